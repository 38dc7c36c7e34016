"""The folded layer on given routes against the oracle's experts and the definitions of the fold."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import synth_inputs as si
from harness import A, Case, check_output

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    from paper_2608_24938_b200 import binding
    return binding


def small(name, **kw):
    base = dict(name=name, n_experts=16, hidden=256, inter=384, top_k=4, prefill_tokens=96, k_pre=(2,), decode_batch=24, pool_m=(6,))
    base.update(kw)
    return si.scaled(si.CONFIGS["qwen3"], **base)


CONFIGS = {
    "tiny": si.CONFIGS["tiny"],
    "f32_shared": small("routed-f32", dtype="f32", n_shared=1, hidden=132, inter=70),
    "bf16": small("routed-bf16"),
    "bf16_shared": small("routed-shared", n_shared=1, n_experts=40, top_k=8),
    "bf16_top1": small("routed-top1", top_k=1, k_pre=(1,)),
}


def routes(cfg, T, seed=0, spread=True):
    """K different experts per token in random order, positive weights that do not sum to 1."""
    rng = np.random.default_rng([seed, cfg.n_experts, T])
    ids = np.stack([rng.permutation(cfg.n_experts)[:cfg.top_k] for _ in range(T)]).astype(np.int32)
    w = rng.uniform(0.05, 1.0, size=ids.shape).astype(np.float32) * np.float32(1.7)
    return ids, w


def fold64(ids, w, Kp, S, L, h, threshold=np.inf, rescale=False, confidence=False):
    T, K = ids.shape
    out_i, out_w = np.zeros((T, Kp), np.int32), np.zeros((T, Kp))
    src, tgt = np.zeros((T, K - Kp), np.int32), np.zeros((T, K - Kp), np.int32)
    for i in range(T):
        key = w[i] * h[ids[i]] if Kp < K else w[i]  # one fp32 product
        order = sorted(range(K), key=lambda j: (-key[j], ids[i, j]))
        kept = [int(ids[i, j]) for j in order[:Kp]]
        orig = {int(ids[i, j]): float(w[i, j]) for j in order[:Kp]}
        new = dict(orig)
        for n, j in enumerate(order[Kp:]):
            s = int(ids[i, j])
            adm = [t for t in kept if not L[s, t] > threshold]
            t = min(adm, key=lambda e: (L[s, e], e)) if adm else -1
            src[i, n], tgt[i, n] = s, t
            if t >= 0:
                c = min(max(1.0 - float(L[s, t]), 0.0), 1.0) if confidence else 1.0
                if confidence:
                    for e in kept:
                        new[e] += float(w[i, j]) * (1 - c) * orig[e] / sum(orig.values())
                new[t] += float(w[i, j]) * c * float(S[s, t])
        if rescale and sum(new.values()) > 0:
            f = float(w[i].astype(np.float64).sum()) / sum(new.values())
            new = {e: v * f for e, v in new.items()}
        out_i[i], out_w[i] = kept, [new[e] for e in kept]
    return out_i, out_w, src, tgt


def pool64(ids, w, M, S, L, h):
    N = len(h)
    total = np.zeros(N)
    np.add.at(total, ids, w.astype(np.float64))
    union = np.unique(ids)
    pool = sorted(union.tolist(), key=lambda e: (-total[e] * float(h[e]), e))[:M]
    target = np.array([e if e in pool else min(pool, key=lambda p: (L[e, p], p)) for e in range(N)], np.int32)
    scale = np.array([1.0 if target[e] == e else S[e, target[e]] for e in range(N)], np.float32)
    return pool, target, scale, target[ids], w.astype(np.float64) * scale[ids]


def experts(case, x, ids, w):
    cfg = case.cfg
    return oracle.moe_apply(A(x), A(case.wg), A(case.wu), A(case.wd), ids.astype(np.int32), w.astype(np.float32), cfg.n_experts,
                            cfg.n_shared)


def run_prefill(case, x, ids, w, Kp, tables=True, meta=True, **kw):
    ex, cfg, T = case.ex, case.cfg, len(ids)
    ws = case.workspace(T, Kp)
    y = torch.full((T, cfg.hidden), float("nan"), dtype=case.d_wg.dtype, device=case.dev)
    i32 = dict(dtype=torch.int32, device=case.dev)
    m = dict(ids=torch.full((T, Kp), -7, **i32), w=torch.full((T, Kp), float("nan"), device=case.dev),
             omit_src=torch.full((T, cfg.top_k - Kp), -7, **i32), omit_tgt=torch.full((T, cfg.top_k - Kp), -7, **i32)) if meta else None
    ex.exfold_moe_prefill_routed(case.layer, x.to(case.dev), torch.from_numpy(ids).to(case.dev), torch.from_numpy(w).to(case.dev),
                                 case.d_wg, case.d_wu, case.d_wd, case.tables if tables else None, Kp, y, ws, meta=m, **kw)
    assert ex.exfold_device_status(ws) == 0
    return y.float().cpu().numpy(), {k: v.cpu().numpy() for k, v in (m or {}).items()}


def run_decode(case, x, ids, w, M, meta=True):
    ex, cfg, B = case.ex, case.cfg, len(ids)
    K, N = cfg.top_k, cfg.n_experts
    ws = case.workspace(B, K)
    y = torch.full((B, cfg.hidden), float("nan"), dtype=case.d_wg.dtype, device=case.dev)
    i32, f32 = dict(dtype=torch.int32, device=case.dev), dict(dtype=torch.float32, device=case.dev)
    m = dict(pool_ids=torch.full((M,), -7, **i32), pool_size=torch.full((1,), -7, **i32), ids=torch.full((B, K), -7, **i32),
             w=torch.full((B, K), float("nan"), **f32), target=torch.full((N,), -7, **i32),
             scale=torch.full((N,), float("nan"), **f32)) if meta else None
    ex.exfold_moe_decode_routed(case.layer, x.to(case.dev), torch.from_numpy(ids).to(case.dev), torch.from_numpy(w).to(case.dev),
                                case.d_wg, case.d_wu, case.d_wd, case.tables, M, y, ws, meta=m)
    assert ex.exfold_device_status(ws) == 0
    return y.float().cpu().numpy(), {k: v.cpu().numpy() for k, v in (m or {}).items()}


@pytest.mark.parametrize("name", list(CONFIGS))
@pytest.mark.parametrize("T", [1, 3, 8, 9, 96, 2100])
def test_prefill_routed(ex, name, T):
    cfg = CONFIGS[name]
    case = Case(dataclasses.replace(cfg, calib_tokens=0), T=T)
    S, L, h, _ = case.np_tables()
    ids, w = routes(cfg, T)
    for Kp in sorted({1, (cfg.top_k + 1) // 2, cfg.top_k}):
        ri, rw, src, tgt = fold64(ids, w, Kp, S, L, h)
        y, m = run_prefill(case, case.x, ids, w, Kp)
        assert np.array_equal(m["ids"], ri) and np.array_equal(m["omit_src"], src) and np.array_equal(m["omit_tgt"], tgt)
        # at most K additions of rounded products
        tol = (cfg.top_k + 2) * 2.0 ** -23 * np.abs(w).sum(1, keepdims=True) * 4.0
        assert bool((np.abs(m["w"] - rw) <= tol).all())
        check_output(y, experts(case, case.x, ri, rw), cfg.dtype)
        bare, _ = run_prefill(case, case.x, ids, w, Kp, meta=False)
        assert np.array_equal(bare, y)
    y2, m2 = run_prefill(case, case.x, ids, w, cfg.top_k, tables=False)  # nothing is folded: no tables
    check_output(y2, experts(case, case.x, ids, w), cfg.dtype)
    assert np.array_equal(np.sort(m2["ids"], 1), np.sort(ids, 1))


def test_prefill_routed_safeguards_and_paths(ex):
    cfg = CONFIGS["bf16_shared"]
    case = Case(cfg, T=1500)
    S, L, h, _ = case.np_tables()
    ids, w = routes(cfg, 1500, seed=4)
    for kw in (dict(loss_threshold=0.7), dict(rescale=True), dict(confidence_split=True),
               dict(loss_threshold=0.7, rescale=True, confidence_split=True)):
        ri, rw, src, tgt = fold64(ids, w, 3, S, L, h, kw.get("loss_threshold", np.inf), kw.get("rescale", False),
                                  kw.get("confidence_split", False))
        y, m = run_prefill(case, case.x, ids, w, 3, **kw)
        assert np.array_equal(m["omit_tgt"], tgt)
        np.testing.assert_allclose(m["w"], rw, rtol=2e-5, atol=2e-6)
        for path in (1, 2, 3):
            assert np.array_equal(run_prefill(case, case.x, ids, w, 3, gemm_path=path, **kw)[0], y)


@pytest.mark.parametrize("name", list(CONFIGS))
@pytest.mark.parametrize("B", [1, 5, 8, 9, 40, 200])
def test_decode_routed(ex, name, B):
    cfg = CONFIGS[name]
    case = Case(dataclasses.replace(cfg, calib_tokens=0), B=B)
    S, L, h, _ = case.np_tables()
    ids, w = routes(cfg, B, seed=1)
    for M in sorted({1, cfg.n_experts // 3, cfg.n_experts}):
        pool, target, scale, ri, rw = pool64(ids, w, M, S, L, h)
        y, m = run_decode(case, case.xd, ids, w, M)
        assert m["pool_size"][0] == len(pool) and m["pool_ids"][:len(pool)].tolist() == pool and (m["pool_ids"][len(pool):] == -1).all()
        assert np.array_equal(m["ids"], ri) and np.array_equal(m["target"], target) and np.array_equal(m["scale"], scale)
        assert bool((np.abs(m["w"] - rw) <= 2.0 ** -24 * np.abs(rw) + 1e-30).all())
        check_output(y, experts(case, case.xd, ri, rw), cfg.dtype)
        bare, _ = run_decode(case, case.xd, ids, w, M, meta=False)
        assert np.array_equal(bare, y)


@pytest.mark.parametrize("name", ["tiny", "bf16_shared"])
def test_routes_of_no_expert(ex, name):
    """Ids outside the layer, also all of a token's, and weights of 0: no row but the others' (and the shared expert's)."""
    cfg = CONFIGS[name]
    N, K = cfg.n_experts, cfg.top_k
    for T in (4, 30, 300):
        case = Case(dataclasses.replace(cfg, calib_tokens=0), T=T, B=min(T, 200))
        S, L, h, _ = case.np_tables()
        ids, w = routes(cfg, T, seed=2)
        bad, clean, cw = ids.copy(), ids.copy(), w.copy()
        bad[0], clean[0], cw[0] = -1, np.arange(K), 0.0   # a token without an expert
        bad[1, 0], cw[1, 0] = N + 5, 0.0
        clean[1, 0] = 0 if 0 not in ids[1, 1:] else ids[1, 0]
        w0 = w.copy()
        w0[2, 1:] = cw[2, 1:] = 0.0
        for Kp in {1, K}:
            ri, rw, _, _ = fold64(clean, cw, Kp, S, L, h)
            y, m = run_prefill(case, case.x, bad, w0, Kp)
            assert m["ids"].min() >= 0 and m["ids"].max() < N
            check_output(y, experts(case, case.x, ri, rw), cfg.dtype)
        B = case.B
        y, m = run_decode(case, case.xd, bad[:B], w0[:B], N)
        check_output(y, experts(case, case.xd, clean[:B], cw[:B]), cfg.dtype)


def test_an_expert_named_twice(ex):
    """Not a router's choice, but not a fault either: the weights of the two slots add up."""
    cfg = CONFIGS["bf16"]
    for T in (5, 64):
        case = Case(cfg, T=T, B=T)
        ids, w = routes(cfg, T, seed=3)
        ids[:, 1] = ids[:, 0]
        merged = w.copy()
        merged[:, 0] += merged[:, 1]
        merged[:, 1] = 0.0
        other = ids.copy()
        other[:, 1] = (ids.max(1) + 1) % cfg.n_experts
        y, _ = run_prefill(case, case.x, ids, w, cfg.top_k)
        check_output(y, experts(case, case.x, other, merged), "bf16")
        y, _ = run_decode(case, case.xd, ids, w, cfg.n_experts)
        check_output(y, experts(case, case.xd, other, merged), "bf16")


def test_softmax_routes_reproduce_the_logit_calls(ex):
    """Routes of Eq. 2's router: the same retained experts and outputs as the calls that take the scores."""
    for name in ("tiny", "bf16_shared"):
        cfg = dataclasses.replace(CONFIGS[name], calib_tokens=0)
        case = Case(cfg, T=257, B=40)
        K, N = cfg.top_k, cfg.n_experts
        r = ex.make_router("softmax", renormalise=True)
        for lg, x, T in ((case.d_lg, case.x, 257), (case.d_lgd, case.xd, 40)):
            ids = torch.empty((T, K), dtype=torch.int32, device=case.dev)
            w = torch.empty((T, K), device=case.dev)
            ex.exfold_route(case.layer, lg, r, ids, w)
            if T == 257:
                got = case.run_prefill(max(1, K // 2))
                y, m = run_prefill(case, x, ids.cpu().numpy(), w.cpu().numpy(), max(1, K // 2))
            else:
                got = case.run_decode(N // 3)
                y, m = run_decode(case, x, ids.cpu().numpy(), w.cpu().numpy(), N // 3)
            assert np.array_equal(m["ids"], got["ids"])
            check_output(y, got["y"], cfg.dtype)


def test_block_from_hidden_states_under_capture(ex):
    """As a model uses them together: projection onto the residual stream, router scores, the model's own router, the folded
    experts on its routes, projection back; eager and as one graph, for a decode batch and a prompt."""
    cfg = CONFIGS["bf16_shared"]
    for T, decode in ((24, True), (300, False)):
        case = Case(cfg, T=T, B=T)
        N, K, d = cfg.n_experts, cfg.top_k, cfg.hidden
        g = torch.Generator(device="cuda").manual_seed(5)
        bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
        attn, res, wo, wr, wp = bf(T, d), bf(T, d), bf(d, d) * d ** -0.5, bf(N, d) * d ** -0.5, bf(d, d) * d ** -0.5
        router = ex.make_router("sigmoid", bias=torch.randn(N, generator=g, device="cuda") * 0.1, n_groups=4, top_groups=2,
                                group_score="top2", scale=1.5)
        hid, y, out = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        logits, w = torch.empty((T, N), device="cuda"), torch.empty((T, K), device="cuda")
        ids = torch.empty((T, K), dtype=torch.int32, device="cuda")
        ws = case.workspace(T, K)
        lws = ex.alloc_linear_workspace(d, d, T, torch.bfloat16)

        def block():
            ex.exfold_linear(attn, wo, hid, lws, residual=res)
            ex.exfold_router_logits(case.layer, hid, wr, logits, ws)
            ex.exfold_route(case.layer, logits, router, ids, w)
            args = (case.layer, hid, ids, w, case.d_wg, case.d_wu, case.d_wd, case.tables)
            if decode:
                ex.exfold_moe_decode_routed(*args, N // 3, y, ws)
            else:
                ex.exfold_moe_prefill_routed(*args, 3, y, ws)
            ex.exfold_linear(y, wp, out, lws, residual=hid)

        block()
        torch.cuda.synchronize()
        first = [t.clone() for t in (hid, logits, ids, w, y, out)]
        ref = (attn.double() @ wo.double().T + res.double()).float().cpu().numpy()
        check_output(hid.float().cpu().numpy(), ref, "bf16")
        S, L, h, _ = case.np_tables()
        i_, w_ = ids.cpu().numpy(), w.cpu().numpy()
        ri, rw = pool64(i_, w_, N // 3, S, L, h)[3:] if decode else fold64(i_, w_, 3, S, L, h)[:2]
        check_output(y.float().cpu().numpy(), experts(case, hid.cpu(), ri, rw), "bf16")
        check_output(out.float().cpu().numpy(), (y.double() @ wp.double().T + hid.double()).float().cpu().numpy(), "bf16")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block()
        for t in (hid, logits, w, y, out):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (hid, logits, ids, w, y, out)))


@pytest.mark.parametrize("name", ["tiny", "f32_shared", "bf16_shared"])
@pytest.mark.parametrize("opts", [dict(), dict(rescale=True), dict(loss_threshold=0.7), dict(loss_threshold=0.7, rescale=True)])
@pytest.mark.parametrize("T", [4, 30, 300])
def test_confidence_split_over_weights_of_zero(ex, name, opts, T):
    """Retained routes that all weigh 0 share what is spread equally: nothing is lost, and nothing is divided by their sum."""
    cfg = CONFIGS[name]
    N, K = cfg.n_experts, cfg.top_k
    Kp = (K + 1) // 2
    case = Case(dataclasses.replace(cfg, calib_tokens=0), T=T)
    S, L, h, _ = (t.copy() for t in case.np_tables())
    h[N - 1] = 0.0  # never retained before another
    with np.errstate(divide="ignore"):
        case.set_tables((S, L, h, np.log(h)))
    ids, w = routes(cfg, T, seed=6)
    given = ids.copy()
    given[0], ids[0], w[0] = -1, 0, 0.0  # no expert at all: expert 0, K times
    w[1] = 0.0
    ids[2] = given[2] = [*range(K - 1), N - 1]
    w[2] = [0.0] * (K - 1) + [1.25]
    some = np.arange(T) >= 3
    ri, rw = np.zeros((T, Kp), np.int32), np.zeros((T, Kp))
    if some.any():
        ri[some], rw[some] = fold64(ids[some], w[some], Kp, S, L, h, opts.get("loss_threshold", np.inf), opts.get("rescale", False), True)[:2]
    ri[1] = np.sort(ids[1])[:Kp]
    ri[2] = ids[2, :Kp]
    adm = [t for t in ri[2] if not L[N - 1, t] > opts.get("loss_threshold", np.inf)]
    if adm:
        t = min(adm, key=lambda e: (L[N - 1, e], e))
        c = min(max(1.0 - float(L[N - 1, t]), 0.0), 1.0)
        rw[2] = 1.25 * (1 - c) / Kp
        rw[2, list(ri[2]).index(t)] += 1.25 * c * float(S[N - 1, t])
        if opts.get("rescale") and rw[2].sum() > 0:
            rw[2] *= 1.25 / rw[2].sum()
    y, m = run_prefill(case, case.x, given, w, Kp, confidence_split=True, **opts)
    assert np.array_equal(m["ids"], ri)
    np.testing.assert_allclose(m["w"], rw, rtol=2e-5, atol=2e-6)
    clean = ri.copy()
    clean[0] = np.arange(Kp)  # different experts for the oracle; they weigh 0
    check_output(y, experts(case, case.x, clean, rw), cfg.dtype)
    bare, _ = run_prefill(case, case.x, given, w, Kp, meta=False, confidence_split=True, **opts)
    assert np.array_equal(bare, y)


@pytest.mark.parametrize("name", ["tiny", "f32_shared", "bf16", "bf16_shared"])
@pytest.mark.parametrize("B", [1, 8, 9, 200, 256])
def test_decode_routed_weights_of_any_size(ex, name, B):
    """Pool sums neither wrap where an expert's weights sum to 2048 and more nor take a negative or NaN weight for a large one."""
    cfg = CONFIGS[name]
    case = Case(dataclasses.replace(cfg, calib_tokens=0), B=B)
    S, L, h, _ = case.np_tables()
    N, K = cfg.n_experts, cfg.top_k
    ids, w = routes(cfg, B, seed=7)
    ids[:, 0], ids[:, 1] = 5, 6
    for i in range(B):
        ids[i, 2:] = np.random.default_rng(i).permutation([e for e in range(N) if e not in (5, 6)])[:K - 2]
    w[:, 0], w[:, 1] = 2100.0 / B, 400.0 / B  # a sum of 2100: 52 where it wraps
    w = w.astype(np.float32)
    def pools(weights, counted):
        for M in (1, 2):
            pool, target, scale, ri, rw = pool64(ids, counted, M, S, L, h)
            y, m = run_decode(case, case.xd, ids, weights, M)
            assert m["pool_ids"][:len(pool)].tolist() == pool
            assert np.array_equal(m["ids"], ri) and np.array_equal(m["target"], target)
            if np.isfinite(weights).all():
                check_output(y, experts(case, case.xd, ri, weights.astype(np.float64) * scale[ids]), cfg.dtype)
    pools(w, w)
    w[:, 0] *= np.float32(1e4)
    pools(w, w)
    for bad in (-3.0, -1e10, np.nan):
        v = w.copy()
        v[:, 0] = bad
        pools(v, np.where(v > 0, v, np.float32(0.0)))


@pytest.mark.parametrize("name", list(CONFIGS))
@pytest.mark.parametrize("T", [1, 8, 30, 200, 2100])
def test_every_route_names_one_expert(ex, name, T):
    """All rows are one expert's: K times as many as there are tokens (prefill), one per token (decode)."""
    cfg = CONFIGS[name]
    case = Case(dataclasses.replace(cfg, calib_tokens=0), T=T, B=min(T, 200))
    K = cfg.top_k
    ids, w = np.full((T, K), 3, np.int32), routes(cfg, T, seed=8)[1]
    one = np.full((T, 1), 3, np.int32)
    total = w.astype(np.float64).sum(1, keepdims=True)
    y, m = run_prefill(case, case.x, ids, w, K)
    assert (m["ids"] == 3).all()
    check_output(y, experts(case, case.x, one, total), cfg.dtype)
    bad = np.where(np.arange(K)[None, :] % 2 == 0, -1, cfg.n_experts).astype(np.int32).repeat(T, 0)
    y, m = run_prefill(case, case.x, bad, w, K)  # no expert at all: expert 0 with weights of 0
    assert (m["ids"] == 0).all() and (m["w"] == 0).all()
    check_output(y, experts(case, case.x, one, total * 0), cfg.dtype) if cfg.n_shared else np.testing.assert_array_equal(y, 0)
    B = case.B
    y, m = run_decode(case, case.xd, ids[:B], w[:B], cfg.n_experts)
    assert m["pool_size"][0] == 1 and m["pool_ids"][0] == 3
    check_output(y, experts(case, case.xd, one[:B], total[:B]), cfg.dtype)


@pytest.mark.parametrize("name", ["tiny", "f32_shared", "bf16", "bf16_shared"])
@pytest.mark.parametrize("scale", [16.0, 300.0, 1100.0])
def test_decode_routed_ranks_large_sums(ex, name, scale):
    """Sums of weights beyond 2048 rank as any others."""
    cfg = CONFIGS[name]
    for B in (8, 128, 256):
        case = Case(dataclasses.replace(cfg, calib_tokens=0), B=B)
        S, L, h, _ = case.np_tables()
        ids, w = routes(cfg, B, seed=9)
        w *= np.float32(scale)
        for M in (1, cfg.n_experts // 2, cfg.n_experts):
            pool, target, scale_, ri, rw = pool64(ids, w, M, S, L, h)
            y, m = run_decode(case, case.xd, ids, w, M)
            assert m["pool_ids"][:len(pool)].tolist() == pool and np.array_equal(m["ids"], ri)
            check_output(y, experts(case, case.xd, ri, rw), cfg.dtype)
