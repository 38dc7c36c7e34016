"""Routing by a model's own router and its gradient against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

FMIN = np.finfo(np.float32).min


@pytest.fixture(scope="module")
def ex():
    from paper_2608_24938_b200 import binding
    return binding


def scores64(z, score):
    masked = z <= FMIN
    s = np.zeros(z.shape)
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            s = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
        else:
            zz = np.where(masked, -np.inf, z)
            top = zz.max(1, keepdims=True)
            s = np.exp(zz - top)
            s = s / s.sum(1, keepdims=True)
    return np.where(masked, 0.0, s), masked


def route64(z, K, score, bias=None, n_groups=1, top_groups=1, group_score="max", renormalise=True, scale=1.0):
    """One token at a time, straight from the header's text."""
    z = z.astype(np.float64)
    T, N = z.shape
    s, masked = scores64(z, score)
    by_logit = bias is None and (n_groups == top_groups or group_score == "max")
    c = z.copy() if by_logit else s + (0.0 if bias is None else bias.astype(np.float64))
    c[masked] = -np.inf
    per = N // n_groups
    ids = np.zeros((T, K), np.int64)
    up = lambda v: np.inf if np.isnan(v) else v  # a NaN ranks first
    for i in range(T):
        groups = c[i].reshape(n_groups, per)
        gscore = []
        for g in groups:
            two = sorted((up(v) for v in g), reverse=True)[:2]
            v = two[0]
            if group_score == "top2" and per > 1 and two[1] > -np.inf:
                v = two[0] + two[1]
            gscore.append(v)
        stay = sorted(range(n_groups), key=lambda g: (-gscore[g], g))[:top_groups]
        cand = [e for e in range(N) if e // per in stay]
        ids[i] = sorted(cand, key=lambda e: (0 if np.isnan(c[i, e]) else 1, -up(c[i, e]), e))[:K]
    w = np.take_along_axis(s, ids, 1)
    if renormalise:
        t = w.sum(1, keepdims=True)
        with np.errstate(all="ignore"):
            w = np.where(t != 0, w / t, 0.0)
    return ids, w * float(np.float32(scale))  # the struct holds a float


def run_route(ex, z, K, load=True, **kw):
    dev = "cuda"
    T, N = z.shape
    layer = ex.make_layer(N, 0, 64, 64, K, "f32")
    bias = kw.pop("bias", None)
    r = ex.make_router(kw.pop("score"), bias=None if bias is None else torch.from_numpy(bias).to(dev), **kw)
    ids = torch.full((T, K), -7, dtype=torch.int32, device=dev)
    w = torch.full((T, K), float("nan"), device=dev)
    ld = torch.full((N,), -7, dtype=torch.int32, device=dev) if load else None
    ex.exfold_route(layer, torch.from_numpy(z).to(dev), r, ids, w, ld)
    return ids.cpu().numpy(), w.cpu().numpy().astype(np.float64), None if ld is None else ld.cpu().numpy()


def check_route(ex, z, K, **kw):
    ids, w, load = run_route(ex, z, K, **kw)
    rid, rw = route64(z, K, **kw)
    assert np.array_equal(ids, rid)
    assert np.array_equal(load, np.bincount(rid.ravel(), minlength=z.shape[1]))
    # computed in 64 bits and rounded once: half a step of fp32, below its normal range half a step of 2^-149
    assert bool((np.abs(w - rw) <= np.abs(rw) * (2.0 ** -24 + 1e-12) + 2.0 ** -150).all())


def scores(T, N, seed=0, std=1.0):
    return np.random.default_rng(seed).standard_normal((T, N)).astype(np.float32) * np.float32(std)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("N,K,T", [(2, 1, 1), (8, 2, 64), (31, 31, 5), (32, 32, 3), (33, 4, 17), (64, 6, 9), (100, 10, 301),
                                   (128, 8, 1), (128, 8, 2500), (160, 6, 257), (255, 32, 33), (256, 8, 4097)])
def test_route_sizes(ex, score, N, K, T):
    z = scores(T, N, seed=N * 1000 + K)
    bias = scores(1, N, seed=5, std=0.1)[0]
    check_route(ex, z, K, score=score)
    check_route(ex, z, K, score=score, bias=bias, renormalise=False, scale=2.5)
    check_route(ex, z, K, score=score, bias=bias, renormalise=True, scale=0.7)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("N,G,top,K", [(256, 8, 4, 8), (64, 8, 1, 8), (64, 32, 30, 6), (96, 3, 2, 5), (30, 5, 2, 12), (32, 32, 7, 7),
                                       (256, 2, 1, 32), (248, 31, 3, 4)])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_route_groups(ex, score, N, G, top, K, group_score):
    z = scores(333, N, seed=N + G)
    kw = dict(score=score, n_groups=G, top_groups=top, group_score=group_score)
    check_route(ex, z, K, **kw)
    check_route(ex, z, K, bias=scores(1, N, seed=6, std=0.2)[0], scale=2.5, **kw)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("mask", [-np.inf, FMIN])
@pytest.mark.parametrize("groups", [dict(), dict(n_groups=8, top_groups=3, group_score="top2"), dict(n_groups=8, top_groups=2)])
@pytest.mark.parametrize("bias", [False, True])
def test_route_masks(ex, score, mask, groups, bias):
    """Rows with no, one, few and all experts masked; a mask of the lowest finite value is one too."""
    N, K = 128, 8
    z = scores(200, N, seed=3)
    rng = np.random.default_rng(4)
    z[:100][rng.random((100, N)) < 0.3] = mask
    z[100:120] = mask
    for i in range(120, 140):  # i - 120 experts are left
        z[i, rng.permutation(N)[i - 120:]] = mask
    for i in range(140, 160):  # one expert per group at most
        for g in range(8):
            z[i, g * 16:(g + 1) * 16 - (g % 2)] = mask
    b = scores(1, N, seed=7, std=0.3)[0] if bias else None
    check_route(ex, z, K, score=score, bias=b, **groups)
    check_route(ex, z, K, score=score, bias=b, renormalise=False, **groups)


def test_route_ties_and_near_ties(ex):
    """Equal scores go to the lower id, in fp32 equal but in 64 bits different ones to the larger."""
    N, K = 128, 8
    z = np.zeros((4, N), np.float32)
    z[1] = np.float32(-0.0)
    z[2, ::2] = 1.0
    z[3] = np.repeat(scores(1, 16)[0], 8)
    for score in ("sigmoid", "softmax"):
        check_route(ex, z, K, score=score)
        check_route(ex, z, K, score=score, bias=np.zeros(N, np.float32))
        check_route(ex, z, K, score=score, n_groups=16, top_groups=3, group_score="top2")
    # neighbouring floats near 4, where the sigmoid has a slope of 0.018: their scores agree in fp32
    near = np.float32(4.0) + np.arange(N, dtype=np.float32)[None, :] * np.float32(2.0 ** -21)
    near = np.concatenate([near, near[:, ::-1], near[:, np.random.default_rng(1).permutation(N)]]).astype(np.float32)
    bias = np.full(N, 0.25, np.float32)
    for score in ("sigmoid", "softmax"):
        check_route(ex, near, K, score=score, bias=bias)
        check_route(ex, near, K, score=score, bias=bias, n_groups=8, top_groups=2, group_score="top2")
    # a bias that nearly cancels the scores' order
    z = scores(500, N, seed=9)
    sig, _ = scores64(z.astype(np.float64), "sigmoid")
    for i in range(0, 500, 50):
        b = (0.5 - sig[i]).astype(np.float32)
        check_route(ex, z[i:i + 50], K, score="sigmoid", bias=b)


def test_route_extreme_scores(ex):
    N, K = 64, 4
    z = scores(64, N, seed=2, std=30.0)
    z[0] = np.linspace(-700, -600, N)    # every sigmoid underflows in fp32
    z[1] = np.linspace(600, 700, N)      # every sigmoid is 1 in fp32
    z[2] = 3e38 * np.linspace(-1, 1, N)
    z[3, 5] = np.inf
    check_route(ex, z[:3], K, score="sigmoid")
    check_route(ex, z[4:], K, score="sigmoid", renormalise=False)
    check_route(ex, z[3:4], K, score="sigmoid")
    check_route(ex, np.delete(z, 3, 0), K, score="softmax")
    check_route(ex, np.delete(z, 3, 0), K, score="softmax", renormalise=False)
    # +inf under a softmax and NaN scores: valid, different ids, the token's weights are NaN, the other tokens' are not
    for bad in (np.nan, np.inf):
        z = scores(40, N, seed=8)
        z[7, 13] = bad
        for kw in (dict(score="softmax"), dict(score="sigmoid"), dict(score="sigmoid", bias=scores(1, N)[0]),
                   dict(score="sigmoid", n_groups=4, top_groups=2, group_score="top2")):
            ids, w, load = run_route(ex, z, K, **kw)
            rid, rw = route64(np.delete(z, 7, 0), K, **kw)
            assert np.array_equal(np.delete(ids, 7, 0), rid)
            if np.isinf(bad):  # the largest score, but a bias or a group may speak against it
                assert np.array_equal(ids[7:8], route64(z[7:8], K, **kw)[0]) or kw["score"] == "softmax"
            else:
                assert ids[7, 0] == 13
            assert len(set(ids[7])) == K and ids.min() >= 0 and ids.max() < N and load.sum() == ids.size
            assert np.isfinite(np.delete(w, 7, 0)).all()
            if np.isnan(bad) or kw["score"] == "softmax":
                assert np.isnan(w[7]).all()
    z = scores(3, N, seed=8)
    z[1] = np.nan
    ids, _, _ = run_route(ex, z, K, score="softmax", bias=np.zeros(N, np.float32))
    assert np.array_equal(ids[1], np.arange(K))


def test_route_without_load_unaligned_and_empty(ex):
    N, K, T = 33, 3, 50  # rows of 132 bytes
    z = scores(T, N)
    ids, w, _ = run_route(ex, z, K, load=False, score="softmax")
    rid, rw = route64(z, K, "softmax")
    assert np.array_equal(ids, rid)
    layer, r = ex.make_layer(N, 0, 64, 64, K, "f32"), ex.make_router("softmax")
    buf = torch.from_numpy(np.concatenate([[0.0], z.ravel()]).astype(np.float32)).cuda()
    out_i = torch.full((T * K + 2,), -7, dtype=torch.int32, device="cuda")
    out_w = torch.full((T * K + 2,), -7.0, device="cuda")
    ex.exfold_route(layer, buf[1:].view(T, N), r, out_i[1:-1].view(T, K), out_w[1:-1].view(T, K))
    assert np.array_equal(out_i[1:-1].view(T, K).cpu().numpy(), rid)
    assert out_i[0] == out_i[-1] == -7 and out_w[0] == out_w[-1] == -7.0  # nothing beside the rows
    load = torch.full((N,), 5, dtype=torch.int32, device="cuda")
    ex.exfold_route(layer, buf[:0].view(0, N), r, out_i[:0].view(0, K), out_w[:0].view(0, K), load)
    assert load.sum() == 0


def test_route_captured_and_on_another_stream(ex):
    N, K, T = 128, 8, 3000
    layer, r = ex.make_layer(N, 0, 64, 64, K, "f32"), ex.make_router("sigmoid", bias=torch.zeros(N, device="cuda"))
    z = torch.empty((T, N), device="cuda")
    ids = torch.empty((T, K), dtype=torch.int32, device="cuda")
    w, load = torch.empty((T, K), device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")
    dw, dz = torch.ones((T, K), device="cuda"), torch.empty((T, N), device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    z.copy_(torch.from_numpy(scores(T, N, 1)))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        ex.exfold_route(layer, z, r, ids, w, load)
        ex.exfold_route_backward(layer, z, ids, dw, r, dz)
    for seed in (2, 3):
        host = scores(T, N, seed)
        z.copy_(torch.from_numpy(host))
        graph.replay()
        rid, _ = route64(host, K, "sigmoid", bias=np.zeros(N, np.float32))
        assert np.array_equal(ids.cpu().numpy(), rid)
        assert np.array_equal(load.cpu().numpy(), np.bincount(rid.ravel(), minlength=N))
        eager = torch.empty_like(dz)
        ex.exfold_route_backward(layer, z, ids, dw, r, eager)
        assert torch.equal(eager, dz)


def test_route_refuses_tensors_of_the_host(ex):
    layer, r = ex.make_layer(8, 0, 64, 64, 2, "f32"), ex.make_router()
    z, ids, w = torch.zeros(3, 8, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, 2, device="cuda")
    for bad in ((z.cpu(), ids, w), (z, ids.cpu(), w), (z, ids, w.cpu())):
        with pytest.raises(AssertionError):
            ex.exfold_route(layer, bad[0], r, bad[1], bad[2])
    with pytest.raises(AssertionError):
        ex.exfold_route_backward(layer, z, ids, w, r, z.cpu())
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    ws = ex.alloc_linear_workspace(64, 2, 2, torch.bfloat16)
    for bad in ((x.cpu(), x, ws), (x, x.cpu(), ws), (x, x, ws.cpu())):
        with pytest.raises(AssertionError):
            ex.exfold_linear(bad[0], bad[1], torch.zeros(2, 2, dtype=torch.bfloat16, device="cuda"), bad[2])


# ------------------------------------------------------------------------------------------------ gradient
def grad64(z, ids, g, score, renormalise, scale):
    s, _ = scores64(z.astype(np.float64), score)
    rows = np.arange(len(z))[:, None]
    ok = (ids >= 0) & (ids < z.shape[1])
    at = np.where(ok, ids, 0)
    sk = np.where(ok, s[rows, at], 0.0)
    g = np.where(ok, g.astype(np.float64), 0.0)
    t = sk.sum(1, keepdims=True)
    safe = np.where(t != 0, t, 1.0)
    ds = np.where(t != 0, (g - (g * sk).sum(1, keepdims=True) / safe) / safe, 0.0) if renormalise else g
    full = np.zeros_like(s)
    np.add.at(full, (np.broadcast_to(rows, at.shape), at), np.where(ok, ds * scale, 0.0))
    if score == "sigmoid":
        return full * s * (1 - s)
    return s * (full - (full * s).sum(1, keepdims=True)) if not renormalise else full * s


def grad_bound(z, ids, g, score, renormalise, scale):
    """What rounding may do. Gathered forms: 64-bit arithmetic and one rounding. Softmax over all experts, fp32: a score has the
    rounding of its argument (|z - max| half steps), 2 steps of expf, 13 half steps of the sum, 2 of quotients; a product and the
    tree sum of 32 terms 7 more. Its terms are scale |g| s for a chosen expert and s sum_k scale |g_k| s_k for all."""
    ref = np.abs(grad64(z, ids, g, score, renormalise, scale))
    if score == "sigmoid" or renormalise:
        return ref * (2.0 ** -24) + 1e-12 * scale * np.abs(g).max()
    s, masked = scores64(z.astype(np.float64), score)
    rows = np.arange(len(z))[:, None]
    a = np.abs(g) * scale
    dot = (a * s[rows, ids]).sum(1, keepdims=True)
    terms = s * dot
    np.add.at(terms, (np.broadcast_to(rows, ids.shape), ids), a * s[rows, ids])
    with np.errstate(invalid="ignore"):
        spread = np.where(masked, 0.0, z.max(1, keepdims=True) - z).max()
    return 2 * (spread + 4 + 13 + 2 + 7) * 2.0 ** -24 * terms + 2.0 ** -126


def run_back(ex, z, ids, g, score, renormalise, scale):
    T, N = z.shape
    layer = ex.make_layer(N, 0, 64, 64, ids.shape[1], "f32")
    out = torch.full((T, N), float("nan"), device="cuda")
    ex.exfold_route_backward(layer, torch.from_numpy(z).cuda(), torch.from_numpy(ids.astype(np.int32)).cuda(),
                             torch.from_numpy(g).cuda(), ex.make_router(score, renormalise=renormalise, scale=scale), out)
    return out.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("N,K,T", [(2, 1, 1), (8, 2, 64), (33, 32, 5), (64, 6, 100), (128, 8, 2000), (200, 10, 31), (256, 8, 77)])
def test_route_backward(ex, score, renormalise, N, K, T):
    z = scores(T, N, seed=N + 1)
    ids, _ = route64(z, K, score, renormalise=renormalise)
    g = scores(T, K, seed=N + 2)
    got = run_back(ex, z, ids, g, score, renormalise, 1.5)
    assert bool((np.abs(got - grad64(z, ids, g, score, renormalise, 1.5)) <= grad_bound(z, ids, g, score, renormalise, 1.5)).all())


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward_masks_and_dropped_ids(ex, score, renormalise):
    N, K = 64, 6
    z = scores(30, N, seed=11)
    z[:10, 3:40] = -np.inf
    z[10:15] = FMIN
    z[15:20] = -np.inf
    z[20, :-2] = -np.inf  # fewer experts left than slots
    ids, _ = route64(z, K, score, renormalise=renormalise)
    g = scores(30, K, seed=12)
    got = run_back(ex, z, ids, g, score, renormalise, 1.0)
    assert bool((np.abs(got - grad64(z, ids, g, score, renormalise, 1.0)) <= grad_bound(z, ids, g, score, renormalise, 1.0)).all())
    assert (got[10:20] == 0).all() and (got[:10, 3:40] == 0).all()
    dropped = ids.copy()
    dropped[25, 2], dropped[26, 0], dropped[27] = -1, N, -5
    ok = (dropped >= 0) & (dropped < N)
    got = run_back(ex, z, dropped, g, score, renormalise, 1.0)
    ref = grad64(z, dropped, g, score, renormalise, 1.0)
    bound = grad_bound(z, np.where(ok, dropped, 0), np.where(ok, g, 0.0).astype(np.float32), score, renormalise, 1.0)
    assert bool((np.abs(got - ref) <= bound).all() and (got[27] == 0).all())


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward_against_differences(ex, score, renormalise):
    """The gradient of sum(dw * w) with the choice held: central differences of the 64-bit definition. A step of 1e-4 leaves
    1e-8 / 6 of third derivatives (below 2 scale |g|) and 1e-12 of rounding."""
    N, K = 16, 4
    z = scores(6, N, seed=21)
    ids, _ = route64(z, K, score, renormalise=renormalise)
    g = scores(6, K, seed=22)
    rows = np.arange(6)[:, None]

    def loss(zz):
        s, _ = scores64(zz, score)
        w = s[rows, ids]
        if renormalise:
            w = w / w.sum(1, keepdims=True)
        return (2.0 * w * g).sum(1)

    num = np.zeros((6, N))
    for e in range(N):
        d = np.zeros((6, N))
        d[:, e] = 1e-4
        num[:, e] = (loss(z + d) - loss(z - d)) / 2e-4
    got = run_back(ex, z, ids, g, score, renormalise, 2.0)
    tol = 2 * 2.0 * np.abs(g).sum(1).max() * 1e-8 / 6 + 1e-8 + grad_bound(z, ids, g, score, renormalise, 2.0)
    assert bool((np.abs(got - num) <= tol).all())


def test_route_beyond_32_bit_offsets(ex):
    """More than 2^31 scores: the last tokens' rows are found, and nothing else is written there."""
    N, K, T = 256, 2, (1 << 23) + 5
    z = torch.zeros((T, N), device="cuda")
    tail = scores(5, N, seed=31)
    z[-5:] = torch.from_numpy(tail).cuda()
    layer, r = ex.make_layer(N, 0, 64, 64, K, "f32"), ex.make_router("softmax")
    ids, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    load = torch.empty(N, dtype=torch.int32, device="cuda")
    ex.exfold_route(layer, z, r, ids, w, load)
    rid, rw = route64(tail, K, "softmax")
    assert np.array_equal(ids[-5:].cpu().numpy(), rid) and torch.equal(ids[:-5].amax(0).cpu(), torch.tensor([0, 1], dtype=torch.int32))
    assert bool((np.abs(w[-5:].cpu().numpy() - rw) <= rw * (2.0 ** -24 + 1e-12)).all())
    assert int(load.sum()) == T * K and int(load[0]) >= T - 5
    dz = torch.full((T, N), float("nan"), device="cuda")
    g = torch.ones((T, K), device="cuda")
    g[:, 1] = -1.0
    ex.exfold_route_backward(layer, z, ids, g, r, dz)
    ref = grad64(tail, rid, g[-5:].cpu().numpy(), "softmax", True, 1.0)
    bound = grad_bound(tail, rid, g[-5:].cpu().numpy(), "softmax", True, 1.0)
    assert bool((np.abs(dz[-5:].cpu().numpy() - ref) <= bound).all())
    assert torch.equal(dz[:-5].amax(0)[:2].cpu(), torch.tensor([0.5, -0.5])) and torch.equal(dz[:-5, 2:].abs().amax(), dz.new_zeros(()))


def tied_groups(T, N, G, plus, minus, amp, seed):
    """Scores and a bias whose groups' two largest choices are s + plus and s + minus, with sums `amp` times a few fp32 roundings apart:
    every group has the same scores but for small differences."""
    rng = np.random.default_rng(seed)
    per = N // G
    z = np.tile(rng.standard_normal((T, per)), (1, G)) + rng.uniform(-1, 1, (T, N)) * amp
    bias = np.full((G, per), minus, np.float32)
    bias[:, 0] = plus
    return z.astype(np.float32), bias.ravel()


@pytest.mark.parametrize("score,slope", [("sigmoid", 0.2), ("softmax", 0.008)])
@pytest.mark.parametrize("plus,minus", [(16, -16), (100, -100), (1000, -1000), (-100, 100), (1030, 1030), (-1030, -1030), (1000, 900),
                                        (3e30, -3e30), (3e38, 3e38), (-3e38, -3e38)])
@pytest.mark.parametrize("N,G,top,K", [(256, 8, 4, 8), (8, 2, 1, 1), (96, 3, 2, 5)])
def test_route_groups_of_large_biases(ex, score, slope, plus, minus, N, G, top, K):
    """Sums of two choices are rounded at the size of the choices, which may be far above the sum's."""
    amp = min(0.5, max(abs(plus), abs(minus)) * 2.0 ** -22 / slope)
    z, bias = tied_groups(300, N, G, plus, minus, amp, seed=int(abs(plus) % 1000) + N)
    for group_score in ("top2", "max"):
        check_route(ex, z, K, score=score, bias=bias, n_groups=G, top_groups=top, group_score=group_score)


def test_route_groups_fp32_sums_are_in_the_wrong_order(ex):
    """A token whose groups score 0.948400 and 0.948380, in fp32 0.948364 and 0.948425."""
    z = np.array([[-1.704, -1.145, -0.586, 1.352, -1.632, 0.562, 1.294, 0.458]], np.float32)
    bias = np.tile(np.array([1000, -1000, -1000, -1000], np.float32), 2)
    assert route64(z, 1, "sigmoid", bias=bias, n_groups=2, top_groups=1, group_score="top2")[0][0, 0] == 0
    check_route(ex, z, 1, score="sigmoid", bias=bias, n_groups=2, top_groups=1, group_score="top2")


def peaked_grad64(z, ids, g, scale):
    """The gradient over all experts with 1 - s taken from the other experts' exponentials; and the sum of magnitudes of what each
    entry is made of, once the terms that cancel exactly are gone."""
    T, N = z.shape
    s, _ = scores64(z.astype(np.float64), "softmax")
    rows = np.arange(T)[:, None]
    chosen = np.zeros((T, N), bool)
    chosen[rows, ids] = True
    G = np.zeros((T, N))
    G[rows, ids] = g
    sc = np.where(chosen, s, 0.0)
    rest = np.where(chosen, 0.0, s).sum(1, keepdims=True)
    diff = G[:, :, None] - G[:, None, :]  # [e][k]
    value = np.where(chosen, G * rest + (diff * sc[:, None, :]).sum(2), -(G * sc).sum(1, keepdims=True)) * s * scale
    terms = np.where(chosen, np.abs(G) * rest + (np.abs(diff) * sc[:, None, :]).sum(2), np.abs((G * sc).sum(1, keepdims=True))) * s * scale
    return value, terms


@pytest.mark.parametrize("N,K", [(64, 1), (64, 2), (128, 8), (33, 5), (200, 10), (256, 32)])
@pytest.mark.parametrize("T", [7, 1300, 5000])
def test_route_backward_of_confident_routers(ex, N, K, T):
    """Softmax over all experts with one or two scores far above the others: what is left of a chosen expert's entry is small against
    its own terms. The scores' exponentials are fp32 (argument |z - max|, 4 half steps of expf, 13 of the sum, 7 of products and
    quotients, twice for a numerator and the sum), the chosen ones' and their sums 64-bit."""
    T = min(T, 600000 // N // max(1, N // 32))
    z = scores(T, N, seed=N + K)
    top = np.random.default_rng(3).permutation(N)[:2]
    z[:, top[0]] += np.linspace(0, 18, T, dtype=np.float32)
    z[T // 2:, top[1]] = z[T // 2:, top[0]] - np.float32(0.25)
    ids, _ = route64(z, K, "softmax", renormalise=False)
    g = scores(T, K, seed=N + 2)
    got = run_back(ex, z, ids, g, "softmax", False, 1.5)
    ref, terms = peaked_grad64(z, ids, g, 1.5)
    spread = (z.max(1, keepdims=True) - z).max()
    bound = 2 * (spread + 4 + 13 + 7) * 2.0 ** -24 * terms + 1e-14 * 1.5 * np.abs(g).max() + 2.0 ** -126
    bad = np.abs(got - ref) > bound
    assert not bad.any(), f"{int(bad.sum())} entries, worst {float((np.abs(got - ref) / bound).max()):.1f} of the bound"


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_route_groups_of_one_expert(ex, score):
    """Groups that go by a sum of two rank by scores as others do, also where a group has one expert: sigmoids that are 1 in 64 bits tie."""
    for N, top, K in ((8, 3, 2), (32, 7, 7), (32, 1, 1)):
        z = np.concatenate([scores(20, N, seed=41), scores(20, N, seed=42, std=30.0), 40 + np.abs(scores(20, N, seed=43, std=5.0))])
        for group_score in ("top2", "max"):
            check_route(ex, z.astype(np.float32), K, score=score, n_groups=N, top_groups=top, group_score=group_score)
