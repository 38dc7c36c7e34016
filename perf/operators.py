"""The operators around the folded experts as a set of measurable cases.

`route`            a model's own router: sigmoid or softmax scores, a balance bias, expert groups, Top-K, weights
`route_backward`   the gradient of its weights with respect to the router scores
`linear`           a product with bias, activation and residual: the projections before and after the layer
`prefill_routed`, `decode_routed`   the folded experts on given routes (ids and weights) instead of router scores

A case is one call on one layer of the shapes that the repository's configurations name or of a generic shape. With
`own` false, `run` computes the operator in elementary torch operations; with `own` true it makes the library's call.
"""
import math

import numpy as np
import torch

own = False

# routed experts, shared experts, hidden, intermediate, Top-K, dtype
SHAPES = {
    "tiny": (8, 0, 128, 256, 2, "f32"),
    "mixtral": (8, 0, 4096, 14336, 2, "bf16"),
    "qwen3": (128, 0, 2048, 768, 8, "bf16"),
    "glm45air": (128, 1, 4096, 1408, 8, "bf16"),
}
LAYER = ("experts", "shared", "hidden", "inter", "top_k", "dtype")
MAX_LINEAR_FLOPS = 2.8e11
MAX_EXPERT_FLOPS = 1.6e11
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _route(op, **kw):
    c = {"op": op, "experts": 128, "top_k": 8, "score": "sigmoid", "bias": True, "groups": 1, "top_groups": 1,
         "group_score": "max", "renormalise": True, "scale": 1.0, "masked": False, "zipf": False}
    c.update(kw)
    return c


def _linear(**kw):
    c = {"op": "linear", "dtype": "bf16", "out": "bf16", "bias": False, "act": "none", "residual": False, "pad": 0}
    c.update(kw)
    return c


def _experts(op, shape, **kw):
    c = {"op": op, "zipf": False}
    c.update(zip(LAYER, SHAPES[shape] if isinstance(shape, str) else shape))
    c.update(kw)
    return c


def listed():
    return [
        # one user's next token: the router of a layer of 128 experts with a balance bias
        _route("route", name="route_sigmoid_t1", tokens=1),
        # a ragged prompt through a group-limited router: 4 of 8 groups of 32 experts, some experts masked out
        _route("route", name="route_grouped_t777", tokens=777, experts=256, groups=8, top_groups=4, group_score="top2",
               scale=2.5, masked=True),
        # eight prompts of 2048 tokens through a sigmoid router
        _route("route", name="route_sigmoid_t16384", tokens=16384),
        # tuning a sigmoid router on a short batch
        _route("route_backward", name="route_back_sigmoid_t333", tokens=333),
        # tuning a softmax router whose weights are not renormalised: every score gets a gradient
        _route("route_backward", name="route_back_softmax_t8192", tokens=8192, score="softmax", bias=False,
               renormalise=False, zipf=True),
        # an fp32 layer small enough that latency is the whole cost
        _linear(name="linear_f32_t64", tokens=64, inputs=128, outputs=256, dtype="f32", out="f32", bias=True, act="silu"),
        # one user's next token through a projection back to the residual stream
        _linear(name="linear_t1_res", tokens=1, inputs=4096, outputs=4096, residual=True),
        # an ordinary decode batch through a wide projection
        _linear(name="linear_t64_wide", tokens=64, inputs=4096, outputs=14336, bias=True, act="gelu"),
        # odd sizes, rows apart from each other, an fp32 residual stream
        _linear(name="linear_ragged_t777", tokens=777, inputs=2040, outputs=1411, out="f32", bias=True, act="gelu_tanh",
                residual=True, pad=8),
        # a long prompt's projection back to the residual stream
        _linear(name="linear_t8192_res", tokens=8192, inputs=4096, outputs=4096, bias=True, residual=True),
        # a server's usual decode step on a large layer with a shared expert, on the model's own routes
        _experts("decode_routed", "glm45air", name="glm_decode_routed_b128_m32", tokens=128, budget=32),
        # a long prompt on many small experts of uneven popularity, 8 given routes folded to 4
        _experts("prefill_routed", "qwen3", name="qwen3_prefill_routed_t4096_k4", tokens=4096, budget=4, zipf=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("route", "route", "route_backward", "linear", "linear", "linear", "linear", "experts", "experts"))
    if op in ("route", "route_backward"):
        groups = rng.choice((1, 1, 2, 4, 8))
        n = groups * _log_int(rng, 4, 256 // groups)
        top_groups = rng.randint(1, groups)
        c = _route(op, tokens=_log_int(rng, 1, 16384 * 128 // n if op == "route" else 8192 * 128 // n), experts=n,
                   groups=groups, top_groups=top_groups, top_k=rng.randint(1, min(10, n // groups * top_groups)),
                   group_score=rng.choice(("max", "top2")), score=rng.choice(("sigmoid", "softmax")),
                   bias=rng.random() < 0.6, renormalise=rng.random() < 0.6, scale=rng.choice((1.0, 2.5)),
                   masked=rng.random() < 0.3, zipf=rng.random() < 0.4)
        return c
    if op == "linear":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        t = _log_int(rng, 1, 8192 if dtype == "bf16" else 1024)
        unit = rng.choice((1, 8, 64))
        hi = 14336 if dtype == "bf16" else 2048
        sizes = [max(1, unit * round(_log_int(rng, 64, hi) / unit)) for _ in range(2)]
        while 2.0 * t * sizes[0] * sizes[1] > (MAX_LINEAR_FLOPS if dtype == "bf16" else 4e9):
            t = max(1, t * 3 // 4)
        return _linear(tokens=t, inputs=sizes[0], outputs=sizes[1], dtype=dtype,
                       out="f32" if dtype == "f32" else rng.choice(("bf16", "bf16", "f32")), bias=rng.random() < 0.5,
                       act=rng.choice(ACTIVATIONS), residual=rng.random() < 0.5, pad=rng.choice((0, 0, 8)))
    op = rng.choice(("prefill_routed", "decode_routed"))
    shape = rng.choice(("tiny", "mixtral", "qwen3", "glm45air", None))
    if shape is None:
        n = _log_int(rng, 4, 256)
        shape = (n, rng.randint(0, 1), 64 * _log_int(rng, 2, 32), 64 * _log_int(rng, 2, 16), rng.randint(1, min(n, 10)), "bf16")
    c = _experts(op, shape, zipf=rng.random() < 0.5)
    c["tokens"] = _log_int(rng, 1, 256 if op == "decode_routed" else 4096)
    c["budget"] = _log_int(rng, 1, c["experts"]) if op == "decode_routed" else rng.randint(1, c["top_k"])
    while c["tokens"] > 1 and 6.0 * c["hidden"] * c["inter"] * c["tokens"] * (c["top_k"] + c["shared"]) > MAX_EXPERT_FLOPS * 2:
        c["tokens"] = max(1, c["tokens"] * 3 // 4)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _scores(c, rng_np, normal):
    """Router scores N(0, 1), with a Zipf popularity of the experts on top where the case has one."""
    z = normal((c["tokens"], c["experts"]), 1.0, torch.float32)
    if c["zipf"]:
        p = np.arange(1, c["experts"] + 1, dtype=np.float64) ** -1.1
        z += torch.from_numpy(np.log(p / p.sum())[rng_np.permutation(c["experts"])].astype(np.float32)).to(z.device)
    return z


def _tables(n, rng):
    """Calibrated tables of the geometry that real layers show (norms over a factor of three, S = similarity times norm ratio)."""
    h = np.exp(rng.uniform(0.0, np.log(3.2), size=n))
    c = np.triu(rng.uniform(0.2, 0.9, size=(n, n)), 1)
    c = c + c.T
    S = np.clip(c * h[:, None] / h[None, :], -4.0, 4.0)
    S = np.where(rng.uniform(size=(n, n)) < 0.10, -S, S)
    L = 1.0 - c * c
    np.fill_diagonal(S, 1.0)
    np.fill_diagonal(L, 0.0)
    h = h.astype(np.float32)
    return S.astype(np.float32), L.astype(np.float32), h, np.log(h.astype(np.float64)).astype(np.float32)


def prepare(case, seed):
    c, dev = dict(case), torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng([seed, 13])

    def normal(shape, std, dt):
        return torch.empty(shape, dtype=dt, device=dev).normal_(0.0, std, generator=g)

    st = {"case": c, "seed": seed}
    if c["op"] in ("route", "route_backward"):
        t, n, k = c["tokens"], c["experts"], c["top_k"]
        st["logits"] = _scores(c, rng, normal)
        st["bias"] = normal((n,), 0.1, torch.float32) if c["bias"] else None
        if c["masked"]:  # experts that a token may not use; one token that may use none
            out = torch.rand((t, n), generator=g, device=dev) < 0.08
            st["logits"][out] = float("-inf")
            if t > 2:
                st["logits"][t // 2] = torch.finfo(torch.float32).min
        if c["op"] == "route_backward":
            st["ids"] = _choose(c, st["logits"], st["bias"])[0].to(torch.int32)
            st["dw"] = normal((t, k), 1.0, torch.float32)
        if own:
            from paper_2608_24938_b200 import binding as ex
            st["layer"] = ex.make_layer(n, 0, 64, 64, k, torch.float32)
            st["opts"] = ex.make_router(c["score"], bias=st["bias"], n_groups=c["groups"], top_groups=c["top_groups"],
                                        group_score=c["group_score"], renormalise=c["renormalise"], scale=c["scale"])
            if c["op"] == "route":
                st["ids"] = torch.empty((t, k), dtype=torch.int32, device=dev)
                st["w"] = torch.empty((t, k), dtype=torch.float32, device=dev)
                st["load"] = torch.empty(n, dtype=torch.int32, device=dev)
            else:
                st["dlogits"] = torch.empty((t, n), dtype=torch.float32, device=dev)
        return st
    dt = _dtype(c["dtype"])
    if c["op"] == "linear":
        t, i, o, pad, out = c["tokens"], c["inputs"], c["outputs"], c["pad"], _dtype(c["out"])

        def rows(r, cols, std, dtype):  # rows `pad` elements (and what aligns them to 8) apart
            ld = cols if pad == 0 else (cols + 7) // 8 * 8 + pad
            return normal((r, ld), std, dtype)[:, :cols]

        st["x"], st["w"] = rows(t, i, 1.0, dt), rows(o, i, i ** -0.5, dt)
        st["bias"] = normal((o,), 0.5, dt) if c["bias"] else None
        st["residual"] = rows(t, o, 1.0, out) if c["residual"] else None
        if own:
            from paper_2608_24938_b200 import binding as ex
            st["y"] = torch.empty((t, o), dtype=out, device=dev)
            st["ws"] = ex.alloc_linear_workspace(i, o, t, dt, device=dev)
        return st
    n, s, d, i, k = (c[f] for f in LAYER[:5])
    t = c["tokens"]
    st["x"] = normal((t, d), 1.0, dt)
    std = 0.02 if d >= 1024 else 0.05
    st["w"] = [normal((n + s, i, d), std, dt), normal((n + s, i, d), std, dt), normal((n + s, d, i), std, dt)]
    # the routes of a sigmoid router with renormalised weights
    z = torch.sigmoid(_scores(c, rng, normal))
    top = torch.topk(z, k, dim=1)
    st["ids"], st["rw"] = top.indices.to(torch.int32), top.values / top.values.sum(1, keepdim=True)
    st["tabs"] = [torch.from_numpy(a).to(dev) for a in _tables(n, rng)]
    if own:
        from paper_2608_24938_b200 import binding as ex
        st["layer"] = ex.make_layer(n, s, d, i, k, dt)
        st["tables"] = ex.make_tables(*st["tabs"])
        st["y"] = torch.empty((t, d), dtype=dt, device=dev)
        st["ws"] = ex.alloc_workspace(st["layer"], t, c["budget"] if c["op"] == "prefill_routed" else k, device=dev)
    return st


# ------------------------------------------------------------------------------------------------ the calls
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2608_24938_b200 import binding as ex
    c = st["case"]
    if c["op"] == "route":
        ex.exfold_route(st["layer"], st["logits"], st["opts"], st["ids"], st["w"], st["load"])
        return {"ids": st["ids"], "w": st["w"], "load": st["load"]}
    if c["op"] == "route_backward":
        ex.exfold_route_backward(st["layer"], st["logits"], st["ids"], st["dw"], st["opts"], st["dlogits"])
        return st["dlogits"]
    if c["op"] == "linear":
        ex.exfold_linear(st["x"], st["w"], st["y"], st["ws"], bias=st["bias"], residual=st["residual"], activation=c["act"])
        return st["y"]
    call = ex.exfold_moe_prefill_routed if c["op"] == "prefill_routed" else ex.exfold_moe_decode_routed
    call(st["layer"], st["x"], st["ids"], st["rw"], *st["w"], st["tables"], c["budget"], st["y"], st["ws"])
    return st["y"]


# ------------------------------------------------------------------------------------------------ plain forms
def _choose(c, logits, bias):
    """Chosen experts and every expert's score, in 64 bits: choices lie next to ties."""
    z = logits.double()
    masked = logits <= torch.finfo(torch.float32).min
    if c["score"] == "sigmoid":
        s = torch.sigmoid(z)
    else:
        e = torch.exp(z - z.amax(1, keepdim=True))
        s = e / e.sum(1, keepdim=True)
    s = torch.where(masked, 0.0, s)
    choice = s if bias is None else s + bias.double()
    if bias is None and (c["groups"] == 1 or c["group_score"] == "max"):
        choice = z  # the same order
    choice = torch.where(masked, float("-inf"), choice)
    n, g = c["experts"], c["groups"]
    if g > 1:
        per = choice.view(-1, g, n // g)
        if c["group_score"] == "max" or n == g:
            gs = per.amax(2)
        else:
            two = torch.topk(per, 2, dim=2).values
            gs = two[..., 0] + torch.where(torch.isneginf(two[..., 1]), 0.0, two[..., 1])
        best = torch.sort(gs, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros_like(gs, dtype=torch.bool).scatter_(1, best, True).repeat_interleave(n // g, dim=1)
        # experts of the other groups come last, behind the masked ones of the best groups
        order = torch.sort(choice, dim=1, descending=True, stable=True).indices
        order = order.gather(1, torch.sort((~keep).gather(1, order).to(torch.int8), dim=1, stable=True).indices)
    else:
        order = torch.sort(choice, dim=1, descending=True, stable=True).indices
    return order[:, :c["top_k"]], s


def _plain_route(c, logits, bias):
    ids, s = _choose(c, logits, bias)
    w = s.gather(1, ids)
    if c["renormalise"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total != 0, w / total, 0.0)
    load = torch.zeros(c["experts"], dtype=torch.int64, device=ids.device)
    load.scatter_add_(0, ids.reshape(-1), torch.ones_like(ids.reshape(-1)))
    return {"ids": ids.to(torch.int32), "w": (w * c["scale"]).float(), "load": load.to(torch.int32)}


def _plain_route_backward(c, logits, ids, dw):
    at = ids.long()
    masked = logits <= torch.finfo(torch.float32).min
    if c["score"] == "sigmoid":
        s = torch.sigmoid(logits)
    else:
        e = torch.exp(logits - logits.amax(1, keepdim=True))
        s = e / e.sum(1, keepdim=True)
    s = torch.where(masked, 0.0, s)
    sk = s.gather(1, at)
    if c["renormalise"]:
        total = sk.sum(1, keepdim=True)
        ds = torch.where(total != 0, (dw - (dw * sk).sum(1, keepdim=True) / total) / total, 0.0) * c["scale"]
    else:
        ds = dw * c["scale"]
    if c["score"] == "sigmoid":
        return torch.zeros_like(s).scatter_(1, at, ds * sk * (1.0 - sk))
    return torch.zeros_like(s).scatter_(1, at, ds * sk) - s * (ds * sk).sum(1, keepdim=True)


def _activate(v, name):
    if name == "relu":
        return torch.clamp(v, min=0.0)
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _plain_linear(st, dt):
    c = st["case"]
    v = st["x"].to(dt) @ st["w"].to(dt).t()
    if st["bias"] is not None:
        v = v + st["bias"].to(dt)
    v = _activate(v, c["act"])
    if st["residual"] is not None:
        v = v + st["residual"].to(dt)
    return v


def _plain_fold(c, ids, w, tabs):
    """Executed experts and their weights per slot ([T][slots], weight 0 where a slot was folded away)."""
    S, L, h, _ = tabs
    ids = ids.long()
    if c["op"] == "decode_routed":
        n = c["experts"]
        total = torch.zeros(n, dtype=torch.float64, device=w.device).index_add_(0, ids.reshape(-1), w.double().reshape(-1))
        used = torch.zeros(n, dtype=torch.bool, device=w.device).index_fill_(0, ids.reshape(-1), True)
        rank = torch.where(used, total * h.double(), float("-inf"))
        pool = torch.sort(rank, descending=True, stable=True).indices[:c["budget"]]
        in_pool = torch.zeros(n, dtype=torch.bool, device=w.device).index_fill_(0, pool, True) & used
        target = torch.where(in_pool, L, float("inf")).argmin(1)
        every = torch.arange(n, device=w.device)
        target = torch.where(in_pool, every, target)
        return target[ids], w * torch.where(in_pool, 1.0, S[every, target])[ids]
    key = w * h[ids]
    by_id = torch.sort(ids, dim=1).indices  # ties by the lower id
    order = by_id.gather(1, torch.sort(key.gather(1, by_id), dim=1, descending=True, stable=True).indices)
    ids, w, b = ids.gather(1, order), w.gather(1, order), c["budget"]
    kept, out = ids[:, :b], w[:, :b].clone()
    for j in range(b, ids.shape[1]):  # the omitted routes, in rank order, onto their minimum-loss targets
        loss = L[ids[:, j:j + 1], kept]
        best = loss.amin(1, keepdim=True)
        at = torch.where(loss == best, kept, c["experts"]).argmin(1, keepdim=True)
        out.scatter_add_(1, at, w[:, j:j + 1] * S[ids[:, j:j + 1], kept.gather(1, at)])
    return kept, out


def _plain_experts(st, dt):
    c = st["case"]
    ids, w = _plain_fold(c, st["ids"], st["rw"].to(dt), [t.to(dt) if dt == torch.float64 else t for t in st["tabs"]])
    wg, wu, wd = st["w"]
    x = st["x"].to(dt)
    y = torch.zeros_like(x)

    def expert(e, rows):
        a, b = rows @ wg[e].to(dt).t(), rows @ wu[e].to(dt).t()
        return (a / (1.0 + torch.exp(-a)) * b) @ wd[e].to(dt).t()

    order = torch.sort(ids.reshape(-1), stable=True).indices
    counts = torch.bincount(ids.reshape(-1), minlength=c["experts"]).tolist()
    tok, wt = order // ids.shape[1], w.reshape(-1)[order]
    r = 0
    for e, m in enumerate(counts):
        if m:
            y.index_add_(0, tok[r:r + m], expert(e, x[tok[r:r + m]]) * wt[r:r + m, None])
            r += m
    if c["shared"]:
        y += expert(c["experts"], x)
    return y


def _run_plain(st):
    c = st["case"]
    if c["op"] == "route":
        return _plain_route(c, st["logits"], st["bias"])
    if c["op"] == "route_backward":
        return _plain_route_backward(c, st["logits"], st["ids"], st["dw"])
    if c["op"] == "linear":
        return _plain_linear(st, torch.float32).to(_dtype(c["out"]))
    return _plain_experts(st, torch.float32).to(_dtype(c["dtype"]))


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _exact_scores(c, z):
    masked = z <= np.finfo(np.float32).min
    with np.errstate(over="ignore", invalid="ignore"):
        if c["score"] == "sigmoid":
            s = np.where(z >= 0, 1.0 / (1.0 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1.0 + np.exp(-np.abs(z))))
        else:
            s = np.exp(z - z.max(1, keepdims=True))
            s /= s.sum(1, keepdims=True)
    s[masked] = 0.0
    return s, masked


def _exact_route(c, z, bias):
    t, n = z.shape
    s, masked = _exact_scores(c, z)
    plain_order = bias is None and (c["groups"] == 1 or c["group_score"] == "max")
    choice = z.copy() if plain_order else s + (0.0 if bias is None else bias[None, :])
    choice[masked] = -np.inf
    per = n // c["groups"]
    gs = np.sort(choice.reshape(t, c["groups"], per), axis=2)[:, :, ::-1]
    score = gs[:, :, 0].copy()
    if c["group_score"] == "top2" and per > 1:
        score += np.where(np.isneginf(gs[:, :, 1]), 0.0, gs[:, :, 1])
    place = np.argsort(np.argsort(-score, axis=1, kind="stable"), axis=1, kind="stable")
    out = np.repeat(place >= c["top_groups"], per, axis=1)
    ids = np.empty((t, c["top_k"]), np.int64)
    experts = np.arange(n)
    for i in range(t):
        ids[i] = np.lexsort((experts, -choice[i], out[i]))[:c["top_k"]]
    w = np.take_along_axis(s, ids, 1)
    if c["renormalise"]:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total != 0)
    return ids, w * c["scale"]


def _exact_route_backward(c, z, ids, dw):
    """The weights' Jacobian, product rule on w = scale s_k (/ sum of the chosen s), applied to dw."""
    s, _ = _exact_scores(c, z)
    rows = np.arange(len(z))[:, None]
    sk = s[rows, ids]
    total = sk.sum(1, keepdims=True)
    safe = np.where(total != 0, total, 1.0)
    if c["renormalise"]:
        gs = np.where(total != 0, dw / safe - (dw * sk).sum(1, keepdims=True) / safe ** 2, 0.0)
    else:
        gs = dw
    grad_s = np.zeros_like(s)
    grad_s[rows, ids] = gs * c["scale"]
    if c["score"] == "sigmoid":
        return grad_s * s * (1.0 - s)
    return s * (grad_s - (grad_s * s).sum(1, keepdims=True))


def _exact_activation(v, name):
    if name == "relu":
        return torch.maximum(v, torch.zeros_like(v))
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "gelu_tanh":
        u = (2.0 / math.pi) ** 0.5 * (v + 0.044715 * v * v * v)
        return v * torch.sigmoid(2.0 * u)
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def _exact_experts(st):
    """Token by token on the host for the fold, expert by expert for the products."""
    c = st["case"]
    S, L, h = (_np(t) for t in st["tabs"][:3])
    ids, w, n = st["ids"].cpu().numpy(), _np(st["rw"]), c["experts"]
    t = len(ids)
    gate = np.zeros((t, n))
    if c["op"] == "decode_routed":
        total = np.zeros(n)
        np.add.at(total, ids, w)
        union = np.unique(ids)
        pool = sorted(union.tolist(), key=lambda e: (-total[e] * h[e], e))[:c["budget"]]
        for i in range(t):
            for e, we in zip(ids[i], w[i]):
                to = e if e in pool else min(pool, key=lambda p: (L[e, p], p))
                gate[i, to] += we * S[e, to]
    else:
        w32, h32 = st["rw"].cpu().numpy(), st["tabs"][2].cpu().numpy()
        for i in range(t):
            order = sorted(range(ids.shape[1]), key=lambda j: (-(w32[i, j] * h32[ids[i, j]]), ids[i, j]))
            kept = [int(ids[i, j]) for j in order[:c["budget"]]]
            for j in order[:c["budget"]]:
                gate[i, ids[i, j]] += w[i, j]
            for j in order[c["budget"]:]:
                to = min(kept, key=lambda p: (L[ids[i, j], p], p))
                gate[i, to] += w[i, j] * S[ids[i, j], to]
    gate = torch.from_numpy(gate).to(st["x"].device)
    x = st["x"].double()
    y = torch.zeros_like(x)
    for e in range(n + c["shared"]):
        if e < n:
            rows = torch.nonzero(gate[:, e]).flatten()
            weight = gate[rows, e]
        else:
            rows, weight = torch.arange(t, device=x.device), torch.ones(t, dtype=torch.float64, device=x.device)
        if rows.numel() == 0:
            continue
        up, down = x[rows] @ st["w"][1][e].double().T, x[rows] @ st["w"][0][e].double().T
        y[rows] += weight[:, None] * ((down * torch.sigmoid(down) * up) @ st["w"][2][e].double().T)
    return y


def exact(case, seed):
    st = prepare(case, seed)
    c = st["case"]
    if c["op"] == "route":
        ids, w = _exact_route(c, _np(st["logits"]), _np(st["bias"]))
        return {"ids": torch.from_numpy(ids), "w": torch.from_numpy(w),
                "load": torch.from_numpy(np.bincount(ids.ravel(), minlength=c["experts"]))}
    if c["op"] == "route_backward":
        return torch.from_numpy(_exact_route_backward(c, _np(st["logits"]), st["ids"].cpu().numpy().astype(np.int64), _np(st["dw"])))
    if c["op"] == "linear":
        v = torch.einsum("ti,oi->to", st["x"].double(), st["w"].double())
        if st["bias"] is not None:
            v += st["bias"].double()
        v = _exact_activation(v, c["act"])
        return v if st["residual"] is None else v + st["residual"].double()
    return _exact_experts(st)


# ------------------------------------------------------------------------------------------------ accounting
def _executed(c):
    """(experts whose weights are read, executed routed rows) of one call, from routes of the case's distribution."""
    rng = np.random.default_rng(11)
    n, k = c["experts"], c["top_k"]
    z = rng.standard_normal((c["tokens"], n))
    if c["zipf"]:
        p = np.arange(1, n + 1, dtype=np.float64) ** -1.1
        z += np.log(p / p.sum())[rng.permutation(n)]
    top = np.argsort(-z, axis=1)[:, :k]
    _, L, h, _ = _tables(n, rng)
    w = 1.0 / (1.0 + np.exp(-np.take_along_axis(z, top, 1)))
    w /= w.sum(1, keepdims=True)
    if c["op"] == "prefill_routed":
        kept = np.take_along_axis(top, np.argsort(-(w * h[top]), axis=1)[:, :c["budget"]], 1)
    else:
        score = np.zeros(n)
        np.add.at(score, top, w)
        union = np.flatnonzero(score)
        pool = union[np.argsort(-(score * h)[union])][:c["budget"]]
        kept = np.where(np.isin(np.arange(n), pool), np.arange(n), pool[np.argmin(L[:, pool], axis=1)])[top]
    return len(np.unique(kept)), sum(len(set(r)) for r in kept.tolist())


def work(case):
    c, t = case, case["tokens"]
    if c["op"] in ("route", "route_backward"):
        n, k = c["experts"], c["top_k"]
        if c["op"] == "route":  # the scores, the bias, ids and weights, the load
            return {"bytes": 4.0 * t * n + (4 * n if c["bias"] else 0) + 8.0 * t * k + 4 * n, "flops": 4.0 * t * n}
        # the gradient; all scores, or the chosen ones; ids and weights' gradients
        read = 4.0 * t * (n if c["score"] == "softmax" and not c["renormalise"] else k)
        return {"bytes": 4.0 * t * n + read + 8.0 * t * k, "flops": 2.0 * t * n + 8.0 * t * k}
    el = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "linear":
        i, o, ey = c["inputs"], c["outputs"], 4 if c["out"] == "f32" else 2
        nbytes = float(el) * (t * i + o * i) + (el * o if c["bias"] else 0) + ey * t * o * (2.0 if c["residual"] else 1.0)
        return {"bytes": nbytes, "flops": 2.0 * t * i * o}
    touched, rows = _executed(c)
    d, i, s = c["hidden"], c["inter"], c["shared"]
    return {"bytes": (touched + s) * 3.0 * d * i * el + 2.0 * t * d * el + 8.0 * t * c["top_k"],
            "flops": 6.0 * d * i * (rows + s * t)}
