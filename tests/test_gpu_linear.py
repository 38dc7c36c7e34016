"""The dense product with bias, activation and residual against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def ex():
    from paper_2608_24938_b200 import binding
    return binding


def act64(v, name):
    if name == "relu":
        return torch.relu(v)
    if name == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def reference(x, w, bias, residual, act, out):
    """(value, bound of the error). Products of bf16 are exact in fp32, of fp32 rounded; sums are taken in fp32, on the tensor cores
    in steps of 16 products that may be cut off instead of rounded: (in / 8 + 16) 2^-23 of the sum of magnitudes there, and
    (in + 2) 2^-24 of it where each product is added with one rounding. Activations have slopes up to 1.13 and are computed to
    8 half steps of their argument; then the residual's addition and half a step of the output."""
    X, W = x.double(), w.double()
    K = x.shape[1]
    pre = X @ W.T
    mag = X.abs() @ W.abs().T
    if bias is not None:
        pre = pre + bias.double()
        mag = mag + bias.double().abs()
    steps = max((K / 8 + 16) * 2.0 ** -23 if x.dtype == torch.bfloat16 else 0.0, (K + 2) * 2.0 ** -24)
    err = 1.13 * steps * mag + 8 * 2.0 ** -24 * pre.abs()
    v = act64(pre, act)
    if residual is not None:
        err = err + 2.0 ** -24 * (v.abs() + residual.double().abs())
        v = v + residual.double()
    half = 2.0 ** -8 if out == torch.bfloat16 else 2.0 ** -24
    return v, err + half * (v.abs() + err) + 2.0 ** -126


def rows(r, c, dtype, seed, std=1.0, ld=None, offset=0):
    """r x c with rows ld elements apart, `offset` elements into a buffer; what lies between and around holds NaN."""
    g = torch.Generator().manual_seed(seed)
    ld = c if ld is None else ld
    buf = torch.full((offset + r * ld + 64,), float("nan"), dtype=dtype)
    view = buf[offset:offset + r * ld].view(r, ld)[:, :c]
    view.copy_((torch.randn((r, c), generator=g) * std).to(dtype))
    dev = buf.cuda()
    return dev[offset:offset + r * ld].view(r, ld)[:, :c], dev


def check(ex, T, i, o, dtype=torch.bfloat16, out=None, bias=True, residual=True, act="none", ldx=None, ldw=None, ldy=None, ldr=None,
          offset=0, in_place=False, seed=0):
    out = dtype if out is None else out
    x, _ = rows(T, i, dtype, seed + 1, ld=ldx, offset=offset)
    w, _ = rows(o, i, dtype, seed + 2, std=i ** -0.5, ld=ldw, offset=offset)
    b = rows(1, o, dtype, seed + 3, offset=offset)[0][0] if bias else None
    y, ybuf = rows(T, o, out, seed + 4, ld=ldy, offset=offset)
    r = None
    if residual:
        r = y if in_place else rows(T, o, out, seed + 5, ld=ldr, offset=offset)[0]
    ref, bound = reference(x, w, b, r, act, out)
    if not in_place:
        y.fill_(float("nan"))
    around = torch.ones_like(ybuf, dtype=torch.bool)
    around[offset:offset + T * (ldy or o)].view(T, ldy or o)[:, :o] = False
    ws = ex.alloc_linear_workspace(i, o, T, dtype, out, ldx=ldx or 0, ldw=ldw or 0)
    ws.fill_(0xFF)
    ex.exfold_linear(x, w, y, ws, bias=b, residual=r, activation=act)
    assert ex.exfold_device_status(ws) == 0
    assert ybuf[around].isnan().all(), "something beside the rows was written"
    got = y.double()
    assert got.isfinite().all()
    bad = (got - ref).abs() > bound
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside the bound, worst {float(((got - ref).abs() / bound).max()):.2f}"
    return y


TOKENS = [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33, 64, 65, 100, 127, 128, 129, 200, 256, 257, 300, 513]


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("i,o", [(64, 64), (128, 256), (256, 40), (1024, 520), (2048, 768)])
def test_linear_bf16(ex, T, i, o):
    check(ex, T, i, o, act="silu")
    check(ex, T, i, o, out=torch.float32, bias=False, act="gelu")


@pytest.mark.parametrize("T", [1, 5, 12, 64, 130, 300, 700])
@pytest.mark.parametrize("i,o", [(8, 1), (1, 8), (1, 1), (72, 7), (136, 129), (200, 333), (1000, 1411), (2040, 257), (63, 65), (517, 100),
                                 (6591, 64)])
def test_linear_odd_sizes(ex, T, i, o):
    pad = (i + 7) // 8 * 8 + 8
    check(ex, T, i, o, act="gelu_tanh")
    check(ex, T, i, o, ldx=pad, ldw=pad, ldy=o + 3, ldr=o + 5, act="relu")
    check(ex, T, i, o, out=torch.float32, ldx=pad, ldw=pad + 8, ldy=o + 1)


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
def test_linear_epilogues(ex, dtype, out, act, bias, residual):
    for T in (1, 20, 300):
        check(ex, T, 192, 264, dtype, out, bias, residual, act)


@pytest.mark.parametrize("T", [1, 2, 9, 64, 100, 257, 1000])
@pytest.mark.parametrize("i,o", [(1, 1), (3, 5), (128, 256), (100, 129), (517, 64), (768, 2048)])
def test_linear_f32(ex, T, i, o):
    check(ex, T, i, o, torch.float32, act="silu")
    check(ex, T, i, o, torch.float32, ldx=i + 1, ldw=i + 3, ldy=o + 1, ldr=o, act="none")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 6, 40, 200, 600])
@pytest.mark.parametrize("offset", [1, 4, 8])
def test_linear_unaligned_operands(ex, dtype, T, offset):
    """Operands that start anywhere in a buffer, dense and with odd row distances."""
    check(ex, T, 264, 136, dtype, offset=offset, act="relu")
    check(ex, T, 264, 136, dtype, offset=offset, ldx=267, ldw=265, ldy=137, ldr=139)
    check(ex, T, 265, 135, dtype, offset=offset)


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T", [1, 8, 33, 129, 520])
def test_linear_in_place_residual(ex, dtype, out, T):
    check(ex, T, 256, 512, dtype, out, in_place=True, act="gelu")
    check(ex, T, 256, 500, dtype, out, in_place=True, ldy=504)


@pytest.mark.parametrize("T,i,o", [(2048, 4096, 1408), (1300, 2048, 4096), (4096, 768, 2048), (300, 4096, 14336), (5, 4096, 14336),
                                   (16, 14336, 4096), (777, 2040, 1411)])
def test_linear_large(ex, T, i, o):
    check(ex, T, i, o, act="gelu_tanh")


@pytest.mark.parametrize("T", [1, 9, 140, 700])
@pytest.mark.parametrize("i", [1, 7, 9, 63, 65, 514, 1411])
def test_linear_copied_rows(ex, T, i):
    """bf16 rows at odd distances, from every alignment of the matrix' start; NaN before, between and behind them."""
    for offset in range(0, 9):
        check(ex, T, i, 136, offset=offset, ldx=i + (i + 1) % 2, ldw=i + 2 + (i + 1) % 2)
    check(ex, T, i, 136, ldx=(i + 7) // 8 * 8, ldw=i + 3)
    check(ex, T, i, 136, ldx=i + 3, ldw=(i + 7) // 8 * 8)


def test_linear_zero_tokens_writes_nothing(ex):
    w = torch.ones((8, 64), dtype=torch.bfloat16, device="cuda")
    ws = ex.alloc_linear_workspace(64, 8, 0, torch.bfloat16)
    ex.exfold_linear(w[:0], w, torch.empty((0, 8), dtype=torch.bfloat16, device="cuda"), ws)


@pytest.mark.parametrize("T", [1, 16, 130, 700])
def test_linear_rows_do_not_mix(ex, T):
    """An infinity or NaN in one token's row stays there; weights of unused columns do too."""
    x, _ = rows(T, 256, torch.bfloat16, 1)
    w, _ = rows(264, 256, torch.bfloat16, 2)
    ws = ex.alloc_linear_workspace(256, 264, T, torch.bfloat16)
    y0, y1 = (torch.empty((T, 264), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ex.exfold_linear(x, w, y0, ws)
    w2, x2 = w.clone(), x.clone()
    w2[3, 5] = float("inf")
    x2[T - 1, 7] = float("nan")
    ex.exfold_linear(x2, w2, y1, ws)
    keep = torch.arange(264, device="cuda") != 3
    assert torch.equal(y0[:T - 1, keep], y1[:T - 1, keep])
    assert y1[T - 1].isnan().all() and not y1[:T - 1, 3].isfinite().any()


@pytest.mark.parametrize("T", [1, 24, 200, 1500])
def test_linear_is_reproducible_and_captured(ex, T):
    i, o = 1024, 768
    x, _ = rows(T, i, torch.bfloat16, 1)
    w, _ = rows(o, i, torch.bfloat16, 2)
    ws, ws2 = (ex.alloc_linear_workspace(i, o, T, torch.bfloat16) for _ in range(2))
    y, y2, ref = (torch.empty((T, o), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    ex.exfold_linear(x, w, ref, ws)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        ex.exfold_linear(x, w, y, ws)
        ex.exfold_linear(x, w, y2, ws2)
    for _ in range(3):
        y.zero_(), y2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref) and torch.equal(y2, ref)
    # two streams at once, a workspace each
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    y.zero_(), y2.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        ex.exfold_linear(x, w, y, ws, stream=a)
        ex.exfold_linear(x, w, y2, ws2, stream=b)
    torch.cuda.synchronize()
    assert torch.equal(y, ref) and torch.equal(y2, ref)
    # new inputs right before the call, on the call's stream
    with torch.cuda.stream(a):
        x.mul_(2.0)
        ex.exfold_linear(x, w, y, ws, stream=a)
    torch.cuda.synchronize()
    assert torch.equal(y, ref * 2)


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("T", [3, 9])
def test_linear_rows_far_apart(ex, dtype, out, T):
    """Row offsets beyond 2^31 elements, of x and of y (in place on the residual)."""
    i, o, ld = 128, 64, ((1 << 31) // (T - 1) + 64) // 8 * 8
    x = torch.empty((T - 1) * ld + i, dtype=dtype, device="cuda").as_strided((T, i), (ld, 1))
    y = torch.empty((T - 1) * ld + o, dtype=out, device="cuda").as_strided((T, o), (ld, 1))
    g = torch.Generator(device="cuda").manual_seed(3)
    w = (torch.randn((o, i), generator=g, device="cuda") * i ** -0.5).to(dtype)
    x.copy_(torch.randn((T, i), generator=g, device="cuda").to(dtype))
    y.copy_(torch.randn((T, o), generator=g, device="cuda").to(out))
    ref, bound = reference(x, w, None, y, "silu", out)
    ws = ex.alloc_linear_workspace(i, o, T, dtype, out, ldx=ld)
    ex.exfold_linear(x, w, y, ws, residual=y, activation="silu")
    assert ex.exfold_device_status(ws) == 0
    assert ((y.double() - ref).abs() <= bound).all()


def test_linear_one_workspace_on_one_stream(ex):
    """Calls of different sizes and types one after the other on a stream share a workspace as large as the largest needs."""
    sizes = [(1, 65, 64), (300, 333, 129), (8, 64, 64), (64, 517, 200), (700, 256, 512), (3, 1411, 8)]
    need = max(ex.alloc_linear_workspace(i, o, t, torch.bfloat16).numel() for t, i, o in sizes)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    calls = []
    for n, (t, i, o) in enumerate(sizes * 2):
        g = torch.Generator(device="cuda").manual_seed(n)
        x = torch.randn((t, i), generator=g, device="cuda").bfloat16()
        w = (torch.randn((o, i), generator=g, device="cuda") * i ** -0.5).bfloat16()
        calls.append((x, w, torch.empty((t, o), dtype=torch.bfloat16, device="cuda")))
    for x, w, y in calls:
        ex.exfold_linear(x, w, y, ws, activation="relu")
    assert ex.exfold_device_status(ws) == 0
    for x, w, y in calls:
        ref, bound = reference(x, w, None, None, "relu", torch.bfloat16)
        assert ((y.double() - ref).abs() <= bound).all()


def test_linear_kernels_beside_each_other(ex):
    """Calls of every kernel on streams of their own, at the same time: each has the bits it has alone."""
    sizes = [(1, 1024, 2048, torch.bfloat16), (40, 2048, 1024, torch.bfloat16), (300, 1024, 1024, torch.bfloat16), (100, 2048, 40, torch.bfloat16),
             (2500, 1024, 2048, torch.bfloat16), (70, 517, 333, torch.bfloat16), (100, 512, 512, torch.float32), (6, 512, 512, torch.float32)]
    jobs = []
    for n, (t, i, o, dtype) in enumerate(sizes):
        g = torch.Generator(device="cuda").manual_seed(n)
        x = torch.randn((t, i), generator=g, device="cuda").to(dtype)
        w = (torch.randn((o, i), generator=g, device="cuda") * i ** -0.5).to(dtype)
        r = torch.randn((t, o), generator=g, device="cuda").to(dtype)
        alone, y = torch.empty_like(r), torch.empty_like(r)
        ws = ex.alloc_linear_workspace(i, o, t, dtype)
        ex.exfold_linear(x, w, alone, ws, residual=r, activation="silu")
        assert ex.exfold_device_status(ws) == 0
        jobs.append((x, w, y, ws, r, alone, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(30):
        for x, w, y, ws, r, _, stream in jobs:
            ex.exfold_linear(x, w, y, ws, residual=r, activation="silu", stream=stream)
    torch.cuda.synchronize()
    for x, w, y, ws, r, alone, _ in jobs:
        assert ex.exfold_device_status(ws) == 0 and torch.equal(y, alone)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("o", [4097, 4098, 4099, 4100, 4101, 4102, 4103, 4104, 4112, 4120])
@pytest.mark.parametrize("T,i", [(2001, 512), (3001, 200)])
def test_linear_pairs_write_nothing_behind_the_columns(ex, T, i, o, out):
    """Rows whose distance suits a tensor map but whose length does not: what lies between them is the caller's."""
    gap = (o + 7) // 8 * 8 + 16
    check(ex, T, i, o, out=out, act="relu", ldy=gap, ldr=gap + 8)
    check(ex, T, i, o, out=out, residual=False, ldy=gap)
    check(ex, T, i, o, out=out, bias=False, in_place=True, ldy=gap)


@pytest.mark.parametrize("K", [4096, 520, 517])
def test_linear_single_rows_of_wide_matrices(ex, K):
    """The distance to a next row means nothing where there is none: one token, or one feature, cut from a matrix whose rows lie at
    odd distances, on the workspace of dense rows."""
    pad = (K + 7) // 8 * 8
    for at in range(8):
        wide = rows(9, K + 3 + K % 2, torch.bfloat16, 1 + at)[0]
        row = wide[at:at + 1, :K]
        many = rows(300, K, torch.bfloat16, 20, std=K ** -0.5, ld=pad)[0]
        for T, o in ((1, 300), (1, 1), (5, 1), (300, 1)):
            x, w = (row, many[:o]) if T == 1 else (many[:T], row)
            ws = ex.alloc_linear_workspace(K, o, T, torch.bfloat16, ldx=0 if T == 1 else pad, ldw=0 if o == 1 else pad)
            ws.fill_(0xFF)
            r = rows(T, o, torch.bfloat16, 30)[0]
            y = torch.full((T, o), float("nan"), dtype=torch.bfloat16, device="cuda")
            ex.exfold_linear(x, w, y, ws, residual=r, activation="silu")
            assert ex.exfold_device_status(ws) == 0
            ref, bound = reference(x, w, None, r, "silu", torch.bfloat16)
            assert ((y.double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("K", [512, 517])
@pytest.mark.parametrize("T,o", [(2, 600), (600, 3), (40, 300), (700, 520)])
@pytest.mark.parametrize("odd", ["x", "w"])
def test_linear_copies_only_what_lies_oddly(ex, K, T, o, odd):
    pad = (K + 7) // 8 * 8
    ld = K + 1 + K % 2  # odd
    ldx, ldw = (ld, pad) if odd == "x" else (pad, ld)
    x, w = rows(T, K, torch.bfloat16, 1, ld=ldx)[0], rows(o, K, torch.bfloat16, 2, std=K ** -0.5, ld=ldw)[0]
    ws = ex.alloc_linear_workspace(K, o, T, torch.bfloat16, ldx=ldx, ldw=ldw)
    ws.fill_(0xFF)
    y = torch.full((T, o), float("nan"), dtype=torch.bfloat16, device="cuda")
    ex.exfold_linear(x, w, y, ws)
    assert ex.exfold_device_status(ws) == 0
    ref, bound = reference(x, w, None, None, "none", torch.bfloat16)
    assert ((y.double() - ref).abs() <= bound).all()
    if T > 8 or odd == "x":  # (with few tokens their copy costs nothing)
        copied = int((ws[256:] != 0xFF).sum())
        assert copied <= (T if odd == "x" else o) * ((K + 15) // 16 * 32), "more than the one matrix was copied"


def test_linear_empty_call_leaves_everything(ex):
    """No tokens: no output, no workspace is written, and a new workspace's status reads as no error."""
    n = ex.alloc_linear_workspace(64, 8, 4, torch.bfloat16).numel()
    stale = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    del stale  # the allocator hands these out again
    for dtype in (torch.bfloat16, torch.float32):
        w = torch.ones((8, 64), dtype=dtype, device="cuda")
        ws = ex.alloc_linear_workspace(64, 8, 4, dtype)
        assert ex.exfold_device_status(ws) == 0
        ws[256:] = 0xFF
        before, y = ws.clone(), torch.full((4, 8), 7.0, dtype=dtype, device="cuda")
        ex.exfold_linear(w[:0], w, y[:0], ws, activation="relu")
        assert ex.exfold_device_status(ws) == 0 and torch.equal(ws, before) and bool((y == 7).all())


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype,T,i,o", [(torch.float32, 40, 1, 9), (torch.float32, 300, 3, 70), (torch.float32, 1024, 16, 2048),
                                         (torch.bfloat16, 5, 64, 40), (torch.bfloat16, 300, 64, 264), (torch.bfloat16, 8192, 64, 5000)])
def test_linear_activations_far_out(ex, act, dtype, T, i, o):
    """Every activation in half steps of its own value, also where it tends to 0: one input counts, so that the sum is exact.
    gelu: erfc to 4 steps, its argument to 3 half steps, which count (v^2 + 1) times; gelu_tanh and silu: v / (1 + e^-a), a to 8 half
    steps (silu: exact), exp to 2 steps, the sum and the quotient to 4 half steps."""
    v = torch.linspace(-9, 9, T).to(dtype)
    x = torch.zeros((T, i), dtype=dtype)
    x[:, i // 2] = v
    w = torch.ones((o, i), dtype=dtype)
    y = torch.full((T, o), float("nan"), device="cuda")
    ws = ex.alloc_linear_workspace(i, o, T, dtype, torch.float32)
    ex.exfold_linear(x.cuda(), w.cuda(), y, ws, activation=act)
    assert ex.exfold_device_status(ws) == 0
    d = v.double()
    a = 2 * math.sqrt(2 / math.pi) * (d + 0.044715 * d ** 3)
    ref = {"gelu": 0.5 * d * torch.special.erfc(-d / math.sqrt(2)), "gelu_tanh": d / (1 + torch.exp(-a)), "silu": d / (1 + torch.exp(-d))}[act]
    steps = {"gelu": 8 + 3 * (d * d + 1) + 4, "gelu_tanh": 8 * a.abs() + 8 + 4, "silu": torch.full_like(d, 12.0)}[act]
    bound = (steps * 2.0 ** -24 * ref.abs() + 2.0 ** -126)[:, None].cuda()
    err = (y.double() - ref[:, None].cuda()).abs()
    assert (err <= bound).all(), f"worst {float((err / bound).max()):.1f} of the bound"


# Sizes that take the CTA pairs (linear_prefers_pairs), many of them with several items per pair or bands of row tiles
PAIRS = [(2500, 1024, 2048), (6000, 72, 4099), (4096, 200, 2001), (8192, 4096, 2048), (1029, 4104, 4099), (300, 4096, 14336)]


@pytest.mark.parametrize("T,i,o", PAIRS)
def test_linear_pairs_results_and_residuals(ex, T, i, o):
    """What the CTA-pair kernel does to its sums: results of both types, rows that a tensor map takes and rows that none does, with a
    residual, without, and in place; K that ends inside a block, features that end inside 32 columns."""
    p = (i + 7) // 8 * 8
    p = dict(ldx=p, ldw=p)
    even = (o + 7) // 8 * 8 + 8
    check(ex, T, i, o, out=torch.float32, act="gelu", **p, ldy=even, ldr=even)
    check(ex, T, i, o, out=torch.float32, act="relu", residual=False, **p, ldy=even)
    check(ex, T, i, o, out=torch.float32, **p, ldy=o + 1 + o % 2, ldr=o + 3 + o % 2)
    check(ex, T, i, o, act="silu", residual=False, **p, ldy=even)
    check(ex, T, i, o, act="gelu_tanh", bias=False, **p, ldy=even, ldr=even)
    check(ex, T, i, o, **p, ldy=o + 1 + o % 2, ldr=o + 3 + o % 2)
    check(ex, T, i, o, residual=False, **p, ldy=o + 1 + o % 2)


@pytest.mark.parametrize("T,i,o", PAIRS)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_linear_pairs_in_place(ex, T, i, o, out):
    p = (i + 7) // 8 * 8
    even = (o + 7) // 8 * 8
    check(ex, T, i, o, out=out, in_place=True, act="relu", ldx=p, ldw=p, ldy=even)
    check(ex, T, i, o, out=out, in_place=True, ldx=p, ldw=p, ldy=o + 1 + o % 2)


BIG = [(1000, 100, 2048), (1300, 768, 1411), (500, 258, 2048), (1300, 203, 768), (500, 500, 1000), (1300, 768, 333), (300, 500, 768),
       (1000, 507, 255), (128, 1411, 2048)]


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T,i,o", BIG)
def test_linear_large_cuda_core_tiles(ex, dtype, out, T, i, o):
    """The 128 x 128 tiles on the CUDA cores, with K in 1, 2, 4 and 8 parts: fp32 and bf16 that only starts unaligned, rows in fours and not."""
    offset = 0 if dtype == torch.float32 else 4
    unit = 4 if dtype == torch.float32 else 8
    ld = (i + unit - 1) // unit * unit
    check(ex, T, i, o, dtype, out, act="silu", offset=offset, ldx=ld, ldw=ld)
    check(ex, T, i, o, dtype, out, bias=False, offset=1, ldx=ld, ldw=ld, ldy=o + 3, ldr=o + 1)
    check(ex, T, i, o, dtype, out, residual=False, offset=offset, ldx=ld, ldw=ld, ldy=o + 2)
