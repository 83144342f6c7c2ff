"""GPU parity of the matrix product with bias, activation and residual and of its gradients against the definition in 64 bits:
sizes that no tile divides, single rows, views with strides and odd addresses, streams and graphs.

Tolerances, per element.  A sum of n products in fp32 is off by at most n 2^-24 sum |a_i b_i| (check mode: in double, 2^-53),
a result is rounded once by half a step (bf16 2^-8, fp32 2^-24, relative); an activation passes on the error of z times its
largest slope (1.13) and adds its own evaluation error, at most 2^-20 (check mode: 2^-50) of 1 + |z|."""
import math

import pytest

pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "gelu", "silu")
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
UNIT = {"bf16": 2.0 ** -24, "f32": 2.0 ** -53}      # of the sums
EVAL = {"bf16": 2.0 ** -20, "f32": 2.0 ** -50}      # of the activations
SHAPES = [
    # rows, inputs, outputs
    (1, 1, 1), (1, 64, 64), (1, 4096, 512), (1, 1000, 4096), (2, 10, 10), (3, 33, 1), (5, 1, 7), (7, 8, 8), (16, 512, 4096),
    (17, 100, 65), (31, 4096, 10), (33, 72, 256), (64, 64, 64), (127, 129, 131), (128, 512, 4096), (128, 4096, 10), (200, 2048, 1000),
    (256, 256, 256), (300, 1000, 10), (513, 72, 520), (777, 1032, 264), (1021, 257, 1000), (1024, 1024, 1024), (2049, 640, 1111),
    (2304, 320, 2560),
]


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    from paper_1911_05146_amd import hpf
    return hpf, torch, {m: hpf.Ops(hpf.HPF_BF16 if m == "bf16" else hpf.HPF_F32) for m in HALF}


def tdtype(torch, mode):
    return torch.bfloat16 if mode == "bf16" else torch.float32


def make(torch, mode, M, K, N, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * M + 31 * K + 101 * N)
    t = tdtype(torch, mode)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)
    return dict(x=randn(M, K).to(t), w=randn(K, N) * math.sqrt(1.0 / K), bias=randn(N) * 0.3, residual=randn(M, N).to(t),
                dy=randn(M, N).to(t), z=randn(M, N) * 1.4)


def act64(torch, act, z):
    """act(z), act'(z) in 64 bits."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q * (1 + z * (1 - q))
    return z, torch.ones_like(z)


def z64(torch, mode, x, w, bias):
    """z and the bound of its error."""
    t = tdtype(torch, mode)
    x, w = x.double(), w.to(t).double()
    z, size = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    return z, (x.shape[1] + 8) * UNIT[mode] * size


def check(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got.double() - ref).abs() / tol.clamp(min=1e-300)).max()):.2f} of the bound"


def check_forward(torch, mode, act, y, slope, z, dz, residual):
    ref, sref = act64(torch, act, z)
    err = 1.13 * dz + (EVAL[mode] * (1 + z.abs()) if act in ("gelu", "silu") else 0)
    if residual is not None:
        ref = ref + residual.double()
        err = err + UNIT[mode] * (ref.abs() + residual.double().abs())
    check(y, ref, HALF[mode] * ref.abs() * 1.01 + err + 1e-38, "y")
    if slope is not None:
        tol = HALF[mode] * sref.abs() * 1.01 + dz + EVAL[mode] * (1 + z.abs())
        if act == "relu":
            tol = torch.where(z.abs() <= dz, 1.0, 0.0)        # on the border either is right
        check(slope, sref, tol, "slope")


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_every_activation(env, mode, shape):
    hpf, torch, ops = env
    M, K, N = shape
    print(f"\n[case] forward {shape} {mode}", flush=True)
    d = make(torch, mode, M, K, N)
    weights = ops[mode].linear_weights(d["w"])
    for i, act in enumerate(ACTS):
        bias = d["bias"] if i != 1 else None
        residual = d["residual"] if i in (0, 2) else None
        y, slope = ops[mode].linear_forward(d["x"], weights, bias, residual, act, slope=True)
        assert (slope is None) == (act == "none")
        z, dz = z64(torch, mode, d["x"], d["w"], bias)
        check_forward(torch, mode, act, y, slope, z, dz, residual)
        assert torch.equal(y, ops[mode].linear_forward(d["x"], weights, bias, residual, act)), "same inputs, other bits"


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_backward(env, mode, shape):
    hpf, torch, ops = env
    M, K, N = shape
    print(f"\n[case] backward {shape} {mode}", flush=True)
    d = make(torch, mode, M, K, N, seed=1)
    weights = ops[mode].linear_weights(d["w"])
    t = tdtype(torch, mode)
    w = d["w"].to(t).double()
    for act in ("none", "gelu"):
        slope = None if act == "none" else act64(torch, act, d["z"].double())[1].to(t)
        dz = d["dy"].double()
        if slope is not None:
            dz = (dz * slope.double()).to(t).double()
        dx, dw, db = ops[mode].linear_backward(d["dy"], d["x"], weights, slope)
        ref = dz @ w.t()
        check(dx, ref, HALF[mode] * 1.01 * ref.abs() + (N + 8) * UNIT[mode] * (dz.abs() @ w.t().abs()) + 1e-38, "dx")
        x = d["x"].double()
        ref, size = x.t() @ dz, x.t().abs() @ dz.abs()
        check(dw, ref, 2.0 ** -24 * ref.abs() * 1.01 + (M + 8) * UNIT[mode] * size + 1e-38, "dw")
        bref, bsize = dz.sum(0), dz.abs().sum(0)
        check(db, bref, 2.0 ** -24 * bref.abs() * 1.01 + (M + 8) * UNIT[mode] * bsize + 1e-38, "db")
        again = ops[mode].linear_backward(d["dy"], d["x"], weights, slope)
        assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db))), "same inputs, other bits"
        dw2, db2 = torch.full_like(dw, 3.0), torch.full_like(db, -2.0)
        only = ops[mode].linear_backward(d["dy"], d["x"], weights, slope, need_dx=False, dw=dw2, db=db2, accumulate=True)
        assert only[0] is None and only[1] is dw2
        check(dw2, ref + 3, 2.0 ** -23 * ((ref + 3).abs() + ref.abs() + 3) + (M + 8) * UNIT[mode] * size, "dw added to")
        check(db2, bref - 2, 2.0 ** -23 * ((bref - 2).abs() + bref.abs() + 2) + (M + 8) * UNIT[mode] * bsize, "db added to")


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_wide_products(env, mode):
    """Sizes at which every kernel of the products has many tiles, long sums and ragged ends."""
    hpf, torch, ops = env
    for M, K, N in ((4096, 1536, 2048), (4097, 1001, 1999)) if mode == "bf16" else ((700, 600, 650),):
        print(f"\n[case] wide {M}x{K}x{N} {mode}", flush=True)
        d = make(torch, mode, M, K, N, seed=2)
        weights = ops[mode].linear_weights(d["w"])
        y, slope = ops[mode].linear_forward(d["x"], weights, d["bias"], d["residual"], "silu", slope=True)
        z, err = z64(torch, mode, d["x"], d["w"], d["bias"])
        check_forward(torch, mode, "silu", y, slope, z, err, d["residual"])
        dx, dw, db = ops[mode].linear_backward(d["dy"], d["x"], weights, slope)
        t = tdtype(torch, mode)
        dz, x, w = (d["dy"].double() * slope.double()).to(t).double(), d["x"].double(), d["w"].to(t).double()
        ref = dz @ w.t()
        check(dx, ref, HALF[mode] * 1.01 * ref.abs() + (N + 8) * UNIT[mode] * (dz.abs() @ w.t().abs()), "dx")
        check(dw, x.t() @ dz, 2.0 ** -23 * (x.t() @ dz).abs() + (M + 8) * UNIT[mode] * (x.t().abs() @ dz.abs()), "dw")
        check(db, dz.sum(0), 2.0 ** -23 * dz.sum(0).abs() + (M + 8) * UNIT[mode] * dz.abs().sum(0), "db")


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 64, 40), (9, 40, 24), (130, 200, 136), (300, 520, 264)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("left,right", [(0, 3), (1, 0), (2, 5), (8, 8)])
def test_views_give_what_dense_tensors_give(env, mode, shape, left, right):
    """Rows with a stride, at addresses that are aligned to an element only; what lies between the rows is neither used nor touched."""
    hpf, torch, ops = env
    M, K, N = shape
    print(f"\n[case] views {shape} {mode} {left} {right}", flush=True)
    d = make(torch, mode, M, K, N, seed=3)
    weights = ops[mode].linear_weights(d["w"])

    def view(a):
        wide = torch.full((M, left + a.shape[1] + right), float("nan"), device="cuda", dtype=a.dtype)
        v = wide[:, left:left + a.shape[1]]
        v.copy_(a)
        return v, wide
    x, residual, dy = view(d["x"])[0], view(d["residual"])[0], view(d["dy"])[0]
    out, wide = view(torch.zeros_like(d["residual"]))
    y, slope = ops[mode].linear_forward(d["x"], weights, d["bias"], d["residual"], "gelu", slope=True)
    y2, slope2 = ops[mode].linear_forward(x, weights, d["bias"], residual, "gelu", slope=True, out=out)
    assert y2 is out and torch.equal(y, out) and torch.equal(slope, slope2)
    assert bool(wide[:, :left].isnan().all()) and bool(wide[:, left + N:].isnan().all())
    # residual and output in one place
    inplace = d["residual"].clone()
    assert torch.equal(y, ops[mode].linear_forward(x, weights, d["bias"], inplace, "gelu", out=inplace))
    a, b = ops[mode].linear_backward(d["dy"], d["x"], weights, slope), ops[mode].linear_backward(dy, x, weights, slope)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    a, b = ops[mode].linear_backward(d["dy"], d["x"], weights), ops[mode].linear_backward(dy, x, weights)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_transposed_and_overlapping_views_are_refused(env, mode):
    hpf, torch, ops = env
    d = make(torch, mode, 32, 32, 32)
    weights = ops[mode].linear_weights(d["w"])
    with pytest.raises(ValueError, match="strides"):
        ops[mode].linear_forward(d["x"].t(), weights)
    with pytest.raises(ValueError, match="strides"):
        ops[mode].linear_forward(d["x"][:1].expand(32, 32), weights)
    with pytest.raises(hpf.HpfError, match="overlaps"):
        ops[mode].linear_forward(d["x"], weights, out=d["x"])
    with pytest.raises(ValueError, match="columns"):
        ops[mode].linear_forward(d["x"][:, :31], weights)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_no_rows(env, mode):
    hpf, torch, ops = env
    d = make(torch, mode, 4, 24, 40)
    weights = ops[mode].linear_weights(d["w"])
    y, slope = ops[mode].linear_forward(d["x"][:0], weights, d["bias"], None, "relu", slope=True)
    assert y.shape == (0, 40) and slope.shape == (0, 40)
    dx, dw, db = ops[mode].linear_backward(d["dy"][:0], d["x"][:0], weights)
    assert dx.shape == (0, 24) and not bool(dw.any()) and not bool(db.any())
    dw.fill_(2.0), db.fill_(3.0)
    ops[mode].linear_backward(d["dy"][:0], d["x"][:0], weights, dw=dw, db=db, accumulate=True)
    assert bool((dw == 2).all()) and bool((db == 3).all())


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(3, 40, 24), (130, 100, 70), (300, 520, 264)], ids=lambda s: "x".join(map(str, s)))
def test_infinities_and_nan_stay_in_their_rows(env, mode, shape):
    """A row of x with NaN or infinities makes that row of y NaN or infinite and no other; tails are not padded with neighbours."""
    hpf, torch, ops = env
    M, K, N = shape
    d = make(torch, mode, M, K, N, seed=4)
    weights = ops[mode].linear_weights(d["w"])
    for act in ACTS:
        clean = ops[mode].linear_forward(d["x"], weights, d["bias"], None, act)
        x = d["x"].clone()
        x[1, K - 1] = float("nan")
        x[2, 0] = float("inf")
        y = ops[mode].linear_forward(x, weights, d["bias"], None, act)
        assert bool(y[1].isnan().all())
        if act == "none":
            assert bool(y[2].isinf().all())
        keep = torch.ones(M, dtype=torch.bool, device="cuda")
        keep[1:3] = False
        assert torch.equal(y[keep], clean[keep])


def test_gradient_against_differences(env):
    """Directional differences of the definition in 64 bits: error h^2 times third derivatives, here below 1e-6 of the value's scale."""
    hpf, torch, ops = env
    M, K, N = 37, 50, 41
    d = make(torch, "f32", M, K, N, seed=5)
    weights = ops["f32"].linear_weights(d["w"])
    for act in ("gelu", "silu", "none"):
        y, slope = ops["f32"].linear_forward(d["x"], weights, d["bias"], d["residual"], act, slope=True)
        dx, dw, db = ops["f32"].linear_backward(d["dy"], d["x"], weights, slope)

        def value(x, w, b):
            return float((act64(torch, act, x @ w + b)[0] * d["dy"].double()).sum())
        x, w, b = d["x"].double(), d["w"].double(), d["bias"].double()
        g = torch.Generator(device="cuda").manual_seed(9)
        h = 1e-4
        for which, grad in (("x", dx), ("w", dw), ("b", db)):
            v = torch.randn(grad.shape, device="cuda", generator=g, dtype=torch.float64)
            args = {"x": x, "w": w, "b": b}
            up, down = dict(args), dict(args)
            up[which], down[which] = args[which] + h * v, args[which] - h * v
            diff = (value(**up) - value(**down)) / (2 * h)
            mine = float((grad.double() * v).sum())
            scale = float((grad.double() * v).norm()) + 1e-6
            # fp32 results: half a step each, adding up like a random walk at most; differences: h^2 and 64-bit noise / h
            assert abs(diff - mine) <= 2e-6 * scale * math.sqrt(v.numel()), (act, which, diff, mine)


@pytest.mark.parametrize("shape", [(1, 512, 4096), (130, 200, 136), (600, 1000, 300)], ids=lambda s: "x".join(map(str, s)))
def test_streams_and_graphs(env, shape):
    """Two streams at once, and a captured forward and backward replayed on new inputs with eager calls in between."""
    hpf, torch, ops = env
    M, K, N = shape
    o = ops["bf16"]
    d, d2 = make(torch, "bf16", M, K, N, seed=6), make(torch, "bf16", M, K, N, seed=7)
    weights = o.linear_weights(d["w"])

    def both(x, dy, residual):
        y, slope = o.linear_forward(x, weights, d["bias"], residual, "gelu", slope=True)
        return (y, slope) + tuple(o.linear_backward(dy, x, weights, slope))
    want = [both(e["x"], e["dy"], e["residual"]) for e in (d, d2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for i, e in enumerate((d, d2)):
            with torch.cuda.stream(streams[i]):
                got[i] = both(e["x"], e["dy"], e["residual"])
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(p, q) for p, q in zip(got[i], want[i]))
    x, dy, residual = d["x"].clone(), d["dy"].clone(), d["residual"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        both(x, dy, residual)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=streams[0]):
        out = both(x, dy, residual)
    for i in (0, 1, 0, 1):
        e = (d, d2)[i]
        x.copy_(e["x"]), dy.copy_(e["dy"]), residual.copy_(e["residual"])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[i]))
        assert all(torch.equal(p, q) for p, q in zip(both(e["x"], e["dy"], e["residual"]), want[i]))


def test_new_weights_in_place(env):
    hpf, torch, ops = env
    for mode in HALF:
        d, d2 = make(torch, mode, 20, 100, 70, seed=8), make(torch, mode, 20, 100, 70, seed=9)
        weights = ops[mode].linear_weights(d["w"])
        assert ops[mode].linear_weights(d2["w"], out=weights) is weights
        assert torch.equal(ops[mode].linear_forward(d["x"], weights), ops[mode].linear_forward(d["x"], ops[mode].linear_weights(d2["w"])))
        with pytest.raises(ValueError):
            ops[mode].linear_weights(d["w"][:, :69].contiguous(), out=weights)


@pytest.mark.parametrize("shape", [(4100, 640, 2600), (4097, 40, 2570), (4096, 128, 2560), (4096, 192, 2568), (700, 2600, 4104), (705, 2605, 4099), (40, 2600, 4104),
                                   (130, 2560, 4096), (192, 2568, 4096), (2050, 40, 2050), (2048, 130, 2056)], ids=lambda s: "x".join(map(str, s)))
def test_large_tiles_and_short_sums(env, shape):
    """Forward or dw on the largest tiles, with one, two, three and more steps of the contraction, whole and ending within one."""
    test_forward_every_activation(env, "bf16", shape)
    test_backward(env, "bf16", shape)


@pytest.mark.parametrize("M,K,N", [(1, 4096, 8200), (4, 1024, 17000), (16, 1000, 20011), (16, 600, 16384), (2, 9000, 4096), (16, 20000, 520), (1, 3, 70001)])
def test_few_rows_of_wide_weights(env, M, K, N):
    test_forward_every_activation(env, "bf16", (M, K, N))
    test_backward(env, "bf16", (M, K, N))


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_row_strides_beyond_a_tiles_offsets(env, mode):
    """256 rows, 2^22 + 8 elements apart, are more than 32 bits of bytes from end to end."""
    hpf, torch, ops = env
    M, K, N, ld = 260, 24, 40, (1 << 22) + 8
    d = make(torch, mode, M, K, N, seed=5)
    weights = ops[mode].linear_weights(d["w"])
    wide = torch.empty(M, ld, device="cuda", dtype=tdtype(torch, mode))
    x, dy, out = wide[:, :K], wide[:, K:K + N], wide[:, 128:128 + N]
    x.copy_(d["x"])
    dy.copy_(d["dy"])
    y = ops[mode].linear_forward(d["x"], weights, d["bias"], d["dy"], "relu")
    assert torch.equal(y, ops[mode].linear_forward(x, weights, d["bias"], dy, "relu", out=out))
    a, b = ops[mode].linear_backward(d["dy"], d["x"], weights), ops[mode].linear_backward(dy, x, weights)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_columns_of_one_matrix(env, mode):
    """Input, residual and output side by side in one buffer do not overlap; nothing else in it changes."""
    hpf, torch, ops = env
    M, K, N = 70, 33, 20
    d = make(torch, mode, M, K, N, seed=6)
    weights = ops[mode].linear_weights(d["w"])
    wide = torch.full((M, 101), 7.0, device="cuda", dtype=tdtype(torch, mode))
    x, residual, out = wide[:, 1:1 + K], wide[:, 1 + K:1 + K + N], wide[:, 60:60 + N]
    x.copy_(d["x"])
    residual.copy_(d["residual"])
    before = wide.clone()
    y = ops[mode].linear_forward(d["x"], weights, None, d["residual"], "silu")
    assert torch.equal(y, ops[mode].linear_forward(x, weights, None, residual, "silu", out=out))
    before[:, 60:60 + N] = y
    assert torch.equal(wide, before)
    for cols in (slice(K, K + N), slice(0, N), slice(1 + K - N, 1 + K)):       # these share a column with x
        with pytest.raises(hpf.HpfError):
            ops[mode].linear_forward(x, weights, out=wide[:, cols])
    logits, d_wide = wide[:, :40], wide[:, 40:80]
    labels = torch.randint(0, 40, (M,), device="cuda", dtype=torch.int32)
    logits.normal_()
    r = ops[mode].logprob_forward(logits, labels)
    one = torch.ones(M, device="cuda")
    want = ops[mode].logprob_backward(logits.contiguous(), labels, r.stats, one)
    assert torch.equal(want, ops[mode].logprob_backward(logits, labels, r.stats, one, out=d_wide))
    with pytest.raises(hpf.HpfError):
        ops[mode].logprob_backward(logits, labels, r.stats, one, out=wide[:, 39:79])


@pytest.mark.parametrize("shape", [(4100, 264, 2600), (300, 2560, 4104), (16, 1000, 30000)], ids=lambda s: "x".join(map(str, s)))
def test_streams_and_graphs_on_the_largest_tiles(env, shape):
    test_streams_and_graphs(env, shape)


@pytest.mark.parametrize("shape", [(1 << 21, 3, 2), (1 << 21, 64, 8), (1, 1 << 20, 4), (17, 1 << 20, 8), (2, 5, 1 << 20), (33, 8, 1 << 20)], ids=lambda s: "x".join(map(str, s)))
def test_largest_sizes(env, shape):
    test_forward_every_activation(env, "bf16", shape)
    test_backward(env, "bf16", shape)
