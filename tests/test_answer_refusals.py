"""No-GPU checks of the operators at the answer end of a model: sizes, and what the entry points refuse before any device work (the
addresses here are never used)."""
import pytest

A, B, D, E, F = (i << 40 for i in range(1, 6))       # addresses far apart


@pytest.fixture(scope="module")
def hpf():
    from paper_1911_05146_amd import hpf as h
    return h


def refused(hpf, status, text, f, *args):
    with pytest.raises(hpf.HpfError) as e:
        f(*args)
    assert e.value.status == status and text in str(e.value), str(e.value)


def test_sizes(hpf):
    assert hpf.hpf_op_linear_packed_bytes(1, 1) == 2 * (64 + 64)
    assert hpf.hpf_op_linear_packed_bytes(100, 65) == 2 * (65 * 128 + 100 * 128)
    for bad in ((0, 1), (1, 0), (-4, 8), (1 << 21, 4), (4, 1 << 21)):
        assert hpf.hpf_op_linear_packed_bytes(*bad) == 0
        assert hpf.hpf_op_linear_workspace_bytes(hpf.HPF_BF16, 4, *bad) == 0
    assert hpf.hpf_op_linear_workspace_bytes(7, 4, 4, 4) == 0 and hpf.hpf_op_linear_workspace_bytes(hpf.HPF_F32, 0, 4, 4) == 0
    for bad in ((0, 4, 0), (4, 0, 0), (-1, 4, 0), (4, 4, -1), (4, 4, 65), (4, 1 << 29, 0)):
        assert hpf.hpf_op_logits_workspace_bytes(hpf.HPF_F32, *bad) == 0


def forward(hpf, dtype=None, x=A, ldx=16, w=B, bias=0, r=0, ldr=0, y=D, ldy=8, slope=0, M=4, K=16, N=8, act=0, ws=E, n=1 << 30):
    hpf.hpf_op_linear_forward(hpf.HPF_BF16 if dtype is None else dtype, x, ldx, w, bias, r, ldr, y, ldy, slope, M, K, N, act, ws, n)


def backward(hpf, dtype=None, dy=A, lddy=8, x=B, ldx=16, w=D, slope=0, dx=E, lddx=16, dw=F, db=0, M=4, K=16, N=8, ws=6 << 40, n=1 << 30):
    hpf.hpf_op_linear_backward(hpf.HPF_BF16 if dtype is None else dtype, dy, lddy, x, ldx, w, slope, dx, lddx, dw, db, 0, M, K, N, ws, n)


def test_linear_refusals(hpf):
    EINVAL, ENOMEM, EUN = hpf.HPF_EINVAL, hpf.HPF_ENOMEM, hpf.HPF_EUNSUPPORTED

    def f(status, text, **kw):
        refused(hpf, status, text, lambda: forward(hpf, **kw))

    def b(status, text, **kw):
        refused(hpf, status, text, lambda: backward(hpf, **kw))
    for g in (f, b):
        g(EINVAL, "dtype", dtype=5)
        g(EINVAL, "negative", M=-1)
        g(EINVAL, "positive", K=0)
        g(EINVAL, "positive", N=0)
        g(EUN, "2^20", K=(1 << 20) + 1)
        g(EUN, "2^21", M=(1 << 21) + 1)
        g(EUN, "2^32", M=1 << 21, N=(1 << 11) + 1, **({"ldy": 1 << 12} if g is f else {"lddy": 1 << 12}))
        g(EUN, "2^32", K=1 << 20, N=1 << 13, **({"ldy": 1 << 13} if g is f else {"lddy": 1 << 13}))
        g(EINVAL, "stride", ldx=15)
        g(EINVAL, "aligned", x=A + 1 if g is f else B + 1)
        g(EINVAL, "256-byte", w=(B if g is f else D) + 64)
    f(EINVAL, "activation", act=4)
    f(EINVAL, "activation", act=-1)
    f(EINVAL, "null", x=0)
    f(EINVAL, "null", w=0)
    f(EINVAL, "null", y=0)
    f(EINVAL, "stride", ldy=7)
    f(EINVAL, "stride", r=E, ldr=7)
    f(EINVAL, "aligned", slope=E + 1)
    f(EINVAL, "overlaps", y=A)
    f(EINVAL, "overlaps", y=A + 2 * (3 * 16 + 15))
    f(EINVAL, "overlaps", slope=A)
    f(EINVAL, "overlaps", slope=D)
    f(EINVAL, "overlaps", y=B)
    f(EINVAL, "overlaps", r=D + 2, ldr=8)
    f(EINVAL, "overlaps", r=D, ldr=9)
    b(EINVAL, "null", dy=0)
    b(EINVAL, "null", x=0)
    b(EINVAL, "null", w=0)
    b(EINVAL, "stride", lddy=7)
    b(EINVAL, "stride", lddx=15)
    b(EINVAL, "aligned", slope=6 * (1 << 40) + 1)
    b(EINVAL, "overlaps", dx=A)
    b(EINVAL, "overlaps", dw=D + 256)
    b(EINVAL, "overlap", dw=E)
    b(EINVAL, "overlap", db=F + 16 * 8 * 4 - 4)
    need = hpf.hpf_op_linear_workspace_bytes(hpf.HPF_BF16, 4, 16, 8)
    if need:
        b(EINVAL, "workspace", ws=0)
        b(EINVAL, "256-byte", ws=(6 << 40) + 16)
        b(ENOMEM, "workspace", n=need - 1)
    packed = hpf.hpf_op_linear_packed_bytes(16, 8)
    refused(hpf, EINVAL, "null", hpf.hpf_op_linear_pack, 0, 16, 8, A, packed)
    refused(hpf, EINVAL, "null", hpf.hpf_op_linear_pack, A, 16, 8, 0, packed)
    refused(hpf, EINVAL, "positive", hpf.hpf_op_linear_pack, A, 0, 8, B, packed)
    refused(hpf, EINVAL, "256-byte", hpf.hpf_op_linear_pack, A, 16, 8, B + 128, packed)
    refused(hpf, ENOMEM, "needed", hpf.hpf_op_linear_pack, A, 16, 8, B, packed - 1)
    refused(hpf, EINVAL, "overlap", hpf.hpf_op_linear_pack, A, 16, 8, A, packed)


def test_no_rows_and_nothing_wanted_need_no_tensors(hpf):
    forward(hpf, x=0, w=0, y=0, M=0, ws=0, n=0)
    backward(hpf, dx=0, dw=0, dy=0, x=0, w=0, ws=0, n=0)
    hpf.hpf_op_logprob_forward(hpf.HPF_F32, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 10)
    hpf.hpf_op_logprob_backward(hpf.HPF_F32, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 10)
    hpf.hpf_op_distill(hpf.HPF_F32, 0, 0, 0, 0, 0, 0, 1.0, 0.0, 0, 0, 0, 0, 0, 10)


def test_logits_refusals(hpf):
    EINVAL, EUN = hpf.HPF_EINVAL, hpf.HPF_EUNSUPPORTED

    def f(status, text, dtype=1, s=A, ld=10, labels=B, logprob=D, entropy=0, rank=0, stats=0, ti=0, tl=0, top=0, rows=4, classes=10):
        refused(hpf, status, text, hpf.hpf_op_logprob_forward, dtype, s, ld, labels, logprob, entropy, rank, stats, ti, tl, top, rows, classes, F, 1 << 30)

    def b(status, text, dtype=1, s=A, ld=10, labels=B, stats=D, gl=E, h=0, gh=0, d=F, ldd=10, rows=4, classes=10):
        refused(hpf, status, text, hpf.hpf_op_logprob_backward, dtype, s, ld, labels, stats, gl, h, gh, d, ldd, rows, classes)

    def k(status, text, dtype=1, s=A, ld=10, ti=B, tl=D, top=3, labels=E, T=1.0, hw=0.5, w=0, loss=F, d=6 << 40, ldd=10, rows=4, classes=10):
        refused(hpf, status, text, hpf.hpf_op_distill, dtype, s, ld, ti, tl, top, labels, T, hw, w, loss, d, ldd, rows, classes, 7 << 40, 1 << 30)
    for g in (f, b, k):
        g(EINVAL, "dtype", dtype=2)
        g(EINVAL, "negative", rows=-1)
        g(EINVAL, "positive", classes=0)
        g(EUN, "2^28", classes=(1 << 28) + 1, ld=1 << 30)
        g(EUN, "2^21", rows=(1 << 21) + 1)
        g(EUN, "2^36", rows=1 << 20, classes=1 << 17, ld=1 << 17)
        g(EINVAL, "null", s=0)
        g(EINVAL, "stride", ld=9)
        g(EINVAL, "aligned", s=A + 1)
    for g in (f, k):
        g(EINVAL, "negative", top=-1)
        g(EUN, "at most 64", top=65)
    f(EINVAL, "top_index", top=3, tl=E)
    f(EINVAL, "labels", labels=0)
    f(EINVAL, "labels", labels=0, logprob=0, rank=D)
    b(EINVAL, "stats", stats=0)
    b(EINVAL, "dlogits", d=0)
    b(EINVAL, "labels", labels=0)
    b(EINVAL, "entropy", gh=B)
    b(EINVAL, "stride", ldd=9)
    b(EINVAL, "aligned", d=F + 1)
    b(EINVAL, "overlap", d=A, ldd=11)
    b(EINVAL, "overlap", d=A + 2)
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-5, 1e5):
        k(EINVAL, "temperature", T=T)
    for hw in (-0.1, 1.1, float("nan")):
        k(EINVAL, "hard_weight", hw=hw)
    k(EINVAL, "loss", loss=0)
    k(EINVAL, "top_index", ti=0)
    k(EINVAL, "labels", labels=0)
    k(EINVAL, "stride", ldd=9)
    k(EINVAL, "overlap", d=A)


def test_tensor_checks_of_the_wrapper(hpf):
    """Shapes, types and places are refused before an address is taken (CPU tensors stand in for misplaced ones)."""
    import torch
    o = hpf.Ops(hpf.HPF_BF16)
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    w = hpf.LinearWeights(16, 8, hpf.HPF_BF16, x, 0)
    with pytest.raises(ValueError, match="another type or device"):
        o.linear_forward(x, w)
    with pytest.raises(ValueError, match="on cpu"):
        o.logprob_forward(x)
    with pytest.raises(ValueError, match="float32"):
        o.logprob_forward(x.float())
    with pytest.raises(ValueError, match="w:"):
        o.linear_weights(torch.zeros(4, 4))


def test_columns_that_overlap(hpf):
    """Matrices of one row stride: side by side they do not overlap; a shared column, or one that wraps into the next row, does."""
    def f(y, **kw):
        refused(hpf, hpf.HPF_EINVAL, "overlaps", lambda: forward(hpf, y=y, ldx=40, ldy=40, **kw))
    for at in (0, 15, -7, 40, 2 * 40 + 15, -40 + 39, 33, 33 + 40):          # x: columns 0 to 15 of 40; y: 8 columns from `at`
        f(A + 2 * at)
    f(A + 2 * 17, r=A + 2 * 20, ldr=40)                             # residual within y
    # no overlap: what is refused next is the workspace
    for at in (16, 32, 20 + 40):
        refused(hpf, hpf.HPF_ENOMEM, "workspace", lambda: forward(hpf, y=A + 2 * at, ldx=40, ldy=40, n=1))
