"""GPU tests at the edges of the operators at the answer end of a model: workspaces of exactly the size asked for, with a guard behind them.

Tolerances: a sum of n products in fp32 is off by at most n 2^-24 sum |a_i b_i|, a result in bf16 is rounded once by half a step, 2^-8 of it."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    from paper_1911_05146_amd import hpf
    return hpf, torch


def randn(torch, seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def check(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off"


class Guarded:
    """A workspace of exactly `need` bytes, filled with NaN, and 64 KiB behind it that nobody may touch."""

    def __init__(self, torch, need):
        self.need = need
        self.raw = torch.full((need + 65536 + 256,), 0xff, device="cuda", dtype=torch.uint8)
        self.at = -self.raw.data_ptr() % 256
        self.ptr = self.raw.data_ptr() + self.at
        self.raw[self.at + need:] = 0xa5

    def check(self):
        assert bool((self.raw[self.at + self.need:] == 0xa5).all()), "written behind the workspace"


# up to 16 rows and long contractions, where the number of shares depends on how the contraction is counted; then every other cut
FEW = [(16, 89760, 40), (16, 89760, 48), (1, 53856, 65), (5, 53856, 65), (1, 89736, 40), (3, 40, 48)]
CUTS = FEW + [(16, 4096, 4096), (1, 40, 89760), (16, 40, 89760), (128, 4096, 512), (40, 2600, 4104), (130, 2565, 999), (2560, 512, 4096), (1021, 257, 1000)]


@pytest.mark.parametrize("M,K,N", CUTS)
def test_products_stay_within_a_workspace_of_the_size_asked_for(env, M, K, N):
    hpf, torch = env
    print(f"\n[case] workspace {M}x{K}x{N}", flush=True)
    bf16 = torch.bfloat16
    x, w, dy = randn(torch, 1, M, K).to(bf16), randn(torch, 2, K, N) * K ** -0.5, randn(torch, 3, M, N).to(bf16)
    slope = randn(torch, 4, M, N).to(bf16)
    weights = hpf.Ops(hpf.HPF_BF16).linear_weights(w)
    seen = w.to(bf16).double()
    need = hpf.hpf_op_linear_workspace_bytes(hpf.HPF_BF16, M, K, N)
    stream = torch.cuda.current_stream().cuda_stream
    # rows in place, and rows that are copied because they start off 16 bytes
    wide = torch.empty(M, K + 1, device="cuda", dtype=bf16)
    wide[:, 1:] = x
    sums = []
    for a, lda in ((x, K), (wide[:, 1:], K + 1)):
        ws = Guarded(torch, need)
        y = torch.empty(M, N, device="cuda", dtype=bf16)
        hpf.hpf_op_linear_forward(hpf.HPF_BF16, a.data_ptr(), lda, weights.ptr, 0, 0, 0, y.data_ptr(), N, 0, M, K, N, hpf.HPF_ACT_NONE, ws.ptr, need, stream)
        torch.cuda.synchronize()
        ws.check()
        ref = x.double() @ seen
        check(y, ref, 2.0 ** -8 * 1.01 * ref.abs() + (K + 8) * 2.0 ** -24 * (x.double().abs() @ seen.abs()), "y")
        sums.append(y)
    assert torch.equal(*sums), "the copy of the rows gives other bits"
    for sl in (None, slope):
        dz = dy.double() if sl is None else (dy.double() * sl.double()).to(bf16).double()
        ws = Guarded(torch, need)
        dx, dw, db = torch.empty(M, K, device="cuda", dtype=bf16), torch.empty(K, N, device="cuda"), torch.empty(N, device="cuda")
        hpf.hpf_op_linear_backward(hpf.HPF_BF16, dy.data_ptr(), N, x.data_ptr(), K, weights.ptr, 0 if sl is None else sl.data_ptr(), dx.data_ptr(), K, dw.data_ptr(),
                                   db.data_ptr(), 0, M, K, N, ws.ptr, need, stream)
        torch.cuda.synchronize()
        ws.check()
        ref = dz @ seen.t()
        check(dx, ref, 2.0 ** -8 * 1.01 * ref.abs() + (N + 8) * 2.0 ** -24 * (dz.abs() @ seen.t().abs()) + 1e-38, "dx")
        ref, size = x.double().t() @ dz, x.double().t().abs() @ dz.abs()
        check(dw, ref, 2.0 ** -24 * 1.01 * ref.abs() + (M + 8) * 2.0 ** -24 * size + 1e-38, "dw")
        check(db, dz.sum(0), 2.0 ** -24 * 1.01 * dz.sum(0).abs() + (M + 8) * 2.0 ** -24 * dz.abs().sum(0) + 1e-38, "db")


# every kernel of the distillation: a wave per row, few and many rows of 256 threads, rows with a second launch, long rows, divided rows
DISTILL = [(12, 100), (1100, 300), (12, 1500), (1100, 2100), (140, 20000), (260, 131072), (2, 40000)]


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", DISTILL, ids=lambda s: "x".join(map(str, s)))
def test_entries_of_very_small_teacher_probability(env, mode, shape):
    """A listed class whose teacher probability is a number below 2^-1022, or none at all, gets the student's probability as its gradient."""
    from test_gpu_logits import check_distill, distill64
    hpf, torch = env
    rows, classes = shape
    print(f"\n[case] small probabilities {shape} {mode}", flush=True)
    o = hpf.Ops(hpf.HPF_BF16 if mode == "bf16" else hpf.HPF_F32)
    s = randn(torch, 5, rows, classes).to(o.tdtype)
    index = torch.arange(10, device="cuda", dtype=torch.int32).repeat(rows, 1)
    index[1::4, 9] = 8                                  # a class listed twice, each time all but impossible
    labels = (torch.arange(rows, device="cuda") % 12 - 1).int()
    for T in (1.0, 0.05, 2.0, 3.0):
        gaps = torch.tensor([0.0, 1.0, 690.0, 708.0, 715.0, 720.0, 735.0, 744.0, 744.5, 800.0], device="cuda") * T
        logit = (5.0 - gaps).repeat(rows, 1).contiguous()
        for hw in (0.0, 0.5, 1.0):
            loss, ds = o.distill(s, index, logit, labels, temperature=T, hard_weight=hw)
            assert bool(loss.isfinite().all()) and bool(ds.isfinite().all()), (T, hw)
            check_distill(torch, mode, s, index, logit, labels, T, hw, None, loss, ds)
            if hw == 0.0:
                at = ds.double().gather(1, index.long()[:, 2:])
                q = torch.softmax(s.double() / float(torch.tensor(T)), 1).gather(1, index.long()[:, 2:]) * float(torch.tensor(T))
                # relative to the value, and 2^-126 where it is less than that: there the types have no full set of digits (at T = 0.05 some are 1e-39)
                check(at, q, (2.0 ** -7 if mode == "bf16" else 1e-4) * q + 2.0 ** -126, "the student's probability")
    # a list that has no say (hard_weight 1) leaves loss and gradient those of the label
    logit[0, 3], logit[rows - 1, 0] = float("nan"), float("inf")
    loss, ds = o.distill(s, index, logit, labels, temperature=2.0, hard_weight=1.0)
    want = o.distill(s, None, None, labels, temperature=2.0, hard_weight=1.0)
    assert torch.equal(loss, want[0])
    ref, dref, _ = distill64(torch, s, torch.full_like(index, -1), torch.zeros_like(logit), labels, 2.0, 1.0, None)
    check_distill(torch, mode, s, torch.full_like(index, -1), torch.zeros_like(logit), labels, 2.0, 1.0, None, loss, ds)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(3, 40, 24), (130, 200, 136), (1021, 257, 1000), (2304, 512, 4096), (700, 2600, 4104)])
def test_weight_gradients_in_a_flat_buffer(env, mode, M, K, N):
    """dw and db at any fp32 address of one buffer of gradients, written and added to; the numbers around them stay."""
    hpf, torch = env
    print(f"\n[case] flat gradients {M}x{K}x{N} {mode}", flush=True)
    o = hpf.Ops(hpf.HPF_BF16 if mode == "bf16" else hpf.HPF_F32)
    x, w, dy = randn(torch, 1, M, K).to(o.tdtype), randn(torch, 2, K, N), randn(torch, 3, M, N).to(o.tdtype)
    weights = o.linear_weights(w)
    _, dw, db = o.linear_backward(dy, x, weights)
    for off in (0, 1, 2, 3):
        flat = torch.full((off + K * N + N + 8,), 7.0, device="cuda")
        vw, vb = flat[off:off + K * N].view(K, N), flat[off + K * N:off + K * N + N]
        o.linear_backward(dy, x, weights, dw=vw, db=vb)
        assert torch.equal(vw, dw) and torch.equal(vb, db)
        assert bool((flat[:off] == 7).all()) and bool((flat[off + K * N + N:] == 7).all())
        before = vw.clone()
        o.linear_backward(dy, x, weights, dw=vw, db=vb, accumulate=True)
        # one sum more, rounded once: 2^-24 of it (check mode: from double)
        check(vw, before.double() + dw.double(), 2.0 ** -23 * before.double().abs() * 2, "dw added to")
        assert bool((flat[:off] == 7).all()) and bool((flat[off + K * N + N:] == 7).all())


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("at", [0, 3, 8])
def test_gradients_of_a_few_columns_take_no_more_than_they_hold(env, mode, at):
    """The gradient of logits that are a part of a much wider matrix has rows of its own, which start where the logits' do within 128 bytes."""
    hpf, torch = env
    o = hpf.Ops(hpf.HPF_BF16 if mode == "bf16" else hpf.HPF_F32)
    rows, classes = 40, 1000
    for width in (1 << 16, 1003, 1008, (1 << 15) + 3):
        wide = randn(torch, 6, rows, width + 16).to(o.tdtype)[:, :width]
        s = wide[:, at:at + classes] if at + classes <= width else wide[:, :classes]
        labels = (torch.arange(rows, device="cuda") * 37 % classes).int()
        r = o.logprob_forward(s, labels, 5)
        one = torch.ones(rows, device="cuda")
        d = o.logprob_backward(s, labels, r.stats, one)
        loss, ds = o.distill(s, r.top_index, r.top_logprob, labels, hard_weight=0.5)
        most = rows * (classes * s.element_size() + 128)
        for g, want in ((d, o.logprob_backward(s.contiguous(), labels, r.stats, one)), (ds, None)):
            held = g.untyped_storage().nbytes()
            assert g.shape == s.shape and held <= most
            phase = 128 // s.element_size()
            assert g.stride(0) % phase == s.stride(0) % phase
            if want is not None:
                assert torch.equal(g, want)
        dense = o.distill(s.contiguous(), r.top_index, r.top_logprob, labels, hard_weight=0.5)
        assert bool(((loss - dense[0]).abs() <= 1e-6 * (1 + loss.abs())).all()) and bool(((ds.double() - dense[1].double()).abs() <= 2.0 ** -7 * ds.double().abs() + 1e-7).all())


@pytest.mark.parametrize("M", [1, 20, 300])
def test_tail_of_gelu(env, M):
    """gelu(z) far below zero keeps the digits of its type: relative to its value, which falls to 2^-126 at -13.  The kernel's Phi(-|z|) is off by at
    most 2^-12 of itself (the largest deviation of its polynomial), exp2 of z^2 / 2 by z^2 2^-23 <= 2^-15: together below 2^-11."""
    hpf, torch = env
    print(f"\n[case] gelu tail {M}", flush=True)
    o = hpf.Ops(hpf.HPF_BF16)
    z = torch.linspace(-13, 13, 4096, device="cuda").to(torch.bfloat16).float()
    x = torch.ones(M, 1, device="cuda", dtype=torch.bfloat16)
    y, slope = o.linear_forward(x, o.linear_weights(z[None].contiguous()), activation="gelu", slope=True)
    z = z.double()
    def below(v):                                        # torch.special.ndtr ends where 1 + erf rounds to 0, at -8.3
        return 0.5 * torch.special.erfc(-v * 0.5 ** 0.5)
    phi, density = below(z), torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    off = 2.0 ** -11 * below(-z.abs()) + torch.where(z > 0, 2.0 ** -22, 0.0)
    ref, sref = z * phi, phi + z * density
    check(y, ref.expand(M, -1), 2.0 ** -8 * 1.01 * ref.abs() + z.abs() * off + 2.0 ** -126, "y")
    check(slope, sref.expand(M, -1), 2.0 ** -8 * 1.01 * sref.abs() + off + 2.0 ** -14 * z.abs() * density + 2.0 ** -126, "slope")


@pytest.mark.parametrize("shape", [(6, 1000), (1100, 2052), (200, 20001), (140, 65537), (2, 70001)], ids=lambda s: "x".join(map(str, s)))
def test_lists_of_logits_far_from_zero(env, shape):
    """A common offset that leaves the logits a few hundred or thousand steps of fp32 apart: many distinct values within what a coarse bound tells
    apart, and many equal ones."""
    from test_gpu_logits import check_forward
    hpf, torch = env
    print(f"\n[case] far from zero {shape}", flush=True)
    o = hpf.Ops(hpf.HPF_F32)
    rows, classes = shape
    labels = (torch.arange(rows, device="cuda") * 7919 % classes).int()
    for offset in (1e4, -1e5):
        s = randn(torch, 7, rows, classes) * 2.5 + offset
        for top in (5, 64):
            check_forward(torch, s, labels, top, o.logprob_forward(s, labels, top))
