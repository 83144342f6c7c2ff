"""No-GPU checks of what the operators at the answer end of a model refuse before any device work: arrays that are off their elements (the
addresses here are never used)."""
import pytest

from test_answer_refusals import A, B, D, E, F, backward, forward, refused

G, H = 6 << 40, 7 << 40


@pytest.fixture(scope="module")
def hpf():
    from paper_1911_05146_amd import hpf as h
    return h


def logprob(hpf, s=A, ld=10, labels=B, logprob=D, entropy=D + 4096, rank=E, stats=E + 4096, ti=F, tl=F + 4096, top=3, rows=4, classes=10, ws=G, dtype=1):
    hpf.hpf_op_logprob_forward(dtype, s, ld, labels, logprob, entropy, rank, stats, ti, tl, top, rows, classes, ws, 1 << 30)


def logprob_gradient(hpf, s=A, labels=B, stats=D, gl=E, h=F, gh=F + 4096, d=G, rows=4, classes=10, dtype=1, ld=0):
    hpf.hpf_op_logprob_backward(dtype, s, ld or classes, labels, stats, gl, h, gh, d, ld or classes, rows, classes)


def distill(hpf, s=A, ti=B, tl=D, top=3, labels=E, w=E + 4096, loss=F, d=G, rows=4, classes=10, ws=H, dtype=1):
    hpf.hpf_op_distill(dtype, s, classes, ti, tl, top, labels, 1.0, 0.5, w, loss, d, classes, rows, classes, ws, 1 << 30)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_arrays_off_their_elements(hpf, off):
    def no(f, **kw):
        refused(hpf, hpf.HPF_EINVAL, "aligned", lambda: f(hpf, **kw))
    no(forward, bias=F + off)
    no(forward, dtype=hpf.HPF_F32, w=B + off)
    no(backward, dw=F + off)
    no(backward, db=(7 << 40) + off)
    no(backward, dw=F + off, M=0)
    no(backward, dtype=hpf.HPF_F32, w=D + off)
    refused(hpf, hpf.HPF_EINVAL, "aligned", hpf.hpf_op_linear_pack, A + off, 16, 8, B, 1 << 20)
    for name, at in (("labels", B), ("logprob", D), ("entropy", D), ("rank", E), ("stats", E), ("ti", F), ("tl", F)):
        no(logprob, **{name: at + off})
    for name, at in (("labels", B), ("stats", D), ("gl", E), ("h", F), ("gh", F)):
        no(logprob_gradient, **{name: at + off})
    for name, at in (("ti", B), ("tl", D), ("labels", E), ("w", E), ("loss", F)):
        no(distill, **{name: at + off})


def test_outputs_that_overlap_another_tensor(hpf):
    def no(f, **kw):
        refused(hpf, hpf.HPF_EINVAL, "overlap", lambda: f(hpf, **kw))
    last = 4 * (8 - 1)                                   # of a bias of 8: y or slope from its last element on
    no(forward, bias=D)
    no(forward, bias=F, y=F + last)
    no(forward, bias=F, slope=F + last)
    no(forward, dtype=hpf.HPF_F32, w=B, y=B + 16 * 8 * 4 - 4)
    row, pair, entry = 4 * 4, 2 * 4 * 4, 3 * 4 * 4       # bytes of four rows' numbers, pairs, lists of 3
    out = {"logprob": (D, row), "entropy": (D + 4096, row), "rank": (E, row), "stats": (E + 4096, pair), "ti": (F, entry), "tl": (F + 4096, entry)}
    logits = 2 * (3 * 10 + 10)
    for name, (at, size) in out.items():
        no(logprob, **{name: A + logits - 4})            # the logits' last element
        no(logprob, **{name: A - size + 4})              # their first one
        no(logprob, **{name: B})                         # the labels
        for other, (place, _) in out.items():
            if other != name:
                no(logprob, **{name: place - size + 4})
    for name, size in (("labels", row), ("stats", pair), ("gl", row), ("h", row), ("gh", row)):
        no(logprob_gradient, **{name: G + logits - 4})
        no(logprob_gradient, **{name: G - size + 4})
    for name, size in (("ti", entry), ("tl", entry), ("labels", row), ("w", row)):
        no(distill, **{name: F})
        no(distill, **{name: G + logits - 4})
        no(distill, **{name: G - size + 4})
    no(distill, loss=A + logits - 4)
    no(distill, loss=G)
    no(distill, d=A)


def test_workspaces_that_overlap_a_tensor(hpf):
    def no(f, **kw):
        refused(hpf, hpf.HPF_EINVAL, "overlap", lambda: f(hpf, **kw))
    need = hpf.hpf_op_linear_workspace_bytes(hpf.HPF_BF16, 4, 16, 8)
    assert need >= 256
    for ws in (A, B, D, 8 << 40, 9 << 40, 10 << 40):      # x, weights, y; bias, residual and slope
        for at in (ws, ws + 256 - need):
            no(forward, ws=at, bias=8 << 40, r=9 << 40, ldr=8, slope=10 << 40)
    for ws in (A, B, D, E, F, 8 << 40, 9 << 40):          # dy, x, weights, dx, dw; slope and db
        no(backward, ws=ws, slope=8 << 40, db=9 << 40)
    rows, classes = 4, 1 << 18                            # divided rows
    assert hpf.hpf_op_logits_workspace_bytes(hpf.HPF_BF16, rows, classes, 3)
    for ws in (A, B, D, D + 4096, E, E + 4096, F, F + 4096):
        no(logprob, ws=ws, rows=rows, classes=classes, ld=classes)
    for ws in (A, B, D, E, E + 4096, F, G):
        no(distill, ws=ws, rows=rows, classes=classes)


def test_what_lies_apart_is_not_refused(hpf):
    """Everything side by side in one piece of memory: the call gets as far as its workspace, which is too small."""
    x, at = A, [A]

    def place(n):
        at[0] += n
        return at[0] - n
    x, bias, y, slope, r = place(2 * 4 * 16), place(4 * 8), place(2 * 4 * 8), place(2 * 4 * 8), place(2 * 4 * 8)
    refused(hpf, hpf.HPF_ENOMEM, "workspace", lambda: forward(hpf, x=x, bias=bias, y=y, slope=slope, r=r, ldr=8, n=1))
    refused(hpf, hpf.HPF_ENOMEM, "workspace", lambda: forward(hpf, x=x, bias=bias, y=y, slope=slope, r=y, ldr=8, n=1))
    n = 1 << 18
    s, d, labels = place(2 * 4 * n), place(2 * 4 * n), place(16)
    a, b, c, e, ti, tl = place(16), place(16), place(16), place(32), place(48), place(48)
    refused(hpf, hpf.HPF_ENOMEM, "workspace", hpf.hpf_op_logprob_forward, 1, s, n, labels, a, b, c, e, ti, tl, 3, 4, n, H, 1)
    refused(hpf, hpf.HPF_ENOMEM, "workspace", hpf.hpf_op_distill, 1, s, n, ti, tl, 3, labels, 1.0, 0.5, a, b, d, n, 4, n, H, 1)


def test_weights_of_another_device_or_size(hpf):
    """New weights go into an object of the same device (here the CPU stands in for one, whose memory is never touched); sizes beyond the limits are
    said to be that."""
    import torch
    for dtype in (hpf.HPF_BF16, hpf.HPF_F32):
        o = hpf.Ops(dtype, "cpu")
        elsewhere = hpf.LinearWeights(16, 8, dtype, torch.zeros(16, 8, device="meta"), B)
        with pytest.raises(ValueError, match="another shape, type or device"):
            o.linear_weights(torch.zeros(16, 8), out=elsewhere)
    refused(hpf, hpf.HPF_EUNSUPPORTED, "2^32", hpf.hpf_op_linear_pack, A, 1 << 20, 1 << 13, 0, 0)
    refused(hpf, hpf.HPF_EUNSUPPORTED, "2^20", hpf.hpf_op_linear_pack, A, (1 << 20) + 1, 8, 0, 0)


def test_gradients_beyond_a_launch(hpf):
    """2^24 work-groups of 256 threads and more are no launch: fp32 logits whose rows have 2^24 pieces of 4096 in all."""
    for rows, classes in ((1 << 21, 1 << 15), (1 << 21, 7 * 4096 - 2), (256, 1 << 28), (1 << 12, 1 << 24)):
        refused(hpf, hpf.HPF_EUNSUPPORTED, "2^24", lambda: logprob_gradient(hpf, rows=rows, classes=classes, dtype=hpf.HPF_F32))
    for rows, classes, dtype in ((1 << 21, 7 * 4096 - 4, hpf.HPF_F32), (1 << 21, 1 << 15, hpf.HPF_BF16), (256, 1 << 28, hpf.HPF_BF16)):
        refused(hpf, hpf.HPF_EINVAL, "stats", lambda: logprob_gradient(hpf, rows=rows, classes=classes, dtype=dtype, stats=0))     # refused for another reason
