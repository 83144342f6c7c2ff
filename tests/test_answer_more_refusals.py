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
