"""GPU parity of the row operators on logits -- log probabilities with rank, entropy and list, their gradient, distillation --
against the definitions in 64 bits: row lengths from one class on, odd ones and views, ties, masked classes, broken rows, streams
and graphs.

Tolerances.  exp(s - m) in fp32 is off by at most (|s - m| + 4) 2^-23 relative, a sum of n such terms by n 2^-24 more, where a thread
adds at most classes / 64 + 64 terms and partial sums one after the other; so the sum of all classes but the largest has a relative
error of at most `rel`, and log Z = log1p(rest) one of at most rel * rest / Z.  Results are rounded by half a step (fp32 2^-24, bf16 2^-8)."""
import math

import pytest

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
INF = math.inf
SHAPES = [(1, 1), (1, 2), (3, 7), (300, 10), (5, 64), (4, 65), (9, 511), (70, 1000), (2, 1001), (3, 2048), (3, 4097), (5, 10000), (600, 1200),
          (2, 32768), (3, 50257), (1, 65537), (1, 131072), (2, 131071), (1, 300001)]


@pytest.fixture(scope="module")
def env():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    from paper_1911_05146_amd import hpf
    return hpf, torch, {m: hpf.Ops(hpf.HPF_BF16 if m == "bf16" else hpf.HPF_F32) for m in HALF}


def make(torch, mode, rows, classes, seed=0, left=0, right=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 13 * rows + classes)
    wide = torch.randn(rows, left + classes + right, device="cuda", generator=g) * 3
    wide[:, left:left + 1] += torch.rand(rows, 1, device="cuda", generator=g) * 14
    s = wide.to(torch.bfloat16 if mode == "bf16" else torch.float32)[:, left:left + classes]
    if classes > 40:
        s[:, 5::17] = -INF
    labels = torch.randint(0, classes, (rows,), device="cuda", generator=g)
    labels = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.5, s.argmax(1), labels).int()
    if rows > 2:
        labels[rows // 2] = -1
    return s, labels, g


class Row64:
    """Softmax of every row in 64 bits, and the bounds."""

    def __init__(self, torch, s, scale=1.0):
        s = s.double()
        self.m = s.amax(1, keepdim=True)
        self.t = (s - self.m) * scale
        e = self.t.exp()
        # 1 + rest, rest without the largest: log(1 + rest) of a rounded sum would be off by 2^-53, more than the kernels' error where
        # rest is 1e-12
        rest = e.scatter(1, self.t.argmax(1, keepdim=True), 0.0).sum(1, keepdim=True)
        rest = torch.where(self.m.isinf(), math.nan, rest)
        self.logz = torch.log1p(rest)
        self.logp = self.t - self.logz
        self.p = e / (1 + rest)
        self.tail = rest / (1 + rest)
        # relative to rest = sum' e_i (without the largest): sum' e_i (|t_i| + 4) 2^-23 / sum' e_i, where sum' e_i |t_i| / sum' e_i is
        # sum p_i |t_i| / tail, since the largest has t = 0
        size = (self.p * self.t.clamp(min=-1e30).abs()).sum(1, keepdim=True) / self.tail.clamp(min=1e-300)
        self.rel = 2.0 ** -23 * (size + 4) + (s.shape[1] / 64 + 64) * 2.0 ** -24
        self.entropy = -(self.p * self.logp.clamp(min=-1e300)).sum(1, keepdim=True)


def near(got, ref, tol, what):
    got = got.double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    bad = ~(same | ((got - ref).abs() <= tol))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, first {got[bad][0]} for {ref[bad][0]}"


def before(torch, s, labels):
    mine = s.gather(1, labels.long().clamp(min=0)[:, None])
    b = (s > mine) | ((s == mine) & (torch.arange(s.shape[1], device=s.device) < labels[:, None]))
    return torch.where(labels >= 0, b.sum(1), -1).int()


def check_forward(torch, s, labels, top, r):
    q = Row64(torch, s)
    lab = labels.long().clamp(min=0)[:, None]
    tol = lambda v: 2.0 ** -23 * v.abs() + 1.01 * q.rel * q.tail + 1e-44      # noqa: E731
    lp = torch.where(labels[:, None] >= 0, q.logp.gather(1, lab), 0.0)
    near(r.logprob, lp[:, 0], tol(torch.where(lp.isinf(), 0.0, lp))[:, 0], "logprob")
    near(r.entropy, q.entropy[:, 0], (q.rel * (2 * q.entropy + q.tail) + 1e-30)[:, 0], "entropy")
    assert torch.equal(r.rank, before(torch, s, labels))
    near(r.stats[:, :1], q.m, 0 * q.m, "maximum")
    near(r.stats[:, 1:], q.logz, tol(q.logz), "log sum")
    if top:
        value, index = torch.sort(s.double(), dim=1, descending=True, stable=True)
        n = min(top, s.shape[1])
        masked = value[:, :n] == -INF
        assert torch.equal(r.top_index[:, :n], torch.where(masked, -1, index[:, :n]).int())
        ref = q.logp.gather(1, index[:, :n])
        near(r.top_logprob[:, :n], ref, tol(torch.where(ref.isinf(), 0.0, ref)), "list")
        assert bool((r.top_index[:, n:] == -1).all()) and bool((r.top_logprob[:, n:] == -INF).all())


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_logprob_forward(env, mode, shape):
    hpf, torch, ops = env
    print(f"\n[case] logprob {shape} {mode}", flush=True)
    s, labels, _ = make(torch, mode, *shape)
    for top in (0, 1, 5, 64):
        r = ops[mode].logprob_forward(s, labels, top)
        check_forward(torch, s, labels, top, r)
        again = ops[mode].logprob_forward(s, labels, top)
        assert all(p is None or torch.equal(p, q) for p, q in zip(r, again)), "same inputs, other bits"
    no = ops[mode].logprob_forward(s)
    assert no.logprob is None and no.rank is None and no.top_index is None and torch.equal(no.entropy, r.entropy)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(3, 65), (5, 1000), (130, 1001), (3, 20000), (2, 70001)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("left,right", [(0, 7), (1, 0), (3, 4), (8, 8)])
def test_views_give_what_dense_rows_give(env, mode, shape, left, right):
    hpf, torch, ops = env
    print(f"\n[case] views {shape} {mode} {left} {right}", flush=True)
    s, labels, g = make(torch, mode, *shape, left=left, right=right)
    dense = s.contiguous()
    r, rd = ops[mode].logprob_forward(s, labels, 20), ops[mode].logprob_forward(dense, labels, 20)
    check_forward(torch, s, labels, 20, r)
    assert torch.equal(r.rank, rd.rank) and torch.equal(r.top_index, rd.top_index)
    args = dict(grad_logprob=torch.randn(shape[0], device="cuda", generator=g), entropy=rd.entropy,
                grad_entropy=torch.randn(shape[0], device="cuda", generator=g))
    want = ops[mode].logprob_backward(dense, labels, rd.stats, **args)
    wide = torch.full((shape[0], left + shape[1] + right), 9.0, device="cuda", dtype=s.dtype)
    out = wide[:, left:left + shape[1]]
    assert torch.equal(want, ops[mode].logprob_backward(s, labels, rd.stats, **args))
    assert torch.equal(want, ops[mode].logprob_backward(s, labels, rd.stats, out=out, **args))
    assert bool((wide[:, :left] == 9).all()) and bool((wide[:, left + shape[1]:] == 9).all())
    assert torch.equal(want, ops[mode].logprob_backward(dense, labels, rd.stats, out=dense, **args))       # in place
    top = rd.top_index, torch.where(rd.top_index < 0, 0.0, rd.top_logprob)
    q1, qt = Row64(torch, s), Row64(torch, s, 0.5)
    for e in (s, s.contiguous()):
        loss, ds = ops[mode].distill(e, *top, labels, temperature=2.0, hard_weight=0.5)
        check_distill(torch, mode, e, *top, labels, 2.0, 0.5, None, loss, ds, q1, qt)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_logprob_backward(env, mode, shape):
    hpf, torch, ops = env
    print(f"\n[case] logprob gradient {shape} {mode}", flush=True)
    s, labels, g = make(torch, mode, *shape)
    rows = shape[0]
    r = ops[mode].logprob_forward(s, labels)
    gl, gh = torch.randn(rows, device="cuda", generator=g), torch.randn(rows, device="cuda", generator=g)
    logp = s.double() - r.stats.double().sum(1, keepdim=True)
    p, lc = logp.exp(), logp.clamp(min=-1e300)
    hot = torch.arange(shape[1], device="cuda") == labels[:, None]
    h = r.entropy.double()[:, None]
    for with_l, with_h in ((1, 1), (1, 0), (0, 1)):
        a = (gl.double() * (labels >= 0))[:, None] * with_l
        b = gh.double()[:, None] * with_h
        ref = a * hot - a * p - b * p * (lc + h)
        got = ops[mode].logprob_backward(s, labels if with_l else None, r.stats, gl if with_l else None, r.entropy if with_h else None,
                                         gh if with_h else None)
        # the argument of exp is off by 2^-24 of its terms; at the label 1 - p comes from expm1(log p)
        size = (s.double() - r.stats[:, :1].double()).clamp(min=-1e30).abs() + lc.clamp(min=-1e30).abs() + 4
        rel = torch.where(p > 0, 2.0 ** -23 * size, 0.0)
        tol = HALF[mode] * 1.01 * ref.abs() + rel * (a.abs() * p + b.abs() * p * (lc.abs() + h + 1)) + 2.0 ** -22 * (a * hot).abs() * (1 - p) + 1e-37
        near(got, ref, tol, "dlogits")
        assert torch.equal(got, ops[mode].logprob_backward(s, labels, r.stats, gl if with_l else None, r.entropy, gh if with_h else None))


def teacher(torch, s, top, g):
    t = s.double() * 0.6 + torch.randn(s.shape, device="cuda", generator=g, dtype=torch.float64)
    t = torch.where(s.isinf(), -INF, t)
    value, index = t.topk(min(top, s.shape[1]), dim=1)
    absent = value.isinf()
    absent[::3, index.shape[1] // 2:] = True
    return torch.where(absent, -1, index).int().contiguous(), torch.where(absent, 3.0, value).float().contiguous()


def distill64(torch, s, index, logit, labels, T, hw, weight):
    """(loss, ds, log q and p of the entries) from the definition."""
    rows, classes = s.shape
    T, hw = (float(torch.tensor(v, dtype=torch.float32)) for v in (T, hw))       # the call takes them in fp32: 1 - 0.9f is 2.4e-7 from 0.1
    q1, qt = torch.log_softmax(s.double(), 1), torch.log_softmax(s.double() / T, 1)
    on = (index >= 0) & (logit > -INF)
    some = on.any(1, keepdim=True)
    t = torch.where(on, logit.double() / T, -1e300)
    logt = t - torch.logsumexp(t, 1, keepdim=True)
    p = logt.exp() * on
    idx = index.long().clamp(min=0)
    loss = (1 - hw) * T * T * torch.where(p > 0, p * (logt - qt.gather(1, idx)), 0.0).sum(1)
    has = labels >= 0
    hot = torch.arange(classes, device="cuda") == labels[:, None]
    if hw:
        loss = loss - hw * torch.where(hot, q1, 0.0).sum(1)
    want = torch.zeros_like(q1).scatter_add_(1, idx, p)
    ds = (1 - hw) * T * (qt.exp() * some - want) + hw * (q1.exp() * has[:, None] - hot.double())
    w = torch.ones(rows, 1, device="cuda", dtype=torch.float64) if weight is None else weight.double()[:, None]
    return loss, ds * w, w


def check_distill(torch, mode, s, index, logit, labels, T, hw, weight, loss, ds, q1=None, qt=None):
    q1, qt = q1 or Row64(torch, s), qt or Row64(torch, s, 1 / T)
    ref, dref, w = distill64(torch, s, index, logit, labels, T, hw, weight)
    # the list in double: log q is off by log Z's error alone
    tol = 2.0 ** -23 * ref.abs() + 1.01 * ((1 - hw) * T * T * qt.rel * qt.tail + hw * q1.rel * q1.tail)[:, 0] + 1e-44
    near(loss, ref, torch.where(ref.isinf(), 0.0, tol), "loss")
    if ds is not None:
        soft, hard = (1 - hw) * T * w.abs() * qt.p, hw * w.abs() * q1.p
        arg = 2.0 ** -23 * (q1.t.clamp(min=-1e30).abs() * (1 / T + 1) + 4)
        tol = HALF[mode] * 1.01 * dref.abs() + soft * (qt.rel + arg) + hard * (q1.rel + arg) + 1e-37
        # at the listed classes and the label: the difference of two logarithms, so relative to the smaller tail
        near(ds, dref, torch.where(tol.isnan(), 1e-37, tol), "dlogits")


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_distill(env, mode, shape):
    hpf, torch, ops = env
    print(f"\n[case] distill {shape} {mode}", flush=True)
    s, labels, g = make(torch, mode, *shape)
    rows = shape[0]
    for top, T, hw in ((1, 1.0, 0.0), (5, 2.0, 0.25), (64, 4.0, 0.5), (20, 0.5, 0.9), (3, 1.0, 1.0)):
        index, logit = teacher(torch, s, top, g)
        weight = torch.randn(rows, device="cuda", generator=g) if top != 5 else None
        loss, ds = ops[mode].distill(s, index, logit, labels, temperature=T, hard_weight=hw, row_weight=weight)
        check_distill(torch, mode, s, index, logit, labels, T, hw, weight, loss, ds)
        again = ops[mode].distill(s, index, logit, labels, temperature=T, hard_weight=hw, row_weight=weight)
        assert torch.equal(loss, again[0]) and torch.equal(ds, again[1]), "same inputs, other bits"
        alone, none = ops[mode].distill(s, index, logit, labels, temperature=T, hard_weight=hw, gradient=False)
        assert none is None
        check_distill(torch, mode, s, index, logit, labels, T, hw, weight, alone, None)
    loss, ds = ops[mode].distill(s, None, None, labels, hard_weight=1.0)       # no list: the cross-entropy of the label
    none = torch.full((rows, 1), -1, device="cuda", dtype=torch.int32)
    check_distill(torch, mode, s, none, torch.zeros(rows, 1, device="cuda"), labels, 1.0, 1.0, None, loss, ds)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [3, 100, 5000, 40001])
def test_a_class_that_is_all_but_certain(env, mode, classes):
    """log p and p - 1 of such a class keep their digits: relative, not absolute, in what is left."""
    hpf, torch, ops = env
    s = torch.zeros(4, classes, device="cuda") - 2
    s[torch.arange(4), torch.tensor([0, 1, classes - 1, classes // 2])] = 13.0
    s = s.to(torch.bfloat16 if mode == "bf16" else torch.float32)
    labels = torch.tensor([0, 1, classes - 1, classes // 2], device="cuda", dtype=torch.int32)
    rest = (classes - 1) * math.exp(-15.0)
    r = ops[mode].logprob_forward(s, labels, 2)
    rel = 2.0 ** -23 * 20 + (classes / 64 + 64) * 2.0 ** -24
    near(r.logprob, torch.full((4,), -math.log1p(rest), device="cuda", dtype=torch.float64), torch.tensor(rel * rest, device="cuda"), "logprob")
    want = rest / (1 + rest) * 15 + math.log1p(rest)
    near(r.entropy, torch.full((4,), want, device="cuda", dtype=torch.float64), torch.tensor(2 * rel * want, device="cuda"), "entropy")
    d = ops[mode].logprob_backward(s, labels, r.stats, torch.ones(4, device="cuda"))
    at = d.gather(1, labels.long()[:, None])[:, 0]
    near(at, torch.full((4,), rest / (1 + rest), device="cuda", dtype=torch.float64), torch.tensor((rel + HALF[mode]) * 1.1 * rest, device="cuda"), "gradient")
    loss, ds = ops[mode].distill(s, labels[:, None].contiguous(), torch.zeros(4, 1, device="cuda"), labels, hard_weight=0.5)
    near(loss, torch.full((4,), math.log1p(rest), device="cuda", dtype=torch.float64), torch.tensor(rel * rest * 1.1, device="cuda"), "loss")
    at = ds.gather(1, labels.long()[:, None])[:, 0]
    near(at, torch.full((4,), -rest / (1 + rest), device="cuda", dtype=torch.float64), torch.tensor((rel + HALF[mode]) * 1.1 * rest, device="cuda"), "gradient")


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [6, 1000, 3001, 70000])
def test_masked_and_broken_rows(env, mode, classes):
    hpf, torch, ops = env
    lowest = torch.finfo(torch.bfloat16 if mode == "bf16" else torch.float32).min
    s, _, g = make(torch, mode, 10, classes, seed=3)
    labels = torch.tensor([0, 1, 2, 3, 4, -1, classes - 1, classes, -7, 2], device="cuda", dtype=torch.int32)
    s[0] = -INF                                    # nothing left
    s[1, :] = -INF
    s[1, 1] = 2.0                                  # one class left, the label
    s[2, :] = lowest                               # masks of the type's lowest value
    s[2, 2], s[2, 3] = 1.0, 1.0
    s[3, classes // 2] = float("nan")
    s[4, classes - 2] = INF
    s[5] = -INF
    s[6] = lowest                                  # every class at the lowest value: equal ones
    s[9, :] = -INF
    s[9, 0], s[9, 3] = 0.0, 0.0                    # the label is masked
    r = ops[mode].logprob_forward(s, labels, 4)
    lp, ent, rank, ti, tl = [t.cpu() for t in (r.logprob, r.entropy, r.rank, r.top_index, r.top_logprob)]
    assert lp[0] == -INF and ent[0] == 0 and rank[0] == 0 and ti[0].tolist() == [-1] * 4 and bool((tl[0] == -INF).all())
    assert lp[1] == 0 and ent[1] == 0 and rank[1] == 0 and ti[1].tolist() == [1, -1, -1, -1] and tl[1, 0] == 0 and tl[1, 1] == -INF
    assert abs(float(lp[2]) + math.log(2)) < 1e-6 and rank[2] == 0 and ti[2].tolist() == [2, 3, 0, 1] and tl[2, 2] < -1e38
    for i in (3, 4):
        assert math.isnan(lp[i]) and math.isnan(ent[i]) and rank[i] == -1 and ti[i].tolist() == [-1] * 4 and bool(tl[i].isnan().all())
    assert lp[5] == 0 and rank[5] == -1 and ent[5] == 0
    assert abs(float(lp[6]) + math.log(classes)) < 1e-5 * math.log(classes) and abs(float(ent[6]) - math.log(classes)) < 1e-5 * math.log(classes)
    assert rank[6] == classes - 1 and ti[6].tolist() == [0, 1, 2, 3]
    assert math.isnan(lp[7]) and rank[7] == -1 and math.isnan(lp[8]) and rank[8] == -1
    assert not math.isnan(ent[7]) and ti[7, 0] >= 0
    assert lp[9] == -INF and rank[9] == 3 and ti[9].tolist() == [0, 3, -1, -1]
    one = torch.ones(10, device="cuda")
    d = ops[mode].logprob_backward(s, labels, r.stats, one, r.entropy, one).float().cpu()
    assert not bool(d[0].any()) and not bool(d[1].any()) and not bool(d[5].any())
    for i in (3, 4, 7, 8):
        assert bool(d[i].isnan().all())
    for i in (2, 6, 9):
        assert bool(d[i].isfinite().all())
    assert abs(float(d[2, 2]) - 0.5) < 1e-2 and abs(float(d[2, 3]) + 0.5) < 1e-2 and not bool(d[2, 4:].any())
    assert abs(float(d[9, 0]) + 0.5) < 1e-2 and float(d[9, 2]) == 1.0
    index = torch.tensor([[2, 3]] * 10, device="cuda", dtype=torch.int32)
    logit = torch.zeros(10, 2, device="cuda")
    loss, ds = ops[mode].distill(s, index, logit, labels, hard_weight=0.5)
    loss, ds = loss.cpu(), ds.float().cpu()
    assert loss[0] == 0 and not bool(ds[0].any()) and loss[5] == 0 and not bool(ds[5].any())
    assert loss[1] == INF and float(ds[1, 2]) == -0.25 and float(ds[1, 1]) == 0.5          # listed classes that the student may not answer
    assert abs(float(loss[2]) - 0.5 * math.log(2)) < 1e-6 and abs(float(ds[2, 2]) + 0.25) < 1e-3 and abs(float(ds[2, 3]) - 0.25) < 1e-3
    for i in (3, 4, 7, 8):
        assert math.isnan(loss[i]) and bool(ds[i].isnan().all())
    assert loss[9] == INF and bool(ds[9].isfinite().all())


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [5, 130, 1024, 9000, 66000])
def test_ties_take_the_lowest_index(env, mode, classes):
    hpf, torch, ops = env
    g = torch.Generator(device="cuda").manual_seed(classes)
    s = torch.randint(-2, 3, (6, classes), device="cuda", generator=g).to(torch.bfloat16 if mode == "bf16" else torch.float32)
    s[0] = 1.0                                       # all equal
    s[1] = 0.0
    s[1, ::2] = -0.0                                 # zeros of either sign are equal
    s[2] = torch.arange(classes, device="cuda").float().to(s.dtype)      # rising: the list is at the end of the row
    s[3] = -s[2]
    labels = torch.tensor([classes - 1, 3, 0, classes // 2, 1, 4], device="cuda", dtype=torch.int32)
    for top in (1, 4, 33, 64):
        check_forward(torch, s, labels, top, ops[mode].logprob_forward(s, labels, top))


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [64, 1000, 50000])
def test_lists_whose_classes_lie_together(env, mode, classes):
    """The largest logits side by side, at every 64th, 256th and 1024th class, in one order and the other."""
    hpf, torch, ops = env
    rows = []
    for stride in (1, 8, 64, 256, 1024):
        for sign in (1, -1):
            base = torch.randn(classes, device="cuda") * 0.1
            n = min(100, (classes - 1) // stride + 1)
            base[torch.arange(n, device="cuda") * stride] = 5 + sign * torch.arange(n, device="cuda") * 0.01
            rows.append(base)
    s = torch.stack(rows).to(torch.bfloat16 if mode == "bf16" else torch.float32)
    labels = torch.zeros(len(rows), device="cuda", dtype=torch.int32)
    for top in (3, 64):
        check_forward(torch, s, labels, top, ops[mode].logprob_forward(s, labels, top))


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [12, 900, 30000])
def test_lists_with_repeated_and_absent_and_bad_entries(env, mode, classes):
    hpf, torch, ops = env
    s, labels, g = make(torch, mode, 5, classes, seed=5)
    index = torch.tensor([[3, 3, 7, -1, 3], [-1, -1, -1, -1, -1], [1, 2, 3, 4, classes], [9, 8, 9, 8, 9], [0, 1, 0, 6, -5]], device="cuda", dtype=torch.int32)
    logit = torch.randn(5, 5, device="cuda", generator=g)
    logit[3, 1], logit[3, 3] = -INF, -INF             # both entries of class 8: not there
    labels[:] = torch.tensor([3, 1, 1, 2, -1], device="cuda")
    loss, ds = ops[mode].distill(s, index, logit, labels, temperature=1.5, hard_weight=0.3)
    assert math.isnan(loss[2]) and bool(ds[2].isnan().all())
    keep = torch.tensor([0, 1, 3, 4], device="cuda")
    check_distill(torch, mode, s[keep], index[keep], logit[keep], labels[keep], 1.5, 0.3, None, loss[keep], ds[keep])
    logit[0, 1] = float("nan")
    loss, ds = ops[mode].distill(s, index, logit, labels, temperature=1.5, hard_weight=0.3)
    assert math.isnan(loss[0]) and math.isnan(ds[0, 3])


def test_gradients_against_differences(env):
    """Central differences of the definitions in 64 bits along random directions (h^2 error: below 1e-7 of the scale)."""
    hpf, torch, ops = env
    rows, classes, h = 6, 50, 1e-4
    g = torch.Generator(device="cuda").manual_seed(1)
    s = torch.randn(rows, classes, device="cuda", generator=g) * 2
    labels = torch.randint(0, classes, (rows,), device="cuda", generator=g).int()
    index, logit = teacher(torch, s, 8, g)
    r = ops["f32"].logprob_forward(s, labels)
    gl, gh = torch.randn(rows, device="cuda", generator=g), torch.randn(rows, device="cuda", generator=g)
    d = ops["f32"].logprob_backward(s, labels, r.stats, gl, r.entropy, gh)
    loss, ds = ops["f32"].distill(s, index, logit, labels, temperature=2.0, hard_weight=0.3)

    def scores(x):
        logp = torch.log_softmax(x, 1)
        return float((gl.double() * logp.gather(1, labels.long()[:, None])[:, 0] - gh.double() * (logp.exp() * logp).sum(1)).sum())

    def losses(x):
        return float(distill64(torch, x, index, logit, labels, 2.0, 0.3, None)[0].sum())
    for _ in range(5):
        v = torch.randn(rows, classes, device="cuda", generator=g, dtype=torch.float64)
        for f, grad in ((scores, d), (losses, ds)):
            diff = (f(s.double() + h * v) - f(s.double() - h * v)) / (2 * h)
            mine = float((grad.double() * v).sum())
            # fp32 gradients: 2^-20 relative in each of the terms at most
            assert abs(diff - mine) <= 2.0 ** -20 * float((grad.double() * v).abs().sum()) + 1e-6, (diff, mine)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_no_rows(env, mode):
    hpf, torch, ops = env
    s = torch.zeros(0, 40, device="cuda", dtype=ops[mode].tdtype)
    labels = torch.zeros(0, device="cuda", dtype=torch.int32)
    r = ops[mode].logprob_forward(s, labels, 3)
    assert r.logprob.shape == (0,) and r.top_index.shape == (0, 3)
    assert ops[mode].logprob_backward(s, labels, r.stats, r.logprob).shape == (0, 40)
    loss, ds = ops[mode].distill(s, r.top_index, r.top_logprob, labels, hard_weight=0.5)
    assert loss.shape == (0,) and ds.shape == (0, 40)


@pytest.mark.parametrize("shape", [(1, 131072), (40, 1000), (6, 70001)], ids=lambda s: "x".join(map(str, s)))
def test_streams_and_graphs(env, shape):
    hpf, torch, ops = env
    o = ops["bf16"]
    data = [make(torch, "bf16", *shape, seed=20 + i)[:2] for i in range(2)]
    one = torch.ones(shape[0], device="cuda")

    def every(s, labels):
        r = o.logprob_forward(s, labels, 20)
        d = o.logprob_backward(s, labels, r.stats, one, r.entropy, one)
        return tuple(r) + (d,) + o.distill(s, r.top_index, r.top_logprob, labels, temperature=2.0, hard_weight=0.5)
    want = [every(*e) for e in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(3):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = every(*data[i])
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(p, q) for p, q in zip(got[i], want[i]))
    s, labels = data[0][0].clone(), data[0][1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        every(s, labels)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=streams[0]):
        out = every(s, labels)
    for i in (0, 1, 0, 1):
        s.copy_(data[i][0]), labels.copy_(data[i][1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[i]))
        assert all(torch.equal(p, q) for p, q in zip(every(*data[i]), want[i]))


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes,period,part,top", [(1020, 256, 80, 30), (2040, 512, 160, 30), (7900, 1024, 192, 20), (16000, 2048, 384, 20), (65000, 4096, 128, 5),
                                                     (131072, 8192, 256, 5), (200001, 1024, 192, 40)])
def test_lists_among_thousands_of_large_logits(env, mode, classes, period, part, top):
    """Large logits in the first `part` classes of every `period` and small ones elsewhere: whole threads hold nothing else, and no simple
    bound separates the list from the rest.  Distinct values, then many equal ones."""
    hpf, torch, ops = env
    g = torch.Generator(device="cuda").manual_seed(classes)
    c = torch.arange(classes, device="cuda")
    s = torch.randn(4, classes, device="cuda", generator=g)
    large = (c % period) < part
    s[:2] += 30.0 * large
    s[1:3] = s[1:3].round()
    s[3] = torch.where(large, 7.0, 6.0)
    s = s.to(torch.bfloat16 if mode == "bf16" else torch.float32)
    labels = torch.tensor([0, classes - 1, 5, classes // 2], device="cuda", dtype=torch.int32)
    for n in (top, 64):
        check_forward(torch, s, labels, n, ops[mode].logprob_forward(s, labels, n))
    views = torch.cat([torch.zeros(4, 3, device="cuda", dtype=s.dtype), s], 1)[:, 3:]
    check_forward(torch, views, labels, top, ops[mode].logprob_forward(views, labels, top))


# As many rows as there are when none is divided among work-groups, at lengths on both sides of every kernel's
MANY = [(1100, 2052), (1030, 9001), (200, 20001), (140, 32768), (300, 50001), (140, 65536), (140, 65537), (260, 131072)]


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s)))
def test_many_long_rows(env, mode, shape):
    hpf, torch, ops = env
    print(f"\n[case] many rows {shape} {mode}", flush=True)
    s, labels, g = make(torch, mode, *shape)
    for top in (0, 64):
        r = ops[mode].logprob_forward(s, labels, top)
        check_forward(torch, s, labels, top, r)
        again = ops[mode].logprob_forward(s, labels, top)
        assert all(p is None or torch.equal(p, q) for p, q in zip(r, again)), "same inputs, other bits"
    index, logit = teacher(torch, s, 20, g)
    weight = torch.randn(shape[0], device="cuda", generator=g)
    for T, hw in ((1.0, 0.25), (2.0, 0.5), (4.0, 0.1), (0.7, 0.9), (3.0, 0.0)):
        loss, ds = ops[mode].distill(s, index, logit, labels, temperature=T, hard_weight=hw, row_weight=weight)
        check_distill(torch, mode, s, index, logit, labels, T, hw, weight, loss, ds)
        alone, none = ops[mode].distill(s, index, logit, labels, temperature=T, hard_weight=hw, row_weight=weight, gradient=False)
        assert none is None and torch.equal(loss, alone)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1030, 9001), (200, 20001), (300, 50001), (260, 131000)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("left,right", [(1, 0), (3, 4)])
def test_views_of_many_long_rows(env, mode, shape, left, right):
    test_views_give_what_dense_rows_give(env, mode, shape, left, right)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("copies,classes", [(110, 2100), (20, 20000), (20, 40000), (30, 50000), (30, 131000)])
def test_masked_and_broken_rows_among_many(env, mode, copies, classes):
    """Ten special rows over and over: each copy like the first one, bit for bit, and like the ten alone, which other kernels take: to twice
    the bound that holds for either, with sum p |t| <= 30 and an entropy of at most log(131000) < 12."""
    hpf, torch, ops = env
    lowest = torch.finfo(torch.bfloat16 if mode == "bf16" else torch.float32).min
    s, _, g = make(torch, mode, 10, classes, seed=3)
    labels = torch.tensor([0, 1, 2, 3, 4, -1, classes - 1, classes, -7, 2], device="cuda", dtype=torch.int32)
    s[0] = s[5] = -INF
    s[1, :] = -INF
    s[1, 1] = 2.0
    s[2, :] = lowest
    s[2, 2], s[2, 3] = 1.0, 1.0
    s[3, classes // 2] = float("nan")
    s[4, classes - 2] = INF
    s[6] = lowest
    s[9, :] = -INF
    s[9, 0], s[9, 3] = 0.0, 0.0
    index = torch.tensor([[2, 3, -1]] * 7 + [[5, classes, 1], [1, 1, 0], [0, 3, 7]], device="cuda", dtype=torch.int32)
    logit = torch.tensor([[0.0, 1.0, 2.0]] * 10, device="cuda")
    few = ops[mode].logprob_forward(s, labels, 30)
    many = ops[mode].logprob_forward(s.repeat(copies, 1), labels.repeat(copies), 30)
    few_d = ops[mode].distill(s, index, logit, labels, temperature=2.0, hard_weight=0.5)
    many_d = ops[mode].distill(s.repeat(copies, 1), index.repeat(copies, 1), logit.repeat(copies, 1), labels.repeat(copies), temperature=2.0, hard_weight=0.5)
    rel = 2.0 ** -23 * 64 + (classes / 64 + 64) * 2.0 ** -24
    for name, a, b in [(n, getattr(few, n), getattr(many, n)) for n in few._fields] + [("loss", few_d[0], many_d[0]), ("dlogits", few_d[1], many_d[1])]:
        b = b.view(copies, *a.shape)
        same = (b == b[:1]) | (b.isnan() & b[:1].isnan())
        assert bool(same.all()), f"{name}: copies of a row differ"
        if a.dtype == torch.int32:
            assert torch.equal(a, b[0]), name
            continue
        a = a.double()
        size = 2.0 ** -23 * torch.where(a.isinf() | a.isnan(), 0.0, a.abs())
        tol = 2 * (size + rel * (25 if name == "entropy" else 4 if name == "loss" else 1))
        near(b[0], a, tol if name != "dlogits" else tol + 2 * HALF[mode] * a.abs(), name)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("classes,period,part", [(9000, 1024, 192), (20000, 2048, 384), (50000, 4096, 128), (131072, 8192, 256)])
def test_lists_among_thousands_of_large_logits_of_many_rows(env, mode, classes, period, part):
    hpf, torch, ops = env
    g = torch.Generator(device="cuda").manual_seed(classes)
    c = torch.arange(classes, device="cuda")
    s = torch.randn(260, classes, device="cuda", generator=g)
    large = (c % period) < part
    s[:130] += 30.0 * large
    s[65:195] = s[65:195].round()
    s[195:230] = torch.where(large, 7.0, 6.0)
    s[230:] = 1.0
    s = s.to(torch.bfloat16 if mode == "bf16" else torch.float32)
    labels = torch.randint(0, classes, (260,), device="cuda", generator=g).int()
    for top in (5, 64):
        check_forward(torch, s, labels, top, ops[mode].logprob_forward(s, labels, top))


@pytest.mark.parametrize("shape", [(1030, 9001), (200, 20001), (140, 65536), (300, 70001)], ids=lambda s: "x".join(map(str, s)))
def test_streams_and_graphs_of_many_rows(env, shape):
    test_streams_and_graphs(env, shape)


@pytest.mark.parametrize("shape", [(64, 16500), (65, 16500), (100, 33001), (100, 70001)], ids=lambda s: "x".join(map(str, s)))
def test_rows_around_the_number_that_is_divided(env, shape):
    test_many_long_rows(env, "bf16", shape)
    test_many_long_rows(env, "f32", shape)


@pytest.mark.parametrize("shape", [(1 << 21, 1), (1 << 21, 3), (1, 1 << 28)], ids=lambda s: "x".join(map(str, s)))
def test_largest_sizes(env, shape):
    hpf, torch, ops = env
    print(f"\n[case] largest {shape}", flush=True)
    s, labels, g = make(torch, "bf16", *shape)
    r = ops["bf16"].logprob_forward(s, labels, 5)
    check_forward(torch, s, labels, 5, r)
    index, logit = r.top_index, torch.where(r.top_index < 0, 0.0, r.top_logprob)
    loss, ds = ops["bf16"].distill(s, index, logit, labels, temperature=2.0, hard_weight=0.5)
    check_distill(torch, "bf16", s, index, logit, labels, 2.0, 0.5, None, loss, ds)
