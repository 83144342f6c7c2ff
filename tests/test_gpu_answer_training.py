"""Training a partition through the operators of the answer end: a partition without a head, a classifier of its own behind it, a loss against a
teacher's list; the classifier's dx goes back into the partition as err_in, and its gradients are the whole model's."""
import numpy as np
import pytest

import parity
from paper_1911_05146_amd import workloads as W

pytestmark = pytest.mark.gpu

CLASSES, TOP, T, HARD = 100, 8, 2.0, 0.25


@pytest.mark.parametrize("mode", ["f32", "bf16"])
def test_distillation_trains_a_partition(oracle, mode):
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: these tests need a real MI355X")
    from paper_1911_05146_amd import hpf
    print(f"\n[case] partition behind a distilled classifier {mode}", flush=True)
    blk = W.Block(W.BASIC, 16, 16, 16, 1)
    spec = W.PartitionSpec(name="student", in_h=8, in_w=8, in_c=16, blocks=(blk, blk), microbatch=8, num_microbatches=2, seed=5)
    inp = W.make_inputs(spec, randomize_affine=True)
    dtype = hpf.HPF_BF16 if mode == "bf16" else hpf.HPF_F32
    o, part = hpf.Ops(dtype), hpf.Partition(spec, inp.params, dtype)
    g = torch.Generator(device="cuda").manual_seed(11)
    b, m = spec.microbatch, spec.num_microbatches
    features = int(np.prod(part.out_shape[1:]))
    w, bias = torch.randn(features, CLASSES, device="cuda", generator=g) * features ** -0.5, torch.randn(CLASSES, device="cuda", generator=g) * 0.1
    wt = torch.randn(features, CLASSES, device="cuda", generator=g) * 2 * features ** -0.5
    labels = [torch.randint(0, CLASSES, (b,), device="cuda", generator=g).int() for _ in range(m)]
    weight = torch.full((b,), 1.0 / spec.divisor, device="cuda")
    weights, teacher = o.linear_weights(w), o.linear_weights(wt)
    dw, db = torch.zeros(features, CLASSES, device="cuda"), torch.zeros(CLASSES, device="cuda")
    acts = [torch.from_numpy(a).to("cuda", o.tdtype) for a in inp.act_in]
    try:
        outs, lists, errs, err_out = [], [], [], []
        for i in range(m):
            outs.append(part.forward_microbatch(i, acts[i]))
        for i in range(m):
            x = outs[i].view(b, features)
            t = o.logprob_forward(o.linear_forward(x, teacher), top=TOP)
            s = o.linear_forward(x, weights, bias)
            loss, ds = o.distill(s, t.top_index, t.top_logprob, labels[i], temperature=T, hard_weight=HARD, row_weight=weight)
            dx, _, _ = o.linear_backward(ds, x, weights, dw=dw, db=db, accumulate=True)
            lists.append((t.top_index, t.top_logprob))
            errs.append(dx.view(part.out_shape))
            err_out.append(part.backward_microbatch(i, errs[i]))
        torch.cuda.synchronize()
        res = {"act_out": [a.float().cpu().numpy() for a in outs], "err_out": [e.float().cpu().numpy() for e in err_out], "loss": 0.0,
               "grad": part.grad_accum_read()}
    finally:
        part.close()
    seen_w = w.to(o.tdtype).double()

    def classifier(a, i):
        """Gradient of the micro-batch's loss with respect to the features `a`, W and b in 64 bits."""
        x, p, c = (v.detach().double().requires_grad_() for v in (a.reshape(b, features), seen_w, bias))
        s = x @ p + c
        teach, logq = torch.softmax(lists[i][1].double() / T, 1), torch.log_softmax(s / T, 1)
        kl = (teach * (teach.log() - logq.gather(1, lists[i][0].long()))).sum(1)
        ce = -torch.log_softmax(s, 1).gather(1, labels[i].long()[:, None])[:, 0]
        (((1 - HARD) * T * T * kl + HARD * ce) / spec.divisor).sum().backward()
        return x.grad, p.grad, c.grad
    want = [classifier(outs[i], i) for i in range(m)]
    # 2-norms; bf16 rounds s, ds and dx by 2^-8 each at most, and s moves the gradient by its own size at most; fp32 the same with 2^-24, and sums
    tol = 4 * 2.0 ** -8 if mode == "bf16" else 1e-5
    for i in range(m):
        assert float((errs[i].reshape(b, features).double() - want[i][0]).norm() / want[i][0].norm()) <= tol, "dx"
    for got, k in ((dw, 1), (db, 2)):
        ref = want[0][k] + want[1][k]
        assert float((got.double() - ref).norm() / ref.norm()) <= tol
    # the partition, fed the gradients that the classifier gave it
    host = [e.float().cpu().numpy() for e in errs]
    seen = W.StepInputs(inp.params, [a.float().cpu().numpy() for a in acts], None, host)
    yard = oracle.run_step(spec, seen, np.float32, storage="bf16" if mode == "bf16" else "none")
    seen64 = W.StepInputs(seen.params.astype(np.float64), [a.astype(np.float64) for a in seen.act_in], None, [e.astype(np.float64) for e in host])
    exact = oracle.run_step(spec, seen64, np.float64)
    print(parity.fmt(parity.compare(spec, res, yard, mode, ref64=exact)))
    if mode == "f32":
        # the whole model: the oracle's own features through the classifier and back, without anything of the device's but the teacher's list
        whole = W.StepInputs(seen64.params, seen64.act_in, None, [
            classifier(torch.from_numpy(np.asarray(exact["act_out"][i], np.float64)).cuda(), i)[0].cpu().numpy().reshape(part.out_shape) for i in range(m)])
        ref = oracle.run_step(spec, whole, np.float64)
        assert parity.rel_l2(res["grad"], ref["grad"]) <= parity.TOL["f32"]
