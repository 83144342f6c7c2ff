"""Timing cases of the operators at the answer end of a model (`hpf.Ops`): the matrix product with bias, activation and
residual, the log probabilities that an evaluation reads from logits, and the loss of a student that learns from a
teacher's top logits.

A case:
  task      "linear"            y = act(x W + bias) + residual, with the slope act'(x W + bias) that back-propagation needs if `slope`
            "linear-gradient"   dx, dW, dbias from dy and the slope
            "logprob"           log probability and rank of the labels, entropy, `top` most likely classes
            "logprob-gradient"  gradient of log probability and entropy with respect to the logits
            "distill"           loss against the teacher's `top` logits and the hard label, and its gradient
  dtype     "bf16" or "f32": type of the tensors (weights, their gradients and what there is one of per row: fp32)
  rows, inputs, outputs    sizes of a product
  rows, classes, pad       logits [rows, classes] whose rows lie classes + pad elements apart
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TEMPERATURE, HARD_WEIGHT = 2.0, 0.25
ACTIVATIONS = ("none", "relu", "gelu", "silu")


def listed():
    def linear(name, rows, inputs, outputs, dtype, activation, bias, residual, slope):
        return dict(name=name, task="linear", rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, activation=activation, bias=bias,
                    residual=residual, slope=slope)

    def gradient(name, rows, inputs, outputs, dtype, activation):
        return dict(name=name, task="linear-gradient", rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, activation=activation)

    def rows_of(name, task, rows, classes, pad, top, dtype):
        return dict(name=name, task=task, rows=rows, classes=classes, pad=pad, top=top, dtype=dtype)
    return [
        # one request through VGG-16's widest dense layer: bound by the weights and by latency
        linear("linear-one-row", 1, 4096, 4096, "bf16", "relu", True, False, False),
        # the same layer on a batch of 128
        linear("linear-batch", 128, 4096, 4096, "bf16", "relu", True, False, False),
        # a large batch with everything in the epilogue
        linear("linear-large", 8192, 4096, 4096, "bf16", "gelu", True, True, True),
        # the check mode, sizes that no tile divides
        linear("linear-ragged-f32", 333, 1000, 517, "f32", "silu", True, True, False),
        # gradients: the large batch, and a ragged one of ImageNet's 1000 classes
        gradient("linear-gradient-large", 8192, 4096, 4096, "bf16", "gelu"),
        gradient("linear-gradient-ragged", 1021, 2049, 1000, "bf16", "relu"),
        # one position of a model with many classes: a single row, all alternatives that a service offers
        rows_of("logprob-one-row", "logprob", 1, 131072, 0, 20, "bf16"),
        # evaluation of ImageNet logits as an inference call leaves them: top-1 / top-5
        rows_of("logprob-images", "logprob", 8192, 1000, 0, 5, "f32"),
        # a teacher's list over many classes, rows padded to 128 bytes
        rows_of("logprob-teacher", "logprob", 2048, 50257, 47, 64, "bf16"),
        # learning from rewards: gradient of log probability and entropy
        rows_of("logprob-gradient-wide", "logprob-gradient", 2048, 50257, 47, 0, "bf16"),
        # distillation of an image classifier, and with many classes
        rows_of("distill-images", "distill", 256, 1000, 0, 32, "f32"),
        rows_of("distill-wide", "distill", 2048, 131072, 0, 64, "bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo - 0.49), math.log(hi + 0.49))))))
    task = rng.choice(["linear", "linear-gradient", "logprob", "logprob-gradient", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if task.startswith("linear"):
        rows, inputs, outputs = log_int(1, 8192), log_int(10, 4096), log_int(10, 4096)
        if rng.random() < 0.5:                       # as most layers have it
            inputs, outputs = -(-inputs // 16) * 16, -(-outputs // 16) * 16
        if dtype == "f32":                           # the check mode is for small products
            rows = min(rows, max(1, int(4e9 / (inputs * outputs))))
        case = dict(task=task, rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, activation=rng.choice(ACTIVATIONS))
        if task == "linear":
            case |= dict(bias=rng.random() < 0.8, residual=rng.random() < 0.5)
            # relu's slope jumps where x W + bias is 0 within its rounding, so it is no output to compare
            case["slope"] = case["activation"] != "relu" and rng.random() < 0.6
        return case
    classes = log_int(2, 131072)
    rows = log_int(1, max(1, min(8192, int(1.3e8 / classes))))
    pad = -classes % 64 if rng.random() < 0.3 else 0
    top = min(classes, rng.choice([1, 5, 20, 32, 64])) if task != "logprob-gradient" else 0
    if task == "logprob" and rng.random() < 0.2:
        top = 0
    return dict(task=task, rows=rows, classes=classes, pad=pad, top=top, dtype=dtype)


def sizes(case):
    return case["rows"], case["inputs"], case["outputs"]


# ---- inputs -----------------------------------------------------------------------------------------------------
def logits_of(case, randn, rand):
    """Logits as a trained model gives them: noise, a few classes that stand out, and classes that are masked out."""
    rows, classes = case["rows"], case["classes"]
    s = randn(rows, classes + case["pad"]).mul_(2.5)
    for _ in range(3):
        c = (rand(rows, 1) * classes).long()
        s.scatter_add_(1, c, 12 * rand(rows, 1))
    if classes >= 64:                                # classes that may not be answered
        s[:, (rand(classes // 50) * (classes - 1)).long() + 1] = -math.inf
    return s.to(TYPES[case["dtype"]])[:, :classes]


def teacher_of(case, logits, randn, rand):
    """A teacher's list: the top of logits that resemble the student's, sorted; some rows have a shorter one (-1)."""
    rows, top = case["rows"], case["top"]
    t = logits.float()
    t = torch.where(t.isinf(), t, 0.7 * t + randn(*t.shape))
    value, index = t.topk(top, dim=1)
    length = torch.where(rand(rows, 1) < 0.1, (rand(rows, 1) * (top + 1)).floor(), float(top))
    absent = (torch.arange(top, device=DEVICE) >= length) | value.isinf()
    return torch.where(absent, -1, index).int(), torch.where(absent, 0.0, value)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device=DEVICE, generator=g)

    def rand(*shape):
        return torch.rand(*shape, device=DEVICE, generator=g)
    t = TYPES[case["dtype"]]
    state = {"case": dict(case)}
    if case["task"].startswith("linear"):
        rows, inputs, outputs = sizes(case)
        state["x"] = randn(rows, inputs).to(t)
        state["w"] = randn(inputs, outputs).mul_(math.sqrt(2.0 / inputs))
        if case["task"] == "linear":
            state["bias"] = randn(outputs).mul_(0.3) if case["bias"] else None
            state["residual"] = randn(rows, outputs).to(t) if case["residual"] else None
        else:
            state["dy"] = randn(rows, outputs).mul_(0.1).to(t)
            z = randn(rows, outputs).mul_(1.4)
            state["slope"] = None if case["activation"] == "none" else slope_of(case["activation"], z).to(t)
    else:
        rows, classes = case["rows"], case["classes"]
        state["logits"] = logits_of(case, randn, rand)
        likely = state["logits"].argmax(1)
        other = (rand(rows) * classes).long().clamp_(max=classes - 1)
        state["labels"] = torch.where(rand(rows) < 0.6, likely, other)
        state["labels"] = torch.where(rand(rows) < 0.05, -1, state["labels"]).int()        # rows without a label
        masked = state["logits"].gather(1, state["labels"].long().clamp(min=0)[:, None])[:, 0].isinf()
        state["labels"] = torch.where(masked, likely, state["labels"]).int()
        if case["task"] == "logprob-gradient":
            state["grad_logprob"] = randn(rows)
            state["grad_entropy"] = randn(rows).mul_(0.01)
            m = state["logits"].float().amax(1)
            z = (state["logits"].float() - m[:, None]).double().exp().sum(1)
            state["stats"] = torch.stack([m, z.log().float()], 1)
            logp = state["logits"].float() - state["stats"].sum(1, keepdim=True)
            state["entropy"] = -(logp.exp() * logp.clamp(min=-1e30)).sum(1)
        if case["task"] == "distill":
            state["top_index"], state["top_logit"] = teacher_of(case, state["logits"], randn, rand)
            state["row_weight"] = torch.full((rows,), 1.0 / rows, device=DEVICE)
    if own:      # the handle and the weights' layout that a program keeps from the last update of the weights on
        from paper_1911_05146_amd import hpf
        state["ops"] = hpf.Ops(hpf.HPF_BF16 if case["dtype"] == "bf16" else hpf.HPF_F32, DEVICE)
        if "w" in state:
            state["weights"] = state["ops"].linear_weights(state["w"])
    return state


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(state):
    return run_own(state) if own else run_plain(state)


def run_own(state):
    case, ops = state["case"], state["ops"]
    task = case["task"]
    if task == "linear":
        return ops.linear_forward(state["x"], state["weights"], state["bias"], state["residual"], case["activation"], slope=case["slope"])
    if task == "linear-gradient":
        return ops.linear_backward(state["dy"], state["x"], state["weights"], state["slope"])
    if task == "logprob":
        r = ops.logprob_forward(state["logits"], state["labels"], case["top"])
        return [r.logprob, r.entropy, r.rank] + ([r.top_index, r.top_logprob] if case["top"] else [])
    if task == "logprob-gradient":
        return ops.logprob_backward(state["logits"], state["labels"], state["stats"], state["grad_logprob"], state["entropy"], state["grad_entropy"])
    return ops.distill(state["logits"], state["top_index"], state["top_logit"], state["labels"], temperature=TEMPERATURE,
                       hard_weight=HARD_WEIGHT, row_weight=state["row_weight"])


def normal_below(z):
    """Phi(z): the standard normal distribution."""
    return 0.5 * torch.erfc(-z * math.sqrt(0.5))


def activated(activation, z):
    if activation == "relu":
        return z.clamp(min=0)
    if activation == "gelu":
        return z * normal_below(z)
    return z / (1 + torch.exp(-z)) if activation == "silu" else z


def slope_of(activation, z):
    if activation == "relu":
        return (z > 0).to(z.dtype)
    if activation == "gelu":
        return normal_below(z) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if activation == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    raise ValueError(activation)


def run_plain(state):
    case = state["case"]
    task, t = case["task"], TYPES[case["dtype"]]
    if task.startswith("linear"):
        x, w = state["x"].float(), state["w"].to(t).float()
        if task == "linear":
            z = x @ w
            if state["bias"] is not None:
                z = z + state["bias"]
            y = activated(case["activation"], z)
            if state["residual"] is not None:
                y = y + state["residual"].float()
            if not case["slope"]:
                return y.to(t)
            return y.to(t), slope_of(case["activation"], z).to(t) if case["activation"] != "none" else None
        dz = state["dy"].float()
        if state["slope"] is not None:               # the operand of both products has the tensors' type
            dz = (dz * state["slope"].float()).to(t).float()
        return (dz @ w.t()).to(t), x.t() @ dz, dz.sum(0)
    s = state["logits"].float()
    labels = state["labels"].long()
    label, has = labels.clamp(min=0)[:, None], labels >= 0
    hot = torch.arange(s.shape[1], device=s.device) == labels[:, None]
    if task == "logprob-gradient":
        logp = s - state["stats"][:, :1] - state["stats"][:, 1:]
        p = torch.exp(logp)
        g = torch.where(has, state["grad_logprob"], 0.0)[:, None]
        ds = -g * torch.where(hot, torch.expm1(logp), p)         # 1 - p of a label that is all but certain
        ds = ds - state["grad_entropy"][:, None] * torch.where(p > 0, p * (logp + state["entropy"][:, None]), 0.0)
        return ds.to(t)
    m = s.amax(1, keepdim=True)
    s0 = s - m
    e1 = torch.exp(s0)
    z1 = e1.sum(1, keepdim=True, dtype=torch.float64)            # next to 1 where a class is all but certain
    lz1 = torch.log(z1)
    mine = s0.gather(1, label)
    logprob = torch.where(has, (mine.double() - lz1)[:, 0], 0.0)
    if task == "logprob":
        entropy = torch.where(e1 > 0, e1 * (lz1.float() - s0), 0.0).sum(1) / z1[:, 0].float()
        its = s.gather(1, label)
        before = (s > its) | ((s == its) & (torch.arange(s.shape[1], device=s.device) < label))
        rank = torch.where(has, before.sum(1), -1).int()
        if not case["top"]:
            return [logprob.float(), entropy, rank]
        value, index = torch.sort(s, dim=1, descending=True, stable=True)
        value, index = value[:, :case["top"]], index[:, :case["top"]]
        return [logprob.float(), entropy, rank, torch.where(value == -math.inf, -1, index).int(), ((value - m).double() - lz1).float()]
    # distill: the list's entries and the label in 64 bits, since there two probabilities are subtracted that may be nearly equal
    classes = s.shape[1]
    absent = state["top_index"] < 0
    index = state["top_index"].long()
    teacher = torch.where(absent, -math.inf, state["top_logit"].double() / TEMPERATURE)
    some = ~absent.all(1, keepdim=True)
    teacher = teacher - torch.where(some, teacher.amax(1, keepdim=True), 0.0)
    e = torch.exp(teacher)
    norm = torch.where(some, e.sum(1, keepdim=True), 1.0)
    p, logp = e / norm, torch.where(absent, 0.0, teacher - torch.log(norm))
    soft = s0 / TEMPERATURE
    eq = torch.exp(soft)
    zq = eq.sum(1, keepdim=True, dtype=torch.float64)
    logq = s0.gather(1, index.clamp(min=0)).double() / TEMPERATURE - torch.log(zq)
    kl = torch.where(p > 0, p * (logp - logq), 0.0).sum(1)
    loss = (1 - HARD_WEIGHT) * TEMPERATURE ** 2 * kl - HARD_WEIGHT * logprob
    ws = torch.where(some, state["row_weight"][:, None] * (1 - HARD_WEIGHT) * TEMPERATURE, 0.0)
    wh = torch.where(has, state["row_weight"] * HARD_WEIGHT, 0.0)[:, None]
    ds = torch.empty(s.shape[0], classes + 1, device=s.device)   # entries that the list does not have go to the last column
    ds[:, :classes] = eq * (ws / zq).float()
    ds.scatter_(1, torch.where(absent, classes, index), torch.where(p > 0, ws * p * torch.expm1(logq - logp), 0.0).float())
    ds = ds[:, :classes] + torch.where(hot, (wh * torch.expm1(logprob)[:, None]).float(), e1 * (wh / z1).float())
    return loss.float(), ds.to(t)


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def work(case):
    s = 2 if case["dtype"] == "bf16" else 4
    if case["task"].startswith("linear"):
        rows, inputs, outputs = sizes(case)
        weights = inputs * outputs * s
        if case["task"] == "linear":
            tensors = 1 + case["residual"] + (case["slope"] and case["activation"] != "none")
            return {"bytes": rows * inputs * s + weights + outputs * 4 * case["bias"] + rows * outputs * s * tensors,
                    "flops": 2 * rows * inputs * outputs}
        tensors = 1 + (case["activation"] != "none")
        return {"bytes": 2 * rows * inputs * s + weights + inputs * outputs * 4 + outputs * 4 + rows * outputs * s * tensors,
                "flops": 4 * rows * inputs * outputs}
    rows, classes, top = case["rows"], case["classes"], case["top"]
    values = rows * classes
    if case["task"] == "logprob":
        return {"bytes": values * s + rows * (16 + 8 * top), "flops": 8 * values}
    if case["task"] == "logprob-gradient":
        return {"bytes": 2 * values * s + rows * 24, "flops": 8 * values}
    return {"bytes": 2 * values * s + rows * (12 + 8 * top), "flops": 12 * values}


# ---- the same from the definitions, in 64 bits -------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["task"].startswith("linear"):
        return exact_linear(case, state)
    s = state["logits"].double()
    label = state["labels"].long()
    every = torch.arange(len(label), device=s.device)
    hot = torch.zeros_like(s)
    hot[every[label >= 0], label[label >= 0]] = 1.0
    if case["task"] == "logprob-gradient":
        # p and log p follow from the statistics that the call is given
        logp = s - state["stats"].double().sum(1, keepdim=True)
        p = logp.exp()
        lp = logp.clamp(min=-1e300)
        g = (state["grad_logprob"].double() * (label >= 0))[:, None]
        return g * hot - g * p - state["grad_entropy"].double()[:, None] * p * (lp + state["entropy"].double()[:, None])
    logp = s - torch.logsumexp(s, 1, keepdim=True)
    picked = torch.where(hot > 0, logp, 0.0).sum(1)
    if case["task"] == "logprob":
        entropy = -(logp.exp() * logp.clamp(min=-1e300)).sum(1)
        out = [picked, entropy, None]
        return out + [None, logp.topk(case["top"], dim=1).values] if case["top"] else out
    index, valid = state["top_index"].long(), state["top_index"] >= 0
    some = valid.any(1)
    teacher = (state["top_logit"].double() / TEMPERATURE).masked_fill(~valid, -1e300)
    logt = teacher - torch.logsumexp(teacher, 1, keepdim=True)
    t = logt.exp() * valid
    logq = s / TEMPERATURE
    logq = logq - torch.logsumexp(logq, 1, keepdim=True)
    wanted = torch.zeros_like(s)
    for j in range(index.shape[1]):
        at = valid[:, j]
        wanted[every[at], index[at, j]] += t[at, j]
    kl = torch.where(valid, t * (logt - logq.gather(1, index.clamp(min=0))), 0.0).sum(1)
    loss = (1 - HARD_WEIGHT) * TEMPERATURE ** 2 * kl - HARD_WEIGHT * picked
    w = state["row_weight"].double()[:, None]
    ds = (1 - HARD_WEIGHT) * TEMPERATURE * (logq.exp() * some[:, None] - wanted)
    ds += HARD_WEIGHT * (logp.exp() * (label >= 0)[:, None] - hot)
    return loss, ds * w


def exact_linear(case, state):
    t = TYPES[case["dtype"]]
    x, w = state["x"].double(), state["w"].to(t).double()
    if case["task"] == "linear":
        z = torch.matmul(x, w)
        if case["bias"]:
            z += state["bias"].double()
        below = torch.special.ndtr(z)
        sigmoid = torch.sigmoid(z)
        y, slope = {
            "none": lambda: (z, None),
            "relu": lambda: (torch.relu(z), (z > 0).double()),
            "gelu": lambda: (z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)),
            "silu": lambda: (z * sigmoid, sigmoid + z * sigmoid * (1 - sigmoid)),
        }[case["activation"]]()
        if case["residual"]:
            y = y + state["residual"].double()
        return (y, slope) if case["slope"] else y
    dz = state["dy"].double()
    if state["slope"] is not None:                   # one rounding of the product, which fp32 and bf16 factors leave exact in 64 bits
        dz = (dz * state["slope"].double()).to(t).double()
    return torch.matmul(dz, w.t()), torch.matmul(x.t(), dz), dz.sum(0)
