"""The operators over a vocabulary that a user of this framework times: drawing a token from an ensemble of
language models, listing its likeliest tokens, distilling those into a student, and the 8-bit head product that
makes the logits.

Logits are those of a language model: a bulk of unlikely tokens and some dozens of likely ones, for answers
with a share of the rows restricted to half of the vocabulary by a mask of -inf.  Every row of a sampling batch has its own
temperature and filters, as the requests of a serving batch do.  Activations have a few large channels.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one request to three image classifiers: the smallest draw, where the launch counts
        dict(name="sample_3x1x1000", op="sample", models=3, n=1, classes=1000, dtype="fp32"),
        # a decoding batch of three small text models over the sentiment models' vocabulary
        dict(name="sample_3x16x30000", op="sample", models=3, n=16, classes=30000, dtype="bf16"),
        # a full decoding batch of one large-vocabulary model with fp32 logits
        dict(name="sample_1x256x131072", op="sample", models=1, n=256, classes=131072, dtype="fp32"),
        # top-5 answers of three image classifiers at the batch that they are served with
        dict(name="topk5_3x64x1000", op="topk", models=3, n=64, classes=1000, dtype="fp32", k=5),
        # alternatives with log-probabilities for a few requests, an odd vocabulary (rows on odd addresses)
        dict(name="topk20_2x7x50021", op="topk", models=2, n=7, classes=50021, dtype="bf16", k=20),
        # a teacher ensemble labels a training batch with its 64 likeliest tokens
        dict(name="topk64_2x1024x131072", op="topk", models=2, n=1024, classes=131072, dtype="bf16", k=64),
        # fine-tuning an image classifier on a teacher's top 5, a tiny batch
        dict(name="distill_8x1000", op="distill", n=8, classes=1000, dtype="fp32", k=5, rest=True),
        # an ordinary distillation step: loss and gradient, the rest of the teacher's mass as one class
        dict(name="distill_4096x30000", op="distill", n=4096, classes=30000, dtype="bf16", k=32, rest=True),
        # a large vocabulary of odd size, the teacher renormalised over its top tokens
        dict(name="distill_2047x131071", op="distill", n=2047, classes=131071, dtype="bf16", k=64, rest=False),
        # the head or a hidden layer for one token
        dict(name="fc_1x4096x4096", op="fc", n=1, c_in=4096, c_out=4096, dtype="bf16", out="fp32", relu=False),
        # VGG-16's first classifier layer at the headline batch
        dict(name="fc_64x25088x4096", op="fc", n=64, c_in=25088, c_out=4096, dtype="fp32", out="fp32", relu=True),
        # the head over a batch of sequences
        dict(name="fc_4096x4096x30000", op="fc", n=4096, c_in=4096, c_out=30000, dtype="bf16", out="bf16", relu=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    op = rng.choice(("sample", "topk", "distill", "fc"))
    dtype = rng.choice(("fp32", "bf16"))
    if op == "fc":
        n, c_in, c_out = _log_int(rng, 1, 4096), _log_int(rng, 64, 25088), _log_int(rng, 16, 30000)
        while 2 * n * c_in * c_out > 1.0e12:
            n = max(1, n // 2)
        return dict(op=op, n=n, c_in=c_in, c_out=c_out, dtype=dtype, out=rng.choice(("fp32", "bf16")),
                    relu=rng.random() < 0.5)
    classes = _log_int(rng, 100, 160000)
    if op == "distill":
        n = min(_log_int(rng, 1, 8192), 130_000_000 // classes)
        return dict(op=op, n=n, classes=classes, dtype=dtype, k=_log_int(rng, 1, min(256, classes)),
                    rest=rng.random() < 0.5)
    models = rng.choice((1, 1, 2, 3, 4))
    n = min(_log_int(rng, 1, 512), 33_000_000 // (models * classes))
    case = dict(op=op, models=models, n=max(1, n), classes=classes, dtype=dtype)
    return dict(case, k=_log_int(rng, 1, 128)) if op == "topk" else case


# ---------------------------------------------------------------- inputs

def _logits(g, shape, dtype, restrict):
    """[..., n, C]: bulk of standard deviation 1.5, up to 64 tokens raised by up to 16 (the same ones for every
    model of an ensemble, by other amounts); restrict: one row in eight masked to half of its classes."""
    n, C = shape[-2:]
    z = torch.randn(shape, generator=g, device="cuda") * 1.5
    likely = torch.randint(0, C, (n, min(64, C)), generator=g, device="cuda").expand(*shape[:-1], -1)
    z.scatter_add_(-1, likely, torch.rand(likely.shape, generator=g, device="cuda") * 16)
    if restrict:
        masked = torch.rand((n, C), generator=g, device="cuda") < 0.5
        masked &= torch.arange(n, device="cuda").view(-1, 1) % 8 == 7
        z.masked_fill_(masked, -math.inf)
    return z.to(DTYPES[dtype])


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "fc":
        n, c_in, c_out = case["n"], case["c_in"], case["c_out"]
        x = torch.randn((n, c_in), generator=g, device="cuda")
        x *= 1 + 7 * (rand(c_in) < 0.01)
        pad = (c_in + 15) // 16 * 16
        w = torch.zeros((c_out, pad), dtype=torch.int8, device="cuda")
        w[:, :c_in] = (torch.randn((c_out, c_in), generator=g, device="cuda") * 32).clamp_(-127, 127).round_()
        return {"x": x.to(DTYPES[case["dtype"]]), "w": w[:, :c_in], "w_scale": 0.0005 + 0.001 * rand(c_out),
                "bias": rand(c_out) - 0.5}
    n, C = case["n"], case["classes"]
    if case["op"] == "distill":
        s = {"logits": _logits(g, (n, C), case["dtype"], False)}
        order = torch.randint(0, C, (n, 1), generator=g, device="cuda")
        stride = 2 * torch.randint(0, (C + 1) // 2, (n, 1), generator=g, device="cuda") + 1
        stride = torch.where(torch.gcd(stride, torch.full_like(stride, C)) == 1, stride, torch.ones_like(stride))
        s["labels"] = ((order + stride * torch.arange(case["k"], device="cuda")) % C).int()
        t = torch.randn((n, case["k"]), generator=g, device="cuda") * 2
        s["logp"] = torch.log_softmax(t, -1) + torch.log(0.7 + 0.29 * rand(n, 1))
        s["grad"] = (rand(n) < 0.9) / n                    # padded positions count for nothing
        return s
    s = {"logits": _logits(g, (case["models"], n, C), case["dtype"], True)}
    if case["op"] == "sample":
        style = torch.arange(n, device="cuda") % 4           # plain; top-k and top-p; top-p; min-p
        s["temperature"] = 0.6 + 0.6 * rand(n)
        s["top_k"] = torch.where(style == 1, 20 + (rand(n) * 80).int(), 0).int()
        s["top_p"] = torch.where((style == 1) | (style == 2), 0.8 + 0.18 * rand(n), 1.0)
        s["min_p"] = torch.where(style == 3, 0.02 + 0.1 * rand(n), 0.0)
        s["uniform"] = rand(n)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    out = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    n = case["n"]
    if case["op"] == "fc":
        pad = (case["c_in"] + 15) // 16 * 16
        s["q"], s["x_scale"] = out(n, pad, t=torch.int8)[:, :case["c_in"]], out(n)
        s["y"] = out(n, case["c_out"], t=DTYPES[case["out"]])
    elif case["op"] == "distill":
        s["loss"], s["d"] = out(n), torch.empty_like(s["logits"])
    else:
        shape = (n, case["k"]) if case["op"] == "topk" else (n,)
        s["out"], s["labels"] = out(*shape), out(*shape, t=torch.int32)
    return s


# ---------------------------------------------------------------- one pass

DISTILL_T = 2.0
REST_MIN = 2.0 ** -20      # a rest of the teacher's mass below this is rounding and counts as none
P_MIN = 2.0 ** -1000       # a class below this counts as having no probability


def _mean_softmax(z, t):
    """Mean over models of softmax(z / t) in 64 bits."""
    z = z.double() / t
    e = torch.exp(z - z.amax(-1, keepdim=True))
    return (e / e.sum(-1, keepdim=True)).mean(0)


def _plain_sample(s):
    C = s["logits"].shape[-1]
    col = lambda v: v.view(-1, 1)  # noqa: E731
    p = _mean_softmax(s["logits"], col(s["temperature"]).double())
    q, order = torch.sort(p, dim=-1, descending=True, stable=True)
    top_k = col(torch.where((s["top_k"] <= 0) | (s["top_k"] > C), C, s["top_k"]))
    q = torch.where(torch.arange(C, device=q.device) < top_k, q, 0.0)
    run_sum = torch.cumsum(q, -1)
    keep = (run_sum - q < col(s["top_p"]).double() * run_sum[:, -1:]) & (q >= col(s["min_p"]).double() * q[:, :1])
    keep &= q > P_MIN
    p = torch.where(torch.zeros_like(keep).scatter_(-1, order, keep), p, 0.0)
    run_sum = torch.cumsum(p, -1)
    total = run_sum[:, -1:]
    label = (run_sum <= col(s["uniform"]).double() * total).sum(-1, keepdim=True)
    return {"labels": label[:, 0].int(), "probs": (p.gather(-1, label) / total)[:, 0].float()}


def _plain_topk(s):
    p, order = torch.sort(_mean_softmax(s["logits"], 1.0), dim=-1, descending=True, stable=True)
    k = s["case"]["k"]
    pad = max(0, k - p.shape[-1])
    p = torch.nn.functional.pad(p[:, :k], (0, pad))
    order = torch.nn.functional.pad(order[:, :k], (0, pad))
    return {"labels": torch.where(p > P_MIN, order, -1).int(),
            "logp": torch.where(p > P_MIN, torch.log(p), -math.inf).float()}


def _plain_distill(s):
    T, case = DISTILL_T, s["case"]
    ids = s["labels"].long()
    z = s["logits"].float() / T
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    p = e / e.sum(-1, keepdim=True)
    lse = top + torch.log(e.sum(-1, keepdim=True))
    q = torch.exp(s["logp"])
    log_q, log_p = s["logp"], z.gather(-1, ids) - lse
    if case["rest"]:
        q_r = 1 - q.sum(-1, keepdim=True)
        q_r = torch.where(q_r < REST_MIN, 0.0, q_r)
        others = e.scatter(-1, ids, 0.0).sum(-1, keepdim=True)
        log_pr = top + torch.log(others) - lse
        scale = torch.where(others > 0, q_r / torch.exp(log_pr), 0.0)
        d = p * ((q.sum(-1, keepdim=True) + q_r) - scale)
        d.scatter_(-1, ids, p.gather(-1, ids) * (q.sum(-1, keepdim=True) + q_r))
        rest = torch.where(q_r > 0, q_r * (torch.log(q_r) - log_pr), 0.0)[:, 0]
    else:
        q = q / q.sum(-1, keepdim=True)
        log_q = torch.log(q)
        d, rest = p, 0.0
    loss = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(-1) + rest
    d = d.scatter_add(-1, ids, -q) * (T * s["grad"].view(-1, 1))
    return {"loss": T * T * loss, "grad": d.to(s["logits"].dtype)}


def _plain_fc(s):
    x = s["x"].float()
    scale = x.abs().amax(-1, keepdim=True) / 127
    q = torch.round(x.double() / scale).float()           # next to a half, 32 bits decide otherwise
    y = (q @ s["w"].float().t()) * (scale * s["w_scale"]) + s["bias"]
    return {"y": (y.clamp(min=0) if s["case"]["relu"] else y).to(s["y"].dtype)}


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"sample": _plain_sample, "topk": _plain_topk, "distill": _plain_distill, "fc": _plain_fc}[op](s)
    from paper_1804_06087_amd import binding
    if op == "sample":
        binding.combine_sample(s["logits"], s["uniform"], s["labels"], s["out"], temperature=s["temperature"],
                               top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"labels": s["labels"], "probs": s["out"]}
    if op == "topk":
        binding.combine_topk(s["logits"], s["labels"], s["out"])
        return {"labels": s["labels"], "logp": s["out"]}
    if op == "distill":
        binding.distill_loss(s["logits"], s["labels"], s["logp"], s["loss"], s["d"], grad_loss=s["grad"],
                             temperature=DISTILL_T, rest=s["case"]["rest"])
        return {"loss": s["loss"], "grad": s["d"]}
    binding.quantize_rows_i8(s["x"], s["q"], s["x_scale"])
    binding.fc_i8(s["q"], s["x_scale"], s["w"], s["w_scale"], s["y"], bias=s["bias"], relu=s["case"]["relu"])
    return {"y": s["y"]}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    item = 4 if case["dtype"] == "fp32" else 2
    n = case["n"]
    if case["op"] == "fc":
        c_in, c_out = case["c_in"], case["c_out"]
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": n * c_in * item + c_out * c_in + 8 * c_out + n * c_out * out, "flops": 2 * n * c_in * c_out}
    if case["op"] == "distill":
        return {"bytes": 2 * n * case["classes"] * item + n * (8 * case["k"] + 8), "flops": 0}
    values = case["models"] * n * case["classes"]
    extra = 8 * n * case["k"] if case["op"] == "topk" else 28 * n
    return {"bytes": values * item + extra, "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits, from the definitions

def _combined(z, t):
    """The combined distribution by logarithms of sums, one model after another."""
    p = torch.zeros(z.shape[1:], dtype=torch.float64, device=z.device)
    for m in range(z.shape[0]):
        p += torch.exp(z[m].double() / t - torch.logsumexp(z[m].double() / t, -1, keepdim=True)) / z.shape[0]
    return p


def _exact_sample(case, s):
    p = _combined(s["logits"], s["temperature"].double().view(-1, 1)).cpu().numpy()
    host = {k: s[k].cpu().numpy() for k in ("top_k", "top_p", "min_p", "uniform")}
    labels, probs = [], []
    for i, row in enumerate(p):
        order = np.argsort(-row, kind="stable")
        if host["top_k"][i] > 0:
            order = order[:host["top_k"][i]]
        reached = np.cumsum(row[order])
        if host["top_p"][i] < 1:
            order = order[:1 + int(np.searchsorted(reached, float(host["top_p"][i]) * reached[-1], side="left"))]
        order = order[row[order] >= float(host["min_p"][i]) * row[order[0]]]
        order = np.sort(order[row[order] > P_MIN])
        at = np.cumsum(row[order])
        j = order[int(np.searchsorted(at, float(host["uniform"][i]) * at[-1], side="right"))]
        labels.append(j)
        probs.append(row[j] / at[-1])
    return {"labels": torch.tensor(labels, dtype=torch.int32), "probs": torch.tensor(probs, dtype=torch.float64)}


def _exact_topk(case, s):
    n, k = case["n"], case["k"]
    labels = np.full((n, k), -1, np.int32)
    logp = np.full((n, k), -np.inf)
    for i in range(n):
        row = _combined(s["logits"][:, i:i + 1], 1.0)[0]
        least = torch.topk(row, min(k, row.numel())).values[-1].clamp(min=P_MIN)
        at = torch.nonzero(row >= least)[:, 0].cpu().numpy()
        v = row[row >= least].cpu().numpy()
        best = np.lexsort((at, -v))[:k]
        labels[i, :best.size], logp[i, :best.size] = at[best], np.log(v[best])
    return {"labels": torch.from_numpy(labels), "logp": torch.from_numpy(logp)}


def _exact_distill(case, s):
    """By the derivative of log p of each teacher's class and of the rest, a few rows at a time."""
    T, step = DISTILL_T, 256
    losses, grads = [], []
    for at in range(0, case["n"], step):
        z = s["logits"][at:at + step].double() / T
        ids, log_q = s["labels"][at:at + step].long(), s["logp"][at:at + step].double()
        if not case["rest"]:
            log_q = log_q - torch.logsumexp(log_q, -1, keepdim=True)
        q = torch.exp(log_q)
        log_p = z - torch.logsumexp(z, -1, keepdim=True)
        loss = (q * (log_q - log_p.gather(-1, ids)))
        loss = torch.where(q > 0, loss, 0.0).sum(-1)
        target = torch.zeros_like(z).scatter_add_(-1, ids, q)
        if case["rest"]:
            q_r = 1 - q.sum(-1, keepdim=True)
            q_r = torch.where(q_r < REST_MIN, 0.0, q_r)
            outside = log_p.scatter(-1, ids, -math.inf)
            log_pr = torch.logsumexp(outside, -1, keepdim=True)
            loss += torch.where(q_r > 0, q_r * (torch.log(q_r) - log_pr), 0.0)[:, 0]
            share = torch.exp(outside - log_pr)
            target += torch.where(torch.isfinite(log_pr), q_r * share, 0.0)
        d = torch.exp(log_p) * target.sum(-1, keepdim=True) - target
        losses.append(T * T * loss)
        grads.append((T * s["grad"][at:at + step].double().view(-1, 1) * d))
    return {"loss": torch.cat(losses), "grad": torch.cat(grads)}


def _exact_fc(case, s):
    x = s["x"].double()
    scale = (x.abs().amax(-1, keepdim=True) / 127).float().double()
    q = torch.round(x / scale)
    y = torch.empty((case["n"], case["c_out"]), dtype=torch.float64, device=x.device)
    for at in range(0, case["c_out"], 4096):
        y[:, at:at + 4096] = q @ s["w"][at:at + 4096].double().t().contiguous()
    y = y * scale * s["w_scale"].double() + s["bias"].double()
    return {"y": torch.relu(y) if case["relu"] else y}


def exact(case, seed):
    s = _inputs(case, seed)
    return {"sample": _exact_sample, "topk": _exact_topk, "distill": _exact_distill, "fc": _exact_fc}[case["op"]](case, s)
