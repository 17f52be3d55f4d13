"""The operators that a user of this framework times who trains a language model on its own answers and serves its
head in 4 bits: the log-probabilities of given tokens, a clipped policy loss, a preference loss over pairs of answers, and
the head product in microscaled 4-bit floating point.

Logits are those of a language model: a bulk of unlikely tokens and some dozens of likely ones.  Tokens are mostly likely
ones, as drawn answers are; one in seven positions is a prompt's or padding's and has no token (-1).  Old and reference
policies are near the present one.  Activations have a few large channels.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
TEMPERATURE = 0.9
CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.05
BETA, SMOOTHING = 0.1, 0.02


def listed():
    return [
        # one answer of an image classifier: the smallest call, where the launch counts
        dict(name="logp_1x1000", op="logp", n=1, classes=1000, dtype="fp32", entropy=False, grad=False),
        # backward of a loss of the user's own over a small batch, odd vocabulary (rows on odd addresses)
        dict(name="logp_grad_777x30001", op="logp", n=777, classes=30001, dtype="fp32", entropy=True, grad=True),
        # a reference model's log-probabilities and entropies over a training batch, large vocabulary
        dict(name="logp_8192x131072", op="logp", n=8192, classes=131072, dtype="bf16", entropy=True, grad=False),
        # an ordinary policy step over the sentiment models' vocabulary, with an entropy bonus
        dict(name="policy_4096x30000", op="policy", n=4096, classes=30000, dtype="bf16", entropy=0.01),
        # a policy step with fp32 logits and an odd vocabulary, without the bonus
        dict(name="policy_1500x50021", op="policy", n=1500, classes=50021, dtype="fp32", entropy=0.0),
        # two pairs of short answers over an image classifier's classes: latency
        dict(name="preference_2x5x1000", op="preference", pairs=2, length=5, classes=1000, dtype="fp32", mean=False),
        # an ordinary preference step, ragged answers
        dict(name="preference_8x250x30000", op="preference", pairs=8, length=250, classes=30000, dtype="bf16", mean=False),
        # a large odd vocabulary and long answers, scores by the token
        dict(name="preference_3x1000x131071", op="preference", pairs=3, length=1000, classes=131071, dtype="bf16", mean=True),
        # the head or a hidden layer for one token
        dict(name="fc4_1x4096x4096", op="fc", n=1, c_in=4096, c_out=4096, dtype="bf16", out="fp32", relu=False, fresh=False),
        # VGG-16's first classifier layer at the headline batch
        dict(name="fc4_64x25088x4096", op="fc", n=64, c_in=25088, c_out=4096, dtype="fp32", out="fp32", relu=True, fresh=False),
        # a head in training: its weights have moved and are quantised again, odd sizes
        dict(name="fc4_1000x2050x30001", op="fc", n=1000, c_in=2050, c_out=30001, dtype="bf16", out="bf16", relu=False, fresh=True),
        # the head over a batch of sequences
        dict(name="fc4_4096x4096x30000", op="fc", n=4096, c_in=4096, c_out=30000, dtype="bf16", out="bf16", relu=False, fresh=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    op = rng.choice(("logp", "policy", "preference", "fc"))
    dtype = rng.choice(("fp32", "bf16"))
    if op == "fc":
        n, c_in, c_out = _log_int(rng, 1, 4096), _log_int(rng, 64, 25088), _log_int(rng, 16, 30000)
        while 2 * n * c_in * c_out > 1.0e12:
            n = max(1, n // 2)
        return dict(op=op, n=n, c_in=c_in, c_out=c_out, dtype=dtype, out=rng.choice(("fp32", "bf16")),
                    relu=rng.random() < 0.5, fresh=rng.random() < 0.3)
    classes = _log_int(rng, 100, 160000)
    if op == "preference":
        pairs = _log_int(rng, 1, 64)
        length = min(_log_int(rng, 1, 1000), max(1, 120_000_000 // (2 * pairs * classes)))
        return dict(op=op, pairs=pairs, length=length, classes=classes, dtype=dtype, mean=rng.random() < 0.5)
    n = min(_log_int(rng, 1, 8192), 130_000_000 // classes)
    if op == "policy":
        return dict(op=op, n=n, classes=classes, dtype=dtype, entropy=rng.choice((0.0, 0.01)))
    return dict(op=op, n=n, classes=classes, dtype=dtype, entropy=rng.random() < 0.5, grad=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _offsets(case):
    """First rows of the sequences (chosen, rejected, chosen, ...): lengths of half to one and a half times the mean."""
    spread = torch.arange(2 * case["pairs"], dtype=torch.float64) * 0.6180339887 % 1
    length = (case["length"] * (0.5 + spread)).round().clamp(min=1).to(torch.int32)
    return torch.cat([torch.zeros(1, dtype=torch.int32), length.cumsum(0).to(torch.int32)])


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "fc":
        n, c_in, c_out = case["n"], case["c_in"], case["c_out"]
        x = randn(n, c_in) * (1 + 7 * (rand(c_in) < 0.01))
        s = {"x": x.to(DTYPES[case["dtype"]]), "bias": rand(c_out) - 0.5}
        if case["fresh"]:
            s["w"] = (randn(c_out, c_in) * 0.02).to(DTYPES[case["dtype"]])
            return s
        blocks = (c_in + 31) // 32                           # rows of whole blocks, zeros behind c_in
        s["wq"] = torch.randint(0, 256, (c_out, 16 * blocks), generator=g, device="cuda", dtype=torch.uint8)
        if c_in % 32:
            s["wq"][:, (c_in + 1) // 2:] = 0
            if c_in % 2:
                s["wq"][:, c_in // 2] &= 15
        pad = torch.zeros((c_out, (blocks + 15) // 16 * 16), dtype=torch.uint8, device="cuda")
        pad[:, :blocks] = 127 - torch.randint(6, 10, (c_out, blocks), generator=g, device="cuda")
        s["w_scale"] = pad[:, :blocks]
        return s
    C = case["classes"]
    s = {}
    if case["op"] == "preference":
        offsets = _offsets(case)
        n = int(offsets[-1])
        s["offsets"] = offsets.cuda()
    else:
        n = case["n"]
    z = randn(n, C) * 1.5
    k = min(64, C)                                           # likely tokens, no two of a row alike
    likely = (torch.randint(0, C, (n, 1), generator=g, device="cuda") + C // k * torch.arange(k, device="cuda")) % C
    z.scatter_add_(-1, likely, rand(n, k) * 16)
    s["logits"] = z.to(DTYPES[case["dtype"]])
    del z
    anywhere = torch.randint(0, C, (n,), generator=g, device="cuda")
    labels = torch.where(rand(n) < 0.9, likely[:, 0], anywhere)
    s["labels"] = torch.where((rand(n) < 1 / 7) & (torch.arange(n, device="cuda") > 0), -1, labels).int()
    # log-probabilities near which the old and the reference policy's lie
    logp = torch.empty(n, dtype=torch.float64, device="cuda")
    for at in range(0, n, 1024):
        x = s["logits"][at:at + 1024].double() / TEMPERATURE
        logp[at:at + 1024] = (x.gather(-1, labels[at:at + 1024].view(-1, 1))[:, 0] - torch.logsumexp(x, -1))
    if case["op"] == "preference":
        drift = torch.zeros(n, device="cuda")                # of a sequence's tokens, likelier by now or less likely
        drift[offsets[:-1].long().cuda()] = 1
        drift = (0.05 * randn(2 * case["pairs"]))[drift.cumsum(0).long() - 1]
        s["ref"] = (logp + drift + 0.3 * randn(n)).float()
        s["weight"] = 0.5 + rand(case["pairs"])
    elif case["op"] == "policy":
        step = 0.2 * randn(n).double()
        for border in (1 - CLIP_LOW, 1 + CLIP_HIGH):         # no ratio where the last bit of logp decides
            step = torch.where((step - math.log(border)).abs() < 1e-4, math.log(border) + 2e-4, step)
        s["old"] = (logp - step).float()
        s["ref"] = (logp + 0.5 * randn(n)).float()
        s["advantage"] = randn(n)
        s["weight"] = (s["labels"] >= 0) / n
    elif case["grad"]:
        s["g_logp"], s["g_entropy"] = randn(n), 0.1 * randn(n)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    out = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731

    def mx4(n, c):
        blocks = (c + 31) // 32
        return out(n, 16 * blocks, t=torch.uint8), out(n, (blocks + 15) // 16 * 16, t=torch.uint8)[:, :blocks]

    if case["op"] == "fc":
        s["xq"], s["x_scale"] = mx4(case["n"], case["c_in"])
        if case["fresh"]:
            s["wq"], s["w_scale"] = mx4(case["c_out"], case["c_in"])
        s["y"] = out(case["n"], case["c_out"], t=DTYPES[case["out"]])
        return s
    n = s["logits"].shape[0]
    if case["op"] == "preference":
        s["loss"], s["scores"] = out(case["pairs"]), out(case["pairs"], 2)
    else:
        s["loss"], s["logp"], s["kl"] = out(n), out(n), out(n)
        s["h"] = out(n) if case["entropy"] else None
    if case["op"] != "logp" or case["grad"]:
        s["d"] = torch.empty_like(s["logits"])
    return s


# ---------------------------------------------------------------- one pass

def _softmax(z, labels, dtype=torch.float32):
    """(valid [n], the label's index [n, 1], its log p fp64 [n], p, log p) of rows of logits; log p of the label in
    64 bits, since what follows compares and subtracts it."""
    x = z.to(dtype) / TEMPERATURE
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    valid = labels >= 0
    at = torch.where(valid, labels, 0).long().view(-1, 1)
    logp = z.gather(-1, at).double() / TEMPERATURE - (top.double() + torch.log(total))
    return valid, at, logp[:, 0], e / total.to(dtype), (x - top) - torch.log(total).to(dtype)


def _minus_p(p, at, valid, g):
    """g (1[c = label] - p) / T, 0 in rows without a label."""
    g = torch.where(valid, g, 0.0).view(-1, 1)
    return (p * -g).scatter_add_(-1, at, g) / TEMPERATURE


def _plain_logp(s):
    case = s["case"]
    valid, at, logp, p, log_p = _softmax(s["logits"], s["labels"])
    out = {"logp": torch.where(valid, logp, 0.0).float()}
    if case["entropy"]:
        H = -(p * log_p).sum(-1)
        out["entropy"] = torch.where(valid, H, 0.0)
    if case["grad"]:
        d = _minus_p(p, at, valid, s["g_logp"])
        if case["entropy"]:
            d -= torch.where(valid, s["g_entropy"], 0.0).view(-1, 1) * p * (log_p + H.view(-1, 1)) / TEMPERATURE
        out["grad"] = d.to(s["logits"].dtype)
    return out


def _plain_policy(s):
    valid, at, logp, p, log_p = _softmax(s["logits"], s["labels"])
    A, eta = s["advantage"].double(), s["case"]["entropy"]
    ratio = torch.exp(logp - s["old"].double())
    plain, clipped = ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
    d = s["ref"].double() - logp
    kl = torch.expm1(d) - d
    loss = KL_COEF * kl - torch.minimum(plain, clipped)
    coef = torch.where(plain <= clipped, -plain, 0.0) - KL_COEF * torch.expm1(d)
    grad = _minus_p(p, at, valid, (coef * s["weight"]).float())
    out = {"logp": torch.where(valid, logp, 0.0).float(), "kl": torch.where(valid, kl, 0.0).float()}
    if eta:
        H = -(p * log_p).sum(-1)
        out["entropy"] = torch.where(valid, H, 0.0)
        loss = loss - eta * H
        weight = torch.where(valid, eta * s["weight"], 0.0).view(-1, 1)
        grad += weight * p * (log_p + H.view(-1, 1)) / TEMPERATURE
    return {"loss": torch.where(valid, loss, 0.0).float(), **out, "grad": grad.to(s["logits"].dtype)}


def _plain_preference(s):
    valid, at, logp, p, _ = _softmax(s["logits"], s["labels"], torch.float64)   # a score sums small differences
    first = s["offsets"].long()
    n, sequences = logp.shape[0], first.numel() - 1
    which = torch.bucketize(torch.arange(n, device=logp.device), first[1:], right=True)
    zero = torch.zeros(sequences, dtype=torch.float64, device=logp.device)
    score = zero.index_add(0, which, torch.where(valid, logp - s["ref"].double(), 0.0))
    per_token = torch.ones_like(score)
    if s["case"]["mean"]:
        per_token = 1 / zero.index_add(0, which, valid.double()).clamp(min=1)
    score = BETA * score * per_token
    u = score[0::2] - score[1::2]
    soft = torch.log1p(torch.exp(-u.abs()))
    loss = (1 - SMOOTHING) * (soft + (-u).clamp(min=0)) + SMOOTHING * (soft + u.clamp(min=0))
    du = s["weight"].double() * (SMOOTHING * torch.sigmoid(u) - (1 - SMOOTHING) * torch.sigmoid(-u))
    coef = BETA * per_token * torch.stack([du, -du], 1).view(-1)
    grad = _minus_p(p, at, valid, coef[which])
    return {"loss": loss.float(), "scores": score.view(-1, 2).float(), "grad": grad.to(s["logits"].dtype)}


def _plain_mx4(x):
    """The values that rows in 4 bits stand for: exact in 32 bits but for the last power of a very small block."""
    n, c = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -c % 32)).view(n, -1, 32)
    _, e = torch.frexp(v.abs().amax(-1, keepdim=True))       # max = m 2^e, 0.5 <= m < 1
    e = (e - 3).clamp(-127, 127)
    v = torch.ldexp(v, -e)
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0))
    return torch.ldexp((torch.round(v / step) * step).clamp(-6, 6), e).view(n, -1)


def _values(codes, scale):
    """What codes (two in a byte, the even one in the low half) and scales 2^(byte - 127) stand for."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).view(codes.shape[0], -1, 32)
    return torch.ldexp(v, (scale.int() - 127).unsqueeze(-1)).view(codes.shape[0], -1)


def _plain_fc(s):
    w = _plain_mx4(s["w"]) if s["case"]["fresh"] else _values(s["wq"], s["w_scale"])
    y = _plain_mx4(s["x"]) @ w.t() + s["bias"]
    return {"y": (y.clamp(min=0) if s["case"]["relu"] else y).to(s["y"].dtype)}


def run(state):
    s = state
    case = s["case"]
    op = case["op"]
    if not own:
        return {"logp": _plain_logp, "policy": _plain_policy, "preference": _plain_preference, "fc": _plain_fc}[op](s)
    from paper_1804_06087_amd import binding
    if op == "logp":
        out = {"logp": s["logp"]}
        if case["entropy"]:
            out["entropy"] = s["h"]
        grad = {}
        if case["grad"]:
            out["grad"] = s["d"]
            grad = dict(grad_logits=s["d"], grad_logp=s["g_logp"], grad_entropy=s["g_entropy"] if case["entropy"] else None)
        binding.token_logp(s["logits"], s["labels"], s["logp"], s["h"], temperature=TEMPERATURE, **grad)
        return out
    if op == "policy":
        binding.policy_loss(s["logits"], s["labels"], s["advantage"], s["loss"], s["d"], old_logp=s["old"],
                            ref_logp=s["ref"], grad_loss=s["weight"], out_logp=s["logp"], out_kl=s["kl"],
                            out_entropy=s["h"], temperature=TEMPERATURE, clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                            kl_coef=KL_COEF, entropy_coef=case["entropy"])
        out = {"loss": s["loss"], "logp": s["logp"], "kl": s["kl"]}
        if case["entropy"]:
            out["entropy"] = s["h"]
        return {**out, "grad": s["d"]}
    if op == "preference":
        binding.preference_loss(s["logits"], s["labels"], s["loss"], s["d"], offsets=s["offsets"], ref_logp=s["ref"],
                                grad_loss=s["weight"], out_scores=s["scores"], temperature=TEMPERATURE, beta=BETA,
                                smoothing=SMOOTHING, mean=case["mean"])
        return {"loss": s["loss"], "scores": s["scores"], "grad": s["d"]}
    if case["fresh"]:
        binding.quantize_rows_mx4(s["w"], s["wq"], s["w_scale"])
    binding.quantize_rows_mx4(s["x"], s["xq"], s["x_scale"])
    binding.fc_mx4(s["xq"], s["x_scale"], s["wq"], s["w_scale"], s["y"], bias=s["bias"], relu=case["relu"])
    return {"y": s["y"]}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    item = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "fc":
        n, c_in, c_out = case["n"], case["c_in"], case["c_out"]
        w = c_in * item if case["fresh"] else c_in * 17 / 32    # 16 bytes of codes and one of scale for 32 values
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": n * c_in * item + c_out * (w + 4) + n * c_out * out, "flops": 2 * n * c_in * c_out}
    if case["op"] == "preference":
        n = int(_offsets(case)[-1])
        return {"bytes": n * (2 * case["classes"] * item + 8) + 24 * case["pairs"], "flops": 0}
    n = case["n"]
    if case["op"] == "policy":
        return {"bytes": n * (2 * case["classes"] * item + 36), "flops": 0}
    return {"bytes": n * ((2 if case["grad"] else 1) * case["classes"] * item + 16), "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits, from the definitions

def _exact_tokens(case, s):
    """By autograd in 64 bits of the loss as it is written, some rows at a time; a pair's rows by the chain rule over
    its score."""
    z, ids = s["logits"], s["labels"].long()
    n = z.shape[0]
    step = max(1, (1 << 25) // z.shape[1])
    host = {k: [] for k in ("loss", "logp", "kl", "entropy", "grad")}
    valid = ids >= 0

    def log_softmax(at, wanted):
        x = z[at:at + step].double().requires_grad_(wanted)
        rows = torch.log_softmax(x / TEMPERATURE, -1)
        return x, rows, rows.gather(-1, ids[at:at + step].clamp(min=0).view(-1, 1))[:, 0] * valid[at:at + step]

    def grad_of(total, x):
        return torch.autograd.grad(total, x)[0]

    if case["op"] == "preference":
        with torch.no_grad():
            logp = torch.cat([log_softmax(at, False)[2] for at in range(0, n, step)])
        logp.requires_grad_(True)
        first = s["offsets"].tolist()
        losses, scores = [], []
        for i in range(case["pairs"]):
            r = []
            for a, b in ((first[2 * i], first[2 * i + 1]), (first[2 * i + 1], first[2 * i + 2])):
                v = (logp[a:b] - s["ref"][a:b].double())[valid[a:b]].sum()
                r.append(BETA * v / max(1, int(valid[a:b].sum())) if case["mean"] else BETA * v)
            u = r[0] - r[1]
            losses.append(-(1 - SMOOTHING) * torch.nn.functional.logsigmoid(u) - SMOOTHING * torch.nn.functional.logsigmoid(-u))
            scores.append(torch.stack(r))
        loss, scores = torch.stack(losses), torch.stack(scores)
        g = grad_of((loss * s["weight"].double()).sum(), logp)
        for at in range(0, n, step):
            x, _, part = log_softmax(at, True)
            host["grad"].append(grad_of((part * g[at:at + step]).sum(), x))
        return {"loss": loss.detach(), "scores": scores.detach(), "grad": torch.cat(host["grad"])}
    wanted = case["op"] == "policy" or case["grad"]
    for at in range(0, n, step):
        v = valid[at:at + step]
        cut = lambda k: s[k][at:at + step].double()  # noqa: E731
        with torch.set_grad_enabled(wanted):
            x, rows, logp = log_softmax(at, wanted)
            total = 0.0
            H = -(torch.exp(rows) * rows).sum(-1) * v
            if case["op"] == "policy":
                ratio = torch.exp(logp - cut("old"))
                d = cut("ref") - logp
                kl = torch.exp(d) - d - 1
                gain = torch.minimum(ratio * cut("advantage"), torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * cut("advantage"))
                loss = (KL_COEF * kl - gain) * v - case["entropy"] * H
                host["kl"].append((kl * v).detach())
                host["loss"].append(loss.detach())
                total = (loss * cut("weight")).sum()
            elif wanted:
                total = (logp * cut("g_logp")).sum()
                if case["entropy"]:
                    total = total + (H * cut("g_entropy")).sum()
            if wanted:
                host["grad"].append(grad_of(total, x))
        host["logp"].append(logp.detach())
        if case["entropy"]:
            host["entropy"].append(H.detach())
    return {k: torch.cat(v) for k, v in host.items() if v}


def _exact_mx4(x):
    """The nearest of the 15 values on each side, a tie to the even code, by distances in 64 bits."""
    n, c = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -c % 32)).view(n, -1, 32)
    top = v.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = torch.where(torch.exp2(e) > top, e - 1, torch.where(torch.exp2(e + 1) <= top, e + 1, e))
    scale = torch.exp2((e - 2).clamp(-127, 127))
    u = (v / scale).abs()
    best, at = torch.full_like(u, math.inf), torch.zeros_like(u)
    for value in (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):   # even codes first, and kept in a tie
        near = (u - value).abs()
        at = torch.where(near < best, value, at)
        best = torch.minimum(near, best)
    return (torch.sign(v) * at * scale).view(n, -1)


def _exact_fc(case, s):
    x = _exact_mx4(s["x"])
    y = torch.empty((case["n"], case["c_out"]), dtype=torch.float64, device=x.device)
    code = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    for at in range(0, case["c_out"], 2048):
        if case["fresh"]:
            w = _exact_mx4(s["w"][at:at + 2048])
        else:
            q = s["wq"][at:at + 2048].int()
            w = torch.empty((q.shape[0], 2 * q.shape[1]), dtype=torch.float64, device=x.device)
            for j in (0, 1):
                nibble = (q >> (4 * j)) % 16
                w[:, j::2] = code[nibble % 8] * (1 - 2 * (nibble // 8))
            w = w * torch.exp2(s["w_scale"][at:at + 2048].double() - 127).repeat_interleave(32, 1)
        y[:, at:at + 2048] = x @ w.t().contiguous()
    y += s["bias"].double()
    return {"y": torch.relu(y) if case["relu"] else y}


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_fc(case, s) if case["op"] == "fc" else _exact_tokens(case, s)
