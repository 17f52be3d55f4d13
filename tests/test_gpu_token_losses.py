"""The losses over given tokens on the GPU against the 64-bit oracle: log-probabilities with entropies and their
gradient, the clipped policy loss, the preference loss; at odd sizes, strides, masks and special values, on other
streams, in replayed graphs, and chained with the 4-bit head product and the draw as a training program chains them."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as ot
from paper_1804_06087_amd import RafikiError
from paper_1804_06087_amd import binding as bd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}       # relative rounding error of a stored value


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def full(*shape, dtype=torch.float32):
    return torch.full(shape, -7, dtype=dtype, device=DEV)


def lm_rows(rng, n, C, dtype):
    """Logits [n, C] with a bulk of unlikely classes and some likely ones, and labels, most of them likely; the second
    of every four rows has no token from the fifth row on."""
    z = rng.standard_normal((n, C)) * 1.5
    labels = np.zeros(n, np.int32)
    for i in range(n):
        likely = rng.integers(0, C, min(20, C))
        z[i, likely] += rng.random(likely.size) * 12
        labels[i] = likely[0] if i % 3 else rng.integers(0, C)
        if i % 4 == 1 and i > 4:
            labels[i] = (-1, C, -2 ** 31, 2 ** 31 - 1)[i // 4 % 4]
    return torch.from_numpy(z.astype(np.float32)).to(DT[dtype]), labels


# What 32 bits lose of one row.  A power 2^x, x = (z - top) s, is off by 2^-23 |x| ln 2 (the product and s are rounded)
# and a few units in its own last place; a sum of C of them in runs of at most max(200, C / 1024) and trees by as many 2^-24.
def sum_error(z, y, t):
    x = np.delete(np.asarray(z, np.float64) / t, y)
    x = x[x > -np.inf]
    if not x.size:
        return 2.0 ** -20
    w = np.exp(x - x.max())
    mean_x = (w * (x.max() - x)).sum() / w.sum()
    return (200 + len(z) / 1024) * 2.0 ** -24 + 2.0 ** -22 * (mean_x + 4)


class Bounds:
    """Limits of one row's errors, from its exact values."""

    def __init__(self, z, y, t):
        facts = ot.token_facts(z, y, t)
        self.defined = facts is not None
        if not self.defined:
            return
        self.logp, self.H, self.p, self.log_p = facts
        e = self.eps = sum_error(z, y, t)
        # log p = - log(1 + R): only the others' sum is rounded
        rest = np.delete(self.p, y).sum()
        self.d_logp = e * min(1.0, rest * 2) + 2.0 ** -23 * abs(self.logp) if self.logp > -np.inf else 0.0
        fin = self.p > 0
        self.x = np.where(fin, self.log_p - self.log_p.max(), 0.0)
        spread = (self.p * np.abs(self.x)).sum()
        self.d_H = 4 * e * (1 + self.H + spread)

    def grad(self, t, a, h, da, want, dtype):
        """da: how far a may be off."""
        log_p = np.where(self.p > 0, self.log_p, 0.0)
        inner = abs(a) + abs(h) * (np.abs(log_p) + self.H)
        rel = 2 * self.eps + 2.0 ** -22 * (np.abs(self.x) + 8)
        lost = self.p * (inner * rel + da + abs(h) * (self.d_H + 2.0 ** -20 * (np.abs(log_p) + 1)))
        return lost, np.abs(want) * HALF_STEP[dtype] + 1e-37 * (inner + 1) / t

    def check_grad(self, got, z, y, t, a, h, da, dtype, what):
        want = ot.token_grad(z, y, t, a, h)
        if np.isnan(want).any():
            assert np.isnan(got).all(), what
            return
        lost, kept = self.grad(t, a, h, da, want, dtype)
        rest = np.delete(self.p, y).sum()                    # the label's own: a (1 - p)
        lost[y] += (abs(a) * (2 * self.eps + 2.0 ** -20) + da) * rest
        bad = ~(np.abs(got - want) <= lost / t * (1 + HALF_STEP[dtype]) + kept)
        assert not bad.any(), (what, np.nonzero(bad)[0][:5], got[bad][:5], want[bad][:5])


def near(got, want, limit, what):
    if abs(want) > 3.4028235677973366e38:                     # beyond fp32
        want = math.copysign(math.inf, want)
    assert got == want or (math.isnan(got) and math.isnan(want)) or abs(got - want) <= limit, (what, got, want, limit)


# ---------------------------------------------------------------- log-probabilities

def run_logp(z, labels, t, a=None, h=None, logp=True, entropy=True, grad=True, **kw):
    n = z.shape[0]
    out = (full(n) if logp else None, full(n) if entropy else None,
           torch.full(z.shape, -7, dtype=z.dtype, device=DEV) if grad else None)
    bd.token_logp(z, dev(labels), out[0], out[1], out[2], None if a is None else dev(a), None if h is None else dev(h),
                  temperature=t, **kw)
    torch.cuda.synchronize()
    return out


def check_logp(z, labels, t, a, h, out, dtype):
    zh = host(z)
    for i in range(len(labels)):
        y, ai, hi = int(labels[i]), 0.0 if a is None else float(a[i]), 0.0 if h is None else float(h[i])
        token = 0 <= y < zh.shape[1]
        b = Bounds(zh[i], y, t) if token else None
        if out[0] is not None:
            near(float(out[0][i]), 0.0 if not token else b.logp if b.defined else math.nan,
                 b.d_logp + 2.0 ** -149 if token and b.defined else 0, ("logp", i))
        if out[1] is not None:
            near(float(out[1][i]), 0.0 if not token else b.H if b.defined else math.nan, b.d_H if token and b.defined else 0,
                 ("entropy", i))
        if out[2] is not None:
            got = host(out[2][i])
            if not token or (ai == 0 and hi == 0):
                assert (got == 0).all(), i
            elif not b.defined:
                assert np.isnan(got).all(), i
            else:
                b.check_grad(got, zh[i], y, t, ai, hi, 0.0, dtype, ("grad", i))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C,t", [(7, 1, 1.0), (9, 2, 2.0), (12, 7, 0.5), (12, 8, 1.0), (12, 9, 1.0), (12, 63, 0.7), (16, 64, 1.0),
                                   (12, 65, 3.0), (20, 1000, 0.9), (6, 4099, 1.0), (6, 30001, 0.9), (6, 50021, 1.0),
                                   (6, 131071, 1.3), (6, 131072, 1.0), (6, 200003, 1.0)])
def test_token_logp(n, C, t, dtype):
    rng = np.random.default_rng(n * 7 + C)
    z, labels = lm_rows(rng, n, C, dtype)
    z = z.to(DEV)
    a, h = rng.standard_normal(n).astype(np.float32), (0.3 * rng.standard_normal(n)).astype(np.float32)
    a[2] = h[2] = 0
    a[3] = h[4] = 0
    out = run_logp(z, labels, t, a, h)
    check_logp(z, labels, t, a, h, out, dtype)
    # each output alone gives its values again; without the entropy's weight, the gradient of log p alone
    check_logp(z, labels, t, None, None, run_logp(z, labels, t, grad=False, entropy=False), dtype)
    check_logp(z, labels, t, None, None, run_logp(z, labels, t, grad=False, logp=False), dtype)
    check_logp(z, labels, t, a, None, run_logp(z, labels, t, a, None, entropy=False, logp=False), dtype)
    check_logp(z, labels, t, None, h, run_logp(z, labels, t, None, h, entropy=False, logp=False), dtype)
    again = run_logp(z, labels, t, a, h)
    assert all(torch.equal(x, y) for x, y in zip(out, again))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("chunks", [64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384, 20480])
def test_token_logp_at_every_row_length(chunks, dtype):
    """Both sides of numbers of 16-byte chunks at which a row may take more threads or registers; of the odd lengths
    every row starts at another alignment."""
    V = 8 if dtype == "bf16" else 4
    rng = np.random.default_rng(chunks)
    for C in (chunks * V - 1, chunks * V, chunks * V + 1):
        z, labels = lm_rows(rng, 3, C, dtype)
        labels[:] = (C - 1, 0, C - V)                        # in the last chunk, the first, and on their border
        a = rng.standard_normal(3).astype(np.float32)
        z = z.to(DEV)
        check_logp(z, labels, 0.9, a, a, run_logp(z, labels, 0.9, a, a), dtype)
        check_logp(z, labels, 0.9, a, None, run_logp(z, labels, 0.9, a, entropy=False), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,chunks", [(8195, 257), (8195, 768), (8195, 769), (600, 257), (600, 768), (600, 1024), (600, 1025),
                                      (600, 2048), (600, 2049), (600, 3071), (600, 3073), (600, 4096), (600, 4097), (770, 4097),
                                      (1024, 5000), (1025, 4200), (600, 9000)])
def test_whole_rows_of_many(n, chunks, dtype):
    """Enough rows that none goes in parts, at both sides of the numbers of 16-byte chunks and of rows at which a row takes
    other threads or registers; the rows repeat ten that differ, and equal rows on equal boundaries have equal results."""
    V = 8 if dtype == "bf16" else 4
    rng = np.random.default_rng(chunks)
    for C in (chunks * V, chunks * V - 5):
        rows, labels = lm_rows(rng, 10, C, dtype)
        labels[:3] = (C - 1, 0, C - V)                       # in the last chunk, the first, and on their border
        A, old, ref, g = policy_inputs(rng, rows, labels, 0.9, 0.2, 0.28)
        at = np.arange(n) % 10
        z = rows.to(DEV)[torch.from_numpy(at).to(DEV)]
        sel = list(range(10)) + list(range(n - 10, n))
        for ent in (0.02, 0.0):
            h = g[at] * np.float32(ent) if ent else None
            for grad in (True, False):
                out = run_logp(z, labels[at], 0.9, A[at] if grad else None, h if grad else None, entropy=bool(ent), grad=grad)
                check_logp(z[sel], labels[at][sel], 0.9, A[at][sel], None if h is None else h[sel],
                           [o if o is None else o[sel] for o in out], dtype)
                if C % V == 0:
                    for o in out:
                        assert o is None or torch.equal(o[10:n // 10 * 10].reshape(n // 10 - 1, -1),
                                                        o[:10].reshape(1, -1).expand(n // 10 - 1, -1))
            o = run_policy(z, labels[at], A[at], old[at], ref[at], g[at], 0.9, 0.2, 0.28, 0.05, ent)
            check_policy(z[sel], labels[at][sel], A[at][sel], old[at][sel], ref[at][sel], g[at][sel], 0.9, 0.2, 0.28, 0.05, ent,
                         {k: v[sel] for k, v in o.items()}, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [5, 700, 90001, 200003])
def test_token_logp_special_rows(C, dtype):
    low, high = float(torch.finfo(DT[dtype]).min), float(torch.finfo(DT[dtype]).max)
    z = torch.zeros((13, C))
    labels = np.full(13, 2, np.int32)
    z[0] = -math.inf                           # nothing left
    z[1] = -math.inf
    z[1, 2] = 3.0                              # only the label left: p = 1
    z[2, 2] = -math.inf                        # the label is masked
    z[3] = low                                 # all at the type's lowest value: uniform
    z[4] = low
    z[4, 2] = 1.0                              # the label above masks of the lowest value
    z[5] = low
    z[5, 3] = 1.0                              # another class above them
    z[6, C - 1] = math.nan
    z[7, C - 1] = math.inf
    z[8, 2] = math.inf
    z[9] = high
    z[9, 2] = low                              # further apart than fp32 holds
    z[10, 2] = math.nan
    z[11] = -math.inf
    z[11, [2, C - 1]] = -1.0                   # two classes left
    z[12, 2] = 1000.0
    z = z.to(DT[dtype]).to(DEV)
    a = np.linspace(0.5, 2, 13).astype(np.float32)
    for t in (1.0, 0.25, 2.0 ** 20, 2.0 ** -20):
        for h in (None, -a):
            check_logp(z, labels, t, a, h, run_logp(z, labels, t, a, h), dtype)
        check_logp(z, labels, t, None, None, run_logp(z, labels, t, grad=False), dtype)
    weightless = run_logp(z, labels, 1.0, 0 * a, 0 * a)
    assert (weightless[2] == 0).all()


def test_token_logp_of_a_sure_student():
    """p within 2^-40 of 1: log p and the label's gradient keep their own relative precision."""
    z = torch.zeros((3, 100), device=DEV)
    z[0, 5], z[1, 99], z[2, 0] = 30.0, 40.0, 60.0
    labels = np.int32([5, 99, 0])
    a = np.float32([1, 1, 1])
    logp, _, grad = run_logp(z, labels, 1.0, a)
    for i, top in enumerate((30.0, 40.0, 60.0)):
        want = -math.log1p(99 * math.exp(-top))
        # exp(-top) in fp32: the argument's rounding 2^-24 top, the sum of 99 ones is exact
        rel = 2.0 ** -22 * (top + 4)
        assert abs(float(logp[i]) - want) <= rel * abs(want)
        assert abs(float(grad[i, labels[i]]) + want) <= rel * abs(want) + abs(want) ** 2


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [50, 900, 9000, 70001])
def test_token_logp_of_unlikely_tokens(C, dtype):
    """Labels up to e^-400 below the others, with weights down to 1e-30: the gradient of the likely classes keeps its
    precision, whichever way the row is summed."""
    below = (10.0, 20.0, 30.0, 33.0, 34.0, 60.0, 87.0, 88.0, 89.0, 104.0, 400.0)
    n = len(below)
    rng = np.random.default_rng(C)
    z = torch.from_numpy(rng.standard_normal((n, C)).astype(np.float32))
    labels = rng.integers(0, C, n).astype(np.int32)
    for i, d in enumerate(below):
        z[i, labels[i]] = -d
    z = z.to(DT[dtype]).to(DEV)
    for a in (1.0, 1e-8, 1e-30):
        w = np.full(n, a, np.float32)
        for h in (None, w):
            check_logp(z, labels, 1.0, w, h, run_logp(z, labels, 1.0, w, h), dtype)
    A, g = np.ones(n, np.float32), np.full(n, 1e-8, np.float32)
    check_policy(z, labels, A, None, None, g, 1.0, 0.2, 0.2, 0.0, 0.01, run_policy(z, labels, A, None, None, g, ent=0.01), dtype)
    offsets = [0, 5, n]
    check_preference(z, labels, offsets, None, 1.0, 1e-3, 0.0, False, None,
                     run_preference(z, labels, offsets, None, 1.0, 1e-3), dtype)


def test_token_logp_strided_unaligned_broadcast():
    rng = np.random.default_rng(3)
    n, C = 7, 1001
    for dtype in ("fp32", "bf16"):
        z, labels = lm_rows(rng, n, C, dtype)
        a = rng.standard_normal(n).astype(np.float32)
        buf = torch.zeros(n * 1103 + 3, dtype=DT[dtype], device=DEV)
        v = buf[3:].as_strided((n, C), (1103, 1))
        v.copy_(z)
        gbuf = full(n * 1105 + 5, dtype=DT[dtype])
        grad = gbuf[5:].as_strided((n, C), (1105, 1))
        logp = full(n + 2)
        bd.token_logp(v, dev(labels), logp[1:-1], None, grad, dev(a))
        torch.cuda.synchronize()
        check_logp(v, labels, 1.0, a, None, (logp[1:-1], None, grad), dtype)
        assert (gbuf[:5] == -7).all() and (gbuf[5:].as_strided((n - 1, 104), (1105, 1), 5 + C) == -7).all()
        assert logp[0] == -7 and logp[-1] == -7
        one = z[:1].to(DEV).expand(n, C)                       # one row for all labels
        check_logp(one, labels, 1.0, a, None, run_logp(one, labels, 1.0, a), dtype)
        over = buf[3:].as_strided((n, C), (17, 1))             # rows that overlap
        check_logp(over, labels, 1.0, a, None, run_logp(over, labels, 1.0, a), dtype)


def test_offsets_past_32_bits():
    """Rows of logits and of the gradient more than 2^31 elements from the first."""
    rng = np.random.default_rng(4)
    n, C, ld = 4, 5000, (1 << 30) - 3
    buf = torch.empty(3 * ld + C, dtype=torch.bfloat16, device=DEV)
    grad_buf = torch.empty(3 * ld + C, dtype=torch.bfloat16, device=DEV)
    v, grad = buf.as_strided((n, C), (ld, 1)), grad_buf.as_strided((n, C), (ld, 1))
    z, labels = lm_rows(rng, n, C, "bf16")
    v.copy_(z)
    a = rng.standard_normal(n).astype(np.float32)
    logp = full(n)
    bd.token_logp(v, dev(labels), logp, None, grad, dev(a))
    torch.cuda.synchronize()
    check_logp(v, labels, 1.0, a, None, (logp, None, grad), "bf16")
    loss = full(1)
    offsets = np.int32([0, 3, 4])
    bd.preference_loss(v, dev(labels), loss, grad, offsets=dev(offsets))
    torch.cuda.synchronize()
    check_preference(v, labels, offsets, None, 1.0, 0.1, 0.0, False, None, (loss, None, grad), "bf16")


def test_more_rows_than_one_launch_takes():
    n, C = (1 << 20) + 5, 3
    z = torch.randn((n, C), device=DEV)
    labels = torch.randint(-1, C, (n,), dtype=torch.int32, device=DEV)
    logp, grad, a = full(n), torch.full_like(z, -7), torch.randn(n, device=DEV)
    bd.token_logp(z, labels, logp, None, grad, a)
    rows = torch.log_softmax(z.double(), -1)
    valid = labels >= 0
    want = torch.where(valid, rows.gather(1, labels.clamp(min=0).long()[:, None])[:, 0], 0)
    d = -torch.exp(rows)
    d.scatter_add_(1, labels.clamp(min=0).long()[:, None], torch.ones(n, 1, dtype=torch.float64, device=DEV))
    d *= torch.where(valid, a.double(), 0)[:, None]
    # three terms: 2^-22 (|x| + 4) with |x| < 12, twice
    assert (logp.double() - want).abs().max() < 2.0 ** -17 and (grad.double() - d).abs().max() < 2.0 ** -15
    loss, scores = full(1), full(1, 2)
    bd.preference_loss(z, labels, loss, grad, n_pairs=1, offsets=torch.tensor([1, 9, n - 2], dtype=torch.int32, device=DEV),
                       out_scores=scores)
    score = torch.stack([want[1:9].sum(), want[9:n - 2].sum()]) * 0.1
    assert (scores[0].double() - score).abs().max() < 0.1 * n * 2.0 ** -20
    assert torch.equal(grad[0].double(), grad[0].double()) and (grad[n - 2:].double() - d[n - 2:]).abs().max() < 2.0 ** -15


def test_token_logp_gradient_against_differences():
    """Along a direction v: (f(z + h v) - f(z - h v)) / 2h against the gradient times v, in fp32: truncation
    h^2 |f'''| |v|^3 / 6 with |v| = 1 and f''' below 4, rounding of the two values 2^-23 |f| / h each."""
    rng = np.random.default_rng(8)
    n, C, h = 6, 300, 2.0 ** -5
    z = torch.from_numpy(rng.standard_normal((n, C)).astype(np.float32)).to(DEV)
    labels = rng.integers(0, C, n).astype(np.int32)
    v = rng.standard_normal((n, C))
    v = dev((v / np.sqrt((v * v).sum(1, keepdims=True))).astype(np.float32))
    one = np.ones(n, np.float32)
    for a, w in ((one, 0 * one), (0 * one, one)):
        grad = run_logp(z, labels, 1.0, a, w)[2]
        k = 0 if a[0] else 1
        up, down = run_logp(z + h * v, labels, 1.0, grad=False)[k], run_logp(z - h * v, labels, 1.0, grad=False)[k]
        diff = (up.double() - down.double()) / (2 * h)
        assert (diff - (grad.double() * v.double()).sum(1)).abs().max() < h * h * 4 / 6 + 2 * 2.0 ** -23 * 8 / h * 4


# ---------------------------------------------------------------- policy

def run_policy(z, labels, A, old=None, ref=None, g=None, t=1.0, low=0.2, high=0.2, kl=0.0, ent=0.0, outputs="loss logp kl entropy grad", **kw):
    n = z.shape[0]
    o = {k: (torch.full(z.shape, -7, dtype=z.dtype, device=DEV) if k == "grad" else full(n)) for k in outputs.split()}
    up = lambda v: None if v is None else dev(v)  # noqa: E731
    bd.policy_loss(z, dev(labels), dev(A), o.get("loss"), o.get("grad"), old_logp=up(old), ref_logp=up(ref), grad_loss=up(g),
                   out_logp=o.get("logp"), out_kl=o.get("kl"), out_entropy=o.get("entropy"), temperature=t, clip_low=low,
                   clip_high=high, kl_coef=kl, entropy_coef=ent, **kw)
    torch.cuda.synchronize()
    return o


def check_policy(z, labels, A, old, ref, g, t, low, high, klc, ent, o, dtype):
    zh = host(z)
    for i in range(len(labels)):
        y = int(labels[i])
        at = lambda v, d=None: d if v is None else float(v[i])  # noqa: E731
        gi = at(g, 1.0)
        loss, logp, kl, H, grad = ot.policy(zh[i], y, at(A), at(old), at(ref), t, low, high, klc, ent, gi)
        b = Bounds(zh[i], y, t) if 0 <= y < zh.shape[1] else None
        limits = dict(loss=0.0, logp=0.0, kl=0.0, entropy=0.0)
        slope = da = 0.0
        if b is not None and b.defined:
            dl = b.d_logp
            # r and exp(d) are off by dl and one rounding; the double results are rounded once
            ratio = 0.0 if at(A) == 0 or old is None else min(math.exp(min(b.logp - at(old), 80)), 3e38) if b.logp > -np.inf else 0.0
            e = math.exp(min(at(ref) - b.logp, 80)) if ref is not None and b.logp > -np.inf else 0.0
            d_r = abs(at(A)) * ratio * (dl + 2.0 ** -23)
            d_kl = abs(e - 1) * dl + e * dl * dl if e else 0.0
            da = abs(gi) * (d_r + (abs(klc) * e * (dl + 2.0 ** -40) if klc else 0.0))
            limits = dict(loss=d_r + (abs(klc) * d_kl if klc else 0.0) + abs(ent) * b.d_H + 2.0 ** -23 * (abs(loss) + (abs(klc * kl) if klc else 0.0) + abs(ent * H)),
                          logp=dl + 2.0 ** -149, kl=d_kl + 2.0 ** -23 * abs(kl) + 1e-14, entropy=b.d_H)
            plain = at(A) * (ratio if old is not None else 1.0)
            cut = at(A) * min(max(ratio, 1 - low), 1 + high) if old is not None else plain
            slope = (-plain if plain <= cut else 0.0) - (klc * (e - 1) if klc and ref is not None else 0.0)
        for k, want in (("loss", loss), ("logp", logp), ("kl", kl), ("entropy", H)):
            if k in o:
                got = float(o[k][i])
                if math.isfinite(want) and abs(want) < 3.4e38:
                    near(got, want, limits[k], (k, i))
                else:
                    assert got == want or (math.isnan(got) and math.isnan(want)) or abs(got) >= 3.4e38, (k, i, got, want)
        if "grad" in o:
            got = host(o["grad"][i])
            if np.isnan(grad).any():
                assert np.isnan(got).all(), i
            elif b is None or gi == 0:
                assert (got == 0).all(), i
            else:
                b.check_grad(got, zh[i], y, t, gi * slope, -gi * ent, da + abs(gi * slope) * 2.0 ** -22, dtype, ("grad", i))


def policy_inputs(rng, z, labels, t, low, high):
    """Old and reference log p near the present ones, no ratio next to a border of the clip."""
    zh, n = host(z), len(labels)
    logp = np.zeros(n)
    for i, y in enumerate(labels):
        facts = ot.token_facts(zh[i], y, t) if 0 <= y < zh.shape[1] else None
        logp[i] = facts[0] if facts else 0.0
    step = 0.3 * rng.standard_normal(n)
    for border in (1 - low, 1 + high):
        step[np.abs(step - math.log(border)) < 1e-3] += 3e-3
    f = lambda v: v.astype(np.float32)  # noqa: E731
    return f(rng.standard_normal(n)), f(logp - step), f(logp + 0.5 * rng.standard_normal(n)), f(rng.standard_normal(n))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kl,ent", [(0.0, 0.0), (0.1, 0.0), (0.05, 0.02), (-0.3, -0.1)])
@pytest.mark.parametrize("n,C,t", [(16, 2, 1.0), (24, 65, 0.7), (24, 1000, 0.9), (10, 30001, 1.0), (6, 131071, 0.9), (5, 200003, 1.0)])
def test_policy(n, C, t, kl, ent, dtype):
    rng = np.random.default_rng(n + C)
    z, labels = lm_rows(rng, n, C, dtype)
    A, old, ref, g = policy_inputs(rng, z, labels, t, 0.2, 0.28)
    z = z.to(DEV)
    g[2] = 0
    A[3] = 0
    o = run_policy(z, labels, A, old, ref, g, t, 0.2, 0.28, kl, ent)
    check_policy(z, labels, A, old, ref, g, t, 0.2, 0.28, kl, ent, o, dtype)
    for k in o:                                              # each output alone
        alone = run_policy(z, labels, A, old, ref, g, t, 0.2, 0.28, kl, ent, outputs=k)
        check_policy(z, labels, A, old, ref, g, t, 0.2, 0.28, kl, ent, alone, dtype)
    for o2, r2 in ((None, ref), (old, None), (None, None)):
        o = run_policy(z, labels, A, o2, r2, None, t, 0.2, 0.28, kl, ent)
        check_policy(z, labels, A, o2, r2, None, t, 0.2, 0.28, kl, ent, o, dtype)


def test_policy_clips():
    """Ratios of exactly 1/2, 1, 2 (logits of two equal classes, log p = - log 2 up to one rounding of old) on both
    sides of the clip, with both signs of the advantage."""
    z = torch.zeros((9, 2), device=DEV)
    labels = np.zeros(9, np.int32)
    steps = np.log(np.repeat([0.5, 1.0, 2.0], 3))
    old = (math.log(0.5) - steps).astype(np.float32)
    A = np.float32([1, -1, 0] * 3)
    o = run_policy(z, labels, A, old, low=0.2, high=0.3)
    want = [-0.5, 0.8, 0, -1, 1, 0, -1.3, 2, 0]
    slope = [-0.5, 0, 0, -1, 1, 0, 0, 2, 0]                  # d loss / d log p
    assert np.abs(host(o["loss"]) - want).max() <= 2.0 ** -21
    assert np.abs(host(o["grad"])[:, 0] - np.array(slope) / 2).max() <= 2.0 ** -21
    o = run_policy(z, labels, A, old, low=1.0, high=math.inf)      # no clip
    assert np.abs(host(o["loss"]) - [-0.5, 0.5, 0, -1, 1, 0, -2, 2, 0]).max() <= 2.0 ** -21


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [5, 3000, 200003])
def test_policy_special_rows(C, dtype):
    """Masked labels, empty rows, infinities and NaN, ratios and KL terms beyond fp32."""
    n = 14
    z = torch.zeros((n, C))
    z[0] = -math.inf
    z[1, 2] = -math.inf                                      # p = 0: ratio 0, KL infinite
    z[2, 3] = math.nan
    z[3, 3] = math.inf
    z[4, 2] = 200.0                                          # ratio beyond fp32
    z[5, 2] = 200.0
    z[6] = -math.inf
    z[6, 2] = 1.0                                            # p = 1
    z[7, 2] = -500.0
    z = z.to(DT[dtype]).to(DEV)
    labels = np.full(n, 2, np.int32)
    logp = np.array([ot.token_facts(host(z[i]), 2, 1.0)[0] if i not in (0, 2, 3) else 0.0 for i in range(n)])
    old, ref = (np.where(np.isfinite(logp), logp, -5) + 0.1).astype(np.float32), (np.where(np.isfinite(logp), logp, -5) - 0.2).astype(np.float32)
    A = np.float32([1, 1, 1, 1, 1, -1, 1, -1, 0, math.nan, 1, 1, 1, 0])
    old[4:6] = -200.0
    ref[7] = 1.0
    old[8], ref[10] = math.nan, math.nan
    old[11], ref[12] = -math.inf, -math.inf
    ref[13] = math.inf
    for klc in (0.0, 0.5):
        for r in (ref, None):
            o = run_policy(z, labels, A, old, r, None, kl=klc)
            check_policy(z, labels, A, old, r, None, 1.0, 0.2, 0.2, klc, 0.0, o, dtype)
            o = run_policy(z, labels, A, old, r, np.zeros(n, np.float32), kl=klc)
            assert (o["grad"] == 0).all()


# ---------------------------------------------------------------- preference

def run_preference(z, labels, offsets, ref=None, t=1.0, beta=0.1, smoothing=0.0, mean=False, g=None, pairs=None,
                   outputs="loss scores grad", **kw):
    P = pairs or (len(offsets) - 1) // 2
    o = {k: {"loss": lambda: full(P), "scores": lambda: full(P, 2),
             "grad": lambda: torch.full(z.shape, -7, dtype=z.dtype, device=DEV)}[k]() for k in outputs.split()}
    up = lambda v: None if v is None else dev(v)  # noqa: E731
    bd.preference_loss(z, dev(labels), o.get("loss"), o.get("grad"), offsets=up(None if offsets is None else np.int32(offsets)),
                       n_pairs=pairs, ref_logp=up(ref), grad_loss=up(g), out_scores=o.get("scores"), temperature=t, beta=beta,
                       smoothing=smoothing, mean=mean, **kw)
    torch.cuda.synchronize()
    return o.get("loss"), o.get("scores"), o.get("grad")


def check_preference(z, labels, offsets, ref, t, beta, smoothing, mean, g, out, dtype):
    loss, scores, grad = out
    zh = host(z)
    want_loss, want_scores, want_grad = ot.preference(zh, labels, offsets, ref, t, beta, smoothing, mean, g)
    C = zh.shape[1]
    for p in range(len(want_loss)):
        rows = [[i for i in range(offsets[2 * p + k], offsets[2 * p + k + 1]) if 0 <= labels[i] < C] for k in range(2)]
        bounds = {i: Bounds(zh[i], int(labels[i]), t) for r in rows for i in r}
        per = [1 / len(r) if mean and r else 1.0 for r in rows]
        d_score = [beta * per[k] * sum(bounds[i].d_logp for i in rows[k] if bounds[i].defined) for k in range(2)]
        d_u = sum(d_score)
        for k in range(2):
            if scores is not None:
                near(float(scores[p, k]), want_scores[p, k], d_score[k] + 2.0 ** -23 * abs(want_scores[p, k]), ("score", p, k))
        if loss is not None:
            near(float(loss[p]), want_loss[p], d_u + 2.0 ** -23 * abs(want_loss[p]), ("loss", p))
        if grad is None:
            continue
        gp = 1.0 if g is None else float(g[p])
        u = want_scores[p, 0] - want_scores[p, 1]
        sig = lambda v: 1 / (1 + math.exp(-v)) if v > -700 else 0.0  # noqa: E731
        du = math.nan if math.isnan(u) else smoothing * sig(u) - (1 - smoothing) * sig(-u)
        for k in range(2):
            a = 0.0 if gp == 0 else (-1 if k else 1) * beta * gp * du * per[k]
            # the sigmoid's slope is at most its value and 1/4
            da = 0.0 if gp == 0 or math.isnan(u) else beta * abs(gp) * per[k] * min(0.25, sig(u) * sig(-u)) * d_u * 1.5
            for i in range(offsets[2 * p + k], offsets[2 * p + k + 1]):
                got = host(grad[i])
                if i not in bounds or gp == 0:
                    assert (got == 0).all(), i
                elif math.isnan(a) or not bounds[i].defined:
                    assert np.isnan(got).all(), i
                else:
                    bounds[i].check_grad(got, zh[i], int(labels[i]), t, a, 0.0, da + abs(a) * 2.0 ** -22, dtype, ("grad", i))
    if grad is not None:
        for i in list(range(offsets[0])) + list(range(offsets[-1], len(labels))):
            assert (host(grad[i]) == -7).all(), i


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("C,t,lengths", [(1, 1.0, [1, 2]), (2, 1.0, [1, 1, 2, 3]), (9, 0.5, [3, 0, 1, 4]), (1000, 0.9, [5, 7, 0, 0, 9, 1]),
                                         (4099, 1.0, [4, 4]), (30001, 0.9, [3, 6, 2, 2]), (131071, 1.0, [2, 3]), (200003, 1.0, [1, 2])])
def test_preference(C, t, lengths, mean, dtype):
    rng = np.random.default_rng(C + len(lengths))
    offsets = np.concatenate([[2], 2 + np.cumsum(lengths)])
    n = int(offsets[-1]) + 3
    z, labels = lm_rows(rng, n, C, dtype)
    ref = np.array([ot.token_facts(host(z[i]), y, t)[0] if 0 <= y < C else 0.0 for i, y in enumerate(labels)])
    ref = (ref + rng.standard_normal(n)).astype(np.float32)
    z = z.to(DEV)
    P = len(lengths) // 2
    g = rng.standard_normal(P).astype(np.float32)
    for smoothing in (0.0, 0.1):
        out = run_preference(z, labels, offsets, ref, t, 0.3, smoothing, mean, g)
        check_preference(z, labels, offsets, ref, t, 0.3, smoothing, mean, g, out, dtype)
    out = run_preference(z, labels, offsets, None, t, 0.01, 0.0, mean)
    check_preference(z, labels, offsets, None, t, 0.01, 0.0, mean, None, out, dtype)
    for k, name in enumerate(("loss", "scores", "grad")):    # each output alone
        alone = run_preference(z, labels, offsets, None, t, 0.01, 0.0, mean, outputs=name)
        assert torch.equal(alone[k], out[k])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("chunks", [30, 255, 257, 1024, 1025, 1536, 1537, 2049])
def test_preference_of_many_rows(chunks, dtype):
    """Enough rows for three launches and none in parts, at both sides of the numbers of 16-byte chunks at which a row takes
    other threads; the pairs repeat one whose answers are checked, in rows on other boundaries."""
    V = 8 if dtype == "bf16" else 4
    rng = np.random.default_rng(chunks)
    for C in (chunks * V, chunks * V - 5):
        rows, labels = lm_rows(rng, 11, C, dtype)
        labels[:3] = (C - 1, 0, C - V)
        ref = np.array([ot.token_facts(host(rows[i]), y, 0.9)[0] if 0 <= y < C else 0.0 for i, y in enumerate(labels)])
        ref = (ref + rng.standard_normal(11)).astype(np.float32)
        pairs = 60
        at = np.concatenate([[0], np.tile(np.arange(11), pairs), [0, 0]])
        offsets = np.concatenate([[1], 1 + np.cumsum(np.tile([4, 7], pairs))])
        z = rows.to(DEV)[torch.from_numpy(at).to(DEV)]
        g = rng.standard_normal(pairs).astype(np.float32)
        loss, scores, grad = run_preference(z, labels[at], offsets, ref[at], 0.9, 0.3, 0.1, True, g)
        for p in (0, 1, pairs - 1):
            r = slice(1 + 11 * p, 12 + 11 * p)
            check_preference(z[r], labels, [0, 4, 11], ref, 0.9, 0.3, 0.1, True, g[p:p + 1],
                             (loss[p:p + 1], scores[p:p + 1], grad[r]), dtype)
        if C % V == 0:                                       # equal rows on equal boundaries
            assert (loss == loss[0]).all() and (scores == scores[0]).all()
        assert (grad[0] == -7).all() and (grad[-2:] == -7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("t", [2.0 ** -20, 2.0 ** -12, 2.0 ** -8, 0.02, 0.03, 50.0, 2.0 ** 20])
def test_preference_at_low_and_high_temperatures(t, dtype):
    """Logits near 0, whose label is just above or below the others: what a low temperature makes large differences of."""
    rng = np.random.default_rng(int(math.log2(t)) + 40)
    for C in (2, 9, 700, 40001):
        z = (rng.standard_normal((7, C)) * 0.05).astype(np.float32)
        labels = rng.integers(0, C, 7).astype(np.int32)
        z[1, labels[1]] = z[1].max() + np.float32(0.01)       # the likeliest class
        z[2, labels[2]] = z[2].min() - np.float32(0.01)       # the least likely one
        z[3] -= z[3].max() + np.float32(0.01)                 # all below 0, the label's below the others
        z[3, labels[3]] = -0.0625
        z[4] += 16 - z[4].mean()
        z = torch.from_numpy(z).to(DT[dtype]).to(DEV)
        out = run_preference(z, labels, [0, 2, 4, 5, 7], None, t, min(t, 1.0) * 0.3, 0.1)
        check_preference(z, labels, [0, 2, 4, 5, 7], None, t, min(t, 1.0) * 0.3, 0.1, False, None, out, dtype)


def test_preference_equal_lengths_and_padding():
    rng = np.random.default_rng(12)
    n, C = 24, 500
    z, labels = lm_rows(rng, n, C, "bf16")
    labels[4:6] = labels[10:12] = -1                          # answers padded to 6 rows
    labels[18:24] = -1                                        # one without tokens
    z = z.to(DEV)
    for mean in (False, True):
        out = run_preference(z, labels, None, mean=mean, pairs=2)
        check_preference(z, labels, [0, 6, 12, 18, 24], None, 1.0, 0.1, 0.0, mean, None, out, "bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_preference_special_rows(dtype):
    """A NaN row makes its own pair NaN and no other; padding may hold anything; infinite scores; weights of 0."""
    C = 700
    rng = np.random.default_rng(13)
    offsets = [0, 2, 4, 6, 8, 10, 12, 14, 16, 18, 20, 22, 24]
    z, labels = lm_rows(rng, 24, C, dtype)
    labels[:] = rng.integers(0, C, 24)
    z[1, 5] = math.nan                                        # pair 0
    z[4] = math.nan                                           # pair 1: a row without a token
    labels[4] = -1
    z[9, labels[9]] = -math.inf                               # pair 2: the chosen one impossible
    z[15, labels[15]] = -math.inf                             # pair 3: the rejected one
    z[16, labels[16]] = -math.inf                             # pair 4: both
    z[18, labels[18]] = -math.inf
    z[20] = -math.inf                                         # pair 5: an empty row
    z = z.to(DEV)
    g = np.float32([1, 1, 1, 1, 1, 1])
    for smoothing in (0.0, 0.25):
        out = run_preference(z, labels, offsets, None, 1.0, 0.2, smoothing, False, g)
        check_preference(z, labels, offsets, None, 1.0, 0.2, smoothing, False, g, out, dtype)
    out = run_preference(z, labels, offsets, None, 1.0, 0.2, 0.0, False, 0 * g)
    assert (out[2] == 0).all()


@pytest.mark.parametrize("pairs", [70000, 1 << 20])
def test_preference_of_many_pairs(pairs):
    """More pairs than a grid's second axis takes, most of them without rows or with one."""
    C, n = 5, 150000
    g = torch.Generator(device="cuda").manual_seed(pairs)
    z = torch.randn((n, C), device=DEV, generator=g)
    labels = torch.randint(-1, C, (n,), dtype=torch.int32, device=DEV, generator=g)
    offsets = torch.sort(torch.randint(0, n + 1, (2 * pairs + 1,), dtype=torch.int32, device=DEV, generator=g)).values
    loss, scores, grad = full(pairs), full(pairs, 2), torch.full_like(z, -7)
    bd.preference_loss(z, labels, loss, grad, offsets=offsets, out_scores=scores, beta=0.5)
    rows = torch.log_softmax(z.double(), -1)
    at = labels.clamp(min=0).long()[:, None]
    valid = labels >= 0
    logp = torch.where(valid, rows.gather(1, at)[:, 0], 0)
    run = torch.cat([torch.zeros(1, dtype=torch.float64, device=DEV), logp.cumsum(0)])
    first = offsets.long()
    score = (0.5 * (run[first[1:]] - run[first[:-1]])).view(-1, 2)
    u = score[:, 0] - score[:, 1]
    # five terms: 2^-22 (|x| + 4) with |x| < 14 a row, at most some 20 rows an answer; the running sum is off by 1e-9
    assert (scores.double() - score).abs().max() < 20 * 2.0 ** -17 and (loss.double() + torch.nn.functional.logsigmoid(u)).abs().max() < 40 * 2.0 ** -17
    which = torch.searchsorted(first[1:], torch.arange(n, device=DEV), right=True).clamp(max=2 * pairs - 1)
    a = -0.5 * torch.sigmoid(-u)[which // 2] * (1 - 2 * (which % 2)) * valid
    want = -torch.exp(rows)
    want.scatter_add_(1, at, torch.ones_like(want[:, :1]))
    want *= a[:, None]
    inside = (torch.arange(n, device=DEV) >= first[0]) & (torch.arange(n, device=DEV) < first[-1])
    assert (grad.double() - want)[inside].abs().max() < 2.0 ** -13 and (grad[~inside] == -7).all()


def test_preference_bad_offsets_stay_inside():
    """Decreasing offsets and such beyond the rows: wrong values, but nothing outside of the arrays is written."""
    n, C = 6, 300
    z = torch.randn((n, C), device=DEV)
    buf = full((n + 2) * C)
    grad = buf[C:-C].view(n, C)
    loss = full(4)
    labels = torch.zeros(n, dtype=torch.int32, device=DEV)
    for offsets in ([0, 4, 2, 5, 1], [-5, 3, 100, 2 ** 31 - 1, -2 ** 31], [6, 6, 6, 6, 6], [3, 2, 1, 0, -1]):
        need = bd.preference_workspace(n, C)
        ws = full(need + 32, dtype=torch.uint8)
        ws.fill_(9)
        bd.preference_loss(z, labels, loss[1:3], grad, offsets=dev(np.int32(offsets)), workspace=ws[16:16 + need])
        torch.cuda.synchronize()
        assert (buf[:C] == -7).all() and (buf[-C:] == -7).all() and loss[0] == -7 and loss[3] == -7
        assert (ws[:16] == 9).all() and (ws[16 + need:] == 9).all()


# ---------------------------------------------------------------- streams, graphs, the chain

def chain_setup(seed, pairs=2, length=5, c_in=200, C=3001):
    rng = np.random.default_rng(seed)
    n = 2 * pairs * length
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV)  # noqa: E731
    b = dict(hidden=f(n, c_in).to(torch.bfloat16), head=f(C, c_in) * 0.3, ref_head=f(C, c_in) * 0.3, bias=f(C),
             uniform=torch.from_numpy(rng.random(n).astype(np.float32)).to(DEV), advantage=f(n), logits=full(n, C),
             ref_logits=full(n, C), tokens=full(n, dtype=torch.int32), probs=full(n), old=full(n), ref=full(n), loss=full(n),
             grad=torch.full((n, C), -7.0, device=DEV), pair_loss=full(pairs), scores=full(pairs, 2),
             pair_grad=torch.full((n, C), -7.0, device=DEV))
    b["x"], b["w"], b["ref_w"] = bd.mx4_empty(n, c_in), bd.mx4_empty(C, c_in), bd.mx4_empty(C, c_in)
    need = (bd.combine_workspace(1, n, C), bd.fc_mx4_workspace(n, c_in + -c_in % 32, C), bd.preference_workspace(n, C))
    b["ws"] = [torch.empty(max(k, 16), dtype=torch.uint8, device=DEV) for k in need]
    b["pairs"] = pairs
    return b


def chain(b, stream=None, own_workspace=True):
    """Both heads in 4 bits, tokens drawn from the student, their log p under both, the two losses."""
    ws = b["ws"] if own_workspace else [None] * 3
    s = dict(stream=stream)
    bd.quantize_rows_mx4(b["hidden"], *b["x"], **s)
    bd.quantize_rows_mx4(b["head"], *b["w"], **s)
    bd.quantize_rows_mx4(b["ref_head"], *b["ref_w"], **s)
    bd.fc_mx4(*b["x"], *b["w"], b["logits"], bias=b["bias"], workspace=ws[1], **s)
    bd.fc_mx4(*b["x"], *b["ref_w"], b["ref_logits"], bias=b["bias"], workspace=ws[1], **s)
    bd.combine_sample(b["logits"], b["uniform"], b["tokens"], b["probs"], workspace=ws[0], **s)
    bd.token_logp(b["logits"], b["tokens"], b["old"], **s)
    bd.token_logp(b["ref_logits"], b["tokens"], b["ref"], **s)
    bd.policy_loss(b["logits"], b["tokens"], b["advantage"], b["loss"], b["grad"], old_logp=b["old"], ref_logp=b["ref"],
                   kl_coef=0.1, entropy_coef=0.01, **s)
    bd.preference_loss(b["logits"], b["tokens"], b["pair_loss"], b["pair_grad"], n_pairs=b["pairs"], ref_logp=b["ref"],
                       out_scores=b["scores"], workspace=ws[2], **s)


CHAIN = ("logits", "ref_logits", "tokens", "probs", "old", "ref", "loss", "grad", "pair_loss", "scores", "pair_grad")


def outputs(b):
    return [b[k].clone() for k in CHAIN]


def clear(b):
    for k in CHAIN:
        b[k].fill_(-7)


def test_chain_against_the_oracle():
    b = chain_setup(1)
    chain(b)
    torch.cuda.synchronize()
    for head, logits in (("head", "logits"), ("ref_head", "ref_logits")):
        xq, xs = ot.quantize_mx4(host(b["hidden"]))
        wq, ws = ot.quantize_mx4(host(b[head]))
        want = ot.fc_mx4(xq, xs, wq, ws, host(b["bias"]))
        size = np.abs(ot.mx4_values(xq, xs)) @ np.abs(ot.mx4_values(wq, ws)).T
        assert (np.abs(host(b[logits]) - want) <= size * 224 * 2.0 ** -23 + np.abs(want) * 2.0 ** -23).all()
    tokens = b["tokens"].cpu().numpy()
    z = b["logits"]
    for i, row in enumerate(host(z)):
        assert tokens[i] == ot.sample(row[None], float(b["uniform"][i]))[0]
        assert abs(math.log(float(b["probs"][i])) - float(b["old"][i])) < 1e-4
    check_logp(z, tokens, 1.0, None, None, (b["old"], None, None), "fp32")
    check_logp(b["ref_logits"], tokens, 1.0, None, None, (b["ref"], None, None), "fp32")
    n, L = len(tokens), len(tokens) // 4
    old, ref = b["old"].cpu().numpy(), b["ref"].cpu().numpy()
    check_policy(z, tokens, b["advantage"].cpu().numpy(), old, ref, None, 1.0, 0.2, 0.2, 0.1, 0.01,
                 dict(loss=b["loss"], grad=b["grad"]), "fp32")
    check_preference(z, tokens, [0, L, 2 * L, 3 * L, n], ref, 1.0, 0.1, 0.0, False, None,
                     (b["pair_loss"], b["scores"], b["pair_grad"]), "fp32")


def test_two_streams_at_once_repeat_the_same_bits():
    one, two = chain_setup(1), chain_setup(2, pairs=3, length=7, C=5003)
    chain(one)
    chain(two)
    torch.cuda.synchronize()
    want = [outputs(one), outputs(two)]
    clear(one), clear(two)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for own in (True, False):
        for _ in range(3):
            for b, s in zip((one, two), streams):
                chain(b, stream=s, own_workspace=own)
        torch.cuda.synchronize()
        for b, w in zip((one, two), want):
            assert all(torch.equal(x, y) for x, y in zip(outputs(b), w))
        clear(one), clear(two)
        torch.cuda.synchronize()


def test_replayed_graphs():
    """Two captured chains, replayed in turn with eager work between, give the eager results every time."""
    sets = [chain_setup(5), chain_setup(6, pairs=1, length=3, C=1001)]
    graphs = []
    for b in sets:
        chain(b)                                             # loads every kernel before the capture
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            chain(b)
        graphs.append(g)
    rng = np.random.default_rng(7)
    for _ in range(3):
        for b, g in zip(sets, graphs):
            b["hidden"].copy_(torch.from_numpy(rng.standard_normal(b["hidden"].shape).astype(np.float32)))
            chain(b)
            torch.cuda.synchronize()
            want = outputs(b)
            clear(b)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(outputs(b), want))


def test_inputs_and_surroundings_are_left_alone():
    rng = np.random.default_rng(9)
    n, C = 8, 777
    z, labels = lm_rows(rng, n, C, "bf16")
    z = z.to(DEV)
    before = z.clone()
    buf = full(n + 4)
    A = torch.randn(n, device=DEV)
    bd.policy_loss(z, dev(labels), A, buf[2:-2])
    bd.token_logp(z, dev(labels), buf[2:-2])
    need = bd.preference_workspace(n, C)
    ws = torch.full((need + 32,), 9, dtype=torch.uint8, device=DEV)
    loss = full(3)
    bd.preference_loss(z, dev(labels), loss[1:2], n_pairs=1, workspace=ws[16:16 + need])
    torch.cuda.synchronize()
    assert torch.equal(z, before) and (buf[:2] == -7).all() and (buf[-2:] == -7).all()
    assert loss[0] == -7 and loss[2] == -7 and (ws[:16] == 9).all() and (ws[16 + need:] == 9).all()


def test_refusals_on_the_device():
    z, f, i = torch.zeros((4, 6), device=DEV), torch.zeros(4, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    o = torch.tensor([0, 1, 4], dtype=torch.int32, device=DEV)
    for call in (lambda: bd.token_logp(z, i.long(), f), lambda: bd.token_logp(z, i, f[:3]), lambda: bd.token_logp(z, None, f),
                 lambda: bd.token_logp(z.half(), i, f), lambda: bd.token_logp(z.t(), i, f),
                 lambda: bd.token_logp(z, i, f, grad_logits=z.bfloat16(), grad_logp=f), lambda: bd.token_logp(z, i.cpu(), f),
                 lambda: bd.policy_loss(z, i, None, f), lambda: bd.policy_loss(z, i, f, f, old_logp=f.double()),
                 lambda: bd.preference_loss(z, i, f[:1], offsets=o[:2]), lambda: bd.preference_loss(z, i, f[:1]),
                 lambda: bd.preference_loss(z, i, f[:1], offsets=o.long()), lambda: bd.preference_loss(z, i, f[:2], offsets=o),
                 lambda: bd.preference_loss(z, i, f[:1], offsets=o, n_pairs=2),
                 lambda: bd.preference_loss(z, i, f[:1], offsets=o, out_scores=torch.zeros(2, 1, device=DEV))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: bd.token_logp(z, i), lambda: bd.token_logp(z, i, f, temperature=0.0),
                 lambda: bd.token_logp(z, i, f, grad_logits=torch.empty_like(z)), lambda: bd.policy_loss(z, i, f),
                 lambda: bd.policy_loss(z, i, f, f, clip_low=2.0), lambda: bd.preference_loss(z, i, f[:3], n_pairs=3),
                 lambda: bd.preference_loss(z, i, f[:1], offsets=o, beta=0.0),
                 lambda: bd.preference_loss(z, i, f[:1], offsets=o, workspace=torch.empty(8, dtype=torch.uint8, device=DEV)),
                 lambda: bd.token_logp(z[:0], i[:0], f[:0])):
        with pytest.raises(RafikiError):
            call()


def test_gradient_in_the_logits_place_is_refused():
    z, i, f = torch.zeros(4, 6, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(4, device=DEV)
    for call in (lambda: bd.token_logp(z, i, None, None, z, f), lambda: bd.policy_loss(z, i, f, None, z),
                 lambda: bd.preference_loss(z, i, None, z, n_pairs=2)):
        with pytest.raises(ValueError, match="read again"):
            call()
