"""How precise the losses over given tokens are, on the GPU against 64 bits: log-probabilities without a bias and a KL term that
keeps its digits next to the reference.

What 32 bits lose here, relative to a class's power 2^x, x = (z - the row's maximum) log2(e) / T in units of powers: the
difference and the product are rounded, 2^-24 |x| ln 2 each; the power is off by one unit, 2^-23; a chunk's additions by 2^-24 each,
three in a row; a move of a sum to another maximum, in a row and where its parts are joined, by a unit each.  Together
2^-23 (4.5 + |ln of the power|)."""
import math

import numpy as np
import pytest
import torch

from paper_1804_06087_amd import binding as bd

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
T = 0.71                                                     # log2(e) / T is 3e-8 of itself away from an fp32 number


def full(*shape, dtype=torch.float32):
    return torch.full(shape, -7, dtype=dtype, device=DEV)


def rows_of(n, C, dtype, gap, seed):
    """Logits [n, C] of a language model, and labels about `gap` T below the row's likeliest class."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.randn((n, C), device=DEV, generator=g) * 1.5
    at = torch.randint(0, C, (n, 40), device=DEV, generator=g)
    z.scatter_(1, at, 8 + 8 * torch.rand((n, 40), device=DEV, generator=g))
    labels = torch.randint(0, C, (n,), device=DEV, generator=g)
    z.scatter_(1, labels[:, None], z.amax(1, keepdim=True) - gap * T - torch.rand((n, 1), device=DEV, generator=g))
    return z.to(DT[dtype]), labels.int()


class Exact:
    """log p [n] of the labels in 64 bits, and the bound of a row's error by the rule above."""

    def __init__(self, z, labels, t=T):
        n = z.shape[0]
        self.logp, self.bound = (torch.empty(n, dtype=torch.float64, device=DEV) for _ in range(2))
        step = max(1, (1 << 26) // z.shape[1])
        for i in range(0, n, step):
            x = z[i:i + step].double() / t
            log_p = torch.log_softmax(x, 1)
            self.logp[i:i + step] = log_p.gather(1, labels[i:i + step, None].long())[:, 0]
            below = log_p.amax(1, keepdim=True) - log_p
            self.bound[i:i + step] = 2.0 ** -23 * (4.5 + (log_p.exp() * below.clamp(max=1e4)).sum(1))

    def check(self, delta):
        """Errors delta [n] of log p: every one within its row's bound; on average, since roundings go either way, within half a
        unit of the power (which may have a side) and four deviations of that average."""
        assert (delta.abs() <= self.bound).all(), (delta / self.bound).abs().max()
        deviation = self.bound.square().mean().sqrt().item() / math.sqrt(3 * delta.numel())
        assert abs(delta.mean().item()) <= 2.0 ** -24 + 4 * deviation, (delta.mean().item(), deviation)


# rows in a wave, in several, in many with the rest read again, and in parts
KINDS = [(500, 100), (500, 1000), (500, 2300), (300, 9000), (300, 30001), (64, 131071), (600, 50021), (600, 131072), (9, 200003)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C", KINDS)
@pytest.mark.parametrize("gap", [0.0, 4.0, 24.0])
def test_kl_next_to_the_reference(n, C, gap, dtype):
    """kl = exp(d) - d - 1 with d near 0.01: log p off by delta changes it by (exp(d) - 1) delta, and the fp32 result is rounded
    by 2^-24 of 5e-5, 3e-10 of log p."""
    z, labels = rows_of(n, C, dtype, gap, n + C)
    exact = Exact(z, labels)
    ref = (exact.logp + 0.01 * (1 + torch.rand(n, device=DEV, dtype=torch.float64))).float()
    d = ref.double() - exact.logp
    want = torch.expm1(d) - d
    for ent in (0.0, 0.01):
        for grad in (True, False):
            kl, loss = full(n), full(n)
            bd.policy_loss(z, labels, torch.ones(n, device=DEV), loss, torch.empty_like(z) if grad else None, ref_logp=ref,
                           out_kl=kl, temperature=T, kl_coef=0.1, entropy_coef=ent)
            exact.check((want - kl.double()) / torch.expm1(d))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C", KINDS)
def test_log_p_has_no_bias(n, C, dtype):
    z, labels = rows_of(n, C, dtype, 24.0, n + C + 1)
    exact = Exact(z, labels)
    for entropy in (True, False):
        logp = full(n)
        bd.token_logp(z, labels, logp, full(n) if entropy else None, temperature=T)
        rounded = exact.logp.abs().max().item() * 2.0 ** -24
        delta = logp.double() - exact.logp
        exact.bound += rounded
        exact.check(delta)
        exact.bound -= rounded


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C", KINDS)
def test_preference_scores_next_to_the_reference(n, C, dtype):
    """Scores of one token each: beta (log p - ref), whose fp32 rounding is 2^-24 of the difference."""
    n -= n % 2
    z, labels = rows_of(n, C, dtype, 24.0, n + C + 2)
    exact = Exact(z, labels)
    ref = exact.logp.float()
    scores = full(n // 2, 2)
    bd.preference_loss(z, labels, None, None, n_pairs=n // 2, ref_logp=ref, out_scores=scores, temperature=T, beta=0.5)
    exact.check(scores.double().view(-1) / 0.5 - (exact.logp - ref.double()))


# ---------------------------------------------------------------- entropy

HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


class ExactEntropy:
    """H [n] and its gradient [n, C] in 64 bits with their bounds.

    With weights w_c = 2^x_c off by rho_c relatively (the rule above; the maximum's x is 0, its power 1 and nothing of it is
    lost), H = ln sum w - sum w x ln 2 / sum w moves by sum p_c rho_c |1 - ln p_c - H|, ln sum w by sum p_c rho_c.  A chunk's
    moment is summed in fp32, at most 9 roundings of 2^-24 of what is a sum of one sign; H is rounded once.
    dH / dz_c = - p_c (log p_c + H) / T: a factor of two fp32 terms of the size of log p_c and H, and p_c with rho_c."""

    def __init__(self, z, t):
        x = z.double() / t
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        is_top = torch.zeros_like(x, dtype=torch.bool).scatter_(1, x.argmax(1, keepdim=True), True)
        rest = e.masked_fill(is_top, 0).sum(1, keepdim=True)
        log_p = (x - top) - torch.log1p(rest)
        p = log_p.exp()
        finite = torch.where(p > 0, log_p, 0)
        self.H = -(p * finite).sum(1)
        below = torch.where(p > 0, top - x, 0)
        rho = (2.0 ** -23 * (4.5 + below)).masked_fill(is_top, 0)
        lost = p * rho
        H = self.H[:, None]
        self.d_H = (lost * (1 + finite.abs() + H)).sum(1) + 9 * 2.0 ** -24 * (p * below).sum(1) + 2.0 ** -23 * self.H
        self.grad = torch.where(p > 0, -p * (finite + H), 0) / t
        shift = (self.d_H + lost.sum(1))[:, None]
        self.d_grad = p * ((rho + 2.0 ** -22) * (finite.abs() + H) + shift) / t

    def check(self, H, grad, dtype):
        assert (H >= 0).all()
        off = (H.double() - self.H).abs()
        assert (off <= self.d_H).all(), ((off / self.d_H).max(), self.H[(off / self.d_H).argmax()])
        off = (grad.double() - self.grad).abs()
        limit = self.d_grad * 1.01 + self.grad.abs() * HALF_STEP[dtype] + 1e-37
        assert (off <= limit).all(), ((off / limit).max(), (off / limit).argmax())


def check_entropy(z, labels, t, dtype):
    n = z.shape[0]
    exact = ExactEntropy(z, t)
    one = torch.ones(n, device=DEV)
    H, grad = full(n), torch.empty_like(z)
    bd.token_logp(z, labels, None, H, grad, None, one, temperature=t)
    exact.check(H, grad, dtype)
    bd.token_logp(z, labels, None, H, temperature=t)           # without a gradient
    exact.check(H, grad, dtype)
    # the policy loss takes the same: - H, without an advantage
    loss = full(n)
    bd.policy_loss(z, labels, 0 * one, loss, grad, out_entropy=H, temperature=t, entropy_coef=-1.0)
    exact.check(H, grad, dtype)
    assert torch.equal(loss, H)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C", [(64, 2), (64, 5), (64, 9), (64, 100), (48, 1000), (48, 2300), (300, 9000), (300, 30001), (600, 60000),
                                 (8, 131071), (3, 200003)])
def test_entropy_of_sure_rows(n, C, dtype):
    """One class far above a bulk, with the label that class, in the bulk, the first and the last one: H does not
    depend on it, is never negative and keeps its digits however small it is."""
    g = torch.Generator(device=DEV).manual_seed(C)
    base = torch.randn((n, C), device=DEV, generator=g)
    at = torch.randint(0, C, (n,), device=DEV, generator=g)
    at[0], at[-1] = 0, C - 1
    for gap in (6.0, 10.0, 14.0, 18.0, 22.0, 26.0, 28.0, 40.0):
        z = base.scatter(1, at[:, None], gap).to(DT[dtype])
        for labels in (at, torch.randint(0, C, (n,), device=DEV, generator=g), 0 * at, 0 * at + C - 1):
            check_entropy(z, labels.int(), 1.0, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C", KINDS)
def test_entropy(n, C, dtype):
    n = min(n, 150_000_000 // (C * 8) + 1) if n < 600 else n // 4
    z, labels = rows_of(n, C, dtype, 6.0, n + C + 3)
    check_entropy(z, labels, T, dtype)
    check_entropy(torch.zeros_like(z) + z[:, :1], labels, T, dtype)      # classes that are all alike


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_entropy_of_many_sure_rows(dtype):
    """Enough rows of each length that none goes in parts."""
    for n, C in ((9000, 700), (9000, 2000), (600, 5000), (600, 12000), (600, 30000), (800, 30001)):
        g = torch.Generator(device=DEV).manual_seed(C)
        z = torch.randn((n, C), device=DEV, generator=g)
        at = torch.randint(0, C, (n, 1), device=DEV, generator=g)
        z = z.scatter_(1, at, 6 + 30 * torch.rand((n, 1), device=DEV, generator=g)).to(DT[dtype])
        check_entropy(z, torch.randint(0, C, (n,), device=DEV, generator=g).int(), 1.0, dtype)


# ---------------------------------------------------------------- ratio

def test_ratio_next_to_the_clip():
    """Rows of C equal classes: log p = - ln C to 1e-15, and old that rounded to fp32, so that r - 1 is up to 1e-7.  With a clip
    on either side of it, r is clipped, and the gradient 0, or it is not."""
    for C in range(2, 60):
        logp = -math.log(C)
        old = np.float32(logp)
        step = math.expm1(logp - float(old))
        if abs(step) < 1e-9:
            continue
        z = torch.zeros((2, C), device=DEV)
        labels = torch.tensor([0, C - 1], dtype=torch.int32, device=DEV)
        A = torch.full((2,), math.copysign(1.0, step), device=DEV)
        for width, clipped in ((abs(step) / 2, True), (abs(step) * 2, False)):
            loss, grad = full(2), torch.empty_like(z)
            bd.policy_loss(z, labels, A, loss, grad, old_logp=torch.full((2,), float(old), device=DEV), clip_low=width,
                           clip_high=width)
            assert (grad == 0).all() if clipped else (grad != 0).all(), (C, step, width)


# ---------------------------------------------------------------- more rows than a launch takes

@pytest.mark.parametrize("n,C,dtype", [((1 << 20) + 5, 1100, "fp32"), ((1 << 20) + 5, 9001, "bf16"), ((1 << 25) + 37, 3, "fp32")])
def test_rows_of_a_second_launch(n, C, dtype):
    """A launch takes 2^20 workgroups: of one row each, or of 32 short ones.  All rows are one row of logits."""
    g = torch.Generator(device=DEV).manual_seed(C)
    z = (3 * torch.randn((1, C), device=DEV, generator=g)).to(DT[dtype])
    log_p = torch.log_softmax(z[0].double(), 0)
    H = -(log_p.exp() * log_p).sum()
    labels = torch.randint(-1, C, (n,), dtype=torch.int32, device=DEV, generator=g)
    logp, entropy = full(n), full(n)
    bd.token_logp(z.expand(n, C), labels, logp, entropy)
    want = torch.where(labels >= 0, log_p[labels.clamp(min=0).long()], 0)
    # the rule above with powers down to e^-40, and the results' own rounding, 2^-24 of 40
    assert (logp.double() - want).abs().max() <= 2.0 ** -23 * (4.5 + 40) + 2.0 ** -24 * 40
    assert (entropy.double() - torch.where(labels >= 0, H, 0)).abs().max() <= 2.0 ** -23 * (4.5 + 40) * (2 + H) * 2


# ---------------------------------------------------------------- gradients beside the logits

def test_gradient_over_the_logits_is_refused():
    """Rows of the gradient that share elements with rows of the logits: refused, however they meet; rows that lie between
    them are written."""
    n, C = 6, 40
    buf = torch.randn(4 * n * 100, device=DEV)
    at = lambda first, ld: buf.as_strided((n, C), (ld, 1), first)  # noqa: E731
    labels, f = torch.arange(n, dtype=torch.int32, device=DEV), torch.ones(n, device=DEV)
    for z, grad in ((at(0, 40), at(40, 40)), (at(40, 40), at(0, 40)), (at(0, 100), at(39, 100)), (at(0, 100), at(61, 100)),
                    (at(0, 100), at(500, 40)), (at(500, 40), at(0, 100)), (at(0, 0), at(39, 40)), (at(500, 17), at(0, 100))):
        for call in (lambda: bd.token_logp(z, labels, None, None, grad, f), lambda: bd.policy_loss(z, labels, f, None, grad),
                     lambda: bd.preference_loss(z, labels, None, grad, n_pairs=3)):
            with pytest.raises(ValueError, match="read again"):
                call()
    for z, grad in ((at(0, 100), at(40, 100)), (at(60, 100), at(0, 100)), (at(0, 40), at(240, 40)), (at(0, 0), at(40, 40)),
                    (at(0, 200), at(50, 400)), (at(0, 400), at(50, 200))):
        apart = torch.empty((n, C), device=DEV)
        bd.token_logp(z, labels, None, None, apart, f)
        bd.token_logp(z, labels, None, None, grad, f)
        assert torch.equal(grad, apart)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,chunks", [(4100, 129), (4100, 257), (4100, 448), (4100, 449), (4100, 1024), (4100, 1025), (4090, 1024), (600, 4095)])
def test_rows_at_the_borders_of_their_length(n, chunks, dtype):
    """Both sides of the numbers of rows and of 16-byte chunks at which a row takes other threads: every value by its bound."""
    V = 8 if dtype == "bf16" else 4
    for C in (chunks * V, chunks * V - 3):
        z, labels = rows_of(n, C, dtype, 4.0, n + C + 4)
        exact = Exact(z, labels)
        ref = (exact.logp + 0.02).float()
        d = ref.double() - exact.logp
        for ent in (0.0, 0.01):
            for grad in (True, False):
                kl = full(n)
                bd.policy_loss(z, labels, torch.ones(n, device=DEV), None, torch.empty_like(z) if grad else None, ref_logp=ref,
                               out_kl=kl, temperature=T, entropy_coef=ent)
                exact.check((torch.expm1(d) - d - kl.double()) / torch.expm1(d))
        check_entropy(z, labels, T, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [100, 900, 3000])
def test_rows_do_not_depend_on_their_neighbours(C, dtype):
    """Rows that share a wave: with other rows between them the even rows keep every bit of log p (through scores of one token and
    KL estimates, which show 1e-15 and 1e-10 of it), H and the gradient."""
    n = 4000
    z, labels = rows_of(n, C, dtype, 3.0, C)
    ref = Exact(z, labels).logp.float()
    one = torch.ones(n, device=DEV)

    def results(z, labels):
        scores, loss, kl, H, grad = full(n // 2, 2), full(n), full(n), full(n), torch.empty_like(z)
        bd.preference_loss(z, labels, None, None, n_pairs=n // 2, ref_logp=ref, out_scores=scores, temperature=T)
        bd.policy_loss(z, labels, one, loss, grad, ref_logp=ref + 0.01, out_kl=kl, out_entropy=H, temperature=T, entropy_coef=0.1)
        kl2 = full(n)
        bd.policy_loss(z, labels, one, None, None, ref_logp=ref + 0.01, out_kl=kl2, temperature=T)
        return [v.reshape(n, -1)[::2].clone() for v in (scores, loss, kl, H, grad, kl2)]

    first = results(z, labels)
    z[1::2], labels[1::2] = z[1::2].flip(0), labels[1::2].flip(0)
    for a, b in zip(first, results(z, labels)):
        assert torch.equal(a, b)
