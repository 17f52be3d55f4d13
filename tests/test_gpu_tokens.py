"""The vocabulary operators on the GPU against the 64-bit oracle: sampling, top-k, distillation with its
gradient, row quantisation and the 8-bit FC layer, at odd sizes, strides, masks and special values, on other
streams, in replayed graphs, and chained as a serving and training program chains them."""
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
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def lm_logits(rng, S, n, C, dtype, masked=True):
    """A bulk of unlikely classes, some likely ones, every third row half masked; values as stored in dtype."""
    z = rng.standard_normal((S, n, C)) * 1.5
    for i in range(n):
        likely = rng.integers(0, C, min(20, C))
        z[:, i, likely] += rng.random((S, likely.size)) * 12
        if masked and i % 3 == 2 and C > 1:
            m = rng.random(C) < 0.5
            m[rng.integers(0, C)] = False
            z[:, i, m] = -np.inf
    return torch.from_numpy(z.astype(np.float32)).to(DT[dtype])


def empty_sample(n):
    return torch.full((n,), -7, dtype=torch.int32, device=DEV), torch.full((n,), -7.0, device=DEV)


def check_sample(z, par, labels, probs):
    """Labels equal the oracle's; probabilities within one fp32 rounding and the 64-bit sums' (far below it)."""
    zh, lab, pr = host(z).astype(np.float64), host(labels), host(probs)
    for i in range(zh.shape[1]):
        get = lambda k, d: d if par.get(k) is None else par[k][i]  # noqa: E731
        label, p = ot.sample(zh[:, i], get("uniform", 0), float(get("temperature", 1.0)), int(get("top_k", 0)),
                             float(get("top_p", 1.0)), float(get("min_p", 0.0)))
        assert lab[i] == label, (i, lab[i], label, {k: v[i] for k, v in par.items() if v is not None})
        if math.isnan(p):
            assert math.isnan(pr[i])
        else:
            assert abs(pr[i] - p) <= 2.0 ** -23 * p, (i, pr[i], p)


def run_sample(z, par, **kw):
    n = z.shape[-2]
    labels, probs = empty_sample(n)
    bd.combine_sample(z, dev(par["uniform"]), labels, probs,
                      **{k: dev(v) for k, v in par.items() if k != "uniform" and v is not None}, **kw)
    torch.cuda.synchronize()
    return labels, probs


def mixed_params(rng, n):
    f = lambda a: np.asarray(a, np.float32)  # noqa: E731
    style = np.arange(n) % 6                  # plain, top-k, top-p, min-p, all, greedy
    return {"uniform": f(rng.random(n)), "temperature": f(np.where(style == 5, 0, 0.5 + rng.random(n))),
            "top_k": np.where((style == 1) | (style == 4), rng.integers(1, 60, n), 0).astype(np.int32),
            "top_p": f(np.where((style == 2) | (style == 4), 0.3 + 0.69 * rng.random(n), 1.0)),
            "min_p": f(np.where((style == 3) | (style == 4), 0.2 * rng.random(n), 0.0))}


# ---------------------------------------------------------------- sampling

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("S,n,C", [(1, 6, 1), (1, 6, 2), (2, 6, 63), (1, 12, 64), (3, 12, 65), (1, 12, 255),
                                   (2, 12, 256), (1, 12, 257), (3, 24, 1000), (1, 24, 4099), (32, 6, 300),
                                   (2, 12, 30001), (1, 12, 131073)])
def test_sample(S, n, C, dtype):
    rng = np.random.default_rng(S * 1000003 + n * 1009 + C)
    z = lm_logits(rng, S, n, C, dtype).to(DEV)
    par = mixed_params(rng, n)
    check_sample(z, par, *run_sample(z, par))


def test_sample_null_filters_are_off():
    rng = np.random.default_rng(1)
    z = lm_logits(rng, 2, 9, 777, "fp32").to(DEV)
    par = {"uniform": rng.random(9).astype(np.float32)}
    check_sample(z, par, *run_sample(z, par))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sample_flat_rows(dtype):
    """Nuclei of thousands of classes: hardly any class is likely, and bf16 leaves long runs of ties."""
    rng = np.random.default_rng(2)
    C = 40000
    z = torch.from_numpy((rng.standard_normal((1, 8, C)) * 0.3).astype(np.float32)).to(DT[dtype]).to(DEV)
    par = {"uniform": rng.random(8).astype(np.float32),
           "top_p": np.float32([0.5, 0.9, 0.99, 0.999, 0.3, 1.0, 1.0, 0.9]),
           "top_k": np.int32([0, 0, 0, 30000, 0, 5000, 20000, 1500]),
           "min_p": np.float32([0, 0, 0.1, 0, 0.5, 0.2, 0, 0])}
    check_sample(z, par, *run_sample(z, par))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("S,C", [(2, 40000), (3, 1025), (32, 5003)])
def test_sample_flat_rows_of_several_models(S, C, dtype):
    """The mean of several flat distributions; every fourth row holds few distinct values, so its cuts fall into ties."""
    rng = np.random.default_rng(S + C)
    z = (rng.standard_normal((S, 8, C)) * 0.3).astype(np.float32)
    z[:, 3::4] = np.round(z[:1, 3::4] * 2) / 2
    z = torch.from_numpy(z).to(DT[dtype]).to(DEV)
    par = {"uniform": rng.random(8).astype(np.float32),
           "temperature": np.float32([1, 0.7, 2, 1, 1, 1, 0, 1]),
           "top_p": np.float32([0.5, 0.9, 0.99, 1.0, 0.3, 1.0, 1.0, 1.0]),
           "top_k": np.int32([0, C - 1, C - 100, C // 2, 0, C // 2, 5000, 1024]),
           "min_p": np.float32([0, 0, 0.1, 0, 0.5, 0.2, 0, 0])}
    check_sample(z, par, *run_sample(z, par))


def test_sample_ties_are_cut_by_index():
    """Rows of few distinct values: top-k, top-p and min-p cut inside runs of equal classes.  All sums are exact
    (powers of two), so every border is exact too."""
    C = 4096
    z = torch.zeros((1, 8, C), device=DEV)
    par = {"uniform": np.float32([0, 0.25, 0.5, 0.999, 0.75, 0.5, 0.5, 0.0]),
           "top_k": np.int32([7, 1000, 0, 0, 0, 2048, 0, 1]),
           "top_p": np.float32([1, 1, 0.5, 0.25, 2.0 ** -13, 0.5, 1, 1]),
           "min_p": np.float32([0, 0, 0, 0, 0, 1.0, 5.0, 0])}
    labels, probs = run_sample(z, par)
    # kept: 7, 1000, 2048, 1024, 1, 1024 (half of 2048), all, 1
    assert host(labels).tolist() == [0, 250, 1024, 1022, 0, 512, 2048, 0]
    assert np.allclose(host(probs), [1 / 7, 1 / 1000, 1 / 2048, 1 / 1024, 1, 1 / 1024, 1 / 4096, 1], rtol=2.0 ** -23, atol=0)


def test_sample_greedy_rows_of_equal_classes():
    """More equal first classes than any list holds: the lowest index, with and without filters."""
    z = torch.zeros((2, 3, 5000), device=DEV)
    z[:, 1, :7] = -1.0
    z[:, 2] = -math.inf
    z[:, 2, 1234:4000] = 2.0
    for par in ({}, {"top_k": np.int32([50] * 3)}, {"top_p": np.float32([0.0] * 3)}):
        par = {"uniform": np.float32([0.9] * 3), "temperature": np.float32([0] * 3), **par}
        labels, probs = run_sample(z, par)
        assert host(labels).tolist() == [0, 7, 1234] and host(probs).tolist() == [1, 1, 1]


def test_sample_special_rows():
    lowest = float(torch.finfo(torch.float32).min)
    C = 500
    z = torch.zeros((2, 14, C), device=DEV)
    z[:, 0] = -math.inf                        # masked out altogether
    z[1, 1] = -math.inf                        # one model masked out
    z[0, 2, 499] = math.nan
    z[1, 3, 0] = math.inf
    z[:, 4] = lowest                           # all at the type's lowest value: uniform
    z[:, 5] = lowest
    z[:, 5, 77] = 0.0                          # all but one at the lowest value
    z[:, 6] = -math.inf
    z[:, 6, 13] = -3.0                         # one class left
    z[0, 7, 5], z[0, 7, 6] = 3e38, -3e38       # the range of the type
    par = {"uniform": np.float32([.5, .5, .5, .5, .5, .5, .5, .5, 1.0, math.nan, -1.0, .5, .5, .5]),
           "temperature": np.float32([1, 1, 1, 1, .01, .01, 1, 1, 1, 1, 1, math.nan, -1, math.inf])}
    labels, probs = run_sample(z, par)
    check_sample(z, par, labels, probs)
    lab, pr = host(labels), host(probs)
    assert lab[[0, 1, 2, 3, 11, 12]].tolist() == [-1] * 6
    assert pr[0] == 0 and pr[1] == 0 and np.isnan(pr[[2, 3, 11, 12]]).all()
    assert lab[[4, 5, 6, 8, 9, 10, 13]].tolist() == [250, 77, 13, 499, 0, 0, 250]


def test_sample_temperatures_and_infinite_temperature_with_a_mask():
    rng = np.random.default_rng(9)
    z = lm_logits(rng, 2, 6, 900, "fp32")
    par = {"uniform": rng.random(6).astype(np.float32),
           "temperature": np.float32([1e-3, 1e-30, 50.0, 1e30, math.inf, 0.0])}
    z = z.to(DEV)
    check_sample(z, par, *run_sample(z, par))


def test_sample_strided_unaligned_and_broadcast():
    rng = np.random.default_rng(3)
    S, n, C = 3, 7, 1001
    z = lm_logits(rng, S, n, C, "bf16")
    par = mixed_params(rng, n)
    buf = torch.zeros(S * n * 1100 * 2 + 3, dtype=torch.bfloat16, device=DEV)
    v = buf[3:].as_strided((S, n, C), (1100, 1100 * S + 1, 1))       # row-major by request, odd distances
    v.copy_(z)
    check_sample(v, par, *run_sample(v, par))
    one = z[:1].to(DEV).expand(S, n, C)                                # one model's rows for all members
    check_sample(one, par, *run_sample(one, par))
    row = z[:, :1].to(DEV).expand(S, n, C)                             # one row for all requests
    check_sample(row, par, *run_sample(row, par))
    two_dims = z[0].to(DEV)
    check_sample(two_dims[None], par, *run_sample(two_dims, par))


def test_sample_offsets_past_32_bits():
    """Rows more than 2^31 elements from the first."""
    rng = np.random.default_rng(4)
    n, C, ld = 4, 5000, (1 << 30) - 3
    buf = torch.empty(3 * ld + C, dtype=torch.bfloat16, device=DEV)
    v = buf.as_strided((1, n, C), (0, ld, 1))
    v.copy_(lm_logits(rng, 1, n, C, "bf16"))
    par = mixed_params(rng, n)
    check_sample(v, par, *run_sample(v, par))
    labels = torch.empty((n, 5), dtype=torch.int32, device=DEV)
    logp = torch.empty((n, 5), device=DEV)
    bd.combine_topk(v, labels, logp)
    torch.cuda.synchronize()
    check_topk(v, 5, 1.0, labels, logp)


def test_sample_leaves_the_rest_alone():
    """Outputs are views into larger buffers: nothing around them changes, nor do the inputs."""
    rng = np.random.default_rng(6)
    z = lm_logits(rng, 2, 5, 600, "fp32").to(DEV)
    before = z.clone()
    lab, pr = torch.full((9,), 42, dtype=torch.int32, device=DEV), torch.full((9,), 42.0, device=DEV)
    bd.combine_sample(z, torch.rand(5, device=DEV), lab[2:7], pr[2:7])
    need = bd.combine_workspace(2, 5, 600)
    ws = torch.full((need + 64,), 9, dtype=torch.uint8, device=DEV)
    bd.combine_sample(z, torch.rand(5, device=DEV), lab[2:7], pr[2:7], workspace=ws[16:16 + need])
    torch.cuda.synchronize()
    assert torch.equal(z, before)
    assert (lab[[0, 1, 7, 8]] == 42).all() and (pr[[0, 1, 7, 8]] == 42).all() and (lab[2:7] >= 0).all()
    assert (ws[:16] == 9).all() and (ws[16 + need:] == 9).all()


# ---------------------------------------------------------------- top-k

def check_topk(z, k, t, labels, logp):
    zh, lab, lp = host(z).astype(np.float64), host(labels), host(logp)
    for i in range(zh.shape[1]):
        want, want_lp = ot.topk(zh[:, i], k, t)
        assert np.array_equal(lab[i], want), (i, lab[i], want)
        # one fp32 rounding of log p; the 64-bit p is off by some 1e-14, which log p near 0 shows as such
        with np.errstate(invalid="ignore"):
            ok = (np.abs(lp[i] - want_lp) <= 2.0 ** -23 * np.abs(want_lp) + 1e-12) | (lp[i] == want_lp)
        assert (ok | (np.isnan(lp[i]) & np.isnan(want_lp))).all(), (i, lp[i], want_lp)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("S,n,C,k,t", [(1, 4, 1, 1, 1.0), (1, 5, 7, 9, 2.0), (3, 64, 1000, 5, 1.0), (2, 5, 64, 64, 0.5),
                                       (1, 6, 300, 257, 1.0), (2, 7, 50021, 20, 1.0), (1, 5, 131072, 64, 3.0),
                                       (32, 4, 513, 33, 1.0), (1, 4, 20000, 1024, 1.0), (4, 3, 9000, 1023, 0.7),
                                       (1, 3, 700, 1024, 1.0)])
def test_topk(S, n, C, k, t, dtype):
    rng = np.random.default_rng(S * 31 + n * 17 + C + k)
    z = lm_logits(rng, S, n, C, dtype).to(DEV)
    labels = torch.full((n, k), -7, dtype=torch.int32, device=DEV)
    logp = torch.full((n, k), -7.0, device=DEV)
    bd.combine_topk(z, labels, logp, temperature=t)
    torch.cuda.synchronize()
    check_topk(z, k, np.float32(t), labels, logp)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("S,C,k", [(3, 5003, 1024), (2, 40000, 1000), (32, 2500, 900), (1, 1025, 1024)])
def test_topk_flat_rows_of_several_models(S, C, k, dtype):
    """The k-th class among thousands of nearly equal ones; the last row's k-th class is one of many equal ones."""
    rng = np.random.default_rng(61 + S)
    z = (rng.standard_normal((S, 4, C)) * 0.01).astype(np.float32)
    z[:, 3] = np.round(z[:1, 3] * 50) / 50
    z = torch.from_numpy(z).to(DT[dtype]).to(DEV)
    labels = torch.full((4, k), -7, dtype=torch.int32, device=DEV)
    logp = torch.full((4, k), -7.0, device=DEV)
    bd.combine_topk(z, labels, logp)
    torch.cuda.synchronize()
    check_topk(z, k, 1.0, labels, logp)


def test_topk_ties_order_and_special_rows():
    C, k = 3000, 600
    z = torch.zeros((1, 8, C), device=DEV)
    z[0, 1] = torch.arange(C, device=DEV) % 3                 # three values, cut inside the second
    z[0, 2] = -math.inf
    z[0, 3, 10:20] = math.nan
    z[0, 4] = -math.inf
    z[0, 4, [2999, 5, 1000]] = torch.tensor([1.0, 1.0, 2.0], device=DEV)
    z[0, 5] = torch.arange(C, device=DEV).float() * 0.5        # ascending; most have no probability to speak of
    z[0, 6] = -torch.arange(C, device=DEV).float() * 3         # below 2^-1000 from class 232 on
    z[0, 7] = torch.finfo(torch.float32).min
    labels = torch.empty((8, k), dtype=torch.int32, device=DEV)
    logp = torch.empty((8, k), device=DEV)
    bd.combine_topk(z, labels, logp)
    torch.cuda.synchronize()
    check_topk(z, k, 1.0, labels, logp)
    assert labels[4, :4].tolist() == [1000, 5, 2999, -1] and (labels[2] == -1).all() and (labels[3] == -1).all()


@pytest.mark.parametrize("S", [1, 2, 32])
@pytest.mark.parametrize("k", [300, 430, 440, 446, 700])
def test_topk_far_below_the_best(S, k):
    """Probabilities over more octaves than fp32 has: 0.29 octaves a class (0.58 from class 600 on), in 79 groups."""
    C = 5000
    c = torch.arange(C, device=DEV).float()
    z = torch.stack([-(c * 0.2 + torch.relu(c - 600) * 0.2)] * S)[:, None].repeat(1, 2, 1)
    z[:, 1] = z[:, 1].flip(-1)
    labels = torch.empty((2, k), dtype=torch.int32, device=DEV)
    logp = torch.empty((2, k), device=DEV)
    bd.combine_topk(z.contiguous(), labels, logp)
    torch.cuda.synchronize()
    check_topk(z, k, 1.0, labels, logp)


# ---------------------------------------------------------------- distillation

def teacher(rng, n, C, k, rest):
    ids = np.stack([rng.permutation(C)[:k] if k <= C else rng.integers(0, C, k) for _ in range(n)]).astype(np.int32)
    t = rng.standard_normal((n, k)) * 2
    logp = t - np.log(np.exp(t).sum(1, keepdims=True)) + np.log(0.6 + 0.39 * rng.random((n, 1)))
    return ids, logp.astype(np.float32)


def distill_bounds(z, C, k, t, q_total, dtype):
    """What 32 bits lose, for one row: x = z / t and the log of the sum are off by 2^-22 of their size in units of
    the exponent, a sum of C terms in runs of C / 1024 and trees by (C / 1024 + k + 64) 2^-24, exp and log by a few
    2^-23; everything multiplies terms of at most Q + 1."""
    fin = z[np.isfinite(z)]
    x = np.abs(fin).max() / t + math.log(C) if fin.size else 0.0
    return 2.0 ** -22 * (2 * x + 8) + (C / 1024 + k + 64) * 2.0 ** -24


def run_distill(z, ids, logp, t, rest, g=None, loss=True, grad=True, **kw):
    n = z.shape[0]
    out = torch.full((n,), -7.0, device=DEV) if loss else None
    d = torch.full(z.shape, -7.0, dtype=z.dtype, device=DEV) if grad else None
    bd.distill_loss(z, dev(ids), dev(logp), out, d, grad_loss=None if g is None else dev(g), temperature=t, rest=rest, **kw)
    torch.cuda.synchronize()
    return out, d


def check_distill(z, ids, logp, t, rest, g, loss, grad, dtype):
    zh = host(z).astype(np.float64)
    n, C = zh.shape
    for i in range(n):
        gi = 1.0 if g is None else float(g[i])
        want, want_d = ot.distill(zh[i], ids[i], logp[i], float(np.float32(t)), rest, gi)
        valid = (ids[i] >= 0) & (ids[i] < C)
        q = np.exp(logp[i][valid].astype(np.float64)).sum() + 1 if rest else 1.0
        eps = distill_bounds(zh[i], C, ids.shape[1], t, q, dtype)
        if loss is not None:
            got = float(loss[i])
            if math.isfinite(want):
                size = 1 + (np.abs(logp[i][valid]).max() if valid.any() else 0)
                # the teacher's mass 1 - sum q of the rest is itself off by k 2^-24, times log p_r
                assert abs(got - want) <= t * t * (q + 1) * size * (eps + ids.shape[1] * 2.0 ** -24 * 40), (i, got, want)
            else:
                assert got == want or (math.isnan(got) and math.isnan(want)), (i, got, want)
        if grad is not None:
            got = host(grad[i]).astype(np.float64)
            if np.isnan(want_d).any():
                assert np.isnan(got).all(), i
                continue
            # relative to each of the terms: Q p_c, q_c, q_r p_c / p_r
            lse = ot._lse(zh[i] / t)
            terms = np.exp(zh[i] / t - lse) * (q + 1) + np.abs(want_d) / max(t * abs(gi), 1e-300)
            np.add.at(terms, ids[i][valid], np.exp(logp[i][valid].astype(np.float64)) if rest else 1.0)
            limit = t * abs(gi) * terms * (2 * eps + ids.shape[1] * 2.0 ** -22) + np.abs(want_d) * HALF_STEP[dtype] + 1e-37
            bad = np.abs(got - want_d) > limit
            assert not bad.any(), (i, np.nonzero(bad)[0][:5], got[bad][:5], want_d[bad][:5])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,C,k,t", [(3, 1, 1, 1.0), (5, 2, 1, 2.0), (4, 33, 33, 1.0), (6, 64, 7, 0.5), (8, 1000, 5, 2.0),
                                     (3, 1025, 100, 1.0), (5, 30000, 32, 2.0), (3, 131071, 64, 1.0), (2, 160001, 256, 2.0),
                                     (3, 5000, 1024, 1.5), (2, 10, 40, 1.0)])
def test_distill(n, C, k, t, dtype, rest):
    rng = np.random.default_rng(n * 7 + C + k)
    z = lm_logits(rng, 1, n, C, dtype, masked=False)[0].to(DEV)
    ids, logp = teacher(rng, n, C, k, rest)
    g = (rng.random(n) - 0.3).astype(np.float32)
    g[0] = 0
    loss, grad = run_distill(z, ids, logp, t, rest, g)
    check_distill(z, ids, logp, t, rest, g, loss, grad, dtype)
    # each output alone gives the same bits
    assert torch.equal(run_distill(z, ids, logp, t, rest, g, grad=False)[0], loss)
    assert torch.equal(run_distill(z, ids, logp, t, rest, g, loss=False)[1], grad)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("chunks", [256, 1024, 2048, 4096, 8192, 16384, 20480])
def test_distill_at_every_row_length(chunks, dtype, rest):
    """Both sides of each number of 16-byte chunks at which a row takes more threads or registers; of the odd
    lengths every row starts at another alignment."""
    V = 8 if dtype == "bf16" else 4
    for C in (chunks * V + V + 1, chunks * V + V + 2):
        test_distill(3, C, 9, 1.5, dtype, rest)


@pytest.mark.parametrize("rest", [False, True])
def test_distill_slots_empty_repeated_and_masked(rest):
    rng = np.random.default_rng(21)
    n, C, k = 9, 300, 6
    z = lm_logits(rng, 1, n, C, "fp32", masked=False)[0]
    ids, logp = teacher(rng, n, C, k, rest)
    ids[0] = -1                                          # no teacher
    ids[1, 2:] = -1                                      # few slots
    ids[2] = 17                                          # one class in every slot
    ids[3, :3], ids[3, 3:] = C, C + 100                  # beyond the vocabulary: empty
    z[4, ::2] = -math.inf                                # a masked student, some teacher classes among the masked
    ids[4] = [1, 3, 5, 7, 9, 11]
    z[5, 100:] = -math.inf
    ids[5] = [200, 1, 2, 3, 4, 5]                        # p = 0 where the teacher has mass: infinite loss
    logp[6, 1:] = -math.inf                              # slots without mass
    z[7] = -math.inf
    z[7, ids[7]] = 1.0                                   # the others have no probability
    z[8] = -math.inf                                     # nothing left
    z = z.to(DEV)
    loss, grad = run_distill(z, ids, logp, 1.3, rest)
    check_distill(z, ids, logp, 1.3, rest, None, loss, grad, "fp32")
    if not rest:
        assert loss[0] == 0 and (grad[0] == 0).all() and loss[3] == 0
    assert math.isinf(float(loss[5])) and torch.isnan(loss[8])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [5, 700, 90001])
def test_distill_masks_of_the_lowest_value(C, dtype, rest):
    """Rows masked with the type's lowest value: one of nothing else is uniform; the rest has p = 0.  Scores 0 and
    powers 1 are exact: what is left are sums of equal terms (2^-24 an addition, C / 1024 + 64 of them), quotients
    and log2 C (2^-22 relative), times the T^2 (Q + 1) of the formula.  Row 1's other classes are equal, so that
    p_c / p_r = 1 / (C - 2) however small p_r is; its log is finite as long as fp32 holds the difference of the
    logits over T, in powers of 2."""
    z = torch.full((3, C), float(torch.finfo(DT[dtype]).min), dtype=DT[dtype], device=DEV)
    z[1, 2] = z[1, C - 1] = 1.0
    z[2] = float(torch.finfo(DT[dtype]).max)
    ids = np.int32([[2, C - 1]] * 3)
    logp = np.log(np.float32([[0.5, 0.25]] * 3))
    for t in (0.5, 2.0):
        loss, grad = run_distill(z, ids, logp, t, rest)
        q = np.float64([0.5, 0.25]) if rest else np.float64([2 / 3, 1 / 3])
        q_r = 0.25 if rest else 0.0
        eps = (C / 1024 + 64) * 2.0 ** -24 + 2.0 ** -20
        for i, p in ((0, 1 / C), (1, 0.5), (2, 1 / C)):
            want = (q * (np.log(q) - math.log(p))).sum()
            other = (C - 2) * p if i != 1 else 0.0
            if rest:
                log_other = math.log(other) if i != 1 else (float(z[1, 0]) - 1.0) / t
                if -log_other / math.log(2) > torch.finfo(torch.float32).max:
                    log_other = -math.inf
                want += q_r * (math.log(q_r) - log_other)
            got = float(loss[i])
            limit = t * t * 2 * max(math.log(4 * C), abs(want)) * eps if math.isfinite(want) else 0.0
            assert got == t * t * want or abs(got - t * t * want) <= limit, (i, got, want)
            d = host(grad[i]).astype(np.float64)
            assert np.abs(d[ids[i]] - t * (p - q)).max() <= t * (eps * 2 + HALF_STEP[dtype]), i
            outside = np.delete(d, ids[i])
            wanted = t * (other - q_r) / (C - 2)
            assert np.abs(outside - wanted).max() <= t * 2 * eps / C + abs(wanted) * HALF_STEP[dtype], (i, wanted)


def test_distill_smallest_and_largest_temperatures():
    """T so small that one class has all, and so large that all classes are alike."""
    z = torch.tensor([[1.0, 3.0, 2.0, -math.inf], [0.0, 0.0, 0.0, 0.0]], device=DEV)
    ids, logp = np.int32([[1], [1]]), np.float32([[0.0], [0.0]])
    loss, grad = run_distill(z, ids, logp, 1e-39, False)
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all() and float(loss[0]) == 0 and (grad[0] == 0).all()
    loss, grad = run_distill(z, ids, logp, 1e19, False)
    for i, n in ((0, 3), (1, 4)):
        assert abs(float(loss[i]) / 1e38 - math.log(n)) <= 2.0 ** -20
        want = np.array([1 / n, 1 / n - 1, 1 / n, 1 / n if n == 4 else 0.0])
        assert np.abs(host(grad[i]) / 1e19 - want).max() <= 2.0 ** -20


@pytest.mark.parametrize("rest", [False, True])
def test_distill_not_finite(rest):
    rng = np.random.default_rng(22)
    z = lm_logits(rng, 1, 5, 700, "fp32", masked=False)[0]
    ids, logp = teacher(rng, 5, 700, 4, rest)
    z[0, 600] = math.nan
    z[1, 3] = math.inf
    logp[2, 1] = math.nan
    z[3, 5] = math.nan                                   # of no weight: no gradient
    g = np.float32([1, 1, 1, 0, 1])
    z = z.to(DEV)
    loss, grad = run_distill(z, ids, logp, 1.0, rest, g)
    assert torch.isnan(loss[:4]).all() and torch.isfinite(loss[4])
    assert torch.isnan(grad[:3]).all() and (grad[3] == 0).all() and torch.isfinite(grad[4]).all()


def test_distill_tail_of_a_sure_student():
    """p_r far below fp32's 1 - sum p: the rest's own sum keeps it."""
    C = 2000
    z = torch.full((1, C), -30.0, device=DEV)
    z[0, 3], z[0, 8] = 10.0, 9.0
    ids, logp = np.int32([[3, 8]]), np.log(np.float32([[0.6, 0.3]]))
    loss, grad = run_distill(z, ids, logp, 1.0, True)
    check_distill(z, ids, logp, 1.0, True, None, loss, grad, "fp32")
    assert float(loss[0]) > 0.1 * 30 * 0.9


@pytest.mark.parametrize("rest", [False, True])
def test_distill_gradient_against_differences(rest):
    """The kernel's gradient against central differences of the 64-bit loss."""
    rng = np.random.default_rng(23)
    C, k, t, h = 40, 5, 1.5, 1e-5
    z = rng.standard_normal((1, C)).astype(np.float32)
    ids, logp = teacher(rng, 1, C, k, rest)
    _, grad = run_distill(dev(z), ids, logp, t, rest)
    z64 = z[0].astype(np.float64)
    for c in range(C):
        up, down = z64.copy(), z64.copy()
        up[c] += h
        down[c] -= h
        diff = (ot.distill(up, ids[0], logp[0], t, rest)[0] - ot.distill(down, ids[0], logp[0], t, rest)[0]) / (2 * h)
        assert abs(diff - float(grad[0, c])) < 4e-6       # fp32 terms of at most 1.5, some ten roundings; 1e-9 of differences


def test_distill_strided_unaligned_and_broadcast():
    rng = np.random.default_rng(24)
    n, C, k = 6, 1003, 9
    z = lm_logits(rng, 1, n, C, "bf16", masked=False)[0]
    ids, logp = teacher(rng, n, C, k, True)
    buf = torch.zeros(n * 1111 + 5, dtype=torch.bfloat16, device=DEV)
    v = buf[1:].as_strided((n, C), (1111, 1))
    v.copy_(z)
    gbuf = torch.full((n * 1207 + 7,), 42.0, dtype=torch.bfloat16, device=DEV)
    gv = gbuf[3:].as_strided((n, C), (1207, 1))
    loss = torch.empty(n, device=DEV)
    bd.distill_loss(v, dev(ids), dev(logp), loss, gv, temperature=1.0, rest=True)
    torch.cuda.synchronize()
    check_distill(v, ids, logp, 1.0, True, None, loss, gv, "bf16")
    outside = torch.ones_like(gbuf, dtype=torch.bool)
    outside[3:].as_strided((n, C), (1207, 1)).fill_(False)
    assert (gbuf[outside] == 42).all()                   # nothing written between the rows
    same = z[:1].to(DEV).expand(n, C)
    loss, grad = run_distill(same, ids, logp, 1.0, True)
    check_distill(same, ids, logp, 1.0, True, None, loss, grad, "bf16")


def test_distill_largest_vocabulary():
    rng = np.random.default_rng(25)
    C = 1 << 20
    z = lm_logits(rng, 1, 2, C, "bf16", masked=False)[0].to(DEV)
    ids, logp = teacher(rng, 2, C, 16, True)
    loss, grad = run_distill(z, ids, logp, 2.0, True)
    check_distill(z, ids, logp, 2.0, True, None, loss, grad, "bf16")
    par = mixed_params(rng, 2)
    check_sample(z[None], par, *run_sample(z, par))


# ---------------------------------------------------------------- 8-bit FC

def padded(a, pad=None, fill=0):
    """int8 matrix on the GPU as a view of a wider one whose padding holds `fill`."""
    n, c = a.shape
    wide = torch.full((n, (c + 15) // 16 * 16 if pad is None else pad), fill, dtype=torch.int8, device=DEV)
    wide[:, :c] = torch.from_numpy(a).to(DEV)
    return wide[:, :c]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 5), (4, 64), (7, 1000), (2, 4096), (33, 2048), (1, 25088), (5, 12289)])
def test_quantize(n, c, dtype):
    rng = np.random.default_rng(n * 100 + c)
    x = torch.from_numpy((rng.standard_normal((n, c)) * 3).astype(np.float32)).to(DT[dtype])
    if n > 2:
        x[1] = 0
        x[2, c // 2:] = x[2, 0] * 0.5                    # ties where the largest is x[2, 0]
    xh = host(x)
    want_q, want_s = ot.quantize_rows(xh)
    buf = torch.full((n, c + 11), 99, dtype=torch.int8, device=DEV)
    scale = torch.empty(n, device=DEV)
    bd.quantize_rows_i8(x.to(DEV), buf[:, :c], scale)
    torch.cuda.synchronize()
    assert np.array_equal(host(scale), want_s)
    assert np.array_equal(buf[:, :c].cpu().numpy(), want_q)
    assert (buf[:, c:] == 99).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("c", [8192, 8193, 28672, 28673, 60001, 131071])
def test_quantize_long_rows(c, dtype):
    test_quantize(3, c, dtype)


def test_quantize_special_rows():
    x = np.zeros((8, 37), np.float32)
    x[0, 5] = np.nan
    x[1, 36] = -np.inf
    x[2, :] = 1e-40                                       # below the smallest scale
    x[3, :5] = [127, 0.5, 1.5, -2.5, 63.5]                # scale 1, ties to even
    x[4, 0] = 3.4e38
    x[5, :3] = [3e-37, -1.5e-37, 1e-38]
    x[6, :4] = [1.0, 0.5, -0.5, 0.25]
    x[7, :] = np.float32(1.1) * np.arange(37)
    want_q, want_s = ot.quantize_rows(x)
    q, s = torch.full((8, 37), 99, dtype=torch.int8, device=DEV), torch.empty(8, device=DEV)
    bd.quantize_rows_i8(dev(x), q, s)
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(host(s), want_s, equal_nan=True)
    assert q[3, :5].tolist() == [127, 0, 2, -2, 64]


def check_fc(x, sx, w, sw, bias, relu, y, dtype):
    acc = np.abs(x.astype(np.float64) @ w.astype(np.float64).T) * (sx[:, None].astype(np.float64) * sw)
    want = ot.fc_i8(x, sx, w, sw, bias, relu)
    # int to fp32, two products, one sum: half a step each; then the stored value
    limit = 3 * 2.0 ** -24 * acc + (2.0 ** -24 + HALF_STEP[dtype]) * np.abs(want) * 1.01 + 1e-37
    limit += 2.0 ** -24 * (0 if bias is None else np.abs(bias)[None, :])
    got = host(y).astype(np.float64)
    bad = np.abs(got - want) > limit
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


FC_SIZES = [(1, 1, 1), (1, 16, 5), (2, 17, 16), (5, 63, 33), (16, 64, 64), (17, 100, 65), (1, 4096, 4096), (3, 4097, 1000),
            (64, 2048, 1000), (33, 25088, 257), (130, 300, 129), (256, 512, 256), (257, 511, 300), (128, 4096, 30000),
            (1000, 1111, 777), (31, 64, 4096), (300, 16, 300), (8, 131071, 40), (512, 1024, 2048), (1, 8192, 3)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,c_in,c_out", FC_SIZES)
def test_fc(n, c_in, c_out, dtype):
    rng = np.random.default_rng(n + c_in * 3 + c_out * 7)
    x = rng.integers(-128, 128, (n, c_in), dtype=np.int8)
    w = rng.integers(-128, 128, (c_out, c_in), dtype=np.int8)
    sx, sw = rng.random(n).astype(np.float32) + 0.5, rng.random(c_out).astype(np.float32) * 0.01
    bias = None if c_out % 3 == 0 else rng.standard_normal(c_out).astype(np.float32)
    relu = c_out % 2 == 1
    buf = torch.full((n, c_out + 3), 42.0, dtype=DT[dtype], device=DEV)
    y = buf[:, :c_out]
    bd.fc_i8(padded(x, fill=77), dev(sx), padded(w, fill=-55), dev(sw), y, bias=None if bias is None else dev(bias),
             relu=relu)
    torch.cuda.synchronize()
    check_fc(x, sx, w, sw, bias, relu, y, dtype)
    assert (buf[:, c_out:] == 42).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,c_in,c_out", [(4100, 130, 4200), (3841, 256, 4351), (2050, 300, 2049), (4097, 17, 4097)])
def test_fc_many_tiles(n, c_in, c_out, dtype):
    """Enough rows and columns for the larger tiles, with ragged edges and K ends inside a chunk."""
    test_fc(n, c_in, c_out, dtype)


def test_fc_extremes():
    """The largest sums: -128 * -128 over 131071 terms is 2^31 - 2^14."""
    x = np.full((2, 131071), -128, np.int8)
    w = np.full((3, 131071), -128, np.int8)
    w[1] = 127
    y = torch.empty((2, 3), device=DEV)
    one = lambda n: torch.ones(n, device=DEV)  # noqa: E731
    bd.fc_i8(padded(x), one(2), padded(w), one(3), y)
    torch.cuda.synchronize()
    check_fc(x, np.ones(2, np.float32), w, np.ones(3, np.float32), None, False, y, "fp32")


def test_fc_strides_and_nan_scale():
    rng = np.random.default_rng(31)
    n, c_in, c_out = 40, 200, 90
    x = rng.integers(-128, 128, (n, c_in), dtype=np.int8)
    w = rng.integers(-128, 128, (c_out, c_in), dtype=np.int8)
    sx, sw = rng.random(n).astype(np.float32), rng.random(c_out).astype(np.float32)
    buf = torch.full((n * 101 + 9,), 42.0, dtype=torch.bfloat16, device=DEV)
    y = buf[1:].as_strided((n, c_out), (101, 1))          # odd distances, odd start
    bd.fc_i8(padded(x, 320), dev(sx), padded(w, 1024), dev(sw), y)
    torch.cuda.synchronize()
    check_fc(x, sx, w, sw, None, False, y, "bf16")
    sx[3] = np.nan
    out = torch.empty((n, c_out), device=DEV)
    bd.fc_i8(padded(x, 320), dev(sx), padded(w, 1024), dev(sw), out, relu=True)
    torch.cuda.synchronize()
    assert torch.isnan(out[3]).all() and torch.isfinite(out[4:]).all()


def test_refusals_on_the_device():
    z, i, f = torch.zeros(2, 3, 50, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, device=DEV)
    with pytest.raises(ValueError):
        bd.combine_sample(z.transpose(1, 2), f, i, f)          # classes not contiguous
    with pytest.raises(ValueError):
        bd.combine_sample(z.half(), f, i, f)
    with pytest.raises(ValueError):
        bd.combine_sample(z, f, i, f, top_k=f)                 # a filter of the wrong type
    with pytest.raises(ValueError):
        bd.combine_sample(z, f[:2], i, f)
    with pytest.raises(RafikiError):
        bd.combine_sample(z, f, i, f, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(RafikiError):
        bd.combine_topk(z, torch.zeros((3, 2), dtype=torch.int32, device=DEV), torch.zeros((3, 2), device=DEV), temperature=0.0)
    with pytest.raises(ValueError):
        bd.distill_loss(z[0], i.view(3, 1), f.view(3, 1), grad_logits=z[0].bfloat16())
    with pytest.raises(RafikiError):
        bd.distill_loss(z[0], i.view(3, 1), f.view(3, 1))       # no output
    q = torch.zeros((3, 50), dtype=torch.int8, device=DEV)
    with pytest.raises((RafikiError, ValueError)):
        bd.fc_i8(q, f, q, f, torch.zeros((3, 3), device=DEV))   # rows of 50 bytes
    w = torch.zeros(3 * 64 - 10, dtype=torch.int8, device=DEV).as_strided((3, 50), (64, 1))
    with pytest.raises(ValueError):
        bd.fc_i8(w, f, w, f, torch.zeros((3, 3), device=DEV))   # the last row ends short of a multiple of 16


# ---------------------------------------------------------------- streams, graphs, the chain

def chain(h, w, sw, S, n, C, k, u, bufs, stream=None):
    """Hidden states of an ensemble -> 8-bit heads -> logits -> a token and the teacher's top k -> a student's loss."""
    for m in range(S):
        bd.quantize_rows_i8(h[m], bufs["q"][m], bufs["sx"][m], stream=stream)
        bd.fc_i8(bufs["q"][m], bufs["sx"][m], w[m], sw[m], bufs["z"][m], stream=stream)
    bd.combine_sample(bufs["z"], u, bufs["tok"], bufs["p"], top_p=bufs["top_p"], workspace=bufs["ws"], stream=stream)
    bd.combine_topk(bufs["z"], bufs["ids"], bufs["logp"], temperature=2.0, workspace=bufs["ws"], stream=stream)
    bd.distill_loss(bufs["student"], bufs["ids"], bufs["logp"], bufs["loss"], bufs["grad"], temperature=2.0, rest=True,
                    stream=stream)


def chain_setup(seed, S=2, n=9, c_in=200, C=3001, k=16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    h = r(S, n, c_in).bfloat16()
    w = torch.zeros((S, C, 208), dtype=torch.int8, device=DEV)
    w[:, :, :c_in] = (r(S, C, c_in) * 40).clamp(-127, 127).round().to(torch.int8)
    e = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device=DEV)  # noqa: E731
    bufs = dict(q=e(S, n, 208, t=torch.int8)[:, :, :c_in], sx=e(S, n), z=e(S, n, C), tok=e(n, t=torch.int32), p=e(n),
                ids=e(n, k, t=torch.int32), logp=e(n, k), student=r(n, C).bfloat16(), loss=e(n),
                grad=e(n, C, t=torch.bfloat16), top_p=e(n) + 0.9,
                ws=e(max(bd.combine_workspace(S, n, C), 16), t=torch.uint8))
    u = torch.rand(n, generator=g, device=DEV)
    return h, w[:, :, :c_in], torch.full((S, C), 0.005, device=DEV), S, n, C, k, u, bufs


def outputs(bufs):
    return [bufs[x].clone() for x in ("q", "sx", "z", "tok", "p", "ids", "logp", "loss", "grad")]


def test_chain_against_the_oracle():
    args = chain_setup(1)
    chain(*args)
    torch.cuda.synchronize()
    h, w, sw, S, n, C, k, u, b = args
    for m in range(S):
        q, s = ot.quantize_rows(host(h[m]))
        assert np.array_equal(b["q"][m].cpu().numpy(), q) and np.array_equal(host(b["sx"][m]), s)
        check_fc(q, s, w[m].cpu().numpy(), host(sw[m]), None, False, b["z"][m], "fp32")
    check_sample(b["z"], {"uniform": host(u), "top_p": host(b["top_p"])}, b["tok"], b["p"])
    check_topk(b["z"], k, 2.0, b["ids"], b["logp"])
    check_distill(b["student"], host(b["ids"]), host(b["logp"]), 2.0, True, None, b["loss"], b["grad"], "bf16")


def test_more_rows_than_one_launch_takes():
    """2^20 + 77 rows: every operator gives a row what it gives the same row of a short call."""
    m, n, C, k = 997, (1 << 20) + 77, 5, 3
    gen = torch.Generator().manual_seed(3)
    z = torch.randn(2, m, C, generator=gen).to(DEV)
    z[:, 5] = -math.inf
    u = torch.rand(m, generator=gen).to(DEV)
    which = torch.arange(n, device=DEV) % m

    def run(z, u):
        n = u.numel()
        ints = lambda *shape: torch.full(shape, -7, dtype=torch.int32, device=DEV)  # noqa: E731
        floats = lambda *shape: torch.full(shape, -7.0, device=DEV)  # noqa: E731
        token, prob, labels, logp, loss, grad = ints(n), floats(n), ints(n, k), floats(n, k), floats(n), floats(n, C)
        bd.combine_sample(z, u, token, prob, top_p=torch.full((n,), 0.9, device=DEV))
        bd.combine_topk(z, labels, logp)
        bd.distill_loss(z[0], labels, logp, loss, grad, rest=True)
        x, q, scale = torch.where(z[1].isinf(), 0.5, z[1]), torch.zeros(n, 16, dtype=torch.int8, device=DEV), floats(n)
        bd.quantize_rows_i8(x, q[:, :C], scale)
        w = torch.arange(-24, 24, device=DEV).to(torch.int8).reshape(3, 16)
        y = floats(n, 3)
        bd.fc_i8(q[:, :C], scale, w[:, :C], torch.ones(3, device=DEV), y)
        torch.cuda.synchronize()
        return token, prob, labels, logp, loss, grad, q, scale, y

    for few, many in zip(run(z, u), run(z[:, which].contiguous(), u[which].contiguous())):
        assert torch.equal(torch.nan_to_num(few[which], nan=-99.0), torch.nan_to_num(many, nan=-99.0))


def test_two_streams_at_once_repeat_the_same_bits():
    one, two = chain_setup(2), chain_setup(3)
    want = []
    for args in (one, two):
        chain(*args)
        torch.cuda.synchronize()
        want.append(outputs(args[-1]))
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        chain(*one, stream=sa)
        with torch.cuda.stream(sb):
            chain(*two)
        torch.cuda.synchronize()
        for args, w in zip((one, two), want):
            assert all(torch.equal(x, y) for x, y in zip(outputs(args[-1]), w))


def test_workspace_from_the_allocator_on_another_stream():
    """Without a workspace the binding takes one from torch's allocator; on another stream than the current one it
    stays theirs until that stream has passed."""
    rng = np.random.default_rng(41)
    z = lm_logits(rng, 1, 64, 30000, "fp32").to(DEV)
    par = mixed_params(rng, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = []
    u = dev(par["uniform"])
    for _ in range(4):
        labels, probs = empty_sample(64)
        s.wait_stream(torch.cuda.current_stream())
        bd.combine_sample(z, u, labels, probs, stream=s)
        junk = torch.full((1 << 22,), 3.0, device=DEV)           # would take a freed workspace's place
        got.append((labels, probs, junk))
    torch.cuda.synchronize()
    for labels, probs, _ in got:
        check_sample(z, {"uniform": par["uniform"]}, labels, probs)


def test_replayed_graphs():
    """Two captured chains with a workspace each, replayed in turn between eager calls, on new inputs."""
    args = [chain_setup(4), chain_setup(5)]
    graphs = []
    for a in args:
        chain(*a)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            chain(*a)
        graphs.append(g)
    for step in range(4):
        for a, g in zip(args, graphs):
            h, u, b = a[0], a[7], a[-1]
            gen = torch.Generator(device=DEV).manual_seed(100 + step)
            h.copy_(torch.randn(h.shape, generator=gen, device=DEV))
            u.copy_(torch.rand(u.shape, generator=gen, device=DEV))
            g.replay()
            torch.cuda.synchronize()
            got = outputs(b)
            chain(*a)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, outputs(b)))
    other = chain_setup(6)                                       # an eager run of other sizes in between
    chain(*other)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [3, 700, 90001])
@pytest.mark.parametrize("low", [-104.0, -1000.0])
def test_distill_empty_rest_far_below_zero(low, C, dtype):
    """Nothing above -inf outside the teacher's classes, whose logits all lie far below 0: the same bits as with `low`
    taken off (the values and their differences are exact), and the oracle's."""
    z = torch.full((2, C), -math.inf, dtype=DT[dtype])
    z[:, [0, C // 2, C - 1]] = torch.tensor([[0.0, -8.0, -16.0], [0.0, 0.0, -8.0]], dtype=DT[dtype])
    ids = np.int32([[C // 2, 0, C - 1]] * 2)
    logp = np.log(np.float32([[0.5, 0.25, 0.25], [0.125, 0.75, 0.125]]))
    near = run_distill(z.to(DEV), ids, logp, 4.0, True)
    check_distill(z, ids, logp, 4.0, True, None, *near, dtype)
    assert torch.isfinite(near[0]).all() and torch.isfinite(near[1]).all()
    for t in (4.0, 0.125):
        near, far = (run_distill((z + shift).to(DEV), ids, logp, t, True) for shift in (0.0, low))
        assert torch.equal(near[0], far[0]) and torch.equal(near[1], far[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [3, 64, 30001])
def test_distill_rest_that_no_class_can_take(C, dtype):
    """A teacher with mass for the other classes and a student that masks all of them: the loss is infinite, and the
    gradient that of the teacher's classes alone, which sums to 0."""
    z = torch.full((3, C), -math.inf, dtype=DT[dtype])
    z[0, 0] = 1.0
    z[1, :2] = torch.tensor([0.5, -1.0], dtype=DT[dtype])
    z[2, [0, C - 1]] = torch.tensor([-300.0, -301.0], dtype=DT[dtype])
    ids = np.int32([[0, -1], [0, 1], [C - 1, 0]])
    logp = np.log(np.float32([[0.75, 1.0], [0.5, 0.125], [0.25, 0.25]]))
    loss, grad = run_distill(z.to(DEV), ids, logp, 2.0, True)
    check_distill(z, ids, logp, 2.0, True, None, loss, grad, dtype)
    assert (loss == math.inf).all()
    assert (grad[0] == 0).all()                            # p = 1 and all of the mass: exactly
    # T times two terms of at most 1/2, off by some 8 roundings of 2^-24 each, and stored once
    assert (grad.double().sum(1).abs() <= 2 * (2 * 0.5 * (8 * 2.0 ** -24 + HALF_STEP[dtype]))).all()
    assert (grad[:, 2:C - 1] == 0).all()


@pytest.mark.parametrize("which", ["null", "default", "side", "number"])
def test_workspace_belongs_to_the_stream_of_the_call(which):
    """Without a workspace, on another stream than the current one: the block is not one that the current stream's queued
    work still reads, and not one that its next allocations get while the call runs.  Blocks of one size, each
    stream kept busy first."""
    rng = np.random.default_rng(42)
    n, C = 64, 30000
    z = lm_logits(rng, 1, n, C, "fp32").to(DEV)
    par = mixed_params(rng, n)
    need = bd.combine_workspace(1, n, C)
    args = {k: dev(v) for k, v in par.items()}
    u = args.pop("uniform")
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    a = torch.randn(2048, 2048, device=DEV)
    target = {"null": torch.cuda.default_stream(), "default": torch.cuda.default_stream(), "side": other,
              "number": other}[which]
    given = {"null": 0, "default": target, "side": target, "number": other.cuda_stream}[which]
    labels, probs = empty_sample(n)
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            block = torch.full((need,), 5, dtype=torch.uint8, device=DEV)
            for _ in range(8):
                b = a @ a
            copy = block.clone()                                 # read late; the block is free again for this stream
            del block
            with torch.cuda.stream(target):
                for _ in range(8):
                    c = a @ a
            bd.combine_sample(z, u, labels, probs, stream=given, **args)
            junk = [torch.full((need,), 3, dtype=torch.uint8, device=DEV) for _ in range(4)]
        torch.cuda.synchronize()
        assert (copy == 5).all() and all((j == 3).all() for j in junk)
        check_sample(z[:, ::7], {k: v[::7] for k, v in par.items()}, labels[::7], probs[::7])
        del b, c, junk


def test_replayed_graph_of_calls_that_take_their_workspace():
    """Captured without workspaces: the graph's own memory holds them, which eager calls and allocations between the
    replays leave alone."""
    rng = np.random.default_rng(43)
    z = lm_logits(rng, 2, 9, 3001, "fp32").to(DEV)
    par = mixed_params(rng, 9)
    args = {k: dev(v) for k, v in par.items()}
    u = args.pop("uniform")
    n, c_in, c_out = 64, 4096, 1000                              # few tiles: K is split through a workspace
    assert bd.fc_i8_workspace(n, c_in, c_out) > 0
    x = torch.from_numpy(rng.integers(-128, 128, (n, c_in), dtype=np.int8)).to(DEV)
    w = torch.from_numpy(rng.integers(-128, 128, (c_out, c_in), dtype=np.int8)).to(DEV)
    one = lambda k: torch.full((k,), 0.01, device=DEV)  # noqa: E731
    sx, sw = one(n), one(c_out)
    out = [empty_sample(9), torch.empty((n, c_out), device=DEV)]

    def calls():
        bd.combine_sample(z, u, *out[0], **args)
        bd.fc_i8(x, sx, w, sw, out[1])

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        gen = torch.Generator(device=DEV).manual_seed(step)
        u.copy_(torch.rand(9, generator=gen, device=DEV))
        x.copy_(torch.randint(-128, 128, x.shape, generator=gen, device=DEV))
        for t in (*out[0], out[1]):
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out[0], out[1])]
        junk = [torch.full((1 << s,), 9, dtype=torch.uint8, device=DEV) for s in (16, 18, 20, 22)]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*out[0], out[1])))
        del junk


# Logits of both signs that lie further apart than fp32 can hold: their differences and bounds stay finite.

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("S", [1, 2])
@pytest.mark.parametrize("C", [900, 2000])
def test_sample_span_beyond_fp32(C, S, dtype):
    rng = np.random.default_rng(51)
    n = 8
    z = torch.from_numpy(np.float32(3.3e38) * (2 * rng.random((S, n, C)).astype(np.float32) - 1)).to(DT[dtype])
    z[:, 0] = -3e38
    z[:, 0, :64] = 3e38
    z[:, 1] = z[:, 0]
    z = z.to(DEV)
    par = {"uniform": np.float32([0.9, 0.9, 0.9, 0.3, 0.999, 0.7, 0.6, 0.4]),
           "temperature": np.float32([math.inf, 3e38, math.inf, 3e38, 3e38, 2e38, 0, math.inf]),
           "top_k": np.int32([0, 0, 0, C * 3 // 4, 600, 0, 0, C - 1]),
           "top_p": np.float32([1, 0.9, 0.75, 1, 1, 0.97, 1, 1]),
           "min_p": np.float32([0.1, 0, 0, 0, 0, 0.05, 0, 0.5])}
    check_sample(z, par, *run_sample(z, par))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("S", [1, 3])
@pytest.mark.parametrize("C,k", [(2000, 20), (2000, 700), (2000, 1000), (700, 300), (70000, 64)])
def test_topk_span_beyond_fp32(C, k, S, dtype):
    rng = np.random.default_rng(52)
    t = np.float32(3e37)
    z = (np.float32(3.3e38) * (2 * rng.random((S, 4, C)).astype(np.float32) - 1))
    z[:, 1] = -3e38
    z[:, 1, ::97] = 3e38
    z[:, 2] *= np.float32(0.01)
    z = torch.from_numpy(z).to(DT[dtype]).to(DEV)
    labels = torch.empty((4, k), dtype=torch.int32, device=DEV)
    logp = torch.empty((4, k), device=DEV)
    bd.combine_topk(z, labels, logp, temperature=float(t))
    torch.cuda.synchronize()
    check_topk(z, k, t, labels, logp)


@pytest.mark.parametrize("S", [1, 2])
def test_temperatures_and_logits_below_the_normal_range(S):
    """T and the logits' differences of the size of fp32's smallest values: their quotients are ordinary numbers."""
    rng = np.random.default_rng(54)
    C, k = 3000, 40
    z = np.float32(1e-41) * rng.integers(-1000, 1000, (S, 4, C)).astype(np.float32)
    t = np.float32(2e-39)
    par = {"uniform": np.float32([0.2, 0.5, 0.8, 0.3]), "temperature": np.float32([t] * 4),
           "top_k": np.int32([50, 0, 0, 1500]), "top_p": np.float32([1, 0.5, 1, 0.99]), "min_p": np.float32([0, 0, 0.2, 0])}
    z = dev(z)
    check_sample(z, par, *run_sample(z, par))
    labels = torch.empty((4, k), dtype=torch.int32, device=DEV)
    logp = torch.empty((4, k), device=DEV)
    bd.combine_topk(z, labels, logp, temperature=float(t))
    torch.cuda.synchronize()
    check_topk(z, k, t, labels, logp)


def test_sample_top_p_cut_at_the_border_of_the_list():
    """A nucleus that ends among equal classes exactly where the row kernel's list of classes ends.  One class leads; the
    upper 64 groups of 64 classes hold one second class each, which set the list's bound; every group holds one of the equal
    classes, whose log2 p differs from the bound in the last places only (T was picked for the fp32 rounding of 1 / T).
    The first of them, by index, are in the nucleus, whichever group they are in."""
    C, groups = 8192, 128
    t = np.float32(1.4425914287567139)
    k = 1.4426950408889634 / float(t)
    z, top_p = [], []
    for b in range(24, 232):
        border = np.float32(((b + 1) / 16 + 1 / 32) / k)
        for step in range(-2, 3):
            third = (border.view(np.int32) + step).view(np.float32)
            second = np.float32((b + 0.5) / 16 / k)
            row = np.full(C, -np.inf, np.float32)
            row[1::64] = -third
            row[C // 2::64] = -second
            row[C // 2 + 5] = 0
            z.append(row)
            p2, p3 = 2.0 ** (-float(second) * k), 2.0 ** (-float(third) * k)
            # half a class off the next border: 2^-16 of the whole at least, far above the fp32 step of top_p
            top_p.append((1 + groups // 2 * p2 + 10.5 * p3) / (1 + groups // 2 * p2 + groups * p3))
    n = len(z)
    z = dev(np.stack(z)[None])
    par = {"uniform": np.zeros(n, np.float32), "temperature": np.full(n, t), "top_p": np.float32(top_p)}
    labels, probs = run_sample(z, par)
    assert (labels == 1).all(), torch.nonzero(labels != 1)[:, 0].tolist()
    check_sample(z[:, ::37], {k: v[::37] for k, v in par.items()}, labels[::37], probs[::37])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C,t", [(5, 1e38), (700, 1e38), (90001, 1e38), (1001, 3e38), (170000, 1.4e36), (301, 1.3e36), (301, 1e36)])
def test_distill_span_beyond_fp32(C, t, dtype, rest):
    """Student logits of both signs further apart than fp32 can hold, at a temperature of their size: T^2 is beyond fp32
    and the loss with it, the gradient is not.  The terms Q p_c, q_c and q_r p_c / p_r (at most 2 together) are off by the
    bounds of 32 bits relative to each; and a power below 2^-126 is 0, which T times it may not be: T 2^-125."""
    rng = np.random.default_rng(53)
    t = float(np.float32(t))
    z = torch.from_numpy(np.float32(3.3e38) * (2 * rng.random((3, C)).astype(np.float32) - 1)).to(DT[dtype])
    z[1] = -3e38
    z[1, [1, C - 2]] = 3e38
    z[2] = 3e38
    z[2, [0, C - 1]] = -3e38
    ids = np.int32([[0, C - 1]] * 3)
    logp = np.log(np.float32([[0.5, 0.25]] * 3))
    loss, grad = run_distill(z.to(DEV), ids, logp, t, rest)
    zh, got = host(z).astype(np.float64), host(grad).astype(np.float64)
    for i in range(3):
        _, want = ot.distill(zh[i], ids[i], logp[i], t, rest)
        terms = 2 * np.exp(zh[i] / t - ot._lse(zh[i] / t)) + np.abs(want) / t
        np.add.at(terms, ids[i], 1.0)
        eps = 2 * distill_bounds(zh[i], C, 2, t, 1.0, dtype) + 2 * 2.0 ** -22
        assert (np.abs(got[i] - want) <= t * (terms * eps + 2.0 ** -125) + np.abs(want) * HALF_STEP[dtype]).all(), i
    assert (loss == math.inf).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_distill_loss_of_a_span_beyond_fp32(dtype, rest):
    """The type's lowest value beside its largest at an ordinary temperature: log p = -2 max / T is within fp32, and so is the
    loss, T times the difference for each class, of little weight."""
    top = float(torch.finfo(DT[dtype]).max)
    t, q = 8.0, 2.0 ** -8
    z = torch.full((1, 100), -top, dtype=DT[dtype], device=DEV)
    z[0, 5] = top
    loss, grad = run_distill(z, np.int32([[5, 50]]), np.log(np.float32([[1 - q, q]])), t, rest)
    want = t * q * 2 * top
    assert abs(float(loss) - want) <= 1e-5 * want          # q = exp(log q): 2^-24 (1 + |log q|), some 10 roundings
    check_distill(z, np.int32([[5, 50]]), np.log(np.float32([[1 - q, q]])), t, rest, None, None, grad, dtype)


@pytest.mark.parametrize("t", [1e-20, 1e-25, 1e-30])
def test_distill_loss_where_the_square_of_t_underflows(t):
    """T^2 is below fp32, T^2 times the loss's sum is not: one class against a sure student, loss = T (difference)."""
    z = torch.tensor([[1.0, 3.0, 2.0], [0.5, -1.0, 0.25]], device=DEV)
    loss, _ = run_distill(z, np.int32([[0], [1]]), np.float32([[0.0], [0.0]]), t, False)
    want = float(np.float32(t)) * np.array([2.0, 1.5])
    assert np.abs(host(loss).astype(np.float64) - want).max() <= 1e-6 * want.min()       # some 10 roundings of 2^-24


def test_distill_loss_where_the_square_of_t_overflows():
    """A student that agrees exactly has loss 0 whatever T is."""
    z = torch.tensor([[7.0], [-3.0]], device=DEV)
    for t in (1e19, 1e25, 3e38):
        loss, grad = run_distill(z, np.int32([[0], [0]]), np.float32([[0.0], [0.0]]), t, False)
        assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("C", [3, 500])
def test_distill_nan_teacher_with_nothing_outside(C):
    """NaN in the teacher gives NaN throughout the row, also where the student masks every other class."""
    z = torch.full((1, C), -math.inf, device=DEV)
    z[0, :2] = 1.0
    loss, grad = run_distill(z, np.int32([[0, 1]]), np.float32([[math.nan, -1.0]]), 1.0, True)
    assert torch.isnan(loss).all() and torch.isnan(grad).all()


def test_fc_one_row_of_any_distance():
    """A matrix of one row has no distance between rows: only the row's own place counts."""
    rng = np.random.default_rng(55)
    c_in, c_out = 200, 33
    x = rng.integers(-128, 128, (1, c_in), dtype=np.int8)
    w = rng.integers(-128, 128, (c_out, c_in), dtype=np.int8)
    sx, sw = rng.random(1).astype(np.float32), rng.random(c_out).astype(np.float32)
    xp, wp = padded(x), padded(w)
    for row in (xp[0].unsqueeze(0), xp.as_strided((1, c_in), (1 << 23, 1)), xp.as_strided((1, c_in), (0, 1))):
        y = torch.empty((1, c_out), device=DEV)
        bd.fc_i8(row, dev(sx), wp, dev(sw), y)
        torch.cuda.synchronize()
        check_fc(x, sx, w, sw, None, False, y, "fp32")
    y = torch.empty((3, 1), device=DEV)                   # one output, three rows
    bd.fc_i8(wp[:3], dev(sw[:3]), xp[0].unsqueeze(0), dev(sx), y)
    torch.cuda.synchronize()
    check_fc(w[:3], sw[:3], x, sx, None, False, y, "fp32")
    with pytest.raises(ValueError):                       # not readable up to the next multiple of 16
        bd.fc_i8(torch.zeros(c_in, dtype=torch.int8, device=DEV).unsqueeze(0), dev(sx), wp, dev(sw),
                 torch.empty((1, c_out), device=DEV))


@pytest.mark.parametrize("S", [1, 2, 32])
def test_topk_near_the_least_probability(S):
    """Classes that one model gives 2^-980 to 2^-1000 and the others nothing: what the others' powers are cut at does not
    show in the logarithm."""
    C, k = 400, 300
    x = torch.full((S, 3, C), -math.inf)
    x[:, :, 0] = 0.0
    likely = torch.arange(1, C)
    x[0, :, 1:] = -(978.0 + 24.0 * likely / C) * math.log(2)      # to 2^-1002 and, of S models, S times less
    x[:, 1, 1:] = torch.where(x[:, 1, 1:] == -math.inf, -5000.0, x[:, 1, 1:])
    x[:, 2] = x[:, 2].flip(-1)
    x = x.to(DEV)
    labels = torch.empty((3, k), dtype=torch.int32, device=DEV)
    logp = torch.empty((3, k), device=DEV)
    bd.combine_topk(x, labels, logp)
    torch.cuda.synchronize()
    check_topk(x, k, 1.0, labels, logp)
