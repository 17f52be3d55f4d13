"""The losses over given tokens and the 4-bit FC layer without a GPU: argument refusals of the C entry points and of
the binding (before any device call), workspace sizes, and the 64-bit oracle against independent statements of the
definitions (gradients against differences, codes against every representable neighbour)."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_1804_06087_amd as pkg
from oracle import tokens as ot
from paper_1804_06087_amd import binding as bd

INVALID = bd.RAFIKI_ERR_INVALID
P = 4096          # a stand-in for a device pointer: never read, every call below is refused


def _logp(**over):
    a = dict(logits=P, dtype=0, ld_row=10, n=4, C=10, labels=P, t=1.0, g_logp=P, g_entropy=P, logp=P, entropy=P, grad=P,
             ld_grad=10, ws=P, ws_bytes=1 << 20, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_token_logp(*a.values())


def _policy(**over):
    a = dict(logits=P, dtype=0, ld_row=10, n=4, C=10, labels=P, advantage=P, old=P, ref=P, t=1.0, low=0.2, high=0.2,
             kl=0.1, ent=0.0, g=None, loss=P, logp=P, out_kl=P, entropy=P, grad=P, ld_grad=10, ws=P,
             ws_bytes=1 << 20, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_policy_loss(*a.values())


def _preference(**over):
    a = dict(logits=P, dtype=0, ld_row=10, n=8, C=10, labels=P, offsets=P, pairs=2, ref=P, t=1.0, beta=0.1, smoothing=0.0,
             mean=0, g=None, loss=P, scores=P, grad=P, ld_grad=10, ws=P, ws_bytes=1 << 20, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_preference_loss(*a.values())


def _quantize(**over):
    a = dict(x=P, dtype=0, ld_x=40, n=4, c=40, q=P, ld_q=32, scale=P, ld_scale=2, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_quantize_rows_mx4(*a.values())


def _fc(**over):
    a = dict(x=P, ld_x=32, xs=P, ld_xs=16, w=P, ld_w=32, ws_=P, ld_ws=16, bias=None, n=4, c_in=64, c_out=5, relu=0, y=P,
             dtype=0, ld_y=5, ws=P, ws_bytes=1 << 30, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_fc_mx4(*a.values())


ROWS = ({"logits": None}, {"labels": None}, {"dtype": 2}, {"dtype": -1}, {"n": 0}, {"n": -1}, {"n": (1 << 30) + 1}, {"C": 0}, {"C": (1 << 20) + 1},
        {"t": 0.0}, {"t": -1.0}, {"t": math.nan}, {"t": math.inf}, {"t": 2.0 ** -21}, {"t": 2.0 ** 21}, {"ld_row": -1},
        {"ld_grad": 9}, {"logits": P + 2}, {"grad": P + 2}, {"dtype": 1, "logits": P + 1})


@pytest.mark.parametrize("call,over", [
    *[(c, o) for c in (_logp, _policy, _preference) for o in ROWS],
    *[(c, {"C": 1 << 20, "ld_grad": 1 << 20, **o}) for c in (_logp, _policy)
      for o in ({"ws": None}, {"ws": P + 8}, {"ws_bytes": 15})],          # few rows that are long
    *[(_logp, o) for o in ({"logp": None, "entropy": None, "grad": None}, {"g_logp": None, "g_entropy": None})],
    *[(_policy, o) for o in ({"advantage": None}, {"loss": None, "logp": None, "out_kl": None, "entropy": None, "grad": None},
                             {"low": -0.1}, {"low": 1.1}, {"low": math.nan}, {"high": -0.1}, {"high": math.nan},
                             {"kl": math.inf}, {"kl": math.nan}, {"ent": math.inf}, {"ent": math.nan})],
    *[(_preference, o) for o in ({"loss": None, "scores": None, "grad": None}, {"pairs": 0}, {"pairs": (1 << 20) + 1},
                                 {"offsets": None, "pairs": 3}, {"beta": 0.0}, {"beta": -1.0}, {"beta": math.inf},
                                 {"beta": math.nan}, {"smoothing": -0.1}, {"smoothing": 0.6}, {"smoothing": math.nan},
                                 {"ws": None}, {"ws": P + 8}, {"ws_bytes": 8})],
    *[(_quantize, o) for o in ({"x": None}, {"q": None}, {"scale": None}, {"n": 0}, {"c": 0}, {"ld_q": 31}, {"ld_scale": 1},
                               {"ld_x": -1}, {"dtype": 2}, {"x": P + 1}, {"c": (1 << 30) + 1, "ld_q": 1 << 40, "ld_scale": 1 << 40})],
    *[(_fc, o) for o in ({"x": None}, {"xs": None}, {"w": None}, {"ws_": None}, {"y": None}, {"n": 0}, {"c_out": 0},
                         {"c_in": 0}, {"c_in": 33}, {"c_in": (1 << 20) + 32, "ld_x": 1 << 22, "ld_w": 1 << 22},
                         {"ld_x": 16}, {"ld_x": 40}, {"ld_w": 0}, {"ld_xs": 8}, {"ld_xs": 0}, {"ld_ws": 24},
                         {"x": P + 4}, {"w": P + 8}, {"xs": P + 1}, {"ws_": P + 2}, {"ld_y": 4}, {"dtype": 2}, {"y": P + 2},
                         {"ld_w": (1 << 22) + 16}, {"n": (1 << 24) + 1}, {"c_out": (1 << 24) + 1, "ld_y": 1 << 25})],
])
def test_refusals(call, over):
    assert call(**over) == INVALID, over
    assert bd.last_error()


def test_workspace_sizes():
    lib, b = pkg.load_library(), C.c_longlong(-1)
    for f in (lib.rafiki_preference_workspace, lib.rafiki_token_workspace):
        assert f(1, 1, None) == INVALID
        for bad in ((0, 1), (1, 0), (1, (1 << 20) + 1), ((1 << 30) + 1, 1)):
            assert f(*bad, C.byref(b)) == INVALID
    assert bd.preference_workspace(1 << 30, 1) > 1 << 32                 # 64-bit size
    assert bd.token_workspace(1 << 30, 1 << 20) >= 0
    assert lib.rafiki_fc_mx4_workspace(1, 32, 1, None) == INVALID
    for bad in ((0, 32, 1), (1, 0, 1), (1, 32, 0), (1, 48, 1), (1, (1 << 20) + 32, 1)):
        assert lib.rafiki_fc_mx4_workspace(*bad, C.byref(b)) == INVALID
    assert bd.fc_mx4_workspace(1, 1 << 20, 1) >= 0


def test_valid_calls_without_a_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in (_logp, _policy, _preference, _quantize, _fc):
        assert call() == bd.RAFIKI_ERR_HIP and "launch" in bd.last_error()


def test_binding_refuses_host_tensors():
    import torch
    z, f, i = torch.zeros(4, 5), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    q, s = bd.mx4_empty(4, 5, device="cpu")
    for call in (lambda: bd.token_logp(z, i, f), lambda: bd.policy_loss(z, i, f, f),
                 lambda: bd.preference_loss(z, i, f[:2], n_pairs=2), lambda: bd.quantize_rows_mx4(z, q, s),
                 lambda: bd.fc_mx4(q, s, q, s, torch.zeros(4, 4))):
        with pytest.raises(ValueError):
            call()


def test_mx4_empty_layout():
    for c in (1, 32, 33, 512, 513, 4100):
        q, s = bd.mx4_empty(3, c, device="cpu")
        b = (c + 31) // 32
        assert q.shape == (3, 16 * b) and s.shape == (3, b)
        assert q.stride() == (16 * b, 1) and s.stride(0) % 16 == 0 and s.stride(0) >= b


# ---------------------------------------------------------------- the oracle

def _differences(f, z, h=1e-5):
    d = np.zeros(z.size)
    for c in range(z.size):
        up, down = z.copy(), z.copy()
        up[c] += h
        down[c] -= h
        d[c] = (f(up) - f(down)) / (2 * h)
    return d


# truncation h^2 |f'''| / 6 with |f'''| below 50 for these values, rounding 2^-52 |f| / h
CLOSE = 2e-9


def test_oracle_token_gradient_against_differences():
    z = np.random.default_rng(3).standard_normal(9)
    got = ot.token_grad(z, 4, 1.7, 0.8, -0.3)

    def f(v):
        logp, H = ot.token_facts(v, 4, 1.7)[:2]
        return 0.8 * logp - 0.3 * H
    assert np.abs(got - _differences(f, z)).max() < CLOSE


@pytest.mark.parametrize("A", [1.3, -0.7, 0.0])
@pytest.mark.parametrize("shift", [-0.5, 0.05, 0.5])
def test_oracle_policy_gradient_against_differences(A, shift):
    z = np.random.default_rng(4).standard_normal(9)
    logp = ot.token_facts(z, 2, 0.8)[0]
    f = lambda v: ot.policy(v, 2, A, logp + shift, logp + 0.4, 0.8, 0.2, 0.3, 0.1, 0.02)[0]  # noqa: E731
    got = ot.policy(z, 2, A, logp + shift, logp + 0.4, 0.8, 0.2, 0.3, 0.1, 0.02)[4]
    assert np.abs(got - _differences(f, z)).max() < CLOSE


@pytest.mark.parametrize("mean", [False, True])
def test_oracle_preference_gradient_against_differences(mean):
    rng = np.random.default_rng(5)
    z = rng.standard_normal((7, 6))
    labels, offsets, ref = np.array([1, -1, 3, 0, 5, 9, 2]), [0, 2, 3, 3, 6], rng.standard_normal(7)
    g = [0.7, -1.2]
    _, _, got = ot.preference(z, labels, offsets, ref, 1.3, 0.4, 0.1, mean, g)
    f = lambda v: float(np.dot(g, ot.preference(v.reshape(7, 6), labels, offsets, ref, 1.3, 0.4, 0.1, mean)[0]))  # noqa: E731
    assert np.isnan(got[6]).all()                            # a row of no answer
    assert np.abs(got[:6] - _differences(f, z.ravel()).reshape(7, 6)[:6]).max() < CLOSE


def test_oracle_codes_are_the_nearest():
    """Every magnitude, the midpoints between them and their neighbours in fp32, under several scales."""
    mids = np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    want = [0, 2, 2, 4, 4, 6, 6]                             # ties to the even code
    for e in (-127, -100, -1, 0, 1, 60, 125):
        s = 2.0 ** e
        with np.errstate(over="ignore"):
            row = np.concatenate([[4.0], mids, np.nextafter(mids, np.float32(0)), np.nextafter(mids, np.float32(9))])
            x = (np.pad(row, (0, 32 - row.size)) * s).astype(np.float32)[None]
        exact = x.astype(np.float64)[0, :row.size] / s == row
        codes, scale = ot.quantize_mx4(x)
        assert scale[0, 0] == e + 127
        if exact.all():
            assert codes[0, 1:8].tolist() == want
            assert codes[0, 8:15].tolist() == [0, 1, 2, 3, 4, 5, 6] and codes[0, 15:22].tolist() == [1, 2, 3, 4, 5, 6, 7]
    codes, scale = ot.quantize_mx4(np.float32([[7.9] + [0] * 31, [np.nan] + [1] * 31, [0] * 32, [1e-45] + [0] * 31]))
    assert codes[0, 0] == 7 and scale[:, 0].tolist() == [127, 255, 0, 0] and (codes[1] == 0).all()
