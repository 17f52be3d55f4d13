"""The vocabulary operators without a GPU: argument refusals of the C entry points and of the binding (before
any device call), workspace sizes, and the 64-bit oracle against independent statements of the definitions
(gradients against differences, sampling against its distribution)."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_1804_06087_amd as pkg
from oracle import tokens as ot
from paper_1804_06087_amd import binding as bd

INVALID = bd.RAFIKI_ERR_INVALID
P = 4096          # a stand-in for a device pointer: never read, every call below is refused


def _sample(**over):
    a = dict(logits=P, dtype=0, ld_model=100, ld_row=10, S=2, n=4, C=10, temperature=None, top_k=None, top_p=None,
             min_p=None, uniform=P, labels=P, out=P, ws=P, ws_bytes=1 << 20, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_combine_sample(*a.values())


def _topk(**over):
    a = dict(logits=P, dtype=0, ld_model=100, ld_row=10, S=2, n=4, C=10, t=1.0, k=3, labels=P, out=P, ws=P,
             ws_bytes=1 << 20, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_combine_topk(*a.values())


def _distill(**over):
    a = dict(logits=P, dtype=0, ld_row=10, n=4, C=10, ids=P, logp=P, k=3, t=1.0, rest=0, g=None, loss=P, grad=P,
             ld_grad=10, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_distill_loss(*a.values())


def _quantize(**over):
    a = dict(x=P, dtype=0, ld_x=10, n=4, c=10, q=P, ld_q=16, scale=P, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_quantize_rows_i8(*a.values())


def _fc(**over):
    a = dict(x=P, ld_x=16, sx=P, w=P, ld_w=16, sw=P, bias=None, n=4, c_in=10, c_out=5, relu=0, y=P, dtype=0, ld_y=5,
             ws=P, ws_bytes=1 << 30, stream=None)
    a.update(over)
    return pkg.load_library().rafiki_fc_i8(*a.values())


@pytest.mark.parametrize("call,over", [
    *[(_sample, o) for o in ({"logits": None}, {"uniform": None}, {"labels": None}, {"out": None}, {"dtype": 2},
                             {"dtype": -1}, {"S": 0}, {"S": 33}, {"n": 0}, {"n": -1}, {"C": 0}, {"C": (1 << 20) + 1},
                             {"ld_row": -1}, {"ld_model": -1}, {"ws": None}, {"ws_bytes": 8}, {"ws": P + 8},
                             {"logits": P + 2}, {"dtype": 1, "logits": P + 1})],
    *[(_topk, o) for o in ({"logits": None}, {"labels": None}, {"out": None}, {"k": 0}, {"k": 1025}, {"t": 0.0},
                           {"t": -1.0}, {"t": math.inf}, {"t": math.nan}, {"C": 0}, {"ws": None}, {"dtype": 3})],
    *[(_distill, o) for o in ({"logits": None}, {"ids": None}, {"logp": None}, {"loss": None, "grad": None}, {"k": 0},
                              {"k": 1025}, {"n": 0}, {"C": 0}, {"C": (1 << 20) + 1}, {"t": 0.0}, {"t": math.nan},
                              {"ld_row": -1}, {"ld_grad": 9}, {"dtype": 5}, {"grad": P + 2}, {"logits": P + 1})],
    *[(_quantize, o) for o in ({"x": None}, {"q": None}, {"scale": None}, {"n": 0}, {"c": 0}, {"ld_q": 9},
                               {"ld_x": -1}, {"dtype": 2}, {"x": P + 1}, {"c": (1 << 30) + 1, "ld_q": 1 << 31})],
    *[(_fc, o) for o in ({"x": None}, {"w": None}, {"sx": None}, {"sw": None}, {"y": None}, {"n": 0}, {"c_out": 0},
                         {"c_in": 0}, {"c_in": 131072, "ld_x": 131072, "ld_w": 131072}, {"ld_x": 15}, {"ld_x": 0},
                         {"ld_w": 24}, {"x": P + 4}, {"w": P + 8}, {"ld_y": 4}, {"dtype": 2}, {"y": P + 2},
                         {"ld_w": (1 << 22) + 16}, {"n": (1 << 24) + 1}, {"c_out": (1 << 24) + 1, "ld_y": 1 << 25})],
])
def test_refusals(call, over):
    assert call(**over) == INVALID, over
    assert bd.last_error()


def test_workspace_sizes():
    lib, b = pkg.load_library(), C.c_longlong(-1)
    assert lib.rafiki_combine_workspace(1, 1, 1, None) == INVALID
    for bad in ((0, 1, 1), (33, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 20) + 1)):
        assert lib.rafiki_combine_workspace(*bad, C.byref(b)) == INVALID
    assert bd.combine_workspace(32, 1 << 20, 1 << 20) > 1 << 31          # 64-bit size
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 131072, 1)):
        assert lib.rafiki_fc_i8_workspace(*bad, C.byref(b)) == INVALID
    assert bd.fc_i8_workspace(1, 131071, 1) >= 0


def test_valid_calls_without_a_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in (_sample, _topk, _distill, _quantize, _fc):
        assert call() == bd.RAFIKI_ERR_HIP and "launch" in bd.last_error()


def test_binding_refuses_host_tensors():
    import torch
    z, f, i = torch.zeros(2, 3, 5), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        bd.combine_sample(z, f, i, f)
    with pytest.raises(ValueError):
        bd.combine_topk(z, i.view(3, 1), f.view(3, 1))
    with pytest.raises(ValueError):
        bd.distill_loss(z[0], i.view(3, 1), f.view(3, 1), f)
    with pytest.raises(ValueError):
        bd.quantize_rows_i8(f.view(3, 1), torch.zeros(3, 1, dtype=torch.int8), f)
    with pytest.raises(ValueError):
        bd.fc_i8(i.view(3, 1).to(torch.int8), f, i.view(3, 1).to(torch.int8), f, f.view(3, 1))


# ---------------------------------------------------------------- the oracle

def test_oracle_sampling_follows_the_kept_distribution():
    """Uniforms at the midpoints of 4000 equal steps draw every kept class as often as its share, within one step."""
    rng = np.random.default_rng(5)
    z = rng.standard_normal((2, 12)).astype(np.float32) * 2
    p = ot.combined(z, 0.7)
    order = ot.ranked(p)[:9]
    cum = np.cumsum(p[order]) / p[order].sum()
    kept = [c for j, c in enumerate(order) if j == 0 or cum[j - 1] < 0.9]
    kept = [c for c in kept if p[c] >= 0.05 * p[order[0]]]
    steps = 4000
    drawn = np.bincount([ot.sample(z, (i + 0.5) / steps, 0.7, 9, 0.9, 0.05)[0] for i in range(steps)], minlength=12)
    share = np.zeros(12)
    share[kept] = p[kept] / p[kept].sum()
    assert np.abs(drawn - steps * share).max() <= 1


def test_oracle_exact_borders():
    z = np.zeros((1, 8), np.float32)                     # p = 1/8 each, exactly
    assert [ot.sample(z, u / 4, top_p=0.5)[0] for u in range(4)] == [0, 1, 2, 3]
    assert ot.sample(z, 0.99, top_p=0.5625)[0] == 4       # 4.5 of 8: five classes
    assert ot.sample(z, 0.99, top_k=3) == (2, 1 / 3)
    assert ot.sample(z, 0.0, min_p=1.0) == (0, 1 / 8)
    assert ot.sample(np.full((1, 4), -np.inf), 0.5) == (-1, 0.0)


@pytest.mark.parametrize("rest", [False, True])
def test_oracle_gradient_against_differences(rest):
    rng = np.random.default_rng(11)
    z = rng.standard_normal(9)
    labels = np.array([4, 1, -1, 4, 7, 30], np.int32)          # a class twice, two empty slots
    logp = np.log(np.array([0.2, 0.3, 0.9, 0.1, 0.15, 0.9]))
    t, h = 1.7, 1e-5
    _, d = ot.distill(z, labels, logp, t, rest)
    for c in range(9):
        up, down = z.copy(), z.copy()
        up[c] += h
        down[c] -= h
        diff = (ot.distill(up, labels, logp, t, rest)[0] - ot.distill(down, labels, logp, t, rest)[0]) / (2 * h)
        # truncation h^2 |f'''| / 6 with |f'''| <= 2, rounding 2^-52 |loss| / h
        assert abs(diff - d[c]) < 1e-9


def test_oracle_quantisation_ties():
    x = np.array([[127.0, 0.5, 1.5, -2.5, 63.5]], np.float32)        # scale 1
    q, s = ot.quantize_rows(x)
    assert s[0] == 1 and q.tolist() == [[127, 0, 2, -2, 64]]


def test_oracle_gradient_of_a_rest_that_no_class_can_take():
    """p_r = 0: q_r drops out of the gradient, which then sums to 0 over the classes that are left."""
    loss, d = ot.distill(np.array([1.0, -np.inf, -np.inf]), np.array([0], np.int32), np.log([0.75]), 1.0, True)
    assert loss == math.inf and np.array_equal(d, np.zeros(3))
    loss, d = ot.distill(np.array([0.5, -1.0, -np.inf]), np.array([0, 1], np.int32), np.log([0.5, 0.125]), 2.0, True)
    p = 1 / (1 + math.exp(-0.75))
    assert loss == math.inf and abs(d[0] - 2 * (0.625 * p - 0.5)) < 1e-15 and abs(d.sum()) < 1e-15 and d[2] == 0


# ---------------------------------------------------------------- workspaces that the binding takes itself

@pytest.mark.parametrize("stream", ["none", "null", "number", "default", "object"])
def test_workspace_is_the_stream_s_own(monkeypatch, stream):
    """A workspace that the caller does not give is allocated with the stream of the call current, so that neither what
    the current stream still does with a block nor its next allocation meets the work on the other stream.  torch's
    streams and allocator are stand-ins here: what counts is which stream was current at the allocation."""
    import contextlib
    import types

    import torch
    device = torch.device("cuda", 0)
    make = lambda handle: types.SimpleNamespace(cuda_stream=handle, device=device)  # noqa: E731
    current, default = make(7), make(0)
    state, taken, calls = {"current": current}, [], []

    @contextlib.contextmanager
    def use(s):
        before, state["current"] = state["current"], s
        yield
        state["current"] = before

    def external(handle, device=None):
        assert handle, "torch makes a new stream of an external one without a handle"
        return make(handle)

    class Block:
        def data_ptr(self):
            return P

    def empty(need, dtype, device):
        assert need == 640
        taken.append(state["current"].cuda_stream)
        return Block()

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: state["current"].cuda_stream, raising=False)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: default)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch, "empty", empty)
    given, want = {"none": (None, 7), "null": (0, 0), "number": (99, 99), "default": (default, 0),
                   "object": (make(55), 55)}[stream]
    bd._call(types.SimpleNamespace(device=device), given, 640, None, lambda *a: calls.append(a) or 0, "x")
    assert taken == [want] and calls == [("x", P, 640, want)] and state["current"] is current
