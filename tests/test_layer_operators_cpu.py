"""Refusals of the gated scan, the norm with a residual's addition and the product with its
epilogue, which need no GPU, and their definitions against one another."""
import os

import numpy as np
import pytest

from oracle import sequence_oracle as Q
from paper_2609_32479_gb300 import trackfit as T

P = 1 << 20     # an address that is never read
INVALID, UNSUPPORTED, OK = T.ERR_INVALID_ARG, T.ERR_UNSUPPORTED, T.OK
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return T.load()


def call(fn, base, **kw):
    assert set(kw) <= set(base), kw
    return fn(*{**base, **kw}.values())


SCAN = dict(dtype=1, gate=P, gate_stride=128, cand=P, cand_stride=128, n_rows=100000, offsets=P, n_seq=3, channels=64,
            reverse=0, state_in=None, state_out=None, saved=None, out=P, out_stride=64, workspace=P,
            workspace_size=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(n_rows=1 << 41), INVALID),
    (dict(n_seq=-1), INVALID), (dict(n_seq=1 << 31), INVALID), (dict(channels=0), UNSUPPORTED),
    (dict(channels=12), UNSUPPORTED), (dict(channels=65544), UNSUPPORTED), (dict(reverse=2), INVALID),
    (dict(offsets=None), INVALID), (dict(offsets=P + 4), INVALID), (dict(gate=None), INVALID), (dict(cand=P + 8), INVALID),
    (dict(out=None), INVALID), (dict(out_stride=56), INVALID), (dict(gate_stride=132), INVALID),
    (dict(cand_stride=-64), INVALID), (dict(dtype=0, out_stride=66), INVALID), (dict(state_in=P + 8), INVALID),
    (dict(state_out=P + 4), INVALID), (dict(saved=P + 4), INVALID), (dict(workspace=P + 8), INVALID),
    (dict(n_seq=0, offsets=None, gate=None), OK)])
def test_scan_refusals(lib, kw, want):
    assert call(lib.trackfit_gated_scan, SCAN, **kw) == want


BACK = dict(dtype=2, gate=P, gate_stride=128, cand=P, cand_stride=128, n_rows=100000, offsets=P, n_seq=3, channels=64,
            reverse=1, state_in=None, saved=P, d_out=P, d_out_stride=64, d_state_out=None, d_state_in=None, d_gate=P,
            d_gate_stride=128, d_cand=P, d_cand_stride=128, workspace=P, workspace_size=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=4), INVALID), (dict(n_rows=-1), INVALID), (dict(n_seq=-1), INVALID), (dict(channels=4), UNSUPPORTED),
    (dict(reverse=-1), INVALID), (dict(offsets=None), INVALID), (dict(gate=P + 2), INVALID), (dict(cand=None), INVALID),
    (dict(d_out=None), INVALID), (dict(d_out_stride=63), INVALID), (dict(d_gate=None), INVALID),
    (dict(d_gate_stride=60), INVALID), (dict(d_cand=P + 8), INVALID), (dict(d_cand_stride=0), INVALID),
    (dict(saved=None), INVALID), (dict(saved=P + 4), INVALID), (dict(state_in=P + 8), INVALID),
    (dict(d_state_out=P + 8), INVALID), (dict(d_state_in=P + 4), INVALID), (dict(workspace=P + 4), INVALID),
    (dict(n_seq=0, offsets=None, gate=None, saved=None), OK)])
def test_scan_backward_refusals(lib, kw, want):
    assert call(lib.trackfit_gated_scan_backward, BACK, **kw) == want


def test_scan_sizes(lib):
    saved, ws = lib.trackfit_gated_scan_saved, lib.trackfit_gated_scan_workspace
    assert saved(0, 64) == 0 and saved(-1, 64) == 0 and saved(100, 12) == 0
    assert saved(1, 64) == 64 * 4 and saved(32, 8) == 8 * 4 and saved(33, 8) == 2 * 8 * 4
    assert 4 * T.gated_scan_saved(1000, 24) == saved(1000, 24) >= 8 * 24 * 4
    for bad in ((5, 100, 1, 64), (1, -1, 1, 64), (1, 100, -1, 64), (1, 100, 1, 60)):
        assert ws(*bad) == 0
    assert ws(1, 1280, 20, 64) == 0 and ws(1, 1281, 20, 64) > 0
    for t in range(3):
        n = ws(t, 100000, 3, 64)
        assert ws(t, 0, 3, 64) == 0 and ws(t, 200000, 3, 64) >= n
        if n:
            assert call(lib.trackfit_gated_scan, SCAN, dtype=t, workspace_size=n - 1) == INVALID
            assert call(lib.trackfit_gated_scan, SCAN, dtype=t, workspace=None) == INVALID
            assert call(lib.trackfit_gated_scan_backward, BACK, dtype=t, workspace_size=n - 1) == INVALID


STEP = dict(dtype=0, gate=P, gate_stride=128, cand=P, cand_stride=128, n_seq=7, channels=64, slots=None, n_slots=7,
            state_in=P, state_out=P, out=P, out_stride=64, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=5), INVALID), (dict(n_seq=-1), INVALID), (dict(n_slots=-1), INVALID), (dict(n_slots=6), INVALID),
    (dict(channels=20), UNSUPPORTED), (dict(slots=P + 2), INVALID), (dict(state_in=None), INVALID),
    (dict(state_out=None), INVALID), (dict(state_in=P + 4), INVALID), (dict(gate=None), INVALID),
    (dict(cand_stride=32), INVALID), (dict(out=P + 4), INVALID), (dict(n_seq=0, gate=None, state_in=None), OK)])
def test_step_refusals(lib, kw, want):
    assert call(lib.trackfit_gated_scan_step, STEP, **kw) == want


NORM = dict(dtype=1, x=P, x_stride=128, delta=P, delta_stride=128, n_rows=10, channels=128, gain=P, eps=1e-6, sum_out=P,
            sum_stride=128, out_type=1, out=P, out_stride=128, scales=None, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), INVALID), (dict(out_type=0), INVALID), (dict(out_type=4), INVALID), (dict(n_rows=-1), INVALID),
    (dict(n_rows=1 << 41), INVALID), (dict(channels=4), UNSUPPORTED), (dict(channels=16392, x_stride=20000), UNSUPPORTED),
    (dict(channels=100), UNSUPPORTED), (dict(channels=120, out_type=3, scales=P), UNSUPPORTED), (dict(eps=0.0), INVALID),
    (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(x=None), INVALID), (dict(out=None), INVALID),
    (dict(x=P + 8), INVALID), (dict(delta=P + 4), INVALID), (dict(sum_out=P + 2), INVALID), (dict(x_stride=120), INVALID),
    (dict(delta_stride=0), INVALID), (dict(sum_stride=100), INVALID), (dict(out_stride=132), INVALID),
    (dict(gain=P + 2), INVALID), (dict(out_type=3), INVALID), (dict(scales=P), INVALID),
    (dict(out_type=3, scales=P + 1), INVALID), (dict(out_type=3, scales=P, out_stride=136), INVALID),
    (dict(n_rows=0, x=None, out=None), OK)])
def test_norm_refusals(lib, kw, want):
    assert call(lib.trackfit_add_norm, NORM, **kw) == want


PROD = dict(dtype=1, operand_type=1, x=P, x_stride=128, x_scales=None, weight=P, weight_stride=128, weight_scales=None,
            n_rows=10, in_dim=128, out_dim=64, bias=P, activation=2, gate=P, gate_stride=64, residual=P,
            residual_stride=64, out=P, out_stride=64, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), INVALID), (dict(operand_type=0), INVALID), (dict(operand_type=2), INVALID), (dict(n_rows=-1), INVALID),
    (dict(in_dim=4), UNSUPPORTED), (dict(in_dim=100), UNSUPPORTED), (dict(in_dim=16392), UNSUPPORTED),
    (dict(out_dim=0), UNSUPPORTED), (dict(out_dim=60), UNSUPPORTED), (dict(out_dim=65544), UNSUPPORTED),
    (dict(operand_type=3, x_scales=P, weight_scales=P, in_dim=120), UNSUPPORTED), (dict(activation=4), INVALID),
    (dict(activation=-1), INVALID), (dict(x=None), INVALID), (dict(weight=None), INVALID), (dict(out=None), INVALID),
    (dict(x=P + 8), INVALID), (dict(weight=P + 4), INVALID), (dict(out=P + 2), INVALID), (dict(gate=P + 8), INVALID),
    (dict(residual=P + 8), INVALID), (dict(x_stride=120), INVALID), (dict(weight_stride=132), INVALID),
    (dict(out_stride=56), INVALID), (dict(gate_stride=0), INVALID), (dict(residual_stride=-64), INVALID),
    (dict(bias=P + 2), INVALID), (dict(x_scales=P), INVALID), (dict(operand_type=3), INVALID),
    (dict(operand_type=3, x_scales=P), INVALID), (dict(operand_type=3, x_scales=P, weight_scales=P + 2), INVALID),
    (dict(n_rows=0, x=None, out=None), OK)])
def test_product_refusals(lib, kw, want):
    assert call(lib.trackfit_product, PROD, **kw) == want


def test_the_binding_refuses_tensors_on_the_host(lib):
    torch = pytest.importorskip("torch")
    x, off, s = torch.zeros((4, 16)), torch.tensor([0, 4]), torch.zeros((4, 16))
    for call_it in (lambda: T.gated_scan(x, x, off, x), lambda: T.gated_scan_step(x, x, s, s, x),
                    lambda: T.gated_scan_backward(x, x, off, torch.zeros(16), x, x, x), lambda: T.add_norm(x, x),
                    lambda: T.product(x, x, torch.zeros((4, 4)))):
        with pytest.raises(ValueError):
            call_it()


def test_checks_of_matrices():
    torch = pytest.importorskip("torch")
    a = object.__new__(T._OpArgs)
    a.what, a.device, a.dtype, a.torch = "op", torch.device("cpu"), torch.float32, torch
    x = torch.zeros((6, 32))
    assert a.matrix("x", None, (6, 32)) == (None, 0)
    assert a.matrix("x", x, (6, 32)) == (x.data_ptr(), 32) and a.matrix("x", x[:, 8:16], (6, 8)) == (x.data_ptr() + 32, 32)
    assert a.matrix("x", x[::2], (3, 32))[1] == 64 and a.matrix("x", x[:1, :8], (1, 8))[1] == 8
    for bad, shape in ((x, (6, 16)), (x.half(), (6, 32)), (x[:, ::2], (6, 16)), (x.t(), (32, 6))):
        with pytest.raises(ValueError):
            a.matrix("x", bad, shape)
    assert a.kept("saved", None, 6, 32) is None and a.kept("saved", torch.zeros(32), 6, 32) is not None
    with pytest.raises(ValueError):
        a.kept("saved", torch.zeros(31), 6, 32)


# ---------------------------------------------------------------- the definitions

@pytest.mark.parametrize("reverse", [False, True])
def test_the_gradients_are_those_of_the_scan(reverse):
    """Against central differences: their error is h^2 / 6 of a third derivative plus 2^-53 / h of
    the sums, below 1e-7 for h = 1e-4 and values of a few units."""
    r = np.random.default_rng(1)
    off, C = [0, 0, 5, 6, 6, 13], 3
    p, n, s0 = r.normal(size=(13, C)), r.normal(size=(13, C)), r.normal(size=(5, C))
    g, gs = r.normal(size=(13, C)), r.normal(size=(5, C))

    def loss():
        out, s = Q.gated_scan(p, n, off, reverse, s0)
        return np.sum(out * g) + np.sum(s * gs)

    grads = Q.gated_scan_backward(p, n, off, g, reverse, s0, gs)
    for x, d in zip((p, n, s0), grads):
        for i in np.ndindex(x.shape):
            keep = x[i]
            x[i] = keep + 1e-4
            up = loss()
            x[i] = keep - 1e-4
            down = loss()
            x[i] = keep
            assert abs((up - down) / 2e-4 - d[i]) < 1e-7, (i, d[i])


def test_values_of_the_8_bit_type():
    torch = pytest.importorskip("torch")
    x = np.concatenate([np.linspace(-448, 448, 4001), np.geomspace(2.0 ** -12, 448, 999), [0.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(Q.e4m3(np.float32(x)), want)


def test_the_definitions_make_up_the_layer():
    """The norm, the products and the scans, put together, are the encoder's layer, written out a
    hit at a time (both in 64 bits: 1e-12 is 2^13 roundings of values of a few units)."""
    r = np.random.default_rng(2)
    D, H, T_ = 16, 24, 11
    x = r.normal(size=(T_, D))
    w = {k: r.normal(size=s) * 0.2 for k, s in dict(w_in=(4 * H + D, D), w_m=(D, 2 * H), w1=(H, D), w2=(D, H)).items()}
    b = {k: r.normal(size=s) * 0.2 for k, s in dict(w_in=4 * H + D, w_m=D, w1=H, w2=D).items()}
    gain = 1 + 0.1 * r.normal(size=D)
    _, y = Q.add_norm(x, None, gain, 1e-5)
    u = Q.product(y, w["w_in"], b["w_in"])
    off = [0, T_]
    hf, _ = Q.gated_scan(u[:, :H], u[:, H:2 * H], off)
    hb, _ = Q.gated_scan(u[:, 2 * H:3 * H], u[:, 3 * H:4 * H], off, True)
    x1 = Q.product(np.concatenate([hf, hb], 1), w["w_m"], b["w_m"], gate=u[:, 4 * H:], residual=x)
    x2 = Q.product(Q.product(x1, w["w1"], b["w1"], "silu"), w["w2"], b["w2"], residual=x1)
    ref = layer_reference(x, w, b, gain, 1e-5, H)
    np.testing.assert_allclose(x2, ref, rtol=0, atol=1e-12)


def layer_reference(x, w, b, gain, eps, H):
    """The layer's formulas, a hit at a time."""
    sig = lambda v: 1 / (1 + np.exp(-v))
    T_, D = x.shape
    xh = [v / np.sqrt(sum(c * c for c in v) / D + eps) * gain for v in x]
    u = [w["w_in"] @ v + b["w_in"] for v in xh]
    hf, hb = np.zeros((T_, H)), np.zeros((T_, H))
    h = np.zeros(H)
    for t in range(T_):
        h = h + sig(u[t][:H]) * (u[t][H:2 * H] - h)
        hf[t] = h
    h = np.zeros(H)
    for t in range(T_ - 1, -1, -1):
        h = h + sig(u[t][2 * H:3 * H]) * (u[t][3 * H:4 * H] - h)
        hb[t] = h
    out = []
    for t in range(T_):
        x1 = x[t] + (w["w_m"] @ np.concatenate([hf[t], hb[t]]) + b["w_m"]) * sig(u[t][4 * H:])
        a = w["w1"] @ x1 + b["w1"]
        out.append(x1 + w["w2"] @ (a * sig(a)) + b["w2"])
    return np.array(out)
