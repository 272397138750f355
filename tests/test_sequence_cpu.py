"""Refusals of the operators on packed sequences, which need no GPU: the library's checks of
pointers, strides, widths and counts, and the binding's of tensors."""
import ctypes
import os

import pytest

from paper_2609_32479_gb300 import trackfit as T

P = 1 << 20     # an address that is never read
INVALID, UNSUPPORTED, OK = T.ERR_INVALID_ARG, T.ERR_UNSUPPORTED, T.OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(T.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return T.load()


def call(fn, base, **kw):
    assert set(kw) <= set(base), kw
    return fn(*{**base, **kw}.values())


NORM = dict(dtype=1, q=P, q_stride=384, q_heads=4, k=P, k_stride=384, k_heads=4, head_dim=32, n_rows=10, q_gain=P,
            k_gain=P, eps=1e-6, positions=P, rot_dim=32, rot_base=1e4, q_out=P, q_out_stride=128, k_out=P,
            k_out_stride=128, stream=None)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(n_rows=1 << 41), INVALID),
    (dict(head_dim=20), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
    (dict(q_heads=0), UNSUPPORTED), (dict(q_heads=257), UNSUPPORTED), (dict(k_heads=-1), UNSUPPORTED),
    (dict(rot_dim=8), UNSUPPORTED), (dict(rot_dim=48), UNSUPPORTED), (dict(rot_dim=-16), UNSUPPORTED),
    (dict(eps=0.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID),
    (dict(rot_base=0.5), INVALID), (dict(rot_base=NAN), INVALID), (dict(rot_base=INF), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(q_out=None), INVALID), (dict(k_out=None), INVALID),
    (dict(q=P + 8), INVALID), (dict(k_out=P + 2), INVALID), (dict(q_stride=120), INVALID), (dict(q_stride=388), INVALID),
    (dict(k_out_stride=-128), INVALID), (dict(k_stride=0), INVALID), (dict(dtype=0, q_stride=386), INVALID),
    (dict(positions=None), INVALID), (dict(positions=P + 2), INVALID), (dict(q_gain=P + 1), INVALID),
    (dict(n_rows=0, q=None, k=None), OK)])
def test_norm_refusals(lib, kw, want):
    assert call(lib.trackfit_qk_norm, NORM, **kw) == want


LINEAR = dict(dtype=1, q=P, q_stride=128, k=P, k_stride=128, v=P, v_stride=128, log_decay=P, decay_stride=4,
              n_rows=1000, offsets=P, n_seq=3, n_heads=4, key_dim=32, value_dim=32, scale=1.0, reverse=0, state_in=None,
              state_out=None, out=P, out_stride=128, workspace=P, workspace_size=1 << 30, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=7), INVALID), (dict(n_rows=-5), INVALID), (dict(n_seq=-1), INVALID), (dict(n_seq=1 << 31), INVALID),
    (dict(n_heads=0), UNSUPPORTED), (dict(key_dim=4), UNSUPPORTED), (dict(value_dim=132), UNSUPPORTED),
    (dict(value_dim=33), UNSUPPORTED), (dict(scale=NAN), INVALID), (dict(reverse=2), INVALID),
    (dict(offsets=None), INVALID), (dict(offsets=P + 4), INVALID), (dict(state_in=P + 4), INVALID),
    (dict(state_out=P + 8), INVALID), (dict(q=None), INVALID), (dict(k=P + 4), INVALID), (dict(v=None), INVALID),
    (dict(out=None), INVALID), (dict(q_stride=127), INVALID), (dict(v_stride=132), INVALID), (dict(out_stride=96), INVALID),
    (dict(log_decay=None), INVALID), (dict(log_decay=P + 2), INVALID), (dict(decay_stride=3), INVALID),
    (dict(workspace=None), INVALID), (dict(workspace=P + 8), INVALID), (dict(workspace_size=100), INVALID),
    (dict(n_seq=0, offsets=None, q=None), OK)])
def test_linear_refusals(lib, kw, want):
    assert call(lib.trackfit_linear_attention, LINEAR, **kw) == want


def test_linear_workspace(lib):
    f = lib.trackfit_linear_attention_workspace
    assert f(512, 1, 4, 32, 32) == 0 and f(0, 1, 4, 32, 32) == 0
    assert f(513, 1, 4, 32, 32) >= 4 * 32 * 32 * 4
    assert f(16384, 256, 4, 32, 32) == 0 and f(16384, 255, 4, 32, 32) > 0 and f(16385, 1000, 4, 32, 32) > 0
    assert f(-1, 1, 4, 32, 32) == 0 and f(1000, 1, 0, 32, 32) == 0 and f(1000, 1, 4, 20, 32) == 0 and f(1000, 0, 4, 32, 32) == 0
    n = f(1 << 20, 4, 8, 64, 64)
    assert 0 < n < 1 << 30
    assert call(lib.trackfit_linear_attention, LINEAR, workspace_size=f(1000, 3, 4, 32, 32) - 1) == INVALID


STEP = dict(dtype=2, q=P, q_stride=128, k=P, k_stride=128, v=P, v_stride=128, log_decay=P, decay_stride=4, n_seq=7,
            n_heads=4, key_dim=32, value_dim=32, scale=1.0, slots=None, n_slots=7, state_in=P, state_out=P, out=P,
            out_stride=128, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=5), INVALID), (dict(n_seq=-1), INVALID), (dict(n_slots=-1), INVALID), (dict(n_slots=6), INVALID),
    (dict(n_heads=300), UNSUPPORTED), (dict(key_dim=12), UNSUPPORTED), (dict(value_dim=0), UNSUPPORTED),
    (dict(scale=INF), INVALID), (dict(slots=P + 2), INVALID), (dict(state_in=None), INVALID),
    (dict(state_out=None), INVALID), (dict(state_in=P + 4), INVALID), (dict(q=None), INVALID), (dict(k_stride=64), INVALID),
    (dict(log_decay=None), INVALID), (dict(decay_stride=1), INVALID), (dict(out=P + 6), INVALID),
    (dict(n_seq=0, q=None, state_in=None), OK)])
def test_step_refusals(lib, kw, want):
    assert call(lib.trackfit_linear_attention_step, STEP, **kw) == want


CROSS = dict(dtype=1, q=P, q_stride=128, q_offsets=P, n_q_rows=100, k=P, k_stride=64, v=P, v_stride=64, kv_offsets=P,
             n_kv_rows=200, n_seq=3, q_heads=4, kv_heads=2, head_dim=32, scale=0.2, out=P, out_stride=128, workspace=P,
             workspace_size=1 << 40, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), INVALID), (dict(n_q_rows=-1), INVALID), (dict(n_kv_rows=-1), INVALID), (dict(n_seq=-2), INVALID),
    (dict(n_seq=1 << 31), INVALID), (dict(q_heads=3), UNSUPPORTED), (dict(kv_heads=0), UNSUPPORTED),
    (dict(head_dim=36), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(scale=NAN), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q_offsets=None), INVALID), (dict(kv_offsets=P + 4), INVALID),
    (dict(k=None), INVALID), (dict(v=P + 2), INVALID), (dict(k_stride=56), INVALID), (dict(q_stride=130), INVALID),
    (dict(n_seq=0, q=None), OK), (dict(n_q_rows=0, q=None, k=None), OK)])
def test_cross_refusals(lib, kw, want):
    assert call(lib.trackfit_cross_attention, CROSS, **kw) == want


def test_wait_hook_refusals(lib):
    for bad in ((-1, 0), (2_000_000_001, 0), (0, 2), (0, -1)):
        assert lib.trackfit_debug_operator_wait(*bad) == INVALID
    assert lib.trackfit_debug_operator_wait(0, 0) == OK


def test_the_binding_refuses_tensors_on_the_host(lib):
    torch = pytest.importorskip("torch")
    x, off = torch.zeros((4, 2, 16)), torch.tensor([0, 4])
    for call_it in (lambda: T.qk_norm(x, x, x, x),
                    lambda: T.linear_attention(x, x, x, torch.zeros((4, 2)), off, x),
                    lambda: T.linear_attention_step(x, x, x, torch.zeros((4, 2)), torch.zeros((4, 2, 16, 16)),
                                                    torch.zeros((4, 2, 16, 16)), x),
                    lambda: T.cross_attention(x, x, x, off, off, x)):
        with pytest.raises(ValueError):
            call_it()


def test_checks_of_rows_and_vectors():
    """The binding's rules of shapes, types and strides, on host tensors."""
    torch = pytest.importorskip("torch")
    a = object.__new__(T._OpArgs)
    a.what, a.device, a.dtype, a.torch = "op", torch.device("cpu"), torch.float32, torch
    x = torch.zeros((6, 4, 8))
    assert a.rows("x", x, (6, 4, 8)) == (x.data_ptr(), 32)
    assert a.rows("x", x[::2], (3, 4, 8))[1] == 64
    assert a.rows("x", x[:, 1:3], (6, 2, 8)) == (x.data_ptr() + 32, 32)
    for bad, shape in ((x, (6, 4, 16)), (x.half(), (6, 4, 8)), (x[:, ::2], (6, 2, 8)), (x[:, :, ::2], (6, 4, 4)),
                       (x.transpose(0, 1), (4, 6, 8))):
        with pytest.raises(ValueError):
            a.rows("x", bad, shape)
    v = torch.zeros(8)
    assert a.vector("v", None, torch.float32, (8,)) is None and a.vector("v", v, torch.float32, (8,)) == v.data_ptr()
    for bad in (v[:4], v.double(), torch.zeros(16)[::2]):
        with pytest.raises(ValueError):
            a.vector("v", bad, torch.float32, (8,))
    g = torch.zeros((6, 10))
    assert a.decay(g[:, 2:6], 6, 4) == (g.data_ptr() + 8, 10)
    for bad in (g, g[:, ::2], g[:, :4].half()):
        with pytest.raises(ValueError):
            a.decay(bad, 6, 4)


def test_ctypes_signatures_have_as_many_arguments_as_the_header(lib):
    import re
    header = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "trackfit.h")
    src = re.sub(r"/\*.*?\*/", "", open(header).read(), flags=re.S)
    for name in ("trackfit_qk_norm", "trackfit_linear_attention", "trackfit_linear_attention_workspace",
                 "trackfit_linear_attention_step", "trackfit_cross_attention", "trackfit_cross_attention_workspace"):
        params = re.search(name + r"\s*\(([^)]*)\)", src).group(1)
        want = []
        for p in params.split(","):
            want.append(ctypes.c_void_p if "*" in p else {
                "int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "double": ctypes.c_double,
                "size_t": ctypes.c_size_t}[p.split()[0]])
        assert getattr(lib, name).argtypes == want, name
