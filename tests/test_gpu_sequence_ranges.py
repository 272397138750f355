"""The operators on packed sequences at the ends of their types' ranges and over long sums.

u = 2^-24 is a rounding of fp32, e = finfo(type).eps / 2 one of the rows' type."""
import numpy as np
import pytest

from oracle import sequence_oracle as Q
from tests.test_gpu_sequence import T, TYPES, U, dev, half_step, hold, host, linear_tol, rounding, slab  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---------------------------------------------------------------- attention: long sums of one sign

def one_sign(T, t, nq, nk, D, seed):
    r = np.random.default_rng(seed)
    q, k = (dev(0.25 * r.normal(size=(m, 1, D)), t) for m in (nq, nk))
    v = dev(0.5 + r.random((nk, 1, D)), t)
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev([0, nq], "int64"), dev([0, nk], "int64"), out)
    x = torch.einsum("qhd,khd->hqk", q.double(), k.double()) * D ** -0.5
    ref = torch.einsum("hqk,khd->qhd", torch.softmax(x, -1), v.double())
    top = D ** -0.5 * float(q.double().norm(dim=-1).max() * k.double().norm(dim=-1).max())
    return host(out), ref.cpu().numpy(), top


@pytest.mark.parametrize("nq,nk,D", [(16, 16000, 64), (700, 16000, 32), (90, 60000, 64), (2000, 20000, 128)])
def test_cross_fp32_of_values_of_one_sign(T, nq, nk, D):
    """Errors that are rounded to nearest grow with the square root of the states, not with them: each
    sum of n / 16 chunks has a deviation of u sqrt(n / 48) at most, 8 sqrt(n / 16) u holds it for all."""
    out, ref, top = one_sign(T, "float32", nq, nk, D, 24)
    hold(out, ref, ref * (2 * (D + 8) * top + 16 + 8 * np.sqrt(nk / 16)) * U)
    # and they have no sign: their mean is that of the weights' errors, which are common to the channels
    assert abs(np.mean(out / ref - 1)) < 32 * U
