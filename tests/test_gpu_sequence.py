"""The operators on packed sequences on the GPU against their fp64 definitions.

Tolerances.  u = finfo(float32).eps / 2 = 2^-24 is a rounding of fp32, e = finfo(type).eps / 2
one of the rows' type.  An output is held to e |y| (fp16 also to 2^-25, half the distance
of its values below 2^-14, where e no longer says it) for its own rounding plus the roundings on
the way, each relative to the sum of the absolute values of what is added up (the same
definition of |q|, |k|, |v|):
  norm    the sum of D squares, rsqrt, the products with 1/rms and gain, the angle (pi u as a
          fraction of a turn held in 24 bits), sine and cosine, the turned sum: at most 24 u
          of |a| + |b|, the pair's values.
  linear  a decay, a product and two sums a row and head, K products: (6 n + K + 16) u over
          n rows, of the absolute sums; the 16-bit types round the state, or its parts, to 16
          bits as operands, 2 e of the absolute sums.  States: fp32 throughout, (6 n + 16) u.
  cross   a score's error, (D + 8) u of its absolute sum, is the relative error of its weight;
          the sums over n states, (n + 16) u; 16-bit types round the weights once, e.  fp32
          operands are two parts of 11 bits, which loses 8 u more of each product: 2 (D + 8) u
          holds both."""
import numpy as np
import pytest

from oracle import sequence_oracle as Q

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]


@pytest.fixture(scope="module")
def T():
    import os
    from paper_2609_32479_gb300 import trackfit
    if not os.path.exists(trackfit.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    trackfit.load()
    return trackfit


def half_step(t):
    return torch.finfo(getattr(torch, t)).eps / 2 if t != "float32" else U


def rounding(t, y):
    return half_step(t) * np.abs(y) + (2.0 ** -25 if t == "float16" else 0.0)


def dev(x, t="float32"):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda").to(getattr(torch, t))


def host(x):
    return x.detach().double().cpu().numpy()


def hold(got, ref, tol, what=""):
    """|got - ref| <= tol element by element, NaN where the reference is."""
    got, ref = host(got) if torch.is_tensor(got) else got, np.asarray(ref)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref), err_msg=what)
    off = np.where(np.isnan(ref), 0.0, np.abs(got - ref) - tol)
    worst = float(off.max()) if off.size else 0.0
    if worst > 0:
        at = int(np.argmax(off))
        pytest.fail(f"{what}: {got.flat[at]:.6g} for {ref.flat[at]:.6g} at {np.unravel_index(at, off.shape)}, "
                    f"{worst:.3g} over the tolerance of {np.broadcast_to(tol, ref.shape).flat[at]:.3g}")


def slab(r, shapes, t, pad=0):
    """Row arrays that are column blocks of one buffer, with `pad` heads' worth of other columns between."""
    n = shapes[0][0]
    widths = [h * d for _, h, d in shapes]
    x = dev(r.normal(size=(n, sum(widths) + pad * len(shapes))), t)
    out, c = [], 0
    for (_, h, d), w in zip(shapes, widths):
        out.append(x[:, c:c + w].unflatten(1, (h, d)))
        c += w + pad
    return out


# ---------------------------------------------------------------- norms and rotation

def norm_tol(x, gain, eps, rot, t, y):
    z = np.abs(Q.qk_norm(x, gain, eps))
    h = rot // 2
    pair = z.copy()
    pair[..., :h] += z[..., h:rot]
    pair[..., h:rot] += z[..., :h]
    return rounding(t, y) + 24 * U * pair


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,hq,hk,d,rot", [(1, 1, 0, 8, 0), (1, 1, 1, 16, 16), (5, 4, 4, 32, 32), (33, 6, 2, 48, 32),
                                           (64, 3, 1, 24, 16), (777, 8, 8, 64, 64), (130, 5, 5, 40, 0),
                                           (257, 2, 1, 128, 128), (40, 2, 2, 128, 48), (41000, 2, 1, 16, 16)])
def test_norm(T, t, n, hq, hk, d, rot):
    r = np.random.default_rng(n + d)
    q, k, _ = slab(r, [(n, hq, d), (n, max(hk, 1), d), (n, 1, d)], t)
    k = k if hk else None
    gq, gk = r.normal(size=d).astype(np.float32), r.normal(size=d).astype(np.float32)
    pos = r.integers(-5, 5000, n).astype(np.int32)
    qo = torch.empty((n, hq, d), dtype=q.dtype, device="cuda")
    ko = torch.empty((n, hk, d), dtype=q.dtype, device="cuda") if hk else None
    T.qk_norm(q, k, qo, ko, q_gain=dev(gq), k_gain=dev(gk), eps=1e-5, positions=dev(pos, "int32"), rot_dim=rot)
    for x, g, o in ((q, gq, qo), (k, gk, ko))[:2 if hk else 1]:
        ref = Q.qk_norm(host(x), g, 1e-5, pos, rot)
        hold(o, ref, norm_tol(host(x), g, 1e-5, rot, t, ref))


@pytest.mark.parametrize("t", TYPES)
def test_norm_in_place_at_far_positions_and_of_zeros(T, t):
    r = np.random.default_rng(3)
    n, h, d = 50, 2, 32
    q, k = slab(r, [(n, h, d), (n, h, d)], t)
    q[7] = 0
    x, y = host(q), host(k)
    pos = r.integers(-2 ** 31, 2 ** 31 - 1, n).astype(np.int32)
    pos[:4] = [2 ** 31 - 1, -2 ** 31, 0, 1]
    T.qk_norm(q, k, q, k, positions=dev(pos, "int32"), rot_dim=32)
    # the definition's own angle is off by its rounding in 64 bits: |angle| 2^-53 a step, three steps
    more = 3 * 2.0 ** 31 * 2.0 ** -53
    for a, got in ((x, q), (y, k)):
        ref = Q.qk_norm(a, None, 1e-6, pos, 32)
        z = np.abs(Q.qk_norm(a, None, 1e-6))
        hold(got, ref, norm_tol(a, None, 1e-6, 32, t, ref) + more * (z + np.roll(z, 16, -1)))


def test_norm_keeps_a_row_that_is_not_finite_to_itself(T):
    r = np.random.default_rng(4)
    q, k = slab(r, [(9, 2, 16), (9, 2, 16)], "float32")
    q[4, 1, 3] = float("nan")
    k[2, 0, 0] = float("inf")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    T.qk_norm(q, k, qo, ko, positions=torch.arange(9, dtype=torch.int32, device="cuda"), rot_dim=16)
    bad = torch.zeros((9, 2), dtype=torch.bool)
    bad[4, 1] = True
    assert torch.equal(torch.isnan(qo).any(-1).cpu(), bad)
    bad = torch.zeros((9, 2), dtype=torch.bool)
    bad[2, 0] = True
    assert torch.equal(torch.isnan(ko).any(-1).cpu(), bad)


# ---------------------------------------------------------------- linear attention

def linear_tol(q, k, v, g, off, scale, rev, s0, t, o, s):
    """(tolerance of out, of the states)"""
    n = int(np.max(np.diff(off))) if len(off) > 1 else 0
    oa, sa = Q.linear_attention(np.abs(q), np.abs(k), np.abs(v), g, off, abs(scale), rev,
                                None if s0 is None else np.abs(s0))
    K = q.shape[2]
    # rows behind a decay to nothing do not add roundings: n counts at most what 2^-24 leaves of the slowest head
    slow = float(np.max(np.mean(np.maximum(g, -30.0), 0))) if len(g) else 0.0
    n = min(n, 17 / max(-slow, 1e-9) + 64)
    e = half_step(t)
    to = rounding(t, o) + ((6 * n + K + 16) * U + (2 * e if t != "float32" else 0.0)) * oa
    return to, (6 * n + 16) * U * sa


def check_linear(T, lengths, H, K, V, t, rev=False, states=True, lead=0, tail=0, seed=0, resets=0.01, strong=0.5,
                 shared_out=False):
    r = np.random.default_rng(seed + 1000 * K + V)
    off = lead + np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    n, B = int(off[-1]) + tail, len(lengths)
    q, k, v = slab(r, [(n, H, K), (n, H, K), (n, H, V)], t, pad=8)
    g = -strong * r.random((n, H)) * 10.0 ** -r.integers(0, 3, H)
    g[r.random((n, H)) < resets] = -40.0
    g[r.random((n, H)) < resets] = -np.inf
    gd = dev(g)
    g = host(gd)
    s0 = r.normal(size=(B, H, K, V)).astype(np.float32) if states else None
    out = torch.full((n, H, V), float("nan"), dtype=q.dtype, device="cuda")
    s1 = torch.full((B, H, K, V), float("nan"), device="cuda") if states else None
    T.linear_attention(q, k, v, gd, dev(off, "int64"), out, scale=0.3, reverse=rev,
                       state_in=dev(s0) if states else None, state_out=s1)
    args = host(q), host(k), host(v), g, off, 0.3, rev, s0
    o, s = Q.linear_attention(*args)
    to, ts = linear_tol(*args, t, o, s)
    hold(out, o, to, "out")
    if states:
        hold(s1, s, ts, "state")
    return out, s1


SHORT = [0, 1, 2, 7, 8, 9, 15, 16, 17, 0, 0, 31, 32, 33, 63, 64, 65, 20, 1]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("K,V", [(8, 8), (16, 16), (32, 32), (24, 40), (64, 64), (40, 128), (128, 24), (128, 128), (96, 80)])
def test_linear_short(T, t, rev, K, V):
    check_linear(T, SHORT, 2, K, V, t, rev, states=True)
    check_linear(T, SHORT, 3, K, V, t, rev, states=False, lead=5, tail=9)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lengths", [[512, 513, 0, 511], [1100], [3, 2500, 1, 0, 600, 255, 256, 257], [256, 768, 1024, 1]])
def test_linear_long(T, t, rev, lengths):
    check_linear(T, lengths, 2, 32, 32, t, rev, states=True, seed=1)
    check_linear(T, lengths, 1, 64, 40, t, rev, states=False, lead=7, tail=300, seed=2)


@pytest.mark.parametrize("t", TYPES)
def test_linear_many_tracks(T, t):
    r = np.random.default_rng(11)
    check_linear(T, r.integers(8, 21, 1500), 4, 32, 32, t, states=False)
    check_linear(T, r.integers(0, 65, 300), 4, 32, 48, t, True, states=True)


@pytest.mark.parametrize("t", TYPES)
def test_linear_without_decay_and_of_single_rows(T, t):
    check_linear(T, [1] * 70, 2, 32, 32, t, strong=0.0, resets=0.0)
    check_linear(T, [700, 40], 2, 16, 16, t, strong=0.0, resets=0.0, states=True)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("length", [40, 1300])
def test_linear_keeps_what_is_not_finite_to_its_sequence(T, t, length):
    r = np.random.default_rng(5)
    H, K = 2, 32
    off = np.array([0, 20, 20 + length, 40 + length], np.int64)
    n = int(off[-1])
    q, k, v = slab(r, [(n, H, K)] * 3, t)
    for x, at in ((q, 30), (k, 31), (v, 32)):
        x[at, 0, 5] = float("nan")
    v[33, 1, 3] = float("inf")
    g = dev(-0.1 * r.random((n, H)))
    out = torch.empty((n, H, K), dtype=q.dtype, device="cuda")
    s1 = torch.empty((3, H, K, K), device="cuda")
    T.linear_attention(q, k, v, g, dev(off, "int64"), out, state_out=s1)
    ok = torch.isfinite(out).all(-1).all(-1).cpu()
    assert ok[:30].all() and ok[20 + length:].all() and not ok[33]
    assert torch.isfinite(s1[[0, 2]]).all() and not torch.isfinite(s1[1]).all()


@pytest.mark.parametrize("t", TYPES)
def test_linear_states_in_place_and_in_parts(T, t):
    """A sequence in three calls, its state in one array, is the sequence in one."""
    r = np.random.default_rng(6)
    H, K, n = 2, 32, 700
    q, k, v = slab(r, [(n, H, K)] * 3, t)
    g = dev(-0.05 * r.random((n, H)))
    whole, s1 = torch.empty((n, H, K), dtype=q.dtype, device="cuda"), torch.empty((1, H, K, K), device="cuda")
    T.linear_attention(q, k, v, g, dev([0, n], "int64"), whole, state_out=s1)
    parts, s2 = torch.empty_like(whole), torch.zeros((1, H, K, K), device="cuda")
    for lo, hi in ((0, 100), (100, 101), (101, n)):
        T.linear_attention(q[lo:hi], k[lo:hi], v[lo:hi], g[lo:hi], dev([0, hi - lo], "int64"), parts[lo:hi],
                           state_in=s2, state_out=s2)
    args = host(q), host(k), host(v), host(g), [0, n], 1.0, False, None
    o, s = Q.linear_attention(*args)
    to, ts = linear_tol(*args, t, o, s)
    hold(parts, o, to)
    hold(whole, o, to)
    hold(s2, s, ts)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
def test_linear_states_in_place_of_long_sequences(T, t, rev):
    """The parts of a long sequence run in any order: its first part still begins with the state
    before the call, though the last part may put the state after it in the same place.  (More
    parts than the GPU holds at a time, the first in the recurrence's direction last.)"""
    H, K, n = 8, 64, 200000 if t != "float32" else 60000
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((n, H, K), generator=g, device="cuda").to(getattr(torch, t)) for _ in range(3))
    d = -0.02 * torch.rand((n, H), generator=g, device="cuda")
    off = dev([0, 600, n - 700, n], "int64")
    s0 = 10 * torch.randn((3, H, K, K), generator=g, device="cuda")
    s1, s2 = torch.empty_like(s0), s0.clone()
    a, b = torch.empty_like(q), torch.empty_like(q)
    T.linear_attention(q, k, v, d, off, a, reverse=rev, state_in=s0, state_out=s1)
    T.linear_attention(q, k, v, d, off, b, reverse=rev, state_in=s2, state_out=s2)
    assert torch.equal(s1, s2) and torch.equal(a, b)


def test_linear_is_the_same_wherever_a_sequence_stands(T):
    """Bit for bit: the other sequences of a batch, their order and number do not matter."""
    r = np.random.default_rng(7)
    lengths = r.integers(0, 40, 200)
    off = np.concatenate([[0], np.cumsum(lengths)])
    n = int(off[-1])
    q, k, v = slab(r, [(n, 2, 32)] * 3, "bfloat16")
    g = dev(-r.random((n, 2)))
    out = torch.empty((n, 2, 32), dtype=q.dtype, device="cuda")
    T.linear_attention(q, k, v, g, dev(off, "int64"), out)
    p = r.permutation(200)
    rows = torch.from_numpy(np.concatenate([np.arange(off[b], off[b + 1]) for b in p])).cuda()
    out2 = torch.empty_like(out)
    T.linear_attention(q[rows].contiguous(), k[rows].contiguous(), v[rows].contiguous(), g[rows].contiguous(),
                       dev(np.concatenate([[0], np.cumsum(lengths[p])]), "int64"), out2)
    assert torch.equal(out[rows], out2)


# ---------------------------------------------------------------- a single row

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,H,K,V", [(1, 1, 8, 8), (5, 4, 32, 32), (97, 3, 24, 40), (33, 2, 64, 64), (7, 2, 128, 128),
                                     (9, 1, 96, 16)])
@pytest.mark.parametrize("slots", [False, True])
def test_step(T, t, B, H, K, V, slots):
    r = np.random.default_rng(B + K)
    q, k, v = slab(r, [(B, H, K), (B, H, K), (B, H, V)], t)
    g = dev(-r.random((B, H)) * np.where(r.random((B, H)) < 0.1, np.inf, 1.0))
    ns = B + 5
    s0 = dev(r.normal(size=(ns, H, K, V)))
    s1 = torch.full_like(s0, 7.0)
    out = torch.empty((B, H, V), dtype=q.dtype, device="cuda")
    at = r.permutation(ns)[:B] if slots else np.arange(B)
    T.linear_attention_step(q, k, v, g, s0, s1, out, scale=0.5, slots=dev(at, "int32") if slots else None)
    args = host(q), host(k), host(v), host(g), host(s0)[at], 0.5
    o, s = Q.linear_attention_step(*args)
    oa, sa = Q.linear_attention_step(*(np.abs(x) for x in args[:3]), args[3], np.abs(args[4]), 0.5)
    hold(out, o, rounding(t, o) + (K + 12) * U * oa)
    hold(s1[torch.from_numpy(at).cuda()], s, 5 * U * sa)
    others = np.setdiff1d(np.arange(ns), at)
    assert bool((s1[torch.from_numpy(others).cuda()] == 7.0).all())
    T.linear_attention_step(q, k, v, g, s0, s0, out, scale=0.5, slots=dev(at, "int32") if slots else None)
    assert torch.equal(s0[torch.from_numpy(at).cuda()], s1[torch.from_numpy(at).cuda()])


def test_step_of_a_padded_batch(T):
    r = np.random.default_rng(1)
    B, H, K = 6, 2, 16
    q, k, v = slab(r, [(B, H, K)] * 3, "bfloat16")
    s = dev(r.normal(size=(4, H, K, K)))
    before = s.clone()
    out = torch.zeros((B, H, K), dtype=q.dtype, device="cuda")
    T.linear_attention_step(q, k, v, torch.zeros((B, H), device="cuda"), s, s, out,
                            slots=torch.tensor([2, -1, 4, 0, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda"))
    assert torch.isnan(out[[1, 2, 4, 5]]).all() and torch.isfinite(out[[0, 3]]).all()
    assert torch.equal(s[[1, 3]], before[[1, 3]]) and not torch.equal(s[[0, 2]], before[[0, 2]])


@pytest.mark.parametrize("t", TYPES)
def test_steps_after_a_sequence_go_on_with_it(T, t):
    """A prompt of 40 rows, then 5 single rows, is the sequence of 45."""
    r = np.random.default_rng(2)
    B, H, K, n = 3, 2, 32, 45
    q, k, v = (x.unflatten(0, (B, n)) for x in slab(r, [(B * n, H, K)] * 3, t))
    g = dev(-0.2 * r.random((B, n, H)))
    s = torch.zeros((B, H, K, K), device="cuda")
    first = [x[:, :40].reshape(B * 40, *x.shape[2:]).contiguous() for x in (q, k, v, g)]
    out = torch.empty((B * 40, H, K), dtype=q.dtype, device="cuda")
    T.linear_attention(*first, torch.arange(0, B * 40 + 1, 40, device="cuda"), out, state_out=s)
    last = torch.empty((B, H, K), dtype=q.dtype, device="cuda")
    for i in range(40, n):
        T.linear_attention_step(q[:, i], k[:, i], v[:, i], g[:, i], s, s, last)
    flat = [host(x).reshape(B * n, *x.shape[2:]) for x in (q, k, v, g)]
    args = (*flat, np.arange(0, B * n + 1, n), 1.0, False, None)
    o, st = Q.linear_attention(*args)
    to, ts = linear_tol(*args, t, o, st)
    hold(last, o.reshape(B, n, H, K)[:, -1], to.reshape(B, n, H, K)[:, -1])
    hold(s, st, ts)


# ---------------------------------------------------------------- attention to states

def check_cross(T, nq, nk, Hq, Hk, D, t, lead=0, tail=0, seed=0, scale=None, spread=1.0):
    r = np.random.default_rng(seed + 100 * D + Hq)
    qo = lead + np.concatenate([[0], np.cumsum(nq)]).astype(np.int64)
    ko = 2 * lead + np.concatenate([[0], np.cumsum(nk)]).astype(np.int64)
    Nq, Nk = int(qo[-1]) + tail, int(ko[-1]) + tail
    (q,) = slab(r, [(Nq, Hq, D)], t, pad=8)
    q *= spread
    k, v = slab(r, [(Nk, Hk, D), (Nk, Hk, D)], t, pad=16)
    out = torch.full((Nq, Hq, D), float("nan"), dtype=q.dtype, device="cuda")
    sc = D ** -0.5 if scale is None else scale
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), out, scale=scale)
    ref = Q.cross_attention(host(q), host(k), host(v), qo, ko, sc)
    # the weights' errors act on values of both signs: held against the weighted sum of |v|
    absv = np.nan_to_num(Q.cross_attention(host(q), host(k), np.abs(host(v)), qo, ko, sc))
    top = sc * float(np.max(np.linalg.norm(host(q), axis=-1), initial=0.0)) * float(
        np.max(np.linalg.norm(host(k), axis=-1), initial=0.0))   # of |score|, and of its absolute sum up to sqrt(D)
    e = half_step(t)
    n = int(np.max(nk, initial=0))
    tol = rounding(t, np.nan_to_num(ref)) + absv * (2 * (D + 8) * abs(top) * U + (n + 16) * U + (e if t != "float32" else 0))
    hold(out, ref, tol)
    return out


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("Hq,Hk,D", [(1, 1, 8), (4, 4, 32), (4, 2, 24), (6, 1, 64), (2, 2, 40), (16, 4, 128), (3, 3, 96)])
def test_cross_short(T, t, Hq, Hk, D):
    check_cross(T, [5, 1, 0, 5, 2, 17, 3, 16, 33, 1], [12, 1, 7, 0, 20, 16, 64, 65, 33, 15], Hq, Hk, D, t)
    check_cross(T, [5] * 40, np.random.default_rng(1).integers(0, 21, 40), Hq, Hk, D, t, lead=3, tail=6)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("nq,nk", [([1], [3000]), ([1, 2, 1, 0, 4], [700, 0, 2049, 33, 1]), ([130], [1025]),
                                   ([300, 0, 129], [257, 63, 0]), ([64, 257, 1], [511, 640, 1300])])
def test_cross_long(T, t, nq, nk):
    check_cross(T, nq, nk, 2, 2, 64, t)
    check_cross(T, nq, nk, 4, 1, 32, t, lead=2, tail=5, seed=1)
    check_cross(T, nq, nk, 2, 1, 128, t, seed=2)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("nq,nk", [([1, 2] * 10, [700] * 20), ([2, 0, 3, 1], [3000, 10, 1, 5000]),
                                   ([1] * 70, list(range(200, 1600, 20))), ([7, 7, 7], [900, 1000, 0])])
def test_cross_of_few_queries(T, t, nq, nk):
    """Few tiles: split ranges, and tiles of fewer rows."""
    check_cross(T, nq, nk, 4, 4, 64, t)
    check_cross(T, nq, nk, 6, 2, 32, t, lead=1, tail=3, seed=4)
    check_cross(T, nq, nk, 3, 1, 128, t, seed=5)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D", [64, 8, 40, 72, 128])
@pytest.mark.parametrize("nq,nk", [([128], [512]), ([300, 40, 0, 500], [3000, 100, 50, 128]),
                                   ([1, 129, 127, 700], [1, 2047, 127, 4097]), ([64] * 9, [513] * 9)])
def test_cross_of_many_queries_to_many_states(T, t, D, nq, nk):
    """Averages of 64 queries and 512 states and more; among them sequences of few."""
    check_cross(T, nq, nk, 2, 2, D, t)
    check_cross(T, nq, nk, 6, 2, D, t, lead=3, tail=140, seed=3)


@pytest.mark.parametrize("t", TYPES)
def test_cross_of_growing_scores(T, t):
    """Later states score higher and higher: the maximum that the weights are taken against moves."""
    r = np.random.default_rng(12)
    n, m, D = 200, 1500, 64
    q = dev(1.0 + 0.1 * r.normal(size=(n, 1, D)), t)
    k = dev(np.linspace(-6, 6, m)[:, None, None] * np.ones((m, 1, D)) + 0.1 * r.normal(size=(m, 1, D)), t)
    v = dev(r.normal(size=(m, 1, D)), t)
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev([0, n], "int64"), dev([0, m], "int64"), out)
    args = host(q), host(k)
    ref = Q.cross_attention(*args, host(v), [0, n], [0, m], D ** -0.5)
    absv = Q.cross_attention(*args, np.abs(host(v)), [0, n], [0, m], D ** -0.5)
    # a score of up to 60 is a sum of D terms of one sign: its error is D + 8 roundings of the score
    tol = rounding(t, ref) + absv * (2 * (D + 8) * 60 * U + (m + 16) * U + (half_step(t) if t != "float32" else 0))
    hold(out, ref, tol)


@pytest.mark.parametrize("t", TYPES)
def test_cross_of_sharp_and_flat_scores(T, t):
    check_cross(T, [40, 3], [100, 900], 2, 2, 32, t, spread=16.0)
    check_cross(T, [40, 3], [100, 900], 2, 2, 32, t, scale=0.0)
    check_cross(T, [40, 3], [100, 900], 2, 2, 32, t, scale=-0.25)
    check_cross(T, [200], [900], 2, 2, 32, t, spread=16.0)
    check_cross(T, [200], [900], 2, 2, 32, t, scale=0.0)
    check_cross(T, [200], [900], 2, 2, 32, t, scale=-0.25)


@pytest.mark.parametrize("t", TYPES)
def test_cross_keeps_what_is_not_finite_to_its_sequence(T, t):
    r = np.random.default_rng(9)
    nq, nk = [5, 5, 200, 5], [12, 12, 100, 12]
    qo, ko = np.concatenate([[0], np.cumsum(nq)]), np.concatenate([[0], np.cumsum(nk)])
    (q,) = slab(r, [(qo[-1], 2, 32)], t)
    k, v = slab(r, [(ko[-1], 2, 32)] * 2, t)
    k[13, 0, 3] = float("nan")
    v[30, 1, 3] = float("inf")
    q[11, 0, 0] = float("nan")
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), out)
    ok = torch.isfinite(out).cpu()
    assert ok[:5].all() and ok[-5:].all()
    assert not ok[5:10, 0].any() and ok[5:10, 1].all()
    assert not ok[11, 0].any() and ok[12:210, 0].all()
    assert not ok[10:210, 1, 3].any() and ok[10:210, 1, :3].all()


@pytest.mark.parametrize("t", TYPES)
def test_cross_of_many_keeps_what_is_not_finite_to_its_sequence(T, t):
    r = np.random.default_rng(10)
    nq, nk = [100, 90, 200], [600, 700, 600]
    qo, ko = np.concatenate([[0], np.cumsum(nq)]), np.concatenate([[0], np.cumsum(nk)])
    (q,) = slab(r, [(qo[-1], 2, 32)], t)
    k, v = slab(r, [(ko[-1], 2, 32)] * 2, t)
    k[700, 0, 3] = float("nan")
    v[1200, 1, 3] = float("inf")
    q[250, 0, 0] = float("nan")
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), out)
    ok = torch.isfinite(out).cpu()
    assert ok[:100].all() and ok[190:250].all() and ok[251:].all() and ok[250, 1].all()
    assert not ok[100:190, 0].any() and not ok[250, 0].any()
    assert not ok[100:190, 1, 3].any() and ok[100:190, 1, :3].all()


def test_an_expired_wait_is_reported_and_the_next_call_is_right(T):
    """A loader that holds its first block back: the waits for it give up after 20 ms, the call
    returns, the error is reported once, and the same call afterwards is right."""
    torch.cuda.synchronize()
    assert T.operator_errors() == T.OK
    x = torch.randn((700, 1, 64), device="cuda").to(torch.bfloat16)
    off = dev([0, 700], "int64")
    want, out = torch.empty_like(x), torch.empty_like(x)
    T.cross_attention(x, x, x, off, off, want)
    T.debug_operator_wait(20_000_000, True)
    try:
        T.cross_attention(x, x, x, off, off, out)
        assert T.operator_errors() == T.ERR_TIMEOUT
        assert T.operator_errors() == T.OK
    finally:
        T.debug_operator_wait()
    T.cross_attention(x, x, x, off, off, out)
    assert T.operator_errors() == T.OK and torch.equal(out, want)


def test_no_wait_has_expired(T):
    torch.cuda.synchronize()
    assert T.operator_errors() == T.OK


def test_cross_of_scores_that_are_all_minus_infinity_is_zero(T):
    q = torch.ones((2, 1, 16), device="cuda")
    k = torch.full((9, 1, 16), float("-inf"), device="cuda")
    v = torch.ones((9, 1, 16), device="cuda")
    for t in TYPES:
        out = torch.full((2, 1, 16), 5.0, device="cuda", dtype=getattr(torch, t))
        T.cross_attention(q.to(out.dtype), k.to(out.dtype), v.to(out.dtype), dev([0, 2], "int64"), dev([0, 9], "int64"), out)
        assert bool((out == 0).all())
        many = torch.full((150, 1, 16), 5.0, device="cuda", dtype=out.dtype)
        T.cross_attention(torch.ones_like(many), k[:1].expand(700, 1, 16).to(out.dtype).contiguous(),
                          v[:1].expand(700, 1, 16).to(out.dtype).contiguous(), dev([0, 150], "int64"),
                          dev([0, 700], "int64"), many)
        assert bool((many == 0).all())


# ---------------------------------------------------------------- together, streams, graphs

def layer(T, x, offsets, cross_kv, kv_offsets, positions, gain, out, stream=None, work=(None, None)):
    """What mixes the rows of an encoder layer, out of a projection x [N, 3 H D + ...]: the norms with
    rotation, linear attention both ways, then attention of the result to other states."""
    H, D = 4, 32
    n = x.shape[0]
    q, k, v = (x[:, i * H * D:(i + 1) * H * D].unflatten(1, (H, D)) for i in range(3))
    T.qk_norm(q, k, out["q"], out["k"], q_gain=gain, k_gain=gain, positions=positions, rot_dim=32, stream=stream)
    T.linear_attention(out["q"], out["k"], v, out["g"], offsets, out["f"], scale=D ** -0.5, stream=stream, workspace=work[0])
    T.linear_attention(out["q"], out["k"], v, out["g"], offsets, out["b"], scale=D ** -0.5, reverse=True, stream=stream,
                       workspace=work[0])
    T.qk_norm(out["f"], out["b"], out["f"], out["b"], stream=stream)
    T.cross_attention(out["f"], cross_kv[0], cross_kv[1], offsets, kv_offsets, out["y"], stream=stream, workspace=work[1])
    return n


def layer_inputs(seed, lengths, nk, t):
    r = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(lengths)])
    ko = np.concatenate([[0], np.cumsum(nk)])
    n, H, D = int(off[-1]), 4, 32
    x = dev(r.normal(size=(n, 3 * H * D)), t)
    kv = slab(r, [(int(ko[-1]), H, D)] * 2, t)
    out = {c: torch.full((n, H, D), float("nan"), dtype=x.dtype, device="cuda") for c in "qkfby"}
    out["g"] = dev(-0.3 * r.random((n, H)))
    pos = np.concatenate([np.arange(m) for m in lengths]).astype(np.int32)
    return x, dev(off, "int64"), kv, dev(ko, "int64"), dev(pos, "int32"), dev(1 + 0.1 * r.normal(size=D)), out


@pytest.mark.parametrize("t", TYPES)
def test_layer(T, t):
    """The operators one after the other, each against its definition of what it was given."""
    lengths, nk = [20, 13, 0, 600, 8], [9, 0, 4, 700, 30]
    x, off, kv, ko, pos, gain, out = layer_inputs(1, lengths, nk, t)
    layer(T, x, off, kv, ko, pos, gain, out)
    H, D = 4, 32
    q, k, v = (host(x)[:, i * H * D:(i + 1) * H * D].reshape(-1, H, D) for i in range(3))
    for a, c in ((q, "q"), (k, "k")):
        ref = Q.qk_norm(a, host(gain), 1e-6, host(pos), 32)
        hold(out[c], ref, norm_tol(a, host(gain), 1e-6, 32, t, ref), c)
    for c, rev in (("f", False), ("b", True)):
        args = host(out["q"]), host(out["k"]), v, host(out["g"]), off.tolist(), D ** -0.5, rev, None
        o, s = Q.linear_attention(*args)
        to, _ = linear_tol(*args, t, o, s)
        # the norm divides by a head's rms and turns an error of tol into tol / rms, and as much again by the rms' own
        rms = np.sqrt(np.mean(o * o, -1, keepdims=True) + 1e-6)
        ref = Q.qk_norm(o, None, 1e-6)
        slack = to / rms + np.abs(ref) * np.sqrt(np.mean(to * to, -1, keepdims=True)) / rms
        hold(out[c], ref, 2 * slack + norm_tol(o, None, 1e-6, 0, t, ref), c)
    ref = Q.cross_attention(host(out["f"]), host(kv[0]), host(kv[1]), off.tolist(), ko.tolist(), D ** -0.5)
    absv = Q.cross_attention(host(out["f"]), host(kv[0]), np.abs(host(kv[1])), off.tolist(), ko.tolist(), D ** -0.5)
    top = D ** -0.5 * np.linalg.norm(host(out["f"]), axis=-1).max() * np.linalg.norm(host(kv[0]), axis=-1).max()
    e = half_step(t)
    hold(out["y"], ref, rounding(t, ref) + absv * (2 * (D + 8) * top * U + 716 * U + (e if t != "float32" else 0)), "y")


def test_layer_on_a_stream_and_in_a_graph(T):
    lengths, nk = [20, 13, 0, 900, 8], [9, 0, 4, 3000, 30]
    x, off, kv, ko, pos, gain, out = layer_inputs(2, lengths, nk, "bfloat16")
    layer(T, x, off, kv, ko, pos, gain, out)
    torch.cuda.synchronize()
    want = {c: t.clone() for c, t in out.items()}

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for t in "qkfby":
        out[t].fill_(float("nan"))
    torch.cuda.synchronize()
    layer(T, x, off, kv, ko, pos, gain, out, stream=st)
    st.synchronize()
    for c in "qkfby":
        assert torch.equal(out[c], want[c]), c

    n = x.shape[0]
    work = tuple(torch.empty(max(b, 16), dtype=torch.uint8, device="cuda") for b in (
        T.linear_attention_workspace(n, len(lengths), 4, 32, 32),
        int(T.load().trackfit_cross_attention_workspace(1, n, kv[0].shape[0], len(lengths), 4, 4, 32))))
    for use in (work, (None, None)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(T, x, off, kv, ko, pos, gain, out, work=use)
        for _ in range(2):
            for t in "qkfby":
                out[t].fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for c in "qkfby":
                assert torch.equal(out[c], want[c]), c
    # other offsets and rows of the same total, replayed: nothing was kept from the capture
    off.copy_(dev(np.concatenate([[0], np.cumsum([8, 900, 0, 20, 13])]), "int64"))
    ko.copy_(dev(np.concatenate([[0], np.cumsum([3000, 9, 30, 4, 0])]), "int64"))
    x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    got = {c: t.clone() for c, t in out.items()}
    layer(T, x, off, kv, ko, pos, gain, out)
    torch.cuda.synchronize()
    for c in "qkfby":
        assert torch.equal(out[c], got[c]), c


def test_calls_at_once_on_two_streams(T):
    """Two streams with workspaces of their own do not disturb one another."""
    both = [layer_inputs(s, [1500, 3, 700], [2000, 1, 40], "float16") for s in (3, 4)]
    want = []
    for x, off, kv, ko, pos, gain, out in both:
        layer(T, x, off, kv, ko, pos, gain, out)
        torch.cuda.synchronize()
        want.append({c: out[c].clone() for c in "qkfby"})
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (x, off, kv, ko, pos, gain, out) in zip(streams, both):
            layer(T, x, off, kv, ko, pos, gain, out, stream=st)
    torch.cuda.synchronize()
    for (x, off, kv, ko, pos, gain, out), w in zip(both, want):
        for c in "qkfby":
            assert torch.equal(out[c], w[c]), c


def test_empty_calls(T):
    e = lambda *s: torch.empty(s, device="cuda")
    T.qk_norm(e(0, 2, 16), None, e(0, 2, 16), None)
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    s0, s1 = torch.randn((3, 2, 16, 8), device="cuda"), e(3, 2, 16, 8)
    T.linear_attention(e(0, 2, 16), e(0, 2, 16), e(0, 2, 8), e(0, 2), off, e(0, 2, 8), state_in=s0, state_out=s1)
    assert torch.equal(s0, s1)
    T.linear_attention(e(0, 2, 16), e(0, 2, 16), e(0, 2, 8), e(0, 2), off, e(0, 2, 8), state_out=s1)
    assert bool((s1 == 0).all())
    T.linear_attention(e(5, 2, 16), e(5, 2, 16), e(5, 2, 8), e(5, 2), off[:1], e(5, 2, 8))
    T.linear_attention_step(e(0, 2, 16), e(0, 2, 16), e(0, 2, 8), e(0, 2), s0, s1, e(0, 2, 8))
    out = torch.ones((3, 2, 16), device="cuda")
    T.cross_attention(torch.ones((3, 2, 16), device="cuda"), e(0, 1, 16), e(0, 1, 16),
                      torch.tensor([0, 1, 1, 3], device="cuda"), off, out)
    assert bool((out == 0).all())
    T.cross_attention(e(0, 2, 16), e(4, 1, 16), e(4, 1, 16), off, off, e(0, 2, 16))
