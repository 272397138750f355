"""The gated scan with its gradients and its single row, the norm with a residual's addition and
the product with its epilogue on the GPU, against their fp64 definitions.

Tolerances.  u = 2^-24 is a rounding of fp32, e a rounding of the rows' type (half its eps); an
output is held to e |y| (fp16 also to 2^-25, half the distance of its values below 2^-14; e4m3
below) plus the roundings on the way:
  scan     z and 1 - z are off by k u of themselves, k = 2 |p| + 10, as the header says.  So a
           state's error is at most E_t = (1 - z) E_{t-1} + (k + 6) u ((1 - z) H_{t-1} + z |n|),
           H the scan of |n|, |h_0|: six more roundings for w h + z n and the joining of a
           part's w products.  Parts of rows are joined through (factor, sum) pairs, two
           roundings a part: 2 u H for each of the at most n / 16 + 16 of a sequence.
  back     likewise for D with |g|: F_t = (1 - z) F_{t+1} + ... ; dn is z D, dp is
           z (1 - z) (n - h) D: products of values with these errors, (2 k + 8) u more.
  step     w h + z n: (k + 6) u (w |h| + z |n|).
  norm     the sum's rounding and that of the squares' sum, sqrt, quotient and the products:
           (C / 32 + 16) u |y| holds any order of adding C squares in lanes (all of one sign),
           and x + delta is rounded once in fp32 (u of |x| + |delta|, relative to the row's
           norm).
           e4m3: y / scale is off by those and a division; its nearest value is either of two
           where it lies that near to a border, so the result is within half a step of the
           8-bit type (2^-4 of the value, 2^-10 below 2^-6) and the error before it.
  product  exact products, K sums, each off by 2 u of the absolute sum at most: (2 K + 8) u S;
           the activations' slopes are at most 1.13, their own error 16 u of the value, and
           4 y^2 u of it for the far tail of gelu (the argument's rounding); sigma(gate) as
           above."""
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


@pytest.fixture(autouse=True)
def no_wait_expires(T):
    yield
    assert T.operator_errors() == T.OK


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


def slab(r, n, widths, t, pad=8, size=1.0):
    """Matrices that are column blocks of one buffer, `pad` other columns between."""
    x = dev(size * r.normal(size=(n, sum(widths) + pad * len(widths))), t)
    out, c = [], 0
    for w in widths:
        out.append(x[:, c:c + w])
        c += w + pad
    return out


def offsets_of(lengths, lead=0):
    return lead + np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


# ---------------------------------------------------------------- scan

def k_of(p):
    return 2 * np.minimum(np.abs(p), 100.0) + 10


def scan_bounds(p, n, off, rev, s0):
    """(E [N, C], of the states [B, C], H [N, C])."""
    z, w = Q.logistic(p), Q.logistic(-p)
    B, C = len(off) - 1, p.shape[1]
    H, Hs = Q.gated_scan(p, np.abs(n), off, rev, None if s0 is None else np.abs(s0))
    E, Es = np.full(p.shape, np.nan), np.zeros((B, C))
    top = 1.0
    for b in range(B):
        rows = list(range(int(off[b]), int(off[b + 1])))
        if rev:
            rows.reverse()
        e = np.zeros(C)
        h = np.zeros(C) if s0 is None else np.abs(s0[b])
        most = h.copy()
        for t in rows:
            e = w[t] * e + (k_of(p[t]) + 6) * U * (w[t] * h + z[t] * np.abs(n[t]))
            h = H[t]
            E[t] = e + 2 * U * (len(rows) / 16 + 16) * h
        Es[b] = e + 2 * U * (len(rows) / 16 + 16) * (h if rows else 0.0)
    return E, Es, H


def back_bounds(p, n, off, g, rev, s0, ds):
    z, w = Q.logistic(p), Q.logistic(-p)
    B, C = len(off) - 1, p.shape[1]
    E, _, H = scan_bounds(p, n, off, rev, s0)
    h, _ = Q.gated_scan(p, n, off, rev, s0)
    ep, en, es = np.full(p.shape, np.nan), np.full(p.shape, np.nan), np.zeros((B, C))
    for b in range(B):
        rows = list(range(int(off[b]), int(off[b + 1])))
        if rev:
            rows.reverse()
        f, d = np.zeros(C), np.zeros(C) if ds is None else np.abs(ds[b])
        more = 2 * U * (len(rows) / 16 + 16)
        for i in range(len(rows) - 1, -1, -1):
            t = rows[i]
            d = d + np.abs(g[t])
            f = f + 2 * U * d
            k = k_of(p[t])
            before = h[rows[i - 1]] if i else (np.zeros(C) if s0 is None else s0[b])
            hb = H[rows[i - 1]] if i else np.abs(before)
            eb = E[rows[i - 1]] if i else np.zeros(C)
            ft = f + more * d
            v = np.abs(n[t] - before)
            en[t] = z[t] * (ft + (k + 4) * U * d)
            ep[t] = z[t] * w[t] * ((2 * k + 8) * U * (np.abs(n[t]) + hb) * d + (eb + U * (np.abs(n[t]) + hb)) * (d + ft) +
                                   v * ft)
            f = w[t] * (f + (k + 4) * U * d)
            d = w[t] * d
        es[b] = f + more * d
    return ep, en, es


def check_scan(T, lengths, C, t, rev=False, states=True, lead=0, tail=0, seed=0, spread=(1.0, -7.0), size=1.0, back=True):
    r = np.random.default_rng(seed + C)
    off = offsets_of(lengths, lead)
    n, B = int(off[-1]) + tail, len(lengths)
    p, c, g, dp, dc = slab(r, n, [C] * 5, t, size=size)
    p += torch.linspace(*spread, C, device="cuda").to(p.dtype)
    P, N, G = host(p), host(c), host(g)
    s0 = r.normal(size=(B, C)).astype(np.float32) if states else None
    s1 = torch.full((B, C), float("nan"), device="cuda") if states else None
    out = torch.full((n, C), float("nan"), dtype=p.dtype, device="cuda")
    saved = torch.full((T.gated_scan_saved(n, C),), float("nan"), device="cuda")
    od = dev(off, "int64")
    T.gated_scan(p, c, od, out, reverse=rev, state_in=dev(s0) if states else None, state_out=s1, saved=saved)
    o, s = Q.gated_scan(P, N, off, rev, s0)
    E, Es, _ = scan_bounds(P, N, off, rev, s0)
    hold(out, o, rounding(t, o) + np.nan_to_num(E), "out")
    if states:
        hold(s1, s, rounding("float32", s) + Es, "state")
    out2 = torch.empty_like(out)
    T.gated_scan(p, c, od, out2, reverse=rev, state_in=dev(s0) if states else None)
    assert torch.equal(out[lead:n - tail], out2[lead:n - tail])
    if not back:
        return
    dp.fill_(float("nan"))
    dc.fill_(float("nan"))
    ds = r.normal(size=(B, C)).astype(np.float32) if states else None
    d0 = torch.full((B, C), float("nan"), device="cuda") if states else None
    T.gated_scan_backward(p, c, od, saved, g, dp, dc, reverse=rev, state_in=dev(s0) if states else None,
                          d_state_out=dev(ds) if states else None, d_state_in=d0)
    rp, rn, rs = Q.gated_scan_backward(P, N, off, G, rev, s0, ds)
    ep, en, es = back_bounds(P, N, off, G, rev, s0, ds)
    hold(dc, rn, rounding(t, rn) + np.nan_to_num(en), "d_cand")
    hold(dp, rp, rounding(t, rp) + np.nan_to_num(ep), "d_gate")
    if states:
        hold(d0, rs, rounding("float32", rs) + es, "d_state")


SHORT = [0, 1, 2, 7, 8, 9, 15, 16, 17, 0, 0, 31, 32, 33, 63, 64, 65, 20, 1, 0]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("C", [8, 24, 64, 72, 192, 264])
def test_scan_short(T, t, rev, C):
    check_scan(T, SHORT, C, t, rev, states=True)
    check_scan(T, SHORT, C, t, rev, states=False, lead=5, tail=9, seed=1)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lengths", [[1], [128], [127, 0, 129], [1000, 0, 3, 513], [5000], [2, 9000, 1], [4095, 1], [4097]])
def test_scan_long(T, t, rev, lengths):
    check_scan(T, lengths, 72, t, rev, states=True)
    check_scan(T, lengths, 16, t, rev, states=False, lead=130, tail=300, seed=2)


@pytest.mark.parametrize("t", TYPES)
def test_scan_many_tracks(T, t):
    r = np.random.default_rng(3)
    check_scan(T, r.integers(8, 21, 700), 40, t, states=False)
    check_scan(T, r.integers(0, 3, 3000), 8, t, True, states=True)
    check_scan(T, [0] * 500, 8, t, True, states=True)


def scan_on_gpu(p, n, g, off, rev):
    """The definition in 64 bits, a row at a time on the GPU: h, dp, dn and their bounds as above."""
    z, w = torch.sigmoid(p.double()), torch.sigmoid(-p.double())
    N, G = n.double(), g.double()
    k = 2 * p.double().abs().clamp(max=100.0) + 10
    h, E, H, before, Eb, Hb = (torch.zeros_like(N) for _ in range(6))
    dp, dn, ep, en = (torch.zeros_like(N) for _ in range(4))
    for b in range(len(off) - 1):
        rows = range(off[b + 1] - 1, off[b] - 1, -1) if rev else range(off[b], off[b + 1])
        x, e, a = (torch.zeros_like(N[0]) for _ in range(3))
        for t in rows:
            before[t], Eb[t], Hb[t] = x, e, a
            e = w[t] * e + (k[t] + 6) * U * (w[t] * a + z[t] * N[t].abs())
            x, a = w[t] * x + z[t] * N[t], w[t] * a + z[t] * N[t].abs()
            h[t], E[t], H[t] = x, e, a
        more = 2 * U * (len(rows) / 16 + 16)
        d, da, f = (torch.zeros_like(N[0]) for _ in range(3))
        for t in reversed(rows):
            d, da = d + G[t], da + G[t].abs()
            f = f + 2 * U * da
            ft = f + more * da
            size = N[t].abs() + Hb[t]
            dn[t], dp[t] = z[t] * d, z[t] * w[t] * (N[t] - before[t]) * d
            en[t] = z[t] * (ft + (k[t] + 4) * U * da)
            ep[t] = z[t] * w[t] * ((2 * k[t] + 8) * U * size * da + (Eb[t] + U * size) * (da + ft) +
                                   (N[t] - before[t]).abs() * ft)
            f = w[t] * (f + (k[t] + 4) * U * da)
            d, da = w[t] * d, w[t] * da
        E[off[b]:off[b + 1]] += more * H[off[b]:off[b + 1]]
    return h, dp, dn, E, ep, en


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lead", [0, 1, 3, 31, 33, 127])
def test_scan_whose_first_rows_are_of_no_sequence(T, t, rev, lead):
    """A first window of fewer rows goes on into the next one of the same warp: enough windows that a warp has
    several."""
    C, n = 1024, 9000
    x = torch.randn((n, 2 * C), generator=torch.Generator(device="cuda").manual_seed(lead), device="cuda")
    x[:, :C] -= 3
    x = x.to(getattr(torch, t))
    p, c = x[:, :C], x[:, C:]
    out, whole = torch.empty((n, C), dtype=x.dtype, device="cuda"), torch.empty((n, C), dtype=x.dtype, device="cuda")
    rows = slice(lead, n - lead)
    T.gated_scan(p, c, dev([lead, n - lead], "int64"), out, reverse=rev)
    T.gated_scan(p[rows], c[rows], dev([0, n - 2 * lead], "int64"), whole[rows], reverse=rev)
    # the same sequence cut into other windows: both are within a rounding of the type and
    # 2 (2 |p| + 16) u of the exact state a row it remembers (|p| up to 8, about 20 rows, states below 4)
    tol = 2 * half_step(t) * whole[rows].double().abs() + 2 * 32 * U * 20 * 4
    assert bool(((out[rows].double() - whole[rows].double()).abs() <= tol).all())


@pytest.mark.parametrize("rev", [False, True])
def test_scan_of_many_channels_and_many_windows_a_warp(T, rev):
    """Long sequences of 2,048 channels: every warp of the sums has eight windows."""
    C, off = 2048, [3, 3000, 3001, 11203, 14000]
    n = off[-1] + 5
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((n, 3 * C), generator=gen, device="cuda")
    x[:, :C] += torch.linspace(1.0, -7.0, C, device="cuda")
    x = x.to(torch.bfloat16)
    p, c, g = x[:, :C], x[:, C:2 * C], x[:, 2 * C:]
    out, dp, dn = (torch.empty((n, C), dtype=x.dtype, device="cuda") for _ in range(3))
    saved = torch.empty(T.gated_scan_saved(n, C), device="cuda")
    T.gated_scan(p, c, dev(off, "int64"), out, reverse=rev, saved=saved)
    T.gated_scan_backward(p, c, dev(off, "int64"), saved, g, dp, dn, reverse=rev)
    ref = scan_on_gpu(p, c, g, off, rev)
    rows, e = slice(off[0], off[-1]), half_step("bfloat16")
    for got, want, tol in zip((out, dp, dn), ref[:3], ref[3:]):
        off_by = (got.double() - want).abs() - e * want.abs() - tol
        assert bool((off_by[rows] <= 0).all()), float(off_by[rows].max())


def test_rows_far_beyond_32_bits(T):
    """Arrays of more than 2^32 elements: the last rows of each operator."""
    n, C = 1060000, 2048
    x = torch.zeros((n, 2 * C), dtype=torch.bfloat16, device="cuda")       # 4.3e9 elements
    last = torch.randn((300, 2 * C), device="cuda").to(torch.bfloat16)
    x[-300:] = last
    off = [0, n - 300, n - 280, n]
    out = torch.empty((n, C), dtype=x.dtype, device="cuda")
    small = torch.empty((300, C), dtype=x.dtype, device="cuda")
    T.gated_scan(x[:, :C], x[:, C:], dev(off, "int64"), out)
    T.gated_scan(last[:, :C], last[:, C:], dev([0, 20, 300], "int64"), small)
    z = torch.sigmoid(last[:, :C].double())
    h = torch.zeros(C, dtype=torch.float64, device="cuda")
    for t in range(300):
        h = (torch.zeros_like(h) if t in (0, 20) else h) * (1 - z[t]) + z[t] * last[t, C:].double()
        for got in (out[n - 300 + t], small[t]):
            assert bool(((got.double() - h).abs() <= half_step("bfloat16") * h.abs() + 2.0 ** -16).all())    # (values of a few units)
    T.add_norm(x, x)
    T.add_norm(last, last)
    assert torch.equal(x[-300:], last)
    del out
    w = torch.randn((72, 2 * C), device="cuda").to(torch.bfloat16)
    y, ys = torch.empty((n, 72), dtype=x.dtype, device="cuda"), torch.empty((300, 72), dtype=x.dtype, device="cuda")
    T.product(x, w, y)
    ref = last.double() @ w.double().T
    T.product(last, w, ys)
    for got in (y[-300:], ys):
        tol = half_step("bfloat16") * ref.abs() + (2 * 2 * C + 8) * U * (last.double().abs() @ w.double().abs().T)
        assert bool(((got.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("t", TYPES)
def test_scan_that_hardly_forgets_and_that_forgets_all(T, t):
    """Gates of 2^-14, where the parts of a sequence all count, and of nearly one."""
    check_scan(T, [6000, 500], 16, t, spread=(-9.7, -9.0), size=0.1)
    check_scan(T, [6000, 500], 16, t, True, spread=(9.0, 60.0), seed=5)
    check_scan(T, [700], 16, t, spread=(-80.0, -60.0), seed=6)


def test_scan_of_gates_at_the_ends(T):
    """Infinite gates: all of the candidate, or none; they pass no gradient of their own."""
    inf = float("inf")
    p = torch.tensor([[inf], [-inf], [inf], [0.0], [-inf]], device="cuda").repeat(1, 8)
    n = torch.arange(1.0, 6.0, device="cuda")[:, None].repeat(1, 8)
    out, saved = torch.empty_like(n), torch.empty(T.gated_scan_saved(5, 8), device="cuda")
    off = dev([0, 5], "int64")
    T.gated_scan(p, n, off, out, saved=saved)
    assert out[:, 0].tolist() == [1.0, 1.0, 3.0, 3.5, 3.5]
    dp, dn = torch.empty_like(n), torch.empty_like(n)
    T.gated_scan_backward(p, n, off, saved, torch.ones_like(n), dp, dn)
    assert dn[:, 0].tolist() == [2.0, 0.0, 2.0, 1.0, 0.0] and dp[:, 0].tolist() == [0.0, 0.0, 0.0, 0.5, 0.0]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("length", [40, 1300, 9000])
@pytest.mark.parametrize("rev", [False, True])
def test_scan_keeps_what_is_not_finite_to_its_sequence(T, t, length, rev):
    r = np.random.default_rng(5)
    off = np.array([0, 20, 20 + length, 40 + length], np.int64)
    n = int(off[-1])
    p, c, g = slab(r, n, [16] * 3, t)
    p[25, 3], c[26, 4], c[27, 5], g[28, 6] = float("nan"), float("nan"), float("inf"), float("nan")
    out, dp, dn = (torch.empty((n, 16), dtype=p.dtype, device="cuda") for _ in range(3))
    s1, d0 = torch.empty((3, 16), device="cuda"), torch.empty((3, 16), device="cuda")
    saved = torch.empty(T.gated_scan_saved(n, 16), device="cuda")
    T.gated_scan(p, c, dev(off, "int64"), out, reverse=rev, state_out=s1, saved=saved)
    T.gated_scan_backward(p, c, dev(off, "int64"), saved, g, dp, dn, reverse=rev, d_state_in=d0)
    others = [i for i in range(16) if i not in (3, 4, 5, 6)]
    for x in (out, dp, dn):
        ok = torch.isfinite(x).cpu()
        assert ok[:20].all() and ok[20 + length:].all() and ok[:, others].all()
    assert torch.isnan(out[25, 3]) and torch.isnan(out[26, 4]) and not torch.isfinite(out[27, 5]) and torch.isnan(dn[28, 6])
    for x in (s1, d0):
        assert torch.isfinite(x[[0, 2]]).all() and torch.isfinite(x[1, others]).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rev", [False, True])
def test_scan_states_in_place_and_the_same_each_time(T, t, rev):
    """state_out may be state_in, d_state_in d_state_out; and nothing depends on the order in which
    the parts of the rows run."""
    n, C = 60000, 136
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((n, 3 * C), generator=g, device="cuda")
    x[:, :C] -= 6
    x = x.to(getattr(torch, t))
    p, c, do = x[:, :C], x[:, C:2 * C], x[:, 2 * C:]
    off = dev([0, 600, n - 700, n], "int64")
    s0 = 10 * torch.randn((3, C), generator=g, device="cuda")
    ws = torch.empty(T.gated_scan_workspace(x.dtype, n, 3, C), dtype=torch.uint8, device="cuda")
    ws.random_(0, 256, generator=g)
    got = []
    for i in range(6):
        out, dp, dn = (torch.empty((n, C), dtype=x.dtype, device="cuda") for _ in range(3))
        saved = torch.empty(T.gated_scan_saved(n, C), device="cuda")
        s1 = s0.clone() if i % 2 else torch.empty_like(s0)
        T.gated_scan(p, c, off, out, reverse=rev, state_in=s1 if i % 2 else s0, state_out=s1, saved=saved, workspace=ws)
        d0 = s0.clone() if i % 2 else torch.empty_like(s0)
        T.gated_scan_backward(p, c, off, saved, do, dp, dn, reverse=rev, state_in=s0, d_state_out=d0 if i % 2 else s0,
                              d_state_in=d0, workspace=ws)
        got.append((out, s1, dp, dn, d0))
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("t", TYPES)
def test_scan_in_parts(T, t):
    """A sequence in three calls, its state in one array, and back again."""
    r = np.random.default_rng(6)
    C, n = 24, 700
    p, c, g = slab(r, n, [C] * 3, t)
    parts, dp, dn = (torch.empty((n, C), dtype=p.dtype, device="cuda") for _ in range(3))
    s, first, saved = torch.zeros((1, C), device="cuda"), [], []
    cuts = ((0, 100), (100, 101), (101, n))
    for lo, hi in cuts:
        first.append(s.clone())
        saved.append(torch.empty(T.gated_scan_saved(hi - lo, C), device="cuda"))
        T.gated_scan(p[lo:hi], c[lo:hi], dev([0, hi - lo], "int64"), parts[lo:hi], state_in=s, state_out=s, saved=saved[-1])
    d = torch.zeros((1, C), device="cuda")
    for i in (2, 1, 0):
        lo, hi = cuts[i]
        T.gated_scan_backward(p[lo:hi], c[lo:hi], dev([0, hi - lo], "int64"), saved[i], g[lo:hi], dp[lo:hi], dn[lo:hi],
                              state_in=first[i], d_state_out=d, d_state_in=d)
    args = host(p), host(c), [0, n]
    o, so = Q.gated_scan(*args)
    E, Es, _ = scan_bounds(*args, False, None)
    hold(parts, o, rounding(t, o) + E)
    hold(s, so, rounding("float32", so) + Es)
    rp, rn, rs = Q.gated_scan_backward(*args, host(g))
    ep, en, es = back_bounds(*args, host(g), False, None, None)
    hold(dn, rn, rounding(t, rn) + en)
    hold(dp, rp, rounding(t, rp) + ep)
    hold(d, rs, rounding("float32", rs) + es)


def test_scan_of_nothing(T):
    x = torch.zeros((0, 16), device="cuda")
    s = torch.arange(48.0, device="cuda").reshape(3, 16)
    s1 = torch.empty_like(s)
    T.gated_scan(x, x, dev([0, 0, 0, 0], "int64"), x, state_in=s, state_out=s1, saved=x.flatten())
    assert torch.equal(s, s1)
    d0 = torch.empty_like(s)
    T.gated_scan_backward(x, x, dev([0, 0, 0, 0], "int64"), torch.empty(4, device="cuda")[:0], x, x, x, d_state_out=s,
                          d_state_in=d0)
    assert torch.equal(s, d0)
    T.gated_scan(x, x, dev([0, 0, 0, 0], "int64"), x, state_out=s1)
    assert bool((s1 == 0).all())
    T.gated_scan(x, x, dev([0], "int64"), x)


# ---------------------------------------------------------------- a single row

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,C", [(1, 8), (5, 24), (97, 192), (700, 1032), (3, 2048)])
@pytest.mark.parametrize("slots", [False, True])
def test_step(T, t, B, C, slots):
    r = np.random.default_rng(B + C)
    p, c = slab(r, B, [C, C], t, size=3.0)
    ns = B + 5
    s0 = dev(r.normal(size=(ns, C)))
    s1 = torch.full_like(s0, 7.0)
    out = torch.empty((B, C), dtype=p.dtype, device="cuda")
    at = r.permutation(ns)[:B] if slots else np.arange(B)
    T.gated_scan_step(p, c, s0, s1, out, slots=dev(at, "int32") if slots else None)
    P, N, S = host(p), host(c), host(s0)[at]
    z, w = Q.logistic(P), Q.logistic(-P)
    ref = S + z * (N - S)
    tol = (k_of(P) + 6) * U * (w * np.abs(S) + z * np.abs(N))
    hold(out, ref, rounding(t, ref) + tol)
    atd = torch.from_numpy(at).cuda()
    hold(s1[atd], ref, rounding("float32", ref) + tol)
    others = np.setdiff1d(np.arange(ns), at)
    assert bool((s1[torch.from_numpy(others).cuda()] == 7.0).all())
    T.gated_scan_step(p, c, s0, s0, out, slots=dev(at, "int32") if slots else None)
    assert torch.equal(s0[atd], s1[atd])


def test_step_of_a_padded_batch(T):
    r = np.random.default_rng(1)
    p, c = slab(r, 6, [40, 40], "bfloat16")
    s = dev(r.normal(size=(4, 40)))
    before = s.clone()
    out = torch.zeros((6, 40), dtype=p.dtype, device="cuda")
    T.gated_scan_step(p, c, s, s, out, slots=torch.tensor([2, -1, 4, 0, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32,
                                                          device="cuda"))
    assert torch.isnan(out[[1, 2, 4, 5]]).all() and torch.isfinite(out[[0, 3]]).all()
    assert torch.equal(s[[1, 3]], before[[1, 3]]) and not torch.equal(s[[0, 2]], before[[0, 2]])


@pytest.mark.parametrize("t", TYPES)
def test_steps_are_the_scan(T, t):
    r = np.random.default_rng(2)
    B, C, n = 7, 48, 30
    p, c = slab(r, B * n, [C, C], t)
    off = dev(np.arange(B + 1) * n, "int64")
    out, s1 = torch.empty((B * n, C), dtype=p.dtype, device="cuda"), torch.empty((B, C), device="cuda")
    T.gated_scan(p, c, off, out, state_out=s1)
    s, rows = torch.zeros((B, C), device="cuda"), torch.empty((B, C), dtype=p.dtype, device="cuda")
    args = host(p), host(c), np.arange(B + 1) * n
    E, Es, _ = scan_bounds(*args, False, None)
    o, so = Q.gated_scan(*args)
    for i in range(n):
        T.gated_scan_step(p[i::n], c[i::n], s, s, rows)
        hold(rows, o[i::n], rounding(t, o[i::n]) + E[i::n])
    hold(s, so, rounding("float32", so) + Es)


# ---------------------------------------------------------------- norm

def check_norm(T, n, C, t, delta, gain, total, eight, size=1.0, seed=0, eps=1e-5):
    r = np.random.default_rng(n + C + seed)
    x, d = slab(r, n, [C, C], t, size=size)
    x *= dev(0.2 + 2 * np.abs(r.normal(size=C)), t)
    g = dev(1 + 0.3 * r.normal(size=C)) if gain else None
    out = torch.empty((n, C), dtype=torch.float8_e4m3fn if eight else x.dtype, device="cuda")
    sums = torch.full((n, C), 7.0, dtype=x.dtype, device="cuda") if total else None
    scales = torch.empty(n, device="cuda") if eight else None
    X, D, G = host(x), host(d) if delta else None, host(g) if gain else None
    T.add_norm(x, out, delta=d if delta else None, sum_out=sums, gain=g, eps=eps, scales=scales)
    s, y = Q.add_norm(X, D, G, eps)
    size = np.abs(X) + (np.abs(D) if delta else 0.0)
    lost = U * size * (np.abs(y) / np.maximum(np.abs(s), 1e-300) if delta else 0.0)
    # the row's norm from rounded sums: u of the mean of |x| + |delta| against the sum's
    rel = (C / 32 + 16) * U + (U * np.sqrt((size ** 2).mean(-1) / (s ** 2).mean(-1))[:, None] if delta else 0.0)
    tol = rel * np.abs(y) + np.where(s == 0, U * size / np.sqrt((s ** 2).mean(-1, keepdims=True) + eps), lost)
    if total:
        hold(sums, s, rounding(t, s) + U * size, "sum")
    if not eight:
        hold(out, y, rounding(t, y) + tol, "out")
        return
    most = np.maximum(np.abs(y).max(-1) / 448.0, 2.0 ** -100)
    hold(scales, most, (np.max(tol, -1) / 448.0) + 2 * U * most, "scales")
    q = y / host(scales)[:, None]
    near = tol / host(scales)[:, None] + 2 * U * np.abs(q)
    hold(out, np.clip(q, -448, 448), np.maximum(2.0 ** -4 * np.abs(q), 2.0 ** -10) + near, "out")
    # and no value further than its own scale says from the nearest one: at most two steps either side of a border
    lo, hi = Q.e4m3(np.clip(q - near, -448, 448)), Q.e4m3(np.clip(q + near, -448, 448))
    o = host(out)
    assert np.all((o >= lo) & (o <= hi))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,C", [(1, 16), (3, 48), (33, 128), (700, 192), (2600, 256), (65, 1024), (40, 2064), (9, 4096),
                                 (5, 16384), (150, 272), (31, 528), (20, 8208)])
@pytest.mark.parametrize("eight", [False, True])
def test_add_norm(T, t, n, C, eight):
    check_norm(T, n, C, t, True, True, True, eight)
    check_norm(T, n, C, t, False, False, False, eight, seed=1)
    check_norm(T, n, C, t, True, False, False, eight, size=30.0, seed=2)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [8, 24, 200, 1000, 2056, 16376])
def test_add_norm_of_widths_that_16_does_not_divide(T, t, C):
    check_norm(T, 77, C, t, True, True, True, False)
    check_norm(T, 6, C, t, False, True, True, False, seed=3)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [64, 2048])
def test_add_norm_in_place(T, t, C):
    r = np.random.default_rng(1)
    x, d = slab(r, 50, [C, C], t)
    out, s = torch.empty((50, C), dtype=x.dtype, device="cuda"), torch.empty((50, C), dtype=x.dtype, device="cuda")
    T.add_norm(x, out, delta=d, sum_out=s)
    a, b = x.clone(), d.clone()
    T.add_norm(a, b, delta=b, sum_out=a)
    assert torch.equal(a, s) and torch.equal(b, out)
    a, b = x.clone(), d.clone()
    T.add_norm(a, a, delta=b, sum_out=b)
    assert torch.equal(b, s) and torch.equal(a, out)


def test_add_norm_of_zeros_and_of_rows_that_are_not_finite(T):
    x = torch.zeros((5, 32), device="cuda")
    x[1, 3], x[2, 4] = float("nan"), float("inf")
    x[3] = 1e-30
    x[4] = 2.0
    out, scales = torch.empty((5, 32), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(5, device="cuda")
    T.add_norm(x, out, scales=scales)
    y = out.float()
    assert bool((y[0] == 0).all()) and scales[0].item() == 2.0 ** -100
    assert torch.isfinite(y[[0, 3, 4]]).all() and bool((y[[3, 4]] == 448).all())
    z = torch.empty_like(x)
    T.add_norm(x, z)
    assert torch.isfinite(z[[0, 3, 4]]).all() and torch.isnan(z[1]).all() and torch.isnan(z[2, 4])
    # a row's largest sum of squares: fp32's range left, as documented, gives zeros
    big = torch.full((1, 32), 1e30, device="cuda")
    T.add_norm(big, z[:1])
    assert bool((z[0] == 0).all())


# ---------------------------------------------------------------- product

ACTS = ["none", "relu", "silu", "gelu"]


def check_product(T, n, K, M, t, act="none", bias=True, gate=False, residual=False, eight=False, seed=0, size=1.0,
                  in_place=False):
    r = np.random.default_rng(n + 3 * K + 7 * M + seed)
    if eight:
        x = dev(r.normal(size=(n, K + 16)) * 100, "float8_e4m3fn")[:, :K]
        w = dev(r.normal(size=(M, K + 32)) * 100, "float8_e4m3fn")[:, 16:K + 16]
        xs, ws = dev(size * 0.01 * (0.5 + r.random(n))), dev(0.01 / np.sqrt(K) * (0.5 + r.random(M)))
        X, W = host(x) * host(xs)[:, None], host(w) * host(ws)[:, None]
    else:
        x = slab(r, n, [K], t, size=size)[0]
        w = slab(r, M, [K], t, size=1 / np.sqrt(K))[0]
        xs = ws = None
        X, W = host(x), host(w)
    b = dev(r.normal(size=M)) if bias else None
    g, res, out = slab(r, n, [M, M, M], t)
    g, res = g if gate else None, res if residual else None
    R = host(res) if residual else None
    if in_place:
        out = res
    T.product(x, w, out, bias=b, activation=act, gate=g, residual=res, x_scales=xs, weight_scales=ws)
    B = host(b) if bias else None
    y = Q.product(X, W, B)
    S = np.abs(X) @ np.abs(W).T + (np.abs(B) if bias else 0.0)
    before = (2 * K + 8) * U * S
    v = Q.product(X, W, B, act)
    tol = before * (1.13 if act != "none" else 1.0) + 16 * U * np.abs(v) + (4 * y * y * U * np.abs(v) if act == "gelu" else 0.0)
    if act == "gelu":     # below what fp32 holds: erfc's smallest normal value times |y|
        tol = tol + 2.0 ** -126 * np.abs(y)
    if act == "silu":
        tol = tol + (2 * np.minimum(np.abs(y), 100.0)) * U * np.abs(v) + 2.0 ** -126 * np.abs(y)
    if gate:
        Gt = host(g)
        sg = Q.logistic(Gt)
        tol, v = tol * sg + (k_of(Gt) + 2) * U * np.abs(v) * sg, v * sg
    if residual:
        v = v + R
        tol = tol + 2 * U * (np.abs(v) + np.abs(R))
    hold(out, v, rounding(t, v) + tol, f"{n} {K} {M} {act}")
    return out


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,K,M", [(1, 8, 8), (2, 64, 64), (7, 4096, 256), (8, 200, 40), (9, 264, 1032), (16, 1000, 24),
                                   (17, 128, 128), (33, 72, 520), (64, 512, 192), (65, 48, 264), (127, 256, 128),
                                   (128, 128, 256), (129, 136, 200), (300, 512, 512), (1000, 24, 72), (513, 264, 1000),
                                   (2049, 128, 64), (700, 1024, 640)])
def test_product(T, t, n, K, M):
    check_product(T, n, K, M, t)
    check_product(T, n, K, M, t, "silu", gate=True, residual=True, seed=1)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,K,M", [(1, 16, 8), (7, 4096, 256), (12, 528, 40), (17, 128, 128), (64, 512, 200), (130, 48, 264),
                                   (500, 256, 136), (300, 1040, 512), (2100, 272, 64)])
def test_product_of_8_bits(T, t, n, K, M):
    check_product(T, n, K, M, t, eight=True)
    check_product(T, n, K, M, t, "gelu", gate=True, residual=True, eight=True, seed=1)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("residual", [False, True])
def test_product_epilogues(T, t, act, gate, residual):
    for n in (5, 40, 333):
        check_product(T, n, 64, 136, t, act, bias=False, gate=gate, residual=residual, size=3.0)
        check_product(T, n, 64, 136, t, act, gate=gate, residual=residual, in_place=residual, size=3.0)


@pytest.mark.parametrize("t", TYPES)
def test_product_of_many_rows(T, t):
    check_product(T, 40001, 64, 72, t, gate=True, residual=True, in_place=True)
    check_product(T, 20000, 40, 8, t, "relu")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,K,M,eight", [(17, 512, 8, False), (100, 4096, 72, False), (70, 2048, 24, False), (200, 1032, 264, False),
                                         (90, 4096, 200, True), (65, 1040, 16, True), (128, 2048, 520, True)])
def test_product_of_few_tiles(T, t, n, K, M, eight):
    """A long K for few outputs: parts of K side by side."""
    check_product(T, n, K, M, t, eight=eight)
    check_product(T, n, K, M, t, "gelu", gate=True, residual=True, eight=eight, in_place=True, seed=1)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n,K,M,eight", [(16400, 64, 136, False), (16385, 200, 256, False), (9001, 96, 264, False),
                                         (8200, 128, 520, False), (16385, 272, 144, True), (8300, 64, 520, True)])
def test_product_of_wide_tiles(T, t, n, K, M, eight):
    """Enough rows for tiles of 256 by pairs of CTAs: outputs of one tile and of several, rows and outputs that
    end inside a tile."""
    check_product(T, n, K, M, t, "relu", eight=eight)
    check_product(T, n, K, M, t, "silu", gate=True, residual=True, eight=eight, in_place=True, seed=1)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("n", [3, 60, 400])
def test_product_keeps_a_row_that_is_not_finite_to_itself(T, t, n):
    r = np.random.default_rng(4)
    x = dev(r.normal(size=(n, 72)), t)
    w = dev(r.normal(size=(136, 72)), t)
    x[1, 5] = float("nan")
    x[2, 6] = float("inf")
    out = torch.empty((n, 136), dtype=x.dtype, device="cuda")
    T.product(x, w, out)
    ok = torch.isfinite(out)
    keep = [i for i in range(n) if i not in (1, 2)]
    assert ok[keep].all() and torch.isnan(out[1]).all() and not ok[2].any()


@pytest.mark.parametrize("t", TYPES)
def test_product_leaves_what_is_beside_its_rows(T, t):
    """Columns beyond out_dim of a wider array, rows behind the last, stay as they are."""
    for n, K, M in ((5, 64, 40), (200, 64, 136), (130, 200, 264)):
        x, w = torch.randn((n, K), device="cuda").to(getattr(torch, t)), torch.randn((M, K), device="cuda").to(getattr(torch, t))
        wide = torch.full((n + 3, M + 24), 5.0, device="cuda").to(x.dtype)
        T.product(x, w, wide[1:n + 1, 8:M + 8])
        assert bool((wide[:, :8] == 5).all()) and bool((wide[:, M + 8:] == 5).all())
        assert bool((wide[0] == 5).all()) and bool((wide[n + 1:] == 5).all())


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
def test_product_of_long_sums_of_one_sign(T, t):
    """All products positive: an order of adding that loses the same way each time shows here."""
    for n in (4, 300):
        x, w = torch.rand((n, 16384), device="cuda").to(getattr(torch, t)) / 64, torch.rand((64, 16384), device="cuda").to(getattr(torch, t))
        out = torch.empty((n, 64), dtype=x.dtype, device="cuda")
        T.product(x, w, out)
        ref = host(x) @ host(w).T
        # 1,024 steps of 16 channels, each off by 2^-22 of the sum so far: at most 2^-12 in all
        hold(out, ref, rounding(t, ref) + 2.0 ** -12 * ref)


# ---------------------------------------------------------------- streams, graphs, a layer of them

def layer(T, x, w, b, gain, off, H, buf):
    D = x.shape[1]
    T.add_norm(x, buf["y"], gain=gain, eps=1e-5)
    T.product(buf["y"], w["w_in"], buf["u"], bias=b["w_in"])
    u = buf["u"]
    T.gated_scan(u[:, :H], u[:, H:2 * H], off, buf["h"][:, :H])
    T.gated_scan(u[:, 2 * H:3 * H], u[:, 3 * H:4 * H], off, buf["h"][:, H:], reverse=True)
    T.product(buf["h"], w["w_m"], buf["x1"], bias=b["w_m"], gate=u[:, 4 * H:4 * H + D], residual=x)
    T.product(buf["x1"], w["w1"], buf["a"], bias=b["w1"], activation="silu")
    T.product(buf["a"], w["w2"], buf["x2"], bias=b["w2"], residual=buf["x1"])


def layer_inputs(n, D, H, t, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g, device="cuda")
    ty = getattr(torch, t)
    shapes = dict(w_in=(4 * H + D, D), w_m=(D, 2 * H), w1=(H, D), w2=(D, H))
    w = {k: (f(*s) / s[1] ** 0.5).to(ty) for k, s in shapes.items()}
    b = {k: 0.2 * f(s[0]) for k, s in shapes.items()}
    e = lambda *s: torch.empty(s, dtype=ty, device="cuda")
    buf = dict(y=e(n, D), u=e(n, 4 * H + D), h=e(n, 2 * H), x1=e(n, D), a=e(n, H), x2=e(n, D))
    return f(n, D).to(ty), w, b, 1 + 0.1 * f(D), buf


def layer_reference(x, w, b, gain, off, H):
    _, y = Q.add_norm(x, None, gain, 1e-5)
    u = Q.product(y, w["w_in"], b["w_in"])
    hf, _ = Q.gated_scan(u[:, :H], u[:, H:2 * H], off)
    hb, _ = Q.gated_scan(u[:, 2 * H:3 * H], u[:, 3 * H:4 * H], off, True)
    x1 = Q.product(np.concatenate([hf, hb], 1), w["w_m"], b["w_m"], gate=u[:, 4 * H:], residual=x)
    return Q.product(Q.product(x1, w["w1"], b["w1"], "silu"), w["w2"], b["w2"], residual=x1)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("D,H", [(128, 192), (40, 64)])
def test_a_layer_of_them(T, t, D, H):
    """Norm, projection, both scans, merge and MLP as they follow one another.  Each of the six
    intermediate results is rounded to the rows' type once, and what follows is at most about
    threefold as large for it (norms of the matrices about 2, slopes about 1): 6 * 3^2 roundings of
    values up to 8 in 16 bits; fp32 256 times as many for its sums."""
    r = np.random.default_rng(8)
    lengths = np.concatenate([r.integers(0, 30, 40), [500, 3]])
    off = offsets_of(lengths)
    n = int(off[-1])
    x, w, b, gain, buf = layer_inputs(n, D, H, t, 1)
    layer(T, x, w, b, gain, dev(off, "int64"), H, buf)
    ref = layer_reference(host(x), {k: host(v) for k, v in w.items()}, {k: host(v) for k, v in b.items()}, host(gain),
                          off, H)
    hold(buf["x2"], ref, (54 if t != "float32" else 54 * 256) * half_step(t) * 8)


def test_a_layer_captured_and_replayed_beside_another(T):
    """Two graphs of the same layer with workspaces of their own, replayed on two streams at once, on
    inputs that changed since the capture."""
    D, H, off = 64, 96, dev([0, 0, 40, 7000, 7013], "int64")
    sets = [layer_inputs(7013, D, H, "bfloat16", s) for s in (1, 2)]
    graphs = []
    for x, w, b, gain, buf in sets:
        layer(T, x, w, b, gain, off, H, buf)      # the first calls stay outside of a capture
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer(T, x, w, b, gain, off, H, buf)
        graphs.append(g)
    new = [layer_inputs(7013, D, H, "bfloat16", s)[0] for s in (3, 4)]
    for s, x in zip(sets, new):
        s[0].copy_(x)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for x, w, b, gain, buf in sets:
        got = buf["x2"].clone()
        layer(T, x, w, b, gain, off, H, buf)
        assert torch.equal(got, buf["x2"])


def test_another_stream(T):
    s = torch.cuda.Stream()
    x, w, b, gain, buf = layer_inputs(900, 64, 96, "float16", 5)
    off = dev([0, 800, 900], "int64")
    layer(T, x, w, b, gain, off, 96, buf)
    want = buf["x2"].clone()
    for v in buf.values():
        v.zero_()
    s.wait_stream(torch.cuda.current_stream())
    u, H = buf["u"], 96
    T.add_norm(x, buf["y"], gain=gain, eps=1e-5, stream=s)
    T.product(buf["y"], w["w_in"], u, bias=b["w_in"], stream=s)
    T.gated_scan(u[:, :H], u[:, H:2 * H], off, buf["h"][:, :H], stream=s)
    T.gated_scan(u[:, 2 * H:3 * H], u[:, 3 * H:4 * H], off, buf["h"][:, H:], reverse=True, stream=s.cuda_stream)
    T.product(buf["h"], w["w_m"], buf["x1"], bias=b["w_m"], gate=u[:, 4 * H:], residual=x, stream=s)
    T.product(buf["x1"], w["w1"], buf["a"], bias=b["w1"], activation="silu", stream=s)
    T.product(buf["a"], w["w2"], buf["x2"], bias=b["w2"], residual=buf["x1"], stream=s)
    s.synchronize()
    assert torch.equal(buf["x2"], want)


def test_the_binding_refuses(T):
    x = torch.zeros((4, 16), device="cuda")
    h, off = x.half(), dev([0, 4], "int64")
    e8 = torch.zeros((4, 16), dtype=torch.float8_e4m3fn, device="cuda")
    for bad in (lambda: T.gated_scan(x, h, off, x), lambda: T.gated_scan(x, x, off.int(), x),
                lambda: T.gated_scan(x, x, off, x[:, ::2]), lambda: T.gated_scan(x, x, off, x, saved=x),
                lambda: T.gated_scan(x, x, off, x, state_in=torch.zeros((2, 16), device="cuda")),
                lambda: T.add_norm(x, e8), lambda: T.add_norm(x, x, scales=torch.zeros(4, device="cuda")),
                lambda: T.add_norm(x, x, gain=torch.zeros(8, device="cuda")), lambda: T.product(x, x, x),
                lambda: T.product(e8, e8, torch.zeros((4, 4), device="cuda")),
                lambda: T.product(x, x[:, :8], torch.zeros((4, 4), device="cuda")),
                lambda: T.product(x, torch.zeros((16, 16), device="cuda"), x, activation="tanh")):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: T.product(x, x, torch.zeros((4, 4), device="cuda")),     # a width that 8 does not divide
                lambda: T.add_norm(x[:, :12], torch.zeros((4, 12), device="cuda"))):
        with pytest.raises(T.TrackfitError):
            bad()
