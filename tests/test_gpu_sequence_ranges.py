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


@pytest.mark.parametrize("bits", [0x7fffffff, 0x7fc00000, 0x7f800001, -1])
def test_cross_fp32_of_any_nan(T, bits):
    """Whatever its payload, a NaN stays one."""
    r = np.random.default_rng(30)
    for at in range(3):
        x = [dev(r.normal(size=(40, 1, 16))) for _ in range(3)]
        x[at][7, 0, 5:6].view(torch.int32).fill_(bits)
        out = torch.empty_like(x[0])
        T.cross_attention(*x, dev([0, 20, 40], "int64"), dev([0, 20, 40], "int64"), out)
        assert bool(torch.isfinite(out[20:]).all())
        bad = torch.isnan(out[:20, 0]).cpu()
        assert bool(bad[7].all()) if at == 0 else bool(bad.all()) if at == 1 else bool(bad[:, 5].all())
        assert int(bad.sum()) == (16, 320, 20)[at]


# ---------------------------------------------------------------- attention: values next to the largest

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("nq,nk", [(3, 9), (1, 3000), (100, 700)])
def test_cross_of_one_state_of_the_largest_values(T, t, sign, nq, nk):
    """One state of them, whose weight is next to one or next to zero."""
    r = np.random.default_rng(21)
    D = 32
    big = sign * torch.finfo(getattr(torch, t)).max
    q, k, v = (dev(r.normal(size=(m, 1, D)), t) for m in (nq, nk, nk))
    v[nk // 2] = big
    out = torch.empty_like(q)
    for ahead in (30.0, -8.0):
        q[..., 0], k[..., 0], k[nk // 2, :, 0] = 1.0, 0.0, ahead
        T.cross_attention(q, k, v, dev([0, nq], "int64"), dev([0, nk], "int64"), out, scale=1.0)
        args = host(q), host(k)
        ref = Q.cross_attention(*args, host(v), [0, nq], [0, nk], 1.0)
        absv = Q.cross_attention(*args, np.abs(host(v)), [0, nq], [0, nk], 1.0)
        top = np.linalg.norm(args[0], axis=-1).max() * np.linalg.norm(args[1], axis=-1).max()
        hold(out, ref, rounding(t, ref) + absv * (2 * (D + 8) * top * U + (nk + 16) * U + (half_step(t) if t != "float32" else 0)))


def test_cross_of_keys_next_to_the_largest_fp32(T):
    """Scores are finite where the queries are small."""
    D, n = 16, 40
    top = torch.finfo(torch.float32).max
    q = torch.full((5, 1, D), 2.0 ** -125, device="cuda")
    k = torch.zeros((n, 1, D), device="cuda")
    k[:, 0, 0] = top * torch.linspace(-1, 1, n, device="cuda")
    k[3, 0, 1] = -top
    v = dev(np.random.default_rng(22).normal(size=(n, 1, D)))
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev([0, 5], "int64"), dev([0, n], "int64"), out, scale=1.0)
    ref = Q.cross_attention(host(q), host(k), host(v), [0, 5], [0, n], 1.0)
    hold(out, ref, 2 * (D + 8) * 16 * U * np.abs(host(v)).max())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("nq,nk", [(3, 9), (1, 3000), (100, 700)])
def test_cross_of_the_largest_values_alone(T, t, sign, nq, nk):
    """All values are the largest: their average is it, though their sum is none."""
    r = np.random.default_rng(23)
    D = 32
    big = sign * torch.finfo(getattr(torch, t)).max
    q, k = (dev(r.normal(size=(m, 1, D)), t) for m in (nq, nk))
    v = torch.full_like(k, big)
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev([0, nq], "int64"), dev([0, nk], "int64"), out)
    ref = np.full(out.shape, float(big))
    # the weights' errors act on both sums
    hold(out, ref, rounding(t, ref) + np.abs(ref) * (nk + 64) * U + (half_step(t) if t != "float32" else 0) * np.abs(ref))


# ---------------------------------------------------------------- attention: small weights

def weights_tol(t):
    """(relative, absolute against a row's largest) error of a weight as an operand.  fp16: two to the
    13 and up are what the largest weight may be taken as, half of the type's smallest step is 2^-25."""
    return half_step(t) if t != "float32" else 8 * U, 2.0 ** -38 if t == "float16" else 0.0


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("nq", [1, 100])
@pytest.mark.parametrize("gap,n,first", [(12.0, 30011, 0.0), (15.0, 30011, 0.0), (18.0, 30011, 0.0), (20.0, 30011, 0.0),
                                         (17.4, 30011, 1.0), (17.4, 300000, 1.0), (16.0, 600, 0.0)])
def test_cross_of_one_state_far_ahead(T, t, nq, gap, n, first):
    """One state whose score is `gap` above all others', which are equal: their weights are e^-gap each."""
    D = 64
    q = torch.zeros((nq, 1, D), device="cuda")
    q[:, :, 0] = 1
    k = torch.zeros((n, 1, D), device="cuda")
    k[n // 3, 0, 0] = 1
    v = torch.ones((n, 1, D), device="cuda")
    v[n // 3] = first
    q, k, v = (x.to(getattr(torch, t)) for x in (q, k, v))
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev([0, nq], "int64"), dev([0, n], "int64"), out, scale=gap)
    w = (n - 1) * np.exp(-float(np.float32(gap)))
    y = np.full((nq, 1, D), (first + w) / (1 + w))
    rel, least = weights_tol(t)
    # the others' weights: their scores are 0, the first one's is exact; n sums; 64 u for the exponent's product
    tol = rounding(t, y) + (rel + (np.sqrt(n) + 64) * U) * y + least * n
    hold(out, y, tol)


# ---------------------------------------------------------------- linear attention: the whole range, long decays

@pytest.mark.parametrize("t", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [1e33, 1e-33])
@pytest.mark.parametrize("length", [40, 1300])
def test_linear_of_values_at_the_ends_of_fp32(T, t, size, length):
    """Sums of 1e33 are finite, and those of 1e-33 keep their bits."""
    r = np.random.default_rng(20)
    H, K, V = 2, 32, 32
    n = length + 25
    q, k, v = slab(r, [(n, H, K), (n, H, K), (n, H, V)], t)
    k, v = (0.1 * k.abs()).contiguous(), (v.abs() * size).contiguous()
    q = (0.1 * q).contiguous()
    g = dev(-0.9 * np.ones((n, H)))
    off = np.array([0, 25, n])
    out, s1 = torch.empty_like(v), torch.empty((2, H, K, V), device="cuda")
    T.linear_attention(q, k, v, g, dev(off, "int64"), out, state_out=s1)
    args = host(q), host(k), host(v), host(g), off, 1.0, False, None
    o, s = Q.linear_attention(*args)
    to, ts = linear_tol(*args, t, o, s)
    hold(out, o, to, "out")
    hold(s1, s, ts, "state")


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rate,length,others", [(0.001, 16000, 383), (0.003, 2048, 100), (0.0005, 40000, 1)])
def test_linear_of_a_constant_decay_over_a_long_sequence(T, t, rate, length, others):
    """One rate for all rows: the errors of its exponentials are all alike and add up.  (Uncut among
    many sequences of one row; cut with few.)"""
    H, K, V = 1, 8, 16
    n = length + others
    off = np.concatenate([[0], length + np.arange(others + 1)]).astype(np.int64)
    x = torch.ones((n, H, K), device="cuda").to(getattr(torch, t))
    v = torch.ones((n, H, V), device="cuda").to(x.dtype)
    g = torch.full((n, H), -rate, device="cuda")
    out, s1 = torch.empty_like(v), torch.empty((others + 1, H, K, V), device="cuda")
    T.linear_attention(x, x, v, g, dev(off, "int64"), out, scale=0.125, state_out=s1)
    gd = float(np.float32(-rate))
    s = np.ones(others + 1)
    s[0] = np.expm1(gd * length) / np.expm1(gd)
    # a row: its exponential (an ulp, u below 1), a product, a sum, over what is left of all rows
    tol = 3 * U * s[0] + 16 * U
    hold(s1, np.broadcast_to(s[:, None, None, None], s1.shape), tol * s[:, None, None, None])
    y = np.expm1(gd * np.arange(1, length + 1)) / np.expm1(gd)
    y = np.broadcast_to(y[:, None, None], (length, H, V))
    hold(out[:length], y, rounding(t, y) + (3 * U * s[0] + 32 * U + (2 * half_step(t) if t != "float32" else 0)) * y)


@pytest.mark.parametrize("rev", [False, True])
def test_linear_of_a_sequence_longer_than_31_bits_count(T, rev):
    """All rows are ones and a row forgets half: the outputs stand at 16 from the tenth row on."""
    n = 2 ** 31 + 5000
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GB")
    x = torch.ones((n, 1, 8), dtype=torch.bfloat16, device="cuda")
    g = torch.full((n, 1), -float(np.log(2.0)), device="cuda")
    out = torch.zeros_like(x)
    s1 = torch.zeros((1, 1, 8, 8), device="cuda")
    work = torch.empty(T.linear_attention_workspace(n, 1, 1, 8, 8), dtype=torch.uint8, device="cuda")
    T.linear_attention(x, x, x, g, dev([0, n], "int64"), out, reverse=rev, state_out=s1, workspace=work)
    flat = out.view(-1)
    step = 1 << 28
    bad = sum(int((flat[at:at + step] != 16).sum()) for at in range(0, flat.numel(), step))
    del x, g, out, flat, work
    torch.cuda.empty_cache()
    # the first rows, by how much a bf16 can tell 16 from: 16 (1 - 2^-i) rounds to it from i = 9 on
    assert bad <= 9 * 8 and bool(torch.isclose(s1, torch.full_like(s1, 2.0), rtol=1e-5).all())


# ---------------------------------------------------------------- expired waits, asked for by several

def test_an_expired_wait_is_reported_to_every_thread_and_stream_that_asks(T):
    import threading
    torch.cuda.synchronize()
    device = torch.cuda.current_device()
    streams = [torch.cuda.current_stream(), torch.cuda.Stream()]
    x = torch.randn((700, 1, 64), device="cuda").to(torch.bfloat16)
    off, out = dev([0, 700], "int64"), torch.empty_like(x)
    go, asked, seen = threading.Event(), threading.Event(), []

    def other():
        torch.cuda.set_device(device)
        for s in streams:                  # what expired before this test is told to whoever first asks
            T.operator_errors(s)
        seen.append([T.operator_errors(s) for s in streams])
        asked.set()
        go.wait(60)
        seen.append([T.operator_errors(s) for s in streams])
        seen.append([T.operator_errors(s) for s in streams])

    thread = threading.Thread(target=other)
    thread.start()
    assert asked.wait(60) and seen[0] == [T.OK] * 2
    for s in streams:
        T.operator_errors(s)
    assert [T.operator_errors(s) for s in streams] == [T.OK, T.OK]
    T.debug_operator_wait(20_000_000, True)
    try:
        T.cross_attention(x, x, x, off, off, out, stream=streams[0])
        torch.cuda.synchronize()
    finally:
        T.debug_operator_wait()
    go.set()
    thread.join(60)
    assert seen[1:] == [[T.ERR_TIMEOUT] * 2, [T.OK] * 2]
    # what the other thread was told is still told here, for each stream once
    assert [T.operator_errors(s) for s in reversed(streams)] == [T.ERR_TIMEOUT] * 2
    assert [T.operator_errors(s) for s in streams] == [T.OK] * 2


# ---------------------------------------------------------------- linear attention: fp16 values of any size

@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("K,V", [(16, 16), (32, 48), (64, 64), (128, 40)])
@pytest.mark.parametrize("size", [1e-2, 1e-4, 3e-7, 3e4])
def test_linear_states_of_values_of_any_size(T, t, K, V, size):
    """States are fp32 sums of decayed rows, however small these are in their own type."""
    r = np.random.default_rng(26)
    H = 2
    lengths = [0, 1, 2, 15, 16, 17, 20, 33, 700]
    off = np.concatenate([[0], np.cumsum(lengths)])
    n = int(off[-1])
    q, k, v = slab(r, [(n, H, K), (n, H, K), (n, H, V)], t)
    v = (v * size * torch.logspace(-3, 0, V, device="cuda").to(v.dtype)).clamp(-6e4, 6e4)
    g = dev(-0.3 * r.random((n, H)))
    out, s1 = torch.empty_like(v), torch.empty((len(lengths), H, K, V), device="cuda")
    T.linear_attention(q, k, v, g, dev(off, "int64"), out, scale=1e-3 if size > 1 else 1.0, state_out=s1)
    args = host(q), host(k), host(v), host(g), off, 1e-3 if size > 1 else 1.0, False, None
    o, s = Q.linear_attention(*args)
    to, ts = linear_tol(*args, t, o, s)
    # a row of which less than fp32's smallest, 2^-126, is left counts nothing: as many of them as there are
    # rows, with |k| of 6, are below 2^-113
    hold(s1, s, ts + 2.0 ** -113, "state")
    hold(out, o, to, "out")
    T.linear_attention(q, k, v, g, dev(off, "int64"), out, scale=args[5])
    hold(out, o, to, "out without states")


# ---------------------------------------------------------------- operands of 16 bits: two parts

@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("K,V", [(16, 16), (32, 32), (32, 48), (64, 64), (128, 40)])
@pytest.mark.parametrize("states", [False, True])
def test_linear_holds_its_state_and_weights_in_two_parts(T, t, rev, K, V, states):
    """Outputs are off by their own rounding and by e^2 of what is added up, not by e of it."""
    r = np.random.default_rng(27)
    H = 2
    lengths = [1, 15, 16, 17, 20, 33, 64, 900]
    off = np.concatenate([[0], np.cumsum(lengths)])
    n = int(off[-1])
    q, k, v = slab(r, [(n, H, K), (n, H, K), (n, H, V)], t)
    g = dev(-0.5 * r.random((n, H)))
    s0 = dev(r.normal(size=(len(lengths), H, K, V))) if states else None
    out = torch.empty_like(v, memory_format=torch.contiguous_format)
    s1 = torch.empty_like(s0) if states else None
    T.linear_attention(q, k, v, g, dev(off, "int64"), out, scale=0.2, reverse=rev, state_in=s0, state_out=s1)
    args = host(q), host(k), host(v), host(g), off, 0.2, rev, None if s0 is None else host(s0)
    o, s = Q.linear_attention(*args)
    oa, _ = Q.linear_attention(*(np.abs(x) for x in args[:3]), args[3], off, 0.2, rev, None if s0 is None else np.abs(args[7]))
    e, steps = half_step(t), 17 / 0.25 + 64
    # (6 n + K + 16) u as in linear_tol, n the rows that count at a mean decay of 0.25; the state's parts
    # and the weights' each leave e^2
    hold(out, o, rounding(t, o) + ((6 * steps + K + 16) * U + 2 * e * e) * oa, "out")


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("nq,nk,D", [([5, 3, 17], [20, 8, 33], 32), ([1, 2], [3000, 900], 64), ([4, 0, 40], [700, 3, 60], 128),
                                     ([200, 90], [900, 1300], 64), ([200, 90], [900, 1300], 128), ([150], [600], 24)])
def test_cross_holds_its_weights_in_two_parts(T, t, nq, nk, D):
    """Outputs are off by their own rounding and by e^2 of the weighted |v|."""
    r = np.random.default_rng(28)
    qo, ko = np.concatenate([[0], np.cumsum(nq)]), np.concatenate([[0], np.cumsum(nk)])
    q = dev(r.normal(size=(int(qo[-1]), 4, D)), t)
    k, v = (dev(r.normal(size=(int(ko[-1]), 2, D)), t) for _ in range(2))
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), out)
    sc = D ** -0.5
    ref = Q.cross_attention(host(q), host(k), host(v), qo, ko, sc)
    absv = Q.cross_attention(host(q), host(k), np.abs(host(v)), qo, ko, sc)
    top = sc * np.linalg.norm(host(q), axis=-1).max() * np.linalg.norm(host(k), axis=-1).max()
    e, n = half_step(t), max(nk)
    # fp16: the lower part's smallest step, 2^-38 of the largest weight a state, on values up to the largest
    least = n * 2.0 ** -38 * np.abs(host(v)).max() if t == "float16" else 0.0
    hold(out, ref, rounding(t, ref) + absv * (2 * (D + 8) * top * U + (16 + 8 * np.sqrt(n)) * U + 2 * e * e) + least)


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("nq,nk", [(16, 30000), (100, 120000), (2100, 30000), (20000, 30000)])
def test_cross_16_bits_of_values_of_one_sign(T, t, nq, nk):
    """No output is further off than its rounding and its weights'.  The mean of all is that of the
    definition rounded alike (outputs near one gather at few values, so that the rounding by itself
    has a mean): an output that rounds the other way is 2 e off, to either side, and six deviations
    of as many as there are hold it.  What the products cut off does not grow with the states: 256
    steps at most, up to 2^-23 each of a sum that grows as they go."""
    out, ref, top = one_sign(T, t, nq, nk, 64, 25)
    e = half_step(t)
    hold(out, ref, ref * (2 * e + 2 * 72 * top * U + (16 + 8 * np.sqrt(nk / 16)) * U))
    near = torch.from_numpy(ref).to(getattr(torch, t)).double().numpy()
    off = np.mean(out / near - 1)
    assert abs(off) < 12 * e * np.sqrt(np.mean(out != near) / out.size) + 256 * U, off


# ---------------------------------------------------------------- attention: what is put aside

@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("D", [40, 64, 128])
@pytest.mark.parametrize("growth", [-6.0, 3.0, 14.0])
def test_cross_of_scores_that_grow_over_a_long_range(T, t, D, growth):
    """Many heads, so that a range is one part: O is put aside several times, and the maximum that the
    weights are taken against moves in between, or never again."""
    r = np.random.default_rng(31)
    H, nq, nk = 80, 500, [7000, 0, 130, 2048, 2049]
    ko, qo = np.concatenate([[0], np.cumsum(nk)]), np.array([0, 300, 310, 350, 430, nq])
    q, k = dev(0.3 * r.normal(size=(nq, H, D)), t), dev(0.3 * r.normal(size=(ko[-1], H, D)), t)
    v = dev(r.normal(size=(ko[-1], H, D)), t)
    q[..., 0] = 1.0
    for a, n in zip(ko, nk):
        k[a:a + n, :, 0] = torch.linspace(0, growth, max(n, 1), device="cuda")[:n, None].to(k.dtype)
    out = torch.full_like(q, float("nan"))
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), out, scale=1.0)
    e = half_step(t)
    for b, n in enumerate(nk):
        rows, at = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        if n == 0:
            assert bool((out[rows] == 0).all())
            continue
        x = torch.softmax(torch.einsum("qhd,khd->hqk", q[rows].double(), k[at].double()), -1)
        ref = torch.einsum("hqk,khd->qhd", x, v[at].double()).cpu().numpy()
        absv = torch.einsum("hqk,khd->qhd", x, v[at].double().abs()).cpu().numpy()
        top = float(q[rows].double().norm(dim=-1).max() * k[at].double().norm(dim=-1).max())
        # 256 steps of a product's accumulation, up to 2^-23 each of a sum that grows
        tol = rounding(t, ref) + absv * (2 * (D + 8) * top * U + (256 + 8 * np.sqrt(n)) * U + 2 * e * e)
        hold(out[rows], ref, tol + (n * 2.0 ** -38 * 6 if t == "float16" else 0.0), f"sequence {b}")


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
def test_cross_of_long_ranges_keeps_what_is_not_finite_to_its_sequence(T, t):
    r = np.random.default_rng(32)
    H, D, nq, nk = 160, 64, [100, 90, 66], [2500, 3000, 2600]
    qo, ko = np.concatenate([[0], np.cumsum(nq)]), np.concatenate([[0], np.cumsum(nk)])
    q, k, v = (dev(r.normal(size=(m, H, D)), t) for m in (qo[-1], ko[-1], ko[-1]))
    want, out = torch.empty_like(q), torch.empty_like(q)
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), want)
    k[2600, 0, 3] = float("nan")
    v[2700, 1, 3] = float("inf")
    v[5400, 2, 5] = float("nan")
    T.cross_attention(q, k, v, dev(qo, "int64"), dev(ko, "int64"), out)
    same = (out == want).cpu()
    assert same[:100].all() and same[190:].all() and same[100:190, 3:].all()
    ok = torch.isfinite(out[100:190]).cpu()
    assert not ok[:, 0].any() and not ok[:, 1, 3].any() and not ok[:, 2, 5].any()
    assert ok[:, 1, :3].all() and ok[:, 1, 4:].all() and ok[:, 2, :5].all() and ok[:, 2, 6:].all()


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
def test_cross_of_two_widths_at_once(T, t):
    """Kernels that take different parts of tensor memory, on two streams, one call after the other."""
    r = np.random.default_rng(33)
    calls = []
    for D, H in ((64, 24), (128, 12), (128, 24), (40, 12)):
        q, k, v = (dev(r.normal(size=(m, H, D)), t) for m in (900, 4000, 4000))
        off, ko, out = dev([0, 500, 900], "int64"), dev([0, 2500, 4000], "int64"), torch.empty_like(q)
        T.cross_attention(q, k, v, off, ko, out)
        calls.append((q, k, v, off, ko, out, out.clone()))
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(6):
        for s, (q, k, v, off, ko, out, _) in zip(streams, calls):
            T.cross_attention(q, k, v, off, ko, out, stream=s)
    torch.cuda.synchronize()
    assert T.operator_errors() == T.OK
    for *_, out, want in calls:
        assert torch.equal(out, want)


# ---------------------------------------------------------------- fp32: errors that no sum lessens

@pytest.mark.parametrize("D", [16, 64, 96, 128])
@pytest.mark.parametrize("nq,nk", [(40, 350), (1, 900), (300, 40)])
def test_cross_fp32_is_as_near_as_fp32_products(T, D, nq, nk):
    """Scores of a few, each a sum of groups of 16 channels that are off by 2^-22 of their size: weights
    are off by a few u, and 12 u holds their average."""
    r = np.random.default_rng(35)
    H = 3
    q, k, v = (dev(r.normal(size=(m, H, D))) for m in (nq, nk, nk))
    q = 1.5 * q
    out = torch.empty_like(q)
    T.cross_attention(q, k, v, dev([0, nq], "int64"), dev([0, nk], "int64"), out)
    ref = Q.cross_attention(host(q), host(k), host(v), [0, nq], [0, nk], D ** -0.5)
    assert np.linalg.norm(host(out) - ref) < 12 * U * np.linalg.norm(ref)


def test_linear_fp32_over_slow_decays(T):
    """A row's two roundings a value, 0.4 u each as a deviation, over the 700 rows that count, leave 15 u of
    a state's size and of an output's; an error of the decay, which all values share, would add to it."""
    r = np.random.default_rng(34)
    n, H, K = 4000, 3, 32
    q, k, v = (dev(r.normal(size=(n, H, K))) for _ in range(3))
    g = dev(-0.001 * (0.5 + r.random((n, H))) * np.array([1.0, 2.0, 0.7]))
    out, s1 = torch.empty_like(v), torch.empty((1, H, K, K), device="cuda")
    T.linear_attention(q, k, v, g, dev([0, n], "int64"), out, state_out=s1)
    o, s = Q.linear_attention(host(q), host(k), host(v), host(g), [0, n])
    for got, ref in ((out, o), (s1, s)):
        assert np.linalg.norm(host(got) - ref) < 24 * U * np.linalg.norm(ref)
