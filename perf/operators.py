"""What the sequence operators are timed on: norms with rotation, decayed linear
attention over whole sequences and by single tokens, and attention to the states
of an encoder.

All of them read packed sequences, as trackfit.forward_packed does: the rows of all
sequences back to back, and offsets [sequences + 1].  The heads are those that this
repository configures (d_model 128 in 4 heads of 32) and wider ones; the sequences are
tracks of 8 to 20 hits, an event's hits as one long sequence, or both mixed.

Keys of a case
  kind    "norm"    queries and keys normalised per head and rotated, out of a projection
          "linear"  linear attention with a decay a head, whole sequences
          "step"    the same by one token a sequence
          "cross"   attention of packed queries to packed states of other lengths
  type    "bf16" | "fp16" | "fp32", the type of the rows; states are fp32 always
  sequences, shortest, longest   their number and their lengths, uniform in between
  heads, kv_heads, key, value    heads, and the widths of a head's keys and values
  rotated, far                   norm: rotated channels of a head, positions up to far
  states, reverse                linear: states in and out; from the last row to the first
  slots                          step: the states lie in slots of their own order
  queries_from, queries_to       cross: queries a sequence
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BASE = 10000.0         # the rotation's angles are position * BASE ** (-2 i / rotated)
EPS = 1e-6
MOST_BYTES = 2.2e9     # of a drawn case
MOST_FLOPS = 3e11


def _norm(name, type, rows, heads, kv_heads, key, rotated, far):
    return dict(name=name, kind="norm", type=type, rows=rows, heads=heads, kv_heads=kv_heads, key=key,
                rotated=rotated, far=far)


def _linear(name, type, sequences, shortest, longest, heads, key, value, states=False, reverse=False):
    return dict(name=name, kind="linear", type=type, sequences=sequences, shortest=shortest, longest=longest,
                heads=heads, key=key, value=value, states=states, reverse=reverse)


def _step(name, type, sequences, heads, key, value, slots):
    return dict(name=name, kind="step", type=type, sequences=sequences, heads=heads, key=key, value=value,
                slots=slots)


def _cross(name, type, sequences, queries_from, queries_to, shortest, longest, heads, kv_heads, key):
    return dict(name=name, kind="cross", type=type, sequences=sequences, queries_from=queries_from,
                queries_to=queries_to, shortest=shortest, longest=longest, heads=heads, kv_heads=kv_heads, key=key)


def listed():
    return [
        # the hits of one event's tracks between the projection and the attention: latency
        _norm("norm_event_bf16", "bf16", 2600, 4, 4, 32, 32, 64),
        # an offline batch of 100,000 tracks
        _norm("norm_batch_bf16", "bf16", 1310003, 4, 4, 32, 32, 64),
        # fp32 rows of an event-long sequence, shared keys, a part of an odd head rotated, far positions
        _norm("norm_far_fp32", "fp32", 77777, 6, 2, 48, 32, 1 << 20),
        # one event's tracks through an encoder layer, against the hits' order: latency
        _linear("linear_event_fp16", "fp16", 211, 8, 20, 4, 32, 32, reverse=True),
        # an offline batch of tracks
        _linear("linear_tracks_bf16", "bf16", 131072, 8, 20, 4, 32, 32),
        # all hits of four events, each one sequence, with the states to go on from
        _linear("linear_long_bf16", "bf16", 4, 20000, 40000, 8, 64, 64, states=True),
        # fp32 tracks and parts of tracks, none of them longer than 64 hits, some empty, odd widths
        _linear("linear_parts_fp32", "fp32", 20011, 0, 64, 4, 32, 48, states=True),
        # the candidates of one event extended by a hit: latency
        _step("step_event_bf16", "bf16", 97, 4, 32, 32, True),
        # the candidates of many events at a time
        _step("step_batch_fp16", "fp16", 8192, 8, 64, 64, False),
        # the five parameters' queries of each track of a batch, reading the track's hits
        _cross("cross_readout_bf16", "bf16", 131072, 5, 5, 8, 20, 4, 4, 32),
        # single queries against event-long states, shared keys and values
        _cross("cross_single_bf16", "bf16", 61, 1, 2, 1, 16384, 16, 4, 128),
        # the track candidates of an event reading all of its hits
        _cross("cross_event_fp16", "fp16", 1, 4099, 4099, 30011, 30011, 8, 8, 64),
    ]


def draw(rng):
    """One more case of the ranges above: sizes over their logarithm, odd ones among them."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["norm", "linear", "linear", "step", "cross", "cross"])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    heads = rng.choice([1, 2, 4, 6, 8])
    width = rng.choice([16, 24, 32, 40, 64, 64, 96, 128])
    if kind == "norm":
        kv_heads = rng.choice([h for h in (1, 2, 4, 6, 8) if heads % h == 0])
        c = _norm(None, type, log_int(64, 1500000), heads, kv_heads, width, 16 * rng.randint(0, width // 16),
                  rng.choice([64, 1 << 20]))
        size = "rows"
    elif kind == "linear":
        value = width if rng.random() < 0.7 else rng.choice([16, 24, 32, 40, 64, 96, 128])
        if rng.random() < 0.6:
            longest = log_int(4, 64)
            c = _linear(None, type, log_int(64, 131072), rng.randint(0, longest), longest, heads, width, value,
                        rng.random() < 0.3, rng.random() < 0.5)
            size = "sequences"
        else:
            longest = log_int(100, 40000)
            c = _linear(None, type, log_int(1, 16), rng.randint(0, longest), longest, heads, width, value,
                        rng.random() < 0.5, rng.random() < 0.5)
            size = "longest"
    elif kind == "step":
        c = _step(None, type, log_int(16, 16384), heads, width, width, rng.random() < 0.5)
        size = "sequences"
    else:
        kv_heads = rng.choice([h for h in (1, 2, 4, 6, 8) if heads % h == 0])
        p = rng.random()
        if p < 0.4:
            longest, most = log_int(4, 64), rng.randint(1, 24)
            n, size = log_int(64, 131072), "sequences"
        elif p < 0.7:
            longest, most = log_int(256, 16384), rng.randint(1, 4)
            n, size = log_int(1, 64), "longest"
        else:
            longest, most = log_int(256, 30000), log_int(64, 4096)
            n, size = rng.randint(1, 3), "longest"
        c = _cross(None, type, n, rng.randint(1, most), most, rng.randint(0, longest), longest, heads, kv_heads, width)
    del c["name"]
    most_flops = MOST_FLOPS if c["kind"] == "cross" and type != "fp32" else MOST_FLOPS / 8
    while work(c)["bytes"] > MOST_BYTES or work(c)["flops"] > most_flops:
        c[size] = max(1, c[size] * 2 // 3)
        if size == "longest":
            c["shortest"] = min(c["shortest"], c["longest"])
    return c


def _lengths(n, lo, hi, seed=None):
    """The same lengths for every seed, in an order of its own (the rows are as many)."""
    g = torch.Generator()
    g.manual_seed(17)
    lengths = torch.randint(lo, hi + 1, (n,), generator=g, dtype=torch.int64)
    if seed is None:
        return lengths
    g.manual_seed(seed)
    return lengths[torch.randperm(n, generator=g)]


def _offsets(lengths):
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(lengths, 0)])


def _unit(x):
    return x / torch.sqrt(torch.mean(x * x, -1, keepdim=True) + EPS)


def _places(offsets, longest, reverse=False):
    """For sequences padded to `longest`: the row of every place, and whether there is one."""
    t = torch.arange(longest, device=offsets.device)
    n = offsets[1:] - offsets[:-1]
    there = t[None, :] < n[:, None]
    at = offsets[1:, None] - 1 - t[None, :] if reverse else offsets[:-1, None] + t[None, :]
    return torch.where(there, at, 0), there


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = dict(case=case)
    if case["kind"] == "norm":
        N, Hq, Hk, D = case["rows"], case["heads"], case["kv_heads"], case["key"]
        # a projection's output: queries, keys and values of a row side by side
        x = (normal(N, Hq + 2 * Hk, D) * (0.5 + normal(Hq + 2 * Hk, D).abs())).to(t)
        s["q"], s["k"] = x[:, :Hq], x[:, Hq:Hq + Hk]
        s["q_gain"], s["k_gain"] = 1 + 0.2 * normal(D), 1 + 0.2 * normal(D)
        s["positions"] = torch.randint(0, case["far"], (N,), generator=g, device=dev, dtype=torch.int32)
        s["q_out"] = torch.empty((N, Hq, D), dtype=t, device=dev)
        s["k_out"] = torch.empty((N, Hk, D), dtype=t, device=dev)
        return s
    if case["kind"] == "cross":
        nq = _lengths(case["sequences"], case["queries_from"], case["queries_to"], seed + 1)
        nk = _lengths(case["sequences"], case["shortest"], case["longest"], seed)
        s["q_offsets"], s["kv_offsets"] = _offsets(nq).to(dev), _offsets(nk).to(dev)
        s["most_q"], s["most_kv"] = int(nq.max()), int(nk.max())
        Nq, Nk = int(nq.sum()), int(nk.sum())
        D = case["key"]
        s["scale"] = 1.0 / math.sqrt(D)
        s["q"] = (1.5 * _unit(normal(Nq, case["heads"], D))).to(t)
        kv = normal(Nk, 2 * case["kv_heads"], D)
        kv[:, :case["kv_heads"]] = _unit(kv[:, :case["kv_heads"]])
        kv = kv.to(t)
        s["k"], s["v"] = kv[:, :case["kv_heads"]], kv[:, case["kv_heads"]:]
        s["out"] = torch.empty((Nq, case["heads"], D), dtype=t, device=dev)
        return s
    H, K, V = case["heads"], case["key"], case["value"]
    B = case["sequences"]
    if case["kind"] == "linear":
        n = _lengths(B, case["shortest"], case["longest"], seed)
        s["offsets"] = _offsets(n).to(dev)
        s["most"] = int(n.max())
        N = int(n.sum())
    else:
        N = B
    s["scale"] = 1.0 / math.sqrt(K)
    s["q"], s["k"] = _unit(normal(N, H, K)).to(t), _unit(normal(N, H, K)).to(t)
    s["v"] = normal(N, H, V).to(t)
    # a head forgets within about one row, or within about a thousand, and a few rows forget nearly all
    rate = torch.exp2(-torch.linspace(0.0, 10.0, H, device=dev))
    x = -rate * torch.nn.functional.softplus(normal(N, H) + 0.5)
    s["log_decay"] = torch.where(torch.rand((N, H), generator=g, device=dev) < 0.002, -30.0, x)
    s["out"] = torch.empty((N, H, V), dtype=t, device=dev)
    if case["kind"] == "step" or case["states"]:
        s["state_in"] = normal(B, H, K, V)
        s["state_out"] = torch.empty((B, H, K, V), device=dev)
    if case["kind"] == "step":
        s["slots"] = torch.randperm(B, generator=g, device=dev).to(torch.int32) if case["slots"] else None
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "linear": _plain_linear, "step": _plain_step, "cross": _plain_cross}[
        s["case"]["kind"]](s)


def _run_own(s):
    from paper_2609_32479_gb300 import trackfit
    c = s["case"]
    if c["kind"] == "norm":
        trackfit.qk_norm(s["q"], s["k"], s["q_out"], s["k_out"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS,
                         positions=s["positions"], rot_dim=c["rotated"], rot_base=BASE)
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "linear":
        states = dict(state_in=s["state_in"], state_out=s["state_out"]) if c["states"] else {}
        trackfit.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], s["out"], scale=s["scale"],
                                  reverse=c["reverse"], **states)
        return {"out": s["out"], "state": s["state_out"]} if c["states"] else {"out": s["out"]}
    if c["kind"] == "step":
        trackfit.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state_in"], s["state_out"], s["out"],
                                       scale=s["scale"], slots=s["slots"])
        return {"out": s["out"], "state": s["state_out"]}
    trackfit.cross_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["kv_offsets"], s["out"], scale=s["scale"])
    return {"out": s["out"]}


def _plain_norm(s):
    c = s["case"]
    half = c["rotated"] // 2
    i = torch.arange(half, device=s["q"].device, dtype=torch.float64)
    # in 64 bits: a far position's angle is of the order of a million
    angle = s["positions"].to(torch.float64)[:, None, None] * BASE ** (-i / max(half, 1))
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def one(x, gain):
        x = x.float()
        x = x * torch.rsqrt(torch.mean(x * x, -1, keepdim=True) + EPS) * gain
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1)

    s["q_out"].copy_(one(s["q"], s["q_gain"]))
    s["k_out"].copy_(one(s["k"], s["k_gain"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _plain_linear(s):
    """Chunks of rows: within one the decayed products, between them the chunks' states, each chunk's
    from all before it."""
    c = s["case"]
    B, H, K, V = c["sequences"], c["heads"], c["key"], c["value"]
    C = min(128, max(1, s["most"]))
    n = max(1, -(-s["most"] // C))
    if s["q"].shape[0]:
        at, there = _places(s["offsets"], n * C, c["reverse"])

        def chunks(x):   # [B, H, n, C, ...]
            x = torch.where(there[..., None, None], x.float()[at], 0.0)
            return x.view(B, n, C, H, -1).permute(0, 3, 1, 2, 4)

        q, k, v = chunks(s["q"]), chunks(s["k"]), chunks(s["v"])
        # sums of logarithms in 64 bits, only differences of which are used
        g = chunks(s["log_decay"][..., None])[..., 0].double().cumsum(-1)
        i = torch.arange(C, device=g.device)
        w = torch.where(i[:, None] >= i, torch.exp((g[..., :, None] - g[..., None, :]).float()), 0.0)
        o = torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * w, v)
        del w
        u = torch.matmul((k * torch.exp((g[..., -1:] - g).float())[..., None]).transpose(-1, -2), v)
        a = g[..., -1].cumsum(-1)                      # up to the end of each chunk
        before = torch.cat([torch.zeros_like(a[..., :1]), a], -1)
        j = torch.arange(n + 1, device=g.device)
        w = torch.where(j[:, None] > j[:-1], torch.exp((before[..., :, None] - a[..., None, :]).float()), 0.0)
        st = torch.matmul(w, u.reshape(B, H, n, K * V)).view(B, H, n + 1, K, V)
        if c["states"]:
            st = st + torch.exp(before.float())[..., None, None] * s["state_in"][:, :, None]
        o = o + torch.matmul(q * torch.exp(g.float())[..., None], st[:, :, :-1])
        o = (s["scale"] * o).permute(0, 2, 3, 1, 4).reshape(B, n * C, H, V)
        s["out"][at[there]] = o[there].to(s["out"].dtype)
        if c["states"]:
            s["state_out"].copy_(st[:, :, -1])
    elif c["states"]:
        s["state_out"].copy_(s["state_in"])
    return {"out": s["out"], "state": s["state_out"]} if c["states"] else {"out": s["out"]}


def _plain_step(s):
    at = s["slots"].long() if s["slots"] is not None else None
    st = s["state_in"] if at is None else s["state_in"][at]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    st = torch.exp(s["log_decay"])[..., None, None] * st + k[..., :, None] * v[..., None, :]
    s["out"].copy_(s["scale"] * torch.matmul(q[..., None, :], st)[..., 0, :])
    if at is None:
        s["state_out"].copy_(st)
    else:
        s["state_out"][at] = st
    return {"out": s["out"], "state": s["state_out"]}


def _plain_cross(s):
    c = s["case"]
    if s["q"].shape[0] == 0 or s["most_kv"] == 0:
        s["out"].zero_()
        return {"out": s["out"]}
    G = c["heads"] // c["kv_heads"]
    qat, qthere = _places(s["q_offsets"], s["most_q"])
    kat, kthere = _places(s["kv_offsets"], s["most_kv"])
    q = s["q"].float()[qat].permute(0, 2, 1, 3)                                       # [B, H, Q, D]
    k = s["k"].float()[kat].permute(0, 2, 1, 3).repeat_interleave(G, 1)               # [B, H, K, D]
    v = torch.where(kthere[..., None, None], s["v"].float()[kat], 0.0).permute(0, 2, 1, 3).repeat_interleave(G, 1)
    x = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    x = torch.where(kthere[:, None, None], x, -math.inf)
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    n = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / torch.where(n > 0, n, 1.0)
    s["out"].copy_(o.permute(0, 2, 1, 3)[qthere])
    return {"out": s["out"]}


def exact(case, seed):
    """The definitions, row by row, in 64 bits."""
    s = prepare(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "step": _exact_step, "cross": _exact_cross}[case["kind"]](s)


def _exact_norm(s):
    r = s["case"]["rotated"]
    rate = torch.pow(torch.tensor(BASE, dtype=torch.float64, device="cuda"),
                     -torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / max(r, 1))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), rate))

    def one(x, gain):
        x = x.double()
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn[:, None]
        return torch.cat([z.real, z.imag, x[..., r:]], -1)

    return {"q": one(s["q"], s["q_gain"]), "k": one(s["k"], s["k_gain"])}


def _exact_linear(s):
    """S <- exp(g) S + k v^T and o = scale S^T q, a row at a time."""
    c = s["case"]
    off = s["offsets"]
    n = off[1:] - off[:-1]
    st = s["state_in"].double() if c["states"] else torch.zeros(
        (c["sequences"], c["heads"], c["key"], c["value"]), dtype=torch.float64, device="cuda")
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    by_length = torch.argsort(n, descending=True)      # the sequences that reach row t come first
    off, last, length = off[:-1][by_length], off[1:][by_length] - 1, n[by_length].tolist()
    st = st[by_length]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    live = len(length)
    for t in range(s["most"]):
        while live and length[live - 1] <= t:
            live -= 1
        row = last[:live] - t if c["reverse"] else off[:live] + t
        st[:live] *= torch.exp(s["log_decay"][row].double())[..., None, None]
        st[:live] += k[row][..., :, None] * v[row][..., None, :]
        out[row] = s["scale"] * torch.einsum("bhk,bhkv->bhv", q[row], st[:live])
    if not c["states"]:
        return {"out": out}
    state = torch.empty_like(st)
    state[by_length] = st
    return {"out": out, "state": state}


def _exact_step(s):
    B = s["case"]["sequences"]
    at = torch.arange(B, device="cuda") if s["slots"] is None else s["slots"].long()
    st = s["state_in"].double()
    st[at] = torch.exp(s["log_decay"].double())[..., None, None] * st[at] + torch.einsum(
        "bhk,bhv->bhkv", s["k"].double(), s["v"].double())
    return {"out": s["scale"] * torch.einsum("bhk,bhkv->bhv", s["q"].double(), st[at]), "state": st}


def _exact_cross(s):
    """softmax(scale q k^T) v: tracks padded, a few sequences one after the other."""
    c = s["case"]
    G = c["heads"] // c["kv_heads"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    if out.shape[0] == 0 or s["most_kv"] == 0:
        return {"out": out}
    if c["sequences"] <= 64:
        a, b = s["q_offsets"].tolist(), s["kv_offsets"].tolist()
        for i in range(c["sequences"]):
            if b[i + 1] == b[i]:
                continue
            for h in range(c["heads"]):
                k, v = s["k"][b[i]:b[i + 1], h // G].double(), s["v"][b[i]:b[i + 1], h // G].double()
                x = s["scale"] * (s["q"][a[i]:a[i + 1], h].double() @ k.T)
                out[a[i]:a[i + 1], h] = torch.softmax(x, -1) @ v
        return {"out": out}
    qat, qthere = _places(s["q_offsets"], s["most_q"])
    kat, kthere = _places(s["kv_offsets"], s["most_kv"])
    for h in range(c["heads"]):
        x = s["scale"] * torch.einsum("bqd,bkd->bqk", s["q"][:, h][qat].double(), s["k"][:, h // G][kat].double())
        p = torch.exp(x - x.amax(-1, keepdim=True)) * kthere[:, None]
        p = p / p.sum(-1, keepdim=True).clamp_min(1e-300)
        out[:, h] = torch.einsum("bqk,bkd->bqd", p, s["v"][:, h // G][kat].double())[qthere]
    return {"out": out}


def work(case):
    """Each input read once, each output written once.  Operations: a multiply and an add count two."""
    e = 4 if case["type"] == "fp32" else 2
    if case["kind"] == "norm":
        n = case["rows"] * (case["heads"] + case["kv_heads"]) * case["key"]
        return {"bytes": 2 * e * n + 4 * case["rows"] + 8 * case["key"], "flops": 7 * n}
    B = case["sequences"]
    H, K = case["heads"], case["key"]
    if case["kind"] == "step":
        V = case["value"]
        return {"bytes": B * H * (2 * e * (K + V) + 4 + 8 * K * V), "flops": 5 * B * H * K * V}
    n = _lengths(B, case["shortest"], case["longest"])
    N = int(n.sum())
    if case["kind"] == "cross":
        # the queries' order goes with the seed: each sequence counted with the mean number of queries
        nq = int(_lengths(B, case["queries_from"], case["queries_to"]).sum())
        return {"bytes": 2 * e * K * (nq * H + N * case["kv_heads"]) + 16 * (B + 1), "flops": 4 * K * H * nq * N // B}
    V = case["value"]
    # a short sequence's products of queries and keys are fewer than a state's
    flops = H * (4 * K * V * N if case["states"] else int(torch.minimum(4 * K * V * n, n * (n + 1) * (K + V)).sum()))
    return {"bytes": N * H * (2 * e * (K + V) + 4) + 8 * (B + 1) + (8 * B * H * K * V if case["states"] else 0),
            "flops": flops}
