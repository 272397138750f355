"""What the operators of a gated recurrent layer are timed on: the gated scan over packed
sequences (forward, with its gradients, by single rows), the norm with the residual's
addition, and the product with its epilogue.

Sequences stand back to back, as trackfit.forward_packed has them: offsets [sequences + 1].
The widths are those that this repository configures (128 and 256 channels, 192 in the
paper's layers) and wider ones; the sequences are tracks of 8 to 20 hits, an event's hits as
one long sequence, or both mixed.

Keys of a case
  kind      "scan"     h <- h + sigma(p) (n - h) along whole sequences
            "train"    the same, and the gradients of p, n and the first states
            "step"     one row more of each sequence
            "norm"     root-mean-square norm of x + delta
            "product"  residual + act(x W^T + bias) * sigma(gate)
  type      "bf16" | "fp16" | "fp32", the type of the rows; states are fp32 always
  sequences, shortest, longest   their number and their lengths, uniform in between
  channels  of the scan and the norm
  states, reverse   scan, train: states in and out; from the last row to the first
  slots     step: the states lie in slots of their own order
  rows      norm, product
  delta     norm: whether there is one (the sum is an output then)
  eight     norm: the output in e4m3 with a scale a row; product: operands in e4m3 with scales
  inner, outer      product: channels of x and of the output
  act       product: "none" | "relu" | "silu" | "gelu"
  gate, residual    product: whether there is one
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
LARGEST = 448.0             # of e4m3
LEAST_SCALE = 2.0 ** -100   # of a row in 8 bits
MOST_BYTES = 2.4e9          # of a drawn case
MOST_FLOPS = {"bf16": 2.7e11, "fp16": 2.7e11, "fp32": 7e10}


def _scan(name, type, sequences, shortest, longest, channels, states=False, reverse=False, kind="scan"):
    return dict(name=name, kind=kind, type=type, sequences=sequences, shortest=shortest, longest=longest,
                channels=channels, states=states, reverse=reverse)


def _step(name, type, sequences, channels, slots):
    return dict(name=name, kind="step", type=type, sequences=sequences, channels=channels, slots=slots)


def _norm(name, type, rows, channels, delta, eight=False):
    return dict(name=name, kind="norm", type=type, rows=rows, channels=channels, delta=delta, eight=eight)


def _product(name, type, rows, inner, outer, act="none", gate=False, residual=False, eight=False):
    return dict(name=name, kind="product", type=type, rows=rows, inner=inner, outer=outer, act=act, gate=gate,
                residual=residual, eight=eight)


def listed():
    return [
        # one event's tracks through a layer, against the hits' order: latency
        _scan("scan_event_fp16", "fp16", 211, 8, 20, 192, reverse=True),
        # all hits of four events, each one sequence, with the states to go on from
        _scan("scan_long_fp32", "fp32", 4, 20000, 40000, 200, states=True),
        # a training batch of tracks, forward and backward
        _scan("train_tracks_bf16", "bf16", 65536, 8, 20, 192, kind="train"),
        # event-long sequences and empty ones, forward and backward, with the gradients of the first states
        _scan("train_long_bf16", "bf16", 5, 0, 30000, 512, states=True, reverse=True, kind="train"),
        # the candidates of one event extended by a hit: latency
        _step("step_event_bf16", "bf16", 97, 192, True),
        # the candidates of many events at a time
        _step("step_batch_fp16", "fp16", 65536, 1024, False),
        # one event's hits before a layer: latency
        _norm("norm_event_bf16", "bf16", 2600, 128, True),
        # an offline batch's hits before a layer whose products are in 8 bits
        _norm("norm_batch_eight", "bf16", 1835003, 256, True, eight=True),
        # a few candidates through a wide layer: the weights are what is read
        _product("product_single_bf16", "bf16", 7, 4096, 4096, act="silu"),
        # the merge of a layer over an offline batch's hits: gated, onto the residual stream
        _product("product_merge_bf16", "bf16", 1310003, 256, 128, gate=True, residual=True),
        # a wide layer over a few events' hits
        _product("product_wide_fp16", "fp16", 8011, 4096, 4096, act="gelu"),
        # the same in 8 bits, back onto the residual stream
        _product("product_wide_eight", "bf16", 8011, 4096, 4096, residual=True, eight=True),
    ]


def draw(rng):
    """One more case of the ranges above: sizes over their logarithm, odd ones among them."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["scan", "train", "step", "norm", "product", "product"])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    channels = 8 * log_int(1, 256)
    if kind in ("scan", "train"):
        if rng.random() < 0.5:
            longest = log_int(4, 64)
            sequences, size = log_int(64, 131072), "sequences"
        else:
            longest = log_int(100, 40000)
            sequences, size = log_int(1, 64), "longest"
        c = _scan(None, type, sequences, rng.randint(0, longest), longest, channels, rng.random() < 0.5,
                  rng.random() < 0.5, kind)
    elif kind == "step":
        c, size = _step(None, type, log_int(16, 65536), channels, rng.random() < 0.5), "sequences"
    elif kind == "norm":
        eight = rng.random() < 0.4
        c, size = _norm(None, type, log_int(64, 2000000), channels * (2 if eight else 1), rng.random() < 0.7, eight), "rows"
    else:
        eight = rng.random() < 0.25
        c, size = _product(None, type, log_int(1, 2000000), (16 if eight else 8) * log_int(1, 512), 8 * log_int(1, 512),
                           rng.choice(["none", "relu", "silu", "gelu"]), rng.random() < 0.3, rng.random() < 0.4,
                           eight), "rows"
    del c["name"]
    most = MOST_FLOPS["bf16" if c.get("eight") else type]
    while work(c)["bytes"] > MOST_BYTES or work(c)["flops"] > most:
        c[size] = max(1, c[size] * 2 // 3)
        if size == "longest":
            c["shortest"] = min(c["shortest"], c["longest"])
    return c


def _lengths(case, seed=None):
    """The same lengths for every seed, in an order of its own (the rows are as many)."""
    g = torch.Generator()
    g.manual_seed(23)
    n = case["sequences"]
    lengths = torch.randint(case["shortest"], case["longest"] + 1, (n,), generator=g, dtype=torch.int64)
    if seed is None:
        return lengths
    g.manual_seed(seed)
    return lengths[torch.randperm(n, generator=g)]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = dict(case=case)
    if case["kind"] in ("scan", "train", "step"):
        B, C = case["sequences"], case["channels"]
        if case["kind"] == "step":
            N = B
        else:
            n = _lengths(case, seed)
            N = int(n.sum())
            s["most"] = int(n.max())
            s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(n, 0)]).to(dev)
        # gates and candidates side by side, out of a projection: a channel forgets within a row or
        # two, or within about a thousand
        x = normal(N, 2 * C)
        x[:, :C] += torch.linspace(1.0, -7.0, C, device=dev)
        x = x.to(t)
        s["gate"], s["cand"] = x[:, :C], x[:, C:]
        s["out"] = torch.empty((N, C), dtype=t, device=dev)
        if case["kind"] == "step" or case["states"]:
            s["state_in"], s["state_out"] = normal(B, C), torch.empty((B, C), device=dev)
        if case["kind"] == "step":
            s["slots"] = torch.randperm(B, generator=g, device=dev).to(torch.int32) if case["slots"] else None
        if case["kind"] == "train":
            s["d_out"] = normal(N, C).to(t)
            d = torch.empty((N, 2 * C), dtype=t, device=dev)
            s["d_gate"], s["d_cand"] = d[:, :C], d[:, C:]
            if case["states"]:
                s["d_state_out"], s["d_state_in"] = normal(B, C), torch.empty((B, C), device=dev)
        return s
    N = case["rows"]
    if case["kind"] == "norm":
        C = case["channels"]
        # a residual stream whose channels are of different sizes, and a branch's output
        s["x"] = (normal(N, C) * (0.3 + 2.0 * normal(C).abs())).to(t)
        s["delta"] = normal(N, C).to(t) if case["delta"] else None
        s["gain"] = 1 + 0.2 * normal(C)
        s["sum"] = torch.empty((N, C), dtype=t, device=dev) if case["delta"] else None
        s["out"] = torch.empty((N, C), dtype=torch.float8_e4m3fn if case["eight"] else t, device=dev)
        s["scales"] = torch.empty(N, device=dev) if case["eight"] else None
        return s
    K, M = case["inner"], case["outer"]
    if case["eight"]:
        def eight(x):
            scale = (x.abs().amax(-1) / LARGEST).clamp_min(LEAST_SCALE)
            return (x / scale[:, None]).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn), scale
        s["x"], s["x_scales"] = eight(normal(N, K))
        s["weight"], s["weight_scales"] = eight(normal(M, K) / math.sqrt(K))
    else:
        s["x"] = normal(N, K).to(t)
        s["weight"] = (normal(M, K) / math.sqrt(K)).to(t)
    s["bias"] = 0.5 * normal(M)
    s["gate"] = normal(N, M).to(t) if case["gate"] else None
    s["residual"] = normal(N, M).to(t) if case["residual"] else None
    s["out"] = torch.empty((N, M), dtype=t, device=dev)
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"scan": _plain_scan, "train": _plain_train, "step": _plain_step, "norm": _plain_norm,
            "product": _plain_product}[s["case"]["kind"]](s)


def _run_own(s):
    from paper_2609_32479_gb300 import trackfit
    c = s["case"]
    if c["kind"] == "scan":
        trackfit.gated_scan(s["gate"], s["cand"], s["offsets"], s["out"], reverse=c["reverse"],
                            state_in=s.get("state_in"), state_out=s.get("state_out"))
        return {"out": s["out"], "state": s["state_out"]} if c["states"] else {"out": s["out"]}
    if c["kind"] == "train":
        saved = torch.empty(trackfit.gated_scan_saved(s["gate"].shape[0], c["channels"]), device=s["gate"].device)
        trackfit.gated_scan(s["gate"], s["cand"], s["offsets"], s["out"], reverse=c["reverse"],
                            state_in=s.get("state_in"), state_out=s.get("state_out"), saved=saved)
        trackfit.gated_scan_backward(s["gate"], s["cand"], s["offsets"], saved, s["d_out"], s["d_gate"], s["d_cand"],
                                     reverse=c["reverse"], state_in=s.get("state_in"),
                                     d_state_out=s.get("d_state_out"), d_state_in=s.get("d_state_in"))
        return _trained(s)
    if c["kind"] == "step":
        trackfit.gated_scan_step(s["gate"], s["cand"], s["state_in"], s["state_out"], s["out"], slots=s["slots"])
        return {"out": s["out"], "state": s["state_out"]}
    if c["kind"] == "norm":
        trackfit.add_norm(s["x"], s["out"], delta=s["delta"], sum_out=s["sum"], gain=s["gain"], eps=EPS,
                          scales=s["scales"])
        return _normed(s)
    scales = dict(x_scales=s["x_scales"], weight_scales=s["weight_scales"]) if c["eight"] else {}
    trackfit.product(s["x"], s["weight"], s["out"], bias=s["bias"], activation=c["act"], gate=s["gate"],
                     residual=s["residual"], **scales)
    return {"out": s["out"]}


def _trained(s):
    r = {"out": s["out"], "d_gate": s["d_gate"], "d_cand": s["d_cand"]}
    if s["case"]["states"]:
        r["state"], r["d_state"] = s["state_out"], s["d_state_in"]
    return r


def _normed(s):
    r = {"out": s["out"]}
    if s["case"]["delta"]:
        r["sum"] = s["sum"]
    if s["case"]["eight"]:
        r["scales"] = s["scales"]
    return r


def _doubling(a, b, most):
    """y_t = a_t y_{t-1} + b_t along the rows, in place of b: pairs of rows, of pairs, and so on; a is
    zero where a sequence begins, and used up."""
    step = 1
    while step < most:
        b[step:] += a[step:] * b[:-step]
        a[step:] = a[step:] * a[:-step]
        step *= 2
    return b


def _directed(s):
    """Gates, candidates and their sequences in the direction of the recurrence: first and last rows of the
    sequences that have rows, these sequences, and how to put rows back."""
    turn = (lambda x: x.flip(0)) if s["case"]["reverse"] else (lambda x: x)
    off = s["offsets"]
    has = torch.nonzero(off[1:] > off[:-1])[:, 0]
    first, last = off[:-1][has], off[1:][has] - 1
    if s["case"]["reverse"]:
        N = s["gate"].shape[0]
        first, last = N - 1 - last, N - 1 - first
    return turn(torch.sigmoid(s["gate"].float())), turn(s["cand"].float()), first, last, has, turn


def _states(s, z, n, first, has):
    """All states h."""
    b = z * n
    a = 1 - z
    if s["case"]["states"]:
        b[first] += a[first] * s["state_in"][has]
    a[first] = 0
    return _doubling(a, b, s["most"])


def _plain_scan(s):
    z, n, first, last, has, turn = _directed(s)
    h = _states(s, z, n, first, has)
    s["out"].copy_(turn(h))
    if not s["case"]["states"]:
        return {"out": s["out"]}
    s["state_out"].copy_(s["state_in"])
    s["state_out"][has] = h[last]
    return {"out": s["out"], "state": s["state_out"]}


def _plain_train(s):
    z, n, first, last, has, turn = _directed(s)
    h = _states(s, z, n, first, has)
    s["out"].copy_(turn(h))
    states = s["case"]["states"]
    if states:
        s["state_out"].copy_(s["state_in"])
        s["state_out"][has] = h[last]
    # n_t - h_{t-1}
    e = n.clone()
    e[1:] -= h[:-1]
    e[first] = n[first]
    if states:
        e[first] -= s["state_in"][has]
    del h
    # the state's gradient, from the last row on: what comes from the row behind has that row's 1 - z
    d = turn(s["d_out"].float())
    if s["case"]["reverse"] is False:
        d = d.clone()
    if states:
        d[last] += s["d_state_out"][has]
    a = torch.zeros_like(z)
    a[:-1] = 1 - z[1:]
    a[last] = 0
    d = _doubling(a.flip(0), d.flip(0), s["most"]).flip(0)
    del a
    s["d_cand"].copy_(turn(z * d))
    s["d_gate"].copy_(turn(z * (1 - z) * e * d))
    if states:
        s["d_state_in"].copy_(s["d_state_out"])
        s["d_state_in"][has] = (1 - z[first]) * d[first]
    return _trained(s)


def _plain_step(s):
    at = s["slots"].long() if s["slots"] is not None else None
    h = s["state_in"] if at is None else s["state_in"][at]
    h = h + torch.sigmoid(s["gate"].float()) * (s["cand"].float() - h)
    s["out"].copy_(h)
    if at is None:
        s["state_out"].copy_(h)
    else:
        s["state_out"][at] = h
    return {"out": s["out"], "state": s["state_out"]}


def _plain_norm(s):
    x = s["x"].float()
    if s["case"]["delta"]:
        x = x + s["delta"].float()
        s["sum"].copy_(x)
    y = x * torch.rsqrt(torch.mean(x * x, -1, keepdim=True) + EPS) * s["gain"]
    if s["case"]["eight"]:
        scale = (y.abs().amax(-1) / LARGEST).clamp_min(LEAST_SCALE)
        s["scales"].copy_(scale)
        y = (y / scale[:, None]).clamp(-LARGEST, LARGEST)
    s["out"].copy_(y)
    return _normed(s)


def _plain_product(s):
    c = s["case"]
    y = torch.matmul(s["x"].float(), s["weight"].float().T)
    if c["eight"]:
        y = y * s["x_scales"][:, None] * s["weight_scales"]
    y = y + s["bias"]
    if c["act"] == "relu":
        y = torch.where(y > 0, y, 0.0)
    elif c["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    elif c["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if c["gate"]:
        y = y / (1 + torch.exp(-s["gate"].float()))
    if c["residual"]:
        y = y + s["residual"].float()
    s["out"].copy_(y)
    return {"out": s["out"]}


def exact(case, seed):
    """The definitions, in 64 bits; the recurrences row by row."""
    s = prepare(case, seed)
    return {"scan": _exact_scan, "train": _exact_scan, "step": _exact_step, "norm": _exact_norm,
            "product": _exact_product}[case["kind"]](s)


def _logistic(x):
    """1 / (1 + exp(-x)) in 64 bits."""
    return 0.5 * (1 + torch.tanh(0.5 * x.double()))


def _exact_scan(s):
    c = s["case"]
    off, B = s["offsets"], c["sequences"]
    h = s["state_in"].double() if c["states"] else torch.zeros((B, c["channels"]), dtype=torch.float64, device="cuda")
    z, n = _logistic(s["gate"]), s["cand"].double()
    out = torch.zeros_like(n)
    train = c["kind"] == "train"
    e = torch.zeros_like(n) if train else None
    length = off[1:] - off[:-1]
    order = torch.argsort(length, descending=True)     # the sequences that reach row t come first
    lo, hi, h = off[:-1][order], off[1:][order] - 1, h[order]
    lengths = length[order].tolist()
    live, alive = B, []
    for t in range(s["most"]):
        while live and lengths[live - 1] <= t:
            live -= 1
        alive.append(live)
        row = hi[:live] - t if c["reverse"] else lo[:live] + t
        v = n[row] - h[:live]
        h[:live] += z[row] * v
        out[row] = h[:live]
        if train:
            e[row] = v
    back = torch.empty_like(order)
    back[order] = torch.arange(B, device="cuda")
    r = {"out": out}
    if c["states"]:
        r["state"] = h[back]
    if not train:
        return r
    d = s["d_state_out"].double()[order] if c["states"] else torch.zeros_like(h)
    dg, dc = torch.zeros_like(out), torch.zeros_like(out)
    for t in range(s["most"] - 1, -1, -1):
        live = alive[t]
        row = hi[:live] - t if c["reverse"] else lo[:live] + t
        d[:live] += s["d_out"][row].double()
        x = z[row]
        dc[row] = x * d[:live]
        d[:live] *= 1 - x
        dg[row] = x * e[row] * d[:live]
    r["d_gate"], r["d_cand"] = dg, dc
    if c["states"]:
        r["d_state"] = d[back]
    return r


def _exact_step(s):
    at = torch.arange(s["case"]["sequences"], device="cuda") if s["slots"] is None else s["slots"].long()
    state = s["state_in"].double()
    z = _logistic(s["gate"])
    h = (1 - z) * state[at] + z * s["cand"].double()
    state[at] = h
    return {"out": h, "state": state}


def _nearest_e4m3(x):
    """Three bits behind the leading one, steps of 2^-9 below 2^-6; halves to the even value."""
    exponent = torch.frexp(x.abs().clamp_min(2.0 ** -6))[1].double() - 1
    step = torch.exp2(exponent - 3)
    return torch.round(x / step) * step


def _exact_norm(s):
    x = s["x"].double()
    r = {}
    if s["case"]["delta"]:
        x = x + s["delta"].double()
        r["sum"] = x
    y = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * s["gain"].double()
    if s["case"]["eight"]:
        scale = torch.clamp(y.abs().amax(-1) / LARGEST, min=LEAST_SCALE)
        r["scales"], y = scale, _nearest_e4m3(torch.clamp(y / scale[:, None], -LARGEST, LARGEST))
    r["out"] = y
    return r


def _exact_product(s):
    c = s["case"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    w = s["weight"].double()
    if c["eight"]:
        w = w * s["weight_scales"].double()[:, None]
    for a in range(0, c["rows"], 1 << 17):
        b = min(a + (1 << 17), c["rows"])
        x = s["x"][a:b].double()
        if c["eight"]:
            x = x * s["x_scales"][a:b].double()[:, None]
        y = torch.addmm(s["bias"].double(), x, w.T)
        if c["act"] == "relu":
            y = torch.clamp(y, min=0.0)
        elif c["act"] == "silu":
            y = y * _logistic(y)
        elif c["act"] == "gelu":
            y = 0.5 * y * torch.special.erfc(-y / math.sqrt(2.0))
        if c["gate"]:
            y = y * _logistic(s["gate"][a:b])
        if c["residual"]:
            y = y + s["residual"][a:b].double()
        out[a:b] = y
    return {"out": out}


def work(case):
    """Each input read once, each output written once.  Operations: a multiply and an add count two."""
    e = 4 if case["type"] == "fp32" else 2
    if case["kind"] in ("scan", "train"):
        B, C = case["sequences"], case["channels"]
        N = int(_lengths(case).sum())
        bytes, flops = 3 * e * N * C + 8 * (B + 1), 8 * N * C
        if case["states"]:
            bytes += 8 * B * C
        if case["kind"] == "train":
            bytes, flops = bytes + 5 * e * N * C + 8 * (B + 1) + (12 * B * C if case["states"] else 0), flops + 20 * N * C
        return {"bytes": bytes, "flops": flops}
    if case["kind"] == "step":
        return {"bytes": case["sequences"] * case["channels"] * (3 * e + 8) + (4 * case["sequences"] if case["slots"] else 0),
                "flops": 8 * case["sequences"] * case["channels"]}
    N = case["rows"]
    if case["kind"] == "norm":
        C = case["channels"]
        return {"bytes": N * C * (e * (3 if case["delta"] else 1) + (1 if case["eight"] else e)) + 4 * C +
                (4 * N if case["eight"] else 0), "flops": 6 * N * C}
    K, M = case["inner"], case["outer"]
    i = 1 if case["eight"] else e
    return {"bytes": i * K * (N + M) + e * N * M * (1 + case["gate"] + case["residual"]) + 4 * M +
            (4 * (N + M) if case["eight"] else 0), "flops": 2 * N * M * K}
