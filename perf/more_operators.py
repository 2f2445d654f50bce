"""The operators of a delta-rule layer (GDN, KDA) and of its 8-bit integer projections, as a program that serves a model calls them.

`perf/operators.py` measures those around the Mamba-2 recurrence; the cases here are what the other two recurrences run before and after
their decode steps, through the public calls of `binding.SketchSSM`:
- op "scan":   the gated delta rule over packed prompts, with the keys' and queries' norms and the gates, which leaves the state that the
               decode steps go on from (GDN: a decay for each head, KDA: one for each channel of a key);
- op "token":  the convolution, the norms and the gates of one token of every sequence, laid out as the decode calls want them;
- op "norm":   the root-mean-square norm with the residual's addition before it, or of every head's output with the gate behind it, and its
               rows in 8-bit integers with a scale for each token;
- op "matmul": the product of such rows by 8-bit integer weights with a scale for each channel.

With `own` false each is computed by elementary torch operations in 32 bits (sums of log decays in 64).
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_EPS_QK, _EPS = 1e-6, 1e-5

_SCAN = dict(op="scan", kind="gdn", tokens=16384, sequences=1, heads=32, groups=16, dk=128, dv=128, io="bf16", out="bf16", resume=False)
_TOKEN = dict(op="token", kind="gdn", batch=512, heads=32, groups=16, dk=128, dv=128, width=4, io="bf16")
_NORM = dict(op="norm", rows=16384, width=2048, mode="residual", group=2048, act="silu", io="bf16", x="bf16")
_MATMUL = dict(op="matmul", rows=16384, cols=12352, inner=2048, out="bf16")


def _case(base, name, **kw):
    return dict(base, name=name, **kw)


def listed():
    return [
        # one short prompt: less than two chunks, where the call's latency counts
        _case(_SCAN, "scan_short", tokens=100),
        # one long prompt of the GDN layer workload's heads
        _case(_SCAN, "scan_long"),
        # many prompts of ragged lengths that go on from stored states
        _case(_SCAN, "scan_ragged", sequences=48, resume=True),
        # KDA: a few prompts admitted together, keys and queries for every head, a decay for every channel
        _case(_SCAN, "scan_kda", kind="kda", tokens=4096, sequences=8, groups=32, resume=True),
        # 32-bit tensors and 80 value channels
        _case(_SCAN, "scan_v80_f32", tokens=1500, sequences=7, heads=24, groups=12, dv=80, io="f32", out="f32"),
        # a single user's token
        _case(_TOKEN, "token_one", batch=1),
        # a decode step of the KDA layer workload's batch
        _case(_TOKEN, "token_kda", kind="kda", groups=32),
        # the norm before a layer's first projection over a batch of prompts
        _case(_NORM, "norm_prompts"),
        # the heads' norm and gate behind a decode step, its input as the step leaves it
        _case(_NORM, "norm_gated_token", rows=512, width=4096, mode="gated", group=128, x="f32"),
        # a layer's first projection for a decode step: the weights are what is read
        _case(_MATMUL, "matmul_token", rows=64),
        # an odd number of rows and columns, 32-bit result
        _case(_MATMUL, "matmul_odd_f32", rows=777, cols=2049, inner=4096, out="f32"),
        # the first projection of the prompts: the largest product
        _case(_MATMUL, "matmul_prompts"),
    ]


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["scan", "scan", "scan", "scan", "token", "token", "norm", "norm", "matmul", "matmul"])
    if op == "scan":
        c = dict(_SCAN)
        c["kind"] = rng.choice(["gdn", "gdn", "kda"])
        c["heads"] = rng.choice([4, 8, 16, 24, 32, 48])
        c["groups"] = c["heads"] // rng.choice([1, 1, 2, 4])
        c["dk"], c["dv"] = rng.choice([(128, 128)] * 5 + [(128, 64), (128, 80), (64, 64)])
        c["io"], c["out"] = rng.choice([("bf16", "bf16")] * 4 + [("bf16", "f32"), ("f32", "f32")])
        most = 16384 * 32 if c["kind"] == "gdn" and c["io"] == "bf16" and c["dk"] == c["dv"] == 128 else 1500 * 24
        c["tokens"] = _log(rng, 1, min(16384, most // c["heads"]))
        c["sequences"] = _log(rng, 1, min(64, c["tokens"]))
        c["resume"] = rng.random() < 0.5
    elif op == "token":
        c = dict(_TOKEN)
        c["kind"] = rng.choice(["gdn", "kda"])
        c["batch"] = _log(rng, 1, 512)
        c["heads"] = rng.choice([4, 8, 16, 24, 32])
        c["groups"] = c["heads"] // rng.choice([1, 1, 2, 4])
        c["dk"], c["dv"] = rng.choice([(128, 128), (128, 128), (128, 64), (128, 80), (64, 64)])
        c["width"] = rng.choice([4, 4, 3, 2])
        c["io"] = rng.choice(["bf16", "bf16", "f32"])
    elif op == "norm":
        c = dict(_NORM)
        c["rows"] = _log(rng, 1, 16384)
        c["mode"] = rng.choice(["residual", "plain", "gated"])
        c["io"] = rng.choice(["bf16", "bf16", "f32"])
        if c["mode"] == "gated":
            c["group"] = rng.choice([64, 80, 128, 128])
            c["width"] = c["group"] * _log(rng, 2, 40)
            c["act"] = rng.choice(["silu", "sigmoid"])
            c["x"] = rng.choice(["f32", c["io"]])
        else:
            c["width"] = c["group"] = 8 * _log(rng, 16, 640)
            c["x"] = c["io"]
        c["rows"] = max(1, min(c["rows"], 16384 * 2048 // c["width"] // (2 if "f32" in (c["io"], c["x"]) else 1)))
    else:
        c = dict(_MATMUL)
        c["rows"] = _log(rng, 1, 16384)
        c["cols"] = rng.choice([8 * _log(rng, 8, 1544), _log(rng, 64, 12352)])
        c["inner"] = 16 * _log(rng, 8, 512)
        c["out"] = rng.choice(["bf16", "bf16", "f32"])
        c["rows"] = max(1, min(c["rows"], 16384 * 12352 // c["cols"] * 2048 // c["inner"]))
    return c


# ---- what a program has in hand ---------------------------------------------------------------------------------------


def _lengths(tokens, sequences, seed):
    """Ragged lengths that sum to `tokens`; with many sequences one of them is empty."""
    r = random.Random(seed)
    w = [r.uniform(0.05, 1.0) ** 2 for _ in range(sequences)]
    if sequences > 4:
        w[r.randrange(sequences)] = 0.0
    ends = [0]
    for i in range(sequences):
        ends.append(round(tokens * sum(w[:i + 1]) / sum(w)))
    return [ends[i + 1] - ends[i] for i in range(sequences)]


def _batch(c, seed):
    """Packed prompts: lengths, first rows, where each sequence's state goes and where it comes from (-1: from nothing)."""
    n = c["sequences"]
    lens = _lengths(c["tokens"], n, seed)
    starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    r = random.Random(seed + 1)
    slots = list(range(n))
    r.shuffle(slots)
    resume = [n + i if c["resume"] and r.random() < 0.75 else -1 for i in range(n)]
    return dict(lens=lens, starts=starts, slots=torch.tensor(slots, dtype=torch.int32).cuda(),
                resume=torch.tensor(resume, dtype=torch.int32).cuda())


def _layer(c, batch):
    from paper_2609_33051_b200 import binding
    return binding.SketchSSM(c.get("kind", "gdn"), batch, c.get("heads", 1), c.get("dk", 64), c.get("dv", 64), 8, 4, io=c.get("io", "bf16"),
                             out="f32", device=torch.cuda.current_device())


def prepare(case, seed):
    c, gen = dict(case), torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=c)

    def normal(*shape, dtype="f32"):
        return torch.randn(*shape, device="cuda", generator=gen).to(_TORCH[dtype])

    def gates():
        """a [H] < 0, and the bias of the step size of every head, or of every channel: decays of a token from nothing to a fifth."""
        h = c["heads"]
        a = -1.0 - 15.0 * torch.rand(h, device="cuda", generator=gen)
        step = torch.exp(math.log(1e-3) + math.log(100.0) * torch.rand(*((h, c["dk"]) if c["kind"] == "kda" else (h,)), device="cuda", generator=gen))
        return a, torch.log(torch.expm1(step))

    if c["op"] == "scan":
        n, t, h, g, k, v, io = c["sequences"], c["tokens"], c["heads"], c["groups"], c["dk"], c["dv"], c["io"]
        s["batch"] = _batch(c, seed)
        # a row of the convolution's output: values, keys, queries
        row = normal(t, h * v + 2 * g * k, dtype=io)
        s["v"] = row[:, :h * v].unflatten(1, (h, v))
        s["k"] = row[:, h * v:h * v + g * k].unflatten(1, (g, k))
        s["q"] = row[:, h * v + g * k:].unflatten(1, (g, k))
        # the projection's columns behind them: step sizes and the decays' arguments
        row = normal(t, h + (h * k if c["kind"] == "kda" else h), dtype=io)
        s["b"], s["dt"] = row[:, :h], row[:, h:]
        s["a"], s["dt_bias"] = gates()
        state = normal(2 * n, h, k, v) / math.sqrt(k)
        if own:
            from paper_2609_33051_b200 import binding
            s["m"] = _layer(c, 2 * n)
            s["prompts"] = binding.Prompts(s["batch"]["starts"], t, slots=s["batch"]["slots"], resume=s["batch"]["resume"])
            s["m"].state.copy_(state)
            s["y"] = torch.empty(t, h, v, dtype=_TORCH[c["out"]], device="cuda")
            s["work"] = s["m"].new_delta_work(n, t)
        else:
            s["state"] = state
    elif c["op"] == "token":
        h, g, k, v, w = c["heads"], c["groups"], c["dk"], c["dv"], c["width"]
        ch = h * v + 2 * g * k
        # a row of the layer's first projection: gate, convolved channels, step sizes, the decays' arguments
        row = normal(c["batch"], h * v + ch + h + (h * k if c["kind"] == "kda" else h), dtype=c["io"])
        s["x"], s["b"], s["dt"] = row[:, h * v:h * v + ch], row[:, h * v + ch:h * v + ch + h], row[:, h * v + ch + h:]
        s["w"] = normal(ch, w) / math.sqrt(w)
        s["a"], s["dt_bias"] = gates()
        s["conv"] = normal(c["batch"], w - 1, ch, dtype=c["io"])
        if own:
            s["m"] = _layer(c, c["batch"])
            s["token"] = s["m"].new_token_buffers()
    elif c["op"] == "norm":
        t, d, io = c["rows"], c["width"], c["io"]
        s["x"] = normal(t, d, dtype=c["x"])
        s["w"] = 1.0 + 0.1 * normal(c["group"])
        if c["mode"] == "residual":
            s["residual"] = 4.0 * normal(t, d, dtype=io)
            s["residual_out"] = torch.empty_like(s["residual"])
        if c["mode"] == "gated":
            s["gate"] = normal(t, d, dtype=io)
        s["values"] = torch.empty(t, d, dtype=torch.bfloat16, device="cuda")
        if own:
            s["m"] = _layer(c, 1)
            s["out8"] = torch.empty(t, d, dtype=torch.int8, device="cuda")
            s["scale"] = torch.empty(t, device="cuda")
    else:
        m, n, k = c["rows"], c["cols"], c["inner"]
        s["a"], s["a_scale"] = _quantise(normal(m, k))
        s["w"], s["w_scale"] = _quantise(normal(n, k) / math.sqrt(k))
        s["out"] = torch.empty(m, n, dtype=_TORCH[c["out"]], device="cuda")
        if own:
            s["m"] = _layer(c, 1)
    return s


def _quantise(x):
    """8-bit integers and a scale for each row."""
    scale = x.abs().amax(1) / 127.0
    return torch.round(x / scale[:, None]).to(torch.int8), scale


# ---- one pass ----------------------------------------------------------------------------------------------------------


def run(s):
    return globals()[("_own_" if own else "_plain_") + s["case"]["op"]](s)


def _anew(t):
    """Columns behind KDA's step sizes in rows that begin on 16 bytes, as the calls take them: few heads leave them, and the rows, off that."""
    return t if (t.data_ptr() | t.stride(0) * t.element_size()) % 16 == 0 else t.clone(memory_format=torch.contiguous_format)


def _own_scan(s):
    m, dt = s["m"], s["dt"]
    if s["case"]["kind"] == "kda":
        dt = _anew(dt)
    m.delta_scan(s["prompts"], s["q"], s["k"], s["v"], s["b"], dt, s["a"], s["y"], dt_bias=s["dt_bias"], eps=_EPS_QK, work=s["work"])
    return dict(y=s["y"], state=m.state)


def _own_token(s):
    t, x, dt = s["token"], s["x"], s["dt"]
    if s["case"]["kind"] == "kda":
        x, dt = _anew(x), _anew(dt)
    s["m"].delta_step(x, s["b"], dt, s["w"], None, s["conv"], s["a"], s["dt_bias"], t, groups=s["case"]["groups"], eps=_EPS_QK)
    return dict(q=t["q"], k=t["k"], v=t["v"], beta=t["beta"], decay=t["decay"], conv=s["conv"])


def _own_norm(s):
    c = s["case"]
    s["m"].integer_norm(s["x"], s["w"], s["out8"], s["scale"], residual=s.get("residual"), residual_out=s.get("residual_out"),
                     gate=s.get("gate"), act=c["act"], eps=_EPS)
    return _norm_result(s, s["out8"], s["scale"])


def _norm_result(s, out8, scale):
    # the values that the integers stand for
    torch.mul(out8, scale[:, None], out=s["values"])
    res = dict(values=s["values"], scale=scale)
    return dict(res, residual=s["residual_out"]) if s["case"]["mode"] == "residual" else res


def _own_matmul(s):
    s["m"].integer_matmul(s["a"], s["a_scale"], s["w"], s["w_scale"], s["out"])
    return dict(out=s["out"])


_Q = 64


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))


def _unit(x):
    x = x.float()
    return x * torch.rsqrt((x * x).sum(-1, keepdim=True) + _EPS_QK)


def _plain_scan(s):
    """Chunks of 64 tokens of one sequence each.  With u_t = beta_t (v_t - decayed state before t, read by k_t) a chunk is
        (I + L) U = beta (V - (e^c K) S),   Y = (e^c Q) S + P U,   S <- e^c_end S + (e^(c_end - c) K)^T U,
    L strictly lower and P lower triangular, both with the decays between two tokens; I + L is inverted row by row, for all chunks at
    once, and what passes from chunk to chunk goes through all sequences together."""
    c, b = s["case"], s["batch"]
    h, per_group, kda = c["heads"], c["heads"] // c["groups"], c["kind"] == "kda"
    lens = torch.tensor(b["lens"])
    per = (lens + _Q - 1) // _Q
    seq = torch.repeat_interleave(torch.arange(len(lens)), per)
    first = torch.arange(len(seq)) - (per.cumsum(0) - per)[seq]
    pos = (first * _Q)[:, None] + torch.arange(_Q)
    ok = (pos < lens[seq][:, None]).cuda()
    at = ((lens.cumsum(0) - lens)[seq][:, None] + pos).clamp(max=c["tokens"] - 1).cuda()
    wide = lambda z: z.repeat_interleave(per_group, 2).transpose(1, 2)  # noqa: E731        [N, H, Q, K]
    live = ok[:, None, :, None]
    q, k = wide(_unit(s["q"])[at]) * c["dk"] ** -0.5, wide(_unit(s["k"])[at]) * live
    beta = torch.sigmoid(s["b"].float())[at].transpose(1, 2)[..., None] * live
    v = s["v"].float()[at].transpose(1, 2) * live
    dt = s["dt"].float().unflatten(1, (h, -1)) + s["dt_bias"].reshape(h, -1)
    cum = ((_softplus(dt) * s["a"][:, None])[at].transpose(1, 2) * live).double().cumsum(2)              # [N, H, Q, 1 or K]
    t = torch.arange(_Q, device="cuda")
    below = t[:, None] > t
    if kda:
        L, P = torch.empty(2, len(seq), h, _Q, _Q, device="cuda")
        for j in range(_Q):
            kj = k[:, :, j:j + 1] * torch.exp(torch.clamp(cum - cum[:, :, j:j + 1], max=0)).float()
            L[..., j], P[..., j] = (k * kj).sum(-1), (q * kj).sum(-1)
    else:
        gap = torch.exp(torch.clamp(cum - cum.transpose(2, 3), max=0)).float()
        L, P = (k @ k.transpose(2, 3)) * gap, (q @ k.transpose(2, 3)) * gap
        del gap
    L = torch.where(below, beta * L, 0.0)
    P = torch.where(below.T, 0.0, P)
    T = torch.eye(_Q, device="cuda").expand_as(L).clone()
    for i in range(1, _Q):
        T[:, :, i, :i] = -(L[:, :, i, None, :i] @ T[:, :, :i, :i])[:, :, 0]
    e, end = torch.exp(cum).float(), cum[:, :, -1:]
    U, W = T @ (beta * v), T @ (beta * e * k)
    qe, ke, keep = q * e, (k * torch.exp(end - cum).float()).transpose(2, 3), torch.exp(end).float().transpose(2, 3)
    del L, T, e, q, k, v
    src = b["resume"].long()
    S = s["state"][src.clamp(min=0)] * (src >= 0)[:, None, None, None]
    order = torch.argsort(per, descending=True)
    firsts, counts = (per.cumsum(0) - per)[order].cuda(), per[order].tolist()
    back, S = order.cuda(), S[order.cuda()]
    out = torch.empty(c["tokens"], h, c["dv"], dtype=_TORCH[c["out"]], device="cuda")
    n = len(counts)
    for i in range(max(counts)):
        while counts[n - 1] <= i:
            n -= 1
        x = firsts[:n] + i
        u = U[x] - W[x] @ S[:n]
        y = qe[x] @ S[:n] + P[x] @ u
        S[:n] = keep[x] * S[:n] + ke[x] @ u
        out[at[x][ok[x]]] = y.transpose(1, 2)[ok[x]].to(out.dtype)
    s["state"][b["slots"].long()[back]] = S
    return dict(y=out, state=s["state"])


def _plain_token(s):
    c = s["case"]
    h, g, k, v, io = c["heads"], c["groups"], c["dk"], c["dv"], _TORCH[c["io"]]
    rows = torch.cat([s["conv"], s["x"][:, None]], 1)
    acc = (rows.float() * s["w"].T).sum(1)
    y = acc * torch.sigmoid(acc)
    s["conv"].copy_(rows[:, 1:])
    wide = lambda z: _unit(z.unflatten(1, (g, k))).repeat_interleave(h // g, 1)  # noqa: E731
    dt = s["dt"].float().unflatten(1, (h, -1)) + s["dt_bias"].reshape(h, -1)
    decay = torch.exp(_softplus(dt) * s["a"][:, None])
    return dict(q=(wide(y[:, h * v + g * k:]) * k ** -0.5).to(io), k=wide(y[:, h * v:h * v + g * k]).to(io),
                v=y[:, :h * v].unflatten(1, (h, v)).to(io), beta=torch.sigmoid(s["b"].float()),
                decay=decay.to(io) if c["kind"] == "kda" else decay[..., 0], conv=s["conv"])


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float()
    if c["mode"] == "residual":
        x = x + s["residual"].float()
        s["residual_out"].copy_(x)
    u = x.unflatten(1, (-1, c["group"]))
    y = (u * torch.rsqrt((u * u).mean(-1, keepdim=True) + _EPS) * s["w"]).flatten(1)
    if c["mode"] == "gated":
        z = s["gate"].float()
        y = y * torch.sigmoid(z) * (z if c["act"] == "silu" else 1.0)
    top = y.abs().amax(1)
    out8 = torch.round(y * torch.where(top > 1e-30, 127.0 / top, 0.0)[:, None])
    return _norm_result(s, out8, top * (1.0 / 127.0))


def _plain_matmul(s):
    s["out"].copy_((s["a"].float() @ s["w"].float().T) * s["a_scale"][:, None] * s["w_scale"])
    return dict(out=s["out"])


# ---- what a pass cannot do without, and its results in 64 bits ---------------------------------------------------------


def work(case):
    c = case
    if c["op"] == "scan":
        t, h, z = c["tokens"], c["heads"], _SIZE[c["io"]]
        state = c["sequences"] * h * c["dk"] * c["dv"] * 4
        per = h * c["dv"] * (z + _SIZE[c["out"]]) + 2 * c["groups"] * c["dk"] * z + h * z * (1 + (c["dk"] if c["kind"] == "kda" else 1))
        # a token's reading by its key and its query, and its outer product
        return {"bytes": t * per + (1.75 if c["resume"] else 1.0) * state, "flops": 6 * t * h * c["dk"] * c["dv"]}
    if c["op"] == "token":
        z, w, b, h, k = _SIZE[c["io"]], c["width"], c["batch"], c["heads"], c["dk"]
        ch = h * c["dv"] + 2 * c["groups"] * k
        gate = (2 * z * k if c["kind"] == "kda" else z + 4) + z + 4
        return {"bytes": b * ((2 * w - 1) * ch * z + h * (2 * k + c["dv"]) * z + h * gate) + ch * w * 4, "flops": 2 * w * b * ch}
    if c["op"] == "norm":
        t, d, z = c["rows"], c["width"], _SIZE[c["io"]]
        per = _SIZE[c["x"]] + {"plain": 0, "residual": 2 * z, "gated": z}[c["mode"]] + 1
        return {"bytes": t * (d * per + 4) + c["group"] * 4, "flops": 8 * t * d}
    m, n, k = c["rows"], c["cols"], c["inner"]
    return {"bytes": (m + n) * (k + 4) + m * n * _SIZE[c["out"]], "flops": 2 * m * n * k}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return globals()["_exact_" + case["op"]](s)


def _sigmoid64(x):
    return 1 / (1 + torch.exp(-x))


def _unit64(x):
    return x / torch.sqrt((x ** 2).sum(-1, keepdim=True) + _EPS_QK)


def _log_decay64(s):
    """[T, H, 1 or K]"""
    h = s["a"].shape[0]
    x = s["dt"].double().unflatten(1, (h, -1)) + s["dt_bias"].double().reshape(h, -1)
    return torch.logaddexp(x, torch.zeros_like(x)) * s["a"].double()[:, None]


def _exact_scan(s):
    """Token by token: S <- D S, S <- S + beta k (v - S^T k)^T, y = S^T q, all sequences that are still running at once."""
    c, b = s["case"], s["batch"]
    per_group = c["heads"] // c["groups"]
    if max(b["lens"]) * c["sequences"] * c["heads"] * c["dk"] * c["dv"] > 3e11:
        return None
    src, lens = b["resume"].long(), torch.tensor(b["lens"]).cuda()
    order = torch.argsort(lens, descending=True)
    begin = b["starts"].long()[:-1][order]
    S = (s["state"][src.clamp(min=0)].double() * (src >= 0)[:, None, None, None])[order]
    decay, beta = torch.exp(_log_decay64(s)), _sigmoid64(s["b"].double())
    query, key = (_unit64(s[z].double()).repeat_interleave(per_group, 1) for z in ("q", "k"))
    query = query / math.sqrt(c["dk"])
    y = torch.empty(c["tokens"], c["heads"], c["dv"], dtype=torch.float64, device="cuda")
    ends = sorted(b["lens"], reverse=True)
    n = len(ends)
    for t in range(max(b["lens"])):
        while n and ends[n - 1] <= t:
            n -= 1
        at = begin[:n] + t
        k, live = key[at], S[:n]
        live.mul_(decay[at][..., None])
        new = beta[at][..., None] * (s["v"][at].double() - torch.matmul(k[..., None, :], live).squeeze(-2))
        live.addcmul_(k[..., None], new[..., None, :])
        y[at] = torch.matmul(query[at][..., None, :], live).squeeze(-2)
    state = s["state"].clone().double()
    state[b["slots"].long()[order]] = S
    return dict(y=y, state=state)


def _exact_token(s):
    c = s["case"]
    h, g, k, v = c["heads"], c["groups"], c["dk"], c["dv"]
    full = torch.cat([s["conv"].double(), s["x"].double()[:, None]], 1)
    y = torch.einsum("bwc,cw->bc", full, s["w"].double())
    x, key, query = (y * _sigmoid64(y)).split([h * v, g * k, g * k], 1)
    spread = lambda z: _unit64(z.view(-1, g, 1, k)).expand(-1, g, h // g, k).reshape(-1, h, k)  # noqa: E731
    decay = torch.exp(_log_decay64(s))
    return dict(q=spread(query) / math.sqrt(k), k=spread(key), v=x.reshape(-1, h, v), beta=_sigmoid64(s["b"].double()),
                decay=decay if c["kind"] == "kda" else decay[..., 0], conv=full[:, 1:])


def _exact_norm(s):
    c, x, res = s["case"], s["x"].double(), {}
    if c["mode"] == "residual":
        x = x + s["residual"].double()
        res = dict(residual=x)
    y = torch.cat([p / torch.sqrt((p ** 2).mean(1, keepdim=True) + _EPS) * s["w"].double() for p in x.split(c["group"], 1)], 1)
    if c["mode"] == "gated":
        z = s["gate"].double()
        y = y * _sigmoid64(z) * (z if c["act"] == "silu" else 1)
    scale = y.abs().amax(1) / 127
    return dict(values=torch.round(y / scale[:, None]) * scale[:, None], scale=scale, **res)


def _exact_matmul(s):
    # (whole numbers below 2^53: the sums are exact)
    return dict(out=(s["a"].double() @ s["w"].double().T) * s["a_scale"].double()[:, None] * s["w_scale"].double())
