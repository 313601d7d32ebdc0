"""What the speed of the sequence-layer operators is measured on: the calls a program makes that serves a state space
mixer layer (matrix products around a short causal convolution and a selective scan).

Kinds of case:

  linear      y = act(x w^T + bias) + residual
  conv        short causal convolution over ragged prompts, continuing from and leaving a state per request
  conv_step   the same for one token of every request
  scan        selective state space scan over ragged prompts, continuing from and leaving a state per request
  scan_step   the same for one token of every request

A mixer's first product leaves one row per token, [z | x | B | C | dt], so the operators behind it read slices of longer
rows; the cases lay their inputs out like that.
"""
import math

import torch
import torch.nn.functional as F

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_CHUNK = 64   # tokens that the plain scan takes at once


# ---- the cases ---------------------------------------------------------------------------------
def _linear(name, m, n, k, dtype, act="none", bias=True, residual=False):
    return dict(name=name, kind="linear", m=m, n=n, k=k, dtype=dtype, act=act, bias=bias, residual=residual)


def _conv(name, sequences, tokens, channels, width, dtype, spread, resume):
    return dict(name=name, kind="conv", sequences=sequences, tokens=tokens, channels=channels, width=width, dtype=dtype,
                spread=spread, resume=resume)


def _scan(name, sequences, tokens, heads, head_dim, groups, state_dim, dtype, spread, resume, gate=True):
    return dict(name=name, kind="scan", sequences=sequences, tokens=tokens, heads=heads, head_dim=head_dim, groups=groups,
                state_dim=state_dim, dtype=dtype, spread=spread, resume=resume, gate=gate)


def _scan_step(name, sequences, heads, head_dim, groups, state_dim, dtype, gate=True):
    return dict(name=name, kind="scan_step", sequences=sequences, heads=heads, head_dim=head_dim, groups=groups,
                state_dim=state_dim, dtype=dtype, gate=gate)


def listed():
    return [
        # one token through a small layer's output product: latency
        _linear("linear_token_bf16", 1, 1024, 2048, "bf16", bias=False, residual=True),
        # a batch of requests, one token each, through the mixer's wide first product: its weights' bytes
        _linear("linear_decode32_bf16", 32, 8512, 2048, "bf16"),
        # the classifier behind a ResNet-50's pooled features over a large batch, in this library's own type
        _linear("linear_classifier_f32", 777, 1000, 2048, "f32"),
        # a ragged batch of prompts through a gated layer's first product, activation fused, sizes that fit no tile
        _linear("linear_ragged_gelu_f16", 1777, 2304, 1544, "f16", act="gelu"),
        # long prompts through the output product with its residual: the largest product
        _linear("linear_prompt_bf16", 16384, 4096, 4096, "bf16", bias=False, residual=True),
        # one token of every request through the short convolution
        dict(name="conv_step_bf16", kind="conv_step", sequences=64, channels=2304, width=4, dtype="bf16"),
        # ragged prompts through the short convolution of x, B and C together
        _conv("conv_ragged_bf16", 37, 16384, 4352, 4, "bf16", spread=3.0, resume=True),
        # one token of a few requests through the recurrence: latency
        _scan_step("step_few_bf16", 4, 32, 64, 1, 128, "bf16"),
        # one token of many requests: the states' bytes
        _scan_step("step_many_bf16", 256, 64, 64, 1, 128, "bf16"),
        # a single long prompt, few heads: parallel along the tokens or not at all
        _scan("scan_long_bf16", 1, 16384, 32, 64, 1, 128, "bf16", spread=1.0, resume=False),
        # ragged prompts, some of them the next part of a longer one
        _scan("scan_ragged_bf16", 24, 12000, 64, 64, 2, 128, "bf16", spread=4.0, resume=True),
        # short odd prompts of a small layer whose sizes fit no tile, half precision, no gate
        _scan("scan_odd_f16", 9, 1001, 10, 48, 2, 72, "f16", spread=2.0, resume=True, gate=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "conv", "conv_step", "scan", "scan", "scan_step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "linear":
        while True:
            m, n, k = _log_int(rng, 1, 16384), _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
            if rng.random() < 0.75:      # most layers' widths are multiples of something; some are not
                n, k = max(64, n // 8 * 8), max(64, k // 8 * 8)
            if m * n * k <= 2 ** 37:
                break
        return dict(kind=kind, m=m, n=n, k=k, dtype=dtype, act=rng.choice(["none", "relu", "silu", "gelu"]),
                    bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    if kind in ("conv", "conv_step"):
        channels, width = _log_int(rng, 64, 4352), rng.choice([2, 3, 4])
        if kind == "conv_step":
            return dict(kind=kind, sequences=_log_int(rng, 1, 256), channels=channels, width=width, dtype=dtype)
        tokens = _log_int(rng, 16, 16384 if dtype != "f32" else 8192)
        return dict(kind=kind, sequences=_log_int(rng, 1, min(64, tokens)), tokens=tokens, channels=channels, width=width,
                    dtype=dtype, spread=rng.uniform(1.0, 6.0), resume=rng.random() < 0.5)
    groups = rng.choice([1, 1, 2, 4])
    heads = groups * _log_int(rng, 1, 64 // groups)
    head_dim = rng.choice([32, 48, 64, 64, 128, rng.randint(16, 128)])
    state_dim = rng.choice([16, 64, 128, 128, 256, rng.randint(16, 256)])
    gate = rng.random() < 0.5
    area = heads * head_dim * state_dim
    if kind == "scan_step":
        return dict(kind=kind, sequences=_log_int(rng, 1, max(1, min(256, 2 ** 27 // area))), heads=heads,
                    head_dim=head_dim, groups=groups, state_dim=state_dim, dtype=dtype, gate=gate)
    tokens = _log_int(rng, 1, max(64, min(16384, 2 ** 32 // area)))
    return dict(kind=kind, sequences=_log_int(rng, 1, min(32, tokens)), tokens=tokens, heads=heads, head_dim=head_dim,
                groups=groups, state_dim=state_dim, dtype=dtype, spread=rng.uniform(1.0, 6.0),
                resume=rng.random() < 0.5, gate=gate)


# ---- inputs --------------------------------------------------------------------------------------
def _lengths(case, seed):
    """Ragged lengths that add up to the case's tokens, the longest about `spread` times the mean; one is empty where
    there are enough."""
    s, total = case["sequences"], case["tokens"]
    g = torch.Generator().manual_seed(seed * 2 + 1)
    w = torch.rand(s, generator=g, dtype=torch.float64) ** (2.0 * (case["spread"] - 1.0)) + 0.02
    if s >= 8:
        w[int(torch.randint(0, s, (1,), generator=g))] = 0.0
    cut = torch.round(torch.cumsum(w, 0) / w.sum() * total).to(torch.int64).tolist()
    return [b - a for a, b in zip([0] + cut[:-1], cut)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale


def _slices(g, rows, widths, dtype):
    """Normal values in one buffer of `rows` rows, and the slices of the given widths side by side in it."""
    pad = (-sum(widths)) % 8
    buf = _randn(g, (rows, sum(widths) + pad)).to(_TYPES[dtype])
    return list(torch.split(buf, list(widths) + [pad], dim=1)[:len(widths)])


def _inputs(case, seed):
    """Everything that a pass reads, on the GPU."""
    g, kind, ty = _gen(seed), case["kind"], _TYPES[case["dtype"]]
    i = {}
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        i["x"] = _randn(g, (m, k)).to(ty)
        i["w"] = _randn(g, (n, k), k ** -0.5).to(ty)
        i["bias"] = _randn(g, (n,), 0.5).to(ty) if case["bias"] else None
        i["residual"] = _randn(g, (m, n)).to(ty) if case["residual"] else None
        return i
    s = case["sequences"]
    slots = s + 3                # a pool holds states of requests that are not in this call too
    perm = torch.randperm(slots, generator=torch.Generator().manual_seed(seed))[:s]
    i["slots"], i["slot_map"] = slots, perm.to(torch.int32).cuda()
    step = kind.endswith("_step")
    i["lengths"] = [1] * s if step else _lengths(case, seed)
    tokens = sum(i["lengths"])
    starts = [0]
    for n in i["lengths"]:
        starts.append(starts[-1] + n)
    i["starts"] = torch.tensor(starts, dtype=torch.int32).cuda()
    resume = [1] * s if step else [1 if case["resume"] and r % 2 == 0 else 0 for r in range(s)]
    i["resume_host"], i["resume"] = resume, torch.tensor(resume, dtype=torch.int32).cuda()
    if kind in ("conv", "conv_step"):
        c, width = case["channels"], case["width"]
        i["x"] = _slices(g, tokens, [64, c], case["dtype"])[1]
        i["w"] = _randn(g, (c, width), width ** -0.5).to(ty)
        i["bias"] = _randn(g, (c,), 0.1).to(ty)
        i["state"] = _randn(g, (slots, width - 1, c)).to(ty)
        return i
    h, p, gr, n = case["heads"], case["head_dim"], case["groups"], case["state_dim"]
    z, x, b, c, dt = _slices(g, tokens, [h * p, h * p, gr * n, gr * n, h], case["dtype"])
    i.update(x=x, b=b, c=c, dt=dt, z=z if case["gate"] else None)
    i["a"] = -(1.0 + 15.0 * torch.rand(h, generator=g, device="cuda"))
    d0 = torch.exp(math.log(1e-3) + (math.log(1e-1) - math.log(1e-3)) * torch.rand(h, generator=g, device="cuda"))
    i["dt_bias"] = d0 + torch.log(-torch.expm1(-d0))      # softplus of it is d0
    i["d"] = _randn(g, (h,), 0.2) + 1.0
    i["state"] = _randn(g, (slots, h, p, n), 0.5)
    return i


def prepare(case, seed):
    st = {"case": case, "in": _inputs(case, seed)}
    i, kind = st["in"], case["kind"]
    ty = _TYPES[case["dtype"]]
    if own:
        from paper_2008_04567_amd import binding as B
        st["B"] = B
        code = {"f32": B.F32, "bf16": B.BF16, "f16": B.F16}[case["dtype"]]
        empty = lambda shape, t=ty: torch.empty(shape, device="cuda", dtype=t)
        if kind == "linear":
            act = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}[case["act"]]
            st["desc"] = B.make_linear_desc(case["m"], case["n"], case["k"], dtype=code, act=act)
            st["y"] = empty((case["m"], case["n"]))
            need = B.linear_workspace(st["desc"])
        elif kind in ("conv", "conv_step"):
            st["desc"] = B.make_causal_conv_desc(
                case["sequences"], i["x"].shape[0], case["channels"], case["width"], max_length=max(i["lengths"]),
                slots=i["slots"], dtype=code, act=B.ACT_SILU, x_stride=i["x"].stride(0))
            st["y"] = empty(i["x"].shape)
            need = 0
        else:
            z = i["z"]
            st["desc"] = B.make_ssm_desc(
                case["sequences"], i["x"].shape[0], case["heads"], case["head_dim"], case["groups"], case["state_dim"],
                max_length=max(i["lengths"]), slots=i["slots"], dtype=code, dt_softplus=True, x_stride=i["x"].stride(0),
                dt_stride=i["dt"].stride(0), b_stride=i["b"].stride(0), c_stride=i["c"].stride(0),
                z_stride=z.stride(0) if z is not None else None)
            st["y"] = empty((i["x"].shape[0], case["heads"] * case["head_dim"]))
            need = B.ssm_workspace(st["desc"]) if kind == "scan" else 0
        st["workspace"] = torch.empty(need, device="cuda", dtype=torch.uint8) if need else None
        if "state" in i:         # the pool that the call leaves, the old one kept, so that a pass can be repeated
            st["state_out"] = i["state"].clone()
    elif kind == "conv":
        st["plan"] = _conv_plan(case, i)
    elif kind == "scan":
        st["plan"] = _scan_plan(i)
    return st


# ---- the framework's calls -----------------------------------------------------------------------
def _run_own(st):
    B, case, i, desc, y = st["B"], st["case"], st["in"], st["desc"], st["y"]
    kind, stream = case["kind"], torch.cuda.current_stream()
    if kind == "linear":
        B.linear_fwd(desc, i["x"], i["w"], y, bias=i["bias"], residual=i["residual"], workspace=st["workspace"],
                     stream=stream)
        return y
    if kind == "conv":
        B.causal_conv1d_fwd(desc, i["x"], i["w"], y, bias=i["bias"], starts=i["starts"], slot_map=i["slot_map"],
                            resume=i["resume"], state_in=i["state"], state_out=st["state_out"], stream=stream)
    elif kind == "conv_step":
        B.causal_conv1d_step(desc, i["x"], i["w"], y, bias=i["bias"], slot_map=i["slot_map"], state_in=i["state"],
                             state_out=st["state_out"], stream=stream)
    elif kind == "scan":
        B.ssm_scan_fwd(desc, i["x"], i["dt"], i["a"], i["b"], i["c"], y, d=i["d"], z=i["z"], dt_bias=i["dt_bias"],
                       starts=i["starts"], slot_map=i["slot_map"], resume=i["resume"], state_in=i["state"],
                       state_out=st["state_out"], workspace=st["workspace"], stream=stream)
    else:
        B.ssm_scan_step(desc, i["x"], i["dt"], i["a"], i["b"], i["c"], y, d=i["d"], z=i["z"], dt_bias=i["dt_bias"],
                        slot_map=i["slot_map"], state_in=i["state"], state_out=st["state_out"], stream=stream)
    return y, st["state_out"]


# ---- the plain forms -----------------------------------------------------------------------------
def _act(v, act):
    if act == "relu":
        return torch.clamp_min(v, 0.0)
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return v


def _plain_linear(case, i):
    v = i["x"].float() @ i["w"].float().T
    if i["bias"] is not None:
        v = v + i["bias"].float()
    v = _act(v, case["act"])
    if i["residual"] is not None:
        v = v + i["residual"].float()
    return v.to(i["x"].dtype)


def _conv_plan(case, i):
    """Rows of [histories of all requests | tokens] in the order history, tokens, history, tokens ..., where each token's
    window starts in that order, and where each request's last rows are."""
    past, s = case["width"] - 1, case["sequences"]
    order, first, tail, t = [], [], [], 0
    for r, n in enumerate(i["lengths"]):
        at = len(order)
        order += range(r * past, (r + 1) * past)
        order += range(s * past + t, s * past + t + n)
        first += range(at, at + n)
        tail += range(at + n, at + n + past)
        t += n
    cuda = lambda v: torch.tensor(v, dtype=torch.int64).cuda()
    return dict(order=cuda(order), first=cuda(first), tail=cuda(tail))


def _plain_conv(case, i, plan):
    past = case["width"] - 1
    slot = i["slot_map"].long()
    hist = i["state"][slot] * i["resume"].to(i["state"].dtype).view(-1, 1, 1)
    rows = torch.cat([hist.reshape(-1, case["channels"]), i["x"]])[plan["order"]]
    v, w = i["bias"].float(), i["w"].float()
    for j in range(past + 1):
        v = v + rows[plan["first"] + j].float() * w[:, j]
    state = i["state"].clone()
    state[slot] = rows[plan["tail"]].view(-1, past, case["channels"])
    return _act(v, "silu").to(i["x"].dtype), state


def _plain_conv_step(case, i):
    slot = i["slot_map"].long()
    rows = torch.cat([i["state"][slot], i["x"].unsqueeze(1)], 1)
    v = i["bias"].float() + (rows.float() * i["w"].float().T).sum(1)
    state = i["state"].clone()
    state[slot] = rows[:, 1:]
    return _act(v, "silu").to(i["x"].dtype), state


def _softplus(v):
    return torch.clamp_min(v, 0.0) + torch.log1p(torch.exp(-torch.abs(v)))


def _scan_plan(i):
    """Tokens of chunks (a request's last chunk filled up with row `tokens`), and the chunks of each turn: the j-th of
    every request that has one, longest requests first."""
    tokens, start, chunks = sum(i["lengths"]), 0, []
    rows, row = [], 0
    for n in i["lengths"]:
        k = (n + _CHUNK - 1) // _CHUNK
        chunks.append(list(range(row, row + k)))
        for j in range(k):
            rows += [start + j * _CHUNK + t if j * _CHUNK + t < n else tokens for t in range(_CHUNK)]
        start, row = start + n, row + k
    order = sorted(range(len(chunks)), key=lambda r: -len(chunks[r]))
    turns = []
    for j in range(max(len(c) for c in chunks)):
        turns.append(torch.tensor([chunks[r][j] for r in order if len(chunks[r]) > j], dtype=torch.int64).cuda())
    where = torch.tensor(rows, dtype=torch.int64).cuda()
    return dict(rows=where, valid=(where < tokens), order=torch.tensor(order, dtype=torch.int64).cuda(), turns=turns,
                back=torch.nonzero(where < tokens).flatten())


def _plain_scan(case, i, plan):
    h, p, gr, n, q = case["heads"], case["head_dim"], case["groups"], case["state_dim"], _CHUNK
    rep = h // gr
    take = lambda v: torch.cat([v, v.new_zeros(1, v.shape[1])])[plan["rows"]].float().view(-1, q, v.shape[1])
    x, dt, b, c = take(i["x"]), take(i["dt"]), take(i["b"]), take(i["c"])
    k = x.shape[0]
    x = x.view(k, q, h, p).permute(0, 2, 1, 3).contiguous()                              # k h q p
    b, c = [v.view(k, q, gr, n).permute(0, 2, 1, 3).contiguous() for v in (b, c)]        # k g q n
    dt = (_softplus(dt + i["dt_bias"]) * plan["valid"].view(k, q, 1)).permute(0, 2, 1)   # k h q
    s = torch.cumsum(dt * i["a"].view(1, h, 1), 2)
    tri = torch.ones(q, q, device=x.device, dtype=torch.bool).tril()
    decay = torch.exp(torch.where(tri, s.unsqueeze(3) - s.unsqueeze(2), -math.inf))      # k h t s
    bt = b.transpose(2, 3).contiguous()
    m = torch.matmul(c, bt).repeat_interleave(rep, 1) * decay * dt.unsqueeze(2)
    y = torch.matmul(m, x)
    end = s[:, :, -1:]
    xw = (x * (torch.exp(end - s) * dt).unsqueeze(3)).transpose(2, 3).contiguous()       # k h p q
    local = torch.matmul(xw, b.repeat_interleave(rep, 1))                                # k h p n
    left = torch.exp(end).unsqueeze(3)
    before = torch.empty_like(local)
    slot = i["slot_map"].long()
    cur = (i["state"][slot] * i["resume"].view(-1, 1, 1, 1))[plan["order"]]
    for turn in plan["turns"]:
        before[turn] = cur[:len(turn)]
        cur[:len(turn)] = cur[:len(turn)] * left[turn] + local[turn]
    y = y + torch.matmul(c.repeat_interleave(rep, 1), before.transpose(2, 3).contiguous()) * torch.exp(s).unsqueeze(3)
    y = y + x * i["d"].view(1, h, 1, 1)
    y = y.permute(0, 2, 1, 3).reshape(k * q, h * p)[plan["back"]]
    if i["z"] is not None:
        y = y * _act(i["z"].float(), "silu")
    state = i["state"].clone()
    state[slot[plan["order"]]] = cur
    return y.to(i["x"].dtype), state


def _plain_scan_step(case, i):
    h, p, gr, n, s = case["heads"], case["head_dim"], case["groups"], case["state_dim"], case["sequences"]
    slot = i["slot_map"].long()
    x = i["x"].float().view(s, h, p)
    b, c = [i[v].float().view(s, gr, n).repeat_interleave(h // gr, 1) for v in ("b", "c")]
    dt = _softplus(i["dt"].float() + i["dt_bias"])
    cur = i["state"][slot] * torch.exp(dt * i["a"]).view(s, h, 1, 1) + (x * dt.unsqueeze(2)).unsqueeze(3) * b.unsqueeze(2)
    y = (cur * c.unsqueeze(2)).sum(3) + x * i["d"].view(1, h, 1)
    y = y.view(s, h * p)
    if i["z"] is not None:
        y = y * _act(i["z"].float(), "silu")
    state = i["state"].clone()
    state[slot] = cur
    return y.to(i["x"].dtype), state


def run(state):
    if own:
        return _run_own(state)
    case, i = state["case"], state["in"]
    kind = case["kind"]
    if kind == "linear":
        return _plain_linear(case, i)
    if kind == "conv":
        return _plain_conv(case, i, state["plan"])
    if kind == "conv_step":
        return _plain_conv_step(case, i)
    if kind == "scan":
        return _plain_scan(case, i, state["plan"])
    return _plain_scan_step(case, i)


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    e, kind = _BYTES[case["dtype"]], case["kind"]
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        cells = m * k + n * k + m * n * (2 if case["residual"] else 1) + (n if case["bias"] else 0)
        return {"bytes": e * cells, "flops": 2.0 * m * n * k}
    s = case["sequences"]
    tokens = s if kind.endswith("_step") else case["tokens"]
    read = s if kind.endswith("_step") else (s + 1) // 2 if case["resume"] else 0     # states that a pass continues from
    if kind in ("conv", "conv_step"):
        c, width = case["channels"], case["width"]
        return {"bytes": e * c * (2 * tokens + (read + s) * (width - 1) + width + 1),
                "flops": 2.0 * tokens * c * width}
    h, p, gr, n = case["heads"], case["head_dim"], case["groups"], case["state_dim"]
    row = h * p * (3 if case["gate"] else 2) + 2 * gr * n + h
    return {"bytes": e * tokens * row + 4 * (read + s) * h * p * n + 12 * h, "flops": 5.0 * tokens * h * p * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------
def exact(case, seed):
    i, kind = _inputs(case, seed), case["kind"]
    f64 = lambda v: None if v is None else v.double()
    if kind == "linear":
        v = torch.matmul(f64(i["x"]), f64(i["w"]).T)
        if case["bias"]:
            v += f64(i["bias"])
        act = case["act"]
        v = {"none": lambda t: t, "relu": torch.relu, "silu": F.silu, "gelu": F.gelu}[act](v)
        return v if i["residual"] is None else v + f64(i["residual"])
    slot, starts = i["slot_map"].tolist(), i["starts"].tolist()
    if kind in ("conv", "conv_step"):
        past = case["width"] - 1
        x, w, bias, state = f64(i["x"]), f64(i["w"]), f64(i["bias"]), f64(i["state"])
        y, after = torch.empty_like(x), state.clone()
        for r in range(case["sequences"]):
            hist = state[slot[r]] if i["resume_host"][r] else torch.zeros_like(state[0])
            line = torch.cat([hist, x[starts[r]:starts[r + 1]]])
            n = line.shape[0] - past
            if n:
                y[starts[r]:starts[r + 1]] = F.silu((line.unfold(0, past + 1, 1) * w).sum(2) + bias)
            after[slot[r]] = line[n:]
        return y, after
    h, p, gr, n = case["heads"], case["head_dim"], case["groups"], case["state_dim"]
    s, lengths = case["sequences"], i["lengths"]
    if max(lengths) > 40000:
        return None
    order = sorted(range(s), key=lambda r: -lengths[r])      # the requests still running are the first ones
    idx = torch.tensor(order, device="cuda")
    at = i["starts"].long()[:-1][idx]
    state = f64(i["state"])
    sl = i["slot_map"].long()[idx]
    cur = state[sl] * i["resume"].double()[idx].view(-1, 1, 1, 1)
    y = torch.empty(i["x"].shape, device="cuda", dtype=torch.float64)
    a, d, dt_bias = f64(i["a"]), f64(i["d"]), f64(i["dt_bias"])
    dt_all = F.softplus(f64(i["dt"]) + dt_bias, threshold=1000.0)
    da_all = torch.exp(dt_all * a)
    live = s
    for t in range(max(lengths)):
        while live and lengths[order[live - 1]] <= t:
            live -= 1
        tok, hs = at[:live] + t, cur[:live]
        xt = i["x"][tok].double().view(live, h, p)
        bt = i["b"][tok].double().view(live, gr, 1, 1, n).expand(-1, -1, h // gr, -1, -1).reshape(live, h, 1, n)
        ct = i["c"][tok].double().view(live, gr, 1, n, 1).expand(-1, -1, h // gr, -1, -1).reshape(live, h, n, 1)
        hs *= da_all[tok].view(live, h, 1, 1)
        hs.addcmul_((xt * dt_all[tok].unsqueeze(2)).unsqueeze(3), bt)
        yt = torch.matmul(hs, ct).squeeze(3) + xt * d.view(1, h, 1)
        y[tok] = yt.view(live, h * p)
    if i["z"] is not None:
        y *= F.silu(i["z"].double())
    after = state.clone()
    after[sl] = cur
    return y, after
