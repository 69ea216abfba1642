"""The operators of a prompt's layer around a decode worker's 8-bit cache and microscaled 4-bit weights, as cases that can be timed and compared:
attention of a chunk of new tokens of each request over the cache, the gated pair of a feed-forward block (both projections, the activation and
the product), and a projection with bias, activation and residual behind it.

A case is a dict of plain values:
  op "chunk": `batch` requests of lengths in [lo, hi], of which the last tokens are new: `new` of each ("even"), uneven counts up to `new`, none
              among them ("ragged"), `new` of every eighth request and one of the others ("mixed"), or all of them ("prompts"); `pad` rows behind the
              last; a token sees itself and what is in front of it, `window` positions of it (0: all).  Heads are `hq` query heads over `hkv` KV
              heads of `d` dims
  op "gated": `rows` rows through a pair of matrices [n, k] in the microscaled format, out = act(x Wg^T) * (x Wu^T)
  op "fused": out = act(x W^T + bias) + residual, `bias` and `act` where the case has them
Activations x (or queries) are `dtype`, "f32" or "bf16", and so is what comes out, or `out` where the case names it.  Sizes are the repository's own shapes
(8B, 14B, small, tiny).

`own` false: the plain forms, elementary torch operations in 32 bits.  `own` true: the library's calls.  exact() has the same results in 64 bits,
written apart from the plain forms."""
import math

import torch

own = False

PAGE = 16
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
DEV = "cuda:0"


def listed():
    return [
        # the smallest call: a few new tokens of short requests
        {"name": "chunk_tiny_b8_f32", "op": "chunk", "mode": "ragged", "batch": 8, "new": 5, "pad": 2, "hq": 4, "hkv": 2, "d": 64, "dtype": "f32", "lo": 16, "hi": 128, "window": 0},
        # four drafted tokens of every request of a medium batch are looked over at once, 8B heads
        {"name": "chunk_8b_b64_draft4_bf16", "op": "chunk", "mode": "even", "batch": 64, "new": 4, "pad": 0, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "lo": 512, "hi": 4096, "window": 0},
        # a block of a long prompt behind what earlier blocks have cached
        {"name": "chunk_8b_2048_of_8191_bf16", "op": "chunk", "mode": "even", "batch": 1, "new": 2048, "pad": 0, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "lo": 8191, "hi": 8191, "window": 0},
        # whole prompts of different lengths side by side, padded
        {"name": "chunk_8b_prompts_bf16", "op": "chunk", "mode": "prompts", "batch": 4, "new": 0, "pad": 9, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "lo": 300, "hi": 1500, "window": 0},
        # uneven chunks with a sliding window, five query heads per KV head, fp32 activations
        {"name": "chunk_14b_window_f32", "op": "chunk", "mode": "ragged", "batch": 5, "new": 500, "pad": 3, "hq": 40, "hkv": 8, "d": 128, "dtype": "f32", "lo": 700, "hi": 4000, "window": 1000},
        # prompts and decode steps in one batch
        {"name": "chunk_8b_b24_mixed_bf16", "op": "chunk", "mode": "mixed", "batch": 24, "new": 256, "pad": 1, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "lo": 256, "hi": 4096, "window": 0},
        # one user: the gate and up matrices are all there is to read
        {"name": "gated_14336x4096_1_bf16", "op": "gated", "n": 14336, "k": 4096, "rows": 1, "dtype": "bf16", "act": "silu"},
        # the benchmark's default batch
        {"name": "gated_14336x4096_64_bf16", "op": "gated", "n": 14336, "k": 4096, "rows": 64, "dtype": "bf16", "act": "silu"},
        # a ragged batch of the 14B shape, fp32 activations
        {"name": "gated_13824x5120_150_f32", "op": "gated", "n": 13824, "k": 5120, "rows": 150, "dtype": "f32", "act": "gelu_tanh"},
        # a prefill block
        {"name": "gated_14336x4096_2048_bf16", "op": "gated", "n": 14336, "k": 4096, "rows": 2048, "dtype": "bf16", "act": "silu"},
        # one user: the output projection onto a 32-bit residual stream
        {"name": "fused_4096x4096_1_bf16", "op": "fused", "n": 4096, "k": 4096, "rows": 1, "dtype": "bf16", "out": "f32", "act": "none", "bias": False},
        # a down projection with a bias, an odd number of rows
        {"name": "fused_5120x13824_333_bf16", "op": "fused", "n": 5120, "k": 13824, "rows": 333, "dtype": "bf16", "out": "bf16", "act": "gelu", "bias": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("chunk", "chunk", "chunk", "gated", "gated", "fused"))
    dtype = rng.choice(("f32", "bf16", "bf16"))
    if op != "chunk":
        case = {"op": op, "n": _log_int(rng, 17, 14336), "k": 32 * _log_int(rng, 2, 128), "rows": _log_int(rng, 1, 2048), "dtype": dtype,
                "act": rng.choice(("silu", "gelu", "gelu_tanh", "none"))}
        return case if op == "gated" else {**case, "out": rng.choice(("f32", "bf16")), "bias": rng.random() < 0.5}
    d = rng.choice((64, 128))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.randint(1, 8)
    if hq * d % 128:
        hq, hkv = 2 * hq, 2 * hkv
    mode = rng.choice(("even", "ragged", "mixed", "prompts"))
    batch = _log_int(rng, 1, 64)
    # the plain form holds every request's longest chunk against the longest cache
    most = 1 << 24
    hi = _log_int(rng, 16, min(8192, int(math.sqrt(most / batch)) if mode == "prompts" else 8192))
    new = 0 if mode == "prompts" else _log_int(rng, 1, max(1, min(hi, 2048 // batch, most // (batch * hi))))
    return {"op": op, "mode": mode, "batch": batch, "new": new, "pad": rng.randint(0, 5), "hq": hq, "hkv": hkv, "d": d, "dtype": dtype,
            "lo": rng.randint(1, max(1, hi // 2)), "hi": hi, "window": rng.choice((0, 0, 0, _log_int(rng, 1, hi)))}


# ------------------------------------------------------------------ what a case's requests look like

def _requests(case):
    """(length, new tokens) of every request, the longest among them; the same for every seed."""
    n = case["batch"]
    lens = [case["lo"] + int((case["hi"] - case["lo"] + 1) * ((i + 1) * 0.6180339887498949 % 1.0)) for i in range(n)]
    lens[n // 2] = case["hi"]
    if case["mode"] == "prompts":
        return [(x, x) for x in lens]
    if case["mode"] == "even":
        return [(x, min(x, case["new"])) for x in lens]
    if case["mode"] == "mixed":
        return [(x, min(x, case["new"] if i % 8 == 0 else 1)) for i, x in enumerate(lens)]
    return [(x, min(x, int((case["new"] + 1) * ((i + 1) * 0.7548776662466927 % 1.0)) if i != n // 2 else case["new"])) for i, x in enumerate(lens)]


def _page_bytes(case):
    return 2 * case["hkv"] * PAGE * case["d"], 2 * case["hkv"] * PAGE   # codes, scales


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 31)
    dt = DT[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEV) * scale

    s = {"case": case}
    if case["op"] != "chunk":
        n, k, rows = case["n"], case["k"], case["rows"]
        to = DT[case.get("out", case["dtype"])]
        s["x"] = normal(rows, k).to(dt)
        for name in ("", "_up") if case["op"] == "gated" else ("",):
            s["codes" + name] = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
            # weights of standard deviation about 0.02: blocks whose largest value lies in [1/32, 1/8)
            s["scales" + name] = torch.randint(120, 122, (n, k // 32), generator=g, device=DEV, dtype=torch.uint8)
        if case["op"] == "fused":
            s["residual"] = normal(rows, n).to(to)
            s["bias"] = normal(n, scale=0.5).to(to) if case["bias"] else None
        s["out"] = torch.zeros(rows, n, device=DEV, dtype=to)
        return s
    lens, new = zip(*_requests(case))
    pages = [-(-n // PAGE) for n in lens]
    width, total = max(pages), sum(pages)
    n_pages = total + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    where = torch.zeros(len(lens), width, dtype=torch.int64)
    at = 0
    for r, n in enumerate(pages):
        where[r, :n] = torch.arange(at, at + n)
        table[r, :n] = 0
        at += n
    s["table"] = torch.where(table.to(DEV) < 0, -1, perm[where.to(DEV)]).to(torch.int32)
    s["n_pages"] = n_pages
    # one layer's pool: codes of K [head][token][dim] and V [head][dim][token] of every page, then the scales of all pages
    codes, scales = (n_pages * b for b in _page_bytes(case))
    mem = torch.empty(codes + scales, device=DEV, dtype=torch.uint8)
    for lo in range(0, codes, 1 << 28):
        hi = min(codes, lo + (1 << 28))
        mem[lo:hi] = normal(hi - lo, scale=110.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    mem[codes:] = torch.randint(119, 122, (scales,), generator=g, device=DEV, dtype=torch.uint8)
    s["mem"], s["codes"], s["scales"] = mem, mem[:codes], mem[codes:]
    rows = sum(new) + case["pad"]
    s["q"] = normal(rows, case["hq"] * case["d"], scale=1.5).to(dt)
    s["n_tokens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    starts = [0]
    for c in new:
        starts.append(starts[-1] + c)
    s["row_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["most_new"] = max(new)
    s["out"] = torch.zeros(rows, case["hq"] * case["d"], device=DEV, dtype=dt)
    return s


# ------------------------------------------------------------------ the plain forms

def _plain_chunk(s):
    """Every request's rows, as many as the longest chunk has, against its pages, as many as the table is wide."""
    case = s["case"]
    hkv, d, batch, most = case["hkv"], case["d"], case["batch"], s["most_new"]
    group = case["hq"] // hkv
    table, n, starts = s["table"].long(), s["n_tokens"].long(), s["row_starts"].long()
    count = starts[1:] - starts[:-1]
    j = torch.arange(most, device=DEV)
    there = j < count[:, None]                                     # [batch, most]
    row = torch.where(there, starts[:-1, None] + j, 0)
    position = (n - count)[:, None] + j
    at = torch.arange(table.shape[1] * PAGE, device=DEV)
    seen = (at <= position[..., None]) & (table >= 0).repeat_interleave(PAGE, 1)[:, None]
    if case["window"]:
        seen &= at > position[..., None] - case["window"]
    seen = seen[:, None, :, None]                                  # [batch, 1, most, 1, tokens]
    page = table.clamp(min=0)
    codes = s["codes"].view(torch.float8_e4m3fn).view(s["n_pages"], 2, hkv, PAGE * d)
    powers = torch.exp2(s["scales"].view(s["n_pages"], 2, hkv, PAGE).float() - 127.0)
    k = codes[:, 0].float().view(-1, hkv, PAGE, d) * powers[:, 0, :, :, None]
    v = codes[:, 1].float().view(-1, hkv, d, PAGE) * powers[:, 1, :, None, :]
    k = k[page].permute(0, 2, 4, 1, 3).reshape(batch, hkv, d, -1)
    v = v[page].permute(0, 2, 1, 4, 3).reshape(batch, hkv, -1, d)
    q = (s["q"].float() * (1.0 / math.sqrt(d)))[row].view(batch, most, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(batch, hkv, most * group, d)
    score = torch.matmul(q, k).view(batch, hkv, most, group, -1)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True).view(batch, hkv, most * group, 1)
    out = torch.matmul(p.view(batch, hkv, most * group, -1), v) / torch.where(total > 0, total, 1.0)
    out = out.view(batch, hkv, most, group, d).permute(0, 2, 1, 3, 4).reshape(batch * most, -1).to(s["out"].dtype)
    r = torch.arange(s["out"].shape[0], device=DEV)
    of = (r[:, None] >= starts[1:]).sum(-1).clamp(max=batch - 1)
    mine = torch.where(r < starts[-1], of * most + r - starts[of], 0)
    s["out"].copy_(torch.where((r < starts[-1])[:, None], out[mine], s["out"]))
    return s["out"]


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _plain_values(codes, scales):
    n, half = codes.shape
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEV)
    code = torch.stack([codes & 15, codes >> 4], -1).view(n, half * 2).int()
    power = torch.ldexp(torch.ones((), device=DEV), scales.int() - 127)
    power = torch.where(scales == 255, math.nan, power)
    return (table[code].view(n, -1, 32) * power[..., None]).view(n, half * 2)


def _plain_act(x, act):
    if act == "silu":
        return x / (1.0 + torch.exp(-x))
    if act == "gelu":
        return 0.5 * x * torch.erfc(x * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return x / (1.0 + torch.exp(x * (1.0 + 0.044715 * x * x) * -2.0 * math.sqrt(2.0 / math.pi)))
    return x


def _plain_product(s):
    case = s["case"]
    x = s["x"].float()
    y = torch.matmul(x, _plain_values(s["codes"], s["scales"]).t())
    if case["op"] == "gated":
        y = _plain_act(y, case["act"]) * torch.matmul(x, _plain_values(s["codes_up"], s["scales_up"]).t())
    else:
        if s["bias"] is not None:
            y = y + s["bias"].float()
        y = _plain_act(y, case["act"]) + s["residual"].float()
    return y.to(s["out"].dtype)


# ------------------------------------------------------------------ one pass

def run(state):
    if own:
        return _own(state)
    return _plain_chunk(state) if state["case"]["op"] == "chunk" else _plain_product(state)


def _own(s):
    from paper_2603_02599_amd import binding as sun
    case = s["case"]
    act = {"none": sun.SUN_ACT_NONE, "silu": sun.SUN_ACT_SILU, "gelu": sun.SUN_ACT_GELU, "gelu_tanh": sun.SUN_ACT_GELU_TANH}[case.get("act", "none")]
    if case["op"] == "gated":
        if "workspace" not in s:
            s["workspace"] = torch.empty(sun.sun_mx4_gated_workspace_bytes(case["n"], case["k"], case["rows"]), dtype=torch.uint8, device=DEV)
        sun.sun_mx4_gated(s["codes"], s["scales"], s["codes_up"], s["scales_up"], s["x"], s["out"], s["workspace"], activation=act)
        return s["out"]
    if case["op"] == "fused":
        if "workspace" not in s:
            s["workspace"] = torch.empty(sun.sun_mx4_linear_workspace_bytes(case["n"], case["k"], case["rows"]), dtype=torch.uint8, device=DEV)
        sun.sun_mx4_linear_fused(s["codes"], s["scales"], s["x"], s["out"], s["workspace"], bias=s["bias"], activation=act, residual=s["residual"])
        return s["out"]
    if "pool" not in s:
        from paper_2603_02599_amd import workloads as wl
        cfg = sun.make_cfg(wl.Shape("case", 1, case["hq"] * case["d"], case["hq"], case["hkv"], case["d"], 128, 32), "f32")
        s["pool"] = sun.sun_kv8_pool_create(cfg, s["mem"])
        s["workspace"] = torch.empty(sun.sun_kv8_chunk_attention_workspace_bytes(cfg, s["table"].shape[0], s["q"].shape[0], s["table"].shape[1]), dtype=torch.uint8, device=DEV)
    sun.sun_kv8_chunk_attention(s["pool"], 0, s["q"], s["row_starts"], s["table"], s["n_tokens"], s["out"], s["workspace"], window=case["window"])
    return s["out"]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] != "chunk":
        n, k, rows = case["n"], case["k"], case["rows"]
        pair, to = (2, size) if case["op"] == "gated" else (1, SIZE[case["out"]])
        return {"bytes": pair * n * k * (0.5 + 1 / 32) + rows * (k * size + n * to * (1 if pair == 2 else 2)) + (n * to if case.get("bias") else 0), "flops": 2 * pair * n * k * rows}
    hq, hkv, d, window = case["hq"], case["hkv"], case["d"], case["window"]
    read = pairs = rows = 0
    for n, c in _requests(case):
        if not c:
            continue
        rows += c
        read += min(n, window + c - 1) if window else n
        # row j of c sees n - c + 1 + j positions, at most the window
        full = sum(min(n - c + 1 + j, window) for j in range(c)) if window else c * (n - c + 1) + c * (c - 1) // 2
        pairs += full
    return {"bytes": read * hkv * 2 * (d + 1) + read / PAGE * 4 + rows * 2 * hq * d * size + case["batch"] * 8, "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------ the same in 64 bits

def _exact_chunk(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    numbers = torch.tensor([(-1.0) ** (b >> 7) * ((b & 7) / 8.0 * 2.0 ** -6 if not (b >> 3 & 15) else (1 + (b & 7) / 8.0) * 2.0 ** ((b >> 3 & 15) - 7)) for b in range(256)],
                           dtype=torch.float64, device=DEV)
    codes = s["codes"].view(s["n_pages"], 2, hkv, PAGE * d)
    power = torch.pow(2.0, s["scales"].view(s["n_pages"], 2, hkv, PAGE).double() - 127)
    out = s["out"].double().view(-1, hq, d)
    q = s["q"].double().view(-1, hq, d)
    row = 0
    for i, (n, c) in enumerate(_requests(case)):
        if not c:
            continue
        page = s["table"][i, :-(-n // PAGE)].long()
        position = torch.arange(n - c, n, device=DEV)[:, None]
        token = torch.arange(n, device=DEV)
        hidden = (token > position) | (token + case["window"] <= position) if case["window"] else token > position
        for h in range(hkv):
            k = (numbers[codes[page, 0, h].int()].view(-1, PAGE, d) * power[page, 0, h, :, None]).view(-1, d)[:n]
            v = (numbers[codes[page, 1, h].int()].view(-1, d, PAGE) * power[page, 1, h, None, :]).transpose(1, 2).reshape(-1, d)[:n]
            kt = k.t().contiguous()
            for e in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                w = torch.matmul(q[row:row + c, e].contiguous(), kt) / math.sqrt(d)
                out[row:row + c, e] = torch.matmul(torch.softmax(w.masked_fill_(hidden, -math.inf), -1), v)
        row += c
    return out.view(-1, hq * d)


def _exact_weights(codes, scales):
    numbers = torch.tensor([(-1.0) ** (c >> 3) * ((c & 1) / 2.0 if not (c >> 1 & 3) else (1 + (c & 1) / 2.0) * 2.0 ** ((c >> 1 & 3) - 1)) for c in range(16)], dtype=torch.float64, device=DEV)
    w = torch.empty(codes.shape[0], codes.shape[1] * 2, dtype=torch.float64, device=DEV)
    w[:, 0::2], w[:, 1::2] = numbers[(codes % 16).int()], numbers[(codes // 16).int()]
    return w * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "chunk":
        return _exact_chunk(s)
    act = {"none": lambda y: y, "silu": lambda y: y * torch.sigmoid(y), "gelu": lambda y: y * (1.0 + torch.erf(y / math.sqrt(2.0))) / 2.0,
           "gelu_tanh": lambda y: y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))) / 2.0}[case["act"]]
    x = s["x"].double()
    y = torch.matmul(x, _exact_weights(s["codes"], s["scales"]).t())
    if case["op"] == "gated":
        return act(y) * torch.matmul(x, _exact_weights(s["codes_up"], s["scales_up"]).t())
    return act(y if s["bias"] is None else y + s["bias"].double()) + s["residual"].double()
