"""The operators around a decode worker's 8-bit cache and its microscaled 4-bit weights, as cases that can be timed and compared:
keys and values appended to the cache with the rotation on the way, attention of one new token over it, quantisation to (and values of) the
microscaled format, and the product with weights held in it.

A case is a dict of plain values:
  op "append":    `rows` rows of `requests` requests, `pad` of them padding; one row per request ("decode") or prompts of uneven lengths
  op "attention": one new token of `batch` requests with lengths in [lo, hi], `window` positions of each (0: all)
  op "quantize":  a matrix [n, k] into the format and its values back
  op "linear":    `rows` rows through a matrix [n, k] in the format
Heads are `hq` query heads over `hkv` KV heads of `d` dims; `dtype` is "f32" or "bf16".  Sizes are the repository's own shapes (8B, 14B, small, tiny).

`own` false: the plain forms, elementary torch operations in 32 bits (in 64 where a value is rounded to few bits behind it).  `own` true: the
library's calls.  exact() has the same results in 64 bits, written apart from the plain forms."""
import math

import torch

own = False

PAGE = 16
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
DEV = "cuda:0"
EPS = 1e-6


def listed():
    return [
        # a decode step of a medium batch, 8B heads
        {"name": "append_8b_b64_bf16", "op": "append", "mode": "decode", "rows": 64, "pad": 0, "requests": 64, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "norm": False, "scaled": True, "base": 500000.0, "lo": 512, "hi": 4096},
        # uneven prompts of one prefill batch, padded; 14B heads with head norms
        {"name": "append_14b_prompts_4096_f32", "op": "append", "mode": "prompts", "rows": 4096, "pad": 6, "requests": 5, "hq": 40, "hkv": 8, "d": 128, "dtype": "f32", "norm": True, "scaled": False, "base": 1000000.0, "lo": 0, "hi": 300},
        # the smallest call: launches and latency are all there is
        {"name": "attention_tiny_b8_f32", "op": "attention", "batch": 8, "hq": 4, "hkv": 2, "d": 64, "dtype": "f32", "lo": 16, "hi": 128, "window": 0},
        # one user, one long conversation: the length has to be split for the chip to be filled
        {"name": "attention_8b_b1_bf16", "op": "attention", "batch": 1, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "lo": 8191, "hi": 8191, "window": 0},
        # a full batch with a sliding window, fp32 activations
        {"name": "attention_8b_b256_window_f32", "op": "attention", "batch": 256, "hq": 32, "hkv": 8, "d": 128, "dtype": "f32", "lo": 1, "hi": 4096, "window": 1500},
        # long contexts, five query heads per KV head: the cache is all there is
        {"name": "attention_14b_b24_long_bf16", "op": "attention", "batch": 24, "hq": 40, "hkv": 8, "d": 128, "dtype": "bf16", "lo": 2048, "hi": 32768, "window": 0},
        # a small model's q/k/v matrix
        {"name": "quantize_1024x512_f32", "op": "quantize", "n": 1024, "k": 512, "dtype": "f32"},
        # the gate/up pair of the 8B shape
        {"name": "quantize_28672x4096_bf16", "op": "quantize", "n": 28672, "k": 4096, "dtype": "bf16"},
        # one user: q/k/v of the 8B shape, the weights are all there is to read
        {"name": "linear_6144x4096_1_bf16", "op": "linear", "n": 6144, "k": 4096, "rows": 1, "dtype": "bf16"},
        # the benchmark's default batch through gate/up
        {"name": "linear_28672x4096_64_bf16", "op": "linear", "n": 28672, "k": 4096, "rows": 64, "dtype": "bf16"},
        # a ragged batch through the 14B shape's down projection, fp32 activations
        {"name": "linear_5120x13824_150_f32", "op": "linear", "n": 5120, "k": 13824, "rows": 150, "dtype": "f32"},
        # a prefill block through gate/up: matrix cores
        {"name": "linear_28672x4096_2048_bf16", "op": "linear", "n": 28672, "k": 4096, "rows": 2048, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "quantize", "linear", "linear"))
    dtype = rng.choice(("f32", "bf16"))
    if op in ("append", "attention"):
        d = rng.choice((64, 128))
        hkv = rng.choice((1, 2, 4, 8))
        hq = hkv * rng.randint(1, 8)
        if hq * d % 128:
            hq, hkv = 2 * hq, 2 * hkv
    if op == "append":
        mode = rng.choice(("decode", "prompts"))
        rows = _log_int(rng, 1, 256) if mode == "decode" else _log_int(rng, 8, 2500)
        requests = rows if mode == "decode" else rng.randint(1, 6)
        return {"op": op, "mode": mode, "rows": rows, "pad": rng.randint(0, min(rows - 1, 5)), "requests": requests, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype,
                "norm": rng.random() < 0.5, "scaled": rng.random() < 0.5, "base": rng.choice((10000.0, 500000.0, 1000000.0)), "lo": rng.randint(0, 64), "hi": _log_int(rng, 64, 4096)}
    if op == "attention":
        batch = _log_int(rng, 1, 256)
        hi = _log_int(rng, 2, min(32768, 400000 // batch))
        return {"op": op, "batch": batch, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "lo": rng.randint(0, hi // 2), "hi": hi,
                "window": rng.choice((0, 0, 0, _log_int(rng, 1, hi)))}
    if op == "quantize":
        return {"op": op, "n": _log_int(rng, 1, 20000), "k": 32 * _log_int(rng, 1, 160), "dtype": dtype}
    return {"op": op, "n": _log_int(rng, 17, 20000), "k": 32 * _log_int(rng, 2, 160), "rows": _log_int(rng, 1, 2048), "dtype": dtype}


# ------------------------------------------------------------------ what a case's requests look like

def _lens(case):
    """Uneven lengths in [lo, hi], the longest among them; the same for every seed."""
    n = case["batch"] if case["op"] == "attention" else case["requests"]
    at = [case["lo"] + int((case["hi"] - case["lo"] + 1) * ((i + 1) * 0.6180339887498949 % 1.0)) for i in range(n)]
    at[n // 2] = case["hi"]
    return at


def _new_rows(case):
    """(position, request) of every row of an append; position -1: padding."""
    lens, live = _lens(case), case["rows"] - case["pad"]
    if case["mode"] == "decode":
        rows = [(lens[i], i) for i in range(live)]
    else:
        n, rows, left = case["requests"], [], live
        for r in range(n):
            count = left if r == n - 1 else min(left, live * (r + 1) * 2 // (n * (n + 1)) + r % 3)
            rows += [(lens[r] + t, r) for t in range(count)]
            left -= count
    return rows + [(-1, 0)] * case["pad"]


def _positions_needed(case):
    """Positions that each request's table has pages for."""
    if case["op"] == "attention":
        return _lens(case)
    need = [1] * case["requests"]
    for p, r in _new_rows(case):
        need[r] = max(need[r], p + 1)
    return need


def _page_bytes(case):
    return 2 * case["hkv"] * PAGE * case["d"], 2 * case["hkv"] * PAGE   # codes, scales


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    dt = DT[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device=DEV) * scale

    s = {"case": case}
    if case["op"] == "quantize":
        s["x"] = normal(case["n"], case["k"], scale=0.02).to(dt)
        return s
    if case["op"] == "linear":
        n, k = case["n"], case["k"]
        s["x"] = normal(case["rows"], k).to(dt)
        s["codes"] = torch.randint(0, 256, (n, k // 2), generator=g, device=DEV, dtype=torch.uint8)
        # weights of standard deviation about 0.02: blocks whose largest value lies in [1/32, 1/8)
        s["scales"] = torch.randint(120, 122, (n, k // 32), generator=g, device=DEV, dtype=torch.uint8)
        s["out"] = torch.zeros(case["rows"], n, device=DEV, dtype=dt)
        return s
    need = _positions_needed(case)
    pages = [-(-n // PAGE) for n in need]
    width, total = max(max(pages), 1), max(sum(pages), 1)
    n_pages = total + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(need), width), -1, dtype=torch.int32)
    where = torch.zeros(len(need), width, dtype=torch.int64)
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
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "attention":
        s["q"] = normal(case["batch"], hq * d, scale=1.5).to(dt)
        s["n_tokens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEV)
        s["out"] = torch.zeros(case["batch"], hq * d, device=DEV, dtype=dt)
        return s
    rows = _new_rows(case)
    s["positions"] = torch.tensor([p for p, _ in rows], dtype=torch.int32, device=DEV)
    s["requests"] = torch.tensor([r for _, r in rows], dtype=torch.int32, device=DEV)
    # q, k and v side by side, as one projection leaves them
    qkv = normal(len(rows), (hq + 2 * hkv) * d).to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :hq * d], qkv[:, hq * d:(hq + hkv) * d], qkv[:, (hq + hkv) * d:]
    s["q_norm"] = (1.0 + normal(d, scale=0.1)).to(dt) if case["norm"] else None
    s["k_norm"] = (1.0 + normal(d, scale=0.1)).to(dt) if case["norm"] else None
    s["q_out"] = torch.zeros(len(rows), hq * d, device=DEV, dtype=dt)
    return s


# ------------------------------------------------------------------ the plain forms

def _thetas(case):
    """Rotation frequencies in 64 bits, rescaled by wavelength where the case says so."""
    j = torch.arange(case["d"] // 2, dtype=torch.float64, device=DEV)
    theta = torch.exp(j * (-2.0 * math.log(case["base"]) / case["d"]))
    if not case["scaled"]:
        return theta
    factor, low, high, orig = 8.0, 1.0, 4.0, 8192.0
    wave = 2.0 * math.pi / theta
    smooth = (orig / wave - low) / (high - low)
    mixed = (1.0 - smooth) * theta / factor + smooth * theta
    return torch.where(wave > orig / low, theta / factor, torch.where(wave >= orig / high, mixed, theta))


def _to_e4m3(y):
    """Codes and scale bytes of the vectors along the last axis (fp32)."""
    top = torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y)).amax(-1)
    m, x = torch.frexp(top)
    e = torch.where(top > 0, x - 9 + (m > 0.875), -100).clamp(min=-100)
    return torch.ldexp(y, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _plain_append(s):
    case = s["case"]
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], case["rows"]
    pos = s["positions"].long()
    live = (pos >= 0)
    ang = pos.clamp(min=0).double()[:, None] * _thetas(case)
    cos, sin = (f(ang).float().double()[:, None, :] for f in (torch.cos, torch.sin))

    def rotated(x, heads, gain):
        x = x.reshape(n, heads, d).double()
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + float(torch.tensor(EPS, dtype=torch.float32))) * gain.double()
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).float()

    q = rotated(s["q"], hq, s["q_norm"]).to(s["q_out"].dtype).reshape(n, hq * d)
    s["q_out"].copy_(torch.where(live[:, None], q, s["q_out"]))
    page = s["table"].long()[s["requests"].long(), pos.clamp(min=0) // PAGE]
    keep = live & (page >= 0)
    page, slot = page[keep], (pos % PAGE)[keep]
    codes = s["codes"].view(s["n_pages"], 2, hkv, PAGE * d)
    scales = s["scales"].view(s["n_pages"], 2, hkv, PAGE)
    kc, ks = _to_e4m3(rotated(s["k"], hkv, s["k_norm"])[keep])
    vc, vs = _to_e4m3(s["v"].reshape(n, hkv, d).float()[keep])
    codes[:, 0].view(-1, hkv, PAGE, d)[page, :, slot] = kc
    codes[:, 1].view(-1, hkv, d, PAGE)[page, :, :, slot] = vc
    scales[page, 0, :, slot] = ks
    scales[page, 1, :, slot] = vs
    return s["q_out"]


def _plain_attention(s):
    case = s["case"]
    hkv, d, batch = case["hkv"], case["d"], case["batch"]
    group = case["hq"] // hkv
    n = s["n_tokens"].long()
    table = s["table"].long()
    at = torch.arange(table.shape[1] * PAGE, device=DEV)
    seen = (at < n[:, None]) & (table >= 0).repeat_interleave(PAGE, 1)
    if case["window"]:
        seen &= at >= n[:, None] - case["window"]
    page = table.clamp(min=0)
    codes = s["codes"].view(torch.float8_e4m3fn).view(s["n_pages"], 2, hkv, PAGE * d)
    powers = torch.exp2(s["scales"].view(s["n_pages"], 2, hkv, PAGE).float() - 127.0)
    q = s["q"].float().reshape(batch, hkv, group, d) * (1.0 / math.sqrt(d))
    k = codes[:, 0].float().view(-1, hkv, PAGE, d) * powers[:, 0, :, :, None]
    v = codes[:, 1].float().view(-1, hkv, d, PAGE) * powers[:, 1, :, None, :]
    k = k[page].permute(0, 2, 4, 1, 3).reshape(batch, hkv, d, -1)
    v = v[page].permute(0, 2, 1, 4, 3).reshape(batch, hkv, -1, d)
    score = torch.where(seen[:, None, None], torch.matmul(q, k), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen[:, None, None], torch.exp(score - torch.where(torch.isfinite(top), top, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.reshape(batch, -1).to(s["q"].dtype)


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _plain_quantize(x):
    """4-bit codes (two a byte, even column low) and scale bytes of a matrix, 32 columns a block."""
    n, k = x.shape
    x = x.float().view(n, k // 32, 32)
    top = x.abs().amax(-1)
    _, e = torch.frexp(top)
    e = torch.where(top > 0, e - 3, -127).clamp(min=-127)
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for edge in (0.75, 1.25, 1.75, 2.5, 3.5, 5.0):   # halfway values go to the even code
        code += (a >= edge) if edge in (0.75, 1.75, 3.5) else (a > edge)
    code |= torch.signbit(y).to(torch.uint8) << 3
    bad = ~torch.isfinite(top)
    code = torch.where(bad[..., None], 0, code).view(n, k)
    return code[:, 0::2] | code[:, 1::2] << 4, torch.where(bad, 255, e + 127).to(torch.uint8)


def _plain_values(codes, scales):
    n, half = codes.shape
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEV)
    code = torch.stack([codes & 15, codes >> 4], -1).view(n, half * 2).int()
    power = torch.ldexp(torch.ones((), device=DEV), scales.int() - 127)
    power = torch.where(scales == 255, math.nan, power)
    return (table[code].view(n, -1, 32) * power[..., None]).view(n, half * 2)


# ------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    if own:
        return _own(state)
    if case["op"] == "append":
        return {"q": _plain_append(state), "codes": state["codes"].view(torch.float8_e4m3fn), "scales": state["scales"]}
    if case["op"] == "attention":
        return _plain_attention(state)
    if case["op"] == "quantize":
        return _plain_values(*_plain_quantize(state["x"])).to(state["x"].dtype)
    return torch.matmul(state["x"].float(), _plain_values(state["codes"], state["scales"]).t()).to(state["x"].dtype)


def _own(s):
    from paper_2603_02599_amd import binding as sun
    case = s["case"]
    if case["op"] == "quantize":
        codes, scales = sun.sun_mx4_quantize(s["x"])
        return sun.sun_mx4_dequantize(codes, scales, s["x"].dtype)
    if case["op"] == "linear":
        if "workspace" not in s:
            s["workspace"] = torch.empty(max(sun.sun_mx4_linear_workspace_bytes(case["n"], case["k"], case["rows"]), 256), dtype=torch.uint8, device=DEV)
        sun.sun_mx4_linear(s["codes"], s["scales"], s["x"], s["out"], s["workspace"])
        return s["out"]
    if "pool" not in s:
        from paper_2603_02599_amd import workloads as wl
        shape = wl.Shape("case", 1, case["hq"] * case["d"], case["hq"], case["hkv"], case["d"], 128, 32, rms_eps=EPS, rope_base=case.get("base", 10000.0),
                         qk_norm=case.get("norm", False), rope_scaling=(8.0, 1.0, 4.0, 8192) if case.get("scaled") else None)
        s["cfg"] = sun.make_cfg(shape, "f32")
        s["pool"] = sun.sun_kv8_pool_create(s["cfg"], s["mem"])
    if case["op"] == "append":
        sun.sun_kv8_append(s["pool"], 0, s["q"], s["k"], s["v"], s["positions"], s["requests"], s["table"], s["q_out"], s["q_norm"], s["k_norm"])
        return {"q": s["q_out"], "codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"]}
    if "workspace" not in s:
        s["workspace"] = torch.empty(sun.sun_kv8_attention_workspace_bytes(s["cfg"], *s["table"].shape), dtype=torch.uint8, device=DEV)
    sun.sun_kv8_attention(s["pool"], 0, s["q"], s["table"], s["n_tokens"], s["out"], s["workspace"], window=case["window"])
    return s["out"]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "quantize":   # the matrix in, codes and scales out, values out
        n = case["n"] * case["k"]
        return {"bytes": n * (2 * SIZE[case["dtype"]] + 0.5 + 1 / 32), "flops": 2 * n}
    if case["op"] == "linear":
        n, k, rows = case["n"], case["k"], case["rows"]
        return {"bytes": n * k * (0.5 + 1 / 32) + rows * (n + k) * SIZE[case["dtype"]], "flops": 2 * n * k * rows}
    hq, hkv, d, size = case["hq"], case["hkv"], case["d"], SIZE[case["dtype"]]
    if case["op"] == "append":
        rows = case["rows"] - case["pad"]
        return {"bytes": rows * ((2 * hq + 2 * hkv) * d * size + 2 * hkv * (d + 1) + 12), "flops": rows * (hq + hkv) * d * 3}
    tokens = sum(min(n, case["window"]) if case["window"] else n for n in _lens(case))
    return {"bytes": tokens * hkv * 2 * (d + 1) + tokens / PAGE * 4 + case["batch"] * (2 * hq * d * size + 4), "flops": 4 * tokens * hq * d}


# ------------------------------------------------------------------ the same in 64 bits

def _grid(y, mantissa, least):
    """y rounded to `mantissa` bits behind the leading one, half to even, spaced as at 2^least below it."""
    _, x = torch.frexp(y)
    step = torch.pow(2.0, (x.double() - 1).clamp(min=least) - mantissa)
    return torch.round(y / step) * step   # torch.round takes halves to even


def _exact_entry(y):
    """e4m3 numbers and scale bytes of one vector each along the last axis (64 bits)."""
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-40) / 448.0))
    e = torch.where(top <= 448.0 * torch.pow(2.0, e - 1), e - 1, e)
    e = torch.where(top > 448.0 * torch.pow(2.0, e), e + 1, e).clamp(min=-100)
    e = torch.where(top == 0, torch.full_like(e, -100.0), e)
    return _grid(y / torch.pow(2.0, e), 3, -6), (e[..., 0] + 127)


def _exact_append(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    theta = [case["base"] ** (-2.0 * j / d) for j in range(d // 2)]
    if case["scaled"]:
        for j, t in enumerate(theta):
            turns = 8192.0 * t / (2.0 * math.pi)
            share = min(1.0, max(0.0, (turns - 1.0) / 3.0))
            theta[j] = t / 8.0 if turns < 1.0 else t if turns > 4.0 else t / 8.0 * (1.0 - share) + t * share
    theta = torch.tensor(theta, dtype=torch.float64, device=DEV)
    pos = s["positions"].double()
    c, z = torch.cos(pos[:, None] * theta).float().double(), torch.sin(pos[:, None] * theta).float().double()

    def turn(x, heads, gain):
        x = x.double().reshape(-1, heads, d)
        if gain is not None:
            eps = float(torch.tensor(EPS, dtype=torch.float32))
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + eps) * gain.double()
        w = torch.complex(x[..., :d // 2], x[..., d // 2:]) * torch.complex(c, z)[:, None]
        return torch.cat([w.real, w.imag], -1)

    live = s["positions"] >= 0
    q = turn(s["q"], hq, s["q_norm"]).reshape(-1, hq * d)
    q = torch.where(live[:, None], q, s["q_out"].double())
    codes = s["codes"].view(torch.float8_e4m3fn).float().double()
    scales = s["scales"].double()
    kc, ks = _exact_entry(turn(s["k"], hkv, s["k_norm"]).float().double())
    vc, vs = _exact_entry(s["v"].double().reshape(-1, hkv, d))
    r = torch.nonzero(live)[:, 0]
    p = s["positions"].long()[r]
    page, slot = s["table"].long()[s["requests"].long()[r], p // PAGE], p % PAGE
    h, t = torch.arange(hkv, device=DEV), torch.arange(d, device=DEV)
    block = (page[:, None] * 2 * hkv + h)[..., None]
    codes[block * PAGE * d + slot[:, None, None] * d + t] = kc[r]
    codes[(block + hkv) * PAGE * d + t * PAGE + slot[:, None, None]] = vc[r]
    scales[block[..., 0] * PAGE + slot[:, None]] = ks[r]
    scales[(block[..., 0] + hkv) * PAGE + slot[:, None]] = vs[r]
    return {"q": q, "codes": codes, "scales": scales.to(torch.int64)}


def _exact_attention(s):
    case = s["case"]
    hkv, d = case["hkv"], case["d"]
    numbers = torch.tensor([(-1.0) ** (b >> 7) * ((b & 7) / 8.0 * 2.0 ** -6 if not (b >> 3 & 15) else (1 + (b & 7) / 8.0) * 2.0 ** ((b >> 3 & 15) - 7)) for b in range(256)],
                           dtype=torch.float64, device=DEV)
    codes = s["codes"].view(s["n_pages"], 2, hkv, PAGE * d)
    power = torch.pow(2.0, s["scales"].view(s["n_pages"], 2, hkv, PAGE).double() - 127)
    out = torch.zeros(case["batch"], hkv, case["hq"] // hkv, d, dtype=torch.float64, device=DEV)
    q = s["q"].double().view(case["batch"], hkv, -1, d)
    for i, n in enumerate(_lens(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == first:
            continue
        page = s["table"][i, :-(-n // PAGE)].long()
        got, by = numbers[codes[page].int()], power[page]
        k = (got[:, 0].view(-1, hkv, PAGE, d) * by[:, 0, ..., None]).transpose(0, 1).reshape(hkv, -1, d)[:, first:n]
        v = (got[:, 1].view(-1, hkv, d, PAGE) * by[:, 1, :, None]).permute(1, 0, 3, 2).reshape(hkv, -1, d)[:, first:n]
        w = torch.softmax(torch.matmul(q[i], k.transpose(1, 2).contiguous()) / math.sqrt(d), -1)
        out[i] = torch.matmul(w, v.contiguous())
    return out.view(case["batch"], -1)


def _exact_quantize(x):
    x = x.double().view(x.shape[0], -1, 32)
    top = x.abs().amax(-1, keepdim=True)
    _, e = torch.frexp(top)
    power = torch.pow(2.0, (e.double() - 3).clamp(min=-127))
    return (_grid(x / power, 1, 0).clamp(-6, 6) * power).view(x.shape[0], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "attention":
        return _exact_attention(s)
    if case["op"] == "quantize":
        return _exact_quantize(s["x"])
    numbers = torch.tensor([(-1.0) ** (c >> 3) * ((c & 1) / 2.0 if not (c >> 1 & 3) else (1 + (c & 1) / 2.0) * 2.0 ** ((c >> 1 & 3) - 1)) for c in range(16)], dtype=torch.float64, device=DEV)
    w = torch.empty(case["n"], case["k"], dtype=torch.float64, device=DEV)
    w[:, 0::2], w[:, 1::2] = numbers[(s["codes"] % 16).int()], numbers[(s["codes"] // 16).int()]
    w *= torch.pow(2.0, s["scales"].double() - 127).repeat_interleave(32, 1)
    return torch.matmul(s["x"].double(), w.t())
