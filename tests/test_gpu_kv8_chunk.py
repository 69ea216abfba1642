"""Attention of a chunk of new tokens over the 8-bit cache on the GPU against its 64-bit plain form: chunk lengths from none to whole prompts, windows,
pages and values that are not there, parts of long caches, graphs and streams."""
import math

import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2603_02599_amd import binding as sun
from test_gpu_kv8 import DEV, DT, HEADS, Cache, host, i32, make_shape

pytestmark = pytest.mark.gpu


def starts_of(counts, first=0):
    return np.concatenate([[first], first + np.cumsum(counts)]).astype(np.int64)


def queries(shape, rows, dtype, seed=3, scale=1.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(rows, shape.n_q_heads * shape.head_dim, generator=g, device=DEV) * scale).to(DT[dtype])


def attend(cache, layer, q, starts, lens, window=0, out=None, flags=0, stream=None, table=None):
    table = cache.dev_table if table is None else table
    out = torch.full_like(q, 33.0) if out is None else out
    nbytes = sun.sun_kv8_chunk_attention_workspace_bytes(cache.cfg, table.shape[0], q.shape[0], table.shape[1])
    ws = torch.full((nbytes + 256,), 0xff, dtype=torch.uint8, device=DEV)
    sun.sun_kv8_chunk_attention(cache.pool, layer, q, i32(starts), table, i32(lens), out, ws[:nbytes], window=window, flags=flags, stream=stream)
    torch.cuda.synchronize()
    assert (ws[nbytes:] == 0xff).all(), "written behind the workspace"
    return out


def reference(q, views, layer, table, n, window, shape, n_pages):
    """One request: q [c, Hq, d] of its last c positions -> out and, per element, sum_t p_t |v_t| and the scale of the scores' error."""
    c, hq, d = q.shape
    hkv = shape.n_kv_heads
    k_codes, v_codes, k_scales, v_scales = (v[layer] for v in views)
    out, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros((c, hq))
    t = np.array([t for t in range(max(0, n - c - window + 1) if window else 0, n) if 0 <= table[t // 16] < n_pages], dtype=np.int64)
    if not t.size:
        return out, mass, reach
    pos = np.arange(n - c, n)[:, None]
    seen = (t <= pos) & ((t > pos - window) if window else True)
    any_seen = seen.any(1)
    page, slot = table[t // 16], t % 16
    for h in range(hkv):
        k = R.E4M3[k_codes[page, h, slot]] * np.exp2(k_scales[page, h, slot].astype(np.float64) - 127)[:, None]
        v = R.E4M3[v_codes[page, h, :, slot]] * np.exp2(v_scales[page, h, slot].astype(np.float64) - 127)[:, None]
        for i in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
            with np.errstate(invalid="ignore"):
                s = np.where(seen, q[:, i] @ k.T / math.sqrt(d), -np.inf)
                top = s.max(1, keepdims=True)
                p = np.exp(s - np.where(any_seen[:, None], top, 0.0))
                p = np.where(seen, p / np.where(any_seen[:, None], p.sum(1, keepdims=True), 1.0), 0.0)
            clean = np.isfinite(v).all(1)
            out[:, i], mass[:, i] = p[:, clean] @ v[clean], p[:, clean] @ np.abs(v[clean])
            for j in np.nonzero(~clean)[0]:
                out[:, i] += np.where(seen[:, j:j + 1], p[:, j:j + 1] * v[j], 0.0)
            reach[:, i] = np.where(seen, np.abs(q[:, i]) @ np.abs(k).T, 0.0).max(1) / math.sqrt(d)
    return out, mass, reach


def bound(ref, mass, reach, n, d, dtype):
    """Scores: d products summed in 32 bits (three planes of a 32-bit query: 3 d) and four roundings behind them; weights e^s off by twice that, an exponential
    good to 2^-22, rounded to bf16 (half a step: 2^-8) or carried in 24 bits; two sums over n weights in 32 bits, three times as many products for three
    planes; the output's own rounding."""
    planes = 1 if dtype == "bf16" else 3
    score = reach[..., None] * (planes * d + 4) * 2.0 ** -24
    weight = 2 * score + 2.0 ** -21 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
    return mass * (weight + (planes + 1) * (n + 8) * 2.0 ** -24) + np.abs(ref) * R.HALF[dtype] * 1.01 + 1e-37


def check(cache, layer, counts, lens, dtype, window=0, pad=0, first=0, seed=3, scale=1.5, change=None):
    s = cache.shape
    starts = starts_of(counts, first)
    q = queries(s, int(starts[-1]) + pad, dtype, seed, scale)
    if change is not None:
        change(q)
    before = cache.mem.clone()
    out = attend(cache, layer, q, starts, lens, window)
    assert torch.equal(before, cache.mem)
    got, views, qh = host(out).reshape(-1, s.n_q_heads, s.head_dim), cache.views(), host(q).reshape(-1, s.n_q_heads, s.head_dim)
    assert (got[:first] == 33).all() and (got[starts[-1]:] == 33).all(), "rows of no request were written"
    for i, n in enumerate(lens):
        if not counts[i]:
            continue
        n = min(max(n, 0), 16 * cache.table.shape[1])
        rows = slice(starts[i], starts[i + 1])
        ref, mass, reach = reference(qh[rows], views, layer, cache.table[i], n, window, s, cache.n_pages)
        over = np.abs(got[rows] - ref) / bound(ref, mass, reach, n, s.head_dim, dtype)
        nan = np.isnan(ref)
        assert np.array_equal(nan, np.isnan(got[rows])), f"request {i}: not-a-numbers elsewhere"
        assert (over[~nan] <= 1).all(), f"request {i}, {counts[i]} of {n} tokens: {over[~nan].max(initial=0):.2f} of the bound"
    return q, out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d", HEADS)
def test_uneven_chunks(hq, hkv, d, dtype):
    """From one token to a whole prompt, with requests that have nothing new between them, and rows in front of and behind all of them."""
    lens = [1, 16, 33, 200, 64, 300, 5, 129, 1000]
    counts = [1, 4, 33, 0, 17, 150, 5, 1, 40]
    cache = Cache(make_shape(hq, hkv, d), lens)
    cache.fill(1, lens)
    check(cache, 1, counts, lens, dtype, pad=3, first=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts, lens", [([1], [1]), ([2], [2]), ([31], [31]), ([32], [32]), ([33], [47]), ([128], [128]), ([129], [129]), ([1], [5000]), ([8], [5000]),
                                          ([100], [4099]), ([500], [500]), ([0, 1], [0, 65])])
@pytest.mark.parametrize("hq, hkv, d", [(4, 1, 64), (2, 2, 128), (7, 1, 128)])
def test_one_request(hq, hkv, d, counts, lens, dtype):
    cache = Cache(make_shape(hq, hkv, d), lens)
    cache.fill(0, lens)
    check(cache, 0, counts, lens, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 2, 16, 17, 64, 100, 5000])
def test_window(window, dtype):
    """Pages that no row sees are not read: their table entries are -1 and the slots hold not-a-numbers."""
    lens, counts = [1, 40, 130, 700, 2000], [1, 7, 130, 3, 90]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    for r, (n, c) in enumerate(zip(lens, counts)):
        cache.table[r, :max(0, n - c - window + 1) // 16] = -1
    cache.dev_table = i32(cache.table)
    check(cache, 0, counts, lens, dtype, window=window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lost_pages_and_counts_beyond(dtype):
    """Entries outside the pool: their tokens do not count; a row that sees none gets zeros, and so do rows in front of position 0."""
    lens, counts = [100, 700, 64, 200, 3, 50], [60, 20, 10, 200, 3, 50]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    cache.table[0, 2] = -1
    cache.table[1, :30] = cache.n_pages
    cache.table[2, :] = -3
    cache.table[3, 0] = 2 ** 31 - 1
    cache.dev_table = i32(cache.table)
    _, out = check(cache, 0, counts, lens, dtype)
    assert (out[80:90] == 0).all() and (out[90:106] == 0).all()
    check(cache, 0, counts, [100, 12, 4, 100, -7, 0], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_not_a_numbers_stay_where_they_belong(d, dtype):
    """A key or value that is not a number reaches the rows that see it, a value in its dim alone, and no row in front of it."""
    lens, counts = [300, 260, 40], [300, 9, 40]
    cache = Cache(make_shape(4, 2, d), lens)
    cache.fill(0, lens)
    lay, starts = cache.lay, starts_of(counts)
    q = queries(cache.shape, int(starts[-1]), dtype)
    clean = attend(cache, 0, q, starts, lens).view(-1, 4, d).clone()
    bad = torch.zeros_like(clean, dtype=torch.bool)
    for r, t, head, dim in ((0, 150, 1, 9), (0, 77, 0, 11), (1, 255, 0, 3), (2, 5, 1, 60), (2, 6, 1, 60)):
        cache.mem[lay.v_off + int(cache.table[r, t // 16]) * lay.v_page + head * lay.v_head + t % 16 * lay.v_token + dim * lay.v_dim] = 127 + 128 * (t & 1)
        bad[starts[r] + max(0, t - lens[r] + counts[r]):starts[r + 1], 2 * head:2 * head + 2, dim] = True
    r, t, head = 2, 33, 0
    cache.mem[lay.k_off + int(cache.table[r, t // 16]) * lay.k_page + head * lay.k_head + t % 16 * lay.k_token + 7] = 255
    bad[starts[r] + t:starts[r + 1], :2] = True
    got = attend(cache, 0, q, starts, lens).view(-1, 4, d)
    assert torch.equal(torch.isnan(got), bad)
    assert torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens, counts", [([300, 40, 5000], [2, 40, 3]), ([300, 400], [300, 70])])
def test_queries_that_are_not_numbers(lens, counts, dtype):
    """A head whose query holds an infinity or a not-a-number is not-a-number where it sees a token, and nobody else is."""
    cache = Cache(make_shape(4, 2, 128), lens)
    cache.fill(0, lens)
    starts = starts_of(counts)
    q = queries(cache.shape, int(starts[-1]), dtype)
    clean = attend(cache, 0, q, starts, lens).view(-1, 4, 128)
    v = q.view(-1, 4, 128)
    bad = torch.zeros(len(v), 4, dtype=torch.bool, device=DEV)
    for row, head, value in ((0, 1, math.inf), (1, 3, -math.inf), (int(starts[1]) + 9, 2, math.nan), (int(starts[2]) - 1, 0, math.inf)):
        v[row, head, 70] = value
        bad[row, head] = True
    v[int(starts[1]), 1] = -math.inf
    bad[int(starts[1]), 1] = True
    got = attend(cache, 0, q, starts, lens).view(-1, 4, 128)
    assert torch.equal(torch.isnan(got).all(-1), bad) and torch.equal(torch.isnan(got).any(-1), bad)
    assert torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_apart_and_equal(dtype):
    lens, counts = [300, 1000], [200, 5]
    cache = Cache(make_shape(4, 2, 64), lens)
    cache.fill(0, lens, spread=0)
    check(cache, 0, counts, lens, dtype, scale=40.0)
    check(cache, 0, counts, lens, dtype, scale=1e-20)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d, counts, lens", [(8, 2, 128, [3], [9000]), (4, 1, 64, [40, 1], [9001, 3]), (32, 8, 128, [70], [4100]), (5, 1, 128, [600, 0, 9], [8000, 0, 7000])])
def test_long_caches_in_parts(hq, hkv, d, counts, lens, dtype):
    cache = Cache(make_shape(hq, hkv, d), lens)
    cache.fill(0, lens)
    check(cache, 0, counts, lens, dtype)
    check(cache, 0, counts, lens, dtype, window=2500)
