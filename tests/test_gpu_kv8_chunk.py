"""Attention of a chunk of new tokens over the 8-bit cache on the GPU against its 64-bit plain form: chunk lengths from none to whole prompts, windows,
pages and values that are not there, parts of long caches, graphs and streams."""
import math

import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2603_02599_amd import binding as sun
from test_gpu_kv8 import DEV, DT, HEADS, Cache, host, i32, make_shape, two_tokens

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
    for window in (0, 2 ** 31 - 1, 2 ** 30, 3):
        check(cache, 0, counts, [100, 12, 4, 100, -7, 0], dtype, window=window)


@pytest.mark.parametrize("counts", [[5, 1], [60, 33]])
def test_lost_pages_of_many_heads(counts):
    """More heads than a page's stand-in has powers for: the values' powers of a page lie 16 bytes a head behind its keys'."""
    cache = Cache(make_shape(192, 192, 64), [70, 40])
    cache.fill(0, [70, 40])
    cache.table[0, 1] = -1
    cache.table[1, 2] = cache.n_pages
    cache.dev_table = i32(cache.table)
    check(cache, 0, counts, [70, 40], "bf16")


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
@pytest.mark.parametrize("hq, hkv", [(16, 16), (32, 8)])
def test_tiles_of_many_lengths(hq, hkv, dtype):
    """Enough groups of heads and tiles for no parts, so that tiles start by their lengths: long, short and empty requests, some with fewer positions than rows, with and without a window."""
    lens = [600, 3, 900, 0, 513, 64, 700, 1, 130, 40, 520, 512, 33, 200, 0, 5, 640, 1, 100, 16]
    counts = [600, 3, 300, 5, 1, 64, 0, 1, 130, 60, 33, 512, 33, 9, 0, 5, 16, 1, 100, 17]
    cache = Cache(make_shape(hq, hkv, 64), lens, extra_cols=0)
    cache.fill(0, lens)
    for window in (0, 90, 700):
        check(cache, 0, counts, lens, dtype, window=window, pad=20 if hq == hkv else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d, counts, lens", [(8, 2, 128, [3], [9000]), (4, 1, 64, [40, 1], [9001, 3]), (32, 8, 128, [70], [4100]), (5, 1, 128, [600, 0, 9], [8000, 0, 7000])])
def test_long_caches_in_parts(hq, hkv, d, counts, lens, dtype):
    cache = Cache(make_shape(hq, hkv, d), lens)
    cache.fill(0, lens)
    check(cache, 0, counts, lens, dtype)
    check(cache, 0, counts, lens, dtype, window=2500)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_other_requests_hold_does_not_matter(dtype):
    lens, counts = [500, 20, 3000, 64, 700], [40, 3, 2, 64, 1]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    starts = starts_of(counts)
    q = queries(cache.shape, int(starts[-1]), dtype)
    a = attend(cache, 0, q, starts, lens)
    assert torch.equal(a, attend(cache, 0, q, starts, lens))
    b = attend(cache, 0, q, starts, [500, 3, 2, 64, 1])
    for r in (0, 3):
        assert torch.equal(a[starts[r]:starts[r + 1]], b[starts[r]:starts[r + 1]])
    # another order of the same requests
    order = [2, 3, 0, 4, 1]
    moved = torch.cat([q[starts[r]:starts[r + 1]] for r in order])
    c = attend(cache, 0, moved, starts_of([counts[r] for r in order]), [lens[r] for r in order], table=cache.dev_table[order].contiguous())
    assert torch.equal(c, torch.cat([a[starts[r]:starts[r + 1]] for r in order]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_requests_and_room_for_far_more(dtype):
    """1024 requests, and tables far wider than the caches are long."""
    rng = np.random.default_rng(4)
    lens = rng.integers(1, 40, 1024).tolist()
    counts = [int(min(n, rng.integers(0, 4))) for n in lens]
    counts[700] = lens[700]
    cache = Cache(make_shape(4, 2, 64), lens)
    cache.fill(0, lens)
    check(cache, 0, counts, lens, dtype, pad=1)
    cache = Cache(make_shape(8, 1, 128), [700, 90], extra_cols=60000)
    cache.fill(0, [700, 90])
    check(cache, 0, [3, 90], [700, 90], dtype)
    check(cache, 0, [300, 1], [700, 90], dtype, window=200)


def test_row_starts_that_are_none_stay_inside():
    """Falling, negative and too large ones: rows outside what the arrays hold are neither read nor written, and the other requests are right."""
    lens, counts = [50, 300, 40, 17], [5, 40, 3, 2]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    starts = starts_of(counts)
    q = queries(cache.shape, 50, "bf16")
    good = attend(cache, 0, q, starts, lens)
    room = torch.full((60, q.shape[1]), 33.0, device=DEV, dtype=torch.bfloat16)
    for bad in ([0, 5, 45, 48, 2 ** 31 - 1], [-7, 5, 45, 48, 50], [0, 5, 45, 20, 10], [50, 0, 50, 0, 50], [60, 70, 80, 90, 100]):
        room.fill_(33.0)
        attend(cache, 0, q, bad, lens, out=room[:50])
        assert (room[50:] == 33).all()
        if bad[:3] == [0, 5, 45]:
            assert torch.equal(room[:45], good[:45])


def test_checks_of_device_arrays():
    cache = Cache(make_shape(4, 2, 64), [40, 40])
    cache.fill(0, [40, 40])
    q = queries(cache.shape, 10, "f32")
    for starts, n, window, status in (([0, 5, 11], [40, 40], 0, 6), ([0, 5, 4], [40, 40], 0, 6), ([-1, 5, 10], [40, 40], 0, 6), ([0, 5, 10], [4, 40], 0, 6), ([0, 5, 10], [40, -1], 0, 6),
                                      ([0, 5, 10], [40, 100], 0, 6), ([0, 5, 10], [40, 50], 0, 5), ([0, 1, 2], [50, 40], 2, 5)):
        with pytest.raises(sun.SunError) as e:
            attend(cache, 0, q, starts, n, window, flags=sun.SUN_VALIDATE)
        assert e.value.status == status, (starts, n)
    cache.table[:, 0] = -1   # in front of what a window lets them see
    cache.dev_table = i32(cache.table)
    attend(cache, 0, q, [0, 5, 10], [40, 40], 16, flags=sun.SUN_VALIDATE)
    cache.table[1, :] = -1
    cache.dev_table = i32(cache.table)
    attend(cache, 0, q, [0, 5, 5], [40, 40], 16, flags=sun.SUN_VALIDATE)   # a request without new rows reads nothing


def test_binding_refuses_other_shapes_types_and_devices():
    cache = Cache(make_shape(4, 2, 64), [40, 40])
    cache.fill(0, [40, 40])
    q, at = torch.zeros(5, 256, device=DEV), i32([40, 40])
    ws = torch.zeros(sun.sun_kv8_chunk_attention_workspace_bytes(cache.cfg, 2, 5, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
    ok = dict(q=q, row_starts=i32([0, 2, 5]), page_tables=cache.dev_table, n_tokens=at, out=q.clone(), workspace=ws)
    sun.sun_kv8_chunk_attention(cache.pool, 0, **ok)
    for change in (dict(q=q.bfloat16()), dict(q=q.half(), out=q.half()), dict(out=q.bfloat16()), dict(out=q[:4]), dict(out=q), dict(n_tokens=at.long()), dict(n_tokens=i32([1])), dict(row_starts=i32([0, 5])),
                   dict(row_starts=i32([0, 2, 5]).long()), dict(page_tables=cache.dev_table[:1]), dict(page_tables=cache.dev_table[0]), dict(q=torch.zeros(5, 512, device=DEV)[:, ::2]),
                   dict(q=q[0]), dict(workspace=ws.cpu()), dict(q=q.cpu()), dict(window=1 << 31), dict(window=-1)):
        with pytest.raises(sun.SunError) as e:
            sun.sun_kv8_chunk_attention(cache.pool, 0, **{**ok, **change})
        assert e.value.status == 2, change


def attend_two_tokens(cache, q):
    """A chunk of both tokens of every request: the last rows, which see both."""
    batch, hq, d = q.shape
    rows = torch.from_numpy(np.repeat(q.reshape(batch, -1), 2, 0)).to(DEV)
    out = attend(cache, 0, rows, starts_of([2] * batch), [2] * batch)
    return host(out).reshape(batch, 2, hq, d)[:, 1]


@pytest.mark.parametrize("d", [64, 128])
def test_32_bit_queries_and_weights_carry_24_bits(d):
    """Scores that are what the last 8 of a query's 24 bits leave, and values that cancel but for what the weights' last bits leave."""
    q_a, q_b = R.close_queries(12, 8)
    places = [(0, d - 1), (5, 6), (33, 2), (d // 2, 1), (31, 32), (17, 16)] * 2
    q = np.zeros((12, 8, d), np.float32)
    for r, (a, b) in enumerate(places):
        q[r, :, a], q[r, :, b] = q_a[r], q_b[r]
    cache = two_tokens([[(0, a, 0x38), (0, b, 0xb8)] for a, b in places], (0x38, 0), d, 8, 12)
    ref, off = R.close_queries_out(q_a, q_b, d)
    assert (np.abs(attend_two_tokens(cache, q) - ref[..., None]) <= off[..., None]).all()
    gaps = R.close_gaps(12, 8, d)
    q = np.zeros((12, 8, d), np.float32)
    for r in range(12):
        q[r, :, 3 * r] = gaps[r]
    cache = two_tokens([[(1, 3 * r, 0xb8)] for r in range(12)], (0x38, 0xb8), d, 8, 12)
    ref, off = R.close_gaps_out(gaps, d)
    assert (np.abs(attend_two_tokens(cache, q) - ref[..., None]) <= off[..., None]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_beyond_32_bit_offsets(dtype):
    """Pages at the end of a pool of more than 2^32 bytes a layer: the same results as in a small pool."""
    shape = make_shape(16, 8, 128)
    small = Cache(shape, [40, 900], poison=False)
    small.fill(1, [40, 900])
    n_pages = (9 << 30) // 2 // sun.sun_kv8_pool_bytes(small.cfg, 1) * 2 + 7
    mem = torch.zeros(sun.sun_kv8_pool_bytes(small.cfg, n_pages), dtype=torch.uint8, device=DEV)
    pool = sun.sun_kv8_pool_create(small.cfg, mem)
    lay, first = pool.layout(), n_pages - small.n_pages
    assert lay.k_layer > 1 << 32 and lay.n_pages == n_pages
    for off, layer, page, to_off, to_layer, to_page in ((lay.k_off, lay.k_layer, lay.k_page, small.lay.k_off, small.lay.k_layer, small.lay.k_page),
                                                       (lay.ks_off, lay.s_layer, lay.s_page, small.lay.ks_off, small.lay.s_layer, small.lay.s_page)):
        mem[off + layer + first * page:][:small.n_pages * page].copy_(small.mem[to_off + to_layer:][:small.n_pages * to_page])
    q = queries(shape, 240, dtype)
    outs = []
    for p, table in ((small.pool, small.dev_table), (pool, torch.where(small.dev_table >= 0, small.dev_table + first, small.dev_table))):
        out = torch.zeros_like(q)
        ws = torch.zeros(sun.sun_kv8_chunk_attention_workspace_bytes(small.cfg, 2, 240, table.shape[1]), dtype=torch.uint8, device=DEV)
        sun.sun_kv8_chunk_attention(p, 1, q, i32([0, 10, 240]), table, i32([40, 900]), out, ws)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and outs[0].abs().max() > 0


# ------------------------------------------------------------------ together

class Layer:
    """A layer over chunks of new tokens, as a caller that runs it itself puts it together: projection, append, chunk attention, output projection onto the residual
    stream, gated pair, down projection onto the residual stream."""

    def __init__(self, lens, counts, dtype, hidden=256, ffn=352, hq=8, hkv=2, d=64, seed=0, pad=2):
        self.cache = Cache(make_shape(hq, hkv, d, qk_norm=True), [n + c * 4 for n, c in zip(lens, counts)])
        self.cache.fill(0, lens)
        self.hq, self.hkv, self.d, self.dtype, self.counts = hq, hkv, d, DT[dtype], counts
        g = torch.Generator(device=DEV).manual_seed(seed)
        weights = lambda n, k: sun.sun_mx4_quantize(torch.randn(n, k, generator=g, device=DEV) * k ** -0.5)
        self.wqkv, self.wo, self.gate, self.up, self.down = weights((hq + 2 * hkv) * d, hidden), weights(hidden, hq * d), weights(ffn, hidden), weights(ffn, hidden), weights(hidden, ffn)
        self.bias = torch.randn(hidden, generator=g, device=DEV) * 0.1
        self.gains = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(self.dtype) for _ in range(2)]
        rows = sum(counts) + pad
        empty = lambda n, t=self.dtype: torch.zeros(rows, n, dtype=t, device=DEV)
        self.x = torch.randn(rows, hidden, generator=g, device=DEV).to(self.dtype)
        self.stream = torch.randn(rows, hidden, generator=g, device=DEV)      # 32 bits
        self.starts, self.lens = i32(starts_of(counts)), i32(lens)
        self.new = i32(counts)
        self.req = i32(np.concatenate([np.repeat(np.arange(len(lens)), counts), np.zeros(pad, int)]))
        self.step_of = i32(np.concatenate([*[np.arange(c) for c in counts], np.full(pad, -1 << 20)]))   # padding stays below 0
        self.n, self.pos = i32(lens) * 0, self.req * 0
        self.qkv, self.q, self.att, self.mid = empty((hq + 2 * hkv) * d), empty(hq * d), empty(hq * d), empty(ffn)
        self.after_o, self.act = empty(hidden, torch.float32), empty(hidden)
        width = self.cache.table.shape[1]
        nbytes = max(sun.sun_mx4_linear_workspace_bytes(max(hidden, (hq + 2 * hkv) * d), max(hidden, ffn, hq * d), rows), sun.sun_mx4_gated_workspace_bytes(ffn, hidden, rows),
                     sun.sun_mx4_linear_workspace_bytes(hidden, ffn, rows), sun.sun_mx4_linear_workspace_bytes(hidden, hq * d, rows),
                     sun.sun_mx4_linear_workspace_bytes((hq + 2 * hkv) * d, hidden, rows), sun.sun_kv8_chunk_attention_workspace_bytes(self.cache.cfg, len(lens), rows, width))
        self.ws = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)

    def run(self):
        qd, kd = self.hq * self.d, self.hkv * self.d
        torch.add(self.lens[self.req], self.step_of, out=self.pos)
        torch.add(self.lens, self.new, out=self.n)
        sun.sun_mx4_linear(*self.wqkv, self.x, self.qkv, self.ws)
        q, k, v = self.qkv[:, :qd], self.qkv[:, qd:qd + kd], self.qkv[:, qd + kd:]
        sun.sun_kv8_append(self.cache.pool, 0, q, k, v, self.pos, self.req, self.cache.dev_table, self.q, *self.gains)
        sun.sun_kv8_chunk_attention(self.cache.pool, 0, self.q, self.starts, self.cache.dev_table, self.n, self.att, self.ws)
        sun.sun_mx4_linear_fused(*self.wo, self.att, self.after_o, self.ws, residual=self.stream)
        self.act.copy_(self.after_o)
        sun.sun_mx4_gated(*self.gate, *self.up, self.act, self.mid, self.ws)
        sun.sun_mx4_linear_fused(*self.down, self.mid, self.after_o, self.ws, bias=self.bias, residual=self.after_o)
        self.lens.copy_(self.n)


def product(w, x):
    values = R.mx4_values(w[0].cpu().numpy(), w[1].cpu().numpy())
    return x @ values.T, (3 * x.shape[1] + 8) * 2.0 ** -24 * (np.abs(x) @ np.abs(values).T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_over_chunks(dtype):
    """Every operator's result against the plain form of its own inputs, over three steps; padding rows go through the products alone."""
    lens, counts = [0, 15, 500, 33], [40, 1, 4, 0]
    b = Layer(lens, counts, dtype)
    half = R.HALF[dtype]
    for step in range(3):
        stream = host(b.stream)
        b.run()
        torch.cuda.synchronize()
        views = b.cache.views()
        at = 0
        for i, c in enumerate(counts):
            n = lens[i] + c * (step + 1)
            assert int(b.lens[i]) == n
            if c:
                q = host(b.q[at:at + c]).reshape(c, b.hq, b.d)
                ref, mass, reach = reference(q, views, 0, b.cache.table[i], n, 0, b.cache.shape, b.cache.n_pages)
                assert (np.abs(host(b.att[at:at + c]).reshape(q.shape) - ref) <= bound(ref, mass, reach, n, b.d, dtype)).all()
            at += c
        g, g_off = product(b.gate, host(b.act))
        u, u_off = product(b.up, host(b.act))
        a = g / (1 + np.exp(-g))
        off = (1.13 * g_off + np.abs(a) * (6 * np.abs(g) + 8) * 2.0 ** -24) * (np.abs(u) + u_off) + np.abs(a) * u_off + np.abs(a * u) * (half * 1.01 + 2.0 ** -23)
        assert (np.abs(host(b.mid) - a * u) <= off + 1e-37).all()
        o, o_off = product(b.wo, host(b.att))
        mid = stream + o   # what the stream was before the down projection, up to o's error
        d, d_off = product(b.down, host(b.mid))
        ref = mid + d + host(b.bias)
        assert (np.abs(host(b.after_o) - ref) <= o_off + d_off + (np.abs(mid) + np.abs(d) + np.abs(ref) + 1) * 2.0 ** -22).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_in_a_graph(dtype):
    """Captured and replayed with the program's own eager work between: every replay's bits are the eager run's."""
    lens, counts = [0, 15, 500, 33], [40, 1, 4, 0]
    eager, graphed = Layer(lens, counts, dtype), Layer(lens, counts, dtype)
    start = (graphed.lens.clone(), graphed.cache.mem.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())   # behind the copies: the run changes what they are of
    with torch.cuda.stream(side):
        graphed.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.run()
    graphed.lens.copy_(start[0])
    graphed.cache.mem.copy_(start[1])
    for step in range(3):
        x = torch.randn_like(eager.x.float()).to(eager.x.dtype)
        eager.x.copy_(x)
        graphed.x.copy_(x)
        eager.run()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((eager.after_o, graphed.after_o), (eager.att, graphed.att), (eager.mid, graphed.mid), (eager.cache.mem, graphed.cache.mem), (eager.lens, graphed.lens)):
            assert torch.equal(a, b), step


def test_layers_on_streams():
    """On another stream than the current one, and two at once with workspaces of their own: what they give alone."""
    setups = [([40, 700, 3], [5, 2, 1]), ([2000, 5], [70, 5])]
    alone, together = ([Layer(*s, "bf16", seed=i) for i, s in enumerate(setups)] for _ in range(2))
    for b in alone:
        for _ in range(3):
            b.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in setups]
    for _ in range(3):
        for b, s in zip(together, streams):
            with torch.cuda.stream(s):
                b.run()
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert torch.equal(a.after_o, b.after_o) and torch.equal(a.att, b.att) and torch.equal(a.cache.mem, b.cache.mem)


def test_calls_take_a_stream():
    """stream= names the stream of a call: work queued in front of it there is seen."""
    lens, counts = [3000, 90], [100, 90]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    q = queries(cache.shape, 190, "bf16")
    want = attend(cache, 0, q, starts_of(counts), lens)
    side = torch.cuda.Stream()
    late = torch.zeros_like(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(q)
    got = attend(cache, 0, late, starts_of(counts), lens, stream=side)
    assert torch.equal(want, got)


def test_two_graphs_share_a_workspace():
    """Graphs replayed one behind the other on a stream may use the same workspace."""
    lens, counts = [[5000, 90], [4000, 700, 3]], [[3, 2], [100, 2, 1]]
    setups = []
    for n, c in zip(lens, counts):
        cache = Cache(make_shape(8, 2, 128), n)
        cache.fill(0, n)
        setups.append((cache, queries(cache.shape, sum(c), "bf16"), i32(starts_of(c)), i32(n)))
    nbytes = max(sun.sun_kv8_chunk_attention_workspace_bytes(cache.cfg, len(n), q.shape[0], cache.table.shape[1]) for (cache, q, _, n) in setups)
    ws = torch.full((nbytes,), 0xff, dtype=torch.uint8, device=DEV)
    outs, graphs = [], []
    for cache, q, starts, n in setups:
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sun.sun_kv8_chunk_attention(cache.pool, 0, q, starts, cache.dev_table, n, out, ws)
        outs.append(out)
        graphs.append(g)
    for step in range(3):
        for (cache, q, starts, n), seed in zip(setups, (5, 6)):
            q.copy_(queries(cache.shape, q.shape[0], "bf16", seed + step))
        want = [attend(cache, 0, q, host(starts), host(n)) for cache, q, starts, n in setups]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), step
