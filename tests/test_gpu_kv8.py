"""The 8-bit cache on the GPU against its 64-bit plain form: appends (codes, powers, rotated queries, and nothing else written), attention
of one new token, and both with the 4-bit product as the attention block of a decode worker."""
import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2603_02599_amd import binding as sun
from paper_2603_02599_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEAR = 2.0 ** -22   # how far the two sides' keys may be apart before they are rounded (each is a 32-bit number)


def host(t):
    return t.detach().cpu().double().numpy()


def i32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device=DEV)


def make_shape(hq, hkv, d, **kw):
    return wl.Shape("s", kw.pop("n_layers", 2), 256, hq, hkv, d, 128, 32, **kw)


class Cache:
    """A pool whose every byte is a code or power that must not be used (not-a-numbers), tables of shuffled pages, -1 elsewhere."""

    def __init__(self, shape, need, seed=0, extra_cols=2, poison=True):
        self.shape, self.cfg = shape, sun.make_cfg(shape, "f32")
        rng = np.random.default_rng(seed)
        pages = [-(-n // 16) for n in need]
        self.n_pages = sum(pages) + 3
        perm = rng.permutation(self.n_pages)
        self.table = np.full((len(need), max(pages + [1]) + extra_cols), -1, np.int32)
        at = 0
        for r, n in enumerate(pages):
            self.table[r, :n] = perm[at:at + n]
            at += n
        nbytes = sun.sun_kv8_pool_bytes(self.cfg, self.n_pages)
        self.mem = torch.full((nbytes,), 0xff if poison else 0, dtype=torch.uint8, device=DEV)
        self.pool = sun.sun_kv8_pool_create(self.cfg, self.mem)
        self.lay = self.pool.layout()
        self.dev_table = i32(self.table)

    def views(self, mem=None):
        m = np.ascontiguousarray((self.mem if mem is None else mem).cpu().numpy())
        return R.pool_views(m, self.lay, self.shape.n_layers, self.shape.n_kv_heads, self.shape.head_dim)

    def fill(self, layer, lens, seed=1, spread=3):
        """Random entries at positions 0 .. len - 1 of every request."""
        rng = np.random.default_rng(seed)
        m = self.mem.cpu().numpy().copy()
        k, v, ks, vs = R.pool_views(m, self.lay, self.shape.n_layers, self.shape.n_kv_heads, self.shape.head_dim)
        hkv, d = self.shape.n_kv_heads, self.shape.head_dim
        for r, n in enumerate(lens):
            if n == 0:
                continue
            t = np.arange(n)
            page, slot = self.table[r, t // 16], t % 16
            def draw():
                return R.to_e4m3(np.clip(rng.standard_normal((n, hkv, d)) * 110, -448, 448))
            k[layer][page, :, slot] = draw()
            v[layer][page, :, :, slot] = draw()
            ks[layer][page, :, slot] = rng.integers(121 - spread, 121 + 1, (n, hkv))
            vs[layer][page, :, slot] = rng.integers(121 - spread, 121 + 1, (n, hkv))
        self.mem.copy_(torch.from_numpy(m))


# ------------------------------------------------------------------ append

def run_append(cache, layer, rows, dtype, seed=0, with_q=True, scale=1.0, change=None, norm=False, in_place=False, flags=0, slices=True):
    """rows: (position, request) pairs.  Checks q_out and the whole pool against the plain form."""
    s = cache.shape
    hq, hkv, d, n = s.n_q_heads, s.n_kv_heads, s.head_dim, len(rows)
    g = torch.Generator(device=DEV).manual_seed(seed)
    qkv = (torch.randn(n, (hq + 2 * hkv) * d, generator=g, device=DEV) * scale)
    if change is not None:
        change(qkv)
    qkv = qkv.to(DT[dtype])
    q, k, v = (qkv[:, a * d:b * d] for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    if not slices:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    gains = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(DT[dtype]) for _ in range(2)] if norm else [None, None]
    before = cache.mem.clone()
    q_host, k_host, v_host = host(q), host(k), host(v)
    out = q if in_place else torch.full((n, hq * d), 55.0, device=DEV, dtype=DT[dtype])
    pos, req = [p for p, _ in rows], [r for _, r in rows]
    sun.sun_kv8_append(cache.pool, layer, q if with_q else None, k, v, i32(pos), i32(req), cache.dev_table, out if with_q else None,
                       gains[0] if with_q else None, gains[1], flags=flags)
    torch.cuda.synchronize()
    live = np.array(pos) >= 0
    if with_q:
        want = R.rotated(q_host, hq, cache.cfg, np.maximum(pos, 0), None if not norm else host(gains[0])).reshape(n, -1)
        # operands of a rotation: two products and a sum of the pair's values; a norm of 2^-24 (d / 4 + 8) at most before it
        a = np.abs(q_host if not norm else R.rotated(q_host, hq, cache.cfg, np.zeros(n), host(gains[0])).reshape(n, -1)).reshape(n, hq, 2, d // 2)
        pair = np.repeat(a.sum(2, keepdims=True), 2, 2).reshape(n, -1)
        bound = pair * (4 + (d / 4 + 8 if norm else 0)) * 2.0 ** -24 + np.abs(want) * R.HALF[dtype] * 1.01
        got = host(out)
        with np.errstate(invalid="ignore"):
            off = np.where(np.isfinite(want), np.abs(got - want) - bound, 0.0)
        assert (off[live] <= 0).all()
        assert np.array_equal(np.isfinite(got[live]), np.isfinite(want[live]))
        assert in_place or (got[~live] == 55).all()
    # The pool: the key's code, or that of either neighbour where it lies within NEAR of a border; everything else bit for bit.  The key
    # as it is stands beside the two that are moved: beside a largest value of 448 (power 0) a value of 1.5 * 2^-9 lies between the codes 1 and 2 and goes to
    # the even one, 2; moved down it goes to 1, and moved up the largest value takes the next power.
    expect = before.cpu().numpy().copy()
    near = [expect.copy(), expect.copy(), expect.copy()]
    kr = R.rotated(k_host, hkv, cache.cfg, np.maximum(pos, 0), None if not norm else host(gains[1]))
    vr = v_host.reshape(n, hkv, d)
    for mem, f in zip(near, (1.0, 1 - NEAR, 1 + NEAR)):
        views = R.pool_views(mem, cache.lay, s.n_layers, hkv, d)
        for i in range(n):
            if pos[i] < 0 or not 0 <= req[i] < len(cache.table) or pos[i] // 16 >= cache.table.shape[1]:
                continue
            page, slot = cache.table[req[i], pos[i] // 16], pos[i] % 16
            if not 0 <= page < cache.n_pages:
                continue
            kc, ks = R.entry(kr[i] * f)
            vc, vs = R.entry(vr[i])
            views[0][layer, page, :, slot], views[1][layer, page, :, :, slot] = kc, vc
            views[2][layer, page, :, slot], views[3][layer, page, :, slot] = ks, vs
    got = cache.mem.cpu().numpy()
    bad = np.nonzero((got != near[0]) & (got != near[1]) & (got != near[2]))[0]
    assert bad.size == 0, f"{bad.size} bytes, first at {bad[0]}: {got[bad[0]]} not {near[0][bad[0]]}"
    return out


HEADS = [(4, 2, 64), (8, 8, 128), (10, 2, 128), (8, 1, 128), (2, 2, 64), (7, 1, 128), (40, 8, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d", HEADS)
def test_append_one_row_per_request(hq, hkv, d, dtype):
    lens = [0, 1, 15, 16, 17, 200, 31, 4000]
    cache = Cache(make_shape(hq, hkv, d), [n + 1 for n in lens])
    run_append(cache, 1, [(n, r) for r, n in enumerate(lens)], dtype, flags=sun.SUN_VALIDATE)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d", [(4, 2, 64), (10, 2, 128)])
@pytest.mark.parametrize("counts, firsts", [((16,), (0,)), ((16,), (5,)), ((1,), (16,)), ((33, 50), (0, 7)), ((15, 17, 3, 64), (1, 16, 31, 0)), ((700, 340), (3, 1000)), ((2050, 63, 1, 2001), (3, 1000, 15, 7))])
def test_append_prompts(counts, firsts, hq, hkv, d, dtype):
    """Runs of positions that start and end anywhere in a page, of several requests in one call (4096 rows and more: four a workgroup)."""
    cache = Cache(make_shape(hq, hkv, d), [f + c for f, c in zip(firsts, counts)])
    run_append(cache, 0, [(f + t, r) for r, (f, c) in enumerate(zip(firsts, counts)) for t in range(c)], dtype, flags=sun.SUN_VALIDATE)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [37, 1061, 4133])
def test_append_padding_and_any_order(rows, dtype):
    """Rows in any order with padding between them; a row of the last block stays within the arrays."""
    rng = np.random.default_rng(rows)
    need = [rows, 64, 100]
    cache = Cache(make_shape(4, 2, 128), need)
    at = [(t, 0) for t in range(rows - 30)] + [(t, 1) for t in range(11)] + [(t + 3, 2) for t in range(9)] + [(-1, 0)] * 6 + [(-7, 99)] * 4
    order = rng.permutation(len(at))
    run_append(cache, 1, [at[i] for i in order], dtype)
    cache2 = Cache(make_shape(4, 2, 128), need)
    run_append(cache2, 1, at[:20] + [(-1, 2)] * 3 + at[20:], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_without_pages_leaves_the_pool(dtype):
    """Positions beyond the table, entries outside the pool and requests that are none: q is rotated, the pool stays."""
    cache = Cache(make_shape(4, 2, 64), [40, 40])
    cache.table[1, 1] = cache.n_pages
    cache.table[0, 2] = -5
    cache.dev_table = i32(cache.table)
    rows = [(0, 0), (16, 1), (33, 0), (16 * cache.table.shape[1], 0), (2 ** 31 - 1, 1), (3, 2), (3, -1), (5, 1)]
    run_append(cache, 0, rows, dtype)
    run_append(cache, 0, [(t, 0) for t in range(36)], dtype)   # a run that loses its page half way


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [make_shape(8, 2, 64, qk_norm=True, rms_eps=1e-6, rope_base=1e6), make_shape(10, 2, 128, qk_norm=True),
                                   make_shape(8, 4, 128, rope_base=500000.0, rope_scaling=(8.0, 1.0, 4.0, 256))])
def test_append_backbone_options(shape, dtype):
    cache = Cache(shape, [300, 5000])
    rows = [(t, 0) for t in range(257, 300)] + [(4999, 1), (0, 1)]
    run_append(cache, 0, rows, dtype, norm=shape.qk_norm)
    run_append(cache, 1, rows, dtype, norm=shape.qk_norm, with_q=False, slices=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_in_place_and_far_positions(dtype):
    cache = Cache(make_shape(4, 2, 128, rope_base=10000.0), [32], extra_cols=0)
    wide = np.full((1, 1 << 20), -1, np.int32)
    wide[0, -1] = cache.table[0, 0]
    cache.table, cache.dev_table = wide, i32(wide)
    run_append(cache, 0, [((1 << 24) - 3, 0)], dtype, in_place=True, slices=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_values_at_the_edges(dtype):
    """Zero vectors, subnormal and huge ones, powers that are just reached, infinities and not-a-numbers (row by row; position 0 turns nothing)."""
    d = 64
    def change(x):
        x[0] = 0
        x[1] = -0.0
        x[2] *= 1e-42
        x[3] *= 1e38 / 4
        x[4] = 448.0
        x[5] = 449.0
        x[6, ::3] = float("nan")
        x[7, 1::5] = float("inf")
        x[8] = float("nan")
        x[9, ::2] = 2.0 ** -9 * 1.5
        x[9, 1::2] = 448.0
        x[10] *= 2.0 ** -110
    cache = Cache(make_shape(4, 2, d), [1] * 11)
    run_append(cache, 0, [(0, r) for r in range(11)], dtype, change=change)


# ------------------------------------------------------------------ attention

def run_attention(cache, layer, lens, dtype, window=0, seed=3, q_scale=1.5, batch_rows=None):
    s = cache.shape
    rows = list(range(len(lens))) if batch_rows is None else batch_rows
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn(len(lens), s.n_q_heads * s.head_dim, generator=g, device=DEV) * q_scale).to(DT[dtype])[rows].contiguous()
    table = cache.dev_table[rows].contiguous()
    out = torch.full_like(q, 33.0)
    nbytes = sun.sun_kv8_attention_workspace_bytes(cache.cfg, len(rows), table.shape[1])
    ws = torch.full((nbytes + 256,), 0xff, dtype=torch.uint8, device=DEV)
    sun.sun_kv8_attention(cache.pool, layer, q, table, i32([lens[r] for r in rows]), out, ws, window=window)
    torch.cuda.synchronize()
    assert (ws[nbytes:] == 0xff).all(), "written behind the workspace"
    return q, out


def check_attention(cache, layer, lens, dtype, window=0, **kw):
    s = cache.shape
    before = cache.mem.clone()
    q, out = run_attention(cache, layer, lens, dtype, window, **kw)
    assert torch.equal(before, cache.mem)
    views, got = cache.views(), host(out).reshape(len(lens), s.n_q_heads, s.head_dim)
    for i, n in enumerate(lens):
        n = min(max(n, 0), 16 * cache.table.shape[1])
        ref, mass, reach = R.attention(host(q[i]).reshape(s.n_q_heads, s.head_dim), views, layer, cache.table[i], n, window, s.n_kv_heads, cache.n_pages)
        over = np.abs(got[i] - ref) / R.attention_bound(ref, mass, reach, n, s.head_dim, dtype)
        nan = np.isnan(ref)   # a count that reaches slots nobody wrote: the plain form reads the same not-a-numbers
        assert np.array_equal(nan, np.isnan(got[i])) and (over[~nan] <= 1).all(), f"request {i} of {n} tokens: {over[~nan].max(initial=0):.2f} of the bound"
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d", HEADS)
def test_attention_lengths(hq, hkv, d, dtype):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 128, 200, 1000]
    cache = Cache(make_shape(hq, hkv, d), lens)
    cache.fill(1, lens)
    check_attention(cache, 1, lens, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 2, 16, 17, 64, 100, 5000])
def test_attention_window(window, dtype):
    """Pages in front of the window are gone from the tables."""
    lens = [0, 1, 16, 40, 64, 65, 100, 333, 700]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    for r, n in enumerate(lens):
        cache.table[r, :max(0, n - window) // 16] = -1
    cache.dev_table = i32(cache.table)
    check_attention(cache, 0, lens, dtype, window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d, lens", [(8, 2, 128, [5000]), (4, 1, 64, [9001, 3]), (32, 8, 128, [4100]), (5, 1, 128, [30000, 0, 17000])])
def test_attention_split_over_long_caches(hq, hkv, d, lens, dtype):
    cache = Cache(make_shape(hq, hkv, d, n_layers=1), lens)
    cache.fill(0, lens)
    check_attention(cache, 0, lens, dtype)
    check_attention(cache, 0, lens, dtype, window=2500)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_full_batch(dtype):
    lens = [int(x) for x in np.random.default_rng(5).integers(0, 700, 256)]
    cache = Cache(make_shape(8, 2, 64, n_layers=1), lens)
    cache.fill(0, lens)
    check_attention(cache, 0, lens, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_leaves_lost_pages_out(dtype):
    """Entries outside the pool: their tokens do not count; a request that has none left gets zeros.  Counts beyond the table are cut."""
    lens = [100, 700, 64, 5000]
    cache = Cache(make_shape(8, 2, 128), [100, 700, 64, 100])
    cache.fill(0, [100, 700, 64, 100])
    cache.table[0, 2] = -1
    cache.table[1, :30] = cache.n_pages
    cache.table[2, :] = -3
    cache.dev_table = i32(cache.table)
    out = check_attention(cache, 0, lens, dtype)
    assert (out[2] == 0).all()
    check_attention(cache, 0, [-5, 3, 64, 2 ** 31 - 1], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_peaked_and_flat(dtype):
    """Scores far apart (one token takes all, the maximum grows in the last page) and equal ones."""
    lens = [300, 1000]
    cache = Cache(make_shape(4, 2, 64), lens)
    cache.fill(0, lens, spread=0)
    check_attention(cache, 0, lens, dtype, q_scale=40.0)
    check_attention(cache, 0, lens, dtype, q_scale=1e-20)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_not_a_numbers_stay_where_they_belong(dtype):
    """A key or value that is not a number makes its KV head's heads of its request so (a value: its dim), and nothing else."""
    lens = [70, 900, 40]
    cache = Cache(make_shape(4, 2, 64), lens)
    cache.fill(0, lens)
    clean = run_attention(cache, 0, lens, dtype)[1].clone()
    lay = cache.lay
    k_at = lay.k_off + int(cache.table[1, 20]) * lay.k_page + 1 * lay.k_head + 3 * lay.k_token + 9
    v_at = lay.v_off + int(cache.table[2, 1]) * lay.v_page + 0 * lay.v_head + 5 * lay.v_token + 11 * lay.v_dim
    cache.mem[k_at] = 127
    cache.mem[v_at] = 127
    got = run_attention(cache, 0, lens, dtype)[1].view(3, 4, 64)
    bad = torch.zeros(3, 4, 64, dtype=torch.bool, device=DEV)
    bad[1, 2:] = True
    bad[2, :2, 11] = True
    assert torch.equal(torch.isnan(got), bad)
    assert torch.equal(got[~bad], clean.view(3, 4, 64)[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_does_not_depend_on_batch_mates(dtype):
    lens = [500, 20, 3000, 64]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    a = run_attention(cache, 0, lens, dtype)[1]
    b = run_attention(cache, 0, [500, 0, 1, 64], dtype)[1]
    assert torch.equal(a[0], b[0]) and torch.equal(a[3], b[3])
    c = run_attention(cache, 0, lens, dtype, batch_rows=[2, 3, 0, 1])[1]
    assert torch.equal(a[[2, 3, 0, 1]], c)
    assert torch.equal(a, run_attention(cache, 0, lens, dtype)[1])


# ------------------------------------------------------------------ checks of device arrays

def test_validate_names_what_is_wrong():
    cache = Cache(make_shape(4, 2, 64), [40, 40])
    run_append(cache, 0, [(0, 0), (20, 1)], "f32", flags=sun.SUN_VALIDATE)
    before = cache.mem.clone()
    for rows, status in (([(0, 5)], 5), ([(0, -1)], 5), ([(48, 0)], 5), ([(16 * cache.table.shape[1], 0)], 6), ([(3, 1), (3, 1)], 6)):
        x = torch.zeros(len(rows), 128, device=DEV)
        with pytest.raises(sun.SunError) as e:
            sun.sun_kv8_append(cache.pool, 0, None, x, x, i32([p for p, _ in rows]), i32([r for _, r in rows]), cache.dev_table, None, flags=sun.SUN_VALIDATE)
        assert e.value.status == status, rows
    q = torch.zeros(2, 256, device=DEV)
    ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(cache.cfg, 2, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
    for n, window, status in (([1, -1], 0, 6), ([1, 100], 0, 6), ([1, 50], 0, 5), ([50, 1], 2, 5)):
        with pytest.raises(sun.SunError) as e:
            sun.sun_kv8_attention(cache.pool, 0, q, cache.dev_table, i32(n), q.clone(), ws, window=window, flags=sun.SUN_VALIDATE)
        assert e.value.status == status, (n, window)
    torch.cuda.synchronize()
    assert torch.equal(before, cache.mem)


def test_binding_refuses_other_shapes_types_and_devices():
    cache = Cache(make_shape(4, 2, 64), [40, 40])
    k, q = torch.zeros(2, 128, device=DEV), torch.zeros(2, 256, device=DEV)
    at = i32([0, 1])
    ok = dict(q=q, k=k, v=k, positions=at, requests=at * 0, page_tables=cache.dev_table, q_out=q.clone())
    sun.sun_kv8_append(cache.pool, 0, **ok)
    for change in (dict(k=k.half()), dict(v=k.bfloat16()), dict(v=k[:, :64]), dict(q=q[:1]), dict(positions=at.long()), dict(requests=at[:1]), dict(page_tables=cache.dev_table[0]),
                   dict(q_out=None), dict(v=k.cpu()), dict(k=torch.zeros(128, 2, device=DEV).t()), dict(q_norm=q[0, :64])):
        with pytest.raises(sun.SunError) as e:
            sun.sun_kv8_append(cache.pool, 0, **{**ok, **change})
        assert e.value.status == 2, change
    ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(cache.cfg, 2, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
    ok = dict(q=q, page_tables=cache.dev_table, n_tokens=at, out=q.clone(), workspace=ws)
    for change in (dict(q=q.bfloat16()), dict(out=q.bfloat16()), dict(n_tokens=at.long()), dict(page_tables=cache.dev_table[:1]), dict(q=torch.zeros(2, 512, device=DEV)[:, ::2]),
                   dict(workspace=ws.cpu()), dict(q=q.cpu())):
        with pytest.raises(sun.SunError) as e:
            sun.sun_kv8_attention(cache.pool, 0, **{**ok, **change})
        assert e.value.status == 2, change


# ------------------------------------------------------------------ together

class Block:
    """The attention block of a decode worker: 4-bit projections around the 8-bit cache."""

    def __init__(self, lens, dtype, hidden=256, hq=8, hkv=2, d=64, seed=0):
        self.cache = Cache(make_shape(hq, hkv, d, qk_norm=True), [n + 4 for n in lens])
        self.cache.fill(0, lens)
        self.hq, self.hkv, self.d, self.dtype = hq, hkv, d, DT[dtype]
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.wqkv = sun.sun_mx4_quantize(torch.randn((hq + 2 * hkv) * d, hidden, generator=g, device=DEV) * 0.1)
        self.wo = sun.sun_mx4_quantize(torch.randn(hidden, hq * d, generator=g, device=DEV) * 0.1)
        self.gains = [(1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(self.dtype) for _ in range(2)]
        b = len(lens)
        self.x = torch.randn(b, hidden, generator=g, device=DEV).to(self.dtype)
        self.lens, self.req = i32(lens), torch.arange(b, dtype=torch.int32, device=DEV)
        self.qkv = torch.zeros(b, (hq + 2 * hkv) * d, dtype=self.dtype, device=DEV)
        self.q, self.att = (torch.zeros(b, hq * d, dtype=self.dtype, device=DEV) for _ in range(2))
        self.out = torch.zeros(b, hidden, dtype=self.dtype, device=DEV)
        self.n = i32(lens) * 0
        nbytes = max(sun.sun_mx4_linear_workspace_bytes(self.qkv.shape[1], hidden, b), sun.sun_mx4_linear_workspace_bytes(hidden, hq * d, b),
                     sun.sun_kv8_attention_workspace_bytes(self.cache.cfg, b, self.cache.table.shape[1]))
        self.ws = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)

    def step(self):
        qd, kd = self.hq * self.d, self.hkv * self.d
        sun.sun_mx4_linear(*self.wqkv, self.x, self.qkv, self.ws)
        q, k, v = self.qkv[:, :qd], self.qkv[:, qd:qd + kd], self.qkv[:, qd + kd:]
        sun.sun_kv8_append(self.cache.pool, 0, q, k, v, self.lens, self.req, self.cache.dev_table, self.q, *self.gains)
        torch.add(self.lens, 1, out=self.n)
        sun.sun_kv8_attention(self.cache.pool, 0, self.q, self.cache.dev_table, self.n, self.att, self.ws)
        sun.sun_mx4_linear(*self.wo, self.att, self.out, self.ws)
        self.lens += 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_decode_workers_attention_block(dtype):
    """Each operator's result against the plain form of its own inputs, over three steps."""
    lens = [0, 15, 16, 500, 33]
    b = Block(lens, dtype)
    s, cfg = b.cache.shape, b.cache.cfg
    for step in range(3):
        now = [n + step for n in lens]
        b.step()
        torch.cuda.synchronize()
        for w, x, out in ((b.wqkv, b.x, b.qkv), (b.wo, b.att, b.out)):
            wv, xs = R.mx4_values(w[0].cpu().numpy(), w[1].cpu().numpy()), host(x)
            ref = xs @ wv.T
            assert (np.abs(host(out) - ref) <= R.linear_bound(xs, wv, ref, dtype)).all()
        views, qkv = b.cache.views(), host(b.qkv)
        k = R.rotated(qkv[:, b.hq * b.d:(b.hq + b.hkv) * b.d], b.hkv, cfg, now, host(b.gains[1]))
        v = qkv[:, (b.hq + b.hkv) * b.d:].reshape(-1, b.hkv, b.d)
        for i, n in enumerate(now):
            page, slot = b.cache.table[i, n // 16], n % 16
            for y, code, scale in ((k[i], views[0][0, page, :, slot], views[2][0, page, :, slot]), (v[i], views[1][0, page, :, :, slot], views[3][0, page, :, slot])):
                got = R.E4M3[code] * np.exp2(scale.astype(np.float64) - 127)[:, None]
                top = np.abs(y).max(-1, keepdims=True)
                assert (np.abs(got - y) <= np.abs(y) * 2.0 ** -4 * 1.001 + top * 2.0 ** -17).all()   # half a step, the subnormals' 2^-10 of 448
            ref, mass, reach = R.attention(host(b.q[i]).reshape(b.hq, b.d), views, 0, b.cache.table[i], n + 1, 0, b.hkv, b.cache.n_pages)
            assert (np.abs(host(b.att[i]).reshape(b.hq, b.d) - ref) <= R.attention_bound(ref, mass, reach, n + 1, b.d, dtype)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_in_a_graph(dtype):
    """Captured and replayed with the program's own eager work between: every replay's bits are the eager step's."""
    lens = [0, 15, 500, 33]
    eager, graphed = Block(lens, dtype), Block(lens, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    start = (graphed.lens.clone(), graphed.cache.mem.clone())
    with torch.cuda.stream(side):
        graphed.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    graphed.lens.copy_(start[0])
    graphed.cache.mem.copy_(start[1])
    for step in range(4):
        x = torch.randn_like(eager.x.float()).to(eager.x.dtype)
        eager.x.copy_(x)
        graphed.x.copy_(x)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((eager.out, graphed.out), (eager.q, graphed.q), (eager.cache.mem, graphed.cache.mem), (eager.lens, graphed.lens)):
            assert torch.equal(a, b), step


def test_block_on_another_stream():
    lens = [40, 700, 3]
    a, b = Block(lens, "bf16"), Block(lens, "bf16")
    torch.cuda.synchronize()
    a.step()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.step()
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.out) and torch.equal(a.cache.mem, b.cache.mem)


def test_blocks_on_two_streams_at_once():
    """Two blocks with workspaces of their own, their steps under way together, give what they give alone."""
    lens = [[40, 700, 3], [2000, 5]]
    alone, together = ([Block(n, "bf16", seed=i) for i, n in enumerate(lens)] for _ in range(2))
    for b in alone:
        for _ in range(8):
            b.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in lens]
    for _ in range(8):
        for b, s in zip(together, streams):
            with torch.cuda.stream(s):
                b.step()
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert torch.equal(a.out, b.out) and torch.equal(a.cache.mem, b.cache.mem)


def test_two_graphs_share_a_workspace():
    """Graphs replayed one behind the other on a stream may use the same workspace."""
    lens = [[3000, 90], [40, 700, 3]]
    eager, graphed = ([Block(n, "bf16", seed=i) for i, n in enumerate(lens)] for _ in range(2))
    ws = max((b.ws for b in graphed), key=lambda t: t.numel())
    graphs = []
    for b in graphed:
        b.ws = ws
        start = (b.lens.clone(), b.cache.mem.clone())
        b.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.step()
        graphs.append(g)
        b.lens.copy_(start[0])
        b.cache.mem.copy_(start[1])
    for step in range(4):
        for b in eager:
            b.step()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, graphed):
            assert torch.equal(a.out, b.out) and torch.equal(a.cache.mem, b.cache.mem), step


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_beyond_32_bit_offsets(dtype):
    """Pages at the end of a pool of more than 2^32 bytes a layer: the same bytes and results as in a small pool."""
    shape = make_shape(16, 8, 128)
    small = Cache(shape, [40, 900], poison=False)
    small.fill(1, [37, 893])
    cols = small.table.shape[1]
    n_pages = (9 << 30) // 2 // sun.sun_kv8_pool_bytes(small.cfg, 1) * 2 + 7
    mem = torch.zeros(sun.sun_kv8_pool_bytes(small.cfg, n_pages), dtype=torch.uint8, device=DEV)
    pool = sun.sun_kv8_pool_create(small.cfg, mem)
    lay, first = pool.layout(), n_pages - small.n_pages
    assert lay.k_layer > 1 << 32 and lay.n_pages == n_pages

    def blocks(m, l, page, pages):   # codes and scales of the second layer's pages
        c, s = l.k_off + l.k_layer + page * l.k_page, l.ks_off + l.s_layer + page * l.s_page
        return m[c:c + pages * l.k_page], m[s:s + pages * l.s_page]
    for a, b in zip(blocks(mem, lay, first, small.n_pages), blocks(small.mem, small.lay, 0, small.n_pages)):
        a.copy_(b)
    table = torch.where(small.dev_table >= 0, small.dev_table + first, small.dev_table)
    g = torch.Generator(device=DEV).manual_seed(1)
    pos, req = i32([37, 38, 39, 893, 894, 895, 896, 897, 898, 899]), i32([0] * 3 + [1] * 7)
    q, k, v = (torch.randn(10, h * 128, generator=g, device=DEV).to(DT[dtype]) for h in (16, 8, 8))
    outs = []
    for p, t in ((small.pool, small.dev_table), (pool, table)):
        q_out, out = torch.zeros_like(q), torch.zeros(2, 16 * 128, device=DEV, dtype=DT[dtype])
        sun.sun_kv8_append(p, 1, q, k, v, pos, req, t, q_out)
        ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(small.cfg, 2, cols), dtype=torch.uint8, device=DEV)
        sun.sun_kv8_attention(p, 1, q_out[[2, 9]], t, i32([40, 900]), out, ws)
        outs.append((q_out, out))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and outs[0][1].abs().min() > 0
    for a, b in zip(blocks(mem, lay, first, small.n_pages), blocks(small.mem, small.lay, 0, small.n_pages)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq, hkv, d, batch", [(8, 8, 64, 11), (16, 8, 128, 300), (4, 2, 128, 1024)])
def test_attention_with_room_for_far_more(hq, hkv, d, batch, dtype):
    """A table that is far wider than the caches are long: the same bits, whichever way the chunks are dealt."""
    lens = [(0, 1, 700, 16, 2500, 0, 257)[i % 7] for i in range(batch)]
    cache = Cache(make_shape(hq, hkv, d), lens, extra_cols=0)
    cache.fill(1, lens)
    q = torch.randn(batch, hq * d, device=DEV).to(DT[dtype])
    results = []
    for cols in (cache.table.shape[1], 16000):
        table = torch.full((batch, cols), -1, device=DEV, dtype=torch.int32)
        table[:, :cache.table.shape[1]] = cache.dev_table
        ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(cache.cfg, batch, cols), dtype=torch.uint8, device=DEV)
        for window in (0, 600):
            out = torch.full_like(q, 9.0)
            sun.sun_kv8_attention(cache.pool, 1, q, table, i32(lens), out, ws, window=window)
            results.append(out)
    assert torch.equal(results[0], results[2]) and torch.equal(results[1], results[3])
    assert not torch.equal(results[0], results[1]) and (results[0][[i for i, n in enumerate(lens) if n == 0]] == 0).all()
    check_attention(cache, 1, lens, dtype)


def test_workspace_of_a_larger_batch_serves_a_smaller():
    """Five requests are cut finer than eight: the workspace made for eight holds their parts."""
    lens = [16 * 300] * 5
    cache = Cache(make_shape(8, 8, 64), lens, extra_cols=0)
    cache.fill(0, lens)
    q = torch.randn(5, 8 * 64, device=DEV)
    results = []
    for batch in (5, 8):
        out = torch.zeros_like(q)
        ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(cache.cfg, batch, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
        sun.sun_kv8_attention(cache.pool, 0, q, cache.dev_table, i32(lens), out, ws)
        results.append(out)
    assert torch.equal(*results)


# ------------------------------------------------------------------ queries that are not numbers

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols, window", [(0, 0), (0, 300), (8000, 0), (8000, 300), (150000, 0)])
@pytest.mark.parametrize("hq, hkv, d", [(8, 2, 64), (8, 2, 128)])
def test_attention_queries_that_are_not_numbers(hq, hkv, d, cols, window, dtype):
    """A query with an infinity or a not-a-number has no softmax: not-a-numbers in its head, whether its scores are infinities of one sign, of both or
    not-a-numbers themselves.  Zeros stay where no token is, and every other head keeps its bits."""
    lens = [1, 700, 3, 2500, 0, 90, 16, 257]
    cache = Cache(make_shape(hq, hkv, d, n_layers=1), lens)
    cache.fill(0, lens)
    m = cache.mem.cpu().numpy().copy()
    k = R.pool_views(m, cache.lay, 1, hkv, d)[0][0]
    for r, n in enumerate(lens):
        for t in range(n):
            k[cache.table[r, t // 16], :, t % 16, 5] = 0x38   # every key's dim 5 is 1 times its power: an infinite query there gives scores of one sign
    cache.mem.copy_(torch.from_numpy(m))
    cache.table[6, 0] = -1                                    # a request whose page is gone
    table = torch.full((len(lens), max(cols, cache.table.shape[1])), -1, device=DEV, dtype=torch.int32)
    table[:, :cache.table.shape[1]] = i32(cache.table)
    ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(cache.cfg, len(lens), table.shape[1]), dtype=torch.uint8, device=DEV)
    q = (torch.randn(len(lens), hq, d, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV) * 1.5).to(DT[dtype])

    def attend(q):
        out = torch.full_like(q, 33.0)
        sun.sun_kv8_attention(cache.pool, 0, q.view(len(lens), -1), table, i32(lens), out.view(len(lens), -1), ws, window=window)
        return out

    clean = attend(q)
    assert torch.isfinite(clean).all() and (clean[4] == 0).all() and (clean[6] == 0).all()
    bad = q.clone()
    inf, nan = float("inf"), float("nan")
    places = [(0, 0, 5, -inf), (0, 1, 5, inf), (0, 5, 9, nan), (1, 2, 5, -inf), (1, 4, 5, inf), (1, 7, 40, -inf), (2, 3, 5, -inf), (3, 6, 5, -inf), (3, 1, 63, nan),
              (4, 0, 5, -inf), (4, 1, 5, nan), (5, 7, 5, -inf), (5, 0, 11, inf), (6, 2, 5, -inf), (7, 5, 5, -inf), (7, 4, 5, inf)]
    want = torch.zeros(len(lens), hq, d, dtype=torch.bool, device=DEV)
    for r, h, j, value in places:
        bad[r, h, j] = value
        want[r, h] = r not in (4, 6)
    got = attend(bad)
    assert torch.equal(torch.isnan(got), want)
    assert torch.equal(got[~want], clean[~want])
    views = cache.views()
    for r, n in enumerate(lens):   # the plain form says the same
        with np.errstate(invalid="ignore"):
            ref = R.attention(host(bad[r]), views, 0, cache.table[r], n, window, hkv, cache.n_pages)[0]
        assert np.array_equal(np.isnan(ref), want[r].cpu().numpy())


# ------------------------------------------------------------------ what only the low bits decide

def two_tokens(dims, values, d, hq, batch):
    """Requests of two tokens whose keys are zero but for `dims` (request -> [(token, dim, code)], power 0) and whose values are `values` in every dim."""
    cache = Cache(make_shape(hq, 1, d, n_layers=1), [2] * batch)
    m = cache.mem.cpu().numpy().copy()
    k, v, ks, vs = (x[0] for x in R.pool_views(m, cache.lay, 1, 1, d))
    for r in range(batch):
        page = cache.table[r, 0]
        k[page, 0, :2] = 0
        ks[page, 0, :2] = vs[page, 0, :2] = 127
        for t in range(2):
            v[page, 0, :, t] = values[t]
        for t, j, code in dims[r]:
            k[page, 0, t, j] = code
    cache.mem.copy_(torch.from_numpy(m))
    return cache


def attend_two(cache, q):
    batch, hq, d = q.shape
    out = torch.full((batch, hq * d), 33.0, device=DEV)
    ws = torch.zeros(sun.sun_kv8_attention_workspace_bytes(cache.cfg, batch, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
    sun.sun_kv8_attention(cache.pool, 0, torch.from_numpy(q.reshape(batch, -1)).to(DEV), cache.dev_table, i32([2] * batch), out, ws)
    return host(out).reshape(batch, hq, d)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_32_bit_queries_carry_24_bits(d):
    """Scores that are what the last 8 of a query's 24 bits leave."""
    q_a, q_b = R.close_queries(12, 8)
    places = [(0, d - 1), (5, 6), (33, 2), (d // 2, 1), (31, 32), (17, 16)] * 2
    q = np.zeros((12, 8, d), np.float32)
    for r, (a, b) in enumerate(places):
        q[r, :, a], q[r, :, b] = q_a[r], q_b[r]
    cache = two_tokens([[(0, a, 0x38), (0, b, 0xb8)] for a, b in places], (0x38, 0), d, 8, 12)   # token 0: 1 at a, -1 at b, value 1; token 1: zeros
    got = attend_two(cache, q)
    ref, bound = R.close_queries_out(q_a, q_b, d)
    assert (np.abs(got - ref[..., None]) <= bound[..., None]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_attention_32_bit_weights_carry_24_bits(d):
    """Values that cancel but for what the weights' last bits leave."""
    gaps = R.close_gaps(12, 8, d)
    q = np.zeros((12, 8, d), np.float32)
    for r in range(12):
        q[r, :, 3 * r] = gaps[r]
    cache = two_tokens([[(1, 3 * r, 0xb8)] for r in range(12)], (0x38, 0xb8), d, 8, 12)   # scores 0 and -gap / sqrt d, values 1 and -1
    got = attend_two(cache, q)
    ref, bound = R.close_gaps_out(gaps, d)
    assert (np.abs(got - ref[..., None]) <= bound[..., None]).all()


def test_keys_that_are_no_matrix_are_refused():
    cache = Cache(make_shape(4, 2, 64), [40])
    k, at = torch.zeros(1, 128, device=DEV), i32([0])
    for bad in (k[0, 0], k[0], k[None]):
        with pytest.raises(sun.SunError) as e:
            sun.sun_kv8_append(cache.pool, 0, None, bad, bad, at, at, cache.dev_table, None)
        assert e.value.status == 2
