"""The 8-bit cache and the microscaled 4-bit format without a GPU: the reference forms against hand-made values, the pool's
layout, workspace sizes, and every refusal that happens before anything is enqueued."""
import ctypes as C
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2603_02599_amd import binding as sun
from paper_2603_02599_amd import workloads as wl

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000  # aligned, never dereferenced: these calls fail (or only store it) before any GPU work


@pytest.fixture(scope="module")
def lib():
    from paper_2603_02599_amd.build import build_lib
    build_lib()
    return sun.lib()


def test_e4m3_by_hand():
    assert _same(R.E4M3[[0, 1, 8, 0x38, 0x7e, 0xfe]], [0, 2.0 ** -9, 2.0 ** -6, 1, 448, -448]) and math.isnan(R.E4M3[127])
    # halves go to the even code, in the subnormals and above
    got = R.to_e4m3(np.array([2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875, 447.9, -1.0, np.nan, np.inf]))
    assert got.tolist() == [0, 2, 0x38, 0x3a, 0x7e, 0xb8, 127, 127]
    every = np.delete(np.arange(256), [127, 255])
    assert _same(R.E4M3[R.to_e4m3(R.E4M3[every])], R.E4M3[every])
    t = torch.linspace(-460, 460, 100001)
    t = t[t.abs() <= 448]
    assert _same(R.to_e4m3(t.double().numpy()), t.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def _same(a, b):
    return np.array_equal(np.asarray(a), np.asarray(b), equal_nan=np.asarray(a).dtype.kind == "f")


def test_entry_exponent_is_the_smallest_that_holds():
    for top, e in ((448.0, 0), (448.5, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -100), (1e-44, -100), (3.4e38, 120)):
        assert R.entry_exponent(np.array(top)) == e, top
        assert top <= 448 * 2.0 ** e and (e == -100 or top > 448 * 2.0 ** (e - 1))


def test_mx4_by_hand():
    x = np.zeros((1, 64))
    x[0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9]      # halfway values go to the even code, 7.9 stops at 6
    x[0, 32:35] = [0.5 * 2.0 ** -30, -4.0 * 2.0 ** -30, 0.0]
    codes, scales = R.mx4_quantize(x)
    assert [codes[0, i // 2] >> 4 * (i % 2) & 15 for i in range(8)] == [0, 2, 2, 4, 4, 6, 6, 7]
    assert scales.tolist() == [[127, 97]]
    assert _same(R.mx4_values(codes, scales)[0, :8], [0, 1, 1, 2, 2, 4, 4, 6])
    assert _same(R.mx4_values(codes, scales)[0, 32:35], x[0, 32:35])
    x[0, 5] = np.inf
    codes, scales = R.mx4_quantize(x)
    assert scales.tolist() == [[255, 97]] and np.isnan(R.mx4_values(codes, scales)[0, :32]).all()
    assert R.mx4_quantize(np.zeros((1, 32)))[1].tolist() == [[0]]


def test_layout_struct_matches_the_header(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "sun.h"\nint main(void) { printf("%zu\\n", sizeof(sun_kv8_layout)); return 0; }\n')
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "s")], check=True)
    assert int(subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout) == C.sizeof(sun.Kv8Layout)


def make_pool(lib, shape=wl.TINY, n_pages=5, extra=0):
    cfg, out = sun.make_cfg(shape, "f32"), C.c_void_p()
    nbytes = lib.sun_kv8_pool_bytes(C.byref(cfg), n_pages, 16) + extra
    return cfg, lib.sun_kv8_pool_create(C.byref(cfg), FAKE, nbytes, 16, C.byref(out)), out


@pytest.mark.parametrize("shape", [wl.TINY, wl.SMALL128])
def test_pool_layout_places_every_entry_once(lib, shape):
    cfg, rc, pool = make_pool(lib, shape, 5, 17)
    assert rc == 0
    lay = sun.Kv8Layout()
    assert lib.sun_kv8_pool_layout(pool, C.byref(lay)) == 0
    lib.sun_kv8_pool_destroy(pool)
    nl, hkv, d = shape.n_layers, shape.n_kv_heads, shape.head_dim
    assert (lay.n_pages, lay.page_tokens, lay.total_bytes) == (5, 16, nl * 5 * hkv * 32 * (d + 1))
    mem = np.zeros(lay.total_bytes, np.uint8)
    for v in R.pool_views(mem, lay, nl, hkv, d):
        v += 1
    assert (mem == 1).all()
    assert lay.k_page % 128 == 0 and lay.ks_off % 128 == 0 and (lay.k_token, lay.k_dim, lay.v_token, lay.v_dim) == (d, 1, 1, 16)


def test_pool_refusals(lib):
    cfg, out = sun.make_cfg(wl.TINY, "f32"), C.c_void_p()
    make = lambda *a: lib.sun_kv8_pool_create(*a, C.byref(out))  # noqa: E731
    assert make(None, FAKE, 1 << 20, 16) == 1 and make(C.byref(cfg), None, 1 << 20, 16) == 1
    assert make(C.byref(cfg), FAKE, 1 << 20, 8) == 2
    assert make(C.byref(cfg), FAKE + 16, 1 << 20, 16) == 3 and make(C.byref(cfg), FAKE, 100, 16) == 3
    assert lib.sun_kv8_pool_create(C.byref(cfg), FAKE, 1 << 20, 16, None) == 1
    assert lib.sun_kv8_pool_layout(None, None) == 1
    assert lib.sun_kv8_pool_bytes(C.byref(cfg), 4, 8) == 0
    bad = sun.make_cfg(wl.TINY, "f32")
    bad.head_dim = 96
    assert make(C.byref(bad), FAKE, 1 << 20, 16) == 2


def append_args(pool, **kw):
    a = dict(pool=pool, layer=0, rows=3, dtype=0, q=FAKE, ld_q=256, k=FAKE, ld_k=128, v=FAKE, ld_v=128, positions=FAKE, requests=FAKE,
             tables=FAKE, n_requests=2, max_pages=4, q_norm=None, k_norm=None, q_out=FAKE + 4096, stream=None, flags=0)
    assert set(kw) <= set(a)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("change, status", [
    (dict(pool=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(positions=None), 1), (dict(requests=None), 1), (dict(tables=None), 1),
    (dict(q=None), 2), (dict(q_out=None), 2), (dict(layer=2), 2), (dict(layer=-1), 2), (dict(rows=0), 2), (dict(n_requests=0), 2),
    (dict(max_pages=0), 2), (dict(max_pages=(1 << 26) + 1), 2), (dict(dtype=2), 2), (dict(dtype=-1), 2), (dict(k=FAKE + 8), 2),
    (dict(q_out=FAKE + 4), 2), (dict(ld_k=127), 2), (dict(ld_k=130), 2), (dict(ld_v=64), 2), (dict(ld_q=252), 2), (dict(dtype=1, ld_v=132), 2),
    (dict(q_norm=FAKE), 2), (dict(k_norm=FAKE), 2), (dict(q_out=FAKE, ld_q=512), 2)])
def test_append_refusals(lib, change, status):
    _, rc, pool = make_pool(lib)
    assert rc == 0
    if "pool" not in change:
        change = dict(change, pool=pool)
    assert lib.sun_kv8_append(*append_args(change.pop("pool"), **change)) == status
    assert lib.sun_last_error()
    lib.sun_kv8_pool_destroy(pool)


def test_append_wants_the_gains_of_a_head_norm(lib):
    _, rc, pool = make_pool(lib, wl.TINY_QWEN)
    assert rc == 0
    assert lib.sun_kv8_append(*append_args(pool)) == 1 and lib.sun_kv8_append(*append_args(pool, k_norm=FAKE)) == 1
    assert lib.sun_kv8_append(*append_args(pool, q=None, q_out=None, q_norm=FAKE, k_norm=FAKE)) == 2
    lib.sun_kv8_pool_destroy(pool)


@pytest.mark.parametrize("change, status", [
    (dict(pool=None), 1), (dict(q=None), 1), (dict(tables=None), 1), (dict(n=None), 1), (dict(out=None), 1), (dict(ws=None), 1),
    (dict(layer=2), 2), (dict(layer=-1), 2), (dict(batch=0), 2), (dict(batch=1025), 2), (dict(max_pages=0), 2), (dict(max_pages=(1 << 26) + 1), 2),
    (dict(window=-1), 2), (dict(dtype=7), 2), (dict(q=FAKE + 4), 2), (dict(out=FAKE + 8), 2), (dict(ws=FAKE + 128), 4), (dict(ws_bytes=100), 4)])
def test_attention_refusals(lib, change, status):
    cfg, rc, pool = make_pool(lib)
    assert rc == 0
    a = dict(pool=pool, layer=0, batch=2, dtype=0, q=FAKE, tables=FAKE, max_pages=100, n=FAKE, window=0, out=FAKE, ws=FAKE,
             ws_bytes=lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), 2, 100), stream=None, flags=0)
    assert set(change) <= set(a)
    a.update(change)
    assert lib.sun_kv8_attention(*a.values()) == status
    lib.sun_kv8_pool_destroy(pool)


def chunk(span, batch, hkv):
    ch = 256
    while ch < 2048 and 2 * ch <= span * hkv * batch // 512:
        ch *= 2
    return ch


@pytest.mark.parametrize("hkv, hq", [(1, 8), (2, 4), (8, 40)])
def test_attention_workspace_holds_the_chunks_of_any_length(lib, hkv, hq):
    """Whatever the lengths up to the table's, no request has more chunks than the workspace has room for."""
    shape = wl.Shape("s", 1, 256, hq, hkv, 128, 128, 32)
    cfg = sun.make_cfg(shape, "f32")
    for batch in (1, 3, 24, 64, 256, 1024):
        for pages in (1, 3, 4, 5, 40, 250, 2049):
            most = max(-(-n // chunk(n, batch, hkv)) for n in range(1, pages * 16 + 1))
            room = lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), batch, pages)
            need = batch * most * hq * 130 * 4 if most > 1 else 0
            assert need <= room, (batch, pages)   # and no more than some smaller batch needs, see the next test
    assert lib.sun_kv8_attention_workspace_bytes(None, 1, 1) == 0
    assert lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), 0, 1) == 0 and lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), 1, 0) == 0


@pytest.mark.parametrize("hkv, hq", [(1, 8), (2, 4), (8, 40)])
def test_attention_workspace_serves_fewer_requests(lib, hkv, hq):
    """Fewer requests are cut finer: whatever the batch up to the one that was asked for, its partial results fit."""
    cfg = sun.make_cfg(wl.Shape("s", 1, 256, hq, hkv, 128, 128, 32), "f32")
    for pages in (16, 32, 40, 250, 2049):
        need, room = 0, []
        for batch in range(1, 1025):
            n = pages * 16
            # the most chunks of any length: the longest request of each chunk size
            ends = [n] + [e for ch in (256, 512, 1024, 2048) for e in ((2 * ch * 512 - 1) // (hkv * batch),) if 0 < e <= n]
            most = max(-(-e // chunk(e, batch, hkv)) for e in ends)
            need = max(need, batch * most * hq * 130 * 4 if most > 1 else 0)
            room.append(lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), batch, pages))
            assert room[-1] >= need, (pages, batch)
        assert room == sorted(room) and room[-1] <= need + 256


def test_sizes_beyond_one_launch_are_refused(lib):
    """A launch holds fewer than 2^32 threads: what would take more is an error before anything is enqueued, and has no workspace."""
    cfg, rc, pool = make_pool(lib)
    assert rc == 0
    hkv = wl.TINY.n_kv_heads
    big = C.c_size_t(-1)
    for rows in (1 << 30, (1 << 31) - 1, 1 << 24):
        ld = wl.TINY.n_kv_heads * wl.TINY.head_dim
        assert lib.sun_kv8_append(pool, 0, rows, 0, None, 0, FAKE, ld, FAKE, ld, FAKE, FAKE, FAKE, 1, 1, None, None, None, None, 0) == 2
    for batch, pages in ((1024, 1 << 26), (1024, (1 << 29) // hkv // 128 + 128)):
        assert lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), batch, pages) == 0
        assert lib.sun_kv8_attention(pool, 0, batch, 0, FAKE, FAKE, pages, FAKE, 0, FAKE, FAKE, big, None, 0) == 2
        assert lib.sun_kv8_attention(pool, 0, batch, 0, FAKE, FAKE, pages, FAKE, 4096, FAKE, FAKE, 0, None, 0) == 4   # a window bounds it
    assert lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), 1024, 1 << 16) > 0 and lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), 1025, 4) == 0
    lib.sun_kv8_pool_destroy(pool)
    for n, k, rows in (((1 << 28) + 1, 32, 1), ((1 << 31) - 1, 32, 128), (1, (1 << 31) - 32, 1), (1, 32, (1 << 31) - 1), (1 << 20, 32, 1 << 20)):
        assert lib.sun_mx4_linear_workspace_bytes(n, k, rows) == 0
        assert lib.sun_mx4_linear(FAKE, FAKE, n, k, rows, FAKE, 1, k, FAKE, 1, n, FAKE, big, None) == 2


def test_binding_refuses_counts_beyond_32_bits():
    for good in (0, -1, (1 << 31) - 1, -1 << 31):
        sun._int32(n=good)
    for bad in (1 << 31, 1 << 32, -(1 << 31) - 1):
        with pytest.raises(sun.SunError) as e:
            sun._int32(n=bad)
        assert e.value.status == 2


@pytest.mark.parametrize("args, status", [
    ((None, 0, 4, 64, FAKE, FAKE), 1), ((FAKE, 0, 4, 64, None, FAKE), 1), ((FAKE, 0, 4, 64, FAKE, None), 1), ((FAKE, 2, 4, 64, FAKE, FAKE), 2),
    ((FAKE, 0, 0, 64, FAKE, FAKE), 2), ((FAKE, 0, 4, 0, FAKE, FAKE), 2), ((FAKE, 0, 4, 48, FAKE, FAKE), 2), ((FAKE + 4, 0, 4, 64, FAKE, FAKE), 2),
    ((FAKE, 0, 4, 64, FAKE + 1, FAKE), 2)])
def test_quantize_refusals(lib, args, status):
    w, dtype, rows, cols, codes, scales = args
    assert lib.sun_mx4_quantize(w, dtype, rows, cols, codes, scales, None) == status
    assert lib.sun_mx4_dequantize(codes, scales, rows, cols, dtype, w, None) == status


@pytest.mark.parametrize("change, status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(x=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(N=0), 2), (dict(K=0), 2),
    (dict(K=63), 2), (dict(rows=0), 2), (dict(x_dtype=2), 2), (dict(out_dtype=-1), 2), (dict(codes=FAKE + 8), 2), (dict(x=FAKE + 4), 2), (dict(ld_x=60), 2),
    (dict(ld_x=66), 2), (dict(x_dtype=1, ld_x=68), 2), (dict(ld_out=99), 2), (dict(out=FAKE + 2), 2), (dict(ws=FAKE + 64), 4), (dict(ws_bytes=8), 4)])
def test_linear_refusals(lib, change, status):
    a = dict(codes=FAKE, scales=FAKE, N=100, K=64, rows=40, x=FAKE, x_dtype=0, ld_x=64, out=FAKE, out_dtype=0, ld_out=100, ws=FAKE,
             ws_bytes=lib.sun_mx4_linear_workspace_bytes(100, 64, 40), stream=None)
    assert set(change) <= set(a)
    a.update(change)
    assert lib.sun_mx4_linear(*a.values()) == status


def test_linear_workspace_sizes(lib):
    assert lib.sun_mx4_linear_workspace_bytes(0, 64, 1) == lib.sun_mx4_linear_workspace_bytes(8, 48, 1) == lib.sun_mx4_linear_workspace_bytes(8, 64, 0) == 0
    assert lib.sun_mx4_linear_workspace_bytes(128256, 16384, 4096) >= 3 * 2 * 16384 * 4096   # sizes past 32 bits


@pytest.mark.parametrize("N, K", [(17, 5120), (1000, 4096), (6144, 13824), (28672, 4096)])
def test_linear_workspace_holds_fewer_rows_too(lib, N, K):
    """A call with any number of rows finds enough in a workspace made for more: the size never falls as rows are added."""
    sizes = [lib.sun_mx4_linear_workspace_bytes(N, K, r) for r in range(1, 1200)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("N, K", [(17, 5120), (1000, 4096), (5120, 13824), (28672, 4096), (300, 2080)])
@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls get as far as the launch, which must find no GPU")
def test_linear_workspace_is_enough(lib, N, K):
    """No call with the bytes that were asked for finds them too few: it fails for want of a GPU instead."""
    for rows in list(range(1, 700)) + list(range(700, 6000, 61)):
        need = lib.sun_mx4_linear_workspace_bytes(N, K, rows)
        for x_dtype in (0, 1):
            assert lib.sun_mx4_linear(FAKE, FAKE, N, K, rows, FAKE, x_dtype, K, FAKE, 1, N, FAKE, need, None) not in (0, 2, 4), rows


def test_binding_refuses_what_does_not_fit():
    """Types, shapes and devices are looked at before the library is called; tensors here are on the CPU, which is refused last."""
    x = torch.zeros(4, 64)
    for bad in (lambda: sun.sun_mx4_quantize(x.half()), lambda: sun.sun_mx4_quantize(x[:, :40]), lambda: sun.sun_mx4_quantize(x[0]),
                lambda: sun.sun_mx4_quantize(x[:, ::2]), lambda: sun.sun_mx4_quantize(x),
                lambda: sun.sun_mx4_dequantize(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 3, dtype=torch.uint8)),
                lambda: sun.sun_mx4_dequantize(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), torch.float16)):
        with pytest.raises(sun.SunError) as e:
            bad()
        assert e.value.status == 2


def test_binding_loads_without_a_gpu_build_of_torch(lib):
    """The names that only a GPU build of torch has are not needed to load the module, to ask for sizes or to be refused."""
    code = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2603_02599_amd import binding as sun
assert sun.sun_mx4_linear_workspace_bytes(100, 64, 40) > 0
try:
    sun.sun_mx4_quantize(torch.zeros(4, 64))
except sun.SunError as e:
    print(e.status)
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout.strip() == "2", done.stderr


@pytest.mark.parametrize("d", [64, 128])
def test_bounds_of_the_low_planes_reject_two_planes(d):
    """What 32-bit attention is measured by where only its low bits decide: three planes pass, two do not."""
    q_a, q_b = R.close_queries(12, 8)
    ref, bound = R.close_queries_out(q_a, q_b, d)
    assert (R.cut(q_a, 3) == q_a).all() and (R.cut(q_b, 3) == q_b).all()
    for planes, passes in ((3, True), (2, False)):
        s = ((R.cut(q_a, planes) - R.cut(q_b, planes)) / math.sqrt(d)).astype(np.float32)
        w = np.exp(-np.abs(s))
        out = np.where(s > 0, 1 / (1 + w), w / (1 + w))
        assert ((np.abs(out - ref) <= bound) == passes).all()
    q = R.close_gaps(12, 8, d)
    ref, bound = R.close_gaps_out(q, d)
    w = np.exp(-(q / np.float32(math.sqrt(d)))).astype(np.float32)
    bf16 = lambda x: torch.from_numpy(x).bfloat16().float().numpy()  # noqa: E731
    hi = bf16(w)
    lo = bf16(w - hi)
    for kept, passes in ((hi.astype(np.float64) + lo + bf16(w - hi - lo), True), (hi.astype(np.float64) + lo, False)):
        out = (1 - kept) / (1 + w.astype(np.float64))
        assert (np.abs(out - ref) <= bound).all() == passes
    two = np.abs((1 - hi.astype(np.float64) - lo) / (1 + w.astype(np.float64)) - ref) / bound
    assert (two > 2).sum() > 20


@pytest.mark.parametrize("hkv, hq", [(1, 8), (2, 4), (8, 40)])
def test_attention_window_workspace_is_enough(lib, hkv, hq):
    """Every windowed call that is accepted has a size: it holds the chunks of any length in the window, for fewer requests and shorter windows too."""
    cfg = sun.make_cfg(wl.Shape("s", 1, 256, hq, hkv, 128, 128, 32), "f32")
    whole = lambda b, p: lib.sun_kv8_attention_workspace_bytes(C.byref(cfg), b, p)  # noqa: E731
    size = lambda b, p, w: lib.sun_kv8_attention_window_workspace_bytes(C.byref(cfg), b, p, w)  # noqa: E731
    for pages in (1, 40, 2049, 1 << 26):
        need = 0
        rooms = {w: [] for w in (1, 241, 242, 700, 1500, 40000)}
        for batch in range(1, 1025):
            assert size(batch, pages, 0) == whole(batch, pages) and (whole(batch, pages) == 0 or size(batch, pages, 700) <= whole(batch, pages))
            for window, rooms_of in rooms.items():
                most = min(pages * 16, window + 15)   # the pages in front of a window are whole
                ends = [most] + [e for ch in (256, 512, 1024, 2048) for e in ((2 * ch * 512 - 1) // (hkv * batch),) if 0 < e <= most]
                chunks = max(-(-e // chunk(e, batch, hkv)) for e in ends)
                rooms_of.append((size(batch, pages, window), batch * chunks * hq * 130 * 4 if chunks > 1 else 0))
        for window, rooms_of in rooms.items():
            got, needs = zip(*rooms_of)
            assert all(g >= n and g > 0 for g, n in zip(got, np.maximum.accumulate(needs))), (pages, window)
            assert list(got) == sorted(got) and got[-1] <= max(needs) + 256
        assert all(a[0] <= b[0] for w, v in ((1, 241), (241, 242), (242, 700), (700, 1500), (1500, 40000)) for a, b in zip(rooms[w], rooms[v]))
    assert size(2, 40, -1) == size(0, 40, 5) == size(1025, 40, 5) == size(2, 0, 5) == size(2, (1 << 26) + 1, 5) == 0
    assert lib.sun_kv8_attention_window_workspace_bytes(None, 1, 1, 1) == 0
    assert sun.sun_kv8_attention_window_workspace_bytes(cfg, 256, 8192, 1500) == size(256, 8192, 1500)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls get as far as the launch, which must find no GPU")
def test_windowed_calls_have_the_size_that_they_ask_for(lib):
    """Batches and tables that no call without a window may have: with the bytes that were asked for a windowed one fails for want of a GPU only."""
    cfg, rc, pool = make_pool(lib)
    assert rc == 0
    hkv = wl.TINY.n_kv_heads
    for batch, pages in ((1024, 1 << 26), (1024, (1 << 29) // hkv // 128 + 128), (256, 8192), (1, 1 << 26)):
        for window in (1, 4096, 100000):
            need = lib.sun_kv8_attention_window_workspace_bytes(C.byref(cfg), batch, pages, window)
            assert need > 0
            for w in (1, window // 2 + 1, window):
                assert lib.sun_kv8_attention(pool, 0, batch, 0, FAKE, FAKE, pages, FAKE, w, FAKE, FAKE, need, None, 0) not in (0, 2, 4), (batch, pages, window, w)
    lib.sun_kv8_pool_destroy(pool)


def test_binding_has_no_size_for_counts_beyond_32_bits(lib):
    """Counts that the library takes in 32 bits are not cut to some smaller call's."""
    cfg, far = sun.make_cfg(wl.TINY, "f32"), 1 << 32
    assert sun.sun_mx4_linear_workspace_bytes(100, 64, 40) > 0 and sun.sun_kv8_attention_workspace_bytes(cfg, 2, 100) > 0
    for n, k, rows in ((far + 100, 64, 40), (100, far + 64, 40), (100, 64, far + 40)):
        assert sun.sun_mx4_linear_workspace_bytes(n, k, rows) == 0
    for batch, pages in ((far + 2, 100), (2, far + 100)):
        assert sun.sun_kv8_attention_workspace_bytes(cfg, batch, pages) == sun.sun_kv8_attention_window_workspace_bytes(cfg, batch, pages, 5) == 0
    assert sun.sun_kv8_attention_window_workspace_bytes(cfg, 2, 100, far + 5) == 0
    assert sun.sun_kv8_pool_bytes(cfg, 4, far + 16) == 0 < sun.sun_kv8_pool_bytes(cfg, 4, 16)
