"""Chunk attention over the 8-bit cache, the gated pair and the product with an epilogue without a GPU: workspace sizes and every refusal that happens before anything is
enqueued."""
import ctypes as C

import pytest
import torch

from paper_2603_02599_amd import binding as sun
from paper_2603_02599_amd import workloads as wl
from test_lowbit_cpu import FAKE, lib, make_pool  # noqa: F401

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the calls get as far as the launch, which must find no GPU")


def chunk_args(lib, cfg, pool, **change):
    a = dict(pool=pool, layer=0, batch=2, rows=5, dtype=0, q=FAKE, starts=FAKE, tables=FAKE, max_pages=100, n=FAKE, window=0, out=FAKE + 65536, ws=FAKE,
             ws_bytes=lib.sun_kv8_chunk_attention_workspace_bytes(C.byref(cfg), 2, 5, 100), stream=None, flags=0)
    assert set(change) <= set(a)
    a.update(change)
    return list(a.values())


@pytest.mark.parametrize("change, status", [
    (dict(pool=None), 1), (dict(q=None), 1), (dict(starts=None), 1), (dict(tables=None), 1), (dict(n=None), 1), (dict(out=None), 1), (dict(ws=None), 1),
    (dict(layer=2), 2), (dict(layer=-1), 2), (dict(batch=0), 2), (dict(batch=1025), 2), (dict(rows=0), 2), (dict(rows=-4), 2), (dict(max_pages=0), 2), (dict(max_pages=(1 << 26) + 1), 2),
    (dict(window=-1), 2), (dict(dtype=7), 2), (dict(q=FAKE + 4), 2), (dict(out=FAKE + 8), 2), (dict(out=FAKE), 2), (dict(rows=(1 << 31) - 1), 2), (dict(ws=FAKE + 128), 4), (dict(ws_bytes=100), 4)])
def test_chunk_attention_refusals(lib, change, status):  # noqa: F811
    cfg, rc, pool = make_pool(lib)
    assert rc == 0
    assert lib.sun_kv8_chunk_attention(*chunk_args(lib, cfg, **{"pool": pool, **change})) == status
    assert lib.sun_last_error()
    lib.sun_kv8_pool_destroy(pool)


@no_gpu
@pytest.mark.parametrize("shape", [wl.TINY, wl.SMALL_G5, wl.LLAMA_8B])
def test_chunk_attention_workspace_is_enough_for_fewer(lib, shape):  # noqa: F811
    """No call with the bytes that were asked for finds them too few, with as many rows and requests or fewer: it fails for want of a GPU instead."""
    cfg, rc, pool = make_pool(lib, shape)
    assert rc == 0
    for batch, rows in ((1, 1), (1, 2048), (3, 40), (64, 256), (17, 3000), (1024, 1024), (700, 20000)):
        for pages in (1, 16, 17, 512, 1 << 20):
            size = lib.sun_kv8_chunk_attention_workspace_bytes(C.byref(cfg), batch, rows, pages)
            for b in {1, 2, batch // 2, batch - 1, batch} - {0}:
                for r in {1, 2, 7, 31, 33, rows // 3, rows // 2, rows - 1, rows}:
                    if b <= batch and 0 < r <= rows:
                        assert lib.sun_kv8_chunk_attention(*chunk_args(lib, cfg, pool, batch=b, rows=r, max_pages=pages, ws_bytes=size)) == 8, (b, r, batch, rows, pages)
    lib.sun_kv8_pool_destroy(pool)


def test_chunk_attention_has_no_size_for_what_it_refuses(lib):  # noqa: F811
    cfg = sun.make_cfg(wl.TINY, "f32")
    size = lib.sun_kv8_chunk_attention_workspace_bytes
    assert size(None, 1, 1, 1) == size(C.byref(cfg), 0, 1, 1) == size(C.byref(cfg), 1025, 1, 1) == size(C.byref(cfg), 1, 0, 1) == size(C.byref(cfg), 1, 1, 0) == 0
    assert size(C.byref(cfg), 1, 1, (1 << 26) + 1) == size(C.byref(cfg), 1, (1 << 31) - 1, 1) == 0 and size(C.byref(cfg), 1024, 1 << 24, 1 << 26) > 0
    big = sun.make_cfg(wl.LLAMA_8B, "f32")
    assert size(C.byref(big), 1024, 1 << 23, 1 << 26) > 0   # as documented
    assert sun.sun_kv8_chunk_attention_workspace_bytes(cfg, 1 << 31, 1, 1) == sun.sun_kv8_chunk_attention_workspace_bytes(cfg, 1, 1 << 32, 1) == 0
    assert sun.sun_mx4_gated_workspace_bytes(1 << 31, 32, 1) == 0


LINEAR = dict(N=100, K=64, rows=40, x=FAKE, x_dtype=0, ld_x=64)


@pytest.mark.parametrize("change, status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(x=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(N=0), 2), (dict(K=63), 2), (dict(rows=0), 2), (dict(x_dtype=2), 2),
    (dict(out_dtype=-1), 2), (dict(codes=FAKE + 8), 2), (dict(ld_x=60), 2), (dict(ld_out=99), 2), (dict(out=FAKE + 2), 2), (dict(ws=FAKE + 64), 4), (dict(ws_bytes=8), 4),
    (dict(activation=4), 2), (dict(activation=-1), 2), (dict(bias=FAKE + 2), 2), (dict(residual=FAKE + 2), 2), (dict(residual=FAKE, ld_residual=99), 2), (dict(out_dtype=1, bias=FAKE + 1), 2),
    (dict(residual=FAKE + 4096, ld_residual=104), 2), (dict(N=(1 << 28) + 1), 2), (dict(rows=(1 << 31) - 1), 2)])
def test_fused_refusals(lib, change, status):  # noqa: F811
    a = dict(codes=FAKE, scales=FAKE, **LINEAR, bias=FAKE, activation=1, residual=FAKE + 4096, ld_residual=100, out=FAKE + 4096, out_dtype=0, ld_out=100, ws=FAKE,
             ws_bytes=lib.sun_mx4_linear_workspace_bytes(100, 64, 40), stream=None)
    assert set(change) <= set(a)
    a.update(change)
    assert lib.sun_mx4_linear_fused(*a.values()) == status


@pytest.mark.parametrize("change, status", [
    (dict(gate=None), 1), (dict(gate_scales=None), 1), (dict(up=None), 1), (dict(up_scales=None), 1), (dict(x=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(N=0), 2), (dict(K=63), 2),
    (dict(rows=0), 2), (dict(x_dtype=2), 2), (dict(out_dtype=-1), 2), (dict(gate=FAKE + 8), 2), (dict(up=FAKE + 8), 2), (dict(ld_x=60), 2), (dict(ld_out=99), 2), (dict(out=FAKE + 2), 2),
    (dict(ws=FAKE + 64), 4), (dict(ws_bytes=8), 4), (dict(activation=4), 2), (dict(N=(1 << 27) + 1), 2), (dict(N=(1 << 31) - 1), 2)])
def test_gated_refusals(lib, change, status):  # noqa: F811
    a = dict(gate=FAKE, gate_scales=FAKE, up=FAKE, up_scales=FAKE, **LINEAR, activation=1, out=FAKE, out_dtype=0, ld_out=100, ws=FAKE,
             ws_bytes=lib.sun_mx4_gated_workspace_bytes(100, 64, 40), stream=None)
    assert set(change) <= set(a)
    a.update(change)
    assert lib.sun_mx4_gated(*a.values()) == status


@no_gpu
@pytest.mark.parametrize("N, K", [(17, 5120), (1000, 4096), (300, 2080)])
def test_gated_workspace_is_enough(lib, N, K):  # noqa: F811
    sizes = []
    for rows in list(range(1, 300)) + list(range(300, 4000, 61)):
        need = lib.sun_mx4_gated_workspace_bytes(N, K, rows)
        sizes.append(need)
        for x_dtype in (0, 1):
            assert lib.sun_mx4_gated(FAKE, FAKE, FAKE, FAKE, N, K, rows, FAKE, x_dtype, K, 1, FAKE, 1, N, FAKE, need, None) == 8, rows
    assert sizes == sorted(sizes)   # enough for fewer rows too


def test_binding_refuses_on_the_cpu():
    x = torch.zeros(4, 64)
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8)
    for bad in (lambda: sun.sun_mx4_linear_fused(codes, scales, x, torch.zeros(4, 8), x), lambda: sun.sun_mx4_gated(codes, scales, codes, scales, x, torch.zeros(4, 8), x)):
        with pytest.raises(sun.SunError) as e:
            bad()
        assert e.value.status == 2
