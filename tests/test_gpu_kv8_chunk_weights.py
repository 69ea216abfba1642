"""The softmax's weights of chunk attention in bf16 calls: 16 bits, as in the attention of single tokens, against the sum of the same weights."""
import numpy as np
import pytest
import torch

import lowbit_ref as R
import test_gpu_kv8_chunk as chunk
from test_gpu_kv8 import DEV, Cache, i32, make_shape
from test_gpu_kv8_chunk import attend, check, starts_of

pytestmark = pytest.mark.gpu


def bound(ref, mass, reach, n, d, dtype):
    """test_gpu_kv8_chunk.py's with weights of two planes: bf16 of the weight, off by 2^-8 of it, and bf16 of what is left, off by 2^-8 of that.  Twice as many products are summed."""
    assert dtype == "bf16"
    score = reach[..., None] * (d + 4) * 2.0 ** -24
    weight = 2 * score + 2.0 ** -21 + 2.0 ** -16
    return mass * (weight + 3 * (n + 8) * 2.0 ** -24) + np.abs(ref) * R.HALF[dtype] * 1.01 + 1e-37


@pytest.mark.parametrize("hq, hkv, d, counts, lens", [
    (4, 1, 64, [1, 5, 8], [40, 100, 600]), (8, 2, 128, [9, 16, 12], [90, 300, 16]), (8, 2, 128, [200, 33, 70], [200, 700, 70]), (5, 1, 128, [3, 60, 9], [6000, 300, 4000]),
    (64, 64, 64, [520, 30, 200], [520, 600, 200])])
@pytest.mark.parametrize("window", [0, 50])
def test_what_values_that_cancel_leave(hq, hkv, d, counts, lens, window, monkeypatch):
    """Values of both signs: much of their weighted sum cancels, so that the output's own rounding is small against what the weights' would be."""
    monkeypatch.setattr(chunk, "bound", bound)
    cache = Cache(make_shape(hq, hkv, d), lens)
    cache.fill(0, lens)
    check(cache, 0, counts, lens, "bf16", window=window)
    check(cache, 0, counts, lens, "bf16", window=window, scale=0.3)   # weights close to each other


@pytest.mark.parametrize("count", [1, 7, 16, 30, 60, 300])
@pytest.mark.parametrize("n", [400, 5000])
def test_weights_that_all_round_alike(n, count):
    """One token with a high score in front of many with 0, all values 1: a mean of ones, whatever the weights are.  The high score, (5.5 + 2^-6) / sqrt(64), makes the others'
    weights 1.0037 times a power of two, which 8 bits would all take down to it."""
    cache = Cache(make_shape(4, 2, 64), [n])
    m = cache.mem.cpu().numpy().copy()
    k, v, ks, vs = R.pool_views(m, cache.lay, 2, 2, 64)
    t = np.arange(n)
    page, slot = cache.table[0, t // 16], t % 16
    k[0][page, :, slot], ks[0][page, :, slot] = 0, 127
    v[0][page, :, :, slot], vs[0][page, :, slot] = 0x38, 127   # 1
    k[0][cache.table[0, 0], :, 0, :2] = 0x38
    cache.mem.copy_(torch.from_numpy(m))
    q = torch.zeros(count, 4, 64, device=DEV)
    q[..., 0], q[..., 1] = 5.5, 2.0 ** -6
    out = attend(cache, 0, q.view(count, -1).bfloat16(), starts_of([count]), [n])
    assert (out == 1).all()


def test_a_chunk_of_one_token_is_as_good_as_the_single_token_call():
    """Both within the same bound of the 64-bit value."""
    lens = [1, 17, 300, 2500]
    cache = Cache(make_shape(8, 2, 128), lens)
    cache.fill(0, lens)
    q = chunk.queries(cache.shape, 4, "bf16")
    got = attend(cache, 0, q, range(5), lens)
    single = torch.zeros_like(q)
    ws = torch.zeros(chunk.sun.sun_kv8_attention_workspace_bytes(cache.cfg, 4, cache.table.shape[1]), dtype=torch.uint8, device=DEV)
    chunk.sun.sun_kv8_attention(cache.pool, 0, q, cache.dev_table, i32(lens), single, ws)
    views = cache.views()
    for i, n in enumerate(lens):
        ref, mass, reach = R.attention(chunk.host(q[i]).reshape(8, 128), views, 0, cache.table[i], n, 0, 2, cache.n_pages)
        for out in (got, single):
            assert (np.abs(chunk.host(out[i]).reshape(8, 128) - ref) <= bound(ref, mass, reach, n, 128, "bf16")).all(), n
