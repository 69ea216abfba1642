"""Scale bytes of 255, which sun_kv8_append never writes but another writer of the published layout may: not-a-numbers for the rows that see the token, and for nobody else."""
import pytest
import torch

from test_gpu_kv8 import Cache, make_shape
from test_gpu_kv8_chunk import attend, queries, starts_of

pytestmark = pytest.mark.gpu

# Rows of two query heads a KV head: up to 16 are few places, up to 32 are shared by pairs of waves, and whole tiles; alone, in parts of a long cache, and as tiles that start by their lengths
LAYOUTS = [(4, 2, [12], [90]), (4, 2, [30], [90]), (4, 2, [90], [90]), (4, 2, [200], [300]), (4, 2, [14, 1], [3000, 40]), (4, 2, [29, 3], [3000, 40]), (4, 2, [150, 20], [3000, 40]),
           (128, 64, [600, 20, 9, 31], [600, 530, 9, 31])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [0, 1, 20])
@pytest.mark.parametrize("of", ["v", "k"])
@pytest.mark.parametrize("hq, hkv, counts, lens", LAYOUTS)
def test_a_power_that_is_none_reaches_those_who_see_it(hq, hkv, counts, lens, of, window, dtype):
    cache = Cache(make_shape(hq, hkv, 64), lens)
    cache.fill(0, lens)
    lay, starts = cache.lay, starts_of(counts)
    q = queries(cache.shape, int(starts[-1]), dtype)
    clean = attend(cache, 0, q, starts, lens, window).view(-1, hq, 64).clone()
    assert not torch.isnan(clean).any()
    fine = cache.mem.clone()
    n, c = lens[0], counts[0]
    for t in sorted({n - 1, n - 2, n - c, n - c + 1, n - c // 2, max(n - c - 25, 0), 0}):   # the last token, which one row sees, to one that all see
        cache.mem.copy_(fine)
        head = hkv - 1
        cache.mem[(lay.vs_off if of == "v" else lay.ks_off) + int(cache.table[0, t // 16]) * lay.s_page + head * lay.s_head + t % 16] = 255
        got = attend(cache, 0, q, starts, lens, window).view(-1, hq, 64)
        position = torch.arange(n - c, n, device=got.device)
        bad = torch.zeros(got.shape[:2], dtype=torch.bool, device=got.device)
        bad[:c, 2 * head:] = ((t <= position) & ((t > position - window) if window else True))[:, None]
        assert torch.equal(torch.isnan(got), bad[..., None].expand_as(got)), t
        assert torch.equal(got[~bad], clean[~bad]), t
