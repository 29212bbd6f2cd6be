"""A key with a scale that is no number, beside keys whose K scales binary16 does not hold (below 2^-17) or whose codes it does not
hold times the scale (8192 and more): every query that sees the bad key gets NaN, no other one is touched by it."""
import numpy as np
import pytest

import kv4_reference as ref
from test_kv4_gpu import _attend, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TINY, LARGE, LARGEST = 0x3580, 0x4600, 0x4612     # 2^-20, 8192, 9344
# few rows, one and two row tiles; prompts: alone, heads of 64; alone; cut along the keys; pairs; pairs cut along the keys
FORMS = [([5], [90], 2, 1, 64), ([4], [700], 2, 4, 128), ([300], [900], 80, 2, 64), ([130] * 20, [500] * 20, 8, 1, 128),
         ([200], [3000], 2, 1, 128), ([600], [2700], 20, 2, 128), ([600], [3500], 2, 1, 128)]


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("kv,bits", [(1, 0x7F80), (1, 0x7FC0), (3, 0x7F80), (3, 0x7FC0), (3, 0xBF80)])
@pytest.mark.parametrize("odd", [TINY, LARGE, LARGEST])
def test_a_bad_key_beside_odd_scales(dp, ns, lens, H, g, D, kv, bits, odd):  # noqa: F811
    rng = np.random.default_rng(H + D + odd)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    q = _rows(rng, sum(ns), H * g, D)
    n, L = ns[0], int(lens[0])
    key = L - n // 2 - 1                       # (some rows of the first sequence see it, some do not)
    # the other one of two neighbours, both in the same 16 bytes of every lane's rows
    cache[1][table[0, (key ^ 1) // 16], :, (key ^ 1) % 16] = odd
    dirty = [a.copy() for a in cache]
    dirty[kv][table[0, key // 16], :, key % 16] = bits
    clean, _ = _attend(dp, cache, q, cu, lens, table)
    got, _ = _attend(dp, dirty, q, cu, lens, table)
    hit = np.zeros(got.shape[0], bool)
    hit[:n] = L - n + np.arange(n) >= key
    assert 0 < hit.sum() < n and not np.isnan(clean).any()
    assert np.isnan(got[hit]).all()
    assert np.array_equal(got[~hit], clean[~hit])
    dp.dptq_last_device_error()
