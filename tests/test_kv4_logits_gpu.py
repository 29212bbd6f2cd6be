"""Logits over the 4-bit cache where a channel of the query is far larger than the others and the keys have the code 0 there: their
error goes by the sum of |q k|, not by the sum of |q|."""
import numpy as np
import pytest

import kv4_reference as ref
from test_kv4_gpu import _check, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ns,lens,H,g,D", [([1], [300], 2, 1, 128), ([1, 1], [2000, 33], 2, 8, 128), ([1, 1], [700, 5], 2, 4, 64),
                                           ([4], [900], 1, 4, 128), ([3], [500], 2, 5, 64), ([40], [500], 1, 2, 128)])
@pytest.mark.parametrize("large", [300.0, 30000.0])
def test_a_large_query_channel_over_codes_of_zero(dp, ns, lens, H, g, D, large):  # noqa: F811
    rng = np.random.default_rng(D + H + g)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    codes = ref.unpack(cache[0])
    codes[..., [5, D // 2 + 2]] = 0
    cache[0] = ref.pack(codes)
    cache[1][:] = ref.bf16_bits(rng.uniform(1.0, 3.0, cache[1].shape).astype(np.float32))
    q = _rows(rng, sum(ns), H * g, D)
    q[:, :, 5], q[:, :, D // 2 + 2] = large, 0.75 * large
    _check(dp, cache, q, cu, lens, table, scale=0.02)
