"""Prompts that pairs of CTAs take (heads of 128, at least 512 rows of a sequence and KV head, a grid
that fills the GPU)."""
import math

import numpy as np
import pytest

import kv8_reference as ref
from test_kv8_gpu import _attend, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P", [16, 128])
def test_many_tiles_of_unlike_pages_the_same_bits_every_time(dp, P):  # noqa: F811
    """Scales that differ by binades from page to page, in each of 24 tiles of keys: a tile that met
    another one's codes or scales would be far outside the tolerance."""
    rng = np.random.default_rng(P)
    ns, lens, H, g = [700, 513, 300], [3000, 2500, 300], 16, 2
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, 128)
    q = _rows(rng, sum(ns), H * g, 128)
    got, scale = _attend(dp, cache, q, cu, lens, table)
    want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, scale)
    assert (np.abs(got - want) <= tol).all()
    assert scale == 1 / math.sqrt(128)
    for _ in range(10):
        again, _ = _attend(dp, cache, q, cu, lens, table)
        assert np.array_equal(got, again)
    dp.dptq_last_device_error()
