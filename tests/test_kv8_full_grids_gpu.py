"""dptq_kv8_attention on grids that fill the GPU: prompts there are not split along the keys, and long
ones with heads of 128 are taken by pairs of CTAs."""
import numpy as np
import pytest

import kv8_reference as ref
from test_kv8_gpu import _attend, _check_attend, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ns,lens,H,g,P", [
    ([700, 1, 300, 513], [1500, 5, 300, 640], 8, 2, 16),       # ragged, behind contexts
    ([256] * 3, [256, 400, 1000], 16, 2, 64),                  # whole tiles of rows
    ([257, 130], [257, 2000], 12, 3, 128),                     # odd groups, the last pair nearly empty
    ([90] * 40, list(range(90, 130)), 4, 1, 32)])              # one row tile a sequence
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 5)])
def test_prompts(dp, D, ns, lens, H, g, P, window, sinks):  # noqa: F811
    rng = np.random.default_rng(D + H + window)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    _check_attend(dp, cache, _rows(rng, sum(ns), H * g, D, 8), cu, lens, table, window, sinks)


def test_rows_without_keys_zero_pages_and_a_nan_query(dp):  # noqa: F811
    rng = np.random.default_rng(4)
    ns, lens = [600, 520, 300], [0, 500, 900]                  # nothing cached; 20 rows without a place
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, 8, 16, 128)
    for b in rng.choice(blocks, blocks // 3, replace=False):
        for a in cache:
            a[b] = 0
    q = _rows(rng, sum(ns), 16, 128)
    _check_attend(dp, cache, q, cu, lens, table)
    got, _ = _attend(dp, cache, q, cu, lens, table)
    again, _ = _attend(dp, cache, q, cu, lens, table)
    assert np.array_equal(got, again)
    bad = q.clone()
    bad[1400, 5, 3] = float("nan")
    again, _ = _attend(dp, cache, bad, cu, lens, table)
    assert np.isnan(again[1400, 5]).all()
    got[1400, 5] = again[1400, 5] = 0
    assert np.array_equal(got, again)


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_flat_and_sharp_softmax(dp, scale):  # noqa: F811
    rng = np.random.default_rng(9)
    cu, lens, table, blocks = ref.random_batch(rng, [520, 300], [777, 300], 64)
    cache = ref.random_cache(rng, blocks, 16, 64, 128)
    cache[1][:] = np.float32(1 / 127)
    _check_attend(dp, cache, _rows(rng, 820, 32, 128), cu, lens, table, scale=scale)
