"""Infinite values that reach the cache, and scales that are no numbers: what a row does not see does not touch it, in any form of the
kernels, and a row that sees a page with such a scale is NaN."""
import math

import numpy as np
import pytest

import kv8_reference as ref
from test_kv8_gpu import _attend, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
P = 16

# rows of a sequence, cached tokens with them, KV heads, query heads of each, head dims: single tokens, a few,
# prompts split along the keys, CTAs alone (heads of 64, few rows), pairs
FORMS = [([1, 1], [300, 290], 2, 4, 128), ([3, 2], [300, 290], 1, 4, 64), ([200], [1500], 1, 2, 128),
         ([300], [300], 80, 2, 64), ([140] * 10, [140] * 10, 16, 2, 128), ([600, 520], [900, 520], 16, 2, 128)]


def _rows_that_see(lens, ns, page, window, sinks):
    """For the first sequence: which of its rows see a key of that page."""
    return ref.sees(lens[0] - ns[0] + np.arange(ns[0]), lens[0], window, sinks)[:, page * P:(page + 1) * P].any(axis=1)


def _check(dp, cache, dirty, q, cu, lens, table, see, window, sinks):  # noqa: F811
    scale = 1 / math.sqrt(q.shape[2])
    want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, scale, window, sinks)
    got, _ = _attend(dp, dirty, q, cu, lens, table, window, sinks)
    hit = np.zeros(got.shape[0], bool)
    hit[cu[0]:cu[1]] = see
    assert np.isnan(got[hit]).all(), np.argwhere(~np.isnan(got[hit]))[:5]
    bad = ~(np.abs(got[~hit] - want[~hit]) <= tol[~hit])
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist())
    dp.dptq_last_device_error()


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
@pytest.mark.parametrize("at", [0.4, 0.97])     # of the rows: where the page lies
def test_an_infinite_v_scale_stays_with_the_rows_that_see_it(dp, ns, lens, H, g, D, window, sinks, at):  # noqa: F811
    rng = np.random.default_rng(D + ns[0] + window)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    page = int((lens[0] - ns[0] + at * ns[0] - 1) // P)
    dirty = [a.copy() for a in cache]
    dirty[3][table[0, page]] = np.inf
    dirty[2][table[0, page]] = 0                # as append leaves such a page
    q = _rows(rng, sum(ns), H * g, D)
    see = _rows_that_see(lens, ns, page, window, sinks)
    assert see.any() and (ns[0] < 100 or not see.all())
    _check(dp, cache, dirty, q, cu, lens, table, see, window, sinks)


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS[2:])
def test_an_infinite_value_in_a_prompt_leaves_earlier_tokens_alone(dp, ns, lens, H, g, D):  # noqa: F811
    """Through the cache's own append: one infinite V value in the middle of the first 128 new tokens."""
    rng = np.random.default_rng(D)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    k, v = _rows(rng, sum(ns), H, D), _rows(rng, sum(ns), H, D)
    q = _rows(rng, sum(ns), H * g, D)
    caches = []
    for row in (None, 70):
        now = [a.copy() for a in cache]
        w = v.clone()
        if row is not None:
            w[row, :, 5] = float("inf")
        ref.append(now[0], now[1], k.cpu().numpy(), cu, lens, table)
        ref.append(now[2], now[3], w.cpu().numpy(), cu, lens, table)
        caches.append(now)
    page = int(lens[0] - ns[0] + 70) // P
    assert np.isinf(caches[1][3][table[0, page]]).all()
    _check(dp, caches[0], caches[1], q, cu, lens, table, _rows_that_see(lens, ns, page, 0, 0), 0, 0)


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("kv,value", [(1, np.nan), (1, np.inf), (3, np.nan)])
def test_scales_that_are_no_numbers(dp, ns, lens, H, g, D, kv, value):  # noqa: F811
    """A caller's own cache: a NaN, or an infinite K scale, whatever the page's codes are."""
    rng = np.random.default_rng(D + ns[0])
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    page = int((lens[0] - ns[0] // 2 - 1) // P)
    dirty = [a.copy() for a in cache]
    dirty[kv][table[0, page]] = value
    _check(dp, cache, dirty, _rows(rng, sum(ns), H * g, D), cu, lens, table, _rows_that_see(lens, ns, page, 0, 0), 0, 0)
