"""Prompts over the 4-bit cache that pairs of CTAs take (heads of 128, at least 512 rows of a sequence and KV head that see some
2000 keys), whole tasks (20 heads) and tasks cut along their keys (4)."""
import numpy as np
import pytest

import kv4_reference as ref
from test_kv4_gpu import _attend, _rows, dp  # noqa: F401  (dp: the fixture)
from test_kv4_prompts_gpu import _against_doubles

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NS, LENS, G = [600, 0, 530], [2700, 40, 2500], 2


def _case(H, P=16, seed=0, ns=NS, lens=LENS):
    rng = np.random.default_rng(seed + H)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P, spare=3)
    return rng, cu, lens, table, ref.random_cache(rng, blocks, H, P, 128), _rows(rng, sum(ns), H * G, 128, pad=24)


@pytest.mark.parametrize("H", [20, 4])
@pytest.mark.parametrize("P,window,sinks", [(16, 0, 0), (128, 0, 0), (32, 2600, 3), (64, 2300, 400)])
def test_values(dp, H, P, window, sinks):  # noqa: F811
    _, cu, lens, table, cache, q = _case(H, P)
    _against_doubles(dp, cache, q, cu, lens, table, window, sinks)


@pytest.mark.parametrize("H", [20, 4])
def test_the_same_bits_every_time(dp, H):  # noqa: F811
    _, cu, lens, table, cache, q = _case(H)
    first, _ = _attend(dp, cache, q, cu, lens, table)
    for _ in range(5):
        again, _ = _attend(dp, cache, q, cu, lens, table)
        assert np.array_equal(first, again)


@pytest.mark.parametrize("H", [20, 4])
@pytest.mark.parametrize("kv,bits", [(1, 0x7F80), (1, 0x7FC0), (3, 0xFF80), (3, 0x7FFF)])
def test_a_scale_that_is_no_number_stays_with_the_rows_that_see_it(dp, H, kv, bits):  # noqa: F811
    _, cu, lens, table, cache, q = _case(H)
    for key in (5, 2400):
        dirty = [a.copy() for a in cache]
        dirty[kv][table[0, key // 16], :, key % 16] = bits
        got, _ = _attend(dp, dirty, q, cu, lens, table, 0, 0)
        clean, _ = _attend(dp, cache, q, cu, lens, table, 0, 0)
        hit = np.zeros(got.shape[0], bool)
        hit[:600] = 2100 + np.arange(600) >= key
        assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])
    dp.dptq_last_device_error()


@pytest.mark.parametrize("H", [20, 4])
def test_nan_queries_and_what_no_query_sees(dp, H):  # noqa: F811
    rng, cu, lens, table, cache, q = _case(H)
    W = 2100
    got, _ = _attend(dp, cache, q, cu, lens, table, W, 3)
    other, bad = [a.copy() for a in cache], q.clone()
    hidden = [b for b in range(cache[0].shape[0]) if b not in table[2] and b not in table[0]]
    for b in hidden:
        other[1][b], other[3][b], other[0][b], other[2][b] = 0x7FC0, 0x7F80, 0x88, 0x77
    last, used = table[2, 2499 // 16], 2499 % 16 + 1
    other[1][last, :, used:], other[3][last, :, used:], other[2][last, :, used:] = 0x4612, 0x4612, 0x88
    bad[3, 1, 100] = float("nan")
    again, _ = _attend(dp, other, bad, cu, lens, table, W, 3)
    assert np.isnan(again[3, 1]).all()
    got[3, 1] = again[3, 1] = 0
    assert np.array_equal(got, again)
    dp.dptq_last_device_error()


@pytest.mark.parametrize("H", [20, 4])
def test_scales_far_apart_and_growing_maxima(dp, H):  # noqa: F811
    rng, cu, lens, table, cache, q = _case(H)
    cache[3][:] = ref.bf16_bits((2.0 ** rng.uniform(-30, 10, cache[3].shape)).astype(np.float32))
    for x in (1, 3):
        cache[x][rng.random(cache[x].shape) < 0.25] = 0
    _against_doubles(dp, cache, q, cu, lens, table)
    cache[0][:] = 0x11
    for s in (0, 2):
        for p in range(-(-int(lens[s]) // 16)):
            cache[1][table[s, p]] = ref.bf16_bits(((p * 16 + np.arange(16)) / 512).astype(np.float32))
    cache[3][:] = ref.bf16_bits(np.float32(0.5))
    _against_doubles(dp, cache, (1 + 0.1 * q).half(), cu, lens, table)


@pytest.mark.parametrize("H", [20, 4])
def test_pages_that_are_not_there(dp, H):  # noqa: F811
    """They read as pages without keys and are reported; the other sequence is served."""
    _, cu, lens, table, cache, q = _case(H)
    want, _ = _attend(dp, cache, q, cu, lens, table)
    missing = table.copy()
    missing[0, 3], missing[0, 80], missing[0, 168] = 1 << 30, -9, cache[0].shape[0]
    c2 = [a.copy() for a in cache]
    got, _ = _attend(dp, c2, q, cu, lens, missing)
    with pytest.raises(dp.DptqError) as e:
        dp.dptq_last_device_error()
    assert e.value.status == 1
    assert np.array_equal(got[600:], want[600:]) and np.isfinite(got).all()
    # the same as a cache whose keys there have no weight: their logits far below all others
    direct = torch.from_numpy(got[599].astype(np.float64))
    pages = [p for p in range(-(-2700 // 16)) if p not in (3, 80, 168)]
    K, V = (ref.values(cache[i], cache[i + 1])[table[0, pages]].transpose(1, 0, 2, 3).reshape(H, -1, 128).astype(np.float64)
            for i in (0, 2))
    keys = np.concatenate([np.arange(16 * p, 16 * p + 16) for p in pages]) < 2700
    x = q[599].cpu().numpy().astype(np.float64)
    for h in range(H):
        a = x[h * G:(h + 1) * G] @ K[h][keys].T / np.sqrt(128)
        w = np.exp(a - a.max(axis=1, keepdims=True))
        o = (w / w.sum(axis=1, keepdims=True)) @ V[h][keys]
        # weights and output rounded to binary16, values up to 9
        assert np.abs(direct[h * G:(h + 1) * G].numpy() - o).max() < 2.0 ** -10 * 9
