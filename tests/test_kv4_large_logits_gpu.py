"""Attention over the 4-bit cache with logits up to 10^10: the largest queries and K scales that there are.  fp32 has steps of more
than 2^10 there, so what is expected does not depend on roundings: one key far above the others, all keys alike, keys far
below the others that the same rows see."""
import numpy as np
import pytest

import kv4_reference as ref
from test_kv4_gpu import _attend, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LARGEST = 0x4612     # 9344
# few rows, one and two row tiles; prompts: alone, heads of 64; alone; cut along the keys; pairs; pairs cut along the keys
FORMS = [([1], [90], 2, 1, 64), ([1, 1], [2000, 700], 2, 8, 128), ([4], [700], 2, 4, 128), ([300], [900], 8, 2, 64),
         ([130] * 20, [500] * 20, 8, 1, 128), ([200], [3000], 2, 1, 128), ([600], [2700], 20, 2, 128), ([600], [3500], 2, 1, 128)]


def _case(ns, lens, H, g, D):
    rng = np.random.default_rng(H + D + sum(ns))
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    cache[3][:] = ref.bf16_bits(np.float32(0.5))
    return cu, lens, table, cache, _rows(rng, sum(ns), H * g, D)


def _values(cache, table, s, L, H, D):
    """V of a sequence's keys, float64 [heads, L, D]."""
    pages = table[s, :-(-L // 16)]
    return ref.values(cache[2][pages], cache[3][pages]).transpose(1, 0, 2, 3).reshape(H, -1, D)[:, :L].astype(np.float64)


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("size", [65504.0, 3000.0, 100.0, -65504.0])
def test_keys_alike(dp, ns, lens, H, g, D, size):  # noqa: F811
    """The mean of V over what a row sees: the same products in the same order give every key the same logit."""
    cu, lens, table, cache, q = _case(ns, lens, H, g, D)
    cache[0][:], cache[1][:] = 0x77, LARGEST
    q[:] = size
    got, _ = _attend(dp, cache, q, cu, lens, table)
    for s, (n, L) in enumerate(zip(ns, lens)):
        V = _values(cache, table, s, L, H, D)
        count = np.arange(1, L + 1)[:, None]
        mean, mag = (np.cumsum(v, axis=1)[:, L - n:] / count[L - n:] for v in (V, np.abs(V)))      # [H, n, D]
        mean, mag = (np.repeat(v, g, axis=0).transpose(1, 0, 2) for v in (mean, mag))
        # weights rounded to binary16 (alike: a power of two, none), fp32 sums of up to L terms, the output's rounding
        tol = 2.0 ** -11 * np.abs(mean) + (2.0 ** -11 + (L / 16 + 64) * 2.0 ** -23) * mag + 2.0 ** -24
        assert (np.abs(got[cu[s]:cu[s + 1]] - mean) <= tol).all()
    dp.dptq_last_device_error()


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("size", [65504.0, 2000.0, 20.0])
@pytest.mark.parametrize("growing", [False, True])
def test_one_key_above_all_others(dp, ns, lens, H, g, D, size, growing):  # noqa: F811
    """Its V, to one rounding: with 2^-4 of its logit, 10^4 and more, between it and the next one.  growing: every key's
    logit is above the one before."""
    cu, lens, table, cache, q = _case(ns, lens, H, g, D)
    cache[0][:] = 0x77
    q[:] = size
    at = []
    for s, (n, L) in enumerate(zip(ns, lens)):
        cache[1][table[s]] = ref.bf16_bits(np.float32(8192 / 16))
        keys = [0, L // 3] if not growing else [L // 5, L // 4, L // 2, L - n]      # (every row sees them all)
        for i, k in enumerate(keys):
            cache[1][table[s, k // 16], :, k % 16] = ref.bf16_bits(np.float32(8192 * (16 - len(keys) + 1 + i) / 16))
        at.append(keys[-1])
    got, _ = _attend(dp, cache, q, cu, lens, table)
    for s, L in enumerate(lens):
        want = np.repeat(_values(cache, table, s, L, H, D)[:, at[s]], g, axis=0)
        assert np.array_equal(got[cu[s]:cu[s + 1]], np.broadcast_to(want, got[cu[s]:cu[s + 1]].shape).astype(np.float16))
    dp.dptq_last_device_error()


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
def test_keys_far_below(dp, ns, lens, H, g, D):  # noqa: F811
    """The first third of the keys has logits of -10^9 and less: the result is that of the others alone."""
    cu, lens, table, cache, q = _case(ns, lens, H, g, D)
    # ordinary logits come from the first half of the dims, over codes of zero in the second one, where queries are large
    q[:, :, :D // 2] *= 2 ** 9
    q[:, :, D // 2:] = -(q[:, :, D // 2:].abs() + 2 ** 13)
    codes = ref.unpack(cache[0])
    codes[..., D // 2:] = 0
    cache[0], cache[1][:] = ref.pack(codes), ref.bf16_bits(np.float32(2.0 ** -10))
    others = table.copy()
    for s, L in enumerate(lens):
        below = table[s, :L // 48]
        cache[0][below], cache[1][below] = 0x77, LARGEST
        others[s, :L // 48] = -1
    got, scale = _attend(dp, cache, q, cu, lens, table)
    want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, others, scale)
    assert tol.max() < 0.1 and (np.abs(got - want) <= tol).all()
    dp.dptq_last_device_error()


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (77, 3)])
def test_rows_beside_large_ones(dp, ns, lens, H, g, D, window, sinks):  # noqa: F811
    """A row's bits do not depend on rows of far larger logits beside it, whose own results stay among the values of V."""
    cu, lens, table, cache, q = _case(ns, lens, H, g, D)
    clean, _ = _attend(dp, cache, q, cu, lens, table, window, sinks)
    large = np.zeros(clean.shape[:2], bool)
    large[::3, 0], large[-1, H * g - 1] = True, True
    mixed = q.clone()
    mixed[torch.from_numpy(large)] *= 10000.0
    got, _ = _attend(dp, cache, mixed, cu, lens, table, window, sinks)
    assert np.array_equal(got[~large], clean[~large])
    assert (np.abs(got[large]) <= 3.5 * (1 + 2.0 ** -10)).all() and np.abs(got[large]).max() > 1
    dp.dptq_last_device_error()
