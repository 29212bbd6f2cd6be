"""Argument checks of the 4-bit cache's entry points that are made before CUDA is touched, and the test
reference's own pins."""
import ctypes
import math

import numpy as np
import pytest

import kv4_reference as ref

P, F = ctypes.c_void_p, ctypes.c_float


@pytest.fixture(scope="module")
def dp():
    from paper_2606_12487_gb300 import dptq
    dptq.load()
    return dptq


def _handles(dp, cache=None, batch=None):
    c = dp._Kv4CacheC(*([64] * 4), 10, 2, 16, 128)
    b = dp._Kv8BatchC(*([64] * 3), 3, 5, 7, 4, 80)
    for k, v in (cache or {}).items():
        setattr(c, k, v)
    for k, v in (batch or {}).items():
        setattr(b, k, v)
    return c, b


@pytest.mark.parametrize("cache,batch,want", [
    (dict(head_dim=96), {}, 2), (dict(head_dim=256), {}, 2), (dict(head_dim=0), {}, 1), (dict(block_tokens=8), {}, 2),
    (dict(block_tokens=48), {}, 2), (dict(block_tokens=256), {}, 2), (dict(block_tokens=-16), {}, 1),
    (dict(num_blocks=1 << 27), {}, 2), (dict(num_blocks=0), {}, 1), (dict(kv_heads=0), {}, 1), (dict(kv_heads=1024), {}, 2), (dict(k_codes=None), {}, 1),
    (dict(v_codes=72), {}, 1), (dict(k_scales=None), {}, 1), (dict(k_scales=72), {}, 1), (dict(v_scales=66), {}, 1),
    ({}, dict(seqs=-1), 1), ({}, dict(seqs=65536), 2), ({}, dict(tokens=-1), 1), ({}, dict(max_tokens=-1), 1),
    ({}, dict(max_tokens=65536, tokens=70000), 2), ({}, dict(max_len=(1 << 27) + 1, table_stride=1 << 28), 2),
    ({}, dict(max_len=-1), 1), ({}, dict(max_len=81), 1), ({}, dict(block_table=None), 1), ({}, dict(cu_tokens=None), 1),
    ({}, dict(seq_lens=None), 1), ({}, dict(cu_tokens=66), 1), ({}, dict(seq_lens=67), 1), ({}, dict(block_table=65), 1),
    ({}, dict(seqs=0), 0), ({}, dict(tokens=0), 0), ({}, dict(max_tokens=0), 0)])
def test_cache_and_batch(dp, cache, batch, want):
    c, b = _handles(dp, cache, batch)
    lib = dp.load()
    cp, bp = ctypes.addressof(c), ctypes.addressof(b)
    assert lib.dptq_kv4_append(cp, bp, P(64), P(64), 256, None) == want
    assert lib.dptq_kv4_read(cp, bp, P(64), P(64), 256, None) == want
    heads = 8 * max(1, c.kv_heads)
    assert lib.dptq_kv4_attention(cp, bp, P(64), 8 * heads * 128, heads, F(0.1), 0, 0, P(64), 8 * heads * 128, None) == want


def test_scalars(dp):
    c, b = _handles(dp)
    lib = dp.load()
    cp, bp, att = ctypes.addressof(c), ctypes.addressof(b), lib.dptq_kv4_attention
    for call in (lib.dptq_kv4_append, lib.dptq_kv4_read):
        assert call(None, bp, P(64), P(64), 256, None) == 1
        assert call(cp, None, P(64), P(64), 256, None) == 1
    assert att(cp, None, P(64), 1024, 8, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 0, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 7, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 130 * 128, 130, F(0.1), 0, 0, P(64), 130 * 128, None) == 2
    for scale in (math.inf, math.nan):
        assert att(cp, bp, P(64), 1024, 8, F(scale), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 8, F(0.1), -1, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 8, F(0.1), 0, -1, P(64), 1024, None) == 1


def test_reference_quantizer():
    x = np.array([[7.0, 0.5, 1.5, -2.5], [0, 0, 0, 0], [np.nan, 3.5, -1, 0.25], [np.inf, 1, 2, 3]], np.float16)
    c, b = ref.quant(x)
    s = ref.bf16_value(b)
    assert s.tolist() == [1.0, 0.0, 0.5, math.inf]
    assert c.tolist() == [[7, 0, 2, -2], [0] * 4, [0, 7, -2, 0], [0] * 4]
    assert (ref.unpack(ref.pack(c)) == c).all()
    assert ref.pack(np.array([[-1, 7]], np.int8)).tolist() == [[0x7F]]
    v = ref.values(ref.pack(c), b)
    assert v[0].tolist() == [7, 0, 2, -2] and np.isnan(v[3]).all()


def test_codes_fit_and_values_are_exact():
    """Over every binary16 maximum: codes stay in -7..7 and scale times code needs no rounding (from 2^-17 on)."""
    x = np.arange(1, 0x7C00, dtype=np.uint16).view(np.float16)
    c, b = ref.quant(x[:, None])
    assert (np.abs(c) <= 7).all() and (c >= 6).all()
    s = ref.bf16_value(b).astype(np.float64)
    for k in range(-7, 8):
        exact = s[s >= 2.0 ** -17] * k
        assert (exact.astype(np.float16).astype(np.float64) == exact).all()


def test_a_grid_of_2_to_the_minus_13_decides_every_quotient():
    """x r on that grid, r = 1 / s a unit in its last place up or down, rounds to an integer as the IEEE quotient does, for
    every binary16 x that a scale covers: what the kernel's codes rest on."""
    x = np.arange(0x7C00, dtype=np.uint16).view(np.float16).astype(np.float32)
    one = np.float32(1)
    for e in (-27, -24, -17, -3, 0, 13):
        for k in range(128, 256, 5 if e else 1):
            s = np.float32(k / 128 * 2.0 ** e)
            v, r = x[x <= np.float32(7.03) * s], one / s
            want = np.rint(v / s)
            for r in (np.nextafter(r, np.float32(0)), r, np.nextafter(r, np.float32(np.inf))):
                t = (v.astype(np.float64) * r + 1536).astype(np.float32) - np.float32(1536)
                assert np.array_equal((t + np.float32(12582912)) - np.float32(12582912), want)


def test_reference_attention_is_a_weighted_mean():
    rng = np.random.default_rng(0)
    cu, lens, table, blocks = ref.random_batch(rng, [3], [20], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, 64)
    out, tol = ref.attend(cache, np.zeros((3, 1, 64), np.float16), cu, lens, table, 0.1, window=4, sinks=1)
    v = ref.values(cache[2][table[0], 0], cache[3][table[0], 0]).reshape(-1, 64).astype(float)
    assert np.allclose(out[2, 0], v[[0, 16, 17, 18, 19]].mean(0)) and (tol > 0).all()
