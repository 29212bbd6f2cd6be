"""Argument checks of the norm and KV8 entry points that are made before CUDA is touched, and the
test reference's own pins."""
import ctypes
import math

import numpy as np
import pytest

import kv8_reference as ref


@pytest.fixture(scope="module")
def dp():
    from paper_2606_12487_gb300 import dptq
    dptq.load()
    return dptq


P = ctypes.c_void_p
F = ctypes.c_float


def test_norm_checks_arguments(dp):
    call = dp.load().dptq_add_rmsnorm_quant
    d, odd = P(64), P(72)
    ok = dict(x=d, r=d, g=d, M=4, K=256, eps=F(1e-5), bits=8, out=d, c=d, s=d)
    for bad, want in ((dict(bits=5), 1), (dict(M=-1), 1), (dict(K=0), 1), (dict(K=48), 2), (dict(K=49152 + 32), 2),
                      (dict(eps=F(-1)), 1), (dict(eps=F(math.nan)), 1), (dict(x=None), 1), (dict(c=None), 1),
                      (dict(s=None), 1), (dict(r=None), 1), (dict(out=None), 1), (dict(x=odd), 1), (dict(g=odd), 1),
                      (dict(r=odd), 1), (dict(out=odd), 1), (dict(c=P(68)), 1), (dict(c=P(66), bits=4), 1),
                      (dict(s=P(66)), 1), (dict(M=0), 0)):
        a = ok | bad
        got = call(a["x"], a["r"], a["g"], a["M"], a["K"], a["eps"], a["bits"], a["out"], a["c"], a["s"], None)
        assert got == want, bad
        assert got == 0 or dp.load().dptq_last_error_message()


def _handles(dp, cache=None, batch=None):
    c = dp._Kv8CacheC(*([64] * 4), 10, 2, 16, 128)
    b = dp._Kv8BatchC(*([64] * 3), 3, 5, 7, 4, 80)
    for k, v in (cache or {}).items():
        setattr(c, k, v)
    for k, v in (batch or {}).items():
        setattr(b, k, v)
    return c, b


@pytest.mark.parametrize("cache,batch,want", [
    (dict(head_dim=96), {}, 2), (dict(head_dim=0), {}, 1), (dict(block_tokens=8), {}, 2), (dict(block_tokens=48), {}, 2),
    (dict(block_tokens=-16), {}, 1), (dict(num_blocks=0), {}, 1), (dict(kv_heads=0), {}, 1),
    (dict(kv_heads=1024), {}, 2), (dict(k_codes=None), {}, 1), (dict(v_codes=72), {}, 1), (dict(k_scales=None), {}, 1),
    ({}, dict(seqs=-1), 1), ({}, dict(seqs=65536), 2), ({}, dict(tokens=-1), 1), ({}, dict(max_tokens=-1), 1),
    ({}, dict(max_len=-1), 1), ({}, dict(max_len=81), 1), ({}, dict(block_table=None), 1), ({}, dict(cu_tokens=None), 1),
    ({}, dict(seq_lens=None), 1), ({}, dict(seqs=0), 0), ({}, dict(tokens=0), 0), ({}, dict(max_tokens=0), 0)])
def test_kv8_checks_cache_and_batch(dp, cache, batch, want):
    c, b = _handles(dp, cache, batch)
    lib = dp.load()
    assert lib.dptq_kv8_append(ctypes.addressof(c), ctypes.addressof(b), P(64), P(64), 256, None) == want
    heads = 8 * max(1, c.kv_heads)
    assert lib.dptq_kv8_attention(ctypes.addressof(c), ctypes.addressof(b), P(64), 8 * heads * 128, heads, F(0.1), 0, 0,
                                  P(64), 8 * heads * 128, None) == want


def test_kv8_checks_scalars(dp):
    c, b = _handles(dp)
    lib = dp.load()
    cp, bp = ctypes.addressof(c), ctypes.addressof(b)
    att = lib.dptq_kv8_attention
    assert lib.dptq_kv8_append(None, bp, P(64), P(64), 256, None) == 1
    assert att(cp, None, P(64), 1024, 8, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 0, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 7, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 130 * 128, 130, F(0.1), 0, 0, P(64), 130 * 128, None) == 2
    assert att(cp, bp, P(64), 1024, 8, F(math.inf), 0, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 8, F(0.1), -1, 0, P(64), 1024, None) == 1
    assert att(cp, bp, P(64), 1024, 8, F(0.1), 0, -1, P(64), 1024, None) == 1


def test_reference_quantizers():
    x = np.array([[[127.0, 0.5, 1.5, -2.5]]], np.float16)
    codes, scales = np.zeros((1, 1, 4, 4), np.int8), np.zeros((1, 1), np.float32)
    table = np.zeros((1, 1), np.int32)
    ref.append(codes, scales, x, [0, 1], [1], table)
    assert scales[0, 0] == 1 and codes[0, 0, 0].tolist() == [127, 0, 2, -2]
    ref.append(codes, scales, 2 * x, [0, 1], [2], table)          # the page's scale doubles
    assert scales[0, 0] == 2 and codes[0, 0, 0].tolist() == [64, 0, 1, -1] and codes[0, 0, 1].tolist() == [127, 0, 2, -2]
    h, c, s = ref.norm_quant(np.array([[3, 4]], np.float16), None, None, 0.0, 4)
    assert c.tolist() == [[5, 7]] and abs(s[0] - 4 / 7 / math.sqrt(12.5)) < 1e-7


def test_reference_attention_is_a_weighted_mean():
    rng = np.random.default_rng(0)
    cu, lens, table, blocks = ref.random_batch(rng, [3], [20], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, 64)
    q = np.zeros((3, 1, 64), np.float16)
    out, tol = ref.attend(cache, q, cu, lens, table, 0.1, window=4, sinks=1)
    v = (cache[2][table[0], 0].astype(float) * cache[3][table[0], 0][:, None, None]).reshape(-1, 64)
    assert np.allclose(out[2, 0], v[[0, 16, 17, 18, 19]].mean(0)) and (tol > 0).all()
    assert ref.sees([2], 5, 2, 0).tolist() == [[False, True, True, False, False]]


@pytest.mark.parametrize("batch", [dict(max_tokens=65536, tokens=70000), dict(max_len=(1 << 27) + 1, table_stride=1 << 28)])
def test_kv8_refuses_what_its_indexes_do_not_hold(dp, batch):
    c, b = _handles(dp, batch=batch)
    lib = dp.load()
    cp, bp = ctypes.addressof(c), ctypes.addressof(b)
    assert lib.dptq_kv8_append(cp, bp, P(64), P(64), 256, None) == 2
    assert lib.dptq_kv8_attention(cp, bp, P(64), 1024, 8, F(0.1), 0, 0, P(64), 1024, None) == 2


@pytest.mark.parametrize("cache,batch", [(dict(k_scales=66), {}), (dict(v_scales=65), {}), ({}, dict(cu_tokens=66)),
                                         ({}, dict(seq_lens=67)), ({}, dict(block_table=66))])
def test_kv8_refuses_misaligned_scales_and_arrays(dp, cache, batch):
    """4-byte values that the kernels read whole: a misaligned read would fault."""
    c, b = _handles(dp, cache, batch)
    lib = dp.load()
    cp, bp = ctypes.addressof(c), ctypes.addressof(b)
    assert lib.dptq_kv8_append(cp, bp, P(64), P(64), 256, None) == 1
    assert lib.dptq_kv8_attention(cp, bp, P(64), 1024, 8, F(0.1), 0, 0, P(64), 1024, None) == 1
    assert b"aligned" in lib.dptq_last_error_message()
