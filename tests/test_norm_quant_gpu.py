"""dptq_add_rmsnorm_quant against its definition: the residual and the codes bit for bit, the
scales in 64 bits."""
import numpy as np
import pytest

import kv8_reference as ref
import parity

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_12487_gb300 import dptq
    dptq.load()
    return dptq


def _call(dp, x, r, g, bits, eps=EPS, inplace=None):
    M, K = x.shape
    X = torch.from_numpy(x).cuda()
    R = None if r is None else torch.from_numpy(r).cuda()
    G = None if g is None else torch.from_numpy(g).cuda()
    out = None if r is None else X if inplace == "x" else R if inplace == "r" else torch.empty_like(X)
    codes = torch.empty((M, K // 2) if bits == 4 else (M, K), dtype=torch.uint8 if bits == 4 else torch.int8,
                        device="cuda")
    scales = torch.full((M,), -1.0, device="cuda")
    dp.dptq_add_rmsnorm_quant(X, R, G, eps, bits, out, codes, scales)
    torch.cuda.synchronize()
    c = codes.cpu().numpy()
    c = parity.unpack_public_a4(c, K) if bits == 4 else c
    return None if out is None else out.cpu().numpy(), c.astype(np.int64), scales.cpu().numpy()


def _check(got, want, K):
    h, c, s = got
    h_ref, c_ref, s_ref = want
    if h is not None:
        assert np.array_equal(h.view(np.uint16), h_ref.view(np.uint16))
    assert np.array_equal(c, c_ref)
    # a sum of K squares in fp32 (any order with at most K / 32 + 32 terms in a chain), then a
    # division, a root, a reciprocal and a product
    rel = ((K / 32 + 32) / 2 + 8) * 2.0 ** -24
    ok = np.isfinite(s_ref)
    np.testing.assert_allclose(s[ok], s_ref[ok], rtol=rel, atol=0)


def _inputs(M, K, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((M, K)).astype(np.float16)
    r = (rng.standard_normal((M, K)) * 2).astype(np.float16)
    r[:, rng.choice(K, min(K, 3), replace=False)] *= 50
    g = (1 + 0.2 * rng.standard_normal(K)).astype(np.float16)
    return x, r, g


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,K", [(1, 32), (3, 96), (5, 2080), (1, 4096), (9, 4096), (64, 8192), (333, 5120),
                                 (2, 11008), (700, 1024), (1, 16384), (3, 16416), (2, 28672), (2, 49152)])
def test_norm_quant_matches_its_definition(dp, M, K, bits):
    x, r, g = _inputs(M, K, M * 100003 + K)
    for rr in (r, None):
        for gg in (g, None):
            _check(_call(dp, x, rr, gg, bits), ref.norm_quant(x, rr, gg, EPS, bits), K)


@pytest.mark.parametrize("inplace", ["x", "r"])
@pytest.mark.parametrize("M,K", [(4, 4096), (3, 20000 - 20000 % 32)])
def test_norm_quant_in_place(dp, inplace, M, K):
    x, r, g = _inputs(M, K, K)
    _check(_call(dp, x, r, g, 8, inplace=inplace), ref.norm_quant(x, r, g, EPS, 8), K)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("K", [64, 4096, 20480])
def test_norm_quant_ties_zeros_and_non_finite_values(dp, bits, K):
    rng = np.random.default_rng(K)
    q = 2 ** (bits - 1) - 1
    x = (rng.integers(-2 * q, 2 * q + 1, (8, K)) * 0.5).astype(np.float16)      # half of the values tie
    x[:, 0] = q                                                                  # s' = 1
    x[1] = 0                                                                     # all zero
    x[2] = 0
    x[2, K - 1] = np.float16(6e-8)                                               # one subnormal
    x[3, 5:9] = np.nan
    x[4, 7] = np.inf
    x[5] = np.float16(65504)                                                     # squares sum to 4e9 K
    r = np.zeros_like(x)
    r[6] = x[6]                                                                  # the sum is exact
    r[7] = -x[7]
    for eps in (EPS, 0.0):
        got, want = _call(dp, x, r, None, bits, eps), ref.norm_quant(x, r, None, eps, bits)
        assert np.array_equal(got[1], want[1])
        rows = [0, 1, 2, 5, 6] if eps == 0.0 else [0, 1, 2, 5, 6, 7]
        rows = [i for i in rows if eps or i != 1]                                # (0 / 0 without eps)
        np.testing.assert_allclose(got[2][rows], want[2][rows], rtol=((K / 32 + 32) / 2 + 8) * 2.0 ** -24, atol=0)
        assert np.isnan(got[2][3]) and not np.isfinite(got[2][4])


def test_norm_quant_feeds_the_gemm(dp, orc):
    """The codes and scales go through dptq_qgemm_codes as dptq_rotate_quant_act's do."""
    M, N, K = 37, 272, 512
    x, r, g = _inputs(M, K, 3)
    W = np.random.default_rng(1).standard_normal((N, K)).astype(np.float16)
    layer = dp.dptq_pack_weights(torch.from_numpy(W).cuda(), 1)
    wq, sw = dp.dptq_get_packed(layer)
    w = parity.unpack_public_a4(wq, K).astype(np.float64) * sw[:, None]
    for bits in (4, 8):
        codes = torch.empty((M, K // 2) if bits == 4 else (M, K), dtype=torch.uint8 if bits == 4 else torch.int8,
                            device="cuda")
        scales = torch.empty((M,), device="cuda")
        h = torch.empty((M, K), dtype=torch.float16, device="cuda")
        out = torch.empty((M, N), dtype=torch.float16, device="cuda")
        dp.dptq_add_rmsnorm_quant(torch.from_numpy(x).cuda(), torch.from_numpy(r).cuda(), torch.from_numpy(g).cuda(),
                                  EPS, bits, h, codes, scales)
        dp.dptq_qgemm_codes(layer, codes, scales, bits, out)
        _, c, s = ref.norm_quant(x, r, g, EPS, bits)
        want = (c * s[:, None]) @ w.T
        # exact integer products; fp32 scales and one rounding to binary16
        np.testing.assert_allclose(out.cpu().numpy(), want, rtol=2.0 ** -10, atol=2.0 ** -24)


def test_norm_quant_refusals(dp):
    x = torch.zeros((2, 64), dtype=torch.float16, device="cuda")
    c, s = torch.empty((2, 64), dtype=torch.int8, device="cuda"), torch.empty((2,), device="cuda")
    call = dp.dptq_add_rmsnorm_quant
    for bad in (dict(residual=x), dict(residual_out=x), dict(bits=5), dict(eps=-1.0), dict(eps=float("nan"))):
        a = dict(residual=None, gamma=None, eps=EPS, bits=8, residual_out=None, codes=c, scales=s) | bad
        with pytest.raises((dp.DptqError, ValueError, TypeError)):
            call(x, **a)
    odd = torch.zeros((129,), dtype=torch.float16, device="cuda")[1:].view(2, 64)
    with pytest.raises(dp.DptqError):
        call(odd, None, None, EPS, 8, None, c, s)
    narrow = torch.zeros((2, 48), dtype=torch.float16, device="cuda")
    with pytest.raises(dp.DptqError):
        call(narrow, None, None, EPS, 8, None, torch.empty((2, 48), dtype=torch.int8, device="cuda"), s)
    with pytest.raises(TypeError):
        call(x.float(), None, None, EPS, 8, None, c, s)
    empty = torch.zeros((0, 64), dtype=torch.float16, device="cuda")
    call(empty, None, None, EPS, 8, None, c[:0], s[:0])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("K", [64, 4096, 20480])
@pytest.mark.parametrize("eps", [EPS, 0.0])
def test_a_token_of_zeros_has_scale_zero(dp, bits, K, eps):
    """With eps = 0 too, where the norm's own factor is 1 / 0; also where only the sum is zero, or only the
    weighted values are."""
    rng = np.random.default_rng(K)
    x = rng.standard_normal((4, K)).astype(np.float16)
    x[0] = 0
    r = np.zeros_like(x)
    r[1] = -x[1]
    for rr, gg, zero in ((r, None, [0, 1]), (None, None, [0]), (r, np.zeros(K, np.float16), [0, 1, 2, 3])):
        _, c, s = _call(dp, x, rr, gg, bits, eps)
        _, c_ref, s_ref = ref.norm_quant(x, rr, gg, eps, bits)
        assert np.array_equal(c, c_ref) and not c[zero].any() and not s[zero].any()
        rest = [i for i in range(4) if i not in zero]
        np.testing.assert_allclose(s[rest], s_ref[rest], rtol=((K / 32 + 32) / 2 + 8) * 2.0 ** -24, atol=0)
    x[0, 3] = np.nan                             # no number, and nothing else in the token
    _, c, s = _call(dp, x, None, None, bits, eps)
    assert not c[0].any() and np.isnan(s[0])
