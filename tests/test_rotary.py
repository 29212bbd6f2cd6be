"""Rotary positions: frequencies and turn fractions (host), refusals before CUDA is touched, and the kernel against
64-bit angles."""
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


# ---------------------------------------------------------------------------------- host
@pytest.mark.parametrize("r", [2, 4, 20, 64, 128])
@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
                                        ("wavelength", dict(factor=8.0, trained_len=8192.0)),
                                        ("wavelength", dict(factor=2.0, trained_len=300.0, low=0.5, high=9.0)),
                                        ("ramp", dict(factor=16.0, trained_len=4096.0)),
                                        ("ramp", dict(factor=4.0, trained_len=7.0, low=0.1, high=0.9))])
def test_frequencies(dp, r, scaling, kw):
    if scaling == "ntk" and r < 4:
        with pytest.raises(dp.DptqError):
            dp.dptq_rotary_frequencies(r, 10000.0, scaling, **kw)
        return
    got = dp.dptq_rotary_frequencies(r, 10000.0, scaling, **kw)
    want = ref.frequencies(r, 10000.0, scaling, **({"high": 32.0 if scaling == "ramp" else 4.0} | kw))
    assert got.shape == (r // 2,)
    # each of a few operations rounds by 2^-53; pow and log to a few units
    assert np.allclose(got, want, rtol=2.0 ** -46, atol=0)


def test_frequencies_scale_what_they_should(dp):
    f = dp.dptq_rotary_frequencies(128)
    s = dp.dptq_rotary_frequencies(128, scaling="wavelength", factor=8.0, trained_len=8192.0)
    turns = 8192 * f / (2 * math.pi)
    assert (s[turns >= 4] == f[turns >= 4]).all() and np.allclose(s[turns <= 1], f[turns <= 1] / 8)
    s = dp.dptq_rotary_frequencies(128, scaling="ramp", factor=8.0, trained_len=8192.0)
    assert s[0] == f[0] and math.isclose(s[-1], f[-1] / 8) and (np.diff(s) < 0).all()
    s = dp.dptq_rotary_frequencies(128, scaling="ntk", factor=8.0)
    assert s[0] == f[0] and math.isclose(s[-1], f[-1] / 8, rel_tol=1e-12)


def test_turns_are_exact_fractions(dp):
    """Whole positions times the 64-bit fraction, modulo 2^64, against exact rationals of the double frequency."""
    from fractions import Fraction
    pi = Fraction(3141592653589793238462643383279502884197169399375105820974944592307816406286, 10 ** 75)
    f = np.array([0.0, 1.0, -1.0, 1e-4, 0.8659643, 7.5, 2 * math.pi, 1e-9, 1000.25])
    t = dp.dptq_rotary_turns(f)
    assert t.dtype == np.uint64 and t[0] == 0 and int(t[1]) == (1 << 64) - int(t[2])
    for k, v in enumerate(f):
        want = Fraction(float(v)) / (2 * pi)
        for p in (1, 1000, 131071, 1 << 27):
            got = Fraction((int(t[k]) * p) % (1 << 64), 1 << 64)
            off = (got - want * p) % 1
            off = min(off, 1 - off)
            # the quotient by 2 pi: three roundings of 2^-53 of the whole angle; the fraction 2^-65
            assert off <= p * (abs(want) * Fraction(3, 1 << 53) + Fraction(1, 1 << 65))


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=-2), dict(base=1.0), dict(base=math.nan),
                                 dict(base=math.inf), dict(scaling="linear", factor=0.0),
                                 dict(scaling="linear", factor=math.nan), dict(scaling="ramp", trained_len=0.0),
                                 dict(scaling="wavelength", trained_len=9.0, low=4.0, high=4.0),
                                 dict(scaling="wavelength", trained_len=9.0, low=0.0)])
def test_frequencies_refuse(dp, bad):
    with pytest.raises(dp.DptqError) as e:
        dp.dptq_rotary_frequencies(**({"rot_dim": 64} | bad))
    assert e.value.status == 1


def test_tables_refuse(dp):
    with pytest.raises(ValueError):
        dp.dptq_rotary_frequencies(64, scaling="cubic")
    for bad in ([1.0, math.inf], [math.nan]):
        with pytest.raises(dp.DptqError):
            dp.dptq_rotary_turns(bad)
    with pytest.raises(ValueError):
        dp.dptq_rotary_turns([[1.0]])
    with pytest.raises(ValueError):
        dp.Rotary(8, frequencies=[1.0, 0.1], device="cpu")
    with pytest.raises(ValueError):
        dp.Rotary(5, frequencies=[1.0, 0.1], device="cpu")
    assert dp.dptq_rotary_turns([]).shape == (0,)
    lib = dp.load()
    assert lib.dptq_rotary_turns(None, 3, P(64)) == 1 and lib.dptq_rotary_turns(P(64), -1, P(64)) == 1
    assert lib.dptq_rotary_frequencies(8, 10.0, 9, 1.0, 1.0, 1.0, 2.0, P(64)) == 1
    assert lib.dptq_rotary_frequencies(8, 10.0, 0, 1.0, 1.0, 1.0, 2.0, None) == 1


@pytest.mark.parametrize("bad,want", [
    (dict(b=None), 1), (dict(x=None), 1), (dict(out=None), 1), (dict(turns=None), 1), (dict(x=72), 1), (dict(out=72), 1),
    (dict(turns=68), 1), (dict(xs=1020), 1), (dict(os=1020), 1), (dict(xs=504), 1), (dict(heads=0), 1), (dict(heads=-1), 1),
    (dict(dim=0), 1), (dict(dim=132), 2), (dict(dim=520, xs=4160, os=4160), 2), (dict(heads=65536), 2), (dict(rot=0), 1),
    (dict(rot=63), 1), (dict(rot=130), 1), (dict(amp=math.nan), 1), (dict(amp=math.inf), 1), (dict(seqs=-1), 1),
    (dict(seqs=65536), 2), (dict(max_tokens=65536), 2), (dict(max_len=(1 << 27) + 1), 2), (dict(cu=None), 1),
    (dict(lens=None), 1), (dict(cu=66), 1), (dict(lens=66), 1), (dict(out=64, os=1032), 1), (dict(seqs=0), 0),
    (dict(tokens=0), 0), (dict(max_tokens=0), 0)])
def test_rotary_checks_arguments(dp, bad, want):
    a = dict(x=64, out=128, turns=64, xs=512, os=512, heads=4, dim=128, rot=64, amp=1.0, seqs=3, tokens=7, max_tokens=4,
             max_len=80, cu=64, lens=64, b=0) | bad
    b = dp._Kv8BatchC(a["cu"], a["lens"], None, a["seqs"], 0, a["tokens"], a["max_tokens"], a["max_len"])
    got = dp.load().dptq_rotary(None if a["b"] is None else ctypes.addressof(b), P(a["x"]), a["xs"], a["heads"], a["dim"],
                                P(a["turns"]), a["rot"], 0, F(a["amp"]), P(a["out"]), a["os"], None)
    assert got == want


# ---------------------------------------------------------------------------------- GPU
def _batch(dp, torch, ns, lens, tokens=None, **kw):
    cu = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    b = dict(tokens=int(cu[-1]) if tokens is None else tokens, max_tokens=max(ns), max_len=max(max(lens), 1)) | kw
    return dp.Kv8Batch(torch.tensor(cu, **i32), torch.tensor(lens, **i32), torch.zeros((len(ns), 1), **i32), **b)


def _positions(ns, lens):
    return np.concatenate([np.arange(l - n, l) for n, l in zip(ns, lens)])


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    return t


# rows of each sequence, lengths with them (0: a padding slot), heads, head dim, rotated dims
SHAPES = [([1], [5001], 40, 128, 128), ([1, 1, 1], [1, 131072, 7], 1, 64, 64), ([37, 5, 2], [37, 9005, 0], 9, 128, 64),
          ([3, 4], [2, 4], 5, 80, 32), ([70], [100070], 3, 256, 256), ([5, 1], [134217728, 3], 72, 128, 32),
          ([6], [60], 7, 64, 20), ([2, 9], [1, 33], 3, 72, 72), ([4], [1000], 2, 8, 2), ([300], [301], 80, 128, 128),
          ([3], [3], 2, 512, 496)]


@pytest.mark.gpu
@pytest.mark.parametrize("ns,lens,H,D,r", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("place", ["apart", "in place", "strided in place"])
def test_rotary(dp, torch, ns, lens, H, D, r, interleaved, place):
    rng = np.random.default_rng(r + H)
    T = sum(ns)
    extra = 0 if place == "in place" else 3
    rows = torch.from_numpy(rng.standard_normal((T + 2, H * D + 8 * extra)).astype(np.float16)).cuda()
    x = rows[:T, :H * D].unflatten(1, (H, D))
    kw = dict(scaling="linear", factor=2.0) if H % 2 else {}
    rot = dp.Rotary(r, interleaved=interleaved, amplitude=1.25 if H % 3 else 1.0, **kw)
    b = _batch(dp, torch, ns, lens)
    before = rows.clone()
    pos = _positions(ns, lens)
    want, tol = ref.rotate(x.cpu().numpy(), pos, rot.frequencies, interleaved, rot.amplitude)
    if place == "apart":
        out = torch.full((T + 2, H * D), 7.0, dtype=torch.float16, device="cuda")
        dp.dptq_rotary(rot, b, x, out[:T].unflatten(1, (H, D)))
        assert torch.equal(rows, before) and (out[T:] == 7).all()
        got = out[:T].unflatten(1, (H, D)).cpu().numpy()
        assert (got[pos < 0] == 7).all()
        got[pos < 0] = want[pos < 0]
    else:
        dp.dptq_rotary(rot, b, x)
        got = x.cpu().numpy()
        assert torch.equal(rows[T:], before[T:]) and torch.equal(rows[:, H * D:], before[:, H * D:])
    assert np.array_equal(got[..., r:], want[..., r:].astype(np.float16))
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist())
    dp.dptq_last_device_error()


@pytest.mark.gpu
def test_rotary_back_and_forth(dp, torch):
    """Negative frequencies undo it: two roundings to binary16 of values of the pair's length."""
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.standard_normal((50, 4, 128)).astype(np.float16)).cuda()
    b = _batch(dp, torch, [50], [70000])
    there, f = torch.empty_like(x), dp.dptq_rotary_frequencies(128)
    dp.dptq_rotary(dp.Rotary(128), b, x, there)
    dp.dptq_rotary(dp.Rotary(128, frequencies=-f), b, there)
    pair = x.float().unflatten(2, (2, 64)).norm(dim=2).repeat(1, 1, 2)
    assert ((there.float() - x.float()).abs() <= (2 ** -11 + 2 ** -10 + 2 ** -19) * pair + 2 ** -23).all()


@pytest.mark.gpu
def test_relative_positions(dp, torch):
    """q . k after rotation depends on the distance alone, at far positions as at near ones: what both roundings
    allow, 2^-11 of each product for each side."""
    rng = np.random.default_rng(3)
    q, k = (torch.from_numpy(rng.standard_normal((1, 1, 128)).astype(np.float16)).cuda() for _ in range(2))
    rot, dots = dp.Rotary(128), []
    for p in (100, 131000, 100_000_000):
        y = []
        for t, at in ((q, p), (k, p - 57)):
            o = torch.empty_like(t)
            dp.dptq_rotary(rot, _batch(dp, torch, [1], [at + 1]), t, o)
            y.append(o.double())
        dots.append(((y[0] * y[1]).sum().item(), (y[0].abs() * y[1].abs()).sum().item()))
    for d, mag in dots[1:]:
        # (pairs' lengths in place of the values: another sqrt 2)
        assert abs(d - dots[0][0]) <= 2 * 2 ** 0.5 * 2 * 2 ** -11 * max(mag, dots[0][1])


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_pairs(dp, torch):
    rng = np.random.default_rng(1)
    for D, r in ((128, 128), (64, 20)):
        x = torch.from_numpy(rng.standard_normal((5, 3, D)).astype(np.float16)).cuda()
        b, rot, clean, out = _batch(dp, torch, [5], [905]), dp.Rotary(r), torch.empty_like(x), torch.empty_like(x)
        dp.dptq_rotary(rot, b, x, clean)
        x[2, 1, 3], x[4, 0, 1] = float("nan"), float("inf")
        dp.dptq_rotary(rot, b, x, out)
        hit = torch.zeros_like(x, dtype=torch.bool)
        for t, h, d in ((2, 1, 3), (4, 0, 1)):
            hit[t, h, [d, d + r // 2]] = True
        assert torch.equal(out[~hit], clean[~hit]) and not torch.isfinite(out[hit]).any()


@pytest.mark.gpu
def test_rotary_leaves_what_contradicts_the_batch(dp, torch):
    for cu, lens, served in (([0, 3, 9], [1 << 30, 9], [3, 9]), ([0, 12, 9], [9, 9], None), ([-1, 3, 9], [9, 9], [3, 9])):
        i32 = dict(dtype=torch.int32, device="cuda")
        x = torch.ones((12, 2, 64), dtype=torch.float16, device="cuda")
        b = dp.Kv8Batch(torch.tensor(cu, **i32), torch.tensor(lens, **i32), torch.zeros((2, 1), **i32), tokens=12,
                        max_tokens=9, max_len=100)
        dp.dptq_rotary(dp.Rotary(64), b, x)
        with pytest.raises(dp.DptqError) as e:
            dp.dptq_last_device_error()
        assert e.value.status == 1
        stay = torch.ones((12,), dtype=torch.bool, device="cuda")
        if served:
            stay[served[0]:served[1]] = False
            assert not (x[~stay] == 1).all(dim=2).all(dim=1)[1:].any()
        assert (x[stay] == 1).all()


@pytest.mark.gpu
def test_rotary_stream_and_graph(dp, torch):
    """On a side stream, and replayed from a graph with other lengths in the same arrays."""
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((3, 6, 128)).astype(np.float16)).cuda()
    out, rot = torch.empty_like(x), dp.Rotary(128)
    b = _batch(dp, torch, [1, 2], [9, 50], max_len=1 << 20)
    dp.dptq_kv8_reserve()

    def expect(lens):
        want, tol = ref.rotate(x.cpu().numpy(), _positions([1, 2], lens), rot.frequencies, False)
        assert (np.abs(out.cpu().numpy() - want) <= tol).all()
        out.fill_(float("nan"))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dp.dptq_rotary(rot, b, x, out)
    side.synchronize()
    expect([9, 50])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dp.dptq_rotary(rot, b, x, out)
    for lens in ([9, 50], [700000, 2], [1, 1 << 20]):
        b.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        expect(lens)


@pytest.mark.gpu
def test_rotary_refuses(dp, torch):
    b, rot = _batch(dp, torch, [2], [9]), dp.Rotary(64)
    x = torch.zeros((2, 3, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(TypeError):
        dp.dptq_rotary(rot, b, x.float())
    with pytest.raises(ValueError):
        dp.dptq_rotary(rot, b, x[:1])
    with pytest.raises(ValueError):
        dp.dptq_rotary(rot, b, x, x[:, :2])
    with pytest.raises(ValueError):
        dp.dptq_rotary(rot, b, x.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(dp.DptqError):
        dp.dptq_rotary(rot, b, x[:, :, :32].contiguous())
    b.device += 1                                     # (as if its arrays were on another GPU)
    with pytest.raises(ValueError):
        dp.dptq_rotary(rot, b, x)
