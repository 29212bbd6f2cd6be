"""The paged 4-bit cache: append bit for bit, read-back exactly, attention within the roundings it declares."""
import math

import numpy as np
import pytest

import kv4_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2606_12487_gb300 import dptq
    dptq.load()
    return dptq


def _cuda(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def _bf16(bits):
    return torch.from_numpy(bits.astype(np.int32)).to(torch.int16).cuda().view(torch.bfloat16)


def _bits(t):
    return t.view(torch.int16).cpu().numpy().astype(np.uint16)


def _handles(dp, cache, cu, lens, table, **kw):
    kc, vc = _cuda(cache[0], cache[2])
    c = dp.Kv4Cache(kc, vc, _bf16(cache[1]), _bf16(cache[3]))
    sizes = dict(tokens=int(cu[-1]), max_tokens=int(max(np.diff(cu), default=0)), max_len=int(max(lens, default=0))) | kw
    return c, dp.Kv8Batch(*_cuda(cu, lens, table), **sizes)


def _rows(rng, T, heads, D, pad=0):
    """Rows of heads side by side, `pad` values between tokens."""
    x = torch.from_numpy(rng.standard_normal((max(T, 1), heads * D + pad)).astype(np.float16)).cuda()
    return x[:T, :heads * D].unflatten(1, (heads, D))


def _attend(dp, cache, q, cu, lens, table, window=0, sinks=0, scale=None, **kw):
    c, b = _handles(dp, cache, cu, lens, table, **kw)
    scale = 1 / math.sqrt(q.shape[2]) if scale is None else scale
    T, H, D = q.shape
    out = torch.full((T + 2, H * D + 16), 7.0, dtype=torch.float16, device="cuda")
    dp.dptq_kv4_attention(c, b, q, out[:T, :H * D].unflatten(1, (H, D)), scale, window, sinks)
    assert (out[T:] == 7).all() and (out[:, H * D:] == 7).all()
    return out[:T, :H * D].unflatten(1, (H, D)).cpu().numpy(), scale


def _check(dp, cache, q, cu, lens, table, window=0, sinks=0, scale=None, **kw):
    got, scale = _attend(dp, cache, q, cu, lens, table, window, sinks, scale, **kw)
    want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, scale, window, sinks)
    for s in range(len(lens)):      # rows that have no place see nothing
        n = cu[s + 1] - cu[s]
        assert not got[cu[s]:cu[s] + max(n - lens[s], 0)].any()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5])
    dp.dptq_last_device_error()
    return got


# ---------------------------------------------------------------------------------- append, read
BATCHES = [([1], [1]), ([1, 1, 1], [16, 17, 400]), ([3, 0, 5], [3, 9, 130]), ([33, 1, 70], [50, 64, 70]),
           ([2, 4], [0, 3]), ([300], [1000])]


@pytest.mark.parametrize("ns,lens", BATCHES)
@pytest.mark.parametrize("H,D,P,pad", [(1, 64, 16, 0), (3, 128, 32, 0), (8, 128, 128, 24), (5, 64, 64, 8)])
def test_append_and_read(dp, ns, lens, H, D, P, pad):
    rng = np.random.default_rng(D + P + sum(ns))
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    c, b = _handles(dp, cache, cu, lens, table)
    T = sum(ns)
    k, v = _rows(rng, T, H, D, pad), _rows(rng, T, H, D, pad)
    k[:, :, 3] *= 30
    dp.dptq_kv4_append(c, b, k, v)
    want = [a.copy() for a in cache]
    ref.append(want[0], want[1], k.cpu().numpy(), cu, lens, table)
    ref.append(want[2], want[3], v.cpu().numpy(), cu, lens, table)
    for got, w in zip((c.k_codes, c.v_codes), (want[0], want[2])):
        assert np.array_equal(got.cpu().numpy(), w)
    for got, w in zip((c.k_scales, c.v_scales), (want[1], want[3])):
        assert np.array_equal(_bits(got), w)
    # back again, into rows that keep what the batch has no place for
    flat = torch.full((2, T + 1, H * D + pad), 7.0, dtype=torch.float16, device="cuda")
    outs = [f[:T, :H * D].unflatten(1, (H, D)) for f in flat]
    dp.dptq_kv4_read(c, b, *outs)
    for f, o, w in zip(flat, outs, (want[:2], want[2:])):
        e = np.full((T, H, D), 7, np.float16)
        ref.read(*w, e, cu, lens, table)
        assert np.array_equal(o.cpu().numpy(), e)
        assert (f[T:] == 7).all() and (f[:, H * D:] == 7).all()
    dp.dptq_last_device_error()


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_values_at_the_edges(dp, D):
    """Zeros, the smallest and largest binary16 numbers, halves (ties), scales that round up and down,
    NaN and infinities, each in a row of its own."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 2, D)).astype(np.float16)
    x[0], x[1, 0], x[2] = 0, -0.0, 0
    x[2, :, 5], x[3] = 2.0 ** -24, np.float16(65504) * np.sign(x[3])
    x[4], x[4, :, 0] = rng.integers(-14, 15, (2, D)) / 2, 7      # ties
    x[5], x[5, :, 0] = rng.integers(-14, 15, (2, D)) / 128, 7 / 64
    x[6, 0, 9], x[6, 1, 0], x[7, 0, D - 1] = np.nan, -np.inf, np.inf
    x[8] = np.nan
    x[9] = (rng.integers(0, 64, (2, D)) * 2.0 ** -24).astype(np.float16)
    for i in range(10, 40):
        x[i] *= np.float16(2.0 ** (i - 26))
    cu, lens, table, blocks = ref.random_batch(rng, [40], [45], 16)
    cache = ref.random_cache(rng, blocks, 2, 16, D)
    c, b = _handles(dp, cache, cu, lens, table)
    k = _cuda(x)[0]
    dp.dptq_kv4_append(c, b, k, k)
    ref.append(cache[0], cache[1], x, cu, lens, table)
    assert np.array_equal(c.k_codes.cpu().numpy(), cache[0]) and np.array_equal(_bits(c.k_scales), cache[1])
    outs = [torch.empty_like(k) for _ in range(2)]
    dp.dptq_kv4_read(c, b, *outs)
    e = np.zeros(x.shape, np.float16)
    ref.read(cache[0], cache[1], e, cu, lens, table)
    assert np.array_equal(outs[0].cpu().numpy(), e, equal_nan=True)
    dp.dptq_last_device_error()


# ---------------------------------------------------------------------------------- attention
# new rows and cached tokens of each sequence, KV heads, query heads of each, head dim, page
FEW = [([1], [1], 1, 1, 128, 16), ([1], [32], 2, 3, 64, 16), ([1, 1, 1], [33, 31, 700], 2, 4, 128, 16),
       ([1] * 5, [1, 0, 2047, 130, 64], 1, 8, 64, 128), ([3, 2], [3, 95], 3, 5, 128, 32), ([4], [1300], 2, 4, 64, 64),
       ([1], [9000], 8, 8, 128, 128), ([1, 1], [5000, 77], 4, 16, 128, 64), ([16, 9, 0], [16, 2000, 5], 2, 1, 128, 16),
       ([2, 3], [1, 2], 2, 4, 64, 16)]
MANY = [([17], [17], 1, 1, 128, 16), ([40, 33], [40, 500], 2, 4, 64, 32), ([130, 1, 0, 64], [130, 900, 7, 64], 2, 2, 128, 16),
        ([257], [1024], 1, 3, 128, 128), ([9], [3000], 2, 20, 128, 64), ([5, 8], [3, 8], 1, 64, 64, 16),
        ([2], [300], 1, 64, 128, 32), ([600], [600], 2, 1, 64, 16)]


@pytest.mark.parametrize("ns,lens,H,g,D,P", FEW + MANY)
def test_attention(dp, ns, lens, H, g, D, P):
    rng = np.random.default_rng(D + P + g + sum(lens))
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    _check(dp, ref.random_cache(rng, blocks, H, P, D), _rows(rng, sum(ns), H * g, D, pad=8 * (g % 3)), cu, lens, table)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (17, 0), (128, 4), (500, 130), (100000, 3), (33, 100000)])
@pytest.mark.parametrize("ns,lens,H,g,D,P", [FEW[2], FEW[5], FEW[8], MANY[1], MANY[3], MANY[4]])
def test_windows(dp, ns, lens, H, g, D, P, window, sinks):
    rng = np.random.default_rng(window + D)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    _check(dp, ref.random_cache(rng, blocks, H, P, D), _rows(rng, sum(ns), H * g, D), cu, lens, table, window, sinks)


@pytest.mark.parametrize("n", [1, 3, 130, 600])
def test_what_no_query_sees_does_not_matter(dp, n):
    """Pages behind the window, positions past the length, pages of nobody: NaN and infinite scales included."""
    rng = np.random.default_rng(5 + n)
    P, H, D, W = 16, 2, 128, 40
    cu, lens, table, blocks = ref.random_batch(rng, [n], [400 + n], P, spare=4)
    cache = ref.random_cache(rng, blocks, H, P, D)
    q = _rows(rng, n, 8, D)
    got, _ = _attend(dp, cache, q, cu, lens, table, W, 3)
    first = (lens[0] - n - W + 1) // P          # the first page that a window reaches
    other = [a.copy() for a in cache]
    hidden = [b for b in range(blocks) if b not in table[0, first:] and b != table[0, 0]]
    for b in hidden:
        other[1][b], other[3][b] = 0x7FC0, 0x7F80
        other[0][b], other[2][b] = 0x88, 0x77
    last, used = table[0, (lens[0] - 1) // P], (lens[0] - 1) % P + 1
    other[1][last, :, used:], other[3][last, :, used:] = 0xFF80, 0x7FC0
    other[0][last, :, used:], other[2][last, :, used:] = 0x77, 0x88
    other[1][table[0, 0], :, 3:], other[3][table[0, 0], :, 3:] = 0x7FC0, 0xFFFF     # behind the first three
    t2 = table.copy()
    t2[0, 1:first] = -1                          # pages that no query sees need not be there
    again, _ = _attend(dp, other, q, cu, lens, t2, W, 3)
    assert np.array_equal(got, again)
    dp.dptq_last_device_error()


# rows, lengths, KV heads, query heads of each, dims: single tokens, a few, split along the keys, CTAs alone, pairs
FORMS = [([1, 1], [300, 290], 2, 4, 128), ([3, 2], [300, 290], 1, 4, 64), ([200], [1500], 1, 2, 128),
         ([300], [300], 80, 2, 64), ([140] * 10, [140] * 10, 16, 2, 128), ([600, 520], [900, 520], 16, 2, 128)]


@pytest.mark.parametrize("ns,lens,H,g,D", FORMS)
@pytest.mark.parametrize("kv,bits", [(1, 0x7F80), (1, 0x7FC0), (3, 0x7F80), (3, 0xFF80), (3, 0x7FFF)])
@pytest.mark.parametrize("at", [0.4, 0.97])
def test_a_scale_that_is_no_number_stays_with_the_rows_that_see_it(dp, ns, lens, H, g, D, kv, bits, at):
    rng = np.random.default_rng(D + ns[0] + bits)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    key = int(lens[0] - ns[0] + at * ns[0] - 1)
    window = 50 if at < 0.5 else 0
    dirty = [a.copy() for a in cache]
    dirty[kv][table[0, key // 16], :, key % 16] = bits
    dirty[kv - 1][table[0, key // 16], :, key % 16] &= 0x0F
    q = _rows(rng, sum(ns), H * g, D)
    got, scale = _attend(dp, dirty, q, cu, lens, table, window, 0)
    clean, _ = _attend(dp, cache, q, cu, lens, table, window, 0)
    hit = np.zeros(got.shape[0], bool)
    hit[cu[0]:cu[1]] = ref.sees(lens[0] - ns[0] + np.arange(ns[0]), lens[0], window, 0)[:, key]
    assert hit.any() and np.isnan(got[hit]).all()
    assert np.array_equal(got[~hit], clean[~hit])
    dp.dptq_last_device_error()


@pytest.mark.parametrize("n", [1, 3, 150, 600])
def test_a_nan_query_stays_in_its_row(dp, n):
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n, n], [200 + n, 50 + n], 16)
    cache = ref.random_cache(rng, blocks, 2, 16, 128)
    q = _rows(rng, 2 * n, 8, 128)
    got, _ = _attend(dp, cache, q, cu, lens, table)
    bad = q.clone()
    bad[0, 3, 7] = float("nan")
    again, _ = _attend(dp, cache, bad, cu, lens, table)
    assert np.isnan(again[0, 3]).all()
    got[0, 3] = again[0, 3] = 0
    assert np.array_equal(got, again)


@pytest.mark.parametrize("n", [1, 6, 130, 520])
def test_zeros_and_scales_far_apart(dp, n):
    """Scales of 0 and from 2^-20 to 2^10 side by side, in K (where q is small) and in V."""
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n, n], [300 + n, 90 + n], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, 64)
    cache[3][:] = ref.bf16_bits((2.0 ** rng.uniform(-20, 10, cache[3].shape)).astype(np.float32))
    for x in (1, 3):
        cache[x][rng.random(cache[x].shape) < 0.25] = 0
    _check(dp, cache, _rows(rng, 2 * n, 4, 64), cu, lens, table)
    cache[1][:] = ref.bf16_bits((2.0 ** rng.uniform(-16, 10, cache[1].shape)).astype(np.float32))
    _check(dp, cache, _rows(rng, 2 * n, 4, 64), cu, lens, table, scale=2.0 ** -10)
    cache[2][:], cache[3][:] = 0, 0
    got, _ = _attend(dp, cache, _rows(rng, 2 * n, 4, 64), cu, lens, table)
    assert not got.any()


@pytest.mark.parametrize("n", [1, 200])
def test_a_first_token_that_takes_almost_all_the_weight(dp, n):
    """A sink whose values are zero: what is left to see are weights of 2^-20 and less of the largest."""
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n], [500 + n], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, 128)
    cache[1][:] = ref.bf16_bits(np.float32(0.25))
    cache[0][table[0, 0], :, 0] = 0x77
    cache[3][table[0, 0], :, 0] = 0
    q = (0.3 + 0.1 * _rows(rng, n, 4, 128)).half()
    _check(dp, cache, q, cu, lens, table)


@pytest.mark.parametrize("n", [1, 200, 550])
@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_flat_and_sharp_softmax(dp, n, scale):
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n], [333 + n], 32)
    _check(dp, ref.random_cache(rng, blocks, 2, 32, 128), _rows(rng, n, 4, 128), cu, lens, table, scale=scale)


def test_maxima_that_grow_with_every_tile(dp):
    """Keys whose logits rise by far more than a kernel lets its maximum lag."""
    rng = np.random.default_rng(3)
    for n in (1, 300, 560):
        cu, lens, table, blocks = ref.random_batch(rng, [n], [900 + n], 16)
        cache = ref.random_cache(rng, blocks, 1, 16, 64)
        cache[0][:] = 0x11
        s = np.zeros(cache[1].shape, np.float32)
        for p in range(len(table[0])):
            s[table[0, p]] = (p * 16 + np.arange(16)) / 256
        cache[1] = ref.bf16_bits(s)
        q = (1 + 0.1 * _rows(rng, n, 2, 64)).half()
        _check(dp, cache, q, cu, lens, table, scale=0.25)


def test_offsets_past_32_bits(dp):
    """Pages whose codes lie beyond 2^31 and 2^32 bytes."""
    H, P, D = 8, 128, 128
    blocks = (1 << 32) // (H * P * D // 2) + 3
    codes = [torch.zeros((blocks, H, P, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones((blocks, H, P), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c = dp.Kv4Cache(codes[0], codes[1], scales[0], scales[1])
    pages = [blocks - 1, 0, blocks // 2 + 1, blocks - 2]
    rng = np.random.default_rng(0)
    for n in (1, 470):
        cu, lens = np.array([0, n], np.int32), np.array([500], np.int32)
        b = dp.Kv8Batch(*_cuda(cu, lens, np.array([pages], np.int32)), tokens=n, max_tokens=n, max_len=500)
        k, v = _rows(rng, n, H, D), _rows(rng, n, H, D)
        dp.dptq_kv4_append(c, b, k, v)
        small = [codes[0][pages].cpu().numpy(), _bits(scales[0][pages]), codes[1][pages].cpu().numpy(),
                 _bits(scales[1][pages])]
        q, out = _rows(rng, n, H, D), torch.empty((n, H, D), dtype=torch.float16, device="cuda")
        dp.dptq_kv4_attention(c, b, q, out, 0.1)
        near = np.arange(4, dtype=np.int32)[None]
        want, tol = ref.attend(small, q.cpu().numpy(), cu, lens, near, 0.1)
        assert (np.abs(out.cpu().numpy() - want) <= tol).all()
        dp.dptq_kv4_read(c, b, k, v)
        e = np.zeros((n, H, D), np.float16)
        ref.read(small[0], small[1], e, cu, lens, near)
        assert np.array_equal(k.cpu().numpy(), e) and codes[0][pages[-1]].any()
    dp.dptq_last_device_error()


def test_the_same_bits_every_time(dp):
    rng = np.random.default_rng(2)
    for ns, lens, H in (([1] * 5, [3000, 17, 900, 5000, 64], 2), ([64, 300], [9000, 300], 2), ([700, 513], [2000, 513], 16)):
        cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 32)
        cache = ref.random_cache(rng, blocks, H, 32, 128)
        q = _rows(rng, sum(ns), H * 4, 128)
        first, _ = _attend(dp, cache, q, cu, lens, table)
        for _ in range(5):
            again, _ = _attend(dp, cache, q, cu, lens, table)
            assert np.array_equal(first, again)


@pytest.mark.parametrize("n", [1, 40])
def test_a_step_on_another_stream_and_captured(dp, n):
    """Rotary positions, append, attention and read-back as a decoder layer runs them: on a side stream, and replayed
    from a graph with new lengths in the same arrays."""
    rng = np.random.default_rng(11)
    H, g, P, D = 2, 4, 16, 128
    cu, lens, table, blocks = ref.random_batch(rng, [n, n], [600, 40 + n], P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    c, b = _handles(dp, cache, cu, lens, table)
    qkv = torch.empty((2 * n, (g + 2) * H * D), dtype=torch.float16, device="cuda")
    src = _rows(rng, 2 * n, (g + 2) * H, D).flatten(1)
    qk = qkv[:, :(g + 1) * H * D].unflatten(1, ((g + 1) * H, D))
    q, k, v = qkv.unflatten(1, ((g + 2) * H, D)).split([g * H, H, H], dim=1)
    rot = dp.Rotary(D)
    out = torch.empty((2 * n, H * g, D), dtype=torch.float16, device="cuda")
    back = [torch.empty((2 * n, H, D), dtype=torch.float16, device="cuda") for _ in range(2)]

    def step():
        dp.dptq_rotary(rot, b, qk)
        dp.dptq_kv4_append(c, b, k, v)
        dp.dptq_kv4_attention(c, b, q, out, 0.09)
        dp.dptq_kv4_read(c, b, *back)

    def expect(lens):
        pos = np.concatenate([np.arange(l - n, l) for l in lens])
        y, tol = ref.rotate(src.unflatten(1, ((g + 2) * H, D))[:, :(g + 1) * H].cpu().numpy(), pos, rot.frequencies, False)
        assert (np.abs(qk.cpu().numpy() - y) <= tol).all()
        want = [a.copy() for a in cache]
        ref.append(want[0], want[1], k.cpu().numpy(), cu, lens, table)
        ref.append(want[2], want[3], v.cpu().numpy(), cu, lens, table)
        o, tol = ref.attend(want, q.cpu().numpy(), cu, lens, table, 0.09)
        assert (np.abs(out.cpu().numpy() - o) <= tol).all()
        for i in range(2):
            e = np.full((2 * n, H, D), 3, np.float16)
            ref.read(want[2 * i], want[2 * i + 1], e, cu, lens, table)
            assert np.array_equal(back[i].cpu().numpy(), e)

    def reset():
        for t, a in zip((c.k_codes, c.v_codes), (cache[0], cache[2])):
            t.copy_(torch.from_numpy(a))
        for t, a in zip((c.k_scales, c.v_scales), (cache[1], cache[3])):
            t.copy_(_bf16(a))
        qkv.copy_(src)
        out.fill_(float("nan"))
        for t in back:
            t.fill_(3)

    dp.dptq_kv8_reserve()
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    expect(lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for now in ([600, 40], [33, 16], [1, 0], [599, 1]):
        reset()
        now = np.array(now, np.int32)
        b.seq_lens.copy_(torch.from_numpy(now))
        graph.replay()
        torch.cuda.synchronize()
        expect(now)
    dp.dptq_last_device_error()


# ---------------------------------------------------------------------------------- refusals
@pytest.mark.parametrize("n", [1, 140])
@pytest.mark.parametrize("what", ["page", "long", "many", "order"])
def test_batches_that_contradict_themselves_are_reported(dp, n, what):
    rng = np.random.default_rng(1)
    H, P, D = 2, 16, 64
    cu, lens, table, blocks = ref.random_batch(rng, [n, n], [150 + n, 200 + n], P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    q, k = _rows(rng, 2 * n, 4, D), _rows(rng, 2 * n, H, D)
    cu2, lens2, t2, kw = cu.copy(), lens.copy(), table.copy(), {}
    if what == "page":
        t2[0, 0], t2[0, 3] = blocks, -7
        t2[0, (150 + n - 1) // P] = 1 << 30
    elif what == "long":
        kw["max_len"] = int(lens[1])
        lens2[0] = 1 << 30
    elif what == "many":
        cu2[1] = 2 * n + 5
    else:
        cu2[1] = -3
    c, b = _handles(dp, cache, cu2, lens2, t2, max_tokens=n, tokens=2 * n, **kw)
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    outs = [torch.full(k.shape, 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]

    def reported(call):
        call()
        with pytest.raises(dp.DptqError) as e:
            dp.dptq_last_device_error()
        assert e.value.status == 1
        dp.dptq_last_device_error()                                   # cleared

    reported(lambda: dp.dptq_kv4_attention(c, b, q, out, 0.1))
    reported(lambda: dp.dptq_kv4_read(c, b, *outs))
    before = [t.clone() for t in (c.k_codes, c.k_scales)]
    reported(lambda: dp.dptq_kv4_append(c, b, k, k))
    if what in ("long", "page"):      # the other sequence is served
        want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, 0.1)
        assert (np.abs(out.cpu().numpy() - want)[n:] <= tol[n:]).all()
        e = np.zeros(k.shape, np.float16)
        ref.read(cache[0], cache[1], e, cu, lens, table)
        assert np.array_equal(outs[0].cpu().numpy()[n:], e[n:])
    if what == "long":
        own = table[0][table[0] >= 0]
        assert (out[:n] == 7).all() and (outs[0][:n] == 7).all()
        assert torch.equal(c.k_codes[own], before[0][own]) and torch.equal(c.k_scales[own], before[1][own])
    if what == "page":                # rows without a page: left as they are
        assert (outs[0][n - 1] == 7).all()


def test_refusals(dp):
    H, P, D = 2, 16, 64
    rng = np.random.default_rng(1)
    cu, lens, table, blocks = ref.random_batch(rng, [1], [20], P)
    c, b = _handles(dp, ref.random_cache(rng, blocks, H, P, D), cu, lens, table)
    q, k = _rows(rng, 1, 4, D), _rows(rng, 1, H, D)
    out = torch.empty_like(q)
    ok = dict(scale=0.1, window=0, sinks=0)
    for bad in (dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(dp.DptqError):
            dp.dptq_kv4_attention(c, b, q, out, **(ok | bad))
    with pytest.raises(dp.DptqError):                                     # 3 query heads over 2
        dp.dptq_kv4_attention(c, b, q[:, :3].contiguous(), out[:, :3].contiguous(), 0.1)
    with pytest.raises(ValueError):
        dp.dptq_kv4_attention(c, b, q, out[:, :2], 0.1)
    for call in (dp.dptq_kv4_append, dp.dptq_kv4_read):
        with pytest.raises(TypeError):
            call(c, b, k.float(), k)
        with pytest.raises(ValueError):
            call(c, b, k[:, :, :32], k)
        two = _rows(rng, 2, H, D, 3)                                      # rows 2-byte aligned
        b2 = _handles(dp, ref.random_cache(rng, blocks, H, P, D), np.array([0, 2], np.int32), lens, table)[1]
        with pytest.raises(dp.DptqError):
            call(c, b2, two, two)
        with pytest.raises(ValueError):                                   # distances that differ
            call(c, b2, _rows(rng, 2, H, D, 8), _rows(rng, 2, H, D))
        shift = torch.zeros((H * D + 8,), dtype=torch.float16, device="cuda")[1:1 + H * D].view(1, H, D)
        with pytest.raises(dp.DptqError):
            call(c, b, shift, shift)
    with pytest.raises(TypeError):
        dp.Kv4Cache(c.k_codes.view(torch.int8), c.v_codes, c.k_scales, c.v_scales)
    with pytest.raises(TypeError):
        dp.Kv4Cache(c.k_codes, c.v_codes, c.k_scales.half(), c.v_scales)
    with pytest.raises(ValueError):
        dp.Kv4Cache(c.k_codes, c.v_codes, c.k_scales[:, :, 0].contiguous(), c.v_scales)
    for blk, dim in ((8, 64), (48, 64), (256, 64), (16, 32), (16, 96), (16, 256)):
        bad = dp.Kv4Cache.empty(3, H, blk, dim)
        bb = dp.Kv8Batch(b.cu_tokens, b.seq_lens, b.block_table, tokens=1, max_tokens=1, max_len=16)
        qq = torch.zeros((1, 4, dim), dtype=torch.float16, device="cuda")
        with pytest.raises(dp.DptqError) as e:
            dp.dptq_kv4_attention(bad, bb, qq, torch.empty_like(qq), 0.1)
        assert e.value.status == 2
    # nothing to do
    none = dp.Kv8Batch(torch.zeros(1, dtype=torch.int32, device="cuda"),
                       torch.zeros(0, dtype=torch.int32, device="cuda"),
                       torch.zeros((0, 1), dtype=torch.int32, device="cuda"), tokens=0, max_tokens=0, max_len=0)
    dp.dptq_kv4_append(c, none, k[:0], k[:0])
    dp.dptq_kv4_read(c, none, k[:0], k[:0])
    dp.dptq_kv4_attention(c, none, q[:0], out[:0], 0.1)
    b.device += 1                                     # (as if its arrays were on another GPU)
    for call in (lambda: dp.dptq_kv4_append(c, b, k, k), lambda: dp.dptq_kv4_read(c, b, k, k),
                 lambda: dp.dptq_kv4_attention(c, b, q, out, 0.1)):
        with pytest.raises(ValueError):
            call()
