"""The int8 paged KV cache: dptq_kv8_append bit for bit against its definition, and
dptq_kv8_attention against a plain form in 64 bits, for single tokens, a few tokens and prompts."""
import math

import numpy as np
import pytest

import kv8_reference as ref

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


def _handles(dp, cache, cu, lens, table, max_tokens=None, max_len=None):
    kc, ks, vc, vs = _cuda(*cache)
    c = dp.Kv8Cache(kc, vc, ks, vs)
    n = np.diff(cu)
    cut, lt, tt = _cuda(cu, lens, table)
    b = dp.Kv8Batch(cut, lt, tt, tokens=int(cu[-1]), max_tokens=max_tokens or max(1, int(n.max(initial=0))),
                    max_len=int(lens.max(initial=0)) if max_len is None else max_len)
    return c, b


def _rows(rng, T, H, D, pad=0):
    """float16 [T, H, D] as a view into rows of H D + pad values."""
    x = torch.from_numpy(rng.standard_normal((T, H * D + pad)).astype(np.float16)).cuda()
    return x[:, :H * D].unflatten(1, (H, D))


def _attend(dp, cache, q, cu, lens, table, window=0, sinks=0, scale=None, **kw):
    D = q.shape[2]
    scale = 1 / math.sqrt(D) if scale is None else scale
    c, b = _handles(dp, cache, cu, lens, table, **kw)
    out = torch.full(q.shape, float("nan"), dtype=torch.float16, device="cuda")
    dp.dptq_kv8_attention(c, b, q, out, scale, window=window, sinks=sinks)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64), scale


def _check_attend(dp, cache, q, cu, lens, table, window=0, sinks=0, scale=None, **kw):
    got, scale = _attend(dp, cache, q, cu, lens, table, window, sinks, scale, **kw)
    want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, scale, window, sinks)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], tol[bad][:5])
    dp.dptq_last_device_error()


# ---------------------------------------------------------------------------------- append
@pytest.mark.parametrize("H,D,P", [(1, 64, 16), (3, 128, 16), (2, 64, 32), (8, 128, 64), (5, 128, 128), (2, 64, 128)])
def test_append_matches_its_definition(dp, H, D, P):
    rng = np.random.default_rng(H * 1000 + D + P)
    # a first token, a page's last row, its first, prompts over several pages, a prefix that ends
    # inside a page, no rows, a padding slot of length 0, a sequence shorter than its rows
    ns = [1, 1, 1, 5 * P + 3, 2 * P, 0, 1, 4, P - 1]
    lens = [1, 2 * P, 2 * P + 1, 5 * P + 3, 2 * P + P // 2, 7, 0, 3, 3 * P]
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    want = [a.copy() for a in cache]
    c, b = _handles(dp, cache, cu, lens, table)
    k, v = _rows(rng, int(cu[-1]), H, D, 8), _rows(rng, int(cu[-1]), H, D, 8)
    k[::3] *= 40
    v[1] = 0
    for _ in range(2):      # the second call finds its own codes and scales
        dp.dptq_kv8_append(c, b, k, v)
        ref.append(want[0], want[1], k.cpu().numpy(), cu, lens, table)
        ref.append(want[2], want[3], v.cpu().numpy(), cu, lens, table)
        for name, t, w in zip("kc ks vc vs".split(), (c.k_codes, c.k_scales, c.v_codes, c.v_scales), want):
            assert np.array_equal(t.cpu().numpy(), w), name
    dp.dptq_last_device_error()


@pytest.mark.parametrize("P", [16, 128])
def test_append_token_by_token_keeps_a_page_of_growing_rows(dp, P):
    H, D, steps = 2, 128, P + 5
    rng = np.random.default_rng(P)
    cu, lens, table, blocks = ref.random_batch(rng, [1, 1], [steps, steps], P)
    cache = [np.zeros((blocks, H, P, D), np.int8), np.full((blocks, H), np.nan, np.float32),
             np.zeros((blocks, H, P, D), np.int8), np.full((blocks, H), np.nan, np.float32)]
    want = [a.copy() for a in cache]
    c, b = _handles(dp, cache, cu, lens, table)
    for t in range(1, steps + 1):
        now = np.array([t, t], np.int32)
        b.seq_lens.copy_(torch.from_numpy(now))
        k, v = _rows(rng, 2, H, D) * (1 + 0.3 * t), _rows(rng, 2, H, D)
        dp.dptq_kv8_append(c, b, k, v)
        ref.append(want[0], want[1], k.cpu().numpy(), cu, now, table)
        ref.append(want[2], want[3], v.cpu().numpy(), cu, now, table)
    for t, w in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales), want):
        assert np.array_equal(t.cpu().numpy(), w, equal_nan=w.dtype == np.float32)


def test_append_zeros_ties_and_non_finite_values(dp):
    H, D, P = 2, 64, 16
    rng = np.random.default_rng(0)
    cu, lens, table, blocks = ref.random_batch(rng, [P, P, P], [P, P, P], P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    x = (rng.integers(-254, 255, (3 * P, H, D)) * 0.5).astype(np.float16)
    x[:, :, 0] = 127.0                      # s = 1: half of the values tie
    x[P:2 * P] = 0                          # a page of zeros
    x[2 * P, 0, 3] = np.nan
    x[2 * P + 1, 1, 5] = np.inf
    want = [a.copy() for a in cache]
    c, b = _handles(dp, cache, cu, lens, table)
    k = torch.from_numpy(x).cuda()
    dp.dptq_kv8_append(c, b, k, k)
    ref.append(want[0], want[1], x, cu, lens, table)
    ref.append(want[2], want[3], x, cu, lens, table)
    for t, w in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales), want):
        assert np.array_equal(t.cpu().numpy(), w)


# ---------------------------------------------------------------------------------- attention
LENS = [1, 2, 15, 16, 17, 31, 64, 100, 127, 128, 129, 500, 1025]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("H,g", [(1, 1), (2, 4), (1, 8), (3, 5), (2, 16), (1, 40)])
def test_single_tokens(dp, D, P, H, g):
    rng = np.random.default_rng(D + P + 10 * g)
    cu, lens, table, blocks = ref.random_batch(rng, [1] * len(LENS), LENS, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    _check_attend(dp, cache, _rows(rng, len(LENS), H * g, D, 16), cu, lens, table)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 16), (33, 1), (100, 40), (128, 200), (5000, 3)])
@pytest.mark.parametrize("n", [1, 3])
def test_single_and_few_tokens_with_window_and_sinks(dp, window, sinks, n):
    rng = np.random.default_rng(window + sinks)
    lens = [l + n - 1 for l in LENS]
    cu, lens, table, blocks = ref.random_batch(rng, [n] * len(lens), lens, 32)
    cache = ref.random_cache(rng, blocks, 2, 32, 128)
    _check_attend(dp, cache, _rows(rng, len(lens) * n, 8, 128), cu, lens, table, window, sinks)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,g", [(1, 1), (2, 2), (1, 8), (1, 3), (1, 64)])
def test_few_tokens(dp, D, H, g):
    """Two to five rows a sequence, ragged, behind contexts of zero to a thousand tokens."""
    rng = np.random.default_rng(D + g)
    ns = [2, 5, 3, 1, 4, 2]
    lens = [2, 5, 20, 300, 130, 1000]
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    _check_attend(dp, cache, _rows(rng, sum(ns), H * g, D), cu, lens, table)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 64, 128])
@pytest.mark.parametrize("H,g", [(2, 1), (1, 4), (1, 7)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3), (200, 0)])
def test_prompts(dp, D, P, H, g, window, sinks):
    """Ragged prompts, some behind a context, with a sequence of one row among them."""
    rng = np.random.default_rng(D + P + g + window)
    ns = [257, 1, 100, 333, 64]
    lens = [257, 77, 100, 700, 1300]
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    _check_attend(dp, cache, _rows(rng, sum(ns), H * g, D, 24), cu, lens, table, window, sinks)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_one_long_sequence(dp, n):
    """Few rows and a long axis: the work is split along it and joined."""
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n], [20011], 64)
    cache = ref.random_cache(rng, blocks, 1, 64, 128)
    q = _rows(rng, n, 4, 128)
    _check_attend(dp, cache, q, cu, lens, table)
    _check_attend(dp, cache, q, cu, lens, table, 3000, 70)


@pytest.mark.parametrize("n", [1, 3, 130])
def test_rows_that_see_nothing_are_zero(dp, n):
    rng = np.random.default_rng(n)
    ns, lens = [n, n, n, 0], [0, max(0, n - 2), 40 + n, 9]
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, 2, 16, 128)
    _check_attend(dp, cache, _rows(rng, sum(ns), 4, 128), cu, lens, table)
    if n == 130:
        _check_attend(dp, cache, _rows(rng, sum(ns), 4, 128), cu, lens, table, 5, 2)


@pytest.mark.parametrize("n", [1, 130])
def test_what_is_not_seen_does_not_count(dp, n):
    """Codes past the end, pages outside the window and other sequences' pages may hold anything,
    NaN and infinite scales included."""
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
        other[1][b], other[3][b] = np.nan, np.inf
        other[0][b], other[2][b] = -128, 127
    last, used = table[0, (lens[0] - 1) // P], (lens[0] - 1) % P + 1
    other[0][last, :, used:], other[2][last, :, used:] = 127, -128
    t2 = table.copy()
    t2[0, 1:first] = -1                          # pages that no query sees need not be there
    again, _ = _attend(dp, other, q, cu, lens, t2, W, 3)
    assert np.array_equal(got, again)
    dp.dptq_last_device_error()


@pytest.mark.parametrize("n", [1, 130])
def test_pages_of_zeros_and_scales_far_apart(dp, n):
    """V scales from 2^-40 to 2^9 and pages of zeros (scale 0) side by side."""
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n, n], [300 + n, 90 + n], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, 64)
    cache[3][:] = (2.0 ** rng.uniform(-30, 2, cache[3].shape)).astype(np.float32)
    for b in rng.choice(blocks, blocks // 4, replace=False):
        cache[2][b], cache[3][b] = 0, 0
        cache[0][b], cache[1][b] = 0, 0
    _check_attend(dp, cache, _rows(rng, 2 * n, 4, 64), cu, lens, table)
    cache[2][:], cache[3][:] = 0, 0
    got, _ = _attend(dp, cache, _rows(rng, 2 * n, 4, 64), cu, lens, table)
    assert not got.any()


@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_flat_and_sharp_softmax(dp, n, scale):
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n], [333], 32)
    cache = ref.random_cache(rng, blocks, 2, 32, 128)
    cache[1][:] = np.float32(1 / 127)
    _check_attend(dp, cache, _rows(rng, n, 4, 128), cu, lens, table, scale=scale)


@pytest.mark.parametrize("n", [1, 3, 150])
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


def test_offsets_past_32_bits(dp):
    """Pages whose codes lie beyond 2^31 and 2^32 bytes."""
    H, P, D = 8, 128, 128
    blocks = (1 << 32) // (H * P * D) + 3
    codes = [torch.zeros((blocks, H, P, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.ones((blocks, H), device="cuda") for _ in range(2)]
    c = dp.Kv8Cache(codes[0], codes[1], scales[0], scales[1])
    pages = [blocks - 1, 0, blocks // 2 + 1, blocks - 2]
    rng = np.random.default_rng(0)
    for n in (1, 470):
        cu, lens = np.array([0, n], np.int32), np.array([500], np.int32)
        table = np.array([pages], np.int32)
        b = dp.Kv8Batch(*_cuda(cu, lens, table), tokens=n, max_tokens=n, max_len=500)
        k, v = _rows(rng, n, H, D), _rows(rng, n, H, D)
        dp.dptq_kv8_append(c, b, k, v)
        small = [codes[0][pages].cpu().numpy(), scales[0][pages].cpu().numpy(), codes[1][pages].cpu().numpy(),
                 scales[1][pages].cpu().numpy()]
        q = _rows(rng, n, H, D)
        out = torch.empty((n, H, D), dtype=torch.float16, device="cuda")
        dp.dptq_kv8_attention(c, b, q, out, 0.1)
        want, tol = ref.attend(small, q.cpu().numpy(), cu, lens, np.arange(4, dtype=np.int32)[None], 0.1)
        assert (np.abs(out.cpu().numpy() - want) <= tol).all()
        assert codes[0][pages[-1]].any()
    dp.dptq_last_device_error()


def test_the_same_bits_every_time(dp):
    rng = np.random.default_rng(2)
    for ns, lens in (([1] * 5, [3000, 17, 900, 5000, 64]), ([64, 300], [9000, 300])):
        cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 32)
        cache = ref.random_cache(rng, blocks, 2, 32, 128)
        q = _rows(rng, sum(ns), 8, 128)
        first, _ = _attend(dp, cache, q, cu, lens, table)
        for _ in range(5):
            again, _ = _attend(dp, cache, q, cu, lens, table)
            assert np.array_equal(first, again)


def test_another_stream_and_a_captured_step(dp):
    """Append then attend on a side stream, and the same step replayed from a CUDA graph with new
    lengths in the same arrays."""
    rng = np.random.default_rng(11)
    H, g, P, D = 2, 4, 16, 128
    cu, lens, table, blocks = ref.random_batch(rng, [1, 1], [600, 40], P)
    cache = ref.random_cache(rng, blocks, H, P, D)
    c, b = _handles(dp, cache, cu, lens, table)
    k, v, q = _rows(rng, 2, H, D), _rows(rng, 2, H, D), _rows(rng, 2, H * g, D)
    out = torch.empty((2, H * g, D), dtype=torch.float16, device="cuda")

    def step():
        dp.dptq_kv8_append(c, b, k, v)
        dp.dptq_kv8_attention(c, b, q, out, 0.09)

    def expect(lens):
        want = [a.copy() for a in cache]
        ref.append(want[0], want[1], k.cpu().numpy(), cu, lens, table)
        ref.append(want[2], want[3], v.cpu().numpy(), cu, lens, table)
        o, tol = ref.attend(want, q.cpu().numpy(), cu, lens, table, 0.09)
        assert (np.abs(out.cpu().numpy() - o) <= tol).all()

    def reset():
        for t, a in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales), cache):
            t.copy_(torch.from_numpy(a))
        out.fill_(float("nan"))

    dp.dptq_kv8_reserve()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    expect(lens)
    reset()
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
def test_batches_that_contradict_themselves_are_reported(dp):
    rng = np.random.default_rng(1)
    H, P, D = 2, 16, 64
    for n in (1, 140):
        cu, lens, table, blocks = ref.random_batch(rng, [n, n], [150 + n, 200 + n], P)
        cache = ref.random_cache(rng, blocks, H, P, D)
        q, k = _rows(rng, 2 * n, 4, D), _rows(rng, 2 * n, H, D)
        for what in ("page", "long", "many", "order"):
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
            c, b = _handles(dp, cache, cu2, lens2, t2, max_tokens=n, **kw)
            out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
            dp.dptq_kv8_attention(c, b, q, out, 0.1)
            with pytest.raises(dp.DptqError) as e:
                dp.dptq_last_device_error()
            assert e.value.status == 1
            dp.dptq_last_device_error()                                   # cleared
            before = [t.clone() for t in (c.k_codes, c.k_scales)]
            dp.dptq_kv8_append(c, b, k, k)
            with pytest.raises(dp.DptqError):
                dp.dptq_last_device_error()
            if what in ("long", "page"):      # the other sequence is served
                want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, 0.1)
                assert (np.abs(out.cpu().numpy() - want)[n:] <= tol[n:]).all()
                assert what == "page" or (out[:n] == 7).all()
                own = table[0][table[0] >= 0]
                if what == "long":
                    assert torch.equal(c.k_codes[own], before[0][own]) and torch.equal(c.k_scales[own], before[1][own])


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
            dp.dptq_kv8_attention(c, b, q, out, **(ok | bad))
    with pytest.raises(dp.DptqError):                                     # 3 query heads over 2
        dp.dptq_kv8_attention(c, b, q[:, :3].contiguous(), out[:, :3].contiguous(), 0.1)
    with pytest.raises(ValueError):
        dp.dptq_kv8_attention(c, b, q, out[:, :2], 0.1)
    with pytest.raises(TypeError):
        dp.dptq_kv8_append(c, b, k.float(), k)
    with pytest.raises(ValueError):
        dp.dptq_kv8_append(c, b, k[:, :, :32], k)
    two = _rows(rng, 2, H, D, 3)                                          # rows 2-byte aligned
    b2 = _handles(dp, ref.random_cache(rng, blocks, H, P, D), np.array([0, 2], np.int32), lens, table)[1]
    with pytest.raises(dp.DptqError):
        dp.dptq_kv8_append(c, b2, two, two)
    shift = torch.zeros((H * D + 8,), dtype=torch.float16, device="cuda")[1:1 + H * D].view(1, H, D)
    with pytest.raises(dp.DptqError):
        dp.dptq_kv8_append(c, b, shift, shift)
    for blk, dim in ((8, 64), (48, 64), (256, 64), (16, 32), (16, 96), (16, 256)):
        codes = torch.zeros((3, H, blk, dim), dtype=torch.int8, device="cuda")
        s = torch.zeros((3, H), device="cuda")
        bad = dp.Kv8Cache(codes, codes.clone(), s, s.clone())
        bb = dp.Kv8Batch(b.cu_tokens, b.seq_lens, b.block_table, tokens=1, max_tokens=1, max_len=16)
        qq = torch.zeros((1, 4, dim), dtype=torch.float16, device="cuda")
        with pytest.raises(dp.DptqError) as e:
            dp.dptq_kv8_attention(bad, bb, qq, torch.empty_like(qq), 0.1)
        assert e.value.status == 2
    long = dp.Kv8Batch(b.cu_tokens, b.seq_lens, b.block_table, tokens=1, max_tokens=1, max_len=1000)
    with pytest.raises(dp.DptqError):
        dp.dptq_kv8_attention(c, long, q, out, 0.1)
    # nothing to do
    none = dp.Kv8Batch(torch.zeros(1, dtype=torch.int32, device="cuda"),
                       torch.zeros(0, dtype=torch.int32, device="cuda"),
                       torch.zeros((0, 1), dtype=torch.int32, device="cuda"), tokens=0, max_tokens=0, max_len=0)
    dp.dptq_kv8_append(c, none, k[:0], k[:0])
    dp.dptq_kv8_attention(c, none, q[:0], out[:0], 0.1)
