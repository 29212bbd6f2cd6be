"""Prompts over the 4-bit cache in every form of the kernel: tasks cut along the keys, many sequences, scales that
binary16 does not hold, and decode batches of many sequences; against 64 bits on the GPU."""
import math

import numpy as np
import pytest

import kv4_reference as ref
from test_kv4_gpu import _attend, _check, _cuda, _rows, dp  # noqa: F401  (dp: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _against_doubles(dp, cache, q, cu, lens, table, window=0, sinks=0):  # noqa: F811
    """As the reference's attend, on the GPU (its tolerance per row from the row's own largest terms)."""
    got, scale = _attend(dp, cache, q, cu, lens, table, window, sinks)
    kc, vc = (torch.from_numpy(ref.values(c, b)).cuda() for c, b in (cache[:2], cache[2:]))
    H, P, D = kc.shape[1:]
    g = q.shape[1] // H
    out = torch.from_numpy(got).cuda().double()
    for s in range(len(lens)):
        n, L = int(cu[s + 1] - cu[s]), int(lens[s])
        if n == 0:
            continue
        pages = torch.from_numpy(table[s, :-(-L // P)]).long().cuda()
        pos = torch.arange(L - n, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        vis = j <= pos
        if window:
            vis = vis & ((j > pos - window) | (j < sinks))
        for h in range(H):
            K, V = (t[pages, h].reshape(-1, D)[:L].double() for t in (kc, vc))
            x = q[cu[s]:cu[s] + n, h * g:(h + 1) * g].double().transpose(0, 1)
            a = (x @ K.t() * scale).masked_fill(~vis, -math.inf)
            w = torch.softmax(a, dim=2)
            mag = (x.abs() @ K.abs().t() * abs(scale)).masked_fill(~vis, 0).amax(dim=2, keepdim=True)
            o = w @ V
            rel = 2.0 ** -11 + 2 * (D + 16) * 2.0 ** -23 * mag + (L / 16 + 64) * 2.0 ** -23
            big = V.abs().amax()
            # (below the weights' normal range 2^-32 of the largest weight, for every key)
            tol = rel * (w @ V.abs()) + 2.0 ** -32 * w.amax(dim=2, keepdim=True) * L * big + 2.0 ** -11 * o.abs() + 2.0 ** -24
            y = out[cu[s]:cu[s] + n, h * g:(h + 1) * g].transpose(0, 1)
            bad = ~((y - o).abs() <= tol)
            assert not bad.any(), (s, h, int(bad.sum()), (y - o)[bad][:5].tolist(), tol[bad][:5].tolist())
    dp.dptq_last_device_error()


# rows and lengths, KV heads, query heads of each, dims, window: one wave of tasks in up to ten parts; some more than
# whole waves of CTAs alone, and of pairs; tasks of half a wave in three parts; with a window and sinks
CUT = [([70], [9000], 1, 8, 128, 0, 0), ([40, 33, 0, 64], [7000, 2600, 77, 3000], 2, 4, 128, 0, 0), ([300], [3200], 80, 1, 128, 0, 0),
       ([600, 520], [3300, 3200], 22, 1, 128, 0, 0), ([270, 260], [3000, 2900], 45, 1, 64, 0, 0), ([520], [4000], 5, 8, 128, 0, 0),
       ([300, 260], [6000, 5000], 4, 2, 128, 3000, 5), ([513], [5000], 3, 1, 128, 2700, 200), ([256], [2700], 1, 2, 64, 0, 0)]


@pytest.mark.parametrize("ns,lens,H,g,D,window,sinks", CUT)
def test_tasks_cut_along_their_keys(dp, ns, lens, H, g, D, window, sinks):  # noqa: F811
    rng = np.random.default_rng(H + D)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 32)
    cache = ref.random_cache(rng, blocks, H, 32, D)
    q = _rows(rng, sum(ns), H * g, D)
    _against_doubles(dp, cache, q, cu, lens, table, window, sinks)
    first, _ = _attend(dp, cache, q, cu, lens, table, window, sinks)
    again, _ = _attend(dp, cache, q, cu, lens, table, window, sinks)
    assert np.array_equal(first, again)


@pytest.mark.parametrize("n,S,g,D", [(17, 40, 1, 64), (9, 33, 8, 128), (90, 35, 6, 128)])
def test_more_sequences_than_a_warp_has_lanes(dp, n, S, g, D):  # noqa: F811
    rng = np.random.default_rng(S)
    ns = [int(v) for v in rng.integers(0, n + 1, S)]
    ns[3] = n
    lens = [k + int(v) for k, v in zip(ns, rng.integers(0, 300, S))]
    lens[5] = 0
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    _check(dp, ref.random_cache(rng, blocks, 2, 16, D), _rows(rng, sum(ns), 2 * g, D), cu, lens, table)


@pytest.mark.parametrize("S,top,H,g,D", [(300, 700, 1, 4, 128), (150, 90, 2, 1, 64), (129, 2000, 1, 16, 128), (1, 30000, 1, 8, 128),
                                         (2, 11000, 3, 5, 64), (8, 2048, 8, 8, 128), (3, 1400, 8, 1, 128)])
def test_single_tokens_of_many_and_of_long_sequences(dp, S, top, H, g, D):  # noqa: F811
    """Steps shared equally and cut by heads, results joined at once and in two levels."""
    rng = np.random.default_rng(S)
    lens = [int(v) for v in rng.integers(0, top, S)]
    lens[S // 2] = top
    cu, lens, table, blocks = ref.random_batch(rng, [1] * S, lens, 64)
    _check(dp, ref.random_cache(rng, blocks, H, 64, D), _rows(rng, S, H * g, D), cu, lens, table)


@pytest.mark.parametrize("ns,lens,H,g,D", [([1, 2], [300, 290], 2, 4, 128), ([40], [900], 1, 2, 128), ([300], [300], 3, 2, 64),
                                           ([600, 520], [900, 520], 2, 2, 128)])
def test_scales_below_binary16(dp, ns, lens, H, g, D):  # noqa: F811
    """Scales from the smallest bfloat16 to 2^-17, alone and beside ordinary ones: values are rounded once, and where all
    of a cache's values are that small, so is the output."""
    rng = np.random.default_rng(D)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    q = _rows(rng, sum(ns), H * g, D)
    tiny = ref.bf16_bits((2.0 ** rng.uniform(-30, -16.5, cache[1].shape)).astype(np.float32))
    tiny[rng.random(tiny.shape) < 0.1] = 1
    some = rng.random(tiny.shape) < 0.5
    for kv in (1, 3):
        cache[kv] = np.where(some, tiny, cache[kv])
    _against_doubles(dp, cache, q, cu, lens, table)
    cache[3] = ref.bf16_bits((2.0 ** rng.uniform(-18.5, -17, cache[3].shape)).astype(np.float32))
    got, scale = _attend(dp, cache, q, cu, lens, table)
    want, tol = ref.attend(cache, q.cpu().numpy(), cu, lens, table, scale)
    # (each cached value is a rounding of at most 2^-25 away from what the decode kernel takes)
    assert (np.abs(got - want) <= tol + 2.0 ** -25).all() and np.abs(got).max() > 2.0 ** -17


@pytest.mark.parametrize("n", [1, 60, 600])
def test_the_largest_scale_and_those_above(dp, n):  # noqa: F811
    """9344 serves; above it, and below zero, a scale is no number for the rows that see its key."""
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n], [200 + n], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, 128)
    cache[3][table[0, 2], 0, 5] = 0x4612
    q = _rows(rng, n, 2, 128)
    _against_doubles(dp, cache, q, cu, lens, table)
    for kv, bits in ((1, 0x4613), (3, 0x4613), (1, 0x8000), (3, 0xBF80)):
        bad = [a.copy() for a in cache]
        bad[kv][table[0, 12], 0, 2] = bits         # position 194: all rows
        got, _ = _attend(dp, bad, q, cu, lens, table)
        assert np.isnan(got).all()


def test_two_streams_in_turn_share_the_scratch(dp):  # noqa: F811
    """Calls ordered by events on two streams, cut along the keys and joined in the same scratch."""
    rng = np.random.default_rng(0)
    data = []
    for n in (70, 1):
        cu, lens, table, blocks = ref.random_batch(rng, [n], [9000], 32)
        cache = ref.random_cache(rng, blocks, 1, 32, 128)
        kc, vc, cut, lt, tt = _cuda(cache[0], cache[2], cu, lens, table)
        scales = [torch.from_numpy(b.astype(np.int32)).to(torch.int16).cuda().view(torch.bfloat16) for b in (cache[1], cache[3])]
        q = _rows(rng, n, 8, 128)
        data.append((dp.Kv4Cache(kc, vc, *scales), dp.Kv8Batch(cut, lt, tt, tokens=n, max_tokens=n, max_len=9000), q,
                     torch.empty_like(q), (kc, vc, scales, cut, lt, tt)))
    torch.cuda.synchronize()
    for c, b, q, out, _ in data:
        dp.dptq_kv4_attention(c, b, q, out, 0.1)
    torch.cuda.synchronize()
    first = [d[3].clone() for d in data]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(10):
        c, b, q, out, _ = data[i % 2]
        with torch.cuda.stream(streams[i % 2]):
            streams[i % 2].wait_stream(streams[1 - i % 2])
            out.zero_()
            dp.dptq_kv4_attention(c, b, q, out, 0.1)
    torch.cuda.synchronize()
    assert all(torch.equal(a, d[3]) for a, d in zip(first, data))


@pytest.mark.parametrize("n", [1, 60, 600])
@pytest.mark.parametrize("D", [64, 128])
def test_the_largest_values_where_no_query_looks(dp, n, D):  # noqa: F811
    """Unused memory may hold the code -8, which append does not make: times 9344 it is no binary16 number."""
    rng = np.random.default_rng(n)
    cu, lens, table, blocks = ref.random_batch(rng, [n], [200 + n], 16)
    cache = ref.random_cache(rng, blocks, 1, 16, D)
    q = _rows(rng, n, 2, D)
    got, _ = _attend(dp, cache, q, cu, lens, table, window=50)
    last, used = table[0, (lens[0] - 1) // 16], (lens[0] - 1) % 16 + 1
    for page, slots in ((last, slice(used, 16)), (table[0, 2], slice(0, 16))):
        for kv in (0, 2):
            cache[kv][page, :, slots], cache[kv + 1][page, :, slots] = 0x88, 0x4612
    again, _ = _attend(dp, cache, q, cu, lens, table, window=50)
    assert np.array_equal(got, again)


@pytest.mark.parametrize("ns,lens,g", [([64, 40], [0, 9000], 8), ([20, 40, 30], [7, 7000, 0], 4)])
def test_padding_slots_beside_tasks_that_are_cut(dp, ns, lens, g):  # noqa: F811
    """Rows of sequences of length zero, or longer than their sequence, see nothing in any part."""
    rng = np.random.default_rng(g)
    cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 32)
    _check(dp, ref.random_cache(rng, blocks, 2, 32, 128), _rows(rng, sum(ns), 2 * g, 128), cu, lens, table)


def test_fewer_rows_than_declared(dp):  # noqa: F811
    """A batch padded to its bounds: more tokens, rows and length declared than there are; the rest stays as it is."""
    rng = np.random.default_rng(1)
    for ns, lens, g in (([3, 1], [40, 900], 2), ([30, 90], [2000, 300], 4), ([560], [3000], 1)):
        cu, lens, table, blocks = ref.random_batch(rng, ns, lens, 16)
        table = np.pad(table, ((0, 0), (0, 100)), constant_values=-1)
        cache = ref.random_cache(rng, blocks, 2, 16, 128)
        T = sum(ns)
        kc, vc, cut, lt, tt = _cuda(cache[0], cache[2], cu, lens, table)
        ks, vs = (torch.from_numpy(b.astype(np.int32)).to(torch.int16).cuda().view(torch.bfloat16) for b in (cache[1], cache[3]))
        c = dp.Kv4Cache(kc, vc, ks, vs)
        b = dp.Kv8Batch(cut, lt, tt, tokens=T + 900, max_tokens=max(ns) + 700, max_len=int(lens.max()) + 1500)
        q, out = _rows(rng, T + 900, 2 * g, 128), torch.full((T + 900, 2 * g, 128), 7.0, dtype=torch.float16, device="cuda")
        dp.dptq_kv4_attention(c, b, q, out, 0.09)
        want, tol = ref.attend(cache, q[:T].cpu().numpy(), cu, lens, table, 0.09)
        assert (np.abs(out[:T].cpu().numpy() - want) <= tol).all() and (out[T:] == 7).all()
        k, v = (torch.full((T + 900, 2, 128), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
        dp.dptq_kv4_read(c, b, k, v)
        e = np.full((T + 900, 2, 128), 7, np.float16)
        ref.read(cache[0], cache[1], e, cu, lens, table)
        assert np.array_equal(k.cpu().numpy(), e)
        x = q.clone()
        dp.dptq_rotary(dp.Rotary(128), b, x)
        assert torch.equal(x[T:], q[T:]) and not torch.equal(x[:T], q[:T])
        new = _rows(rng, T + 900, 2, 128)
        dp.dptq_kv4_append(c, b, new, new)
        ref.append(cache[0], cache[1], new[:T].cpu().numpy(), cu, lens, table)
        assert np.array_equal(c.k_codes.cpu().numpy(), cache[0])
        dp.dptq_last_device_error()


@pytest.mark.parametrize("H,D", [(1023, 64), (1000, 128)])
def test_many_heads(dp, H, D):  # noqa: F811
    rng = np.random.default_rng(H)
    cu, lens, table, blocks = ref.random_batch(rng, [2, 1], [18, 5], 16)
    cache = ref.random_cache(rng, blocks, H, 16, D)
    q = _rows(rng, 3, H, D)
    _check(dp, cache, q, cu, lens, table)
    kc, vc, cut, lt, tt = _cuda(cache[0], cache[2], cu, lens, table)
    ks, vs = (torch.from_numpy(b.astype(np.int32)).to(torch.int16).cuda().view(torch.bfloat16) for b in (cache[1], cache[3]))
    c, b = dp.Kv4Cache(kc, vc, ks, vs), dp.Kv8Batch(cut, lt, tt, tokens=3, max_tokens=2, max_len=18)
    k, v = _rows(rng, 3, H, D), _rows(rng, 3, H, D)
    dp.dptq_kv4_append(c, b, k, v)
    ref.append(cache[0], cache[1], k.cpu().numpy(), cu, lens, table)
    ref.append(cache[2], cache[3], v.cpu().numpy(), cu, lens, table)
    assert np.array_equal(c.k_codes.cpu().numpy(), cache[0]) and np.array_equal(c.v_codes.cpu().numpy(), cache[2])
    back = [torch.empty_like(k) for _ in range(2)]
    dp.dptq_kv4_read(c, b, *back)
    e = np.zeros((3, H, D), np.float16)
    ref.read(cache[2], cache[3], e, cu, lens, table)
    assert np.array_equal(back[1].cpu().numpy(), e)
    dp.dptq_last_device_error()
