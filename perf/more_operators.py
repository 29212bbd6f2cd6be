"""What rotary positions and the paged cache of 4-bit codes are timed on.

A case is a dict of plain values.  `kind` names the operator:

  rotary  rotary positions of the query and key heads that a projection left side by side: pairs of
          both layouts, the whole head or its first part, frequencies scaled for long contexts
          (dptq_rotary)
  write   new K and V rows quantized into the cache (dptq_kv4_append) and read back as the values
          that the cache now stands for (dptq_kv4_read): what an evaluation of the 4-bit cache does
          with every token, and the only way to have the codes as values
  read    whole cached sequences back as binary16 rows (dptq_kv4_read): a prefix that another
          program continues, or a cache that moves to another format
  attend  causal attention over the cache, for single tokens, for chunks of new tokens behind a
          context and for prompts, with an optional sliding window and first tokens that stay
          visible (dptq_kv4_attention)

Head counts and widths are those of the LLaMA geometries in paper_2606_12487_gb300/inputs.py (7B: 32
heads of 128; 13B: 40; LLaMA-3-8B: 32 over 8; 70B: 64 over 8).

The cache: two's complement nibbles, low nibble first, and a bfloat16 scale for every token and head;
a value is scale times code.  Every step of the quantizer is defined in 32 bits, so codes and
scales are the same on both sides.

`own` false: the plain form, elementary operations in 32 bits (angles in 64).  True: the library's
calls.
"""
import math

import torch

own = False
DEV = "cuda"


def listed():
    return [
        # One token of LLaMA-3-8B behind a middling context: launch latency.
        dict(name="rotary_s1_h40", kind="rotary", S=1, new=1, lo=5000, hi=5000, H=40, D=128, rot=128,
             interleaved=False, scaling="none", factor=1.0),
        # A prompt of odd length, LLaMA-2-13B, half of each head rotated, neighbouring pairs.
        dict(name="rotary_n1333_part", kind="rotary", S=1, new=1333, lo=0, hi=0, H=80, D=128, rot=64,
             interleaved=True, scaling="linear", factor=4.0),
        # The next 8192 tokens of a LLaMA-2-70B document of 100000, frequencies scaled by wavelength.
        dict(name="rotary_n8192_far", kind="rotary", S=1, new=8192, lo=100000, hi=100000, H=72, D=128, rot=128,
             interleaved=False, scaling="wavelength", factor=8.0),
        # One new token of each of 32 LLaMA-2-7B sequences.
        dict(name="write_step_s32", kind="write", S=32, new=1, lo=100, hi=4000, Hkv=32, Hq=32, D=128, bs=16),
        # Four LLaMA-2-70B prompts of ragged lengths, three of them behind a cached prefix.
        dict(name="write_prompts_s4", kind="write", S=4, new=2048, lo=0, hi=1000, Hkv=8, Hq=64, D=128, bs=64),
        # Three LLaMA-3-8B sequences of odd lengths.
        dict(name="read_s3_l1500", kind="read", S=3, new=1, lo=700, hi=1500, Hkv=8, Hq=32, D=128, bs=16),
        # A batch of 32 LLaMA-2-7B sequences moves to another format.
        dict(name="read_s32_l4096", kind="read", S=32, new=1, lo=200, hi=4095, Hkv=32, Hq=32, D=128, bs=32),
        # One LLaMA-3-8B sequence, a short context: launch latency.
        dict(name="decode_s1_l512", kind="attend", S=1, new=1, lo=511, hi=511, Hkv=8, Hq=32, D=128, bs=16,
             window=0, sinks=0),
        # A decode step of 64 LLaMA-2-70B sequences, ragged contexts.
        dict(name="decode_s64_l16384", kind="attend", S=64, new=1, lo=1000, hi=16383, Hkv=8, Hq=64, D=128, bs=64,
             window=0, sinks=0),
        # One LLaMA-2-70B sequence of 131072 tokens: few rows, a long axis.
        dict(name="decode_s1_l131072", kind="attend", S=1, new=1, lo=131071, hi=131071, Hkv=8, Hq=64, D=128, bs=128,
             window=0, sinks=0),
        # Chunks of up to 500 new tokens of three LLaMA-2-70B documents, each token sees 4096 and the first four.
        dict(name="chunk_s3_n500_window", kind="attend", S=3, new=500, lo=3001, hi=12001, Hkv=8, Hq=64, D=128, bs=32,
             window=4096, sinks=4),
        # The largest: a LLaMA-2-70B prompt of 8192 tokens.
        dict(name="prompt_s1_n8192", kind="attend", S=1, new=8192, lo=0, hi=0, Hkv=8, Hq=64, D=128, bs=64,
             window=0, sinks=0),
    ]


_MAX_FLOPS = 4.0 * 128 * 64 * 8192 * 8192 / 2
_MAX_SCORES = 1 << 32     # scores of one plain pass
_MAX_CACHE = 1 << 31      # values of K or of V


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "write", "read", "attend", "attend", "attend", "attend"])
    if kind == "rotary":
        D = rng.choice([64, 128, 128])
        scaling = rng.choice(["none", "none", "linear", "wavelength", "ramp"])
        hi = rng.choice([0, _log_int(rng, 1, 131072)])
        c = dict(kind=kind, S=_log_int(rng, 1, 64), new=_log_int(rng, 1, 8192), lo=hi // 3, hi=hi,
                 H=rng.choice([2, 9, 40, 64, 72, 80]), D=D, rot=rng.choice([D, D, D // 2, D // 4, 20]),
                 interleaved=rng.random() < 0.4, scaling=scaling,
                 factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]))
        c["S"] = max(1, min(c["S"], 8192 * 72 // (c["new"] * c["H"])))
        return c
    Hkv = rng.choice([1, 4, 8, 8, 32, 40])
    g = rng.choice([1, 2, 4, 8]) if Hkv <= 8 else 1
    heads = dict(Hkv=Hkv, Hq=Hkv * g, D=rng.choice([64, 128, 128]), bs=rng.choice([16, 32, 64, 128]))
    while kind in ("write", "read"):
        hi = _log_int(rng, 2, 8000)
        if kind == "read":
            c = dict(kind=kind, S=_log_int(rng, 1, 64), new=1, lo=hi // 4, hi=hi, **heads)
        elif rng.random() < 0.5:
            c = dict(kind=kind, S=_log_int(rng, 1, 128), new=1, lo=hi // 2, hi=hi, **heads)
        else:
            c = dict(kind=kind, S=rng.randint(1, 8), new=_log_int(rng, 2, 2048), lo=0, hi=hi, **heads)
        if c["S"] * (hi + c["new"]) * Hkv * c["D"] <= _MAX_CACHE // 8:
            return c
    window = rng.choice([0, 0, _log_int(rng, 32, 4096)])
    masks = dict(window=window, sinks=rng.choice([0, 1, 4, 64]) if window else 0)
    while True:
        if rng.random() < 0.5:     # decode, or a few speculative tokens
            S, new, hi = _log_int(rng, 1, 128), rng.choice([1, 1, 1, 3]), _log_int(rng, 16, 131072)
            c = dict(kind=kind, S=S, new=new, lo=hi // 3, hi=hi, **heads, **masks)
        else:
            S, new, hi = rng.randint(1, 4), _log_int(rng, 17, 4096), rng.choice([0, 0, _log_int(rng, 16, 32768)])
            c = dict(kind=kind, S=S, new=new, lo=hi // 2, hi=hi, **heads, **masks)
        cells = S * (hi + new)
        if (work(c)["flops"] <= _MAX_FLOPS and cells * Hkv * c["D"] <= _MAX_CACHE and
                cells * new * c["Hq"] <= _MAX_SCORES):
            return c


# ------------------------------------------------------------------------------ shapes
def _spread(case):
    """New tokens and context of each sequence: fixed by the case, spread over its range."""
    S, out = case["S"], []
    for i in range(S):
        f = (i * 0.6180339887498949) % 1.0
        n = case["new"] if i == 0 else max(1, case["new"] - int(f * case["new"] / 2))
        # (from the top of the range downwards; the first sequence is the longest)
        c = case["hi"] - int(round(f * (case["hi"] - case["lo"])))
        # (a read takes every cached token of a sequence)
        out.append((n + c, 0) if case["kind"] == "read" else (n, c))
    return out


def _seen(n, ctx, window, sinks):
    """(pairs of a query and a key it sees, keys that any query sees) of one sequence."""
    pairs = 0
    for p in range(ctx, ctx + n):
        pairs += p + 1 if not window else min(p + 1, window + min(sinks, max(0, p + 1 - window)))
    if not window:
        return pairs, ctx + n
    first = max(0, ctx - window + 1)
    return pairs, ctx + n - first + min(sinks, first)


# Rotary frequencies: base 10000; a training length of 8192 and, for "wavelength", wavelengths that fit it
# 1 to 4 times between scaled and kept, for "ramp" dims between 1 and 32 turns in it.
_BASE, _TRAINED = 10000.0, 8192.0


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "ramp" else 1.0


def _frequencies(case):
    r, s = case["rot"], case["factor"]
    f = [_BASE ** (-2.0 * i / r) for i in range(r // 2)]
    if case["scaling"] == "linear":
        f = [v / s for v in f]
    elif case["scaling"] == "wavelength":
        keep = [min(1.0, max(0.0, (_TRAINED * v / (2 * math.pi) - 1.0) / (4.0 - 1.0))) for v in f]
        f = [v * (k + (1 - k) / s) for v, k in zip(f, keep)]
    elif case["scaling"] == "ramp":
        dim = [r * math.log(_TRAINED / (2 * math.pi * b)) / (2 * math.log(_BASE)) for b in (32.0, 1.0)]
        lo, hi = max(math.floor(dim[0]), 0), min(math.ceil(dim[1]), r - 1)
        far = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001))) for i in range(r // 2)]
        f = [v * (1 - w + w / s) for v, w in zip(f, far)]
    return f


# ------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + 7919 * stream + 1)
    return g


def _half(x):
    return x.clamp_(-65504.0, 65504.0).to(torch.float16)


def _sink(D):
    """A direction that queries share and the keys of the first tokens are strong in."""
    return torch.where(torch.arange(D, device=DEV) % 3 == 0, 1.0, -1.0)


def _quantize(x):
    """Codes, two to a byte, and bfloat16 scales of float32 rows [..., D]."""
    step = torch.tensor(1.0 / 7.0, dtype=torch.float32, device=x.device)
    s = (x.abs().amax(dim=-1) * step).to(torch.bfloat16)
    d = torch.where(s > 0, s.float(), 1.0).unsqueeze(-1)
    c = torch.round(x / d).to(torch.int8)
    return ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8), s


def _values(codes, scales):
    """float32 values [..., D] of codes [..., D / 2] and scales [...]."""
    b = codes.view(torch.int8)
    low = (b << 4) >> 4
    return torch.stack((low, b >> 4), dim=-1).flatten(-2).float().mul_(scales.float().unsqueeze(-1))


def _codes(blocks, H, bs, D, firsts, seed, stream):
    """A filled cache: rows of unit variance with strong channels in each head (and, for keys,
    first tokens in the direction that queries share), quantized row by row."""
    g = _gen(seed, stream)
    codes = torch.empty((blocks, H, bs, D // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((blocks, H, bs), dtype=torch.bfloat16, device=DEV)
    gain = torch.where(torch.rand((H, 1, D), generator=g, device=DEV) < 0.03, 6.0, 1.0)
    step = max(1, (1 << 27) // (H * bs * D))
    for b in range(0, blocks, step):
        n = min(step, blocks - b)
        x = torch.randn((n, H, bs, D), generator=g, device=DEV) * gain
        if firsts is not None:
            x[:, :, :4] += 2.0 * firsts[b:b + n, None, None, None] * _sink(D)
        codes[b:b + n], scales[b:b + n] = _quantize(x)
    return codes, scales


def prepare(case, seed):
    seqs = _spread(case)
    ns, lens = [n for n, _ in seqs], [n + c for n, c in seqs]
    S, T, D = case["S"], sum(ns), case["D"]
    i32 = dict(dtype=torch.int32, device=DEV)
    cu = torch.tensor([sum(ns[:i]) for i in range(S + 1)], **i32)
    st = dict(case=case, cu=cu, lens=torch.tensor(lens, **i32), max_new=max(ns), max_len=max(lens))
    bounds = dict(tokens=T, max_tokens=max(ns), max_len=max(lens))
    g = _gen(seed, 0)
    if case["kind"] == "rotary":
        # q and k as the projection leaves them: the heads of a token, then its values
        H = case["H"]
        rows = _half(torch.randn((T, (H + 2) * D), generator=g, device=DEV))
        st.update(x=rows[:, :H * D].unflatten(1, (H, D)), out=torch.empty((T, H, D), dtype=torch.float16, device=DEV))
        if own:     # the tables and the step's batch that a serving program keeps
            from paper_2606_12487_gb300 import dptq
            st["rotary"] = dptq.Rotary(case["rot"], base=_BASE, interleaved=case["interleaved"], scaling=case["scaling"],
                                       factor=case["factor"], trained_len=_TRAINED, amplitude=_amplitude(case))
            st["batch"] = dptq.Kv8Batch(cu, st["lens"], torch.zeros((S, 1), **i32), **bounds)
        else:
            st["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
        return st
    Hq, Hkv, bs = (case[k] for k in ("Hq", "Hkv", "bs"))
    pages = [-(-n // bs) for n in lens]
    cols, blocks = max(pages), sum(pages) + 1      # (the last page is nobody's)
    order = torch.randperm(blocks - 1, generator=g, device=DEV).to(torch.int32)
    at = torch.tensor([sum(pages[:i]) for i in range(S)], device=DEV)
    col = torch.arange(cols, device=DEV)
    held = col < torch.tensor(pages, device=DEV)[:, None]
    table = torch.where(held, order[(at[:, None] + col).clamp(max=blocks - 2)], -1).to(torch.int32)
    firsts = torch.zeros((blocks,), device=DEV)
    firsts[table[:, 0].long()] = 1.0
    kc, ks = _codes(blocks, Hkv, bs, D, firsts, seed, 1)
    vc, vs = _codes(blocks, Hkv, bs, D, None, seed, 2)
    st.update(k_codes=kc, k_scales=ks, v_codes=vc, v_scales=vs, table=table)
    half = dict(dtype=torch.float16, device=DEV)
    if case["kind"] == "attend":
        q = torch.randn((T, (Hq + 2 * Hkv) * D), generator=g, device=DEV)
        q[:, :Hq * D].view(T, Hq, D).add_(0.25 * _sink(D))
        st.update(q=_half(q)[:, :Hq * D].unflatten(1, (Hq, D)), out=torch.empty((T, Hq, D), **half))
    else:
        st.update(k_out=torch.empty((T, Hkv, D), **half), v_out=torch.empty((T, Hkv, D), **half))
    if case["kind"] == "write":
        kv = _half(torch.randn((T, 2 * Hkv * D), generator=g, device=DEV) * 1.3)
        k, v = kv.split([Hkv * D, Hkv * D], dim=1)
        st.update(k=k.unflatten(1, (Hkv, D)), v=v.unflatten(1, (Hkv, D)))
    if own:     # the handles that a serving program keeps for its cache and for a step's batch
        from paper_2606_12487_gb300 import dptq
        st["cache"] = dptq.Kv4Cache(kc, vc, ks, vs)
        st["batch"] = dptq.Kv8Batch(cu, st["lens"], table, **bounds)
    return st


# ------------------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"rotary": _plain_rotary, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[kind](state)
    from paper_2606_12487_gb300 import dptq
    if kind == "rotary":
        dptq.dptq_rotary(state["rotary"], state["batch"], state["x"], state["out"])
        return state["out"]
    if kind == "attend":
        dptq.dptq_kv4_attention(state["cache"], state["batch"], state["q"], state["out"], 1.0 / math.sqrt(case["D"]),
                                window=case["window"], sinks=case["sinks"])
        return state["out"]
    if kind == "write":
        dptq.dptq_kv4_append(state["cache"], state["batch"], state["k"], state["v"])
    dptq.dptq_kv4_read(state["cache"], state["batch"], state["k_out"], state["v_out"])
    scales = [state["k_scales"], state["v_scales"]] if kind == "write" else []
    return [state["k_out"], state["v_out"]] + scales


def _positions(st, T):
    """Sequence and position of each of the call's rows."""
    t = torch.arange(T, device=DEV)
    seq = torch.searchsorted(st["cu"][1:].contiguous(), t.to(torch.int32), right=True)
    return seq, st["lens"].long()[seq] - st["cu"].long()[seq + 1] + t


def _plain_rotary(st):
    case = st["case"]
    x, r = st["x"], case["rot"]
    _, pos = _positions(st, x.shape[0])
    a = pos.double()[:, None, None] * st["freq"]
    cos, sin = (a.cos() * _amplitude(case)).float(), (a.sin() * _amplitude(case)).float()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    u, v = x[:, :, first].float(), x[:, :, second].float()
    y = x.clone()
    y[:, :, first] = (u * cos - v * sin).half()
    y[:, :, second] = (u * sin + v * cos).half()
    return y


def _plain_write(st):
    bs = st["case"]["bs"]
    seq, pos = _positions(st, st["k"].shape[0])
    blk = st["table"].long()[seq, pos // bs]
    for rows, codes, scales in ((st["k"], st["k_codes"], st["k_scales"]), (st["v"], st["v_codes"], st["v_scales"])):
        codes[blk, :, pos % bs], scales[blk, :, pos % bs] = _quantize(rows.float())
    return _plain_read(st) + [st["k_scales"], st["v_scales"]]


def _plain_read(st):
    bs = st["case"]["bs"]
    seq, pos = _positions(st, st["k_out"].shape[0])
    blk = st["table"].long()[seq, pos // bs]
    return [_values(st[c][blk, :, pos % bs], st[s][blk, :, pos % bs]).half()
            for c, s in (("k_codes", "k_scales"), ("v_codes", "v_scales"))]


def _plain_attend(st):
    """The batch padded to its longest sequence; the query heads of a KV head side by side."""
    case = st["case"]
    Hkv, D, W = case["Hkv"], case["D"], case["window"]
    g, N = case["Hq"] // Hkv, st["max_new"]
    blk = st["table"].long().clamp(min=0)
    S = blk.shape[0]

    def cached(codes, scales):
        x = _values(codes[blk], scales[blk])                                            # [S, pages, H, bs, D]
        return x.permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, D)

    n = (st["cu"][1:] - st["cu"][:-1]).long()
    i = torch.arange(N, device=DEV)
    pos = (st["lens"].long() - n)[:, None] + i                                          # [S, N]
    token = (st["cu"][:-1].long()[:, None] + i).clamp(max=st["q"].shape[0] - 1)
    q = st["q"][token].float().view(S, N, Hkv, g, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, g * N, D)
    k = cached(st["k_codes"], st["k_scales"])
    a = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D))
    del k
    j = torch.arange(a.shape[3], device=DEV)
    seen = j <= pos[:, :, None]
    if W:
        seen = seen & ((j > pos[:, :, None] - W) | (j < case["sinks"]))
    a.view(S, Hkv, g, N, -1).masked_fill_(~seen[:, None, None], -math.inf)
    a.sub_(a.amax(dim=3, keepdim=True)).exp_()
    o = torch.matmul(a, cached(st["v_codes"], st["v_scales"])).div_(a.sum(dim=3, keepdim=True))
    o = o.view(S, Hkv, g, N, D).permute(0, 3, 1, 2, 4).reshape(S * N, Hkv * g, D)
    # the rows of the tokens that there are, in their order
    t = torch.arange(st["q"].shape[0], device=DEV)
    seq = torch.searchsorted(st["cu"][1:].contiguous(), t.to(torch.int32), right=True)
    return o[seq * N + t - st["cu"].long()[seq]].half()


# ------------------------------------------------------------------------------ work
def work(case):
    seqs, D = _spread(case), case["D"]
    T = sum(n for n, _ in seqs)
    if case["kind"] == "rotary":
        return {"bytes": 4 * T * case["H"] * D + 8 * case["rot"] // 2 + 8 * len(seqs),
                "flops": 3.0 * T * case["H"] * case["rot"]}
    H, bs = case["Hkv"], case["bs"]
    if case["kind"] == "read":        # codes and scales in, binary16 out
        return {"bytes": 2 * T * H * (D // 2 + 2 + 2 * D), "flops": 2.0 * T * H * D}
    if case["kind"] == "write":       # binary16 in, codes and scales out, and their values
        return {"bytes": 2 * T * H * (2 * D + D // 2 + 2 + 2 * D), "flops": 8.0 * T * H * D}
    pairs = keys = 0
    for n, c in seqs:
        a, b = _seen(n, c, case["window"], case["sinks"])
        pairs, keys = pairs + a, keys + b
    return {"bytes": 2 * keys * H * (D // 2 + 2) + 4 * (keys // bs + 1) + 4 * T * case["Hq"] * D,
            "flops": 4.0 * pairs * case["Hq"] * D}


# ------------------------------------------------------------------------------ 64-bit results
def exact(case, seed):
    st = prepare(case, seed)
    seqs, D = _spread(case), case["D"]
    cu = st["cu"].tolist()
    if case["kind"] == "rotary":
        # pairs as complex numbers, each turned by the power of its frequency's unit number
        x, r, H = st["x"].double(), case["rot"], case["H"]
        out = x.clone()
        pairs = (H, r // 2, 2) if case["interleaved"] else (H, 2, r // 2)
        for b, (n, c) in enumerate(seqs):
            z = x[cu[b]:cu[b] + n, :, :r].reshape(n, *pairs)
            z = z if case["interleaved"] else z.transpose(2, 3)
            z = torch.complex(z[..., 0].contiguous(), z[..., 1].contiguous())
            f = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
            angle = torch.arange(c, c + n, device=DEV, dtype=torch.float64)[:, None, None] * f
            z = torch.view_as_real(z * torch.polar(torch.full_like(angle, _amplitude(case)), angle))
            z = z if case["interleaved"] else z.transpose(2, 3)
            out[cu[b]:cu[b] + n, :, :r] = z.reshape(n, H, r)
        return out
    bs, H = case["bs"], case["Hkv"]
    table = st["table"].cpu()
    if case["kind"] == "read":
        res = []
        for codes, scales in ((st["k_codes"], st["k_scales"]), (st["v_codes"], st["v_scales"])):
            rows = []
            for b, (n, _) in enumerate(seqs):
                blk = table[b, :-(-n // bs)].long().to(DEV)
                byte = codes[blk].transpose(1, 2).flatten(0, 1)[:n].to(torch.int16)
                c = torch.stack((byte % 16, byte // 16), dim=3).flatten(2).double()
                rows.append(torch.where(c > 7, c - 16, c) * scales[blk].transpose(1, 2).flatten(0, 1)[:n, :, None].double())
            res.append(torch.cat(rows))
        return res
    if case["kind"] == "write":
        # (codes are whole numbers, and so what they stand for has no 64-bit value of its own)
        res = []
        for rows, scales in ((st["k"], st["k_scales"]), (st["v"], st["v_scales"])):
            s = scales.double()
            for b, (n, c) in enumerate(seqs):
                pos = torch.arange(c, c + n)
                blk = table[b, pos // bs].long().to(DEV)
                s[blk, :, (pos % bs).to(DEV)] = rows[cu[b]:cu[b] + n].double().abs().amax(dim=2) / 7.0
            res.append(s)
        return [None, None] + res
    g, W = case["Hq"] // H, case["window"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, c) in enumerate(seqs):
        L = c + n
        blk = table[b, :-(-L // bs)].long().to(DEV)
        rows = max(1, (1 << 27) // L)
        for h in range(H):
            kv = []
            for codes, scales in ((st["k_codes"], st["k_scales"]), (st["v_codes"], st["v_scales"])):
                byte = codes[blk, h].reshape(-1, D // 2)[:L].to(torch.int16)
                code = torch.stack((byte % 16, byte // 16), dim=2).flatten(1).double()
                kv.append(torch.where(code > 7, code - 16, code) * scales[blk, h].reshape(-1)[:L, None].double())
            for e in range(h * g, (h + 1) * g):
                for at in range(0, n, rows):
                    q = st["q"][cu[b] + at:cu[b] + min(n, at + rows), e].double()
                    pos = c + at + torch.arange(q.shape[0], device=DEV)[:, None]
                    j = torch.arange(L, device=DEV)[None, :]
                    hide = j > pos
                    if W:
                        hide = hide | ((j <= pos - W) & (j >= case["sinks"]))
                    logit = (q @ kv[0].t() / math.sqrt(D)).masked_fill(hide, -math.inf)
                    out[cu[b] + at:cu[b] + at + q.shape[0], e] = torch.softmax(logit, dim=1) @ kv[1]
    return out
