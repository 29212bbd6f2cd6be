"""What the operators around the quantized linear layer are timed on.

A case is a dict of plain values.  `kind` names the operator:

  norm    residual addition, RMS norm and per-token int8 quantization in one call
          (dptq_add_rmsnorm_quant), what q|k|v and gate|up read
  append  new K and V rows into a paged cache of int8 codes with a scale for each page and
          head (dptq_kv8_append)
  attend  causal attention over that cache, for single tokens and for prompts, with an
          optional sliding window and first tokens that stay visible (dptq_kv8_attention)

Head counts, widths and token counts are those of the LLaMA geometries in
paper_2606_12487_gb300/inputs.py (7B: 32 heads of 128; LLaMA-3-8B: 32 over 8; 70B: 64 over 8).

`own` false: the plain form, elementary operations in 32 bits.  True: the library's calls.
The codes are whole numbers and the same on both sides: every step of the quantizers is
defined in 32 bits.  They are returned as they are, beside their scales.
"""
import math

import torch

own = False
DEV = "cuda"
EPS = 1e-5


def listed():
    return [
        # One token of LLaMA-2-7B: launch latency.
        dict(name="norm_m1_k4096", kind="norm", M=1, K=4096, res=True, gamma=True),
        # A decode step of LLaMA-2-70B at 64 sequences.
        dict(name="norm_m64_k8192", kind="norm", M=64, K=8192, res=True, gamma=True),
        # A prompt of odd length, LLaMA-2-13B, the norm's weight folded into the projections.
        dict(name="norm_m1333_k5120", kind="norm", M=1333, K=5120, res=True, gamma=False),
        # LLaMA-2-70B, four sequences of 2048 tokens.
        dict(name="norm_m8192_k8192", kind="norm", M=8192, K=8192, res=True, gamma=True),
        # One new token of each of 32 LLaMA-2-7B sequences.
        dict(name="append_step_s32", kind="append", S=32, new=1, lo=100, hi=4000, Hq=32, Hkv=32, D=128, bs=16),
        # Four LLaMA-2-70B prompts of ragged lengths, three of them behind a cached prefix.
        dict(name="append_prompts_s4", kind="append", S=4, new=2048, lo=0, hi=1000, Hq=64, Hkv=8, D=128, bs=64),
        # One LLaMA-3-8B sequence, a short context: launch latency.
        dict(name="decode_s1_l512", kind="attend", S=1, new=1, lo=511, hi=511, Hq=32, Hkv=8, D=128, bs=16,
             window=0, sinks=0),
        # A decode step of 32 LLaMA-2-7B sequences (a KV head for each query head), ragged contexts.
        dict(name="decode_s32_mha", kind="attend", S=32, new=1, lo=200, hi=4095, Hq=32, Hkv=32, D=128, bs=32,
             window=0, sinks=0),
        # 64 LLaMA-2-70B sequences, each token sees 4096 tokens and the first four.
        dict(name="decode_s64_window", kind="attend", S=64, new=1, lo=1000, hi=16383, Hq=64, Hkv=8, D=128, bs=64,
             window=4096, sinks=4),
        # One LLaMA-2-70B sequence of 131072 tokens: few rows, a long axis.
        dict(name="decode_s1_l131072", kind="attend", S=1, new=1, lo=131071, hi=131071, Hq=64, Hkv=8, D=128, bs=128,
             window=0, sinks=0),
        # Three LLaMA-3-8B prompts of odd lengths up to 2048.
        dict(name="prompt_s3_n2048", kind="attend", S=3, new=2048, lo=0, hi=0, Hq=32, Hkv=8, D=128, bs=16,
             window=0, sinks=0),
        # The largest: a LLaMA-2-70B prompt of 8192 tokens.
        dict(name="prompt_s1_n8192", kind="attend", S=1, new=8192, lo=0, hi=0, Hq=64, Hkv=8, D=128, bs=64,
             window=0, sinks=0),
    ]


_MAX_FLOPS = 4.0 * 128 * 64 * 8192 * 8192 / 2
_MAX_SCORES = 1 << 32     # scores of one plain pass
_MAX_CACHE = 1 << 31      # codes of K or of V


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append", "attend", "attend", "attend"])
    if kind == "norm":
        return dict(kind=kind, M=_log_int(rng, 1, 8192), K=rng.choice([1024, 2080, 4096, 5120, 8192]),
                    res=rng.random() < 0.8, gamma=rng.random() < 0.7)
    Hkv = rng.choice([1, 4, 8, 8, 32, 40])
    g = rng.choice([1, 2, 4, 8]) if Hkv <= 8 else 1
    heads = dict(Hq=Hkv * g, Hkv=Hkv, D=rng.choice([64, 128, 128]), bs=rng.choice([16, 32, 64, 128]))
    while kind == "append":
        hi = _log_int(rng, 2, 8000)
        if rng.random() < 0.5:
            c = dict(kind=kind, S=_log_int(rng, 1, 128), new=1, lo=hi // 2, hi=hi, **heads)
        else:
            c = dict(kind=kind, S=rng.randint(1, 8), new=_log_int(rng, 2, 2048), lo=0, hi=hi, **heads)
        if c["S"] * (hi + c["new"]) * Hkv * c["D"] <= _MAX_CACHE // 8:
            return c
    window = rng.choice([0, 0, _log_int(rng, 32, 4096)])
    masks = dict(window=window, sinks=rng.choice([0, 1, 4, 64]) if window else 0)
    while True:
        if rng.random() < 0.6:     # decode, or a few speculative tokens
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
        out.append((n, case["hi"] - int(round(f * (case["hi"] - case["lo"])))))
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


def _codes(blocks, H, bs, D, firsts, seed, stream):
    """A filled cache: rows of unit variance with strong channels in each head (and, for keys,
    first tokens in the direction that queries share), quantized page by page."""
    g = _gen(seed, stream)
    codes = torch.empty((blocks, H, bs, D), dtype=torch.int8, device=DEV)
    scales = torch.empty((blocks, H), dtype=torch.float32, device=DEV)
    gain = torch.where(torch.rand((H, 1, D), generator=g, device=DEV) < 0.03, 6.0, 1.0)
    step = max(1, (1 << 27) // (H * bs * D))
    for b in range(0, blocks, step):
        n = min(step, blocks - b)
        x = torch.randn((n, H, bs, D), generator=g, device=DEV) * gain
        if firsts is not None:
            x[:, :, :4] += 2.0 * firsts[b:b + n, None, None, None] * _sink(D)
        s = x.abs().amax(dim=(2, 3)) / 127.0
        codes[b:b + n] = torch.round(x / s[:, :, None, None]).to(torch.int8)
        scales[b:b + n] = s
    return codes, scales


def prepare(case, seed):
    if case["kind"] == "norm":
        M, K = case["M"], case["K"]
        g = _gen(seed, 0)
        x = torch.randn((M, K), generator=g, device=DEV)
        r = torch.randn((M, K), generator=g, device=DEV) * 2.0
        r[:, torch.randperm(K, generator=g, device=DEV)[:4]] *= 40.0        # massive activations
        st = dict(case=case, x=_half(x), residual=_half(r) if case["res"] else None, gamma=None,
                  codes=torch.empty((M, K), dtype=torch.int8, device=DEV),
                  scales=torch.empty((M,), dtype=torch.float32, device=DEV),
                  residual_out=torch.empty((M, K), dtype=torch.float16, device=DEV) if case["res"] else None)
        if case["gamma"]:
            st["gamma"] = _half(1.0 + 0.2 * torch.randn((K,), generator=g, device=DEV))
        return st
    S, Hq, Hkv, D, bs = (case[k] for k in ("S", "Hq", "Hkv", "D", "bs"))
    seqs = _spread(case)
    ns, lens = [n for n, _ in seqs], [n + c for n, c in seqs]
    pages = [-(-l // bs) for l in lens]
    T, cols, blocks = sum(ns), max(pages), sum(pages) + 1      # (the last page is nobody's)
    g = _gen(seed, 0)
    order = torch.randperm(blocks - 1, generator=g, device=DEV).to(torch.int32)
    at = torch.tensor([sum(pages[:i]) for i in range(S)], device=DEV)
    col = torch.arange(cols, device=DEV)
    held = col < torch.tensor(pages, device=DEV)[:, None]
    table = torch.where(held, order[(at[:, None] + col).clamp(max=blocks - 2)], -1).to(torch.int32)
    firsts = torch.zeros((blocks,), device=DEV)
    firsts[table[:, 0].long()] = 1.0
    kc, ks = _codes(blocks, Hkv, bs, D, firsts, seed, 1)
    vc, vs = _codes(blocks, Hkv, bs, D, None, seed, 2)
    # q, k and v of the new tokens as the projection leaves them: one row for each token
    qkv = torch.randn((T, (Hq + 2 * Hkv) * D), generator=g, device=DEV)
    q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], dim=1)
    q.view(T, Hq, D).add_(0.25 * _sink(D))
    k.mul_(1.3)
    qkv = _half(qkv)
    q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], dim=1)
    cu = torch.tensor([sum(ns[:i]) for i in range(S + 1)], dtype=torch.int32, device=DEV)
    st = dict(case=case, k_codes=kc, k_scales=ks, v_codes=vc, v_scales=vs, cu=cu, table=table,
              lens=torch.tensor(lens, dtype=torch.int32, device=DEV), max_new=max(ns), max_len=max(lens),
              q=q.unflatten(1, (Hq, D)), k=k.unflatten(1, (Hkv, D)), v=v.unflatten(1, (Hkv, D)),
              out=torch.empty((T, Hq, D), dtype=torch.float16, device=DEV))
    if own:     # the handles that a serving program keeps for its cache and for a step's batch
        from paper_2606_12487_gb300 import dptq
        st["cache"] = dptq.Kv8Cache(kc, vc, ks, vs)
        st["batch"] = dptq.Kv8Batch(cu, st["lens"], table, tokens=T, max_tokens=max(ns), max_len=max(lens))
    return st


# ------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2606_12487_gb300 import dptq
        if kind == "norm":
            dptq.dptq_add_rmsnorm_quant(state["x"], state["residual"], state["gamma"], EPS, 8, state["residual_out"],
                                        state["codes"], state["scales"])
            return [state["residual_out"], state["codes"], state["scales"]]
        if kind == "append":
            dptq.dptq_kv8_append(state["cache"], state["batch"], state["k"], state["v"])
            return [state["k_codes"], state["k_scales"], state["v_codes"], state["v_scales"]]
        case = state["case"]
        dptq.dptq_kv8_attention(state["cache"], state["batch"], state["q"], state["out"],
                                1.0 / math.sqrt(case["D"]), window=case["window"], sinks=case["sinks"])
        return state["out"]
    return {"norm": _plain_norm, "append": _plain_append, "attend": _plain_attend}[kind](state)


def _plain_norm(st):
    h = st["x"].float()
    if st["residual"] is not None:
        h = (h + st["residual"].float()).half()
        out, h = h, h.float()
    else:
        out = None
    p = h if st["gamma"] is None else h * st["gamma"].float()
    s = p.abs().amax(dim=1, keepdim=True) / 127.0
    c = torch.round(p / torch.where(s > 0, s, 1.0)).to(torch.int8)
    rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + EPS)
    return [out, c, s.squeeze(1) * rstd]


def _plain_append(st):
    """All pages that new tokens fall into, [S, pages of a sequence, page], at once."""
    case = st["case"]
    bs = case["bs"]
    n = (st["cu"][1:] - st["cu"][:-1]).long()
    start = st["lens"].long() - n
    per = (st["max_new"] + bs - 2) // bs + 1
    page = (start // bs)[:, None] + torch.arange(per, device=DEV)                       # [S, per]
    i = (page * bs)[:, :, None] + torch.arange(bs, device=DEV) - start[:, None, None]   # token of the call
    new = (i >= 0) & (i < n[:, None, None])
    old = i < 0
    touched = new.any(dim=2)
    cols = st["table"].shape[1]
    blk = torch.gather(st["table"].long(), 1, page.clamp(max=cols - 1))
    blk = torch.where(touched, blk, st["k_codes"].shape[0] - 1)
    token = (st["cu"][:-1].long()[:, None, None] + i).clamp(0, st["k"].shape[0] - 1)
    earlier = (old.any(dim=2) & touched)[:, :, None]
    new, old, keep = new[:, :, None, :, None], old[:, :, None, :, None], touched[:, :, None, None, None]
    for rows, codes, scales in ((st["k"], st["k_codes"], st["k_scales"]), (st["v"], st["v_codes"], st["v_scales"])):
        x = rows[token].permute(0, 1, 3, 2, 4).float()                                  # [S, per, H, bs, D]
        x = torch.where(new, x, 0.0)
        c0, s_held = codes[blk], scales[blk]
        s0 = torch.where(earlier, s_held, 0.0)
        s1 = torch.maximum(s0, x.abs().amax(dim=(3, 4)) / 127.0)
        d = torch.where(s1 > 0, s1, 1.0)[:, :, :, None, None]
        c1 = torch.where(new, torch.round(x / d),
                         torch.where(old, torch.round(c0.float() * s0[:, :, :, None, None] / d), c0.float()))
        codes[blk] = torch.where(keep, c1.to(torch.int8), c0)
        scales[blk] = torch.where(touched[:, :, None], s1, s_held)
    return [st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"]]


def _plain_attend(st):
    """The batch padded to its longest sequence; the query heads of a KV head side by side."""
    case = st["case"]
    Hkv, D, W = case["Hkv"], case["D"], case["window"]
    g, N = case["Hq"] // Hkv, st["max_new"]
    blk = st["table"].long().clamp(min=0)
    S = blk.shape[0]

    def cached(codes, scales):
        x = codes[blk].float().mul_(scales[blk][:, :, :, None, None])                   # [S, pages, H, bs, D]
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
    if case["kind"] == "norm":
        n, M, K = case["M"] * case["K"], case["M"], case["K"]
        return {"bytes": 2 * n + (4 * n if case["res"] else 0) + n + 4 * M + (2 * K if case["gamma"] else 0),
                "flops": 8.0 * n}
    seqs, H, D, bs = _spread(case), case["Hkv"], case["D"], case["bs"]
    T = sum(n for n, _ in seqs)
    if case["kind"] == "append":
        pages = sum((n + c + bs - 1) // bs - c // bs for n, c in seqs)
        return {"bytes": 2 * (3 * T * H * D + 8 * pages * H), "flops": 6.0 * T * H * D}
    pairs = keys = 0
    for n, c in seqs:
        a, b = _seen(n, c, case["window"], case["sinks"])
        pairs, keys = pairs + a, keys + b
    return {"bytes": 2 * keys * H * D + 8 * H * (keys // bs + 1) + 4 * T * case["Hq"] * D,
            "flops": 4.0 * pairs * case["Hq"] * D}


# ------------------------------------------------------------------------------ 64-bit results
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "norm":
        h = st["x"].double()
        out = None
        if case["res"]:
            h = h + st["residual"].double()
            out = h.half().double()
            h, exact_out = out, h
        p = h * st["gamma"].double() if case["gamma"] else h
        rms = (h.square().mean(dim=1) + EPS).sqrt()
        # (the codes are whole numbers: no 64-bit value)
        return [exact_out if case["res"] else None, None, p.abs().amax(dim=1) / 127.0 / rms]
    seqs, bs, D, H = _spread(case), case["bs"], case["D"], case["Hkv"]
    table = st["table"].cpu()
    cu = st["cu"].tolist()
    if case["kind"] == "append":
        # page by page: the scale that covers the earlier rows' codes and the new rows
        res = []
        for rows, scales in ((st["k"], st["k_scales"]), (st["v"], st["v_scales"])):
            s = scales.double()
            for b, (n, c) in enumerate(seqs):
                for page in range(c // bs, (c + n - 1) // bs + 1):
                    lo, hi = max(c, page * bs), min(c + n, (page + 1) * bs)
                    blk = int(table[b, page])
                    top = rows[cu[b] + lo - c:cu[b] + hi - c].double().abs().amax(dim=(0, 2)) / 127.0
                    s[blk] = torch.maximum(s[blk], top) if lo > page * bs else top
            res += [None, s]
        return res
    g, W = case["Hq"] // H, case["window"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n, c) in enumerate(seqs):
        L = c + n
        blk = table[b, :-(-L // bs)].long().to(DEV)
        rows = max(1, (1 << 27) // L)
        for h in range(H):
            kv = [(codes[blk, h].double() * scales[blk, h].double()[:, None, None]).reshape(-1, D)[:L]
                  for codes, scales in ((st["k_codes"], st["k_scales"]), (st["v_codes"], st["v_scales"]))]
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
