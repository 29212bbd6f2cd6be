"""A small LLaMA-shaped decoder on the library: prompts, then single tokens, for a ragged batch.

    python examples/decoder_layers.py

Each layer runs, in order (d the width, random weights):

  dptq_add_rmsnorm_quant   residual addition, RMS norm, codes       -> q|k|v (dptq_qgemm_codes)
  (rotary embedding, plain torch)
  dptq_kv8_append          the new k and v into the int8 paged cache
  dptq_kv8_attention       over it, causal, with a window and sinks if asked for
  dptq_qlinear             o, behind the online Hadamard rotation
  dptq_add_rmsnorm_quant                                            -> gate|up (dptq_qgemm_codes)
  (SwiGLU, plain torch)
  dptq_qlinear             down, behind the online rotation

The projections that read the residual stream are packed with had_block = 1 (their rotation is
folded into the stream offline, Section 2 Eq. 5); layers of the mask run 8-bit activations.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_12487_gb300 import dptq  # noqa: E402

EPS = 1e-5


class Decoder:
    def __init__(self, layers=4, d=1024, heads=16, kv_heads=4, f=2816, mask_a8=(0, 1, 3), pages=256, page=16,
                 had_block=256, window=0, sinks=0, seed=0):
        self.d, self.heads, self.kv, self.dim, self.f = d, heads, kv_heads, d // heads, f
        self.page, self.window, self.sinks = page, window, sinks
        self.bits = [8 if i in mask_a8 else 4 for i in range(layers)]
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(n, k):
            return (torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)).half()

        def gamma():
            return (1 + 0.1 * torch.randn((d,), generator=g, device="cuda")).half()

        n_qkv = (heads + 2 * kv_heads) * self.dim
        self.layers = [dict(qkv=dptq.dptq_pack_weights(w(n_qkv, d), 1), o=dptq.dptq_pack_weights(w(d, d), had_block),
                            up=dptq.dptq_pack_weights(w(2 * f, d), 1), down=dptq.dptq_pack_weights(w(d, f), had_block),
                            g1=gamma(), g2=gamma(), cache=dptq.Kv8Cache.empty(pages, kv_heads, page, self.dim))
                       for _ in range(layers)]
        self.free = list(range(pages))
        self.tables, self.lens = {}, {}

    def batch(self, new):
        """The batch of a step that gives sequence s new[s] tokens: pages are handed out here."""
        cu, lens = [0], []
        for s, n in new.items():
            self.lens[s] = self.lens.get(s, 0) + n
            table = self.tables.setdefault(s, [])
            while len(table) * self.page < self.lens[s]:
                table.append(self.free.pop())
            cu.append(cu[-1] + n)
            lens.append(self.lens[s])
        cols = max(len(self.tables[s]) for s in new)
        table = [self.tables[s] + [-1] * (cols - len(self.tables[s])) for s in new]
        i32 = dict(dtype=torch.int32, device="cuda")
        pos = torch.cat([torch.arange(self.lens[s] - n, self.lens[s]) for s, n in new.items()])
        return dptq.Kv8Batch(torch.tensor(cu, **i32), torch.tensor(lens, **i32), torch.tensor(table, **i32),
                             tokens=cu[-1], max_tokens=max(new.values()), max_len=max(lens)), pos.cuda()

    def rotary(self, x, pos):
        half = self.dim // 2
        a = pos[:, None, None] * 10000.0 ** (-torch.arange(half, device="cuda") / half)
        u, v = x[..., :half].float(), x[..., half:].float()
        x.copy_(torch.cat([u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()], dim=-1))

    def step(self, x, new):
        """Hidden states float16 [tokens, d] of the new tokens of the sequences in `new` (a dict of
        counts) through all layers; returns the residual stream after the last one."""
        batch, pos = self.batch(new)
        T, half = x.shape[0], dict(dtype=torch.float16, device="cuda")
        h, update = torch.zeros_like(x), x
        scales, att = torch.empty((T,), device="cuda"), torch.empty((T, self.heads, self.dim), **half)
        for layer, bits in zip(self.layers, self.bits):
            codes = torch.empty((T, self.d if bits == 8 else self.d // 2), device="cuda",
                                dtype=torch.int8 if bits == 8 else torch.uint8)
            qkv, proj = torch.empty((T, layer["qkv"].N), **half), torch.empty((T, self.d), **half)
            up, down = torch.empty((T, 2 * self.f), **half), torch.empty((T, self.d), **half)
            dptq.dptq_add_rmsnorm_quant(update, h, layer["g1"], EPS, bits, h, codes, scales)
            dptq.dptq_qgemm_codes(layer["qkv"], codes, scales, bits, qkv)
            rows = qkv.unflatten(1, (self.heads + 2 * self.kv, self.dim))
            q, k, v = rows.split([self.heads, self.kv, self.kv], dim=1)
            self.rotary(q, pos)
            self.rotary(k, pos)
            dptq.dptq_kv8_append(layer["cache"], batch, k, v)
            dptq.dptq_kv8_attention(layer["cache"], batch, q, att, 1 / math.sqrt(self.dim), self.window, self.sinks)
            dptq.dptq_qlinear(layer["o"], att.flatten(1), bits, proj)
            dptq.dptq_add_rmsnorm_quant(proj, h, layer["g2"], EPS, bits, h, codes, scales)
            dptq.dptq_qgemm_codes(layer["up"], codes, scales, bits, up)
            gate, value = up.split(self.f, dim=1)
            dptq.dptq_qlinear(layer["down"], (torch.nn.functional.silu(gate) * value).contiguous(), bits, down)
            update = down
        return h + update


def main():
    model = Decoder()
    g = torch.Generator(device="cuda").manual_seed(1)
    new = {0: 37, 1: 120, 2: 5}
    y = model.step(torch.randn((sum(new.values()), model.d), generator=g, device="cuda").half(), new)
    print("prompt: %d tokens of %d sequences, |h| %.3f" % (y.shape[0], len(new), y.float().norm(dim=1).mean()))
    steps = 32
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for i in range(steps):
        if i == 2:
            ev[0].record()
        y = model.step(torch.randn((3, model.d), generator=g, device="cuda").half(), {0: 1, 1: 1, 2: 1})
    ev[1].record()
    torch.cuda.synchronize()
    dptq.dptq_last_device_error()
    print("decode: %d steps, lengths %s, %.0f us a step, |h| %.3f"
          % (steps, list(model.lens.values()), ev[0].elapsed_time(ev[1]) * 1e3 / (steps - 2), y.float().norm(dim=1).mean()))


if __name__ == "__main__":
    main()
