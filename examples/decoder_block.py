"""A stack of blocks around the STEM layer, trained for some steps and then served in 8-bit integers.

    n = N(x)                            stem_block_enter_forward   (in front of the first block)
    f = layer(n, ids)                   stem_ffn_forward
    x = x + scale * drop(N(f) w)        stem_block_leave_forward, which also gives the next block's n

Attention is left out: the layer's own path is what is shown.  Run from the repository's root on an MI355X:

    python -m examples.decoder_block
"""
from __future__ import annotations

import torch

from paper_2601_10639_amd import inputs, stemlib as L

DEV, EPS = "cuda:0", 1e-5


class Stack:
    def __init__(self, blocks=2, d=256, F=1024, V=1000, T=512, p=0.1, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        bf = torch.bfloat16

        def normal(*shape, std):
            return torch.empty(*shape, device=DEV).normal_(0.0, std, generator=gen).to(bf)

        self.d, self.F, self.V, self.T = d, F, V, T
        self.embed = normal(V, d, std=1.0)
        self.blocks, self.step = [], torch.zeros(1, dtype=torch.int64, device=DEV)   # counts on: another dropout mask each step
        for k in range(blocks):
            b = dict(Wg=normal(F, d, std=d ** -0.5), Wd=normal(d, F, std=F ** -0.5), E=normal(V, F, std=1.0),
                     w_out=torch.ones(d, device=DEV, dtype=bf), w_in=torch.ones(d, device=DEV, dtype=bf), scale=torch.full((d,), 0.5, device=DEV, dtype=bf))
            b["ctx"] = L.stem_create(d, F, V, L.STEM_BF16, T, reserve=L.STEM_RESERVE_QUANT)
            b.update(master=b["E"].float(), m=torch.zeros(V, F, device=DEV), v=torch.zeros(V, F, device=DEV))
            self.blocks.append(b)
        for k, b in enumerate(self.blocks):   # a block's end brings the next one's norm along
            nxt = self.blocks[k + 1]["w_in"] if k + 1 < blocks else None
            b["norm"] = L.stem_norm(L.STEM_NORM_RMS, EPS, b["w_in"])
            b["leave"] = [L.stem_leave(out=L.stem_norm(L.STEM_NORM_RMS, EPS, b["w_out"]), next=L.stem_norm(L.STEM_NORM_RMS, EPS, nxt) if nxt is not None else None,
                                       gate_kind=L.STEM_GATE_CHANNEL, gate=b["scale"], p=q, seed=17 + k, step=self.step) for q in (p, 0.0)]

    def forward(self, ids, train):
        """The last residual stream and what the backward pass needs."""
        x = self.embed[ids.long()]
        n, saved = torch.empty_like(x), []
        L.stem_block_enter_forward(self.blocks[0]["ctx"], x, self.blocks[0]["norm"], n)
        for k, b in enumerate(self.blocks):
            G, H = (torch.empty(len(ids), self.F, dtype=x.dtype, device=DEV) for _ in range(2))
            f, y, after = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x) if k + 1 < len(self.blocks) else None
            L.stem_ffn_forward(b["ctx"], n, ids, b["Wg"], b["Wd"], b["E"], f, save_G=G, save_H=H)
            L.stem_block_leave_forward(b["ctx"], f, x, b["leave"][not train], y, after)
            saved.append((x, n, G, H, f, y))
            x, n = y, after
        return x, saved

    def train_step(self, ids, target, lr=0.05):
        """One step on mean (x - target)^2; the loss before it."""
        self.step.add_(1)
        x, saved = self.forward(ids, True)
        diff = x.float() - target
        loss = diff.square().mean()
        dy, dn = (diff * (2.0 / self.d)).to(x.dtype), None
        for k in reversed(range(len(self.blocks))):
            b, (x0, n, G, H, f, y) = self.blocks[k], saved[k]
            ctx, T, d, F = b["ctx"], len(ids), self.d, self.F
            f32 = dict(device=DEV, dtype=torch.float32)
            dx, df, dlayer, dU = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(G)
            dscale, dw_out, dw_next = torch.empty(d, **f32), torch.empty(d, **f32), torch.empty(d, **f32) if dn is not None else None
            L.stem_block_leave_backward(ctx, dy, dn, f, y, b["leave"][0], dx, df, dscale, dw_out, dw_next)
            dWg, dWd = torch.empty(F, d, **f32), torch.empty(d, F, **f32)
            L.stem_ffn_backward(ctx, df, n, ids, b["Wg"], b["Wd"], b["E"], G, H, dlayer, dWg, dWd, dU)
            i32 = dict(device=DEV, dtype=torch.int32)
            uniq, count, rows = torch.empty(T, **i32), torch.empty(1, **i32), torch.empty(min(T, self.V), F, **f32)
            L.stem_embed_grad(ctx, ids, dU, torch.empty(T, **i32), torch.empty(T, **i32), uniq, torch.empty(T + 1, **i32), count, rows)
            L.stem_embed_sparse_adamw(ctx, uniq, count, rows, b["E"], b["master"], b["m"], b["v"], 1e-2, 0.9, 0.95, 1e-8, 0.0, int(self.step))
            grads = [(b["Wg"], dWg), (b["Wd"], dWd), (b["scale"], dscale), (b["w_out"], dw_out)]
            if dn is not None:
                grads.append((self.blocks[k + 1]["w_in"], dw_next))
            for w, g in grads:
                w.sub_((lr / T * g).to(w.dtype))
            dy, dn = dx, dlayer
        dx, dw = torch.empty_like(x), torch.empty(self.d, device=DEV)
        b = self.blocks[0]
        L.stem_block_enter_backward(b["ctx"], dn, saved[0][0], b["norm"], dx, dw, dres=dy)
        b["w_in"].sub_((lr / len(ids) * dw).to(b["w_in"].dtype))
        return float(loss)

    def quantise(self):
        for b in self.blocks:
            b["q"] = (L.stem_quant_weights(b["ctx"], b["Wg"]), L.stem_quant_weights(b["ctx"], b["Wd"]))

    def serve(self, ids):
        """The same stack for inference on 8-bit weights: the norm in front is part of the layer's call, the norm behind it of the block's end."""
        x = self.embed[ids.long()]
        f = torch.empty_like(x)
        for b in self.blocks:
            L.stem_quant_ffn_forward(b["ctx"], x, ids, *b["q"], b["E"], f, norm=b["norm"])
            end = L.stem_leave(out=b["leave"][1].norms[0], gate_kind=L.STEM_GATE_CHANNEL, gate=b["scale"])
            L.stem_block_leave_forward(b["ctx"], f, x, end, x)
        return x


def main(steps=30):
    stack = Stack()
    ids = torch.from_numpy(inputs.zipf_ids(stack.T, stack.V, seed=1)).to(torch.int32).to(DEV)
    target = torch.randn(stack.V, stack.d, generator=torch.Generator().manual_seed(2)).to(DEV)[ids.long()]   # a row to learn for each token id
    losses = [stack.train_step(ids, target) for _ in range(steps)]
    stack.quantise()
    x, _ = stack.forward(ids, False)
    apart = []
    for T in (1, 16, len(ids)):
        y = stack.serve(ids[:T])
        apart.append(float((y.float() - x[:T].float()).norm() / x[:T].float().norm()))
    return losses, apart


if __name__ == "__main__":
    losses, apart = main()
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    print("served in 8 bits, relative distance from bf16 at 1, 16 and all tokens:", " ".join(f"{a:.4f}" for a in apart))
