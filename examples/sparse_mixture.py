"""A mixture of sparse networks, served and trained: every token's row goes through a few of several networks.

    x      = embed(table, ids)                          rows by token id
    chosen = route(x @ router)                          the networks of each row, and their weights
    xs     = dispatch(x, chosen)                        rows sorted by network
    ys     = network_e(xs) + gain_e * xs                each network on its own batch, with a learned skip around it
    out    = x + combine(ys)                            back to the tokens' order, weighted, onto the residual

The networks are pruned ones that stay as they are; table, router and gains are learned.  Run it on a GPU:

    python examples/sparse_mixture.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2007_14152_amd as sp  # noqa: E402
import synth  # noqa: E402


class Mixture:
    """`experts` sparse networks of N neurons and L layers behind a router that picks k of them."""

    def __init__(self, vocab, N=1024, L=4, experts=8, k=2, seed=1, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.N, self.experts, self.k = N, experts, k
        bias = np.full(N, -0.05, dtype=np.float32)
        self.nets = []
        for e in range(experts):
            idx = [synth.gen_layer(N, l, seed * 1000 + e) for l in range(L)]
            val = [synth.gen_values(N) for _ in range(L)]
            self.nets.append(sp.Model(idx, val, bias, device=device))
        self.table = torch.rand(vocab, N, generator=g, device=device) * 0.1
        self.router = torch.randn(N, experts, generator=g, device=device) * 0.05
        self.gain = torch.randn(experts, N, generator=g, device=device) * 0.1

    def _networks(self, xs, offsets):
        """Every network on its batch; rows that a network prunes are zero."""
        ys = torch.zeros_like(xs)
        for e, net in enumerate(self.nets):
            first, last = offsets[e], offsets[e + 1]
            if first < last:
                n, rows, Y = net.infer(xs[first:last])
                ys[first + rows[:n].long()] = Y
        return ys

    def forward(self, ids):
        """(out [n, N], what a gradient step needs)."""
        x = sp.embed(self.table, ids)
        logits = x @ self.router
        chosen, weight = sp.route(logits, self.k, keep=ids >= 0)
        xs, offsets, place = sp.dispatch(x, chosen, self.experts)
        at = offsets.tolist()
        expert = torch.repeat_interleave(torch.arange(self.experts, device=x.device), torch.diff(offsets).long())
        skip = self.gain[expert]  # a row per pair; the pairs without an expert stand behind them
        ys = self._networks(xs, at)
        ys[:at[-1]] += skip * xs[:at[-1]]
        out = sp.combine(ys, place, weight=weight, add=x)
        return out, (ids, x, logits, chosen, weight, xs, offsets, place, ys, expert, skip)

    def gradients(self, dout, saved):
        """Of table, router and gain, for the gradient dout of the output; the networks' outputs are taken as given."""
        ids, x, logits, chosen, weight, xs, offsets, place, ys, expert, skip = saved
        dys, dweight = sp.combine_grad(dout, ys, place, weight, offsets)
        used = len(expert)
        dgain = torch.zeros_like(self.gain).index_add_(0, expert, dys[:used] * xs[:used])
        dxs = torch.zeros_like(xs)
        dxs[:used] = dys[:used] * skip
        dlogits = sp.route_grad(dweight, logits, chosen)
        dx = dout + sp.dispatch_grad(dxs, place) + dlogits @ self.router.t()
        dtable = sp.embed_grad(dx, ids, self.table.shape[0])
        return dtable, x.t() @ dlogits, dgain

    def close(self):
        for net in self.nets:
            net.close()


def main():
    torch.manual_seed(0)
    vocab, n = 5000, 2000
    m = Mixture(vocab)
    ids = torch.randint(0, vocab, (n,), device="cuda:0")
    ids[-20:] = -1  # padding
    # a prompt, then token by token
    out, saved = m.forward(ids)
    print("prompt of %d tokens: rows per network %s" % (n, torch.diff(saved[6]).tolist()))
    one = torch.cat([m.forward(ids[t:t + 1])[0] for t in range(5)])
    print("one token at a time: the same to %.1e" % float((one - out[:5]).abs().max()))
    # a few steps towards outputs that are given
    target = out + torch.randn_like(out) * 0.1
    for step in range(5):
        out, saved = m.forward(ids)
        loss = float(((out - target)[ids >= 0] ** 2).mean())
        print("step %d: loss %.6f" % (step, loss))
        dout = torch.where((ids >= 0)[:, None], out - target, 0.0)
        for p, d in zip((m.table, m.router, m.gain), m.gradients(dout, saved)):
            p -= 0.05 * d / d.abs().max().clamp(min=1e-12) * p.abs().mean()
    m.close()


if __name__ == "__main__":
    main()
