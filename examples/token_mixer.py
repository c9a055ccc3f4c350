"""A token model with a memory that fades, trained and then served.

  x = scaled rows of a table by token             nsd_embed
  q, k = norm and rotation of x W_q, x W_k          nsd_qk_rotate
  o = attention with a decay per head over x's
      packed sequences                              nsd_attn_decay
  y = o W_o,  L = 1/2 mean |y - target|^2

A training step takes the gradients back through the same operators
(nsd_attn_decay_vjp, nsd_qk_rotate_vjp, nsd_embed_vjp: the decays, the norms'
weights and the table learn too), measures all of them and clips what the
optimizer takes (optim.AdamW with max_norm).  Serving holds one state per
sequence and head, whatever the sequence's length, and moves it on token by
token (nsd_attn_decay_step).  The dense projections are plain matrix products.

  python examples/token_mixer.py [--vocab V] [--tokens T] [--sequences S] [--steps K]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2303_07030_amd import nsd, optim  # noqa: E402


class TokenMixer:
    """Weights, buffers and one step over batches of up to `tokens` tokens, all of them in one
    of up to `sequences` packed sequences."""

    def __init__(self, vocab, tokens, sequences, width=128, heads=4, kv_heads=2, d=32, dv=32,
                 out=32, dtype=torch.bfloat16, lr=1e-2, max_norm=1.0, seed=0, device="cuda"):
        self.vocab, self.width, self.n, self.seqs = vocab, width, tokens, sequences
        self.heads, self.kv_heads, self.d, self.dv, self.dtype = heads, kv_heads, d, dv, dtype
        dev = torch.device(device)
        g = torch.Generator(device=dev)
        g.manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, device=dev, generator=g) / math.sqrt(rows)).to(dtype)

        self.table = (torch.randn(vocab, width, device=dev, generator=g) * 0.1).to(dtype)
        self.wq, self.wk = weight(width, heads * d), weight(width, kv_heads * d)
        self.wv, self.wo = weight(width, kv_heads * dv), weight(heads * dv, out)
        self.nq, self.nk = torch.ones(d, device=dev), torch.ones(d, device=dev)
        # heads that forget over some tokens to some hundred
        self.decay = -(2.0 ** -torch.linspace(2.0, 8.0, heads, device=dev))
        self.params = [self.table, self.wq, self.wk, self.wv, self.wo, self.nq, self.nk,
                       self.decay]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.optim = optim.AdamW(self.params, self.grads, lr=lr, masters=True, max_norm=max_norm,
                                 weight_decay=[0.01] * 5 + [0.0] * 3)

        def rows(w):
            return torch.empty(tokens, w, dtype=dtype, device=dev)

        self.x, self.dx = rows(width), rows(width)
        self.q, self.k, self.v = rows(heads * d), rows(kv_heads * d), rows(kv_heads * dv)
        self.qr, self.kr = torch.empty_like(self.q), torch.empty_like(self.k)
        self.dqr, self.dkr, self.dvv = (torch.empty_like(t) for t in (self.q, self.k, self.v))
        self.o, self.do = rows(heads * dv), rows(heads * dv)
        self.freq = 10_000.0 ** (-torch.arange(0, d, 2, device=dev, dtype=torch.float64) / d)
        self.embedding = nsd.embed_desc(self.table, self.x, math.sqrt(width), grad=self.grads[0])
        self.turn = nsd.qk_desc(heads, kv_heads, d, self.q, self.k, self.qr, self.kr)
        self.attn = nsd.decay_desc(heads, kv_heads, d, dv, self.qr, self.kr, self.v, self.o,
                                   1.0 / math.sqrt(d))
        self.ws = [torch.empty(size, dtype=torch.uint8, device=dev) for size in (
            nsd.nsd_embed_vjp_workspace_size(tokens, self.embedding),
            nsd.nsd_qk_rotate_vjp_workspace_size(tokens, self.turn),
            nsd.nsd_attn_decay_workspace_size(tokens, sequences, tokens, self.attn, True))]

    def forward(self, ids, seqptr, pos):
        n, seqs = ids.numel(), seqptr.numel() - 1
        if n > self.n or seqs > self.seqs:
            raise ValueError(f"{n} tokens in {seqs} sequences, room for {self.n} in {self.seqs}")
        x, q, k, v, o = (t[:n] for t in (self.x, self.q, self.k, self.v, self.o))
        nsd.nsd_embed(n, self.embedding, ids, self.table, x)
        torch.mm(x, self.wq, out=q)
        torch.mm(x, self.wk, out=k)
        torch.mm(x, self.wv, out=v)
        nsd.nsd_qk_rotate(n, self.turn, q, k, self.nq, self.nk, pos, self.freq, self.qr, self.kr)
        nsd.nsd_attn_decay(n, seqs, seqptr, n, self.attn, self.qr, self.kr, v, self.decay, None,
                           o, None, self.ws[2])
        return o @ self.wo

    def backward(self, ids, seqptr, pos, y, target):
        """The loss; leaves every parameter's gradient in `grads`."""
        n, seqs = ids.numel(), seqptr.numel() - 1
        x, o, dx, do, dqr, dkr, dvv = (t[:n] for t in (self.x, self.o, self.dx, self.do, self.dqr,
                                                       self.dkr, self.dvv))
        gtable, gwq, gwk, gwv, gwo, gnq, gnk, gdecay = self.grads
        diff = y.float() - target
        dy = (diff / n).to(self.dtype)
        torch.mm(o.t(), dy, out=gwo)
        torch.mm(dy, self.wo.t(), out=do)
        nsd.nsd_attn_decay_vjp(n, seqs, seqptr, n, self.attn, self.qr, self.kr, self.v, self.decay,
                               None, do, None, dqr, dkr, dvv, gdecay, None, self.ws[2])
        # (the rotated rows' gradients become those of the projections' outputs in place)
        nsd.nsd_qk_rotate_vjp(n, self.turn, self.q, self.k, self.nq, self.nk, pos, self.freq,
                              dqr, dkr, dqr, dkr, gnq, gnk, self.ws[1])
        for w, dproj in ((gwq, dqr), (gwk, dkr), (gwv, dvv)):
            torch.mm(x.t(), dproj, out=w)
        torch.mm(dqr, self.wq.t(), out=dx)
        dx.addmm_(dkr, self.wk.t()).addmm_(dvv, self.wv.t())
        nsd.nsd_embed_vjp(n, self.embedding, ids, dx, False, gtable, self.ws[0])
        return 0.5 * (diff * diff).sum() / n

    def step(self, ids, seqptr, pos, target):
        y = self.forward(ids, seqptr, pos)
        loss = self.backward(ids, seqptr, pos, y, target)
        self.optim.step()
        self.decay.clamp_(max=0.0)
        return loss

    def state(self, slots):
        """States of `slots` sequences that have not begun."""
        return torch.zeros(slots, self.heads, self.d, self.dv, device=self.decay.device)

    def serve(self, ids, slot, pos, state):
        """Outputs for one new token each of the sequences in slots `slot`, at positions `pos`;
        the states move on."""
        n, dev = ids.numel(), ids.device

        def rows(w):
            return torch.empty(n, w, dtype=self.dtype, device=dev)

        x = rows(self.width)
        nsd.nsd_embed(n, nsd.embed_desc(self.table, x, self.embedding.scale), ids, self.table, x)
        q, k, v = x @ self.wq, x @ self.wk, x @ self.wv
        turn = nsd.qk_desc(self.heads, self.kv_heads, self.d, q, k, q, k)
        nsd.nsd_qk_rotate(n, turn, q, k, self.nq, self.nk, pos, self.freq, q, k)
        o = rows(self.heads * self.dv)
        attn = nsd.decay_desc(self.heads, self.kv_heads, self.d, self.dv, q, k, v, o,
                              self.attn.scale)
        nsd.nsd_attn_decay_step(n, slot, state.shape[0], attn, q, k, v, self.decay, state, o)
        return o @ self.wo


def packed(lens, device="cuda"):
    """(seqptr, positions) of packed sequences."""
    ptr = torch.zeros(len(lens) + 1, dtype=torch.int32, device=device)
    ptr[1:] = torch.tensor(lens, device=device).cumsum(0)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(device)
    return ptr, pos


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--sequences", type=int, default=6)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    net = TokenMixer(a.vocab, a.tokens, a.sequences)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ids = torch.randint(a.vocab, (a.tokens,), device="cuda", generator=g, dtype=torch.int32)
    lens = [a.tokens // a.sequences] * a.sequences
    lens[0] += a.tokens - sum(lens)
    seqptr, pos = packed(lens)
    # what a token's answer has to be depends on it and the one before it
    code = torch.randn(a.vocab, 32, device="cuda", generator=g)
    target = code[ids.long()] + 0.5 * code[ids.roll(1).long()]
    for i in range(a.steps):
        loss = net.step(ids, seqptr, pos, target)
        if i == 0 or (i + 1) % 5 == 0:
            print(f"step {i + 1:4d}  loss {loss.item():.5f}  gradient norm "
                  f"{net.optim.grad_norm.norm.item():.4f}", flush=True)
    # serve the first tokens of every sequence one by one
    y = net.forward(ids, seqptr, pos)
    state, worst = net.state(a.sequences), 0.0
    slot = torch.arange(a.sequences, dtype=torch.int32, device="cuda")
    first = seqptr[:-1].long()
    for t in range(min(8, min(lens))):
        out = net.serve(ids[first + t], slot, pos[first + t], state)
        worst = max(worst, (out.float() - y[first + t].float()).abs().max().item())
    print(f"served {a.sequences} sequences, largest difference from the batch: {worst:.2e}")


if __name__ == "__main__":
    main()
