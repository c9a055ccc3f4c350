"""A layer that learns over a sparse pattern, trained and then served.

  o = attention of x over the stored keys of a mask     nsd_attn_diff
  S = the top-k gates of o W_r, a CSR [nodes x experts]  nsd_route
  y = S E, one row of E an expert                        nsd_spmm
  L = 1/2 mean |y - target|^2 + the balance loss of S

A training step takes the gradients back through the same operators
(nsd_spmm_vjp on S's pattern, nsd_route_vjp, nsd_attn_diff_vjp) and updates
every tensor in one launch (optim.AdamW).  Serving holds keys and values as
caches and answers single nodes from lists of slots (nsd_attn_diff_decode),
then routes and mixes them.  The dense projections are plain matrix products.

  python examples/sparse_mixture.py [--nodes N] [--degree D] [--steps K]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2303_07030_amd import nsd, optim  # noqa: E402
from paper_2303_07030_amd.operand import DeviceCsr  # noqa: E402

BALANCE = 0.01


def regular_rows(n, k, device):
    """rowptr of n rows of k entries."""
    return torch.arange(n + 1, dtype=torch.int32, device=device) * k


class SparseMixture:
    """Buffers, weights and one step of the layer over a fixed mask of `nodes`
    rows (rowptr, colind: a CSR with sorted rows)."""

    def __init__(self, rowptr, colind, width, heads=8, kv_heads=2, d=32, dv=64, experts=16,
                 topk=2, out=32, dtype=torch.bfloat16, state_bits=8, lr=1e-2, seed=0):
        dev = rowptr.device
        self.n = n = rowptr.numel() - 1
        self.heads, self.kv_heads, self.d, self.dv = heads, kv_heads, d, dv
        self.experts, self.topk, self.out, self.dtype = experts, topk, out, dtype
        g = torch.Generator(device=dev)
        g.manual_seed(seed)

        def weight(rows, cols, dt=dtype):
            w = torch.randn(rows, cols, device=dev, generator=g) / math.sqrt(rows)
            return w.to(dt)

        # projections, router, experts, lambda a head
        self.wq = weight(width, heads * 2 * d)
        self.wk = weight(width, kv_heads * 2 * d)
        self.wv = weight(width, kv_heads * dv)
        self.wr = weight(heads * dv, experts)
        self.we = weight(experts, out, torch.float32)
        self.lam = torch.full((heads,), 0.5, device=dev)
        self.params = [self.wq, self.wk, self.wv, self.wr, self.we, self.lam]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.optim = optim.AdamW(self.params, self.grads, lr=lr, state_bits=state_bits,
                                 masters=True, weight_decay=[0.01] * 5 + [0.0])

        # what the forward leaves for the gradient
        def rows(w):
            return torch.empty(n, w, dtype=dtype, device=dev)

        self.q, self.k, self.v = rows(heads * 2 * d), rows(kv_heads * 2 * d), rows(kv_heads * dv)
        self.o, self.do = rows(heads * dv), rows(heads * dv)
        self.dq, self.dk, self.dv_ = (torch.empty_like(t) for t in (self.q, self.k, self.v))
        self.stat = torch.empty(n, heads, 4, device=dev)
        self.attn = nsd.attn_desc(heads, kv_heads, d, dv, self.q, self.k, self.v, self.o,
                                  1.0 / math.sqrt(d))
        self.mask = DeviceCsr(n, n, rowptr, colind, torch.zeros(colind.numel(), device=dev),
                              item_len=nsd.nsd_attn_item_len(colind.numel(), self.attn))
        self.attn_ws = self._bytes(nsd.nsd_attn_diff_workspace_size(self.mask.desc,
                                                                    self.mask.csc, self.attn))
        self.logits = torch.empty(n, experts, dtype=dtype, device=dev)
        self.dlogits = torch.empty_like(self.logits)
        self.router = nsd.router_desc(experts, topk, self.logits)
        self.route_ws = self._bytes(nsd.nsd_route_workspace_size(n, self.router))
        self.gate_col = torch.empty(n * topk, dtype=torch.int32, device=dev)
        self.gate = torch.empty(n * topk, device=dev)
        self.dgate = torch.empty_like(self.gate)
        self.counts = torch.empty(experts + 1, dtype=torch.int32, device=dev)
        self.balance = torch.empty(1, dtype=torch.float64, device=dev)
        self.gate_rowptr = regular_rows(n, topk, dev)
        self.y = torch.empty(n, out, device=dev)

    def _bytes(self, n):
        return torch.empty(max(n, 256), dtype=torch.uint8, device=self.lam.device)

    def mix(self, rows, col, gate, rowptr, y, build_csc):
        """y = S E; S holds views of the gates (no copy)."""
        S = DeviceCsr(rows, self.experts, rowptr, col, gate, build_csc=build_csc, k_hint=self.out)
        nsd.nsd_spmm(S.desc, self.we, self.out, y, S.workspace(self.out))
        return S

    def forward(self, x, build_csc=True):
        torch.mm(x, self.wq, out=self.q)
        torch.mm(x, self.wk, out=self.k)
        torch.mm(x, self.wv, out=self.v)
        nsd.nsd_attn_diff(self.mask.desc, self.attn, self.q, self.k, self.v, self.lam, None,
                          self.o, self.stat, self.attn_ws)
        torch.mm(self.o, self.wr, out=self.logits)
        nsd.nsd_route(self.n, self.router, self.logits, None, BALANCE, self.gate_col, self.gate,
                      self.counts, self.balance, self.route_ws)
        return self.mix(self.n, self.gate_col, self.gate, self.gate_rowptr, self.y, build_csc)

    def backward(self, x, S, target):
        """The loss; leaves every weight's gradient in `grads`."""
        diff = self.y - target
        loss = 0.5 * (diff * diff).sum() / self.n + self.balance[0]
        gwq, gwk, gwv, gwr, gwe, glam = self.grads
        nsd.nsd_spmm_vjp(S.desc, S.csc, self.we, diff / self.n, self.out, self.dgate, gwe,
                         S.workspace(self.out))
        nsd.nsd_route_vjp(self.n, self.router, self.logits, None, self.gate_col, self.gate,
                          self.counts, BALANCE, 1.0, self.dgate, self.dlogits)
        torch.mm(self.o.t(), self.dlogits, out=gwr)
        torch.mm(self.dlogits, self.wr.t(), out=self.do)
        nsd.nsd_attn_diff_vjp(self.mask.desc, self.mask.csc, self.attn, self.q, self.k, self.v,
                              self.lam, None, self.stat, self.do, self.dq, self.dk, self.dv_,
                              glam, None, self.attn_ws)
        for w, dy in ((gwq, self.dq), (gwk, self.dk), (gwv, self.dv_)):
            torch.mm(x.t(), dy, out=w)
        return loss

    def step(self, x, target):
        S = self.forward(x)
        loss = self.backward(x, S, target)
        self.optim.step()
        return loss

    def serve(self, x, rowptr, slots, longest):
        """Answers for single nodes with features x against the cached keys and
        values of the last forward: row i reads the slots
        slots[rowptr[i]:rowptr[i + 1]], at most `longest` of them."""
        rows, dev = x.shape[0], x.device
        q = x @ self.wq
        o = torch.empty(rows, self.heads * self.dv, dtype=self.dtype, device=dev)
        attn = nsd.attn_desc(self.heads, self.kv_heads, self.d, self.dv, q, self.k, self.v, o,
                             1.0 / math.sqrt(self.d))
        ws = self._bytes(nsd.nsd_attn_diff_decode_workspace_size(rows, longest, attn))
        nsd.nsd_attn_diff_decode(rows, rowptr, slots, longest, attn, q, self.k, self.v, self.lam,
                                 None, o, ws)
        logits = o @ self.wr
        col = torch.empty(rows * self.topk, dtype=torch.int32, device=dev)
        gate = torch.empty(rows * self.topk, device=dev)
        router = nsd.router_desc(self.experts, self.topk, logits)
        nsd.nsd_route(rows, router, logits, None, 0.0, col, gate, None, None, None)
        y = torch.empty(rows, self.out, device=dev)
        self.mix(rows, col, gate, regular_rows(rows, self.topk, dev), y, False)
        return y


def random_mask(n, degree, device, seed=0):
    """CSR with up to `degree` distinct random keys a row (some rows fewer, one
    in 64 none)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    col = torch.randint(n, (n, degree), device=device, generator=g).sort(dim=1).values
    keep = torch.ones_like(col, dtype=torch.bool)
    keep[:, 1:] = col[:, 1:] != col[:, :-1]
    keep[::64] = False
    rowptr = torch.zeros(n + 1, dtype=torch.int32, device=device)
    rowptr[1:] = keep.sum(dim=1).cumsum(0)
    return rowptr, col[keep].to(torch.int32)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--nodes", type=int, default=20000)
    ap.add_argument("--degree", type=int, default=24)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    dev = "cuda"
    rowptr, colind = random_mask(a.nodes, a.degree, dev)
    net = SparseMixture(rowptr, colind, a.width)
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    x = torch.randn(a.nodes, a.width, device=dev, generator=g).to(net.dtype)
    target = torch.randn(a.nodes, 1, device=dev, generator=g) * 0.1 + \
        torch.randn(1, net.out, device=dev, generator=g)
    for i in range(a.steps):
        loss = net.step(x, target)
        if i == 0 or (i + 1) % 5 == 0:
            print(f"step {i + 1:4d}  loss {loss.item():.5f}  balance {net.balance.item():.5f}",
                  flush=True)
    # serve the last nodes with the slots of their rows
    net.forward(x, build_csc=False)
    m = min(8, a.nodes)
    first = int(rowptr[-m - 1])
    ptr = rowptr[-m - 1:] - first
    y = net.serve(x[-m:], ptr, colind[first:], a.degree)
    print(f"served {m} nodes, largest difference from the batch: "
          f"{(y - net.y[-m:]).abs().max().item():.2e}")


if __name__ == "__main__":
    main()
