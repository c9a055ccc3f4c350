"""The operators as one model uses them (examples/sparse_mixture.py): the
gradients of a training step against a plain fp64 model, its loss, and single
nodes against the batch.

Tolerance of the fp32 comparisons: a gradient passes sums of at most the width
(24), the keys of a row (10), the values of all heads (32), the experts (6),
the keys of a column and the nodes (80), 250 terms in all, each rounding to
2^-24 of what it adds up; the differences in the gradients of the two softmaxes
and of the normalised gates can raise that against their results, for which
eightfold is allowed: 250 * 8 * 2^-24 = 1.2e-4 of a tensor's largest value.
"""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

TOL = 250 * 8 * 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "sparse_mixture.py")
    spec = importlib.util.spec_from_file_location("sparse_mixture", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def make(example, dtype, state_bits, n=80, lr=1e-2):
    import torch
    rowptr, colind = example.random_mask(n, 10, "cuda", seed=3)
    net = example.SparseMixture(rowptr, colind, 24, heads=4, kv_heads=2, d=8, dv=8, experts=6,
                                topk=2, out=8, dtype=dtype, state_bits=state_bits, lr=lr)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(n, 24, device="cuda", generator=g).to(dtype)
    target = torch.randn(n, 8, device="cuda", generator=g)
    return net, x, target, rowptr, colind


def plain(net, params, x, target, rowptr, colind, balance):
    """The model in fp64 on the CPU, with dense masked maps: (loss, y)."""
    import torch
    wq, wk, wv, wr, we, lam = params
    n, H, Hk, d, dv = net.n, net.heads, net.kv_heads, net.d, net.dv
    q = (x @ wq).view(n, H, 2, d)
    k = (x @ wk).view(n, Hk, 2, d)
    v = (x @ wv).view(n, Hk, dv)
    held = torch.zeros(n, n, dtype=torch.bool)
    ptr, col = rowptr.cpu().tolist(), colind.cpu()
    for i in range(n):
        held[i, col[ptr[i]:ptr[i + 1]].long()] = True
    some = held.any(1, keepdim=True).double()
    o = []
    for h in range(H):
        g = h * Hk // H
        maps = []
        for m in range(2):
            s = q[:, h, m] @ k[:, g, m].t() / math.sqrt(d)
            s = s.masked_fill(~held, -1e30)
            maps.append(torch.softmax(s, 1) * some)
        o.append((maps[0] - lam[h] * maps[1]) @ v[:, g])
    logits = torch.cat(o, 1) @ wr
    p = torch.softmax(logits, 1)
    # ties (rows without keys) to the lowest expert
    tie = logits.detach() - torch.arange(net.experts) * 1e-12
    top = tie.topk(net.topk, dim=1).indices
    chosen = torch.zeros_like(p).scatter(1, top, 1.0)
    gates = p * chosen
    gates = gates / gates.sum(1, keepdim=True)
    y = gates @ we
    use = chosen.sum(0)
    aux = balance * net.experts * ((use / use.sum()) * (p.sum(0) / n)).sum()
    return 0.5 * ((y - target) ** 2).sum() / n + aux, y


def close(got, want, what):
    err = (got.double().cpu() - want).abs().max().item()
    assert err <= TOL * want.abs().max().item(), (what, err, want.abs().max().item())


def test_step_gradients_are_the_models(example):
    import torch
    net, x, target, rowptr, colind = make(example, torch.float32, 32)
    S = net.forward(x)
    loss = net.backward(x, S, target)
    params = [p.detach().double().cpu().requires_grad_() for p in net.params]
    args = (x.double().cpu(), target.double().cpu(), rowptr, colind, example.BALANCE)
    want, y = plain(net, params, *args)
    want.backward()
    close(net.y, y.detach(), "y")
    assert abs(loss.item() - want.item()) <= TOL * want.item()
    for name, g, p in zip(("wq", "wk", "wv", "wr", "we", "lam"), net.grads, params):
        close(g, p.grad, name)
    # the same gradients along one direction, against the plain model's difference: h^2
    # curvature and the choice of experts (unchanged at this h) leave h = 1e-6 about 1e-9
    torch.manual_seed(0)
    way = [torch.randn_like(p) for p in params]
    h = 1e-6
    with torch.no_grad():
        ends = [plain(net, [p + s * h * w for p, w in zip(params, way)], *args)[0].item()
                for s in (1, -1)]
    slope = (ends[0] - ends[1]) / (2 * h)
    along = sum((g.double().cpu() * w).sum().item() for g, w in zip(net.grads, way))
    room = sum((g.double().cpu().abs().max() * w.abs().sum()).item()
               for g, w in zip(net.grads, way))
    assert abs(along - slope) <= TOL * room


@pytest.mark.parametrize("bits", [8, 32])
def test_training_lowers_the_loss(example, bits):
    import torch
    net, x, target, *_ = make(example, torch.bfloat16, bits)
    target = target * 0.1 + target[:1]
    losses = [net.step(x, target).item() for _ in range(30)]
    assert all(math.isfinite(v) for v in losses)
    assert losses[-1] < losses[0]


def test_served_nodes_are_the_batchs(example):
    import torch
    net, x, _, rowptr, colind = make(example, torch.float32, 32)
    net.forward(x)
    y = net.serve(x, rowptr, colind, 10)
    close(y, net.y.double().cpu(), "all rows")
    first = int(rowptr[-4])
    y = net.serve(x[-3:], rowptr[-4:] - first, colind[first:], 10)
    close(y, net.y[-3:].double().cpu(), "the last rows")


def test_the_command(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["sparse_mixture.py", "--nodes", "200", "--degree", "8",
                                     "--steps", "5"])
    example.main()
    out = capsys.readouterr().out
    assert "step    5" in out and "served 8 nodes" in out
