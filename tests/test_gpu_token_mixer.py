"""The operators around an attention with a decay as one model uses them
(examples/token_mixer.py): the gradients of a training step against a plain fp64
model, the clipped step, single tokens against the batch; and keys and values that
nsd_qk_append writes, read by the attention over lists of cache slots.

Tolerance of the fp32 comparisons: a gradient passes sums of at most the width (24),
a head's values twice (8 and 8), the tokens (70), all heads' values (32), the words'
tokens (70) and the norms' and products' roundings, below 300 terms in all, each
rounding to 2^-24 of what it adds up; the differences in the norm's gradient and the
projections' can raise that against their results, for which eightfold is allowed:
300 * 8 * 2^-24 = 1.5e-4 of a tensor's largest value.
"""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

TOL = 300 * 8 * 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "token_mixer.py")
    spec = importlib.util.spec_from_file_location("token_mixer", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


LENS = [40, 0, 1, 29]


def make(example, dtype, **kw):
    import torch
    n = sum(LENS)
    net = example.TokenMixer(30, n, len(LENS), width=24, heads=4, kv_heads=2, d=8, dv=8, out=6,
                             dtype=dtype, **kw)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    ids = torch.randint(-2, 30, (n,), device="cuda", generator=g, dtype=torch.int32)
    ids[::3] = 7  # a frequent word
    seqptr, pos = example.packed(LENS)
    target = torch.randn(n, 6, device="cuda", generator=g)
    return net, ids, seqptr, pos, target


def plain(net, params, ids, pos, target):
    """The model in fp64 on the CPU, every pair of tokens of a sequence: (loss, y)."""
    import torch
    table, wq, wk, wv, wo, nq, nk, decay = params
    H, Hk, d, dv = net.heads, net.kv_heads, net.d, net.dv
    keep = (ids >= 0) & (ids < net.vocab)
    x = table[ids.clamp(0, net.vocab - 1).long()] * math.sqrt(net.width) * keep[:, None]
    angle = pos.double()[:, None] * net.freq.cpu()
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turned(z, w):
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + net.turn.eps) * w
        a, b = z[..., :d // 2], z[..., d // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    n = ids.numel()
    q, k = turned((x @ wq).view(n, H, d), nq), turned((x @ wk).view(n, Hk, d), nk)
    v = (x @ wv).view(n, Hk, dv)
    o, first = [], 0
    for m in LENS:
        rows = slice(first, first + m)
        first += m
        t = torch.arange(m, dtype=torch.float64)
        apart = (t[:, None] - t).clamp_min(0)
        seen = (t[:, None] >= t).double()
        for h in range(H):
            e = h * Hk // H
            w = torch.exp(decay[h] * apart) * seen / math.sqrt(d)
            o.append(((q[rows, h] @ k[rows, e].t()) * w) @ v[rows, e])
    o = torch.cat([torch.cat(o[i * H:(i + 1) * H], 1) for i in range(len(LENS))])
    y = o @ wo
    return 0.5 * ((y - target) ** 2).sum() / n, y


def close(got, want, what):
    err = (got.double().cpu() - want).abs().max().item()
    assert err <= TOL * want.abs().max().item(), (what, err, want.abs().max().item())


def test_step_gradients_are_the_models(example):
    import torch
    net, ids, seqptr, pos, target = make(example, torch.float32)
    y = net.forward(ids, seqptr, pos)
    loss = net.backward(ids, seqptr, pos, y, target)
    params = [p.detach().double().cpu().requires_grad_() for p in net.params]
    args = (ids.cpu(), pos.cpu(), target.double().cpu())
    want, want_y = plain(net, params, *args)
    want.backward()
    close(y, want_y.detach(), "y")
    assert abs(loss.item() - want.item()) <= TOL * want.item()
    for name, g, p in zip(("table", "wq", "wk", "wv", "wo", "nq", "nk", "decay"), net.grads,
                          params):
        close(g, p.grad, name)
    # along one direction, against the plain model's difference: h^2 curvature at this h
    # leaves h = 1e-6 about 1e-9
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


def test_the_step_takes_clipped_gradients(example):
    """The optimizer measures the gradients that the operators wrote."""
    import torch
    net, ids, seqptr, pos, target = make(example, torch.float32, max_norm=1e-3)
    net.step(ids, seqptr, pos, target)
    norm = math.sqrt(sum((g.double() ** 2).sum().item() for g in net.grads))
    p = net.optim.grad_norm
    assert abs(p.norm.item() - norm) <= 1e-9 * norm and norm > 1e-3
    assert abs(p.scale.item() - 1e-3 / (norm + 1e-6)) <= 2.0 ** -22 * p.scale.item()


def test_a_shorter_batch(example):
    """Fewer tokens and sequences than there is room for: the gradients of a model that has
    room for them alone (sums of the dense products may have another order); more are refused."""
    import torch
    net, ids, seqptr, pos, target = make(example, torch.float32)
    room = example.TokenMixer(30, 20_000, 9, width=24, heads=4, kv_heads=2, d=8, dv=8, out=6,
                              dtype=torch.float32)
    for t in (room.x, room.q, room.k, room.v, room.o, room.do, room.dqr, room.dkr, room.dvv):
        t.fill_(float("nan"))
    losses = []
    for m in (net, room):
        y = m.forward(ids, seqptr, pos)
        losses.append(m.backward(ids, seqptr, pos, y, target).item())
    assert abs(losses[0] - losses[1]) <= TOL * losses[0]
    for a, b in zip(net.grads, room.grads):
        close(b, a.double().cpu(), tuple(a.shape))
    more = torch.zeros(71, dtype=torch.int32, device="cuda")
    for args in ((more, seqptr, more), (ids, torch.zeros(6, dtype=torch.int32, device="cuda"), pos)):
        with pytest.raises(ValueError, match="room for 70 in 4"):
            net.forward(*args)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_training_runs(example, dtype):
    import torch
    net, ids, seqptr, pos, target = make(example, getattr(torch, dtype))
    losses = [net.step(ids, seqptr, pos, target).item() for _ in range(10)]
    assert all(math.isfinite(v) for v in losses)
    assert all(torch.isfinite(p.float()).all() for p in net.params)


def test_served_tokens_are_the_batchs(example):
    import torch
    net, ids, seqptr, pos, target = make(example, torch.float32)
    y = net.forward(ids, seqptr, pos)
    state = net.state(6)
    slots = torch.tensor([4, 0, 2, 5], dtype=torch.int32, device="cuda")
    first = seqptr[:-1].long()
    for t in range(max(LENS)):
        live = [i for i, m in enumerate(LENS) if t < m]
        at = first[live] + t
        out = net.serve(ids[at], slots[live], pos[at], state)
        close(out, y[at].double().cpu(), t)
    assert torch.all(state[[0, 1, 3]] == 0)  # the empty sequence's, and nobody's


def test_the_command(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["token_mixer.py", "--vocab", "50", "--tokens", "600",
                                     "--sequences", "3", "--steps", "5"])
    example.main()
    out = capsys.readouterr().out
    assert "step    5" in out and "served 3 sequences" in out


def test_appended_keys_and_values_are_what_attention_reads():
    """Tokens appended one batch after the other to scattered slots of a cache, then read
    by the differential attention over lists of slots: as over rows that were rotated in
    one call."""
    import torch
    from paper_2303_07030_amd import nsd
    H, Hk, d, dv, n, slots = 4, 2, 16, 24, 60, 100
    g = torch.Generator(device="cuda")
    g.manual_seed(2)

    def rows(m, w):
        return torch.randn(m, w, device="cuda", generator=g)

    # (a head of the differential attention is two halves, each with its norm and rotation)
    q, k, v = rows(n, H * 2 * d), rows(n, Hk * 2 * d), rows(n, Hk * dv)
    wq, wk = rows(1, d)[0], rows(1, d)[0]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    freq = 100.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    kc, vc = rows(slots, Hk * 2 * d), rows(slots, Hk * dv)
    slot = torch.randperm(slots, device="cuda", generator=g)[:n].int()
    qo = torch.empty_like(q)
    for a, b in ((0, 1), (1, 40), (40, n)):
        s = nsd.qk_desc(2 * H, 2 * Hk, d, q[a:b], k[a:b], qo[a:b], kc)
        nsd.nsd_qk_append(b - a, s, q[a:b], k[a:b], v[a:b], wq, wk, pos[a:b], freq, slot[a:b],
                          slots, qo[a:b], kc, vc)
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    s = nsd.qk_desc(2 * H, 2 * Hk, d, q, k, qr, kr)
    nsd.nsd_qk_rotate(n, s, q, k, wq, wk, pos, freq, qr, kr)
    lam = torch.full((H,), 0.3, device="cuda")
    outs = []
    for queries, keys, values, cols in ((qo, kc, vc, slot),
                                        (qr, kr, v, torch.arange(n, device="cuda").int())):
        o = torch.empty(3, H * dv, device="cuda")
        lens = [n, 1, 40]
        rowptr = torch.tensor([0, n, n + 1, n + 41], dtype=torch.int32, device="cuda")
        lists = torch.cat([cols[:m] for m in lens])
        last = queries[[n - 1, 0, 39]].contiguous()
        attn = nsd.attn_desc(H, Hk, d, dv, last, keys, values, o, d ** -0.5)
        ws = torch.empty(max(256, nsd.nsd_attn_diff_decode_workspace_size(3, n, attn)),
                         dtype=torch.uint8, device="cuda")
        nsd.nsd_attn_diff_decode(3, rowptr, lists, n, attn, last, keys, values, lam, None, o, ws)
        outs.append(o)
    assert torch.equal(*outs)
