"""Workloads of the operators that learn: attention over a sparse mask, the
router of a sparse mixture, and the optimizer's step.

Each case is one call, or the calls of one training step, on data already in
HBM.  With `own` the operators are those of this package; without it they are
computed in their plain form, by elementary torch operations in 32 bits.

attn    differential attention over the stored keys of a CSR mask: the
        difference of two softmax maps, the second weighted by a learned
        number per head; the forward pass, or a training step with every
        gradient
decode  the same for one new token per sequence over lists of cache slots
route   the top-k gates of a router, the use of every expert, the balance
        loss; with the gradient in training
adamw   one step of AdamW over a model's tensors

All inputs are drawn on the GPU from a seed.
"""
import math
import random

import torch

own = False
DEV = "cuda"
BLOCK = 256       # values that share a scale in 8-bit optimizer states
HYPER = dict(lr=2e-4, beta1=0.9, beta2=0.98, eps=1e-8)


# ------------------------------------------------------------------ cases

def listed():
    return [
        # the next token of four chats of some hundred tokens each, the cache
        # shared and paged: a call of microseconds, all latency
        dict(name="decode_4x700", kind="decode", rows=4, len=700, slots=8192, heads=8, kv=2,
             d=64, dv=128, dtype="bf16"),
        # sixteen long documents being continued: the cache is read once
        dict(name="decode_16x32k", kind="decode", rows=16, len=32_000, slots=600_000, heads=16,
             kv=4, d=64, dv=128, dtype="bf16"),
        # a training step of graph attention on the SpMM workload's pattern and
        # hidden size (64), in 32 bits
        dict(name="attn_graph_100k_1m", kind="attn", mode="train", mask="graph", nq=100_000,
             nk=100_000, nnz=1_000_000, s=1.1, cap=5000, heads=4, kv=4, d=8, dv=16, dtype="f32",
             bias=False),
        # a training step over a document: a window of 256 tokens and 16 tokens
        # that all see, queries, keys and values from one projection
        dict(name="attn_window_8k", kind="attn", mode="train", mask="window", nq=8192, nk=8192,
             win=256, glob=16, heads=8, kv=4, d=64, dv=128, dtype="bf16", bias=False),
        # odd sizes: a rectangular pattern with empty rows, a learned bias per
        # stored key that masks a tenth of them, heads sharing keys
        dict(name="attn_odd_20k_400k", kind="attn", mode="train", mask="graph", nq=20_011,
             nk=12_007, nnz=400_009, s=0.0, cap=0, heads=6, kv=3, d=40, dv=72, dtype="bf16",
             bias=True),
        # inference on a graph of the layer workload's pattern and half its width
        dict(name="attn_fwd_200k_4m", kind="attn", mode="fwd", mask="graph", nq=200_000,
             nk=200_000, nnz=4_000_000, s=1.05, cap=20_000, heads=8, kv=8, d=16, dv=32,
             dtype="bf16", bias=False),
        # the router of a serving step: a few tokens, all latency
        dict(name="route_16_e64_k8", kind="route", mode="fwd", tokens=16, experts=64, topk=8,
             norm=True, skip=0.0, dtype="bf16"),
        # the router of a training step
        dict(name="route_131k_e128_k8", kind="route", mode="train", tokens=131_072, experts=128,
             topk=8, norm=True, skip=0.0, dtype="bf16"),
        # odd sizes, padded tokens, gates that are not normalised
        dict(name="route_10k_e60_k4", kind="route", mode="train", tokens=10_007, experts=60,
             topk=4, norm=False, skip=0.1, dtype="f32"),
        # a model of many small tensors
        dict(name="adamw_300_small", kind="adamw", tensors=300, total=2_000_000, states=32,
             weights="f32", grads="f32"),
        # a model in bf16 with 32-bit copies of its weights
        dict(name="adamw_200m_f32", kind="adamw", tensors=24, total=200_000_000, states=32,
             weights="copy", grads="bf16"),
        # the same without copies, states in 8 bits
        dict(name="adamw_200m_8bit", kind="adamw", tensors=24, total=200_000_000, states=8,
             weights="bf16", grads="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    """Heads of usual widths (values twice as wide as a query's half), or odd ones."""
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    if rng.random() < 0.5:
        d = rng.choice([8, 16, 32, 64])
        return dict(heads=heads, kv=kv, d=d, dv=2 * d)
    return dict(heads=heads, kv=kv, d=_log(rng, 5, 100), dv=_log(rng, 5, 200))


def draw(rng):
    kind = rng.choice(["decode", "attn", "attn", "route", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "decode":
        rows, length = _log(rng, 1, 32), _log(rng, 1, 32_000)
        c = dict(kind=kind, rows=rows, len=length, slots=max(64, int(1.2 * rows * length)),
                 dtype=dtype, **_heads(rng))
        while rows * length * c["kv"] * (2 * c["d"] + c["dv"]) > 5e8 and c["kv"] > 1:
            c.update(heads=c["heads"] // c["kv"], kv=1)
        return c
    if kind == "attn":
        h = _heads(rng)
        nnz = _log(rng, 2000, 3_000_000)
        nnz = min(nnz, int(1.2e9 / (h["heads"] * (2 * h["d"] + h["dv"]))))
        c = dict(kind=kind, mode=rng.choice(["train", "train", "fwd"]), dtype=dtype,
                 bias=rng.random() < 0.5, **h)
        if rng.random() < 0.3:
            win, glob = _log(rng, 8, 512), rng.choice([0, 1, 16])
            n = max(64, nnz // (win + glob))
            return dict(c, mask="window", nq=n, nk=n, win=win, glob=glob)
        nq, nk = (max(32, nnz // _log(rng, 4, 60)) for _ in range(2))
        return dict(c, mask="graph", nq=nq, nk=nk, nnz=min(nnz, nq * nk // 8),
                    s=rng.choice([0.0, 1.1]), cap=max(64, nk // 16))
    if kind == "route":
        experts = rng.choice([4, 8, 16, 64, 128, 256, _log(rng, 5, 512)])
        tokens = min(_log(rng, 1, 200_000), 20_000_000 // experts)
        return dict(kind=kind, mode=rng.choice(["train", "fwd"]), tokens=tokens, experts=experts,
                    topk=min(experts, rng.choice([1, 2, 4, 6, 8])), norm=rng.random() < 0.5,
                    skip=rng.choice([0.0, 0.1]), dtype=dtype)
    return dict(kind=kind, tensors=_log(rng, 1, 200), total=_log(rng, 10_000, 100_000_000),
                states=rng.choice([32, 8]), weights=rng.choice(["f32", "bf16", "copy"]),
                grads=rng.choice(["f32", "bf16"]))


# ----------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _type(c, key="dtype"):
    return torch.float32 if c[key] == "f32" else torch.bfloat16


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).mul_(std).to(dtype)


def _graph(g, c):
    """nnz distinct (row, column) pairs: rows by a Zipf profile over a random
    ranking (none over `cap` on average) or uniform, a twentieth of the rows
    empty; columns uniform."""
    nq, nk, nnz = c["nq"], c["nk"], c["nnz"]
    used = max(1, nq - nq // 20)
    order = torch.randperm(nq, generator=g, device=DEV)
    if c["s"] > 0:
        w = torch.arange(1, used + 1, device=DEV, dtype=torch.float64) ** -c["s"]
        w = torch.clamp(w / w.sum(), max=c["cap"] / nnz)
        cdf = torch.cumsum(w / w.sum(), 0)
    keys = torch.empty(0, dtype=torch.int64, device=DEV)
    while keys.numel() < nnz:
        m = nnz + nnz // 8 + 64
        if c["s"] > 0:
            u = torch.rand(m, generator=g, device=DEV, dtype=torch.float64)
            r = torch.searchsorted(cdf, u).clamp_(max=used - 1)
        else:
            r = torch.randint(used, (m,), generator=g, device=DEV)
        col = torch.randint(nk, (m,), generator=g, device=DEV)
        keys = torch.unique(torch.cat([keys, order[r] * nk + col]))
    at = torch.arange(nnz, device=DEV) * keys.numel() // nnz
    return keys[at] // nk, keys[at] % nk


def _window(c):
    """Row i stores the `glob` first keys and the `win` keys up to its own."""
    n, w, glob = c["nq"], c["win"], c["glob"]
    i = torch.arange(n, device=DEV)[:, None]
    j = torch.cat([torch.arange(glob, device=DEV).expand(n, glob),
                   i + torch.arange(1 - w, 1, device=DEV)], 1)
    keep = j >= 0
    keep[:, :glob] &= j[:, :glob] <= i - w
    return i.expand_as(j)[keep], j[keep]


def _lens(c):
    """Lengths of a decode case's rows: ragged, one of them a first token."""
    r = random.Random(c["rows"] * 1_000_003 + c["len"])
    n = [r.randint((c["len"] + 1) // 2, c["len"]) for _ in range(c["rows"])]
    if len(n) > 2:
        n[1] = 1
    return n


def _entries(c):
    if c["kind"] == "decode":
        return sum(_lens(c))
    if c["mask"] == "graph":
        return c["nnz"]
    n, w, glob = c["nq"], c["win"], c["glob"]
    return sum(min(i + 1, w) + max(0, min(glob, i - w + 1)) for i in range(n))


def _attn_inputs(c, g):
    H, Hk, d, dv, T = c["heads"], c["kv"], c["d"], c["dv"], _type(c)
    if c["kind"] == "decode":
        nq, nk = c["rows"], c["slots"]
        row = torch.repeat_interleave(torch.arange(nq, device=DEV),
                                      torch.tensor(_lens(c), device=DEV))
        col = torch.randperm(nk, generator=g, device=DEV)[:row.numel()]
    else:
        nq, nk = c["nq"], c["nk"]
        row, col = _graph(g, c) if c["mask"] == "graph" else _window(c)
    rowptr = torch.zeros(nq + 1, dtype=torch.int32, device=DEV)
    rowptr[1:] = torch.cumsum(torch.bincount(row, minlength=nq), 0)
    S = dict(rowptr=rowptr, row=row, col=col.int())
    if c.get("mask") == "window":  # one projection's output: a token's q, k, v side by side
        qkv = _normal(g, nq, H * 2 * d + Hk * 2 * d + Hk * dv, dtype=T)
        q, k, v = qkv.split([H * 2 * d, Hk * 2 * d, Hk * dv], 1)
    else:
        q, k, v = (_normal(g, n, w, dtype=T) for n, w in
                   ((nq, H * 2 * d), (nk, Hk * 2 * d), (nk, Hk * dv)))
    S.update(q=q, k=k, v=v, lam=0.2 + 0.6 * torch.rand(H, generator=g, device=DEV), bias=None)
    if c.get("bias"):  # a tenth of the keys masked, and every key of some rows
        b = _normal(g, row.numel())
        off = torch.rand(row.numel(), generator=g, device=DEV) < 0.1
        off |= (torch.rand(nq, generator=g, device=DEV) < 0.01)[row]
        S["bias"] = b.masked_fill_(off, -math.inf)
    if c.get("mode") == "train":
        S["dO"] = _normal(g, nq, H * dv, dtype=T)
    return S


def _sizes(c):
    """Lengths of a model's tensors: a few take most of the weights, none of
    them of a round size, the smallest of one value."""
    n, total = c["tensors"], c["total"]
    w = [1.0 / (i + 1) ** 0.7 for i in range(n)]
    sizes = [max(1, int(total * x / sum(w))) for x in w]
    if n > 2:
        sizes[-1], sizes[-2] = 1, 3
    return sizes


def _padded(c):
    """Each tensor's room in the flat buffers: whole blocks."""
    return [-(-n // BLOCK) * BLOCK for n in _sizes(c)]


def _tensors(c, flat, per=1):
    """The tensors in a flat buffer of one value for each `per` weights."""
    return [t[: -(-n // per)] for t, n in zip(flat.split([n // per for n in _padded(c)]),
                                              _sizes(c))]


def _adamw_inputs(c, g):
    """A model's tensors in flat buffers, one for each kind, zeros between them."""
    room, sizes = _padded(c), torch.tensor(_sizes(c), device=DEV)
    total = sum(room)
    starts = torch.tensor([0] + room[:-1], device=DEV).cumsum(0)
    at = torch.arange(total, device=DEV)
    of = torch.repeat_interleave(torch.arange(len(room), device=DEV),
                                 torch.tensor(room, device=DEV))
    on = (at - starts[of] < sizes[of]).float()
    p = _normal(g, total, std=0.02).mul_(on)
    S = dict(p=p.to(torch.float32 if c["weights"] == "f32" else torch.bfloat16),
             copy=p if c["weights"] == "copy" else None,
             g=_normal(g, total, std=1e-3).mul_(on).to(_type(c, "grads")), ms=None, vs=None)
    # states as some hundred steps leave them
    m, v = _normal(g, total, std=2e-4), _normal(g, total, std=1e-3).square_().add_(1e-8)
    m, v = m.mul_(on), v.mul_(on)
    if c["states"] == 8:
        S["ms"] = _blocks(m).abs().amax(1) / 448.0
        S["vs"] = _blocks(v).amax(1) / 57344.0
        m = (_blocks(m) / S["ms"][:, None]).view(-1).to(torch.float8_e4m3fn)
        v = (_blocks(v) / S["vs"][:, None]).view(-1).to(torch.float8_e5m2)
    return dict(S, m=m, v=v)


def prepare(case, seed):
    c, g = case, _gen(seed)
    S = dict(c=c)
    if c["kind"] in ("attn", "decode"):
        S.update(_attn_inputs(c, g))
    elif c["kind"] == "route":
        T, E = c["tokens"], c["experts"]
        S["x"] = _normal(g, T, E, std=2.0, dtype=_type(c))
        S["skip"] = ((torch.rand(T, generator=g, device=DEV) < c["skip"]).to(torch.uint8)
                     if c["skip"] else None)
        if c["mode"] == "train":
            S["dgate"] = _normal(g, T, c["topk"], std=1.0 / T)
    else:
        S.update(_adamw_inputs(c, g))
    if own:
        S.update(_handles(c, S))
    return S


# ------------------------------------------------- the framework's operators

def _empty_like_rows(x):
    """Rows of x's width without x's strides (a packed row's parts)."""
    return torch.empty(x.shape, dtype=x.dtype, device=DEV)


def _handles(c, S):
    """What a program keeps between calls: operands, plans, outputs, workspaces."""
    from paper_2303_07030_amd import nsd, operand, optim
    if c["kind"] in ("attn", "decode"):
        H, Hk, d, dv = c["heads"], c["kv"], c["d"], c["dv"]
        o = torch.empty(S["q"].shape[0], H * dv, dtype=S["q"].dtype, device=DEV)
        a = nsd.attn_desc(H, Hk, d, dv, S["q"], S["k"], S["v"], o, 1.0 / math.sqrt(d))
        out = dict(attn=a, o=o)
        if c["kind"] == "decode":
            n = nsd.nsd_attn_diff_decode_workspace_size(c["rows"], c["len"], a)
        else:
            nnz, train = S["col"].numel(), c["mode"] == "train"
            val = S["bias"] if c["bias"] else torch.zeros(nnz, device=DEV)
            A = operand.DeviceCsr(c["nq"], c["nk"], S["rowptr"], S["col"], val,
                                  build_csc=train, perm_plans=False,
                                  item_len=nsd.nsd_attn_item_len(nnz, a))
            n = nsd.nsd_attn_diff_workspace_size(A.desc, A.csc, a)
            out["A"] = A
            if train:
                out["stat"] = torch.empty(c["nq"], H, 4, device=DEV)
                if c["mask"] == "window":  # gradients of one projection, packed as it is
                    w = [t.shape[1] for t in (S["q"], S["k"], S["v"])]
                    out["grads"] = torch.empty(c["nq"], sum(w), dtype=o.dtype,
                                               device=DEV).split(w, 1)
                else:
                    out["grads"] = [_empty_like_rows(t) for t in (S["q"], S["k"], S["v"])]
                out["dlam"] = torch.empty(H, device=DEV)
                out["dbias"] = torch.empty(nnz, device=DEV) if c["bias"] else None
        return dict(out, ws=torch.empty(max(n, 256), dtype=torch.uint8, device=DEV))
    if c["kind"] == "route":
        T, E, k = c["tokens"], c["experts"], c["topk"]
        r = nsd.router_desc(E, k, S["x"], c["norm"])
        out = dict(router=r, col=torch.empty(T, k, dtype=torch.int32, device=DEV),
                   gate=torch.empty(T, k, device=DEV))
        if c["mode"] == "train":
            n = nsd.nsd_route_workspace_size(T, r)
            out.update(counts=torch.empty(E + 1, dtype=torch.int32, device=DEV),
                       loss=torch.empty(1, dtype=torch.float64, device=DEV),
                       dx=torch.empty_like(S["x"]),
                       ws=torch.empty(max(n, 256), dtype=torch.uint8, device=DEV))
        return out
    t = {x: None if S[x] is None else _tensors(c, S[x], BLOCK if x in ("ms", "vs") else 1)
         for x in ("p", "g", "copy", "m", "v", "ms", "vs")}
    return dict(opt=optim.AdamW(t["p"], t["g"], masters=t["copy"], state_bits=c["states"],
                                m=t["m"], v=t["v"], m_scale=t["ms"], v_scale=t["vs"],
                                weight_decay=0.01, step=99, **HYPER))


def _own(c, S):
    from paper_2303_07030_amd import nsd
    if c["kind"] == "decode":
        nsd.nsd_attn_diff_decode(c["rows"], S["rowptr"], S["col"], c["len"], S["attn"], S["q"],
                                 S["k"], S["v"], S["lam"], None, S["o"], S["ws"])
        return S["o"]
    if c["kind"] == "attn":
        A, a = S["A"], S["attn"]
        nsd.nsd_attn_diff(A.desc, a, S["q"], S["k"], S["v"], S["lam"], S["bias"], S["o"],
                          S.get("stat"), S["ws"])
        if c["mode"] == "fwd":
            return S["o"]
        nsd.nsd_attn_diff_vjp(A.desc, A.csc, a, S["q"], S["k"], S["v"], S["lam"], S["bias"],
                              S["stat"], S["dO"], *S["grads"], S["dlam"], S["dbias"], S["ws"])
        return dict(o=S["o"], dq=S["grads"][0], dk=S["grads"][1], dv=S["grads"][2],
                    dlam=S["dlam"], dbias=S["dbias"])
    if c["kind"] == "route":
        if c["mode"] == "fwd":
            nsd.nsd_route(c["tokens"], S["router"], S["x"], S["skip"], 0.0, S["col"], S["gate"],
                          None, None, None)
            return dict(col=S["col"], gate=S["gate"])
        nsd.nsd_route(c["tokens"], S["router"], S["x"], S["skip"], 0.01, S["col"], S["gate"],
                      S["counts"], S["loss"], S["ws"])
        nsd.nsd_route_vjp(c["tokens"], S["router"], S["x"], S["skip"], S["col"], S["gate"],
                          S["counts"], 0.01, 1.0, S["dgate"], S["dx"])
        return dict(col=S["col"], gate=S["gate"], counts=S["counts"], loss=S["loss"].float(),
                    dx=S["dx"])
    S["opt"].step()
    return {x: S[x] for x in ("p", "copy", "m", "v", "ms", "vs")}


# ------------------------------------------------------------ the plain forms

def _by_row(x, row, n, how):
    """Sums or maxima of x's leading entries by row."""
    out = torch.full((n,) + x.shape[1:], 0.0 if how == "sum" else -math.inf, device=DEV)
    if how == "sum":
        return out.index_add_(0, row, x)
    return out.scatter_reduce_(0, row.view(-1, 1, 1).expand_as(x), x, "amax")


def _plain_attn(c, S):
    H, Hk, d, dv = c["heads"], c["kv"], c["d"], c["dv"]
    row, col, T = S["row"], S["col"].long(), S["q"].dtype
    n, nk, grp, scale = S["q"].shape[0], S["k"].shape[0], H // Hk, 1.0 / math.sqrt(d)
    q = S["q"].float().view(n, H, 2, d)[row]
    k = S["k"].float().view(nk, Hk, 2, d)[col].repeat_interleave(grp, 1)
    v = S["v"].float().view(nk, Hk, dv)[col].repeat_interleave(grp, 1)
    s = (q * k).sum(-1) * scale
    if S["bias"] is not None:
        s = s + S["bias"][:, None, None]
    top = _by_row(s, row, n, "max")
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(s - top[row])
    z = _by_row(e, row, n, "sum")
    a = e / z[row].clamp_min_(1e-30)
    lam = S["lam"][:, None]
    w = a[..., 0:1] - lam * a[..., 1:2]
    o = _by_row(w * v, row, n, "sum").view(n, H * dv).to(T)
    if c.get("mode") != "train":
        return o
    go = S["dO"].float().view(n, H, dv)[row]
    t = (go * v).sum(-1, keepdim=True)
    D = _by_row(a * t, row, n, "sum")
    ds = a * (t - D[row])
    ds = torch.stack([ds[..., 0], -S["lam"] * ds[..., 1]], -1)
    dq = _by_row((ds * scale)[..., None] * k, row, n, "sum")
    dk = (ds * scale)[..., None] * q
    dk = dk.view(-1, Hk, grp, 2, d).sum(2)
    dv_ = (w * go).view(-1, Hk, grp, dv).sum(2)
    return dict(o=o, dq=dq.view(n, -1).to(T),
                dk=_by_row(dk, col, nk, "sum").view(nk, -1).to(T),
                dv=_by_row(dv_, col, nk, "sum").view(nk, -1).to(T), dlam=-D[..., 1].sum(0),
                dbias=None if S["bias"] is None else ds.sum((1, 2)))


def _plain_route(c, S):
    k, E = c["topk"], c["experts"]
    x = S["x"].float()
    e = torch.exp(x - x.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    col = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k].sort(dim=1)[0]
    gate = p.gather(1, col)
    total = gate.sum(1, keepdim=True)
    if c["norm"]:
        gate = gate / total
    on = torch.ones(x.shape[0], 1, device=DEV) if S["skip"] is None else 1.0 - S["skip"][:, None]
    gate = gate * on
    col = torch.where(on > 0, col, torch.arange(k, device=DEV))
    if c["mode"] == "fwd":
        return dict(col=col.int(), gate=gate)
    n = torch.zeros(E, device=DEV, dtype=torch.int32)
    n.index_add_(0, col.reshape(-1), on.int().expand_as(col).reshape(-1))
    routed = on.sum()
    f = n / n.sum().clamp_min(1)
    loss = 0.01 * E * (f * (p * on).sum(0)).sum() / routed.clamp_min(1)
    u = (0.01 * E * f / routed.clamp_min(1)).expand_as(p)
    dg = S["dgate"]
    if c["norm"]:
        back = gate * (dg - (gate * dg).sum(1, keepdim=True))
    else:
        u = u.scatter_add(1, col, dg)
        back = torch.zeros_like(dg)
    dx = p * (u - (p * u).sum(1, keepdim=True))
    dx = dx.scatter_add(1, col, back) * on
    return dict(col=col.int(), gate=gate, counts=torch.cat([n, routed.int().view(1)]),
                loss=loss.view(1), dx=dx.to(S["x"].dtype))


def _blocks(x):
    """x as rows of the values that share a scale."""
    return x.view(-1, BLOCK)


def _mix(x):
    """32 mixed bits of each 32-bit number (held in 64)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _noise(c, step):
    """The 32 bits that the rounding of every value draws: by the step, its
    tensor's number and its place in it."""
    room = torch.tensor(_padded(c), device=DEV)
    key = _mix((torch.arange(room.numel(), device=DEV) + step * 0x9E3779B1) & 0xFFFFFFFF)
    start = torch.cumsum(room, 0) - room
    n = sum(_padded(c))
    at = torch.arange(n, device=DEV) - torch.repeat_interleave(start, room, output_size=n)
    key = torch.repeat_interleave(key, room, output_size=n)
    return _mix((at * 0x9E3779B1 + key) & 0xFFFFFFFF)


def _to_eight(x, bits, T):
    """x to 8 bits, a scale for every block: rounded up or down at random so
    that the mean is kept; `bits` are 16 random bits for every value."""
    mant, low, sub, top = ((3, -6, 512.0, 448.0) if T == torch.float8_e4m3fn
                           else (2, -14, 65536.0, 57344.0))
    s = _blocks(x).abs().amax(1) * (1.0 / top)
    s = torch.where(s < 2.0 ** -126, 0.0, s)
    inv = torch.where(s > 0, 1.0 / s, 0.0)
    y = (_blocks(x).abs() * inv[:, None]).view(-1)
    drop = 23 - mant
    raw = y.view(torch.int32) + ((bits << (drop - 16)) + (1 << (drop - 17))).int()
    code = (raw >> drop) - ((126 + low) << mant)
    small = torch.floor(y * sub + (bits.float() + 0.5) * 2.0 ** -16).int()
    code = torch.where(y < 2.0 ** low, small, code)
    code = code.clamp_max(0x7E if mant == 3 else 0x7B)
    if mant == 2:  # a second moment that is not zero stays so
        code = torch.where(y > 0, code.clamp_min(1), code)
    else:
        code = code | ((x.view(torch.int32) >> 31) & 0x80)
    return code.to(torch.uint8).view(T), s


def _from_eight(x, s):
    return (_blocks(x.float()) * s[:, None]).view(-1)


def _plain_adamw(c, S):
    t = S["t"] = S.get("t", 99) + 1
    b1, b2, lr = HYPER["beta1"], HYPER["beta2"], HYPER["lr"]
    eight = c["states"] == 8
    g = S["g"].float()
    m = _from_eight(S["m"], S["ms"]) if eight else S["m"]
    v = _from_eight(S["v"], S["vs"]) if eight else S["v"]
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * (1.0 - b2)) * g
    w = S["p"].float() if S["copy"] is None else S["copy"]
    den = v.sqrt() * (1.0 / math.sqrt(1.0 - b2 ** t)) + HYPER["eps"]
    w = w * (1.0 - lr * 0.01) - (m / den) * (lr / (1.0 - b1 ** t))
    bits = _noise(c, t) if eight or c["weights"] == "bf16" else None
    if eight:
        m, s = _to_eight(m, bits & 0xFFFF, S["m"].dtype)
        S["ms"].copy_(s)
        v, s = _to_eight(v, bits >> 16, S["v"].dtype)
        S["vs"].copy_(s)
    S["m"].copy_(m)
    S["v"].copy_(v)
    if c["weights"] == "bf16":  # rounded up or down at random, too
        up = (_mix(bits ^ 0x9E3779B1) & 0xFFFF).int()
        w = ((w.view(torch.int32) + up) & -65536).view(torch.float32)
    S["p"].copy_(w)
    if S["copy"] is not None:
        S["copy"].copy_(w)
    return {x: S[x] for x in ("p", "copy", "m", "v", "ms", "vs")}


def run(state):
    c = state["c"]
    if own:
        return _own(c, state)
    if c["kind"] in ("attn", "decode"):
        return _plain_attn(c, state)
    return _plain_route(c, state) if c["kind"] == "route" else _plain_adamw(c, state)


# ------------------------------------------------------- work and definition

def work(case):
    c = case
    if c["kind"] in ("attn", "decode"):
        es = 4 if c["dtype"] == "f32" else 2
        H, Hk, d, dv, nnz = c["heads"], c["kv"], c["d"], c["dv"], _entries(c)
        nq = c["rows"] if c["kind"] == "decode" else c["nq"]
        nk = nnz if c["kind"] == "decode" else c["nk"]
        rows = es * (nq * H * 2 * d + nk * Hk * (2 * d + dv))
        b = 1 if c.get("bias") else 0
        if c.get("mode") != "train":
            return dict(bytes=rows + es * nq * H * dv + 4 * (1 + b) * nnz,
                        flops=nnz * H * (4 * d + 2 * dv))
        # q, k, v, dO and the pattern in; o and every gradient out
        return dict(bytes=2 * rows + 2 * es * nq * H * dv + 4 * (1 + 2 * b) * nnz,
                    flops=nnz * H * (12 * d + 6 * dv))
    if c["kind"] == "route":
        T, E, k = c["tokens"], c["experts"], c["topk"]
        es = 4 if c["dtype"] == "f32" else 2
        if c["mode"] == "fwd":
            return dict(bytes=T * (E * es + 8 * k), flops=4 * T * E)
        return dict(bytes=T * (2 * E * es + 12 * k), flops=10 * T * E)
    per = {"f32": 8, "bf16": 4, "copy": 10}[c["weights"]]
    per += 4 if c["grads"] == "f32" else 2
    per += 16 if c["states"] == 32 else 4 + 16 / BLOCK
    return dict(bytes=per * sum(_sizes(c)), flops=14 * sum(_sizes(c)))


def _exact_attn(c, S):
    """Head by head from the definition: the softmax of the keys that are
    stored and not masked; the gradients by differentiating it."""
    H, Hk, d, dv = c["heads"], c["kv"], c["d"], c["dv"]
    n, nk, train = S["q"].shape[0], S["k"].shape[0], c.get("mode") == "train"
    row, col = S["row"], S["col"].long()
    at = torch.arange(row.numel(), device=DEV)
    if S["bias"] is not None:
        at = torch.nonzero(S["bias"] > -math.inf).view(-1)
        row, col = row[at], col[at]
    o = torch.zeros(n, H, dv, dtype=torch.float64, device=DEV)
    dq = torch.zeros(n, H, 2 * d, dtype=torch.float64, device=DEV)
    dk = torch.zeros(nk, Hk, 2 * d, dtype=torch.float64, device=DEV)
    dvv = torch.zeros(nk, Hk, dv, dtype=torch.float64, device=DEV)
    dlam = torch.zeros(H, dtype=torch.float64, device=DEV)
    dbias = torch.zeros(S["row"].numel(), dtype=torch.float64, device=DEV)

    def softmax(s):
        m = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
        m = m.index_reduce(0, row, s.detach(), "amax")
        x = torch.exp(s - m[row])
        z = torch.zeros(n, dtype=torch.float64, device=DEV).index_add(0, row, x)
        return x / z[row]

    for h in range(H):
        g = h // (H // Hk)
        q = S["q"][:, h * 2 * d:(h + 1) * 2 * d].double()
        k = S["k"][:, g * 2 * d:(g + 1) * 2 * d].double()
        v = S["v"][:, g * dv:(g + 1) * dv].double()
        lam = S["lam"][h].double()
        b = torch.zeros(row.numel(), dtype=torch.float64, device=DEV) if S["bias"] is None \
            else S["bias"][at].double()
        wrt = [q, k, v, lam, b]
        with torch.set_grad_enabled(train):
            if train:
                [t.requires_grad_() for t in wrt]
            qr, kr = q[row], k[col]
            s1 = (qr[:, :d] * kr[:, :d]).sum(1) / math.sqrt(d) + b
            s2 = (qr[:, d:] * kr[:, d:]).sum(1) / math.sqrt(d) + b
            w = softmax(s1) - lam * softmax(s2)
            oh = torch.zeros(n, dv, dtype=torch.float64, device=DEV)
            oh = oh.index_add(0, row, w[:, None] * v[col])
        o[:, h] = oh.detach()
        if train:
            up = S["dO"][:, h * dv:(h + 1) * dv].double()
            gq, gk, gv, gl, gb = torch.autograd.grad(oh, wrt, up)
            dq[:, h] = gq
            dk[:, g] += gk
            dvv[:, g] += gv
            dlam[h] = gl
            dbias.index_add_(0, at, gb)
    if not train:
        return o.view(n, -1)
    return dict(o=o.view(n, -1), dq=dq.view(n, -1), dk=dk.view(nk, -1), dv=dvv.view(nk, -1),
                dlam=dlam, dbias=None if S["bias"] is None else dbias)


def _exact_route(c, S):
    k, E = c["topk"], c["experts"]
    x = S["x"].double().requires_grad_(c["mode"] == "train")
    on = torch.ones(x.shape[0], dtype=torch.bool, device=DEV) if S["skip"] is None \
        else S["skip"] == 0
    # the k largest, ties to the lowest expert: order by value, then by index
    key = x.detach() - 0.0
    rank = torch.argsort(-key, dim=1, stable=True)
    chosen = torch.zeros_like(key).scatter_(1, rank[:, :k], 1.0)
    col = torch.nonzero(chosen)[:, 1].view(-1, k)
    p = torch.softmax(x, 1)
    gate = p.gather(1, col)
    if c["norm"]:
        gate = torch.softmax(x.gather(1, col), 1)
    gate = gate * on[:, None]
    shown = torch.where(on[:, None], col, torch.arange(k, device=DEV)).int()
    if c["mode"] == "fwd":
        return dict(col=shown, gate=gate.detach())
    n = chosen[on].sum(0)
    routed = on.sum()
    loss = 0.01 * E * ((n / n.sum().clamp_min(1)) * p[on].sum(0)).sum() / routed.clamp_min(1)
    dx, = torch.autograd.grad([loss, gate], x, [torch.ones_like(loss), S["dgate"].double()])
    return dict(col=shown, gate=gate.detach(), counts=torch.cat([n, routed.view(1)]).int(),
                loss=loss.detach().view(1), dx=dx)


def _exact_adamw(c, S):
    b1, b2, lr, t = HYPER["beta1"], HYPER["beta2"], HYPER["lr"], 100
    g, m, v = (S[x].double() for x in ("g", "m", "v"))
    if c["states"] == 8:
        m, v = (torch.repeat_interleave(S[s].double(), BLOCK) * x
                for x, s in ((m, "ms"), (v, "vs")))
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
    w = (S["p"] if S["copy"] is None else S["copy"]).double()
    w = w - lr * 0.01 * w - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t))
                                                         + HYPER["eps"])
    out = dict(p=w, copy=None if S["copy"] is None else w, m=m, v=v, ms=None, vs=None)
    if c["states"] == 8:  # the scales are defined, the codes rounded at random
        out.update(m=None, v=None, ms=_blocks(m).abs().amax(1) / 448,
                   vs=_blocks(v).amax(1) / 57344)
    return out


def exact(case, seed):
    S = prepare(case, seed)
    if case["kind"] in ("attn", "decode"):
        return _exact_attn(case, S)
    return _exact_route(case, S) if case["kind"] == "route" else _exact_adamw(case, S)
