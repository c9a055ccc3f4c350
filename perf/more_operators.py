"""Workloads of the operators around attention and the optimizer: token rows,
norms and rotation of queries and keys, attention with a decay, and the norm of
all gradients.

Each case is one call, or the calls of one training step, on data already in
HBM.  With `own` the operators are those of this package; without it they are
computed in their plain form, by elementary torch operations in 32 bits.

embed   rows of a table by token, and the table's gradient
qk      norm and rotation of every head's query and key; with the gradient in
        training; in serving the keys and values go to slots of a cache
decay   linear attention with a decay for each head over packed sequences; with
        the gradient in training
step    the same for one new token per sequence, the states held in slots
norm    the norm of a model's gradients and the factor that clips them, for an
        optimizer that takes it, or applied in place

All inputs are drawn on the GPU from a seed.
"""
import math
import random

import torch

own = False
DEV = "cuda"
CHUNK = 128       # tokens that the plain form of the decay takes at once


# ------------------------------------------------------------------ cases

def listed():
    return [
        # the tokens of one serving step: all latency
        dict(name="embed_16", kind="embed", mode="fwd", tokens=16, vocab=32_000, width=1024,
             table="bf16", rows="bf16", grad="bf16", skip=0.0, add=False),
        # a training step's batch; words as frequent as in text
        dict(name="embed_32k_train", kind="embed", mode="train", tokens=32_768, vocab=50_000,
             width=1024, table="bf16", rows="bf16", grad="bf16", skip=0.0, add=False),
        # odd sizes, padded tokens, added to the gradient that a tied head left
        dict(name="embed_odd_10k", kind="embed", mode="train", tokens=10_007, vocab=5_003,
             width=333, table="f32", rows="f32", grad="f32", skip=0.1, add=True),
        # eight chats' next tokens on their way into the cache
        dict(name="qk_append_8", kind="qk", mode="append", tokens=8, heads=16, kv=4, d=64, rot=64,
             pairs="half", far=4096, slots=65_536, dv=128, dtype="bf16", norm=True),
        # a training step over 16 thousand tokens
        dict(name="qk_train_16k", kind="qk", mode="train", tokens=16_384, heads=32, kv=8, d=128,
             rot=128, pairs="half", far=8192, slots=0, dv=0, dtype="bf16", norm=True),
        # odd sizes, a part of each head rotated, pairs side by side, far positions
        dict(name="qk_odd_10k", kind="qk", mode="train", tokens=10_007, heads=6, kv=3, d=40,
             rot=24, pairs="next", far=1_000_000, slots=0, dv=0, dtype="f32", norm=True),
        # a serving step of sixty-four sequences: the states are read and written
        dict(name="step_64", kind="step", rows=64, slots=100, heads=16, kv=16, d=64, dv=128,
             dtype="bf16"),
        # a long prompt, one sequence
        dict(name="decay_prompt_64k", kind="decay", mode="fwd", seqs=1, tokens=65_536, heads=8,
             kv=8, d=128, dv=128, dtype="bf16", start=False),
        # a training step over packed documents, one of them of a single token
        dict(name="decay_train_32k", kind="decay", mode="train", seqs=12, tokens=32_768, heads=16,
             kv=16, d=64, dv=128, dtype="bf16", start=False),
        # odd sizes in 32 bits, heads that share keys, sequences that go on from a state
        dict(name="decay_odd_5k", kind="decay", mode="train", seqs=7, tokens=5_003, heads=6, kv=3,
             d=40, dv=72, dtype="f32", start=True),
        # the gradients of a model of many small tensors
        dict(name="norm_300_small", kind="norm", tensors=300, total=2_000_000, grads="f32",
             order=2, clip=False),
        # those of a large model, clipped in place
        dict(name="clip_200m", kind="norm", tensors=24, total=200_000_000, grads="bf16", order=2,
             clip=True),
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8, 16])
    heads = kv * rng.choice([1, 1, 2, 4])
    if rng.random() < 0.5:
        d = rng.choice([16, 32, 64, 128])
        return dict(heads=heads, kv=kv, d=d, dv=rng.choice([d, min(2 * d, 128)]))
    return dict(heads=heads, kv=kv, d=_log(rng, 5, 128), dv=_log(rng, 5, 200))


def draw(rng):
    kind = rng.choice(["embed", "embed", "qk", "qk", "decay", "decay", "step", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "embed":
        width = _log(rng, 16, 2048)
        vocab = min(_log(rng, 100, 60_000), 80_000_000 // width)
        tokens = min(_log(rng, 1, 100_000), 60_000_000 // width)
        return dict(kind=kind, mode=rng.choice(["train", "train", "fwd"]), tokens=tokens,
                    vocab=vocab, width=width, table=dtype, rows=rng.choice([dtype, "bf16"]),
                    grad=rng.choice([dtype, "f32"]), skip=rng.choice([0.0, 0.1]),
                    add=rng.random() < 0.5)
    if kind == "qk":
        h = _heads(rng)
        rot = rng.choice([h["d"] // 2 * 2, h["d"] // 4 * 2])
        mode = rng.choice(["train", "train", "append"])
        most = 60_000_000 // ((h["heads"] + h["kv"]) * h["d"])
        tokens = _log(rng, 1, 64) if mode == "append" else min(_log(rng, 1, 40_000), most)
        return dict(h, kind=kind, mode=mode, tokens=tokens, rot=rot,
                    pairs=rng.choice(["half", "next"]), far=_log(rng, 100, 1_000_000),
                    slots=_log(rng, 200, 100_000) if mode == "append" else 0,
                    dv=h["dv"] if mode == "append" else 0, dtype=dtype, norm=rng.random() < 0.7)
    if kind == "step":
        h = _heads(rng)
        rows = min(_log(rng, 1, 300), max(1, 40_000_000 // (h["heads"] * h["d"] * h["dv"])))
        return dict(h, kind=kind, rows=rows, slots=rows + rng.randint(0, 50), dtype=dtype)
    if kind == "decay":
        h = _heads(rng)
        seqs = _log(rng, 1, 40)
        train = rng.random() < 0.6
        most = (4e9 if train else 1e10) / (h["heads"] * h["d"] * h["dv"])
        tokens = min(_log(rng, 1, 60_000), int(most),
                     25_000_000 // (h["heads"] * max(h["d"], h["dv"])))
        return dict(h, kind=kind, mode="train" if train else "fwd", seqs=seqs,
                    tokens=max(1, tokens), dtype=dtype, start=rng.random() < 0.5)
    return dict(kind=kind, tensors=_log(rng, 1, 300), total=_log(rng, 10_000, 140_000_000),
                grads=rng.choice(["f32", "bf16", "bf16"]), order=rng.choice([2, 2, 0]),
                clip=rng.random() < 0.5)


# ----------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).mul_(std).to(dtype)


def _lens(c):
    """Lengths of packed sequences: ragged, one of a single token, one empty."""
    r = random.Random(c["seqs"] * 1_000_003 + c["tokens"])
    n, left = c["seqs"], c["tokens"]
    if n == 1:
        return [left]
    w = [0.3 + r.random() for _ in range(n)]
    if n > 3:
        w[1], w[2] = 0.0, 0.0
    lens = [int(left * x / sum(w)) for x in w]
    if n > 3 and sum(lens) < left:
        lens[1] = 1
    lens[0] += left - sum(lens)
    return lens


def _sizes(c):
    """Lengths of a model's tensors: a few take most of the weights, none of
    them of a round size, the smallest of one value."""
    n, total = c["tensors"], c["total"]
    w = [1.0 / (i + 1) ** 0.7 for i in range(n)]
    sizes = [max(1, int(total * x / sum(w))) for x in w]
    if n > 2:
        sizes[-1], sizes[-2] = 1, 3
    return sizes


def _embed_inputs(c, g):
    n, V, w = c["tokens"], c["vocab"], c["width"]
    # words by their frequency in text (the k-th as 1 / k), at random places in the table
    p = 1.0 / torch.arange(1, V + 1, device=DEV, dtype=torch.float64)
    cdf = torch.cumsum(p / p.sum(), 0)
    at = torch.searchsorted(cdf, torch.rand(n, generator=g, device=DEV, dtype=torch.float64))
    ids = torch.randperm(V, generator=g, device=DEV)[at.clamp_(max=V - 1)].int()
    if c["skip"]:  # padding
        ids.masked_fill_(torch.rand(n, generator=g, device=DEV) < c["skip"], -1)
    S = dict(ids=ids, W=_normal(g, V, w, std=0.02, dtype=_type(c["table"])), scale=math.sqrt(w))
    if c["mode"] == "train":
        S["dout"] = _normal(g, n, w, dtype=_type(c["rows"]))
        S["dW"] = (_normal(g, V, w, dtype=_type(c["grad"])) if c["add"]
                   else torch.empty(V, w, dtype=_type(c["grad"]), device=DEV))
    return S


def _qk_inputs(c, g):
    n, H, Hk, d, T = c["tokens"], c["heads"], c["kv"], c["d"], _type(c["dtype"])
    wide = _normal(g, n, H * d + Hk * d + Hk * c["dv"], dtype=T)  # one projection's output
    q, k, v = wide.split([H * d, Hk * d, Hk * c["dv"]], 1)
    S = dict(q=q, k=k, v=v, wq=None, wk=None, eps=1e-6)
    if c["norm"]:
        S["wq"], S["wk"] = (1.0 + _normal(g, d, std=0.1) for _ in range(2))
    S["pos"] = torch.randint(c["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
    r = c["rot"]
    S["freq"] = 10_000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / max(r, 1))
    if c["mode"] == "append":  # rows of a cache, one token not kept
        S["slot"] = torch.randperm(c["slots"], generator=g, device=DEV)[:n].int()
        if n > 2:
            S["slot"][1] = -1
        S["kc"] = _normal(g, c["slots"], Hk * d, dtype=T)
        S["vc"] = _normal(g, c["slots"], Hk * c["dv"], dtype=T)
    else:
        S["dq"], S["dk"] = _normal(g, n, H * d, dtype=T), _normal(g, n, Hk * d, dtype=T)
    return S


def _decay_inputs(c, g):
    H, Hk, d, dv, T = c["heads"], c["kv"], c["d"], c["dv"], _type(c["dtype"])
    n = c["rows"] if c["kind"] == "step" else c["tokens"]
    S = dict(q=_normal(g, n, H * d, dtype=T), k=_normal(g, n, Hk * d, dtype=T),
             v=_normal(g, n, Hk * dv, dtype=T), scale=1.0 / math.sqrt(d))
    # heads that remember from about two tokens to some thousand
    S["decay"] = -(2.0 ** -torch.linspace(1.0, 10.0, H, device=DEV))
    if c["kind"] == "step":
        S["state"] = _normal(g, c["slots"], H, d, dv)
        S["slot"] = torch.randperm(c["slots"], generator=g, device=DEV)[:n].int()
        return S
    lens = torch.tensor([0] + _lens(c), device=DEV)
    S["seqptr"] = torch.cumsum(lens, 0).int()
    S["longest"] = max(_lens(c))
    S["s0"] = _normal(g, c["seqs"], H, d, dv) if c["start"] else None
    if c["mode"] == "train":
        S["do"] = _normal(g, n, H * dv, dtype=T)
        S["ds1"] = _normal(g, c["seqs"], H, d, dv) if c["start"] else None
    return S


def _norm_inputs(c, g):
    sizes = _sizes(c)
    flat = _normal(g, sum(sizes), std=1e-3, dtype=_type(c["grads"]))
    S = dict(flat=flat, grads=list(flat.split(sizes)), max_norm=1.0, turn=0)
    # the loss's scale is taken out on one pass and put back on the next, so that
    # the gradients are changed by every pass and stay what they are
    S["factors"] = [torch.full((1,), f, device=DEV) for f in (0.125, 8.0)]
    return S


def prepare(case, seed):
    c, g = case, _gen(seed)
    make = dict(embed=_embed_inputs, qk=_qk_inputs, decay=_decay_inputs, step=_decay_inputs,
                norm=_norm_inputs)[c["kind"]]
    S = dict(make(c, g), c=c)
    if own:
        S.update(_handles(c, S))
    return S


# ------------------------------------------------- the framework's operators

def _bytes(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)


def _rows_like(t):
    """Rows of t's width without t's strides (a packed row's parts)."""
    return torch.empty(t.shape, dtype=t.dtype, device=DEV)


def _handles(c, S):
    """What a program keeps between calls: shapes, plans, outputs, workspaces."""
    from paper_2303_07030_amd import nsd, optim
    if c["kind"] == "embed":
        out = torch.empty(c["tokens"], c["width"], dtype=_type(c["rows"]), device=DEV)
        e = nsd.embed_desc(S["W"], out, S["scale"], grad=S.get("dW"))
        ws = _bytes(nsd.nsd_embed_vjp_workspace_size(c["tokens"], e)) if "dW" in S else None
        return dict(desc=e, out=out, ws=ws)
    if c["kind"] == "qk":
        qo = _rows_like(S["q"])
        ko = S["kc"] if c["mode"] == "append" else _rows_like(S["k"])
        a = nsd.qk_desc(c["heads"], c["kv"], c["d"], S["q"], S["k"], qo, ko, rot=c["rot"],
                        interleaved=c["pairs"] == "next", norm=c["norm"], eps=S["eps"])
        out = dict(desc=a, qo=qo, ko=ko)
        if c["mode"] == "train":
            out["ws"] = _bytes(nsd.nsd_qk_rotate_vjp_workspace_size(c["tokens"], a))
            # gradients of one projection, packed as it is
            w = [S["q"].shape[1], S["k"].shape[1]]
            out["gq"], out["gk"] = torch.empty(c["tokens"], sum(w), dtype=qo.dtype,
                                               device=DEV).split(w, 1)
            if c["norm"]:
                out["gwq"], out["gwk"] = (torch.empty(c["d"], device=DEV) for _ in range(2))
        return out
    if c["kind"] in ("decay", "step"):
        o = torch.empty(S["q"].shape[0], c["heads"] * c["dv"], dtype=S["q"].dtype, device=DEV)
        a = nsd.decay_desc(c["heads"], c["kv"], c["d"], c["dv"], S["q"], S["k"], S["v"], o,
                           S["scale"])
        if c["kind"] == "step":
            return dict(desc=a, o=o)
        train = c["mode"] == "train"
        n = nsd.nsd_attn_decay_workspace_size(c["tokens"], c["seqs"], S["longest"], a, train)
        state = (c["seqs"], c["heads"], c["d"], c["dv"])
        out = dict(desc=a, o=o, s1=torch.empty(state, device=DEV), ws=_bytes(n))
        if train:
            out.update(gq=_rows_like(S["q"]), gk=_rows_like(S["k"]), gv=_rows_like(S["v"]),
                       gdecay=torch.empty(c["heads"], device=DEV),
                       gs0=torch.empty(state, device=DEV) if c["start"] else None)
        return out
    return dict(plan=optim.GradNorm(S["grads"], max_norm=S["max_norm"],
                                    order=math.inf if c["order"] == 0 else c["order"]))


def _own(c, S):
    from paper_2303_07030_amd import nsd
    if c["kind"] == "embed":
        nsd.nsd_embed(c["tokens"], S["desc"], S["ids"], S["W"], S["out"])
        if c["mode"] == "fwd":
            return S["out"]
        nsd.nsd_embed_vjp(c["tokens"], S["desc"], S["ids"], S["dout"], c["add"], S["dW"], S["ws"])
        return dict(out=S["out"], dW=S["dW"])
    if c["kind"] == "qk":
        if c["mode"] == "append":
            nsd.nsd_qk_append(c["tokens"], S["desc"], S["q"], S["k"], S["v"], S["wq"], S["wk"],
                              S["pos"], S["freq"], S["slot"], c["slots"], S["qo"], S["kc"],
                              S["vc"])
            return dict(q=S["qo"], k=S["kc"], v=S["vc"])
        nsd.nsd_qk_rotate(c["tokens"], S["desc"], S["q"], S["k"], S["wq"], S["wk"], S["pos"],
                          S["freq"], S["qo"], S["ko"])
        gwq, gwk = S.get("gwq"), S.get("gwk")
        nsd.nsd_qk_rotate_vjp(c["tokens"], S["desc"], S["q"], S["k"], S["wq"], S["wk"], S["pos"],
                              S["freq"], S["dq"], S["dk"], S["gq"], S["gk"], gwq, gwk, S["ws"])
        return dict(q=S["qo"], k=S["ko"], dq=S["gq"], dk=S["gk"], dwq=gwq, dwk=gwk)
    if c["kind"] == "step":
        nsd.nsd_attn_decay_step(c["rows"], S["slot"], c["slots"], S["desc"], S["q"], S["k"],
                                S["v"], S["decay"], S["state"], S["o"])
        return dict(o=S["o"], state=S["state"])
    if c["kind"] == "decay":
        args = (c["tokens"], c["seqs"], S["seqptr"], S["longest"], S["desc"], S["q"], S["k"],
                S["v"], S["decay"], S["s0"])
        nsd.nsd_attn_decay(*args, S["o"], S["s1"], S["ws"])
        if c["mode"] == "fwd":
            return dict(o=S["o"], s1=S["s1"])
        nsd.nsd_attn_decay_vjp(*args, S["do"], S["ds1"], S["gq"], S["gk"], S["gv"], S["gdecay"],
                               S["gs0"], S["ws"])
        return dict(o=S["o"], s1=S["s1"], dq=S["gq"], dk=S["gk"], dv=S["gv"], ddecay=S["gdecay"],
                    ds0=S["gs0"])
    p = S["plan"]
    if not c["clip"]:
        p.measure()
        return dict(norm=p.norm, scale=p.scale, norms=p.norms)
    p.measure(grad_scale=_factor(S))
    p.clip()
    return dict(norm=p.norm, scale=p.scale, norms=p.norms, grads=S["flat"])


# ------------------------------------------------------------ the plain forms

def _plain_embed(c, S):
    keep = S["ids"] >= 0
    at = S["ids"].clamp_min(0).long()
    out = (S["W"][at].float() * S["scale"] * keep[:, None]).to(_type(c["rows"]))
    if c["mode"] == "fwd":
        return out
    g = torch.zeros(c["vocab"], c["width"], device=DEV)
    g.index_add_(0, at, S["dout"].float() * (S["scale"] * keep[:, None]))
    S["dW"].copy_(S["dW"].float() + g if c["add"] else g)
    return dict(out=out, dW=S["dW"])


def _rotated(x, c, cos, sin):
    """The first `rot` values of the last dimension, rotated in pairs."""
    r = c["rot"]
    if c["pairs"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([y, x[..., r:]], -1)


def _plain_qk(c, S):
    n, d, T = c["tokens"], c["d"], S["q"].dtype
    angle = S["pos"].double()[:, None] * S["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = {}
    for x, w, g, name in ((S["q"], S["wq"], S.get("dq"), "q"), (S["k"], S["wk"], S.get("dk"), "k")):
        x = x.float().reshape(n, -1, d)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + S["eps"]) if c["norm"] else 1.0
        u = x * r
        y = u * w if c["norm"] else u
        out[name] = _rotated(y, c, cos, sin).reshape(n, -1).to(T)
        if g is not None:
            g = _rotated(g.float().view(n, -1, d), c, cos, -sin)
            if c["norm"]:
                out["dw" + name] = (g * u).sum((0, 1))
                g = g * w
                g = r * (g - u * (g * u).mean(-1, keepdim=True))
            out["d" + name] = g.reshape(n, -1).to(T)
    if c["mode"] == "append":
        on = S["slot"] >= 0
        at = S["slot"][on].long()
        S["kc"][at] = out["k"][on]
        S["vc"][at] = S["v"][on]
        return dict(q=out["q"], k=S["kc"], v=S["vc"])
    return out


def _powers(decay, n):
    """exp(decay n) for whole n >= 0, 0 for n < 0: [heads, *n.shape]."""
    e = torch.exp(decay.view(-1, *[1] * n.dim()) * n.clamp_min(0))
    return torch.where(n >= 0, e, torch.zeros_like(e))


def _chunks(q, k, v, decay, s0, lens, scale):
    """Outputs and last states of padded sequences [seqs, n, heads, *], n whole
    chunks: within a chunk every pair of tokens, between chunks their states."""
    B, n, H, d = q.shape
    dv, C = v.shape[-1], CHUNK
    nc = n // C
    q, k, v = (x.view(B, nc, C, H, -1).permute(0, 3, 1, 2, 4) for x in (q * scale, k, v))
    i = torch.arange(C, device=DEV)
    j = torch.arange(nc, device=DEV)
    near = _powers(decay, i[:, None] - i)[:, None]
    o = (q @ k.transpose(-1, -2) * near) @ v
    kv = (k * _powers(decay, C - 1 - i)[:, None, :, None]).transpose(-1, -2) @ v
    far = _powers(decay, (j[:, None] - 1 - j) * C)
    state = (far @ kv.reshape(B, H, nc, d * dv)).view(B, H, nc, d, dv)
    if s0 is not None:
        state = state + _powers(decay, j * C)[:, :, None, None] * s0[:, :, None]
    o = o + (q * _powers(decay, i + 1)[:, None, :, None]) @ state
    # the state after each sequence's own last token
    t = torch.arange(n, device=DEV)
    w = _powers(decay, lens[:, None] - 1 - t).transpose(0, 1).view(B, H, nc, C, 1)
    last = ((k * w).flatten(2, 3)).transpose(-1, -2) @ v.flatten(2, 3)
    if s0 is not None:
        last = last + _powers(decay, lens).t()[:, :, None, None] * s0
    return o.permute(0, 2, 3, 1, 4).reshape(B, n, H * dv), last


def _plain_decay(c, S):
    H, Hk, d, dv, T = c["heads"], c["kv"], c["d"], c["dv"], S["q"].dtype
    lens = S["seqptr"].diff()
    n = -(-S["longest"] // CHUNK) * CHUNK
    t = torch.arange(n, device=DEV)
    on = t < lens[:, None]
    at = (S["seqptr"][:-1, None] + t)[on]

    def padded(x, heads):
        y = torch.zeros(c["seqs"], n, x.shape[1], device=DEV)
        y[on] = x[at].float()
        return y.view(c["seqs"], n, heads, -1)

    def unpadded(x):
        return x.reshape(c["seqs"], n, -1)[on].to(T)

    train, grp = c["mode"] == "train", H // Hk
    q, k, v = padded(S["q"], H), padded(S["k"], Hk), padded(S["v"], Hk)
    wrt = [q, k, v, S["decay"].clone()] + ([S["s0"].clone()] if c["start"] else [])
    with torch.set_grad_enabled(train):
        for x in wrt:
            x.requires_grad_(train)
        o, s1 = _chunks(q, k.repeat_interleave(grp, 2), v.repeat_interleave(grp, 2), wrt[3],
                        wrt[4] if c["start"] else None, lens, S["scale"])
    out = dict(o=unpadded(o.detach()), s1=s1.detach())
    if train:
        up = padded(S["do"], 1).view(o.shape)
        ends, ups = ([o, s1], [up, S["ds1"]]) if c["start"] else ([o], [up])
        g = torch.autograd.grad(ends, wrt, ups)
        out.update(dq=unpadded(g[0]), dk=unpadded(g[1]), dv=unpadded(g[2]), ddecay=g[3],
                   ds0=g[4] if c["start"] else None)
    return out


def _plain_step(c, S):
    H, Hk, d, dv, n = c["heads"], c["kv"], c["d"], c["dv"], c["rows"]
    at = S["slot"].long()
    q = S["q"].float().view(n, H, d, 1)
    k = S["k"].float().view(n, Hk, d, 1).repeat_interleave(H // Hk, 1)
    v = S["v"].float().view(n, Hk, 1, dv).repeat_interleave(H // Hk, 1)
    s = S["state"][at] * torch.exp(S["decay"]).view(H, 1, 1) + k * v
    S["state"][at] = s
    o = (q * s).sum(2) * S["scale"]
    return dict(o=o.view(n, H * dv).to(S["q"].dtype), state=S["state"])


def _factor(S):
    S["turn"] += 1
    return S["factors"][(S["turn"] - 1) % 2]


def _plain_norm(c, S):
    f = _factor(S) if c["clip"] else None
    if c["order"] == 2:  # in 64 bits: squares of what 32 bits hold, sums of millions
        norms = torch.stack([t.double().square().sum() for t in S["grads"]]).sqrt()
    else:
        norms = torch.stack([t.abs().amax().double() for t in S["grads"]])
    if f is not None:
        norms = norms * f.abs()
    norm = (norms.square().sum().sqrt() if c["order"] == 2 else norms.amax()).view(1)
    scale = (S["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    scale = (scale * f if f is not None else scale).float()
    out = dict(norm=norm, scale=scale, norms=norms)
    if c["clip"]:
        S["flat"].copy_(S["flat"].float() * scale)
        out["grads"] = S["flat"]
    return out


def run(state):
    c = state["c"]
    if own:
        return _own(c, state)
    return dict(embed=_plain_embed, qk=_plain_qk, decay=_plain_decay, step=_plain_step,
                norm=_plain_norm)[c["kind"]](c, state)


# ------------------------------------------------------- work and definition

def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    c = case
    if c["kind"] == "embed":
        n, V, w = c["tokens"], c["vocab"], c["width"]
        # rows that some token names, in the mean
        h = sum(1.0 / k for k in range(1, V + 1))
        used = int(sum(-math.expm1(n * math.log1p(-1.0 / (k * h))) for k in range(1, V + 1)))
        b = n * (4 + w * _size(c["rows"])) + used * w * _size(c["table"])
        if c["mode"] == "fwd":
            return dict(bytes=b, flops=n * w)
        back = 2 * used if c["add"] else V
        return dict(bytes=b + n * w * _size(c["rows"]) + back * w * _size(c["grad"]),
                    flops=3 * n * w)
    if c["kind"] == "qk":
        values = c["tokens"] * (c["heads"] + c["kv"]) * c["d"]
        es, per = _size(c["dtype"]), 4 if c["norm"] else 0
        if c["mode"] == "append":
            return dict(bytes=es * 2 * (values + c["tokens"] * c["kv"] * c["dv"]),
                        flops=(per + 3) * values)
        return dict(bytes=es * 4 * values, flops=(3 * per + 6) * values)
    if c["kind"] in ("decay", "step"):
        H, Hk, d, dv, es = c["heads"], c["kv"], c["d"], c["dv"], _size(c["dtype"])
        n = c["rows"] if c["kind"] == "step" else c["tokens"]
        rows = es * n * (H + Hk) * (d + dv)
        if c["kind"] == "step":
            return dict(bytes=rows + 8 * n * H * d * dv, flops=5 * n * H * d * dv)
        states = 4 * c["seqs"] * H * d * dv * (2 if c["start"] else 1)
        if c["mode"] == "fwd":
            return dict(bytes=rows + states, flops=4 * n * H * d * dv)
        # q, k, v, dO in; o and the gradients of q, k, v out; the states' gradients
        return dict(bytes=2 * rows + 2 * states, flops=14 * n * H * d * dv)
    n = sum(_sizes(c))
    return dict(bytes=n * _size(c["grads"]) * (2 if c["clip"] else 1),
                flops=n * (3 if c["clip"] else 2))


def _exact_embed(c, S):
    """As the product with a one-hot matrix's definition has it, word by word in
    the order of the sorted tokens."""
    n, V, w = c["tokens"], c["vocab"], c["width"]
    on = torch.nonzero((S["ids"] >= 0) & (S["ids"] < V)).view(-1)
    word = S["ids"][on].long()
    out = torch.zeros(n, w, dtype=torch.float64, device=DEV)
    out[on] = S["W"].double().index_select(0, word) * S["scale"]
    if c["mode"] == "fwd":
        return out
    order = torch.argsort(word, stable=True)
    ends = torch.cumsum(torch.bincount(word, minlength=V), 0)
    dW = torch.empty(V, w, dtype=torch.float64, device=DEV)
    for lo in range(0, w, 64):
        g = S["dout"][on[order], lo:lo + 64].double()
        run_ = torch.cat([torch.zeros(1, g.shape[1], dtype=torch.float64, device=DEV),
                          torch.cumsum(g, 0)])[ends]
        run_ = torch.cat([run_[:1], run_.diff(dim=0)])
        dW[:, lo:lo + 64] = run_ * S["scale"]
    return dict(out=out, dW=dW + S["dW"].double() if c["add"] else dW)


def _exact_qk(c, S):
    """Each pair as a complex number that is turned; gradients by differentiation."""
    n, d, r = c["tokens"], c["d"], c["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       S["pos"].double()[:, None] * S["freq"][None])[:, None]
    re, im = ((torch.arange(r // 2), torch.arange(r // 2) + r // 2) if c["pairs"] == "half"
              else (torch.arange(0, r, 2), torch.arange(1, r, 2)))
    back = torch.argsort(torch.cat([re, im])).to(DEV)
    re, im = re.to(DEV), im.to(DEV)
    out = {}
    for name in ("q", "k"):
        train = c["mode"] == "train"
        x = S[name].double().reshape(n, -1, d).requires_grad_(train)
        w = S["w" + name]
        w = w.double().requires_grad_(train) if w is not None else None
        y = x
        if c["norm"]:
            y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + S["eps"]) * w
        z = torch.complex(y[..., re], y[..., im]) * turn
        y = torch.cat([torch.cat([z.real, z.imag], -1)[..., back], y[..., r:]], -1)
        out[name] = y.detach().reshape(n, -1)
        if train:
            wrt = [x, w] if c["norm"] else [x]
            got = torch.autograd.grad(y, wrt, S["d" + name].double().view(n, -1, d))
            out["d" + name] = got[0].reshape(n, -1)
            if c["norm"]:
                out["dw" + name] = got[1]
    if c["mode"] == "append":
        kc, vc = S["kc"].double(), S["vc"].double()
        for t, slot in enumerate(S["slot"].tolist()):
            if slot >= 0:
                kc[slot], vc[slot] = out["k"][t], S["v"][t].double()
        return dict(q=out["q"], k=kc, v=vc)
    return out


def _exact_decay(c, S):
    """Head by head and sequence by sequence, every pair of tokens."""
    H, Hk, d, dv, n = c["heads"], c["kv"], c["d"], c["dv"], c["tokens"]
    train, scale, f64 = c["mode"] == "train", S["scale"], torch.float64
    z = lambda *shape: torch.zeros(*shape, dtype=f64, device=DEV)  # noqa: E731
    o, s1 = z(n, H, dv), z(c["seqs"], H, d, dv)
    dq, dk, dv_, dg, ds0 = z(n, H, d), z(n, Hk, d), z(n, Hk, dv), z(H), z(c["seqs"], H, d, dv)
    first = 0
    for b, m in enumerate(_lens(c)):
        rows = slice(first, first + m)
        first += m
        t = torch.arange(m, device=DEV, dtype=f64)
        for h in range(H):
            e, g = h // (H // Hk), S["decay"][h].double()
            q = S["q"][rows, h * d:(h + 1) * d].double()
            k = S["k"][rows, e * d:(e + 1) * d].double()
            v = S["v"][rows, e * dv:(e + 1) * dv].double()
            up = S["do"][rows, h * dv:(h + 1) * dv].double() if train else None
            rest = torch.exp(g * (m - 1 - t))[:, None]
            s1[b, h] = (k * rest).t() @ v
            if train and c["start"]:
                ds1 = S["ds1"][b, h].double()
                dk[rows, e] += rest * (v @ ds1.t())
                dv_[rows, e] += rest * (k @ ds1)
                dg[h] += ((m - 1 - t)[:, None] * rest * (k @ ds1) * v).sum()
            if c["start"]:
                s0, since = S["s0"][b, h].double(), torch.exp(g * (t + 1))[:, None] * scale
                s1[b, h] += torch.exp(g * m) * s0
                o[rows, h] += since * (q @ s0)
                if train:
                    dq[rows, h] += since * (up @ s0.t())
                    ds0[b, h] += (since * q).t() @ up + torch.exp(g * m) * ds1
                    dg[h] += ((t + 1)[:, None] * since * (q @ s0) * up).sum()
                    dg[h] += m * torch.exp(g * m) * (s0 * ds1).sum()
            for lo in range(0, m, 4096):
                hi = min(m, lo + 4096)
                apart = t[lo:hi, None] - t[:hi]
                keep = torch.where(apart >= 0, torch.exp(g * apart.clamp_min(0)), 0.0) * scale
                a = (q[lo:hi] @ k[:hi].t()) * keep
                o[first - m + lo:first - m + hi, h] += a @ v[:hi]
                if train:
                    u = up[lo:hi] @ v[:hi].t()
                    dg[h] += (a * u * apart).sum()
                    dv_[first - m:first - m + hi, e] += a.t() @ up[lo:hi]
                    u = u * keep
                    dq[first - m + lo:first - m + hi, h] += u @ k[:hi]
                    dk[first - m:first - m + hi, e] += u.t() @ q[lo:hi]
    out = dict(o=o.view(n, -1), s1=s1)
    if train:
        out.update(dq=dq.view(n, -1), dk=dk.view(n, -1), dv=dv_.view(n, -1), ddecay=dg,
                   ds0=ds0 if c["start"] else None)
    return out


def _exact_step(c, S):
    H, Hk, d, dv = c["heads"], c["kv"], c["d"], c["dv"]
    state, o = S["state"].double(), []
    keep = torch.exp(S["decay"].double())[:, None, None]
    of = torch.arange(H, device=DEV) // (H // Hk)
    for r, slot in enumerate(S["slot"].tolist()):
        k, v = S["k"][r].double().view(Hk, d, 1)[of], S["v"][r].double().view(Hk, 1, dv)[of]
        state[slot] = keep * state[slot] + k @ v
        o.append((S["q"][r].double().view(H, 1, d) @ state[slot]).flatten() * S["scale"])
    return dict(o=torch.stack(o), state=state)


def _exact_norm(c, S):
    f = abs(S["factors"][0].item()) if c["clip"] else 1.0
    norms = torch.stack([torch.linalg.vector_norm(t.double(), math.inf if c["order"] == 0 else 2)
                         for t in S["grads"]]) * f
    norm = torch.linalg.vector_norm(norms, math.inf if c["order"] == 0 else 2)
    scale = min(1.0, S["max_norm"] / (norm.item() + 1e-6)) * f
    out = dict(norm=norm.view(1), scale=torch.tensor([scale], dtype=torch.float64, device=DEV),
               norms=norms)
    if c["clip"]:
        out["grads"] = S["flat"].double() * scale
    return out


def exact(case, seed):
    S = prepare(case, seed)
    return dict(embed=_exact_embed, qk=_exact_qk, decay=_exact_decay, step=_exact_step,
                norm=_exact_norm)[case["kind"]](case, S)
