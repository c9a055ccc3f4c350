"""AdamW over many tensors: against the formula in 64 bits, the 8-bit states
against their definition bit by bit, what rounding at random keeps, and the
refusals."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2303_07030_amd import nsd

EPS32 = 2.0 ** -24
H = dict(lr=1e-2, beta1=0.9, beta2=0.98, eps=1e-8)
WD = 0.05
SIZES = [1, 3, 255, 256, 257, 4095, 4096, 4097, 20_001, 0, 64]


# ------------------------------------------------------------- refusals

def record(n=8, ptr=0x1000, p=0, g=0, master=None, scales=0x1000):
    return nsd.nsd_adamw_tensor(n, ptr, master, ptr, ptr, ptr, scales, scales, p, g, 0.0)


@pytest.mark.parametrize("t, bits", [
    (record(n=-1), 32), (record(ptr=None), 32), (record(p=7), 32), (record(g=-1), 32),
    (record(master=0x1000), 32), (record(scales=None), 8), (record(), 16)])
def test_bad_tensors_are_refused(t, bits):
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_adamw_plan_build([t], bits, torch.empty(4096, dtype=torch.uint8))
    assert e.value.status == nsd.NSD_ERR_INVALID_ARG


def test_too_long_a_tensor_is_refused():
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_adamw_plan_build([record(n=2 ** 31)], 32, torch.empty(4096, dtype=torch.uint8))
    assert e.value.status == nsd.NSD_ERR_TOO_LARGE


def test_more_chunks_than_a_launch_has_blocks_are_refused():
    many = [record(n=2 ** 31 - 5000)] * 33  # 2^24 chunks: a grid's threads take 32 bits
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_adamw_plan_build(many, 32, torch.empty(4096, dtype=torch.uint8))
    assert e.value.status == nsd.NSD_ERR_TOO_LARGE


def apart(n, first, **change):
    """A record of bf16 weights whose arrays follow each other from `first` on."""
    sizes = dict(param=2 * n, master=4 * n, grad=2 * n, m=n, v=n, m_scale=4 * -(-n // 256),
                 v_scale=4 * -(-n // 256))
    t = nsd.nsd_adamw_tensor(n, param_dtype=nsd.BF16, grad_dtype=nsd.BF16)
    for name, size in sizes.items():
        setattr(t, name, first)
        first += size
    for name, value in change.items():
        setattr(t, name, value)
    return t, first


def test_arrays_that_share_memory_are_refused():
    table = torch.empty(4096, dtype=torch.uint8)
    a, end = apart(600, 0x1000)
    for change in (dict(param=a.param), dict(param=a.param + 1198), dict(m=a.v), dict(grad=a.master),
                   dict(v_scale=a.m_scale + 8), dict(m=a.grad), dict(master=end - 4)):
        b, _ = apart(40, end, **change)
        for records in ([a, b], [b, a], [a, apart(0, end)[0], b]):
            with pytest.raises(nsd.NsdError) as e:
                nsd.nsd_adamw_plan_build(records, 8, table)
            assert e.value.status == nsd.NSD_ERR_INVALID_ARG and "share" in str(e.value)
    for field in ("master", "grad", "m", "v", "m_scale", "v_scale"):  # within one tensor
        c, _ = apart(600, 0x1000)
        setattr(c, field, c.param)
        with pytest.raises(nsd.NsdError) as e:
            nsd.nsd_adamw_plan_build([c], 8, table)
        assert e.value.status == nsd.NSD_ERR_INVALID_ARG and "share" in str(e.value)


@pytest.mark.gpu
def test_neighbours_and_shared_gradients_are_taken():
    """Arrays side by side in one buffer, and one gradient of two tensors."""
    from paper_2303_07030_amd.optim import AdamW
    buf = torch.zeros(4 * 300, device="cuda")
    p, m, v, g = buf.split(300)
    g.fill_(0.5)
    q = torch.zeros(300, device="cuda")
    AdamW([p, q], [g, g], m=[m, torch.zeros_like(m)], v=[v, torch.zeros_like(v)], **H).step()
    assert torch.equal(p, q) and bool((p < 0).all())
    with pytest.raises(nsd.NsdError):
        AdamW([p, p], [g, g])


def test_a_small_table_is_refused():
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_adamw_plan_build([record()], 32, torch.empty(8, dtype=torch.uint8))
    assert e.value.status == nsd.NSD_ERR_WORKSPACE


@pytest.mark.parametrize("change", [dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=math.nan),
                                    dict(eps=0.0), dict(eps=math.inf), dict(lr=math.nan),
                                    dict(step=0)])
def test_bad_hyperparameters_are_refused(change):
    plan = nsd.nsd_adamw_plan(1, 1, 32, 0x1000)
    h = nsd.nsd_adamw(**{**dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1), **change})
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_adamw_step(plan, h)
    assert e.value.status == nsd.NSD_ERR_INVALID_ARG


def test_a_plan_never_built_is_refused():
    h = nsd.nsd_adamw(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1)
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_adamw_step(nsd.nsd_adamw_plan(1, 1, 0, None), h)
    assert e.value.status == nsd.NSD_ERR_INVALID_ARG
    nsd.nsd_adamw_step(nsd.nsd_adamw_plan(0, 0, 32, None), h)  # no tensors: nothing to do


# --------------------------------------------------- definition, on the CPU

def mix(x):
    x = np.asarray(x, np.uint32).copy()
    x ^= x >> np.uint32(16)
    x *= np.uint32(0x6A09E667)
    x ^= x >> np.uint32(15)
    x *= np.uint32(0xBB67AE85)
    return x ^ (x >> np.uint32(16))


def noise(n, tensor, step):
    key = mix(np.array([(step * 0x9E3779B1 + tensor) & 0xFFFFFFFF], np.uint32))[0]
    with np.errstate(over="ignore"):
        return mix(np.arange(n, dtype=np.uint32) * np.uint32(0x9E3779B1) + key)


def decode(codes, mant):
    """Value of every code of an 8-bit float with `mant` mantissa bits."""
    c = codes.astype(np.int64)
    bias = 7 if mant == 3 else 15
    e, f = (c & 0x7F) >> mant, c & ((1 << mant) - 1)
    v = np.where(e == 0, f * 2.0 ** (1 - bias - mant), (1 + f / 2.0 ** mant) * 2.0 ** (e - bias))
    return np.where(c & 0x80, -v, v)


def blocks(x):
    return np.pad(x, (0, -len(x) % 256)).reshape(-1, 256)


def to_eight(x, rnd, mant):
    """(codes, scales) of fp32 values, in fp32 as the header defines them."""
    top = np.float32(448 if mant == 3 else 57344)
    s = np.abs(blocks(x)).max(1) * np.float32(1 / float(top))
    s = np.where(s < 2.0 ** -126, np.float32(0), s)
    with np.errstate(divide="ignore"):
        inv = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
    y = (np.abs(blocks(x)) * inv[:, None]).reshape(-1)[: len(x)]
    low, drop = (-6, 20) if mant == 3 else (-14, 21)
    raw = y.view(np.uint32) + (rnd << np.uint32(drop - 16)) + np.uint32(1 << (drop - 17))
    code = (raw >> np.uint32(drop)).astype(np.int64) - ((126 + low) << mant)
    frac = (rnd.astype(np.float32) + np.float32(0.5)) * np.float32(2.0 ** -16)
    small = np.floor(y * np.float32(2.0 ** (mant - low)) + frac).astype(np.int64)
    code = np.minimum(np.where(y < 2.0 ** low, small, code), 0x7E if mant == 3 else 0x7B)
    if mant == 2:
        code = np.where((y > 0) & (code == 0), 1, code)
    else:
        code = code | np.where(np.signbit(x), 0x80, 0)
    return code.astype(np.uint8), s.astype(np.float32)


def test_codes_stand_for_torch_values():
    c = np.arange(256, dtype=np.uint8)
    for mant, T, fine in ((3, torch.float8_e4m3fn, (c & 0x7F) != 0x7F),
                          (2, torch.float8_e5m2, (c & 0x7F) < 0x7C)):
        assert np.array_equal(torch.from_numpy(c).view(T).float().numpy()[fine],
                              decode(c, mant)[fine].astype(np.float32))


# ------------------------------------------------------------------ on a GPU

def gpu(x, dtype=torch.float32, shift=0):
    """A device copy `shift` elements off the allocation's alignment."""
    t = torch.empty(len(x) + shift, dtype=dtype, device="cuda")[shift:]
    t.copy_(torch.from_numpy(np.asarray(x)))
    return t


def make(rng, weights, grads, shift):
    W = torch.float32 if weights == "f32" else torch.bfloat16
    G = torch.float32 if grads == "f32" else torch.bfloat16
    p = [rng.standard_normal(n).astype(np.float32) for n in SIZES]
    g = [(rng.standard_normal(n) * 10.0 ** rng.uniform(-6, 1, n)).astype(np.float32)
         for n in SIZES]
    P, Gr = [gpu(x, W, shift) for x in p], [gpu(x, G, shift) for x in g]
    copies = [gpu(x, torch.float32, shift) for x in p] if weights == "copy" else None
    return P, Gr, copies


def as64(t):
    return t.double().cpu().numpy()


def formula(w, g, m, v, t, scale=1.0):
    g = scale * g
    m = H["beta1"] * m + (1 - H["beta1"]) * g
    v = H["beta2"] * v + (1 - H["beta2"]) * g * g
    step = H["lr"] * (m / (1 - H["beta1"] ** t)) / (np.sqrt(v / (1 - H["beta2"] ** t)) + H["eps"])
    return w * (1 - H["lr"] * WD) - step, m, v, np.abs(step)


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("weights", ["f32", "bf16", "copy"])
def test_32_bit_states_follow_the_formula(weights, grads, shift):
    from paper_2303_07030_amd.optim import AdamW
    rng = np.random.default_rng(5)
    P, G, copies = make(rng, weights, grads, shift)
    opt = AdamW(P, G, masters=copies, weight_decay=WD, **H)
    clip = torch.tensor(0.5, device="cuda")
    for t in (1, 2, 3):
        before = [(as64(copies[i] if copies else P[i]), as64(G[i]), as64(opt.m[i]),
                   as64(opt.v[i])) for i in range(len(P))]
        opt.step(grad_scale=clip if t == 2 else None)
        for i, (w0, g, m0, v0) in enumerate(before):
            w, m, v, step = formula(w0, g, m0, v0, t, 0.5 if t == 2 else 1.0)
            # four roundings each of the moments' terms
            assert np.all(np.abs(as64(opt.m[i]) - m)
                          <= 4 * EPS32 * (np.abs(m0) + np.abs(g)) + 1e-44)
            assert np.all(np.abs(as64(opt.v[i]) - v) <= 5 * EPS32 * (v0 + g * g) + 1e-44)
            # the weight's product and sum; the step's dozen roundings, and what
            # the rounding of a moment that cancels makes of it
            root = np.sqrt(v / (1 - H["beta2"] ** t)) + H["eps"]
            off = H["lr"] * 4 * EPS32 * (np.abs(m0) + np.abs(g)) / (1 - H["beta1"] ** t) / root
            tol = 3 * EPS32 * np.abs(w0) + 16 * EPS32 * step + off
            got = as64(copies[i] if copies else P[i])
            if weights == "bf16":  # to a neighbour: less than one unit of bf16
                tol = tol + 2.0 ** -7 * np.abs(w)
            assert np.all(np.abs(got - w) <= tol), (weights, t, i)
            if copies:  # the nearest bf16 of the copy
                assert torch.equal(P[i], copies[i].bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("weights, grads, shift", [("f32", "f32", 0), ("bf16", "bf16", 1),
                                                   ("copy", "bf16", 0)])
def test_8_bit_states_bit_by_bit(weights, grads, shift):
    from paper_2303_07030_amd.optim import AdamW
    rng = np.random.default_rng(6)
    P, G, copies = make(rng, weights, grads, shift)
    one = torch.float8_e4m3fn
    m = [torch.zeros(n + shift, dtype=torch.uint8, device="cuda")[shift:].view(one) for n in SIZES]
    opt = AdamW(P, G, masters=copies, weight_decay=WD, state_bits=8, m=m, **H)
    f = np.float32
    for t in (1, 2, 3):
        if t == 3:  # a block whose gradients vanish beside it keeps a finite state
            G[8][256:512] *= 1e-30
        before = []
        for i in range(len(P)):
            cm, cv = (x[i].view(torch.uint8).cpu().numpy() for x in (opt.m, opt.v))
            sm, sv = (x[i].cpu().numpy() for x in (opt.m_scale, opt.v_scale))
            before.append((as64(copies[i] if copies else P[i]), G[i].float().cpu().numpy(),
                           cm, sm, cv, sv))
        opt.step()
        for i, (w0, g, cm, sm, cv, sv) in enumerate(before):
            n = len(g)
            if n == 0:
                continue
            m0 = decode(cm, 3).astype(f) * np.repeat(sm, 256)[:n]
            v0 = decode(cv, 2).astype(f) * np.repeat(sv, 256)[:n]
            m1 = m0 * f(H["beta1"]) + g * f(1 - H["beta1"])
            v1 = v0 * f(H["beta2"]) + (g * f(1 - H["beta2"])) * g
            rnd = noise(n, i, t)
            for x, mant, codes, scales, r in ((m1, 3, opt.m[i], opt.m_scale[i],
                                               rnd & np.uint32(0xFFFF)),
                                              (v1, 2, opt.v[i], opt.v_scale[i],
                                               rnd >> np.uint32(16))):
                want, s = to_eight(x, r, mant)
                assert np.array_equal(scales.cpu().numpy(), s)
                assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), want)
                # a neighbour: within a code's distance of what it stands for
                back = decode(want, mant) * np.repeat(s, 256)[:n].astype(np.float64)
                unit = np.maximum(np.abs(x) * 2.0 ** -mant,
                                  np.repeat(s, 256)[:n] * 2.0 ** (-9 if mant == 3 else -16))
                assert np.all(np.abs(back - x) <= unit * (1 + 1e-6))
            w, _, _, step = formula(w0, g.astype(np.float64), m0.astype(np.float64),
                                    v0.astype(np.float64), t)
            root = np.sqrt(v1.astype(np.float64) / (1 - H["beta2"] ** t)) + H["eps"]
            off = H["lr"] * 4 * EPS32 * (np.abs(m0) + np.abs(g)) / (1 - H["beta1"] ** t) / root
            tol = 3 * EPS32 * np.abs(w0) + 16 * EPS32 * step + off
            if weights == "bf16":
                tol = tol + 2.0 ** -7 * np.abs(w)
            got = as64(copies[i] if copies else P[i])
            assert np.all(np.abs(got - w) <= tol), (weights, t, i)


@pytest.mark.gpu
def test_rounding_at_random_keeps_means_and_repeats():
    """A constant gradient on 2^18 weights: the codes' mean is the state's
    within five standard deviations, and so is the bf16 weights'."""
    from paper_2303_07030_amd.optim import AdamW
    n = 1 << 18
    out = []
    for _ in range(2):
        p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
        g = torch.full((n,), 0.3, device="cuda")
        g[::256] = 1.0  # the blocks' largest
        opt = AdamW([p], [g], lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0,
                    state_bits=8)
        opt.step()
        out.append((p, opt.m[0].view(torch.uint8), opt.v[0].view(torch.uint8)))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    rest = torch.arange(n, device="cuda") % 256 != 0
    k = int(rest.sum())
    for codes, scale, x, mant in ((opt.m[0], opt.m_scale[0], 0.1 * 0.3, 3),
                                  (opt.v[0], opt.v_scale[0], 0.001 * 0.09, 2)):
        y = codes.float().double() * scale.double().repeat_interleave(256)
        unit = x * 2.0 ** -mant  # a bound of the two neighbours' distance
        assert abs(float(y[rest].mean()) - x) <= 5 * unit / 2 / math.sqrt(k) + 1e-6 * x
        assert len(torch.unique(codes.view(torch.uint8)[rest])) == 2
    # the step moves a weight by 1e-4, a fortieth of bf16's unit below 1
    w = p[rest].double()
    assert abs(float(w.mean()) - (1 - 1e-4)) <= 5 * 2.0 ** -8 / 2 / math.sqrt(k) + 1e-8


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_what_is_not_finite_stays_where_the_header_says(bits):
    from paper_2303_07030_amd.optim import AdamW
    p, g = torch.ones(600, device="cuda"), torch.full((600,), 0.1, device="cuda")
    g[10], g[300] = math.nan, math.inf
    opt = AdamW([p], [g], state_bits=bits, **H)
    opt.step()
    g.fill_(0.1)
    opt.step()
    bad = torch.isnan(p).cpu().numpy()
    want = np.zeros(600, bool)
    want[10] = want[300] = True
    if bits == 8:
        want[256:512] = True
    assert np.array_equal(bad, want)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_step_counts_its_replays(bits):
    from paper_2303_07030_amd.optim import AdamW
    rng = np.random.default_rng(8)
    n = 5000
    w, g = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    eager, graph = [], []
    p, gr = gpu(w), gpu(g)
    opt = AdamW([p], [gr], state_bits=bits, **H)
    for t in range(4):
        opt.step(lr=1e-2 / (t + 1))
        eager.append((p.clone(), opt.m[0].view(torch.uint8).clone()))
    p, gr = gpu(w), gpu(g)
    opt = AdamW([p], [gr], state_bits=bits, **H)
    t = torch.zeros(1, dtype=torch.int32, device="cuda")
    lr = torch.zeros(1, device="cuda")
    side = torch.cuda.Stream()
    cg = torch.cuda.CUDAGraph()
    with torch.cuda.graph(cg, stream=side):
        t.add_(1)
        opt.step(step_dev=t, lr_dev=lr)
    for k in range(4):
        lr.fill_(1e-2 / (k + 1))
        cg.replay()
        torch.cuda.synchronize()
        graph.append((p.clone(), opt.m[0].view(torch.uint8).clone()))
    for (pe, me), (pg, mg) in zip(eager, graph):
        assert torch.equal(me, mg)
        # the corrections in fp32 instead of fp64: a few units of the step
        assert float((pe - pg).abs().max()) <= 64 * EPS32 * 4


@pytest.mark.gpu
def test_an_optimizer_refuses_what_does_not_fit():
    from paper_2303_07030_amd.optim import AdamW
    p, g = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    for params, grads, kw in (([p], [g[:9]], {}), ([p], [], {}), ([p], [g.double()], {}),
                              ([p.cpu()], [g], {}), ([p], [g], dict(state_bits=4)),
                              ([torch.ones(20, device="cuda")[::2]], [g], {}),
                              ([p], [g], dict(weight_decay=[0.1, 0.2])),
                              ([p], [g], dict(masters=[g[:9]]))):
        with pytest.raises(ValueError):
            AdamW(params, grads, **kw)
    with pytest.raises(nsd.NsdError):
        AdamW([p], [g], masters=[torch.ones(10, device="cuda")])
    AdamW([], []).step()
    assert ctypes.sizeof(nsd.nsd_adamw_tensor) == 80


@pytest.mark.gpu
@pytest.mark.parametrize("weights", ["f32", "copy"])
def test_second_moments_below_the_normal_numbers(weights):
    """Gradients of 1e-20: v is denormal, its root is not, and eps is smaller."""
    from paper_2303_07030_amd.optim import AdamW
    rng = np.random.default_rng(9)
    n, lr, b1, b2, eps = 1027, 1e-2, 0.9, 0.98, 1e-30
    g = (10.0 ** rng.uniform(-20, -18, n)).astype(np.float32)
    p = gpu(np.ones(n), torch.float32 if weights == "f32" else torch.bfloat16)
    opt = AdamW([p], [gpu(g)], lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=0.0,
                masters=True if weights == "copy" else None)
    opt.step()
    got = as64(opt.masters[0] if weights == "copy" else p)
    # of the first step m / sqrt(v) is 1; v is a multiple u of 2^-149, rounded three
    # times, of which the root keeps half; the weight's own rounding
    u = (1 - b2) * g.astype(np.float64) ** 2 / 2.0 ** -149
    tol = lr * (1.5 / (u - 1.5) + 16 * EPS32) + 2 * EPS32
    assert np.all(np.abs(got - (1.0 - lr)) <= tol)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("weights", ["f32", "copy"])
@pytest.mark.parametrize("lr, wd", [(1e-4, 0.01), (2e-4, 0.01), (1e-5, 0.012), (1e-2, 0.05)])
def test_a_small_decay_is_not_rounded_before_the_weight(lr, wd, weights, bits):
    """Without gradients only w (1 - lr wd) is left: to the nearest, but for lr and
    the product in 32 bits."""
    from paper_2303_07030_amd.optim import AdamW
    rng = np.random.default_rng(10)
    w = rng.standard_normal(5000).astype(np.float32)
    w[7], w[8] = np.inf, -np.inf
    p = gpu(w, torch.float32 if weights == "f32" else torch.bfloat16)
    copies = [gpu(w)] if weights == "copy" else None
    opt = AdamW([p], [torch.zeros(5000, device="cuda")], lr=lr, weight_decay=wd, masters=copies,
                state_bits=bits)
    opt.step()
    got = as64(copies[0] if copies else p)
    assert got[7] == np.inf and got[8] == -np.inf
    fine = np.isfinite(w)
    want = w[fine].astype(np.float64) * (1 - lr * wd)
    off = np.abs(got[fine] - want)
    assert np.all(off <= np.spacing(np.abs(want).astype(np.float32)) / 2.0
                  + 4 * EPS32 * lr * wd * np.abs(want))


@pytest.mark.gpu
def test_a_refused_step_changes_nothing():
    from paper_2303_07030_amd.optim import AdamW
    rng = np.random.default_rng(11)
    w, g = rng.standard_normal(700).astype(np.float32), rng.standard_normal(700).astype(np.float32)
    opts = [AdamW([gpu(w, torch.bfloat16)], [gpu(g)], state_bits=8, **H) for _ in range(2)]
    opts[1].step(lr=0.02)
    opts[0].step(lr=0.02)
    for bad in (math.nan, math.inf):
        with pytest.raises(nsd.NsdError):
            opts[0].step(lr=bad)
    assert opts[0].t == 1 and opts[0].hyper.lr == 0.02
    for o in opts:
        o.step()
    a, b = ((o.params[0], o.m[0].view(torch.uint8), o.v[0].view(torch.uint8)) for o in opts)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    # the caller's count, then the optimizer's
    count = torch.full((1,), 3, dtype=torch.int32, device="cuda")
    opts[0].step(step_dev=count)
    assert opts[0].t == 2
    opts[0].t = 3
    opts[1].step()
    for o in opts:
        o.step()
    assert opts[0].t == opts[1].t == 4
