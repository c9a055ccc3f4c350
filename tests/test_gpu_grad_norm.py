"""The norm of many gradients and the factor that clips them: against sums in 64
bits, the extremes of 32 bits, what is not finite, AdamW's own measure, and the
refusals."""
import math

import numpy as np
import pytest
import torch

from paper_2303_07030_amd import nsd

P = 0x1000
SIZES = [1, 3, 0, 255, 4097, 16_383, 16_384, 16_385, 70_001, 7]


# ------------------------------------------------------------- refusals

@pytest.mark.parametrize("t, status", [
    ((-1, P, 0), nsd.NSD_ERR_INVALID_ARG), ((8, None, 0), nsd.NSD_ERR_INVALID_ARG),
    ((8, P, 2), nsd.NSD_ERR_INVALID_ARG), ((8, P + 2, 0), nsd.NSD_ERR_INVALID_ARG),
    ((8, P + 1, 1), nsd.NSD_ERR_INVALID_ARG), ((2 ** 31 - 1, P, 0), nsd.NSD_ERR_TOO_LARGE)])
def test_bad_tensors_are_refused(t, status):
    for call in (lambda r: nsd.nsd_grad_plan_size(r),
                 lambda r: nsd.nsd_grad_plan_build(r, torch.empty(4096, dtype=torch.uint8))):
        with pytest.raises(nsd.NsdError) as e:
            call([nsd.nsd_grad_tensor(*t)])
        assert e.value.status == status


def test_more_chunks_than_a_launch_has_blocks_are_refused():
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_grad_plan_size([nsd.nsd_grad_tensor(2 ** 31 - 20_000, P, 0)] * 129)
    assert e.value.status == nsd.NSD_ERR_TOO_LARGE


def test_bad_calls_are_refused():
    plan = nsd.nsd_grad_plan(2, 3, 0, P)
    h = nsd.nsd_clip(1.0, 2, None)
    ws = torch.empty(4096, dtype=torch.uint8)
    for args, status in (((nsd.nsd_grad_plan(1, 1, 0, None), h, P, P, None, ws), "INVALID"),
                         ((plan, nsd.nsd_clip(1.0, 1, None), P, P, None, ws), "INVALID"),
                         ((plan, nsd.nsd_clip(0.0, 2, None), P, P, None, ws), "INVALID"),
                         ((plan, nsd.nsd_clip(math.nan, 2, None), P, P, None, ws), "INVALID"),
                         ((plan, h, None, P, None, ws), "INVALID"),
                         ((plan, h, P, None, None, ws), "INVALID"),
                         ((plan, h, P, P, None, None), "WORKSPACE")):
        with pytest.raises(nsd.NsdError, match=status):
            nsd.nsd_grad_norm(*args)
    with pytest.raises(nsd.NsdError, match="INVALID"):
        nsd.nsd_grad_clip(plan, None)
    with pytest.raises(nsd.NsdError, match="share memory"):
        nsd.nsd_grad_clip(nsd.nsd_grad_plan(2, 3, 1, P), P)
    with pytest.raises(ValueError, match="norms"):
        nsd.nsd_grad_norm(plan, h, P, P, torch.zeros(1, dtype=torch.float64), ws)
    with pytest.raises(ValueError, match="scale"):
        nsd.nsd_grad_clip(plan, torch.zeros(1, dtype=torch.float64))


@pytest.mark.parametrize("change", [
    dict(grad_scale=("scale", 0)), dict(grad_scale=("norm", 4)), dict(grad_scale=("norms", 12)),
    dict(grad_scale=("ws", 8)), dict(scale=("norm", 0)), dict(norm=("norms", 8)),
    dict(scale=("ws", 64)), dict(norms=("ws", 0)), dict(norms=("table", 0))])
def test_what_is_written_is_apart(change):
    hold = torch.empty((1 << 12) + 256, dtype=torch.uint8)
    at = {n: (i + 1) << 24 for i, n in enumerate(("norm", "scale", "norms", "grad_scale", "table"))}
    ws = hold[-hold.data_ptr() % 256:]
    at["ws"] = ws.data_ptr()
    for name, (other, offset) in change.items():
        at[name] = at[other] + offset
    plan = nsd.nsd_grad_plan(2, 40, 0, at["table"])
    with pytest.raises(nsd.NsdError, match="shares memory") as e:
        nsd.nsd_grad_norm(plan, nsd.nsd_clip(1.0, 2, at["grad_scale"]), at["norm"], at["scale"],
                          at["norms"], ws)
    assert e.value.status == nsd.NSD_ERR_INVALID_ARG


def test_bad_orders_are_refused():
    from paper_2303_07030_amd import optim
    with pytest.raises(ValueError, match="order"):
        optim.GradNorm([], order=1)
    with pytest.raises(ValueError, match="contiguous device tensor"):
        optim.GradNorm([torch.zeros(4)])


# ------------------------------------------------------------- on the GPU

def grads_of(dtype, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    flat = (torch.randn(sum(SIZES) + 1, generator=g) * std).to(dtype).cuda()
    return list(flat[1:].split(SIZES))  # no tensor at a round address


def want(grads, order, f, top):
    """(norm, scale, norms) in 64 bits."""
    each = [np.abs(t.double().cpu().numpy()) for t in grads]
    if order == 2:
        norms = np.array([math.sqrt(math.fsum(x * x)) for x in each])
        norm = math.sqrt(math.fsum(norms ** 2))
    else:
        norms = np.array([x.max(initial=0.0) for x in each])
        norm = norms.max(initial=0.0)
    norm, norms = norm * abs(f), norms * abs(f)
    return norm, f * min(1.0, top / (norm + 1e-6)), norms


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", [2, math.inf])
@pytest.mark.parametrize("top, f", [(1.0, None), (1e9, None), (math.inf, -0.25), (0.5, 3.0)])
def test_norms_and_factor(dtype, order, top, f):
    """A sum of n squares in 64 bits is off by n 2^-53 at most of itself, its root by
    half of that and a rounding; the factor is rounded to 32 bits once."""
    from paper_2303_07030_amd import optim
    grads = grads_of(dtype)
    p = optim.GradNorm(grads, top, order)
    p.measure(None if f is None else torch.full((1,), f, device="cuda"))
    norm, scale, norms = want(grads, order, 1.0 if f is None else f, top)
    room = (sum(SIZES) + 8) * 2.0 ** -53
    assert abs(p.norm.item() - norm) <= room * norm
    assert np.all(np.abs(p.norms.cpu().numpy() - norms) <= room * norms)
    assert abs(p.scale.item() - scale) <= (2.0 ** -24 + room) * abs(scale)
    old = [g.clone() for g in grads]
    p.clip()
    for g, o in zip(grads, old):
        assert torch.equal(g, (o.float() * p.scale).to(dtype))


@pytest.mark.gpu
def test_the_extremes_of_32_bits():
    from paper_2303_07030_amd import optim
    big = [torch.full((1000,), 3e38, device="cuda"),
           torch.full((1000,), 1e-44, device="cuda"),
           torch.full((5,), 3e38, device="cuda", dtype=torch.bfloat16)]
    p = optim.GradNorm(big, 1.0)
    p.measure()
    norm, scale, norms = want(big, 2, 1.0, 1.0)
    assert norms[1] > 0
    np.testing.assert_allclose(p.norms.cpu().numpy(), norms, rtol=1e-12)
    assert math.isclose(p.norm.item(), norm, rel_tol=1e-12)
    # 1e-40 is below 2^-126, the least normal number of 32 bits: there numbers lie 2^-149
    # apart, and a rounding is off by half of that
    assert abs(p.scale.item() - scale) <= 2.0 ** -150


@pytest.mark.gpu
@pytest.mark.parametrize("order", [2, math.inf])
@pytest.mark.parametrize("tensor, place", [(0, 0), (1, 2), (8, 70_000), (8, 16_384)])
def test_what_is_not_finite_shows(order, tensor, place):
    from paper_2303_07030_amd import optim
    for bad in (math.nan, math.inf, -math.inf):
        grads = grads_of(torch.float32, seed=1)
        grads[tensor][place] = bad
        p = optim.GradNorm(grads, 1.0, order)
        p.measure()
        assert [i for i, v in enumerate(p.norms.tolist()) if not math.isfinite(v)] == [tensor]
        if math.isnan(bad):
            assert math.isnan(p.norm.item()) and math.isnan(p.scale.item())
        else:
            assert p.norm.item() == math.inf and p.scale.item() == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("order", [2, math.inf])
@pytest.mark.parametrize("f", [None, -0.25])
def test_nothing_is_clipped_without_a_bound(order, f):
    """An infinite gradient included; one that is not a number shows in the factor."""
    from paper_2303_07030_amd import optim
    for bad in (math.inf, -math.inf, math.nan):
        grads = grads_of(torch.float32, seed=1)
        grads[8][16_384] = bad
        p = optim.GradNorm(grads, order=order)
        p.measure(None if f is None else torch.full((1,), f, device="cuda"))
        if math.isnan(bad):
            assert math.isnan(p.norm.item()) and math.isnan(p.scale.item())
        else:
            assert p.norm.item() == math.inf and p.scale.item() == (1.0 if f is None else f)


@pytest.mark.gpu
def test_empty_lists_and_zero_gradients():
    from paper_2303_07030_amd import optim
    for grads in ([], [torch.zeros(0, device="cuda")], [torch.zeros(40, device="cuda")]):
        p = optim.GradNorm(grads, 2.0)
        p.measure()
        p.clip()
        assert p.norm.item() == 0.0 and p.scale.item() == 1.0
        assert p.norms.tolist() == [0.0] * len(grads)


@pytest.mark.gpu
def test_a_measures_own_factor_is_not_its_input():
    """Refused, and nothing changes; another measure's factor is an input like any."""
    from paper_2303_07030_amd import optim
    g = torch.full((100,), 2.0, device="cuda")
    p, other = optim.GradNorm([g], 1.0), optim.GradNorm([g], 5.0)
    p.measure()
    old = p.norm.item(), p.scale.item()
    with pytest.raises(nsd.NsdError, match="shares memory"):
        p.measure(grad_scale=p.scale)
    assert (p.norm.item(), p.scale.item()) == old
    other.measure(grad_scale=p.scale)
    assert math.isclose(other.norm.item(), 20.0 * old[1], rel_tol=1e-12)
    w = torch.ones(100, device="cuda")
    opt = optim.AdamW([w], [g], max_norm=1.0)
    with pytest.raises(nsd.NsdError, match="shares memory"):
        opt.step(grad_scale=opt.grad_norm.scale)
    assert opt.t == 0 and torch.all(w == 1.0)


@pytest.mark.gpu
def test_gradients_of_several_tensors():
    """One gradient listed twice counts twice, and is not clipped in place."""
    from paper_2303_07030_amd import optim
    g = torch.full((100,), 2.0, device="cuda")
    p = optim.GradNorm([g, g, g[3:]], 1.0)
    p.measure()
    assert math.isclose(p.norm.item(), math.sqrt(4.0 * 297), rel_tol=1e-12)
    with pytest.raises(nsd.NsdError, match="share memory"):
        p.clip()
    assert torch.all(g == 2.0)


@pytest.mark.gpu
def test_a_measure_on_another_stream():
    """What the measure leaves is not overwritten by the first values, which a busy current
    stream would come to later."""
    from paper_2303_07030_amd import optim
    g = torch.full((1000,), 2.0, device="cuda")
    side = torch.cuda.Stream()
    a, b = torch.randn(2, 4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for built, stream in ((side, side), (side.cuda_stream, side.cuda_stream), (None, side)):
        for _ in range(40):
            torch.mm(a, b)
        p = optim.GradNorm([g], 1.0, stream=built)
        p.measure(stream=stream)
        torch.cuda.synchronize()
        assert math.isclose(p.norm.item(), math.sqrt(4000.0), rel_tol=1e-12)
        assert math.isclose(p.norms.item(), math.sqrt(4000.0), rel_tol=1e-12)
        assert math.isclose(p.scale.item(), 1.0 / math.sqrt(4000.0), rel_tol=1e-6)


@pytest.mark.gpu
def test_a_captured_measure_and_clip_follow_the_gradients():
    from paper_2303_07030_amd import optim
    grads = grads_of(torch.bfloat16, seed=2)
    p = optim.GradNorm(grads, 1.0)
    side = torch.cuda.Stream()
    p.measure()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        p.measure()
        p.clip()
    for seed in (3, 4, 5):
        fresh = grads_of(torch.bfloat16, seed=seed, std=float(seed))
        for g, x in zip(grads, fresh):
            g.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        norm, scale, _ = want(fresh, 2, 1.0, 1.0)
        assert math.isclose(p.norm.item(), norm, rel_tol=1e-10)
        for g, x in zip(grads, fresh):
            assert torch.equal(g, (x.float() * p.scale).bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("f", [None, 0.5])
def test_adamw_clips_what_it_takes(f):
    """AdamW(max_norm) is AdamW given the factor; the gradients stay."""
    from paper_2303_07030_amd import optim
    sizes = [5, 300, 4097]
    g = torch.Generator(device="cuda").manual_seed(7)
    weights = [torch.randn(n, device="cuda", generator=g) for n in sizes]
    grads = [torch.randn(n, device="cuda", generator=g) for n in sizes]
    gs = None if f is None else torch.full((1,), f, device="cuda")
    a = [w.clone() for w in weights]
    b = [w.clone() for w in weights]
    one = optim.AdamW(a, grads, max_norm=0.7)
    two = optim.AdamW(b, grads)
    kept = [x.clone() for x in grads]
    for _ in range(3):
        one.step(grad_scale=gs)
        norm = math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in grads))
        norm *= 1.0 if f is None else f
        factor = torch.full((1,), (1.0 if f is None else f) * 0.7 / (norm + 1e-6), device="cuda")
        two.step(grad_scale=factor)
    assert abs(one.grad_norm.norm.item() - norm) <= 1e-9 * norm
    # the factor may be rounded the other way (2^-23); three steps of 1e-3 each
    for x, y in zip(a, b):
        assert (x - y).abs().max().item() <= 3e-3 * 8 * 2.0 ** -23 + 2.0 ** -22
    for x, y in zip(grads, kept):
        assert torch.equal(x, y)
