"""The router: the chosen experts, gates, counts and balance loss against plain
formulas in 64 bits, the gradient against the formula's and against
differences, closed experts, skipped tokens, ties, and the refusals."""
import math

import numpy as np
import pytest
import torch

from paper_2303_07030_amd import nsd

EPS32 = 2.0 ** -24


# ------------------------------------------------------------- refusals

@pytest.mark.parametrize("change, status", [
    (dict(experts=0), nsd.NSD_ERR_INVALID_ARG), (dict(topk=0), nsd.NSD_ERR_INVALID_ARG),
    (dict(topk=9), nsd.NSD_ERR_INVALID_ARG), (dict(dtype=5), nsd.NSD_ERR_INVALID_ARG),
    (dict(ld=7), nsd.NSD_ERR_INVALID_ARG),
    (dict(experts=1025, ld=1025), nsd.NSD_ERR_UNSUPPORTED)])
def test_bad_descriptors_are_refused(change, status):
    s = nsd.nsd_router(**{**dict(experts=8, topk=2, dtype=0, normalize=1, ld=8), **change})
    for call in (lambda: nsd.nsd_route_workspace_size(4, s),
                 lambda: nsd.nsd_route(4, s, 0x1000, None, 0.0, 0x1000, 0x1000, None, None, None),
                 lambda: nsd.nsd_route_vjp(4, s, 0x1000, None, 0x1000, 0x1000, None, 0.0, 1.0,
                                           0x1000, 0x1000)):
        with pytest.raises(nsd.NsdError) as e:
            call()
        assert e.value.status == status


def test_bad_arguments_are_refused():
    s = nsd.router_desc(8, 2, nsd.F32)
    P = 0x1000
    for args, status in (((-1, P, P, P, None, None), nsd.NSD_ERR_INVALID_ARG),
                         ((4, None, P, P, None, None), nsd.NSD_ERR_INVALID_ARG),
                         ((4, P, None, P, None, None), nsd.NSD_ERR_INVALID_ARG),
                         ((4, P, P, None, None, None), nsd.NSD_ERR_INVALID_ARG),
                         ((4, P, P, P, P, None), nsd.NSD_ERR_INVALID_ARG),
                         ((4, P, P, P, P, P), nsd.NSD_ERR_WORKSPACE),
                         ((2 ** 30, P, P, P, None, None), nsd.NSD_ERR_TOO_LARGE)):
        n, x, col, gate, counts, loss = args
        with pytest.raises(nsd.NsdError) as e:
            nsd.nsd_route(n, s, x, None, 0.0, col, gate, counts, loss, None)
        assert e.value.status == status, args
    with pytest.raises(nsd.NsdError) as e:
        nsd.nsd_route_vjp(4, s, P, None, None, P, None, 0.0, 1.0, P, P)
    assert e.value.status == nsd.NSD_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        nsd.router_desc(8, 2, torch.zeros(4, 9))
    with pytest.raises(ValueError):
        nsd.router_desc(8, 2, torch.zeros(8, 4).t())
    with pytest.raises(ValueError):
        nsd.router_desc(8, 2, torch.zeros(4, 8, dtype=torch.float64))


# ---------------------------------------------- definition in 64 bits (numpy)

def test_gradients_that_are_not_whole_rows_are_refused():
    """dlogits is written row after row: as part of wider rows, or of fewer bits than
    the logits, it would be written beside its place."""
    T, E, k, P = 6, 8, 2, 0x1000
    s = nsd.router_desc(E, k, torch.zeros(T, E))
    wide = torch.zeros(T, E + 4)
    for dlogits, dgate, name in ((wide[:, :E], torch.zeros(T, k), "dlogits"),
                                 (torch.zeros(T, E, dtype=torch.bfloat16), None, "dlogits"),
                                 (torch.zeros(T - 1, E), None, "dlogits"),
                                 (torch.zeros(T, E), wide[:, :k], "dgate"),
                                 (torch.zeros(T, E), torch.zeros(T, k).double(), "dgate")):
        with pytest.raises(ValueError, match=name):
            nsd.nsd_route_vjp(T, s, P, None, P, P, P, 1.0, 1.0, dgate, dlogits)
    nsd.nsd_route_vjp(0, s, P, None, P, P, P, 1.0, 1.0, torch.zeros(0, k), torch.zeros(0, E))


def softmax64(x):
    m = x.max(1, keepdims=True)
    m = np.where(np.isinf(m) & (m < 0), 0.0, m)
    e = np.exp(x - m)
    s = e.sum(1, keepdims=True)
    return np.divide(e, s, out=np.zeros_like(e), where=s > 0)


def definition(x, k, norm, skip, weight):
    """(col, gate, counts with the tokens routed, loss, p) of fp64 logits."""
    T, E = x.shape
    p = softmax64(x)
    col = np.sort(np.argsort(-x, 1, kind="stable")[:, :k], 1)
    on = np.ones(T, bool) if skip is None else skip == 0
    col = np.where(on[:, None], col, np.arange(k))
    gate = np.take_along_axis(p, col, 1)
    if norm:
        s = gate.sum(1, keepdims=True)
        gate = np.divide(gate, s, out=np.zeros_like(gate), where=s > 0)
    gate = gate * on[:, None]
    there = np.take_along_axis(x, col, 1) > -np.inf
    n = np.bincount(col[there & on[:, None]], minlength=E)
    rows = int((on & (x > -np.inf).any(1)).sum())
    P = p[on].sum(0)
    loss = weight * E * (n * P).sum() / n.sum() / rows if rows else 0.0
    return col, gate, np.append(n, rows), loss, p


def gradient(x, k, norm, skip, weight, seed, dgate, parts):
    col, gate, n, _, p = parts
    T, E = x.shape
    on = np.ones(T) if skip is None else (skip == 0).astype(float)
    u = np.zeros((T, E))
    if n[-1]:
        u += seed * weight * E * n[:E] / n[:E].sum() / n[-1]
    back = np.zeros((T, E))
    if norm:
        np.put_along_axis(back, col, gate * (dgate - (gate * dgate).sum(1, keepdims=True)), 1)
    else:
        d = np.zeros((T, E))
        np.put_along_axis(d, col, dgate, 1)
        u = u + d
    dx = (p * (u - (p * u).sum(1, keepdims=True)) + back) * on[:, None]
    mag = (p * (np.abs(u) + (p * np.abs(u)).sum(1, keepdims=True))
           + np.abs(back)) * on[:, None]
    if norm:  # what the two terms of a normalised gate's gradient hold
        m = np.zeros((T, E))
        np.put_along_axis(m, col, gate * (np.abs(dgate)
                                          + (gate * np.abs(dgate)).sum(1, keepdims=True)), 1)
        mag += m * on[:, None]
    return dx, mag


@pytest.mark.parametrize("norm", [False, True])
def test_the_gradient_is_that_of_the_definition(norm):
    """Central differences of loss and gates, the counts held."""
    rng = np.random.default_rng(1)
    T, E, k, w, seed = 5, 7, 3, 0.3, 1.7
    x, dgate = rng.standard_normal((T, E)), rng.standard_normal((T, k))
    skip = np.array([0, 0, 1, 0, 0])
    parts = definition(x, k, norm, skip, w)
    dx, _ = gradient(x, k, norm, skip, w, seed, dgate, parts)
    for t in range(T):
        for e in range(E):
            side = []
            for h in (1e-5, -1e-5):
                y = x.copy()
                y[t, e] += h
                q = definition(y, k, norm, skip, w)
                assert np.array_equal(q[0], parts[0])
                side.append(seed * q[3] + (q[1] * dgate).sum())
            assert abs((side[0] - side[1]) / 2e-5 - dx[t, e]) <= 1e-8


# ------------------------------------------------------------------ on a GPU

def run(x, k, norm, skip, weight, seed=1.0, dgate=None, stats=True):
    T, E = x.shape
    s = nsd.router_desc(E, k, x, norm)
    col = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    gate = torch.full((T, k), math.nan, device="cuda")
    counts = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda") if stats else None
    loss = torch.full((1,), math.nan, dtype=torch.float64, device="cuda") if stats else None
    ws = torch.empty(nsd.nsd_route_workspace_size(T, s), dtype=torch.uint8, device="cuda")
    nsd.nsd_route(T, s, x, skip, weight, col, gate, counts, loss, ws if stats else None)
    dx = None
    if dgate is not None:
        dx = torch.full((T, E), math.nan, dtype=x.dtype, device="cuda")
        nsd.nsd_route_vjp(T, s, x, skip, col, gate, counts, weight, seed, dgate, dx)
    torch.cuda.synchronize()
    return col, gate, counts, loss, dx


def rows(rng, T, E, dtype, pad):
    """Device rows `pad` values apart beyond E, one off a round address."""
    x = torch.from_numpy(rng.standard_normal((T, E + pad)).astype(np.float32) * 2)
    buf = torch.empty(T * (E + pad) + 1, dtype=dtype, device="cuda")[1 if pad else 0:]
    buf = buf[: T * (E + pad)].view(T, E + pad)
    buf.copy_(x)
    return buf[:, :E]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T, E, k, pad", [
    (1, 1, 1, 0), (1, 64, 8, 0), (3, 5, 5, 0), (37, 8, 2, 0), (200, 9, 3, 2), (129, 16, 4, 0),
    (64, 60, 4, 0), (65, 33, 6, 1), (300, 64, 8, 0), (5000, 128, 8, 0), (777, 129, 7, 3),
    (1000, 256, 1, 0), (500, 500, 10, 0), (90, 513, 6, 0), (700, 1024, 16, 0), (40, 96, 96, 0)])
@pytest.mark.parametrize("norm", [False, True])
def test_route_and_gradient(T, E, k, pad, norm, dtype):
    rng = np.random.default_rng(T * 1000 + E)
    x = rows(rng, T, E, dtype, pad)
    skip = torch.from_numpy((rng.random(T) < 0.2).astype(np.uint8)).cuda() if T > 3 else None
    dgate = torch.from_numpy(rng.standard_normal((T, k)).astype(np.float32)).cuda()
    col, gate, counts, loss, dx = run(x, k, norm, skip, 0.05, 0.7, dgate)
    x64, s64 = x.double().cpu().numpy(), None if skip is None else skip.cpu().numpy()
    parts = definition(x64, k, norm, s64, 0.05)
    assert np.array_equal(col.cpu().numpy(), parts[0])
    assert np.array_equal(counts.cpu().numpy(), parts[2])
    # exp2's argument and result, the sum of up to 1024 terms (each slot's by
    # halves: eight or sixteen in a lane, then log2 of the lanes), a quotient
    tol = 64 * EPS32
    assert np.all(np.abs(gate.cpu().numpy() - parts[1]) <= tol * parts[1] + 1e-30)
    assert abs(float(loss) - parts[3]) <= tol * abs(parts[3])
    ref, mag = gradient(x64, k, norm, s64, 0.05, 0.7, dgate.double().cpu().numpy(), parts)
    out = 2.0 ** -8 * np.abs(ref) if dtype == torch.bfloat16 else 0.0
    assert np.all(np.abs(dx.double().cpu().numpy() - ref) <= 4 * tol * mag + out + 1e-30)
    # the gates alone are the same bits
    col2, gate2, _, _, _ = run(x, k, norm, skip, 0.05, stats=False)
    assert torch.equal(col, col2) and torch.equal(gate, gate2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E", [6, 64, 200, 600])
def test_ties_fall_to_the_lowest_expert(E, dtype):
    x = torch.zeros(4, E, device="cuda", dtype=dtype)
    x[1, 2:] = 1.0
    x[2, ::2] = -0.0
    x[3] = torch.arange(E, device="cuda") % 3 == 1
    col, gate, counts, _, _ = run(x, 2, True, None, 1.0)
    assert col.cpu().tolist() == [[0, 1], [2, 3], [0, 1], [1, 4]]
    assert torch.all(gate == 0.5)
    assert int(counts[:E].sum()) == 8 and int(counts[E]) == 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("norm", [False, True])
def test_closed_experts_and_values_that_are_not_finite(norm, dtype):
    rng = np.random.default_rng(3)
    T, E, k = 70, 20, 3
    x = rows(rng, T, E, dtype, 0)
    low = torch.finfo(dtype).min
    x[0] = -math.inf                    # nothing is open: not routed
    x[1, 1:] = -math.inf                # one open: two stored zeros
    x[2] = low                          # the lowest value is a value
    x[3, 5:] = low
    x[4, 7] = math.nan
    x[5, 9] = math.inf
    x[6, :18] = -math.inf
    skip = torch.zeros(T, dtype=torch.uint8, device="cuda")
    skip[8] = 1
    x[8] = math.nan                     # a skipped token's logits do not matter
    dgate = torch.ones(T, k, device="cuda")
    col, gate, counts, loss, dx = run(x, k, norm, skip, 1.0, 1.0, dgate)
    c, g, d = col.cpu().numpy(), gate.cpu().numpy(), dx.float().cpu().numpy()
    assert np.all((np.diff(c, axis=1) > 0) & (c[:, 1:] < E) & (c[:, :-1] >= 0))
    assert c[0].tolist() == [0, 1, 2] and np.all(g[0] == 0) and np.all(d[0] == 0)
    assert c[1].tolist() == [0, 1, 2] and g[1].tolist() == [1, 0, 0]
    assert c[2].tolist() == [0, 1, 2] and np.allclose(g[2], 1 / 3 if norm else 1 / E, rtol=1e-6)
    assert np.all(c[3] < 5) and 7 in c[4] and 9 in c[5]
    assert np.all(np.isnan(g[4])) and np.all(np.isnan(g[5]))
    assert c[6].tolist() == [0, 18, 19] and g[6, 0] == 0
    assert c[8].tolist() == [0, 1, 2] and np.all(g[8] == 0) and np.all(d[8] == 0)
    rest = np.setdiff1d(np.arange(T), [4, 5])
    assert np.all(np.isfinite(g[rest])) and np.all(np.isfinite(d[[0, 1, 2, 3, 6, 8]]))
    n = counts.cpu().numpy()
    # all but the first and the skipped one; row 1 chose one open expert, row 6 two
    assert n[E] == T - 2 and n[:E].sum() == (T - 2) * k - 2 - 1


@pytest.mark.gpu
def test_nobody_routed_and_no_tokens():
    x = torch.randn(9, 12, device="cuda")
    skip = torch.ones(9, dtype=torch.uint8, device="cuda")
    dgate = torch.ones(9, 2, device="cuda")
    col, gate, counts, loss, dx = run(x, 2, True, skip, 1.0, 1.0, dgate)
    assert not counts.any() and float(loss) == 0 and not gate.any() and not dx.any()
    _, _, counts, loss, _ = run(x[:0], 2, True, None, 1.0, 1.0, dgate[:0])
    assert not counts.any() and float(loss) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [False, True])
def test_parts_of_the_gradient(norm):
    """Without dgate the loss's alone, without counts the gates' alone."""
    rng = np.random.default_rng(5)
    x = rows(rng, 300, 40, torch.float32, 0)
    s = nsd.router_desc(40, 4, x, norm)
    dgate = torch.from_numpy(rng.standard_normal((300, 4)).astype(np.float32) * 1e-3).cuda()
    col, gate, counts, _, _ = run(x, 4, norm, None, 1.0)
    a, b = torch.empty_like(x), torch.empty_like(x)
    nsd.nsd_route_vjp(300, s, x, None, None, None, counts, 1.0, 2.0, None, a)
    nsd.nsd_route_vjp(300, s, x, None, col, gate, None, 1.0, 2.0, dgate, b)
    x64, d64 = x.double().cpu().numpy(), dgate.double().cpu().numpy()
    parts = definition(x64, 4, norm, None, 1.0)
    for got, seed, d in ((a, 2.0, 0 * d64), (b, 0.0, d64)):
        ref, mag = gradient(x64, 4, norm, None, 1.0, seed, d, parts)
        assert np.all(np.abs(got.double().cpu().numpy() - ref) <= 256 * EPS32 * mag + 1e-30)


@pytest.mark.gpu
def test_gates_are_a_csr_of_the_library():
    """S E and its gradient through nsd_spmm and nsd_spmm_vjp."""
    from paper_2303_07030_amd.operand import DeviceCsr
    T, E, k, width = 200, 24, 3, 16
    x = torch.randn(T, E, device="cuda")
    col, gate, _, _, _ = run(x, k, True, None, 0.0)
    A = DeviceCsr(T, E, torch.arange(T + 1, dtype=torch.int32, device="cuda") * k, col.view(-1),
                  gate.view(-1), k_hint=width)
    nsd.nsd_validate_csr(A.desc, True, torch.empty(256, dtype=torch.uint8, device="cuda"))
    B, C = torch.randn(E, width, device="cuda"), torch.empty(T, width, device="cuda")
    nsd.nsd_spmm(A.desc, B, width, C, A.workspace(width))
    want = (gate.double()[..., None] * B.double()[col.long()]).sum(1)
    assert bool(((C - want).abs() <= 1e-5 * (1 + want.abs())).all())


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    x = torch.randn(4000, 64, device="cuda", dtype=torch.bfloat16)
    want = run(x, 8, True, None, 0.1, 1.0, torch.ones(4000, 8, device="cuda"))
    s = nsd.router_desc(64, 8, x, True)
    out = [torch.zeros_like(t) for t in want]
    ws = torch.empty(nsd.nsd_route_workspace_size(4000, s), dtype=torch.uint8, device="cuda")
    dgate = torch.ones(4000, 8, device="cuda")
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        nsd.nsd_route(4000, s, y, None, 0.1, *out[:4], ws)
        nsd.nsd_route_vjp(4000, s, y, None, out[0], out[1], out[2], 0.1, 1.0, dgate, out[4])
    for _ in range(3):
        y.copy_(x)
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        y.zero_()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E, k", [(8, 4), (20, 7), (64, 8), (300, 40)])
@pytest.mark.parametrize("norm", [False, True])
def test_nothing_comes_back_through_the_gates_of_closed_experts(norm, E, k, dtype):
    rng = np.random.default_rng(6)
    T = 90
    x = rows(rng, T, E, dtype, 0)
    opened = torch.from_numpy(rng.integers(0, k, T)).cuda()  # fewer than k, of some none
    order = torch.from_numpy(rng.random((T, E))).cuda().argsort(1).argsort(1)
    x.masked_fill_(order >= opened[:, None], -math.inf)
    dgate = torch.from_numpy(rng.standard_normal((T, k)).astype(np.float32)).cuda()
    col, _, _, _, _ = run(x, k, norm, None, 0.3)
    closed = x.gather(1, col.long()) == -math.inf
    assert bool(closed.any(1).all())
    want = run(x, k, norm, None, 0.3, 1.3, dgate.masked_fill(closed, 0.0))[4]
    assert bool(torch.isfinite(want).all()) and bool(want.any())
    for what in (math.nan, math.inf, -1e38):
        assert torch.equal(run(x, k, norm, None, 0.3, 1.3, dgate.masked_fill(closed, what))[4], want)
