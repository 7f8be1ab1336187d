"""The norm of many gradients and their clipping against fp64 sums."""
import numpy as np
import pytest
import torch

import workloads as W
from gpu_util import DEV, to_np
from oracle import operators as O
from paper_2302_08005_amd import binding as B

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half a step among the subnormal numbers


def arrays(sizes, dtypes, scale=1.0, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return [(torch.randn(n, device=DEV, generator=gen) * scale).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def clip(grads, out, max_norm, norm=True):
    plan = B.GradPlan(grads, out)
    sumsq, n = torch.full((1,), 9.0, dtype=torch.float64, device=DEV), torch.full((1,), 9.0, device=DEV)
    B.slapo_grad_sumsq(plan, sumsq)
    B.slapo_grad_clip(plan, sumsq, max_norm, n if norm else None)
    return sumsq.item(), n.item()


def check(grads, clipped, sumsq, norm, max_norm, before):
    want, wnorm = O.clip([to_np(b) for b in before], max_norm)
    assert abs(sumsq - wnorm ** 2) <= 1e-12 * wnorm ** 2       # 64-bit sums: n 2^-53 at the very most, n below 4e6 here and added in trees
    assert abs(norm - wnorm) <= 2.0 ** -24 * wnorm * 1.0001
    for w, c, b in zip(want, clipped, before):
        if wnorm <= max_norm:
            assert torch.equal(c, b)
        else:   # the factor and the product in 32 bits, rounded once more
            assert (np.abs(to_np(c) - w) <= np.abs(w) * (HALF_STEP[c.dtype] + 3 * 2.0 ** -24) + TINY[c.dtype]).all()


SIZES = [[1], [8], [7, 9, 0, 1, 15, 4096, 4097, 33], [3 << 18, 5, 100003], [17] * 200 + [0, 70001], [1 << 21]]
KINDS = [[torch.float32], [torch.bfloat16], [torch.float16], [torch.float32, torch.bfloat16, torch.float16]]


@pytest.mark.parametrize("kinds", KINDS, ids=lambda k: "-".join(str(x)[6:] for x in k))
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}-{sum(s)}")
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("part", [0.37, 2.0])
def test_clipping(sizes, kinds, in_place, part):
    grads = arrays(sizes, kinds)
    before = [g.clone() for g in grads]
    norm = O.clip([to_np(b) for b in before], 1.0)[1]
    out = None if in_place else [torch.full_like(g, 3.0) for g in grads]
    sumsq, got = clip(grads, out, part * norm)
    check(grads, grads if in_place else out, sumsq, got, np.float32(part * norm).item(), before)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))


@pytest.mark.parametrize("value", [1e30, 3e38, 1e-30, 1e-40])
def test_norms_that_32_bits_do_not_hold_the_square_of(value):
    g = [torch.full((1000,), value, device=DEV), torch.full((24,), value, device=DEV)]
    before = [x.clone() for x in g]
    bound = float(np.float32(g[0][0].item()) * 4) if value < 1 else 1.0
    sumsq, norm = clip(g, None, bound)
    want = before[0][0].double().item() * 32.0   # sqrt(1024)
    assert abs(sumsq - want ** 2) <= 1e-12 * want ** 2
    assert norm == float("inf") if want > 3.4e38 else abs(norm - want) <= 2.0 ** -24 * want + 2.0 ** -150
    for x, b in zip(g, before):
        w = to_np(b) * (bound / want)
        assert (np.abs(to_np(x) - w) <= np.abs(w) * 4 * 2.0 ** -24 + 2.0 ** -149).all()


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), float("-inf")])
def test_a_norm_that_is_no_number_leaves_the_gradients(bad):
    g = arrays([100, 5000], [torch.bfloat16])
    g[1][4321] = bad
    out = [torch.zeros_like(x) for x in g]
    _, norm = clip(g, out, 1.0)
    assert not np.isfinite(norm) and all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(g, out))


def test_no_gradients_and_an_infinite_bound():
    assert clip([], None, 1.0) == (0.0, 0.0)
    assert clip([torch.zeros(0, device=DEV)], None, 1.0) == (0.0, 0.0)
    g = arrays([100], [torch.float32])
    before = g[0].clone()
    clip(g, None, float("inf"), norm=False)
    assert torch.equal(g[0], before)


def test_accumulated_sums_same_bits_and_another_order_of_calls():
    a, b = arrays([5000, 77], [torch.bfloat16]), arrays([1 << 20], [torch.float32], seed=1)
    pa, pb = B.GradPlan(a), B.GradPlan(b)
    s, t = (torch.zeros(1, dtype=torch.float64, device=DEV) for _ in range(2))
    seen = set()
    for _ in range(3):
        B.slapo_grad_sumsq(pa, s)
        B.slapo_grad_sumsq(pb, s, accumulate=1)
        seen.add(s.item())
    B.slapo_grad_sumsq(pb, t)
    assert len(seen) == 1 and abs(s.item() - t.item() - O.clip([to_np(x) for x in a], 1.0)[1] ** 2) <= 1e-12 * s.item()


def test_replayed():
    """Captured with its plan, replayed on new values between eager calls of the same plan."""
    g = arrays([300000, 17, 4096], [torch.bfloat16, torch.float32])
    out = [torch.empty_like(x) for x in g]
    plan = B.GradPlan(g, out)
    s, n = torch.zeros(1, dtype=torch.float64, device=DEV), torch.zeros(1, device=DEV)

    def step():
        B.slapo_grad_sumsq(plan, s)
        B.slapo_grad_clip(plan, s, 2.0, n)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for x in g:
            x.copy_(torch.randn(x.shape, device=DEV) * 10.0 ** (-3 * (i % 2)))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out + [s, n]]
        for x in out + [s, n]:
            x.fill_(1.0)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, out + [s, n])), i


def test_holders_clip_their_own_gradients():
    cfg = W.CONFIGS["C1"].replace(dtype=W.BF16)
    stack = B.Stack(cfg, [W.make_params(cfg, layer_id=i) for i in range(2)])
    for layer in stack.grads:
        for g in layer.values():
            g.copy_(torch.randn(g.shape, device=DEV))
    before = [g.clone() for layer in stack.grads for g in layer.values()]
    norm = stack.clip_gradients(3.0)
    want, wnorm = O.clip([to_np(b) for b in before], 3.0)
    assert abs(norm.item() - wnorm) <= 2.0 ** -24 * wnorm * 1.0001
    for w, c in zip(want, [g for layer in stack.grads for g in layer.values()]):
        assert (np.abs(to_np(c) - w) <= np.abs(w) * (2.0 ** -8 + 3 * 2.0 ** -24) + TINY[c.dtype]).all()


def test_refused():
    g = arrays([100, 100], [torch.float32])
    for grads, out in (([g[0].cpu()], None), ([g[0].long()], None), (g, [g[0]]), ([g[0]], [g[1][:50]]), ([g[0]], [g[1].half()]), ([g[0][::2]], None)):
        with pytest.raises(ValueError):
            B.GradPlan(grads, out)
    for grads, out, status in (([g[0], g[0]], None, -2), ([g[0], g[0][:50]], None, -2), ([g[0][1:]], None, -4), ([g[0], g[1]], [g[1], g[0]], -2),
                               ([g[0], g[0]], [g[1], torch.empty_like(g[1])], None), ([g[0], g[1]], [g[1], None], -2)):
        if status is None:   # the same gradient twice counts twice
            B.GradPlan(grads, out)
            continue
        with pytest.raises(B.SlapoError) as e:
            B.GradPlan(grads, out)
        assert e.value.status == status
    plan = B.GradPlan(g)
    s = torch.zeros(1, dtype=torch.float64, device=DEV)
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(B.SlapoError):
            B.slapo_grad_clip(plan, s, bad)
    with pytest.raises(ValueError):
        B.slapo_grad_sumsq(plan, s.float())


def test_an_array_of_more_than_2_31_elements():
    """Sum and clipped values of its last elements: 2^31 + 77 of 1/2, and one of 3 behind them."""
    n = 2 ** 31 + 77
    g = torch.full((n + 1,), 0.5, dtype=torch.bfloat16, device=DEV)
    g[n] = 3.0
    plan = B.GradPlan([g])
    s, norm = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(1, device=DEV)
    B.slapo_grad_sumsq(plan, s)
    assert s.item() == n / 4 + 9.0   # (exact in 64 bits)
    B.slapo_grad_clip(plan, s, 1.0, norm)
    want = 1.0 / s.item() ** 0.5
    tail = g[-100:].double()
    assert bool(((tail[:-1] - 0.5 * want).abs() <= 0.5 * want * 2.0 ** -8 * 1.01).all()) and abs(tail[-1].item() - 3 * want) <= 3 * want * 2.0 ** -8 * 1.01
    assert bool((g[:-1] == g[0]).all())


def test_on_another_stream_than_the_plan_was_built_on():
    g = arrays([100000, 3], [torch.float32])
    before = [x.clone() for x in g]
    side = torch.cuda.Stream()
    s, norm = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(1, device=DEV)
    plan = B.GradPlan(g)
    side.wait_stream(torch.cuda.current_stream())
    B.slapo_grad_sumsq(plan, s, stream=side)
    with torch.cuda.stream(side):
        B.slapo_grad_clip(plan, s, 1.0, norm)
    torch.cuda.current_stream().wait_stream(side)
    check(g, g, s.item(), norm.item(), 1.0, before)


@pytest.mark.parametrize("in_place", [True, False])
def test_many_megabytes(in_place):
    """Beyond 64 MB what is written goes past the caches: every type, with ends that fill no segment; against 64 bits on the device."""
    grads = [torch.randn(n, device=DEV).to(t) for n, t in ((17 * 2 ** 20 + 5, torch.float32), (9 * 2 ** 20 + 1, torch.bfloat16), (8 * 2 ** 20 - 3, torch.float16))]
    before = [g.clone() for g in grads]
    out = None if in_place else [torch.zeros_like(g) for g in grads]
    sumsq, norm = clip(grads, out, 3.0)
    want = sum(b.double().square().sum() for b in before).item()
    assert abs(sumsq - want) <= 1e-12 * want and abs(norm - want ** 0.5) <= 2.0 ** -24 * 1.0001 * want ** 0.5
    for b, c in zip(before, grads if in_place else out):
        w = b.double() * (3.0 / want ** 0.5)
        assert bool(((c.double() - w).abs() <= w.abs() * (HALF_STEP[c.dtype] + 3 * 2.0 ** -24) + TINY[c.dtype]).all())
