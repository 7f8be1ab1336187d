"""Cross attention, forward and backward, against the fp64 definition, element by element within derived bounds."""
import numpy as np
import pytest
import torch

import workloads as W
from gpu_util import DEV, store, tdtype, to_np
from oracle import operators as O
from paper_2302_08005_amd import binding as B

pytestmark = pytest.mark.gpu

ROUND = {W.FP32: 2.0 ** -24, W.FP16: 2.0 ** -11, W.BF16: 2.0 ** -8}   # half a step, relative
TINY = {W.FP32: 0.0, W.FP16: 2.0 ** -25, W.BF16: 0.0}                  # half a step among the subnormal numbers of IEEE half


def view(a, dtype, stride, gap=np.nan):
    """[B,S,w] host array -> device view with `stride` elements from token to token, `gap` between the rows; and the array behind it."""
    b, s, w = a.shape
    back = torch.full((b, s, stride), gap, dtype=tdtype(dtype), device=DEV)
    back[..., :w] = torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(tdtype(dtype))
    return back[..., :w], back


class Problem:
    def __init__(self, batch, q_len, kv_len, heads, kv_heads, width, dtype=W.BF16, lens=None, scale=0.0, strided=False, big=1.0, seed=0, poison=True, steps=False):
        rng = np.random.default_rng(seed + q_len * 1000 + kv_len)
        self.__dict__.update(batch=batch, q_len=q_len, kv_len=kv_len, heads=heads, kv_heads=kv_heads, width=width, dtype=dtype)
        w, kw = heads * width, kv_heads * width
        self.lens = None if lens is None else np.resize(np.array(lens, dtype=np.int32), batch)
        qs, os_ = (w + 24, w + 8) if strided else (0, 0)
        ks = 2 * kw if strided else 0   # keys and values side by side
        self.desc = B.make_cross_attn_desc(batch=batch, q_len=q_len, kv_len=kv_len, heads=heads, kv_heads=kv_heads, head_dim=width, dtype=dtype,
                                           scale=scale, q_stride=qs, kv_stride=ks, out_stride=os_)
        self.scale = scale or None
        q, k, v, do = (store(rng.standard_normal(s), dtype) for s in ((batch, q_len, w), (batch, kv_len, kw), (batch, kv_len, kw), (batch, q_len, w)))
        q = store(q * big, dtype)
        if steps:   # values that differ in their last bit
            v = store(1.0 + 2 * ROUND[dtype] * (v > 0), dtype)
        if self.lens is not None and poison:   # what lies behind the visible states reaches nothing
            for b, n in enumerate(np.clip(self.lens, 0, kv_len)):
                k[b, n:], v[b, n:] = (np.nan, np.inf) if b % 2 else (-np.inf, np.nan)
        self.host = [x.reshape(*x.shape[:2], -1, width).astype(np.float64) for x in (q, k, v, do)]
        self.q, self.q_back = view(q, dtype, qs or w)
        self.do, _ = view(do, dtype, os_ or w)
        self.out, self.out_back = view(np.zeros_like(do), dtype, os_ or w, gap=7.0)
        self.dq, self.dq_back = view(np.zeros_like(q), dtype, qs or w, gap=7.0)
        self.kv, self.dkv = (torch.full((batch, kv_len, 2 * kw), 7.0, dtype=tdtype(dtype), device=DEV) for _ in range(2))
        if strided:
            self.kv[..., :kw], self.kv[..., kw:] = (torch.from_numpy(x).to(DEV) for x in (k, v))
            self.k, self.v, self.dk, self.dv = self.kv[..., :kw], self.kv[..., kw:], self.dkv[..., :kw], self.dkv[..., kw:]
        else:
            self.k, self.v = (view(x, dtype, kw)[0] for x in (k, v))
            self.dk, self.dv = (torch.full((batch, kv_len, kw), 7.0, dtype=tdtype(dtype), device=DEV) for _ in range(2))
        self.lse = torch.full((batch, heads, q_len), 7.0, device=DEV)
        self.dlens = None if lens is None else torch.from_numpy(self.lens).to(DEV)
        need = B.slapo_cross_attn_workspace(self.desc)
        self.ws = [torch.full((n,), 0xff, dtype=torch.uint8, device=DEV) if n else None for n in need]   # (NaN all over)

    def forward(self, lse=True):
        B.slapo_cross_attn_fwd(self.desc, self.q, self.k, self.v, self.dlens, self.out, self.lse if lse else None, self.ws[0])

    def backward(self):
        B.slapo_cross_attn_bwd(self.desc, self.q, self.k, self.v, self.dlens, self.out, self.do, self.lse, self.dq, self.dk, self.dv, self.ws[1])

    def heads_of(self, t):
        return to_np(t).reshape(*t.shape[:2], -1, self.width)

    def check(self, backward=True):
        q, k, v, do = self.host
        self.forward()
        out, lse = O.cross_forward(q, k, v, self.lens, self.scale)
        bounds = O.cross_bounds(q, k, v, do, self.lens, self.scale, ROUND[self.dtype], TINY[self.dtype], 0 if self.dtype == W.FP32 else 64)
        within(self.heads_of(self.out), out, bounds[0], "out")
        got = to_np(self.lse)
        assert np.array_equal(np.isneginf(got), np.isneginf(lse))
        seen = np.isfinite(lse)
        within(got[seen], lse[seen], bounds[1][seen], "lse")
        if backward:
            self.backward()
            for name, want, bound in zip(("dq", "dk", "dv"), O.cross_backward(q, k, v, do, self.lens, self.scale), bounds[2:]):
                within(self.heads_of(getattr(self, name)), want, bound, name)
        for back, w in ((self.out_back, self.out), (self.dq_back, self.dq)):   # columns between the rows are left alone
            gap = back[..., w.shape[-1]:]
            assert gap.numel() == 0 or bool((gap == 7.0).all())


def within(got, want, bound, name):
    off = np.abs(got - want)
    ok = off <= bound   # (NaN: not)
    assert ok.all(), (name, int((~ok).sum()), ok.size, np.argwhere(~ok)[:3].tolist(), float(np.nanmax(off / bound)))


SHAPES = [   # batch, q_len, kv_len, heads, kv_heads, head width
    (1, 1, 1, 1, 1, 64), (2, 1, 70, 4, 4, 64), (3, 1, 1000, 8, 2, 128), (2, 5, 33, 6, 2, 64), (1, 129, 257, 2, 1, 128), (3, 64, 64, 4, 4, 64),
    (2, 200, 77, 8, 2, 128), (1, 31, 1000, 2, 2, 64), (2, 333, 130, 6, 2, 64), (1, 1, 5000, 3, 1, 64), (1, 700, 1, 2, 2, 128), (9, 3, 15, 5, 5, 128),
    (1, 65, 2100, 12, 1, 64), (2, 1100, 300, 2, 2, 64),
]


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16, W.FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_all_states_visible(shape, dtype):
    Problem(*shape, dtype=dtype, big=2.0).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16, W.FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[2] > 1], ids=lambda s: "x".join(map(str, s)))
def test_lengths_with_infinities_and_nan_behind_them_and_strides(shape, dtype):
    kv = shape[2]
    lens = [kv // 2 + 1, 0, kv, 1, kv + 5, -4, kv - 1, min(kv, 64), min(kv, 65)]
    start = shape[1] % 3
    Problem(*shape, dtype=dtype, lens=lens[start:] + lens[:start], strided=True).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16, W.FP32], ids=["bf16", "fp16", "fp32"])
def test_every_length_around_a_tile(dtype):
    Problem(70, 3, 69, 2, 1, 64, dtype=dtype, lens=list(range(70))).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", [(2, 300, 900, 20, 20, 128), (3, 700, 800, 16, 16, 64), (1, 1100, 1300, 24, 8, 128)], ids=lambda s: "x".join(map(str, s)))
def test_lengths_inside_a_group_of_states_with_blocks_for_every_unit(shape, dtype):
    """Enough blocks of the widest kind: the states end inside a wavefront's 32, and rows inside the last tile."""
    Problem(*shape, dtype=dtype, lens=[shape[2] - 47, 513, 500]).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16, W.FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [(3, 200, 1, 4, 2, 64), (3, 40, 1, 2, 2, 128), (3, 4, 300, 4, 2, 64), (3, 4, 300, 2, 2, 128), (3, 100, 300, 4, 2, 64), (3, 100, 90, 2, 2, 128),
                                   (3, 600, 300, 48, 48, 128)], ids=lambda s: "x".join(map(str, s)))
def test_a_state_alone_has_gradients_of_zero(shape, dtype):
    """Its probability is 1 whatever its score."""
    p = Problem(*shape, dtype=dtype, lens=[1, shape[2], 1])
    p.forward()
    p.backward()
    for b in range(shape[0]):
        if p.lens[b] == 1:
            assert not p.dq[b].any() and not p.dk[b].any() and bool(p.dv[b, 0].any())


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", [(9, 32, 1500, 1, 1, 64), (9, 3, 1500, 8, 1, 128), (9, 1, 140, 40, 40, 128), (9, 7, 161, 8, 2, 64)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_few_rows(shape, dtype):
    """Lengths around the tiles of 32 states, of one and two tiles (which take delta another way), and whole tiles that are hidden."""
    kv = shape[2]
    Problem(*shape, dtype=dtype, lens=[1, 0, 31, 32, 33, 64, 65, kv - 1, kv - 33], strided=True).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("shape", [(2, 130, 777, 4, 2, 64), (1, 64, 5000, 1, 1, 64), (3, 700, 800, 16, 16, 64), (1, 100, 700, 2, 2, 128),
                                   (1, 40, 4000, 2, 1, 128), (2, 33, 150, 1, 1, 64), (2, 16, 3000, 2, 1, 64), (2, 8, 999, 2, 2, 128)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_where_values_differ_by_less_than_the_rounding_of_their_mean(shape, dtype):
    """dp - delta is then no larger than what the stored out is off by, which without a correction puts R = 1.3 to 5.5 times dq into dq.

    In the 2-norm, roundings being independent, relative to dq: u for the result, u (1 + R) for the gradients of the scores that are rounded in
    front of the correction, u R for the correction's factor. 32 bits: dp and delta are sums of `width` values and of size sqrt(width), off by no more than
    sqrt(width) 2^-24 of that, 8e-6, four times over with the probabilities and their sums, where dp - delta is about half of sqrt(width) 2 u, 8 u, and its
    correction R of that."""
    p = Problem(*shape, dtype=dtype, lens=[shape[2], 2 * shape[2] // 3], steps=True)
    p.check()
    q, k, v, do = p.host
    u = ROUND[dtype]
    want, out = O.cross_backward(q, k, v, do, p.lens)[0], O.cross_forward(q, k, v, p.lens)
    s, kk, _ = O._scores(q, k, v, p.lens, shape[5] ** -0.5)
    mean = (np.exp(s - out[1][..., None]) @ kk).transpose(0, 2, 1, 3) * shape[5] ** -0.5
    stored = (do * (store(out[0].astype(np.float32), dtype) - out[0])).sum(-1, keepdims=True) * mean
    norm = np.linalg.norm(want)
    times = np.linalg.norm(stored) / norm
    limit = u * (2 + 2 * times) + (1 + times) * 4 * 8e-6 / (8 * u)
    assert times > 1 and times > 10 * limit    # (else this says nothing)
    assert np.linalg.norm(p.heads_of(p.dq) - want) <= limit * norm


@pytest.mark.parametrize("width", [64, 128])
@pytest.mark.parametrize("kv_len", [31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 192])
def test_lengths_around_the_forms_of_the_kernels(kv_len, width):
    for q_len, heads, kv_heads in ((31, 2, 2), (33, 2, 2), (8, 12, 3), (130, 3, 1)):
        Problem(2, q_len, kv_len, heads, kv_heads, width, lens=[kv_len, kv_len - 1], strided=True).check()


@pytest.mark.parametrize("batch", [63, 64, 65])
def test_batches_around_those_that_are_ordered_by_length(batch):
    """Blocks of samples of several lengths are put in order up to 64 samples: every sample is still computed once."""
    Problem(batch, 2, 300, 2, 1, 64, lens=[(37 * i) % 301 for i in range(batch)]).check()
    Problem(batch, 40, 140, 1, 1, 64, lens=[140 - (i % 3) * 70 for i in range(batch)]).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16, W.FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("scale", [1e-38, 0.01, 1.0])
def test_scales(dtype, scale):
    Problem(2, 70, 150, 4, 2, 64, dtype=dtype, scale=scale, lens=[150, 99]).check()


@pytest.mark.parametrize("dtype", [W.BF16, W.FP32], ids=["bf16", "fp32"])
def test_a_state_that_takes_a_row_alone(dtype):
    """Scores of up to several hundred: the softmax is one state, late in the walk, and every earlier sum is scaled away."""
    p = Problem(1, 40, 700, 2, 2, 64, dtype=dtype, big=1.0, lens=[650])
    q, k = p.host[0], p.host[1]
    k[0, 640] = store(q[0, 7] * 16, dtype)
    p.k[0, 640] = torch.from_numpy(k[0, 640].reshape(-1)).to(DEV)
    p.check()


def test_without_lse_and_the_same_bits_again():
    p = Problem(3, 20, 500, 4, 2, 64, lens=[500, 0, 321])
    p.forward()
    p.backward()
    first = [x.clone() for x in (p.out, p.lse, p.dq, p.dk, p.dv)]
    p.out.zero_()
    p.forward(lse=False)
    assert torch.equal(p.out, first[0])
    p.forward()
    p.backward()
    for a, b in zip(first, (p.out, p.lse, p.dq, p.dk, p.dv)):
        assert torch.equal(a, b)


def test_gradients_against_differences():
    """Of sum(out * dout) in the fp32 mode: central differences along random directions, fp64 sums of fp32 outputs (2^-24 of a sum of
    ~5e3 terms of size 1 over a step of 2^-4: 3e-4 off at most by rounding; the third-order term is below 1e-3 of the slope's scale)."""
    p = Problem(2, 9, 40, 4, 2, 64, dtype=W.FP32, lens=[40, 23], poison=False)
    p.forward()
    p.backward()
    gen = torch.Generator(device=DEV).manual_seed(3)
    for t, g in ((p.q, p.dq), (p.k, p.dk), (p.v, p.dv)):
        way = torch.randn(t.shape, device=DEV, generator=gen)
        way /= way.norm()
        old, f = t.clone(), []
        for h in (2.0 ** -4, -2.0 ** -4):
            t.copy_(old + h * way)
            p.forward()
            f.append((p.out.double() * p.do.double()).sum().item())
        t.copy_(old)
        slope, want = (f[0] - f[1]) / 2.0 ** -3, (g.double() * way.double()).sum().item()
        assert abs(slope - want) <= 3e-4 + 1e-3 * g.double().norm().item(), (slope, want)


def test_refused_tensors():
    """What the library cannot see is refused before an address is taken: other types, extents, strides and places."""
    p = Problem(2, 5, 33, 4, 2, 64)
    ok = dict(q=p.q, k=p.k, v=p.v, kv_lens=None, out=p.out, lse=p.lse, ws=p.ws[0])
    bad = [dict(q=p.q.float()), dict(q=p.q[:, :4]), dict(k=p.k[..., :64]), dict(k=p.k.transpose(0, 1).contiguous().transpose(0, 1)), dict(v=p.v.cpu()),
           dict(out=p.out.half()), dict(lse=p.lse[:, :3]), dict(kv_lens=torch.ones(2, dtype=torch.int64, device=DEV)),
           dict(kv_lens=torch.ones(3, dtype=torch.int32, device=DEV))]
    for kw in bad:
        with pytest.raises(ValueError):
            B.slapo_cross_attn_fwd(p.desc, **{**ok, **kw})
    p.forward()
    for ws, status in ((p.ws[1][:16], -5), (None, -1)):
        with pytest.raises(B.SlapoError) as e:
            B.slapo_cross_attn_bwd(p.desc, p.q, p.k, p.v, None, p.out, p.do, p.lse, p.dq, p.dk, p.dv, ws)
        assert e.value.status == status
    with pytest.raises(ValueError):
        B.slapo_cross_attn_bwd(p.desc, p.q, p.k, p.v, None, p.out, p.do, p.lse, p.dq, p.dk, p.dv, p.ws[1].cpu())


def test_on_another_stream_and_replayed():
    """Captured forward and backward, replayed on new inputs between eager calls, against the eager results."""
    p = Problem(2, 37, 600, 4, 2, 64, lens=[600, 401])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.forward()
        p.backward()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward()
        p.backward()
    for i in range(4):
        p.q.copy_(torch.randn(p.q.shape, device=DEV))
        p.dlens.copy_(torch.tensor([600 - 100 * i, 64 * i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (p.out, p.lse, p.dq, p.dk, p.dv)]
        for x in (p.out, p.lse, p.dq, p.dk, p.dv):
            x.fill_(3.0)
        p.forward()
        p.backward()
        for a, b in zip(got, (p.out, p.lse, p.dq, p.dk, p.dv)):
            assert torch.equal(a, b), i


def test_samples_whose_states_lie_beyond_32_bits():
    """Three samples of 2.1 GB of states each, columns of a wide array: the last ones against 64-bit products on the device."""
    batch, kv_len, stride, w = 3, 65000, 16384, 64
    gen = torch.Generator(device=DEV).manual_seed(1)
    kv = torch.empty((batch, kv_len, stride), dtype=torch.bfloat16, device=DEV)
    kv[..., -2 * w:] = torch.randn((batch, kv_len, 2 * w), device=DEV, generator=gen)
    k, v = kv[..., -2 * w:-w], kv[..., -w:]
    for q_len in (1, 70):
        d = B.make_cross_attn_desc(batch=batch, q_len=q_len, kv_len=kv_len, heads=1, head_dim=w, kv_stride=stride)
        q = torch.randn((batch, q_len, w), device=DEV, generator=gen).to(torch.bfloat16)
        out, lse = torch.empty_like(q), torch.empty((batch, 1, q_len), device=DEV)
        need = B.slapo_cross_attn_workspace(d)
        ws = torch.empty(max(need), dtype=torch.uint8, device=DEV)
        B.slapo_cross_attn_fwd(d, q, k, v, None, out, lse, ws)
        dkv = torch.empty_like(kv)
        dq, dk, dv = torch.empty_like(q), dkv[..., -2 * w:-w], dkv[..., -w:]
        do = torch.randn(q.shape, device=DEV, generator=gen).to(torch.bfloat16)
        B.slapo_cross_attn_bwd(d, q, k, v, None, out, do, lse, dq, dk, dv, ws)
        for b in range(batch):
            p = torch.softmax(q[b].double() @ k[b].double().t().contiguous() / 8, 1)
            want = p @ v[b].double()
            # (u of the result and of the probabilities: sum p |v| is below 1 here, sqrt(2 / pi) on average; 1.1 for the 32-bit sums)
            assert bool(((out[b].double() - want).abs() <= 2.0 ** -8 * 1.1 * (want.abs() + p @ v[b].double().abs())).all())
            wdv = p.t().contiguous() @ do[b].double()
            assert bool(((dv[b].double() - wdv).abs() <= 2.0 ** -8 * 1.1 * (wdv.abs() + p.t().contiguous() @ do[b].double().abs())).all())
        del dkv


def test_two_streams_at_once_and_two_graphs_with_one_workspace():
    """Calls side by side have a workspace each; graphs that are replayed one after the other may share one."""
    a, b = Problem(2, 33, 900, 4, 2, 64, lens=[900, 77]), Problem(3, 5, 2100, 8, 2, 64, seed=5)
    want = []
    for p in (a, b):
        p.forward()
        p.backward()
        want.append([x.clone() for x in (p.out, p.lse, p.dq, p.dk, p.dv)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for p, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                p.forward()
                p.backward()
    torch.cuda.synchronize()
    for p, w in zip((a, b), want):
        assert all(torch.equal(x, y) for x, y in zip((p.out, p.lse, p.dq, p.dk, p.dv), w))
    n = max(x.numel() for p in (a, b) for x in p.ws if x is not None)
    shared = torch.empty(n, dtype=torch.uint8, device=DEV)
    graphs = []
    for p in (a, b):
        p.ws = [shared, shared]
        p.forward()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.forward()
            p.backward()
        graphs.append(g)
    for _ in range(3):
        for p, g, w in zip((a, b), graphs, want):
            for x in (p.out, p.lse, p.dq, p.dk, p.dv):
                x.fill_(3.0)
            g.replay()
        torch.cuda.synchronize()
        for p, w in zip((a, b), want):
            assert all(torch.equal(x, y) for x, y in zip((p.out, p.lse, p.dq, p.dk, p.dv), w))
