"""Host-only checks of the operators' C ABI: bad arguments are refused before a device is touched."""
import ctypes as C

import pytest
import torch

from paper_2302_08005_amd import binding as B

P = 4096   # an aligned address that nothing reads


def cross(**kw):
    return B.make_cross_attn_desc(**{**dict(batch=2, q_len=8, kv_len=16, heads=4, kv_heads=2, head_dim=64), **kw})


def test_cross_attention_descriptor():
    fwd, bwd = B.slapo_cross_attn_workspace(cross())
    assert fwd >= 0 and bwd >= 2 * 4 * 8 * 4
    for kw, status in ((dict(batch=0), -2), (dict(q_len=0), -2), (dict(kv_len=-1), -2), (dict(kv_heads=3), -2), (dict(kv_heads=0), -2), (dict(head_dim=32), -3),
                       (dict(dtype=5), -3), (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2), (dict(q_stride=248), -2),
                       (dict(q_stride=260), -4), (dict(kv_stride=120), -2), (dict(kv_stride=-256), -2), (dict(out_stride=257), -4),
                       (dict(kv_len=1 << 23), -3), (dict(q_len=1 << 24), -3), (dict(batch=70000), -3), (dict(kv_len=4096, kv_stride=1 << 20), -3),
                       (dict(batch=60000, heads=64, kv_heads=64), -3), (dict(q_len=1 << 22, heads=32), -3)):
        with pytest.raises(B.SlapoError) as e:
            B.slapo_cross_attn_workspace(cross(**kw))
        assert e.value.status == status, (kw, e.value.status)


def test_cross_attention_pointers():
    L, d = B.lib(), C.byref(cross())
    assert L.slapo_cross_attn_workspace(d, None, None) == -1 and L.slapo_cross_attn_workspace(None, C.byref(C.c_size_t()), C.byref(C.c_size_t())) == -1
    for i in (0, 1, 2, 4):
        args = [P, P, P, None, P, None, P, 1 << 30, None]
        args[i] = None
        assert L.slapo_cross_attn_fwd(d, *args) == -1, i
        args[i] = P + 8
        assert L.slapo_cross_attn_fwd(d, *args) == -4, i
    for i in (0, 1, 2, 4, 5, 7, 8, 9, 10):
        args = [P, P, P, None, P, P, P, P, P, P, P, 1 << 30, None]
        args[i] = None
        assert L.slapo_cross_attn_bwd(d, *args) == -1, i
        args[i] = P + 8
        assert L.slapo_cross_attn_bwd(d, *args) == -4, i


def test_workspaces_that_are_too_small():
    L, d = B.lib(), cross(batch=1, q_len=1, kv_len=4096)   # (few blocks: the walk is split)
    fwd, bwd = B.slapo_cross_attn_workspace(d)
    assert fwd > 0 and bwd > 0
    assert L.slapo_cross_attn_fwd(C.byref(d), P, P, P, None, P, None, P, fwd - 1, None) == -5
    assert L.slapo_cross_attn_fwd(C.byref(d), P, P, P, None, P, None, None, fwd, None) == -1
    assert L.slapo_cross_attn_bwd(C.byref(d), P, P, P, None, P, P, P, P, P, P, P, bwd - 1, None) == -5


def test_division_by_the_group_is_exact():
    """The invariant that the kernels divide row numbers with, for every group size up to 300 and some beyond, at the ends of its range."""
    for g in list(range(1, 300)) + [1000, 4097, 65535]:
        bits = (g - 1).bit_length()
        mul = ((((1 << bits) - g) << 32) // g + 1) & 0xffffffff
        for r in {0, 1, g - 1, g, g + 1, 7 * g - 1, (1 << 31) - 1, (1 << 31) // g * g - 1, (1 << 30) + 3}:
            assert (((r * mul) >> 32) + r) >> bits == r // g


def rope(**kw):
    return B.make_rope_axes_desc(**{**dict(rows=6, heads=2, head_dim=64, pairs=(16, 16)), **kw})


def test_rotary_arguments():
    L = B.lib()
    call = lambda d, pos=P, x=1 << 20, y=1 << 24: L.slapo_rope_axes(C.byref(d), pos, x, y, 0, None)   # noqa: E731
    for kw, status in ((dict(rows=0), -2), (dict(heads=0), -2), (dict(head_dim=60), -4), (dict(head_dim=264), -3), (dict(pairs=(16, 17)), -2),
                       (dict(pairs=(-1, 3)), -2), (dict(pairs=()), -2), (dict(base=1.0), -2), (dict(base=float("nan")), -2), (dict(ladder=2), -3),
                       (dict(dtype=9), -3), (dict(in_stride=64), -2), (dict(out_stride=132), -4), (dict(in_stride=1 << 28), -3), (dict(rows=1 << 31), -3)):
        assert call(rope(**kw)) == status, kw
    d = rope()
    assert call(d, pos=None) == -1 and call(d, x=None) == -1 and call(d, y=None) == -1 and call(d, x=(1 << 20) + 8) == -4
    assert L.slapo_rope_axes(None, P, P, P, 0, None) == -1
    assert call(d, y=(1 << 20) + 256) == -2 and call(rope(in_stride=136), y=1 << 20) == -2   # shared memory that is not the same rows
    with pytest.raises(ValueError):
        rope(pairs=(1, 1, 1, 1, 1))


def grads(*entries):
    return len(entries), (B._Grad * max(1, len(entries)))(*[B._Grad(*e) for e in entries])


def test_gradient_plans():
    L, need, plan = B.lib(), C.c_size_t(0), B._GradPlan()
    f = B.FP32
    assert L.slapo_grad_plan_bytes(*grads((P, None, 100, f), (None, None, 0, B.BF16)), C.byref(need)) == 0 and need.value > 0
    assert L.slapo_grad_plan_bytes(0, None, C.byref(need)) == 0
    assert L.slapo_grad_plan_bytes(1, None, C.byref(need)) == -1 and L.slapo_grad_plan_bytes(-1, None, C.byref(need)) == -2
    assert L.slapo_grad_plan_bytes(*grads((P, None, 100, f)), None) == -1
    big = 1 << 20
    for entries, status in (([(P, None, -1, f)], -2), ([(P, None, 8, 7)], -3), ([(None, None, 8, f)], -1), ([(P + 8, None, 8, f)], -4), ([(P, P + 4, 8, f)], -4),
                            ([(P, None, 1 << 40, f)], -3), ([(P, None, 100, f), (P, None, 8, f)], -2), ([(P, None, 100, f), (P + 384, None, 8, f)], -2),
                            ([(P, P + 64, 100, f)], -2), ([(P, big, 100, f), (big, P, 100, f)], -2), ([(P, big, 100, f), (2 * P, big + 400 - 16, 8, f)], -2),
                            ([(P, big, 100, f), (P, 2 * big, 100, f), (P + 16, P, 4, f)], -2)):
        assert L.slapo_grad_plan_build(*grads(*entries), P, C.byref(plan), None) == status, entries
    assert L.slapo_grad_plan_build(*grads((P, None, 8, f)), None, C.byref(plan), None) == -1
    assert L.slapo_grad_plan_build(*grads((P, None, 8, f)), P + 8, C.byref(plan), None) == -4
    assert L.slapo_grad_plan_build(*grads((P, None, 8, f)), P, None, None) == -1
    good = B._GradPlan(P, 1)
    assert L.slapo_grad_sumsq(None, 0, P, None) == -1 and L.slapo_grad_sumsq(C.byref(B._GradPlan()), 0, P, None) == -1
    assert L.slapo_grad_sumsq(C.byref(good), 0, None, None) == -1 and L.slapo_grad_sumsq(C.byref(good), 0, P + 4, None) == -4
    assert L.slapo_grad_clip(C.byref(good), P, 0.0, None, None) == -2 and L.slapo_grad_clip(C.byref(good), P, float("nan"), None, None) == -2
    assert L.slapo_grad_clip(C.byref(good), None, 1.0, None, None) == -1 and L.slapo_grad_clip(C.byref(good), P, 1.0, P + 2, None) == -4


def test_host_tensors_are_refused():
    """The binding takes no address of a tensor that lies elsewhere."""
    t = torch.zeros(2, 8, 256)
    with pytest.raises(ValueError):
        B._arg("q", t, torch.float32, (2, 8, 256), t.stride(), 0)
    with pytest.raises(ValueError):
        B._room(t, 0)
    with pytest.raises(ValueError):
        B._rows("x", t, torch.float32, 16, 256, 256, 0)
    assert B._room(None, 0) == (None, 0)
