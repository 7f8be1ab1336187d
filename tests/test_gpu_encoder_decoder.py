"""The operators in a row, as a training step of an encoder-decoder pair uses them: image states with row and column positions through
self attention, keys and values of them, cross attention of a decoder's queries, all gradients back to the weights, and their clipping.
Against the same step in fp64 with autograd."""
import numpy as np
import pytest
import torch

import workloads as W
from gpu_util import DEV, TOL, err, store, tdtype
from oracle import operators as O
from paper_2302_08005_amd import binding as B

pytestmark = pytest.mark.gpu

BATCH, SIDE, Q, HIDDEN, HEADS, WIDTH = 2, 9, 37, 256, 4, 64
S, T, TQ = SIDE * SIDE, BATCH * SIDE * SIDE, BATCH * Q


def tensors(dtype):
    rng = np.random.default_rng(11)
    shapes = dict(x=(T, HIDDEN), z=(TQ, HIDDEN), dy=(TQ, HIDDEN), wqkv=(3 * HIDDEN, HIDDEN), wq=(HIDDEN, HIDDEN), wkv=(2 * HIDDEN, HIDDEN))
    return {k: store(rng.standard_normal(s) * (0.06 if k[0] == "w" else 1.0), dtype) for k, s in shapes.items()}


def positions():
    rows, cols = np.divmod(np.arange(S), SIDE)
    return np.tile(np.stack([rows, cols], 1).astype(np.int32) + 1000, (BATCH, 1))


def reference(t, lens, max_norm):
    """torch autograd in fp64 on the host."""
    t = {k: torch.from_numpy(v.astype(np.float64)).requires_grad_(k[0] == "w") for k, v in t.items()}
    angle = torch.from_numpy(O.rotary_angles(positions(), WIDTH, (16, 16), 10000.0, True))[:, None]

    def turn(a):
        z = torch.view_as_complex(a.reshape(T, HEADS, WIDTH // 2, 2)) * torch.polar(torch.ones_like(angle), angle)
        return torch.view_as_real(z).reshape(T, HIDDEN)

    def attend(q, k, v, mask=None):
        q, k, v = (a.reshape(BATCH, -1, HEADS, WIDTH).transpose(1, 2) for a in (q, k, v))
        return torch.nn.functional.scaled_dot_product_attention(q, k, v, attn_mask=mask).transpose(1, 2).reshape(-1, HIDDEN)

    qkv = t["x"] @ t["wqkv"].T
    states = attend(turn(qkv[:, :HIDDEN]), turn(qkv[:, HIDDEN:2 * HIDDEN]), qkv[:, 2 * HIDDEN:])
    kv = states @ t["wkv"].T
    mask = (torch.arange(S) < torch.from_numpy(lens)[:, None])[:, None, None]
    out = attend(t["z"] @ t["wq"].T, kv[:, :HIDDEN], kv[:, HIDDEN:], mask)
    out.backward(t["dy"])
    grads = {k: t[k].grad.numpy() for k in ("wqkv", "wq", "wkv")}
    clipped, norm = O.clip(list(grads.values()), max_norm)
    return out.detach().numpy(), dict(zip(grads, clipped)), norm


@pytest.mark.parametrize("dtype", [W.BF16, W.FP16, W.FP32], ids=["bf16", "fp16", "fp32"])
def test_step(dtype):
    host, lens, max_norm = tensors(dtype), np.array([S, 50], dtype=np.int32), 0.5
    want, wgrads, wnorm = reference(host, lens, max_norm)
    assert wnorm > max_norm
    dt = tdtype(dtype)
    d = {k: torch.from_numpy(v).to(DEV).to(dt) for k, v in host.items()}
    new = lambda *s: torch.empty(s, dtype=dt, device=DEV)   # noqa: E731
    pos, dlens = torch.from_numpy(positions()).to(DEV), torch.from_numpy(lens).to(DEV)
    self_desc = B.make_desc(batch=BATCH, seq=S, hidden=HIDDEN, heads=HEADS, ffn=HIDDEN, dtype=dtype)
    turn = B.make_rope_axes_desc(T, 2 * HEADS, WIDTH, (16, 16), ladder=B.ROPE_PER_AXIS, dtype=dtype, in_stride=3 * HIDDEN, out_stride=3 * HIDDEN)
    cross = B.make_cross_attn_desc(batch=BATCH, q_len=Q, kv_len=S, heads=HEADS, head_dim=WIDTH, dtype=dtype, kv_stride=2 * HIDDEN)
    ws = torch.empty(max(B.slapo_cross_attn_workspace(cross)), dtype=torch.uint8, device=DEV)
    # forward
    qkv, states, lse = new(T, 3 * HIDDEN), new(T, HIDDEN), torch.empty(BATCH, HEADS, S, device=DEV)
    B.slapo_gemm(dtype, B.NT, B.EPI_NONE, B.GELU, T, 3 * HIDDEN, HIDDEN, d["x"], d["wqkv"], qkv)
    B.slapo_rope_axes(turn, pos, qkv, qkv)
    B.slapo_attn_fwd(self_desc, qkv, None, states, lse)
    kv, q, out, clse = new(BATCH, S, 2 * HIDDEN), new(BATCH, Q, HIDDEN), new(BATCH, Q, HIDDEN), torch.empty(BATCH, HEADS, Q, device=DEV)
    B.slapo_gemm(dtype, B.NT, B.EPI_NONE, B.GELU, T, 2 * HIDDEN, HIDDEN, states, d["wkv"], kv)
    B.slapo_gemm(dtype, B.NT, B.EPI_NONE, B.GELU, TQ, HIDDEN, HIDDEN, d["z"], d["wq"], q)
    k, v = kv[..., :HIDDEN], kv[..., HIDDEN:]
    B.slapo_cross_attn_fwd(cross, q, k, v, dlens, out, clse, ws)
    # backward
    dq, dkv, dstates, dqkv = new(BATCH, Q, HIDDEN), new(BATCH, S, 2 * HIDDEN), new(T, HIDDEN), new(T, 3 * HIDDEN)
    B.slapo_cross_attn_bwd(cross, q, k, v, dlens, out, d["dy"].view(BATCH, Q, HIDDEN), clse, dq, dkv[..., :HIDDEN], dkv[..., HIDDEN:], ws)
    grads = {n: torch.empty_like(d[n]) for n in wgrads}
    B.slapo_weight_grad(dtype, 0, HIDDEN, HIDDEN, TQ, dq, d["z"], grads["wq"])
    B.slapo_weight_grad(dtype, 0, 2 * HIDDEN, HIDDEN, T, dkv, states, grads["wkv"])
    B.slapo_gemm(dtype, B.NN, B.EPI_NONE, B.GELU, T, HIDDEN, 2 * HIDDEN, dkv, d["wkv"], dstates)
    B.slapo_attn_bwd(self_desc, qkv, None, states, dstates, lse, torch.empty_like(lse), dqkv)
    B.slapo_rope_axes(turn, pos, dqkv, dqkv, inverse=1)
    B.slapo_weight_grad(dtype, 0, 3 * HIDDEN, HIDDEN, T, dqkv, d["x"], grads["wqkv"])
    norm = B.clip_gradients(grads.values(), max_norm)
    assert err(out.view(TQ, HIDDEN), want) <= TOL[dtype]
    assert abs(norm.item() - wnorm) <= TOL[dtype] * wnorm
    for n in wgrads:
        assert err(grads[n], wgrads[n]) <= TOL[dtype], n
