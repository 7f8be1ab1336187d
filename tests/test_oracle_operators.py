"""Pins of the fp64 definitions in oracle/operators.py: differences, library functions in 64 bits, invariants."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import llama_layer as LL
from oracle import operators as O


def draw(rng, b, sq, sk, h, hk, d):
    return rng.standard_normal((b, sq, h, d)), rng.standard_normal((b, sk, hk, d)), rng.standard_normal((b, sk, hk, d)), rng.standard_normal((b, sq, h, d))


@pytest.mark.parametrize("lens", [None, [3, 0]])
def test_cross_gradients_against_differences(lens):
    rng = np.random.default_rng(1)
    q, k, v, do = draw(rng, 2, 3, 5, 4, 2, 6)
    lens = None if lens is None else np.array(lens)
    got = O.cross_backward(q, k, v, do, lens, 0.7)
    for x, g in zip((q, k, v), got):
        for i in np.ndindex(x.shape):
            old, f = x[i], []
            for h in (1e-6, -1e-6):
                x[i] = old + h
                f.append(float((O.cross_forward(q, k, v, lens, 0.7)[0] * do).sum()))
            x[i] = old
            assert abs((f[0] - f[1]) / 2e-6 - g[i]) <= 1e-7 * (1 + abs(g[i]))


def test_cross_attention_against_library_in_64_bits():
    rng = np.random.default_rng(2)
    q, k, v, do = draw(rng, 2, 7, 11, 6, 2, 8)
    lens = np.array([11, 4])
    t = [torch.from_numpy(x.copy()).requires_grad_() for x in (q, k, v)]
    kk, vv = (x.repeat_interleave(3, 2).transpose(1, 2) for x in t[1:])
    mask = (torch.arange(11) < torch.from_numpy(lens)[:, None])[:, None, None]
    out = torch.nn.functional.scaled_dot_product_attention(t[0].transpose(1, 2), kk, vv, attn_mask=mask).transpose(1, 2)
    out.backward(torch.from_numpy(do))
    o, lse = O.cross_forward(q, k, v, lens)
    assert np.abs(o - out.detach().numpy()).max() < 1e-13
    for g, x in zip(O.cross_backward(q, k, v, do, lens), t):
        assert np.abs(g - x.grad.numpy()).max() < 1e-13
    s = np.einsum("bqhd,bkhd->bhqk", q, np.repeat(k, 3, 2)) / np.sqrt(8)
    assert np.abs(np.exp(s[1, :, :, :4] - lse[1][..., None]).sum(-1) - 1).max() < 1e-13


def test_cross_rows_without_states():
    rng = np.random.default_rng(3)
    q, k, v, do = draw(rng, 3, 2, 4, 2, 1, 4)
    k[1], v[1] = np.nan, np.inf
    lens = np.array([2, -3, 9])   # (beyond either end: the end)
    k[0, 2:], v[0, 2:] = np.inf, np.nan
    o, lse = O.cross_forward(q, k, v, lens)
    assert (o[1] == 0).all() and np.isneginf(lse[1]).all() and np.isfinite(o).all()
    dq, dk, dv = O.cross_backward(q, k, v, do, lens)
    assert (dq[1] == 0).all() and (dk[1] == 0).all() and (dv[1] == 0).all() and (dk[0, 2:] == 0).all() and (dv[0, 2:] == 0).all()
    assert all(np.isfinite(x).all() for x in (dq, dk, dv))


@pytest.mark.parametrize("per_axis", [False, True])
def test_rotary_turns_pairs_and_its_inverse_is_the_transpose(per_axis):
    rng = np.random.default_rng(4)
    x, w = rng.standard_normal((5, 3, 16)), rng.standard_normal((5, 3, 16))
    pos = rng.integers(-50, 2 ** 31 - 1, (5, 3)).astype(np.int32)
    pairs = (3, 0, 4)
    y = O.rotary(x, pos, pairs, per_axis=per_axis)
    assert np.array_equal(y[..., 14:], x[..., 14:])
    assert np.allclose((y * w).sum(), (x * O.rotary(w, pos, pairs, per_axis=per_axis, inverse=True)).sum(), rtol=1e-12)
    z = x[..., 0::2] + 1j * x[..., 1::2]
    step = np.array([0 / 3, 1 / 3, 2 / 3, 0 / 4, 1 / 4, 2 / 4, 3 / 4]) if per_axis else 2 * np.arange(7) / 16
    z[..., :7] *= np.exp(1j * pos[:, [0, 0, 0, 2, 2, 2, 2]] * 10000.0 ** -step)[:, None]
    assert np.abs(y[..., 0::2] - z.real).max() < 1e-6 and np.abs(y[..., 1::2] - z.imag).max() < 1e-6


def test_rotary_of_one_axis_is_the_layers_rotary():
    cfg = W.small_config(batch=2, seq=7, hidden=24, heads=3, arch=W.LLAMA, pre_ln=1)
    qkv = np.random.default_rng(5).standard_normal((14, 72))
    want = LL.rope_apply(cfg, qkv)
    pos = np.tile(np.arange(7, dtype=np.int32), 2)[:, None]
    got = O.rotary(qkv[..., :48].reshape(14, 6, 8), pos, (4,), base=cfg.rope_base)
    assert np.abs(got.reshape(14, 48) - want[:, :48]).max() < 1e-13


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]]), np.zeros(0)]
    c, norm = O.clip(g, 1.0)
    assert norm == 5.0 and np.allclose(c[0], [0.6, 0]) and np.allclose(c[1], 0.8)
    assert O.clip(g, 5.0)[0][1][0, 0] == 4.0 and O.clip([np.array([np.inf, 2.0])], 1.0)[0][0][1] == 2.0
