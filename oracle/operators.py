"""Plain fp64 definitions of the operators beside the layers: cross attention, rotary positions of several axes, gradient clipping.

`cross_bounds` and `rotary_bound` give, element by element, how far a result may be off that takes the same sums in 32 bits and rounds
what the kernels round: u = half a step of the storage type, relative to the value (eps / 2)."""
from __future__ import annotations

import numpy as np


def _scores(q, k, v, lens, scale):
    """q [B,Sq,h,d], k, v [B,Sk,hk,d] -> scores [B,h,Sq,Sk] (hidden: -inf), k and v per query head [B,h,Sk,d] with zeros for hidden states."""
    group = q.shape[2] // k.shape[2]
    k, v = (np.repeat(x, group, axis=2).transpose(0, 2, 1, 3) for x in (k, v))
    hidden = np.zeros((k.shape[0], 1, 1, k.shape[2]), bool) if lens is None else \
        (np.arange(k.shape[2]) >= np.clip(lens, 0, k.shape[2])[:, None])[:, None, None]
    seen = ~np.swapaxes(np.broadcast_to(hidden, hidden.shape), 2, 3)
    k, v = np.where(seen, k, 0.0), np.where(seen, v, 0.0)
    s = q.transpose(0, 2, 1, 3) @ k.transpose(0, 1, 3, 2) * scale
    return np.where(hidden, -np.inf, s), k, v


def cross_forward(q, k, v, lens=None, scale=None):
    """out [B,Sq,h,d], lse [B,h,Sq]; a row without states: 0 and -inf."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    s, _, v = _scores(q, k, v, lens, scale)
    top = s.max(-1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    e = np.exp(s - top)
    total = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = (top + np.log(total))[..., 0]
        p = np.where(total > 0, e / total, 0.0)
    return (p @ v).transpose(0, 2, 1, 3), lse


def cross_backward(q, k, v, dout, lens=None, scale=None):
    """dq, dk, dv in the shapes of q, k, v."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    group = q.shape[2] // k.shape[2]
    s, kk, vv = _scores(q, k, v, lens, scale)
    o, lse = cross_forward(q, k, v, lens, scale)
    with np.errstate(invalid="ignore"):
        p = np.where(np.isfinite(s), np.exp(s - lse[..., None]), 0.0)
    do, qt = dout.transpose(0, 2, 1, 3), q.transpose(0, 2, 1, 3)
    ds = p * (do @ vv.transpose(0, 1, 3, 2) - (do * o.transpose(0, 2, 1, 3)).sum(-1, keepdims=True))

    def over_group(x):   # [B,h,Sk,d] -> [B,Sk,hk,d]
        return x.reshape(x.shape[0], -1, group, *x.shape[2:]).sum(2).transpose(0, 2, 1, 3)

    return ((ds @ kk).transpose(0, 2, 1, 3) * scale, over_group(ds.transpose(0, 1, 3, 2) @ qt) * scale,
            over_group(p.transpose(0, 1, 3, 2) @ do))


def cross_bounds(q, k, v, dout, lens, scale, u, tiny, stored_above):
    """Bounds on the errors of (out, lse, dq, dk, dv). In samples of more than `stored_above` visible states backward takes delta = dout . out of the
    stored out, which is off by its own bound, else as the sum of p dp.

    e = 2^-24. A score is a sum of d products: off by at most (d + 2) e scale sum|q k|, and with the exponential (3e relative, and the
    argument's own rounding, 2e times its size) a probability by `es` relative; its row sum as much again, and n e for the additions. What
    multiplies v (and dout, k, q in backward) is rounded to the storage type: u relative, `tiny` absolute (half a step among the
    subnormal numbers of IEEE half, where the largest probability of a row is 1 in forward; 0 for types with the exponents of fp32).
    The sums of the products add n e of their absolute values, the result is rounded once (u, or `tiny` where it is subnormal)."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    group, d, e = q.shape[2] // k.shape[2], q.shape[3], 2.0 ** -24
    s, kk, vv = _scores(q, k, v, lens, scale)
    o, lse = cross_forward(q, k, v, lens, scale)
    with np.errstate(invalid="ignore"):
        p = np.where(np.isfinite(s), np.exp(s - lse[..., None]), 0.0)
        size = np.where(np.isfinite(s), np.abs(s), 0.0).max(-1, keepdims=True) + np.where(np.isfinite(lse), np.abs(lse), 0.0)[..., None]
    qt, do = q.transpose(0, 2, 1, 3), dout.transpose(0, 2, 1, 3)
    n, m = s.shape[-1], s.shape[-2] * group
    es = (d + 2) * e * scale * (np.abs(qt) @ np.abs(kk).transpose(0, 1, 3, 2)).max(-1, keepdims=True) + 2 * e * size + 3 * e
    row = es + (n + 4) * e                       # of a row sum, relative
    b_out = u * np.abs(o.transpose(0, 2, 1, 3)) + p @ np.abs(vv) * (u + es + row + (n + 4) * e) + tiny * np.abs(vv).sum(2, keepdims=True)
    b_lse = (row + 2 * e * (1 + size))[..., 0]
    ep = es + row + 2 * e * (1 + size)           # of a probability taken from lse, relative
    dp = do @ vv.transpose(0, 1, 3, 2)
    delta = (do * o.transpose(0, 2, 1, 3)).sum(-1, keepdims=True)
    seen = np.isfinite(s).any(2, keepdims=True).sum(-1, keepdims=True)
    size_dp = np.abs(do) @ np.abs(vv).transpose(0, 1, 3, 2)   # (as much for delta = sum p dp, and n e and es more for its sum)
    size_delta = (p * size_dp).sum(-1, keepdims=True)
    sums = (d + 2) * e * (size_dp + size_delta) + (es + row + (n + 4) * e) * size_delta + \
        np.where(seen > stored_above, (np.abs(do) * (b_out + tiny)).sum(-1, keepdims=True), 0.0)
    ds = p * (dp - delta)
    b_ds = p * sums + np.abs(ds) * (ep + u + 2 * e) + tiny
    b_p = p * (ep + u) + tiny

    def over_group(x):
        return x.reshape(x.shape[0], -1, group, *x.shape[2:]).sum(2).transpose(0, 2, 1, 3)

    hidden = np.isinf(s)   # (exactly 0 there)
    b_ds, b_p = np.where(hidden, 0.0, b_ds), np.where(hidden, 0.0, b_p)
    dq, dk, dv = cross_backward(q, k, v, dout, lens, scale)
    b_dq = u * np.abs(dq) + ((b_ds + (n + 4) * e * np.abs(ds)) @ np.abs(kk)).transpose(0, 2, 1, 3) * scale
    b_dk = u * np.abs(dk) + over_group((b_ds + (m + 4) * e * np.abs(ds)).transpose(0, 1, 3, 2) @ np.abs(qt)) * scale
    b_dv = u * np.abs(dv) + over_group((b_p + (m + 4) * e * p).transpose(0, 1, 3, 2) @ np.abs(do))
    return tuple(b + 1e-30 + (0.0 if i == 1 else tiny) for i, b in enumerate((b_out.transpose(0, 2, 1, 3), b_lse, b_dq, b_dk, b_dv)))


def rotary_angles(positions, head_dim, pairs, base, per_axis):
    """[rows, sum(pairs)] angles."""
    out, first = [], 0
    for a, n in enumerate(pairs):
        i = np.arange(n, dtype=np.float64)
        step = i / max(n, 1) if per_axis else 2.0 * (first + i) / head_dim
        out.append(positions[:, a:a + 1].astype(np.float64) * np.float64(base) ** -step)
        first += n
    return np.concatenate(out, 1)


def rotary(x, positions, pairs, base=10000.0, per_axis=False, inverse=False):
    """x [rows, heads, head_dim]."""
    angle = rotary_angles(positions, x.shape[-1], pairs, base, per_axis)[:, None]
    t = 2 * angle.shape[-1]
    c, s = np.cos(angle), -np.sin(angle) if inverse else np.sin(angle)
    y = np.array(x, dtype=np.float64)
    a, b = y[..., 0:t:2].copy(), y[..., 1:t:2].copy()
    y[..., 0:t:2], y[..., 1:t:2] = a * c - b * s, a * s + b * c
    return y


def rotary_bound(x, y, positions, pairs, u, tiny, base=10000.0, per_axis=False):
    """The angle in 64 bits is off by 4 of their roundings relative to it, the cosine and sine by 6 roundings of 32 bits (argument, function), the
    pair's two products and their sum by 3, the result by u (or `tiny` where it is subnormal)."""
    angle = np.abs(rotary_angles(positions, x.shape[-1], pairs, base, per_axis))[:, None]
    b = np.zeros(y.shape)
    t = 2 * angle.shape[-1]
    pair = np.hypot(x[..., 0:t:2], x[..., 1:t:2]) * 1.5 * (4 * 2.0 ** -53 * angle + 9 * 2.0 ** -24)
    b[..., 0:t:2], b[..., 1:t:2] = pair, pair
    b[..., :t] += u * np.abs(y[..., :t]) + tiny
    return b


def clip(grads, max_norm):
    """(clipped, norm) of a list of arrays."""
    norm = float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))
    factor = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return [g.astype(np.float64) * factor for g in grads], norm
