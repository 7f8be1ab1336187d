"""ctypes binding of libslapo_mi355x.so: same entry-point names as include/slapo.h, arguments
marshalled from torch tensors (used for device memory and streams only). No arithmetic here."""
from __future__ import annotations

import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SLAPO_LIB", os.path.join(HERE, "libslapo_mi355x.so"))

BF16, FP32, FP16 = 0, 1, 2
GELU, RELU = 0, 1
NT, NN, TN = 0, 1, 2
EPI_NONE, EPI_BIAS, EPI_BIAS_ACT, EPI_DACT, EPI_ADD, EPI_GATE, EPI_DGATE = 0, 1, 2, 3, 4, 5, 6
CLASSIC, LLAMA = 0, 1
ROPE_SHARED, ROPE_PER_AXIS = 0, 1
PARAM_NAMES = ("wqkv", "bqkv", "wo", "bo", "ln1_g", "ln1_b", "w1", "b1", "w2", "b2", "ln2_g", "ln2_b")


class LayerDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("seq", C.c_int32), ("hidden", C.c_int32), ("heads", C.c_int32),
                ("ffn", C.c_int32), ("causal", C.c_int32), ("dropout_p", C.c_float), ("seed", C.c_uint64),
                ("dtype", C.c_int32), ("act", C.c_int32), ("pre_ln", C.c_int32), ("layer_id", C.c_int32),
                ("ln_eps", C.c_float), ("accumulate_grads", C.c_int32), ("checkpoint", C.c_int32), ("attn_dropout_p", C.c_float),
                ("arch", C.c_int32), ("rope_base", C.c_float), ("attn_dim", C.c_int32)]


class _Ptrs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in PARAM_NAMES]


class CrossAttnDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("q_len", C.c_int32), ("kv_len", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float), ("q_stride", C.c_int64), ("kv_stride", C.c_int64),
                ("out_stride", C.c_int64)]


class RopeAxesDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("heads", C.c_int32), ("head_dim", C.c_int32), ("axes", C.c_int32), ("pairs", C.c_int32 * 4),
                ("ladder", C.c_int32), ("base", C.c_float), ("dtype", C.c_int32), ("in_stride", C.c_int64), ("out_stride", C.c_int64)]


class _Grad(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("count", C.c_int64), ("dtype", C.c_int32)]


class _GradPlan(C.Structure):
    _fields_ = [("memory", C.c_void_p), ("segments", C.c_int64)]


class SlapoError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib():
    """Loads the HIP library; there is no fallback if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(LIB_PATH)
        L.slapo_status_string.restype = C.c_char_p
        L.slapo_status_string.argtypes = [C.c_int]
        vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
        dp = C.POINTER(LayerDesc)
        sigs = {
            "slapo_layer_workspace": [dp, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)],
            "slapo_layer_saved_region": [dp, C.c_char_p, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)],
            "slapo_layer_fwd": [dp, C.POINTER(_Ptrs), vp, vp, vp, vp, vp, vp],
            "slapo_layer_bwd": [dp, C.POINTER(_Ptrs), vp, vp, vp, vp, vp, C.POINTER(_Ptrs), vp, vp],
            "slapo_stack_workspace": [dp, i32, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)],
            "slapo_stack_fwd": [dp, i32, C.POINTER(_Ptrs), vp, vp, vp, vp, vp, vp, vp],
            "slapo_stack_bwd": [dp, i32, C.POINTER(_Ptrs), vp, vp, vp, vp, vp, vp, C.POINTER(_Ptrs), vp, vp],
            "slapo_gemm": [i32, i32, i32, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp],
            "slapo_gemm_ex": [i32, i32, i32, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, i32, vp, C.c_size_t, vp],
            "slapo_gemm_workspace": [i32, i32, i32, i64, i64, i64, C.POINTER(C.c_size_t)],
            "slapo_gemm_kernel_name": [i32, i32, i32, i64, i64, i64, i32, i32, i32, C.c_char_p, C.c_size_t],
            "slapo_attn_fwd": [dp, vp, vp, vp, vp, vp],
            "slapo_attn_bwd": [dp, vp, vp, vp, vp, vp, vp, vp, vp],
            "slapo_bdrln_fwd": [dp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "slapo_bdrln_bwd": [dp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp],
            "slapo_bdrln_bwd_blocks": [i64],
            "slapo_colsum_partials": [i32, i64, i64, vp, vp, vp],
            "slapo_colsum_blocks": [i64],
            "slapo_colreduce_partials": [i32, i64, i64, i64, vp, vp, i32, vp],
            "slapo_dropout_mask": [dp, i32, i64, vp, vp],
            "slapo_rope": [dp, vp, vp, i32, vp],
            "slapo_weight_grad_workspace": [i32, i64, i64, i64, C.POINTER(C.c_size_t)],
            "slapo_weight_grad": [i32, i32, i64, i64, i64, vp, vp, vp, vp, vp],
            "slapo_weight_grad_static": [i32, i32, i64, i64, i64, vp, vp, vp, vp],
            "slapo_cross_attn_workspace": [C.POINTER(CrossAttnDesc), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)],
            "slapo_cross_attn_fwd": [C.POINTER(CrossAttnDesc), vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp],
            "slapo_cross_attn_bwd": [C.POINTER(CrossAttnDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp],
            "slapo_rope_axes": [C.POINTER(RopeAxesDesc), vp, vp, vp, i32, vp],
            "slapo_grad_plan_bytes": [i32, C.POINTER(_Grad), C.POINTER(C.c_size_t)],
            "slapo_grad_plan_build": [i32, C.POINTER(_Grad), vp, C.POINTER(_GradPlan), vp],
            "slapo_grad_sumsq": [C.POINTER(_GradPlan), i32, vp, vp],
            "slapo_grad_clip": [C.POINTER(_GradPlan), vp, C.c_float, vp, vp],
        }
        for name, args in sigs.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = C.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().slapo_status_string(int(status)).decode()


def _check(rc, where):
    if rc != 0:
        raise SlapoError(rc, where)


def _p(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors must be contiguous"
    return t.data_ptr()


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def make_desc(cfg=None, **kw) -> LayerDesc:
    """Builds a descriptor from a workloads.LayerConfig-like object and/or keyword overrides."""
    vals = dict(batch=1, seq=1, hidden=64, heads=1, ffn=64, causal=0, dropout_p=0.0, seed=0, dtype=BF16, act=GELU,
                pre_ln=0, layer_id=0, ln_eps=1e-5, accumulate_grads=0, checkpoint=0, attn_dropout_p=0.0,
                arch=CLASSIC, rope_base=10000.0, attn_dim=0)
    if cfg is not None:
        for k in vals:
            if hasattr(cfg, k):
                vals[k] = getattr(cfg, k)
    vals.update(kw)
    return LayerDesc(**vals)


def torch_dtype(desc: LayerDesc):
    return {FP32: torch.float32, FP16: torch.float16}.get(desc.dtype, torch.bfloat16)


def slapo_layer_workspace(desc: LayerDesc):
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().slapo_layer_workspace(C.byref(desc), C.byref(a), C.byref(b)), "slapo_layer_workspace")
    return a.value, b.value


def slapo_layer_saved_region(desc: LayerDesc, name: str):
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().slapo_layer_saved_region(C.byref(desc), name.encode(), C.byref(a), C.byref(b)),
           "slapo_layer_saved_region")
    return a.value, b.value


def _ptr_table(tensors: dict) -> _Ptrs:
    return _Ptrs(**{n: _p(tensors.get(n)) for n in PARAM_NAMES})   # entries a layer family does not have stay NULL


def slapo_layer_fwd(desc, params: dict, x, seqlens, y, saved, scratch, stream=None):
    pt = _ptr_table(params)
    _check(lib().slapo_layer_fwd(C.byref(desc), C.byref(pt), _p(x), _p(seqlens), _p(y), _p(saved), _p(scratch),
                                 _stream(stream)), "slapo_layer_fwd")


def slapo_layer_bwd(desc, params: dict, x, seqlens, dy, saved, dx, grads: dict, scratch, stream=None):
    pt, gt = _ptr_table(params), _ptr_table(grads)
    _check(lib().slapo_layer_bwd(C.byref(desc), C.byref(pt), _p(x), _p(seqlens), _p(dy), _p(saved), _p(dx),
                                 C.byref(gt), _p(scratch), _stream(stream)), "slapo_layer_bwd")


def slapo_gemm(dtype, layout, epilogue, act, M, N, K, A, B, Cout, bias=None, aux_in=None, aux_out=None, stream=None):
    _check(lib().slapo_gemm(dtype, layout, epilogue, act, M, N, K, _p(A), _p(B), _p(Cout), _p(bias), _p(aux_in),
                            _p(aux_out), _stream(stream)), "slapo_gemm")


GEMM_SHARED = 1


def slapo_gemm_workspace(dtype, layout, epilogue, M, N, K) -> int:
    a = C.c_size_t(0)
    _check(lib().slapo_gemm_workspace(dtype, layout, epilogue, M, N, K, C.byref(a)), "slapo_gemm_workspace")
    return a.value


def slapo_gemm_ex(dtype, layout, epilogue, act, M, N, K, A, B, Cout, bias=None, aux_in=None, aux_out=None, flags=0, ws=None,
                  stream=None):
    _check(lib().slapo_gemm_ex(dtype, layout, epilogue, act, M, N, K, _p(A), _p(B), _p(Cout), _p(bias), _p(aux_in),
                               _p(aux_out), flags, _p(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                               _stream(stream)), "slapo_gemm_ex")


def slapo_gemm_kernel_name(dtype, layout, epilogue, M, N, K, flags=0, weight_grad=0, with_ws=0) -> str:
    buf = C.create_string_buffer(320)
    _check(lib().slapo_gemm_kernel_name(dtype, layout, epilogue, M, N, K, flags, weight_grad, with_ws, buf, len(buf)),
           "slapo_gemm_kernel_name")
    return buf.value.decode()


def slapo_weight_grad_workspace(dtype, M, N, K) -> int:
    a = C.c_size_t(0)
    _check(lib().slapo_weight_grad_workspace(dtype, M, N, K, C.byref(a)), "slapo_weight_grad_workspace")
    return a.value


def slapo_weight_grad(dtype, accumulate, M, N, K, A, B, Cout, ws=None, stream=None):
    _check(lib().slapo_weight_grad(dtype, accumulate, M, N, K, _p(A), _p(B), _p(Cout), _p(ws), _stream(stream)),
           "slapo_weight_grad")


def slapo_weight_grad_static(dtype, accumulate, M, N, K, A, B, Cout, stream=None):
    _check(lib().slapo_weight_grad_static(dtype, accumulate, M, N, K, _p(A), _p(B), _p(Cout), _stream(stream)),
           "slapo_weight_grad_static")


# Which launches of several products the library's backward makes, and such a launch by itself: no entry points of its interface, but
# functions that it holds anyway, for measurements.
APART, BEHIND, BLOCKS = 0, 1, 2


class _Product(C.Structure):
    _fields_ = [("layout", C.c_int), ("M", C.c_int), ("N", C.c_int), ("K", C.c_int), ("A", C.c_void_p), ("B", C.c_void_p),
                ("C", C.c_void_p), ("aux", C.c_void_p)]


def backward_form(desc: LayerDesc) -> int:
    """A launch per product (APART), one of the layer's input gradient and all weight gradients (BEHIND), or one per block (BLOCKS)."""
    return lib()._ZN5slapo17products_togetherEPK16slapo_layer_desc(C.byref(desc))


def launch_products(dtype, products, stream=None):
    """products: (layout, M, N, K, A, B, C, aux or None) each, the tensors of those sizes; at most five."""
    if len(products) > 5:
        raise ValueError(len(products))
    table = (_Product * len(products))(*[_Product(l, m, n, k, _p(a), _p(b), _p(c), _p(aux)) for l, m, n, k, a, b, c, aux in products])
    fn = lib()._ZN5slapo15launch_productsEiiPKNS_7ProductEP12ihipStream_t
    fn.restype, fn.argtypes = None, [C.c_int, C.c_int, C.c_void_p, C.c_void_p]
    fn(dtype, len(products), C.cast(table, C.c_void_p), _stream(stream))


def slapo_attn_fwd(desc, qkv, seqlens, out, lse, stream=None):
    _check(lib().slapo_attn_fwd(C.byref(desc), _p(qkv), _p(seqlens), _p(out), _p(lse), _stream(stream)),
           "slapo_attn_fwd")


def slapo_attn_bwd(desc, qkv, seqlens, out, dout, lse, delta, dqkv, stream=None):
    _check(lib().slapo_attn_bwd(C.byref(desc), _p(qkv), _p(seqlens), _p(out), _p(dout), _p(lse), _p(delta),
                                _p(dqkv), _stream(stream)), "slapo_attn_bwd")


def slapo_bdrln_fwd(desc, site, T, r, bias, res, gamma, beta, z_out, out, mu, rstd, stream=None):
    _check(lib().slapo_bdrln_fwd(C.byref(desc), site, T, _p(r), _p(bias), _p(res), _p(gamma), _p(beta), _p(z_out),
                                 _p(out), _p(mu), _p(rstd), _stream(stream)), "slapo_bdrln_fwd")


def slapo_bdrln_bwd_blocks(T) -> int:
    return lib().slapo_bdrln_bwd_blocks(T)


def slapo_bdrln_bwd(desc, site, T, dout, z, mu, rstd, gamma, dres_in, dz_out, dr_out, partials, stream=None):
    _check(lib().slapo_bdrln_bwd(C.byref(desc), site, T, _p(dout), _p(z), _p(mu), _p(rstd), _p(gamma), _p(dres_in),
                                 _p(dz_out), _p(dr_out), _p(partials), _stream(stream)), "slapo_bdrln_bwd")


def slapo_colsum_blocks(T) -> int:
    return lib().slapo_colsum_blocks(T)


def slapo_colsum_partials(dtype, T, N, a, partials, stream=None):
    _check(lib().slapo_colsum_partials(dtype, T, N, _p(a), _p(partials), _stream(stream)), "slapo_colsum_partials")


def slapo_colreduce_partials(dtype, nblk, stride, N, partials, out, accumulate=0, stream=None):
    _check(lib().slapo_colreduce_partials(dtype, nblk, stride, N, _p(partials), _p(out), accumulate,
                                          _stream(stream)), "slapo_colreduce_partials")


def slapo_dropout_mask(desc, site, T, mask, stream=None):
    _check(lib().slapo_dropout_mask(C.byref(desc), site, T, _p(mask), _stream(stream)), "slapo_dropout_mask")


def slapo_rope(desc, qkv, table, inverse=0, stream=None):
    _check(lib().slapo_rope(C.byref(desc), _p(qkv), _p(table), inverse, _stream(stream)), "slapo_rope")


# ---- operators beside the layers. Their tensors may be views, so each is checked against the descriptor before its address is taken:
# its type, its extent, where it lies. (A wrong one would be read or written out of bounds, which the library cannot see.)
_TORCH = {BF16: torch.bfloat16, FP32: torch.float32, FP16: torch.float16}
_DTYPE = {v: k for k, v in _TORCH.items()}


def _refuse(name, t, want):
    raise ValueError(f"{name}: {tuple(t.shape)} with strides {t.stride()}, {t.dtype}, on {t.device}: {want} is wanted on the stream's device")


def _arg(name, t, dtype, shape, strides, device, optional=False):
    """Address of a tensor of exactly this kind."""
    if t is None and optional:
        return None
    # (the stride of a dimension of one element says nothing)
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_cuda or \
            (t.stride() != strides and not all(n == 1 or a == b for n, a, b in zip(shape, t.stride(), strides))):
        _refuse(name, t, f"{dtype} of shape {tuple(shape)} with strides {tuple(strides)}")
    return t.data_ptr()


def _room(t, device):
    """Address and bytes of a workspace (the library knows how many it wants)."""
    if t is None:
        return None, 0
    if not t.is_cuda or t.get_device() != device or not t.is_contiguous():
        _refuse("ws", t, "a contiguous workspace")
    return t.data_ptr(), t.numel() * t.element_size()


def _stream_and_device(stream):
    device = torch.cuda.current_device()
    if stream is None:   # (its address without a Stream object around it, which takes 1 us of a call's 6)
        return torch._C._cuda_getCurrentRawStream(device), device
    if stream.device_index != device:   # (kernels are launched on the current device)
        raise ValueError(f"the stream belongs to device {stream.device_index}, the current device is {device}")
    return stream.cuda_stream, device


def make_cross_attn_desc(**kw) -> CrossAttnDesc:
    """kv_heads defaults to heads, the strides to packed rows, scale to 1 / sqrt(head_dim)."""
    vals = dict(batch=1, q_len=1, kv_len=1, heads=1, kv_heads=kw.get("heads", 1), head_dim=64, dtype=BF16, scale=0.0, q_stride=0,
                kv_stride=0, out_stride=0)
    vals.update(kw)
    return CrossAttnDesc(**vals)


def slapo_cross_attn_workspace(desc: CrossAttnDesc):
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().slapo_cross_attn_workspace(C.byref(desc), C.byref(a), C.byref(b)), "slapo_cross_attn_workspace")
    return a.value, b.value


def _cross_shapes(d):
    """(shape, strides) of q, of k and v, of out, and of lse."""
    w, kw = d.heads * d.head_dim, d.kv_heads * d.head_dim
    qs, ks, os = d.q_stride or w, d.kv_stride or kw, d.out_stride or w
    return (((d.batch, d.q_len, w), (d.q_len * qs, qs, 1)), ((d.batch, d.kv_len, kw), (d.kv_len * ks, ks, 1)),
            ((d.batch, d.q_len, w), (d.q_len * os, os, 1)), ((d.batch, d.heads, d.q_len), (d.heads * d.q_len, d.q_len, 1)))


def slapo_cross_attn_fwd(desc, q, k, v, kv_lens, out, lse=None, ws=None, stream=None):
    """q, out [batch, q_len, heads * head_dim], k, v [batch, kv_len, kv_heads * head_dim], views with the descriptor's strides."""
    st, dev = _stream_and_device(stream)
    dt, f32, (a, b, c, e) = _TORCH[desc.dtype], torch.float32, _cross_shapes(desc)
    _check(lib().slapo_cross_attn_fwd(C.byref(desc), _arg("q", q, dt, *a, dev), _arg("k", k, dt, *b, dev), _arg("v", v, dt, *b, dev),
                                      _arg("kv_lens", kv_lens, torch.int32, (desc.batch,), (1,), dev, True), _arg("out", out, dt, *c, dev),
                                      _arg("lse", lse, f32, *e, dev, True), *_room(ws, dev), st), "slapo_cross_attn_fwd")


def slapo_cross_attn_bwd(desc, q, k, v, kv_lens, out, dout, lse, dq, dk, dv, ws, stream=None):
    st, dev = _stream_and_device(stream)
    dt, (a, b, c, e) = _TORCH[desc.dtype], _cross_shapes(desc)
    _check(lib().slapo_cross_attn_bwd(C.byref(desc), _arg("q", q, dt, *a, dev), _arg("k", k, dt, *b, dev), _arg("v", v, dt, *b, dev),
                                      _arg("kv_lens", kv_lens, torch.int32, (desc.batch,), (1,), dev, True), _arg("out", out, dt, *c, dev),
                                      _arg("dout", dout, dt, *c, dev), _arg("lse", lse, torch.float32, *e, dev), _arg("dq", dq, dt, *a, dev),
                                      _arg("dk", dk, dt, *b, dev), _arg("dv", dv, dt, *b, dev), *_room(ws, dev), st),
           "slapo_cross_attn_bwd")


def make_rope_axes_desc(rows, heads, head_dim, pairs, base=10000.0, ladder=ROPE_SHARED, dtype=BF16, in_stride=0, out_stride=0) -> RopeAxesDesc:
    """pairs: how many pairs of a head each axis turns."""
    if len(pairs) > 4:
        raise ValueError(f"{len(pairs)} axes: at most 4 are supported")
    return RopeAxesDesc(rows=rows, heads=heads, head_dim=head_dim, axes=len(pairs), pairs=(C.c_int32 * 4)(*pairs), ladder=ladder, base=base,
                        dtype=dtype, in_stride=in_stride, out_stride=out_stride)


def slapo_rope_axes(desc, positions, x, out, inverse=0, stream=None):
    """x, out: tensors whose rows (all dimensions but the last, `rows` of them, evenly `in_stride` / `out_stride` apart) hold the heads in
    front; positions int32 [rows, axes]."""
    st, dev = _stream_and_device(stream)
    dt, width = _TORCH[desc.dtype], desc.heads * desc.head_dim
    _check(lib().slapo_rope_axes(C.byref(desc), _arg("positions", positions, torch.int32, (desc.rows, desc.axes), (desc.axes, 1), dev),
                                 _rows("x", x, dt, desc.rows, width, desc.in_stride or width, dev),
                                 _rows("out", out, dt, desc.rows, width, desc.out_stride or width, dev), inverse, st), "slapo_rope_axes")


def _rows(name, t, dtype, rows, width, stride, device):
    """Address of a tensor of `rows` rows of at least `width` elements, `stride` apart."""
    shape, strides = t.shape, t.stride()
    ok = t.dtype is dtype and t.is_cuda and t.get_device() == device and shape[-1] >= width and strides[-1] == 1
    if len(shape) == 2:
        ok = ok and shape[0] == rows and (rows == 1 or strides[0] == stride)
    else:
        n = 1
        for size, step in zip(reversed(shape[:-1]), reversed(strides[:-1])):
            ok = ok and (size == 1 or step == n * stride)
            n *= size
        ok = ok and n == rows
    if not ok:
        _refuse(name, t, f"{dtype}, {rows} rows of {width} or more elements, {stride} from one to the next,")
    return t.data_ptr()


class GradPlan:
    """Which gradients take part in a norm, and where the clipped ones go (`out`, tensors of the same types and sizes; None: back where they came
    from). Built once for arrays that stay where they are; it keeps the tensors alive. One call at a time uses it."""

    def __init__(self, grads, out=None, stream=None):
        grads = list(grads)
        out = [None] * len(grads) if out is None else list(out)
        if len(out) != len(grads):
            raise ValueError(f"{len(out)} outputs for {len(grads)} gradients")
        st, self.device = _stream_and_device(stream)
        table = (_Grad * max(1, len(grads)))()
        for i, (g, o) in enumerate(zip(grads, out)):
            for t in (g, o):
                if t is not None and (t.dtype not in _DTYPE or t.dtype is not g.dtype or t.numel() != g.numel() or not t.is_contiguous()
                                      or not t.is_cuda or t.get_device() != self.device):
                    _refuse(f"gradient {i}", t, f"contiguous {g.dtype} of {g.numel()} elements")
            table[i] = _Grad(g.data_ptr(), None if o is None else o.data_ptr(), g.numel(), _DTYPE[g.dtype])
        need = C.c_size_t(0)
        _check(lib().slapo_grad_plan_bytes(len(grads), table, C.byref(need)), "slapo_grad_plan_bytes")
        self.memory = torch.empty(need.value, dtype=torch.uint8, device=f"cuda:{self.device}")
        self.tensors, self.plan, self.stream = (grads, out), _GradPlan(), st
        _check(lib().slapo_grad_plan_build(len(grads), table, self.memory.data_ptr(), C.byref(self.plan), st), "slapo_grad_plan_build")


def _scalar(name, t, dtype, device, optional=False):
    if t is None and optional:
        return None
    if t.dtype is not dtype or t.numel() != 1 or not t.is_cuda or t.get_device() != device:
        _refuse(name, t, f"one {dtype}")
    return t.data_ptr()


def _plan_stream(plan, stream):
    st, dev = _stream_and_device(stream)
    if dev != plan.device:
        raise ValueError(f"the plan belongs to device {plan.device}, the stream to {dev}")
    if st != plan.stream:   # (torch must not hand the plan's memory to others while this stream uses it)
        plan.memory.record_stream(stream if stream is not None else torch.cuda.current_stream(dev))
    return st, dev


def slapo_grad_sumsq(plan: GradPlan, sumsq, accumulate=0, stream=None):
    """sumsq: one float64."""
    st, dev = _plan_stream(plan, stream)
    _check(lib().slapo_grad_sumsq(C.byref(plan.plan), accumulate, _scalar("sumsq", sumsq, torch.float64, dev), st), "slapo_grad_sumsq")


def slapo_grad_clip(plan: GradPlan, sumsq, max_norm, norm=None, stream=None):
    """norm: one float32, or None."""
    st, dev = _plan_stream(plan, stream)
    _check(lib().slapo_grad_clip(C.byref(plan.plan), _scalar("sumsq", sumsq, torch.float64, dev), max_norm,
                                 _scalar("norm", norm, torch.float32, dev, True), st), "slapo_grad_clip")


def clip_gradients(grads, max_norm):
    """Clips the gradients in place to a norm of at most max_norm, all of them taken together; returns the norm that they had (one float32 on
    the device; nothing waits for it). Programs that clip the same arrays step by step keep a GradPlan instead."""
    plan = GradPlan(grads)
    sumsq = torch.empty(1, dtype=torch.float64, device=plan.memory.device)
    norm = torch.empty(1, dtype=torch.float32, device=plan.memory.device)
    slapo_grad_sumsq(plan, sumsq)
    slapo_grad_clip(plan, sumsq, max_norm, norm)
    return norm


def slapo_stack_workspace(desc: LayerDesc, n_layers: int):
    a, b, c = C.c_size_t(0), C.c_size_t(0), C.c_size_t(0)
    _check(lib().slapo_stack_workspace(C.byref(desc), n_layers, C.byref(a), C.byref(b), C.byref(c)),
           "slapo_stack_workspace")
    return a.value, b.value, c.value


def _ptr_tables(layers: list):
    arr = (_Ptrs * len(layers))()
    for i, t in enumerate(layers):
        arr[i] = _ptr_table(t)
    return arr


def slapo_stack_fwd(desc, params: list, x, seqlens, y, acts, saved, scratch, stream=None):
    _check(lib().slapo_stack_fwd(C.byref(desc), len(params), _ptr_tables(params), _p(x), _p(seqlens), _p(y), _p(acts),
                                 _p(saved), _p(scratch), _stream(stream)), "slapo_stack_fwd")


def slapo_stack_bwd(desc, params: list, x, seqlens, dy, acts, saved, dx, grads: list, scratch, stream=None):
    _check(lib().slapo_stack_bwd(C.byref(desc), len(params), _ptr_tables(params), _p(x), _p(seqlens), _p(dy), _p(acts),
                                 _p(saved), _p(dx), _ptr_tables(grads), _p(scratch), _stream(stream)), "slapo_stack_bwd")


class Stack:
    """Convenience holder for a stack of layers of one shape: per-layer parameters and gradients, shared workspaces."""

    def __init__(self, cfg, params_np: list, device="cuda:0", **desc_kw):
        self.desc = make_desc(cfg, **desc_kw)
        self.device = torch.device(device)
        self.dt = torch_dtype(self.desc)
        self.params = [{k: torch.from_numpy(v).to(self.device).to(self.dt).contiguous() for k, v in p.items()}
                       for p in params_np]
        self.grads = [{k: torch.zeros_like(v) for k, v in p.items()} for p in self.params]
        ab, sb, wb = slapo_stack_workspace(self.desc, len(self.params))
        mk = lambda n: torch.empty(n, dtype=torch.uint8, device=self.device) if n else None
        self.acts, self.saved, self.scratch = mk(ab), mk(sb), mk(wb)

    def to_device(self, a_np):
        return torch.from_numpy(a_np).to(self.device).to(self.dt).contiguous()

    def forward(self, x, seqlens=None):
        y = torch.empty_like(x)
        slapo_stack_fwd(self.desc, self.params, x, seqlens, y, self.acts, self.saved, self.scratch)
        return y

    def backward(self, x, seqlens, dy):
        dx = torch.empty_like(x)
        slapo_stack_bwd(self.desc, self.params, x, seqlens, dy, self.acts, self.saved, dx, self.grads, self.scratch)
        return dx

    def clip_gradients(self, max_norm):
        """Of all layers together, in place; returns their norm before."""
        return clip_gradients([g for layer in self.grads for g in layer.values()], max_norm)


class Layer:
    """Convenience holder: device parameters, gradients and the two workspaces of one layer."""

    def __init__(self, cfg, params_np: dict, device="cuda:0", **desc_kw):
        self.desc = make_desc(cfg, **desc_kw)
        self.device = torch.device(device)
        self.dt = torch_dtype(self.desc)
        self.params = {k: torch.from_numpy(v).to(self.device).to(self.dt).contiguous() for k, v in params_np.items()}
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        sb, wb = slapo_layer_workspace(self.desc)
        self.saved = torch.empty(sb, dtype=torch.uint8, device=self.device) if sb else None   # None: checkpoint mode
        self.scratch = torch.empty(wb, dtype=torch.uint8, device=self.device)

    def to_device(self, a_np):
        return torch.from_numpy(a_np).to(self.device).to(self.dt).contiguous()

    def forward(self, x, seqlens=None):
        y = torch.empty_like(x)
        slapo_layer_fwd(self.desc, self.params, x, seqlens, y, self.saved, self.scratch)
        return y

    def backward(self, x, seqlens, dy):
        dx = torch.empty_like(x)
        slapo_layer_bwd(self.desc, self.params, x, seqlens, dy, self.saved, dx, self.grads, self.scratch)
        return dx

    def clip_gradients(self, max_norm):
        """In place; returns their norm before."""
        return clip_gradients(self.grads.values(), max_norm)

    def saved_tensor(self, name):
        off, nbytes = slapo_layer_saved_region(self.desc, name)
        raw = self.saved[off:off + nbytes]
        if name in ("lse", "mu1", "rstd1", "mu2", "rstd2"):
            return raw.view(torch.float32)
        return raw.view(self.dt)
