"""Binding over the C ABI of include/attn_layer.h: attention's backward pass, and the norm and position rotation of queries
and keys with their gradient.  Allocates results and workspaces with torch and runs on torch's current stream; every step of the
computation runs in the HIP kernels of csrc/attn_bwd.hip and csrc/qk_norm_rope.hip."""
import contextlib
import ctypes
import os

import paper_2603_24517_amd as _attn

LAYER_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libattn_layer_mi355x.so")
LAYER_CALL_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_layer_call.so")
HEAD = 128

ROPE_HALVES, ROPE_ADJACENT = 0, 1
BF16, FP32 = 0, 1
INT32, INT64 = 0, 1

_layer = None


class Heads(ctypes.Structure):
    """attn_heads: a BF16 tensor [B, S, H, D], strides in elements."""
    _fields_ = [("ptr", ctypes.c_void_p), ("batch", ctypes.c_longlong), ("token", ctypes.c_longlong), ("head", ctypes.c_longlong)]


class Rope(ctypes.Structure):
    """attn_rope"""
    _fields_ = [("B", ctypes.c_int), ("S", ctypes.c_int), ("Hq", ctypes.c_int), ("Hkv", ctypes.c_int), ("D", ctypes.c_int),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("weight_type", ctypes.c_int),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("places", ctypes.c_longlong), ("rotated", ctypes.c_int),
                ("pairing", ctypes.c_int), ("positions", ctypes.c_void_p), ("position_type", ctypes.c_int), ("eps", ctypes.c_float)]


def load_layer():
    """Load the built library (never builds, never falls back)."""
    global _layer
    if _layer is None:
        if not os.path.exists(LAYER_PATH):
            raise ImportError(f"{LAYER_PATH} is missing: build it with `python -m paper_2603_24517_amd.build [--all]` "
                              "(there is no fallback path)")
        lib = ctypes.CDLL(LAYER_PATH)
        vp, ci, ll, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
        rope, heads = ctypes.POINTER(Rope), ctypes.POINTER(Heads)
        lib.attn_bwd.argtypes = [vp] * 11 + [size] + [ci] * 7 + [ctypes.c_float, vp]
        lib.attn_bwd_workspace.argtypes = [ci] * 7
        lib.attn_qk_norm_rope.argtypes = [rope] + [heads] * 6 + [vp]
        lib.attn_qk_norm_rope_bwd.argtypes = [rope] + [heads] * 8 + [vp, vp, vp, size, vp]
        lib.attn_qk_norm_rope_bwd_workspace.argtypes = [rope]
        lib.attn_bwd.restype = lib.attn_qk_norm_rope.restype = lib.attn_qk_norm_rope_bwd.restype = ci
        lib.attn_bwd_workspace.restype = lib.attn_qk_norm_rope_bwd_workspace.restype = ll
        _layer = lib
    return _layer


def attn_bwd_workspace(B, Hq, Hkv, Sq, Skv, D, causal):
    """C-ABI call attn_bwd_workspace(...): bytes, or a negative status code."""
    return int(load_layer().attn_bwd_workspace(int(B), int(Hq), int(Hkv), int(Sq), int(Skv), int(D), int(bool(causal))))


def attn_bwd(dout, dlse, q, k, v, o, lse, dq, dk, dv, workspace, workspace_bytes, B, Hq, Hkv, Sq, Skv, D, causal, scale,
             stream=None):
    """C-ABI call attn_bwd(...).  Tensors (anything with .data_ptr()) or raw device addresses; returns the status code."""
    p = _attn._ptr
    return load_layer().attn_bwd(p(dout), p(dlse), p(q), p(k), p(v), p(o), p(lse), p(dq), p(dk), p(dv), p(workspace),
                                 int(workspace_bytes), int(B), int(Hq), int(Hkv), int(Sq), int(Skv), int(D),
                                 int(bool(causal)), float(scale), stream)


class _Native:
    """csrc/layer_call.cpp, loaded with the first call: attention_backward(), qk_norm_rope() and qk_norm_rope_backward() as one native
    call each.  None from one of them leaves the call to the general form here, which also words the refusals."""

    def __getattr__(self, name):
        if not os.path.exists(LAYER_CALL_PATH):
            raise ImportError(f"{LAYER_CALL_PATH} is missing: build it with `python -m paper_2603_24517_amd.build [--all]`")
        import importlib.util
        import torch  # noqa: F401  (its libraries are the module's dependencies)
        spec = importlib.util.spec_from_file_location(_attn.__name__ + "._layer_call", LAYER_CALL_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        lib = load_layer()
        module.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            lib.attn_bwd, lib.attn_bwd_workspace, lib.attn_qk_norm_rope, lib.attn_qk_norm_rope_bwd, lib.attn_qk_norm_rope_bwd_workspace)))
        self.backward, self.rope, self.rope_backward = module.backward, module.rope, module.rope_backward
        return getattr(self, name)


_native = _Native()


def _on(index):
    """A context in which device `index` is the current one (none where it is already)."""
    import torch
    return contextlib.nullcontext() if index == torch.cuda.current_device() else torch.cuda.device(index)


def _stream(index):
    from torch._C import _cuda_getCurrentRawStream
    return _cuda_getCurrentRawStream(index)


def _same_device(tensors):
    index = tensors[0].get_device()
    for t in tensors:
        if t.get_device() != index:
            raise ValueError("all tensors must be on one device")
    return index


def attention_backward(do, q, k, v, o, lse, causal=False, scale=None, dlse=None):
    """Gradients (dq, dk, dv) of attention(q, k, v, causal, scale) = (o, lse), given those of o and (if lse was used) of lse.

    do, q, o [B,Sq,Hq,D], k/v [B,Skv,Hkv,D], BF16; lse, dlse [B,Hq,Sq], FP32; contiguous, on one ROCm device.
    Returns BF16 tensors of the shapes of q, k and v.  Gradients of heads that share K and V are added up.
    """
    res = _native.backward(do, q, k, v, o, lse, causal, scale, dlse)
    if type(res) is tuple:
        return res
    if res is None:
        return _attention_backward(do, q, k, v, o, lse, causal, scale, dlse)
    raise _attn.AttnError(res, "attn_bwd")


def _attention_backward(do, q, k, v, o, lse, causal, scale, dlse):
    """attention_backward() in general: tensor subclasses, torch function modes; and its refusals."""
    import torch
    (B, Sq, Hq, D), (_, Skv, Hkv, _) = _attn._check(q, k, v)
    for t in (do, o):
        if t.dtype != torch.bfloat16 or not t.is_contiguous() or t.shape != q.shape:
            raise ValueError("do and o must be contiguous BF16 tensors of q's shape")
    for t in (lse,) if dlse is None else (lse, dlse):
        if t.dtype != torch.float32 or not t.is_contiguous() or t.shape != (B, Hq, Sq):
            raise ValueError("lse and dlse must be contiguous FP32 tensors [B, Hq, Sq]")
    index = _same_device([q, k, v, do, o, lse] + ([] if dlse is None else [dlse]))
    if scale is None:
        scale = D ** -0.5
    lib = load_layer()
    nbytes = lib.attn_bwd_workspace(B, Hq, Hkv, Sq, Skv, D, 1 if causal else 0)
    if nbytes < 0:
        raise _attn.AttnError(nbytes, "attn_bwd")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    with _on(index):
        rc = lib.attn_bwd(do.data_ptr(), None if dlse is None else dlse.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                          o.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), nbytes,
                          B, Hq, Hkv, Sq, Skv, D, 1 if causal else 0, float(scale), _stream(index))
    if rc != _attn.ATTN_OK:
        raise _attn.AttnError(rc, "attn_bwd")
    return dq, dk, dv


def rope_table(places, rotated=HEAD, base=10000.0, device="cuda"):
    """cos and sin, FP32 [places, rotated / 2], of place * base ** (-2 i / rotated); the angles are formed in 64 bits."""
    import torch
    rate = base ** (-torch.arange(0, rotated, 2, dtype=torch.float64, device=device) / rotated)
    angle = torch.arange(places, dtype=torch.float64, device=device)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def _heads(t):
    s = t.stride()
    return Heads(t.data_ptr(), s[0], s[1], s[2])


def _check_heads(name, t, shape, device_index):
    import torch
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor; there is no CPU path")
    if t.dtype != torch.bfloat16 or t.dim() != 4 or tuple(t.shape) != tuple(shape) or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"{name} must be a BF16 tensor {list(shape)} with its last dimension contiguous")
    if t.get_device() != device_index:
        raise ValueError("all tensors must be on one device")
    return t


def _check_out(out):
    """An output may be any view, but two of its elements must not share memory (strides 0, overlapping windows)."""
    for t in out:
        need = 1
        for size, stride in sorted(zip(t.shape, t.stride()), key=lambda x: x[1]):
            if size > 1:
                if stride < need:
                    raise ValueError("the elements of an output must not overlap")
                need = stride * (size - 1) + need
    return out


def _check_distinct(out):
    if len({t.data_ptr() for t in out}) < len(out):
        raise ValueError("outputs must not share memory")


def _written(out):
    """Autograd's counts of the tensors, which the kernels write to behind its back."""
    from torch.autograd.graph import increment_version
    for t in out:
        increment_version(t)


def _rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved):
    """(attn_rope, device index) of the arguments that both directions share."""
    import torch
    if not q.is_cuda:
        raise ValueError("qk_norm_rope needs device tensors; there is no CPU path")
    if q.dim() != 4 or k.dim() != 4 or k.shape[:2] != q.shape[:2] or k.shape[3] != q.shape[3]:
        raise ValueError("q and k must be [B, S, H, D] with the same B, S and D")
    index = q.get_device()
    B, S, Hq, D = q.shape
    _check_heads("q", q, q.shape, index)
    _check_heads("k", k, k.shape, index)
    if (q_weight is None) != (k_weight is None):
        raise ValueError("q_weight and k_weight: both or neither")
    weight_type = BF16
    if q_weight is not None:
        for w in (q_weight, k_weight):
            if w.dtype not in (torch.bfloat16, torch.float32) or w.dtype != q_weight.dtype or not w.is_contiguous() or w.shape != (D,):
                raise ValueError("q_weight and k_weight must be contiguous tensors [D], both BF16 or both FP32")
        weight_type = FP32 if q_weight.dtype == torch.float32 else BF16
    for t in (cos, sin):
        if t.dtype != torch.float32 or not t.is_contiguous() or t.dim() != 2 or t.shape != cos.shape:
            raise ValueError("cos and sin must be contiguous FP32 tensors [places, rotated / 2]")
    position_type = INT32
    if positions is not None:
        if positions.dtype not in (torch.int32, torch.int64) or not positions.is_contiguous() or positions.shape != (B, S):
            raise ValueError("positions must be a contiguous int32 or int64 tensor [B, S]")
        position_type = INT64 if positions.dtype == torch.int64 else INT32
    _same_device([q, cos, sin] + [t for t in (q_weight, k_weight, positions) if t is not None])
    ptr = _attn._ptr
    rope = Rope(B, S, Hq, k.shape[2], D, ptr(q_weight), ptr(k_weight), weight_type, cos.data_ptr(), sin.data_ptr(), cos.shape[0],
                2 * cos.shape[1], ROPE_ADJACENT if interleaved else ROPE_HALVES, ptr(positions), position_type, float(eps))
    return rope, index


def qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False, v=None, out=None):
    """The RMS norm of each head of q and k and the rotation of its leading elements by the token's place, in one pass.

    q [B,S,Hq,D], k (and v) [B,S,Hkv,D]: BF16, last dimension contiguous, other strides as they come (multiples of 8), so that
    slices of one projection serve.  q_weight, k_weight [D], BF16 or FP32, or None for none.  cos, sin: FP32
    [places, rotated / 2] (rope_table); positions [B,S], int32 or int64, the row of the table for each token, or
    None: token s takes row s.  A token whose place lies outside the table gets NaN.  interleaved: the pairs are
    (2 i, 2 i + 1), otherwise (i, i + rotated / 2).

    Returns (q, k), or (q, k, v) with v copied, contiguous as attention() takes them; or writes to the tensors `out`, as many,
    of any strides (a slice of a cache, say), and returns those.  They must not share memory with each other or with the inputs.
    """
    if out is not None:
        out = tuple(out)
    res = _native.rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, v, out)
    if type(res) is tuple:
        return res if out is None else out
    if res is None:
        return _qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, v, out)
    raise _attn.AttnError(res, "attn_qk_norm_rope")


def _qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, v, out):
    """qk_norm_rope() in general."""
    import torch
    rope, index = _rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    ins = [q, k] if v is None else [q, k, _check_heads("v", v, k.shape, index)]
    if out is None:
        out = tuple(torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in ins)
    else:
        if len(out) != len(ins):
            raise ValueError("out must hold a tensor for each of q, k and (if given) v")
        for t, x in zip(out, ins):
            _check_heads("out", t, x.shape, index)
        _check_out(out)
        _check_distinct(out)
    null = Heads(None, 0, 0, 0)
    args = [_heads(t) for t in ins] + [null] * (3 - len(ins)) + [_heads(t) for t in out] + [null] * (3 - len(ins))
    with _on(index):
        rc = load_layer().attn_qk_norm_rope(rope, *args, _stream(index))
    if rc != _attn.ATTN_OK:
        raise _attn.AttnError(rc, "attn_qk_norm_rope")
    _written(out)
    return out


def qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False, dv=None,
                          out=None):
    """The gradient of qk_norm_rope(q, k, ...): from the gradients dq, dk (and dv) of its results to those of its inputs.

    Arguments as there; dq, dk, dv: BF16, of the shapes of q and k, last dimension contiguous.  Returns (dq, dk, dq_weight, dk_weight)
    or, with dv, (dq, dk, dv, dq_weight, dk_weight): BF16 like the inputs, contiguous or in the tensors `out` (the slices of
    the gradient of one projection, say), which must not share memory with each other or with the inputs; the weights' gradients
    FP32 [D], None without weights.  A token whose place lies outside the table gets NaN in dq and dk and is left out of the weights' gradients.
    """
    if out is not None:
        out = tuple(out)
    res = _native.rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, dv, out)
    if type(res) is tuple:
        return res if out is None else (*out, *res[-2:])
    if res is None:
        return _qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, dv, out)
    raise _attn.AttnError(res, "attn_qk_norm_rope_bwd")


def _qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, dv, out):
    """qk_norm_rope_backward() in general."""
    import torch
    rope, index = _rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    grads = [_check_heads("dq", dq, q.shape, index), _check_heads("dk", dk, k.shape, index)]
    if dv is not None:
        grads.append(_check_heads("dv", dv, k.shape, index))
    if out is None:
        out = tuple(torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in grads)
    else:
        if len(out) != len(grads):
            raise ValueError("out must hold a tensor for each of dq, dk and (if given) dv")
        for t, x in zip(out, grads):
            _check_heads("out", t, x.shape, index)
        _check_out(out)
        _check_distinct(out)
    lib = load_layer()
    dqw = dkw = workspace = None
    nbytes = 0
    if q_weight is not None:
        nbytes = lib.attn_qk_norm_rope_bwd_workspace(rope)
        if nbytes < 0:
            raise _attn.AttnError(nbytes, "attn_qk_norm_rope_bwd")
        dqw, dkw = (torch.empty(q.shape[3], dtype=torch.float32, device=q.device) for _ in range(2))
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    null = Heads(None, 0, 0, 0)
    pad = [null] * (3 - len(grads))
    args = [_heads(t) for t in grads] + pad + [_heads(q), _heads(k)] + [_heads(t) for t in out] + pad
    ptr = _attn._ptr
    with _on(index):
        rc = lib.attn_qk_norm_rope_bwd(rope, *args, ptr(dqw), ptr(dkw), ptr(workspace), nbytes, _stream(index))
    if rc != _attn.ATTN_OK:
        raise _attn.AttnError(rc, "attn_qk_norm_rope_bwd")
    _written(out)
    return (*out, dqw, dkw)
