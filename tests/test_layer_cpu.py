"""Host-side checks of the library of the operators around the attention forward: its symbols, its refusals (none of which may
reach the device: the pointers are fake addresses), its kernels' registers; and the references of the GPU tests against differences."""
import ctypes
import math

import pytest
import torch

import layer_util as L
import paper_2603_24517_amd as A
from paper_2603_24517_amd import build as B
from paper_2603_24517_amd import codeobj
from paper_2603_24517_amd import layer
from test_abi_cpu import _declared_symbols


def test_library_exports_its_header_and_nothing_else():
    import subprocess
    out = subprocess.run(["nm", "-D", "--defined-only", B.LAYER_LIB], check=True, capture_output=True, text=True).stdout
    names = {ln.split()[-1] for ln in out.splitlines()}
    want = {"attn_bwd", "attn_bwd_workspace", "attn_qk_norm_rope", "attn_qk_norm_rope_bwd", "attn_qk_norm_rope_bwd_workspace"}
    assert {n for n in names if not n.startswith("__hip_cuid_")} == want == set(_declared_symbols("attn_layer.h"))


def test_kernels_have_no_scratch():
    meta = codeobj.kernel_metadata(B.LAYER_LIB)
    assert len(meta) >= 8
    for name, f in meta.items():
        assert f["private_segment_fixed_size"] == 0 and f["vgpr_spill_count"] == 0, (name, f)


BWD = dict(dout=4096, dlse=None, q=8192, k=12288, v=16384, o=20480, lse=24576, dq=28672, dk=32768, dv=36864, workspace=40960,
           workspace_bytes=1 << 30, B=1, Hq=4, Hkv=2, Sq=8, Skv=8, D=128, causal=0, scale=0.1)


@pytest.mark.parametrize("kw,code", [(dict([(n, None)]), A.ATTN_E_NULL) for n in
                                     ("dout", "q", "k", "v", "o", "lse", "dq", "dk", "dv", "workspace")] + [
    (dict(B=0), A.ATTN_E_SHAPE), (dict(Hq=0), A.ATTN_E_SHAPE), (dict(Hkv=-1), A.ATTN_E_SHAPE), (dict(Sq=0), A.ATTN_E_SHAPE),
    (dict(Skv=0), A.ATTN_E_SHAPE), (dict(D=0), A.ATTN_E_SHAPE), (dict(Hq=5), A.ATTN_E_SHAPE),
    (dict(D=64), A.ATTN_E_UNSUPPORTED), (dict(Sq=2**31 - 200, Skv=1), A.ATTN_E_UNSUPPORTED), (dict(Hq=65536), A.ATTN_E_UNSUPPORTED),
    (dict(B=1 << 20, Sq=1 << 12, Hq=1 << 10, Hkv=1 << 10), A.ATTN_E_UNSUPPORTED),
    (dict(B=(1 << 31) - 1, Hq=32768, Hkv=32768, Sq=1 << 30, Skv=1 << 29), A.ATTN_E_UNSUPPORTED),
    (dict(dout=4096 + 8), A.ATTN_E_ALIGN), (dict(dv=36864 + 2), A.ATTN_E_ALIGN), (dict(workspace=40960 + 4), A.ATTN_E_ALIGN),
    (dict(lse=24576 + 2), A.ATTN_E_ALIGN), (dict(dlse=4097), A.ATTN_E_ALIGN),
    (dict(scale=math.nan), A.ATTN_E_SCALE), (dict(scale=-math.inf), A.ATTN_E_SCALE),
    (dict(workspace_bytes=100), A.ATTN_E_WORKSPACE),
])
def test_bwd_refuses_on_the_host(kw, code):
    assert A.attn_bwd(*{**BWD, **kw}.values()) == code


def test_bwd_workspace():
    assert A.attn_bwd_workspace(1, 4, 2, 8, 8, 128, False) > 0
    assert A.attn_bwd_workspace(1, 4, 3, 8, 8, 128, False) == A.ATTN_E_SHAPE
    assert A.attn_bwd_workspace(1, 4, 2, 8, 8, 64, True) == A.ATTN_E_UNSUPPORTED
    assert A.attn_bwd_workspace(1, 4, 2, 0, 8, 128, True) == A.ATTN_E_SHAPE


ROPE = dict(B=2, S=8, Hq=4, Hkv=2, D=128, q_weight=4096, k_weight=8192, weight_type=layer.FP32, cos=12288, sin=16384, places=64,
            rotated=128, pairing=0, positions=None, position_type=0, eps=1e-6)


def _rope_call(backward, rope, tensors=None, extra=()):
    r = layer.Rope(**{**ROPE, **rope})
    t = {n: layer.Heads(1 << 20, 8 * 512, 512, 128) for n in range(8 if backward else 6)}
    t.update(tensors or {})
    lib = A.load_layer()
    args = [None if x is None else ctypes.byref(x) for x in t.values()]
    if not backward:
        return lib.attn_qk_norm_rope(ctypes.byref(r), *args, None)
    return lib.attn_qk_norm_rope_bwd(ctypes.byref(r), *args, *(extra or (4096, 8192, 12288, 1 << 20)), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(cos=None), A.ATTN_E_NULL), (dict(sin=None), A.ATTN_E_NULL), (dict(q_weight=None), A.ATTN_E_NULL),
    (dict(k_weight=None), A.ATTN_E_NULL), (dict(B=0), A.ATTN_E_SHAPE), (dict(S=0), A.ATTN_E_SHAPE), (dict(Hq=-1), A.ATTN_E_SHAPE),
    (dict(Hkv=0), A.ATTN_E_SHAPE), (dict(places=0), A.ATTN_E_SHAPE), (dict(S=65), A.ATTN_E_SHAPE), (dict(D=64), A.ATTN_E_UNSUPPORTED),
    (dict(rotated=0), A.ATTN_E_UNSUPPORTED), (dict(rotated=24), A.ATTN_E_UNSUPPORTED), (dict(rotated=144), A.ATTN_E_UNSUPPORTED),
    (dict(pairing=2), A.ATTN_E_UNSUPPORTED), (dict(weight_type=2), A.ATTN_E_UNSUPPORTED), (dict(position_type=-1), A.ATTN_E_UNSUPPORTED),
    (dict(B=1 << 20, S=1 << 10, places=1 << 20), A.ATTN_E_UNSUPPORTED), (dict(Hq=(1 << 31) - 1), A.ATTN_E_UNSUPPORTED),
    (dict(B=1 << 16, S=1 << 16, places=1 << 20), A.ATTN_E_UNSUPPORTED),
    (dict(eps=-1.0), A.ATTN_E_SCALE), (dict(eps=math.nan), A.ATTN_E_SCALE), (dict(cos=12288 + 8), A.ATTN_E_ALIGN),
    (dict(q_weight=4098), A.ATTN_E_ALIGN), (dict(positions=4098), A.ATTN_E_ALIGN), (dict(positions=4100, position_type=1), A.ATTN_E_ALIGN),
])
def test_norm_rope_refuses_on_the_host(kw, code, backward):
    assert _rope_call(backward, kw) == code


@pytest.mark.parametrize("backward", [False, True])
def test_norm_rope_refuses_tensors(backward):
    pos = (0, 1, 2, 3, 4, 5, 6, 7) if backward else (0, 1, 2, 3, 4, 5)
    optional = (2, 7) if backward else (2, 5)      # values, in and out
    for n in pos:
        if n != 2:      # without values to read there is none to write
            assert _rope_call(backward, {}, {n: layer.Heads(None, 4096, 512, 128)}) == A.ATTN_E_NULL, n
            assert _rope_call(backward, {}, {n: None}) == A.ATTN_E_NULL, n
        for bad in (layer.Heads((1 << 20) + 8, 4096, 512, 128), layer.Heads(1 << 20, 4100, 512, 128), layer.Heads(1 << 20, 4096, 516, 128),
                    layer.Heads(1 << 20, 4096, 512, 129)):
            assert _rope_call(backward, {}, {n: bad}) == A.ATTN_E_ALIGN, n
        assert _rope_call(backward, {}, {n: layer.Heads(1 << 20, 1 << 60, 512, 128)}) == A.ATTN_E_UNSUPPORTED
    assert optional[0] == 2


def test_norm_rope_refuses_more_rows_than_a_launch_takes():
    sizes = dict(B=1 << 12, S=1 << 12, places=1 << 12, Hkv=8)
    assert _rope_call(False, dict(sizes, Hq=16)) == A.ATTN_E_UNSUPPORTED
    assert _rope_call(False, dict(sizes, Hq=24), {2: layer.Heads(None, 0, 0, 0)}) == A.ATTN_E_UNSUPPORTED


def test_norm_rope_backward_refuses_its_own():
    for extra, code in (((4096, None, 12288, 1 << 20), A.ATTN_E_NULL), ((4096, 8192, None, 1 << 20), A.ATTN_E_NULL),
                        ((4096, 8192, 12288, 100), A.ATTN_E_WORKSPACE), ((4097, 8192, 12288, 1 << 20), A.ATTN_E_ALIGN),
                        ((4096, 8192, 12296, 1 << 20), A.ATTN_E_ALIGN)):
        assert _rope_call(True, {}, extra=extra) == code
    assert A.load_layer().attn_qk_norm_rope_bwd_workspace(ctypes.byref(layer.Rope(**{**ROPE, "D": 96}))) == A.ATTN_E_UNSUPPORTED
    assert A.load_layer().attn_qk_norm_rope_bwd_workspace(None) == A.ATTN_E_NULL


def test_no_cpu_fallback():
    x = torch.zeros(1, 8, 2, 128, dtype=torch.bfloat16)
    lse = torch.zeros(1, 2, 8)
    cos, sin = A.rope_table(8, device="cpu")
    with pytest.raises(ValueError):
        A.attention_backward(x, x, x, x, x, lse)
    with pytest.raises(ValueError):
        A.qk_norm_rope(x, x, None, None, cos, sin)
    with pytest.raises(ValueError):
        A.qk_norm_rope_backward(x, x, x, x, None, None, cos, sin)


def test_outputs_that_overlap_are_refused():
    x = torch.zeros(2, 8, 4, 128)
    layer._check_out([x, x.transpose(1, 2), x[:, ::2], x[:, :, 1:3], x[:, :1]])
    for bad in (x[:1].expand(2, 8, 4, 128), x[:, :, :1].expand(2, 8, 4, 128), x.as_strided((2, 8, 4, 128), (4096, 512, 120, 1))):
        with pytest.raises(ValueError):
            layer._check_out([bad])


def test_rope_table():
    cos, sin = A.rope_table(1000, 64, base=500.0, device="cpu")
    c, s = L.table(1000, 64, base=500.0)
    assert cos.dtype == torch.float32 and torch.equal(cos, c) and torch.equal(sin, s)


# ----------------------------------------------------------------------------- the references against differences of the forward
@pytest.mark.parametrize("Sq,Skv,causal,Hq,Hkv", [(5, 7, True, 4, 2), (6, 4, True, 2, 1), (3, 5, False, 2, 2)])
def test_backward_reference_against_autograd(Sq, Skv, causal, Hq, Hkv):
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(2, s, h, 16, generator=g, dtype=torch.float64, requires_grad=True) for s, h in ((Sq, Hq), (Skv, Hkv), (Skv, Hkv)))
    ok = L.valid_pairs(Sq, Skv, causal)
    kk, vv = (t.repeat_interleave(Hq // Hkv, 2) for t in (k, v))
    s = torch.matmul(q.transpose(1, 2), kk.transpose(1, 2).transpose(-1, -2)) * 0.3
    rows = ok.any(-1)
    s = s.masked_fill(~ok, -1e300)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None]) * rows[:, None]
    o = torch.matmul(p, vv.transpose(1, 2)).transpose(1, 2)
    do, dlse = torch.randn(o.shape, generator=g, dtype=torch.float64), torch.randn(lse.shape, generator=g, dtype=torch.float64) * rows
    want = torch.autograd.grad([o, lse], [q, k, v], [do, dlse])
    lse_in = torch.where(rows, lse, -math.inf).detach()
    got, _, _ = L.backward64(do, q.detach(), k.detach(), v.detach(), o.detach(), lse_in, causal, 0.3, dlse)
    for a, b in zip(got, want):
        torch.testing.assert_close(a, b, rtol=1e-10, atol=1e-10)


def test_differences_reject_wrong_gradients():
    """check_slopes, which the GPU tests hold the kernel's gradients against, takes rounded gradients and refuses scaled, negated and incomplete ones."""
    Hq, Hkv, S, scale = 4, 2, 150, 128 ** -0.5
    do, dl = L.rand(1, 1, S, Hq, 128), L.rand(2, 1, Hq, S, mul=4.0).float()
    q, k, v = L.rand(3, 1, S, Hq, 128), L.rand(4, 1, S, Hkv, 128), L.rand(5, 1, S, Hkv, 128)
    o, lse = L.forward64(q, k, v, True, scale)
    good = [t.to(torch.bfloat16) for t in L.backward64(do, q, k, v, o, lse, True, scale, dl)[0]]
    L.check_slopes(good, do, dl, q, k, v, True, scale)
    for n, name in enumerate(("dq", "dk", "dv")):
        for factor in (0.0, 0.5, 0.75, 1.25, 2.0, -1.0):
            with pytest.raises(AssertionError, match=name):
                L.check_slopes([t * factor if i == n else t for i, t in enumerate(good)], do, dl, q, k, v, True, scale)
    no_delta = L.backward64(do, q, k, v, torch.zeros_like(o), lse, True, scale, dl)[0]
    no_lse = L.backward64(do, q, k, v, o, lse, True, scale)[0]
    one_head = L.backward64(do[:, :, ::2], q[:, :, ::2], k, v, o[:, :, ::2], lse[:, ::2], True, scale, dl[:, ::2])[0]
    for bad in ([no_delta[0], good[1], good[2]], [good[0], no_delta[1], good[2]], [no_lse[0], good[1], good[2]], [good[0], no_lse[1], good[2]],
                [good[0], one_head[1], good[2]], [good[0], good[1], one_head[2]]):
        with pytest.raises(AssertionError):
            L.check_slopes(bad, do, dl, q, k, v, True, scale)


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_reference_against_differences(interleaved):
    g = torch.Generator().manual_seed(6)
    x, dz = (torch.randn(1, 2, 1, 32, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(32, generator=g, dtype=torch.float64)
    cos, sin = L.table(9, 16)
    pos = torch.tensor([[7, 2]])

    def f(x, w):
        return (L.norm_rope64(x, w, cos, sin, pos, 1e-3, interleaved)[0] * dz).sum()

    (dx, _), (dw, _) = L.norm_rope_backward64(dz, x, w, cos, sin, pos, 1e-3, interleaved)
    h = 1e-6
    for t, d in ((x, dx), (w, dw)):
        for i in range(t.numel()):
            e = torch.zeros_like(t).view(-1)
            e[i] = h
            e = e.view(t.shape)
            diff = (f(x + e, w) - f(x - e, w)) / (2 * h) if t is x else (f(x, w + e) - f(x, w - e)) / (2 * h)
            assert abs(diff - d.reshape(-1)[i]) < 1e-7



# ------------------------------------------------------------------------------------------------------- the binding without a device
def test_exception_of_a_dispatch_mode_reaches_the_caller():
    from torch._subclasses.fake_tensor import FakeTensorMode
    from torch.utils._python_dispatch import TorchDispatchMode

    class Refuse(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            if func in (torch.ops.aten.empty_like.default, torch.ops.aten.empty.memory_format):
                raise KeyError("no")
            return func(*args, **(kwargs or {}))

    with FakeTensorMode():
        fake = [torch.empty(1, 4, 2, 128, device="cuda", dtype=torch.bfloat16) for _ in range(5)]
        lse, cos = torch.empty(1, 2, 4, device="cuda"), torch.empty(4, 64, device="cuda")
    do, q, k, v, o, lse, cos = (torch._to_functional_tensor(t) for t in (*fake, lse, cos))       # (torch.Tensor itself, on a device)
    for call in (lambda: A.attention_backward(do, q, k, v, o, lse), lambda: A.qk_norm_rope(q, k, None, None, cos, cos),
                 lambda: A.qk_norm_rope_backward(do, k, q, k, None, None, cos, cos)):
        with Refuse(), pytest.raises(KeyError):
            call()


@pytest.mark.parametrize("current", [0, 1])
def test_device_of_the_tensors_is_made_current_and_its_stream_taken(monkeypatch, current):
    log = []

    class Context:
        def __init__(self, index):
            log.append(("device", index))

        __enter__ = __exit__ = lambda self, *a: None

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    monkeypatch.setattr(torch.cuda, "device", Context)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 7 + index, raising=False)
    with layer._on(0):
        log.append(layer._stream(0))
    assert log == ([7] if current == 0 else [("device", 0), 7])


def test_tensors_of_several_devices_are_refused():
    class On:
        def __init__(self, index):
            self.get_device = lambda: index

    assert layer._same_device([On(1), On(1)]) == 1
    with pytest.raises(ValueError):
        layer._same_device([On(0), On(1)])


def test_autograd_forms_refuse_what_the_functions_refuse():
    from paper_2603_24517_amd import autograd as AG
    x = torch.zeros(1, 8, 4, 128, dtype=torch.bfloat16, requires_grad=True)
    cos, sin = A.rope_table(8, device="cpu")
    for call in (lambda: AG.attention(x, x, x), lambda: AG.qk_norm_rope(x, x, None, None, cos, sin), lambda: AG.qkv_norm_rope(x, 2, 1, None, None, cos, sin),
                 lambda: AG.qkv_norm_rope(x, 2, 2, None, None, cos, sin)):
        with pytest.raises(ValueError):
            call()
