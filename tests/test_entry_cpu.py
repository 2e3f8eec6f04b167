"""What smoke() holds a layer's gradients against: wrong ones do not pass."""
import math

import pytest
import torch

import __graft_entry__ as E
import layer_util as L


def _layer():
    """Tensors as the kernels leave them, from the references of the GPU tests."""
    B, S, H = 2, 300, 8
    qkv, do = L.rand(1, B, S, 3 * H, 128), L.rand(2, B, S, H, 128)
    weight = 1 + 0.2 * torch.randn(128, generator=torch.Generator().manual_seed(3))
    cos, sin = L.table(S, 128)
    at = torch.arange(S).expand(B, S)
    x = qkv.split(H, 2)
    q, k = (L.norm_rope64(t, weight, cos, sin, at, 1e-6, False)[0].to(torch.bfloat16) for t in x[:2])
    v = x[2].contiguous()
    scale = 128 ** -0.5
    o, lse = L.forward64(q, k, v, True, scale)
    dq, dk, dv = (t.to(torch.bfloat16) for t in L.backward64(do, q, k, v, o, lse, True, scale)[0])
    (dxq, _), (dwq, _) = L.norm_rope_backward64(dq, x[0], weight, cos, sin, at, 1e-6, False)
    (dxk, _), (dwk, _) = L.norm_rope_backward64(dk, x[1], weight, cos, sin, at, 1e-6, False)
    return dict(qkv=qkv, weight=weight, cos=cos, sin=sin, do=do, q=q, k=k, v=v, dq=dq, dk=dk, dv=dv,
                dqkv=torch.cat((dxq, dxk, dv.double()), 2).to(torch.bfloat16), dweight=(dwq + dwk).float())


def test_smoke_takes_right_gradients_and_no_others():
    t = _layer()
    E.check_layer(**t)
    for name in ("dq", "dk", "dv", "dqkv", "dweight"):
        for factor in (0.0, 0.9, 2.0, -1.0, math.nan):
            with pytest.raises(AssertionError, match=name):
                E.check_layer(**{**t, name: t[name] * factor})
    for part in range(3):           # queries', keys' and values' share of the projection's gradient
        bad = t["dqkv"].clone()
        bad[:, :, 8 * part:8 * part + 8] *= 0.5
        with pytest.raises(AssertionError, match="dqkv"):
            E.check_layer(**{**t, "dqkv": bad})
