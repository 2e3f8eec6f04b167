"""The differentiable forms: one projection -> norm and rotation -> attention -> a number, and back.  Each stage's gradient is held against
64-bit arithmetic on the tensors that the stage really got (layer_util says how far it may be off)."""
import math

import pytest
import torch

import layer_util as L
import paper_2603_24517_amd as A
from paper_2603_24517_amd import autograd as AG

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


def leaf(t):
    return t.detach().cuda().requires_grad_()


@pytest.mark.parametrize("B,S,Hq,Hkv,rotated,dtype,interleaved,causal", [
    (2, 70, 4, 2, 128, torch.float32, False, True), (1, 133, 8, 2, 64, torch.bfloat16, True, True), (1, 40, 3, 3, 96, None, False, False)])
def test_layer(B, S, Hq, Hkv, rotated, dtype, interleaved, causal):
    qkv = leaf(L.rand(1, B, S, Hq + 2 * Hkv, 128))
    g = torch.Generator().manual_seed(2)
    qw = kw = None
    if dtype is not None:
        qw, kw = (leaf((1 + 0.3 * torch.randn(128, generator=g)).to(dtype)) for _ in range(2))
    cos, sin = (t.cuda() for t in L.table(200, rotated))
    pos = torch.randint(0, 200, (B, S), generator=g).cuda()
    q, k, v = AG.qkv_norm_rope(qkv, Hq, Hkv, qw, kw, cos, sin, pos, 1e-6, interleaved)
    o, lse = AG.attention(q, k, v, causal)
    for t in (q, k, v, o):
        t.retain_grad()
    do, dl = L.rand(3, B, S, Hq, 128).cuda(), L.rand(4, B, Hq, S).float().cuda()
    ((o.float() * do.float()).sum() + (lse * dl).sum()).backward()
    assert torch.equal(o.grad, do)
    c = [t.detach().cpu() for t in (do, q, k, v, o, lse)]
    L.check_backward((q.grad, k.grad, v.grad), L.backward64(*c, causal, SCALE, dl.cpu()), "attention")
    x, at = qkv.detach().cpu(), pos.cpu()
    parts = [Hq, Hkv, Hkv]
    xs, gs = x.split(parts, 2), qkv.grad.split(parts, 2)
    for n, (t, w) in enumerate(((q, qw), (k, kw))):
        want_x, want_w = L.norm_rope_backward64(t.grad.cpu(), xs[n], None if w is None else w.detach().cpu(), cos.cpu(), sin.cpu(), at, 1e-6, interleaved)
        L.check_close(gs[n], want_x, f"projection {n}")
        if w is not None:
            assert w.grad.dtype == w.dtype
            ref, bound = want_w
            L.check_close(w.grad, (ref, bound + (L.H * ref.abs() if dtype == torch.bfloat16 else 0)), f"weight {n}")
    assert torch.equal(gs[2], v.grad)


def test_separate_projections_and_strided_gradients():
    B, S, Hq, Hkv = 2, 33, 4, 2
    q, k, v = leaf(L.rand(11, B, S, Hq, 128)), leaf(L.rand(12, B, S, Hkv, 128)), leaf(L.rand(13, B, S, Hkv, 128))
    cos, sin = (t.cuda() for t in L.table(S, 128))
    dq, dk, dv = L.rand(14, B, Hq, S, 128).cuda(), L.rand(15, B, S, Hkv, 128).cuda(), L.rand(16, B, S, Hkv, 128).cuda()
    out = AG.qk_norm_rope(q, k, None, None, cos, sin, v=v)
    got = torch.autograd.grad(out, (q, k, v), (dq.transpose(1, 2), dk, dv))         # heads before tokens
    want = A.qk_norm_rope_backward(dq.transpose(1, 2).contiguous(), dk, q.detach(), k.detach(), None, None, cos, sin)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], dv)
    odd = torch.zeros(B * S * Hq * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(B, S, Hq, 128).copy_(dq.transpose(1, 2))       # 8 bytes off
    q2, k2 = AG.qk_norm_rope(q, k, None, None, cos, sin)
    again = torch.autograd.grad(q2, (q, k), odd)
    assert torch.equal(again[0], want[0]) and (again[1] == 0).all()
    one = torch.autograd.grad(AG.qk_norm_rope(q, k, None, None, cos, sin)[0].sum(), q)[0]       # an expanded gradient
    assert torch.equal(one, A.qk_norm_rope_backward(torch.ones_like(q), dk, q.detach(), k.detach(), None, None, cos, sin)[0])
    none = AG.qk_norm_rope(q, k, None, None, cos, sin, v=v)[2].sum()
    assert torch.equal(torch.autograd.grad(none, v)[0], torch.ones_like(v))


def test_gradients_off_a_16_byte_boundary():
    B, S, H = 1, 20, 2
    q, k, v = (leaf(L.rand(17 + n, B, S, H, 128)) for n in range(3))
    cos, sin = (t.cuda() for t in L.table(S, 128))
    odd = lambda seed: torch.cat([torch.zeros(1, dtype=torch.bfloat16), L.rand(seed, B * S * H * 128)]).cuda()[1:].view(B, S, H, 128)
    do, dk = odd(20), odd(21)
    assert do.is_contiguous() and do.data_ptr() % 16
    for f in (lambda: AG.attention(q, k, v, True)[:1], lambda: AG.qk_norm_rope(q, k, None, None, cos, sin)):
        out = f()
        got = torch.autograd.grad(out, (q, k), (do, dk)[:len(out)])
        out = f()
        want = torch.autograd.grad(out, (q, k), (do.clone(), dk.clone())[:len(out)])
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_attention_gradients_of_one_result_only():
    q, k, v = leaf(L.rand(21, 1, 50, 4, 128)), leaf(L.rand(22, 1, 60, 2, 128)), leaf(L.rand(23, 1, 60, 2, 128))
    o, lse = A.attention(q.detach(), k.detach(), v.detach(), causal=True)
    got = torch.autograd.grad(AG.attention(q, k, v, True)[1].sum(), (q, k, v))
    want = A.attention_backward(torch.zeros_like(o), q.detach(), k.detach(), v.detach(), o, lse, True, dlse=torch.ones_like(lse))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (got[2] == 0).all()
    got = torch.autograd.grad(AG.attention(q, k, v, True)[0].float().sum(), (q, k, v))      # an expanded gradient
    want = A.attention_backward(torch.ones_like(o), q.detach(), k.detach(), v.detach(), o, lse, True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x = AG.attention(q, k, v, True)[0].float().sum()
    dq, = torch.autograd.grad(x, q, create_graph=True)
    with pytest.raises(RuntimeError):           # once differentiable
        dq.float().sum().backward()
    with torch.no_grad():
        assert not AG.attention(q, k, v, True)[0].requires_grad


def test_step_in_a_graph():
    """Forward and backward of a layer captured together, replayed with other inputs, each time against the same step outside."""
    B, S, Hq, Hkv = 1, 96, 8, 2
    cos, sin = (t.cuda() for t in L.table(S, 128))
    qkv0 = L.rand(31, B, S, Hq + 2 * Hkv, 128).cuda()
    w0 = torch.ones(128, device="cuda")
    do = L.rand(32, B, S, Hq, 128).cuda()

    def step():
        qkv, qw, kw = (t.detach().requires_grad_() for t in (qkv0, w0, w0))
        o, _ = AG.attention(*AG.qkv_norm_rope(qkv, Hq, Hkv, qw, kw, cos, sin), True)
        return torch.autograd.grad(o, (qkv, qw, kw), do)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for n in range(4):
        qkv0.copy_(L.rand(40 + n, *qkv0.shape))
        do.copy_(L.rand(50 + n, *do.shape))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step())), n


def test_one_token_then_the_next():
    """Serving: a prompt into a cache, then token by token, each with its own place: the same as all tokens at once."""
    S, Hq, Hkv = 21, 4, 2
    cos, sin = (t.cuda() for t in L.table(64, 128))
    w = (1 + 0.2 * torch.randn(128, generator=torch.Generator().manual_seed(5))).cuda()
    qkv = L.rand(61, 1, S, Hq + 2 * Hkv, 128).cuda()
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=2)
    whole = A.qk_norm_rope(q, k, w, w, cos, sin, v=v)
    want, _ = A.attention(*whole, causal=True)
    cache = [torch.zeros(1, 64, Hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n = 17
    for a, b in [(0, n)] + [(i, i + 1) for i in range(n, S)]:
        at = torch.arange(a, b, device="cuda")[None]
        rows = torch.empty(1, b - a, Hq, 128, dtype=torch.bfloat16, device="cuda")
        A.qk_norm_rope(q[:, a:b], k[:, a:b], w, w, cos, sin, at, v=v[:, a:b], out=(rows, cache[0][:, a:b], cache[1][:, a:b]))
        o, _ = A.attention(rows, cache[0][:, :b].contiguous(), cache[1][:, :b].contiguous(), causal=True)
        assert torch.equal(rows, whole[0][:, a:b])
        # (other kernels of the forward pass for other numbers of rows: two roundings of probabilities and one of O, each way)
        assert (o.float() - want[:, a:b].float()).abs().max() <= 2.0 ** -6 * want.abs().max()
    assert torch.equal(cache[0][:, :S], whole[1]) and torch.equal(cache[1][:, :S], whole[2]) and (cache[0][:, S:] == 0).all()


def test_refuses():
    x = L.rand(71, 1, 8, 8, 128).cuda()
    cos, sin = (t.cuda() for t in L.table(8, 128))
    with pytest.raises(ValueError):
        AG.qkv_norm_rope(x, 4, 3, None, None, cos, sin)
    with pytest.raises(ValueError):
        AG.qkv_norm_rope(x[0], 4, 2, None, None, cos, sin)
    with pytest.raises(ValueError):
        AG.attention(x, x.float(), x)
    with pytest.raises(ValueError):
        AG.qk_norm_rope(x.cpu(), x, None, None, cos, sin)
