"""64-bit references of the operators around the attention forward, written from their formulas, and how far the kernels may be off.

H = 2^-8 is half a step of a BF16 value, relative to it.  attention_backward rounds P and dS to BF16 before they multiply and each result
once, everything else is FP32; so an element of dV = sum_i P_i dO_i is off by at most H * sum |P_i dO_i| + H * |dV|, one of dQ and dK
likewise with dS.  FP32 adds to each pair's P and dS at most F times its magnitude before cancellation (128 products of a score and their
sum, an exponent's argument of up to 2^7: 2^-24 * 2^7 each, with room for both: 2^-16).  Roundings of different pairs are independent with
a root mean square of at most H / sqrt(3) of each term, so over a whole result the 2-norm of the error stays below 0.75 H times that of
its terms and itself."""
import math

import numpy as np
import torch

H = 2.0 ** -8
F = 2.0 ** -16


def valid_pairs(Sq, Skv, causal):
    i, j = torch.arange(Sq)[:, None], torch.arange(Skv)[None]
    return j <= i + (Skv - Sq) if causal else torch.ones(Sq, Skv, dtype=torch.bool)


def forward64(q, k, v, causal, scale):
    """O (BF16) and LSE (FP32) from 64-bit arithmetic, CPU tensors."""
    B, Sq, Hq, D = q.shape
    _, Skv, Hkv, _ = k.shape
    o, lse = torch.zeros(q.shape, dtype=torch.float64), torch.empty(B, Hq, Sq, dtype=torch.float64)
    ok = valid_pairs(Sq, Skv, causal)
    for b in range(B):
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = (q[b, :, h].double() @ k[b, :, g].double().T * scale).masked_fill(~ok, -math.inf)
            l = torch.logsumexp(s, -1)
            lse[b, h] = l
            p = torch.where(ok & torch.isfinite(l)[:, None], torch.exp(s - l[:, None]), 0.0)
            o[b, :, h] = p @ v[b, :, g].double()
    return o.to(torch.bfloat16), lse.float()


def backward64(do, q, k, v, o, lse, causal, scale, dlse=None):
    """(reference, bound of each element, root of the sum of squares of its terms) for dq, dk, dv; CPU tensors."""
    B, Sq, Hq, D = q.shape
    _, Skv, Hkv, _ = k.shape
    f64 = torch.float64
    shapes = (q.shape, k.shape, v.shape)
    ref, bound, square = ([torch.zeros(s, dtype=f64) for s in shapes] for _ in range(3))
    ok = valid_pairs(Sq, Skv, causal)
    for b in range(B):
        for h in range(Hq):
            g = h // (Hq // Hkv)
            qh, kh, vh, gh, oh = (x.double() for x in (q[b, :, h], k[b, :, g], v[b, :, g], do[b, :, h], o[b, :, h]))
            l = lse[b, h].double()[:, None]
            p = torch.where(ok & torch.isfinite(l), torch.exp(qh @ kh.T * scale - l), 0.0)
            delta = (gh * oh).sum(-1, keepdim=True)
            size = (gh * oh).abs().sum(-1, keepdim=True)
            if dlse is not None:
                delta = delta - dlse[b, h].double()[:, None]
                size = size + dlse[b, h].double().abs()[:, None]
            ds = p * (gh @ vh.T - delta)
            # what FP32 may do to a pair, before cancellation
            fp = F * p
            fds = F * p * (gh.abs() @ vh.abs().T + size)
            for n, at, left, err, right in ((0, (b, slice(None), h), ds * scale, fds * abs(scale), kh),
                                            (1, (b, slice(None), g), ds.T * scale, fds.T * abs(scale), qh),
                                            (2, (b, slice(None), g), p.T, fp.T, gh)):
                ref[n][at] += left @ right
                bound[n][at] += (H * left.abs() + err) @ right.abs()
                square[n][at] += left ** 2 @ right ** 2
    for n in range(3):
        bound[n] += H * ref[n].abs() + 1e-30
    return ref, bound, [s.sqrt() for s in square]


def check_backward(got, want, what=""):
    ref, bound, terms = want
    for name, x, r, b, t in zip(("dq", "dk", "dv"), got, ref, bound, terms):
        err = (x.cpu().double() - r).abs()
        assert not torch.isnan(err).any(), f"{what} {name}: NaN"
        worst = (err / b).max().item()
        assert worst <= 1.0, f"{what} {name}: {worst:.2f} times the bound"
        # (2-norms; + 1e-3 of the bound for the FP32 parts, which are not independent)
        norm = 0.75 * H * math.sqrt(t.square().sum().item() + r.square().sum().item()) + 1e-3 * b.norm().item()
        assert err.norm().item() <= norm + 1e-30, f"{what} {name}: {err.norm().item() / norm:.2f} times the 2-norm's bound"


def rand(seed, *shape, mul=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * mul).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------- norm and rotation
def table(places, rotated, base=10000.0):
    rate = base ** (-torch.arange(0, rotated, 2, dtype=torch.float64) / rotated)
    angle = torch.arange(places, dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def _members(rotated, interleaved):
    i = np.arange(rotated // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotated // 2)


def _turn(x, cos, sin, positions, interleaved, back=False):
    a, b = _members(2 * cos.shape[1], interleaved)
    c, s = (t.double()[positions][:, :, None] for t in (cos, sin))
    s = -s if back else s
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size = x.abs()
    size[..., a] = (x[..., a] * c).abs() + (x[..., b] * s).abs()
    size[..., b] = (x[..., b] * c).abs() + (x[..., a] * s).abs()
    return y, size


def norm_rope64(x, w, cos, sin, positions, eps, interleaved):
    """(reference, bound): one rounding, and FP32 relative to the terms of the rotation."""
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    y, size = _turn(y, cos, sin, positions, interleaved)
    return y, H * y.abs() + F * size + 1e-30


def norm_rope_backward64(dz, x, w, cos, sin, positions, eps, interleaved):
    """((dx, bound), (dweight, bound)).  A weight's gradient is a sum in FP32 of up to a few hundred terms in line per lane, then of 32 lanes,
    then of 1024 workgroups in 64 runs: 2^-24 * 2^9 of the sum of magnitudes."""
    x = x.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xhat = x * r
    dy, size = _turn(dz.double(), cos, sin, positions, interleaved, back=True)
    dw, dw_size = (dy * xhat).sum((0, 1, 2)), (size * xhat.abs()).sum((0, 1, 2))
    g, g_size = (dy, size) if w is None else (dy * w.double(), size * w.double().abs())
    dx = r * (g - xhat * (g * xhat).mean(-1, keepdim=True))
    dx_size = r * (g_size + xhat.abs() * (g_size * xhat.abs()).mean(-1, keepdim=True))
    return (dx, H * dx.abs() + F * dx_size + 1e-30), (dw, 2.0 ** -15 * dw_size + 1e-30)


def check_close(got, want, what=""):
    ref, bound = want
    err = (got.cpu().double() - ref).abs()
    assert not torch.isnan(err).any(), f"{what}: NaN"
    assert (err <= bound).all(), f"{what}: {(err / bound).max().item():.2f} times the bound"


# ------------------------------------------------------------------------------------------------- against differences of the forward
def forward_exact(q, k, v, causal, scale):
    """(O, LSE, P) in 64 bits, nothing rounded; CPU tensors, O [B, S, H, D], P [B, H, Sq, Skv]."""
    G = q.shape[2] // k.shape[2]
    q, k, v = (t.double().transpose(1, 2) for t in (q, k.repeat_interleave(G, 2), v.repeat_interleave(G, 2)))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    s = s.masked_fill(~valid_pairs(q.shape[2], k.shape[2], causal), -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(torch.isneginf(lse), 0.0, lse)[..., None])
    return torch.matmul(p, v).transpose(1, 2), lse, p


def check_slopes(grads, do, dlse, q, k, v, causal, scale):
    """Gradients of sum(do O) + sum(dlse LSE), from the forward kernel's O and LSE, against differences of that number in 64 bits: along the signs of
    the gradient itself, and of the shares in it that come through O and through LSE, so that all elements of one add up and a factor, a sign or a
    lost term cannot hide.  The tolerance comes from the 64-bit gradient alone: `bound` of backward64 for each element; and delta's share of the
    forward kernel's roundings, of its probabilities and of O, each at most H, which reaches all pairs of a row.  (Differences of steps h of a smooth
    function are off by h^2: 1e-6 of the slope has room for it.)"""
    o, lse, p = forward_exact(q, k, v, causal, scale)
    ref, bound, _ = backward64(do, q, k, v, o, lse, causal, scale, dlse)
    without_o, without_lse = (backward64(do, q, k, v, x, lse, causal, scale, y)[0] for x, y in ((torch.zeros_like(o), dlse), (o, None)))
    G = q.shape[2] // k.shape[2]
    kk, vv = k.double().repeat_interleave(G, 2), v.double().repeat_interleave(G, 2)
    size = torch.matmul(p, vv.abs().transpose(1, 2)).transpose(1, 2) + o.abs()
    delta = H * (do.double().abs() * size).sum(-1).transpose(1, 2)         # [B, H, Sq]

    def value(q, k, v):
        o, l, _ = forward_exact(q, k, v, causal, scale)
        return (do.double() * o).sum().item() + (dlse.double() * l)[torch.isfinite(l)].sum().item()

    for n, name in enumerate(("dq", "dk", "dv")):
        shares = {"": ref[n]} if n == 2 else {"": ref[n], " through O": ref[n] - without_o[n], " through LSE": ref[n] - without_lse[n]}
        for share, part in shares.items():
            way = torch.sign(part)
            at, h = [q.double(), k.double(), v.double()], 1e-5
            up, down = (at[:n] + [at[n] + s * h * way] + at[n + 1:] for s in (1, -1))
            slope = (value(*up) - value(*down)) / (2 * h)
            # what an error of delta does along `way`
            s = torch.zeros_like(p)
            if n == 0:
                s = torch.matmul(way.transpose(1, 2), kk.transpose(1, 2).transpose(2, 3).contiguous())
            elif n == 1:
                s = torch.matmul(q.double().transpose(1, 2), way.repeat_interleave(G, 2).transpose(1, 2).transpose(2, 3).contiguous())
            tolerance = bound[n].sum().item() + (delta * (abs(scale) * p * s).sum(-1).abs()).sum().item() + 1e-6 * ref[n].abs().sum().item()
            got = (grads[n].cpu().double() * way).sum().item()
            assert tolerance <= 0.6 * part.abs().sum().item(), f"{name}{share}: too much room, {tolerance} of {part.abs().sum().item()}"
            assert abs(got - slope) <= tolerance, f"{name}{share}: {got} along its signs, differences {slope}, tolerance {tolerance}"
