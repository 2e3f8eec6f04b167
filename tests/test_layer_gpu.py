"""attention_backward, qk_norm_rope and qk_norm_rope_backward against 64-bit arithmetic (layer_util says how far they may be off)."""
import math

import pytest
import torch

import layer_util as L
import paper_2603_24517_amd as A

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


def cuda(*tensors):
    return [None if t is None else t.cuda() for t in tensors]


def inputs(B, Hq, Hkv, Sq, Skv, causal, seed, scale=SCALE, q_mul=1.0, do_mul=1.0, dlse=False):
    q = L.rand(seed, B, Sq, Hq, 128, mul=q_mul)
    k, v = L.rand(seed + 1, B, Skv, Hkv, 128), L.rand(seed + 2, B, Skv, Hkv, 128)
    do = L.rand(seed + 3, B, Sq, Hq, 128, mul=do_mul)
    o, lse = L.forward64(q, k, v, causal, scale)
    dl = L.rand(seed + 4, B, Hq, Sq, mul=do_mul).float() if dlse else None
    return do, q, k, v, o, lse, dl


# B, Hq, Hkv, Sq, Skv, causal: one token; tile borders of 32, 64, 128, 256 rows; more queries than keys (rows without a key under the mask); fewer;
# head groups of 1, 2, 3, 4, 6, 8
SHAPES = [
    (1, 1, 1, 1, 1, True), (2, 2, 1, 1, 1, False), (1, 4, 2, 1, 77, True), (3, 2, 2, 1, 600, False),
    (1, 2, 2, 31, 31, True), (1, 2, 1, 32, 32, True), (2, 2, 2, 33, 33, True), (1, 2, 2, 33, 65, False),
    (1, 4, 1, 64, 64, True), (1, 3, 1, 65, 63, False), (1, 6, 2, 100, 100, True), (2, 4, 4, 127, 129, True),
    (1, 8, 1, 130, 130, True), (1, 2, 2, 255, 257, False), (1, 1, 1, 256, 256, True), (1, 1, 1, 257, 257, True),
    (1, 2, 1, 300, 40, True), (1, 2, 2, 300, 1, True), (2, 2, 1, 70, 33, True), (1, 4, 4, 520, 520, True),
    (1, 2, 1, 40, 700, True), (1, 8, 2, 17, 1030, True), (1, 2, 2, 600, 90, False), (1, 12, 2, 50, 200, True),
    (5, 4, 2, 200, 200, True), (1, 32, 8, 96, 160, True), (1, 1, 1, 1500, 900, True), (1, 1, 1, 900, 1500, False),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape):
    n = SHAPES.index(shape)
    causal = shape[5]
    do, q, k, v, o, lse, dl = inputs(*shape, seed=100 + 10 * n, dlse=n % 3 == 0, q_mul=2.0 if n % 4 == 1 else 1.0,
                                     do_mul=2.0 ** -10 if n % 5 == 2 else 1.0)
    d = cuda(do, q, k, v, o, lse, dl)
    got = A.attention_backward(*d[:6], causal=causal, dlse=d[6])
    assert [x.dtype for x in got] == [torch.bfloat16] * 3 and [x.shape for x in got] == [q.shape, k.shape, v.shape]
    L.check_backward(got, L.backward64(do, q, k, v, o, lse, causal, SCALE, dl), str(shape))


@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.02, 0.5])
@pytest.mark.parametrize("causal", [False, True])
def test_backward_scales(scale, causal):
    do, q, k, v, o, lse, _ = inputs(1, 4, 2, 90, 110, causal, seed=2000, scale=scale)
    got = A.attention_backward(*cuda(do, q, k, v, o, lse), causal=causal, scale=scale)
    L.check_backward(got, L.backward64(do, q, k, v, o, lse, causal, scale), f"scale {scale}")


@pytest.mark.parametrize("scale", [1.2e-38, 1e-40, -1e-44, 1e-46])
def test_backward_of_scales_below_the_normal_range(scale):
    """Scores of no size beside a mask of infinity: all keys that a row sees have the same probability.  (In FP32 the last of them is 0.)"""
    do, q, k, v, o, lse, dl = inputs(1, 4, 2, 70, 90, True, seed=2050, scale=scale, dlse=True)
    got = A.attention_backward(*cuda(do, q, k, v, o, lse), causal=True, scale=scale, dlse=dl.cuda())
    L.check_backward(got, L.backward64(do, q, k, v, o, lse, True, scale, dl), f"scale {scale}")


def test_backward_of_rows_without_a_key():
    """Under the mask, with more queries than keys, the first rows see nothing: no gradient of theirs, whatever arrives."""
    do, q, k, v, o, lse, dl = inputs(1, 2, 1, 170, 100, True, seed=2100, dlse=True)
    assert torch.isneginf(lse[:, :, :70]).all()
    got = A.attention_backward(*cuda(do, q, k, v, o, lse), causal=True, dlse=dl.cuda())
    assert (got[0][:, :70] == 0).all()
    L.check_backward(got, L.backward64(do, q, k, v, o, lse, True, SCALE, dl))
    q2, do2 = q.clone(), do.clone()
    q2[:, :40], do2[:, :40] = 7.0, -3.0         # rows that nothing sees
    again = A.attention_backward(*cuda(do2, q2, k, v, o, lse), causal=True, dlse=dl.cuda())
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_backward_of_large_and_small_scores():
    """One dominant key per row, and rows whose probabilities all underflow but one."""
    do, q, k, v, _, _, _ = inputs(1, 2, 2, 80, 80, True, seed=2200)
    q = q * 16
    k[:, ::7] *= 8
    o, lse = L.forward64(q, k, v, True, SCALE)
    got = A.attention_backward(*cuda(do, q, k, v, o, lse), causal=True)
    # (arguments of the exponent reach 2^12 here, so FP32 leaves P 2^-24 * 2^12 relative: 2^4 times what the bound assumes.  Errors of that
    # kind may all point one way: over at most 80 terms, 2^-12 * sqrt(80) = 0.56 H of their 2-norm, within as much again as the 0.75 H)
    ref, bound, terms = L.backward64(do, q, k, v, o, lse, True, SCALE)
    L.check_backward(got, (ref, [b * (1 + 2.0 ** 4 * L.F / L.H) + 2.0 ** 4 * L.F * b / L.H for b in bound], [t * 2 for t in terms]))


@pytest.mark.parametrize("shape", [(1, 8, 2, 1500, 1500, True), (2, 2, 2, 700, 1300, False), (1, 4, 1, 60, 9000, True), (1, 4, 4, 512, 512, False)],
                         ids=str)
def test_backward_same_bits_always(shape):
    """Repeated, on another stream, and beside other launches; results of a call do not depend on what its memory held."""
    do, q, k, v, o, lse, _ = cuda(*inputs(*shape, seed=2300))
    first = A.attention_backward(do, q, k, v, o, lse, causal=shape[5])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(3):
        junk = torch.full((8 << 20,), float("nan"), device="cuda")
        del junk
        outs.append(A.attention_backward(do, q, k, v, o, lse, causal=shape[5]))
        with torch.cuda.stream(side):
            outs.append(A.attention_backward(do, q, k, v, o, lse, causal=shape[5]))
    torch.cuda.synchronize()
    for got in outs:
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_backward_against_differences():
    """The gradient of a number made of O and LSE against differences of the forward pass itself, along random directions."""
    B, Hq, Hkv, S, causal = 1, 4, 2, 150, True
    do, q, k, v, _, _, dl = inputs(B, Hq, Hkv, S, S, causal, seed=2400, dlse=True)
    do, q, k, v, dl = cuda(do, q, k, v, dl)
    o, lse = A.attention(q, k, v, causal=causal)
    grads = A.attention_backward(do, q, k, v, o, lse, causal=causal, dlse=dl)

    def value(q, k, v):
        o, lse = L.forward64(q.cpu(), k.cpu(), v.cpu(), causal, SCALE)      # (O rounded: its error, H |O| per element, enters the tolerance)
        return (do.cpu().double() * o.double()).sum().item() + (dl.cpu().double() * lse.double()).sum().item()

    o_round = L.H * (do.double().square() * o.double().square()).sum().sqrt().item()
    for n, x in enumerate((q, k, v)):
        step = torch.where(torch.rand(x.shape, generator=torch.Generator().manual_seed(n)) < 0.5, -1, 1).cuda()
        # one bit pattern up or down for every element: steps of half a unit in the last place, exactly representable on both sides
        up, down = ((x.view(torch.int16) + s * step.to(torch.int16) * 4).view(torch.bfloat16) for s in (1, -1))
        args = [q, k, v]
        args[n] = up
        hi = value(*args)
        args[n] = down
        lo = value(*args)
        want = (grads[n].double() * (up.double() - down.double())).sum().item()
        size = (grads[n].double() * (up.double() - down.double())).square().sum().sqrt().item()
        # two rounded O's, 4-sigma; BF16 gradients, 4-sigma; second order: steps are 2^-5 relative, so a few per cent of the size
        assert abs((hi - lo) - want) <= 4 * math.sqrt(2) * o_round + 4 * L.H * size + 0.1 * size * math.sqrt(8), (n, hi - lo, want)


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv,causal", [(1, 4, 2, 150, 150, True), (2, 2, 2, 70, 40, True), (1, 3, 1, 33, 200, False)])
def test_backward_against_differences_along_its_signs(B, Hq, Hkv, Sq, Skv, causal):
    """The gradient from the forward pass's own O and LSE; a factor or a lost term does not pass (layer_util.check_slopes)."""
    do, q, k, v, _, lse, dl = inputs(B, Hq, Hkv, Sq, Skv, causal, seed=2450, dlse=True)
    dl = 4 * dl.masked_fill(torch.isneginf(lse), 0.0)       # (rows without a key: LSE is -inf, and no slope of it)
    d = cuda(do, q, k, v, dl)
    o, lse = A.attention(*d[1:4], causal=causal)
    grads = A.attention_backward(*d[:4], o, lse, causal=causal, dlse=d[4])
    L.check_slopes(grads, do, dl, q, k, v, causal, SCALE)


NOT_FINITE = [(1, 4, 2, 500, 500), (2, 2, 1, 200, 450), (1, 2, 2, 450, 200), (24, 8, 8, 200, 200)]


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("shape", NOT_FINITE, ids=str)
def test_backward_of_values_that_are_not_finite(shape, value):
    """Under the mask: NaN where the formulas have it, the same bits in what such a value is masked for, from 160 positions on (a value of v, o or of
    LSE's gradient: from the first position on) and in other heads and batch entries.  (An infinity leaves infinities as well: P > 0 times one is one.)"""
    B, Hq, Hkv, Sq, Skv = shape
    G, off, nan = Hq // Hkv, Skv - Sq, math.isnan(value)
    clean = inputs(*shape, True, seed=2800, dlse=True)
    want = A.attention_backward(*cuda(*clean[:6]), causal=True, dlse=clean[6].cuda())
    names = ("do", "q", "k", "v", "o", "lse", "dlse")
    b, h = B - 1, G - 1             # the head of a group's queries, the first of the keys

    def run(**changed):
        t = {**dict(zip(names, clean)), **changed}
        got = A.attention_backward(*cuda(*(t[n] for n in names[:6])), causal=True, dlse=t["dlse"].cuda())
        return [x.cpu() for x in got]

    def same(got, ref, but=slice(None), heads=slice(0, 0)):
        """Everything the same but positions `but` of heads `heads` of batch entry b, which are returned."""
        ref, x = ref.cpu(), got.clone()
        part = got[b, but, heads].float()
        x[b, but, heads] = ref[b, but, heads]
        assert torch.equal(x, ref)
        return part

    bad = lambda name, *at: (lambda t: (t.__setitem__(at, value), t)[1])(clean[names.index(name)].clone())
    spoilt = lambda x: torch.isnan(x).all() if nan else not torch.isfinite(x).any()
    group = slice(0, 1)
    for i in sorted({0, max(0, -off - 1), max(0, -off), 37, Sq // 2, Sq - 1}):
        seen = max(0, i + off + 1)          # keys that row i sees
        reach = min(Skv, max(0, i + off + 160))
        row = (slice(i, i + 1), slice(h, h + 1))
        for name, column in (("q", 5), ("do", 77)):
            x = bad(name, b, i, h, column)
            changed = {name: x}
            if name == "q":
                changed["lse"] = clean[5].clone()
                if seen:
                    changed["lse"][b, h, i] = math.nan
            dq, dk, dv = run(**changed)
            part = same(dq, want[0], *row)
            assert spoilt(part) if seen else (part == 0).all()
            part = same(dk, want[1], slice(0, reach), group)
            assert spoilt(part[:seen])
            part = same(dv, want[2], slice(0, reach), group)
            assert spoilt(part[:seen, :, 77]) and (name == "q" or torch.equal(dv[..., :77], want[2].cpu()[..., :77]))
        for name, at in (("o", (b, i, h, 3)), ("dlse", (b, h, i))):
            dq, dk, dv = run(**{name: bad(name, *at)})
            part = same(dq, want[0], *row)
            assert not torch.isfinite(part).any() if seen else (part == 0).all()
            part = same(dk, want[1], slice(0, seen), group)
            assert not torch.isfinite(part).any()
            same(dv, want[2])
    for j in sorted({0, 100, Skv // 2, Skv - 33, Skv - 1}):
        sees = max(0, j - off)              # the first row that sees key j
        for name in ("k", "v"):
            changed = {name: bad(name, b, j, 0, 9)}
            if name == "k":
                changed["lse"] = clean[5].clone()
                changed["lse"][b, :G, sees:] = math.nan
            else:
                changed["o"] = clean[4].clone()
                changed["o"][b, sees:, :G, 9] = value
            dq, dk, dv = run(**changed)
            part = same(dq, want[0], slice(max(0, sees - 159) if name == "k" else sees, Sq), slice(0, G))
            assert spoilt(part[-(Sq - sees):])
            same(dk, want[1], slice(0, Skv), group)
            if name == "k":
                same(dv, want[2], slice(0, Skv), group)
            else:
                same(dv, want[2])


def test_backward_refuses():
    do, q, k, v, o, lse, dl = cuda(*inputs(2, 4, 2, 20, 30, True, seed=2500, dlse=True))
    good = dict(do=do, q=q, k=k, v=v, o=o, lse=lse, dlse=dl)
    for name, bad in (("do", do.float()), ("do", do[:, :19]), ("do", do.transpose(1, 2)), ("do", do.cpu()), ("q", q.float()), ("q", q[0]),
                      ("k", k[:, ::2]), ("k", k[:1]), ("v", v[:, 1:].contiguous()), ("o", o.transpose(1, 2).contiguous()), ("o", o.cpu()),
                      ("lse", lse.double()), ("lse", lse[:, :2]), ("lse", lse.cpu()), ("dlse", dl.bfloat16()), ("dlse", dl.transpose(1, 2)),
                      ("dlse", dl.cpu())):
        with pytest.raises(ValueError):
            A.attention_backward(**{**good, name: bad}, causal=True)
    with pytest.raises(A.AttnError) as e:
        A.attention_backward(**good, scale=math.inf)
    assert e.value.code == A.ATTN_E_SCALE and "attn_bwd" in str(e.value)
    with pytest.raises(A.AttnError) as e:
        A.attention_backward(do, q, k[:, :, :1].expand(2, 30, 3, 128).contiguous(), v[:, :, :1].expand(2, 30, 3, 128).contiguous(), o, lse)
    assert e.value.code == A.ATTN_E_SHAPE


def _graph(call):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    return g, out


@pytest.mark.parametrize("shape", [(1, 4, 2, 300, 300, True), (1, 2, 2, 64, 3000, True)], ids=str)
def test_backward_in_a_graph(shape):
    """Captured, replayed with other inputs in place, each replay against the call itself, with other work between."""
    do, q, k, v, o, lse, _ = cuda(*inputs(*shape, seed=2600))
    g, out = _graph(lambda: A.attention_backward(do, q, k, v, o, lse, causal=shape[5]))
    for n in range(4):
        do.copy_(L.rand(2700 + n, *do.shape))
        g.replay()
        torch.cuda.synchronize()
        want = A.attention_backward(do, q, k, v, o, lse, causal=shape[5])
        assert all(torch.equal(a, b) for a, b in zip(out, want)), n


# ------------------------------------------------------------------------------------------------- norm and rotation
# B, S, Hq, Hkv, rotated, weight type, positions, interleaved, fused, with v
ROPES = [
    (1, 1, 1, 1, 128, torch.float32, None, False, False, False), (64, 1, 32, 8, 128, torch.bfloat16, torch.int64, False, True, True),
    (3, 37, 4, 2, 64, torch.float32, torch.int32, False, True, True), (2, 5, 3, 3, 16, torch.bfloat16, None, True, False, True),
    (1, 200, 5, 1, 96, None, torch.int64, True, True, True), (2, 33, 16, 16, 128, torch.float32, None, True, True, False),
    (1, 7, 2, 5, 112, None, torch.int32, False, False, False), (5, 129, 8, 4, 32, torch.bfloat16, torch.int64, False, True, True),
]


def rope_inputs(B, S, Hq, Hkv, rotated, weight, positions, interleaved, fused, with_v, seed):
    if fused:
        q, k, v = L.rand(seed, B, S, Hq + 2 * Hkv, 128).split([Hq, Hkv, Hkv], dim=2)
    else:
        q, k, v = L.rand(seed, B, S, Hq, 128), L.rand(seed + 1, B, S, Hkv, 128), L.rand(seed + 2, B, S, Hkv, 128)
    g = torch.Generator().manual_seed(seed + 3)
    qw = kw = None
    if weight is not None:
        qw, kw = ((1 + 0.3 * torch.randn(128, generator=g)).to(weight) for _ in range(2))
    cos, sin = L.table(300, rotated)
    pos = None if positions is None else torch.randint(0, 300, (B, S), generator=g).to(positions)
    return q, k, v if with_v else None, qw, kw, cos, sin, pos


def on_device(t):
    """The same strides on the device (slices of one projection stay that)."""
    base = t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,), 0).cuda()
    return base.as_strided(t.shape, t.stride(), t.storage_offset())


@pytest.mark.parametrize("case", ROPES, ids=str)
def test_norm_rope(case):
    B, S = case[:2]
    q, k, v, qw, kw, cos, sin, pos = rope_inputs(*case, seed=3000 + 10 * ROPES.index(case))
    inter = case[7]
    dev = [on_device(q), on_device(k), *cuda(qw, kw, cos, sin, pos)]
    got = A.qk_norm_rope(*dev, eps=1e-5, interleaved=inter, v=None if v is None else on_device(v))
    at = torch.arange(S).expand(B, S) if pos is None else pos.long()
    for x, t, w, name in ((got[0], q, qw, "q"), (got[1], k, kw, "k")):
        assert x.is_contiguous() and x.dtype == torch.bfloat16
        L.check_close(x, L.norm_rope64(t, w, cos, sin, at, 1e-5, inter), f"{case} {name}")
    assert len(got) == (2 if v is None else 3)
    if v is not None:
        assert got[2].is_contiguous() and torch.equal(got[2].cpu(), v.contiguous())


@pytest.mark.parametrize("case", ROPES, ids=str)
def test_norm_rope_backward(case):
    B, S, Hq, Hkv = case[:4]
    seed = 4000 + 10 * ROPES.index(case)
    q, k, v, qw, kw, cos, sin, pos = rope_inputs(*case, seed=seed)
    inter = case[7]
    dq, dk, dv = L.rand(seed + 5, B, S, Hq, 128), L.rand(seed + 6, B, S, Hkv, 128), L.rand(seed + 7, B, S, Hkv, 128)
    dev = [on_device(q), on_device(k), *cuda(qw, kw, cos, sin, pos)]
    out = None
    whole = torch.full((B, S, Hq + 2 * Hkv, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    if case[8]:
        out = whole.split([Hq, Hkv, Hkv], dim=2)[:2 if v is None else 3]
    got = A.qk_norm_rope_backward(dq.cuda(), dk.cuda(), *dev, eps=1e-5, interleaved=inter, dv=None if v is None else dv.cuda(), out=out)
    at = torch.arange(S).expand(B, S) if pos is None else pos.long()
    *dx, dqw, dkw = got
    if out is not None:
        assert all(a.data_ptr() == b.data_ptr() for a, b in zip(dx, out))
        if v is None:
            assert (whole[:, :, Hq + Hkv:] == 9.0).all()
    for x, dw, dz, t, w, name in ((dx[0], dqw, dq, q, qw, "q"), (dx[1], dkw, dk, k, kw, "k")):
        want_x, want_w = L.norm_rope_backward64(dz, t, w, cos, sin, at, 1e-5, inter)
        L.check_close(x, want_x, f"{case} d{name}")
        if w is None:
            assert dw is None
        else:
            assert dw.dtype == torch.float32
            L.check_close(dw, want_w, f"{case} d{name}_weight")
    if v is not None:
        assert torch.equal(dx[2].cpu(), dv)


@pytest.mark.parametrize("strides", ["transposed", "every other", "broadcast", "cache"])
def test_norm_rope_strides(strides):
    """Heads before tokens, every other head, one head for all, and results into a slice of a cache with the rest left as it was."""
    B, S, H = 2, 19, 4
    cos, sin = L.table(40, 128)
    out = cache = None
    if strides == "transposed":
        q = L.rand(1, B, H, S, 128).transpose(1, 2)
    elif strides == "every other":
        q = L.rand(2, B, S, 2 * H, 128)[:, :, ::2]
    elif strides == "broadcast":
        q = L.rand(3, B, S, 1, 128).expand(B, S, H, 128)
    else:
        q = L.rand(4, B, S, H, 128)
        cache = [torch.full((B, 60, H, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        out = [c[:, 20:20 + S] for c in cache]
    k, v = L.rand(5, B, S, H, 128), L.rand(6, B, S, H, 128)
    got = A.qk_norm_rope(on_device(q), k.cuda(), None, None, *cuda(cos, sin), v=v.cuda(), out=out)
    at = torch.arange(S).expand(B, S)
    L.check_close(got[0], L.norm_rope64(q, None, cos, sin, at, 1e-6, False), strides)
    L.check_close(got[1], L.norm_rope64(k, None, cos, sin, at, 1e-6, False), strides)
    assert torch.equal(got[2].cpu(), v)
    if cache:
        for c in cache:
            assert (c[:, :20] == 3.0).all() and (c[:, 20 + S:] == 3.0).all()


def test_norm_rope_places_outside_the_table():
    q, k = L.rand(1, 1, 4, 2, 128).cuda(), L.rand(2, 1, 4, 1, 128).cuda()
    cos, sin = cuda(*L.table(10, 128))
    for dtype in (torch.int32, torch.int64):
        pos = torch.tensor([[0, 10, -1, 9]], dtype=dtype, device="cuda")
        for x in A.qk_norm_rope(q, k, None, None, cos, sin, pos):
            assert torch.isnan(x[:, 1:3].float()).all() and not torch.isnan(x[:, ::3].float()).any()
    pos = torch.tensor([[0, 1 << 40, 3, -(1 << 40)]], device="cuda")
    x = A.qk_norm_rope(q, k, None, None, cos, sin, pos)[0]
    assert torch.isnan(x[:, 1::2].float()).all() and not torch.isnan(x[:, ::2].float()).any()


@pytest.mark.parametrize("S,dtype", [(4, torch.int32), (4, torch.int64), (700, torch.int64)])
def test_norm_rope_backward_of_places_outside_the_table(S, dtype):
    """NaN in these tokens' own gradients; the weights' gradients are those of the other tokens, whatever arrives for these."""
    q, k, dq, dk = (L.rand(30 + n, 2, S, h, 128) for n, h in enumerate((3, 1, 3, 1)))
    g = torch.Generator().manual_seed(34)
    qw, kw = ((1 + 0.3 * torch.randn(128, generator=g)) for _ in range(2))
    cos, sin = L.table(S, 64)
    pos = torch.arange(S).repeat(2, 1).to(dtype)
    pos[0, 1], pos[1, 2] = -1, S
    if dtype == torch.int64:
        pos[0, 3] = 1 << 40
    out = (pos < 0) | (pos >= S)
    dq[0, 1] = 0.0
    dk[1, 2] = math.nan
    got = A.qk_norm_rope_backward(*cuda(dq, dk, q, k, qw, kw, cos, sin, pos))
    at = torch.where(out, 0, pos).long()
    for x, dw, dz, t, w, name in ((got[0], got[2], dq, q, qw, "q"), (got[1], got[3], dk, k, kw, "k")):
        assert torch.isnan(x[out.cuda()].float()).all()
        (ref, bound), (ref_w, bound_w) = L.norm_rope_backward64(dz.masked_fill(out[:, :, None, None], 0.0), t, w, cos, sin, at, 1e-6, False)
        L.check_close(x[~out.cuda()], (ref[~out], bound[~out]), f"d{name}")
        L.check_close(dw, (ref_w, bound_w), f"d{name}_weight")


def test_norm_rope_beyond_the_squares_range():
    """Heads whose squares add up to more than FP32 holds come out as zeros, and so do their gradients; their neighbours do not notice."""
    q, dq = L.rand(50, 1, 6, 2, 128), L.rand(51, 1, 6, 2, 128)
    q[0, 2, 0, 7], q[0, 4, 1] = 1e20, 3e38
    cos, sin = L.table(6, 128)
    at, big = torch.arange(6)[None], torch.zeros(1, 6, 2, dtype=torch.bool)
    big[0, 2, 0] = big[0, 4, 1] = True
    w = torch.ones(128)
    got = A.qk_norm_rope(*cuda(q, q, w, w, cos, sin))[0].cpu()
    ref, bound = L.norm_rope64(q, w, cos, sin, at, 1e-6, False)
    assert not got[big].any()
    L.check_close(got[~big], (ref[~big], bound[~big]))
    dx, _, dw, _ = A.qk_norm_rope_backward(*cuda(dq, dq, q, q, w, w, cos, sin))
    (ref, bound), want_w = L.norm_rope_backward64(dq.masked_fill(big[..., None], 0.0), q, w, cos, sin, at, 1e-6, False)
    assert not dx.cpu()[big].any()
    L.check_close(dx.cpu()[~big], (ref[~big], bound[~big]))
    L.check_close(dw, want_w)


@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_norm_rope_of_values_that_are_not_finite(value):
    """They stay in their own head of their own token, but for the weights' gradients, which are sums over all."""
    q, k, dq, dk = (L.rand(40 + n, 2, 50, h, 128) for n, h in enumerate((4, 2, 4, 2)))
    w, cos, sin = torch.ones(128), *L.table(50, 128)
    forward = lambda q: A.qk_norm_rope(*cuda(q, k, w, w, cos, sin), v=k.cuda())
    backward = lambda dq, q: A.qk_norm_rope_backward(*cuda(dq, dk, q, k, w, w, cos, sin))
    bad = lambda t: t.index_put((torch.tensor(1), torch.tensor(17), torch.tensor(2), torch.tensor(60)), torch.tensor(value, dtype=t.dtype))
    for want, got in ((forward(q), forward(bad(q))), (backward(dq, q), backward(dq, bad(q))), (backward(dq, q), backward(bad(dq), q))):
        a, x = want[0], got[0].clone()
        assert not torch.isfinite(x[1, 17, 2]).all()
        x[1, 17, 2] = a[1, 17, 2]
        assert torch.equal(x, a) and torch.equal(got[1], want[1])
        if len(got) == 3:           # values
            assert torch.equal(got[2], want[2])
        else:
            assert not torch.isfinite(got[2]).all() and torch.equal(got[3], want[3])
    odd = torch.tensor([0x7fc1, 0xffff - 65536, 0x7f80, 0xff80 - 65536, 0x8000 - 65536, 1], dtype=torch.int16).view(torch.bfloat16)
    v = k.clone()
    v[1, 3, 1, :6] = odd
    assert torch.equal(A.qk_norm_rope(*cuda(q, k, w, w, cos, sin), v=v.cuda())[2].cpu().view(torch.int16), v.view(torch.int16))       # bit by bit


def test_norm_rope_zeros_and_extremes():
    """Rows of zeros (with eps; their gradient is that of x / sqrt(eps)), and rows whose squares leave BF16's but not FP32's precision."""
    q = torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16)
    q[:, 1] = 1e15
    q[:, 2] = L.rand(9, 2, 128) * 2.0 ** -30
    cos, sin = L.table(3, 128)
    at = torch.arange(3)[None]
    for eps in (1e-6, 1e-18):
        got, _ = A.qk_norm_rope(q.cuda(), q.cuda(), None, None, *cuda(cos, sin), eps=eps)
        L.check_close(got, L.norm_rope64(q, None, cos, sin, at, eps, False), f"eps {eps}")
        dz = L.rand(10, 1, 3, 2, 128)
        dx = A.qk_norm_rope_backward(dz.cuda(), dz.cuda(), q.cuda(), q.cuda(), None, None, *cuda(cos, sin), eps=eps)[0]
        L.check_close(dx, L.norm_rope_backward64(dz, q, None, cos, sin, at, eps, False)[0], f"eps {eps}")


def test_norm_rope_refuses():
    q, k = L.rand(1, 2, 6, 4, 128).cuda(), L.rand(2, 2, 6, 2, 128).cuda()
    cos, sin = cuda(*L.table(16, 64))
    w = torch.ones(128, device="cuda")
    pos = torch.zeros(2, 6, dtype=torch.int32, device="cuda")
    good = dict(q=q, k=k, q_weight=w, k_weight=w, cos=cos, sin=sin, positions=pos)
    bads = [("q", q.float()), ("q", q[0]), ("q", q.cpu()), ("k", k[:1]), ("k", k.cpu()), ("k", k.transpose(2, 3)), ("q_weight", None),
            ("q_weight", w.bfloat16()), ("k_weight", w[:64]), ("k_weight", w.cpu()), ("cos", cos.double()), ("cos", cos[:, :16]),
            ("sin", sin.t().contiguous().t()), ("sin", sin.cpu()), ("positions", pos.float()), ("positions", pos[:, :3]), ("positions", pos.cpu()),
            ("v", q), ("v", k.float()), ("out", (q,)), ("out", (q, q)), ("out", (torch.empty_like(q[:, :, :1]).expand_as(q), k))]
    for name, bad in bads:
        with pytest.raises(ValueError):
            A.qk_norm_rope(**{**good, name: bad})
        if name not in ("v", "out"):
            with pytest.raises(ValueError):
                A.qk_norm_rope_backward(q, k, **{**good, name: bad})
    for kw in (dict(dq=q.float()), dict(dk=q), dict(dv=q), dict(dv=k.cpu()), dict(out=(q,))):
        with pytest.raises(ValueError):
            A.qk_norm_rope_backward(**{**good, "dq": q, "dk": k, **kw})
    for change, code in ((dict(cos=cos[:, :20].contiguous(), sin=sin[:, :20].contiguous()), A.ATTN_E_UNSUPPORTED), (dict(eps=-1.0), A.ATTN_E_SCALE),
                         (dict(cos=cos[:3], sin=sin[:3], positions=None), A.ATTN_E_SHAPE),
                         (dict(q=torch.zeros(2 * 6 * 4 * 128 + 8, dtype=torch.bfloat16, device="cuda")[4:-4].view(2, 6, 4, 128)), A.ATTN_E_ALIGN)):
        with pytest.raises(A.AttnError) as e:
            A.qk_norm_rope(**{**good, **change})
        assert e.value.code == code


def test_norm_rope_in_a_graph_and_on_another_stream():
    case = (2, 50, 8, 2, 128, torch.float32, torch.int64, False, True, True)
    q, k, v, qw, kw, cos, sin, pos = rope_inputs(*case, seed=5000)
    q, k, v = on_device(q), on_device(k), on_device(v)
    qw, kw, cos, sin, pos = cuda(qw, kw, cos, sin, pos)
    dq, dk = L.rand(5001, *q.shape).cuda(), L.rand(5002, *k.shape).cuda()
    both = lambda: (*A.qk_norm_rope(q, k, qw, kw, cos, sin, pos, v=v), *A.qk_norm_rope_backward(dq, dk, q, k, qw, kw, cos, sin, pos))
    g, out = _graph(both)
    for n in range(4):
        dq.copy_(L.rand(5100 + n, *dq.shape))
        pos.copy_((pos + 13) % 300)
        g.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(other, want))


def test_norm_rope_out_counts_as_written():
    """Tensors given as `out` were written to: an autograd graph that saved one says so; and the same one twice is refused."""
    q, k = L.rand(5200, 1, 4, 2, 128).cuda(), L.rand(5201, 1, 4, 2, 128).cuda()
    cos, sin = cuda(*L.table(4, 128))
    args = (None, None, cos, sin)
    forward = lambda out: A.qk_norm_rope(q, k, *args, out=out)
    backward = lambda out: A.qk_norm_rope_backward(q, k, q, k, *args, out=out)
    general = (lambda out: A.layer._qk_norm_rope(q, k, *args, None, 1e-6, False, None, out),
               lambda out: A.layer._qk_norm_rope_backward(q, k, q, k, *args, None, 1e-6, False, None, out))
    for call in (forward, backward, *general):
        out = (torch.zeros_like(q), torch.zeros_like(k))
        x = torch.ones_like(q).requires_grad_()
        product = (x * out[1]).sum()
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            product.backward()
        with torch.inference_mode():
            made_here = (torch.empty_like(q), torch.empty_like(k))
            call(made_here)
        assert _equal(made_here, out)
        call(made_here)
        with pytest.raises(ValueError):
            call((out[0], out[0]))


def test_threads_on_streams_of_their_own():
    """Calls made at once, from several threads: workspaces and results of each are its own."""
    import threading
    do, q, k, v, o, lse, _ = cuda(*inputs(2, 4, 2, 260, 260, True, seed=5300))
    w, (cos, sin) = torch.ones(128, device="cuda"), cuda(*L.table(260, 128))

    def calls():
        return (*A.attention_backward(do, q, k, v, o, lse, causal=True), *A.qk_norm_rope(q, k, w, w, cos, sin),
                *A.qk_norm_rope_backward(do, k, q, k, w, w, cos, sin))

    want, right = calls(), []
    torch.cuda.synchronize()

    def run(n):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(15):
                got = calls()
                torch.cuda.current_stream().synchronize()
                if _equal(got, want):
                    right.append(n)

    threads = [threading.Thread(target=run, args=(n,)) for n in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(right) == 4 * 15


# --------------------------------------------------------------------------------------------- native call and general form
class Sub(torch.Tensor):
    pass


def _equal(a, b):
    return len(a) == len(b) and all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b))


def test_forms_agree():
    """The native call, the general form (subclasses, parameters, function modes) and the C entry."""
    do, q, k, v, o, lse, dl = cuda(*inputs(2, 4, 2, 70, 90, True, seed=6000, dlse=True))
    ref = A.attention_backward(do, q, k, v, o, lse, True, None, dl)
    assert type(ref) is tuple
    assert _equal(A.layer._attention_backward(do, q, k, v, o, lse, True, None, dl), ref)
    assert _equal(A.attention_backward(do.as_subclass(Sub), q, k, v, o, lse, 1, SCALE, dl), ref)
    assert _equal(A.attention_backward(do, torch.nn.Parameter(q), k, v, o, lse, causal=True, scale=torch.tensor(SCALE, dtype=torch.float64), dlse=dl), ref)
    with torch.device("cpu"):
        assert _equal(A.attention_backward(do, q, k, v, o, lse, True, dlse=dl), ref)
    nbytes = A.attn_bwd_workspace(2, 4, 2, 70, 90, 128, True)
    out, ws = [torch.empty_like(t) for t in (q, k, v)], torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    assert A.attn_bwd(do, dl, q, k, v, o, lse, *out, ws, nbytes, 2, 4, 2, 70, 90, 128, True, SCALE, torch.cuda.current_stream().cuda_stream) == 0
    assert _equal(out, ref)

    case = (2, 30, 6, 2, 96, torch.bfloat16, torch.int32, True, True, True)
    q, k, v, qw, kw, cos, sin, pos = rope_inputs(*case, seed=6100)
    q, k, v = on_device(q), on_device(k), on_device(v)
    qw, kw, cos, sin, pos = cuda(qw, kw, cos, sin, pos)
    dq, dk, dv = L.rand(6101, *q.shape).cuda(), L.rand(6102, *k.shape).cuda(), L.rand(6103, *v.shape).cuda()
    args = (qw, kw, cos, sin, pos, 1e-6, True)
    ref = A.qk_norm_rope(q, k, *args, v=v)
    assert _equal(A.layer._qk_norm_rope(q, k, *args, v, None), ref)
    assert _equal(A.qk_norm_rope(q.as_subclass(Sub), k, *args, v=v), ref)
    assert _equal(A.qk_norm_rope(q, k, torch.nn.Parameter(qw), *args[1:], v), ref)
    outs = [torch.zeros_like(t) for t in ref]
    got = A.qk_norm_rope(q, k, *args, v=v, out=outs)
    assert all(a is b for a, b in zip(got, outs)) and _equal(got, ref)
    ref = A.qk_norm_rope_backward(dq, dk, q, k, *args, dv=dv)
    assert _equal(A.layer._qk_norm_rope_backward(dq, dk, q, k, *args, dv, None), ref)
    with torch.device("cpu"):
        assert _equal(A.qk_norm_rope_backward(dq, dk, q, k, *args, dv=dv), ref)
    got = A.qk_norm_rope_backward(dq, dk, q, k, *args, dv=dv, out=outs)
    assert all(a is b for a, b in zip(got, outs)) and _equal(got, ref)
    assert _equal(A.qk_norm_rope_backward(dq, dk, q, k, None, None, *args[2:]), A.layer._qk_norm_rope_backward(dq, dk, q, k, None, None, *args[2:], None, None))


# ----------------------------------------------------------------------------------------------------------- sizes
def _device_rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16)


def test_backward_of_queries_beyond_32_bit_offsets():
    """4.6 GB of Q: a few rows with a gradient, the last ones among them, against the same rows alone."""
    B, Hq, Hkv, Sq, Skv = 1, 128, 2, 140000, 40
    q, k, v = _device_rand(1, B, Sq, Hq, 128), _device_rand(2, B, Skv, Hkv, 128), _device_rand(3, B, Skv, Hkv, 128)
    o, lse = A.attention(q, k, v)
    rows = torch.tensor([0, 1, 70001, 131071, 131072, Sq - 2, Sq - 1], device="cuda")
    do = torch.zeros_like(q)
    do[:, rows] = _device_rand(4, B, len(rows), Hq, 128)
    dq, dk, dv = A.attention_backward(do, q, k, v, o, lse)
    few = [t[:, rows].cpu() for t in (do, q, o)]
    want = L.backward64(few[0], few[1], k.cpu(), v.cpu(), few[2], lse[:, :, rows].cpu(), False, SCALE)
    L.check_backward((dq[:, rows], dk, dv), want)
    rest = torch.ones(Sq, dtype=torch.bool, device="cuda")
    rest[rows] = False
    assert not dq[:, rest].any()


def test_backward_of_keys_beyond_32_bit_offsets():
    B, Hq, Hkv, Sq, Skv = 1, 128, 128, 3, 140000
    q, do = _device_rand(5, B, Sq, Hq, 128), _device_rand(6, B, Sq, Hq, 128)
    k, v = _device_rand(7, B, Skv, Hkv, 128), _device_rand(8, B, Skv, Hkv, 128)
    o, lse = A.attention(q, k, v)
    dq, dk, dv = A.attention_backward(do, q, k, v, o, lse)
    keys = torch.tensor([0, 70001, 131071, 131072, Skv - 2, Skv - 1], device="cuda")
    # these keys alone: LSE and O stay those of all of them
    ref, bound, _ = L.backward64(do.cpu(), q.cpu(), k[:, keys].cpu(), v[:, keys].cpu(), o.cpu(), lse.cpu(), False, SCALE)
    for got, n in ((dk[:, keys], 1), (dv[:, keys], 2)):
        L.check_close(got, (ref[n], bound[n]))
    for h in (0, 127):      # dq of a head, which is a sum over all keys
        ref, bound, _ = L.backward64(*(t[:, :, h:h + 1].cpu() for t in (do, q, k, v, o)), lse[:, h:h + 1].cpu(), False, SCALE)
        L.check_close(dq[:, :, h:h + 1], (ref[0], bound[0]))


def test_backward_of_many_short_sequences():
    B = 70000
    q, k, v, do = (_device_rand(10 + n, B, 1, h, 128) for n, h in enumerate((2, 1, 1, 2)))
    o, lse = A.attention(q, k, v, causal=True)
    dl = torch.randn(B, 2, 1, device="cuda")
    dq, dk, dv = A.attention_backward(do, q, k, v, o, lse, causal=True, dlse=dl)
    # one key: P = 1, so dV is the sum of the heads' dO; dS = dLSE, so dQ = scale dLSE K
    want = do.float().sum(2, keepdim=True)
    # (P and dS each rounded, the results rounded, P off by 2^-16 before)
    assert ((dv.float() - want).abs() <= 2.1 * L.H * do.float().abs().sum(2, keepdim=True)).all()
    want = SCALE * dl.transpose(1, 2)[..., None] * k.float()
    size = SCALE * (dl.abs().transpose(1, 2)[..., None] + 2 * L.F * (do.float().abs() * v.float().abs()).sum(-1, keepdim=True)) * k.float().abs()
    assert ((dq.float() - want).abs() <= 2.1 * L.H * size + 2 * L.F * SCALE * (do.float().abs() * v.float().abs()).sum(-1, keepdim=True) * k.float().abs()).all()


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv,causal", [(512, 8, 4, 62, 62, True), (96, 16, 16, 200, 200, True), (208, 12, 4, 90, 200, False)])
def test_backward_of_large_batches_of_short_sequences(B, Hq, Hkv, Sq, Skv, causal):
    """Inputs beyond every cache, whose two kinds of items are dealt side by side: three sequences, over and over."""
    do, q, k, v, o, lse, _ = inputs(3, Hq, Hkv, Sq, Skv, causal, seed=5400)
    at = torch.arange(B) % 3
    got = A.attention_backward(*(t.cuda()[at.cuda()].contiguous() for t in (do, q, k, v, o, lse)), causal=causal)
    L.check_backward([x[:3] for x in got], L.backward64(do, q, k, v, o, lse, causal, SCALE))
    assert all(torch.equal(x, x[at.cuda()]) for x in got)


def test_norm_rope_beyond_32_bit_offsets():
    S, Hq, Hkv = 70000, 256, 1
    q, k = _device_rand(20, 1, S, Hq, 128), _device_rand(21, 1, S, Hkv, 128)
    cos, sin = A.rope_table(S)
    got = A.qk_norm_rope(q, k, None, None, cos, sin)
    at = torch.tensor([0, 1, 32767, 65535, 65536, S - 1], device="cuda")
    places = at.cpu()[None]
    L.check_close(got[0][:, at], L.norm_rope64(q[:, at].cpu(), None, cos.cpu(), sin.cpu(), places, 1e-6, False))
    L.check_close(got[1][:, at], L.norm_rope64(k[:, at].cpu(), None, cos.cpu(), sin.cpu(), places, 1e-6, False))
    w = torch.ones(128, device="cuda")
    dq = torch.zeros_like(q)
    dq[:, at] = _device_rand(22, 1, len(at), Hq, 128)
    dx, _, dqw, _ = A.qk_norm_rope_backward(dq, torch.zeros_like(k), q, k, w, w, cos, sin)
    (ref, bound), (dw, dw_bound) = L.norm_rope_backward64(dq[:, at].cpu(), q[:, at].cpu(), w.cpu(), cos.cpu(), sin.cpu(), places, 1e-6, False)
    L.check_close(dx[:, at], (ref, bound))
    L.check_close(dqw, (dw, dw_bound))


def test_calls_inside_torch_func_raise():
    """torch.func hands on tensors without storage: torch's own exception for those, and the next call is none the worse."""
    do, q, k, v, o, lse, _ = cuda(*inputs(1, 2, 1, 40, 40, True, seed=6200))
    cos, sin = cuda(*L.table(40, 128))
    want = A.attention_backward(do, q, k, v, o, lse, causal=True)
    for call in (lambda x: A.attention_backward(do, x, k, v, o, lse, causal=True)[0], lambda x: A.qk_norm_rope(x, k, None, None, cos, sin)[0],
                 lambda x: A.qk_norm_rope_backward(x, k, q, k, None, None, cos, sin)[0]):
        with pytest.raises(RuntimeError, match="storage"):
            torch.func.grad(lambda x: call(x).float().sum())(q)
    assert _equal(A.attention_backward(do, q, k, v, o, lse, causal=True), want)


@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv,causal", [(13, 8, 8, 600, 600, True), (11, 16, 8, 1300, 1300, True), (97, 8, 8, 300, 300, True), (29, 8, 8, 450, 700, False)])
def test_backward_of_group_counts_without_divisors(B, Hq, Hkv, Sq, Skv, causal):
    """Windows of groups, the last one longer than the others, each kind of items by itself and both side by side: two sequences, over and over."""
    do, q, k, v, o, lse, _ = inputs(2, Hq, Hkv, Sq, Skv, causal, seed=5500)
    at = (torch.arange(B) % 2).cuda()
    got = A.attention_backward(*(t.cuda()[at].contiguous() for t in (do, q, k, v, o, lse)), causal=causal)
    G = Hq // Hkv
    for h in (0, Hkv - 1):          # (the 64-bit form of two heads)
        part = slice(h * G, h * G + G)
        few = (do[:, :, part], q[:, :, part], k[:, :, h:h + 1], v[:, :, h:h + 1], o[:, :, part], lse[:, part])
        L.check_backward((got[0][:2, :, part], got[1][:2, :, h:h + 1], got[2][:2, :, h:h + 1]), L.backward64(*few, causal, SCALE))
    assert all(torch.equal(x, x[at]) for x in got)
