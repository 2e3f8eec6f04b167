"""What the operators around the attention forward are timed on: its backward pass, the per-head norm of queries and keys
with the position rotation, and the gradient of that.  Each as a layer calls it: BF16 tensors [B, S, H, 128] that are on
the device, queries, keys and values as slices of one fused projection where the layer has one.

Sizes: the head counts and sequence lengths of `paper_2603_24517_amd/workloads.py` (8 x 4096, 4 x 8192, 2 x 16384,
1 x 512), and generic ones for what that list leaves out: ragged prompts, odd lengths, few tokens.
"""
import math

import torch

own = False

D = 128
SCALE = D ** -0.5
BASE = 10000.0
EPS = 1e-6
TABLE = 32768           # positions of the rotation tables


def _bwd(name, B, Hq, Hkv, Sq, Skv, causal, q_mul=1.0, do_mul=1.0, dlse=False):
    return {"name": name, "op": "attention_backward", "B": B, "Hq": Hq, "Hkv": Hkv, "Sq": Sq, "Skv": Skv, "causal": causal,
            "q_mul": q_mul, "do_mul": do_mul, "dlse": dlse}


def _norm(name, op, B, Hq, Hkv, S, rot=128, weight="bf16", positions="none", interleaved=False, fused=True):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "S": S, "rot": rot, "weight": weight,
            "positions": positions, "interleaved": interleaved, "fused": fused}


def listed():
    return [
        # the smallest problem of the workload list, trained: one short sequence, four heads, bidirectional
        _bwd("bwd_full_1x512", 1, 4, 4, 512, 512, False),
        # a batch of short ragged prompts (fine-tuning), one query head per K/V head; gradients of a mean loss are small
        _bwd("bwd_causal_24x200", 24, 16, 16, 200, 200, True, do_mul=2.0 ** -10),
        # one document of odd length through a grouped-query layer
        _bwd("bwd_gqa4_causal_1x1111", 1, 32, 8, 1111, 1111, True),
        # a piece of a long document against the keys before it, merged with other pieces through LSE, which has a gradient
        _bwd("bwd_gqa4_chunk_512_of_8192", 1, 32, 8, 512, 8192, True, dlse=True),
        # pre-training batches: the headline shape, bidirectional
        _bwd("bwd_full_8x4096", 8, 16, 16, 4096, 4096, False),
        # the longest listed: grouped-query heads, causal, long documents
        _bwd("bwd_gqa4_causal_2x16384", 2, 32, 8, 16384, 16384, True),
        # generation: one token of each of 64 sequences, each at a place of its own
        _norm("norm_rope_64x1", "qk_norm_rope", 64, 32, 8, 1, positions="int64"),
        # a ragged prompt, half of each head rotated, separate projections
        _norm("norm_rope_3x1111", "qk_norm_rope", 3, 32, 8, 1111, rot=64, weight="fp32", positions="int32", fused=False),
        # a training batch through a fused projection
        _norm("norm_rope_8x4096", "qk_norm_rope", 8, 16, 16, 4096),
        # gradients: one short sequence; documents packed into rows, adjacent pairs rotated; a training batch
        _norm("norm_rope_bwd_1x512", "qk_norm_rope_backward", 1, 4, 4, 512, weight="fp32"),
        _norm("norm_rope_bwd_3x1111", "qk_norm_rope_backward", 3, 32, 8, 1111, positions="int64", interleaved=True, fused=False),
        _norm("norm_rope_bwd_8x4096", "qk_norm_rope_backward", 8, 16, 16, 4096),
    ]


HEADS = [(16, 16), (32, 8), (32, 4), (64, 8), (4, 4)]       # the head counts of the workload list
MOST_FLOPS = 10.0 * D * 2 * 32 * 16384 * 16384 / 2          # the last listed backward pass
MOST_ROWS = 8 * 4096 * 48                                   # (token, head) rows of the largest listed norm


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    Hq, Hkv = rng.choice(HEADS)
    op = rng.choice(["attention_backward", "attention_backward", "qk_norm_rope", "qk_norm_rope_backward"])
    if op == "attention_backward":
        kind = rng.choice(["same", "same", "chunk", "more_rows"])
        if kind == "same":
            Sq = Skv = _log(rng, 64, 16384)
            B = _log(rng, 1, max(1, 32768 // Sq))
            causal = rng.random() < 0.7
        elif kind == "chunk":
            Sq = _log(rng, 1, 2048)
            Skv = Sq + _log(rng, 64, 14000)
            B = rng.choice([1, 1, 2, 3])
            causal = True
        else:                                   # more queries than keys; with the mask the first rows have no key
            Skv = _log(rng, 40, 2048)
            Sq = Skv + _log(rng, 1, 2000)
            B = rng.choice([1, 2, 4])
            causal = rng.random() < 0.5
        case = _bwd("", B, Hq, Hkv, Sq, Skv, causal, q_mul=rng.choice([1.0, 1.0, 2.0]), do_mul=rng.choice([1.0, 2.0 ** -10]),
                    dlse=rng.random() < 0.3)
        while case["B"] > 1 and work(case)["flops"] > MOST_FLOPS:
            case["B"] //= 2
        while work(case)["flops"] > MOST_FLOPS:
            case["Hq"] //= 2
            case["Hkv"] = max(1, case["Hkv"] // 2)
    else:
        S = rng.choice([1, _log(rng, 2, 16384), _log(rng, 2, 16384)])
        B = _log(rng, 1, max(1, min(256, MOST_ROWS // (S * (Hq + 2 * Hkv)))))
        case = _norm("", op, B, Hq, Hkv, S, rot=rng.choice([32, 64, 96, 128, 128]), weight=rng.choice(["bf16", "fp32", "none"]),
                     positions=rng.choice(["none", "int32", "int64"]), interleaved=rng.random() < 0.4, fused=rng.random() < 0.6)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _forward(q, k, v, causal):
    """O (BF16) and LSE of the forward pass, in pieces of the score matrix."""
    B, Sq, Hq, _ = q.shape
    _, Skv, Hkv, _ = k.shape
    o = torch.empty_like(q)
    lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device)
    for b, heads, kv, r0, r1 in _pieces(B, Hq, Hkv, Sq, Skv):
        s = _scores(q, k, b, heads, kv, r0, r1, causal)
        l = torch.logsumexp(s, dim=-1)
        p = torch.exp(s - torch.where(l == -math.inf, 0.0, l)[..., None])
        o[b, r0:r1, heads] = (p @ _heads(v, b, kv)).transpose(0, 1).to(torch.bfloat16)
        lse[b, heads, r0:r1] = l
    return o, lse


def _rotation_tables(rot):
    angle = torch.arange(TABLE, dtype=torch.float64, device="cuda")[:, None] * BASE ** (
        -torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    return angle.cos().float(), angle.sin().float()


def prepare(case, seed):
    g = _generator(seed)
    B, Hq, Hkv = case["B"], case["Hq"], case["Hkv"]
    st = {"case": case}
    if case["op"] == "attention_backward":
        Sq, Skv = case["Sq"], case["Skv"]
        st["q"] = _normal(g, B, Sq, Hq, D) * case["q_mul"]         # exact: powers of two
        st["k"], st["v"] = _normal(g, B, Skv, Hkv, D), _normal(g, B, Skv, Hkv, D)
        st["do"] = _normal(g, B, Sq, Hq, D) * case["do_mul"]
        st["o"], st["lse"] = _forward(st["q"], st["k"], st["v"], case["causal"])
        st["dlse"] = None
        if case["dlse"]:
            st["dlse"] = torch.randn((B, Hq, Sq), generator=g, device="cuda") * case["do_mul"]
        return st
    S = case["S"]

    def projection():
        if case["fused"]:
            return list(_normal(g, B, S, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], dim=2))
        return [_normal(g, B, S, Hq, D), _normal(g, B, S, Hkv, D), _normal(g, B, S, Hkv, D)]

    st["q"], st["k"], st["v"] = projection()
    st["qw"] = st["kw"] = None
    if case["weight"] != "none":
        dtype = torch.float32 if case["weight"] == "fp32" else torch.bfloat16
        st["qw"], st["kw"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype) for _ in range(2))
    st["cos"], st["sin"] = _rotation_tables(case["rot"])
    st["positions"] = None
    if case["positions"] != "none":
        dtype = torch.int32 if case["positions"] == "int32" else torch.int64
        if S == 1:          # generation: every sequence at a place of its own
            st["positions"] = torch.randint(0, TABLE, (B, 1), generator=g, device="cuda").to(dtype)
        else:               # documents packed into rows: places start again with each
            start = torch.randint(0, S, (B, 1), generator=g, device="cuda")
            i = torch.arange(S, device="cuda")[None]
            st["positions"] = torch.where(i < start, i, i - start).to(dtype).contiguous()
    if case["op"] == "qk_norm_rope_backward":
        st["dq"], st["dk"], st["dv"] = _normal(g, B, S, Hq, D), _normal(g, B, S, Hkv, D), _normal(g, B, S, Hkv, D)
    return st


# ------------------------------------------------------------------------------------------------------------ plain forms
def _pieces(B, Hq, Hkv, Sq, Skv, most=1 << 27):
    """(batch entry, query heads, K/V heads, first row, last row) of pieces of at most `most` scores: whole heads where they fit."""
    G = Hq // Hkv
    kv = max(1, min(Hkv, most // (G * Sq * Skv)))
    rows = Sq if kv > 1 else max(1, min(Sq, most // (G * Skv)))
    for b in range(B):
        for h in range(0, Hkv, kv):
            top = min(Hkv, h + kv)
            for r0 in range(0, Sq, rows):
                yield b, slice(h * G, top * G), (slice(h, top), G), r0, min(Sq, r0 + rows)


def _heads(x, b, kv):
    """K or V of these heads, one per query head, [heads, Skv, D] in 32 bits."""
    heads, G = kv
    return x[b, :, heads].transpose(0, 1).float().repeat_interleave(G, dim=0).contiguous()


def _scores(q, k, b, heads, kv, r0, r1, causal):
    s = (q[b, r0:r1, heads].transpose(0, 1).float().contiguous() @ _heads(k, b, kv).transpose(1, 2)) * SCALE
    if causal:
        off = k.shape[1] - q.shape[1]
        i = torch.arange(r0, r1, device=q.device)[:, None]
        s = s.masked_fill(torch.arange(k.shape[1], device=q.device)[None] > i + off, -math.inf)
    return s


def _plain_attention_backward(st):
    q, k, v, o, lse, do = (st[n] for n in ("q", "k", "v", "o", "lse", "do"))
    B, Sq, Hq, _ = q.shape
    _, Skv, Hkv, _ = k.shape
    G = Hq // Hkv
    dq = torch.empty_like(q)
    dk = torch.zeros(k.shape, dtype=torch.float32, device=k.device)
    dv = torch.zeros(v.shape, dtype=torch.float32, device=v.device)
    delta = (do.float() * o.float()).sum(-1).transpose(1, 2)
    if st["dlse"] is not None:
        delta = delta - st["dlse"]
    for b, heads, kv, r0, r1 in _pieces(B, Hq, Hkv, Sq, Skv):
        l = lse[b, heads, r0:r1, None]
        p = torch.exp(_scores(q, k, b, heads, kv, r0, r1, st["case"]["causal"]) - torch.where(l == -math.inf, 0.0, l))
        dor = do[b, r0:r1, heads].transpose(0, 1).float().contiguous()
        dv[b, :, kv[0]] += (p.transpose(1, 2) @ dor).unflatten(0, (-1, G)).sum(1).transpose(0, 1)
        ds = p * (dor @ _heads(v, b, kv).transpose(1, 2) - delta[b, heads, r0:r1, None]) * SCALE
        del p
        dq[b, r0:r1, heads] = (ds @ _heads(k, b, kv)).transpose(0, 1).to(torch.bfloat16)
        qr = q[b, r0:r1, heads].transpose(0, 1).float().contiguous()
        dk[b, :, kv[0]] += (ds.transpose(1, 2) @ qr).unflatten(0, (-1, G)).sum(1).transpose(0, 1)
    return dq, dk.to(torch.bfloat16), dv.to(torch.bfloat16)


def _angles(st):
    """cos and sin of each token, [B or 1, S, 1, rot / 2]."""
    S = st["q"].shape[1]
    if st["positions"] is None:
        return st["cos"][None, :S, None], st["sin"][None, :S, None]
    i = st["positions"].long()
    return st["cos"][i][:, :, None], st["sin"][i][:, :, None]


def _pairs(x, rot, interleaved):
    """The two members of each rotated pair."""
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2]
    return x[..., :rot // 2], x[..., rot // 2:rot]


def _rotated(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    a, b = _pairs(x, rot, interleaved)
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_norm_rope(st):
    cos, sin = _angles(st)

    def one(x, w):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if w is not None:
            y = y * w.float()
        return _rotated(y, cos, sin, st["case"]["interleaved"]).to(torch.bfloat16)

    out = one(st["q"], st["qw"]), one(st["k"], st["kw"])
    return (*out, st["v"].contiguous()) if st["case"]["fused"] else out


def _plain_norm_rope_backward(st):
    cos, sin = _angles(st)

    def one(dz, x, w):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xhat = x * r
        dy = _rotated(dz.float(), cos, -sin, st["case"]["interleaved"])
        dw = None if w is None else (dy * xhat).sum((0, 1, 2), dtype=torch.float64).float()
        g = dy if w is None else dy * w.float()
        return (r * (g - xhat * (g * xhat).mean(-1, keepdim=True))).to(torch.bfloat16), dw

    dq, dqw = one(st["dq"], st["q"], st["qw"])
    dk, dkw = one(st["dk"], st["k"], st["kw"])
    out = [torch.cat((dq, dk, st["dv"]), dim=2)] if st["case"]["fused"] else [dq, dk]
    return out if dqw is None else out + [dqw, dkw]


# ------------------------------------------------------------------------------------------------------------------ a pass
def run(st):
    case = st["case"]
    if not own:
        return {"attention_backward": _plain_attention_backward, "qk_norm_rope": _plain_norm_rope,
                "qk_norm_rope_backward": _plain_norm_rope_backward}[case["op"]](st)
    import paper_2603_24517_amd as attn
    if case["op"] == "attention_backward":
        return attn.attention_backward(st["do"], st["q"], st["k"], st["v"], st["o"], st["lse"], causal=case["causal"],
                                       dlse=st["dlse"])
    common = (st["q"], st["k"], st["qw"], st["kw"], st["cos"], st["sin"], st["positions"], EPS, case["interleaved"])
    if case["op"] == "qk_norm_rope":
        if case["fused"]:
            return attn.qk_norm_rope(*common, v=st["v"])
        return attn.qk_norm_rope(*common)
    if case["fused"]:
        B, S, Hq, Hkv = case["B"], case["S"], case["Hq"], case["Hkv"]
        dqkv = torch.empty((B, S, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
        *_, dqw, dkw = attn.qk_norm_rope_backward(st["dq"], st["dk"], *common, dv=st["dv"],
                                                  out=dqkv.split([Hq, Hkv, Hkv], dim=2))
        out = [dqkv]
    else:
        *out, dqw, dkw = attn.qk_norm_rope_backward(st["dq"], st["dk"], *common)
    return out if dqw is None else out + [dqw, dkw]


def _unmasked(case):
    """(query, key) pairs that are not masked, per head."""
    B, Sq, Skv = case["B"], case["Sq"], case["Skv"]
    if not case["causal"]:
        return B * Sq * Skv
    full = min(Sq, Skv)             # rows that see a part of the last `full` keys
    return B * (full * (Skv - full) + full * (full + 1) // 2)


def work(case):
    B, Hq, Hkv = case["B"], case["Hq"], case["Hkv"]
    if case["op"] == "attention_backward":
        Sq, Skv = case["Sq"], case["Skv"]
        # q, o, do read and dq written; k, v read and dk, dv written; lse (and its gradient) read
        nbytes = 2 * D * B * (4 * Hq * Sq + 4 * Hkv * Skv) + 4 * B * Hq * Sq * (2 if case["dlse"] else 1)
        return {"bytes": nbytes, "flops": 10.0 * D * Hq * _unmasked(case)}
    S = case["S"]
    rows = B * S * (Hq + Hkv)
    copied = B * S * Hkv if case["fused"] else 0
    # each token's place, and the table rows of the places that there are
    places = 0 if case["positions"] == "none" else B * S * (4 if case["positions"] == "int32" else 8)
    table = (min(TABLE, B) if S == 1 and case["positions"] != "none" else S) * case["rot"] * 4
    if case["op"] == "qk_norm_rope":
        return {"bytes": 2 * D * 2 * (rows + copied) + places + table, "flops": 8.0 * D * rows}
    return {"bytes": 2 * D * (3 * rows + 2 * copied) + places + table, "flops": 18.0 * D * rows}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attention_backward":
        return _exact_attention_backward(st)
    x = {n: st[n].double().requires_grad_(n in "qk") for n in "qkv"}
    w = {n: None if st[n] is None else st[n].double().requires_grad_() for n in ("qw", "kw")}
    S, rot = case["S"], case["rot"]
    i = torch.arange(S, device="cuda")[None] if st["positions"] is None else st["positions"].long()
    turn = torch.complex(st["cos"].double(), st["sin"].double())[i][:, :, None]

    def one(x, w):
        y = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / D + EPS)
        if w is not None:
            y = w * y
        head, tail = y[..., :rot], y[..., rot:]
        head = head.unflatten(-1, (-1, 2)) if case["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat((z.flatten(-2), tail), -1)

    q, k = one(x["q"], w["qw"]), one(x["k"], w["kw"])
    if case["op"] == "qk_norm_rope":
        return (q.detach(), k.detach(), x["v"].detach()) if case["fused"] else (q.detach(), k.detach())
    leaves = [x["q"], x["k"]] + ([] if w["qw"] is None else [w["qw"], w["kw"]])
    dq, dk, *dw = torch.autograd.grad([q, k], leaves, [st["dq"].double(), st["dk"].double()])
    return ([torch.cat((dq, dk, st["dv"].double()), dim=2)] if case["fused"] else [dq, dk]) + dw


def _exact_attention_backward(st):
    q, k, v, o, do, lse = (st[n].double() for n in ("q", "k", "v", "o", "do", "lse"))
    dlse = 0.0 if st["dlse"] is None else st["dlse"].double()
    B, Sq, Hq, _ = q.shape
    _, Skv, Hkv, _ = k.shape
    G = Hq // Hkv
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    part = max(1, (1 << 26) // Skv)
    key = torch.arange(Skv, device="cuda")
    for b in range(B):
        for h in range(Hq):
            kh, vh = k[b, :, h // G].contiguous(), v[b, :, h // G].contiguous()
            for r in range(0, Sq, part):
                at = slice(r, min(Sq, r + part))
                qh, gh = q[b, at, h].contiguous(), do[b, at, h].contiguous()
                d = torch.linalg.vecdot(gh, o[b, at, h])
                if st["dlse"] is not None:
                    d = d - dlse[b, h, at]
                valid = torch.isfinite(lse[b, h, at])[:, None]
                if st["case"]["causal"]:
                    valid = valid & (key[None] <= torch.arange(at.start, at.stop, device="cuda")[:, None] + (Skv - Sq))
                p = torch.where(valid, torch.exp(torch.mm(qh, kh.t()) / math.sqrt(D) - lse[b, h, at, None]), 0.0)
                dv[b, :, h // G] += torch.mm(p.t(), gh)
                p *= torch.mm(gh, vh.t()) - d[:, None]
                p /= math.sqrt(D)
                dq[b, at, h] = torch.mm(p, kh)
                dk[b, :, h // G] += torch.mm(p.t(), qh)
    return dq, dk, dv
