"""The serving operators over a paged K/V cache: what is measured of them, and their plain forms.

Three operators of one serving step, each with its head dimension fixed at 128:

  norm_rope   RMS norm of every query and key head, then the rotary encoding, in one pass
  append      a batch's new keys and values into a paged cache, keys normalised and rotated on the way
  attend      causal attention of a batch's new tokens (one of them, a few, or a chunk) over the paged cache

With `own` false `run` computes the operator in elementary torch operations (32 bits; angles in 64); with `own` true it
makes the calls a user of the library makes.  `exact` evaluates the definitions in 64 bits.
"""
import math
import random

import torch

own = False

D = 128
THETA = 500000.0
EPS = 1e-6
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # One decode step of 64 short requests: every request's one new token, the projection's output read in place.
        dict(name="norm_rope_step", op="norm_rope", dtype="bf16", tokens=64, hq=32, hkv=8, norm=True, fused=True),
        # A prefill chunk of 8192 tokens of a model with 64 query heads.
        dict(name="norm_rope_chunk", op="norm_rope", dtype="bf16", tokens=8192, hq=64, hkv=8, norm=True, fused=True),
        # The accuracy path: 32-bit heads, an odd number of tokens, separate tensors.
        dict(name="norm_rope_f32", op="norm_rope", dtype="f32", tokens=1021, hq=8, hkv=8, norm=True, fused=False),
        # One decode step of 64 requests: 64 tokens land in 64 different pages.
        dict(name="append_step", op="append", dtype="bf16", requests=64, new=1, context=1000, spread=1, hkv=8, page=16, head_major=False, norm=False),
        # Five requests' prefill chunks, 8192 new tokens in all, keys normalised as well.
        dict(name="append_chunks", op="append", dtype="bf16", requests=5, new=1638, context=500, spread=2, hkv=8, page=64, head_major=False, norm=True),
        # 32-bit cache, a head-major layout, a page size that is no power of two.
        dict(name="append_f32", op="append", dtype="f32", requests=3, new=333, context=100, spread=3, hkv=8, page=24, head_major=True, norm=False),
        # The smallest step: one request's one token.
        dict(name="attend_one", op="attend", dtype="bf16", requests=1, new=1, context=4099, spread=0, hq=32, hkv=8, page=16, head_major=False),
        # A decode step of 64 requests of mixed lengths.
        dict(name="attend_step", op="attend", dtype="bf16", requests=64, new=1, context=3000, spread=4, hq=32, hkv=8, page=64, head_major=False),
        # A decode step of three long requests (the long-context case), 64 query heads.
        dict(name="attend_long", op="attend", dtype="bf16", requests=3, new=1, context=131072, spread=5, hq=64, hkv=8, page=128, head_major=True),
        # One prefill chunk resumed on a long stored prefix.
        dict(name="attend_chunk", op="attend", dtype="bf16", requests=1, new=2048, context=30720, spread=0, hq=32, hkv=8, page=64, head_major=False),
        # A mixed batch: chunks of several requests beside requests with a few tokens or none, odd page size.
        dict(name="attend_mixed", op="attend", dtype="bf16", requests=24, new=300, context=2000, spread=6, hq=32, hkv=8, page=48, head_major=False),
        # The accuracy path, 32-bit cache.
        dict(name="attend_f32", op="attend", dtype="f32", requests=3, new=200, context=500, spread=7, hq=8, hkv=8, page=16, head_major=False),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], even in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["norm_rope", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 5, 7, 8])
    page = 8 * _between(rng, 1, 32)
    if op == "norm_rope":
        return dict(op=op, dtype=dtype, tokens=_between(rng, 1, 8192), hq=hq, hkv=hkv, norm=rng.random() < 0.8, fused=rng.random() < 0.5)
    if op == "append":
        requests = _between(rng, 1, 64)
        return dict(op=op, dtype=dtype, requests=requests, new=_between(rng, 1, max(1, 8192 // requests)), context=_between(rng, 1, 2000),
                    spread=rng.randrange(1, 1 << 20), hkv=hkv, page=page, head_major=rng.random() < 0.5, norm=rng.random() < 0.5)
    kind = rng.choice(["step", "chunk"])
    if kind == "step":
        requests = _between(rng, 1, 64)
        new, context = _between(rng, 1, 8), _between(rng, 1, min(65536, 262144 // requests))
    else:
        requests = _between(rng, 1, 8)
        new, context = _between(rng, 9, 1500 // requests), _between(rng, 1, 16384 // requests)
    if dtype == "f32":
        context = min(context, 2048)
    return dict(op=op, dtype=dtype, requests=requests, new=new, context=context, spread=rng.randrange(0, 1 << 20), hq=hq, hkv=hkv, page=page,
                head_major=rng.random() < 0.5)


def lengths(case):
    """(new tokens, cached tokens with the new ones) of every request: around `new` and `context`, from the case alone."""
    b, r = case["requests"], random.Random(case["spread"] + 77)
    if case["spread"] == 0:
        return [case["new"]] * b, [case["context"] + case["new"]] * b
    if case["new"] == 1:
        n = [1] * b
    else:  # from none to twice as many; every fourth request is in its decode phase
        n = [1 if i % 4 == 3 else r.randint(0, 2 * case["new"]) for i in range(b)]
        n[0] = case["new"]
    ctx = [max(0, int(case["context"] * math.exp(r.uniform(-1.5, 0.7)))) for _ in range(b)]
    ctx[0] = case["context"]
    return n, [c + m for c, m in zip(ctx, n)]


def _tokens_heads(case):
    n, kv = lengths(case)
    return sum(n), n, kv


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm_rope":
        t, h = case["tokens"], case["hq"] + case["hkv"]
        return {"bytes": 2 * t * h * D * size + 4 * t, "flops": t * h * D * 8}
    t, n, kv = _tokens_heads(case)
    if case["op"] == "append":
        return {"bytes": 4 * t * case["hkv"] * D * size + 4 * (2 * case["requests"] + t // case["page"]), "flops": t * case["hkv"] * D * 8}
    seen = sum(k for k, m in zip(kv, n) if m > 0)
    pairs = sum(m * k - m * (m - 1) // 2 for k, m in zip(kv, n))
    return {"bytes": 2 * seen * case["hkv"] * D * size + 2 * t * case["hq"] * D * size + 4 * t * case["hq"] + 4 * seen // case["page"],
            "flops": 4 * D * case["hq"] * pairs}


# ------------------------------------------------------------------------------------------ the inputs
def _table(n_pos):
    """The rotary table of the library's documented layout: fine cosines and sines by channel, coarse ones by 64 positions."""
    f = torch.exp2(-torch.arange(64, dtype=torch.float64, device=DEV) / 64 * math.log2(THETA))
    b = torch.arange(64, dtype=torch.float64, device=DEV)
    a = 64.0 * torch.arange((n_pos + 63) // 64, dtype=torch.float64, device=DEV)
    fine, coarse = f[:, None] * b[None, :], a[:, None] * f[None, :]
    return torch.cat([t.reshape(-1) for t in (fine.cos(), fine.sin(), coarse.cos(), coarse.sin())]).float()


def _heads(gen, tokens, heads, dtype):
    return torch.randn((tokens, heads, D), generator=gen, device=DEV).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    s = dict(case)
    if case["op"] != "attend":
        s["q_weight"] = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dtype)
        s["k_weight"] = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dtype)
    if case["op"] == "norm_rope":
        t, hq, hkv = case["tokens"], case["hq"], case["hkv"]
        if case["fused"]:  # column slices of one fused projection
            qkv = _heads(gen, t, hq + 2 * hkv, dtype)
            s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]
        else:
            s["q"], s["k"] = _heads(gen, t, hq, dtype), _heads(gen, t, hkv, dtype)
        s["n_pos"] = 131072
        s["positions"] = torch.randint(0, s["n_pos"], (t,), generator=gen, device=DEV, dtype=torch.int32)
        s["table"] = _table(s["n_pos"])
        return s
    t, n, kv = _tokens_heads(case)
    b, page, hkv = case["requests"], case["page"], case["hkv"]
    need = [-(-k // page) for k in kv]
    total = sum(need) + 3
    order = torch.randperm(total, generator=gen, device=DEV).int()
    table = torch.zeros((b, max(max(need), 1)), dtype=torch.int32, device=DEV)
    rows = torch.arange(table.shape[1], device=DEV)[None, :]
    need_t = torch.tensor(need, device=DEV)[:, None]
    first = torch.tensor([sum(need[:i]) for i in range(b)], device=DEV)[:, None]
    s["block_table"] = torch.where(rows < need_t, order[(first + rows).clamp(max=total - 1)], table)
    shape = (total, hkv, page, D) if case["head_major"] else (total, page, hkv, D)
    pages = [torch.randn(shape, generator=gen, device=DEV).to(dtype) for _ in range(2)]
    if case["head_major"]:
        pages = [p.transpose(1, 2) for p in pages]
    s["k_pages"], s["v_pages"] = pages
    cu = [sum(n[:i]) for i in range(b + 1)]
    s["cu_q"] = torch.tensor(cu, dtype=torch.int32, device=DEV)
    s["kv_lens"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    s["most_new"], s["most_kv"] = max(n), max(kv)
    if case["op"] == "append":
        s["k"], s["v"] = _heads(gen, t, hkv, dtype), _heads(gen, t, hkv, dtype)
        s["n_pos"] = max(kv)
        s["table"] = _table(s["n_pos"])
    else:
        s["q"] = _heads(gen, t, case["hq"], dtype)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    if s["op"] == "norm_rope":
        return _own_norm_rope(s) if own else _plain_norm_rope(s)
    if s["op"] == "append":
        return _own_append(s) if own else _plain_append(s)
    return _own_attend(s) if own else _plain_attend(s)


def _own_norm_rope(s):
    from paper_2409_15104_b200 import binding
    q, k = binding.pec_qk_norm_rope(s["q"], s["k"], norm=s["norm"], q_weight=s["q_weight"] if s["norm"] else None,
                                    k_weight=s["k_weight"] if s["norm"] else None, eps=EPS, tables=(s["table"], s["n_pos"]),
                                    positions=s["positions"])
    return {"q": q, "k": k}


def _own_append(s):
    from paper_2409_15104_b200 import binding
    binding.pec_kv_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["block_table"], s["cu_q"], s["kv_lens"], norm=s["norm"],
                          k_weight=s["k_weight"] if s["norm"] else None, eps=EPS, tables=(s["table"], s["n_pos"]))
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _own_attend(s):
    from paper_2409_15104_b200 import binding
    o, lse = binding.pec_paged_attn(s["q"], s["k_pages"], s["v_pages"], s["block_table"], s["cu_q"], s["kv_lens"], max_q_len=s["most_new"])
    return {"o": o, "lse": lse}


def _norm(x, weight):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)


def _turn(x, positions):
    """The rotate-half pairing: channel i < 64 with channel i + 64, by position * theta^(-2 i / 128)."""
    f = torch.exp2(-torch.arange(64, dtype=torch.float64, device=x.device) / 64 * math.log2(THETA))
    angle = positions.double()[:, None, None] * f
    c, t = angle.cos().to(x.dtype), angle.sin().to(x.dtype)
    lo, hi = x[..., :64], x[..., 64:]
    return torch.cat([lo * c - hi * t, hi * c + lo * t], -1)


def _plain_norm_rope(s):
    q, k = s["q"].float(), s["k"].float()
    if s["norm"]:
        q, k = _norm(q, s["q_weight"]), _norm(k, s["k_weight"])
    return {"q": _turn(q, s["positions"]).to(s["q"].dtype), "k": _turn(k, s["positions"]).to(s["k"].dtype)}


def _places(s):
    """Request and position of every new token."""
    cu, t = s["cu_q"].long(), s["k"].shape[0]
    row = torch.arange(t, device=cu.device)
    b = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return b, s["kv_lens"].long()[b] - cu[b + 1] + row


def _plain_append(s):
    b, pos = _places(s)
    k = s["k"].float()
    if s["norm"]:
        k = _norm(k, s["k_weight"])
    page, slot = s["block_table"][b, pos // s["page"]].long(), pos % s["page"]
    s["k_pages"][page, slot] = _turn(k, pos).to(s["k"].dtype)
    s["v_pages"][page, slot] = s["v"]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attend(s):
    q, cu, kv_len = s["q"], s["cu_q"].long(), s["kv_lens"].long()
    dev, (t, hq, _), hkv = q.device, q.shape, s["hkv"]
    n = cu[1:] - cu[:-1]
    i, j = torch.arange(s["most_new"], device=dev), torch.arange(s["most_kv"], device=dev)
    rows = (cu[:-1, None] + i).clamp(max=t - 1)
    real = i < n[:, None]                                                       # [B, n]
    pages = s["block_table"].long()
    keys = s["k_pages"][pages].flatten(1, 2)[:, :s["most_kv"]].float()         # [B, kv, Hkv, D]
    vals = s["v_pages"][pages].flatten(1, 2)[:, :s["most_kv"]].float()
    held = (j < kv_len[:, None])[:, :, None, None]
    keys, vals = keys.masked_fill(~held, 0.0), vals.masked_fill(~held, 0.0)
    x = q[rows].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)      # [B, Hkv, g n, D]
    score = (x @ keys.permute(0, 2, 3, 1)).unflatten(2, (hq // hkv, s["most_new"])) * (1 / math.sqrt(D))
    pos = kv_len[:, None] - n[:, None] + i
    score.masked_fill_(~(j <= pos[:, :, None])[:, None, None], float("-inf"))
    most = score.amax(-1, keepdim=True)
    score.sub_(most).exp_()
    total = score.sum(-1, keepdim=True)
    o = (score.flatten(2, 3) @ vals.transpose(1, 2)).unflatten(2, (hq // hkv, s["most_new"])) / total
    lse = (most + total.log()).squeeze(-1)
    o, lse = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[real], lse.permute(0, 3, 1, 2).flatten(2, 3)[real]
    return {"o": o.to(q.dtype), "lse": lse}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm_rope":
        return {"q": _exact_heads(s["q"], s["q_weight"] if s["norm"] else None, s["positions"]),
                "k": _exact_heads(s["k"], s["k_weight"] if s["norm"] else None, s["positions"])}
    n, kv = lengths(case)
    page = case["page"]
    if case["op"] == "append":
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        row = 0
        for b in range(case["requests"]):
            if n[b] == 0:
                continue
            pos = torch.arange(kv[b] - n[b], kv[b], device=DEV)
            new_k = _exact_heads(s["k"][row:row + n[b]], s["k_weight"] if s["norm"] else None, pos)
            where = s["block_table"][b].long()[torch.div(pos, page, rounding_mode="floor")]
            kp[where, pos % page] = new_k
            vp[where, pos % page] = s["v"][row:row + n[b]].double()
            row += n[b]
        return {"k_pages": kp, "v_pages": vp}
    hq, hkv = case["hq"], case["hkv"]
    g, row = hq // hkv, 0
    o = torch.zeros((sum(n), hq, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((sum(n), hq), dtype=torch.float64, device=DEV)
    for b in range(case["requests"]):
        if n[b] == 0:
            continue
        at = torch.arange(kv[b], device=DEV)
        where = s["block_table"][b].long()[torch.div(at, page, rounding_mode="floor")]
        hidden = at[None, :] > torch.arange(kv[b] - n[b], kv[b], device=DEV)[:, None]
        for h in range(hkv):
            keys = s["k_pages"][where, at % page, h].double()
            vals = s["v_pages"][where, at % page, h].double()
            for r in range(h * g, h * g + g):
                z = (s["q"][row:row + n[b], r].double() @ keys.T) / math.sqrt(D)
                z[hidden] = -math.inf
                total = torch.logsumexp(z, 1)
                lse[row:row + n[b], r] = total
                o[row:row + n[b], r] = torch.exp(z - total[:, None]) @ vals
        row += n[b]
    return {"o": o, "lse": lse}


def _exact_heads(x, weight, positions):
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * weight.double()
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV),
                       positions.double()[:, None] * THETA ** (-2.0 * torch.arange(64, dtype=torch.float64, device=DEV) / D))
    z = torch.complex(x[..., :64].contiguous(), x[..., 64:].contiguous()) * turn[:, None, :]
    return torch.cat([z.real, z.imag], -1)
