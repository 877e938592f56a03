"""The serving operators over a paged K/V cache held in 4 bits: what is measured of them, and their plain forms.

Three operators of one serving step, each with its head dimension fixed at 128:

  append    a batch's new keys (normalised and rotated on the way) and values, quantised into the cache as they are written;
            the whole cache is then read back as the values it stands for
  read      the cached keys and values of a batch's requests, read back into packed tensors
  attend    causal attention of a batch's new tokens (one of them, a few, or a chunk) over the cache

A head of a token is 128 codes of 4 bits (sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6, two in a byte,
the even channel in the low half) and one scale: the smallest number of six significant bits that brings the head's largest
magnitude to 6 or below, held as bf16.  Codes are the nearest ones, ties to the even code.

With `own` false `run` computes the operator in elementary torch operations (32 bits; what is quantised and the angles in 64,
from the entries of the rotary table, which is an input); with `own` true it makes the calls a user of the library makes.
`exact` evaluates the definitions in 64 bits.
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
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
LEAST, MOST = 2.0 ** -100, 1.3125 * 2.0 ** 125          # of a scale


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # One decode step of 64 young requests: 64 tokens land in 64 different pages.
        dict(name="append_step", op="append", dtype="bf16", requests=64, new=1, context=40, spread=1, hkv=8, page=16, head_major=False, norm=False),
        # Five requests' prefill chunks, 7302 new tokens in all, keys normalised as well.
        dict(name="append_chunks", op="append", dtype="bf16", requests=5, new=1638, context=500, spread=2, hkv=8, page=64, head_major=True, norm=True),
        # 32-bit heads, a page size that is no power of two.
        dict(name="append_f32", op="append", dtype="f32", requests=3, new=333, context=100, spread=3, hkv=8, page=24, head_major=True, norm=False),
        # A long request's whole stored prefix, to resume its prefill through contiguous attention or to hand it to another GPU.
        dict(name="read_long", op="read", dtype="bf16", requests=1, new=131072, context=0, spread=0, hkv=8, page=64, head_major=True),
        # The stored tokens of a batch of short requests, in 32 bits, small token-major pages.
        dict(name="read_batch", op="read", dtype="f32", requests=9, new=700, context=0, spread=8, hkv=8, page=16, head_major=False),
        # The smallest step: one request's one token.
        dict(name="attend_one", op="attend", dtype="bf16", requests=1, new=1, context=4099, spread=0, hq=32, hkv=8, page=16, head_major=False),
        # A decode step of 64 requests of mixed lengths.
        dict(name="attend_step", op="attend", dtype="bf16", requests=64, new=1, context=3000, spread=4, hq=32, hkv=8, page=64, head_major=True),
        # A decode step of three long requests (the long-context case), 64 query heads.
        dict(name="attend_long", op="attend", dtype="bf16", requests=3, new=1, context=131072, spread=5, hq=64, hkv=8, page=128, head_major=True),
        # Four tokens a request at once (a draft that is being verified), token-major pages.
        dict(name="attend_verify", op="attend", dtype="bf16", requests=16, new=4, context=9000, spread=0, hq=32, hkv=8, page=32, head_major=False),
        # One prefill chunk resumed on a long stored prefix.
        dict(name="attend_chunk", op="attend", dtype="bf16", requests=1, new=2048, context=30720, spread=0, hq=32, hkv=8, page=64, head_major=True),
        # A mixed batch: chunks of several requests beside requests with a few tokens or none, odd page size.
        dict(name="attend_mixed", op="attend", dtype="bf16", requests=24, new=300, context=2000, spread=6, hq=32, hkv=8, page=48, head_major=False),
        # The accuracy path: 32-bit queries and output.
        dict(name="attend_f32", op="attend", dtype="f32", requests=3, new=200, context=500, spread=7, hq=8, hkv=8, page=16, head_major=False),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], even in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 5, 7, 8])
    page = 8 * _between(rng, 1, 32)
    place = dict(hkv=hkv, page=page, head_major=rng.random() < 0.5)
    if op == "append":
        requests = _between(rng, 1, 64)
        return dict(op=op, dtype=dtype, requests=requests, new=_between(rng, 1, max(1, 8192 // requests)), context=_between(rng, 1, 500),
                    spread=rng.randrange(1, 1 << 20), norm=rng.random() < 0.5, **place)
    if op == "read":
        requests = _between(rng, 1, 64)
        return dict(op=op, dtype=dtype, requests=requests, new=_between(rng, 1, 65536 // requests), context=0, spread=rng.randrange(1, 1 << 20), **place)
    kind = rng.choice(["step", "step", "chunk"])
    if kind == "step":
        requests = _between(rng, 1, 64)
        new, context = _between(rng, 1, 8), _between(rng, 1, min(65536, 262144 // requests))
    else:
        requests = _between(rng, 1, 8)
        new, context = _between(rng, 9, 1500 // requests), _between(rng, 1, 16384 // requests)
    if dtype == "f32":
        context = min(context, 2048)
    return dict(op=op, dtype=dtype, requests=requests, new=new, context=context, spread=rng.randrange(0, 1 << 20), hq=hq, **place)


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


def _pool(case):
    """Pages of every request, and of the whole cache (three of them nobody's)."""
    need = [-(-k // case["page"]) for k in lengths(case)[1]]
    return need, sum(need) + 3


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    n, kv = lengths(case)
    t, hkv, held = sum(n), case["hkv"], 2 * (D // 2 + 2)           # bytes of a token's key and value of one head, as held
    if case["op"] == "append":
        pool = _pool(case)[1] * case["page"]
        return {"bytes": t * hkv * (2 * D * size + held) + pool * hkv * (held + 2 * D * size) + 4 * (2 * case["requests"] + t // case["page"]),
                "flops": t * hkv * D * 16}
    if case["op"] == "read":
        return {"bytes": t * hkv * (held + 2 * D * size) + 4 * (2 * case["requests"] + t // case["page"]), "flops": t * hkv * D * 2}
    seen = sum(k for k, m in zip(kv, n) if m > 0)
    pairs = sum(m * k - m * (m - 1) // 2 for k, m in zip(kv, n))
    return {"bytes": seen * hkv * held + 2 * t * case["hq"] * D * size + 4 * t * case["hq"] + 4 * seen // case["page"],
            "flops": 4 * D * case["hq"] * pairs}


# ------------------------------------------------------------------------------------------ the inputs
def _table(n_pos):
    """The rotary table of the library's documented layout: fine cosines and sines by channel, coarse ones by 64 positions."""
    f = torch.exp2(-torch.arange(64, dtype=torch.float64, device=DEV) / 64 * math.log2(THETA))
    b = torch.arange(64, dtype=torch.float64, device=DEV)
    a = 64.0 * torch.arange((n_pos + 63) // 64, dtype=torch.float64, device=DEV)
    fine, coarse = f[:, None] * b[None, :], a[:, None] * f[None, :]
    return torch.cat([t.reshape(-1) for t in (fine.cos(), fine.sin(), coarse.cos(), coarse.sin())]).float()


def _heads(gen, shape):
    """Heads whose magnitudes differ from token to token."""
    x = torch.randn((*shape, D), generator=gen, device=DEV)
    return x.mul_(torch.exp(0.3 * torch.randn((*shape, 1), generator=gen, device=DEV)))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    s = dict(case)
    n, kv = lengths(case)
    t, b, page, hkv = sum(n), case["requests"], case["page"], case["hkv"]
    need, total = _pool(case)
    order = torch.randperm(total, generator=gen, device=DEV).int()
    table = torch.zeros((b, max(max(need), 1)), dtype=torch.int32, device=DEV)
    rows = torch.arange(table.shape[1], device=DEV)[None, :]
    need_t = torch.tensor(need, device=DEV)[:, None]
    first = torch.tensor([sum(need[:i]) for i in range(b)], device=DEV)[:, None]
    s["block_table"] = torch.where(rows < need_t, order[(first + rows).clamp(max=total - 1)], table)
    # The cache as earlier steps have left it.
    shape = (total, hkv, page) if case["head_major"] else (total, page, hkv)
    for which in ("k", "v"):
        codes = torch.empty((*shape, D // 2), dtype=torch.uint8, device=DEV)
        scales = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
        for i in range(0, total, max(1, (1 << 26) // (page * hkv * D))):          # (a piece of the pool at a time)
            part = slice(i, i + max(1, (1 << 26) // (page * hkv * D)))
            codes[part], scales[part] = _quantise(_heads(gen, scales[part].shape))
        s[which + "_pages"], s[which + "_scales"] = (codes.transpose(1, 2), scales.transpose(1, 2)) if case["head_major"] else (codes, scales)
    s["cu_q"] = torch.tensor([sum(n[:i]) for i in range(b + 1)], dtype=torch.int32, device=DEV)
    s["kv_lens"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    s["tokens"], s["most_new"], s["most_kv"] = t, max(n), max(kv)
    if case["op"] == "append":
        s["k"], s["v"] = _heads(gen, (t, hkv)).to(dtype), _heads(gen, (t, hkv)).to(dtype)
        s["k_weight"] = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dtype)
        s["n_pos"] = max(max(kv), 1)
        s["table"] = _table(s["n_pos"])
        # The whole cache as one request, to read it back.
        s["all_pages"] = torch.arange(total, dtype=torch.int32, device=DEV)[None]
        s["all_cu"] = torch.tensor([0, total * page], dtype=torch.int32, device=DEV)
        s["all_len"] = torch.tensor([total * page], dtype=torch.int32, device=DEV)
        s["all_tokens"] = total * page
    elif case["op"] == "attend":
        s["q"] = torch.randn((t, case["hq"], D), generator=gen, device=DEV).to(dtype)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    if s["op"] == "append":
        return _own_append(s) if own else _plain_append(s)
    if s["op"] == "read":
        return _own_read(s) if own else _plain_read(s)
    return _own_attend(s) if own else _plain_attend(s)


def _own_append(s):
    from paper_2409_15104_b200 import binding
    cache = s["k_pages"], s["k_scales"], s["v_pages"], s["v_scales"]
    binding.pec_kv_append_q4(s["k"], s["v"], *cache, s["block_table"], s["cu_q"], s["kv_lens"], norm=s["norm"],
                             k_weight=s["k_weight"] if s["norm"] else None, eps=EPS, tables=(s["table"], s["n_pos"]))
    k, v = binding.pec_kv_read_q4(*cache, s["all_pages"], s["all_cu"], s["all_len"], s["all_tokens"], dtype=TYPES[s["dtype"]])
    return {"k": k, "v": v}


def _own_read(s):
    from paper_2409_15104_b200 import binding
    k, v = binding.pec_kv_read_q4(s["k_pages"], s["k_scales"], s["v_pages"], s["v_scales"], s["block_table"], s["cu_q"], s["kv_lens"],
                                  s["tokens"], dtype=TYPES[s["dtype"]])
    return {"k": k, "v": v}


def _own_attend(s):
    from paper_2409_15104_b200 import binding
    o, lse = binding.pec_paged_attn_q4(s["q"], s["k_pages"], s["k_scales"], s["v_pages"], s["v_scales"], s["block_table"], s["cu_q"],
                                       s["kv_lens"], max_q_len=s["most_new"])
    return {"o": o, "lse": lse}


def _quantise(x):
    """(bytes, scales) of heads [..., D], in x's own precision."""
    most = x.abs().amax(-1).double()
    sixth = most / torch.full_like(most, 6)                    # (a division: by a number it would be a product with 1 / 6)
    low = (1 << 47) - 1                                        # of the 52 bits after the first, five stay
    scale = ((sixth.view(torch.int64) + low) & ~low).view(torch.float64).clamp(LEAST, MOST).to(x.dtype)
    t = x.abs() / scale[..., None]
    code = (t > 0.25).to(torch.uint8)
    for border, up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += t >= border if up else t > border
    code |= (x < 0).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4, scale.to(torch.bfloat16)


def _values(pages, scales):
    """Heads [..., D] in 32 bits."""
    code = torch.stack([pages & 15, pages >> 4], -1).flatten(-2)
    magnitude = torch.tensor(MAGNITUDES, device=pages.device)[(code & 7).int()]
    return torch.where(code > 7, -magnitude, magnitude).mul_(scales.float()[..., None])


def _turn(x, table, n_pos, positions):
    """The rotate-half pairing in 64 bits, cosines and sines from the table's entries by the addition theorem."""
    t = table.double()
    a, b, na = positions // 64, positions % 64, (n_pos + 63) // 64
    fine = t[:8192].view(2, 64, 64)
    coarse = t[8192:8192 + 128 * na].view(2, na, 64)
    fc, fs, cc, cs = fine[0].T[b], fine[1].T[b], coarse[0][a], coarse[1][a]
    c, s = (cc * fc - cs * fs)[:, None], (cs * fc + cc * fs)[:, None]
    lo, hi = x[..., :64], x[..., 64:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def _places(s):
    """Request, position, page and slot of every new token."""
    cu = s["cu_q"].long()
    row = torch.arange(s["tokens"], device=cu.device)
    b = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    pos = s["kv_lens"].long()[b] - cu[b + 1] + row
    return pos, s["block_table"][b, pos // s["page"]].long(), pos % s["page"]


def _plain_append(s):
    pos, page, slot = _places(s)
    k = s["k"].double()
    if s["norm"]:
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * s["k_weight"].double()
    s["k_pages"][page, slot], s["k_scales"][page, slot] = _quantise(_turn(k, s["table"], s["n_pos"], pos))
    s["v_pages"][page, slot], s["v_scales"][page, slot] = _quantise(s["v"].double())
    k, v = _values(s["k_pages"], s["k_scales"]), _values(s["v_pages"], s["v_scales"])
    dtype = s["k"].dtype
    return {"k": k.flatten(0, 1).to(dtype), "v": v.flatten(0, 1).to(dtype)}


def _plain_read(s):
    _, page, slot = _places(s)
    dtype = TYPES[s["dtype"]]
    return {"k": _values(s["k_pages"][page, slot], s["k_scales"][page, slot]).to(dtype),
            "v": _values(s["v_pages"][page, slot], s["v_scales"][page, slot]).to(dtype)}


def _plain_attend(s):
    q, cu, kv_len = s["q"], s["cu_q"].long(), s["kv_lens"].long()
    dev, (t, hq, _), hkv = q.device, q.shape, s["hkv"]
    n = cu[1:] - cu[:-1]
    i, j = torch.arange(s["most_new"], device=dev), torch.arange(s["most_kv"], device=dev)
    rows = (cu[:-1, None] + i).clamp(max=t - 1)
    real = i < n[:, None]                                                       # [B, n]
    pages = s["block_table"].long()
    held = (j < kv_len[:, None])[:, :, None, None]

    def gathered(which):                                                        # [B, kv, Hkv, D], zeros past a request's end
        codes, scales = (s[which + end][pages].flatten(1, 2)[:, :s["most_kv"]] for end in ("_pages", "_scales"))
        return _values(codes, scales).masked_fill_(~held, 0.0)

    x = q[rows].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)      # [B, Hkv, g n, D]
    score = (x @ gathered("k").permute(0, 2, 3, 1)).unflatten(2, (hq // hkv, s["most_new"])) * (1 / math.sqrt(D))
    pos = kv_len[:, None] - n[:, None] + i
    score.masked_fill_(~(j <= pos[:, :, None])[:, None, None], float("-inf"))
    most = score.amax(-1, keepdim=True)
    score.sub_(most).exp_()
    total = score.sum(-1, keepdim=True)
    o = (score.flatten(2, 3) @ gathered("v").transpose(1, 2)).unflatten(2, (hq // hkv, s["most_new"])) / total
    lse = (most + total.log()).squeeze(-1)
    o, lse = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[real], lse.permute(0, 3, 1, 2).flatten(2, 3)[real]
    return {"o": o.to(q.dtype), "lse": lse}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    n, kv = lengths(case)
    page = case["page"]
    if case["op"] == "append":
        k, v = _exact_held(s["k_pages"], s["k_scales"]), _exact_held(s["v_pages"], s["v_scales"])
        row = 0
        for b in range(case["requests"]):
            new, new_v = s["k"][row:row + n[b]].double(), s["v"][row:row + n[b]].double()
            row += n[b]
            if n[b] == 0:
                continue
            pos = torch.arange(kv[b] - n[b], kv[b], device=DEV)
            if case["norm"]:
                new = new / torch.sqrt((new * new).sum(-1, keepdim=True) / D + EPS) * s["k_weight"].double()
            turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV),
                               pos.double()[:, None] * THETA ** (-2.0 * torch.arange(64, dtype=torch.float64, device=DEV) / D))
            z = torch.complex(new[..., :64].contiguous(), new[..., 64:].contiguous()) * turn[:, None, :]
            where = s["block_table"][b].long()[torch.div(pos, page, rounding_mode="floor")]
            k[where, pos % page] = _exact_rounded(torch.cat([z.real, z.imag], -1))
            v[where, pos % page] = _exact_rounded(new_v)
        return {"k": k.flatten(0, 1), "v": v.flatten(0, 1)}

    def held(b, which, h=slice(None)):
        at = torch.arange(kv[b] - n[b] if case["op"] == "read" else 0, kv[b], device=DEV)
        where = s["block_table"][b].long()[torch.div(at, page, rounding_mode="floor")]
        return _exact_held(s[which + "_pages"][where, at % page, h], s[which + "_scales"][where, at % page, h])

    if case["op"] == "read":
        return {w: torch.cat([held(b, w) for b in range(case["requests"])]) for w in "kv"}
    hq, hkv = case["hq"], case["hkv"]
    g, row = hq // hkv, 0
    o = torch.zeros((sum(n), hq, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((sum(n), hq), dtype=torch.float64, device=DEV)
    for b in range(case["requests"]):
        if n[b] == 0:
            continue
        hidden = torch.arange(kv[b], device=DEV)[None, :] > torch.arange(kv[b] - n[b], kv[b], device=DEV)[:, None]
        for h in range(hkv):
            keys, vals = held(b, "k", h), held(b, "v", h)
            for r in range(h * g, h * g + g):
                z = (s["q"][row:row + n[b], r].double() @ keys.T) / math.sqrt(D)
                z[hidden] = -math.inf
                total = torch.logsumexp(z, 1)
                lse[row:row + n[b], r] = total
                o[row:row + n[b], r] = torch.exp(z - total[:, None]) @ vals
        row += n[b]
    return {"o": o, "lse": lse}


def _exact_held(codes, scales):
    """What codes and scales stand for, written out from the bits: (1 + m / 2) 2^(e - 1), or m / 2 where e is 0."""
    c = torch.stack([codes % 16, torch.div(codes, 16, rounding_mode="floor")], -1).flatten(-2).double()
    sign, rest = torch.div(c, 8, rounding_mode="floor"), c % 8
    e, m = torch.div(rest, 2, rounding_mode="floor"), rest % 2
    return (1 - 2 * sign) * torch.where(e > 0, (1 + m / 2) * 2.0 ** (e - 1), m / 2) * scales.double()[..., None]


def _exact_rounded(x):
    """The nearest representable head, from the distances to all eight magnitudes (the even code of two that are as near)."""
    most = x.abs().amax(-1)
    m, e = torch.frexp(most / torch.full_like(most, 6))
    two_to_e = ((e.long() + 1023) << 52).view(torch.float64)   # (the power function of the GPU is not exact)
    scale = (torch.ceil(m * 64) * two_to_e).div_(torch.full_like(most, 64)).clamp(LEAST, MOST)[..., None]
    best, off = torch.zeros_like(x), (x.abs() / scale).clone()
    for code in (2, 4, 6, 1, 3, 5, 7):
        d = (x.abs() / scale - MAGNITUDES[code]).abs()
        best, off = torch.where(d < off, MAGNITUDES[code], best), torch.minimum(d, off)
    return torch.sign(x) * best * scale
