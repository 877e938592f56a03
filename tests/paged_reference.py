"""The paged serving operators in 64 bits, written out request by request, with error bounds that follow from the arithmetic."""
import numpy as np
import torch

D = 128
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # largest relative rounding error of a value


def rope(x, positions, theta):
    """x [T, H, 128] fp64, positions [T]: channel i < 64 turned with channel i + 64."""
    f = theta ** (-2.0 * np.arange(64) / D)
    a = np.asarray(positions, dtype=np.float64)[:, None, None] * f
    lo, hi = x[..., :64], x[..., 64:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def norm_rope(x, weight, eps, positions, theta, norm=True, turn=True):
    """(value, size): size is what a rounding error of the step's fp32 arithmetic scales with - the pair's magnitudes."""
    x = x.detach().double().cpu().numpy()
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * weight.double().cpu().numpy()
    size = np.abs(x) + np.abs(np.concatenate([x[..., 64:], x[..., :64]], -1))
    return (rope(x, positions, theta) if turn else x), size


def norm_rope_bound(want, size, dtype):
    """fp32 arithmetic: the sum of squares is a tree of 4 + 5 additions over rounded squares, halved by the root; root,
    division and two products one rounding each; cosines and sines within 3e-7: below 1e-6 of the pair's magnitudes in all.
    Then one rounding to the output type."""
    return HALF[dtype] * np.abs(want) + 1e-6 * size


def attend(q, k_pages, v_pages, block_table, cu_q, kv_lens, causal=True, scale=None):
    """Values and bounds: o, lse, and per element A = sum_j p_j |v_j| and per row B = max_j scale sum_c |q_c k_jc|.
    q [T, Hq, D], pages [num, page, Hkv, D] (any strides), host lists cu_q, kv_lens.  Padding rows are NaN."""
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    q = q.detach().double().cpu()
    T, Hq, _ = q.shape
    page, Hkv = k_pages.shape[1], k_pages.shape[2]
    o = np.full((T, Hq, D), np.nan)
    A = np.zeros((T, Hq, D))
    lse = np.full((T, Hq), np.nan)
    B = np.zeros((T, Hq))
    for b in range(len(kv_lens)):
        s, e, kv = cu_q[b], cu_q[b + 1], kv_lens[b]
        n = e - s
        if n == 0:
            continue
        need = -(-kv // page)
        ids = block_table[b, :need].long().to(k_pages.device)
        keys = k_pages[ids].double().cpu().reshape(need * page, Hkv, D)[:kv]
        vals = v_pages[ids].double().cpu().reshape(need * page, Hkv, D)[:kv]
        for h in range(Hq):
            kh, vh, qh = keys[:, h // (Hq // Hkv)], vals[:, h // (Hq // Hkv)], q[s:e, h]
            z = scale * (qh @ kh.T)
            seen = torch.ones((n, kv), dtype=torch.bool)
            if causal:
                seen = torch.arange(kv)[None, :] <= (kv - n + torch.arange(n))[:, None]
            z = z.masked_fill(~seen, -float("inf"))
            some = seen.any(1)
            m = torch.where(some, z.max(1).values if kv else torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64))
            p = torch.exp(z - m[:, None])
            l = p.sum(1)
            inv = torch.where(some, 1 / l, torch.zeros_like(l))
            o[s:e, h] = ((p @ vh) * inv[:, None]).numpy()
            A[s:e, h] = ((p @ vh.abs()) * inv[:, None]).numpy()
            lse[s:e, h] = torch.where(some, m + l.log(), torch.full_like(l, -float("inf"))).numpy()
            if kv:
                B[s:e, h] = (scale * (qh.abs() @ kh.abs().T)).masked_fill(~seen, 0.0).max(1).values.numpy()
    return o, lse, A, B


def check_attend(got_o, got_l, want, dtype, what="", p_error=None):
    """Bounds: a score is a sum of 128 products in fp32, off by at most 128 * 2^-23 * B (each addition to a full ulp, which
    covers truncating adders), and so is the scaling's rounding; e^x turns that into a relative error of p, twice (p and the
    sum).  2^x is approximated to 2^-21.  bf16 rounds p by 2^-8 of itself; fp32 sums of up to 2^18 terms in pieces and
    merges stay below 2e-6 of A.  The output is rounded once to its type.  p_error: another relative error of p than a bf16
    rounding's."""
    o, lse, A, B = want
    got_o, got_l = got_o.detach(), got_l.detach()
    out_t = got_o.dtype
    go, gl = got_o.double().cpu().numpy(), got_l.double().cpu().numpy()
    real = ~np.isnan(lse)
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(gl)[real], empty[real]), f"{what}: which rows are empty differs"
    assert (go[empty] == 0).all(), f"{what}: empty rows must be zero"
    delta = 130 * 2.0 ** -23 * B
    full = real & ~empty
    assert np.isfinite(go[real]).all() and np.isfinite(gl[full]).all(), f"{what}: not finite"
    if p_error is None:
        p_error = HALF[torch.bfloat16] if dtype == torch.bfloat16 else 0.0
    bound = (2 * delta[..., None] + 2.0 ** -20 + 2e-6 + p_error) * A + HALF[out_t] * np.abs(o) + 1e-30
    off = np.abs(go - o)[full] / bound[full]
    bl = (delta + 2.0 ** -20 + 2e-6 + 2.0 ** -23 * np.abs(np.where(full, lse, 0.0)))[full]
    off_l = np.abs(gl[full] - lse[full]) / bl
    if off.size:
        print(f"[parity] {what}: o at {off.max():.3f} of its bound, lse at {off_l.max():.3f}")
        assert off.max() <= 1 and off_l.max() <= 1, (what, off.max(), off_l.max())


def make_cache(seed, kv_lens, page, hkv, dtype, device, head_major=False, spare=2, poison=True, wild=True):
    """A paged cache whose requests' keys and values are N(0, 1), pages in random order; slots past a request's end and spare
    pages hold NaN (poison), table entries a request does not reach are far out of range (wild)."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-k // page) for k in kv_lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g)
    fill = float("nan") if poison else 0.0
    pages = [torch.full((total, page, hkv, D), fill, dtype=dtype) for _ in range(2)]
    width = max(max(need), 1) + 1
    table = torch.full((len(kv_lens), width), 2 ** 30 if wild else 0, dtype=torch.int32)
    at = 0
    for b, kv in enumerate(kv_lens):
        ids = order[at:at + need[b]]
        at += need[b]
        table[b, :need[b]] = ids.int()
        for p in pages:
            rows = torch.full((need[b] * page, hkv, D), fill, dtype=dtype)
            rows[:kv] = torch.randn((kv, hkv, D), generator=g).to(dtype)
            p[ids] = rows.view(need[b], page, hkv, D)
    if head_major:
        pages = [p.transpose(1, 2).contiguous().to(device).transpose(1, 2) for p in pages]
    else:
        pages = [p.to(device) for p in pages]
    return pages[0], pages[1], table.to(device)


def offsets(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out
