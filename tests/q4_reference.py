"""The 4-bit cache in 64 bits: what codes and scales stand for, what a head is quantised to, and caches to test with."""
import numpy as np
import torch

import paged_reference as ref

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LEAST, MOST = 2.0 ** -100, 1.3125 * 2.0 ** 125


def values(pages, scales):
    """[.., 64] bytes and [..] bf16 -> [.., 128] fp64."""
    b = pages.view(torch.uint8).cpu().numpy()
    code = np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], 128)
    v = np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    with np.errstate(invalid="ignore"):
        return v * scales.double().cpu().numpy()[..., None]


def quantise(x):
    """What is held of heads [.., 128] in fp64: (values, scales); heads that are not finite become NaN."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x).all(-1)
    y = np.where(fine[..., None], x, 0.0)
    m, e = np.frexp(np.abs(y).max(-1) / 6)
    s = np.clip(np.ldexp(np.ceil(m * 64) / 64, e), LEAST, MOST)[..., None]
    t = np.abs(y) / s
    d = np.abs(t[..., None] - MAGNITUDES)
    d[..., 1::2] *= 1 + 1e-13                                   # of two codes as near, the even one
    v = np.copysign(MAGNITUDES[d.argmin(-1)], y) * s
    return np.where(fine[..., None], v, np.nan), np.where(fine, s[..., 0], np.nan)


def pack(x):
    """fp64 heads -> (bytes, bf16 scales) tensors, for filling caches."""
    v, s = quantise(x)
    code = np.abs(v / s[..., None])[..., None] == MAGNITUDES
    code = code.argmax(-1).astype(np.uint8) | ((v < 0).astype(np.uint8) << 3)
    return torch.from_numpy(code[..., 0::2] | code[..., 1::2] << 4), torch.from_numpy(s).to(torch.bfloat16)


def make_cache(seed, kv_lens, page, hkv, device, head_major=False, spare=2, wild=True, size=1.0):
    """As paged_reference.make_cache, held in 4 bits: (k_pages, k_scales, v_pages, v_scales, block_table).  Slots past a request's end
    and spare pages hold any codes with scales that are not finite."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-k // page) for k in kv_lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g)
    width = max(max(need), 1) + 1
    table = torch.full((len(kv_lens), width), 2 ** 30 if wild else 0, dtype=torch.int32)
    out = []
    for which in range(2):
        codes = torch.randint(0, 256, (total, page, hkv, 64), generator=g, dtype=torch.uint8)
        scales = torch.full((total, page, hkv), float("nan"), dtype=torch.bfloat16)
        scales[:, ::2] = float("inf")
        at = 0
        for b, kv in enumerate(kv_lens):
            ids = order[at:at + need[b]]
            at += need[b]
            table[b, :need[b]] = ids.int()
            c, s = codes[ids].view(-1, hkv, 64), scales[ids].view(-1, hkv)
            x = torch.randn((kv, hkv, 128), generator=g) * torch.exp(0.5 * torch.randn((kv, hkv, 1), generator=g)) * size
            if kv:
                c[:kv], s[:kv] = pack(x.double().numpy())
            codes[ids], scales[ids] = c.view(need[b], page, hkv, 64), s.view(need[b], page, hkv)
        for t in (codes, scales):
            out.append(t.transpose(1, 2).contiguous().to(device).transpose(1, 2) if head_major else t.to(device))
    return (*out, table.to(device))


def attend(q, cache, cu_q, kv_lens, causal=True, scale=None):
    """paged_reference.attend over what the cache holds (bf16 numbers all of them, so fp32 tensors hold them too)."""
    kp, ks, vp, vs, table = cache
    k, v = (torch.from_numpy(values(p, s)).float() for p, s in ((kp, ks), (vp, vs)))
    return ref.attend(q, k, v, table.cpu(), cu_q, kv_lens, causal, scale)
