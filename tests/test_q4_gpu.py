"""The calls over a paged cache held in 4 bits on the GPU against 64-bit references: append, read back, attention, and a serving step
made of them."""
import ctypes

import numpy as np
import pytest
import torch

import paged_reference as ref
import q4_reference as q4
from paper_2409_15104_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 500000.0
BF16, F32 = torch.bfloat16, torch.float32


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------ append
def angles(tables, positions):
    """Cosines and sines [T, 64] in fp64 from the table's fp32 entries."""
    t, n_pos = tables[0].double().cpu().numpy(), tables[1]
    na = (n_pos + 63) // 64
    F, G = t[:4096].reshape(64, 64), t[4096:8192].reshape(64, 64)
    C, S = t[8192:8192 + 64 * na].reshape(na, 64), t[8192 + 64 * na:8192 + 128 * na].reshape(na, 64)
    p = np.asarray(positions)
    a, b = p // 64, p % 64
    return C[a] * F.T[b] - S[a] * G.T[b], S[a] * F.T[b] + C[a] * G.T[b]


def check_held(pages, scales, x, weight, positions, norm, tables):
    """What is held of the heads x [T, H, 128]: exactly the definition's numbers.  (Its arithmetic and the library's both err by
    some 1e-15, so a head that comes out differently with probability 1e-12 would fail; the inputs here do not.)"""
    z = x.detach().double().cpu().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        if norm:
            z = z / np.sqrt((z * z).mean(-1, keepdims=True) + float(np.float32(1e-6)))
            if weight is not None:
                z = z * weight.double().cpu().numpy()
        if tables is not None:
            c, s = (v[:, None] for v in angles(tables, positions))
            lo, hi = z[..., :64], z[..., 64:]
            z = np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)
    want, want_s = q4.quantise(z)
    got, got_s = q4.values(pages, scales), scales.double().cpu().numpy()
    assert np.array_equal(got_s, want_s, equal_nan=True), np.argwhere(got_s != want_s)[:5]
    assert np.array_equal(got, want, equal_nan=True), (np.argwhere(got != want)[:5], np.abs(got - want).max())


CACHES = [
    ([1], [1], 16, 1, False), ([1] * 40, list(range(1, 41)), 16, 8, False), ([5, 0, 1, 33, 0], [5, 9, 64, 100, 0], 24, 3, True),
    ([200, 3], [200, 130], 128, 2, False), ([1] * 33 + [70], [17 * (i % 9) + 1 for i in range(33)] + [1000], 8, 4, True),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,kv,page,hkv,head_major", CACHES)
@pytest.mark.parametrize("norm,turn", [(False, True), (True, True), (False, False), (True, False)])
def test_append(pec, dtype, n, kv, page, hkv, head_major, norm, turn):
    kp, ks, vp, vs, table = q4.make_cache(11, kv, page, hkv, DEV, head_major)
    before = [t.clone() for t in (kp, ks, vp, vs)]
    cu = ref.offsets(n)
    T = cu[-1] + 3                                                # three rows of padding
    g = torch.Generator().manual_seed(7)
    kvs = (torch.randn((T, 2 * hkv, 128), generator=g) * torch.exp(2 * torch.randn((T, 2 * hkv, 1), generator=g))).to(dtype).to(DEV)
    k, v = kvs[:, :hkv], kvs[:, hkv:]
    w = (1 + 0.2 * torch.randn(128, generator=g)).to(dtype).to(DEV) if norm else None
    tables = pec.pec_rope_table(THETA, 2000, DEV) if turn else None
    pec.pec_kv_append_q4(k, v, kp, ks, vp, vs, table, dev(cu), dev(kv), norm=norm, k_weight=w, tables=tables)
    pec.check_status()
    places = [(int(table[b, (kv[b] - n[b] + i) // page]), (kv[b] - n[b] + i) % page, kv[b] - n[b] + i, cu[b] + i) for b in range(len(n)) for i in range(n[b])]
    pg, slot, pos, row = (list(x) for x in zip(*places))
    check_held(kp[pg, slot], ks[pg, slot], k[row], w, pos, norm, tables)
    check_held(vp[pg, slot], vs[pg, slot], v[row], None, pos, False, None)
    other = torch.ones(kp.shape[:2], dtype=torch.bool, device=DEV)
    other[pg, slot] = False
    for now, was in zip((kp, ks, vp, vs), before):
        assert torch.equal(now[other].view(torch.uint8), was[other].view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_decides_borders_exactly(pec, dtype):
    """Channels on the borders between two codes and next to them, in units of scales of all six-bit mantissas and many exponents."""
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows = []
    for m in range(32, 64):
        for e in (-90, -20, 0, 3, 60):
            s = m * 2.0 ** e / 64
            x = np.zeros(128)
            x[0] = 6 * s
            x[1:8], x[8:15] = borders * s, -borders * s
            near = torch.from_numpy(np.concatenate([borders * s, s * np.arange(1, 11) / 2])).to(dtype)
            bits = near.view(torch.int16 if dtype == BF16 else torch.int32)
            x[20:37] = (bits + 1).view(dtype).double().numpy()
            x[40:57] = (bits - 1).view(dtype).double().numpy()
            rows.append(x)
    x = torch.from_numpy(np.stack(rows)).to(dtype)[:, None].to(DEV)
    T = x.shape[0]
    kp, ks, vp, vs, table = q4.make_cache(1, [T], 16, 1, DEV)
    pec.pec_kv_append_q4(x, -x, kp, ks, vp, vs, table, dev([0, T]), dev([T]))
    pec.check_status()
    ids = table[0, :-(-T // 16)].long()
    flat = lambda t: t[ids].flatten(0, 1)[:T]
    check_held(flat(kp), flat(ks), x, None, None, False, None)
    check_held(flat(vp), flat(vs), -x, None, None, False, None)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norm,turn", [(False, False), (True, True)])
def test_append_extreme_values(pec, dtype, norm, turn):
    """Zero heads, huge and tiny ones; a head that is not finite becomes NaN and spoils no other."""
    x = torch.randn((10, 2, 128), generator=torch.Generator().manual_seed(4)).to(DEV)
    x[0] = 0
    x[1] *= 2.0 ** 125 / x[1].abs().max()
    x[2] = 0
    x[2, :, 5] = torch.finfo(dtype).max
    x[3] *= 1e-36
    x[4] *= 1e-30
    x[5, 0, 5] = float("nan")
    x[6, 1, 77] = float("inf")
    x[7, 0] = float("-inf")
    x[8, 0, :] = 0
    x[8, 0, 127] = -1e-44
    x = x.to(dtype)
    kp, ks, vp, vs, table = q4.make_cache(1, [10], 8, 2, DEV)
    tables = pec.pec_rope_table(THETA, 16, DEV) if turn else None
    pec.pec_kv_append_q4(x, x, kp, ks, vp, vs, table, dev([0, 10]), dev([10]), norm=norm, tables=tables)
    pec.check_status()
    ids = table[0, :2].long()
    flat = lambda t: t[ids].flatten(0, 1)[:10]
    check_held(flat(vp), flat(vs), x, None, None, False, None)
    check_held(flat(kp), flat(ks), x, None, list(range(10)), norm, tables)
    assert (flat(ks)[0].float() == 2.0 ** -100).all() and not torch.isfinite(flat(ks)[5, 0])


def test_append_reports_what_is_out_of_range_and_stores_the_rest(pec):
    page, hkv = 16, 2
    kp, ks, vp, vs, table = q4.make_cache(12, [40, 40, 40, 40], page, hkv, DEV)
    table[1, 2] = kp.shape[0]                                     # one page past the cache
    table[2, 2] = -1
    before = [t.clone() for t in (kp, ks, vp, vs)]
    k, v = torch.randn((4, hkv, 128), device=DEV), torch.randn((4, hkv, 128), device=DEV)
    pec.pec_kv_append_q4(k, v, kp, ks, vp, vs, table, dev([0, 1, 2, 3, 4]), dev([40, 40, 40, 4000]))   # the last one is past its row of the table
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
    at = (int(table[0, 2]), 39 % page)
    check_held(kp[at][None], ks[at][None], k[:1], None, [39], False, None)
    other = torch.ones(kp.shape[:2], dtype=torch.bool, device=DEV)
    other[at] = False
    for now, was in zip((kp, ks, vp, vs), before):
        assert torch.equal(now[other].view(torch.uint8), was[other].view(torch.uint8))
    for cu, lens in (([0, 3, 1, 4, 4], [40] * 4), ([0, 1, 2, 3, 9], [40] * 4), ([0, 4, 4, 4, 4], [2, 1, 1, 1])):
        pec.pec_kv_append_q4(k, v, kp, ks, vp, vs, table.clamp(0, kp.shape[0] - 1), dev(cu), dev(lens))
        with pytest.raises(binding.PecError):
            pec.check_status()


# ------------------------------------------------------------------------------------------ read back
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,kv,page,hkv,head_major", CACHES + [([300, 7], [300, 900], 48, 17, True)])
def test_read(pec, dtype, n, kv, page, hkv, head_major):
    kp, ks, vp, vs, table = q4.make_cache(21, kv, page, hkv, DEV, head_major)
    cu = ref.offsets(n)
    T = cu[-1] + 2
    out = torch.full((T, 2 * hkv + 1, 128), 7.0, dtype=dtype, device=DEV)
    k, v = pec.pec_kv_read_q4(kp, ks, vp, vs, table, dev(cu), dev(kv), T, dtype=dtype, k_out=out[:, :hkv], v_out=out[:, hkv:2 * hkv])
    pec.check_status()
    for got, pages, scales in ((k, kp, ks), (v, vp, vs)):
        want = q4.values(pages, scales)
        for b in range(len(n)):
            pos = np.arange(kv[b] - n[b], kv[b])
            ids = table[b].cpu().numpy()[pos // page]
            assert np.array_equal(got[cu[b]:cu[b + 1]].double().cpu().numpy(), want[ids, pos % page])
    assert (out[cu[-1]:] == 7.0).all() and (out[:, 2 * hkv] == 7.0).all()
    # new tensors, whole requests
    whole = ref.offsets(kv)
    k, v = pec.pec_kv_read_q4(kp, ks, vp, vs, table, dev(whole), dev(kv), whole[-1], dtype=dtype)
    assert k.shape == v.shape == (whole[-1], hkv, 128) and k.dtype == dtype
    rows = [whole[b] + kv[b] - n[b] + i for b in range(len(n)) for i in range(n[b])]
    assert torch.equal(k[rows], out[:cu[-1], :hkv]) and torch.equal(v[rows], out[:cu[-1], hkv:2 * hkv])


def test_read_reports_what_is_out_of_range_and_leaves_its_rows(pec):
    kp, ks, vp, vs, table = q4.make_cache(12, [40, 40, 40], 16, 2, DEV)
    table[1, 2] = kp.shape[0]
    out = torch.full((2, 6, 2, 128), 7.0, device=DEV)
    pec.pec_kv_read_q4(kp, ks, vp, vs, table, dev([0, 2, 4, 6]), dev([40, 40, 4000]), 6, dtype=F32, k_out=out[0], v_out=out[1])
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
    assert (out[:, 2:] == 7.0).all() and not (out[:, :2] == 7.0).all(-1).any()


def test_heads_that_are_not_finite_are_read_as_nan(pec):
    kp, ks, vp, vs, table = q4.make_cache(12, [9], 8, 2, DEV)
    x = torch.randn((9, 2, 128), device=DEV)
    x[4, 1, 3] = float("inf")
    pec.pec_kv_append_q4(x, x, kp, ks, vp, vs, table, dev([0, 9]), dev([9]))
    for dtype in (BF16, F32):
        k, v = pec.pec_kv_read_q4(kp, ks, vp, vs, table, dev([0, 9]), dev([9]), 9, dtype=dtype)
        for t in (k, v):
            assert torch.isnan(t[4, 1]).all() and torch.isnan(t).sum() == 128
    pec.check_status()


# ------------------------------------------------------------------------------------------ attention
def check(o, lse, want, dtype, cache, kv, most_rows, what):
    """paged_reference.check_attend with the rounding of the probabilities here.  fp32 q: none.  bf16 q: fp16 parts, off by half a step,
    2^-11 of themselves, and in its subnormals (steps of 2^-24) by 2^-25.
    At most 16 packed rows: p sv 2^10 / v_ref, v_ref a power of two of at most twice the largest scale s, the row's largest p 1 or more:
    2^-25 is 2^-35 v_ref <= 2^-34 s for each key, times a code of at most 6.
    More: p times 2^10 or more, so 2^-35 of the largest p, times 6 s, for each key; and values in units in which s is 2^9 or more, so
    2^-34 s once (the p sum to 1): 2^-35 * 6 s * keys + 2^-34 s <= 2^-34 * 6 s * keys, the same."""
    o64, lse64, A, B = want
    error = None
    if dtype == BF16:
        error = 2.0 ** -11
        scales = cache[3].float()
        A = A + max(kv) * 2.0 ** -34 * 6 * float(scales[torch.isfinite(scales)].max() if torch.isfinite(scales).any() else 0.0) / error
    ref.check_attend(o, lse, (o64, lse64, A, B), dtype, f"{what}, {most_rows} rows", error)


def attend(pec, seed, n, kv, hq, hkv, page, dtype, *, head_major=False, causal=True, out_dtype=None, pad=0, fused=False, known=True,
           scale=0.0, size=1.0, what=""):
    cache = q4.make_cache(seed, kv, page, hkv, DEV, head_major, size=size)
    cu = ref.offsets(n)
    T = cu[-1] + pad
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((T, hq + (2 if fused else 0), 128), generator=g).to(dtype).to(DEV)[:, :hq]
    out_dtype = dtype if out_dtype is None else out_dtype
    o = torch.full((T, hq, 128), 7.0, dtype=out_dtype, device=DEV)
    lse = torch.full((T, hq), 7.0, device=DEV)
    call = lambda: pec.pec_paged_attn_q4(q, *cache, dev(cu), dev(kv), max_q_len=max(n) if known else 0, causal=causal, softmax_scale=scale, o=o, lse=lse)
    call()
    pec.check_status()
    want = q4.attend(q, cache, cu, kv, causal, scale or None)
    if pad:
        assert (o[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all(), "padding rows were written"
    check(o, lse, want, dtype, cache, kv, max(n) * (hq // hkv), what)
    first = (o.clone(), lse.clone())
    call()
    assert torch.equal(first[0], o) and torch.equal(first[1], lse), "the same call gave other bits"
    return o, lse


SHAPES = [
    # n, kv, hq, hkv, page
    ([1], [1], 1, 1, 16), ([1], [1], 8, 1, 8), ([1], [128], 4, 4, 16), ([1], [129], 8, 2, 16), ([1], [127], 16, 2, 128),
    ([1], [0], 4, 2, 16),                                          # a token before its request's first position: sees nothing
    ([3], [1], 4, 2, 16), ([5, 2], [0, 1], 8, 8, 16),              # leading rows that see nothing
    ([1] * 7, [1, 2, 63, 64, 65, 300, 1000], 32, 8, 16), ([1] * 64, [37 * (i % 11) + 1 for i in range(64)], 8, 2, 48),
    ([1] * 70, [(i * i) % 700 + 1 for i in range(70)], 4, 1, 64), ([1, 0, 1, 0, 0], [500, 30, 0, 0, 700], 8, 4, 24),
    ([4, 1, 2, 3], [400, 129, 128, 131], 14, 2, 16), ([18], [200], 7, 1, 136), ([42], [170], 3, 1, 32), ([128], [128], 1, 1, 16),
    ([1], [5000], 64, 8, 128), ([2], [9000], 5, 1, 256), ([1], [20000], 8, 1, 16), ([1, 1], [1, 12000], 16, 2, 64),
    ([1], [700], 128, 1, 16), ([2], [300], 128, 1, 40), ([1], [300], 67, 1, 16),
    ([129], [129], 1, 1, 16), ([130], [500], 4, 4, 16), ([200], [200], 8, 2, 16), ([33], [1000], 32, 8, 64), ([300], [1000], 8, 8, 24),
    ([257, 1, 100, 0, 64], [257, 900, 1100, 50, 64], 8, 2, 48), ([100], [3000], 7, 1, 104), ([513], [2049], 4, 2, 128),
    ([40, 1, 1, 90], [6000, 3000, 10, 95], 16, 2, 16), ([150], [100], 4, 2, 16), ([3, 300], [9000, 310], 8, 1, 8),
    ([1, 1, 1], [3000, 1, 700], 16, 1, 16), ([4, 3, 1], [2000, 40, 9], 16, 4, 32), ([8], [4000], 2, 1, 64), ([16, 2], [600, 5], 1, 1, 8),
    ([9], [1000], 1, 1, 16), ([17, 16], [800, 900], 2, 2, 16),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_attention(pec, dtype, i):
    n, kv, hq, hkv, page = SHAPES[i]
    attend(pec, 100 + i, n, kv, hq, hkv, page, dtype, head_major=i % 2 == 1, pad=i % 3, fused=i % 2 == 0, known=i % 4 != 3,
           what=f"{n} of {kv}, {hq}/{hkv} heads, pages of {page}"[:120])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", [1, 3, 5, 6, 12, 17, 26, 28, 31, 35])
def test_attention_without_the_causal_mask(pec, dtype, i):
    n, kv, hq, hkv, page = SHAPES[i]
    attend(pec, 300 + i, n, kv, hq, hkv, page, dtype, causal=False, what=f"not causal, {n} of {kv}"[:100])


@pytest.mark.parametrize("i", [2, 8, 16, 18, 24, 28, 30, 31, 34])
def test_attention_fp32_output_and_scale(pec, i):
    n, kv, hq, hkv, page = SHAPES[i]
    attend(pec, 400 + i, n, kv, hq, hkv, page, BF16, out_dtype=F32, scale=0.3, what=f"fp32 output, {n} of {kv}"[:100])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-8, 1e-3, 30.0])
def test_attention_at_other_magnitudes(pec, dtype, size):
    attend(pec, 500, [1, 40, 2], [900, 300, 5000], 8, 2, 16, dtype, size=size, what=f"keys and values of {size}")


def test_a_serving_step(pec):
    """Prefill in chunks, then decode steps: append, attention; and the same through what is read back of the cache."""
    hq, hkv, page, S = 16, 4, 32, 700
    g = torch.Generator().manual_seed(9)
    tables = pec.pec_rope_table(THETA, 2000, DEV)
    qkv = torch.randn((S, hq + 2 * hkv, 128), generator=g).to(BF16).to(DEV)
    q, _ = pec.pec_qk_norm_rope(qkv[:, :hq], tables=tables, pos0=0)
    kp, ks, vp, vs, table = cache = q4.make_cache(3, [S, 0], page, hkv, DEV, head_major=True)
    at = 0
    outs = []
    for n in (300, 1, 1, 129, 64, 1, 204):
        cu, kv = dev([0, n, n]), dev([at + n, 0])
        pec.pec_kv_append_q4(qkv[at:at + n, hq:hq + hkv], qkv[at:at + n, hq + hkv:], *cache, cu, kv, norm=True, tables=tables)
        outs.append(pec.pec_paged_attn_q4(q[at:at + n], *cache, cu, kv, max_q_len=n))
        at += n
    assert at == S
    pec.check_status()
    o, lse = torch.cat([x for x, _ in outs]), torch.cat([x for _, x in outs])
    want = q4.attend(q, cache, [0, S, S], [S, 0])
    ref.check_attend(o, lse, want, BF16, "chunks and steps")
    k, v = pec.pec_kv_read_q4(*cache, dev([0, S, S]), dev([S, 0]), S)
    o2, lse2 = pec.pec_prefill_attn(q.contiguous(), k, v)
    ref.check_attend(o2, lse2, want, BF16, "the prefill path over what is read back")
