"""How exactly the tensor-core kernels over a cache held in 4 bits hold what their products take: the documented bounds, from the
conversions' arithmetic on the CPU, and on the GPU where a single key or a single channel shows them."""
import numpy as np
import pytest
import torch

import q4_reference as q4
from paper_2409_15104_b200 import binding

BF16, F32, DEV = torch.bfloat16, torch.float32, "cuda:0"


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------ the conversions
def test_codes_times_scales_in_fp16():
    """In units in which the largest scale is 2^9 (values) or 2^12 (keys) at least: fp16 takes the scale, then the product."""
    scales = (np.arange(32, 64) / 32)[:, None] * 2.0 ** np.arange(-40, 13)[None]
    held = scales.astype(np.float16)[..., None] * q4.MAGNITUDES.astype(np.float16)
    assert held.dtype == np.float16
    off = np.abs(held.astype(np.float64) - scales[..., None] * q4.MAGNITUDES)
    assert off.max() == 6 * 2.0 ** -25
    assert off[scales >= 2.0 ** -18].max() == 0 and off[scales >= 2.0 ** -19].max() > 0
    # 2^-18 is 2^-27 of 2^9 and 2^-30 of 2^12; 6 * 2^-25 is 6 * 2^-34 and 6 * 2^-37 of them.


def _bf16_below(top):
    bits = torch.arange(0, 1 << 15, dtype=torch.int32).to(torch.int16)
    x = bits.view(BF16).double()
    return x[torch.isfinite(x) & (x < top)]


def test_queries_in_two_parts_of_e4m3():
    """A row's largest channel is brought to [2^7, 2^8)."""
    x = _bf16_below(2.0 ** 8)
    one = x.float().to(torch.float8_e4m3fn)
    two = ((x - one.double()) * 16).float().to(torch.float8_e4m3fn)
    off = (x - one.double() - two.double() / 16).abs()
    assert off.max() == 2.0 ** -14                                 # 2^-21 of 2^7
    assert off[x >= 2.0 ** -6].max() == 0                          # 2^-13 of 2^7


def test_queries_in_fp16():
    """A row's largest channel is brought to [2^14, 2^15)."""
    x = _bf16_below(2.0 ** 15)
    off = (x - x.float().half().double()).abs()
    assert off.max() <= 2.0 ** -25 and off[x >= 2.0 ** -17].max() == 0   # 2^-39 and 2^-31 of 2^14


# ------------------------------------------------------------------------------------------ the kernels
@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("below", [24, 29, 31])
def test_a_small_value_behind_a_large_one(pec, n, below):
    """A key that all rows see with all their weight (e^-200 on the others), whose value's scale lies far below one seen before: off by at most
    6 * 2^-34 of the largest scale, by the probability's rounding to fp16 (2^-11 of the value) and by fp32's (2^-20, with that of 2^x)."""
    kv = 300
    x = np.zeros((2, kv, 2, 128))                                  # keys, values
    x[0, :, :, 0] = -6.0
    x[0, kv - n, :, 0] = 6.0
    x[1, :kv - n] = np.random.RandomState(5).choice(q4.MAGNITUDES, (kv - n, 2, 128))
    x[1, 3, :, 0] = 6.0
    mantissas = np.arange(32, 64) / 32
    worst = 0.0
    for m in mantissas[1::6]:
        x[1, kv - n] = m * 2.0 ** -below * np.resize([6, 4, 3, 2, 1.5, 1, 0.5, 0, -6, -1.5], 128)
        cache = q4.make_cache(1, [kv], 16, 2, DEV, wild=False)
        ids = cache[4][0, :-(-kv // 16)].long()
        for which in range(2):
            codes, scales = q4.pack(x[which])
            full, s = cache[2 * which][ids].flatten(0, 1), cache[2 * which + 1][ids].flatten(0, 1)
            full[:kv], s[:kv] = codes.to(DEV), scales.to(DEV)
            cache[2 * which][ids], cache[2 * which + 1][ids] = full.view(-1, 16, 2, 64), s.view(-1, 16, 2)
        q = torch.zeros((n, 8, 128), dtype=BF16, device=DEV)
        q[..., 0] = 200.0
        o, _ = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([kv]), max_q_len=n, out_dtype=F32)
        pec.check_status()
        want = q4.values(cache[2], cache[3])[ids.cpu().numpy()].reshape(-1, 2, 128)[kv - n].repeat(4, 0)
        off = np.abs(o.double().cpu().numpy() - want)
        worst = max(worst, off.max())
        assert (off <= 6 * 2.0 ** -34 + (2.0 ** -11 + 2.0 ** -20) * np.abs(want)).all(), (m, off.max() * 2.0 ** 34)
    print(f"[parity] {n} tokens, 2^-{below}: off by {worst * 2.0 ** 34:.3f} * 2^-34 of the largest scale")


@pytest.mark.gpu
@pytest.mark.parametrize("n,bound,scale", [(1, 2.0 ** -21, 2.0 ** 12), (40, 2.0 ** -39, 2.0 ** 30)])
def test_a_small_channel_of_a_query(pec, n, bound, scale):
    """A key of one channel, against rows whose largest channel (1) it does not have: a row's LSE over this one key is the score of that
    channel, by a scale that makes the bound large beside fp32's roundings."""
    kv, hkv = n, 1
    small = (1 + torch.arange(128).double() / 128) * 2.0 ** -torch.arange(13, 45).repeat(4).double()
    q = torch.zeros((n, 16, 128), dtype=BF16)
    q[..., 0] = 1.0
    cache = q4.make_cache(2, [kv], 16, hkv, DEV, wild=False)
    x = np.zeros((1, 1, 128))
    x[..., 1] = 6.0
    codes, scales = q4.pack(x)
    cache[0][cache[4][0, 0].long(), 0], cache[1][cache[4][0, 0].long(), 0] = codes[0].to(DEV), scales[0].to(DEV)
    worst = 0.0
    for part in range(0, 128, 16):
        q[0, :, 1] = small[part:part + 16].to(BF16)                # row 0 is at position 0 and sees the first key only
        _, lse = pec.pec_paged_attn_q4(q.to(DEV), *cache, dev([0, n]), dev([kv]), max_q_len=n, softmax_scale=scale)
        pec.check_status()
        want = 6.0 * scale * q[0, :, 1].double()
        off = (lse[0].double().cpu() - want).abs()
        # fp32: the score's scale, its product, log2 units and back, 2^-24 of it each; ln of a sum beside them, 2^-20.
        assert (off <= 6 * scale * bound + 4 * 2.0 ** -24 * want + 2.0 ** -20).all(), (off / (6 * scale * bound)).max()
        worst = max(worst, float((off / (6 * scale)).max()))
    print(f"[parity] {n} tokens: off by {worst / bound:.3f} of the bound")


# ------------------------------------------------------------------------------------------ what four bits cost
def test_what_heads_are_held_to():
    """The documented errors of held heads against what was quantised (2-norm, relative): means over 4000 heads, whose own errors differ by a
    tenth, so that a mean is known to 0.0005 and its third digit to be tested."""
    x = np.random.RandomState(7).standard_normal((4000, 128))
    outliers, pair = x.copy(), x.copy()
    outliers[:, [5, 69, 40, 104]] *= 10
    pair[:, [3, 77]] *= 10
    for y, want in ((x, 0.109), (pair, 0.198), (outliers, 0.195)):
        off = np.linalg.norm(q4.quantise(y)[0] - y) / np.linalg.norm(y)
        assert abs(off - want) <= 0.003, (off, want)
