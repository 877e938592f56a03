"""Append and read of a cache held in 4 bits: how a call's work is divided changes no bit of what it does."""
import pytest
import torch

import q4_reference as q4
from test_q4_gpu import BF16, DEV, F32, THETA, angles, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,hkv", [(2100, 8), (700, 3), (16000, 40), (1400, 33), (5000, 5), (4500, 1)])
def test_large_calls_do_what_small_ones_do(pec, dtype, T, hkv):
    """One call against calls of a few tokens at a time, which are divided otherwise: the same cache, the same tensors read back."""
    page, piece = 64, 97 if T < 10000 else 997
    tables = pec.pec_rope_table(THETA, T + 100, DEV)
    pages = -(-T // page) + 1
    order = torch.randperm(pages, device=DEV)[None].int()
    g = torch.Generator(device=DEV).manual_seed(3)
    x = (torch.randn((T, 2 * hkv, 128), generator=g, device=DEV) * torch.exp(torch.randn((T, 2 * hkv, 1), generator=g, device=DEV))).to(dtype)
    caches = []
    for _ in range(2):
        codes = [torch.zeros((pages, page, hkv, 64), dtype=torch.uint8, device=DEV) for _ in range(2)]
        scales = [torch.zeros((pages, page, hkv), dtype=BF16, device=DEV) for _ in range(2)]
        caches.append((codes[0], scales[0], codes[1], scales[1], order))
    k, v = x[:, :hkv], x[:, hkv:]
    pec.pec_kv_append_q4(k, v, *caches[0], dev([0, T]), dev([T]), norm=True, tables=tables)
    whole = pec.pec_kv_read_q4(*caches[0], dev([0, T]), dev([T]), T, dtype=dtype)
    for s in range(0, T, piece):
        n = min(piece, T - s)
        args = (dev([0, n]), dev([s + n]))
        pec.pec_kv_append_q4(k[s:s + n], v[s:s + n], *caches[1], *args, norm=True, tables=tables)
        part = pec.pec_kv_read_q4(*caches[0], *args, n, dtype=dtype)
        assert all(torch.equal(a[s:s + n], b) for a, b in zip(whole, part))
    pec.check_status()
    for a, b in zip(caches[0], caches[1]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # ... which is the definition's: a row of every class, and the values that it stands for.
    at = T // 2
    for which in range(2):
        codes, scales = caches[0][2 * which], caches[0][2 * which + 1]
        pg, slot = int(order[0, at // page]), at % page
        held = q4.values(codes[pg, slot], scales[pg, slot])
        assert torch.equal(whole[which][at].double().cpu(), torch.from_numpy(held))
        if which:
            assert (held == q4.quantise(v[at].double().cpu().numpy())[0]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("turn", [False, True])
def test_heads_that_norm_brings_next_to_borders(pec, dtype, turn):
    """Heads whose channels are all of one magnitude become the weight's to within eps / x^2, which lies on borders of codes and scales or
    just below them: the scale and the codes are the definition's to 2^-50 and 2^-41 (and the 2^-50 that the check's own fp64 is off by)."""
    T, hkv, page = 600, 4, 64
    g = torch.Generator().manual_seed(12)
    size = torch.exp(torch.rand((T, hkv, 1), generator=g).double() * 30 - 3)
    x = (size * torch.sign(torch.randn((T, hkv, 128), generator=g).double())).to(dtype).to(DEV)
    w = (torch.randn(128, generator=g) * 3).to(BF16).to(dtype).to(DEV)
    pages = -(-T // page)
    order = torch.randperm(pages, device=DEV)[None].int()
    codes = [torch.zeros((pages, page, hkv, 64), dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros((pages, page, hkv), dtype=BF16, device=DEV) for _ in range(2)]
    tables = pec.pec_rope_table(THETA, T, DEV) if turn else None
    pec.pec_kv_append_q4(x, x, codes[0], scales[0], codes[1], scales[1], order, dev([0, T]), dev([T]), norm=True, k_weight=w, tables=tables)
    pec.check_status()
    pos = torch.arange(T, device=DEV)
    pg, slot = order[0, pos // page].long(), pos % page
    held = torch.from_numpy(q4.values(codes[0][pg, slot], scales[0][pg, slot]))
    s = scales[0][pg, slot].double().cpu()[..., None]
    z = x.double().cpu()
    z = z * torch.rsqrt(z.square().mean(-1, keepdim=True) + float(torch.tensor(1e-6))) * w.double().cpu()
    if turn:
        c, t = (torch.from_numpy(v)[:, None] for v in angles(tables, list(range(T))))
        z = torch.cat([z[..., :64] * c - z[..., 64:] * t, z[..., 64:] * c + z[..., :64] * t], -1)
    most = z.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(s)                                          # the number before s has six significant bits as well
    before = torch.ldexp(torch.where(m == 0.5, torch.tensor(63 / 128, dtype=torch.float64), m - 1 / 64), e)
    assert (6 * s >= most * (1 - 2.0 ** -49)).all() and (6 * before < most * (1 + 2.0 ** -49)).all()
    off = (z - held).abs()
    nearest = ((z.abs() / s)[..., None] - torch.from_numpy(q4.MAGNITUDES)).abs().amin(-1) * s
    assert (off <= nearest + z.abs() * 2.0 ** -40).all()           # (a channel off a border by d is off one code by 2 d more than the other)
