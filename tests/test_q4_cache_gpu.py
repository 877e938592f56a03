"""Append and read of a cache held in 4 bits: how a call's work is divided changes no bit of what it does."""
import pytest
import torch

import q4_reference as q4
from test_q4_gpu import BF16, DEV, F32, THETA, dev

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
