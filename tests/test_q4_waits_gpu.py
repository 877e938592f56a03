"""Attention over a cache held in 4 bits where what a kernel reads is late, or is written by another warp: queries that come from memory
while the cache is at hand, and calls that run beside others."""
import pytest
import torch

import paged_reference as ref
import q4_reference as q4
from test_q4_gpu import BF16, DEV, F32, attend, check, dev

pytestmark = pytest.mark.gpu


def one_token_requests(q, cache, kv, hkv):
    """paged_reference.attend for requests of one token each over the same kv cached tokens, all at once: o, lse, A, B."""
    kp, ks, vp, vs, table = cache
    page = kp.shape[1]
    ids = table[0, :-(-kv // page)].cpu().numpy()
    k, v = (torch.from_numpy(q4.values(p, s)[ids].reshape(-1, hkv, 128)[:kv]).to(DEV) for p, s in ((kp, ks), (vp, vs)))
    x = q.double().unflatten(1, (hkv, -1))                         # [T, Hkv, g, D]
    z = torch.einsum("thgd,khd->thgk", x, k) / 128 ** 0.5
    B = torch.einsum("thgd,khd->thgk", x.abs(), k.abs()).amax(-1) / 128 ** 0.5
    p = torch.softmax(z, -1)
    o, A = (torch.einsum("thgk,khd->thgd", p, y) for y in (v, v.abs()))
    return [t.flatten(1, 2).cpu().numpy() for t in (o, torch.logsumexp(z, -1), A, B)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kv,hq,hkv", [(64, 8, 8), (40, 8, 2), (200, 16, 4)])
def test_queries_that_come_late(pec, dtype, kv, hq, hkv):
    """Queries out of memory, beside a cache, tables and a plan that are in L2: the first scores wait for them."""
    T = 4000
    cache = q4.make_cache(17, [kv], 16, hkv, DEV)
    table = cache[4].expand(T, -1).contiguous()                    # (pages may be shared for reading)
    q = torch.randn((T, hq, 128), generator=torch.Generator().manual_seed(18)).to(dtype).to(DEV)
    args = (*cache[:4], table, dev(list(range(T + 1))), dev([kv] * T))
    want = one_token_requests(q, cache, kv, hkv)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device=DEV)    # (twice the L2)
    for most in (1, 0):
        for _ in range(3):
            flush.fill_(1)
            pec.pec_kv_read_q4(*cache, dev([0, kv]), dev([kv]), kv)
            args[4].sum(), args[5].sum(), args[6].sum()
            o, lse = pec.pec_paged_attn_q4(q, *args, max_q_len=most)
            pec.check_status()
            check(o, lse, want, dtype, cache, [kv], hq // hkv, f"late queries, {kv} keys")


def test_calls_of_both_types_at_once(pec):
    """fp32 and bf16 batches on streams of their own, beside copies that keep the memory busy: the same bits as alone."""
    cases = []
    for seed, dtype, n, kv in ((31, F32, [1] * 30, [300 + 31 * i for i in range(30)]), (32, F32, [200, 1, 70], [900, 4000, 70]), (33, F32, [3], [9000]),
                               (34, BF16, [300, 2], [2000, 500])):
        cache = q4.make_cache(seed, kv, 16, 2, DEV)
        q = torch.randn((sum(n), 8, 128), generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)
        args = (q, *cache, dev(ref.offsets(n)), dev(kv))
        want = pec.pec_paged_attn_q4(*args, max_q_len=max(n))
        check(*want, q4.attend(q, cache, ref.offsets(n), kv), dtype, cache, kv, 4 * max(n), f"alone {n[:3]}")
        cases.append((args, max(n), want))
    room = torch.empty((2, 1 << 28), dtype=torch.uint8, device=DEV)
    streams = [torch.cuda.Stream() for _ in range(len(cases) + 1)]
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(streams[-1]):
            room[0].copy_(room[1])
        got = [pec.pec_paged_attn_q4(*args, max_q_len=most, stream=s) for (args, most, _), s in zip(cases, streams)]
        torch.cuda.synchronize()
        for (_, _, want), have in zip(cases, got):
            assert torch.equal(want[0], have[0]) and torch.equal(want[1], have[1])
    pec.check_status()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,kv,hq,hkv,page", [([200], [100], 4, 2, 16), ([300], [70], 8, 2, 24), ([256, 3, 400], [100, 50, 270], 1, 1, 8), ([700], [596], 16, 1, 64),
                                              ([200] * 30, [100] * 30, 16, 8, 16)])
def test_leading_rows_that_see_nothing(pec, n, kv, hq, hkv, page, causal):
    """Requests with more new tokens than cached ones: whole stages without keys beside stages with some, many times over."""
    for seed in range(4):
        attend(pec, 200 + seed, n, kv, hq, hkv, page, BF16, causal=causal, out_dtype=F32 if seed % 2 else None, what=f"{n[:3]} of {kv[:3]}")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("prefix", [128, 1152, 3968])
def test_leading_rows_of_a_slice_that_see_nothing_of_it(pec, prefix, bad):
    """Keys cut into slices of which a block's first stage sees none and its second one some; a query that is not finite in the first
    stage's rows stays in its row."""
    n, kv, bad_row = 256, prefix + 256, 70
    cache = q4.make_cache(51, [kv], 16, 1, DEV)
    q = torch.randn((n, 1, 128), generator=torch.Generator().manual_seed(52)).to(BF16).to(DEV)
    want = q4.attend(q, cache, [0, n], [kv])
    want[1][bad_row, 0] = want[0][bad_row, 0] = float("nan")       # (rows that check passes over)
    q[bad_row, 0, 7] = bad
    for _ in range(8):
        o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([kv]), max_q_len=n)
        pec.check_status()
        assert torch.isnan(o[bad_row]).all() and torch.isnan(lse[bad_row]).all()
        check(o, lse, want, BF16, cache, [kv], n, f"beside a query of {bad}, prefix {prefix}")
