"""The paged cache held in 4 bits as programs use it: graphs, streams and workspaces, shared and far pages, orders of the cache, large
batches, bad tables, numbers that are not finite, and rows whose weight lies where rounding costs the most."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import q4_reference as q4
from paper_2409_15104_b200 import binding
from test_q4_gpu import BF16, DEV, F32, THETA, attend, check, check_held, dev

pytestmark = pytest.mark.gpu


def queries(seed, T, hq, dtype):
    return torch.randn((T, hq, 128), generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("norm,turn", [(True, True), (False, True), (True, False)])
def test_append_decides_every_code_of_many_heads(pec, dtype, norm, turn):
    """Some 10000 heads with half a percent of them beside a border of two codes or of two scales: exactly the definition's numbers.
    Weights of either sign and size, heads of few and of equal channels."""
    n, hkv, page = 1300, 8, 64
    kp, ks, vp, vs, table = q4.make_cache(41, [n + 60], page, hkv, DEV)
    g = torch.Generator().manual_seed(42)
    k = torch.randn((n, hkv, 128), generator=g)
    k[::7] *= torch.exp(6 * torch.randn((n, hkv, 1), generator=g))[::7]
    k[3::50, :, 5:] = 0
    k[4::50] = 1.5
    k[5::50, :, ::2] *= 1e-4
    k = k.to(dtype).to(DEV)
    w = (torch.randn(128, generator=g) * 3).to(dtype).to(DEV) if norm else None
    tables = pec.pec_rope_table(THETA, 3000, DEV) if turn else None
    pec.pec_kv_append_q4(k, k, kp, ks, vp, vs, table, dev([0, n]), dev([n + 60]), norm=norm, k_weight=w, tables=tables)
    pec.check_status()
    pos = list(range(60, n + 60))
    pg, slot = [int(table[0, p // page]) for p in pos], [p % page for p in pos]
    check_held(kp[pg, slot], ks[pg, slot], k, w, pos, norm, tables)
    check_held(vp[pg, slot], vs[pg, slot], k, None, pos, False, None)


@pytest.mark.parametrize("T,cu", [(8, [5, 3, 8]), (4, [0, 4, 9, 9]), (4, [0, 4, 100, 50]), (6, [0] * 40 + [6] * 40 + [2, 6]), (3, [0] + [3] * 700 + [1] + [3] * 20)])
def test_offsets_that_no_row_meets_are_reported(pec, T, cu):
    """Offsets that descend before the first row or after the last one, or pass T, in any group of requests."""
    B = len(cu) - 1
    kp, ks, vp, vs, table = q4.make_cache(43, [20] * B, 16, 1, DEV, wild=False)
    x = torch.randn((T, 1, 128), device=DEV)
    for call in (lambda: pec.pec_kv_append_q4(x, x, kp, ks, vp, vs, table, dev(cu), dev([20] * B)),
                 lambda: pec.pec_kv_read_q4(kp, ks, vp, vs, table, dev(cu), dev([20] * B), T),
                 lambda: pec.pec_paged_attn_q4(x, kp, ks, vp, vs, table, dev(cu), dev([20] * B))):
        call()
        with pytest.raises(binding.PecError) as e:
            pec.check_status()
        assert e.value.code == binding.PEC_ERR_BAD_INDEX


@pytest.mark.parametrize("T", [70, 9000])
def test_read_of_many_requests_and_paddings(pec, T):
    """Warps whose rows are of several requests, of none, or of a bad table: everyone's own rows, the others as they were."""
    g = np.random.RandomState(6)
    n = []
    while sum(n) + 10 < T - 9:
        n.append(int(g.choice([0, 1, 2, 3, 5, 9])))
    kv = [m + int(g.choice([0, 3, 40])) for m in n]
    kp, ks, vp, vs, table = q4.make_cache(44, kv, 16, 2, DEV)
    bad = [b for b in range(len(n)) if n[b] >= 2][::5]
    for b in bad:
        table[b, (kv[b] - 1) // 16] = -3
    cu = [c + 5 for c in ref.offsets(n)]
    out = torch.full((2, T, 2, 128), 7.0, dtype=BF16, device=DEV)
    pec.pec_kv_read_q4(kp, ks, vp, vs, table, dev(cu), dev(kv), T, k_out=out[0], v_out=out[1])
    with pytest.raises(binding.PecError):
        pec.check_status()
    want = torch.full((2, T, 2, 128), 7.0, dtype=BF16)
    held = [torch.from_numpy(q4.values(p, s)).to(BF16) for p, s in ((kp, ks), (vp, vs))]
    t = table.cpu()
    for b in range(len(n)):
        for i in range(n[b]):
            at = kv[b] - n[b] + i
            if int(t[b, at // 16]) >= 0:
                for which in range(2):
                    want[which, cu[b] + i] = held[which][int(t[b, at // 16]), at % 16]
    assert torch.equal(out.cpu(), want)


# ------------------------------------------------------------------------------------------ pages
def test_pages_beyond_32_bits_of_bytes(pec):
    """Append, read and attend at the far end of a cache of 2 x 4.5 GB."""
    page, hkv = 64, 8
    num = (1 << 32) // (page * hkv * 64) + 8000
    kp, vp = (torch.empty((num, page, hkv, 64), dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.ones((num, page, hkv), dtype=BF16, device=DEV) for _ in range(2))
    for dtype in (BF16, F32):
        for n, kv in ((1, 100), (170, 250)):
            table = dev([[num - 1, num - 7, num - 3, num - 20, 0]])
            for t in (kp, vp):
                t[-40:].random_(0, 256)
            k, v, q = (torch.randn((n, h, 128), device=DEV).to(dtype) for h in (hkv, hkv, 16))
            cu, lens = dev([0, n]), dev([kv])
            pec.pec_kv_append_q4(k, v, kp, ks, vp, vs, table, cu, lens)
            o, lse = pec.pec_paged_attn_q4(q, kp, ks, vp, vs, table, cu, lens, max_q_len=n)
            k2, _ = pec.pec_kv_read_q4(kp, ks, vp, vs, table, cu, lens, n, dtype=dtype)
            pec.check_status()
            near = table.clone()
            near[0, :4] -= num - 40
            cache = tuple(t[-40:] for t in (kp, ks, vp, vs)) + (near,)
            check(o, lse, q4.attend(q, cache, [0, n], [kv]), dtype, cache, [kv], 2 * n, f"far pages {n}")
            assert np.array_equal(k2.double().cpu().numpy(), q4.quantise(k.double().cpu().numpy())[0])
    del kp, vp, ks, vs
    torch.cuda.empty_cache()


@pytest.mark.parametrize("page,total", [(1024, 5000), (65536, 70000), (512, 512), (8, 2999)])
def test_page_sizes_and_a_cache_of_one_page(pec, page, total):
    for n in (1, 140):
        attend(pec, page + n, [n], [total], 4, 1, page, BF16, known=n == 1, what=f"pages of {page}, {n} new")


def test_requests_that_share_pages(pec):
    kp, ks, vp, vs, table = cache = q4.make_cache(61, [333, 333], 16, 2, DEV)
    table[1, :20] = table[0, :20]
    for n in ([1, 1], [100, 13]):
        cu = ref.offsets(n)
        q = queries(62, sum(n), 8, BF16)
        o, lse = pec.pec_paged_attn_q4(q, *cache, dev(cu), dev([333, 333]), max_q_len=max(n))
        pec.check_status()
        check(o, lse, q4.attend(q, cache, cu, [333, 333]), BF16, cache, [333], max(n) * 4, f"shared pages {n}")


def other_order(codes, scales, order):
    """The same cache behind other strides."""
    P, page, hkv, _ = codes.shape
    if order == "heads first":
        return codes.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3), scales.permute(2, 0, 1).contiguous().permute(1, 2, 0)
    if order == "between a token's others":
        full = torch.full((P, page, hkv, 2, 64), 0xff, dtype=torch.uint8, device=DEV)
        full[:, :, :, 1] = codes
        sc = torch.full((P, page, hkv, 3), float("nan"), dtype=BF16, device=DEV)
        sc[..., 2] = scales
        return full[:, :, :, 1], sc[..., 2]
    st = hkv * 96 + 32                                             # strides whose greatest common divisor is 32 bytes
    full = torch.full((P * (page * st + 32),), 0xff, dtype=torch.uint8, device=DEV)
    out = full.as_strided(codes.shape, (page * st + 32, st, 96, 1))
    out.copy_(codes)
    return out, scales


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k_order,v_order", [("heads first", "heads first"), ("between a token's others", "odd strides"), ("odd strides", "heads first")])
@pytest.mark.parametrize("n,kv,hq,hkv,page", [([1, 1, 1], [700, 130, 33], 8, 2, 16), ([3, 20], [900, 260], 6, 3, 24), ([200, 1], [500, 300], 8, 1, 64),
                                              ([1], [200], 4, 4, 256)])
def test_orders_of_the_cache(pec, dtype, k_order, v_order, n, kv, hq, hkv, page):
    kp, ks, vp, vs, table = cache = q4.make_cache(71, kv, page, hkv, DEV)
    cu, T = ref.offsets(n), sum(n)
    q = queries(72, T, hq, dtype)
    plain = pec.pec_paged_attn_q4(q, *cache, dev(cu), dev(kv), max_q_len=max(n))
    other = (*other_order(kp, ks, k_order), *other_order(vp, vs, v_order), table)
    o, lse = pec.pec_paged_attn_q4(q, *other, dev(cu), dev(kv), max_q_len=max(n))
    read = [pec.pec_kv_read_q4(*c, dev(cu), dev(kv), T, dtype=dtype) for c in (cache, other)]
    pec.check_status()
    check(o, lse, q4.attend(q, cache, cu, kv), dtype, cache, kv, max(n) * (hq // hkv), f"{k_order}, {v_order}")
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1]), "the order of the cache changed bits"
    assert torch.equal(read[0][0], read[1][0]) and torch.equal(read[0][1], read[1][1])
    x = torch.randn((T, hkv, 128), device=DEV).to(dtype)
    for c in (cache, other):
        pec.pec_kv_append_q4(x, x, *c, dev(cu), dev(kv))
    pec.check_status()
    assert all(torch.equal(a, b) or torch.equal(a.isnan(), b.isnan()) for a, b in zip(cache[1::2], other[1::2]))
    assert torch.equal(cache[0], other[0]) and torch.equal(cache[2], other[2])


@pytest.mark.skipif(not hasattr(torch, "float4_e2m1fn_x2"), reason="torch without the type")
def test_pages_of_torchs_own_type(pec):
    kp, ks, vp, vs, table = q4.make_cache(73, [100, 40], 16, 2, DEV)
    q = queries(74, 2, 8, BF16)
    args = (dev([0, 1, 2]), dev([100, 40]))
    a = pec.pec_paged_attn_q4(q, kp, ks, vp, vs, table, *args)
    b = pec.pec_paged_attn_q4(q, kp.view(torch.float4_e2m1fn_x2), ks, vp.view(torch.float4_e2m1fn_x2), vs, table, *args)
    pec.check_status()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------------------------------ streams, graphs, workspaces
def test_streams_graphs_and_a_shared_workspace(pec):
    """Steps captured and replayed after lengths and inputs have changed; graphs that share a workspace and run one after the other; an
    eager call on a stream of its own."""
    page, hkv, hq = 16, 2, 8
    binding.status_word(torch.device(DEV))
    cache = q4.make_cache(31, [900, 400, 333], page, hkv, DEV, wild=False)
    for t in (cache[1], cache[3]):
        t[~torch.isfinite(t)] = 1.0
    tables = pec.pec_rope_table(THETA, 4000, DEV)
    ws = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    steps = []
    for n, dtype in (([1, 1, 1], BF16), ([40, 1, 150], BF16), ([3, 1, 70], F32)):
        T = sum(n)
        q, k, v = (torch.randn((T, h, 128), device=DEV).to(dtype) for h in (hq, hkv, hkv))
        steps.append(dict(n=n, dtype=dtype, cu=dev(ref.offsets(n)), kv=dev([900, 400, 333]), q=q, k=k, v=v, o=torch.empty_like(q), lse=torch.empty((T, hq), device=DEV)))

    def issue(s):
        pec.pec_kv_append_q4(s["k"], s["v"], *cache, s["cu"], s["kv"], norm=True, tables=tables)
        pec.pec_paged_attn_q4(s["q"], *cache, s["cu"], s["kv"], max_q_len=max(s["n"]), o=s["o"], lse=s["lse"], workspace=ws)

    graphs = []
    for s in steps:
        issue(s)                                                  # warm up outside the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            issue(s)
        graphs.append(graph)
    for lens in ([900, 400, 333], [700, 123, 208]):
        for s in steps:
            s["kv"].copy_(dev(lens))
            s["q"].normal_()
        for s, graph in zip(steps, graphs):
            graph.replay()
            pec.check_status()
            got = s["o"].clone(), s["lse"].clone()
            check(*got, q4.attend(s["q"], cache, s["cu"].tolist(), lens), s["dtype"], cache, lens, 4 * max(s["n"]), f"replayed {lens}")
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            o, lse = pec.pec_paged_attn_q4(s["q"], *cache, s["cu"], s["kv"], max_q_len=max(s["n"]), stream=side)
            side.synchronize()
            assert torch.equal(o, got[0]) and torch.equal(lse, got[1])


def test_two_calls_at_once(pec):
    """Batches on streams and workspaces of their own, many times: the same bits as one after the other."""
    cases = []
    for seed, n, kv in ((51, [1] * 20, [700 + 31 * i for i in range(20)]), (52, [200, 1, 70], [900, 4000, 70]), (53, [4], [9000])):
        cache = q4.make_cache(seed, kv, 16, 2, DEV)
        args = (queries(seed, sum(n), 8, BF16), *cache, dev(ref.offsets(n)), dev(kv))
        cases.append((args, max(n), pec.pec_paged_attn_q4(*args, max_q_len=max(n))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        got = [pec.pec_paged_attn_q4(*args, max_q_len=most, stream=s) for (args, most, _), s in zip(cases, streams)]
        torch.cuda.synchronize()
        for (_, _, want), have in zip(cases, got):
            assert torch.equal(want[0], have[0]) and torch.equal(want[1], have[1])
    pec.check_status()


def test_calls_on_another_stream_keep_their_tensors(pec):
    """Inputs of the current stream that are dropped as soon as the call returns, while the call's stream is still busy."""
    cache = q4.make_cache(27, [600], 16, 2, DEV)
    q = queries(28, 64, 8, BF16)
    want = pec.pec_paged_attn_q4(q, *cache, dev([0, 64]), dev([600]), max_q_len=64)
    want_k, _ = pec.pec_kv_read_q4(*cache, dev([0, 64]), dev([600]), 64)
    once = [t.clone() for t in cache[:4]]
    pec.pec_kv_append_q4(q[:, :2], q[:, 2:4], *once, cache[4], dev([0, 64]), dev([600]))
    twice = [t.clone() for t in cache[:4]]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for call in (lambda: pec.pec_paged_attn_q4(q.clone(), *(t.clone() for t in cache), dev([0, 64]), dev([600]), max_q_len=64, stream=side),
                 lambda: pec.pec_kv_read_q4(*(t.clone() for t in cache), dev([0, 64]), dev([600]), 64, stream=side)[:1],
                 lambda: pec.pec_kv_append_q4(q.clone()[:, :2], q.clone()[:, 2:4], *twice, cache[4].clone(), dev([0, 64]), dev([600]), stream=side)):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)                        # 50 ms
        out = call()
        for _ in range(20):                                       # whatever small blocks are free now
            torch.full((64, 8, 128), 100.0, dtype=BF16, device=DEV)
            torch.full((64,), 99, dtype=torch.int32, device=DEV)
        torch.cuda.synchronize()
        if out is not None:
            assert torch.equal(out[0], want[0] if len(out) == 2 else want_k)
    for a, b in zip(twice, once):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    pec.check_status()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cu", [[0, 200] * 32 + [0], [200, 0] * 32 + [200], [0, 200, 200, 0] * 16 + [200]])
def test_overlapping_offsets_stay_inside_the_workspace(pec, dtype, cu):
    """Offsets that go back and forth have together many times the blocks of T tokens.  The workspace has exactly the size asked for;
    what lies around it is not written."""
    kp, ks, vp, vs, table = q4.make_cache(26, [1024] * 64, 128, 1, DEV)
    q = queries(27, 200, 1, dtype)
    a = binding.pec_paged_q4_args()
    a.q, a.o, a.lse, a.status = [1 << 20] * 4
    c = a.cache
    c.k_pages, c.v_pages, c.k_scales, c.v_scales, c.block_table, c.cu_q, c.kv_lens = [1 << 20] * 7
    c.k_pages_stride_p = c.v_pages_stride_p = 128 * 64
    c.k_pages_stride_t = c.v_pages_stride_t = c.k_pages_stride_h = c.v_pages_stride_h = 64
    c.k_scales_stride_p = c.v_scales_stride_p = 128
    c.k_scales_stride_t = c.v_scales_stride_t = c.k_scales_stride_h = c.v_scales_stride_h = 1
    c.page_size, c.num_pages, c.table_stride, c.max_pages, c.B, c.T, c.Hkv, c.D = 128, kp.shape[0], table.shape[1], table.shape[1], 64, 200, 1, 128
    a.q_stride_t = a.q_stride_h = 128
    a.dtype = a.o_dtype = binding.PEC_BF16 if dtype == BF16 else binding.PEC_F32
    a.Hq, a.causal = 1, 1
    need = binding.pec_paged_q4_workspace_size(a)
    assert need > 0
    guard = 4 << 20
    room = torch.full(((need + 2 * guard) // 4 + 4,), 1000.0, device=DEV)
    bytes_ = room.view(torch.uint8)
    o, lse = torch.full((200, 1, 128), 7.0, dtype=dtype, device=DEV), torch.full((200, 1), 7.0, device=DEV)
    pec.pec_paged_attn_q4(q, kp, ks, vp, vs, table, dev(cu), dev([1024] * 64), o=o, lse=lse, workspace=bytes_[guard:guard + need])
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
    assert (bytes_[:guard].view(torch.float32) == 1000.0).all() and (room[(guard + need + 3) // 4:] == 1000.0).all()
    assert o.float().abs().max() < 100 and lse.abs().max() < 100


@pytest.mark.parametrize("n,kv,hq", [([1] * 40, [2500] * 40, 8), ([4] * 9, [3000] * 9, 8), ([300, 300], [2500, 2500], 8)])
def test_a_wait_that_runs_out_is_reported(pec, n, kv, hq):
    """The last value tile of each CTA is left out: the waits for it run out within the limit, the status word says so, and the next
    launch is right."""
    cache = q4.make_cache(81, kv, 16, 2, DEV)
    q, cu = queries(82, sum(n), hq, BF16), ref.offsets(n)
    args = (q, *cache, dev(cu), dev(kv))
    try:
        pec.pec_control(binding.PEC_CTL_WAIT_LIMIT_CYCLES, 4_000_000)
        pec.pec_control(binding.PEC_CTL_TEST_SKIP_LAST_LOAD, 1)
        pec.pec_paged_attn_q4(*args, max_q_len=max(n))
        with pytest.raises(binding.PecError) as e:
            pec.check_status()
        assert e.value.code == binding.PEC_ERR_TIMEOUT
    finally:
        pec.pec_control(binding.PEC_CTL_TEST_SKIP_LAST_LOAD, 0)
        pec.pec_control(binding.PEC_CTL_WAIT_LIMIT_CYCLES, 2_000_000_000)
    o, lse = pec.pec_paged_attn_q4(*args, max_q_len=max(n))
    pec.check_status()
    check(o, lse, q4.attend(q, cache, cu, kv), BF16, cache, kv, max(n) * (hq // 2), "after a wait that ran out")


# ------------------------------------------------------------------------------------------ batches
def test_calls_without_tokens(pec):
    cache = q4.make_cache(45, [20], 16, 2, DEV)
    before = [t.clone() for t in cache[:4]]
    none = torch.empty((0, 2, 128), dtype=BF16, device=DEV)
    pec.pec_kv_append_q4(none, none, *cache, dev([0, 0]), dev([20]))
    k, v = pec.pec_kv_read_q4(*cache, dev([0, 0]), dev([20]), 0)
    o, lse = pec.pec_paged_attn_q4(torch.empty((0, 8, 128), dtype=BF16, device=DEV), *cache, dev([0, 0]), dev([20]))
    pec.check_status()
    assert k.shape == v.shape == (0, 2, 128) and o.shape == (0, 8, 128) and lse.shape == (0, 8)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache, before))


def test_a_request_per_row_of_a_large_batch(pec):
    """More requests than a warp or a group of the plan looks at once, of both classes, some empty, with room before the first and after
    the last row."""
    g = np.random.RandomState(4)
    for B, pick in ((1500, [0, 1, 1, 2]), (300, [0, 1, 130, 200])):
        n = [int(x) for x in g.choice(pick, B)]
        kv = [m + int(x) for m, x in zip(n, g.choice([0, 1, 30, 200], B))]
        cache = q4.make_cache(B, kv, 16, 1, DEV)
        cu = [c + 3 for c in ref.offsets(n)]
        T = cu[-1] + 2
        q = queries(B, T, 1, BF16)
        o, lse = torch.full((T, 1, 128), 7.0, dtype=BF16, device=DEV), torch.full((T, 1), 7.0, device=DEV)
        pec.pec_paged_attn_q4(q, *cache, dev(cu), dev(kv), o=o, lse=lse)
        pec.check_status()
        for rows in (slice(0, 3), slice(cu[-1], T)):
            assert (o[rows] == 7.0).all() and (lse[rows] == 7.0).all()
        check(o, lse, q4.attend(q, cache, cu, kv), BF16, cache, kv, 1 if max(pick) < 16 else 200, f"{B} requests")


@pytest.mark.parametrize("hq", [4, 8, 16])
def test_short_requests_in_a_row(pec, hq):
    """Several units in a CTA's piece of the line, many of them of one step: a unit begins while the one before the last is still read."""
    g = np.random.RandomState(hq)
    kv = [int(x) for x in g.choice([1, 40, 200, 256, 300, 700], 1100)]
    cache = q4.make_cache(hq, kv, 64, 1, DEV)
    q = queries(hq, len(kv), hq, BF16)
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev(ref.offsets([1] * len(kv))), dev(kv), max_q_len=1)
    pec.check_status()
    check(o, lse, q4.attend(q, cache, ref.offsets([1] * len(kv)), kv), BF16, cache, kv, hq, f"{len(kv)} short requests")


def test_bad_tables_are_reported(pec):
    for dtype in (F32, BF16):
        for n in (1, 5, 200):
            kp, ks, vp, vs, table = q4.make_cache(13, [300], 16, 1, DEV, wild=False)
            q = queries(14, n, 2, dtype)
            cases = []
            for bad in (-1, kp.shape[0], 2 ** 31 - 1):
                t = table.clone()
                t[0, 7] = bad
                cases.append((t, [0, n], [300], n))
            cases += [(table, [0, n + 1], [300], n), (table, [-1, n], [300], n), (table, [n, 0], [300], n), (table, [0, n], [-1], n),
                      (table, [0, n], [10000], n), (table, [0, n], [2 ** 31 - 1], n)]
            if n > 1:
                cases.append((table, [0, n], [300], n - 1))       # more new tokens than max_q_len allows
            for t, cu, kv, most in cases:
                pec.pec_paged_attn_q4(q, kp, ks, vp, vs, t, dev(cu), dev(kv), max_q_len=most)
                with pytest.raises(binding.PecError) as e:
                    pec.check_status()
                assert e.value.code == binding.PEC_ERR_BAD_INDEX
            o, lse = pec.pec_paged_attn_q4(q, kp, ks, vp, vs, table, dev([0, n]), dev([300]), max_q_len=n)
            pec.check_status()
            check(o, lse, q4.attend(q, (kp, ks, vp, vs, table), [0, n], [300]), dtype, (kp, ks, vp, vs), [300], 2 * n, "after bad tables")


# ------------------------------------------------------------------------------------------ numbers
@pytest.mark.parametrize("n,kv", [(1, 40000), (4, 40000), (40, 40000)])
@pytest.mark.parametrize("ahead", [8.0, 17.0, 25.0])
def test_weight_beside_one_key_that_takes_most(pec, n, kv, ahead):
    """A first key that is `ahead` (natural units) of all others and has no value, as long prompts have it: what is left comes from
    probabilities far below the largest."""
    kp, ks, vp, vs, table = cache = q4.make_cache(91, [kv], 64, 1, DEV)
    g = torch.Generator().manual_seed(92)
    along = torch.sign(torch.randn(128, generator=g))
    for p, s, first in ((kp, ks, along.numpy() * 4.0), (vp, vs, np.zeros(128))):
        c, sc = q4.pack(first[None].astype(np.float64))
        p[int(table[0, 0]), 0, 0], s[int(table[0, 0]), 0, 0] = c[0].to(DEV), sc[0].to(DEV)
    q = (0.1 * torch.randn((n, 4, 128), generator=g) + along * ahead / (4 * 128 ** 0.5)).to(BF16).to(DEV)
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([kv]), max_q_len=n, out_dtype=F32)
    pec.check_status()
    want = q4.attend(q, cache, [0, n], [kv])
    check(o, lse, want, BF16, cache, [kv], 4 * n, f"{ahead} ahead, {n} tokens")


@pytest.mark.parametrize("n,hq", [(1, 4), (3, 5), (100, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_of_ten_thousand(pec, dtype, n, hq):
    kp, ks, vp, vs, table = cache = q4.make_cache(9, [1500], 16, 1, DEV)
    ids = table[0, :94].tolist()                                  # 1500 tokens in pages of 16
    ramp = torch.exp2(torch.linspace(0.0, 6.0, 94, device=DEV).floor()).view(94, 1, 1)
    ks[ids] = (ks[ids].float() * ramp).to(BF16)
    q = queries(10, n, hq, dtype)
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([1500]), max_q_len=n, softmax_scale=20.0)
    pec.check_status()
    want = q4.attend(q, cache, [0, n], [1500], scale=20.0)
    assert want[1].max() > 1e4
    check(o, lse, want, dtype, cache, [1500], n * hq, f"scores to {want[1].max():.0f}")


@pytest.mark.parametrize("n", [1, 4, 60])
@pytest.mark.parametrize("step", [2.0 ** 4, 2.0 ** -4])
def test_scales_that_climb_and_fall(pec, n, step):
    """Keys and values whose scales change by 2^4 every hundred tokens, up or down over 2^28: nothing overflows, and what is small beside
    values seen before is held to what its tolerance counts."""
    kp, ks, vp, vs, table = cache = q4.make_cache(93, [800], 16, 2, DEV)
    for j in range(50):
        page = int(table[0, j])
        vs[page] = (vs[page].float() * step ** (j // 7)).to(BF16)
        ks[page] = (ks[page].float() * 2.0 ** -(j // 10)).to(BF16)
    q = queries(94, n, 8, BF16)
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([800]), max_q_len=n, out_dtype=F32)
    pec.check_status()
    check(o, lse, q4.attend(q, cache, [0, n], [800]), BF16, cache, [800], 4 * n, f"values by {step}")


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 40])
@pytest.mark.parametrize("n", [1, 50])
def test_queries_of_other_magnitudes(pec, n, size):
    cache = q4.make_cache(95, [900], 16, 2, DEV, size=1 / size)
    q = queries(96, n, 8, BF16) * size
    q[..., 3] *= 1e-3
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([900]), max_q_len=n)
    pec.check_status()
    check(o, lse, q4.attend(q, cache, [0, n], [900]), BF16, cache, [900], 4 * n, f"queries of {size}")


def test_zero_heads_and_queries(pec):
    """Keys, values and queries of zeros only: means of the values, masked rows as ever."""
    for n in (3, 60):
        kp, ks, vp, vs, table = cache = q4.make_cache(97, [n + 100], 16, 1, DEV)
        first = table[0, :(n + 100) // 16].tolist()                # (whole pages of the request)
        kp[first], ks[first] = 0, 2.0 ** -100
        q = queries(98, n, 4, BF16)
        q[::2] = 0
        o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([n + 100]), max_q_len=n)
        pec.check_status()
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()
        check(o, lse, q4.attend(q, cache, [0, n], [n + 100]), BF16, cache, [n + 100], 4 * n, f"zeros, {n} tokens")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_request_that_is_not_finite_spoils_no_other(pec, dtype):
    n, kv, page = [1, 1, 140, 3], [300, 200, 400, 90], 16
    kp, ks, vp, vs, table = q4.make_cache(21, kv, page, 2, DEV)
    clean = q4.make_cache(21, kv, page, 2, DEV)
    cu = ref.offsets(n)
    q = queries(22, cu[-1], 8, dtype)
    for b in (0, 2):
        ks[int(table[b, 3]), 2] = float("nan")
        vs[int(table[b, 5]), 7] = float("nan")
    o, lse = pec.pec_paged_attn_q4(q, kp, ks, vp, vs, table, dev(cu), dev(kv), max_q_len=140)
    pec.check_status()
    want = q4.attend(q, clean, cu, kv)
    for s, e in ((1, 2), (cu[3], cu[4])):
        check(o[s:e], lse[s:e], [x[s:e] for x in want], dtype, clean, kv, 16 if dtype == F32 else 12, "a neighbour of a request that is not finite")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(1, 100), (3, 100), (20, 100), (1, 3000), (20, 3000), (200, 3000)])
def test_rows_that_see_a_key_that_is_not_finite_say_so(pec, dtype, n, kv):
    """That is not "sees no key" (0 and -inf).  The rows before the key do not see it and keep their values."""
    kp, ks, vp, vs, table = cache = q4.make_cache(22, [kv], 16, 2, DEV)
    q = queries(23, n, 8, dtype)
    want = q4.attend(q, cache, [0, n], [kv])
    at = kv - (n + 1) // 2
    ks[int(table[0, at // 16]), at % 16] = float("nan")
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([kv]), max_q_len=n)
    pec.check_status()
    sees = n - (kv - at)
    assert torch.isnan(o[sees:]).all() and torch.isnan(lse[sees:]).all()
    check(o[:sees], lse[:sees], [x[:sees] for x in want], dtype, cache, [kv], 4 * n, "rows before a key that is not finite")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(1, 100), (1, 40000), (4, 3000), (13, 3000), (200, 3000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_not_finite_stays_so(pec, dtype, n, kv, bad):
    """In every part of its keys and in their merge; the other rows of the same tile keep their values."""
    cache = q4.make_cache(24, [kv], 16, 2, DEV)
    q = queries(25, n, 8, dtype)
    q[n // 2, 3, 7] = bad
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([kv]), max_q_len=n)
    pec.check_status()
    assert torch.isnan(o[n // 2, 3]).all() and torch.isnan(lse[n // 2, 3])
    q[n // 2, 3, 7] = 0
    want = q4.attend(q, cache, [0, n], [kv])
    want[1][n // 2, 3] = want[0][n // 2, 3] = np.nan
    check(o, lse, want, dtype, cache, [kv], 4 * n, f"beside a query of {bad}, {n} of {kv}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 40])
def test_a_value_that_is_not_finite_reaches_the_rows_that_see_it(pec, dtype, n):
    kp, ks, vp, vs, table = cache = q4.make_cache(26, [200], 16, 2, DEV)
    q = queries(27, n, 8, dtype)
    vs[int(table[0, 2]), 5, 1] = float("nan")
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev([0, n]), dev([200]), max_q_len=n)
    pec.check_status()
    assert torch.isnan(o[:, 4:]).all() and torch.isfinite(o[:, :4]).all() and torch.isfinite(lse).all()


# ------------------------------------------------------------------------------------------ refusals
def test_the_binding_refuses_what_the_library_cannot_see(pec):
    kp, ks, vp, vs, table = q4.make_cache(1, [20, 20], 16, 2, DEV, wild=False)
    q, k = torch.zeros((2, 4, 128), dtype=BF16, device=DEV), torch.zeros((2, 2, 128), dtype=BF16, device=DEV)
    cu, kv = dev([0, 1, 2]), dev([20, 20])
    cache = dict(k_pages=kp, k_scales=ks, v_pages=vp, v_scales=vs, block_table=table, cu_q=cu, kv_lens=kv)
    shared = [dict(k_pages=kp.cpu()), dict(v_pages=vp[:-1]), dict(k_pages=kp[..., :32]), dict(k_scales=ks.cpu()), dict(v_scales=vs[:-1]), dict(v_scales=vs[:, :, :1]),
              dict(block_table=table.long()), dict(block_table=table[:1]), dict(cu_q=cu[:2]), dict(cu_q=cu.float()), dict(kv_lens=kv.cpu())]
    for over in shared + [dict(q=q.cpu()), dict(q=q[0]), dict(q=q[..., :64]), dict(o=torch.zeros((2, 4, 64), dtype=BF16, device=DEV)),
                          dict(lse=torch.zeros((2, 4), dtype=BF16, device=DEV)), dict(max_q_len=-1), dict(workspace=torch.zeros(64, dtype=torch.uint8))]:
        with pytest.raises((ValueError, TypeError)):
            pec.pec_paged_attn_q4(**{**cache, "q": q, **over})
    for over in shared + [dict(k=k.cpu()), dict(v=k[:1]), dict(k=k.half()), dict(k=k[..., :64]), dict(v=k.float())]:
        with pytest.raises((ValueError, TypeError)):
            pec.pec_kv_append_q4(**{**cache, "k": k, "v": k, **over})
    for over in shared + [dict(tokens=-1), dict(dtype=torch.float16), dict(k_out=k[:1]), dict(v_out=k.float())]:
        with pytest.raises((ValueError, TypeError)):
            pec.pec_kv_read_q4(**{**cache, "tokens": 2, **over})
    pec.check_status()
