"""The paged serving calls on the GPU against 64-bit references: head norm with rotation, cache append, paged attention, and a
serving step made of them."""
import ctypes

import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2409_15104_b200 import binding, workloads

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 500000.0
BF16, F32 = torch.bfloat16, torch.float32


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------ norm and rotation
def check_heads(got, x, weight, positions, dtype, norm, turn, skip=(), before=None):
    want, size = ref.norm_rope(x, weight, 1e-6, positions, THETA, norm, turn)
    off = np.abs(got.double().cpu().numpy() - want)
    bound = ref.norm_rope_bound(want, size, dtype) + 1e-37
    keep = [t for t in range(x.shape[0]) if t not in skip]
    assert (off[keep] <= bound[keep]).all(), float((off / bound)[keep].max())
    for t in skip:
        assert torch.equal(got[t], before[t])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,hq,hkv", [(1, 1, 1), (1, 32, 8), (3, 5, 1), (64, 32, 8), (257, 7, 7), (1000, 64, 8), (5, 100, 3), (2048, 2, 1)])
@pytest.mark.parametrize("norm,turn", [(True, True), (False, True), (True, False)])
def test_norm_rope(pec, dtype, T, hq, hkv, norm, turn):
    n_pos = 200000
    tables = pec.pec_rope_table(THETA, n_pos, DEV) if turn else None
    g = torch.Generator().manual_seed(T * 100 + hq)
    qkv = torch.randn((T, hq + 2 * hkv, 128), generator=g).to(dtype).to(DEV)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    qw, kw = [(1 + 0.2 * torch.randn(128, generator=g)).to(dtype).to(DEV) for _ in range(2)] if norm else (None, None)
    pos = torch.randint(0, n_pos, (T,), generator=g).int()
    skip = [t for t in range(T) if t % 7 == 5]
    pos[skip] = -1
    qo = torch.full((T, hq, 128), 7.0, dtype=dtype, device=DEV)
    ko = torch.full((T, hkv, 128), 7.0, dtype=dtype, device=DEV)
    before = qkv.clone()
    pec.pec_qk_norm_rope(q, k, norm=norm, q_weight=qw, k_weight=kw, tables=tables, positions=pos.to(DEV), q_out=qo, k_out=ko)
    pec.check_status()
    seven = torch.full((T, 128, 128), 7.0, dtype=dtype, device=DEV)
    p = pos.clamp(min=0).numpy()
    check_heads(qo, q, qw, p, dtype, norm, turn, skip, seven[:, :hq])
    check_heads(ko, k, kw, p, dtype, norm, turn, skip, seven[:, :hkv])
    assert torch.equal(qkv, before)
    # in place, on slices of the fused tensor: the same bits, and the value columns as they were
    pec.pec_qk_norm_rope(q, k, norm=norm, q_weight=qw, k_weight=kw, tables=tables, positions=pos.to(DEV), inplace=True)
    keep = [t for t in range(T) if t not in skip]
    assert torch.equal(q[keep], qo[keep]) and torch.equal(k[keep], ko[keep])
    assert torch.equal(qkv[:, hq + hkv:], before[:, hq + hkv:]) and torch.equal(qkv[skip], before[skip])


def test_norm_rope_of_queries_alone_at_a_chunks_positions(pec):
    tables = pec.pec_rope_table(THETA, 5000, DEV)
    q = torch.randn((100, 6, 128), device=DEV)
    out, none = pec.pec_qk_norm_rope(q, norm=False, tables=tables, pos0=4900)
    assert none is None
    check_heads(out, q, None, np.arange(4900, 5000), F32, False, True)
    with pytest.raises(binding.PecError):
        pec.pec_qk_norm_rope(q, norm=False, tables=tables, pos0=4901)


def test_norm_rope_extreme_values(pec):
    """Zero heads stay zero; large and tiny magnitudes are normalised; a head that is not finite spoils no other."""
    x = torch.randn((6, 2, 128), device=DEV).to(BF16)
    x[0] = 0
    x[1] *= 1e15
    x[2] *= 1e-15
    x[3, 0, 5] = float("nan")
    x[4, 1, 77] = float("inf")
    out, _ = pec.pec_qk_norm_rope(x, tables=pec.pec_rope_table(THETA, 64, DEV), pos0=3)
    assert (out[0] == 0).all() and torch.isnan(out[3, 0]).all()
    for t, h in [(1, 0), (2, 1), (3, 1), (4, 0), (5, 0)]:
        check_heads(out[t:t + 1, h:h + 1], x[t:t + 1, h:h + 1], None, [3 + t], BF16, True, True)


def test_norm_rope_reports_positions_past_the_table(pec):
    tables = pec.pec_rope_table(THETA, 100, DEV)
    q = torch.randn((4, 2, 128), device=DEV)
    out = torch.full_like(q, 7.0)
    pec.pec_qk_norm_rope(q, tables=tables, positions=dev([3, 100, 99, 2 ** 31 - 1]), q_out=out)
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
    assert (out[[1, 3]] == 7.0).all() and not (out[[0, 2]] == 7.0).any()
    pec.check_status()


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,kv,page,hkv,head_major", [
    ([1], [1], 16, 1, False), ([1] * 40, list(range(1, 41)), 16, 8, False), ([5, 0, 1, 33, 0], [5, 9, 64, 100, 0], 24, 3, True),
    ([200, 3], [200, 130], 128, 2, False), ([1] * 33 + [70], [17 * (i % 9) + 1 for i in range(33)] + [1000], 8, 4, True),
])
@pytest.mark.parametrize("norm,turn", [(False, True), (True, True), (False, False)])
def test_append(pec, dtype, n, kv, page, hkv, head_major, norm, turn):
    kp, vp, table = ref.make_cache(11, kv, page, hkv, dtype, DEV, head_major, poison=False)
    k0, v0 = kp.clone(), vp.clone()
    cu = ref.offsets(n)
    T = cu[-1] + 3                                                # three rows of padding
    g = torch.Generator().manual_seed(7)
    kvs = torch.randn((T, 2 * hkv, 128), generator=g).to(dtype).to(DEV)
    k, v = kvs[:, :hkv], kvs[:, hkv:]
    w = (1 + 0.2 * torch.randn(128, generator=g)).to(dtype).to(DEV) if norm else None
    tables = pec.pec_rope_table(THETA, 2000, DEV) if turn else None
    pec.pec_kv_append(k, v, kp, vp, table, dev(cu), dev(kv), norm=norm, k_weight=w, tables=tables)
    pec.check_status()
    seen = torch.zeros(kp.shape[:2], dtype=torch.bool, device=DEV)
    for b in range(len(n)):
        for i in range(n[b]):
            pos, t = kv[b] - n[b] + i, cu[b] + i
            pg, slot = int(table[b, pos // page]), pos % page
            seen[pg, slot] = True
            assert torch.equal(vp[pg, slot], v[t])
            if norm or turn:
                check_heads(kp[pg, slot][None], k[t:t + 1], w, [pos], dtype, norm, turn)
            else:
                assert torch.equal(kp[pg, slot], k[t])
    assert torch.equal(kp[~seen], k0[~seen]) and torch.equal(vp[~seen], v0[~seen])


def test_append_reports_what_is_out_of_range_and_stores_the_rest(pec):
    page, hkv = 16, 2
    kp, vp, table = ref.make_cache(12, [40, 40, 40, 40], page, hkv, F32, DEV, poison=False)
    k0 = kp.clone()
    table[1, 2] = kp.shape[0]                                     # one page past the cache
    table[2, 2] = -1
    k, v = torch.randn((4, hkv, 128), device=DEV), torch.randn((4, hkv, 128), device=DEV)
    kv = dev([40, 40, 40, 4000])                                  # the last one's position is past its row of the table
    pec.pec_kv_append(k, v, kp, vp, table, dev([0, 1, 2, 3, 4]), kv)
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
    at = (int(table[0, 2]), 39 % page)
    assert torch.equal(kp[at], k[0])
    k0[at] = k[0]
    assert torch.equal(kp, k0)
    for cu, lens in (([0, 3, 1, 4, 4], [40] * 4), ([0, 1, 2, 3, 9], [40] * 4), ([0, 4, 4, 4, 4], [2, 1, 1, 1])):
        pec.pec_kv_append(k, v, kp, vp, table.clamp(0, kp.shape[0] - 1), dev(cu), dev(lens))
        with pytest.raises(binding.PecError):
            pec.check_status()


# ------------------------------------------------------------------------------------------ attention
def attend(pec, seed, n, kv, hq, hkv, page, dtype, *, head_major=False, causal=True, out_dtype=None, pad=0, fused=False, known=True,
           scale=0.0, what=""):
    kp, vp, table = ref.make_cache(seed, kv, page, hkv, dtype, DEV, head_major)
    cu = ref.offsets(n)
    T = cu[-1] + pad
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((T, hq + (2 if fused else 0), 128), generator=g).to(dtype).to(DEV)[:, :hq]
    out_dtype = dtype if out_dtype is None else out_dtype
    o = torch.full((T, hq, 128), 7.0, dtype=out_dtype, device=DEV)
    lse = torch.full((T, hq), 7.0, device=DEV)
    call = lambda: pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev(kv), max_q_len=max(n) if known else 0, causal=causal, softmax_scale=scale, o=o, lse=lse)
    call()
    pec.check_status()
    want = ref.attend(q, kp, vp, table, cu, kv, causal, scale or None)
    if pad:
        assert (o[cu[-1]:] == 7.0).all() and (lse[cu[-1]:] == 7.0).all(), "padding rows were written"
    ref.check_attend(o, lse, want, dtype, what)
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
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_paged_attention(pec, dtype, i):
    n, kv, hq, hkv, page = SHAPES[i]
    attend(pec, 100 + i, n, kv, hq, hkv, page, dtype, head_major=i % 2 == 1, pad=i % 3, fused=i % 2 == 0, known=i % 4 != 3,
           what=f"{n} of {kv}, {hq}/{hkv} heads, pages of {page}"[:120])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("i", [1, 3, 5, 6, 12, 17, 26, 28, 31])
def test_paged_attention_without_the_causal_mask(pec, dtype, i):
    n, kv, hq, hkv, page = SHAPES[i]
    attend(pec, 300 + i, n, kv, hq, hkv, page, dtype, causal=False, what=f"not causal, {n} of {kv}"[:100])


@pytest.mark.parametrize("i", [2, 8, 16, 18, 24, 28, 30, 31])
def test_paged_attention_fp32_output_and_scale(pec, i):
    n, kv, hq, hkv, page = SHAPES[i]
    attend(pec, 400 + i, n, kv, hq, hkv, page, BF16, out_dtype=F32, scale=0.3, what=f"fp32 output, {n} of {kv}"[:100])


@pytest.mark.parametrize("seed", range(12))
def test_paged_attention_random_batches(pec, seed):
    r = np.random.RandomState(seed)
    g, hkv = int(r.choice([1, 2, 3, 4, 5, 7, 8, 16])), int(r.choice([1, 2, 4]))
    B = int(r.randint(1, 20))
    n = [int(x) for x in r.choice([0, 1, 1, 1, 2, 7, 40, 150], B)]
    if sum(n) == 0:
        n[0] = 1
    kv = [int(m + r.choice([0, 1, 5, 127, 128, 400, 2000])) for m in n]
    attend(pec, 500 + seed, n, kv, g * hkv, hkv, 8 * int(r.randint(1, 33)), BF16 if seed % 3 else F32, head_major=bool(r.randint(2)),
           pad=int(r.randint(4)), known=bool(r.randint(2)), what=f"random {seed}")


def test_moving_maxima_and_large_scores(pec):
    """Scores that grow along the keys move the running maximum in every tile; scores near +-1e4 stay exact enough."""
    for dtype in (F32, BF16):
        for n in (1, 130):
            kp, vp, table = ref.make_cache(9, [1500], 16, 1, dtype, DEV)
            q = torch.randn((n, 4, 128), device=DEV).to(dtype)
            ids = table[0, :94].long()
            ramp = torch.linspace(0.1, 40.0, 94 * 16, device=DEV).view(94, 16, 1, 1)
            kp[ids] = (kp[ids].float() * ramp).to(dtype)
            o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([1500]), max_q_len=n)
            pec.check_status()
            ref.check_attend(o, lse, ref.attend(q, kp, vp, table, [0, n], [1500]), dtype, f"ramp {dtype} {n}")


def test_a_request_that_is_not_finite_spoils_no_other(pec):
    for dtype in (F32, BF16):
        n, kv, page = [1, 1, 140, 3], [300, 200, 400, 90], 16
        kp, vp, table = ref.make_cache(21, kv, page, 2, dtype, DEV)
        clean = ref.make_cache(21, kv, page, 2, dtype, DEV)
        cu = ref.offsets(n)
        q = torch.randn((cu[-1], 8, 128), device=DEV).to(dtype)
        for b in (0, 2):
            kp[table[b, 3].long(), 2] = float("inf")
            vp[table[b, 5].long(), 7] = float("nan")
        o, lse = pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev(kv), max_q_len=140)
        pec.check_status()
        want = ref.attend(q, *clean, cu, kv)
        for s, e in ((1, 2), (cu[3], cu[4])):
            ref.check_attend(o[s:e], lse[s:e], [x[s:e] for x in want], dtype, "a neighbour of a request that is not finite")


def test_bad_tables_are_reported(pec):
    for dtype in (F32, BF16):
        for n in (1, 200):
            kp, vp, table = ref.make_cache(13, [300], 16, 1, dtype, DEV, poison=False, wild=False)
            q = torch.randn((n, 2, 128), device=DEV).to(dtype)
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
                pec.pec_paged_attn(q, kp, vp, t, dev(cu), dev(kv), max_q_len=most)
                with pytest.raises(binding.PecError) as e:
                    pec.check_status()
                assert e.value.code == binding.PEC_ERR_BAD_INDEX
            o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([300]), max_q_len=n)
            pec.check_status()
            ref.check_attend(o, lse, ref.attend(q, kp, vp, table, [0, n], [300]), dtype, "after bad tables")


def test_pages_beyond_32_bits_of_elements(pec):
    """Pages whose offsets pass 2^32 elements: append and attend at the far end of a 10 GB cache."""
    page, hkv = 64, 8
    num = (1 << 32) // (page * hkv * 128) + 50
    kp = torch.empty((num, page, hkv, 128), dtype=BF16, device=DEV)
    vp = torch.empty((num, page, hkv, 128), dtype=BF16, device=DEV)
    for n, kv in ((1, 100), (170, 250)):
        table = dev([[num - 1, num - 7, num - 3, num - 20, 0]])
        kp[-40:].normal_()
        vp[-40:].normal_()
        k, v, q = (torch.randn((n, h, 128), device=DEV).to(BF16) for h in (hkv, hkv, 16))
        pec.pec_kv_append(k, v, kp, vp, table, dev([0, n]), dev([kv]))
        o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([kv]), max_q_len=n)
        pec.check_status()
        small_k, small_v, small_t = kp[-40:], vp[-40:], table.clone()
        small_t[0, :4] -= num - 40
        at = kv - 1
        assert torch.equal(small_k[small_t[0, at // page].long(), at % page], k[-1])
        ref.check_attend(o, lse, ref.attend(q, small_k, small_v, small_t, [0, n], [kv]), BF16, f"far pages {n}")
    del kp, vp
    torch.cuda.empty_cache()


def test_streams_graphs_and_a_shared_workspace(pec):
    """A step captured on one stream and replayed after the tables and inputs have changed; two graphs that share a workspace
    and run one after the other; an eager call on a stream of its own."""
    page, hkv, hq = 16, 2, 8
    binding.status_word(torch.device(DEV))
    kp, vp, table = ref.make_cache(31, [900, 400, 333], page, hkv, BF16, DEV, poison=False, wild=False)
    tables = pec.pec_rope_table(THETA, 4000, DEV)
    steps = []
    for n in ([1, 1, 1], [40, 1, 150]):
        cu, kv = dev(ref.offsets(n)), dev([900, 400, 333])
        T = sum(n)
        q, k, v = (torch.randn((T, h, 128), device=DEV).to(BF16) for h in (hq, hkv, hkv))
        o, lse = torch.empty((T, hq, 128), dtype=BF16, device=DEV), torch.empty((T, hq), device=DEV)
        steps.append(dict(n=n, cu=cu, kv=kv, q=q, k=k, v=v, o=o, lse=lse))
    ws = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)

    def issue(s):
        qr, _ = pec.pec_qk_norm_rope(s["q"], norm=True, tables=tables, positions=s["pos"])
        pec.pec_kv_append(s["k"], s["v"], kp, vp, table, s["cu"], s["kv"], norm=True, tables=tables)
        pec.pec_paged_attn(qr, kp, vp, table, s["cu"], s["kv"], max_q_len=max(s["n"]), o=s["o"], lse=s["lse"], workspace=ws)

    def positions(n, kv):
        return [kv[b] - n[b] + i for b in range(len(n)) for i in range(n[b])]

    graphs = []
    for s in steps:
        s["pos"] = dev(positions(s["n"], [900, 400, 333]))
        issue(s)                                                  # warm up outside the capture
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            issue(s)
        graphs.append(g)
    for lens in ([900, 400, 333], [700, 123, 208]):
        for s in steps:
            s["kv"].copy_(dev(lens))
            s["pos"].copy_(dev(positions(s["n"], lens)))
            s["q"].normal_()
        for s, g in zip(steps, graphs):
            g.replay()
            pec.check_status()
            got = s["o"].clone(), s["lse"].clone()
            qr, _ = pec.pec_qk_norm_rope(s["q"], tables=tables, positions=s["pos"])
            ref.check_attend(*got, ref.attend(qr, kp, vp, table, s["cu"].tolist(), lens), BF16, f"replayed {lens}")
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            o, lse = pec.pec_paged_attn(qr, kp, vp, table, s["cu"], s["kv"], max_q_len=max(s["n"]), stream=side)
            side.synchronize()
            assert torch.equal(o, got[0]) and torch.equal(lse, got[1])


def test_a_serving_step_against_the_prefill_path(pec):
    """A prompt fed as chunks, then single tokens, through projection, norm and rotation, append and paged attention; the
    result of the last rows against pec_prefill_attn over the whole request's contiguous q, k, v."""
    hq, hkv, page, S, width = 8, 2, 16, 700, 512
    torch.manual_seed(3)
    x = (torch.randn((S, width), device=DEV) / 4).to(BF16)
    w = (torch.randn(((hq + 2 * hkv) * 128, width), device=DEV) / 16).to(BF16)
    qw, kw = [(1 + 0.1 * torch.randn(128, device=DEV)).to(BF16) for _ in range(2)]
    tables = pec.pec_rope_table(THETA, 1024, DEV)
    num = -(-S // page) + 1
    kp, vp = [torch.full((num, page, hkv, 128), float("nan"), dtype=BF16, device=DEV) for _ in range(2)]
    table = torch.randperm(num, device=DEV)[None, :num - 1].int()
    whole = pec.pec_linear(x, w).view(S, hq + 2 * hkv, 128)
    q_all, k_all = pec.pec_qk_norm_rope(whole[:, :hq], whole[:, hq:hq + hkv], q_weight=qw, k_weight=kw, tables=tables)
    want_o, want_l = pec.pec_prefill_attn(q_all, k_all, whole[:, hq + hkv:], out_dtype=BF16)
    at = 0
    for n in (300, 1, 37, 256, 5, 1, 100):
        qkv = pec.pec_linear(x[at:at + n], w).view(n, hq + 2 * hkv, 128)
        at += n
        q, _ = pec.pec_qk_norm_rope(qkv[:, :hq], q_weight=qw, tables=tables, pos0=at - n)
        pec.pec_kv_append(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], kp, vp, table, dev([0, n]), dev([at]), norm=True, k_weight=kw, tables=tables)
        o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([at]), max_q_len=n)
        pec.check_status()
        assert torch.equal(q, q_all[at - n:at])
        # two roundings of o to bf16 and two of p: the values are averages of |v| of order 1
        assert (o.float() - want_o[at - n:at].float()).abs().max() <= 4 * 2.0 ** -8 * whole.float().abs().max()
        assert (lse - want_l[at - n:at]).abs().max() <= 1e-4
        ref.check_attend(o, lse, ref.attend(q, kp, vp, table, [0, n], [at]), BF16, f"step of {n} at {at}")
    assert at == S


def test_calls_without_tokens(pec):
    kp, vp, table = ref.make_cache(1, [20], 16, 2, BF16, DEV)
    none = torch.empty((0, 4, 128), dtype=BF16, device=DEV)
    o, lse = pec.pec_paged_attn(none, kp, vp, table, dev([0, 0]), dev([20]))
    assert o.shape == (0, 4, 128) and lse.shape == (0, 4)
    pec.pec_kv_append(none[:, :2], none[:, :2], kp, vp, table, dev([0, 0]), dev([20]))
    pec.pec_qk_norm_rope(none)
    q = torch.full((3, 4, 128), 1.0, dtype=BF16, device=DEV)       # padding alone
    o = torch.full_like(q, 7.0)
    pec.pec_paged_attn(q, kp, vp, table, dev([0, 0]), dev([20]), o=o)
    pec.check_status()
    assert (o == 7.0).all()


def test_a_request_per_row_of_a_large_batch(pec):
    """More requests than a warp, a plan group (256) or a block looks at once, of both classes, some empty, with room before the
    first and after the last row."""
    g = np.random.RandomState(4)
    for B, pick in ((1500, [0, 1, 1, 2]), (300, [0, 1, 130, 200])):
        n = [int(x) for x in g.choice(pick, B)]
        kv = [m + int(x) for m, x in zip(n, g.choice([0, 1, 30, 200], B))]
        kp, vp, table = ref.make_cache(B, kv, 16, 1, BF16, DEV)
        cu = [c + 3 for c in ref.offsets(n)]                          # three rows that belong to no request
        T = cu[-1] + 2
        q = torch.randn((T, 1, 128), device=DEV).to(BF16)
        o, lse = torch.full((T, 1, 128), 7.0, dtype=BF16, device=DEV), torch.full((T, 1), 7.0, device=DEV)
        pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev(kv), o=o, lse=lse)
        pec.check_status()
        for rows in (slice(0, 3), slice(cu[-1], T)):
            assert (o[rows] == 7.0).all() and (lse[rows] == 7.0).all()
        ref.check_attend(o, lse, ref.attend(q, kp, vp, table, cu, kv), BF16, f"{B} requests")
        k, v = torch.randn((T, 1, 128), device=DEV).to(BF16), torch.randn((T, 1, 128), device=DEV).to(BF16)
        pec.pec_kv_append(k, v, kp, vp, table, dev(cu), dev(kv))
        pec.check_status()
        last = [b for b in range(B) if n[b]][-1]
        assert torch.equal(kp[int(table[last, (kv[last] - 1) // 16]), (kv[last] - 1) % 16], k[cu[last + 1] - 1])


def test_two_calls_at_once(pec):
    """Two batches on two streams with workspaces of their own, many times: the same bits as one after the other."""
    cases = []
    for seed, n, kv in ((51, [1] * 20, [700 + 31 * i for i in range(20)]), (52, [200, 1, 70], [900, 4000, 70])):
        kp, vp, table = ref.make_cache(seed, kv, 16, 2, BF16, DEV)
        q = torch.randn((sum(n), 8, 128), device=DEV).to(BF16)
        args = (q, kp, vp, table, dev(ref.offsets(n)), dev(kv))
        cases.append((args, max(n), pec.pec_paged_attn(*args, max_q_len=max(n))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        got = [pec.pec_paged_attn(*args, max_q_len=most, stream=s) for (args, most, _), s in zip(cases, streams)]
        torch.cuda.synchronize()
        for (_, _, want), have in zip(cases, got):
            assert torch.equal(want[0], have[0]) and torch.equal(want[1], have[1])
    pec.check_status()


def test_requests_that_share_pages(pec):
    """A common prefix in the same pages of two requests, each with its own last page."""
    kp, vp, table = ref.make_cache(61, [333, 333], 16, 2, BF16, DEV)
    table[1, :20] = table[0, :20]
    for n in ([1, 1], [100, 13]):
        q = torch.randn((sum(n), 8, 128), device=DEV).to(BF16)
        cu = ref.offsets(n)
        o, lse = pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev([333, 333]), max_q_len=max(n))
        pec.check_status()
        ref.check_attend(o, lse, ref.attend(q, kp, vp, table, cu, [333, 333]), BF16, f"shared pages {n}")


@pytest.mark.parametrize("page,total", [(1024, 5000), (65536, 70000), (512, 512), (8, 3000)])
def test_page_sizes_and_a_cache_of_one_page(pec, page, total):
    for n in (1, 140):
        attend(pec, page + n, [n], [total], 4, 1, page, BF16, known=n == 1, what=f"pages of {page}, {n} new")


def _other_order(pages, order):
    """The same pages [P, page, Hkv, 128] behind other strides; what lies between them is NaN."""
    P, page, hkv, d = pages.shape
    if order == "heads first":
        return pages.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    if order == "between a token's others":
        full = torch.full((P, page, hkv, 2, d), float("nan"), dtype=pages.dtype, device=DEV)
        full[:, :, :, 1] = pages
        return full[:, :, :, 1]
    if order == "a layer's pages":
        full = torch.full((P, 3, page, hkv, d), float("nan"), dtype=pages.dtype, device=DEV)
        full[:, 1] = pages
        return full[:, 1]
    st = hkv * 136 + 8                                             # strides whose greatest common divisor is 8 elements
    full = torch.full((P * (page * st + 24),), float("nan"), dtype=pages.dtype, device=DEV)
    out = full.as_strided(pages.shape, (page * st + 24, st, 136, 1))
    out.copy_(pages)
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k_order,v_order", [("heads first", "heads first"), ("between a token's others", "a layer's pages"),
                                             ("a layer's pages", "odd strides"), ("odd strides", "heads first")])
@pytest.mark.parametrize("n,kv,hq,hkv,page", [([1, 1, 1], [700, 130, 33], 8, 2, 16), ([3, 20], [900, 260], 6, 3, 24),
                                              ([200, 1], [500, 300], 8, 1, 64), ([1], [200], 4, 4, 256)])
def test_orders_of_the_cache(pec, dtype, k_order, v_order, n, kv, hq, hkv, page):
    kp, vp, table = ref.make_cache(71, kv, page, hkv, dtype, DEV)
    cu = ref.offsets(n)
    q = torch.randn((cu[-1], hq, 128), generator=torch.Generator().manual_seed(72)).to(dtype).to(DEV)
    plain = pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev(kv), max_q_len=max(n))
    o, lse = pec.pec_paged_attn(q, _other_order(kp, k_order), _other_order(vp, v_order), table, dev(cu), dev(kv), max_q_len=max(n))
    pec.check_status()
    ref.check_attend(o, lse, ref.attend(q, kp, vp, table, cu, kv), dtype, f"{k_order}, {v_order}")
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1]), "the order of the cache changed bits"


def test_partials_of_two_caches_merge(pec):
    """A long request's cache on two holders (Section 5.2): the new token's fp32 partials over either part, merged."""
    kp, vp, table = ref.make_cache(71, [900, 500], 16, 2, BF16, DEV)
    q = torch.randn((1, 8, 128), device=DEV).to(BF16)
    parts = []
    for b, kv in ((0, 900), (1, 500)):
        parts.append(pec.pec_paged_attn(q, kp, vp, table[b:b + 1], dev([0, 1]), dev([kv]), max_q_len=1, causal=False, out_dtype=F32))
    o, lse = pec.pec_attn_merge(*parts[0], *parts[1])
    pec.check_status()
    both = torch.cat([kp[table[0, :57].long()].reshape(-1, 2, 128)[:900], kp[table[1, :32].long()].reshape(-1, 2, 128)[:500]]).view(1, 1400, 2, 128)
    bothv = torch.cat([vp[table[0, :57].long()].reshape(-1, 2, 128)[:900], vp[table[1, :32].long()].reshape(-1, 2, 128)[:500]]).view(1, 1400, 2, 128)
    want = ref.attend(q, both, bothv, torch.zeros((1, 1), dtype=torch.int32), [0, 1], [1400])
    ref.check_attend(o, lse, want, BF16, "two partials merged")


@pytest.mark.parametrize("n,kv", [([1] * 40, [2500] * 40), ([300, 300], [2500, 2500])])
def test_a_wait_that_runs_out_is_reported(pec, n, kv):
    """The loader of each CTA leaves its last value tile out: the waits for it run out within the limit, the status word says so,
    and the next launch is right."""
    kp, vp, table = ref.make_cache(81, kv, 16, 2, BF16, DEV)
    q = torch.randn((sum(n), 8, 128), device=DEV).to(BF16)
    cu = ref.offsets(n)
    args = (q, kp, vp, table, dev(cu), dev(kv))
    try:
        pec.pec_control(binding.PEC_CTL_WAIT_LIMIT_CYCLES, 4_000_000)
        pec.pec_control(binding.PEC_CTL_TEST_SKIP_LAST_LOAD, 1)
        pec.pec_paged_attn(*args, max_q_len=max(n))
        with pytest.raises(binding.PecError) as e:
            pec.check_status()
        assert e.value.code == binding.PEC_ERR_TIMEOUT
    finally:
        pec.pec_control(binding.PEC_CTL_TEST_SKIP_LAST_LOAD, 0)
        pec.pec_control(binding.PEC_CTL_WAIT_LIMIT_CYCLES, 2_000_000_000)
    o, lse = pec.pec_paged_attn(*args, max_q_len=max(n))
    pec.check_status()
    ref.check_attend(o, lse, ref.attend(q, kp, vp, table, cu, kv), BF16, "after a wait that ran out")


@pytest.mark.parametrize("n,kv,hq,hkv", [([1], [3000], 8, 1), ([1] * 9, [5, 128, 700, 129, 1, 2000, 64, 300, 1111], 32, 8), ([2, 1, 2], [900, 40, 2], 16, 2),
                                         ([16], [333], 1, 1), ([5, 3], [4000, 3], 3, 1)])
def test_few_rows_keep_more_of_the_probabilities(pec, n, kv, hq, hkv):
    """At most 16 packed rows: p is the sum of two bf16 values, each rounded to half a step: 2^-8 of what the first left, 2^-16
    of p."""
    kp, vp, table = ref.make_cache(91, kv, 16, hkv, BF16, DEV)
    cu = ref.offsets(n)
    q = torch.randn((sum(n), hq, 128), device=DEV).to(BF16)
    o, lse = pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev(kv), max_q_len=max(n), out_dtype=F32)
    pec.check_status()
    ref.check_attend(o, lse, ref.attend(q, kp, vp, table, cu, kv), BF16, f"fp32 output, {n} of {kv}"[:100], p_error=2.0 ** -16)


def test_the_binding_refuses_what_the_library_cannot_see(pec):
    kp, vp, table = ref.make_cache(1, [20, 20], 16, 2, BF16, DEV, wild=False)
    q, k = torch.zeros((2, 4, 128), dtype=BF16, device=DEV), torch.zeros((2, 2, 128), dtype=BF16, device=DEV)
    cu, kv = dev([0, 1, 2]), dev([20, 20])
    wide = torch.zeros((2, 4, 256), dtype=BF16, device=DEV)[:, :, ::2]
    attn = dict(q=q, k_pages=kp, v_pages=vp, block_table=table, cu_q=cu, kv_lens=kv)
    for over in (dict(q=q.cpu()), dict(q=q[0]), dict(q=wide), dict(q=q[..., :64]), dict(k_pages=kp.float()), dict(v_pages=vp[:-1]), dict(k_pages=kp.cpu()),
                 dict(block_table=table.long()), dict(block_table=table[:1]), dict(cu_q=cu[:2]), dict(cu_q=cu.float()), dict(kv_lens=kv.cpu()),
                 dict(o=torch.zeros((2, 4, 64), dtype=BF16, device=DEV)), dict(o=torch.zeros_like(q), out_dtype=F32), dict(lse=torch.zeros((2, 4), dtype=BF16, device=DEV)),
                 dict(max_q_len=-1), dict(workspace=torch.zeros(64, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            pec.pec_paged_attn(**{**attn, **over})
    for over in (dict(q=q.half()), dict(k_pages=None), dict(out_dtype=torch.float16), dict(max_q_len="many")):
        with pytest.raises(TypeError):
            pec.pec_paged_attn(**{**attn, **over})
    with pytest.raises(binding.PecError) as e:
        pec.pec_paged_attn(**attn, workspace=torch.zeros(64, dtype=torch.uint8, device=DEV))
    assert e.value.code == -4
    append = dict(k=k, v=k, k_pages=kp, v_pages=vp, block_table=table, cu_q=cu, kv_lens=kv)
    w = torch.ones(128, dtype=BF16, device=DEV)
    for over in (dict(v=k[:1]), dict(k=q, v=q), dict(k_weight=w), dict(norm=True, k_weight=w[:64]), dict(norm=True, k_weight=w.float()),
                 dict(tables=(torch.zeros(100, device=DEV), 10)), dict(v=k.cpu())):
        with pytest.raises(ValueError):
            pec.pec_kv_append(**{**append, **over})
    for over in (dict(k=k[:1]), dict(positions=dev([1])), dict(positions=torch.zeros(2, device=DEV)), dict(q_out=k), dict(norm=False, q_weight=w)):
        with pytest.raises(ValueError):
            pec.pec_qk_norm_rope(**{**dict(q=q, k=k), **over})
    with pytest.raises(binding.PecError):
        pec.pec_qk_norm_rope(q, eps=0.0)
    pec.check_status()


def _chain(pec, hq, hkv, page, S, seed):
    """State and one step of a decode chain whose kernels follow each other without a pause: projection output -> norm and rotation ->
    append -> attention -> the next step's input."""
    torch.manual_seed(seed)
    num = -(-S // page)
    st = dict(kp=torch.zeros((num, page, hkv, 128), dtype=BF16, device=DEV), vp=torch.zeros((num, page, hkv, 128), dtype=BF16, device=DEV),
              ids=torch.randperm(num, device=DEV)[None].int(), cu=dev([0, 1]), kv=dev([0]), pos=dev([0]), tables=pec.pec_rope_table(THETA, S, DEV),
              x=torch.randn((1, hq * 128), device=DEV).to(BF16), w=(torch.randn(((hq + 2 * hkv) * 128, hq * 128), device=DEV) / 30).to(BF16))

    def step():
        st["kv"] += 1                                             # torch kernels, copies and a GEMM in between
        st["pos"].copy_(st["kv"])
        st["pos"] -= 1
        qkv = pec.pec_linear(st["x"], st["w"]).view(1, hq + 2 * hkv, 128)
        q, _ = pec.pec_qk_norm_rope(qkv[:, :hq], tables=st["tables"], positions=st["pos"])
        pec.pec_kv_append(qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], st["kp"], st["vp"], st["ids"], st["cu"], st["kv"], norm=True, tables=st["tables"])
        o, _ = pec.pec_paged_attn(q, st["kp"], st["vp"], st["ids"], st["cu"], st["kv"], max_q_len=1)
        st["x"].copy_(o.view(1, hq * 128))

    return st, step


def test_steps_without_a_pause_give_the_bits_of_steps_with_one(pec):
    """300 decode steps back to back, with a synchronisation after every kernel's step, and replayed from a graph."""
    ends = []
    for mode in ("paused", "flowing", "graph"):
        st, step = _chain(pec, 8, 2, 16, 400, 5)
        graph = None
        for i in range(300):
            if mode == "graph" and i == 10:
                graph = torch.cuda.CUDAGraph()
                kept = {k: st[k].clone() for k in ("kv", "pos", "x", "kp", "vp")}
                with torch.cuda.graph(graph):
                    step()
                for k, v in kept.items():
                    st[k].copy_(v)
            graph.replay() if graph else step()
            if mode == "paused":
                torch.cuda.synchronize()
        pec.check_status()
        assert int(st["kv"]) == 300
        ends.append((st["x"].clone(), st["kp"].clone(), st["vp"].clone()))
    for other in ends[1:]:
        assert all(torch.equal(a, b) for a, b in zip(ends[0], other))


def test_a_capture_with_other_nodes_and_a_fork(pec):
    """Captured behind copies, fills, torch kernels and a joined side stream; replays read what those nodes wrote."""
    binding.status_word(torch.device(DEV))
    kv = [700, 300]
    kp, vp, table = ref.make_cache(95, kv, 16, 2, BF16, DEV, poison=False, wild=False)
    for n in ([1, 1], [150, 2]):
        cu, lens, true_lens, src = dev(ref.offsets(n)), dev(kv), dev(kv), torch.randn((sum(n), 8, 128), device=DEV).to(BF16)
        q = torch.empty_like(src)
        o, lse = torch.empty_like(src), torch.empty(src.shape[:2], device=DEV)
        call = lambda: pec.pec_paged_attn(q, kp, vp, table, cu, lens, max_q_len=max(n), o=o, lse=lse)
        q.copy_(src)
        call()
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.graph(g):
            q.zero_()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                lens.fill_(0)
                lens.add_(true_lens)
            q.copy_(src)
            torch.cuda.current_stream().wait_stream(side)
            call()
        for _ in range(3):
            src.normal_()
            o.fill_(7.0)
            g.replay()
            pec.check_status()
            ref.check_attend(o, lse, ref.attend(src, kp, vp, table, cu.tolist(), kv), BF16, f"captured behind other nodes {n}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cu", [[0, 200] * 32 + [0], [200, 0] * 32 + [200], [0, 200, 200, 0] * 16 + [200]])
def test_overlapping_offsets_stay_inside_the_workspace(pec, dtype, cu):
    """Offsets that go back and forth: every second request is in order by itself, together they have many times the blocks of
    T tokens.  The workspace has exactly the size asked for; what lies around it is neither written nor merged into a result."""
    kp, vp, table = ref.make_cache(26, [1024] * 64, 128, 1, dtype, DEV)
    q = torch.randn((200, 1, 128), device=DEV).to(dtype)
    a = binding.pec_paged_args()
    a.q, a.k_pages, a.v_pages, a.block_table, a.cu_q, a.kv_lens, a.o, a.lse, a.status = [1 << 20] * 9
    a.q_stride_t = a.q_stride_h = a.k_pages_stride_h = a.v_pages_stride_h = a.k_pages_stride_t = a.v_pages_stride_t = 128
    a.k_pages_stride_p = a.v_pages_stride_p = 128 * 128
    a.dtype = a.o_dtype = binding.PEC_BF16 if dtype == BF16 else binding.PEC_F32
    a.page_size, a.num_pages, a.table_stride, a.max_pages, a.B, a.T = 128, kp.shape[0], table.shape[1], table.shape[1], 64, 200
    a.Hq, a.Hkv, a.D, a.causal = 1, 1, 128, 1
    need = binding.pec_paged_workspace_size(a)
    guard = 4 << 20
    room = torch.full(((need + 2 * guard) // 4 + 4,), 1000.0, device=DEV)
    bytes_ = room.view(torch.uint8)
    ws = bytes_[guard:guard + need]
    o, lse = torch.full((200, 1, 128), 7.0, dtype=dtype, device=DEV), torch.full((200, 1), 7.0, device=DEV)
    pec.pec_paged_attn(q, kp, vp, table, dev(cu), dev([1024] * 64), o=o, lse=lse, workspace=ws)
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
    assert (bytes_[:guard].view(torch.float32) == 1000.0).all() and (room[(guard + need + 3) // 4:] == 1000.0).all()
    assert o.float().abs().max() < 100 and lse.abs().max() < 100


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(1, 100), (20, 100), (1, 3000), (20, 3000), (200, 3000)])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_rows_that_see_a_key_that_is_not_finite_say_so(pec, dtype, n, kv, bad):
    """A NaN score, or one of +inf (exp(inf - inf)), makes a row's sum NaN: that is not "sees no key" (0 and -inf), in a request of
    one tile (kv = 100) as in one whose keys are cut (a part that were left out would give a plausible result).  The rows before
    the key do not see it and keep their values."""
    kp, vp, table = ref.make_cache(22, [kv], 16, 2, dtype, DEV)
    q = torch.randn((n, 8, 128), generator=torch.Generator().manual_seed(23))
    q[..., 5] = q[..., 5].abs() + 0.1                             # the score of a key with +inf there is +inf
    q = q.to(dtype).to(DEV)
    want = ref.attend(q, kp, vp, table, [0, n], [kv])
    at = kv - (n + 1) // 2
    kp[int(table[0, at // 16]), at % 16, :, 5] = float(bad)
    o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([kv]), max_q_len=n)
    pec.check_status()
    sees = n - (kv - at)
    assert not torch.isfinite(o[sees:]).any()
    assert not torch.isfinite(lse[sees:]).any() and not torch.isneginf(lse[sees:]).any()
    ref.check_attend(o[:sees], lse[:sees], [x[:sees] for x in want], dtype, f"rows before a key with {bad}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(1, 100), (1, 3000), (1, 40000), (13, 3000), (200, 3000)])
def test_a_query_that_is_not_finite_stays_so_when_its_parts_are_merged(pec, dtype, n, kv):
    """Every partial of such a row has a NaN for its LSE; the merge must not take that for parts without keys.  The other rows of
    the same tile keep their values."""
    kp, vp, table = ref.make_cache(24, [kv], 16, 2, dtype, DEV)
    q = torch.randn((n, 8, 128), generator=torch.Generator().manual_seed(25)).to(dtype).to(DEV)
    q[n // 2, 3, 7] = float("nan")
    o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([kv]), max_q_len=n)
    pec.check_status()
    assert torch.isnan(o[n // 2, 3]).all() and torch.isnan(lse[n // 2, 3])
    want = ref.attend(q, kp, vp, table, [0, n], [kv])
    assert np.isnan(want[1]).sum() == 1                           # that row's LSE: left out by the comparison
    ref.check_attend(o, lse, want, dtype, f"beside a query that is not finite, {n} of {kv}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("norm", [False, True])
def test_without_a_table_channels_do_not_meet(pec, dtype, norm):
    """No rotation: z = y.  What is not finite in channel i stays there (a rotation by zero would bring inf * 0 into channel
    i + 64 or i - 64), and without a norm the heads are copied."""
    x = torch.randn((5, 3, 128), generator=torch.Generator().manual_seed(8)).to(dtype).to(DEV)
    x[1, 0, 5], x[2, 1, 100], x[3, 2, 64], x[4, 0, 0] = float("inf"), float("-inf"), float("nan"), -0.0
    kp, vp, table = ref.make_cache(14, [5], 16, 3, dtype, DEV, poison=False)
    v = torch.randn((5, 3, 128), device=DEV).to(dtype)
    pec.pec_kv_append(x, v, kp, vp, table, dev([0, 5]), dev([5]), norm=norm)
    outs = [*pec.pec_qk_norm_rope(x, x.clone(), norm=norm), kp[int(table[0, 0]), :5]]
    pec.check_status()
    for out in outs:
        if not norm:
            assert torch.equal(out.isnan(), x.isnan())
            assert torch.equal(out.nan_to_num(nan=9.0), x.nan_to_num(nan=9.0)) and torch.equal(torch.signbit(out[4]), torch.signbit(x[4]))
            continue
        for t, h, c in ((1, 0, 5), (2, 1, 100)):                  # x / sqrt(inf): 0, and NaN where x is inf
            rest = [i for i in range(128) if i != c]
            assert torch.isnan(out[t, h, c]) and (out[t, h, rest] == 0).all()
        assert torch.isnan(out[3, 2]).all()
        for t in range(5):
            for h in range(3):
                if (t, h) not in ((1, 0), (2, 1), (3, 2)):
                    check_heads(out[t:t + 1, h:h + 1], x[t:t + 1, h:h + 1], None, [0], dtype, True, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("norm", [False, True])
def test_without_a_table_channels_do_not_meet(pec, dtype, norm):
    """No rotation: z = y.  What is not finite in channel i stays there (a rotation by zero would bring inf * 0 into channel
    i + 64 or i - 64), and without a norm the heads are copied."""
    x = torch.randn((5, 3, 128), generator=torch.Generator().manual_seed(8)).to(dtype).to(DEV)
    x[1, 0, 5], x[2, 1, 100], x[3, 2, 64], x[4, 0, 0] = float("inf"), float("-inf"), float("nan"), -0.0
    kp, vp, table = ref.make_cache(14, [5], 16, 3, dtype, DEV, poison=False)
    v = torch.randn((5, 3, 128), device=DEV).to(dtype)
    pec.pec_kv_append(x, v, kp, vp, table, dev([0, 5]), dev([5]), norm=norm)
    outs = [*pec.pec_qk_norm_rope(x, x.clone(), norm=norm), kp[int(table[0, 0]), :5]]
    pec.check_status()
    for out in outs:
        if not norm:
            assert torch.equal(out.isnan(), x.isnan())
            assert torch.equal(out.nan_to_num(nan=9.0), x.nan_to_num(nan=9.0)) and torch.equal(torch.signbit(out[4]), torch.signbit(x[4]))
            continue
        for t, h, c in ((1, 0, 5), (2, 1, 100)):                  # x / sqrt(inf): 0, and NaN where x is inf
            rest = [i for i in range(128) if i != c]
            assert torch.isnan(out[t, h, c]) and (out[t, h, rest] == 0).all()
        assert torch.isnan(out[3, 2]).all()
        for t in range(5):
            for h in range(3):
                if (t, h) not in ((1, 0), (2, 1), (3, 2)):
                    check_heads(out[t:t + 1, h:h + 1], x[t:t + 1, h:h + 1], None, [0], dtype, True, False)


def test_a_status_word_made_on_a_busy_stream_loses_no_report(pec, monkeypatch):
    """The device's word is zeroed on the stream of whoever asks first; a call on another stream may not run before that."""
    tables = pec.pec_rope_table(THETA, 100, DEV)
    q, at = torch.randn((1, 2, 128), device=DEV), dev([100])
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_status_words", {})
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                            # 0.2 s
        binding.status_word(DEV)
    pec.pec_qk_norm_rope(q, tables=tables, positions=at)          # a position past the table
    torch.cuda.synchronize()
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX


def test_check_status_waits_for_calls_on_other_streams(pec):
    tables = pec.pec_rope_table(THETA, 100, DEV)
    q, at = torch.randn((1, 2, 128), device=DEV), dev([100])
    pec.check_status()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)                            # 0.2 s
        pec.pec_qk_norm_rope(q, tables=tables, positions=at)      # a position past the table
    try:
        with pytest.raises(binding.PecError) as e:
            pec.check_status()
        assert e.value.code == binding.PEC_ERR_BAD_INDEX
    finally:
        torch.cuda.synchronize()
        binding.status_word(DEV).zero_()
    pec.check_status()


def test_a_dimension_past_32_bits_is_refused(pec):
    """A head dimension of 2^32 + 128 is not one of 128."""
    q = torch.empty((1, 1, (1 << 32) + 128), dtype=BF16, device=DEV)
    for args in ((q,), (q[..., :128], q)):
        with pytest.raises(ValueError):
            pec.pec_qk_norm_rope(*args, norm=False)
    del q
    torch.cuda.empty_cache()


def test_norm_rope_without_a_table_at_any_first_position(pec):
    """Positions pos0 + t past 2^63 are not padding."""
    q = torch.randn((20, 2, 128), device=DEV).to(BF16)
    out = torch.full_like(q, 7.0)
    pec.pec_qk_norm_rope(q, pos0=(1 << 63) - 1, q_out=out)
    pec.check_status()
    assert torch.equal(out, pec.pec_qk_norm_rope(q)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,hq", [(1, 4), (3, 16), (130, 4)])
def test_scores_of_ten_thousand(pec, dtype, n, hq):
    """Scores past +-1e4 in natural units (the narrow, the wide and the chunk form), where the maximum's subtraction and the LSE
    lose the most bits: the bound's score term grows with sum |q k| and covers them."""
    kp, vp, table = ref.make_cache(9, [1500], 16, 1, dtype, DEV)
    q = torch.randn((n, hq, 128), generator=torch.Generator().manual_seed(10)).to(dtype).to(DEV)
    ids = table[0, :94].long()
    ramp = torch.linspace(0.1, 40.0, 94 * 16, device=DEV).view(94, 16, 1, 1)
    kp[ids] = (kp[ids].float() * ramp).to(dtype)
    o, lse = pec.pec_paged_attn(q, kp, vp, table, dev([0, n]), dev([1500]), max_q_len=n, softmax_scale=20.0)
    pec.check_status()
    want = ref.attend(q, kp, vp, table, [0, n], [1500], scale=20.0)
    assert want[1].max() > 1e4
    ref.check_attend(o, lse, want, dtype, f"scores to {want[1].max():.0f}, {n} tokens")


def test_calls_on_another_stream_keep_their_tensors(pec):
    """Inputs of the current stream that are dropped as soon as the call returns, while the call's stream is still busy: their memory
    may not be handed out before the call has read it.  The same for a result that is dropped while the current stream reads it."""
    kp, vp, table = ref.make_cache(27, [600], 16, 2, BF16, DEV)
    q = torch.randn((64, 8, 128), device=DEV).to(BF16)
    tables = pec.pec_rope_table(THETA, 1000, DEV)
    want_h, _ = pec.pec_qk_norm_rope(q, tables=tables)
    want, want_l = pec.pec_paged_attn(q, kp, vp, table, dev([0, 64]), dev([600]), max_q_len=64)
    k2, v2 = kp.clone(), vp.clone()
    pec.pec_kv_append(q[:, :2], q[:, 2:4], k2, v2, table, dev([0, 64]), dev([600]), tables=tables)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    k3, v3 = kp.clone(), vp.clone()

    def overwrite():                                              # whatever small blocks are free now
        for _ in range(20):
            torch.full((64, 8, 128), 100.0, dtype=BF16, device=DEV)
            torch.full((64,), 99, dtype=torch.int32, device=DEV)

    for call in (lambda: pec.pec_qk_norm_rope(q.clone(), tables=tables, stream=side)[0],
                 lambda: pec.pec_paged_attn(q.clone(), kp, vp, table.clone(), dev([0, 64]), dev([600]), max_q_len=64, stream=side),
                 lambda: pec.pec_kv_append(q.clone()[:, :2], q.clone()[:, 2:4], k3, v3, table.clone(), dev([0, 64]), dev([600]), tables=tables, stream=side)):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)                        # 50 ms
        out = call()
        overwrite()
        torch.cuda.synchronize()
        if isinstance(out, tuple):
            assert torch.equal(out[0], want) and torch.equal(out[1], want_l)
        elif out is not None:
            assert torch.equal(out, want_h)
    assert torch.equal(k3.view(torch.int16), k2.view(torch.int16)) and torch.equal(v3.view(torch.int16), v2.view(torch.int16))
    # A result read by the current stream and dropped; the call's stream takes the next result's memory.
    out = pec.pec_qk_norm_rope(q, tables=tables, stream=side)[0]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(100_000_000)
    kept = out.clone()
    del out
    for _ in range(5):
        other = pec.pec_qk_norm_rope(q + 1, tables=tables, stream=side)[0]
        del other
    torch.cuda.synchronize()
    assert torch.equal(kept, want_h)
    pec.check_status()


@pytest.mark.parametrize("T,cu", [(8, [5, 3, 8]), (4, [0, 4, 9, 9]), (4, [0, 4, 100, 50]), (6, [0] * 40 + [6] * 40 + [2, 6]), (3, [0] + [3] * 700 + [1] + [3] * 20),
                                  (0, None)])
def test_append_reports_offsets_that_no_row_meets(pec, T, cu):
    """Offsets that descend before the first row or after the last one, or pass T, in any group of requests: their tokens are not
    stored, and the call says so.  Ascending ones with empty requests anywhere are fine."""
    ok = cu is None
    if ok:
        T, cu = 6, [2] * 300 + [3] * 300 + [6] * 300
    B = len(cu) - 1
    kp, vp, table = ref.make_cache(15, [20] * B, 24, 1, F32, DEV, poison=False, wild=False)
    k = torch.randn((T, 1, 128), device=DEV)
    pec.pec_kv_append(k, k, kp, vp, table, dev(cu), dev([20] * B))
    if ok:
        pec.check_status()
        return
    with pytest.raises(binding.PecError) as e:
        pec.check_status()
    assert e.value.code == binding.PEC_ERR_BAD_INDEX
