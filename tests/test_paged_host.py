"""CPU checks of the paged serving calls: what the library refuses before any launch, workspace sizes, and the binding's own
checks; and that the 64-bit reference they are tested against agrees with the oracle."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paged_reference as ref
from paper_2409_15104_b200 import binding

BIG = 1 << 20                                                     # addresses are never dereferenced: validation fails first


def _norm_rope(**over):
    a = binding.pec_norm_rope_args()
    a.q = a.q_out = a.k = a.k_out = a.status = BIG
    for f in ("q_stride_h", "k_stride_h", "q_out_stride_h", "k_out_stride_h"):
        setattr(a, f, 128)
    a.q_stride_t = a.q_out_stride_t = 8 * 128
    a.k_stride_t = a.k_out_stride_t = 2 * 128
    a.dtype, a.Hq, a.Hkv, a.D, a.T, a.norm, a.eps = binding.PEC_BF16, 8, 2, 128, 0, 1, 1e-6
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code", [
    ({}, 0), (dict(q=None), -1), (dict(k_out=None), -1), (dict(k=None, k_out=None, Hkv=0, k_stride_t=0), 0), (dict(q=None, q_out=None, Hq=0), 0),
    (dict(Hq=0, Hkv=0), -1), (dict(Hq=-1), -1), (dict(T=-1), -1), (dict(D=64), -2), (dict(dtype=7), -2), (dict(norm=2), -1),
    (dict(eps=0.0), -1), (dict(eps=float("nan")), -1), (dict(eps=0.0, norm=0), 0), (dict(rope_table=BIG, n_pos=0), -1),
    (dict(rope_table=BIG + 4, n_pos=10), -3), (dict(rope_table=BIG, n_pos=10, pos0=11), -1), (dict(rope_table=BIG, n_pos=10, T=11), -1),
    (dict(pos0=-1), -1), (dict(status=None), -1), (dict(q_stride_h=64), -1), (dict(k_stride_t=260), -3), (dict(q_out=BIG + 8), -3),
    (dict(q_weight=BIG + 2), -3), (dict(positions=BIG + 2), -3), (dict(q_out_stride_t=9 * 128), -1), (dict(q_out=BIG + 4096, q_out_stride_t=9 * 128), 0),
    (dict(Hq=70000), -2), (dict(T=(1 << 30) + 1), -2),
])
def test_norm_rope_validates_on_the_host(over, code):
    assert binding.load().pec_qk_norm_rope(ctypes.byref(_norm_rope(**over)), None) == code, binding.pec_last_error()
    assert binding.load().pec_qk_norm_rope(None, None) == -1


def _cache(a, **over):
    a.k_pages = a.v_pages = a.block_table = a.cu_q = a.kv_lens = a.status = BIG
    for side in "kv":
        setattr(a, f"{side}_pages_stride_p", 16 * 8 * 128)
        setattr(a, f"{side}_pages_stride_t", 8 * 128)
        setattr(a, f"{side}_pages_stride_h", 128)
    a.page_size, a.num_pages, a.max_pages, a.table_stride, a.B, a.T = 16, 100, 10, 10, 4, 0
    a.Hkv, a.D, a.dtype = 8, 128, binding.PEC_BF16
    for k, v in over.items():
        setattr(a, k, v)
    return a


CACHE_REFUSALS = [
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(block_table=None), -1), (dict(cu_q=None), -1), (dict(kv_lens=None), -1),
    (dict(status=None), -1), (dict(D=64), -2), (dict(dtype=3), -2), (dict(Hkv=0), -1), (dict(B=0), -1), (dict(T=-1), -1),
    (dict(T=(1 << 30) + 1), -2), (dict(page_size=12), -2), (dict(page_size=0), -2), (dict(page_size=4), -2), (dict(num_pages=0), -1),
    (dict(num_pages=1 << 31), -1), (dict(max_pages=0), -1), (dict(table_stride=9), -1), (dict(table_stride=9, B=1), 0),
    (dict(max_pages=1 << 27, table_stride=1 << 27), -2), (dict(k_pages_stride_t=64), -1), (dict(v_pages_stride_h=132), -3),
    (dict(k_pages_stride_p=0), -1), (dict(v_pages=BIG + 8), -3), (dict(kv_lens=BIG + 2), -3),
]


@pytest.mark.parametrize("over,code", [({}, 0)] + CACHE_REFUSALS + [
    (dict(k=None), -1), (dict(v=BIG + 8), -3), (dict(k_stride_t=64), -1), (dict(v_stride_h=132), -3), (dict(norm=3), -1),
    (dict(norm=1, eps=0.0), -1), (dict(rope_table=BIG, n_pos=-1), -1), (dict(k_weight=BIG + 8), -3),
])
def test_append_validates_on_the_host(over, code):
    a = _cache(binding.pec_kv_append_args())
    a.k = a.v = BIG
    a.k_stride_t = a.v_stride_t = 8 * 128
    a.k_stride_h = a.v_stride_h = 128
    a.eps = 1e-6
    for k, v in over.items():
        setattr(a, k, v)
    assert binding.load().pec_kv_append(ctypes.byref(a), None) == code, binding.pec_last_error()
    assert binding.load().pec_kv_append(None, None) == -1


def _paged(**over):
    a = _cache(binding.pec_paged_args())
    a.q = a.o = a.lse = BIG
    a.q_stride_t, a.q_stride_h, a.Hq, a.o_dtype, a.causal = 32 * 128, 128, 32, binding.PEC_BF16, 1
    a.workspace, a.workspace_bytes = BIG, 1 << 40
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code", [({}, 0)] + CACHE_REFUSALS + [
    (dict(q=None), -1), (dict(o=None), -1), (dict(lse=None), -1), (dict(Hq=33), -1), (dict(Hq=8 * 129), -1), (dict(o_dtype=4), -2),
    (dict(dtype=binding.PEC_F32), -2), (dict(causal=2), -1), (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=-1.0), -1),
    (dict(max_q_len=-1), -1), (dict(q=BIG + 8), -3), (dict(q_stride_t=132), -3), (dict(o=BIG + 8), -3), (dict(lse=BIG + 2), -3),
])
def test_paged_attn_validates_on_the_host(over, code):
    lib = binding.load()
    a = _paged(**over)
    assert lib.pec_paged_attn(ctypes.byref(a), None) == code, binding.pec_last_error()
    if code:
        assert lib.pec_paged_workspace_size(ctypes.byref(a)) == 0
    assert lib.pec_paged_attn(None, None) == -1


@pytest.mark.parametrize("over,bf16", [
    (dict(k_pages_stride_p=16 * 8 * 128 + 8, num_pages=(1 << 31) - 1), -2),          # common divisor 8: page numbers times 2049
    (dict(k_pages_stride_p=16 * 8 * 128 + 8, num_pages=1 << 20), -2), (dict(k_pages_stride_p=16 * 8 * 128 + 8, num_pages=1 << 19), 0),
    (dict(num_pages=(1 << 24) - 1), 0), (dict(v_pages_stride_h=1 << 45), -2),
    (dict(v_pages_stride_h=1 << 45, Hkv=1), 0), (dict(v_pages_stride_p=(1 << 45) + 8, num_pages=1), 0), (dict(v_pages_stride_p=(1 << 45) + 8), -2),
])
def test_strides_that_the_tensor_maps_cannot_hold(over, bf16):
    lib = binding.load()
    for dtype, code in ((binding.PEC_BF16, bf16), (binding.PEC_F32, 0)):
        a = _paged(dtype=dtype, o_dtype=binding.PEC_F32, **over)
        assert lib.pec_paged_attn(ctypes.byref(a), None) == code, binding.pec_last_error()


def test_paged_attn_asks_for_its_workspace():
    lib = binding.load()
    a = _paged(T=64, max_q_len=1, max_pages=1000, table_stride=1000, num_pages=100000, B=64)
    need = lib.pec_paged_workspace_size(ctypes.byref(a))
    assert need > 0
    for ws, size in ((None, need), (BIG, need - 1), (BIG + 8, need)):
        a.workspace, a.workspace_bytes = ws, size
        assert lib.pec_paged_attn(ctypes.byref(a), None) == -4, binding.pec_last_error()


def test_binding_checks_what_the_library_cannot_see():
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.pec_qk_norm_rope(x)                                # not a CUDA tensor
    with pytest.raises(TypeError):
        binding.pec_qk_norm_rope(x.half())
    with pytest.raises(ValueError):
        binding.pec_paged_attn(x, x, x, x, x, x)


def test_reference_agrees_with_the_oracle():
    """Contiguous prefill and decode rows of the oracle against the paged reference on the same keys and values."""
    torch.manual_seed(5)
    kv, n, hq, hkv, page = 77, 30, 4, 2, 16
    kp, vp, table = ref.make_cache(3, [kv, 5], page, hkv, torch.float32, "cpu")
    q = torch.randn((n + 5, hq, 128))
    o, lse, _, _ = ref.attend(q, kp, vp, table, [0, n, n + 5], [kv, 5])
    keys = kp[table[0, :5].long()].reshape(-1, hkv, 128)[:kv]
    vals = vp[table[0, :5].long()].reshape(-1, hkv, 128)[:kv]
    full = torch.cat([torch.zeros((kv - n, hq, 128)), q[:n]])
    want_o, want_l = oracle.prefill_attn(full, keys.contiguous(), vals.contiguous(), seq_len=kv, chunk_start=kv - n, chunk_len=n, kv_len=kv)
    assert np.abs(o[:n] - want_o).max() < 1e-12 and np.abs(lse[:n] - want_l).max() < 1e-12
    x = torch.randn((3, 2, 128))
    pos = [0, 17, 40000]
    want = oracle.rope(x.double().numpy().reshape(3, 256), pos, 1e4, 256).reshape(3, 2, 128)
    assert np.abs(ref.rope(x.double().numpy(), pos, 1e4) - want).max() < 1e-9


@pytest.mark.parametrize("n_pos", [10, (1 << 31) - 1])
def test_norm_rope_refuses_positions_that_wrap(n_pos):
    """pos0 + T past 2^63 is past the table, not before it."""
    for pos0 in ((1 << 63) - 1, (1 << 63) - 2):
        assert binding.load().pec_qk_norm_rope(ctypes.byref(_norm_rope(rope_table=BIG, n_pos=n_pos, pos0=pos0, T=2)), None) == -1, binding.pec_last_error()


@pytest.mark.parametrize("dtype", [binding.PEC_BF16, binding.PEC_F32])
@pytest.mark.parametrize("hkv,g", [(1, 1), (1, 128), (8, 4), (24, 1), (64, 8), (128, 5), (1024, 67), (65535, 1)])
@pytest.mark.parametrize("T,B,most", [(1, 1, 1), (64, 64, 1), (4096, 1, 0), (8192, 300, 2048)])
def test_workspace_stays_below_its_documented_bound(dtype, hkv, g, T, B, most):
    """148 SMs: 137 MB and 0.133 MB for every KV head, and the list of row blocks."""
    a = _paged(T=T, B=B, max_q_len=most, max_pages=8192, table_stride=8192, num_pages=1000, Hkv=hkv, Hq=hkv * g, dtype=dtype,
               o_dtype=binding.PEC_F32, q_stride_t=hkv * g * 128)
    for side in "kv":
        setattr(a, f"{side}_pages_stride_t", hkv * 128)
        setattr(a, f"{side}_pages_stride_p", 16 * hkv * 128)
    need = binding.load().pec_paged_workspace_size(ctypes.byref(a))
    block = 2 * (128 // g) * g if dtype == binding.PEC_BF16 else 64                # packed rows
    lists = 48 * (T * g / block + min(T, B) + 1100 + hkv)
    assert 0 < need <= 137e6 + 0.133e6 * hkv + lists, (need, binding.pec_last_error())
