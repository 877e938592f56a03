"""CPU checks of the calls over a cache held in 4 bits: what the library refuses before any launch, workspace sizes, the binding's own
checks, and the reference that the GPU tests compare with."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import q4_reference as q4
from paper_2409_15104_b200 import binding

BIG = 1 << 20                                                     # addresses are never dereferenced: validation fails first


def test_library_exports_every_declared_symbol():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = open(os.path.join(root, "include", "pec.h")).read()
    assert set(re.findall(r"^(?:int|size_t) (pec_[a-z_]*q4[a-z_]*)\(", header, re.M)) == set(binding.EXPORTS_Q4)
    for name in binding.EXPORTS_Q4:
        assert getattr(binding.load(), name) is not None


def _cache(c, **over):
    c.k_pages = c.v_pages = c.k_scales = c.v_scales = c.block_table = c.cu_q = c.kv_lens = BIG
    for side in "kv":
        for what, unit in (("pages", 64), ("scales", 1)):
            setattr(c, f"{side}_{what}_stride_p", 16 * 8 * unit)
            setattr(c, f"{side}_{what}_stride_t", 8 * unit)
            setattr(c, f"{side}_{what}_stride_h", unit)
    c.page_size, c.num_pages, c.max_pages, c.table_stride, c.B, c.T, c.Hkv, c.D = 16, 100, 10, 10, 4, 0, 8, 128
    for k, v in over.items():
        setattr(c, k, v)


def _apply(a, over):
    names = {f for f, _ in binding.pec_q4_cache._fields_}
    for k, v in over.items():
        setattr(a.cache if k in names else a, k, v)
    return a


CACHE_REFUSALS = [
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(k_scales=None), -1), (dict(v_scales=None), -1), (dict(block_table=None), -1),
    (dict(cu_q=None), -1), (dict(kv_lens=None), -1), (dict(status=None), -1), (dict(D=64), -2), (dict(dtype=3), -2), (dict(Hkv=0), -1),
    (dict(B=0), -1), (dict(T=-1), -1), (dict(T=(1 << 30) + 1), -2), (dict(page_size=12), -2), (dict(page_size=0), -2), (dict(num_pages=0), -1),
    (dict(num_pages=1 << 31), -1), (dict(max_pages=0), -1), (dict(table_stride=9), -1), (dict(table_stride=9, B=1), 0),
    (dict(max_pages=1 << 27, table_stride=1 << 27), -2), (dict(k_pages_stride_t=32), -1), (dict(v_pages_stride_h=80), -3),
    (dict(k_pages_stride_p=0), -1), (dict(v_pages=BIG + 16), -3), (dict(k_scales=BIG + 1), -3), (dict(v_scales_stride_t=0), -1),
    (dict(k_scales_stride_h=-1), -1), (dict(kv_lens=BIG + 2), -3), (dict(k_scales_stride_h=7), 0),
]


def _append(**over):
    a = binding.pec_kv_append_q4_args()
    _cache(a.cache)
    a.k = a.v = a.status = BIG
    a.k_stride_t = a.v_stride_t = 8 * 128
    a.k_stride_h = a.v_stride_h = 128
    a.dtype, a.eps = binding.PEC_BF16, 1e-6
    return _apply(a, over)


@pytest.mark.parametrize("over,code", [({}, 0)] + CACHE_REFUSALS + [
    (dict(k=None), -1), (dict(v=BIG + 8), -3), (dict(k_stride_t=64), -1), (dict(v_stride_h=132), -3), (dict(norm=3), -1),
    (dict(norm=1, eps=0.0), -1), (dict(rope_table=BIG, n_pos=-1), -1), (dict(rope_table=BIG + 4, n_pos=9), -3), (dict(k_weight=BIG + 8), -3),
])
def test_append_validates_on_the_host(over, code):
    assert binding.load().pec_kv_append_q4(ctypes.byref(_append(**over)), None) == code, binding.pec_last_error()
    assert binding.load().pec_kv_append_q4(None, None) == -1


@pytest.mark.parametrize("over,code", [({}, 0)] + CACHE_REFUSALS + [
    (dict(k_out=None), -1), (dict(v_out=None), -1), (dict(k_out=BIG + 8), -3), (dict(k_out_stride_t=64), -1), (dict(v_out_stride_h=132), -3),
])
def test_read_validates_on_the_host(over, code):
    a = binding.pec_kv_read_q4_args()
    _cache(a.cache)
    a.k_out = a.v_out = a.status = BIG
    a.k_out_stride_t = a.v_out_stride_t = 8 * 128
    a.k_out_stride_h = a.v_out_stride_h = 128
    a.dtype = binding.PEC_BF16
    assert binding.load().pec_kv_read_q4(ctypes.byref(_apply(a, over)), None) == code, binding.pec_last_error()
    assert binding.load().pec_kv_read_q4(None, None) == -1


def _paged(**over):
    a = binding.pec_paged_q4_args()
    _cache(a.cache)
    a.q = a.o = a.lse = a.status = BIG
    a.q_stride_t, a.q_stride_h, a.Hq, a.dtype, a.o_dtype, a.causal = 32 * 128, 128, 32, binding.PEC_BF16, binding.PEC_BF16, 1
    a.workspace, a.workspace_bytes = BIG, 1 << 40
    return _apply(a, over)


@pytest.mark.parametrize("over,code", [({}, 0)] + CACHE_REFUSALS + [
    (dict(q=None), -1), (dict(o=None), -1), (dict(lse=None), -1), (dict(Hq=33), -1), (dict(Hq=8 * 129), -1), (dict(o_dtype=4), -2),
    (dict(dtype=binding.PEC_F32), -2), (dict(causal=2), -1), (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=-1.0), -1),
    (dict(max_q_len=-1), -1), (dict(q=BIG + 8), -3), (dict(q_stride_t=132), -3), (dict(o=BIG + 8), -3), (dict(lse=BIG + 2), -3),
])
def test_paged_attn_validates_on_the_host(over, code):
    lib = binding.load()
    a = _paged(**over)
    assert lib.pec_paged_attn_q4(ctypes.byref(a), None) == code, binding.pec_last_error()
    if code:
        assert lib.pec_paged_q4_workspace_size(ctypes.byref(a)) == 0
    assert lib.pec_paged_attn_q4(None, None) == -1


def test_paged_attn_asks_for_its_workspace():
    lib = binding.load()
    a = _paged(T=64, max_q_len=1, max_pages=1000, table_stride=1000, num_pages=100000, B=64)
    need = lib.pec_paged_q4_workspace_size(ctypes.byref(a))
    assert need > 0
    for ws, size in ((None, need), (BIG, need - 1), (BIG + 8, need)):
        a.workspace, a.workspace_bytes = ws, size
        assert lib.pec_paged_attn_q4(ctypes.byref(a), None) == -4, binding.pec_last_error()


def test_binding_checks_what_the_library_cannot_see():
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.pec_kv_append_q4(x, x, x, x, x, x, x, x, x)         # not a CUDA tensor
    with pytest.raises(ValueError):
        binding.pec_paged_attn_q4(x, x, x, x, x, x, x, x)
    with pytest.raises(TypeError):
        binding.pec_paged_attn_q4(x.half(), x, x, x, x, x, x, x)
    with pytest.raises(ValueError):
        binding.pec_kv_read_q4(x, x, x, x, x, x, x, 4)


def test_the_reference_quantises_by_definition():
    """Hand-worked heads; every representable number is a fixed point; the held head is within half a step, and exact in bf16."""
    x = np.zeros((5, 128))
    x[0, :8] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, -0.25]           # scale 1: every border goes to its even code
    x[1, :3] = [6.01, -1, 0.3]                                     # scale 33 / 32
    x[2, 7] = 1e-35                                                # below the least scale
    x[3, 0] = 3e38
    x[4, 1] = np.nan
    v, s = q4.quantise(x)
    assert v[0, :8].tolist() == [6, 4, 4, 2, 2, 1, 1, 0] and s[0] == 1
    assert s[1] == 33 / 32 and v[1, :3].tolist() == [6 * 33 / 32, -33 / 32, 0.5 * 33 / 32]
    assert s[2] == q4.LEAST and (v[2] == 0).all() and np.isnan(v[4]).all() and np.isnan(s[4])
    g = np.random.default_rng(3)
    y = g.standard_normal((300, 128)) * np.exp(g.standard_normal((300, 1)) * 5)
    v, s = q4.quantise(y)
    assert (s >= np.abs(y).max(-1) / 6).all() and (s <= np.abs(y).max(-1) / 6 * (1 + 2.0 ** -5)).all()
    assert (np.abs(v - y) <= s[:, None] * np.where(np.abs(y) > 4 * s[:, None], 1.0, np.where(np.abs(y) > 2 * s[:, None], 0.5, 0.25))).all()
    t = torch.from_numpy(v)
    assert torch.equal(t.to(torch.bfloat16).double(), t) and torch.equal(torch.from_numpy(q4.values(*q4.pack(y))), t)
    again, _ = q4.quantise(v)
    assert np.array_equal(again, v)
