"""Values that are not finite in a cache held in 4 bits, where some rows of their request see them and others do not yet."""
import pytest
import torch

import paged_reference as ref
import q4_reference as q4
from test_q4_gpu import BF16, DEV, F32, check, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,kv", [(2, 50), (4, 50), (4, 3000), (5, 50), (20, 700), (200, 300), (200, 3000)])
@pytest.mark.parametrize("back", [1, 2])
def test_a_value_that_some_rows_do_not_see_yet(pec, dtype, n, kv, back):
    """The last tokens but one or two hold a value that is not finite.  Rows that see it get NaN; those before it get NaN or what they
    would get without it - the latter, where 16 packed rows or fewer of bf16 queries make a request; LSEs, the other KV head and the
    request beside it are as without it."""
    ns, kvs, page = [n, 3], [kv, 90], 16
    kp, ks, vp, vs, table = cache = q4.make_cache(41, kvs, page, 2, DEV)
    cu = ref.offsets(ns)
    q = torch.randn((cu[-1], 8, 128), generator=torch.Generator().manual_seed(42)).to(dtype).to(DEV)
    want = q4.attend(q, cache, cu, kvs)
    at = kv - back
    clean = [t.clone() for t in cache[:4]]
    vs[int(table[0, at // page]), at % page, 1] = float("nan")
    o, lse = pec.pec_paged_attn_q4(q, *cache, dev(cu), dev(kvs), max_q_len=max(ns))
    pec.check_status()
    sees = n - back
    assert torch.isnan(o[sees:n, 4:]).all()
    spoilt = torch.isnan(o[:sees, 4:]).all(-1)
    assert torch.equal(spoilt, torch.isnan(o[:sees, 4:]).any(-1))
    if dtype == BF16 and 4 * n <= 16:
        assert not spoilt.any()
    o[sees:n, 4:] = torch.from_numpy(want[0][sees:n, 4:]).to(o)
    o[:sees, 4:][spoilt] = torch.from_numpy(want[0][:sees, 4:]).to(o)[spoilt]
    check(o, lse, want, dtype, (*clean, table), kvs, 4 * n, f"{n} tokens of {kv}, {int(spoilt.sum())} rows spoilt")
