"""The plan of the verify attention over 8-bit blocks (no GPU): wavefronts with keys of their own for little work, the shared ring for much."""
import ctypes

import pytest

from paper_2510_07535_amd import binding as B
from test_abi_rows import _desc


@pytest.mark.parametrize("n,hq,hkv,batch,ctx,dtype,own", [
    (1, 32, 8, 1, 65536, B.OWL_BF16, True), (16, 32, 8, 1, 1 << 20, B.OWL_BF16, True), (60, 32, 8, 1, 5003, B.OWL_BF16, True),
    (60, 32, 8, 1, 65001, B.OWL_BF16, False), (60, 32, 8, 1, 20000, B.OWL_BF16, False), (60, 32, 8, 1, 20000, B.OWL_F16, True),
    (26, 32, 8, 16, 65536, B.OWL_F16, False), (24, 32, 8, 16, 65536, B.OWL_F16, True), (16, 32, 8, 16, 65536, B.OWL_BF16, True),
    (16, 32, 8, 16, 8192, B.OWL_BF16, False), (40, 64, 8, 1, 131072, B.OWL_BF16, False),
])
@pytest.mark.parametrize("D", [64, 128])
def test_plan(n, hq, hkv, batch, ctx, dtype, own, D):
    d = _desc(n_draft=n, n_q_heads=hq, n_kv_heads=hkv, batch=batch, max_ctx_len=ctx, max_pages_per_seq=(ctx + n + 15) // 16, qkv_dtype=dtype, head_dim=D)
    p = B.owl_verify_attn_quant_plan(d)
    assert p.workspace_bytes == B.owl_verify_attn_quant_workspace_size(d)
    assert (p.kernel_variant >= 47) == own and p.kernel_variant >= 27
    assert p.row_tiles == (n * hq // hkv + 15) // 16 and (not own or p.tiles_per_wave <= 2 and p.row_groups == (p.row_tiles + 1) // 2)
    assert p.split_tokens % 64 == 0 and p.split_tokens * p.max_splits >= ctx + n


def test_plan_refuses():
    plan = B.Plan()
    assert B.lib().owl_verify_attn_quant_plan(ctypes.byref(_desc()), None) == B.OWL_ERR_INVALID_ARG
    assert B.lib().owl_verify_attn_quant_plan(None, ctypes.byref(plan)) == B.OWL_ERR_INVALID_ARG
    assert B.lib().owl_verify_attn_quant_plan(ctypes.byref(_desc(qkv_dtype=B.OWL_F32)), ctypes.byref(plan)) == B.OWL_ERR_UNSUPPORTED
