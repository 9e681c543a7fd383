"""Calls whose grids would have more threads along a dimension than a launch can have are refused on the host (no GPU)."""
import pytest

from paper_2510_07535_amd import binding as B
from test_abi_rows import _append, _append_desc, _desc

MANY = 1 << 24


@pytest.mark.parametrize("quant,n", [(False, MANY), (False, 1 << 30), (True, (1 << 28) - 30), (True, 1 << 30)])
def test_append_refuses_more_tokens_than_a_grid_holds(quant, n):
    d = _desc(max_pages_per_seq=1 << 27, n_pool_pages=1 << 27)
    assert _append(d, _append_desc(n_tokens=n), quant) == B.OWL_ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,vocab,code", [
    (1 << 22, 100, B.OWL_ERR_UNSUPPORTED), ((1 << 22) - 1, 100, None), (1 << 22, 8185, B.OWL_ERR_UNSUPPORTED), (1 << 22, 8186, None),
    (1 << 23, 8186, B.OWL_ERR_UNSUPPORTED), ((1 << 23) - 1, 40000, None), ((1 << 31) - 1, 1, B.OWL_ERR_UNSUPPORTED),
])
def test_logprobs_refuse_more_rows_than_a_grid_holds(rows, vocab, code):
    d = B.LogprobDesc(rows=rows, vocab=vocab, n_given=0, n_top=1, dtype=B.OWL_F32, scale=1.0, row_stride=vocab)
    if code is None:
        assert B.owl_token_logprobs_workspace_size(d) > 0
        return
    with pytest.raises(B.OwlError) as e:
        B.owl_token_logprobs_workspace_size(d)
    assert e.value.code == code
