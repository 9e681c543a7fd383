"""The verify attention over 8-bit blocks on pieces as long as they get in use, loop by loop: hundreds of stages of 64 tokens, rings that
turn over, page lists that are asked for again.  The plan is asserted, so that a case reaches the loop it is meant for.  Needs an
MI355X (-m gpu)."""
import functools

import numpy as np
import pytest
import torch

import oracle
from block_helpers import DEV, BlockCase, QuantStep, assert_attention, block_case, i32, oracle_out, rng
from oracle import cache_blocks as C
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from util import sample_rows

pytestmark = pytest.mark.gpu


@functools.lru_cache(maxsize=2)
def _pools(pages, Hkv, D, dtype):
    """Blocks of numbers of about one, the scales of neighbours apart by up to four, and the same numbers in 16 bits."""
    r = rng(pages + Hkv + D + dtype)
    strides, out = (Hkv * 16 * D, 16 * D, D), []
    for _ in range(2):
        raw = C.e4m3_bytes(np.clip(r.standard_normal((pages, Hkv, 16, D)) * 64.0, -448.0, 448.0))
        scale = r.integers(120, 123, (pages, Hkv)).astype(np.uint8)
        numbers = C.e4m3_values(raw) * np.exp2(scale.astype(np.float64) - 127.0)[:, :, None, None]
        out.append((C.Blocks(raw, scale, strides, D, dtype), W.store(numbers.astype(np.float32), dtype)))
    return out


def _case(seed, dtype, n, group, Hkv, D, ctx, pages, spread):
    """One sequence whose pages are drawn from the pool (each once where there are enough); scores have a standard deviation of ``spread``."""
    r = rng(seed)
    need = (ctx + n + 15) // 16
    table = (r.permutation(pages) if need <= pages else r.integers(0, pages, need))[:need].astype(np.int32)[None]
    (k, k16), (v, v16) = _pools(pages, Hkv, D, dtype)
    q = W.store(r.standard_normal((1, n, Hkv * group, D)).astype(np.float32), dtype)
    case = W.Case("long", seed, dtype, 1, n, Hkv * group, Hkv, D, float(np.float32(spread / np.sqrt(D))), q, k16, v16, table, np.array([ctx], np.int32),
                  W.random_tree(n, 6, r)[None], need, *k.strides, pages)
    return BlockCase(case, k, v)


def _variant(own_keys, index, dtype, D):
    """Numbers of the instantiated kernels: 27 for 16- and 32-bit caches, five a type and head size of the ring, three of own keys."""
    kind = [(W.DT_BF16, 128), (W.DT_BF16, 64), (W.DT_F16, 128), (W.DT_F16, 64)].index((dtype, D))
    return 27 + 20 + 3 * kind + index if own_keys else 27 + 5 * kind + index


def _check(bc, step, what):
    step.run()
    got, rows = step.result(), sample_rows(bc.case, 48, always=[(0, bc.case.N - 1, bc.case.Hq - 1)])
    want = oracle.verify_attn_case(bc.case, rows=rows)
    assert_attention(got[rows[:, 0], rows[:, 1], rows[:, 2]], bc, want, what)
    assert np.isfinite(got).all() and step.flags() == 0
    step.out.fill_(float("nan"))                         # and again: the same bits
    step.run()
    assert np.array_equal(step.result(), got), what


# Equal splits of 256 stages, the longest a caller can ask for, and a rest: (nodes, query heads, KV heads, greatest length announced, own
# keys, kernel, tiles a wavefront, row groups)
SPLITS = {
    "own keys, 1 tile": (4, 4, 2, None, True, 0, 1, 1), "own keys, 2 tiles": (8, 4, 2, None, True, 1, 2, 1),
    "own keys, 2 groups": (16, 4, 2, None, True, 2, 2, 2), "own keys, 8 groups": (60, 4, 1, None, True, 2, 2, 8),
    "two key groups": (60, 4, 1, 1 << 20, False, 0, 1, 4), "pipelined, 1 tile": (20, 4, 1, 1 << 22, False, 1, 1, 1),
    "pairs of 7 tiles": (14, 8, 1, 1 << 22, False, 2, 2, 1), "pairs of 8 tiles": (16, 8, 1, 1 << 22, False, 2, 2, 1),
    "pipelined, 2 tiles": (60, 4, 1, 1 << 22, False, 3, 2, 1), "3 tiles": (40, 8, 1, 1 << 22, False, 4, 3, 1),
}


@pytest.mark.parametrize("spread", [1.0, 6.0, 60.0])         # (from 60 on bf16 pieces are done again, fp16 from 6)
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", list(SPLITS))
def test_equal_splits_of_256_stages(layout, D, dtype, spread):
    n, group, Hkv, announced, own, index, tiles, groups = SPLITS[layout]
    bc = _case(n + D, dtype, n, group, Hkv, D, 16384 + 64 * 70 + 37, 1400, spread)
    step = QuantStep(bc, split_tokens=16384, max_ctx_len=announced)
    if announced is not None:
        width = (announced + n + 15) // 16
        table = np.full((1, width), -1, np.int32)
        table[:, :bc.case.page_table.shape[1]] = bc.case.page_table
        step.table, step.desc.max_pages_per_seq = i32(table), width
        step.workspace = torch.empty(B.owl_verify_attn_quant_workspace_size(step.desc), dtype=torch.uint8, device=DEV)
    plan = B.owl_verify_attn_quant_plan(step.desc)
    assert (plan.kernel_variant, plan.tiles_per_wave, plan.row_groups, plan.split_tokens) == (_variant(own, index, dtype, D), tiles, groups, 16384)
    _check(bc, step, layout)


# Shares of a library-chosen size: 64 KV heads leave each four workers on 256 compute units, some 400 stages each.
SHARES = {
    "own keys, 1 tile": (4, 4, True, 0, 1, 1), "own keys, 2 tiles": (8, 4, True, 1, 2, 1), "own keys, 2 groups": (16, 4, True, 2, 2, 2),
    "pipelined, 1 tile": (20, 4, False, 1, 1, 1), "pairs": (32, 4, False, 2, 2, 1), "pipelined, 2 tiles": (60, 4, False, 3, 2, 1),
    "3 tiles": (40, 8, False, 4, 3, 1),
}


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("layout", list(SHARES))
def test_shares_of_hundreds_of_stages(layout, dtype):
    n, group, own, index, tiles, groups = SHARES[layout]
    bc = _case(n, dtype, n, group, 64, 128, 64 * 1600 - 77, 200, 1.0)
    step = QuantStep(bc)
    plan = B.owl_verify_attn_quant_plan(step.desc)
    assert (plan.kernel_variant, plan.tiles_per_wave, plan.row_groups) == (_variant(own, index, dtype, 128), tiles, groups)
    assert 1600 * 64 * groups // plan.n_workgroups >= 300          # stages of a worker
    _check(bc, step, layout)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("n,tiles,groups", [(4, 1, 1), (7, 2, 1), (15, 2, 2)])
def test_equal_splits_of_a_batch_with_keys_of_their_own(n, tiles, groups, dtype):
    r = rng(n)
    hkv, announced = 3, 20000 if dtype == W.DT_BF16 else None       # (four tiles in bf16: from 16K tokens on)
    bc = block_case("own-split", n, dtype=dtype, Hq=4 * hkv, Hkv=hkv, D=128, ctx_lens=[700, 33, 0, 1500], trees=[W.random_tree(n, 5, r) for _ in range(4)])
    for counts in (None, [n, 0, 1, n // 2]):
        step = QuantStep(bc, counts=counts, split_tokens=192, max_ctx_len=announced)
        if announced is not None:
            table = np.full((4, (announced + n + 15) // 16), -1, np.int32)
            table[:, :bc.case.page_table.shape[1]] = bc.case.page_table
            step.table, step.desc.max_pages_per_seq = i32(table), table.shape[1]
            step.workspace = torch.empty(B.owl_verify_attn_quant_workspace_size(step.desc), dtype=torch.uint8, device=DEV)
        plan = B.owl_verify_attn_quant_plan(step.desc)
        assert plan.kernel_variant >= 47 and (plan.tiles_per_wave, plan.row_groups, plan.split_tokens) == (tiles, groups, 192)
        step.run()
        assert_attention(step.result(), bc, oracle_out(bc, counts), str(counts))
        assert step.flags() == 0
