"""The verify attention over caches of 4-bit groups on pieces as long as they get in use: both kernels hold where the pages of 8192 tokens of a piece lie
(64 stages of 128, 32 chunks for each of eight wavefronts) and then ask again.  Pieces end on both sides of that and of twice as much, and the plan is
asserted, so that a case reaches the loop it is meant for.  Needs an MI355X (-m gpu)."""
import functools

import numpy as np
import pytest
import torch

import oracle
from block_helpers import DEV, assert_attention, i32, rng
from group_helpers import GroupCase, GroupStep, values
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from util import sample_rows

pytestmark = pytest.mark.gpu

FIRST_OWN = 77                   # of the instantiated kernels, those with keys of a wavefront's own are the last


@functools.lru_cache(maxsize=2)
def _pools(pages, Hkv, D, dtype):
    """K and V: bytes, scales, and the same numbers, of about one, in 16 bits."""
    r, out = rng(pages + Hkv + D + dtype), []
    for _ in range(2):
        raw = r.integers(0, 256, (pages, Hkv, 16, D // 2)).astype(np.uint8)
        scale = r.integers(125, 127, (pages, Hkv, 16, D // 32)).astype(np.uint8)
        out.append((raw, scale, W.store(values(raw, scale).astype(np.float32), dtype)))
    return out


def _case(seed, dtype, n, group, Hkv, D, lens, pages, spread):
    """Sequences whose pages are drawn from the pool (each once where there are enough); scores have a standard deviation of about ``spread``."""
    r = rng(seed)
    need = [(L + n + 15) // 16 for L in lens]
    drawn = r.permutation(pages) if sum(need) <= pages else r.integers(0, pages, sum(need))
    table, at = np.full((len(lens), max(need)), -1, np.int32), 0
    for b, k in enumerate(need):
        table[b, :k] = drawn[at:at + k]
        at += k
    (k, ks, k16), (v, vs, v16) = _pools(pages, Hkv, D, dtype)
    q = W.store(r.standard_normal((len(lens), n, Hkv * group, D)).astype(np.float32), dtype)
    trees = np.stack([W.random_tree(n, 6, r) for _ in lens])
    case = W.Case("long", seed, dtype, len(lens), n, Hkv * group, Hkv, D, float(np.float32(spread / np.sqrt(D))), q, k16, v16, table, np.array(lens, np.int32),
                  trees, max(need), Hkv * 16 * D, 16 * D, D, pages)
    return GroupCase(case, (k, v), (ks, vs), (Hkv * 8 * D, 8 * D, D // 2))


def _check(gc, step, what):
    got, rows = step.result(), sample_rows(gc.case, 48, always=[(b, gc.case.N - 1, gc.case.Hq - 1) for b in range(gc.case.B)])
    want = oracle.verify_attn_case(gc.case, rows=rows)
    assert_attention(got[rows[:, 0], rows[:, 1], rows[:, 2]].astype(np.float64), gc, want, what)
    assert np.isfinite(got).all() and int(step.status.item()) == 0
    step.out.fill_(float("nan"))                         # and again: the same bits
    assert np.array_equal(step.result(), got), what


# (nodes, query heads a KV head, KV heads, greatest length announced, own keys, tiles a wavefront and row groups in bf16, in fp16)
SPLITS = {
    "own keys, 1 tile": (4, 4, 2, None, True, (1, 1), (1, 1)), "own keys, 2 tiles": (8, 4, 1, 1 << 18, True, (2, 1), (2, 1)),
    "own keys, 2 groups": (16, 4, 1, 1 << 17, True, (2, 2), (2, 2)), "own keys, 8 groups": (60, 4, 1, None, True, (2, 8), (2, 8)),
    "shared, 2 tiles in all": (8, 4, 1, None, False, (1, 1), (1, 1)), "shared, 3 tiles in all": (12, 4, 1, 1 << 22, False, (2, 1), (2, 1)),
    "shared, 4 tiles": (16, 4, 1, 1 << 22, False, (2, 1), (2, 1)), "shared, 7 tiles": (28, 4, 1, 1 << 22, False, (2, 1), (2, 1)),
    "shared, 15 tiles": (60, 4, 1, 1 << 22, False, (2, 1), (2, 1)), "shared, 20 tiles": (40, 8, 1, 1 << 22, False, (3, 1), (2, 2)),
}


def _split_step(layout, dtype, D, ctx, split, spread):
    n, group, Hkv, announced, own, bf16, fp16 = SPLITS[layout]
    gc = _case(n + D, dtype, n, group, Hkv, D, [ctx], 1700, spread)
    step = GroupStep(gc, split_tokens=split, max_ctx_len=announced)
    if announced is not None:
        width = (announced + n + 15) // 16
        table = np.full((1, width), -1, np.int32)
        table[:, :gc.case.page_table.shape[1]] = gc.case.page_table
        step.table, step.desc.max_pages_per_seq = i32(table), width
        step.ws = torch.full((B.owl_verify_attn_groups_workspace_size(step.desc),), 0xFF, dtype=torch.uint8, device=DEV)
    plan = B.owl_verify_attn_groups_plan(step.desc)
    assert (plan.kernel_variant >= FIRST_OWN, plan.tiles_per_wave, plan.row_groups) == (own, *(fp16 if dtype == W.DT_F16 else bf16)), plan.as_dict()
    assert plan.split_tokens == split
    return gc, step


# the longest split a caller can ask for, and a rest of a little less and a little more than 8192 tokens
@pytest.mark.parametrize("ctx,spread", [(24500, 1.0), (24700, 6.0), (24576, 60.0)])
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", list(SPLITS))
def test_equal_splits_of_128_stages(layout, D, dtype, ctx, spread):
    _check(*_split_step(layout, dtype, D, ctx, 16384, spread), layout)


@pytest.mark.parametrize("split", [8128, 8192, 8256, 8320])
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("layout", list(SPLITS))
def test_pieces_about_where_the_page_lists_end(layout, dtype, split):
    _check(*_split_step(layout, dtype, 128, 24990, split, 1.0), f"{layout} {split}")


# (nodes, query heads a KV head, own keys, tiles a wavefront and row groups in bf16, in fp16)
SHARES = {
    "own keys, 1 tile": (4, 4, True, (1, 1), (1, 1)), "own keys, 2 tiles": (8, 4, True, (2, 1), (2, 1)), "shared, 4 tiles": (16, 4, False, (2, 1), (2, 1)),
    "shared, 7 tiles": (26, 4, False, (2, 1), (2, 1)), "shared, 15 tiles": (60, 4, False, (2, 1), (2, 1)), "shared, 20 tiles": (40, 8, False, (3, 1), (2, 2)),
}


def _shares_plan(step, layout, dtype):
    own, bf16, fp16 = SHARES[layout][2:]
    plan = B.owl_verify_attn_groups_plan(step.desc)
    assert (plan.kernel_variant >= FIRST_OWN, plan.tiles_per_wave, plan.row_groups) == (own, *(fp16 if dtype == W.DT_F16 else bf16)), plan.as_dict()
    return plan


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("layout", list(SHARES))
def test_shares_of_hundreds_of_stages(layout, dtype, D):
    """64 KV heads leave each four workers on 256 compute units, of two row groups two: 25000 tokens each and more."""
    n, group = SHARES[layout][:2]
    T = 64 * 1600 - 77
    gc = _case(n, dtype, n, group, 64, D, [T], 200, 1.0)
    step = GroupStep(gc)
    plan = _shares_plan(step, layout, dtype)
    assert T * 64 * plan.row_groups // plan.n_workgroups >= 20000
    _check(gc, step, layout)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("layout", list(SHARES))
def test_shares_of_long_batches(layout, dtype):
    """16 sequences over 32 workers a head: pieces begin and end within sequences, some are two or three times 8192 tokens long."""
    n, group = SHARES[layout][:2]
    lens = [20011, 64000, 31, 40005, 0, 52345, 8191, 8192, 8193, 16384 - n, 16385, 61440, 24576, 33000, 47777, 58001]
    gc = _case(n + 1, dtype, n, group, 8, 128, lens, 400, 1.0)
    step = GroupStep(gc)
    plan = _shares_plan(step, layout, dtype)
    assert sum(lens) * 8 * plan.row_groups // plan.n_workgroups >= 12000
    _check(gc, step, layout)
