"""The verify attention over 8-bit blocks where its numbers lie far apart: references of pieces and of key groups that differ by more
than 32 bits hold, and keys, values and scales towards the ends of the types.  Needs an MI355X (-m gpu)."""
import dataclasses

import numpy as np
import pytest
import torch

from block_helpers import DEV, HALF, NAN_BYTE, BlockCase, QuantStep, assert_attention, i32, oracle_out, rng
from oracle import cache_blocks as C
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W

pytestmark = pytest.mark.gpu

# Layouts of the loops: (nodes, query heads a KV head, KV heads, sequences, greatest length announced, tokens a split).  Announced as
# long, or in a batch, rows go to the shared ring.
LONG = 1 << 20
LAYOUTS = {
    "own keys, 1 tile": (4, 4, 2, 1, None, 512), "own keys, 3 groups": (20, 4, 2, 1, None, 512), "two key groups": (10, 4, 2, 2, None, 512),
    "pipelined, 1 tile": (20, 4, 1, 1, LONG, 512), "pairs": (16, 8, 1, 1, LONG, 2048), "pipelined, 2 tiles": (60, 4, 1, 1, LONG, 512),
    "3 tiles": (40, 8, 1, 1, LONG, 512),
}


def make_blocks(case, k_wide, v_wide):
    """The blocks of a case's rows, k_wide and v_wide in the pools' layout (64 bits); slots behind the last row are no number."""
    strides = (case.stride_page, case.stride_head, case.stride_token)
    blocks, pools = [], []
    for wide in (k_wide, v_wide):
        held = C.Blocks(np.full(wide.shape, NAN_BYTE), np.full((case.n_pool_pages, case.Hkv), 255), strides, case.D, case.dtype)
        numbers = np.zeros_like(wide)
        for b in range(case.B):
            T = int(case.ctx_lens[b]) + case.N
            for lp in range((T + 15) // 16):
                page = int(case.page_table[b, lp])
                for g in range(case.Hkv):
                    at = [held._at(page, g, s) for s in range(min(16, T - lp * 16))]
                    held.write(page, g, np.stack([wide.reshape(-1)[a] for a in at]))
                    for s, a in enumerate(at):
                        numbers.reshape(-1)[a] = held.row(page, g, s)
        blocks.append(held)
        pools.append(W.store(numbers.astype(np.float32), case.dtype))
    return BlockCase(dataclasses.replace(case, k_pool=pools[0], v_pool=pools[1]), *blocks)


def make_step(bc, announced, split):
    step = QuantStep(bc, split_tokens=split, max_ctx_len=announced)
    if announced is not None:
        width = (announced + bc.case.N + 15) // 16
        table = np.full((bc.case.B, width), -1, np.int32)
        table[:, :bc.case.page_table.shape[1]] = bc.case.page_table
        step.table, step.desc.max_pages_per_seq = i32(table), width
        step.workspace = torch.empty(B.owl_verify_attn_quant_workspace_size(step.desc), dtype=torch.uint8, device=DEV)
    return step


def scored_case(layout, dtype, D, ctx, score_of, value_of):
    """Every row's score with the key at position t is score_of(t), as a power of two, and its value value_of(t) in all channels."""
    n, group, hkv, batch, announced, split = LAYOUTS[layout]
    unit = 130.0 / 128.0                                 # so that -128, 9 and the like, exact in a block, are -130, 9.14
    case = W.make_case("scored", 5, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=[ctx] * batch, trees=[W.chain_tree(n)] * batch,
                       scale=unit / (16.0 * np.log2(np.e)))
    q = np.zeros(case.q.shape)
    q[..., 0] = 16.0
    k, v = np.zeros(case.k_pool.shape), np.zeros(case.v_pool.shape)
    for b in range(batch):
        for t in range(ctx + n):
            page = int(case.page_table[b, t // 16])
            k[page, :, t % 16, 0] = score_of(t)
            v[page, :, t % 16, :] = value_of(t)
    case = dataclasses.replace(case, q=W.store(q.astype(np.float32), dtype))
    bc = make_blocks(case, k, v)
    return make_step(bc, announced, split), bc


def assert_rows(got, bc, want, what):
    """As assert_attention, element by element; here all channels of a row are rounded alike."""
    greatest = np.abs(W.widen(bc.case.v_pool, bc.case.dtype)).max()
    err, bound = np.abs(got - want), (2 * HALF[bc.case.dtype] + 2.0 ** -10) * greatest
    assert got.shape == want.shape and np.isfinite(got).all() and err.max() <= bound, f"{what}: {err.max():.3e} > {bound:.3e}"


# --------------------------------------------------------------------------- references far apart
# A key of weight 2^9.14 = 565 whose piece (or key group) began with scores of -130, against as many as 2048 keys of weight 1 elsewhere,
# whose values have the other sign.  Lost, it would leave an answer of 1.
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_the_greatest_score_in_a_piece_that_began_far_below(layout, D, dtype):
    split = LAYOUTS[layout][-1]
    late = split + split // 2 + 13
    step, bc = scored_case(layout, dtype, D, 2 * split, lambda t: 0.0 if t < split else 9.0 if t == late else -128.0,
                           lambda t: 1.0 if t < split else -1.0)
    step.run()
    assert_rows(step.result(), bc, oracle_out(bc), layout)
    assert step.flags() == 0


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("layout", ["two key groups", "pairs", "own keys, 1 tile"])
def test_the_greatest_score_among_keys_that_began_far_below(layout, odd, D, dtype):
    """The same between the wavefronts of one piece: 32 keys at a time belong to one key group or the other."""
    split = LAYOUTS[layout][-1]
    low = lambda t: t // 32 % 2 == odd or t >= split - 64
    late = split // 2 + 32 * odd + 7
    assert late // 32 % 2 == odd
    step, bc = scored_case(layout, dtype, D, split, lambda t: 9.0 if t == late else -128.0 if low(t) else 0.0, lambda t: -1.0 if low(t) else 1.0)
    step.run()
    assert_rows(step.result(), bc, oracle_out(bc), layout)
    assert step.flags() == 0


# --------------------------------------------------------------------------- towards the ends of the types
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_great_values_where_scores_outgrow_the_first_ones(layout, D):
    """A weight of up to 2^99 beside its piece's reference, times values of 2^60."""
    split = LAYOUTS[layout][-1]
    step, bc = scored_case(layout, W.DT_BF16, D, split, lambda t: 9.0 if t == split // 2 + 13 else -128.0, lambda t: 2.0 ** 60 * (1 + t % 2))
    step.run()
    assert_rows(step.result(), bc, oracle_out(bc), layout)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype,k_power,v_power", [
    (W.DT_BF16, 0, -100), (W.DT_BF16, 0, -111), (W.DT_BF16, 0, 80), (W.DT_BF16, 60, 0), (W.DT_BF16, -60, -70), (W.DT_F16, 0, -10), (W.DT_F16, 0, 12), (W.DT_F16, 6, 3),
    (W.DT_F16, -6, 0),
])
def test_keys_and_values_far_from_one(layout, dtype, k_power, v_power):
    """Powers of two on all keys, taken off the queries, and on all values, which come out again."""
    n, group, hkv, batch, announced, split = LAYOUTS[layout]
    r = rng(n + 100)
    case = W.make_case("far", 11, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=128, ctx_lens=[2 * split + 77] * batch,
                       trees=[W.random_tree(n, 6, r) for _ in range(batch)])
    case = dataclasses.replace(case, q=W.store((W.widen(case.q, dtype) * 2.0 ** -k_power).astype(np.float32), dtype))
    bc = make_blocks(case, W.widen(case.k_pool, dtype) * 2.0 ** k_power, W.widen(case.v_pool, dtype) * 2.0 ** v_power)
    step = make_step(bc, announced, split)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc), layout)


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_values_of_zero(layout):
    n, group, hkv, batch, announced, split = LAYOUTS[layout]
    case = W.make_case("zero", 12, dtype=W.DT_BF16, Hq=hkv * group, Hkv=hkv, D=64, ctx_lens=[split + 130] * batch, trees=[W.chain_tree(n)] * batch)
    bc = make_blocks(case, W.widen(case.k_pool, W.DT_BF16), np.zeros(case.v_pool.shape))
    step = make_step(bc, announced, split)
    step.run()
    assert not step.result().any() and step.flags() == 0


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_answers_below_the_least_normal_number(layout):
    """Values of a few of the smallest steps that a block has, 2^-126, of both signs: their means are subnormal in 32 bits."""
    n, group, hkv, batch, announced, split = LAYOUTS[layout]
    case = W.make_case("least", 13, dtype=W.DT_BF16, Hq=hkv * group, Hkv=hkv, D=128, ctx_lens=[2 * split + 77] * batch, trees=[W.chain_tree(n)] * batch)
    bc = make_blocks(case, W.widen(case.k_pool, W.DT_BF16), W.widen(case.v_pool, W.DT_BF16) * 2.0 ** -125)
    step = make_step(bc, announced, split)
    step.run()
    assert_rows(step.result(), bc, oracle_out(bc), layout)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_a_draft_key_that_is_no_number_stays_in_its_subtree(layout, D, dtype):
    n, group, hkv, batch, announced, split = LAYOUTS[layout]
    r = rng(n + D)
    tree = W.random_tree(n, 4, r)
    case = W.make_case("nan", 14, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=[split + 200] * batch, trees=[tree] * batch)
    bc = make_blocks(case, W.widen(case.k_pool, dtype), W.widen(case.v_pool, dtype))
    want, node = oracle_out(bc), n // 2
    step = make_step(bc, announced, split)
    page, slot = int(case.page_table[0, (split + 200 + node) // 16]), (split + 200 + node) % 16
    for g in range(hkv):
        step.k[bc.k._at(page, g, slot).start + 7] = NAN_BYTE
    step.run()
    got = step.result()
    sees = np.zeros(n, bool)
    for i in range(n):
        sees[i] = i == node or (tree[i] >= 0 and sees[tree[i]])
    assert sees.any() and not sees.all() and np.isnan(got[0, sees]).all()
    got[0, sees] = want[0, sees]
    assert_attention(got, bc, want, layout)
