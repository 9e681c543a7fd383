"""The verify attention over caches of 4-bit groups with queries and keys from one end of bf16 to the other: a row's answer is what the 64-bit
oracle says wherever its products of queries and keys fit into 32 bits, as in a 16-bit cache.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from block_helpers import DEV, assert_attention, i32, oracle_out, rng
from group_helpers import GroupStep, group_case
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from paper_2510_07535_amd.runner import _to_dev

pytestmark = pytest.mark.gpu

# (nodes, query heads a KV head, greatest length announced, keys of a wavefront's own, tiles a wavefront, row groups): both kernels, each loop
LAYOUTS = {
    "own keys, 1 tile": (4, 4, None, True, 1, 1), "own keys, 2 tiles": (7, 4, 1 << 17, True, 2, 1), "own keys, 2 groups": (16, 4, 40000, True, 2, 2),
    "shared, groups of 2 tiles": (12, 4, None, False, 1, 2), "shared, 3 tiles in all": (12, 4, 1 << 20, False, 2, 1),
    "shared, 7 tiles": (28, 4, 1 << 20, False, 2, 1), "shared, 15 tiles": (60, 4, 1 << 20, False, 2, 1), "shared, 20 tiles": (40, 8, 1 << 20, False, 3, 1),
}
FIRST_OWN = 77                   # of the instantiated kernels, those with keys of a wavefront's own are the last


def _step(layout, D, q_exp, k_exp, scale_exp, spread=0):
    """Queries of about 2^q_exp (rows of up to 2^spread less), keys of about 2^k_exp, scores of up to a few dozen."""
    n, group, announced, own, tiles, groups = LAYOUTS[layout]
    r = rng(n + D)
    gc = group_case("groups-range", n, dtype=W.DT_BF16, Hq=2 * group, Hkv=2, D=D, ctx_lens=[900], trees=[W.random_tree(n, 6, r)], scale=2.0 ** scale_exp)
    c = gc.case
    fine = gc.scale[0] != 255
    gc.scale[0][fine] += np.uint8(k_exp % 256)
    assert gc.scale[0][fine].min() >= 2 and gc.scale[0][fine].max() <= 252
    c.k_pool[...] = W.store(W.widen(c.k_pool, c.dtype) * np.float32(2.0 ** k_exp), c.dtype)
    rows = np.exp2(q_exp - r.integers(0, spread + 1, c.q.shape[:-1] + (1,)).astype(np.float64))
    c.q[...] = W.store((W.widen(c.q, c.dtype) * rows).astype(np.float32), c.dtype)
    step = GroupStep(gc, max_ctx_len=announced)
    if announced is not None:
        wide = (announced + n + 15) // 16
        table = np.full((1, wide), -1, np.int32)
        table[:, :c.page_table.shape[1]] = c.page_table
        step.table, step.desc.max_pages_per_seq = i32(table), wide
        step.ws = torch.full((B.owl_verify_attn_groups_workspace_size(step.desc),), 0xFF, dtype=torch.uint8, device=DEV)
    plan = B.owl_verify_attn_groups_plan(step.desc)
    assert (plan.kernel_variant >= FIRST_OWN, plan.tiles_per_wave, plan.row_groups) == (own, tiles, groups)
    return step, gc


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_exp,k_exp,scale_exp", [(0, 115, -118), (0, 120, -123), (-15, 124, -112), (-60, 124, -67), (-110, 114, -7), (-120, 124, -7),
                                                   (3, 112, -118), (60, 60, -123), (118, -118, -3), (100, -60, -43), (-100, -20, 117), (0, 0, -3)])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_queries_and_keys_of_all_sizes(layout, q_exp, k_exp, scale_exp, D):
    step, gc = _step(layout, D, q_exp, k_exp, scale_exp)
    assert_attention(step.result(), gc, oracle_out(gc), layout)
    assert int(step.status.item()) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_exp,k_exp,scale_exp,spread", [(0, 120, -123, 100), (-20, 124, -107, 60), (10, 112, -125, 30)])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_rows_of_different_sizes_against_great_keys(layout, q_exp, k_exp, scale_exp, spread, D):
    step, gc = _step(layout, D, q_exp, k_exp, scale_exp, spread)
    assert_attention(step.result(), gc, oracle_out(gc), layout)
    assert int(step.status.item()) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_a_great_channel_that_no_key_has(layout, D):
    """Queries of 2^113 .. 2^114 but for one channel of 2^122, which is 0 in all keys; the keys' others are 0 or 2^-126; a scale of 2^15.  The scores are
    some dozens."""
    step, gc = _step(layout, D, 0, 0, 0)
    c, r = gc.case, rng(D)
    step.desc.scale = c.scale = 2.0 ** 15
    signs = r.integers(0, 3, c.k_pool.shape).astype(np.uint8)
    signs[..., 0] = 0
    codes = np.where(signs == 2, 9, signs).astype(np.uint8)              # 0, 1/2, -1/2
    live = (gc.scale[0] != 255).repeat(32, -1).reshape(signs.shape)
    step.k.copy_(torch.from_numpy(codes[..., 0::2] | codes[..., 1::2] << 4).reshape(step.k.shape))
    step.ks[step.ks != 255] = 2                                          # 2^-125
    c.k_pool[...] = np.where(live, W.store(np.array([0.0, 2.0 ** -126, -2.0 ** -126], np.float32)[signs], W.DT_BF16), 0)
    c.q[...] = W.store((r.choice([-1.0, 1.0], c.q.shape) * r.uniform(1.0, 1.99, c.q.shape) * 2.0 ** 113).astype(np.float32), W.DT_BF16)
    c.q[..., 0] = W.store(np.full(1, 2.0 ** 122, np.float32), W.DT_BF16)
    step.q.copy_(_to_dev(c.q, DEV))
    assert_attention(step.result(), gc, oracle_out(gc), layout)
    assert int(step.status.item()) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,above", [(W.DT_BF16, 7), (W.DT_BF16, 9), (W.DT_BF16, 10), (W.DT_BF16, 12), (W.DT_F16, 4), (W.DT_F16, 6), (W.DT_F16, 9), (W.DT_F16, 12)])
@pytest.mark.parametrize("layout", [k for k in LAYOUTS if k != "shared, 20 tiles"])
def test_channels_far_below_their_rows_greatest(layout, dtype, above, D):
    """One channel of q is 2^above greater than the others, with keys that are all 1 there, so that the others' products decide."""
    n, group, announced, own, tiles, groups = LAYOUTS[layout]
    r = rng(n + above + D)
    gc = group_case("groups-channels", n, dtype=dtype, Hq=2 * group, Hkv=2, D=D, ctx_lens=[900], trees=[W.random_tree(n, 6, r)])
    c, hot = gc.case, 37
    byte, scale = gc.raw[0][..., hot // 2], gc.scale[0][..., hot // 32]
    fine = scale != 255
    code = np.zeros(scale.shape, np.uint8)
    for e, k in ((-2, 6), (-1, 4), (0, 2)):                              # 1 as 4 / 4, 2 / 2, 1
        code[scale == 127 + e] = k
    assert (code[fine] > 0).all()
    byte[fine] = (byte[fine] & 15) | code[fine] << 4                     # (an odd channel: the upper half)
    c.k_pool[..., hot][fine] = W.store(np.ones(1, np.float32), dtype)
    q = W.widen(c.q, dtype)
    q[..., hot] = np.sign(q[..., hot]) * 2.0 ** above
    c.q[...] = W.store(q.astype(np.float32), dtype)
    step = GroupStep(gc, max_ctx_len=announced)
    if announced is not None:
        wide = (announced + n + 15) // 16
        table = np.full((1, wide), -1, np.int32)
        table[:, :c.page_table.shape[1]] = c.page_table
        step.table, step.desc.max_pages_per_seq = i32(table), wide
        step.ws = torch.full((B.owl_verify_attn_groups_workspace_size(step.desc),), 0xFF, dtype=torch.uint8, device=DEV)
    plan = B.owl_verify_attn_groups_plan(step.desc)
    assert (plan.kernel_variant >= FIRST_OWN, plan.tiles_per_wave, plan.row_groups) == (own, tiles, groups)
    assert_attention(step.result(), gc, oracle_out(gc), layout)
    assert int(step.status.item()) == 0
