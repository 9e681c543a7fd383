"""The verify attention over caches of 4-bit groups, against the fp64 oracle of the 16-bit path on the numbers that the groups stand for.
Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

import oracle
from block_helpers import DEV, assert_attention, i32, oracle_out, rng
from group_helpers import GroupStep, group_case
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from util import sample_rows

pytestmark = pytest.mark.gpu

# (assert_attention's bound beside the weights' rounding, 2^-10 of the greatest value, holds here too: a query is off by at most 2^-17 of its
# row's greatest number in channels below 2^-9 of that (bf16; fp16 2^-6), which moves a score of D products with keys of a few units by less than 2^-12 as well.)


def _trees(kind, n, count, r):
    return [W.chain_tree(n) if kind == "chain" or (kind == "mix" and i % 2) else W.random_tree(n, 6, r) for i in range(count)]


def _announced(gc, most, **kw):
    """A step whose sequences may be ``most`` long: its work is dealt out as that of long ones."""
    step = GroupStep(gc, **kw)
    wide = (most + gc.case.N + 15) // 16
    table = np.full((gc.case.B, wide), -1, np.int32)
    table[:, :gc.case.page_table.shape[1]] = gc.case.page_table
    step.table = i32(table)
    step.desc.max_ctx_len, step.desc.max_pages_per_seq = most, wide
    step.ws = torch.full((B.owl_verify_attn_groups_workspace_size(step.desc),), 0xFF, dtype=torch.uint8, device=DEV)
    return step


def _check(step, gc, what="", counts=None):
    assert_attention(step.result(), gc, oracle_out(gc, counts), what)
    assert int(step.status.item()) == 0


# rows per KV head from one tile to several row groups, pieces shorter and longer than a page, odd lengths
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group,hkv,ctx", [
    (1, 4, 2, [0]), (1, 1, 1, [1]), (1, 4, 2, [15]), (3, 4, 2, [16]), (6, 4, 2, [17]), (4, 8, 1, [63]), (60, 1, 2, [64]), (16, 4, 2, [1000]),
    (26, 4, 2, [2047]), (40, 4, 1, [700]), (40, 8, 2, [1500]), (60, 8, 1, [900]), (64, 8, 1, [333]), (5, 3, 3, [5003]), (2, 4, 8, [4500]),
])
def test_attention_matches_the_oracle(dtype, D, n, group, hkv, ctx):
    r = rng(n * 1000 + D + dtype)
    gc = group_case("groups", 7 + n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=ctx, trees=_trees("tree", n, 1, r), head_major=n % 2 == 0,
                    spare_pages=3)
    _check(GroupStep(gc), gc, f"{n} {group} {hkv} {ctx}")


@pytest.mark.parametrize("dtype,D,n,group,hkv,ctx,split", [
    (W.DT_BF16, 128, 26, 4, 2, [0, 1, 700, 33, 1029], 0), (W.DT_F16, 128, 7, 4, 2, [300, 0, 0, 2000], 0),
    (W.DT_BF16, 64, 40, 8, 1, [500, 16, 48, 15, 17, 900], 0), (W.DT_F16, 64, 12, 4, 4, [640] * 9, 0),
    (W.DT_BF16, 128, 20, 8, 2, [513, 64, 65], 128), (W.DT_F16, 128, 60, 4, 1, [1300, 77], 192), (W.DT_BF16, 128, 1, 4, 2, [300, 5, 64, 2000], 64),
    (W.DT_BF16, 128, 2, 4, 2, [40 * i for i in range(70)], 0),
])
def test_batches_with_drafts_of_different_sizes(dtype, D, n, group, hkv, ctx, split):
    r = rng(len(ctx) * 100 + n)
    gc = group_case("groups-batch", 31 + n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=ctx, trees=_trees("mix", n, len(ctx), r))
    for counts in (None, r.integers(0, n + 1, len(ctx))):
        step = GroupStep(gc, counts=counts, split_tokens=split, flags=B.OWL_FLAG_FP32_PARTIALS if split else 0)
        _check(step, gc, str(counts), counts)


@pytest.mark.parametrize("dtype,D,n,group,hkv,ctx,split", [
    (W.DT_BF16, 128, 16, 4, 2, 5000, 128), (W.DT_F16, 64, 28, 4, 8, 9000, 256), (W.DT_BF16, 128, 5, 4, 2, 3001, 64), (W.DT_BF16, 128, 40, 8, 2, 6000, 512),
    (W.DT_F16, 128, 1, 8, 1, 2500, 192), (W.DT_BF16, 64, 60, 4, 4, 2111, 320),
])
def test_lone_sequences_in_equal_splits(dtype, D, n, group, hkv, ctx, split):
    r = rng(ctx + n)
    gc = group_case("groups-splits", 41 + n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=[ctx], trees=_trees("tree", n, 1, r))
    _check(GroupStep(gc, split_tokens=split), gc)


@pytest.mark.parametrize("n,group,hkv,ctx", [(26, 4, 2, 20000), (60, 4, 2, 9000), (40, 8, 1, 30000), (6, 4, 1, 40000), (1, 4, 1, 70001)])
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
def test_long_contexts(n, group, hkv, ctx, dtype):
    """Many stages a piece, row groups: sampled rows."""
    r = rng(ctx)
    gc = group_case("groups-long", ctx, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=128, ctx_lens=[ctx], trees=_trees("tree", n, 1, r), outlier_frac=0.02)
    step = GroupStep(gc)
    got, rows = step.result(), sample_rows(gc.case, 64)
    assert_attention(got[rows[:, 0], rows[:, 1], rows[:, 2]], gc, oracle.verify_attn_case(gc.case, rows=rows))
    assert np.isfinite(got).all() and int(step.status.item()) == 0


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("group,n", [(4, 1), (4, 6), (4, 26), (8, 40)])
def test_pages_of_very_different_scales(dtype, group, n):
    r = rng(5 * n)
    top = 5 if dtype == W.DT_BF16 else 3
    gc = group_case("groups-scales", 3, gain=lambda g, k: 2.0 ** g.integers(-top, top + 1, k), dtype=dtype, Hq=2 * group, Hkv=2, D=128, ctx_lens=[1111],
                    trees=_trees("tree", n, 1, r), scale=0.02)
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("dtype,gain", [(W.DT_BF16, 8.0), (W.DT_BF16, 32.0), (W.DT_BF16, 64.0), (W.DT_F16, 4.0), (W.DT_F16, 16.0)])
@pytest.mark.parametrize("group,n,ctx", [(4, 1, 5000), (4, 5, 3000), (4, 26, 2500), (8, 40, 1800), (4, 60, 1200)])
def test_scores_that_outgrow_the_first_ones(group, n, ctx, dtype, gain):
    """Late keys far longer than the early ones: references move, by up to some 320 powers of two."""
    r = rng(ctx + int(gain))
    gc = group_case("groups-outgrown", 17, dtype=dtype, Hq=2 * group, Hkv=2, D=128, ctx_lens=[ctx], trees=_trees("tree", n, 1, r), outlier_frac=0.05,
                    outlier_gain=gain)
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ctx", [[2111], [900, 31, 1500]])
@pytest.mark.parametrize("n", [4, 8, 11, 16, 20, 24, 28, 32, 36, 40, 44, 48, 52, 60, 64])
def test_every_number_of_row_tiles(n, ctx, D):
    r = rng(n * 3 + D)
    gc = group_case("groups-tiles", n + D, dtype=W.DT_F16 if n % 8 else W.DT_BF16, Hq=8, Hkv=2, D=D, ctx_lens=ctx, trees=_trees("tree", n, len(ctx), r))
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group", [(1, 4), (5, 4), (9, 4), (20, 4), (28, 4), (32, 4), (40, 4), (60, 4), (40, 8), (64, 8), (50, 16)])
def test_sequences_announced_as_long_ones(n, group, D, dtype):
    """Every layout of the loops, on lengths of a few stages to some seventy."""
    r = rng(n + group + D)
    for hkv, ctx in ((2, [4500]), (1, [700]), (2, [1, 1030, 64])):
        gc = group_case("groups-announced", n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=ctx, trees=_trees("tree", n, len(ctx), r))
        _check(_announced(gc, 1 << 20), gc, f"{hkv} {ctx}")


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [9, 16, 20, 28, 41, 60])
def test_row_groups_with_keys_of_their_own(n, D, dtype):
    """A lone sequence of two KV heads that may be 40000 long: up to eight groups of two row tiles."""
    r = rng(n + 3 * D)
    for ctx in (4500, 700, 31, 0):
        gc = group_case("groups-own", n, dtype=dtype, Hq=8, Hkv=2, D=D, ctx_lens=[ctx], trees=_trees("tree", n, 1, r))
        step = _announced(gc, 40000)
        plan, tiles = B.owl_verify_attn_groups_plan(step.desc), (4 * n + 15) // 16
        assert (plan.tiles_per_wave, plan.row_groups) == (2, (tiles + 1) // 2)
        _check(step, gc, str(ctx))


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
def test_more_row_groups_than_an_xcd_has_compute_units(dtype):
    r = rng(9)
    gc = group_case("groups-rows", 9, dtype=dtype, Hq=32, Hkv=1, D=128, ctx_lens=[500], trees=_trees("tree", 64, 1, r))
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 6, 40, 60])
def test_gaps_between_rows_heads_and_pages(n, D, dtype):
    r = rng(n + D)
    gc = group_case("groups-gaps", 4, dtype=dtype, Hq=8, Hkv=2, D=D, ctx_lens=[1203], trees=_trees("tree", n, 1, r), head_major=True)
    for step in (GroupStep(gc), _announced(gc, 1 << 20)):
        w = D // 2
        token = 2 * (w + 16) + 32
        strides = (16 * token + 48, w + 16, token)
        for name, raw in zip(("k", "v"), gc.raw):
            wide = np.full(gc.case.n_pool_pages * strides[0], 0xFF, np.uint8)
            for page in range(gc.case.n_pool_pages):
                for g in range(2):
                    for slot in range(16):
                        at = page * strides[0] + g * strides[1] + slot * token
                        wide[at:at + w] = raw[page, g, slot]
            setattr(step, name, torch.from_numpy(wide).to(DEV))
        step.desc.kv_stride_page, step.desc.kv_stride_head, step.desc.kv_stride_token = strides
        _check(step, gc)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,spread", [(W.DT_BF16, 30), (W.DT_F16, 6)])
@pytest.mark.parametrize("n", [1, 6, 60])
def test_queries_of_very_different_sizes(n, dtype, spread, D):
    """Rows from 2^-spread to 2^spread, keys to match: every row has a scale of its own.  Channels of a row differ by up to 2^8."""
    r = rng(n + spread)
    gc = group_case("groups-queries", 6, dtype=dtype, Hq=4, Hkv=1, D=D, ctx_lens=[777], trees=_trees("tree", n, 1, r), scale=2.0 ** -8)
    q = W.widen(gc.case.q, dtype).astype(np.float64)
    rows = 2.0 ** r.integers(-spread, 4, q.shape[:-1] + (1,))
    chans = 2.0 ** r.integers(-8, 1, q.shape)
    gc.case.q[...] = W.store((q * rows * chans).astype(np.float32), dtype)
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("n", [1, 26])
def test_queries_of_zeros_and_of_the_types_ends(n, dtype):
    """Rows of zeros weigh all keys alike; the greatest and the least numbers are taken."""
    r = rng(n)
    gc = group_case("groups-ends", 6, dtype=dtype, Hq=4, Hkv=1, D=128, ctx_lens=[300], trees=[W.chain_tree(n)], scale=2.0 ** (-126 if dtype == W.DT_BF16 else -16))
    q = W.widen(gc.case.q, dtype).astype(np.float64)
    q[:, :, 0] = 0.0
    q[:, :, 1] = {W.DT_BF16: 2.0 ** 126, W.DT_F16: 2.0 ** 15}[dtype] * np.sign(q[:, :, 1])
    q[:, :, 2] *= {W.DT_BF16: 2.0 ** -126, W.DT_F16: 2.0 ** -14}[dtype]
    gc.case.q[...] = W.store(q.astype(np.float32), dtype)
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n", [1, 7, 40])
def test_queries_that_are_no_numbers_spoil_their_own_rows_only(n, bad):
    gc = group_case("groups-none", 8, dtype=W.DT_BF16, Hq=8, Hkv=2, D=128, ctx_lens=[500], trees=[W.chain_tree(n)])
    want = GroupStep(gc).result()
    q = W.widen(gc.case.q, W.DT_BF16)
    q[0, n // 2, 5, 77] = bad
    gc.case.q[...] = W.store(q, W.DT_BF16)
    got = GroupStep(gc).result()
    assert np.isnan(got[0, n // 2, 5]).all()
    got[0, n // 2, 5] = want[0, n // 2, 5]
    assert np.array_equal(got, want)


@pytest.mark.parametrize("n", [2, 7, 40])
def test_keys_and_values_that_are_no_numbers(n):
    """A draft's key that is none spoils the rows that see it, a value that is none all rows of its sequence and KV head."""
    gc = group_case("groups-none", 8, dtype=W.DT_F16, Hq=8, Hkv=2, D=64, ctx_lens=[200, 300], trees=[W.chain_tree(n)] * 2)
    want = GroupStep(gc).result()
    at = lambda b, p: (int(gc.case.page_table[b, p // 16]), p % 16)
    step = GroupStep(gc)
    page, slot = at(0, 200 + n - 1)                      # the last node of the chain: only it sees itself
    step.ks[page, 1, slot, 0] = 255
    got = step.result()
    assert np.isnan(got[0, n - 1, 4:]).all()
    got[0, n - 1, 4:] = want[0, n - 1, 4:]
    assert np.array_equal(got, want)
    step = GroupStep(gc)
    page, slot = at(1, 33)
    step.vs[page, 0, slot, 1] = 255                      # channels 32 .. 63
    got = step.result()
    assert np.isnan(got[1, :, :4, 32:]).all()
    got[1, :, :4] = want[1, :, :4]
    assert np.array_equal(got, want)


def test_captured_calls_on_two_streams_at_once():
    r = rng(12)
    steps, graphs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for long, n, dtype in ((False, 2, W.DT_F16), (True, 40, W.DT_BF16)):
        gc = group_case("groups-two", n, dtype=dtype, Hq=16, Hkv=2, D=128, ctx_lens=[2100], trees=_trees("tree", n, 1, r))
        step = _announced(gc, 1 << 20) if long else GroupStep(gc)
        B.owl_verify_attn_groups_init(step.desc)
        steps.append((step, step.result(), gc))
    for (step, _, _), stream in zip(steps, streams):
        graph = torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                step.run()
        graphs.append(graph)
    torch.cuda.synchronize()
    for rep in range(4):
        for step, _, _ in steps:
            step.out.fill_(float("nan"))
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for step, want, gc in steps:
            assert np.array_equal(step.out.cpu().numpy(), want), rep
    for step, want, gc in steps:
        assert_attention(want, gc, oracle_out(gc))


def test_graphs_that_share_a_workspace_one_after_the_other():
    r = rng(13)
    cases = [group_case("groups-shared", n, dtype=W.DT_BF16, Hq=8, Hkv=2, D=128, ctx_lens=[ctx], trees=_trees("tree", n, 1, r)) for n, ctx in ((3, 900), (30, 2000))]
    steps = [GroupStep(gc) for gc in cases]
    big = torch.empty(max(s.ws.numel() for s in steps), dtype=torch.uint8, device=DEV)
    want, graphs = [], []
    for s in steps:
        s.ws = big
        want.append(s.result())
    for s in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        graphs.append(graph)
    for rep in range(3):
        for i in (0, 1, 1, 0):
            steps[i].out.fill_(float("nan"))
            graphs[i].replay()
            torch.cuda.synchronize()
            assert np.array_equal(steps[i].out.cpu().numpy(), want[i]), rep


def test_graph_replays_follow_the_lengths():
    r = rng(3)
    gc = group_case("groups-graph", 61, stale_none=False, dtype=W.DT_BF16, Hq=16, Hkv=4, D=128, ctx_lens=[1500, 40, 700], trees=_trees("tree", 12, 3, r))
    step = GroupStep(gc)
    B.owl_verify_attn_groups_init(step.desc)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for rep in range(4):
        step.lens.copy_(torch.tensor([1500 - 100 * rep, 40, 700 - 300 * (rep % 2)], dtype=torch.int32))
        step.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = step.out.cpu().numpy()
        step.out.fill_(float("nan"))
        assert np.array_equal(got, step.result()), rep
    assert int(step.status.item()) == 0


@pytest.mark.parametrize("n,long", [(1, False), (6, False), (60, True)])
def test_pages_beyond_32_bit_offsets(n, long):
    """Pages 4 GB behind the first one."""
    r = rng(n)
    gc = group_case("groups-far", 4, dtype=W.DT_BF16, Hq=32, Hkv=8, D=128, ctx_lens=[700], trees=_trees("tree", n, 1, r))
    step = _announced(gc, 1 << 20) if long else GroupStep(gc)
    page, count = 8 * 16 * 64, gc.case.n_pool_pages
    pages = (1 << 32) // page + 2 * count
    far = pages - count
    for name in ("k", "v", "ks", "vs"):
        near = getattr(step, name)
        wide = torch.empty(pages * (near.numel() // count), dtype=torch.uint8, device=DEV)
        wide[far * (near.numel() // count):] = near.reshape(-1)
        setattr(step, name, wide)
    step.table = torch.where(step.table >= 0, step.table + far, step.table)
    step.desc.n_pool_pages = pages
    _check(step, gc)


def test_answers_in_16_bits_and_zeros_of_absent_nodes():
    r = rng(1)
    for dtype, kind in ((W.DT_BF16, B.OWL_BF16), (W.DT_F16, B.OWL_F16)):
        gc = group_case("groups-out", 5, dtype=dtype, Hq=8, Hkv=2, D=128, ctx_lens=[300, 20], trees=_trees("tree", 9, 2, r))
        full, half = GroupStep(gc, counts=[9, 4]), GroupStep(gc, out_dtype=kind, counts=[9, 4])
        full.run()
        half.run()
        torch.cuda.synchronize()
        assert torch.equal(half.out, full.out.to(half.out.dtype)) and not half.out[1, 4:].any()


def test_identity_paging():
    gc = group_case("groups-flat", 8, dtype=W.DT_BF16, Hq=4, Hkv=1, D=128, ctx_lens=[777], trees=[W.chain_tree(4)], paged=False, head_major=True)
    assert gc.case.page_table is None
    _check(GroupStep(gc), gc)


@pytest.mark.parametrize("n", [2, 5, 30])
def test_bad_pages_lengths_and_counts_are_flagged_and_stay_in_bounds(n):
    r = rng(2)
    gc = group_case("groups-bad", 9, stale_none=False, dtype=W.DT_BF16, Hq=8, Hkv=2, D=128, ctx_lens=[400, 200], trees=_trees("tree", n, 2, r))
    want = GroupStep(gc).result()
    step = GroupStep(gc)
    step.table[0, 3] = gc.case.n_pool_pages
    got = step.result()
    assert int(step.status.item()) == B.OWL_DEV_BAD_PAGE and np.array_equal(got[1], want[1])
    step = GroupStep(gc, counts=[99, -1])
    assert not step.result()[1].any() and int(step.status.item()) == B.OWL_DEV_BAD_NDRAFT
    step = GroupStep(gc)
    step.lens[1] = 100000                                # (counts as the greatest: the shares, and the order of the first sequence's sums, are others)
    assert_attention(step.result()[:1], gc, oracle_out(gc)[:1])
    assert int(step.status.item()) & B.OWL_DEV_BAD_CTX_LEN
    step = GroupStep(gc)
    step.dparent[0, 1] = 7
    got = step.result()
    assert np.array_equal(got[1], want[1]) and int(step.status.item()) == B.OWL_DEV_BAD_PARENT


def test_two_calls_give_the_same_bits():
    r = rng(4)
    for n, ctx in ((1, [9000]), (26, [3000, 17, 800])):
        gc = group_case("groups-twice", 4, dtype=W.DT_BF16, Hq=16, Hkv=4, D=128, ctx_lens=ctx, trees=_trees("tree", n, len(ctx), r))
        step = GroupStep(gc)
        assert np.array_equal(step.result(), step.result())
