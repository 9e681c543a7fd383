"""The verify attention over caches of 8-bit blocks and the commit in them, against the oracles.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from block_helpers import DEV, NAN_BYTE, QuantStep, assert_attention, block_case, i32, oracle_out, rng
from oracle import cache_blocks as C
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W

pytestmark = pytest.mark.gpu


def _trees(kind, n, count, r):
    return [W.chain_tree(n) if kind == "chain" or (kind == "mix" and i % 2) else W.random_tree(n, 6, r) for i in range(count)]


# --------------------------------------------------------------------------- attention
# rows per KV head from one tile to several row groups, pieces shorter and longer than a page, odd lengths
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group,hkv,ctx", [
    (1, 4, 2, [0]), (1, 1, 1, [1]), (1, 4, 2, [15]), (3, 4, 2, [16]), (6, 4, 2, [17]), (4, 8, 1, [63]), (60, 1, 2, [64]), (16, 4, 2, [1000]),
    (26, 4, 2, [2047]), (40, 4, 1, [700]), (40, 8, 2, [1500]), (60, 8, 1, [900]), (64, 8, 1, [333]), (5, 3, 3, [5003]), (2, 4, 8, [4500]),
])
def test_attention_matches_the_oracle(dtype, D, n, group, hkv, ctx):
    r = rng(n * 1000 + D + dtype)
    bc = block_case("quant", 7 + n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=ctx, trees=_trees("tree", n, 1, r),
                    head_major=n % 2 == 0, spare_pages=3)
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc), f"{n} {group} {hkv} {ctx}")
    assert step.flags() == 0


@pytest.mark.parametrize("dtype,D,n,group,hkv,ctx,split", [
    (W.DT_BF16, 128, 26, 4, 2, [0, 1, 700, 33, 1029], 0), (W.DT_F16, 128, 7, 4, 2, [300, 0, 0, 2000], 0),
    (W.DT_BF16, 64, 40, 8, 1, [500, 16, 48, 15, 17, 900], 0), (W.DT_F16, 64, 12, 4, 4, [640] * 9, 0),
    (W.DT_BF16, 128, 20, 8, 2, [513, 64, 65], 128), (W.DT_F16, 128, 60, 4, 1, [1300, 77], 192),
])
def test_batches_with_drafts_of_different_sizes(dtype, D, n, group, hkv, ctx, split):
    r = rng(len(ctx) * 100 + n)
    bc = block_case("quant-batch", 31 + n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=ctx, trees=_trees("mix", n, len(ctx), r))
    for counts in (None, r.integers(0, n + 1, len(ctx))):
        step = QuantStep(bc, counts=counts, split_tokens=split, flags=B.OWL_FLAG_FP32_PARTIALS if split else 0)
        step.run()
        assert_attention(step.result(), bc, oracle_out(bc, counts), str(counts))
        assert step.flags() == 0


@pytest.mark.parametrize("n,group,hkv,ctx", [(26, 4, 2, 20000), (60, 4, 2, 9000), (40, 8, 1, 30000), (6, 4, 1, 40000)])
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
def test_long_contexts(n, group, hkv, ctx, dtype):
    """Many stages a piece, pairs of wavefronts, row groups: against the 16-bit path's oracle on sampled rows."""
    import oracle
    from util import sample_rows
    r = rng(ctx)
    bc = block_case("quant-long", ctx, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=128, ctx_lens=[ctx], trees=_trees("tree", n, 1, r), outlier_frac=0.02)
    step = QuantStep(bc)
    step.run()
    got, rows = step.result(), sample_rows(bc.case, 64)
    want = oracle.verify_attn_case(bc.case, rows=rows)
    assert_attention(got[rows[:, 0], rows[:, 1], rows[:, 2]], bc, want)
    assert np.isfinite(got).all() and step.flags() == 0


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("group,n", [(4, 6), (4, 26), (8, 40)])
def test_pages_of_very_different_scales(dtype, group, n):
    """Neighbouring pages differ by up to 2^10 (fp16: 2^6) in their scales, of K and of V each."""
    r = rng(5 * n)
    top = 5 if dtype == W.DT_BF16 else 3
    bc = block_case("quant-scales", 3, page_gain=lambda g, k: 2.0 ** g.integers(-top, top + 1, k), dtype=dtype, Hq=2 * group, Hkv=2, D=128,
                    ctx_lens=[1111], trees=_trees("tree", n, 1, r), scale=0.02)
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


@pytest.mark.parametrize("group,n,ctx", [(4, 5, 3000), (4, 26, 2500), (8, 40, 1800), (4, 60, 1200)])
def test_fp16_scores_that_outgrow_the_first_ones(group, n, ctx):
    """Late keys far longer than the early ones: the frozen references of the fp16 loops overflow and pieces are redone."""
    r = rng(ctx)
    bc = block_case("quant-overflow", 17, page_gain=None, dtype=W.DT_F16, Hq=2 * group, Hkv=2, D=128, ctx_lens=[ctx],
                    trees=_trees("tree", n, 1, r), outlier_frac=0.05, outlier_gain=16.0)
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


@pytest.mark.parametrize("gain", [8.0, 32.0, 64.0])
@pytest.mark.parametrize("group,n,ctx", [(4, 5, 3000), (4, 26, 2500), (8, 40, 1800), (4, 60, 1200)])
def test_bf16_scores_that_outgrow_the_first_ones(group, n, ctx, gain):
    """The same in bf16, with its exponents: scores that lie some 40, 160 and 320 (as powers of two) above the first ones."""
    r = rng(ctx + int(gain))
    bc = block_case("quant-overflow", 17, page_gain=None, dtype=W.DT_BF16, Hq=2 * group, Hkv=2, D=128, ctx_lens=[ctx],
                    trees=_trees("tree", n, 1, r), outlier_frac=0.05, outlier_gain=gain)
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ctx", [[2111], [900, 31, 1500]])
@pytest.mark.parametrize("n", [4, 8, 11, 16, 20, 24, 28, 32, 36])
def test_every_number_of_row_tiles(n, ctx, D):
    r = rng(n * 3 + D)
    bc = block_case("quant-tiles", n + D, dtype=W.DT_F16 if n % 8 else W.DT_BF16, Hq=8, Hkv=2, D=D, ctx_lens=ctx, trees=_trees("tree", n, len(ctx), r))
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))
    assert step.flags() == 0


def _announced(bc, most):
    """A step whose sequences may be ``most`` long: its work is dealt out as that of long ones."""
    step = QuantStep(bc)
    wide = (most + bc.case.N + 15) // 16
    table = np.full((bc.case.B, wide), -1, np.int32)
    table[:, :bc.case.page_table.shape[1]] = bc.case.page_table
    step.table = i32(table)
    step.desc.max_ctx_len, step.desc.max_pages_per_seq = most, wide
    step.workspace = torch.empty(B.owl_verify_attn_quant_workspace_size(step.desc), dtype=torch.uint8, device=DEV)
    return step


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,group", [(20, 4), (28, 4), (32, 4), (40, 4), (60, 4), (40, 8), (64, 8), (50, 16)])
def test_sequences_announced_as_long_ones(n, group, D, dtype):
    """Every layout of the loop that many rows share, on lengths of a few stages to some seventy."""
    r = rng(n + group + D)
    for hkv, ctx in ((2, [4500]), (1, [700]), (2, [1, 1030, 64])):
        bc = block_case("quant-announced", n, dtype=dtype, Hq=hkv * group, Hkv=hkv, D=D, ctx_lens=ctx, trees=_trees("tree", n, len(ctx), r))
        step = _announced(bc, 1 << 20)
        step.run()
        assert_attention(step.result(), bc, oracle_out(bc), f"{hkv} {ctx}")
        assert step.flags() == 0


@pytest.mark.parametrize("dtype,gain", [(W.DT_BF16, 32.0), (W.DT_BF16, 64.0), (W.DT_F16, 4.0), (W.DT_F16, 16.0)])
@pytest.mark.parametrize("n,group", [(28, 4), (32, 4), (60, 4), (40, 8)])
def test_outgrown_references_of_sequences_announced_as_long_ones(n, group, dtype, gain):
    r = rng(n + int(gain))
    bc = block_case("quant-outgrown", 3, dtype=dtype, Hq=2 * group, Hkv=2, D=128, ctx_lens=[3001], trees=_trees("tree", n, 1, r), outlier_frac=0.05,
                    outlier_gain=gain)
    step = _announced(bc, 1 << 20)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
def test_more_row_groups_than_an_xcd_has_compute_units(dtype):
    r = rng(9)
    bc = block_case("quant-rows", 9, dtype=dtype, Hq=32, Hkv=1, D=128, ctx_lens=[500], trees=_trees("tree", 64, 1, r))
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,long", [(6, False), (40, False), (60, True)])
def test_gaps_between_rows_heads_and_pages(n, long, D, dtype):
    r = rng(n + D)
    bc = block_case("quant-gaps", 4, dtype=dtype, Hq=8, Hkv=2, D=D, ctx_lens=[1203], trees=_trees("tree", n, 1, r))
    step = _announced(bc, 1 << 20) if long else QuantStep(bc)
    token = 2 * (D + 16) + 32
    strides = (16 * token + 48, D + 16, token)
    for name, blocks in (("k", bc.k), ("v", bc.v)):
        wide = C.Blocks(np.full(bc.case.n_pool_pages * strides[0], NAN_BYTE, np.uint8), blocks.scale, strides, D, dtype)
        for page in range(bc.case.n_pool_pages):
            for g in range(2):
                for slot in range(16):
                    wide.flat[wide._at(page, g, slot)] = blocks.flat[blocks._at(page, g, slot)]
        setattr(step, name, torch.from_numpy(wide.flat).to(DEV))
    step.desc.kv_stride_page, step.desc.kv_stride_head, step.desc.kv_stride_token = strides
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


def test_captured_calls_on_two_streams_at_once():
    """A short and an announced-as-long sequence, each in a graph on its own stream with its own workspace, replayed side by side."""
    r = rng(12)
    steps, graphs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for long, n, dtype in ((False, 12, W.DT_F16), (True, 40, W.DT_BF16)):
        bc = block_case("quant-two", n, dtype=dtype, Hq=16, Hkv=2, D=128, ctx_lens=[2100], trees=_trees("tree", n, 1, r))
        step = _announced(bc, 1 << 20) if long else QuantStep(bc)
        B.owl_verify_attn_quant_init(step.desc)
        step.run()
        steps.append((step, step.result(), bc))
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
        for step, want, bc in steps:
            got = step.result()
            assert np.array_equal(got, want), rep
    for step, want, bc in steps:
        assert_attention(want, bc, oracle_out(bc))


@pytest.mark.parametrize("n,long", [(6, False), (60, True)])
def test_pages_beyond_32_bit_offsets(n, long):
    """The attention and the commit where pages lie 4 GB behind the first one."""
    r = rng(n)
    bc = block_case("quant-far", 4, dtype=W.DT_BF16, Hq=32, Hkv=8, D=128, ctx_lens=[700], trees=_trees("tree", n, 1, r))
    step = _announced(bc, 1 << 20) if long else QuantStep(bc)
    page, count = 8 * 16 * 128, bc.case.n_pool_pages
    pages = (1 << 32) // page + 2 * count
    far = pages - count
    for name in ("k", "v", "ks", "vs"):
        near = getattr(step, name)
        wide = torch.empty(pages * (near.numel() // count), dtype=torch.uint8, device=DEV)
        wide[far * (near.numel() // count):] = near.reshape(-1)
        setattr(step, name, wide)
    step.table = torch.where(step.table >= 0, step.table + far, step.table)
    step.desc.n_pool_pages = pages
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))
    acc = np.full((1, n), -1, np.int32)
    acc[0, :3] = 1, 2, 5
    B.owl_commit_kv_quant(step.desc, step.k, step.v, step.ks, step.vs, step.table, step.lens, i32(acc), i32([3]), None, step.status)
    for blocks, raw, scale in ((bc.k, step.k, step.ks), (bc.v, step.v, step.vs)):
        want = blocks.copy()
        want.commit(bc.case.page_table, bc.case.ctx_lens, acc, [3])
        assert np.array_equal(scale[far * 8:].cpu().numpy().reshape(want.scale.shape), want.scale)
        assert C.same_bytes(raw[far * page:].cpu().numpy(), want.flat)
    assert step.flags() == 0


def test_answers_in_16_bits_and_zeros_of_absent_nodes():
    r = rng(1)
    for dtype, kind in ((W.DT_BF16, B.OWL_BF16), (W.DT_F16, B.OWL_F16)):
        bc = block_case("quant-out", 5, dtype=dtype, Hq=8, Hkv=2, D=128, ctx_lens=[300, 20], trees=_trees("tree", 9, 2, r))
        full, half = QuantStep(bc, counts=[9, 4]), QuantStep(bc, out_dtype=kind, counts=[9, 4])
        full.run()
        half.run()
        want = full.out.to(half.out.dtype)
        torch.cuda.synchronize()
        assert torch.equal(half.out, want) and not half.out[1, 4:].any()


def test_identity_paging():
    bc = block_case("quant-flat", 8, dtype=W.DT_BF16, Hq=4, Hkv=1, D=128, ctx_lens=[777], trees=[W.chain_tree(4)], paged=False, head_major=False)
    assert bc.case.page_table is None
    step = QuantStep(bc)
    step.run()
    assert_attention(step.result(), bc, oracle_out(bc))


def test_bad_pages_lengths_and_counts_are_flagged_and_stay_in_bounds():
    r = rng(2)
    bc = block_case("quant-bad", 9, dtype=W.DT_BF16, Hq=8, Hkv=2, D=128, ctx_lens=[400, 200], trees=_trees("tree", 5, 2, r))
    ref = QuantStep(bc)
    ref.run()
    want = ref.result()
    step = QuantStep(bc)
    step.table[0, 3] = bc.case.n_pool_pages
    step.run()
    got = step.result()
    assert step.flags() == B.OWL_DEV_BAD_PAGE and np.array_equal(got[1], want[1])
    step = QuantStep(bc, counts=[9, -1])
    step.run()
    assert not step.result()[1].any() and step.flags() == B.OWL_DEV_BAD_NDRAFT
    step = QuantStep(bc)
    step.lens[1] = 100000
    step.run()
    assert np.array_equal(step.result()[0], want[0]) and step.flags() & B.OWL_DEV_BAD_CTX_LEN


def test_graph_replays_match_eager():
    r = rng(3)
    bc = block_case("quant-graph", 61, dtype=W.DT_BF16, Hq=16, Hkv=4, D=128, ctx_lens=[1500, 40, 700], trees=_trees("tree", 12, 3, r))
    step = QuantStep(bc)
    B.owl_verify_attn_quant_init(step.desc)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step.run()
    torch.cuda.synchronize()
    for rep in range(4):
        step.lens.copy_(torch.tensor([1500 - 100 * rep, 40, 700 - 300 * (rep % 2)], dtype=torch.int32))
        step.ks.copy_(torch.from_numpy(bc.k.scale + np.where(bc.k.scale < 200, rep % 3, 0).astype(np.uint8)))
        step.out.fill_(float("nan"))
        graph.replay()
        got = step.result()
        step.out.fill_(float("nan"))
        step.run()
        assert np.array_equal(got, step.result()), rep
    assert step.flags() == 0


# --------------------------------------------------------------------------- commit
def _commit(bc, acc, na, table=None, new=True):
    c = bc.case
    step = QuantStep(bc)
    if table is not None:
        step.table = i32(table)
    new_lens = torch.full((c.B,), -7, dtype=torch.int32, device=DEV) if new else None
    B.owl_commit_kv_quant(step.desc, step.k, step.v, step.ks, step.vs, step.table, step.lens, i32(acc), i32(na), new_lens, step.status)
    return step, new_lens


def _same(step, k, v):
    torch.cuda.synchronize()
    for got, scale, want in ((step.k, step.ks, k), (step.v, step.vs, v)):
        assert np.array_equal(scale.cpu().numpy(), want.scale)
        assert C.same_bytes(got.cpu().numpy(), want.flat)


def _paths(B_, N, r, most):
    acc, na = np.full((B_, N), -1, np.int32), np.zeros(B_, np.int32)
    for b in range(B_):
        na[b] = r.integers(0, most + 1)
        acc[b, :na[b]] = np.sort(r.choice(N, na[b], replace=False))
    return acc, na


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,most,head_major", [(1, 1, True), (6, 6, True), (40, 8, False), (64, 64, True), (64, 20, False)])
def test_commit_matches_the_oracle(dtype, D, N, most, head_major):
    r = rng(N * 10 + D + dtype)
    ctx = [0, 1, 15, 16, 31, 100, 333]
    bc = block_case("commit", N, page_gain=lambda g, k: 2.0 ** g.integers(-9, 7, k), dtype=dtype, Hq=3, Hkv=3, D=D, ctx_lens=ctx,
                    trees=[W.chain_tree(N)] * len(ctx), head_major=head_major, spare_pages=2)
    acc, na = _paths(len(ctx), N, r, most)
    if N == 64 and most == 64:
        acc[0], na[0] = np.arange(64), 64                # all in place
        acc[2, :63], na[2] = np.arange(1, 64), 63        # all move by one
        acc[2, 63] = -1
        na[4], acc[4] = 0, -1
    k, v = bc.k.copy(), bc.v.copy()
    for blocks in (k, v):
        blocks.commit(bc.case.page_table, bc.case.ctx_lens, acc, na)
    step, new_lens = _commit(bc, acc, na)
    _same(step, k, v)
    assert step.flags() == 0 and new_lens.cpu().numpy().tolist() == (bc.case.ctx_lens + na).tolist()


def test_commit_without_lengths_and_with_identity_paging():
    bc = block_case("commit-flat", 4, dtype=W.DT_BF16, Hq=2, Hkv=2, D=128, ctx_lens=[21], trees=[W.chain_tree(20)], paged=False)
    acc, na = np.full((1, 20), -1, np.int32), np.array([3], np.int32)
    acc[0, :3] = [2, 9, 19]
    k, v = bc.k.copy(), bc.v.copy()
    for blocks in (k, v):
        blocks.commit(None, [21], acc, na)
    step, _ = _commit(bc, acc, na, new=False)
    _same(step, k, v)


def test_commit_flags_bad_lists_pages_and_lengths_and_moves_nothing_there():
    r = rng(8)
    bc = block_case("commit-bad", 6, dtype=W.DT_BF16, Hq=2, Hkv=2, D=64, ctx_lens=[30, 100, 50, 60], trees=[W.chain_tree(12)] * 4)
    acc, na = np.full((4, 12), -1, np.int32), np.array([2, 3, 2, 2], np.int32)
    acc[0, :2], acc[1, :3], acc[2, :2], acc[3, :2] = [3, 3], [0, 1, 12], [4, 7], [5, 11]
    table = bc.case.page_table.copy()
    table[3, (60 + 11) // 16] = -1
    k, v = bc.k.copy(), bc.v.copy()
    for blocks in (k, v):
        blocks.commit(bc.case.page_table, bc.case.ctx_lens, acc, [0, 0, 2, 0])
    step, new_lens = _commit(bc, acc, na, table=table)
    _same(step, k, v)
    assert step.flags() == B.OWL_DEV_BAD_ACCEPT | B.OWL_DEV_BAD_PAGE
    assert new_lens.cpu().numpy().tolist() == [30, 100, 52, 60]
    step, new_lens = _commit(bc, acc, np.array([0, 99, 0, -3], np.int32))
    _same(step, bc.k, bc.v)
    assert step.flags() == B.OWL_DEV_BAD_ACCEPT


def test_a_second_commit_of_rows_in_place_changes_nothing():
    r = rng(12)
    bc = block_case("commit-twice", 14, dtype=W.DT_F16, Hq=2, Hkv=2, D=128, ctx_lens=[45], trees=[W.chain_tree(10)])
    acc, na = np.full((1, 10), -1, np.int32), np.array([4], np.int32)
    acc[0, :4] = [1, 4, 5, 9]
    step, _ = _commit(bc, acc, na)
    torch.cuda.synchronize()
    before = [x.clone() for x in (step.k, step.v, step.ks, step.vs)]
    B.owl_commit_kv_quant(step.desc, step.k, step.v, step.ks, step.vs, step.table, step.lens, i32([[0, 1, 2, 3] + [-1] * 6]), i32(na), None, step.status)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (step.k, step.v, step.ks, step.vs)))
