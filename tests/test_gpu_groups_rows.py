"""Caches of 4-bit groups: the commit of accepted rows and reading rows back, bit for bit.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from block_helpers import DEV, i32, rng
from group_helpers import values
from oracle import cache_groups as G
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W

pytestmark = pytest.mark.gpu


class Cache:
    def __init__(self, seed, *, Hkv, D, ctx, n, dtype=W.DT_BF16, head_major=True, table=True, gap=0):
        r = rng(seed)
        self.Hkv, self.D, self.n, self.dtype, self.ctx = Hkv, D, n, dtype, np.asarray(ctx, np.int32)
        pages = [(int(L) + n + 15) // 16 for L in ctx]
        self.n_pages = sum(pages) + 3
        self.table = None
        if table:
            self.table = np.full((len(ctx), max(pages)), -1, np.int32)
            order, at = r.permutation(self.n_pages), 0
            for b, p in enumerate(pages):
                self.table[b, :p] = order[at:at + p]
                at += p
        w = D // 2
        self.strides = (Hkv * 16 * w + gap, 16 * w, w) if head_major else (16 * Hkv * w + gap, w, Hkv * w)
        low, high = G.ENDS[dtype]
        self.held = [G.Groups(r.integers(0, 256, (self.n_pages, self.strides[0])), r.integers(low + 127, high + 128, (self.n_pages, Hkv, 16, D // 32)),
                              self.strides, D, dtype) for _ in range(2)]
        for h in self.held:
            h.scale[r.random(h.scale.shape) < 0.02] = 255
        self.dev = [torch.from_numpy(x).to(DEV) for x in (self.held[0].flat, self.held[1].flat, self.held[0].scale, self.held[1].scale)]
        self.desc = B.make_desc(batch=len(ctx), n_draft=min(n, 64), n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=D,
                                max_pages_per_seq=0 if self.table is None else self.table.shape[1], max_ctx_len=int(self.ctx.max()), qkv_dtype=dtype,
                                scale=1.0, kv_stride_page=self.strides[0], kv_stride_head=self.strides[1], kv_stride_token=self.strides[2],
                                n_pool_pages=self.n_pages)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.dtable, self.lens = i32(self.table), i32(self.ctx)

    def same(self, held):
        torch.cuda.synchronize()
        return all(np.array_equal(d.cpu().numpy(), h.flat) and np.array_equal(s.cpu().numpy(), h.scale) for d, s, h in zip(self.dev[:2], self.dev[2:], held))

    def commit(self, accepted, count, new=True, stream=None):
        self.new = torch.full((len(self.ctx),), -9, dtype=torch.int32, device=DEV) if new else None
        B.owl_commit_kv_groups(self.desc, *self.dev, self.dtable, self.lens, i32(accepted), i32(count), self.new, self.status, stream)


def _paths(r, Bn, n, depth):
    accepted, count = np.full((Bn, n), -1, np.int32), r.integers(0, depth + 1, Bn).astype(np.int32)
    count[0] = depth
    for b in range(Bn):
        accepted[b, :count[b]] = np.sort(r.permutation(n)[:count[b]])
    return accepted, count


@pytest.mark.parametrize("Hkv,D,ctx,n,depth,head_major,table", [
    (8, 128, [65], 60, 6, True, True), (2, 64, [0, 15, 16, 100], 40, 8, False, True), (1, 128, [47, 1], 64, 64, True, True), (3, 64, [7], 1, 1, True, True),
    (5, 128, [1000, 31, 32, 33, 5], 13, 13, False, True), (2, 128, [50], 20, 9, True, False), (1, 64, [3, 90], 64, 33, True, True),
])
def test_commit_moves_rows_with_their_scales(Hkv, D, ctx, n, depth, head_major, table):
    c = Cache(n + depth, Hkv=Hkv, D=D, ctx=ctx, n=n, head_major=head_major, table=table, gap=32)
    accepted, count = _paths(rng(n), len(ctx), n, depth)
    c.commit(accepted, count)
    for h in c.held:
        h.commit(c.table, ctx, accepted, count)
    assert c.same(c.held)
    assert np.array_equal(c.new.cpu().numpy(), c.ctx + count) and int(c.status.item()) == 0


@pytest.mark.parametrize("path,count,bit", [
    ([3, 3, 5], 3, B.OWL_DEV_BAD_ACCEPT), ([5, 3, 6], 3, B.OWL_DEV_BAD_ACCEPT), ([1, 2, 9], 3, B.OWL_DEV_BAD_ACCEPT), ([-1, 2, 3], 3, B.OWL_DEV_BAD_ACCEPT),
    ([1, 2, 3], 10, B.OWL_DEV_BAD_ACCEPT), ([1, 2, 3], -1, B.OWL_DEV_BAD_ACCEPT), ([0, 1, 2], 3, 0), ([2, 4, 8], 0, 0),
])
def test_commit_bad_paths_and_paths_in_place_move_nothing(path, count, bit):
    c = Cache(5, Hkv=2, D=128, ctx=[30, 9], n=9)
    accepted = np.full((2, 9), -1, np.int32)
    accepted[0, :3] = path
    accepted[1, :2] = [2, 7]
    count = np.array([count, 2], np.int32)
    c.commit(accepted, count)
    for h in c.held:
        h.commit(c.table, [30, 9], np.stack([np.arange(9), accepted[1]]), [0, 2])
    assert c.same(c.held) and int(c.status.item()) == bit
    assert c.new.tolist() == [30 + (3 if bit == 0 and count[0] == 3 else 0), 11]


def test_commit_bad_pages_and_lengths():
    c = Cache(6, Hkv=2, D=64, ctx=[30, 9, 4], n=9)
    c.dtable[0, 2] = c.n_pages                           # positions 32 .. 38 of the first sequence
    c.lens[2] = 31                                       # beyond max_ctx_len: clamped, its pages end before
    accepted = np.array([[1, 4, 8] + [-1] * 6, [0, 5] + [-1] * 7, [3] + [-1] * 8], np.int32)
    c.commit(accepted, np.array([3, 2, 0], np.int32))
    for h in c.held:
        h.commit(c.table, [30, 9, 4], accepted, [0, 2, 0])
    assert c.same(c.held)
    assert int(c.status.item()) == B.OWL_DEV_BAD_PAGE | B.OWL_DEV_BAD_CTX_LEN and c.new.tolist() == [30, 11, 30]


def test_commit_without_new_lengths_captured_and_on_a_stream():
    c = Cache(7, Hkv=4, D=128, ctx=[40], n=12)
    accepted = np.array([[2, 3, 7, 11] + [-1] * 8], np.int32)
    da, dn = i32(accepted), i32(np.array([4], np.int32))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.owl_commit_kv_groups(c.desc, *c.dev, c.dtable, c.lens, da, dn, None, c.status)
    for _ in range(3):                                   # each moves what the one before left
        graph.replay()
        torch.cuda.synchronize()
        for h in c.held:
            h.commit(c.table, [40], accepted, [4])
        assert c.same(c.held)


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("Hkv,D,ctx,first,n,head_major,table", [
    (8, 128, [200], 0, 200, True, True), (8, 128, [200], 13, 1, True, True), (3, 64, [100, 77], 5, 80, False, True), (1, 128, [64], 15, 18, True, False),
    (5, 64, [40], 0, 1, True, True), (9, 128, [33], 16, 17, False, True), (2, 64, [3000], 1, 2999, True, True), (17, 64, [31], 7, 20, True, True),
])
def test_gather_reads_what_groups_stand_for(dtype, Hkv, D, ctx, first, n, head_major, table):
    c = Cache(first + n, Hkv=Hkv, D=D, ctx=ctx, n=8, dtype=dtype, head_major=head_major, table=table, gap=16)
    t = {W.DT_BF16: torch.bfloat16, W.DT_F16: torch.float16}[dtype]
    seq = len(ctx) - 1
    n = min(n, ctx[seq] + 8 - first)
    for which in (0, 1):
        dst = torch.full((n + 2, Hkv, D), 5.0, dtype=t, device=DEV)
        B.owl_gather_kv_groups(c.desc, c.dev[which], c.dev[2 + which], c.dtable, seq, first, n, dst, c.status)
        torch.cuda.synchronize()
        want = np.stack([[c.held[which].row(p // 16 if c.table is None else int(c.table[seq, p // 16]), g, p % 16) for g in range(Hkv)]
                         for p in range(first, first + n)])
        got = dst[:n].double().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)
        assert (dst[n:] == 5).all()
    assert int(c.status.item()) == 0


def test_gather_of_no_rows_and_of_bad_pages():
    c = Cache(9, Hkv=2, D=128, ctx=[60], n=4)
    dst = torch.full((40, 2, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    B.owl_gather_kv_groups(c.desc, c.dev[0], c.dev[2], c.dtable, 0, 3, 0, dst, c.status)
    torch.cuda.synchronize()
    assert (dst == 5).all() and int(c.status.item()) == 0
    c.dtable[0, 1] = -7
    B.owl_gather_kv_groups(c.desc, c.dev[0], c.dev[2], c.dtable, 0, 10, 40, dst, c.status)
    torch.cuda.synchronize()
    page = lambda p: 0 if p // 16 == 1 else int(c.table[0, p // 16])
    want = np.stack([[c.held[0].row(page(p), g, p % 16) for g in range(2)] for p in range(10, 50)])
    assert np.array_equal(dst.double().cpu().numpy(), want, equal_nan=True) and int(c.status.item()) == B.OWL_DEV_BAD_PAGE
    c.status.zero_()
    B.owl_gather_kv_groups(c.desc, c.dev[0], c.dev[2], c.dtable, 0, c.table.shape[1] * 16 - 2, 4, dst, c.status)      # past the table
    torch.cuda.synchronize()
    assert int(c.status.item()) == B.OWL_DEV_BAD_PAGE


def test_gather_far_pages():
    """Pages more than 4 GB behind the first one."""
    free, _ = torch.cuda.mem_get_info()
    assert free > 12 << 30
    Hkv, D = 1, 128
    stride = 1 << 20
    pages = 4500
    pool = torch.zeros(pages * stride, dtype=torch.uint8, device=DEV)
    r = rng(10)
    raw = r.integers(0, 256, (16, 64)).astype(np.uint8)
    scale = r.integers(110, 140, (pages, Hkv, 16, 4)).astype(np.uint8)
    pool[4400 * stride:4400 * stride + 1024] = torch.from_numpy(raw.reshape(-1)).to(DEV)
    desc = B.make_desc(batch=1, n_draft=1, n_q_heads=1, n_kv_heads=1, head_dim=D, max_pages_per_seq=1, max_ctx_len=10, qkv_dtype=W.DT_BF16, scale=1.0,
                       kv_stride_page=stride, kv_stride_head=1024, kv_stride_token=64, n_pool_pages=pages)
    dst = torch.empty((16, 1, D), dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.owl_gather_kv_groups(desc, pool, torch.from_numpy(scale).to(DEV), i32(np.array([[4400]])), 0, 0, 16, dst, status)
    torch.cuda.synchronize()
    assert np.array_equal(dst[:, 0].double().cpu().numpy(), values(raw, scale[4400, 0])) and int(status.item()) == 0
