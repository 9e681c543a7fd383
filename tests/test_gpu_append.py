"""Appending rows to the paged cache, rotated on the way, in 16 and 32 bits and in 8-bit blocks: bit for bit what the oracle
says (64-bit arithmetic on both sides, rounded once).  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from block_helpers import DEV, i32, rng
from oracle import cache_blocks as C
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from paper_2510_07535_amd.runner import _to_dev

pytestmark = pytest.mark.gpu


class Append:
    """New rows and a cache with something in it already."""

    def __init__(self, seed, *, dtype, quant, Hq, Hkv, D, ctx, n, rot_dim, pairs=False, rot_scale=1.0, head_major=True, counts=None, pos=None,
                 fused=True, spread=4, rows=None, base=10000.0):
        r = rng(seed)
        self.dtype, self.quant, self.Hq, self.Hkv, self.D, self.n, self.rot_dim, self.pairs = dtype, quant, Hq, Hkv, D, n, rot_dim, pairs
        self.ctx, Bn = np.asarray(ctx, np.int32), len(ctx)
        self.counts = counts
        pages = [(int(L) + n + 15) // 16 for L in ctx]
        self.n_pages, self.table = sum(pages) + 2, np.full((Bn, max(pages)), -1, np.int32)
        order = r.permutation(self.n_pages)
        at = 0
        for b, p in enumerate(pages):
            self.table[b, :p] = order[at:at + p]
            at += p
        self.strides = (Hkv * 16 * D, 16 * D, D) if head_major else (16 * Hkv * D, D, Hkv * D)
        shape = (self.n_pages, Hkv, 16, D) if head_major else (self.n_pages, 16, Hkv, D)
        if quant:
            self.k, self.v = (C.Blocks(r.integers(0, 256, shape).astype(np.uint8) & 0xF7, r.integers(118, 128, (self.n_pages, Hkv)), self.strides, D, dtype)
                              for _ in range(2))
        else:
            self.k, self.v = (W.store(r.standard_normal(shape).astype(np.float32), dtype) for _ in range(2))
        heads = Hq + 2 * Hkv
        x = r.standard_normal((Bn, n, heads, D)) * np.exp2(r.integers(-spread, spread + 1, (Bn, n, heads, 1)))
        self.x = W.store(x.astype(np.float32), dtype) if rows is None else rows(W.store(x.astype(np.float32), dtype))
        self.inv_freq = (base ** (-np.arange(rot_dim // 2) / max(1, rot_dim // 2))).astype(np.float32)
        self.pos = pos
        es = 4 if dtype == W.DT_F32 else 2
        wide = heads * D
        self.desc = B.make_desc(batch=Bn, n_draft=min(n, 64), n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, max_pages_per_seq=self.table.shape[1],
                                max_ctx_len=int(self.ctx.max()), qkv_dtype=dtype, scale=1.0, kv_stride_page=self.strides[0], kv_stride_head=self.strides[1],
                                kv_stride_token=self.strides[2], n_pool_pages=self.n_pages)
        self.app = B.AppendDesc(n_tokens=n, rot_dim=rot_dim, rot_style=B.OWL_ROT_PAIRS if pairs else B.OWL_ROT_HALVES, rot_scale=rot_scale,
                                q_stride=wide if fused else Hq * D, k_stride=wide if fused else Hkv * D, v_stride=wide if fused else Hkv * D)
        self.rot_scale = rot_scale
        x = _to_dev(self.x.reshape(Bn, n, wide), DEV)
        self.dq, self.dk, self.dv = x.split([Hq * D, Hkv * D, Hkv * D], dim=-1)
        if not fused:
            self.dq, self.dk, self.dv = self.dq.contiguous(), self.dk.contiguous(), self.dv.contiguous()
        self.fused_rows = x
        self.q_out = torch.full((Bn, n, Hq, D), 7, dtype=x.dtype, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.dtable, self.dlens, self.dcounts = i32(self.table), i32(self.ctx), i32(counts)
        self.freq = torch.from_numpy(self.inv_freq).to(DEV) if rot_dim else None
        if quant:
            self.dev = [torch.from_numpy(t).to(DEV) for t in (self.k.flat, self.v.flat, self.k.scale, self.v.scale)]
        else:
            self.dev = [_to_dev(t, DEV) for t in (self.k, self.v)]

    def run(self, q=True, q_out=None):
        a = (self.desc, self.app, self.dq if q else None, self.dk, self.dv, self.freq, i32(self.pos), (self.q_out if q_out is None else q_out) if q else None)
        call = B.owl_append_kv_quant if self.quant else B.owl_append_kv
        call(*a, *self.dev, self.dtable, self.dlens, self.dcounts, self.status)
        torch.cuda.synchronize()

    def want(self):
        """(q [B][n][Hq][D], K, V) as the oracle has them; rows of absent tokens of q are left at 7."""
        counts = np.full(len(self.ctx), self.n) if self.counts is None else np.clip(self.counts, 0, self.n)
        pos = self.pos if self.pos is not None else self.ctx[:, None] + np.arange(self.n)
        q, k, v = self.x[:, :, :self.Hq], self.x[:, :, self.Hq:self.Hq + self.Hkv], self.x[:, :, self.Hq + self.Hkv:]
        q, k, v = C.rotated_rows(q, k, v, pos, self.inv_freq, self.rot_dim, self.pairs, self.rot_scale, self.dtype)
        full = np.full(q.shape, 7, q.dtype)
        for b, c in enumerate(counts):
            full[b, :c] = q[b, :c]
        if not self.quant:
            return full, *(C.append(p, x, self.table, self.ctx, counts, self.strides) for p, x in ((self.k, k), (self.v, v)))
        pools = self.k.copy(), self.v.copy()
        for p, x in zip(pools, (k, v)):
            p.append(x, self.table, self.ctx, counts)
        return full, *pools

    def check(self, want=None, q=True):
        wq, wk, wv = self.want() if want is None else want
        if q:
            got = self.q_out.cpu().numpy().view(wq.dtype)
            assert np.array_equal(got, wq), f"{np.sum(got != wq)} of {wq.size}"
        if not self.quant:
            for d, w in zip(self.dev, (wk, wv)):
                assert np.array_equal(d.cpu().numpy().view(w.dtype).reshape(w.shape), w)
            return
        for d, s, w in zip(self.dev[:2], self.dev[2:], (wk, wv)):
            assert np.array_equal(s.cpu().numpy(), w.scale)
            assert C.same_bytes(d.cpu().numpy(), w.flat)


TYPES = [(W.DT_BF16, False), (W.DT_F16, False), (W.DT_F32, False), (W.DT_BF16, True), (W.DT_F16, True)]


@pytest.mark.parametrize("dtype,quant", TYPES)
@pytest.mark.parametrize("Hq,Hkv,D,ctx,n,rot_dim,pairs,head_major,fused", [
    (4, 1, 64, [0], 1, 64, False, True, True), (8, 2, 128, [5003], 1, 128, False, True, True), (8, 2, 128, [15, 16, 17, 0], 6, 128, False, False, True),
    (6, 2, 128, [100, 31], 60, 64, True, True, False), (8, 8, 64, [33], 64, 32, False, False, False), (3, 1, 128, [1, 47], 17, 16, True, True, True),
    (4, 4, 128, [250], 33, 0, False, True, True), (32, 8, 128, [70], 5, 128, True, True, True), (2, 2, 64, [12], 300, 64, False, True, True),
])
def test_append_matches_the_oracle(dtype, quant, Hq, Hkv, D, ctx, n, rot_dim, pairs, head_major, fused):
    a = Append(n + D + rot_dim, dtype=dtype, quant=quant, Hq=Hq, Hkv=Hkv, D=D, ctx=ctx, n=n, rot_dim=rot_dim, pairs=pairs, head_major=head_major, fused=fused)
    a.run()
    a.check()
    assert int(a.status.item()) == 0


@pytest.mark.parametrize("dtype,quant", TYPES)
def test_positions_of_a_tree_far_ones_and_a_scale(dtype, quant):
    """Position ids of their own, up to 2^31 - 1 and below zero, and a factor on the turned channels."""
    pos = np.array([[0, 131071, 1 << 20, (1 << 31) - 1, -5, 99999, 7], [3, 3, 4, 4, 5, 1 << 30, 1000003]], np.int64)
    a = Append(3, dtype=dtype, quant=quant, Hq=4, Hkv=2, D=128, ctx=[40, 7], n=7, rot_dim=128, pos=pos, rot_scale=1.1386, base=500000.0)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype,quant", TYPES)
def test_sequences_with_fewer_new_tokens_and_without_queries(dtype, quant):
    counts = np.array([9, 0, 4, 1, 12, -3], np.int32)
    a = Append(4, dtype=dtype, quant=quant, Hq=4, Hkv=2, D=64, ctx=[30, 5, 16, 0, 47, 3], n=9, rot_dim=64, counts=counts)
    a.run()
    a.check()
    assert int(a.status.item()) == B.OWL_DEV_BAD_NDRAFT  # 12 and -3
    a = Append(5, dtype=dtype, quant=quant, Hq=4, Hkv=2, D=64, ctx=[30, 5], n=9, rot_dim=64)
    a.run(q=False)
    a.check(q=False)
    assert (a.q_out == 7).all()


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("Hkv,D,pairs", [(2, 128, False), (3, 64, True)])
def test_blocks_with_gaps_between_their_rows(dtype, Hkv, D, pairs):
    """Bytes between rows, heads and pages, that stay as they are."""
    a = Append(15, dtype=dtype, quant=True, Hq=2 * Hkv, Hkv=Hkv, D=D, ctx=[21, 40, 0], n=19, rot_dim=D // 2, pairs=pairs)
    head, token = D + 16, Hkv * (D + 16) + 32
    page = 16 * token + 48
    a.strides, r = (page, head, token), rng(16)
    a.desc.kv_stride_page, a.desc.kv_stride_head, a.desc.kv_stride_token = a.strides
    a.k, a.v = (C.Blocks(r.integers(0, 256, a.n_pages * page).astype(np.uint8) & 0xF7, x.scale, a.strides, D, dtype) for x in (a.k, a.v))
    a.dev = [torch.from_numpy(t).to(DEV) for t in (a.k.flat, a.v.flat, a.k.scale, a.v.scale)]
    a.run()
    a.check()


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
def test_a_sequence_without_new_tokens_keeps_its_block(dtype):
    """Its rows could do with a smaller scale; the other sequence's block, of the same kind, gets one."""
    a = Append(14, dtype=dtype, quant=True, Hq=4, Hkv=2, D=64, ctx=[5, 5, 0], n=3, rot_dim=64, counts=np.array([0, 3, 0], np.int32), spread=0)
    for blocks, raw, scale in ((a.k, a.dev[0], a.dev[2]), (a.v, a.dev[1], a.dev[3])):
        blocks.flat &= 0xBF                              # magnitudes below 2
        blocks.scale += 4
        raw &= 0xBF
        scale += 4
    before = [t.clone() for t in a.dev]
    a.run()
    a.check()
    for got, was in zip(a.dev[2:], before[2:]):
        assert torch.equal(got[a.table[0, 0]], was[a.table[0, 0]]) and (got[a.table[1, 0]] < was[a.table[1, 0]]).all()


@pytest.mark.parametrize("dtype,quant", [(W.DT_BF16, False), (W.DT_F32, False), (W.DT_F16, True)])
def test_queries_in_place(dtype, quant):
    a = Append(6, dtype=dtype, quant=quant, Hq=8, Hkv=2, D=128, ctx=[11], n=21, rot_dim=96, fused=False)
    a.run(q_out=a.dq)
    a.q_out = a.dq.view(a.q_out.shape)
    a.check()


@pytest.mark.parametrize("dtype,quant", TYPES)
def test_bad_pages_and_lengths_drop_their_rows_only(dtype, quant):
    a = Append(7, dtype=dtype, quant=quant, Hq=2, Hkv=2, D=64, ctx=[30, 20, 40], n=40, rot_dim=64)
    wq, wk, wv = a.want()
    # the second page of sequence 0's new rows, and all rows of sequence 2
    table = a.table.copy()
    table[0, 3] = a.n_pages
    a.dtable, a.dlens = i32(table), i32([30, 20, 41])
    lost = [int(a.table[0, 3])] + [int(p) for p in a.table[2] if p >= 0]
    a.run()
    assert int(a.status.item()) == B.OWL_DEV_BAD_PAGE | B.OWL_DEV_BAD_CTX_LEN
    if quant:
        for w, old in ((wk, a.k), (wv, a.v)):
            for page in lost:
                for g in range(2):
                    for slot in range(16):
                        w.flat[w._at(page, g, slot)] = old.flat[old._at(page, g, slot)]
                w.scale[page] = old.scale[page]
    else:
        for w, old in ((wk, a.k), (wv, a.v)):
            w[lost] = old[lost]
    a.check((wq, wk, wv), q=False)
    got = a.q_out.cpu().numpy().view(wq.dtype)
    assert np.array_equal(got[:2], wq[:2])


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
def test_blocks_of_extreme_rows(dtype):
    """Zeros, infinities and no numbers, the ends of the type, numbers that sink below a block's steps, ties."""
    def rows(x):
        wide = W.widen(x, dtype).astype(np.float32)
        wide[0, :16] = 0.0
        wide[0, 16, :, 0], wide[0, 17, :, 1], wide[0, 18, :, 2] = np.nan, np.inf, -np.inf
        wide[0, 32:48] *= {W.DT_BF16: 2.0 ** 120, W.DT_F16: 2.0 ** 11}[dtype]
        wide[0, 40, :, 5] = {W.DT_BF16: 3.3895e38, W.DT_F16: 65504.0}[dtype]
        wide[0, 48:64] *= {W.DT_BF16: 2.0 ** -125, W.DT_F16: 2.0 ** -18}[dtype]
        wide[0, 64:80] = np.exp2(np.arange(16) % 16 - 13.0)[:, None, None] * 1.0625       # ties of the coarse steps
        with np.errstate(over="ignore"):
            return W.store(wide, dtype)
    a = Append(8, dtype=dtype, quant=True, Hq=1, Hkv=1, D=64, ctx=[0], n=80, rot_dim=0, rows=rows)
    a.run()
    a.check()


def test_appending_the_same_rows_again_changes_nothing():
    a = Append(9, dtype=W.DT_BF16, quant=True, Hq=2, Hkv=2, D=128, ctx=[23], n=10, rot_dim=128)
    a.run()
    before = [t.clone() for t in a.dev]
    a.run()
    assert all(torch.equal(x, y) for x, y in zip(before, a.dev))


@pytest.mark.parametrize("quant", [False, True])
def test_graph_replays_match_eager(quant):
    a = Append(10, dtype=W.DT_BF16, quant=quant, Hq=8, Hkv=2, D=128, ctx=[90, 33], n=24, rot_dim=128)
    b = Append(10, dtype=W.DT_BF16, quant=quant, Hq=8, Hkv=2, D=128, ctx=[90, 33], n=24, rot_dim=128)
    a.run()
    b.run()                                              # (loads the kernel)
    call = B.owl_append_kv_quant if quant else B.owl_append_kv
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call(a.desc, a.app, a.dq, a.dk, a.dv, a.freq, None, a.q_out, *a.dev, a.dtable, a.dlens, None, a.status)
    for rep in range(3):
        for s in (a, b):
            s.dlens.copy_(torch.tensor([90 - 20 * rep, 33 - rep], dtype=torch.int32))
            s.fused_rows.copy_(s.fused_rows.flip(-1))
        graph.replay()
        b.run()
        assert torch.equal(a.q_out, b.q_out) and all(torch.equal(x, y) for x, y in zip(a.dev, b.dev)), rep


def test_a_far_place_in_a_large_pool():
    """Offsets beyond 2^32 bytes."""
    D, Hkv, pages = 128, 8, 150000                        # 4.9 GB a tensor in 16 bits
    for quant in (False, True):
        kind = torch.uint8 if quant else torch.bfloat16
        k, v = (torch.zeros((pages, Hkv, 16, D), dtype=kind, device=DEV) for _ in range(2))
        if quant:
            k, v = k.repeat(2, 1, 1, 1), v.repeat(2, 1, 1, 1)
        last = k.shape[0] - 1
        scales = [torch.full((k.shape[0], Hkv), 127, dtype=torch.uint8, device=DEV) for _ in range(2)] if quant else []
        x = torch.randn((1, 2, 3 * Hkv * D), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(torch.bfloat16)
        x = x.clamp(-1.75, 1.75).mul(4).round().div(4)                    # exact in a block
        desc = B.make_desc(batch=1, n_draft=2, n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=D, max_pages_per_seq=2, max_ctx_len=15, qkv_dtype=B.OWL_BF16,
                           scale=1.0, kv_stride_page=Hkv * 16 * D, kv_stride_head=16 * D, kv_stride_token=D, n_pool_pages=k.shape[0])
        app = B.AppendDesc(n_tokens=2, rot_dim=0, rot_style=0, rot_scale=1.0, q_stride=3 * Hkv * D, k_stride=3 * Hkv * D, v_stride=3 * Hkv * D)
        q, kn, vn = x.split(Hkv * D, dim=-1)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        call = B.owl_append_kv_quant if quant else B.owl_append_kv
        call(desc, app, None, kn, vn, None, None, None, k, v, *scales, i32([[last - 1, last]]), i32([15]), None, status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for pool, rows, t in ((k, kn, 0), (v, vn, 1)):
            for page, slot, i in ((last - 1, 15, 0), (last, 0, 1)):
                got = pool[page, :, slot]
                if quant:
                    got = got.view(torch.float8_e4m3fn).float() * torch.exp2(scales[t][page].float() - 127)[:, None]
                assert torch.equal(got.float(), rows[0, i].view(Hkv, D).float())
        del k, v
