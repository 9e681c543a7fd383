"""Appending rows with norms of the heads, to caches of 16 and 32 bits and of 8-bit blocks, and with or without them to caches of 4-bit
groups: bit for bit what the oracle says (64-bit arithmetic on both sides, rounded once).  Needs an MI355X (-m gpu)."""
import ctypes

import numpy as np
import pytest
import torch

from block_helpers import DEV, i32, rng
from oracle import cache_blocks as C
from oracle import cache_groups as G
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from paper_2510_07535_amd.runner import _to_dev

pytestmark = pytest.mark.gpu


class Rows:
    """New rows, norms and a cache with something in it already.  cache: "own", "blocks" or "groups"."""

    def __init__(self, seed, *, dtype, cache, Hq, Hkv, D, ctx, n, rot_dim, pairs=False, rot_scale=1.0, head_major=True, counts=None, pos=None,
                 fused=True, spread=4, norm=True, gains=True, eps=1e-5, rows=None, page_gap=0):
        r = rng(seed)
        self.dtype, self.cache, self.Hq, self.Hkv, self.D, self.n, self.rot_dim, self.pairs = dtype, cache, Hq, Hkv, D, n, rot_dim, pairs
        self.ctx, Bn = np.asarray(ctx, np.int32), len(ctx)
        self.counts, self.pos, self.rot_scale, self.norm, self.eps = counts, pos, rot_scale, norm, eps
        pages = [(int(L) + n + 15) // 16 for L in ctx]
        self.n_pages, self.table = sum(pages) + 2, np.full((Bn, max(pages)), -1, np.int32)
        order, at = r.permutation(self.n_pages), 0
        for b, p in enumerate(pages):
            self.table[b, :p] = order[at:at + p]
            at += p
        w = D // 2 if cache == "groups" else D
        self.strides = (Hkv * 16 * w + page_gap, 16 * w, w) if head_major else (16 * Hkv * w + page_gap, w, Hkv * w)
        shape = (self.n_pages, self.strides[0])
        if cache == "groups":
            self.k, self.v = (G.Groups(r.integers(0, 256, shape), r.integers(110, 140, (self.n_pages, Hkv, 16, D // 32)), self.strides, D, dtype) for _ in range(2))
        elif cache == "blocks":
            self.k, self.v = (C.Blocks(r.integers(0, 256, shape).astype(np.uint8) & 0xF7, r.integers(118, 128, (self.n_pages, Hkv)), self.strides, D, dtype)
                              for _ in range(2))
        else:
            self.k, self.v = (W.store(r.standard_normal(shape).astype(np.float32), dtype) for _ in range(2))
        heads = Hq + 2 * Hkv
        x = r.standard_normal((Bn, n, heads, D)) * np.exp2(r.integers(-spread, spread + 1, (Bn, n, heads, 1)))
        self.x = W.store(x.astype(np.float32), dtype)
        if rows is not None:
            self.x = rows(self.x)
        self.q_gain, self.k_gain = ((1 + 0.3 * r.standard_normal(D)).astype(np.float32) if norm and gains else None for _ in range(2))
        self.inv_freq = (10000.0 ** (-np.arange(rot_dim // 2) / max(1, rot_dim // 2))).astype(np.float32)
        wide = heads * D
        self.desc = B.make_desc(batch=Bn, n_draft=min(n, 64), n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, max_pages_per_seq=self.table.shape[1],
                                max_ctx_len=int(self.ctx.max()), qkv_dtype=dtype, scale=1.0, kv_stride_page=self.strides[0], kv_stride_head=self.strides[1],
                                kv_stride_token=self.strides[2], n_pool_pages=self.n_pages)
        self.app = B.AppendDesc(n_tokens=n, rot_dim=rot_dim, rot_style=B.OWL_ROT_PAIRS if pairs else B.OWL_ROT_HALVES, rot_scale=rot_scale,
                                q_stride=wide if fused else Hq * D, k_stride=wide if fused else Hkv * D, v_stride=wide if fused else Hkv * D)
        x = _to_dev(self.x.reshape(Bn, n, wide), DEV)
        self.dq, self.dk, self.dv = x.split([Hq * D, Hkv * D, Hkv * D], dim=-1)
        if not fused:
            self.dq, self.dk, self.dv = self.dq.contiguous(), self.dk.contiguous(), self.dv.contiguous()
        self.q_out = torch.full((Bn, n, Hq, D), 7, dtype=x.dtype, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.dtable, self.dlens, self.dcounts, self.dpos = i32(self.table), i32(self.ctx), i32(counts), i32(pos)
        self.freq = torch.from_numpy(self.inv_freq).to(DEV) if rot_dim else None
        self.gains = [None if g is None else torch.from_numpy(g).to(DEV) for g in (self.q_gain, self.k_gain)]
        if cache == "own":
            self.dev = [_to_dev(t, DEV) for t in (self.k, self.v)] + [None, None]
        else:
            self.dev = [torch.from_numpy(t).to(DEV) for t in (self.k.flat, self.v.flat, self.k.scale, self.v.scale)]

    def run(self, q=True, stream=None):
        call = B.owl_append_kv_groups if self.cache == "groups" else B.owl_append_kv_norm
        call(self.desc, self.app, B.NormDesc(eps=self.eps) if self.norm else None, self.dq if q else None, self.dk, self.dv, *self.gains, self.freq,
             self.dpos, self.q_out if q else None, *self.dev, self.dtable, self.dlens, self.dcounts, self.status, stream)

    def want(self):
        counts = np.full(len(self.ctx), self.n) if self.counts is None else np.clip(self.counts, 0, self.n)
        pos = self.pos if self.pos is not None else self.ctx[:, None] + np.arange(self.n)
        q, k, v = self.x[:, :, :self.Hq], self.x[:, :, self.Hq:self.Hq + self.Hkv], self.x[:, :, self.Hq + self.Hkv:]
        a = (q, k, v, pos, self.inv_freq, self.rot_dim, self.pairs, self.rot_scale, self.dtype)
        q, k, v = G.normalised_rows(*a, self.q_gain, self.k_gain, self.eps) if self.norm else C.rotated_rows(*a)
        full = np.full(q.shape, 7, q.dtype)              # (16-bit rows are held as their bits)
        for b, c in enumerate(counts):
            full[b, :c] = q[b, :c]
        if self.cache == "own":
            return full, *(C.append(p, x, self.table, self.ctx, counts, self.strides) for p, x in ((self.k, k), (self.v, v)))
        pools = self.k.copy(), self.v.copy()
        for p, x in zip(pools, (k, v)):
            p.append(x, self.table, self.ctx, counts)
        return full, *pools

    def check(self, q=True):
        torch.cuda.synchronize()
        wq, wk, wv = self.want()
        if q:
            got = self.q_out.view(torch.int16 if self.dtype != W.DT_F32 else torch.int32).cpu().numpy().view(wq.dtype)
            same = (got == wq) | (np.isnan(C.widen(got, self.dtype)) & np.isnan(C.widen(wq, self.dtype)))
            assert same.all(), f"{np.sum(~same)} of {wq.size}"
        if self.cache == "own":
            for d, w in zip(self.dev[:2], (wk, wv)):
                got = d.view(torch.int16 if self.dtype != W.DT_F32 else torch.int32).cpu().numpy().view(w.dtype).reshape(w.shape)
                assert ((got == w) | (np.isnan(C.widen(got, self.dtype)) & np.isnan(C.widen(w, self.dtype)))).all()
            return
        for d, s, w in zip(self.dev[:2], self.dev[2:], (wk, wv)):
            assert np.array_equal(s.cpu().numpy(), w.scale)
            if self.cache == "groups":
                assert np.array_equal(d.cpu().numpy(), w.flat), f"{np.sum(d.cpu().numpy() != w.flat)} of {w.flat.size}"
            else:
                assert C.same_bytes(d.cpu().numpy(), w.flat)


KINDS = [(W.DT_BF16, "own", True), (W.DT_F16, "own", True), (W.DT_F32, "own", True), (W.DT_BF16, "blocks", True), (W.DT_F16, "blocks", True),
         (W.DT_BF16, "groups", True), (W.DT_F16, "groups", True), (W.DT_BF16, "groups", False), (W.DT_F16, "groups", False)]


@pytest.mark.parametrize("dtype,cache,norm", KINDS)
@pytest.mark.parametrize("Hq,Hkv,D,ctx,n,rot_dim,pairs,head_major,fused", [
    (4, 1, 64, [0], 1, 64, False, True, True), (8, 2, 128, [5003], 1, 128, False, True, True), (8, 2, 128, [15, 16, 17, 0], 6, 128, False, False, True),
    (6, 2, 128, [100, 31], 60, 64, True, True, False), (8, 8, 64, [33], 64, 32, False, False, False), (3, 1, 128, [1, 47], 17, 16, True, True, True),
    (4, 4, 128, [250], 33, 0, False, True, True), (32, 8, 128, [70], 5, 128, True, True, True), (2, 2, 64, [12], 300, 64, False, True, True),
    (5, 5, 128, [3], 7, 48, False, True, True), (5, 5, 128, [30], 7, 80, True, False, True), (7, 7, 64, [9], 11, 48, False, True, False), (1, 1, 64, [2], 3, 0, False, True, True),
])
def test_rows_match_the_oracle(dtype, cache, norm, Hq, Hkv, D, ctx, n, rot_dim, pairs, head_major, fused):
    a = Rows(n + D + rot_dim, dtype=dtype, cache=cache, norm=norm, Hq=Hq, Hkv=Hkv, D=D, ctx=ctx, n=n, rot_dim=rot_dim, pairs=pairs,
             head_major=head_major, fused=fused, page_gap=64)
    a.run()
    a.check()
    assert int(a.status.item()) == 0


@pytest.mark.parametrize("dtype,cache,norm", KINDS)
@pytest.mark.parametrize("Hq,Hkv,D,ctx,n,rot_dim,pairs", [(3, 1, 128, [5], 768, 128, False), (3, 1, 128, [5], 769, 64, False), (7, 1, 64, [9, 0, 40], 300, 64, True),
                                                          (20, 2, 128, [33, 1], 500, 128, True)])
def test_many_tokens(dtype, cache, norm, Hq, Hkv, D, ctx, n, rot_dim, pairs):
    a = Rows(n + D, dtype=dtype, cache=cache, norm=norm, Hq=Hq, Hkv=Hkv, D=D, ctx=ctx, n=n, rot_dim=rot_dim, pairs=pairs)
    a.run()
    a.check()
    assert int(a.status.item()) == 0


@pytest.mark.parametrize("dtype,cache,norm", KINDS)
def test_far_positions_a_scale_and_no_gains(dtype, cache, norm):
    pos = np.array([[0, 131071, 1 << 20, (1 << 31) - 1, -5, 99999, 7], [3, 3, 4, 4, 5, 1 << 30, 1000003]], np.int64)
    a = Rows(3, dtype=dtype, cache=cache, norm=norm, gains=False, Hq=4, Hkv=2, D=128, ctx=[40, 7], n=7, rot_dim=128, pos=pos, rot_scale=1.1386)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype,cache,norm", KINDS)
def test_sequences_with_fewer_new_tokens_and_without_queries(dtype, cache, norm):
    counts = np.array([9, 0, 4, 1, 12, -3], np.int32)
    a = Rows(4, dtype=dtype, cache=cache, norm=norm, Hq=4, Hkv=2, D=64, ctx=[30, 5, 16, 0, 47, 3], n=9, rot_dim=64, counts=counts)
    a.run()
    a.check()
    assert int(a.status.item()) == B.OWL_DEV_BAD_NDRAFT  # 12 and -3
    a = Rows(5, dtype=dtype, cache=cache, norm=norm, Hq=4, Hkv=2, D=64, ctx=[30, 5], n=9, rot_dim=64)
    a.run(q=False)
    a.check(q=False)
    assert (a.q_out == 7).all()


@pytest.mark.parametrize("dtype,cache,norm", KINDS)
@pytest.mark.parametrize("eps", [0.0, 1e-6, 3.0])
def test_rows_of_zeros_tiny_and_huge_numbers(dtype, cache, norm, eps):
    """Zeros (0 / 0 with eps 0), the type's least and greatest numbers, rows that differ by many binades."""
    def rows(x):
        w = C.widen(x, dtype)
        w[0, 0] = 0.0
        w[0, 1] *= 2.0 ** (-140 if dtype != W.DT_F16 else -20)
        w[0, 2] *= 2.0 ** (120 if dtype != W.DT_F16 else 11)
        w[0, 3, :, ::2] *= 2.0 ** -30
        w[0, 4] = np.sign(w[0, 4]) * {W.DT_BF16: 3.3895e38, W.DT_F16: 65504.0, W.DT_F32: 3.4e38}[dtype]
        return C.store(w, dtype)
    a = Rows(6, dtype=dtype, cache=cache, norm=norm, Hq=2, Hkv=2, D=128, ctx=[20], n=6, rot_dim=0 if not norm else 128, spread=2, rows=rows, eps=eps)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("norm", [False, True])
def test_infinite_numbers_and_none_make_their_groups_none(dtype, norm):
    def rows(x):
        w = C.widen(x, dtype)
        w[0, 0, :, 40] = np.inf
        w[0, 1, :, 100] = np.nan
        w[0, 2, :, 0] = -np.inf
        return C.store(w, dtype)
    a = Rows(7, dtype=dtype, cache="groups", norm=norm, Hq=2, Hkv=2, D=128, ctx=[13], n=5, rot_dim=64, rows=rows)
    a.run()
    a.check()
    got = a.dev[2].cpu().numpy()[a.table[0, 0]][:, 13]   # K's scales of the first new token
    assert (got[:, 1] == 255).all() if not norm else True


@pytest.mark.parametrize("dtype,cache,norm", KINDS)
def test_bad_pages_and_lengths_are_dropped(dtype, cache, norm):
    a = Rows(8, dtype=dtype, cache=cache, norm=norm, Hq=2, Hkv=2, D=64, ctx=[14, 3], n=5, rot_dim=64)
    before = [None if t is None else t.clone() for t in a.dev]
    a.dtable[0, 1] = a.n_pages                           # tokens 2 .. 4 of the first sequence
    a.dlens[1] = 15                                      # beyond max_ctx_len
    a.run()
    torch.cuda.synchronize()
    assert int(a.status.item()) == B.OWL_DEV_BAD_PAGE | B.OWL_DEV_BAD_CTX_LEN
    a.ctx, a.counts = a.ctx[:1], np.array([2])           # what is left: two rows of the first sequence
    a.x, a.q_out = a.x[:1], a.q_out[:1]
    table = a.table
    a.table = table[:1]
    _, wk, wv = a.want()
    for d, s, w, old in zip(a.dev[:2], a.dev[2:], (wk, wv), before):
        d = d.cpu().numpy() if cache != "own" else d.view(torch.int16 if dtype != W.DT_F32 else torch.int32).cpu().numpy().view(w.dtype)
        if cache == "own":
            assert np.array_equal(d.reshape(w.shape), w)
        elif cache == "groups":
            assert np.array_equal(d, w.flat) and np.array_equal(s.cpu().numpy(), w.scale)
        else:
            assert C.same_bytes(d, w.flat) and np.array_equal(s.cpu().numpy(), w.scale)


def test_queries_in_place_and_a_stream_of_ones_own():
    a = Rows(9, dtype=W.DT_BF16, cache="groups", Hq=4, Hkv=2, D=128, ctx=[33], n=6, rot_dim=128, fused=False)
    a.q_out = a.dq.view(a.q_out.shape)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a.run(stream=s.cuda_stream)
    s.synchronize()
    a.check()


@pytest.mark.parametrize("cache,norm", [("own", True), ("blocks", True), ("groups", True), ("groups", False)])
def test_captured_appends_and_their_replays(cache, norm):
    """The first call of a shape inside a capture; replays with other rows and lengths in the same places."""
    a = Rows(10, dtype=W.DT_F16, cache=cache, norm=norm, Hq=4, Hkv=2, D=128, ctx=[33, 90], n=6, rot_dim=128)
    b = Rows(11, dtype=W.DT_F16, cache=cache, norm=norm, Hq=4, Hkv=2, D=128, ctx=[70, 17], n=6, rot_dim=128)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    graph.replay()
    a.check()
    # b's rows, cache and lengths through a's buffers (the tables have the same number of columns)
    assert a.table.shape[1] >= b.table.shape[1]
    a.table = np.full_like(a.table, -1)
    a.table[:, :b.table.shape[1]] = b.table % a.n_pages
    keep = {tuple(x) for x in a.table.tolist()}
    assert len(keep) == 2
    used = [p for i, L in enumerate(b.ctx) for p in a.table[i, L // 16:(L + 5) // 16 + 1]]
    if len(set(used)) != len(used):
        a.table = np.arange(a.table.size, dtype=np.int32).reshape(a.table.shape) % a.n_pages
    a.dtable.copy_(i32(a.table))
    torch.cuda.synchronize()
    a.ctx, a.x = b.ctx, b.x
    a.dlens.copy_(b.dlens)
    whole = torch.cat([b.dq, b.dk, b.dv], -1)
    for mine, theirs in zip((a.dq, a.dk, a.dv), whole.split([a.Hq * a.D, a.Hkv * a.D, a.Hkv * a.D], dim=-1)):
        mine.copy_(theirs)
    if cache == "own":
        a.k, a.v = (t.view(torch.int16).cpu().numpy().view(a.k.dtype).reshape(a.k.shape) for t in a.dev[:2])
    else:
        for held, d, s in ((a.k, a.dev[0], a.dev[2]), (a.v, a.dev[1], a.dev[3])):
            held.flat[:], held.scale[:] = d.cpu().numpy(), s.cpu().numpy()
    a.desc.max_ctx_len = 90
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
    a.check()


def test_two_sequences_one_after_the_other_fill_a_page():
    """Rows of other tokens stay as they are, bit for bit: single tokens appended one by one give the page that one call gives."""
    one = Rows(12, dtype=W.DT_BF16, cache="groups", Hq=2, Hkv=2, D=128, ctx=[5], n=20, rot_dim=128)
    one.run()
    one.check()
    many = Rows(12, dtype=W.DT_BF16, cache="groups", Hq=2, Hkv=2, D=128, ctx=[5], n=20, rot_dim=128)
    many.app.n_tokens = 1
    many.desc.max_ctx_len = 25
    many.desc.max_pages_per_seq = many.table.shape[1]
    for i in range(20):
        lens = i32(np.array([5 + i]))
        B.owl_append_kv_groups(many.desc, many.app, B.NormDesc(eps=many.eps), None, many.dk[:, i:], many.dv[:, i:], *many.gains, many.freq, None, None,
                               *many.dev, many.dtable, lens, i32(np.array([1])), many.status)
    torch.cuda.synchronize()
    for x, y in zip(one.dev, many.dev):
        assert torch.equal(x, y)


def test_prompt_of_thousands_of_tokens():
    """Against the call in pieces: every row the same, whatever else is in the call."""
    a = Rows(13, dtype=W.DT_BF16, cache="groups", Hq=8, Hkv=2, D=128, ctx=[0], n=3000, rot_dim=128)
    b = Rows(13, dtype=W.DT_BF16, cache="groups", Hq=8, Hkv=2, D=128, ctx=[0], n=3000, rot_dim=128)
    a.run()
    b.desc.max_ctx_len = 3000
    for first in range(0, 3000, 777):
        n = min(777, 3000 - first)
        b.app.n_tokens = n
        out = torch.empty((1, n, 8, 128), dtype=b.q_out.dtype, device=DEV)
        B.owl_append_kv_groups(b.desc, b.app, B.NormDesc(eps=b.eps), b.dq[:, first:], b.dk[:, first:], b.dv[:, first:], *b.gains, b.freq, None, out,
                               *b.dev, b.dtable, i32(np.array([first])), i32(np.array([n])), b.status)
        b.q_out[:, first:first + n] = out
    torch.cuda.synchronize()
    assert torch.equal(a.q_out, b.q_out) and all(torch.equal(x, y) for x, y in zip(a.dev, b.dev))


def test_the_norm_descriptor_has_the_headers_size():
    assert ctypes.sizeof(B.NormDesc) == 4
