"""Caches of 8-bit blocks for the GPU tests: a workloads.Case whose cache has gone through the oracle's blocks."""
import dataclasses

import numpy as np
import torch

import oracle
from oracle import cache_blocks as C
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from paper_2510_07535_amd.runner import _to_dev

DEV = "cuda:0"
NAN_BYTE = 0x7F


def rng(k):
    return np.random.Generator(np.random.Philox(key=k))


def i32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


@dataclasses.dataclass
class BlockCase:
    case: W.Case                 # 16-bit pools that hold the same numbers, bit for bit
    k: C.Blocks
    v: C.Blocks


def block_case(name, seed, page_gain=None, **kw):
    """Blocks of every cached row; slots behind the last one hold bytes that are no number, pages that no sequence
    has such a scale too.  ``page_gain(rng, n)``: powers of two that the n pages' values are multiplied by."""
    case = W.make_case(name, seed, **kw)
    strides = (case.stride_page, case.stride_head, case.stride_token)
    pools, blocks = [], []
    r = rng(seed + 77)
    for pool in (case.k_pool, case.v_pool):
        held = C.Blocks(np.full(pool.shape, NAN_BYTE), np.full((case.n_pool_pages, case.Hkv), 255), strides, case.D, case.dtype)
        gain = np.ones(case.n_pool_pages) if page_gain is None else page_gain(r, case.n_pool_pages)
        wide = W.widen(pool, case.dtype)
        wide16 = np.zeros_like(wide)
        for b in range(case.B):
            T = int(case.ctx_lens[b]) + case.N
            for lp in range((T + 15) // 16):
                page = lp if case.page_table is None else int(case.page_table[b, lp])
                n = min(16, T - lp * 16)
                for g in range(case.Hkv):
                    at = [held._at(page, g, s) for s in range(n)]
                    held.write(page, g, np.stack([wide.reshape(-1)[a] for a in at]) * gain[page])
                    for s, a in enumerate(at):
                        wide16.reshape(-1)[a] = held.row(page, g, s)
        blocks.append(held)
        pools.append(W.store(wide16.astype(np.float32), case.dtype))
    return BlockCase(dataclasses.replace(case, k_pool=pools[0], v_pool=pools[1]), *blocks)


class QuantStep:
    """Device buffers of one owl_verify_attn_quant."""

    def __init__(self, bc, out_dtype=B.OWL_F32, counts=None, split_tokens=0, max_ctx_len=None, flags=0):
        c = self.case = bc.case
        self.desc = B.make_desc(batch=c.B, n_draft=c.N, n_q_heads=c.Hq, n_kv_heads=c.Hkv, head_dim=c.D, max_pages_per_seq=c.max_pages_per_seq,
                                max_ctx_len=c.max_ctx_len if max_ctx_len is None else max_ctx_len, qkv_dtype=c.dtype, scale=c.scale,
                                kv_stride_page=c.stride_page, kv_stride_head=c.stride_head, kv_stride_token=c.stride_token,
                                n_pool_pages=c.n_pool_pages, out_dtype=out_dtype, split_tokens=split_tokens, flags=flags)
        self.q = _to_dev(c.q, DEV)
        self.k, self.v = (torch.from_numpy(x.flat).to(DEV) for x in (bc.k, bc.v))
        self.ks, self.vs = (torch.from_numpy(x.scale).to(DEV) for x in (bc.k, bc.v))
        self.table, self.lens, self.parent, self.counts = i32(c.page_table), i32(c.ctx_lens), i32(c.tree_parent), i32(counts)
        kind = {B.OWL_F32: torch.float32, B.OWL_BF16: torch.bfloat16, B.OWL_F16: torch.float16}[out_dtype]
        self.out = torch.full((c.B, c.N, c.Hq, c.D), float("nan"), dtype=kind, device=DEV)
        self.workspace = torch.empty(B.owl_verify_attn_quant_workspace_size(self.desc), dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def run(self):
        B.owl_verify_attn_quant(self.desc, self.q, self.k, self.v, self.ks, self.vs, self.table, self.lens, self.parent, self.counts,
                                self.out, self.workspace, self.status)

    def result(self):
        torch.cuda.synchronize()
        return self.out.double().cpu().numpy()

    def flags(self):
        torch.cuda.synchronize()
        return int(self.status.item())


# Relative half steps of the types, torch.finfo(t).eps / 2
HALF = {W.DT_BF16: 2.0 ** -8, W.DT_F16: 2.0 ** -11, W.DT_F32: 2.0 ** -24}


def assert_attention(got, bc, want, what=""):
    """A weight is rounded to the queries' type, in numerator and denominator: an output is off by at most 2 h of the greatest value
    that its KV head holds; a partial is held to 2^-12 of its row's greatest; scores are sums of D products in 32 bits, a few
    hundred in magnitude at most, off by less than 2^-12 of one, and with them their weights: 2^-10 in all beside the rounding.  That
    much at the worst element; over all outputs the roundings are independent, and their 2-norm is h at most."""
    c = bc.case
    assert got.shape == want.shape and np.isfinite(got).all(), what
    greatest = np.abs(W.widen(c.v_pool, c.dtype)).max()
    err = np.abs(got - want)
    bound = (2 * HALF[c.dtype] + 2.0 ** -10) * greatest
    assert err.max() <= bound, f"{what}: {err.max():.3e} > {bound:.3e}"
    assert np.linalg.norm(got - want) <= (HALF[c.dtype] + 2.0 ** -11) * np.linalg.norm(want), what


def oracle_out(bc, counts=None):
    return oracle.verify_attn_case(bc.case) if counts is None else oracle.verify_attn_ragged_case(bc.case, counts)
