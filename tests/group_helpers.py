"""Caches of 4-bit groups for the tests: a workloads.Case whose cache has gone through the oracle's groups."""
import dataclasses

import numpy as np
import torch

from block_helpers import DEV, i32, rng
from oracle import cache_groups as G
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from paper_2510_07535_amd.runner import _to_dev


def quantise(x, dtype):
    """Rows [..., D] of numbers in 64 bits -> (bytes [..., D / 2], scales [..., D / 32]): the oracle's group_of, many at once."""
    x = np.asarray(x, np.float64)
    shape = x.shape
    x = x.reshape(*shape[:-1], -1, 32)
    fine = np.isfinite(x).all(-1)
    x = np.where(fine[..., None], x, 0.0)
    low, high = G.ENDS[dtype]
    big = np.abs(x).max(-1)
    with np.errstate(divide="ignore"):
        e = np.where(big > 0, np.ceil(np.log2(np.where(big > 0, big, 1.0) / 7.0)), low)
    e = np.where(big > 7.0 * np.exp2(e), e + 1, e)
    e = np.where((big > 0) & (big <= 7.0 * np.exp2(e - 1)), e - 1, e)
    e = np.clip(e, low, high)
    y = np.abs(x) * np.exp2(-e)[..., None]
    code = (y > 0.25).astype(np.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    code = np.where(fine[..., None], code + 8 * np.signbit(x), 0).astype(np.uint8).reshape(shape)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(fine, e + 127, 255).astype(np.uint8)


def values(raw, scale):
    """What rows of bytes [..., D / 2] with scales [..., D / 32] stand for."""
    codes = np.stack([raw & 15, raw >> 4], -1).reshape(*raw.shape[:-1], -1)
    x = np.where(codes > 7, -1.0, 1.0) * G.MAGNITUDES[codes & 7]
    with np.errstate(over="ignore"):
        e = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127.0))
    return x * np.repeat(e, 32, -1)


@dataclasses.dataclass
class GroupCase:
    case: W.Case                 # 16-bit pools that hold the same numbers, bit for bit
    raw: tuple                   # K, V: bytes in the case's layout, D / 2 for D
    scale: tuple                 # [pages][Hkv][16][D / 32] each
    strides: tuple               # bytes


def group_case(name, seed, gain=None, stale_none=True, **kw):
    """Groups of every cached row; rows behind the last one, and pages that no sequence has, are no numbers (scale 255) unless
    ``stale_none`` is false.  ``gain(rng, n)``: powers of two that the n pages' values are multiplied by."""
    case = W.make_case(name, seed, **kw)
    r = rng(seed + 77)
    head_major = case.stride_head > case.stride_token
    raws, scales, pools = [], [], []
    for pool in (case.k_pool, case.v_pool):
        x = W.widen(pool, case.dtype).astype(np.float64)
        x = x.reshape(case.n_pool_pages, case.Hkv, 16, case.D) if head_major else x.reshape(case.n_pool_pages, 16, case.Hkv, case.D).swapaxes(1, 2)
        if gain is not None:
            x = x * gain(r, case.n_pool_pages)[:, None, None, None]
        raw, scale = quantise(x, case.dtype)
        live = np.zeros((case.n_pool_pages, 16), bool)
        for b in range(case.B):
            t = np.arange(int(case.ctx_lens[b]) + case.N)
            page = t // 16 if case.page_table is None else case.page_table[b, t // 16]
            live[page, t % 16] = True
        if stale_none:
            scale = np.where(live[:, None, :, None], scale, 255).astype(np.uint8)
        wide = np.where(live[:, None, :, None], values(raw, scale), 0.0)
        layout = (lambda a: a) if head_major else (lambda a: a.swapaxes(1, 2))
        raws.append(np.ascontiguousarray(layout(raw)))
        scales.append(np.ascontiguousarray(scale))
        pools.append(W.store(np.ascontiguousarray(layout(wide)).astype(np.float32), case.dtype).reshape(pool.shape))
    H, D = case.Hkv, case.D
    strides = (H * 16 * D // 2, 16 * D // 2, D // 2) if head_major else (16 * H * D // 2, D // 2, H * D // 2)
    return GroupCase(dataclasses.replace(case, k_pool=pools[0], v_pool=pools[1]), tuple(raws), tuple(scales), strides)


class GroupStep:
    """Device buffers of one owl_verify_attn_groups."""

    def __init__(self, gc, *, split_tokens=0, out_dtype=B.OWL_F32, flags=0, max_ctx_len=None, counts=None, parent=None):
        c = gc.case
        self.case, self.gc = c, gc
        self.parent = c.tree_parent if parent is None else parent
        self.counts = counts
        self.desc = B.make_desc(batch=c.B, n_draft=c.N, n_q_heads=c.Hq, n_kv_heads=c.Hkv, head_dim=c.D,
                                max_pages_per_seq=0 if c.page_table is None else c.page_table.shape[1],
                                max_ctx_len=int(c.ctx_lens.max()) if max_ctx_len is None else max_ctx_len, qkv_dtype=c.dtype, scale=c.scale,
                                kv_stride_page=gc.strides[0], kv_stride_head=gc.strides[1], kv_stride_token=gc.strides[2],
                                n_pool_pages=c.n_pool_pages, split_tokens=split_tokens, out_dtype=out_dtype, flags=flags)
        self.k, self.v = (torch.from_numpy(x).to(DEV) for x in gc.raw)
        self.ks, self.vs = (torch.from_numpy(x).to(DEV) for x in gc.scale)
        self.q = _to_dev(c.q, DEV)
        self.table, self.lens, self.dparent, self.dcounts = i32(c.page_table), i32(c.ctx_lens), i32(self.parent), i32(counts)
        t = {0: torch.bfloat16, 1: torch.float32, 2: torch.float16}[out_dtype]
        self.out = torch.full((c.B, c.N, c.Hq, c.D), 123.0, dtype=t, device=DEV)
        self.ws = torch.full((B.owl_verify_attn_groups_workspace_size(self.desc),), 0xFF, dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def run(self, stream=None):
        B.owl_verify_attn_groups(self.desc, self.q, self.k, self.v, self.ks, self.vs, self.table, self.lens, self.dparent, self.dcounts,
                                 self.out, self.ws, self.status, stream)

    def result(self):
        self.run()
        torch.cuda.synchronize()
        return self.out.float().cpu().numpy()
