"""Refusals of the calls over caches of 4-bit groups and of the append with norms: what the host can see is refused before anything is
launched (no GPU)."""
import ctypes

import pytest

from paper_2510_07535_amd import binding as B
from test_abi_rows import A, _append_desc, _desc

NORM = B.NormDesc(eps=1e-6)


def _desc4(**over):
    kw = dict(kv_stride_page=2 * 16 * 64, kv_stride_head=16 * 64, kv_stride_token=64)
    kw.update(over)
    return _desc(**kw)


def _call(fn, desc, app, norm=NORM, **over):
    p = dict(q=A, k_new=A, v_new=A, q_gain=A, k_gain=A, inv_freq=A, pos=0, q_out=2 * A, k_cache=A, v_cache=A, k_scale=A, v_scale=A, table=A, lens=A, n_new=0)
    p.update(over)
    return getattr(B.lib(), fn)(ctypes.byref(desc), None if app is None else ctypes.byref(app), None if norm is None else ctypes.byref(norm),
                                *[p[x] for x in ("q", "k_new", "v_new", "q_gain", "k_gain", "inv_freq", "pos", "q_out", "k_cache", "v_cache", "k_scale",
                                                 "v_scale", "table", "lens", "n_new")], 0, 0)


FORMS = [("owl_append_kv_norm", _desc, dict(k_scale=0, v_scale=0)), ("owl_append_kv_norm", _desc, {}), ("owl_append_kv_groups", _desc4, {})]


@pytest.mark.parametrize("fn,desc,scales", FORMS)
@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=0), B.OWL_ERR_INVALID_ARG), (dict(n_tokens=200), B.OWL_ERR_INVALID_ARG), (dict(rot_dim=-16), B.OWL_ERR_UNSUPPORTED),
    (dict(rot_dim=24), B.OWL_ERR_UNSUPPORTED), (dict(rot_dim=144), B.OWL_ERR_UNSUPPORTED), (dict(rot_style=2), B.OWL_ERR_UNSUPPORTED),
    (dict(rot_scale=float("nan")), B.OWL_ERR_INVALID_ARG), (dict(q_stride=1016), B.OWL_ERR_INVALID_ARG), (dict(k_stride=248), B.OWL_ERR_INVALID_ARG),
    (dict(v_stride=260), B.OWL_ERR_INVALID_ARG),
])
def test_append_refuses_shapes(fn, desc, scales, over, code):
    assert _call(fn, desc(), _append_desc(**over), **scales) == code


@pytest.mark.parametrize("fn,desc,scales", FORMS)
@pytest.mark.parametrize("over", [
    dict(k_new=0), dict(v_new=0), dict(inv_freq=0), dict(k_cache=0), dict(v_cache=0), dict(lens=0), dict(q=0), dict(q_out=0), dict(table=0),
    dict(q=A + 8), dict(k_new=A + 2), dict(v_new=A + 4), dict(q_out=A + 8), dict(k_cache=A + 1), dict(v_cache=A + 8), dict(q_gain=A + 2), dict(k_gain=A + 1),
])
def test_append_refuses_pointers(fn, desc, scales, over):
    assert _call(fn, desc(), _append_desc(), **{**scales, **over}) == B.OWL_ERR_INVALID_ARG


@pytest.mark.parametrize("fn,desc,scales", FORMS)
@pytest.mark.parametrize("eps", [-1e-9, float("nan"), float("inf")])
def test_append_refuses_eps(fn, desc, scales, eps):
    assert _call(fn, desc(), _append_desc(), B.NormDesc(eps=eps), **scales) == B.OWL_ERR_INVALID_ARG


def test_norms_and_scales_that_do_not_belong_together():
    assert _call("owl_append_kv_norm", _desc(), _append_desc(), None) == B.OWL_ERR_INVALID_ARG
    assert _call("owl_append_kv_norm", _desc(), _append_desc(), k_scale=0) == B.OWL_ERR_INVALID_ARG
    assert _call("owl_append_kv_norm", _desc(), _append_desc(), v_scale=0) == B.OWL_ERR_INVALID_ARG
    for over in (dict(k_scale=0), dict(v_scale=0), dict(k_scale=A + 8), dict(v_scale=A + 4)):
        assert _call("owl_append_kv_groups", _desc4(), _append_desc(), **over) == B.OWL_ERR_INVALID_ARG
    assert _call("owl_append_kv_groups", _desc4(), _append_desc(), None) == B.OWL_ERR_INVALID_ARG          # gains without norms
    assert _call("owl_append_kv_groups", _desc4(), _append_desc(), None, q_gain=0) == B.OWL_ERR_INVALID_ARG


BAD4 = [
    (dict(qkv_dtype=B.OWL_F32), B.OWL_ERR_UNSUPPORTED), (dict(kv_stride_token=72), B.OWL_ERR_INVALID_ARG), (dict(kv_stride_token=48), B.OWL_ERR_INVALID_ARG),
    (dict(kv_stride_head=16 * 64 + 8), B.OWL_ERR_INVALID_ARG), (dict(kv_stride_page=-16), B.OWL_ERR_INVALID_ARG), (dict(head_dim=96), B.OWL_ERR_UNSUPPORTED),
    (dict(page_size=32), B.OWL_ERR_UNSUPPORTED), (dict(kv_stride_token=(1 << 26) + 16), B.OWL_ERR_UNSUPPORTED), (dict(n_q_heads=7), B.OWL_ERR_INVALID_ARG),
]


@pytest.mark.parametrize("over,code", BAD4)
def test_descriptors(over, code):
    d = _desc4(**over)
    wide = _append_desc(k_stride=512, v_stride=512, q_stride=2048, rot_dim=64)
    assert _call("owl_append_kv_groups", d, wide) == code
    assert B.lib().owl_commit_kv_groups(ctypes.byref(d), A, A, A, A, A, A, A, A, 0, 0, 0) == code
    assert B.lib().owl_gather_kv_groups(ctypes.byref(d), A, A, A, 0, 0, 10, A, 0, 0) == code


def test_rows_of_half_a_byte_a_channel_are_legal_strides_here_only():
    """64-byte rows of 128 channels: too short for the 8-bit calls."""
    with pytest.raises(B.OwlError):
        B.owl_verify_attn_quant_workspace_size(_desc4())


def test_append_beyond_a_grid():
    d = _desc4(max_pages_per_seq=1 << 27, n_pool_pages=1 << 27)
    assert _call("owl_append_kv_groups", d, _append_desc(n_tokens=1 << 24)) == B.OWL_ERR_UNSUPPORTED
    assert _call("owl_append_kv_groups", _desc4(batch=70000), _append_desc()) == B.OWL_ERR_UNSUPPORTED


def test_commit_refuses():
    call = lambda d=None, **o: B.lib().owl_commit_kv_groups(
        ctypes.byref(d or _desc4()), *[o.get(x, A) for x in ("k", "v", "ks", "vs", "table", "lens", "accepted", "count")], o.get("new", 2 * A), 0, 0)
    for x in ("k", "v", "ks", "vs", "lens", "accepted", "count", "table"):
        assert call(**{x: 0}) == B.OWL_ERR_INVALID_ARG, x
    for x in ("k", "v", "ks", "vs"):
        assert call(**{x: A + 8}) == B.OWL_ERR_INVALID_ARG, x
    assert call(new=A) == B.OWL_ERR_INVALID_ARG          # the lengths themselves
    assert call(_desc4(max_pages_per_seq=62)) == B.OWL_ERR_INVALID_ARG
    assert call(_desc4(n_draft=65)) == B.OWL_ERR_TOO_MANY_DRAFT
    assert call(_desc4(batch=70000)) == B.OWL_ERR_UNSUPPORTED


def test_gather_refuses():
    call = lambda d=None, **o: B.lib().owl_gather_kv_groups(
        ctypes.byref(d or _desc4()), o.get("cache", A), o.get("scale", A), o.get("table", A), o.get("seq", 0), o.get("first", 0), o.get("n", 10), o.get("dst", A), 0, 0)
    for o in (dict(cache=0), dict(scale=0), dict(dst=0), dict(table=0), dict(seq=-1), dict(seq=2), dict(first=-1), dict(n=-1), dict(cache=A + 8),
              dict(scale=A + 4), dict(dst=A + 2)):
        assert call(**o) == B.OWL_ERR_INVALID_ARG, o
    for o in (dict(first=(1 << 32) + 1), dict(n=(1 << 32) + 1)):
        assert call(**o) == B.OWL_ERR_UNSUPPORTED, o


@pytest.mark.parametrize("missing", ["q", "k", "v", "ks", "vs", "lens", "parent", "out"])
def test_verify_refuses_missing_pointers(missing):
    p = {x: 0 if x == missing else A for x in ("q", "k", "v", "ks", "vs", "table", "lens", "parent", "out", "ws")}
    assert B.lib().owl_verify_attn_groups(ctypes.byref(_desc4()), p["q"], p["k"], p["v"], p["ks"], p["vs"], p["table"], p["lens"], p["parent"], 0,
                                          p["out"], p["ws"], 1 << 30, 0, 0) == B.OWL_ERR_INVALID_ARG


def test_verify_refuses_workspaces_tables_and_alignment():
    d = _desc4()
    size = B.owl_verify_attn_groups_workspace_size(d)
    call = lambda **o: B.lib().owl_verify_attn_groups(
        ctypes.byref(o.get("d", d)), o.get("q", A), o.get("k", A), A, o.get("ks", A), o.get("vs", A), A, A, A, 0, A, o.get("ws", A), o.get("bytes", size), 0, 0)
    assert call(ws=0) == B.OWL_ERR_WORKSPACE and call(bytes=size - 1) == B.OWL_ERR_WORKSPACE
    for o in (dict(ws=A + 128), dict(q=A + 8), dict(k=A + 8), dict(ks=A + 8), dict(vs=A + 4)):
        assert call(**o) == B.OWL_ERR_INVALID_ARG, o
    assert call(d=_desc4(max_pages_per_seq=62), bytes=1 << 30) == B.OWL_ERR_INVALID_ARG


@pytest.mark.parametrize("over,code", BAD4)
def test_verify_refuses_descriptors(over, code):
    d, plan = _desc4(**over), B.Plan()
    for call in (B.owl_verify_attn_groups_workspace_size, B.owl_verify_attn_groups_init, B.owl_verify_attn_groups_plan):
        with pytest.raises(B.OwlError) as e:
            call(d)
        assert e.value.code == code
    assert B.lib().owl_verify_attn_groups_plan(ctypes.byref(_desc4()), None) == B.OWL_ERR_INVALID_ARG
    assert B.lib().owl_verify_attn_groups_plan(None, ctypes.byref(plan)) == B.OWL_ERR_INVALID_ARG


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [B.OWL_BF16, B.OWL_F16])
@pytest.mark.parametrize("group", [1, 4, 8, 64])
def test_every_plan_has_a_kernel_that_covers_its_rows(group, dtype, D):
    for n in range(1, 65):
        for batch, ctx, hkv in ((1, 0, 1), (1, 5003, 8), (1, 1 << 20, 2), (16, 65536, 8), (300, 700, 4)):
            d = _desc4(n_draft=n, n_q_heads=group * hkv, n_kv_heads=hkv, batch=batch, max_ctx_len=ctx, max_pages_per_seq=(ctx + n + 15) // 16, qkv_dtype=dtype,
                       head_dim=D)
            p = B.owl_verify_attn_groups_plan(d)
            assert p.workspace_bytes == B.owl_verify_attn_groups_workspace_size(d) > 0
            assert p.row_tiles == (n * group + 15) // 16 and p.kernel_variant >= 59
            per_group = -(-p.row_tiles // p.row_groups)
            assert 1 <= p.tiles_per_wave <= 3 and per_group <= 8 * p.tiles_per_wave
            assert p.split_tokens % 64 == 0 and p.split_tokens * p.max_splits >= ctx + n


def test_every_kernel_is_some_calls():
    taken = set()
    for dtype in (B.OWL_BF16, B.OWL_F16):
        for D in (64, 128):
            for ctx in (1000, 20000, 131072):
                for batch in (1, 16):
                    for n in (1, 5, 16, 28, 48, 64):
                        for group in (4, 8):
                            d = B.make_desc(batch=batch, n_draft=n, n_q_heads=8 * group, n_kv_heads=8, head_dim=D, max_pages_per_seq=(ctx + n + 15) // 16,
                                            max_ctx_len=ctx, qkv_dtype=dtype, scale=0.1, kv_stride_page=64 * D, kv_stride_head=8 * D, kv_stride_token=D // 2,
                                            n_pool_pages=1 << 20, out_dtype=dtype)
                            taken.add(B.owl_verify_attn_groups_plan(d).kernel_variant)
    assert taken == set(range(59, 89))
