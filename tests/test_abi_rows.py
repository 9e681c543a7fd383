"""Refusals of the calls that write the cache's rows, read 8-bit blocks or look at logits: what the host can see is refused
before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2510_07535_amd import binding as B

A = 0x10000                                              # stands for an address; nothing here gets as far as using one


def _desc(**over):
    kw = dict(batch=2, n_draft=6, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_seq=70, max_ctx_len=1000,
              qkv_dtype=B.OWL_BF16, scale=0.09, kv_stride_page=2 * 16 * 128, kv_stride_head=16 * 128, kv_stride_token=128,
              n_pool_pages=200)
    kw.update(over)
    return B.make_desc(**kw)


def _append_desc(**over):
    kw = dict(n_tokens=60, rot_dim=128, rot_style=B.OWL_ROT_HALVES, rot_scale=1.0, q_stride=1024, k_stride=256, v_stride=256)
    kw.update(over)
    return B.AppendDesc(**kw)


def _append(desc, app, quant, **over):
    p = dict(q=A, k_new=A, v_new=A, inv_freq=A, pos=0, q_out=2 * A, k_cache=A, v_cache=A, k_scale=A, v_scale=A, table=A, lens=A, n_new=0)
    p.update(over)
    head = [ctypes.byref(desc), ctypes.byref(app) if app is not None else None] + [p[x] for x in ("q", "k_new", "v_new", "inv_freq", "pos", "q_out", "k_cache", "v_cache")]
    tail = [p["table"], p["lens"], p["n_new"], 0, 0]
    if quant:
        return B.lib().owl_append_kv_quant(*head, p["k_scale"], p["v_scale"], *tail)
    return B.lib().owl_append_kv(*head, *tail)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=0), B.OWL_ERR_INVALID_ARG), (dict(n_tokens=200), B.OWL_ERR_INVALID_ARG),          # beyond the table
    (dict(rot_dim=-16), B.OWL_ERR_UNSUPPORTED), (dict(rot_dim=24), B.OWL_ERR_UNSUPPORTED), (dict(rot_dim=144), B.OWL_ERR_UNSUPPORTED),
    (dict(rot_style=2), B.OWL_ERR_UNSUPPORTED), (dict(rot_scale=float("nan")), B.OWL_ERR_INVALID_ARG),
    (dict(q_stride=1016), B.OWL_ERR_INVALID_ARG), (dict(k_stride=248), B.OWL_ERR_INVALID_ARG), (dict(v_stride=260), B.OWL_ERR_INVALID_ARG),
    (dict(q_stride=1028), B.OWL_ERR_INVALID_ARG),
])
def test_append_refuses_shapes(quant, over, code):
    assert _append(_desc(), _append_desc(**over), quant) == code


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("over", [
    dict(k_new=0), dict(v_new=0), dict(inv_freq=0), dict(k_cache=0), dict(v_cache=0), dict(lens=0), dict(q=0), dict(q_out=0), dict(table=0),
    dict(q=A + 8), dict(k_new=A + 2), dict(v_new=A + 4), dict(q_out=A + 8), dict(k_cache=A + 1), dict(v_cache=A + 8),
])
def test_append_refuses_pointers(quant, over):
    assert _append(_desc(), _append_desc(), quant, **over) == B.OWL_ERR_INVALID_ARG


def test_append_refuses_queries_in_place_with_gaps():
    assert _append(_desc(), _append_desc(q_stride=1536), False, q=A, q_out=A) == B.OWL_ERR_INVALID_ARG


@pytest.mark.parametrize("quant", [False, True])
def test_append_refuses_descriptors(quant):
    assert _append(_desc(), None, quant) == B.OWL_ERR_INVALID_ARG
    assert _append(_desc(head_dim=96), _append_desc(rot_dim=64), quant) == B.OWL_ERR_UNSUPPORTED
    assert _append(_desc(batch=70000), _append_desc(), quant) == B.OWL_ERR_UNSUPPORTED
    assert _append(_desc(n_q_heads=7), _append_desc(), quant) == B.OWL_ERR_INVALID_ARG


def test_8_bit_blocks_refuse_token_strides_beyond_32_bit_page_offsets():
    d = _desc(kv_stride_token=(1 << 26) + 16)
    assert _append(d, _append_desc(), True) == B.OWL_ERR_UNSUPPORTED
    with pytest.raises(B.OwlError):
        B.owl_verify_attn_quant_workspace_size(d)


def test_8_bit_blocks_refuse_32_bit_numbers_odd_strides_and_missing_scales():
    for d, code in ((_desc(qkv_dtype=B.OWL_F32), B.OWL_ERR_UNSUPPORTED), (_desc(kv_stride_token=136), B.OWL_ERR_INVALID_ARG),
                    (_desc(kv_stride_head=16 * 128 + 8), B.OWL_ERR_INVALID_ARG)):
        assert _append(d, _append_desc(k_stride=512, v_stride=512, q_stride=2048), True) == code
        with pytest.raises(B.OwlError) as e:
            B.owl_verify_attn_quant_workspace_size(d)
        assert e.value.code == code
        with pytest.raises(B.OwlError) as e:
            B.owl_verify_attn_quant_init(d)
        assert e.value.code == code
        assert B.lib().owl_commit_kv_quant(ctypes.byref(d), A, A, A, A, A, A, A, A, 0, 0, 0) == code
    assert _append(_desc(), _append_desc(), True, k_scale=0) == B.OWL_ERR_INVALID_ARG
    assert _append(_desc(), _append_desc(), True, v_scale=0) == B.OWL_ERR_INVALID_ARG


@pytest.mark.parametrize("missing", ["q", "k", "v", "ks", "vs", "lens", "parent", "out"])
def test_verify_quant_refuses_missing_pointers(missing):
    p = {x: 0 if x == missing else A for x in ("q", "k", "v", "ks", "vs", "table", "lens", "parent", "out", "ws")}
    d = _desc()
    assert B.lib().owl_verify_attn_quant(ctypes.byref(d), p["q"], p["k"], p["v"], p["ks"], p["vs"], p["table"], p["lens"], p["parent"], 0,
                                         p["out"], p["ws"], 1 << 30, 0, 0) == B.OWL_ERR_INVALID_ARG


def test_verify_quant_refuses_workspaces_tables_and_alignment():
    d = _desc()
    size = B.owl_verify_attn_quant_workspace_size(d)
    call = lambda **o: B.lib().owl_verify_attn_quant(
        ctypes.byref(o.get("d", d)), o.get("q", A), o.get("k", A), A, A, A, A, A, A, 0, A, o.get("ws", A), o.get("bytes", size), 0, 0)
    assert call(ws=0) == B.OWL_ERR_WORKSPACE and call(bytes=size - 1) == B.OWL_ERR_WORKSPACE
    assert call(ws=A + 128) == B.OWL_ERR_INVALID_ARG and call(q=A + 8) == B.OWL_ERR_INVALID_ARG and call(k=A + 8) == B.OWL_ERR_INVALID_ARG
    assert call(d=_desc(max_pages_per_seq=62), bytes=1 << 30) == B.OWL_ERR_INVALID_ARG


def test_commit_quant_refuses():
    call = lambda d=None, **o: B.lib().owl_commit_kv_quant(
        ctypes.byref(d or _desc()), *[o.get(x, A) for x in ("k", "v", "ks", "vs", "table", "lens", "accepted", "count")], o.get("new", 2 * A), 0, 0)
    for x in ("k", "v", "ks", "vs", "lens", "accepted", "count", "table"):
        assert call(**{x: 0}) == B.OWL_ERR_INVALID_ARG, x
    assert call(new=A) == B.OWL_ERR_INVALID_ARG          # the lengths themselves
    assert call(k=A + 8) == B.OWL_ERR_INVALID_ARG
    assert call(_desc(max_pages_per_seq=62)) == B.OWL_ERR_INVALID_ARG
    assert call(_desc(n_draft=65)) == B.OWL_ERR_TOO_MANY_DRAFT


@pytest.mark.parametrize("over,code", [
    (dict(rows=0), B.OWL_ERR_INVALID_ARG), (dict(vocab=0), B.OWL_ERR_INVALID_ARG), (dict(row_stride=999), B.OWL_ERR_INVALID_ARG),
    (dict(scale=0.0), B.OWL_ERR_INVALID_ARG), (dict(scale=float("inf")), B.OWL_ERR_INVALID_ARG), (dict(scale=float("nan")), B.OWL_ERR_INVALID_ARG),
    (dict(n_given=-1), B.OWL_ERR_INVALID_ARG), (dict(n_top=-1), B.OWL_ERR_INVALID_ARG), (dict(n_given=65), B.OWL_ERR_UNSUPPORTED),
    (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), B.OWL_ERR_UNSUPPORTED),
    (dict(n_top=33), B.OWL_ERR_UNSUPPORTED), (dict(dtype=3), B.OWL_ERR_UNSUPPORTED),
])
def test_logprobs_refuse_descriptors(over, code):
    kw = dict(rows=4, vocab=1000, n_given=2, n_top=5, dtype=B.OWL_F32, scale=1.0, row_stride=1000)
    kw.update(over)
    with pytest.raises(B.OwlError) as e:
        B.owl_token_logprobs_workspace_size(B.LogprobDesc(**kw))
    assert e.value.code == code
    assert B.lib().owl_token_logprobs(ctypes.byref(B.LogprobDesc(**kw)), A, A, A, A, A, A, A, 1 << 30, 0, 0) == code


def test_logprobs_refuse_pointers_and_workspaces():
    d = B.LogprobDesc(rows=4, vocab=1000, n_given=2, n_top=5, dtype=B.OWL_F32, scale=1.0, row_stride=1000)
    size = B.owl_token_logprobs_workspace_size(d)
    call = lambda **o: B.lib().owl_token_logprobs(ctypes.byref(d), o.get("x", A), o.get("tok", A), o.get("lp", A), A, A, A, o.get("ws", A), o.get("bytes", size), 0, 0)
    for o in (dict(x=0), dict(x=A + 2), dict(tok=0), dict(lp=0), dict(ws=A + 64)):
        assert call(**o) == B.OWL_ERR_INVALID_ARG, o
    assert call(ws=0) == B.OWL_ERR_WORKSPACE and call(bytes=0) == B.OWL_ERR_WORKSPACE


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(B.AppendDesc) == 4 * 4 + 3 * 8 and B.AppendDesc.q_stride.offset == 16
    assert ctypes.sizeof(B.LogprobDesc) == 6 * 4 + 8 and B.LogprobDesc.row_stride.offset == 24
