"""A decoding loop over a cache of 4-bit groups with normalised heads, from the prompt on: append, Prepare, append of the drafted tree, verify
attention, what the target says, acceptance, commit, every array staying on the device, against the same loop on the oracles; at the end the sequences
are read back.  Needs an MI355X (-m gpu)."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
from block_helpers import DEV, assert_attention, i32, rng
from group_helpers import GroupCase, values
from oracle import cache_groups as G
from oracle import logprobs as P
from oracle import steps as S
from paper_2510_07535_amd import binding as B
from paper_2510_07535_amd import workloads as W
from paper_2510_07535_amd.runner import _to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,n,other_stream", [(W.DT_BF16, 128, 10, False), (W.DT_F16, 64, 10, True), (W.DT_F16, 128, 1, False), (W.DT_BF16, 64, 3, True)])
def test_decoding_loop_over_4_bit_groups(dtype, D, n, other_stream):
    r = rng(dtype + D + n)
    Hq, Hkv, rounds, vocab, eps = 8, 2, 8, 700, 1e-5
    N, Bn = 2 * n, 3
    prompts, most = np.array([37, 300, 0], np.int32), 300
    room = most + rounds * n + N
    width = (room + 15) // 16
    n_pages = Bn * width
    table = r.permutation(n_pages).astype(np.int32).reshape(Bn, width)
    strides = (Hkv * 16 * D // 2, 16 * D // 2, D // 2)
    shape = (n_pages, Hkv, 16, D // 2)
    inv_freq = (10000.0 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)
    gains = [r.uniform(0.5, 2.0, D).astype(np.float32) for _ in range(2)]
    scale = float(np.float32(D ** -0.5))
    k_o, v_o = (G.Groups(np.zeros(shape), np.full((n_pages, Hkv, 16, D // 32), 127), strides, D, dtype) for _ in range(2))
    stored = lambda x, pos: G.normalised_rows(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, inv_freq, D, False, 1.0, dtype, *gains, eps)
    numbers = lambda c: W.store(values(c.flat.reshape(shape), c.scale).astype(np.float32), dtype)

    heads, wide = Hq + 2 * Hkv, (Hq + 2 * Hkv) * D
    desc = B.make_desc(batch=Bn, n_draft=N, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, max_pages_per_seq=width, max_ctx_len=room - N, qkv_dtype=dtype,
                       scale=scale, kv_stride_page=strides[0], kv_stride_head=strides[1], kv_stride_token=strides[2], n_pool_pages=n_pages)
    app = lambda count: B.AppendDesc(n_tokens=count, rot_dim=D, rot_style=B.OWL_ROT_HALVES, rot_scale=1.0, q_stride=wide, k_stride=wide, v_stride=wide)
    norm = B.NormDesc(eps=eps)
    stream = torch.cuda.Stream() if other_stream else torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        k, v, ks, vs = (torch.from_numpy(x).to(DEV) for x in (k_o.flat, v_o.flat, k_o.scale, v_o.scale))
        freq, d_table, status = torch.from_numpy(inv_freq).to(DEV), i32(table), torch.zeros(1, dtype=torch.int32, device=DEV)
        q_gain, k_gain = (torch.from_numpy(x).to(DEV) for x in gains)
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        p2, depth, pos, acc, na, bonus, last = z(Bn, N), z(Bn, N), z(Bn, N), z(Bn, N), z(Bn), z(Bn), z(Bn)
        anc = torch.zeros((Bn, N), dtype=torch.int64, device=DEV)
        said, root = z(Bn, N), z(Bn, 1)
        lens = [z(Bn), z(Bn)]
        q_out, out = torch.zeros((Bn, N, Hq, D), dtype=torch.int16, device=DEV), torch.zeros((Bn, N, Hq, D), device=DEV)
        ws = torch.empty(B.owl_verify_attn_groups_workspace_size(desc), dtype=torch.uint8, device=DEV)
        rows = B.LogprobDesc(rows=Bn * N, vocab=vocab, n_given=0, n_top=1, dtype=B.OWL_F32, scale=1.0, row_stride=vocab)
        ends = B.LogprobDesc(rows=Bn, vocab=vocab, n_given=0, n_top=1, dtype=B.OWL_F32, scale=1.0, row_stride=vocab)
        lws = torch.empty(B.owl_token_logprobs_workspace_size(rows), dtype=torch.uint8, device=DEV)

    # the prompts, all of them in one call
    x = W.store(r.standard_normal((Bn, most, heads, D)).astype(np.float32), dtype)
    _, kr, vr = stored(x, np.tile(np.arange(most), (Bn, 1)))
    k_o.append(kr, table, [0] * Bn, prompts)
    v_o.append(vr, table, [0] * Bn, prompts)
    with torch.cuda.stream(stream):
        _, dk, dv = _to_dev(x.reshape(Bn, most, wide), DEV).split([Hq * D, Hkv * D, Hkv * D], dim=-1)
        B.owl_append_kv_groups(desc, app(most), norm, None, dk, dv, None, k_gain, freq, None, None, k, v, ks, vs, d_table, lens[0], i32(prompts), status)
        lens[0].copy_(i32(prompts))
    ctx_o, grew = prompts.copy(), 0
    for it in range(rounds):
        trees = np.stack([W.chain_tree(n) if b == it % Bn else W.random_tree(n, 4, r) for b in range(Bn)])
        x = W.store(r.standard_normal((Bn, N, heads, D)).astype(np.float32), dtype)
        logits = r.standard_normal((Bn * N + Bn, vocab)).astype(np.float32)
        tokens = r.integers(0, vocab, (Bn, N)).astype(np.int32)
        _, _, best, _ = P.token_logprobs(logits, None, 1, 1.0)
        said_o, root_o = best[:Bn * N, 0].reshape(Bn, N), best[Bn * N:, 0]
        for b in range(Bn):                              # drafts that agree with the target on the path to one node
            node = int(r.integers(n // 2, n))
            while node >= 0:
                up = int(trees[b, node])
                tokens[b, node] = said_o[b, up] if up >= 0 else root_o[b]
                node = up
        # the oracles' round
        p2_o, _, _, pos_o = S.prepare_spec_tree(trees, ctx_o)
        q_o, kr, vr = stored(x, pos_o)
        k_o.append(kr, table, ctx_o, [N] * Bn)
        v_o.append(vr, table, ctx_o, [N] * Bn)
        case = W.Case("loop", 0, dtype, Bn, N, Hq, Hkv, D, scale, q_o, numbers(k_o), numbers(v_o), table, ctx_o, p2_o, width, *(2 * s for s in strides), n_pages)
        want = oracle.verify_attn_case(case)
        acc_o, na_o, bonus_o, last_o = S.accept_greedy(tokens, p2_o, root_o, said_o, n)
        k_o.commit(table, ctx_o, acc_o, na_o)
        v_o.commit(table, ctx_o, acc_o, na_o)
        # the device's
        cur, nxt = lens[it % 2], lens[(it + 1) % 2]
        with torch.cuda.stream(stream):
            dq, dk, dv = _to_dev(x.reshape(Bn, N, wide), DEV).split([Hq * D, Hkv * D, Hkv * D], dim=-1)
            d_logits = torch.from_numpy(logits).to(DEV)
            B.owl_prepare_spec_tree(i32(trees), cur, p2, anc, depth, pos, status)
            B.owl_append_kv_groups(desc, app(N), norm, dq, dk, dv, q_gain, k_gain, freq, pos, q_out, k, v, ks, vs, d_table, cur, None, status)
            B.owl_verify_attn_groups(desc, q_out, k, v, ks, vs, d_table, cur, p2, None, out, ws, status)
            B.owl_token_logprobs(rows, d_logits, None, None, None, said, None, lws, status)
            B.owl_token_logprobs(ends, d_logits[Bn * N:], None, None, None, root, None, lws, status)
            B.owl_accept_greedy(i32(tokens), p2, root, said, n, acc, na, bonus, last, status)
            B.owl_commit_kv_groups(desc, k, v, ks, vs, d_table, cur, acc, na, nxt, status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0, it
        assert np.array_equal(q_out.cpu().numpy().view(np.uint16), q_o), it
        assert_attention(out.double().cpu().numpy(), GroupCase(dataclasses.replace(case), (k_o.flat, v_o.flat), (k_o.scale, v_o.scale), strides), want, str(it))
        assert np.array_equal(said.cpu().numpy(), said_o) and np.array_equal(root.cpu().numpy()[:, 0], root_o), it
        for got, ref in ((p2, p2_o), (pos, pos_o), (acc, acc_o), (na, na_o), (bonus, bonus_o), (last, last_o), (nxt, ctx_o + na_o)):
            assert np.array_equal(got.cpu().numpy(), ref), it
        for raw, sc, ref in ((k, ks, k_o), (v, vs, v_o)):
            assert np.array_equal(sc.cpu().numpy(), ref.scale) and np.array_equal(raw.cpu().numpy(), ref.flat), it
        grew += int(na_o.sum())
        ctx_o = (ctx_o + na_o).astype(np.int32)
    assert grew > rounds
    for b in range(Bn):                                  # what the loop has kept, in 16 bits
        L = int(ctx_o[b])
        for raw, sc, ref in ((k, ks, k_o), (v, vs, v_o)):
            with torch.cuda.stream(stream):
                back = torch.zeros((L, Hkv, D), dtype=torch.int16, device=DEV)
                B.owl_gather_kv_groups(desc, raw, sc, d_table, b, 0, L, back, status)
            torch.cuda.synchronize()
            kept = np.stack([[ref.row(table[b, t // 16], g, t % 16) for g in range(Hkv)] for t in range(L)]).reshape(L, Hkv, D)
            assert int(status.item()) == 0 and np.array_equal(back.cpu().numpy().view(np.uint16), W.store(kept.astype(np.float32), dtype)), b
