"""Log probabilities of given tokens, entropies and top alternatives against the oracle.  Needs an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from block_helpers import DEV, i32, rng
from oracle import logprobs as P
from paper_2510_07535_amd import binding as B

pytestmark = pytest.mark.gpu
KIND = {B.OWL_F32: torch.float32, B.OWL_BF16: torch.bfloat16, B.OWL_F16: torch.float16}


class Call:
    def __init__(self, x, tokens, n_top, scale=1.0, pad=0, offset=0, dtype=B.OWL_F32):
        """x [rows][vocab] (numpy); rows lie ``pad`` numbers apart, the first one ``offset`` behind an aligned address."""
        rows, vocab = x.shape
        wide = vocab + pad
        flat = torch.full((offset + rows * wide,), float("nan"), dtype=KIND[dtype], device=DEV)
        self.x = torch.as_strided(flat, (rows, vocab), (wide, 1), offset)
        self.x.copy_(torch.from_numpy(x).to(DEV).to(KIND[dtype]))
        self.n_given = 0 if tokens is None else tokens.shape[1]
        self.tokens = i32(tokens)
        self.desc = B.LogprobDesc(rows=rows, vocab=vocab, n_given=self.n_given, n_top=n_top, dtype=dtype, scale=scale, row_stride=wide)
        nan = lambda *s: torch.full(s, 123.0, device=DEV)
        self.logprob, self.entropy, self.top = nan(rows, max(self.n_given, 1))[:, :self.n_given].contiguous(), nan(rows), nan(rows, n_top)
        self.ids = torch.full((rows, n_top), -9, dtype=torch.int32, device=DEV)
        self.workspace = torch.empty(max(256, B.owl_token_logprobs_workspace_size(self.desc)), dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def run(self):
        B.owl_token_logprobs(self.desc, self.x, self.tokens if self.n_given else None, self.logprob if self.n_given else None, self.entropy,
                             self.ids, self.top, self.workspace, self.status)
        torch.cuda.synchronize()
        return self

    def check(self):
        x = self.x.double().cpu().numpy()
        lp, h, ids, top = P.token_logprobs(x, None if not self.n_given else self.tokens.cpu().numpy(), self.desc.n_top, self.desc.scale)
        assert np.array_equal(self.ids.cpu().numpy(), ids)
        # An exponential is off by 2^-22 (its argument, at most 2^7 in magnitude where it counts, and itself by half a step each), the sums of
        # the others to less: ln l by 2^-21; x - m - ln l rounds at the magnitude of its parts.
        seen = np.where(np.isfinite(x), np.abs(x), 0.0).max(1, keepdims=True) * float(np.float32(self.desc.scale))
        bound = 2.0 ** -20 + 2.0 ** -23 * (2 * seen + 20)
        # (the answer is in float32, where -6e38, of 3e38 against -3e38, is -infinity)
        with np.errstate(over="ignore"):
            lp, top = (w.astype(np.float32).astype(np.float64) for w in (lp, top))
        for got, want in ((self.logprob, lp), (self.top, top)):
            got = got.double().cpu().numpy()
            fine = np.isfinite(want)
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
            assert (np.abs(np.where(fine, got, 0.0) - np.where(fine, want, 0.0)) <= bound).all()
        got = self.entropy.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(h))
        assert (np.abs(np.nan_to_num(got) - np.nan_to_num(h)) <= 2 * bound[:, 0]).all()
        return self


@pytest.mark.parametrize("dtype", [B.OWL_F32, B.OWL_BF16, B.OWL_F16])
@pytest.mark.parametrize("rows,vocab,n_given,n_top,scale,pad,offset", [
    (1, 1, 1, 1, 1.0, 0, 0), (3, 2, 2, 5, 1.0, 1, 1), (2, 255, 1, 1, 0.7, 0, 3), (4, 257, 0, 10, 1.0, 3, 0), (1, 32003, 4, 10, 1.0, 0, 1), (5, 8191, 3, 32, 1.25, 1, 5),
    (2, 8193, 64, 0, 1.0, 7, 2), (3, 40000, 2, 17, 1.0, 0, 0), (2, 128256, 1, 1, 1.0, 0, 0), (1, 200001, 5, 32, 0.5, 0, 7), (70, 1000, 1, 4, 2.0, 24, 0),
])
def test_matches_the_oracle(dtype, rows, vocab, n_given, n_top, scale, pad, offset):
    r = rng(vocab + rows)
    x = (2.5 * r.standard_normal((rows, vocab))).astype(np.float32)
    tokens = r.integers(0, vocab, (rows, n_given)).astype(np.int32) if n_given else None
    c = Call(x, tokens, n_top, scale, pad, offset, dtype).run().check()
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("dtype", [B.OWL_F32, B.OWL_BF16])
@pytest.mark.parametrize("n_top", [1, 10, 32])
def test_equal_logits_go_by_their_index(dtype, n_top):
    r = rng(n_top)
    x = np.zeros((6, 20000), np.float32)                 # row 0: all equal
    x[1] = r.integers(0, 3, 20000)
    x[2] = np.where(np.arange(20000) % 2, -0.0, 0.0)     # equal as well
    x[3] = np.arange(20000)                              # the greatest last (bf16: in runs of equal ones), all in one place
    x[4] = -np.arange(20000)
    x[5, [19999, 3, 8191, 8192]] = 5.0
    Call(x, None, n_top, dtype=dtype).run().check()


def test_excluded_tokens_rows_without_any_and_what_is_no_number():
    r = rng(2)
    x = (3 * r.standard_normal((8, 9000))).astype(np.float32)
    x[0, r.random(9000) < 0.99] = -np.inf
    x[1] = -np.inf
    x[2, 1:] = -np.inf
    x[3, 8999] = np.nan
    x[4, 17] = np.inf
    x[5, 100:] = -np.inf
    x[6] = np.where(np.arange(9000) == 4321, 3.0e38, -3.0e38)
    tokens = r.integers(0, 9000, (8, 3)).astype(np.int32)
    tokens[2] = 0, 1, -1
    tokens[7] = 9000, -2, 5
    c = Call(x, tokens, 12).run().check()
    assert int(c.status.item()) == B.OWL_DEV_BAD_LOGIT | B.OWL_DEV_BAD_TOKEN


@pytest.mark.parametrize("dtype", [B.OWL_F32, B.OWL_BF16])
@pytest.mark.parametrize("rows,vocab", [(300, 8185), (300, 8186), (300, 9000), (2, 32761), (2, 32762), (1, 1 << 20)])
def test_rows_at_the_borders_between_one_launch_and_two(rows, vocab, dtype):
    r = rng(vocab)
    x = r.standard_normal((rows, vocab)).astype(np.float32)
    x[-1] = np.sort(x[-1])                               # the greatest side by side
    x[0, :] = -4.0
    x[0, r.integers(0, vocab, 40)] = 3.0                 # few great ones, the rest equal
    Call(x, r.integers(0, vocab, (rows, 2)).astype(np.int32), 32, dtype=dtype).run().check()


def test_outputs_that_are_not_wanted():
    r = rng(3)
    x = r.standard_normal((3, 500)).astype(np.float32)
    c = Call(x, r.integers(0, 500, (3, 2)).astype(np.int32), 4).run()
    d = Call(x, c.tokens.cpu().numpy(), 4)
    B.owl_token_logprobs(d.desc, d.x, d.tokens, d.logprob, None, d.ids, None, d.workspace)
    torch.cuda.synchronize()
    assert torch.equal(c.logprob, d.logprob) and torch.equal(c.ids, d.ids) and (d.entropy == 123).all() and (d.top == 123).all()


def test_the_same_call_gives_the_same_bits_and_replays():
    r = rng(4)
    x = (2 * r.standard_normal((9, 70000))).astype(np.float32)
    tokens = r.integers(0, 70000, (9, 2)).astype(np.int32)
    c, d = Call(x, tokens, 10).run(), Call(x, tokens, 10).run()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            B.owl_token_logprobs(c.desc, c.x, c.tokens, c.logprob, c.entropy, c.ids, c.top, c.workspace, c.status)
    for rep in range(3):
        for s in (c, d):
            s.x.copy_(s.x.flip(0) * (1.0 + 0.5 * rep))
            s.workspace.fill_(0xFF)
        graph.replay()
        d.run()
        assert all(torch.equal(p, q) for p, q in ((c.logprob, d.logprob), (c.entropy, d.entropy), (c.ids, d.ids), (c.top, d.top))), rep
    c.check()


def test_rows_far_behind_the_first():
    """Offsets beyond 2^32 bytes: the last of 9000 rows of 128256 in 32 bits."""
    rows, vocab = 9000, 128256
    x = torch.zeros((rows, vocab), device=DEV)
    x[-1] = torch.randn(vocab, device=DEV, generator=torch.Generator(DEV).manual_seed(5))
    desc = B.LogprobDesc(rows=rows, vocab=vocab, n_given=0, n_top=3, dtype=B.OWL_F32, scale=1.0, row_stride=vocab)
    ids, top = torch.zeros((rows, 3), dtype=torch.int32, device=DEV), torch.zeros((rows, 3), device=DEV)
    ws = torch.empty(B.owl_token_logprobs_workspace_size(desc), dtype=torch.uint8, device=DEV)
    B.owl_token_logprobs(desc, x, None, None, None, ids, top, ws)
    torch.cuda.synchronize()
    want = x[-1].double().log_softmax(-1).sort(descending=True, stable=True)
    assert torch.equal(ids[-1].long(), want.indices[:3]) and (top[-1].double() - want.values[:3]).abs().max() < 1e-5
    assert (ids[:-1] == torch.arange(3, device=DEV)).all()
