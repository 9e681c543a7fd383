"""Log probabilities of near-certain tokens, at temperatures other than one, and of logits towards the ends of their type.  Needs an
MI355X (-m gpu)."""
import numpy as np
import pytest

from block_helpers import i32, rng
from oracle import logprobs as P
from paper_2510_07535_amd import binding as B
from test_gpu_logprobs import Call

pytestmark = pytest.mark.gpu


def check(c):
    """x - m is rounded once, its product with the scale once: 2^-23 of a log probability's magnitude; ln l is off by 2^-21 as the
    exponentials are (2^-22, and the sum to less), and the difference rounds once more.  Nothing grows with the logits themselves,
    and with the greatest at x - m = 0 and l >= 1 no log probability is above 0."""
    lp, h, ids, top = P.token_logprobs(c.x.double().cpu().numpy(), None if not c.n_given else c.tokens.cpu().numpy(), c.desc.n_top, c.desc.scale)
    assert np.array_equal(c.ids.cpu().numpy(), ids)
    for got, want in ((c.logprob, lp), (c.top, top)):
        got = got.double().cpu().numpy()
        with np.errstate(over="ignore"):                 # what lies beyond float32 is -infinity there
            want = want.astype(np.float32).astype(np.float64)
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~fine], want[~fine], equal_nan=True)
        got, want = got[fine], want[fine]
        assert (got <= 0).all() and (np.abs(got - want) <= 2.0 ** -20 + 2.0 ** -22 * np.abs(want)).all(), np.abs(got - want).max()
    # (the entropy's mean of x - m: its terms' roundings weigh as the terms do)
    got = c.entropy.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(h)) and (np.abs(np.nan_to_num(got) - np.nan_to_num(h)) <= 2.0 ** -19 + 2.0 ** -20 * np.abs(np.nan_to_num(h))).all()
    return c


# one launch, and two
SHAPES = [(40, 1000), (3, 30000), (300, 9000), (4, 70001)]


@pytest.mark.parametrize("dtype", [B.OWL_F32, B.OWL_BF16])
@pytest.mark.parametrize("scale", [0.7, 1.25, 0.1, 3.0])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_near_certain_tokens(rows, vocab, scale, dtype):
    r = rng(rows + vocab)
    x = r.standard_normal((rows, vocab)).astype(np.float32)
    token = r.integers(0, vocab, rows)
    x[np.arange(rows), token] = np.exp(r.uniform(np.log(20.0), np.log(1000.0), rows))
    given = np.stack([token, (token + 1) % vocab], axis=1).astype(np.int32)
    c = check(Call(x, given, 3, scale, dtype=dtype).run())
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("dtype", [B.OWL_F32, B.OWL_BF16, B.OWL_F16])
@pytest.mark.parametrize("scale", [1.25, 2.0, 0.5])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_rows_of_the_types_least_and_greatest_numbers(rows, vocab, scale, dtype):
    """All logits the type's lowest number, a usual mask: every token is as likely as any other.  All but one: that one is certain.
    The greatest number beside usual ones: certain as well."""
    end = {B.OWL_F32: 3.4028234663852886e38, B.OWL_BF16: 3.3895313892515355e38, B.OWL_F16: 65504.0}[dtype]
    r = rng(vocab)
    x = np.full((rows, vocab), -end, np.float32)
    x[1, vocab // 2] = 1.5
    x[2] = r.standard_normal(vocab)
    x[2, vocab - 1] = end
    given = r.integers(0, vocab, (rows, 2)).astype(np.int32)
    given[1, 0], given[2, 0] = vocab // 2, vocab - 1
    c = check(Call(x, given, 4, scale, dtype=dtype).run())
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_scales_towards_the_ends_of_the_type(rows, vocab):
    r = rng(rows)
    x = np.where(r.random((rows, vocab)) < 0.5, 3.0e38, -3.0e38).astype(np.float32)
    check(Call(x, r.integers(0, vocab, (rows, 2)).astype(np.int32), 2, 1.0e-38).run())
    x = -np.exp2(r.integers(-2, 9, (rows, vocab))).astype(np.float32)
    c = check(Call(x, r.integers(0, vocab, (rows, 2)).astype(np.int32), 2, 1.0e38).run())
    assert int(c.status.item()) == 0
