"""sssd_op_logprobs against 64 bits where one workgroup goes over a whole row (from 1024 rows on) of a real vocabulary, and where the true log-probability is -infinity.

Bounds, u = 2^-24, for rows whose logits are about as far apart as those of a model.  A term of S is off by (4 |x| + 2) u of itself (the difference, the factor log2(e) / T, their product, exp2), x
relative to a logit within four octaves of the largest, 2.8 more than the row's own x: (4 |x| + 13) u.  A lane adds vocab / 256 + 1 terms, a wave its lanes in 6 steps; the sums are moved to
another reference at most once on the way and once at the end, by up to four octaves, 16 u each, and three joins of waves cost as much: log S is off by (4 E|x| + c) u and its own rounding, with c = vocab / 256 + 1 + 6
+ 5 * 16 + 13.  A log-probability has 4 |x| u (difference, 1 / T, product) and two roundings more; the entropy (4 E x^2 + (2 + 2 c) E|x| + 4 (E|x|)^2 + 4 E|x| + c) u and three roundings of
its parts, with x relative to the reference.  The roundings of a chain of sums are independent: in the root mean square over rows the bounds hold without its vocab / 256."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_logprobs as base
from paper_2411_05894_amd import binding as sv

DEV = "cuda:0"
U = 2.0 ** -24
SHIFT = 4 * math.log(2)


def close(got, want, bound, mean_bound):
    """-infinity exactly where the truth is; else within bounds.  Squared errors in units of the bound for the root mean square."""
    got = got.double()
    assert not got.isnan().any() and not want.isnan().any()
    none = want == -math.inf
    assert (got[none] == -math.inf).all() and got[~none].isfinite().all()
    err = (got - want)[~none].abs()
    bound, mean_bound = bound.expand(want.shape)[~none], mean_bound.expand(want.shape)[~none]
    assert (err <= bound).all(), float((err / bound).max())
    if err.numel() >= 1000:
        assert float(((err / mean_bound) ** 2).mean()) <= 1


def check(z, tokens, n_top, temperature=1.0, at_a_time=256):
    rows, vocab = z.shape
    lp, ranks, entropy, ids, top = sv.sssd_op_logprobs(z, tokens.int(), n_top, temperature)
    parts = []
    for i in range(0, rows, at_a_time):
        t = tokens[i:i + at_a_time]
        w = base.want(z[i:i + at_a_time], t, n_top, temperature)
        first = w["order"][:, :n_top]
        assert torch.equal(ranks[i:i + at_a_time].long(), torch.gather(w["place"], 1, t)) and torch.equal(ids[i:i + at_a_time].long(), first)
        parts.append((torch.gather(w["lp"], 1, t), torch.gather(w["x"], 1, t), torch.gather(w["lp"], 1, first), torch.gather(w["x"], 1, first), w["e1"], w["e2"], w["log_s"], w["entropy"]))
    lw, xw, tw, xt, e1, e2, log_s, hw = (torch.cat(p) for p in zip(*parts))

    def bound(c, want, x):
        x = x.nan_to_num(0, 0, 0).abs()
        return (4 * e1[:, None] + c) * U + 4 * x * U + (want.abs().nan_to_num(0, 0, 0) + log_s[:, None]) * 4 * U
    chain, rest = vocab / 256 + 1, 6 + 5 * 16 + 13
    close(lp, lw, bound(chain + rest, lw, xw), bound(rest, lw, xw))
    close(top, tw, bound(chain + rest, tw, xt), bound(rest, tw, xt))
    a, b = e1 + SHIFT, e2 + 2 * SHIFT * e1 + SHIFT ** 2
    h = lambda c: (4 * b + (2 + 2 * c) * a + 4 * a ** 2 + 4 * a + c) * U + 3 * (a + log_s) * U  # noqa: E731
    close(entropy, hw, h(chain + rest), h(rest))
    return lp, ranks, entropy, ids, top


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [768, 1023, 1024, 1501])
@pytest.mark.parametrize("m,n_top,temperature", [(1, 1, 1.0), (7, 20, 0.7)])
def test_whole_rows_of_a_real_vocabulary(dtype, rows, m, n_top, temperature):
    z, tokens = base.random_rows(rows, 128256, rows + m, dtype)
    a = check(z, tokens[:, :m].contiguous(), n_top, temperature)
    assert all(torch.equal(x, y) for x, y in zip(a, sv.sssd_op_logprobs(z, tokens[:, :m].int().contiguous(), n_top, temperature)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(6, 20011), (1, 300007), (1200, 9001), (1024, 128256)])
def test_masked_tokens(dtype, rows, vocab):
    """Log-probabilities of masked tokens are -infinity, whether they are given or among the first because nothing else is left."""
    z, tokens = base.random_rows(rows, vocab, vocab, dtype)
    for r in range(0, rows, 6):
        z[r, 1:] = -math.inf                 # one token left
        if r + 1 < rows:
            z[r + 1, 3:] = -math.inf         # three
        if r + 2 < rows:
            z[r + 2, ::2] = -math.inf
        if r + 3 < rows:
            z[r + 3, :-40] = -math.inf
        if r + 4 < rows:
            z[r + 4, 17:] = -math.inf
            z[r + 4, 100] = 2.0
    tokens[:, 0], tokens[:, 1], tokens[:, 2], tokens[:, 3] = 0, 1, vocab - 1, 100
    lp, ranks, entropy, ids, top = check(z, tokens, 64)
    assert (lp[0, 1:4] == -math.inf).all() and lp[0, 0] == 0 and entropy[0] == 0 and (top[0, 1:] == -math.inf).all() and torch.equal(ids[0], torch.arange(64, dtype=torch.int32, device=DEV))


def test_far_rows():
    """Numbers of rows beyond 2^31 bytes."""
    vocab, rows = 128256, 9000
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    part, tokens = base.random_rows(40, vocab, 10, torch.bfloat16)
    z[-40:] = part
    all_tokens = torch.full((rows, 2), 5, dtype=torch.int64, device=DEV)
    all_tokens[-40:] = tokens[:, :2]
    lp, ranks, entropy, ids, top = far = sv.sssd_op_logprobs(z, all_tokens.int(), 3)
    for got in (lp[:-40], top[:-40]):        # equal logits: one of vocab
        assert ((got.double() + math.log(vocab)).abs() <= (vocab / 256 + 100 + 8 * math.log(vocab)) * U).all()
    assert ((entropy[:-40].double() - math.log(vocab)).abs() <= (vocab / 256 + 100 + 8 * math.log(vocab)) * U).all()
    assert (ranks[:-40] == 5).all() and torch.equal(ids[:-40], torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEV).expand(rows - 40, 3))
    again = torch.zeros(1100, vocab, dtype=torch.bfloat16, device=DEV)
    again[:40] = part
    t = torch.full((1100, 2), 5, dtype=torch.int64, device=DEV)
    t[:40] = tokens[:, :2]
    near = check(again, t, 3)
    assert all(torch.equal(x[-40:], y[:40]) for x, y in zip(far, near))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_are_the_same_among_others(dtype):
    """What a row gives does not depend on the others, nor on how many there are while the workgroups go over whole rows."""
    z, tokens = base.random_rows(2000, 32001, 3, dtype)
    t = tokens[:, :3].int().contiguous()
    all_rows = sv.sssd_op_logprobs(z, t, 5)
    some = sv.sssd_op_logprobs(z[700:1800], t[700:1800].contiguous(), 5)
    assert all(torch.equal(x[700:1800], y) for x, y in zip(all_rows, some))
