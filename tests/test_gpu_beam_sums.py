"""How near beam_select's sums of exponentials are to the exact ones, where their roundings
weigh most: one peak, and as many equal values as a wave holds some way below it; and what it
picks where 64 bits cannot tell scores apart."""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import DEV
from paper_2609_34380_amd import dps

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -24


def mean_distance(n):
    """The largest mean of |d| that n values d <= 0, the largest of them 0, have under the
    weights e^d.  With p = e^d / z the mean is the entropy of p less log z, and the value 0 has
    p = 1 / z, so the others are equal: (n - 1) t / (e^t + n - 1) for some t."""
    t = np.linspace(0.01, 30, 100000)
    return float(((n - 1) * t / (np.exp(t) + n - 1)).max())


def bound(n, pairs):
    """Of a sum over n values a wave, relative.  A term e^d: d rounded once, times log2 e, a
    constant 0.224 units off and a product rounded once, each of |d| in the exponent; 2 units for
    the exponential; then `pairs` roundings of sums in fp32.  The rest is in 64 bits."""
    log2e = float(np.float32(1.4426950408889634))
    const = abs(log2e / 1.4426950408889634 - 1) / UNIT
    assert const < 0.225
    return ((2 + const) * mean_distance(n) + 2 + pairs) * UNIT * 1.001


@pytest.mark.parametrize("dtype,per", [(torch.float32, 4), (torch.float16, 8), (torch.bfloat16, 8)])
def test_a_peak_over_equal_values(dtype, per):
    rows, vecs, threads = 1024, 8, 256
    piece = threads * vecs * per
    rng = np.random.default_rng(per)
    at = np.arange(piece)
    wave = at // per % threads < 64              # what the first wave of the block holds
    peak = rng.uniform(-15, 15, rows)
    peak[::2] = 0.0
    logits = torch.full((rows, piece), float("-inf"), dtype=torch.float64)
    logits[:, wave] = torch.from_numpy(peak - rng.uniform(3, 11, rows))[:, None]
    logits[:, 0] = torch.from_numpy(peak)
    logits = logits.to(dtype)
    exact = logits.double().numpy()
    lse = exact.max(1) + np.log(np.exp(exact - exact.max(1)[:, None]).sum(1))
    # so near to the sum's logarithm that the rest keeps its last bits in fp32
    score = (lse - exact[:, 0]).astype(np.float32)
    got = dps.beam_select(logits.to(DEV), torch.from_numpy(score).to(DEV), 1)
    assert got.token.flatten().tolist() == [0] * rows
    want = score.astype(np.float64) + (exact[:, 0] - lse)
    off = np.abs(got.score.cpu().double().numpy().reshape(-1) - want)
    limit = bound(64 * vecs * per, int(math.log2(per)))
    print("%s: %.2f of 2^-24, at most %.2f" % (dtype, off.max() / UNIT, limit / UNIT))
    assert off.max() <= limit
    assert limit < 2.0 ** -19


@pytest.mark.parametrize("vocab,keep", [(50, 4), (70000, 4), (70000, 256)])
def test_scores_that_swallow_the_logits(vocab, keep):
    """A score so large that every token's is the same in 64 bits: different tokens of the
    first beam, all of that score; equal logits still by their tokens."""
    rng = np.random.default_rng(vocab + keep)
    x = torch.from_numpy(rng.normal(size=(4, vocab)).astype(np.float32))
    x[2:] = 1.5
    score = np.array([-1e20, -1e20, -1e20, -1e20], np.float32)
    got = dps.beam_select(x.to(DEV), torch.from_numpy(score).to(DEV), 2, keep=keep)
    token, parent = got.token.tolist(), got.parent.tolist()
    n = min(keep, vocab)
    assert parent[0][:n] == [0] * n and len(set(token[0][:n])) == n
    assert all(0 <= t < vocab for t in token[0][:n])
    assert parent[1][:n] == [2] * n and token[1][:n] == list(range(n))
    assert bool((got.score == float(score[0])).all())
