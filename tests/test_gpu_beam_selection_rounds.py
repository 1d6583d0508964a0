"""Beam selection over rows so many or so long that a wavefront goes through several rounds of a stretch: the threshold, the list and the sums
carried from one to the next."""
import math

import pytest
import torch

import continuation_util as U
from gpu_util import announce

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def P():
    import paper_2405_16444_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def ctx(P):
    c = P.cb_create(U.model(4, 2, 64, "bf16"), 8)
    yield c
    P.cb_destroy(c)


def test_sums_over_many_rounds(P, ctx):
    """2048 rows of 4 M logits, 1024 rounds to a wavefront: each lane's first logit is the largest, all others lie the same step below it, a step at which
    1024 float additions of a round's sum would be off by 200 units of 2^-24 in one direction"""
    rows, vocab, step = 2048, 1 << 22, 0.75
    announce("selection, many rounds", rows, vocab)
    x = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda").fill_(-step)
    for piece in range(2):                 # of a row, as 4096 wavefronts take them
        x[:, piece * (vocab // 2):piece * (vocab // 2) + 512:8] = 0.0
    scores = torch.linspace(-40, 0, rows, device="cuda")
    s, b, t = P.cb_beam_select(ctx, x, scores, rows, 3)
    lse = math.log(2 * 64 + (vocab - 2 * 64) * math.exp(-step))
    err = (s.double() - (scores.double() - lse)[:, None]).abs()
    assert bool((err <= U.sum_error(vocab) + (scores.double() - lse).abs()[:, None] * 2.0 ** -24).all()), float(err.max()) * 2 ** 24
    assert not bool(b.any()) and torch.equal(t, torch.tensor([[0, 8, 16]], dtype=torch.int32, device="cuda").expand(rows, 3))
