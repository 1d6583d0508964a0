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


# rows, vocabularies and beams that make two and more rounds to a wavefront; the last stretch and the last round of other lengths than the rest
MANY = [(256, 64000, 8), (256, 64007, 4), (1024, 32000, 4), (1024, 33333, 16), (4500, 9001, 3), (320, 100003, 5)]


def rounds_of(rows, vocab):
    """2048 logits each, of a wavefront: as many as leave no more than 4096 wavefronts"""
    return -(-(-(-vocab // 2048)) // max(1, 4096 // rows))


def check(P, ctx, x, scores, beams, keep, done=None, end=0):
    """the call on all rows, some groups of them against the definition"""
    groups = x.shape[0] // beams
    got = P.cb_beam_select(ctx, x, scores, groups, keep, done, end)
    some = sorted({0, 1, groups // 3, groups // 2, groups - 2, groups - 1})
    rows = torch.tensor([g * beams + b for g in some for b in range(beams)], device="cuda")
    U.check_selection([t[some] for t in got], x[rows], scores[rows], len(some), None if done is None else done[rows], end)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,beams", MANY)
def test_several_rounds(P, ctx, dtype, rows, vocab, beams):
    announce("selection, several rounds", dtype, rows, vocab, beams)
    assert rounds_of(rows, vocab) > 1
    scores = (U.normal((rows,), vocab, std=2.0) - 10).cuda()
    x = U.normal((rows, vocab), rows + beams, U.TYPES[dtype], 3.0).cuda()
    done = (torch.arange(rows) % 11 == 3).to(torch.int32).cuda()
    for keep in (1, 16, 64):
        check(P, ctx, x, scores, beams, keep, done, vocab - 1)
        check(P, ctx, x.round(), scores, beams, keep)          # few distinct values


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,beams", MANY[1:4])
def test_every_round_is_better_than_the_last(P, ctx, dtype, rows, vocab, beams):
    """every logit of a round passes the threshold that the rounds before it left, so that lists overflow with entries kept; and the other way round"""
    announce("selection, rising and falling logits", dtype, rows, vocab, beams)
    base = torch.linspace(-6, 6, vocab)[None, :] + U.normal((rows, 1), 3, std=0.3)
    scores = U.normal((rows,), 4, std=0.2).cuda()
    for x in (base, base.flip(1), (base * 4).floor() / 4):
        x = x.to(U.TYPES[dtype]).cuda()
        for keep in (1, 9, 64):
            check(P, ctx, x, scores, beams, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,beams", MANY[:5])
def test_values_that_are_not_finite_in_some_rounds(P, ctx, dtype, rows, vocab, beams):
    announce("selection, rounds that are not finite", dtype, rows, vocab, beams)
    n, dt = rounds_of(rows, vocab), U.TYPES[dtype]
    nth = (torch.arange(vocab, device="cuda") // 2048) % n       # round of its stretch that a logit belongs to
    first, last = (nth == 0).nonzero().flatten(), (nth == n - 1).nonzero().flatten()
    scores = U.normal((rows,), 6, std=1.0).cuda()
    base = U.normal((rows, vocab), 5, dt, 2.0).cuda()
    for where in (first, last):
        for fill in (-INF, NAN, torch.finfo(dt).min):
            x = base.clone()
            x[:, where] = fill                                     # all of these rounds
            x[::3, where[5]] = 1.0
            for keep in (1, 64):
                check(P, ctx, x, scores, beams, keep)
        x = base.clone()
        x[1::2, where[7]] = INF                                    # one infinite logit, and two of different lanes and stretches
        x[2::4, where[-1]] = INF
        x[2::4, where[3]] = INF
        for keep in (1, 64):
            check(P, ctx, x, scores, beams, keep)
    x = torch.full_like(base, -INF)                                # nothing but a last logit, and nothing at all
    x[::2, -1] = 0.5
    check(P, ctx, x, scores, beams, 5)
