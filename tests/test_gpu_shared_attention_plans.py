"""Attention of several continuations on every kind of launch that its plan chooses between: the result must not tell which one a size takes."""
import random

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


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def inputs(m, plens, n_seqs, n_q, stride, row_tail, seed, pstride):
    groups, dt = len(plens), U.TYPES[m.dtype]
    q = U.normal((groups * n_seqs * n_q, m.n_q_heads, m.head_dim), seed, dt)
    kp, vp = (U.normal((groups, pstride, m.n_kv_heads, m.head_dim), seed + i, dt) for i in (1, 2))
    kt, vt = (U.normal((groups * n_seqs, stride, m.n_kv_heads, m.head_dim), seed + i, dt) for i in (3, 4))
    return [t.cuda() for t in (q, kp, vp, kt, vt)] + [torch.tensor(row_tail, dtype=torch.int32, device="cuda")]


def call(P, ctx, q, kp, vp, plens, kt, vt, row_tail, n_seqs, n_q, **kw):
    flat = [t.view(-1, *t.shape[2:]) for t in (kp, vp, kt, vt)]
    return P.cb_shared_prefix_attention(ctx, q, len(plens), n_seqs, n_q, flat[0], flat[1], plens, flat[2], flat[3], row_tail, **kw)


def ragged(seqs, n_q, stride, seed):
    """tail rows seen by every query row: up to itself, padding behind the continuation's last new token"""
    rng, out = random.Random(seed), []
    for _ in range(seqs):
        new, before = rng.randint(max(1, n_q // 2), n_q), rng.randint(0, stride - n_q)
        out += [before + i + 1 if i < new else -1 for i in range(n_q)]
    return out


# few queries, and enough queries and keys for a launch of 32 queries per wavefront: one piece of the keys, several, one token and many, one
# request and two; the last tile of every context is filled in part
SHAPES = [(8, 2, 128, [700], 3, 1), (16, 2, 64, [333, 70], 2, 5), (16, 8, 64, [500], 8, 256), (16, 2, 128, [1111, 1999], 3, 200),
          (64, 2, 64, [13001], 4, 1), (24, 4, 128, [7001], 41, 1)]


@pytest.mark.parametrize("hq,hkv,dh,plens,n_seqs,n_q", SHAPES)
def test_a_visible_infinity_gives_an_infinity_whatever_the_launch(P, hq, hkv, dh, plens, n_seqs, n_q):
    """Values that are not finite in rows that every query sees: an infinity of their sign in their channel and key/value head, nothing
    anywhere else.  Every context row's probability is positive in these inputs, so that is what the definition gives."""
    m, stride, g = U.model(hq, hkv, dh, "bf16"), n_q + 20, hq // hkv
    seqs = len(plens) * n_seqs
    rt = ragged(seqs, n_q, stride, n_q)
    announce("visible infinities", hq, hkv, dh, plens, n_seqs, n_q)
    q, kp, vp, kt, vt, r = inputs(m, plens, n_seqs, n_q, stride, rt, 71, max(plens) + 3)
    ctx = P.cb_create(m, 8)
    ref = call(P, ctx, q, kp, vp, plens, kt, vt, r, n_seqs, n_q)
    assert bool(torch.isfinite(ref).all())
    real = torch.tensor([v >= 0 for v in rt], device="cuda")
    # one row: of either half of the first tile, on both sides of a tile's border, the last; and the second half of every tile
    for rows in ([3], [40], [63], [64], [-1], [-2, -1], "second halves"):
        for bad in (INF, -INF):
            v = vp.clone()
            for grp, n in enumerate(plens):
                at = torch.arange(n)[torch.arange(n) % 64 >= 32] if rows == "second halves" else [i % n for i in rows]
                v[grp, at, hkv - 1, 5] = bad
            out = call(P, ctx, q, kp, v, plens, kt, vt, r, n_seqs, n_q)
            hit = torch.zeros_like(out, dtype=torch.bool)
            hit[real, (hkv - 1) * g:, 5] = True
            assert bool((out[hit] == bad).all()), (rows, bad)
            assert same(out[~hit], ref[~hit]), (rows, bad)
    P.cb_destroy(ctx)


def test_more_workgroups_than_a_launch_numbers_are_refused(P):
    """2^23 tails' heads of 512 threads each: refused before anything is read, as the size query says"""
    import ctypes as C
    from paper_2405_16444_amd import binding
    ctx = P.cb_create(U.model(32, 32, 128, "bf16"), 8)
    assert P.cb_shared_prefix_workspace_bytes(ctx, 64, 4096, 1, 40, 1) == 0 and P.cb_shared_prefix_workspace_bytes(ctx, 64, 3900, 1, 40, 1) > 0
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p, lens = buf.data_ptr(), (C.c_int32 * 64)(*[40] * 64)
    assert binding._lib.cb_shared_prefix_attention(ctx._h, p, 64, 4096, 1, p, p, lens, 40, p, p, 1, p, p, p, 1 << 60, None) == -4
    P.cb_destroy(ctx)


EVERY = [(dh, *shape) for dh in (64, 128) for shape, _ in U.plan_shapes(dh)]


@pytest.mark.parametrize("dh,hq,hkv,prefix,n_seqs,n_q", EVERY)
def test_every_tile_counts_once(P, dh, hq, hkv, prefix, n_seqs, n_q):
    """values that give every tile of the context, and of the tails, a channel which few others share"""
    m, stride = U.model(hq, hkv, dh, "bf16"), n_q + 20
    rt = ragged(n_seqs, n_q, stride, prefix)
    announce("every tile counts", dh, hq, hkv, prefix, n_seqs, n_q)
    q, kp, _, kt, _, r = inputs(m, [prefix], n_seqs, n_q, stride, rt, 81, prefix)
    vp = U.coded_values(prefix, hkv, dh).to(torch.bfloat16)[None].cuda()
    vt = U.coded_values(stride, hkv, dh, prefix // 32 + 1).to(torch.bfloat16)[None].expand(n_seqs, -1, -1, -1).contiguous().cuda()
    check(P, m, q, kp, vp, prefix, kt, vt, r, n_seqs, n_q)


@pytest.mark.parametrize("dh,hq,hkv,prefix,n_seqs,n_q", EVERY)
def test_rows_at_the_borders_count(P, dh, hq, hkv, prefix, n_seqs, n_q):
    """a few context rows, at tile borders and the ends, and all tail rows have most of the probability"""
    m, stride = U.model(hq, hkv, dh, "bf16"), n_q + 20
    rt = ragged(n_seqs, n_q, stride, prefix + 1)
    announce("border rows", dh, hq, hkv, prefix, n_seqs, n_q)
    q, kp, vp, kt, vt, r = inputs(m, [prefix], n_seqs, n_q, stride, rt, 91, prefix + 40)
    q, kp, kt = U.towards_borders(q, kp, kt, prefix)
    check(P, m, q, kp, vp, prefix, kt, vt, r, n_seqs, n_q)


def check(P, m, q, kp, vp, prefix, kt, vt, r, n_seqs, n_q):
    ctx = P.cb_create(m, 8)
    out = call(P, ctx, q, kp, vp, [prefix], kt, vt, r, n_seqs, n_q)
    ref, bound = U.attention(q, kp, vp, [prefix], kt, vt, r.cpu(), n_seqs, n_q, m.dtype)
    off = (out.double() - ref).abs()
    assert bool(torch.isfinite(out).all()) and bool((off <= bound).all()), float((off / bound.clamp_min(1e-30)).max())
    assert not bool(out[r < 0].any())
    assert same(call(P, ctx, q, kp, vp, [prefix], kt, vt, r, n_seqs, n_q, out=q), out)      # over the queries
    P.cb_destroy(ctx)
