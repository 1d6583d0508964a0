"""The operators that carry several continuations of one fused context, each against its definition in 64 bits: attention over a
shared context and the continuations' tails, head norms with rotation and cache append, beam selection, reordering."""
import math
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
    return torch.equal(a.contiguous().view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32),
                       b.contiguous().view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


# ---- attention ---------------------------------------------------------------------------------------------------
def attention_case(m, plens, n_seqs, n_q, stride, row_tail, seed, pstride=None):
    groups, dt = len(plens), U.TYPES[m.dtype]
    pstride = max(plens) if pstride is None else pstride
    rows = groups * n_seqs * n_q
    assert len(row_tail) == rows
    q = U.normal((rows, m.n_q_heads, m.head_dim), seed, dt)
    kp, vp = (U.normal((groups, pstride, m.n_kv_heads, m.head_dim), seed + i, dt) for i in (1, 2))
    kt, vt = (U.normal((groups * n_seqs, stride, m.n_kv_heads, m.head_dim), seed + i, dt) for i in (3, 4))
    return [t.cuda() for t in (q, kp, vp, kt, vt)] + [torch.tensor(row_tail, dtype=torch.int32, device="cuda")]


def call_attention(P, ctx, q, kp, vp, plens, kt, vt, row_tail, n_seqs, n_q, **kw):
    flat = [t.view(-1, *t.shape[2:]) for t in (kp, vp, kt, vt)]
    return P.cb_shared_prefix_attention(ctx, q, len(plens), n_seqs, n_q, flat[0], flat[1], plens, flat[2], flat[3], row_tail, **kw)


def check_attention(P, m, plens, n_seqs, n_q, stride, row_tail, seed, pstride=None):
    announce("shared attention", vars(m), plens, n_seqs, n_q, stride, row_tail[:8], pstride)
    q, kp, vp, kt, vt, rt = attention_case(m, plens, n_seqs, n_q, stride, row_tail, seed, pstride)
    ctx = P.cb_create(m, 8)
    out = call_attention(P, ctx, q, kp, vp, plens, kt, vt, rt, n_seqs, n_q)
    torch.cuda.synchronize()
    ref, bound = U.attention(q, kp, vp, plens, kt, vt, rt, n_seqs, n_q, m.dtype)
    off = (out.double() - ref).abs()
    assert bool(torch.isfinite(out).all()) and bool((off <= bound).all()), float((off / bound.clamp_min(1e-30)).max())
    P.cb_destroy(ctx)


HEADS = [("bf16", 4, 4, 64), ("bf16", 8, 2, 128), ("bf16", 14, 2, 128), ("bf16", 16, 2, 64), ("bf16", 5, 1, 128), ("f32", 4, 2, 64),
         ("f32", 6, 2, 128)]


@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
@pytest.mark.parametrize("prefix", [1, 31, 32, 33, 127, 129, 545, 1999])
def test_attention_decoding_step(P, dtype, hq, hkv, dh, prefix):
    """one new token per continuation, tails of every length from one to the whole slab"""
    m = U.model(hq, hkv, dh, dtype)
    check_attention(P, m, [prefix], 5, 1, 70, [1, 70, 33, 32, 17], 100 + prefix)


@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
def test_attention_groups_with_contexts_of_their_own(P, dtype, hq, hkv, dh):
    m = U.model(hq, hkv, dh, dtype)
    check_attention(P, m, [300, 0, 77, 1], 3, 1, 40, [5, 40, 1, 2, 9, 33, 0, 31, 32, 8, 0, 3], 7, pstride=311)


@pytest.mark.parametrize("n_seqs", [1, 2, 7, 16, 33])
def test_attention_numbers_of_continuations(P, n_seqs):
    for dtype, hq, hkv, dh in HEADS[1:3] + HEADS[5:6]:
        check_attention(P, U.model(hq, hkv, dh, dtype), [700], n_seqs, 1, 24, [1 + (7 * i) % 24 for i in range(n_seqs)], n_seqs)


@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
@pytest.mark.parametrize("n_seqs,n_q", [(3, 4), (2, 37), (5, 64)])
def test_attention_several_new_tokens_padded(P, dtype, hq, hkv, dh, n_seqs, n_q):
    """questions and drafts of different lengths: token i sees the tail up to itself, rows behind the last one are padding"""
    stride, rt, rng = n_q + 20, [], random.Random(n_q)
    for _ in range(n_seqs):
        new, before = rng.randint(1, n_q), rng.randint(0, 20)
        rt += [before + i + 1 if i < new else -1 for i in range(n_q)]
    check_attention(P, U.model(hq, hkv, dh, dtype), [431], n_seqs, n_q, stride, rt, n_q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_many_query_rows(P, dtype):
    """more query rows than one block of the kernels takes, context and tails of several pieces"""
    m = U.model(8, 2, 128, dtype)
    rt = [40 + i // 2 for _ in range(3) for i in range(150)]
    check_attention(P, m, [900], 3, 150, 600, rt, 3)
    check_attention(P, m, [350], 1, 1, 3000, [2999], 4)
    check_attention(P, m, [100], 2, 5, 1900, [600, 601, 602, 603, 604, 1895, 1896, 1897, -1, -1], 5)


WIDE = [  # enough queries and keys for the launch that takes 32 queries per wavefront: one, two and many pieces, one token and many
    (16, 8, 64, [500], 8, 256, 300), (16, 2, 128, [1111, 1999], 3, 200, 250), (64, 2, 64, [13001], 4, 1, 40), (24, 4, 128, [7001], 41, 1, 33),
    (16, 2, 64, [5000], 5, 9, 700)]


@pytest.mark.parametrize("hq,hkv,dh,plens,n_seqs,n_q,stride", WIDE)
def test_attention_wide(P, hq, hkv, dh, plens, n_seqs, n_q, stride):
    m, rt, rng = U.model(hq, hkv, dh, "bf16"), [], random.Random(n_q)
    for _ in range(len(plens) * n_seqs):
        new, before = rng.randint(max(1, n_q // 2), n_q), rng.randint(0, stride - n_q)
        rt += [before + i + 1 if i < new else -1 for i in range(n_q)]
    rt[0] = 0
    check_attention(P, m, plens, n_seqs, n_q, stride, rt, n_q, pstride=max(plens) + 5)
    q, kp, vp, kt, vt, r = attention_case(m, plens, n_seqs, n_q, stride, rt, n_q, max(plens) + 5)
    ctx = P.cb_create(m, 8)
    ref = call_attention(P, ctx, q, kp, vp, plens, kt, vt, r, n_seqs, n_q)
    assert same(call_attention(P, ctx, q, kp, vp, plens, kt, vt, r, n_seqs, n_q, out=q), ref)      # over the queries
    P.cb_destroy(ctx)


@pytest.mark.parametrize("hq,hkv,dh,plens,n_seqs,n_q,stride", WIDE[:1] + WIDE[3:])
def test_attention_wide_hidden_rows_have_no_influence(P, hq, hkv, dh, plens, n_seqs, n_q, stride):
    m = U.model(hq, hkv, dh, "bf16")
    rt = [(5 + i if i < n_q - n_q // 3 else -1) for _ in range(n_seqs) for i in range(n_q)]
    q, kp, vp, kt, vt, r = attention_case(m, plens, n_seqs, n_q, stride, rt, 22, pstride=max(plens) + 70)
    announce("wide shared attention, hidden rows", hq, hkv, dh, plens, n_seqs, n_q)
    ctx = P.cb_create(m, 8)
    ref = call_attention(P, ctx, q, kp, vp, plens, kt, vt, r, n_seqs, n_q)
    seen = [max(v for v in rt[s * n_q:(s + 1) * n_q]) for s in range(n_seqs)]
    kp[0, plens[0]:], vp[0, plens[0]:] = NAN, INF
    for s in range(n_seqs):
        kt[s, seen[s]:], vt[s, seen[s]:] = INF, NAN
    kt[1, :], vt[1, :] = NAN, NAN          # all of one continuation's tail: the others do not notice
    out = call_attention(P, ctx, q, kp, vp, plens, kt, vt, r, n_seqs, n_q)
    mine = torch.zeros(len(rt), dtype=torch.bool)
    mine[n_q:2 * n_q] = True
    assert same(out[~mine], ref[~mine])
    assert bool(out[mine][torch.tensor(rt)[mine] >= 0].isnan().all()) and not bool(out[mine][torch.tensor(rt)[mine] < 0].any())
    P.cb_destroy(ctx)


@pytest.mark.parametrize("hq,hkv,dh,plens,n_seqs", [(8, 8, 128, [24641, 100], 3), (32, 8, 128, [25013], 7), (48, 8, 64, [50111], 8)])
def test_attention_contexts_larger_than_the_caches(P, hq, hkv, dh, plens, n_seqs):
    """of 100 MB and more: loaded past the caches, one, two and four query blocks"""
    m, rng = U.model(hq, hkv, dh, "bf16"), random.Random(hq)
    rt = [rng.randint(-1, 60) for _ in range(len(plens) * n_seqs)]
    check_attention(P, m, plens, n_seqs, 1, 60, rt, 9, pstride=max(plens) + 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_more_groups_than_one_launch_numbers(P, dtype):
    m = U.model(2, 1, 64, dtype)
    rng = random.Random(5)
    check_attention(P, m, [rng.randint(0, 50) for _ in range(131)], 2, 1, 9, [rng.randint(-1, 9) for _ in range(262)], 6, pstride=50)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_without_contexts_without_tails_and_without_keys(P, dtype):
    m = U.model(6, 2, 64, dtype)
    check_attention(P, m, [0], 3, 2, 12, [1, 2, -1, 0, 12, 40], 8, pstride=0)       # more than the slab counts as the slab
    check_attention(P, m, [100], 3, 2, 0, [0, 0, -1, 5, 0, 0], 9)
    check_attention(P, m, [0], 2, 1, 0, [0, 3], 10, pstride=0)                      # nothing at all: zeros
    check_attention(P, m, [0, 0], 1, 1, 7, [0, 0], 11, pstride=20)


@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_attention_hidden_rows_have_no_influence(P, dtype, hq, hkv, dh, bad):
    """Context rows behind their length, tail rows behind a query's and other continuations' tails hold values that are not
    finite: bit for bit the result of finite ones, for every row that does not see them; NaN reaches those that do."""
    m, n_q, stride = U.model(hq, hkv, dh, dtype), 5, 45
    rt = [10, 11, 12, 13, 14, 0, 1, 2, 3, -1, 30, 31, 32, 33, 34]
    q, kp, vp, kt, vt, r = attention_case(m, [200], 3, n_q, stride, rt, 21, pstride=260)
    announce("shared attention, hidden rows", dtype, hq, hkv, dh, bad)
    ctx = P.cb_create(m, 8)
    ref = call_attention(P, ctx, q, kp, vp, [200], kt, vt, r, 3, n_q)
    for t in (kp, vp):
        t[:, 200:] = bad
    for t in (kt, vt):
        t[0, 14:] = bad
        t[1, 3:] = bad
        t[2, 32:] = bad                  # seen by the last two rows of the third continuation
    out = call_attention(P, ctx, q, kp, vp, [200], kt, vt, r, 3, n_q)
    assert same(out[:13], ref[:13])
    assert not bool(torch.isfinite(out[13:]).any())
    vt2, kt2 = vt.clone(), kt.clone()
    kt2[2, 32:] = 0.5                    # finite keys: the values alone spread
    out = call_attention(P, ctx, q, kp, vp, [200], kt2, vt2, r, 3, n_q)
    assert same(out[:13], ref[:13])
    if math.isnan(bad):
        assert bool(out[13:].isnan().all())
    else:                                # a visible infinity gives an infinity of its sign, not NaN
        assert bool((out[13:] == bad).all())
    P.cb_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("last", [0, 5, 31, 63])
def test_attention_visible_infinity_in_a_partly_filled_tile(P, dtype, last):
    """the last visible row holds an infinite value, the tile behind it is empty"""
    m = U.model(4, 2, 64, dtype)
    q, kp, vp, kt, vt, r = attention_case(m, [64], 1, 1, 100, [last + 1], 31)
    ctx = P.cb_create(m, 8)
    vt[0, last] = INF
    out = call_attention(P, ctx, q, kp, vp, [64], kt, vt, r, 1, 1)
    assert bool((out == INF).all())
    vp[0, 63], vt[0, last] = -INF, 1.0
    out = call_attention(P, ctx, q, kp, vp, [64], kt, vt, r, 1, 1)
    assert bool((out == -INF).all())
    P.cb_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_and_equal_scores(P, dtype):
    """scores far apart (one key takes everything), far below zero, and all equal"""
    m = U.model(4, 2, 128, dtype)
    q, kp, vp, kt, vt, r = attention_case(m, [300], 2, 1, 40, [20, 40], 41)
    ctx = P.cb_create(m, 8)
    for scale in (30.0, -30.0, 0.0):
        out = call_attention(P, ctx, q * scale, kp, vp, [300], kt, vt, r, 2, 1)
        ref, bound = U.attention(q * scale, kp, vp, [300], kt, vt, r, 2, 1, m.dtype)
        assert bool(((out.double() - ref).abs() <= bound).all()), scale
    P.cb_destroy(ctx)


def test_attention_output_over_the_queries_other_streams_and_repetition(P):
    m = U.model(8, 2, 128, "bf16")
    q, kp, vp, kt, vt, r = attention_case(m, [777], 4, 3, 50, [1, 2, 3, 10, 11, 12, 48, 49, 50, 7, -1, -1], 51)
    ctx = P.cb_create(m, 8)
    ref = call_attention(P, ctx, q, kp, vp, [777], kt, vt, r, 4, 3)
    for _ in range(3):
        assert same(call_attention(P, ctx, q, kp, vp, [777], kt, vt, r, 4, 3), ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        over = q.clone()
        call_attention(P, ctx, over, kp, vp, [777], kt, vt, r, 4, 3, out=over)
    torch.cuda.synchronize()
    assert same(over, ref)
    P.cb_destroy(ctx)


def test_calls_on_a_stream_of_their_own_keep_their_workspaces(P):
    """workspaces and outputs that the binding allocates are not handed out again while the other stream works on them"""
    m = U.model(8, 2, 128, "bf16")
    q, kp, vp, kt, vt, r = attention_case(m, [3000], 6, 1, 50, [1, 2, 3, 10, 11, 50], 52)
    x = U.normal((24, 20011), 17, std=3.0).cuda()
    s = U.normal((24,), 18).cuda()
    ctx = P.cb_create(m, 8)
    ref, best = call_attention(P, ctx, q, kp, vp, [3000], kt, vt, r, 6, 1), P.cb_beam_select(ctx, x, s, 3, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(10):
        got.append((call_attention(P, ctx, q, kp, vp, [3000], kt, vt, r, 6, 1, stream=side), P.cb_beam_select(ctx, x, s, 3, 16, stream=side)))
        junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(3)]       # takes freed memory on the current stream
        del junk
    torch.cuda.synchronize()
    for out, sel in got:
        assert same(out, ref) and all(torch.equal(a, b) for a, b in zip(sel, best))
    P.cb_destroy(ctx)


def test_attention_long_context_past_32_bit_offsets(P):
    """tails whose slabs lie more than 2^32 bytes into the array"""
    m = U.model(8, 8, 128, "bf16")
    rows = 2 ** 21 + 4096                                     # of 2 KB
    announce("shared attention, slabs past 2^32 bytes")
    big = torch.zeros((rows, 8, 128), dtype=torch.bfloat16, device="cuda")
    stride = rows // 2
    q, kp, vp, _, _, _ = attention_case(m, [50], 2, 1, 1, [1, 1], 61)
    kt, vt = big.view(2, stride, 8, 128), torch.zeros_like(big).view(2, stride, 8, 128)
    n = 9
    for t, seed in ((kt, 62), (vt, 63)):
        t[1, :n] = U.normal((n, 8, 128), seed, torch.bfloat16).cuda()
        t[0, stride - n:] = U.normal((n, 8, 128), seed + 2, torch.bfloat16).cuda()
    r = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    ctx = P.cb_create(m, 8)
    out = call_attention(P, ctx, q, kp, vp, [50], kt, vt, r, 2, 1)
    ref, bound = U.attention(q, kp, vp, [50], kt, vt, r, 2, 1, m.dtype)
    assert bool(((out.double() - ref).abs() <= bound).all())
    # a context that long: all but its last rows are equal keys and zero values
    kp2, vp2 = big.view(1, rows, 8, 128), vt.reshape(1, rows, 8, 128)
    kp2.zero_()
    kp2[0, -n:], vp2[0, -n:] = 8 * q[0].sign(), U.normal((n, 8, 128), 64, torch.bfloat16).cuda()
    r.zero_()
    out = call_attention(P, ctx, q[:1], kp2, vp2, [rows], kt[:1, :0], vt[:1, :0], r[:1], 1, 1)
    s = (8 * q[0].double().abs().sum(-1) / math.sqrt(128)).view(8, 1)
    w = torch.exp(s) / (n * torch.exp(s) + ((rows - n) - int((vp2[0, :-n].abs().sum((1, 2)) > 0).sum())))
    assert bool(((out[0].double() - w * vp2[0, -n:].double().sum(0)).abs() <= 0.02).all())
    P.cb_destroy(ctx)


# ---- head norms, rotation, cache append ------------------------------------------------------------------------------
@pytest.mark.parametrize("rope", ["adjacent", "half"])
@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("rows", [1, 7, 130])
def test_norm_rope_append(P, rope, dtype, hq, hkv, dh, norms, rows):
    announce("norm, rope, append", rope, dtype, hq, hkv, dh, norms, rows)
    m, dt, slots, far = U.model(hq, hkv, dh, dtype, rope=rope), U.TYPES[dtype], rows + 9, 5000
    ctx = P.cb_create(m, far)
    qkv = U.normal((rows, (hq + 2 * hkv) * dh), rows, dt).cuda()
    g = torch.Generator().manual_seed(rows)
    pos = torch.randint(0, far, (rows,), generator=g).to(torch.int32)
    pos[0] = far - 1
    slot = torch.randperm(slots, generator=g)[:rows].to(torch.int32)
    if rows > 5:                          # padding rows, rows that are not kept
        pos[2], pos[3] = -1, far
        slot[4], slot[5] = -1, slots
    gains = [(1 + U.normal((dh,), 5 + i, std=0.2)).to(dt).cuda() if norms else None for i in (0, 1)]
    k, v = (U.normal((slots, hkv, dh), 11 + i, dt).cuda() for i in (0, 1))
    k0, v0 = k.clone(), v.clone()
    q_out = U.normal((rows, hq, dh), 13, dt).cuda()
    q0 = q_out.clone()
    P.cb_qkv_norm_rope(ctx, qkv, pos.cuda(), slot.cuda(), k, v, gains[0], gains[1], q_out=q_out)
    x = qkv.view(rows, hq + 2 * hkv, dh)
    live = ((pos >= 0) & (pos < far)).cuda()
    ref, bound = U.rope(x[:, :hq], pos.cuda(), gains[0], m)
    assert bool(((q_out.double() - ref).abs() <= bound)[live].all()) and same(q_out[~live], q0[~live])
    ref, bound = U.rope(x[:, hq:hq + hkv], pos.cuda(), gains[1], m)
    kept = live & (slot >= 0).cuda() & (slot < slots).cuda()
    at = slot.cuda()[kept].long()
    assert bool(((k[at].double() - ref[kept]).abs() <= bound[kept]).all()) and same(v[at], x[kept, hq + hkv:])
    rest = torch.ones(slots, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert same(k[rest], k0[rest]) and same(v[rest], v0[rest])
    # three tensors of their own strides, the queries rotated in place
    q2 = x[:, :hq].reshape(rows, -1).clone()
    wide = torch.zeros((rows, hkv * dh + 16), dtype=dt, device="cuda")
    wide[:, :hkv * dh] = x[:, hq:hq + hkv].reshape(rows, -1)
    k2, v2 = k0.clone(), v0.clone()
    P.cb_qkv_norm_rope(ctx, (q2, wide[:, :hkv * dh], qkv[:, (hq + hkv) * dh:]), pos.cuda(), slot.cuda(), k2, v2, gains[0], gains[1],
                       q_out=q2.view(rows, hq, dh))
    assert same(q2.view(rows, hq, dh)[live], q_out[live]) and same(k2, k) and same(v2, v)
    P.cb_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_zero_and_large_heads(P, dtype):
    m = U.model(4, 2, 64, dtype)
    ctx, dt = P.cb_create(m, 16), U.TYPES[dtype]
    qkv = U.normal((3, 8 * 64), 3, dt)
    qkv[0] = 0
    qkv[1] *= 1e15
    gain = torch.ones(64, dtype=dt).cuda()
    pos, k = torch.tensor([3, 4, 5], dtype=torch.int32).cuda(), torch.zeros((3, 2, 64), dtype=dt, device="cuda")
    out = P.cb_qkv_norm_rope(ctx, qkv.cuda(), pos, pos - 3, k, torch.zeros_like(k), gain, gain)
    ref, bound = U.rope(qkv.view(3, 8, 64)[:, :4].cuda(), pos, gain, m)
    assert bool(((out.double() - ref).abs() <= bound).all())
    P.cb_destroy(ctx)


# ---- beam selection --------------------------------------------------------------------------------------------------
def check_select(P, ctx, logits, scores, n_groups, n_keep, finished=None, end_token=0):
    """Whole numbers as the definition gives them wherever its scores are further apart than the kernel's can be off: the sum of the
    exponentials is a float sum over 32 logits of a lane, 6 levels of a wavefront, the rest in double, each exponential 4 units off: 48 units of
    2^-24, and one rounding of the result."""
    got = [t.cpu() for t in P.cb_beam_select(ctx, logits, scores, n_groups, n_keep, finished, end_token)]
    every = U.beam_scores(logits, scores, finished, end_token)
    vocab, beams = logits.shape[1], logits.shape[0] // n_groups
    wants = U.best(every, n_groups, min(n_keep + 1, beams * vocab))
    every = every.cpu()
    for g in range(n_groups):
        want, seen = wants[g] + [(-INF, -1, -1)] * (n_keep + 1), set()
        for i in range(n_keep):
            s, b, t = float(got[0][g, i]), int(got[1][g, i]), int(got[2][g, i])
            ws, wb, wt = want[i]
            if ws == -INF:
                assert (s, b, t) == (-INF, -1, -1), (g, i, s, b, t)
                continue
            tol = 48 * 2.0 ** -24 + abs(ws) * 2.0 ** -24 if math.isfinite(ws) else 0.0
            assert s == ws or abs(s - ws) <= tol, (g, i, s, ws)
            assert (b, t) not in seen and 0 <= b < beams and 0 <= t < vocab
            seen.add((b, t))
            rest = torch.cat((every[g * beams:g * beams + wb], every[g * beams + wb + 1:(g + 1) * beams])) - ws
            if not bool(((rest.abs() <= 2 * tol) & (rest != 0)).any()):
                assert (b, t) == (wb, wt), (g, i, (s, b, t), want[i])
            else:                         # another beam's score is nearer than the float sums of both resolve, and not the same
                assert abs(float(every[g * beams + b, t]) - ws) <= 2 * tol


@pytest.fixture(scope="module")
def select_ctx(P):
    ctx = P.cb_create(U.model(4, 2, 64, "bf16"), 8)
    yield ctx
    P.cb_destroy(ctx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 500, 2047, 2048, 2049, 32000, 50257])
@pytest.mark.parametrize("groups,beams,keep", [(1, 1, 1), (1, 4, 8), (3, 5, 16), (2, 8, 64)])
def test_select(P, select_ctx, dtype, vocab, groups, beams, keep):
    announce("beam selection", dtype, vocab, groups, beams, keep)
    rows = groups * beams
    logits = U.normal((rows, vocab), vocab + beams, U.TYPES[dtype], 3.0).cuda()
    scores = (U.normal((rows,), vocab, std=2.0) - 10).cuda()
    check_select(P, select_ctx, logits, scores, groups, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_strided_rows_of_every_alignment(P, select_ctx, dtype):
    for pad, first in ((1, 0), (3, 1), (5, 2), (8, 3), (16, 0), (7, 7)):
        wide = U.normal((6, 3001 + pad + first), pad, U.TYPES[dtype], 2.0).cuda()
        wide[:, :first] = 100.0
        wide[:, first + 3001:] = 100.0                         # outside the rows: must not be looked at
        check_select(P, select_ctx, wide[:, first:first + 3001], torch.zeros(6, device="cuda"), 2, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", [1, 5, 64])
def test_select_ties_go_to_the_lower_beam_then_the_lower_token(P, select_ctx, dtype, keep):
    dt = U.TYPES[dtype]
    for fill in (0.0, -0.0, -7.5):
        x = torch.full((4, 5000), fill, dtype=dt)
        x[:, 1::3] = abs(fill) if fill else -fill              # +0 and -0 are equal
        check_select(P, select_ctx, x.cuda(), torch.zeros(4, device="cuda"), 2, keep)
    x = torch.zeros((8, 9000), dtype=dt)                       # more equal continuations than the lists hold
    check_select(P, select_ctx, x.cuda(), torch.zeros(8, device="cuda"), 1, keep)
    x = U.normal((3, 9000), 3, dt, 1.0).round()                # few distinct values, identical beams
    x[1:] = x[0]
    check_select(P, select_ctx, x.cuda(), torch.zeros(3, device="cuda"), 1, keep)
    x = torch.zeros((2, 4100), dtype=dt)
    x[:, [0, 2047, 2048, 4099]] = 1.0                          # equal ones in every stretch
    check_select(P, select_ctx, x.cuda(), torch.tensor([-1.0, -1.0], device="cuda"), 1, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_values_that_are_not_finite(P, select_ctx, dtype):
    x = U.normal((8, 6000), 9, U.TYPES[dtype], 2.0)
    x[0] = -INF                                                # nothing allowed
    x[1] = -INF
    x[1, [5, 4000, 5999]] = torch.tensor([1.0, 2.0, 2.0]).to(x.dtype)
    x[2] = NAN
    x[3, 100:] = NAN
    x[4, [7, 3000]] = INF
    x[5, :] = torch.finfo(x.dtype).min                         # a mask of the type's lowest value
    x[5, 17] = 0.5
    x[6, 0] = -INF
    scores = torch.tensor([0.0, -1.0, 0.0, -2.0, -3.0, -30.0, INF, NAN])
    for keep in (1, 6, 64):
        for rows in ([0, 1, 2, 3], [3, 4, 5, 6], [0, 2, 6, 7], [7, 5, 4, 1], [1, 1, 1, 1]):
            check_select(P, select_ctx, x[rows].cuda(), scores[rows].cuda(), 1, keep)
        check_select(P, select_ctx, x.cuda(), scores.cuda(), 2, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_finished_beams_go_on_with_the_end_token(P, select_ctx, dtype):
    x = U.normal((6, 4000), 13, U.TYPES[dtype], 2.0)
    x[1] = NAN                                                 # a finished beam's logits are not looked at
    scores = torch.tensor([-4.0, -5.0, -6.5, -40.0, -1.0, -INF])
    for done in ([0, 1, 0, 0, 1, 0], [1, 1, 1, 1, 1, 1], [0, 1, 0, 5, -1, 1]):
        for keep in (1, 4, 9, 64):
            check_select(P, select_ctx, x.cuda(), scores.cuda(), 2, keep, torch.tensor(done, dtype=torch.int32).cuda(), 3999)


def test_select_large_logits_and_scores_lose_nothing(P, select_ctx):
    """a common offset of the logits changes no score; beams whose scores differ by less than a float step at their size stay apart
    as long as their float inputs do"""
    x = U.normal((4, 3000), 15, std=1.0)
    for offset in (-1e4, 1e4):
        check_select(P, select_ctx, (x + offset).cuda(), torch.tensor([-1.0, -2.0, -3.0, -4.0]).cuda(), 1, 12)
    check_select(P, select_ctx, (x * 40).cuda(), torch.tensor([-1000.0, -1000.5, -1001.0, -900.0]).cuda(), 1, 12)


def test_select_repeats_bit_for_bit(P, select_ctx):
    x, s = U.normal((24, 20011), 17, std=3.0).cuda(), U.normal((24,), 18).cuda()
    ref = P.cb_beam_select(select_ctx, x, s, 3, 16)
    for _ in range(3):
        got = P.cb_beam_select(select_ctx, x, s, 3, 16)
        assert same(got[0], ref[0]) and torch.equal(got[1], ref[1]) and torch.equal(got[2], ref[2])


# ---- reordering ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,hkv,dh", [("bf16", 8, 128), ("bf16", 1, 64), ("f32", 2, 64)])
@pytest.mark.parametrize("groups,beams,stride,layers", [(1, 2, 1, 1), (3, 4, 17, 2), (2, 8, 33, 3), (1, 13, 50, 2), (2, 31, 9, 1),
                                                        (1, 64, 12, 2), (1, 3, 40, 131)])
def test_reorder(P, dtype, hkv, dh, groups, beams, stride, layers):
    announce("reorder", dtype, hkv, dh, groups, beams, stride, layers)
    m, n = U.model(hkv, hkv, dh, dtype, layers), groups * beams
    ctx = P.cb_create(m, 8)
    rng = random.Random(beams)
    shape = (n * stride, hkv, dh)
    ks = [U.normal(shape, 2 * l, U.TYPES[dtype]).cuda() for l in range(layers)]
    vs = [U.normal(shape, 2 * l + 1, U.TYPES[dtype]).cuda() for l in range(layers)]
    for kind in ("random", "rotate", "first", "same", "outside", "whole"):
        parent = {"rotate": [(b + 1) % beams for b in range(beams)] * groups, "first": [0] * n,
                  "same": list(range(beams)) * groups, "outside": [rng.choice([-1, beams, 0, 2 ** 31 - 1]) for _ in range(n)]
                  }.get(kind, [rng.randrange(beams) for _ in range(n)])
        lens = None if kind == "whole" else [rng.randint(0, stride) for _ in range(n)]
        refs = []
        for t in ks + vs:
            old, new = t.view(n, stride, -1).clone(), t.view(n, stride, -1).clone()
            for b, p in enumerate(parent):
                if 0 <= p < beams:
                    a = b // beams * beams + p
                    ln = stride if lens is None else lens[a]
                    new[b, :ln] = old[a, :ln]
            refs.append(new)
        P.cb_beam_reorder(ctx, ks, vs, groups, torch.tensor(parent, dtype=torch.int32, device="cuda"),
                          None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        for t, ref in zip(ks + vs, refs):
            assert same(t.view(n, stride, -1), ref), kind
    # all layers of one tensor; lengths outside a slab count as its ends
    both = torch.stack(ks), torch.stack(vs)
    parent = torch.tensor([(b + 1) % beams for b in range(beams)] * groups, dtype=torch.int32, device="cuda")
    lens = torch.tensor([stride + 5 if i % 2 else -3 for i in range(n)], dtype=torch.int32, device="cuda")
    P.cb_beam_reorder(ctx, ks, vs, groups, parent, lens.clamp(0, stride))
    P.cb_beam_reorder(ctx, both[0], both[1], groups, parent, lens)
    assert same(both[0], torch.stack(ks)) and same(both[1], torch.stack(vs))
    P.cb_destroy(ctx)
