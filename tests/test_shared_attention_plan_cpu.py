"""The launches of attention over a shared context, asked of the library's planner without a device."""
import itertools
import re

import pytest
import torch

import continuation_util as U


def threads(m, n_groups, n_seqs, n_q, prefix, stride):
    """of the launch that reads contexts and tails, from its plan: a work item for every piece of every block of queries and key/value head"""
    p = U.attention_plan(m, n_groups, n_seqs, n_q, prefix, stride)
    items = n_groups * n_seqs * p.tail_blocks * p.tail_pieces + (0 if p.wide else n_groups * p.ctx_blocks * p.ctx_pieces)
    return items * m.n_kv_heads * (256 if p.qb == 1 else 512)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(32, 32), (32, 8), (64, 1), (128, 1), (8, 1), (1, 1)])
def test_accepted_launches_number_their_threads_with_32_bits(dtype, hq, hkv):
    m, accepted = U.model(hq, hkv, 128, dtype), 0
    for groups in (1, 3, 64):
        for n_q in (1, 2, 64):
            for shift in range(0, 24):
                for n_seqs in ((1 << shift) - 1, 1 << shift):
                    for prefix in (0, 1, 40, 100000):
                        for stride in (0, 1, 700, 40000):
                            if n_seqs == 0 or n_seqs * groups * n_q * hq > 1 << 23:
                                continue
                            if U.attention_plan(m, groups, n_seqs, n_q, prefix, stride) is None:
                                assert groups * n_seqs * n_q * hq > 1 << 22
                            else:
                                accepted += 1
                                assert threads(m, groups, n_seqs, n_q, prefix, stride) < 1 << 32
    assert accepted > 1000


def test_the_largest_launch_is_refused():
    m = U.model(32, 32, 128, "bf16")
    # a tail of one row, and none: 2^23 key/value heads of 512 threads
    assert U.attention_plan(m, 64, 4096, 1, 0, 1) is None and U.attention_plan(m, 64, 4096, 1, 40, 1) is None
    assert U.attention_plan(m, 64, 4096, 1, 40, 0) is not None and U.attention_plan(m, 64, 3900, 1, 40, 1) is not None
    assert U.attention_plan(m, 64, 4097, 1, 40, 0) is None


def test_every_kernel_that_is_built_is_reached_by_some_plan():
    from paper_2405_16444_amd import build
    names = re.findall(rb"shared_attn_bf16_kernelILi(\d+)ELi(\d)ELi\dELi\dELb(\d)ELb(\d)ELb(\d)E", open(build.LIB_PATH, "rb").read())
    built = {tuple(map(int, n)) for n in names}                      # head_dim, query blocks, several tokens, past the caches, folding
    reached = set()
    for dh, (hq, hkv), n_seqs, n_q, prefix in itertools.product(
            (64, 128), ((32, 32), (32, 8), (64, 8), (32, 1), (64, 1), (128, 1), (5, 5), (48, 8)), (1, 3, 8, 64, 128, 256, 512, 1024),
            (1, 2, 4, 8, 64), (40, 600, 3000, 30000, 100000)):
        p = U.attention_plan(U.model(hq, hkv, dh, "bf16"), 1, n_seqs, n_q, prefix, 32)
        if p is not None:
            reached.add((dh, p.qb, int(n_q > 1), p.stream, p.fold))
    assert len(built) == 38 and built == reached, (sorted(built - reached), sorted(reached - built))


def test_the_shapes_of_the_gpu_test_reach_every_kernel():
    every = {(dh, *what, int(shape[4] > 1)) for dh in (64, 128) for shape, what in U.plan_shapes(dh)}
    assert len(every) == 38
    for dh in (64, 128):
        for (hq, hkv, prefix, n_seqs, n_q), what in U.plan_shapes(dh):
            p = U.attention_plan(U.model(hq, hkv, dh, "bf16"), 1, n_seqs, n_q, prefix, n_q + 20)
            assert (p.qb, p.stream, p.fold) == what, (dh, hq, hkv, prefix, n_seqs, n_q, p)


@pytest.mark.parametrize("dh", [64, 128])
def test_bound_notices_a_lost_tile_of_the_longest_context(dh):
    """with the coded values; with normal ones the output shrinks with the number of keys and the bound does not"""
    prefix = U.plan_shapes(dh)[0][0][2]
    q, k = U.normal((1, 2, dh), 1, torch.bfloat16), U.normal((1, prefix, 2, dh), 2, torch.bfloat16)
    v = U.coded_values(prefix, 2, dh).to(torch.bfloat16)
    none = torch.zeros((1, 0, 2, dh), dtype=torch.bfloat16)
    ref, bound = U.attention(q, k, v[None], [prefix], none, none, [0], 1, 1, "bf16")
    for h in range(2):
        p = torch.softmax(k[0, :, h].double() @ q[0, h].double() / dh ** 0.5, 0)
        part = torch.zeros(((prefix + 31) // 32, dh), dtype=torch.float64).index_add_(0, torch.arange(prefix) // 32, p[:, None] * v[:, h].double())
        share = torch.zeros(len(part), dtype=torch.float64).index_add_(0, torch.arange(prefix) // 32, p)
        assert torch.allclose(part.sum(0), ref[0, h], rtol=0, atol=1e-12)
        lost = (part.sum(0) - part) / (1 - share)[:, None]
        twice = (part.sum(0) + part) / (1 + share)[:, None]
        for wrong in (lost[:-1], twice[:-1]):              # the last tile has a few rows only
            assert bool(((wrong - ref[0, h]).abs() > bound[0, h]).any(1).all())


@pytest.mark.parametrize("dh,prefix,tail", [(64, 437, 83), (64, 25033, 20), (128, 1003, 83), (128, 12745, 20)])
def test_bound_notices_a_border_row(dh, prefix, tail):
    dt = torch.bfloat16
    q, kp, vp = U.normal((1, 2, dh), 1, dt), U.normal((1, prefix + 40, 2, dh), 2, dt), U.normal((1, prefix + 40, 2, dh), 3, dt)
    kt, vt = U.normal((1, tail + 1, 2, dh), 4, dt), U.normal((1, tail + 1, 2, dh), 5, dt)
    q, kp, kt = U.towards_borders(q, kp, kt, prefix)

    def call(kp, vp, prefix, tail):
        return U.attention(q, kp, vp, [prefix], kt, vt, [tail], 1, 1, "bf16")
    ref, bound = call(kp, vp, prefix, tail)
    wrong = [call(kp, vp, prefix + 1, tail), call(kp, vp, prefix, tail - 1), call(kp, vp, prefix, tail + 1)]
    for row in U.border_rows(prefix):
        left = [i for i in range(prefix) if i != row]
        wrong.append(call(kp[:, left], vp[:, left], prefix - 1, tail))
    for out, _ in wrong:
        assert bool(((out - ref).abs() > bound).any())
