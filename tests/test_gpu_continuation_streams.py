"""The continuations' calls on a stream of their own, with results and workspaces that the binding allocates, while the current stream has work waiting
on memory that it has already given back."""
import pytest
import torch

import continuation_util as U
from gpu_util import announce

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2405_16444_amd as pkg
    return pkg


def busy(slow):
    """some 50 ms of work for the current stream"""
    for _ in range(200):
        slow.fill_(1.0)


def calls(P):
    m = U.model(8, 2, 128, "bf16")
    ctx = P.cb_create(m, 64)
    q, kp, vp = U.normal((6, 8, 128), 1, torch.bfloat16).cuda(), *(U.normal((3000, 2, 128), i, torch.bfloat16).cuda() for i in (2, 3))
    kt, vt = (U.normal((300, 2, 128), i, torch.bfloat16).cuda() for i in (4, 5))
    r = torch.tensor([1, 2, 3, 10, 11, 50], dtype=torch.int32, device="cuda")
    x, s = U.normal((24, 20011), 6, std=3.0).cuda(), U.normal((24,), 7).cuda()
    qkv = U.normal((6, 12 * 128), 8, torch.bfloat16).cuda()
    return ctx, [
        lambda **kw: [P.cb_shared_prefix_attention(ctx, q, 1, 6, 1, kp, vp, [3000], kt, vt, r, **kw)],
        lambda **kw: list(P.cb_beam_select(ctx, x, s, 3, 16, **kw)),
        lambda **kw: [P.cb_qkv_norm_rope(ctx, qkv, r, r - 100, kt, vt, **kw)]]                  # the caches are left as they are


@pytest.mark.parametrize("which", [0, 1, 2])
def test_memory_that_waiting_work_still_writes_is_not_taken(P, which):
    ctx, every = calls(P)
    call = every[which]
    announce("calls beside waiting work", which)
    want = [t.clone() for t in call()]
    size = [P.cb_shared_prefix_workspace_bytes(ctx, 1, 6, 1, 3000, 50), P.cb_beam_select_workspace_bytes(ctx, 3, 8, 20011, 16), 512][which]
    slow, side = torch.empty(1 << 26, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(slow)
    junk = [torch.full_like(t, 77) for t in want for _ in range(3)] + [torch.full((size,), 77, dtype=torch.uint8, device="cuda") for _ in range(3)]
    taken = {t.data_ptr() for t in junk}
    del junk                                      # the fills still wait behind the slow work
    got = call(stream=side)
    assert not torch.cuda.current_stream().query()
    side.synchronize()
    assert not taken & {t.data_ptr() for t in got}
    torch.cuda.synchronize()                      # the fills are over
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    P.cb_destroy(ctx)


@pytest.mark.parametrize("which", [0, 1, 2])
def test_results_that_waiting_work_still_reads_are_not_written_over(P, which):
    ctx, every = calls(P)
    call = every[which]
    announce("results read late", which)
    slow, side = torch.empty(1 << 26, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(stream=side)
    want = [t.clone() for t in call()]
    torch.cuda.current_stream().wait_stream(side)
    busy(slow)
    read = [t.clone() for t in got]               # waits behind the slow work
    at = {t.data_ptr() for t in got}
    del got
    again = [call(stream=side) for _ in range(3)]
    assert not torch.cuda.current_stream().query()
    assert not at & {t.data_ptr() for ts in again for t in ts}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(read, want))
    P.cb_destroy(ctx)
