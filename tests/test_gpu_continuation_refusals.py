"""What the operators of the continuations refuse, before any launch: through the C ABI with tensors that the calls must not touch, and
through the binding's own checks."""
import ctypes as C

import pytest
import torch

import continuation_util as U

pytestmark = pytest.mark.gpu

OK, EINVAL, ENULL, EWORKSPACE, EUNSUPPORTED = 0, -1, -2, -3, -4


@pytest.fixture(scope="module")
def env():
    import paper_2405_16444_amd as P
    from paper_2405_16444_amd import binding
    ctx = P.cb_create(U.model(4, 2, 64, "bf16", layers=3), 32)
    buf = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    yield P, binding._lib, ctx, buf
    torch.cuda.synchronize()
    assert not bool(buf.any())                       # no refused call wrote anything
    P.cb_destroy(ctx)


def call(fn, args, **change):
    return fn(*{**args, **change}.values())


def test_norm_rope_refusals(env):
    P, lib, ctx, buf = env
    p = buf.data_ptr()
    good = dict(ctx=ctx._h, q=p, qs=512, k=p, ks=512, v=p, vs=512, qn=None, kn=None, pos=p, row=p, n=3, out=p, kc=p, vc=p, rows=8, s=None)
    f = lib.cb_qkv_norm_rope
    assert call(f, good, n=0) == OK
    for name in ("ctx", "q", "k", "v", "pos", "row", "out", "kc", "vc"):
        assert call(f, good, **{name: None}) == ENULL, name
    for name in ("q", "k", "v", "qn", "kn", "out", "kc", "vc"):
        assert call(f, good, **{name: p + 8}) == EINVAL, name
    assert call(f, good, n=1 << 24) == EUNSUPPORTED
    for bad in (dict(pos=p + 2), dict(row=p + 1), dict(n=-1), dict(rows=-1), dict(qs=248), dict(ks=127), dict(vs=120), dict(qs=257), dict(ks=132)):
        assert call(f, good, **bad) == EINVAL, bad


def test_attention_refusals(env):
    P, lib, ctx, buf = env
    p, lens = buf.data_ptr(), (C.c_int32 * 2)(5, 9)
    size = P.cb_shared_prefix_workspace_bytes(ctx, 2, 3, 1, 9, 4)
    good = dict(ctx=ctx._h, q=p, g=2, n=3, nq=1, kp=p, vp=p, lens=lens, ps=9, kt=p, vt=p, ts=4, rt=p, o=p, ws=p, size=size, s=None)
    f = lib.cb_shared_prefix_attention
    for name in ("ctx", "q", "kp", "vp", "lens", "kt", "vt", "rt", "o", "ws"):
        assert call(f, good, **{name: None}) == ENULL, name
    for name in ("q", "kp", "vp", "kt", "vt", "o"):
        assert call(f, good, **{name: p + 8}) == EINVAL, name
    for bad in (dict(ws=p + 128), dict(rt=p + 2), dict(g=0), dict(n=0), dict(nq=-1), dict(ps=8), dict(ps=-1), dict(ts=-1),
                dict(lens=(C.c_int32 * 2)(5, -1))):
        assert call(f, good, **bad) == EINVAL, bad
    assert call(f, good, size=size - 1) == EWORKSPACE
    assert call(f, good, n=1 << 22, nq=1 << 22) == EUNSUPPORTED and call(f, good, n=1 << 30) == EUNSUPPORTED and call(f, good, g=1, n=(1 << 21) + 1) == EUNSUPPORTED
    for bad in ((0, 1, 1, 5, 5), (1, 0, 1, 5, 5), (1, 1, 0, 5, 5), (1, 1, 1, -1, 5), (1, 1, 1, 5, -1), (1 << 20, 1 << 20, 1, 5, 5)):
        assert P.cb_shared_prefix_workspace_bytes(ctx, *bad) == 0, bad
    assert lib.cb_shared_prefix_workspace_bytes(None, 1, 1, 1, 1, 1) == 0


def test_attention_workspace_holds_for_shorter_contexts(env):
    P, _, ctx, _ = env
    for shape in ((1, 4, 1), (5, 2, 3), (130, 1, 1), (1, 16, 64)):
        sizes = [P.cb_shared_prefix_workspace_bytes(ctx, *shape, n, 50) for n in range(0, 9000, 37)]
        assert sizes == sorted(sizes)


def test_select_refusals(env):
    P, lib, ctx, buf = env
    p = buf.data_ptr()
    size = P.cb_beam_select_workspace_bytes(ctx, 2, 3, 100, 5)
    good = dict(ctx=ctx._h, x=p, dt=0, ld=100, g=2, b=3, vocab=100, sc=p, done=None, end=0, keep=5, so=p, bo=p, to=p, ws=p, size=size, s=None)
    f = lib.cb_beam_select
    for name in ("ctx", "x", "sc", "so", "bo", "to", "ws"):
        assert call(f, good, **{name: None}) == ENULL, name
    for bad in (dict(x=p + 2), dict(dt=1, x=p + 1), dict(dt=2), dict(dt=-1), dict(ld=99), dict(g=0), dict(b=0), dict(vocab=0), dict(keep=0),
                dict(sc=p + 2), dict(done=p + 2), dict(done=p, end=100), dict(done=p, end=-1), dict(so=p + 1), dict(bo=p + 2), dict(to=p + 3),
                dict(ws=p + 16)):
        assert call(f, good, **bad) == EINVAL, bad
    assert call(f, good, size=size - 1) == EWORKSPACE
    for bad in (dict(keep=65), dict(b=65), dict(g=30000), dict(vocab=(1 << 30) + 1, ld=1 << 31)):
        assert call(f, good, **bad) == EUNSUPPORTED, bad
    for bad in ((0, 1, 10, 1), (1, 65, 10, 1), (1, 1, 0, 1), (1, 1, 10, 65), (40000, 2, 10, 1)):
        assert P.cb_beam_select_workspace_bytes(ctx, *bad) == 0, bad


def test_reorder_refusals(env):
    P, lib, ctx, buf = env
    p = buf.data_ptr()
    ptrs, others = (C.c_void_p * 3)(p, p, p), (C.c_void_p * 3)(p + 64, p + 64, p + 64)
    good = dict(ctx=ctx._h, k=ptrs, v=others, l0=0, l1=3, g=2, b=4, ts=8, parent=p, len=None, s=None)
    f = lib.cb_beam_reorder
    for name in ("ctx", "k", "v", "parent"):
        assert call(f, good, **{name: None}) == ENULL, name
    assert call(f, good, k=(C.c_void_p * 3)(p, None, p)) == ENULL and call(f, good, v=(C.c_void_p * 3)(p + 64, p + 64, p + 4)) == EINVAL
    assert call(f, good, v=ptrs) == EINVAL                                            # K and V of a layer in one array
    assert call(f, good, k=(C.c_void_p * 3)(p, None, p), l0=2) == OK                # layers outside the range are not looked at
    for bad in (dict(l0=-1), dict(l1=4), dict(l0=2, l1=1), dict(g=0), dict(b=0), dict(ts=-1), dict(parent=p + 2), dict(len=p + 1)):
        assert call(f, good, **bad) == EINVAL, bad
    for bad in (dict(b=65), dict(g=65536)):
        assert call(f, good, **bad) == EUNSUPPORTED, bad
    for empty in (dict(l0=3), dict(ts=0), dict(b=1)):
        assert call(f, good, **empty) == OK, empty


def test_binding_checks_what_it_is_given(env):
    P, _, ctx, _ = env
    dt, i32 = torch.bfloat16, torch.int32

    def z(*shape, dtype=dt, device="cuda"):
        return torch.zeros(shape, dtype=dtype, device=device)
    idx = z(3, dtype=i32)
    k = z(8, 2, 64)
    for args in ((z(3, 511), idx, idx, k, k), (z(3, 512, dtype=torch.float32), idx, idx, k, k), (z(3, 512), z(3, dtype=torch.int64), idx, k, k),
                 (z(3, 512), idx, z(2, dtype=i32), k, k), (z(3, 512), idx, idx, z(8, 1, 64), k), (z(3, 512, device="cpu"), idx, idx, k, k),
                 (z(512, 3).T, idx, idx, k, k), (z(3, 512), idx, idx, k, z(16, 2, 64)[::2])):
        with pytest.raises(AssertionError):
            P.cb_qkv_norm_rope(ctx, *args)
    q, kt, rt = z(4, 4, 64), z(40, 2, 64), z(4, dtype=i32)
    for args in ((q, 1, 3, 1, k, k, [8], kt, kt, rt), (q, 1, 4, 1, k, k, [8, 8], kt, kt, rt), (q, 1, 4, 1, k, k, [8], z(39, 2, 64), z(39, 2, 64), rt),
                 (q, 1, 4, 1, k, k, [8], kt, kt, rt.long()), (z(4, 4, 64, device="cpu"), 1, 4, 1, k, k, [8], kt, kt, rt),
                 (q, 1, 4, 1, k, z(9, 2, 64), [8], kt, kt, rt)):
        with pytest.raises(AssertionError):
            P.cb_shared_prefix_attention(ctx, *args)
    with pytest.raises(P.CacheBlendError) as e:
        P.cb_shared_prefix_attention(ctx, q, 1, 4, 1, k, k, [9], kt, kt, rt)
    assert e.value.status == EINVAL
    x, s = z(4, 50, dtype=torch.float32), z(4, dtype=torch.float32)
    for args in ((x.half(), s, 1, 2), (x, s.double(), 1, 2), (x, s[:3], 1, 2), (x, s, 3, 2), (x.cpu(), s, 1, 2), (x.T, s, 1, 2), (x, s, 1, 2, rt.long())):
        with pytest.raises(AssertionError):
            P.cb_beam_select(ctx, *args)
    with pytest.raises(P.CacheBlendError) as e:
        P.cb_beam_select(ctx, x, s, 1, 65)
    assert e.value.status == EUNSUPPORTED
    for args in (([kt], [kt, kt], 1, rt), ([kt], [kt[:20]], 1, rt), ([kt], [kt.clone()], 3, rt), ([kt], [kt.clone()], 1, rt.long()),
                 ([kt.float()], [kt.float()], 1, rt)):
        with pytest.raises(AssertionError):
            P.cb_beam_reorder(ctx, *args)


def test_calls_are_timed_under_their_class(env):
    P, _, ctx, _ = env
    P.cb_profile_enable(ctx, 1)
    k, rt = torch.zeros((8, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    P.cb_qkv_norm_rope(ctx, torch.zeros((4, 512), dtype=torch.bfloat16, device="cuda"), rt, rt, k, k.clone())
    P.cb_shared_prefix_attention(ctx, torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda"), 1, 4, 1, k, k, [8], k, k, rt)
    P.cb_beam_select(ctx, torch.zeros((4, 50), device="cuda"), torch.zeros(4, device="cuda"), 1, 2)
    P.cb_beam_reorder(ctx, [k], [k.clone()], 1, rt)
    got = P.cb_profile_read(ctx)
    P.cb_profile_enable(ctx, 0)
    assert {c: got[c]["launches"] for c in ("norm", "attention", "first_token", "other")} == dict.fromkeys(("norm", "attention", "first_token", "other"), 1)
