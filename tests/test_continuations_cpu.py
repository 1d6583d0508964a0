"""The continuations' operators without a device: refusals that come before any device call, and the references that the GPU tests hold
the kernels to, against library routines and against mistakes planted in their inputs."""
import ctypes
import math

import pytest
import torch

import continuation_util as U


def test_calls_without_a_context_are_refused():
    from paper_2405_16444_amd.binding import _lib
    lens = (ctypes.c_int32 * 1)(1)
    ptrs = (ctypes.c_void_p * 1)(16)
    assert _lib.cb_qkv_norm_rope(None, 16, 8, 16, 8, 16, 8, None, None, 16, 16, 1, 16, 16, 16, 1, None) == -2
    assert _lib.cb_shared_prefix_attention(None, 16, 1, 1, 1, 16, 16, lens, 1, 16, 16, 1, 16, 16, 256, 0, None) == -2
    assert _lib.cb_beam_select(None, 16, 0, 8, 1, 1, 8, 16, None, 0, 1, 16, 16, 16, 256, 0, None) == -2
    assert _lib.cb_beam_reorder(None, ptrs, ptrs, 0, 1, 1, 1, 1, 16, None, None) == -2
    assert _lib.cb_shared_prefix_workspace_bytes(None, 1, 1, 1, 1, 1) == 0
    assert _lib.cb_beam_select_workspace_bytes(None, 1, 1, 8, 1) == 0


def attention_inputs():
    q, kp, vp = U.normal((6, 4, 64), 1), U.normal((1, 40, 2, 64), 2), U.normal((1, 40, 2, 64), 3)
    kt, vt = U.normal((3, 9, 2, 64), 4), U.normal((3, 9, 2, 64), 5)
    return q, kp, vp, kt, vt, [3, 4, 9, -1, 0, 1]


def test_attention_reference_is_a_masked_softmax():
    q, kp, vp, kt, vt, seen = attention_inputs()
    out, bound = U.attention(q, kp, vp, [37], kt, vt, torch.tensor(seen), 3, 2, "f32")
    for r, n in enumerate(seen):
        if n < 0:
            assert not bool(out[r].any())
            continue
        k, v = (torch.cat((c[0, :37], t[r // 2, :n])).double().repeat_interleave(2, 1).transpose(0, 1) for c, t in ((kp, kt), (vp, vt)))
        ref = torch.nn.functional.scaled_dot_product_attention(q[r].double()[:, None], k, v)[:, 0]
        assert torch.allclose(out[r], ref, rtol=0, atol=1e-12)
    # with values of at most 4.5: 2 x 4.5 x 68 x 2^-24 x (64 x 4.5^2 / 8)
    assert bool((bound[:3] > 0).all()) and float(bound.max()) < 6e-3


@pytest.mark.parametrize("mistake", ["one key more", "a hidden row", "another tail", "the other group's head"])
def test_attention_reference_notices(mistake):
    q, kp, vp, kt, vt, seen = attention_inputs()
    ref, bound = U.attention(q, kp, vp, [37], kt, vt, torch.tensor(seen), 3, 2, "bf16")
    if mistake == "one key more":
        out, _ = U.attention(q, kp, vp, [38], kt, vt, torch.tensor(seen), 3, 2, "bf16")
    elif mistake == "a hidden row":
        out, _ = U.attention(q, kp, vp, [37], kt, vt, torch.tensor([v + 1 if v >= 0 else v for v in seen]), 3, 2, "bf16")
    elif mistake == "another tail":
        out, _ = U.attention(q, kp, vp, [37], kt.roll(1, 0), vt.roll(1, 0), torch.tensor(seen), 3, 2, "bf16")
    else:
        out, _ = U.attention(q, kp.flip(2), vp.flip(2), [37], kt, vt, torch.tensor(seen), 3, 2, "bf16")
    assert bool(((out - ref).abs() > bound).any())


@pytest.mark.parametrize("layout", ["adjacent", "half"])
def test_rope_reference_is_a_complex_product(layout):
    m = U.model(3, 1, 64, "f32", rope=layout, theta=5e5)
    x, pos, gain = U.normal((7, 3, 64), 1), torch.tensor([0, 1, 5, 100, 4095, 30000, 2]), 1 + U.normal((64,), 2, std=0.1)
    y = torch.nn.functional.rms_norm(x.double(), (64,), gain.double(), m.rms_eps)
    z = torch.complex(y[..., 0::2], y[..., 1::2]) if layout == "adjacent" else torch.complex(y[..., :32], y[..., 32:])
    z = z * torch.polar(torch.ones(1, dtype=torch.float64), pos.double()[:, None, None] * m.rope_theta ** (-torch.arange(32).double() / 32))
    ref = torch.stack((z.real, z.imag), -1).flatten(-2) if layout == "adjacent" else torch.cat((z.real, z.imag), -1)
    assert torch.allclose(U.rope(x, pos, gain, m)[0], ref, rtol=0, atol=1e-11)


def test_selection_reference_is_a_log_softmax():
    x, s = U.normal((4, 50), 1, std=2.0), torch.tensor([-1.0, -2.0, float("-inf"), -0.5])
    every = U.beam_scores(x, s)
    assert torch.allclose(every[[0, 1, 3]], (s.double()[:, None] + torch.log_softmax(x.double(), -1))[[0, 1, 3]], rtol=0, atol=1e-12)
    assert bool((every[2] == -math.inf).all())
    flat = sorted(((-float(v), b, t) for b, row in enumerate(every) for t, v in enumerate(row) if v > -math.inf))
    assert U.best(every, 1, 9)[0] == [(-v, b, t) for v, b, t in flat[:9]]
    x[1, 7] = x[1, 9] = math.inf
    x[0, 3] = math.nan
    every = U.beam_scores(x, s, torch.tensor([0, 0, 0, 1]), 5)
    assert every[1, 7] == every[1, 9] == -2.0 - math.log(2) and every[1].isinf().sum() == 48
    assert every[0, 3] == -math.inf and every[3, 5] == -0.5 and every[3].isinf().sum() == 49
    assert len(U.best(every, 2, 60)[1]) == 60 and U.best(every, 2, 60)[1][-1] == (-math.inf, -1, -1)
