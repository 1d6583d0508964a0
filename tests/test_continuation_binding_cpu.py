"""What the binding of the continuations' calls hands to the library, without a device: a library that only takes notes, and tensors of the host that
stand for a device's (both have the number -1)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2405_16444_amd import binding as B


class Notes:
    """Stands for the library: every call is noted and succeeds"""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or (256 if name.endswith("workspace_bytes") else 0)


@pytest.fixture
def lib(monkeypatch):
    notes = Notes()
    monkeypatch.setattr(B, "_lib", notes)
    monkeypatch.setattr(B, "_current_stream", lambda ctx, stream: 0)
    return notes


def context():
    model = SimpleNamespace(n_layers=3, n_q_heads=4, n_kv_heads=2, head_dim=64)
    return SimpleNamespace(_h=1, model=model, dtype=torch.bfloat16, device=SimpleNamespace(index=-1))


class Elsewhere:
    """A workspace on another device than the context's"""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def attention(workspace):
    z = lambda *shape, dt=torch.bfloat16: torch.zeros(shape, dtype=dt)
    k, kt = z(8, 2, 64), z(20, 2, 64)
    return B.cb_shared_prefix_attention(context(), z(4, 4, 64), 1, 4, 1, k, k, [8], kt, kt, z(4, dt=torch.int32), out=z(4, 4, 64), workspace=workspace)


def select(workspace):
    out = (torch.zeros(1, 2), torch.zeros((1, 2), dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32))
    return B.cb_beam_select(context(), torch.zeros(4, 50), torch.zeros(4), 1, 2, workspace=workspace, out=out)


@pytest.mark.parametrize("call,size_at", [(attention, -2), (select, -2)])
def test_workspaces_are_checked_like_every_tensor(lib, call, size_at):
    room = torch.zeros(1024, dtype=torch.uint8)
    call(room)
    assert lib.calls[-1][1][size_at] == 1024
    call(room.view(torch.float32))                   # bytes, whatever the type
    assert lib.calls[-1][1][size_at] == 1024
    n = len(lib.calls)
    for bad in (Elsewhere(room), room[::2]):
        with pytest.raises(AssertionError):
            call(bad)
    assert len(lib.calls) == n
