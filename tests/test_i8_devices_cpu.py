"""Tensors of two devices in one call of rs_residual_norm_fwd are refused before anything is launched; host side only: the tensors are
stand-ins that say where they are, the library one that notes what reaches it."""
import pytest
import torch

import paper_2508_00367_amd as rs
from paper_2508_00367_amd import binding


class _There:
    """What the binding asks of a tensor."""
    dtype = torch.float32

    def __init__(self, device, *shape):
        self.device_index, self.shape = device, shape

    def get_device(self):
        return self.device_index

    def stride(self, i=None):
        return {-1: 1, 0: self.shape[-1]}[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return torch.Size(self.shape).numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000000 * (self.device_index + 1)


class _Library:
    def __init__(self):
        self.calls = 0

    def rs_residual_norm_fwd(self, *args):
        self.calls += 1
        return rs.RS_OK


@pytest.fixture
def machine(monkeypatch):
    """Two devices; machine(i) makes device i the current one."""
    library, current = _Library(), [0]
    monkeypatch.setattr(binding, "_lib", library)
    monkeypatch.setattr(binding, "_current_device", lambda: current[0])
    monkeypatch.setattr(binding, "_stream", lambda stream=None: None)

    def go(i):
        current[0] = i
        return library
    return go


def test_vectors_of_another_device_are_refused(machine):
    cfg = rs.make_residual_norm_cfg(1, 4, 16, rs.RS_F32)
    library = machine(0)
    w = rs.make_residual_norm_weights(dict(pre_g=_There(0, 16)))
    rs.rs_residual_norm_fwd(cfg, w, _There(0, 1, 4, 16), None, _There(0, 1, 4, 16), None)
    assert library.calls == 1
    machine(1)
    with pytest.raises(AssertionError, match="device"):
        rs.rs_residual_norm_fwd(cfg, w, _There(1, 1, 4, 16), None, _There(1, 1, 4, 16), None)
    with pytest.raises(AssertionError, match="device"):
        rs.rs_residual_norm_fwd(cfg, w, _There(0, 1, 4, 16), None, _There(0, 1, 4, 16), None)
    assert library.calls == 1
    rs.rs_residual_norm_fwd(cfg, rs.make_residual_norm_weights({}), _There(1, 1, 4, 16), None, _There(1, 1, 4, 16), None)
    assert library.calls == 2
    machine(0)
    rs.rs_residual_norm_fwd(cfg, w, _There(0, 1, 4, 16), None, _There(0, 1, 4, 16), None)
    assert library.calls == 3
