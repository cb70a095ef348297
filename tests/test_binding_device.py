"""The calls on 8-bit matrices run on the current device: the binding refuses what lies on another one, in every argument, before
the library is called.  On the CPU, with tensors that only say where they lie."""
import types

import pytest
import torch

from paper_2607_22614_amd import dr

P = 1 << 20


class Somewhere:
    """A dense tensor's face: shape, type and device."""

    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, device=0):
        self.shape, self.dtype, self.device = shape, dtype, device

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.dtype.itemsize

    @property
    def nbytes(self):
        return self.numel() * self.element_size()

    def stride(self, i=None):
        steps = (self.shape[1], 1)
        return steps if i is None else steps[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P

    def get_device(self):
        return self.device


def _codes(rows, cols, device=0, scales=None):
    stride = -(-cols // 128) * 128
    return dr.QMatrix(Somewhere(rows, stride, dtype=torch.uint8, device=device),
                      Somewhere(-(-stride // 512), rows, 4, dtype=torch.uint8, device=device if scales is None else scales), rows, cols)


def _bytes(device):
    return Somewhere(64, dtype=torch.uint8, device=device)


# each call with its arguments' devices in turn
CALLS = {
    "dr_quantize": (3, lambda a, b, c: dr.dr_quantize(Somewhere(3, 200, device=a), _codes(3, 200, b), _codes(200, 3, c), stream=0)),
    "dr_qmatmul": (4, lambda a, b, c, w: dr.dr_qmatmul(_codes(3, 200, a), _codes(8, 200, b), Somewhere(3, 8, device=c), workspace=_bytes(w), stream=0)),
    "dr_qlinear": (4, lambda a, b, c, w: dr.dr_qlinear(Somewhere(3, 200, device=a), _codes(8, 200, b), Somewhere(3, 8, device=c), workspace=_bytes(w), stream=0)),
    "dr_qgated": (4, lambda a, b, c, w: dr.dr_qgated(Somewhere(3, 200, device=a), _codes(8, 200, b), Somewhere(3, 4, device=c), workspace=_bytes(w), stream=0)),
    "dr_qgated_save": (6, lambda a, b, c, d, e, w: dr.dr_qgated_save(_codes(3, 200, a), _codes(8, 200, b), _codes(3, 4, c), _codes(3, 4, d), _codes(3, 4, e),
                                                                     workspace=_bytes(w), stream=0)),
    "dr_gated_backward": (6, lambda a, b, c, d, e, f: dr.dr_gated_backward(Somewhere(3, 4, device=a), _codes(3, 4, b), _codes(3, 4, c), _codes(3, 8, d),
                                                                           _codes(8, 3, e), _codes(4, 3, f), stream=0)),
    "dr_qtranspose": (2, lambda a, b: dr.dr_qtranspose(_codes(3, 4, a), _codes(4, 3, b), stream=0)),
}


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("name", CALLS)
def test_every_argument(name, current, monkeypatch):
    count, call = CALLS[name]
    reached = []

    def library(*_):
        reached.append(name)
        return dr.DR_OK

    monkeypatch.setattr(dr, "_lib", types.SimpleNamespace(**{name: library, "dr_qmatrix_sizes": dr._lib.dr_qmatrix_sizes}))
    monkeypatch.setattr(dr, "_device", lambda: current)
    call(*[current] * count)
    assert reached == [name]
    for i in range(count):
        with pytest.raises(ValueError, match="current device"):
            call(*[1 - current if j == i else current for j in range(count)])
    assert reached == [name]


def test_codes_and_scales_lie_together():
    with pytest.raises(ValueError, match="device"):
        _codes(3, 200, 0, 1)
    assert _codes(3, 200, 1, 1).device == 1


@pytest.mark.parametrize("current", [0, 1])
def test_a_stream_of_another_device(current, monkeypatch):
    monkeypatch.setattr(dr, "_device", lambda: current)
    streams = [types.SimpleNamespace(device_index=i, cuda_stream=77 + i) for i in range(2)]
    assert dr._stream_on(current, streams[current], "here") == 77 + current
    with pytest.raises(ValueError, match="current device"):
        dr._stream_on(current, streams[1 - current], "here")
