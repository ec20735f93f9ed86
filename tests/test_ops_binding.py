"""What the binding hands to the entry points of the operators beside the layer, and what it refuses.  No GPU: the tensors are on the host and
say that they are on a device, and a stand-in takes the calls."""
import ctypes as C

import pytest
import torch

from paper_2510_26730_amd import binding as ef


class Device(torch.Tensor):
    """A tensor in host memory that counts as the first device's."""

    def get_device(self):
        return 0


def dev(t):
    return t.as_subclass(Device)


class Calls:
    """Takes the calls of the library; ef_quant_rows* write what the entry points may write."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            if name == "ef_quant_rows":
                x, kind, ldx, rows, K, codes, ldc, scales, s = args
                self.zero(codes, rows, K, ldc, ldc)
            elif name == "ef_quant_rows_within":
                x, kind, ldx, rows, K, codes, width, ldc, scales, s = args
                self.zero(codes, rows, K, width, ldc)
            return 1 << 20 if name.endswith("_work") else 0
        return call

    @staticmethod
    def zero(codes, rows, K, width, ldc):
        for r in range(rows):
            C.memset(codes + r * ldc, 0, min((K + 63) // 64 * 64, width))


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(ef, "lib", lambda: c)
    return c


@pytest.mark.parametrize("rows,first,last", [(4, 100, 200), (4, 0, 100), (1, 100, 200), (3, 30, 190), (2, 0, 200)])
def test_codes_in_columns_of_a_wider_matrix(calls, rows, first, last):
    """Nothing behind the columns is written, not in the next row and not behind the last one."""
    room = torch.full((rows * 200 + 256,), 99, dtype=torch.int8)
    codes = dev(room[:rows * 200].view(rows, 200)[:, first:last])
    ef.ef_quant_rows(dev(torch.zeros(rows, 100)), codes, dev(torch.zeros(rows)))
    assert len(calls.made) == 1
    wide = room[:rows * 200].view(rows, 200)
    assert (room[rows * 200:] == 99).all() and (wide[:, :first] == 99).all() and (wide[:, last:] == 99).all()
    assert (wide[:, first:first + 100] == 0).all()


def test_width_is_checked():
    refuse = lambda width, ldc: ef.lib().ef_quant_rows_within(4096, ef.EF_BF16, 64, 2, 64, 4096, width, ldc, 4096, None)  # noqa: E731
    for width, ldc in ((63, 64), (65, 64), (200, 128)):
        assert refuse(width, ldc) == ef.EF_EINVAL and "width" in ef.ef_last_error(None)
