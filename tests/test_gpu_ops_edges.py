"""The operators beside the layer where numbers are at the edge of their types and tensors at the edge of others, and the forms of the
products by name."""
import numpy as np
import pytest
import torch

import oracle.ops as ops
from paper_2510_26730_amd import binding as ef
from test_gpu_ops import TYPES, f64, stream

pytestmark = pytest.mark.gpu


# ---- rows to 8 bits ------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,first,last,pitch", [(4, 100, 100, 200, 200), (7, 100, 0, 110, 200), (1, 65, 16, 90, 90), (5, 96, 16, 112, 128),
                                                     (1200, 96, 32, 144, 144), (3, 1000, 16, 1020, 1040), (6, 64, 16, 80, 80), (9, 2056, 0, 2100, 2112)])
def test_codes_in_columns_of_a_wider_matrix(rows, K, first, last, pitch, dtype):
    """Codes and zeros go into the columns given, and nowhere else: not into the next row, not behind the last."""
    gen = torch.Generator().manual_seed(rows + K)
    x = torch.randn(rows, K, generator=gen).to(TYPES[dtype])
    room = torch.full((rows * pitch + 512,), 99, dtype=torch.int8, device="cuda")
    wide = room[:rows * pitch].view(rows, pitch)
    scales = torch.empty(rows, device="cuda")
    ef.ef_quant_rows(x.cuda(), wide[:, first:last], scales, stream=stream())
    torch.cuda.synchronize()
    q, s = ops.quant_rows(f64(x))
    padded = min((K + 63) // 64 * 64, last - first)
    assert np.array_equal(wide[:, first:first + K].cpu().numpy(), q) and np.array_equal(f64(scales), s)
    assert (wide[:, first + K:first + padded] == 0).all()
    assert (wide[:, :first] == 99).all() and (wide[:, first + padded:] == 99).all() and (room[rows * pitch:] == 99).all()
