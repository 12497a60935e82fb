"""Continuations of beams, and what rows keep, at the ends of what the calls accept."""

import numpy as np
import pytest

from test_gpu_beams import _stream, _xgm

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("source", [[1, 2, 0], [-1, 0, 0]])
def test_more_parts_than_a_launch_has_workgroups(source):
    xgm = _xgm()
    n = (1 << 24) + 7                                            # parts of a byte each, and of two
    x = torch.randint(0, 256, (3, n), dtype=torch.uint8, device="cuda")
    y = torch.randint(-99, 99, (2, 3, n // 2), dtype=torch.int16, device="cuda")
    used = torch.tensor([1, 0, 5], dtype=torch.int32, device="cuda")
    want = x.clone(), y.clone()
    for b, a in enumerate(source):
        if a >= 0:
            want[0][b] = x[a]
            if used[a] > 0:
                want[1][:, b] = y[:, a]
    on = torch.tensor(source, dtype=torch.int32, device="cuda")
    kept = xgm.RowSet(xgm.RowData(d_data=x.data_ptr(), row_stride=n, part_stride=1, part_bytes=1, n_outer=1, n_parts=n),
                      xgm.RowData(d_data=y.data_ptr(), row_stride=n // 2 * 2, outer_stride=n // 2 * 6, part_stride=2, part_bytes=2, n_outer=2, n_parts=n // 2,
                                  d_used=used.data_ptr(), used_bytes=2))
    xgm.reorder_rows(kept, on.data_ptr(), 3, _stream())
    torch.cuda.synchronize()
    assert torch.equal(x, want[0]) and torch.equal(y, want[1])
