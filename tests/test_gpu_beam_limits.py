"""Continuations of beams, and what rows keep, at the ends of what the calls accept.

Tolerances.  A sum y + (score - (top + log(weights / weight of top))), top the row's largest logit, is off by less than (18 + |y| + |score| + |top|) 2^-50 before it is
rounded to 32 bits.  In steps of 2^-52: a weight is off by 2 + |y| of itself, the weights together by 2 + |top| + 14 (the mean of top - y under the weights is at most
log 2^20 < 14) and by half a step for each of 39 additions at most, the largest one's own by 2 + |top|, the logarithm of at most 14 by 8: 46 + 2 |top|.  Three additions
round by half a step of their results: (42 + |y| + 2 |score| + 3 |top|) / 2.  Together 67 + |y| / 2 + |score| + 3.5 |top|, a fourth of which in steps of 2^-50."""

import time

import numpy as np
import pytest

from test_gpu_beams import Beams, _stream, _xgm

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


@pytest.mark.parametrize("parts", [1 << 21, 1 << 24])
def test_short_parts_take_what_their_bytes_take(parts):
    """Workgroups that each have a part of 4 bytes, or of 16, beside an array of long ones: not as long as if they had a long one."""
    xgm = _xgm()
    x = torch.randint(0, 99, (2, parts), dtype=torch.int32, device="cuda")
    y = torch.randint(0, 99, (2, parts // 4, 4), dtype=torch.int32, device="cuda")
    z = torch.randint(0, 99, (2, 1 << 26), dtype=torch.int32, device="cuda")
    kept = xgm.RowSet(xgm.RowData(d_data=x.data_ptr(), row_stride=4 * parts, part_stride=4, part_bytes=4, n_outer=1, n_parts=parts),
                      xgm.RowData(d_data=y.data_ptr(), row_stride=4 * parts, part_stride=16, part_bytes=16, n_outer=1, n_parts=parts // 4),
                      xgm.RowData(d_data=z.data_ptr(), row_stride=4 << 26, part_bytes=4 << 26, n_outer=1, n_parts=1))
    on = torch.tensor([-1, 0], dtype=torch.int32, device="cuda")
    begin = time.perf_counter()
    xgm.reorder_rows(kept, on.data_ptr(), 2, _stream())
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    assert torch.equal(x[0], x[1]) and torch.equal(y[0], y[1]) and torch.equal(z[0], z[1])
    assert took < 0.1 + parts * 30e-9          # (3 us a workgroup, of which a card has more than 100 at a time)


def test_a_lookup_of_the_most_rows():
    """2^24 rows of more columns than 256 threads take at once: a workgroup a row, and more of them than a launch may have.  69 GB."""
    xgm = _xgm()
    n, K, V = 1 << 24, 2064, 300
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("not as much memory")
    codes = torch.randint(0, 126, (V, K), dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-V // 128), -(-K // 128)), 0.25, device="cuda")
    ids = torch.randint(-1, V, (n,), dtype=torch.int32, device="cuda")
    out = torch.empty((n, K), dtype=torch.bfloat16, device="cuda")
    xgm.f8_embed(ids.data_ptr(), n, codes.data_ptr(), scales.data_ptr(), V, K, 0.5, out.data_ptr(), xgm.DTYPE_BF16, K, _stream())
    torch.cuda.synchronize()
    table = torch.cat([codes.view(torch.float8_e4m3fn).float() / 8, torch.zeros((1, K), device="cuda")]).bfloat16()      # (exact; -1 is the last one)
    for b in range(0, n, 1 << 19):
        assert torch.equal(out[b:b + (1 << 19)], table[ids[b:b + (1 << 19)].long()]), b
    del out
    torch.cuda.empty_cache()


def _bound(y, score, top):
    return (18 + abs(y) + abs(score) + abs(top)) * 2.0 ** -50


@pytest.mark.parametrize("score", [0.0, -3.0, 700.0])
@pytest.mark.parametrize("top", [1.0, 40.0, 1000.0, 30000.0])
def test_order_behind_a_token_that_has_all_the_weight(top, score):
    """Two rows alike but for their second token, which is worth 0 and `more`, down to what 64 bits do not tell apart beside the largest logit."""
    R, V = 60, 300
    b = Beams(R, 2, V, "f32", seed=1)
    x = b.logits
    x[:] = -torch.rand(V, device="cuda") - 1.0
    x[:, 7], x[:, 100] = top, 0.0
    more = 2.0 ** -np.arange(R)
    x[1::2, 100] = torch.from_numpy(more.astype(np.float32)).cuda() * min(0.5, top / 2)
    b.scores[:] = score
    rows, ids, sums = b.run(4)
    y = x[1::2, 100].double().cpu().numpy()
    told = 0
    for r in range(R):
        if y[r] / 2 > _bound(y[r], score, top) + _bound(0.0, score, top):      # (y itself raises the row's weight by less than half of it)
            assert ids[r, 2] == 100 and ids[r, 3] == 100 and (rows[r, 2:] == [2 * r + 1, 2 * r]).all(), (r, y[r])
            told += 1
    assert told >= 30


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0.0, 3.0, 300.0, 30000.0, -30000.0])
def test_sums_next_to_zero(top, dtype):
    """Scores as near to the logarithms of the rows' weights as 32 bits let them be: what is left of the second token's sum shows more of its bits."""
    R, V = 64, 9000
    b = Beams(R, 1, V, dtype, seed=3)
    x = b.logits
    x[:] = (x.float() * 0.5 + top).to(x.dtype)
    y = x.double().cpu().numpy().astype(np.longdouble)
    most = y.max(1, keepdims=True)
    lse = (most + np.log(np.exp(y - most).sum(1, keepdims=True)))[:, 0]
    order = np.argsort(-y.astype(np.float64), axis=1, kind="stable")[:, :3]
    b.scores[:] = (lse - y[np.arange(R), order[:, 1]]).astype(np.float32)
    rows, ids, sums = b.run(3)
    assert np.array_equal(ids, order)
    for k in range(3):
        of = y[np.arange(R), order[:, k]]
        want = of + (b.scores.astype(np.longdouble) - lse)
        tol = 2.0 ** -24 * np.abs(want) + _bound(of, b.scores, most[:, 0])
        assert (np.abs(sums[:, k] - want) <= tol).all(), (k, float((np.abs(sums[:, k] - want) / tol).max()))
