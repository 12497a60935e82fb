"""Sums of the projection with a matrix in 8 bits where neighbouring products differ much.

Tolerances.  Logits in 32 bits and f16, of any batch: sums in 32 bits, as in test_gpu_f8.py, and half a step of the type.  Logits in bf16 of more than 64 rows
may come from the instructions for 8 bits (with more columns than LDS holds for 32 rows they do): of each group of 8 neighbouring columns, what the products have below 2^-13 of the largest one's power of two is cut off.
The largest loses nothing, the 7 others less than 2^-13 of it each: 7 * 2^-13 of the sum of the groups' largest, whatever the signs."""

import numpy as np
import pytest

import plain_beams as plain
import plain_logits
from test_gpu_f8 import TYPES, Projection, _np, tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _tops(p):
    """Sums over groups of 8 columns of the largest product of each logit."""
    table, K = plain.e4m3(), p.K
    h = np.abs(table[p.eight[0]] * np.repeat(p.eight[1], 128, 1)[:, :K])
    w = np.abs(table[p.codes.cpu().numpy()] * np.repeat(np.repeat(p.scales.double().cpu().numpy(), 128, 0)[:p.V], 128, 1)[:, :K])
    return sum((h[:, None, k:k + 8] * w[None, :, k:k + 8]).max(2) for k in range(0, K, 8))


def _check(p, out, with_work=True):
    want, size = p.want()
    got = _np(p.run(out, with_work=with_work))
    tol = tolerance(want, size, p.K, out)
    if out == "bf16" and p.B > 64:
        tol = tol + 7 * 2.0 ** -13 * _tops(p)
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


def _states(p, values):
    """Gives the projection these hidden states, which 8 bits hold (the largest of a block is 256: its scale is 1)."""
    table = plain.e4m3()
    codes = np.array([int(np.flatnonzero(table == v)[0]) for v in np.unique(values)], np.uint8)[np.searchsorted(np.unique(values), values)]
    scales = np.ones((p.B, plain.blocks(p.K)))
    p.eight = codes, scales
    if p.dtype == "f8":
        p.hidden, p.hidden_scales = torch.from_numpy(codes).cuda(), torch.ones(scales.shape, device="cuda")
    else:
        p.hidden = torch.from_numpy(values).to(TYPES[p.dtype][0]).cuda()


@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("dtype", ["f8", "f16"])
@pytest.mark.parametrize("B,K,V", [(40, 256, 300), (65, 5120, 129), (70, 512, 200), (128, 4608, 300), (130, 4624, 333), (300, 6144, 200)])
def test_products_beside_one_that_is_8192_times_as_large(B, K, V, dtype, out):
    rng = np.random.default_rng(B + K)
    large = (np.arange(0, K, 8) + rng.integers(0, 8, K // 8))
    p = Projection(B, K, V, dtype, whole=True, seed=B)
    h, w = np.full((B, K), 1.875), np.full((V, K), 3.75)         # 7.03 each: just below 2^16 / 8192
    h[:, large], w[:, large] = 256.0, 256.0
    h *= rng.choice([-1.0, 1.0], (B, 1))
    w[::3] *= -1
    _states(p, h)
    p.codes = torch.from_numpy(np.where(np.abs(w) == 256.0, 120, 71).astype(np.uint8) | np.where(w < 0, 128, 0).astype(np.uint8)).cuda()
    assert np.array_equal(plain.e4m3()[p.codes.cpu().numpy()], w)
    p.scales[:] = 2.0 ** -10
    _check(p, out)


@pytest.mark.parametrize("out", ["f16", "bf16"])
@pytest.mark.parametrize("signs", ["all alike", "any"])
@pytest.mark.parametrize("B,K,V", [(65, 8192, 100), (128, 4624, 515), (200, 640, 129), (300, 5120, 300)])
def test_sums_of_products_of_all_sizes(B, K, V, signs, out):
    p = Projection(B, K, V, "f8", seed=K)
    if signs == "all alike":
        p.codes &= 127
        p.hidden &= 127
        p.eight = p.eight[0] & 127, p.eight[1]
    p.scales *= 2.0 ** -8
    _check(p, out)


@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,K,V", [(70, 4624, 601), (130, 4624, 1100), (300, 5120, 129)])
def test_sums_of_many_rows_under_masks(B, K, V, out):
    p = Projection(B, K, V, "f16", seed=V)
    p.scales *= 2.0 ** -6
    want, size = p.want()
    tol = tolerance(want, size, K, out) + (7 * 2.0 ** -13 * _tops(p) if out == "bf16" else 0.0)
    for share in (0.0, 0.002, 0.6, 1.0):
        allowed = np.random.default_rng(B).random((B, V)) < share
        allowed[B // 2] = False
        allowed[B - 1, V - 1] = True
        got = _np(p.run(out, mask=torch.from_numpy(plain_logits.pack(allowed)).cuda(), stride=V + B % 4, offset=B % 3))
        assert (got[~allowed] == -np.inf).all() and (np.abs(got - want) <= tol)[allowed].all(), share


@pytest.mark.parametrize("B", [65, 128, 200])
def test_a_row_is_the_same_in_a_batch_of_any_size(B):
    """f16: sums of 24 bits whatever the batch; a row's neighbours change the order of blocks, no more."""
    p = Projection(B, 4864, 300, "f16", seed=5)
    p.scales *= 2.0 ** -6
    many = p.run("f16").double()
    p.B, few = 16, None
    p.hidden = p.hidden[:16].contiguous()
    few = p.run("f16").double()
    size = torch.from_numpy(plain.project(p.eight[0][:16], p.eight[1][:16], p.codes.cpu().numpy(), p.scales.double().cpu().numpy())[1])
    tol = tolerance(0.0, _np(size), 4864, "f16")
    assert (np.abs(_np(many[:16] - few)) <= 2 * tol + torch.finfo(torch.float16).eps * np.abs(_np(few))).all()
    assert float((many[:16] != few).double().mean()) < 0.01


@pytest.mark.parametrize("B,V,stride", [(200, 40000, (1 << 31) // 200 // 4 * 4 + 4096), (1100, 2000, 2000)])
def test_logits_beyond_2_to_the_31_bytes_are_rounded_once(B, V, stride):
    """Whole numbers, so that every sum is exact in 32 bits, and its products in the cut ones."""
    p = Projection(B, 128, V, "bf16", whole=True, seed=2)
    got = p.run("bf16", stride=stride)
    want = torch.from_numpy(p.want()[0]).to(torch.float32)        # (exact)
    assert torch.equal(got.cpu(), want.to(torch.bfloat16))
