"""Continuations of beams under all rules on logits at once (histories with prompts, the three penalties, biases, masks shorter than the rows), against
their definitions.  Tolerances as in test_gpu_beams.py: rows and tokens the same, sums rounded once to 32 bits beside what 64 bits lose."""

import numpy as np
import pytest

import plain_beams
from test_gpu_logits import TYPES, Batch, _dev, _stream, _xgm

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _check(c, beams, n_out, search=None, ended=None):
    xgm = _xgm()
    requests = c.rows // beams
    scores = (-1 - 3 * np.random.default_rng(c.V).random(c.rows)).astype(np.float32)
    y = c.want()
    want = plain_beams.select(y, scores, ended, beams, n_out, False)
    out = [torch.full((requests, n_out), 99, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    search = search or xgm.BeamSearch(c.rows, c.V, _stream())
    on = [_dev(scores), None if ended is None else _dev(ended)]
    before = c.buf.clone()
    search.select(c.address(), TYPES[c.dtype][1], requests, beams, c.V, c.stride, c.rules, on[0].data_ptr(), 0 if ended is None else on[1].data_ptr(), n_out, False,
                  *(t.data_ptr() for t in out), _stream())
    torch.cuda.synchronize()
    rows, ids, sums = (t.cpu().numpy() for t in out)
    assert np.array_equal(rows, want[0]) and np.array_equal(ids, want[1])
    some = np.isfinite(want[2])
    size = np.where(np.isfinite(y), np.abs(y), 0).max()
    assert np.array_equal(sums[~some], want[2][~some])
    assert (np.abs(sums[some] - want[2][some]) <= 2.0 ** -24 * np.abs(want[2][some]) + (22 + 2 * size) * 2.0 ** -50).all()
    assert torch.equal(c.buf.view(torch.uint8), before.view(torch.uint8))      # nothing is written back


CASES = [dict(rows=2, V=31, dtype="bf16", history=8, bias=3), dict(rows=6, V=5000, dtype="f32", history=700, bias=40, mask="full"),
         dict(rows=8, V=8193, dtype="bf16", history=300, bias=9, mask="short", pad=3, offset=1), dict(rows=6, V=50001, dtype="f16", history=5000, bias=300, offset=5),
         dict(rows=4, V=20011, dtype="f32", history=64, prompt=False, pad=13), dict(rows=12, V=30011, dtype="bf16", bias=25, mask="full"),
         dict(rows=4, V=9000, dtype="bf16", history=9, bias=6000), dict(rows=64, V=1031, dtype="f32", history=50, bias=5, mask="full")]


@pytest.mark.parametrize("beams,n_out", [(1, 1), (2, 4), (2, 40)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c['rows']}x{c['V']}-{c['dtype']}")
def test_all_rules_at_once(case, beams, n_out):
    _check(Batch(**case, seed=case["V"]), beams, n_out)


def test_biases_that_open_and_close_tokens():
    """A bias of +inf counts as the largest finite number, -inf closes a token, NaN counts as -inf; the last of several of a token."""
    c = Batch(6, 9001, "f32", seed=3, history=20, bias=1)
    inf, nan = float("inf"), float("nan")
    c.bias = [[(8999, 60.0)], [(i, -inf) for i in range(9000)], [(5, inf), (8500, 3.0)], [(4, nan), (8193, 55.0), (8193, 50.0)], [(7, 1e30), (7, -1e30), (8, 40.0)],
              [(i, -inf) for i in range(9001)]]
    c.upload()
    for beams, n_out in ((1, 3), (2, 9), (3, 20), (6, 128)):
        _check(c, beams, n_out)


def test_a_search_goes_from_rules_to_none_and_back():
    search = _xgm().BeamSearch(12, 30011, _stream())
    ended = np.array([0, 0, 1, 0] * 3, np.int32)
    for k, how in enumerate([dict(history=60, bias=9), dict(), dict(mask="full"), dict(history=3000, bias=2, mask="short"), dict(bias=400)]):
        _check(Batch(12, 30011 - 977 * k, "bf16", seed=k, **how), 4, 8, search, ended)
