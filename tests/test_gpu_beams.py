"""Continuations of beams, and what rows keep, against their definitions; and the operators of a decode step with beams together.

Tolerances.  Rows and tokens: the same.  Sums: off by (4 + |y| + |score|) 2^-50 before they are rounded to 32 bits, so that they are
within 2^-24 of themselves and that.  What moves: bit for bit."""

import numpy as np
import pytest

import plain_beams as plain
import plain_logits

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": (torch.float32, 0), "bf16": (torch.bfloat16, 1), "f16": (torch.float16, 2)}


def _xgm():
    import paper_2411_15100_amd as xgm
    return xgm


def _stream():
    return int(torch.cuda.current_stream().cuda_stream)


def _at(t):
    return 0 if t is None else t.data_ptr()


class Beams:
    """A batch of beams.  mask: the share of tokens that each row allows (a list that rows go round), or None."""

    def __init__(self, requests, beams, V, dtype="f32", mask=None, seed=0, sigma=2.0, history=0, ended=False, pad=0, offset=0):
        rng = np.random.default_rng(seed)
        self.requests, self.beams, self.V, self.dtype = requests, beams, V, dtype
        self.rows = rows = requests * beams
        self.stride = V + pad
        t = TYPES[dtype][0]
        logits = torch.from_numpy((sigma * rng.standard_normal((rows, V))).astype(np.float32)).to(t)
        self.buf = torch.full((offset + rows * self.stride,), float("nan"), dtype=t)
        self.buf[offset:].view(rows, self.stride)[:, :V] = logits
        self.buf, self.offset = self.buf.cuda(), offset
        self.scores = (-5 - 2 * rng.random(rows)).astype(np.float32)
        self.ended = (rng.random(rows) < 0.25).astype(np.int32) * 9 if ended else None
        self.allowed = None if mask is None else rng.random((rows, V)) < np.resize(mask, rows)[:, None]
        self.history = None
        if history:
            n = rng.integers(0, history + 1, rows).astype(np.int32)
            self.history = dict(tokens=rng.integers(0, V, (rows, history)).astype(np.int32), n_tokens=n,
                                repetition=(1 + rng.random(rows)).astype(np.float32), presence=rng.random(rows).astype(np.float32))

    @property
    def logits(self):
        return self.buf[self.offset:].view(self.rows, self.stride)[:, :self.V]

    def want(self, n_out, placed):
        x = self.logits.float().cpu().numpy()
        y = np.stack([plain_logits.processed(x[b], b, None if self.allowed is None else self.allowed[b], **(self.history or {})) for b in range(self.rows)])
        return plain.select(y, self.scores, self.ended, self.beams, n_out, placed)

    def run(self, n_out, placed=False, search=None, in_place=False):
        xgm = _xgm()
        on = dict(mask=None if self.allowed is None else torch.from_numpy(plain_logits.pack(self.allowed)).cuda(),
                  scores=torch.from_numpy(self.scores).cuda(), ended=None if self.ended is None else torch.from_numpy(self.ended).cuda())
        rules = {}
        if self.allowed is not None:
            rules |= dict(d_bitmask=on["mask"].data_ptr(), v_mask=self.V)
        if self.history:
            h = {k: torch.from_numpy(v).cuda() for k, v in self.history.items()}
            rules |= dict(d_tokens=h["tokens"].data_ptr(), token_stride=h["tokens"].shape[1], d_n_tokens=h["n_tokens"].data_ptr(),
                          d_repetition=h["repetition"].data_ptr(), d_presence=h["presence"].data_ptr())
        search = search or xgm.BeamSearch(self.rows, self.V, _stream())
        ids, rows = (torch.full((self.requests * n_out + 4,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        sums = on["scores"] if in_place else torch.full((self.requests * n_out + 4,), 99.0, device="cuda")
        search.select(self.buf.data_ptr() + self.offset * self.buf.element_size(), TYPES[self.dtype][1], self.requests, self.beams, self.V, self.stride,
                      xgm.LogitRules(**rules) if rules else None, on["scores"].data_ptr(), _at(on["ended"]), n_out, placed, rows.data_ptr(), ids.data_ptr(),
                      sums.data_ptr(), _stream())
        torch.cuda.synchronize()
        n = self.requests * n_out
        for t in (rows, ids) + (() if in_place else (sums,)):
            assert bool((t[n:] == 99).all())
        return tuple(t[:n].view(self.requests, n_out).cpu().numpy() for t in (rows, ids, sums))

    def check(self, n_out, placed=False, **how):
        want, got = self.want(n_out, placed), self.run(n_out, placed, **how)
        assert np.array_equal(got[0], want[0]), np.argwhere(got[0] != want[0])[:3]
        assert np.array_equal(got[1], want[1]), np.argwhere(got[1] != want[1])[:3]
        some = np.isfinite(want[2])
        assert np.array_equal(got[2][~some], want[2][~some])
        size = 4 + 3 * float(self.logits.float().abs().max()) + np.abs(self.scores[np.isfinite(self.scores)]).max(initial=0.0)
        assert (np.abs(got[2][some] - want[2][some]) <= 2.0 ** -24 * np.abs(want[2][some]) + size * 2.0 ** -50).all()
        return got


SIZES = [(1, 1, 1), (1, 1, 7), (1, 4, 4096), (3, 2, 8191), (2, 5, 8192), (2, 3, 8193), (7, 3, 50001), (1, 64, 3000), (5, 8, 20000), (40, 4, 1000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("requests,beams,V", SIZES)
def test_continuations_are_those_of_the_definition(requests, beams, V, dtype):
    for n_out in sorted({1, beams, min(2 * beams, 128)}):
        b = Beams(requests, beams, V, dtype, seed=n_out, pad=V % 3, offset=V % 2, ended=beams == 8)
        b.check(n_out)
    b.check(beams, placed=True)
    b.check(beams, placed=True, in_place=True)


@pytest.mark.parametrize("n_out", [1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_any_number_of_continuations(dtype, n_out):
    Beams(3, 2, 9001, dtype, seed=n_out, mask=[1.0, 0.5, 0.01]).check(n_out)
    Beams(2, 6, 300, dtype, seed=n_out, ended=True).check(n_out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("requests,beams,V", [(4, 4, 5000), (2, 8, 50001), (9, 3, 333)])
def test_continuations_under_rules(requests, beams, V, dtype):
    for seed, mask in enumerate([[0.96], [0.0, 0.01, 0.9], [0.0], [2.0 / V], [1.0, 0.0]]):
        b = Beams(requests, beams, V, dtype, mask=mask, seed=seed, history=40 * (seed % 2), ended=seed > 1, pad=seed)
        b.check(beams, placed=True)
        b.check(2 * beams)


@pytest.mark.parametrize("beams,V,n_out", [(64, 128256, 128), (32, 151936, 64), (19, 77650, 38), (64, 300000, 128), (9, 40000, 20)])
def test_wide_searches(beams, V, n_out):
    b = Beams(1, beams, V, "bf16", seed=n_out, ended=beams == 32)
    b.check(n_out)
    scores = b.scores.copy()
    for live in ([0], [beams - 1], [beams // 2, 3], list(range(0, beams, 5))):          # a first step, and texts that are not there
        b.scores[:] = -np.inf
        b.scores[live] = scores[live]
        b.check(n_out)
    b.scores[:] = scores
    b.scores[beams // 3] += 40                                                          # one row has all of it
    b.check(n_out)


@pytest.mark.parametrize("n_out", [8, 9, 40, 128])
def test_masks_that_leave_stretches(n_out):
    V = 50001
    b = Beams(4, 3, V, "bf16", mask=[0.0], seed=n_out)
    for row, parts in enumerate([[(0, 1100)], [(8192 - 600, 8192 + 600)], [(0, 700), (4096, 4796)], [(V - 849, V)], [(16384, 24576)], [(8, 16), (4104, 4112)],
                                 [(100, 100 + n_out)], [(i, i + 3) for i in range(0, V, 61)], [(0, V)], [(20000, 22100)], [(0, 2048), (40000, 40001)], [(3, 4)]]):
        for first, last in parts:
            b.allowed[row, first:last] = True
    b.check(n_out)
    b.check(3, placed=True)


def test_rows_that_masks_leave_nothing_and_beams_without_a_text():
    b = Beams(6, 4, 10000, "bf16", mask=[0.5], seed=2)
    b.scores[4:8] = [0.0, -np.inf, -np.inf, -np.inf]            # a first step
    b.scores[8:12] = -np.inf                                    # a request that is not there
    b.scores[12:16] = [np.nan, np.inf, -3.0, -3.0]
    b.allowed[16:20] = False                                    # nothing is allowed
    b.allowed[20:23] = False
    b.allowed[23] = np.arange(10000) == 9999                    # one continuation of one row
    for n_out in (4, 9):
        got = b.check(n_out)
        assert (got[0][2] == -1).all() and (got[0][4] == -1).all() and (got[1][5][1:] == -1).all() and got[1][5][0] == 9999
        assert got[2][5][0] == b.scores[23]                     # (a token that is alone costs nothing)
    got = b.check(4, placed=True)
    assert got[1][5].tolist() == [-1, -1, -1, 9999]


def test_ended_rows_compete_with_their_scores():
    b = Beams(3, 4, 3000, "f32", seed=4)
    b.ended = np.zeros(12, np.int32)
    b.ended[[1, 4, 5, 6, 7, 8]] = 1
    b.scores[1], b.scores[8] = 5.0, -1e30
    got = b.check(4)
    assert got[0][0][0] == 1 and got[1][0][0] == -1
    assert sorted(got[0][1]) == [4, 5, 6, 7] and (got[1][1] == -1).all()
    assert 8 not in got[0][2]
    got = b.check(4, placed=True)
    assert got[0][1].tolist() == [4, 5, 6, 7]                   # all stay where they are


@pytest.mark.parametrize("n_out", [1, 8, 64, 128])
@pytest.mark.parametrize("V", [5, 700, 8192, 40000])
def test_equal_logits_go_by_row_and_id(V, n_out):
    """All logits equal: as many candidates as there are tokens at every bound, in a slice and in a request."""
    b = Beams(2, 4, V, "bf16", seed=0, sigma=0.0)
    b.scores[:] = -1.0
    got = b.check(n_out)
    k = min(n_out, V)
    assert (got[0][:, :k] == np.array([[0], [4]])).all() and (got[1][:, :k] == np.arange(k)).all()


def test_equal_beams_with_many_continuations():
    """64 beams alike: equal sums of all rows, more than a workgroup keeps at once."""
    b = Beams(2, 64, 20000, "bf16", seed=5, sigma=3.0)
    x = b.logits
    x[:] = x[0]
    b.scores[:] = -2.0
    for n_out in (64, 128):
        got = b.check(n_out)
        assert (got[1][:, :64] == got[1][0, 0]).all() and (got[0][0, :64] == np.arange(64)).all()
    assert (b.check(64, placed=True)[0] == np.arange(128).reshape(2, 64)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logits_that_are_not_finite_and_the_largest(dtype):
    b = Beams(2, 3, 9000, dtype, seed=6)
    x = b.logits
    most = torch.finfo(TYPES[dtype][0]).max
    x[0] = float("nan")
    x[1, :] = -float("inf")
    x[1, 8500] = -most
    x[2, ::7] = float("nan")
    x[3, 5] = float("inf") if dtype == "f32" else most
    x[4, 8999] = -0.0
    x[5, :] = 1e-3
    x[5, 100:200] = 0.0
    want, got = b.want(6, False), b.run(6)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_near_sums_are_ordered_as_in_64_bits():
    """Two rows whose best tokens are worth the same but for 1e-12 of it."""
    V = 3000
    b = Beams(64, 2, V, "f32", seed=7, sigma=1.0)
    x = b.logits.double().cpu().numpy()
    lse = np.log(np.exp(x).sum(1))
    want = np.empty(64, int)
    for r in range(64):      # the second row's score, as near as 32 bits let it be to a tie; the definition says who is ahead
        b.scores[2 * r + 1] = np.float32(b.scores[2 * r] + x[2 * r].max() - lse[2 * r] - x[2 * r + 1].max() + lse[2 * r + 1])
        worth = [np.float64(b.scores[2 * r + k]) + x[2 * r + k].max() - lse[2 * r + k] for k in (0, 1)]
        want[r] = 2 * r + (worth[1] > worth[0])
    got = b.check(1)
    assert np.array_equal(got[0][:, 0], want) and len(set(want % 2)) == 2


def test_a_search_is_used_again_with_other_sizes():
    xgm = _xgm()
    search = xgm.BeamSearch(64, 30000, _stream())
    for k, (requests, beams, V, n_out) in enumerate([(8, 8, 30000, 16), (1, 1, 5, 1), (16, 4, 20000, 128), (64, 1, 8193, 2), (8, 8, 30000, 8)]):
        Beams(requests, beams, V, "bf16", seed=k, mask=[0.9, 0.01]).check(n_out, search=search)


def test_the_widest_rows():
    Beams(1, 3, 1 << 20, "bf16", seed=1, sigma=1.0).check(6)


# ------------------------------------------------------------------------------------------------ what rows keep
def _moved(t, source, used=None, unit=1, rows_axis=1, length_axis=3):
    want = t.clone()
    for b, a in enumerate(source):
        if 0 <= a < len(source) and a != b:
            n = t.shape[length_axis] if used is None else max(0, min(int(used[a]), t.shape[length_axis] // unit)) * unit
            want.narrow(rows_axis, b, 1).narrow(length_axis, 0, n).copy_(t.narrow(rows_axis, a, 1).narrow(length_axis, 0, n))
    return want


SOURCES = {
    "stay": lambda B, rng: np.arange(B),
    "turn": lambda B, rng: (np.arange(B) + 1) % B,
    "swap": lambda B, rng: np.arange(B)[::-1],
    "one": lambda B, rng: np.full(B, B - 1),
    "any": lambda B, rng: rng.integers(0, B, B),
    "outside": lambda B, rng: np.where(np.arange(B) % 3 == 0, -1, np.where(np.arange(B) % 3 == 1, B + 5, rng.integers(0, B, B))),
}


@pytest.mark.parametrize("kind", sorted(SOURCES))
@pytest.mark.parametrize("layers,B,heads,length,dim,dtype", [
    (1, 1, 1, 5, 8, torch.float32), (2, 4, 3, 17, 64, torch.bfloat16), (3, 7, 1, 33, 1, torch.int32), (1, 128, 2, 100, 16, torch.bfloat16),
    (2, 5, 2, 9, 3, torch.int8), (1, 1024, 1, 40, 4, torch.int16), (1, 3, 1, 70000, 2, torch.float64), (2, 33, 2, 21, 20, torch.bfloat16),
    (1, 1000, 1, 3, 1, torch.int8)])
def test_rows_move_in_place_whatever_goes_where(layers, B, heads, length, dim, dtype, kind):
    xgm = _xgm()
    rng = np.random.default_rng(B)
    source = SOURCES[kind](B, rng).astype(np.int32)
    t = torch.from_numpy(rng.integers(-128, 128, (layers, B, heads, length, dim)).astype(np.int8)).to(dtype).cuda()
    e = t.element_size()
    on = torch.from_numpy(source).cuda()
    for lengths in (None, np.full(B, length), rng.integers(0, length + 1, B), np.where(np.arange(B) % 2, -3, length + 9)):
        x = t.clone()
        used = None if lengths is None else torch.from_numpy(lengths.astype(np.int32)).cuda()
        data = xgm.RowData(d_data=x.data_ptr(), row_stride=x.stride(1) * e, outer_stride=x.stride(0) * e, part_stride=x.stride(2) * e,
                           part_bytes=length * dim * e, d_used=_at(used), used_bytes=dim * e, n_outer=layers, n_parts=heads)
        xgm.reorder_rows(xgm.RowSet(data), on.data_ptr(), B, _stream())
        torch.cuda.synchronize()
        assert torch.equal(x, _moved(t, source, lengths)), lengths


def test_several_arrays_move_at_once_with_strides_and_odd_addresses():
    xgm = _xgm()
    B, rng = 11, np.random.default_rng(3)
    source = rng.integers(0, B, B).astype(np.int32)
    on, used = torch.from_numpy(source).cuda(), torch.from_numpy(rng.integers(0, 50, B).astype(np.int32)).cuda()
    text = torch.from_numpy(rng.integers(0, 99, (B, 64)).astype(np.int32)).cuda()
    flag = torch.from_numpy(rng.integers(0, 99, 3 * B + 1).astype(np.uint8)).cuda()          # every third byte, from the second on
    heads_last = torch.from_numpy(rng.standard_normal((2, B, 50, 3, 6)).astype(np.float32)).cuda()      # [outer, row, position, head, dim]
    score = torch.from_numpy(rng.standard_normal(B)).cuda()
    before = [t.clone() for t in (text, flag, heads_last, score)]
    xgm.reorder_rows(xgm.RowSet(
        xgm.RowData(d_data=text.data_ptr(), row_stride=256, part_bytes=200, n_outer=1, n_parts=1, d_used=used.data_ptr(), used_bytes=4),
        xgm.RowData(d_data=flag.data_ptr() + 1, row_stride=3, part_bytes=1, n_outer=1, n_parts=1),
        xgm.RowData(d_data=heads_last.data_ptr(), row_stride=50 * 72, outer_stride=B * 50 * 72, part_bytes=50 * 72, n_outer=2, n_parts=1,
                    d_used=used.data_ptr(), used_bytes=72),
        xgm.RowData(d_data=score.data_ptr(), row_stride=8, part_bytes=8, n_outer=1, n_parts=1)), on.data_ptr(), B, _stream())
    torch.cuda.synchronize()
    want = [t.clone() for t in before]
    for b, a in enumerate(source):
        n = int(used[a])
        want[0][b, :n] = before[0][a, :n]
        want[1][1 + 3 * b] = before[1][1 + 3 * a]
        want[2][:, b, :n] = before[2][:, a, :n]
        want[3][b] = before[3][a]
    for g, w in zip((text, flag, heads_last, score), want):
        assert torch.equal(g, w)


def test_lengths_at_their_ends_and_units_that_do_not_divide_a_part():
    xgm = _xgm()
    B, part = 6, 100
    for unit in (1, 3, 7, 100, 160, 2 ** 40):
        for value in (0, -1, -2 ** 31, 1, 13, 2 ** 31 - 1):
            t = torch.randint(0, 256, (B, 2, part), dtype=torch.uint8, device="cuda")
            want = t.clone()
            n = max(0, min(part, value * unit))
            want[:, :, :n] = t[[1, 2, 3, 4, 5, 0], :, :n]
            on, used = torch.tensor([1, 2, 3, 4, 5, 0], dtype=torch.int32, device="cuda"), torch.full((B,), value, dtype=torch.int32, device="cuda")
            xgm.reorder_rows(xgm.RowSet(xgm.RowData(d_data=t.data_ptr(), row_stride=2 * part, part_bytes=part, part_stride=part, n_outer=1, n_parts=2,
                                                    d_used=used.data_ptr(), used_bytes=unit)), on.data_ptr(), B, _stream())
            torch.cuda.synchronize()
            assert torch.equal(t, want), (unit, value)


def test_rows_beyond_2_to_the_31_bytes():
    xgm = _xgm()
    t = torch.zeros((3, 1 << 30), dtype=torch.int32, device="cuda")      # 4 GiB a row
    t[1, -5:] = 7
    t[1, 12345] = 9
    on = torch.tensor([1, 2, -1], dtype=torch.int32, device="cuda")
    xgm.reorder_rows(xgm.RowSet(xgm.RowData(d_data=t.data_ptr(), row_stride=4 << 30, part_bytes=4 << 30, n_outer=1, n_parts=1)), on.data_ptr(), 3, _stream())
    torch.cuda.synchronize()
    assert bool((t[0, -5:] == 7).all()) and int(t[0, 12345]) == 9 and int(t[0].sum()) == 44 and not bool(t[1:].any())


# ------------------------------------------------------------------------------------------------ together, streams, graphs
class Step:
    """A decode step with beams: lookup, (no model), projection in 8 bits, continuations, and what the rows keep."""

    def __init__(self, requests, beams, V, K, length, seed=0):
        xgm = _xgm()
        self.requests, self.beams, self.V, self.K, self.length = requests, beams, V, K, length
        self.rows = rows = requests * beams
        g = torch.Generator(device="cuda").manual_seed(seed)
        codes = torch.randint(0, 256, (V, K), generator=g, device="cuda", dtype=torch.uint8)
        codes[codes & 127 == 127] = 0
        self.codes, self.scales = codes, 0.002 * torch.rand((plain.blocks(V), plain.blocks(K)), generator=g, device="cuda")
        self.hidden = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
        self.work = torch.empty(xgm.f8_work_bytes(rows, K), dtype=torch.uint8, device="cuda")
        self.logits = torch.empty((rows, V), dtype=torch.bfloat16, device="cuda")
        self.mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, xgm.bitmask_words(V)), generator=g, device="cuda", dtype=torch.int32)
        self.cache = torch.zeros((2, rows, 2, length, 8), dtype=torch.bfloat16, device="cuda")
        self.text = torch.zeros((rows, length), dtype=torch.int32, device="cuda")
        self.n = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.ids = torch.arange(rows, dtype=torch.int32, device="cuda") // beams
        self.from_rows = torch.empty(rows, dtype=torch.int32, device="cuda")
        self.scores = torch.full((rows,), -float("inf"), device="cuda")
        self.scores[::beams] = 0.0
        self.search = xgm.BeamSearch(rows, V, _stream())
        self.rules = xgm.LogitRules(d_bitmask=self.mask.data_ptr(), v_mask=V)
        self.kept = xgm.RowSet(
            xgm.RowData(d_data=self.cache.data_ptr(), row_stride=2 * length * 16, outer_stride=rows * 2 * length * 16, n_outer=2, part_stride=length * 16, n_parts=2,
                        part_bytes=length * 16, d_used=self.n.data_ptr(), used_bytes=16),
            xgm.RowData(d_data=self.text.data_ptr(), row_stride=4 * length, part_bytes=4 * length, n_outer=1, n_parts=1, d_used=self.n.data_ptr(), used_bytes=4))
        self.lengths = xgm.RowSet(xgm.RowData(d_data=self.n.data_ptr(), row_stride=4, part_bytes=4, n_outer=1, n_parts=1))

    def state(self):
        return [self.hidden, self.logits, self.cache, self.text, self.n, self.ids, self.from_rows, self.scores]

    def __call__(self):
        xgm = _xgm()
        rows, V, K = self.rows, self.V, self.K
        xgm.f8_embed(self.ids.data_ptr(), rows, self.codes.data_ptr(), self.scales.data_ptr(), V, K, 3.0, self.hidden.data_ptr(), 1, K, _stream())
        xgm.f8_logits(self.hidden.data_ptr(), 1, 0, rows, K, K, self.codes.data_ptr(), self.scales.data_ptr(), V, self.logits.data_ptr(), 1, V,
                      self.mask.data_ptr(), self.work.data_ptr(), _stream())
        self.search.select(self.logits.data_ptr(), 1, self.requests, self.beams, V, V, self.rules, self.scores.data_ptr(), 0, self.beams, True,
                           self.from_rows.data_ptr(), self.ids.data_ptr(), self.scores.data_ptr(), _stream())
        xgm.reorder_rows(self.kept, self.from_rows.data_ptr(), rows, _stream())
        xgm.reorder_rows(self.lengths, self.from_rows.data_ptr(), rows, _stream())
        at = self.n.long()[:, None]
        self.text.scatter_(1, at, self.ids[:, None])
        self.cache.scatter_(3, at[None, :, None, :, None].expand(2, rows, 2, 1, 8), self.hidden[None, :, None, None, :8].expand(2, rows, 2, 1, 8).contiguous())
        self.n += 1


def test_a_decode_step_with_beams_follows_the_definition():
    s = Step(3, 4, 700, 256, 16)
    table = plain.e4m3()
    w = s.codes.cpu().numpy()
    ws = s.scales_np = s.scales.double().cpu().numpy()
    wide = table[w] * np.repeat(np.repeat(ws, 128, 0)[:700], 128, 1)
    texts = [[] for _ in range(12)]
    ids = s.ids.cpu().numpy()
    for step in range(10):
        scores = s.scores.cpu().numpy()
        s()
        torch.cuda.synchronize()
        hidden = torch.from_numpy(wide[ids] * 3.0).bfloat16()
        assert torch.equal(s.hidden.cpu(), hidden)
        want, size = plain.project(*plain.quantized(hidden.double().numpy()), w, ws)
        allowed = plain_logits.unpack(s.mask.cpu().numpy(), 700)
        got = s.logits.double().cpu().numpy()
        assert np.array_equal(got > -np.inf, allowed)
        tol = 2.0 ** -8 * np.abs(want) + (2 * np.sqrt(256) * 2.0 ** -23 + 3 * 2.0 ** -24) * size
        assert (np.abs(got - want)[allowed] <= tol[allowed]).all()
        rows, tokens, sums = plain.select(got.astype(np.float32), scores, None, 4, 4, True)
        assert np.array_equal(s.from_rows.cpu().numpy(), rows.ravel()) and np.array_equal(s.ids.cpu().numpy(), tokens.ravel())
        assert np.allclose(s.scores.cpu().numpy(), sums.ravel(), rtol=2.0 ** -23, atol=0)
        ids = tokens.ravel()
        texts = [texts[a] + [int(v)] for a, v in zip(rows.ravel(), ids)]
        text, n = s.text.cpu().numpy(), s.n.cpu().numpy()
        assert (n == step + 1).all() and [text[b, :n[b]].tolist() for b in range(12)] == texts


def test_the_step_replays_from_a_graph_and_runs_on_another_stream():
    s = Step(4, 8, 20000, 512, 40, seed=1)
    start = [t.clone() for t in s.state()]

    def back():
        for t, v in zip(s.state(), start):
            t.copy_(v)
        torch.cuda.synchronize()

    s()
    torch.cuda.synchronize()
    back()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s()
    back()
    wants = []
    for _ in range(5):
        s()
        torch.cuda.synchronize()
        wants.append([t.clone() for t in s.state()])
    back()
    for turn in range(5):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(wants[turn], s.state())), turn
        torch.randn(1000, device="cuda").sum().item()                   # (the program's own work between replays)
    back()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for turn in range(5):
            s()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(wants[turn], s.state())), turn


def test_two_searches_run_at_once():
    a, b = Beams(4, 4, 60000, "bf16", seed=1), Beams(8, 2, 60000, "f32", seed=2)
    want = a.want(8, False), b.want(8, False)
    xgm = _xgm()
    searches = [xgm.BeamSearch(16, 60000, _stream()) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for turn in range(6):
        for x, search, stream in zip((a, b), searches, streams):
            rows, ids = (torch.zeros((x.requests, 8), dtype=torch.int32, device="cuda") for _ in range(2))
            sums, scores = torch.zeros((x.requests, 8), device="cuda"), torch.from_numpy(x.scores).cuda()
            torch.cuda.synchronize()
            search.select(x.buf.data_ptr(), TYPES[x.dtype][1], x.requests, x.beams, x.V, x.stride, None, scores.data_ptr(), 0, 8, False, rows.data_ptr(),
                          ids.data_ptr(), sums.data_ptr(), int(stream.cuda_stream))
            outs.append((rows, ids, sums, scores, x is b))
    torch.cuda.synchronize()
    for rows, ids, _, _, which in outs:
        assert np.array_equal(rows.cpu().numpy(), want[which][0]) and np.array_equal(ids.cpu().numpy(), want[which][1])


def test_beams_of_a_grammar_fork_and_accept():
    """Masks, continuations, states: every text that is left is one that its grammar accepts."""
    import synth_inputs as si
    from paper_2411_15100_amd import workloads as wl
    xgm = _xgm()
    vocab = si.make_vocab("bpe", 4096, 0)
    cache = xgm.Cache(xgm.Grammar(si.JSON_GRAMMAR, "root"), wl.make_xgm_vocab(vocab))
    requests, beams, V, steps = 3, 4, 4096, 24
    rows = requests * beams
    states = xgm.DeviceBatch([xgm.Matcher(cache=cache) for _ in range(rows)], history=1, stream=_stream())
    search = xgm.BeamSearch(rows, V, _stream())
    mask = torch.zeros((rows, xgm.bitmask_words(V)), dtype=torch.int32, device="cuda")
    rules = xgm.LogitRules(d_bitmask=mask.data_ptr(), v_mask=V)
    scores = torch.full((rows,), -float("inf"), device="cuda")
    scores[::beams] = 0.0
    ended = torch.zeros(rows, dtype=torch.int32, device="cuda")
    stops = torch.zeros(V, dtype=torch.bool, device="cuda")
    stops[torch.from_numpy(np.asarray(vocab.stop_ids, dtype=np.int64)).cuda()] = True
    parents, ids = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    texts = [[] for _ in range(rows)]
    g = torch.Generator(device="cuda").manual_seed(0)
    for _ in range(steps):
        states.fill_next_token_bitmask(mask.data_ptr(), _stream())
        logits = 2 * torch.randn((rows, V), generator=g, device="cuda")
        logits[:, stops] += 4
        search.select(logits.data_ptr(), 0, requests, beams, V, V, rules, scores.data_ptr(), ended.data_ptr(), beams, True, parents.data_ptr(), ids.data_ptr(),
                      scores.data_ptr(), _stream())
        states.fork(parents.data_ptr(), _stream())
        assert not states.status(_stream()).any()
        states.accept_tokens(ids.data_ptr(), _stream())
        assert not states.status(_stream()).any()
        ended = ended[parents.clamp(min=0).long()] | (stops[ids.clamp(min=0).long()] & (ids >= 0)).int()
        texts = [(texts[a] + ([v] if v >= 0 else [])) if a >= 0 else [] for a, v in zip(parents.tolist(), ids.tolist())]
    assert (scores > -np.inf).sum() > requests
    for b, text in enumerate(texts):
        m = xgm.Matcher(cache=cache)
        assert all(m.try_accept_token(t) == 0 for t in text)
        assert bool(ended[b]) == m.is_terminated() or not text
