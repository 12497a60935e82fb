"""The operators around the mask (4-bit output projection, rules on logits, drawing a token) against their definitions in
64 bits.

Tolerances.  Projection: the result is rounded once to its type (eps / 2 of the value) after sums in 32 bits; with codes
shifted by 16 or 8 the terms add up to at most S = sum |hidden| * 32 * scale, every addition rounds by at most 2^-24 of S,
and K such roundings of random signs stay within 2 * sqrt(K) * 2^-24 * S.  Where hidden states are small whole numbers and scales
powers of two all sums are exact, and so must the result be.  Rules: 64 bits rounded to 32 and then to the type, the same
bits.  Draws: the same ids (the random numbers lie in the middle of a token's stretch); logprobs: 64 bits rounded to 32."""

import numpy as np
import pytest

import plain_logits as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": (torch.float32, 0), "bf16": (torch.bfloat16, 1), "f16": (torch.float16, 2)}


def _xgm():
    import paper_2411_15100_amd as xgm
    return xgm


def _stream():
    return int(torch.cuda.current_stream().cuda_stream)


def _dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _at(t):
    return 0 if t is None else t.data_ptr()


def _np(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ projection
class Projection:
    def __init__(self, B, K, V, group, dtype, zeros=False, whole=False, seed=0, pad=0):
        g = torch.Generator().manual_seed(seed)
        t = TYPES[dtype][0]
        self.B, self.K, self.V, self.group, self.dtype, self.pad = B, K, V, group, dtype, pad
        h = torch.randint(-3, 4, (B, K + pad), generator=g).float() if whole else torch.randn((B, K + pad), generator=g)
        s = 2.0 ** torch.randint(-3, 1, (V, K // group), generator=g).float() if whole else 0.01 * torch.exp(0.5 * torch.randn((V, K // group), generator=g))
        self.hidden, self.scales = h.to(t).cuda(), s.to(t).cuda()
        self.codes = torch.randint(0, 256, (V, K // 2), generator=g, dtype=torch.uint8).cuda()
        self.zeros = torch.randint(0, 16, (V, K // group), generator=g, dtype=torch.uint8).cuda() if zeros else None

    def want(self):
        return plain.project(_np(self.hidden)[:, :self.K], self.codes.cpu().numpy(), _np(self.scales),
                             None if self.zeros is None else self.zeros.cpu().numpy(), self.group)

    def run(self, out="f32", mask=None, stride=None, offset=0):
        xgm = _xgm()
        stride = stride or self.V
        buf = torch.full((offset + self.B * stride + 8,), 7.0, dtype=TYPES[out][0], device="cuda")
        xgm.q4_logits(self.hidden.data_ptr(), TYPES[self.dtype][1], self.B, self.K, self.K + self.pad, self.codes.data_ptr(), self.scales.data_ptr(),
                      _at(self.zeros), self.V, self.group, buf.data_ptr() + offset * buf.element_size(), TYPES[out][1], stride, _at(mask), _stream())
        torch.cuda.synchronize()
        assert bool((buf[:offset] == 7).all()) and bool((buf[offset + self.B * stride:] == 7).all())
        rows = buf[offset:offset + self.B * stride].view(self.B, stride)
        assert bool((rows[:, self.V:] == 7).all())      # nothing but the logits is written
        return rows[:, :self.V]


SHAPES = [(1, 32, 1, 32), (1, 64, 17, 32), (3, 96, 33, 96), (2, 160, 100, 32), (1, 1024, 257, 128), (5, 288, 130, 32), (4, 4096, 515, 128),
          (16, 2080, 97, 32), (17, 512, 64, 64), (24, 1344, 201, 64), (33, 640, 333, 128), (64, 2048, 129, 256), (100, 384, 1000, 64),
          (128, 4096, 300, 128), (130, 736, 259, 32), (257, 256, 65, 64), (2, 8192, 70, 128), (7, 12288, 40, 64), (40, 16384, 36, 512)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,K,V,group", SHAPES)
def test_projection_is_exact_on_small_whole_numbers(B, K, V, group, dtype):
    for zeros in (False, True):
        p = Projection(B, K, V, group, dtype, zeros, whole=True, seed=B + V)
        want, _ = p.want()
        assert np.array_equal(_np(p.run()), want), (zeros,)


@pytest.mark.parametrize("out", ["f32", "same"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,K,V,group", SHAPES)
def test_projection_of_real_numbers(B, K, V, group, dtype, out):
    out = dtype if out == "same" else out
    p = Projection(B, K, V, group, dtype, zeros=(B + K // 32) % 2 == 0, seed=K + V, pad=8 * (B % 3))
    want, size = p.want()
    got = _np(p.run(out, stride=V + B % 5, offset=B % 4))
    tol = torch.finfo(TYPES[out][0]).eps / 2 * np.abs(want) + 2 * np.sqrt(K) * 2.0 ** -24 * size
    if out == "f16":
        tol += 2.0 ** -25
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("B,K,V,group", [(1, 65536, 40, 32), (1, 65536, 40, 128), (1, 65536, 33, 64), (2, 32768, 20, 32), (3, 24576, 50, 96), (9, 8192, 70, 32),
                                         (5, 12800, 30, 256), (17, 4096, 40, 32), (20, 3200, 50, 32)])
def test_projection_of_columns_around_what_fits_lds(B, K, V, group):
    p = Projection(B, K, V, group, "bf16", zeros=True, whole=True, seed=B)
    want, _ = p.want()
    assert np.array_equal(_np(p.run()), want)


@pytest.mark.parametrize("B,K,V,group", [(1, 1024, 5000, 128), (4, 2080, 3001, 32), (20, 512, 2050, 64), (70, 384, 777, 32), (130, 256, 600, 128)])
def test_projection_under_masks(B, K, V, group):
    rng = np.random.default_rng(B)
    p = Projection(B, K, V, group, "bf16", zeros=True, whole=True, seed=3)
    want, _ = p.want()
    allowed = rng.random((B, V)) < rng.choice([0.0, 0.003, 0.5, 0.97], (B, 1))
    for kind in ("random", "none", "one", "all", "a stretch"):
        if kind != "random":
            allowed[:] = kind == "all"
        if kind == "one":
            allowed[B // 2, V - 1] = True
        if kind == "a stretch":
            allowed[0, V // 3:V // 3 + 40] = True
        got = _np(p.run(mask=_dev(plain.pack(allowed)), offset=1))
        assert np.array_equal(got, np.where(allowed, want, -np.inf)), kind


@pytest.mark.parametrize("B,K,V,group", [(1, 256, 1000, 128), (5, 128, 2049, 32), (20, 512, 2050, 64), (70, 384, 777, 32), (130, 256, 600, 128)])
def test_projection_under_masks_of_another_vocabulary(B, K, V, group):
    """A matrix that is padded behind the masks' tokens, and one that is a part of a larger one."""
    xgm = _xgm()
    rng = np.random.default_rng(V)
    p = Projection(B, K, V, group, "bf16", whole=True, seed=4)
    want, _ = p.want()
    for v_mask, first in ((V - 1, 0), (V - 33, 0), (V - V // 3, 0), (1, 0), (V + 95, 0), (V + 3000, 0), (V + 3000, 64), (V + 640, 640)):
        allowed = rng.random((B, v_mask)) < rng.choice([0.002, 0.5, 0.97], (B, 1))
        words = plain.pack(allowed)
        if v_mask % 32:
            words[:, -1] |= np.int32(-1 << v_mask % 32)         # bits behind the vocabulary say nothing
        d_mask = _dev(words)
        out = torch.full((B, V + 3), 7.0, device="cuda")
        xgm.q4_logits(p.hidden.data_ptr(), 1, B, K, K, p.codes.data_ptr(), p.scales.data_ptr(), 0, V, group, out.data_ptr(), 0, V + 3,
                      d_mask.data_ptr() + first // 32 * 4, _stream(), v_mask=v_mask)
        got = _np(out)
        here = np.zeros((B, V), bool)
        here[:, :v_mask - first] = allowed[:, first:first + V]
        assert np.array_equal(got[:, :V], np.where(here, want, -np.inf)) and (got[:, V:] == 7).all(), (v_mask, first)


@pytest.mark.parametrize("B,K,V,group", [(4, 16384, 700, 128), (3, 16384, 5000, 32), (1, 32768, 333, 128), (1, 40960, 200, 64), (1, 65536, 130, 65536)])
def test_projection_of_many_columns_under_masks_that_leave_workgroups_nothing(B, K, V, group):
    """More steps than a workgroup has waves, and no row of the matrix to share them out over."""
    p = Projection(B, K, V, group, "bf16", whole=True, seed=7)
    want, _ = p.want()
    rng = np.random.default_rng(V)
    for share in (0.0, 0.004, 0.3):
        allowed = rng.random((B, V)) < share
        allowed[:, V // 2:V // 2 + 64] = False
        assert np.array_equal(_np(p.run(mask=_dev(plain.pack(allowed)))), np.where(allowed, want, -np.inf)), share


# (a workgroup of the projection of many rows takes ceil(tiles / 256) tiles of 16 rows of the matrix: 2, 5, 17, 19, 38 and 40)
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,K,V,group", [(40, 64, 5000, 64), (33, 160, 8179, 32), (128, 128, 20001, 128), (65, 96, 70000, 32), (100, 256, 77777, 64), (64, 192, 151936, 192),
                                         (130, 64, 151936, 32), (50, 384, 160001, 128)])
def test_projection_of_many_rows_with_many_tiles_a_workgroup(B, K, V, group, masked):
    p = Projection(B, K, V, group, "bf16" if V % 2 else "f16", zeros=B % 2 == 0, whole=True, seed=B)
    want = torch.from_numpy(p.want()[0]).float().cuda()             # (exact: small whole numbers)
    mask = None
    if masked:
        rng = np.random.default_rng(V)
        allowed = rng.random((B, V)) < rng.choice([0.0, 0.001, 0.4, 0.97], (B, 1))
        allowed[:, V // 5:V // 2] = False                           # workgroups without a row, and some with few
        allowed[B // 2, V // 3] = True
        mask = _dev(plain.pack(allowed))
        want.masked_fill_(_dev(~allowed), -float("inf"))
    assert torch.equal(p.run("f32", mask, stride=V + 3), want)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,K,V,group", [(1, 128, 300001, 128), (3, 64, 600007, 32), (20, 128, 9000, 32), (32, 64, 70001, 64), (17, 256, 20000, 128), (24, 64, 300001, 32),
                                         (40, 64, 300001, 64)])
def test_projection_of_few_rows_with_many_tiles_or_long_lists(B, K, V, group, masked):
    """Two times 16 rows with more than one tile a workgroup, and more than 1024 rows of the matrix, which are listed in parts."""
    p = Projection(B, K, V, group, "f16" if V % 2 else "bf16", zeros=B % 2 == 1, whole=True, seed=B + 1)
    want = torch.from_numpy(p.want()[0]).float().cuda()
    mask = None
    if masked:
        rng = np.random.default_rng(V)
        allowed = rng.random((B, V)) < rng.choice([0.002, 0.5, 1.0], (B, 1))
        allowed[:, V // 5:V // 2] = False
        allowed[B // 2, V // 3] = True
        mask = _dev(plain.pack(allowed))
        want.masked_fill_(_dev(~allowed), -float("inf"))
    assert torch.equal(p.run("f32", mask), want)


def test_projection_of_what_is_not_finite():
    p = Projection(3, 256, 200, 32, "bf16", whole=True)
    p.hidden[1, 100] = float("inf")
    p.hidden[2, 17] = float("nan")
    allowed = np.random.default_rng(0).random((3, 200)) < 0.5
    finite = p.hidden.clone()
    got = _np(p.run(mask=_dev(plain.pack(allowed))))
    p.hidden = torch.where(finite.isfinite(), finite, torch.zeros_like(finite))
    want, _ = p.want()
    assert np.array_equal(got[0], np.where(allowed[0], want[0], -np.inf))
    assert (got[~allowed] == -np.inf).all() and not np.isfinite(got[1:][allowed[1:]]).any()


def test_projection_of_a_matrix_beyond_2_to_the_31_bytes():
    V, K = 589824, 8192
    free, _ = torch.cuda.mem_get_info()
    if free < 8 << 30:
        pytest.skip("needs 8 GiB of device memory")
    p = Projection(1, K, 64, 128, "bf16", whole=True)
    codes = torch.zeros((V, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.ones((V, K // 128), dtype=torch.bfloat16, device="cuda")
    codes[-64:], scales[-64:] = p.codes, p.scales
    want, _ = p.want()
    p.V, p.codes, p.scales = V, codes, scales
    got = _np(p.run()[:, -64:])
    assert np.array_equal(got, want)


# ------------------------------------------------------------------------------------------------ rules
class Batch:
    """Logits and rules: numpy on the host, tensors on the device."""

    def __init__(self, rows, V, dtype, seed=0, history=0, bias=0, mask=None, prompt=True, pad=0, offset=0, sigma=2.0):
        rng = np.random.default_rng(seed)
        self.rows, self.V, self.dtype, self.stride, self.offset = rows, V, dtype, V + pad, offset
        buf = torch.from_numpy((sigma * rng.standard_normal(offset + rows * self.stride)).astype(np.float32)).to(TYPES[dtype][0])
        self.buf = buf.cuda()
        self.h = dict(tokens=None)
        if history:
            ids = (rng.random((rows, history)) ** 4 * V).astype(np.int32)
            ids[rng.random(ids.shape) < 0.02] = -1
            ids[rng.random(ids.shape) < 0.02] = V + 3
            n = rng.integers(0, history + 1, rows).astype(np.int32)
            n[0] = history + 5                          # cut off at the stride
            self.h = dict(tokens=ids, n_tokens=n, n_prompt=(n * rng.random(rows)).astype(np.int32) if prompt else None,
                          repetition=(0.8 + 0.6 * rng.random(rows)).astype(np.float32), frequency=rng.standard_normal(rows).astype(np.float32),
                          presence=rng.standard_normal(rows).astype(np.float32))
        self.bias = None
        if bias:
            self.bias = [[(int(rng.integers(-2, V + 2)), float(np.float32(rng.standard_normal()))) for _ in range(int(rng.integers(0, bias + 1)))]
                         for _ in range(rows)]
        self.allowed, self.v_mask = None, 0
        if mask is not None:
            self.v_mask = V if mask != "short" else max(1, V - V // 5)
            self.allowed = rng.random((rows, self.v_mask)) < rng.choice([0.0, 0.01, 0.5, 0.97], (rows, 1))
            if rows > 1:
                self.allowed[rows // 2] = False         # a row without a token
        self.upload()

    def upload(self):
        h = self.h
        self.d = {k: _dev(v) for k, v in h.items()}
        r = {"d_" + k: _at(v) for k, v in self.d.items()}
        if h["tokens"] is not None:
            r["token_stride"] = h["tokens"].shape[1]
        if self.bias is not None:
            flat = [e for row in self.bias for e in row] + [(0, 0.0)]
            self.d_bias = [_dev(np.array([t for t, _ in flat], np.int32)), _dev(np.array([v for _, v in flat], np.float32)),
                           _dev(np.concatenate([[0], np.cumsum([len(x) for x in self.bias])]).astype(np.int32))]
            r |= dict(d_bias_ids=_at(self.d_bias[0]), d_bias=_at(self.d_bias[1]), d_bias_offsets=_at(self.d_bias[2]), n_bias=len(flat) - 1)
        if self.allowed is not None:
            self.d_mask = _dev(plain.pack(self.allowed))
            r |= dict(d_bitmask=_at(self.d_mask), v_mask=self.v_mask)
        self.rules = _xgm().LogitRules(**r)

    @property
    def logits(self):
        return self.buf[self.offset:].view(self.rows, self.stride)[:, :self.V]

    def address(self):
        return self.buf.data_ptr() + self.offset * self.buf.element_size()

    def want(self):
        x = self.logits.float().cpu().numpy()
        return np.stack([plain.processed(x[b], b, None if self.allowed is None else self.allowed[b], bias=None if self.bias is None else self.bias[b],
                                         **self.h) for b in range(self.rows)])


RULES = [dict(rows=1, V=1, dtype="f32", history=3, bias=2), dict(rows=2, V=31, dtype="bf16", history=8, mask="full"),
         dict(rows=3, V=33, dtype="f16", bias=9, mask="short", pad=3, offset=1), dict(rows=4, V=8192, dtype="bf16", history=700, bias=40, mask="full"),
         dict(rows=5, V=8193, dtype="f32", history=300, mask="full", offset=3), dict(rows=3, V=50001, dtype="bf16", history=5000, bias=300, offset=5),
         dict(rows=2, V=100003, dtype="f16", history=33000, bias=1, mask="short"), dict(rows=7, V=32000, dtype="f32", mask="full"),
         dict(rows=9, V=4099, dtype="bf16"), dict(rows=6, V=20011, dtype="f16", history=64, prompt=False, pad=13, mask="full"),
         dict(rows=1, V=151936, dtype="bf16", history=2048, bias=16, mask="full"), dict(rows=65, V=1031, dtype="f32", history=50, bias=5, mask="full"), dict(rows=3, V=5000, dtype="bf16", history=9, bias=6000)]


@pytest.mark.parametrize("how", ["apart", "in place", "shifted"])
@pytest.mark.parametrize("case", RULES, ids=lambda c: f"{c['rows']}x{c['V']}-{c['dtype']}")
def test_rules_give_the_bits_of_the_definition(case, how):
    xgm = _xgm()
    c = Batch(**case, seed=case["V"])
    want = torch.from_numpy(c.want()).to(TYPES[c.dtype][0])
    if how == "in place":
        out, stride, at = c.logits, c.stride, c.address()
        before = c.buf.clone()
    else:
        stride = c.V + (3 if how == "shifted" else 0)
        buf = torch.full((1 + c.rows * stride,), 7.0, dtype=TYPES[c.dtype][0], device="cuda")
        k = 1 if how == "shifted" else 0
        out, at = buf[k:k + c.rows * stride].view(c.rows, stride)[:, :c.V], buf.data_ptr() + k * buf.element_size()
    xgm.process_logits(c.address(), TYPES[c.dtype][1], c.rows, c.V, c.stride, c.rules, at, stride, _stream())
    torch.cuda.synchronize()
    view = torch.int32 if c.dtype == "f32" else torch.int16
    assert torch.equal(out.cpu().contiguous().view(view), want.view(view))
    if how == "in place":
        now = c.buf.clone()
        now[c.offset:].view(c.rows, c.stride)[:, :c.V] = before[c.offset:].view(c.rows, c.stride)[:, :c.V]
        assert torch.equal(now.view(view), before.view(view))       # the columns beyond V and what lies in front
    else:
        rest = torch.full_like(buf, 7.0)
        rest[k:k + c.rows * stride].view(c.rows, stride)[:, :c.V] = out
        assert torch.equal(buf.view(view), rest.view(view))


def test_a_history_in_the_last_columns_of_a_wider_array():
    xgm = _xgm()
    c = Batch(3, 700, "f32", seed=2, history=90, bias=3)
    wide = torch.full((3, 150), 5, dtype=torch.int32, device="cuda")     # tokens that would count if they were taken
    wide[:, 60:] = c.d["tokens"]
    c.h["n_tokens"] = np.array([90, 0, 71], np.int32)                   # within the array: the rows lie 150 apart
    c.h["n_prompt"] = np.array([95, 3, 0], np.int32)
    c.upload()
    want = torch.from_numpy(c.want())
    c.rules._s.d_tokens, c.rules._s.token_stride = wide[:, 60:].data_ptr(), 150
    out = torch.empty((3, 700), device="cuda")
    xgm.process_logits(c.address(), 0, 3, 700, c.stride, c.rules, out.data_ptr(), 700, _stream())
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().view(torch.int32), want.view(torch.int32))


@pytest.mark.parametrize("rule", ["bias", "presence"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rules_round_once(dtype, rule):
    """Sums that lie so close beside the middle of two neighbours of the type that 32 bits take them for the middle go to the nearer
    neighbour, not to the even one."""
    xgm = _xgm()
    bits, V, t = {"bf16": 7, "f16": 10}[dtype], 4000, TYPES[dtype][0]
    rng = np.random.default_rng(3)
    low = (1 + rng.integers(0, 2 ** bits, V) * 2.0 ** -bits) * 2.0 ** rng.integers(5, 9, V)      # of the two neighbours, whose middle is
    middle = low + 2.0 ** -(bits + 1) * 2.0 ** np.floor(np.log2(low))                            # exact in 32 bits
    sign, side = rng.choice([-1.0, 1.0], V), rng.choice([-1.0, 1.0], V)
    x = side * 2.0 ** -24                                                                        # less than 2^-25 of the sum
    n = 1 if rule == "bias" else V
    want = torch.from_numpy(np.where(sign * side > 0, 2 * middle - low, low) * sign).to(t)
    assert (np.float32(sign * middle + x) == sign * middle).all() and (sign * middle + x != sign * middle).all()
    if rule == "bias":
        d = [_dev(np.arange(V, dtype=np.int32)), _dev((sign * middle).astype(np.float32)), _dev(np.array([0, V], np.int32))]
        rules = xgm.LogitRules(d_bias_ids=_at(d[0]), d_bias=_at(d[1]), d_bias_offsets=_at(d[2]), n_bias=V)
        logits = torch.from_numpy(x).to(t).cuda()[None]
    else:       # row b generated token b
        d = [torch.arange(V, dtype=torch.int32, device="cuda"), torch.ones(V, dtype=torch.int32, device="cuda"), _dev((-sign * middle).astype(np.float32))]
        rules = xgm.LogitRules(d_tokens=_at(d[0]), token_stride=1, d_n_tokens=_at(d[1]), d_presence=_at(d[2]))
        logits = torch.from_numpy(x).to(t).cuda()[None].expand(V, V).contiguous()
    out = torch.empty((n, V), dtype=t, device="cuda")
    xgm.process_logits(logits.data_ptr(), TYPES[dtype][1], n, V, V, rules, out.data_ptr(), V, _stream())
    got = out[0] if rule == "bias" else out.diagonal().contiguous()
    assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rules_on_what_is_not_finite(dtype):
    xgm = _xgm()
    c = Batch(3, 3000, dtype, seed=1, history=400, mask="full")
    low = torch.finfo(TYPES[dtype][0]).min
    for k, v in enumerate([float("nan"), float("inf"), -float("inf"), low, 0.0, -0.0]):
        c.buf[k::7] = v
    want = torch.from_numpy(c.want())
    out = torch.empty((3, 3000), dtype=TYPES[dtype][0], device="cuda")
    xgm.process_logits(c.address(), TYPES[dtype][1], 3, 3000, c.stride, c.rules, out.data_ptr(), 3000, _stream())
    got = out.float().cpu()
    want = want.to(TYPES[dtype][0]).float()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=5.0, posinf=1e38, neginf=-1e38), want.nan_to_num(nan=5.0, posinf=1e38, neginf=-1e38))
    assert bool((got[torch.from_numpy(~c.allowed)] == -float("inf")).all())


# ------------------------------------------------------------------------------------------------ draws
def _draw(c, temperature=None, top_k=None, top_p=None, min_p=None, uniform=None, sampler=None, logprobs=True):
    xgm = _xgm()
    d = [_dev(np.asarray(v, t)) if v is not None else None
         for v, t in ((temperature, np.float32), (top_k, np.int32), (top_p, np.float32), (min_p, np.float32), (uniform, np.float64))]
    draw = xgm.DrawRules(d_temperature=_at(d[0]), d_top_k=_at(d[1]), d_top_p=_at(d[2]), d_min_p=_at(d[3]), d_uniform=_at(d[4]))
    s = sampler or xgm.Sampler(c.rows, c.V, _stream())
    ids = torch.full((c.rows + 1,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((c.rows + 1,), 7.0, dtype=torch.float32, device="cuda")
    before = c.buf.clone()
    s.sample(c.address(), TYPES[c.dtype][1], c.rows, c.V, c.stride, c.rules, draw, ids.data_ptr(), lp.data_ptr() if logprobs else 0, _stream())
    torch.cuda.synchronize()
    assert int(ids[-1]) == -7 and float(lp[-1]) == 7.0
    assert torch.equal(c.buf.view(torch.uint8), before.view(torch.uint8))          # the logits are read only
    return ids[:-1].cpu().numpy(), lp[:-1].cpu().numpy()


def _check_logprob(got, want):
    if want == -np.inf:
        assert got == -np.inf
    else:
        assert abs(float(got) - want) <= 2.0 ** -24 * abs(want) + 1e-9, (got, want)


def _p_between(row, rng):
    """A top_p (float32) whose cut lies in the middle of a token's stretch; 1 where there is no such place."""
    share = row.run_sorted / row.run_sorted[-1]
    gap = np.diff(np.concatenate([[0.0], share]))
    can = np.flatnonzero(gap > 1e-5)
    if not can.size:
        return np.float32(1.0)
    k = int(can[rng.integers(can.size)])
    return np.float32(share[k] - 0.5 * gap[k])


DRAWS = [dict(rows=1, V=1, dtype="f32"), dict(rows=4, V=7, dtype="bf16", mask="full"), dict(rows=8, V=33, dtype="f16", history=20, bias=4),
         dict(rows=5, V=1000, dtype="f32", sigma=0.0), dict(rows=6, V=8192, dtype="bf16", history=100, mask="full"),
         dict(rows=12, V=8191, dtype="f32", sigma=8.0, offset=1), dict(rows=7, V=8193, dtype="bf16", pad=7, offset=3, bias=30),
         dict(rows=3, V=50001, dtype="bf16", sigma=0.02), dict(rows=9, V=32000, dtype="f16", history=3000, bias=50, mask="short", sigma=3.0),
         dict(rows=4, V=100003, dtype="f32", sigma=1.0), dict(rows=2, V=151936, dtype="bf16", history=700, mask="full"),
         dict(rows=33, V=2500, dtype="bf16", mask="full", sigma=1.0), dict(rows=2, V=300000, dtype="f32", sigma=0.0), dict(rows=1, V=589824, dtype="bf16")]


@pytest.mark.parametrize("what", ["all", "k", "p", "m", "kp", "kpm"])
@pytest.mark.parametrize("case", DRAWS, ids=lambda c: f"{c['rows']}x{c['V']}-{c['dtype']}-{c.get('sigma', 2.0)}")
def test_draws_are_those_of_the_definition(case, what):
    c = Batch(**case, seed=case["V"] + 1)
    rng = np.random.default_rng(len(what))
    y = c.want()
    s = _xgm().Sampler(c.rows + 2, c.V + 5, _stream())
    for turn in range(3):
        t = np.where(rng.random(c.rows) < 0.15, 0.0, rng.choice([0.3, 0.7, 1.0, 1.7], c.rows)).astype(np.float32)
        k = rng.choice([0, 1, 2, 5, 50, 400, 3000, c.V, c.V + 9], c.rows) if "k" in what else np.zeros(c.rows, int)
        m = rng.choice([0.0, 0.01, 0.2, 1.0], c.rows).astype(np.float32) if "m" in what else np.zeros(c.rows, np.float32)
        p, u, want = np.ones(c.rows, np.float32), np.zeros(c.rows), []
        for b in range(c.rows):
            row = plain.Row(y[b], float(t[b]), int(k[b]))
            if "p" in what and not row.empty:
                p[b] = _p_between(row, rng)
            row = plain.Row(y[b], float(t[b]), int(k[b]), float(p[b]), float(m[b]))
            if row.empty:
                want.append((-1, -np.inf))
                continue
            u[b], v = row.middle(rng)
            v = int(row.order[0]) if t[b] == 0 else v
            want.append((v, row.logprob(v)))
        ids, lp = _draw(c, t, k if "k" in what else None, p if "p" in what else None, m if "m" in what else None, u, s)
        assert ids.tolist() == [v for v, _ in want], (turn, t, k, p, m, u)
        for got, (_, w) in zip(lp, want):
            _check_logprob(got, w)


@pytest.mark.parametrize("what", ["k", "p", "m", "kpm"])
@pytest.mark.parametrize("case", [dict(rows=128, V=70000, dtype="bf16", history=300, bias=4, mask="full", sigma=3.0), dict(rows=1100, V=2000, dtype="f32", sigma=2.0),
                                  dict(rows=200, V=50001, dtype="f16", sigma=0.0), dict(rows=64, V=151936, dtype="bf16", sigma=2.5, offset=3)],
                         ids=lambda c: f"{c['rows']}x{c['V']}-{c['dtype']}")
def test_large_batches_that_keep_few_tokens(case, what):
    """More than 1024 slices, where no list of the kept tokens is made; in a small batch the same rows are drawn from a list."""
    c = Batch(**case, seed=case["rows"])
    rng = np.random.default_rng(len(what))
    y, rows = c.want(), c.rows
    assert rows * -(-c.V // 8192) > 1024
    t = rng.choice([0.3, 0.7, 1.0, 1.7], rows).astype(np.float32)
    k = rng.choice([1, 2, 5, 50], rows) if "k" in what else np.zeros(rows, int)
    m = rng.choice([0.01, 0.2, 1.0], rows).astype(np.float32) if "m" in what else np.zeros(rows, np.float32)
    p, u, want = np.ones(rows, np.float32), np.zeros(rows), []
    for b in range(rows):
        row = plain.Row(y[b], float(t[b]), int(k[b]))
        if row.empty:
            want.append((-1, -np.inf))
            continue
        if "p" in what:                     # the middle of the stretch of one of the first 60
            share = row.run_sorted[:60] / row.run_sorted[-1]
            at = int(rng.integers(0, share.size))
            p[b] = np.float32(0.5 * (share[at] + (share[at - 1] if at else 0.0)))
        row.__init__(y[b], float(t[b]), int(k[b]), float(p[b]), float(m[b]))
        u[b], v = row.middle(rng)
        want.append((v, row.logprob(v)))

    def draw(n):
        c.rows = n
        ids, lp = _draw(c, t[:n], k[:n] if "k" in what else None, p[:n] if "p" in what else None, m[:n] if "m" in what else None, u[:n])
        c.rows = rows
        return ids, lp

    buf, (ids, lp) = c.buf, draw(rows)
    assert ids.tolist() == [v for v, _ in want]
    for got, (_, w) in zip(lp, want):
        _check_logprob(got, w)
    few = 9
    assert few * -(-c.V // 8192) <= 1024
    some, some_lp = draw(few)
    assert np.array_equal(some, ids[:few]) and np.array_equal(some_lp, lp[:few]) and c.buf is buf


def test_the_likeliest_token_is_taken_without_random_numbers():
    c = Batch(6, 9001, "bf16", seed=5, mask="full", sigma=0.5)      # many equal logits at the top
    y = c.want()
    for kw in (dict(), dict(temperature=[0.0, -1.0, 0.5, float("nan"), 1.0, 2.0])):
        ids, lp = _draw(c, **kw)
        for b in range(6):
            row = plain.Row(y[b])
            want = -1 if row.empty else int(row.order[0])
            assert ids[b] == want
            _check_logprob(lp[b], row.logprob(want) if want >= 0 else -np.inf)
    ids, _ = _draw(c, temperature=[0.0, -1.0, 0.0, float("nan"), 0.0, -2.0], uniform=[0.3] * 6, top_p=[0.5] * 6, logprobs=False)
    assert ids.tolist() == [-1 if plain.Row(r).empty else int(plain.Row(r).order[0]) for r in y]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_min_p_whose_border_lies_at_a_logit_of_0(dtype):
    """Next to 0 thousands of floats have the same weight in 64 bits: those that weigh min_p are kept, all of them."""
    tiny = [-1e-38, -1e-30, -1e-20, -1e-17, 0.0, 1e-20]
    rows = [([0.0] + tiny, 1.0, 1.0), ([0.0] + tiny, 0.7, 1.0), ([1.0] + tiny, 1.0 / np.log(4.0), 0.25), ([0.5] + tiny, 0.5 / np.log(2.0), 0.5),
            ([1e-30, -1.0] + tiny, 1.0, 1.0), ([-1e-25] + tiny[:2], 3.0, 1.0)]
    c = Batch(len(rows), 64, dtype)
    c.rules = None
    x = torch.full((len(rows), 64), -50.0)
    for b, (v, _, _) in enumerate(rows):
        x[b, :len(v)] = torch.tensor(v)
    c.buf[:] = x.reshape(-1).to(c.buf.dtype).cuda()
    y, t, m = c.logits.float().cpu().numpy(), np.float32([r[1] for r in rows]), np.float32([r[2] for r in rows])
    plains = [plain.Row(y[b], float(t[b]), 0, 1.0, float(m[b])) for b in range(len(rows))]
    for k in range(64):
        u = [(min(k, len(r.kept) - 1) + 0.5) / len(r.kept) if b in (0, 1, 4) else (k + 0.5) / 64 for b, r in enumerate(plains)]
        ids, _ = _draw(c, t, None, None, m, u)
        assert ids.tolist() == [r.pick(u[b]) for b, r in enumerate(plains)], k


def test_random_numbers_and_settings_at_their_ends():
    c = Batch(8, 5003, "f32", seed=2, sigma=3.0)
    y = c.want()
    u = [0.0, np.nextafter(1.0, 0.0), 1.0, 5.0, -1.0, float("nan"), 0.0, 0.5]
    p = [0.9, 0.9, 0.9, 0.9, 0.0, float("nan"), -1.0, 2.0]
    k = [-3, 0, 2, 10 ** 9, 0, 0, 0, 1]
    m = [0.0, float("nan"), -1.0, 0.0, 0.0, 0.0, 7.0, 0.0]
    ids, _ = _draw(c, [1.0] * 8, k, p, m, u)
    rows = [plain.Row(y[b], 1.0, max(0, k[b]), p[b] if p[b] < 1 else 1.0, m[b] if m[b] > 0 else 0.0) for b in range(8)]
    seen = [b for b in range(8) if b not in (1, 2, 3)]
    assert [int(ids[b]) for b in seen] == [rows[b].pick(u[b] if u[b] >= 0 else 0.0) for b in seen]
    for b in (1, 2, 3):                                 # the last kept token that weighs enough to count
        kept = rows[b].kept[rows[b].w[rows[b].kept] > 2.0 ** -40]
        assert ids[b] >= kept[-1] and ids[b] in rows[b].kept


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_draws_from_what_is_not_finite(dtype):
    V, low = 9000, torch.finfo(TYPES[dtype][0]).min
    c = Batch(7, V, dtype, seed=4)
    x = c.logits
    x[0] = float("nan")
    x[1] = -float("inf")
    x[2] = low
    x[3, ::2] = float("nan")
    x[4, 17::1000] = float("inf")
    x[5, :8500] = -float("inf")
    x[6, 1::2] = low
    y = c.want()
    rng = np.random.default_rng(1)
    for top_p in (1.0, 0.6):
        p = np.full(7, top_p, np.float32)
        rows = [plain.Row(y[b], 0.8, 0, float(p[b])) for b in range(7)]
        picks = [(0.0, -1) if r.empty else r.middle(rng) for r in rows]
        ids, lp = _draw(c, [0.8] * 7, None, p, None, [u for u, _ in picks])
        assert ids.tolist() == [v for _, v in picks]
        assert ids[0] == -1 and ids[1] == -1 and np.isneginf(lp[:2]).all() and (ids[2:] >= 0).all()
        for b in range(2, 7):
            _check_logprob(lp[b], rows[b].logprob(int(ids[b])))


def test_draws_follow_their_probabilities():
    c = Batch(1, 6, "f32", seed=9, sigma=1.0)
    n = 4096
    c.buf = c.buf.repeat(n, 1).reshape(-1).contiguous()
    c.rows = n
    c.rules = None
    row = plain.Row(c.logits[0].cpu().numpy(), 0.9)
    u = (np.arange(n) + 0.5) / n
    ids, _ = _draw(c, [0.9] * n, uniform=u)
    share = np.bincount(ids, minlength=6) / n
    assert np.abs(share - row.w / row.w.sum()).max() <= 1.0 / n


@pytest.mark.parametrize("sigma", [0.3, 2.0])
def test_weights_have_the_bits_of_64(sigma):
    """A random number 1e-14 beside the border between two tokens falls on its side.  A weight is off by at most (2 + |logit|) 2^-52
    of itself with logits below 12, the border by twice that, and four additions and the product with the number by 2^-53 each: 7e-15."""
    rows, V = 8192, 4
    rng = np.random.default_rng(8)
    c = Batch(rows, V, "f32", sigma=sigma)
    c.rules = None
    y = c.logits.cpu().numpy().astype(np.longdouble)
    assert np.abs(y).max() < 12 and np.finfo(np.longdouble).nmant >= 63
    run = np.cumsum(np.exp(y - y.max(1, keepdims=True)), 1)
    border = rng.integers(0, V - 1, rows)
    upper = rng.random(rows) < 0.5
    share = run[np.arange(rows), border] / run[:, -1]
    u = (share * (1 + np.where(upper, 1, -1) * np.longdouble(1e-14))).astype(np.float64)
    ids, _ = _draw(c, uniform=u)
    assert (ids == border + upper).all(), int((ids != border + upper).sum())


@pytest.mark.parametrize("V,sigma,top_p,rows", [(20000, 1.0, 0.999, 64), (40000, 2.0, 0.9, 48), (3000, 1.0, 0.06, 256), (3000, 1.0, 0.06, 1500), (16500, 1.0, 0.03, 500)])
def test_a_cut_row_is_drawn_from_to_2_to_the_minus_35(V, sigma, top_p, rows):
    """A random number 2^-34 of itself beside a border falls on its side (borders are off by 2^-35): by the sums of the slices, where
    hundreds of tokens are kept or there are more than 1024 slices, and from a list of the kept ones."""
    c = Batch(rows, V, "f32", seed=6, sigma=sigma)
    rng = np.random.default_rng(6)
    y, u, want = c.want(), np.zeros(rows), []
    for b in range(rows):
        row = plain.Row(y[b], 1.0, 0, float(np.float32(top_p)))
        k, upper = int(rng.integers(0, len(row.kept) - 1)), bool(rng.random() < 0.5)
        u[b] = row.run[k] / row.run[-1] * (1 + (2.0 ** -34 if upper else -2.0 ** -34))
        want.append(int(row.kept[k + upper]))
    ids, _ = _draw(c, top_p=[top_p] * rows, uniform=u)
    assert ids.tolist() == want


@pytest.mark.parametrize("top_p", [None, 0.9])
@pytest.mark.parametrize("V", [7, 2140, 20000])
def test_a_token_that_is_alone_has_logprob_0(V, top_p):
    rows = 24
    c = Batch(rows, V, "bf16", seed=V, history=331, bias=194, mask="full")
    only = np.random.default_rng(V).integers(0, V, rows)
    c.allowed = np.zeros((rows, V), bool)
    c.allowed[np.arange(rows), only] = True
    c.upload()
    ids, lp = _draw(c, np.linspace(0.3, 1.9, rows), top_p=None if top_p is None else [top_p] * rows, uniform=np.linspace(0.0, 0.999, rows))
    assert ids.tolist() == only.tolist() and (lp == 0).all()


def test_top_p_takes_lower_ids_first_among_equal_logits():
    c = Batch(4, 20000, "bf16", seed=0, sigma=0.0)                  # all equal
    n = [1, 2, 9999, 20000]
    p = [(k - 0.5) / 20000 for k in n]
    ids, lp = _draw(c, None, None, p, None, [1 - 1e-9] * 4)
    assert ids.tolist() == [k - 1 for k in n]
    assert np.allclose(lp, -np.log(20000.0), rtol=1e-6)
    ids, _ = _draw(c, None, n, None, None, [1 - 1e-9] * 4)
    assert ids.tolist() == [k - 1 for k in n]


@pytest.mark.parametrize("rows,V,history,bias", [(128, 151936, 1500, 40), (48, 70001, 0, 3), (300, 9000, 200, 0), (2, 1000003, 3000, 9)])
def test_draws_without_a_cut_under_rules_are_those_from_logits_that_went_through_the_rules_before(rows, V, history, bias):
    xgm = _xgm()
    c = Batch(rows, V, "f32", seed=V, history=history, bias=bias, mask="full")
    done = torch.empty((rows, V), device="cuda")
    xgm.process_logits(c.address(), 0, rows, V, c.stride, c.rules, done.data_ptr(), V, _stream())
    ids, lp = torch.empty((2, rows), dtype=torch.int32, device="cuda"), torch.empty((2, rows), device="cuda")
    temperature, sampler = torch.linspace(0.5, 1.6, rows, device="cuda"), xgm.Sampler(rows, V, _stream())
    seen = set()
    for turn in range(30):
        u = torch.rand(rows, dtype=torch.float64, generator=torch.Generator().manual_seed(turn)).cuda()
        draw = xgm.DrawRules(d_temperature=temperature.data_ptr(), d_uniform=u.data_ptr())
        for k, (at, stride, rules) in enumerate([(c.address(), c.stride, c.rules), (done.data_ptr(), V, None)]):
            sampler.sample(at, 0, rows, V, stride, rules, draw, ids[k].data_ptr(), lp[k].data_ptr(), _stream())
        torch.cuda.synchronize()
        assert torch.equal(ids[0], ids[1]) and torch.equal(lp[0], lp[1]), turn
        seen |= set((ids[0] // 8192).tolist())
    assert len(seen - {-1}) > 1                                     # (more than one slice was drawn from)


# ------------------------------------------------------------------------------------------------ streams and graphs
def test_the_chain_replays_from_a_graph_and_runs_on_another_stream():
    xgm = _xgm()
    B, K, V = 6, 512, 12345
    p = Projection(B, K, V, 64, "bf16", zeros=True)
    logits = torch.empty((B, V), dtype=torch.bfloat16, device="cuda")
    c = Batch(B, V, "bf16", seed=1, history=60, bias=5, mask="full")
    c.h["n_tokens"][0] = 60
    c.upload()
    u = torch.rand(B, dtype=torch.float64, device="cuda")
    draw = xgm.DrawRules(d_uniform=u.data_ptr(), d_top_p=(top_p := torch.full((B,), 0.9, device="cuda")).data_ptr())
    sampler = xgm.Sampler(B, V, _stream())
    ids, lp = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
    out = torch.empty_like(logits)

    def step():
        xgm.q4_logits(p.hidden.data_ptr(), 1, B, K, K, p.codes.data_ptr(), p.scales.data_ptr(), p.zeros.data_ptr(), V, 64, logits.data_ptr(), 1, V,
                      c.d_mask.data_ptr(), _stream())
        xgm.process_logits(logits.data_ptr(), 1, B, V, V, c.rules, out.data_ptr(), V, _stream())
        sampler.sample(logits.data_ptr(), 1, B, V, V, c.rules, draw, ids.data_ptr(), lp.data_ptr(), _stream())

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for turn in range(5):
        p.hidden.copy_(torch.randn((B, K), device="cuda"))
        u.copy_(torch.rand(B, dtype=torch.float64, device="cuda"))
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (logits, out, ids, lp)]
        for t in (logits, out, ids, lp):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (logits, out, ids, lp))), turn
        for t in (logits, out, ids, lp):
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (logits, out, ids, lp))), turn
    assert float(top_p[0]) > 0
