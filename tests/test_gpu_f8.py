"""The output matrix in 8 bits (projection, hidden states to 8 bits) and rows of output matrices as hidden states, against their
definitions in 64 bits.

Tolerances.  Codes and scales: the same, bit for bit.  Projection: products are exact (two numbers of 4 bits), K of them are added in
32 bits, each addition off by at most 2^-23 of S = sum |hidden * weight| (the matrix instruction may cut off what it does not keep),
with random signs within 2 sqrt(K) 2^-23 S; the product of two scales, the product with it and the addition of a block add 3 * 2^-24 S;
the result is rounded once to its type (eps / 2 of the value, and half of the smallest number).  Where values are small whole numbers and scales powers of two all
sums are exact, and so must the result be.  Lookups: 64 bits rounded once, the same bits.

Logits of 16 bits in batches of more than 64 rows come from the instructions for 8 bits, which cut a product off at 2^-13 of the largest of
its group of at most 8 neighbours.  With p the products of a logit and m their groups' largest, the K cuts are independent and each less than
2^-13 m, so that their sum has a deviation of at most 2^-13 / sqrt(3) sqrt(sum of m^2) <= 2^-13 / sqrt(3) sqrt(8 sum of p^2); six of
those are allowed for: 2^-13 sqrt(96) sqrt(sum of p^2)."""

import numpy as np
import pytest

import plain_beams as plain
import plain_logits

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"f32": (torch.float32, 0), "bf16": (torch.bfloat16, 1), "f16": (torch.float16, 2), "f8": (torch.uint8, 3)}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def _xgm():
    import paper_2411_15100_amd as xgm
    return xgm


def _stream():
    return int(torch.cuda.current_stream().cuda_stream)


def _np(t):
    return t.detach().double().cpu().numpy()


def _at(t):
    return 0 if t is None else t.data_ptr()


# ------------------------------------------------------------------------------------------------ hidden states to 8 bits
def _quantize(x, pad=0, gap=0):
    xgm = _xgm()
    B, K = x.shape
    e = 16 // x.element_size()
    wide = torch.zeros((B, K + pad * e), dtype=x.dtype, device="cuda")
    wide[:, :K] = x
    codes = torch.full((B + 1, K + 16 * gap), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((B * plain.blocks(K) + 3,), 5.0, device="cuda")
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[x.dtype]
    xgm.f8_quantize(wide.data_ptr(), code, B, K, wide.stride(0), codes.data_ptr(), codes.stride(0), scales.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert bool((codes[B] == 77).all()) and bool((codes[:, K:] == 77).all()) and bool((scales[B * plain.blocks(K):] == 5).all())
    return codes[:B, :K].cpu().numpy(), scales[:B * plain.blocks(K)].view(B, -1).double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,K", [(1, 16), (3, 128), (2, 144), (17, 1024), (5, 2080), (130, 272)])
def test_values_in_8_bits_are_those_of_the_definition(B, K, dtype):
    g = torch.Generator().manual_seed(B + K)
    x = torch.randn((B, K), generator=g) * torch.exp(3 * torch.randn((B, 1), generator=g))
    x = x.to(TYPES[dtype][0])
    want = plain.quantized(_np(x))
    got = _quantize(x.cuda(), pad=B % 3, gap=B % 2)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0])


def test_every_step_and_every_middle_of_8_bits():
    values = plain.e4m3()[:127]
    middles = (values[1:] + values[:-1]) / 2
    near = np.concatenate([np.nextafter(middles.astype(np.float32), np.float32(s)) for s in (0, 1e9)])
    x = np.concatenate([values, -values, middles, -middles, near, -near]).astype(np.float32)
    x = np.resize(x, (-(-x.size // 127), 127))
    x = np.concatenate([x, np.full((x.shape[0], 1), 448, np.float32)], 1)             # every block keeps scale 1
    for scale in (1.0, 2.0 ** -100, 2.0 ** 100):
        t = torch.from_numpy(x * np.float32(scale))
        want, got = plain.quantized(_np(t)), _quantize(t.cuda())
        assert (want[1] == scale).all() and np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_scales_at_their_ends_and_values_that_are_not_finite(dtype):
    t = TYPES[dtype][0]
    info = torch.finfo(t)
    x = torch.zeros((9, 256), dtype=t)
    x[1, :3] = torch.tensor([info.smallest_normal, -info.smallest_normal, 0.0])
    x[2, 5] = info.max
    x[3, 7] = float("inf")
    x[4, 9] = float("nan")
    x[4, 10] = 3.0
    x[5, 130] = -float("inf")
    x[6, :] = float("nan")
    x[7, 0] = 1.75
    x[8, 0] = float(np.nextafter(np.float32(1.75), np.float32(2))) if dtype == "f32" else 1.75 + info.eps
    want, got = plain.quantized(_np(x)), _quantize(x.cuda())
    assert np.array_equal(got[1], want[1])
    nan = lambda c: c & 127 == 127      # noqa: E731
    assert np.array_equal(nan(got[0]), nan(want[0])) and np.array_equal(got[0][~nan(got[0])], want[0][~nan(want[0])])
    assert nan(got[0])[3, 7] and nan(got[0])[5, 130] and nan(got[0])[6].all() and not nan(got[0])[[0, 1, 2, 7, 8]].any()


# ------------------------------------------------------------------------------------------------ projection
class Projection:
    def __init__(self, B, K, V, dtype, whole=False, seed=0, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.K, self.V, self.dtype = B, K, V, dtype
        nb, nv = plain.blocks(K), plain.blocks(V)
        if whole:
            h = torch.randint(-4, 5, (B, K), generator=g).float()
            small = torch.from_numpy(np.flatnonzero(np.isin(plain.e4m3(), [-3, -2, -1, -.5, 0, .5, 1, 2, 3, 4]) & (np.arange(256) != 128)))
            codes = small[torch.randint(0, len(small), (V, K), generator=g)].to(torch.uint8)
            scales = 2.0 ** torch.randint(-3, 2, (nv, nb), generator=g).float()
            hidden_scales = 2.0 ** torch.randint(-2, 3, (B, nb), generator=g).float()
        else:
            h = torch.randn((B, K), generator=g) * torch.exp(0.5 * torch.randn(K, generator=g))
            codes = torch.randint(0, 256, (V, K), generator=g, dtype=torch.uint8)
            codes[codes & 127 == 127] = 3
            scales = 0.01 * torch.exp(0.5 * torch.randn((nv, nb), generator=g))
            hidden_scales = 0.01 * torch.exp(0.5 * torch.randn((B, nb), generator=g))
        e = 1 if dtype == "f8" else 2
        pad *= 16 // e
        self.codes, self.scales = codes.cuda(), scales.cuda()
        if dtype == "f8":
            if whole:
                hidden = small[torch.randint(0, len(small), (B, K), generator=g)].to(torch.uint8)
            else:
                hidden = torch.randint(0, 256, (B, K), generator=g, dtype=torch.uint8)
                hidden[hidden & 127 == 127] = 130
            self.hidden_scales = hidden_scales.cuda()
            self.eight = hidden.numpy(), hidden_scales.double().numpy()
        else:
            hidden = h.to(TYPES[dtype][0])
            self.hidden_scales = None
            self.eight = plain.quantized(_np(hidden))
        wide = torch.full((B, K + pad), 127 if dtype == "f8" else float("nan"), dtype=hidden.dtype)      # (what lies behind a row is not read)
        wide[:, :K] = hidden
        self.hidden = wide.cuda()

    def want(self):
        return plain.project(*self.eight, self.codes.cpu().numpy(), self.scales.double().cpu().numpy())

    def squares(self, out):
        if self.B <= 64 or out == "f32":
            return None
        table, K = plain.e4m3(), self.K
        h = table[self.eight[0]] * np.repeat(self.eight[1], 128, 1)[:, :K]
        w = table[self.codes.cpu().numpy()] * np.repeat(np.repeat(self.scales.double().cpu().numpy(), 128, 0)[:self.V], 128, 1)[:, :K]
        return (h * h) @ (w * w).T

    def run(self, out="f32", mask=None, stride=None, offset=0, v_mask=None, with_work=False):
        xgm = _xgm()
        stride = stride or self.V
        buf = torch.full((offset + self.B * stride + 8,), 7.0, dtype=TYPES[out][0], device="cuda")
        n = xgm.f8_work_bytes(self.B, self.K)
        work = torch.full((n + 64,), 127, dtype=torch.uint8, device="cuda")
        xgm.f8_logits(self.hidden.data_ptr(), TYPES[self.dtype][1], _at(self.hidden_scales), self.B, self.K, self.hidden.stride(0), self.codes.data_ptr(),
                      self.scales.data_ptr(), self.V, buf.data_ptr() + offset * buf.element_size(), TYPES[out][1], stride, _at(mask),
                      0 if self.dtype == "f8" and not with_work else work.data_ptr(), _stream(), v_mask)
        torch.cuda.synchronize()
        assert bool((work[n:] == 127).all())
        assert bool((buf[:offset] == 7).all()) and bool((buf[offset + self.B * stride:] == 7).all())
        rows = buf[offset:offset + self.B * stride].view(self.B, stride)
        assert bool((rows[:, self.V:] == 7).all())      # nothing but the logits is written
        return rows[:, :self.V]


def tolerance(want, size, K, out, squares=None):
    """squares: sums of the squares of the products, where the instructions for 8 bits make them."""
    t = TYPES[out][0]
    if squares is not None:
        return torch.finfo(t).eps / 2 * np.abs(want) + TINY[out] / 2 + 2.0 ** -13 * np.sqrt(96 * squares) + 2.0 ** -20 * size
    return torch.finfo(t).eps / 2 * np.abs(want) + TINY[out] / 2 + (2 * np.sqrt(K) * 2.0 ** -23 + 3 * 2.0 ** -24) * size


SHAPES = [(1, 16, 1), (1, 128, 17), (3, 112, 33), (2, 144, 100), (1, 1024, 257), (5, 272, 130), (4, 4096, 515), (16, 2080, 97), (17, 512, 64),
          (24, 1344, 201), (32, 640, 300), (33, 640, 333), (64, 2048, 129), (100, 384, 1000), (128, 4096, 300), (130, 736, 259), (256, 256, 520),
          (257, 256, 65), (300, 1040, 777), (2, 8192, 70), (7, 12288, 40), (40, 16384, 36), (515, 400, 513)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f8"])
@pytest.mark.parametrize("B,K,V", SHAPES)
def test_projection_is_exact_on_small_whole_numbers(B, K, V, dtype):
    p = Projection(B, K, V, dtype, whole=True, seed=B + V)
    assert np.array_equal(_np(p.run()), p.want()[0])


@pytest.mark.parametrize("out", ["f32", "same"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f8"])
@pytest.mark.parametrize("B,K,V", SHAPES)
def test_projection_of_real_numbers(B, K, V, dtype, out):
    out = ("bf16" if dtype == "f8" else dtype) if out == "same" else out
    p = Projection(B, K, V, dtype, seed=K + V, pad=B % 3)
    if out == "f16":
        p.scales *= 2.0 ** -6          # (within the type's range)
    want, size = p.want()
    got = _np(p.run(out, stride=V + B % 5, offset=B % 4))
    tol = tolerance(want, size, K, out, p.squares(out))
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,K,V", [(5, 272, 130), (40, 144, 300), (100, 384, 1000), (257, 256, 65), (300, 1040, 777), (700, 512, 300)])
def test_projection_of_states_in_8_bits_with_working_memory(B, K, V, out):
    p = Projection(B, K, V, "f8", whole=True, seed=K, pad=1)
    want = p.want()[0]
    got = p.run(out, with_work=True)
    assert torch.equal(got, p.run(out)) and (out != "f32" or np.array_equal(_np(got), want))


@pytest.mark.parametrize("B,K,V", [(1, 65536, 40), (2, 32768, 20), (16, 10240, 33), (17, 9216, 30), (9, 24576, 70), (33, 65536, 36)])
def test_projection_of_columns_around_what_fits_lds(B, K, V):
    p = Projection(B, K, V, "bf16", whole=True, seed=B)
    p.scales.clamp_(max=0.25)
    assert np.array_equal(_np(p.run()), p.want()[0])


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "f8"])
@pytest.mark.parametrize("B,K,V", [(3, 49152, 130), (16, 16400, 2049), (9, 24576, 300), (17, 9232, 777), (32, 8208, 4100), (30, 16384, 64)])
def test_projection_of_few_rows_and_many_columns(B, K, V, dtype, masked):
    mask, allowed = None, np.ones((B, V), bool)
    if masked:
        allowed = np.random.default_rng(V).random((B, V)) < 0.2
        allowed[:, V // 3:V // 2] = False
        allowed[0, V // 2:] = V % 2 == 0
        mask = torch.from_numpy(plain_logits.pack(allowed)).cuda()
    p = Projection(B, K, V, dtype, whole=True, seed=K, pad=B % 2)
    p.scales.clamp_(max=0.25)
    want = np.where(allowed, p.want()[0], -np.inf)
    for stride, offset in ((V, 0), (V + 4 - V % 4, 0), (V + 3, 1)):
        assert np.array_equal(_np(p.run("f32", mask=mask, stride=stride, offset=offset)), want), stride
    if dtype == "f8":
        assert np.array_equal(_np(p.run("f32", mask=mask, with_work=True)), want)
    p = Projection(B, K, V, dtype, seed=B)
    if dtype == "f16":
        p.scales *= 2.0 ** -6
    want, size = p.want()
    got = _np(p.run("f16" if dtype == "f16" else "bf16", mask=mask, stride=V + 8 - V % 8))
    tol = tolerance(want, size, K, "f16" if dtype == "f16" else "bf16", None)
    assert (got[~allowed] == -np.inf).all() and (np.abs(got - want) <= tol)[allowed].all()


@pytest.mark.parametrize("dtype", ["bf16", "f8"])
@pytest.mark.parametrize("B,K,V", [(1, 1024, 5000), (4, 2080, 3001), (20, 512, 2050), (70, 384, 777), (130, 256, 600), (300, 128, 3000)])
def test_projection_under_masks(B, K, V, dtype):
    rng = np.random.default_rng(B)
    p = Projection(B, K, V, dtype, whole=True, seed=3)
    want, _ = p.want()
    allowed = rng.random((B, V)) < rng.choice([0.0, 0.003, 0.5, 0.97], (B, 1))
    for kind in ("random", "none", "one", "all", "a stretch"):
        if kind != "random":
            allowed[:] = kind == "all"
        if kind == "one":
            allowed[B // 2, V - 1] = True
        if kind == "a stretch":
            allowed[0, V // 3:V // 3 + 40] = True
        mask = torch.from_numpy(plain_logits.pack(allowed)).cuda()
        assert np.array_equal(_np(p.run(mask=mask)), np.where(allowed, want, -np.inf)), kind


@pytest.mark.parametrize("B,K,V", [(1, 256, 1000), (5, 128, 2049), (20, 512, 2050), (70, 384, 777), (130, 256, 600)])
def test_projection_under_masks_of_another_vocabulary(B, K, V):
    p = Projection(B, K, V, "bf16", whole=True, seed=4)
    want, _ = p.want()
    for v_mask in (1, 31, V // 2 + 5, V - 1, V + 1, V + 999):
        allowed = np.random.default_rng(v_mask).random((B, v_mask)) < 0.6
        words = plain_logits.pack(allowed)
        words.view(np.uint32)[:] |= np.where(np.arange(words.shape[1]) == v_mask // 32, np.uint32((0xffffffff << v_mask % 32) & 0xffffffff), np.uint32(0)) if v_mask % 32 else 0
        ok = np.zeros((B, max(V, v_mask)), bool)
        ok[:, :v_mask] = allowed
        got = _np(p.run(mask=torch.from_numpy(words).cuda(), v_mask=v_mask))
        assert np.array_equal(got, np.where(ok[:, :V], want, -np.inf)), v_mask


def test_a_part_of_a_larger_matrix_under_its_masks():
    B, K, V, first = 6, 384, 1000, 256
    p = Projection(B, K, V, "bf16", whole=True, seed=6)
    want, _ = p.want()
    allowed = np.random.default_rng(0).random((B, V)) < 0.4
    mask = torch.from_numpy(plain_logits.pack(allowed)).cuda()
    part = Projection(B, K, V - first, "bf16", whole=True, seed=6)
    part.hidden, part.codes, part.scales = p.hidden, p.codes[first:].contiguous(), p.scales[first // 128:].contiguous()
    got = _np(part.run(mask=mask[:, first // 32:], v_mask=V))
    assert np.array_equal(got, np.where(allowed, want, -np.inf)[:, first:])


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,K,V", [(2000, 128, 1000), (1100, 272, 20001), (40000, 16, 64), (66000 - 465, 32, 17), (129, 512, 30001), (257, 1024, 9000), (48, 640, 70001), (11, 2080, 50001), (16, 1040, 151936), (27, 2080, 50001)])
def test_projection_of_large_batches_and_large_matrices(B, K, V, masked, out):
    p = Projection(B, K, V, "f16", whole=True, seed=V)
    mask, allowed = None, None
    if masked:
        allowed = torch.rand((B, V), generator=torch.Generator().manual_seed(1)) < 0.3
        allowed[:, V // 4:V // 2] = False
        allowed[B // 2:] = False
        mask = torch.from_numpy(plain_logits.pack(allowed.numpy())).cuda()
    got = p.run(out, mask=mask)
    table = torch.from_numpy(plain.e4m3()).float().cuda()
    h = table[torch.from_numpy(p.eight[0]).cuda().int()] * torch.from_numpy(p.eight[1]).float().cuda().repeat_interleave(128, 1)[:, :K]
    w = table[p.codes.int()] * p.scales.repeat_interleave(128, 0)[:V].repeat_interleave(128, 1)[:, :K]
    for b in range(0, B, 8192):          # (exact: whole numbers below 2^24)
        want = h[b:b + 8192] @ w.T
        if masked:
            want.masked_fill_(~allowed[b:b + 8192].cuda(), -float("inf"))
        assert torch.equal(got[b:b + 8192], want.to(got.dtype)), b


def test_projection_of_what_is_not_finite():
    p = Projection(40, 256, 300, "bf16", seed=1)
    p.hidden[3, 5], p.hidden[39, 200] = float("inf"), float("nan")
    p.codes[17, 130], p.codes[299, 0] = 127, 255
    keep = np.ones((40, 300), bool)
    keep[[3, 39]] = False
    keep[:, [17, 299]] = False
    p.eight = plain.quantized(_np(p.hidden)[:, :256])
    table, want = plain.e4m3(), None
    with np.errstate(invalid="ignore"):
        want, size = p.want()
    got = _np(p.run())
    assert np.isnan(got[~keep]).all() and table[127] != table[127]
    assert (np.abs(got - want)[keep] <= tolerance(want, size, 256, "f32")[keep]).all()


def test_projection_of_a_matrix_beyond_2_to_the_31_bytes():
    """Codes, logits and masks whose offsets do not fit 32 bits: 2.4 GB of codes."""
    V, K, B = 589824, 4096, 20
    codes = torch.zeros((V, K), dtype=torch.uint8, device="cuda")
    scales = torch.ones((V // 128, 32), device="cuda")
    rows = torch.tensor([0, 1, 300000, 524287, 524288, 524289, V - 1], device="cuda")
    codes[rows] = torch.randint(0, 120, (len(rows), K), device="cuda", dtype=torch.uint8)
    p = Projection(B, K, 8, "bf16", whole=True)
    p.V, p.codes, p.scales = V, codes, scales
    got = _np(p.run()[:, rows])
    h = plain.e4m3()[p.eight[0]] * np.repeat(p.eight[1], 128, 1)
    w = plain.e4m3()[codes[rows].cpu().numpy()]
    tol = tolerance(h @ w.T, np.abs(h) @ np.abs(w).T, K, "f32")
    assert (np.abs(got - h @ w.T) <= tol).all()


@pytest.mark.parametrize("B,V", [(200, 40000), (1100, 2000)])
def test_logits_beyond_2_to_the_31_bytes_from_the_first(B, V):
    p = Projection(B, 128, V, "bf16", whole=True, seed=2)
    stride = (1 << 31) // B // 4 * 4 + 4096 if B == 200 else V
    got = p.run("bf16", stride=stride)[:, :: 997].float().cpu().numpy()
    assert np.array_equal(got, p.want()[0].astype(np.float32)[:, :: 997].astype(np.float32)) or \
        np.abs(got - p.want()[0][:, :: 997]).max() <= 2.0 ** -8 * np.abs(got).max()


# ------------------------------------------------------------------------------------------------ lookups
def _ids(n, V, seed):
    ids = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    ids[::5] = -1
    ids[n // 2] = V - 1
    if n > 8:
        ids[3], ids[7], ids[8] = V, 2 ** 31 - 1, -2 ** 31
    return ids


def _once(value, out):
    """Numbers in 64 bits rounded to a type, once (torch goes by way of 32 bits: 1 + 2^-11 + 2^-40 would become 1 in f16)."""
    if out == "f32":
        return value.astype(np.float32)
    if out == "f16":
        return value.astype(np.float16).astype(np.float32)
    m, e = np.frexp(value)                                 # (bf16, normal numbers: 8 bits)
    return np.ldexp(np.rint(m * 256), e - 8).astype(np.float32)


def test_the_rounding_above():
    x = np.array([1 + 2.0 ** -11 + 2.0 ** -40, 1 + 2.0 ** -11, 1 + 3 * 2.0 ** -11, -1 - 2.0 ** -11 - 2.0 ** -40])
    assert _once(x, "f16").tolist() == [1 + 2.0 ** -10, 1, 1 + 2.0 ** -9, -1 - 2.0 ** -10]
    x = np.array([1 + 2.0 ** -8 + 2.0 ** -40, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 0.0])
    assert _once(x, "bf16").tolist() == [1 + 2.0 ** -7, 1, 1 + 2.0 ** -6, 0.0]


def _lookup_matches(got, value, factor, out):
    want = _once(value * np.float64(np.float32(factor)), out)
    assert np.array_equal(got.cpu().float().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,K", [(1, 1, 16), (3, 200, 144), (64, 130, 1024), (300, 5000, 2080), (9, 40, 65536)])
def test_rows_of_an_8_bit_matrix(n, V, K, out):
    p = Projection(1, K, V, "f8", seed=n)
    p.codes[-1, K // 2] = 127
    ids, factor, pad = _ids(n, V, n), 0.37, n % 3
    buf = torch.full((n + 1, K + pad), 7.0, dtype=TYPES[out][0], device="cuda")
    _xgm().f8_embed(ids.cuda().data_ptr(), n, p.codes.data_ptr(), p.scales.data_ptr(), V, K, factor, buf.data_ptr(), TYPES[out][1], K + pad, _stream())
    torch.cuda.synchronize()
    assert bool((buf[n] == 7).all()) and bool((buf[:, K:] == 7).all())
    v = ids.numpy().astype(np.int64)
    there = (v >= 0) & (v < V)
    at = np.where(there, v, 0)
    value = plain.e4m3()[p.codes.cpu().numpy()[at]] * np.repeat(p.scales.double().cpu().numpy()[at // 128], 128, 1)[:, :K]
    _lookup_matches(buf[:n, :K], np.where(there[:, None], value, 0.0), factor, out)


@pytest.mark.parametrize("out,low", [("bf16", False), ("f16", False), ("f16", True)])
def test_products_next_to_the_middle_of_two_numbers(out, low):
    """Products that 32 bits would put onto the middle, from either side; low: of numbers below the type's normal ones."""
    V, K, factor = 512, 65536, np.float32(0.37)
    rng = np.random.default_rng(5)
    digits = 256 if out == "bf16" else 1024
    shape = V // 128, K // 128
    middle = (rng.integers(0, 200, shape) + 0.5) * 2.0 ** -24 if low else (digits // 2 + rng.integers(0, digits // 2, shape) + 0.5) * 2.0 ** rng.integers(-12, -6, shape)
    scales = (middle / np.float64(factor)).astype(np.float32)
    product = scales.astype(np.float64) * np.float64(factor)
    assert ((product.astype(np.float32) == middle) & (product < middle)).sum() > 200 and ((product.astype(np.float32) == middle) & (product > middle)).sum() > 200
    some = np.flatnonzero(np.isin(plain.e4m3(), [1, -1, 2, -2, 0.5, 4, 3, 0, -7]))
    codes = torch.from_numpy(some[rng.integers(0, len(some), (V, K))]).to(torch.uint8).cuda()
    ids = torch.arange(0, V, 64, dtype=torch.int32, device="cuda")
    buf = torch.zeros((len(ids), K), dtype=TYPES[out][0], device="cuda")
    on = torch.from_numpy(scales).cuda()
    _xgm().f8_embed(ids.data_ptr(), len(ids), codes.data_ptr(), on.data_ptr(), V, K, float(factor), buf.data_ptr(), TYPES[out][1], K, _stream())
    torch.cuda.synchronize()
    at = ids.cpu().numpy()
    _lookup_matches(buf, plain.e4m3()[codes.cpu().numpy()[at]] * np.repeat(scales.astype(np.float64)[at // 128], 128, 1), factor, out)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scales_dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,V,K,group", [(1, 1, 32, 32), (3, 200, 160, 32), (64, 130, 1024, 128), (300, 5000, 2112, 64), (9, 40, 65536, 65536), (33, 77, 288, 96)])
def test_rows_of_a_4_bit_matrix(n, V, K, group, scales_dtype, out):
    g = torch.Generator().manual_seed(n)
    codes = torch.randint(0, 256, (V, K // 2), generator=g, dtype=torch.uint8)
    scales = (0.01 * torch.exp(torch.randn((V, K // group), generator=g))).to(TYPES[scales_dtype][0])
    zeros = torch.randint(0, 16, (V, K // group), generator=g, dtype=torch.uint8) if n != 3 else None
    ids, factor, pad = _ids(n, V, n), -11.3, n % 3
    buf = torch.full((n + 1, K + pad), 7.0, dtype=TYPES[out][0], device="cuda")
    on = [codes.cuda(), scales.cuda(), None if zeros is None else zeros.cuda(), ids.cuda()]
    _xgm().q4_embed(on[3].data_ptr(), n, on[0].data_ptr(), on[1].data_ptr(), TYPES[scales_dtype][1], _at(on[2]), V, K, group, factor, buf.data_ptr(),
                    TYPES[out][1], K + pad, _stream())
    torch.cuda.synchronize()
    assert bool((buf[n] == 7).all()) and bool((buf[:, K:] == 7).all())
    v = ids.numpy().astype(np.int64)
    there = (v >= 0) & (v < V)
    at = np.where(there, v, 0)
    c = np.empty((n, K))
    c[:, 0::2], c[:, 1::2] = codes.numpy()[at] & 15, codes.numpy()[at] >> 4
    c -= 8.0 if zeros is None else np.repeat(zeros.double().numpy()[at], group, 1)
    _lookup_matches(buf[:n, :K], np.where(there[:, None], c * np.repeat(_np(scales)[at], group, 1), 0.0), factor, out)


def test_a_lookup_of_many_rows_of_a_matrix_beyond_2_to_the_31_bytes():
    V, K, n = 560000, 4096, 600000 // 4096 * 4096
    codes = torch.zeros((V, K), dtype=torch.uint8, device="cuda")
    scales = torch.ones((V // 128, 32), device="cuda")
    codes[V - 1] = 0x38                                                    # 1.0
    codes[524288] = 0x40                                                   # 2.0
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[n - 1], ids[n - 2] = V - 1, 524288
    out = torch.full((n, K), 5.0, dtype=torch.bfloat16, device="cuda")     # (offsets of the output pass 32 bits too)
    _xgm().f8_embed(ids.data_ptr(), n, codes.data_ptr(), scales.data_ptr(), V, K, 1.5, out.data_ptr(), 1, K, _stream())
    torch.cuda.synchronize()
    assert bool((out[n - 1] == 1.5).all()) and bool((out[n - 2] == 3.0).all()) and not bool(out[:n - 2].any())
