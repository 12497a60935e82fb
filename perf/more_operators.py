"""A decode step with an 8-bit matrix and several beams a request, as measurable cases: tokens to hidden states, hidden states to
logits, logits to the beams that go on, and what these beams keep.

  embed    rows of a tied output matrix, in 4 or in 8 bits, as the next hidden states of given tokens
  f8       the output projection with a matrix in 8-bit floating point (e4m3), a scale for each block of 128 x 128; hidden states
           are given in 8 bits with a scale for each 128 columns, or are brought there
  beam     which continuations of a request's beams go on: the best of all beams' tokens by the sum of log-probabilities
  reorder  the caches and texts of the beams that go on move to their rows, in place

A case's fields: `op`; `rows` (requests times `beams`); `vocab` tokens; `k` columns; `dtype` of hidden states, logits or cached values
("f8": hidden states in 8 bits); `out` type of what is made.  Of the masks, `mask`: "none"; "mixed" (five rows of thirteen are inside
a string and allow 96 % of the vocabulary, the others up to `allowed` tokens); "few" (every row up to `allowed` tokens).
beam: `n_out` continuations a request; `first` (only a request's first beam has a text yet).  reorder: a cache [layers, rows, heads,
length, dim] for keys and values each, of which a row has filled between a half and all of `length`; `moved` rows of a request are dropped
and take over another's text.  embed: `bits`, and `group` columns to a scale in 4 bits.

Hidden states in 8 bits: the scale of a block is the smallest power of two 2^e, -126 <= e <= 120, for which no |x| is above
448 * 2^e; values are x / scale, rounded to the nearest, ties to even.
Continuations are in falling order of score + logit - log(sum of exp of the row's logits), taken as logit + (score - log sum); among
equals the lower row comes first, within a row the larger logit, then the lower id.  An ended row has one continuation: itself, with token -1.
Where `n_out` is the number of beams they are placed: the first continuation of a row takes the row's own place, the others in their
order the places that are left, lowest first.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
SIZES = {"f32": 4, "bf16": 2, "f16": 2, "f8": 1}
OPEN = 0.96           # share of the vocabulary that a row inside a string allows
WIDEST = 151936
BLOCK = 128
MOST_PRODUCTS = 1024 * 128256 * 4096
MOST_MOVED = 128 * 4 * 2 * 8 * 1024 * 128


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # ---- output projection in 8 bits
        # a draft model of a toy vocabulary: nothing but latency
        dict(name="f8-toy-1", op="f8", rows=1, vocab=4096, k=1024, dtype="bf16", out="bf16", mask="none", allowed=0),
        # one local user, no grammar: the whole matrix is read for one row
        dict(name="f8-local-1", op="f8", rows=1, vocab=128256, k=4096, dtype="bf16", out="f32", mask="none", allowed=0),
        # six requests of four beams, some inside strings; an odd vocabulary, columns that fill no block
        dict(name="f8-ragged-24", op="f8", rows=24, vocab=50001, k=2080, dtype="f16", out="f32", mask="mixed", allowed=100),
        # the serving batch, of which some requests have no grammar
        dict(name="f8-serving-128", op="f8", rows=128, vocab=151936, k=4096, dtype="bf16", out="bf16", mask="none", allowed=0),
        # log-probabilities of a given text's tokens, hidden states brought to 8 bits by the norm in front
        dict(name="f8-scoring-1024", op="f8", rows=1024, vocab=128256, k=4096, dtype="f8", out="bf16", mask="none", allowed=0),
        # ---- continuations of beams
        # one user's first step
        dict(name="beam-local-4", op="beam", rows=4, beams=4, vocab=32000, dtype="bf16", out="f32", mask="none", allowed=0, n_out=4, first=True),
        # seven requests of three beams, twice as many continuations for a program that ends texts by itself; an odd vocabulary, unpadded rows
        dict(name="beam-ragged-21", op="beam", rows=21, beams=3, vocab=50001, dtype="f32", out="f32", mask="mixed", allowed=400, n_out=6,
             first=False),
        # a serving batch of eight beams
        dict(name="beam-serving-128", op="beam", rows=128, beams=8, vocab=151936, dtype="bf16", out="f32", mask="mixed", allowed=400, n_out=8,
             first=False),
        # ---- what the beams keep
        # one user's beams on a small model, a short text
        dict(name="reorder-local-4", op="reorder", rows=4, beams=4, layers=4, heads=4, length=256, dim=64, dtype="bf16", moved=2),
        # a serving batch, four layers at a time
        dict(name="reorder-serving-128", op="reorder", rows=128, beams=8, layers=4, heads=8, length=1024, dim=128, dtype="bf16", moved=3),
        # ---- tokens to hidden states
        # the tokens of a decode step
        dict(name="embed-step-128", op="embed", rows=128, vocab=151936, k=4096, bits=4, group=128, dtype="bf16", out="bf16"),
        # prompts, all requests' tokens one behind the other
        dict(name="embed-prompt-16384", op="embed", rows=16384, vocab=128256, k=4096, bits=8, group=128, dtype="f8", out="bf16"),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["f8", "f8", "beam", "beam", "reorder", "embed"])
    vocab = _spread(rng, 1024, WIDEST)
    mask = rng.choice(["none", "mixed", "few"])
    allowed = 0 if mask == "none" else _spread(rng, 1, 1000)
    if op == "f8":
        k = rng.choice([1024, 2048, 4096, 16 * (_spread(rng, 16, 256) | 1)])     # a usual one, or one that ends inside a block
        rows = min(_spread(rng, 1, 1024), MOST_PRODUCTS // (vocab * k))
        dtype = rng.choice(["bf16", "f16", "f8"])
        return dict(op=op, rows=rows, vocab=vocab, k=k, dtype=dtype, out=rng.choice(["f32", "bf16" if dtype == "f8" else dtype]), mask=mask,
                    allowed=allowed)
    if op == "beam":
        beams = _spread(rng, 1, 32)
        rows = beams * _spread(rng, 1, 128 // beams)
        return dict(op=op, rows=rows, beams=beams, vocab=vocab, dtype=rng.choice(["bf16", "f16", "f32"]), out="f32", mask=mask, allowed=allowed,
                    n_out=rng.choice([beams, 2 * beams]), first=rng.random() < 0.2)
    if op == "reorder":
        beams = _spread(rng, 2, 32)
        rows = beams * _spread(rng, 1, 128 // beams)
        c = dict(op=op, rows=rows, beams=beams, layers=rng.choice([1, 2, 4]), heads=_spread(rng, 1, 8), length=_spread(rng, 16, 4096),
                 dim=rng.choice([64, 80, 128]), dtype=rng.choice(["bf16", "f32"]), moved=rng.randint(1, max(1, beams // 2)))
        c["length"] = min(c["length"], MOST_MOVED // (rows * 2 * c["layers"] * c["heads"] * c["dim"]) * 2 // SIZES[c["dtype"]])
        return c
    bits = rng.choice([4, 8])
    group = rng.choice([32, 64, 128]) if bits == 4 else BLOCK
    k = rng.choice([1024, 2048, 4096, 16 * (_spread(rng, 16, 256) | 1) if bits == 8 else group * (_spread(rng, 256 // group, 4000 // group) | 1)])
    return dict(op=op, rows=_spread(rng, 1, 16384), vocab=vocab, k=k, bits=bits, group=group, dtype=rng.choice(["bf16", "f16"]) if bits == 4 else "f8",
                out=rng.choice(["bf16", "f16", "f32"]))


# ------------------------------------------------------------------------------------------------ inputs
def _words(vocab):
    return (vocab + 31) // 32


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _open(b):
    """Whether row b of a mixed batch is inside a string."""
    return b * 5 % 13 < 5


def _pack(allowed):
    """Truth values [rows, vocab] as mask words: token i is bit i % 32 of word i // 32."""
    rows, vocab = allowed.shape
    out = torch.empty((rows, _words(vocab)), dtype=torch.int32, device=allowed.device)
    for b in range(0, rows, 128):
        part = allowed[b:b + 128]
        bits = torch.zeros((part.shape[0], _words(vocab) * 32), dtype=torch.int64, device=allowed.device)
        bits[:, :vocab] = part
        words = (bits.view(part.shape[0], -1, 32) << torch.arange(32, device=allowed.device)).sum(-1)
        out[b:b + 128] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return out


def _mask(case, gen):
    rows, vocab = case["rows"], case["vocab"]
    if case["mask"] == "none":
        return None
    allowed = torch.zeros((rows, vocab), dtype=torch.bool, device="cuda")
    allowed.scatter_(1, torch.randint(0, vocab, (rows, max(1, case["allowed"])), generator=gen, device="cuda"), True)
    if case["mask"] == "mixed":
        for b in range(rows):
            if _open(b):
                allowed[b] = torch.rand(vocab, generator=gen, device="cuda") < OPEN
    return _pack(allowed)


def _f8_matrix(case, gen):
    """Codes [vocab, k] and scales of their blocks, as a program loads them."""
    vocab, k = case["vocab"], case["k"]
    codes = torch.empty((vocab, k), dtype=torch.uint8, device="cuda")
    for v in range(0, vocab, 32768):
        part = codes[v:v + 32768]
        part.copy_((110.0 * torch.randn(part.shape, generator=gen, device="cuda")).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    scales = 2e-4 * torch.exp(0.3 * torch.randn((_blocks(vocab), _blocks(k)), generator=gen, device="cuda"))
    return dict(codes=codes, scales=scales)


def _f8_inputs(case, gen):
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    s = _f8_matrix(case, gen)
    hidden = torch.randn((rows, k), generator=gen, device="cuda")              # behind a norm, some columns larger than others
    hidden *= torch.exp(0.5 * torch.randn((k,), generator=gen, device="cuda"))
    if case["dtype"] == "f8":
        s["hidden_scales"] = 0.01 * torch.exp(0.2 * torch.randn((rows, _blocks(k)), generator=gen, device="cuda"))     # not powers of two
        wide = s["hidden_scales"].repeat_interleave(BLOCK, 1)[:, :k]
        s["hidden"] = (hidden / wide).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        s |= dict(hidden=hidden.to(TYPES[case["dtype"]]), hidden_scales=None)
    return s | dict(bitmask=_mask(case, gen), logits=torch.empty((rows, vocab), dtype=TYPES[case["out"]], device="cuda"))


def _beam_inputs(case, gen):
    rows, vocab, beams = case["rows"], case["vocab"], case["beams"]
    logits = 2.0 * torch.randn((rows, vocab), generator=gen, device="cuda")
    likely = torch.randint(0, vocab, (rows, 24), generator=gen, device="cuda")
    logits.scatter_reduce_(1, likely, 4.0 + 3.0 * torch.randn((rows, 24), generator=gen, device="cuda").abs(), "amax")
    scores = -8.0 - 2.0 * torch.rand((rows,), generator=gen, device="cuda")       # beams of a request are close to each other
    ended = torch.zeros((rows,), dtype=torch.int32, device="cuda")
    if case["first"]:
        scores.view(-1, beams)[:, 1:] = -math.inf
        scores.view(-1, beams)[:, 0] = 0.0
    elif rows > 6:
        ended[torch.randint(0, rows, (rows // 7,), generator=gen, device="cuda")] = 1
    shape = (rows // beams, case["n_out"])
    return dict(logits=logits.to(TYPES[case["dtype"]]), bitmask=_mask(case, gen), scores=scores, ended=ended,
                next_rows=torch.empty(shape, dtype=torch.int32, device="cuda"), ids=torch.empty(shape, dtype=torch.int32, device="cuda"),
                next_scores=torch.empty(shape, dtype=torch.float32, device="cuda"))


def _reorder_inputs(case, gen):
    rows, beams, length = case["rows"], case["beams"], case["length"]
    shape = (case["layers"], rows, case["heads"], length, case["dim"])
    keys, values = (torch.randint(-8192, 8192, shape, generator=gen, device="cuda", dtype=torch.int16).to(TYPES[case["dtype"]]) for _ in range(2))
    # of each request some rows are dropped, and take over the text of one that stays
    order = torch.rand((rows // beams, beams), generator=gen, device="cuda").argsort(1)
    gone, stay = order[:, :case["moved"]], order[:, case["moved"]:]
    source = torch.arange(beams, device="cuda").repeat(rows // beams, 1)
    picks = torch.randint(0, beams - case["moved"], gone.shape, generator=gen, device="cuda")
    source.scatter_(1, gone, stay.gather(1, picks))
    source += torch.arange(0, rows, beams, device="cuda")[:, None]
    used = torch.randint((length + 1) // 2, length + 1, (rows // beams,), generator=gen, device="cuda", dtype=torch.int32).repeat_interleave(beams)
    return dict(keys=keys, values=values, tokens=torch.randint(0, WIDEST, (rows, length), generator=gen, device="cuda", dtype=torch.int32),
                source=source.reshape(-1).int(), used=used)


def _embed_inputs(case, gen):
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    if case["bits"] == 8:
        s = _f8_matrix(case, gen)
    else:
        t = TYPES[case["dtype"]]
        s = dict(codes=torch.randint(0, 256, (vocab, k // 2), generator=gen, device="cuda", dtype=torch.uint8),
                 scales=(0.01 * torch.exp(0.3 * torch.randn((vocab, k // case["group"]), generator=gen, device="cuda"))).to(t),
                 zeros=torch.randint(0, 16, (vocab, k // case["group"]), generator=gen, device="cuda", dtype=torch.uint8))
    usual = torch.rand((rows,), generator=gen, device="cuda") ** 4      # few tokens make up most of a text
    ids = (usual * vocab).to(torch.int32).clamp_(max=vocab - 1)
    ids[::11] = torch.where(torch.rand((ids[::11].numel(),), generator=gen, device="cuda") < 0.5, -1, ids[::11])     # rows that have ended
    return s | dict(ids=ids, factor=math.sqrt(k), hidden=torch.empty((rows, k), dtype=TYPES[case["out"]], device="cuda"))


def _address(t):
    return 0 if t is None else t.data_ptr()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"f8": _f8_inputs, "beam": _beam_inputs, "reorder": _reorder_inputs, "embed": _embed_inputs}[case["op"]](case, gen)
    s["case"] = dict(case)
    if own:      # a program keeps these from step to step: addresses of its arrays, working memory
        import paper_2411_15100_amd as xgm
        if case["op"] == "f8":
            s["work"] = torch.empty((xgm.f8_work_bytes(case["rows"], case["k"]),), dtype=torch.uint8, device="cuda")
        if case["op"] == "beam":
            s["rules"] = xgm.LogitRules(d_bitmask=_address(s["bitmask"]), v_mask=case["vocab"])
            s["search"] = xgm.BeamSearch(case["rows"], case["vocab"], torch.cuda.current_stream().cuda_stream)
        if case["op"] == "reorder":
            e = SIZES[case["dtype"]]
            a_position, a_head, a_row = case["dim"] * e, case["length"] * case["dim"] * e, case["heads"] * case["length"] * case["dim"] * e
            cache = [xgm.RowData(d_data=t.data_ptr(), row_stride=a_row, n_outer=case["layers"], outer_stride=a_row * case["rows"],
                                 n_parts=case["heads"], part_stride=a_head, part_bytes=a_head, d_used=s["used"].data_ptr(), used_bytes=a_position)
                     for t in (s["keys"], s["values"])]
            text = xgm.RowData(d_data=s["tokens"].data_ptr(), row_stride=4 * case["length"], n_outer=1, n_parts=1, part_bytes=4 * case["length"],
                               d_used=s["used"].data_ptr(), used_bytes=4)
            s["kept"] = xgm.RowSet(*cache, text)
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls
def _run_own(s):
    import paper_2411_15100_amd as xgm
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    code = {"f32": xgm.DTYPE_F32, "bf16": xgm.DTYPE_BF16, "f16": xgm.DTYPE_F16, "f8": xgm.DTYPE_F8}
    rows = case["rows"]
    if case["op"] == "f8":
        vocab, k = case["vocab"], case["k"]
        xgm.f8_logits(s["hidden"].data_ptr(), code[case["dtype"]], _address(s["hidden_scales"]), rows, k, k, s["codes"].data_ptr(),
                      s["scales"].data_ptr(), vocab, s["logits"].data_ptr(), code[case["out"]], vocab, _address(s["bitmask"]),
                      s["work"].data_ptr(), stream)
        return s["logits"]
    if case["op"] == "beam":
        s["search"].select(s["logits"].data_ptr(), code[case["dtype"]], rows // case["beams"], case["beams"], case["vocab"], case["vocab"], s["rules"],
                           s["scores"].data_ptr(), s["ended"].data_ptr(), case["n_out"], case["n_out"] == case["beams"], s["next_rows"].data_ptr(),
                           s["ids"].data_ptr(), s["next_scores"].data_ptr(), stream)
        return s["next_rows"], s["ids"], s["next_scores"]
    if case["op"] == "reorder":
        xgm.reorder_rows(s["kept"], s["source"].data_ptr(), rows, stream)
        return s["keys"], s["values"], s["tokens"]
    if case["bits"] == 8:
        xgm.f8_embed(s["ids"].data_ptr(), rows, s["codes"].data_ptr(), s["scales"].data_ptr(), case["vocab"], case["k"], s["factor"],
                     s["hidden"].data_ptr(), code[case["out"]], case["k"], stream)
    else:
        xgm.q4_embed(s["ids"].data_ptr(), rows, s["codes"].data_ptr(), s["scales"].data_ptr(), code[case["dtype"]], s["zeros"].data_ptr(),
                     case["vocab"], case["k"], case["group"], s["factor"], s["hidden"].data_ptr(), code[case["out"]], case["k"], stream)
    return s["hidden"]


# ------------------------------------------------------------------------------------------------ the plain forms
def _allowed(words, vocab):
    bits = words[:, :, None] >> torch.arange(32, dtype=torch.int32, device=words.device) & 1
    return bits.view(words.shape[0], -1)[:, :vocab].bool()


def _to_blocks(x):
    """[rows, k] as [rows, blocks, 128], zeros behind the last column."""
    rows, k = x.shape
    y = torch.zeros((rows, _blocks(k) * BLOCK), dtype=x.dtype, device=x.device)
    y[:, :k] = x
    return y.view(rows, -1, BLOCK)


def _plain_f8(s):
    case = s["case"]
    vocab, k = case["vocab"], case["k"]
    if case["dtype"] == "f8":
        h = _to_blocks(s["hidden"].view(torch.float8_e4m3fn).float()) * s["hidden_scales"][:, :, None]
    else:
        x = _to_blocks(s["hidden"].float())
        part, e = torch.frexp(x.abs().amax(2, keepdim=True))
        e = torch.where(part <= 0.875, e - 9, e - 8).clamp(-126, 120)          # 448 is 0.875 * 2^9
        h = torch.ldexp(torch.ldexp(x, -e).to(torch.float8_e4m3fn).float(), e)
    w = _to_blocks(s["codes"].view(torch.float8_e4m3fn).float())
    w *= s["scales"].repeat_interleave(BLOCK, 0)[:vocab, :, None]
    y = h.view(h.shape[0], -1) @ w.view(vocab, -1).T
    if s["bitmask"] is not None:
        y.masked_fill_(~_allowed(s["bitmask"], vocab), -math.inf)
    return y.to(TYPES[case["out"]])


def _plain_beam(s):
    """In 64 bits: which of two near sums is larger decides a beam."""
    case = s["case"]
    rows, beams, n_out, vocab = case["rows"], case["beams"], case["n_out"], case["vocab"]
    y = s["logits"].double()
    if s["bitmask"] is not None:
        y = y.masked_fill(~_allowed(s["bitmask"], vocab), -math.inf)
    n = min(n_out, vocab)
    best, ids = torch.sort(y, dim=1, descending=True, stable=True)
    best, ids = best[:, :n], ids[:, :n]
    top = y.amax(1, keepdim=True).clamp(min=-1e300)
    base = s["scores"].double()[:, None] - (top + (y - top).exp().sum(1, keepdim=True).log())
    total = torch.where(best > -math.inf, best + base, -math.inf)
    ended = s["ended"][:, None] != 0
    first = torch.arange(n, device="cuda") == 0
    total = torch.where(ended, torch.where(first, s["scores"].double()[:, None], -math.inf), total)
    total = torch.where(s["scores"][:, None] > -math.inf, total, -math.inf)
    ids = torch.where(ended, -1, ids)
    row = torch.arange(rows, device="cuda")[:, None].expand(rows, n)
    total, at = torch.sort(total.view(-1, beams * n), dim=1, descending=True, stable=True)
    m = min(n_out, beams * n)
    there = total[:, :m] > -math.inf
    out = [torch.full((rows // beams, n_out), v, dtype=t, device="cuda") for v, t in ((-1, torch.int32), (-1, torch.int32), (-math.inf, torch.float32))]
    out[0][:, :m] = torch.where(there, row.reshape(-1, beams * n).gather(1, at[:, :m]), -1).int()
    out[1][:, :m] = torch.where(there, ids.reshape(-1, beams * n).gather(1, at[:, :m]), -1).int()
    out[2][:, :m] = torch.where(there, total[:, :m], -math.inf).float()
    if n_out != beams:
        return tuple(out)
    # placed: the first continuation of a row in the row's own place, the others where places are left
    place = torch.arange(beams, device="cuda").expand(rows // beams, beams)
    parent = torch.where(out[0] >= 0, out[0] - torch.arange(0, rows, beams, device="cuda")[:, None], -1)
    same = parent[:, :, None] == parent[:, None, :]
    is_first = (parent >= 0) & ~(same & (place[:, None, :] < place[:, :, None])).any(2)
    taken = torch.zeros((rows // beams, beams + 1), dtype=torch.bool, device="cuda")
    taken.scatter_(1, torch.where(is_first, parent, beams).long(), True)
    left = torch.sort(taken[:, :beams].int(), dim=1, stable=True).indices           # free places first, in order
    number = (~is_first).int().cumsum(1) - 1
    to = torch.where(is_first, parent, left.gather(1, number.clamp(min=0).long())).long()
    return tuple(torch.empty_like(t).scatter_(1, to, t) for t in out)


def _plain_reorder(s):
    at = torch.arange(s["case"]["length"], device="cuda")
    source = s["source"].long()
    there = at < s["used"].long()[source][:, None]
    outs = [torch.where(there[None, :, None, :, None], t[:, source], t) for t in (s["keys"], s["values"])]
    return outs[0], outs[1], torch.where(there, s["tokens"][source], s["tokens"])


def _plain_embed(s):
    case = s["case"]
    there = (s["ids"] >= 0)[:, None]
    ids = s["ids"].clamp(min=0).long()
    if case["bits"] == 8:
        scales = s["scales"][ids // BLOCK].repeat_interleave(BLOCK, 1)[:, :case["k"]]
        y = s["codes"][ids].view(torch.float8_e4m3fn).float() * scales
    else:
        codes = s["codes"][ids]
        y = torch.stack([codes & 15, codes >> 4], -1).view(len(ids), -1, case["group"]).float() - s["zeros"][ids].float()[:, :, None]
        y = (y * s["scales"][ids].float()[:, :, None]).view(len(ids), -1)
    return torch.where(there, y * s["factor"], 0.0).to(TYPES[case["out"]])


def run(state):
    if own:
        return _run_own(state)
    return {"f8": _plain_f8, "beam": _plain_beam, "reorder": _plain_reorder, "embed": _plain_embed}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _allowed_rows(case):
    """Allowed tokens of all rows together, and how many different ones."""
    rows, vocab = case["rows"], case["vocab"]
    shares = [1.0 if case["mask"] == "none" else OPEN if case["mask"] == "mixed" and _open(b) else 1.0 - (1.0 - 1.0 / vocab) ** case["allowed"]
              for b in range(rows)]
    return vocab * sum(shares), vocab * (1.0 - math.prod(1.0 - x for x in shares))


def work(case):
    rows = case["rows"]
    if case["op"] == "reorder":
        moved = rows // case["beams"] * case["moved"] * 0.75 * case["length"]          # positions of rows that move
        each = 2 * case["layers"] * case["heads"] * case["dim"] * SIZES[case["dtype"]] + 4
        return {"bytes": 2.0 * moved * each + 8 * rows, "flops": 0.0}
    vocab, out = case["vocab"], SIZES[case["out"]]
    if case["op"] == "embed":
        edge = np.linspace(0.0, 1.0, vocab + 1) ** 0.25
        different = float((1.0 - (1.0 - np.diff(edge)) ** (0.95 * rows)).sum())
        a_row = case["k"] if case["bits"] == 8 else case["k"] / 2 + 3 * case["k"] / case["group"]
        return {"bytes": different * a_row + rows * (4 + case["k"] * out), "flops": 2.0 * rows * case["k"]}
    pairs, tokens = _allowed_rows(case)
    mask = 0 if case["mask"] == "none" else 4 * rows * _words(vocab)
    if case["op"] == "f8":
        k, e = case["k"], SIZES[case["dtype"]]
        return {"bytes": tokens * (k + 4 * _blocks(k) / BLOCK) + rows * k * e + mask + rows * vocab * out, "flops": 2.0 * pairs * k}
    live = 1.0 / case["beams"] if case["first"] else 1.0
    return {"bytes": live * (pairs * SIZES[case["dtype"]] + mask) + rows * 8 + rows // case["beams"] * case["n_out"] * 12, "flops": 15.0 * live * pairs}


# ------------------------------------------------------------------------------------------------ the definitions, in 64 bits
def _bits(words, vocab):
    return np.unpackbits(words.view(np.uint8), bitorder="little")[:vocab].astype(bool)


def _e4m3_values():
    """The value of each of the 256 codes."""
    out = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = math.nan if c & 127 == 127 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[c] = -x if c & 128 else x
    return out


def _exact_states(x):
    """Hidden states as what they stand for in 8 bits, by the definition."""
    x = x.double().cpu().numpy()
    values = np.sort(_e4m3_values()[:127])       # 0 .. 448
    middles = (values[1:] + values[:-1]) / 2
    out = np.empty_like(x)
    for k in range(0, x.shape[1], BLOCK):
        part = x[:, k:k + BLOCK]
        most = np.abs(part).max(1)
        with np.errstate(divide="ignore"):
            e = np.clip(np.ceil(np.log2(most / 448.0)), -126, 120)
        scale = 2.0 ** np.where(most > 448.0 * 2.0 ** e, e + 1, np.where((most <= 448.0 * 2.0 ** (e - 1)) & (e > -126), e - 1, e))
        size = np.abs(part) / scale[:, None]
        at = np.searchsorted(middles, size, side="left")          # below or at a middle: the lower one
        tie = (at < 126) & (middles[np.minimum(at, 125)] == size) & (at % 2 == 1)     # an odd code is not even
        out[:, k:k + BLOCK] = np.copysign(values[at + tie], part) * scale[:, None]
    return torch.from_numpy(out).cuda()


def _exact_f8(s):
    case = s["case"]
    vocab, k = case["vocab"], case["k"]
    table = torch.from_numpy(_e4m3_values()).cuda()
    column = torch.arange(k, device="cuda") // BLOCK
    if case["dtype"] == "f8":
        h = table[s["hidden"].long()] * s["hidden_scales"].double()[:, column]
    else:
        h = _exact_states(s["hidden"])
    out = torch.empty((case["rows"], vocab), dtype=torch.float64, device="cuda")
    for v in range(0, vocab, 16384):
        part = slice(v, min(v + 16384, vocab))
        rows = torch.arange(part.start, part.stop, device="cuda") // BLOCK
        w = table[s["codes"][part].int()] * s["scales"].double()[rows][:, column]
        out[:, part] = (w @ h.T).T
    if s["bitmask"] is not None:
        for b, words in enumerate(s["bitmask"].cpu().numpy()):
            out[b, torch.from_numpy(~_bits(words, vocab)).cuda()] = -math.inf
    return out


def _exact_beam(s):
    case = s["case"]
    beams, n_out, vocab = case["beams"], case["n_out"], case["vocab"]
    logits, scores, ended = s["logits"].float().cpu().numpy(), s["scores"].cpu().numpy(), s["ended"].cpu().numpy()
    masks = None if s["bitmask"] is None else s["bitmask"].cpu().numpy()
    rows_out, ids_out, scores_out = [], [], []
    for r in range(case["rows"] // beams):
        found = []
        for b in range(r * beams, (r + 1) * beams):
            if not scores[b] > -np.inf:
                continue
            if ended[b]:
                found.append((-float(scores[b]), b, 0.0, -1))
                continue
            y = logits[b].astype(np.float64)
            if masks is not None:
                y[~_bits(masks[b], vocab)] = -np.inf
            top = y.max()
            if top == -np.inf:
                continue
            base = np.float64(scores[b]) - (top + np.log(np.exp(y - top).sum()))
            n = min(n_out, vocab)
            least = np.partition(y, vocab - n)[vocab - n]
            there = np.flatnonzero((y >= least) & (y > -np.inf))
            there = there[np.lexsort((there, -y[there]))][:n]
            found += [(-(y[v] + base), b, -y[v], int(v)) for v in there]
        found = sorted(found)[:n_out]
        got = [(b, v, -minus) for minus, b, _, v in found] + [(-1, -1, -math.inf)] * (n_out - len(found))
        if n_out == beams:
            placed, others = {}, []
            for g in got:
                if g[0] >= 0 and g[0] - r * beams not in placed:
                    placed[g[0] - r * beams] = g
                else:
                    others.append(g)
            got = [placed[i] if i in placed else others.pop(0) for i in range(beams)]
        for out, i in ((rows_out, 0), (ids_out, 1), (scores_out, 2)):
            out.append([g[i] for g in got])
    return torch.tensor(rows_out, dtype=torch.int32), torch.tensor(ids_out, dtype=torch.int32), torch.tensor(scores_out, dtype=torch.float64)


def _exact_reorder(s):
    case = s["case"]
    source, used = s["source"].tolist(), s["used"].tolist()
    keys, values, tokens = s["keys"].clone(), s["values"].clone(), s["tokens"].clone()
    for b, a in enumerate(source):
        n = used[a]
        if a != b:
            keys[:, b, :, :n], values[:, b, :, :n], tokens[b, :n] = s["keys"][:, a, :, :n], s["values"][:, a, :, :n], s["tokens"][a, :n]
    return keys.double(), values.double(), tokens


def _exact_embed(s):
    case = s["case"]
    k = case["k"]
    out = torch.zeros((case["rows"], k), dtype=torch.float64, device="cuda")
    at = torch.nonzero(s["ids"] >= 0)[:, 0]
    ids = s["ids"][at].long()
    if case["bits"] == 8:
        y = torch.from_numpy(_e4m3_values()).cuda()[s["codes"][ids].int()]
        y *= s["scales"].double()[ids // BLOCK][:, torch.arange(k, device="cuda") // BLOCK]
    else:
        group = torch.arange(k, device="cuda") // case["group"]
        y = torch.empty((len(ids), k), dtype=torch.float64, device="cuda")
        y[:, 0::2], y[:, 1::2] = s["codes"][ids].remainder(16).double(), s["codes"][ids].div(16, rounding_mode="floor").double()
        y = (y - s["zeros"][ids].double()[:, group]) * s["scales"][ids].double()[:, group]
    out[at] = y * s["factor"]
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"f8": _exact_f8, "beam": _exact_beam, "reorder": _exact_reorder, "embed": _exact_embed}[case["op"]](s)
