"""The end of a decode step, as measurable cases: what lies between the last hidden state and the token that a grammar accepts.

  head    the output projection with 4-bit weights, under the masks of the grammars: logits from hidden states
  rules   penalties for repeated tokens, biases and masks on logits, as a pass of its own
  draw    one token a row from logits: the same rules, temperature, top-k, top-p, min-p and a draw

A case's fields: `op`; `rows` requests; `vocab` tokens; `dtype` of hidden states or logits.  Of the masks, `mask`:
"none"; "mixed" (a serving batch: five rows of thirteen are inside a string and allow 96 % of the vocabulary, the others
up to `allowed` tokens); "few" (every row at a structural place: `allowed` tokens).  `k` columns, `group` columns to a scale,
`zeros` (zero points, or the middle of the range), `out` type of the logits made by head.  `history`: tokens that the longest
row has behind it; `bias`: biased tokens a row.  `top_k` (0: off), `top_p` (1: off), `min_p` (0: off).

Rows have their own lengths, penalties and temperatures; the seed decides them.  In larger batches a row has no history
yet, and a draw has rows that take the likeliest token (temperature 0).
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
OPEN = 0.96           # share of the vocabulary that a row inside a string allows
WIDEST = 151936


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # ---- output projection
        # a draft model of a toy vocabulary: nothing but latency
        dict(name="head-toy-1", op="head", rows=1, vocab=4096, k=1024, group=32, zeros=False, dtype="bf16", out="bf16", mask="none",
             allowed=0),
        # one local user, no grammar: the whole matrix is read for one row
        dict(name="head-local-1", op="head", rows=1, vocab=128256, k=4096, group=128, zeros=False, dtype="bf16", out="f32", mask="none",
             allowed=0),
        # a few requests at brackets, commas and keys: hardly any row of the matrix is wanted
        dict(name="head-structure-4", op="head", rows=4, vocab=151936, k=4096, group=128, zeros=True, dtype="f16", out="f16", mask="few",
             allowed=400),
        # beams over an odd vocabulary, columns that fill no tile, small groups
        dict(name="head-ragged-24", op="head", rows=24, vocab=50001, k=2080, group=32, zeros=True, dtype="f16", out="f32", mask="mixed",
             allowed=100),
        # the serving batch, of which some requests have no grammar
        dict(name="head-serving-128", op="head", rows=128, vocab=151936, k=4096, group=128, zeros=False, dtype="bf16", out="bf16",
             mask="none", allowed=0),
        # ---- rules as a pass of their own
        # one user of a small vocabulary
        dict(name="rules-local-1", op="rules", rows=1, vocab=32000, dtype="bf16", mask="none", allowed=0, history=512, bias=0),
        # long texts, many biases, an odd vocabulary with unpadded rows
        dict(name="rules-ragged-23", op="rules", rows=23, vocab=50001, dtype="f32", mask="none", allowed=0, history=8000, bias=200),
        # the serving batch
        dict(name="rules-serving-128", op="rules", rows=128, vocab=151936, dtype="bf16", mask="mixed", allowed=400, history=2048, bias=16),
        # ---- draws
        # one local user with the usual settings, free text
        dict(name="draw-local-1", op="draw", rows=1, vocab=151936, dtype="bf16", mask="none", allowed=0, history=512, bias=0, top_k=50,
             top_p=0.95, min_p=0.0),
        # rollouts for training: the whole distribution, nothing cut off, no rule
        dict(name="draw-rollout-48", op="draw", rows=48, vocab=128256, dtype="bf16", mask="none", allowed=0, history=0, bias=0, top_k=0,
             top_p=1.0, min_p=0.0),
        # every setting at once on logits in 32 bits, an odd vocabulary with unpadded rows
        dict(name="draw-ragged-16", op="draw", rows=16, vocab=100003, dtype="f32", mask="none", allowed=0, history=3000, bias=100,
             top_k=1000, top_p=0.9, min_p=0.02),
        # the serving batch
        dict(name="draw-serving-128", op="draw", rows=128, vocab=151936, dtype="bf16", mask="mixed", allowed=400, history=1024, bias=0,
             top_k=0, top_p=0.9, min_p=0.0),
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["head", "rules", "draw"])
    rows, vocab = _spread(rng, 1, 128), _spread(rng, 1024, WIDEST)
    mask = rng.choice(["none", "mixed", "few"])
    c = dict(op=op, rows=rows, vocab=vocab, dtype=rng.choice(["bf16", "f16"] if op == "head" else ["bf16", "f16", "f32"]), mask=mask,
             allowed=0 if mask == "none" else _spread(rng, 1, 1000))
    if op == "head":
        group = rng.choice([32, 64, 128])
        k = rng.choice([1024, 2048, 4096, group * (_spread(rng, 256 // group, 4000 // group) | 1)])     # a usual one, or one that fills no tile
        c |= dict(k=k, group=group, zeros=rng.random() < 0.5, out=rng.choice(["f32", c["dtype"]]))
        return c
    c |= dict(history=rng.choice([0, _spread(rng, 16, 8192)]), bias=rng.choice([0, _spread(rng, 1, 300)]))
    if op == "draw":
        c |= dict(top_k=rng.choice([0, _spread(rng, 1, 1000)]), top_p=rng.choice([1.0, round(rng.uniform(0.5, 0.99), 3)]),
                  min_p=rng.choice([0.0, 0.05]))
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _words(vocab):
    return (vocab + 31) // 32


def _open(b):
    """Whether row b of a mixed batch is inside a string."""
    return b * 5 % 13 < 5


def _pack(allowed):
    """Truth values [rows, vocab] as mask words: token i is bit i % 32 of word i // 32."""
    rows, vocab = allowed.shape
    bits = torch.zeros((rows, _words(vocab) * 32), dtype=torch.int64, device=allowed.device)
    bits[:, :vocab] = allowed
    words = (bits.view(rows, -1, 32) << torch.arange(32, device=allowed.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _mask(case, gen):
    rows, vocab = case["rows"], case["vocab"]
    if case["mask"] == "none":
        return None
    dice = torch.rand((rows, vocab), generator=gen, device="cuda")
    few = torch.zeros((rows, vocab), dtype=torch.bool, device="cuda")
    few.scatter_(1, torch.randint(0, vocab, (rows, max(1, case["allowed"])), generator=gen, device="cuda"), True)
    if case["mask"] == "mixed":
        inside = torch.tensor([_open(b) for b in range(rows)], device="cuda")
        few = torch.where(inside[:, None], dice < OPEN, few)
    return _pack(few)


def _head_inputs(case, gen):
    rows, vocab, k, group, t = case["rows"], case["vocab"], case["k"], case["group"], TYPES[case["dtype"]]
    s = dict(
        hidden=torch.randn((rows, k), generator=gen, device="cuda").to(t),     # behind a norm
        codes=torch.randint(0, 256, (vocab, k // 2), generator=gen, device="cuda", dtype=torch.uint8),
        scales=(0.01 * torch.exp(0.3 * torch.randn((vocab, k // group), generator=gen, device="cuda"))).to(t),
        zeros=torch.randint(0, 16, (vocab, k // group), generator=gen, device="cuda", dtype=torch.uint8) if case["zeros"] else None,
        bitmask=_mask(case, gen))
    s["logits"] = torch.empty((rows, vocab), dtype=TYPES[case["out"]], device="cuda")
    return s


def _rule_inputs(case, gen):
    rows, vocab, t = case["rows"], case["vocab"], TYPES[case["dtype"]]
    logits = 2.0 * torch.randn((rows, vocab), generator=gen, device="cuda")
    likely = torch.randint(0, vocab, (rows, 24), generator=gen, device="cuda")
    logits.scatter_reduce_(1, likely, 4.0 + 3.0 * torch.randn((rows, 24), generator=gen, device="cuda").abs(), "amax")
    s = dict(logits=logits.to(t), bitmask=_mask(case, gen), tokens=None, bias_ids=None)
    if case["history"]:
        n = torch.randint(max(1, case["history"] // 4), case["history"] + 1, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        n[0] = case["history"]
        if rows > 3:
            n[2] = 0
        usual = torch.rand((rows, case["history"]), generator=gen, device="cuda") ** 4     # few tokens make up most of a text
        s |= dict(tokens=(usual * vocab).to(torch.int32).clamp_(max=vocab - 1), n_tokens=n,
                  n_prompt=(n * torch.rand((rows,), generator=gen, device="cuda")).to(torch.int32),
                  repetition=1.0 + 0.3 * torch.rand((rows,), generator=gen, device="cuda"),
                  frequency=0.5 * torch.rand((rows,), generator=gen, device="cuda"),
                  presence=0.5 * torch.rand((rows,), generator=gen, device="cuda"))
    if case["bias"]:
        n = min(case["bias"], vocab)
        ids = torch.rand((rows, vocab), generator=gen, device="cuda").topk(n, 1).indices.to(torch.int32)     # all different
        s |= dict(bias_ids=ids.reshape(-1).contiguous(), bias=2.0 * torch.randn((rows * n,), generator=gen, device="cuda"),
                  bias_offsets=torch.arange(0, rows * n + 1, n, dtype=torch.int32, device="cuda"))
    return s


def _draw_inputs(case, gen):
    rows = case["rows"]
    s = _rule_inputs(case, gen)
    t = 0.6 + 0.6 * torch.rand((rows,), generator=gen, device="cuda")
    if rows >= 8:
        t[5::16] = 0.0
    s |= dict(temperature=t, uniform=torch.rand((rows,), generator=gen, device="cuda", dtype=torch.float64),
              top_k=None, top_p=None, min_p=None)
    if case["top_k"]:
        s["top_k"] = torch.full((rows,), case["top_k"], dtype=torch.int32, device="cuda")
    if case["top_p"] < 1:
        s["top_p"] = torch.full((rows,), case["top_p"], dtype=torch.float32, device="cuda")
    if case["min_p"]:
        s["min_p"] = torch.full((rows,), case["min_p"], dtype=torch.float32, device="cuda")
    s["ids"] = torch.empty((rows,), dtype=torch.int32, device="cuda")
    s["logprobs"] = torch.empty((rows,), dtype=torch.float32, device="cuda")
    return s


def _address(t):
    return 0 if t is None else t.data_ptr()


def _rules_of(xgm, s, vocab):
    """The rules as a program hands them over: the addresses of its arrays."""
    r = dict(d_bitmask=_address(s["bitmask"]), v_mask=vocab)
    if s["tokens"] is not None:
        r |= dict(d_tokens=_address(s["tokens"]), token_stride=s["tokens"].stride(0), d_n_tokens=_address(s["n_tokens"]),
                  d_n_prompt=_address(s["n_prompt"]), d_repetition=_address(s["repetition"]), d_frequency=_address(s["frequency"]),
                  d_presence=_address(s["presence"]))
    if s["bias_ids"] is not None:
        r |= dict(d_bias_ids=_address(s["bias_ids"]), d_bias=_address(s["bias"]), d_bias_offsets=_address(s["bias_offsets"]),
                  n_bias=s["bias_ids"].numel())
    return xgm.LogitRules(**r)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"head": _head_inputs, "rules": _rule_inputs, "draw": _draw_inputs}[case["op"]](case, gen)
    s["case"] = dict(case)
    if case["op"] == "rules":
        s["out"] = torch.empty_like(s["logits"])
    if own and case["op"] != "head":      # a program keeps these from step to step: addresses of its arrays, working memory
        import paper_2411_15100_amd as xgm
        s["rules"] = _rules_of(xgm, s, case["vocab"])
        if case["op"] == "draw":
            s["draw"] = xgm.DrawRules(d_temperature=_address(s["temperature"]), d_top_k=_address(s["top_k"]),
                                      d_top_p=_address(s["top_p"]), d_min_p=_address(s["min_p"]), d_uniform=_address(s["uniform"]))
            s["sampler"] = xgm.Sampler(case["rows"], case["vocab"])
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls
def _run_own(s):
    import paper_2411_15100_amd as xgm
    case = s["case"]
    code = {"f32": xgm.DTYPE_F32, "bf16": xgm.DTYPE_BF16, "f16": xgm.DTYPE_F16}
    rows, vocab, stream = case["rows"], case["vocab"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "head":
        xgm.q4_logits(s["hidden"].data_ptr(), code[case["dtype"]], rows, case["k"], case["k"], s["codes"].data_ptr(),
                      s["scales"].data_ptr(), _address(s["zeros"]), vocab, case["group"], s["logits"].data_ptr(), code[case["out"]],
                      vocab, _address(s["bitmask"]), stream)
        return s["logits"]
    if case["op"] == "rules":
        xgm.process_logits(s["logits"].data_ptr(), code[case["dtype"]], rows, vocab, vocab, s["rules"], s["out"].data_ptr(), vocab, stream)
        return s["out"]
    s["sampler"].sample(s["logits"].data_ptr(), code[case["dtype"]], rows, vocab, vocab, s["rules"], s["draw"], s["ids"].data_ptr(),
                        s["logprobs"].data_ptr(), stream)
    return s["ids"], s["logprobs"]


# ------------------------------------------------------------------------------------------------ the plain forms
def _allowed(words, vocab):
    bits = words[:, :, None] >> torch.arange(32, dtype=torch.int32, device=words.device) & 1
    return bits.view(words.shape[0], -1)[:, :vocab].bool()


def _plain_head(s):
    case = s["case"]
    vocab, k, group = case["vocab"], case["k"], case["group"]
    n = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(vocab, k // group, group).float()
    n -= 8.0 if s["zeros"] is None else s["zeros"].float()[:, :, None]
    y = s["hidden"].float() @ (n * s["scales"].float()[:, :, None]).view(vocab, k).T
    if s["bitmask"] is not None:
        y = y.masked_fill(~_allowed(s["bitmask"], vocab), -math.inf)
    return y.to(TYPES[case["out"]])


def _plain_rules(s, exact):
    """The logits under the rules, computed in 32 bits, or in 64 for a draw: which of two near logits is larger decides a token."""
    t = torch.float64 if exact else torch.float32
    y = s["logits"].to(t)
    rows, vocab = y.shape
    if s["tokens"] is not None:
        at = torch.arange(s["tokens"].shape[1], device="cuda")
        there, prompt = at < s["n_tokens"][:, None], at < s["n_prompt"][:, None]
        ids, zero = s["tokens"].long(), torch.zeros((rows, vocab), dtype=t, device="cuda")
        count = zero.scatter_add(1, ids, (there & ~prompt).to(t))
        seen = zero.scatter_add(1, ids, there.to(t)) > 0
        r = s["repetition"].to(t)[:, None]
        y = torch.where(seen, torch.where(y > 0, y / r, y * r), y)
        y = torch.where(count > 0, y - s["frequency"].to(t)[:, None] * count - s["presence"].to(t)[:, None], y)
    if s["bias_ids"] is not None:
        y = y.scatter_add(1, s["bias_ids"].long().view(rows, -1), s["bias"].to(t).view(rows, -1))
    if s["bitmask"] is not None:
        y = y.masked_fill(~_allowed(s["bitmask"], vocab), -math.inf)
    return y.float()


def _plain_draw(s):
    y = _plain_rules(s, True)
    y = torch.where(y.isnan(), -math.inf, y).clamp(max=torch.finfo(torch.float32).max)
    rows, vocab = y.shape
    greedy = ~(s["temperature"] > 0)
    t = torch.where(greedy, 1.0, s["temperature"].double())[:, None]
    top = y.max(1, keepdim=True).values
    w = torch.where(y > -math.inf, torch.exp((y.double() - top.double()) / t), 0.0)
    whole = w.sum(1)
    kept = w
    if s["top_k"] is not None or s["top_p"] is not None:
        order = torch.sort(y, dim=1, descending=True, stable=True).indices
        sorted_w = w.gather(1, order)
        if s["top_k"] is not None:
            sorted_w = sorted_w * (torch.arange(vocab, device="cuda") < s["top_k"][:, None])
        if s["top_p"] is not None:
            run = sorted_w.cumsum(1)
            sorted_w = sorted_w * (run - sorted_w < s["top_p"].double()[:, None] * sorted_w.sum(1, keepdim=True))
        kept = torch.zeros_like(w).scatter(1, order, sorted_w)
    if s["min_p"] is not None:
        kept = kept * (kept >= s["min_p"].double()[:, None])
    run = kept.cumsum(1)
    ids = (run <= s["uniform"][:, None] * run[:, -1:]).sum(1)
    first = torch.where(y == top, torch.arange(vocab, device="cuda"), vocab).min(1).values
    ids = torch.where(greedy, first, ids.clamp(max=vocab - 1))
    logprobs = (y.gather(1, ids[:, None]).double() - top.double())[:, 0] / t[:, 0] - whole.log()
    none = top[:, 0] == -math.inf
    return torch.where(none, -1, ids).int(), torch.where(none, -math.inf, logprobs).float()


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "head":
        return _plain_head(state)
    return _plain_draw(state) if op == "draw" else _plain_rules(state, False).to(TYPES[state["case"]["dtype"]])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _allowed_rows(case):
    """Allowed tokens of all rows together, and how many different ones."""
    rows, vocab = case["rows"], case["vocab"]
    a = min(1.0, case["allowed"] / vocab)
    shares = [1.0 if case["mask"] == "none" else OPEN if case["mask"] == "mixed" and _open(b) else 1.0 - (1.0 - 1.0 / vocab) ** case["allowed"]
              for b in range(rows)]
    return vocab * sum(shares), vocab * (1.0 - math.prod(1.0 - x for x in shares))


def work(case):
    rows, vocab, e = case["rows"], case["vocab"], SIZES[case["dtype"]]
    pairs, tokens = _allowed_rows(case)
    mask = 0 if case["mask"] == "none" else 4 * rows * _words(vocab)
    if case["op"] == "head":
        a_row = case["k"] / 2 + case["k"] / case["group"] * (2 + (1 if case["zeros"] else 0))
        return {"bytes": tokens * a_row + rows * case["k"] * e + mask + rows * vocab * SIZES[case["out"]], "flops": 2.0 * pairs * case["k"]}
    text = rows * case["history"] * 4 * 0.6 + rows * case["bias"] * 8
    if case["op"] == "rules":
        return {"bytes": pairs * e + mask + text + rows * vocab * e, "flops": 2.0 * pairs}
    return {"bytes": pairs * e + mask + text + rows * 8, "flops": 15.0 * pairs}


# ------------------------------------------------------------------------------------------------ the definitions, in 64 bits
def _bits(words, vocab):
    return np.unpackbits(words.view(np.uint8), bitorder="little")[:vocab].astype(bool)


def _exact_head(s):
    case = s["case"]
    out = torch.empty((case["rows"], case["vocab"]), dtype=torch.float64, device="cuda")
    h = s["hidden"].double()
    for v in range(0, case["vocab"], 16384):
        part = slice(v, min(v + 16384, case["vocab"]))
        w = torch.empty((part.stop - v, case["k"]), dtype=torch.float64, device="cuda")
        w[:, 0::2] = s["codes"][part].remainder(16)
        w[:, 1::2] = s["codes"][part].div(16, rounding_mode="floor")
        w -= 8 if s["zeros"] is None else s["zeros"][part].double().repeat_interleave(case["group"], 1)
        w *= s["scales"][part].double().repeat_interleave(case["group"], 1)
        out[:, part] = (w @ h.T).T
    if s["bitmask"] is not None:
        for b, words in enumerate(s["bitmask"].cpu().numpy()):
            out[b, torch.from_numpy(~_bits(words, case["vocab"])).cuda()] = -math.inf
    return out


def _exact_rules(h, b, vocab):
    y = h["logits"][b].copy()
    if h["tokens"] is not None:
        n, p = int(h["n_tokens"][b]), int(h["n_prompt"][b])
        made = np.bincount(h["tokens"][b, p:n], minlength=vocab)
        seen = np.flatnonzero(np.bincount(h["tokens"][b, :n], minlength=vocab))
        r = np.float64(h["repetition"][b])
        y[seen] = [v / r if v > 0 else v * r for v in y[seen]]
        for v in np.flatnonzero(made):
            y[v] -= np.float64(h["frequency"][b]) * made[v] + np.float64(h["presence"][b])
    if h["bias_ids"] is not None:
        part = slice(h["bias_offsets"][b], h["bias_offsets"][b + 1])
        y[h["bias_ids"][part]] += h["bias"][part].astype(np.float64)
    if h["bitmask"] is not None:
        y[~_bits(h["bitmask"][b], vocab)] = -np.inf
    return y


def _exact_draw(h, b, vocab):
    y = _exact_rules(h, b, vocab).astype(np.float32).astype(np.float64)    # a draw is from logits in 32 bits
    order = np.lexsort((np.arange(vocab), -y))                             # falling, ties by the lower id
    t = float(h["temperature"][b])
    if y[order[0]] == -np.inf:
        return -1, -math.inf
    w = np.exp((y - y[order[0]]) / (t if t > 0 else 1.0))
    if not t > 0:
        return int(order[0]), -math.log(w.sum())
    n = int(np.count_nonzero(y > -np.inf))
    if h["top_k"] is not None:
        n = min(n, int(h["top_k"][b]))
    if h["top_p"] is not None:
        run = np.cumsum(w[order[:n]])
        n = min(n, int(np.searchsorted(run, np.float64(h["top_p"][b]) * run[-1])) + 1)
    kept = order[:n]
    if h["min_p"] is not None:
        kept = kept[w[kept] >= np.float64(h["min_p"][b])]
    kept = np.sort(kept)
    run = np.cumsum(w[kept])
    v = int(kept[min(len(kept) - 1, np.searchsorted(run, h["uniform"][b] * run[-1], side="right"))])
    return v, (y[v] - y[order[0]]) / t - math.log(w.sum())


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "head":
        return _exact_head(s)
    h = {k: (v.double() if k == "logits" else v).cpu().numpy() if isinstance(v, torch.Tensor) else v for k, v in s.items()
         if k != "out"}
    if case["op"] == "rules":
        return torch.from_numpy(np.stack([_exact_rules(h, b, case["vocab"]) for b in range(case["rows"])]))
    got = [_exact_draw(h, b, case["vocab"]) for b in range(case["rows"])]
    return torch.tensor([g[0] for g in got], dtype=torch.int32), torch.tensor([g[1] for g in got], dtype=torch.float64)
