"""What the operators around the mask compute, from their definitions in 64 bits (numpy)."""

import numpy as np


def unpack(words, V):
    """Truth values [rows, V] of mask words int32 [rows, (V + 31) // 32]."""
    bits = np.unpackbits(np.ascontiguousarray(words).view(np.uint8), axis=-1, bitorder="little")
    return bits[..., :V].astype(bool)


def pack(allowed):
    rows, V = allowed.shape
    bits = np.zeros((rows, (V + 31) // 32 * 32), dtype=np.uint8)
    bits[:, :V] = allowed
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32)


def project(hidden, codes, scales, zeros, group):
    """hidden [B, K], codes [V, K / 2], scales and zeros [V, K / group] -> [B, V] and the sum of the absolute terms that a
    kernel with codes shifted by up to 32 adds up."""
    n = np.empty((codes.shape[0], 2 * codes.shape[1]))
    n[:, 0::2] = codes & 15
    n[:, 1::2] = codes >> 4
    s = np.repeat(scales, group, 1)
    z = 8.0 if zeros is None else np.repeat(zeros.astype(np.float64), group, 1)
    return hidden @ ((n - z) * s).T, np.abs(hidden) @ np.abs(32.0 * s).T


def processed(x, b, allowed=None, tokens=None, n_tokens=None, n_prompt=None, repetition=None, frequency=None, presence=None, bias=None):
    """Row b of the logits under the rules, as float32; bias: a list of (id, value)."""
    y = x.astype(np.float64)
    V = y.shape[0]
    if tokens is not None:
        history = tokens[b, :min(int(n_tokens[b]), tokens.shape[1])]
        prompt = 0 if n_prompt is None else int(n_prompt[b])
        made = {}
        for i, t in enumerate(history):
            if 0 <= t < V:
                made[int(t)] = made.get(int(t), 0) + (1 if i >= prompt else 0)
        for t, count in made.items():
            if repetition is not None:
                r = np.float64(repetition[b])
                y[t] = y[t] / r if y[t] > 0 else y[t] * r
            if count:
                y[t] = y[t] - (np.float64(frequency[b]) if frequency is not None else 0.0) * count - (np.float64(presence[b]) if presence is not None else 0.0)
    if bias is not None:
        for t, v in dict(bias).items():
            if 0 <= t < V:
                y[t] += np.float64(np.float32(v))
    if allowed is not None:
        y[:allowed.shape[0]][~allowed[:V]] = -np.inf
        y[allowed.shape[0]:] = -np.inf
    with np.errstate(over="ignore"):
        return y.astype(np.float32)


class Row:
    """The distribution of a row of processed logits (float32): weights, kept tokens in order of ids, running sums."""

    def __init__(self, y, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
        y = np.where(np.isnan(y), np.float32(-np.inf), np.minimum(y, np.finfo(np.float32).max)).astype(np.float64)
        y = y + 0.0
        self.y, self.t = y, temperature if temperature > 0 else 1.0
        self.order = np.lexsort((np.arange(y.size), -y))
        self.top = y[self.order[0]]
        self.empty = self.top == -np.inf
        if self.empty:
            return
        with np.errstate(under="ignore"):
            self.w = np.where(y > -np.inf, np.exp((y - self.top) / self.t), 0.0)
        n = y.size
        if top_k > 0:
            n = min(n, top_k)
        self.run_sorted = np.cumsum(self.w[self.order[:n]])
        if top_p < 1:
            n = max(1, int(np.searchsorted(self.run_sorted, np.float64(top_p) * self.run_sorted[-1])) + 1)
        kept = self.order[:n]
        if min_p > 0:
            kept = kept[(self.w[kept] >= min(1.0, float(min_p))) | (kept == self.order[0])]
        self.kept = np.sort(kept)
        self.run = np.cumsum(self.w[self.kept])

    def logprob(self, v):
        return -np.inf if v < 0 else (self.y[v] - self.top) / self.t - np.log(self.w.sum())

    def pick(self, u):
        return int(self.kept[min(len(self.kept) - 1, np.searchsorted(self.run, u * self.run[-1], side="right"))])

    def middle(self, rng):
        """(u, id): a random number in the middle of the stretch of one kept token that has room for it."""
        w = self.w[self.kept] / self.run[-1]
        can = np.flatnonzero(w > 1e-7)
        k = int(can[rng.integers(can.size)]) if rng.random() < 0.5 else int(can[np.argmax(rng.random(can.size) * w[can])])
        return float((self.run[k] - 0.5 * self.w[self.kept[k]]) / self.run[-1]), int(self.kept[k])
