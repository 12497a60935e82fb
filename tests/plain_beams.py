"""What the operators for 8-bit matrices and beams compute, from their definitions in 64 bits (numpy)."""

import numpy as np

BLOCK = 128


def e4m3():
    """The value of each of the 256 codes."""
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    x = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e.astype(float) - 7))
    x = np.where(c & 127 == 127, np.nan, x)
    return np.where(c & 128, -x, x)


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def quantized(x):
    """Codes [B, K] and scales [B, blocks] of values in 64 bits."""
    B, K = x.shape
    values = e4m3()[:127]                                # rising: 0 .. 448
    middles = (values[1:] + values[:-1]) / 2
    codes, scales = np.zeros((B, K), np.uint8), np.zeros((B, blocks(K)))
    for j in range(blocks(K)):
        part = x[:, j * BLOCK:(j + 1) * BLOCK]
        for b in range(B):
            row = part[b]
            most = np.abs(row[~np.isnan(row)]).max(initial=0.0)
            e = -126
            while e < 120 and most > 448.0 * 2.0 ** e:
                e += 1
            scales[b, j] = 2.0 ** e
            size = np.abs(row) / 2.0 ** e
            with np.errstate(invalid="ignore"):
                at = np.searchsorted(middles, size, side="left")
                tie = (at < 126) & (middles[np.minimum(at, 125)] == size) & (at % 2 == 1)
            c = (at + tie).astype(np.uint8) | np.where(np.signbit(row), 128, 0).astype(np.uint8)
            codes[b, j * BLOCK:(j + 1) * BLOCK] = np.where(np.isfinite(row), c, 127)
    return codes, scales


def project(codes, scales, matrix, matrix_scales):
    """[B, V] logits and the sums of the absolute terms."""
    table = e4m3()
    K, V = matrix.shape[1], matrix.shape[0]
    h = table[codes] * np.repeat(scales, BLOCK, 1)[:, :K]
    w = table[matrix] * np.repeat(np.repeat(matrix_scales, BLOCK, 0)[:V], BLOCK, 1)[:, :K]
    return h @ w.T, np.abs(h) @ np.abs(w).T


def select(y, scores, ended, beams, n_out, placed):
    """Continuations from processed logits y (float32 [rows, V]): rows, ids, sums (64 bits), each [requests, n_out]."""
    requests = y.shape[0] // beams
    rows, ids = np.full((requests, n_out), -1), np.full((requests, n_out), -1)
    sums = np.full((requests, n_out), -np.inf)
    for r in range(requests):
        found = []
        for b in range(r * beams, (r + 1) * beams):
            if not np.isfinite(scores[b]):
                continue
            if ended is not None and ended[b]:
                found.append((-np.float64(scores[b]), b, 0.0, -1))
                continue
            x = y[b].astype(np.float64)
            x[np.isnan(x)] = -np.inf
            x = np.minimum(x, np.finfo(np.float32).max)
            top = x.max()
            if top == -np.inf:
                continue
            base = np.float64(scores[b]) - (top + np.log(np.exp(x - top).sum()))
            order = np.lexsort((np.arange(x.size), -x))[:n_out]
            found += [(-(x[v] + base), b, -x[v], int(v)) for v in order if x[v] > -np.inf]
        found = sorted(found)[:n_out]
        got = [(b, v, -s) for s, b, _, v in found] + [(-1, -1, -np.inf)] * (n_out - len(found))
        if placed:
            first, others = {}, []
            for g in got:
                if g[0] >= 0 and g[0] not in first:
                    first[g[0]] = g
                else:
                    others.append(g)
            got = [first[r * beams + i] if r * beams + i in first else others.pop(0) for i in range(beams)]
        for j, g in enumerate(got):
            rows[r, j], ids[r, j], sums[r, j] = g
    return rows, ids, sums
