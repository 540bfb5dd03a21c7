"""Float64 forms of the packed cache's quantiser, of attention over it and of the
choice of beams (NumPy)."""
import numpy as np


def packed(x, bits):
    """What a cache of `bits` (8 or 4) makes of rows x [...][size]: values, and
    per group of 64 numbers the step and the zero."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 64)
    top, digits = 2 ** bits - 1, 4 if bits == 4 else 1
    ok = (np.abs(g) < 2.0 ** 125).all(-1)
    y = np.where(ok[..., None], g, 0.0)
    lo, hi = np.minimum(y.min(-1), 0.0), np.maximum(y.max(-1), 0.0)
    spread = (hi - lo).astype(np.float32).astype(np.float64)  # a range is held in fp32
    frac, exp = np.frexp(spread / top)
    step = np.maximum(np.ldexp(np.ceil(np.ldexp(frac, digits)), exp - digits), 2.0 ** -100)
    zero = np.rint(-lo / step)
    code = np.clip(np.rint(y / step[..., None]) + zero[..., None], 0, top)
    v = np.where(ok[..., None], (code - zero[..., None]) * step[..., None], np.nan)
    return v.reshape(x.shape), np.where(ok, step, np.nan), np.where(ok, zero, 0.0)


def continuations(scores, logits, n_best, suppress=()):
    """The n_best likeliest continuations of one group of beams: parents, tokens,
    scores. scores [width], logits [width][ids]."""
    total = []
    for c, row in zip(scores, logits):
        l = np.array(row, np.float64)
        l[list(suppress)] = -np.inf
        l[np.isnan(l)] = -np.inf
        m = l.max()
        if not np.isfinite(c) or m == -np.inf:
            total.append(np.full(len(l), -np.inf))
            continue
        d = np.where(l == np.inf, 0.0, -np.inf) if m == np.inf else l - m
        total.append(float(c) + (d - np.log(np.exp(d).sum())))
    total = np.concatenate(total)
    at = np.argsort(-total, kind="stable")[:n_best]
    at = at[total[at] > -np.inf]
    n = len(logits[0])
    gap = n_best - len(at)
    return (np.concatenate([at // n, np.full(gap, -1)]), np.concatenate([at % n, np.full(gap, -1)]),
            np.concatenate([total[at], np.full(gap, -np.inf)]))
