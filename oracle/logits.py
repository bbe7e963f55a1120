"""CPU oracle for the calls on logits -- TEST INFRASTRUCTURE ONLY.

Adjusted logits and choices are defined to the bit in fp32 (every operation rounded by itself), so
``adjust`` computes them in numpy fp32, a row at a time.  Distillation is computed in fp64 from its
definition (``distill``), with the gradient by differences of the loss beside it (``loss_difference``).
Shares no code with the library.
"""
from __future__ import annotations

import numpy as np

F = np.float32


def allowed_bits(words, V):
    """The mask's bits of one row: bit v % 32 of word v / 32."""
    words = np.asarray(words).view(np.uint32)
    return ((words[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1).astype(bool)


def mask_words(allowed):
    """int32 words [n, (V + 31) // 32] of boolean rows."""
    allowed = np.atleast_2d(allowed)
    n, V = allowed.shape
    W = (V + 31) // 32
    pad = np.zeros((n, W * 32), bool)
    pad[:, :V] = allowed
    return np.packbits(pad, axis=1, bitorder="little").view(np.int32).reshape(n, W)


def _row(a, r):
    return None if a is None else a[r % len(a)]


def adjust(rows, logits, *, history=None, lengths=None, repetition=None, frequency=None, presence=None,
           bias=None, inv_temperature=None, mask=None, noise=None):
    """(adjusted fp32 [rows, V], choice int64 [rows]); operands as in the library, logits as fp32."""
    V = logits.shape[1]
    out = np.empty((rows, V), F)
    choice = np.full(rows, -1, np.int64)
    with np.errstate(all="ignore"):
        for r in range(rows):
            x = _row(logits, r).astype(F)
            if history is not None:
                ids = np.asarray(_row(history, r), np.int64)
                if lengths is not None:
                    ids = ids[:max(0, min(int(_row(lengths, r)), len(ids)))]
                n = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)
                seen = n > 0
                if repetition is not None:
                    rep = F(_row(repetition, r))
                    x = np.where(seen, np.where(x > 0, x / rep, x * rep), x)
                if frequency is not None:
                    x = np.where(seen, x - n.astype(F) * F(_row(frequency, r)), x)
                if presence is not None:
                    x = np.where(seen, x - F(_row(presence, r)), x)
            if bias is not None:
                x = x + _row(bias, r)
            if inv_temperature is not None:
                x = x * F(_row(inv_temperature, r))
            if mask is not None:
                x = np.where(allowed_bits(_row(mask, r), V), x, F(-np.inf))
            out[r] = x
            y = x if noise is None else np.where(x == -np.inf, F(-np.inf), x + _row(noise, r))
            y = np.where(np.isnan(y), F(-np.inf), y)
            if y.max() > -np.inf:
                choice[r] = int(np.argmax(y))       # the first of the greatest
    assert out.dtype == F
    return out, choice


def valid_entries(ids, teacher, allowed, V):
    ids = np.asarray(ids, np.int64)
    ok = (ids >= 0) & (ids < V)
    if allowed is not None:
        ok &= allowed[np.clip(ids, 0, V - 1)]
    return ok & ~(np.asarray(teacher, np.float64) == -np.inf)


def distill(logits, ids, teacher, tau, mask=None, scale=None):
    """Per row, in fp64: loss, (m, s) and the gradient; and what error bounds are made of: the
    probabilities q and p (summed by entry), the greatest |log q| of a listed entry, the greatest
    distance of a listed teacher logit below the greatest one."""
    N, V = logits.shape
    res = {"loss": np.zeros(N), "stats": np.zeros((N, 2)), "grad": np.zeros((N, V)), "q": np.zeros((N, V)), "p": np.zeros((N, V)),
           "away": np.zeros((N, V)), "term": np.zeros(N), "spread": np.zeros(N), "has": np.zeros(N, bool)}
    with np.errstate(all="ignore"):
        for r in range(N):
            x = logits[r].astype(np.float64)
            ok = None
            if mask is not None:
                ok = allowed_bits(_row(mask, r), V)
                x = np.where(ok, x, -np.inf)
            m = np.fmax.reduce(x)
            m = -np.inf if np.isnan(m) else m
            s = np.exp((x - (m if m > -np.inf else 0.0)) / tau).sum()
            res["stats"][r] = m, s
            if ids.shape[1] == 0:
                continue
            t = np.asarray(_row(teacher, r), np.float64)
            i = np.asarray(_row(ids, r), np.int64)
            v = valid_entries(i, t, ok, V)
            if not v.any():
                continue
            res["has"][r] = True
            i, t = i[v], t[v]
            w = np.exp((t - np.fmax.reduce(t)) / tau)
            p = w / w.sum()
            d = (x - m) / tau
            logq = d[i] - np.log(s)
            terms = np.where(p == 0, 0.0, p * logq)
            res["loss"][r] = -tau * tau * terms.sum()
            res["term"][r] = np.abs(logq).max()
            res["spread"][r] = ((t.max() - t) / tau).max()
            np.add.at(res["p"][r], i, p)
            res["q"][r] = np.exp(d) / s
            res["away"][r] = np.where(res["q"][r] > 0, -d, 0.0)
            g = tau * (1.0 if scale is None else float(_row(scale, r))) * (res["q"][r] - res["p"][r])
            res["grad"][r] = g if ok is None else np.where(ok, g, 0.0)
    return res


def loss_difference(logits, ids, teacher, tau, mask, r, v, h=1e-4):
    """Central difference of row r's loss by its logit v."""
    one = np.repeat(logits[r:r + 1].astype(np.float64), 2, 0)
    one[0, v] += h
    one[1, v] -= h
    pick = [np.repeat(_row(a, r)[None], 2, 0) if a is not None else None for a in (ids, teacher, mask)]
    a, b = distill(one, pick[0], pick[1], tau, pick[2])["loss"]
    return (a - b) / (2 * h)
