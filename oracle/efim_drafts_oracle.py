"""CPU oracle of a step with drafted tokens: q/k norms with rotation, look-up of drafts, verification of drafts.

TEST INFRASTRUCTURE ONLY; shares no code with the library.  Everything in float64 (or whole numbers), one token, place or row after
the other, as the definitions read.

Readings (the paper leaves the model as it is and does not speak of drafts): the norm is the root mean square norm of one head's
values with a weight per dimension, rounded to bf16 once, behind the rotation; drafts are judged by the rejection rule of speculative
sampling (accept x with probability min(1, p(x)/q(x)), else draw from (p - q)^+), whose draw is made as the argmax of w_j / e_j with
exponential e; the look-up takes the longest agreeing suffix, the latest place among equals, and repeats itself past the end.
"""
import math

import numpy as np


def qk_norm(x, weight, eps, offset=0.0):
    """x: float64 [..., D]; weight: float64 [D] or None."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    return y if weight is None else y * (np.asarray(weight, np.float64) + offset)


def rotate(y, table_row, interleaved):
    """y: float64 [H, D]; table_row: cos of the D/2 angles, then their sines (the table the library is given).  Returns the rotated rows
    and, per value, the sum of the two products' magnitudes."""
    half = y.shape[1] // 2
    c, s = np.asarray(table_row[:half], np.float64), np.asarray(table_row[half:], np.float64)
    a = np.arange(0, 2 * half, 2) if interleaved else np.arange(half)
    b = a + 1 if interleaved else a + half
    out, size = np.empty_like(y), np.empty_like(y)
    out[:, a] = y[:, a] * c - y[:, b] * s
    out[:, b] = y[:, b] * c + y[:, a] * s
    size[:, a] = np.abs(y[:, a] * c) + np.abs(y[:, b] * s)
    size[:, b] = np.abs(y[:, b] * c) + np.abs(y[:, a] * s)
    return out, size


def draft_lookup(history, min_ngram, max_ngram, num_drafts):
    """history: list of token ids.  -> list of num_drafts ids, or None."""
    n = len(history)
    best = (0, 0)
    for e in range(1, n):
        m = 0
        while m < max_ngram and m < e and history[e - 1 - m] == history[n - 1 - m]:
            m += 1
        if m >= min_ngram:
            best = max(best, (m, e))
    if best[0] == 0:
        return None
    e = best[1]
    return [history[e + i % (n - e)] for i in range(num_drafts)]


def distribution(logits, temperature):
    """softmax(logits / temperature) in float64 (temperature <= 0: at 1), or None where there is none."""
    x = np.asarray(logits, np.float64)
    if np.isnan(x).any() or not (x > -np.inf).any():
        return None
    if (x == np.inf).any():
        w = (x == np.inf).astype(np.float64)
    else:
        w = np.exp((x - x.max()) / (temperature if temperature > 0 else 1.0))
    return w / w.sum()


def verify(tokens, rows, uniform, noise, draft_probs=None, temperature=1.0, probs=False):
    """One sequence.  tokens: its new tokens (pending, then drafts); rows: float64 [len(tokens)][vocab], logits or probabilities.
    noise None: greedy.  -> (accepted, next, log-probabilities of what it goes on with, margin): margin is the smallest
    relative distance that any decision had from going the other way."""
    greedy = not probs and (noise is None or not temperature > 0)
    vocab = len(rows[0]) if len(rows) else 0
    logs, margin = [], math.inf
    for i in range(len(tokens)):
        p = np.asarray(rows[i], np.float64) if probs else distribution(rows[i], temperature)
        if p is None:
            return i, -1, logs + [0.0], margin
        draft = int(tokens[i + 1]) if i + 1 < len(tokens) else None
        best = int(np.argmax(rows[i]))                 # the first of equals
        left = p
        if draft is not None:
            q = None if draft_probs is None else np.asarray(draft_probs[i], np.float64)
            inside = 0 <= draft < vocab
            if inside:
                if greedy:
                    taken = draft == best
                else:
                    lhs, rhs = float(uniform[i]) * (1.0 if q is None else q[draft]), p[draft]
                    taken = lhs < rhs
                    margin = min(margin, abs(lhs - rhs) / max(lhs, rhs, 1e-300))
                if taken:
                    logs.append(math.log(p[draft]))
                    continue
            if q is not None:
                left = np.maximum(p - q, 0.0)
            elif inside:
                left = p.copy()
                left[draft] = 0.0
            if not left.max() > 0:
                left = p
        if greedy:
            nxt = best
        else:
            score = np.where(left > 0, left, 0) / np.asarray(noise, np.float64)
            nxt = int(np.argmax(score))
            rest = np.delete(score, nxt)
            if rest.size and rest.max() > 0:
                margin = min(margin, 1 - rest.max() / score[nxt])
        return i, nxt, logs + [math.log(p[nxt])], margin
    return 0, -1, [0.0], margin                        # no rows
