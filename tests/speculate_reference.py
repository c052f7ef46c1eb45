"""Plain host forms of the calls for speculative decoding over the paged pool (numpy, 64 bits unless a call's steps are stated in 32)."""
from __future__ import annotations

import math

import numpy as np

import pages_reference as pages


def random_tree(n, rng, reach=4):
    """Parents of n rows: -1 for the first, else one of the `reach` rows in front."""
    return [-1] + [int(rng.integers(max(0, j - reach), j)) for j in range(1, n)] if n else []


def path(parent, j):
    found = []
    while j >= 0:
        found.append(j)
        j = parent[j]
    return found


def tables(first, n_pos, rot_dim, theta, factor=1.0, original_len=0.0, turns=(1.0, 32.0), amplitude=1.0):
    """cos, sin in 64 bits; angles in the host's extended type, whole turns taken away before the functions."""
    L = np.longdouble
    i = np.arange(rot_dim // 2).astype(L)
    f = np.exp(-2 * i / L(rot_dim) * np.log(L(theta)))
    two_pi = 2 * L("3.14159265358979323846264338327950288")
    g = np.clip((original_len * f / two_pi - turns[0]) / (L(turns[1]) - L(turns[0])), 0, 1) if original_len else np.zeros_like(f)
    turn = (first + np.arange(n_pos)).astype(L)[:, None] * (f * (g + (1 - g) / L(factor)) / two_pi)
    angle = ((turn - np.rint(turn)) * two_pi).astype(np.float64)
    return amplitude * np.cos(angle), amplitude * np.sin(angle)


def turned(x, gain, eps, cos, sin, interleaved, half, tiny):
    """Heads x [rows][heads][d] normalised (gain not None) and rotated by cos, sin [rows][rot/2].  Returns values and bounds on the errors.

    Bounds.  half, tiny: half a step of the 16-bit type, relative and at its smallest values; the result is rounded once.  The norm in fp32: a sum
    of d squares (at most d 2^-24 relative), the reciprocal root (2^-22) and two products; the rotation: two products and a sum, 3 2^-24 of the
    products' magnitudes.  (d + 16) 2^-24 of the magnitudes that are added covers both.
    """
    x = x.astype(np.float64)
    d, r = x.shape[-1], 2 * cos.shape[-1]
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain.astype(np.float64)
    y, big = x.copy(), np.abs(x)
    if r:
        at = np.arange(r // 2)
        i, j = (2 * at, 2 * at + 1) if interleaved else (at, at + r // 2)
        c, s = cos[:, None, :].astype(np.float64), sin[:, None, :].astype(np.float64)
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
        big[..., i], big[..., j] = (np.abs(x[..., u] * c) + np.abs(x[..., v] * s) for u, v in ((i, j), (j, i)))
    exact = gain is None and r == 0
    return y, np.zeros_like(y) if exact else half * np.abs(y) + 2 * (d + 16) * 2.0 ** -24 * big + tiny


def tree_attention(k, v, q, n, nq, ratio, scale, half, seen):
    """As pages.attention, row j over the keys that seen[j] [n] says: the same bounds."""
    got = []
    for j in range(nq):
        at = np.nonzero(seen[j])[0]
        got.append(pages.attention(k[at], v[at], q[j:j + 1], len(at), 1, ratio, scale, half))
    return tuple(np.concatenate(x) for x in zip(*got))


def seen_by(parent, n):
    """[nq][n]: what the rows of a tree see of a sequence of n rows."""
    nq = len(parent)
    s = np.zeros((nq, n), bool)
    s[:, :n - nq] = True
    for j in range(nq):
        s[j, [n - nq + a for a in path(parent, j)]] = True
    return s


def logits(x, prompt, made, rep, freq, pres, bias, allowed, t=np.float32):
    """One row by the stated steps in type t: x [vocab] and the token picked.  bias: (token, value) in order, the last of a token stands."""
    vocab = len(x)
    x = x.astype(t)
    inside = lambda a: np.array([y for y in a if 0 <= y < vocab], np.int64)  # noqa: E731
    c = np.bincount(inside(made), minlength=vocab)
    seen = (c + np.bincount(inside(prompt), minlength=vocab)) > 0
    with np.errstate(all="ignore"):
        x = np.where(seen, np.where(x > 0, x / t(rep), x * t(rep)), x)
        x = np.where(c > 0, x - t(freq) * c.astype(t), x)
        x = np.where(c > 0, x - t(pres), x)
        for tok, val in dict(bias).items():
            if 0 <= tok < vocab:
                x[tok] = x[tok] + t(val)
        x = np.where(allowed, x, t(-np.inf))
        key = np.where(np.isnan(x), np.inf, x)
    nan = np.nonzero(np.isnan(x) & allowed)[0]
    if len(nan):
        return x, int(nan[0])
    at = np.nonzero(allowed)[0]
    return x, int(at[np.argmax(key[at])]) if len(at) else -1


def accept(parent, drafted, chosen):
    """The path from row 0: the first child whose drafted token is the one chosen at the row."""
    got = [0] if len(parent) else []
    while got:
        r = got[-1]
        nxt = [c for c in range(r + 1, len(parent)) if parent[c] == r and drafted[c] == chosen[r] and chosen[r] >= 0]
        if not nxt:
            break
        got.append(nxt[0])
    return got
