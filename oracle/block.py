"""TEST INFRASTRUCTURE - the block operators (attention over packed prompts, 4-bit cache and the attention over it,
root-mean-square norm, requantization by row scales) written from their definitions in ``include/iptq.h``,
in numpy's 64-bit integers and Python's whole numbers.  Never touches the HIP library."""

from __future__ import annotations

import math
from dataclasses import dataclass, field

import numpy as np

from .ref import Dyadic

GROUP = 64
SAT = 2 ** 23 - 1


@dataclass
class Attention:
    variant: int = 0
    i0: int = 256
    n_shift: int = 6
    score_shift: int = 0
    causal: int = 0
    post: Dyadic = field(default_factory=lambda: Dyadic(1, 8, 0, -128, 127))


def rshr_round(x, s):
    return x if s == 0 else (x + (1 << (s - 1))) >> s


def dyadic(x, p):
    return np.clip(rshr_round(np.asarray(x, np.int64) * p.m, p.s) + p.zp, p.qmin, p.qmax)


def weights(x, seen, p):
    """Qexp of the rows of x [rows, keys], of which row i sees the first seen[i] keys (or seen is a mask)."""
    x = rshr_round(x.astype(np.int64), p.score_shift)
    seen = np.asarray(seen)
    keep = seen if seen.dtype == bool else np.arange(x.shape[1])[None, :] < seen[:, None]
    if x.shape[1] == 0:
        return np.zeros_like(x)
    top = np.where(keep, x, -2 ** 60).max(1, keepdims=True)
    d = np.where(keep, x - top, 0)
    n = -(d + (d >> 1) - (d >> 4))
    q, r = n // p.i0, n % p.i0
    if p.variant == 0:
        base = p.i0 + ((-r) >> 1)
    else:
        y = ((-r) >> 1) + ((-r) >> 3) + ((-r) >> 4)
        base = p.i0 + y + (y * y // (2 * p.i0) if p.variant == 2 else 0)
    return np.where(keep & (q < 32), (base << p.n_shift) >> np.minimum(q, 31), 0)


def mean(acc, total, shift, post):
    f = np.array([(1 << 54) // int(t) if t else 0 for t in total], np.int64)[:, None]
    return dyadic((f * acc) >> shift, post).astype(np.int8)


def _product(a, b):
    """Whole numbers: every partial sum stays below 2^53, where doubles hold them exactly."""
    return (a.astype(np.float64) @ b.astype(np.float64)).astype(np.int64)


def attention(q, k, v, p, seen=None):
    """One sequence: q [nq, heads, d], k and v [nk, kv heads, d] int8."""
    (nq, heads, d), (nk, kv_heads, _) = q.shape, k.shape
    if seen is None:
        seen = np.arange(nq) + 1 + (nk - nq) if p.causal else np.full(nq, nk)
    out = np.zeros(q.shape, np.int8)
    for h in range(heads):
        g = h // (heads // kv_heads)
        x = _product(q[:, h], k[:, g].T)
        w = weights(x, seen, p)
        out[:, h] = mean(_product(w, v[:, g]), w.sum(1), 46, p.post)
    return out


def packed(q, k, v, q_offsets, k_offsets, max_q, p, out):
    """Packed sequences into a copy of out; rows that no sequence has, or beyond max_q, stay."""
    out = out.copy()
    for i in range(len(q_offsets) - 1):
        (a, b), (c, d) = q_offsets[i:i + 2], k_offsets[i:i + 2]
        n = min(b - a, max_q)
        out[a:a + n] = attention(q[a:b], k[c:d], v[c:d], p)[:n]
    return out


def groups(d):
    return -(-d // GROUP)


def quantize(x):
    """int8 [..., d] -> codes in [-7, 7] and steps [..., groups]."""
    d = x.shape[-1]
    x = np.pad(x.astype(np.int64), [(0, 0)] * (x.ndim - 1) + [(0, -d % GROUP)]).reshape(x.shape[:-1] + (groups(d), GROUP))
    a = np.abs(x).max(-1, keepdims=True)
    c = np.sign(x) * ((14 * np.abs(x) + a) // np.maximum(2 * a, 1))
    return c.reshape(c.shape[:-2] + (c.shape[-2] * GROUP,))[..., :d], a[..., 0]


def pack(c):
    c = c & 15
    return (c[..., 0::2] | c[..., 1::2] << 4).astype(np.uint8)


def unpack(b):
    b = b.astype(np.int64)
    c = np.stack((b & 15, b >> 4), -1).reshape(b.shape[:-1] + (2 * b.shape[-1],))
    return np.where(c > 7, c - 16, c)


def store(cache, k, v, slots):
    """cache: [k codes, k steps, v codes, v steps] as in the header; returns the updated copies."""
    kc, ks, vc, vs = (x.copy() for x in cache)
    pages, _, page = kc.shape[:3]
    for i, slot in enumerate(slots):
        if not 0 <= slot < pages * page:
            continue
        at, pos = divmod(int(slot), page)
        for x, codes, steps in ((k, kc, ks), (v, vc.transpose(0, 1, 3, 2), vs)):
            c, a = quantize(x[i])
            codes[at, :, pos] = pack(c)
            steps[at, :, pos] = a
    return [kc, ks, vc, vs]


def attention_cache(q, cache, pages, lengths, q_tokens, p):
    """q [n_seq * q_tokens, heads, d]; pages [n_seq, max_pages]."""
    kc, ks, vc, vs = cache
    n_pages, kv_heads, page, half = kc.shape
    d, heads = 2 * half, q.shape[1]
    out = np.zeros(q.shape, np.int8)
    for i in range(len(lengths)):
        n = min(max(int(lengths[i]), 0), pages.shape[1] * page)
        token = np.arange(n)
        at = pages[i][token // page].astype(np.int64)
        there = (at >= 0) & (at < n_pages)
        at, pos = np.where(there, at, 0), token % page
        last = n - q_tokens + np.arange(q_tokens) if p.causal else np.full(q_tokens, n - 1)
        keep = there[None, :] & (token[None, :] <= last[:, None])
        rows = slice(i * q_tokens, (i + 1) * q_tokens)
        for h in range(heads):
            g = h // (heads // kv_heads)
            spread = lambda a: np.repeat(a.astype(np.int64), GROUP, 1)[:, :d]  # noqa: E731
            x = _product(q[rows, h], (unpack(kc[at, g, pos]) * spread(ks[at, g, pos])).T)
            w = weights(x, keep, p)
            c = unpack(vc.transpose(0, 1, 3, 2)[at, g, pos])
            acc = np.concatenate([_product(rshr_round(w * vs[at, g, pos][:, j].astype(np.int64), 7), c[:, j * GROUP:(j + 1) * GROUP])
                                  for j in range(groups(d))], 1)
            out[rows, h] = mean(acc, w.sum(1), 39, p.post)
    return out


def rmsnorm(x, residual, gain, in_m, in_s, eps, post, row_scales):
    """(codes, stream, row scales or None) of one tensor [rows, cols]; Python's whole numbers per row."""
    rows, cols = (x if x is not None else residual).shape
    r = np.zeros((rows, cols), np.int64) if x is None else rshr_round(x.astype(np.int64) * in_m, in_s)
    if residual is not None:
        r = r + residual
    r = np.clip(r, -SAT, SAT)
    codes, scales = np.zeros((rows, cols), np.int8), np.zeros(rows, np.int32)
    for i in range(rows):
        s = min(sum(int(v) * int(v) for v in r[i]) + cols * eps, 2 ** 62 - 1)
        t = (62 - s.bit_length()) // 2
        f = (math.isqrt(cols << 32) * ((1 << 61) // math.isqrt(s << (2 * t)))) >> 24 if s else 0
        z = rshr_round(r[i] * f, 41 - t)
        y = rshr_round(z * gain.astype(np.int64), 6)
        if row_scales:
            scales[i] = np.abs(y).max()
            codes[i] = rshr_round(y * ((127 << 40) // int(scales[i]) if scales[i] else 0), 40)
        else:
            codes[i] = dyadic(y, post)
    return codes, r.astype(np.int32), scales if row_scales else None


def requant_rows(x, row_scales, row_shift, p):
    """Python's whole numbers: a product of two int32 and a shift of up to 62 bits may pass 64."""
    wide = x.astype(object) * row_scales.astype(object)[:, None]
    v = np.vectorize(lambda a: min(max(rshr_round(a, row_shift), -2 ** 31), 2 ** 31 - 1), otypes=[np.int64])(wide)
    return dyadic(v, p)
