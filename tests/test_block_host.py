"""The block operators without a GPU: refusals and no-ops of every entry point, the constants derived from real scales,
the oracle's hand-worked values, integer helpers and address rules compiled for the host, and the instructions of the kernels."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_2511_15369_amd as ip
from oracle import block as ob
from oracle.ref import Dyadic
from paper_2511_15369_amd import block, build

NULL, SHAPE, PARAM, RANGE, ALIGN, WORKSPACE = -1, -2, -3, -4, -6, -7
BASE = 1 << 40                                       # addresses that are never followed


def params(**k):
    f = dict(variant=1, i0=512, n_shift=5, score_shift=2, causal=1, post=ip.Dyadic(20000, 20, 0, -128, 127))
    f.update(k)
    return ip.AttentionParams(*[f[n] for n, _ in ip.AttentionParams._fields_])


def attention(p=params(), stream=None, **k):
    f = dict(q=BASE, qs=8 * 64, k=2 * BASE, ks=2 * 64, v=3 * BASE, vs=2 * 64, qo=4 * BASE, ko=5 * BASE, n=0, max_q=10, qt=20, kt=20,
             heads=8, kv=2, dim=64, out=6 * BASE, os=8 * 64)
    f.update(k)
    return block._lib().iptq_attention_i8(f["q"], f["qs"], f["k"], f["ks"], f["v"], f["vs"], f["qo"], f["ko"], f["n"], f["max_q"],
                                          f["qt"], f["kt"], f["heads"], f["kv"], f["dim"], f["out"], f["os"],
                                          None if p is None else ctypes.byref(p), stream)


@pytest.mark.parametrize("code,change", [
    (0, {}), (NULL, dict(p=None)), (PARAM, dict(p=params(i0=15))), (PARAM, dict(p=params(i0=1025))), (PARAM, dict(p=params(n_shift=-1))),
    (RANGE, dict(p=params(n_shift=6))), (0, dict(p=params(i0=32639 >> 5))), (PARAM, dict(p=params(score_shift=17))),
    (PARAM, dict(p=params(score_shift=-1))), (PARAM, dict(p=params(causal=2))), (PARAM, dict(p=params(variant=3))),
    (PARAM, dict(p=params(post=ip.Dyadic(1, 63, 0, -128, 127)))), (PARAM, dict(p=params(post=ip.Dyadic(1, 0, 0, 0, 255)))),
    (SHAPE, dict(heads=0)), (SHAPE, dict(heads=7)), (SHAPE, dict(kv=0)), (SHAPE, dict(dim=48)), (SHAPE, dict(dim=256)), (SHAPE, dict(n=-1)),
    (SHAPE, dict(max_q=-1)), (SHAPE, dict(qt=-1)), (SHAPE, dict(kt=1 << 31)), (SHAPE, dict(qt=(1 << 31) - 256)), (NULL, dict(n=1, qt=(1 << 31) - 257, q=None)), (SHAPE, dict(qs=511)), (SHAPE, dict(ks=127)),
    (SHAPE, dict(vs=127)), (SHAPE, dict(os=511)), (SHAPE, dict(os=1 << 31)), (NULL, dict(qo=None)), (NULL, dict(ko=None)),
    (SHAPE, dict(qo=None, ko=None)), (SHAPE, dict(qo=None, ko=None, n=3)), (SHAPE, dict(qo=None, ko=None, n=1, kt=65537)),
    (0, dict(qo=None, ko=None, n=0, qt=0, kt=0)), (0, dict(n=1, max_q=0)), (0, dict(n=1, qt=0)), (SHAPE, dict(n=1 << 30, max_q=1 << 20)),
    (NULL, dict(n=1, q=None)), (NULL, dict(n=1, k=None)), (NULL, dict(n=1, v=None)), (NULL, dict(n=1, out=None)),
    (ALIGN, dict(n=1, qo=4 * BASE + 2)), (ALIGN, dict(n=1, ko=5 * BASE + 1)), (PARAM, dict(n=1, out=BASE)),
    (PARAM, dict(n=1, out=2 * BASE + 19 * 128)), (PARAM, dict(n=1, out=3 * BASE - 19 * 512 - 511)), (PARAM, dict(n=1, out=4 * BASE)),
    (PARAM, dict(n=1, out=5 * BASE + 4))])
def test_attention_refuses(code, change):
    assert attention(**change) == code


def cache(**k):
    f = dict(kc=BASE, ks=2 * BASE, vc=3 * BASE, vs=4 * BASE, pages=10, tokens=32, heads=2, dim=64)
    f.update(k)
    return ip.CacheI4(*[f[n] for n in ("kc", "ks", "vc", "vs", "pages", "tokens", "heads", "dim")])


CACHES = [(NULL, None), (NULL, dict(kc=None)), (NULL, dict(ks=None)), (NULL, dict(vc=None)), (NULL, dict(vs=None)), (ALIGN, dict(kc=BASE + 8)),
          (ALIGN, dict(ks=BASE + 1)), (ALIGN, dict(vc=BASE + 4)), (ALIGN, dict(vs=BASE + 8)), (SHAPE, dict(pages=0)), (SHAPE, dict(tokens=8)),
          (SHAPE, dict(tokens=48)), (SHAPE, dict(tokens=8192)), (SHAPE, dict(heads=0)), (SHAPE, dict(dim=80)),
          (SHAPE, dict(pages=1 << 26))]


def store(c, **k):
    f = dict(k=6 * BASE, ks=128, v=7 * BASE, vs=128, slots=8 * BASE, tokens=5)
    f.update(k)
    return block._lib().iptq_cache_store_i4(None if c is None else ctypes.byref(c), f["k"], f["ks"], f["v"], f["vs"], f["slots"],
                                            f["tokens"], None)


@pytest.mark.parametrize("code,change", CACHES)
def test_a_cache_is_checked(code, change):
    c = None if change is None else cache(**change)
    assert store(c) == code
    size = ctypes.c_int64(-5)
    ref = None if c is None else ctypes.byref(c)
    assert block._lib().iptq_attention_cache_i4_workspace(ref, 1, 1, 2, 1, ctypes.byref(size)) == code and size.value == -5
    assert attend(c) == code


@pytest.mark.parametrize("code,change", [
    (0, dict(tokens=0)), (SHAPE, dict(tokens=-1)), (SHAPE, dict(tokens=1 << 31)), (SHAPE, dict(ks=127)), (SHAPE, dict(vs=1 << 31)),
    (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(slots=None)), (ALIGN, dict(slots=8 * BASE + 2)), (PARAM, dict(k=BASE)),
    (PARAM, dict(v=4 * BASE + 639)), (PARAM, dict(slots=2 * BASE - 16)), (PARAM, dict(k=3 * BASE - 639)), (SHAPE, dict(tokens=1 << 27)),
    (NULL, dict(tokens=(1 << 27) - 16, k=None))])
def test_a_store_refuses(code, change):
    assert store(cache(), **change) == code


def attend(c, p=params(), **k):
    f = dict(q=6 * BASE, qs=512, pages=7 * BASE, max_pages=4, lengths=8 * BASE, n=0, t=1, heads=8, out=9 * BASE, os=512, work=10 * BASE,
             size=1 << 40)
    f.update(k)
    return block._lib().iptq_attention_cache_i4(f["q"], f["qs"], None if c is None else ctypes.byref(c), f["pages"], f["max_pages"],
                                                f["lengths"], f["n"], f["t"], f["heads"], f["out"], f["os"], f["work"], f["size"],
                                                None if p is None else ctypes.byref(p), None)


@pytest.mark.parametrize("code,change", [
    (0, {}), (NULL, dict(p=None)), (0, dict(p=params(score_shift=20))), (PARAM, dict(p=params(score_shift=21))), (PARAM, dict(p=params(i0=8))),
    (SHAPE, dict(n=-1)), (SHAPE, dict(t=0)), (SHAPE, dict(t=65)), (SHAPE, dict(max_pages=-1)), (SHAPE, dict(max_pages=4097)),
    (SHAPE, dict(heads=0)), (SHAPE, dict(heads=9)), (SHAPE, dict(n=1 << 22)), (SHAPE, dict(qs=511)), (SHAPE, dict(os=511)),
    (SHAPE, dict(size=-1)), (NULL, dict(n=1, q=None)), (NULL, dict(n=1, out=None)), (NULL, dict(n=1, lengths=None)),
    (NULL, dict(n=1, pages=None)), (ALIGN, dict(n=1, pages=7 * BASE + 1)), (ALIGN, dict(n=1, lengths=8 * BASE + 2)),
    (PARAM, dict(n=1, out=6 * BASE + 511)), (PARAM, dict(n=1, out=BASE)), (PARAM, dict(n=1, out=7 * BASE + 15)),
    (PARAM, dict(n=1, out=8 * BASE)), (PARAM, dict(n=1, out=3 * BASE + 10 * 2 * 32 * 32 - 1)), (SHAPE, dict(n=1 << 21)), (NULL, dict(n=(1 << 21) - 1, q=None)),
    (SHAPE, dict(n=1 << 20, max_pages=33)), (NULL, dict(n=(1 << 20) - 1, max_pages=33, q=None)), (SHAPE, dict(n=1 << 14, max_pages=4096))])
def test_cache_attention_refuses(code, change):
    assert attend(cache(), **change) == code


@pytest.mark.parametrize("n,heads,t,max_pages", [(0, 8, 1, 4096), (0, 8, 64, 0), (1 << 20, 8, 1, 0), (65535, 2, 1, 4096), ((1 << 24) // 2 - 1, 2, 1, 3)])
def test_cache_workspaces_at_their_ends(n, heads, t, max_pages):
    """No sequence, no page, as many as there may be: a size that is none or fits its scores and sums."""
    size = ctypes.c_int64(-1)
    assert block._lib().iptq_attention_cache_i4_workspace(ctypes.byref(cache()), n, t, heads, max_pages, ctypes.byref(size)) == 0
    keys = max_pages * 32
    whole = n * 2 <= 1 << 22 and keys <= 1024            # (heads on two kv heads)
    assert size.value % 16 == 0 and (size.value == 0) == (n == 0 or whole)
    assert size.value == 0 or n * heads * t * keys * 2 < size.value < n * heads * t * (keys * 2 + 256 + 128 * 280)


@pytest.mark.parametrize("heads,t,max_pages", [(2, 1, 4096), (128, 4, 4096), (8, 1, 3)])
def test_cache_attention_wants_its_workspace(heads, t, max_pages):
    size = ctypes.c_int64()
    assert block._lib().iptq_attention_cache_i4_workspace(ctypes.byref(cache()), 2, t, heads, max_pages, ctypes.byref(size)) == 0
    assert size.value >= 0
    assert block._lib().iptq_attention_cache_i4_workspace(ctypes.byref(cache()), 2, t, heads, max_pages, None) == NULL
    if size.value:
        k = dict(n=2, t=t, heads=heads, max_pages=max_pages, qs=64 * heads, os=64 * heads)
        assert attend(cache(), size=size.value - 1, **k) == WORKSPACE
        assert attend(cache(), work=None, **k) == NULL
        assert attend(cache(), work=10 * BASE + 8, **k) == ALIGN
        for at in (6 * BASE, 7 * BASE, 8 * BASE, 9 * BASE, BASE, 2 * BASE, 3 * BASE, 4 * BASE):
            assert attend(cache(), work=at, **k) == PARAM
    assert "workspace" in ip.strerror(WORKSPACE)


def norm(p=ip.RmsnormParams(20000, 16, 1, ip.Dyadic(20000, 29, 0, -128, 127)), **k):
    f = dict(x=BASE, r=2 * BASE, g=3 * BASE, ro=2 * BASE, out=4 * BASE, s=5 * BASE, rows=0, cols=100)
    f.update(k)
    return block._lib().iptq_rmsnorm_i32(f["x"], f["r"], f["g"], f["ro"], f["out"], f["s"], f["rows"], f["cols"],
                                         None if p is None else ctypes.byref(p), None)


def norm_params(**k):
    f = dict(m=20000, s=16, eps=1, post=ip.Dyadic(20000, 29, 0, -128, 127))
    f.update(k)
    return ip.RmsnormParams(f["m"], f["s"], f["eps"], f["post"])


@pytest.mark.parametrize("code,change", [
    (0, {}), (NULL, dict(p=None)), (SHAPE, dict(rows=-1)), (SHAPE, dict(rows=1 << 31)), (SHAPE, dict(cols=0)), (SHAPE, dict(cols=16385)),
    (PARAM, dict(p=norm_params(m=32768))), (PARAM, dict(p=norm_params(m=-32768))), (PARAM, dict(p=norm_params(s=63))),
    (PARAM, dict(p=norm_params(eps=-1))), (PARAM, dict(p=norm_params(eps=2 ** 46 + 1))), (PARAM, dict(p=norm_params(post=ip.Dyadic(1, 0, 0, 0, 128)))),
    (NULL, dict(rows=1, x=None, r=None, ro=None)), (NULL, dict(rows=1, g=None)), (NULL, dict(rows=1, out=None)), (ALIGN, dict(rows=1, x=BASE + 2)),
    (ALIGN, dict(rows=1, r=BASE + 1, ro=None)), (ALIGN, dict(rows=1, g=3 * BASE + 1)), (ALIGN, dict(rows=1, s=5 * BASE + 2)),
    (PARAM, dict(rows=1, ro=2 * BASE + 4)), (PARAM, dict(rows=1, ro=BASE)), (PARAM, dict(rows=1, out=BASE + 399)), (PARAM, dict(rows=1, out=2 * BASE)),
    (PARAM, dict(rows=1, out=3 * BASE + 199)), (PARAM, dict(rows=2, s=4 * BASE + 196)), (PARAM, dict(rows=1, s=2 * BASE)),
    (PARAM, dict(rows=1, ro=6 * BASE, s=6 * BASE + 396))])
def test_norm_refuses(code, change):
    assert norm(**change) == code


@pytest.mark.parametrize("code,change", [
    (0, {}), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=0)), (SHAPE, dict(cols=1048577)), (PARAM, dict(shift=63)), (PARAM, dict(shift=-1)),
    (PARAM, dict(signed=2)), (PARAM, dict(p=ip.Dyadic(1, 0, 0, -1, 127), signed=0)), (NULL, dict(p=None)), (NULL, dict(rows=1, x=None)),
    (NULL, dict(rows=1, s=None)), (NULL, dict(rows=1, out=None)), (ALIGN, dict(rows=1, x=BASE + 1)), (ALIGN, dict(rows=1, s=2 * BASE + 2)),
    (PARAM, dict(rows=1, out=BASE + 39)), (PARAM, dict(rows=3, out=2 * BASE + 11))])
def test_requant_rows_refuses(code, change):
    f = dict(x=BASE, s=2 * BASE, shift=22, out=3 * BASE, rows=0, cols=10, signed=1, p=ip.Dyadic(20000, 20, 0, -128, 127))
    f.update(change)
    assert block._lib().iptq_requant_rows(f["x"], f["s"], f["shift"], f["out"], f["rows"], f["cols"], f["signed"],
                                          None if f["p"] is None else ctypes.byref(f["p"]), None) == code


def test_prepare_from_real_scales():
    rng = np.random.default_rng(0)
    for _ in range(300):
        of_cache, variant, causal = int(rng.integers(2)), int(rng.integers(3)), int(rng.integers(2))
        s, sv, so = (float(2.0 ** rng.uniform(-20, -5)) for _ in range(3))
        scale = s / 7 if of_cache else s
        shift = 0
        while 1 / (scale * 2 ** shift) >= 1025:
            shift += 1
        if shift > (20 if of_cache else 16):
            with pytest.raises(ip.IptqError):
                ip.attention_prepare(s, sv, so, 3, variant, causal, of_cache)
            continue
        p = ip.attention_prepare(s, sv, so, 3, variant, causal, of_cache)
        assert (p.variant, p.score_shift, p.causal, p.i0) == (variant, shift, causal, int(1 / (scale * 2 ** shift)))
        assert p.i0 << p.n_shift <= 32639 < p.i0 << (p.n_shift + 1)
        ratio = sv / (256 * so) / (7 if of_cache else 1)
        assert abs(p.post.m / 2 ** p.post.s / ratio - 1) <= 2 ** -14 and (p.post.zp, p.post.qmin, p.post.qmax) == (3, -128, 127)
    for bad in ((0.0, 1, 1), (1.0, 1, 1), (1e-3, -1.0, 1), (1e-3, 1, float("inf")), (float("nan"), 1, 1), (1e-12, 1, 1)):
        with pytest.raises(ip.IptqError):
            ip.attention_prepare(*bad, 0, 0, 0)
    for bad in ((3, 0, 0), (0, 2, 0), (0, 0, 2)):
        with pytest.raises(ip.IptqError):
            ip.attention_prepare(1e-3, 0.02, 0.02, 0, *bad)


# ----------------------------------------------------------------------------- the oracle, by hand
def test_oracle_attention_by_hand():
    # i0 = 16, N = 0: scores 0, -8, -16 have d = 0, -8, -16; Qp = 0, -8 - 4 + 1 = -11, -16 - 8 + 1 = -23
    # n = 0, 11, 23: q = 0, 0, 1, r = 0, 11, 7: base (variant 0) = 16, 16 - 6 = 10, 16 - 4 = 12 -> 16, 10, 6
    p = ob.Attention(variant=0, i0=16, n_shift=0, post=Dyadic(1, 8, 0, -128, 127))
    x = np.array([[0, -8, -16]])
    assert ob.weights(x, np.array([3]), p).tolist() == [[16, 10, 6]]
    assert ob.weights(x, np.array([2]), p).tolist() == [[16, 10, 0]]
    # variant 1: -r = -11: -6 - 2 - 1 = -9, -7: -4 - 1 - 1 = -6 -> 16, 7, 10 >> 1 = 5; variant 2: 81 // 32 = 2, 36 // 32 = 1
    p.variant = 1
    assert ob.weights(x, np.array([3]), p).tolist() == [[16, 7, 5]]
    p.variant = 2
    assert ob.weights(x, np.array([3]), p).tolist() == [[16, 9, 5]]
    # values 10, -20, 40 with weights 16, 10, 6: sum 32, 160 - 200 + 240 = 200; f = 2^49, o = 200 * 2^49 >> 46 = 1600, 6.25 in
    # eight fractional bits, rounded 6
    p.variant = 0
    q, k, v = np.zeros((1, 1, 32), np.int8), np.zeros((3, 1, 32), np.int8), np.zeros((3, 1, 32), np.int8)
    q[0, 0, 0], k[:, 0, 0], v[:, 0, 5] = 8, (0, -1, -2), (10, -20, 40)
    out = ob.attention(q, k, v, p)
    assert out[0, 0, 5] == 6 and np.count_nonzero(out) == 1
    p.causal = 1
    assert ob.attention(np.repeat(q, 3, 0), k, v, p)[:, 0, 5].tolist() == [10, (160 - 200) * (2 ** 54 // 26) // 2 ** 46 + 128 >> 8, 6]


def test_oracle_cache_by_hand():
    # step 70: 5 -> (70 + 70) // 140 = 1; 4 -> 126 // 140 = 0; -70 -> -7; 34 -> 546 // 140 = 3; step 0: all 0
    x = np.zeros((1, 128), np.int8)
    x[0, :4] = (5, 4, -70, 34)
    c, a = ob.quantize(x)
    assert c[0, :4].tolist() == [1, 0, -7, 3] and a.tolist() == [[70, 0]] and not c[0, 4:].any()
    assert ob.pack(c)[0, :2].tolist() == [0x01, 0x39] and np.array_equal(ob.unpack(ob.pack(c)), c)
    every = np.arange(-128, 128).astype(np.int8)
    for a in range(1, 129):                               # no code is further than half a step of a / 7 from its value
        v = every[np.abs(every.astype(int)) <= a].astype(int)
        code = np.sign(v) * ((14 * np.abs(v) + a) // (2 * a))
        assert np.abs(code).max() <= 7 and np.all(np.abs(14 * v - 2 * a * code) <= a)


def test_oracle_norm_by_hand():
    # a row of equal values r: every z is 2^12 (its own root mean square), whatever r, within the rounding of F
    for r in (1, 7, 12345, ob.SAT):
        x = np.full((1, 64), r, np.int32)
        codes, stream, s = ob.rmsnorm(None, x, np.full(64, 64, np.int16), 1, 0, 0, Dyadic(1, 12 - 6, 0, -128, 127), False)
        assert np.all(codes == 64) and np.all(stream == r)
    codes, _, s = ob.rmsnorm(None, np.array([[3, -4, 0, 0]], np.int32), np.full(4, 64, np.int16), 1, 0, 0, None, True)
    # root mean square 2.5: -4 / 2.5 = -1.6 -> y = -1.6 * 4096
    assert abs(s[0] - 1.6 * 4096) <= 1 and codes[0].tolist() == [95, -127, 0, 0]
    zero = ob.rmsnorm(None, np.zeros((1, 4), np.int32), np.ones(4, np.int16), 1, 0, 0, Dyadic(1, 0, 5, -128, 127), False)
    assert zero[0].tolist() == [[5] * 4]
    assert ob.rmsnorm(np.array([[2 ** 31 - 1]], np.int32), None, np.ones(1, np.int16), 32767, 0, 0, Dyadic(), False)[1][0, 0] == ob.SAT
    assert ob.requant_rows(np.array([[-3, 2 ** 31 - 1]], np.int32), np.array([2 ** 31 - 1], np.int32), 1, Dyadic(1, 0, 0, -128, 127)).tolist() \
        == [[-128, 127]]


# ----------------------------------------------------------------------------- helpers on the host
DRIVER = r"""
#include "block.h"
#include <stdio.h>
#include <vector>
using namespace iptq;
static uint64_t s = 0x9E3779B97F4A7C15ull;
static uint64_t rnd() { s ^= s << 13; s ^= s >> 7; s ^= s << 17; return s; }
int main()
{
    for (long i = 0; i < 4000000; ++i) {
        const uint32_t d = (1u << 30) | (uint32_t)(i < 100000 ? i : i < 200000 ? 0x3fffffffl - (i - 100000) : (long)(rnd() >> 34));
        if (floor_div_2_61(d) != (1ull << 61) / d) return printf("%u\n", d), 1;
    }
    for (long i = 0; i < 4000000; ++i) {
        const uint32_t d = i < 600000 ? (uint32_t)i : i < 700000 ? 0x80050000u - (uint32_t)(i - 600000) * 7 : i < 1200000 ? 0u - (uint32_t)(i - 700000) * 211
                           : (uint32_t)(rnd() >> (32 + rnd() % 32));
        if (floor_div_scaled(1, 54, d) != (d ? (1ull << 54) / d : 0) || floor_div_scaled(127, 40, d) != (d ? (127ull << 40) / d : 0)) return printf("%u\n", d), 9;
    }
    for (long i = 0; i < 300000; ++i) {
        const uint64_t v = i < 4 ? (1ull << 62) - 1 - i : i < 8 ? (1ull << 60) + i - 4 : (1ull << 60) + rnd() % (3ull << 60);
        const unsigned __int128 r = root_u62(v);
        if (r * r > v || (r + 1) * (r + 1) <= v) return 3;
    }
    for (uint32_t d = 1; d < 5000; d += 1 + d / 50) {
        const DivDev D = div_of(d);
        for (int i = 0; i < 2000; ++i) {
            const uint32_t n = i < 10 ? 0x7fffffffu - i : (uint32_t)(rnd() >> (33 + rnd() % 20));
            if (div_by(n, D) != n / d) return 4;
        }
    }
    // what a table says is followed only inside the cache: ids outside it, keys behind the length
    std::vector<int32_t> table = {3, -1, 4, 2147483647, 0};
    for (int32_t key = 0; key < 5 * 32; ++key)
        for (int32_t length : {0, 1, 31, 32, 33, 100, 160}) {
            const int32_t id = table[key / 32], want = key < length && id >= 0 && id < 4 ? id : -1;
            if (page_of_key(table.data(), 5, 4, key, length) != want) return 5;
        }
    if (page_of_key(nullptr, 5, 4, 0, 0) != -1 || page_of_key(nullptr, 5, 4, 1 << 30, 160) != -1) return 6;
    // offsets are clamped: [from, from + n) always lies inside the tokens
    const int32_t wild[] = {INT32_MIN, -7, 0, 1, 5, 9, 10, 11, INT32_MAX};
    for (int32_t a : wild)
        for (int32_t b : wild)
            for (int32_t tokens : {0, 1, 10, INT32_MAX}) {
                int32_t from, n;
                clamped_range(a, b, tokens, &from, &n);
                if (from < 0 || n < 0 || (int64_t)from + n > tokens) return 7;
                if (a >= 0 && a <= b && b <= tokens && (from != a || n != b - a)) return 8;
            }
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not installed")
def test_integer_helpers_and_address_rules(tmp_path):
    src, exe = str(tmp_path / "driver.cpp"), str(tmp_path / "driver")
    with open(src, "w") as f:
        f.write(DRIVER)
    subprocess.check_call(["hipcc", "-x", "hip", "--cuda-host-only", "-O2", "-std=c++17", "-I" + build.BLOCK, "-Xarch_host",
                           "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", src,
                           os.path.join(build.CSRC, "plan.cpp"), "-o", exe], stderr=subprocess.DEVNULL)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)


# ----------------------------------------------------------------------------- the kernels' instructions
FORBIDDEN = re.compile(r"^\s+(v_(?!mfma_i32_)[a-z0-9_]*_(f16|f32|f64|bf16)\b|v_cvt_(?!pk_[iu]16_[iu]32)|v_rcp|v_rsq|v_sqrt|v_mfma_(?!i32_)|v_smfmac|"
                       r"v_exp|v_log|v_pk_[a-z]+_f|v_dot[0-9]*_f|v_fma|v_mad_f|v_mac_f|v_div_)", re.M)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not installed")
@pytest.mark.parametrize("src", [s for s in build.BLOCK_SOURCES if s.endswith(".hip")])
def test_integer_instructions_only(src, tmp_path):
    """No floating point, matrix products in their integer forms only, no register spilled."""
    out = str(tmp_path / "a.s")
    subprocess.check_call(["hipcc", "-x", "hip", "--cuda-device-only", "-S", os.path.join(build.BLOCK, src), "-o", out]
                          + [f for f in build.FLAGS if f != "-fPIC"], stderr=subprocess.DEVNULL)
    text = open(out).read()
    if ".amdhsa_kernel" not in text:
        assert "__global__" not in open(os.path.join(build.BLOCK, src)).read()
        return
    hits = FORBIDDEN.findall(text)
    assert not hits, hits[:5]
    scratch = re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text)
    assert scratch and all(int(b) == 0 for b in scratch), scratch
    assert ("v_mfma_i32_" in text) == (re.match(r"attention_\w+_\d+\.hip", src) is not None)


def test_every_source_is_built():
    assert sorted(f for f in os.listdir(build.BLOCK) if f.endswith((".hip", ".cpp"))) == sorted(build.BLOCK_SOURCES)
