"""The block operators on the GPU against the oracle's 64-bit integers: every value has to be equal."""
import numpy as np
import pytest

import paper_2511_15369_amd as ip
from oracle import block as ob
from oracle.ref import Dyadic

pytestmark = pytest.mark.gpu


def _cuda(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _dyadic(d):
    return ip.Dyadic(d.m, d.s, d.zp, d.qmin, d.qmax)


def _params(p):
    return ip.AttentionParams(p.variant, p.i0, p.n_shift, p.score_shift, p.causal, _dyadic(p.post))


def _attention(rng, dim, spread, variant=1, causal=1, i0=None, keys=64, cache=False):
    """Parameters for scores of that standard deviation, an exponent of 1 to 4 of them."""
    inv = spread / float(rng.uniform(1, 4))
    shift = max(0, int(np.ceil(np.log2(inv / 1024))))
    i0 = int(i0 or max(16, min(1024, inv / 2 ** shift)))
    n = 0
    while i0 << (n + 1) <= 32639:
        n += 1
    n = int(rng.integers(max(0, n - 3), n + 1))
    post = Dyadic(int(rng.integers(2 ** 13, 2 ** 15)) * int(rng.choice([1, 1, 1, -1])), 21 + 3 * cache - int(np.log2(keys + 1) / 2), int(rng.integers(-9, 9)),
                  -128, int(rng.choice([127, 100])))
    return ob.Attention(variant, i0, n, shift, causal, post)


# ----------------------------------------------------------------------------- attention over prompts
def _packed(rng, q_lens, k_lens, heads, kv_heads, dim, p, fused=True, max_q=None, gap=5, sigma=27, offset=0):
    """Runs a packed problem, rows of other tokens around and between the sequences' rows, and compares all of them."""
    import torch
    def edges(lens):
        return (np.cumsum([0] + list(lens)) + gap).astype(np.int32)
    qo, ko = edges(q_lens), edges(k_lens)
    nq, nk = int(qo[-1]) + gap, int(ko[-1]) + gap
    def int8(n, h):
        return np.clip(np.rint(rng.normal(0, sigma, (n, h, dim))), -128, 127).astype(np.int8)
    q, k, v = int8(nq, heads), int8(nk, kv_heads), int8(nk, kv_heads)
    before = rng.integers(-128, 128, (nq, heads, dim)).astype(np.int8)
    if fused:                                            # views of one tensor, at any byte
        rows = torch.zeros(offset + max(nq, nk) * (heads + 2 * kv_heads) * dim, dtype=torch.int8, device="cuda")
        rows = rows[offset:].view(max(nq, nk), heads + 2 * kv_heads, dim)
        dq, dk, dv = rows[:nq, :heads], rows[:nk, heads:heads + kv_heads], rows[:nk, heads + kv_heads:]
        dq.copy_(_cuda(q)), dk.copy_(_cuda(k)), dv.copy_(_cuda(v))
    else:
        dq, dk, dv = _cuda(q), _cuda(k), _cuda(v)
    out = torch.zeros(offset + nq * (heads + 1) * dim, dtype=torch.int8, device="cuda")[offset:].view(nq, heads + 1, dim)
    out[:, heads] = 77
    out[:, :heads] = _cuda(before)
    most = max(q_lens) if max_q is None else max_q
    ip.attention_i8(dq, dk, dv, _cuda(qo), _cuda(ko), len(q_lens), most, out[:, :heads], _params(p))
    torch.cuda.synchronize()
    want = ob.packed(q, k, v, qo, ko, most, p, before)
    got = out.cpu().numpy()
    assert np.array_equal(got[:, :heads], want)
    assert np.all(got[:, heads] == 77)
    return want


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("variant", [0, 1, 2])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("heads", [3, 6, 27])             # 10 sequences of up to two tiles of 128 queries: either kernel
def test_packed_lengths(dim, variant, causal, heads):
    """Lengths around the tiles' edges, sequences without queries, without keys, with fewer keys than queries."""
    rng = np.random.default_rng([dim, variant, causal, heads])
    q_lens = [1, 0, 31, 33, 64, 129, 65, 5, 130, 1]
    k_lens = [1, 4, 31, 40, 63, 129, 257, 0, 100, 300]
    p = _attention(rng, dim, 27 * 27 * dim ** 0.5, variant, causal, keys=100)
    _packed(rng, q_lens, k_lens, heads, heads // 3, dim, p, offset=int(rng.integers(0, 16)))


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (8, 1), (5, 5), (40, 8), (12, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_heads(heads, kv_heads, dim):
    rng = np.random.default_rng([heads, dim])
    for fused in (False, True):
        _packed(rng, [70, 3, 40], [70, 9, 41], heads, kv_heads, dim, _attention(rng, dim, 27 * 27 * dim ** 0.5, keys=40), fused)


@pytest.mark.parametrize("n,dim,variant,heads", [(1000, 128, 0, 2), (1537, 64, 1, 2), (2111, 32, 2, 2), (700, 96, 1, 2), (1000, 128, 1, 32), (1537, 64, 0, 20),
                                                 (1999, 32, 1, 16), (700, 96, 2, 48), (641, 128, 2, 48), (1537, 64, 1, 40), (1999, 32, 0, 40)])
@pytest.mark.parametrize("causal", [0, 1])
def test_long_prompts(n, dim, variant, heads, causal):
    rng = np.random.default_rng([n, causal])
    _packed(rng, [n], [n + (37 if causal else 0)], heads, heads // 2, dim, _attention(rng, dim, 27 * 27 * dim ** 0.5, variant, causal, keys=n))


@pytest.mark.parametrize("heads,kv_heads", [(160, 40), (120, 10), (84, 42), (63, 21), (64, 1)])
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
def test_heads_that_share_a_workgroup(heads, kv_heads, dim):
    """Four heads, two or one to a workgroup; sequences of every remainder, of one tile and of several."""
    rng = np.random.default_rng([heads, dim])
    p = _attention(rng, dim, 27 * 27 * dim ** 0.5, 1, int(rng.integers(2)), keys=100)
    _packed(rng, [200, 1, 31, 33, 95, 129, 64], [200, 1, 40, 33, 95, 160, 64], heads, kv_heads, dim, p, offset=3)
    _packed(rng, [60, 1, 31, 33, 8, 64, 2, 50], [60, 1, 40, 20, 8, 64, 130, 50], heads, kv_heads, dim, p)


@pytest.mark.parametrize("n,k", [(1, 1), (3, 508), (5, 509), (1, 3000), (32, 255), (33, 256), (2, 257), (4, 2049)])
def test_few_queries_of_many_keys(n, k):
    """Keys divided over wavefronts: around one block each, and where a sum no longer fits with its upper half in one."""
    rng = np.random.default_rng([n, k])
    for dim in (32, 64, 96, 128):
        for causal in (0, 1):
            _packed(rng, [n], [k], 2, 1, dim, _attention(rng, dim, 27 * 27 * dim ** 0.5, 1, causal, keys=k))


def test_more_queries_than_max_q_and_wild_offsets_stay():
    rng = np.random.default_rng(3)
    _packed(rng, [50, 200, 7], [60, 200, 90], 4, 2, 64, _attention(rng, 64, 27 * 27 * 8), max_q=40)


@pytest.mark.parametrize("i0", [16, 17, 255, 256, 1023, 1024])
@pytest.mark.parametrize("sigma", [3, 27, 200])
def test_extreme_scores_and_scales(i0, sigma):
    """Scales from the coarsest to the finest, bytes from small ones to all at their ends."""
    rng = np.random.default_rng([i0, sigma])
    for variant in (0, 1, 2):
        for shift in (0, 1, 5, 16):
            p = _attention(rng, 128, 27 * 27 * 11.0, variant, 1, i0)
            p.score_shift = shift
            _packed(rng, [40], [67], 2, 1, 128, p, sigma=sigma)
            if shift == 5:
                _packed(rng, [40] * 6, [67] * 6, 48, 1, 32, p, sigma=sigma)


def test_bytes_at_their_ends():
    """All -128: the largest products, the largest sums of weights, every weight at its most."""
    import torch
    n = 4096
    for q, k, v in ((-128, -128, -128), (-128, 127, 127), (0, 0, -128), (127, 127, 127)):
        for i0 in (1019, 1018):                  # 1019 << 5 is the largest weight but 31
            p = ob.Attention(1, i0, 5, 4, 0, Dyadic(1, 8, 0, -128, 127))
            for heads in (1, 256):
                t = [torch.full((m, h, 128), x, dtype=torch.int8, device="cuda") for m, h, x in ((40, heads, q), (n, 1, k), (n, 1, v))]
                out = torch.empty_like(t[0])
                ip.attention_i8(*t, None, None, 1, 40, out, _params(p))
                assert torch.all(out == v)               # (rounding down by f may take a unit of 2^-8, never half of one)


def test_longest_keys():
    """65536 keys; one more is not served and leaves its rows."""
    import torch
    rng = np.random.default_rng(5)
    n = 65537
    q, k, v = (np.clip(np.rint(rng.normal(0, 30, (m, 1, 32))), -127, 127).astype(np.int8) for m in (6, n, n))
    p = _attention(rng, 32, 900 * 32 ** 0.5, 1, 0, keys=n)
    dq, dk, dv = _cuda(q), _cuda(k), _cuda(v)
    out = torch.full_like(dq, 55)
    qo, ko = np.array([0, 3, 6], np.int32), np.array([0, 65536, 65536], np.int32)
    ip.attention_i8(dq, dk, dv, _cuda(qo), _cuda(ko), 2, 3, out, _params(p))
    assert np.array_equal(out.cpu().numpy(), ob.packed(q, k, v, qo, ko, 3, p, np.full_like(q, 55)))
    ip.attention_i8(dq, dk, dv, _cuda(np.array([0, 6], np.int32)), _cuda(np.array([0, n], np.int32)), 1, 6, out.fill_(55), _params(p))
    assert torch.all(out == 55)


def test_equal_lengths_without_offsets():
    import torch
    rng = np.random.default_rng(6)
    for n, lq, lk in ((3, 197, 197), (5, 49, 49), (2, 1, 30), (4, 16, 0), (70, 49, 49), (65, 16, 0)):
        q, k, v = (rng.integers(-90, 90, (n * m, 4, 64)).astype(np.int8) for m in (lq, lk, lk))
        p = _attention(rng, 64, 52 * 52 * 8.0, causal=0, keys=lk)
        out = torch.full((n * lq, 4, 64), 9, dtype=torch.int8, device="cuda")
        ip.attention_i8(_cuda(q), _cuda(k), _cuda(v), None, None, n, lq, out, _params(p))
        want = np.concatenate([ob.attention(q[i * lq:(i + 1) * lq], k[i * lk:(i + 1) * lk], v[i * lk:(i + 1) * lk], p) for i in range(n)])
        assert np.array_equal(out.cpu().numpy(), want)


def test_the_softmax_of_the_library_gives_the_same_weights():
    """The fused operator beside the library's softmax: products, softmax_i32 and products again with probabilities cut to
    eight bits lie within what that cut allows (each probability is at most a unit of 2^-7 too small)."""
    import torch
    rng = np.random.default_rng(8)
    n, d = 197, 64
    q, k, v = (np.clip(np.rint(rng.normal(0, 27, (n, 1, d))), -127, 127).astype(np.int8) for _ in range(3))
    p = ob.Attention(1, 800, 5, 0, 0, Dyadic(1, 8, 0, -128, 127))
    out = torch.empty((n, 1, d), dtype=torch.int8, device="cuda")
    ip.attention_i8(_cuda(q), _cuda(k), _cuda(v), None, None, 1, n, out, _params(p))
    scores = (q[:, 0].astype(np.int32) @ k[:, 0].astype(np.int32).T).astype(np.int32)
    probs = torch.empty((n, n), dtype=torch.uint8, device="cuda")
    sp = ip.SoftmaxParams(1, 800, 5, 30, 8, 1, 0, ip.Dyadic(1, 0, 0, 0, 255), 0, 0)
    ip.softmax_i32(_cuda(scores), None, 0, probs, n, n, sp)
    probs = probs.cpu().numpy().astype(np.int64)
    w = ob.weights(scores, np.full(n, n), p)
    assert np.array_equal(probs, (((1 << 30) // w.sum(1))[:, None] * w) >> 23)
    cut = 1 + 2.0 ** 7 * n * 2.0 ** -15                        # per probability: the floor, and f's
    off = np.abs(out.cpu().numpy()[:, 0] - (probs @ v[:, 0].astype(np.int64)) / 128.0)
    assert np.all(off <= cut / 128 * np.abs(v[:, 0].astype(np.int64)).sum(0) + 0.5 + 2.0 ** -7)


# ----------------------------------------------------------------------------- the cache
def _cache(rng, pages, kv_heads, page, dim):
    shape, g = (pages, kv_heads, page), ob.groups(dim)
    return [rng.integers(0, 256, shape + (dim // 2,)).astype(np.uint8), rng.integers(0, 129, shape + (g,)).astype(np.uint8),
            rng.integers(0, 256, (pages, kv_heads, dim // 2, page)).astype(np.uint8), rng.integers(0, 129, shape + (g,)).astype(np.uint8)]


def _on_gpu(cache):
    d = [_cuda(x) for x in cache]
    return d, ip.cache_i4(*d, cache[0].shape[-1] * 2)


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("page", [16, 64, 4096])
def test_store(dim, page):
    """Scattered and consecutive slots, padding, slots outside the cache; what is not named stays."""
    rng = np.random.default_rng([dim, page])
    pages = 3 if page == 4096 else 20
    for tokens, consecutive in ((1, 0), (7, 0), (70, 0), (230, 1), (64, 1), (257, 2)):
        kv_heads = int(rng.choice([1, 2, 3, 8]))
        cache = _cache(rng, pages, kv_heads, page, dim)
        if consecutive == 1:
            slots = np.arange(tokens) + int(rng.integers(0, pages * page - tokens))
        else:
            slots = rng.permutation(pages * page)[:tokens]
        slots = slots.astype(np.int32)
        if tokens > 1:
            at = rng.permutation(tokens)[:5]
            slots[at] = (-1, pages * page, -2 ** 31, 2 ** 31 - 1, -7)
        rows = rng.integers(-128, 128, (tokens, 2 * kv_heads + 1, dim)).astype(np.int8)
        rows[rng.random(rows.shape[:2]) < 0.1] = 0
        rows[rng.random(rows.shape[:2]) < 0.1] //= 40
        drows = _cuda(rows)
        d, c = _on_gpu(cache)
        ip.cache_store_i4(c, drows[:, :kv_heads], drows[:, kv_heads:2 * kv_heads], _cuda(slots), tokens)
        want = ob.store(cache, rows[:, :kv_heads], rows[:, kv_heads:2 * kv_heads], slots)
        for a, b in zip(d, want):
            assert np.array_equal(a.cpu().numpy(), b)


def test_store_every_byte():
    """Every value beside every step."""
    rng = np.random.default_rng(1)
    x = np.zeros((129, 1, 128), np.int8)
    y = np.zeros((129, 1, 128), np.int8)
    for a in range(129):
        v = np.arange(-a, a + 1)[:128 if a < 64 else None]
        s = -1 if a == 128 else 1
        x[a, 0, :64], x[a, 0, 64:] = rng.permutation(np.resize(v, 256))[:64], np.resize(v, 256)[64:128]
        y[a, 0, :64], y[a, 0, 64:] = np.resize(v, 256)[128:192], np.resize(v, 256)[192:]
        x[a, 0, 5], y[a, 0, 70] = np.int8(s * a), np.int8(-a)
    cache = _cache(rng, 9, 1, 16, 128)
    d, c = _on_gpu(cache)
    slots = rng.permutation(144)[:129].astype(np.int32)
    ip.cache_store_i4(c, _cuda(x), _cuda(y), _cuda(slots), 129)
    for a, b in zip(d, ob.store(cache, x, y, slots)):
        assert np.array_equal(a.cpu().numpy(), b)


def _attend(rng, lengths, heads, kv_heads, dim, page, t, p, spare=0, bad=(), sigma=27, codes=None, strided=True):
    import torch
    most = max(1, max(-(-max(n, 0) // page) for n in lengths)) + spare
    pages = sum(-(-max(n, 0) // page) for n in lengths) + 2
    cache = _cache(rng, pages, kv_heads, page, dim) if codes is None else codes(pages)
    table = rng.integers(-9, 1 << 30, (len(lengths), most)).astype(np.int32)        # what lies behind a length is not read
    order, at = rng.permutation(pages), 0
    for i, n in enumerate(lengths):
        m = -(-max(n, 0) // page)
        table[i, :m] = order[at:at + m]
        at += m
    for i, j, v in bad:
        table[i, j] = v
    q = np.clip(np.rint(rng.normal(0, sigma, (len(lengths) * t, heads, dim))), -128, 127).astype(np.int8)
    dq = _cuda(np.concatenate([q, q[:, :1]], 1))[:, :heads] if strided else _cuda(q)
    out = torch.full((len(lengths) * t + 1, heads + 1, dim), 77, dtype=torch.int8, device="cuda")
    d, c = _on_gpu(cache)
    size = ip.attention_cache_i4_workspace(c, len(lengths), t, heads, most)
    work = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    for _ in range(2):                                   # what a call leaves in the workspace means nothing to the next
        ip.attention_cache_i4(dq, c, _cuda(table), _cuda(np.array(lengths, np.int32)), len(lengths), t, out[:-1, :heads], work[:size],
                              _params(p))
        got = out.cpu().numpy()
        assert np.array_equal(got[:-1, :heads], ob.attention_cache(q, cache, table, lengths, t, p))
        assert np.all(got[-1] == 77) and np.all(got[:, heads] == 77) and torch.all(work[size:] == 0xA5)


def _spread(dim):
    return 27 * 4.6 * 64 * dim ** 0.5


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("variant", [0, 1, 2])
@pytest.mark.parametrize("t", [1, 3])
def test_cache_attention_lengths(dim, variant, t):
    """Lengths around tiles and pages, none, fewer tokens than queries, negative and beyond the table."""
    rng = np.random.default_rng([dim, variant, t])
    for page in (16, 64):
        p = _attention(rng, dim, _spread(dim), variant, 1, cache=True)
        _attend(rng, [0, 1, 2, 15, 16, 17, 63, 64, 65, 129, 255, 256, 257, 600, -4], 6, 2, dim, page, t, p, spare=int(rng.integers(0, 3)))


@pytest.mark.parametrize("heads,kv_heads,t", [(1, 1, 1), (8, 8, 1), (16, 1, 1), (17, 1, 1), (32, 8, 4), (64, 8, 4), (7, 1, 5), (40, 8, 2),
                                              (33, 1, 2), (4, 2, 64)])
def test_cache_attention_columns(heads, kv_heads, t):
    rng = np.random.default_rng([heads, t])
    for causal in (0, 1):
        _attend(rng, [300, 70, 5], heads, kv_heads, 128, 32, t, _attention(rng, 128, _spread(128), 1, causal, cache=True))


@pytest.mark.parametrize("heads,n", [(4, 1023), (4, 1024), (4, 1025), (40, 512), (40, 513), (40, 1024), (24, 1024), (4, 64), (4, 65)])
def test_cache_attention_at_the_limits_of_one_workgroup(heads, n):
    rng = np.random.default_rng([heads, n])
    for dim in (32, 64, 96, 128):
        _attend(rng, [n, 3, n - 1], heads, 2, dim, 16, 1, _attention(rng, dim, _spread(dim), 2, 1, keys=n, cache=True))


@pytest.mark.parametrize("n,dim,t,heads", [(1500, 128, 1, 4), (2600, 64, 2, 8), (5000, 128, 4, 8), (9000, 32, 1, 2), (20011, 96, 1, 2)])
def test_cache_attention_long(n, dim, t, heads):
    rng = np.random.default_rng(n)
    for lengths in ([n], [n, 40, n // 2, n - 1]):
        _attend(rng, lengths, heads, 2, dim, 64, t, _attention(rng, dim, _spread(dim), 1, 1, keys=n, cache=True))


def test_cache_attention_longest():
    """131072 tokens: the sums of weights pass 2^31."""
    rng = np.random.default_rng(2)
    n, page = 131072, 4096
    p = ob.Attention(0, 1000, 5, 20, 1, Dyadic(20000, 20, 0, -128, 127))
    _attend(rng, [n, 3], 2, 1, 32, page, 1, p)


@pytest.mark.parametrize("i0", [1018, 1019])
def test_cache_attention_every_weight_at_its_most(i0):
    """Equal scores of as many keys as there may be: the weights add up to more than 2^31."""
    rng = np.random.default_rng(i0)
    p = ob.Attention(1, i0, 5, 0, 1, Dyadic(32000, 19, 0, -128, 127))
    _attend(rng, [131072, 70000, 131071], 3, 1, 32, 256, 1, p, sigma=0)


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("page,heads", [(16, 5), (32, 3), (128, 4), (256, 20), (4096, 9)])
def test_cache_attention_page_sizes(dim, page, heads):
    """Tiles of several pages, of one, pages of many tiles; over one workgroup and several."""
    rng = np.random.default_rng([dim, page])
    p = _attention(rng, dim, _spread(dim), 1, 1, cache=True)
    _attend(rng, [900, 641, 63, 130], heads, 1, dim, page, 1, p)
    _attend(rng, [4500, 4097, 1, 2111], heads, 1, dim, page, 2, p, spare=1)


def test_cache_attention_pages_that_are_not_there():
    """Tokens in a page outside the cache count as masked; a sequence of such pages sees nothing."""
    rng = np.random.default_rng(4)
    for page, lengths in ((16, [100, 64, 33]), (64, [500, 64, 200])):
        m = -(-lengths[1] // page)
        bad = [(0, 1, -1), (0, 3, 2 ** 31 - 1), (2, 0, -2 ** 31)] + [(1, j, 1 << 20) for j in range(m)]
        for t in (1, 2):
            _attend(rng, lengths, 4, 2, 64, page, t, _attention(rng, 64, _spread(64), 1, 1, cache=True), bad=bad)


@pytest.mark.parametrize("i0,shift", [(16, 20), (16, 0), (1024, 0), (777, 9), (1019, 20)])
def test_cache_attention_extremes(i0, shift):
    """Codes and steps at their ends, queries of -128."""
    rng = np.random.default_rng([i0, shift])
    n = 0
    while i0 << (n + 1) <= 32639:
        n += 1
    for fill, step in ((0x99, 128), (0x77, 128), (0x88, 128), (0x00, 0), (0x79, 1)):
        codes = lambda pages: [np.full((pages, 1, 32, 64), fill, np.uint8), np.full((pages, 1, 32, 2), step, np.uint8),  # noqa: E731
                               np.full((pages, 1, 64, 32), fill, np.uint8), np.full((pages, 1, 32, 2), step, np.uint8)]
        p = ob.Attention(1, i0, n, shift, 1, Dyadic(30000, 22, 1, -128, 127))
        _attend(rng, [700, 33], 2, 1, 128, 32, 1, p, sigma=500, codes=codes)


# ----------------------------------------------------------------------------- norm and row scales
def _norm(rng, rows, cols, scales, x=True, residual=True, keep=True, in_place=False, mag=9000, eps=3, in_ms=(20000, 16), post=None, gain=None, offset=0):
    import torch
    wide = 1 + 40 * (rng.random(cols) < 0.01)
    hx = np.clip(rng.normal(0, 3 * mag, (rows, cols)), -2 ** 31, 2 ** 31 - 1).astype(np.int64).astype(np.int32) if x else None
    hr = np.clip(rng.normal(0, mag, (rows, cols)) * wide, -2 ** 31, 2 ** 31 - 1).astype(np.int64).astype(np.int32) if residual else None
    if rows > 2:
        for h in (hx, hr):
            if h is not None:
                h[1] = 0
    g = rng.integers(-2 ** 15, 2 ** 15, cols).astype(np.int16) if gain is None else np.full(cols, gain, np.int16)
    post = post or Dyadic(int(rng.integers(2 ** 14, 2 ** 15)), 29, int(rng.integers(-3, 4)), -128, 127)
    want = ob.rmsnorm(hx, hr, g, *in_ms, eps, post, scales)

    def at(h, kind):
        if h is None:
            return None
        t = torch.zeros(h.size + offset, dtype=kind, device="cuda")[offset:].view(h.shape)
        return t.copy_(_cuda(h))

    dx, dr = at(hx, torch.int32), at(hr, torch.int32)
    out = torch.full((rows * cols + offset + 16,), 77, dtype=torch.int8, device="cuda")
    stream = (dr if in_place else torch.empty((rows, cols), dtype=torch.int32, device="cuda")) if keep else None
    s = torch.full((rows + 1,), 77, dtype=torch.int32, device="cuda") if scales else None
    ip.rmsnorm_i32(dx, dr, at(g, torch.int16), stream, out[offset:], s, rows, cols, ip.RmsnormParams(*in_ms, eps, _dyadic(post)))
    got = out.cpu().numpy()
    assert np.array_equal(got[offset:offset + rows * cols].reshape(rows, cols), want[0])
    assert np.all(got[:offset] == 77) and np.all(got[offset + rows * cols:] == 77)
    if keep:
        assert np.array_equal(stream.cpu().numpy(), want[1])
    if residual and not in_place:
        assert np.array_equal(dr.cpu().numpy(), hr)
    if scales:
        assert np.array_equal(s.cpu().numpy()[:rows], want[2]) and int(s[rows]) == 77


@pytest.mark.parametrize("cols", [1, 2, 3, 63, 64, 65, 255, 256, 257, 1000, 1023, 1024, 2047, 2048, 2052, 4096, 4100, 5120, 8191, 8192, 8193, 12288, 12289, 16383, 16384])
@pytest.mark.parametrize("scales", [False, True])
def test_norm_lengths(cols, scales):
    rng = np.random.default_rng([cols, scales])
    for rows in (1, 5):
        _norm(rng, rows, cols, scales, in_place=bool(rng.integers(2)), offset=int(rng.choice([0, 0, 1, 3])))


@pytest.mark.parametrize("rows", [1, 2, 63, 300, 2100])
def test_norm_rows(rows):
    rng = np.random.default_rng(rows)
    for cols in (48, 384, 770):
        for scales in (False, True):
            _norm(rng, rows, cols, scales, in_place=scales)


@pytest.mark.parametrize("scales", [False, True])
@pytest.mark.parametrize("cols", [130, 4096])
def test_norm_inputs(cols, scales):
    """Without a product, without a residual, without the stream's new value; in place."""
    rng = np.random.default_rng([cols, scales])
    _norm(rng, 4, cols, scales, x=False)
    _norm(rng, 4, cols, scales, x=False, in_place=True)
    _norm(rng, 4, cols, scales, residual=False)
    _norm(rng, 4, cols, scales, residual=False, keep=False)
    _norm(rng, 4, cols, scales, keep=False)


@pytest.mark.parametrize("mag", [0.4, 3, 2 ** 20, 2 ** 24, 2 ** 30])
@pytest.mark.parametrize("cols", [70, 3000])
def test_norm_magnitudes(mag, cols):
    """Streams of small values, saturated ones; eps from none to the most; the steps' shifts from 0 to 62."""
    rng = np.random.default_rng([int(mag * 10), cols])
    for eps in (0, 1, 2 ** 46):
        for in_ms in ((1, 0), (-32767, 15), (32767, 0), (5, 62)):
            _norm(rng, 3, cols, bool(rng.integers(2)), mag=mag, eps=eps, in_ms=in_ms, in_place=True)
    for post in (Dyadic(1, 0, 0, -128, 127), Dyadic(-32767, 40, 7, -100, 100), Dyadic(32767, 62, 2 ** 24, -128, 127), Dyadic(32767, 0, -2 ** 24, -5, 5)):
        for gain in (-2 ** 15, 2 ** 15 - 1, 0, 1):
            _norm(rng, 2, cols, False, mag=mag, post=post, gain=gain)
            _norm(rng, 2, cols, True, mag=mag, gain=gain)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 1000), (700, 33), (64, 6144), (5, 65536), (33, 1023), (2, 100001)])
@pytest.mark.parametrize("signed", [0, 1])
def test_requant_rows(rows, cols, signed):
    import torch
    rng = np.random.default_rng([rows, cols, signed])
    for offset in (0, 1, 3):
        shift = int(rng.choice([0, 1, 16, 22, 30, 40, 62]))
        x = rng.integers(-2 ** 31, 2 ** 31, (rows, cols)) if rng.random() < 0.3 else rng.normal(0, 60000, (rows, cols))
        x = x.astype(np.int64).astype(np.int32)
        s = rng.integers(-2 ** 31, 2 ** 31, rows).astype(np.int32) if rng.random() < 0.4 else rng.integers(2 ** 20, 2 ** 25, rows).astype(np.int32)
        p = Dyadic(int(rng.integers(-2 ** 15 + 1, 2 ** 15)), int(rng.choice([0, 8, 20, 26, 45, 62])), int(rng.integers(-20, 20)), *((-128, 127) if signed else (3, 255)))
        out = torch.full((rows * cols + offset + 16,), 77, dtype=torch.int8 if signed else torch.uint8, device="cuda")
        dx = torch.zeros(rows * cols + offset, dtype=torch.int32, device="cuda")[offset:].copy_(_cuda(x).view(-1))
        ip.requant_rows(dx, _cuda(s), out[offset:], rows, cols, shift, signed, _dyadic(p))
        got = out.cpu().numpy()
        assert np.array_equal(got[offset:offset + rows * cols].reshape(rows, cols), ob.requant_rows(x, s, shift, p))
        assert np.all(got[:offset] == 77) and np.all(got[offset + rows * cols:] == 77)


# ----------------------------------------------------------------------------- together, as a model runs them
class _Block:
    """One transformer block in integers over a 4-bit cache: norm -> product -> row scales -> cache and attention ->
    product -> norm -> product -> GELU; prompts by attention_i8, single tokens by attention_cache_i4."""
    heads, kv_heads, dim, cols, hidden, page, pages = 8, 2, 64, 320, 512, 32, 24

    def __init__(self, seed):
        rng = self.rng = np.random.default_rng(seed)
        width = (self.heads + 2 * self.kv_heads) * self.dim
        w8 = lambda *s: np.clip(np.rint(rng.normal(0, 30, s)), -127, 127).astype(np.int8)  # noqa: E731
        self.w_qkv, self.w_out, self.w_up = w8(self.cols, width), w8(self.heads * self.dim, self.cols), w8(self.cols, self.hidden)
        self.gain = rng.integers(3000, 20000, self.cols).astype(np.int16)
        self.norm = dict(in_m=20000, in_s=20, eps=4, post=Dyadic(20000, 29, 0, -128, 127))
        self.rows = dict(shift=22, p=Dyadic(20000, 26, 0, -128, 127))
        self.prompt = ob.Attention(1, 700, 5, 5, 1, Dyadic(20000, 21, 0, -128, 127))
        self.decode = ob.Attention(1, 900, 5, 7, 1, Dyadic(20000, 24, 0, -128, 127))
        self.gelu = ip.gelu_prepare(0.03, 0.03, 0, 0, 1, 255)
        self.gelu.pre_m, self.gelu.pre_s = 20000, 24

    # a product of codes: exact in float64 on either side
    @staticmethod
    def _product(a, b):
        return (a.double() @ b.double()).int()

    def on_gpu(self):
        import torch
        self.d = {k: _cuda(getattr(self, k)) for k in ("w_qkv", "w_out", "w_up", "gain")}
        self.cache_np = _cache(self.rng, self.pages, self.kv_heads, self.page, self.dim)
        self.cache_d, self.cache = _on_gpu(self.cache_np)
        size = ip.attention_cache_i4_workspace(self.cache, 3, 1, self.heads, 8)
        self.work = torch.empty((size,), dtype=torch.uint8, device="cuda")

    def gpu(self, x, stream, slots, attend):
        import torch
        n = stream.shape[0]
        new = lambda kind, *s: torch.empty(s, dtype=kind, device="cuda")  # noqa: E731
        np_ = ip.RmsnormParams(self.norm["in_m"], self.norm["in_s"], self.norm["eps"], _dyadic(self.norm["post"]))
        codes, scales = new(torch.int8, n, self.cols), new(torch.int32, n)
        ip.rmsnorm_i32(x, stream, self.d["gain"], stream, codes, scales, n, self.cols, np_)
        acc = self._product(codes, self.d["w_qkv"])
        qkv = new(torch.int8, n, self.heads + 2 * self.kv_heads, self.dim)
        ip.requant_rows(acc, scales, qkv, n, acc.shape[1], self.rows["shift"], 1, _dyadic(self.rows["p"]))
        q, k, v = qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv_heads], qkv[:, self.heads + self.kv_heads:]
        ip.cache_store_i4(self.cache, k, v, slots, n)
        o = new(torch.int8, n, self.heads, self.dim)
        attend(q, k, v, o)
        acc = self._product(o.view(n, -1), self.d["w_out"])
        codes2 = new(torch.int8, n, self.cols)
        ip.rmsnorm_i32(acc, stream, self.d["gain"], stream, codes2, None, n, self.cols, np_)
        up = self._product(codes2, self.d["w_up"])
        y = new(torch.int8, n, self.hidden)
        ip.gelu_i32(up.view(-1), y, up.numel(), self.gelu)
        return [codes, scales, qkv, o, codes2, stream, y]

    def oracle(self, x, stream, slots, attend):
        from oracle import ref
        n = self.norm
        codes, stream, scales = ob.rmsnorm(x, stream, self.gain, n["in_m"], n["in_s"], n["eps"], n["post"], True)
        acc = codes.astype(np.int64) @ self.w_qkv.astype(np.int64)
        qkv = ob.requant_rows(acc.astype(np.int32), scales, self.rows["shift"], self.rows["p"]).astype(np.int8)
        qkv = qkv.reshape(len(codes), -1, self.dim)
        q, k, v = qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv_heads], qkv[:, self.heads + self.kv_heads:]
        self.cache_np = ob.store(self.cache_np, k, v, slots)
        o = attend(q, k, v)
        acc = (o.reshape(len(codes), -1).astype(np.int64) @ self.w_out.astype(np.int64)).astype(np.int32)
        codes2, stream, _ = ob.rmsnorm(acc, stream, self.gain, n["in_m"], n["in_s"], n["eps"], n["post"], False)
        up = (codes2.astype(np.int64) @ self.w_up.astype(np.int64)).astype(np.int32)
        g = self.gelu
        gp = ref.GeluParams(g.variant, g.q_b, g.q_c, g.k, g.zp_in, g.max_abs_q, g.pre_m, g.pre_s, Dyadic(*[getattr(g.post, f) for f in ("m", "s", "zp", "qmin", "qmax")]))
        return [codes, scales, qkv, o, codes2, stream, ref.gelu_i32(up, gp)]


def test_a_block_over_prompts_then_tokens():
    """Three prompts go through a block and into the cache, then two steps of one token each, the second captured
    into a graph and replayed with other inputs; every tensor on the way is compared."""
    import torch
    b = _Block(0)
    b.on_gpu()
    lens, most = [70, 1, 33], 8
    tables = np.full((3, most), -1, np.int32)
    order = b.rng.permutation(b.pages)
    for i in range(3):
        tables[i, :4] = order[4 * i:4 * i + 4]
    slot = lambda i, t: tables[i, t // b.page] * b.page + t % b.page  # noqa: E731
    total = sum(lens)
    stream = b.rng.integers(-20000, 20000, (total, b.cols)).astype(np.int32)
    slots = np.array([slot(i, t) for i in range(3) for t in range(lens[i])], np.int32)
    offsets = np.cumsum([0] + lens).astype(np.int32)
    d_off = _cuda(offsets)
    got = b.gpu(None, _cuda(stream), _cuda(slots),
                lambda q, k, v, o: ip.attention_i8(q, k, v, d_off, d_off, 3, max(lens), o, _params(b.prompt)))
    want = b.oracle(None, stream, slots, lambda q, k, v: ob.packed(q, k, v, offsets, offsets, max(lens), b.prompt, np.zeros_like(q)))
    assert sum(np.count_nonzero(w) for w in want) > 0.5 * sum(w.size for w in want)
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy().reshape(w.shape), w)

    d_tables = _cuda(tables)
    d_x, d_stream, d_slots, d_lengths = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((3, b.cols), (3, b.cols), (3,), (3,)))

    def step():
        return b.gpu(d_x, d_stream, d_slots, lambda q, k, v, o: ip.attention_cache_i4(q, b.cache, d_tables, d_lengths, 3, 1, o, b.work,
                                                                                      _params(b.decode)))

    graph, outs = None, None
    for token in range(4):
        x, stream = b.rng.integers(-10 ** 6, 10 ** 6, (3, b.cols)).astype(np.int32), b.rng.integers(-20000, 20000, (3, b.cols)).astype(np.int32)
        slots = np.array([slot(i, lens[i]) for i in range(3)], np.int32)
        lens = [n + 1 for n in lens]
        for d, h in ((d_x, x), (d_stream, stream), (d_slots, slots), (d_lengths, np.array(lens, np.int32))):
            d.copy_(_cuda(h))
        if token == 0:
            outs = step()
        else:
            if graph is None:
                torch.cuda.synchronize()
                held = d_stream.clone()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    outs = step()
                d_stream.copy_(held)
            graph.replay()
        torch.cuda.synchronize()
        want = b.oracle(x, stream, slots, lambda q, k, v: ob.attention_cache(q, b.cache_np, tables, lens, 1, b.decode))
        for g, w in zip(outs, want):
            assert np.array_equal(g.cpu().numpy().reshape(w.shape), w)
    for a, w in zip(b.cache_d, b.cache_np):
        assert np.array_equal(a.cpu().numpy(), w)


@pytest.mark.parametrize("native", [True, False])
def test_either_binding(native, monkeypatch):
    """The native call module and ctypes take the same arguments and make the same calls."""
    import torch
    b = _Block(1)
    b.on_gpu()
    ip.requant_rows(*[torch.zeros(s, dtype=t, device="cuda") for s, t in (((1, 8), torch.int32), (1, torch.int32), ((1, 8), torch.int8))], 1, 8, 1, 1,
                    ip.Dyadic(1, 0, 0, -128, 127))       # (the module is bound with a process's first call)
    if not native:
        monkeypatch.setattr(ip.binding, "_fast", None)
    elif ip.binding._fast is None:
        pytest.skip("the native call module is not built")
    n = 40
    stream, slots = b.rng.integers(-20000, 20000, (n, b.cols)).astype(np.int32), b.rng.permutation(b.pages * b.page)[:n].astype(np.int32)
    off = np.array([0, n], np.int32)
    got = b.gpu(None, _cuda(stream), _cuda(slots), lambda q, k, v, o: ip.attention_i8(q, k, v, _cuda(off), _cuda(off), 1, n, o, _params(b.prompt)))
    want = b.oracle(None, stream, slots, lambda q, k, v: ob.packed(q, k, v, off, off, n, b.prompt, np.zeros_like(q)))
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy().reshape(w.shape), w)
    tables, lengths = b.rng.permutation(b.pages)[None, :8].astype(np.int32), [250]
    q = b.rng.integers(-90, 90, (1, b.heads, b.dim)).astype(np.int8)
    o = torch.empty(q.shape, dtype=torch.int8, device="cuda")
    ip.attention_cache_i4(_cuda(q), b.cache, _cuda(tables), _cuda(np.array(lengths, np.int32)), 1, 1, o, b.work, _params(b.decode))
    assert np.array_equal(o.cpu().numpy(), ob.attention_cache(q, b.cache_np, tables, lengths, 1, b.decode))
    if not native:
        test_the_binding_refuses()


# ----------------------------------------------------------------------------- sizes that pass 32 bits, launches of more workgroups than one may have
def test_rows_past_32_bits():
    """Tokens 2 MiB apart: the last rows lie behind 4 GiB."""
    import torch
    rng = np.random.default_rng(11)
    n, heads, kv_heads, dim, apart = 2200, 2, 1, 64, 2 << 20
    rows = [torch.empty(n * apart, dtype=torch.int8, device="cuda").view(n, apart) for _ in range(2)]
    view = lambda t, at, h: t[:, at:at + h * dim].unflatten(1, (h, dim))  # noqa: E731
    q, k, v = (rng.integers(-60, 60, (n, h, dim)).astype(np.int8) for h in (heads, kv_heads, kv_heads))
    dq, dk, dv, out = view(rows[0], 8, heads), view(rows[0], 500, kv_heads), view(rows[0], 701, kv_heads), view(rows[1], 77, heads)
    for d, h in ((dq, q), (dk, k), (dv, v)):
        d.copy_(_cuda(h))
    p = _attention(rng, dim, 1200 * dim ** 0.5, keys=n)
    ip.attention_i8(dq, dk, dv, None, None, 1, n, out, _params(p))
    assert np.array_equal(out.cpu().numpy(), ob.attention(q, k, v, p))
    cache = _cache(rng, n // 16 + 1, kv_heads, 16, dim)
    d, c = _on_gpu(cache)
    slots = rng.permutation((n // 16 + 1) * 16)[:n].astype(np.int32)
    ip.cache_store_i4(c, dk, dv, _cuda(slots), n)
    for a, w in zip(d, ob.store(cache, k, v, slots)):
        assert np.array_equal(a.cpu().numpy(), w)


def test_a_cache_past_32_bits():
    """Pages behind 4 GiB of codes."""
    import torch
    rng = np.random.default_rng(12)
    pages, page, dim = 1 << 21, 64, 64
    d = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in ((pages, 1, page, 32), (pages, 1, page, 1), (pages, 1, 32, page), (pages, 1, page, 1))]
    c = ip.cache_i4(*d, dim)
    used = np.array([pages - 1, 3, pages // 2 + 1, pages - 2, 0], np.int32)
    n = 5 * page - 7
    k, v = (rng.integers(-90, 90, (n, 1, dim)).astype(np.int8) for _ in range(2))
    slots = (used[np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page).astype(np.int32)
    ip.cache_store_i4(c, _cuda(k), _cuda(v), _cuda(slots), n)
    small = ob.store([np.zeros(t.shape[1:], np.uint8)[None].repeat(5, 0) for t in d], k, v, np.arange(n, dtype=np.int32))
    q = rng.integers(-90, 90, (1, 4, dim)).astype(np.int8)
    for spare in (0, 200):                               # one workgroup, and several
        p = _attention(rng, dim, _spread(dim), cache=True)
        table = np.concatenate([used, np.full(spare, -1)]).astype(np.int32)[None]
        out = torch.empty(q.shape, dtype=torch.int8, device="cuda")
        size = ip.attention_cache_i4_workspace(c, 1, 1, 4, table.shape[1])
        ip.attention_cache_i4(_cuda(q), c, _cuda(table), _cuda(np.array([n], np.int32)), 1, 1, out, torch.empty(size, dtype=torch.uint8, device="cuda"),
                              _params(p))
        assert np.array_equal(out.cpu().numpy(), ob.attention_cache(q, small, np.arange(5, dtype=np.int32)[None], [n], 1, p))


def test_values_past_32_bits():
    """Rows of the norm and of the requantization behind 2^31 values."""
    import torch
    rng = np.random.default_rng(13)
    rows, cols, last = (1 << 20) + 9, 2052, 5
    x, stream = (torch.zeros((rows, cols), dtype=torch.int32, device="cuda") for _ in range(2))
    hx = rng.integers(-2 ** 20, 2 ** 20, (last, cols)).astype(np.int32)
    x[-last:] = _cuda(hx)
    gain, post = rng.integers(-2 ** 14, 2 ** 14, cols).astype(np.int16), Dyadic(20000, 29, 2, -128, 127)
    out, scales = torch.empty((rows, cols), dtype=torch.int8, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    ip.rmsnorm_i32(x, stream, _cuda(gain), stream, out, scales, rows, cols, ip.RmsnormParams(20000, 16, 3, _dyadic(post)))
    want = ob.rmsnorm(hx, np.zeros_like(hx), gain, 20000, 16, 3, post, True)
    for d, w in zip((out, stream, scales), want):
        assert np.array_equal(d[-last:].cpu().numpy(), w) and not d[-last - 3:-last].any()
    ip.requant_rows(x, scales, out, rows, cols, 30, 1, _dyadic(post))
    assert np.array_equal(out[-last:].cpu().numpy(), ob.requant_rows(hx, want[2], 30, post)) and torch.all(out[:-last] == 2)


@pytest.mark.parametrize("cols", [2, 5])
def test_norm_of_more_rows_than_a_launch_has(cols):
    import torch
    rng = np.random.default_rng(cols)
    rows, cut = (1 << 22) + 77, 1 << 21
    x = torch.randint(-2 ** 20, 2 ** 20, (rows, cols), dtype=torch.int32, device="cuda")
    gain, p = _cuda(rng.integers(-2 ** 14, 2 ** 14, cols).astype(np.int16)), ip.RmsnormParams(20000, 16, 3, ip.Dyadic(20000, 29, 0, -128, 127))
    got = [torch.empty((rows, cols), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2)]
    ip.rmsnorm_i32(x, None, gain, None, got[0], scales[0], rows, cols, p)
    for a, b in ((0, cut), (cut, rows)):
        ip.rmsnorm_i32(x[a:b], None, gain, None, got[1][a:b], scales[1][a:b], b - a, cols, p)
    assert torch.equal(*got) and torch.equal(*scales)
    want = ob.rmsnorm(x[-90:].cpu().numpy(), None, gain.cpu().numpy(), 20000, 16, 3, Dyadic(20000, 29, 0, -128, 127), True)
    assert np.array_equal(got[0][-90:].cpu().numpy(), want[0])


def test_prompts_of_more_workgroups_than_a_launch_has():
    """65536 sequences of one token and one of 8960: tiles for the longest of each, over several launches."""
    import torch
    rng = np.random.default_rng(14)
    n, long, dim = 65537, 8960, 32
    at = np.concatenate([np.arange(n), [n - 1 + long]]).astype(np.int32)
    tokens = int(at[-1])
    q, k, v = (rng.integers(-60, 60, (tokens, 1, dim)).astype(np.int8) for _ in range(3))
    p = _attention(rng, dim, 1200 * dim ** 0.5, keys=400)
    d, d_at = [_cuda(x) for x in (q, k, v)], _cuda(at)
    out = torch.empty((tokens, 1, dim), dtype=torch.int8, device="cuda")
    ip.attention_i8(*d, d_at, d_at, n, long, out, _params(p))
    apart = torch.empty_like(out)
    ip.attention_i8(*d, d_at, d_at, n - 1, 1, apart, _params(p))
    ip.attention_i8(*d, d_at[-2:], d_at[-2:], 1, long, apart, _params(p))
    assert torch.equal(out, apart)
    few = np.array([0, 1, 2, 3], np.int32)
    assert np.array_equal(out[:3].cpu().numpy(), ob.packed(q[:3], k[:3], v[:3], few, few, 1, p, np.zeros_like(q[:3])))


def test_short_caches_of_more_workgroups_than_a_launch_has():
    import torch
    rng = np.random.default_rng(15)
    n, heads, dim = 1 << 17, 33, 32
    cache = _cache(rng, 3, heads, 16, dim)
    d, c = _on_gpu(cache)
    p = _attention(rng, dim, _spread(dim), 1, 1, cache=True)
    q = torch.randint(-90, 90, (n, heads, dim), dtype=torch.int8, device="cuda")
    table, lengths = torch.randint(0, 3, (n, 2), dtype=torch.int32, device="cuda"), torch.randint(0, 33, (n,), dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]
    size = ip.attention_cache_i4_workspace(c, n, 1, heads, 2)
    assert size > 0 and ip.attention_cache_i4_workspace(c, n // 2, 1, heads, 2) == 0
    ip.attention_cache_i4(q, c, table, lengths, n, 1, outs[0], torch.empty(size, dtype=torch.uint8, device="cuda"), _params(p))
    for a in (0, n // 2):
        b = a + n // 2
        ip.attention_cache_i4(q[a:b], c, table[a:b], lengths[a:b], n // 2, 1, outs[1][a:b], None, _params(p))
    assert torch.equal(*outs)
    want = ob.attention_cache(q[-9:].cpu().numpy(), cache, table[-9:].cpu().numpy(), lengths[-9:].cpu().numpy(), 1, p)
    assert np.array_equal(outs[0][-9:].cpu().numpy(), want)


def test_calls_go_to_the_current_stream():
    """Two streams at once, each with its own workspace: every call waits for what its stream wrote before."""
    import torch
    rng = np.random.default_rng(9)
    p = _attention(rng, 128, _spread(128), 1, 1, keys=6000, cache=True)
    cache = _cache(rng, 100, 1, 64, 128)
    d, c = _on_gpu(cache)
    table = rng.permutation(100)[None, :94].astype(np.int32)
    q = [rng.integers(-90, 90, (1, 4, 128)).astype(np.int8) for _ in range(2)]
    want = [ob.attention_cache(x, cache, table, [6000], 1, p) for x in q]
    size = ip.attention_cache_i4_workspace(c, 1, 1, 4, 94)
    streams = [torch.cuda.Stream() for _ in range(2)]
    dt, dl, dq = _cuda(table), _cuda(np.array([6000], np.int32)), [_cuda(x) for x in q]
    held = [torch.zeros_like(x) for x in dq]
    outs, works = [torch.empty_like(x) for x in dq], [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in q]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, h, x, o, w in zip(streams, held, dq, outs, works):
            with torch.cuda.stream(s):
                h.zero_()
                torch.cuda._sleep(20000)
                h.copy_(x)
                ip.attention_cache_i4(h, c, dt, dl, 1, 1, o, w, _params(p))
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert np.array_equal(o.cpu().numpy(), w)


def test_the_binding_refuses():
    """Shapes, types and strides that do not belong together never reach the library."""
    import torch
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    p = ip.attention_prepare(1e-3, 0.02, 0.02, 0, 1, 1)
    q, k, o = i8(4, 4, 64), i8(6, 2, 64), i8(4, 4, 64)
    off = i32(2)
    for bad in ((q.cpu(), k, k, off, off, o), (q.int(), k, k, off, off, o), (q.view(4, 256), k, k, off, off, o), (q, k, i8(5, 2, 64), off, off, o),
                (q, i8(6, 2, 32), i8(6, 2, 32), off, off, o), (q, k, k, off, off, i8(3, 4, 64)), (q, k, k, off.long(), off, o),
                (q, k, k, i32(1), off, o), (q.transpose(0, 1), k, k, off, off, o.transpose(0, 1)), (q, k, k, off, off, o[:1].expand(4, 4, 64)),
                (i8(4, 64, 4).transpose(1, 2), k, k, off, off, o)):
        with pytest.raises((TypeError, ValueError)):
            ip.attention_i8(*bad[:5], 1, 4, bad[5], p)
    with pytest.raises(ip.IptqError):
        ip.attention_i8(q, k, k, off, None, 1, 4, o, p)
    parts = lambda: [u8(3, 2, 16, 32), u8(3, 2, 16, 1), u8(3, 2, 32, 16), u8(3, 2, 16, 1)]  # noqa: E731
    for i, t in ((0, u8(3, 2, 16, 16)), (1, u8(3, 2, 16, 2)), (2, u8(3, 2, 16, 32)), (3, u8(2, 2, 16, 1)), (0, i8(3, 2, 16, 32)), (2, u8(3, 2, 32, 16).cpu())):
        c = parts()
        c[i] = t
        with pytest.raises((TypeError, ValueError)):
            ip.cache_i4(*c, 64)
    c = ip.cache_i4(*parts(), 64)
    with pytest.raises(ValueError):
        ip.cache_store_i4(c, k, i8(6, 1, 64), i32(6), 6)
    with pytest.raises(ValueError):
        ip.cache_store_i4(c, k, k, i32(5), 6)
    for args in ((q, c, i32(4, 1), i32(4), 5, 1, o), (q, c, i32(4), i32(4), 4, 1, o), (q, c, i32(3, 1), i32(4), 4, 1, o), (q, c, i32(4, 1), i32(3), 4, 1, o),
                 (i8(4, 4, 32), c, i32(4, 1), i32(4), 4, 1, i8(4, 4, 32))):
        with pytest.raises(ValueError):
            ip.attention_cache_i4(*args, None, p)
    n = ip.RmsnormParams(1, 0, 0, ip.Dyadic(1, 0, 0, -128, 127))
    with pytest.raises(ValueError):
        ip.rmsnorm_i32(i32(2, 7), None, torch.zeros(8, dtype=torch.int16, device="cuda"), None, i8(2, 8), None, 2, 8, n)
    with pytest.raises(TypeError):
        ip.rmsnorm_i32(i32(2, 8), None, i32(8), None, i8(2, 8), None, 2, 8, n)
    with pytest.raises(ValueError):
        ip.requant_rows(i32(2, 8), i32(1), i8(2, 8), 2, 8, 1, 1, ip.Dyadic(1, 0, 0, -128, 127))
