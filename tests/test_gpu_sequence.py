"""The sequence operators (include/rh_seq.h) against their plain implementations in 64 bits (oracle/sequence.py):
block tables and slots exactly, computed numbers within bounds worked out from the arithmetic.

Bounds.  u = 2^-24 is half an ulp of 1 in fp32, 2^-8 of bf16, 2^-4 of e4m3.
  attend  a score is a sum of dim products: off by at most (dim + 8) u sum|q k| scale; a weight exp(s - top) is then off by
          twice that (its own score and the top's, which cancels in the quotient but not in the bound), by 4 u (|s| + |top|) for the
          exponent's scaling and by a few u for the function.  Over n tokens of one sum, of at most n u more (sums are blocked: far
          less).  An output is a mean of values with these weights: off by at most twice the weights' error times max|v|; a bf16
          result by half an ulp more, with weights rounded to 16 bits of mantissa (2^-16) where they meet 16-bit values.
  norm    the mean square is a sum of cols squares: off by at most (cols + 4) u relative, its root by half; three more roundings.
  matvec  products with a 2-bit mantissa; a sum of n_in of them: (n_in + 8) u sum|x w|.
"""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import sequence as S
from paper_2407_16990_amd import RH, KVCache, RhError

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def rh():
    return _context()


def _context(**kw):
    net = wl.Net("plain", 4, 2, 2)
    return RH(frame_w=64, frame_h=64, max_frames=1, halo=2, bin_size=32, max_bins=4, net=net, weights=wl.make_weights(net, 0, "fp32"),
              precision="fp32", **kw)


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _np(t):
    return t.double().cpu().numpy() if t.dtype != E4M3 else S.e4m3_values()[t.view(torch.uint8).cpu().numpy()]


# ---------------------------------------------------------------------------------------------------- cache_plan
def _plan_inputs(rng, n, page, history, chunk, ended, room, slack=0):
    old = rng.integers(0, history + 1, n)
    new = rng.integers(0, chunk + 1, n) if chunk > 1 else np.ones(n, int)
    new[rng.random(n) < ended] = -1
    have = -(-old // page)
    width = max(1, -(-(history + chunk) // page) - slack)
    old = np.minimum(old, width * page); have = -(-old // page)
    spare = int(sum(-(-(o + x) // page) - h for o, x, h in zip(old, new, have) if x > 0) * room)
    pages = int(have.sum()) + spare + 1
    ids = rng.permutation(pages)
    table = np.full((n, width), -1)
    at = 0
    for b in range(n):
        table[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    free = np.full(pages, -1)
    free[:spare] = ids[at:at + spare]
    return new, old, table, free, spare, max(1, int(new[new > 0].sum()))


def _check_plan(rh, new, old, table, free, count, page, n_slots, in_place=False):
    want = S.plan(new, old, table, free, count, page, n_slots)
    d_old, d_table, d_free, d_count = _i32(old), _i32(table), _i32(free), _i32([count])
    kw = dict(new_lengths=d_old, new_count=d_count) if in_place else {}
    slots, off, lengths, left = rh.cache_plan(_i32(new), d_old, d_table, d_free, d_count, page, n_slots, **kw)
    for name, g, w in zip(("slots", "off", "lengths", "count", "table", "free"), (slots, off, lengths, left, d_table, d_free), want):
        assert np.array_equal(g.cpu().numpy().reshape(np.shape(w)), w), name


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,page,history,chunk,ended,room", [
    (1, 1, 0, 1, 0, 1.0), (1, 16, 15, 1, 0, 1.0), (1, 16, 16, 1, 0, 1.0), (8, 16, 300, 1, 0, 1.5), (255, 16, 500, 1, 0.2, 1.0),
    (256, 7, 60, 40, 0.1, 1.0), (257, 20, 100, 300, 0.3, 0.5), (700, 48, 900, 200, 0.1, 0.9), (2048, 64, 200, 33, 0.5, 0.0),
    (2047, 1, 30, 9, 0.4, 0.7), (3, 128, 100000, 70000, 0.0, 1.0), (40, 4096, 10, 10, 0.5, 1.0)])
def test_plan(rh, n, page, history, chunk, ended, room, in_place):
    rng = np.random.default_rng(n * 7 + page)
    new, old, table, free, count, n_slots = _plan_inputs(rng, n, page, history, chunk, ended, room)
    _check_plan(rh, new, old, table, free, count, page, n_slots, in_place)
    _check_plan(rh, new, old, table, free, count, page, max(1, n_slots // 2), in_place)       # too few slots
    _check_plan(rh, new, old, table, free, count, page, n_slots + 1000, in_place)             # room behind the last


def test_plan_rows_that_are_too_short(rh):
    rng = np.random.default_rng(5)
    new, old, table, free, count, n_slots = _plan_inputs(rng, 300, 16, 100, 90, 0.1, 1.0, slack=4)
    _check_plan(rh, new, old, table, free, count, 16, n_slots)


def test_plan_extremes(rh):
    big = 2 ** 31 - 1
    table = np.full((6, 3), -1)
    # negative and huge lengths, huge requests, a stack height that lies
    _check_plan(rh, [5, big, -1, 3, big, -(2 ** 31)], [-7, 10, big, 0, big, 5], table, np.arange(20)[::-1].copy(), 4, 16, 64)
    _check_plan(rh, [1, 2], [0, 0], table[:2], np.arange(4), 1000, 2, 8)
    _check_plan(rh, [1, 2], [0, 0], table[:2], np.arange(4), -3, 2, 8)
    _check_plan(rh, [-1, -1], [6, 6], np.arange(6).reshape(2, 3), np.full(3, 9), 0, 2, 8)      # more pages come back than the stack holds


def test_plan_over_many_steps_hands_every_page_out_once(rh):
    """Streams that come, grow and go: at every step the live streams' pages and the free ones are a partition of the pool."""
    rng = np.random.default_rng(0)
    n, page, pages, width = 37, 8, 220, 12
    lengths, table, free, count = _i32(np.zeros(n)), _i32(np.full((n, width), -1)), _i32(rng.permutation(pages)), _i32([pages])
    for _ in range(40):
        new = rng.integers(0, 9, n)
        new[rng.random(n) < 0.1] = -1
        rh.cache_plan(_i32(new), lengths, table, free, count, page, 400, new_lengths=lengths, new_count=count)
        held = [p for row, ln in zip(table.cpu().numpy(), lengths.cpu().numpy()) for p in row[:-(-int(ln) // page)]]
        left = free.cpu().numpy()[:int(count)]
        assert sorted(held + left.tolist()) == list(range(pages))


# ---------------------------------------------------------------------------------------------------- cache_write
def _empty_cache(pages, page, heads, dim, dtype, order, gap=0):
    shape = (pages, page, heads, dim + gap) if order == "token" else (pages, heads, page, dim + gap)
    def one():
        t = torch.full(shape, 85, dtype=torch.uint8, device="cuda").view(E4M3) if dtype == E4M3 else torch.full(shape, 7.0, dtype=dtype, device="cuda")
        t = t[..., :dim]
        return t if order == "token" else t.transpose(1, 2)
    sc = (lambda: torch.full((pages, heads, page), 3.0, device="cuda")) if dtype == E4M3 else (lambda: None)
    return KVCache(one(), one(), sc(), sc())


@pytest.mark.parametrize("src,dst", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, E4M3),
                                     (torch.bfloat16, torch.bfloat16), (torch.bfloat16, E4M3)])
@pytest.mark.parametrize("n,heads,dim,page,order,offset", [(1, 1, 32, 1, "token", 0), (65, 3, 96, 16, "head", 0), (33, 8, 128, 20, "token", 1),
                                                           (200, 5, 160, 48, "head", 3), (17, 2, 256, 64, "token", 0), (0, 2, 64, 16, "token", 0)])
def test_write(rh, src, dst, n, heads, dim, page, order, offset):
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    pages = (n + n // 2) // page + 2
    # rows out of a wider projection, at any element: the kernel's loads need no alignment
    row = torch.randn((n, 2 * heads * dim + 5 + offset), generator=g, device="cuda").to(src)
    k, v = row[:, offset:offset + heads * dim].reshape(n, heads, dim) if n == 0 else row[:, offset:offset + heads * dim].unflatten(1, (heads, dim)), \
        row[:, offset + heads * dim:offset + 2 * heads * dim].unflatten(1, (heads, dim)) if n else row[:, :heads * dim].reshape(n, heads, dim)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n].to(torch.int32)
    if n > 4:
        k[0, 0, 3], v[1, 0, :] = float("nan"), 0.0                # a NaN stays one; a head of zeros
        slots[3], slots[4] = -1, pages * page                     # skipped
    cache = _empty_cache(pages, page, heads, dim, dst, order, gap=16)
    rh.cache_write(cache, k, v, slots)
    at = slots.cpu().numpy()
    for x, c, sc in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        x, got = _np(x), _np(c)
        blank = float(S.e4m3_values()[85]) if dst == E4M3 else 7.0
        want, tol = np.full(got.shape, blank), np.zeros(got.shape)
        for i in range(n):
            if not 0 <= at[i] < pages * page:
                continue
            p, line = divmod(int(at[i]), page)
            if dst != E4M3:
                want[p, line] = x[i]
                tol[p, line] = np.abs(x[i]) * (0 if src == dst else HALF[dst])
                continue
            most = np.maximum(np.abs(x[i]).max(-1), S.AMAX_MIN)
            g_sc = sc[p, :, line].double().cpu().numpy()
            bad = np.isnan(most)
            assert np.array_equal(np.isnan(g_sc), bad) and np.isnan(got[p, line][bad]).all()
            assert (np.abs(g_sc - most / 448)[~bad] <= 2 * U * most[~bad] / 448).all()
            want[p, line] = np.where(bad[:, None], np.nan, x[i] / (most / 448)[:, None])
            # half an ulp of e4m3 (3 bits below the leading one, 2^-10 below the smallest normal), of a quotient off by 3 ulp
            tol[p, line] = np.maximum(np.abs(want[p, line]) * 2.0 ** -4, 2.0 ** -10) * (1 + 1e-5) + 448 * 4 * U
        assert np.array_equal(np.isnan(want), np.isnan(got))
        assert (np.abs(got - want) <= tol)[~np.isnan(want)].all()
        if sc is not None and n == 0:
            assert bool((sc == 3.0).all())


# ---------------------------------------------------------------------------------------------------- cache_attend
def _attend_inputs(seed, lengths, heads, group, dim, page, q_dtype, c_dtype, order="token", spread=1.0, spare=1, q_gap=0, poison=True):
    """Pages in random order; everything in the cache that is no stream's token is NaN (or infinite)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    have = [-(-int(n) // page) for n in lengths]
    pages, width = sum(have) + spare, max(1, max(have))
    ids = rng.permutation(pages)
    table = np.full((len(lengths), width), -1)
    used = np.zeros((pages, page), bool)
    at = 0
    for b, n in enumerate(have):
        table[b, :n] = ids[at:at + n]
        for j in range(n):
            used[ids[at + j], : min(page, int(lengths[b]) - j * page)] = True
        at += n
    shape = (pages, page, heads, dim) if order == "token" else (pages, heads, page, dim)
    used = torch.from_numpy(used).cuda()
    def one(bad):
        x = torch.randn(shape, generator=g, device="cuda")
        x = x if order == "token" else x.transpose(1, 2)
        x = (x * 100).clamp(-448, 448).to(E4M3) if c_dtype == E4M3 else x.to(c_dtype)
        if poison and c_dtype == E4M3:
            x.view(torch.uint8)[~used] = 0x7F
        elif poison:
            x[~used] = bad
        sc = None
        if c_dtype == E4M3:
            sc = torch.rand((pages, heads, page), generator=g, device="cuda") * 0.01 + 0.005
            if poison:
                sc[~used[:, None, :].expand(-1, heads, -1)] = float("nan")
        return x, sc
    (k, ks), (v, vs) = one(float("nan")), one(float("inf"))
    cols = heads * group * dim
    q = (torch.randn((len(lengths), cols + q_gap), generator=g, device="cuda") * spread).to(q_dtype)[:, q_gap:].unflatten(1, (heads * group, dim))
    return q, KVCache(k, v, ks, vs), _i32(table), _i32(lengths)


def _values(x, sc):
    v = _np(x)
    return v if sc is None else v * sc.double().cpu().numpy().transpose(0, 2, 1)[..., None]


def _check_attend(rh, q, cache, table, lengths, scale, window=0, got=None):
    out, lse = rh.cache_attend(q, cache, table, lengths, scale=scale, window=window, want_lse=True) if got is None else got
    page = cache.page
    k, v = _values(cache.k, cache.k_scale), _values(cache.v, cache.v_scale)
    qn, t = _np(q), table.cpu().numpy()
    w_out, w_lse = S.attend(qn, k, v, t, lengths.cpu().numpy(), page, scale, window)
    out, lse = _np(out), _np(lse)
    group, dim = q.shape[1] // k.shape[2], q.shape[2]
    worst = 0.0
    for b in range(q.shape[0]):
        n = min(max(0, int(lengths[b])), table.shape[1] * page)
        pos = np.arange(max(0, n - window) if window else 0, n)
        p = t[b][pos // page] if n else np.zeros(0, int)
        ok = (p >= 0) & (p < k.shape[0])
        p, line = p[ok], (pos % page)[ok]
        if len(p) == 0:
            assert (out[b] == 0).all() and np.isneginf(lse[b]).all()
            continue
        for h in range(q.shape[1]):
            kk, vv = k[p, line, h // group], v[p, line, h // group]
            most = (np.abs(kk) @ np.abs(qn[b, h])).max() * scale
            e = 2 * (dim + 8) * U * most + 8 * U * most + (16 + len(p) / 16) * U
            half = HALF[q.dtype]
            tol = (2 * e + (2.0 ** -16 if q.dtype == torch.bfloat16 else 0)) * np.abs(vv).max() + half * np.abs(w_out[b, h])
            err = np.abs(out[b, h] - w_out[b, h])
            assert (err <= tol).all(), (b, h, len(p), float((err / tol).max()))
            assert abs(lse[b, h] - w_lse[b, h]) <= e + 2 * U * abs(w_lse[b, h]), (b, h)
            worst = max(worst, float((err / tol).max()))
    return worst


KINDS = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, E4M3)]


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
def test_attend_head_sizes(rh, q_dtype, c_dtype, dim):
    for order, group, page in (("token", 1, 16), ("head", 5, 20)):
        q, cache, table, lengths = _attend_inputs(dim + group, [1, 33, 0, 150], 2, group, dim, page, q_dtype, c_dtype, order)
        _check_attend(rh, q, cache, table, lengths, dim ** -0.5)


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("heads,group", [(1, 1), (1, 16), (2, 17), (3, 2), (8, 4), (1, 40), (4, 8), (1, 33)])
def test_attend_head_layouts(rh, q_dtype, c_dtype, heads, group):
    q, cache, table, lengths = _attend_inputs(heads * 100 + group, [70, 5, 129], heads, group, 64, 16, q_dtype, c_dtype, "head", q_gap=3)
    _check_attend(rh, q, cache, table, lengths, 0.125)


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("page", [1, 3, 8, 16, 31, 32, 33, 64, 100, 1000])
def test_attend_lengths_around_every_boundary(rh, q_dtype, c_dtype, page):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 1025]
    q, cache, table, lengths = _attend_inputs(page, lens, 2, 3, 64, page, q_dtype, c_dtype, "token" if page % 2 else "head")
    _check_attend(rh, q, cache, table, lengths, 0.125)


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 129, 4000])
def test_attend_window(rh, q_dtype, c_dtype, window):
    q, cache, table, lengths = _attend_inputs(window, [0, 1, 32, 33, 64, 131, 700, 2500], 2, 4, 96, 20, q_dtype, c_dtype)
    _check_attend(rh, q, cache, table, lengths, 96 ** -0.5, window)
    # what lies before the window does not matter either
    page, t = 20, table.cpu().numpy()
    for b, n in enumerate(lengths.tolist()):
        for pos in range(0, max(0, n - window)):
            p, line = int(t[b, pos // page]), pos % page
            if c_dtype == E4M3:
                cache.k.view(torch.uint8)[p, line] = 0x7F
            else:
                cache.k[p, line] = float("nan")
                cache.v[p, line] = float("nan")
            if pos > 60:
                break
    out = rh.cache_attend(q, cache, table, lengths, scale=96 ** -0.5, window=window)
    assert bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("n,length,heads,group", [(1, 30000, 1, 1), (1, 20001, 2, 8), (3, 9000, 1, 20), (60, 300, 8, 2), (300, 40, 4, 1),
                                                    (64, 30, 8, 2), (64, 100, 16, 1), (100, 5000, 2, 4), (8, 12000, 2, 20), (2048, 20, 2, 1), (65, 1000, 1, 17)])
def test_attend_split_and_joined(rh, q_dtype, c_dtype, n, length, heads, group):
    """One long stream among short ones, and many: whatever the split, and the same bits on every run."""
    lens = [length] + [(7 * i * length // n) % (length // 3) for i in range(1, n)]
    q, cache, table, lengths = _attend_inputs(n + length, lens, heads, group, 128, 16, q_dtype, c_dtype, "head")
    out, lse = rh.cache_attend(q, cache, table, lengths, want_lse=True)
    _check_attend(rh, q, cache, table, lengths, 128 ** -0.5, got=(out, lse))
    for _ in range(4):
        again = rh.cache_attend(q, cache, table, lengths, want_lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
@pytest.mark.parametrize("dim,heads,group", [(96, 4, 3), (32, 3, 1), (64, 5, 18)])
def test_attend_many_chunks_of_heads_that_share_lines(rh, q_dtype, c_dtype, dim, heads, group):
    lens = [3000 + 211 * i for i in range(20)] + [0, 1, 17]
    q, cache, table, lengths = _attend_inputs(dim, lens, heads, group, dim, 16, q_dtype, c_dtype, "token")
    got = rh.cache_attend(q, cache, table, lengths, want_lse=True)
    again = rh.cache_attend(q, cache, table, lengths, want_lse=True)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    pick = [0, 7, 19, 20, 21, 22]                              # the reference takes its time: some of the streams
    _check_attend(rh, q[pick], cache, table[pick].contiguous(), lengths[pick].contiguous(), dim ** -0.5, got=(got[0][pick], got[1][pick]))


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
def test_attend_peaked_scores(rh, q_dtype, c_dtype):
    """Scores hundreds apart: tokens whose weight is nothing, tops that come late, and a scale of zero or below."""
    q, cache, table, lengths = _attend_inputs(3, [500, 77, 1, 260], 2, 4, 64, 16, q_dtype, c_dtype, spread=20.0)
    for scale in (1.0, 0.0, -0.5):
        out, lse = rh.cache_attend(q, cache, table, lengths, scale=scale, want_lse=True)
        w_out, w_lse = S.attend(_np(q), _values(cache.k, cache.k_scale), _values(cache.v, cache.v_scale), table.cpu().numpy(), lengths.cpu().numpy(), 16, scale)
        # a score's error is (dim + 16) u sum|q k| <= 80 u * 64 * 60 * 4.5 = 0.08 of a weight, where tops are close to each other
        bar = 0.2 * np.abs(_values(cache.v, cache.v_scale)[np.isfinite(_values(cache.v, cache.v_scale))]).max()
        assert np.abs(_np(out) - w_out).max() <= bar and np.isfinite(_np(out)).all()
        assert np.abs(_np(lse) - w_lse).max() <= 0.1


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
def test_attend_leaves_out_pages_that_do_not_exist(rh, q_dtype, c_dtype):
    q, cache, table, lengths = _attend_inputs(8, [100, 64, 31, 200], 2, 2, 64, 16, q_dtype, c_dtype, poison=False)
    table[0, 2], table[1, :], table[2, 0], table[3, 5], table[3, 12] = -1, 10 ** 6, -5, cache.n_pages, -(2 ** 31)
    cache.v[0].view(torch.uint8)[:] = 0x7F                         # page 0 may hold anything where nobody owns it
    cache.k[0].view(torch.uint8)[:] = 0x7F
    table[table == 0] = -1
    _check_attend(rh, q, cache, table, lengths, 0.125)


def test_attend_lengths_past_the_table(rh):
    q, cache, table, lengths = _attend_inputs(9, [96, 48], 1, 2, 64, 16, torch.bfloat16, torch.bfloat16)
    full = rh.cache_attend(q, cache, table, lengths)
    table = table[:, :6].contiguous()
    long = rh.cache_attend(q, cache, table, _i32([2 ** 31 - 1, 48]))
    assert torch.equal(full, long)
    none = rh.cache_attend(q, cache, table, _i32([-4, -(2 ** 31)]))
    assert bool((none == 0).all())


@pytest.mark.parametrize("q_dtype,c_dtype", KINDS)
def test_attend_infinities_are_what_the_formula_makes_of_them(rh, q_dtype, c_dtype):
    """A NaN among a stream's own keys or values reaches that stream's outputs and no other's."""
    q, cache, table, lengths = _attend_inputs(4, [40, 40, 40], 1, 2, 64, 16, q_dtype, c_dtype)
    p = int(table[1, 1])
    if c_dtype == E4M3:
        cache.v.view(torch.uint8)[p, 3, 0, 5] = 0x7F
    else:
        cache.v[p, 3, 0, 5] = float("nan")
    out = rh.cache_attend(q, cache, table, lengths).float()
    assert bool(torch.isnan(out[1, :, 5]).all()) and bool(torch.isfinite(out[[0, 2]]).all())
    assert bool(torch.isfinite(out[1, :, :5]).all()) and bool(torch.isfinite(out[1, :, 6:]).all())
    if c_dtype == E4M3:
        cache.k.view(torch.uint8)[p, 3, 0, 5] = 0x7F
    else:
        cache.k[p, 3, 0, 5] = float("nan")
    out, lse = rh.cache_attend(q, cache, table, lengths, want_lse=True)
    assert bool(torch.isnan(out[1].float()).all()) and bool(torch.isnan(lse[1]).all())
    assert bool(torch.isfinite(out[[0, 2]].float()).all()) and bool(torch.isfinite(lse[[0, 2]]).all())


@pytest.mark.parametrize("c_dtype", [torch.bfloat16, E4M3, torch.float32])
def test_attend_offsets_past_32_bits(rh, c_dtype):
    """A cache of more than 2^32 elements, its last pages in use."""
    heads, dim, page = 8, 128, 64
    pages = 2 ** 32 // (heads * dim * page) + 9
    size = {torch.bfloat16: 2, torch.float32: 4, E4M3: 1}[c_dtype]
    k, v = (torch.empty((pages, page, heads, dim * size), dtype=torch.uint8, device="cuda") for _ in range(2))
    k, v = k.view(c_dtype), v.view(c_dtype)
    ks, vs = (torch.empty((pages, heads, page), device="cuda") for _ in range(2)) if c_dtype == E4M3 else (None, None)
    cache = KVCache(k, v, ks, vs)
    q_dtype = torch.float32 if c_dtype == torch.float32 else torch.bfloat16
    table = _i32([[pages - 1, 0, pages - 3], [pages - 2, 5, pages - 5]])
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((300, 2, heads, dim), generator=g, device="cuda").to(q_dtype)
    slots = (table[:, torch.arange(150, device="cuda") // page] * page + torch.arange(150, device="cuda") % page).reshape(-1).to(torch.int32)
    rh.cache_write(cache, x[:, 0], x[:, 1], slots)
    q = torch.randn((2, heads * 2, dim), generator=g, device="cuda").to(q_dtype)
    out, lse = rh.cache_attend(q, cache, table, _i32([150, 150]), want_lse=True)
    small = KVCache(*[t[table.reshape(-1).long()].contiguous() if t.dtype != E4M3 else t.view(torch.uint8)[table.reshape(-1).long()].view(E4M3)
                      for t in (k, v)], *[None if t is None else t[table.reshape(-1).long()].contiguous() for t in (ks, vs)])
    o2, l2 = rh.cache_attend(q, small, _i32([[0, 1, 2], [3, 4, 5]]), _i32([150, 150]), want_lse=True)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    _check_attend(rh, q, small, _i32([[0, 1, 2], [3, 4, 5]]), _i32([150, 150]), dim ** -0.5)


# ---------------------------------------------------------------------------------------------------- norm_residual
def _check_norm(rh, x, w, r, eps, outputs, sum_out=None):
    want_s, want_y, want_sc = S.norm(_np(x), _np(w), None if r is None else _np(r), eps)
    total, y, y8, sc = rh.norm_residual(x, w, r, eps=eps, outputs=outputs, sum_out=sum_out)
    half = HALF[x.dtype]
    rel = (x.shape[1] / 2 + 8) * U
    if r is not None:
        assert (np.abs(_np(total) - want_s) <= half * np.abs(want_s) * (1 + 1e-6) + U * np.abs(want_s)).all()
    # a sum s of two rounded inputs is itself rounded once before it is squared and scaled
    bar = (rel + 2 * U) * np.abs(want_y)
    if outputs != "e4m3":
        assert (np.abs(_np(y) - want_y) <= bar + half * np.abs(want_y) * (1 + 1e-6)).all()
    if outputs != "same":
        assert (np.abs(_np(sc) - want_sc) <= (rel + 6 * U) * want_sc).all()
        q = want_y / want_sc[:, None]
        tol = np.maximum(np.abs(q) * 2.0 ** -4, 2.0 ** -10) * (1 + 1e-3) + 448 * (2 * rel + 8 * U)
        assert (np.abs(_np(y8) - q) <= tol).all()
        assert np.abs(_np(y8)).max() <= 448
        if np.abs(want_y).max() > 1e-20:
            assert (np.abs(_np(y8)).max(-1) == 448).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 3), (3, 4), (4, 8), (9, 63), (2, 255), (7, 256), (6, 510), (5, 513), (8, 1024), (3, 1025), (3, 2048), (2, 2049),
                                       (3, 4095), (2, 4096), (2, 4097), (2, 8193), (2, 16384), (1, 16389), (1, 32767), (1, 32768), (1000, 64), (333, 2000)])
def test_norm(rh, dtype, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows * 40000 + cols)
    x, r = (torch.randn((rows, cols), generator=g, device="cuda").to(dtype) for _ in range(2))
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    for outputs in ("same", "e4m3", "both"):
        _check_norm(rh, x, w, r, 1e-6, outputs)
    _check_norm(rh, x, w, None, 1e-5, "both")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_strided_rows_and_in_place(rh, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn((6, 1300), generator=g, device="cuda").to(dtype)
    other = torch.randn((6, 900), generator=g, device="cuda").to(dtype)
    w = torch.rand(500, generator=g, device="cuda") + 0.5
    x, r = wide[:, 3:503], other[:, 1:501]
    keep = other.clone()
    fresh = rh.norm_residual(x, w, r, outputs="both")
    _check_norm(rh, x, w, r.clone(), 1e-6, "both", sum_out=torch.empty((6, 640), dtype=dtype, device="cuda")[:, :500])
    placed = rh.norm_residual(x, w, r, outputs="both", sum_out=r)              # the residual stream, in place
    assert placed[0].data_ptr() == r.data_ptr()
    for a, b in zip(fresh, placed):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    assert torch.equal(other[:, 501:], keep[:, 501:]) and torch.equal(other[:, :1], keep[:, :1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_every_rest_of_a_row(rh, dtype):
    """Rows that end anywhere in a piece, at the wave's and the workgroup's ends too; what lies beside a row (NaN) is neither read into it nor
    written; the residual stream in place."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for base in (0, 504, 512, 1016, 2040, 4088, 8184, 16376):
        for cols in range(base + 1, base + 18):
            wide = torch.full((5, cols + 13), float("nan"), device="cuda").to(dtype)
            x = wide[:, 5:5 + cols]
            x.copy_(torch.randn((5, cols), generator=g, device="cuda"))
            w = torch.randn(cols, generator=g, device="cuda")
            r_wide = wide.clone()
            r = r_wide[:, 5:5 + cols]
            _check_norm(rh, x, w, r.clone(), 1e-6, "both")
            want = rh.norm_residual(x, w, r.clone(), outputs="both")
            got = rh.norm_residual(x, w, r, outputs="both", sum_out=r)
            assert all(torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else a, b.view(torch.uint8) if b.dtype == E4M3 else b) for a, b in zip(got, want))
            assert bool(r_wide[:, :5].isnan().all()) and bool(r_wide[:, 5 + cols:].isnan().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_short_rows_side_by_side(rh, dtype):
    """Rows that share a wave keep to themselves: a NaN, an infinity or zeros in one change no other."""
    g = torch.Generator(device="cuda").manual_seed(11)
    for rows in (1, 3, 37, 300):
        for cols in (1, 7, 30, 32, 33, 63, 64, 65, 100, 128, 129, 200, 256, 257):
            x = torch.randn((rows, cols), generator=g, device="cuda").to(dtype)
            w = torch.rand(cols, generator=g, device="cuda") + 0.5
            _check_norm(rh, x, w, None, 1e-6, "both")
            want = rh.norm_residual(x, w, outputs="both")
            bad = x.clone()
            bad[1::4, cols // 2] = float("nan")
            bad[2::8, -1] = float("inf")
            bad[3::8] = 0
            got = rh.norm_residual(bad, w, outputs="both")
            same = torch.ones(rows, dtype=torch.bool, device="cuda")
            same[1::4] = False; same[2::8] = False; same[3::8] = False
            for a, b in zip(got[1:], want[1:]):                     # without a residual there is no sum
                a, b = a[same], b[same]
                assert torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else a, b.view(torch.uint8) if b.dtype == E4M3 else b)
            assert bool(got[1][1::4].isnan().all()) and bool((got[1][3::8] == 0).all())


def test_norm_extreme_rows(rh):
    x = torch.zeros((6, 300), device="cuda")
    x[1], x[2, 5], x[3, 7], x[4], x[5] = 1e-30, float("inf"), float("nan"), 1e30, 1e-3
    w = torch.ones(300, device="cuda")
    _, y, y8, sc = rh.norm_residual(x, w, None, eps=0.0 + 1e-12, outputs="both")
    assert bool((y[0] == 0).all()) and bool((y8[0].float() == 0).all()) and float(sc[0]) > 0
    assert bool(torch.isfinite(y[1]).all()) and bool(torch.isnan(y8[3].float()).all()) and bool(torch.isnan(sc[3]))
    assert bool(torch.isnan(y[2, 5])) and bool((y[2, :5] == 0).all()) and bool(torch.isnan(sc[2]))    # infinity / infinity, finite / infinity
    assert bool((y[4] == 0).all())                                              # the squares pass fp32, as the formula in 32 bits has it
    assert np.allclose(_np(y[5]), 1e-3 / np.sqrt(1e-6 + 1e-12), rtol=1e-6)


# ---------------------------------------------------------------------------------------------------- matvec_packed
def _weights(g, n_out, n_in, wide=False):
    blocks = (n_in + 31) // 32
    w = torch.randint(0, 256, (n_out, 16 * blocks), generator=g, device="cuda").to(torch.uint8)
    sc = torch.randint(60 if wide else 118, 190 if wide else 128, (n_out, blocks), generator=g, device="cuda").to(torch.uint8)
    return w, sc


def _rows(g, rows, n_in, dtype, gap=0):
    x = torch.randn((rows, n_in + gap), generator=g, device="cuda")
    x = (x * 100).clamp(-448, 448).to(E4M3) if dtype == E4M3 else x.to(dtype)
    return x[:, gap:]


def _check_matvec(rh, x, w, sc, xs, relu, out_dtype):
    y = rh.matvec_packed(x, w, sc, x_scale=xs, relu=relu, out_dtype=out_dtype)
    xn = _np(x)
    real = S.unpack_weights(w.cpu().numpy(), sc.cpu().numpy(), x.shape[1])
    xsn = None if xs is None else _np(xs)
    want = S.matvec(xn, w.cpu().numpy(), sc.cpu().numpy(), xsn, relu)
    most = np.abs(xn) @ np.abs(real).T * (1 if xs is None else xsn[:, None])
    tol = (x.shape[1] + 8) * U * most + HALF[out_dtype] * np.abs(want) * (1 + 1e-5)
    err = np.abs(_np(y) - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())
    return y


TYPES = [torch.float32, torch.bfloat16, E4M3]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_out,n_in", [(1, 1, 1), (1, 16, 32), (1, 17, 31), (2, 5, 33), (3, 100, 127), (1, 64, 129), (5, 33, 510), (16, 1024, 512), (17, 130, 920),
                                             (1, 4096, 1024), (33, 200, 300), (64, 96, 2048), (65, 70, 700), (130, 40, 64), (4, 2, 8192), (1, 500, 16384), (8, 48, 20000), (15, 1, 511),
                                             (64, 9000, 2100), (16, 5000, 2048), (24, 8300, 3500)])
def test_matvec(rh, dtype, rows, n_out, n_in):
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + n_out * 3 + n_in)
    w, sc = _weights(g, n_out, n_in)
    x = _rows(g, rows, n_in, dtype, gap=(n_out % 3) * 5)
    xs = torch.rand(rows, generator=g, device="cuda") * 0.1 if dtype == E4M3 or n_out % 2 else None
    for relu, out in ((False, torch.float32), (True, torch.bfloat16)):
        _check_matvec(rh, x, w, sc, xs, relu, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_out,n_in", [(1, 200, 16000), (16, 7, 4096), (16, 300, 16384), (13, 260, 15361), (31, 500, 7777), (40, 1000, 8000), (64, 129, 12288), (64, 2100, 5000), (200, 33, 9000),
                                             (1, 16, 40000), (64, 3000, 16384)])
def test_matvec_long_rows(rh, dtype, rows, n_out, n_in):
    """Long rows, whose inner index several workgroups share: what they add up, and that it is the same every time, also between calls of
    other shapes that use the same scratch memory."""
    g = torch.Generator(device="cuda").manual_seed(rows + n_out + n_in)
    w, sc = _weights(g, n_out, n_in)
    x = _rows(g, rows, n_in, dtype, gap=rows % 2 * 3)
    xs = torch.rand(rows, generator=g, device="cuda") * 0.1 if n_out % 2 else None
    w2, sc2 = _weights(g, 400, 16384)
    x2 = _rows(g, 16, 16384, torch.float32)
    other = rh.matvec_packed(x2, w2, sc2)
    for relu, out in ((False, torch.float32), (True, torch.bfloat16)):
        y = _check_matvec(rh, x, w, sc, xs, relu, out)
        for _ in range(3):
            assert torch.equal(rh.matvec_packed(x2, w2, sc2), other)
            assert torch.equal(rh.matvec_packed(x, w, sc, x_scale=xs, relu=relu, out_dtype=out), y)


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_every_rest_of_a_row(rh, dtype):
    """Rows that end anywhere in a piece, block or stretch of 512; what lies beside a row (NaN) does not matter."""
    g = torch.Generator(device="cuda").manual_seed(9)
    for base in (0, 500, 1010, 4080):
        for n_in in range(base + 1, base + 37):
            w, sc = _weights(g, 20, n_in)
            x = torch.full((19, n_in + 9), float("nan"), device="cuda").to(dtype)[:, 4:4 + n_in]
            x.copy_(_rows(g, 19, n_in, dtype))
            for out in (torch.float32, torch.bfloat16):
                _check_matvec(rh, x, w, sc, None, False, out)


def test_matvec_long_rows_hold_what_is_not_finite(rh):
    """An infinity or NaN of a row stays in that row's outputs, wherever along the row it lies."""
    g = torch.Generator(device="cuda").manual_seed(8)
    w, sc = _weights(g, 70, 16384)
    w |= 0x11                                                      # no weight is zero
    for dtype in TYPES:
        x = _rows(g, 16, 16384, dtype).clone()
        want = rh.matvec_packed(x, w, sc, out_dtype=torch.float32)
        for at in (0, 511, 8000, 16383):
            bad = x.clone()
            bad[5, at] = float("nan")
            y = rh.matvec_packed(bad, w, sc, out_dtype=torch.float32)
            assert bool(y[5].isnan().all()), at
            y[5] = want[5]
            assert torch.equal(y, want)


def test_matvec_long_rows_in_a_graph(rh):
    g = torch.Generator(device="cuda").manual_seed(12)
    w, sc = _weights(g, 300, 16384)
    x = torch.zeros((16, 16384), device="cuda")
    rh.matvec_packed(x, w, sc)                                     # the scratch memory is there
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    rh.lib.rh_set_stream(rh.h, side.cuda_stream)
    rh._stream = side
    try:
        with torch.cuda.graph(graph, stream=side):
            got = rh.matvec_packed(x, w, sc)
    finally:
        rh._stream = torch.cuda.current_stream()
        rh.lib.rh_set_stream(rh.h, rh._stream.cuda_stream)
    for i in range(5):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = rh.matvec_packed(x, w, sc)
        torch.cuda.synchronize()
        assert torch.equal(got, want), i


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_every_code_and_scale(rh, dtype):
    """One weight a row of outputs: every code at every scale byte (255 is not a number), an input of one."""
    w = torch.zeros((4096, 16), dtype=torch.uint8, device="cuda")
    w[:, 0] = torch.arange(4096, device="cuda") % 16
    sc = (torch.arange(4096, device="cuda") // 16).to(torch.uint8)[:, None].contiguous()
    x = torch.zeros((1, 32), device="cuda")
    x[0, 0] = 1
    y = rh.matvec_packed(x.to(dtype), w, sc, out_dtype=torch.float32)[0].double().cpu().numpy()
    want = S.unpack_weights(w.cpu().numpy(), sc.cpu().numpy(), 1)[:, 0]
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32).astype(np.float64)        # 6 * 2^127 and the like pass fp32
    assert np.isnan(y[4080:]).all()
    # numbers below the normal ones of fp32 may come out as zeros
    ok = (y == want32) | ((np.abs(want32) < 2.0 ** -126) & (np.abs(y) < 2.0 ** -126))
    assert ok[:4080].all(), np.nonzero(~ok[:4080])


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_scales_far_apart(rh, dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    w, sc = _weights(g, 60, 400, wide=True)
    _check_matvec(rh, _rows(g, 3, 400, dtype), w, sc, None, False, torch.float32)


def test_matvec_codes_past_the_row_do_not_matter(rh):
    g = torch.Generator(device="cuda").manual_seed(4)
    w, sc = _weights(g, 50, 70)
    x = torch.randn((2, 200), generator=g, device="cuda")
    x[:, 70:] = float("nan")                                       # nor does what follows a row of x
    a = rh.matvec_packed(x[:, :70], w, sc)
    w2 = w.clone()
    w2[:, 35:] = 255 - w2[:, 35:]
    assert torch.equal(a, rh.matvec_packed(x[:, :70], w2, sc)) and bool(torch.isfinite(a).all())


def test_matvec_infinities(rh):
    g = torch.Generator(device="cuda").manual_seed(6)
    w, sc = _weights(g, 40, 64)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn((3, 64), generator=g, device="cuda").to(dtype)
        x[1, 9] = float("nan")
        y = rh.matvec_packed(x, w, sc, out_dtype=torch.float32)
        assert bool(torch.isnan(y[1]).all()) and bool(torch.isfinite(y[[0, 2]]).all())


def test_matvec_strided_output(rh):
    g = torch.Generator(device="cuda").manual_seed(5)
    w, sc = _weights(g, 37, 96)
    x = torch.randn((4, 96), generator=g, device="cuda").to(torch.bfloat16)
    out = torch.full((4, 60), 9.0, dtype=torch.bfloat16, device="cuda")
    rh.matvec_packed(x, w, sc, out=out[:, 2:39])
    assert torch.equal(out[:, 2:39], rh.matvec_packed(x, w, sc)) and bool((out[:, :2] == 9).all()) and bool((out[:, 39:] == 9).all())


# ---------------------------------------------------------------------------------------------------- streams, graphs, refusals
def test_on_another_stream():
    """A context on a stream that is not torch's current one: inputs are ready, outputs are held back from reuse."""
    side = torch.cuda.Stream()
    rh2 = _context(stream=side)
    q, cache, table, lengths = _attend_inputs(1, [300, 5, 90], 2, 4, 64, 16, torch.bfloat16, torch.bfloat16)
    torch.cuda.synchronize()
    out = rh2.cache_attend(q, cache, table, lengths)
    side.synchronize()
    rh1 = _context()
    assert torch.equal(out, rh1.cache_attend(q, cache, table, lengths))


def test_a_captured_step_replays_what_the_calls_give(rh):
    """plan, write, norm, matvec and attend in one graph, replayed with other contents in between."""
    n, heads, group, dim, page, width, pages = 9, 2, 4, 64, 16, 8, 80
    g = torch.Generator(device="cuda").manual_seed(0)
    cols = heads * (group + 2) * dim
    w, sc = _weights(g, cols, 256)
    weight = torch.ones(256, device="cuda")

    def state():
        c = KVCache(*[torch.zeros((pages, page, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)])
        return dict(c=c, lengths=_i32(np.zeros(n)), table=_i32(np.full((n, width), -1)), free=_i32(np.arange(pages)), count=_i32([pages]),
                    new=_i32(np.ones(n)), x=torch.zeros((n, 256), dtype=torch.bfloat16, device="cuda"))

    def step(s):
        _, _, y8, ys = rh.norm_residual(s["x"], weight, outputs="e4m3")
        row = rh.matvec_packed(y8, w, sc, x_scale=ys)
        slots, _, _, _ = rh.cache_plan(s["new"], s["lengths"], s["table"], s["free"], s["count"], page, n, new_lengths=s["lengths"], new_count=s["count"])
        h = heads * group * dim
        rh.cache_write(s["c"], row[:, h:h + heads * dim].unflatten(1, (heads, dim)), row[:, h + heads * dim:].unflatten(1, (heads, dim)), slots)
        return rh.cache_attend(row[:, :h].unflatten(1, (heads * group, dim)), s["c"], s["table"], s["lengths"])

    eager, cap = state(), state()
    step(state())                                                   # the scratch memory is there
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    rh.lib.rh_set_stream(rh.h, side.cuda_stream)
    rh._stream = side
    try:
        with torch.cuda.graph(graph, stream=side):
            got = step(cap)
    finally:
        rh._stream = torch.cuda.current_stream()
        rh.lib.rh_set_stream(rh.h, rh._stream.cuda_stream)
    for i in range(6):
        x = torch.randn((n, 256), generator=g, device="cuda").to(torch.bfloat16)
        new = _i32([-1 if (i + b) % 5 == 4 else 1 for b in range(n)])
        for s in (eager, cap):
            s["x"].copy_(x); s["new"].copy_(new)
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
        assert all(torch.equal(eager[k], cap[k]) for k in ("lengths", "table", "free", "count"))


def _refused(status, call, *a, **kw):
    with pytest.raises(RhError) as ei:
        call(*a, **kw)
    assert ei.value.status == status and len(str(ei.value)) > 20
    return str(ei.value)


def test_refusals(rh):
    INVALID, SHAPE, CAPACITY, UNIMPLEMENTED = 1, 2, 3, 7
    q, cache, table, lengths = _attend_inputs(1, [30, 5], 2, 4, 64, 16, torch.bfloat16, torch.bfloat16)
    z = torch.zeros
    dev = dict(device="cuda")
    # plan
    args = lambda n: (_i32(np.ones(n)), _i32(np.zeros(n)), _i32(np.zeros((n, 2))), _i32(np.zeros(4)), _i32([4]))  # noqa: E731
    _refused(CAPACITY, rh.cache_plan, *args(2049), 16, 8)
    _refused(SHAPE, rh.cache_plan, *args(2), 0, 8)
    _refused(SHAPE, rh.cache_plan, *args(2), 16, 0)
    _refused(SHAPE, rh.cache_plan, *args(2), 2 ** 30, 8)
    # caches
    def cache_of(dim=64, dtype=torch.bfloat16, gap=0, off=0, scales=False):
        t = z(4 * 16 * 2 * (dim + gap) + off, dtype=dtype, **dev)[off:].view(4, 16, 2, dim + gap)[..., :dim]
        return KVCache(t, t, *([z((4, 2, 16), **dev)] * 2 if scales else []))
    x = z((3, 2, 64), dtype=torch.bfloat16, **dev)
    slots = _i32([0, 1, 2])
    _refused(SHAPE, rh.cache_write, cache_of(48), x[..., :48], x[..., :48], slots)
    _refused(SHAPE, rh.cache_write, cache_of(288), z((3, 2, 288), **dev), z((3, 2, 288), **dev), slots)
    _refused(SHAPE, rh.cache_write, cache_of(gap=4), x, x, slots)
    _refused(INVALID, rh.cache_write, cache_of(off=4), x, x, slots)
    _refused(INVALID, rh.cache_write, cache_of(scales=True), x, x, slots)
    _refused(INVALID, rh.cache_write, cache_of(dtype=E4M3), x, x, slots)
    _refused(UNIMPLEMENTED, rh.cache_write, cache_of(dtype=torch.float32), x, x, slots)
    _refused(INVALID, rh.cache_write, cache_of(), x.to(E4M3), x.to(E4M3), slots)
    # attend
    _refused(SHAPE, rh.cache_attend, q[:, :7], cache, table, lengths)
    _refused(UNIMPLEMENTED, rh.cache_attend, q.float(), cache, table, lengths)
    _refused(UNIMPLEMENTED, rh.cache_attend, q, cache_of(dtype=torch.float32), table, lengths)
    _refused(INVALID, rh.cache_attend, q, cache, table, lengths, window=-1)
    _refused(CAPACITY, rh.cache_attend, q[:1].expand(2049, 8, 64), cache, table[:1].expand(2049, -1).contiguous(), _i32(np.ones(2049)))
    _refused(INVALID, rh.cache_attend, q, cache, table, lengths, out=z(2 * 8 * 64 + 1, dtype=torch.bfloat16, **dev)[1:].view(2, 8, 64))
    # norm
    w = torch.ones(64, **dev)
    big = z((1, 32769), **dev)
    _refused(SHAPE, rh.norm_residual, big, z(32769, **dev))
    _refused(INVALID, rh.norm_residual, z((2, 64), **dev), w, eps=-1.0)
    _refused(INVALID, rh.norm_residual, z((2, 64), **dev), w, eps=float("nan"))
    _refused(INVALID, rh.norm_residual, z((2, 64), **dev).to(E4M3), w)
    _refused(SHAPE, rh.norm_residual, z((1, 64), **dev).expand(2, 64), w)
    # matvec
    cw, cs = z((8, 32), dtype=torch.uint8, **dev), z((8, 2), dtype=torch.uint8, **dev)
    _refused(INVALID, rh.matvec_packed, z((2, 64), **dev), cw, cs, out_dtype=E4M3)
    _refused(SHAPE, rh.matvec_packed, z((1, 64), **dev).expand(2, 64), cw, cs)
    _refused(INVALID, rh.matvec_packed, z((2, 64), **dev), z(8 * 32 + 1, dtype=torch.uint8, **dev)[1:].view(8, 32), cs)
    # nothing was launched and the context goes on
    _check_attend(rh, q, cache, table, lengths, 0.125)


def test_empty_batches(rh):
    z = torch.zeros
    assert rh.norm_residual(z((0, 64), device="cuda"), z(64, device="cuda"))[1].shape == (0, 64)
    assert rh.matvec_packed(z((0, 64), device="cuda"), z((8, 32), dtype=torch.uint8, device="cuda"), z((8, 2), dtype=torch.uint8, device="cuda")).shape == (0, 8)


def test_tensors_that_do_not_fit_are_refused_in_the_binding(rh):
    q, cache, table, lengths = _attend_inputs(1, [30, 5], 2, 4, 64, 16, torch.bfloat16, torch.bfloat16)
    x, w32 = torch.zeros((2, 64), device="cuda"), torch.ones(64, device="cuda")
    cw, cs = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), dtype=torch.uint8, device="cuda")
    i = _i32(np.zeros(2))
    calls = [
        lambda: rh.cache_attend(q[:1], cache, table, lengths), lambda: rh.cache_attend(q[..., :32], cache, table, lengths),
        lambda: rh.cache_attend(q, cache, table.long(), lengths), lambda: rh.cache_attend(q, cache, table, lengths[:1]),
        lambda: rh.cache_attend(q, cache, table, lengths, out=torch.zeros((2, 8, 64), device="cuda")),
        lambda: rh.cache_attend(q.cpu(), cache, table, lengths),
        lambda: KVCache(cache.k, cache.v.float()), lambda: KVCache(cache.k, cache.v[:, :, :1]), lambda: KVCache(cache.k.transpose(2, 3), cache.v.transpose(2, 3)),
        lambda: KVCache(cache.k, cache.v, i.float(), i.float()),
        lambda: rh.cache_write(cache, q[:, :2], q[:, :3], i), lambda: rh.cache_write(cache, q[:, :2], q[:, 2:4], i.long()), lambda: rh.cache_write(cache, q[:1, :2], q[:1, 2:4], i),
        lambda: rh.cache_plan(i, i[:1], table, i, i[:1], 16, 4), lambda: rh.cache_plan(i, i, table[:1], i, i[:1], 16, 4), lambda: rh.cache_plan(i, i, table, i, i, 16, 4),
        lambda: rh.cache_plan(i, i, table, i, i[:1], 16, 4, new_lengths=i[:1]), lambda: rh.cache_plan(i.float(), i, table, i, i[:1], 16, 4),
        lambda: rh.norm_residual(x, w32[:5]), lambda: rh.norm_residual(x, w32, x.bfloat16()), lambda: rh.norm_residual(x, w32, x[:1]), lambda: rh.norm_residual(x, w32, outputs="bf16"),
        lambda: rh.norm_residual(x, w32.double()), lambda: rh.norm_residual(x.t(), w32[:2]), lambda: rh.norm_residual(x, w32, x, sum_out=x.bfloat16()),
        lambda: rh.matvec_packed(x[:, :32], cw, cs), lambda: rh.matvec_packed(x, cw[:4], cs), lambda: rh.matvec_packed(x, cw, cs, x_scale=w32), lambda: rh.matvec_packed(x, cw.int(), cs),
        lambda: rh.matvec_packed(x.double(), cw, cs), lambda: rh.matvec_packed(x, cw, cs, out=x), lambda: rh.matvec_packed(x, cw, cs, out=torch.zeros((2, 8), device="cuda"), out_dtype=torch.bfloat16),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(AssertionError):
            call()
            print("call", k, "was taken")
    with pytest.raises(TypeError):
        rh.cache_attend(q, cache, table, lengths, scale="1")
