"""The key-value cache in K-means codes on the GPU: codes equal to the stated
fp32 definition bit for bit, values read back exactly, attention within bounds
that are derived from its roundings."""
import math

import numpy as np
import pytest
import torch

import paper_1402_3788_amd as km

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0") if torch.cuda.is_available() else None
BF, FP = torch.bfloat16, torch.float16


def make_cache(heads, dim, sub, K, dtype, pages, page, seed=0, random_codes=True):
    g = torch.Generator().manual_seed(seed)
    S = dim // sub
    kc, vc = (torch.randn(heads, S, K, sub, generator=g).to(dtype).to(DEV) for _ in range(2))
    cache = km.KVCodes.empty(kc, vc, pages, page)
    if random_codes:
        for t in (cache.k_codes, cache.v_codes):
            t.copy_(torch.randint(0, K, t.shape, generator=g, dtype=torch.uint8))
    return cache


def nearest(x, centres):
    """The definition in include/kmeans.h, in numpy fp32: x [n, H, D], centres
    [H, S, K, sub] -> [n, H, S]."""
    x, c = x.float().cpu().numpy(), centres.float().cpu().numpy()
    H, S, K, sub = c.shape
    out = np.zeros((x.shape[0], H, S), np.uint8)
    with np.errstate(all="ignore"):
        for i in range(0, x.shape[0], 64):
            e = x[i:i + 64].reshape(-1, H, S, 1, sub) - c
            d = e * e
            while d.shape[-1] > 1:
                d = d[..., 0::2] + d[..., 1::2]
            d = d[..., 0]
            d = np.where(np.isnan(d), np.float32(np.inf), d)      # never the least
            out[i:i + 64] = d.argmin(-1)
    return out


def codes_at(cache, slots):
    slots = np.asarray(slots)
    p, o = slots // cache.page, slots % cache.page
    return cache.k_codes.cpu().numpy()[p, :, o, :], cache.v_codes.cpu().numpy()[p, :, :, o]


def tokens(cache, n, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, cache.heads, cache.dim, generator=g).to(cache.dtype).to(DEV)
            for _ in range(2)]


WRITE = [
    # heads, dim, sub, K, dtype, tokens, page
    (1, 64, 2, 1, BF, 1, 8),
    (8, 128, 4, 256, BF, 1, 16),
    (3, 96, 8, 200, FP, 67, 16),
    (2, 64, 2, 256, FP, 300, 32),
    (5, 128, 8, 256, BF, 131, 1024),
    (2, 96, 4, 33, BF, 257, 64),
    (1, 128, 2, 16, FP, 33, 8),
    (2, 96, 2, 255, BF, 32, 128),
    (4, 64, 8, 31, BF, 64, 16),
    (2, 64, 4, 129, FP, 31, 8),
]


@pytest.mark.parametrize("heads,dim,sub,K,dtype,n,page", WRITE)
def test_write_codes(heads, dim, sub, K, dtype, n, page):
    pages = -(-n // page) + 2
    cache = make_cache(heads, dim, sub, K, dtype, pages, page, seed=n, random_codes=False)
    cache.k_codes.fill_(251)
    cache.v_codes.fill_(251)
    k, v = tokens(cache, n, 1)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(3))[:n]
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    kc, vc = codes_at(cache, slots)
    assert np.array_equal(kc, nearest(k, cache.k_centres))
    assert np.array_equal(vc, nearest(v, cache.v_centres))
    # nothing else is touched
    rest = np.setdiff1d(np.arange(pages * page), slots.numpy())
    kc, vc = codes_at(cache, rest)
    assert (kc == 251).all() and (vc == 251).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
def test_write_is_the_nearest_in_64_bits(dtype, sub):
    cache = make_cache(2, 64, sub, 256, dtype, 20, 32, seed=sub)
    k, v = tokens(cache, 600, 2)
    slots = torch.arange(600)
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    for x, c, codes in zip((k, v), (cache.k_centres, cache.v_centres), codes_at(cache, slots)):
        H, S, K, _ = c.shape
        e = x.double().cpu().view(-1, H, S, 1, sub) - c.double().cpu()
        d = (e * e).sum(-1)
        got = d.gather(-1, torch.from_numpy(codes).long()[..., None])[..., 0]
        # subtraction, square and three additions: 6 roundings either side
        assert (got <= d.amin(-1) * (1 + 13 * 2.0 ** -24)).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
def test_write_close_calls(dtype, sub):
    """Tokens half way between two centres, and next to that; centres that occur
    twice; centres with one far away, which widens every bound on rounding."""
    cache = make_cache(2, 64, sub, 256, dtype, 40, 32, seed=9)
    for c in (cache.k_centres, cache.v_centres):
        c[:, :, 77] = c[:, :, 12]
        c[:, :, 200:208] = c[:, :, 30:38]
        c[:, 1::2, 255] = 700.0
    g = torch.Generator().manual_seed(5)
    n = 1000
    H, S = 2, 64 // sub
    rows = []
    for c in (cache.k_centres, cache.v_centres):
        c = c.float().cpu()
        i, j = (torch.randint(0, 256, (n, H, S), generator=g) for _ in range(2))
        h, s = torch.arange(H)[:, None], torch.arange(S)
        mid = 0.5 * (c[h, s, i] + c[h, s, j])
        mid[: n // 4] = c[h, s, i][: n // 4]
        rows.append(mid.reshape(n, H, 64).to(dtype).to(DEV))
    k, v = rows
    slots = torch.arange(n)
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    kc, vc = codes_at(cache, slots)
    assert np.array_equal(kc, nearest(k, cache.k_centres))
    assert np.array_equal(vc, nearest(v, cache.v_centres))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
def test_write_unusual_values(dtype, sub):
    cache = make_cache(1, 64, sub, 256, dtype, 8, 16, seed=11)
    k, v = tokens(cache, 64, 4)
    big = 3e38 if dtype is BF else 65504.0
    small = 1e-40 if dtype is BF else 6e-8
    for t in (k, v):
        t[3, 0, 5] = math.nan
        t[4, 0, 9] = math.inf
        t[5, 0, 10] = -math.inf
        t[6] = big
        t[7, 0, ::2] = -big
        t[8] = 0.0
        t[9] = small
        t[10, 0, 1] = 1e4
        t[11] = 0.01 * t[11]
    if dtype is BF:
        cache.v_centres[0, 3] *= 2e19         # squares overflow
        cache.v_centres[0, 5] *= 1e-22        # and underflow
    cache.k_centres[0, 7] *= 1e-6
    slots = torch.arange(64)
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    kc, vc = codes_at(cache, slots)
    assert np.array_equal(kc, nearest(k, cache.k_centres))
    assert np.array_equal(vc, nearest(v, cache.v_centres))
    s = 5 // sub
    assert kc[3, 0, s] == 0 and kc[4, 0, 9 // sub] == 0 and kc[5, 0, 10 // sub] == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
def test_write_below_the_normal_range(dtype, sub):
    """Centres and tokens among the least numbers of the type, and tokens of
    ordinary size that such centres tell apart."""
    cache = make_cache(2, 64, sub, 256, dtype, 20, 32, seed=12)
    tiny = 2.0 ** -17 if dtype is FP else 2.0 ** -130
    cache.k_centres.copy_((tiny * torch.randn(cache.k_centres.shape, device=DEV)).to(dtype))
    k, v = tokens(cache, 600, 6)
    k[:200] = (tiny * k[:200].float()).to(dtype)
    cache.v_centres[..., 0] = (4 * tiny * torch.randn(2, 64 // sub, 256, device=DEV)).to(dtype)
    cache.v_centres[..., 1:] = 0
    v[..., ::sub] = 1.0
    slots = torch.arange(600)
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    kc, vc = codes_at(cache, slots)
    assert np.array_equal(kc, nearest(k, cache.k_centres))
    assert np.array_equal(vc, nearest(v, cache.v_centres))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
@pytest.mark.parametrize("n", [5, 900])
def test_write_few_and_many(n, sub, dtype):
    """The forms for few tokens and for many: ties, values that are no numbers and
    an odd number of centres, in tokens that both take."""
    for n_all in (n, 900):
        cache = make_cache(1, 64, sub, 77, dtype, 60, 16, seed=21, random_codes=False)
        cache.k_centres[:, :, 40:44] = cache.k_centres[:, :, 9:13]
        k, v = tokens(cache, 900, 8)
        k[0, 0, :sub] = cache.k_centres[0, 0, 41]
        k[1, 0, 3], k[2, 0, 7], k[3] = math.nan, -math.inf, 0.0
        v[4] = 3e38 if dtype is BF else 65504.0
        slots = torch.arange(900, device=DEV)
        for i in range(0, n_all, n):
            km.kmeans_kv_write(cache, k[i:i + n], v[i:i + n], slots[i:i + n])
        kc, vc = codes_at(cache, np.arange(n_all))
        assert np.array_equal(kc, nearest(k[:n_all], cache.k_centres))
        assert np.array_equal(vc, nearest(v[:n_all], cache.v_centres))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
def test_write_many_unusual(sub, dtype):
    """The screen for many tokens where its bound is no finite number or every
    centre is within it, from strided tokens, among them padding."""
    n = 1100
    cache = make_cache(1, 64, sub, 250, dtype, 70, 16, seed=22, random_codes=False)
    big = 3e38 if dtype is BF else 65504.0
    both = torch.randn(1, n, 2, 64, device=DEV).to(dtype)
    k, v = both[:, :, 0].transpose(0, 1), both[:, :, 1].transpose(0, 1)
    for t in (k, v):
        t[3, 0, 5], t[4, 0, 9], t[5, 0, 10] = math.nan, math.inf, -math.inf
        t[6] = big
        t[7, 0, ::2] = -big
        t[8] = 0.0
        t[9] = 1e-40 if dtype is BF else 6e-8
        t[10, 0, 1] = 1e4
        t[700:900] *= 0.001
    cache.v_centres[0, 1:3, 17] = big          # its square overflows in the first type
    cache.v_centres[0, 3] *= 2e19 if dtype is BF else 1000.0
    cache.v_centres[0, 5] *= 1e-22 if dtype is BF else 1e-6
    cache.k_centres[0, 2:4] = cache.k_centres[0, 2:4, :1]        # all the same
    slots = torch.arange(n)
    slots[100], slots[200], slots[300] = -1, 70 * 16, 2 ** 45
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    live = np.array([i for i in range(n) if i not in (100, 200, 300)])
    kc, vc = codes_at(cache, live)
    assert np.array_equal(kc, nearest(k, cache.k_centres)[live])
    assert np.array_equal(vc, nearest(v, cache.v_centres)[live])
    kc, vc = codes_at(cache, np.setdiff1d(np.arange(70 * 16), live))
    assert not kc.any() and not vc.any()


@pytest.mark.parametrize("n", [129, 2000, 5000])
def test_write_many_tokens(n):
    """More tokens than one round of the launch takes."""
    cache = make_cache(1 if n > 4000 else 6, 64, 4, 64, BF, -(-n // 64), 64, seed=n)
    k, v = tokens(cache, n, 7)
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(n))
    km.kmeans_kv_write(cache, k, v, slots.to(DEV))
    kc, vc = codes_at(cache, slots)
    assert np.array_equal(kc, nearest(k, cache.k_centres))
    assert np.array_equal(vc, nearest(v, cache.v_centres))


def test_write_strides_and_padding():
    cache = make_cache(3, 64, 4, 50, BF, 10, 16, random_codes=False)
    n = 45
    both = torch.randn(3, n, 2, 64, device=DEV).to(BF)          # heads outermost, k and v mixed
    k, v = both[:, :, 0].transpose(0, 1), both[:, :, 1].transpose(0, 1)
    slots = torch.arange(n) + 7
    slots[5], slots[6], slots[7] = -1, 160, 2 ** 45
    slots[8] = -(2 ** 40)
    wide = torch.stack((slots, slots + 1), 1).to(DEV)
    km.kmeans_kv_write(cache, k, v, wide[:, 0])
    live = np.array([i for i in range(n) if i not in (5, 6, 7, 8)])
    kc, vc = codes_at(cache, slots.numpy()[live])
    assert np.array_equal(kc, nearest(k, cache.k_centres)[live])
    assert np.array_equal(vc, nearest(v, cache.v_centres)[live])
    rest = np.setdiff1d(np.arange(160), slots.numpy()[live])
    kc, vc = codes_at(cache, rest)
    assert not kc.any() and not vc.any()
    # rows that start off 16 bytes, features that are not contiguous, one row for all heads
    odd = torch.randn(n, 3 * 65 + 1, device=DEV).to(BF)[:, 1:].unflatten(1, (3, 65))[:, :, :64]
    turned = torch.randn(n, 64, 3, device=DEV).to(BF).transpose(1, 2)
    one = torch.randn(n, 1, 64, device=DEV).to(BF).expand(n, 3, 64)
    slots = torch.arange(n)
    for a, b in ((odd, turned), (turned, odd), (one, k), (k, one)):
        km.kmeans_kv_write(cache, a, b, slots.to(DEV))
        kc, vc = codes_at(cache, slots)
        assert np.array_equal(kc, nearest(a, cache.k_centres))
        assert np.array_equal(vc, nearest(b, cache.v_centres))


READ = [
    (1, 64, 2, 1, BF, 1, 8),
    (8, 128, 4, 256, BF, 700, 16),
    (3, 96, 8, 200, FP, 67, 32),
    (2, 96, 2, 77, BF, 129, 8),
    (2, 96, 4, 256, FP, 1025, 64),
    (5, 64, 8, 16, FP, 2000, 1024),
    (1, 128, 2, 256, BF, 4099, 16),
    (64, 64, 2, 256, BF, 1030, 16),
    (64, 96, 8, 31, FP, 1500, 8),
    (32, 128, 4, 256, FP, 5003, 64),
    (40, 64, 8, 256, BF, 2047, 32),
    (32, 96, 4, 200, BF, 1999, 16),
    (33, 96, 2, 256, FP, 1024, 128),
    (64, 128, 2, 255, BF, 1111, 8),
    (48, 64, 4, 256, FP, 1201, 1024),
    (64, 128, 8, 256, BF, 513, 16),
]


@pytest.mark.parametrize("heads,dim,sub,K,dtype,n,page", READ)
def test_read(heads, dim, sub, K, dtype, n, page):
    pages = 7
    cache = make_cache(heads, dim, sub, K, dtype, pages, page, seed=n)
    g = torch.Generator().manual_seed(1)
    slots = torch.randint(0, pages * page, (n,), generator=g)
    slots[n // 2] = -5 if n > 1 else slots[0]
    if n > 3:
        slots[n // 3], slots[n // 4] = pages * page, 2 ** 50
    k, v = km.kmeans_kv_read(cache, slots.to(DEV))
    live = (slots >= 0) & (slots < pages * page)
    kc, vc = codes_at(cache, torch.where(live, slots, 0))
    H, S = heads, dim // sub
    h, s = torch.arange(H)[:, None], torch.arange(S)
    for got, codes, c in ((k, kc, cache.k_centres), (v, vc, cache.v_centres)):
        want = c.cpu()[h, s, torch.from_numpy(codes).long()].reshape(n, H, dim)
        want[~live] = 0
        assert torch.equal(got.cpu(), want)
    # into the caller's tensors, heads outermost
    out = [torch.full((heads, n, dim + 8), 7.0, device=DEV, dtype=dtype) for _ in range(2)]
    km.kmeans_kv_read(cache, slots.to(DEV),
                      out=[o[:, :, :dim].transpose(0, 1) for o in out])
    for o, t in zip(out, (k, v)):
        assert torch.equal(o[:, :, :dim].transpose(0, 1), t)
        assert (o[:, :, dim:] == 7.0).all()


READ_RUNS = [
    # heads, dim, sub, K, dtype, tokens, page, first place
    (32, 128, 4, 256, FP, 5003, 64, 0),
    (8, 128, 4, 256, BF, 1031, 8, 0),
    (64, 64, 2, 256, BF, 1030, 16, 8),
    (40, 64, 8, 250, BF, 2047, 32, 3),
    (64, 96, 8, 31, FP, 1500, 16, 5),
    (33, 96, 2, 256, FP, 1024, 128, 1),
    (32, 96, 4, 200, BF, 1999, 1024, 7),
    (48, 64, 4, 256, FP, 1201, 8, 4),
    (64, 128, 2, 255, BF, 1111, 16, 0),
    (64, 128, 8, 256, BF, 513, 64, 9),
]


@pytest.mark.parametrize("heads,dim,sub,K,dtype,n,page,place", READ_RUNS)
def test_read_of_contexts(heads, dim, sub, K, dtype, n, page, place):
    """Tokens side by side on pages in any order, up to the last of the cache, some
    of them left out or elsewhere, from places that are on no boundary."""
    pages = -(-(n + place) // page)
    cache = make_cache(heads, dim, sub, K, dtype, pages, page, seed=n)
    g = torch.Generator().manual_seed(2)
    pos = torch.arange(place, place + n)
    slots = torch.randperm(pages, generator=g)[pos // page] * page + pos % page
    odd = torch.randint(0, n, (5,), generator=g)
    slots[odd] = torch.tensor([-1, pages * page, 0, pages * page - 1, -2 ** 63])
    slots[n - 1] = pages * page - 1
    slots[16:24] = torch.arange(pages * page - 8, pages * page)
    slots[24:32] = torch.arange(7, -1, -1)
    slots[32:40] = torch.arange(-4, 4)
    k, v = km.kmeans_kv_read(cache, slots.to(DEV))
    live = (slots >= 0) & (slots < pages * page)
    kc, vc = codes_at(cache, torch.where(live, slots, 0))
    h, s = torch.arange(heads)[:, None], torch.arange(dim // sub)
    for got, codes, c in ((k, kc, cache.k_centres), (v, vc, cache.v_centres)):
        want = c.cpu()[h, s, torch.from_numpy(codes).long()].reshape(n, heads, dim)
        want[~live] = 0
        assert torch.equal(got.cpu(), want)


def test_codes_past_the_centres_are_zeros():
    cache = make_cache(2, 64, 4, 20, BF, 4, 16)
    cache.k_codes[1, 0, 3, 2] = 20
    cache.v_codes[1, 1, 5, 3] = 255
    k, v = km.kmeans_kv_read(cache, torch.tensor([19], device=DEV))
    assert not k[0, 0, 8:12].any() and k[0, 0, :8].any()
    assert not v[0, 1, 20:24].any() and v[0, 1, 24:].any()
    check_attend(cache, [30], table=[[1, 2]], group=2)


# ---------------------------------------------------------------------------
# attention


def dense(cache, codes, centres):
    """codes [n, H, S] -> [H, n, D] in 64 bits; a code past the centres is zeros."""
    H, S, K, sub = centres.shape
    c = torch.cat((centres.double().cpu(), torch.zeros(H, S, 256 - K, sub, dtype=torch.float64)), 2)
    h, s = torch.arange(H)[:, None], torch.arange(S)
    return c[h, s, codes.long()].reshape(-1, H, cache.dim).transpose(0, 1)


def reference(cache, q, table, lengths, starts, scale):
    """Formula in 64 bits, and bounds on what the kernel's roundings may change:
    (out, lse, bound of out, bound of lse)."""
    B, Hq, D = q.shape
    H = cache.heads
    G = Hq // H
    u = 2.0 ** -9 if q.dtype is BF else 2.0 ** -12        # half a unit of the 16-bit type
    qd = q.double().cpu()
    kc, vc = cache.k_codes.cpu(), cache.v_codes.cpu()
    out = torch.zeros(B, Hq, D, dtype=torch.float64)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64)
    bo, bl = torch.zeros_like(out), torch.zeros(B, Hq, dtype=torch.float64)
    for b in range(B):
        a, n = max(0, starts[b]), lengths[b]
        if n <= a:
            continue
        pos = torch.arange(a, n)
        p, o = table[b][pos // cache.page].long(), pos % cache.page
        k, v = dense(cache, kc[p, :, o, :], cache.k_centres), dense(cache, vc[p, :, :, o], cache.v_centres)
        qb = qd[b].view(H, G, D)
        z = torch.matmul(qb, k.transpose(1, 2)) * scale
        total = torch.logsumexp(z, -1)
        w = torch.exp(z - total[..., None])
        out[b] = torch.matmul(w, v).reshape(Hq, D)
        lse[b] = total.reshape(Hq)
        # a score: D products added in fp32 in any order, the scaling and the
        # change to base 2 (three roundings, each of a value up to the sum of
        # magnitudes); the exponent function to two units
        size = torch.matmul(qb.abs(), k.abs().transpose(1, 2)) * abs(scale)
        ez = ((D + 6) * 2.0 ** -23 * size).amax(-1) + 2.0 ** -20
        # each weight: its rounding to 16 bits (also below the least normal
        # number of fp16, 2^-25 of the largest weight, here of a sum >= 1/64),
        # twice the score's error, and the fp32 sums over n positions
        rel = u + 2 * ez + (n / 32 + 64) * 2.0 ** -23
        sub = 0.0 if q.dtype is BF else 64 * 2.0 ** -25
        spread = torch.matmul(w, v.abs())
        bo[b] = (rel[..., None] * spread + sub * v.abs().sum(1)[:, None]
                 + u * out[b].view(H, G, D).abs() + 2.0 ** -24).reshape(Hq, D)
        bl[b] = (ez + (n / 32 + 64) * 2.0 ** -23 + 2.0 ** -22 * total.abs()).reshape(Hq)
    return out, lse, bo, bl


def run_attend(cache, lengths, table=None, group=1, starts=None, scale=None, seed=0, extra=1,
               spread=2.0, **kw):
    """The call's inputs and outputs; table: rows of pages (None: drawn)."""
    B = len(lengths)
    g = torch.Generator().manual_seed(100 + seed)
    width = max(1, max(-(-x // cache.page) for x in lengths)) + extra
    if table is None:
        table = torch.full((B, width), -1, dtype=torch.int32)
        table[:, ::2] = 2 ** 31 - 1                     # no pages: never followed
        for b, x in enumerate(lengths):
            need = -(-x // cache.page)
            first = (max(0, starts[b]) // cache.page) if starts is not None and x > starts[b] else 0
            table[b, first:need] = torch.randint(0, cache.pages, (need - first,), generator=g,
                                                 dtype=torch.int32)
    else:
        table = torch.tensor(table, dtype=torch.int32)
    q = (spread * torch.randn(B, cache.heads * group, cache.dim, generator=g)).to(cache.dtype)
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV)
    got = km.kmeans_kv_attend(cache, q.to(DEV), table.to(DEV),
                              torch.tensor(lengths, dtype=torch.int32, device=DEV), scale,
                              starts=st, **kw)
    return q, table, got


def check_against(cache, q, table, lengths, starts, scale, got):
    scale = 1 / math.sqrt(cache.dim) if scale is None else scale
    out, lse, bo, bl = reference(cache, q, table, lengths,
                                 [0] * len(lengths) if starts is None else starts, scale)
    o, ls = got[0].double().cpu(), got[1].double().cpu()
    assert torch.equal(torch.isinf(ls), torch.isinf(lse))
    empty = torch.isinf(lse)
    assert (ls[empty] == -math.inf).all() and not o[empty].any()
    worst = ((o - out).abs() / bo.clamp(min=1e-300))[~empty]
    assert not worst.numel() or worst.max() <= 1, worst.max()
    worst = ((ls - lse).abs() / bl.clamp(min=1e-300))[~empty]
    assert not worst.numel() or worst.max() <= 1, worst.max()


def check_attend(cache, lengths, table=None, group=1, starts=None, scale=None, seed=0, **kw):
    q, table, got = run_attend(cache, lengths, table, group, starts, scale, seed, **kw)
    check_against(cache, q, table, lengths, starts, scale, got)
    return got


ATTEND = [
    # heads, dim, sub, K, dtype, page, group
    (1, 64, 2, 256, BF, 16, 1),
    (2, 64, 4, 256, FP, 8, 3),
    (1, 64, 8, 100, BF, 32, 16),
    (2, 96, 2, 200, FP, 16, 4),
    (1, 96, 4, 256, BF, 64, 5),
    (3, 96, 8, 17, FP, 32, 2),
    (2, 128, 2, 256, BF, 8, 8),
    (8, 128, 4, 256, BF, 16, 4),
    (1, 128, 4, 256, FP, 1024, 17),
    (1, 128, 8, 256, BF, 128, 32),
    (2, 128, 8, 1, FP, 16, 1),
]


@pytest.mark.parametrize("heads,dim,sub,K,dtype,page,group", ATTEND)
def test_attend_lengths(heads, dim, sub, K, dtype, page, group):
    cache = make_cache(heads, dim, sub, K, dtype, 70, page, seed=dim + sub)
    check_attend(cache, [1], group=group)
    check_attend(cache, [0], group=group)
    check_attend(cache, [0, 1, 2, 7, 8, 9, 31, 32, 33, 0, 63, 64, 65, 100, 255, 256, 257, 0],
                 group=group, seed=1)
    check_attend(cache, [1000, 3, 517], group=group, seed=2, extra=40)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_attend_every_form(dim, sub, dtype):
    """Up to 8 query heads to a key head and more, few and more than 64 sequences."""
    cache = make_cache(1, dim, sub, 256, dtype, 30, 16, seed=dim * sub)
    check_attend(cache, [70, 5, 411], group=9)
    check_attend(cache, [70, 5, 411], group=8, seed=1)
    check_attend(cache, list(range(65)) + [300], group=2, seed=2)
    check_attend(cache, [33] * 64, group=12, seed=3)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("dim,sub", [(64, 2), (96, 8), (128, 4)])
def test_attend_starts(dtype, dim, sub):
    cache = make_cache(2, dim, sub, 256, dtype, 50, 16, seed=3)
    lengths = [1, 40, 40, 40, 100, 100, 333, 333, 333, 64, 5, 0]
    starts = [0, 39, 40, 55, 31, 32, 300, -7, 95, 63, 9, 0]
    check_attend(cache, lengths, starts=starts, group=3)


def test_attend_split_over_the_length():
    """Sequences that many workgroups share, alone and among short ones."""
    cache = make_cache(2, 128, 4, 256, BF, 300, 64, seed=4)
    check_attend(cache, [20011], group=4)
    check_attend(cache, [3, 9000, 0, 1, 12345, 64, 0], group=2, seed=1)
    cache = make_cache(1, 64, 2, 256, FP, 300, 16, seed=5)
    check_attend(cache, [17, 16411, 900], starts=[0, 1000, 880], group=1, seed=2)


def test_attend_many_sequences():
    cache = make_cache(1, 64, 4, 64, BF, 40, 8, seed=6)
    g = torch.Generator().manual_seed(6)
    lengths = torch.randint(0, 70, (1500,), generator=g).tolist()
    check_attend(cache, lengths, group=2)
    cache = make_cache(1, 128, 8, 64, FP, 40, 8, seed=6)
    lengths = torch.randint(0, 9, (4096,), generator=g).tolist()
    check_attend(cache, lengths, group=1)
    # mostly empty, the rest long, some beyond what is looked up in LDS
    lengths = [0] * 3000
    for b, n in ((0, 700), (63, 40), (64, 33), (1023, 1500), (1024, 64), (2999, 2000)):
        lengths[b] = n
    cache = make_cache(1, 64, 8, 64, BF, 300, 16, seed=7)
    check_attend(cache, lengths, group=2)


def test_attend_head_layouts():
    cache = make_cache(1, 64, 4, 256, BF, 40, 16, seed=7)
    for group in (16, 17, 31, 128):
        check_attend(cache, [5, 200], group=group, seed=group)
    cache = make_cache(33, 64, 4, 16, FP, 40, 16, seed=8)
    check_attend(cache, [5, 200, 90], group=1)


def test_attend_scales():
    cache = make_cache(2, 64, 4, 256, BF, 40, 16, seed=9)
    for scale in (0.0, 1.0, -0.5, 1e-6, 5.0):
        check_attend(cache, [300, 40], group=2, scale=scale)


def test_attend_rising_and_falling_scores():
    """The largest score first, last, and ever larger along the sequence."""
    for dtype in (BF, FP):
        cache = make_cache(1, 64, 8, 256, dtype, 64, 8, seed=10)
        q0 = torch.randn(64, generator=torch.Generator().manual_seed(1))
        for c in range(8):
            cache.k_centres[0, c] = (q0[c * 8:c * 8 + 8] * torch.linspace(-2, 2, 256)[:, None]).to(
                dtype).to(DEV)
        ramp = torch.arange(512, dtype=torch.int64) // 2
        for codes in (ramp, ramp.flip(0), (ramp * 37) % 256):
            cache.k_codes.copy_(codes.to(torch.uint8).view(64, 1, 8, 1).expand(64, 1, 8, 8))
            table = [list(range(64))]
            q = q0.to(dtype).view(1, 1, 64).expand(1, 3, 64).contiguous()
            for scale in (0.125, 1.0):
                got = km.kmeans_kv_attend(cache, q.to(DEV), torch.tensor(table, dtype=torch.int32,
                                                                         device=DEV),
                                          torch.tensor([511], dtype=torch.int32, device=DEV), scale)
                check_against(cache, q, torch.tensor(table), [511], None, scale, got)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attend_long_tail_of_small_weights(dtype):
    """120000 positions that weigh 2^-16.3 of the first one each, 1.5 together."""
    n = 120001
    cache = make_cache(1, 64, 4, 4, dtype, 1876, 64, seed=15)
    cache.k_centres.zero_()
    cache.v_centres.zero_()
    cache.k_centres[0, 0, 1, 0] = 1.0
    cache.v_centres[0, :, 2] = 1.0
    cache.k_codes.zero_()
    cache.v_codes.fill_(2)
    table = torch.arange(1876, dtype=torch.int32, device=DEV)[None]
    cache.k_codes[0, 0, 0, 0] = 1
    cache.v_codes[0, 0, :, 0] = 0
    q = torch.zeros(1, 1, 64, device=DEV, dtype=dtype)
    q[0, 0, 0] = 1.0
    out, lse = km.kmeans_kv_attend(cache, q, table, torch.tensor([n], dtype=torch.int32, device=DEV),
                                   scale=16.3 * math.log(2.0))
    tail = (n - 1) * 2.0 ** -16.3
    want = tail / (1 + tail)
    # the output's own rounding (it lies in [1/2, 1)), the weights' 16 (bf16) or 20 bits, what fp16 cuts
    # off below 2^-24 of weights lifted by 2^7, and the score's rounding
    u, w = (2.0 ** -9, 2.0 ** -15) if dtype is BF else (2.0 ** -12, 2.0 ** -20 + 2.0 ** (16.3 - 31))
    assert (out.double() - want).abs().max() <= u + want * (w + 16.3 * 2.0 ** -21)
    assert abs(lse.item() - (16.3 * math.log(2.0) + math.log1p(tail))) < 1e-5


def test_attend_infinite_scores_and_masked_nan():
    """Scores of +inf give NaN and of -inf weight nothing, as the formula says;
    a centre that only positions outside the span name does not enter, NaN
    included."""
    cache = make_cache(1, 64, 4, 256, BF, 8, 16, seed=11)
    cache.k_centres[0, 0, 255] = math.inf
    cache.v_centres[0, :, 255] = math.nan
    for t in (cache.k_codes, cache.v_codes):
        t[t == 255] = 254
    cache.v_codes[2, :, :, 5:] = 255          # positions 37.. of the sequence
    cache.v_codes[0, :, :, :3] = 255
    table = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device=DEV)
    n, st = (torch.tensor([x], dtype=torch.int32, device=DEV) for x in (37, 3))
    q = torch.randn(1, 2, 64, device=DEV).to(BF)
    q[:, :, 0], q[:, :, 1], q[:, :, 2], q[:, :, 3] = 1.0, 1.0, 1.0, 1.0
    clean, lse = km.kmeans_kv_attend(cache, q, table, n, starts=st)
    assert torch.isfinite(clean).all() and torch.isfinite(lse).all()
    cache.k_codes[1, 0, 4, 0] = 255           # z = +inf at position 20
    out, lse = km.kmeans_kv_attend(cache, q, table, n, starts=st)
    assert torch.isnan(out).all()
    q[:, :, :4] = -1.0                        # z = -inf there: as if it were not attended
    out, lse = km.kmeans_kv_attend(cache, q, table, n, starts=st)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    # -inf everywhere: nothing is attended
    cache.k_codes[:3, 0, :, 0] = 255
    out, lse = km.kmeans_kv_attend(cache, q, table, n, starts=st)
    assert not out.any() and (lse == -math.inf).all()


def test_attend_parts_join():
    """Attention over a span is that of its two parts joined by their lse."""
    cache = make_cache(2, 96, 4, 256, FP, 60, 16, seed=12)
    q, table, (o, l) = run_attend(cache, [700], group=2)
    args = (q.to(DEV), table.to(DEV))
    at = lambda x: torch.tensor([x], dtype=torch.int32, device=DEV)  # noqa: E731
    o1, l1 = km.kmeans_kv_attend(cache, *args, at(333))
    o2, l2 = km.kmeans_kv_attend(cache, *args, at(700), starts=at(333))
    whole = torch.logaddexp(l1, l2)
    joined = (torch.exp(l1 - whole)[..., None] * o1.float()
              + torch.exp(l2 - whole)[..., None] * o2.float())
    assert (whole - l).abs().max() < 1e-4
    # three outputs rounded to fp16, weights likewise: 4 halves of a unit of |v| <= 5
    assert (joined - o.float()).abs().max() < 4 * 2.0 ** -12 * 5


def test_attend_strides_streams_and_repeats():
    cache = make_cache(2, 128, 4, 256, BF, 200, 16, seed=13)
    lengths = [2500, 3, 0, 777]
    q, table, (o, l) = run_attend(cache, lengths, group=4)
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    qd, td = q.to(DEV), table.to(DEV)
    # the same bits again, on another stream, from strided inputs, into the caller's outputs
    o2, l2 = km.kmeans_kv_attend(cache, qd, td, n)
    assert torch.equal(o, o2) and torch.equal(l, l2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        big = torch.zeros(8, 4, 2 * 128 + 8, device=DEV, dtype=BF).transpose(0, 1)
        big[:, :, :128] = qd
        wide = torch.zeros(4, td.shape[1] + 5, device=DEV, dtype=torch.int32)
        wide[:, :td.shape[1]] = td
        out = torch.full((8, 4, 136), 7.0, device=DEV, dtype=BF).transpose(0, 1)
        lse = torch.empty(4, 8, device=DEV)
        ws = torch.full((cache.attend_workspace_bytes(4, 8, td.shape[1]),), 255, device=DEV,
                        dtype=torch.uint8)
        nn = torch.stack((n, n), 1)[:, 0]
        got = km.kmeans_kv_attend(cache, big[:, :, :128], wide[:, :td.shape[1]], nn,
                                  out=out[:, :, :128], lse=lse, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert got[1] is lse
    assert torch.equal(out[:, :, :128], o) and torch.equal(lse, l)
    assert (out[:, :, 128:] == 7.0).all()
    # a query that starts off 16 bytes, features not contiguous
    odd = torch.zeros(4 * 8 * 128 + 1, device=DEV, dtype=BF)[1:].view(4, 8, 128)
    odd.copy_(qd)
    turned = qd.transpose(1, 2).contiguous().transpose(1, 2)
    for x in (odd, turned):
        o2, l2 = km.kmeans_kv_attend(cache, x, td, n)
        assert torch.equal(o, o2) and torch.equal(l, l2)


def test_attend_table_of_zero_width_and_zero_sequences():
    cache = make_cache(2, 64, 4, 16, BF, 4, 16)
    q = torch.randn(3, 4, 64, device=DEV).to(BF)
    n = torch.tensor([5, 0, 2], dtype=torch.int32, device=DEV)
    out, lse = km.kmeans_kv_attend(cache, q, torch.zeros(3, 0, dtype=torch.int32, device=DEV), n)
    assert not out.any() and (lse == -math.inf).all()
    out, lse = km.kmeans_kv_attend(cache, q[:0], torch.zeros(0, 2, dtype=torch.int32, device=DEV),
                                   n[:0])
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    # lengths past the table and below zero
    table = torch.tensor([[0, 1], [2, 3], [1, 2]], dtype=torch.int32, device=DEV)
    big = torch.tensor([2 ** 31 - 1, -9, 32], dtype=torch.int32, device=DEV)
    got = km.kmeans_kv_attend(cache, q, table, big)
    check_against(cache, q.cpu(), table.cpu(), [32, 0, 32], None, None, got)


def test_write_read_zero_tokens():
    cache = make_cache(2, 64, 4, 16, BF, 4, 16)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    empty = torch.zeros(0, 2, 64, device=DEV, dtype=BF)
    km.kmeans_kv_write(cache, empty, empty, none)
    k, v = km.kmeans_kv_read(cache, none)
    assert k.shape == v.shape == (0, 2, 64)


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB of key codes, used at its far end."""
    heads, dim, sub, page = 8, 128, 4, 64
    kc, vc = (torch.randn(heads, 32, 256, 4, device=DEV).to(BF) for _ in range(2))
    pages = (1 << 32) // (heads * page * 32) + 40
    codes = [torch.empty(s, dtype=torch.uint8, device=DEV)
             for s in ((pages, heads, page, 32), (pages, heads, 32, page))]
    cache = km.KVCodes(kc, vc, *codes)
    n = 300
    k, v = tokens(cache, n, 1)
    table = torch.arange(pages - 1, pages - 6, -1, dtype=torch.int32, device=DEV)[None]
    pos = torch.arange(n, device=DEV)
    slots = table[0][pos // page].long() * page + pos % page
    km.kmeans_kv_write(cache, k, v, slots)
    small = km.KVCodes(kc, vc, *(c[-6:].clone() for c in codes))
    shift = (pages - 6) * page
    for a, b in zip(km.kmeans_kv_read(cache, slots), km.kmeans_kv_read(small, slots - shift)):
        assert torch.equal(a, b)
    cs = small.k_codes.cpu().numpy()[(slots - shift).cpu() // page, :, (slots - shift).cpu() % page]
    assert np.array_equal(cs, nearest(k, kc))
    q = torch.randn(1, 32, dim, device=DEV).to(BF)
    ln = torch.tensor([n], dtype=torch.int32, device=DEV)
    for a, b in zip(km.kmeans_kv_attend(cache, q, table, ln),
                    km.kmeans_kv_attend(small, q, table - (pages - 6), ln)):
        assert torch.equal(a, b)


def test_graph_replays():
    """A decode step captured in a graph: write, then attend, replayed with the
    program's own work between."""
    cache = make_cache(2, 128, 4, 256, BF, 64, 16, seed=14, random_codes=True)
    q = torch.zeros(3, 8, 128, device=DEV, dtype=BF)
    k, v = (torch.zeros(3, 2, 128, device=DEV, dtype=BF) for _ in range(2))
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    n = torch.zeros(3, dtype=torch.int32, device=DEV)
    table = torch.randperm(60, generator=torch.Generator().manual_seed(1)).view(3, 20).to(
        torch.int32).to(DEV)
    out, lse = torch.empty(3, 8, 128, device=DEV, dtype=BF), torch.empty(3, 8, device=DEV)
    ws = torch.empty(cache.attend_workspace_bytes(3, 8, 20), dtype=torch.uint8, device=DEV)

    def step():
        km.kmeans_kv_write(cache, k, v, slots)
        km.kmeans_kv_attend(cache, q, table, n, out=out, lse=lse, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(2)
    start = torch.tensor([0, 100, 250])
    for i in range(5):
        q.copy_(torch.randn(q.shape, generator=g))
        k.copy_(torch.randn(k.shape, generator=g))
        v.copy_(torch.randn(v.shape, generator=g))
        pos = start + 13 * i
        slots.copy_(table.cpu().long().gather(1, (pos // 16)[:, None])[:, 0] * 16 + pos % 16)
        n.copy_((pos + 1).to(torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        step()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
        check_against(cache, q.cpu(), table.cpu(), (pos + 1).tolist(), None, None, got)


# ---------------------------------------------------------------------------
# refusals


def test_refusals_of_the_binding():
    cache = make_cache(2, 64, 4, 16, BF, 4, 16)
    k, v = tokens(cache, 3, 1)
    slots = torch.arange(3, device=DEV)
    with pytest.raises(ValueError):
        km.kmeans_kv_write(cache, k.float(), v, slots)
    with pytest.raises(ValueError):
        km.kmeans_kv_write(cache, k, v[:2], slots)
    with pytest.raises(ValueError):
        km.kmeans_kv_write(cache, k[:, :1], v, slots)
    with pytest.raises(ValueError):
        km.kmeans_kv_write(cache, k, v, slots.int())
    with pytest.raises(ValueError):
        km.kmeans_kv_write(cache, k.cpu(), v, slots)
    with pytest.raises(ValueError):
        km.kmeans_kv_read(cache, slots[:, None])
    with pytest.raises(ValueError):
        km.kmeans_kv_read(cache, slots, out=(k[:1].expand(3, 2, 64), v))
    q = torch.randn(3, 4, 64, device=DEV).to(BF)
    table = torch.zeros(3, 2, dtype=torch.int32, device=DEV)
    n = torch.ones(3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q[:, :3], table, n)
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q.half(), table, n)
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q, table[:2], n)
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q, table.long(), n)
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q, table, n[:2])
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q, table, n, starts=n.long())
    with pytest.raises(ValueError):
        km.kmeans_kv_attend(cache, q, table, n, lse=torch.empty(3, 4, device=DEV, dtype=BF))
    with pytest.raises(km.KmeansError):
        km.kmeans_kv_attend(cache, q, table, n, scale=math.inf)
    with pytest.raises(km.KmeansError):
        km.kmeans_kv_attend(cache, q, table, n, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    c = cache.k_centres
    with pytest.raises(ValueError):
        km.KVCodes(c, cache.v_centres.half(), cache.k_codes, cache.v_codes)
    with pytest.raises(ValueError):
        km.KVCodes(c, c, cache.k_codes, cache.v_codes[:3])
    with pytest.raises(ValueError):
        km.KVCodes(c, c, cache.k_codes.int(), cache.v_codes)
    for shape, page in (((2, 16, 16, 5), 16), ((2, 16, 300, 4), 16), ((2, 16, 16, 4), 24),
                        ((2, 16, 16, 4), 4), ((2, 20, 16, 4), 16)):
        bad = torch.zeros(shape, device=DEV, dtype=BF)
        with pytest.raises(km.KmeansError):
            km.KVCodes.empty(bad, bad, 4, page)
