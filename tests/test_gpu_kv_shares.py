"""Attention over K-means codes, whose positions are shared by waves and workgroups:
bounds so close that no wave's share can be missing from an output.

Keys are multiples of 1/8 and queries of 1/4, so that fp32 holds every score
exactly; what remains are the weights' and the sums' roundings."""
import math

import pytest
import torch

import paper_1402_3788_amd as km

BF, FP = torch.bfloat16, torch.float16

CASES = [
    # dim, sub, heads, group, dtype, page, (starts, lengths)
    (64, 2, 1, 1, FP, 16, ([0, 1000, 880], [17, 16411, 900])),
    (64, 4, 2, 8, FP, 32, ([0], [9001])),
    (96, 8, 1, 9, FP, 16, ([5, 0], [8200, 33])),
    (128, 4, 2, 12, FP, 64, ([0, 0, 40], [3000, 0, 2600])),
    (128, 4, 2, 4, BF, 64, ([0], [20011])),
    (64, 2, 1, 3, BF, 8, ([0, 7], [5000, 6000])),
    (96, 4, 1, 16, BF, 128, ([0, 0], [4100, 700])),
    (128, 8, 4, 1, BF, 16, ([0, 30, 0], [2000, 2500, 31])),
    # one workgroup to a head and many tiles: nothing is left to the second launch
    (64, 8, 130, 1, FP, 32, ([0, 0, 100], [1500, 40, 1200])),
    (64, 4, 300, 1, BF, 16, ([0, 9], [1100, 700])),
    (128, 8, 5, 128, BF, 16, ([0, 0, 3], [500, 1300, 77])),
    (96, 2, 12, 33, FP, 64, ([17, 0], [900, 1000])),
    # more of them than compute units
    (128, 4, 97, 40, BF, 32, ([0, 2], [200, 450])),
]


class Inputs:
    """Centres, codes, queries and a table, on the host."""

    def __init__(self, dim, sub, heads, group, dtype, page, spans, K=256):
        g = torch.Generator().manual_seed(dim * sub + heads)
        self.dim, self.sub, self.heads, self.group, self.dtype, self.page = (
            dim, sub, heads, group, dtype, page)
        self.starts, self.lengths = spans
        S = dim // sub
        self.k_centres = (torch.randn(heads, S, K, sub, generator=g).clamp(-3, 3) * 8).round() / 8
        self.v_centres = torch.randn(heads, S, K, sub, generator=g).to(dtype).double()
        need = [-(-n // page) for n in self.lengths]
        self.pages = sum(need) + 1
        self.k_codes = torch.randint(0, K, (self.pages, heads, page, S), generator=g,
                                     dtype=torch.uint8)
        self.v_codes = torch.randint(0, K, (self.pages, heads, S, page), generator=g,
                                     dtype=torch.uint8)
        self.table = torch.full((len(need), max(need) + 1), -1, dtype=torch.int32)
        free = torch.randperm(self.pages, generator=g).to(torch.int32)
        for b, n in enumerate(need):
            self.table[b, :n], free = free[:n], free[n:]
        self.q = (torch.randn(len(need), heads * group, dim, generator=g) * 4).round() / 4
        self.scale = 1.0 / math.sqrt(dim)

    def rows(self, b, h):
        """Keys and values that head h of sequence b attends, in 64 bits."""
        pos = torch.arange(self.starts[b], self.lengths[b])
        p, off = self.table[b][pos // self.page].long(), pos % self.page
        s = torch.arange(self.dim // self.sub)
        k = self.k_centres[h].double()[s, self.k_codes[p, h, off].long()]
        v = self.v_centres[h][s, self.v_codes[p, h, :, off].long()]
        return k.reshape(-1, self.dim), v.reshape(-1, self.dim)

    def reference(self, b, h, also=()):
        """(out, lse, bound of out, bound of lse) of the group's queries, and for each
        stretch of positions in `also` what it adds to out and its part of the sum."""
        k, v = self.rows(b, h)
        q = self.q[b, h * self.group:(h + 1) * self.group].double()
        z = (q @ k.T) * self.scale
        lse = torch.logsumexp(z, -1)
        w = torch.exp(z - lse[:, None])
        out, spread = w @ v, w @ v.abs()
        n, top = z.shape[1], z.amax(-1)
        bf16 = self.dtype is BF
        # A weight against the largest: the scale in base 2 (three roundings) and the
        # argument's own, each of a distance that the reference, up to 8 + 7 in base 2
        # behind the largest score, adds to; the exponential, and 8 changes of the
        # reference and joinings, two roundings each.
        off = 2.0 ** -20 + 2.0 ** -22 * (top[:, None] - z + 15 * math.log(2))
        # Its two parts: of bf16 8 bits each, to nearest; of fp16 11 bits each, cut
        # off, and below 2^-31 of the largest weight nothing.
        parts = 2.0 ** -17 if bf16 else 2.0 ** -21
        lost = 0.0 if bf16 else 2.0 ** -31 * torch.exp(top - lse)
        # fp32 sums over 32 positions at a time, and over lanes, waves and workgroups
        sums = (n / 32 + 64) * 2.0 ** -24
        half = 2.0 ** -8 if bf16 else 2.0 ** -11          # of a unit of the output
        total = (w * off).sum(-1) + sums
        bound_out = ((w * (off + parts)) @ v.abs() + sums * spread + total[:, None] * out.abs()
                     + half * out.abs() + 2.0 ** -25)
        if not bf16:
            bound_out += lost[:, None] * v.abs().sum(0)
        bound_lse = total + 2.0 ** -21 * (lse.abs() + 15)
        parts_of = [(w[:, a:e] @ v[a:e], w[:, a:e].sum(-1)) for a, e in also]
        return (out, lse, bound_out, bound_lse), parts_of

    def shares(self):
        """The stretches [sequence, first, end) (positions from `starts`) that a wave
        or a workgroup takes: the tiles of 32 positions of all sequences in a row,
        shared evenly by the workgroups of a head and their waves."""
        waves = 16 if self.dim == 64 else 12
        ranges, tiles = [], 0
        for a, n in zip(self.starts, self.lengths):
            count = -(-n // 32) - a // 32 if n > a else 0
            ranges.append((tiles, tiles + count))
            tiles += count
        blocks = self.heads * -(-self.group // 16)
        splits = min(max(1, 256 // blocks), max(1, -(-tiles // waves)))

        def even(lo, hi, count):
            each, more = divmod(hi - lo, count)
            at = [lo + i * each + min(i, more) for i in range(count + 1)]
            return list(zip(at, at[1:]))

        groups = even(0, tiles, splits)
        got = []
        for lo, hi in groups + [w for g in groups for w in even(*g, waves)]:
            for b, (first, end) in enumerate(ranges):
                x, y = max(lo, first), min(hi, end)
                if x < y:
                    a, n = self.starts[b], self.lengths[b]
                    p = [(t - first + a // 32) * 32 for t in (x, y)]
                    got.append((b, max(p[0], a) - a, min(p[1], n) - a))
        return sorted(set(got))


@pytest.mark.parametrize("case", CASES[:8], ids=str)
def test_no_share_can_be_missing(case):
    """Every share's part of an output is more than the bound somewhere, so that an
    output without it would not pass, and so is its part of the sum."""
    x = Inputs(*case)
    shares = x.shares()
    assert len(shares) > 40
    for b in range(len(x.lengths)):
        mine = [(a, e) for s, a, e in shares if s == b]
        if not mine:
            continue
        (out, lse, bound_out, bound_lse), parts = x.reference(b, 0, mine)
        for (a, e), (part, weight) in zip(mine, parts):
            assert (part.abs() > bound_out).any(), (b, a, e)
            assert (-torch.log1p(-weight.clamp(max=1 - 1e-9)) > bound_lse).any(), (b, a, e)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_all_shares_are_in(case):
    x = Inputs(*case)
    dev = torch.device("cuda:0")
    cache = km.KVCodes(x.k_centres.to(x.dtype).to(dev), x.v_centres.to(x.dtype).to(dev),
                       x.k_codes.to(dev), x.v_codes.to(dev))
    at = [torch.tensor(t, dtype=torch.int32, device=dev) for t in (x.lengths, x.starts)]
    out, lse = km.kmeans_kv_attend(cache, x.q.to(x.dtype).to(dev), x.table.to(dev), at[0],
                                   x.scale, starts=at[1])
    out, lse = out.double().cpu(), lse.double().cpu()
    heads = range(x.heads) if x.heads < 8 else (0, 1, x.heads // 2, x.heads - 1)
    for b in range(len(x.lengths)):
        for h in heads:
            mine = slice(h * x.group, (h + 1) * x.group)
            if x.lengths[b] <= x.starts[b]:
                assert not out[b, mine].any() and (lse[b, mine] == -math.inf).all()
                continue
            (o, l, bo, bl), _ = x.reference(b, h)
            assert ((out[b, mine] - o).abs() <= bo).all(), (b, h, ((out[b, mine] - o).abs() / bo).max())
            assert ((lse[b, mine] - l).abs() <= bl).all(), (b, h, ((lse[b, mine] - l).abs() / bl).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, FP])
def test_long_tail_of_small_weights_of_many_queries(dtype):
    """120000 positions that weigh 2^-16.3 of the first one each, 1.5 together, in
    the form for more than 8 queries to a key head."""
    dev = torch.device("cuda:0")
    n = 120001
    centres = [torch.zeros(1, 16, 4, 4, device=dev, dtype=dtype) for _ in range(2)]
    centres[0][0, 0, 1, 0] = 1.0
    centres[1][0, :, 2] = 1.0
    cache = km.KVCodes.empty(*centres, 1876, 64)
    cache.v_codes.fill_(2)
    table = torch.arange(1876, dtype=torch.int32, device=dev)[None]
    cache.k_codes[0, 0, 0, 0] = 1
    cache.v_codes[0, 0, :, 0] = 0
    q = torch.zeros(1, 12, 64, device=dev, dtype=dtype)
    q[:, :, 0] = 1.0
    out, lse = km.kmeans_kv_attend(cache, q, table, torch.tensor([n], dtype=torch.int32, device=dev),
                                   scale=16.3 * math.log(2.0))
    tail = (n - 1) * 2.0 ** -16.3
    want = tail / (1 + tail)
    # the output's own rounding (it lies in [1/2, 1)), the weights' parts, what fp16 cuts
    # off below 2^-31 of the largest, and the score's rounding
    u, w = (2.0 ** -9, 2.0 ** -17) if dtype is BF else (2.0 ** -12, 2.0 ** -21 + 2.0 ** (16.3 - 31))
    assert (out.double() - want).abs().max() <= u + want * (w + 16.3 * 2.0 ** -21)
    assert (lse.double() - (16.3 * math.log(2.0) + math.log1p(tail))).abs().max() < 1e-5
