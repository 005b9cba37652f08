"""What kmeans_kv_rotate, kmeans_kv_attend_tokens, kmeans_kv_weigh and kmeans_kv_evict
are defined to return, in 64 bits and plain steps (helpers of test_gpu_kv_serve*.py)."""
import math

import torch

import paper_1402_3788_amd as km

DEV = torch.device("cuda:0") if torch.cuda.is_available() else None
BF, FP = torch.bfloat16, torch.float16


def make_cache(heads, dim, sub, K, dtype, pages, page, seed=0):
    g = torch.Generator().manual_seed(seed)
    S = dim // sub
    kc, vc = (torch.randn(heads, S, K, sub, generator=g).to(dtype).to(DEV) for _ in range(2))
    cache = km.KVCodes.empty(kc, vc, pages, page)
    for t in (cache.k_codes, cache.v_codes):
        t.copy_(torch.randint(0, K, t.shape, generator=g, dtype=torch.uint8))
    return cache


class Call:
    """A cache, sequences in it and new tokens: sizes is a list of (cached positions
    with the new ones, new tokens)."""

    def __init__(self, sizes, heads=2, group=2, dim=64, sub=4, K=256, dtype=BF, page=16, seed=0,
                 more_tokens=0, q_scale=2.0):
        g = torch.Generator().manual_seed(seed + 1)
        self.sizes, self.heads, self.group = sizes, heads, group
        need = [-(-n // page) for n, _ in sizes]
        self.pages, width = sum(need) + 3, max(max(need, default=0), 1)
        self.cache = make_cache(heads, dim, sub, K, dtype, self.pages, page, seed)
        perm = torch.randperm(self.pages, generator=g).to(torch.int32)
        # entries that no position needs are numbers of no page
        table = torch.full((len(sizes), width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = perm[at:at + n]
            at += n
        self.spare = perm[at:]
        self.table = table.to(DEV)
        self.lengths = torch.tensor([n for n, _ in sizes], dtype=torch.int32, device=DEV)
        bounds = [0]
        for _, n in sizes:
            bounds.append(bounds[-1] + n)
        self.bounds = torch.tensor(bounds, dtype=torch.int32, device=DEV)
        self.q = (q_scale * torch.randn(bounds[-1] + more_tokens, heads * group, dim, generator=g)
                  ).to(dtype).to(DEV)
        self.scale = 1.0 / math.sqrt(dim)
        self.more = {}

    def attend(self, **kw):
        return km.kmeans_kv_attend_tokens(self.cache, self.q, self.bounds, self.table, self.lengths,
                                          **{**self.more, **kw})

    def weigh(self, lse, weights=None, **kw):
        return km.kmeans_kv_weigh(self.cache, self.q, lse, self.bounds, self.table, self.lengths,
                                  weights, **{**self.more, **kw})


def values(codes, book):
    """codes [n, H, S] -> [H, n, dim], zeros for a code past the centres."""
    H, S, K, sub = book.shape
    book = torch.cat((book.double(), torch.zeros(H, S, 256 - K, sub, dtype=torch.float64,
                                                 device=book.device)), 2)
    h, s = torch.arange(H, device=book.device)[:, None], torch.arange(S, device=book.device)
    return book[h, s, codes.long()].reshape(codes.shape[0], H, S * sub).transpose(0, 1)


def sequence(call, b):
    """Keys and values [H, n, dim] of a sequence's positions, and its new tokens'
    numbers and positions."""
    c = call.cache
    n = min(max(int(call.lengths[b]), 0), call.table.shape[1] * c.page)
    T = call.q.shape[0]
    t0 = min(max(int(call.bounds[b]), 0), T)
    t1 = min(max(int(call.bounds[b + 1]), t0), T)
    i = torch.arange(n, device=DEV)
    p = call.table[b][i // c.page].long().clamp(0, c.pages - 1)
    k = values(c.k_codes[p, :, i % c.page], c.k_centres)
    v = values(c.v_codes[p, :, :, i % c.page], c.v_centres)
    return k, v, t0, t1, n - (t1 - t0) + torch.arange(t1 - t0, device=DEV)


def scores(call, b):
    """z [H, G, new, n] in fp64 with -inf where nothing is seen, how far fp32 may take
    each, k, v, t0, t1."""
    m = call.more
    k, v, t0, t1, pos = sequence(call, b)
    n = k.shape[1]
    H, G, D = call.heads, call.group, k.shape[2]
    q = call.q[t0:t1].double().view(t1 - t0, H, G, D).permute(1, 2, 0, 3)
    kt = k.transpose(1, 2)[:, None]
    scale = m.get("scale")
    scale = 1 / math.sqrt(D) if scale is None else scale
    z = torch.matmul(q, kt) * scale
    # a sum of D products in any order: D - 1 additions; the product with the scale
    off = torch.matmul(q.abs(), kt.abs()) * abs(scale) * (D + 4) * 2.0 ** -24
    cap = m.get("cap", 0.0)
    if cap:
        z = cap * torch.tanh(z / cap)
        # the derivative of tanh is at most 1; 2 / (1 + e) to three roundings
        off = off + cap * 2.0 ** -21
    i = torch.arange(n, device=DEV)
    far = (pos[:, None] - i).abs().double()
    if m.get("slopes") is not None:
        slopes = m["slopes"].double().view(H, G, 1, 1)
        z = z - slopes * far
        off = off + (slopes * far).abs() * 2.0 ** -22
    high = pos + 1
    if m.get("prefixes") is not None:
        high = torch.maximum(high, m["prefixes"][b].long())
    high = high.clamp(max=n)
    low = torch.zeros_like(pos)
    if m.get("window"):
        low = torch.maximum(low, pos - m["window"] + 1)
    if m.get("starts") is not None:
        low = torch.maximum(low, m["starts"][t0:t1].long())
    seen = (i >= low[:, None]) & (i < high[:, None])
    off = off + z.abs().nan_to_num(0, 0, 0) * 2.0 ** -22 + 2.0 ** -21
    return z.masked_fill(~seen, -math.inf), off.masked_fill(~seen, 0.0), k, v, t0, t1


def attention(call):
    """(out, lse) in fp64 of the tokens in sequences, and the bounds of their errors;
    NaN for the tokens outside."""
    T, Hq, D = call.q.shape
    out = torch.full((T, Hq, D), math.nan, dtype=torch.float64, device=DEV)
    lse = torch.full((T, Hq), math.nan, dtype=torch.float64, device=DEV)
    d_out, d_lse = torch.zeros_like(out), torch.zeros_like(lse)
    half = torch.finfo(call.cache.dtype).eps / 2
    tiny = torch.finfo(call.cache.dtype).smallest_normal
    for b in range(len(call.sizes)):
        z, off, k, v, t0, t1 = scores(call, b)
        if z.shape[-1] == 0:
            z, off = z.new_full((*z.shape[:-1], 1), -math.inf), off.new_zeros((*off.shape[:-1], 1))
            v = v.new_zeros(v.shape[0], 1, D)
        total = torch.logsumexp(z, -1)
        w = torch.exp(z - torch.where(total == -math.inf, 0.0, total)[..., None])
        vv = v[:, None]
        o = torch.matmul(w, vv)
        top = off.amax(-1, keepdim=True)

        def rows(x):
            return x.permute(2, 0, 1, *range(3, x.dim())).reshape(t1 - t0, Hq, *x.shape[3:])

        out[t0:t1], lse[t0:t1] = rows(o), rows(total)
        # every weight off by its score's error, once more by the sum's, and by the
        # rounding to 16 bits; sums of n fp32 numbers; the result's own rounding
        n = z.shape[-1]
        rel = 2 * top + half + (n ** 0.5 + 64) * 2.0 ** -22
        d_out[t0:t1] = rows(half * o.abs() + rel * torch.matmul(w, vv.abs()) + tiny)
        d_lse[t0:t1] = rows((top + (n ** 0.5 + 64) * 2.0 ** -22)[..., 0]
                            + total.abs().nan_to_num(0, 0, 0) * 2.0 ** -22)
    return out, lse, d_out, d_lse


def check_attention(call, got=None):
    out, lse = call.attend() if got is None else got
    o, s, d_o, d_s = attention(call)
    inside = ~torch.isnan(s)
    o, d_o, got_o = o[inside], d_o[inside], out.double()[inside]
    assert torch.isfinite(got_o).all()
    worst = ((got_o - o).abs() / d_o).max().item() if o.numel() else 0.0
    assert worst <= 1.0, f"out off by {worst} of its bound"
    s, d_s, got_s = s[inside], d_s[inside], lse.double()[inside]
    none = s == -math.inf
    assert torch.equal(none, got_s == -math.inf)
    assert (got_o[none] == 0).all()
    assert ((got_s - s).abs()[~none] <= d_s[~none]).all()
    return out, lse


def weights_of(call, lse, positions):
    """[seqs, heads, positions] in fp64 and the bounds of their errors."""
    B, H = len(call.sizes), call.heads
    w = torch.zeros(B, H, positions, dtype=torch.float64, device=DEV)
    d = torch.zeros_like(w)
    for b in range(B):
        z, off, k, v, t0, t1 = scores(call, b)
        n = min(z.shape[-1], positions)
        x = lse[t0:t1].double().view(t1 - t0, H, call.group).permute(1, 2, 0)[..., None]
        none = x == -math.inf
        e = torch.exp(z - torch.where(none, 0.0, x)).masked_fill(none, 0.0)
        w[b, :, :n] = e.sum((1, 2))[:, :n]
        count = e.shape[1] * e.shape[2]
        e = e * (off + torch.where(none, 0.0, x.abs()) * 2.0 ** -23 + (count + 8) * 2.0 ** -24)
        d[b, :, :n] = e.sum((1, 2))[:, :n]
    return w, d + 1e-30


def evicted(weights, lengths, keep, recent, first):
    """(kept, lengths, weights) by sorting on the host."""
    w = weights.cpu()
    B, H, P = w.shape
    kept = torch.full((B, H, keep), -1, dtype=torch.int32)
    out = torch.zeros_like(w)
    left = []
    for b, n in enumerate(lengths.tolist()):
        left.append(min(n, keep))
        for h in range(H):
            x = w[b, h].tolist() + [0.0] * max(0, n - P)
            if n <= keep:
                got = list(range(n))
            else:
                sure = set(range(first)) | set(range(n - recent, n))
                rest = sorted((i for i in range(n) if i not in sure),
                              key=lambda i: (x[i] != x[i], -x[i] if x[i] == x[i] else 0.0, i))
                got = sorted(sure | set(rest[:keep - len(sure)]))
            for j, i in enumerate(got):
                kept[b, h, j] = i
                if j < P:
                    out[b, h, j] = x[i]
    return kept, torch.tensor(left, dtype=torch.int32), out
