"""Serving from the key-value cache in K-means codes, as measurable cases: queries
and keys turned by their positions, attention of many new tokens with caps, biases
and masks, the weight that attention gave to every position, and the eviction of
positions that got little.

The cache: keys are [pages][heads][page][dim/sub] codes of one byte, values
[pages][heads][dim/sub][page], each the number of a centre of its head and
sub-vector. A case is a dict of plain values:

    op      "rotate" (new queries and keys are turned), "attend" (new tokens attend
            over the cache), "weigh" (the attention weights of new tokens are summed
            for each cached position), "evict" (positions of large summed weight
            move to fresh pages)
    dtype   "bf16" or "fp16"
    heads   key-value heads; group: query heads of each
    dim, sub, centres, page   as above; page tokens to a page
    tokens, rot, interleaved, inverse, stretch, amplitude     of "rotate": features
            [0, rot) of a head are turned; frequencies base 10000 ** (-2 i / rot),
            divided by stretch
    seqs, lo, hi     sequences with cached positions spaced from lo to hi on their
            logarithm (lo 0: the first has none)
    new_lo, new_hi   of "attend" and "weigh": new tokens of each, at the end of its
            positions (which they add to)
    cap (0: none), slopes (a distance bias or not), window (0: none), prefix (first
            positions that every token sees), docs (0, or the length of documents:
            a token sees its own; every 17th token is padding and sees nothing)
    keep, recent, first       of "evict": kept positions, of them always the last
            `recent` and the first `first`
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    score = dict(cap=0.0, slopes=False, window=0, prefix=0, docs=0)
    return [
        # A decode step of 37 sequences, half of each head turned, fp16.
        dict(name="rotate-37-part", op="rotate", dtype="fp16", tokens=37, heads=5, group=4, dim=96,
             rot=48, interleaved=True, inverse=False, stretch=1.0, amplitude=1.0),
        # A prompt of 8192 tokens in a context stretched four times.
        dict(name="rotate-8192", op="rotate", dtype="bf16", tokens=8192, heads=8, group=8, dim=128,
             rot=128, interleaved=False, inverse=False, stretch=4.0, amplitude=1.14),
        # One sequence that has just begun, scores capped: latency.
        dict(name="attend-1x77-cap", op="attend", dtype="bf16", seqs=1, lo=76, hi=76, new_lo=1,
             new_hi=1, heads=8, group=4, dim=128, sub=4, centres=256, page=16,
             **{**score, "cap": 30.0}),
        # A decode step of a serving batch, scores that fall with the distance.
        dict(name="attend-32x4096-slopes", op="attend", dtype="bf16", seqs=32, lo=512, hi=4096,
             new_lo=1, new_hi=1, heads=8, group=4, dim=128, sub=4, centres=256, page=16,
             **{**score, "slopes": True}),
        # Five proposed tokens of each sequence checked at once, a sliding window,
        # one bit a feature and an odd code book.
        dict(name="attend-17x8191-verify", op="attend", dtype="fp16", seqs=17, lo=100, hi=8191,
             new_lo=5, new_hi=5, heads=3, group=5, dim=96, sub=8, centres=200, page=64,
             **{**score, "window": 1000}),
        # Ragged prompts of several documents each, with a common prefix and padding.
        dict(name="attend-8x1000-docs", op="attend", dtype="fp16", seqs=8, lo=0, hi=0, new_lo=101,
             new_hi=1000, heads=12, group=1, dim=64, sub=2, centres=256, page=32,
             **{**score, "prefix": 40, "docs": 150}),
        # A question of 256 tokens about a document of 65536.
        dict(name="attend-1x64k-chunk", op="attend", dtype="bf16", seqs=1, lo=65536, hi=65536,
             new_lo=256, new_hi=256, heads=8, group=8, dim=128, sub=4, centres=256, page=64,
             **{**score, "cap": 50.0, "slopes": True}),
        # The last 4096 tokens of a prompt of 16384.
        dict(name="attend-1x16k-prompt", op="attend", dtype="bf16", seqs=1, lo=12288, hi=12288,
             new_lo=4096, new_hi=4096, heads=8, group=8, dim=128, sub=4, centres=256, page=64,
             **score),
        # The decode step's weights, added up for eviction.
        dict(name="weigh-32x4096", op="weigh", dtype="bf16", seqs=32, lo=512, hi=4096, new_lo=1,
             new_hi=1, heads=8, group=4, dim=128, sub=4, centres=256, page=16, **score),
        # What the last tokens of long prompts look at.
        dict(name="weigh-4x8000-last", op="weigh", dtype="fp16", seqs=4, lo=5000, hi=8000, new_lo=33,
             new_hi=64, heads=8, group=8, dim=128, sub=4, centres=256, page=64,
             **{**score, "cap": 50.0}),
        # Short dialogues brought down to 300 positions.
        dict(name="evict-9x1000", op="evict", dtype="fp16", seqs=9, lo=50, hi=1000, heads=5, dim=96,
             sub=8, centres=200, page=16, keep=300, recent=32, first=4),
        # A batch of long contexts brought down to half.
        dict(name="evict-64x8192", op="evict", dtype="bf16", seqs=64, lo=5000, hi=8192, heads=8,
             dim=128, sub=4, centres=256, page=64, keep=4096, recent=128, first=4),
    ]


def _between(rng, lo, hi):
    """A whole number of lo..hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotate", "attend", "attend", "attend", "weigh", "evict"))
    case = dict(op=op, dtype=rng.choice(("bf16", "fp16")), heads=rng.randint(1, 8),
                dim=rng.choice((64, 96, 128)))
    if op == "rotate":
        case["group"] = rng.choice((1, 2, 4, 5, 8))
        case["tokens"] = _between(rng, 1, 8192)
        case["rot"] = rng.choice((case["dim"], case["dim"], case["dim"] // 2,
                                  2 * rng.randint(1, case["dim"] // 2)))
        case["interleaved"] = rng.choice((False, True))
        case["inverse"] = rng.choice((False, False, True))
        case["stretch"] = rng.choice((1.0, 1.0, 8.0))
        case["amplitude"] = rng.choice((1.0, 1.0, 1.2))
        return case
    case.update(sub=rng.choice((2, 4, 4, 8)), centres=rng.choice((256, 256, _between(rng, 16, 256))),
                page=rng.choice((16, 32, 64)))
    if op == "evict":
        case["seqs"] = _between(rng, 1, 64)
        case["hi"] = _between(rng, 1, min(65536, 32 * 8192 // case["seqs"]))
        case["lo"] = rng.randint(0, case["hi"])
        case["keep"] = _between(rng, 1, case["hi"])
        case["recent"] = rng.randint(0, case["keep"])
        case["first"] = rng.randint(0, min(4, case["keep"] - case["recent"]))
        return case
    case["group"] = rng.choice((1, 2, 4, 5, 8))
    # decode steps, verifications, and pieces of prompts
    case["new_hi"] = rng.choice((1, rng.randint(2, 8), _between(rng, 9, 2048)))
    case["new_lo"] = rng.randint(1, case["new_hi"])
    most = 1 << 26                                       # new tokens times positions
    case["seqs"] = _between(rng, 1, 64 if case["new_hi"] < 9 else 8)
    room = min(65536, most // (4 * case["seqs"] * case["new_hi"]))
    case["hi"] = _between(rng, 1, max(1, room))
    case["lo"] = rng.randint(0, case["hi"])
    case["cap"] = rng.choice((0.0, 0.0, 20.0, 50.0))
    case["slopes"] = rng.choice((False, False, True))
    case["window"] = rng.choice((0, 0, _between(rng, 1, case["hi"])))
    case["prefix"] = rng.choice((0, 0, _between(rng, 1, case["hi"])))
    case["docs"] = rng.choice((0, 0, _between(rng, 1, case["hi"])))
    return case


def _spaced(lo, hi, n):
    """n whole numbers from lo to hi, spaced on their logarithm."""
    if n == 1:
        return [hi]
    a = max(lo, 1)
    got = [int(round(a * (max(hi, a) / a) ** (i / (n - 1)))) for i in range(n)]
    return [0 if hi == 0 else min(x, hi) for x in ([0] if lo == 0 else got[:1]) + got[1:]]


def _sizes(case, seed):
    """Cached positions before, and new tokens, of every sequence (in an order that
    the seed gives)."""
    g = torch.Generator()
    g.manual_seed(seed)
    n = case["seqs"]
    cached = torch.tensor(_spaced(case["lo"], case["hi"], n))[torch.randperm(n, generator=g)]
    if case["op"] == "evict":
        return cached, torch.zeros_like(cached)
    new = torch.tensor(_spaced(case["new_lo"], case["new_hi"], n))[torch.randperm(n, generator=g)]
    return cached, new


def _frequencies(case):
    half = case["rot"] // 2
    return 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half) / case["stretch"]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    H, D = case["heads"], case["dim"]

    def rand(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    if case["op"] == "rotate":
        T, Hq = case["tokens"], H * case["group"]
        # tokens of several sequences, some far into a long context
        start = torch.randint(0, 1 << 20, (1,), generator=g, device=dev)
        return dict(case=case, q=rand(T, Hq, D).to(dt), k=rand(T, H, D).to(dt),
                    positions=start + torch.randperm(T, generator=g, device=dev),
                    frequencies=_frequencies(case).to(dev))
    sub, K, page = case["sub"], case["centres"], case["page"]
    S, B = D // sub, case["seqs"]
    # channels of unlike spread, as keys and values have them
    spread = torch.exp(0.4 * rand(2, H, 1, D))
    books = [(rand(H, K, D) * spread[i]).view(H, K, S, sub).transpose(1, 2).contiguous().to(dt)
             for i in (0, 1)]
    cached, new = _sizes(case, seed)
    lengths = cached + new
    most = max(1, int(lengths.max()))
    width = -(-most // page)
    need = (lengths + page - 1) // page

    def table(need, rows, at, perm):
        first = torch.cumsum(need, 0) - need
        col = torch.arange(rows, device=dev)
        where = (at + first[:, None] + col).clamp(max=perm.numel() - 1)
        # entries past a sequence's end are not pages
        return torch.where(col < need[:, None], perm[where], -1).to(torch.int32)

    used = int(need.sum())
    goal = torch.clamp(lengths, max=case["keep"]) if case["op"] == "evict" else lengths * 0
    fresh = (goal + page - 1) // page
    pages = used + int(fresh.sum()) + 3
    perm = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    s = dict(case=case, k_centres=books[0], v_centres=books[1],
             lengths=lengths.to(dev).to(torch.int32), table=table(need.to(dev), width, 0, perm))
    s["k_codes"] = torch.randint(0, K, (pages, H, page, S), generator=g, device=dev,
                                 dtype=torch.uint8)
    s["v_codes"] = torch.randint(0, K, (pages, H, S, page), generator=g, device=dev,
                                 dtype=torch.uint8)
    if case["op"] == "evict":
        s["to"] = table(fresh.to(dev), max(1, -(-int(goal.max()) // page)), used, perm)
        # summed attention weights: a few large, many small, of them many alike
        w = torch.exp(3.0 * rand(B, H, width * page) - 6.0)
        s["weights"] = torch.where(w < 1e-3, 2.0 ** -11, w)
    else:
        T, G = int(new.sum()), case["group"]
        bounds = torch.zeros(B + 1, dtype=torch.int32)
        bounds[1:] = torch.cumsum(new, 0)
        seq = torch.repeat_interleave(torch.arange(B), new)
        pos = cached[seq] + torch.arange(T) - bounds[seq]
        s["bounds"] = bounds.to(dev)
        # queries that prefer some keys to others
        s["q"] = (2.0 * rand(T, H * G, D)).to(dt)
        s["scale"] = 1.0 / math.sqrt(D)
        s["slopes"] = s["prefixes"] = s["starts"] = None
        if case["slopes"]:
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H * G + 1, device=dev) / (H * G))
        if case["prefix"]:
            s["prefixes"] = torch.full((B,), case["prefix"], dtype=torch.int32, device=dev)
        if case["docs"]:
            starts = pos // case["docs"] * case["docs"]
            starts = torch.where(torch.arange(T) % 17 == 16, lengths[seq], starts)
            s["starts"] = starts.to(dev).to(torch.int32)
        if case["op"] == "weigh":
            s["lse"] = _plain_attend(s)[1]
    if own:
        import paper_1402_3788_amd as km
        s["cache"] = km.KVCodes(s["k_centres"], s["v_centres"], s["k_codes"], s["v_codes"])
    return s


def _plain_rotate(s):
    case = s["case"]
    half = case["rot"] // 2
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos = (case["amplitude"] * torch.cos(angle)).float()[:, None]
    sin = (case["amplitude"] * torch.sin(angle)).float()[:, None]
    if case["inverse"]:
        sin = -sin

    def turned(x):
        y = x.float()
        if case["interleaved"]:
            at = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
        else:
            at = slice(0, half), slice(half, 2 * half)
        a, b = y[..., at[0]], y[..., at[1]]
        out = y.clone()
        out[..., at[0]] = a * cos - b * sin
        out[..., at[1]] = a * sin + b * cos
        return out.to(x.dtype)

    return turned(s["q"]), turned(s["k"])


def _values(codes, centres):
    """codes [..., H, n, S] -> the centres' values, [..., H, n, dim]."""
    H, S, K, sub = centres.shape
    base = (torch.arange(H, device=codes.device)[:, None, None] * S
            + torch.arange(S, device=codes.device)) * K
    return centres.view(H * S * K, sub)[base + codes].flatten(-2)


def _rows(s):
    """The new tokens in rows of each sequence: their numbers [B, n] (past a
    sequence's last: some token), which are there, their positions, and the bounds of
    what each sees."""
    case = s["case"]
    n, T = case["new_hi"], s["q"].shape[0]
    row = torch.arange(n, device=s["q"].device)
    count = s["bounds"].diff()
    there = row < count[:, None]
    token = (s["bounds"][:-1, None] + row).clamp(max=T - 1).long()
    pos = (s["lengths"] - count)[:, None] + row
    low = s["starts"][token].clamp(min=0) if s["starts"] is not None else torch.zeros_like(pos)
    if case["window"]:
        low = torch.maximum(low, pos - case["window"] + 1)
    high = pos + 1
    if s["prefixes"] is not None:
        high = torch.maximum(high, s["prefixes"][:, None])
    return token, there, pos, low, torch.minimum(high, s["lengths"][:, None])


def _plain_scores(s):
    """[B, H, n, G, positions] fp32, -inf where a token does not see a position, and
    the rows they stand for."""
    case = s["case"]
    H, G, D = case["heads"], case["group"], case["dim"]
    B, L = s["table"].shape[0], s["table"].shape[1] * case["page"]
    token, there, pos, low, high = _rows(s)
    pages = s["table"].clamp(min=0).long()
    kc = s["k_codes"][pages].transpose(1, 2).reshape(B, H, L, -1)
    k = _values(kc, s["k_centres"]).float()
    n = token.shape[1]
    q = s["q"].float()[token].view(B, n, H, G, D).transpose(1, 2).reshape(B, H, n * G, D)
    z = torch.matmul(q, k.transpose(2, 3)).view(B, H, n, G, L)
    z *= s["scale"]
    if case["cap"]:
        z = torch.tanh(z / case["cap"]) * case["cap"]
    i = torch.arange(L, device=z.device)
    if s["slopes"] is not None:
        far = (pos[..., None] - i).abs().float()
        z -= s["slopes"].view(H, 1, G, 1) * far[:, None, :, None]
    seen = (i >= low[..., None]) & (i < high[..., None]) & there[..., None]
    return z.masked_fill_(~seen[:, None, :, None], -math.inf), token, there


def _plain_attend(s):
    case = s["case"]
    H, G, D = case["heads"], case["group"], case["dim"]
    z, token, there = _plain_scores(s)
    B, L, n = z.shape[0], z.shape[-1], token.shape[1]
    pages = s["table"].clamp(min=0).long()
    vc = s["v_codes"][pages].permute(0, 2, 1, 4, 3).reshape(B, H, L, -1)
    v = _values(vc, s["v_centres"]).float()
    top = z.amax(-1, keepdim=True)
    z -= torch.where(top == -math.inf, 0.0, top)
    e = z.exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, H, n * G, L), v).view(B, H, n, G, D)
    o = o / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1)
    # rows of sequences back to the tokens' order
    o = o.permute(0, 2, 1, 3, 4).reshape(B, n, H * G, D)[there]
    return o.to(s["q"].dtype), lse.permute(0, 2, 1, 3).reshape(B, n, H * G)[there]


def _plain_weigh(s):
    case = s["case"]
    z, token, there = _plain_scores(s)
    lse = s["lse"][token].view(*token.shape, case["heads"], case["group"]).transpose(1, 2)
    z -= torch.where(lse == -math.inf, 0.0, lse)[..., None]
    return z.exp_().sum((2, 3))


def _plain_evict(s):
    case = s["case"]
    w, page, keep = s["weights"], case["page"], case["keep"]
    B, H, W = w.shape
    i = torch.arange(W, device=w.device)
    n = s["lengths"][:, None, None]
    always = (i < case["first"]) | (i >= n - case["recent"])
    order = torch.where(always, math.inf, w)
    order = torch.where(i < n, order, -math.inf)
    order = torch.sort(order, dim=-1, descending=True, stable=True).indices[..., :keep]
    j = torch.arange(order.shape[-1], device=w.device)
    left = s["lengths"].clamp(max=keep)
    here = (j < left[:, None]).unsqueeze(1).expand(B, H, -1)
    order = torch.where(here, order, W).sort(-1).values
    weights = torch.zeros_like(w)
    weights[..., :order.shape[-1]] = torch.where(here, w.gather(-1, order.clamp(max=W - 1)), 0.0)
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device=w.device)
    kept[..., :order.shape[-1]] = torch.where(here, order, -1)
    b, h, to = here.nonzero(as_tuple=True)
    at = order[b, h, to]
    p, q = s["table"][b, at // page].long(), s["to"][b, to // page].long()
    s["k_codes"][q, h, to % page] = s["k_codes"][p, h, at % page]
    s["v_codes"][q, h, :, to % page] = s["v_codes"][p, h, :, at % page]
    return kept, left, weights, s["k_codes"], s["v_codes"]


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"rotate": _plain_rotate, "attend": _plain_attend, "weigh": _plain_weigh,
                "evict": _plain_evict}[op](state)
    import paper_1402_3788_amd as km
    if op == "rotate":
        return km.kmeans_kv_rotate(state["q"], state["k"], state["positions"],
                                   state["frequencies"], interleaved=case["interleaved"],
                                   inverse=case["inverse"], amplitude=case["amplitude"])
    cache = state["cache"]
    if op == "evict":
        kept, left, weights = km.kmeans_kv_evict(cache, state["weights"], state["table"],
                                                 state["lengths"], case["keep"],
                                                 recent=case["recent"], first=case["first"],
                                                 to=state["to"])
        return kept, left, weights, cache.k_codes, cache.v_codes
    more = dict(scale=state["scale"], cap=case["cap"], slopes=state["slopes"],
                window=case["window"], prefixes=state["prefixes"], starts=state["starts"])
    if op == "weigh":
        return km.kmeans_kv_weigh(cache, state["q"], state["lse"], state["bounds"], state["table"],
                                  state["lengths"], **more)
    return km.kmeans_kv_attend_tokens(cache, state["q"], state["bounds"], state["table"],
                                      state["lengths"], **more)


def _pairs(case):
    """Pairs of a token and a position that it sees, and positions that any sees."""
    pairs = some = 0
    cached, new = _sizes(case, 0)
    token = 0
    for c, n in zip(cached.tolist(), new.tolist()):
        pos = c + torch.arange(n)
        low = torch.zeros(n, dtype=torch.long)
        if case["docs"]:
            pad = (token + torch.arange(n)) % 17 == 16
            low = torch.where(pad, c + n, pos // case["docs"] * case["docs"])
        token += n
        if case["window"]:
            low = torch.maximum(low, pos - case["window"] + 1)
        high = torch.clamp(pos + 1, min=case["prefix"]).clamp(max=c + n)
        wide = (high - low).clamp(min=0)
        pairs += int(wide.sum())
        if int(wide.max()):
            some += int(high[wide > 0].max() - low[wide > 0].min())
    return pairs, some


def work(case):
    H, D = case["heads"], case["dim"]
    if case["op"] == "rotate":
        T, Hq = case["tokens"], H * case["group"]
        return {"bytes": T * ((Hq + H) * D * 4 + 8) + 4 * case["rot"],
                "flops": 3 * T * (Hq + H) * case["rot"]}
    S, B, page = D // case["sub"], case["seqs"], case["page"]
    cached, new = _sizes(case, 0)
    lengths = cached + new
    width = -(-max(1, int(lengths.max())) // page)
    table = 4 * int(((lengths + page - 1) // page).sum())
    if case["op"] == "evict":
        left = int(lengths.clamp(max=case["keep"]).sum())
        # weights of all positions, codes of the kept ones from and to the cache
        return {"bytes": 4 * H * int(lengths.sum()) + 4 * H * B * (width * page + case["keep"])
                + 4 * S * H * left + table + 8 * B, "flops": 0}
    T, Hq = int(new.sum()), H * case["group"]
    pairs, some = _pairs(case)
    book = 2 * H * D * case["centres"]
    rows = T * Hq * (2 * D + 4) + table + 8 * B
    if case["op"] == "weigh":
        return {"bytes": S * H * some + book + rows + 4 * B * H * width * page,
                "flops": 2 * D * Hq * pairs}
    return {"bytes": 2 * (S * H * some + book) + rows + 2 * D * T * Hq,
            "flops": 4 * D * Hq * pairs}


def _exact_rotate(s, case):
    half = case["rot"] // 2
    angle = torch.outer(s["positions"].double(), s["frequencies"].double())
    turn = torch.polar(torch.full_like(angle, case["amplitude"]),
                       -angle if case["inverse"] else angle)[:, None]
    out = []
    for x in (s["q"].double(), s["k"].double()):
        part = x[..., :2 * half]
        part = part.unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        part = part if case["interleaved"] else part.transpose(-1, -2)
        part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
        part = part if case["interleaved"] else part.transpose(-1, -2)
        out.append(torch.cat((part.flatten(-2), x[..., 2 * half:]), -1))
    return tuple(out)


def _exact_evict(s, case):
    """By sequence and head, on the host, by sorting tuples."""
    w, table, to = s["weights"].cpu(), s["table"].cpu(), s["to"].cpu()
    page, keep = case["page"], case["keep"]
    kc, vc = s["k_codes"].cpu(), s["v_codes"].cpu()
    B, H, W = w.shape
    kept = torch.full((B, H, keep), -1, dtype=torch.int32)
    weights = torch.zeros_like(w)
    left = []
    for b, n in enumerate(s["lengths"].tolist()):
        m = min(n, keep)
        left.append(m)
        for h in range(H):
            sure = set(range(min(case["first"], n))) | set(range(max(0, n - case["recent"]), n))
            if n <= keep:
                got = list(range(n))
            else:
                x = w[b, h, :n].tolist()
                rest = sorted((i for i in range(n) if i not in sure), key=lambda i: (-x[i], i))
                got = sorted(sure | set(rest[:keep - len(sure)]))
            at, j = torch.tensor(got, dtype=torch.long), torch.arange(m)
            kept[b, h, :m] = at
            weights[b, h, :m] = w[b, h, at]
            p, q = table[b, at // page].long(), to[b, j // page].long()
            kc[q, h, j % page], vc[q, h, :, j % page] = kc[p, h, at % page], vc[p, h, :, at % page]
    return kept, torch.tensor(left, dtype=torch.int32), weights.double(), kc, vc


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return _exact_rotate(s, case)
    if case["op"] == "evict":
        # the sorts of a long batch take the host longer than is wanted
        return _exact_evict(s, case) if case["seqs"] * case["hi"] * case["heads"] < 1 << 20 else None
    dev = s["q"].device
    H, G, D, page = case["heads"], case["group"], case["dim"], case["page"]
    kb, vb = s["k_centres"].double(), s["v_centres"].double()
    S = D // case["sub"]
    ss = torch.arange(S, device=dev)
    B, W = s["table"].shape[0], s["table"].shape[1] * page
    T = s["q"].shape[0]
    out = torch.zeros(T, H * G, D, dtype=torch.float64, device=dev)
    lse = torch.full((T, H * G), -math.inf, dtype=torch.float64, device=dev)
    weights = torch.zeros(B, H, W, dtype=torch.float64, device=dev)
    bounds, lengths = s["bounds"].tolist(), s["lengths"].tolist()
    for b in range(B):
        t0, t1, n = bounds[b], bounds[b + 1], lengths[b]
        i = torch.arange(n, device=dev)
        p, off = s["table"][b][i // page].long(), i % page
        pos = n - (t1 - t0) + torch.arange(t1 - t0, device=dev)[:, None]
        seen = i <= pos
        if case["window"]:
            seen &= i > pos - case["window"]
        if case["prefix"]:
            ahead = i < case["prefix"]
            if case["window"]:
                ahead = ahead & (i > pos - case["window"])
            seen |= ahead
        if s["starts"] is not None:
            seen &= i >= s["starts"][t0:t1, None]
        for h in range(H):
            k = kb[h, ss, s["k_codes"][p, h, off].long()].reshape(n, D)
            v = vb[h, ss, s["v_codes"][p, h, :, off].long()].reshape(n, D)
            for hq in range(h * G, (h + 1) * G):
                z = (s["q"][t0:t1, hq].double() @ k.T) * s["scale"]
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][hq].double() * (pos - i).abs()
                z = z.masked_fill(~seen, -math.inf)
                if case["op"] == "weigh":
                    x = s["lse"][t0:t1, hq, None].double()
                    weights[b, h, :n] += torch.exp(z - torch.where(x == -math.inf, 0.0, x)).sum(0)
                    continue
                total = torch.logsumexp(z, -1)
                lse[t0:t1, hq] = total
                w = torch.exp(z - torch.where(total == -math.inf, 0.0, total)[:, None])
                out[t0:t1, hq] = w @ v
    return weights if case["op"] == "weigh" else (out, lse)
