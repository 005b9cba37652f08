"""The key-value cache in K-means codes, as measurable cases.

A head's vector of `dim` features is held as dim/sub codes of one byte, each the
number of the centre nearest to a sub-vector of `sub` features (Eq. (2), ties to
the lowest number); the centres are what kmeans_run learned, rounded to the
model's 16-bit type. Keys are [pages][heads][page][dim/sub] codes, values
[pages][heads][dim/sub][page]. A case is a dict of plain values:

    op      "store" (new tokens are encoded into the cache and read back as the
            values that the codes stand for), "read" (cached tokens are read
            back), "attend" (one new token of every sequence attends over the
            cache)
    dtype   "bf16" or "fp16"
    heads   key-value heads; group: query heads of each ("attend")
    dim, sub, centres, page   as above; page tokens to a page
    tokens  of "store" and "read"
    seqs, lo, hi, window      of "attend": sequences with lengths spaced from lo
            to hi (on their logarithm; lo 0: the first is empty), of which the
            last `window` positions are attended (0: all)
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One token of one sequence enters the cache: latency.
        dict(name="store-1", op="store", dtype="bf16", tokens=1, heads=8, dim=128, sub=4,
             centres=256, page=16),
        # A decode step of 100 sequences, four bits a feature.
        dict(name="store-100-fp16", op="store", dtype="fp16", tokens=100, heads=4, dim=64, sub=2,
             centres=256, page=32),
        # A ragged piece of a prompt, one bit a feature and an odd code book.
        dict(name="store-1021-k200", op="store", dtype="fp16", tokens=1021, heads=5, dim=96, sub=8,
             centres=200, page=16),
        # A prompt of 4096 tokens.
        dict(name="store-4096", op="store", dtype="bf16", tokens=4096, heads=8, dim=128, sub=4,
             centres=256, page=64),
        # A short context read back.
        dict(name="read-333", op="read", dtype="fp16", tokens=333, heads=5, dim=96, sub=4,
             centres=256, page=16),
        # A long context read back, as for a layer that needs whole keys.
        dict(name="read-64k", op="read", dtype="bf16", tokens=65536, heads=8, dim=128, sub=4,
             centres=256, page=64),
        # One sequence that has just begun: latency.
        dict(name="attend-1x77", op="attend", dtype="bf16", seqs=1, lo=77, hi=77, window=0,
             heads=8, group=4, dim=128, sub=4, centres=256, page=16),
        # Many short dialogues of uneven lengths, every head with its own keys,
        # the last 400 positions of each.
        dict(name="attend-100x1000-mha", op="attend", dtype="fp16", seqs=100, lo=0, hi=1000,
             window=400, heads=12, group=1, dim=64, sub=2, centres=256, page=32),
        # A serving batch.
        dict(name="attend-32x4096", op="attend", dtype="bf16", seqs=32, lo=512, hi=4096, window=0,
             heads=8, group=4, dim=128, sub=4, centres=256, page=16),
        # One key head for 16 query heads, one bit a feature, an odd code book.
        dict(name="attend-17x8191-mqa", op="attend", dtype="bf16", seqs=17, lo=100, hi=8191,
             window=0, heads=1, group=16, dim=96, sub=8, centres=200, page=64),
        # One document of 131072 positions: the length is split or the card is idle.
        dict(name="attend-1x128k", op="attend", dtype="bf16", seqs=1, lo=131072, hi=131072,
             window=0, heads=8, group=8, dim=128, sub=4, centres=256, page=64),
        # The largest batch of long contexts.
        dict(name="attend-64x16k", op="attend", dtype="bf16", seqs=64, lo=8192, hi=16384,
             window=0, heads=8, group=8, dim=128, sub=4, centres=256, page=64),
    ]


def _between(rng, lo, hi):
    """A whole number of lo..hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("store", "read", "attend", "attend"))
    case = dict(op=op, dtype=rng.choice(("bf16", "fp16")), heads=rng.randint(1, 8),
                dim=rng.choice((64, 96, 128)), sub=rng.choice((2, 4, 4, 8)),
                centres=rng.choice((256, 256, _between(rng, 16, 256))),
                page=rng.choice((16, 32, 64)))
    if op == "attend":
        case["seqs"] = _between(rng, 1, 128)
        case["hi"] = _between(rng, 1, min(131072, 20 * 16384 // case["seqs"]))
        case["lo"] = rng.randint(0, case["hi"])
        case["window"] = rng.choice((0, 0, _between(rng, 1, case["hi"])))
        case["group"] = rng.choice((1, 2, 4, 5, 7, 8))
    else:
        case["tokens"] = _between(rng, 1, 4096 if op == "store" else 65536)
    return case


def _lengths(case):
    """The lengths of an "attend" case, ascending."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    if n == 1:
        return [hi]
    a = max(lo, 1)
    got = [int(round(a * (hi / a) ** (i / (n - 1)))) for i in range(n)]
    return ([0] if lo == 0 else got[:1]) + got[1:]


def _starts(case, lengths):
    w = case["window"]
    return [max(0, x - w) if w else 0 for x in lengths]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    H, D, sub, K, page = (case[k] for k in ("heads", "dim", "sub", "centres", "page"))
    S = D // sub
    # channels of unlike spread, as keys and values have them
    spread = torch.exp(0.4 * torch.randn(2, H, 1, D, generator=g, device=dev))

    def rows(kind, n):
        return torch.randn(H, n, D, generator=g, device=dev) * spread[kind]

    def centres(kind):
        return rows(kind, K).view(H, K, S, sub).transpose(1, 2).contiguous().to(dt)

    s = dict(case=case, k_centres=centres(0), v_centres=centres(1))
    if case["op"] == "attend":
        order = torch.randperm(case["seqs"], generator=g, device=dev)
        lengths = torch.tensor(_lengths(case), dtype=torch.int32, device=dev)
        starts = torch.tensor(_starts(case, _lengths(case)), dtype=torch.int32, device=dev)
        s["lengths"], s["starts"] = lengths[order], starts[order]
        need = (s["lengths"].long() + page - 1) // page
        width = max(1, -(-case["hi"] // page))
        used = sum(-(-x // page) for x in _lengths(case))
        pages = used + 3
        perm = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
        first = torch.cumsum(need, 0) - need
        col = torch.arange(width, device=dev)
        at = (first[:, None] + col).clamp(max=pages - 1)
        # entries past a sequence's end are not pages
        s["table"] = torch.where(col < need[:, None], perm[at], -1).to(torch.int32)
        # queries that prefer some keys to others
        q = 2.0 * torch.randn(case["seqs"], H * case["group"], D, generator=g, device=dev)
        s["q"] = q.to(dt)
        s["scale"] = 1.0 / math.sqrt(D)
    else:
        T = case["tokens"]
        pages = -(-T // page) + 3
        perm = torch.randperm(pages, generator=g, device=dev)
        pos = torch.arange(T, device=dev)
        s["slots"] = perm[pos // page] * page + pos % page
        if case["op"] == "store":
            s["k"], s["v"] = (rows(kind, T).transpose(0, 1).contiguous().to(dt)
                              for kind in (0, 1))
    s["k_codes"] = torch.randint(0, K, (pages, H, page, S), generator=g, device=dev,
                                 dtype=torch.uint8)
    s["v_codes"] = torch.randint(0, K, (pages, H, S, page), generator=g, device=dev,
                                 dtype=torch.uint8)
    if own:
        import paper_1402_3788_amd as km
        s["cache"] = km.KVCodes(s["k_centres"], s["v_centres"], s["k_codes"], s["v_codes"])
    return s


def _fold(x):
    """The sum over the last axis, neighbours first, every addition rounded."""
    return x[..., 0] if x.shape[-1] == 1 else _fold(x[..., 0::2] + x[..., 1::2])


def _nearest(x, centres):
    """x [T][H][D] -> the number of the nearest centre, [T][H][S] uint8."""
    H, S, K, sub = centres.shape
    diff = x.float().view(-1, H, S, 1, sub) - centres.float()
    return _fold(diff * diff).argmin(-1).to(torch.uint8)


def _values(codes, centres):
    """codes [..., H, n, S] -> the centres' values, [..., H, n, dim]."""
    H, S, K, sub = centres.shape
    base = (torch.arange(H, device=codes.device)[:, None, None] * S
            + torch.arange(S, device=codes.device)) * K
    return centres.view(H * S * K, sub)[base + codes].flatten(-2)


def _plain_read(s):
    page = s["case"]["page"]
    p, off = s["slots"] // page, s["slots"] % page
    k = _values(s["k_codes"][p, :, off, :].unsqueeze(2), s["k_centres"]).squeeze(2)
    v = _values(s["v_codes"][p, :, :, off].unsqueeze(2), s["v_centres"]).squeeze(2)
    return k, v


def _plain_store(s):
    page = s["case"]["page"]
    p, off = s["slots"] // page, s["slots"] % page
    s["k_codes"][p, :, off, :] = _nearest(s["k"], s["k_centres"])
    s["v_codes"][p, :, :, off] = _nearest(s["v"], s["v_centres"])
    return _plain_read(s)


def _plain_attend(s):
    B, Hq, D = s["q"].shape
    H, G, L = s["case"]["heads"], s["case"]["group"], s["table"].shape[1] * s["case"]["page"]
    pages = s["table"].clamp(min=0).long()
    kc = s["k_codes"][pages].transpose(1, 2).reshape(B, H, L, -1)
    vc = s["v_codes"][pages].permute(0, 2, 1, 4, 3).reshape(B, H, L, -1)
    k, v = _values(kc, s["k_centres"]).float(), _values(vc, s["v_centres"]).float()
    pos = torch.arange(L, device=pages.device)
    seen = (pos >= s["starts"][:, None]) & (pos < s["lengths"][:, None])
    z = torch.matmul(s["q"].float().view(B, H, G, D), k.transpose(2, 3)) * s["scale"]
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    lse = top + torch.log(total)
    return o.view(B, Hq, D).to(s["q"].dtype), lse.view(B, Hq)


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"store": _plain_store, "read": _plain_read, "attend": _plain_attend}[op](state)
    import paper_1402_3788_amd as km
    cache = state["cache"]
    if op == "attend":
        return km.kmeans_kv_attend(cache, state["q"], state["table"], state["lengths"],
                                   state["scale"], starts=state["starts"])
    if op == "store":
        km.kmeans_kv_write(cache, state["k"], state["v"], state["slots"])
    return km.kmeans_kv_read(cache, state["slots"])


def work(case):
    H, D, sub, K = (case[k] for k in ("heads", "dim", "sub", "centres"))
    S = D // sub
    books = 2 * H * D * K * 2
    if case["op"] == "attend":
        lengths = _lengths(case)
        n = sum(b - a for a, b in zip(_starts(case, lengths), lengths))
        Hq = H * case["group"]
        table = sum(-(-x // case["page"]) for x in lengths) * 4
        return {"bytes": 2 * S * H * n + books + table + case["seqs"] * (Hq * (4 * D + 4) + 8),
                "flops": 4 * D * Hq * n}
    T = case["tokens"]
    read = 2 * T * H * (S + 2 * D) + books + 8 * T
    if case["op"] == "read":
        return {"bytes": read, "flops": 0}
    # the codes just written need not be fetched again to be read back
    return {"bytes": read + 2 * T * H * 2 * D, "flops": 2 * T * H * D * K * 3}


def exact(case, seed):
    s = prepare(case, seed)
    kb, vb = s["k_centres"].double(), s["v_centres"].double()
    H, S, K, sub = kb.shape
    D, page = S * sub, case["page"]
    hh = torch.arange(H, device=kb.device).view(1, H, 1)
    ss = torch.arange(S, device=kb.device).view(1, 1, S)
    if case["op"] == "attend":
        G, out, lse = case["group"], [], []
        for b in range(case["seqs"]):
            a, n = int(s["starts"][b]), int(s["lengths"][b])
            if n <= a:
                out.append(torch.zeros(H * G, D, dtype=torch.float64, device=kb.device))
                lse.append(torch.full((H * G,), -math.inf, dtype=torch.float64, device=kb.device))
                continue
            pos = torch.arange(a, n, device=kb.device)
            p, off = s["table"][b][pos // page].long(), pos % page
            k = kb[hh, ss, s["k_codes"][p, :, off, :].long()].reshape(n - a, H, D)
            v = vb[hh, ss, s["v_codes"][p, :, :, off].long()].reshape(n - a, H, D)
            q = s["q"][b].double().view(H, G, D)
            z = torch.bmm(q, k.permute(1, 2, 0).contiguous()) * s["scale"]
            total = torch.logsumexp(z, -1)
            w = torch.exp(z - total[..., None])
            out.append(torch.bmm(w, v.permute(1, 0, 2).contiguous()).view(H * G, D))
            lse.append(total.view(H * G))
        return torch.stack(out), torch.stack(lse)
    got = []
    for name, book in (("k", kb), ("v", vb)):
        if case["op"] == "read":
            p, off = s["slots"] // page, s["slots"] % page
            codes = s["k_codes"][p, :, off, :] if name == "k" else s["v_codes"][p, :, :, off]
            got.append(book[hh, ss, codes.long()].reshape(-1, H, D))
            continue
        parts = []
        for x in s[name].split(128):
            e = x.double().view(-1, H, S, 1, sub) - book
            parts.append(book[hh, ss, (e * e).sum(-1).argmin(-1)].reshape(-1, H, D))
        got.append(torch.cat(parts))
    return tuple(got)
