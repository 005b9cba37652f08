"""A key-value cache in K-means codes, from the sample tokens to the answers.

    python examples/kv_codes.py [--heads 2] [--group 4] [--dim 64] [--sub 4]
                                [--centres 256] [--prompt 700] [--steps 8]

1. The centres of every head and sub-vector are learned with kmeans_run on the
   keys and values of sample tokens.
2. Prompts of unlike lengths are encoded into the pages of a cache.
3. Each decode step writes one new token of every sequence and attends over all
   of its codes; the last tokens, kept as they are, could be attended to apart
   and joined by the returned logarithms of the sums.

Keys and values are synthetic: tokens of a few kinds, each head with channels of
unlike spread. Printed: bytes of the cache, how far values read back are from
those written, and how far the attention over codes is from attention over the
keys and values themselves and over those read back.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1402_3788_amd as km  # noqa: E402


def sample_tokens(n, heads, dim, gen, kinds):
    """[n, heads, dim]: tokens of a kind are near each other."""
    which = torch.randint(0, kinds.shape[0], (n,), generator=gen, device=kinds.device)
    noise = torch.randn(n, heads, dim, generator=gen, device=kinds.device)
    return kinds[which] + 0.25 * noise


def learn_centres(x, sub, K, gen, max_iter=15):
    """The centres of every head's sub-vectors, [heads, dim / sub, K, sub] fp32: one
    kmeans_run for each, from K of the tokens."""
    n, heads, dim = x.shape
    first = torch.randperm(n, generator=gen, device=x.device)[:K]
    ws = km.workspace(n, sub, K, x.device)
    out = torch.empty(heads, dim // sub, K, sub, device=x.device)
    for h in range(heads):
        for s in range(dim // sub):
            part = x[:, h, s * sub:(s + 1) * sub].float().contiguous()
            out[h, s] = km.kmeans_run(part, K, part[first], max_iter, ws=ws)[1]
    return out


def attention(q, k, v):
    """One new token over [n, heads, dim], in fp32."""
    heads = k.shape[1]
    k, v = (t.float().transpose(0, 1).contiguous() for t in (k, v))
    q = q.float().view(heads, -1, q.shape[-1])
    w = torch.softmax(torch.matmul(q, k.transpose(1, 2)) / math.sqrt(q.shape[-1]), -1)
    return torch.matmul(w, v).reshape(-1, q.shape[-1])


def relative(a, b):
    return ((a - b).norm() / b.norm()).item()


def run(heads=2, group=4, dim=64, sub=4, centres=256, prompt=700, steps=8, page=16, seed=0,
        dtype=torch.bfloat16, device="cuda:0"):
    dev = torch.device(device)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    spread = torch.exp(0.5 * torch.randn(2, 1, heads, dim, generator=gen, device=dev))
    kinds = [s * torch.randn(400, heads, dim, generator=gen, device=dev) for s in spread]

    sample = [sample_tokens(8192, heads, dim, gen, x) for x in kinds]
    books = [learn_centres(x, sub, centres, gen).to(dtype) for x in sample]

    lengths = [prompt, prompt // 3 + 1, 1]
    per_seq = [-(-(n + steps) // page) for n in lengths]
    pages = sum(per_seq)
    cache = km.KVCodes.empty(*books, pages, page)
    free = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    table = torch.full((len(lengths), max(per_seq)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(per_seq):
        table[b, :n] = free[at:at + n]
        at += n

    def slots(b, pos):
        return table[b, pos // page].long() * page + pos % page

    history = []
    for b, n in enumerate(lengths):
        k, v = (sample_tokens(n, heads, dim, gen, x).to(dtype) for x in kinds)
        km.kmeans_kv_write(cache, k, v, slots(b, torch.arange(n, device=dev)))
        history.append([k, v])

    n = torch.tensor(lengths, dtype=torch.int32, device=dev)
    seqs = torch.arange(len(lengths), device=dev)
    for _ in range(steps):
        k, v = (sample_tokens(len(lengths), heads, dim, gen, x).to(dtype) for x in kinds)
        pos = n.long()
        km.kmeans_kv_write(cache, k, v, table[seqs, pos // page].long() * page + pos % page)
        n += 1
        for b, h in enumerate(history):
            h[0], h[1] = torch.cat((h[0], k[b:b + 1])), torch.cat((h[1], v[b:b + 1]))
        q = torch.randn(len(lengths), heads * group, dim, generator=gen, device=dev).to(dtype)
        out, lse = km.kmeans_kv_attend(cache, q, table, n)

    got = dict(codes=cache.k_codes.numel() + cache.v_codes.numel(),
               plain=2 * 2 * pages * page * heads * dim, key=0.0, value=0.0, exact=0.0, same=0.0)
    for b, (k, v) in enumerate(history):
        kk, vv = km.kmeans_kv_read(cache, slots(b, torch.arange(k.shape[0], device=dev)))
        got["key"] = max(got["key"], relative(kk.float(), k.float()))
        got["value"] = max(got["value"], relative(vv.float(), v.float()))
        got["exact"] = max(got["exact"], relative(out[b].float(), attention(q[b], k, v)))
        got["same"] = max(got["same"], relative(out[b].float(), attention(q[b], kk, vv)))
    return got


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("heads", 2), ("group", 4), ("dim", 64), ("sub", 4), ("centres", 256),
                        ("prompt", 700), ("steps", 8)):
        p.add_argument("--" + name, type=int, default=value)
    got = run(**vars(p.parse_args()))
    print(f"cache: {got['codes']} bytes of codes, {got['plain']} as 16-bit keys and values")
    print(f"read back: keys off by {got['key']:.3f}, values by {got['value']:.3f} (relative)")
    print(f"attention: off by {got['exact']:.3f} from that over the keys and values themselves, "
          f"by {got['same']:.5f} from that over those read back")


if __name__ == "__main__":
    main()
