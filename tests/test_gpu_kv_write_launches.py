"""Encoding with as many tokens as the launch of six workgroups to a compute unit
takes, several steps to each: the stated fp32 definition, bit for bit."""
import pytest
import torch

import paper_1402_3788_amd as km

pytestmark = pytest.mark.gpu


def nearest(x, centres):
    """The least of the distances, neighbours added first, every operation rounded;
    x [n, H, D], centres [H, S, K, sub] -> [n, H, S]."""
    H, S, K, sub = centres.shape
    got = []
    for part in x.float().split(32):
        e = part.view(-1, H, S, 1, sub) - centres.float()
        d = e * e
        while d.shape[-1] > 1:
            d = d[..., 0::2] + d[..., 1::2]
        got.append(d[..., 0].argmin(-1).to(torch.uint8))
    return torch.cat(got)


@pytest.mark.parametrize("heads,dim,sub,K,dtype,n", [
    (8, 128, 4, 256, torch.bfloat16, 1003), (8, 128, 4, 256, torch.bfloat16, 2500),
    (16, 64, 2, 256, torch.float16, 801), (12, 96, 8, 200, torch.float16, 2999),
    (4, 128, 2, 131, torch.bfloat16, 1111), (40, 64, 8, 256, torch.bfloat16, 1300),
])
def test_many_steps(heads, dim, sub, K, dtype, n):
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(n)
    steps, kinds = -(-n // 32), 2 * heads * (dim // sub // 4)
    assert steps * kinds > 12 * 256 and steps > -(-6 * 256 // kinds)
    page, pages = 64, -(-n // 64) + 1
    centres = [torch.randn(heads, dim // sub, K, sub, generator=g).to(dtype).to(dev)
               for _ in range(2)]
    cache = km.KVCodes.empty(*centres, pages, page)
    k, v = (torch.randn(n, heads, dim, generator=g).to(dtype).to(dev) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g)[:n].to(dev)
    km.kmeans_kv_write(cache, k, v, slots)
    p, off = slots // page, slots % page
    assert torch.equal(cache.k_codes[p, :, off], nearest(k, centres[0]))
    assert torch.equal(cache.v_codes[p, :, :, off], nearest(v, centres[1]))
    rest = torch.ones(pages * page, dtype=torch.bool, device=dev)
    rest[slots] = False
    rest = rest.nonzero()[:, 0]
    assert not cache.k_codes[rest // page, :, rest % page].any()
    assert not cache.v_codes[rest // page, :, :, rest % page].any()
