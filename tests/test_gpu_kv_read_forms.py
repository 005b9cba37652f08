"""Reading back around the numbers of tokens at which centres are taken from LDS
instead of looked up in the L2: the same values from both."""
import pytest
import torch

import paper_1402_3788_amd as km

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,dim,sub,limit", [
    (8, 128, 2, 1024), (3, 96, 2, 2731), (2, 64, 2, 4096), (8, 128, 4, 1024), (5, 96, 4, 2185),
    (3, 64, 8, 10923), (16, 128, 8, 1024),
])
def test_either_side_of_the_limit(heads, dim, sub, limit, dtype):
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(limit)
    page, pages = 32, limit // 32 + 2
    S = dim // sub
    centres = [torch.randn(heads, S, 256, sub, generator=g).to(dtype).to(dev) for _ in range(2)]
    codes = [torch.randint(0, 256, s, generator=g, dtype=torch.uint8).to(dev)
             for s in ((pages, heads, page, S), (pages, heads, S, page))]
    cache = km.KVCodes(*centres, *codes)
    slots = torch.randperm(pages * page, generator=g).to(dev)
    h, s = torch.arange(heads, device=dev)[:, None], torch.arange(S, device=dev)
    for n in (limit // 2, limit - 1, limit, limit + 1):
        at = slots[:n]
        k, v = km.kmeans_kv_read(cache, at)
        kc, vc = codes[0][at // page, :, at % page], codes[1][at // page, :, :, at % page]
        for got, c, code in ((k, centres[0], kc), (v, centres[1], vc)):
            assert torch.equal(got, c[h, s, code.long()].reshape(n, heads, dim))
