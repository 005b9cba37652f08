"""Attention over K-means codes: what the 16-bit parts of a weight leave of it.

A cache in which the scores are exact, half of the weights are exactly 1 and the
values' signs make the sum of weight times value nearly vanish: what the weights
lose stands alone in the output."""
import math

import numpy as np
import pytest
import torch

import paper_1402_3788_amd as km

BF, FP = torch.bfloat16, torch.float16
N_ONES = 161
LOSSY = np.exp(-np.arange(1, 256) / 256.0)       # the weights that 16 bits do not hold


def balance():
    """The value of the last position that weighs 1: with it, 160 of -1 and +1 for
    the others the sum is below half a step of 8 bits."""
    return float(torch.tensor(160.0 - LOSSY.sum()).to(BF))


def wanted():
    return (LOSSY.sum() - (N_ONES - 1) + balance()) / (LOSSY.sum() + N_ONES)


def bound():
    """A weight is off by at most 2^-17 of itself, rounded to nearest twice to 8
    bits: errors that do not lean to one side add up as their squares do, 6
    standard deviations of them (uniform ones, each over its whole range). Each
    exponential and its argument, of at most 1.45, to 2^-22; 13 tiles' sums, joined,
    to 2^-22 of what they add up; the output itself to 2^-8."""
    total = LOSSY.sum() + N_ONES
    off = 6 * 2.0 ** -17 / math.sqrt(3) * math.sqrt((LOSSY ** 2).sum())
    return (off + 2.0 ** -22 * LOSSY.sum() + 2.0 ** -22 * total) / total + 2.0 ** -8 * abs(wanted())


def cut(x):
    return (x.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)


def nearest(x):
    return torch.from_numpy(x).to(BF).float().numpy()


@pytest.mark.parametrize("part,inside", [(nearest, True), (cut, False)])
def test_the_bound_tells_rounding_from_cutting(part, inside):
    """Both ways of taking two bf16 parts of each weight, in 64 bits otherwise."""
    w = LOSSY.astype(np.float32)
    high = part(w)
    kept = high.astype(np.float64) + part(w - high)
    got = (kept.sum() - (N_ONES - 1) + balance()) / (LOSSY.sum() + N_ONES)
    assert (abs(got - wanted()) <= bound()) == inside


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("dim,sub", [(64, 2), (96, 8), (128, 4)])
@pytest.mark.parametrize("group", [1, 8, 9])
def test_weights_lean_to_no_side(group, dim, sub, dtype):
    dev = torch.device("cuda:0")
    n, page = N_ONES + 255, 16
    centres = [torch.zeros(1, dim // sub, 256, sub) for _ in range(2)]
    # keys: code j is -j / 256 along the query, exact in 8 bits; code 0 weighs 1
    centres[0][0, 0, :, 0] = -torch.arange(256) / 256.0
    # values: codes 0, 1, 2 are -1, +1 and what balances them
    centres[1][0, :, 0], centres[1][0, :, 1], centres[1][0, :, 2] = -1.0, 1.0, balance()
    cache = km.KVCodes.empty(*(c.to(dtype).to(dev) for c in centres), n // page, page)
    key = torch.cat((torch.zeros(N_ONES, dtype=torch.long), torch.arange(1, 256)))
    value = torch.cat((torch.zeros(N_ONES - 1, dtype=torch.long), torch.tensor([2]),
                       torch.ones(255, dtype=torch.long)))
    # in an order in which the sum stays small; a weight of 1 first, so that it is
    # the reference
    order = torch.randperm(n - 1, generator=torch.Generator().manual_seed(1)) + 1
    order = torch.cat((torch.zeros(1, dtype=torch.long), order))
    key, value = key[order].to(torch.uint8), value[order].to(torch.uint8)
    cache.k_codes[:, 0, :, 0] = key.view(-1, page).to(dev)
    cache.v_codes[:, 0] = value.view(-1, 1, page).expand(-1, dim // sub, page).to(dev)
    q = torch.zeros(1, group, dim, device=dev, dtype=dtype)
    q[:, :, 0] = 1.0
    table = torch.arange(n // page, dtype=torch.int32, device=dev)[None]
    out, lse = km.kmeans_kv_attend(cache, q, table,
                                   torch.tensor([n], dtype=torch.int32, device=dev), scale=1.0)
    assert (out.double() - wanted()).abs().max().item() <= bound()
    # the sum and the base-2 logarithm (of 8.3) to 2^-20, its rounding, the change of base
    assert (lse.double() - math.log(LOSSY.sum() + N_ONES)).abs().max().item() <= 2.0 ** -19
