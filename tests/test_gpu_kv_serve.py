"""Serving from the key-value cache on the GPU: turned queries and keys, attention of
many new tokens and summed weights within bounds derived from their roundings,
evicted positions and moved codes exactly."""
import math

import pytest
import torch
import torch.autograd.forward_ad

import paper_1402_3788_amd as km
from kv_serve_reference import (BF, DEV, FP, Call, attention, check_attention, evicted, make_cache,
                                weights_of)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- rotary positions

def turned(x, positions, frequencies, interleaved, inverse, amplitude):
    half = frequencies.shape[0]
    y = x.double().cpu().clone()
    w = positions.double().cpu()[:, None] * frequencies.cpu()
    c, s = amplitude * torch.cos(w)[:, None], amplitude * torch.sin(w)[:, None]
    s = -s if inverse else s
    at = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved
          else (slice(0, half), slice(half, 2 * half)))
    a, b = y[..., at[0]].clone(), y[..., at[1]].clone()
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    size = x.double().cpu().abs().clone()
    size[..., at[0]] = size[..., at[1]] = amplitude * (a.abs() + b.abs())
    return y, size


def near(got, want, size):
    """One rounding to 16 bits, and 2^-21 of the products for the fp32 before it
    (cosine, sine and amplitude, two products, one sum)."""
    half = torch.finfo(got.dtype).eps / 2
    off = (got.double().cpu() - want).abs()
    tiny = 2.0 ** -25 if got.dtype == FP else 0.0        # half a step of the least numbers
    assert (off <= half * want.abs() + 2.0 ** -21 * size * (1 + half) + tiny).all()


ROTATE = [
    # tokens, q heads, k heads, dim, half, interleaved, inverse, amplitude, dtype
    (1, 1, 1, 64, 32, False, False, 1.0, BF),
    (1, 32, 8, 128, 64, True, False, 1.0, FP),
    (37, 20, 5, 96, 24, True, True, 1.25, FP),
    (37, 20, 5, 96, 24, False, False, 0.5, BF),
    (5, 3, 1, 128, 1, False, True, 1.0, BF),
    (5, 3, 1, 128, 1, True, False, 1.0, FP),
    (9, 4, 0, 72, 33, False, False, 2.0, BF),
    (9, 4, 2, 72, 35, True, True, 1.0, BF),
    (3, 2, 2, 8, 4, False, False, 1.0, FP),
    (3, 70, 10, 512, 256, False, True, 1.0, BF),
    (3, 7, 10, 512, 256, True, False, 1.0, FP),
    (600, 8, 2, 64, 0, False, False, 3.0, BF),
    (1500, 5, 1, 64, 32, True, False, 1.0, BF),
    # halves that are no whole runs of 16 bytes, heads that fill no wave
    (33, 13, 3, 40, 19, False, False, 1.0, FP),
    (20, 9, 2, 512, 255, False, True, 1.0, BF),
    (20, 9, 2, 512, 251, True, False, 1.0, FP),
    (7, 70, 9, 96, 46, False, False, 1.5, BF),
    (2, 300, 8, 24, 12, False, False, 1.0, FP),
    (2, 300, 8, 24, 11, True, False, 1.0, BF),
    (3, 5, 5, 8, 3, False, False, 1.0, BF),
]


@pytest.mark.parametrize("T,hq,hk,dim,half,inter,inverse,amp,dtype", ROTATE)
@pytest.mark.parametrize("in_place", [False, True])
def test_rotate(T, hq, hk, dim, half, inter, inverse, amp, dtype, in_place):
    g = torch.Generator().manual_seed(T + dim)
    q = torch.randn(T, hq, dim, generator=g).to(dtype).to(DEV)
    k = torch.randn(T, hk, dim, generator=g).to(dtype).to(DEV) if hk else None
    pos = torch.randint(-5, 1 << 21, (T,), generator=g).to(DEV)
    f = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).to(DEV)
    want = [turned(x, pos, f, inter, inverse, amp) for x in (q, k) if x is not None]
    was = [x.clone() for x in (q, k) if x is not None]
    got = km.kmeans_kv_rotate(q, k, pos, f, interleaved=inter, inverse=inverse, amplitude=amp,
                              out=(q, k) if in_place else None)
    assert (got[0] is q) == in_place and (got[1] is None) == (k is None)
    for x, (y, size), old, src in zip(got, want, was, (q, k)):
        near(x, y, size)
        assert torch.equal(x[..., 2 * half:], old[..., 2 * half:])
        if not in_place:
            assert torch.equal(src, old)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("half", [3, 8, 12, 16])
def test_rotate_leaves_features_behind_as_they_are(half, inter):
    """Infinities and NaN there reach no feature that is turned, and stay themselves."""
    g = torch.Generator().manual_seed(half)
    q = torch.randn(5, 6, 64, generator=g).to(BF).to(DEV)
    pos = torch.arange(5).to(DEV)
    f = torch.rand(half, generator=g, dtype=torch.float64).to(DEV)
    want = km.kmeans_kv_rotate(q, None, pos, f, interleaved=inter)[0]
    q[..., 2 * half:] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0]).to(BF).to(
        DEV).repeat(16)[:64 - 2 * half]
    got = km.kmeans_kv_rotate(q, None, pos, f, interleaved=inter)[0]
    assert torch.equal(got[..., :2 * half], want[..., :2 * half])
    assert torch.equal(got[..., 2 * half:].view(torch.int16), q[..., 2 * half:].view(torch.int16))


def test_rotate_far_positions_and_gradient():
    """Positions past 2^31, and the inverse as the gradient: by the formula and by
    differences in 64 bits."""
    g = torch.Generator().manual_seed(1)
    q = torch.randn(4, 2, 64, generator=g).to(BF).to(DEV)
    pos = torch.tensor([2 ** 33 + 1, -2 ** 35, 2 ** 40 + 12345, 7], device=DEV)
    f = (2.0 ** -torch.arange(32, dtype=torch.float64)).to(DEV)
    got, _ = km.kmeans_kv_rotate(q, None, pos, f)
    near(got, *turned(q, pos, f, False, False, 1.0))
    grad = torch.randn(4, 2, 64, generator=g).to(BF).to(DEV)
    back, _ = km.kmeans_kv_rotate(grad, None, pos, f, inverse=True, amplitude=1.5)
    x = q.double().cpu().requires_grad_()
    w = pos.double().cpu()[:, None, None] * f.cpu()
    a, b = x[..., :32], x[..., 32:]
    y = 1.5 * torch.cat((a * torch.cos(w) - b * torch.sin(w), a * torch.sin(w) + b * torch.cos(w)), -1)
    y.backward(grad.double().cpu())
    _, size = turned(grad, pos, f, False, True, 1.5)
    near(back, x.grad, size)
    # linear in x: a difference of whole steps is exact in 64 bits but for rounding
    for at in ((0, 0, 3), (2, 1, 40)):
        e = torch.zeros_like(x)
        e[at] = 1.0
        plus, minus = (turned((q.double().cpu() + s * e), pos, f, False, False, 1.5)[0] for s in (1, -1))
        slope = ((plus - minus) / 2 * grad.double().cpu()).sum()
        assert abs(slope - x.grad[at]) <= 1e-9 * size[at]


def test_rotate_strides_and_others():
    g = torch.Generator().manual_seed(2)
    big = torch.randn(6, 24, 96, generator=g).to(FP).to(DEV)
    f = torch.rand(20, dtype=torch.float64, generator=g).to(DEV)
    pos = torch.arange(12, device=DEV)[::2]
    q, k = big[:, 3:11, :64], big.transpose(0, 1)[11:12].transpose(0, 1)[:, :, 24:88]
    want = [turned(x, pos, f, False, False, 1.0) for x in (q, k)]
    for x, y in zip(km.kmeans_kv_rotate(q, k, pos, f), want):
        near(x, *y)
    # heads between are untouched in place
    was = big.clone()
    km.kmeans_kv_rotate(q, k, pos, f, out=(q, k))
    for x, y in zip((q, k), want):
        near(x, *y)
    was[:, 3:11, :64], was[:, 11:12, 24:88] = q, k
    assert torch.equal(was, big)
    # features that are not contiguous are copied first
    odd = torch.randn(6, 64, 3, generator=g).to(FP).to(DEV).transpose(1, 2)
    got, none = km.kmeans_kv_rotate(odd, None, pos, f)
    near(got, *turned(odd, pos, f, False, False, 1.0))
    assert none is None
    # one token's row for many
    row = torch.randn(1, 2, 64, generator=g).to(FP).to(DEV).expand(6, 2, 64)
    near(km.kmeans_kv_rotate(row, None, pos, f)[0], *turned(row, pos, f, False, False, 1.0))
    empty = torch.empty(0, 2, 64, dtype=FP, device=DEV)
    assert km.kmeans_kv_rotate(empty, empty, pos[:0], f)[0].shape == (0, 2, 64)


# ------------------------------------------------------------- attention of many tokens

SIZES = [
    # one token of one sequence, one position
    ([(1, 1)], dict(dim=64, sub=2)),
    # single tokens of uneven sequences
    ([(77, 1), (1, 1), (300, 1), (0, 0), (129, 1)], dict(dim=128, sub=4, group=4, heads=3)),
    # a few tokens each, an odd code book, pages that end inside a tile
    ([(5, 5), (203, 5), (64, 3)], dict(dim=96, sub=8, K=200, dtype=FP, group=5, heads=1, page=8)),
    # prompts from their first token
    ([(97, 97), (1, 1), (260, 260)], dict(dim=64, sub=2, dtype=FP, group=1, heads=3, page=32)),
    # pieces of prompts, some without tokens
    ([(500, 120), (33, 0), (700, 1), (64, 64)], dict(dim=128, sub=4, group=8, heads=2, page=64)),
    ([(600, 70)], dict(dim=96, sub=4, group=3, heads=2, page=1024)),
    ([(130, 130), (257, 100)], dict(dim=64, sub=8, group=2, heads=1, page=16)),
    ([(300, 40)], dict(dim=128, sub=2, group=4, heads=1, K=31, dtype=FP)),
    ([(300, 40)], dict(dim=128, sub=8, group=16, heads=1)),
    ([(200, 3)], dict(dim=64, sub=4, group=128, heads=1)),
    ([(290, 33)], dict(dim=96, sub=2, group=1, heads=2)),
    # more new tokens than positions: the first see nothing
    ([(10, 40), (0, 5), (45, 40)], dict(dim=64, sub=4, group=2)),
]

MODES = ["plain", "cap", "slopes", "window", "prefix", "starts", "all"]


def set_mode(call, mode, seed=3):
    g = torch.Generator().manual_seed(seed)
    T, Hq = call.q.shape[:2]
    if mode in ("cap", "all"):
        call.more["cap"] = 3.0
    if mode in ("slopes", "all"):
        call.more["slopes"] = torch.linspace(-0.01, 0.3, Hq, device=DEV)
    if mode in ("window", "all"):
        call.more["window"] = 37
    if mode in ("prefix", "all"):
        call.more["prefixes"] = torch.tensor([(7 * b + 50) % 90 - 10 for b in range(len(call.sizes))],
                                             dtype=torch.int32, device=DEV)
    if mode in ("starts", "all"):
        # some past everything, some negative
        most = max(n for n, _ in call.sizes)
        call.more["starts"] = torch.randint(-3, max(most, 1) + 3, (T,), generator=g,
                                            dtype=torch.int32).to(DEV)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_attend_and_weigh(case, mode):
    sizes, kw = SIZES[case]
    call = Call(sizes, seed=case, **kw)
    set_mode(call, mode)
    _, lse = check_attention(call)
    positions = call.table.shape[1] * call.cache.page
    w, d = weights_of(call, lse, positions)
    got = call.weigh(lse)
    assert got.shape == w.shape
    assert ((got.double() - w).abs() <= d).all()
    # added to what is there, in rows of another length
    there = torch.rand(len(sizes), call.heads, positions + 5, device=DEV)
    want = there.double()
    want[..., :positions] += w
    again = call.weigh(lse, there)
    assert again is there
    bound = torch.zeros_like(want)
    bound[..., :positions] = d
    assert ((there.double() - want).abs() <= bound + 2.0 ** -23 * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_every_form(dim, sub, dtype):
    for sizes in ([(150, 1), (90, 2)], [(400, 90), (70, 70)]):
        call = Call(sizes, heads=2, group=4, dim=dim, sub=sub, dtype=dtype, seed=dim + sub)
        set_mode(call, "slopes")
        _, lse = check_attention(call)
        w, d = weights_of(call, lse, call.table.shape[1] * call.cache.page)
        assert ((call.weigh(lse).double() - w).abs() <= d).all()


# More rows than units of few are taken for.
MANY = [
    ([(400, 390), (330, 330), (0, 0), (70, 5), (3, 9)], dict(group=8, heads=1)),
    ([(1100, 1100)], dict(group=4, heads=2, page=64)),
    ([(290, 33)] + [(120 - b, 120 - b) for b in range(0, 110, 3)], dict(group=4, heads=3, page=8)),
    ([(500, 40), (77, 35)], dict(group=128, heads=1, page=1024)),
    ([(700, 300), (33, 0), (50, 60), (650, 300)], dict(group=8, heads=2, K=31)),
]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("case", range(len(MANY)))
def test_many_rows(case, mode):
    sizes, kw = MANY[case]
    dim, sub, dtype = [(64, 2, BF), (128, 4, FP), (96, 8, FP), (128, 8, BF), (96, 4, BF)][case]
    call = Call(sizes, dim=dim, sub=sub, dtype=dtype, seed=200 + case, **kw)
    set_mode(call, mode)
    out, lse = check_attention(call)
    again = call.attend()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sub", [2, 4, 8])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_every_form_of_many_rows(dim, sub, dtype):
    for page in (16, 32):
        call = Call([(520, 510), (90, 90)], heads=1, group=8, dim=dim, sub=sub, dtype=dtype, seed=dim + sub,
                    page=page)
        set_mode(call, "slopes")
        check_attention(call)


def test_long_context_of_many_rows():
    """Cut by many workgroups; captured, and replayed with other lengths and bounds."""
    call = Call([(3000, 600), (6000, 500)], heads=2, group=4, dim=64, page=64, seed=240)
    out, lse = check_attention(call)
    n = km.kmeans_kv_attend_tokens_workspace_bytes(call.cache, call.q.shape[0], 2, 8, call.table.shape[1])
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    o, l = torch.zeros_like(out), torch.zeros_like(lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call.attend(out=o, lse=l, ws=ws)
    for _ in range(3):
        ws.fill_(255)
        o.fill_(1.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse)
    call.lengths[0] = 700
    call.bounds[1] = 650
    ws.fill_(255)
    g.replay()
    check_attention(call, (o, l))


# Rows and positions that are shared out in other ways: to units of few and of many rows, to
# waves alone and to all of a workgroup.
SHARES = [
    ([(100, 41), (33, 20), (0, 0), (64, 64)], dict(dim=64, group=5, heads=1, page=8)),
    ([(70, 45), (40, 40)], dict(dim=64, sub=8, group=2, heads=128)),
    ([(50, 20)], dict(dim=64, sub=8, group=4, heads=300)),
    ([(40, 40)], dict(dim=128, group=8, heads=2)),
    ([(30, 9)], dict(dim=96, group=128, heads=1, sub=8, dtype=FP)),
    ([(300, 30)], dict(dim=128, group=4, heads=2)),
    ([(60 - b % 7, 25) for b in range(40)], dict(dim=64, group=4, heads=1)),
    ([(60 - b % 7, 16) for b in range(40)], dict(dim=64, group=4, heads=1)),
]


@pytest.mark.parametrize("mode", ["plain", "all"])
@pytest.mark.parametrize("case", range(len(SHARES)))
def test_shares(case, mode):
    sizes, kw = SHARES[case]
    call = Call(sizes, seed=100 + case, **kw)
    set_mode(call, mode)
    _, lse = check_attention(call)
    w, d = weights_of(call, lse, call.table.shape[1] * call.cache.page)
    got = call.weigh(lse)
    assert ((got.double() - w).abs() <= d).all()
    assert torch.equal(call.weigh(lse), got)


def test_long_contexts():
    """Contexts long enough to be shared by many workgroups, with few and many rows."""
    for sizes in ([(9000, 1), (20001, 1)], [(9000, 9)], [(12345, 200)], [(5000, 1), (6000, 150), (33, 33)]):
        call = Call(sizes, heads=2, group=4, dim=128, page=64, seed=len(sizes))
        _, lse = check_attention(call)
        w, d = weights_of(call, lse, call.table.shape[1] * call.cache.page)
        assert ((call.weigh(lse).double() - w).abs() <= d).all()


def test_many_sequences():
    sizes = [((37 * b) % 90 + (b % 3), b % 3) for b in range(1200)]
    call = Call(sizes, heads=1, group=2, dim=64, seed=5)
    _, lse = check_attention(call)
    w, d = weights_of(call, lse, call.table.shape[1] * call.cache.page)
    assert ((call.weigh(lse).double() - w).abs() <= d).all()


def test_one_token_equals_kv_attend():
    """The same positions through kmeans_kv_attend: both within their bounds of the
    definition, and their weights sum to the number of query heads."""
    call = Call([(200, 1), (1, 1), (77, 1)], heads=2, group=4, dim=128, seed=9)
    out, lse = check_attention(call)
    out1, lse1 = km.kmeans_kv_attend(call.cache, call.q, call.table, call.lengths)
    check_attention(call, (out1, lse1))
    for x in (lse, lse1):
        total = call.weigh(x).double().sum(-1)
        assert (total - call.group).abs().max() <= call.group * 1e-4


def test_tokens_outside_sequences_are_left():
    call = Call([(40, 7), (90, 20)], more_tokens=6, seed=4)
    call.bounds += 3                                     # three before, three behind
    out = torch.full_like(call.q, 7.0)
    lse = torch.full(call.q.shape[:2], 5.0, device=DEV)
    got = call.attend(out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    check_attention(call, got)
    for s in (slice(0, 3), slice(30, None)):
        assert (out[s] == 7).all() and (lse[s] == 5).all()
    # bounds past the tokens, and descending ones, are cut
    call.bounds[-1] = 1000
    check_attention(call)
    call.bounds[:] = torch.tensor([-5, 10, 4], dtype=torch.int32)
    call.lengths[0] = 30
    out, lse = call.attend()
    assert torch.isfinite(out[:10]).all()


def test_garbage_in_device_data():
    """Lengths and page numbers that nothing belongs to are never followed."""
    call = Call([(40, 7), (90, 20)], seed=4)
    call.lengths[:] = torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32)
    call.table[0, 1::2] = torch.tensor([2 ** 31 - 1], dtype=torch.int32)
    call.table[0, ::3] = -2 ** 31
    out, lse = call.attend()
    assert torch.isfinite(out).all() and (lse[7:] == -math.inf).all() and (out[7:] == 0).all()
    w = call.weigh(lse)
    assert torch.isfinite(w).all() and (w[1] == 0).all()


@pytest.mark.parametrize("seqs,new", [(40, 1), (64, 2), (200, 1), (30, 40), (300, 90)])
def test_bounds_that_descend(seqs, new):
    """Bounds that make more rows of the tokens than there are give undefined outputs and
    touch nothing else: the call's neighbours in memory stay, and so do later calls."""
    call = Call([(60, new)] * seqs, heads=1, group=4, dim=64, seed=7)
    T = call.q.shape[0]
    want, lse0 = call.attend()
    w0 = call.weigh(lse0)
    good = call.bounds.clone()
    n = km.kmeans_kv_attend_tokens_workspace_bytes(call.cache, T, seqs, 4, call.table.shape[1])
    room = torch.full((n + 4096,), 77, dtype=torch.uint8, device=DEV)
    out = torch.full((T + 8, 4, 64), 5.0, dtype=BF, device=DEV)
    for bad in (torch.arange(seqs + 1) % 2 * T, T - good.cpu(), good.cpu().roll(1)):
        call.bounds.copy_(bad)
        _, lse = call.attend(out=out[:T], ws=room[:n])
        assert (room[n:] == 77).all() and (out[T:] == 5).all()
        w = call.weigh(lse0)
        assert w.shape == w0.shape
    call.bounds.copy_(good)
    out, lse = call.attend()
    assert torch.equal(out, want) and torch.equal(lse, lse0) and torch.equal(call.weigh(lse0), w0)


def test_infinities_and_nan_in_what_is_not_seen():
    """NaN in the query of one token stays there, and the largest centres in positions
    that are not seen (scores of infinity) change nothing."""
    call = Call([(100, 4)], heads=1, group=2, dim=64, seed=6)
    starts = torch.tensor([10, 10, 10, 10], dtype=torch.int32, device=DEV)
    call.more["starts"] = starts
    # centre 255 is named by positions below 10 only
    call.cache.v_codes[call.cache.v_codes == 255] = 1
    call.cache.k_codes[call.cache.k_codes == 255] = 1
    want, lse0 = check_attention(call)
    w0 = call.weigh(lse0)
    p = call.table[0, 0].long()
    call.cache.v_codes[p, :, :, 3] = 255
    call.cache.k_codes[p, :, 3] = 255
    call.cache.v_centres[:, :, 255] = torch.finfo(BF).max
    call.cache.k_centres[:, :, 255] = torch.finfo(BF).max
    out, lse = call.attend()
    assert torch.equal(out, want) and torch.equal(lse, lse0) and torch.equal(call.weigh(lse0), w0)
    call.q[3] = math.nan
    out, lse = call.attend()
    assert torch.equal(out[:3], want[:3]) and torch.equal(lse[:3], lse0[:3])
    assert torch.isnan(out[3]).all() and torch.isnan(lse[3]).all()
    # a token whose every score is -infinity
    call = Call([(3, 1)], heads=1, group=1, dim=64, seed=6)
    call.cache.k_centres.fill_(1.0)
    call.q.fill_(-math.inf)
    out, lse = call.attend()
    assert (out == 0).all() and (lse == -math.inf).all()
    assert (call.weigh(lse) == 0).all()


def test_scales_and_caps():
    for more in (dict(scale=0.0), dict(scale=-0.3), dict(scale=30.0), dict(scale=30.0, cap=50.0),
                 dict(scale=-1.0, cap=0.01), dict(scale=1.0, cap=1e6)):
        call = Call([(60, 20), (300, 2)], heads=1, group=3, dim=64, seed=8)
        call.more.update(more)
        if more.get("cap") == 1e6:
            # tanh near 0 is off by a rounding of 1, times the cap: within the bound too
            check_attention(call)
            continue
        _, lse = check_attention(call)
        w, d = weights_of(call, lse, call.table.shape[1] * call.cache.page)
        assert ((call.weigh(lse).double() - w).abs() <= d).all()


def test_strides_streams_and_graphs():
    call = Call([(200, 30), (90, 1), (333, 40)], heads=2, group=2, dim=64, seed=11)
    set_mode(call, "all")
    want, lse = check_attention(call)
    wide = torch.zeros(call.q.shape[0], 9, 80, dtype=BF, device=DEV)
    wide[:, 2:6, 8:72] = call.q
    out = torch.full_like(wide, 3.0)
    q0, call.q = call.q, wide[:, 2:6, 8:72]
    call.attend(out=out[:, 4:8, 8:72], lse=torch.empty_like(lse))
    assert torch.equal(out[:, 4:8, 8:72], want)
    out[:, 4:8, 8:72] = 3.0
    assert (out == 3).all()
    # a table that is a slice of a larger one
    t0 = call.table
    big = torch.full((3, t0.shape[1] + 3), 2 ** 30, dtype=torch.int32, device=DEV)
    big[:, 2:-1] = t0
    call.table = big[:, 2:-1]
    assert torch.equal(call.attend()[0], want)
    call.table, call.q = t0, q0
    w0 = call.weigh(lse)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call.attend()[0]
        w = call.weigh(lse)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(w, w0)
    # two graphs that share a workspace
    n = km.kmeans_kv_attend_tokens_workspace_bytes(call.cache, call.q.shape[0], 3, 4, t0.shape[1])
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    graphs = []
    for _ in range(2):
        out, l = torch.zeros_like(want), torch.zeros_like(lse)
        w = torch.zeros_like(w0)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call.attend(out=out, lse=l, ws=ws)
            call.weigh(l, w)
        graphs.append((g, out, l, w))
    for turn in range(3):
        for g, out, l, w in graphs:
            out.fill_(1.0)
            l.fill_(1.0)
            w.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(l, lse) and torch.equal(w, w0)
        ws.fill_(255)
    # the lengths of a captured call may change between replays
    call.lengths[2] = 250
    graphs[0][0].replay()
    check_attention(call, graphs[0][1:3])


def test_same_bits():
    call = Call([(4000, 100), (3000, 1)], heads=2, group=4, dim=128, seed=12)
    out, lse = call.attend()
    w = call.weigh(lse)
    for _ in range(3):
        o, l = call.attend()
        assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(call.weigh(l), w)


def test_nothing_to_do():
    call = Call([(5, 0), (0, 0)], seed=1)
    out, lse = call.attend()
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    w = call.weigh(lse)
    assert w.shape == (2, 2, 16) and (w == 0).all()
    call = Call([(0, 3), (0, 2)], seed=1)
    call.table = call.table[:, :0]
    out, lse = call.attend()
    assert (out == 0).all() and (lse == -math.inf).all()
    assert call.weigh(lse).shape == (2, 2, 0)


# ------------------------------------------------------------------------ eviction

EVICT = [
    # lengths, keep, recent, first, positions of the weights beside the table's (None: those)
    ([1], 1, 0, 0, None), ([2], 1, 1, 0, None), ([2], 1, 0, 1, None), ([2], 1, 0, 0, None),
    ([300, 0, 17, 64], 40, 8, 4, None),
    ([300, 41, 40, 39], 40, 40, 0, None), ([300, 41], 40, 0, 40, None),
    ([1000, 3000, 2049], 1024, 100, 3, None),
    ([777, 500], 513, 0, 0, 600), ([777, 500], 100, 10, 10, 900),
    ([100, 90], 4000, 5, 5, None),
    ([20000, 5], 9001, 64, 4, None),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lengths,keep,recent,first,positions", EVICT)
def test_evict(lengths, keep, recent, first, positions, in_place):
    dims = [(64, 8, 8), (96, 8, 16), (64, 4, 16), (96, 4, 64), (128, 4, 64), (96, 2, 32), (128, 2, 1024)]
    for dim, sub, page in dims[keep % 2::2]:
        run_evict(lengths, keep, recent, first, positions, in_place, dim, sub, page)


def run_evict(lengths, keep, recent, first, positions, in_place, dim, sub, page, heads=3, kind="ties"):
    B = len(lengths)
    need = [-(-n // page) for n in lengths]
    fresh = [-(-min(n, keep) // page) for n in lengths]
    pages = sum(need) + sum(fresh) + 2
    cache = make_cache(heads, dim, sub, 256, BF, pages, page, seed=keep)
    g = torch.Generator().manual_seed(keep)
    perm = torch.randperm(pages, generator=g).to(torch.int32)
    width = max(need) or 1
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    to = torch.full((B, max(-(-min(keep, width * page) // page), 1)), -1, dtype=torch.int32)
    for b, n in enumerate(fresh):
        to[b, :n] = perm[at:at + n]
        at += n
    P = width * page if positions is None else positions
    w = torch.randint(0, 50, (B, heads, P), generator=g).float() * 0.25
    if kind == "odd":
        w[:, :, ::5] = -1.0
        w[:, :, 1::7] = math.nan
        w[:, :, 2::11] = math.inf
        w[:, :, 3::13] = -math.inf
        w[:, :, 4::17] = -0.0
        w[:, :, 5::17] = 0.0
    kept, left, ww = evicted(w, torch.tensor(lengths), keep, recent, first)
    kc, vc = cache.k_codes.cpu(), cache.v_codes.cpu()
    want_k, want_v = kc.clone(), vc.clone()
    goal = table if in_place else to
    for b, n in enumerate(left.tolist()):
        for h in range(heads):
            src, j = kept[b, h, :n].long(), torch.arange(n)
            p, q = table[b, src // page].long(), goal[b, j // page].long()
            want_k[q, h, j % page] = kc[p, h, src % page]
            want_v[q, h, :, j % page] = vc[p, h, :, src % page]
    dl, dw, dt = (torch.tensor(lengths, dtype=torch.int32, device=DEV), w.to(DEV), table.to(DEV))
    got = km.kmeans_kv_evict(cache, dw, dt, dl, keep, recent=recent, first=first,
                             to=None if in_place else to.to(DEV))
    assert (got[1] is dl) == in_place and (got[2] is dw) == in_place
    assert torch.equal(got[0].cpu(), kept) and torch.equal(got[1].cpu(), left)
    assert torch.equal(got[2].cpu().nan_to_num(-77.0), ww.nan_to_num(-77.0))
    assert torch.equal(cache.k_codes.cpu(), want_k) and torch.equal(cache.v_codes.cpu(), want_v)
    if not in_place:
        assert dl.tolist() == lengths and torch.equal(dw.cpu().nan_to_num(-77.0), w.nan_to_num(-77.0))


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_from_long_rows(in_place):
    """Rows beyond what a workgroup holds, beside short ones."""
    run_evict([70000, 9000, 100, 4097], 5000, 100, 4, None, in_place, 64, 8, 1024, heads=2)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_unusual_weights(in_place):
    run_evict([500, 300], 250, 20, 3, None, in_place, 64, 4, 16, kind="odd")
    run_evict([500, 300], 450, 0, 0, None, in_place, 64, 4, 16, kind="odd")


def test_evict_pages_that_are_none():
    """Entries outside the cache: nothing is written for those of `to`, some page is
    read for those of table."""
    cache = make_cache(2, 64, 4, 256, BF, 12, 16)
    table = torch.arange(4, dtype=torch.int32, device=DEV)[None]
    to = torch.tensor([[-1, 2 ** 31 - 1, 12]], dtype=torch.int32, device=DEV)
    w = torch.rand(1, 2, 64, device=DEV)
    n = torch.tensor([60], dtype=torch.int32, device=DEV)
    k, v = cache.k_codes.clone(), cache.v_codes.clone()
    kept, left, _ = km.kmeans_kv_evict(cache, w, table, n, 40, to=to)
    assert left.tolist() == [40] and (kept >= 0).all()
    assert torch.equal(k, cache.k_codes) and torch.equal(v, cache.v_codes)
    table[0, 2] = 2 ** 30
    km.kmeans_kv_evict(cache, w, table, n, 40, to=torch.tensor([[5, 6, 7]], dtype=torch.int32,
                                                             device=DEV))
    keep = [0, 1, 2, 3, 4, 8, 9, 10, 11]
    assert torch.equal(k[keep], cache.k_codes[keep]) and torch.equal(v[keep], cache.v_codes[keep])


def test_evict_in_a_graph():
    cache = make_cache(2, 64, 4, 256, BF, 12, 16)
    table = torch.arange(10, dtype=torch.int32, device=DEV)[None]
    k, v = cache.k_codes.clone(), cache.v_codes.clone()
    w0 = torch.rand(1, 2, 160, device=DEV)
    n = torch.tensor([150], dtype=torch.int32, device=DEV)
    w = w0.clone()
    want = km.kmeans_kv_evict(cache, w, table, n, 60, recent=10)
    kk, vv = cache.k_codes.clone(), cache.v_codes.clone()

    def again():
        cache.k_codes.copy_(k)
        cache.v_codes.copy_(v)
        n.fill_(150)
        w.copy_(w0)

    again()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = km.kmeans_kv_evict(cache, w, table, n, 60, recent=10)
    for _ in range(3):
        again()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and n.tolist() == [60]
        assert torch.equal(kk, cache.k_codes) and torch.equal(vv, cache.v_codes)


# ------------------------------------------------------------------ a run of them

def test_a_run_of_them():
    """Prompts and decode steps with rotary positions, weights summed, and evictions
    between: every call against the definition on the cache as it is."""
    heads, group, dim, page = 2, 4, 64, 16
    call = Call([(200, 200), (77, 77)], heads=heads, group=group, dim=dim, page=page, seed=20)
    cache, g = call.cache, torch.Generator().manual_seed(21)
    # 13 and 7 pages of its cache
    width, pages = 13, torch.randperm(call.pages, generator=g).to(torch.int32)
    call.table = torch.full((2, width), -1, dtype=torch.int32)
    call.table[0], call.table[1, :7] = pages[:13], pages[13:20]
    call.table = call.table.to(DEV)
    f = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).to(DEV)
    weights = torch.zeros(2, heads, width * page, device=DEV)
    at = torch.tensor([0, 0])                            # positions of the sequences so far
    call.lengths = torch.zeros(2, dtype=torch.int32, device=DEV)
    for step, new in enumerate([(150, 60), (1, 1), (1, 1), (7, 1), (1, 1)]):
        T = sum(new)
        q = torch.randn(T, heads * group, dim, generator=g).to(BF).to(DEV)
        k, v = (torch.randn(T, heads, dim, generator=g).to(BF).to(DEV) for _ in range(2))
        positions = torch.cat([at[b] + torch.arange(new[b]) for b in range(2)]).to(DEV)
        q0 = q.clone()
        q, k = km.kmeans_kv_rotate(q, k, positions, f)
        near(q, *turned(q0, positions, f, False, False, 1.0))
        at += torch.tensor(new)
        slots = []
        for b in range(2):
            place = int(call.lengths[b]) + torch.arange(new[b], device=DEV)
            slots.append(call.table[b, place // page].long() * page + place % page)
        km.kmeans_kv_write(cache, k, v, torch.cat(slots))
        call.lengths += torch.tensor(new, dtype=torch.int32, device=DEV)
        call.q, call.bounds = q, torch.tensor([0, new[0], T], dtype=torch.int32, device=DEV)
        out, lse = check_attention(call)
        before = weights.double().clone()
        w, d = weights_of(call, lse, width * page)
        call.weigh(lse, weights)
        assert ((weights.double() - before - w).abs() <= d + 2.0 ** -23 * weights.abs()).all()
        if step % 2 == 1:
            n = call.lengths.cpu()
            want = evicted(weights, n, 70, 16, 2)
            codes = [cache.k_codes.clone(), cache.v_codes.clone()]
            kept, left, ww = km.kmeans_kv_evict(cache, weights, call.table, call.lengths, 70,
                                                recent=16, first=2)
            assert torch.equal(kept.cpu(), want[0]) and torch.equal(call.lengths.cpu(), want[1])
            assert torch.equal(weights.cpu(), want[2])
            for b in range(2):
                for h in range(heads):
                    src = kept[b, h][kept[b, h] >= 0].long()
                    j = torch.arange(src.numel(), device=DEV)
                    p, to = call.table[b, src // page].long(), call.table[b, j // page].long()
                    assert torch.equal(cache.k_codes[to, h, j % page], codes[0][p, h, src % page])
                    assert torch.equal(cache.v_codes[to, h, :, j % page], codes[1][p, h, :, src % page])


# ------------------------------------------------------------------------ refusals

def refused(fn, *args, match=None, **kw):
    with pytest.raises((ValueError, km.KmeansError), match=match):
        fn(*args, **kw)


def test_refusals_of_rotate():
    q, k = torch.zeros(3, 4, 64, dtype=BF, device=DEV), torch.zeros(3, 2, 64, dtype=BF, device=DEV)
    pos, f = torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(32, dtype=torch.float64,
                                                                        device=DEV)
    r = km.kmeans_kv_rotate
    refused(r, q.float(), k, pos, f)
    refused(r, q, k.half(), pos, f)
    refused(r, q, k[:2], pos, f)
    refused(r, q, k[..., :32], pos, f)
    refused(r, q.cpu(), k, pos, f)
    refused(r, q, k, pos.int(), f)
    refused(r, q, k, pos[:2], f)
    refused(r, q, k, pos, f.float())
    refused(r, q, k, pos, f.cpu())
    refused(r, q, k, pos, torch.zeros(33, dtype=torch.float64, device=DEV))
    refused(r, q, k, pos, f, amplitude=math.inf)
    refused(r, q[..., :12].contiguous(), None, pos, f[:6])
    refused(r, q, k, pos, f, out=(q[:2], k))
    refused(r, q, k, pos, f, out=(q.new_zeros(1, 4, 64).expand(3, 4, 64), k))
    refused(r, q.clone().requires_grad_(), k, pos, f, match="gradient")
    odd = torch.zeros(3, 64, 4, dtype=BF, device=DEV).transpose(1, 2)
    refused(r, odd, None, pos, f, out=(odd, None))


def test_refusals_of_the_others():
    call = Call([(40, 3), (20, 2)], seed=2)
    _, lse = call.attend()
    w = call.weigh(lse)
    good = dict(q=call.q, bounds=call.bounds, table=call.table, lengths=call.lengths)

    def both(match=None, **kw):
        a = {**good, **kw}
        refused(km.kmeans_kv_attend_tokens, call.cache, match=match, **a)
        refused(km.kmeans_kv_weigh, call.cache, lse=lse, match=match, **a)

    both(q=call.q.half())
    both(q=call.q.cpu())
    both(q=call.q[:, :3])
    both(q=call.q.clone().requires_grad_(), match="gradient")
    both(bounds=call.bounds.long())
    both(bounds=call.bounds[:2])
    both(table=call.table.long())
    both(table=call.table[:1])
    both(lengths=call.lengths.long())
    both(window=-1)
    both(cap=-1.0)
    both(cap=math.nan)
    both(scale=math.inf)
    both(slopes=torch.zeros(3, device=DEV))
    both(slopes=torch.zeros(4, device=DEV, dtype=torch.float64))
    both(prefixes=torch.zeros(3, dtype=torch.int32, device=DEV))
    both(starts=torch.zeros(4, dtype=torch.int32, device=DEV))
    a = km.kmeans_kv_attend_tokens
    refused(a, call.cache, **good, out=call.q[:3])
    refused(a, call.cache, **good, lse=lse.double())
    refused(a, call.cache, **good, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    refused(a, call.cache, **good, ws=torch.empty(1 << 20, dtype=torch.uint8))
    refused(call.weigh, lse[:2])
    refused(call.weigh, lse.double())
    refused(call.weigh, lse, w[:1])
    refused(call.weigh, lse, w.double())
    refused(call.weigh, lse, w[:, :1].expand(2, 2, -1))
    refused(call.weigh, lse, w.transpose(1, 2).contiguous().transpose(1, 2))
    e = km.kmeans_kv_evict
    n = call.lengths
    refused(e, call.cache, w, call.table, n, 0)
    refused(e, call.cache, w, call.table, n, 5, recent=3, first=3)
    refused(e, call.cache, w, call.table, n, 5, recent=-1)
    refused(e, call.cache, w[:1], call.table, n, 5)
    refused(e, call.cache, w.half(), call.table, n, 5)
    refused(e, call.cache, w, call.table.long(), n, 5)
    refused(e, call.cache, w, call.table, n.long(), 5)
    refused(e, call.cache, w, call.table, n, 30, to=call.table[:, :1])
    refused(e, call.cache, w, call.table, torch.stack((n, n), 1)[:, 0], 5)
    refused(e, call.cache, w[:, :1].expand(2, 2, -1), call.table, n, 5)


# ------------------------------------------------------------------ other ways to the calls

def test_same_bits_without_the_call_module(monkeypatch):
    """The calls that the C++ module makes and those through ctypes are the same."""
    call = Call([(200, 30), (90, 1), (0, 0)], heads=2, group=2, dim=64, seed=21)
    set_mode(call, "all")
    positions = torch.arange(call.q.shape[0], device=DEV)
    f = torch.rand(20, dtype=torch.float64, device=DEV)

    def everything():
        q, k = km.kmeans_kv_rotate(call.q, call.q[:, :2], positions, f, interleaved=True, amplitude=1.5)
        out, lse = call.attend()
        w = call.weigh(lse)
        codes = call.cache.k_codes.clone(), call.cache.v_codes.clone()
        table = torch.arange(6, dtype=torch.int32, device=DEV).view(3, 2)
        kept, left, ww = km.kmeans_kv_evict(call.cache, w, call.table, call.lengths, 24, recent=5, first=2,
                                            to=table)
        moved = call.cache.k_codes.clone(), call.cache.v_codes.clone()
        for t, x in zip((call.cache.k_codes, call.cache.v_codes), codes):
            t.copy_(x)
        return q, k, out, lse, w, kept, left, ww, *moved

    # pages 0 to 5 take what is kept: no sequence may have them
    used = call.table[call.table >= 0]
    call.table[call.table >= 0] = used.argsort().argsort().to(torch.int32) + 6
    pages = 6 + used.numel()
    old = call.cache
    call.cache = make_cache(2, 64, 4, 256, BF, pages, old.page, seed=22)
    want = everything()
    monkeypatch.setattr(km.kv, "_fast", None)
    for a, b in zip(everything(), want):
        assert torch.equal(a, b)


def test_calls_that_need_a_gradient():
    call = Call([(40, 7)], heads=2, group=2, dim=64, seed=23)
    positions = torch.arange(7, device=DEV)
    f = torch.rand(8, dtype=torch.float64, device=DEV)
    out, lse = call.attend()
    q = call.q
    fwd = torch.autograd.forward_ad
    for leaf in (q.clone().requires_grad_(), q.clone().requires_grad_() * 1):
        call.q = leaf
        for run in (call.attend, lambda: call.weigh(lse),
                    lambda: km.kmeans_kv_rotate(leaf, None, positions, f)):
            with pytest.raises(ValueError, match="gradient"):
                run()
        with torch.no_grad():
            assert torch.equal(call.attend()[0], out)
    with fwd.dual_level():
        call.q = fwd.make_dual(q, q)
        for run in (call.attend, lambda: call.weigh(lse),
                    lambda: km.kmeans_kv_rotate(call.q, None, positions, f)):
            with pytest.raises(ValueError, match="gradient"):
                run()
    call.q = q
    w = call.weigh(lse)
    with pytest.raises(ValueError, match="gradient"):
        call.weigh(lse, w.clone().requires_grad_())
    with pytest.raises(ValueError, match="gradient"):
        call.weigh(lse.clone().requires_grad_())
    with pytest.raises(ValueError, match="gradient"):
        km.kmeans_kv_evict(call.cache, w.clone().requires_grad_(), call.table, call.lengths, 8)


def test_two_streams_at_once():
    calls = [Call([(3000, 70), (500, 1)], heads=2, group=4, dim=128, seed=31),
             Call([(900, 1), (2000, 5)], heads=2, group=4, dim=128, seed=32)]
    want = []
    for c in calls:
        out, lse = c.attend()
        want.append((out, lse, c.weigh(lse)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[], []]
    for _ in range(10):
        for c, s, g in zip(calls, streams, got):
            with torch.cuda.stream(s):
                out, lse = c.attend()
                g.append((out, lse, c.weigh(lse)))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for x in g:
            for a, b in zip(x, w):
                assert torch.equal(a, b)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lengths,keep,kind", [
    # a tile of kept positions that lie far from each other, and near; many heads, whose
    # workgroups take one tile after the other
    ([20000, 9000], 300, "ties"), ([1500] * 6, 1400, "ties"), ([700, 20000], 650, "ties"),
])
def test_evict_far_and_near(lengths, keep, kind, in_place):
    for dim, sub in ((64, 8), (128, 2), (96, 8)):
        run_evict(lengths, keep, 10, 2, None, in_place, dim, sub, 32, heads=3 if len(lengths) < 3 else 80,
                  kind=kind)


def test_offsets_past_32_bits():
    """The last pages of a cache whose codes are more than 2^32 bytes, and weights whose
    rows are more than 2^31 elements apart."""
    heads, dim, sub, page = 8, 128, 2, 64
    each = heads * page * (dim // sub)
    pages = (1 << 32) // each + 200
    g = torch.Generator().manual_seed(41)
    centres = torch.randn(heads, dim // sub, 256, sub, generator=g).to(BF).to(DEV)
    cache = km.KVCodes.empty(centres, centres, pages, page)
    n = 40                                               # pages of a sequence
    low = torch.arange(n, dtype=torch.int32, device=DEV).view(1, n)
    high = low + (pages - n)
    for t in (cache.k_codes, cache.v_codes):
        t[:n].copy_(torch.randint(0, 256, t[:n].shape, generator=g, dtype=torch.uint8))
        t[-n:] = t[:n]
    lengths = torch.tensor([n * page - 5], dtype=torch.int32, device=DEV)
    for new in (1, 40):
        q = torch.randn(new, heads * 4, dim, generator=g).to(BF).to(DEV)
        bounds = torch.tensor([0, new], dtype=torch.int32, device=DEV)
        want = km.kmeans_kv_attend_tokens(cache, q, bounds, low, lengths)
        got = km.kmeans_kv_attend_tokens(cache, q, bounds, high, lengths)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        w = km.kmeans_kv_weigh(cache, q, want[1], bounds, low, lengths)
        assert torch.equal(km.kmeans_kv_weigh(cache, q, want[1], bounds, high, lengths), w)
    # the same weights to both, in rows far apart
    room = torch.zeros((1 << 31) + heads * n * page, device=DEV)
    far = room.as_strided((2, heads, n * page), (1 << 31, n * page, 1))
    both, two = torch.cat((low, high)), torch.cat((lengths, lengths))
    km.kmeans_kv_weigh(cache, q.repeat(2, 1, 1), want[1].repeat(2, 1),
                       torch.tensor([0, 40, 80], dtype=torch.int32, device=DEV), both, two, far)
    assert torch.equal(far[0], far[1])
    # one sequence and two share rows out in different ways: sums of the same 160 weights, none
    # below zero, in two orders, each off by at most 159 roundings of at most the sum
    assert ((far[0].double() - w[0]).abs() <= 2 * 159 * 2.0 ** -24 * w[0].double()).all()
    was = far.clone()
    kept, left, ww = km.kmeans_kv_evict(cache, far, both, two, 1000, recent=30)
    assert ww is far and left is two and left.tolist() == [1000, 1000]
    assert torch.equal(kept[0], kept[1]) and torch.equal(far[0], far[1])
    assert (kept[0].diff(dim=-1) > 0).all() and torch.equal(far[0, :, :1000], was[0].gather(1, kept[0].long()))
    for t in (cache.k_codes, cache.v_codes):
        assert torch.equal(t[:n], t[-n:])
