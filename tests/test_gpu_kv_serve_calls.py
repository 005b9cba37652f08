"""Calls of serving from the key-value cache that its documentation allows, or refuses,
with tensors that share memory or carry gradients."""
import math

import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_1402_3788_amd as km
from kv_serve_reference import BF, DEV, evicted, make_cache
from paper_1402_3788_amd.kv import _call
from paper_1402_3788_amd.kv_serve import _Evict

pytestmark = pytest.mark.gpu


def rotate_inputs(tokens=3, heads=4, half=16, seed=0):
    g = torch.Generator().manual_seed(seed)
    room = torch.randn(heads, tokens, 64, generator=g).to(BF).to(DEV)
    positions = torch.arange(5, 5 + tokens, device=DEV)
    return room, positions, torch.rand(half, dtype=torch.float64, generator=g).to(DEV)


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("fast", [True, False])
def test_rotate_to_another_view_of_the_same_memory(which, fast, monkeypatch):
    """An output that begins where its input does has the input's strides, or the call is
    refused and nothing written."""
    if not fast:
        monkeypatch.setattr(km.kv, "_fast", None)
    room, positions, f = rotate_inputs()
    was = room.clone()
    x = room.transpose(0, 1)                             # [tokens, heads, dim]
    other = torch.randn(3, 4, 64).to(BF).to(DEV)
    view = room.view(3, 4, 64)
    args, out = ((x, other), (view, None)) if which == "q" else ((other, x), (None, view))
    with pytest.raises((ValueError, km.KmeansError)):
        km.kmeans_kv_rotate(*args, positions, f, out=out)
    torch.cuda.synchronize()
    assert torch.equal(room, was)
    # another tensor of the same layout is in place
    want = km.kmeans_kv_rotate(x, None, positions, f)[0]
    again = room.as_strided((3, 4, 64), x.stride())
    args, out = ((x, other), (again, None)) if which == "q" else ((other, x), (None, again))
    got = km.kmeans_kv_rotate(*args, positions, f, out=out)[0 if which == "q" else 1]
    assert got is again and torch.equal(x, want)


@pytest.mark.parametrize("shape,strides", [
    ((1, 4, 64), (4096, 64, 1)), ((1, 4, 64), (3, 64, 1)), ((3, 1, 64), (64, 1000, 1)),
    ((3, 1, 64), (64, 5, 1)),
])
def test_rotate_in_place_whatever_the_stride_of_a_single_row(shape, strides):
    room, positions, f = rotate_inputs(tokens=3, heads=4)
    x = room.flatten()[:math.prod(shape)].view(shape)
    again = room.as_strided(shape, strides)
    want = km.kmeans_kv_rotate(x, None, positions[:shape[0]], f)[0]
    was = room.clone()
    for q, out in ((x, again), (again, x), (again, again)):
        room.copy_(was)
        got = km.kmeans_kv_rotate(q, None, positions[:shape[0]], f, out=(out, None))[0]
        assert got is out and torch.equal(x, want)


@pytest.mark.parametrize("fast", [True, False])
def test_rotate_by_frequencies_that_need_a_gradient(fast, monkeypatch):
    """Learned frequencies would lose their gradient without a word."""
    if not fast:
        monkeypatch.setattr(km.kv, "_fast", None)
    room, positions, f = rotate_inputs()
    x = room.transpose(0, 1)
    want = km.kmeans_kv_rotate(x, None, positions, f)[0]
    leaf = f.clone().requires_grad_()
    for t in (leaf, leaf * 1):
        with pytest.raises(ValueError, match="gradient"):
            km.kmeans_kv_rotate(x, None, positions, t)
        with pytest.raises(ValueError, match="gradient"):
            km.kmeans_kv_rotate(x, None, positions, t, out=(torch.empty_like(want), None))
        with torch.no_grad():
            assert torch.equal(km.kmeans_kv_rotate(x, None, positions, t)[0], want)
        assert torch.equal(km.kmeans_kv_rotate(x, None, positions, t.detach())[0], want)
    with fwd.dual_level():
        with pytest.raises(ValueError, match="gradient"):
            km.kmeans_kv_rotate(x, None, positions, fwd.make_dual(f, f))
        assert torch.equal(km.kmeans_kv_rotate(x, None, positions, f)[0], want)


@pytest.mark.parametrize("positions", [700, 2000, 2100, 9000, 70000])
@pytest.mark.parametrize("codes,weights", [("to", "in place"), ("in place", "apart"), ("to", "apart")])
def test_evict_weights_in_place_whether_codes_are_or_not(positions, codes, weights):
    """weights_out may be weights and lengths_out lengths, through the C entry point, where
    the codes go to other pages, and need not be where they stay; rows of one workgroup's
    tile of weights (2048), and of many."""
    heads, page, B, keep = 4, 64, 3, positions * 2 // 5
    g = torch.Generator().manual_seed(positions)
    lengths = torch.tensor([positions, positions - 13, positions // 2], dtype=torch.int32)
    width = -(-positions // page)
    fresh = -(-keep // page)
    perm = torch.randperm(B * (width + fresh), generator=g).to(torch.int32)
    table = perm[:B * width].view(B, width).to(DEV)
    to = perm[B * width:].view(B, fresh).to(DEV)
    cache = make_cache(heads, 64, 4, 256, BF, B * (width + fresh), page)
    # rows with room behind them
    room = torch.full((B, heads, positions + 24), 7.0)
    room[..., :positions] = torch.rand(B, heads, positions, generator=g)
    want = evicted(room[..., :positions], lengths, keep, 5, 3)
    kc, vc = cache.k_codes.clone(), cache.v_codes.clone()
    n, w = lengths.to(DEV), room.to(DEV)
    n_out, w_out = (n, w) if weights == "in place" else (torch.zeros_like(n), torch.full_like(w, 7.0))
    kept = torch.empty(B, heads, keep, dtype=torch.int32, device=DEV)
    goal = to if codes == "to" else table
    e = _Evict(table.data_ptr(), width, width, n.data_ptr(), w.data_ptr(), w.stride(0), w.stride(1),
               positions, B, keep, 5, 3, to.data_ptr() if codes == "to" else None, fresh, fresh)
    _call(cache, km._lib.kmeans_kv_evict, "kmeans_kv_evict", e, kept.data_ptr(), n_out.data_ptr(),
          w_out.data_ptr(), w.stride(0), w.stride(1))
    torch.cuda.synchronize()
    assert torch.equal(kept.cpu(), want[0]) and torch.equal(n_out.cpu(), want[1])
    assert torch.equal(w_out[..., :positions].cpu(), want[2]) and (w_out[..., positions:] == 7).all()
    if weights == "apart":
        assert torch.equal(w.cpu(), room) and torch.equal(n.cpu(), lengths)
    for b, m in enumerate(want[1].tolist()):
        j = torch.arange(m, device=DEV)
        for h in range(heads):
            src = kept[b, h, :m].long()
            p, q = table[b, src // page].long(), goal[b, j // page].long()
            assert torch.equal(cache.k_codes[q, h, j % page], kc[p, h, src % page])
            assert torch.equal(cache.v_codes[q, h, :, j % page], vc[p, h, :, src % page])
