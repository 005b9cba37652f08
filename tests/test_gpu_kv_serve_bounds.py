"""Attention of new tokens and summed weights within bounds that count each rounding
once: caps far above all scores, and weights that units of few rows give to the values
in two 16-bit parts."""
import math

import pytest
import torch

import kv_serve_reference as ref
from kv_serve_reference import BF, FP, Call, check_attention, weights_of

pytestmark = pytest.mark.gpu

_scores = ref.scores


def capped(call, b):
    """kv_serve_reference.scores, with the error that a cap adds bounded by what the
    scores are, not by the cap.

    Up to 5/8 of the cap, y = cap tanh(x) with x = z scale / cap is off, in steps of 2^-24
    of itself, by 3 for x (the scale, its quotient with the cap, the product; the condition of
    tanh is at most 1), 3 for the cap to base 2 and its product with x, 1 for the last sum,
    and less than 1 for the polynomial (2^-27) and for the roundings of its terms past the
    first, which are less than an eighth of it: 8. Beyond, by roundings of numbers up
    to 2 cap."""
    more = call.more
    cap = more["cap"]
    call.more = {k: v for k, v in more.items() if k not in ("cap", "slopes")}
    z, off, *others = _scores(call, b)
    call.more = more
    x = z / cap
    y = (cap * torch.tanh(x)).masked_fill(z == -math.inf, -math.inf)
    near = x.abs() <= 0.62
    size = y.abs().nan_to_num(0, 0, 0)
    off = off + torch.where(near, size * 8 * 2.0 ** -24, cap * 2.0 ** -21).masked_fill(y == -math.inf, 0.0)
    assert more.get("slopes") is None
    return (y, off, *others)


# Few and many rows to a unit.
@pytest.mark.parametrize("sizes", [[(60, 20), (300, 2)], [(400, 390), (330, 330)]])
@pytest.mark.parametrize("scale,cap", [(1.0, 1e6), (1.0, 1e30), (0.3, 300.0), (0.125, 30.0), (-0.125, 5.0)])
def test_caps(monkeypatch, scale, cap, sizes):
    monkeypatch.setattr(ref, "scores", capped)
    call = Call(sizes, heads=1, group=4, dim=64, dtype=FP, seed=8)
    call.more.update(scale=scale, cap=cap)
    _, lse = check_attention(call)
    w, d = weights_of(call, lse, call.table.shape[1] * call.cache.page)
    assert ((call.weigh(lse).double() - w).abs() <= d).all()


@pytest.mark.parametrize("mode", ["plain", "masks", "exact scores"])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sizes,kw", [
    ([(77, 1), (300, 1), (129, 1)], dict(dim=128, group=4)),            # 4 and 8 rows of 8
    ([(500, 1), (33, 1)], dict(dim=64, group=8, sub=2)),
    ([(203, 5), (64, 3), (40, 4)], dict(dim=96, group=5, sub=8)),       # up to 25 in units of 16
    ([(3000, 2)], dict(dim=128, group=16)),                             # joined by a second launch
])
def test_weights_in_two_parts(sizes, kw, dtype, mode):
    """Two parts leave 2^-17 of a weight in bf16; in fp16 2^-21 of it, 2^-31 of the largest and
    what lies below both parts' least numbers, 2^-24 of a weight lifted by 2^7: one part, with
    half a step of the type, would be seen in outputs that are small beside their terms: those
    of bf16 in all modes, of fp16 where the scores are sums of few bits without a rounding."""
    call = Call(sizes, heads=2, dtype=dtype, seed=50, q_scale=0.5, **kw)
    if mode == "masks":
        call.more["window"] = 45
        call.more["starts"] = torch.arange(call.q.shape[0], dtype=torch.int32, device=ref.DEV) % 3 * 20
    if mode == "exact scores":
        call.q.copy_((call.q * 4).round().clamp(-4, 4) / 4)
        call.cache.k_centres.copy_((call.cache.k_centres * 2).round().clamp(-4, 4) / 2)
        call.more["scale"] = 0.125
    out, lse = call.attend()
    half = torch.finfo(dtype).eps / 2
    part, least = (2.0 ** -17, 0.0) if dtype is BF else (2.0 ** -21, 2.0 ** -31 + 2.0 ** -31)
    tiny = 0.0 if dtype is BF else 2.0 ** -25            # half a step of the least outputs
    for b in range(len(sizes)):
        z, off, k, v, t0, t1 = ref.scores(call, b)
        if mode == "exact scores":
            off = z.abs() * 2.0 ** -22 + 2.0 ** -21      # to base 2, and its power
        total = torch.logsumexp(z, -1)
        w = torch.exp(z - torch.where(total == -math.inf, 0.0, total)[..., None])
        v, n = v[:, None], z.shape[-1]
        o, size = torch.matmul(w, v), torch.matmul(w, v.abs())
        rel = 2 * off.amax(-1, keepdim=True) + part + (n ** 0.5 + 64) * 2.0 ** -22
        seen = (z > -math.inf).double()
        bound = (half * o.abs() + rel * (1 + half) * size + tiny
                 + least * w.amax(-1, keepdim=True) * torch.matmul(seen, v.abs()))
        rows = lambda x: x.permute(2, 0, 1, 3).reshape(t1 - t0, -1, x.shape[-1])  # noqa: E731
        assert ((out[t0:t1].double() - rows(o)).abs() <= rows(bound)).all()
