"""Gradients of the norm with eps = 0: slots of a thread block that hold no row must not count, where 1 / sqrt(0) is infinite."""
import pytest
import torch

from paper_2509_22323_b200 import binding
from tests import plain_operators as plain
from tests.test_gpu_rotary import DEV, make, rotary_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,Hk,N,D,layout", [
    (1, 3, 1, 17, 64, "halves"),     # tokens behind the last in the last tile, heads that are no multiple of a step
    (2, 5, 2, 1, 128, "pairs"),      # one token, whose heads leave slots empty
    (1, 1, 0, 1, 16, "pairs"),
    (2, 24, 8, 300, 96, "halves"),   # and lanes without channels
])
def test_gradients_with_an_eps_of_zero(kind, B, H, Hk, N, D, layout):
    gen = torch.Generator(device=DEV).manual_seed(N + D)
    rotary, angle = rotary_of(layout, D, 1, B, N, gen)
    x = [make((B, h, N, D), kind, "heads", gen, 1.7) if h else None for h in (H, Hk)]
    d = [make((B, h, N, D), kind, "heads", gen, 0.3) if h else None for h in (H, Hk)]
    gains = [torch.rand(D, generator=gen, device=DEV) + 0.5 for _ in range(2)]
    got = binding.rapid3_norm_rotary_backward(d[0], d[1], x[0], x[1], gains[0], gains[1] if Hk else None, 0.0, rotary)
    for i in range(2 if Hk else 1):
        X, gain = x[i].double(), gains[i].double()
        assert (X.square().sum(-1) > 0).all()
        g, size = plain.turn(d[i].double(), -angle, layout), plain.pair_size(d[i].double(), D, layout)
        r = torch.rsqrt(X.square().mean(-1, keepdim=True))
        u = X * r
        want = r * (g * gain - u * (g * gain * u).mean(-1, keepdim=True))
        # fp32 arithmetic and a result rounded once, as with any eps: 2^-19 of the magnitudes, half a step
        magnitude = r * (size * gain + u.abs() * 4 * (size * gain * u.abs()).mean(-1, keepdim=True))
        bound = plain.half_step(x[i].dtype) * want.abs() + 2.0 ** -19 * magnitude + plain.smallest(x[i].dtype)
        assert ((got[i].double() - want).abs() <= bound).all()
        # 2^-15 of the terms: each off by 2^-18, sums of at most 2^8 rows
        terms = (size * u.abs()).sum((0, 1, 2))
        assert ((got[2 + i].double() - (g * u).sum((0, 1, 2))).abs() <= 2.0 ** -15 * terms + 1e-30).all()
