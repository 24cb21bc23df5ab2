"""Rows that see fewer than 256 keys behind rows that see every key: their dq is off by the rounding of dS and its own, and by no more, as it is
where no row is full (h sqrt(E[1 / m^2] / 3) = 0.425 h each in the mean square, m the mantissa, evenly spread in its logarithm; a tenth is left
for what is not spread so)."""
import math

import pytest
import torch

from paper_2509_22323_b200 import binding
from tests import plain_operators as plain
from tests.window_cases import DEV, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_full,left", [(128, -1), (140, -1), (128, 30), (300, 60)])
def test_rows_of_few_keys_behind_full_rows(D, n_full, left):
    N = 512
    c = Case("bf16", 4, 8, 4, D, N, N, left, 0, 0, n_full)
    out, lse = binding.rapid3_window_attn(c.q, c.k, c.v, None, torch.empty((4, 8, N), device=DEV), **c.rule)
    dq, _, _ = binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, **c.rule)
    off = size = 0.0
    for b in range(4):
        few = c.seen[b].sum(-1) < 256
        assert few.any() and not few[:n_full].any()
        for h in range(8):
            q, k, v, d = c.q[b, h].double(), c.k[b, h // 2].double(), c.v[b, h // 2].double(), c.dout[b, h].double()
            o, _, p = plain.attention(q, k, v, c.seen[b], c.scale)
            want = plain.attention_gradients(q, k, v, o, p, d, c.scale)[0]
            off += (dq[b, h].double() - want)[few].square().sum().item()
            size += want[few].square().sum().item()
    assert math.sqrt(off / size) <= 1.1 * math.sqrt(2) * 0.4246 * 2.0 ** -8, math.sqrt(off / size) * 2 ** 8
