"""Gradients where a warp's group of sixteen keys holds one key alone, the last, and a row sees that key and no other: every row of the
block sees the key, so that nothing has to be hidden, and yet the row has no gradient of its score."""
import pytest
import torch

from paper_2509_22323_b200 import binding
from tests.window_cases import DEV, Case

pytestmark = pytest.mark.gpu

CASES = [  # B, H, Hkv, n_q, n_kv, left, right, q_len, kv_len: keys = 1 modulo 16; the last row sees the last key
    (1, 2, 1, 64, 65, 0, -1, None, None),
    (1, 2, 2, 64, 65, 0, 63, None, None),
    (1, 2, 1, 64, 17, 0, -1, None, None),
    (1, 3, 1, 128, 17, 0, -1, None, None),
    (2, 4, 2, 128, 129, 0, -1, None, None),
    (1, 4, 2, 128, 145, 0, -1, None, None),
    (1, 2, 1, 320, 321, 0, 100, None, None),
    (3, 4, 2, 200, 200, 0, -1, [128, 64, 192], [145, 33, 193]),
]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,Hkv,n_q,n_kv,left,right,q_len,kv_len", CASES)
def test_a_lone_key_seen_by_whole_blocks(kind, D, B, H, Hkv, n_q, n_kv, left, right, q_len, kv_len):
    c = Case(kind, B, H, Hkv, D, n_q, n_kv, left, right, 0, 0, q_len, kv_len)
    for b, (r, n) in enumerate(c.lens):
        assert n % 16 == 1 and c.seen[b][r - 1].sum() == 1 and c.seen[b][r - 1, n - 1] and c.seen[b][r - 64:, n - 1].all()
    out, lse = c.fresh(H, n_q), torch.full((B, H, n_q), 77.0, device=DEV)
    binding.rapid3_window_attn(c.q, c.k, c.v, out, lse, **c.rule)
    grads = c.fresh(H, n_q), c.fresh(Hkv, n_kv), c.fresh(Hkv, n_kv)
    binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, *grads, **c.rule)
    assert binding.rapid3_window_status() == 0
    c.check(out, lse, grads)
    for b, (r, n) in enumerate(c.lens):
        assert (grads[0][b, :, r - 1] == 0).all()
