"""Refusals of the windowed attention before any GPU call, and its plain 64-bit form against differences and by hand."""
import ctypes
import math

import pytest
import torch

from paper_2509_22323_b200 import binding
from tests import plain_operators as plain


def call(fn="rapid3_window_attn", shape=None, rows=None, q=True, lse=4096, workspace=4096, size=None):
    lib = binding.load()
    s = dict(type=0, B=2, H=4, H_kv=2, D=64, n_q=5, n_kv=9, left=3, right=0, n_sink=1, n_full=0, softmax_scale=0.125, q_len=None, kv_len=None)
    w = binding.Window(**(s | (shape or {})))
    t = binding.Rows(**(dict(data=8192, stride_b=4000, stride_h=800, stride_n=72) | (rows or {})))
    if fn == "rapid3_window_attn":
        return lib.rapid3_window_attn(w, t if q else None, t, t, t, None, None)
    if size is None:
        size = max(0, lib.rapid3_window_workspace_bytes(w))
    return lib.rapid3_window_attn_backward(w, t, t, t, t, lse, t, t, t, t, workspace, size, None)


BAD = [(-2, dict(type=2)), (-1, dict(type=3)), (-2, dict(D=96)), (-1, dict(B=0)), (-1, dict(H=0)), (-1, dict(H_kv=0)), (-1, dict(H=5)), (-1, dict(n_q=0)),
       (-1, dict(n_kv=0)), (-2, dict(n_q=1 << 30)), (-2, dict(n_kv=1 << 30)), (-2, dict(H=131072)), (-1, dict(left=-2)), (-1, dict(right=-2)),
       (-1, dict(n_sink=-1)), (-1, dict(n_full=-1)), (-1, dict(softmax_scale=0.0)), (-1, dict(softmax_scale=math.nan)), (-1, dict(softmax_scale=3e38)), (-2, dict(B=1 << 20, n_kv=1 << 22))]


@pytest.mark.parametrize("fn", ["rapid3_window_attn", "rapid3_window_attn_backward"])
@pytest.mark.parametrize("code,shape", BAD)
def test_shapes_refused(fn, code, shape):
    assert call(fn, shape) == code


@pytest.mark.parametrize("fn", ["rapid3_window_attn", "rapid3_window_attn_backward"])
@pytest.mark.parametrize("rows", [dict(data=None), dict(data=8194), dict(stride_n=56), dict(stride_n=76), dict(stride_h=0), dict(stride_b=-4000)])
def test_rows_refused(fn, rows):
    assert call(fn, rows=rows) == -1


def test_other_refusals():
    lib = binding.load()
    assert call(rows=dict(stride_b=1 << 39)) == -2
    assert call(q=False) == -1
    assert call("rapid3_window_attn_backward", lse=None) == -1
    assert call("rapid3_window_attn_backward", workspace=None) == -1
    assert call("rapid3_window_attn_backward", workspace=4104) == -1
    assert call("rapid3_window_attn_backward", size=16) == -3
    assert call("rapid3_window_attn_backward", dict(B=70000, H=2, H_kv=1)) == -2
    assert lib.rapid3_window_attn(None, None, None, None, None, None, None) == -1
    assert lib.rapid3_window_workspace_bytes(None) == -1
    assert lib.rapid3_window_status(None) == -1


def test_visible_by_hand():
    rows = lambda *a: ["".join("x" if v else "." for v in r) for r in plain.visible(*a).tolist()]
    assert rows(4, 6, 1, 0, 1, 0, 4, 6) == ["xxx...", "x.xx..", "x..xx.", "x...xx"]       # the last rows; first token and two near ones
    assert rows(3, 4, 0, 0, 0, 0, 3, 2) == ["....", "x...", ".x.."]                       # the first row stands before the first key
    assert rows(3, 4, 0, 0, 0, 1, 3, 2) == ["....", "xx..", ".x.."]                       # and is none of the full rows, the first of which is at position 0
    assert rows(3, 3, 1, 1, 1, 1, 3, 3) == ["xxx", "xxx", "xxx"]
    assert rows(4, 4, 0, 0, 2, 2, 4, 4) == ["xxxx", "xxxx", "xxx.", "xx.x"]                # two text tokens
    assert rows(2, 3, -1, -1, 0, 0, 1, 2) == ["xx.", "..."]                               # places behind the lengths


def test_plain_attention_gradients_against_differences():
    gen = torch.Generator().manual_seed(1)
    q, k, v, w = (torch.randn((n, 8), generator=gen, dtype=torch.float64) for n in (5, 7, 7, 5))
    seen = plain.visible(5, 7, 2, 0, 1, 0, 5, 7)
    loss = lambda q, k, v: (w * plain.attention(q, k, v, seen, 0.4)[0]).sum().item()
    out, _, p = plain.attention(q, k, v, seen, 0.4)
    for i, g in enumerate(plain.attention_gradients(q, k, v, out, p, w, 0.4)):
        for at in ((0, 0), (3, 5), (4, 7)):
            args = [[q, k, v], [q, k, v]]
            for sign in (0, 1):
                x = args[sign][i].clone()
                x[at] += (1e-5, -1e-5)[sign]
                args[sign][i] = x
            assert math.isclose((loss(*args[0]) - loss(*args[1])) / 2e-5, g[at].item(), rel_tol=1e-6, abs_tol=1e-8)
