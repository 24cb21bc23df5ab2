"""Rotary frequencies, the plain 64-bit forms against differences, and refusals: no GPU needed."""
import ctypes
import math

import pytest
import torch

from paper_2509_22323_b200 import binding
from tests import plain_operators as plain


def test_frequencies_by_hand():
    f, a = binding.rapid3_rotary_freqs(8, 10000.0)
    assert a == 1.0
    torch.testing.assert_close(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14, atol=0)
    f, a = binding.rapid3_rotary_freqs(8, 10000.0, "linear", 4.0)
    assert a == 1.0
    torch.testing.assert_close(f, torch.tensor([0.25, 0.025, 0.0025, 0.00025], dtype=torch.float64), rtol=1e-14, atol=0)
    # a larger base: the fastest pair as it was, the slowest slower by the factor
    f, _ = binding.rapid3_rotary_freqs(8, 10000.0, "base", 4.0)
    assert f[0] == 1.0 and math.isclose(f[3].item(), 0.001 / 4, rel_tol=1e-13)
    # two pairs: 32 turns and more keep their frequency, one and fewer are interpolated, between them in proportion
    trained = 4096
    f0, _ = binding.rapid3_rotary_freqs(64, 10000.0)
    f, a = binding.rapid3_rotary_freqs(64, 10000.0, "parts", 8.0, trained, 32.0, 1.0)
    assert math.isclose(a, 1 + 0.1 * math.log(8.0), rel_tol=1e-6)
    turns = trained * f0 / (2 * math.pi)
    assert torch.equal(f[turns >= 32], f0[turns >= 32])
    torch.testing.assert_close(f[turns <= 1], f0[turns <= 1] / 8, rtol=1e-14, atol=0)
    mid = (turns > 1) & (turns < 32)
    assert mid.any()
    share = (turns[mid] - 1) / 31
    torch.testing.assert_close(f[mid], f0[mid] * share + f0[mid] / 8 * (1 - share), rtol=1e-13, atol=0)


@pytest.mark.parametrize("args", [(7, 1e4), (0, 1e4), (8, 1.0), (8, math.inf), (8, 1e4, "linear", 0.5), (8, 1e4, "sideways", 2.0),
                                  (8, 1e4, "parts", 2.0, 0), (8, 1e4, "parts", 2.0, 100, 1.0, 1.0), (8, 1e4, "base", math.nan)])
def test_frequencies_refused(args):
    with pytest.raises(binding.Rapid3Error) as e:
        binding.rapid3_rotary_freqs(*args)
    assert e.value.code == -1


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_plain_gradients_against_differences(layout):
    """The formulas that the kernels' gradients are tested with, against differences of the plain forward form."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((1, 2, 3, 16), generator=gen, dtype=torch.float64)
    w, gain = torch.randn(x.shape, generator=gen, dtype=torch.float64), torch.randn(16, generator=gen, dtype=torch.float64)
    angle = plain.angles(torch.rand(4, generator=gen, dtype=torch.float64), torch.tensor([[[3], [5], [1000]]]), [4])
    loss = lambda x, gain: (w * plain.turn(plain.norm(x, gain, 1e-3), angle, layout, 1.25)).sum()
    g = 1.25 * plain.turn(w, -angle, layout)
    g[..., 8:] = w[..., 8:]
    u = plain.norm(x, 1.0, 1e-3)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-3)
    dx, dgain = r * (g * gain - u * (g * gain * u).mean(-1, keepdim=True)), (g * u).sum((0, 1, 2))
    step = 1e-5
    for at in [(0, 0, 0, 0), (0, 1, 2, 5), (0, 1, 1, 9), (0, 0, 2, 15)]:
        d = torch.zeros_like(x)
        d[at] = step
        assert math.isclose((loss(x + d, gain) - loss(x - d, gain)).item() / (2 * step), dx[at].item(), rel_tol=1e-6, abs_tol=1e-8)
    for c in (0, 6, 13):
        d = torch.zeros_like(gain)
        d[c] = step
        assert math.isclose((loss(x, gain + d) - loss(x, gain - d)).item() / (2 * step), dgain[c].item(), rel_tol=1e-6, abs_tol=1e-8)


def call(fn="rapid3_rotary", shape=None, rows=None, turn=None, **other):
    """The C entry with pointers that are never followed: every refusal comes before the first CUDA call."""
    lib = binding.load()
    s = dict(type=0, B=2, N=5, D=64, H_q=4, H_k=2) | (shape or {})
    t = dict(layout=1, channels=64, axes=1, axis_pairs=(32, 0, 0, 0), freq=4096, pos=None, pos_stride_b=0, pos_stride_n=1, pos0=0, amplitude=1.0)
    t |= turn or {}
    t["axis_pairs"] = (ctypes.c_int32 * 4)(*t["axis_pairs"])
    S, T = binding.Heads(**s), binding.Turn(**t)
    r = dict(data=8192, stride_b=2000, stride_h=400, stride_n=72) | (rows or {})
    q, k, qo, ko = (binding.Rows(**r) for _ in range(4))
    k = other.get("k", k)
    if fn == "rapid3_rotary":
        return lib.rapid3_rotary(S, q, k, T, 0, qo, ko, None)
    gain, eps = other.get("gain", 4096), other.get("eps", 1e-6)
    if fn == "rapid3_norm_rotary":
        return lib.rapid3_norm_rotary(S, q, k, gain, gain, eps, T, qo, ko, None)
    size = lib.rapid3_norm_rotary_workspace_bytes(S)
    return lib.rapid3_norm_rotary_backward(S, q, k, q, k, gain, gain, eps, T, qo, ko, other.get("dgain", 4096), 4096, other.get("workspace", 4096),
                                           other.get("size", size), None)


@pytest.mark.parametrize("code,what", [
    (-1, dict(shape=dict(type=3))), (-1, dict(shape=dict(type=-1))), (-1, dict(shape=dict(B=0))), (-1, dict(shape=dict(N=0))),
    (-1, dict(shape=dict(H_q=0))), (-1, dict(shape=dict(H_k=-1))), (-2, dict(shape=dict(D=8))), (-2, dict(shape=dict(D=72))),
    (-2, dict(shape=dict(D=512))), (-2, dict(shape=dict(B=70000, N=70000))),
    (-1, dict(rows=dict(data=None))), (-1, dict(rows=dict(data=8200))), (-1, dict(rows=dict(stride_n=36))), (-1, dict(rows=dict(stride_n=0))),
    (-1, dict(rows=dict(stride_h=401))), (-1, dict(rows=dict(stride_b=-2000))),
    (-1, dict(turn=dict(layout=2))), (-1, dict(turn=dict(channels=63))), (-1, dict(turn=dict(channels=128, axis_pairs=(64, 0, 0, 0)))),
    (-2, dict(turn=dict(channels=20, axis_pairs=(10, 0, 0, 0)))), (-1, dict(turn=dict(axes=0))), (-1, dict(turn=dict(axes=5))),
    (-1, dict(turn=dict(axis_pairs=(31, 0, 0, 0)))), (-1, dict(turn=dict(freq=None))), (-1, dict(turn=dict(amplitude=math.inf))),
    (-1, dict(turn=dict(pos0=-1))), (-1, dict(turn=dict(axes=2, axis_pairs=(16, 16, 0, 0)))), (-1, dict(turn=dict(pos=4096, pos_stride_n=-1))),
    (-1, dict(k=None)),
    (-1, dict(fn="rapid3_norm_rotary", gain=None)), (-1, dict(fn="rapid3_norm_rotary", eps=-1.0)), (-1, dict(fn="rapid3_norm_rotary", eps=math.nan)),
    (-1, dict(fn="rapid3_norm_rotary_backward", dgain=None)), (-1, dict(fn="rapid3_norm_rotary_backward", workspace=None)),
    (-1, dict(fn="rapid3_norm_rotary_backward", workspace=4100)), (-3, dict(fn="rapid3_norm_rotary_backward", size=1000)),
])
def test_refused_before_any_gpu_call(code, what):
    assert call(**what) == code


def test_null_shapes_are_refused():
    lib = binding.load()
    assert lib.rapid3_rotary(None, None, None, None, 0, None, None, None) == -1
    assert lib.rapid3_norm_rotary_workspace_bytes(None) == -2
    assert lib.rapid3_norm_rotary_workspace_bytes(binding.Heads(0, 1, 1, 128, 1, 1)) >= 2 * 128 * 4


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError):
        binding.Rotary("halves", torch.ones(4, dtype=torch.float64))
