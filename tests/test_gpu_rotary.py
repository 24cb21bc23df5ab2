"""rapid3_rotary, rapid3_norm_rotary and rapid3_norm_rotary_backward on the GPU against the plain 64-bit forms.

Tolerances.  A result is rounded once: half a step of its type.  Before that the fp32 arithmetic is off by, relative to the
magnitudes that are added: the fraction of a turn rounded to fp32, at most half a turn, 2 pi 2^-26 = 2^-23.3; sine and cosine 2 ulp,
2^-22; products, sums and amplitude 6 roundings of 2^-24; the norm's sum of squares 12 roundings halved by the root and rsqrt 2 ulp:
below 2^-20.5 in all.  FP32 = 2^-19 leaves a factor of two."""
import math

import pytest
import torch

from paper_2509_22323_b200 import binding
from tests import plain_operators as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
FP32 = 2.0 ** -19
T = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def make(shape, kind, order, gen, scale=1.0):
    B, H, N, D = shape
    x = torch.randn((B, N, H, D) if order == "tokens" else shape, generator=gen, device=DEV).mul_(scale).to(T[kind])
    if order == "tokens":
        return x.transpose(1, 2)
    if order == "packed":                                            # every other row of a wider buffer
        wide = torch.full((B, H, 2 * N, D + 16), math.nan, dtype=T[kind], device=DEV)
        wide[:, :, ::2, 16:] = x
        return wide[:, :, ::2, 16:]
    return x


def rotary_of(layout, channels, axes, B, N, gen, far=100000, amplitude=1.0, shared=False):
    pairs = channels // 2
    counts = [pairs] if axes == 1 else [pairs // 4, pairs - pairs // 4 - pairs // 3, pairs // 3]
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in counts]).to(DEV)
    pos = torch.randint(0, far, (1 if shared else B, N, axes), generator=gen, device=DEV, dtype=torch.int32)
    return binding.Rotary(layout, freq, pos, amplitude=amplitude, axis_pairs=counts), plain.angles(freq, pos, counts)


def close(got, want, size, what):
    """|got - want| <= half a step of the type + FP32 of the magnitudes that made it."""
    bound = plain.half_step(got.dtype) * want.abs() + FP32 * size + plain.smallest(got.dtype)
    worst = ((got.double() - want).abs() / bound).nan_to_num(nan=math.inf).max().item()
    assert worst <= 1.0, (what, worst)


CASES = [  # type, B, H, Hk, N, D, layout, channels, axes, order
    ("bf16", 1, 1, 1, 1, 64, "halves", 64, 1, "heads"),
    ("bf16", 3, 5, 2, 1, 128, "pairs", 128, 1, "heads"),
    ("f16", 2, 4, 1, 17, 128, "halves", 128, 1, "tokens"),
    ("f32", 2, 3, 3, 33, 64, "halves", 32, 1, "packed"),
    ("bf16", 1, 2, 0, 70, 96, "halves", 24, 1, "heads"),
    ("f16", 2, 3, 1, 31, 16, "pairs", 6, 1, "tokens"),
    ("f32", 1, 7, 2, 16, 256, "halves", 256, 1, "heads"),
    ("bf16", 2, 24, 24, 257, 128, "pairs", 128, 3, "tokens"),
    ("f16", 1, 3, 1, 5, 48, "halves", 48, 3, "packed"),
    ("f32", 1, 2, 2, 9, 80, "pairs", 0, 1, "heads"),
    ("bf16", 1, 40, 8, 1500, 64, "halves", 64, 1, "heads"),
]


@pytest.mark.parametrize("kind,B,H,Hk,N,D,layout,channels,axes,order", CASES)
def test_forward_and_backward(kind, B, H, Hk, N, D, layout, channels, axes, order):
    gen = torch.Generator(device=DEV).manual_seed(7 * N + D)
    amplitude = 1.2079 if channels else 1.0
    rotary, angle = rotary_of(layout, channels, axes, B, N, gen, amplitude=amplitude)
    q, k = make((B, H, N, D), kind, order, gen, 1.7), make((B, Hk, N, D), kind, order, gen) if Hk else None
    gains = [torch.randn(D, generator=gen, device=DEV) for _ in range(2)]
    size = lambda x: plain.pair_size(x, channels, layout, amplitude)
    # the rotation alone, and transposed
    for back in (False, True):
        got = binding.rapid3_rotary(q, k, rotary, backward=back)
        for name, x, z in zip("qk", (q, k), got):
            if x is not None:
                close(z, plain.turn(x.double(), -angle if back else angle, layout, amplitude), size(x.double()), (name, back))
    # behind the norm
    got = binding.rapid3_norm_rotary(q, k, gains[0], gains[1] if Hk else None, 1e-5, rotary)
    for name, x, z, g in zip("qk", (q, k), got, gains):
        if x is not None:
            y = plain.norm(x.double(), g.double(), 1e-5)
            close(z, plain.turn(y, angle, layout, amplitude), size(y), ("norm", name))
    # gradients: a result is a difference of two terms, whose magnitudes are added up for the bound
    d = [make((B, H, N, D), kind, order, gen, 0.3), make((B, Hk, N, D), kind, order, gen, 0.3) if Hk else None]
    dq, dk, dgq, dgk = binding.rapid3_norm_rotary_backward(d[0], d[1], q, k, gains[0], gains[1] if Hk else None, 1e-5, rotary)
    for name, x, dz, gain, dx, dgain in zip("qk", (q, k), d, gains, (dq, dk), (dgq, dgk)):
        if x is None:
            assert dx is None
            continue
        x, gain = x.double(), gain.double()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)
        g, gs = plain.turn(dz.double(), -angle, layout, amplitude), size(dz.double())
        u = x * r
        want = r * (g * gain - u * (g * gain * u).mean(-1, keepdim=True))
        # the mean of D products: each off by 2 FP32 of its size, 12 roundings in its sum
        magnitude = r * (gs * gain.abs() + u.abs() * 4 * (gs * gain.abs() * u.abs()).mean(-1, keepdim=True))
        close(dx, want, magnitude, ("gradient", name))
        # terms off by 2 FP32, and a lane's sum of at most 2^8 rows (2^-16), fixed trees behind it
        terms = (gs * u.abs()).sum((0, 1, 2))
        assert ((dgain.double() - (g * u).sum((0, 1, 2))).abs() <= 2.0 ** -15 * terms + 1e-30).all(), ("gain", name)


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_gradients_against_differences(layout):
    """The kernel's gradients along a direction against central differences of the 64-bit forward form."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    B, H, N, D = 2, 3, 19, 64
    rotary, angle = rotary_of(layout, 32, 1, B, N, gen)
    x, w = make((B, H, N, D), "f32", "heads", gen), make((B, H, N, D), "f32", "heads", gen)
    gain = torch.rand(D, generator=gen, device=DEV) + 0.5
    dx, _, dgain, _ = binding.rapid3_norm_rotary_backward(w, None, x, None, gain, None, 1e-6, rotary)
    loss = lambda a, b: (w.double() * plain.turn(plain.norm(a, b, 1e-6), angle, layout)).sum().item()
    along, along_gain, step = torch.randn(x.shape, generator=gen, device=DEV).double(), torch.randn(D, generator=gen, device=DEV).double(), 1e-5
    X, G = x.double(), gain.double()
    for got, size, there, back in (((dx.double() * along).sum(), (dx.double() * along).abs().sum(), loss(X + step * along, G), loss(X - step * along, G)),
                                   ((dgain.double() * along_gain).sum(), (dgain.double() * along_gain).abs().sum(),
                                    loss(X, G + step * along_gain), loss(X, G - step * along_gain))):
        # fp32 gradients: 2^-15 of the summands; the differences' own error is third order, 1e-10, and 1e-16 |loss| / step
        assert abs(got.item() - (there - back) / (2 * step)) <= 2.0 ** -15 * size.item() + 1e-6


def test_in_place_and_positions_from_an_offset():
    gen = torch.Generator(device=DEV).manual_seed(5)
    q, k = make((2, 4, 37, 128), "bf16", "tokens", gen), make((2, 2, 37, 128), "bf16", "tokens", gen)
    freq, amplitude = binding.rapid3_rotary_freqs(128, 10000.0, "parts", 8.0, 4096)
    by_offset = binding.Rotary("halves", freq.to(DEV), pos0=(1 << 30) - 37, amplitude=amplitude)
    pos = torch.arange((1 << 30) - 37, 1 << 30, device=DEV, dtype=torch.int32).view(1, 37, 1)
    by_list = binding.Rotary("halves", freq.to(DEV), pos, amplitude=amplitude)
    want = binding.rapid3_rotary(q, k, by_list)
    for z, x in zip(want, (q, k)):
        close(z, plain.turn(x.double(), plain.angles(freq.to(DEV), pos, [64]), "halves", amplitude), plain.pair_size(x.double(), 128, "halves", amplitude), "far")
    binding.rapid3_rotary(q, k, by_offset, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_backward_in_place_and_twice_the_same_bits():
    gen = torch.Generator(device=DEV).manual_seed(6)
    q, d = make((2, 24, 700, 64), "bf16", "heads", gen), make((2, 24, 700, 64), "bf16", "heads", gen)
    gain = torch.rand(64, generator=gen, device=DEV)
    rotary, _ = rotary_of("pairs", 64, 1, 2, 700, gen)
    first = binding.rapid3_norm_rotary_backward(d, None, q, None, gain, None, 1e-6, rotary)
    again = binding.rapid3_norm_rotary_backward(d, None, q, None, gain, None, 1e-6, rotary)
    assert torch.equal(first[0], again[0]) and torch.equal(first[2], again[2])
    binding.rapid3_norm_rotary_backward(d, None, q, None, gain, None, 1e-6, rotary, dq=d)
    assert torch.equal(d, first[0])


def test_rows_beyond_32_bits():
    """Heads 2^31 + 64 elements apart: offsets in bytes and in elements pass 32 bits."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    apart = (1 << 31) + 64
    buffer = torch.empty(2 * apart, dtype=torch.bfloat16, device=DEV)
    q = buffer.as_strided((1, 2, 20, 64), (2 * apart, apart, 64, 1))
    x = torch.randn((1, 2, 20, 64), generator=gen, device=DEV).to(torch.bfloat16)
    q.copy_(x)
    rotary, angle = rotary_of("halves", 64, 1, 1, 20, gen)
    out, _ = binding.rapid3_rotary(x, None, rotary)
    binding.rapid3_rotary(q, None, rotary, q)
    assert torch.equal(q, out)


def test_captured_and_on_another_stream():
    """Two captured graphs, replayed in turn on inputs and positions refilled in place, and an eager call on a stream of its own."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    q, d = make((1, 8, 300, 128), "f16", "heads", gen), make((1, 8, 300, 128), "f16", "heads", gen)
    gain = torch.rand(128, generator=gen, device=DEV)
    rotary, _ = rotary_of("halves", 128, 1, 1, 300, gen)
    binding.rapid3_norm_rotary_backward(d, None, q, None, gain, None, 1e-6, rotary)
    got, graphs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(binding.rapid3_norm_rotary_backward(d, None, q, None, gain, None, 1e-6, rotary))
        graphs.append(g)
    q.copy_(make((1, 8, 300, 128), "f16", "heads", gen))
    rotary.pos.add_(17)
    for g in graphs + graphs:
        g.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = binding.rapid3_norm_rotary_backward(d, None, q, None, gain, None, 1e-6, rotary)
    torch.cuda.synchronize()
    for x in got:
        assert torch.equal(x[0], want[0]) and torch.equal(x[2], want[2])


def test_refusals_of_the_binding():
    gen = torch.Generator(device=DEV).manual_seed(1)
    q, k = make((1, 2, 4, 64), "bf16", "heads", gen), make((1, 1, 4, 64), "bf16", "heads", gen)
    rotary, _ = rotary_of("halves", 64, 1, 1, 4, gen)
    gain = torch.ones(64, device=DEV)
    binding.rapid3_norm_rotary(q, k, gain, gain, 1e-6, rotary)
    for bad in (dict(q=q.cpu()), dict(k=k.half()), dict(k=k[..., :32]), dict(q=q[:, :, :3]), dict(q=q.double()), dict(q_gain=gain.double()),
                dict(k_gain=gain[:32]), dict(k_gain=None), dict(q_out=torch.empty_like(k)), dict(q=q[..., ::2]),
                dict(rotary=rotary_of("halves", 64, 1, 3, 4, gen)[0])):
        args = dict(q=q, k=k, q_gain=gain, k_gain=gain, eps=1e-6, rotary=rotary) | bad
        with pytest.raises(ValueError):
            binding.rapid3_norm_rotary(**args)
    for bad in (dict(eps=-1.0), dict(rotary=binding.Rotary("halves", rotary.freq.repeat(2), rotary.pos)),
                dict(q=torch.zeros(257, dtype=torch.bfloat16, device=DEV)[1:].view(1, 1, 4, 64), k=None, k_gain=None),
                dict(q=q[:, :, :1].expand(-1, -1, 4, -1))):
        args = dict(q=q, k=k, q_gain=gain, k_gain=gain, eps=1e-6, rotary=rotary) | bad
        with pytest.raises(binding.Rapid3Error):
            binding.rapid3_norm_rotary(**args)
