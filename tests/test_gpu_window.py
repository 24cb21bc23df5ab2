"""rapid3_window_attn and rapid3_window_attn_backward on the GPU against the plain 64-bit forms, head by head."""
import math

import pytest
import torch

from paper_2509_22323_b200 import binding
from tests.window_cases import DEV, Case

pytestmark = pytest.mark.gpu

PROMPTS = [  # type, B, H, Hkv, D, n_q, n_kv, left, right, sink, full, q_len, kv_len, order
    ("bf16", 1, 1, 1, 64, 17, 17, -1, -1, 0, 0, None, None, "heads"),                    # everything visible, one ragged tile
    ("bf16", 1, 2, 2, 128, 64, 64, -1, 0, 0, 0, None, None, "heads"),                    # causal
    ("f16", 1, 4, 2, 128, 200, 200, 63, 0, 4, 0, None, None, "tokens"),                  # causal window and sinks, pairs of heads
    ("bf16", 2, 3, 3, 64, 321, 321, 64, 64, 65, 65, None, None, "packed"),               # joint: text rows see everything
    ("f16", 2, 3, 1, 64, 300, 300, 0, 0, 0, 0, None, None, "heads"),                     # every row sees itself alone
    ("bf16", 1, 6, 2, 128, 129, 700, 100, 0, 70, 0, None, None, "heads"),                # the last rows of a longer sequence
    ("bf16", 3, 4, 1, 64, 257, 190, 50, 0, 3, 0, [257, 130, 190], [190, 190, 5], "heads"),   # more rows than keys: the first see nothing
    ("f16", 4, 2, 2, 128, 130, 260, 31, 7, 0, 0, [130, 0, 1, 64], [260, 260, 0, 65], "tokens"),  # lengths of zero and one
    ("bf16", 2, 8, 4, 64, 100, 1000, 127, 0, 1, 0, [100, 37], [777, 64], "packed"),
    ("bf16", 1, 2, 1, 128, 400, 400, -1, 30, 0, 0, None, None, "heads"),                 # bounded on the right alone
    ("f16", 1, 2, 1, 64, 400, 400, 30, -1, 0, 10, None, None, "heads"),                  # bounded on the left alone
    ("bf16", 1, 2, 2, 64, 260, 260, 20, 0, 200, 0, None, None, "heads"),                 # first tokens that reach into the window
    ("bf16", 1, 2, 2, 64, 260, 260, 20, 0, 1 << 30, 0, None, None, "heads"),             # as good as causal
    ("f16", 1, 2, 2, 128, 150, 150, (1 << 31) - 1, (1 << 31) - 1, 0, 0, None, None, "heads"),    # bounds beyond any length
    ("bf16", 2, 2, 2, 128, 150, 150, 40, 3, 2, 1 << 30, [150, 99], [150, 150], "heads"), # every row is full
    ("bf16", 2, 40, 8, 64, 500, 500, 99, 0, 4, 0, None, None, "heads"),                  # several units for each thread block
    ("f16", 3, 20, 4, 128, 650, 650, 200, 200, 64, 64, [650, 649, 1], [650, 649, 1], "tokens"),
    ("bf16", 2, 39, 13, 128, 300, 300, 80, 0, 0, 0, None, None, "heads"),                # an odd number of heads for each key head: 256 rows a unit
    ("bf16", 1, 39, 13, 64, 1500, 1500, 300, 0, 10, 0, [1400], [1450], "heads"),
    ("f16", 1, 16, 1, 128, 1100, 1100, 99, 0, 4, 0, None, None, "heads"),                # gradients: many units for the one tile of first tokens
    ("bf16", 2, 32, 1, 64, 900, 1000, 40, 5, 130, 0, [900, 60], [1000, 140], "tokens"),  # and for two, of sequences that fill few of them
]


def prompt(case):
    *args, order = case
    c = Case(*args, order=order)
    out, lse = c.fresh(c.H, c.n_q), torch.full((c.B, c.H, c.n_q), 77.0, device=DEV)
    binding.rapid3_window_attn(c.q, c.k, c.v, out, lse, **c.rule)
    return c, out, lse


@pytest.mark.parametrize("case", PROMPTS)
def test_prompt(case):
    c, out, lse = prompt(case)
    assert binding.rapid3_window_status() == 0
    c.check(out, lse)


@pytest.mark.parametrize("case", PROMPTS)
def test_gradients(case):
    c, out, lse = prompt(case)
    grads = c.fresh(c.H, c.n_q), c.fresh(c.Hkv, c.n_kv), c.fresh(c.Hkv, c.n_kv)
    binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, *grads, **c.rule)
    assert binding.rapid3_window_status() == 0
    c.check(out, lse, grads)


TOKENS = [
    ("bf16", 1, 1, 1, 64, 1, 1, 0, 0, 0, 0, None, None, "heads"),
    ("f16", 2, 8, 2, 128, 1, 100, 15, 0, 4, 0, None, [100, 3], "heads"),
    ("bf16", 3, 16, 1, 128, 1, 999, 127, 0, 1, 0, None, [999, 0, 128], "tokens"),        # one sequence has no key
    ("bf16", 2, 6, 2, 64, 5, 333, 40, 0, 7, 0, [5, 2], [333, 1], "packed"),              # several rows, some before the first key
    ("f16", 1, 4, 4, 64, 16, 16, -1, 0, 0, 0, None, None, "heads"),
    ("bf16", 1, 8, 1, 128, 2, 5000, -1, -1, 0, 0, None, None, "heads"),                  # a cluster of thread blocks for each key head
    ("f16", 1, 8, 8, 64, 1, 40000, -1, 0, 0, 0, None, [39990], "heads"),
    ("bf16", 2, 32, 8, 128, 1, 3000, 1023, 0, 4, 0, None, [3000, 1500], "heads"),
    ("bf16", 2, 4, 2, 64, 3, 300, 9, 2, 20, 290, [3, 3], [300, 292], "heads"),           # full rows among them
    ("bf16", 64, 16, 8, 128, 1, 200, 90, 0, 0, 0, None, None, "tokens"),
]


@pytest.mark.parametrize("case", TOKENS)
def test_tokens(case):
    c, out, lse = prompt(case)
    c.check(out, lse)


@pytest.mark.parametrize("case", [TOKENS[0], TOKENS[3], TOKENS[8]])
def test_gradients_of_few_rows(case):
    c, out, lse = prompt(case)
    grads = c.fresh(c.H, c.n_q), c.fresh(c.Hkv, c.n_kv), c.fresh(c.Hkv, c.n_kv)
    binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, *grads, **c.rule)
    assert binding.rapid3_window_status() == 0
    c.check(out, lse, grads)


@pytest.mark.parametrize("n_q", [1, 300])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_scores_that_rise_along_the_keys(kind, n_q):
    """The running maximum moves again and again: scores from about -100 to 100, peaked weights."""
    c = Case(kind, 1, 2, 2, 64, n_q, 1200, -1, 0, 0, 0, spread=1.0, scale=1.0)
    c.k.copy_(c.k * 0.1 + torch.linspace(-1, 1, 1200, device=DEV)[:, None])
    c.q.copy_(c.q * 0.1 + 1.0)
    out, lse = c.fresh(2, n_q), torch.full((1, 2, n_q), 77.0, device=DEV)
    binding.rapid3_window_attn(c.q, c.k, c.v, out, lse, **c.rule)
    import tests.window_cases as wc
    was = wc.S
    wc.S = 2.0 ** -12                                                # scores up to 2^7, sums of 64 of 2 each: 2^-23 * 2^7 * 8
    try:
        c.check(out, lse)
    finally:
        wc.S = was


def test_gradients_against_differences():
    """dq along a direction against differences of the 64-bit loss; so far from rounded weights that 16 bits allow."""
    from tests import plain_operators as plain
    c, out, lse = prompt(("f16", 1, 2, 1, 64, 90, 90, 30, 0, 2, 0, None, None, "heads"))
    dq, dk, dv = binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, **c.rule)
    w = c.dout[0].double()
    loss = lambda q, k, v: sum((w[h] * plain.attention(q[h], k, v, c.seen[0], c.scale)[0]).sum() for h in range(2)).item()
    args = [c.q[0].double(), c.k[0, 0].double(), c.v[0, 0].double()]
    for i, g in enumerate((dq[0], dk[0, 0], dv[0, 0])):
        along = torch.randn(g.shape, generator=c.gen, device=DEV).double()
        step = [x + 1e-5 * along if j == i else x for j, x in enumerate(args)], [x - 1e-5 * along if j == i else x for j, x in enumerate(args)]
        want = (loss(*step[0]) - loss(*step[1])) / 2e-5
        # every element of the gradient is off by a few half steps of it and of its summands: 8 h of the magnitudes, of random signs
        assert abs((g.double() * along).sum().item() - want) <= 8 * 2.0 ** -11 * (g.double() * along).norm().item() + 1e-5


def test_twice_the_same_bits_and_shared_layouts():
    """The same call twice; and Q, K, V as views of one packed projection with gradients into one packed tensor."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    B, N, H, Hkv, D = 2, 500, 8, 2, 128
    packed = torch.randn((B, N, H + 2 * Hkv, D), generator=gen, device=DEV).to(torch.bfloat16)
    views = lambda t: (t[:, :, :H].transpose(1, 2), t[:, :, H:H + Hkv].transpose(1, 2), t[:, :, H + Hkv:].transpose(1, 2))
    q, k, v = views(packed)
    rule = dict(left=100, right=0, n_sink=3)
    out = torch.empty((B, N, H, D), dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    lse = torch.empty((B, H, N), device=DEV)
    dout = torch.randn((B, N, H, D), generator=gen, device=DEV).to(torch.bfloat16).transpose(1, 2)
    binding.rapid3_window_attn(q, k, v, out, lse, **rule)
    grads = [torch.empty_like(packed) for _ in range(2)]
    for g in grads:
        binding.rapid3_window_attn_backward(q, k, v, out, lse, dout, *views(g), **rule)
    assert torch.equal(*grads)
    apart = [x.contiguous() for x in (q, k, v)]
    out2, lse2 = binding.rapid3_window_attn(*apart, None, torch.empty_like(lse), **rule)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    for a, b in zip(binding.rapid3_window_attn_backward(*apart, out2, lse2, dout.contiguous(), **rule), views(grads[0])):
        assert torch.equal(a, b)


def test_captured_with_lengths_that_change_and_two_streams():
    """A training pass captured twice; lengths and inputs are refilled in place, the graphs replayed in turn, and eager calls run on two
    streams beside one another."""
    c = Case("bf16", 2, 8, 2, 64, 400, 400, 90, 0, 4, 0, [400, 300], [400, 350])
    run = lambda: (lambda o: o + binding.rapid3_window_attn_backward(c.q, c.k, c.v, o[0], o[1], c.dout, **c.rule))(
        binding.rapid3_window_attn(c.q, c.k, c.v, None, torch.zeros((2, 8, 400), device=DEV), **c.rule))
    run()
    graphs, got = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(run())
        graphs.append(g)
    for t in (c.q, c.k, c.v, c.dout):
        t.copy_(torch.randn(t.shape, generator=c.gen, device=DEV))
    lens = [[250, 17], [399, 17]]
    c.rule["q_len"].copy_(torch.tensor(lens[0]))
    c.rule["kv_len"].copy_(torch.tensor(lens[1]))
    for g in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    streams, eager = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            eager.append(run())
    torch.cuda.synchronize()
    assert binding.rapid3_window_status() == 0
    for other in got[1:] + eager:
        for x, y in zip(got[0], other):
            for b in range(2):
                n = lens[1 if x.shape[1] == 2 else 0][b]
                assert torch.equal(x[b, :, :n], y[b, :, :n])


def test_a_cache_beyond_32_bits():
    """Key heads 2^31 + 64 elements apart, for single tokens and for a prompt."""
    apart = (1 << 31) + 64
    for n_q in (1, 100):
        c = Case("bf16", 1, 4, 2, 64, n_q, 300, 99, 0, 4, 0)
        far = []
        for x in (c.k, c.v):
            buffer = torch.empty(apart + 300 * 64, dtype=torch.bfloat16, device=DEV)
            far.append(buffer.as_strided((1, 2, 300, 64), (2 * apart, apart, 64, 1)))
            far[-1].copy_(x)
        out, lse = c.fresh(4, n_q), torch.full((1, 4, n_q), 77.0, device=DEV)
        binding.rapid3_window_attn(c.q, *far, out, lse, **c.rule)
        c.check(out, lse)


def test_together_as_a_block_uses_them():
    """Raw projections, normed and turned, into the windowed attention, and all the way back: against the 64-bit chain.  Then the same
    Q and K through the block-sparse step of the library at ratio 1, whose dense attention is the window without bounds."""
    from tests import plain_operators as plain
    gen = torch.Generator(device=DEV).manual_seed(12)
    H, N, D, text = 2, 320, 64, 64
    raw = [torch.randn((1, H, N, D), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(3)]
    dout = torch.randn((1, H, N, D), generator=gen, device=DEV).to(torch.bfloat16)
    gains = [torch.rand(D, generator=gen, device=DEV) + 0.5 for _ in range(2)]
    freq, _ = binding.rapid3_rotary_freqs(D)
    pos = torch.arange(N, device=DEV, dtype=torch.int32).view(1, N, 1)
    rotary = binding.Rotary("halves", freq.to(DEV), pos)
    rule = dict(left=64, right=64, n_sink=text, n_full=text)
    q, k = binding.rapid3_norm_rotary(raw[0], raw[1], *gains, 1e-6, rotary)
    out, lse = binding.rapid3_window_attn(q, k, raw[2], None, torch.empty((1, H, N), device=DEV), **rule)
    dq, dk, dv = binding.rapid3_window_attn_backward(q, k, raw[2], out, lse, dout, **rule)
    draw = binding.rapid3_norm_rotary_backward(dq, dk, raw[0], raw[1], *gains, 1e-6, rotary)
    seen = plain.visible(N, N, 64, 64, text, text, N, N).to(DEV)
    leaves = [x.double().requires_grad_() for x in raw + gains]
    angle = plain.angles(freq.to(DEV), pos, [D // 2])
    with torch.enable_grad():
        Q, K = (plain.turn(plain.norm(x, g, 1e-6), angle, "halves") for x, g in ((leaves[0], leaves[3]), (leaves[1], leaves[4])))
        O = torch.softmax((Q @ K.transpose(-1, -2) * D ** -0.5).masked_fill(~seen, -math.inf), -1) @ leaves[2]
        want = torch.autograd.grad(O, leaves, dout.double())
    # each step rounds once, relative to itself; errors of random signs pass on: within 6 half steps in the norm
    for got, x in [(out, O.detach()), (dv, want[2]), (draw[0], want[0]), (draw[1], want[1]), (draw[2], want[3]), (draw[3], want[4])]:
        assert ((got.double() - x).norm() / x.norm()).item() <= 6 * 2.0 ** -8
    ctx = binding.Context(1, H, D, text, N - text)
    dense = ctx.rapid3_gated_step(q, k, raw[2], torch.zeros_like(q), [binding.ACT_ATTEND], [1.0])
    free, _ = binding.rapid3_window_attn(q, k, raw[2])
    # both round weights and results once: two half steps of each, of magnitudes below 4
    assert (dense.double() - free.double()).abs().max().item() <= 4 * 4 * 2.0 ** -8 * 0.5


def test_refusals_of_the_binding():
    c = Case("bf16", 1, 4, 2, 64, 20, 30, 5, 0, 0, 0, [20], [30])
    out, lse = binding.rapid3_window_attn(c.q, c.k, c.v, None, torch.empty((1, 4, 20), device=DEV), **c.rule)
    for bad in (dict(q=c.q.cpu()), dict(k=c.k.half()), dict(v=c.v[:, :, :29]), dict(q=c.q.float()), dict(out=out[:, :2]), dict(k=c.k[:, :, :, :32]),
                dict(lse=lse.half()), dict(lse=lse[:, :, :10]), dict(q_len=c.rule["q_len"].long()), dict(kv_len=c.rule["kv_len"].cpu()),
                dict(kv_len=c.rule["kv_len"].repeat(2))):
        args = dict(q=c.q, k=c.k, v=c.v, out=out, lse=lse, **c.rule) | bad
        with pytest.raises(ValueError):
            binding.rapid3_window_attn(**args)
    wide = torch.zeros((1, 4, 20, 96), dtype=torch.bfloat16, device=DEV)
    for bad in (dict(left=-2), dict(right=-2), dict(n_sink=-1), dict(n_full=-1), dict(softmax_scale=0.0), dict(softmax_scale=math.inf),
                dict(k=c.k[:, :1].expand(-1, 2, -1, -1)), dict(k=c.k.repeat(1, 2, 1, 1)[:, :3], v=c.v.repeat(1, 2, 1, 1)[:, :3]),
                dict(q=wide, k=wide, v=wide, out=wide)):
        args = dict(q=c.q, k=c.k, v=c.v, out=out, lse=lse, **c.rule) | bad
        with pytest.raises(binding.Rapid3Error):
            binding.rapid3_window_attn(**args)
    with pytest.raises(ValueError):
        binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, None, c.dout, **c.rule)


ONE_KEY = [  # D, n_q, n_kv, left, right, sink, full, q_len, kv_len: every row sees one key
    (64, 1, 1, -1, 0, 0, 0, None, None),
    (128, 1, 1, 20, 20, 256, 256, None, None),
    (64, 300, 300, 0, 0, 0, 0, None, None),
    (128, 300, 300, 0, 0, 0, 0, None, None),
    (64, 200, 400, -1, -1, 0, 0, [200, 130], [1, 1]),
    (128, 200, 400, -1, -1, 0, 0, [200, 130], [1, 1]),
]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,n_q,n_kv,left,right,sink,full,q_len,kv_len", ONE_KEY)
def test_rows_that_see_one_key_have_no_gradient_of_scores(kind, D, n_q, n_kv, left, right, sink, full, q_len, kv_len):
    """The weight of a single key is 1 whatever its score: dq and dk are exactly zero, dv is the sum of dout."""
    c = Case(kind, 2, 4, 2, D, n_q, n_kv, left, right, sink, full, q_len, kv_len)
    assert all((s.sum(-1) == 1).all() for s in c.seen)
    out, lse = c.fresh(4, n_q), torch.full((2, 4, n_q), 77.0, device=DEV)
    binding.rapid3_window_attn(c.q, c.k, c.v, out, lse, **c.rule)
    grads = c.fresh(4, n_q), c.fresh(2, n_kv), c.fresh(2, n_kv)
    binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, *grads, **c.rule)
    assert binding.rapid3_window_status() == 0
    for b, (r, n) in enumerate(c.lens):
        assert (grads[0][b, :, :r] == 0).all() and (grads[1][b, :, :n] == 0).all()
    c.check(out, lse, grads)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,left,sink", [(20, -1, 0), (41, 186, 4), (300, 15, 0), (900, -1, 0)])
def test_gradients_where_rows_see_few_keys(D, N, left, sink):
    """dq and dk are off by the rounding of dS and their own, of random signs, and by no more: a rounding to nearest is off by
    h sqrt(E[1 / m^2] / 3) = 0.425 h in the mean square, m the mantissa, evenly spread in its logarithm; two of them by 0.60 h; a tenth is left
    for what is not spread so.  (With delta from the rounded output alone it is 0.66 to 0.78 h here.)"""
    from tests import plain_operators as plain
    c = Case("bf16", 4, 8, 4, D, N, N, left, 0, sink, 0)
    out, lse = binding.rapid3_window_attn(c.q, c.k, c.v, None, torch.empty((4, 8, N), device=DEV), **c.rule)
    dq, dk, _ = binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, **c.rule)
    off, size = [0.0, 0.0], [0.0, 0.0]
    for b in range(4):
        for hk in range(4):
            k, v, want_dk = c.k[b, hk].double(), c.v[b, hk].double(), 0.0
            for h in (2 * hk, 2 * hk + 1):
                q, d = c.q[b, h].double(), c.dout[b, h].double()
                o, _, p = plain.attention(q, k, v, c.seen[b], c.scale)
                g = plain.attention_gradients(q, k, v, o, p, d, c.scale)
                off[0] += (dq[b, h].double() - g[0]).square().sum().item()
                size[0] += g[0].square().sum().item()
                want_dk = want_dk + g[1]
            off[1] += (dk[b, hk].double() - want_dk).square().sum().item()
            size[1] += want_dk.square().sum().item()
    for x, y in zip(off, size):
        assert math.sqrt(x / y) <= 1.1 * math.sqrt(2) * 0.4246 * 2.0 ** -8, math.sqrt(x / y) * 2 ** 8


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("what", [math.inf, -math.inf])
def test_infinities_behind_the_lengths(D, what):
    c = Case("bf16", 3, 4, 2, D, 200, 210, 60, 0, 3, 0, [200, 131, 64], [210, 131, 65])
    for b, (r, n) in enumerate(c.lens):
        for t, m in ((c.q, r), (c.dout, r), (c.k, n), (c.v, n)):
            t[b, :, m:] = what
    out, lse = c.fresh(4, 200), torch.full((3, 4, 200), 77.0, device=DEV)
    binding.rapid3_window_attn(c.q, c.k, c.v, out, lse, **c.rule)
    grads = c.fresh(4, 200), c.fresh(2, 210), c.fresh(2, 210)
    binding.rapid3_window_attn_backward(c.q, c.k, c.v, out, lse, c.dout, *grads, **c.rule)
    assert binding.rapid3_window_status() == 0
    c.check(out, lse, grads)


FIRST = '''
import torch
from paper_2509_22323_b200 import binding as b
q, k = torch.randn(2, 4, 200, {D}, device="cuda").half(), torch.randn(2, 2, 200, {D}, device="cuda").half()
v, one, gain = torch.randn_like(k), torch.randn_like(q[:, :, :1]).contiguous(), torch.ones({D}, device="cuda")
lse, dout = torch.zeros(2, 4, 200, device="cuda"), torch.randn_like(q)
rot = b.Rotary("halves", b.rapid3_rotary_freqs({D})[0].cuda())
s = torch.cuda.Stream()
s.wait_stream(torch.cuda.current_stream())
def run():
    o, _ = b.rapid3_window_attn(q, k, v, None, lse, left=50, right=0, n_sink=2)
    g = b.rapid3_window_attn_backward(q, k, v, o, lse, dout, left=50, right=0, n_sink=2)
    t, _ = b.rapid3_window_attn(one, k, v, left=50, right=0)
    return (o, t) + g + b.rapid3_norm_rotary(q, k, gain, gain, 1e-6, rot) + b.rapid3_norm_rotary_backward(g[0], g[1], q, k, gain, gain, 1e-6, rot)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=s):
    got = run()
graph.replay()
torch.cuda.synchronize()
assert b.rapid3_window_status() == 0
for x, y in zip(got, run()):
    assert torch.equal(x, y)
print("the same")
'''


@pytest.mark.parametrize("D", [64, 128])
def test_the_first_calls_of_a_process_are_captured(D):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST.format(D=D)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stderr[-2000:]
