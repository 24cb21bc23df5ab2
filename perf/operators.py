"""The operators of an attention block beside the block-sparse attention: what is measured of them, and their plain forms.

  rotary   rotary positions of Q and K heads (adjacent pairs or halves, all of a head or its first channels, frequencies as given)
  norm     RMS normalisation of each Q and K head with a gain, and the rotation, in the same pass; forward or backward
  window   attention with a sliding window and first tokens that every row sees; forward, one training pass, single tokens

A case is a dict of plain values:

  kind     "rotary", "norm", "norm_backward", "window", "window_train" or "window_token"
  type     "bf16", "f16" or "f32": of the tensors (gains, frequencies and statistics have types of their own)
  B, H, Hkv, D   sequences, query heads, key (and value) heads, head dimension
  N        tokens of a sequence ("window_token": places of the cache)
  ragged   sequences of different lengths, in tensors of N places
  rotary and norm:  layout "pairs" | "halves", rot channels turned, axes coordinates of a position (1 or 3), far the largest position,
           order "heads" [B, H, N, D] | "tokens" views of [B, N, H, D]
  window:  left, right (-1: no bound), sinks, full (rows at the first `full` positions see every key)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def _rot(name, kind, type, B, H, Hkv, D, N, layout, rot, axes, far, order="heads"):
    case = {"name": name} if name else {}
    case.update(kind=kind, type=type, B=B, H=H, Hkv=Hkv, D=D, N=N, layout=layout, rot=rot, axes=axes, far=far, order=order)
    return case


def _win(name, kind, type, B, H, Hkv, D, N, left, right, sinks, full, ragged):
    case = {"name": name} if name else {}
    case.update(kind=kind, type=type, B=B, H=H, Hkv=Hkv, D=D, N=N, left=left, right=right, sinks=sinks, full=full, ragged=ragged)
    return case


def listed():
    return [
        # one new token of each of 64 sequences of very different lengths: all latency and the launch
        _rot("rotary_tokens", "rotary", "bf16", 64, 32, 8, 128, 1, "halves", 128, 1, 120000),
        # prompts in full precision, of whose heads only the first half is turned; an odd length, token by token as a projection leaves it
        _rot("rotary_part_f32", "rotary", "f32", 2, 16, 16, 64, 2047, "halves", 32, 1, 4096, "tokens"),
        # Q and K of three joint sequences of 512 text and 64 x 64 image tokens, with positions of three coordinates
        _rot("norm_joint", "norm", "bf16", 3, 24, 24, 128, 4608, "pairs", 128, 3, 64),
        # the same step for two new tokens' heads with shared key heads: latency
        _rot("norm_tokens", "norm", "bf16", 2, 32, 8, 128, 1, "halves", 128, 1, 30000),
        # fine-tuning a joint block of 333 text and 64 x 64 image tokens: the gradients of the raw projections and of the gains
        _rot("norm_backward_joint", "norm_backward", "f16", 2, 24, 24, 64, 4429, "pairs", 64, 3, 64),
        # training on one long sequence with shared key heads, token by token
        _rot("norm_backward_shared", "norm_backward", "bf16", 1, 32, 8, 128, 8191, "halves", 128, 1, 8192, "tokens"),
        # a joint sequence whose image tokens see the text and eight rows of the grid on either side; text rows see everything
        _win("window_joint", "window", "bf16", 1, 24, 24, 128, 4608, 512, 512, 512, 512, False),
        # a prompt, causal, 1024 tokens back and four first tokens, key heads shared by four
        _win("window_prompt_shared", "window", "f16", 1, 32, 8, 128, 8192, 1023, 0, 4, 0, False),
        # a padded batch of short prompts of odd lengths at 64 channels
        _win("window_ragged", "window", "bf16", 4, 16, 4, 64, 1000, 255, 0, 1, 0, True),
        # one training pass through the joint attention of two images of 333 text and 32 x 32 image tokens at 64 channels
        _win("window_train_joint", "window_train", "bf16", 2, 24, 24, 64, 1357, 256, 256, 333, 333, False),
        # one training pass over a causal sequence, key heads shared by four
        _win("window_train_shared", "window_train", "f16", 1, 32, 8, 128, 4095, 1023, 0, 4, 0, False),
        # one new token of each of 64 sequences against long caches, of which 4096 places and four first ones are seen
        _win("window_tokens", "window_token", "bf16", 64, 64, 8, 128, 16384, 4095, 0, 4, 0, True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "norm", "norm_backward", "window", "window_train", "window_token"])
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    H = Hkv * rng.choice([1, 2, 4, 8])
    if kind in ("rotary", "norm", "norm_backward"):
        layout = rng.choice(["pairs", "halves"])
        N, B = _spread(rng, 1, 8000), rng.randint(1, 4)
        axes = rng.choice([1, 1, 3])
        rot = D if axes == 3 or kind == "norm" else rng.choice([D, D // 2, D // 4])
        return _rot(None, kind, rng.choice(["bf16", "f16", "f32"]), B, H, Hkv, D, max(1, N // B), layout, rot, axes,
                    64 if axes == 3 else _spread(rng, 100, 200000), rng.choice(["heads", "tokens"]))
    type = rng.choice(["bf16", "f16"])
    if kind == "window_token":
        N = _spread(rng, 64, 12000)
        return _win(None, kind, type, _spread(rng, 1, 48), H, Hkv, D, N, _spread(rng, 16, 4096) - 1, 0, rng.choice([0, 1, 4, 16]), 0, True)
    H, Hkv = min(H, 32), min(Hkv, 8)
    N = _spread(rng, 1, 4000 if H <= 16 else 2600)
    causal = rng.random() < 0.6
    left = _spread(rng, 16, 1500) - 1
    sinks = rng.choice([0, 1, 4, 77]) if causal else rng.choice([0, 77, 256])
    return _win(None, kind, type, rng.randint(1, 2) if N > 1500 else rng.randint(1, 4), H, Hkv, D, N, left, 0 if causal else left, sinks,
                0 if causal else sinks, rng.random() < 0.4)


# ------------------------------------------------------------------------------------------------ inputs

def _frequencies(c):
    """Radians per position of every turned channel pair, and how many pairs each coordinate turns."""
    pairs = c["rot"] // 2
    if c["axes"] == 3:
        first = pairs // 8
        counts = [first, (pairs - first) // 2, pairs - first - (pairs - first) // 2]
    else:
        counts = [pairs]
    # a long context beyond the trained one slows the frequencies down: a larger base
    base = 500000.0 if c["far"] > 50000 else 10000.0
    freq = torch.cat([torch.tensor([base ** (-i / n) for i in range(n)], dtype=torch.float64) for n in counts])
    return freq, counts


def _positions(c, gen):
    B, N = c["B"], c["N"]
    if c["axes"] == 3:                      # first coordinate unused, then row and column of the image grid; text at (0, 0, 0)
        side = max(1, min(c["far"], math.isqrt(N)))
        text = max(0, N - side * side)
        i = torch.arange(N, device="cuda") - text
        at = torch.stack([torch.zeros_like(i), torch.div(i, side, rounding_mode="floor"), i % side], -1)
        return torch.where(i[:, None] >= 0, at, 0).clamp_(min=0).to(torch.int32)[None].contiguous()
    start = torch.randint(0, max(1, c["far"] - N), (B, 1), generator=gen, device="cuda")
    return (start + torch.arange(N, device="cuda")).to(torch.int32)[..., None].contiguous()


def _tensor(c, gen, H, N, order="heads", scale=1.0):
    shape = (c["B"], N, H, c["D"]) if order == "tokens" else (c["B"], H, N, c["D"])
    t = torch.empty(shape, dtype=TYPES[c["type"]], device="cuda")
    t.normal_(0.0, scale, generator=gen)
    return t.transpose(1, 2) if order == "tokens" else t


def _lengths(c, gen):
    if not c["ragged"]:
        return None
    # at least one sequence fills its places
    n = torch.randint(max(1, c["N"] // 3), c["N"] + 1, (c["B"],), generator=gen, device="cuda")
    n[0] = c["N"]
    return n.to(torch.int32)


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["kind"] in ("rotary", "norm", "norm_backward"):
        for name, H in (("q", c["H"]), ("k", c["Hkv"])):
            s[name] = _tensor(c, gen, H, c["N"], c["order"], 1.3)
            s[name + "_out"] = torch.empty_like(s[name])
            if c["kind"] == "norm_backward":
                s["d" + name] = _tensor(c, gen, H, c["N"], c["order"], 0.1)
            if c["kind"] != "rotary":
                s[name + "_gain"] = 1.0 + 0.2 * torch.randn(c["D"], generator=gen, device="cuda")
                s["d" + name + "_gain"] = torch.empty_like(s[name + "_gain"])
        freq, counts = _frequencies(c)
        s["freq"], s["counts"], s["pos"] = freq.cuda(), counts, _positions(c, gen)
        if own:
            from paper_2509_22323_b200 import binding
            s["rotary"] = binding.Rotary(c["layout"], s["freq"], s["pos"], axis_pairs=counts)
        return s
    rows = 1 if c["kind"] == "window_token" else c["N"]
    s["q"], s["k"], s["v"] = _tensor(c, gen, c["H"], rows), _tensor(c, gen, c["Hkv"], c["N"]), _tensor(c, gen, c["Hkv"], c["N"])
    n = _lengths(c, gen)
    s["kv_len"], s["q_len"] = n, None if rows == 1 else n
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q"].shape[:3], dtype=torch.float32, device="cuda")
    if c["kind"] == "window_train":
        s["dout"] = _tensor(c, gen, c["H"], rows)
        s["dq"], s["dk"], s["dv"] = (torch.zeros_like(s[x]) for x in "qkv")
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls

def _run_own(s):
    from paper_2509_22323_b200 import binding as b
    c = s["case"]
    if c["kind"] == "rotary":
        b.rapid3_rotary(s["q"], s["k"], s["rotary"], s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if c["kind"] == "norm":
        b.rapid3_norm_rotary(s["q"], s["k"], s["q_gain"], s["k_gain"], EPS, s["rotary"], s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if c["kind"] == "norm_backward":
        b.rapid3_norm_rotary_backward(s["dq"], s["dk"], s["q"], s["k"], s["q_gain"], s["k_gain"], EPS, s["rotary"], s["q_out"], s["k_out"],
                                      s["dq_gain"], s["dk_gain"])
        return s["q_out"], s["k_out"], s["dq_gain"], s["dk_gain"]
    seen = dict(left=c["left"], right=c["right"], n_sink=c["sinks"], n_full=c["full"], q_len=s["q_len"], kv_len=s["kv_len"])
    b.rapid3_window_attn(s["q"], s["k"], s["v"], s["out"], s["lse"], **seen)
    if c["kind"] != "window_train":
        return s["out"], s["lse"]
    b.rapid3_window_attn_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], **seen)
    return s["out"], s["lse"], s["dq"], s["dk"], s["dv"]


# ------------------------------------------------------------------------------------------------ the plain forms

def _cos_sin(s):
    """[B or 1, 1, N, pairs]: angles in 64 bits, whose cosine and sine are then held in 32."""
    c = s["case"]
    axis = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(s["counts"])).to("cuda")
    angle = (s["pos"].double()[..., axis] * s["freq"])[:, None]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turn(x, cos, sin, layout, rot):
    if layout == "pairs":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _visible(s, rows, keys):
    """[B or 1, rows, keys] truth values, and [B or 1, rows]: the rows that are there."""
    c = s["case"]
    i, j = torch.arange(rows, device="cuda")[None, :, None], torch.arange(keys, device="cuda")[None, None]
    kv = s["kv_len"][:, None, None].long() if s["kv_len"] is not None else torch.full((1, 1, 1), keys, device="cuda")
    q = s["q_len"][:, None, None].long() if s["q_len"] is not None else torch.full((1, 1, 1), rows, device="cuda")
    at = i + kv - q
    seen = (j >= at - c["left"]) | (j < c["sinks"]) if c["left"] >= 0 else torch.ones_like(j, dtype=torch.bool)
    if c["right"] >= 0:
        seen = seen & (j <= at + c["right"])
    seen = (seen | (at < c["full"])) & (j < kv)
    return seen, (i < q)[..., 0]


def _window(s, q, k, v, seen, there):
    """q: [B, Hkv, group, rows, D] and k, v: [B, Hkv, keys, D] in 32 bits -> the weights, the output and log sum exp."""
    B, Hkv, G, R, D = q.shape
    score = (q.reshape(B, Hkv, G * R, D) @ k.transpose(-1, -2)).mul_(D ** -0.5).view(B, Hkv, G, R, -1)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, 1.0, total))
    out = (p.view(B, Hkv, G * R, -1) @ v).view(B, Hkv, G, R, D)
    return p, torch.where(there[:, None, None, :, None], out, 0.0), torch.where(there[:, None, None], (total.log() + top)[..., 0], 0.0)


def _run_plain(s):
    c = s["case"]
    kind = TYPES[c["type"]]
    if c["kind"] in ("rotary", "norm"):
        cos, sin = _cos_sin(s)
        got = []
        for name in "qk":
            x = s[name].float()
            if c["kind"] == "norm":
                x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s[name + "_gain"]
            got.append(_turn(x, cos, sin, c["layout"], c["rot"]).to(kind))
        return tuple(got)
    if c["kind"] == "norm_backward":
        cos, sin = _cos_sin(s)
        raw, gains = [], []
        for name in "qk":
            x, g = s[name].float(), _turn(s["d" + name].float(), cos, -sin, c["layout"], c["rot"])
            r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
            unit = x * r
            gains.append((g * unit).sum((0, 1, 2)))
            g = g * s[name + "_gain"]
            raw.append(((g - unit * (g * unit).mean(-1, keepdim=True)) * r).to(kind))
        return raw[0], raw[1], gains[0], gains[1]
    B, H, Hkv, D = c["B"], c["H"], c["Hkv"], c["D"]
    q = s["q"].float().view(B, Hkv, H // Hkv, -1, D)
    if c["kind"] == "window_token":
        # the places that the one row sees, gathered: first ones and the window
        n = s["kv_len"].long()[:, None]
        start = (n - 1 - c["left"]).clamp(min=0)
        at = start + torch.arange(c["left"] + 1, device="cuda")
        first = torch.arange(c["sinks"], device="cuda")[None].expand(B, -1)
        seen = torch.cat([first < torch.minimum(start, n), at < n], 1)
        at = torch.cat([first, at], 1).clamp(max=c["N"] - 1)
        k, v = (torch.gather(s[x], 2, at[:, None, :, None].expand(-1, Hkv, -1, D)).float() for x in "kv")
        _, out, lse = _window(s, q, k, v, seen[:, None], torch.ones(1, 1, dtype=torch.bool, device="cuda"))
        return out.view(B, H, 1, D).to(kind), lse.view(B, H, 1)
    k, v = s["k"].float(), s["v"].float()
    seen, there = _visible(s, c["N"], c["N"])
    p, out, lse = _window(s, q, k, v, seen, there)
    outs = (out.view(B, H, -1, D).to(kind), lse.view(B, H, -1))
    if c["kind"] == "window":
        return outs
    R = c["N"]
    d = torch.where(there[:, None, None, :, None], s["dout"].float().view(B, Hkv, H // Hkv, R, D), 0.0)
    dv = p.flatten(2, 3).transpose(-1, -2) @ d.flatten(2, 3)
    dp = (d.flatten(2, 3) @ v.transpose(-1, -2)).view_as(p)
    ds = dp.sub_((d * out).sum(-1, keepdim=True)).mul_(p).mul_(D ** -0.5)
    ds = torch.where(there[:, None, None, :, None], ds, 0.0).flatten(2, 3)
    dq = (ds @ k).view(B, H, R, D)
    dk = ds.transpose(-1, -2) @ q.flatten(2, 3)
    return outs + (dq.to(kind), dk.to(kind), dv.to(kind))


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ work and exact values

def _pairs_seen(c):
    """Visible (row, key) pairs of one head, over all sequences of full length, and keys that some row sees."""
    n = c["N"]
    if c["kind"] == "window_token":
        near = min(n, c["left"] + 1)
        keys = near + min(c["sinks"], n - near)
        return keys * c["B"], keys * c["B"]
    p = np.arange(n, dtype=np.int64)
    hi = np.minimum(n, p + c["right"] + 1) if c["right"] >= 0 else np.full(n, n, dtype=np.int64)
    lo = np.maximum(0, p - c["left"]) if c["left"] >= 0 else np.zeros(n, dtype=np.int64)
    count = hi - lo + np.minimum(lo, c["sinks"])
    count[: c["full"]] = n
    return int(count.sum()) * c["B"], n * c["B"]


def work(case):
    c = case
    if c["kind"] in ("rotary", "norm", "norm_backward"):
        numbers = c["B"] * c["N"] * (c["H"] + c["Hkv"]) * c["D"]
        moved = {"rotary": 2, "norm": 2, "norm_backward": 3}[c["kind"]] * numbers * BYTES[c["type"]]
        at = c["N"] * c["axes"] * 4 * (1 if c["axes"] == 3 else c["B"])
        return {"bytes": moved + at, "flops": {"rotary": 3, "norm": 7, "norm_backward": 14}[c["kind"]] * numbers}
    pairs, keys = _pairs_seen(c)
    q_numbers = c["B"] * c["H"] * (1 if c["kind"] == "window_token" else c["N"]) * c["D"]
    kv_numbers = 2 * keys * c["Hkv"] * c["D"]
    lse = q_numbers // c["D"] * 4
    if c["ragged"]:                          # lengths between a third and all of the places: two thirds of the work, in the mean
        share = 2 / 3 if c["kind"] != "window_token" else 1.0
        pairs, q_numbers, kv_numbers = int(pairs * share), int(q_numbers * share), int(kv_numbers * share)
    if c["kind"] == "window_train":          # q, k, v, dout read; out, dq, dk, dv written
        return {"bytes": (4 * q_numbers + 2 * kv_numbers) * 2 + lse, "flops": 14 * pairs * c["H"] * c["D"]}
    return {"bytes": (2 * q_numbers + kv_numbers) * 2 + lse, "flops": 4 * pairs * c["H"] * c["D"]}


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] in ("rotary", "norm", "norm_backward"):
        axis = [a for a, n in enumerate(s["counts"]) for _ in range(n)]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"][..., axis].double() * s["freq"]).unsqueeze(1)
        half = c["rot"] // 2
        got = {}
        for name in "qk":
            raw = s[name].double().requires_grad_(c["kind"] == "norm_backward")
            gain = s[name + "_gain"].double().requires_grad_(True) if c["kind"] != "rotary" else None
            with torch.enable_grad():
                x = raw if gain is None else raw / (raw.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * gain
                head, rest = x[..., : c["rot"]], x[..., c["rot"]:]
                if c["layout"] == "halves":
                    head = head.unflatten(-1, (2, half)).transpose(-1, -2)
                else:
                    head = head.unflatten(-1, (half, 2))
                z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
                y = torch.cat([(z.transpose(-1, -2) if c["layout"] == "halves" else z).flatten(-2), rest], -1)
            if c["kind"] == "norm_backward":
                got[name] = torch.autograd.grad(y, (raw, gain), s["d" + name].double())
            else:
                got[name] = (y.detach(),)
        return got["q"][:1] + got["k"][:1] + got["q"][1:] + got["k"][1:]
    # one head at a time, row by row of truth values from the definition; gradients by differentiation
    B, H, G, D = c["B"], c["H"], c["H"] // c["Hkv"], c["D"]
    rows, keys = s["q"].shape[2], c["N"]
    train = c["kind"] == "window_train"
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    grads = [torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in "qkv"] if train else []
    for b in range(B):
        kv = int(s["kv_len"][b]) if s["kv_len"] is not None else keys
        nq = int(s["q_len"][b]) if s["q_len"] is not None else rows
        at = torch.arange(nq, device="cuda").unsqueeze(1) + (kv - nq)
        key = torch.arange(kv, device="cuda").unsqueeze(0)
        hidden = torch.zeros((nq, kv), dtype=torch.bool, device="cuda")
        if c["left"] >= 0:
            hidden |= (at - key > c["left"]) & (key >= c["sinks"])
        if c["right"] >= 0:
            hidden |= key - at > c["right"]
        hidden &= at >= c["full"]
        for h in range(H):
            q = s["q"][b, h, :nq].double().requires_grad_(train)
            k, v = (s[x][b, h // G, :kv].double().requires_grad_(train) for x in "kv")
            with torch.enable_grad():
                score = ((q @ k.T) / math.sqrt(D)).masked_fill(hidden, float("-inf"))
                o = torch.softmax(score, -1) @ v
            out[b, h, :nq] = o.detach()
            lse[b, h, :nq] = torch.logsumexp(score.detach(), -1)
            if train:
                g = torch.autograd.grad(o, (q, k, v), s["dout"][b, h, :nq].double())
                grads[0][b, h, :nq] = g[0]
                grads[1][b, h // G, :kv] += g[1]
                grads[2][b, h // G, :kv] += g[2]
    return (out, lse, *grads)
