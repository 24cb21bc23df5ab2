"""What the tests of the windowed attention share: inputs, and bounds from the roundings that the kernels make.

Bounds, on top of the 64-bit result.  h is half a step of the tensors' type.
  scores   products of 16-bit numbers are exact in fp32; sums of 128 of them, and lse, are off by less than S = 2^-16 of a unit at
           the sizes used here (magnitudes below 2^5, 2^-23 a step, a tree of a few steps), and so is a weight, relative to itself
  out      each weight rounded (h), the sum rounded (h): h |out| + (h + S) (P |V|); fp16 weights below 2^-14 are off by up to
           2^-25 of the row's largest: 2^-25 sum |V|
  delta    made of the rounded out: sum |dout| times out's bound
  dS       h |dS| + P (S (|dP| + |delta|) + 2^-19 |dout| |V| + delta's bound), fp16 2^-25 in all
  dq, dk   h |dq| + scale (dS's bound) |K|, and so on;  dv as out with P^T |dout|."""
import math

import torch

from tests import plain_operators as plain

DEV = "cuda"
S = 2.0 ** -16
T = {"bf16": torch.bfloat16, "f16": torch.float16}


def tensor(shape, kind, order, gen, scale=1.0):
    B, H, N, D = shape
    x = torch.randn((B, N, H, D) if order == "tokens" else shape, generator=gen, device=DEV).mul_(scale).to(T[kind])
    if order == "tokens":
        return x.transpose(1, 2)
    if order == "packed":
        wide = torch.full((B, H, N + 3, D + 8), math.nan, dtype=T[kind], device=DEV)
        wide[:, :, :N, 8:] = x
        return wide[:, :, :N, 8:]
    return x


class Case:
    def __init__(self, kind, B, H, Hkv, D, n_q, n_kv, left, right, sink, full, q_len=None, kv_len=None, order="heads", seed=0, scale=None, spread=1.0):
        self.gen = torch.Generator(device=DEV).manual_seed(1000 * n_q + n_kv + seed)
        self.kind, self.B, self.H, self.Hkv, self.D, self.n_q, self.n_kv = kind, B, H, Hkv, D, n_q, n_kv
        self.scale = D ** -0.5 if scale is None else scale
        self.q = tensor((B, H, n_q, D), kind, order, self.gen, spread)
        self.k, self.v = (tensor((B, Hkv, n_kv, D), kind, order, self.gen) for _ in range(2))
        self.dout = tensor((B, H, n_q, D), kind, order, self.gen)
        self.lens = [[n_q if q_len is None else min(max(q_len[b], 0), n_q), n_kv if kv_len is None else min(max(kv_len[b], 0), n_kv)] for b in range(B)]
        as_len = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
        self.rule = dict(left=left, right=right, n_sink=sink, n_full=full, q_len=as_len(q_len), kv_len=as_len(kv_len), softmax_scale=self.scale)
        for b, (r, n) in enumerate(self.lens):                       # what lies behind the lengths may be anything
            for t, m in ((self.q, r), (self.dout, r), (self.k, n), (self.v, n)):
                t[b, :, m:] = math.nan
        self.seen = [plain.visible(n_q, n_kv, left, right, sink, full, r, n)[:r, :n].to(DEV) for r, n in self.lens]

    def fresh(self, heads, n):
        """A result's tensor, filled with something to be found again where nothing is written."""
        return torch.full((self.B, heads, n, self.D), 77.0, dtype=T[self.kind], device=DEV)

    def check(self, out, lse, grads=None, heads=None):
        h, tiny = plain.half_step(T[self.kind]), (2.0 ** -25 if self.kind == "f16" else 0.0)
        small = plain.smallest(T[self.kind])
        G = self.H // self.Hkv
        for b, (r, n) in enumerate(self.lens):
            rest = [("out", out[b, :, r:], 77.0), ("lse", lse[b, :, r:], 77.0)]
            if grads:
                rest += [("dq", grads[0][b, :, r:], 77.0), ("dk", grads[1][b, :, n:], 77.0), ("dv", grads[2][b, :, n:], 77.0)]
            for name, t, was in rest:
                assert (t == was).all(), (name, "written behind the sequence", b)
            for hk in range(self.Hkv) if heads is None else sorted({x // G for x in heads}):
                k, v = self.k[b, hk, :n].double(), self.v[b, hk, :n].double()
                sums = [0.0, 0.0, 0.0, 0.0]
                for head in range(hk * G, hk * G + G):
                    q = self.q[b, head, :r].double()
                    want, want_lse, p = plain.attention(q, k, v, self.seen[b], self.scale)
                    bound = h * want.abs() + (h + S) * (p @ v.abs()) + tiny * v.abs().sum(0) + small
                    self.within(out[b, head, :r], want, bound, ("out", b, head))
                    empty = torch.isinf(want_lse)
                    assert torch.equal(torch.isinf(lse[b, head, :r]), empty) and (lse[b, head, :r][empty] < 0).all(), ("lse", b, head)
                    self.within(lse[b, head, :r][~empty], want_lse[~empty], S + 2.0 ** -22 * want_lse[~empty].abs(), ("lse", b, head))
                    if not grads:
                        continue
                    d = self.dout[b, head, :r].double()
                    dq, dk, dv = plain.attention_gradients(q, k, v, want, p, d, self.scale)
                    dp, delta = d @ v.T, (d * want).sum(-1, keepdim=True)
                    ds = p * (dp - delta)
                    ds_off = h * ds.abs() + p * (S * (dp.abs() + delta.abs()) + 2.0 ** -19 * (d.abs() @ v.abs().T) + (d.abs() * bound).sum(-1, keepdim=True)) + tiny
                    ds_off = torch.where(self.seen[b], ds_off, 0.0)
                    self.within(grads[0][b, head, :r], dq, h * dq.abs() + self.scale * (ds_off @ k.abs()) + small, ("dq", b, head))
                    p_off = torch.where(self.seen[b], (h + S) * p + tiny, 0.0)
                    for i, x in enumerate((dk, self.scale * (ds_off.T @ q.abs()), dv, p_off.T @ d.abs())):
                        sums[i] = sums[i] + x
                if grads:
                    self.within(grads[1][b, hk, :n], sums[0], h * sums[0].abs() + sums[1] + small, ("dk", b, hk))
                    self.within(grads[2][b, hk, :n], sums[2], h * sums[2].abs() + sums[3] + small, ("dv", b, hk))

    @staticmethod
    def within(got, want, bound, what):
        if want.numel():
            worst = ((got.double() - want).abs() / bound).nan_to_num(nan=math.inf).max().item()
            assert worst <= 1.0, (what, worst)
