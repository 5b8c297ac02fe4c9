"""Plain 64-bit forms of the serving operators and the bounds their results are held to."""
import math

import torch

F64 = torch.float64
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}     # of a value rounded once, relative


def rotate(x, pos, turns_per_pos, neighbours):
    """x [..., tokens, D] in 64 bits, rotated by 2 pi pos * turns (pos [..., tokens], turns [D / 2])."""
    D = x.shape[-1]
    angle = 2.0 * math.pi * torch.remainder(pos.to(F64)[..., None] * turns_per_pos, 1.0)
    c, s = angle.cos(), angle.sin()
    a, b = (x[..., 0::2], x[..., 1::2]) if neighbours else (x[..., :D // 2], x[..., D // 2:])
    ra, rb = a * c - b * s, b * c + a * s
    return torch.stack([ra, rb], -1).flatten(-2) if neighbours else torch.cat([ra, rb], -1)


def turns(D, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / D) / (2.0 * math.pi) for i in range(D // 2)], dtype=F64)


class Rows:
    """softmax(scale q K^T) V of rows q [m, D] over K, V [n, D], all in 64 bits, with what the bounds need."""

    def __init__(self, q, K, V, scale):
        q, K, V = q.to(F64), K.to(F64), V.to(F64)
        n, D = K.shape
        self.n, self.D = n, D
        if n == 0:
            self.O, self.lse = torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=F64)
            self.mass, self.vmax, self.dot = torch.zeros_like(q), 0.0, torch.zeros(q.shape[0], dtype=F64)
            return
        x = scale * (q @ K.T)
        self.lse = torch.logsumexp(x, -1)
        p = torch.exp(x - self.lse[:, None])
        self.O, self.mass = p @ V, p @ V.abs()
        self.vmax = float(V.abs().max())
        self.dot = (scale * (q.abs() @ K.abs().T)).amax(-1)                       # sum |q_i k_i| of the worst key

    def joined(self, O_in, lse_in):
        O_in, lse_in = O_in.to(F64), lse_in.to(F64)
        z = torch.logaddexp(self.lse, lse_in)
        a, b = torch.exp(self.lse - z), torch.exp(lse_in - z)
        a, b = (torch.where(torch.isfinite(z), w, torch.zeros_like(w)) for w in (a, b))
        O_in = torch.where(b[:, None] > 0, O_in, torch.zeros_like(O_in))          # what has no weight may be anything
        self.O, self.mass = a[:, None] * self.O + b[:, None] * O_in, a[:, None] * self.mass + b[:, None] * O_in.abs()
        self.vmax = max(self.vmax, float(O_in.abs().max()))
        self.lse = z
        return self

    # A logit is a sum of D products and is scaled once: it is off by at most (D + 4) 2^-24 of sum |q_i k_i|.  A weight, an
    # exponential of it, is off relatively by that plus the exponential's own 2^-21 (argument and result); sums of n terms add
    # n 2^-24; joining adds a few more.  That many times the largest |v|, twice (numerator and denominator), is how far O can be
    # off in fp32.  With bf16 the weights are rounded once more, 2^-8 of each, and divided by the sum of the rounded ones:
    # twice 2^-8 of sum p |v|.  The store rounds once.
    def weight_error(self):
        return (self.D + 4) * 2.0 ** -24 * self.dot + 2.0 ** -21 + (self.n + 32) * 2.0 ** -24

    def O_bound(self, dtype):
        rounded = 2.0 * HALF_STEP[dtype] if dtype == torch.bfloat16 else 0.0
        return 2.0 * self.weight_error()[:, None] * self.vmax + rounded * self.mass * 1.01 + HALF_STEP[dtype] * self.O.abs() * 1.01 + 1e-30

    def lse_bound(self):
        return self.weight_error() + 2.0 ** -22 * (self.lse.abs().nan_to_num(posinf=0.0) + 1.0)


def close(got, want, bound, what=""):
    got = got.to("cpu").to(F64)
    same = (got == want) | ((got - want).abs() <= bound)                          # (== for infinities)
    assert bool(same.all()), (what, float(((got - want).abs() / bound).nan_to_num(nan=math.inf)[~same].max()), int((~same).sum()))


def page_rows_of(K, table_row, n):
    """The first n rows of a unit, from its pages."""
    R = K.shape[1]
    return torch.cat([K[int(table_row[i])] for i in range(-(-n // R))])[:n] if n else K.new_zeros(0, K.shape[2])


def make_cache(g, B, Hkv, D, R, lengths, dtype, spare=0, room=0):
    """Pools whose pages belong to the units in random order, on the CPU.  Rows past the lengths hold NaN; table entries past a unit's
    pages numbers far outside.  `room`: rows a unit has pages for beyond its length; `spare`: pages of nobody."""
    U = B * Hkv
    need = [-(-(int(n) + room) // R) for n in lengths.view(-1)]
    width = max(1, max(need))
    order = torch.randperm(sum(need) + spare, generator=g).to(torch.int32)
    table = torch.full((U, width), 1 << 30, dtype=torch.int32)
    table[:, 1::2] = -7
    K, V = (torch.full((max(1, len(order)), R, D), math.nan, dtype=dtype) for _ in range(2))
    at = 0
    for u in range(U):
        table[u, :need[u]] = order[at:at + need[u]]
        at += need[u]
        for i in range(int(lengths.view(-1)[u])):
            page = int(table[u, i // R])
            K[page, i % R] = torch.randn(D, generator=g).to(dtype)
            V[page, i % R] = torch.randn(D, generator=g).to(dtype)
    return K, V, table
