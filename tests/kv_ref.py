"""Plain references for the paged key-value cache and its attention: a list
model of the page bookkeeping, one step after another, and attention and
rotary positions in float64 with a bound on what the kernels may be off by."""
from __future__ import annotations

import math

import torch

UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half an ulp, relative
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def div_up(a, b):
    return -(-a // b)


class PageModel:
    """np_kv_* on lists.  data[page][slot] is whatever a test puts there."""

    def __init__(self, S, N, M, P):
        self.S, self.N, self.M, self.P = S, N, M, P
        self.table = [[] for _ in range(S)]
        self.len = [0] * S
        self.refs = [0] * N
        self.data = [[None] * P for _ in range(N)]

    def extend(self, seqs, new):
        P = self.P
        served, holders, seen = [], {}, set()
        for i, (s, n) in enumerate(zip(seqs, new)):
            ok = 0 <= s < self.S and s not in seen and n >= 0 and self.len[s] + n <= self.M * P
            seen.add(s)
            served.append(ok)
            if ok and self.len[s] % P and n > 0:
                holders.setdefault(self.table[s][-1], []).append(i)
        plan, need = [], 0
        for i, (s, n) in enumerate(zip(seqs, new)):
            if not served[i]:
                plan.append(None)
                continue
            split = False
            if self.len[s] % P and n > 0:
                page = self.table[s][-1]
                h = holders[page]
                split = not (self.refs[page] == len(h) and h[0] == i)
            fresh = div_up(self.len[s] + n, P) - len(self.table[s])
            plan.append((split, fresh))
            need += split + fresh
        free = [p for p in range(self.N) if self.refs[p] == 0]
        if need > len(free):
            return [-1] * len(seqs)
        pos0 = []
        drop = []
        for i, (s, n) in enumerate(zip(seqs, new)):
            if plan[i] is None:
                pos0.append(-1)
                continue
            split, fresh = plan[i]
            pos0.append(self.len[s])
            if split:
                old, page = self.table[s][-1], free.pop(0)
                r = self.len[s] % P
                self.data[page][:r] = self.data[old][:r]
                self.table[s][-1] = page
                self.refs[page] = 1
                drop.append(old)
            for _ in range(fresh):
                page = free.pop(0)
                self.table[s].append(page)
                self.refs[page] = 1
            self.len[s] += n
        for p in drop:
            self.refs[p] -= 1
        return pos0

    def fork(self, src, dst, lens=None):
        before_len = list(self.len)
        before_table = [list(t) for t in self.table]
        taken = set()
        for i, (a, b) in enumerate(zip(src, dst)):
            if not (0 <= a < self.S and 0 <= b < self.S):
                if 0 <= b < self.S:
                    taken.add(b)
                continue
            first = b not in taken
            taken.add(b)
            n = before_len[a] if lens is None else lens[i]
            if not first or before_len[b] or not 0 <= n <= before_len[a]:
                continue
            self.table[b] = before_table[a][:div_up(n, self.P)]
            self.len[b] = n
            for p in self.table[b]:
                self.refs[p] += 1

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < self.S:
                for p in self.table[s]:
                    self.refs[p] -= 1
                self.table[s], self.len[s] = [], 0

    def compact(self):
        used = [p for p in range(self.N) if self.refs[p] > 0]
        U = len(used)
        holes = [p for p in range(U) if self.refs[p] == 0]
        to = dict(zip([p for p in used if p >= U], holes))
        for a, b in to.items():
            self.data[b] = list(self.data[a])
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return len(to)

    def tables(self):
        return [t + [-1] * (self.M - len(t)) for t in self.table]


def attention(q, keys, values, p0, scale, window, dtype):
    """One batch row in float64: q [n][Hq][D], keys/values [Hkv][len][D] (as
    stored), first position p0.  Returns (out, bound), both [n][Hq][D]: the
    exact result and how far a correct kernel may be off.

    The bound, elementwise, with W = sum_j w_j |v_j| over the softmax weights:
      - the scores' fp32 error ds (a dot product of D terms and the scaling:
        (D + 8) 2^-24 sum |q||k| scale, plus 2^-22 |s| for the base-2
        exponent) moves a weight by at most e^(2 ds) - 1 of itself;
      - exponentials and fp32 sums over the keys add (len + 32) 2^-23;
      - 16-bit types round each probability (u each, and fp16 by 2^-25 of the
        largest where it goes subnormal) and the result (u |o|)."""
    n, Hq, D = q.shape
    Hkv, ln, _ = keys.shape
    q, keys, values = q.double(), keys.double(), values.double()
    out = torch.zeros(n, Hq, D, dtype=torch.float64)
    bound = torch.zeros_like(out)
    u = UNIT[dtype]
    for i in range(n):
        p = p0 + i
        if p0 < 0:
            continue
        lo = max(0, p - window + 1) if window else 0
        for h in range(Hq):
            k, v = keys[h * Hkv // Hq, lo:p + 1], values[h * Hkv // Hq, lo:p + 1]
            s = (k @ q[i, h]) * scale
            w = torch.softmax(s, 0)
            out[i, h] = w @ v
            W = w @ v.abs()
            ds = float(((D + 8) * 2.0 ** -24 * abs(scale) * (k.abs() @ q[i, h].abs())
                        + 2.0 ** -22 * s.abs()).max())
            rel = math.expm1(2 * ds) + (p + 1 - lo + 32) * 2.0 ** -23
            b = rel * W + u * out[i, h].abs() * (1 + rel)
            if dtype != "f32":
                b = b + u * W * (1 + rel)
            if dtype == "f16":
                # weights relative to the largest are at least w / max w
                b = b + 2.0 ** -25 * float(w.max()) * v.abs().sum(0) * (1 + rel) + 2.0 ** -25
            bound[i, h] = b + 1e-30
    return out, bound


def rotate(x, cos, sin, pos, interleaved):
    """Rotary positions of x [n][H][D] in float64; pos [n] longs."""
    x = x.double()
    R = 2 * cos.shape[1]
    c, s = cos.double()[pos][:, None], sin.double()[pos][:, None]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = a * c - b * s, b * c + a * s
    return y
