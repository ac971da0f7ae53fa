"""64-bit references, inputs and error bounds of the attention operators (written from the formulas; no code of the library)."""
import math

import torch

from linear_ref import UNIT

BF16, F16 = torch.bfloat16, torch.float16


def rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


class Batch:
    """A paged cache with sequences of `lengths` tokens whose last `new` ones are a call's rows, in scattered pages; every place
    of the cache that holds no token is NaN. layout: 'heads' [pages][heads][tokens][D], 'tokens' [pages][tokens][heads][D] seen
    as the former. behind: rows behind the last sequence. prefix: leading tokens that all sequences share."""

    def __init__(self, new, lengths, Hq, Hkv, D, dtype, page, seed=1, layout="heads", behind=0, prefix=0, single=False, spare=2, wide=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g, self.new, self.lengths, self.Hq, self.Hkv, self.D, self.dtype, self.page = g, new, lengths, Hq, Hkv, D, dtype, page
        self.T, self.B = sum(new) + behind, len(new)
        need = [-(-n // page) for n in lengths]
        shared = prefix // page
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        width = max([1] + need) + wide
        table = torch.full((self.B, width), -7, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            if shared and b:
                table[b, :min(n, shared)] = table[0, :min(n, shared)]
            at += n
        shape = (pages, Hkv, page, D) if layout == "heads" else (pages, page, Hkv, D)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        if layout == "tokens":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.table = table
        self.K, self.V = [], []                      # each sequence's own tokens, [n][Hkv][D]
        for b, n in enumerate(lengths):
            k, v = (rand(g, n, Hkv, D).to(dtype) for _ in range(2))
            if prefix and b:
                k[:prefix], v[:prefix] = self.K[0][:min(n, prefix)], self.V[0][:min(n, prefix)]
            self.K.append(k)
            self.V.append(v)
        self.write()
        self.len_t = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        self.first = starts
        self.starts = None if single else torch.tensor(starts, dtype=torch.int32, device="cuda")

    def write(self):
        for b, n in enumerate(self.lengths):
            if n:
                p = torch.arange(n, device="cuda")
                page = self.table[b].long()[p // self.page]
                self.k[page, :, p % self.page] = self.K[b]
                self.v[page, :, p % self.page] = self.V[b]

    def queries(self, scale=1.5, pad=0, lead=0):
        """[T][Hq][D], cut out of rows that are `pad` elements longer and start `lead` elements past an allocation."""
        cols = self.Hq * self.D
        buf = torch.full((self.T * (cols + pad) + lead,), float("nan"), device="cuda", dtype=self.dtype)
        v = buf[lead:].view(self.T, cols + pad)[:, :cols] if self.T else buf.new_empty(0, cols)
        v.copy_(scale * rand(self.g, self.T, cols))
        return v.unflatten(1, (self.Hq, self.D))

    def args(self):
        return self.k, self.v, self.table, self.len_t

    def exact(self, q, window=0, sinks=0, scale=None):
        """[T][Hq][D] in 64 bits, and the bound of an output's error; rows of no sequence are NaN in both."""
        G, D = self.Hq // self.Hkv, self.D
        scale = 1 / math.sqrt(D) if scale is None else scale
        out = torch.full((self.T, self.Hq, D), float("nan"), dtype=torch.float64, device="cuda")
        tol = out.clone()
        u = UNIT[self.dtype]
        for b, (a, n) in enumerate(zip(self.new, self.lengths)):
            t = self.first[b]
            if not a:
                continue
            x = q[t:t + a].double().unflatten(1, (self.Hkv, G))
            k, v = self.K[b].double(), self.V[b].double()
            p = torch.arange(n - a, n, device="cuda")[:, None]
            j = torch.arange(n, device="cuda")
            seen = j <= p
            if window:
                seen = seen & ((j > p - window) | (j < sinks))
            s = torch.einsum("thgd,jhd->thgj", x, k) * scale
            size = torch.einsum("thgd,jhd->thgj", x.abs(), k.abs()) * scale      # what the scores' rounding scales with
            m = seen[:, None, None]
            s = torch.where(m, s, -math.inf)
            top = s.amax(3, keepdim=True).clamp_min(-1e300) if n else s.new_zeros(a, self.Hkv, G, 1)
            w = torch.where(m, torch.exp(s - top), 0.0)
            l = w.sum(3, keepdim=True)
            w = w / torch.where(l > 0, l, 1.0)
            o = torch.einsum("thgj,jhd->thgd", w, v)
            A = torch.einsum("thgj,jhd->thgd", w, v.abs())
            # A weight e^x is off by the score's error (D products of exact 32-bit values, summed with at most 2^-23 lost of the
            # sum of sizes at each of D additions, then two products), by the exponent's rounding (|x| 2^-23 log2 e), by the
            # exponential's two units; each weight is rounded to u for the product with v; two sums over the keys of at most
            # 2^-23 lost an addition (joined in another order).
            big = torch.where(m, size, 0.0).amax(3, keepdim=True) if n else s.new_zeros(a, self.Hkv, G, 1)
            e = (D + 4) * 2.0 ** -23 * big + (big + 16) * 2.0 ** -21 + (2 * n + 64) * 2.0 ** -23
            tol_b = A * (u + 2 * e) * (1 + 1e-3) + u * o.abs()
            if self.dtype == F16:      # weights below 2^-14 and outputs lie on the grid of 2^-24; the largest weight is at least 1
                tol_b += 2.0 ** -25 * (torch.einsum("thgj,jhd->thgd", m.expand_as(w).double(), v.abs()) + 2)
            out[t:t + a], tol[t:t + a] = o.flatten(1, 2), tol_b.flatten(1, 2) + 2.0 ** -130
        return out, tol


def check(got, want, tol, valid):
    got, want, tol = got[:valid].double(), want[:valid], tol[:valid]
    assert torch.isfinite(got).all()
    off = (got - want).abs()
    bad = off > tol
    assert not bad.any(), (int(bad.sum()), float((off / tol).max()), torch.nonzero(bad)[:5].tolist())
    return float((off / tol).max()) if off.numel() else 0.0
