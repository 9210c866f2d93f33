"""The paged key-value cache in plain form: attention in 64 bits with bounds on its rounding, bookkeeping on Python lists."""
from __future__ import annotations

import math
import types

import torch


def ceil_div(a, b):
    return -(-a // b)


def visible(p, window, sinks, upto):
    """Positions that a token at position p sees, of 0 .. upto-1."""
    return [j for j in range(max(0, min(p + 1, upto))) if window <= 0 or j > p - window or j < sinks]


def attend(q, k, v, table, lens, n_new=None, scale=None, window=0, sinks=0, weight_bits=24):
    """(out float64 [B, n, Hq, D], bound of the same shape, written [B, n]) for tensors on any device.

    The bound is on |kernel - out|, by arithmetic.  With w_j the weights (summing to one), v_j the values and u = 2^-24:
      scores   a dot product of D terms in fp32 and its scaling by scale log2(e): off by at most (D + 4) u S, S = scale sum |q_d k_jd|,
               and the subtraction of the reference by another u (S + 16); with the exponential's 2^-22 a weight is off by at most
               e_j = (2 D + 24) u (max_j S + 1) + 2^-22, relative (twice that for the normaliser, in which the same errors sit);
      weights  rounded to `weight_bits` bits of mantissa (8 in bf16, of which half a step is 2^-8): r = 2^-weight_bits, relative
      sums     of N terms and the N / 32 joins and rescalings around them, in fp32: at most (N + 64) 2^-23 of the sum of their magnitudes
               (2^-23: a tensor core may cut off instead of rounding)
      result   rounded once to the output's type, half a step: eps / 2.
    An error d_j of weight j moves out by w_j d_j (v_j - out), so the weights' errors count with sum_j w_j |v_j - out|.
    """
    B, n, Hq, D = q.shape
    P, Hkv, page, _ = k.shape
    group = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    u = 2.0 ** -24
    out = torch.zeros((B, n, Hq, D), dtype=torch.float64)
    bound = torch.zeros_like(out)
    written = torch.zeros((B, n), dtype=torch.bool)
    tab, ls = table.cpu().tolist(), lens.cpu().tolist()
    news = [n] * B if n_new is None else [max(0, min(n, x)) for x in n_new.cpu().tolist()]
    half = torch.finfo(q.dtype).eps / 2
    for b in range(B):
        if news[b] == 0:
            continue
        L = ls[b]
        bad = L < 0 or L > len(tab[b]) * page
        L = 0 if bad else L
        pages = tab[b][:ceil_div(L, page)]
        if pages:
            at = torch.tensor([x if 0 <= x < P else 0 for x in pages], device=k.device)
            keys = k[at].transpose(1, 2).reshape(-1, Hkv, D)[:L].double().cpu()
            vals = v[at].transpose(1, 2).reshape(-1, Hkv, D)[:L].double().cpu()
        for t in range(news[b]):
            written[b, t] = True
            if bad:
                out[b, t] = math.nan
                continue
            see = visible(L - news[b] + t, window, sinks, L)
            if not see:
                continue
            if any(not 0 <= pages[j // page] < P for j in see):
                out[b, t] = math.nan
                continue
            kk, vv = keys[see], vals[see]
            qq = q[b, t].double().cpu().view(Hkv, group, D)
            s = torch.einsum("hgd,jhd->hgj", qq, kk) * scale
            S = torch.einsum("hgd,jhd->hgj", qq.abs(), kk.abs()).amax(-1) * abs(scale)       # [Hkv, group]
            w = torch.softmax(s, -1)
            o = torch.einsum("hgj,jhd->hgd", w, vv)
            A = torch.stack([torch.einsum("gj,jgd->gd", w[h], (vv[:, h][:, None] - o[h][None]).abs()) for h in range(Hkv)])
            mag = torch.einsum("hgj,jhd->hgd", w, vv.abs())
            e = 2 * ((2 * D + 24) * u * (S + 1) + 2.0 ** -22)
            r = 2.0 ** -weight_bits
            err = (e[..., None] + r * (1 + 2 * r)) * A + (len(see) + 64) * 2.0 ** -23 * (mag + o.abs())
            out[b, t] = o.reshape(Hq, D)
            bound[b, t] = (err + half * (o.abs() + err)).reshape(Hq, D)
    return out, bound, written


class Book:
    """The pages' bookkeeping on lists."""

    def __init__(self, table, lens, refs, page):
        self.table, self.lens, self.refs, self.page = table.cpu().tolist(), lens.cpu().tolist(), refs.cpu().tolist(), page

    def held(self, tokens):
        return ceil_div(tokens, self.page)

    def ok(self, b):
        return 0 <= self.lens[b] <= len(self.table[b]) * self.page

    def extend(self, n, n_new=None):
        P, new, copies, drop = len(self.refs), [], [], []
        before = list(self.refs)
        free = [p for p in range(P) if before[p] == 0]
        asked = 0
        for b, L in enumerate(self.lens):
            m = n if n_new is None else n_new[b]
            new.append(-1)
            copies.append([-1, -1])
            if not 0 <= m <= n or not self.ok(b) or L + m > len(self.table[b]) * self.page or L + m > 2**31 - 1:
                continue
            first, pages, replace = self.held(L), self.held(L + m) - self.held(L), False
            if m > 0 and L % self.page:
                last = self.table[b][first - 1]
                if not 0 <= last < P:
                    continue
                if before[last] > 1:
                    replace, first, pages = True, first - 1, pages + 1
            asked += pages
            if pages and asked > len(free):
                continue
            for i in range(pages):
                p = free[asked - pages + i]
                if i == 0 and replace:
                    copies[b] = [self.table[b][first], p]
                    drop.append(self.table[b][first])
                self.table[b][first + i] = p
                self.refs[p] = 1
            self.lens[b] += m
            new[b] = m
        for p in drop:
            self.refs[p] -= 1
        return new, copies

    def give(self, p):
        if 0 <= p < len(self.refs) and self.refs[p] > 0:
            self.refs[p] -= 1

    def truncate(self, keep, n=0, n_new=None):
        for b, L in enumerate(self.lens):
            if not self.ok(b):
                continue
            m = L if n == 0 else min(L, max(0, n if n_new is None else n_new[b]))
            left = L - m + max(0, min(m, keep[b]))
            for j in range(self.held(left), self.held(L)):
                self.give(self.table[b][j])
                self.table[b][j] = -1
            self.lens[b] = left

    def fork(self, src, dst):
        B, ok = len(self.lens), []
        rows, lens = [list(r) for r in self.table], list(self.lens)
        for i, (s, d) in enumerate(zip(src, dst)):
            bad = not (0 <= s < B and 0 <= d < B) or d in src or any(dst[g] == d for g in range(len(dst)) if g != i)
            bad = bad or not (0 <= lens[s] <= len(rows[s]) * self.page and 0 <= lens[d] <= len(rows[d]) * self.page)
            ok.append(-1 if bad else 0)
            if bad:
                continue
            for p in rows[s][:self.held(lens[s])]:
                if 0 <= p < len(self.refs):
                    self.refs[p] += 1
            for p in rows[d][:self.held(lens[d])]:
                self.give(p)
            self.table[d] = rows[s][:self.held(lens[s])] + [-1] * (len(rows[s]) - self.held(lens[s]))
            self.lens[d] = lens[s]
        return ok

    def compact(self):
        P = len(self.refs)
        live = sum(1 for r in self.refs if r != 0)
        holes = [p for p in range(live) if self.refs[p] == 0]
        sources = [p for p in range(live, P) if self.refs[p] != 0]
        to = dict(zip(sources, holes))
        for b in range(len(self.lens)):
            if self.ok(b):
                for j in range(self.held(self.lens[b])):
                    self.table[b][j] = to.get(self.table[b][j], self.table[b][j])
        for s, h in to.items():
            self.refs[h], self.refs[s] = self.refs[s], 0
        moves = [[s, h] for s, h in zip(sources, holes)]
        return moves + [[-1, -1]] * (P // 2 - len(moves)), len(moves)


def make(B, n, Hq, Hkv, D, page, lens, dtype=torch.bfloat16, device="cuda", seed=0, spare=5, layout="heads", width=None, q_scale=1.5):
    """A cache with the given sequence lengths on pages in no order; layout "tokens": rows of a page by token first in memory."""
    g = torch.Generator().manual_seed(seed)
    held = [ceil_div(max(0, x), page) for x in lens]
    width = width or max(1, max(held))
    P = sum(held) + spare
    order = torch.randperm(P, generator=g).tolist()
    table = [[-1] * width for _ in range(B)]
    for b in range(B):
        for j in range(min(held[b], width)):
            table[b][j] = order.pop()
    def rand(*shape):
        return torch.randn(shape, generator=g)
    if layout == "tokens":
        k, v = (rand(P, page, Hkv, D).to(dtype).to(device).transpose(1, 2) for _ in range(2))
    else:
        k, v = (rand(P, Hkv, page, D).to(dtype).to(device) for _ in range(2))
    refs = torch.zeros((P,), dtype=torch.int32)
    for row, h in zip(table, held):
        for p in row[:h]:
            refs[p] += 1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=device)      # noqa: E731
    return types.SimpleNamespace(q=(rand(B, n, Hq, D) * q_scale).to(dtype).to(device), k=k, v=v, table=i32(table), lens=i32(list(lens)), refs=refs.to(device),
                                 k_new=rand(B, n, Hkv, D).to(dtype).to(device), v_new=rand(B, n, Hkv, D).to(dtype).to(device), page=page)
