"""The attention cache in 8 bits, written down in 64 bits on the host: what the GPU tests of slicer_kv_* compare with."""
from __future__ import annotations

import math

import numpy as np
import torch

PAGE = 64
TINY = 2.0 ** -119


def f32(x):
    return np.asarray(x, dtype=np.float64).astype(np.float32).astype(np.float64)


def hold(x):
    """[64, D] bf16 values of a page and head (float64) -> (codes, scale)."""
    amax = np.abs(x).max()
    if amax < TINY:
        return np.zeros_like(x), 0.0
    scale, inv = f32(amax / 127.0), f32(127.0 / amax)          # quotients and products of fp32 numbers, rounded from 64 bits: as rounded once
    return np.clip(np.rint(f32(x * inv)), -127, 127), float(scale)


class Sequence:
    """One sequence: pages of held values, then open tokens; a page or token that has met a value that is not finite is marked."""

    def __init__(self, heads, dim):
        self.G, self.D = heads, dim
        self.pages = []           # (k [64, G, D], v, bad [G])
        self.open = []            # (k [G, D], v, bad [G])

    def append(self, k, v):
        """k, v: [n, G, D] torch tensors."""
        k, v = (t.detach().cpu().to(torch.bfloat16).double().numpy() for t in (k, v))
        for i in range(k.shape[0]):
            bad = ~(np.isfinite(k[i]).all(1) & np.isfinite(v[i]).all(1))
            self.open.append((np.where(bad[:, None], 0.0, k[i]), np.where(bad[:, None], 0.0, v[i]), bad))
            if len(self.open) == PAGE:
                held = []
                for which in (0, 1):
                    x = np.stack([t[which] for t in self.open])
                    y = np.empty_like(x)
                    for g in range(self.G):
                        codes, scale = hold(x[:, g])
                        y[:, g] = codes * scale
                    held.append(y)
                self.pages.append((held[0], held[1], np.stack([t[2] for t in self.open]).any(0)))
                self.open = []

    def __len__(self):
        return PAGE * len(self.pages) + len(self.open)

    def values(self):
        """(k, v [len, G, D], bad [len, G])"""
        if not len(self):
            z = np.zeros((0, self.G, self.D))
            return z, z, np.zeros((0, self.G), bool)
        ks = [p[0] for p in self.pages] + [t[0][None] for t in self.open]
        vs = [p[1] for p in self.pages] + [t[1][None] for t in self.open]
        bad = [np.repeat(p[2][None], PAGE, 0) for p in self.pages] + [t[2][None] for t in self.open]
        return np.concatenate(ks), np.concatenate(vs), np.concatenate(bad)

    def attend(self, q, scale, causal=True):
        """q [n, H, D] -> out, lse, mass [G, pages], and for tolerances: sum p |v|, the largest sum |q k| of the rows and sum |v|."""
        q = q.detach().cpu().double().numpy()
        n, H, D = q.shape
        R, total = H // self.G, len(self)
        k, v, bad = self.values()
        pages = -(-total // PAGE)
        out, absv, lse = np.zeros((n, H, D)), np.zeros((n, H, D)), np.full((n, H), -np.inf)
        size, allv = np.zeros((n, H)), np.zeros((n, H, D))
        mass = np.zeros((self.G, max(pages, 1)))
        for h in range(H):
            g = h // R
            s = scale * (q[:, h] @ k[:, g].T)
            seen = np.ones((n, total), bool)
            if causal:
                seen = np.arange(total)[None] < (total - n + np.arange(n)[:, None] + 1)
            for i in range(n):
                sel = np.nonzero(seen[i])[0]
                if not len(sel):
                    continue
                if bad[sel, g].any():
                    out[i, h], lse[i, h] = np.nan, np.nan
                    mass[g, sel // PAGE] += np.nan
                    continue
                si = s[i, sel]
                m = si.max()
                p = np.exp(si - m)
                lse[i, h] = m + math.log(p.sum())
                p /= p.sum()
                out[i, h] = p @ v[sel, g]
                absv[i, h] = p @ np.abs(v[sel, g])
                allv[i, h] = np.abs(v[sel, g]).sum(0)
                size[i, h] = abs(scale) * (np.abs(k[sel, g]) @ np.abs(q[i, h])).max()
                np.add.at(mass[g], sel // PAGE, p)
        return out, lse, mass[:, :pages], absv, size, allv


def evict(mass, pages, keep, sink, recent):
    """mass [G, >= pages] of one sequence -> the places of the full pages that stay."""
    if pages <= keep:
        return list(range(pages))
    w = mass.astype(np.float64).sum(0)
    free = sorted(range(sink, pages - recent), key=lambda p: (0, 0, p) if np.isnan(w[p]) else (1, -w[p], p))
    return sorted(list(range(sink)) + list(range(pages - recent, pages)) + free[: keep - sink - recent])
