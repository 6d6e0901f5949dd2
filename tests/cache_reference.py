"""Plain 64-bit definitions of the cache operators, on the CPU, with the tolerances that their tests use.

A result may be off by the rounding to its type (torch.finfo(t).eps / 2 of its size) and by what 32-bit arithmetic costs.  With E = 2^-24
(a rounding of fp32), n keys and D dimensions:
  * a score is a sum of D products, scaled: off by at most (D + 3) E scale sum_c |q_c k_c|, which its weight is off by as a factor; the maximum that is subtracted cancels
    but for one rounding of the difference of the two, at most 2 E of their size;
  * exp2 of a number x: one rounding of x (as above) and 2 E of the hardware's;
  * the sums of n weights, and of n products, are off by at most n E of the sums of sizes, rescalings by 2 E each time the maximum rises (at most n / 32 times) and at the joins;
  * as a pair of bf16 numbers weights are kept to 2^-16, and queries of fp32 to 2^-16 as a factor of every product.
Weights appear above and below the fraction, so that all of it counts twice:
  |error| <= rounding |o| + 2 (score + (n + n / 16 + 16) E + pair) sum_j p_j |v_j|
"""
import math

import numpy as np
import torch

E = 2.0 ** -24


def pack(k, v):
    """Caches [.., B, rows, heads, D] as bpd.h lays them out."""
    if not (k.dtype == torch.bfloat16 and k.shape[-1] in (64, 128)):
        return k.contiguous(), v.contiguous()
    *lead, b, cap, h, d = k.shape
    assert cap % 32 == 0
    out_k, out_v = torch.empty((*lead, b, h, cap // 32, 32 * d), dtype=k.dtype), torch.empty((*lead, b, h, cap // 32, 32 * d), dtype=k.dtype)
    key, c = torch.meshgrid(torch.arange(32), torch.arange(d), indexing="ij")
    a, t, r, s, q, e = key // 8, key // 4 % 2, key % 4, c // 32, c // 8 % 4, c % 8
    at_k = ((((t * (d // 32) + s) * 4 + q) * 4 + a) * 4 + r) * 8 + e
    at_v = (((c // 16) * 4 + key // 8) * 16 + c % 16) * 8 + key % 8
    for x, y, at in ((k, out_k, at_k), (v, out_v, at_v)):
        rows = x.movedim(-2, -3).reshape(*lead, b, h, cap // 32, 32 * d)       # [.., key * d + c]
        y[..., at.reshape(-1)] = rows
    shape = (*lead, b, h, cap // 32, 32, d)
    return out_k.view(shape), out_v.view(shape)


def unpack(k, v):
    """The other way round."""
    if not (k.dtype == torch.bfloat16 and k.shape[-1] in (64, 128)):
        return k, v
    *lead, b, h, g, _, d = k.shape
    key, c = torch.meshgrid(torch.arange(32), torch.arange(d), indexing="ij")
    a, t, r, s, q, e = key // 8, key // 4 % 2, key % 4, c // 32, c // 8 % 4, c % 8
    at_k = (((((t * (d // 32) + s) * 4 + q) * 4 + a) * 4 + r) * 8 + e).reshape(-1)
    at_v = ((((c // 16) * 4 + key // 8) * 16 + c % 16) * 8 + key % 8).reshape(-1)
    return tuple(x.reshape(*lead, b, h, g, 32 * d)[..., at].reshape(*lead, b, h, g * 32, d).movedim(-2, -3).contiguous() for x, at in ((k, at_k), (v, at_v)))


def ancestors(parent, there):
    """Per node the list of its ancestors and itself, None for absent ones."""
    out = []
    for i, p in enumerate(parent):
        p = int(p)
        if i >= there or p < -1 or p >= i or (p >= 0 and out[p] is None):
            out.append(None)
        else:
            out.append(([] if p < 0 else out[p]) + [i])
    return out


def choose(q, k, n, block, first, recent, top):
    """Blocks that the heads q [G, D] see of n rows k [rows, D] (64 bits)."""
    done = n // block
    always = [j for j in range(done) if j < first or j >= done - recent]
    rest = [j for j in range(done) if j not in set(always)]
    bound = {}
    for j in rest:
        rows = k[j * block:(j + 1) * block]
        lo, hi = rows.amin(0), rows.amax(0)
        bound[j] = float(torch.maximum(q * lo, q * hi).sum())
    rest.sort(key=lambda j: (math.isnan(bound[j]), -bound[j] if not math.isnan(bound[j]) else 0, j))
    return sorted(always + rest[:top])


def attention(q, k, v, lengths, parents, scale=None, blocks=None):
    """q [B, T, H, D], k, v [B, rows, heads, D], parents [B, T] or None.  Returns (out, bound of the error without the rounding of the result, chosen)."""
    b, t, h, d = q.shape
    cap, kv = k.shape[1], k.shape[2]
    g = h // kv
    scale = d ** -0.5 if scale is None else scale
    out, off = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    chosen = np.zeros((b, kv, t, (cap // blocks["block"] + 31) // 32 * 32 if blocks else 0), bool)
    pair_q = q.dtype == torch.float32 and k.dtype == torch.bfloat16 and d != 16
    pair_p = k.dtype == torch.bfloat16 and d != 16
    for s in range(b):
        n = int(lengths[s])
        there = 0 if n < 0 else max(0, min(t, cap - n))
        anc = ancestors(parents[s] if parents is not None else range(-1, t - 1), there)
        n = max(0, min(n, cap))
        for i in range(t):
            if anc[i] is None:
                continue
            own = [n + a for a in anc[i]]
            for hk in range(kv):
                qq = q[s, i, hk * g:(hk + 1) * g].double()
                rows = list(range(n))
                if blocks:
                    picks = choose(qq, k[s, :, hk].double(), n, **blocks)
                    chosen[s, hk, i, picks] = True
                    rows = [r for j in picks for r in range(j * blocks["block"], (j + 1) * blocks["block"])] + list(range(n // blocks["block"] * blocks["block"], n))
                kk, vv = k[s, rows + own, hk].double(), v[s, rows + own, hk].double()
                score = qq @ kk.T * scale
                p = torch.softmax(score, 1)
                o = p @ vv
                size = (p[:, :, None] * vv.abs()[None]).sum(1)
                most = (qq.abs() @ kk.abs().T).amax(1, keepdim=True) * abs(scale)
                nk = kk.shape[0]
                rel = (d + 3 + 4) * E * most + (2.0 ** -16 * most if pair_q else 0) + (nk + nk / 16 + 16) * E + (2.0 ** -16 if pair_p else 0)
                out[s, i, hk * g:(hk + 1) * g], off[s, i, hk * g:(hk + 1) * g] = o, 2 * rel * size
    words = chosen.reshape(b, kv, t, -1, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)
    return out, off, torch.from_numpy(words.sum(-1).astype(np.uint32).view(np.int32))


def check(got, want, off, what=""):
    got = got.detach().cpu()
    none = torch.isnan(want)                       # (a key that a node sees is not a number)
    assert torch.equal(torch.isnan(got), none), f"{what}: not a number"
    got, want, off = got[~none], want[~none], off[~none]
    bound = off + want.abs() * (torch.finfo(got.dtype).eps / 2) * (1 + 2.0 ** -10) + 1e-37
    err = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    worst = float((err / bound).max()) if err.numel() else 0.0
    assert worst <= 1, f"{what}: {worst} times the bound, at {np.unravel_index(int((err / bound).argmax()), err.shape)}"


def accept(parent, token, expect, best, length, room, eos, cap):
    """One sequence: (path, next)."""
    path, want, cur = [], int(expect), -1
    most = len(parent) if room is None else min(len(parent), int(room))
    there = len(parent) if cap is None else min(len(parent), cap - int(length))
    if length < 0:
        most = 0
    while len(path) < most:
        step = [i for i in range(cur + 1, there) if int(parent[i]) == cur and int(token[i]) == want]
        if not step:
            break
        cur = step[0]
        path.append(cur)
        want = int(best[cur])
        if eos >= 0 and int(token[cur]) == eos:
            break
    return path, want


def summaries(k, block):
    """[B, heads, blocks, 2, D] of k [B, rows, heads, D]."""
    b, cap, h, d = k.shape
    n = cap // block
    x = k[:, :n * block].reshape(b, n, block, h, d)
    return torch.stack([x.amin(2), x.amax(2)], 2).permute(0, 3, 1, 2, 4)


def summaries_unpacked(s, n):
    """Summaries as the operators keep them, as [B, heads, blocks, 2, D]."""
    b, h, tiles, _, d8, _, _ = s.shape
    return s.permute(0, 1, 2, 5, 3, 4, 6).reshape(b, h, tiles * 64, 2, d8 * 8)[:, :, :n]
