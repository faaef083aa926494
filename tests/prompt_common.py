"""References for the calls between a prompt and its paged cache, in plain Python and 64 bits, apart from the library."""
import math

import numpy as np
import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # of a rounding, relative


def attend(q, k, v, cu, scale, window=0):
    """softmax(scale q k^T) v of packed causal sequences in 64 bits, and how far a result in q's type may be off.

    With w the weights, u half a step of the type and d the head dimension: the weights in front of the product with V are rounded (u
    each; their sum is taken as rounded, so numerator and denominator move by u sum w|v| each at most), the output is rounded (u |o|),
    a score's fp32 sum is off by at most (d + 2) 2^-24 sum |q_i k_i| scale (which moves a weight by as much, relatively, twice that
    with the denominator), an fp32 exp2 and its argument by 2^-22 each, the fp32 sums over n keys by (n + 64) 2^-23 (twice: numerator and denominator; running
    rescales included).  fp16 weights below 2^-14 are off by 2^-25 at most, absolutely, where the largest of a row is at least 1: n 2^-25 max|v|,
    twice with the denominator.  Outputs below 2^-14 likewise: 2^-25."""
    T, hq, d = q.shape
    g = hq // k.shape[1]
    out = torch.zeros((T, hq, d), dtype=torch.float64)
    tol = torch.zeros_like(out)
    u = HALF_STEP[q.dtype]
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(hq if b > a else 0):
            qd, kd, vd = (x[a:b, i].double().cpu() for x, i in ((q, h), (k, h // g), (v, h // g)))
            n = b - a
            back = torch.arange(n).unsqueeze(1) - torch.arange(n)
            hidden = (back < 0) | ((back >= window) if window else torch.zeros((n, n), dtype=torch.bool))
            w = torch.softmax((qd @ kd.t() * scale).masked_fill(hidden, -math.inf), dim=-1)
            o, spread = w @ vd, w @ vd.abs()
            score = abs(scale) * (d + 2) * 2.0 ** -24 * (qd.abs() @ kd.abs().t()).masked_fill(hidden, 0).amax(-1, keepdim=True)
            small = (n * 2.0 ** -24 * vd.abs().max() + 2.0 ** -25) if q.dtype == torch.float16 else 0.0
            out[a:b, h] = o
            tol[a:b, h] = u * o.abs() + (2 * u + 2 * score + 2.0 ** -20 + (n + 64) * 2.0 ** -22) * spread + small
    return out, tol


def quantize(x, group):
    """Eq. 2-3 from fp16 or bf16 [..., d], every fp32 step rounded by itself: packed codes, scales, zero-points as numpy."""
    f = x.float().cpu().numpy().reshape(tuple(x.shape[:-1]) + (-1, group))
    with np.errstate(over="ignore"):
        mn, mx = f.min(-1, keepdims=True), f.max(-1, keepdims=True)
        s = np.minimum((mx - mn) / np.float32(15), np.float32(65504)).astype(np.float16)
        s[s == 0] = 1
        z = np.clip((-mn / s.astype(np.float32)), np.float32(-65504), np.float32(65504)).astype(np.float16) + np.float16(0)
        c = np.clip(np.rint(f / s.astype(np.float32) + z.astype(np.float32)), 0, 15).astype(np.uint8).reshape(x.shape)
    return c[..., 0::2] | c[..., 1::2] << 4, s[..., 0], z[..., 0]


def append(lens, table, free, n_free, new, page, bound):
    """tq_pages_append, one sequence and one token at a time."""
    lens, table, n_pages = list(lens), [list(r) for r in table], len(free)
    n_free = min(max(n_free, 0), n_pages)
    left, wanted = n_free, 0               # pages nobody has asked for yet (may go below zero)
    cu, served, slots = [0], [], []
    for b, row in enumerate(table):
        have, want = max(lens[b], 0), max(new[b], 0)
        wanted += want
        cu.append(min(wanted, bound))
        fits = have + want <= len(row) * page and (want == 0 or wanted <= bound)
        need = -(-(have + want) // page) - -(-have // page) if fits else 0
        left -= need
        ok = fits and (need == 0 or left >= 0)
        served.append(int(ok))
        lens[b] = have + want if ok else have
        for i in range(need if ok else 0):
            n_free -= 1
            row[-(-have // page) + i] = free[n_free]
        for t in range(cu[-1] - cu[-2]):
            p = have + t
            num = row[p // page] if ok else -1
            slots.append(num * page + p % page if 0 <= num < n_pages else -1)
    return dict(seq_lens=lens, block_table=table, n_free=n_free, cu_seqlens=cu, served=served,
                slots=slots + [-1] * (bound - len(slots)))


def trim(lens, table, free, n_free, keep, page):
    lens, free = list(lens), list(free)
    n_free = min(max(n_free, 0), len(free))
    for b, row in enumerate(table):
        have = max(lens[b], 0)
        lens[b] = min(max(keep[b], 0), have)
        for i in range(-(-lens[b] // page), min(-(-have // page), len(row))):
            if n_free < len(free):
                free[n_free] = row[i]
                n_free += 1
    return dict(seq_lens=lens, free_pages=free, n_free=n_free)
