"""Independent reference of the 8-bit key-value cache (test infrastructure only): fp64 on the CPU, one block, row or
slot after the other, no code shared with the library."""
from __future__ import annotations

import math

import torch

CODES = 256
# e4m3: sign, four bits of exponent (bias 7), three of fraction; 0x7f and 0xff are NaN
TABLE = torch.tensor([(-1.0 if c > 127 else 1.0) * (math.nan if c % 128 == 127 else
                      (8 + c % 8) * 2.0 ** (c // 8 % 16 - 10) if c // 8 % 16 else (c % 8) * 2.0 ** -9)
                      for c in range(CODES)], dtype=torch.float64)
POSITIVE = TABLE[:127]      # 0 .. 448, ascending


def encode(x: torch.Tensor) -> torch.Tensor:
    """Codes of fp64 numbers: nearest, ties to the even code; beyond 448 the largest; NaN 0x7f."""
    a = x.abs().nan_to_num(nan=0.0, posinf=1e9).clamp(max=448.0)
    hi = torch.searchsorted(POSITIVE, a).clamp(max=126)        # first number >= a
    lo = (hi - 1).clamp(min=0)
    down, up = a - POSITIVE[lo], POSITIVE[hi] - a
    code = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = torch.where(a == POSITIVE[hi], hi, code)
    code = torch.where(torch.signbit(x), code + 128, code)
    return torch.where(x.isnan(), torch.full_like(code, 127), code).to(torch.uint8)


def least_scale(largest: float) -> float:
    """Least power of two s with largest <= 448 s, from 2^-100 to 2^119."""
    e = -100
    while e < 119 and largest > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(codes, scale, x, cached, offsets, block):
    """codes [n, kv, L, hd] uint8, scale [n, kv, L/block] fp64 (both changed in place), x [rows, kv, hd]."""
    n, kv = codes.shape[:2]
    for s in range(n):
        rows = x[offsets[s]:offsets[s + 1]].double()
        c, m = cached[s], offsets[s + 1] - offsets[s]
        if m == 0:
            continue
        for h in range(kv):
            for b in range(c // block, (c + m - 1) // block + 1):
                lo, hi = max(c, b * block), min(c + m, (b + 1) * block)
                part = rows[lo - c:hi - c, h]
                fin = part[part.isfinite()].abs()
                sc = least_scale(float(fin.max()) if fin.numel() else 0.0)
                if lo > b * block:
                    old = float(scale[s, h, b])
                    sc = max(sc, old)
                    codes[s, h, b * block:lo] = encode(TABLE[codes[s, h, b * block:lo].long()] * (old / sc))
                scale[s, h, b] = sc
                codes[s, h, lo:hi] = encode(part / sc)


def values(codes, scale, block):
    return TABLE[codes.long()] * scale.double().repeat_interleave(block, -1)[..., None]


def attend(codes_k, scale_k, codes_v, scale_v, q, cached, offsets, block, weight_in=None, softmax_scale=None):
    """(out [rows, heads, hd], weight [n, kv, L], spread [rows, heads, hd], mag [rows, heads]): spread is sum_j p_j |v_j|,
    mag the largest sum_i |q_i k_ji| * softmax_scale, for error bounds.  Slots that nobody holds: weight NaN."""
    n, kv, L, hd = codes_k.shape
    rows, heads = q.shape[0], q.shape[1]
    g = heads // kv
    scale = softmax_scale if softmax_scale else 1 / math.sqrt(hd)
    out = torch.full((rows, heads, hd), math.nan, dtype=torch.float64)
    spread, mag = torch.zeros_like(out), torch.zeros((rows, heads), dtype=torch.float64)
    weight = torch.full((n, kv, L), math.nan, dtype=torch.float64)
    for s in range(n):
        c, m = cached[s], offsets[s + 1] - offsets[s]
        k = values(codes_k[s], scale_k[s], block)[:, :c + m]
        v = values(codes_v[s], scale_v[s], block)[:, :c + m]
        weight[s, :, :c + m] = 0
        if weight_in is not None:
            weight[s, :, :c] = weight_in[s, :, :c].double()
        for h in range(heads):
            x = q[offsets[s]:offsets[s] + m, h].double()
            z = x @ k[h // g].T * scale
            sees = torch.arange(c + m)[None, :] <= c + torch.arange(m)[:, None]
            z = z.masked_fill(~sees, -math.inf)
            p = torch.softmax(z, -1) if m else z
            out[offsets[s]:offsets[s] + m, h] = p @ v[h // g]
            spread[offsets[s]:offsets[s] + m, h] = p @ v[h // g].abs()
            if m:
                mag[offsets[s]:offsets[s] + m, h] = (x.abs() @ k[h // g].abs().T * scale).amax(-1)
            weight[s, h // g, :c + m] += p.sum(0)
    return out, weight, spread, mag


def evict(codes, scales, weight, position, held, keep, recent, next_position, block):
    """codes = (k, v), scales = (k, v) changed in place; returns (weight_out, position_out, kept) with NaN / -1 where
    nothing is written."""
    n, kv, L = weight.shape
    w_out = torch.full((n, kv, keep), math.nan, dtype=torch.float64)
    p_out = torch.full((n, kv, keep), -1, dtype=torch.int64)
    kept = torch.full((n, kv, keep), -1, dtype=torch.int64)
    for s in range(n):
        for h in range(kv):
            m = held[s]
            now = list(range(min(m, keep)))
            if m > keep:
                w, pos = weight[s, h, :m].tolist(), position[s, h, :m].tolist()
                young = [recent > 0 and p >= next_position[s] - recent for p in pos]
                order = sorted(range(m), key=lambda i: (not young[i], math.isnan(w[i]) and not young[i],
                                                        0.0 if young[i] or math.isnan(w[i]) else -w[i], i))
                stay = set(order[:keep])
                come = iter(sorted(i for i in stay if i >= keep))
                for i in range(keep):
                    if i not in stay:
                        now[i] = next(come)
            for i, f in enumerate(now):
                kept[s, h, i], w_out[s, h, i], p_out[s, h, i] = f, weight[s, h, f], position[s, h, f]
            if m <= keep:
                continue
            for c, sc in zip(codes, scales):
                for b in range(keep // block):
                    part = now[b * block:(b + 1) * block]
                    old = float(sc[s, h, b])
                    top = max([old] + [float(sc[s, h, f // block]) for f in part])
                    for i, f in enumerate(part):
                        c[s, h, b * block + i] = encode(TABLE[c[s, h, f].long()] * (float(sc[s, h, f // block]) / top))
                    sc[s, h, b] = top
    return w_out, p_out, kept
