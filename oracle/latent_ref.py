"""Independent reference of rotary positions and of attention over a latent cache (test infrastructure only): fp64 on the CPU,
pair by pair and sequence by sequence, no code shared with the library."""
from __future__ import annotations

import math

import torch


def frequencies(rot, theta, factor=1.0, original_len=0, low=1.0, high=32.0):
    out = []
    for i in range(rot // 2):
        w = theta ** (-2.0 * i / rot)
        keep = 0.0
        if original_len:
            keep = min(1.0, max(0.0, (original_len * w / (2 * math.pi) - low) / (high - low)))
        out.append(w * (keep + (1 - keep) / factor))
    return out


def rotate(x, positions, rot, theta, first=0, interleaved=False, factor=1.0, original_len=0, low=1.0, high=32.0, magnitude=1.0):
    """x [rows, heads, head_dim] (any type) -> fp64; positions: whole numbers."""
    out = x.double().clone()
    for i, w in enumerate(frequencies(rot, theta, factor, original_len, low, high)):
        a, b = (first + 2 * i, first + 2 * i + 1) if interleaved else (first + i, first + i + rot // 2)
        t = positions.double() * w
        c, s = torch.cos(t)[:, None] * magnitude, torch.sin(t)[:, None] * magnitude
        out[:, :, a], out[:, :, b] = x[:, :, a].double() * c - x[:, :, b].double() * s, x[:, :, b].double() * c + x[:, :, a].double() * s
    return out


def append(rows, x, cached, offsets, latent, norm=None, eps=0.0, rope=None, position=None, max_len=None):
    """rows [n_seq, max_len, latent + rope] fp64, changed in place.  position: of each sequence's first new token."""
    for s in range(rows.shape[0]):
        for i in range(offsets[s + 1] - offsets[s]):
            slot = cached[s] + i
            if slot >= rows.shape[1]:
                break
            v = x[offsets[s] + i].double()
            c, p = v[:latent], v[latent:]
            if norm is not None:
                c = c / torch.sqrt((c * c).mean() + eps) * norm.double()
            if rope is not None:
                p = rotate(p[None, None], torch.tensor([position[s] + i]), **rope)[0, 0]
            rows[s, slot] = torch.cat((c, p))


def attend(rows, q, w_k, w_v, cached, offsets, prefix=None, scale=None):
    """(out [rows, heads, v], spread, wide, mag): spread is sum_j p_j |v_j|, wide |w_v| sum_j p_j |c_j|; mag[form] [rows, heads] the largest
    sum of magnitudes behind a score, of the terms as the form (absorbed, expanded) has them; all for error bounds.  Rows of no
    sequence: NaN."""
    heads, nope, latent = w_k.shape
    n_seq, max_len = rows.shape[:2]
    scale = scale or 1 / math.sqrt(q.shape[2])
    out = torch.full((q.shape[0], heads, w_v.shape[1]), math.nan, dtype=torch.float64)
    spread, wide = torch.zeros_like(out), torch.zeros_like(out)
    mag = {f: torch.zeros(out.shape[:2], dtype=torch.float64) for f in ("absorbed", "expanded")}
    w_k, w_v = w_k.double(), w_v.double()
    for s in range(n_seq):
        c, m = cached[s], min(offsets[s + 1] - offsets[s], max_len - cached[s])
        if m <= 0:
            continue
        x = rows[s, :c + m].double()
        before = 0
        if prefix is not None:
            x = torch.cat((prefix.double(), x))
            before = prefix.shape[0]
        at = slice(offsets[s], offsets[s] + m)
        for h in range(heads):
            k = torch.cat((x[:, :latent] @ w_k[h].T, x[:, latent:]), 1)
            v = x[:, :latent] @ w_v[h].T
            y = q[at, h].double()
            z = y @ k.T * scale
            late = torch.arange(before + c + m)[None, :] > before + c + torch.arange(m)[:, None]
            p = torch.softmax(z.masked_fill(late, -math.inf), -1)
            o = torch.where(late[:, :, None], torch.zeros((), dtype=torch.float64), p[:, :, None] * v[None]).sum(1) if not v.isfinite().all() else p @ v
            out[at, h] = o
            spread[at, h] = p @ v.abs()
            wide[at, h] = p @ x[:, :latent].abs() @ w_v[h].abs().T
            near = y[:, nope:].abs() @ x[:, latent:].abs().T
            big = {"absorbed": (y[:, :nope] @ w_k[h]).abs() @ x[:, :latent].abs().T, "expanded": y[:, :nope].abs() @ k[:, :nope].abs().T}
            for f in big:
                mag[f][at, h] = ((big[f] + near) * scale).masked_fill(late, 0).amax(-1)
    return out, spread, wide, mag
