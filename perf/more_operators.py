"""Rotary positions and attention over one shared latent vector a token, as cases that can be timed and checked: rotating
rows of queries and keys (rope), filling the latent cache (append), and attending over it (attend), for single tokens, for
prompts, and for batches that share a long prefix.

A latent cache holds, for every sequence and slot, one row of `latent` + `rope` elements in bf16: a latent vector c from which
all heads' keys and values are made, k = (w_k c, p) and v = w_v c, and the part p of the key that carries the position and that
the heads share.  The plain forms below are the operators' definitions in elementary torch operations; with `own` set, `run`
makes the calls of `paper_2502_06888_amd.rope_binding` and `paper_2502_06888_amd.latent_binding`.

Lengths are those of this repository's attention workloads: its decode group (512 sequences after 512-token prompts), prompts in
batches of 512 tokens and of about 4000, and conversations of thousands of positions.  Head layouts are those of its attention
workloads for the rotation, and generic for the latent cache: 8 to 128 heads over 512 + 64 elements, 16 over 256 + 32.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


# ---- cases -----------------------------------------------------------------------------------

def _rope(name, rows, heads, kv_heads, head_dim, rot, first, interleaved, dtype, far, factor=1.0, original=0):
    return dict(name=name, kind="rope", rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot=rot, first=first,
                interleaved=interleaved, dtype=dtype, far=far, factor=factor, original=original)


def _latent(name, kind, seqs, heads, dims, cached, new, prefix=0):
    """dims: latent, rope, key part without position, value; cached, new: (least, most) per sequence, spread over them."""
    return dict(name=name, kind=kind, seqs=seqs, heads=heads, latent=dims[0], rope=dims[1], nope=dims[2], value=dims[3],
                cached_lo=cached[0], cached_hi=cached[1], new_lo=new[0], new_hi=new[1], prefix=prefix)


WIDE, SMALL = (512, 64, 128, 128), (256, 32, 64, 64)


def listed():
    return [
        # one token of one conversation: latency counts
        _rope("rope_1", 1, 32, 8, 128, 128, 0, False, "bf16", 700),
        # a group of prompts at far positions, frequencies scaled by parts for a context 16 times as long
        _rope("rope_8192_scaled", 8192, 32, 8, 128, 128, 0, False, "bf16", 131072, 16.0, 8192),
        # queries of latent attention: the last third of each head, interleaved pairs; one shared key
        _rope("rope_part_2051_f32", 2051, 20, 1, 192, 64, 128, True, "f32", 9000),
        # the decode group and ragged chunks of prompts being stored
        _latent("append_512x1", "append", 512, 32, WIDE, (512, 575), (1, 1)),
        _latent("append_37x449", "append", 37, 32, WIDE, (3, 900), (301, 597)),
        # one conversation, one token: latency counts
        _latent("decode_1x700", "attend", 1, 32, WIDE, (700, 700), (1, 1)),
        # the benchmark's decode group: 8 batches of 64 sequences after 512-token prompts
        _latent("decode_512x512", "attend", 512, 32, WIDE, (512, 512), (1, 1)),
        # requests of all ages in one batch, many heads
        _latent("decode_48x3000_128", "attend", 48, 128, WIDE, (1, 6001), (1, 1)),
        # two long prompts
        _latent("prompt_2x4096", "attend", 2, 32, WIDE, (0, 0), (3907, 4096)),
        # chunks of prompts behind what is cached already, ragged, smaller heads
        _latent("chunk_3x533", "attend", 3, 16, SMALL, (0, 6001), (267, 800)),
        # a decode batch whose sequences began with the same long instruction
        _latent("prefix_64x4096", "attend", 64, 32, WIDE, (1, 500), (1, 1), prefix=4096),
        # prompts behind the same documents
        _latent("prefix_5x300", "attend", 5, 20, WIDE, (0, 0), (97, 300), prefix=8001),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "append", "decode", "decode", "decode", "prompt", "prompt", "prefix", "prefix"])
    if kind == "rope":
        heads, kv, hd = rng.choice([(32, 8, 128), (48, 8, 128), (16, 8, 128), (32, 8, 64), (16, 16, 64), (8, 4, 32), (20, 1, 192), (5, 0, 96)])
        rot = rng.choice([hd, hd // 2, 32, 2 * rng.randint(1, hd // 2)])
        far, factor = _log_int(rng, 1, 1 << 20), rng.choice([1.0, 1.0, 4.0, 32.0])
        return _drop(_rope("", _log_int(rng, 1, 16384), heads, kv, hd, rot, rng.choice([0, hd - rot]), rng.random() < 0.5,
                           rng.choice(["bf16", "bf16", "f32"]), far, factor, rng.choice([0, 4096]) if factor > 1 else 0))
    heads, dims = rng.choice([(8, WIDE), (20, WIDE), (32, WIDE), (40, WIDE), (128, WIDE), (16, SMALL), (5, SMALL), (16, (512, 64, 64, 64)),
                              (32, (128, 32, 32, 64))])
    seqs = _log_int(rng, 1, 512)
    if kind == "append":
        new = _log_int(rng, 1, max(1, min(4096, 32768 // seqs)))
        before = rng.randint(0, 600)
        return _drop(_latent("", "append", seqs, heads, dims, (before // 2, before), (rng.randint(0, new), new)))
    if kind == "decode":
        hi = _log_int(rng, 1, max(1, min(32000, 262144 // seqs)))
        return _drop(_latent("", "attend", seqs, heads, dims, (rng.randint(0, hi), hi), (1, rng.choice([1, 1, 1, 2, 4]) if heads <= 40 else 1)))
    seqs = min(seqs, 32)
    new = _log_int(rng, 2, max(2, min(4096, 8192 // seqs)))
    if kind == "prompt":
        before = rng.choice([0, 0, rng.randint(1, max(1, min(4000, 16384 // seqs)))])
        if seqs * heads * new * (new + 2 * before) > 2 * 32 * 4096 * 4096:
            before, new = 0, min(new, 700)
        return _drop(_latent("", "attend", seqs, heads, dims, (before // 2, before), (rng.randint(1, new), new)))
    prefix = _log_int(rng, 1, 16384)
    if rng.random() < 0.5 or seqs * heads * new * (2 * prefix + new) > 2 * 32 * 4096 * 4096:
        own_len = rng.randint(0, 600)
        return _drop(_latent("", "attend", min(4 * seqs, max(1, 524288 // prefix)), heads, dims, (own_len // 3, own_len), (1, 1), prefix))
    return _drop(_latent("", "attend", seqs, heads, dims, (0, 0), (rng.randint(1, new), new), prefix))


def _drop(case):
    case.pop("name")
    return case


def _spread(lo, hi, n):
    """n whole numbers from lo to hi in no order, the first one hi."""
    return [hi - int((hi - lo + 1) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _lengths(case):
    return (_spread(case["cached_lo"], case["cached_hi"], case["seqs"]),
            _spread(case["new_lo"], case["new_hi"], case["seqs"]))


# ---- inputs ----------------------------------------------------------------------------------

def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _settings(case):
    """What a model's configuration says of its rotation."""
    if case["kind"] == "rope":
        return dict(rot_dim=case["rot"], theta=1e6, first=case["first"], interleaved=case["interleaved"], factor=case["factor"],
                    original_len=case["original"], magnitude=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0)
    return dict(rot_dim=case["rope"], theta=1e4, interleaved=True)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    st = dict(case=case)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)

    if case["kind"] == "rope":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        st["positions"] = torch.randint(0, case["far"] + 1, (case["rows"],), generator=g, device=DEV, dtype=torch.int32)
        st["q"] = normal(case["rows"], case["heads"], case["head_dim"], dtype=dtype)
        st["q_out"] = torch.zeros_like(st["q"])
        st["k"] = st["k_out"] = None
        if case["kv_heads"]:
            st["k"] = normal(case["rows"], case["kv_heads"], case["head_dim"], dtype=dtype)
            st["k_out"] = torch.zeros_like(st["k"])
        if own:
            from paper_2502_06888_amd import rope_binding as R
            st["rope"] = R.Rope(**_settings(case))
        return st

    seqs, latent, rope = case["seqs"], case["latent"], case["rope"]
    cached, new = _lengths(case)
    st["max_len"] = st["most"] = max(1, max(c + n for c, n in zip(cached, new)))
    st["n_rows"], st["max_new"], st["max_cached"] = sum(new), max(new), max(cached)
    st["cached"], st["next"] = _int32(cached), _int32([c + case["prefix"] for c in cached])
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    st["offsets"], st["uniform"] = _int32(offsets), min(new) == max(new)
    rows = max(1, st["n_rows"])
    st["rows"] = normal(seqs, st["max_len"], latent + rope)
    st["prefix"] = normal(case["prefix"], latent + rope) if case["prefix"] else None
    if case["kind"] == "append":
        st["x"] = normal(rows, latent + rope, std=3.0)
        st["norm"] = (1 + 0.1 * torch.randn(latent, generator=g, device=DEV)).to(torch.bfloat16)
    else:
        heads = case["heads"]
        st["w_k"] = normal(heads, case["nope"], latent, std=latent ** -0.5)
        st["w_v"] = normal(heads, case["value"], latent, std=latent ** -0.5)
        # some heads look sharply, others broadly
        sharp = torch.exp(0.5 * torch.randn((heads, 1), generator=g, device=DEV))
        st["q"] = (torch.randn((rows, heads, case["nope"] + rope), generator=g, device=DEV) * sharp).to(torch.bfloat16)
        st["out"] = torch.zeros((rows, heads, case["value"]), dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2502_06888_amd import kv8_binding as Q
        from paper_2502_06888_amd import latent_binding as L
        st["cache"] = L.LatentCache(st["rows"], rope, prefix=st["prefix"])
        st["step"] = Q.Kv8Step(st["cached"], st["n_rows"], st["max_new"], st["max_cached"],
                               row_offsets=None if st["uniform"] else st["offsets"], next_position=st["next"])
        if case["kind"] == "append":
            from paper_2502_06888_amd import rope_binding as R
            st["rope"] = R.Rope(**_settings(case))
        else:
            st["heads"] = L.LatentHeads(st["w_k"], st["w_v"])
            st["workspace"] = L.attend_workspace(st["cache"], st["step"], st["heads"])
    return st


# ---- the operators ---------------------------------------------------------------------------

def run(st):
    return {"rope": _rotate, "append": _append, "attend": _attend}[st["case"]["kind"]](st)


def _frequencies(s):
    """Angle per position of each pair, in 64 bits."""
    rot = s["rot_dim"]
    w = s["theta"] ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if s.get("factor", 1.0) != 1.0:
        part = torch.zeros_like(w)
        if s["original_len"]:     # pairs that turn often over the original length keep their frequency
            part = ((w * (s["original_len"] / (2 * math.pi)) - 1.0) / 31.0).clamp(0, 1)
        w = w * (part + (1 - part) / s["factor"])
    return w


def _rotated(x, positions, s):
    """x [rows, heads, head_dim] in 32 bits, turned by its positions."""
    angle = positions.double()[:, None] * _frequencies(s)
    cos, sin = (f(angle).float().mul_(s.get("magnitude", 1.0))[:, None] for f in (torch.cos, torch.sin))
    first, rot = s.get("first", 0), s["rot_dim"]
    part = x[..., first:first + rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if s["interleaved"] else (part[..., :rot // 2], part[..., rot // 2:])
    c, d = a * cos - b * sin, b * cos + a * sin
    out = x.clone()
    out[..., first:first + rot] = torch.stack((c, d), -1).flatten(-2) if s["interleaved"] else torch.cat((c, d), -1)
    return out


def _rotate(st):
    if own:
        from paper_2502_06888_amd import rope_binding as R
        R.rotate(st["rope"], st["positions"], st["q"], q_out=st["q_out"], k=st["k"], k_out=st["k_out"])
        return (st["q_out"],) if st["k"] is None else (st["q_out"], st["k_out"])
    s = _settings(st["case"])
    outs = []
    for name in "qk":
        if st[name] is not None:
            st[name + "_out"].copy_(_rotated(st[name].float(), st["positions"], s))
            outs.append(st[name + "_out"])
    return tuple(outs)


def _places(st):
    """Sequence of each row of the new tokens, and its place among them."""
    row = torch.arange(st["n_rows"], device=DEV)
    seq = torch.searchsorted(st["offsets"][1:].long(), row, right=True)
    return seq, row - st["offsets"].long()[seq]


def _append(st):
    case = st["case"]
    if own:
        from paper_2502_06888_amd import latent_binding as L
        L.append(st["cache"], st["step"], st["x"], norm=st["norm"], eps=EPS, rope=st["rope"])
    elif st["n_rows"] > 0:
        latent = case["latent"]
        seq, at = _places(st)
        x = st["x"][:st["n_rows"]].float()
        c = x[:, :latent]
        c = c * torch.rsqrt(c.square().mean(-1, keepdim=True) + EPS) * st["norm"].float()
        p = _rotated(x[:, None, latent:], st["next"].long()[seq] + at, _settings(case))[:, 0]
        st["rows"][seq, st["cached"].long()[seq] + at] = torch.cat((c, p), -1).to(torch.bfloat16)
    return (st["rows"],)


def _attend(st):
    case = st["case"]
    if own:
        from paper_2502_06888_amd import latent_binding as L
        L.attend(st["cache"], st["step"], st["heads"], st["q"], st["out"], workspace=st["workspace"])
        return (st["out"],)
    seqs, heads, latent, nope, rope, value = (case[n] for n in ("seqs", "heads", "latent", "nope", "rope", "value"))
    prefix, n = case["prefix"], st["max_new"]
    seq, at = _places(st)
    q = torch.zeros((seqs, n, heads, nope + rope), device=DEV)
    q[seq, at] = st["q"][:st["n_rows"]].float()
    q = q.permute(0, 2, 1, 3)                                              # [seqs, heads, new, nope + rope]
    c = st["rows"][:, :st["most"]].float()
    if prefix:
        c = torch.cat((st["prefix"].float().expand(seqs, -1, -1), c), 1)
    slots = c.shape[1]
    flat = c.transpose(1, 2).contiguous()                                  # [seqs, latent + rope, slots]
    w_k, w_v = st["w_k"].float(), st["w_v"].float()
    near = torch.matmul(q[..., nope:].reshape(seqs, heads * n, rope), flat[:, latent:].contiguous())
    sees = prefix + st["cached"][:, None] + torch.arange(n, device=DEV) + 1
    hidden = (torch.arange(slots, device=DEV) >= sees[:, :, None])[:, None]
    many = n > 128                                                         # then keys and values are made for every head
    if many:
        k = torch.matmul(w_k.view(heads * nope, latent), flat[:, :latent]).view(seqs, heads, nope, slots)
        z = torch.matmul(q[..., :nope].contiguous(), k)
        del k
    else:
        a = torch.matmul(q[..., :nope].permute(1, 0, 2, 3).reshape(heads, seqs * n, nope), w_k)
        a = a.view(heads, seqs, n, latent).transpose(0, 1).reshape(seqs, heads * n, latent)
        z = torch.matmul(a, flat[:, :latent].contiguous()).view(seqs, heads, n, slots)
    z = z.add_(near.view(seqs, heads, n, slots)).mul_(1 / math.sqrt(nope + rope)).masked_fill_(hidden, -math.inf)
    del near
    p = torch.exp_(z.sub_(z.amax(-1, keepdim=True)))
    p = p.div_(p.sum(-1, keepdim=True))
    if many:
        v = torch.matmul(c[..., :latent].reshape(seqs * slots, latent), w_v.view(heads * value, latent).T.contiguous())
        o = torch.matmul(p, v.view(seqs, slots, heads, value).transpose(1, 2).contiguous())
    else:
        u = torch.matmul(p.view(seqs, heads * n, slots), c[..., :latent].contiguous())
        u = u.view(seqs, heads, n, latent).transpose(0, 1).reshape(heads, seqs * n, latent)
        o = torch.matmul(u, w_v.transpose(1, 2).contiguous()).view(heads, seqs, n, value).transpose(0, 1)
    out = torch.zeros_like(st["out"])
    out[:st["n_rows"]] = o.transpose(1, 2)[seq, at].to(torch.bfloat16)
    return (out,)


# ---- work --------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "rope":
        elements = case["rows"] * (case["heads"] + case["kv_heads"]) * case["head_dim"]
        turned = case["rows"] * (case["heads"] + case["kv_heads"]) * case["rot"]
        return {"bytes": elements * 2 * (2 if case["dtype"] == "bf16" else 4) + 4 * case["rows"], "flops": 3 * turned}
    cached, new = _lengths(case)
    heads, latent, rope, nope, value, prefix = (case[n] for n in ("heads", "latent", "rope", "nope", "value", "prefix"))
    width = latent + rope
    if case["kind"] == "append":
        return {"bytes": 4 * sum(new) * width, "flops": 6 * sum(new) * width}
    slots = prefix + sum(c + n for c, n in zip(cached, new) if n)
    pairs = sum(n * (prefix + c) + n * (n + 1) // 2 for c, n in zip(cached, new))
    size = 2 * (slots * width + sum(new) * heads * (nope + rope + value) + heads * (nope + value) * latent)
    # keys and values made for every slot, or queries and outputs brought into the latent space: whichever is less
    made = slots * heads * 2 * latent * (nope + value) + pairs * heads * 2 * (nope + rope + value)
    brought = sum(new) * heads * 2 * latent * (nope + value) + pairs * heads * 2 * (2 * latent + rope)
    return {"bytes": size, "flops": min(made, brought)}


# ---- the definition in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"rope": _rotate64, "append": _append64, "attend": _attend64}[case["kind"]](st, case)


def _turn64(x, positions, s):
    """x [rows, heads, head_dim] as complex numbers times e^(i angle), pair by pair."""
    rot, first = s["rot_dim"], s.get("first", 0)
    out = x.clone()
    for i in range(rot // 2):
        w = s["theta"] ** (-2.0 * i / rot)
        if s.get("factor", 1.0) != 1.0:
            keep = 0.0
            if s["original_len"]:
                keep = min(1.0, max(0.0, (s["original_len"] * w / (2 * math.pi) - 1.0) / (32.0 - 1.0)))
            w = keep * w + (1.0 - keep) * w / s["factor"]
        a, b = (first + 2 * i, first + 2 * i + 1) if s["interleaved"] else (first + i, first + i + rot // 2)
        turn = torch.polar(torch.full_like(positions, s.get("magnitude", 1.0)), positions * w)
        z = torch.complex(x[..., a], x[..., b]) * turn[:, None]
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _rotate64(st, case):
    s, positions = _settings(case), st["positions"].double()
    return tuple(_turn64(st[n].double(), positions, s) for n in "qk" if st[n] is not None)


def _append64(st, case):
    cached, new = _lengths(case)
    latent, row = case["latent"], 0
    out = st["rows"].double()
    for s, (c, n) in enumerate(zip(cached, new)):
        if n == 0:
            continue
        x = st["x"][row:row + n].double()
        row += n
        norm = torch.sqrt((x[:, :latent] ** 2).sum(1, keepdim=True) / latent + EPS)
        positions = torch.arange(n, device=DEV, dtype=torch.float64) + (c + case["prefix"])
        out[s, c:c + n, :latent] = x[:, :latent] / norm * st["norm"].double()
        out[s, c:c + n, latent:] = _turn64(x[:, None, latent:], positions, _settings(case))[:, 0]
    return (out,)


def _attend64(st, case):
    cached, new = _lengths(case)
    heads, latent, nope, prefix = case["heads"], case["latent"], case["nope"], case["prefix"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    w_k, w_v = st["w_k"].double(), st["w_v"].double()
    shared = st["prefix"].double() if prefix else None
    row = 0
    for s, (c, n) in enumerate(zip(cached, new)):
        if n == 0:
            continue
        x = st["rows"][s, :c + n].double()
        if prefix:
            x = torch.cat((shared, x))
        q = st["q"][row:row + n].double()
        late = torch.arange(x.shape[0], device=DEV)[None, :] > prefix + c + torch.arange(n, device=DEV)[:, None]
        step = max(1, (1 << 27) // (n * x.shape[0] + x.shape[0] * (nope + case["value"])))   # heads at a time
        lat = x[:, :latent].T.contiguous()
        for h in range(0, heads, step):
            k = torch.matmul(w_k[h:h + step], lat)                           # [some heads, nope, slots]
            v = torch.matmul(w_v[h:h + step], lat).transpose(1, 2).contiguous()
            y = q[:, h:h + step].transpose(0, 1).contiguous()
            z = torch.matmul(y[..., :nope].contiguous(), k) + torch.matmul(y[..., nope:].contiguous(), x[:, latent:].T.contiguous())
            p = torch.softmax((z / math.sqrt(q.shape[-1])).masked_fill(late, -math.inf), -1)
            out[row:row + n, h:h + step] = torch.matmul(p, v).transpose(0, 1)
        row += n
    return (out,)
