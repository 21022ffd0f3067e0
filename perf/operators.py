"""The key-value cache held in 8 bits, as cases that can be timed and checked: filling it (append), attending
over it (attend) and evicting from it by accumulated attention weight (evict).

A cache holds, for every sequence and key-value head, `max_len` slots of `head_dim` elements as e4m3 codes, and one
scale, a power of two, for each block of slots; the value of a code is code * scale.  The plain forms below are the
operators' definitions in elementary torch operations; with `own` set, `run` makes the calls of
`paper_2502_06888_amd.kv8_binding`.

Head layouts are those of this repository's attention workloads (32/8, 48/8 and 16/8 heads of 128, 32/8 of 64) and a
layer without shared heads; lengths are those of its decode group (512 sequences after 512-token prompts), prompts
(batches of 512 tokens) and long conversations (4 sequences of about 8000 positions).

Codes are returned as float8_e4m3fn tensors, so as the numbers they are, with the scales beside them.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
MAX_CODE = 448.0                  # largest finite e4m3 number
SCALE_EXP = (-100, 119)           # exponents of a scale: dequantised values stay normal and finite in bf16


# ---- cases -----------------------------------------------------------------------------------

def _case(name, kind, seqs, heads, kv_heads, head_dim, block, cached, new=(0, 0), **more):
    """cached, new: (least, most) per sequence, spread over the sequences."""
    return dict(name=name, kind=kind, seqs=seqs, heads=heads, kv_heads=kv_heads, head_dim=head_dim, block=block,
                cached_lo=cached[0], cached_hi=cached[1], new_lo=new[0], new_hi=new[1], **more)


def listed():
    return [
        # one conversation, one token: latency counts
        _case("decode_1x700", "attend", 1, 32, 8, 128, 32, (700, 700), (1, 1), weights=False),
        # the benchmark's decode group: 8 batches of 64 sequences after 512-token prompts
        _case("decode_512x512", "attend", 512, 32, 8, 128, 64, (512, 512), (1, 1), weights=False),
        # a few long conversations whose cache will be evicted from: weights summed
        _case("decode_4x8000_weights", "attend", 4, 48, 8, 128, 64, (7003, 8000), (1, 1), weights=True),
        # requests of all ages in one batch, small heads
        _case("decode_96x1500_weights", "attend", 96, 32, 8, 64, 16, (1, 3001), (1, 1), weights=True),
        # the benchmark's prompt batches: 32 prompts of 512 tokens into an empty cache
        _case("prompt_32x512", "attend", 32, 32, 8, 128, 64, (0, 0), (512, 512), weights=False),
        # two long prompts
        _case("prompt_2x4096", "attend", 2, 32, 8, 128, 128, (0, 0), (3907, 4096), weights=False),
        # chunks of prompts behind what is cached already, ragged, weights summed
        _case("chunk_3x533_weights", "attend", 3, 16, 8, 128, 32, (0, 6001), (267, 800), weights=True),
        # the same prompts and decode group being stored, and ragged chunks
        _case("append_32x512", "append", 32, 32, 8, 128, 64, (0, 0), (512, 512)),
        _case("append_512x1", "append", 512, 32, 8, 128, 64, (512, 575), (1, 1)),
        _case("append_7x229", "append", 7, 32, 8, 64, 16, (3, 900), (11, 447)),
        # the decode group brought back to 512 slots; long conversations cut to half
        _case("evict_512x576", "evict", 512, 32, 8, 128, 64, (513, 576), keep=512, recent=64),
        _case("evict_4x8000", "evict", 4, 48, 8, 128, 64, (7003, 8000), keep=4096, recent=256),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "prompt", "prompt", "append", "evict"])
    heads, kv, hd = rng.choice([(32, 8, 128), (48, 8, 128), (16, 8, 128), (32, 8, 64), (16, 16, 64), (8, 4, 32)])
    block = rng.choice([16, 32, 64, 128])
    seqs = _log_int(rng, 1, 512)
    if kind == "decode":
        hi = _log_int(rng, 1, max(1, min(32000, 262144 // seqs)))
        return _drop(_case("", "attend", seqs, heads, kv, hd, block, (rng.randint(0, hi), hi), (1, rng.choice([1, 1, 1, 2, 4])),
                           weights=rng.random() < 0.5))
    if kind == "prompt":
        seqs = min(seqs, 32)
        new = _log_int(rng, 2, max(2, min(4096, 16384 // seqs)))
        before = rng.choice([0, 0, rng.randint(1, max(1, min(4000, 16384 // seqs)))])
        if seqs * heads * new * (new + before) > 2 * 32 * 4096 * 4096:
            before = 0
        return _drop(_case("", "attend", seqs, heads, kv, hd, block, (before // 2, before), (rng.randint(1, new), new),
                           weights=rng.random() < 0.5))
    if kind == "append":
        new = _log_int(rng, 1, max(1, min(4096, 32768 // seqs)))
        before = rng.randint(0, 600)
        return _drop(_case("", "append", seqs, heads, kv, hd, block, (before // 2, before), (rng.randint(0, new), new)))
    hi = _log_int(rng, block + 1, max(block + 1, min(32000, 262144 // seqs)))
    keep = block * rng.randint(1, max(1, hi // block))
    return _drop(_case("", "evict", seqs, heads, kv, hd, block, (rng.randint(0, hi), hi), keep=keep,
                       recent=rng.randint(0, keep)))


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

def _power(e):
    """2^e in 32 bits, from its bits (ldexp takes a power that is not exact everywhere)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _least_scale(largest):
    """The least power of two s with largest <= MAX_CODE * s, in the range of the exponents."""
    m, e = torch.frexp(largest)                       # largest = m * 2^e, 0.5 <= m < 1;  448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(largest > 0, e, torch.full_like(e, SCALE_EXP[0])).clamp(*SCALE_EXP)
    return _power(e)


def _codes(x, scale):
    """x / scale as e4m3 numbers, rounded to nearest even; what is too large becomes the largest."""
    return (x / scale).clamp(-MAX_CODE, MAX_CODE).to(torch.float8_e4m3fn)


def _filled(g, seqs, kv, max_len, hd, block):
    """Codes and scales of a cache that holds normal draws, some channels wider than others."""
    wide = torch.exp(0.5 * torch.randn((1, kv, 1, hd), generator=g, device=DEV))
    codes = torch.empty((seqs, kv, max_len, hd), dtype=torch.uint8, device=DEV)
    scale = torch.empty((seqs, kv, max_len // block), device=DEV)
    step = max(1, (1 << 26) // (kv * max_len * hd))   # sequences at a time
    for s in range(0, seqs, step):
        x = torch.randn((min(step, seqs - s), kv, max_len, hd), generator=g, device=DEV) * wide
        b = x.view(x.shape[0], kv, max_len // block, block * hd)
        sc = _least_scale(b.abs().amax(-1))
        codes[s:s + step] = _codes(b, sc[..., None]).view(x.shape).view(torch.uint8)
        scale[s:s + step] = sc
    return codes, scale


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    seqs, kv, hd, block = case["seqs"], case["kv_heads"], case["head_dim"], case["block"]
    cached, new = _lengths(case)
    most = max(c + n for c, n in zip(cached, new))
    max_len = max(1, -(-most // block)) * block
    st = dict(case=case, max_len=max_len, most=most, max_new=max(new), max_cached=max(cached), n_rows=sum(new))
    st["k"], st["k_scale"] = _filled(g, seqs, kv, max_len, hd, block)
    st["v"], st["v_scale"] = _filled(g, seqs, kv, max_len, hd, block)
    st["cached"] = _int32(cached)
    if case["kind"] == "evict":
        # sums of softmax weights: most slots got little, some much; half of the conversation has been evicted from
        u = torch.rand((seqs, kv, max_len), generator=g, device=DEV).clamp_min(1e-7)
        st["weight_in"] = (-torch.log(u)) ** 3
        st["weight_out"] = torch.zeros_like(st["weight_in"])
        order = torch.rand((seqs, kv, max_len), generator=g, device=DEV).argsort(-1).to(torch.int32)
        st["position"] = torch.where(order * 2 < max_len, order, order + 1000)
        st["position_out"] = torch.zeros_like(st["position"])
        st["next"] = _int32([max_len + 1000] * seqs)
        st["kept"] = torch.full((seqs, kv, case["keep"]), -1, dtype=torch.int32, device=DEV)
    else:
        offsets = [0]
        for n in new:
            offsets.append(offsets[-1] + n)
        st["offsets"] = _int32(offsets)
        st["uniform"] = min(new) == max(new)
        st["next"] = st["cached"] + 17
        rows = max(1, st["n_rows"])
        if case["kind"] == "append":
            st["k_new"] = torch.randn((rows, kv, hd), generator=g, device=DEV).to(torch.bfloat16)
            st["v_new"] = torch.randn((rows, kv, hd), generator=g, device=DEV).to(torch.bfloat16)
            st["position"] = torch.zeros((seqs, kv, max_len), dtype=torch.int32, device=DEV)
        else:
            st["q"] = torch.randn((rows, case["heads"], hd), generator=g, device=DEV).to(torch.bfloat16)
            st["out"] = torch.zeros((rows, case["heads"], hd), dtype=torch.bfloat16, device=DEV)
            if case["weights"]:
                st["weight_in"] = torch.rand((seqs, kv, max_len), generator=g, device=DEV)
                st["weight_out"] = torch.zeros_like(st["weight_in"])
    if own:
        from paper_2502_06888_amd import kv8_binding as Q
        st["cache"] = Q.Kv8Cache(st["k"], st["v"], st["k_scale"], st["v_scale"], block, position=st.get("position"))
        if case["kind"] == "evict":
            st["workspace"] = Q.evict_workspace(st["cache"], case["keep"])
        else:
            st["step"] = Q.Kv8Step(st["cached"], st["n_rows"], st["max_new"], st["max_cached"],
                                   row_offsets=None if st["uniform"] else st["offsets"], next_position=st["next"])
        if case["kind"] == "attend":
            st["workspace"] = Q.attend_workspace(st["cache"], st["step"], case["heads"], case["weights"])
    return st


# ---- the operators ---------------------------------------------------------------------------

def run(st):
    return {"append": _append, "attend": _attend, "evict": _evict}[st["case"]["kind"]](st)


def _values(codes, scale, block, slots):
    """The numbers that the first `slots` slots hold."""
    return codes[:, :, :slots].view(torch.float8_e4m3fn).float() * scale.repeat_interleave(block, 2)[:, :, :slots, None]


def _rows(st):
    """Sequence of each row of the new tokens, and its place among them."""
    row = torch.arange(st["n_rows"], device=DEV)
    seq = torch.searchsorted(st["offsets"][1:].long(), row, right=True)
    return seq, row - st["offsets"].long()[seq]


def _append(st):
    case = st["case"]
    block, kv, hd = case["block"], case["kv_heads"], case["head_dim"]
    if own:
        from paper_2502_06888_amd import kv8_binding as Q
        Q.append(st["cache"], st["step"], st["k_new"], st["v_new"])
    elif st["n_rows"] > 0:
        seq, at = _rows(st)
        cached = st["cached"].long()
        slot = cached[seq] + at
        which = torch.arange(case["seqs"], device=DEV)
        part = (cached // block).clamp(max=st["max_len"] // block - 1)     # block that may hold tokens already
        inside = cached - part * block                                     # how many
        for codes, scales, x in ((st["k"], st["k_scale"], st["k_new"]), (st["v"], st["v_scale"], st["v_new"])):
            x = x[:st["n_rows"]].float()
            flat = scales.permute(0, 2, 1).reshape(-1, kv)                 # one row for each (sequence, block)
            place = seq * flat.shape[0] // case["seqs"] + slot // block
            largest = torch.zeros_like(flat).scatter_reduce(0, place[:, None].expand(-1, kv), x.abs().amax(-1), "amax")
            touched = torch.zeros_like(flat[:, 0], dtype=torch.bool).index_fill(0, place, True)
            begun = torch.zeros_like(touched).view(case["seqs"], -1)
            begun[which, part] = inside > 0
            before = torch.where(begun.view(-1, 1), flat, torch.zeros_like(flat))
            after = torch.where(touched[:, None], torch.maximum(_least_scale(largest), before), flat)
            after = after.view(case["seqs"], -1, kv).permute(0, 2, 1)
            old, now = scales[which, :, part], after[which, :, part]       # [seqs, kv]
            span = part[:, None] * block + torch.arange(block, device=DEV)
            here = codes[which[:, None], :, span]                          # [seqs, block, kv, hd]
            again = _codes(here.view(torch.float8_e4m3fn).float() * old[:, None, :, None], now[:, None, :, None])
            keeps = (torch.arange(block, device=DEV) < inside[:, None])[:, :, None, None]
            codes[which[:, None], :, span] = torch.where(keeps, again.view(torch.uint8), here)
            scales.copy_(after)
            codes[seq, :, slot] = _codes(x, after[seq, :, slot // block][..., None]).view(torch.uint8)
        st["position"][seq, :, slot] = (st["next"].long()[seq] + at).to(torch.int32)[:, None].expand(-1, kv)
    return (st["k"].view(torch.float8_e4m3fn), st["v"].view(torch.float8_e4m3fn), st["k_scale"], st["v_scale"], st["position"])


def _attend(st):
    case = st["case"]
    seqs, heads, kv, hd, block = case["seqs"], case["heads"], case["kv_heads"], case["head_dim"], case["block"]
    if own:
        from paper_2502_06888_amd import kv8_binding as Q
        Q.attend(st["cache"], st["step"], st["q"], st["out"], weight_in=st.get("weight_in"), weight_out=st.get("weight_out"),
                 workspace=st["workspace"])
        return (st["out"], st["weight_out"]) if case["weights"] else (st["out"],)
    out = torch.zeros_like(st["out"])
    seq, at = _rows(st)
    k, v = (_values(st[n], st[n + "_scale"], block, st["most"]) for n in "kv")
    q = torch.zeros((seqs, st["max_new"], heads, hd), device=DEV)
    q[seq, at] = st["q"][:st["n_rows"]].float()
    q = q.view(seqs, st["max_new"], kv, heads // kv, hd).permute(0, 2, 3, 1, 4).reshape(seqs, kv, -1, hd)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(seqs, kv, heads // kv, st["max_new"], -1).mul_(1 / math.sqrt(hd))
    rows = torch.arange(st["max_new"], device=DEV)
    sees = st["cached"][:, None] + rows + 1                                # slots that a row sees
    there = rows < (st["offsets"][1:] - st["offsets"][:-1])[:, None]
    hidden = (torch.arange(st["most"], device=DEV) >= sees[:, :, None]) | ~there[:, :, None]
    hidden = hidden[:, None, None]
    s = s.masked_fill_(hidden, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp_(s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)))
    p = p.div_(p.sum(-1, keepdim=True).clamp_min(1e-30))
    o = torch.matmul(p.view(seqs, kv, -1, st["most"]), v).view(seqs, kv, heads // kv, st["max_new"], hd)
    o = o.permute(0, 3, 1, 2, 4).reshape(seqs, st["max_new"], heads, hd)
    out[:st["n_rows"]] = o[seq, at].to(torch.bfloat16)
    if not case["weights"]:
        return (out,)
    slots = torch.arange(st["max_len"], device=DEV)
    new = st["offsets"][1:] - st["offsets"][:-1]
    weight = torch.where(slots < st["cached"][:, None, None], st["weight_in"], torch.zeros_like(st["weight_in"]))
    weight[:, :, :st["most"]] += p.sum((2, 3))
    return out, torch.where(slots < (st["cached"] + new)[:, None, None], weight, torch.zeros_like(weight))


def _evict(st):
    case = st["case"]
    block, keep = case["block"], case["keep"]
    if own:
        from paper_2502_06888_amd import kv8_binding as Q
        Q.evict(st["cache"], st["cached"], st["max_cached"], keep, case["recent"], st["next"], st["weight_in"], st["weight_out"],
                position_out=st["position_out"], kept=st["kept"], workspace=st["workspace"])
        return (st["k"].view(torch.float8_e4m3fn), st["v"].view(torch.float8_e4m3fn), st["k_scale"], st["v_scale"],
                st["weight_out"], st["position_out"], st["kept"])
    n = min(keep, st["max_len"])
    slot = torch.arange(st["max_len"], device=DEV)
    held = st["cached"][:, None, None]
    key = torch.where(st["position"] >= st["next"][:, None, None] - case["recent"], torch.full_like(st["weight_in"], math.inf),
                      st["weight_in"])
    key = torch.where(slot < held, key, torch.full_like(key, -math.inf))
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :, :n]
    chosen = torch.zeros_like(key, dtype=torch.bool).scatter(2, best, True) & (slot < held)
    hole = ~chosen & (slot < keep) & (held > keep)
    source = chosen & (slot >= keep)
    rank = torch.where(source, source.cumsum(-1) - 1, torch.full_like(best[:, :, :1], st["max_len"]))
    moved = torch.zeros(key.shape[:2] + (st["max_len"] + 1,), dtype=torch.long, device=DEV)
    moved.scatter_(2, rank, slot.expand(key.shape).contiguous())
    kept = torch.where(hole, moved.gather(2, (hole.cumsum(-1) - 1).clamp_min(0)), slot)[:, :, :n]
    there = (slot < held)[:, :, :n].expand(kept.shape)
    weight, position = torch.zeros_like(st["weight_out"]), torch.zeros_like(st["position_out"])
    weight[:, :, :n] = torch.where(there, st["weight_in"].gather(2, kept), weight[:, :, :n])
    position[:, :, :n] = torch.where(there, st["position"].gather(2, kept), position[:, :, :n])
    outs = []
    for codes, scales in ((st["k"], st["k_scale"]), (st["v"], st["v_scale"])):
        codes, scales = codes.clone(), scales.clone()
        came = torch.where(there, scales.gather(2, kept // block), torch.zeros_like(scales[:, :, :1]))
        blocks = scales[:, :, :n // block]
        blocks.copy_(torch.maximum(blocks, came.view(blocks.shape + (block,)).amax(-1)))
        x = codes.gather(2, kept[..., None].expand(kept.shape + codes.shape[3:])).view(torch.float8_e4m3fn).float()
        x = _codes(x * came[..., None], blocks.repeat_interleave(block, 2)[..., None])
        codes[:, :, :n] = torch.where(there[..., None], x.view(torch.uint8), codes[:, :, :n])
        outs.append((codes.view(torch.float8_e4m3fn), scales))
    result = torch.full_like(st["kept"], -1)
    result[:, :, :n] = torch.where(there, kept, torch.full_like(kept, -1)).to(torch.int32)
    return outs[0][0], outs[1][0], outs[0][1], outs[1][1], weight, position, result


# ---- work --------------------------------------------------------------------------------------

def work(case):
    cached, new = _lengths(case)
    heads, kv, hd, block = case["heads"], case["kv_heads"], case["head_dim"], case["block"]
    if case["kind"] == "append":
        # new rows in (bf16), their codes and positions out, the block begun before read and its scale written
        return {"bytes": sum(new) * kv * (2 * hd * (2 + 1) + 4) + sum(-(-n // block) for n in new) * kv * 8, "flops": 0}
    if case["kind"] == "attend":
        slots = sum(c + n for c, n in zip(cached, new) if n)
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cached, new))
        size = slots * kv * (2 * hd + 8 / block) + 4 * sum(new) * heads * hd
        if case["weights"]:
            size += (sum(c + n for c, n in zip(cached, new)) + sum(cached)) * kv * 4
        return {"bytes": size, "flops": 4 * hd * heads * pairs}
    size = 0.0
    for c in cached:
        n = min(c, case["keep"])
        # weights and positions in and out, the list of what is kept; about as many slots move as have to
        moved = max(0, c - case["keep"]) * n / max(1, c)
        size += kv * (8 * c + 12 * n + 4 * hd * moved)
    return {"bytes": size, "flops": 0}


# ---- the definition in 64 bits -------------------------------------------------------------------

def _e4m3(x):
    """Nearest e4m3 number (ties to even): three bits behind the leading one, steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(x)
    step = ((e.long() - 1).clamp_min(-6) - 3 + 1023 << 52).view(torch.float64)
    return (torch.round(x / step) * step).clamp(-MAX_CODE, MAX_CODE)


def _scale64(largest):
    """Least power of two that brings `largest` (a number) to 448 or less."""
    if largest <= 0:
        return 2.0 ** SCALE_EXP[0]
    e = math.ceil(math.log2(largest / MAX_CODE) - 1e-9)
    while largest > MAX_CODE * 2.0 ** e:
        e += 1
    while largest <= MAX_CODE * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** min(max(e, SCALE_EXP[0]), SCALE_EXP[1])


def _decode(codes):
    """e4m3 codes as numbers, from the format: sign, four bits of exponent (bias 7), three of fraction."""
    table = [(-1.0 if c > 127 else 1.0) * math.ldexp(*((8 + c % 8, c // 8 % 16 - 10) if c // 8 % 16 else (c % 8, -9)))
             for c in range(256)]
    return torch.tensor(table, dtype=torch.float64, device=DEV)[codes.long()]


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _append64, "attend": _attend64, "evict": _evict64}[case["kind"]](st, case)


def _append64(st, case):
    cached, new = _lengths(case)
    block, kv = case["block"], case["kv_heads"]
    if sum(-(-n // block) + 1 for n in new) * kv > 40000:   # blocks one by one would take too long
        return None
    outs = []
    for name in "kv":
        values, scales = _decode(st[name]), st[name + "_scale"].double()
        row = 0
        for s, (c, n) in enumerate(zip(cached, new)):
            x = st[name + "_new"][row:row + n].double().transpose(0, 1)     # [kv, n, hd]
            row += n
            for b in range(c // block, -(-(c + n) // block) if n else 0):
                lo, hi = max(c, b * block), min(c + n, (b + 1) * block)
                part = x[:, lo - c:hi - c]
                least = torch.tensor([_scale64(a) for a in part.abs().amax((1, 2)).tolist()], dtype=torch.float64, device=DEV)
                if lo > b * block:
                    after = torch.maximum(least, scales[s, :, b])
                    values[s, :, b * block:lo] = _e4m3(values[s, :, b * block:lo] * (scales[s, :, b] / after)[:, None, None])
                else:
                    after = least
                scales[s, :, b] = after
                values[s, :, lo:hi] = _e4m3(part / after[:, None, None])
        outs.append((values, scales))
    return outs[0][0], outs[1][0], outs[0][1], outs[1][1], None


def _attend64(st, case):
    cached, new = _lengths(case)
    heads, kv, hd, block = case["heads"], case["kv_heads"], case["head_dim"], case["block"]
    group = heads // kv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    weight = torch.zeros((case["seqs"], kv, st["max_len"]), dtype=torch.float64, device=DEV)
    row = 0
    for s, (c, n) in enumerate(zip(cached, new)):
        if case["weights"]:
            weight[s, :, :c] = st["weight_in"][s, :, :c].double()
        if n == 0:
            continue
        k, v = (_decode(st[x][s, :, :c + n]) * st[x + "_scale"][s].double().repeat_interleave(block, 1)[:, :c + n, None] for x in "kv")
        q = st["q"][row:row + n].double().view(n, kv, group, hd)
        late = torch.arange(c + n, device=DEV)[None, :] > torch.arange(c, c + n, device=DEV)[:, None]
        for h in range(kv):
            z = torch.matmul(q[:, h].reshape(n * group, hd), k[h].T.contiguous()) / math.sqrt(hd)
            z = z.view(n, group, c + n).masked_fill(late[:, None, :], -math.inf)
            p = torch.softmax(z, -1)
            out[row:row + n, h * group:(h + 1) * group] = torch.matmul(p.view(n * group, -1), v[h]).view(n, group, hd)
            weight[s, h, :c + n] += p.sum((0, 1))
        row += n
    return (out, weight) if case["weights"] else (out,)


def _evict64(st, case):
    held, keep, block, kv = _lengths(case)[0], case["keep"], case["block"], case["kv_heads"]
    if sum(held) * kv > 4000000:   # one (sequence, head) after the other would take too long
        return None
    weight, position = st["weight_in"].double().cpu(), st["position"].cpu()
    next_position = st["next"].tolist()
    values = {x: _decode(st[x]) for x in "kv"}
    scales = {x: st[x + "_scale"].double() for x in "kv"}
    moved = torch.zeros(st["weight_out"].shape, dtype=torch.float64)
    for s, n in enumerate(held):
        for h in range(kv):
            if n <= keep:
                moved[s, h, :n] = weight[s, h, :n]
                continue
            w, late = weight[s, h, :n].tolist(), (position[s, h, :n] >= next_position[s] - case["recent"]).tolist()
            order = sorted(range(n), key=lambda i: (not late[i], 0.0 if late[i] else -w[i], i))
            stay = set(order[:keep])
            to = [i for i in range(keep) if i not in stay]
            come = sorted(i for i in stay if i >= keep)
            now = list(range(keep))
            for a, b in zip(to, come):
                now[a] = b
            moved[s, h, :keep] = weight[s, h][torch.tensor(now)]
            now = torch.tensor(now, device=DEV)
            for x in "kv":
                sc = scales[x][s, h]
                came = sc[now // block]
                after = torch.maximum(sc[:keep // block], came.view(-1, block).amax(1))
                values[x][s, h, :keep] = _e4m3(values[x][s, h][now] * (came / after.repeat_interleave(block))[:, None])
                sc[:keep // block] = after
    return values["k"], values["v"], scales["k"], scales["v"], moved.to(DEV), None, None
