"""The attention layer over an 8-bit cache (moe_attn_forward_kv8): prompts, single tokens and eviction, layer after layer,
against an fp64 reference with the layer's roundings to bf16; and the calls it refuses."""
import math

import pytest
import torch

from oracle import kv8_ref as R
from paper_2502_06888_amd import attn_binding as A
from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import inputs as I
from paper_2502_06888_amd import kv8_binding as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
RTOL, ATOL = 2e-2, 1e-2          # the layer's tolerance for bf16, as for the bf16 caches
NAMES = ("norm", "wq", "wk", "wv", "wo")


def bf16(x):
    return x.to(torch.bfloat16).double()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def rotate(x, pos, theta):
    """x [rows, heads, hd], pos [rows]: pairs (i, i + hd/2) by pos * theta^(-2i/hd)."""
    half = x.shape[2] // 2
    ang = pos.double()[:, None] * torch.tensor([theta ** (-i / half) for i in range(half)], dtype=torch.float64)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def project(w, ws, x, pos):
    """(q, k, v) as the layer rounds them."""
    x = x.double()
    xn = bf16(x / torch.sqrt((x * x).mean(-1, keepdim=True) + w.rms_eps) * ws["norm"].double())
    n = x.shape[0]
    q = (xn @ ws["wq"].double().T).view(n, w.n_q_heads, w.head_dim)
    k, v = ((xn @ ws[m].double().T).view(n, w.n_kv_heads, w.head_dim) for m in ("wk", "wv"))
    # xn is formed in 32 bits there: an element within 2^-23 of the middle between two bf16 numbers may be rounded the other
    # way (one in 2^14 or so), which moves a projection by a step of that element, 2^-7 |xn_j|, times its weight; the
    # rotation adds two of them.  Room for one such element per row:
    flip = 2.0 ** -7 * xn.abs().amax(-1) * max(float(ws[m].abs().max()) for m in ("wk", "wv")) * 2 ** 0.5
    return bf16(rotate(q, pos, w.rope_theta)), bf16(rotate(k, pos, w.rope_theta)), bf16(v), flip


def workload(heads, kv, hd, d, rows):
    return I.AttnWorkload("kv8", d, heads, kv, hd, (rows,), (0,), 128, w_std=0.06, seed=heads + hd)


@pytest.mark.parametrize("heads,kv,hd,d", [(8, 2, 32, 256), (8, 8, 64, 256), (4, 4, 32, 512), (8, 2, 128, 384), (6, 1, 64, 256)])
def test_conversation_over_two_layers(heads, kv, hd, d):
    layers, n, L, block, keep, recent = 2, 3, 112, 16, 48, 8
    w = workload(heads, kv, hd, d, 128)
    cfg = A.config_for(w, n_layers=layers)
    ctx = A.AttnContext(cfg, DEV)
    ws = [I.gen_attn_weights(w, l) for l in range(layers)]
    for l in range(layers):
        ctx.set_weights(*[ws[l][m].to(DEV) for m in NAMES], layer=l)
    caches = [Q.Kv8Cache.empty(n, kv, hd, L, block, DEV) for _ in range(layers)]
    weight = [torch.zeros((n, kv, L), device=DEV) for _ in range(layers)]
    g = torch.Generator().manual_seed(heads * hd)
    held, seen = [0] * n, [0] * n
    torch.cuda.synchronize()
    for new in ([37, 1, 64], [1, 1, 1], [0, 5, 2], "evict", [1, 1, 1], [20, 3, 30], "evict", [1, 1, 1]):
        if new == "evict":
            for c, wt in zip(caches, weight):
                Q.evict(c, ints(held), max(held), keep, recent, ints(seen), wt, stream=ctx.compute)
            held = [min(h, keep) for h in held]
            ctx.synchronize()
            continue
        off = [0]
        for m in new:
            off.append(off[-1] + m)
        step = Q.Kv8Step(ints(held), off[-1], max(new), max(held), row_offsets=ints(off), next_position=ints(seen))
        space = ctx.kv8_workspace(caches[0], step, True)
        x = torch.randn((off[-1], d), generator=g).to(torch.bfloat16)
        pos = torch.cat([torch.arange(p, p + m) for p, m in zip(seen, new)])
        for l, (c, wt) in enumerate(zip(caches, weight)):
            h_in = x.to(DEV)
            h_out = torch.zeros_like(h_in) if l == 0 else h_in              # the second layer in place
            w_in = wt.cpu().clone()
            torch.cuda.synchronize()
            ctx.forward_kv8(c, step, h_in, h_out, space, layer=l, weight_in=wt, weight_out=wt)
            ctx.synchronize()
            q, k, v, flip = project(w, ws[l], x, pos)
            for codes, scale, ref in ((c.k, c.k_scale, k), (c.v, c.v_scale, v)):
                got = R.values(codes.cpu(), scale.cpu(), block)
                s_all = scale.cpu().double().repeat_interleave(block, -1)
                for s, (a, m) in enumerate(zip(held, new)):
                    want = ref[off[s]:off[s] + m].transpose(0, 1)
                    # half a step of e4m3, one of bf16 (the sums differ in their last bits), and half the least step of the scale
                    room = (2.0 ** -4 + 2.0 ** -7) * want.abs() + s_all[s, :, a:a + m, None] * 2.0 ** -10 + 1.125 * flip[off[s]:off[s] + m, None]
                    far = ((got[s, :, a:a + m] - want).abs() - room).clamp_min(0)
                    assert float(far.amax() if m else 0) == 0, (int((far > 0).sum()), far.numel(), float(far.max()))
            o, wr, _, _ = R.attend(c.k.cpu(), c.k_scale.cpu(), c.v.cpu(), c.v_scale.cpu(), q, held, off, block, w_in)
            ref = x.double() + bf16(o).reshape(off[-1], -1) @ ws[l]["wo"].double().T
            got = h_out.cpu()
            assert bool(((got.double() - ref).abs() <= ATOL + RTOL * ref.abs()).all())
            ok = ~wr.isnan()
            assert torch.allclose(wt.cpu().double()[ok], wr[ok], rtol=RTOL, atol=ATOL)
            for s, (a, m) in enumerate(zip(held, new)):
                assert torch.equal(c.position[s, 0, a:a + m].cpu().long(), torch.arange(seen[s], seen[s] + m))
            x = got
        held, seen = [h + m for h, m in zip(held, new)], [h + m for h, m in zip(seen, new)]
    ctx.close()


def test_single_tokens_agree_with_the_layer_over_bf16_caches():
    """The same sequences through both layers: a cache in 8 bits moves an output by no more than its codes' half steps do."""
    heads, kv, hd, d, n, length = 8, 2, 64, 256, 5, 70
    w = workload(heads, kv, hd, d, n)
    ctx = A.AttnContext(A.config_for(w), DEV)
    ws = I.gen_attn_weights(w, 0)
    ctx.set_weights(*[ws[m].to(DEV) for m in NAMES])
    wide = [torch.zeros((n, kv, 128, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache = Q.Kv8Cache.empty(n, kv, hd, 128, 32, DEV, positions=False)
    g = torch.Generator().manual_seed(3)
    old = [torch.randn((n, kv, 128, hd), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2)]
    # values that e4m3 holds, so that both caches hold the same numbers
    old = [(t.float() * 4).to(torch.float8_e4m3fn).to(torch.bfloat16) for t in old]
    for t, o in zip(wide, old):
        t[:, :, :length] = o[:, :, :length]
    for s in range(n):   # rows of a bf16 cache, one sequence after the other, by their strides
        one = Q.Kv8Cache(*(t[s:s + 1] for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), 32)
        Q.append(one, Q.Kv8Step(ints([0]), length, length, 0), *(t[s].transpose(0, 1)[:length] for t in wide))
    x = torch.randn((n, d), generator=g).to(torch.bfloat16).to(DEV)
    y, y8 = torch.zeros_like(x), torch.zeros_like(x)
    torch.cuda.synchronize()
    step = Q.Kv8Step(ints([length] * n), n, 1, length)
    ctx.forward_kv8(cache, step, x, y8, ctx.kv8_workspace(cache, step, False))
    ctx.forward_group([A.AttnBatch(wide[0], wide[1], x, y, length)])
    ctx.synchronize()
    # what differs: the new token's own k and v (half a step of e4m3 in one slot of 71) and the roundings of q
    assert bool(((y8.double() - y.double()).abs() <= 3 * (ATOL + RTOL * y.double().abs())).all())
    ctx.close()


def test_rows_of_no_sequence_stay_and_a_captured_step_replays():
    heads, kv, hd, d, n, L, block = 8, 2, 64, 256, 3, 64, 16
    w = workload(heads, kv, hd, d, 16)
    ctx = A.AttnContext(A.config_for(w), DEV)
    ws = I.gen_attn_weights(w, 0)
    ctx.set_weights(*[ws[m].to(DEV) for m in NAMES])
    cache = Q.Kv8Cache.empty(n, kv, hd, L, block, DEV)
    for t in (cache.k, cache.v):
        t.fill_(0x30)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(1.0)
    lens, nxt = ints([5, 0, 20]), ints([5, 0, 20])
    step = Q.Kv8Step(lens, 8, 4, L, row_offsets=ints([1, 2, 2, 6]), next_position=nxt)
    x = torch.randn((8, d), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    y = torch.full_like(x, -3.0)
    space = ctx.kv8_workspace(cache, step, False)
    torch.cuda.synchronize()
    ctx.forward_kv8(cache, step, x, y, space)
    ctx.synchronize()
    assert bool((y[[0, 6, 7]] == -3).all()) and bool((y[1:6] != -3).any(-1).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=ctx.compute):
        ctx.forward_kv8(cache, step, x, y, space)
    keep = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    for lengths in ([5, 0, 20], [30, 9, 40], [0, 0, 0]):
        lens.copy_(ints(lengths))
        nxt.copy_(ints(lengths))
        out = []
        for replay in (False, True):
            for t, k in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), keep):
                t.copy_(k)
            y.fill_(-3.0)
            torch.cuda.synchronize()
            if replay:
                graph.replay()
            else:
                ctx.forward_kv8(cache, step, x, y, space)
            torch.cuda.synchronize()
            out.append([t.clone() for t in (y, cache.k, cache.v)])
        for a, b in zip(*out):
            assert torch.equal(a, b)
    ctx.close()


def test_refusals():
    heads, kv, hd, d = 8, 2, 64, 256
    w = workload(heads, kv, hd, d, 16)
    ctx = A.AttnContext(A.config_for(w), DEV)
    cache = Q.Kv8Cache.empty(4, kv, hd, 64, 16, DEV)
    step = Q.Kv8Step(ints([0] * 4), 4, 1, 63)
    x = torch.zeros((4, d), dtype=torch.bfloat16, device=DEV)
    space = ctx.kv8_workspace(cache, step, False)

    def refused(status, text, *a, **k):
        with pytest.raises(B.MoeError) as e:
            ctx.forward_kv8(*a, **k)
        assert e.value.status == status and text in str(e.value)

    refused(B.MOE_ERR_STATE, "set_weights", cache, step, x, x, space)
    ws = I.gen_attn_weights(w, 0)
    ctx.set_weights(*[ws[m].to(DEV) for m in NAMES])
    refused(B.MOE_ERR_INVALID_ARG, "layer", cache, step, x, x, space, layer=1)
    refused(B.MOE_ERR_SHAPE, "heads", Q.Kv8Cache.empty(4, kv, 32, 64, 16, DEV), step, x, x, space)
    many = Q.Kv8Step(ints([0] * 4), 20, 5, 59)
    refused(B.MOE_ERR_SHAPE, "rows", cache, many, torch.zeros((20, d), dtype=torch.bfloat16, device=DEV), torch.zeros((20, d), dtype=torch.bfloat16, device=DEV), ctx.kv8_workspace(cache, many, False))
    refused(B.MOE_ERR_INVALID_ARG, "h_in", cache, step, x[:3], x, space)
    refused(B.MOE_ERR_INVALID_ARG, "device memory", cache, step, x.cpu(), x, space)
    wt = torch.zeros((4, kv, 64), device=DEV)
    long, far = Q.Kv8Cache.empty(4, kv, hd, 4096, 16, DEV), Q.Kv8Step(ints([0] * 4), 4, 1, 4000)
    refused(B.MOE_ERR_OOM, "workspace", long, far, x, x, torch.empty(16, dtype=torch.uint8, device=DEV))
    refused(B.MOE_ERR_INVALID_ARG, "weight_in", cache, step, x, x, space, weight_in=wt)
    torch.cuda.synchronize()
    ctx.forward_kv8(cache, step, x, x, space)                                # a refused call leaves the context usable
    ctx.synchronize()
    ctx.close()
