"""The attention layer over an 8-bit cache with prompts of hundreds of tokens, on inputs for which its projections are exact: what
the attention adds to the hidden state and to the accumulated weights is then bounded element by element."""
import math

import pytest
import torch

from oracle import kv8_ref as R
from paper_2502_06888_amd import attn_binding as A
from paper_2502_06888_amd import kv8_binding as Q
from test_gpu_kv8 import bounds, ints, offsets_of, same
from test_gpu_kv8_layer import bf16, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 10000.0


@pytest.mark.parametrize("heads,kv,hd,block", [
    (8, 1, 64, 32),      # 34 row tiles of one pair: dequantised ahead, several ranges
    (4, 4, 128, 64),     # no shared heads: few row tiles, dequantised on the way
    (6, 2, 64, 16),      # three heads of a group
])
def test_long_prompts_through_the_layer(heads, kv, hd, block):
    """x is +1 or -1 and the norm's weights are 1, so xn is x; the projections' weights are whole numbers of 64ths, so q, k and v are
    exact sums, and v is the same to the last bit; Wo is the identity, so y - x is the attention's output."""
    n, L, d, cap = 3, 1280, heads * hd, 640
    group = heads // kv
    # the context keeps no bf16 cache here: its max_len sizes staging buffers of moe_attn_forward_group alone
    ctx = A.AttnContext(A.MoeAttnConfig(d, heads, kv, hd, 1, 1, 1, cap, THETA, 0.0), DEV)
    g = torch.Generator().manual_seed(heads * 10 + kv)
    wq, wk, wv = ((torch.randint(-8, 9, (h * hd, d), generator=g) / 64).to(torch.bfloat16) for h in (heads, kv, kv))
    ctx.set_weights(*[t.to(DEV) for t in (torch.ones(d, dtype=torch.bfloat16), wq, wk, wv, torch.eye(d, dtype=torch.bfloat16))])
    cache = Q.Kv8Cache.empty(n, kv, hd, L, block, DEV)
    for t in cache.tensors[:4]:
        t.zero_()
    weight = torch.zeros((n, kv, L), device=DEV)
    v_codes, v_scale = torch.zeros((n, kv, L, hd), dtype=torch.uint8), torch.zeros((n, kv, L // block), dtype=torch.float64)
    held = [0] * n
    for new in ([530, 1, 60], [1, 530, 7], [1, 1, 1], [0, 3, 600], [1, 1, 1]):
        off = offsets_of(new)
        rows = off[-1]
        seen = [h + 9 for h in held]
        step = Q.Kv8Step(ints(held), rows, max(new), max(held), row_offsets=ints(off), next_position=ints(seen))
        space = ctx.kv8_workspace(cache, step, True)
        x = (torch.randint(0, 2, (rows, d), generator=g) * 2 - 1).to(torch.bfloat16)
        y = torch.zeros_like(x, device=DEV)
        w_in, h_in = weight.clone(), x.to(DEV)
        torch.cuda.synchronize()
        ctx.forward_kv8(cache, step, h_in, y, space, weight_in=weight, weight_out=weight)
        ctx.synchronize()
        pos = torch.cat([torch.arange(p, p + m) for p, m in zip(seen, new)])
        q, k, v = ((x.double() @ w.double().T).view(rows, -1, hd) for w in (wq, wk, wv))
        q, k, v = bf16(rotate(q, pos, THETA)), bf16(rotate(k, pos, THETA)), bf16(v)
        R.append(v_codes, v_scale, v.to(torch.bfloat16), held, off, block)
        same(cache.v, v_codes)
        for s, (a, m) in enumerate(zip(held, new)):
            if m == 0:
                continue
            first, last = a // block, (a + m - 1) // block + 1
            assert torch.equal(cache.v_scale[s, :, first:last].cpu().double(), v_scale[s, :, first:last])
            want = k[off[s]:off[s] + m].transpose(0, 1)
            got = R.values(cache.k[s:s + 1].cpu(), cache.k_scale[s:s + 1].cpu(), block)[0, :, a:a + m]
            step_of = cache.k_scale[s].cpu().double().repeat_interleave(block, -1)[:, a:a + m, None] * 2.0 ** -10
            # half a step of e4m3, and a rotation in 32 bits that may round to the next bf16 number
            assert bool(((got - want).abs() <= (2.0 ** -4 + 2.0 ** -7) * want.abs() + step_of).all())
            assert torch.equal(cache.position[s, 0, a:a + m].cpu().long(), torch.arange(seen[s], seen[s] + m))
        codes = [t.cpu() for t in cache.tensors[:4]]
        o, more, spread, mag = R.attend(codes[0], codes[2], codes[1], codes[3], q, held, off, block)
        # q's rotation is in 32 bits: an element within 2^-22 of the middle between two bf16 numbers, one in 2^14, may be rounded
        # the other way.  Room for three of the hd elements of a (row, head), each a step (2^-7) of the largest product of a score:
        most = float(q.abs().max()) * float(R.values(codes[0], codes[2], block).nan_to_num(0).abs().max()) / math.sqrt(hd)
        lean = math.expm1(2 * 3 * 2.0 ** -7 * most)
        ref = x.double() + o.reshape(rows, -1)
        room = (bounds(o, spread, mag, hd) + lean * spread).reshape(rows, -1) + 2.0 ** -8 * ref.abs()
        assert bool(((y.cpu().double() - ref).abs() <= room * (1 + 2.0 ** -8)).all())
        total = [h + m for h, m in zip(held, new)]
        for s, h in enumerate(held):
            w_in[s, :, h:] = 0                                               # new slots start from nothing
        rise, after = (weight.double() - w_in.double()).cpu(), weight.cpu().double()
        for s, t in enumerate(total):
            # what the step gave a slot: 32-bit scores and sums, one addition to what was there
            loose = 2 * (hd + 4) * 2.0 ** -24 * float(mag.max()) + 2.0 ** -19
            assert bool(((rise[s, :, :t] - more[s, :, :t]).abs() <= (lean + loose) * more[s, :, :t] + 2.0 ** -23 * after[s, :, :t] + 1e-30).all())
            # the softmax weights of a row are 1 in all, whatever q is
            given = rise[s, :, :t].sum(-1)
            assert bool(((given - new[s] * group).abs() <= loose * new[s] * group + 2.0 ** -23 * after[s, :, :t].sum(-1)).all())
        held = total
    ctx.close()
