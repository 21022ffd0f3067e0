"""The 8-bit key-value cache on the GPU against the fp64 reference: append and evict bit for bit, attention within bounds
that are derived from the formats."""
import pytest
import torch

from oracle import kv8_ref as R
from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import kv8_binding as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def same(got, want):
    """Equal bit for bit (NaN equals NaN); says where not."""
    got, want = got.cpu(), want.cpu()
    if want.dtype == torch.uint8:                                            # codes: NaN has two
        got, want = (torch.where(t & 127 == 127, torch.full_like(t, 127), t) for t in (got, want))
    if want.dtype.is_floating_point:
        got, want = got.double().nan_to_num(-1e300), want.double().nan_to_num(-1e300)
    bad = (got != want).nonzero()
    assert bad.numel() == 0, f"{bad.shape[0]} differ, first at {bad[0].tolist()}: {got[tuple(bad[0])]} for {want[tuple(bad[0])]}"


def offsets_of(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def rand(g, shape, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16)


def filled(g, n, kv, L, hd, block, cached, poison=True):
    """A cache with codes in the held slots and, behind them, what must not be used: NaN codes and NaN scales."""
    codes = torch.randint(0, 256, (2, n, kv, L, hd), generator=g, dtype=torch.uint8)
    codes[(codes & 127) > 0x70] = 0x30                                       # no NaN, magnitudes up to 128
    scale = torch.pow(2.0, torch.randint(-9, -5, (2, n, kv, L // block), generator=g).double())
    if poison:
        for s, c in enumerate(cached):
            codes[:, s, :, c:] = 0x7f
            scale[:, s, :, -(-c // block):] = float("nan")
    pos = torch.full((n, kv, L), -7, dtype=torch.int32)
    cache = Q.Kv8Cache(codes[0].to(DEV), codes[1].to(DEV), scale[0].float().to(DEV), scale[1].float().to(DEV), block, pos.to(DEV))
    return cache, codes, scale


def step_for(cached, new, slack=(0, 0), next_position=None, uniform=False):
    off = offsets_of(new)
    return Q.Kv8Step(ints(cached), off[-1], max(new) + slack[0], max(cached) + slack[1],
                     row_offsets=None if uniform else ints(off), next_position=None if next_position is None else ints(next_position)), off


# ---- append ------------------------------------------------------------------------------------------

APPENDS = [
    # block, hd, kv, cached, new
    (16, 32, 1, [0], [1]),
    (32, 64, 2, [5, 0, 31, 32, 63], [1, 1, 1, 1, 1]),
    (64, 128, 8, [63, 64, 65, 1, 0, 127], [1, 1, 1, 1, 1, 1]),
    (128, 128, 3, [127, 5], [3, 4]),
    (16, 128, 2, [3, 0, 15, 40], [0, 37, 16, 1]),
    (64, 64, 4, [0, 64, 100], [64, 128, 29]),
    (128, 32, 5, [0, 11], [300, 117]),
    (32, 128, 1, [33], [700]),
]


@pytest.mark.parametrize("block,hd,kv,cached,new", APPENDS)
def test_append_has_the_codes_and_scales_of_the_reference(block, hd, kv, cached, new):
    g = torch.Generator().manual_seed(block * 1000 + hd + len(new))
    n = len(cached)
    L = -(-max(c + m for c, m in zip(cached, new)) // block) * block + block
    cache, codes, scale = filled(g, n, kv, L, hd, block, cached)
    nxt = [c + 11 for c in cached]
    step, off = step_for(cached, new, next_position=nxt)
    rows = off[-1] + 2                                                       # rows of no sequence behind the last one
    x = [rand(g, (rows, kv, hd)) * torch.exp2(torch.randint(-4, 5, (rows, 1, 1), generator=g)).to(torch.bfloat16) for _ in range(2)]
    for t in x:
        t[off[-1]:] = float("nan")
    pos = cache.position.cpu().clone()
    Q.append(cache, step, x[0].to(DEV), x[1].to(DEV))
    torch.cuda.synchronize()
    for i, (c, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        R.append(codes[i], scale[i], x[i], cached, off, block)
        same(c, codes[i])
        same(s, scale[i])
    for s, (c, m) in enumerate(zip(cached, new)):
        pos[s, :, c:c + m] = torch.arange(nxt[s], nxt[s] + m, dtype=torch.int32)
    assert torch.equal(cache.position.cpu(), pos)


def test_append_of_infinities_nan_zeros_and_the_ends_of_the_range():
    block, hd, kv = 16, 32, 1
    g = torch.Generator().manual_seed(5)
    cached, new = [0, 8, 0, 0, 0, 8], [16, 1, 3, 2, 2, 2]
    cache, codes, scale = filled(g, 6, kv, 32, hd, block, cached)
    step, off = step_for(cached, new)
    x = rand(g, (off[-1], kv, hd))
    x[3, 0, 4], x[3, 0, 5], x[5, 0, 6] = float("inf"), -float("inf"), float("nan")
    x[16] = float("inf")                                                     # a token without any finite element
    x[17:20] = 0
    x[20:22] = 3.3e38                                                        # beyond what the largest scale reaches
    x[22:24] = 1e-38
    x[24, 0, :] = 1e30                                                       # everything held falls to zero
    Q.append(cache, step, x.to(DEV), x.to(DEV))
    torch.cuda.synchronize()
    for i, (c, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        R.append(codes[i], scale[i], x, cached, off, block)
        same(c, codes[i])
        same(s, scale[i])


def test_tokens_beyond_the_last_slot_do_not_exist():
    """The second sequence has room for two of its five tokens."""
    block, hd, heads, kv, L = 16, 32, 4, 2, 64
    g = torch.Generator().manual_seed(8)
    cached, new, fit = [10, 62], [5, 5], [5, 2]
    cache, codes, scale = filled(g, 2, kv, L, hd, block, cached)
    step, off = step_for(cached, new)
    k, q = rand(g, (10, kv, hd)), rand(g, (10, heads, hd))
    Q.append(cache, step, k.to(DEV), k.to(DEV))
    there = [0, 1, 2, 3, 4, 5, 6]
    for i in range(2):
        R.append(codes[i], scale[i], k[there], cached, offsets_of(fit), block)
    same(cache.k, codes[0])
    same(cache.v, codes[1])
    out = torch.full((10, heads, hd), -3.0, dtype=torch.bfloat16, device=DEV)
    Q.attend(cache, step, q.to(DEV), out)
    ref, _, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q[there], cached, offsets_of(fit), block)
    assert bool(((out[:7].cpu().double() - ref).abs() <= bounds(ref, spread, mag, hd)).all())
    assert bool((out[7:] == -3).all())


def test_append_takes_slices_of_a_fused_projection_and_is_repeatable():
    block, hd, kv, heads = 32, 64, 2, 4
    g = torch.Generator().manual_seed(6)
    cached, new = [7, 40], [5, 9]
    cache, codes, scale = filled(g, 2, kv, 64, hd, block, cached)
    step, off = step_for(cached, new)
    qkv = rand(g, (off[-1], (heads + 2 * kv), hd)).to(DEV)
    k, v = qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    for _ in range(2):                                                       # the second time changes nothing
        Q.append(cache, step, k, v)
        torch.cuda.synchronize()
        if _ == 0:
            R.append(codes[0], scale[0], k.cpu(), cached, off, block)
            R.append(codes[1], scale[1], v.cpu(), cached, off, block)
        same(cache.k, codes[0])
        same(cache.v, codes[1])
        same(cache.k_scale, scale[0])


def test_prompt_token_by_token_gives_the_codes_of_the_whole_prompt():
    """Tokens of similar size: no code falls below the smallest normal one, so the order of the appends does not show."""
    block, hd, kv, n = 16, 32, 2, 3
    g = torch.Generator().manual_seed(7)
    x = [(torch.rand((n * 37, kv, hd), generator=g) + 0.5).to(torch.bfloat16).to(DEV) for _ in range(2)]
    whole = Q.Kv8Cache.empty(n, kv, hd, 48, block, DEV)
    Q.append(whole, Q.Kv8Step(ints([0] * n), n * 37, 37, 0), *x)
    single = Q.Kv8Cache.empty(n, kv, hd, 48, block, DEV)
    cached = ints([0] * n)
    step = Q.Kv8Step(cached, n, 1, 47)
    for t in range(37):
        Q.append(single, step, *(y.view(n, 37, kv, hd)[:, t].contiguous() for y in x))
        cached += 1
    torch.cuda.synchronize()
    for a, b in ((whole.k, single.k), (whole.v, single.v), (whole.position, single.position)):
        assert torch.equal(a[:, :, :37], b[:, :, :37])
    assert torch.equal(whole.k_scale, single.k_scale) and torch.equal(whole.v_scale, single.v_scale)


# ---- attend ------------------------------------------------------------------------------------------

def bounds(out, spread, mag, hd):
    """|error| of an output: half a bf16 step (2^-8) of the result; each softmax weight off by half a bf16 step (it is
    rounded before it multiplies V), by twice the absolute error of a score (hd + 4 roundings of 2^-24 of the sum of
    magnitudes, once in the weight and once in the sum) and by 2^-20 for the exponential and the sums in 32 bits."""
    delta = (hd + 4) * 2.0 ** -24 * mag
    return 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * delta + 2.0 ** -20)[..., None] * spread + 1e-30


def weight_bounds(weight, mag, hd):
    return weight.abs() * (2 * (hd + 4) * 2.0 ** -24 * float(mag.max() if mag.numel() else 0) + 2.0 ** -19) + 1e-30


ATTENDS = [
    # block, hd, heads, kv, cached, new
    (16, 32, 1, 1, [0], [1]),                                    # one token sees itself
    (32, 64, 4, 4, [0, 1, 31, 32, 33], [1, 1, 1, 1, 1]),
    (64, 128, 32, 8, [0, 63, 64, 511, 700], [1, 1, 1, 1, 1]),
    (64, 128, 6, 1, [2500, 17], [1, 1]),                          # a long cache beside a short one
    (128, 128, 8, 1, [1300], [1]),
    (16, 64, 14, 2, [5000, 3, 0], [1, 1, 1]),
    (32, 32, 15, 5, [260], [1]),
    (64, 128, 8, 2, [100, 3, 0], [2, 0, 4]),                      # a few tokens, one sequence without any
    (32, 128, 16, 8, [511, 64], [3, 5]),
    (16, 32, 8, 4, [0, 5], [33, 1]),                              # prompts
    (64, 64, 8, 2, [0, 0, 129], [64, 65, 131]),
    (64, 128, 4, 4, [0], [128]),
    (128, 128, 32, 8, [0, 300], [257, 90]),
    (32, 128, 7, 1, [77], [200]),
    (16, 64, 16, 8, [1000, 0, 3], [17, 0, 300]),
    (64, 128, 12, 2, [2100], [40]),
    (128, 32, 4, 1, [600, 1], [70, 700]),
    (16, 32, 64, 64, [0] * 9, [530, 512, 31, 500, 64, 65, 1, 0, 400]),      # many row tiles: two and more per workgroup
    (64, 64, 64, 32, [3, 0, 100], [600, 580, 33]),
    (64, 128, 48, 16, [0, 5], [350, 400]),
    (32, 64, 8, 2, [60, 5, 0, 33], [0, 200, 0, 0]),                          # sequences without tokens before and behind
    (32, 64, 128, 128, [0, 70, 64, 1], [250, 200, 129, 128]),               # two row tiles per pair
    (64, 128, 8, 1, [0, 37, 500], [530, 1, 450]),                            # 32 row tiles and more: dequantised ahead
    (16, 64, 8, 1, [1, 900], [600, 33]),
    (128, 32, 16, 2, [0, 70], [513, 515]),
    (32, 64, 8, 2, [1700, 3], [1, 1]),                                       # a few ranges of slots, and whole beside them
    (64, 32, 4, 4, [1800, 1600, 0], [2, 1, 0]),
    (64, 128, 8, 2, [900, 20], [4, 1]),                                      # 16 rows, and 12
    (16, 64, 12, 3, [2000], [3]),
    (64, 128, 16, 2, [4000, 130, 0], [5, 0, 3]),                             # 40 rows over many ranges
    (16, 64, 512, 128, [2100, 700, 3, 0], [1, 1, 1, 1]),                     # scores of more than 32 KiB in LDS: one range of 512 pairs,
    (32, 64, 16, 2, [999, 31, 500], [1, 0, 1]),                              # 8 rows of 1000 slots,
    (64, 32, 10, 2, [600, 0, 697, 64], [3, 1, 2, 0]),                        # 15 rows of 700
    (32, 32, 64, 64, [2000, 30], [203, 7]),                                  # ranges of many rows
]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("block,hd,heads,kv,cached,new", ATTENDS)
def test_attention_is_within_its_bounds(block, hd, heads, kv, cached, new, weights):
    g = torch.Generator().manual_seed(block + hd + heads + sum(cached) + sum(new))
    n = len(cached)
    total = [c + m for c, m in zip(cached, new)]
    L = -(-max(total) // block) * block + block
    cache, codes, scale = filled(g, n, kv, L, hd, block, total)
    step, off = step_for(cached, new, slack=(0, 0))
    rows = off[-1] + 3
    q = rand(g, (rows, heads, hd), 2.0)
    out = torch.full((rows, heads, hd), -3.0, dtype=torch.bfloat16, device=DEV)
    w_in = torch.rand((n, kv, L), generator=g)
    w_out = torch.full((n, kv, L), -5.0, device=DEV)
    for s, c in enumerate(cached):
        w_in[s, :, c:] = float("nan")                                        # of new slots nothing is taken over
    Q.attend(cache, step, q.to(DEV), out, *((w_in.to(DEV), w_out) if weights else ()))
    torch.cuda.synchronize()
    ref, weight, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q, cached, off, block, w_in)
    got = out.cpu().double()
    m = off[-1]
    assert bool(((got[:m] - ref[:m]).abs() <= bounds(ref, spread, mag, hd)[:m]).all())
    assert bool((got[m:] == -3).all())                                       # rows of no sequence
    if weights:
        w = w_out.cpu().double()
        held = ~weight.isnan()
        assert bool(((w - weight).abs() <= weight_bounds(weight, mag[:m], hd))[held].all())
        assert bool((w[~held] == -5).all())


def test_attention_of_infinite_and_nan_values_stays_with_those_who_see_them():
    """A NaN code in the last slot of a prompt reaches the last token alone."""
    block, hd, heads, kv = 16, 64, 4, 2
    g = torch.Generator().manual_seed(9)
    cache, codes, scale = filled(g, 1, kv, 64, hd, block, [40])
    cache.v[0, 0, 39, 7] = 0x7f
    codes[1][0, 0, 39, 7] = 0x7f
    for cached, new in ([0, 40], [38, 2], [36, 4], [32, 8], [10, 30], [39, 1]):
        q = rand(g, (new, heads, hd))
        out = torch.zeros((new, heads, hd), dtype=torch.bfloat16, device=DEV)
        Q.attend(cache, Q.Kv8Step(ints([cached]), new, new, cached), q.to(DEV), out)
        got = out.cpu()
        nan = torch.zeros_like(got, dtype=torch.bool)
        nan[-1, :heads // kv, 7] = True
        assert torch.equal(got.isnan(), nan)


def test_nan_codes_in_prompts_stay_with_those_who_see_them():
    """Four row tiles and more, dequantised ahead: NaN codes at slots 70 and 300 of a prompt of 400 tokens."""
    block, hd, heads, kv, new = 32, 64, 8, 2, 400
    g = torch.Generator().manual_seed(19)
    for cached in (0, 75):
        cache, codes, scale = filled(g, 1, kv, 480, hd, block, [cached + new])
        for slot, e in ((70, 3), (300, 60)):
            cache.v[0, 1, slot, e] = 0xff
        q = rand(g, (new, heads, hd))
        out = torch.zeros((new, heads, hd), dtype=torch.bfloat16, device=DEV)
        Q.attend(cache, Q.Kv8Step(ints([cached]), new, new, cached), q.to(DEV), out)
        nan = torch.zeros((new, heads, hd), dtype=torch.bool)
        nan[max(0, 70 - cached):, heads // kv:, 3] = True
        nan[300 - cached:, heads // kv:, 60] = True
        assert torch.equal(out.cpu().isnan(), nan)


@pytest.mark.parametrize("hd,kv,cached", [(32, 1, 0), (64, 2, 75), (128, 1, 1100)])
def test_nan_codes_dequantised_ahead_stay_with_those_who_see_them(hd, kv, cached):
    """The same with 32 row tiles and more, in one range of slots and in several."""
    block, heads, new = 32, 8 * kv, 520
    g = torch.Generator().manual_seed(20)
    cache, codes, scale = filled(g, 1, kv, 1664, hd, block, [cached + new])
    for slot, e in ((70, 3), (cached + 300, hd - 4), (cached + new - 1, 0)):
        cache.v[0, kv - 1, slot, e] = 0xff
    q = rand(g, (new, heads, hd))
    out = torch.zeros((new, heads, hd), dtype=torch.bfloat16, device=DEV)
    Q.attend(cache, Q.Kv8Step(ints([cached]), new, new, cached), q.to(DEV), out)
    nan = torch.zeros((new, heads, hd), dtype=torch.bool)
    nan[max(0, 70 - cached):, -8:, 3] = True
    nan[300:, -8:, hd - 4] = True
    nan[-1:, -8:, 0] = True
    assert torch.equal(out.cpu().isnan(), nan)


@pytest.mark.parametrize("query,power,code,fifth", [
    (-1.0625, 119, 0x7e, False),           # every score is -3.16e38, close to the lowest number
    (1.0625 * 2.0 ** 60, 0, 0x7d, False),  # every score is 5.1e20
    (1.0625 * 2.0 ** 30, 0, 0x7d, True),   # of every five slots the first wins by 4.8e11
    (-1.0625 * 2.0 ** 60, 9, 0x7d, True),  # of every five slots the first is the only one that does not lose by 2.6e23
])
@pytest.mark.parametrize("cached,new", [(700, 1), (40, 4), (0, 150), (300, 520)])
def test_equal_scores_of_any_size_share_alike(cached, new, query, power, code, fifth):
    block, hd, heads, kv, L = 32, 32, 8, 1, 832
    g = torch.Generator().manual_seed(21)
    cache, codes, scale = filled(g, 1, kv, L, hd, block, [L], poison=False)
    loses = torch.arange(L) % 5 != 0
    codes[0][:] = 0
    codes[0][..., 5] = torch.where(loses == (query < 0), code, 0) if fifth else code
    cache.k.copy_(codes[0])
    cache.k_scale.fill_(2.0 ** power)
    q = torch.zeros((new, heads, hd), dtype=torch.bfloat16)
    q[..., 5] = query
    out = torch.zeros((new, heads, hd), dtype=torch.bfloat16, device=DEV)
    w = torch.zeros((1, kv, L), device=DEV)
    Q.attend(cache, Q.Kv8Step(ints([cached]), new, new, cached), q.to(DEV), out, None, w, softmax_scale=0.6875)
    v = R.TABLE[codes[1][0, 0].long()] * scale[1][0, 0].repeat_interleave(block)[:, None]
    want, mean = torch.zeros(L, dtype=torch.float64), torch.zeros((new, 1, hd), dtype=torch.float64)
    for i in range(new):
        share = (~loses if fifth else torch.ones(L)).double() * (torch.arange(L) <= cached + i)
        share /= share.sum()
        want += heads * share
        mean[i, 0] = share @ v
    # equal scores are equal in 32 bits too, and the others' weights are zero: what is left is the rounding of the weights and of
    # the result, and sums in 32 bits
    assert bool(((out.cpu().double() - mean).abs() <= 2.0 ** -8 * mean.abs() + (2.0 ** -8 + 2.0 ** -20) * v.abs().max()).all())
    assert bool(((w[0, 0].cpu().double() - want).abs() <= 2.0 ** -18 * want).all())


@pytest.mark.parametrize("cached,new", [(700, 1), (0, 150), (300, 5)])
def test_scores_far_apart_and_equal_scores(cached, new):
    """One slot far above all others takes everything; equal scores give the mean."""
    block, hd, heads, kv, L = 32, 128, 8, 2, 736
    g = torch.Generator().manual_seed(10)
    cache, codes, scale = filled(g, 1, kv, L, hd, block, [L], poison=False)
    for big in (False, True):
        codes[0][:] = 0
        if big:
            codes[0][:, :, ::97] = 0x70                                      # scores of thousands at a few slots
        cache.k.copy_(codes[0])
        q = torch.full((new, heads, hd), 8.0).to(torch.bfloat16)
        out = torch.zeros((new, heads, hd), dtype=torch.bfloat16, device=DEV)
        Q.attend(cache, Q.Kv8Step(ints([cached]), new, new, cached), q.to(DEV), out)
        ref, _, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q, [cached], [0, new], block)
        # all products of a score are the same here, so its rounding is no larger than the derived bound
        assert bool(((out.cpu().double() - ref).abs() <= bounds(ref, spread, mag, hd)).all())


def test_strides_scale_and_output_in_place():
    block, hd, heads, kv = 32, 64, 8, 2
    g = torch.Generator().manual_seed(11)
    for cached, new in (([100, 31], [1, 1]), ([10, 64], [40, 23])):
        total = [c + m for c, m in zip(cached, new)]
        cache, codes, scale = filled(g, 2, kv, 160, hd, block, total)
        step, off = step_for(cached, new)
        wide = rand(g, (off[-1], heads + 3, hd + 8)).to(DEV)
        q = wide[:, 1:1 + heads, :hd]
        before = wide.cpu().clone()
        ref, _, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q.cpu(), cached, off, block, softmax_scale=0.3)
        Q.attend(cache, step, q, q, softmax_scale=0.3)
        torch.cuda.synchronize()
        assert bool(((q.cpu().double() - ref).abs() <= bounds(ref, spread, mag, hd)).all())
        before[:, 1:1 + heads, :hd] = q.cpu()
        assert torch.equal(wide.cpu(), before)                               # nothing beside the heads is written


def test_weights_without_input_in_place_and_without_rows():
    block, hd, heads, kv, L = 32, 64, 8, 2, 128
    g = torch.Generator().manual_seed(12)
    cached, new = [60, 10], [20, 3]
    cache, codes, scale = filled(g, 2, kv, L, hd, block, [80, 13])
    step, off = step_for(cached, new)
    q = rand(g, (off[-1], heads, hd))
    out = torch.empty((off[-1], heads, hd), dtype=torch.bfloat16, device=DEV)
    w = torch.full((2, kv, L), -5.0, device=DEV)
    Q.attend(cache, step, q.to(DEV), out, None, w)
    _, weight, _, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q, cached, off, block)
    held = ~weight.isnan()
    assert bool(((w.cpu().double() - weight).abs() <= weight_bounds(weight, mag, hd))[held].all())
    assert bool((w.cpu()[~held] == -5).all())
    once = w.clone()
    Q.attend(cache, step, q.to(DEV), out, w, w)                              # old slots add up, new ones start anew
    for s, c in enumerate(cached):
        assert torch.allclose(w[s, :, :c], 2 * once[s, :, :c], rtol=2e-6, atol=0)
        assert torch.equal(w[s, :, c:], once[s, :, c:])
    other = torch.full_like(w, -5.0)
    Q.attend(cache, Q.Kv8Step(ints(cached), 0, 0, 60, row_offsets=ints([0, 0, 0])), q.to(DEV), out, w, other)
    for s, c in enumerate(cached):
        assert torch.equal(other[s, :, :c], w[s, :, :c]) and bool((other[s, :, c:] == -5).all())


def test_sequences_do_not_depend_on_each_other():
    block, hd, heads, kv, L = 64, 128, 8, 2, 1024
    g = torch.Generator().manual_seed(13)
    for new in ([1, 1, 1], [40, 7, 90]):
        cached = [900, 3, 500]
        cache, codes, scale = filled(g, 3, kv, L, hd, block, [c + m for c, m in zip(cached, new)])
        step, off = step_for(cached, new)
        q = rand(g, (off[-1], heads, hd)).to(DEV)
        out = [torch.zeros((off[-1], heads, hd), dtype=torch.bfloat16, device=DEV) for _ in range(3)]
        Q.attend(cache, step, q, out[0])
        Q.attend(cache, step, q, out[1])
        assert torch.equal(out[0], out[1])                                   # run to run
        cache.k[0] = 0x7f                                                    # another sequence turns to NaN
        Q.attend(cache, step, q, out[2])
        assert torch.equal(out[0][off[1]:], out[2][off[1]:])


# ---- evict -------------------------------------------------------------------------------------------

EVICTS = [
    # block, hd, kv, held, keep, recent, kind of weights
    (16, 32, 1, [17], 16, 0, "random"),
    (32, 64, 2, [96, 64, 33, 0, 128], 64, 10, "random"),
    (64, 128, 4, [700, 513, 512, 100], 512, 64, "random"),
    (16, 128, 2, [300, 17], 160, 160, "random"),                  # only recent ones stay
    (128, 32, 3, [1000, 129], 128, 0, "ties"),
    (32, 64, 1, [257], 32, 7, "nan"),
    (16, 64, 2, [70], 64, 3, "zeros"),
    (64, 128, 1, [5000], 2048, 256, "random"),
    (16, 32, 1, [1024, 1, 1025], 1008, 1, "random"),              # around what a wavefront takes
    (128, 32, 2, [4097, 4095], 3968, 100, "ties"),
    (128, 32, 1, [16384, 9000], 16256, 8000, "random"),
    (128, 32, 1, [20000, 70], 128, 0, "ties"),                    # more than 16 per lane
    (128, 32, 2, [17000], 16896, 3, "random"),
    (128, 32, 1, [32768, 20000], 16384, 100, "random"),
    (128, 32, 2, [40000], 4096, 3, "random"),                     # longer than any lanes hold
    (128, 32, 1, [33000, 50, 2000], 1024, 0, "ties"),
    (128, 32, 1, [36000], 33024, 500, "nan"),
]


def evict_state(block, hd, kv, held, kind, seed):
    g = torch.Generator().manual_seed(seed)
    n, L = len(held), -(-max(max(held), 1) // block) * block + block
    cache, codes, scale = filled(g, n, kv, L, hd, block, held)
    w = torch.rand((n, kv, L), generator=g) ** 3
    if kind == "ties":
        w = torch.randint(0, 4, (n, kv, L), generator=g).float() * torch.where(torch.rand((n, kv, L), generator=g) < 0.3, -0.0, 1.0)
    elif kind == "nan":
        w = torch.where(torch.rand((n, kv, L), generator=g) < 0.9, torch.tensor(float("nan")), w)
        w[..., ::13] = float("inf")
    elif kind == "zeros":
        w = torch.zeros_like(w)
    pos = torch.stack([torch.randperm(L, generator=g) for _ in range(n * kv)]).view(n, kv, L).to(torch.int32)
    cache.position.copy_(pos)
    return cache, codes, scale, w, pos, [L] * n


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("block,hd,kv,held,keep,recent,kind", EVICTS)
def test_eviction_keeps_what_the_reference_keeps(block, hd, kv, held, keep, recent, kind, in_place):
    cache, codes, scale, w, pos, nxt = evict_state(block, hd, kv, held, kind, block + hd + keep)
    n, L = len(held), w.shape[2]
    w_ref, p_ref, kept_ref = R.evict(codes, scale, w, pos, held, keep, recent, nxt, block)
    w_in = w.to(DEV)
    w_out = w_in if in_place else torch.full_like(w_in, -5.0)
    p_out = None if in_place else torch.full_like(cache.position, -5)
    kept = None if in_place else torch.full((n, kv, keep), -9, dtype=torch.int32, device=DEV)
    Q.evict(cache, ints(held), max(held), keep, recent, ints(nxt), w_in, None if in_place else w_out, p_out, kept)
    torch.cuda.synchronize()
    for i, (c, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        same(c, codes[i])
        same(s, scale[i])
    p_got = cache.position if in_place else p_out
    for s, m in enumerate(held):
        e = min(m, keep)
        same(w_out[s, :, :e], w_ref[s, :, :e])
        assert torch.equal(p_got[s, :, :e].cpu().long(), p_ref[s, :, :e])
        if in_place:
            same(w_out[s, :, e:], w[s, :, e:])
            assert torch.equal(p_got[s, :, e:].cpu(), pos[s, :, e:])
        else:
            assert bool((w_out[s, :, e:] == -5).all()) and bool((p_got[s, :, e:] == -5).all())
            assert torch.equal(kept[s].cpu().long(), kept_ref[s])


# ---- together ----------------------------------------------------------------------------------------

def test_prompt_decode_evict_decode():
    """A conversation: ragged prompts, single tokens, eviction, single tokens again; after each step the outputs and weights
    are compared with the reference on the codes as they are."""
    block, hd, heads, kv, n, L, keep = 16, 64, 8, 2, 3, 96, 48
    g = torch.Generator().manual_seed(20)
    cache = Q.Kv8Cache.empty(n, kv, hd, L, block, DEV)
    weight = torch.zeros((n, kv, L), device=DEV)
    held, seen = [0] * n, [0] * n
    for new in ([40, 7, 61], [1, 1, 1], [2, 3, 1], "evict", [1, 1, 1], [9, 20, 12], "evict", [1, 1, 1]):
        if new == "evict":
            codes = torch.stack((cache.k, cache.v)).cpu()
            scale = torch.stack((cache.k_scale, cache.v_scale)).cpu().double()
            w, pos = weight.cpu(), cache.position.cpu()
            w_ref, p_ref, _ = R.evict(codes, scale, w, pos, held, keep, 8, seen, block)
            Q.evict(cache, ints(held), max(held), keep, 8, ints(seen), weight)
            assert torch.equal(torch.stack((cache.k, cache.v)).cpu(), codes)
            held = [min(h, keep) for h in held]
            for s, h in enumerate(held):
                assert torch.equal(weight[s, :, :h].cpu().double(), w_ref[s, :, :h])
                assert torch.equal(cache.position[s, :, :h].cpu().long(), p_ref[s, :, :h])
                # what was said last is still there
                assert bool((cache.position[s, :, :h] >= seen[s] - 8).sum() == kv * min(8, seen[s]))
            continue
        step, off = step_for(held, new, next_position=seen)
        q, k, v = (rand(g, (off[-1], h, hd)) for h in (heads, kv, kv))
        out = torch.empty((off[-1], heads, hd), dtype=torch.bfloat16, device=DEV)
        w_in = weight.cpu().clone()
        Q.append(cache, step, k.to(DEV), v.to(DEV))
        Q.attend(cache, step, q.to(DEV), out, weight, weight)
        ref, w, spread, mag = R.attend(cache.k.cpu(), cache.k_scale.cpu(), cache.v.cpu(), cache.v_scale.cpu(), q, held, off, block, w_in)
        assert bool(((out.cpu().double() - ref).abs() <= bounds(ref, spread, mag, hd)).all())
        ok = ~w.isnan()
        assert bool(((weight.cpu().double() - w).abs() <= weight_bounds(w, mag, hd))[ok].all())
        held, seen = [h + m for h, m in zip(held, new)], [h + m for h, m in zip(seen, new)]


@pytest.mark.parametrize("new,cached", [(1, 300), (48, 100)])
def test_a_captured_step_follows_the_lengths_on_the_device(new, cached):
    block, hd, heads, kv, n, L, keep = 32, 64, 8, 2, 4, 512, 96
    g = torch.Generator().manual_seed(21)
    cache, _, _ = filled(g, n, kv, L, hd, block, [cached + 2 * new] * n, poison=False)
    lens = ints([cached, cached // 2, 0, 5])
    nxt = ints([1000] * n)
    step = Q.Kv8Step(lens, n * new, new, L - new, next_position=nxt)
    q, k, v = (rand(g, (n * new, h, hd)).to(DEV) for h in (heads, kv, kv))
    out = torch.zeros_like(q)
    w_in = torch.rand((n, kv, L), generator=g).to(DEV)
    w_out, w_kept, p_out = torch.zeros_like(w_in), torch.zeros_like(w_in), torch.zeros_like(cache.position)
    ws, ws2 = Q.attend_workspace(cache, step, heads, True), Q.evict_workspace(cache, keep)

    def one():
        Q.append(cache, step, k, v)
        Q.attend(cache, step, q, out, w_in, w_out, ws)
        Q.evict(cache, lens, L, keep, 4, nxt, w_in, w_kept, p_out, workspace=ws2)

    stream = torch.cuda.Stream()
    start = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.position)]
    tensors = (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.position, out, w_out, w_kept, p_out)

    def again():
        for t, s in zip(tensors, start):
            t.copy_(s)
        for t in (out, w_out, w_kept, p_out):
            t.zero_()

    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        one()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        one()
    for lengths in ([cached, cached // 2, 0, 5], [cached + new, 1, 97, 0], [0, 0, 200, cached]):
        lens.copy_(ints(lengths))
        again()
        one()
        torch.cuda.synchronize()
        want = [t.clone() for t in tensors]
        again()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(tensors, want):
            assert torch.equal(t, w)


def test_two_streams_at_once():
    block, hd, heads, kv, L = 64, 128, 16, 4, 1024
    g = torch.Generator().manual_seed(22)
    sides = []
    for n, new in ((3, 1), (2, 70)):
        cache, _, _ = filled(g, n, kv, L, hd, block, [900] * n, poison=False)
        step = Q.Kv8Step(ints([800] * n), n * new, new, 800)
        q = rand(g, (n * new, heads, hd)).to(DEV)
        out, w = torch.zeros_like(q), torch.zeros((n, kv, L), device=DEV)
        sides.append((cache, step, q, out, w, Q.attend_workspace(cache, step, heads, True), torch.cuda.Stream()))
    want = []
    for cache, step, q, out, w, ws, _ in sides:
        Q.attend(cache, step, q, out, None, w, ws)
        want.append((out.clone(), w.clone()))
    torch.cuda.synchronize()
    for _ in range(4):
        for cache, step, q, out, w, ws, st in sides:
            Q.attend(cache, step, q, out, None, w, ws, stream=st)
    torch.cuda.synchronize()
    for (_, _, _, out, w, _, _), (o, v) in zip(sides, want):
        assert torch.equal(out, o) and torch.equal(w, v)


def test_numbers_outside_their_bounds_stay_inside_the_tensors():
    """Lengths and offsets beyond what the host said: taken as the nearest ones inside; guards around the tensors stay."""
    block, hd, heads, kv, n, L = 16, 32, 4, 2, 2, 64
    guard = 4096
    g = torch.Generator().manual_seed(23)

    def guarded(shape, dtype):
        import math
        flat = torch.full((math.prod(shape) + 2 * guard,), 77, dtype=dtype, device=DEV)
        return flat, flat[guard:guard + math.prod(shape)].view(shape)

    flats, t = zip(*(guarded(s, d) for s, d in (((n, kv, L, hd), torch.uint8), ((n, kv, L, hd), torch.uint8), ((n, kv, 4), torch.float32),
                                               ((n, kv, 4), torch.float32), ((n, kv, L), torch.int32), ((n, kv, L), torch.float32),
                                               ((n, kv, 32), torch.int32), ((6, heads, hd), torch.bfloat16))))
    cache = Q.Kv8Cache(*t[:4], block, t[4])
    big = 2 ** 31 - 1
    for cached, off in (([big, -5], [0, 3, 6]), ([60, 3], [-9, big, -1]), ([0, 0], [6, 6, 6]), ([-big, big], [3, 0, 9])):
        for x in (cache.k, cache.v):
            x.fill_(0x30)
        for x in (cache.k_scale, cache.v_scale):
            x.fill_(1.0)
        step = Q.Kv8Step(ints(cached), 6, 5, 59, row_offsets=ints(off))
        k = rand(g, (6, kv, hd)).to(DEV)
        Q.append(cache, step, k, k)
        Q.attend(cache, step, rand(g, (6, heads, hd)).to(DEV), t[7], None, t[5])
        Q.evict(cache, ints(cached), 64, 32, 5, None, t[5], kept=t[6])
        torch.cuda.synchronize()
        for f in flats:
            assert bool((f[:guard] == 77).all()) and bool((f[-guard:] == 77).all())


def test_offsets_beyond_32_bits():
    """The last sequence of a cache of 5.4 GB for K alone."""
    block, hd, kv, n, L, keep = 64, 128, 1, 41, 1 << 20, 128
    g = torch.Generator().manual_seed(24)
    cache = Q.Kv8Cache.empty(n, kv, hd, L, block, DEV)
    tail = [t[-1:] for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.position)]
    assert tail[0].data_ptr() - cache.k.data_ptr() > 1 << 32
    small, codes, scale = filled(g, 1, kv, 192, hd, block, [150], poison=False)
    small.position.copy_(torch.arange(192, dtype=torch.int32))
    for t, o in zip(tail, (small.k, small.v, small.k_scale, small.v_scale, small.position)):
        t[:, :, :o.shape[2]] = o
    weight = torch.zeros((n, kv, L), device=DEV)
    for new in (1, 40):
        off = [0] * n + [new]
        step = Q.Kv8Step(ints([0] * (n - 1) + [150]), new, new, 150, row_offsets=ints(off))
        q, k, v = (rand(g, (new, h, hd)) for h in (2, kv, kv))
        out = torch.zeros((new, 2, hd), dtype=torch.bfloat16, device=DEV)
        Q.append(cache, step, k.to(DEV), v.to(DEV))
        Q.attend(cache, step, q.to(DEV), out, None, weight)
        for i, x in enumerate((k, v)):
            R.append(codes[i], scale[i], x, [150], [0, new], block)
        same(tail[0][:, :, :192], codes[0])
        same(tail[1][:, :, :192], codes[1])
        ref, w, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q, [150], [0, new], block)
        assert bool(((out.cpu().double() - ref).abs() <= bounds(ref, spread, mag, hd)).all())
        held = 150 + new
        assert bool(((weight[-1, :, :held].cpu().double() - w[0, :, :held]).abs() <= weight_bounds(w, mag, hd)[0, :, :held]).all())
    held, w_in = [0] * (n - 1) + [190], weight.cpu()[-1:]
    pos = tail[4][:, :, :192].cpu()
    Q.evict(cache, ints(held), 190, keep, 16, None, weight)
    R.evict(codes, scale, w_in[:, :, :192], pos, [190], keep, 16, [190], block)
    same(tail[0][:, :, :192], codes[0])
    same(tail[1][:, :, :192], codes[1])


def test_refusals_that_need_device_memory():
    c = Q.Kv8Cache.empty(2, 2, 64, 128, 32, DEV)
    s = Q.Kv8Step(ints([3, 4]), 2, 1, 4)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=DEV)
    k = q[:, :2]
    w = torch.zeros((2, 2, 128), device=DEV)
    lib = Q.load_library()

    def refused(call, status, text):
        with pytest.raises(B.MoeError) as e:
            call()
        assert e.value.status == status and text in str(e.value)

    odd = torch.zeros((2, 4, 68), dtype=torch.bfloat16, device=DEV)[:, :, :64]
    refused(lambda: Q.append(c, s, odd[:, :2], odd[:, :2]), B.MOE_ERR_INVALID_ARG, "strides")
    shifted = torch.zeros(2 * 4 * 64 + 8, dtype=torch.bfloat16, device=DEV)[1:1 + 512].view(2, 4, 64)
    refused(lambda: Q.attend(c, s, shifted, q), B.MOE_ERR_INVALID_ARG, "aligned")
    refused(lambda: Q.attend(c, s, q, q.cpu()), B.MOE_ERR_INVALID_ARG, "device memory")
    refused(lambda: Q.attend(c, s, q, q, None, w), B.MOE_ERR_INVALID_ARG, "out may be q")
    refused(lambda: Q.attend(c, s, q, torch.zeros((2, 5, 64), dtype=torch.bfloat16, device=DEV)[:, :4], w, None), B.MOE_ERR_INVALID_ARG, "weight_in")
    long, far = Q.Kv8Cache.empty(2, 2, 64, 4096, 32, DEV), Q.Kv8Step(ints([3, 4]), 2, 1, 4000)
    assert Q.attend_workspace_bytes(long, far, 4, False) > 16
    refused(lambda: Q.attend(long, far, q, q.clone(), workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), B.MOE_ERR_OOM, "workspace")
    refused(lambda: Q.evict(c, ints([3, 4]), 4, 32, 0, None, w, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), B.MOE_ERR_OOM, "workspace")
    assert lib.moe_kv8_append(None, c.ref, s.ref, k.data_ptr(), k.data_ptr(), -256, 64) == B.MOE_ERR_INVALID_ARG
    Q.append(c, s, k, k)                                                     # a refused call leaves everything usable
    torch.cuda.synchronize()
