"""The 8-bit key-value cache on the GPU, called in ways that a program may: other streams, large numbers, strides of its own,
long ragged steps.  Compared with the fp64 reference within bounds that are derived from the formats."""
import pytest
import torch

from oracle import kv8_ref as R
from paper_2502_06888_amd import kv8_binding as Q
from test_gpu_kv8 import bounds, evict_state, filled, ints, rand, same, step_for, weight_bounds

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def busy(x, times=40):
    """Work on the current stream that takes some milliseconds and leaves x as it is."""
    for _ in range(times):
        torch.mm(x, x)


def test_workspaces_of_calls_on_another_stream_beside_a_busy_one():
    """What the current stream has freed, but still uses, is not given to a call on another stream."""
    block, hd, heads, kv, L, keep = 64, 128, 16, 4, 4096, 128
    g = torch.Generator().manual_seed(31)
    cache, _, _ = filled(g, 2, kv, L, hd, block, [4000] * 2, poison=False)
    cache.position.copy_(torch.arange(L, dtype=torch.int32))
    step = Q.Kv8Step(ints([3999, 700]), 2, 1, 3999)
    held, nxt = ints([4000, 701]), ints([4000, 701])
    q = rand(g, (2, heads, hd)).to(DEV)
    w_in = torch.rand((2, kv, L), generator=g).to(DEV)
    sizes = [Q.attend_workspace(cache, step, heads, True).numel(), Q.evict_workspace(cache, keep).numel()]
    state = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.position)]
    eye = torch.eye(4096, device=DEV)

    def one(stream):
        for t, s in zip((cache.k, cache.v, cache.k_scale, cache.v_scale, cache.position), state):
            t.copy_(s)
        out, w = torch.zeros_like(q), torch.zeros_like(w_in)
        torch.cuda.synchronize()
        guards = []
        if stream is not None:
            busy(eye)
            for n in sizes:                                      # written behind the busy work, then freed
                t = torch.empty(n, dtype=torch.uint8, device=DEV)
                t.fill_(0x5a)
                guards.append(t.sum(dtype=torch.int64))
                del t
        Q.attend(cache, step, q, out, w_in, w, stream=stream)
        Q.evict(cache, held, 4000, keep, 16, nxt, w, stream=stream)
        torch.cuda.synchronize()
        for n, s in zip(sizes, guards):
            assert int(s) == n * 0x5a
        return [out, w, cache.k.clone(), cache.v.clone(), cache.position.clone()]

    want = one(None)
    side = torch.cuda.Stream()
    for _ in range(2):
        for a, b in zip(want, one(side)):
            assert torch.equal(a, b)


def test_tensors_dropped_behind_a_call_on_another_stream():
    """The lengths of a step, taken by others on the current stream while the other stream is yet to read them."""
    block, hd, heads, kv, L = 32, 64, 8, 2, 512
    g = torch.Generator().manual_seed(32)
    cache, _, _ = filled(g, 3, kv, L, hd, block, [400] * 3, poison=False)
    q, k, v = (rand(g, (3, h, hd)).to(DEV) for h in (heads, kv, kv))
    held = ([399, 20, 111], [60, 200, 7])
    side, eye = torch.cuda.Stream(), torch.eye(4096, device=DEV)
    want, got = [], []
    state = [t.clone() for t in cache.tensors]
    for stream, outs in ((None, want), (side, got)):
        for h in held:
            for t, s in zip(cache.tensors, state):
                t.copy_(s)
            out, w = torch.zeros_like(q), torch.zeros((3, kv, L), device=DEV)
            step = Q.Kv8Step(ints(h), 3, 1, 399, row_offsets=ints([0, 1, 2, 3]), next_position=ints(h))
            torch.cuda.synchronize()
            if stream is not None:
                with torch.cuda.stream(stream):
                    busy(eye)
            Q.append(cache, step, k, v, stream=stream)
            Q.attend(cache, step, q, out, None, w, stream=stream)
            del step
            other = [torch.zeros(4, dtype=torch.int32, device=DEV) for _ in range(3)]
            torch.cuda.synchronize()
            outs += [out, w, cache.k.clone(), cache.position.clone()]
            del other
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("weights", [False, True])
def test_one_long_prompt_among_single_tokens(weights):
    """512 sequences, one of which brings 513 tokens: the bounds allow every pair 33 tiles of rows."""
    block, hd, heads, kv, n = 64, 32, 64, 8, 512
    g = torch.Generator().manual_seed(33)
    cached, new = [(7 * s) % 23 for s in range(n)], [513 if s == 300 else 1 for s in range(n)]
    total = [c + m for c, m in zip(cached, new)]
    L = -(-max(total) // block) * block
    cache, codes, scale = filled(g, n, kv, L, hd, block, total)
    step, off = step_for(cached, new)
    q = rand(g, (off[-1] + 1, heads, hd), 2.0)
    out = torch.full_like(q, -3.0, device=DEV)
    w_in, w = torch.rand((n, kv, L), generator=g), torch.full((n, kv, L), -5.0, device=DEV)
    Q.attend(cache, step, q.to(DEV), out, *((w_in.to(DEV), w) if weights else ()))
    torch.cuda.synchronize()
    ref, want, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q, cached, off, block, w_in)
    m = off[-1]
    assert bool(((out.cpu().double() - ref)[:m].abs() <= bounds(ref, spread, mag, hd)[:m]).all())
    assert bool((out[m:] == -3).all())
    if weights:
        held = ~want.isnan()
        assert bool(((w.cpu().double() - want).abs() <= weight_bounds(want, mag[:m], hd))[held].all())
        assert bool((w.cpu()[~held] == -5).all())


@pytest.mark.parametrize("query", [1.0625 * 2.0 ** 10, 1.0625 * 2.0 ** 18, 1.0625 * 2.0 ** 20, 1.0625 * 2.0 ** 21, -1.0625 * 2.0 ** 21,
                                   1.0625 * 2.0 ** 60, -1.0625 * 2.0 ** 60])
@pytest.mark.parametrize("cached,new", [(700, 1), (3000, 1), (40, 4), (0, 150), (300, 520)])
def test_equal_scores_of_any_size_over_the_largest_values(cached, new, query):
    """Scores from 4.5e5 to 5e20 in magnitude over values up to 448 * 2^119: their mean is finite, so the sums have to be."""
    block, hd, heads, kv, L = 32, 32, 8, 1, 3008
    g = torch.Generator().manual_seed(34)
    cache, codes, scale = filled(g, 1, kv, L, hd, block, [L], poison=False)
    codes[0][:] = 0
    codes[0][..., 5] = 0x7d                                                  # 416
    codes[1] = torch.tensor([0x7e, 0x7e, 0x7a, 0x70], dtype=torch.uint8)[torch.randint(0, 4, codes[1].shape, generator=g)]
    cache.k.copy_(codes[0])
    cache.v.copy_(codes[1])
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(2.0 ** 119)
    q = torch.zeros((new, heads, hd), dtype=torch.bfloat16)
    q[..., 5] = query
    out = torch.zeros((new, heads, hd), dtype=torch.bfloat16, device=DEV)
    w = torch.zeros((1, kv, L), device=DEV)
    Q.attend(cache, Q.Kv8Step(ints([cached]), new, new, cached), q.to(DEV), out, None, w, softmax_scale=0.6875)
    v = R.TABLE[codes[1][0, 0].long()] * 2.0 ** 119
    want, mean = torch.zeros(L, dtype=torch.float64), torch.zeros((new, 1, hd), dtype=torch.float64)
    for i in range(new):
        share = (torch.arange(L) <= cached + i).double() / (cached + i + 1)
        want += heads * share
        mean[i, 0] = share @ v
    # equal scores are equal in 32 bits too: what is left is the rounding of the weights and of the result, and sums in 32 bits
    assert bool(((out.cpu().double() - mean).abs() <= 2.0 ** -8 * mean + (2.0 ** -8 + 2.0 ** -20) * v.max()).all())
    assert bool(((w[0, 0].cpu().double() - want).abs() <= 2.0 ** -18 * want).all())


def test_a_step_without_rows_carries_the_weights_over_and_needs_no_rows():
    block, hd, kv, n, L = 32, 64, 2, 2, 128
    g = torch.Generator().manual_seed(35)
    cache, _, _ = filled(g, n, kv, L, hd, block, [60, 0])
    step = Q.Kv8Step(ints([60, 0]), 0, 0, 60, row_offsets=ints([0, 0, 0]))
    w_in = torch.rand((n, kv, L), generator=g).to(DEV)
    q = torch.zeros(8, dtype=torch.bfloat16, device=DEV)
    for p in (None, q.data_ptr()):
        w = torch.full_like(w_in, -5.0)
        assert Q.load_library().moe_kv8_attend(torch.cuda.current_stream().cuda_stream, cache.ref, step.ref, 4, p, 0, 0, 0.0, p, 0, 0,
                                               w_in.data_ptr(), w.data_ptr(), None, 0) == 0
        assert torch.equal(w[0, :, :60], w_in[0, :, :60]) and bool((w[0, :, 60:] == -5).all()) and bool((w[1] == -5).all())
    rows = torch.zeros((0, 4, hd), dtype=torch.bfloat16, device=DEV)
    w = torch.full_like(w_in, -5.0)
    Q.attend(cache, step, rows, rows, w_in, w)
    assert torch.equal(w[0, :, :60], w_in[0, :, :60]) and bool((w[1] == -5).all())


@pytest.mark.parametrize("hd,heads,kv,cached,new", [
    (128, 8, 2, [100, 31], [1, 1]),                  # decode_kernel, one range
    (64, 12, 2, [5000, 17], [2, 1]),                 # several
    (64, 8, 2, [10, 64], [40, 23]),                  # prompts: four, three, five and eight heads of a group, and one
    (128, 9, 3, [0, 300, 5], [130, 257, 0]),
    (32, 10, 2, [33], [150]),
    (64, 8, 1, [0, 900], [530, 300]),
    (32, 4, 4, [70, 0], [200, 33]),
    (64, 14, 2, [1500], [700]),                      # rows split between workgroups
])
def test_strides_with_weights(hd, heads, kv, cached, new):
    """q as a slice of a fused projection, out as a slice of something wider, rows and heads apart by strides of their own."""
    block = 32
    g = torch.Generator().manual_seed(36 + heads + hd)
    n, total = len(cached), [c + m for c, m in zip(cached, new)]
    L = -(-max(total) // block) * block + block
    cache, codes, scale = filled(g, n, kv, L, hd, block, total)
    step, off = step_for(cached, new)
    m = off[-1]
    fused = rand(g, (m + 2, heads + 2 * kv, hd), 2.0).to(DEV)
    q = fused[:, :heads]
    wide = torch.full((heads + 1, m + 3, hd + 24), -3.0, dtype=torch.bfloat16, device=DEV)
    out = wide[1:, 1:, 8:8 + hd].transpose(0, 1)     # heads farther apart than rows
    w_in = torch.rand((n, kv, L), generator=g)
    w = torch.full((n, kv, L), -5.0, device=DEV)
    before = fused.clone()
    Q.attend(cache, step, q, out, w_in.to(DEV), w)
    torch.cuda.synchronize()
    ref, want, spread, mag = R.attend(codes[0], scale[0], codes[1], scale[1], q.cpu(), cached, off, block, w_in)
    assert bool(((out[:m].cpu().double() - ref[:m]).abs() <= bounds(ref, spread, mag, hd)[:m]).all())
    out[:m] = -3.0
    assert bool((wide == -3).all()) and torch.equal(fused, before)               # nothing beside the heads is written
    held = ~want.isnan()
    assert bool(((w.cpu().double() - want).abs() <= weight_bounds(want, mag[:m], hd))[held].all())
    assert bool((w.cpu()[~held] == -5).all())


@pytest.mark.parametrize("most,keep,recent,kind", [(500, 448, 9, "random"), (700, 512, 0, "ties"), (1000, 512, 64, "random"), (1024, 16, 0, "nan"),
                                                   (1200, 1024, 30, "ties"), (1280, 640, 0, "nan"), (1500, 1024, 64, "random"), (1536, 1520, 3, "ties"),
                                                   (2000, 1024, 0, "nan"), (2048, 1008, 1008, "random")])
def test_many_pairs_keep_what_few_keep(most, keep, recent, kind):
    """Pairs that fill the chip have a wavefront each, few share many: the same result, to the last bit."""
    block, hd, kv, n = 16, 32, 8, 66
    held = [(most - 37 * s) % (most + 1) if s else most for s in range(n)]
    many, _, _, w, pos, nxt = evict_state(block, hd, kv, held, kind, most + keep)
    few = Q.Kv8Cache(*(t.clone() for t in (many.k, many.v, many.k_scale, many.v_scale)), block, many.position.clone())
    outs = []
    for cache, parts in ((many, [(0, n)]), (few, [(s, min(s + 16, n)) for s in range(0, n, 16)])):
        w_out, kept = torch.full((n, kv, w.shape[2]), -5.0, device=DEV), torch.full((n, kv, keep), -9, dtype=torch.int32, device=DEV)
        p_out = torch.full_like(cache.position, -5)
        for a, b in parts:
            one = Q.Kv8Cache(*(t[a:b] for t in cache.tensors[:4]), block, cache.position[a:b])
            Q.evict(one, ints(held[a:b]), most, keep, recent, ints(nxt[a:b]), w[a:b].to(DEV), w_out[a:b], p_out[a:b], kept[a:b])
        torch.cuda.synchronize()
        outs.append((*cache.tensors[:4], w_out, p_out, kept))
    for a, b in zip(*outs):
        same(a, b)


@pytest.mark.parametrize("most", [200, 700, 40000])
def test_a_second_eviction_goes_by_the_positions_that_the_caller_gives(most):
    """Positions run ahead of the slots held once a sequence has been evicted from; without `recent` no slot stays for its position."""
    block, hd, kv, keep = 16, 32, 2, 64
    held, seen = [most, most - 9], [most, most - 9]
    cache, codes, scale, w, pos, _ = evict_state(block, hd, kv, held, "random", most)
    cache.position.copy_(torch.arange(w.shape[2], dtype=torch.int32))
    pos[:] = torch.arange(w.shape[2], dtype=torch.int32)
    weight = w.to(DEV)
    for gone, recent, to in ((0, 20, 64), (5, 16, 48), (10, 0, 16)):         # gone: positions whose tokens are no longer held
        nxt = None if to == 64 else ints(seen)                               # never evicted from: the slots held
        w_ref, p_ref, _ = R.evict(codes, scale, w, pos, held, to, recent, seen, block)
        Q.evict(cache, ints(held), max(held), to, recent, nxt, weight)
        held = [min(h, to) for h in held]
        for s, h in enumerate(held):
            same(weight[s, :, :h], w_ref[s, :, :h])
            assert torch.equal(cache.position[s, :, :h].cpu().long(), p_ref[s, :, :h])
            if recent:
                assert int((cache.position[s, :, :h] >= seen[s] - recent).sum()) == kv * (recent - gone)
        w, pos = weight.cpu(), cache.position.cpu()
        seen = [p + 5 for p in seen]                                         # as if tokens had come and gone
