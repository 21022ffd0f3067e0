"""Attention over a latent cache on the GPU against the definition in 64 bits, within bounds that are derived from the formats.

A rounding to bf16 is off by 2^-8 of the value at most, to fp16 by 2^-11, to two bf16 by 2^-16.  A score is a sum of products: with one
factor of each rounded it is off by that part of the sum of their magnitudes, and by 2^-14 of it for sums of some hundred terms in 32
bits.  An error d of the scores moves a weight by a factor of e^(2d) at most (d of its own, d of the sum's); weights are rounded once
(absorbed: bf16, and so is their sum's part of each; expanded: fp16), values (expanded: fp16) and u (absorbed: two bf16) too, and outputs."""
import math

import pytest
import torch

from oracle import latent_ref as R
from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import kv8_binding as Q
from paper_2502_06888_amd import latent_binding as L
from paper_2502_06888_amd import rope_binding as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def offsets_of(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def rand(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16)


class Layer:
    """A filled cache, heads and queries on the CPU and the GPU; slots that nobody holds and what lies behind outputs are poison."""

    def __init__(self, seed, cached, new, heads, dims, prefix=0, slack=(0, 0), uniform=False, max_len=None, gap=(0, 0), std=1.0, tail=2):
        g = torch.Generator().manual_seed(seed)
        self.latent, self.rope, self.nope, self.value = dims
        self.cached, self.new, self.heads, self.tail = cached, new, heads, tail
        n, width = len(cached), self.latent + self.rope
        self.max_len = max_len or max(c + m for c, m in zip(cached, new)) + 3
        self.off = offsets_of(new)
        self.rows = rand(g, n, self.max_len, width)
        for s, (c, m) in enumerate(zip(cached, new)):
            self.rows[s, c + m:] = NAN
        self.prefix = rand(g, prefix, width) if prefix else None
        self.w_k, self.w_v = rand(g, heads, self.nope, self.latent, std=self.latent ** -0.5), rand(g, heads, self.value, self.latent, std=self.latent ** -0.5)
        self.q = rand(g, self.off[-1] + tail, heads, self.nope + self.rope, std=std)
        self.q[self.off[-1]:] = NAN
        self.cache = L.LatentCache(self.rows.to(DEV), self.rope, None if self.prefix is None else self.prefix.to(DEV))
        self.h = L.LatentHeads(self.w_k.to(DEV), self.w_v.to(DEV))
        self.step = Q.Kv8Step(ints(cached), self.off[-1], max(new) + slack[0], max(cached) + slack[1], row_offsets=None if uniform else ints(self.off))
        self.gap = gap

    def run(self, form, **kw):
        rows, gap = self.q.shape[0], self.gap
        q = torch.full((rows, self.heads + gap[0], self.nope + self.rope + gap[1]), NAN, dtype=torch.bfloat16, device=DEV)
        q = q[:, :self.heads, :self.nope + self.rope]
        q.copy_(self.q)
        whole = torch.full((rows, self.heads + gap[0], self.value + gap[1]), -7.0, dtype=torch.bfloat16, device=DEV)
        out = whole[:, :self.heads, :self.value]
        ws = L.attend_workspace(self.cache, self.step, self.h, form)
        ws.fill_(0xff)                                                       # NaN wherever something unwritten were read
        L.attend(self.cache, self.step, self.h, q, out, form=form, workspace=ws, **kw)
        torch.cuda.synchronize()
        got = out.cpu().clone()
        out[:self.off[-1]] = -7.0
        assert (whole == -7.0).all(), "something beside the rows was written"
        return got

    def reference(self, scale=None):
        return R.attend(self.rows, self.q, self.w_k, self.w_v, self.cached, self.off, self.prefix, scale)


SCORE = {"absorbed": 2.0 ** -16, "expanded": 2.0 ** -11}                     # roundings of a factor of the scores, of the weights
WEIGHT = {"absorbed": 2.0 ** -8, "expanded": 2.0 ** -11}


def tolerance(form, want, spread, wide, mag):
    d = (SCORE[form] + 2.0 ** -14) * mag[form][..., None]
    tol = (2.0 ** -8 + WEIGHT[form]) * want.abs() + spread * (torch.expm1(2 * d) + 1.01 * WEIGHT[form] + 2.0 ** -14)
    return tol + (2.0 ** -11 * spread if form == "expanded" else (2.0 ** -14 + 2.0 ** -16) * wide) + 2.0 ** -100


def check(got, form, ref):
    want, spread, wide, mag = ref
    there = ~want.isnan().all(-1).all(-1)
    err = (got.double() - want).abs()
    over = (err - tolerance(form, *ref))[there]
    assert not over.isnan().any() and over.max() <= 0, f"over by {over.max():.3e}"
    # independent roundings: half a step of bf16 is 2^-8 at most, 0.41 of it in the mean over a binade: the outputs', and in the absorbed
    # form the weights', which a mean over several of them makes smaller
    rel = (err[there].square().mean() / want[there].square().mean()).sqrt()
    assert rel <= 2.0 ** -8 * 0.65, f"off by {rel:.3e} in the mean"


WIDE, SMALL = (512, 64, 128, 128), (256, 32, 64, 64)
ABSORBED, EXPANDED = "absorbed", "expanded"
FORMS = [ABSORBED, EXPANDED]

CASES = [
    # heads, dims, cached, new, prefix
    (1, (128, 32, 32, 32), [0], [1], 0),                                      # one token that sees itself
    (32, WIDE, [700], [1], 0),
    (32, WIDE, [0, 31, 32, 33, 63, 64, 255], [1] * 7, 0),                     # ends within and at tiles
    (8, WIDE, [513, 0, 1200], [1, 1, 1], 0),
    (128, WIDE, [300, 5, 97], [1, 1, 1], 0),
    (64, WIDE, [40, 700], [1, 1], 0),                                         # two wavefronts side by side
    (5, SMALL, [17, 250, 0], [3, 1, 2], 0),
    (16, SMALL, [100, 0, 33, 64], [7, 40, 0, 1], 0),
    (20, WIDE, [3, 200], [67, 31], 0),
    (40, (512, 32, 64, 32), [11, 90], [5, 2], 0),
    (3, (256, 64, 32, 128), [129], [50], 0),
    (2, (128, 64, 128, 64), [1, 2, 3], [33, 64, 1], 0),
    (33, (128, 32, 64, 128), [70], [3], 0),                                   # one row more than a tile
    (7, WIDE, [0, 0], [130, 97], 0),
    (130, (128, 32, 32, 64), [64, 9], [1, 2], 0),
    (32, WIDE, [0, 10, 100], [1, 1, 1], 1),                                   # prefixes
    (20, WIDE, [5, 0, 61], [1, 4, 2], 517),
    (16, SMALL, [0, 0, 0, 0, 9], [3, 1, 20, 0, 1], 1300),
    (128, (256, 32, 128, 64), [31], [1], 95),
    (9, (128, 64, 64, 64), [3, 4], [2, 70], 64),
]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_is_within_its_bounds(case, form):
    heads, dims, cached, new, prefix = CASES[case]
    x = Layer(case + 1, cached, new, heads, dims, prefix)
    check(x.run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("case", [2, 7, 16, 19])
def test_bounds_wider_than_the_lengths_and_strides(case, form):
    heads, dims, cached, new, prefix = CASES[case]
    x = Layer(case + 100, cached, new, heads, dims, prefix, slack=(9, 900), max_len=1600, gap=(3, 8))
    check(x.run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("heads,dims,n_seq,longest,every", [(8, (128, 32, 32, 32), 70, 900, 3), (40, SMALL, 131, 700, 4), (128, WIDE, 9, 1500, 2),
                                                            (4, (128, 32, 32, 32), 300, 1990, 60)])
def test_many_sequences_of_uneven_lengths(heads, dims, n_seq, longest, every, form):
    """Work of sequences with none, one or many ranges, whole or not, with none to three tokens."""
    g = torch.Generator().manual_seed(n_seq)
    cached = [int(torch.randint(0, longest if i % every == 1 else 60, (1,), generator=g)) for i in range(n_seq)]
    cached[every + 1], cached[-1] = longest, 0
    new = [i % 4 if every < 10 else 1 for i in range(n_seq)]
    x = Layer(90 + n_seq, cached, new, heads, dims)
    check(x.run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
def test_steps_without_offsets_scales_and_heads_of_one_matrix(form):
    x = Layer(50, [40, 7, 300], [2, 2, 2], 20, WIDE, prefix=33, uniform=True, tail=0)
    both = torch.cat((x.w_k, x.w_v), 1).to(DEV)                               # [heads, nope + value, latent]
    x.h = L.LatentHeads(both[:, :128], both[:, 128:])
    check(x.run(form, softmax_scale=0.04), form, x.reference(0.04))


@pytest.mark.parametrize("form", FORMS)
def test_a_sequence_does_not_depend_on_the_others(form):
    a = Layer(60, [100, 333, 0], [5, 1, 9], 20, WIDE, prefix=100)
    first = a.run(form)
    a.cache.rows[0] = 1.5
    a.cache.rows[2] = -3.0
    a.q[:5] = 0.25
    a.q[6:15] = 2.0
    assert torch.equal(a.run(form)[5:6], first[5:6])


@pytest.mark.parametrize("form", FORMS)
def test_numbers_outside_their_bounds_stay_within_the_tensors(form):
    """Lengths and offsets that are not what the host said: any result, nothing written outside (poison around the outputs)."""
    x = Layer(70, [60, 3], [4, 4], 8, SMALL, max_len=64)
    for cached, off in (([2 ** 31 - 1, -5], [0, 4, 8]), ([60, 3], [-9, 2 ** 31 - 1, 3]), ([60, 64], [5, 2, 8]), ([-1, 64], [8, 8, 100])):
        x.step.cached.copy_(ints(cached))
        x.step.row_offsets.copy_(ints(off))
        x.run(form)


@pytest.mark.parametrize("form", FORMS)
def test_tokens_beyond_the_last_slot_do_not_exist(form):
    x = Layer(71, [60, 62, 10], [4, 2, 3], 8, SMALL, max_len=62)
    got = x.run(form)
    want = x.reference()
    assert (got[2:6] == -7.0).all()                                           # rows of tokens that found no slot
    check(got, form, want)


@pytest.mark.parametrize("form", FORMS)
def test_a_step_without_rows_and_sequences_without_tokens(form):
    x = Layer(72, [5, 3], [0, 0], 8, SMALL)
    assert L.attend_workspace_bytes(x.cache, x.step, x.h, form) == 0
    out = torch.full((4, 8, 64), -7.0, dtype=torch.bfloat16, device=DEV)
    L.attend(x.cache, x.step, x.h, torch.zeros((4, 8, 96), dtype=torch.bfloat16, device=DEV), out, form=form)
    torch.cuda.synchronize()
    assert (out == -7.0).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("what", ["nan", "inf", "rope"])
@pytest.mark.parametrize("heads,dims,cached,new", [(4, SMALL, [20], [60]), (20, WIDE, [3], [40]), (32, (128, 32, 64, 64), [0, 40], [3, 6])])
def test_what_is_not_finite_reaches_the_rows_that_see_it_and_no_others(heads, dims, cached, new, what, form):
    x = Layer(80, cached, new, heads, dims)
    want = x.reference()
    token = new[0] // 2                                                       # of the first sequence
    slot, bad = cached[0] + token, float("inf") if what == "inf" else NAN
    x.cache.rows[0, slot, dims[0] + 3 if what == "rope" else dims[0] // 2 + 1] = bad
    got = x.run(form)
    row, hit = torch.arange(got.shape[0]), torch.zeros(got.shape[0], dtype=torch.bool)
    hit[token:new[0]] = True
    assert got[:x.off[-1]][hit[:x.off[-1]]].isnan().all()
    good = [t.clone() for t in want[:3]]
    good[0][hit] = NAN                                                        # as rows of no sequence
    check(torch.where(hit[:, None, None], torch.zeros((), dtype=got.dtype), got), form, (*good, want[3]))
    x.cache.rows[0, slot] = 0.5
    x.q[new[0] - 1, 1, 2] = bad                                               # and of the queries
    got = x.run(form)
    assert got[new[0] - 1, 1].isnan().all() and got[:x.off[-1]].isnan().sum() == x.value


@pytest.mark.parametrize("form", FORMS)
def test_a_prefix_that_is_not_finite_reaches_everybody(form):
    x = Layer(81, [5, 9], [1, 3], 8, SMALL, prefix=70)
    x.cache.prefix[33, 7] = NAN
    assert x.run(form)[:4].isnan().all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("size", [30.0, 3e4, 1e12, 1e17])
def test_scores_of_any_size(size, form):
    """The largest score wins; with scores this far apart every row's output is the value of one slot."""
    x = Layer(82, [40, 9], [3, 1], 8, SMALL)
    x.q.mul_(size)
    x.q[x.off[-1]:] = 0
    x.cache = L.LatentCache(torch.nan_to_num(x.rows).to(DEV), x.rope)
    z = R.attend(torch.nan_to_num(x.rows), x.q, x.w_k, x.w_v, x.cached, x.off)[0]
    got = x.run(form)[:x.off[-1]].double()
    if size >= 3e4:
        # the two largest scores of a row may be closer than their errors: rows whose winner leads clearly
        lead = winners(x)
        assert lead.sum() >= 8
        err = (got - z[:x.off[-1]]).abs()[lead]
        wide = 2.0 ** -6 * (1 + z[:x.off[-1]].abs()[lead])
        assert (err <= wide).all()
    else:
        assert got.isfinite().all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sizes", [(1e-6, 1e-6, 1e-6), (1e6, 1e6, 1e6), (1e30, 1e30, 1e30), (1.0, 3e4, 1.0), (3e4, 1.0, 1e-4), (0.0, 1.0, 200.0), (1e-3, 0.0, 0.0)])
def test_latents_of_any_size(sizes, form):
    """Latents of one size in the first 64 slots, of another in the next 64 and another behind them, under queries that keep the scores small."""
    x = Layer(83, [150, 30], [2, 70], 4, (128, 32, 32, 64))
    for i, f in enumerate(sizes):
        x.rows[:, 64 * i:64 * (i + 1) if i < 2 else None, :128] *= f
    x.q[..., :32] /= max(sizes)
    x.cache = L.LatentCache(x.rows.to(DEV), x.rope)
    check(x.run(form), form, x.reference())


def winners(x):
    """(row, head) whose largest score leads the next by more than both can be off, 2 * (2^-8 + 2^-14) of the magnitudes
    behind them."""
    lead = torch.zeros((x.off[-1], x.heads), dtype=torch.bool)
    rows = torch.nan_to_num(x.rows).double()
    for s, (c, m) in enumerate(zip(x.cached, x.new)):
        for i in range(m):
            for h in range(x.heads):
                r = rows[s, :c + i + 1]
                k = torch.cat((r[:, :x.latent] @ x.w_k[h].double().T, r[:, x.latent:]), 1)
                y = x.q[x.off[s] + i, h].double()
                a = torch.cat((y[:x.nope] @ x.w_k[h].double(), y[x.nope:]))
                z, mag = k @ y, r.abs() @ a.abs()
                mag2 = k.abs() @ y.abs()
                top = z.topk(min(2, z.numel())).values
                lead[x.off[s] + i, h] = z.numel() == 1 or bool(top[0] - top[1] > 0.01 * max(mag.max(), mag2.max()))
    return lead


@pytest.mark.parametrize("form", FORMS)
def test_many_slots_in_ranges_and_a_long_prefix(form):
    x = Layer(90, [5000, 17], [1, 2], 4, (128, 32, 32, 32), prefix=3001, max_len=5100)
    check(x.run(form), form, x.reference())
    x = Layer(91, [2900], [1], 130, (128, 32, 32, 32), max_len=2950)
    check(x.run(form), form, x.reference())


@pytest.mark.parametrize("heads,prefix", [(130, 150), (251, 0)])
def test_heads_in_sets_whose_last_one_is_smaller(heads, prefix):
    """Bounds under which the keys and values of all heads do not fit the last-level cache."""
    x = Layer(96, [100, 3, 700], [3, 1, 40], heads, WIDE, prefix=prefix, slack=(0, 1300), max_len=2100)
    check(x.run(EXPANDED), EXPANDED, x.reference())


@pytest.mark.parametrize("form", FORMS)
def test_offsets_beyond_32_bits(form):
    """The last sequence of a cache of more than 2^32 elements."""
    n, max_len, heads = 9, 1 << 20, 2
    dims = (512, 64, 32, 32)
    rows = torch.empty((n, max_len, 576), dtype=torch.bfloat16, device=DEV)    # 10.9 GB
    x = Layer(92, [300] + [0] * (n - 2) + [400], [1] * n, heads, dims, max_len=420)
    rows[:, :420] = x.cache.rows
    x.cache = L.LatentCache(rows, 64)
    check(x.run(form), form, x.reference())


@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("heads", [2, 8])
def test_bounds_beyond_the_last_level_cache(heads, prefix):
    """Slots read past the last-level cache; with a prefix in the same launch (all rows in one tile) and in one of its own."""
    n, max_len = 9, 1 << 15
    x = Layer(99, [300, 0, 1, 63, 64, 65, 200, 31, 400], [1] * n, heads, (512, 64, 32, 32), prefix=prefix, slack=(0, 29000), max_len=420)
    rows = torch.full((n, max_len, 576), NAN, dtype=torch.bfloat16, device=DEV)
    rows[:, :420] = x.cache.rows
    x.cache = L.LatentCache(rows, 64, x.cache.prefix)
    check(x.run(ABSORBED), ABSORBED, x.reference())


@pytest.mark.parametrize("form", FORMS)
def test_replays_of_a_captured_step_follow_the_lengths(form):
    x = Layer(93, [50, 200], [3, 1], 20, WIDE, prefix=40, slack=(2, 100), max_len=420)
    q, out = x.q.to(DEV), torch.zeros((x.q.shape[0], 20, 128), dtype=torch.bfloat16, device=DEV)
    ws = L.attend_workspace(x.cache, x.step, x.h, form)
    L.attend(x.cache, x.step, x.h, q, out, form=form, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.attend(x.cache, x.step, x.h, q, out, form=form, workspace=ws)
    g = torch.Generator().manual_seed(5)
    x.rows = rand(g, 2, 420, 576)
    x.cache.rows.copy_(x.rows)
    for cached, new in (([50, 200], [3, 1]), ([0, 300], [1, 3]), ([299, 7], [4, 0])):
        x.cached, x.new, x.off = cached, new, offsets_of(new)
        x.step.cached.copy_(ints(cached))
        x.step.row_offsets.copy_(ints(x.off))
        out.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(out, -7.0)
        L.attend(x.cache, x.step, x.h, q, eager, form=form)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        check(torch.where(out == -7.0, 0.0, out).cpu(), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
def test_another_stream_and_tensors_dropped_behind_the_call(form):
    x = Layer(94, [30, 600], [2, 1], 20, WIDE, prefix=64)
    want = x.run(form)
    s = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        q, out = x.q.to(DEV), torch.full(want.shape, -7.0, dtype=torch.bfloat16, device=DEV)
    s.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-3                                             # the current stream has work of its own
    L.attend(x.cache, x.step, x.h, q, out, form=form, stream=s)               # with a workspace of its own
    del q
    torch.full((1 << 24,), NAN, device=DEV)                                   # memory that is handed out next
    s.synchronize()
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("form", FORMS)
def test_graphs_that_share_a_workspace_and_calls_at_once(form):
    """Two captured steps of other sizes over one workspace, replayed in turn; then both at once with a workspace each, guards behind."""
    a, b = Layer(97, [700, 3, 90], [1, 1, 1], 128, WIDE), Layer(98, [40, 500], [30, 2], 8, SMALL, prefix=200)
    want = [x.run(form) for x in (a, b)]
    need = [L.attend_workspace_bytes(x.cache, x.step, x.h, form) for x in (a, b)]
    shared = torch.full((max(need),), 0xff, dtype=torch.uint8, device=DEV)
    q, out = [x.q.to(DEV) for x in (a, b)], [torch.full(w.shape, -7.0, dtype=torch.bfloat16, device=DEV) for w in want]
    graphs = []
    for i, x in enumerate((a, b)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            L.attend(x.cache, x.step, x.h, q[i], out[i], form=form, workspace=shared)
    for i in (0, 1, 1, 0, 1, 0):
        out[i].fill_(-7.0)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[i].cpu(), want[i])
        shared.fill_(0xff)
    streams = [torch.cuda.Stream() for _ in range(2)]
    own = [torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device=DEV) for n in need]
    torch.cuda.synchronize()
    for _ in range(8):
        for i, x in enumerate((a, b)):
            L.attend(x.cache, x.step, x.h, q[i], out[i], form=form, workspace=own[i][:need[i]], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i].cpu(), want[i]) and (own[i][need[i]:] == 0xa5).all()


def test_refused_on_the_device():
    x = Layer(95, [5], [1], 8, SMALL, tail=0)
    q, out = x.q.to(DEV), torch.zeros((1, 8, 64), dtype=torch.bfloat16, device=DEV)
    ws = L.attend_workspace(x.cache, x.step, x.h)
    two = torch.zeros((1, 8, 128), dtype=torch.bfloat16, device=DEV)
    for call in (lambda: L.attend(x.cache, x.step, x.h, q, out, workspace=ws[:ws.numel() - 1]), lambda: L.attend(x.cache, x.step, x.h, q, out, workspace=ws[1:]),
                 lambda: L.attend(x.cache, x.step, x.h, q, out.cpu(), workspace=ws), lambda: L.attend(x.cache, x.step, x.h, q, two[:, :, 1:65], workspace=ws),
                 lambda: L.attend(x.cache, x.step, x.h, q, out[:, :1].expand(1, 8, 64), workspace=ws),
                 lambda: L.attend(x.cache, x.step, x.h, q, q[:, :, :64], workspace=ws), lambda: L.append(x.cache, x.step, torch.zeros((1, 288), dtype=torch.bfloat16))):
        with pytest.raises(B.MoeError):
            call()


# ---- append ------------------------------------------------------------------------------------------

ROPES = [None, dict(rot_dim=32, theta=1e4, interleaved=True), dict(rot_dim=10, theta=1e6, first=5, factor=4.0, original_len=4096, magnitude=1.14),
         dict(rot_dim=32, theta=1e4), dict(rot_dim=12, theta=1e4, first=3, interleaved=True)]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("rope", range(len(ROPES)))
@pytest.mark.parametrize("dims", [(512, 64), (256, 32), (128, 64)])
def test_append_writes_the_rows_of_the_new_tokens_only(dims, rope, norm):
    g = torch.Generator().manual_seed(rope * 10 + dims[0])
    latent, width = dims[0], sum(dims)
    cached, new, nxt = [5, 0, 61, 3, 0, 20], [1, 3, 2, 0, 70, 9], [5, 1000000, 61, 3, 0, 7]
    off = offsets_of(new)
    x = rand(g, off[-1] + 3, width + 8, std=3.0)[:, :width]
    x[off[-1]:] = NAN
    w = rand(g, latent) if norm else None
    start = rand(g, 6, 64, width)                                             # the last tokens of 2 and 4 find no slot
    cfg = ROPES[rope]
    cache = L.LatentCache(start.clone().to(DEV), dims[1])
    step = Q.Kv8Step(ints(cached), off[-1], 64, 64, row_offsets=ints(off), next_position=ints(nxt))
    dev = torch.empty((x.shape[0], width + 8), dtype=torch.bfloat16, device=DEV)[:, :width]
    dev.copy_(x)
    L.append(cache, step, dev, norm=None if w is None else w.to(DEV), eps=1e-5, rope=None if cfg is None else P.Rope(**cfg))
    torch.cuda.synchronize()
    want = start.double()
    names = {"rot_dim": "rot"}
    R.append(want, x, cached, off, latent, w, 1e-5, None if cfg is None else {names.get(k, k): v for k, v in cfg.items()}, nxt)
    got = cache.rows.cpu()
    # half a step of bf16; sums of up to 512 squares, a root, a quotient and two products in 32 bits; turned pairs as for rotate
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs()
    tol[..., latent:] += 2.0 ** -21 * 1.2 * 2 * 3.0 * 5.5
    written = torch.zeros((6, 64), dtype=torch.bool)
    for s, (c, m) in enumerate(zip(cached, new)):
        written[s, c:min(c + m, 64)] = True
    assert torch.equal(got[~written], start[~written])
    assert ((got.double() - want).abs() <= tol)[written].all()
    if cfg is None and not norm:
        assert torch.equal(got.double(), want)


def test_append_of_rows_that_are_not_finite_or_zero():
    x = torch.ones((4, 288), dtype=torch.bfloat16)
    x[0, 3], x[1, 260], x[2] = NAN, float("inf"), 0
    cache = L.LatentCache(torch.zeros((4, 2, 288), dtype=torch.bfloat16, device=DEV), 32)
    step = Q.Kv8Step(ints([0] * 4), 4, 1, 0, next_position=ints([1] * 4))
    L.append(cache, step, x.to(DEV), norm=torch.ones(256, dtype=torch.bfloat16, device=DEV), rope=P.Rope(32))
    got = cache.rows[:, 0].cpu()
    assert got[0, :256].isnan().all() and got[0, 256:].isfinite().all()
    assert got[1, :256].isfinite().all() and (~got[1].isfinite()).nonzero().flatten().tolist() == [260, 276]
    assert (got[2] == 0).all() and got[3].isfinite().all() and (cache.rows[:, 1] == 0).all()


def test_append_positions_follow_the_prefix_and_the_slots():
    """Without next_position a token's position is prefix_len + cached + its place."""
    g = torch.Generator().manual_seed(9)
    x, prefix = rand(g, 3, 160).to(DEV), rand(g, 77, 160).to(DEV)
    step = Q.Kv8Step(ints([4]), 3, 3, 4)
    given = Q.Kv8Step(ints([4]), 3, 3, 4, next_position=ints([81]))
    a, b = (L.LatentCache(torch.zeros((1, 8, 160), dtype=torch.bfloat16, device=DEV), 32, prefix) for _ in "ab")
    L.append(a, step, x, rope=P.Rope(32))
    L.append(b, given, x, rope=P.Rope(32))
    assert torch.equal(a.rows, b.rows) and a.rows[0, 5].any()


def test_append_finds_the_sequence_among_thousands():
    n = 5000
    g = torch.Generator().manual_seed(10)
    new = [int(v) for v in torch.randint(0, 3, (n,), generator=g)]
    off = offsets_of(new)
    x = torch.arange(off[-1], dtype=torch.float32)[:, None].expand(-1, 160).contiguous()
    x = torch.cat(((x // 256).to(torch.bfloat16)[:, :128], (x % 256).to(torch.bfloat16)[:, :32]), 1).contiguous()
    cache = L.LatentCache(torch.full((n, 2, 160), -1.0, dtype=torch.bfloat16, device=DEV), 32)
    L.append(cache, Q.Kv8Step(ints([0] * n), off[-1], 2, 0, row_offsets=ints(off)), x.to(DEV))
    want = torch.full((n, 2, 160), -1.0, dtype=torch.bfloat16)
    for s in range(n):
        want[s, :new[s]] = x[off[s]:off[s + 1]]
    assert torch.equal(cache.rows.cpu(), want)


def test_a_run_of_rotation_append_and_attention_as_a_model_makes_it():
    """A shared instruction as a batch of one, prompts behind it, then single tokens: every step against the definition on the rows
    that the cache holds, and the cache against the definition on the rows that came in."""
    g = torch.Generator().manual_seed(11)
    heads, (latent, rope, nope, value) = 8, WIDE
    turn = dict(rot_dim=rope, theta=1e4, interleaved=True)
    on_q = P.Rope(first=nope, **turn)
    ref = dict(rot=rope, theta=1e4, interleaved=True)
    w_k, w_v, norm = rand(g, heads, nope, latent, std=latent ** -0.5), rand(g, heads, value, latent, std=latent ** -0.5), rand(g, latent)
    h = L.LatentHeads(w_k.to(DEV), w_v.to(DEV))

    def step(cache, cached, new, before, form):
        off = offsets_of(new)
        x, q = rand(g, off[-1], latent + rope), rand(g, off[-1], heads, nope + rope)
        s = Q.Kv8Step(ints(cached), off[-1], max(new), max(cached), row_offsets=ints(off))
        was = cache.rows.cpu().double()
        L.append(cache, s, x.to(DEV), norm=norm.to(DEV), rope=P.Rope(**turn))
        place = torch.tensor([before + c + i for c, n in zip(cached, new) for i in range(n)], dtype=torch.int32)
        turned = q.to(DEV)
        P.rotate(on_q, place.to(DEV), turned)
        out = torch.zeros((off[-1], heads, value), dtype=torch.bfloat16, device=DEV)
        L.attend(cache, s, h, turned, out, form=form)
        torch.cuda.synchronize()
        R.append(was, x, cached, off, latent, norm, 1e-6, ref, [before + c for c in cached])
        now = cache.rows.cpu()
        for i, (c, n) in enumerate(zip(cached, new)):
            assert ((now[i, :c + n].double() - was[i, :c + n]).abs() <= (2.0 ** -8 + 2.0 ** -18) * was[i, :c + n].abs() + 2.0 ** -16).all()
        assert ((turned.cpu().double() - R.rotate(q, place, first=nope, **ref)).abs() <= 2.0 ** -8 * 8).all()
        prefix = None if cache.prefix is None else cache.prefix.cpu()
        check(out.cpu(), used(cache, s, h, form), R.attend(now, turned.cpu(), w_k, w_v, cached, off, prefix))
        return [c + n for c, n in zip(cached, new)]

    shared = L.LatentCache(torch.full((1, 90, 576), NAN, dtype=torch.bfloat16, device=DEV), rope)
    assert step(shared, [0], [90], 0, "auto") == [90]
    cache = L.LatentCache(torch.full((3, 60, 576), NAN, dtype=torch.bfloat16, device=DEV), rope, prefix=shared.rows[0])
    held = step(cache, [0, 0, 0], [33, 1, 20], 90, "auto")
    held = step(cache, held, [5, 0, 2], 90, "absorbed")
    for _ in range(4):
        held = step(cache, held, [1, 1, 1], 90, "auto")
    assert held == [42, 5, 26]


def used(cache, step, heads, form):
    """The form that a call takes, by what it asks of memory."""
    if form != "auto":
        return form
    need = {f: L.attend_workspace_bytes(cache, step, heads, f) for f in ("auto", ABSORBED, EXPANDED)}
    assert need[ABSORBED] != need[EXPANDED]
    return ABSORBED if need["auto"] == need[ABSORBED] else EXPANDED
