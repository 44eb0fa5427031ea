"""Attention of several new tokens per sequence (drafted trees, sliding windows) against its definition in 64 bits."""

import math
import random

import pytest
import torch

import token_cases as tc
from paper_2510_13223_amd import bana

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INT_MAX = 2 ** 31 - 1


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def inputs(lens, hq, hkv, rows, seed, width=None):
    cache = tc.Cache(lens, hkv, seed, width)
    g = torch.Generator().manual_seed(seed + 1)
    return cache, torch.randn((rows, hq, tc.D), generator=g).to(torch.bfloat16)


def results(rows, hq, bf16):
    out = torch.full((rows, hq, tc.D), 7.0, dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
    return out, torch.full((rows, hq), 7.0, device=DEV)


def workspace(nbytes):
    return torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV) if nbytes else None  # NaN where it is read unset


def same_outside(out, lse, rb):
    """Rows of no sequence keep what they held."""
    for part in (slice(0, rb[0]), slice(rb[-1], None)):
        assert bool((out[part] == 7.0).all()) and bool((lse[part] == 7.0).all())


def run_tree(cache, q, rb, begin, end, at, masks, scale, bf16, hints=True, ws=True, stream=None):
    rows, hq, _ = q.shape
    k, v = cache.k.to(DEV), cache.v.to(DEV)
    out, lse = results(rows, hq, bf16)
    live = [n for n in cache.lens]
    dims = bana.make_dims(len(cache.lens), hq, cache.hkv, cache.table.shape[1], cache.num_blocks,
                          max_range_tokens=max(live) if hints else 0, total_range_tokens=sum(live) if hints else 0)
    w = workspace(bana.bana_tree_attn_workspace_bytes(dims, rows, len(begin))) if ws else None
    bana.bana_tree_attn(q.to(DEV), ints(rb), k, v, cache.table.to(DEV), ints(begin), ints(end), ints(at),
                        tc.signed(masks).to(DEV), out, lse, scale=scale, workspace=w, dims=dims, stream=stream)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


def run_window(cache, q, rb, seq_lens, window, sinks, scale, bf16, ranges=None, hints=True, ws=True):
    rows, hq, _ = q.shape
    out, lse = results(rows, hq, bf16)
    dims = bana.make_dims(len(cache.lens), hq, cache.hkv, cache.table.shape[1], cache.num_blocks,
                          max_range_tokens=max(cache.lens) if hints else 0,
                          total_range_tokens=sum(cache.lens) if hints else 0)
    w = workspace(bana.bana_window_attn_workspace_bytes(dims, rows, window, sinks)) if ws else None
    more = {} if ranges is None else {"kv_range_begin": ints(ranges[0]), "kv_range_end": ints(ranges[1])}
    bana.bana_window_attn(q.to(DEV), ints(rb), cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV), ints(seq_lens),
                          window, sinks, out, lse, scale=scale, workspace=w, dims=dims, **more)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


def live_rows(out, lse, want, rb):
    s = slice(rb[0], rb[-1])
    ref, ref_lse, bounds = want
    return out[s], lse[s], (ref[s], ref_lse[s], tuple(x[s] for x in bounds))


# (hq, hkv, context lengths, new tokens of each sequence, ranges per sequence)
TREES = [
    (8, 2, [33], [1], 1),
    (4, 1, [0], [5], 1),                                # nothing before the tree
    (32, 8, [100, 17], [8, 3], 2),
    (7, 1, [40, 0, 65], [9, 0, 33], 1),                 # groups of 7, a sequence without rows
    (3, 3, [31, 200], [64, 1], 3),                      # one head per kv head
    (32, 2, [15, 16], [17, 2], 2),                      # groups of 16
    (8, 2, [300], [64], 2),
    (8, 1, [50], [70], 1),                              # more than 64 rows: the nodes behind 64 are not seen
    (12, 4, [1, 2, 3, 40, 5, 90, 7, 8, 9], [2, 1, 0, 12, 1, 1, 0, 6, 2], 2),
    (16, 4, [900, 30], [20, 40], 4),
    (8, 2, [40, 50, 60], [32, 32, 32], 1),              # tiles filled to the last column
    (8, 2, [40, 5, 60, 7, 9], [0, 16, 0, 16, 0], 1),
    (4, 2, [3] * 64, [5] * 64, 1),                      # as many sequences as lanes, and one more
    (4, 2, [3] * 65, [20] * 65, 1),
]


def tree_case(case, seed):
    hq, hkv, lens, news, parts = case
    rng = random.Random(seed)
    rb, rows = tc.rows_of(news, pad=2, first=1)
    cache, q = inputs([n + m for n, m in zip(lens, news)], hq, hkv, rows, seed)
    begin, end = [], []
    for b, n in enumerate(lens):
        cut = [0] + sorted(rng.randint(0, n) for _ in range(parts - 1)) + [n]
        begin.append(cut[:-1])
        end.append(cut[1:])
    begin, end = [list(x) for x in zip(*begin)], [list(x) for x in zip(*end)]
    masks = [0] + [m for n in news for m in tc.random_tree(n, rng)] + [2 ** 64 - 1] * 2
    return cache, q, rb, begin, end, list(lens), masks


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", TREES)
def test_tree(case, bf16):
    cache, q, rb, begin, end, at, masks = tree_case(case, 1)
    want = tc.attention(q, rb, cache, tc.tree_sees(begin, end, at, masks, rb), 0.0884)
    for more in ({}, {"hints": False}, {"ws": False}):
        out, lse = run_tree(cache, q, rb, begin, end, at, masks, 0.0884, bf16, **more)
        same_outside(out, lse, rb)
        tc.check_attention(*live_rows(out, lse, want, rb), bf16)


def test_tree_any_masks_gaps_and_rows_that_see_nothing():
    """Masks that are no tree, ranges with gaps and a token covered twice, rows that see nothing."""
    rng = random.Random(3)
    rb, rows = tc.rows_of([6, 40, 5])
    cache, q = inputs([60, 140, 30], 8, 2, rows, 5)
    begin, end = [[3, 20, 0], [20, 90, 9], [50, 60, 5]], [[18, 55, 0], [20, 95, 9], [52, 85, 5]]
    begin[2][1] = 30  # [30, 85) overlaps [20, 55)
    at = [54, 100, 20]
    masks = [rng.getrandbits(64) & rng.getrandbits(64) for _ in range(rows)]
    masks[3] = masks[46] = masks[50] = 0
    want = tc.attention(q, rb, cache, tc.tree_sees(begin, end, at, masks, rb), 0.1)
    assert bool((want[1][[46, 50]] == -math.inf).all())
    for bf16 in (False, True):
        out, lse = run_tree(cache, q, rb, begin, end, at, masks, 0.1, bf16)
        tc.check_attention(out, lse, want, bf16)
        assert bool((out[[46, 50]] == 0).all())


def test_tree_without_its_nodes_merges_with_them():
    """The context in one call, the nodes in another (tree_begin -1 there), merged: the whole result."""
    case = (8, 2, [100, 37], [9, 20], 1)
    cache, q, rb, begin, end, at, masks = tree_case(case, 7)
    rows, hq, _ = q.shape
    none = [[0] * 2]
    outs = [run_tree(cache, q, rb, begin, end, [-1, -5], masks, 0.1, False),
            run_tree(cache, q, rb, none, none, at, masks, 0.1, False)]
    out, lse = torch.empty((rows, hq, tc.D), device=DEV), torch.empty((rows, hq), device=DEV)
    bana.bana_merge_partials(torch.stack([o for o, _ in outs]).to(DEV), torch.stack([x for _, x in outs]).to(DEV), out,
                             lse)
    want = tc.attention(q, rb, cache, tc.tree_sees(begin, end, at, masks, rb), 0.1)
    # The merge rounds a few times more: 8 steps of 2^-24.
    want[2][2].add_(8)
    tc.check_attention(*live_rows(out.cpu(), lse.cpu(), want, rb), False)


# (hq, hkv, tokens in the cache, of these new, window, sinks)
WINDOWS = [
    (8, 2, [33], [1], 8, 2),
    (32, 8, [500, 90, 17], [1, 1, 1], 64, 4),           # single tokens
    (8, 2, [70], [70], 16, 0),                          # a whole prompt
    (7, 1, [130, 0, 44], [60, 0, 44], 50, 5),
    (3, 3, [129], [128], INT_MAX, 0),                   # plain causal attention
    (32, 2, [90, 31], [40, 31], 1, 1),                  # each row sees itself and the first token
    (4, 1, [200], [150], 33, 64),                       # more sinks than window
    (16, 4, [40, 300], [7, 65], 1000, 3),               # windows that reach past the start
    (8, 1, [16, 17, 15], [16, 17, 15], 5, 0),
    (4, 4, [1, 2], [1, 2], 1, 0),
    (8, 2, [1200], [30], 700, 20),
    (28, 4, [3, 260, 1, 77], [3, 200, 0, 1], 90, 17),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", WINDOWS)
def test_window(case, bf16):
    hq, hkv, lens, news, window, sinks = case
    rb, rows = tc.rows_of(news, pad=3, first=2)
    cache, q = inputs(lens, hq, hkv, rows, 11)
    want = tc.attention(q, rb, cache, tc.window_sees(lens, news, window, sinks), 0.0884)
    for more in ({}, {"hints": False}, {"ws": False}):
        out, lse = run_window(cache, q, rb, lens, window, sinks, 0.0884, bf16, **more)
        same_outside(out, lse, rb)
        tc.check_attention(*live_rows(out, lse, want, rb), bf16)


def test_window_partitions_merge():
    """Tokens split over two calls at any token; the merge gives the whole."""
    lens, news, window, sinks = [150, 61, 20], [50, 1, 20], 40, 6
    rb, rows = tc.rows_of(news)
    cache, q = inputs(lens, 8, 2, rows, 13)
    cut, zero = [101, 3, 20], [0, 0, 0]
    parts = [(zero, cut), (cut, [10 ** 6] * 3)]
    got = []
    for begin, end in parts:
        got.append(run_window(cache, q, rb, lens, window, sinks, 0.1, False, ranges=(begin, end)))
        want = tc.attention(q, rb, cache, tc.window_sees(lens, news, window, sinks, begin, end), 0.1)
        tc.check_attention(*got[-1], want, False)
    out, lse = torch.empty((rows, 8, tc.D), device=DEV), torch.empty((rows, 8), device=DEV)
    bana.bana_merge_partials(torch.stack([o for o, _ in got]).to(DEV), torch.stack([x for _, x in got]).to(DEV), out, lse)
    want = tc.attention(q, rb, cache, tc.window_sees(lens, news, window, sinks), 0.1)
    want[2][2].add_(8)
    tc.check_attention(out.cpu(), lse.cpu(), want, False)


def test_rows_before_the_first_position_see_nothing():
    lens, news = [3, 40], [8, 5]  # five rows of the first sequence lie before its first token
    rb, rows = tc.rows_of(news)
    cache, q = inputs(lens, 8, 2, rows, 17)
    want = tc.attention(q, rb, cache, tc.window_sees(lens, news, 10, 2), 0.1)
    out, lse = run_window(cache, q, rb, lens, 10, 2, 0.1, False)
    tc.check_attention(out, lse, want, False)
    assert bool((out[:5] == 0).all()) and bool((lse[:5] == -math.inf).all())


@pytest.mark.parametrize("nodes", [24, 12])  # tiles of 128 columns and of 64
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_a_row_does_not_see_never_reach_it(bad, nodes):
    """A node and a token whose key and value are not finite: the rows that do not see them are as without them."""
    cache, q, rb, begin, end, at, masks = tree_case((8, 2, [50], [nodes], 1), 19)
    masks = masks[:1] + [1 << i | (1 if i % 2 else 0) for i in range(nodes)] + masks[nodes + 1:]
    clean = [run_tree(cache, q, rb, begin, end, at, masks, 0.1, bf16) for bf16 in (False, True)]
    cache.values[0][50 + 6] = bad
    cache.keys[0][50 + 7] = bad
    cache.values[0][50 + 7, 1, 5] = bad
    cache.store()
    for bf16, (out0, lse0) in zip((False, True), clean):
        out, lse = run_tree(cache, q, rb, begin, end, at, masks, 0.1, bf16)
        other = [r for r in range(rb[0], rb[1]) if r - rb[0] not in (6, 7)]
        assert torch.isfinite(out[other]).all()
        # The slow way round such a block keeps the weights whole: nearer to the definition, not the same bits.
        assert bool(((out[other].double() - out0[other].double()).abs() <= 2.0 ** -6).all())
        assert torch.equal(lse[other], lse0[other])
        assert not torch.isfinite(out[rb[0] + 6]).any()
        if math.isnan(bad):
            assert torch.isnan(out[rb[0] + 7]).all() and torch.isnan(lse[rb[0] + 7]).all()
    # Under a window: a poisoned token in the middle, rows on both sides of its reach.
    cache, q = inputs([100], 8, 2, 60, 23)
    rb = [0, 60]
    clean, lse0 = run_window(cache, q, rb, [100], 20, 3, 0.1, True)
    cache.values[0][55] = bad
    cache.store()
    out, lse = run_window(cache, q, rb, [100], 20, 3, 0.1, True)
    sees = [40 + i >= 55 and 40 + i - 55 < 20 for i in range(60)]
    for i in range(60):
        assert bool(torch.isfinite(out[i]).all()) != sees[i], i
    assert torch.equal(lse, lse0)


def test_nan_and_large_scores():
    """A NaN query makes its row NaN and no other; scores up to 1e4 stay finite."""
    cache, q = inputs([64], 8, 2, 20, 29)
    q[4, 3, 7] = math.nan
    q[9] *= 1000
    out, lse = run_window(cache, q, [0, 20], [64], INT_MAX, 0, 1.0, False)
    assert torch.isnan(out[4, 3]).all() and torch.isnan(lse[4, 3])
    keep = torch.ones(20, 8, dtype=torch.bool)
    keep[4, 3] = False
    assert torch.isfinite(out[keep]).all() and torch.isfinite(lse[keep]).all()
    want = tc.attention(q, [0, 20], cache, tc.window_sees([64], [20], INT_MAX, 0), 1.0)
    s = slice(9, 10)  # one token holds nearly all the weight; a score is off by 2^-23 of its absolute products
    tc.check_attention(out[s], lse[s], (want[0][s], want[1][s], tuple(x[s] for x in want[2])), False)


def test_many_sequences_and_long_ranges_split():
    """300 sequences (the search for a row's sequence takes two rounds), and few rows over long contexts, split."""
    rng = random.Random(31)
    news = [rng.choice([0, 0, 1, 1, 2, 5]) for _ in range(300)]
    lens = [n + rng.randint(0, 20) for n in news]
    rb, rows = tc.rows_of(news, pad=1)
    cache, q = inputs(lens, 4, 2, rows, 37)
    want = tc.attention(q, rb, cache, tc.window_sees(lens, news, 12, 2), 0.1)
    out, lse = run_window(cache, q, rb, lens, 12, 2, 0.1, True)
    tc.check_attention(*live_rows(out, lse, want, rb), True)
    for new, bf16 in ((1, False), (3, True), (40, False)):
        cache, q = inputs([5000, 90 + new], 4, 1, 2 * new, 41 + new)
        rb = [0, new, 2 * new]
        want = tc.attention(q, rb, cache, tc.window_sees([5000, 90 + new], [new, new], 4000, 4), 0.1)
        first = run_window(cache, q, rb, [5000, 90 + new], 4000, 4, 0.1, bf16)
        tc.check_attention(*first, want, bf16)
        for _ in range(3):
            again = run_window(cache, q, rb, [5000, 90 + new], 4000, 4, 0.1, bf16)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_a_tree_of_one_node_is_a_decode_step():
    """One row per sequence over its whole cache: what bana_decode_attn_partial gives, up to rounding."""
    cache, q = inputs([200, 64, 1, 33], 8, 2, 4, 43)
    rb, begin, end = [0, 1, 2, 3, 4], [[0] * 4], [[199, 63, 0, 32]]
    out, lse = run_tree(cache, q, rb, begin, end, [199, 63, 0, 32], [1] * 4, 1.0, False)
    want = torch.empty((4, 8, tc.D), device=DEV), torch.empty((4, 8), device=DEV)
    lens = ints([200, 64, 1, 33])
    bana.bana_decode_attn_partial(q.to(DEV), cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV), lens,
                                  ints([0] * 4), lens, *want)
    assert (out - want[0].cpu()).abs().max() <= 2e-4 and (lse - want[1].cpu()).abs().max() <= 1e-4


def test_streams_and_graphs():
    """On a stream of its own, and captured and replayed with other work between: the eager result each time."""
    cache, q = inputs([700, 50], 8, 2, 14, 47)
    rb, lens = ints([0, 10, 14]), ints([700, 50])
    k, v, table, qd = cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV), q.to(DEV)
    dims = bana.make_dims(2, 8, 2, cache.table.shape[1], cache.num_blocks, max_range_tokens=700, total_range_tokens=750)
    ws = workspace(max(bana.bana_window_attn_workspace_bytes(dims, 14, 600, 4),
                       bana.bana_tree_attn_workspace_bytes(dims, 14, 1)))
    begin, end, at = ints([[0, 0]]), ints([[690, 46]]), ints([690, 46])
    masks = tc.signed([2 ** 10 - 1] * 14).to(DEV)

    def both(stream=None):
        outs = [results(14, 8, True) for _ in range(2)]
        bana.bana_window_attn(qd, rb, k, v, table, lens, 600, 4, *outs[0], workspace=ws, dims=dims, stream=stream)
        bana.bana_tree_attn(qd, rb, k, v, table, begin, end, at, masks, *outs[1], workspace=ws, dims=dims,
                            stream=stream)
        return [x for o in outs for x in o]

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
        got2 = both(side)
    side.synchronize()
    for x, y, z in zip(want, got, got2):
        assert torch.equal(x, y) and torch.equal(x, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for _ in range(4):
        for x in captured:
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, captured):
            assert torch.equal(x, y)
        both()
        torch.cuda.synchronize()


def test_sixty_three_ranges():
    """The most ranges a call may have, one per lane with the nodes: empty ones, single tokens, neighbours."""
    rng = random.Random(53)
    lens, news = [400, 70], [9, 30]
    rb, rows = tc.rows_of(news)
    cache, q = inputs([n + m for n, m in zip(lens, news)], 8, 2, rows, 59)
    begin, end = [[0, 0] for _ in range(63)], [[0, 0] for _ in range(63)]
    for b, n in enumerate(lens):
        cuts = sorted(rng.sample(range(n), 63)) + [n]
        for p in range(63):
            begin[p][b], end[p][b] = cuts[p], rng.choice([cuts[p], cuts[p] + 1, cuts[p + 1], cuts[p + 1]])
    masks = [m for n in news for m in tc.random_tree(n, rng)]
    want = tc.attention(q, rb, cache, tc.tree_sees(begin, end, lens, masks, rb), 0.1)
    for bf16 in (False, True):
        tc.check_attention(*run_tree(cache, q, rb, begin, end, lens, masks, 0.1, bf16), want, bf16)


def test_thousands_of_sequences():
    """More than 64^2 sequences, most of them without a row: the search takes three rounds."""
    rng = random.Random(61)
    news = [rng.choice([0, 0, 0, 1]) for _ in range(4500)]
    news[0], news[-1] = 2, 3
    lens = [n + rng.randint(0, 3) for n in news]
    rb, rows = tc.rows_of(news, pad=2, first=1)
    cache, q = inputs(lens, 2, 1, rows, 67)
    want = tc.attention(q, rb, cache, tc.window_sees(lens, news, 2, 1), 0.1)
    out, lse = run_window(cache, q, rb, lens, 2, 1, 0.1, False)
    same_outside(out, lse, rb)
    tc.check_attention(*live_rows(out, lse, want, rb), False)


def test_calls_at_once_with_workspaces_of_their_own():
    """Two streams, then two graphs, each with its own workspace, under way together: the eager results each time."""
    calls = []
    for new, bf16, seed in ((3, True, 71), (50, False, 73)):
        cache, q = inputs([3000, 900], 8, 2, 2 * new, seed)
        dims = bana.make_dims(2, 8, 2, cache.table.shape[1], cache.num_blocks, max_range_tokens=3000,
                              total_range_tokens=3900)
        ws = workspace(bana.bana_window_attn_workspace_bytes(dims, 2 * new, 2500, 4))
        assert ws is not None
        args = (q.to(DEV), ints([0, new, 2 * new]), cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV),
                ints([3000, 900]), 2500, 4)
        calls.append((args, results(2 * new, 8, bf16), dict(workspace=ws, dims=dims)))
    eager = []
    for args, outs, more in calls:
        bana.bana_window_attn(*args, *outs, **more)
        eager.append([x.clone() for x in outs])
    torch.cuda.synchronize()

    def both_as_eager():
        torch.cuda.synchronize()
        for (_, outs, _), want in zip(calls, eager):
            for x, y in zip(outs, want):
                assert torch.equal(x, y)
                x.fill_(5.0)
        torch.cuda.synchronize()

    streams = [torch.cuda.Stream() for _ in calls]
    both_as_eager()
    for _ in range(10):
        for s, (args, outs, more) in zip(streams, calls):
            bana.bana_window_attn(*args, *outs, stream=s, **more)
    both_as_eager()
    graphs = []
    for args, outs, more in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            bana.bana_window_attn(*args, *outs, **more)
    for _ in range(4):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        both_as_eager()


def test_offsets_past_four_gigabytes():
    """A pool whose tiles lie past 2^32 bytes: the sequence's blocks at its far end."""
    hkv, n = 8, 150000  # 4.9 GB each of keys and values
    cache, q = inputs([100], 16, hkv, 20, 53)
    k = torch.empty((n, hkv, 16, 16, 8), dtype=torch.bfloat16, device=DEV)
    v = torch.empty((n, hkv, 128, 16), dtype=torch.bfloat16, device=DEV)
    far = [n - 1 - 3 * i for i in range(7)]
    table = torch.tensor([far], dtype=torch.int32, device=DEV)
    rb = ints([0, 20])
    key = torch.cat([cache.keys[0]]).to(DEV)
    value = cache.values[0].to(DEV)
    for blk in far:
        k[blk], v[blk] = math.nan, math.nan
    bana.bana_append_kv(key, value, ints([0, 100]), ints([0]), table, k, v)
    out, lse = results(20, 16, False)
    bana.bana_window_attn(q.to(DEV), rb, k, v, table, ints([100]), 30, 4, out, lse, scale=0.1)
    want = tc.attention(q, [0, 20], cache, tc.window_sees([100], [20], 30, 4), 0.1)
    tc.check_attention(out.cpu(), lse.cpu(), want, False)
    del k, v
    torch.cuda.empty_cache()
