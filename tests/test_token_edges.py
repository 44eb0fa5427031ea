"""Calls on new tokens and blocks where the cache or the batch is unusual: scores and values that are not finite, counts
and entries that do not fit together, rows spread unevenly over many sequences."""

import math

import numpy as np
import pytest
import torch

import token_cases as tc
from paper_2510_13223_amd import bana

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def same(x, y):
    """Equal bit for bit (pools hold NaN)."""
    x, y = x.cpu(), y.cpu()
    if x.dtype == torch.bfloat16:
        x, y = x.view(torch.int16), y.view(torch.int16)
    return torch.equal(x, y)


def run(cache, q, rb, bf16, window=None, tree=None, ws=True):
    """(out, lse) of one attention call: window = (seq_lens, window, sinks), tree = (begin, end, tree_begin, masks)."""
    rows, hq, _ = q.shape
    out = torch.full((rows, hq, tc.D), 7.0, dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
    lse = torch.full((rows, hq), 7.0, device=DEV)
    dims = bana.make_dims(len(cache.lens), hq, cache.hkv, cache.table.shape[1], cache.num_blocks,
                          max_range_tokens=max(cache.lens), total_range_tokens=sum(cache.lens))
    n = (bana.bana_window_attn_workspace_bytes(dims, rows, *window[1:]) if window else
         bana.bana_tree_attn_workspace_bytes(dims, rows, len(tree[0])))
    w = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if ws and n else None
    args = (q.to(DEV), ints(rb), cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV))
    more = dict(scale=0.0884, workspace=w, dims=dims)
    if window:
        bana.bana_window_attn(*args, ints(window[0]), *window[1:], out, lse, **more)
    else:
        begin, end, at, masks = tree
        bana.bana_tree_attn(*args, ints(begin), ints(end), ints(at), tc.signed(masks).to(DEV), out, lse, **more)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


def queries(rows, hq, seed):
    return torch.randn((rows, hq, tc.D), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


# ---- scores and values that are not finite ----------------------------------------------------------

@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("news", [3, 60])  # tiles of 64 columns and of 128
def test_scores_of_minus_infinity_give_zero_whatever_the_values(news, bf16, ws):
    """A row whose scores are all -inf is as one that sees nothing, also where its values are infinite or NaN."""
    lens = [900, 100]
    cache = tc.Cache(lens, 2, 3)
    cache.keys[0][:, :, 0] = -math.inf
    cache.values[0][:, :, 5], cache.values[0][:, 1, 70], cache.values[0][899, :, 9] = math.inf, math.nan, -math.inf
    cache.store()
    rb, rows = tc.rows_of([news, news])
    q = queries(rows, 8, 4)
    q[:, :, 0] = 1.0
    before = [n - news for n in lens]
    for call in (dict(window=(lens, 2000, 0)), dict(tree=([[0, 0]], [before], before, [2 ** 64 - 1] * rows))):
        out, lse = run(cache, q, rb, bf16, ws=ws, **call)
        assert bool((out[:news] == 0).all()) and bool((lse[:news] == -math.inf).all())
        assert bool(torch.isfinite(out[news:]).all()) and bool(torch.isfinite(lse[news:]).all())


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("news", [3, 60])  # tiles of 64 columns and of 128
def test_infinite_values_that_rows_see(news, bf16, ws):
    """What the definition gives, wherever the token lies: +-inf for one of them, NaN for both signs or a NaN; no other
    dim, head or row is touched."""
    lens = [700, 90]
    rb, rows = tc.rows_of([news, min(news, 40)])
    q = queries(rows, 8, 6)
    for at in (3, 200, 401, 640, 698):  # blocks that all rows see whole, and blocks that they see in part
        cache = tc.Cache(lens, 2, 5)
        window = (lens, 650, 2)
        clean, clean_lse = run(cache, q, rb, bf16, window=window, ws=ws)
        cache.values[0][at, 0, 17] = math.inf
        cache.values[0][at, 0, 18] = -math.inf
        cache.values[0][at, 0, 19] = math.nan
        cache.values[0][at, 0, 100], cache.values[0][at + 1, 0, 100] = math.inf, -math.inf
        cache.store()
        out, lse = run(cache, q, rb, bf16, window=window, ws=ws)
        want = clean.clone()
        pos = [700 - news + i for i in range(news)]
        sees = [t <= p and (p - t < 650 or t < 2) for t in (at, at + 1) for p in pos]
        one, other = torch.tensor(sees[:news]), torch.tensor(sees[news:])
        first = want[:news, :4]  # the kv head's query heads
        first[one, :, 17], first[one, :, 18], first[one, :, 19] = math.inf, -math.inf, math.nan
        first[one & ~other, :, 100], first[~one & other, :, 100] = math.inf, -math.inf
        first[one & other, :, 100] = math.nan
        assert torch.equal(lse, clean_lse)
        assert torch.equal(torch.isnan(out), torch.isnan(want)), at
        assert torch.equal(torch.nan_to_num(out, 1e30), torch.nan_to_num(want, 1e30)), at


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("nodes", [24, 12])  # tiles of 128 columns and of 64
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_rows_keep_their_bits_beside_values_that_they_do_not_see(bad, nodes, bf16):
    """Nodes whose key or value is not finite: the rows that do not see them keep every bit of the result."""
    cache = tc.Cache([50 + nodes], 2, 19)
    rb, rows = tc.rows_of([nodes], pad=1, first=1)
    q = queries(rows, 8, 20)
    masks = [0] + [1 << i | (1 if i % 2 else 0) for i in range(nodes)] + [2 ** 64 - 1]
    tree = ([[0]], [[50]], [50], masks)
    clean, clean_lse = run(cache, q, rb, bf16, tree=tree)
    cache.values[0][56] = bad
    cache.keys[0][57] = bad
    cache.values[0][57, 1, 5] = bad
    cache.store()
    out, lse = run(cache, q, rb, bf16, tree=tree)
    other = [r for r in range(1, nodes + 1) if r - 1 not in (6, 7)]
    assert torch.equal(out[other], clean[other]) and torch.equal(lse[other], clean_lse[other])
    assert not torch.isfinite(out[7]).any()
    cache = tc.Cache([100], 2, 23)
    q, window = queries(2 * nodes, 8, 24), ([100], 20, 3)
    clean, clean_lse = run(cache, q, [0, 2 * nodes], bf16, window=window)
    cache.values[0][85] = bad
    cache.store()
    out, lse = run(cache, q, [0, 2 * nodes], bf16, window=window)
    sees = torch.tensor([85 <= 100 - 2 * nodes + i < 105 for i in range(2 * nodes)])
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse, clean_lse)
    assert not torch.isfinite(out[sees]).any()


# ---- counts and entries that do not fit together ----------------------------------------------------

class Blocks:
    """A table with its counts and a pool of random tiles, on the device; `lens` tokens a sequence, one count an entry."""

    def __init__(self, lens, num_blocks, width, seed):
        g = torch.Generator().manual_seed(seed)
        perm = torch.randperm(num_blocks, generator=g).tolist()
        self.lens, self.status = ints(lens), ints([0])
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32)
        self.refs = torch.zeros(num_blocks, dtype=torch.int32)
        for b, n in enumerate(lens):
            for j in range(tc.blocks_of(n)):
                self.table[b, j] = perm.pop()
                self.refs[self.table[b, j]] += 1
        self.table, self.refs = self.table.to(DEV), self.refs.to(DEV)
        self.k = torch.randn((num_blocks, 1, 16, 16, 8), generator=g).to(torch.bfloat16).to(DEV)
        self.v = torch.randn((num_blocks, 1, 128, 16), generator=g).to(torch.bfloat16).to(DEV)
        n = bana.bana_kv_blocks_workspace_bytes(len(lens), width, num_blocks)
        self.ws = torch.full((n,), 0x7F, dtype=torch.uint8, device=DEV)

    def copy(self):
        return [x.cpu().clone() for x in (self.k, self.v, self.table, self.lens, self.refs, self.status)]


def fork(src, dst, k, v, table, lens, refs, status):
    """The forks of a call that is in order but for blocks without references among its sources'."""
    width, nb = table.shape[1], len(refs)
    length = [min(max(int(lens[s]), 0), width * tc.BS) for s in src]
    named = {int(table[s, j]) for s, n in zip(src, length) for j in range(tc.blocks_of(n))}
    bad = {x for x in named if not 0 <= x < nb or refs[x] <= 0}
    free = [x for x in range(nb) if refs[x] == 0 and x not in bad]
    if len(free) < sum(n % tc.BS != 0 for n in length):
        status[0] = max(int(status[0]), 1)
        return
    if bad:
        status[0] = 4
    for s, d, n in zip(src, dst, length):
        for j in range(n // tc.BS):
            table[d, j] = table[s, j]
            if int(table[s, j]) not in bad:
                refs[table[s, j]] += 1
        if n % tc.BS:
            blk, fresh = int(table[s, n // tc.BS]), free.pop(0)
            table[d, n // tc.BS] = fresh
            refs[fresh] = 1
            if 0 <= blk < nb:
                k[fresh], v[fresh] = k[blk], v[blk]
        lens[d] = n


def check_fork(p, src, dst, status):
    want = p.copy()
    fork(src, dst, *want)
    bana.bana_fork_kv_seqs(ints(src), ints(dst), p.k, p.v, p.table, p.lens, p.refs, p.status, p.ws)
    for x, y, name in zip(p.copy(), want, ("k", "v", "table", "lens", "refs", "status")):
        assert same(x, y), name
    assert int(p.status) == status


@pytest.mark.parametrize("count", [0, -3])
@pytest.mark.parametrize("entry", [0, 1, 2])
def test_fork_of_a_block_without_references(entry, count):
    """Raised as 4: its entry is copied, its count left alone, and the block, here the one of the lowest number, is no
    free one for this call."""
    p = Blocks([40, 37, 0, 0, 0], 12, 4, 1)
    other = int(p.table[0, entry])
    p.table[p.table == 0] = other
    p.table[0, entry] = 0  # the block's number, and another sequence's if that was it
    p.refs.zero_()
    p.refs[p.table[p.table >= 0].long()] = 1
    p.refs[0] = count
    check_fork(p, [0, 0, 1], [4, 2, 3], 4)


def test_fork_where_only_named_blocks_look_free():
    """Two blocks are free by their counts, and a source names one of them: too few, and nothing else changes."""
    p = Blocks([40, 37, 0, 0], 8, 4, 2)
    free = (p.refs == 0).nonzero().flatten().tolist()
    p.refs[free[1]], p.refs[p.table[1, 2].long()] = 1, 0
    before = p.copy()
    check_fork(p, [0, 1], [2, 3], 1)
    for x, y in zip(p.copy()[:-1], before[:-1]):
        assert same(x, y)


def test_many_forks_of_blocks_without_references():
    """More forks than threads of the plan, sources named many times, one long, blocks without references in some that
    share them."""
    n = 1300
    lens = [5000, 64, 7, 0, 33, 300] + [20] * 1200 + [0] * n
    p = Blocks(lens, 6000, 320, 3)
    for b, j in ((0, 0), (0, 250), (0, 312), (2, 0), (4, 1), (5, 18), (700, 0), (1205, 1)):
        p.refs[p.table[b, j].long()] = 0
    p.table[1, 2] = p.table[0, 250]  # by two sources
    p.table[800, 0] = p.table[700, 0]
    src = [0, 1, 2, 3, 4, 5] * 16 + list(range(6, 1206))
    src += [0] * (n - len(src))
    check_fork(p, src, [1206 + (7 * i) % n for i in range(n)], 4)


def test_fork_beside_unnamed_free_blocks_is_as_before():
    """Blocks in order: no status, the lowest free numbers."""
    p = Blocks([40, 37, 160, 0, 0, 0, 0], 30, 10, 4)
    check_fork(p, [0, 1, 0, 2], [3, 5, 4, 6], 0)


def test_reserve_leaves_entries_that_are_not_minus_one():
    """Only entries of -1 are taken for empty."""
    p = Blocks([16, 0, 0], 20, 6, 5)
    p.table[0, 2], p.table[1, 0], p.table[1, 3], p.table[2, 1] = -7, -2, 99, -2 ** 31
    want = p.copy()
    free = [x for x in range(20) if want[4][x] == 0]
    for b, j in ((0, 1), (0, 3), (1, 1), (1, 2), (1, 4), (2, 0)):
        want[2][b, j] = free.pop(0)
        want[4][want[2][b, j]] = 1
    bana.bana_reserve_kv_blocks(p.table, p.lens, ints([64, 80, 32]), p.refs, p.status, p.ws)
    for x, y in zip(p.copy(), want):
        assert same(x, y)


def test_race_check_build_on_unusual_inputs(monkeypatch):
    """Infinite values in steps that all rows see whole (fp32 lists walked once more), and forks of blocks without
    references, in the LDS race-check build: the same bits."""
    def results():
        found = []
        for news in (3, 60):
            cache = tc.Cache([700, 90], 2, 5)
            cache.values[0][300, 0, 17], cache.values[0][20, 1, 3] = math.inf, math.nan
            cache.store()
            rb, rows = tc.rows_of([news, news])
            found += run(cache, queries(rows, 8, 6), rb, False, window=([700, 90], 650, 2))
        p = Blocks([40, 37, 500, 0, 0, 0, 0], 60, 33, 1)
        p.refs[p.table[0, 1].long()] = p.refs[p.table[2, 31].long()] = 0
        bana.bana_fork_kv_seqs(ints([0, 2, 1, 2]), ints([4, 6, 5, 3]), p.k, p.v, p.table, p.lens, p.refs, p.status, p.ws)
        return found + p.copy()

    want = results()
    assert int(want[-1]) == 4
    monkeypatch.setattr(bana, "_native", bana._PythonChecks())
    monkeypatch.setattr(bana, "_lib", bana.load(bana.RACECHECK_LIB_PATH))
    for x, y in zip(results(), want):
        assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(torch.nan_to_num(x), torch.nan_to_num(y))


def test_captured_forks_replay():
    """Two graphs of forks, each with a workspace of its own, one of blocks without references: every replay leaves what
    the plain form leaves."""
    pools = [Blocks([40, 37, 64, 0, 0, 0], 20, 4, 6), Blocks([33, 16, 9, 0, 0, 0], 20, 4, 7)]
    pools[1].refs[pools[1].table[0, 0].long()] = pools[1].refs[pools[1].table[2, 0].long()] = 0
    names = ("k", "v", "table", "lens", "refs", "status")
    src, dst = [0, 2, 0], [5, 3, 4]
    before = [[getattr(p, n).clone() for n in names] for p in pools]
    want = [p.copy() for p in pools]
    for x in want:
        fork(src, dst, *x)
    s, d, graphs = ints(src), ints(dst), []
    for p in pools:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            bana.bana_fork_kv_seqs(s, d, p.k, p.v, p.table, p.lens, p.refs, p.status, p.ws)
    for _ in range(4):
        for p, old in zip(pools, before):
            for n, x in zip(names, old):
                getattr(p, n).copy_(x)
            p.ws.fill_(0x7F)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for p, ref in zip(pools, want):
            for x, y, n in zip(p.copy(), ref, names):
                assert same(x, y), n
    assert [int(p.status) for p in pools] == [0, 4]


# ---- rows spread unevenly over many sequences -------------------------------------------------------

def rounds_taken(row_begin, x, per_x, first):
    """Rounds of the search for the last sequence b with first(b, row_begin[b]) <= x, 0 where the look at 64 neighbours
    of its place among even sequences settles it."""
    B = len(row_begin) - 1
    starts = np.array([first(b, row_begin[b]) for b in range(B)])
    near = min(max(int(np.float32(x) * np.float32(per_x)) - 31, 0), max(B - 63, 0))
    ok = int((starts[near:near + 64] <= x).sum())
    if B > 1 and ok < 64 and (ok > 0 or near == 0):
        return 0
    rounds, n = 0, B
    while n > 1:
        rounds, n = rounds + 1, -(-n // 64)
    return rounds


def skewed(B, where):
    """Nearly all rows in one sequence; single rows before and behind it, most sequences without."""
    at = {"first": 0, "middle": B // 2 + 3, "last": B - 1}[where]
    news = [1 if b % 9 == 4 and abs(b - at) > 20 or abs(b - at) in (1, 3) else 0 for b in range(B)]
    if B > 1000:
        news = [n if b % 4 == 0 else 0 for b, n in enumerate(news)]
    news[at] = 3000
    return news


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("B,rounds", [(64, 1), (100, 2), (800, 2), (5000, 3)])
def test_append_finds_the_sequences_of_uneven_batches(B, rounds, where):
    news = skewed(B, where)
    rb, rows = tc.rows_of(news, pad=5, first=3)
    first = [(5 * b) % 23 for b in range(B)]
    lens = [f + n if n else 0 for f, n in zip(first, news)]
    cache = tc.Cache(lens, 1, 6)
    places = rows // 16 + 2 * B
    taken = {rounds_taken(rb, x, B / places, lambda b, row: row // 16 + 2 * b) for x in range(places)}
    assert taken == ({0} if B <= 100 and where == "middle" else {0, rounds})  # few sequences: 64 neighbours are most
    g = torch.Generator().manual_seed(7)
    kr, vr = (torch.randn((rows, 1, tc.D), generator=g).to(torch.bfloat16) for _ in range(2))
    k, v, table = cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV)
    tc.append(kr, vr, rb, first, cache.table, cache.k, cache.v)
    bana.bana_append_kv(kr.to(DEV), vr.to(DEV), ints(rb), ints(first), table, k, v)
    assert same(k, cache.k) and same(v, cache.v)


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("B,rounds", [(100, 2), (800, 2), (5000, 3)])
def test_attention_finds_the_sequences_of_uneven_batches(B, rounds, where):
    news = skewed(B, where)
    rb, rows = tc.rows_of(news, pad=5, first=3)
    lens = [n + b % 7 if n else 0 for b, n in enumerate(news)]
    cache = tc.Cache(lens, 1, 8)
    hq, width = 4 if B == 100 else 2, 8
    tile = 64 if rows * hq <= B * 64 else 128
    slots = rows * hq // tile + B
    taken = {rounds_taken(rb, x, B / slots, lambda b, row: row * hq // tile + b) for x in range(slots)}
    assert taken == ({0} if B <= 100 and where == "middle" else {0, rounds})  # few sequences: 64 neighbours are most
    q = queries(rows, hq, 9)
    want = tc.attention(q, rb, cache, tc.window_sees(lens, news, width, 1), 0.0884)
    out, lse = run(cache, q, rb, False, window=(lens, width, 1))
    live = slice(rb[0], rb[-1])
    tc.check_attention(out[live], lse[live], (want[0][live], want[1][live], tuple(x[live] for x in want[2])), False)
    for part in (slice(0, rb[0]), slice(rb[-1], None)):
        assert bool((out[part] == 7.0).all()) and bool((lse[part] == 7.0).all())
