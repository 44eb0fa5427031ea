"""Calls on new tokens and blocks where the cache is unusual: scores and values that are not finite, counts and
entries that do not fit together."""

import math

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
