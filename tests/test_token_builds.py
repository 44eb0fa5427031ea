"""The calls of include/bana_tokens.h in other builds and through the other checks of the Python binding: the same bits.

The LDS race-check build lets odd wavefronts sleep before they write to LDS, or read what other wavefronts overwrite
later, and adds barriers before read-backs: a missing wait or barrier would change results.
"""
import random

import pytest
import torch

import token_cases as tc
from paper_2510_13223_amd import bana

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def same(x, y):
    """Equal bit for bit."""
    if x.is_floating_point():
        kind = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
        x, y = x.view(kind), y.view(kind)
    return torch.equal(x, y)


def attention_results(hq, hkv, lens, news, bf16, poison):
    """Both attention calls over one cache, its lists cut into chunks."""
    rng = random.Random(5)
    cache = tc.Cache(lens, hkv, 3)
    if poison:
        cache.values[0][lens[0] - 2, 0, 9] = float("inf")
        cache.store()
    rb, rows = tc.rows_of(news)
    g = torch.Generator().manual_seed(4)
    q = torch.randn((rows, hq, tc.D), generator=g).to(torch.bfloat16).to(DEV)
    k, v, table = cache.k.to(DEV), cache.v.to(DEV), cache.table.to(DEV)
    dims = bana.make_dims(len(lens), hq, hkv, cache.table.shape[1], cache.num_blocks, max_range_tokens=max(lens),
                          total_range_tokens=sum(lens))
    ws = torch.empty(max(bana.bana_tree_attn_workspace_bytes(dims, rows, 1),
                         bana.bana_window_attn_workspace_bytes(dims, rows, 900, 4)), dtype=torch.uint8, device=DEV)
    outs = [(torch.empty((rows, hq, tc.D), device=DEV, dtype=torch.bfloat16 if bf16 else torch.float32),
             torch.empty((rows, hq), device=DEV)) for _ in range(2)]
    before = [n - m for n, m in zip(lens, news)]
    masks = tc.signed([m for n in news for m in tc.random_tree(n, rng)]).to(DEV)
    bana.bana_tree_attn(q, ints(rb), k, v, table, ints([[0] * len(lens)]), ints([before]), ints(before), masks,
                        *outs[0], scale=0.0884, workspace=ws, dims=dims)
    bana.bana_window_attn(q, ints(rb), k, v, table, ints(lens), 900, 4, *outs[1], scale=0.0884, workspace=ws, dims=dims)
    return [x for o in outs for x in o]


def block_results():
    """Blocks reserved, tokens appended, sequences forked, long and short lists compacted, blocks given back."""
    hkv, B, width, blocks = 4, 5, 80, 400
    g = torch.Generator().manual_seed(6)
    k = torch.zeros((blocks, hkv, 16, 16, 8), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros((blocks, hkv, 128, 16), dtype=torch.bfloat16, device=DEV)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    refs, status = torch.zeros(blocks, dtype=torch.int32, device=DEV), ints([0])
    ws = torch.empty(bana.bana_kv_blocks_workspace_bytes(B, width, blocks), dtype=torch.uint8, device=DEV)
    lens, news = ints([0] * B), [1200, 37, 800, 0, 0]
    rb, rows = tc.rows_of(news)
    kr, vr = (torch.randn((rows, hkv, tc.D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    bana.bana_reserve_kv_blocks(table, lens, ints(news), refs, status, ws)
    bana.bana_append_kv(kr, vr, ints(rb), lens, table, k, v)
    lens = ints(news)
    bana.bana_fork_kv_seqs(ints([1, 1]), ints([4, 3]), k, v, table, lens, refs, status, ws)
    rng = random.Random(8)
    for size in (600, 20):
        kept = torch.tensor([sorted(rng.sample(range(1200), size)) for _ in range(B)], dtype=torch.int32, device=DEV)
        bana.bana_compact_kv_tokens(k, v, table, ints([0] * B), kept, ints([size, 0, size // 2, 0, 0]))
    bana.bana_release_kv_blocks(table, ints([600, 37, 400, 10, 0]), refs, status)
    return [k, v, table, refs, status, lens]


RUNS = [
    lambda: attention_results(8, 2, [700, 90], [12, 5], True, False),     # tiles of 64 columns
    lambda: attention_results(8, 2, [700, 90], [12, 5], False, True),
    lambda: attention_results(8, 2, [1500, 300], [60, 60], True, True),   # of 128
    lambda: attention_results(8, 2, [1500, 300], [60, 60], False, False),
    block_results,
]


@pytest.mark.parametrize("run", RUNS)
def test_lds_race_check_build_bit_identical(run, monkeypatch):
    want = run()
    monkeypatch.setattr(bana, "_native", bana._PythonChecks())
    monkeypatch.setattr(bana, "_lib", bana.load(bana.RACECHECK_LIB_PATH))
    for _ in range(2):
        for a, b in zip(run(), want):
            assert same(a, b)


@pytest.mark.parametrize("run", RUNS)
def test_the_python_checks_make_the_same_calls(run, monkeypatch):
    want = run()
    assert not isinstance(bana._calls(), bana._PythonChecks)
    monkeypatch.setattr(bana, "_native", bana._PythonChecks())
    for a, b in zip(run(), want):
        assert same(a, b)
