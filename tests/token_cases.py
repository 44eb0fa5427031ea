"""Plain 64-bit forms of the calls on new tokens and blocks, and the inputs their tests share."""

import math

import torch

D, BS = 128, 16


def rows_of(news, pad=0, first=0):
    """row_begin (list) for sequences of `news` rows, and the number of rows with `first` before and `pad` behind."""
    rb = [first]
    for n in news:
        rb.append(rb[-1] + n)
    return rb, rb[-1] + pad


class Cache:
    """A paged cache on the CPU with random tokens; blocks and slots that hold none are NaN."""

    def __init__(self, lens, hkv, seed, width=None, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.hkv = list(lens), hkv
        nbs = [-(-n // BS) for n in lens]
        self.num_blocks = max(1, sum(nbs) + spare)
        perm = torch.randperm(self.num_blocks, generator=g).tolist()
        self.table = torch.full((len(lens), width or max(1, max(nbs))), -1, dtype=torch.int32)
        for b, nb in enumerate(nbs):
            for j in range(nb):
                self.table[b, j] = perm.pop()
        self.keys = [torch.randn((n, hkv, D), generator=g).to(torch.bfloat16) for n in lens]
        self.values = [torch.randn((n, hkv, D), generator=g).to(torch.bfloat16) for n in lens]
        self.k = torch.full((self.num_blocks, hkv, D // 8, BS, 8), math.nan, dtype=torch.bfloat16)
        self.v = torch.full((self.num_blocks, hkv, D, BS), math.nan, dtype=torch.bfloat16)
        self.store()

    def store(self):
        for b, n in enumerate(self.lens):
            for t in range(n):
                put(self.k, self.v, int(self.table[b, t // BS]), t % BS, self.keys[b][t], self.values[b][t])


def put(k, v, block, slot, key, value):
    """One token's key and value [Hkv, D] into its slot."""
    k[block, :, :, slot, :] = key.view(-1, D // 8, 8)
    v[block, :, :, slot] = value


def get(k, v, block, slot):
    return k[block, :, :, slot, :].reshape(-1, D), v[block, :, :, slot]


def attention(q, row_begin, cache, sees, scale):
    """(out, lse, bounds) in 64 bits: `sees(b, i)` lists the tokens of row i of sequence b (one twice counts twice).

    bounds: (score, spread, n) per (row, head): spread = sum of weight |value|, n tokens, score the bound of a
    weight's relative error from the scores: products are exact in fp32, 128 of them are summed and scaled, and
    2^x is off by 1 unit at most; each step counts 2^-23 of the sum of absolute products (two roundings)."""
    rows, hq, _ = q.shape
    group = hq // cache.hkv
    out = torch.zeros((rows, hq, D), dtype=torch.float64)
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64)
    spread = torch.zeros((rows, hq, D), dtype=torch.float64)
    score = torch.zeros((rows, hq), dtype=torch.float64)
    count = torch.zeros((rows, hq), dtype=torch.float64)
    for b in range(len(row_begin) - 1):
        for i in range(row_begin[b + 1] - row_begin[b]):
            r, tokens = row_begin[b] + i, torch.tensor(sees(b, i), dtype=torch.long)
            if len(tokens) == 0:
                continue
            for h in range(hq):
                key = cache.keys[b][tokens, h // group].double()
                value = cache.values[b][tokens, h // group].double()
                x = key @ q[r, h].double() * scale
                lse[r, h] = torch.logsumexp(x, 0)
                w = torch.exp(x - lse[r, h])
                out[r, h] = (w[:, None] * value).sum(0)
                spread[r, h] = (w[:, None] * value.abs()).sum(0)
                most = (key.abs() @ q[r, h].double().abs()).max() * scale
                score[r, h] = 2.0 ** -23 * (128 * most + 3 * x.abs().max() + 2)
                count[r, h] = len(tokens)
    return out, lse, (score, spread, count)


def check_attention(out, lse, want, bf16):
    """Against the 64-bit result: weights and their sum are off by `score` each, n + 8 additions by 2^-24 of the
    sum of absolute terms each (counted twice: numerator and denominator), the weights' 24 bits by 2^-24; a bf16
    result rounds the weights and itself by half a step, 2^-8."""
    ref, ref_lse, (score, spread, count) = want
    near = 2 * score + 2 * (count + 10) * 2.0 ** -24
    bound = spread * near[:, :, None]
    if bf16:
        bound = bound + 2.0 ** -8 * (spread + ref.abs() + bound)
    off = (out.double() - ref).abs()
    assert bool((off <= bound + 1e-30).all()), f"out off by {(off - bound).max():.3g} over its bound"
    if lse is not None:
        alive = torch.isfinite(ref_lse)
        assert torch.equal(lse == -math.inf, ~alive)
        bound = score + (count + 10) * 2.0 ** -24 + 2.0 ** -21 * (ref_lse.abs() + 1)
        off = (lse.double() - ref_lse).abs()[alive]
        assert bool((off <= bound[alive]).all()), f"lse off by {(off - bound[alive]).max():.3g} over its bound"


def window_sees(seq_lens, news, window, sinks, begin=None, end=None):
    def sees(b, i):
        pos = seq_lens[b] - news[b] + i
        lo, hi = (0, 1 << 60) if begin is None else (begin[b], end[b])
        return [t for t in range(max(pos + 1, 0)) if (pos - t < window or t < sinks) and lo <= t < hi]
    return sees


def tree_sees(begin, end, tree_begin, masks, row_begin):
    def sees(b, i):
        n = row_begin[b + 1] - row_begin[b]
        tokens = [t for p in range(len(begin)) for t in range(begin[p][b], end[p][b])]
        if tree_begin[b] >= 0:
            tokens += [tree_begin[b] + j for j in range(min(n, 64)) if masks[row_begin[b] + i] >> j & 1]
        return tokens
    return sees


def random_tree(n, rng):
    """Masks of a random tree of n nodes (at most 64 of them can be seen)."""
    seen = []
    for i in range(n):
        parent = rng.randint(-1, i - 1)
        seen.append((seen[parent] if parent >= 0 else 0) | (1 << i if i < 64 else 0))
    return seen


def signed(masks):
    """uint64 masks as the int64 tensor that carries their bits."""
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64)


# ---- blocks -----------------------------------------------------------------------------------------

def blocks_of(tokens):
    return 0 if tokens <= 0 else -(-tokens // BS)


def release(table, keep, refs, status):
    B, width = table.shape
    for b in range(B):
        for j in range(blocks_of(int(keep[b])), width):
            blk = int(table[b, j])
            if blk == -1:
                continue
            table[b, j] = -1
            if not 0 <= blk < len(refs) or refs[blk] <= 0:
                status[0] = max(int(status[0]), 4)
            else:
                refs[blk] -= 1


def reserve(table, lens, need, refs, status):
    B, width = table.shape
    if any(blocks_of(int(x)) > width for x in need):
        status[0] = max(int(status[0]), 3)
        return
    places = [(b, j) for b in range(B) for j in range(blocks_of(int(lens[b])), blocks_of(int(need[b])))
              if table[b, j] < 0]
    free = [i for i in range(len(refs)) if refs[i] == 0]
    if len(free) < len(places):
        status[0] = max(int(status[0]), 1)
        return
    for (b, j), blk in zip(places, free):
        table[b, j] = blk
        refs[blk] = 1


def fork(src, dst, k, v, table, lens, refs, status):
    B, width = table.shape
    src, dst = [int(x) for x in src], [int(x) for x in dst]
    if any(not 0 <= x < B for x in src + dst) or len(set(dst)) < len(dst) or set(dst) & set(src) or \
            any(table[d, 0] != -1 for d in dst):
        status[0] = max(int(status[0]), 2)
        return
    length = [min(max(int(lens[s]), 0), width * BS) for s in src]
    free = [i for i in range(len(refs)) if refs[i] == 0]
    if len(free) < sum(n % BS != 0 for n in length):
        status[0] = max(int(status[0]), 1)
        return
    for s, d, n in zip(src, dst, length):
        for j in range(n // BS):
            blk = int(table[s, j])
            table[d, j] = blk
            if 0 <= blk < len(refs):
                refs[blk] += 1
            else:
                status[0] = max(int(status[0]), 4)
        if n % BS:
            fresh = free.pop(0)
            blk = int(table[s, n // BS])
            table[d, n // BS] = fresh
            refs[fresh] = 1
            if 0 <= blk < len(refs):
                k[fresh], v[fresh] = k[blk], v[blk]
            else:
                status[0] = max(int(status[0]), 4)
        lens[d] = n


def compact(k, v, table, first, kept, n_kept):
    width, nb = table.shape[1], k.shape[0]

    def at(b, t):
        blk = int(table[b, t // BS]) if 0 <= t < width * BS else -1
        return (blk, t % BS) if 0 <= blk < nb else None

    for b in range(table.shape[0]):
        for i in range(min(max(int(n_kept[b]), 0), kept.shape[1])):
            of, to = at(b, int(first[b]) + int(kept[b, i])), at(b, int(first[b]) + i)
            if of is not None and to is not None and of != to:
                put(k, v, *to, *(x.clone() for x in get(k, v, *of)))


def append(k_rows, v_rows, row_begin, first, table, k, v):
    for b in range(table.shape[0]):
        for i in range(row_begin[b + 1] - row_begin[b]):
            t, r = int(first[b]) + i, row_begin[b] + i
            blk = int(table[b, t // BS]) if 0 <= t < table.shape[1] * BS else -1
            if 0 <= blk < k.shape[0]:
                put(k, v, blk, t % BS, k_rows[r], v_rows[r])
