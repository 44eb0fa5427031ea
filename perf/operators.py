"""Cases of the operators on new tokens and on the blocks of the paged K/V cache, and their plain forms.

What a serving program does with the cache besides attending to it from one token per sequence:

* ``tree``     attention of drafted tokens (a tree per sequence) over the cache, ``bana_tree_attn``;
* ``window``   attention of new tokens (prompts, pieces of prompts, single tokens) under a sliding window whose
               first tokens stay visible, ``bana_window_attn``;
* ``append``   the new tokens' keys and values into the cache's tiles, ``bana_append_kv``;
* ``draft``    the blocks of one draft step: what the last step left over goes back, what this one needs is
               taken, ``bana_release_kv_blocks`` and ``bana_reserve_kv_blocks``;
* ``fork``     the children of the last step end, new ones share their parents' blocks, ``bana_release_kv_blocks``
               and ``bana_fork_kv_seqs``;
* ``compact``  the kept tokens of each sequence move together, ``bana_compact_kv_tokens``.

The new tokens of a batch are packed: the rows of sequence b are [row_begin[b], row_begin[b + 1]).  Lengths, numbers of
new tokens and the shapes of the trees come from the case (``lens_seed``), so its work is known without its inputs;
values, the placement of blocks and the kept tokens come from the seed of ``prepare``.  Blocks and slots that hold no
token are NaN where only attention reads the cache.
"""

import math
import random

import numpy as np
import torch

own = False

D, BS = 128, 16
TOKEN_BYTES = 2 * D * 2  # key and value of one token and kv head

# Query / kv heads: GQA groups of 4, 8, 1, 7 and 16, as current decoder layers have them.
HEADS = [(8, 2), (32, 8), (64, 8), (40, 40), (28, 4), (32, 2)]


def _case(name, op, batch, hq, hkv, length, new, **more):
    """``length``: tokens of a sequence before the new ones, ``lens`` fixed / uniform / lognormal around it; ``new``: new
    tokens of a sequence, ``news`` fixed or ragged (from none to ``new``); ``pad``: rows behind the last sequence."""
    c = {"op": op, "batch": batch, "hq": hq, "hkv": hkv, "length": length, "new": new, "lens": "uniform",
         "news": "fixed", "pad": 0, "lens_seed": 0}
    c.update(more)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One user, a short draft: latency only.
        _case("tree_one", "tree", 1, 32, 8, 700, 8, parts=1, bf16=True),
        # A chat server's drafts, ragged, the caches partly migrated; fp32 for a merge with another device's part.
        _case("tree_chat", "tree", 24, 32, 8, 2000, 26, lens="lognormal", news="ragged", pad=5, parts=2, bf16=False),
        # Whole trees of 64 nodes over long contexts, groups of 8.
        _case("tree_wide", "tree", 32, 64, 8, 8000, 64, parts=2, bf16=True),
        # Single tokens of long sequences under a window: what every decode step of such a layer costs.
        _case("window_token", "window", 64, 32, 8, 20000, 1, window=4096, sinks=4, bf16=True),
        # New prompts of ragged lengths, a short window.
        _case("window_prompts", "window", 6, 28, 4, 1, 1500, lens="fixed", news="ragged", pad=11, window=512, sinks=4,
              bf16=True),
        # Pieces of long prompts over what is in the cache already.
        _case("window_chunk", "window", 2, 32, 8, 12000, 4096, window=4096, sinks=64, bf16=True),
        # The keys and values of one token per sequence, and of prompts.
        _case("append_token", "append", 48, 32, 8, 1000, 1),
        _case("append_prompt", "append", 8, 32, 8, 300, 2048, news="ragged", pad=7),
        # The blocks of a draft step in a large pool; new children of beams or samples.
        _case("draft_blocks", "draft", 128, 32, 8, 2000, 64, spare=100000),
        _case("fork_children", "fork", 32, 32, 8, 1500, 0, children=3, spare=2000),
        # The accepted path of each tree; a cache that drops half of its tokens.
        _case("compact_accepted", "compact", 48, 32, 8, 1000, 48, keep=0.15, lens="lognormal"),
        _case("compact_evicted", "compact", 6, 32, 8, 0, 9000, keep=0.5, lens="fixed"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "window", "window", "window", "append", "draft", "fork", "compact"])
    hq, hkv = rng.choice(HEADS)
    more = {"lens": rng.choice(["fixed", "uniform", "lognormal"]), "news": rng.choice(["fixed", "ragged"]),
            "lens_seed": rng.randrange(1 << 30)}
    batch, length, new = _log(rng, 1, 64), _log(rng, 1, 16000), 1
    if op == "tree":
        new = _log(rng, 1, 64)
        more.update(parts=rng.choice([1, 2, 3]), bf16=rng.random() < 0.6, pad=rng.choice([0, 3]))
    elif op == "window":
        new = rng.choice([1, _log(rng, 2, 4096)])
        more.update(window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 17, 64]), bf16=rng.random() < 0.6,
                    pad=rng.choice([0, 9]))
        batch = max(1, min(batch, 8192 // new))
    elif op == "append":
        new = _log(rng, 1, 4096)
        more.update(pad=rng.choice([0, 5]))
        batch = max(1, min(batch, 16384 // new))
    elif op == "draft":
        new = _log(rng, 1, 256)
        more.update(spare=_log(rng, 2000, 200000))
    elif op == "fork":
        new = 0
        more.update(children=rng.choice([1, 2, 4, 7]), spare=_log(rng, 600, 4000))
    elif rng.random() < 0.5:  # compact: drafts
        new = _log(rng, 1, 64)
        more.update(keep=rng.uniform(0.05, 0.5))
    else:  # compact: whole sequences
        length, new = 0, _log(rng, 64, 16000)
        more.update(keep=rng.uniform(0.1, 0.95))
    # At most about 1 GiB of keys and values in a case; the rows times the tokens they see stay below tree_wide's
    # and window_chunk's.
    length = min(length, max(1, (1 << 30) // (hkv * 2 * TOKEN_BYTES)))
    batch = max(1, min(batch, (1 << 30) // (hkv * 2 * TOKEN_BYTES * (length + new))))
    if op in ("tree", "window"):
        seen = length + new if op == "tree" else min(length + new, more["window"] + new)
        batch = max(1, min(batch, int(6e9 / (hq * new * seen * 2))))
    return _case(None, op, batch, hq, hkv, length, new, **more)


# ---- lengths, ranges and trees (host only) ---------------------------------------------------------

def _lens(case):
    r = np.random.default_rng([case["lens_seed"], case["batch"], case["length"]])
    n, mid = case["batch"], case["length"]
    if case["lens"] == "fixed" or mid < 2:
        return np.full(n, mid, dtype=np.int64)
    if case["lens"] == "uniform":
        return r.integers(max(1, int(0.4 * mid)), int(1.6 * mid), size=n, endpoint=True)
    return np.clip(np.rint(mid * np.exp(r.standard_normal(n))), 1, 4 * mid).astype(np.int64)


def _news(case):
    n, new = case["batch"], case["new"]
    if case["news"] == "fixed" or n == 1:
        return np.full(n, new, dtype=np.int64)
    r = np.random.default_rng([case["lens_seed"], n, new, 1])
    return r.integers(0, new, size=n, endpoint=True)


def _row_begin(news):
    return np.concatenate([[0], np.cumsum(news)])


def _masks(case, news):
    """uint64 [rows]: the nodes that each drafted token sees, itself among them; a node's parent is one of the eight
    before it or the sequence itself."""
    r = random.Random(case["lens_seed"] * 31 + case["new"])
    out = []
    for n in news:
        seen = []
        for i in range(int(n)):
            parent = r.randint(max(-1, i - 8), i - 1)
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
        out += seen
    return np.array(out, dtype=np.uint64)


def _parts(case, lens):
    """(begin, end) [parts, B]: the context's ranges, cut at whole blocks."""
    r = random.Random(case["lens_seed"] * 7919 + case["batch"])
    edges = np.zeros((case["parts"] + 1, len(lens)), dtype=np.int64)
    for b, n in enumerate(int(x) for x in lens):
        edges[1:-1, b] = sorted(min(n, BS * r.randint(0, n // BS)) for _ in range(case["parts"] - 1))
        edges[-1, b] = n
    return edges[:-1].copy(), edges[1:].copy()


def _kept_counts(case, news):
    return np.maximum(0, np.rint(news * case["keep"])).astype(np.int64)


# ---- inputs ---------------------------------------------------------------------------------------

def _ints(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


def _table(tokens, blocks, g, dev, width=None):
    """int32 [B, width]: random blocks for `tokens` of each sequence, -1 behind them."""
    nbs = -(-tokens // BS)
    table = torch.full((len(tokens), int(width or max(1, nbs.max()))), -1, dtype=torch.int32, device=dev)
    live = torch.from_numpy(np.arange(table.shape[1])[None, :] < nbs[:, None]).to(dev)
    table[live] = torch.randperm(blocks, generator=g, device=dev).to(torch.int32)[:int(nbs.sum())]
    return table


def _pools(blocks, hkv, g, dev):
    return (torch.randn((blocks, hkv, D // 8, BS, 8), generator=g, device=dev, dtype=torch.bfloat16),
            torch.randn((blocks, hkv, D, BS), generator=g, device=dev, dtype=torch.bfloat16))


def _poison(k, v, table, tokens, dev):
    """NaN in the blocks and slots that hold no token."""
    blocks = k.shape[0]
    used = torch.zeros(blocks, BS, dtype=torch.bool, device=dev)
    where = torch.arange(table.shape[1] * BS, device=dev)
    live = where[None, :] < torch.from_numpy(tokens).to(dev)[:, None]
    slots = table.long().clamp(min=0).repeat_interleave(BS, dim=1) * BS + where[None, :] % BS
    used.view(-1)[slots[live]] = True
    k.masked_fill_(~used[:, None, None, :, None], math.nan)
    v.masked_fill_(~used[:, None, None, :], math.nan)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed * 1000003 + 17)
    op, B, hq, hkv = case["op"], case["batch"], case["hq"], case["hkv"]
    lens, news = _lens(case), _news(case)
    total = lens + news
    used = int((-(-total // BS)).sum())
    s = {"case": case, "lens": lens, "news": news, "hkv": hkv}
    if op in ("tree", "window", "append"):
        rows = int(news.sum()) + case["pad"]
        blocks = max(1, math.ceil(1.1 * used))
        s["live"] = int(news.sum())
        s["table"] = _table(total, blocks, g, dev)
        s["k"], s["v"] = _pools(blocks, hkv, g, dev)
        s["row_begin"] = _ints(_row_begin(news), dev)
        if op == "append":
            s["first"] = _ints(lens, dev)
            s["k_rows"] = torch.randn((max(rows, 1), hkv, D), generator=g, device=dev, dtype=torch.bfloat16)
            s["v_rows"] = torch.randn((max(rows, 1), hkv, D), generator=g, device=dev, dtype=torch.bfloat16)
            return s
        _poison(s["k"], s["v"], s["table"], total, dev)
        s["q"] = 2 * torch.randn((max(rows, 1), hq, D), generator=g, device=dev, dtype=torch.bfloat16)
        s["out"] = torch.full(s["q"].shape, 7.0, dtype=torch.bfloat16 if case["bf16"] else torch.float32, device=dev)
        s["lse"] = torch.full(s["q"].shape[:2], 7.0, dtype=torch.float32, device=dev)
        if op == "tree":
            begin, end = _parts(case, lens)
            s["begin"], s["end"], s["tree_begin"] = _ints(begin, dev), _ints(end, dev), _ints(lens, dev)
            mask = np.concatenate([_masks(case, news), np.zeros(case["pad"], dtype=np.uint64)])
            mask = mask if len(mask) else np.zeros(1, dtype=np.uint64)
            s["mask"] = torch.from_numpy(mask.view(np.int64)).to(dev)
        else:
            s["seq_lens"] = _ints(total, dev)
        return s
    if op == "draft":
        blocks = used + case["spare"]
        s["table"] = _table(lens, blocks, g, dev, width=max(1, int((-(-total // BS)).max())))
        s["seq_lens"], s["need"] = _ints(lens, dev), _ints(total, dev)
    elif op == "fork":
        n = B * case["children"]
        blocks = used + n + case["spare"]
        s["table"] = torch.full((B + n, max(1, int((-(-lens // BS)).max()))), -1, dtype=torch.int32, device=dev)
        s["table"][:B] = _table(lens, blocks, g, dev)
        s["seq_lens"] = torch.cat([_ints(lens, dev), torch.zeros(n, dtype=torch.int32, device=dev)])
        s["src"] = torch.randint(B, (n,), generator=g, device=dev, dtype=torch.int32)
        s["dst"] = (B + torch.randperm(n, generator=g, device=dev)).to(torch.int32)
        s["keep"] = torch.cat([_ints(lens, dev), torch.zeros(n, dtype=torch.int32, device=dev)])
        s["k"], s["v"] = _pools(blocks, hkv, g, dev)
    else:
        s["table"] = _table(total, max(1, math.ceil(1.1 * used)), g, dev)
        s["k"], s["v"] = _pools(max(1, math.ceil(1.1 * used)), hkv, g, dev)
        counts = _kept_counts(case, news)
        most = max(1, int(counts.max()))
        # Random tokens of each sequence, in order; places behind the count hold the row's last possible value.
        score = torch.rand((B, case["new"]), generator=g, device=dev)
        score[torch.arange(case["new"], device=dev)[None, :] >= torch.from_numpy(news).to(dev)[:, None]] = 2.0
        rank = score.argsort(dim=1)[:, :most]
        rank[torch.arange(most, device=dev)[None, :] >= torch.from_numpy(counts).to(dev)[:, None]] = case["new"]
        s["kept"] = rank.sort(dim=1).values.to(torch.int32).contiguous()
        s["n_kept"], s["first"] = _ints(counts, dev), _ints(lens, dev)
        return s
    s["refs"] = torch.zeros(blocks, dtype=torch.int32, device=dev)
    s["refs"][s["table"][s["table"] >= 0].long()] = 1
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    return s


# ---- the framework's calls ------------------------------------------------------------------------

def _workspace(s, need):
    if "workspace" not in s:
        n = need()
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s["workspace"]


def _run_own(s):
    from paper_2510_13223_amd import bana

    case, op = s["case"], s["case"]["op"]
    if op == "append":
        bana.bana_append_kv(s["k_rows"], s["v_rows"], s["row_begin"], s["first"], s["table"], s["k"], s["v"])
        return [s["k"], s["v"]]
    if op == "compact":
        bana.bana_compact_kv_tokens(s["k"], s["v"], s["table"], s["first"], s["kept"], s["n_kept"])
        return [s["k"], s["v"]]
    if op in ("tree", "window"):
        if "dims" not in s:  # the lengths that a serving program knows on the host
            live = s["lens"] + s["news"]
            s["dims"] = bana.make_dims(case["batch"], case["hq"], case["hkv"], s["table"].shape[1], s["k"].shape[0],
                                       max_range_tokens=int(live.max()), total_range_tokens=int(live.sum()))
        rows, scale = s["q"].shape[0], D ** -0.5
        if op == "tree":
            ws = _workspace(s, lambda: bana.bana_tree_attn_workspace_bytes(s["dims"], rows, case["parts"]))
            bana.bana_tree_attn(s["q"], s["row_begin"], s["k"], s["v"], s["table"], s["begin"], s["end"],
                                s["tree_begin"], s["mask"], s["out"], s["lse"], scale=scale, workspace=ws,
                                dims=s["dims"])
        else:
            ws = _workspace(s, lambda: bana.bana_window_attn_workspace_bytes(s["dims"], rows, case["window"],
                                                                             case["sinks"]))
            bana.bana_window_attn(s["q"], s["row_begin"], s["k"], s["v"], s["table"], s["seq_lens"], case["window"],
                                  case["sinks"], s["out"], s["lse"], scale=scale, workspace=ws, dims=s["dims"])
        return [s["out"], s["lse"]]
    B, width = s["table"].shape
    blocks = s["refs"].shape[0]
    if op == "draft":
        ws = _workspace(s, lambda: bana.bana_kv_blocks_workspace_bytes(B, width, blocks))
        bana.bana_release_kv_blocks(s["table"], s["seq_lens"], s["refs"], s["status"])
        bana.bana_reserve_kv_blocks(s["table"], s["seq_lens"], s["need"], s["refs"], s["status"], ws)
        return [s["table"], s["refs"], s["status"]]
    ws = _workspace(s, lambda: bana.bana_kv_blocks_workspace_bytes(B, width, blocks))
    bana.bana_release_kv_blocks(s["table"], s["keep"], s["refs"], s["status"])
    bana.bana_fork_kv_seqs(s["src"], s["dst"], s["k"], s["v"], s["table"], s["seq_lens"], s["refs"], s["status"], ws)
    return [s["table"], s["seq_lens"], s["refs"], s["status"], s["k"], s["v"]]


# ---- the plain forms ------------------------------------------------------------------------------

def _attend(s, pos, visible, scale):
    """Rows of each sequence over the tokens pos [B, S] where visible [B, T, S] says so, in 32 bits."""
    q, k, v, table, rb = s["q"], s["k"], s["v"], s["table"].long(), s["row_begin"].long()
    B, T, S = visible.shape
    hkv, G = s["hkv"], q.shape[1] // s["hkv"]
    i = torch.arange(T, device=q.device)
    row = rb[:-1, None] + i[None, :]
    live = row < rb[1:, None]
    used = visible.any(dim=1)
    block = torch.gather(table, 1, (pos // BS).clamp(0, table.shape[1] - 1)).clamp(min=0)
    block, slot = torch.where(used, block, 0), pos % BS
    keys = k[block, :, :, slot, :].reshape(B, S, hkv, D).float()
    values = torch.where(used[:, :, None, None], v[block, :, :, slot].float(), 0.0)
    queries = q[row.clamp(max=q.shape[0] - 1)].float().reshape(B, T, hkv, G, D)
    queries = queries.permute(0, 2, 1, 3, 4).reshape(B * hkv, T * G, D)
    scores = torch.bmm(queries, keys.permute(0, 2, 3, 1).reshape(B * hkv, D, S).contiguous()) * scale
    scores = scores.view(B, hkv, T, G, S).masked_fill_(~visible[:, None, :, None, :], -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(dim=-1, keepdim=True)
    out = torch.bmm(scores.view(B * hkv, T * G, S), values.permute(0, 2, 1, 3).reshape(B * hkv, S, D).contiguous())
    out = out.view(B, hkv, T, G, D) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).squeeze(-1)
    s["out"][row[live]] = out.permute(0, 2, 1, 3, 4).reshape(B, T, hkv * G, D)[live].to(s["out"].dtype)
    s["lse"][row[live]] = lse.permute(0, 2, 1, 3).reshape(B, T, hkv * G)[live]
    return [s["out"], s["lse"]]


def _plain_tree(s):
    T, S = max(1, int(s["news"].max())), int((s["lens"] + s["news"]).max())
    pos = torch.arange(S, device="cuda").expand(len(s["lens"]), S)
    rb = s["row_begin"].long()
    n = (rb[1:] - rb[:-1])[:, None]
    context = ((pos >= s["begin"][:, :, None]) & (pos < s["end"][:, :, None])).any(dim=0)
    node = pos - s["tree_begin"].long()[:, None]
    row = rb[:-1, None] + torch.arange(T, device="cuda")
    mask = s["mask"][row.clamp(max=s["mask"].shape[0] - 1)]
    node_seen = (mask[:, :, None] >> node.clamp(0, 63)[:, None, :] & 1).bool()
    visible = context[:, None, :] | (node_seen & ((node >= 0) & (node < n))[:, None, :])
    return _attend(s, pos, visible & (row < rb[1:, None])[:, :, None], D ** -0.5)


def _plain_window(s):
    window, sinks = s["case"]["window"], s["case"]["sinks"]
    T, longest = max(1, int(s["news"].max())), int((s["lens"] + s["news"]).max())
    rb, total = s["row_begin"].long(), s["seq_lens"].long()
    at = (total - (rb[1:] - rb[:-1]))[:, None] + torch.arange(T, device="cuda")  # position of each row
    near = min(window + T - 1, longest)
    first = (at[:, :1] - window + 1).clamp(min=sinks)
    pos = torch.cat([torch.arange(sinks, device="cuda").expand(len(total), sinks),
                     first + torch.arange(near, device="cuda")], dim=1)
    back = at[:, :, None] - pos[:, None, :]
    visible = (back >= 0) & ((back < window) | (pos < sinks)[:, None, :]) & (at < total[:, None])[:, :, None]
    return _attend(s, pos, visible, D ** -0.5)


def _plain_append(s):
    rb, n = s["row_begin"].long(), s["live"]
    row = torch.arange(n, device="cuda")
    seq = torch.searchsorted(rb, row, right=True) - 1
    token = s["first"].long()[seq] + row - rb[seq]
    block = s["table"].long()[seq, token // BS]
    s["k"][block, :, :, token % BS, :] = s["k_rows"][:n].view(n, s["hkv"], D // 8, 8)
    s["v"][block, :, :, token % BS] = s["v_rows"][:n]
    return [s["k"], s["v"]]


def _plain_release(table, keep, refs):
    j = torch.arange(table.shape[1], device="cuda")
    drop = (j[None, :] >= ((keep.long() + BS - 1) // BS)[:, None]) & (table >= 0)
    gone = table[drop].long()
    refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    table.masked_fill_(drop, -1)


def _plain_draft(s):
    table, refs = s["table"], s["refs"]
    _plain_release(table, s["seq_lens"], refs)
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    new = (j >= ((s["seq_lens"].long() + BS - 1) // BS)[:, None]) & (j < ((s["need"].long() + BS - 1) // BS)[:, None])
    free = (refs == 0).nonzero().flatten()[:int((new & (table < 0)).sum())]
    table[new & (table < 0)] = free.to(torch.int32)
    refs[free] = 1
    return [table, refs, s["status"]]


def _plain_fork(s):
    table, refs, lens = s["table"], s["refs"], s["seq_lens"]
    _plain_release(table, s["keep"], refs)
    src, dst = s["src"].long(), s["dst"].long()
    whole, part = lens[src].long() // BS, lens[src] % BS > 0
    j = torch.arange(table.shape[1], device="cuda")
    child = torch.where(j[None, :] < whole[:, None], table[src], -1)
    shared = child[child >= 0].long()
    refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    free = (refs == 0).nonzero().flatten()[:int(part.sum())]
    last = table[src[part], whole[part]].long()
    s["k"][free], s["v"][free] = s["k"][last], s["v"][last]
    child[part, whole[part]] = free.to(torch.int32)
    refs[free] = 1
    table[dst], lens[dst] = child, lens[src]
    return [table, lens, refs, s["status"], s["k"], s["v"]]


def _plain_compact(s):
    first, table, k, v = s["first"].long(), s["table"].long(), s["k"], s["v"]
    i = torch.arange(s["kept"].shape[1], device="cuda")
    seq, i = (i[None, :] < s["n_kept"][:, None]).nonzero().unbind(dim=1)
    to, of = first[seq] + i, first[seq] + s["kept"].long()[seq, i]
    to_block, of_block = table[seq, to // BS], table[seq, of // BS]
    k[to_block, :, :, to % BS, :] = k[of_block, :, :, of % BS, :]
    v[to_block, :, :, to % BS] = v[of_block, :, :, of % BS]
    return [k, v]


def run(state):
    if own:
        return _run_own(state)
    plain = {"tree": _plain_tree, "window": _plain_window, "append": _plain_append, "draft": _plain_draft,
             "fork": _plain_fork, "compact": _plain_compact}
    return plain[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    lens, news = _lens(case), _news(case)
    rows = int(news.sum())
    nbs = -(-(lens + news) // BS)
    if op in ("tree", "window"):
        if op == "tree":
            seen = int((lens * news).sum()) + sum(bin(int(m)).count("1") for m in _masks(case, news))
            read = int((lens + news)[news > 0].sum())
        else:
            at = np.concatenate([n0 + np.arange(n) for n0, n in zip(lens, news)] or [np.zeros(0, dtype=np.int64)])
            w, k = case["window"], case["sinks"]
            seen = int((np.minimum(at + 1, w) + np.minimum(k, np.maximum(0, at + 1 - w))).sum())
            first = np.maximum(0, lens - w + 1)
            read = int(((lens + news) - first + np.minimum(k, first))[news > 0].sum())
        each = D * (2 + (2 if case["bf16"] else 4)) + 4
        return {"bytes": read * hkv * TOKEN_BYTES + 4 * (read // BS) + rows * hq * each + 8 * rows,
                "flops": 4 * D * hq * seen}
    if op == "append":
        return {"bytes": 2 * rows * hkv * TOKEN_BYTES + 8 * case["batch"] + 4 * rows // BS, "flops": 0}
    if op == "draft":
        new = int((nbs - -(-lens // BS)).sum())
        return {"bytes": 4 * (8 * new + 3 * case["batch"]), "flops": 0}  # entries and counts, taken and given back
    if op == "fork":
        n = case["batch"] * case["children"]
        entries = int((lens // BS).mean() * n)
        return {"bytes": 8 * 4 * entries + n * (2 * BS * hkv * TOKEN_BYTES + 16), "flops": 0}
    kept = int(_kept_counts(case, news).sum())
    return {"bytes": max(1, kept) * (2 * hkv * TOKEN_BYTES + 4), "flops": 0}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    if case["op"] not in ("tree", "window"):
        return None  # copies and whole numbers
    s = prepare(case, seed)
    out, lse = s["out"].double(), s["lse"].double()
    hkv, group, scale = case["hkv"], case["hq"] // case["hkv"], 1.0 / math.sqrt(D)
    starts = np.concatenate([[0], np.cumsum(s["news"])])
    for b in range(case["batch"]):
        n0, n = int(s["lens"][b]), int(s["news"][b])
        if n == 0:
            continue
        r0, tokens = int(starts[b]), n0 + n
        blocks = s["table"][b, :-(-tokens // BS)].long()
        t = torch.arange(tokens, device="cuda")
        if case["op"] == "tree":
            sees = torch.zeros((n, tokens), dtype=torch.bool, device="cuda")
            for p in range(case["parts"]):
                sees[:, int(s["begin"][p, b]):int(s["end"][p, b])] = True
            bits = s["mask"][r0:r0 + n]
            for j in range(n):
                sees[:, n0 + j] = (bits >> j & 1) == 1
        else:
            at = n0 + torch.arange(n, device="cuda")[:, None]
            sees = (t <= at) & ((t > at - case["window"]) | (t < case["sinks"]))
        for h in range(hkv):
            key = s["k"][blocks, h].permute(0, 2, 1, 3).reshape(-1, D)[:tokens].double()
            value = s["v"][blocks, h].permute(0, 2, 1).reshape(-1, D)[:tokens].double()
            key, value = key.nan_to_num(0.0), value.nan_to_num(0.0)
            for e in range(group):
                x = s["q"][r0:r0 + n, h * group + e].double() @ key.t().contiguous() * scale
                x = x.masked_fill(~sees, -math.inf)
                total = torch.logsumexp(x, dim=1)
                weight = torch.exp(x - torch.where(total == -math.inf, 0.0, total)[:, None])
                out[r0:r0 + n, h * group + e] = weight @ value
                lse[r0:r0 + n, h * group + e] = total
    return [out, lse]
