"""CPU checks of the calls on new tokens and blocks: declared and exported alike, bad arguments refused on the host
before any HIP call, by the C ABI and by the binding; the host code under AddressSanitizer and UBSan."""

import ctypes
import math
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2510_13223_amd import bana

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "bana_tokens.h")
FAKE = ctypes.c_void_p(0x100000)  # 16-byte aligned, never dereferenced: every case below fails validation
ODD = ctypes.c_void_p(0x100008)
BIG = 1 << 40

CALLS = {
    "tree_attn": ["d", 8, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1, FAKE, FAKE, 1.0, FAKE, 0, FAKE, None, 0, None],
    "window_attn": ["d", 8, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 5, 1, 1.0, FAKE, 1, FAKE, None, 0, None],
    "append_kv": ["d", 8, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None],
    "compact_kv_tokens": ["d", FAKE, FAKE, FAKE, FAKE, FAKE, 4, FAKE, None],
    "reserve_kv_blocks": ["d", FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, BIG, None],
    "fork_kv_seqs": ["d", FAKE, FAKE, 2, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, BIG, None],
    "release_kv_blocks": ["d", FAKE, FAKE, FAKE, FAKE, None],
}
# Arguments that may be NULL: lse, the window's partition, the workspace of attention, the stream.
OPTIONAL = {"tree_attn": {15, 16, 18}, "window_attn": {8, 9, 15, 16, 18}, "append_kv": {9}, "compact_kv_tokens": {8},
            "reserve_kv_blocks": {8}, "fork_kv_seqs": {12}, "release_kv_blocks": {5}}
ALIGNED = {"tree_attn": {3, 4, 5, 13, 16}, "window_attn": {3, 4, 5, 13, 16}, "append_kv": {4, 5, 7, 8},
           "compact_kv_tokens": {1, 2}, "reserve_kv_blocks": {6}, "fork_kv_seqs": {4, 5, 10}, "release_kv_blocks": set()}


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(bana_[a-z0-9_]+)\s*\(", text)))


@pytest.fixture(scope="module")
def lib():
    return bana.lib()


def dims(**kw):
    d = bana.make_dims(4, 8, 2, 64, 100)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def call(lib, name, change=None, d=None):
    args = list(CALLS[name])
    args[0] = ctypes.byref(d if d is not None else dims())
    for i, x in (change or {}).items():
        args[i] = x
    return getattr(lib, "bana_" + name)(*args)


def test_every_declared_symbol_is_exported(lib):
    names = declared()
    assert {"bana_" + n for n in CALLS} <= set(names) and len(names) == 10
    for n in names:
        assert hasattr(lib, n), n


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned_pointers_are_invalid(lib, name):
    for i, x in enumerate(CALLS[name]):
        if i == 0 or (x is FAKE and i not in OPTIONAL[name]):
            assert call(lib, name, {i: None}) == -1, i
        if i in ALIGNED[name]:
            assert call(lib, name, {i: ODD}) == -1, i


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kw,expect", [
    (dict(batch=0), -1), (dict(num_kv_heads=3), -1), (dict(num_blocks=0), -1), (dict(max_blocks_per_seq=0), -1),
    (dict(max_range_tokens=-1), -1), (dict(total_range_tokens=-1), -1), (dict(head_dim=64), -2),
    (dict(block_size=32), -2), (dict(num_q_heads=34), -2), (dict(max_blocks_per_seq=1 << 28), -2),
    (dict(batch=1 << 24), -2),
])
def test_bad_dims(lib, name, kw, expect):
    assert call(lib, name, d=dims(**kw)) == expect


def test_bad_sizes_and_kinds(lib):
    for name, rows in (("tree_attn", 1), ("window_attn", 1), ("append_kv", 1)):
        assert call(lib, name, {rows: -1}) == -1
        assert call(lib, name, {rows: 1 << 24}) == -2
        assert call(lib, name, {rows: 1 << 62}) == -2
        assert call(lib, name, {rows: 0}) == 0  # nothing to do
    for name in ("tree_attn", "window_attn"):
        for scale in (0.0, -1.0, math.nan, math.inf, 3e38):
            assert call(lib, name, {12: scale}) == -1
        for kind in (-1, 2):
            assert call(lib, name, {14: kind}) == -1
        assert call(lib, name, {1: 1 << 23}) == -2  # rows x heads
    for parts, expect in ((0, -1), (-3, -1), (64, -2)):
        assert call(lib, "tree_attn", {9: parts}) == expect
    assert call(lib, "tree_attn", {9: 63}, dims(max_blocks_per_seq=1 << 26, batch=1)) == -2
    assert call(lib, "window_attn", {10: 0}) == -1 and call(lib, "window_attn", {10: -5}) == -1
    assert call(lib, "window_attn", {11: -1}) == -1
    assert call(lib, "window_attn", {8: FAKE}) == -1 and call(lib, "window_attn", {9: FAKE}) == -1
    assert call(lib, "compact_kv_tokens", {6: -1}) == -1 and call(lib, "compact_kv_tokens", {6: 0}) == 0
    assert call(lib, "compact_kv_tokens", {6: 1 << 30}) == -2
    assert call(lib, "fork_kv_seqs", {3: -1}) == -1 and call(lib, "fork_kv_seqs", {3: 5}) == -1
    assert call(lib, "fork_kv_seqs", {3: 0}) == 0
    for name in ("reserve_kv_blocks", "fork_kv_seqs", "release_kv_blocks"):
        assert call(lib, name, d=dims(num_blocks=1 << 31)) == -2
    assert call(lib, "reserve_kv_blocks", d=dims(batch=1 << 10, max_blocks_per_seq=1 << 21)) == -2
    need = lib.bana_kv_blocks_workspace_bytes(ctypes.byref(dims()))
    assert need >= 4 * 100
    for name, at in (("reserve_kv_blocks", 7), ("fork_kv_seqs", 11)):
        assert call(lib, name, {at: need - 1}) == -1
    for f in (lambda d: lib.bana_kv_blocks_workspace_bytes(d), lambda d: lib.bana_tree_attn_workspace_bytes(d, 9, 1),
              lambda d: lib.bana_window_attn_workspace_bytes(d, 9, 5, 0)):
        assert f(None) == 0 and f(ctypes.byref(dims(head_dim=64))) == 0
    assert lib.bana_tree_attn_workspace_bytes(ctypes.byref(dims()), -1, 1) == 0
    assert lib.bana_tree_attn_workspace_bytes(ctypes.byref(dims()), 5, 64) == 0
    assert lib.bana_window_attn_workspace_bytes(ctypes.byref(dims()), 5, 0, 0) == 0


def test_the_binding_refuses_host_tensors_and_leaves_them_to_python():
    n = bana._calls()
    x = torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    k, v = torch.zeros(2, 1, 16, 16, 8, dtype=torch.bfloat16), torch.zeros(2, 1, 128, 16, dtype=torch.bfloat16)
    t = torch.zeros(1, 2, dtype=torch.int32)
    assert n.tree(*[x] * 11, 1.0, None, None, None) is None
    assert n.window(*[x] * 6, 5, 0, x, x, 1.0, None, None, None, None, None) is None
    assert n.append(*[x] * 7, None) is None and n.compact(*[x] * 6, None) is None
    assert n.reserve(*[x] * 6, None) is None and n.fork(*[x] * 9, None) is None and n.release(*[x] * 4, None) is None
    assert n.tree() is None and n.window(1) is None and n.release(1, 2) is None
    for f in (lambda: bana.bana_tree_attn(x, i, k, v, t, t, t, i, i, x),
              lambda: bana.bana_window_attn(x, i, k, v, t, i, 5, 0, x),
              lambda: bana.bana_append_kv(x, x, i, i, t, k, v),
              lambda: bana.bana_compact_kv_tokens(k, v, t, i, t, i),
              lambda: bana.bana_reserve_kv_blocks(t, i, i, i, i, i),
              lambda: bana.bana_fork_kv_seqs(i, i, k, v, t, i, i, i, i),
              lambda: bana.bana_release_kv_blocks(t, i, i, i)):
        with pytest.raises(ValueError):
            f()


@pytest.mark.gpu
def test_the_binding_says_what_is_wrong():
    dev = "cuda:0"
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16, device=dev)
    rb = torch.tensor([0, 4], dtype=torch.int32, device=dev)
    k = torch.zeros(3, 2, 16, 16, 8, dtype=torch.bfloat16, device=dev)
    v = torch.zeros(3, 2, 128, 16, dtype=torch.bfloat16, device=dev)
    t = torch.zeros(1, 2, dtype=torch.int32, device=dev)
    one = torch.ones(1, dtype=torch.int32, device=dev)
    out, lse = torch.zeros_like(q), torch.zeros(4, 8, device=dev)
    good = dict(q=q, row_begin=rb, k_cache=k, v_cache=v, block_table=t, seq_lens=4 * one, window=3, sinks=0, out=out,
                lse=lse)
    bana.bana_window_attn(**good)
    for change, error in ((dict(q=q.float()), TypeError), (dict(q=q[:, :, :64]), ValueError),
                          (dict(q=q[:, ::2]), ValueError), (dict(out=out[:3]), ValueError),
                          (dict(out=out.half()), TypeError), (dict(row_begin=rb[:1]), ValueError),
                          (dict(seq_lens=4), TypeError), (dict(seq_lens=rb), ValueError), (dict(window=0), ValueError),
                          (dict(sinks=-1), ValueError), (dict(window=1 << 31), ValueError),
                          (dict(lse=lse.double()), TypeError), (dict(kv_range_begin=one), ValueError),
                          (dict(scale=0.0), bana.BanaError), (dict(scale=math.nan), bana.BanaError),
                          (dict(v_cache=v[:2]), ValueError), (dict(block_table=t[0]), ValueError),
                          (dict(dims=bana.make_dims(2, 8, 2, 2, 3)), ValueError),
                          (dict(q=q.repeat(1, 5, 1), out=out.repeat(1, 5, 1), lse=None), bana.BanaError)):
        with pytest.raises(error):
            bana.bana_window_attn(**{**good, **change})
    bana.bana_window_attn(**{**good, "scale": 1, "lse": None})  # an int scale, no lse
    empty = torch.zeros(0, 8, 128, dtype=torch.bfloat16, device=dev)
    bana.bana_window_attn(**{**good, "q": empty, "out": empty, "lse": None})
    with pytest.raises(ValueError):
        bana.bana_tree_attn(q, rb, k, v, t, t, t, one, torch.zeros(4, device=dev, dtype=torch.int64), out)
    with pytest.raises(TypeError):
        bana.bana_tree_attn(q, rb, k, v, t, one[None], one[None], one, torch.zeros(4, device=dev), out)
    with pytest.raises(ValueError):
        bana.bana_append_kv(q, q, rb, one, t, k, v)  # eight heads into a cache of two
    with pytest.raises(ValueError):
        bana.bana_compact_kv_tokens(k, v, t, one, one, one)
    refs, status = torch.zeros(3, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    with pytest.raises(bana.BanaError):
        bana.bana_reserve_kv_blocks(t, one, one, refs, status, None)
    with pytest.raises(bana.BanaError):
        bana.bana_reserve_kv_blocks(t, one, one, refs, status, refs)
    with pytest.raises(ValueError):
        bana.bana_fork_kv_seqs(one, one, k, v, t, one, refs[:2], status, refs)
    with pytest.raises(ValueError):
        bana.bana_release_kv_blocks(t, rb, refs, status)


def test_host_code_sweep_under_sanitizers(tmp_path):
    """The entry points with stub launchers that check every planned launch against the call's buffers."""
    sys.path.insert(0, os.path.join(ROOT, "tests", "c"))
    import build as c_build

    csrc = os.path.join(ROOT, "paper_2510_13223_amd", "csrc")
    exe = str(tmp_path / "sanitize_tokens")
    cmd = ["g++", "-std=c++17", *c_build.SANITIZE, f"-I{os.path.join(c_build.ROCM, 'include')}",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{csrc}", "-D__HIP_PLATFORM_AMD__", "-DBANA_HOSTCHECK_LIBRARY",
           os.path.join(csrc, "bana_api.cpp"), os.path.join(csrc, "tokens_api.cpp"),
           os.path.join(ROOT, "tests", "c", "sanitize_host.cpp"),
           os.path.join(ROOT, "tests", "c", "sanitize_tokens.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1")
    r = subprocess.run([exe, "20000"], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "launches checked" in r.stdout
