"""Argument checks of the key-value cache's and the attention's entry points: they answer without touching a GPU
(CPU only: no compute call is made here)."""
import ctypes
import os
import subprocess
import sys

import pytest


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    return luvc


FAKE = 4096          # an aligned address that is never dereferenced: the checks fail first


def cache_of(luvc, **changes):
    c = luvc.KvCacheStruct(FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 2, 64, 4, 16, 128, 8, 32, luvc.BF16)
    for name, value in changes.items():
        setattr(c, name, value)
    return c


def test_the_cache_description_is_checked(luvc):
    good = cache_of(luvc)
    assert luvc.lib.luvc_kv_workspace_bytes(good, 8) >= 8 * 32 * 12
    for status, changes in (
        (1, dict(k=None)), (1, dict(table=None)), (1, dict(lengths=None)), (1, dict(dtype=2)),      # e4m3 without scales
        (1, dict(k_scale=FAKE)),                                                                    # scales without e4m3
        (7, dict(dtype=3)), (2, dict(page_size=24)), (2, dict(page_size=0)), (2, dict(D=264)), (2, dict(D=0)),
        (2, dict(pages=0)), (2, dict(layers=0)), (2, dict(slots=0)), (2, dict(max_pages=0)), (2, dict(heads=40000)),
        (2, dict(pages=1 << 26)),                                                                   # 2^32 rows per layer
        (2, dict(max_pages=1 << 28)),                                                               # 2^32 tokens
        (6, dict(D=12)), (6, dict(k=FAKE + 8)), (6, dict(refs=FAKE + 2)),
        (6, dict(dtype=2, D=72, k_scale=FAKE, v_scale=FAKE)),                                       # 72-byte rows
    ):
        c = cache_of(luvc, **changes)
        assert luvc.lib.luvc_kv_reserve(c, None, 4, FAKE, None) == status, changes
        assert luvc.lib.luvc_kv_write(c, 0, None, 4, FAKE, FAKE, 512, 512, 4, None, None, 0, None) == status, changes
        assert luvc.lib.luvc_kv_fork(c, FAKE, FAKE, 4, None) == status, changes
        assert luvc.lib.luvc_kv_free(c, FAKE, 4, None) == status, changes
        assert luvc.lib.luvc_kv_compact(c, None, 4, FAKE, FAKE, FAKE, 4, None, None) == status, changes
        assert luvc.lib.luvc_attn_decode(FAKE, 3584, c, 0, None, 4, 28, 0, FAKE, None) == status, changes
        assert luvc.lib.luvc_kv_workspace_bytes(c, 4) == 0, changes


def test_the_calls_arguments_are_checked(luvc):
    L, c = luvc.lib, cache_of(luvc)
    assert L.luvc_kv_reserve(c, None, 0, FAKE, None) == 2
    assert L.luvc_kv_reserve(c, None, 9, FAKE, None) == 2                 # more sequences than slots
    assert L.luvc_kv_reserve(c, FAKE, 4097, FAKE, None) == 2
    assert L.luvc_kv_reserve(c, None, 4, None, None) == 1
    assert L.luvc_kv_reserve(c, FAKE + 1, 4, FAKE, None) == 6
    write = lambda **k: L.luvc_kv_write(*[k.get(n, d) for n, d in (                                   # noqa: E731
        ("c", c), ("layer", 0), ("seqs", None), ("n", 4), ("k", FAKE), ("v", FAKE), ("ks", 512), ("vs", 512), ("tokens", 4),
        ("starts", None), ("sizes", None), ("dtype", 0), ("opts", None))])
    assert write(k=None) == 1 and write(v=None) == 1
    assert write(dtype=1) == 7 and write(dtype=2) == 7
    assert write(layer=2) == 2 and write(layer=-1) == 2 and write(tokens=5) == 2 and write(ks=504) == 2
    assert write(ks=513, starts=FAKE) == 6 and write(k=FAKE + 8) == 6 and write(sizes=FAKE + 2) == 6
    assert L.luvc_kv_fork(c, None, FAKE, 1, None) == 1 and L.luvc_kv_fork(c, FAKE, None, 1, None) == 1
    assert L.luvc_kv_compact(c, None, 4, None, FAKE, FAKE, 4, None, None) == 1
    assert L.luvc_kv_compact(c, None, 4, FAKE, FAKE, None, 4, None, None) == 1
    assert L.luvc_kv_compact(c, None, 4, FAKE, FAKE, FAKE, -1, None, None) == 4
    o = luvc.KvOpts(workspace=FAKE, workspace_bytes=luvc.lib.luvc_kv_workspace_bytes(c, 4) - 1)
    assert L.luvc_kv_compact(c, None, 4, FAKE, FAKE, FAKE, 4, None, o) == 8
    assert L.luvc_kv_fork(c, FAKE, FAKE, 4, o) == 8
    o = luvc.KvOpts(workspace=FAKE + 128, workspace_bytes=1 << 20)
    assert L.luvc_kv_compact(c, None, 4, FAKE, FAKE, FAKE, 4, None, o) == 8
    assert L.luvc_kv_free(c, FAKE, 4, luvc.KvOpts(device_status=FAKE + 4)) == 6


def test_the_attentions_arguments_are_checked(luvc):
    L, c = luvc.lib, cache_of(luvc)
    attn = lambda **k: L.luvc_attn_decode(*[k.get(n, d) for n, d in (                                  # noqa: E731
        ("q", FAKE), ("stride", 3584), ("c", c), ("layer", 0), ("seqs", None), ("n", 4), ("heads", 28), ("dtype", 0),
        ("out", FAKE), ("opts", None))])
    assert attn(q=None) == 1 and attn(out=None) == 1
    assert attn(dtype=1) == 7 and attn(dtype=2) == 7
    assert attn(heads=30) == 2 and attn(heads=0) == 2                      # not a multiple of the 4 key heads
    assert attn(stride=3576) == 2 and attn(n=0) == 2 and attn(n=9) == 2 and attn(layer=2) == 2
    assert attn(stride=3585) == 6 and attn(q=FAKE + 2) == 6 and attn(seqs=FAKE + 2) == 6
    assert attn(opts=luvc.AttnOpts(scale=float("nan"))) == 2
    assert attn(opts=luvc.AttnOpts(key_bias=FAKE, bias_width=8, bias_stride=7)) == 2
    assert attn(opts=luvc.AttnOpts(key_bias=FAKE + 2, bias_width=8, bias_stride=8)) == 6
    assert attn(opts=luvc.AttnOpts(workspace=FAKE, workspace_bytes=0)) == 8
    assert attn(opts=luvc.AttnOpts(device_status=FAKE + 4)) == 6


def test_the_status_has_a_name(luvc):
    assert luvc.STATUS_NAMES[12] == "LUVC_ERR_PAGES"
    assert b"page" in luvc.lib.luvc_status_string(12)
    assert ctypes.sizeof(luvc.KvCacheStruct) == 7 * 8 + 8 * 4


def test_without_a_gpu_a_call_answers_with_an_error():
    """The number of SMs that launches are sized by cannot be asked of a device that is not there."""
    code = """
import paper_2512_09010_b200 as luvc
A = 4096
c = luvc.KvCacheStruct(A, A, A, A, A, None, None, 2, 64, 4, 16, 128, 8, 32, luvc.BF16)
o = luvc.KvOpts(workspace=A, workspace_bytes=1 << 20, device_status=A)
L = luvc.lib
assert L.luvc_kv_write(c, 0, None, 4, A, A, 512, 512, 4, None, None, 0, o) == 9
assert L.luvc_kv_reserve(c, None, 4, A, o) == 9
assert L.luvc_kv_free(c, A, 4, o) == 9
assert L.luvc_kv_fork(c, A, A, 4, o) == 9
assert L.luvc_kv_compact(c, None, 4, A, A, A, 4, None, o) == 9
a = luvc.AttnOpts(workspace=A, workspace_bytes=1 << 30, device_status=A)
assert L.luvc_attn_decode(A, 3584, c, 0, None, 4, 28, 0, A, a) == 9
print("answered")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True)
    assert r.returncode == 0 and "answered" in r.stdout, (r.returncode, r.stderr[-500:])
