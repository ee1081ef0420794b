"""Argument checks of the attention to an encoder's states: they answer without touching a GPU."""
import os
import subprocess
import sys

import pytest


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    return luvc


FAKE = 4096          # an aligned address that is never dereferenced: the checks fail first


def test_the_arguments_are_checked(luvc):
    call = lambda **k: luvc.lib.luvc_attn_cross(*[k.get(n, d) for n, d in (                            # noqa: E731
        ("q", FAKE), ("qs", 3584), ("k", FAKE), ("ks", 512), ("v", FAKE), ("vs", 512), ("n", 4), ("q_starts", FAKE), ("k_starts", FAKE),
        ("q_tokens", 9), ("k_tokens", 100), ("q_heads", 28), ("heads", 4), ("D", 128), ("dtype", 0), ("out", FAKE), ("opts", None))])
    o = luvc.AttnCrossOpts
    assert call(q=None) == 1 and call(k=None) == 1 and call(v=None) == 1 and call(out=None) == 1 and call(k_starts=None) == 1
    assert call(dtype=2) == 7 and call(dtype=4) == 7
    assert call(n=0) == 2 and call(n=4097) == 2 and call(q_tokens=-1) == 2 and call(k_tokens=-1) == 2 and call(q_starts=None) == 2
    assert call(heads=0) == 2 and call(q_heads=30) == 2 and call(q_heads=0) == 2 and call(q_heads=1 << 17, qs=1 << 24) == 2
    assert call(D=0) == 2 and call(D=264, qs=1 << 14, ks=1 << 14, vs=1 << 14) == 2
    assert call(qs=3576) == 2 and call(ks=504) == 2 and call(vs=504) == 2 and call(opts=o(scale=float("nan"))) == 2
    assert call(D=12) == 6 and call(dtype=1, D=126) == 6 and call(qs=3588) == 6 and call(ks=513) == 6 and call(vs=516) == 6
    assert call(q=FAKE + 8) == 6 and call(k=FAKE + 2) == 6 and call(v=FAKE + 8) == 6 and call(out=FAKE + 4) == 6
    assert call(q_starts=FAKE + 2) == 6 and call(k_starts=FAKE + 1) == 6
    assert call(opts=o(key_bias=FAKE + 2)) == 6 and call(opts=o(lse=FAKE + 1)) == 6 and call(opts=o(device_status=FAKE + 4)) == 6
    size = luvc.lib.luvc_attn_cross_workspace_bytes()
    assert size > 1024
    assert call(opts=o(workspace=FAKE, workspace_bytes=size - 1)) == 8 and call(opts=o(workspace=FAKE + 16, workspace_bytes=size)) == 8
    assert call(q_tokens=0, q=None, out=None) == 0              # nothing to do


def test_without_a_gpu_a_call_answers_with_an_error():
    code = """
import paper_2512_09010_b200 as luvc
A, L = 4096, luvc.lib
o = luvc.AttnCrossOpts(workspace=A, workspace_bytes=1 << 30, device_status=A)
for dtype in (0, 1):
    assert L.luvc_attn_cross(A, 3584, A, 512, A, 512, 4, A, A, 9, 100, 28, 4, 128, dtype, A, o) == 9
assert L.luvc_attn_cross(A, 3584, A, 512, A, 512, 4, A, A, 9, 100, 28, 4, 128, 0, A, None) == 9
assert L.luvc_rope(A, 4096, A, A, 8, 32, 128, 128, 0, A, 4096, None) == 9
c = luvc.KvCacheStruct(A, A, A, A, A, A, A, 2, 64, 4, 16, 128, 8, 32, luvc.E4M3_BLOCK)
k = luvc.KvOpts(workspace=A, workspace_bytes=1 << 20, device_status=A)
assert L.luvc_kv_write(c, 0, None, 4, A, A, 512, 512, 4, None, None, 0, k) == 9
assert L.luvc_kv_read(c, 0, None, 4, None, A, A, 512, 512, 4, None, 0, k) == 9
assert L.luvc_kv_fork(c, A, A, 4, k) == 9
assert L.luvc_attn_decode(A, 3584, c, 0, None, 4, 28, 0, A, luvc.AttnOpts(workspace=A, workspace_bytes=1 << 30, device_status=A)) == 9
print("answered")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True)
    assert r.returncode == 0 and "answered" in r.stdout, (r.returncode, r.stderr[-500:])
