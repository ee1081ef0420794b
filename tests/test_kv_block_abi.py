"""Argument checks of the block-scaled cache and of the rows read back: they answer without touching a GPU."""
import pytest


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    return luvc


FAKE = 4096          # an aligned address that is never dereferenced: the checks fail first


def cache_of(luvc, **changes):
    c = luvc.KvCacheStruct(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 2, 64, 4, 16, 128, 8, 32, luvc.E4M3_BLOCK)
    for name, value in changes.items():
        setattr(c, name, value)
    return c


def test_the_cache_description_is_checked(luvc):
    assert luvc.lib.luvc_kv_workspace_bytes(cache_of(luvc), 8) > 0
    for status, changes in ((1, dict(k_scale=None)), (1, dict(v_scale=None)), (7, dict(dtype=3)), (7, dict(dtype=5)), (6, dict(D=72)),
                            (6, dict(k_scale=FAKE + 2)), (2, dict(page_size=24)), (2, dict(D=272))):
        c = cache_of(luvc, **changes)
        assert luvc.lib.luvc_kv_write(c, 0, None, 4, FAKE, FAKE, 512, 512, 4, None, None, 0, None) == status, changes
        assert luvc.lib.luvc_kv_read(c, 0, None, 4, None, FAKE, FAKE, 512, 512, 4, None, 0, None) == status, changes
        assert luvc.lib.luvc_attn_decode(FAKE, 3584, c, 0, None, 4, 28, 0, FAKE, None) == status, changes
        assert luvc.lib.luvc_kv_workspace_bytes(c, 4) == 0, changes


def test_the_arguments_of_a_read_are_checked(luvc):
    read = lambda **k: luvc.lib.luvc_kv_read(*[k.get(n, d) for n, d in (                              # noqa: E731
        ("c", cache_of(luvc)), ("layer", 0), ("seqs", None), ("n", 4), ("first", None), ("k", FAKE), ("v", FAKE), ("ks", 512), ("vs", 512),
        ("tokens", 4), ("starts", None), ("dtype", 0), ("opts", None))])
    assert read(k=None) == 1 and read(v=None) == 1
    assert read(dtype=1) == 7 and read(dtype=4) == 7
    assert read(layer=2) == 2 and read(layer=-1) == 2 and read(tokens=5) == 2 and read(tokens=-1) == 2 and read(ks=504) == 2 and read(vs=504) == 2
    assert read(n=0) == 2 and read(n=9) == 2 and read(n=4097, seqs=FAKE, starts=FAKE) == 2
    assert read(ks=516) == 6 and read(k=FAKE + 8) == 6 and read(v=FAKE + 4) == 6 and read(first=FAKE + 2) == 6 and read(starts=FAKE + 1) == 6
    assert read(opts=luvc.KvOpts(device_status=FAKE + 4)) == 6
