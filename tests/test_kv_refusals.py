"""Calls on a cache that are refused: argument checks come before anything touches a device, so they run without one."""
import ctypes

import pytest

from paper_2604_24273_b200 import bitrl

P = 1 << 20  # never dereferenced: a 16-byte aligned address


@pytest.fixture(scope="module")
def L():
    from paper_2604_24273_b200 import build

    build.build()
    return bitrl.lib()


def desc(**kw):
    d = dict(k=P, v=P, mass=P, pos=P, page_table=P, used=P, seen=P, n_layers=2, n_pages=8, n_kv_heads=2, page_tokens=16,
             head_dim=64, n_seq=2, max_pages=4)
    d.update(kw)
    return ctypes.byref(bitrl.KvCacheDesc(*d.values()))


def append(L, c=None, layer=0, qkv=P, T=6, off=P, max_new=4, parent=None, nh=4, theta=1e4, q=P):
    return L.bitrl_kv_append(c or desc(), layer, qkv, T, off, max_new, parent, nh, theta, q, None)


def attend(L, c=None, layer=0, q=P, T=6, off=P, max_new=4, parent=None, nh=4, mass=1, att=P, ws=P, nbytes=1 << 40):
    return L.bitrl_attention_cached(c or desc(), layer, q, T, off, max_new, parent, nh, mass, att, ws, nbytes, None)


BAD_CACHES = [
    (dict(k=None), bitrl.ERR_NULL), (dict(v=None), bitrl.ERR_NULL), (dict(pos=None), bitrl.ERR_NULL), (dict(page_table=None), bitrl.ERR_NULL),
    (dict(used=None), bitrl.ERR_NULL), (dict(seen=None), bitrl.ERR_NULL), (dict(page_tokens=24), bitrl.ERR_SHAPE),
    (dict(page_tokens=256), bitrl.ERR_SHAPE), (dict(head_dim=96), bitrl.ERR_SHAPE), (dict(n_seq=0), bitrl.ERR_SHAPE),
    (dict(n_layers=0), bitrl.ERR_SHAPE), (dict(n_pages=0), bitrl.ERR_SHAPE), (dict(max_pages=0), bitrl.ERR_SHAPE),
    (dict(n_kv_heads=0), bitrl.ERR_SHAPE), (dict(max_pages=bitrl.KV_MAX_SLOTS // 16 + 1), bitrl.ERR_LIMIT),
    (dict(k=P + 8), bitrl.ERR_ALIGN), (dict(mass=P + 4), bitrl.ERR_ALIGN),
]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_bad_caches(L, kw, want):
    c = desc(**kw)
    assert append(L, c) == want
    assert attend(L, c) == want
    assert L.bitrl_kv_evict_plan(c, 16, 4, 0, 64, P, P, None) == want
    assert L.bitrl_kv_move(c, P, P, 4, 1, None) == want
    assert L.bitrl_kv_advance(c, P, 4, None, 0, None) == want


BAD_BATCHES = [
    (dict(layer=2), bitrl.ERR_SHAPE), (dict(layer=-1), bitrl.ERR_SHAPE), (dict(nh=3), bitrl.ERR_SHAPE), (dict(nh=0), bitrl.ERR_SHAPE),
    (dict(T=-1), bitrl.ERR_SHAPE), (dict(max_new=-1), bitrl.ERR_SHAPE), (dict(off=None, T=6), bitrl.ERR_SHAPE),
    (dict(max_new=65), bitrl.ERR_SHAPE), (dict(c=desc(max_pages=64), max_new=257, parent=P), bitrl.ERR_LIMIT),
    (dict(c=desc(n_seq=1 << 24, max_pages=64), max_new=512), bitrl.ERR_LIMIT),
]


@pytest.mark.parametrize("kw,want", BAD_BATCHES)
def test_bad_batches(L, kw, want):
    assert append(L, **kw) == want
    assert attend(L, **kw) == want


def test_other_refusals(L):
    assert append(L, theta=0.0) == bitrl.ERR_SHAPE
    assert append(L, qkv=None) == bitrl.ERR_NULL and append(L, q=None) == bitrl.ERR_NULL
    assert append(L, qkv=P + 2) == bitrl.ERR_ALIGN
    assert attend(L, q=None) == bitrl.ERR_NULL and attend(L, att=None) == bitrl.ERR_NULL
    assert attend(L, ws=None) == bitrl.ERR_WORKSPACE and attend(L, nbytes=16) == bitrl.ERR_WORKSPACE
    assert attend(L, c=desc(mass=None)) == bitrl.ERR_NULL
    assert attend(L, q=P + 8) == bitrl.ERR_ALIGN
    c = desc()
    assert L.bitrl_kv_evict_plan(c, 0, 0, 0, 64, P, P, None) == bitrl.ERR_SHAPE
    assert L.bitrl_kv_evict_plan(c, 16, -1, 0, 64, P, P, None) == bitrl.ERR_SHAPE
    assert L.bitrl_kv_evict_plan(c, 16, 0, -1, 64, P, P, None) == bitrl.ERR_SHAPE
    assert L.bitrl_kv_evict_plan(c, 16, 0, 0, 15, P, P, None) == bitrl.ERR_SHAPE  # room for 16 moves is wanted
    assert L.bitrl_kv_evict_plan(c, 16, 0, 0, 16, None, P, None) == bitrl.ERR_NULL
    assert L.bitrl_kv_evict_plan(desc(mass=None), 16, 0, 0, 16, P, P, None) == bitrl.ERR_NULL
    assert L.bitrl_kv_move(c, P, P, -1, 1, None) == bitrl.ERR_SHAPE
    assert L.bitrl_kv_move(c, None, P, 4, 1, None) == bitrl.ERR_NULL
    assert L.bitrl_kv_advance(c, P, -1, None, 0, None) == bitrl.ERR_SHAPE
    assert L.bitrl_kv_advance(c, P, 4, None, -1, None) == bitrl.ERR_SHAPE
    assert L.bitrl_encoder_forward_cached(None, c, P, 4, P, 4, None, 1e4, 1, P, None, P, 1 << 30, None) == bitrl.ERR_NULL


def test_nothing_to_do_is_fine_without_a_device(L):
    assert append(L, T=0, max_new=4, qkv=None, q=None) == bitrl.OK
    assert attend(L, T=0, max_new=4, q=None, att=None, ws=None) == bitrl.OK
    assert L.bitrl_kv_move(desc(), None, None, 0, 1, None) == bitrl.OK


def test_outputs_that_overlap_inputs(L):
    q = 6 * 4 * 64 * 2  # bytes of the six tokens' queries
    for at in (P, P + q - 16, P - q + 16):
        assert append(L, q=at) == bitrl.ERR_SHAPE
        assert attend(L, att=at) == bitrl.ERR_SHAPE
    assert append(L, q=P + 2 * q - 16) == bitrl.ERR_SHAPE  # the values of the last token
    if not bitrl.torch.cuda.is_available():  # beside one another: the next check is the device's
        assert append(L, q=P + 2 * q) not in (bitrl.OK, bitrl.ERR_SHAPE)
        assert attend(L, att=P + q) not in (bitrl.OK, bitrl.ERR_SHAPE) and attend(L, att=P - q) not in (bitrl.OK, bitrl.ERR_SHAPE)


def test_a_group_that_is_too_large(L):
    assert attend(L, desc(n_kv_heads=1), nh=bitrl.KV_MAX_GROUP + 1) == bitrl.ERR_LIMIT
    assert append(L, desc(n_kv_heads=1), nh=bitrl.KV_MAX_GROUP + 1) == bitrl.ERR_LIMIT
    assert L.bitrl_attention_cached_workspace_bytes(desc(n_kv_heads=1), 6, 4, bitrl.KV_MAX_GROUP + 1) == 0


def test_workspace_query(L):
    assert L.bitrl_attention_cached_workspace_bytes(desc(), 6, 4, 4) > 0
    assert L.bitrl_attention_cached_workspace_bytes(desc(head_dim=80), 6, 4, 4) == 0
    assert L.bitrl_attention_cached_workspace_bytes(desc(), 0, 4, 4) == 0
    assert L.bitrl_attention_cached_workspace_bytes(desc(), 6, 4, 3) == 0


def test_the_binding_wants_cuda_tensors():
    import torch

    z = torch.zeros(1, 2, 1, 16, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        bitrl.KVCache(z, z, i[None], i, i)
