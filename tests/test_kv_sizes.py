"""Workspace queries of the calls over a paged cache: a size for what a call takes, 0 for what it refuses."""
import ctypes

import pytest
import torch

from paper_2604_24273_b200 import bitrl
from test_kv_refusals import L, attend, desc  # noqa: F401  (L is the library as a fixture)

INT_MAX = 2**31 - 1
# (cache, T, max_new, heads) that bitrl_attention_cached refuses, and its answer
REFUSED = [
    (desc(), 6, 65, 4, bitrl.ERR_SHAPE),  # more new tokens than a sequence has slots
    (desc(n_kv_heads=1), 6, 4, bitrl.KV_MAX_GROUP + 1, bitrl.ERR_LIMIT),
    (desc(n_kv_heads=1), 6, 4, 129, bitrl.ERR_LIMIT),
    (desc(n_seq=1 << 24, max_pages=64), 6, 512, 4, bitrl.ERR_LIMIT),  # sequences * new tokens * heads
    (desc(), INT_MAX // 4 + 1, 4, 4, bitrl.ERR_LIMIT),  # rows * heads
    (desc(n_pages=1 << 28), 6, 4, 4, bitrl.ERR_LIMIT),  # rows of a layer's pool
    (desc(n_seq=1 << 20, max_pages=1 << 15), 6, 1, 2, bitrl.ERR_LIMIT),  # units of all sequences
]


@pytest.mark.parametrize("cache,T,max_new,nh,status", REFUSED)
def test_no_size_for_a_refused_call(L, cache, T, max_new, nh, status):  # noqa: F811
    assert attend(L, cache, T=T, max_new=max_new, nh=nh) == status
    assert L.bitrl_attention_cached_workspace_bytes(cache, T, max_new, nh) == 0


@pytest.mark.parametrize("nh,nkv", [(4, 2), (64, 1), (128, 2), (6, 6)])
@pytest.mark.parametrize("T,max_new", [(1, 1), (7, 4), (90, 64)])
def test_a_size_for_an_accepted_call(L, nh, nkv, T, max_new):  # noqa: F811
    assert L.bitrl_attention_cached_workspace_bytes(desc(n_kv_heads=nkv), T, max_new, nh) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("group", [65, 129])
def test_an_encoder_whose_group_is_too_large(group):
    """The encoder itself takes any group; over a cache it is refused, and its size query answers 0."""
    nkv, hd, d_ff = 2, 64, 128
    nh = group * nkv
    d, n_qkv = nh * hd, (nh + 2 * nkv) * hd
    gamma = torch.ones(1, device="cuda")
    linear = lambda N, K: bitrl.Linear(torch.zeros(N * K // 4, dtype=torch.uint8, device="cuda"), gamma, N, K)  # noqa: E731
    enc = bitrl.Encoder([(linear(n_qkv, d), linear(d, d), linear(2 * d_ff, d), linear(d, d_ff))], d, d_ff, nh, nkv)
    cache = bitrl.KVCache.empty(1, 2, 64, nkv, hd, page_tokens=16)
    assert enc.cached_workspace_bytes(cache, 2, 1) == 0
    with pytest.raises(bitrl.BitrlError) as e:
        enc.forward_cached(torch.zeros(2, d, dtype=torch.bfloat16, device="cuda"), cache, 1)
    assert e.value.status == bitrl.ERR_LIMIT
    assert ctypes.c_size_t(enc.workspace_bytes(2)).value > 0
    bitrl.poll_status()


def test_a_budget_of_all_slots_needs_no_list(L):  # noqa: F811
    """max_moves >= min(budget, slots - budget) is 0 or less then, and an empty tensor has no address."""
    P = 1 << 20
    if not torch.cuda.is_available():  # past the arguments' checks, the next one is the device's
        for budget in (64, 1000):
            assert L.bitrl_kv_evict_plan(desc(), budget, 4, 0, 0, None, P, None) not in (bitrl.OK, bitrl.ERR_NULL, bitrl.ERR_SHAPE)
    assert L.bitrl_kv_evict_plan(desc(), 63, 4, 0, 0, None, P, None) == bitrl.ERR_SHAPE
    assert L.bitrl_kv_evict_plan(desc(), 63, 4, 0, 1, None, P, None) == bitrl.ERR_NULL
    assert L.bitrl_kv_evict_plan(desc(), 64, 4, 0, 0, None, None, None) == bitrl.ERR_NULL


@pytest.mark.gpu
def test_a_plan_without_moves():
    cache = bitrl.KVCache.empty(2, 3, 64, 2, 64, page_tokens=16)
    cache.used.copy_(torch.tensor([64, 0, 10], dtype=torch.int32))
    moves = torch.empty(2, 3, 2, 0, 2, dtype=torch.int32, device="cuda")
    count = torch.full((2, 3, 2), 7, dtype=torch.int32, device="cuda")
    bitrl.kv_evict_plan(cache, 64, 4, moves=moves, count=count)
    bitrl.kv_move(cache, moves, count)
    bitrl.poll_status()
    assert not count.any()
