"""Rows of logits on both sides of the limit up to which a kernel may use x = z c - R (|R| = 2^24), against the statement in 64 bits
(tests/token_cases.py, which derives the bounds)."""
import math

import numpy as np
import pytest
import torch

import token_cases as tc
from test_gpu_token_loss import B, check_distill, check_logprobs, check_policy, check_ppo, teacher  # noqa: F401 (B: the fixture)

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF, NAN = math.inf, math.nan


def straddling(T, V, tau, sign, seed):
    """fp32 rows whose largest logits lie some ulps to either side of the limit, which is sign * 2^24 temperature / log2(e): anywhere, or those
    beyond it in one place."""
    limit = np.float32(sign * 2.0 ** 24 * tau * math.log(2.0))
    grid = [limit]
    for _ in range(3):
        grid = [np.nextafter(grid[0], np.float32(-INF)), *grid, np.nextafter(grid[-1], np.float32(INF))]
    grid = torch.tensor(np.array(grid, np.float32))  # ascending, the limit in the middle
    g = torch.Generator().manual_seed(seed)
    z = grid[torch.randint(0, 7, (T, V), generator=g)]
    low, high = grid[1], grid[5]
    for t in range(T):
        kind = t % 8
        if kind == 1:
            z[t], z[t, V // 2] = low, high
        elif kind == 2:  # the first element, where a row may begin with an edge
            z[t], z[t, 0] = low, high
        elif kind == 3:  # the last
            z[t], z[t, -1] = low, high
        elif kind == 4:  # the second half: another thread's, chunk's, share's
            z[t] = torch.where(torch.arange(V) < V // 2, low, high)
        elif kind == 5:
            z[t] = torch.where(torch.arange(V) < V // 2, high, low)
        elif kind == 6:  # few of either, all others left out
            keep = torch.rand(V, generator=g) < 3 / V
            keep[0] = keep[-1] = True
            z[t] = torch.where(keep, z[t], -INF)
        elif kind == 7:  # one vector in every 128
            z[t] = torch.where(torch.arange(V) // 8 % 128 == 5, high, low)
    return z


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("tau", [1.0, 1e-3, 1e-6, 2.0 ** 20])
@pytest.mark.parametrize("T,V,ld,offset", [(8, 2, 2, 0), (16, 50, 53, 1), (8, 9000, 9001, 3), (8, 40000, 40000, 0), (1200, 300, 300, 0)])
def test_rows_across_the_limit(B, T, V, ld, offset, tau, sign):
    """Sums that were begun on one side go on on the other: in one vector, between threads, chunks, edges and shares of a cluster."""
    view, store = tc.logits(T, V, F32, 1, ld=ld, offset=offset)
    view.copy_(straddling(T, V, tau, sign, T + V))
    zg = tc.on_gpu(view, store)
    tokens = np.arange(T) * 7 % V
    check_logprobs(B, view, tokens, tau, min(V, 9), zg=zg)
    check_policy(B, view, tokens, tau, np.linspace(-1, 1, T), np.full(T, 0.1), zg=zg)
    check_ppo(B, view, tau, 3, zg=zg)
    for tail in (False, True):
        ids, values = teacher(torch.zeros(T, V), max(1, min(6, V // 2)), tail, 1.0, 4, few=False)
        check_distill(B, view, ids, values, tail, tau, zg=zg)


@pytest.mark.parametrize("tau", [16.0, 100.0, 256.0])
@pytest.mark.parametrize("V", [50, 9000])
def test_half_precision_rows_across_their_lower_limit(B, V, tau):
    """fp16 maxima below -16384 subtract first, those above it do not."""
    g = torch.Generator().manual_seed(V)
    z = (-16384 + 24.0 * torch.randint(-40, 3, (6, V), generator=g)).to(F16)
    z[1, ::2] = -INF
    tokens = np.arange(6) * 5
    check_logprobs(B, z, tokens, tau, 9)
    check_policy(B, z, tokens, tau, np.linspace(-1, 1, 6), np.full(6, 0.1))
    check_ppo(B, z, tau, 3)
    for tail in (False, True):
        ids, values = teacher(torch.zeros(6, V), 6, tail, 1.0, 4, few=False)
        check_distill(B, z, ids, values, tail, tau)


@pytest.mark.parametrize("top,dent", [(20.0, 1e5), (5.0, 1e11)])
@pytest.mark.parametrize("V", [60, 9000])
def test_large_entropy_terms_leave_masked_tokens_without_gradient(B, V, top, dent):
    """At the lowest temperature, with maxima beyond the limit (11.1) and below it: the gradient of a token that is left out is 0, however large the
    entropy's part."""
    tau = 2.0 ** -20
    z = top + tc.logits(4, V, F32, V)[0] * 1e-6
    z[:, 1::3] = -INF
    z[3, 4:] = -INF
    G, E = np.array([1.0, 0.0, -1.0, 1.0]), dent * np.array([1.0, -1.0, 0.5, 1.0])
    got, _ = check_policy(B, z, np.array([0, 2, 3, 0]), tau, G, E)
    assert not got[:, 1::3].any()
    r = tc.Rows(tc.f64(z), tau)
    tokens = np.array([0, 2, 3, 0], np.int32)
    old, one = torch.tensor(r.lp[np.arange(4), tokens], dtype=F32).cuda(), torch.ones(4, device="cuda")
    ppo = B.ppo_token_loss(z.cuda(), torch.from_numpy(tokens).cuda(), old, one, beta=dent, temperature=tau)["dlogits"]
    B.poll_status()
    assert torch.isfinite(ppo).all() and not ppo[:, 1::3].any()
