"""Rows of logits where a number leaves its type: on both sides of the limit up to which a kernel may use x = z c - R (|R| = 2^24), factors of masked
tokens' exponents, masses below what 64 bits hold; against the statement in 64 bits (tests/token_cases.py, which derives the bounds)."""
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


def distill_with_tail(z, ids, values, tau, w, lowest):
    """(loss, its error, dz, its error) of distill_topk with tail, p_r by its logarithm, so that it may lie below what 64 bits hold.  Bounds as those of
    tc.Rows: S outside the names has its terms' errors, 6 |d| + 8 each, and its additions'; log p_r is a difference of 64-bit numbers beside those.
    There, logits of the type's lowest value are a mask."""
    T, V = z.shape
    r = tc.Rows(z, tau)
    loss, err_loss, dz, err_dz = np.zeros(T), np.zeros(T), np.zeros((T, V)), np.zeros((T, V))
    with np.errstate(all="ignore"):
        for t in range(T):
            j, q = ids[t], np.exp(values[t].astype(np.float64))
            outside = np.ones(V, bool)
            outside[j] = False
            rows = tc.Rows(np.where(outside, z[t], -INF)[None], tau)
            gap = (rows.m[0] - r.m[t]) / tau
            log_rest = gap + rows.log_s[0] - r.log_s[t]
            q_rest = max(0.0, 1.0 - q.sum())
            if log_rest < -745 and q_rest <= 2.0 ** -20:
                q_rest = 0.0
            masked = log_rest < -745 and rows.m[0] <= lowest
            if masked:
                log_rest = -INF
            named = q * (values[t] - r.lp[t, j])
            term = q_rest * (np.log(q_rest) - log_rest) if q_rest > 0 else 0.0
            loss[t] = named.sum() + term
            err_rest = rows.err_s[0] + r.err_log_s[t]
            err_loss[t] = (q * r.err_lp[t, j]).sum() + 16 * tc.U * np.abs(named).sum() + q_rest * err_rest + (0.0 if masked else 2.0 ** -50 * abs(log_rest))
            ratio = np.where(outside, 0.0 if masked else rows.p[0], 0.0)  # p_j / p_r
            total = q.sum() + q_rest
            g = total * r.p[t] - q_rest * ratio
            np.subtract.at(g, j, q)
            dz[t] = w[t] * g / tau
            rel = np.where(rows.p[0] > 0, tc.U * (8 * np.abs(np.where(np.isfinite(rows.d[0]), rows.d[0], 0)) + 20) + rows.err_s[0], 0.0)
            size = np.where(outside, total * r.p[t], 1.0)
            err_dz[t] = w[t] / tau * (q_rest * ratio * (rel + 8 * tc.U) + size * (r.rel_p()[t] + 16 * tc.U) + 4 * tc.EXP_MIN)
    return loss, err_loss, dz, err_dz


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("T,V", [(8, 40), (8, 9000), (4, 128000), (1200, 300)])
@pytest.mark.parametrize("tau,gap", [(1.0, 1e4), (0.05, 50.0), (2.0 ** -20, 3.0), (1.0, 700.0), (4.0, 1e4), (1.0, INF), (200.0, INF)])
def test_distill_of_a_mass_outside_the_names_below_64_bits(B, T, V, dtype, tau, gap):
    """Named tokens that lie far above all others (an additive mask of -10000, a low temperature): log p_r is a number as long as a logit is there that is no
    mask, and the gradient outside the names follows it.  With the type's lowest value it is -inf."""
    K = 5
    g = torch.Generator().manual_seed(V)
    z = torch.randn(T, V, generator=g) * tau
    ids = torch.rand(T, V, generator=g).topk(K, 1).indices
    named = z.gather(1, ids)
    z = torch.full_like(z, torch.finfo(dtype).min) if gap == INF else z - gap
    z = z.scatter(1, ids, named).to(dtype)
    z[1::4, 7:] = torch.where(torch.rand(z[1::4, 7:].shape, generator=g) < 0.5, z[1::4, 7:], torch.tensor(-INF, dtype=dtype))  # some left out altogether
    z = z.scatter(1, ids, named.to(dtype))
    q = torch.softmax(torch.randn(T, K, generator=g).double(), 1) * torch.tensor([0.9, 0.3, 0.999, 1.0]).double().repeat(T // 4)[:, None]
    ids, values, w = ids.numpy().astype(np.int32), q.log().float().numpy(), (np.linspace(0.5, 2.0, T) * min(1.0, tau)).astype(np.float32).astype(np.float64)
    out = B.distill_topk(z.cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(values).cuda(), torch.tensor(w, dtype=F32).cuda(), tail=True, temperature=tau)
    B.poll_status()
    loss, el, dz, ed = distill_with_tail(tc.f64(z), ids, values, tau, w, torch.finfo(dtype).min)
    tc.close(out["loss"], loss, el, what="loss")
    tc.close(out["dlogits"], dz, ed, dtype, "gradient")


def test_distill_of_a_student_that_leaves_out_all_but_the_names(B):
    """-inf outside the names, and logits further below than fp32 reaches: p_r = 0, the loss +inf unless what the teacher has outside is rounding."""
    z = torch.full((4, 300), -INF)
    z[2:] = -3.4e38
    z[:, :3] = torch.tensor([3e38, 2.9e38, 3e38])
    values = torch.tensor([[0.3, 0.0, 0.3], [0.5, 0.0, 0.5], [0.3, 0.0, 0.3], [0.5, 0.0, 0.5]]).log()
    out = B.distill_topk(z.cuda(), torch.tensor([[0, 1, 2]] * 4, dtype=torch.int32).cuda(), values.cuda(), tail=True)
    B.poll_status()
    assert torch.isposinf(out["loss"][[0, 2]]).all() and (out["loss"][[1, 3]].abs() < 8 * tc.U).all()
    assert not out["dlogits"][:, 3:].any() and torch.isfinite(out["dlogits"]).all()
