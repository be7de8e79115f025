"""Whole batches of distillation's gradients, every element against its statement in 64 bits."""
import math

import pytest
import torch

import token_cases as tc
from test_gpu_token_rows import LAYOUTS, B, Batch, T  # noqa: F401 (B: the fixture)
from token_cases import U

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,dtype,ld,offset", LAYOUTS)
def test_every_row_of_a_distillation(B, V, dtype, ld, offset, tail):
    """All rows' gradients element by element.  An element is w / temperature times total p_j, less q_j at a named token, less q_r p_j / p_r
    elsewhere: each term is off by the roundings of its exponential, 8 |d| + 12 (d from the row's largest; within the outside ones it is less), of its sums,
    6 sum p |d| + 8 and V / 128 + 64 additions for either, log S's 4 |log S|, and 16 of its own."""
    b = Batch(V, dtype, V + 3, ld, offset)
    tau, K = [1.0, 0.5, 2.0][V % 3], 40
    ids, values = b.teacher(K, tail, tau, 5)
    w = b.weight * (65536.0 if dtype is F16 else 1.0)  # (small gradients as loss scaling has them)
    got = B.distill_topk(b.z, ids, values, w, tail=tail, temperature=tau)["dlogits"]
    B.poll_status()
    seen = []
    for lo in range(0, T, 125):
        z, j, v, wt = b.z[lo : lo + 125].double(), ids[lo : lo + 125].long(), values[lo : lo + 125].double(), w[lo : lo + 125].double()[:, None]
        has = j >= 0
        live = has.any(1, keepdim=True) & ((z > -math.inf).any(1, keepdim=True) | z.isnan().any(1, keepdim=True)) & (wt != 0)
        x = (v if tail else v / tau).masked_fill(~has, -math.inf)
        q = x.exp() if tail else torch.softmax(x, 1).nan_to_num(0.0)
        q_rest = (1 - q.sum(1, keepdim=True)).clamp_min(0.0) if tail else torch.zeros_like(wt)
        named = torch.zeros(len(z), V + 1, dtype=torch.float64, device="cuda").scatter_add_(1, torch.where(has, j, V), q)[:, :V]
        mark = torch.zeros(len(z), V + 1, dtype=torch.bool, device="cuda").scatter_(1, torch.where(has, j, V), True)[:, :V]
        d = (z - z.nan_to_num(-math.inf, posinf=math.inf).amax(1, keepdim=True)) / tau
        log_s = torch.logsumexp(d, 1, keepdim=True)
        p = (d - log_s).exp()
        rest = torch.logsumexp((d - log_s).masked_fill(mark, -math.inf), 1, keepdim=True)
        q_rest = torch.where((q_rest <= 2.0 ** -20) & (rest < -745), 0.0, q_rest)
        masked = (rest < -745) & (z.masked_fill(mark, -math.inf).amax(1, keepdim=True) <= torch.finfo(dtype).min)  # p_r = 0
        outside = torch.where(mark | masked | (q_rest == 0), 0.0, q_rest * (d - log_s - rest).exp())
        total = q.sum(1, keepdim=True) + q_rest
        want = torch.where(live, wt * (total * p - named - outside) / tau, 0.0)
        size = wt * (total * p + named + outside) / tau
        ad = torch.where(p > 0, d.abs(), 0.0)
        n = V / 128 + 64
        roundings = 8 * ad + 12 + 2 * (6 * (p * ad).sum(1, keepdim=True) + 8 + n) + 4 * log_s.abs() + 16 + K
        err = U * roundings * size
        err = err + tc.HALF[dtype] * (want.abs() + err) + tc.TINY[dtype] + 4 * tc.EXP_MIN * wt / tau
        g = got[lo : lo + 125].double()
        ok = (g == want) | (g.isnan() & want.isnan()) | ((g - want).abs() <= err)
        assert ok.all(), f"{(~ok).sum()} differ, first at {(~ok).nonzero()[0].tolist()}: {g[~ok][0]} for {want[~ok][0]}, may be off by {err[~ok][0]}"
        plain = live[:, 0] & want.isfinite().all(1)
        seen.append((want[plain].abs() > 4 * err[plain]).double().mean().item())
    # A bound that zeros would meet shows nothing.  (Half a step of bf16 is 2^-8, subnormals of fp16 begin at 2^-14, and a difference may cancel.)
    assert min(seen) > 0.5
