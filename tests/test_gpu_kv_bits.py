"""Equal calls give equal bits, and what a row cannot see (other rows, unused slots, places without a token) does not move its bits."""
import math

import pytest
import torch

import kv_cases as ref
from test_gpu_kv_cache import fill_new, on_gpu, same

pytestmark = pytest.mark.gpu

# (query heads, kv heads, head dim, page, slots in use, new tokens, tree): groups that do and do not divide a tile of 128 rows
FORMS = [(4, 2, 128, 32, [300, 41], [2, 1], False), (6, 1, 64, 16, [3, 33], [2, 2], False), (20, 5, 128, 64, [9, 0, 200], [15, 40, 31], True),
         (7, 1, 128, 64, [0, 70], [1200, 300], False), (9, 3, 64, 16, [130, 5], [90, 150], True), (33, 1, 128, 64, [70, 500], [50, 3], True),
         (48, 1, 64, 128, [700], [130], False)]


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_24273_b200 import bitrl

    bitrl.lib()
    torch.cuda.set_device(0)
    return bitrl


def trees(seed, news, is_tree):
    return torch.tensor([p for s, m in enumerate(news) for p in ref.tree(seed + s, m, m // 8)], dtype=torch.int32) if is_tree else None


def attend(B, c, q, news, nh, par):
    g = on_gpu(B, c)
    att = B.attention_cached(g, 0, q.cuda(), (ref.offsets(news).cuda(), max(news)), nh, parent=None if par is None else par.cuda())
    return att, g


@pytest.mark.parametrize("nh,nkv,hd,page,used,news,is_tree", FORMS)
def test_equal_calls_give_equal_bits(B, nh, nkv, hd, page, used, news, is_tree):
    """Whatever ran before: other calls leave other queries, of other sizes, on the chip."""
    par = trees(710, news, is_tree)
    c = ref.make(701, used, news, nkv, hd, page)
    q = fill_new(c, 702, news, par, nh)
    other = ref.make(703, used, news, nkv, hd, page, scale=20.0)
    q_other = fill_new(other, 704, news, par, nh, scale=20.0)
    att, g = attend(B, c, q, news, nh, par)
    for i in range(8):
        attend(B, other, q_other * (i + 1), news, nh, par)
        again, h = attend(B, c, q, news, nh, par)
        assert same(again, att) and torch.equal(h.mass, g.mass)
    B.poll_status()


@pytest.mark.parametrize("nh,nkv,hd,page,used,news,is_tree", FORMS)
def test_what_is_not_seen_does_not_move_a_bit(B, nh, nkv, hd, page, used, news, is_tree):
    """Unused slots, the slots and queries of padding, rows behind the last sequence: NaN, zeros or large numbers there."""
    par = trees(720, news, is_tree)
    c = ref.make(705, used, news, nkv, hd, page)  # unused slots hold NaN and infinities
    q = fill_new(c, 706, news, par, nh)
    full = torch.zeros(c["k"].shape[:4], dtype=torch.bool)
    T, off = q.shape[0], ref.offsets(news)
    real = torch.ones(T, dtype=torch.bool) if par is None else par != ref.PAD
    for s, (u, m) in enumerate(zip(used, news)):
        slots = [t for t in range(u + m) if t < u or real[int(off[s]) + t - u]]
        pg, at = ref.at(c, s, slots)
        full[0, pg, :, at] = True
    outs = []
    for fill in (None, 0.0, 3.0e4, -math.inf):
        x, y = dict(c), q.clone()
        if fill is not None:
            for name in ("k", "v"):
                x[name] = torch.where(full[..., None], c[name], fill)
        y[~real] = 0.0 if fill is None else abs(fill) if math.isfinite(fill) else math.nan
        y = torch.cat([y, torch.full((3, y.shape[1]), math.nan if fill is None else 2 * fill, dtype=y.dtype)])
        p = None if par is None else torch.cat([par, torch.zeros(3, dtype=torch.int32)])
        att, g = attend(B, x, y, news, nh, p)
        outs.append((att[:T].cpu(), torch.where(full, g.mass.cpu(), 0.0)))
    B.poll_status()
    for att, mass in outs[1:]:
        assert same(att, outs[0][0]) and torch.equal(mass, outs[0][1])


@pytest.mark.parametrize("nh,nkv,hd,m", [(2, 1, 64, 6), (4, 2, 128, 8), (8, 1, 128, 40), (7, 1, 64, 30)])
def test_a_siblings_token_does_not_move_a_bit(B, nh, nkv, hd, m):
    """A drafted token that is seen by itself alone: its key and value, whatever they hold, leave the others' results as they are."""
    used, news = [21, 70, 0], [m] * 3
    par = torch.tensor(3 * ([ref.PAST, ref.PAST] + [0] * (m - 2)), dtype=torch.int32)
    c = ref.make(707, used, news, nkv, hd, 16)
    q = fill_new(c, 708, news, par, nh)
    others = [r for r in range(3 * m) if r % m != 1]
    outs = []
    for k, v in ((None, None), (0.0, math.inf), (math.nan, math.nan), (9.0, -3.0e4), (1.0, -math.inf)):
        x = {n: t.clone() for n, t in c.items()}
        for s in range(3):
            pg, at = ref.at(c, s, [used[s] + 1])
            if k is not None:
                x["k"][0, pg, :, at], x["v"][0, pg, :, at] = k, v
        att, _ = attend(B, x, q, news, nh, par)
        outs.append(att[others])
        if v is not None and math.isinf(v):
            assert (att[[1, m + 1, 2 * m + 1]] == v).all()
    B.poll_status()
    for att in outs[1:]:
        assert same(att, outs[0])
