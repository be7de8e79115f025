"""How the softmax weights meet the values in attention over the paged cache: with 16 bits, and with values that are not finite."""
import math

import pytest
import torch

import kv_cases as ref
from test_gpu_kv_cache import fill_new, on_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_24273_b200 import bitrl

    bitrl.lib()
    torch.cuda.set_device(0)
    return bitrl


def exact(c, q, off, nh, parent=None, weight=2.0**-16 + 2.0**-19):
    """64-bit (att [T, nh, hd], tolerance): the result is rounded once to bf16 (2^-8 of it); a weight meets the values as two bf16
    halves: of a weight in [1, 2) the first keeps what is above 2^-7, the rest, below 2^-7, is rounded to bf16 (half a step there is
    2^-16) and kept above zero by 2^-20; scores, exponentials and sums in fp32 as in kv_cases.attend.  A row that sees nothing is zero."""
    nkv, hd = c["k"].shape[2], c["k"].shape[4]
    rep = nh // nkv
    att, tol = (torch.zeros(q.shape[0], nh, hd, dtype=torch.float64) for _ in range(2))
    for s in range(len(off) - 1):
        t0, m, u = int(off[s]), int(off[s + 1] - off[s]), int(c["used"][s])
        par = [i - 1 for i in range(m)] if parent is None else parent[t0 : t0 + m].tolist()
        sees = torch.zeros(m, u + m, dtype=torch.bool)
        for i in range(m):
            chain = ref.above(par, i)
            sees[i, :u] = bool(chain)
            sees[i, [u + j for j in chain]] = True
        pages, places = ref.at(c, s, range(u + m))
        for h in range(nkv):
            k, v = c["k"][0][pages, h, places].double(), c["v"][0][pages, h, places].double()
            some = sees.any(0)[:, None]
            k, v = torch.where(some, k, 0.0), torch.where(some, v, 0.0)  # padding's slots
            x = q[t0 : t0 + m].double().reshape(m, nh, hd)[:, h * rep : (h + 1) * rep].transpose(0, 1)
            p = torch.softmax((x @ k.T / math.sqrt(hd)).masked_fill(~sees, -math.inf), 2).nan_to_num(0.0)
            d = 2 * hd * 2.0**-23 * float((x.abs() @ k.abs().T).max()) / math.sqrt(hd) + 2.0**-21 + (u + m) * 2.0**-23
            o = p @ v
            att[t0 : t0 + m, h * rep : (h + 1) * rep] = o.transpose(0, 1)
            tol[t0 : t0 + m, h * rep : (h + 1) * rep] = (2.0**-8 * o.abs() + (weight + d) * (p @ v.abs())).transpose(0, 1)
    return att, tol


# (query heads, kv heads, head dim, page, slots in use, new tokens, tree): few rows, one and two row tiles, several items; histories of
# a few slots, where the roundings of the weights do not average out
FORMS = [(4, 2, 128, 32, [300, 41], [2, 1], False), (6, 1, 64, 16, [3, 33], [2, 2], False), (8, 2, 128, 64, [500, 2], [25, 40], True),
         (20, 5, 128, 64, [9, 0, 200], [15, 40, 31], False), (8, 2, 64, 16, [130, 5], [90, 150], False), (4, 1, 128, 64, [700], [300], False)]


@pytest.mark.parametrize("nh,nkv,hd,page,used,news,is_tree", FORMS)
def test_weights_meet_the_values_with_sixteen_bits(B, nh, nkv, hd, page, used, news, is_tree):
    c = ref.make(201, used, news, nkv, hd, page, scale=0.25)
    par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(210 + s, m, m // 8)], dtype=torch.int32) if is_tree else None
    q = fill_new(c, 202, news, par, nh, scale=0.25)
    off = ref.offsets(news)
    att = B.attention_cached(on_gpu(B, c), 0, q.cuda(), (off.cuda(), max(news)), nh, parent=None if par is None else par.cuda())
    B.poll_status()
    want, tol = exact(c, q, off, nh, par)
    err = (att.cpu().double().reshape(want.shape) - want).abs() - tol
    assert not att.isnan().any() and err.max() <= 0, f"{float(err.max()):.3g} beyond, {int((err > 0).sum())} of {err.numel()}"


@pytest.mark.parametrize("nh,nkv,hd,page,used,news,is_tree", FORMS + [(8, 1, 128, 64, [5000, 130], [1, 1], False)])
def test_infinite_values_reach_those_who_see_them(B, nh, nkv, hd, page, used, news, is_tree):
    """An infinite value in a slot that a row sees makes that dimension of the row's result the same infinity (both signs: NaN),
    whatever the weight's bits are; every other result, and the weights, stay what they were."""
    c = ref.make(221, used, news, nkv, hd, page, scale=0.25)
    par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(230 + s, m)], dtype=torch.int32) if is_tree else None
    q = fill_new(c, 222, news, par, nh, scale=0.25)
    off = ref.offsets(news)
    states = (off.cuda(), max(news))
    gp = None if par is None else par.cuda()
    plain = on_gpu(B, c)
    B.attention_cached(plain, 0, q.cuda(), states, nh, parent=gp)
    g = ref.gen(223)
    up, down = (torch.zeros(q.shape[0], nh, hd, dtype=torch.bool) for _ in range(2))
    for s, (u, m) in enumerate(zip(used, news)):
        t0, rep = int(off[s]), nh // nkv
        tree = [i - 1 for i in range(m)] if par is None else par[t0 : t0 + m].tolist()
        slots = sorted({0, u // 3, u // 2, max(u - 1, 0), u + m // 2, u + m - 1})
        for h in range(nkv):
            for slot in slots:
                dims = torch.randperm(hd, generator=g)[: hd // 6]
                sign = torch.where(torch.rand(len(dims), generator=g) < 0.5, 1.0, -1.0)
                pg, at = ref.at(c, s, [slot])
                c["v"][0, pg[0], h, at[0], dims] = (sign * math.inf).to(torch.bfloat16)
                for i in range(m):
                    if slot < u or slot - u in ref.above(tree, i):
                        for j in range(h * rep, (h + 1) * rep):
                            up[t0 + i, j, dims] |= sign > 0
                            down[t0 + i, j, dims] |= sign < 0
    # what the finite values of a dimension give; the infinite ones count as zero in `want`
    zeroed = {**c, "v": torch.where(c["v"].isinf(), 0.0, c["v"])}
    want, tol = exact(zeroed, q, off, nh, par)
    got = on_gpu(B, c)
    att = B.attention_cached(got, 0, q.cuda(), states, nh, parent=gp).cpu().double().reshape(want.shape)
    B.poll_status()
    assert (up & ~down).any() and (down & ~up).any() and not (up | down).all()
    assert (att[up & ~down] == math.inf).all() and (att[down & ~up] == -math.inf).all() and att[up & down].isnan().all()
    rest = ~(up | down)
    assert ((att - want).abs()[rest] <= tol[rest]).all()
    assert torch.equal(got.mass, plain.mass)


@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
def test_infinities_among_many_short_items(B, hd, page):
    """Sequences of one and of two row tiles in turn, a few with values that some of their drafted tokens must not see."""
    nh, nkv, n_seq = 8, 2, 320
    news = [[40, 9, 12, 7, 20][s % 5] for s in range(n_seq)]
    used = [(37 * s) % 150 for s in range(n_seq)]
    c = ref.make(241, used, news, nkv, hd, page, scale=0.25)
    trees = [[ref.PAST, ref.PAST] + [0] * (m - 2) for m in news]  # token 1 is seen by itself alone
    par = torch.tensor([p for t in trees for p in t], dtype=torch.int32)
    q = fill_new(c, 242, news, par, nh, scale=0.25)
    off = ref.offsets(news)
    want, tol = exact(c, q, off, nh, par)
    odd = [s for s in range(n_seq) if s % 7 in (0, 3)]
    for s in odd:
        pg, at = ref.at(c, s, [used[s] + 1])
        c["v"][0, pg, :, at] = math.inf
        pg, at = ref.at(c, s, [used[s]])  # token 0 is seen by all but token 1
        c["v"][0, pg, 0, at, 5] = -math.inf
    att = B.attention_cached(on_gpu(B, c), 0, q.cuda(), (off.cuda(), max(news)), nh, parent=par.cuda()).cpu().double().reshape(want.shape)
    B.poll_status()
    for s in odd:
        t0, m, rep = int(off[s]), news[s], nh // nkv
        want[t0 + 1] = math.inf
        rows = [t0] + list(range(t0 + 2, t0 + m))
        want[rows, :rep, 5] = -math.inf
    bad = want.isinf()
    assert torch.equal(att[bad], want[bad])
    assert ((att - want).abs()[~bad] <= tol[~bad]).all()
