"""Operators on the paged key/value cache against plain 64-bit forms (tests/kv_cases.py)."""
import math

import pytest
import torch

import kv_cases as ref

pytestmark = pytest.mark.gpu
THETA = 500000.0


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_24273_b200 import bitrl

    bitrl.lib()
    torch.cuda.set_device(0)
    return bitrl


def on_gpu(B, c):
    return B.KVCache(*(c[n].cuda() for n in ("k", "v", "page_table", "used", "seen")), mass=c["mass"].cuda(), pos=c["pos"].cuda())


def put(c, layer, rows):
    """Writes appended rows {(seq, i): (k, v, pos)} of ref.append into the CPU cache."""
    for (s, i), (k, v, p) in rows.items():
        pg, at = ref.at(c, s, [int(c["used"][s]) + i])
        c["k"][layer, pg, :, at] = k.to(torch.bfloat16)
        c["v"][layer, pg, :, at] = v.to(torch.bfloat16)
        c["pos"][layer, pg, :, at] = p
        c["mass"][layer, pg, :, at] = 0.0


def same(x, y):
    """Equal, NaN matching NaN."""
    return torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x, y.view(torch.int16) if y.dtype == torch.bfloat16 else y)


def check_attend(B, c, q, news, nh, parent, behind=2, layer=0, states=None, mass=True):
    """attention_cached on the CPU cache c (new rows already in it) against ref.attend."""
    off = ref.offsets(news)
    T = int(off[-1]) + behind
    q = torch.cat([q, torch.full((behind, q.shape[1]), math.nan, dtype=torch.bfloat16)])
    par = None if parent is None else torch.cat([parent, torch.full((behind,), 99, dtype=torch.int32)])
    want, add, tol, mtol, real = ref.attend(c, layer, q, off, nh, parent)
    g = on_gpu(B, c)
    att = torch.full((T, q.shape[1]), 7.0, dtype=torch.bfloat16, device="cuda")
    B.attention_cached(g, layer, q.cuda(), (off.cuda(), max(news)) if states is None else states, nh,
                       parent=None if par is None else par.cuda(), att=att, accumulate_mass=mass)
    B.poll_status()
    got = att.cpu().double().reshape(T, nh, -1)
    assert (got[~real] == 7.0).all(), "rows behind the last sequence were written"
    err = (got - want).abs()[real] - tol[real]
    assert not got[real].isnan().any() and err.max() <= 0, f"att off by {err.max():.3g} beyond its tolerance"
    if mass:
        m0, m1 = c["mass"][layer].double(), g.mass.cpu()[layer].double()
        bad = (m1 - m0 - add).abs() - (mtol + 2.0**-23 * (m0 + add))
        assert bad.max() <= 0, f"mass off by {bad.max():.3g} beyond its tolerance"
    else:
        assert torch.equal(g.mass.cpu(), c["mass"])
    assert same(g.k.cpu(), c["k"]) and same(g.v.cpu(), c["v"]) and torch.equal(g.pos.cpu(), c["pos"])
    assert torch.equal(g.used.cpu(), c["used"]) and torch.equal(g.seen.cpu(), c["seen"])
    return att, g


def fill_new(c, seed, news, parent, nh, layer=0, scale=1.0):
    """Random keys and values for the new tokens (not for padding) and queries [T, nh*hd]."""
    g = ref.gen(seed)
    off = ref.offsets(news)
    nkv, hd = c["k"].shape[2], c["k"].shape[4]
    rows = {}
    for s, m in enumerate(news):
        for i in range(m):
            k, v = scale * torch.randn(nkv, hd, generator=g), torch.randn(nkv, hd, generator=g)
            if parent is None or int(parent[int(off[s]) + i]) != ref.PAD:
                rows[s, i] = (k, v, i)
    put(c, layer, rows)
    return (2 * torch.randn(int(off[-1]), nh * hd, generator=g)).to(torch.bfloat16)


SHAPES = [(4, 2, 64, 16), (4, 2, 128, 64), (7, 1, 128, 32), (9, 3, 64, 128), (20, 5, 128, 64), (16, 1, 64, 16), (3, 3, 128, 16)]


@pytest.mark.parametrize("nh,nkv,hd,page", SHAPES)
@pytest.mark.parametrize("used,news", [([0], [1]), ([1, 0, 37], [1, 1, 1]), ([300, 16, 0, 65], [5, 0, 3, 17]), ([40, 129], [0, 40])])
def test_append(B, nh, nkv, hd, page, used, news):
    c = ref.make(11, used, news, nkv, hd, page, layers=2)
    off = ref.offsets(news)
    qkv = torch.randn(int(off[-1]) + 1, (nh + 2 * nkv) * hd, generator=ref.gen(12)).to(torch.bfloat16)
    g = on_gpu(B, c)
    q_out = torch.full((qkv.shape[0], nh * hd), 3.0, dtype=torch.bfloat16, device="cuda")
    for par in (None, torch.tensor([p for s, m in enumerate(news) for p in ref.tree(20 + s, m, pads=m // 6)], dtype=torch.int32)):
        full = None if par is None else torch.cat([par, torch.zeros(1, dtype=torch.int32)]).cuda()
        q_out.fill_(3.0)
        B.kv_append(g, 1, qkv.cuda(), (off.cuda(), max(news)), nh, parent=full, theta=THETA, q_out=q_out)
        B.poll_status()
        want_q, rows = ref.append(c, 1, qkv, off, nh, par, THETA)
        put(c, 1, rows)
        got = q_out.cpu()
        for r in range(qkv.shape[0]):
            if r not in want_q:
                assert (got[r] == 3.0).all()
                continue
            x = qkv[r].double().reshape(-1, hd).abs()
            part = x + x.roll(hd // 2, 1)  # |x_i| + |x_{i+hd/2}|: what the rotation's fp32 terms are relative to
            assert ((got[r].double().reshape(nh, hd) - want_q[r]).abs() <= 2.0**-8 * want_q[r].abs() + 2.0**-20 * part[:nh]).all()
        for (s, i), (k, _, _) in rows.items():
            pg, at = ref.at(c, s, [used[s] + i])
            x = qkv[int(off[s]) + i].double().reshape(-1, hd).abs()
            part = (x + x.roll(hd // 2, 1))[nh : nh + nkv]
            gk = g.k[1].cpu()[pg, :, at][0].double()
            assert ((gk - k).abs() <= 2.0**-8 * k.abs() + 2.0**-20 * part).all()
            c["k"][1, pg, :, at] = g.k[1].cpu()[pg, :, at]  # compared above; the rest has to match to the bit
        assert same(g.k.cpu(), c["k"]) and same(g.v.cpu(), c["v"])
        assert torch.equal(g.pos.cpu(), c["pos"]) and torch.equal(g.mass.cpu(), c["mass"])


def test_append_far_positions(B):
    """Angles of far positions: 64-bit, so a position near 2^31 rotates as the definition says."""
    c = ref.make(1, [3], [2], 1, 128, 16)
    c["seen"][0] = 2**31 - 1 - 2
    qkv = torch.randn(2, 3 * 128, generator=ref.gen(2)).to(torch.bfloat16)
    g = on_gpu(B, c)
    q = B.kv_append(g, 0, qkv.cuda(), 2, 1, theta=THETA).cpu().double()
    B.poll_status()
    want, _ = ref.append(c, 0, qkv, ref.offsets([2]), 1, None, THETA)
    for r in range(2):
        # an angle of 2^31 in fp64 is off by 2^31 * 2^-52 (table entry and product): 2^-20 of a turn's rate
        assert ((q[r] - want[r][0]).abs() <= 2.0**-8 * want[r][0].abs() + 2.0**-17 * 4).all()


@pytest.mark.parametrize("nh,nkv,hd,page", SHAPES)
@pytest.mark.parametrize("used,news", [([0], [1]), ([1], [1]), ([15, 16, 17, 0], [1, 1, 1, 1]), ([700, 33], [1, 1])])
def test_single_tokens(B, nh, nkv, hd, page, used, news):
    c = ref.make(3, used, news, nkv, hd, page)
    q = fill_new(c, 4, news, None, nh)
    check_attend(B, c, q, news, nh, None)
    check_attend(B, c, q, news, nh, None, behind=0, states=1, mass=False)


@pytest.mark.parametrize("nh,nkv,hd,page", SHAPES)
@pytest.mark.parametrize("used,news", [([0, 20], [9, 33]), ([130, 0, 64, 5], [17, 0, 1, 64]), ([257], [130])])
def test_causal_tokens(B, nh, nkv, hd, page, used, news):
    c = ref.make(5, used, news, nkv, hd, page)
    check_attend(B, c, fill_new(c, 6, news, None, nh), news, nh, None)


@pytest.mark.parametrize("nh,nkv,hd,page", SHAPES)
@pytest.mark.parametrize("used,news,pads", [([0, 50], [7, 24], 0), ([100, 0, 31, 64], [31, 0, 2, 48], 3), ([63], [256], 40)])
def test_trees(B, nh, nkv, hd, page, used, news, pads):
    c = ref.make(7, used, news, nkv, hd, page)
    par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(30 + s, m, min(pads, m))], dtype=torch.int32)
    check_attend(B, c, fill_new(c, 8, news, par, nh), news, nh, par)


def test_padding_alone(B):
    c = ref.make(9, [40, 3], [4, 2], 2, 64, 16)
    par = torch.tensor([ref.PAD] * 4 + [ref.PAST, ref.PAD], dtype=torch.int32)
    att, _ = check_attend(B, c, fill_new(c, 10, [4, 2], par, 4), [4, 2], 4, par)
    assert (att[:4] == 0).all() and (att[5] == 0).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nh,m", [(2, 6), (8, 40)])
def test_infinities_in_unseen_slots(B, hd, nh, m):
    """A drafted token's key and value that its siblings do not see have no part in the siblings' results."""
    c = ref.make(13, [21, 70], [m, m], 1, hd, 16)
    par = torch.tensor(2 * ([ref.PAST, ref.PAST] + [0] * (m - 2)), dtype=torch.int32)  # token 1 is seen by itself alone
    q = fill_new(c, 14, [m, m], par, nh)
    bad = {k: v.clone() for k, v in c.items()}
    for s in range(2):
        pg, at = ref.at(c, s, [int(c["used"][s]) + 1])
        bad["v"][0, pg, :, at] = math.inf
        bad["k"][0, pg, :, at] = math.nan
    off = ref.offsets([m, m]).cuda()
    got = [B.attention_cached(on_gpu(B, x), 0, q.cuda(), (off, m), nh, parent=par.cuda()).cpu() for x in (c, bad)]
    B.poll_status()
    seers = torch.tensor([r for r in range(2 * m) if r % m != 1])
    want, _, tol, _, _ = ref.attend(c, 0, q, ref.offsets([m, m]), nh, par)
    for x in got:
        x = x.double().reshape(2 * m, nh, hd)[seers]
        assert ((x - want[seers]).abs() <= tol[seers]).all()
    assert got[1][[1, m + 1]].isnan().all()


def test_large_scores(B):
    """Scores of several hundred: the running maximum has to carry them."""
    news = [1, 9]
    c = ref.make(15, [500, 90], news, 2, 128, 64, scale=12.0)
    q = fill_new(c, 16, news, None, 4, scale=12.0)
    check_attend(B, c, q, news, 4, None)


def test_infinite_scores_of_seen_slots(B):
    """A seen key with score -inf has weight zero; the others share the whole."""
    c = ref.make(17, [64], [1], 1, 64, 16)
    q = fill_new(c, 18, [1], None, 2)
    q[:] = q.abs() + 1
    pg, at = ref.at(c, 0, [5])
    c["k"][0, pg, :, at] = -math.inf
    g = on_gpu(B, c)
    att = B.attention_cached(g, 0, q.cuda(), 1, 2).cpu().double()
    B.poll_status()
    w = torch.cat([torch.arange(5), torch.arange(6, 65)])
    pages, places = ref.at(c, 0, w)
    k, v = c["k"][0][pages, 0, places].double(), c["v"][0][pages, 0, places].double()
    for j in range(2):
        p = torch.softmax(k @ q[0, 64 * j : 64 * j + 64].double() / 8, 0)
        assert ((att[0, 64 * j : 64 * j + 64] - p @ v).abs() <= 2.0**-7 * (p @ v.abs()) + 1e-4).all()
    assert g.mass.cpu()[0, pg, 0, at] == c["mass"][0, pg, 0, at]


def test_equal_calls_give_equal_bits(B):
    news = [24, 40, 1]
    c = ref.make(19, [1500, 77, 4000], news, 5, 128, 64)
    par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(40 + s, m)], dtype=torch.int32)
    q = fill_new(c, 20, news, par, 20).cuda()
    off = ref.offsets(news).cuda()
    outs = []
    for _ in range(3):
        g = on_gpu(B, c)
        att = B.attention_cached(g, 0, q, (off, 40), 20, parent=par.cuda())
        outs.append((att, g.mass))
    B.poll_status()
    for att, mass in outs[1:]:
        assert same(att, outs[0][0]) and torch.equal(mass, outs[0][1])


@pytest.mark.parametrize("layers,used,budget,recent,sink,page", [
    (1, [20], 16, 4, 0, 16), (2, [100, 16, 0, 33], 32, 8, 2, 16), (1, [700, 65], 64, 64, 4, 64), (1, [700], 64, 100, 4, 32),
    (3, [500, 499], 1, 0, 0, 128), (1, [5000], 4999, 17, 3, 64), (1, [200], 500, 5, 0, 64), (1, [4096], 2048, 0, 0, 128)])
def test_evict_plan_and_move(B, layers, used, budget, recent, sink, page):
    c = ref.make(21, used, [0] * len(used), 3, 64, page, layers=layers, junk=False)
    # ties (a few values only), zeros of both signs, infinities, NaN
    g = ref.gen(22)
    some = torch.tensor([0.0, -0.0, 0.25, 0.25, 1.5, 3e-40, -2.0, math.inf, math.nan, 1e30])
    pick = torch.rand(c["mass"].shape, generator=g) < 0.3
    c["mass"] = torch.where(pick, some[torch.randint(len(some), c["mass"].shape, generator=g)], c["mass"])
    c["pos"] = torch.where(c["pos"] >= 0, c["pos"] + (torch.rand(c["pos"].shape, generator=g) * 3).int(), c["pos"])
    gpu = on_gpu(B, c)
    moves, count = B.kv_evict_plan(gpu, budget, recent, sink=sink)
    B.poll_status()
    want = ref.plan(c, budget, recent, sink)
    mv, n = moves.cpu(), count.cpu()
    for (layer, s, h), lst in want.items():
        assert int(n[layer, s, h]) == len(lst)
        assert [tuple(x) for x in mv[layer, s, h, : len(lst)].tolist()] == lst
        assert (mv[layer, s, h, len(lst) :] == -1).all()
    B.kv_move(gpu, moves, count)
    B.kv_advance(gpu, 0, budget=budget)
    B.poll_status()
    new = ref.move(c, want)
    for name in ("k", "v", "pos"):
        assert same(getattr(gpu, name).cpu(), new[name])
    assert torch.equal(gpu.mass.cpu().view(torch.int32), new["mass"].view(torch.int32))
    assert gpu.used.cpu().tolist() == [min(u, budget) for u in used]


def test_evict_plan_longer_than_shared_memory(B):
    """More slots than keys fit on chip: the same plan, the keys read again."""
    n = 60000
    c = ref.make(23, [n], [0], 1, 64, 128, junk=False)
    c["mass"] = (c["mass"] * 50).round() / 50
    gpu = on_gpu(B, c)
    moves, count = B.kv_evict_plan(gpu, 20000, 3000, sink=2)
    B.poll_status()
    lst = ref.plan(c, 20000, 3000, 2)[0, 0, 0]
    assert int(count) == len(lst) and [tuple(x) for x in moves[0, 0, 0, : len(lst)].tolist()] == lst


@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64), (128, 128)])
def test_accepting_a_branch(B, hd, page):
    """Overlapping lists: places that a token leaves are taken by a later one."""
    c = ref.make(25, [100, 300, 9], [0, 0, 0], 2, hd, page, layers=3, junk=False)
    lists = [[(60 + 2 * i, 60 + i) for i in range(20)], [(200 + i, 7 + i) for i in range(90)], [(3, 3), (5, 4), (8, 5)]]
    moves = torch.full((3, 95, 2), -5, dtype=torch.int32)
    for s, lst in enumerate(lists):
        moves[s, : len(lst)] = torch.tensor(lst)
    gpu = on_gpu(B, c)
    B.kv_move(gpu, moves.cuda(), torch.tensor([len(x) for x in lists], dtype=torch.int32).cuda())
    B.poll_status()
    new = ref.move(c, {(layer, s, h): lists[s] for layer in range(3) for s in range(3) for h in range(2)})
    for name in ("k", "v", "mass", "pos"):
        assert same(getattr(gpu, name).cpu(), new[name])


def test_advance(B):
    c = ref.make(27, [10, 20, 0], [6, 6, 6], 1, 64, 16, junk=False)
    g = on_gpu(B, c)
    seen = c["seen"].tolist()
    B.kv_advance(g, 3)
    assert g.used.tolist() == [13, 23, 3] and g.seen.tolist() == [x + 3 for x in seen]
    B.kv_advance(g, (torch.tensor([0, 2, 2, 5], dtype=torch.int32).cuda(), 3), n_keep=torch.tensor([1, 0, 3], dtype=torch.int32).cuda())
    assert g.used.tolist() == [14, 23, 6]
    B.kv_advance(g, 0, budget=15)
    assert g.used.tolist() == [14, 15, 6] and g.seen.tolist() == [seen[0] + 4, seen[1] + 3, seen[2] + 6]
    B.poll_status()
    B.kv_advance(g, 1, n_keep=torch.tensor([2, 0, 1], dtype=torch.int32).cuda())  # keeps more than there are
    with pytest.raises(B.BitrlError):
        B.poll_status()
    assert g.used.tolist() == [14, 15, 7]


def test_what_is_wrong_on_the_device_is_reported_and_skipped(B):
    def fresh():
        c = ref.make(29, [20, 30], [3, 3], 2, 64, 16, junk=False)
        return c, fill_new(c, 30, [3, 3], None, 4)

    def run(c, q, par=None, off=(0, 3, 6)):
        g = on_gpu(B, c)
        att = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
        B.attention_cached(g, 0, q.cuda(), (torch.tensor(off, dtype=torch.int32).cuda(), 3), 4, att=att,
                           parent=None if par is None else torch.tensor(par, dtype=torch.int32).cuda())
        qkv = torch.ones(6, 8 * 64, dtype=torch.bfloat16, device="cuda")
        q_out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
        B.kv_append(g, 0, qkv, (torch.tensor(off, dtype=torch.int32).cuda(), 3), 4, q_out=q_out,
                    parent=None if par is None else torch.tensor(par, dtype=torch.int32).cuda())
        with pytest.raises(B.BitrlError) as e:
            B.poll_status()
        assert e.value.status == B.ERR_SHAPE
        return att.cpu(), q_out.cpu(), g

    c, q = fresh()
    for par in ([-1, 0, 1, -1, 2, 1], [-1, 0, 1, -1, 1, 0], [-1, 0, 1, -2, 0, -1], [-1, 0, 1, -1, -3, 0]):
        att, q_out, g = run(c, q, par)  # later, own, padding, unknown: the second sequence's tree is wrong
        assert (att[3:] == 5.0).all() and (att[:3] != 5.0).any() and (q_out[3:] == 5.0).all() and (q_out[:3] != 5.0).any()
    for off in ((0, 3, 7), (0, 4, 6), (3, 1, 1), (-1, 1, 3)):
        run(c, q, off=off)
    c["used"][1] = 1 << 20  # more than its pages hold
    att, q_out, _ = run(c, q)
    assert (att[3:] == 5.0).all() and (q_out[3:] == 5.0).all()
    for page in (-1, 10**6):
        c, q = fresh()
        c["page_table"][1] = page
        run(c, q)
        c["used"] += 3
        g = on_gpu(B, c)
        moves, count = B.kv_evict_plan(g, 16, 2)
        with pytest.raises(B.BitrlError):
            B.poll_status()
        assert int(count[0, 1].sum()) == 0
        B.kv_move(g, torch.tensor([[[20, 3]], [[20, 3]]], dtype=torch.int32).cuda(), torch.tensor([1, 1], dtype=torch.int32).cuda())
        with pytest.raises(B.BitrlError):
            B.poll_status()
    c, q = fresh()
    g = on_gpu(B, c)
    for pair in ([4000, 3], [20, -1]):
        B.kv_move(g, torch.tensor([[pair], [[20, 3]]], dtype=torch.int32).cuda(), torch.tensor([1, 0], dtype=torch.int32).cuda())
        with pytest.raises(B.BitrlError):
            B.poll_status()
    B.kv_move(g, torch.tensor([[[20, 3]], [[20, 3]]], dtype=torch.int32).cuda(), torch.tensor([2, -1], dtype=torch.int32).cuda())
    with pytest.raises(B.BitrlError):
        B.poll_status()
    for name in ("k", "v", "mass", "pos"):
        assert same(getattr(g, name).cpu(), c[name])


def test_pools_beyond_32_bit_offsets(B):
    """k and v hold 2^31 elements and more; the sequence's pages lie at both ends."""
    hd, page, nkv, nh = 128, 128, 1, 4
    n_pages = 2**31 // (hd * page) + 5
    g = torch.Generator(device="cuda").manual_seed(31)
    k = torch.zeros(1, n_pages, nkv, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, 7]], dtype=torch.int32, device="cuda")
    small = torch.randn(2, 4, nkv, page, hd, generator=g, device="cuda").to(torch.bfloat16)
    k[0, table[0].long()], v[0, table[0].long()] = small[0], small[1]
    near = (small[0][None].contiguous(), small[1][None].contiguous(), torch.arange(4, dtype=torch.int32, device="cuda")[None])
    qkv = torch.randn(2, (nh + 2) * hd, generator=g, device="cuda").to(torch.bfloat16)
    outs = []
    for kk, vv, tt in ((k, v, table), near):
        used, seen = (torch.tensor([400], dtype=torch.int32, device="cuda") for _ in range(2))
        c = B.KVCache(kk, vv, tt, used, seen, mass=torch.zeros(kk.shape[:4], device="cuda"))
        q = B.kv_append(c, 0, qkv, 2, nh)
        att = B.attention_cached(c, 0, q, 2, nh)
        B.kv_advance(c, 2)
        moves, count = B.kv_evict_plan(c, 150, 4)
        B.kv_move(c, moves, count)
        t = tt[0].long()
        outs.append((q, att, moves, count, c.k[0, t].clone(), c.v[0, t].clone(), c.mass[0, t].clone(), c.pos[0, t].clone()))
    B.poll_status()
    assert int(outs[0][3]) > 0
    for x, y in zip(*outs):
        assert same(x, y)


def test_other_streams_and_captured_graphs(B):
    """One step (append, attend) on a side stream and as a replayed graph gives the bits of the plain call."""
    news, nh = [17, 5], 8
    c = ref.make(33, [90, 200], news, 2, 128, 32)
    off = ref.offsets(news).cuda()
    qkv = torch.randn(22, 12 * 128, generator=ref.gen(34)).to(torch.bfloat16).cuda()

    def step(g, ws, q, att):
        B.kv_append(g, 0, qkv, (off, 17), nh, q_out=q)
        B.attention_cached(g, 0, q, (off, 17), nh, att=att, workspace=ws)

    g0 = on_gpu(B, c)
    ws = torch.empty(B.attention_cached_workspace_bytes(g0, 22, 17, nh), dtype=torch.uint8, device="cuda")
    q, att = (torch.zeros(22, nh * 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    step(g0, ws, q, att)
    want = att.clone()
    side = torch.cuda.Stream()
    g1 = on_gpu(B, c)
    att.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(g1, ws, q, att)
    torch.cuda.current_stream().wait_stream(side)
    assert same(att, want) and torch.equal(g1.mass, g0.mass)
    g2 = on_gpu(B, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(g2, ws, q, att)
    for _ in range(2):
        att.zero_()
        g2.mass.copy_(c["mass"])
        graph.replay()
        torch.cuda.synchronize()
        assert same(att, want) and torch.equal(g2.mass, g0.mass)
    B.poll_status()


def test_the_binding_checks_its_tensors(B):
    c = ref.make(35, [5, 6], [2, 2], 2, 64, 16, junk=False)
    g = on_gpu(B, c)
    q = torch.zeros(4, 4 * 64, dtype=torch.bfloat16, device="cuda")
    qkv = torch.zeros(4, 8 * 64, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    for bad in (lambda: B.attention_cached(g, 0, q[:, :-1], 2, 4), lambda: B.attention_cached(g, 0, q.float(), 2, 4),
                lambda: B.attention_cached(g, 0, q, 3, 4), lambda: B.attention_cached(g, 0, q, (off[:2], 2), 4),
                lambda: B.attention_cached(g, 0, q, 2, 4, parent=off), lambda: B.attention_cached(g, 0, q, 2, 4, att=q[:2]),
                lambda: B.kv_append(g, 0, qkv[:, 64:], 2, 4), lambda: B.kv_append(g, 0, qkv, 2, 5), lambda: B.kv_append(g, 2, qkv, 2, 4),
                lambda: B.kv_append(g, 0, qkv, 2, 4, q_out=q[:3]), lambda: B.kv_evict_plan(g, 0, 1), lambda: B.kv_evict_plan(g, 4, -1),
                lambda: B.kv_move(g, off, off), lambda: B.KVCache(g.k, g.v[:, 1:].contiguous(), g.page_table, g.used, g.seen),
                lambda: B.KVCache(g.k, g.v, g.page_table, g.used[:1], g.seen)):
        with pytest.raises((TypeError, ValueError, B.BitrlError)):
            bad()
    B.poll_status()


def make_encoder(B, L=2, d=512, d_ff=768, nh=8, nkv=2):
    from paper_2604_24273_b200 import inputs

    dims = {"d": d, "d_ff": d_ff, "n_heads": nh, "n_kv_heads": nkv}
    layers = [tuple(B.Linear.from_master(w.cuda()) for w in inputs.encoder_layer_weights(i, 800, dims)) for i in range(L)]
    return B.Encoder(layers, d, d_ff, nh, nkv), layers


@pytest.mark.parametrize("used,news,is_tree", [([0, 0], [6, 9], False), ([30, 7, 0], [1, 1, 1], False), ([50, 3, 90, 8], [12, 40, 0, 31], True)])
def test_encoder_over_a_cache_is_its_operators_in_turn(B, used, news, is_tree):
    from paper_2604_24273_b200 import inputs

    enc, layers = make_encoder(B)
    c = ref.make(41, used, news, 2, 64, 32, layers=3)
    off = ref.offsets(news)
    T = int(off[-1])
    h = inputs.activations(T, 512, 42).cuda()
    par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(50 + s, m, m // 8)], dtype=torch.int32).cuda() if is_tree else None
    states = (off.cuda(), max(news))
    g = on_gpu(B, c)
    out, pooled = enc.forward_cached(h, g, states, parent=par, want_pooled=True)
    assert torch.equal(g.used.cpu(), c["used"])
    B.poll_status()
    x, g2 = h.clone(), on_gpu(B, c)
    for l, (qkv, o, gu, dn) in enumerate(layers):
        xq, a, rs, _ = B.rmsnorm_quant(x)
        q = B.kv_append(g2, l, B.bitlinear_forward_q(qkv, xq, a, rs), states, 8, parent=par)
        att = B.attention_cached(g2, l, q, states, 8, parent=par)
        xq, a, rs, _ = B.rmsnorm_quant(att)
        x = B.bitlinear_forward_q(o, xq, a, rs, residual=x)
        xq, a, rs, _ = B.rmsnorm_quant(x)
        xq, a, rs, _ = B.relu2gate_rmsnorm_quant(B.bitlinear_forward_q(gu, xq, a, rs))
        x = B.bitlinear_forward_q(dn, xq, a, rs, residual=x)
    real = torch.ones(T, dtype=torch.bool, device="cuda") if par is None else par != ref.PAD
    assert same(out[real], x[real])
    for name in ("k", "v", "mass", "pos"):
        assert same(getattr(g, name), getattr(g2, name))
    for s, m in enumerate(news):
        if m and bool(real[int(off[s + 1]) - 1]):
            assert same(pooled[s], out[int(off[s + 1]) - 1])
        elif m == 0:
            assert (pooled[s] == 0).all()


def test_an_episode_step_by_step(B):
    """Used as meant: a prompt, then single tokens, a drafted tree of which one branch is accepted, and evictions, each
    step checked from the cache that the steps before it left."""
    nh, nkv, hd, page, budget, recent = 4, 2, 64, 16, 48, 12
    c = ref.make(51, [0, 0], [0, 0], nkv, hd, page, room=128, junk=True)
    c["seen"][:] = 0
    g = on_gpu(B, c)
    rnd = ref.gen(52)

    def cpu():
        return {n: getattr(g, n).cpu() for n in ("k", "v", "mass", "pos", "page_table", "used", "seen")}

    for step, (news, is_tree) in enumerate([([40, 25], False), ([1, 1], False), ([15, 0], False), ([20, 12], True), ([1, 1], False), ([30, 16], False)]):
        off = ref.offsets(news)
        T = int(off[-1])
        states = (off.cuda(), max(news))
        par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(60 + s, m)], dtype=torch.int32) if is_tree else None
        gp = None if par is None else par.cuda()
        q = B.kv_append(g, 0, torch.randn(T, (nh + 2 * nkv) * hd, generator=rnd).to(torch.bfloat16).cuda(), states, nh, parent=gp)
        before = cpu()
        att = B.attention_cached(g, 0, q, states, nh, parent=gp)
        want, add, tol, mtol, _ = ref.attend(before, 0, q.cpu(), off, nh, par)
        assert ((att.cpu().double().reshape(T, nh, hd) - want).abs() <= tol).all(), step
        assert ((g.mass.cpu()[0].double() - before["mass"][0].double() - add).abs() <= mtol + 2.0**-23 * (before["mass"][0].double() + add)).all(), step
        if is_tree:
            paths = [ref.above(par[int(off[s]) : int(off[s + 1])].tolist(), m - 1)[::-1] for s, m in enumerate(news)]
            moves = torch.zeros(2, 20, 2, dtype=torch.int32)
            for s, path in enumerate(paths):
                for i, j in enumerate(path):
                    moves[s, i] = torch.tensor([int(before["used"][s]) + j, int(before["used"][s]) + i])
            n = torch.tensor([len(p) for p in paths], dtype=torch.int32)
            B.kv_move(g, moves.cuda(), n.cuda())
            B.kv_advance(g, states, n_keep=n.cuda())
        else:
            B.kv_advance(g, states)
        before = cpu()
        moves, count = B.kv_evict_plan(g, budget, recent, sink=2)
        B.kv_move(g, moves, count)
        B.kv_advance(g, 0, budget=budget)
        after, lists = cpu(), ref.plan(before, budget, recent, 2)
        new = ref.move(before, lists)
        for name in ("k", "v", "pos"):
            assert same(after[name], new[name]), (step, name)
        assert (after["used"] <= budget).all()
        for s in range(2):
            pg, at = ref.at(after, s, range(int(after["used"][s])))
            for h in range(nkv):  # no position twice, the latest ones all there
                p = after["pos"][0][pg, h, at].tolist()
                assert len(set(p)) == len(p) and set(range(max(0, int(after["seen"][s]) - recent), int(after["seen"][s]))) <= set(p)
    B.poll_status()


def dense(c, q, off, nh, parent=None):
    """att and added mass in 64 bits on the GPU, one (sequence, kv head) at a time, with the tolerances of ref.attend."""
    nkv, hd = c["k"].shape[2], c["k"].shape[4]
    rep = nh // nkv
    att, tol = (torch.zeros(q.shape[0], nh, hd, dtype=torch.float64, device="cuda") for _ in range(2))
    add, mtol = (torch.zeros(c["mass"].shape[1:], dtype=torch.float64, device="cuda") for _ in range(2))
    k0, v0, table, q = c["k"][0].cuda(), c["v"][0].cuda(), c["page_table"].cuda(), q.cuda()
    page = k0.shape[2]
    for s in range(len(off) - 1):
        t0, m, u = int(off[s]), int(off[s + 1] - off[s]), int(c["used"][s])
        if m == 0:
            continue
        slot = torch.arange(u + m, device="cuda")
        pg, at = table[s, slot // page].long(), slot % page
        sees = torch.ones(m, u + m, dtype=torch.bool, device="cuda").tril(u)
        if parent is not None:
            sees[:, u:] = False
            for i in range(m):
                chain = ref.above(parent[t0 : t0 + m].tolist(), i)
                sees[i, : u] = bool(chain)
                sees[i, [u + j for j in chain]] = True
        for h in range(nkv):
            k, v = k0[pg, h, at].double(), v0[pg, h, at].double()
            v = torch.where(sees.any(0)[:, None], v, 0.0)
            k = torch.where(sees.any(0)[:, None], k, 0.0)
            x = q[t0 : t0 + m].double().reshape(m, nh, hd)[:, h * rep : (h + 1) * rep].transpose(0, 1)
            sc = (x @ k.T / hd**0.5).masked_fill(~sees, -math.inf)
            p = torch.where(sees, torch.softmax(sc, 2), 0.0)
            d = 2 * hd * 2.0**-23 * float((x.abs() @ k.abs().T).max()) / hd**0.5 + 2.0**-21 + (u + m) * 2.0**-23
            o = p @ v
            att[t0 : t0 + m, h * rep : (h + 1) * rep] = o.transpose(0, 1)
            tol[t0 : t0 + m, h * rep : (h + 1) * rep] = (2.0**-8 * o.abs() + (2.0**-8 + d) * (p @ v.abs())).transpose(0, 1)
            add[pg, h, at] += p.sum((0, 1))
            mtol[pg, h, at] += p.sum((0, 1)) * (d + m * rep * 2.0**-23)
    return att, add, tol, mtol


@pytest.mark.parametrize("nh,nkv,hd,page,used,news,is_tree", [
    (20, 5, 128, 64, [4100], [1500], False), (7, 1, 64, 32, [900, 0, 3000], [700, 333, 40], False), (4, 4, 128, 128, [0], [2100], False),
    (20, 5, 128, 64, [3000 + 41 * i for i in range(9)], [15 + 3 * i for i in range(9)], True),
    (12, 4, 64, 16, [10 * i for i in range(150)], [7 + i % 30 for i in range(150)], False),
    (20, 5, 128, 64, [9000, 100, 5000, 1], [1, 1, 1, 1], False), (16, 4, 64, 16, [33 * i for i in range(200)], [1 + i % 3 for i in range(200)], True),
    (64, 1, 128, 64, [1000], [130], False), (33, 1, 64, 64, [70, 500], [50, 3], True), (3, 1, 128, 16, [20000], [20], False),
    (8, 1, 128, 64, [60000], [1], False)])
def test_long_and_many(B, nh, nkv, hd, page, used, news, is_tree):
    """Items cut between thread blocks, many short sequences, groups that do not divide a tile."""
    c = ref.make(71, used, news, nkv, hd, page)
    par = torch.tensor([p for s, m in enumerate(news) for p in ref.tree(80 + s, m, m // 9)], dtype=torch.int32) if is_tree else None
    q = fill_new(c, 72, news, par, nh)
    off = ref.offsets(news)
    g = on_gpu(B, c)
    att = B.attention_cached(g, 0, q.cuda(), (off.cuda(), max(news)), nh, parent=None if par is None else par.cuda())
    B.poll_status()
    want, add, tol, mtol = dense(c, q, off, nh, par)
    err = (att.double().reshape(want.shape) - want).abs() - tol
    assert not att.isnan().any() and err.max() <= 0, float(err.max())
    m0 = c["mass"][0].double().cuda()
    bad = (g.mass[0].double() - m0 - add).abs() - (mtol + 2.0**-23 * (m0 + add))
    assert bad.max() <= 0, float(bad.max())
