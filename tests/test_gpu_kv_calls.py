"""Calls on the paged key/value cache that the documentation allows and ordinary use seldom makes."""
import math

import pytest
import torch

import kv_cases as ref
from test_gpu_kv_cache import dense, fill_new, on_gpu, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_24273_b200 import bitrl

    bitrl.lib()
    torch.cuda.set_device(0)
    return bitrl


def check(att, mass, c, q, off, nh, parent=None):
    want, add, tol, mtol = dense(c, q, off, nh, parent)
    err = (att.double().reshape(want.shape) - want).abs() - tol
    assert not att.isnan().any() and err.max() <= 0, float(err.max())
    if mass is not None:
        m0 = c["mass"][0].double().cuda()
        assert ((mass[0].double() - m0 - add).abs() - (mtol + 2.0**-23 * (m0 + add))).max() <= 0


# (query heads, kv heads, head dim, page, slots in use, new tokens): one for each kernel that a call can take
FORMS = [(4, 2, 128, 32, [300, 41], [2, 1]), (6, 1, 64, 16, [70, 33], [2, 2]), (8, 2, 128, 64, [500, 90], [25, 40]), (8, 2, 64, 16, [130, 300], [90, 150])]


@pytest.mark.parametrize("nh,nkv,hd,page,used,news", FORMS)
def test_shared_pages_are_read(B, nh, nkv, hd, page, used, news):
    """Two sequences with the same history read the same pages; no weights are accumulated."""
    used = [used[0], used[0]]
    c = ref.make(101, used, news, nkv, hd, page)
    full = used[0] // page
    c["page_table"][1, :full] = c["page_table"][0, :full]
    rest = torch.arange(full * page, used[0])
    if len(rest):
        (p0, a0), (p1, a1) = ref.at(c, 0, rest), ref.at(c, 1, rest)
        c["k"][0, p1, :, a1], c["v"][0, p1, :, a1] = c["k"][0, p0, :, a0], c["v"][0, p0, :, a0]
    q = fill_new(c, 102, news, None, nh)
    off = ref.offsets(news)
    g = B.KVCache(*(c[n].cuda() for n in ("k", "v", "page_table", "used", "seen")))
    att = B.attention_cached(g, 0, q.cuda(), (off.cuda(), max(news)), nh, accumulate_mass=False)
    B.poll_status()
    check(att, None, c, q, off, nh)
    with pytest.raises(B.BitrlError) as e:
        B.attention_cached(g, 0, q.cuda(), (off.cuda(), max(news)), nh)
    assert e.value.status == B.ERR_NULL


@pytest.mark.parametrize("nh,nkv,hd,page,used,news", FORMS)
def test_addresses_that_are_multiples_of_16_only(B, nh, nkv, hd, page, used, news):
    c = ref.make(103, used, news, nkv, hd, page)
    q = fill_new(c, 104, news, None, nh)
    off = ref.offsets(news)
    g = on_gpu(B, c)
    T = q.shape[0]
    place = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device="cuda")
    att = place[8:].view(T, -1)
    qs = torch.empty(q.numel() + 8, dtype=torch.bfloat16, device="cuda")[8:].view(T, -1).copy_(q)
    ws = torch.empty(B.attention_cached_workspace_bytes(g, T, max(news), nh) + 16, dtype=torch.uint8, device="cuda")[16:]
    assert att.data_ptr() % 32 == 16 and ws.data_ptr() % 32 == 16
    B.attention_cached(g, 0, qs, (off.cuda(), max(news)), nh, att=att, workspace=ws)
    B.poll_status()
    check(att, g.mass, c, q, off, nh)
    assert (place[:8] == 0).all()


@pytest.mark.parametrize("nh,nkv,hd,page,used,news", FORMS)
def test_what_is_wrong_is_skipped_by_every_kernel(B, nh, nkv, hd, page, used, news):
    """A bad tree, bad offsets, a bad page: the other sequence's results stay what they are."""
    c = ref.make(105, used, news, nkv, hd, page)
    q = fill_new(c, 106, news, None, nh)
    off = ref.offsets(news)
    T = q.shape[0]
    chain = torch.tensor([i - 1 for m in news for i in range(m)], dtype=torch.int32)
    tree = max(news) <= B.TREE_MAX_TOKENS

    def run(cache, off, parent=None):
        g = on_gpu(B, cache)
        att = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device="cuda")
        B.attention_cached(g, 0, q.cuda(), (off.cuda(), max(news)), nh, att=att, parent=None if parent is None else parent.cuda())
        return att, g

    good, gg = run(c, off)
    B.poll_status()
    n0 = news[0]
    bad_calls = [(c, torch.tensor([0, n0, T + 1], dtype=torch.int32), None)]
    huge = {**c, "used": torch.tensor([used[0], 1 << 20], dtype=torch.int32)}
    bad_calls.append((huge, off, None))
    if tree:
        wrong = chain.clone()
        wrong[n0 + (1 if news[1] > 1 else 0)] = 5000
        bad_calls.append((c, off, wrong))
        whole, _ = run(c, off, chain)
        assert ((whole.double() - good.double()).abs() <= 2.0**-6 * (1 + good.double().abs())).all()
    for cache, o, parent in bad_calls:
        att, g = run(cache, o, parent)
        with pytest.raises(B.BitrlError) as e:
            B.poll_status()
        assert e.value.status == B.ERR_SHAPE
        assert ((att[:n0].double() - good[:n0].double()).abs() <= 2.0**-6 * (1 + good[:n0].double().abs())).all() and (att[n0:] == 5.0).all()
        pg, at = ref.at(c, 1, range(used[1]))
        assert torch.equal(g.mass.cpu()[0][pg, :, at], c["mass"][0][pg, :, at])  # the skipped sequence received nothing
    broken = {**c, "page_table": c["page_table"].clone()}
    broken["page_table"][1, 0] = -3
    att, g = run(broken, off)
    with pytest.raises(B.BitrlError):
        B.poll_status()
    assert ((att[:n0].double() - good[:n0].double()).abs() <= 2.0**-6 * (1 + good[:n0].double().abs())).all()
    pg, at = ref.at(c, 0, range(used[0] + n0))
    assert torch.allclose(g.mass.cpu()[0][pg, :, at], gg.mass.cpu()[0][pg, :, at], rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("nh,nkv,hd,page,used,news", FORMS)
def test_not_a_number_reaches_those_who_see_it(B, nh, nkv, hd, page, used, news):
    """NaN in a key that tokens see, in a value that they see, in one token's query: that and no more."""
    for what in ("key", "value", "query"):
        c = ref.make(107, used, news, nkv, hd, page)
        q = fill_new(c, 108, news, None, nh)
        off = ref.offsets(news)
        rep = nh // nkv
        if what == "query":
            q[0, :hd] = math.nan
        else:
            pg, at = ref.at(c, 1, [used[1]])  # the first new token of the second sequence: seen by all its tokens
            c[what[0]][0, pg, 0, at] = math.nan
        g = on_gpu(B, c)
        att = B.attention_cached(g, 0, q.cuda(), (off.cuda(), max(news)), nh).cpu().reshape(q.shape[0], nh, hd)
        B.poll_status()
        bad = att.isnan().any(2)
        want = torch.zeros_like(bad)
        if what == "query":
            want[0, 0] = True
        else:
            want[news[0] :, :rep] = True
        assert torch.equal(bad, want), what
        mass_bad = g.mass.cpu()[0].isnan()
        expect = torch.zeros_like(mass_bad)
        if what == "query":
            pg, at = ref.at(c, 0, range(used[0] + 1))
            expect[pg, 0, at] = True
        elif what == "key":
            pg, at = ref.at(c, 1, range(used[1] + news[1]))
            expect[pg, 0, at] = True
        assert torch.equal(mass_bad, expect), what


def test_two_graphs_share_a_workspace(B):
    """Replayed one after the other, in any order, they give what plain calls give."""
    nh = 8
    sides = []
    for seed, used, news in ((111, [700, 20], [30, 12]), (112, [64, 900], [1, 2])):
        c = ref.make(seed, used, news, 2, 128, 64)
        q = fill_new(c, seed + 10, news, None, nh).cuda()
        off = ref.offsets(news).cuda()
        want = B.attention_cached(on_gpu(B, c), 0, q, (off, max(news)), nh)
        g = on_gpu(B, c)
        sides.append((c, g, q, off, max(news), torch.zeros_like(q), want))
    ws = torch.empty(max(B.attention_cached_workspace_bytes(g, q.shape[0], m, nh) for _, g, q, _, m, _, _ in sides), dtype=torch.uint8, device="cuda")
    graphs = []
    for _, g, q, off, m, att, _ in sides:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.attention_cached(g, 0, q, (off, m), nh, att=att, workspace=ws)
        graphs.append(graph)
    for order in ((0, 1, 0), (1, 1, 0)):
        for i in order:
            sides[i][5].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in set(order):
            assert same(sides[i][5], sides[i][6])
    B.poll_status()


def test_two_streams_at_once(B):
    nh = 20
    jobs = []
    for seed, used, news in ((121, [3000] * 4, [30] * 4), (122, [2500] * 6, [1] * 6), (123, [800] * 3, [200] * 3)):
        c = ref.make(seed, used, news, 5, 128, 64)
        q = fill_new(c, seed + 10, news, None, nh).cuda()
        off = ref.offsets(news).cuda()
        want = B.attention_cached(on_gpu(B, c), 0, q, (off, max(news)), nh)
        g = on_gpu(B, c)
        ws = torch.empty(B.attention_cached_workspace_bytes(g, q.shape[0], max(news), nh), dtype=torch.uint8, device="cuda")
        jobs.append((g, q, off, max(news), ws, torch.zeros_like(q), want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for g, q, off, m, ws, att, _, st in jobs:
            with torch.cuda.stream(st):
                B.attention_cached(g, 0, q, (off, m), nh, att=att, workspace=ws)
    torch.cuda.synchronize()
    for _, _, _, _, _, att, want, _ in jobs:
        assert same(att, want)
    B.poll_status()


def test_a_fresh_cache_and_an_empty_batch(B):
    cache = B.KVCache.empty(2, 3, 100, 2, 64, page_tokens=16)
    assert cache.max_pages == 7 and cache.page_tokens == 16 and int(cache.used.sum()) == 0
    qkv = torch.randn(6, 8 * 64, generator=ref.gen(131)).to(torch.bfloat16).cuda()
    off = torch.tensor([0, 4, 4, 6], dtype=torch.int32, device="cuda")
    q = B.kv_append(cache, 1, qkv, (off, 4), 4)
    att = B.attention_cached(cache, 1, q, (off, 4), 4)
    B.kv_advance(cache, (off, 4))
    none = torch.zeros(4, dtype=torch.int32, device="cuda")
    empty = torch.zeros(0, 4 * 64, dtype=torch.bfloat16, device="cuda")
    assert B.attention_cached(cache, 1, empty, (none, 4), 4).shape == (0, 256)
    before = cache.mass.clone()
    B.attention_cached(cache, 1, q, (torch.zeros(4, dtype=torch.int32, device="cuda"), 4), 4)  # rows, but nobody's
    B.poll_status()
    assert torch.equal(cache.mass, before) and cache.used.tolist() == [4, 0, 2] and cache.seen.tolist() == [4, 0, 2]
    # each query head hands out weight 1 per token
    assert torch.allclose(cache.mass[1].sum(), torch.tensor(6.0 * 4, device="cuda"), rtol=1e-5) and not cache.mass[0].any()
    assert not att.isnan().any()


def test_many_sequences_of_nothing_much(B):
    """More sequences than threads look them up; most have no new token."""
    n_seq = 1500
    used = [i % 50 for i in range(n_seq)]
    for top in (2, 9):
        news = [(i // 3) % (top + 1) if i % 3 == 0 else 0 for i in range(n_seq)]
        c = ref.make(141, used, news, 1, 64, 16)
        q = fill_new(c, 142, news, None, 5)
        off = ref.offsets(news)
        g = on_gpu(B, c)
        att = B.attention_cached(g, 0, q.cuda(), (off.cuda(), top), 5)
        B.poll_status()
        check(att, g.mass, c, q, off, 5)


def test_counts_that_cannot_be(B):
    """Device-side refusals of the counters and of a list longer than a sequence has slots."""
    c = ref.make(151, [20, 30], [1, 1], 2, 64, 16)
    g = on_gpu(B, c)
    room = c["page_table"].shape[1] * 16
    moves = torch.zeros(2, room + 5, 2, dtype=torch.int32, device="cuda")
    before = [x.clone() for x in (g.k, g.v, g.mass, g.pos)]
    B.kv_move(g, moves, torch.tensor([room + 1, 0], dtype=torch.int32, device="cuda"))
    with pytest.raises(B.BitrlError):
        B.poll_status()
    assert all(same(x, y) for x, y in zip(before, (g.k, g.v, g.mass, g.pos)))
    for name in ("used", "seen"):
        g = on_gpu(B, c)
        getattr(g, name)[0] = -1
        B.kv_advance(g, 1)
        with pytest.raises(B.BitrlError):
            B.poll_status()
        assert int(getattr(g, name)[0]) == -1
        other = "used" if name == "seen" else "seen"
        assert int(getattr(g, other)[0]) == int(c[other][0]) and int(g.used[1]) == 31
