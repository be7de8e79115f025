"""Lists and plans longer than one pass of a thread block takes, and calls whose sequences all bring the same number of tokens."""
import pytest
import torch

import kv_cases as ref
from test_gpu_kv_cache import check_attend, fill_new, on_gpu, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_24273_b200 import bitrl

    bitrl.lib()
    torch.cuda.set_device(0)
    return bitrl


@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
def test_overlapping_lists_of_several_batches(B, hd, page):
    """Sources that earlier destinations of the same list reach, 256 moves a batch; beside lists whose two sides lie apart."""
    c = ref.make(501, [1000, 1000, 1000, 300], [0] * 4, 2, hd, page, layers=2, junk=False)
    lists = [[(7 + i, i) for i in range(900)], [(500 + i, i) for i in range(400)], [(2 * i + 1, i) for i in range(499)], [(i, i) for i in range(300)]]
    moves = torch.full((4, 950, 2), -5, dtype=torch.int32)
    for s, lst in enumerate(lists):
        moves[s, : len(lst)] = torch.tensor(lst)
    gpu = on_gpu(B, c)
    B.kv_move(gpu, moves.cuda(), torch.tensor([len(x) for x in lists], dtype=torch.int32).cuda())
    B.poll_status()
    new = ref.move(c, {(layer, s, h): lists[s] for layer in range(2) for s in range(4) for h in range(2)})
    for name in ("k", "v", "mass", "pos"):
        assert same(getattr(gpu, name).cpu(), new[name]), name


@pytest.mark.parametrize("n,budget,recent,sink", [(60000, 20000, 30000, 2), (60000, 100, 59000, 0), (51204, 51200, 51204, 0), (60000, 59999, 10, 60000)])
def test_plans_beyond_shared_memory_whose_protected_slots_compete(B, n, budget, recent, sink):
    c = ref.make(503, [n, 40], [0, 0], 1, 64, 128, junk=False)
    c["seen"] = c["used"].clone()
    c["mass"] = (c["mass"] * 50).round() / 50
    gpu = on_gpu(B, c)
    moves, count = B.kv_evict_plan(gpu, budget, recent, sink=sink)
    B.poll_status()
    want = ref.plan(c, budget, recent, sink)
    for s in range(2):
        lst = want[0, s, 0]
        assert int(count[0, s, 0]) == len(lst)
        if lst:
            assert torch.equal(moves[0, s, 0, : len(lst)].cpu(), torch.tensor(lst, dtype=torch.int32))


@pytest.mark.parametrize("nh,nkv,hd,page,m,is_tree", [(4, 2, 64, 16, 3, True), (8, 2, 128, 64, 30, True), (20, 5, 128, 32, 40, False),
                                                      (8, 2, 64, 64, 150, False), (8, 1, 64, 16, 200, True)])
def test_the_same_number_of_tokens_everywhere(B, nh, nkv, hd, page, m, is_tree):
    """No offsets: rows s * m .. s * m + m - 1 are sequence s's, in append and attention alike."""
    used = [70, 0, 129]
    c = ref.make(505, used, [m] * 3, nkv, hd, page)
    par = torch.tensor([p for s in range(3) for p in ref.tree(510 + s, m, m // 8)], dtype=torch.int32) if is_tree else None
    q = fill_new(c, 506, [m] * 3, par, nh)
    check_attend(B, c, q, [m] * 3, nh, par, behind=0, states=m)
    qkv = torch.randn(3 * m, (nh + 2 * nkv) * hd, generator=ref.gen(507)).to(torch.bfloat16).cuda()
    outs = []
    for states in (m, (ref.offsets([m] * 3).cuda(), m)):
        g = on_gpu(B, c)
        q_out = B.kv_append(g, 0, qkv, states, nh, parent=None if par is None else par.cuda())
        att = B.attention_cached(g, 0, q_out, states, nh, parent=None if par is None else par.cuda())
        outs.append((q_out, att, g.k, g.v, g.mass, g.pos))
    B.poll_status()
    for x, y in zip(*outs):
        assert same(x, y)


@pytest.mark.parametrize("nh,nkv,hd,page,news", [(4, 2, 64, 16, [2, 1, 0]), (8, 2, 128, 64, [30, 3, 41]), (8, 1, 128, 128, [150, 40, 300])])
def test_a_page_table_with_room_for_half_a_million_slots(B, nh, nkv, hd, page, news):
    """As many entries as a page table may have, of which few name a page: the others are never read as pages."""
    used = [70, 5, 400]
    c = ref.make(521, used, news, nkv, hd, page)
    wide = torch.full((3, B.KV_MAX_SLOTS // page), -1, dtype=torch.int32)
    wide[:, : c["page_table"].shape[1]] = c["page_table"]
    for s in range(3):
        wide[s, -(-(used[s] + news[s]) // page) :] = -1
    c["page_table"] = wide
    q = fill_new(c, 522, news, None, nh)
    check_attend(B, c, q, news, nh, None)
    g = on_gpu(B, c)
    off = ref.offsets(news)
    B.kv_append(g, 0, torch.randn(int(off[-1]), (nh + 2 * nkv) * hd, generator=ref.gen(523)).to(torch.bfloat16).cuda(), (off.cuda(), max(news)), nh)
    B.kv_advance(g, (off.cuda(), max(news)))
    now = {n: getattr(g, n).cpu() for n in ("k", "v", "mass", "pos", "page_table", "used", "seen")}
    moves, count = B.kv_evict_plan(g, 64, 20, sink=2)
    B.kv_move(g, moves, count)
    B.poll_status()
    want = ref.plan(now, 64, 20, 2)
    new = ref.move(now, want)
    for (layer, s, h), lst in want.items():
        assert int(count[layer, s, h]) == len(lst)
    for name in ("k", "v", "mass", "pos"):
        assert same(getattr(g, name).cpu(), new[name]), name
