"""Equal calls give equal bits."""
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
