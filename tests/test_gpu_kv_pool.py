"""What the encoder over a cache hands out as a sequence's latent: its last new token that is one."""
import pytest
import torch

import kv_cases as ref
from test_gpu_kv_cache import make_encoder, on_gpu, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_24273_b200 import bitrl

    bitrl.lib()
    torch.cuda.set_device(0)
    return bitrl


def forward(B, enc, used, trees, h, parent=True):
    news = [len(t) for t in trees]
    c = ref.make(301, used, news, 2, 64, 32, layers=2)
    par = torch.tensor([p for t in trees for p in t], dtype=torch.int32).cuda() if parent else None
    pooled = torch.full((len(used), 512), 9.0, dtype=torch.bfloat16, device="cuda")
    out, pooled = enc.forward_cached(h, on_gpu(B, c), (ref.offsets(news).cuda(), max(news)), parent=par, pooled=pooled)
    return out, pooled, ref.offsets(news).tolist()


TREES = [[-1, 0, 0, 1], [-1, 0, -2, -2], [-2, -2], [], [-1, -2, 0, 2, -2, 0, -2], ref.tree(302, 200, 30), [-2] * 40 + [-1] + [-2] * 150]


def test_the_last_token_of_a_tree(B):
    from paper_2604_24273_b200 import inputs

    enc, _ = make_encoder(B)
    h = inputs.activations(sum(len(t) for t in TREES), 512, 303).cuda()
    out, pooled, off = forward(B, enc, [10, 0, 33, 5, 64, 100, 7], TREES, h)
    B.poll_status()
    for s, t in enumerate(TREES):
        real = [i for i, p in enumerate(t) if p != ref.PAD]
        if real:
            assert same(pooled[s], out[off[s] + real[-1]]), s
        else:
            assert (pooled[s] == 9.0).all(), s


def test_the_last_token_without_a_tree(B):
    from paper_2604_24273_b200 import inputs

    enc, _ = make_encoder(B)
    h = inputs.activations(sum(len(t) for t in TREES), 512, 304).cuda()
    out, pooled, off = forward(B, enc, [10, 0, 33, 5, 64, 100, 7], TREES, h, parent=False)
    B.poll_status()
    for s, t in enumerate(TREES):
        assert same(pooled[s], out[off[s + 1] - 1]) if t else (pooled[s] == 9.0).all(), s


def test_a_sequence_that_is_skipped_is_not_pooled(B):
    from paper_2604_24273_b200 import inputs

    enc, _ = make_encoder(B)
    trees = [[-1, 0, 1], [-1, 0, 5], [-1, 0]]  # the second one's last token continues none before it
    h = inputs.activations(8, 512, 305).cuda()
    out, pooled, off = forward(B, enc, [10, 20, 3], trees, h)
    with pytest.raises(B.BitrlError) as e:
        B.poll_status()
    assert e.value.status == B.ERR_SHAPE
    assert same(pooled[0], out[2]) and (pooled[1] == 9.0).all() and same(pooled[2], out[7])
