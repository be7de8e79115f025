"""The encoder over a cache, step after step without a pause: every launch overlaps its neighbours, and each gives the same bits."""
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


@pytest.mark.parametrize("n_seq,m,used,mass", [(64, 32, 1000, True), (64, 32, 1000, False), (40, 50, 300, True), (3, 300, 700, True), (64, 1, 500, True)])
def test_many_steps_in_a_row(B, n_seq, m, used, mass):
    from paper_2604_24273_b200 import inputs

    enc, _ = make_encoder(B, L=4)
    c = ref.make(601, [used] * n_seq, [m] * n_seq, 2, 64, 64, layers=4)
    g = on_gpu(B, c)
    h = inputs.activations(n_seq * m, 512, 602).cuda()
    out, first = torch.empty_like(h), torch.empty_like(h)
    ws = torch.empty(enc.cached_workspace_bytes(g, n_seq * m, m), dtype=torch.uint8, device="cuda")
    enc.forward_cached(h, g, m, accumulate_mass=mass, h_out=first, workspace=ws)
    once = g.mass.clone()
    B.poll_status()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        enc.forward_cached(h, g, m, accumulate_mass=mass, h_out=out, workspace=ws)
    for step in (lambda: enc.forward_cached(h, g, m, accumulate_mass=mass, h_out=out, workspace=ws), graph.replay):
        for _ in range(10):
            for _ in range(20):
                step()
            B.poll_status()  # no wait has run out
            assert same(out, first)
    g.mass.copy_(c["mass"])
    graph.replay()
    assert torch.equal(g.mass, once)
    B.poll_status()
