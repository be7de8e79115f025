"""Where the binding puts a gradient that it allocates."""
import pytest
import torch

from test_gpu_token_loss import B, ints  # noqa: F401 (B: the fixture)

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,V,ld,offset", [(6, 1001, 1001, 0), (6, 1001, 1001, 1001), (6, 1001, 1024, 0), (6, 1001, 1500, 0), (6, 1001, 1509, 7), (6, 1000, 5003, 20),
                                              (1, 1001, 1001, 1001), (1, 700, 4000, 13), (5, 3, 3, 1), (5, 1, 300, 2), (0, 50, 50, 0)])
def test_new_gradient_lies_as_the_logits(B, rows, V, ld, offset, dtype):
    """Every row at the place of its logits within 32 bytes, so that it is written in whole vectors; no row much longer than V."""
    store = torch.randn(offset + 6 * ld, device="cuda").to(dtype)
    z = torch.as_strided(store, (rows, V), (ld, 1), offset)
    tokens, one = ints([t % V for t in range(rows)]), torch.ones(rows, device="cuda")
    f = B.token_logprobs(z, tokens)
    ids, values = tokens[:, None].contiguous(), torch.zeros(rows, 1, device="cuda")
    for call in (lambda d: B.token_logprobs_backward(z, tokens, f["stats"], dlogp=one, dlogits=d), lambda d: B.ppo_token_loss(z, tokens, f["logp"], one, dlogits=d)["dlogits"],
                 lambda d: B.distill_topk(z, ids, values, dlogits=d)["dlogits"]):
        got = call(None)
        want = call(torch.empty(rows, V, dtype=dtype, device="cuda"))
        assert got.shape == z.shape and got.stride(1) == 1 and (rows < 2 or V <= got.stride(0) < V + 128) and torch.equal(got, want)
        for t in range(rows):
            assert (got[t].data_ptr() - z[t].data_ptr()) % 32 == 0
    B.poll_status()
