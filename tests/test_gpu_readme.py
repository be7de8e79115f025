"""The sequence of calls that the README shows is one that runs."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_episode_of_the_readme():
    from paper_2604_24273_b200 import bitrl, inputs
    from test_gpu_kv_cache import make_encoder

    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        blocks = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "KVCache" in b]
    assert len(blocks) == 1
    enc, _ = make_encoder(bitrl)
    news = [300, 120]
    names = dict(bitrl=bitrl, enc=enc, n_layers=2, n_seq=2, max_tokens=400, n_kv_heads=2, head_dim=64, budget=280, max_new=300,
                 h_in=inputs.activations(420, 512, 401).cuda(), state_off=torch.tensor([0, 300, 420], dtype=torch.int32, device="cuda"))
    exec(compile(blocks[0], "README.md", "exec"), names)
    bitrl.poll_status()
    h, last, cache = names["h"], names["last"], names["cache"]
    assert h.shape == (420, 512) and torch.equal(last, h[[299, 419]])
    assert cache.used.tolist() == [280, 120] and cache.seen.tolist() == news
    assert (names["count"][:, 0] > 0).all() and (names["count"][:, 1] == 0).all()
