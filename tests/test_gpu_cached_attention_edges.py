"""CachedAttention at its ends: prompts without rows, sequences without tokens."""
import numpy as np
import pytest
import torch

from paper_2602_22592_amd import binding as pq
from paper_2602_22592_amd import workloads as wl
from paper_2602_22592_amd.stack import CachedAttention

pytestmark = pytest.mark.gpu
t32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32).cuda()


@pytest.mark.parametrize("kind", [pq.PQ_KV_INT8, pq.PQ_KV_BF16])
def test_a_prompt_without_rows(kind):
    """It returns no rows and leaves the cache alone; one that has rows follows, for one of two sequences."""
    d, H, Hk = 256, 4, 2
    rng = np.random.default_rng(3)
    W = {"W" + n: torch.from_numpy(wl.normal(rng, (d if n in "qo" else Hk * 64, d), 0.06, True)).cuda().bfloat16() for n in "qkvo"}
    layer = CachedAttention(W, H, Hk, n_pages=4, n_seqs=2, max_pages=2, page_tokens=16, kv_kind=kind)
    layer.cache.fill_(255)
    table = t32([[0, 1], [2, 3]])
    out = layer.prompt(torch.empty((0, d), dtype=torch.bfloat16, device="cuda"), t32([0, 0]), table, t32([0, 0, 0]))
    assert out.shape == (0, d) and out.dtype is torch.bfloat16 and (layer.cache == 255).all()
    x = torch.from_numpy(wl.activations(rng, 20, d, bf16=True)).cuda().bfloat16()
    out = layer.prompt(x, t32([0, 20]), table, t32([0, 0, 20]))
    assert torch.isfinite(out.float()).all()
    assert (layer.cache.view(4, -1)[:2] == 255).all() and not (layer.cache.view(4, -1)[2:] == 255).all()
