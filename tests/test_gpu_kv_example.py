"""The serving example: prompts in chunks, tokens by a CUDA graph, an index over the keys."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("batch,prompt,chunk,steps", [(3, 200, 64, 8), (1, 1, 64, 20), (2, 2500, 1000, 3)])
def test_serving_example(cuda_ok, batch, prompt, chunk, steps):
    import kv_serve

    r = kv_serve.run(batch, prompt, chunk, steps)
    lengths = [max(1, prompt * (b + 1) // batch) + steps for b in range(batch)]
    assert r["length"] == lengths
    # a code is off by half of amax / 127, some 0.8% of a value's own size; logits of size 1 then move the
    # weights as much, and a step's two layers add at most 4% of what attention adds to the state
    assert r["error"] < 0.1
    keys = r["keys"].double()
    assert tuple(keys.shape) == (lengths[-1], 2, 64) and torch.isfinite(keys).all()
    for h, (C, assign, wcss) in enumerate(r["fits"]):
        d2 = ((keys[:, h] - C.double()[assign.long()]) ** 2).sum()
        assert wcss == pytest.approx(float(d2), rel=1e-4)
        assert wcss <= float(((keys[:, h] - keys[:, h].mean(0)) ** 2).sum()) * (1 + 1e-4)


def test_capturing_the_step_leaves_the_caches_as_they_were(cuda_ok):
    import kv_serve

    lengths = [20, 33, 41]  # last blocks of 4, 1 and 9 tokens
    server = kv_serve.Server(3, 60)
    g = torch.Generator(device="cuda").manual_seed(5)
    server.prompts([torch.randn(n, 256, generator=g, device="cuda").to(torch.bfloat16) for n in lengths], 16)
    was = [[t.clone() for t in (lay.cache.k, lay.cache.v, lay.cache.scales)] for lay in server.layers]
    table = server.table.clone()
    server.capture()
    torch.cuda.synchronize()
    assert server.start.tolist() == lengths and torch.equal(server.table, table)
    for lay, held in zip(server.layers, was):
        for t, w in zip((lay.cache.k, lay.cache.v, lay.cache.scales), held):
            assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))
