"""Recorded graphs whose caller has let go of what they read."""
import pytest
import torch

from paper_2510_21270_amd import binding as pbs

pytestmark = pytest.mark.gpu


def _fill(x, seed):
    x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))


def test_a_recorded_pipeline_writes_the_slots_it_was_given():
    p = pbs.problem(1, 4, 2, 700, 64, 64, 256, "bf16", tau=0.9)
    Q, K, V = (torch.zeros(1, h, 700, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    cache = pbs.Cache.alloc(60, 16, 2, 64, torch.int8)
    pipe = pbs.Pipeline(p)
    slots = torch.randperm(960, generator=torch.Generator().manual_seed(1))[:700].to(torch.int32)
    for seed, x in enumerate((Q, K, V)):
        _fill(x, seed)
    pipe.capture(Q, K, V, cache=cache, slots=slots[None].cuda())               # nobody else holds these slots
    over = [torch.randint(0, 960, (1, 700), dtype=torch.int32, device="cuda") for _ in range(64)]
    for k in range(3):
        for seed, x in enumerate((Q, K, V)):
            _fill(x, 10 * k + 20 + seed)
        for x in (cache.K, cache.V, cache.k_scale, cache.v_scale):
            x.zero_()
        O = pipe.replay().clone()
        torch.cuda.synchronize()
        got = [x.clone() for x in (cache.K, cache.V, cache.k_scale, cache.v_scale)]
        for x in (cache.K, cache.V, cache.k_scale, cache.v_scale):
            x.zero_()
        assert torch.equal(pipe.run(Q, K, V, cache=cache, slots=slots[None].cuda()), O)
        for x, y in zip((cache.K, cache.V, cache.k_scale, cache.v_scale), got):
            assert torch.equal(x, y)
    assert len(over) == 64
