"""Evictions around 8192 keys, up to which a workgroup has a unit's ranks in its registers (one launch; beyond that several workgroups
have 8192 keys each, in six), and where more keys are protected than may stay."""
import pytest
import torch

from paper_2510_21270_amd import binding as pbs
from test_gpu_evict import Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["random", "ties", "odd", "equal"])
@pytest.mark.parametrize("n,budget,sinks,recent", [(8192, 8191, 4, 64), (8192, 3000, 0, 0), (8193, 8192, 4, 64), (8193, 1, 0, 1), (8193, 5000, 9, 700),
                                                   (16384, 8192, 0, 33), (16385, 8193, 2, 0), (8196, 8190, 0, 0)])
def test_a_workgroup_s_bound(kind, n, budget, sinks, recent):
    Setup(41, 2, 64, "i8", 16, [n, n - 1], kind).check(budget, sinks, recent, max_len=n)


@pytest.mark.parametrize("kind", ["random", "ties"])
def test_one_long_sequence_beside_short_ones(kind):
    # units whose second workgroup has a key, none, and units that keep all of theirs
    Setup(42, 3, 128, "bf16", 16, [8193, 100, 8192, 5000, 0, 300, 8191], kind).check(300, 2, 50, max_len=8193)


@pytest.mark.parametrize("max_len", [None, 16384, 70000])
def test_short_sequences_under_a_large_bound(max_len):
    s = Setup(43, 2, 64, "e4m3", 16, [1040, 1024, 17, 0, 1030], "ties")
    if max_len:                                            # a table of as many pages, those behind the last key none
        s.table = torch.cat([s.table, torch.full((5, -(-max_len // 16) - s.table.shape[1]), -1, dtype=torch.int32)], 1)
    s.check(1000, 4, 64, max_len=max_len)


@pytest.mark.parametrize("n", [100, 8300])
def test_more_protected_keys_than_may_stay(n):
    # positions below 0, and one position many times: of the protected keys those at the lowest places stay, whatever their weights
    s = Setup(44, 2, 64, "i8", 16, [n, n - 7])
    s.position -= n // 4
    s.position.view(-1)[::3] = int(s.position.max())       # a third are the newest
    s.marks = pbs.CacheMarks(s.cache, s.weight.cuda(), s.position.cuda())
    budget = n // 5
    for i in range(2):
        j = torch.arange(s.lens[i])
        p = s.position[s.table[i][j // 16].long(), 0, j % 16]
        assert int(((p < 2) | (p > p.max() - 3)).sum()) > budget
    s.check(budget, 2, 3)


def test_the_order_of_places_among_protected_keys():
    # ten keys at position -1, the later ones heavier: the first four stay
    cache = pbs.Cache.alloc(1, 16, 1, 64)
    cache.K[0, 0] = torch.arange(16.0, device="cuda")[:, None].bfloat16()
    marks = pbs.CacheMarks.alloc(cache)
    marks.weight[0, 0] = torch.arange(16.0, device="cuda")
    marks.position[0, 0] = torch.tensor([3, 4, 5, 6, 7] + [-1] * 10 + [8], dtype=torch.int32, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([16], dtype=torch.int32, device="cuda")
    assert pbs.cache_evict(marks, table, lens, 4).tolist() == [4]
    assert cache.K[0, 0, :4, 0].tolist() == [5.0, 6.0, 7.0, 8.0] and marks.weight[0, 0, :4].tolist() == [5.0, 6.0, 7.0, 8.0]
    assert marks.position[0, 0, :4].tolist() == [-1] * 4
