"""Packed prompts whose keys reach to the end of what a head may span: the last offset of a row lies just below 2 GiB."""
import math

import pytest
import torch

from paper_2510_21270_amd import binding as pbs
from serving_helpers import H16, H32, within

pytestmark = pytest.mark.gpu


def _check(Q, K, V, O, lse):
    """Queries at the end of all keys, causal, in 64 bits on the GPU, a head at a time."""
    m, n, r, d = Q.shape[0], K.shape[0], Q.shape[1] // K.shape[1], Q.shape[2]
    hides = torch.ones(m, n, dtype=torch.bool, device="cuda").triu(n - m + 1)
    # a sum over the keys takes a step to 16 of them
    sums = (n / 16 + 64) * H32
    for h in range(Q.shape[1]):
        q, k, v = Q[:, h].double(), K[:, h // r].double(), V[:, h // r].double()
        s = torch.mm(q, k.t().contiguous()) / math.sqrt(d)
        s.masked_fill_(hides, -math.inf)
        w = torch.softmax(s, 1)
        o = torch.mm(w, v)
        ds = (d + 8) * H32 * float(torch.mm(q.abs(), k.abs().t().contiguous()).max()) / math.sqrt(d) + 8 * H32 * float(s[~hides].abs().max())
        bound = torch.mm(w, v.abs()) * (H16 + 2 * ds + 2 * sums + 2.0 ** -20) + o.abs() * H16
        within(O[:, h], o.cpu(), 1.01 * bound.cpu(), "head %d" % h)
        l = torch.logsumexp(s, 1)
        within(lse[:, h], l.cpu(), (ds + sums + 4 * H32 * l.abs() + 4 * H32).cpu() * 1.01, "lse of head %d" % h)


def _fill(g, K, V, Q):
    K.normal_(generator=g)
    V.normal_(generator=g)
    n, r = K.shape[0], Q.shape[1] // K.shape[1]
    for i, at in enumerate((n - 2, n - 33, n - 290, 5)):   # the keys that weigh most, one to a head in turn
        for h in range(K.shape[1]):
            if h % 4 == i:
                K[at, h] = Q[0, h * r] * 2.0


@pytest.mark.parametrize("n", [1048449, 1048511])
def test_as_many_keys_as_a_head_may_span(n):
    g = torch.Generator(device="cuda").manual_seed(n)
    Q = (1.5 * torch.randn(3, 8, 128, generator=g, device="cuda")).bfloat16()
    K, V = (torch.empty(n, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    _fill(g, K, V, Q)
    cu_q, cu_k = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (3, n))
    O, lse = pbs.prompt_attn(Q, K, V, cu_q, cu_k, want_lse=True)
    _check(Q, K, V, O, lse)
    with pytest.raises(pbs.PbsError):                      # one row more than the limit's
        more = torch.empty(1048512 - n, 8, 128, dtype=torch.bfloat16, device="cuda")
        pbs.prompt_attn(Q, torch.cat((K, more)), torch.cat((V, more)), cu_q, cu_k)


@pytest.mark.parametrize("n", [897, 930, 959])
def test_rows_as_far_apart_as_a_head_may_span(n):
    g = torch.Generator(device="cuda").manual_seed(n)
    Q = (1.5 * torch.randn(40, 8, 64, generator=g, device="cuda")).bfloat16()
    rows = torch.zeros(n, 1 << 20, dtype=torch.bfloat16, device="cuda")
    K, V = rows[:, :512].view(n, 8, 64), rows[:, 1024:1536].view(n, 8, 64)
    k, v = torch.empty(n, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 8, 64, dtype=torch.bfloat16, device="cuda")
    _fill(g, k, v, Q)
    K.copy_(k)
    V.copy_(v)
    cu_q, cu_k = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (40, n))
    O, lse = pbs.prompt_attn(Q, K, V, cu_q, cu_k, want_lse=True)
    _check(Q, k, v, O, lse)
