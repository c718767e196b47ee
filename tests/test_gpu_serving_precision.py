"""How exact the weights of attention over a cache are: two terms in bf16, so that rounding O once is nearly all that is off."""
import math

import pytest
import torch

from paper_2510_21270_amd import binding as pbs            # noqa: F401
from serving_helpers import H16, H32, TYPES, within
from test_gpu_serving import Setup

pytestmark = pytest.mark.gpu


def _ref(q, k, v, sees, scale):
    """One head in 64 bits: q [m, d], k, v [n, d], sees [m, n] -> O and its elementwise bound.  A weight in two terms: the first is off by
    2^-8 of it at most, the second, the rest, by 2^-8 of that."""
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    s = torch.where(sees, (q @ k.T) * scale, torch.full((), -math.inf, dtype=torch.float64))
    some = sees.any(1, keepdim=True)
    w = torch.where(some, torch.softmax(s, 1), torch.zeros((), dtype=torch.float64))
    ds = (q.shape[1] + 8) * H32 * (torch.where(sees, q.abs() @ k.abs().T, 0).amax(1, keepdim=True) * scale) + \
        8 * H32 * torch.where(sees, s.abs(), 0).amax(1, keepdim=True)
    o = w @ v
    return o, ((w @ v.abs()) * (H16 * H16 + 2 * ds + 2 * (sees.sum(1, keepdim=True) + 64) * H32 + 2.0 ** -20) + o.abs() * H16) * 1.01 + 1e-30


def _check(s, O):
    r, P = s.h_q // s.h_kv, s.prefix
    for i, n in enumerate(s.lens):
        t, j = torch.arange(s.q_len)[:, None], torch.arange(P + n)[None]
        sees = ((j < P + n - s.q_len + 1 + t) | (j < P)) & (j < P + n)
        for h in range(s.h_q):
            k = torch.cat((s.k[-1][:, h // r], s.k[i][:, h // r]))
            v = torch.cat((s.v[-1][:, h // r], s.v[i][:, h // r]))
            want, bound = _ref(s.Q[i, :, h], k, v, sees, 1 / math.sqrt(s.d))
            within(O[i, :, h], want, bound, "O of sequence %d (%d keys), head %d" % (i, n, h))


LENS = [1, 2, 3, 16, 17, 33, 64, 100, 130, 0, 700]


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("q_len,h_q,h_kv,d,most", [(1, 8, 2, 64, 700), (1, 8, 2, 128, 700), (1, 8, 8, 128, 100), (3, 8, 2, 64, 700),
                                                   (5, 16, 2, 128, 700), (16, 12, 1, 64, 130)])
def test_weights_of_own_keys(held, q_len, h_q, h_kv, d, most):
    s = Setup(50, q_len, h_q, h_kv, d, held, 16, [n for n in LENS if n <= most])
    _check(s, s.call())


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("n,q_len,h_q,h_kv,d,prefix", [(3, 1, 8, 2, 128, 1), (3, 1, 8, 2, 64, 300), (7, 1, 8, 2, 128, 300), (5, 1, 16, 4, 64, 5)])
def test_weights_of_a_prefix_of_few_rows(held, n, q_len, h_q, h_kv, d, prefix):
    s = Setup(51, q_len, h_q, h_kv, d, held, 32, LENS[:n], prefix)
    _check(s, s.call())
    s.lens = [0] * n                                       # the prefix alone
    s.k[:n], s.v[:n] = [x[:0] for x in s.k[:n]], [x[:0] for x in s.v[:n]]
    _check(s, s.call(max_len=0))


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
@pytest.mark.parametrize("q_len", [1, 2, 16])
def test_values_that_are_not_finite_beside_both_terms(held, q_len):
    # an infinity times a rest of either sign, or of zero, is no infinity of the value's sign
    s = Setup(52, q_len, 8, 2, 128, held, 16, [300, 40, 90])
    clean = s.call()
    odd = []
    for i, at in ((0, 7), (1, 20), (2, 33)):
        page = int(s.table[i, at // 16])
        if held == "bf16":
            s.cache.V[page, :, at % 16, 5 + i] = math.inf if i != 1 else -math.inf
            odd.append(5 + i)
        else:
            s.cache.V.view(torch.uint8)[page, :, at % 16, 5 + i] = 0x7f
            odd.append(5 + i)
    O = s.call()
    for i in range(3):
        seen = O[i, :, :, odd[i]].float()
        sees = torch.ones(q_len, dtype=torch.bool) if i == 0 else torch.arange(q_len) + s.lens[i] - q_len >= (20 if i == 1 else 33)
        if held == "bf16":
            # (its weight may be 0: NaN)
            assert (torch.isnan(seen[sees]) | (seen[sees] == (math.inf if i != 1 else -math.inf))).all()
            assert (seen[sees] == (math.inf if i != 1 else -math.inf)).any()
        else:
            assert torch.isnan(seen[sees]).all()
        same = [f for f in range(128) if f != odd[i]]
        assert torch.equal(O[i][..., same], clean[i][..., same])
