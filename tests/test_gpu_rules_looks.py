"""New tokens over rows with positions under a window where waves look at positions before they bring tiles: many rows to a kv head,
pages that are none, values that are not finite; and one new token to a sequence."""
import math

import pytest
import torch

from test_gpu_rules_decode import Setup

pytestmark = pytest.mark.gpu

WINDOW = 300


def _setup(q_len, h_q, h_kv, held, lens, d=64, **rule):
    s = Setup(31, q_len, h_q, h_kv, d, held, 32, lens, window=WINDOW, marked=True, **rule)
    # what the library goes by: the tiles that all units of the batch may have, to a wave
    rows = q_len * h_q // h_kv
    nt = 1 if rows <= 16 else 2
    shares, units = 2048 if nt == 1 else 1024, h_kv * -(-rows // (16 * nt))
    assert len(lens) * units * s.table.shape[1] > 12 * nt * shares             # (pages of 32 rows: a tile)
    assert sum(n // 32 for n in lens) * units > 9 * shares # and of those that they have
    return s


# 80 and 128 rows of a kv head are three and four tiles of rows, and pass the 64 whose lse are formed together; 40 are two tiles, the
# second with 8 rows
@pytest.mark.parametrize("q_len,h_q,h_kv,held,rule", [(5, 64, 4, "bf16", dict(cap=9.0, slopes=True, sinks=4)), (4, 40, 4, "i8", dict(cap=5.0)),
                                                      (16, 32, 4, "e4m3", dict(slopes=True)), (1, 160, 4, "bf16", dict(sinks=9))])
def test_many_rows_to_a_kv_head(q_len, h_q, h_kv, held, rule):
    s = _setup(q_len, h_q, h_kv, held, [45000, 3, 2000], **rule)
    m = s.marks()
    O, lse = s.call(marks=m, weigh=True, want_lse=True)
    s.check(O, lse, m.weight)
    again = s.marks()
    assert torch.equal(s.call(marks=again, weigh=True), O) and torch.equal(again.weight, m.weight)


@pytest.mark.parametrize("q_len,h_q,h_kv", [(1, 32, 16), (3, 96, 16)])
def test_pages_that_are_none(q_len, h_q, h_kv):
    s = _setup(q_len, h_q, h_kv, "bf16", [40000, 50, 3000], cap=9.0, sinks=2)
    listed, none = s.table.clone(), torch.zeros(40000, dtype=torch.bool)
    # pages with keys that are seen, and one without, are none
    seen = (s.q_pos[0][0] - s.k_pos[0][:, 0] < WINDOW).nonzero()[:, 0]
    for k, page in enumerate([int(seen[2]) // 32, int(seen[len(seen) // 2]) // 32, 1111]):
        s.table[0, page] = (-1, 10 ** 6, -7)[k]
        none[32 * page:32 * page + 32] = True
    m = s.marks()
    O, lse = s.call(marks=m, weigh=True, want_lse=True)
    s.table = listed                                       # (rows of pages that were none get nothing)
    s.check(O, lse, m.weight, hidden=lambda i, j: none[j] if i == 0 else torch.zeros(len(j), dtype=torch.bool))


def _place_of(s, key, distance):
    """Gives a key of sequence 0 a position at this distance from the first query, for every head."""
    where = s.q_pos[0][0] - distance
    at = int(s.slots(0, torch.tensor([key])))
    s.k_pos[0][key], s.position[at // 32, :, at % 32] = where, int(where)
    return at // 32, at % 32


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_values_that_are_not_finite_where_one_query_sees_them(held):
    s = _setup(2, 32, 16, held, [40000, 50, 3000], slopes=True)
    page, off = _place_of(s, 23456, WINDOW - 1)            # the second query is too far
    m = s.marks()
    want, want_lse = s.call(marks=m, weigh=True, want_lse=True)
    s.check(want, want_lse, m.weight)
    if held == "bf16":
        s.cache.V[page, 0, off, 3] = math.inf
    else:
        s.cache.V.view(torch.uint8)[page, 0, off, 3] = 0x7f
    n = s.marks()
    O, lse = s.call(marks=n, weigh=True, want_lse=True)
    assert (O[0, 0, :2, 3] == math.inf).all() if held == "bf16" else torch.isnan(O[0, 0, :2, 3]).all()
    keep = O.clone()
    keep[0, 0, :2, 3] = want[0, 0, :2, 3]
    assert torch.equal(keep, want) and torch.equal(lse, want_lse) and torch.equal(n.weight, m.weight)


@pytest.mark.parametrize("q_len,h_q,held", [(1, 32, "bf16"), (1, 32, "e4m3"), (3, 96, "bf16")])
def test_values_that_are_not_finite_where_every_query_sees_them(q_len, h_q, held):
    # such a wave goes over all of its tiles again, those that it had passed over among them
    s = _setup(q_len, h_q, 16, held, [40000, 50, 3000], cap=9.0)
    page, off = _place_of(s, 23456, 5)
    m = s.marks()
    want, want_lse = s.call(marks=m, weigh=True, want_lse=True)
    s.check(want, want_lse, m.weight)
    if held == "bf16":
        s.cache.V[page, 0, off, 3] = -math.inf
    else:
        s.cache.V.view(torch.uint8)[page, 0, off, 3] = 0xff
    n = s.marks()
    O, lse = s.call(marks=n, weigh=True, want_lse=True)
    r = h_q // 16
    hit = O[0, :, :r, 3]
    assert (hit == -math.inf).all() if held == "bf16" else torch.isnan(hit).all()
    # the logits are the same; of O the values that are finite
    assert torch.equal(lse, want_lse) and torch.equal(n.weight, m.weight)
    O[0, :, :r, 3] = want[0, :, :r, 3]
    s.check(O, lse, n.weight)


def test_keys_that_are_not_finite_behind_the_window():
    # tiles without a key that is seen hold NaN everywhere: neither brought nor weighed
    s = _setup(2, 32, 16, "bf16", [40000, 50, 3000], sinks=1)
    m = s.marks()
    want, lse = s.call(marks=m, weigh=True, want_lse=True)
    s.check(want, lse, m.weight)
    j = torch.arange(40000)
    for kv in range(16):
        near = (s.q_pos[0][-1] - s.k_pos[0][:, kv] < WINDOW + 1) | (s.k_pos[0][:, kv] < 1)
        at = s.slots(0, j[~near]).long()[::5]
        s.cache.K[at // 32, kv, at % 32], s.cache.V[at // 32, kv, at % 32] = math.nan, math.inf
    n = s.marks()
    O, lse2 = s.call(marks=n, weigh=True, want_lse=True)
    assert torch.equal(O, want) and torch.equal(lse, lse2) and torch.equal(n.weight, m.weight)
