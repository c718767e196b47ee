"""Packed prompts under a score rule where there are so many rows that a workgroup has 256 of them, against a plain 64-bit form."""
import math

import pytest
import torch

from paper_2510_21270_amd import binding as pbs
from rule_helpers import ruled_ref
from serving_helpers import within
from test_gpu_rules_prompt import Setup

pytestmark = pytest.mark.gpu


def _wide(s):
    """Whether a workgroup has 256 rows: what the library's rule says for this call."""
    h_q, h_kv = s.Q.shape[1], s.K.shape[1]
    r = h_q // h_kv
    return (sum(s.lens) // (256 // r) + len(s.lens)) * h_kv >= (1792 if r == 1 else 448)


SHORT = [(29 * i) % 77 for i in range(60)]
PREFIX = [(11 * i) % 50 - 3 for i in range(60)]
CASES = [(8, 4, 128, dict(cap=6.0)), (8, 2, 64, dict(cap=5.0, slopes=True)), (8, 4, 128, dict(window=21, sinks=2, prefix=PREFIX)),
         (8, 7, 128, dict(slopes=True, prefix=PREFIX)), (8, 7, 64, dict(cap=70.0, window=33)), (8, 3, 128, dict()),
         (9, 5, 64, dict(cap=4.0, slopes=True, window=40, sinks=60, prefix=PREFIX)), (8, 2, 128, dict(cap=90.0, slopes=True))]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("h_kv,r,d,rule", CASES)
def test_many_short_prompts(h_kv, r, d, rule, causal):
    # one tile or two to a sequence, most with rows left over; keys in front of some, fewer keys than queries in others
    s = Setup(21, SHORT, [(0, 70, -9)[i % 3] for i in range(60)], r * h_kv, h_kv, d, causal=causal, **rule)
    assert _wide(s)
    O, lse = s.call()
    s.check(O, lse, heads=[0, r * h_kv // 2 + 1, r * h_kv - 1])
    for i, n in enumerate(s.lens):
        if n and not s.keys[i]:
            at = slice(int(s.cu_q[i]), int(s.cu_q[i + 1]))
            assert float(O[at].abs().max()) == 0.0 and bool((lse[at] == -math.inf).all())
    again, _ = s.call()
    assert torch.equal(again, O)


@pytest.mark.parametrize("d,rule", [(64, dict(slopes=True, window=50, sinks=1)), (128, dict(cap=7.0)), (64, dict(window=300))])
def test_a_head_to_every_kv_head(d, rule):
    # 256 tokens to a workgroup
    lens = [(37 * i) % 60 for i in range(118)] + [256, 700]
    s = Setup(22, lens, [0] * 120, 16, 16, d, **rule)
    assert _wide(s)
    s.check(*s.call(), rows=[0, 1, 31, 32, 59, 127, 128, 223, 224, 255, 256, 257, 511, 512, 600, 699], heads=[0, 7, 15])


# groups that leave rows of 256 without a query (7: 252, 96: 192, whose last waves have none), and one that fills it with two tokens
@pytest.mark.parametrize("h_kv,r,d,n,rule", [(16, 4, 128, 1500, dict(cap=8.0)), (16, 4, 64, 1500, dict(slopes=True, window=400, sinks=70)),
                                             (12, 7, 128, 1300, dict(window=200, prefix=[300, 5])), (1, 128, 64, 520, dict(cap=3.0)),
                                             (2, 96, 64, 300, dict(slopes=True, prefix=[9, 200])), (4, 40, 128, 400, dict(cap=20.0, slopes=True, window=90))])
def test_long_prompts(h_kv, r, d, n, rule):
    s = Setup(23, [n, n - 101], [77, 0], r * h_kv, h_kv, d, **rule)
    assert _wide(s)
    h_q = r * h_kv
    s.check(*s.call(), rows=[0, 1, 2, 63, 64, 65, 100, 127, 128, 199, 255, 256, 299, 300, 401, 900, 1023, 1024, 1198, 1499, n - 1], heads=sorted({0, 1, h_q // 2, h_q - 1}))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rule", [dict(window=50, sinks=2), dict(cap=9.0), dict(slopes=True, prefix=[5] * 40)])
def test_values_that_are_not_finite(d, rule):
    h_q, heads = 64, [0, 3, 4, 63]                         # of kv heads 0, 0, 1, 15
    s = Setup(24, [300] + [20] * 39, [0] * 40, h_q, 16, d, **rule)
    assert _wide(s)
    clean, lse = s.call()
    s.check(clean, lse, rows=range(0, 300, 17), heads=heads)
    V, twice = s.V.clone(), {}
    odd_values = ((120, 0, 3, math.inf), (170, 0, 3, -math.inf), (250, 1, 7, math.nan), (299, 15, 0, math.inf))
    for key, kv, f, v in odd_values:
        s.V[key, kv, f] = v
    O, lse2 = s.call()
    # rows that are formed a second time have other roundings: each of the two is within its bound of the exact one
    sees, pos, j = s.sees(0, torch.arange(300))
    for h in heads:
        _, _, _, bo, bl, _ = ruled_ref(s.Q[:300, h], s.K[:300, h // 4], V[:300, h // 4], sees, 1 / math.sqrt(d), s.cap,
                                       float(s.slopes[h]) if s.slopes is not None else 0.0, pos, j, weight_bits=8)
        within(lse2[:300, h], lse[:300, h].double().cpu(), 2 * bl, "lse of head %d" % h)
        want, got = clean[:300, h].float().cpu(), O[:300, h].float().cpu()
        for key, kv, f, v in odd_values:
            if h // 4 == kv:
                want[sees[:, key], f] += v
        odd = ~torch.isfinite(want)
        assert odd.any()
        # a weight that has become 0 makes NaN of an infinite value: where there is one, it is not finite
        assert not torch.isfinite(got[odd]).any() and bool(((got - want).abs() <= 2 * bo)[~odd].all())
    # workgroups without such values have stored once
    assert torch.equal(O[300:], clean[300:]) and torch.equal(O[:, 8:60], clean[:, 8:60])


def test_logits_that_grow_along_the_keys():
    # the reference moves again and again, for waves of a workgroup at different tiles
    for step in (0.2, 3.0):
        s = Setup(25, [600, 400], [0, 0], 128, 32, 64, slopes=True)
        assert _wide(s)
        s.Q.abs_()
        for i, n in enumerate(s.lens):
            s.K[int(s.cu_k[i]):int(s.cu_k[i + 1])] = (step * torch.arange(float(n)) / 8)[:, None, None].expand(-1, 32, 64).bfloat16()
        s.check(*s.call(), rows=range(0, 600, 37), heads=[0, 63, 127])


def test_strided_and_captured():
    s = Setup(26, SHORT, [0] * 60, 32, 8, 128, cap=7.0, slopes=True, window=60, sinks=1)
    assert _wide(s)
    want, lse = s.call()
    total = sum(SHORT)
    fused = torch.zeros(total, 50, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, :32], fused[:, 33:41], fused[:, 41:49] = s.Q.cuda(), s.K.cuda(), s.V.cuda()
    out, cu = torch.zeros(32, total, 128, dtype=torch.bfloat16, device="cuda").transpose(0, 1), s.cu_q.cuda()
    pbs.prompt_attn_rule(s.rule, fused[:, :32], fused[:, 33:41], fused[:, 41:49], cu, O=out)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = pbs.prompt_attn_rule(s.rule, fused[:, :32], fused[:, 33:41], fused[:, 41:49], cu)
    for k in range(3):
        fused[:, :32].copy_((1.0 + k) * s.Q.cuda())
        cu[30:].fill_(int(s.cu_q[-1]) - k)
        graph.replay()
        torch.cuda.synchronize()
        eager = pbs.prompt_attn_rule(s.rule, fused[:, :32], fused[:, 33:41], fused[:, 41:49], cu)
        n = int(cu[-1])
        assert torch.equal(O[:n], eager[:n])
