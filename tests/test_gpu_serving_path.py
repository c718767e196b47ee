"""The operators around the prefill path together, as a server uses them: a prompt turned by its positions, attended to by
the block-sparse pipeline (all blocks kept) and by the packed-prompt kernel, its keys cached, a later chunk over keys read back,
then steps of new tokens over the cache, eager and replayed, with a prefix that the batch shares."""
import math

import pytest
import torch

from paper_2510_21270_amd import binding as pbs
from serving_helpers import H16, TYPES, attention_ref, hold_ref, rope_ref, stands_for, within

pytestmark = pytest.mark.gpu


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
def test_prompt_cache_chunk_and_steps(held):
    h_q, h_kv, d, n, page = 8, 2, 128, 700, 32
    r, scale = h_q // h_kv, 1 / math.sqrt(128)
    freq, mag = pbs.rope_frequencies(d, 5e5, "bands", 8.0, 512)
    cache = pbs.Cache.alloc(64, page, h_kv, d, TYPES[held])
    order = torch.randperm(64, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    prefix_pages = order[: -(-n // page)].contiguous()
    t = torch.arange(n)
    slots = (prefix_pages[t // page].long() * page + t % page).to(torch.int32)

    # the prompt, [1, heads, n, d] as the pipeline takes it, turned in place through views
    Q, K, V = _randn(2, 1, h_q, n, d).bfloat16().cuda(), _randn(3, 1, h_kv, n, d).bfloat16().cuda(), _randn(4, 1, h_kv, n, d).bfloat16().cuda()
    raw = [Q.clone(), K.clone()]
    pos = torch.arange(n, dtype=torch.int32).cuda()
    q, k, v = (x[0].transpose(0, 1) for x in (Q, K, V))
    pbs.rope(q, k, pos, freq, magnitude=mag, Qout=q, Kout=k)
    for x, was in ((q, raw[0]), (k, raw[1])):
        want, e = rope_ref(was[0].transpose(0, 1).cpu(), pos.cpu(), freq.cpu(), "half", mag)
        within(x, want, e + H16 * (want.abs() + e))
    p = pbs.problem(1, h_q, h_kv, n, d, 128, 256, "bf16", tau=2.0, flags=pbs.FLAG_FORCE_FIRST_BLOCK)   # keeps every block
    pipe = pbs.Pipeline(p)
    sparse = pipe.run(Q, K, V, cache=cache, slots=slots[None].cuda())
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    dense = pbs.prompt_attn(q, k, v, cu)
    rows = torch.tensor([0, 1, 31, 127, 128, 300, 511, 640, 699])
    hq, hk, hv = q.cpu(), k.cpu(), v.cpu()
    for h in range(h_q):
        sees = torch.arange(n)[None] <= rows[:, None]
        want, _, bound, _ = attention_ref(hq[rows, h], hk[:, h // r], hv[:, h // r], sees, scale)
        within(dense[rows, h], want, bound, "packed prompt, head %d" % h)
        within(sparse[0, h, rows], want, bound, "pipeline, head %d" % h)
    kept = [stands_for(*hold_ref(x, TYPES[held])) for x in (hk, hv)]
    got = pbs.cache_read(cache, slots.cuda())
    assert torch.equal(got[0].cpu(), kept[0].bfloat16()) and torch.equal(got[1].cpu(), kept[1].bfloat16())

    # a chunk of 90 queries behind the keys read back
    m = 90
    cq, ck, cv = _randn(5, m, h_q, d).bfloat16(), _randn(6, m, h_kv, d).bfloat16(), _randn(7, m, h_kv, d).bfloat16()
    keys, values = torch.cat((got[0], ck.cuda())), torch.cat((got[1], cv.cuda()))
    chunk = pbs.prompt_attn(cq.cuda(), keys, values, torch.tensor([0, m], dtype=torch.int32).cuda(),
                            torch.tensor([0, n + m], dtype=torch.int32).cuda())
    rows = torch.tensor([0, 31, 32, 89])
    for h in range(h_q):
        sees = torch.arange(n + m)[None] <= n + rows[:, None]
        want, _, bound, _ = attention_ref(cq[rows, h], keys[:, h // r].cpu(), values[:, h // r].cpu(), sees, scale)
        within(chunk[rows, h], want, bound, "chunk, head %d" % h)

    # steps of 5 sequences that share the prompt as their prefix, two tokens at a time
    n_seq, q_len, steps, max_pages = 5, 2, 3, 2
    table = order[-(-n // page):][: n_seq * max_pages].view(n_seq, max_pages).contiguous()
    step = pbs.DecodeStep(cache, n_seq, h_q, max_pages, freq, q_len, magnitude=mag, prefix_pages=prefix_pages.cuda(), prefix_len=n)
    bufs = [torch.zeros(n_seq, q_len, h_q, d, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(n_seq * q_len, h_kv, d, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(n_seq * q_len, h_kv, d, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(n_seq * q_len, dtype=torch.int32, device="cuda"),
            torch.full((n_seq * q_len,), -1, dtype=torch.int32, device="cuda"), table.cuda(),
            torch.zeros(n_seq, dtype=torch.int32, device="cuda")]
    own_k, own_v = [torch.zeros(n_seq, 0, h_kv, d) for _ in range(2)]
    for s in range(steps):
        new = [_randn(20 + 3 * s + i, *bufs[i].shape).bfloat16() for i in range(3)]
        at = (q_len * s + torch.arange(q_len)).repeat(n_seq)                   # of the sequence's own tokens
        seq = torch.arange(n_seq).repeat_interleave(q_len)
        where = (table[seq, at // page].long() * page + at % page).to(torch.int32)
        values = new + [(n + at).to(torch.int32), where, table, torch.full((n_seq,), q_len * (s + 1), dtype=torch.int32)]
        for buf, x in zip(bufs, values):
            buf.copy_(x)
        if s == 0:
            O = step.run(*bufs)
        else:
            if s == 1:
                step.capture(*bufs)
                for buf, x in zip(bufs, values):           # Q and K have been turned
                    buf.copy_(x)
            O = step.replay()
        torch.cuda.synchronize()
        tq, _ = rope_ref(new[0].view(-1, h_q, d), n + at, freq.cpu(), "half", mag)
        turned_q, turned_k = bufs[0].cpu(), bufs[1].cpu()
        within(turned_q.view(-1, h_q, d), tq, H16 * tq.abs() + 1e-4)
        own_k = torch.cat((own_k, stands_for(*hold_ref(turned_k, TYPES[held])).view(n_seq, q_len, h_kv, d)), 1)
        own_v = torch.cat((own_v, stands_for(*hold_ref(new[2], TYPES[held])).view(n_seq, q_len, h_kv, d)), 1)
        own = q_len * (s + 1)
        for i in range(n_seq):
            sees = torch.arange(n + own)[None] <= n + own - q_len + torch.arange(q_len)[:, None]
            for h in range(h_q):
                a, b = torch.cat((kept[0][:, h // r], own_k[i, :, h // r])), torch.cat((kept[1][:, h // r], own_v[i, :, h // r]))
                want, _, bound, _ = attention_ref(turned_q[i, :, h], a, b, sees, scale)
                within(O[i, :, h], want, bound, "step %d, sequence %d, head %d" % (s, i, h))


def test_two_steps_at_once_on_two_streams():
    # each with a workspace of its own
    caches, outs, wants = [], [], []
    g = torch.Generator(device="cuda").manual_seed(5)
    for k in range(2):
        c = pbs.Cache.alloc(80, 16, 2, 64)
        c.K.normal_(generator=g)
        c.V.normal_(generator=g)
        caches.append(c)
    table = torch.arange(80, dtype=torch.int32).view(2, 40).cuda()
    lens = torch.tensor([640, 333], dtype=torch.int32).cuda()
    Q = torch.randn(2, 1, 8, 64, generator=g, device="cuda").bfloat16()
    for c in caches:
        wants.append(pbs.decode_attn(c, Q, table, lens))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(10):
        for c, s in zip(caches, streams):
            with torch.cuda.stream(s):
                outs.append(pbs.decode_attn(c, Q, table, lens))
    torch.cuda.synchronize()
    for k, o in enumerate(outs):
        assert torch.equal(o, wants[k % 2])
