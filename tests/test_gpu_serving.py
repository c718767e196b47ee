"""Rotary positions, the paged cache and attention of new tokens over it, against plain 64-bit forms."""
import math

import pytest
import torch

from paper_2510_21270_amd import binding as pbs
from serving_helpers import H16, H32, TYPES, attention_ref, hold_ref, rope_ref, stands_for, within

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(seed, *shape):
    return torch.randn(shape, generator=_gen(seed))


# ------------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,h_q,h_kv,d,rot", [(1, 1, 1, 64, 16), (3, 32, 8, 128, 128), (2051, 7, 1, 128, 96),
                                                   (2500, 2, 2, 64, 32), (257, 28, 4, 128, 64)])
def test_rope(tokens, h_q, h_kv, d, rot, dtype, layout):
    dt = TYPES[dtype]
    Q, K = _randn(1, tokens, h_q, d).to(dt), _randn(2, tokens, h_kv, d).to(dt)
    pos = torch.randint(-5, 1 << 20, (tokens,), generator=_gen(3), dtype=torch.int32)
    freq, mag = pbs.rope_frequencies(rot, 5e5, "ramp", 4.0, 8192)
    half = H16 if dtype == "bf16" else H32
    for transpose in (False, True):
        got = pbs.rope(Q.cuda(), K.cuda(), pos.cuda(), freq, layout=layout, magnitude=mag, transpose=transpose)
        for x, y in zip((Q, K), got):
            want, e = rope_ref(x, pos, freq.cpu(), layout, mag, transpose)
            within(y, want, e + half * (want.abs() + e), "rope")
            assert torch.equal(y[..., rot:].cpu(), x[..., rot:])


def test_rope_in_place_on_a_fused_projection_and_transposed_heads():
    tokens, h_q, h_kv, d = 2049, 8, 2, 128
    fused = _randn(1, tokens, (h_q + 2 * h_kv) * d).bfloat16()
    pos = torch.arange(tokens, dtype=torch.int32)
    freq, _ = pbs.rope_frequencies(d, 1e4)
    dev = fused.cuda()
    heads = dev.view(tokens, h_q + 2 * h_kv, d)
    q, k, v = heads[:, :h_q], heads[:, h_q:h_q + h_kv], heads[:, h_q + h_kv:]
    pbs.rope(q, k, pos.cuda(), freq, Qout=q, Kout=k)
    host = fused.view(tokens, h_q + 2 * h_kv, d)
    for x, y in ((host[:, :h_q], q), (host[:, h_q:h_q + h_kv], k)):
        want, e = rope_ref(x, pos, freq.cpu(), "half")
        within(y, want, e + H16 * (want.abs() + e))
    assert torch.equal(v.cpu(), host[:, h_q + h_kv:])
    # the [1, heads, n, d] tensors of the prefill path, seen token by token; partly rotated in place
    x = _randn(4, 1, h_q, tokens, d).bfloat16().cuda()
    before = x.clone()
    freq32, _ = pbs.rope_frequencies(32, 1e4)
    view = x[0].transpose(0, 1)
    pbs.rope(view, None, pos.cuda(), freq32, layout="interleaved", Qout=view)
    want, e = rope_ref(before[0].transpose(0, 1).cpu(), pos, freq32.cpu(), "interleaved")
    within(view, want, e + H16 * (want.abs() + e))
    # keys alone, new memory
    _, k2 = pbs.rope(None, view, pos.cuda(), freq32)
    want, e = rope_ref(view.cpu(), pos, freq32.cpu(), "half")
    within(k2, want, e + H16 * (want.abs() + e))


def test_rope_transpose_is_the_gradient():
    # L = sum(G * rope(x)) in 64 bits by differences, against rope(G, transpose)
    tokens, d = 5, 64
    x, G = _randn(1, tokens, 2, d), _randn(2, tokens, 2, d)
    pos = torch.tensor([0, 1, 7, 1000, 70000], dtype=torch.int32)
    for layout in ("half", "interleaved"):
        freq, mag = pbs.rope_frequencies(32, 1e4, "ramp", 8.0, 4096)
        g, _ = pbs.rope(G.cuda(), None, pos.cuda(), freq, layout=layout, magnitude=mag, transpose=True)
        leaf = x.double().requires_grad_()
        y = rope_ref_differentiable(leaf, pos, freq.cpu(), layout, mag)
        (y * G.double()).sum().backward()
        _, e = rope_ref(G, pos, freq.cpu(), layout, mag, True)
        within(g, leaf.grad, e + H32 * (leaf.grad.abs() + e))
        step = torch.zeros_like(leaf)
        step[3, 1, 2] = 1e-3
        with torch.no_grad():
            hi = (rope_ref_differentiable(leaf + step, pos, freq.cpu(), layout, mag) * G.double()).sum()
            lo = (rope_ref_differentiable(leaf - step, pos, freq.cpu(), layout, mag) * G.double()).sum()
        assert abs(float((hi - lo) / 2e-3) - float(g[3, 1, 2])) < 1e-5     # linear in x: fp32 rounding of g is what is left


def rope_ref_differentiable(x, pos, freq, layout, mag):
    rot = 2 * freq.numel()
    ang = pos.double()[:, None, None] * freq
    cos, sin = ang.cos() * mag, ang.sin() * mag
    if layout == "half":
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        return torch.cat((a * cos - b * sin, a * sin + b * cos, x[..., rot:]), -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), x[..., rot:]), -1)


# ------------------------------------------------------------------------------------------------ cache
@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,h_kv,d,page", [(1, 1, 64, 16), (67, 8, 128, 32), (1000, 3, 64, 64), (513, 8, 128, 1024)])
def test_cache_rows(tokens, h_kv, d, page, dtype, held):
    dt, ht = TYPES[dtype], TYPES[held]
    pages = -(-tokens // page) + 3
    c = pbs.Cache.alloc(pages, page, h_kv, d, ht)
    marks = torch.randint(0, 120, c.K.view(torch.uint8).shape, generator=_gen(9), dtype=torch.uint8).cuda()
    c.K.view(torch.uint8).copy_(marks)
    c.V.view(torch.uint8).copy_(marks.flip(0))
    size = torch.exp(3 * _randn(3, tokens, h_kv, 1))
    K, V = (_randn(1, tokens, h_kv, d) * size).to(dt), (_randn(2, tokens, h_kv, d) * size).to(dt)
    K[0, 0] = 0.0                                          # a row of zeros; a row of one value; the smallest ones
    V[-1, -1] = -3.0
    if tokens > 3:
        K[1, 0] = 1e-38
        V[1, 0, 0] = math.inf
        K[2, 0, 5] = math.nan
        V[3, 0, 7] = -math.inf
    slots = torch.randperm(pages * page, generator=_gen(4))[:tokens].to(torch.int32)
    passed = torch.zeros(tokens, dtype=torch.bool)
    if tokens > 3:                                         # padding
        for i, bad in ((5, -1), (6, pages * page), (7, 2 ** 31 - 1), (8, -2 ** 31)):
            slots[i], passed[i] = bad, True
    want = {"K": c.K.cpu().clone(), "V": c.V.cpu().clone()}
    fact = {"K": None, "V": None} if held == "bf16" else {"K": c.k_scale.cpu().clone(), "V": c.v_scale.cpu().clone()}
    back = {}
    for name, x in (("K", K), ("V", V)):
        q, f = hold_ref(x, ht)
        raw = want[name].view(torch.uint8 if held != "bf16" else torch.int16)
        for t in range(tokens):
            if not passed[t]:
                raw[int(slots[t]) // page, :, int(slots[t]) % page] = q[t].view(raw.dtype)
                if f is not None:
                    fact[name][int(slots[t]) // page, :, int(slots[t]) % page] = f[t]
        back[name] = stands_for(q, f)
        back[name][passed] = 0.0
    pbs.cache_write(c, K.cuda(), V.cuda(), slots.cuda())
    bits = torch.int16 if held == "bf16" else torch.uint8
    for name, got, factors in (("K", c.K, c.k_scale), ("V", c.V, c.v_scale)):
        a, b = got.cpu().view(bits), want[name].view(bits)
        if held == "bf16":                                 # a NaN's bits are not looked at
            a, b = torch.where(torch.isnan(got.cpu()), 0, a), torch.where(torch.isnan(want[name]), 0, b)
        assert torch.equal(a, b), name                     # bit for bit, and nothing else touched
        if factors is not None:
            assert torch.equal(factors.cpu().nan_to_num(-1.0), fact[name].nan_to_num(-1.0)), name
    for out in ("bf16", "f32"):
        k, v = pbs.cache_read(c, slots.cuda(), out)
        for got, name in ((k, "K"), (v, "V")):
            assert torch.equal(got.cpu().nan_to_num(-7.0, -8.0, -9.0), back[name].to(TYPES[out]).nan_to_num(-7.0, -8.0, -9.0)), (out, name)


def test_cache_strided_rows_and_repeated_reads():
    c = pbs.Cache.alloc(4, 32, 2, 128, torch.float8_e4m3fn)
    fused = _randn(1, 50, 6, 128).bfloat16().cuda()
    slots = torch.arange(50, dtype=torch.int32).cuda()
    pbs.cache_write(c, fused[:, 2:4], fused[:, 4:6], slots)
    twice = torch.cat((slots, slots.flip(0)))
    out = torch.full((100, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    pbs.cache_read(c, twice, K=out[:, :2], V=out[:, 2:])
    for at, x in ((0, fused[:, 2:4]), (2, fused[:, 4:6])):
        want = stands_for(*hold_ref(x.cpu(), torch.float8_e4m3fn)).bfloat16()
        assert torch.equal(out[:50, at:at + 2].cpu(), want) and torch.equal(out[50:, at:at + 2].cpu(), want.flip(0))


def test_cache_whose_rows_lie_beyond_4_gib():
    # 5 GiB of bf16 pages: byte offsets pass 32 bits
    pages = 5 * (1 << 30) // (256 * 8 * 128 * 2)
    c = pbs.Cache.alloc(pages, 256, 8, 128)
    slots = torch.tensor([0, pages * 256 - 1, pages * 128 + 3], dtype=torch.int32)
    K, V = _randn(1, 3, 8, 128).bfloat16(), _randn(2, 3, 8, 128).bfloat16()
    pbs.cache_write(c, K.cuda(), V.cuda(), slots.cuda())
    k, v = pbs.cache_read(c, slots.cuda())
    assert torch.equal(k.cpu(), K) and torch.equal(v.cpu(), V)
    assert torch.equal(c.K[-1, :, -1].cpu(), K[1])
    # and the attention reads them there: one sequence in the last page, ten keys
    ten = torch.arange(10, dtype=torch.int32) + (pages - 1) * 256
    K, V = _randn(3, 10, 8, 128).bfloat16(), _randn(4, 10, 8, 128).bfloat16()
    pbs.cache_write(c, K.cuda(), V.cuda(), ten.cuda())
    Q = _randn(5, 1, 1, 8, 128).bfloat16()
    O = pbs.decode_attn(c, Q.cuda(), torch.tensor([[pages - 1]], dtype=torch.int32).cuda(), torch.tensor([10], dtype=torch.int32).cuda())
    for h in range(8):
        want, _, bound, _ = attention_ref(Q[0, :, h], K[:, h], V[:, h], torch.ones(1, 10, dtype=torch.bool), 1 / math.sqrt(128))
        within(O[0, :, h], want, bound)


# ------------------------------------------------------------------------------------------------ decode
class Setup:
    """A cache with sequences and a prefix in shuffled pages; every slot that no key lies in is filled with NaN."""

    def __init__(self, seed, q_len, h_q, h_kv, d, held, page, lens, prefix=0, spare=3):
        self.q_len, self.h_q, self.h_kv, self.d, self.page, self.lens, self.prefix = q_len, h_q, h_kv, d, page, lens, prefix
        need = [-(-n // page) for n in lens]
        pre = -(-prefix // page)
        pages = sum(need) + pre + spare
        order = torch.randperm(pages, generator=_gen(seed))
        ht = TYPES[held]
        self.cache = c = pbs.Cache.alloc(pages, page, h_kv, d, ht)
        if held == "i8":
            for f in (c.k_scale, c.v_scale):
                f.fill_(math.nan)
        else:
            for x in (c.K, c.V):
                x.view(torch.uint8).fill_(0x7f if held == "e4m3" else 0xff)
            if held == "e4m3":
                c.k_scale.fill_(1.0)
                c.v_scale.fill_(math.nan)
        self.table = torch.full((len(lens), max(need + [1])), -1, dtype=torch.int32)
        slots, at = [], 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.prefix_pages = order[at:at + pre].to(torch.int32)
        lines = [self.table[i] for i in range(len(lens))] + [self.prefix_pages]
        counts = list(lens) + [prefix]
        self.k, self.v = [], []
        for i, (line, n) in enumerate(zip(lines, counts)):
            K, V = _randn(seed + 10 + i, n, h_kv, d).bfloat16(), (2 * _randn(seed + 500 + i, n, h_kv, d)).bfloat16()
            j = torch.arange(n)
            slots = (line[j // page].long() * page + j % page).to(torch.int32)
            if n:
                pbs.cache_write(c, K.cuda(), V.cuda(), slots.cuda())
            self.k.append(stands_for(*hold_ref(K, ht)))
            self.v.append(stands_for(*hold_ref(V, ht)))
        self.Q = (1.5 * _randn(seed + 1, len(lens), q_len, h_q, d)).bfloat16()

    def call(self, Q=None, **kw):
        return pbs.decode_attn(self.cache, self.Q.cuda() if Q is None else Q, self.table.cuda(),
                               torch.tensor(self.lens, dtype=torch.int32).cuda(),
                               prefix_pages=self.prefix_pages.cuda() if self.prefix else None, prefix_len=self.prefix, **kw)

    def check(self, O, lse=None, hidden=None, scale=None):
        r, P = self.h_q // self.h_kv, self.prefix
        for i, n in enumerate(self.lens):
            t, j = torch.arange(self.q_len)[:, None], torch.arange(P + n)[None]
            sees = j < P + n - self.q_len + 1 + t
            sees |= j < P
            sees &= j < P + n
            if hidden is not None:
                sees = sees & ~hidden(i, j)
            for h in range(self.h_q):
                k = torch.cat((self.k[-1][:, h // r], self.k[i][:, h // r]))
                v = torch.cat((self.v[-1][:, h // r], self.v[i][:, h // r]))
                o, l, bo, bl = attention_ref(self.Q[i, :, h], k, v, sees, scale or 1 / math.sqrt(self.d))
                within(O[i, :, h], o, bo, "O of sequence %d (%d keys), head %d" % (i, n, h))
                if lse is not None:
                    within(lse[i, :, h], l, bl, "lse of sequence %d, head %d" % (i, h))


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
def test_decode_lengths(held, d, page):
    s = Setup(1, 1, 8, 2, d, held, page, [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 500])
    O, lse = s.call(want_lse=True)
    s.check(O, lse)
    assert float(O[0].abs().max()) == 0.0 and bool((lse[0] == -math.inf).all())


@pytest.mark.parametrize("q_len,h_q,h_kv", [(1, 1, 1), (2, 7, 1), (3, 14, 2), (5, 16, 2), (16, 4, 4), (16, 12, 1), (1, 40, 1), (4, 128, 1)])
def test_decode_several_new_tokens_and_head_groups(q_len, h_q, h_kv):
    s = Setup(2, q_len, h_q, h_kv, 64 if h_q > 14 else 128, "bf16", 32, [q_len - 1, q_len, 1, 77, 200])
    O, lse = s.call(want_lse=True)
    s.check(O, lse)


# units enough that a wave joins a row, or takes a whole unit; one long sequence has more pieces than a wave joins
@pytest.mark.parametrize("n,q_len,h_q,h_kv,d,held,longest,one", [(140, 1, 8, 8, 64, "bf16", 40, 9000), (131, 1, 16, 8, 128, "e4m3", 300, 300),
                                                                 (70, 5, 32, 8, 64, "bf16", 60, 5000), (67, 1, 16, 8, 128, "bf16", 256, 256),
                                                                 (65, 2, 8, 8, 64, "i8", 256, 200), (515, 1, 8, 8, 64, "e4m3", 511, 512)])
def test_decode_many_sequences(n, q_len, h_q, h_kv, d, held, longest, one):
    lens = [(37 * i) % (longest + 1) for i in range(n)]
    lens[n // 3] = one
    s = Setup(5, q_len, h_q, h_kv, d, held, 32, lens)
    O, lse = s.call(want_lse=True, max_len=max(lens))
    s.check(O, lse)


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("n_seq,q_len,h_q,h_kv,d,prefix", [(1, 1, 2, 2, 64, 1), (3, 1, 8, 2, 128, 100), (9, 1, 28, 4, 128, 333), (5, 4, 8, 1, 64, 1025)])
def test_decode_shared_prefix(n_seq, q_len, h_q, h_kv, d, prefix, held):
    lens = [0 if q_len == 1 else 1, 40, 3, 130, 17, 1, 64, 65, 2][:n_seq]
    s = Setup(3, q_len, h_q, h_kv, d, held, 16, lens, prefix)
    O, lse = s.call(want_lse=True)
    s.check(O, lse)


@pytest.mark.parametrize("held", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("h_q,h_kv,d,page,prefix", [(8, 2, 128, 16, 1), (8, 1, 128, 64, 127), (8, 2, 64, 32, 128), (16, 4, 64, 16, 129), (12, 1, 128, 128, 1500),
                                                    (7, 1, 64, 256, 3333)])
def test_decode_prefix_of_a_large_batch(h_q, h_kv, d, page, prefix, held):
    # more rows than a wave takes: several workgroups of 128, the last one partly filled
    n = 13 if prefix < 1000 else 21
    s = Setup(30, 1, h_q, h_kv, d, held, page, [(5 * i) % 40 for i in range(n)], prefix)
    O, lse = s.call(want_lse=True)
    s.check(O, lse)
    again = s.call()
    assert torch.equal(O, again)


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_decode_prefix_of_a_large_batch_with_odd_pages_and_values(held):
    s = Setup(31, 1, 16, 2, 128, held, 16, [3] * 9, 300)
    s.prefix_pages[4], s.prefix_pages[11] = -1, 77777

    def hidden(i, j):
        return ((j >= 64) & (j < 80)) | ((j >= 176) & (j < 192))

    O, lse = s.call(want_lse=True)
    s.check(O, lse, hidden)
    # a value that is not finite in a key that everybody sees
    page = int(s.prefix_pages[2])
    if held == "bf16":
        s.cache.V[page, 1, 3, 9] = math.inf
    else:
        s.cache.v_scale[page, 1, 3] = math.nan
    got = s.call().float().cpu()
    assert torch.isfinite(got[:, :, :8]).all()
    if held == "bf16":
        assert (got[:, :, 8:, 9] == math.inf).all()
        got[:, :, 8:, 9] = 0
        assert torch.isfinite(got).all()
    else:
        assert torch.isnan(got[:, :, 8:]).all()


def test_decode_prefix_of_a_large_batch_in_place_with_values_that_are_not_finite():
    # the prefix alone, in one part: rows that are formed again read their queries again, and O is Q
    s = Setup(33, 1, 40, 1, 64, "bf16", 16, [0], 90)
    s.cache.V[int(s.prefix_pages[1]), 0, 4, 5] = math.inf
    want = s.call()
    Q = s.Q.cuda()
    assert torch.equal(s.call(Q=Q, O=Q, max_len=0), want) and bool((want[..., 5] == math.inf).all())


# rows times keys large enough for the kernel with 128 rows to a workgroup; the last part of the prefix has 65, 1, 127, 5 keys
@pytest.mark.parametrize("n,h_q,h_kv,d,page,prefix", [(8, 16, 1, 64, 16, 4161), (9, 16, 1, 128, 16, 4097), (7, 32, 2, 128, 64, 2431),
                                                      (5, 32, 1, 64, 256, 3333)])
def test_decode_prefix_of_thousands_of_rows(n, h_q, h_kv, d, page, prefix):
    s = Setup(34, 16, h_q, h_kv, d, "bf16", page, [(5 * i) % 40 for i in range(n)], prefix)
    O, lse = s.call(want_lse=True)
    s.check(O, lse)
    assert torch.equal(O, s.call())


@pytest.mark.parametrize("held,n,h_q,h_kv,d,page,prefix", [("e4m3", 9, 32, 1, 64, 16, 3700), ("i8", 10, 32, 2, 128, 32, 3329),
                                                           ("e4m3", 10, 32, 2, 128, 128, 3383)])
def test_decode_prefix_of_thousands_of_rows_8_bit(held, n, h_q, h_kv, d, page, prefix):
    s = Setup(35, 16, h_q, h_kv, d, held, page, [(5 * i) % 40 for i in range(n)], prefix)
    O, lse = s.call(want_lse=True)
    s.check(O, lse)
    assert torch.equal(O, s.call())


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_decode_prefix_of_thousands_of_rows_with_odd_pages_and_values(held):
    n, prefix = (9, 4300) if held == "bf16" else (18, 4300)
    s = Setup(36, 16, 16, 1, 128, held, 16, [3] * n, prefix)
    s.Q *= 8                                               # logits that grow
    s.prefix_pages[4], s.prefix_pages[11], s.prefix_pages[-1] = -1, 77777, -1

    def hidden(i, j):
        return ((j >= 64) & (j < 80)) | ((j >= 176) & (j < 192)) | ((j >= 4288) & (j < 4300))

    O, lse = s.call(want_lse=True)
    s.check(O, lse, hidden)
    page = int(s.prefix_pages[2])
    if held == "bf16":
        s.cache.V[page, 0, 3, 9] = math.inf
        got = s.call().float().cpu()
        assert not torch.isfinite(got[..., 9]).any()       # its probability may be 0: NaN
        got[..., 9] = 0
        assert torch.isfinite(got).all()
    else:
        s.cache.v_scale[page, 0, 3] = math.nan
        assert torch.isnan(s.call()).all()


def test_decode_prefix_of_thousands_of_rows_in_place_with_values_that_are_not_finite():
    # the prefix alone, in one part: rows that are formed again read their queries again, and O is Q
    s = Setup(37, 16, 4, 4, 64, "bf16", 16, [0] * 1024, 200)
    s.cache.V[int(s.prefix_pages[1]), :, 4, 5] = math.inf
    want = s.call()
    Q = s.Q.cuda()
    assert torch.equal(s.call(Q=Q, O=Q, max_len=0), want) and bool((want[..., 5] == math.inf).all())


def test_decode_prefix_of_a_large_batch_logits_that_grow():
    s = Setup(32, 1, 40, 1, 128, "i8", 32, [5], 900)
    s.Q *= 30                                              # hundreds of nats between keys
    O, lse = s.call(want_lse=True)
    s.check(O, lse)


def test_decode_prefix_alone_and_nothing_at_all():
    s = Setup(4, 1, 8, 2, 128, "bf16", 16, [0, 0, 0], 50)
    O, lse = s.call(want_lse=True)
    s.check(O, lse)
    O, lse = s.call(want_lse=True, max_len=0)
    s.check(O, lse)
    s = Setup(4, 1, 8, 2, 128, "bf16", 16, [0, 0])
    O, lse = s.call(want_lse=True, max_len=0)
    assert float(O.abs().max()) == 0.0 and bool((lse == -math.inf).all())


@pytest.mark.parametrize("held", ["bf16", "e4m3"])
def test_decode_long_sequences_in_many_parts(held):
    s = Setup(5, 1, 4, 1, 128, held, 128, [9001, 1, 4097, 4095], 5000)
    O, lse = s.call(want_lse=True)
    s.check(O, lse)
    again, lse2 = s.call(want_lse=True)
    assert torch.equal(O, again) and torch.equal(lse, lse2)
    # another bound on the lengths cuts the work elsewhere; the result is the same up to the order of sums
    O, lse = s.call(want_lse=True, max_len=9001)
    s.check(O, lse)


def test_decode_pages_that_are_none_count_as_keys_nobody_sees():
    s = Setup(6, 2, 8, 2, 64, "bf16", 16, [100, 64], 48)
    s.table[0, 2], s.table[1, 3] = -5, 1 << 30
    s.prefix_pages[1] = 9999
    P = s.prefix

    def hidden(i, j):
        own = (j >= P + 32) & (j < P + 48) if i == 0 else (j >= P + 48) & (j < P + 64)
        return own | ((j >= 16) & (j < 32))

    O, lse = s.call(want_lse=True)
    s.check(O, lse, hidden)


def test_decode_lengths_beyond_their_bound_are_cut_there():
    s = Setup(7, 1, 4, 2, 64, "bf16", 16, [100, 30])
    full = s.call()
    given = s.lens
    s.lens = [60, 30]
    want = s.call()
    s.lens = given
    assert torch.equal(s.call(max_len=60), want) and not torch.equal(full, want)
    s.lens = [-3, 1000]
    O, lse = s.call(want_lse=True)                         # the second reads page_table's entries of -1 behind its 30 keys
    assert float(O[0].abs().max()) == 0.0


def test_decode_values_that_are_not_finite():
    # in a key that the second new token sees and the first does not, and in one that all see
    s = Setup(8, 2, 8, 2, 128, "bf16", 16, [70, 64, 33])
    for i, n in enumerate(s.lens):
        page, at = int(s.table[i, (n - 1) // 16]), (n - 1) % 16
        for place, what in ((3, math.inf), (64, -math.inf), (90, math.nan)):
            s.cache.V[page, :, at, place] = what
            s.v[i][n - 1, :, place] = what
    s.cache.V[int(s.table[0, 0]), :, 5, 7] = -math.inf
    s.v[0][5, :, 7] = -math.inf
    O, lse = s.call(want_lse=True)
    got = O.float().cpu()
    assert torch.isfinite(got[:, 0, :, 8:]).all() and torch.isfinite(got[1:, 0]).all()
    assert (got[:, 1, :, 3] == math.inf).all() and (got[:, 1, :, 64] == -math.inf).all() and torch.isnan(got[:, 1, :, 90]).all()
    assert (got[0, :, :, 7] == -math.inf).all()
    for x in s.v:
        x.nan_to_num_(0.0, 0.0, 0.0)
    clean = torch.ones(s.d, dtype=torch.bool)
    clean[[3, 7, 64, 90]] = False
    s.cache.V.nan_to_num_(0.0, 0.0, 0.0)
    ref = s.call()
    assert torch.equal(ref[..., clean.cuda()], O[..., clean.cuda()])
    s.check(ref, lse)


def test_decode_logits_that_are_not_finite():
    s = Setup(9, 1, 4, 2, 64, "bf16", 16, [50, 50])
    s.Q[0, 0, 1, 3] = math.nan
    s.cache.K[int(s.table[1, 1]), 1, 4, 0] = math.nan      # a key of the second kv head
    O, lse = s.call(want_lse=True)
    got, l = O.float().cpu(), lse.cpu()
    bad = torch.zeros(2, 4, dtype=torch.bool)
    bad[0, 1] = bad[1, 2] = bad[1, 3] = True
    assert torch.isnan(got[:, 0][bad]).all() and torch.isnan(l[:, 0][bad]).all()
    assert torch.isfinite(got[:, 0][~bad]).all() and torch.isfinite(l[:, 0][~bad]).all()


def test_decode_large_logits_and_a_scale_of_the_callers():
    s = Setup(10, 1, 4, 2, 128, "bf16", 16, [300, 20])
    s.Q *= 40                                              # hundreds of nats between keys
    O, lse = s.call(want_lse=True, scale=0.25)
    s.check(O, lse, scale=0.25)


def test_decode_strided_queries_and_outputs():
    s = Setup(11, 2, 8, 2, 64, "e4m3", 32, [45, 90], 20)
    want = s.call()
    fused = torch.zeros(2, 2, 12, 64, dtype=torch.bfloat16, device="cuda")
    fused[:, :, :8] = s.Q.cuda()
    out = torch.full((8, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")     # [heads, tokens, d]
    view = out.view(8, 2, 2, 64).permute(1, 2, 0, 3)
    s.call(Q=fused[:, :, :8], O=view)
    assert torch.equal(view, want)
    O = s.call(Q=fused[:, :, :8], O=fused[:, :, :8])       # in place
    assert torch.equal(O, want) and float(fused[:, :, 8:].abs().max()) == 0.0


def test_decode_on_another_stream_and_captured():
    s = Setup(12, 1, 8, 2, 128, "bf16", 16, [2000, 700, 31], 600)
    want = s.call()
    Q, table, lens, pre = s.Q.cuda(), s.table.cuda(), torch.tensor(s.lens, dtype=torch.int32).cuda(), s.prefix_pages.cuda()
    O = torch.zeros_like(Q)

    def step():
        return pbs.decode_attn(s.cache, Q, table, lens, prefix_pages=pre, prefix_len=s.prefix, O=O)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(O, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):                                     # other lengths and queries in the same memory
        Q.copy_((1.0 + k) * s.Q.cuda())
        lens.copy_(torch.tensor([2000 - 500 * k, 700, 31 - k], dtype=torch.int32))
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone()
        eager = pbs.decode_attn(s.cache, Q, table, lens, prefix_pages=pre, prefix_len=s.prefix)
        assert torch.equal(got, eager)


# ------------------------------------------------------------------------------------------------ prompts
def _cu(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32)


def _prompts(seed, lens, before, h_q, h_kv, d):
    keys = [n + b for n, b in zip(lens, before)]
    Q = (1.5 * _randn(seed, sum(lens), h_q, d)).bfloat16()
    K, V = _randn(seed + 1, sum(keys), h_kv, d).bfloat16(), (2 * _randn(seed + 2, sum(keys), h_kv, d)).bfloat16()
    return Q, K, V, _cu(lens), _cu(keys)


def _check_prompts(Q, K, V, cu_q, cu_k, O, lse, causal=True, scale=None, rows=None):
    r, d = Q.shape[1] // K.shape[1], Q.shape[2]
    for i in range(cu_q.numel() - 1):
        q0, q1, k0, k1 = int(cu_q[i]), int(cu_q[i + 1]), int(cu_k[i]), int(cu_k[i + 1])
        t = torch.arange(q1 - q0) if rows is None else torch.tensor([x for x in rows if x < q1 - q0], dtype=torch.int64)
        if t.numel() == 0:
            continue
        sees = torch.arange(k1 - k0)[None] <= t[:, None] + (k1 - k0) - (q1 - q0)
        if not causal:
            sees = torch.ones_like(sees)
        for h in range(Q.shape[1]):
            o, l, bo, bl = attention_ref(Q[q0 + t, h], K[k0:k1, h // r], V[k0:k1, h // r], sees, scale or 1 / math.sqrt(d))
            within(O[q0 + t, h], o, bo, "O of sequence %d, head %d" % (i, h))
            if lse is not None:
                within(lse[q0 + t, h], l, bl, "lse of sequence %d, head %d" % (i, h))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("h_q,h_kv,d", [(4, 1, 128), (8, 2, 64), (7, 1, 128), (3, 3, 64), (2, 2, 128)])
def test_prompt_lengths(h_q, h_kv, d, causal):
    lens = [1, 0, 2, 15, 17, 31, 32, 33, 0, 64, 65, 130, 1]
    Q, K, V, cu, _ = _prompts(20, lens, [0] * len(lens), h_q, h_kv, d)
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda(), causal=causal, want_lse=True)
    _check_prompts(Q, K, V, cu, cu, O, lse, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (5, 1, 64), (128, 1, 64), (96, 1, 128)])
def test_prompt_chunks_behind_keys_and_queries_that_see_none(h_q, h_kv, d, causal):
    lens, before = [3, 40, 1, 20, 7, 33, 5], [500, 1, 64, -8, -7, 31, -5]
    if h_q > 20:
        lens, before = lens[:5], [100, 1, 64, -8, -7]
    Q, K, V, cu_q, cu_k = _prompts(21, lens, before, h_q, h_kv, d)
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu_q.cuda(), cu_k.cuda(), causal=causal, want_lse=True)
    _check_prompts(Q, K, V, cu_q, cu_k, O, lse, causal)
    if causal:
        a = int(cu_q[3])
        assert float(O[a:a + 8].abs().max()) == 0.0 and bool((lse[a:a + 8] == -math.inf).all())


@pytest.mark.parametrize("h_q,h_kv,d", [(4, 1, 128), (2, 2, 128), (4, 2, 64)])
def test_prompt_long(h_q, h_kv, d):
    Q, K, V, cu_q, cu_k = _prompts(22, [2050, 700], [0, 1333], h_q, h_kv, d)
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu_q.cuda(), cu_k.cuda(), want_lse=True)
    _check_prompts(Q, K, V, cu_q, cu_k, O, lse, rows=[0, 1, 31, 32, 33, 127, 128, 255, 256, 511, 699, 1000, 1024, 2047, 2048, 2049])
    again, lse2 = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu_q.cuda(), cu_k.cuda(), want_lse=True)
    assert torch.equal(O, again) and torch.equal(lse, lse2)


def test_prompt_many_sequences():
    lens = [(7 * i) % 23 for i in range(200)]
    Q, K, V, cu, _ = _prompts(23, lens, [0] * 200, 4, 2, 64)
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda(), want_lse=True)
    _check_prompts(Q, K, V, cu, cu, O, lse)


def test_prompt_rows_of_no_sequence_stay_as_they_were():
    Q, K, V, cu_q, cu_k = _prompts(24, [5, 30, 10], [0, 0, 0], 4, 2, 128)
    O = torch.full((45, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((45, 4), 9.0, device="cuda")
    part = torch.tensor([2, 5, 35], dtype=torch.int32)     # rows 0, 1 and 35 .. belong to none
    pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), part.cuda(), part.cuda(), O=O, lse=lse)
    assert bool((O[:2] == 7).all()) and bool((O[35:] == 7).all()) and bool((lse[:2] == 9).all()) and bool((lse[35:] == 9).all())
    _check_prompts(Q, K, V, part, part, O, lse)
    # places outside the tensors are taken as the nearest inside
    wild = torch.tensor([-4, 5, 1000], dtype=torch.int32)
    got = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), wild.cuda())
    tame = torch.tensor([0, 5, 45], dtype=torch.int32)
    assert torch.equal(got, pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), tame.cuda()))


def test_prompt_strided():
    Q, K, V, cu, _ = _prompts(25, [50, 83], [0, 0], 8, 2, 64)
    want = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda())
    fused = torch.cat((Q, K, V), 1).cuda()                 # a fused projection
    O = torch.zeros(8, 133, 64, dtype=torch.bfloat16, device="cuda")           # [heads, n, d]
    pbs.prompt_attn(fused[:, :8], fused[:, 8:10], fused[:, 10:], cu.cuda(), O=O.transpose(0, 1))
    assert torch.equal(O.transpose(0, 1), want)
    heads = [x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (Q, K, V)]
    assert torch.equal(pbs.prompt_attn(*heads, cu.cuda()), want)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_values_that_are_not_finite(d):
    # keys 40 and 100 hold infinities and NaN: queries in front of them do not see it, nor does the next sequence
    Q, K, V, cu, _ = _prompts(26, [130, 64], [0, 0], 4, 1, d)
    V[40, 0, 3], V[40, 0, 4], V[100, 0, 5], V[100, 0, 6] = math.inf, -math.inf, math.nan, math.inf
    V[41, 0, 4] = math.inf
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda(), want_lse=True)
    got = O.float().cpu()
    assert torch.isfinite(got[:40]).all() and torch.isfinite(got[130:]).all()
    assert (got[40:130, :, 3] == math.inf).all() and (got[40, :, 4] == -math.inf).all() and torch.isnan(got[41:130, :, 4]).all()
    assert torch.isfinite(got[40:100, :, 5:]).all() and torch.isnan(got[100:130, :, 5]).all() and (got[100:130, :, 6] == math.inf).all()
    clean = [i for i in range(d) if i not in (3, 4, 5, 6)]
    V.nan_to_num_(0.0, 0.0, 0.0)
    ref, lse2 = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda(), want_lse=True)
    _check_prompts(Q, K, V, cu, cu, ref, lse2)
    # the other features: keys in tiles with such values are summed relative to another maximum than without, p e^(m - m') for
    # p, so that roundings differ; either is within the bound, each weight's rounding being relative to the weight
    mixed = ref.clone()
    mixed[..., clean] = O[..., clean]
    _check_prompts(Q, K, V, cu, cu, mixed, lse)


def test_prompt_logits_that_are_not_finite():
    Q, K, V, cu, _ = _prompts(27, [70, 40], [0, 0], 4, 2, 64)
    K[50, 1] = math.nan                                    # kv head 1: heads 2 and 3 from query 50 on
    Q[5, 0, 0] = math.nan
    Q[100, 3, 0] = math.inf
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda(), want_lse=True)
    bad = torch.zeros(110, 4, dtype=torch.bool)
    bad[50:70, 2:] = bad[5, 0] = bad[100, 3] = True
    got, l = O.float().cpu(), lse.cpu()
    assert torch.isnan(got[bad]).all() and torch.isfinite(got[~bad]).all() and torch.isfinite(l[~bad]).all() and torch.isnan(l[bad]).all()


def test_prompt_logits_that_grow_along_the_keys():
    # each tile's maximum far above the one before: hundreds of nats from the first key to the last, in steps and in one leap
    n, d = 600, 128
    Q, K, V, cu, _ = _prompts(28, [n], [0], 2, 1, d)
    Q = Q * 0.2
    for shape in ("steps", "leap", "fall"):
        u = torch.zeros(d)
        u[0] = 1.0
        Q[:, :, 0] = 8.0
        k = K.clone()
        ramp = torch.arange(n).float() * 0.5
        k[:, 0, 0] = {"steps": ramp, "leap": (torch.arange(n) >= 300).float() * 400, "fall": 300 - ramp}[shape].bfloat16()
        O, lse = pbs.prompt_attn(Q.cuda(), k.cuda(), V.cuda(), cu.cuda(), want_lse=True)
        _check_prompts(Q, k, V, cu, cu, O, lse, rows=[0, 31, 32, 64, 100, 299, 300, 301, 320, 500, 599])


def test_prompt_on_another_stream_and_captured():
    Q, K, V, cu, _ = [x.cuda() for x in _prompts(29, [300, 20, 77], [0, 0, 0], 8, 2, 128)]
    O = torch.zeros_like(Q)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pbs.prompt_attn(Q, K, V, cu, O=O)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(O, pbs.prompt_attn(Q, K, V, cu))
    with torch.cuda.graph(graph):
        pbs.prompt_attn(Q, K, V, cu, O=O)
    for k in range(3):                                     # other inputs and other lengths in the same memory
        V.mul_(1.5)
        cu.copy_(torch.tensor([0, 300 - 50 * k, 320, 397], dtype=torch.int32))
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, pbs.prompt_attn(Q, K, V, cu))


@pytest.mark.parametrize("prefix", [0, 40])
def test_logits_that_are_all_minus_infinity_count_as_no_key(prefix):
    s = Setup(40, 1, 4, 1, 64, "bf16", 16, [50, 500], prefix)
    s.cache.K[..., 0] = -3e38
    s.Q[:, :, 2, 0] = 3e38                                 # their product leaves float32's range
    s.Q[:, :, [0, 1, 3], 0] = 0
    O, lse = s.call(want_lse=True)
    assert not O[:, :, 2].any() and bool((lse[:, :, 2] == -math.inf).all())
    assert bool(torch.isfinite(lse[:, :, [0, 1, 3]]).all()) and bool(torch.isfinite(O.float()).all())
    Q, K, V, cu, _ = _prompts(41, [70, 300], [0, 0], 4, 1, 64)
    K[..., 0] = -3e38
    Q[:, 2, 0] = 3e38
    Q[:, [0, 1, 3], 0] = 0
    O, lse = pbs.prompt_attn(Q.cuda(), K.cuda(), V.cuda(), cu.cuda(), want_lse=True)
    assert not O[:, 2].any() and bool((lse[:, 2] == -math.inf).all())
    assert bool(torch.isfinite(lse[:, [0, 1, 3]]).all()) and bool(torch.isfinite(O.float()).all())
