"""The operators around the prefill path without a GPU: refusals before any launch, the frequencies of rotary pairs."""
import ctypes
import math
import os

import pytest
import torch

from paper_2510_21270_amd import binding as b


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2510_21270_amd import build
        build.build()
    return b.load_library()


FAKE = ctypes.c_void_p(4096)                               # never dereferenced: calls below are refused first
ODD = ctypes.c_void_p(4096 + 8)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rope(**kw):
    x = dict(tokens=10, h_q=4, h_kv=2, d=64, rot=64, layout=0, dtype=1, magnitude=1.0, flags=0)
    x.update(kw)
    p = b.pbs_rope_problem(**x)
    p.q = p.q_out = b.pbs_strides(4 * 64, 64)
    p.k = p.k_out = b.pbs_strides(2 * 64, 64)
    return p


def test_rope_refusals(lib):
    def call(p, freq=FAKE, pos=FAKE, Q=FAKE, K=FAKE, Qo=FAKE, Ko=FAKE):
        return lib.pbs_rope(ctypes.byref(p) if p is not None else None, freq, pos, Q, K, Qo, Ko, None)

    assert call(None) == 1
    for name in ("freq", "pos", "Q", "K", "Qo", "Ko"):
        assert call(_rope(), **{name: None}) == 1, name
    assert call(_rope(tokens=0)) == 0                      # nothing to do
    for kw in (dict(tokens=-1), dict(h_q=-1), dict(h_q=0, h_kv=0), dict(magnitude=math.nan), dict(magnitude=math.inf)):
        assert call(_rope(**kw)) == 2, kw
    for kw in (dict(d=96), dict(rot=8), dict(rot=80), dict(rot=24), dict(layout=2), dict(dtype=2), dict(tokens=2 ** 31 - 1)):
        assert call(_rope(**kw)) == 3, kw
    assert call(_rope(), Q=ODD) == 2 and call(_rope(), Ko=ODD) == 2 and call(_rope(), freq=ctypes.c_void_p(4100)) == 2
    p = _rope()
    p.q = b.pbs_strides(256, 4)                            # 8 bytes
    assert call(p) == 2
    p = _rope()
    p.q_out = b.pbs_strides(0, 64)                         # rows of the output on top of each other
    assert call(p, Qo=ctypes.c_void_p(1 << 20)) == 2
    p = _rope()
    p.k_out = b.pbs_strides(64, 64)
    assert call(p, Ko=ctypes.c_void_p(1 << 20)) == 2
    p = _rope()
    p.q_out = b.pbs_strides(64, 640)                       # in place with other strides
    assert call(p) == 2
    p = _rope()
    p.q = b.pbs_strides(-256, 64)
    assert call(p) == 2


def test_rope_frequencies_against_their_formulas(lib):
    rot, base, original = 128, 5e5, 8192

    def freq(*a):
        table, mag = (ctypes.c_double * 64)(), ctypes.c_double(0)
        assert lib.pbs_rope_frequencies(*a, table, ctypes.byref(mag)) == 0
        return torch.tensor(list(table), dtype=torch.float64), mag.value

    e = torch.arange(64, dtype=torch.float64)
    plain = base ** (-2 * e / rot)
    got, mag = freq(0, rot, base, 1.0, original, 1.0, 4.0)
    assert mag == 1.0 and torch.allclose(got, plain, rtol=1e-14)
    got, mag = freq(1, rot, base, 8.0, original, 1.0, 4.0)
    assert mag == 1.0 and torch.allclose(got, plain / 8, rtol=1e-14)
    got, mag = freq(2, rot, base, 8.0, original, 1.0, 4.0)
    wave = 2 * math.pi / plain
    assert mag == 1.0
    assert torch.allclose(got[wave < original / 4], plain[wave < original / 4], rtol=1e-14)
    assert torch.allclose(got[wave > original], plain[wave > original] / 8, rtol=1e-14)
    mid = (wave > original / 4) & (wave < original)
    assert mid.any()
    keep = (original / wave[mid] - 1) / 3
    assert torch.allclose(got[mid], plain[mid] * keep + plain[mid] / 8 * (1 - keep), rtol=1e-13)
    got, mag = freq(3, rot, base, 8.0, original, 1.0, 32.0)
    assert abs(mag - (0.1 * math.log(8.0) + 1)) < 1e-15
    lo = math.floor(rot * math.log(original / (32 * 2 * math.pi)) / (2 * math.log(base)))
    hi = math.ceil(rot * math.log(original / (1 * 2 * math.pi)) / (2 * math.log(base)))
    assert torch.allclose(got[: lo + 1], plain[: lo + 1], rtol=1e-14) and torch.allclose(got[hi:], plain[hi:] / 8, rtol=1e-14)
    part = (torch.arange(lo, hi, dtype=torch.float64) - lo) / (hi - lo)
    assert torch.allclose(got[lo:hi], plain[lo:hi] * (1 - part) + plain[lo:hi] / 8 * part, rtol=1e-13)


def test_rope_frequency_refusals(lib):
    t, m = (ctypes.c_double * 64)(), ctypes.c_double(0)

    def call(scaling=2, rot=64, base=1e4, factor=2.0, original=4096.0, low=1.0, high=4.0, table=t, mag=ctypes.byref(m)):
        return lib.pbs_rope_frequencies(scaling, rot, base, factor, original, low, high, table, mag)

    assert call() == 0 and call(table=None) == 1 and call(mag=None) == 1
    assert call(scaling=4) == 3 and call(scaling=-1) == 3
    for kw in (dict(rot=0), dict(rot=63), dict(base=1.0), dict(base=math.nan), dict(factor=0.5), dict(factor=math.inf),
               dict(original=0.0), dict(low=0.0), dict(high=1.0), dict(high=math.nan)):
        assert call(**kw) == 2, kw
    assert call(scaling=0, factor=0.0, original=0.0, low=0.0) == 0             # not looked at


def _cache(**kw):
    x = dict(pages=8, page=16, h_kv=2, d=64, dtype=1, K=4096, V=4096, k_scale=None, v_scale=None)
    x.update(kw)
    return b.pbs_cache(**x)


BAD_CACHES = [(dict(pages=0), 2), (dict(h_kv=0), 2), (dict(page=0), 2), (dict(page=8), 3), (dict(page=48), 3), (dict(page=2048), 3),
              (dict(d=96), 3), (dict(dtype=0), 3), (dict(dtype=4), 3), (dict(pages=2 ** 27), 3), (dict(K=None), 1), (dict(V=None), 1),
              (dict(dtype=2), 1), (dict(dtype=3, k_scale=4096), 1), (dict(K=4104), 2), (dict(dtype=3, k_scale=4096, v_scale=4100), 2)]


def test_cache_refusals(lib):
    s = b.pbs_strides(128, 64)

    def write(c=_cache(), dtype=1, tokens=4, K=FAKE, k=s, V=FAKE, v=s, slots=FAKE):
        return lib.pbs_cache_write(_ref(c), dtype, tokens, K, _ref(k), V, _ref(v), slots, None)

    def read(c=_cache(), dtype=1, tokens=4, slots=FAKE, K=FAKE, k=s, V=FAKE, v=s):
        return lib.pbs_cache_read(_ref(c), dtype, tokens, slots, K, _ref(k), V, _ref(v), None)

    for call in (write, read):
        assert call(c=None) == 1 and call(slots=None) == 1
        assert call(tokens=0) == 0 and call(tokens=-1) == 2
        assert call(dtype=2) == 3 and call(tokens=2 ** 30) == 3
        assert call(K=ODD) == 2 and call(V=ODD) == 2 and call(slots=ctypes.c_void_p(4097)) == 2
        assert call(k=b.pbs_strides(128, 60)) == 2 and call(k=None) == 1
        for kw, st in BAD_CACHES:
            assert call(c=_cache(**kw)) == st, kw
    assert write(K=None) == 1 and write(V=None) == 1 and read(K=None, V=None) == 1
    assert read(k=b.pbs_strides(64, 64)) == 2              # rows of the output on top of each other


def _decode(**kw):
    x = dict(n_seq=3, q_len=1, h_q=4, max_pages=5, max_len=80, prefix_len=0, dtype=1, scale=0.0)
    x.update(kw)
    p = b.pbs_decode_problem(**x)
    p.q = p.o = b.pbs_strides(4 * 64, 64)
    return p


def test_decode_refusals(lib):
    def call(p=None, c=_cache(), Q=FAKE, table=FAKE, lens=FAKE, prefix=FAKE, O=FAKE, lse=None, ws=FAKE, n=1 << 40):
        p = _decode() if p is None else p
        return lib.pbs_decode_attn(ctypes.byref(p), ctypes.byref(c), Q, table, lens, prefix, O, lse, ws, n, None)

    assert lib.pbs_decode_attn(None, ctypes.byref(_cache()), FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == 1
    assert lib.pbs_decode_attn(ctypes.byref(_decode()), None, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == 1
    for name in ("Q", "table", "lens", "O"):
        assert call(**{name: None}) == 1, name
    assert call(_decode(prefix_len=5), prefix=None) == 1
    assert call(_decode(n_seq=0), Q=None) == 0 and call(_decode(n_seq=0, prefix_len=100), Q=None) == 0
    for kw in (dict(n_seq=-1), dict(q_len=0), dict(h_q=0), dict(h_q=3), dict(max_pages=-1), dict(max_len=-1), dict(prefix_len=-1),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf)):
        assert call(_decode(**kw)) == 2, kw
    for kw in (dict(q_len=17), dict(dtype=0), dict(n_seq=70000), dict(n_seq=60000, max_pages=60000), dict(prefix_len=2 ** 31 - 1),
               dict(prefix_len=2 ** 25 + 1), dict(max_len=2 ** 27 + 1)):
        assert call(_decode(**kw)) == 3, kw
    for kw, st in BAD_CACHES:
        assert call(c=_cache(**kw)) == st, kw
    assert call(Q=ODD) == 2 and call(O=ODD) == 2 and call(lse=ctypes.c_void_p(4098)) == 2
    p = _decode(prefix_len=1000)
    need = lib.pbs_decode_workspace_bytes(ctypes.byref(p), ctypes.byref(_cache()))
    assert need > 0
    assert call(p, ws=None) == 1 and call(p, n=need - 1) == 4 and call(p, ws=ODD) == 4
    assert lib.pbs_decode_workspace_bytes(ctypes.byref(_decode(max_len=16)), ctypes.byref(_cache())) == 0   # one part
    assert lib.pbs_decode_workspace_bytes(ctypes.byref(_decode(q_len=0)), ctypes.byref(_cache())) == 0


def test_packed_arguments_are_the_structures():
    import struct
    for made, of, args in ((b._ROPE, b.pbs_rope_problem, tuple(range(1, 8)) + (0.5, 9) + tuple(range(10, 18))),
                           (b._CACHE, b.pbs_cache, (1, 2, 3, 4, 5, 6, 7, 8, 9)),
                           (b._DECODE, b.pbs_decode_problem, (1, 2, 3, 4, 5, 6, 7, 0.25, 9, 10, 11, 12)),
                           (b._PROMPT, b.pbs_prompt_problem, tuple(range(1, 8)) + (0.5, 9) + tuple(range(10, 18))),
                           (b._STRIDES, b.pbs_strides, (3, 4))):
        raw = made(*args)
        assert len(raw) == ctypes.sizeof(of)
        x, flat = of.from_buffer_copy(raw), []
        for name, _ in of._fields_:
            v = getattr(x, name)
            flat += [v.token, v.head] if isinstance(v, b.pbs_strides) else [v]
        assert tuple(flat) == args, of
    assert struct.calcsize("P") == 8


def test_the_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(b.PbsError, match="not on the GPU"):
        b.rope(x, None, torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))
    with pytest.raises(b.PbsError, match="not on the GPU"):
        b.Cache(torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(b.PbsError, match="unknown scaling"):
        b.rope_frequencies(64, scaling="other", device="cpu")
    f, mag = b.rope_frequencies(64, 1e4, device="cpu")
    assert f.shape == (32,) and f.dtype == torch.float64 and mag == 1.0


def test_prompt_refusals(lib):
    def prob(**kw):
        x = dict(n_seq=2, total_q=10, total_k=12, h_q=4, h_kv=2, d=64, dtype=1, scale=0.0, flags=1)
        x.update(kw)
        p = b.pbs_prompt_problem(**x)
        p.q = p.o = b.pbs_strides(256, 64)
        p.k = p.v = b.pbs_strides(128, 64)
        return p

    def call(p=None, Q=FAKE, K=FAKE, V=FAKE, cu_q=FAKE, cu_k=FAKE, O=FAKE, lse=None):
        return lib.pbs_prompt_attn(ctypes.byref(prob() if p is None else p), Q, K, V, cu_q, cu_k, O, lse, None)

    assert lib.pbs_prompt_attn(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None) == 1
    for name in ("Q", "K", "V", "cu_q", "cu_k", "O"):
        assert call(**{name: None}) == 1, name
    assert call(prob(n_seq=0), Q=None) == 0 and call(prob(total_q=0), O=None) == 0
    for kw in (dict(n_seq=-1), dict(total_q=-1), dict(total_k=-1), dict(h_q=0), dict(h_q=3), dict(h_kv=0), dict(scale=-0.5),
               dict(scale=math.nan), dict(scale=math.inf)):
        assert call(prob(**kw)) == 2, kw
    for kw in (dict(dtype=0), dict(dtype=2), dict(d=96), dict(h_q=258, h_kv=2), dict(total_q=2 ** 30), dict(total_k=2 ** 23),
               dict(total_k=2 ** 31 - 1, h_q=1, h_kv=1)):
        assert call(prob(**kw)) == 3, kw
    assert call(Q=ODD) == 2 and call(V=ODD) == 2 and call(O=ODD) == 2 and call(lse=ctypes.c_void_p(4098)) == 2
    p = prob()
    p.o = b.pbs_strides(64, 64)
    assert call(p) == 2
    p = prob()
    p.k = b.pbs_strides(130, 64)
    assert call(p) == 2


def test_a_pipeline_refuses_a_cache_without_slots():
    p = b.problem(batch=1, h_q=2, h_kv=1, n=256, d=128, block=128, segment=256, dtype="bf16", tau=0.9)
    pipe = b.Pipeline(p, device="cpu")
    x = torch.zeros(1, 2, 256, 128, dtype=torch.bfloat16)
    for slots in (None, torch.zeros(256, dtype=torch.int32), torch.zeros(1, 255, dtype=torch.int32)):
        with pytest.raises(b.PbsError, match="slots"):
            pipe.run(x, x[:, :1], x[:, :1], cache=object(), slots=slots)
