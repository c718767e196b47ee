"""Calls of the operators around the prefill path that are refused although each argument is right by itself (no GPU needed)."""
import ctypes

import pytest

from paper_2510_21270_amd import binding as b
from test_serving_cpu import _cache, _decode, lib          # noqa: F401 (the fixture)


def _at(x):
    return ctypes.c_void_p(x)


def _decode_call(lib, p, c, Q, O):
    return lib.pbs_decode_attn(ctypes.byref(p), ctypes.byref(c), _at(Q), _at(4096), _at(4096), _at(4096), _at(O), None, _at(1 << 20), 1 << 40, None)


@pytest.mark.parametrize("prefix", [0, 50, 5000])
def test_new_tokens_in_place_want_the_same_strides(lib, prefix):
    # O at Q's address with other strides: rows would be stored over queries that are still to be read
    c = _cache()
    p = _decode(q_len=2, prefix_len=prefix)
    p.o = b.pbs_strides(64, 6 * 64)
    assert _decode_call(lib, p, c, 8192, 8192) == 2
    p.o = b.pbs_strides(8 * 64, 64)
    assert _decode_call(lib, p, c, 8192, 8192) == 2
    p.o = b.pbs_strides(4 * 64, 128)
    assert _decode_call(lib, p, c, 8192, 8192) == 2


def test_packed_prompts_are_not_attended_to_in_place(lib):
    p = b.pbs_prompt_problem(n_seq=2, total_q=10, total_k=10, h_q=2, h_kv=2, d=64, dtype=1, scale=0.0, flags=1)
    p.q = p.k = p.v = p.o = b.pbs_strides(128, 64)

    def call(Q, K, V, O):
        return lib.pbs_prompt_attn(ctypes.byref(p), _at(Q), _at(K), _at(V), _at(4096), _at(4096), _at(O), None, None)

    for O in (1 << 16, 1 << 17, 1 << 18):
        assert call(1 << 16, 1 << 17, 1 << 18, O) == 2


def test_the_prefix_limits_rows_only_where_there_is_one(lib):
    # 60000 sequences of 16 new tokens: more rows than the grid of a prefix holds, which is not launched without one
    c = _cache(h_kv=2)
    p = _decode(n_seq=60000, q_len=16, h_q=32, max_pages=5, max_len=80)
    p.q = p.o = b.pbs_strides(32 * 64, 64)
    need = lib.pbs_decode_workspace_bytes(ctypes.byref(p), ctypes.byref(c))
    assert need == 0                                       # a wave to a unit
    assert _decode_call(lib, p, c, 4096, 4096 + 8) == 2    # the next check
    p.max_pages = p.max_len = 1000
    assert lib.pbs_decode_workspace_bytes(ctypes.byref(p), ctypes.byref(c)) > 0
    p.prefix_len = 100
    assert lib.pbs_decode_workspace_bytes(ctypes.byref(p), ctypes.byref(c)) == 0 and _decode_call(lib, p, c, 4096, 4096) == 3


# A dispatch holds fewer than 2^32 threads along x; larger calls are refused before anything is enqueued.
def test_rotation_of_more_tokens_than_a_grid_holds(lib):
    p = b.pbs_rope_problem(tokens=2 ** 24, h_q=32, h_kv=8, d=128, rot=128, layout=0, dtype=1, magnitude=1.0, flags=0)
    p.q = p.q_out = b.pbs_strides(32 * 128, 128)
    p.k = p.k_out = b.pbs_strides(8 * 128, 128)
    assert lib.pbs_rope(ctypes.byref(p), _at(4096), _at(4096), _at(4096), _at(4096), _at(1 << 20), _at(1 << 21), None) == 3


@pytest.mark.parametrize("d,tokens", [(128, 2 ** 25), (64, 2 ** 26)])
def test_more_cache_rows_than_a_grid_holds(lib, d, tokens):
    c, s = _cache(d=d, h_kv=8), b.pbs_strides(8 * d, d)
    assert lib.pbs_cache_write(ctypes.byref(c), 1, tokens, _at(4096), ctypes.byref(s), _at(4096), ctypes.byref(s), _at(4096), None) == 3
    assert lib.pbs_cache_read(ctypes.byref(c), 1, tokens, _at(4096), _at(4096), ctypes.byref(s), _at(4096), ctypes.byref(s), None) == 3


@pytest.mark.parametrize("n_seq,q_len,h_q,h_kv,prefix,max_len", [(65535, 16, 32, 4, 100, 0),           # the join of a prefix's parts
                                                                 (65535, 16, 2048, 2048, 0, 16),       # own keys, a wave to a unit
                                                                 (65535, 16, 66, 2, 0, 8000)])         # the join of their pieces
def test_more_rows_of_new_tokens_than_a_grid_holds(lib, n_seq, q_len, h_q, h_kv, prefix, max_len):
    c = _cache(h_kv=h_kv)
    p = _decode(n_seq=n_seq, q_len=q_len, h_q=h_q, max_pages=500, max_len=max_len, prefix_len=prefix)
    p.q = p.o = b.pbs_strides(h_q * 64, 64)
    assert _decode_call(lib, p, c, 4096, 1 << 20) == 3
    assert lib.pbs_decode_workspace_bytes(ctypes.byref(p), ctypes.byref(c)) == 0


def test_more_prompt_tiles_than_a_grid_holds(lib):
    p = b.pbs_prompt_problem(n_seq=1, total_q=2 ** 26, total_k=64, h_q=16, h_kv=16, d=64, dtype=1, scale=0.0, flags=1)
    p.q = p.k = p.v = p.o = b.pbs_strides(16 * 64, 64)
    grid = p.total_q // 128 * 16
    assert grid * 128 < 2 ** 32                            # 2^30 rows: the largest number of tiles stays below
    p = b.pbs_prompt_problem(n_seq=2 ** 22, total_q=2 ** 22, total_k=64, h_q=16, h_kv=16, d=64, dtype=1, scale=0.0, flags=1)
    p.q = p.k = p.v = p.o = b.pbs_strides(16 * 64, 64)
    assert lib.pbs_prompt_attn(ctypes.byref(p), _at(4096), _at(8192), _at(8192), _at(4096), _at(4096), _at(1 << 20), None, None) == 3


def test_a_workspace_that_is_a_strided_view_is_refused(monkeypatch):
    # the kernels write consecutive bytes: every second byte of a buffer would take them over the others
    import torch
    c = b.Cache.__new__(b.Cache)
    c.dev, c.d, c.page, c.c = 0, 64, 16, b._CACHE(8, 16, 2, 64, 1, 4096, 4096, 0, 0)
    monkeypatch.setattr(b, "_same_device", lambda *a: None)
    monkeypatch.setattr(b, "_launch", lambda *a: None)
    Q, table, lens = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 30, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    buf = torch.zeros(1 << 22, dtype=torch.uint8)
    b.decode_attn(c, Q, table, lens, ws=buf)
    with pytest.raises(b.PbsError, match="ws has to be contiguous"):
        b.decode_attn(c, Q, table, lens, ws=buf[::2])


def test_numbers_that_the_structures_cannot_hold_are_refused(monkeypatch):
    import torch
    monkeypatch.setattr(b, "_same_device", lambda *a: None)
    monkeypatch.setattr(b, "_launch", lambda *a: None)
    c = b.Cache.__new__(b.Cache)
    c.dev, c.d, c.page, c.c = 0, 64, 16, b._CACHE(8, 16, 2, 64, 1, 4096, 4096, 0, 0)
    Q, table, lens = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 30, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pages = torch.zeros(30, dtype=torch.int32)
    for kw in (dict(max_len=1 << 31), dict(max_len=1 << 70), dict(prefix_len=-(1 << 40))):
        with pytest.raises(b.PbsError, match="pbs_decode_attn"):
            b.decode_attn(c, Q, table, lens, prefix_pages=pages, **kw)
