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
