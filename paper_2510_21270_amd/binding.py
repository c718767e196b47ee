"""Thin ctypes binding of libpbs.so (include/pbs.h).  Argument marshalling only.

PyTorch is used for device memory and streams; every step of the path runs in the library's HIP kernels.
The functions carry the names of the C entry points.  There is no CPU fallback: if the library is missing
or a call fails, an exception is raised.
"""
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpbs.so")
_lib = None

PBS_F32, PBS_BF16, PBS_E4M3, PBS_I8 = 0, 1, 2, 3
STAGE_KEY_SCORES, STAGE_SEGMENT_PERMUTE, STAGE_BLOCK_MASK, STAGE_ATTN_FWD, STAGE_UNPERMUTE = 1, 2, 3, 4, 5
STAGE_QUERY_PERMUTE = 6
FLAG_FORCE_FIRST_BLOCK, FLAG_TOKEN_ORDER_COPY, FLAG_RUNNING_MAX_ONLY, FLAG_KBAR_IN_WS, FLAG_INDEX_REMAP = 1, 2, 4, 8, 16

EXPORTS = ["pbs_status_string", "pbs_validate", "pbs_workspace_bytes", "pbs_vt_bytes", "pbs_key_scores",
           "pbs_segment_permute", "pbs_permute_rows", "pbs_block_mask", "pbs_attn_fwd", "pbs_unpermute",
           "pbs_mfma_rate_probe", "pbs_key_scores_static", "pbs_key_scores_static_scratch_bytes", "pbs_admitted_lists",
           "pbs_mass_covered", "pbs_key_scores_proxy", "pbs_query_permutation", "pbs_shader_clock_meter",
           "pbs_rope", "pbs_rope_frequencies", "pbs_cache_write", "pbs_cache_read", "pbs_decode_workspace_bytes",
           "pbs_decode_attn", "pbs_prompt_attn", "pbs_decode_rule_workspace_bytes", "pbs_decode_attn_rule", "pbs_cache_mark",
           "pbs_evict_workspace_bytes", "pbs_cache_evict", "pbs_prompt_attn_rule"]


class PbsError(RuntimeError):
    pass


class pbs_problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("h_q", ctypes.c_int32), ("h_kv", ctypes.c_int32), ("n", ctypes.c_int32),
                ("d", ctypes.c_int32), ("block", ctypes.c_int32), ("segment", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("tau", ctypes.c_float), ("scale", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


class pbs_strides(ctypes.Structure):
    _fields_ = [("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class pbs_rope_problem(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("h_q", ctypes.c_int32), ("h_kv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("rot", ctypes.c_int32), ("layout", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("magnitude", ctypes.c_float), ("flags", ctypes.c_uint32), ("q", pbs_strides), ("k", pbs_strides),
                ("q_out", pbs_strides), ("k_out", pbs_strides)]


class pbs_cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int32), ("page", ctypes.c_int32), ("h_kv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("K", ctypes.c_void_p), ("V", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class pbs_decode_problem(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("q_len", ctypes.c_int32), ("h_q", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("max_len", ctypes.c_int32), ("prefix_len", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("q", pbs_strides), ("o", pbs_strides)]


class pbs_prompt_problem(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("total_q", ctypes.c_int32), ("total_k", ctypes.c_int32),
                ("h_q", ctypes.c_int32), ("h_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32), ("q", pbs_strides), ("k", pbs_strides),
                ("v", pbs_strides), ("o", pbs_strides)]


class pbs_score_rule(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("slope", ctypes.c_void_p)]


class pbs_cache_marks(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("position", ctypes.c_void_p)]


class pbs_evict_problem(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seq", "max_pages", "max_len", "budget", "sinks", "recent")]


def load_library():
    """Load libpbs.so built in-tree (python -m paper_2510_21270_amd.build).  Fails loudly when it is missing."""
    global _lib
    if _lib is None:
        path = LIB_PATH
        if not os.path.exists(path):
            raise PbsError("libpbs.so not found at %s: build it with `python -m paper_2510_21270_amd.build`" % path)
        lib = ctypes.CDLL(path)
        P, V, Z = ctypes.POINTER(pbs_problem), ctypes.c_void_p, ctypes.c_size_t
        lib.pbs_status_string.restype = ctypes.c_char_p
        lib.pbs_status_string.argtypes = [ctypes.c_int]
        lib.pbs_validate.argtypes = [P]
        lib.pbs_workspace_bytes.restype = Z
        lib.pbs_workspace_bytes.argtypes = [P, ctypes.c_int]
        lib.pbs_vt_bytes.restype = Z
        lib.pbs_vt_bytes.argtypes = [P]
        lib.pbs_key_scores.argtypes = [P, V, V, V, V, Z, V]
        lib.pbs_key_scores_proxy.argtypes = [P, ctypes.c_int, V, ctypes.c_int32, V, V, V, V, Z, V]
        lib.pbs_key_scores_static.argtypes = [P, V, V, V, V]
        lib.pbs_key_scores_static_scratch_bytes.restype = Z
        lib.pbs_key_scores_static_scratch_bytes.argtypes = []
        lib.pbs_segment_permute.argtypes = [P, V, V, V, V, V, V, V, Z, V]
        lib.pbs_permute_rows.argtypes = [P, ctypes.c_int32, V, V, V, V]
        lib.pbs_block_mask.argtypes = [P, V, V, V, V, V, V, Z, V]
        lib.pbs_attn_fwd.argtypes = [P, V, V, V, V, V, V, V, V, V, V, Z, V]
        lib.pbs_unpermute.argtypes = [P, V, V, V, V]
        lib.pbs_query_permutation.argtypes = [P, V, V, V, V, Z, V]
        lib.pbs_admitted_lists.argtypes = [P, V, V, V]
        lib.pbs_mass_covered.argtypes = [P, V, V, V, V]
        lib.pbs_mfma_rate_probe.argtypes = [ctypes.c_int, ctypes.c_int, V, Z, ctypes.POINTER(ctypes.c_double), V]
        lib.pbs_shader_clock_meter.argtypes = [V, ctypes.c_int, V]
        # (structures of the calls below are passed as addresses: ctypes objects by byref, packed bytes as they are)
        D, I = ctypes.c_double, ctypes.c_int32
        lib.pbs_rope.argtypes = [V, V, V, V, V, V, V, V]
        lib.pbs_rope_frequencies.argtypes = [ctypes.c_int, I, D, D, D, D, D, ctypes.POINTER(D), ctypes.POINTER(D)]
        lib.pbs_cache_write.argtypes = [V, I, I, V, V, V, V, V, V]
        lib.pbs_cache_read.argtypes = [V, I, I, V, V, V, V, V, V]
        lib.pbs_decode_workspace_bytes.restype = Z
        lib.pbs_decode_workspace_bytes.argtypes = [V, V]
        lib.pbs_decode_attn.argtypes = [V, V, V, V, V, V, V, V, V, Z, V]
        lib.pbs_prompt_attn.argtypes = [V, V, V, V, V, V, V, V, V]
        lib.pbs_prompt_attn_rule.argtypes = [V, V, V, V, V, V, V, V, V, V, V]
        lib.pbs_decode_rule_workspace_bytes.restype = Z
        lib.pbs_decode_rule_workspace_bytes.argtypes = [V, V, V, V]
        lib.pbs_decode_attn_rule.argtypes = [V, V, V, V, V, V, V, V, V, V, V, Z, V]
        lib.pbs_cache_mark.argtypes = [V, V, I, V, V, V, V, V]
        lib.pbs_evict_workspace_bytes.restype = Z
        lib.pbs_evict_workspace_bytes.argtypes = [V, V]
        lib.pbs_cache_evict.argtypes = [V, V, V, V, V, V, V, Z, V]
        _lib = lib
    return _lib


def problem(batch, h_q, h_kv, n, d, block, segment, dtype, tau=0.9, scale=0.0, flags=0):
    code = {"bf16": PBS_BF16, "f32": PBS_F32, torch.bfloat16: PBS_BF16, torch.float32: PBS_F32}[dtype]
    return pbs_problem(batch, h_q, h_kv, n, d, block, segment, code, tau, scale, flags)


def torch_dtype(p):
    return torch.bfloat16 if p.dtype == PBS_BF16 else torch.float32


def _check(st, what):
    if st != 0:
        raise PbsError("%s: %s (status %d)" % (what, load_library().pbs_status_string(st).decode(), st))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def validate(p):
    return load_library().pbs_validate(ctypes.byref(p))


def workspace_bytes(p, stage):
    return int(load_library().pbs_workspace_bytes(ctypes.byref(p), stage))


def vt_bytes(p):
    return int(load_library().pbs_vt_bytes(ctypes.byref(p)))


def T_of(p):
    return -(-p.n // p.block)


def alloc_workspace(p, stage, device="cuda"):
    nbytes = workspace_bytes(p, stage)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)   # torch allocations are 512-B aligned


def has_token_copy(p):
    return bool(p.flags & FLAG_TOKEN_ORDER_COPY)


def _tok_rows(p):
    """Rows between the start of a permuted tensor and the start of its token-order copy (PBS_FLAG_TOKEN_ORDER_COPY)."""
    return p.batch * p.h_kv * T_of(p) * p.block


def _alloc_with_copy(p, shape, row_elems, dtype, device):
    """A [batch, h_kv, ...] tensor; with PBS_FLAG_TOKEN_ORDER_COPY it is the head of a larger allocation whose tail
    holds the token-order copy (token_copy() returns that view; the storage lives as long as either view does)."""
    numel = 1
    for v in shape:
        numel *= v
    if not has_token_copy(p):
        return torch.empty(shape, dtype=dtype, device=device)
    flat = torch.empty(_tok_rows(p) * row_elems + numel, dtype=dtype, device=device)
    return flat[:numel].view(shape)


def token_copy(p, x, row_elems):
    """The token-order copy that lies behind a K' (row_elems = d), Vt (d) or kidx (1) tensor from the allocators here."""
    off = x.storage_offset() + _tok_rows(p) * row_elems
    return torch.as_strided(x, x.shape, x.stride(), off)


def alloc_vt(p, device="cuda"):
    G = min(p.block, 32)                                   # keys per transposed group
    return _alloc_with_copy(p, (p.batch, p.h_kv, T_of(p), p.block // G, p.d, G), p.d, torch_dtype(p), device)


def alloc_kp(p, device="cuda"):
    return _alloc_with_copy(p, (p.batch, p.h_kv, p.n, p.d), p.d, torch_dtype(p), device)


def alloc_kidx(p, device="cuda"):
    return _alloc_with_copy(p, (p.batch, p.h_kv, p.n), 1, torch.int32, device)


def _ws_args(p, stage, ws):
    if ws is None:
        ws = alloc_workspace(p, stage)
    return ws, _ptr(ws), ws.numel()


def key_scores(p, Q, K, scores=None, ws=None):
    if scores is None:
        scores = torch.empty((p.batch, p.h_kv, p.n), dtype=torch.float32, device=K.device)
    ws, wp, wn = _ws_args(p, STAGE_KEY_SCORES, ws)
    _check(load_library().pbs_key_scores(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(scores), wp, wn, _stream()),
           "pbs_key_scores")
    return scores


PROXY_LAST_BLOCK, PROXY_QUERY_ROWS, PROXY_AVG_QUERY = 0, 1, 2


def key_scores_proxy(p, proxy, qrows, Q, K, scores=None, ws=None):
    if scores is None:
        scores = torch.empty((p.batch, p.h_kv, p.n), dtype=torch.float32, device=K.device)
    ws, wp, wn = _ws_args(p, STAGE_KEY_SCORES, ws)
    m = 0 if qrows is None else qrows.numel()
    _check(load_library().pbs_key_scores_proxy(ctypes.byref(p), proxy, _ptr(qrows), m, _ptr(Q), _ptr(K), _ptr(scores),
                                               wp, wn, _stream()), "pbs_key_scores_proxy")
    return scores


def key_scores_static(p, Q, K, scores=None):
    if scores is None:
        scores = torch.empty((p.batch, p.h_kv, p.n), dtype=torch.float32, device=K.device)
    _check(load_library().pbs_key_scores_static(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(scores), _stream()),
           "pbs_key_scores_static")
    return scores


def segment_permute(p, scores, K, V, kidx=None, Kp=None, Vt=None, indices_only=False, ws=None):
    dev = (K if K is not None else scores).device
    if kidx is None:
        kidx = alloc_kidx(p, dev)
    if not indices_only:
        if Kp is None and not (p.flags & FLAG_INDEX_REMAP):
            Kp = alloc_kp(p, dev)
        if Vt is None:
            Vt = alloc_vt(p, dev)
    _check(load_library().pbs_segment_permute(ctypes.byref(p), _ptr(scores), _ptr(K), _ptr(V), _ptr(kidx), _ptr(Kp),
                                              _ptr(Vt), _ptr(ws), 0 if ws is None else ws.numel(), _stream()),
           "pbs_segment_permute")
    return kidx, Kp, Vt


def permute_rows(p, X, idx, Xp=None):
    if Xp is None:
        Xp = torch.empty_like(X)
    _check(load_library().pbs_permute_rows(ctypes.byref(p), X.shape[1], _ptr(X), _ptr(idx), _ptr(Xp), _stream()),
           "pbs_permute_rows")
    return Xp


def query_permutation(p, Q, Kc, qidx=None, ws=None):
    if qidx is None:
        qidx = torch.empty((p.batch, p.h_q, p.n), dtype=torch.int32, device=Q.device)
    ws, wp, wn = _ws_args(p, STAGE_QUERY_PERMUTE, ws)
    _check(load_library().pbs_query_permutation(ctypes.byref(p), _ptr(Q), _ptr(Kc), _ptr(qidx), wp, wn, _stream()),
           "pbs_query_permutation")
    return qidx


def block_mask(p, Qp, Kp, mask_bits=None, row_cnt=None, col_idx=None, ws=None):
    T = T_of(p)
    dev = Qp.device
    if mask_bits is None:
        mask_bits = torch.empty((p.batch, p.h_q, T, (T + 63) // 64), dtype=torch.int64, device=dev)
    if row_cnt is None:
        row_cnt = torch.empty((p.batch, p.h_q, T), dtype=torch.int32, device=dev)
    if col_idx is None:
        col_idx = torch.empty((p.batch, p.h_q, T, T), dtype=torch.int32, device=dev)
    ws, wp, wn = _ws_args(p, STAGE_BLOCK_MASK, ws)
    _check(load_library().pbs_block_mask(ctypes.byref(p), _ptr(Qp), _ptr(Kp), _ptr(mask_bits), _ptr(row_cnt),
                                         _ptr(col_idx), wp, wn, _stream()), "pbs_block_mask")
    return mask_bits, row_cnt, col_idx


def attn_fwd(p, Qp, Kp, Vt, qidx, kidx, row_cnt, col_idx, Op=None, lse=None, want_lse=False, ws=None):
    if Op is None:
        Op = torch.empty_like(Qp)
    if lse is None and want_lse:
        lse = torch.empty((p.batch, p.h_q, p.n), dtype=torch.float32, device=Qp.device)
    ws, wp, wn = _ws_args(p, STAGE_ATTN_FWD, ws)
    _check(load_library().pbs_attn_fwd(ctypes.byref(p), _ptr(Qp), _ptr(Kp), _ptr(Vt), _ptr(qidx), _ptr(kidx),
                                       _ptr(row_cnt), _ptr(col_idx), _ptr(Op), _ptr(lse), wp, wn, _stream()),
           "pbs_attn_fwd")
    return (Op, lse) if want_lse else Op


def unpermute(p, Op, qidx, O=None):
    if O is None:
        O = Op if qidx is None else torch.empty_like(Op)
    _check(load_library().pbs_unpermute(ctypes.byref(p), _ptr(Op), _ptr(qidx), _ptr(O), _stream()), "pbs_unpermute")
    return O


def admitted_lists(p, row_cnt=None, col_idx=None, device="cuda"):
    T = T_of(p)
    if row_cnt is None:
        row_cnt = torch.empty((p.batch, p.h_q, T), dtype=torch.int32, device=device)
    if col_idx is None:
        col_idx = torch.empty((p.batch, p.h_q, T, T), dtype=torch.int32, device=device)
    _check(load_library().pbs_admitted_lists(ctypes.byref(p), _ptr(row_cnt), _ptr(col_idx), _stream()),
           "pbs_admitted_lists")
    return row_cnt, col_idx


def mass_covered(p, lse_listed, lse_admitted, covered=None):
    if covered is None:
        covered = torch.empty_like(lse_listed)
    _check(load_library().pbs_mass_covered(ctypes.byref(p), _ptr(lse_listed), _ptr(lse_admitted), _ptr(covered),
                                           _stream()), "pbs_mass_covered")
    return covered


def mfma_rate_probe(random_operands, iters=20000, reps=3):
    """(TFLOP/s, shader clock in MHz) of the matrix units alone: best of `reps` launches timed with events on the
    current stream, and the clock one wave of that launch saw."""
    sink = torch.empty(262144, dtype=torch.float32, device="cuda")
    flop = ctypes.c_double(0.0)
    best, mhz = 0.0, 0.0
    for _ in range(reps + 1):                              # the first launch warms up
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        _check(load_library().pbs_mfma_rate_probe(int(bool(random_operands)), iters, _ptr(sink), sink.numel(),
                                                  ctypes.byref(flop), _stream()), "pbs_mfma_rate_probe")
        e1.record()
        e1.synchronize()
        rate = flop.value / (e0.elapsed_time(e1) * 1e-3) / 1e12
        if rate > best:
            best, mhz = rate, float(sink[0])
    return best, mhz


def shader_clock_beside(fn, micros=20000, delay_s=0.02):
    """Shader clock in MHz while fn()'s kernels run on the current stream: fn() is enqueued, then, after delay_s, one
    watching wave on a second stream (default priority) for `micros` microseconds.  fn's work must outlast both."""
    import time
    out = torch.zeros(2, dtype=torch.float32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    fn()
    time.sleep(delay_s)
    with torch.cuda.stream(side):
        _check(load_library().pbs_shader_clock_meter(_ptr(out), int(micros), ctypes.c_void_p(side.cuda_stream)),
               "pbs_shader_clock_meter")
    torch.cuda.synchronize()
    return float(out[0]), float(out[1])


# ---------------------------------------------------------------------------------------------------------------
# Around the prefill path: tensors of [tokens, heads, d] with any token and head strides (a slice of a fused projection, a
# transposed [heads, n, d] tensor).  The checks here are those that the library cannot make: sizes, types and devices of
# tensors.  A step of single tokens is a handful of these calls, so they are kept short: arguments are packed into the
# library's structures in one go (the layouts of pbs_rope_problem, ... above).
_DTYPE_CODES = {torch.float32: PBS_F32, torch.bfloat16: PBS_BF16, torch.float8_e4m3fn: PBS_E4M3, torch.int8: PBS_I8}
_STRIDES = struct.Struct("2q").pack
_ROPE = struct.Struct("7ifI8q").pack
_CACHE = struct.Struct("5i4P").pack
_DECODE = struct.Struct("7if4q").pack
_PROMPT = struct.Struct("7ifI8q").pack
_RULE = struct.Struct("f2iP").pack                         # 4 bytes, 4, 4, padding, address
_MARKS = struct.Struct("2P").pack
_EVICT = struct.Struct("6i").pack
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _refuse(what, why):
    raise PbsError("%s: %s" % (what, why))


def _packed(what, pack, *numbers):
    try:
        return pack(*numbers)
    except (struct.error, OverflowError) as e:
        raise PbsError("%s: a number that its structure cannot hold (%s)" % (what, e)) from None


def _same_device(what, dev, *tensors):
    """All tensors (None: not given) lie on GPU `dev`."""
    if dev < 0:
        _refuse(what, "a tensor is not on the GPU")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            _refuse(what, "tensors on different devices")


def _launch(what, dev, fn, *args):
    """fn(*args, stream) on the current stream of GPU `dev`, whatever device is current."""
    if dev == torch._C._cuda_getDevice():
        st = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _raw_stream(dev))
    if st != 0:
        _check(st, what)


def _rows(what, x):
    """(token, head) strides of a [tokens, heads, d] tensor whose features are consecutive."""
    (n, h, _), (st, sh, sd) = x.shape, x.stride()
    if sd != 1 and x.numel():
        _refuse(what, "the features of a tensor are not consecutive")
    return (st if n > 1 else 0, sh if h > 1 else 0)


def _ints(what, x, name, *shape):
    if x.dtype != torch.int32 or x.shape != shape or not x.is_contiguous():
        _refuse(what, "%s has to be contiguous int32 of shape %s" % (name, list(shape)))


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {None: 0, "plain": 0, "linear": 1, "bands": 2, "ramp": 3}
ROPE_TRANSPOSE = 1


def rope_frequencies(rot, base=1e4, scaling=None, factor=1.0, original=4096, low=None, high=None, device="cuda"):
    """(frequencies [rot / 2] float64 on `device`, magnitude) of rotary pairs, scaled for contexts longer than `original`:
    None, "linear", "bands" (low, high: turns over the original context, 1 and 4) or "ramp" (1 and 32)."""
    if scaling not in ROPE_SCALINGS:
        _refuse("pbs_rope_frequencies", "unknown scaling %r" % (scaling,))
    low = 1.0 if low is None else low
    high = (32.0 if scaling == "ramp" else 4.0) if high is None else high
    table, mag = (ctypes.c_double * max(1, rot // 2))(), ctypes.c_double(0.0)
    _check(load_library().pbs_rope_frequencies(ROPE_SCALINGS[scaling], rot, base, factor, original, low, high, table,
                                               ctypes.byref(mag)), "pbs_rope_frequencies")
    return torch.tensor(list(table), dtype=torch.float64, device=device), mag.value


def rope(Q, K, positions, freq, layout="half", magnitude=1.0, transpose=False, Qout=None, Kout=None):
    """Q and K (either may be None) turned by their positions; new tensors, or in place with Qout=Q, Kout=K."""
    what = "pbs_rope"
    x = Q if Q is not None else K
    if x is None:
        _refuse(what, "neither Q nor K")
    dev, dt = x.get_device(), x.dtype
    if dev < 0:
        _refuse(what, "a tensor is not on the GPU")
    if Q is not None and Qout is None:
        Qout = torch.empty_like(Q)
    if K is not None and Kout is None:
        Kout = torch.empty_like(K)
    _same_device(what, dev, Q, K, Qout, Kout, positions, freq)
    if x.dim() != 3:
        _refuse(what, "Q and K have to be [tokens, heads, d]")
    tokens, _, d = x.shape
    _ints(what, positions, "positions", tokens)
    if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
        _refuse(what, "freq has to be contiguous float64 [rot / 2]")
    if layout not in ROPE_LAYOUTS or magnitude == 0.0:
        _refuse(what, "unknown layout %r or magnitude 0" % (layout,))
    heads, strides, places = [0, 0], (), []
    for k, (t, out) in enumerate(((Q, Qout), (K, Kout))):
        if t is None:
            if out is not None:
                _refuse(what, "an output without its input")
            strides += (0, 0, 0, 0)
            places.append((None, None))
            continue
        if t.dim() != 3 or t.shape[0] != tokens or t.shape[2] != d or out.shape != t.shape or t.dtype != dt or out.dtype != dt:
            _refuse(what, "tensors of different sizes or types")
        heads[k] = t.shape[1]
        strides += _rows(what, t) + _rows(what, out)
        places.append((t.data_ptr(), out.data_ptr()))
    p = _packed(what, _ROPE, tokens, heads[0], heads[1], d, 2 * freq.shape[0], ROPE_LAYOUTS[layout], _DTYPE_CODES.get(dt, -1),
                magnitude, ROPE_TRANSPOSE if transpose else 0, strides[0], strides[1], strides[4], strides[5], strides[2],
                strides[3], strides[6], strides[7])
    _launch(what, dev, (_lib or load_library()).pbs_rope, p, freq.data_ptr(), positions.data_ptr(), places[0][0], places[1][0],
            places[0][1], places[1][1])
    return Qout, Kout


class Cache:
    """A paged key/value cache over K and V [pages, h_kv, page, d] (bf16, float8_e4m3fn or int8, the 8-bit ones with the
    rows' factors k_scale and v_scale [pages, h_kv, page] float32)."""

    def __init__(self, K, V, k_scale=None, v_scale=None):
        what, dt = "pbs_cache", K.dtype
        dev = K.get_device()
        _same_device(what, dev, V, k_scale, v_scale)
        if K.dim() != 4 or K.shape != V.shape or dt != V.dtype or not K.is_contiguous() or not V.is_contiguous():
            _refuse(what, "K and V have to be contiguous [pages, h_kv, page, d] alike")
        code = _DTYPE_CODES.get(dt, PBS_F32)
        if code == PBS_F32:
            _refuse(what, "a cache holds bf16, float8_e4m3fn or int8")
        if code == PBS_BF16:
            k_scale = v_scale = None
        else:
            for f in (k_scale, v_scale):
                if f is None or f.dtype != torch.float32 or f.shape != K.shape[:3] or not f.is_contiguous():
                    _refuse(what, "factors have to be contiguous float32 [pages, h_kv, page]")
        self.K, self.V, self.k_scale, self.v_scale, self.dev = K, V, k_scale, v_scale, dev
        self.pages, self.h_kv, self.page, self.d = K.shape
        # what the library gets; the tensors above keep the memory
        self.c = _CACHE(self.pages, self.page, self.h_kv, self.d, code, K.data_ptr(), V.data_ptr(),
                        k_scale.data_ptr() if k_scale is not None else 0, v_scale.data_ptr() if v_scale is not None else 0)

    @classmethod
    def alloc(cls, pages, page, h_kv, d, dtype=torch.bfloat16, device="cuda"):
        K = torch.zeros((pages, h_kv, page, d), dtype=torch.uint8 if dtype != torch.bfloat16 else dtype, device=device)
        K, V = K.view(dtype), torch.zeros_like(K).view(dtype)
        f = [None if dtype == torch.bfloat16 else torch.zeros((pages, h_kv, page), dtype=torch.float32, device=device)
             for _ in range(2)]
        return cls(K, V, *f)


def cache_write(cache, K, V, slots):
    """Rows K, V [tokens, h_kv, d] into the slots [tokens] of the cache; a slot outside it is passed over."""
    what, dev = "pbs_cache_write", cache.dev
    _same_device(what, dev, K, V, slots)
    if K.dim() != 3 or K.shape != V.shape or K.dtype != V.dtype or K.shape[1] != cache.h_kv or K.shape[2] != cache.d:
        _refuse(what, "K and V have to be [tokens, h_kv, d] alike")
    n = K.shape[0]
    _ints(what, slots, "slots", n)
    _launch(what, dev, (_lib or load_library()).pbs_cache_write, cache.c, _DTYPE_CODES.get(K.dtype, -1), n, K.data_ptr(),
            _STRIDES(*_rows(what, K)), V.data_ptr(), _STRIDES(*_rows(what, V)), slots.data_ptr())


def cache_read(cache, slots, dtype="bf16", K=None, V=None):
    """(K, V) [tokens, h_kv, d] that the slots stand for; zeros for a slot outside the cache.  Into K and V where given."""
    what, dev = "pbs_cache_read", cache.dev
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32 if dtype == "f32" else dtype
    n = slots.numel()
    _ints(what, slots, "slots", n)
    shape = (n, cache.h_kv, cache.d)
    if K is None:
        K = torch.empty(shape, dtype=dt, device=cache.K.device)
    if V is None:
        V = torch.empty(shape, dtype=dt, device=cache.K.device)
    _same_device(what, dev, slots, K, V)
    if K.shape != shape or V.shape != shape or K.dtype != dt or V.dtype != dt:
        _refuse(what, "K and V have to be [tokens, h_kv, d] of the type asked for")
    _launch(what, dev, (_lib or load_library()).pbs_cache_read, cache.c, _DTYPE_CODES.get(dt, -1), n, slots.data_ptr(),
            K.data_ptr(), _STRIDES(*_rows(what, K)), V.data_ptr(), _STRIDES(*_rows(what, V)))
    return K, V


def _token_strides(what, x):
    """(token, head) strides of a [n_seq, q_len, heads, d] tensor whose first two axes are one axis of tokens."""
    (n, q, h, _), (s, t, sh, e) = x.shape, x.stride()
    if e != 1 and x.numel():
        _refuse(what, "the features of a tensor are not consecutive")
    if n > 1 and q > 1 and s != q * t:
        _refuse(what, "the tokens of a tensor are not evenly spaced")
    return (t if q > 1 else s if n > 1 else 0, sh if h > 1 else 0)


def _new_tokens(what, cache, Q, page_table, lens):
    if Q.dim() != 4 or Q.shape[3] != cache.d or page_table.dim() != 2:
        _refuse(what, "Q has to be [n_seq, q_len, h_q, d] and page_table [n_seq, max_pages]")
    n, q_len, h_q, _ = Q.shape
    max_pages = page_table.shape[1]
    _ints(what, page_table, "page_table", n, max_pages)
    _ints(what, lens, "lens", n)
    return n, q_len, h_q, max_pages


def _new_tokens_out(what, Q, O, lse, want_lse):
    if O is None:
        O = torch.empty_like(Q)
    elif O.shape != Q.shape or O.dtype != Q.dtype:
        _refuse(what, "O has to be like Q")
    if lse is None:
        if want_lse:
            lse = torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device)
    elif lse.dtype != torch.float32 or lse.shape != Q.shape[:3] or not lse.is_contiguous():
        _refuse(what, "lse has to be contiguous float32 [n_seq, q_len, h_q]")
    return O, lse


def decode_attn(cache, Q, page_table, lens, max_len=None, prefix_pages=None, prefix_len=0, scale=0.0, O=None, lse=None,
                want_lse=False, ws=None):
    """Attention of Q [n_seq, q_len, h_q, d], the newest tokens of n_seq sequences, over their cached keys: page_table
    [n_seq, max_pages], lens [n_seq] own keys (the new ones among them, at most max_len), behind prefix_len keys of
    prefix_pages that all sequences share.  O like Q; (O, lse [n_seq, q_len, h_q]) with want_lse."""
    what, dev, lib = "pbs_decode_attn", cache.dev, _lib or load_library()
    n, q_len, h_q, max_pages = _new_tokens(what, cache, Q, page_table, lens)
    if prefix_len:
        if prefix_pages is None or prefix_pages.numel() < -(-prefix_len // cache.page):
            _refuse(what, "prefix_pages is shorter than prefix_len")
        _ints(what, prefix_pages, "prefix_pages", prefix_pages.numel())
    else:
        prefix_pages = None
    if max_len is None:
        max_len = max_pages * cache.page
    O, lse = _new_tokens_out(what, Q, O, lse, want_lse)
    p = _packed(what, _DECODE, n, q_len, h_q, max_pages, max_len, prefix_len, _DTYPE_CODES.get(Q.dtype, -1), scale,
                *_token_strides(what, Q), *_token_strides(what, O))
    need = lib.pbs_decode_workspace_bytes(p, cache.c)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=Q.device) if need else None
    elif not ws.is_contiguous():
        _refuse(what, "ws has to be contiguous")
    _same_device(what, dev, Q, O, page_table, lens, prefix_pages, lse, ws)
    _launch(what, dev, lib.pbs_decode_attn, p, cache.c, Q.data_ptr(), page_table.data_ptr(), lens.data_ptr(),
            prefix_pages.data_ptr() if prefix_pages is not None else None, O.data_ptr(),
            lse.data_ptr() if lse is not None else None, ws.data_ptr() if ws is not None else None,
            ws.numel() * ws.element_size() if ws is not None else 0)
    return O if lse is None else (O, lse)


PROMPT_CAUSAL = 1


def _packed_prompts(what, Q, K, V, cu_q, cu_k, causal, scale, O, lse, want_lse):
    dev, dt = Q.get_device(), Q.dtype
    if Q.dim() != 3 or K.dim() != 3 or K.shape != V.shape or K.shape[2] != Q.shape[2] or K.dtype != dt or V.dtype != dt:
        _refuse(what, "Q, K and V have to be [rows, heads, d] of one type, K and V alike")
    total, h_q, d = Q.shape
    total_k, h_kv, _ = K.shape
    if cu_k is None:
        cu_k = cu_q
        if total_k != total:
            _refuse(what, "without cu_k there is a key to every query")
    n = cu_q.numel()
    if n < 1:
        _refuse(what, "cu_q has to be [n_seq + 1]")
    _ints(what, cu_q, "cu_q", n)
    _ints(what, cu_k, "cu_k", n)
    if O is None:
        O = torch.empty_like(Q)
    elif O.shape != Q.shape or O.dtype != dt:
        _refuse(what, "O has to be like Q")
    if lse is None:
        if want_lse:
            lse = torch.empty((total, h_q), dtype=torch.float32, device=Q.device)
    elif lse.dtype != torch.float32 or lse.shape != (total, h_q) or not lse.is_contiguous():
        _refuse(what, "lse has to be contiguous float32 [total_q, h_q]")
    _same_device(what, dev, K, V, cu_q, cu_k, O, lse)
    p = _packed(what, _PROMPT, n - 1, total, total_k, h_q, h_kv, d, _DTYPE_CODES.get(dt, -1), scale, PROMPT_CAUSAL if causal else 0,
                *_rows(what, Q), *_rows(what, K), *_rows(what, V), *_rows(what, O))
    return dev, n - 1, p, cu_k, O, lse


def prompt_attn(Q, K, V, cu_q, cu_k=None, causal=True, scale=0.0, O=None, lse=None, want_lse=False):
    """Attention of packed prompts: Q [total_q, h_q, d] over K, V [total_k, h_kv, d], sequence i being the rows cu_q[i] ..
    cu_q[i + 1] - 1 and cu_k[i] .. cu_k[i + 1] - 1 (cu_q where cu_k is None).  Causal: the last query sees the last key.
    O like Q, its rows of no sequence as they were (new memory is not cleared); (O, lse [total_q, h_q]) with want_lse."""
    what = "pbs_prompt_attn"
    dev, _, p, cu_k, O, lse = _packed_prompts(what, Q, K, V, cu_q, cu_k, causal, scale, O, lse, want_lse)
    _launch(what, dev, (_lib or load_library()).pbs_prompt_attn, p, Q.data_ptr(), K.data_ptr(), V.data_ptr(), cu_q.data_ptr(),
            cu_k.data_ptr(), O.data_ptr(), lse.data_ptr() if lse is not None else None)
    return O if lse is None else (O, lse)


class ScoreRule:
    """What attention does to its logits, and which keys a query sees: a cap (cap * tanh(x / cap)), slope [h_q] float32 times the
    distance taken off, a window (keys at a distance below it, and those at positions below sinks).  0 or None: without."""

    def __init__(self, cap=0.0, slope=None, window=0, sinks=0):
        what = "pbs_score_rule"
        if slope is not None and (slope.dtype != torch.float32 or slope.dim() != 1 or not slope.is_contiguous()):
            _refuse(what, "slope has to be contiguous float32 [h_q]")
        self.cap, self.slope, self.window, self.sinks = cap, slope, window, sinks
        self.c = _packed(what, _RULE, cap, window, sinks, slope.data_ptr() if slope is not None else 0)   # self.slope keeps the memory

    def check(self, what, h_q):
        if self.slope is not None and self.slope.shape[0] != h_q:
            _refuse(what, "slope has to be [h_q]")


def prompt_attn_rule(rule, Q, K, V, cu_q, cu_k=None, prefix=None, causal=True, scale=0.0, O=None, lse=None, want_lse=False):
    """prompt_attn under a ScoreRule; prefix [n_seq] int32: the first keys of each sequence that all of its queries see."""
    what = "pbs_prompt_attn_rule"
    dev, n, p, cu_k, O, lse = _packed_prompts(what, Q, K, V, cu_q, cu_k, causal, scale, O, lse, want_lse)
    rule.check(what, Q.shape[1])
    if prefix is not None:
        _ints(what, prefix, "prefix", n)
    _same_device(what, dev, rule.slope, prefix)
    _launch(what, dev, (_lib or load_library()).pbs_prompt_attn_rule, p, rule.c, Q.data_ptr(), K.data_ptr(), V.data_ptr(), cu_q.data_ptr(),
            cu_k.data_ptr(), prefix.data_ptr() if prefix is not None else None, O.data_ptr(), lse.data_ptr() if lse is not None else None)
    return O if lse is None else (O, lse)


class CacheMarks:
    """Marks of the rows of a cache: weight (the attention that they have received, float32) and position (int32), [pages, h_kv,
    page]; either may be None."""

    def __init__(self, cache, weight=None, position=None):
        for name, x, dt in (("weight", weight, torch.float32), ("position", position, torch.int32)):
            if x is not None and (x.dtype != dt or x.shape != cache.K.shape[:3] or not x.is_contiguous()):
                _refuse("pbs_cache_marks", "%s has to be contiguous %s [pages, h_kv, page]" % (name, dt))
        _same_device("pbs_cache_marks", cache.dev, weight, position)
        self.cache, self.weight, self.position = cache, weight, position
        at = [x.data_ptr() if x is not None else 0 for x in (weight, position)]
        self.c, self.c_position = _MARKS(*at), _MARKS(0, at[1])

    @classmethod
    def alloc(cls, cache):
        return cls(cache, *(torch.zeros(cache.K.shape[:3], dtype=dt, device=cache.K.device) for dt in (torch.float32, torch.int32)))


def cache_mark(marks, slots, positions=None, weight=None):
    """Marks the rows in the slots [tokens] with positions [tokens] and weight [tokens, h_kv] float32 (any strides; None: 0); a
    slot outside the cache is passed over."""
    what, cache = "pbs_cache_mark", marks.cache
    n = slots.numel()
    _ints(what, slots, "slots", n)
    if positions is not None:
        _ints(what, positions, "positions", n)
    elif marks.position is not None:
        _refuse(what, "positions are missing")
    strides = None
    if weight is not None:
        if marks.weight is None or weight.dtype != torch.float32 or weight.shape != (n, cache.h_kv):
            _refuse(what, "weight has to be float32 [tokens, h_kv], for marks with weights")
        strides = _packed(what, _STRIDES, *weight.stride())
    _same_device(what, cache.dev, slots, positions, weight)
    _launch(what, cache.dev, (_lib or load_library()).pbs_cache_mark, cache.c, marks.c, n, slots.data_ptr(),
            positions.data_ptr() if positions is not None else None, weight.data_ptr() if weight is not None else None, strides)


def cache_evict(marks, page_table, lens, budget, sinks=0, recent=0, max_len=None, new_lens=None, ws=None):
    """Leaves every (sequence, kv head) of the marks' cache with at most `budget` keys, in its first places: positions below sinks, the
    `recent` newest positions, the largest weights.  page_table [n_seq, max_pages], lens [n_seq]; returns the new lengths
    (new_lens=lens: in place)."""
    what, cache, lib = "pbs_cache_evict", marks.cache, _lib or load_library()
    if marks.weight is None or marks.position is None:
        _refuse(what, "marks need weights and positions")
    if page_table.dim() != 2:
        _refuse(what, "page_table has to be [n_seq, max_pages]")
    n, max_pages = page_table.shape
    _ints(what, page_table, "page_table", n, max_pages)
    _ints(what, lens, "lens", n)
    if new_lens is None:
        new_lens = torch.empty_like(lens)
    else:
        _ints(what, new_lens, "new_lens", n)
    p = _packed(what, _EVICT, n, max_pages, max_pages * cache.page if max_len is None else max_len, budget, sinks, recent)
    need = lib.pbs_evict_workspace_bytes(p, cache.c)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=lens.device) if need else None
    elif not ws.is_contiguous():
        _refuse(what, "ws has to be contiguous")
    _same_device(what, cache.dev, page_table, lens, new_lens, marks.weight, marks.position, ws)
    _launch(what, cache.dev, lib.pbs_cache_evict, p, cache.c, marks.c, page_table.data_ptr(), lens.data_ptr(), new_lens.data_ptr(),
            ws.data_ptr() if ws is not None else None, ws.numel() * ws.element_size() if ws is not None else 0)
    return new_lens


def decode_attn_rule(rule, cache, Q, page_table, lens, marks=None, positions=None, weigh=False, max_len=None, scale=0.0, O=None,
                     lse=None, want_lse=False, ws=None):
    """decode_attn (without a prefix) under a ScoreRule.  With marks that have positions the keys' are those, the queries'
    positions [n_seq * q_len]; otherwise places in the sequence.  weigh: what every key receives is added to marks.weight."""
    what, dev, lib = "pbs_decode_attn_rule", cache.dev, _lib or load_library()
    n, q_len, h_q, max_pages = _new_tokens(what, cache, Q, page_table, lens)
    rule.check(what, h_q)
    m = None
    if marks is not None:
        if marks.cache.K.shape != cache.K.shape:
            _refuse(what, "marks of another cache")
        if weigh and marks.weight is None:
            _refuse(what, "marks without weights")
        m = marks.c if weigh else marks.c_position
        if marks.position is not None:
            if positions is None:
                _refuse(what, "positions of the queries are missing")
            _ints(what, positions, "positions", n * q_len)
    elif weigh:
        _refuse(what, "weights need marks")
    if marks is None or marks.position is None:
        positions = None
    if max_len is None:
        max_len = max_pages * cache.page
    O, lse = _new_tokens_out(what, Q, O, lse, want_lse)
    p = _packed(what, _DECODE, n, q_len, h_q, max_pages, max_len, 0, _DTYPE_CODES.get(Q.dtype, -1), scale,
                *_token_strides(what, Q), *_token_strides(what, O))
    need = lib.pbs_decode_rule_workspace_bytes(p, rule.c, cache.c, m)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=Q.device) if need else None
    elif not ws.is_contiguous():
        _refuse(what, "ws has to be contiguous")
    _same_device(what, dev, Q, O, page_table, lens, positions, rule.slope, lse, ws)
    if marks is not None:
        _same_device(what, dev, marks.weight, marks.position)
    _launch(what, dev, lib.pbs_decode_attn_rule, p, rule.c, cache.c, m, Q.data_ptr(),
            positions.data_ptr() if positions is not None else None, page_table.data_ptr(), lens.data_ptr(), O.data_ptr(),
            lse.data_ptr() if lse is not None else None, ws.data_ptr() if ws is not None else None,
            ws.numel() * ws.element_size() if ws is not None else 0)
    return O if lse is None else (O, lse)


class Pipeline:
    """Algorithm 1 end to end on preallocated buffers: the five library calls, nothing else."""

    def __init__(self, p, device="cuda", use_sigma=False):
        self.p = p
        self.p_kbar = pbs_problem.from_buffer_copy(p)
        self.p_kbar.flags |= FLAG_KBAR_IN_WS
        T, dt = T_of(p), torch_dtype(p)
        self.scores = torch.empty((p.batch, p.h_kv, p.n), dtype=torch.float32, device=device)
        self.kidx = alloc_kidx(p, device)
        self.Kp = alloc_kp(p, device)
        self.Vt = alloc_vt(p, device)
        self.mask_bits = torch.empty((p.batch, p.h_q, T, (T + 63) // 64), dtype=torch.int64, device=device)
        self.row_cnt = torch.empty((p.batch, p.h_q, T), dtype=torch.int32, device=device)
        self.col_idx = torch.empty((p.batch, p.h_q, T, T), dtype=torch.int32, device=device)
        self.Op = torch.empty((p.batch, p.h_q, p.n, p.d), dtype=dt, device=device)
        self.O = torch.empty_like(self.Op) if use_sigma else self.Op
        self.Qp = torch.empty_like(self.Op) if use_sigma else None
        self.ws1 = alloc_workspace(p, STAGE_KEY_SCORES, device)
        self.ws3 = alloc_workspace(p, STAGE_BLOCK_MASK, device)
        self.ws4 = alloc_workspace(p, STAGE_ATTN_FWD, device)

    def run(self, Q, K, V, qidx=None, cache=None, slots=None, marks=None, positions=None):
        """With a `cache` the keys and values also go into its slots [batch, n], for the decode steps behind the prompt; with `marks`
        of it the rows get their positions [batch, n] and, as their first weights, the scores of Eq. 4, which sum up to 1 for a kv head (a
        decode step adds q_len * h_q / h_kv; cache_mark with self.scores[b].T times a factor gives them another scale)."""
        p = self.p
        # all refusals of the rows and their marks come before the first row is written
        if cache is not None and (slots is None or slots.shape != (p.batch, p.n)):
            _refuse("pbs_cache_write", "a cache needs slots [batch, n]")
        if marks is not None:
            what = "pbs_cache_mark"
            if cache is None or marks.cache is not cache or (positions is not None and positions.shape != slots.shape):
                _refuse(what, "marks need the cache that they belong to, its slots and positions [batch, n]")
            if marks.position is not None and positions is None:
                _refuse(what, "positions are missing")
            for b in range(p.batch if positions is not None else 0):
                _ints(what, positions[b], "positions", p.n)
            _same_device(what, cache.dev, slots, positions)
        if cache is not None:
            for b in range(p.batch):
                cache_write(cache, K[b].transpose(0, 1), V[b].transpose(0, 1), slots[b])
        key_scores(p, Q, K, self.scores, self.ws1)
        if marks is not None:
            for b in range(p.batch):
                cache_mark(marks, slots[b], None if positions is None else positions[b], self.scores[b].T if marks.weight is not None else None)
        # the block means of K' that Algorithm 2 starts from come out of the gather (PBS_FLAG_KBAR_IN_WS)
        segment_permute(p, self.scores, K, V, self.kidx, self.Kp, self.Vt, ws=self.ws3)
        Qp = Q if qidx is None else permute_rows(p, Q, qidx, self.Qp)
        block_mask(self.p_kbar, Qp, self.Kp, self.mask_bits, self.row_cnt, self.col_idx, self.ws3)
        attn_fwd(p, Qp, self.Kp, self.Vt, qidx, self.kidx, self.row_cnt, self.col_idx, self.Op, ws=self.ws4)
        return unpermute(p, self.Op, qidx, self.O)

    def capture(self, Q, K, V, qidx=None, cache=None, slots=None, marks=None, positions=None):
        """Record the pipeline into a HIP graph that reads these very tensors (refill them in place, then replay()).
        The library allocates nothing, never synchronises and records no memset nodes, so the calls can be captured
        as they are; short sequences, where the dozen launches cost more than the kernels, gain from it.  The tensors, the
        cache and the marks live as long as the graph does."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.run(Q, K, V, qidx, cache, slots, marks, positions)            # everything lazily initialised happens outside the capture
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = self.run(Q, K, V, qidx, cache, slots, marks, positions)
        # a graph has addresses only; one that could not be recorded leaves the former one and its tensors
        self.graph, self._graph_out, self._graph_args = graph, out, (Q, K, V, qidx, cache, slots, marks, positions)
        return self._graph_out

    def replay(self):
        self.graph.replay()
        return self._graph_out


class DecodeStep:
    """One step of a batch behind its prompts on preallocated buffers: rotary positions of the new tokens' Q and K (in
    place), their rows into the cache, attention over the cached keys.  The calls of these names, nothing else.
    With a `rule` attention is decode_attn_rule (without a prefix); with `marks` of the cache the new rows are marked with their
    positions and weight 0, the keys' positions count, and what every key receives is added to its weight."""

    marks = rule = None

    def __init__(self, cache, n_seq, h_q, max_pages, freq, q_len=1, max_len=None, layout="half", magnitude=1.0,
                 prefix_pages=None, prefix_len=0, scale=0.0, rule=None, marks=None):
        self.cache, self.freq, self.layout, self.magnitude, self.scale = cache, freq, layout, magnitude, scale
        self.prefix_pages, self.prefix_len = prefix_pages, prefix_len
        self.max_len = max_pages * cache.page if max_len is None else max_len
        self.O = torch.empty((n_seq, q_len, h_q, cache.d), dtype=torch.bfloat16, device=cache.K.device)
        p = _packed("pbs_decode_attn", _DECODE, n_seq, q_len, h_q, max_pages, self.max_len, prefix_len, PBS_BF16, scale,
                    h_q * cache.d, cache.d, h_q * cache.d, cache.d)
        if marks is not None and marks.cache is not cache:
            _refuse("pbs_decode_attn_rule", "marks of another cache")
        self.marks, self.rule = marks, ScoreRule() if rule is None and marks is not None else rule
        if self.rule is not None:
            if prefix_len:
                _refuse("pbs_decode_attn_rule", "a rule or marks go without a shared prefix")
            need = load_library().pbs_decode_rule_workspace_bytes(p, self.rule.c, cache.c, None if marks is None else marks.c)
        else:
            need = load_library().pbs_decode_workspace_bytes(p, cache.c)
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=cache.K.device)

    def run(self, Q, K, V, positions, slots, page_table, lens):
        """Q [n_seq, q_len, h_q, d], K and V [n_seq * q_len, h_kv, d] of the new tokens (Q and K are turned in place),
        positions and slots [n_seq * q_len], page_table [n_seq, max_pages], lens [n_seq] with the new tokens counted."""
        rows = Q.view(-1, Q.shape[2], Q.shape[3])
        rope(rows, K, positions, self.freq, self.layout, self.magnitude, Qout=rows, Kout=K)
        cache_write(self.cache, K, V, slots)
        if self.marks is not None:
            cache_mark(self.marks, slots, positions)
        if self.rule is not None:
            return decode_attn_rule(self.rule, self.cache, Q, page_table, lens, self.marks, positions,
                                    self.marks is not None and self.marks.weight is not None, self.max_len, self.scale, self.O, ws=self.ws)
        return decode_attn(self.cache, Q, page_table, lens, self.max_len, self.prefix_pages, self.prefix_len, self.scale,
                           self.O, ws=self.ws)

    def evict(self, page_table, lens, budget, sinks=0, recent=0):
        """Between two steps: at most `budget` keys of every sequence and kv head stay (cache_evict), lens is made that in place.  The
        bound on lens is the step's max_len; where the lengths are known to be far below it, cache_evict with theirs is faster."""
        if self.marks is None:
            _refuse("pbs_cache_evict", "a step without marks")
        return cache_evict(self.marks, page_table, lens, budget, sinks, recent, self.max_len, new_lens=lens)

    def capture(self, *args):
        """Record a step into a HIP graph that reads these very tensors (refill them in place, then replay()).  The run ahead of the
        recording turns Q and K and writes and marks the new rows, as every run does; the marks' weights it leaves as they are: only
        replays add to them."""
        with torch.cuda.device(self.cache.K.device):
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            marks = self.marks
            with torch.cuda.stream(side):
                try:
                    if marks is not None and marks.weight is not None:         # weights of its own, for the same kernels
                        self.marks = CacheMarks(self.cache, torch.zeros_like(marks.weight), marks.position)
                    self.run(*args)
                finally:
                    self.marks = marks
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                self.run(*args)
        self.graph, self.args = graph, args                # a graph has addresses only
        return self.O

    def replay(self):
        with torch.cuda.device(self.cache.K.device):
            self.graph.replay()
        return self.O
