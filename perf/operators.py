"""Cases on which the operators around the prefill path are measured: rotary positions, the paged key/value cache,
attention of a step's new tokens over that cache, and attention over whole prompts packed one behind the other.

    op "rope"     rotary positions of Q and K                                      -> Q, K
    op "cache"    keys and values quantised into the pages of a cache, read back   -> K, V as the values that are held
    op "decode"   attention of each sequence's newest tokens over its cached keys  -> O
    op "prompt"   causal attention over packed prompts of different lengths        -> O

`run` computes them with elementary torch operations in 32 bits (angles in 64) where `own` is false, and through
the library where it is true.  `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

FAR = -1e30                                                # stands for a masked logit before the maximum is taken


# ------------------------------------------------------------------------------------------------ cases
def _rope(tokens, h_q, h_kv, d, rot, layout, dtype, scaling, base, factor, original, far, transpose=False, name=None):
    c = dict(op="rope", tokens=tokens, h_q=h_q, h_kv=h_kv, d=d, rot=rot, layout=layout, dtype=dtype, scaling=scaling,
             base=base, factor=factor, original=original, far=far, transpose=transpose)
    return dict(c, name=name) if name else c


def _cache(tokens, h_kv, d, dtype, held, page, name=None):
    c = dict(op="cache", tokens=tokens, h_kv=h_kv, d=d, dtype=dtype, held=held, page=page)
    return dict(c, name=name) if name else c


def _decode(n_seq, q_len, h_q, h_kv, d, held, page, shortest, longest, prefix=0, name=None):
    c = dict(op="decode", n_seq=n_seq, q_len=q_len, h_q=h_q, h_kv=h_kv, d=d, held=held, page=page, shortest=shortest,
             longest=longest, prefix=prefix)
    return dict(c, name=name) if name else c


def _prompt(n_seq, h_q, h_kv, d, shortest, longest, before=0, causal=True, name=None):
    c = dict(op="prompt", n_seq=n_seq, h_q=h_q, h_kv=h_kv, d=d, shortest=shortest, longest=longest, before=before,
             causal=causal)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one step of a batch of 32 sequences far into a long context, frequencies scaled by bands: latency
        _rope(32, 32, 8, 128, 128, "half", "bf16", "bands", 5e5, 8.0, 8192, 131072, name="rope_step"),
        # a whole prompt in front of the prefill path: bytes
        _rope(32768, 32, 8, 128, 128, "half", "bf16", "none", 5e5, 1.0, 32768, 32768, name="rope_prompt_32k"),
        # half of each head rotated, neighbouring features paired, float32, an odd length, the gradient's direction
        _rope(4099, 16, 4, 64, 32, "interleaved", "f32", "ramp", 1e6, 4.0, 32768, 131072, transpose=True,
              name="rope_partial_f32"),
        # one step of 64 sequences: 64 rows of 8 heads appended and read back
        _cache(64, 8, 128, "bf16", "i8", 16, name="cache_step_i8"),
        # a prompt written into its pages and read back for a later chunk
        _cache(32768, 8, 128, "bf16", "e4m3", 64, name="cache_prompt_e4m3"),
        # one short sequence: latency
        _decode(1, 1, 32, 8, 128, "bf16", 16, 1000, 1000, name="decode_one_1k"),
        # a serving batch of 64 sequences of very different lengths over an 8-bit cache
        _decode(64, 1, 32, 8, 128, "e4m3", 64, 7, 16000, name="decode_ragged_e4m3"),
        # 48 answers to one long prefix, seven query heads to a kv head
        _decode(48, 1, 28, 4, 128, "bf16", 32, 1, 700, prefix=8147, name="decode_prefix_8k"),
        # a few sequences at the headline length: bytes
        _decode(8, 1, 32, 8, 128, "bf16", 128, 131072, 131072, name="decode_long_128k"),
        # four short prompts, the shortest of a token or two: latency
        _prompt(4, 32, 8, 128, 1, 200, name="prompt_short"),
        # a batch of prompts too short for block selection to pay
        _prompt(16, 32, 8, 128, 33, 2048, name="prompt_packed"),
        # one long prompt, every block
        _prompt(1, 32, 8, 128, 16384, 16384, name="prompt_16k"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rope", "cache", "decode", "decode", "decode", "prompt", "prompt", "prompt"))
    h_q, h_kv, d = rng.choice(((32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 4, 64), (2, 2, 64), (8, 8, 128), (8, 1, 64)))
    if op == "rope":
        scaling = rng.choice(("none", "linear", "bands", "ramp"))
        return _rope(_log_int(rng, 1, 32768), h_q, h_kv, d, rng.choice((d, d, d // 2, d // 4)),
                     rng.choice(("half", "interleaved")), rng.choice(("bf16", "bf16", "f32")), scaling,
                     rng.choice((1e4, 5e5, 1e6)), 1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)),
                     rng.choice((4096, 8192, 32768)), _log_int(rng, 4096, 1000000), rng.random() < 0.25)
    if op == "cache":
        return _cache(_log_int(rng, 1, 32768), h_kv, d, rng.choice(("bf16", "bf16", "f32")),
                      rng.choice(("bf16", "e4m3", "i8")), rng.choice((16, 32, 64, 128, 256)))
    if op == "decode":
        n_seq = _log_int(rng, 1, 64)
        longest = _log_int(rng, 16, min(131072, 524288 // n_seq))
        q_len = rng.choice((1, 1, 1, 2, 4))
        return _decode(n_seq, q_len, h_q, h_kv, d, rng.choice(("bf16", "e4m3", "i8")), rng.choice((16, 32, 64, 128)),
                       rng.randint(q_len, longest), longest, rng.choice((0, 0, _log_int(rng, 100, 16384))))
    n_seq = _log_int(rng, 1, 32)
    longest = _log_int(rng, 8, 9000 if n_seq == 1 else int(8000 / math.sqrt(n_seq)))
    return _prompt(n_seq, h_q, h_kv, d, longest if n_seq == 1 else rng.randint(1, longest), longest,
                   rng.choice((0, 0, _log_int(rng, 1, max(1, longest // 2)))), rng.random() < 0.85)


def _lengths(c):
    """The lengths of a case's sequences: between shortest and longest, even in their logarithm, shuffled by the case alone."""
    n, lo, hi = c["n_seq"], c["shortest"], c["longest"]
    got = [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) for i in range(n)]
    if n == 1:
        got = [hi]
    random.Random(n * 1000003 + hi).shuffle(got)
    return got


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 16 + stream)
    return g


def _normal(seed, stream, shape, dtype=torch.float32):
    return torch.randn(shape, generator=_generator(seed, stream), device="cuda", dtype=dtype)


def _torch_dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _frequencies(c):
    """Radians per position of every rotated pair in 64 bits, and the factor on the rotated features."""
    rot, base, factor, original = c["rot"], c["base"], c["factor"], c["original"]
    e = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    f = base ** (-2.0 * e / rot)
    if c["scaling"] == "linear":                           # positions squeezed by the factor
        return f / factor, 1.0
    if c["scaling"] == "bands":                            # long wavelengths squeezed, short ones kept
        turns = original * f / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / factor), 1.0
    if c["scaling"] == "ramp":                             # the same, by a ramp over the index of the pair
        def index_of(turns):
            return rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))

        lo = max(math.floor(index_of(32.0)), 0)
        hi = min(math.ceil(index_of(1.0)), rot - 1)
        squeeze = ((e - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (1.0 - squeeze + squeeze / factor), 0.1 * math.log(factor) + 1.0
    return f, 1.0


HELD = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
MOST = {"e4m3": 448.0, "i8": 127.0}                        # what the largest value of a row is mapped to
TINY = 2.0 ** -126


def _quantise(x, held):
    """[..., d] float32 -> what the cache holds, and the factor of each row."""
    if held == "bf16":
        return x.to(torch.bfloat16), None
    s = (x.abs().amax(-1) / MOST[held]).clamp(min=TINY)
    y = x / s[..., None]
    return (y.to(torch.float8_e4m3fn) if held == "e4m3" else y.round().to(torch.int8)), s


def _pages(seed, stream, c, pages):
    """Pages full of normal values as the cache holds them: [pages, h_kv, page, d], and the rows' factors."""
    x = _normal(seed, stream, (pages, c["h_kv"], c["page"], c["d"]), torch.bfloat16)
    return _quantise(x if c["held"] == "bf16" else x.float(), c["held"])


def _shuffled(seed, stream, n):
    return torch.randperm(n, generator=_generator(seed, stream), device="cuda", dtype=torch.int64).to(torch.int32)


def prepare(case, seed):
    c = case
    s = dict(c=c)
    if c["op"] == "rope":
        dt = _torch_dtype(c["dtype"])
        s["Q"] = _normal(seed, 1, (c["tokens"], c["h_q"], c["d"])).to(dt)
        s["K"] = _normal(seed, 2, (c["tokens"], c["h_kv"], c["d"])).to(dt)
        if c["tokens"] <= 64:                              # single tokens of many sequences
            s["positions"] = torch.randint(0, c["far"], (c["tokens"],), generator=_generator(seed, 3), device="cuda",
                                           dtype=torch.int32)
        else:                                              # a stretch of one
            s["positions"] = torch.arange(c["tokens"], device="cuda", dtype=torch.int32) + max(0, c["far"] - c["tokens"])
        s["freq"], s["magnitude"] = _frequencies(c)
    elif c["op"] == "cache":
        dt = _torch_dtype(c["dtype"])
        size = torch.exp(0.5 * _normal(seed, 3, (c["tokens"], c["h_kv"], 1)))   # rows differ in size
        s["K"] = (_normal(seed, 1, (c["tokens"], c["h_kv"], c["d"])) * size).to(dt)
        s["V"] = (_normal(seed, 2, (c["tokens"], c["h_kv"], c["d"])) * size).to(dt)
        page = c["page"]
        pages = c["tokens"] // page + 8
        t = torch.arange(c["tokens"], device="cuda", dtype=torch.int32)
        order = _shuffled(seed, 4, pages)
        if c["tokens"] <= 64:                              # a step: each row in a page of its own sequence
            s["slots"] = _shuffled(seed, 5, pages * page)[: c["tokens"]].contiguous()
        else:
            s["slots"] = order[(t // page).long()] * page + t % page
        s["Kc"], s["ks"] = _pages(seed, 6, c, pages)
        s["Vc"], s["vs"] = _pages(seed, 7, c, pages)
    elif c["op"] == "decode":
        lens = _lengths(c)
        page = c["page"]
        need = [-(-n // page) for n in lens]
        own_pages, pre_pages = sum(need), -(-c["prefix"] // page)
        order = _shuffled(seed, 4, own_pages + pre_pages + 3)
        table = torch.full((c["n_seq"], max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, k in enumerate(need):
            table[i, :k] = order[at:at + k]
            at += k
        s["table"], s["lens"], s["max_len"] = table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens)
        s["prefix_pages"] = order[at:at + pre_pages].contiguous() if pre_pages else None
        s["Q"] = (1.5 * _normal(seed, 1, (c["n_seq"], c["q_len"], c["h_q"], c["d"]))).to(torch.bfloat16)
        s["Kc"], s["ks"] = _pages(seed, 6, c, order.numel())
        s["Vc"], s["vs"] = _pages(seed, 7, c, order.numel())
    else:
        lens = _lengths(c)
        keys = [n + c["before"] for n in lens]
        s["max_q"], s["max_k"] = max(lens), max(keys)
        s["cu_q"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        s["cu_k"] = torch.tensor([sum(keys[:i]) for i in range(len(keys) + 1)], dtype=torch.int32, device="cuda")
        s["Q"] = (1.5 * _normal(seed, 1, (sum(lens), c["h_q"], c["d"]))).to(torch.bfloat16)
        s["K"] = _normal(seed, 2, (sum(keys), c["h_kv"], c["d"]), torch.bfloat16)
        s["V"] = _normal(seed, 3, (sum(keys), c["h_kv"], c["d"]), torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, cos, sin, rot, interleaved):
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., : rot // 2], y[..., rot // 2: rot])
    first, second = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((first, second), -1).flatten(-2) if interleaved else torch.cat((first, second), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _plain_rope(s):
    c = s["c"]
    angle = s["positions"].double()[:, None, None] * s["freq"]
    cos = (angle.cos() * s["magnitude"]).float()
    sin = (angle.sin() * (-s["magnitude"] if c["transpose"] else s["magnitude"])).float()
    flat = c["layout"] == "interleaved"
    return {"Q": _rotate(s["Q"], cos, sin, c["rot"], flat), "K": _rotate(s["K"], cos, sin, c["rot"], flat)}


def _put_and_get(x, pages, factors, slots, held):
    page, at = pages.shape[2], slots.long()
    pg, off = at // page, at % page
    q, f = _quantise(x.float(), held)
    raw = pages if held == "bf16" else pages.view(torch.int8)
    raw[pg, :, off] = q if held == "bf16" else q.view(torch.int8)
    got = raw[pg, :, off].view(pages.dtype).float()
    if f is not None:
        factors[pg, :, off] = f
        got = got * factors[pg, :, off][..., None]
    return got.to(x.dtype)


def _plain_cache(s):
    held = s["c"]["held"]
    return {"K": _put_and_get(s["K"], s["Kc"], s["ks"], s["slots"], held),
            "V": _put_and_get(s["V"], s["Vc"], s["vs"], s["slots"], held)}


def _rows_of(pages, factors, table, count):
    """The first `count` rows behind each line of a page table: [lines, h_kv, count, d] float32."""
    at = table.clamp(min=0).long()
    x = pages.view(torch.int8)[at].view(pages.dtype) if pages.dtype == torch.float8_e4m3fn else pages[at]
    x = x.float()
    if factors is not None:
        x = x * factors[at][..., None]
    n, p, h, page, d = x.shape
    return x.transpose(1, 2).reshape(n, h, p * page, d)[:, :, :count].contiguous()


def _softmax_(x):
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    return x.div_(x.sum(-1, keepdim=True))


def _plain_decode(s):
    c = s["c"]
    n, ql, h_q, d = s["Q"].shape
    h_kv, r, L = c["h_kv"], h_q // c["h_kv"], s["max_len"]
    q = s["Q"].float().reshape(n, ql, h_kv, r, d).permute(0, 2, 1, 3, 4).reshape(n, h_kv, ql * r, d) / math.sqrt(d)
    K = _rows_of(s["Kc"], s["ks"], s["table"], L)
    V = _rows_of(s["Vc"], s["vs"], s["table"], L)
    logits = torch.matmul(q, K.transpose(-1, -2).contiguous())
    last = s["lens"][:, None] - ql + torch.arange(ql, device="cuda")        # the newest key that a query sees
    seen = torch.arange(L, device="cuda") <= last[..., None]                # [n, ql, L]
    logits.masked_fill_(~seen[:, None, :, None].expand(n, 1, ql, r, L).reshape(n, 1, ql * r, L), FAR)
    if not c["prefix"]:
        o = torch.matmul(_softmax_(logits), V)
    else:
        P = c["prefix"]
        Kp = _rows_of(s["Kc"], s["ks"], s["prefix_pages"][None], P)[0]      # [h_kv, P, d], once for all sequences
        Vp = _rows_of(s["Vc"], s["vs"], s["prefix_pages"][None], P)[0]
        rows = q.transpose(0, 1).reshape(h_kv, n * ql * r, d)
        pre = torch.matmul(rows, Kp.transpose(-1, -2).contiguous()).reshape(h_kv, n, ql * r, P).transpose(0, 1)
        w = _softmax_(torch.cat((pre, logits), -1))
        o = torch.matmul(w[..., P:].contiguous(), V)
        wp = w[..., :P].transpose(0, 1).reshape(h_kv, n * ql * r, P)
        o += torch.matmul(wp, Vp).reshape(h_kv, n, ql * r, d).transpose(0, 1)
    return {"O": o.reshape(n, h_kv, ql, r, d).permute(0, 2, 1, 3, 4).reshape(n, ql, h_q, d).to(torch.bfloat16)}


def _padded(x, cu, longest):
    """Packed [total, h, d] -> [sequences, h, longest, d] float32; rows past a sequence's end hold others' values."""
    at = (cu[:-1, None].long() + torch.arange(longest, device="cuda")).clamp(max=x.shape[0] - 1)
    return x[at].float().transpose(1, 2).contiguous()


def _plain_prompt(s):
    c = s["c"]
    total, h_q, d = s["Q"].shape
    h_kv, r, mq, mk = c["h_kv"], h_q // c["h_kv"], s["max_q"], s["max_k"]
    n = c["n_seq"]
    q = (_padded(s["Q"], s["cu_q"], mq) / math.sqrt(d)).reshape(n, h_kv, r * mq, d)
    K, V = _padded(s["K"], s["cu_k"], mk), _padded(s["V"], s["cu_k"], mk)
    len_q, len_k = s["cu_q"].diff(), s["cu_k"].diff()
    t, j = torch.arange(mq, device="cuda"), torch.arange(mk, device="cuda")
    last = (len_k - len_q)[:, None] + t if c["causal"] else (len_k - 1)[:, None].expand(n, mq)
    seen = j <= torch.minimum(last, (len_k - 1)[:, None])[..., None]        # [n, mq, mk]
    w = torch.matmul(q, K.transpose(-1, -2).contiguous()).reshape(n, h_kv, r, mq, mk)
    w.masked_fill_(~seen[:, None, None], FAR)
    o = torch.matmul(_softmax_(w).reshape(n, h_kv, r * mq, mk), V).reshape(n, h_q, mq, d)
    row = torch.arange(total, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu_q"][1:].contiguous(), row, right=True)
    return {"O": o[seq, :, row.long() - s["cu_q"][seq].long()].to(torch.bfloat16)}


def run(state):
    s, c = state, state["c"]
    if own:
        from paper_2510_21270_amd import binding as pbs
        if c["op"] == "rope":
            Q, K = pbs.rope(s["Q"], s["K"], s["positions"], s["freq"], layout=c["layout"], magnitude=s["magnitude"],
                            transpose=c["transpose"])
            return {"Q": Q, "K": K}
        cache = pbs.Cache(s["Kc"], s["Vc"], s["ks"], s["vs"]) if "Kc" in s else None
        if c["op"] == "cache":
            pbs.cache_write(cache, s["K"], s["V"], s["slots"])
            K, V = pbs.cache_read(cache, s["slots"], c["dtype"])
            return {"K": K, "V": V}
        if c["op"] == "decode":
            O = pbs.decode_attn(cache, s["Q"], s["table"], s["lens"], max_len=s["max_len"],
                                prefix_pages=s["prefix_pages"], prefix_len=c["prefix"])
            return {"O": O}
        return {"O": pbs.prompt_attn(s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"], causal=c["causal"])}
    return {"rope": _plain_rope, "cache": _plain_cache, "decode": _plain_decode, "prompt": _plain_prompt}[c["op"]](s)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    c = case
    if c["op"] == "rope":
        heads = c["tokens"] * (c["h_q"] + c["h_kv"])
        return {"bytes": 2 * heads * c["d"] * (2 if c["dtype"] == "bf16" else 4) + 4 * c["tokens"],
                "flops": 3 * heads * c["rot"]}
    if c["op"] == "cache":                                 # read, written, read again, written again
        rows = 2 * c["tokens"] * c["h_kv"]
        inside = c["d"] * 2 if c["held"] == "bf16" else c["d"] + 4
        outside = c["d"] * (2 if c["dtype"] == "bf16" else 4)
        return {"bytes": 2 * rows * (inside + outside) + 8 * c["tokens"], "flops": 3 * rows * c["d"]}
    if c["op"] == "decode":
        row = 2 * c["h_kv"] * (c["d"] * 2 if c["held"] == "bf16" else c["d"] + 4)
        lens = _lengths(c)
        queries = c["n_seq"] * c["q_len"] * c["h_q"]
        pairs = c["q_len"] * c["h_q"] * sum(lens) + queries * c["prefix"]
        return {"bytes": row * (sum(lens) + c["prefix"]) + 4 * queries * c["d"], "flops": 4 * c["d"] * pairs}
    lens, b = _lengths(c), c["before"]
    pairs = sum(n * (n + 1) // 2 + n * b if c["causal"] else n * (n + b) for n in lens)
    return {"bytes": 4 * c["d"] * (c["h_q"] * sum(lens) + c["h_kv"] * sum(n + b for n in lens)),
            "flops": 4 * c["d"] * c["h_q"] * pairs}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_rope(c, s):
    turn = torch.polar(torch.full((1,), float(s["magnitude"]), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * s["freq"][None, :])
    if c["transpose"]:
        turn = turn.conj()
    rot, out = c["rot"], {}
    for name in ("Q", "K"):
        x = s[name].double()
        y = x.clone()
        if c["layout"] == "half":
            z = torch.complex(x[..., : rot // 2], x[..., rot // 2: rot]) * turn[:, None]
            y[..., : rot // 2], y[..., rot // 2: rot] = z.real, z.imag
        else:
            z = torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous()) * turn[:, None]
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        out[name] = y
    return out


def _exact_held(x, held):
    """The values that a cache holds for the rows of x."""
    if held == "bf16":
        step = torch.exp2(torch.frexp(x)[1].double() - 8)  # eight significant bits
        return torch.where(x == 0, x, torch.round(x / step) * step)
    f = (x.abs().amax(-1, keepdim=True) / MOST[held]).clamp(min=TINY)
    y = x / f
    if held == "i8":
        return torch.round(y) * f
    step = torch.exp2(torch.frexp(y)[1].clamp(min=-5).double() - 4)            # four significant bits, 2^-9 at least
    return torch.round(y / step) * step * f


def _exact_rows(pages, factors, line, count):
    x = pages.view(torch.int8)[line.long()].view(pages.dtype) if pages.dtype == torch.float8_e4m3fn else pages[line.long()]
    x = x.double()
    if factors is not None:
        x = x * factors[line.long()].double()[..., None]
    return x.transpose(0, 1).flatten(1, 2)[:, :count]


def _exact_decode(c, s):
    lens, P = s["lens"].tolist(), c["prefix"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    r = c["h_q"] // c["h_kv"]
    pre = [_exact_rows(s[k], s[f], s["prefix_pages"], P) for k, f in (("Kc", "ks"), ("Vc", "vs"))] if P else None
    for i, n in enumerate(lens):
        line = s["table"][i, : -(-n // c["page"])]
        K, V = _exact_rows(s["Kc"], s["ks"], line, n), _exact_rows(s["Vc"], s["vs"], line, n)
        if P:
            K, V = torch.cat((pre[0], K), 1), torch.cat((pre[1], V), 1)
        for t in range(c["q_len"]):
            sees = P + n - c["q_len"] + 1 + t
            for h in range(c["h_kv"]):
                q = s["Q"][i, t, h * r:(h + 1) * r].double()
                out[i, t, h * r:(h + 1) * r] = torch.softmax(q @ K[h, :sees].T / math.sqrt(c["d"]), -1) @ V[h, :sees]
    return {"O": out}


def _exact_prompt(c, s):
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    r, cq, ck = c["h_q"] // c["h_kv"], s["cu_q"].tolist(), s["cu_k"].tolist()
    for i in range(c["n_seq"]):
        for h in range(c["h_q"]):
            K, V = s["K"][ck[i]:ck[i + 1], h // r].double(), s["V"][ck[i]:ck[i + 1], h // r].double()
            for lo in range(cq[i], cq[i + 1], 4096):
                hi = min(lo + 4096, cq[i + 1])
                a = s["Q"][lo:hi, h].double() @ K.T / math.sqrt(c["d"])
                if c["causal"]:
                    a.masked_fill_(torch.ones_like(a, dtype=torch.bool).triu(K.shape[0] - (cq[i + 1] - lo) + 1), -math.inf)
                out[lo:hi, h] = torch.softmax(a, -1) @ V
    return {"O": out}


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "rope":
        return _exact_rope(c, s)
    if c["op"] == "cache":
        return {"K": _exact_held(s["K"].double(), c["held"]), "V": _exact_held(s["V"].double(), c["held"])}
    return _exact_decode(c, s) if c["op"] == "decode" else _exact_prompt(c, s)
