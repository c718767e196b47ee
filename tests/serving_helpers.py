"""Plain 64-bit forms of the operators around the prefill path, on the CPU, with elementwise error bounds.

A rounding to a type is off by at most half a step, finfo(t).eps / 2 relative to the value: bf16 2^-8, fp32 2^-24."""
import math

import torch

H16, H32 = 2.0 ** -8, 2.0 ** -24
MOST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8, "f32": torch.float32}


def rope_ref(x, positions, freq, layout, magnitude=1.0, transpose=False):
    """Turned rows in 64 bits, and how far fp32 arithmetic may be off before the last rounding."""
    x = x.double()
    rot = 2 * freq.numel()
    ang = positions.double()[:, None, None] * freq
    cos, sin = ang.cos() * magnitude, ang.sin() * (-magnitude if transpose else magnitude)
    y, e = x.clone(), torch.zeros_like(x)
    i = torch.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + rot // 2)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    # a turn's rest is rounded to fp32: at most 2^-25 of a turn, 2^-22.3 in the angle; cos and sin two steps, products, sum
    e[..., first] = e[..., second] = (a.abs() + b.abs()) * abs(magnitude) * 2.0 ** -21
    return y, e


def hold_ref(x, dtype):
    """What a cache of `dtype` holds for the rows of x, and the rows' factors."""
    x = x.float()
    if dtype == torch.bfloat16:
        return x.to(dtype), None
    most = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    f = (most / MOST[dtype]).clamp(min=2.0 ** -126)
    y = torch.where(fine[..., None], x / f[..., None], torch.zeros(()))
    q = y.to(dtype) if dtype == torch.float8_e4m3fn else y.round().to(dtype)
    return q, torch.where(fine, f, torch.tensor(math.nan))


def stands_for(q, f):
    return q.float() if f is None else q.float() * f[..., None]


def attention_ref(q, k, v, sees, scale):
    """One head in 64 bits: q [m, d], k, v [n, d], sees [m, n] -> O, lse, and elementwise bounds of a computation whose
    logits and sums are fp32 and whose probabilities enter the second product in bf16.  Rows that see nothing: 0, -inf."""
    q, k, v = q.double(), k.double(), v.double()
    m, n = q.shape[0], k.shape[0]
    o, lse = torch.zeros(m, v.shape[1], dtype=torch.float64), torch.full((m,), -math.inf, dtype=torch.float64)
    bo, bl = torch.zeros_like(o), torch.zeros(m, dtype=torch.float64)
    for i in range(m):
        at = sees[i].nonzero()[:, 0]
        if at.numel() == 0:
            continue
        s = (k[at] @ q[i]) * scale
        # d products and sums in fp32, the factors scale and log2(e), a cached row's factor
        ds = (q.shape[1] + 8) * H32 * float((k[at].abs() @ q[i].abs()).max()) * scale + 8 * H32 * float(s.abs().max())
        w = torch.softmax(s, 0)
        o[i] = w @ v[at]
        lse[i] = torch.logsumexp(s, 0)
        sums = (at.numel() + 64) * H32
        # a probability: its rounding to bf16 (a factor of the value row may sit in it), its logit, exp2; then the output's
        bo[i] = (w @ v[at].abs()) * (H16 + 2 * ds + 2 * sums + 2.0 ** -20) + o[i].abs() * H16
        bl[i] = ds + sums + 4 * H32 * lse[i].abs() + 4 * H32
    return o, lse, bo * 1.01 + 1e-30, bl * 1.01


def within(got, want, bound, what=""):
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    bad = ~(same | (off <= bound))
    assert not bad.any(), "%s: %d of %d off, first at %s: %r instead of %r, bound %.3g" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]), float(bound.expand_as(want)[bad][0]))
