// pbs_rope, pbs_rope_frequencies: rotary positions.
//
// y = magnitude * R(position * f_e) x on every pair of features.  Bytes bound it: 3 operations to a feature that is read and
// written once.  A workgroup takes a few tokens: its threads form the tokens' angles once (fp64 product in turns, the
// whole turns taken off in fp64, which is exact, cos and sin of what is left in fp32) into LDS and then walk over the rows of
// all heads, 16 features to a thread and step, so that a wave moves consecutive memory.  32768 tokens of 32 + 8 heads of 128 in bf16:
// 114 us, 5.9 TB/s read and written; a step of 32 tokens: 3.4 us.
#include "pbs_host.h"
#include "serving.h"

namespace pbs {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 8;                             // most tokens to a workgroup

struct RopeArgs {
    int tokens, h_q, heads, d, rot, per_wg;
    unsigned head_magic;                                   // ceil(2^32 / heads): i / heads for i < 2^16
    float magnitude, sign;
    bool interleaved, in_place_q, in_place_k;
    pbs_strides q, k, qo, ko;
};

// 16 features of a row as the two runs of 8 that a thread moves: for half layout features 8c .. and rot/2 + 8c ..,
// otherwise (interleaved pairs, features behind the rotated ones) 16c .. 16c + 15.
template <typename E>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a, const double *__restrict__ freq,
                                                            const int32_t *__restrict__ positions, const E *Q, const E *K,
                                                            E *Qo, E *Ko)
{
    __shared__ floatx2 turn[kRopeTokens * 64];             // cos, sin of (token, pair)
    const int tid = threadIdx.x;
    const int t0 = blockIdx.x * a.per_wg;
    const int toks = min(a.per_wg, a.tokens - t0);
    const int pairs = a.rot >> 1;
    for (int i = tid; i < toks * pairs; i += kRopeThreads) {
        const int t = i / pairs, e = i - t * pairs;
        const double turns = (double)positions[t0 + t] * (freq[e] * 0.15915494309189535);
        const float part = (float)(turns - rint(turns));   // -0.5 .. 0.5 of a turn
        float s, c;
        sincospif(2.0f * part, &s, &c);
        turn[i] = floatx2{c * a.magnitude, s * a.magnitude * a.sign};
    }
    __syncthreads();

    const int chunks = a.d >> 4, rotated = a.rot >> 4;     // 4 or 8; runs of 16 features
    const int shift = a.d == 128 ? 3 : 2;
    const int items = toks * a.heads << shift;
    for (int i = tid; i < items; i += kRopeThreads) {
        const int c = i & (chunks - 1);
        const int row = i >> shift;
        const int t = a.heads == 1 ? row : (int)__umulhi((unsigned)row, a.head_magic);
        const int h = row - t * a.heads;
        const bool is_q = h < a.h_q;
        const pbs_strides &in = is_q ? a.q : a.k, &out = is_q ? a.qo : a.ko;
        const int hh = is_q ? h : h - a.h_q;
        const E *src = (is_q ? Q : K) + (int64_t)(t0 + t) * in.token + (int64_t)hh * in.head;
        E *dst = (is_q ? Qo : Ko) + (int64_t)(t0 + t) * out.token + (int64_t)hh * out.head;
        if (c >= rotated) {
            if (is_q ? a.in_place_q : a.in_place_k) continue;
            floatx4 v[sizeof(E)];
#pragma unroll
            for (int x = 0; x < (int)sizeof(E); ++x) v[x] = reinterpret_cast<const floatx4 *>(src + 16 * c)[x];
#pragma unroll
            for (int x = 0; x < (int)sizeof(E); ++x) reinterpret_cast<floatx4 *>(dst + 16 * c)[x] = v[x];
            continue;
        }
        const int at0 = a.interleaved ? 16 * c : 8 * c, at1 = a.interleaved ? 16 * c + 8 : pairs + 8 * c;
        float x0[8], x1[8], y0[8], y1[8];
        load8(src + at0, x0);
        load8(src + at1, x1);
        const floatx2 *cs = turn + t * pairs + 8 * c;
        if (a.interleaved) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const floatx2 u = cs[x], v = cs[4 + x];
                y0[2 * x] = x0[2 * x] * u[0] - x0[2 * x + 1] * u[1];
                y0[2 * x + 1] = x0[2 * x] * u[1] + x0[2 * x + 1] * u[0];
                y1[2 * x] = x1[2 * x] * v[0] - x1[2 * x + 1] * v[1];
                y1[2 * x + 1] = x1[2 * x] * v[1] + x1[2 * x + 1] * v[0];
            }
        } else {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const floatx2 u = cs[x];
                y0[x] = x0[x] * u[0] - x1[x] * u[1];
                y1[x] = x0[x] * u[1] + x1[x] * u[0];
            }
        }
        store8(dst + at0, y0);
        store8(dst + at1, y1);
    }
}

}  // namespace pbs

extern "C" pbs_status pbs_rope(const pbs_rope_problem *p, const double *freq, const int32_t *positions, const void *Q,
                               const void *K, void *Qout, void *Kout, void *stream)
{
    using namespace pbs;
    if (!p) return PBS_ERR_NULL;
    if (p->tokens < 0 || p->h_q < 0 || p->h_kv < 0 || (p->h_q == 0 && p->h_kv == 0)) return PBS_ERR_SHAPE;
    if (!(p->magnitude == p->magnitude) || isinf(p->magnitude)) return PBS_ERR_SHAPE;
    if (p->dtype != PBS_F32 && p->dtype != PBS_BF16) return PBS_ERR_UNSUPPORTED;
    if (p->d != 64 && p->d != 128) return PBS_ERR_UNSUPPORTED;
    if (p->layout != PBS_ROPE_HALF && p->layout != PBS_ROPE_INTERLEAVED) return PBS_ERR_UNSUPPORTED;
    if (p->rot < 16 || p->rot > p->d || p->rot % 16 != 0) return PBS_ERR_UNSUPPORTED;
    const long long heads = (long long)p->h_q + p->h_kv;
    if (heads > 8192 || heads * p->tokens > 0x7fffffffLL) return PBS_ERR_UNSUPPORTED;
    if (p->tokens == 0) return PBS_OK;
    if (!freq || !positions || (p->h_q > 0 && (!Q || !Qout)) || (p->h_kv > 0 && (!K || !Kout))) return PBS_ERR_NULL;
    const int es = (int)elem_size(p->dtype);
    if (p->h_q > 0 && (!good_input(Q, p->q, es) || !good_output(Qout, p->q_out, p->tokens, p->h_q, p->d, es)))
        return PBS_ERR_SHAPE;
    if (p->h_kv > 0 && (!good_input(K, p->k, es) || !good_output(Kout, p->k_out, p->tokens, p->h_kv, p->d, es)))
        return PBS_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(freq) & 7u) != 0 || (reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return PBS_ERR_SHAPE;

    RopeArgs a;
    a.tokens = p->tokens; a.h_q = p->h_q; a.heads = (int)heads; a.d = p->d; a.rot = p->rot;
    // As many tokens to a workgroup as its threads have an item each of, while there are workgroups for every compute unit several
    // times over.  Measured in bf16 with 1 / 2 / 4 / 8 tokens: 32768 x (32 + 8) heads of 128, 320 items to a token, 114 / 121 / 126 /
    // 134 us (5.9 TB/s with one); with 1 / 2 / 3 / 8 for 16 + 4 heads of 64, 80 items, 31.3 / 26.1 / 26.3 / 27.0 us.
    const long long items = heads * (p->d / 16);
    a.per_wg = 1;
    while (a.per_wg < kRopeTokens && (a.per_wg + 1) * items <= kRopeThreads && p->tokens >= 1024 * (a.per_wg + 1)) ++a.per_wg;
    a.head_magic = (unsigned)((0x100000000ull + heads - 1) / heads);
    a.magnitude = p->magnitude == 0.0f ? 1.0f : p->magnitude;
    a.sign = (p->flags & PBS_ROPE_TRANSPOSE) ? -1.0f : 1.0f;
    a.interleaved = p->layout == PBS_ROPE_INTERLEAVED;
    a.q = p->q; a.k = p->k; a.qo = p->q_out; a.ko = p->k_out;
    a.in_place_q = Q == Qout;
    a.in_place_k = K == Kout;
    if (p->h_q > 0 && a.in_place_q && (p->q.token != p->q_out.token || p->q.head != p->q_out.head)) return PBS_ERR_SHAPE;
    if (p->h_kv > 0 && a.in_place_k && (p->k.token != p->k_out.token || p->k.head != p->k_out.head)) return PBS_ERR_SHAPE;
    const long long groups = ((long long)p->tokens + a.per_wg - 1) / a.per_wg;
    if (!fits_grid(groups, kRopeThreads)) return PBS_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)groups), block(kRopeThreads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (p->dtype == PBS_BF16)
        return launch(rope_kernel<bf16_t>, grid, block, 0, s, a, freq, positions, static_cast<const bf16_t *>(Q),
                      static_cast<const bf16_t *>(K), static_cast<bf16_t *>(Qout), static_cast<bf16_t *>(Kout));
    return launch(rope_kernel<float>, grid, block, 0, s, a, freq, positions, static_cast<const float *>(Q),
                  static_cast<const float *>(K), static_cast<float *>(Qout), static_cast<float *>(Kout));
}

extern "C" pbs_status pbs_rope_frequencies(int scaling, int32_t rot, double base, double factor, double original,
                                           double low, double high, double *freq, double *magnitude)
{
    if (!freq || !magnitude) return PBS_ERR_NULL;
    if (scaling < PBS_ROPE_PLAIN || scaling > PBS_ROPE_RAMP) return PBS_ERR_UNSUPPORTED;
    if (rot < 2 || rot % 2 != 0 || !(base > 1.0) || isinf(base)) return PBS_ERR_SHAPE;
    if (scaling != PBS_ROPE_PLAIN && (!(factor >= 1.0) || isinf(factor))) return PBS_ERR_SHAPE;
    const double turn = 6.283185307179586;
    double a = 0.0, b = 0.0;
    if (scaling == PBS_ROPE_BANDS || scaling == PBS_ROPE_RAMP) {
        if (!(original >= 1.0) || isinf(original) || !(low > 0.0) || !(high > low) || isinf(high)) return PBS_ERR_SHAPE;
        a = fmax(floor(rot * log(original / (turn * high)) / (2.0 * log(base))), 0.0);
        b = fmin(ceil(rot * log(original / (turn * low)) / (2.0 * log(base))), rot - 1.0);
    }
    *magnitude = scaling == PBS_ROPE_RAMP ? 0.1 * log(factor) + 1.0 : 1.0;
    for (int e = 0; e < rot / 2; ++e) {
        const double f = pow(base, -2.0 * e / rot);
        if (scaling == PBS_ROPE_PLAIN) {
            freq[e] = f;
        } else if (scaling == PBS_ROPE_LINEAR) {
            freq[e] = f / factor;
        } else if (scaling == PBS_ROPE_BANDS) {
            const double keep = fmin(fmax((original * f / turn - low) / (high - low), 0.0), 1.0);
            freq[e] = f * (keep + (1.0 - keep) / factor);
        } else {
            const double squeeze = fmin(fmax((e - a) / fmax(b - a, 0.001), 0.0), 1.0);
            freq[e] = f * (1.0 - squeeze + squeeze / factor);
        }
    }
    return PBS_OK;
}
