// pbs_prompt_attn_rule: attention over packed prompts under a score rule.
//
// Transposed as in the other matrix-core kernels (S^T = K Q^T, O^T += V^T P^T, v_mfma_f32_32x32x16_bf16): a lane owns one query, half of a
// tile's keys.  A wave has 32 rows (row: token, head of the group) against tiles of 64 keys.  A rule's arithmetic (a polynomial and a bias
// for every score) has no place beside one wave's matrix instructions: so two waves share a SIMD, and one's scores are shaped under
// the other's products.  A workgroup is eight waves, the only one of a compute unit, and has two tiles at a time, eight of the
// stages of key_pipeline.h in a ring of two: all of them meet once for 128 keys.  With many rows the waves have 256 of them; with few
// they have 128, four waves one of the two tiles and four the other, and the halves are joined at the end.
//
// Keys that some row sees are a front (the prefix, or the sinks) and a band that ends at the newest row; the tiles between are not
// brought.  A tile that every row of a wave sees whole is not masked.
//
// The softmax keeps a reference m per query and moves it, rescaling O^T and l, when a tile's largest score is more than 2^16 above it;
// tiles come newest first, where a bias leaves the largest scores.  Under a cap alone no reference is needed: scores are within
// 2^+-80, and 32 bits hold their sums.  Values that are not finite (a hidden key's weight is zero, but 0 * inf is NaN) and sums that
// came too near to the ends of the range show when the rows are stored; such a workgroup goes over its keys again, with a
// reference and what is not finite counted apart.  With heads of 128 that pass holds up to 18 values of a lane in scratch memory; the loop
// itself has all of its own in registers.
//
// Probabilities enter the second product as one term in bf16 (off by 2^-8 of each at most), while l sums them as they are.  A second term, what
// the rounding leaves, takes O from 1.9 .. 2.4e-3 off the 64-bit form (rows' norms) to 1.6e-3, which is O's own rounding, but half as many
// matrix instructions again have no slots: 16384 tokens under a cap 2420 -> 3190 us, 16 prompts of 33 .. 2048 under a window 89 -> 109,
// 6 with a bias and prefixes 39 -> 47, 4 of 1 .. 200 11.1 -> 11.9.
//
// Issue slots bound the long prompts, starts and ends of workgroups the short ones.  Measured, us, 32 / 8 heads of 128: 16384 tokens under a cap
// of 50 2400 to 2580, by the card's clock (0.92 to 0.85 PFLOP/s; no cap 2060, a cap of 20, whose logits leave the short polynomial, 2850); 16 prompts of 33 ..
// 2048 under a window 89; 6 of 101 .. 3001, 8 heads of 64, a bias and prefixes 39.
#include "prompt.h"
#include "score_rule.h"

namespace pbs {
namespace prompt {

constexpr int kRuleThreads = 512;
constexpr int kTile = 2 * KS;                              // keys of a wave's tile
constexpr int kWide = 448;                                 // workgroups of 256 rows, see launch_rule
constexpr float kSlack = 16.0f;
constexpr float kLeastSum = 6.310887e-30f;                 // 2^-97
constexpr float kMostCapAlone = 80.0f;                     // in log2 units: 131072 keys at the cap stay below 2^97

struct RuleArgs : Args {                                   // c2: 1 / cap times the scale under a cap
    float cap2;                                            // cap * log2(e), 0: none
    // cap2 tanh(c2 s) as s (t[0] + t[1] s^2 + t[2] s^4 + t[3] s^6) of the products s, up to |s| = small; up to |s| = medium as a longer
    // polynomial of c2 s
    float t[4], small, medium;
    int window, sinks;
    const float *slope;
    const int32_t *prefix;
};

template <int D>
struct Rows32 {                                            // 32 rows of a wave: what State is for 64
    floatx16 o[D / 32][1];
    float m, l;
};

// What a workgroup's rows see, in positions; front: keys that all of them see but for the order among the sinks.
struct Sight {
    int len, prefix, window, sinks;
    bool causal;
    // A query at position pos sees keys 0 .. front - 1 and first .. stop - 1.
    __device__ __forceinline__ void row(int pos, int &front, int &first, int &stop) const
    {
        int64_t a = 0, b = causal ? (int64_t)pos + 1 : len, f = prefix;
        if (window > 0) {
            a = max((int64_t)pos - window + 1, a);
            b = min(b, (int64_t)pos + window);
            f = max(f, causal ? min((int64_t)sinks, (int64_t)pos + 1) : (int64_t)sinks);
        }
        stop = (int)max(min(b, (int64_t)len), (int64_t)0);
        first = (int)min(a, (int64_t)stop);
        front = (int)max(min(f, (int64_t)len), (int64_t)0);
    }
    // whether rows at positions lo .. hi see all keys key0 .. key0 + kTile - 1
    __device__ __forceinline__ bool whole(int lo, int hi, int key0) const
    {
        const int last = key0 + kTile - 1;
        if (last >= len) return false;
        if (last < prefix) return true;
        if (causal && last > lo) return false;
        return window == 0 || last < sinks || (max((int64_t)hi - key0, (int64_t)last - lo) < window);
    }
    // whether none of them sees any
    __device__ __forceinline__ bool none(int lo, int hi, int key0) const
    {
        const int last = key0 + kTile - 1;
        if (key0 < prefix) return false;
        if (causal && key0 > hi) return true;
        return window > 0 && key0 >= sinks && ((int64_t)lo - last >= window || (int64_t)key0 - hi >= window);
    }
    // tiles 0 .. front - 1 and begin .. end - 1 hold all keys that rows at positions lo .. hi see
    __device__ __forceinline__ void tiles(int lo, int hi, int &front, int &begin, int &end) const
    {
        int64_t first = 0, stop = causal ? (int64_t)hi + 1 : len;
        int ahead = prefix;
        if (window > 0) {
            ahead = max(ahead, causal ? min(sinks, max(hi + 1, 0)) : sinks);
            first = max((int64_t)lo - window + 1, (int64_t)0);
            stop = min(stop, (int64_t)hi + window);
        }
        stop = max(min(stop, (int64_t)len), (int64_t)0);
        front = (int)(((int64_t)min(max(ahead, 0), len) + kTile - 1) / kTile);
        end = (int)((stop + kTile - 1) / kTile);
        begin = first < stop ? (int)(first / kTile) : end;
        if (begin <= front) begin = front;
        end = max(end, begin);
    }
};

// the 32 scores of a lane, of keys 32 (x / 16) + 8 (x / 4 % 4) + 4 h + x % 4
__device__ __forceinline__ int key_of(int x) { return 32 * (x >> 4) + 8 * (x >> 2 & 3) + (x & 3); }

// of a lane's query
struct Query { int pos, front, first, stop; float slope2; };

// What becomes of the scores, whose products stand in log2 units afterwards.
enum { kPlain = 0, kCap = 1, kCapAlone = 2 };

template <int D, int CAP, bool SLOPE, bool ODD>
__device__ __forceinline__ void rule_tile(Rows32<D> &st, const Stage<D, false> &sa, const Stage<D, false> &sb, const Offsets<D> &off,
                                          const bf16x8 (&q)[D / 16], const RuleArgs &a, const Query &qu, int key0, bool whole, int h)
{
    floatx16 s[2];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
        const bf16x8 ka = *reinterpret_cast<const bf16x8 *>(sa.k + off.kf[x]), kb = *reinterpret_cast<const bf16x8 *>(sb.k + off.kf[x]);
        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, q[x], x == 0 ? floatx16{0} : s[0], 0, 0, 0);
        s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb, q[x], x == 0 ? floatx16{0} : s[1], 0, 0, 0);
    }
    float y[32];
#pragma unroll
    for (int x = 0; x < 32; ++x) y[x] = s[x >> 4][x & 15];
    constexpr bool kReference = CAP != kCapAlone || ODD;
    // products that go through a multiply-add with the reference below stay what they are
    constexpr bool kLater = CAP == kPlain && !SLOPE;
    if constexpr (CAP != kPlain) {
        float most = 0.0f;
#pragma unroll
        for (int x = 0; x < 32; ++x) most = fmaxf(most, fabsf(y[x]));
        if (__builtin_expect(__any(most > a.medium), 0)) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int x = 0; x < 32; ++x) {
                const float z = y[x] * a.c2;
                float large = tanh_large(z), little = tanh_medium(z);
                asm volatile("" : "+v"(large), "+v"(little));  // both, no branch for every score
                y[x] = a.cap2 * (fabsf(z) > kMediumTanh ? large : little);
            }
        } else if (__any(most > a.small)) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int x = 0; x < 32; ++x) y[x] = a.cap2 * tanh_medium(y[x] * a.c2);
        } else {
#pragma unroll
            for (int x = 0; x < 32; ++x) {
                const float v = y[x] * y[x];
                float p = __builtin_fmaf(v, a.t[3], a.t[2]);
                p = __builtin_fmaf(v, p, a.t[1]);
                p = __builtin_fmaf(v, p, a.t[0]);
                y[x] *= p;
            }
        }
    }
    if constexpr (SLOPE) {
        const float gap = (float)(qu.pos - key0 - 4 * h);
        if (qu.pos >= key0 + kTile) {                      // (of most tiles every query of the wave)
            const float base = -qu.slope2 * gap;
#pragma unroll
            for (int x = 0; x < 32; ++x) {
                const float bias = __builtin_fmaf(qu.slope2, (float)key_of(x), base);
                y[x] = CAP == kPlain ? __builtin_fmaf(y[x], a.c2, bias) : y[x] + bias;
            }
        } else {
#pragma unroll
            for (int x = 0; x < 32; ++x) {
                const float bias = -qu.slope2 * fabsf(gap - (float)key_of(x));
                y[x] = CAP == kPlain ? __builtin_fmaf(y[x], a.c2, bias) : y[x] + bias;
            }
        }
    }
    uint32_t hidden = 0;
    if (!whole) {
        asm volatile("" ::: "memory");                     // keeps this rarer block out of the straight-line code
        const int front = qu.front - key0 - 4 * h, first = qu.first - key0 - 4 * h;
        const uint32_t span = (uint32_t)(qu.stop - qu.first);
#pragma unroll
        for (int x = 0; x < 32; ++x) {
            const bool sees = ((int)(key_of(x) < front) | (int)((uint32_t)(key_of(x) - first) < span)) != 0;   // (no branch)
            if (ODD) hidden |= sees ? 0u : 1u << x;
            y[x] = sees ? y[x] : -INFINITY;
        }
    }
    float ref = 0.0f;
    if constexpr (kReference) {
        float top = y[0];
#pragma unroll
        for (int x = 1; x < 32; ++x) top = fmaxf(top, y[x]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        if constexpr (kLater) top *= a.c2;
        if (__any(top > st.m + kSlack)) {                  // (nothing visible so far: m = -inf)
            const float m = top > st.m + kSlack ? top : st.m;
            const float alpha = m == st.m ? 1.0f : __builtin_amdgcn_exp2f(st.m - m);
            st.m = m;
            st.l *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 16; ++x) st.o[dt][0][x] *= alpha;
        }
        ref = st.m == -INFINITY ? 0.0f : st.m;
    }
    bf16x8 p[4];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
        floatx2 w;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float v = kLater ? __builtin_fmaf(y[x + e], a.c2, -ref) : kReference ? y[x + e] - ref : y[x + e];
            w[e] = __builtin_amdgcn_exp2f(v);
        }
        sum[0] += w[0];
        sum[1] += w[1];
        const bf16x2 t = __builtin_convertvector(w, bf16x2);
        p[x >> 3][x & 7] = t[0];
        p[x >> 3][(x & 7) + 1] = t[1];
    }
    st.l += sum[0] + sum[1];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            const bf16x8 v = read_v<D>(u < 2 ? sa.v : sb.v, off, dt, u & 1);
            if constexpr (!ODD) {
                st.o[dt][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[u], st.o[dt][0], 0, 0, 0);
            } else {
                // the finite values take part, the others count by what a query sees of each kind
                bf16x8 seen;
#pragma unroll
                for (int e = 0; e < 8; ++e) seen[e] = hidden >> (8 * u + e) & 1 ? (bf16_t)0.0f : (bf16_t)1.0f;
                const uintx4 raw = __builtin_bit_cast(uintx4, v);
#pragma unroll 1
                for (int kind = 0; kind < 4; ++kind) {
                    uintx4 w;
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[y] = of_kind(raw[y], kind);
                    const bf16x8 part = __builtin_bit_cast(bf16x8, w);
                    if (kind == 0) {
                        st.o[dt][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part, p[u], st.o[dt][0], 0, 0, 0);
                    } else {
                        const floatx16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part, seen, floatx16{0}, 0, 0, 0);
                        const float add = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : __uint_as_float(0x7fc00000u);
#pragma unroll
                        for (int x = 0; x < 16; ++x)
                            if (n[x] > 0.0f) st.o[dt][0][x] += add;
                    }
                }
            }
        }
}

template <int D>
__device__ __forceinline__ void clear(Rows32<D> &st)
{
    st.m = -INFINITY;
    st.l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) st.o[dt][0] = floatx16{0};
}

// True where the result does not stand: values that are not finite, or, without a reference, a sum near an end of the range.
template <int D, bool REFERENCE>
__device__ __forceinline__ bool store_rows32(const RuleArgs &a, const Place &pl, const Rows32<D> &st, int kv, int t0, int rows, int row0,
                                             int lane, unsigned char *room, bool sees)
{
    bf16_t *const out = a.O + (int64_t)(pl.q0 + t0) * a.o.token + (int64_t)kv * a.r * a.o.head;
    const float l = st.l + __shfl_xor(st.l, 32, 64), inv = l == 0.0f ? 0.0f : 1.0f / l;
    const float zero = rows_out<D, bf16_t>(st, 0, room, lane, [&](floatx4 v) { return __builtin_convertvector(v * inv, bf16x4); },
                                           [&](int x, int piece, uintx4 v) {
                                               const int y = row0 + x, in = token_of(a, y);
                                               if (y < rows)
                                                   *reinterpret_cast<uintx4 *>(out + row_offset(in, y - in * a.r, a.o) + 8 * piece) = v;
                                           });
    const int row = row0 + (lane & 31);
    if (a.lse && lane < 32 && row < rows) {
        const int in = token_of(a, row), head = kv * a.r + row - in * a.r;
        a.lse[(int64_t)(pl.q0 + t0 + in) * a.h_q + head] = l == 0.0f ? -INFINITY : (st.m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
    return __builtin_fmaf(l, 0.0f, zero) != 0.0f || (!REFERENCE && sees && !(l > kLeastSum && l < 1.0f / kLeastSum));
}

// What a wave has summed up, in LDS and out of it; a lane finds its own.
template <int D>
__device__ __forceinline__ void put_rows(const Rows32<D> &st, float *room, int lane)
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int x = 0; x < 16; x += 4)
            *reinterpret_cast<floatx4 *>(room + ((dt * 4 + x / 4) * 64 + lane) * 4) = floatx4{st.o[dt][0][x], st.o[dt][0][x + 1], st.o[dt][0][x + 2], st.o[dt][0][x + 3]};
    room[D / 2 * 64 + lane] = st.m;
    room[D / 2 * 64 + 64 + lane] = st.l;
}
template <int D>
__device__ __forceinline__ void add_rows(Rows32<D> &st, const float *room, int lane)
{
    const float m2 = room[D / 2 * 64 + lane], l2 = room[D / 2 * 64 + 64 + lane], m = fmaxf(st.m, m2);
    const float a = st.m == m ? 1.0f : __builtin_amdgcn_exp2f(st.m - m), b = m2 == m ? 1.0f : __builtin_amdgcn_exp2f(m2 - m);
    st.m = m;
    st.l = st.l * a + l2 * b;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int x = 0; x < 16; x += 4) {
            const floatx4 v = *reinterpret_cast<const floatx4 *>(room + ((dt * 4 + x / 4) * 64 + lane) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[dt][0][x + e] = st.o[dt][0][x + e] * a + v[e] * b;
        }
}

template <int D> struct Ring { Stage<D, false> s[4]; };    // 128 keys
template <int D> constexpr int kRoom = (D / 2 + 2) * 64 * 4;                   // bytes of what a wave has summed up

template <int D, int CAP, bool SLOPE, bool SPLIT>
__global__ __launch_bounds__(kRuleThreads, 2) void prompt_rule_kernel(RuleArgs a)
{
    __shared__ Ring<D> ring0, ring1;                       // apart, so that a read of one does not wait for loads into the other
    __shared__ int bad_rows;
    static_assert(2 * kRoom<D> <= (int)sizeof(Ring<D>), "halves are joined in the ring");
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = blockIdx.x % a.h_kv;
    const Place pl = find_place(a, blockIdx.x / a.h_kv, lane);
    if (pl.seq < 0) return;
    const int t0 = pl.tile * a.tokens, tokens = min(a.tokens, pl.len_q - t0), rows = tokens * a.r;
    const int ahead = pl.len_k - pl.len_q;                 // keys in front of the first query
    const Sight si = {pl.len_k, a.prefix ? a.prefix[pl.seq] : 0, a.window, a.sinks, a.causal};

    const int row0 = (SPLIT ? wave & 3 : wave) * 32, rc = min(row0 + n, rows - 1), in = token_of(a, rc);
    const bool idle = row0 >= rows;                        // (it still brings keys)
    const int pos = t0 + in + ahead;
    // of the wave's rows and of all
    const int lo = t0 + ahead + token_of(a, min(row0, rows - 1)), hi = t0 + ahead + token_of(a, min(row0 + 31, rows - 1));
    int front, begin, end;
    si.tiles(t0 + ahead, t0 + ahead + tokens - 1, front, begin, end);
    const int tiles = front + end - begin, pairs = (tiles + 1) / 2;
    auto tile = [&](int t) { const int x = tiles - 1 - t; return x < front ? x : x - front + begin; };   // newest first
    Query qu;
    qu.pos = pos;
    si.row(pos, qu.front, qu.first, qu.stop);
    qu.slope2 = SLOPE ? a.slope[kv * a.r + rc - in * a.r] * kLog2e : 0.0f;

    // waves 0 .. 3 bring K, the others V, each of 32 keys
    const pbs_strides &ks = wave < 4 ? a.k : a.v;
    const bf16_t *base = (wave < 4 ? a.K : a.V) + (int64_t)pl.k0 * ks.token + (int64_t)kv * ks.head;
    const int step_bytes = (int)ks.token * 2;
    const int size = pl.len_k > 0 ? (pl.len_k - 1) * step_bytes + D * 2 : 0;
    Rows<D, false> src;
    src.rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(base), 0, size, 0x00020000);
    src.size = size;
    src.tiles = (pl.len_k + KS - 1) / KS;
    src.tile_bytes = KS * step_bytes;
    const Offsets<D> off = offsets<D>(wave >> 2, lane, (uint32_t)step_bytes);
    if (threadIdx.x == 0) bad_rows = 0;
    auto get = [&](Ring<D> &to, int pair) {
        const int t = 2 * pair + (wave >> 1 & 1), from = t < tiles ? 2 * tile(t) + (wave & 1) : src.tiles;
        issue_tile(to.s[wave & 3], src, off, from, wave >> 2);
    };

    bf16x8 q[D / 16];
    auto load_queries = [&]() {
        const bf16_t *from = a.Q + (int64_t)(pl.q0 + t0) * a.q.token + (int64_t)kv * a.r * a.q.head + row_offset(in, rc - in * a.r, a.q) + 8 * h;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) q[x] = *reinterpret_cast<const bf16x8 *>(from + 16 * x);
    };
    Rows32<D> st;
    clear(st);
    auto use = [&](const Ring<D> &from, int pair) {
        // both tiles, or the wave's half
#pragma unroll 1
        for (int x = SPLIT ? wave >> 2 : 0; x < (SPLIT ? (wave >> 2) + 1 : 2); ++x) {
            if (idle || 2 * pair + x >= tiles) continue;
            const int key0 = kTile * tile(2 * pair + x);
            if (si.none(lo, hi, key0)) continue;
            rule_tile<D, CAP, SLOPE, false>(st, from.s[2 * x], from.s[2 * x + 1], off, q, a, qu, key0, si.whole(lo, hi, key0), h);
        }
    };
    if (pairs > 0) {
        get(ring0, 0);
        load_queries();
        for (int t = 0;; t += 2) {
            meet();                                        // pair t is there, of every wave; nobody reads pair t - 1 any more
            if (t + 1 < pairs) get(ring1, t + 1);
            use(ring0, t);
            if (t + 1 >= pairs) break;
            meet();
            if (t + 2 < pairs) get(ring0, t + 2);
            use(ring1, t + 1);
            if (t + 2 >= pairs) break;
        }
    }
    __syncthreads();
    if constexpr (CAP == kCapAlone) st.m = 0.0f;
    auto room_of = [&](int x, int bytes) { return reinterpret_cast<unsigned char *>(x < 2 ? &ring0 : &ring1) + (x & 1) * bytes; };
    if constexpr (SPLIT) {
        if (wave >= 4) put_rows(st, reinterpret_cast<float *>(room_of(wave - 4, kRoom<D>)), lane);
        __syncthreads();
        if (wave < 4) add_rows(st, reinterpret_cast<const float *>(room_of(wave, kRoom<D>)), lane);
        __syncthreads();
    }
    // rows leave through LDS, 32 D elements to a wave
    unsigned char *const room = reinterpret_cast<unsigned char *>(wave < 4 ? &ring0 : &ring1) + (wave & 3) * sizeof(Stage<D, false>);
    const bool stores = !idle && (!SPLIT || wave < 4);
    bool bad = false;
    if (stores) bad = store_rows32<D, CAP != kCapAlone>(a, pl, st, kv, t0, rows, row0, lane, room, qu.front > 0 || qu.stop > qu.first);
    if (__any(bad) && lane == 0) bad_rows = 1;
    __syncthreads();
    if (__builtin_expect(bad_rows != 0, 0)) {
        clear(st);
        load_queries();
        for (int t = 0; t < pairs; ++t) {
            __syncthreads();
            get(ring0, t);
            meet();
#pragma unroll 1
            for (int x = 0; x < 2; ++x) {
                if (!stores || 2 * t + x >= tiles) continue;
                const int key0 = kTile * tile(2 * t + x);
                rule_tile<D, CAP, SLOPE, true>(st, ring0.s[2 * x], ring0.s[2 * x + 1], off, q, a, qu, key0, si.whole(lo, hi, key0), h);
            }
        }
        __syncthreads();
        if (stores) store_rows32<D, true>(a, pl, st, kv, t0, rows, row0, lane, room, true);
    }
}

template <int D, bool SPLIT>
pbs_status launch_rows(const RuleArgs &a, long long grid, hipStream_t s)
{
    auto kernel = a.cap2 == 0.0f ? (a.slope ? prompt_rule_kernel<D, kPlain, true, SPLIT> : prompt_rule_kernel<D, kPlain, false, SPLIT>)
                  : a.slope ? prompt_rule_kernel<D, kCap, true, SPLIT>
                  : a.cap2 <= kMostCapAlone ? prompt_rule_kernel<D, kCapAlone, false, SPLIT> : prompt_rule_kernel<D, kCap, false, SPLIT>;
    return launch(kernel, dim3((unsigned)grid), dim3(kRuleThreads), 0, s, a);
}

template <int D>
pbs_status launch_rule(RuleArgs &a, long long grid, hipStream_t s)
{
    // 256 rows to a workgroup where kWide of them or more are left, 1.75 to a compute unit.  Measured, us, 256 rows / 128 in halves, 32 / 8 heads
    // of 128 under a cap: 2000 tokens (256 workgroups) 74 / 60, 2800 (352) 98 / 96, 3200 (408) 113 / 116, 3600 (456) 130 / 144, 4000 (504)
    // 156 / 171, 8000 (1008) 574 / 613; 6 prompts of 500 (416) 39 / 39, 44 of 60 (680) 20 / 28; a window of 512, prompts of 33 .. 2048, 2
    // (272) 28 / 35, 8 (1104) 93 / 117.  A head to every kv head makes rows tokens, and 256 of them see more that is hidden: four times as
    // many are asked for.  8 heads with a bias, prompts of 2000 .. 6000, heads of 64, 4 (528) 168 / 134, 8 (1056) 283 / 244, 14 (1856)
    // 451 / 419, 24 (3184) 732 / 713, heads of 128, 8 (1056) 388 / 358, 14 (1856) 629 / 633; 150 of 60, heads of 64 (1480) 30 / 35.
    const int tokens = 2 * kRows / a.r;
    const long long wide = ((long long)a.total_q / tokens + a.n_seq) * a.h_kv;
    if (wide < (a.r == 1 ? 4 * kWide : kWide)) return launch_rows<D, true>(a, grid, s);
    a.tokens = tokens;
    return launch_rows<D, false>(a, wide, s);
}

}  // namespace prompt
}  // namespace pbs

extern "C" pbs_status pbs_prompt_attn_rule(const pbs_prompt_problem *p, const pbs_score_rule *rule, const void *Q, const void *K,
                                           const void *V, const int32_t *cu_q, const int32_t *cu_k, const int32_t *prefix, void *O,
                                           float *lse, void *stream)
{
    using namespace pbs;
    if (!p || !rule) return PBS_ERR_NULL;
    prompt::RuleArgs a;
    long long grid;
    pbs_status st = prompt::take(p, Q, K, V, cu_q, cu_k, O, lse, prompt::kRuleThreads, a, grid);
    if (st != PBS_OK) return st;
    const float scale = scale_of(p->scale, p->d);
    st = check_rule(rule, scale);
    if (st != PBS_OK) return st;
    if ((reinterpret_cast<uintptr_t>(prefix) & 3u) != 0) return PBS_ERR_SHAPE;
    if (grid == 0) return PBS_OK;
    a.cap2 = rule->cap * kLog2e;
    if (rule->cap > 0.0f) {
        a.c2 = scale / rule->cap;
        const double c = a.c2;
        bool fits = true;                                  // powers of c2 beyond the range of fp32: the longer one for all
        for (int x = 0; x < 4; ++x) {
            const double t = a.cap2 * kLittleTanh[x] * pow(c, 2 * x + 1);
            a.t[x] = (float)t;
            fits = fits && fabs(t) < 1e37 && fabs(t) > 1e-37;
        }
        a.small = fits ? kSmallTanh / a.c2 : -1.0f;
        a.medium = kMediumTanh / a.c2;
    }
    a.window = rule->window;
    a.sinks = rule->sinks;
    a.slope = rule->slope;
    a.prefix = prefix;
    return p->d == 128 ? prompt::launch_rule<128>(a, grid, static_cast<hipStream_t>(stream))
                       : prompt::launch_rule<64>(a, grid, static_cast<hipStream_t>(stream));
}
