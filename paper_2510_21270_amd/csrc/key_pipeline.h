// The pipeline of the attention over dense keys (packed prompts, a prefix shared by a batch): two waves of 64 rows, one wave to a
// SIMD, against tiles of 32 keys that come through LDS.
//
// The softmax of one pass, transposed as in the other matrix-core kernels (S^T = K Q^T, O^T += V^T P^T, v_mfma_f32_32x32x16_bf16):
// a lane owns one query of each 32-row tile, its probabilities are the B operand of the second product as they lie.  K and V
// rows go into LDS as they lie in memory, by asynchronous loads; V^T comes out through the transposing read
// (ds_read_b64_tr_b16: 4 rows x 16 features to 16 lanes).
//
// What bounds it is the matrix pipe and the vector work that has to fit beside it in one wave's instruction stream.  The loop is
// a pipeline in which no matrix instruction of an iteration depends on the vector arithmetic of the same one.  Iteration t:
//     S(t + 1) = K(t + 1) Q^T, then O^T += V^T(t - 1) P^T(t - 1); all along P^T(t) from S(t)
//     LDS: V^T(t - 1) is read under the first matrix instructions; the waves meet; K(t + 4) and V(t + 3) go out into what has
//     been read; K(t + 2) is read under the last ones
// Ring of four stages; stage p holds K tile p and V tile p - 1 (mod 4), which is what iteration p frees.
// The softmax of the loop keeps the reference that the first tile sets (any reference gives the same softmax while nothing
// overflows) and moves it, rescaling O^T and l, when a tile's sum passes 2^40.  What that leaves open (a row whose first
// tile has no finite logit and that ends without a sum; values that are not finite, which a hidden key's zero weight would
// turn into NaN) shows when the rows are stored, and such a workgroup goes over its keys again, tile by tile with the running
// maximum (whole_tile), and stores again.
//
// Probabilities go into the second product rounded to bf16, off by 2^-8 of each at most, while l sums them as they are.  What the
// rounding leaves could go in as a second term, but the matrix units and the instructions beside them are the bound here, and
// registers are taken.  The products of a second term alone, without forming it: 16384 tokens 1.77 -> 2.37 ms, 16 prompts of 33 ..
// 2048 103 -> 127 us, 8000 tokens of 16 / 4 heads of 64 142 -> 176 us, 48 answers to 8147 shared keys 35.0 -> 36.2 us.
//
// F: the keys' and the value rows' factors (of an 8-bit cache whose values lie here as bf16) come along, those of tile t + 3 in
// iteration t into stage t + 3, and are read four keys at a time where they are needed; a key's multiplies its logit, a
// value row's its probability.
#pragma once
#include <utility>

#include "pbs_host.h"
#include "serving.h"

namespace pbs {
namespace prompt {

constexpr int KS = 32;                                     // keys of a tile
constexpr int kRows = 128;                                 // rows of a workgroup: two waves of 64
typedef __attribute__((address_space(3))) void *lptr_t;
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 *tr_ptr_t;

// A tile in LDS.  The 16-byte pieces of a row are stored permuted so that neither read meets itself in a bank:
//   k: piece c of row n at place c ^ (n % 16) (d = 64, 8 pieces to a row: c ^ (n / 2 % 8)): 16 lanes read 16 rows
//   v: piece c of row n at place c ^ 4 (n % 4) (d = 64: c ^ 4 (n / 2 % 2)): 16 lanes read 32 bytes of four rows
template <int D, bool F>
struct __align__(16) Stage {
    unsigned char k[KS * D * 2];
    unsigned char v[KS * D * 2];
    float kf[F ? 2 * KS : 4], vf[F ? 2 * KS : 4];          // (of the tile's rows and the next 32)
};

template <int D> __device__ __forceinline__ int k_place(int row, int c) { return D == 128 ? c ^ (row & 15) : c ^ (row >> 1 & 7); }
template <int D> __device__ __forceinline__ int v_place(int row, int c) { return D == 128 ? c ^ (row & 3) << 2 : c ^ (row >> 1 & 1) << 2; }

template <int D>
struct Offsets {
    static constexpr int kLoads = KS * D * 2 / 1024;       // load instructions of a tile: 1 KiB each
    uint32_t from[kLoads];                                 // byte offset in a tile's rows of the piece this lane moves
    uint32_t kf[D / 16], vf[D / 32];                       // byte offsets in k and v of this lane's fragment reads
};

// wave 0 brings K, wave 1 V; stride: bytes between rows of what this wave brings
template <int D>
__device__ __forceinline__ Offsets<D> offsets(int wave, int lane, uint32_t stride)
{
    constexpr int P = D / 8, RPL = 64 / P;                 // pieces of a row, rows of a load
    Offsets<D> r;
#pragma unroll
    for (int c = 0; c < Offsets<D>::kLoads; ++c) {
        const int row = c * RPL + lane / P, place = lane % P;
        const int piece = wave == 0 ? k_place<D>(row, place) : v_place<D>(row, place);
        r.from[c] = row * stride + piece * 16;
    }
    const int n = lane & 31, h = lane >> 5;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) r.kf[x] = n * (D * 2) + k_place<D>(n, 2 * x + h) * 16;
    // transposing read: lane p of 16 names 4 features of row p / 4; 16 lanes get 16 features, their halves of a wave 4 rows on
    const int p = lane & 15, row = 4 * h + (p >> 2);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
        r.vf[dt] = row * (D * 2) + v_place<D>(row, 4 * dt + 2 * (lane >> 4 & 1) + (p >> 1 & 1)) * 16 + (p & 1) * 8;
    return r;
}

// What a wave brings, wave 0 K and wave 1 V, from consecutive rows (the factors beside them, F).  A tile behind the
// last one starts at the end, where reads give zeros.
template <int D, bool F>
struct Rows {
    __amdgpu_buffer_rsrc_t rows, factors;
    int size, tiles, tile_bytes, factors_size;
    struct At {
        int rows;
        __device__ __forceinline__ void pin() { asm volatile("" : "+s"(rows)); }
    };
    __device__ __forceinline__ At at(int t) const
    {
        if constexpr (F) return {scalar_offset(t * tile_bytes, size)};         // (a part of a prefix: a thousand rows of 256 bytes)
        else return {tile_start(t, tiles, tile_bytes, size)};
    }
    __device__ __forceinline__ void load(unsigned char *dst, int c, const At &w, const Offsets<D> &off) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lptr_t)(dst + c * 1024), 16, off.from[c], w.rows, 0, 0);
    }
    __device__ __forceinline__ void load_factors(float *dst, int t, int lane) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(factors, (lptr_t)dst, 4, lane * 4, scalar_offset(t * KS * 4, factors_size), 0, 0);
    }
};

template <int D, bool F, class SRC>
__device__ __forceinline__ void issue_tile(Stage<D, F> &sg, const SRC &src, const Offsets<D> &off, int t, int wave)
{
    const auto w = src.at(__builtin_amdgcn_readfirstlane(t));
#pragma unroll
    for (int c = 0; c < Offsets<D>::kLoads; ++c) src.load(wave == 0 ? sg.k : sg.v, c, w, off);
}
template <int D, bool F, class SRC>
__device__ __forceinline__ void issue_factors(Stage<D, F> &sg, const SRC &src, int t, int wave, int lane)
{
    if constexpr (F) src.load_factors(wave == 0 ? sg.kf : sg.vf, __builtin_amdgcn_readfirstlane(t), lane);
}

// factors of the 16 keys 8 (x / 4) + 4 h + x % 4 of a tile
__device__ __forceinline__ void read_factors(float (&f)[16], const float *from, int h)
{
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const floatx4 v = *reinterpret_cast<const floatx4 *>(from + 8 * y + 4 * h);
#pragma unroll
        for (int x = 0; x < 4; ++x) f[4 * y + x] = v[x];
    }
}

// V^T fragment (features 32 dt .. + 31, keys 16 u + 8 (e / 4) + 4 h + e % 4): two transposing reads
template <int D>
__device__ __forceinline__ bf16x8 read_v(const unsigned char *v, const Offsets<D> &off, int dt, int u)
{
    const unsigned char *at = v + off.vf[dt] + 16 * u * (D * 2);
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr_t)(at));
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr_t)(at + 8 * (D * 2)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): this wave's loads are in LDS
    __syncthreads();
}

// the same but for this wave's newest N loads
template <int N>
__device__ __forceinline__ void meet_but()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <int D>
struct State {
    floatx16 o[D / 32][2];
    float m[2], l[2];                                      // reference in log2 units; this lane's half of the keys
};

// kind 0: finite values, 1: +inf, 2: -inf, 3: NaN, the latter three as ones
__device__ __forceinline__ uint32_t of_kind(uint32_t pair, int kind)
{
    uint32_t out = 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const uint32_t v = (pair >> (16 * x)) & 0xffffu;
        const bool odd = (v & 0x7f80u) == 0x7f80u, inf = (v & 0x7fffu) == 0x7f80u;
        uint32_t w = 0;
        if (kind == 0) w = odd ? 0u : v;
        else if (kind == 1) w = inf && v < 0x8000u ? 0x3f80u : 0u;
        else if (kind == 2) w = inf && v >= 0x8000u ? 0x3f80u : 0u;
        else w = odd && !inf ? 0x3f80u : 0u;
        out |= w << (16 * x);
    }
    return out;
}

// A tile by itself: scores, mask (keys at or above sees[nt] are hidden), running maximum, sums, second product.  Score x of a
// lane belongs to key 8 (x / 4) + 4 h + x % 4 of the tile.
// `halves`: which halves of the tile's keys exist at all (bits 0 and 1).
template <int D, bool F>
__device__ __forceinline__ void whole_tile(State<D> &st, const Stage<D, F> &sg, const Offsets<D> &off, const bf16x8 (&q)[2][D / 16],
                                           const int (&sees)[2], int key0, int halves, float c2, int h)
{
    float kf[16], vf[16];
    if constexpr (F) {
        read_factors(kf, sg.kf, h);
        read_factors(vf, sg.vf, h);
    }
    floatx16 s[2];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(sg.k + off.kf[x]);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
            s[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[nt][x], x == 0 ? floatx16{0} : s[nt], 0, 0, 0);
    }
    bf16x8 p[2][2];
    bool hides = false;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int lim = sees[nt] - key0 - 4 * h;
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const bool hidden = 8 * (x >> 2) + (x & 3) >= lim || !(halves >> (x >> 3) & 1);
            hides = hides || hidden;
            s[nt][x] = hidden ? -INFINITY : s[nt][x] * (F ? kf[x] * c2 : c2);
            top = fmaxf(top, s[nt][x]);
        }
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m = fmaxf(st.m[nt], top), ref = m == -INFINITY ? 0.0f : m;
        const float alpha = __builtin_amdgcn_exp2f(st.m[nt] - ref);
        st.m[nt] = m;
        float sum = 0.0f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const float w = __builtin_amdgcn_exp2f(s[nt][x] - ref);
            sum += w;
            p[nt][x >> 3][x & 7] = (bf16_t)(F && s[nt][x] != -INFINITY ? w * vf[x] : w);
        }
        st.l[nt] = st.l[nt] * alpha + sum;
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 16; ++x) st.o[dt][nt][x] *= alpha;
        }
    }
    // A hidden key has probability zero, but 0 * inf is NaN: where a tile with hidden keys holds values that are not
    // finite, the product takes the finite ones and the others count by what a query sees of each kind.
    bool odd = false;
    if (__any(hides)) {
#pragma unroll 1
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) {
                const uintx4 v = __builtin_bit_cast(uintx4, read_v<D>(sg.v, off, dt, u));
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    odd = odd || (v[y] & 0x7f80u) == 0x7f80u || (v[y] & 0x7f800000u) == 0x7f800000u;
            }
    }
    if (__any(odd)) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                bf16x8 seen;
                const int lim = sees[nt] - key0 - 4 * h;
#pragma unroll
                for (int e = 0; e < 8; ++e) seen[e] = 16 * u + 8 * (e >> 2) + (e & 3) < lim && (halves >> u & 1) ? (bf16_t)1.0f : (bf16_t)0.0f;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) {
                    const uintx4 v = __builtin_bit_cast(uintx4, read_v<D>(sg.v, off, dt, u));
#pragma unroll 1
                    for (int kind = 0; kind < 4; ++kind) {
                        uintx4 w;
#pragma unroll
                        for (int y = 0; y < 4; ++y) w[y] = of_kind(v[y], kind);
                        const bf16x8 a = __builtin_bit_cast(bf16x8, w);
                        if (kind == 0) {
                            st.o[dt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[nt][u], st.o[dt][nt], 0, 0, 0);
                        } else {
                            const floatx16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, seen, floatx16{0}, 0, 0, 0);
                            const float add = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : __uint_as_float(0x7fc00000u);
#pragma unroll
                            for (int x = 0; x < 16; ++x)
                                if (n[x] > 0.0f) st.o[dt][nt][x] += add;
                        }
                    }
                }
            }
        return;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            const bf16x8 vf = read_v<D>(sg.v, off, dt, u);
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
                st.o[dt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[nt][u], st.o[dt][nt], 0, 0, 0);
        }
}

// ---- the pipeline
// Score matrix instructions are assembly statements, so that the result lies in vector registers (the softmax reads it
// there) and, for d = 128, K and Q in accumulation registers, which nothing else of the loop needs.  The compiler does not see
// inside: scores are read more than a dozen instructions after the last statement, or behind fence(), and no operand may be
// moved into place just ahead of one (a matrix instruction reads two wait states after a vector instruction's write at the
// earliest), which is why d = 64, with registers to spare, has its operands in vector registers.
template <int D>
__device__ __forceinline__ void score_first(floatx16 &s, const bf16x8 &k, const bf16x8 &q)
{
    if (D == 128) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "a"(k), "a"(q));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
}
template <int D>
__device__ __forceinline__ void score_next(floatx16 &s, const bf16x8 &k, const bf16x8 &q)
{
    if (D == 128) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "a"(k), "a"(q));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
__device__ __forceinline__ void fence() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

template <int D>
__device__ __forceinline__ void mask_scores(floatx16 (&s)[2], const int (&sees)[2], int key0, int h)
{
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int lim = sees[nt] - key0 - 4 * h;
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (8 * (x >> 2) + (x & 3) >= lim) s[nt][x] = -INFINITY;
    }
}

// Which of the D / 4 matrix instructions of an iteration brings what (-1: nothing).
template <int D>
struct Slots {
    static constexpr int kAll = D / 4, kScores = D / 8, kFrags = D / 16;      // K and V fragments alike
    static constexpr int kMeet = D == 128 ? 11 : 5;                            // the waves meet after this one
    static constexpr int kFactors = D == 128 ? 29 : 15;                        // the load of the factors
    static constexpr int v_read(int m) { return m < kFrags ? m : -1; }
    static constexpr int load(int m) { return m > kMeet && (m - kMeet) % 2 == 0 && (m - kMeet - 2) / 2 < Offsets<D>::kLoads ? (m - kMeet - 2) / 2 : -1; }
    static constexpr int k_read(int m) { return m >= kScores && m % 2 == 0 && (m - kScores) / 2 < kFrags ? (m - kScores) / 2 : -1; }
    // factors: group g is read when group g - 2, whose place it takes, has been used; group 4 is the next tile's first
    static constexpr int factors_read(int m)
    {
        for (int g = 1; g <= 4; ++g)
            if (m == (D == 128 ? 8 * g - 5 : 4 * g - 2)) return g;
        return -1;
    }
    template <bool F> static constexpr int nt_of(int z) { return F ? z & 1 : z >> 3; }
    template <bool F> static constexpr int pair_of(int z) { return F ? z >> 1 : z & 7; }
    // second products: consecutive ones never share an accumulator
    static constexpr int pv_nt(int n) { return D == 128 ? n >> 3 : n & 1; }
    static constexpr int pv_dt(int n) { return D == 128 ? n & 3 : n >> 1 & 1; }
    static constexpr int pv_u(int n) { return n >> 2 & 1; }
};

template <typename F, int... M>
__device__ __forceinline__ void unrolled(F &f, std::integer_sequence<int, M...>)
{
    (f(std::integral_constant<int, M>{}), ...);
}

constexpr float kBigSum = 1.0995116e12f;                   // 2^40

// A tile outgrew the reference: the reference moves to the tile's maximum, O^T (tiles before this one) and l follow, the tile's
// probabilities are formed again.
template <int D, bool F>
__device__ __forceinline__ void move_reference(State<D> &st, const floatx16 (&s)[2], bf16x8 (&p)[2][2], float (&sum)[2], float c2,
                                               const float (&kf)[16], const float (&vf)[16])
{
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) top = fmaxf(top, F ? s[nt][x] * kf[x] : s[nt][x] * c2);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m = fmaxf(st.m[nt], top), alpha = __builtin_amdgcn_exp2f(st.m[nt] - m);
        st.m[nt] = m;
        st.l[nt] *= alpha;
        sum[nt] = 0.0f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const float w = __builtin_amdgcn_exp2f((F ? s[nt][x] * kf[x] : s[nt][x] * c2) - m);
            sum[nt] += w;
            p[nt][x >> 3][x & 7] = (bf16_t)(F ? w * vf[x] : w);
        }
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int x = 0; x < 16; ++x) st.o[dt][nt][x] *= alpha;
    }
}

// Iteration t (t = P mod 4).  now: scores of tile t; next: receives those of tile t + 1; kf: K fragments of tile t + 1, then of
// t + 2; before: probabilities of tile t - 1; p: receives those of tile t; sv, s1, sk, s3: stages P, P + 1, P + 2, P + 3; fk, fv:
// factors of the tile's first four keys, then of the next tile's.
template <int D, bool F, class SRC>
__device__ __forceinline__ void step(State<D> &st, floatx16 (&now)[2], floatx16 (&next)[2], bf16x8 (&kf)[D / 16],
                                     const bf16x8 (&q)[2][D / 16], const bf16x8 (&before)[2][2], bf16x8 (&p)[2][2], Stage<D, F> &sv,
                                     const Stage<D, F> &s1, const Stage<D, F> &sk, Stage<D, F> &s3, floatx4 (&fk)[2], floatx4 (&fv)[2],
                                     const int (&sees)[2], int t, int all, float c2, int h, const SRC &src, const Offsets<D> &off,
                                     int wave, int lane)
{
    typedef Slots<D> SL;
    bf16x8 vf[D / 16];
    if (__builtin_expect((t + 1) * KS > all, 0)) {
        asm volatile("" ::: "memory");                     // keeps this rare block out of the straight-line code
        mask_scores<D>(now, sees, t * KS, h);
    }
    __builtin_amdgcn_sched_barrier(0);
    // score pair z in three stages, each in another slot: multiply-add, exponentials, sum and pack.  Pairs of the first query tile
    // come first; with factors the two tiles take turns, so that four factors serve four pairs in a row.
    floatx2 sum[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}}, ex = {0.0f, 0.0f}, ar = {0.0f, 0.0f};
    auto pack = [&](auto zc) __attribute__((always_inline)) {
        constexpr int z = decltype(zc)::value;
        if constexpr (z >= 0 && z < 16) {
            constexpr int nt = SL::template nt_of<F>(z), x = 2 * SL::template pair_of<F>(z);
            bf16x2 t2;
            if constexpr (F) t2 = __builtin_convertvector(ex * floatx2{fv[x >> 2 & 1][x & 3], fv[x >> 2 & 1][(x & 3) + 1]}, bf16x2);
            else t2 = __builtin_convertvector(ex, bf16x2);
            asm volatile("" : "+v"(t2));
            if constexpr (x == 0) sum[nt] = ex;
            else sum[nt] += ex;
            asm volatile("" : "+v"(sum[nt]));
            p[nt][x >> 3][x & 7] = t2[0];
            p[nt][x >> 3][(x & 7) + 1] = t2[1];
        }
    };
    auto exps = [&](auto zc) __attribute__((always_inline)) {
        constexpr int z = decltype(zc)::value;
        if constexpr (z >= 0 && z < 16) {
            ex[0] = __builtin_amdgcn_exp2f(ar[0]);
            ex[1] = __builtin_amdgcn_exp2f(ar[1]);
        }
    };
    auto mads = [&](auto zc) __attribute__((always_inline)) {
        constexpr int z = decltype(zc)::value;
        if constexpr (z >= 0 && z < 16) {
            constexpr int nt = SL::template nt_of<F>(z), x = 2 * SL::template pair_of<F>(z);
            if constexpr (F && z % 4 == 0) fk[x >> 2 & 1] *= c2;
            ar[0] = __builtin_fmaf(now[nt][x], F ? fk[x >> 2 & 1][x & 3] : c2, -st.m[nt]);
            ar[1] = __builtin_fmaf(now[nt][x + 1], F ? fk[x >> 2 & 1][(x & 3) + 1] : c2, -st.m[nt]);
        }
    };
    auto softmax_slot = [&](auto mc) __attribute__((always_inline)) {
        constexpr int m = decltype(mc)::value;
        if constexpr (D == 128) {
            if constexpr (m % 2 == 0) {
                pack(std::integral_constant<int, m / 2 - 1>{});
                mads(std::integral_constant<int, m / 2>{});
            } else {
                exps(std::integral_constant<int, m / 2>{});
            }
        } else {
            pack(std::integral_constant<int, m - 2>{});
            exps(std::integral_constant<int, m - 1>{});
            mads(std::integral_constant<int, m>{});
        }
        if constexpr (m >= SL::kScores) asm volatile("" : "+v"(ex), "+v"(ar));
        __builtin_amdgcn_sched_barrier(0);
    };
    typename SRC::At where = {};
    unsigned char *dst = wave == 0 ? sv.k : sv.v;
    auto slot = [&](auto mc) __attribute__((always_inline)) {
        constexpr int m = decltype(mc)::value;
        if constexpr (m < SL::kScores) {
            constexpr int x = m >> 1;
            if constexpr (m == 0) score_first<D>(next[0], kf[0], q[0][0]);
            else if constexpr (m == 1) score_first<D>(next[1], kf[0], q[1][0]);
            else if constexpr ((m & 1) == 0) score_next<D>(next[0], kf[x], q[0][x]);
            else score_next<D>(next[1], kf[x], q[1][x]);
            __builtin_amdgcn_sched_barrier(0);
        } else {
            constexpr int n = m - SL::kScores, nt = SL::pv_nt(n), dt = SL::pv_dt(n), u = SL::pv_u(n);
            st.o[dt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * dt + u], before[nt][u], st.o[dt][nt], 0, 0, 0);
        }
        constexpr int v = SL::v_read(m), k = SL::k_read(m), l = SL::load(m);
        if constexpr (l >= 0) src.load(dst, l, where, off);
        if constexpr (F && m == SL::kFactors) src.load_factors(wave == 0 ? s3.kf : s3.vf, t + 3, lane);
        constexpr int g = SL::factors_read(m);             // factors of four keys, or of the next tile's first four
        if constexpr (F && g >= 0) {
            fk[g & 1] = *reinterpret_cast<const floatx4 *>((g < 4 ? sv.kf : s1.kf) + 8 * (g & 3) + 4 * h);
            fv[g & 1] = *reinterpret_cast<const floatx4 *>((g < 4 ? sv.vf : s1.vf) + 8 * (g & 3) + 4 * h);
        }
        if constexpr (v >= 0) vf[v] = read_v<D>(sv.v, off, v >> 1, v & 1);
        if constexpr (k >= 0) kf[k] = *reinterpret_cast<const bf16x8 *>(sk.k + off.kf[k]);
        if constexpr (m == SL::kMeet - 2) {
            where = src.at(t + (wave == 0 ? 4 : 3));
            where.pin();                                   // formed here
        }
        softmax_slot(mc);
        if constexpr (m == SL::kMeet) {
            // every load but the previous iteration's, and this wave's reads of V, are there
            __builtin_amdgcn_s_waitcnt(0x0070 + Offsets<D>::kLoads + (F ? 1 : 0));   // vmcnt; lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    unrolled(slot, std::make_integer_sequence<int, SL::kAll>{});
    softmax_slot(std::integral_constant<int, SL::kAll>{});
    if constexpr (D == 64) softmax_slot(std::integral_constant<int, SL::kAll + 1>{});
    float tile_sum[2] = {sum[0][0] + sum[0][1], sum[1][0] + sum[1][1]};
    if (__builtin_expect(__any(!(tile_sum[0] <= kBigSum) || !(tile_sum[1] <= kBigSum)), 0)) {
        asm volatile("" ::: "memory");
        float key_f[16], value_f[16];
        if constexpr (F) {
            read_factors(key_f, sv.kf, h);
            read_factors(value_f, sv.vf, h);
#pragma unroll
            for (int x = 0; x < 16; ++x) key_f[x] *= c2;
        }
        move_reference<D, F>(st, now, p, tile_sum, c2, key_f, value_f);
    }
    st.l[0] += tile_sum[0];
    st.l[1] += tile_sum[1];
    __builtin_amdgcn_sched_barrier(0);
}

// the last tile's second product
template <int D, bool F>
__device__ __forceinline__ void drain(State<D> &st, const bf16x8 (&p)[2][2], const Stage<D, F> &sg, const Offsets<D> &off)
{
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            const bf16x8 vf = read_v<D>(sg.v, off, dt, u);
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
                st.o[dt][nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[nt][u], st.o[dt][nt], 0, 0, 0);
        }
}

template <int D>
__device__ __forceinline__ void clear(State<D> &st)
{
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        st.m[nt] = -INFINITY;
        st.l[nt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) st.o[dt][nt] = floatx16{0};
    }
}

// Keys of tiles 0 .. tiles - 1 (at least one), of which the wave's rows all see those below `all`.
// load_queries brings the rows' queries into q, behind the first tiles' loads.  At the end no load into LDS is left, of either wave.
template <int D, bool F, class SRC, class LQ>
__device__ __forceinline__ void all_tiles(State<D> &st, bf16x8 (&q)[2][D / 16], LQ load_queries, const int (&sees)[2], int all,
                                          int tiles, float c2, const SRC &src, const Offsets<D> &off, Stage<D, F> &sg0, Stage<D, F> &sg1,
                                          Stage<D, F> &sg2, Stage<D, F> &sg3, int wave, int lane)
{
    const int h = lane >> 5;
    // stage p: K tile p, V tile p - 1; the V tile of stage 0, number 3, comes again in iteration 0: zero weights need some values
    issue_tile(sg0, src, off, wave == 0 ? 0 : 3, wave);
    issue_factors(sg0, src, 0, wave, lane);
    __builtin_amdgcn_sched_barrier(0);
    load_queries();
    __builtin_amdgcn_sched_barrier(0);
    issue_tile(sg1, src, off, wave == 0 ? 1 : 0, wave);
    issue_factors(sg1, src, 1, wave, lane);
    issue_tile(sg2, src, off, wave == 0 ? 2 : 1, wave);
    issue_factors(sg2, src, 2, wave, lane);
    issue_tile(sg3, src, off, wave == 0 ? 3 : 2, wave);
    constexpr int kEach = Offsets<D>::kLoads + (F ? 1 : 0);
    meet_but<2 * kEach + Offsets<D>::kLoads>();            // the first tile and the queries are there
    floatx16 sa[2], sb[2];
    bf16x8 kf[D / 16], pa[2][2], pb[2][2];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) kf[x] = *reinterpret_cast<const bf16x8 *>(sg0.k + off.kf[x]);
    score_first<D>(sa[0], kf[0], q[0][0]);
    score_first<D>(sa[1], kf[0], q[1][0]);
#pragma unroll
    for (int x = 1; x < D / 16; ++x) {
        score_next<D>(sa[0], kf[x], q[0][x]);
        score_next<D>(sa[1], kf[x], q[1][x]);
    }
    fence();
    __builtin_amdgcn_sched_barrier(0);
    if (KS > all) mask_scores<D>(sa, sees, 0, h);
    {
        float key_f[16];
        if constexpr (F) read_factors(key_f, sg0.kf, h);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float top = -INFINITY;
#pragma unroll
            for (int x = 0; x < 16; ++x) top = fmaxf(top, F ? sa[nt][x] * key_f[x] : sa[nt][x]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            st.m[nt] = top == -INFINITY ? 0.0f : top * c2;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) pa[nt][u][e] = (bf16_t)0.0f;
        }
    }
    meet_but<kEach + Offsets<D>::kLoads>();                // the second one
#pragma unroll
    for (int x = 0; x < D / 16; ++x) kf[x] = *reinterpret_cast<const bf16x8 *>(sg1.k + off.kf[x]);
    __builtin_amdgcn_sched_barrier(0);
    floatx4 fk[2], fv[2];
    if constexpr (F) {
        fk[0] = *reinterpret_cast<const floatx4 *>(sg0.kf + 4 * h);
        fv[0] = *reinterpret_cast<const floatx4 *>(sg0.vf + 4 * h);
    }
    for (int t = 0;; t += 4) {
        step<D, F>(st, sa, sb, kf, q, pa, pb, sg0, sg1, sg2, sg3, fk, fv, sees, t, all, c2, h, src, off, wave, lane);
        step<D, F>(st, sb, sa, kf, q, pb, pa, sg1, sg2, sg3, sg0, fk, fv, sees, t + 1, all, c2, h, src, off, wave, lane);
        step<D, F>(st, sa, sb, kf, q, pa, pb, sg2, sg3, sg0, sg1, fk, fv, sees, t + 2, all, c2, h, src, off, wave, lane);
        step<D, F>(st, sb, sa, kf, q, pb, pa, sg3, sg0, sg1, sg2, fk, fv, sees, t + 3, all, c2, h, src, off, wave, lane);
        if (t + 4 >= tiles) break;                         // (ways out between the four cost 300 spilled registers and more)
    }
    drain<D>(st, pa, sg0, off);
    meet();
}

// Rows of 32 queries out of O^T (lane (n, h), value x of tile dt: feature 32 dt + 8 (x / 4) + 4 h + x % 4 of query n) through
// LDS, so that a store instruction writes whole rows: make() turns four features into elements E, put(row, piece, value) gets 16
// bytes of a row.  room: 32 rows of LDS of the wave's own, at most a stage; piece p of row n lies at place p ^ n.  Returns 0, or
// NaN if a value of the lane's query is not finite.
template <int D, typename E, class MAKE, class PUT>
__device__ __forceinline__ float rows_out(const State<D> &st, int nt, unsigned char *room, int lane, MAKE make, PUT put)
{
    constexpr int kRowB = D * (int)sizeof(E), kPieces = kRowB / 16, kGroup = 4 * (int)sizeof(E);
    typedef E ex4 __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(E) == 4) asm volatile("" : "+v"(lane));  // addresses are formed here, not ahead of the loop
    const int n = lane & 31, h = lane >> 5;
    float zero = 0.0f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const floatx16 &o = st.o[dt][nt];
            const floatx4 v = {o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]};
#pragma unroll
            for (int y = 0; y < 4; ++y) zero = __builtin_fmaf(v[y], 0.0f, zero);
            const int at = (8 * dt + 2 * x + h) * kGroup;
            *reinterpret_cast<ex4 *>(room + n * kRowB + ((at >> 4 ^ (n & (kPieces - 1))) << 4) + (at & 15)) =
                make(v);
        }
#pragma unroll
    for (int y = 0; y < 32 * kPieces / 64; ++y) {
        const int row = (64 * y + lane) / kPieces, piece = lane % kPieces;
        put(row, piece, *reinterpret_cast<const uintx4 *>(room + row * kRowB + ((piece ^ (row & (kPieces - 1))) << 4)));
    }
    return zero;
}

}  // namespace prompt
}  // namespace pbs
