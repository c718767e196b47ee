// pbs_prompt_attn: causal attention over prompts packed one behind the other.
//
// The softmax of one pass, transposed as in the other matrix-core kernels (S^T = K Q^T, O^T += V^T P^T, v_mfma_f32_32x32x16_bf16):
// a lane owns one query of each 32-row tile, its probabilities are the B operand of the second product as they lie.  The rows
// of a tile are (token, head of the group): all query heads of a kv head share every key tile, a tile of 128 rows spans few
// tokens, so that little is multiplied above the diagonal and short prompts fill their tiles.
// A workgroup is two waves of 64 rows, one wave to a SIMD; keys go through LDS in tiles of 32 (K and V rows as they lie in memory, by
// asynchronous loads), V^T comes out of LDS through the transposing read (ds_read_b64_tr_b16: 4 rows x 16 features to 16 lanes).
//
// What bounds it is the matrix pipe and the vector work that has to fit beside it in one wave's instruction stream.  The loop is
// a pipeline in which no matrix instruction of an iteration depends on the vector arithmetic of the same one.  Iteration t:
//     S(t + 1) = K(t + 1) Q^T, then O^T += V^T(t - 1) P^T(t - 1); all along P^T(t) from S(t)
//     LDS: V^T(t - 1) is read under the first matrix instructions; the waves meet; K(t + 4) and V(t + 3) go out into what has
//     been read; K(t + 2) is read under the last ones
// Ring of four stages; stage p holds K tile p and V tile p - 1 (mod 4), which is what iteration p frees.
// The softmax of the loop keeps the reference that the first tile sets (any reference gives the same softmax while nothing
// overflows) and moves it, rescaling O^T and l, when a tile's sum passes 2^40.  What that leaves open (a row whose first
// tile has no finite logit; values that are not finite, which a hidden key's zero weight would turn into NaN) shows in O^T
// or l, and such a workgroup goes over its keys again, tile by tile with the running maximum (whole_tile).
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

struct Args {
    int n_seq, total_q, total_k, h_q, h_kv, r, tokens;     // tokens: of a workgroup's rows
    float c2;                                              // scale * log2(e)
    bool causal;
    pbs_strides q, k, v, o;
    const bf16_t *Q, *K, *V;
    const int32_t *cu_q, *cu_k;
    bf16_t *O;
    float *lse;
};

// A tile in LDS.  The 16-byte pieces of a row are stored permuted so that neither read meets itself in a bank:
//   k: piece c of row n at place c ^ (n % 16) (d = 64, 8 pieces to a row: c ^ (n / 2 % 8)): 16 lanes read 16 rows
//   v: piece c of row n at place c ^ 4 (n % 4) (d = 64: c ^ 4 (n / 2 % 2)): 16 lanes read 32 bytes of four rows
template <int D>
struct __align__(16) Stage {
    unsigned char k[KS * D * 2];
    unsigned char v[KS * D * 2];
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

template <int D>
__device__ __forceinline__ void issue_tile(unsigned char *dst, __amdgpu_buffer_rsrc_t src, const Offsets<D> &off, int from, int size)
{
    const int at = scalar_offset(from, size);
#pragma unroll
    for (int c = 0; c < Offsets<D>::kLoads; ++c)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lptr_t)(dst + c * 1024), 16, off.from[c], at, 0, 0);
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
template <int D>
__device__ __forceinline__ void whole_tile(State<D> &st, const Stage<D> &sg, const Offsets<D> &off, const bf16x8 (&q)[2][D / 16],
                                           const int (&sees)[2], int key0, float c2, int h)
{
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
            const bool hidden = 8 * (x >> 2) + (x & 3) >= lim;
            hides = hides || hidden;
            s[nt][x] = hidden ? -INFINITY : s[nt][x] * c2;
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
            p[nt][x >> 3][x & 7] = (bf16_t)w;
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
                for (int e = 0; e < 8; ++e) seen[e] = 16 * u + 8 * (e >> 2) + (e & 3) < lim ? (bf16_t)1.0f : (bf16_t)0.0f;
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
    static constexpr int v_read(int m) { return m < kFrags ? m : -1; }
    static constexpr int load(int m) { return m > kMeet && (m - kMeet) % 2 == 0 && (m - kMeet - 2) / 2 < Offsets<D>::kLoads ? (m - kMeet - 2) / 2 : -1; }
    static constexpr int k_read(int m) { return m >= kScores && m % 2 == 0 && (m - kScores) / 2 < kFrags ? (m - kScores) / 2 : -1; }
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
template <int D>
__device__ __forceinline__ void move_reference(State<D> &st, const floatx16 (&s)[2], bf16x8 (&p)[2][2], float (&sum)[2], float c2)
{
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) top = fmaxf(top, s[nt][x]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m = fmaxf(st.m[nt], top * c2), alpha = __builtin_amdgcn_exp2f(st.m[nt] - m);
        st.m[nt] = m;
        st.l[nt] *= alpha;
        sum[nt] = 0.0f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const float w = __builtin_amdgcn_exp2f(s[nt][x] * c2 - m);
            sum[nt] += w;
            p[nt][x >> 3][x & 7] = (bf16_t)w;
        }
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int x = 0; x < 16; ++x) st.o[dt][nt][x] *= alpha;
    }
}

template <int D>
struct Source {                                            // what this wave brings: wave 0 K, wave 1 V
    __amdgpu_buffer_rsrc_t rsrc;
    int size, tile_bytes, wave;
};

// Iteration t (t = P mod 4).  now: scores of tile t; next: receives those of tile t + 1; kf: K fragments of tile t + 1, then of
// t + 2; before: probabilities of tile t - 1; p: receives those of tile t; sv: stage P; sk: stage P + 2.
template <int D>
__device__ __forceinline__ void step(State<D> &st, floatx16 (&now)[2], floatx16 (&next)[2], bf16x8 (&kf)[D / 16],
                                     const bf16x8 (&q)[2][D / 16], const bf16x8 (&before)[2][2], bf16x8 (&p)[2][2], Stage<D> &sv,
                                     const Stage<D> &sk, const int (&sees)[2], int t, int all, float c2, int h, const Source<D> &src,
                                     const Offsets<D> &off)
{
    typedef Slots<D> SL;
    bf16x8 vf[D / 16];
    if (__builtin_expect((t + 1) * KS > all, 0)) {
        asm volatile("" ::: "memory");                     // keeps this rare block out of the straight-line code
        mask_scores<D>(now, sees, t * KS, h);
    }
    __builtin_amdgcn_sched_barrier(0);
    // score pair z in three stages, each in another slot: multiply-add, exponentials, sum and pack
    floatx2 sum[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}}, ex = {0.0f, 0.0f}, ar = {0.0f, 0.0f};
    auto pack = [&](auto zc) __attribute__((always_inline)) {
        constexpr int z = decltype(zc)::value, nt = z >> 3;
        if constexpr (z >= 0 && z < 16) {
            bf16x2 t2 = __builtin_convertvector(ex, bf16x2);
            asm volatile("" : "+v"(t2));
            if constexpr ((z & 7) == 0) sum[nt] = ex;
            else sum[nt] += ex;
            asm volatile("" : "+v"(sum[nt]));
            p[nt][(z & 7) >> 2][2 * (z & 3)] = t2[0];
            p[nt][(z & 7) >> 2][2 * (z & 3) + 1] = t2[1];
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
            ar[0] = __builtin_fmaf(now[z >> 3][2 * (z & 7)], c2, -st.m[z >> 3]);
            ar[1] = __builtin_fmaf(now[z >> 3][2 * (z & 7) + 1], c2, -st.m[z >> 3]);
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
    int at = 0;
    unsigned char *dst = src.wave == 0 ? sv.k : sv.v;
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
        if constexpr (l >= 0)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(src.rsrc, (lptr_t)(dst + l * 1024), 16, off.from[l], at, 0, 0);
        if constexpr (v >= 0) vf[v] = read_v<D>(sv.v, off, v >> 1, v & 1);
        if constexpr (k >= 0) kf[k] = *reinterpret_cast<const bf16x8 *>(sk.k + off.kf[k]);
        if constexpr (m == SL::kMeet - 2) {
            at = scalar_offset((t + (src.wave == 0 ? 4 : 3)) * src.tile_bytes, src.size);
            asm volatile("" : "+s"(at));
        }
        softmax_slot(mc);
        if constexpr (m == SL::kMeet) {
            // every load but the previous iteration's, and this wave's reads of V, are there
            __builtin_amdgcn_s_waitcnt(D == 128 ? 0x0078 : 0x0074);
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
        move_reference<D>(st, now, p, tile_sum, c2);
    }
    st.l[0] += tile_sum[0];
    st.l[1] += tile_sum[1];
    __builtin_amdgcn_sched_barrier(0);
}

// the last tile's second product
template <int D>
__device__ __forceinline__ void drain(State<D> &st, const bf16x8 (&p)[2][2], const Stage<D> &sg, const Offsets<D> &off)
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

// Which sequence and which of its tiles workgroup `b` has: the sequences' tiles one behind the other, a sequence's last
// tile, the longest, first.  Every wave looks for itself.  seq = -1: none is left.
struct Place { int seq, tile, q0, len_q, k0, len_k; };
__device__ __forceinline__ Place find_place(const Args &a, int b, int lane)
{
    Place p = {-1, 0, 0, 0, 0, 0};
    int before = 0;
    for (int base = 0; base < a.n_seq; base += 64) {
        const int i = base + lane;
        int q0 = 0, len = 0;
        if (i < a.n_seq) {
            q0 = min(max(a.cu_q[i], 0), a.total_q);
            len = max(min(max(a.cu_q[i + 1], 0), a.total_q) - q0, 0);
        }
        const int tiles = (len + a.tokens - 1) / a.tokens;
        int sum = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int other = __shfl_up(sum, o, 64);
            if (lane >= o) sum += other;
        }
        const int total = __builtin_amdgcn_readlane(sum, 63);
        if (b < before + total) {
            const unsigned long long has = __ballot(b < before + sum);
            const int at = __builtin_ctzll(has);
            p.seq = base + at;
            p.q0 = __builtin_amdgcn_readlane(q0, at);
            p.len_q = __builtin_amdgcn_readlane(len, at);
            const int in = b - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(tiles, at));
            p.tile = __builtin_amdgcn_readlane(tiles, at) - 1 - in;
            const int k0 = min(max(a.cu_k[p.seq], 0), a.total_k);
            p.k0 = __builtin_amdgcn_readfirstlane(k0);
            p.len_k = __builtin_amdgcn_readfirstlane(max(min(max(a.cu_k[p.seq + 1], 0), a.total_k) - k0, 0));
            return p;
        }
        before += total;
    }
    return p;
}

// lane (n, h), value x of O^T tile dt: feature 32 dt + 8 (x / 4) + 4 h + x % 4 of query n
template <int D>
__device__ __forceinline__ void store_rows(const Args &a, const Place &pl, const State<D> &st, int kv, int t0, int rows, int wave, int n, int h)
{
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int row = wave * 64 + 32 * nt + n;
        const float l = st.l[nt] + __shfl_xor(st.l[nt], 32, 64);
        if (row < rows) {
            const int t = t0 + row / a.r, head = kv * a.r + row % a.r;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            bf16_t *dst = a.O + (int64_t)(pl.q0 + t) * a.o.token + (int64_t)head * a.o.head + 4 * h;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const floatx16 &o = st.o[dt][nt];
                    floatx4 v = floatx4{o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]} * inv;
                    if (l == 0.0f) v = floatx4{0};
                    *reinterpret_cast<bf16x4 *>(dst + 32 * dt + 8 * x) = __builtin_convertvector(v, bf16x4);
                }
            if (a.lse && h == 0)
                a.lse[(int64_t)(pl.q0 + t) * a.h_q + head] = l == 0.0f ? -INFINITY : (st.m[nt] + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        }
    }
}

template <int D>
__global__ __launch_bounds__(128) __attribute__((amdgpu_waves_per_eu(1, 1))) void prompt_kernel(Args a)
{
    __shared__ Stage<D> sg0, sg1, sg2, sg3;                // apart, so that a read of one does not wait for loads into another
    __shared__ int bad_rows;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = blockIdx.x % a.h_kv;
    const Place pl = find_place(a, blockIdx.x / a.h_kv, lane);
    if (pl.seq < 0) return;
    const int t0 = pl.tile * a.tokens, rows = min(a.tokens, pl.len_q - t0) * a.r;
    const int ahead = pl.len_k - pl.len_q;                 // keys in front of the first query

    bf16x8 q[2][D / 16];
    int sees[2];
    State<D> st;
    auto init = [&]() {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            st.m[nt] = -INFINITY;
            st.l[nt] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) st.o[dt][nt] = floatx16{0};
        }
    };
    init();
    auto load_queries = [&]() {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const int row = wave * 64 + 32 * nt + n, rc = min(row, rows - 1);
            const int t = t0 + rc / a.r, head = kv * a.r + rc % a.r;
            const bf16_t *src = a.Q + (int64_t)(pl.q0 + t) * a.q.token + (int64_t)head * a.q.head + 8 * h;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) q[nt][x] = *reinterpret_cast<const bf16x8 *>(src + 16 * x);
            sees[nt] = a.causal ? min(max(t + ahead + 1, 0), pl.len_k) : pl.len_k;
        }
    };
    load_queries();
    const int last = a.causal ? min(max(t0 + (rows - 1) / a.r + ahead + 1, 0), pl.len_k) : pl.len_k;   // keys that any row sees
    const int tiles = (last + KS - 1) / KS;

    const pbs_strides &ks = wave == 0 ? a.k : a.v;
    const bf16_t *base = (wave == 0 ? a.K : a.V) + (int64_t)pl.k0 * ks.token + (int64_t)kv * ks.head;
    const int step_bytes = (int)ks.token * 2;
    const int size = pl.len_k > 0 ? (pl.len_k - 1) * step_bytes + D * 2 : 0;
    const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(base), 0, size, 0x00020000);
    const Offsets<D> off = offsets<D>(wave, lane, (uint32_t)step_bytes);

    if (threadIdx.x == 0) bad_rows = 0;
    bool bad = false;
    if (tiles > 0) {
        const Source<D> sr = {src, size, KS * step_bytes, wave};
        auto issue = [&](Stage<D> &sg, int kt, int vt) {
            issue_tile<D>(wave == 0 ? sg.k : sg.v, src, off, (wave == 0 ? kt : vt) * KS * step_bytes, size);
        };
        issue(sg0, 0, 3);                                  // V tile 3 comes again in iteration 0: weights of zero need some values
        issue(sg1, 1, 0);
        issue(sg2, 2, 1);
        issue(sg3, 3, 2);
        meet();
        const int all = __builtin_amdgcn_readfirstlane(sees[0]);               // the wave's first row sees the fewest keys
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
        if (KS > all) mask_scores<D>(sa, sees, 0, h);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float top = -INFINITY;
#pragma unroll
            for (int x = 0; x < 16; ++x) top = fmaxf(top, sa[nt][x]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            st.m[nt] = top == -INFINITY ? 0.0f : top * a.c2;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) pa[nt][u][e] = (bf16_t)0.0f;
        }
#pragma unroll
        for (int x = 0; x < D / 16; ++x) kf[x] = *reinterpret_cast<const bf16x8 *>(sg1.k + off.kf[x]);
        __builtin_amdgcn_sched_barrier(0);
        for (int t = 0;; t += 4) {
            step<D>(st, sa, sb, kf, q, pa, pb, sg0, sg2, sees, t, all, a.c2, h, sr, off);
            step<D>(st, sb, sa, kf, q, pb, pa, sg1, sg3, sees, t + 1, all, a.c2, h, sr, off);
            step<D>(st, sa, sb, kf, q, pa, pb, sg2, sg0, sees, t + 2, all, a.c2, h, sr, off);
            step<D>(st, sb, sa, kf, q, pb, pa, sg3, sg1, sees, t + 3, all, a.c2, h, sr, off);
            if (t + 4 >= tiles) break;                     // (ways out between the four cost 300 spilled registers and more)
        }
        drain<D>(st, pa, sg0, off);
        float zero = 0.0f;                                 // NaN if a value of O^T is not finite
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int x = 0; x < 16; ++x) zero = __builtin_fmaf(st.o[dt][nt][x], 0.0f, zero);
            const float l = st.l[nt] + __shfl_xor(st.l[nt], 32, 64);
            bad = bad || (l == 0.0f && sees[nt] > 0);
            zero = __builtin_fmaf(l, 0.0f, zero);
        }
        bad = bad || zero != 0.0f;
        store_rows<D>(a, pl, st, kv, t0, rows, wave, n, h);
    }
    meet();                                                // loads past the last tile have landed too
    if (__any(bad) && lane == 0) bad_rows = 1;
    __syncthreads();
    if (__builtin_expect(bad_rows != 0 || tiles == 0, 0)) {
        init();
        load_queries();
        for (int t = 0; t < tiles; ++t) {
            __syncthreads();
            issue_tile<D>(wave == 0 ? sg0.k : sg0.v, src, off, t * KS * step_bytes, size);
            meet();
            whole_tile<D>(st, sg0, off, q, sees, t * KS, a.c2, h);
        }
        store_rows<D>(a, pl, st, kv, t0, rows, wave, n, h);
    }

}

}  // namespace prompt
}  // namespace pbs

extern "C" pbs_status pbs_prompt_attn(const pbs_prompt_problem *p, const void *Q, const void *K, const void *V,
                                      const int32_t *cu_q, const int32_t *cu_k, void *O, float *lse, void *stream)
{
    using namespace pbs;
    if (!p) return PBS_ERR_NULL;
    if (p->n_seq < 0 || p->total_q < 0 || p->total_k < 0 || p->h_q < 1 || p->h_kv < 1 || p->h_q % p->h_kv != 0) return PBS_ERR_SHAPE;
    if (!(p->scale >= 0.0f) || isinf(p->scale)) return PBS_ERR_SHAPE;
    if (p->dtype != PBS_BF16 || (p->d != 64 && p->d != 128)) return PBS_ERR_UNSUPPORTED;
    const int r = p->h_q / p->h_kv, tokens = prompt::kRows / (r < prompt::kRows ? r : prompt::kRows);
    if (r > prompt::kRows || (long long)p->total_q * p->h_q > 0x7fffffffLL || (long long)p->total_k * p->h_kv > 0x7fffffffLL)
        return PBS_ERR_UNSUPPORTED;
    if (p->n_seq == 0 || p->total_q == 0) return PBS_OK;
    if (!Q || !cu_q || !cu_k || !O || (p->total_k > 0 && (!K || !V))) return PBS_ERR_NULL;
    if (!good_input(Q, p->q, 2) || !good_output(O, p->o, p->total_q, p->h_q, p->d, 2)) return PBS_ERR_SHAPE;
    if (p->total_k > 0 && (!good_input(K, p->k, 2) || !good_input(V, p->v, 2))) return PBS_ERR_SHAPE;
    if (((reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(cu_k) | reinterpret_cast<uintptr_t>(lse)) & 3u) != 0)
        return PBS_ERR_SHAPE;
    // byte offsets inside a head's rows, a tile past the end included, are 31 bits
    const long long stride = p->k.token > p->v.token ? p->k.token : p->v.token;
    if (((long long)p->total_k + 2 * prompt::KS) * stride * 2 + p->d * 2 >= 0x80000000ll) return PBS_ERR_UNSUPPORTED;
    const long long grid = ((long long)p->total_q / tokens + p->n_seq) * p->h_kv;
    if (grid > 0x7fffffffLL) return PBS_ERR_UNSUPPORTED;

    prompt::Args a;
    a.n_seq = p->n_seq; a.total_q = p->total_q; a.total_k = p->total_k;
    a.h_q = p->h_q; a.h_kv = p->h_kv; a.r = r; a.tokens = tokens;
    a.c2 = (p->scale > 0.0f ? p->scale : (float)(1.0 / sqrt((double)p->d))) * 1.4426950408889634f;
    a.causal = (p->flags & PBS_PROMPT_CAUSAL) != 0;
    a.q = p->q; a.k = p->k; a.v = p->v; a.o = p->o;
    a.Q = static_cast<const bf16_t *>(Q);
    a.K = static_cast<const bf16_t *>(K);
    a.V = static_cast<const bf16_t *>(V);
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.O = static_cast<bf16_t *>(O);
    a.lse = lse;
    return launch(p->d == 128 ? prompt::prompt_kernel<128> : prompt::prompt_kernel<64>, dim3((unsigned)grid), dim3(128), 0,
                  static_cast<hipStream_t>(stream), a);
}
