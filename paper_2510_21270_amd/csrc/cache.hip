// pbs_cache_write, pbs_cache_read: the rows of a paged key/value cache.
//
// A row (token, kv head) is d features: 8 to a lane, 8 or 16 lanes; a thread has its piece of the K row and of the V row.
// Writing in 8 bits finds a row's largest magnitude across these lanes and divides by f = max(largest / M, 2^-126); both
// divisions are IEEE fp32, so that what is held is the same wherever it is formed.  Magnitudes are compared as bit
// patterns: infinite and NaN features are the largest ones and show.  Bytes bound both directions: 32768 tokens of 8 heads of 128
// between bf16 and e4m3 are written in 44 us and read in 34 us (4.6 and 6.0 TB/s read and written).
#include "pbs_host.h"
#include "serving.h"

namespace pbs {

constexpr int kCacheThreads = 256;
constexpr float kTinyFactor = 1.17549435e-38f;             // 2^-126

struct CacheArgs {
    int rows, h_kv, page_log, slots;                       // rows: tokens * h_kv; slots: pages * page
    unsigned d_log;                                        // 6 or 7
    pbs_strides x[2];                                      // K, V
    const int32_t *slot;
};

// Where row h of slot s lies, in rows.
__device__ __forceinline__ int64_t cache_row(int s, int h, int h_kv, int page_log)
{
    return (((int64_t)(s >> page_log) * h_kv + h) << page_log) + (s & ((1 << page_log) - 1));
}

struct Held8 { uint32_t lo, hi; };                         // eight 8-bit values

template <int DTYPE>
__device__ __forceinline__ Held8 round_to_held(const float (&y)[8])
{
    Held8 q;
    if constexpr (DTYPE == PBS_E4M3) {
        int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
        q.lo = lo;
        q.hi = hi;
    } else {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = (uint32_t)(int)rintf(y[i]) & 255u;
        q.lo = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
        q.hi = b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24;
    }
    return q;
}

template <int DTYPE>
__device__ __forceinline__ void held_to_float(const Held8 &q, float (&x)[8])
{
    if constexpr (DTYPE == PBS_E4M3) {
        const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8(q.lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(q.lo, true);
        const floatx2 c = __builtin_amdgcn_cvt_pk_f32_fp8(q.hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(q.hi, true);
        x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
        x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = (float)(int)(int8_t)(q.lo >> (8 * i));
            x[4 + i] = (float)(int)(int8_t)(q.hi >> (8 * i));
        }
    }
}

// x / f, rounded as IEEE division does, by the reciprocal y = 1 / f and two corrections: with y rounded correctly and q within a
// step of the quotient, x - q f is exact and q + y (x - q f) rounds correctly (Markstein 1990).  The first correction brings q
// there.  Exact as long as x - q f does not fall below the smallest numbers, which is what `small` rows are kept away from.
__device__ __forceinline__ float quotient(float x, float f, float y)
{
    float q = x * y;
    q = __builtin_fmaf(__builtin_fmaf(-q, f, x), y, q);
    return __builtin_fmaf(__builtin_fmaf(-q, f, x), y, q);
}

// Eight features of a row in 8 bits, and the row's factor.
template <int DTYPE>
__device__ __forceinline__ Held8 hold8(const float (&x)[8], int lanes, float &factor)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
    for (int o = lanes >> 1; o > 0; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
    const bool finite = most < 0x7f800000u, small = most < 0x21800000u;        // 2^-60
    const float f = fmaxf(__uint_as_float(most) / (DTYPE == PBS_E4M3 ? 448.0f : 127.0f), kTinyFactor), y = 1.0f / f;
    float q[8];
    if (__any(small || !finite)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = finite ? x[i] / f : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = quotient(x[i], f, y);
    }
    factor = finite ? f : __uint_as_float(0x7fc00000u);
    return round_to_held<DTYPE>(q);
}

template <typename E, int DTYPE>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheArgs a, const E *__restrict__ K,
                                                                    const E *__restrict__ V, void *__restrict__ Kc,
                                                                    void *__restrict__ Vc, float *__restrict__ kf,
                                                                    float *__restrict__ vf)
{
    const int lanes = 1 << (a.d_log - 3);                  // to a row
    const int64_t at = (int64_t)blockIdx.x * kCacheThreads + threadIdx.x;
    const int row = (int)(at >> (a.d_log - 3)), lane = (int)at & (lanes - 1);
    if (row >= a.rows) return;                             // whole rows leave together
    const int t = row / a.h_kv, h = row - t * a.h_kv;
    const int s = a.slot[t];
    float k[8], v[8];
    load8(K + (int64_t)t * a.x[0].token + (int64_t)h * a.x[0].head + 8 * lane, k);
    load8(V + (int64_t)t * a.x[1].token + (int64_t)h * a.x[1].head + 8 * lane, v);
    if (s < 0 || s >= a.slots) return;
    const int64_t to = cache_row(s, h, a.h_kv, a.page_log), place = (to << a.d_log) + 8 * lane;
    if constexpr (DTYPE == PBS_BF16) {
        store8(static_cast<bf16_t *>(Kc) + place, k);
        store8(static_cast<bf16_t *>(Vc) + place, v);
    } else {
        float fk, fv;
        const Held8 qk = hold8<DTYPE>(k, lanes, fk), qv = hold8<DTYPE>(v, lanes, fv);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(Kc) + place) = make_uint2(qk.lo, qk.hi);
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(Vc) + place) = make_uint2(qv.lo, qv.hi);
        if (lane == 0) {
            kf[to] = fk;
            vf[to] = fv;
        }
    }
}

// blockIdx.y: 0 = K, 1 = V.
template <typename E, int DTYPE>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(CacheArgs a, E *__restrict__ K, E *__restrict__ V,
                                                                   const void *__restrict__ Kc,
                                                                   const void *__restrict__ Vc,
                                                                   const float *__restrict__ kf,
                                                                   const float *__restrict__ vf)
{
    const int lanes = 1 << (a.d_log - 3);
    const int64_t at = (int64_t)blockIdx.x * kCacheThreads + threadIdx.x;
    const int row = (int)(at >> (a.d_log - 3)), lane = (int)at & (lanes - 1);
    if (row >= a.rows) return;
    const bool is_v = blockIdx.y != 0;
    E *out = is_v ? V : K;
    if (!out) return;
    const int t = row / a.h_kv, h = row - t * a.h_kv;
    const int s = a.slot[t];
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (s >= 0 && s < a.slots) {
        const int64_t from = cache_row(s, h, a.h_kv, a.page_log);
        if constexpr (DTYPE == PBS_BF16) {
            load8(static_cast<const bf16_t *>(is_v ? Vc : Kc) + (from << a.d_log) + 8 * lane, x);
        } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(is_v ? Vc : Kc) +
                                                             (from << a.d_log) + 8 * lane);
            const float f = (is_v ? vf : kf)[from];
            held_to_float<DTYPE>(Held8{v.x, v.y}, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= f;
        }
    }
    const pbs_strides &st = a.x[is_v ? 1 : 0];
    store8(out + (int64_t)t * st.token + (int64_t)h * st.head + 8 * lane, x);
}

inline long long cache_groups(const CacheArgs &a) { return (((int64_t)a.rows << (a.d_log - 3)) + kCacheThreads - 1) / kCacheThreads; }
inline dim3 cache_grid(const CacheArgs &a, int y) { return dim3((unsigned)cache_groups(a), y); }

inline pbs_status cache_args(const pbs_cache *c, int32_t dtype, int32_t tokens, const int32_t *slots, CacheArgs &a)
{
    const pbs_status st = check_cache(c);
    if (st != PBS_OK) return st;
    if (dtype != PBS_F32 && dtype != PBS_BF16) return PBS_ERR_UNSUPPORTED;
    if (tokens < 0) return PBS_ERR_SHAPE;
    if ((long long)tokens * c->h_kv > 0x7fffff00LL) return PBS_ERR_UNSUPPORTED;             // the last workgroup's rows are ints too
    if (tokens > 0 && !slots) return PBS_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(slots) & 3u) != 0) return PBS_ERR_SHAPE;
    a.rows = tokens * c->h_kv;
    a.h_kv = c->h_kv;
    a.page_log = log2_of(c->page);
    a.slots = c->pages * c->page;
    a.d_log = (unsigned)log2_of(c->d);
    a.slot = slots;
    if (!fits_grid(cache_groups(a), kCacheThreads)) return PBS_ERR_UNSUPPORTED;
    return PBS_OK;
}

template <typename E>
pbs_status write_rows(const pbs_cache *c, const CacheArgs &a, const void *K, const void *V, hipStream_t s)
{
    const E *k = static_cast<const E *>(K), *v = static_cast<const E *>(V);
    auto kernel = c->dtype == PBS_BF16 ? cache_write_kernel<E, PBS_BF16>
                  : c->dtype == PBS_E4M3 ? cache_write_kernel<E, PBS_E4M3> : cache_write_kernel<E, PBS_I8>;
    return launch(kernel, cache_grid(a, 1), dim3(kCacheThreads), 0, s, a, k, v, c->K, c->V, c->k_scale, c->v_scale);
}

template <typename E>
pbs_status read_rows(const pbs_cache *c, const CacheArgs &a, void *K, void *V, hipStream_t s)
{
    E *k = static_cast<E *>(K), *v = static_cast<E *>(V);
    auto kernel = c->dtype == PBS_BF16 ? cache_read_kernel<E, PBS_BF16>
                  : c->dtype == PBS_E4M3 ? cache_read_kernel<E, PBS_E4M3> : cache_read_kernel<E, PBS_I8>;
    return launch(kernel, cache_grid(a, 2), dim3(kCacheThreads), 0, s, a, k, v, static_cast<const void *>(c->K),
                  static_cast<const void *>(c->V), static_cast<const float *>(c->k_scale),
                  static_cast<const float *>(c->v_scale));
}

}  // namespace pbs

extern "C" pbs_status pbs_cache_write(const pbs_cache *c, int32_t dtype, int32_t tokens, const void *K,
                                      const pbs_strides *k, const void *V, const pbs_strides *v, const int32_t *slots,
                                      void *stream)
{
    using namespace pbs;
    CacheArgs a;
    const pbs_status st = cache_args(c, dtype, tokens, slots, a);
    if (st != PBS_OK) return st;
    if (tokens == 0) return PBS_OK;
    if (!K || !V || !k || !v) return PBS_ERR_NULL;
    const int es = (int)elem_size(dtype);
    if (!good_input(K, *k, es) || !good_input(V, *v, es)) return PBS_ERR_SHAPE;
    a.x[0] = *k;
    a.x[1] = *v;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == PBS_BF16 ? write_rows<bf16_t>(c, a, K, V, s) : write_rows<float>(c, a, K, V, s);
}

extern "C" pbs_status pbs_cache_read(const pbs_cache *c, int32_t dtype, int32_t tokens, const int32_t *slots, void *K,
                                     const pbs_strides *k, void *V, const pbs_strides *v, void *stream)
{
    using namespace pbs;
    CacheArgs a;
    const pbs_status st = cache_args(c, dtype, tokens, slots, a);
    if (st != PBS_OK) return st;
    if (tokens == 0) return PBS_OK;
    if ((!K && !V) || (K && !k) || (V && !v)) return PBS_ERR_NULL;
    const int es = (int)elem_size(dtype);
    if (K && !good_output(K, *k, tokens, c->h_kv, c->d, es)) return PBS_ERR_SHAPE;
    if (V && !good_output(V, *v, tokens, c->h_kv, c->d, es)) return PBS_ERR_SHAPE;
    a.x[0] = K ? *k : pbs_strides{0, 0};
    a.x[1] = V ? *v : pbs_strides{0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == PBS_BF16 ? read_rows<bf16_t>(c, a, K, V, s) : read_rows<float>(c, a, K, V, s);
}
