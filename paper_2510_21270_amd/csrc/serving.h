// What the operators around the prefill path share: tensors given by strides, the rows of a paged cache.
#pragma once
#include "pbs_host.h"

namespace pbs {

inline bool good_strides(const pbs_strides &s, int es)
{
    return s.token >= 0 && s.head >= 0 && s.token * es % 16 == 0 && s.head * es % 16 == 0 && s.token < (1ll << 31) &&
           s.head < (1ll << 31);
}

inline bool good_input(const void *x, const pbs_strides &s, int es) { return aligned16(x) && good_strides(s, es); }

// Element offset of a row of which token and head are small and not negative: strides have 31 bits, so that two multiply-adds of
// 32 bits do (a product of 64 bits each takes eight instructions of a quarter of the rate).
__host__ __device__ __forceinline__ uint64_t row_offset(uint32_t token, uint32_t head, const pbs_strides &s)
{
    return (uint64_t)token * (uint32_t)s.token + (uint64_t)head * (uint32_t)s.head;
}

// rows of an output do not overlap: the finer of the two steps covers a row, the coarser one all rows of the finer
inline bool good_output(const void *x, const pbs_strides &s, long long tokens, long long heads, int d, int es)
{
    if (!good_input(x, s, es)) return false;
    if (tokens == 1) return heads == 1 || s.head >= d;
    if (heads == 1) return s.token >= d;
    return s.token >= s.head ? s.head >= d && s.token >= s.head * heads : s.token >= d && s.head >= s.token * tokens;
}

// Whether `groups` workgroups of `threads` along x are one launch: a dispatch counts its threads in 32 bits.
inline bool fits_grid(long long groups, int threads) { return groups * threads < 0x100000000ll; }

inline pbs_status check_cache(const pbs_cache *c)
{
    if (!c) return PBS_ERR_NULL;
    if (c->pages < 1 || c->page < 1 || c->h_kv < 1) return PBS_ERR_SHAPE;
    if (c->dtype != PBS_BF16 && c->dtype != PBS_E4M3 && c->dtype != PBS_I8) return PBS_ERR_UNSUPPORTED;
    if (c->d != 64 && c->d != 128) return PBS_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1)) != 0) return PBS_ERR_UNSUPPORTED;
    if ((long long)c->pages * c->page > 0x7fffffffLL || c->h_kv > 65535) return PBS_ERR_UNSUPPORTED;
    if (!c->K || !c->V) return PBS_ERR_NULL;
    if (c->dtype != PBS_BF16 && (!c->k_scale || !c->v_scale)) return PBS_ERR_NULL;
    if (!aligned16(c->K) || !aligned16(c->V)) return PBS_ERR_SHAPE;
    if (c->dtype != PBS_BF16 && (!aligned16(c->k_scale) || !aligned16(c->v_scale))) return PBS_ERR_SHAPE;
    return PBS_OK;
}

inline int log2_of(int v)
{
    int l = 0;
    while ((1 << l) < v) ++l;
    return l;
}

// four 8-bit values as two pairs of bf16
template <int DTYPE>
__device__ __forceinline__ uintx2 widen4(uint32_t w)
{
    if constexpr (DTYPE == PBS_E4M3) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
        return uintx2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    } else {
        const floatx2 a = {(float)(int)(int8_t)w, (float)(int)(int8_t)(w >> 8)};
        const floatx2 b = {(float)(int)(int8_t)(w >> 16), (float)(int)(int8_t)(w >> 24)};
        return uintx2{__builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2)),
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2))};
    }
}

// eight consecutive elements as float, and back with one rounding
__device__ __forceinline__ void load8(const bf16_t *p, float (&x)[8])
{
    const bf16x8 v = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8])
{
    const floatx4 u = reinterpret_cast<const floatx4 *>(p)[0], v = reinterpret_cast<const floatx4 *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&x)[8])
{
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (bf16_t)x[i];
    *reinterpret_cast<bf16x8 *>(p) = v;
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    reinterpret_cast<floatx4 *>(p)[0] = floatx4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<floatx4 *>(p)[1] = floatx4{x[4], x[5], x[6], x[7]};
}

}  // namespace pbs
