// The prefix of pbs_decode_attn against many rows: the queries of the whole batch, 128 to a workgroup, on the pipeline of
// key_pipeline.h.  A part of the keys and a kv head to a workgroup; O, m and l of every part go to the workspace.
//
// A bf16 cache is read where its pages lie.  8-bit values are first written out as bf16, in order, the factors beside them: the
// pipeline has no room for the widening of every tile in every workgroup, and the prefix is short beside what is done with it.
// What bounds it is the start and the end of the workgroups, about 7 us, where a part has few tiles (48 answers to 8147 keys, 28 heads
// on 4 of 128, bf16: 20 us for 5.7 GFLOP), the pipeline from some ten thousand keys on.
#include "decode.h"
#include "key_pipeline.h"

namespace pbs {
namespace prompt {

// Tiles of a part from the pages of a cache.  held: the pages of the part's 32 tiles in a wave's lanes, two to a tile.  The halves of a
// tile have a descriptor each where a page is no more (HALVES), which ends with the keys that exist: what lies behind them reads as
// zeros.
template <int D, bool HALVES>
struct Pages {
    const bf16_t *pool;
    int held, count, begin, page_log, h, h_kv;
    struct At {
        __amdgpu_buffer_rsrc_t lo, hi;
        __device__ __forceinline__ void pin() {}
    };
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t half(int t, int u) const
    {
        const int page = __builtin_amdgcn_readlane(held, (2 * t + u) & 63), rows = min(count - t * KS, KS);
        const int place = (begin + t * KS + 16 * u) & ((1 << page_log) - 1);
        const bf16_t *base = pool + (((((int64_t)max(page, 0)) * h_kv + h) << page_log) + place - 16 * u) * D;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(base), 0, page >= 0 && rows > 16 * u ? rows * D * 2 : 0, 0x00020000);
    }
    __device__ __forceinline__ At at(int t) const
    {
        At w;
        w.lo = half(t, 0);
        if constexpr (HALVES) w.hi = half(t, 1);
        return w;
    }
    __device__ __forceinline__ void load(unsigned char *dst, int c, const At &w, const Offsets<D> &off) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(!HALVES || c < Offsets<D>::kLoads / 2 ? w.lo : w.hi, (lptr_t)(dst + c * 1024), 16, off.from[c], 0, 0, 0);
    }
    __device__ __forceinline__ void load_factors(float *, int, int) const {}
};

// LINE: the keys lie in order as bf16 with factors beside them.  HALVES: in pages of 16.
template <int D, bool LINE, bool HALVES>
__global__ __launch_bounds__(128) __attribute__((amdgpu_waves_per_eu(1, 1))) void prefix_kernel(DecodeArgs a)
{
    __shared__ Stage<D, LINE> sg0, sg1, sg2, sg3;
    __shared__ int bad_rows;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = blockIdx.x, row0 = blockIdx.y * kPrefixRows, part = blockIdx.z;
    const int begin = part * a.p_chunk, count = min(a.p_chunk, a.prefix_len - begin), tiles = (count + KS - 1) / KS;
    const int rows = a.n_seq * a.q_len * a.r;

    int held = -1;
    bool bad = false;
    if (lane < (count + 15) / 16) {
        held = a.prefix[(begin + 16 * lane) >> a.page_log];
        if (held >= a.pages) held = -1;
        bad = held < 0;
    }
    // row / r: the workgroup's first row by a division, its 128 rows by 1 / r, at least 1 / 2 r off the next whole number
    const int t0 = row0 / a.r, rest = row0 - t0 * a.r;
    const float inv_r = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, 1.0f / (float)a.r)));
    auto token_of = [&](int row) { return t0 + (int)(((float)(row - row0 + rest) + 0.5f) * inv_r); };
    bf16x8 q[2][D / 16];
    const int sees[2] = {count, count};
    auto load_queries = [&]() {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const int row = min(row0 + wave * 64 + 32 * nt + n, rows - 1), t = token_of(row);
            const bf16_t *src = a.Q + row_offset(t, kv * a.r + row - t * a.r, a.q) + 8 * h;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) q[nt][x] = *reinterpret_cast<const bf16x8 *>(src + 16 * x);
        }
    };
    auto source = [&]() {
        if constexpr (LINE) {
            Rows<D, true> s;
            const int64_t first = (int64_t)kv * a.p_room + begin;
            s.size = count * D * 2;
            s.tiles = tiles;
            s.tile_bytes = KS * D * 2;
            s.factors_size = min(a.p_chunk, a.p_room - begin) * 4;
            s.rows = __builtin_amdgcn_make_buffer_rsrc((wave == 0 ? a.line_k : a.line_v) + first * D, 0, s.size, 0x00020000);
            s.factors = __builtin_amdgcn_make_buffer_rsrc((wave == 0 ? a.line_kf : a.line_vf) + first, 0, s.factors_size, 0x00020000);
            return s;
        } else {
            return Pages<D, HALVES>{reinterpret_cast<const bf16_t *>(wave == 0 ? a.K : a.V), held, count, begin, a.page_log, kv, a.h_kv};
        }
    };
    unsigned char *const room = reinterpret_cast<unsigned char *>(wave == 0 ? &sg0 : &sg1);
    auto store = [&](const State<D> &st) {                 // true where the result does not stand
        bool bad = false;
        int lane_here = lane;
        asm volatile("" : "+v"(lane_here));                // as in rows_out
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const int first = row0 + wave * 64 + 32 * nt, row = first + (lane_here & 31);
            const float l = st.l[nt] + __shfl_xor(st.l[nt], 32, 64);
            auto out_of = [&](int y) {
                const int t = token_of(y);
                return (int64_t)t * a.h_q + kv * a.r + y - t * a.r;
            };
            const int64_t parts = (int64_t)part * a.n_seq * a.q_len * a.h_q;
            const float zero = rows_out<D, float>(st, nt, room, lane, [&](floatx4 v) { return v; },
                                                  [&](int x, int piece, uintx4 v) {
                                                      if (first + x < rows)
                                                          *reinterpret_cast<uintx4 *>(a.part_o + (parts + out_of(first + x)) * D + 4 * piece) = v;
                                                  });
            if (row < rows && h == 0) {
                const int64_t at = parts + out_of(row);
                a.part_ml[2 * at] = st.m[nt];
                a.part_ml[2 * at + 1] = l;
            }
            bad = bad || __builtin_fmaf(l, 0.0f, zero) != 0.0f || l == 0.0f;
        }
        return bad;
    };
    const auto src = source();
    const Offsets<D> off = offsets<D>(wave, lane, D * 2);
    const unsigned long long missing = __ballot(bad);      // sixteens of keys in no page
    if (threadIdx.x == 0) bad_rows = 0;
    {
        State<D> st;
        clear(st);
        all_tiles<D, LINE>(st, q, load_queries, sees, count, tiles, a.c2, src, off, sg0, sg1, sg2, sg3, wave, lane);
        bad = store(st) || missing != 0;                   // (nobody waits for the stores)
    }
    __syncthreads();
    if (__any(bad) && lane == 0) bad_rows = 1;
    __syncthreads();
    if (__builtin_expect(bad_rows != 0, 0)) {
        State<D> st;
        clear(st);
        load_queries();
        for (int t = 0; t < tiles; ++t) {
            __syncthreads();
            issue_tile(sg0, src, off, t, wave);
            issue_factors(sg0, src, t, wave, lane);
            meet();
            whole_tile<D, LINE>(st, sg0, off, q, sees, t * KS, (int)(~missing >> (2 * t)) & 3, a.c2, h);
        }
        __syncthreads();
        store(st);
    }
}

// The prefix's 8-bit values as bf16, eight to a thread, and their factors; rows behind the prefix and in no page: zeros, 1.
template <int DTYPE, int D>
__global__ __launch_bounds__(256) void line_kernel(DecodeArgs a)
{
    constexpr int L = D / 8;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(at / L), x = (int)at % L, h = blockIdx.y;
    if (row >= a.p_room) return;
    int page = -1;
    if (row < a.prefix_len) page = a.prefix[row >> a.page_log];
    const bool there = page >= 0 && page < a.pages;
    const int64_t from = (((int64_t)(there ? page : 0) * a.h_kv + h) << a.page_log) + (row & ((1 << a.page_log) - 1));
    const int64_t to = (int64_t)h * a.p_room + row;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        uint2 w = make_uint2(0, 0);
        if (there) w = *reinterpret_cast<const uint2 *>((v ? a.V : a.K) + from * D + 8 * x);
        const uintx2 lo = widen4<DTYPE>(w.x), hi = widen4<DTYPE>(w.y);
        *reinterpret_cast<uintx4 *>((v ? a.line_v : a.line_k) + to * D + 8 * x) = uintx4{lo[0], lo[1], hi[0], hi[1]};
        if (x == 0) (v ? a.line_vf : a.line_kf)[to] = there ? (v ? a.vf : a.kf)[from] : 1.0f;
    }
}

}  // namespace prompt

pbs_status launch_prefix(const DecodeArgs &a, int dtype, int d, hipStream_t s)
{
    using namespace prompt;
    const dim3 grid(a.h_kv, a.p_row_tiles, a.p_parts), block(128);
    if (dtype == PBS_BF16) {
        auto kernel = d == 128 ? (a.page_log == 4 ? prefix_kernel<128, false, true> : prefix_kernel<128, false, false>)
                               : (a.page_log == 4 ? prefix_kernel<64, false, true> : prefix_kernel<64, false, false>);
        return launch(kernel, grid, block, 0, s, a);
    }
    auto line = d == 128 ? (dtype == PBS_E4M3 ? line_kernel<PBS_E4M3, 128> : line_kernel<PBS_I8, 128>)
                         : (dtype == PBS_E4M3 ? line_kernel<PBS_E4M3, 64> : line_kernel<PBS_I8, 64>);
    const pbs_status st = launch(line, dim3((unsigned)(((int64_t)a.p_room * (d / 8) + 255) / 256), a.h_kv), dim3(256), 0, s, a);
    if (st != PBS_OK) return st;
    return launch(d == 128 ? prefix_kernel<128, true, false> : prefix_kernel<64, true, false>, grid, block, 0, s, a);
}

}  // namespace pbs
