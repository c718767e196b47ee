// pbs_prompt_attn: causal attention over prompts packed one behind the other, on the pipeline of key_pipeline.h.
//
// The rows of a workgroup are (token, head of the group): all query heads of a kv head share every key tile, 128 rows span few
// tokens, so that little is multiplied above the diagonal and short prompts fill their tiles.  32 heads on 8 of 128: 16384 tokens
// 1.70 ms where calls leave the chip pauses (1.29 PFLOP/s), 1.77 one behind the other (1.24, matrix units 80 % busy), 16 prompts of 33 ..
// 2048 tokens 103 to 110 us (0.74), of which a workgroup's start and end are about 7 of 20 us; 4 prompts of 1 .. 200 tokens 13.2 us.
#include "key_pipeline.h"

namespace pbs {
namespace prompt {

struct Args {
    int n_seq, total_q, total_k, h_q, h_kv, r, tokens;     // tokens: of a workgroup's rows
    float c2, inv_r;                                       // scale * log2(e); 1 / r
    bool causal;
    pbs_strides q, k, v, o;
    const bf16_t *Q, *K, *V;
    const int32_t *cu_q, *cu_k;
    bf16_t *O;
    float *lse;
};

// Which sequence and which of its tiles workgroup `b` has: the sequences' tiles one behind the other, a sequence's last tile, the
// longest, first.  (Tiles with the most keys first over all sequences left no long one for the end, but neighbours no longer
// shared keys in L2: 16 prompts of 33 .. 2048 tokens, 32 / 8 heads, 106 -> 114 us.)  Every wave looks for itself, a lane to a
// sequence.  seq = -1: none is left.
struct Place { int seq, tile, q0, len_q, k0, len_k; };
__device__ __forceinline__ Place find_place(const Args &a, int b, int lane)
{
    Place p = {-1, 0, 0, 0, 0, 0};
    for (int base = 0; base < a.n_seq; base += 64) {
        const int i = base + lane;
        int q0 = 0, len_q = 0, k0 = 0, len_k = 0;
        if (i < a.n_seq) {
            int qa = a.cu_q[i], qb = a.cu_q[i + 1], ka = a.cu_k[i], kb = a.cu_k[i + 1];
            asm volatile("" : "+v"(qa), "+v"(qb), "+v"(ka), "+v"(kb));         // one wait for all four
            q0 = min(max(qa, 0), a.total_q);
            len_q = max(min(max(qb, 0), a.total_q) - q0, 0);
            k0 = min(max(ka, 0), a.total_k);
            len_k = max(min(max(kb, 0), a.total_k) - k0, 0);
        }
        const int tiles = (len_q + a.tokens - 1) / a.tokens;
        int sum = tiles;
        for (int o = 1; o < min(a.n_seq - base, 64); o <<= 1) {
            const int other = __shfl_up(sum, o, 64);
            if (lane >= o) sum += other;
        }
        const unsigned long long has = __ballot(i < a.n_seq && b < sum);
        if (has) {
            const int at = __builtin_ctzll(has);
            p.seq = base + at;
            p.tile = __builtin_amdgcn_readlane(sum, at) - 1 - b;
            p.q0 = __builtin_amdgcn_readlane(q0, at);
            p.len_q = __builtin_amdgcn_readlane(len_q, at);
            p.k0 = __builtin_amdgcn_readlane(k0, at);
            p.len_k = __builtin_amdgcn_readlane(len_k, at);
            return p;
        }
        b -= __builtin_amdgcn_readlane(sum, 63);
    }
    return p;
}

// row / r for the rows of a workgroup: at least 1 / 2 r off the next whole number
__device__ __forceinline__ int token_of(const Args &a, int row) { return (int)(((float)row + 0.5f) * a.inv_r); }

// True where the result does not stand: values that are not finite, or a row that sees keys and has no sum.
template <int D>
__device__ __forceinline__ bool store_rows(const Args &a, const Place &pl, const State<D> &st, const int (&sees)[2], int kv, int t0,
                                           int rows, int wave, int lane, unsigned char *room)
{
    bool bad = false;
    bf16_t *const out = a.O + (int64_t)(pl.q0 + t0) * a.o.token + (int64_t)kv * a.r * a.o.head;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int row0 = wave * 64 + 32 * nt, row = row0 + (lane & 31);
        const float l = st.l[nt] + __shfl_xor(st.l[nt], 32, 64), inv = l == 0.0f ? 0.0f : 1.0f / l;
        // (no sum: O^T is zero as well)
        const float zero = rows_out<D, bf16_t>(st, nt, room, lane, [&](floatx4 v) { return __builtin_convertvector(v * inv, bf16x4); },
                                               [&](int x, int piece, uintx4 v) {
                                                   const int y = row0 + x, in = token_of(a, y);
                                                   if (y < rows)
                                                       *reinterpret_cast<uintx4 *>(out + row_offset(in, y - in * a.r, a.o) + 8 * piece) = v;
                                               });
        bad = bad || __builtin_fmaf(l, 0.0f, zero) != 0.0f || (l == 0.0f && sees[nt] > 0);
        if (a.lse && lane < 32 && row < rows) {
            const int in = token_of(a, row), head = kv * a.r + row - in * a.r;
            a.lse[(int64_t)(pl.q0 + t0 + in) * a.h_q + head] = l == 0.0f ? -INFINITY : (st.m[nt] + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        }
    }
    return bad;
}

template <int D>
__global__ __launch_bounds__(128) __attribute__((amdgpu_waves_per_eu(1, 1))) void prompt_kernel(Args a)
{
    __shared__ Stage<D, false> sg0, sg1, sg2, sg3;         // apart, so that a read of one does not wait for loads into another
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
    clear(st);
    const bf16_t *const first = a.Q + (int64_t)(pl.q0 + t0) * a.q.token + (int64_t)kv * a.r * a.q.head;
    auto load_queries = [&]() {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const int row = wave * 64 + 32 * nt + n, rc = min(row, rows - 1);
            const int in = token_of(a, rc);
            const bf16_t *src = first + row_offset(in, rc - in * a.r, a.q) + 8 * h;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) q[nt][x] = *reinterpret_cast<const bf16x8 *>(src + 16 * x);
        }
    };
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int t = t0 + token_of(a, min(wave * 64 + 32 * nt + n, rows - 1));
        sees[nt] = a.causal ? min(max(t + ahead + 1, 0), pl.len_k) : pl.len_k;
    }
    const int last = a.causal ? min(max(t0 + min(a.tokens, pl.len_q - t0) + ahead, 0), pl.len_k) : pl.len_k;   // keys that any row sees
    const int tiles = (last + KS - 1) / KS;

    const pbs_strides &ks = wave == 0 ? a.k : a.v;
    const bf16_t *base = (wave == 0 ? a.K : a.V) + (int64_t)pl.k0 * ks.token + (int64_t)kv * ks.head;
    const int step_bytes = (int)ks.token * 2;
    const int size = pl.len_k > 0 ? (pl.len_k - 1) * step_bytes + D * 2 : 0;
    Rows<D, false> src;
    src.rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(base), 0, size, 0x00020000);
    src.size = size;
    src.tiles = (pl.len_k + KS - 1) / KS;
    src.tile_bytes = KS * step_bytes;
    const Offsets<D> off = offsets<D>(wave, lane, (uint32_t)step_bytes);
    if (threadIdx.x == 0) bad_rows = 0;
    if (tiles > 0) {
        const int all = __builtin_amdgcn_readfirstlane(sees[0]);               // the wave's first row sees the fewest keys
        all_tiles<D, false>(st, q, load_queries, sees, all, tiles, a.c2, src, off, sg0, sg1, sg2, sg3, wave, lane);
    }
    const bool bad = store_rows<D>(a, pl, st, sees, kv, t0, rows, wave, lane, reinterpret_cast<unsigned char *>(wave == 0 ? &sg0 : &sg1));   // (nobody waits for the stores)
    __syncthreads();
    if (__any(bad) && lane == 0) bad_rows = 1;
    __syncthreads();
    if (__builtin_expect(bad_rows != 0, 0)) {
        clear(st);
        load_queries();
        for (int t = 0; t < tiles; ++t) {
            __syncthreads();
            issue_tile(sg0, src, off, t, wave);
            meet();
            whole_tile<D>(st, sg0, off, q, sees, t * KS, 3, a.c2, h);
        }
        __syncthreads();
        store_rows<D>(a, pl, st, sees, kv, t0, rows, wave, lane, reinterpret_cast<unsigned char *>(wave == 0 ? &sg0 : &sg1));
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
    // byte offsets inside a head's rows have 31 bits
    const long long stride = p->k.token > p->v.token ? p->k.token : p->v.token;
    if (!rows_have_places(p->total_k, prompt::KS, stride * 2, p->d * 2)) return PBS_ERR_UNSUPPORTED;
    const long long grid = ((long long)p->total_q / tokens + p->n_seq) * p->h_kv;
    if (!fits_grid(grid, 128)) return PBS_ERR_UNSUPPORTED;
    if (O == Q || (p->total_k > 0 && (O == K || O == V))) return PBS_ERR_SHAPE;              // rows may be formed a second time

    prompt::Args a;
    a.n_seq = p->n_seq; a.total_q = p->total_q; a.total_k = p->total_k;
    a.h_q = p->h_q; a.h_kv = p->h_kv; a.r = r; a.tokens = tokens;
    a.c2 = (p->scale > 0.0f ? p->scale : (float)(1.0 / sqrt((double)p->d))) * 1.4426950408889634f;
    a.inv_r = 1.0f / r;
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
