// pbs_decode_attn_rule: attention of new tokens over a paged cache under a score rule, and what every key receives of it.
//
// The walk over the keys is that of pbs_decode_attn (decode_walk.h); the rule changes the logits between the two products: a lane
// holds eight keys of one query, so that the cap, the bias by distance and the window are arithmetic within it.  With a window the
// tiles between the sinks and the band that some query sees are not listed, and the shares are cut from the listed ones.  Where rows have
// positions (an eviction has moved them) every tile is listed, and the positions come with the tile.
//
// Weights: what a key receives, the sum of exp(logit - lse) over the rows of its kv head, needs the lse, which is there when the last
// key has been seen.  Reading the keys again would cost half of the attention's bytes: the logits, 4 bytes to a row where a key and its
// value have 128 to 512, go to the workspace instead, and weigh_keys sums them up beside the join of the pieces.  Measured, replayed: 8
// sequences of 131072 keys in bf16, 32 / 8 heads, a bias, 728 us without weights and 943 with them (134 MB of logits out and in again: the
// walk takes 170 us more, of which their bytes are 75, and weigh_keys 38); the same keys' walk alone 6.0 TB/s.
#include "decode_join.h"
#include "decode_rule.h"

namespace pbs {

constexpr int kWeighEach = 2, kWeighKeys = 4 * kDecThreads * kWeighEach, kWeighRows = 64;

// lse in log2 units of row `row` of a sequence's q_len r rows of kv head h; by 16 lanes.  Where the unit is in pieces its own join may not
// have come yet.
__device__ __forceinline__ float joined_lse(const RuleArgs &a, int i, int h, int row, int rows_of_unit)
{
    const int tile = row / rows_of_unit, x = threadIdx.x & 15;
    const int64_t unit = (int64_t)i * a.units + (int64_t)tile * a.h_kv + h;
    const int2 own = a.shares > 0 ? a.pieces[unit] : make_int2(0, 1);
    if (own.y == 1) {
        const int t = row / a.r;
        return a.lse[((int64_t)i * a.q_len + t) * a.h_q + h * a.r + row - t * a.r] * kLog2e;
    }
    const float *ml = a.piece_ml + 2 * ((own.x + unit) * a.slot_rows + row - tile * rows_of_unit);
    float m = -INFINITY, l = 0.0f;
    for (int p = x; p < own.y; p += 16) {
        const floatx2 v = *reinterpret_cast<const floatx2 *>(ml + 2 * (int64_t)p * a.slot_rows);
        const float top = fmaxf(m, v[0]);
        l = (l == 0.0f ? 0.0f : l * __builtin_amdgcn_exp2f(m - top)) + (v[1] == 0.0f ? 0.0f : v[1] * __builtin_amdgcn_exp2f(v[0] - top));
        m = top;
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
        const float m2 = __shfl_xor(m, o, 64), l2 = __shfl_xor(l, o, 64), top = fmaxf(m, m2);
        l = (l == 0.0f ? 0.0f : l * __builtin_amdgcn_exp2f(m - top)) + (l2 == 0.0f ? 0.0f : l2 * __builtin_amdgcn_exp2f(m2 - top));
        m = top;
    }
    return l == 0.0f ? -INFINITY : m + __builtin_amdgcn_logf(l);
}

// Adds to the weights of 2048 listed keys of a (sequence, kv head).  A row without a finite lse (it sees no key, or it has met
// values that are not finite) gives nothing: it would leave NaN in the weights for good.
__device__ __forceinline__ void weigh_keys(const RuleArgs &a, int rows_of_unit, int chunks, unsigned block)
{
    __shared__ float lse[kWeighRows];
    const int64_t unit = block / (unsigned)chunks;
    const int mine = (block - (unsigned)unit * chunks) * kWeighKeys + 4 * threadIdx.x;
    const int i = (int)(unit / a.h_kv), h = (int)(unit - (int64_t)i * a.h_kv), rows = a.q_len * a.r;
    const int len = own_len(a, i), listed = tiles_of_len(a, len) * kTileKeys;
    if (mine - 4 * (int)threadIdx.x >= listed) return;
    floatx4 sum[kWeighEach], v[4][kWeighEach];
    int first[kWeighEach];
    const float *y[kWeighEach];
#pragma unroll
    for (int g = 0; g < kWeighEach; ++g) {
        first[g] = min(mine + 4 * kDecThreads * g, listed - 4);
        sum[g] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        y[g] = a.logits + (unit * a.logit_tiles + first[g] / kTileKeys) * rows * kTileKeys + first[g] % kTileKeys;
    }
    bool live[kWeighEach] = {true, true};
    auto load = [&](int row) __attribute__((always_inline)) {   // four rows at a time, the first ones while the lse are formed
        if (a.live && row % rows_of_unit == 0) {           // (four rows are of one tile of rows)
            const uint8_t *of = a.live + ((int64_t)i * a.units + row / rows_of_unit * a.h_kv + h) * a.logit_tiles;
#pragma unroll
            for (int g = 0; g < kWeighEach; ++g) live[g] = of[first[g] / kTileKeys] != 0;
        }
#pragma unroll
        for (int g = 0; g < kWeighEach; ++g) {
            if (!live[g]) {
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x][g] = floatx4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                continue;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x][g] = *reinterpret_cast<const floatx4 *>(y[g] + min(row + x, rows - 1) * kTileKeys);
        }
    };
    load(0);
    for (int base = 0; base < rows; base += kWeighRows) {
        const int n = min(rows - base, kWeighRows);
        if (base > 0) __syncthreads();
        for (int x = threadIdx.x >> 4; x < n; x += kDecThreads / 16) {
            const float of_row = joined_lse(a, i, h, base + x, rows_of_unit);
            if ((threadIdx.x & 15) == 0) lse[x] = of_row;
        }
        __syncthreads();
        for (int row = 0; row < n; row += 4) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float of_row = lse[min(row + x, n - 1)];
                if (row + x >= n || !(fabsf(of_row) < INFINITY)) continue;
#pragma unroll
                for (int g = 0; g < kWeighEach; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[g][e] += __builtin_amdgcn_exp2f(v[x][g][e] - of_row);
            }
            if (base + row + 4 < rows) load(base + row + 4);
        }
    }
#pragma unroll
    for (int g = 0; g < kWeighEach; ++g) {
        const int key = listed_tiles(a, len).tile(first[g] / kTileKeys) * kTileKeys + first[g] % kTileKeys;
        if (mine + 4 * kDecThreads * g >= listed || key >= len) return;
        const int page = a.table[(int64_t)i * a.max_pages + (key >> a.page_log)];
        if (page < 0 || page >= a.pages) continue;
        float *to = a.weight + ((((int64_t)page * a.h_kv + h) << a.page_log) + (key & ((1 << a.page_log) - 1)));
        if (key + 4 <= len) {
            *reinterpret_cast<floatx4 *>(to) += sum[g];
        } else {
            for (int e = 0; e < len - key; ++e) to[e] += sum[g][e];
        }
    }
}

// The join's workgroups, `joins` of them (none where nothing is joined), and those of the weights: neither waits for the other.
// What is left of a launch between them, graphs of one call: 32 sequences of 200 .. 4097 keys, 3 new tokens, 28 / 4 heads, in int8, 82 -> 75 us; 64 of 7 .. 16000
// keys in e4m3 92 -> 90 (1024 keys to a workgroup, twice as many that form every lse, 94); 8 of 131072 the same.
template <int D, int ROWS>
__global__ __launch_bounds__(kDecThreads) void join_weigh_kernel(RuleArgs a, int rows_of_unit, unsigned joins, int chunks)
{
    const unsigned weighs = gridDim.x - joins;
    if (blockIdx.x < weighs) weigh_keys(a, rows_of_unit, chunks, blockIdx.x);
    else join_rows<D, ROWS>(a, rows_of_unit, blockIdx.x - weighs);
}

inline pbs_status plan_rule(const pbs_decode_problem *p, const pbs_score_rule *r, const pbs_cache *c, const pbs_cache_marks *marks,
                            RulePlan &plan)
{
    if (!p || !r) return PBS_ERR_NULL;
    const bool places = !marks || !marks->position;
    long long most = 1ll << 40;
    if (r->window > 0 && r->sinks >= 0 && places)
        most = 32 * (((long long)r->sinks + 31) / 32 + ((long long)r->window + p->q_len + 30) / 32 + 1);
    pbs_status st = plan_decode(p, c, most, plan);
    if (st != PBS_OK) return st;
    if (p->prefix_len > 0) return PBS_ERR_UNSUPPORTED;
    st = check_rule(r, scale_of(p->scale, c->d));
    if (st != PBS_OK) return st;
    if (marks && (!aligned16(marks->weight) || !aligned16(marks->position))) return PBS_ERR_SHAPE;
    RuleArgs &a = plan.rule;
    static_cast<DecodeArgs &>(a) = plan.a;
    a.cap2 = r->cap * kLog2e;
    if (r->cap > 0.0f) a.c2 = scale_of(p->scale, c->d) / r->cap;
    a.window = r->window;
    a.sinks = r->sinks;
    a.slope = r->slope;
    a.k_pos = places || (a.window == 0 && !a.slope) ? nullptr : marks->position;             // read where something depends on them
    a.weight = marks ? marks->weight : nullptr;
    const long long keys = most > a.max_len ? ((long long)a.max_len + 31) / 32 * 32 : most;
    a.logit_tiles = (int)(keys / kTileKeys);
    a.look = !plan.whole && a.k_pos && a.window > 0 && (long long)a.n_seq * a.units * a.logit_tiles > (long long)kManyTiles * plan.nt * a.shares;
    plan.chunks = a.weight && a.n_seq > 0 ? (keys + kWeighKeys - 1) / kWeighKeys : 0;
    plan.logits = plan.bytes;
    plan.need = plan.bytes;
    if (plan.chunks > 0) {
        const long long grid = plan.chunks * a.n_seq * a.h_kv + plan.join_grid;
        if (grid > 0x7fffffffLL || !fits_grid(grid, kDecThreads)) return PBS_ERR_UNSUPPORTED;
        const size_t rows = (size_t)a.n_seq * a.q_len * a.h_q;
        plan.own_lse = plan.logits + align_up(rows * (size_t)keys * 4, kWsAlign);
        plan.live = plan.own_lse + align_up(rows * 4, kWsAlign);
        plan.need = plan.live + (a.look ? align_up((size_t)a.n_seq * a.units * a.logit_tiles, kWsAlign) : 0);
    }
    return PBS_OK;
}

template <> pbs_status launch_walk<PBS_BF16>(const RulePlan &, int, hipStream_t);
template <> pbs_status launch_walk<PBS_E4M3>(const RulePlan &, int, hipStream_t);
template <> pbs_status launch_walk<PBS_I8>(const RulePlan &, int, hipStream_t);

inline pbs_status launch_rule(const RulePlan &plan, int dtype, int d, hipStream_t s)
{
    if (plan.grid > 0) {
        const pbs_status st = dtype == PBS_BF16 ? launch_walk<PBS_BF16>(plan, d, s)
                              : dtype == PBS_E4M3 ? launch_walk<PBS_E4M3>(plan, d, s) : launch_walk<PBS_I8>(plan, d, s);
        if (st != PBS_OK) return st;
    }
    if (plan.chunks == 0) return plan.join ? launch_join(plan, d, s) : PBS_OK;
    auto kernel = d == 128 ? (plan.join_rows == 1 ? join_weigh_kernel<128, 1> : join_weigh_kernel<128, kDecWaves>)
                           : (plan.join_rows == 1 ? join_weigh_kernel<64, 1> : join_weigh_kernel<64, kDecWaves>);
    const long long joins = plan.join ? plan.join_grid : 0;
    return launch(kernel, dim3((unsigned)(joins + plan.chunks * plan.a.n_seq * plan.a.h_kv)), dim3(kDecThreads), 0, s, plan.rule, 16 * plan.nt,
                  (unsigned)joins, (int)plan.chunks);
}

}  // namespace pbs

extern "C" size_t pbs_decode_rule_workspace_bytes(const pbs_decode_problem *p, const pbs_score_rule *rule, const pbs_cache *c,
                                                  const pbs_cache_marks *marks)
{
    pbs::RulePlan plan;
    return pbs::plan_rule(p, rule, c, marks, plan) == PBS_OK ? plan.need : 0;
}

extern "C" pbs_status pbs_decode_attn_rule(const pbs_decode_problem *p, const pbs_score_rule *rule, const pbs_cache *c,
                                           const pbs_cache_marks *marks, const void *Q, const int32_t *positions,
                                           const int32_t *page_table, const int32_t *lens, void *O, float *lse, void *ws,
                                           size_t ws_bytes, void *stream)
{
    using namespace pbs;
    RulePlan plan;
    pbs_status st = plan_rule(p, rule, c, marks, plan);
    if (st != PBS_OK) return st;
    if (p->n_seq == 0) return PBS_OK;
    if (marks && marks->position && !positions) return PBS_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return PBS_ERR_SHAPE;
    st = take_decode(p, c, Q, page_table, lens, nullptr, O, lse, ws, ws_bytes, plan.need, plan);
    if (st != PBS_OK) return st;
    RuleArgs &a = plan.rule;
    const float c2 = a.c2;
    uint8_t *room = static_cast<uint8_t *>(ws);
    if (plan.chunks > 0 && !lse) plan.a.lse = reinterpret_cast<float *>(room + plan.own_lse);
    static_cast<DecodeArgs &>(a) = plan.a;
    a.c2 = c2;
    a.q_pos = positions;
    a.logits = plan.chunks > 0 ? reinterpret_cast<float *>(room + plan.logits) : nullptr;
    a.live = plan.chunks > 0 && a.look ? room + plan.live : nullptr;
    return launch_rule(plan, c->dtype, c->d, static_cast<hipStream_t>(stream));
}
