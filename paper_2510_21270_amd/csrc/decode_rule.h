// The kernels of pbs_decode_attn_rule (decode_rule.hip has the reasons); instantiated by type in files of their own, which takes
// a third of the time to build.
#pragma once
#include "decode_walk.h"
#include "score_rule.h"

namespace pbs {

typedef int intx4 __attribute__((ext_vector_type(4)));

template <int DTYPE, int D> struct RuleTile;
template <int NT, int FORM> struct RowRule;

// What a kernel is made for: one new token to a sequence, whose queries all see the same keys, without a window, with and without a cap and
// a bias; the same with a window and whatever else; or anything; each with and without logits that are kept, and those with a window also
// for waves that look at positions first.  The walk leaves few
// registers and is bound by latency where there are few keys: what is not asked for is not there.
enum { kCapped = 1, kBiased = 2, kWindow = 4, kAnything = 8, kKept = 16, kLooks = 32 };

struct RuleArgs : DecodeArgs {                             // c2: scale / cap under a cap
    static constexpr bool kRule = true;
    template <int DTYPE, int D> using Tile = RuleTile<DTYPE, D>;

    float cap2;                                            // cap * log2(e), 0: none
    int window, sinks;
    const float *slope;
    const int32_t *q_pos, *k_pos;                          // k_pos NULL: places in the sequence
    float *weight;
    float *logits;                                         // [sequence, kv head][listed tile][row][32] in log2 units, or NULL
    int logit_tiles;
    bool look;                                             // whether waves look at positions before they bring tiles
    uint8_t *live;                                         // [unit][tile]: whether logits are there; NULL: all are
};

template <int FORM>
struct FormArgs : RuleArgs {
    template <int NT> using Rows = RowRule<NT, FORM>;
};

// With positions a window may hide most tiles, and which ones is not known.  Where a wave may have many (by max_len), those that have
// more than kFewTiles look at the positions of 32 tiles before they bring any, and a wave's tiles lie apart, as those that are seen
// lie together.  Measured, a graph of one call, with weights, one new token, 32 / 8 heads, bf16: 8 sequences of 131072 keys, a window of 4096, 955 -> 97 us
// (with neighbouring tiles to a wave 234), 8 of 16384 (16 tiles to a wave) 151 -> 68, and where the window hides nothing 151 / 151; 32 of 200 ..
// 4097 keys, 3 new tokens, 28 / 4 heads, in int8 (16 tiles, each with two of rows) where every tile has a key that is seen 77 -> 80.
constexpr int kFewTiles = 8, kManyTiles = 12;              // (the latter for 16 rows)

// The newest query's window hides the most: with places the tiles in front of the oldest query's window are seen by nobody.
__device__ __forceinline__ Listed listed_tiles(const RuleArgs &a, int len)
{
    if (a.window == 0) return {0, 0, 0};
    if (a.k_pos) return {0, 0, a.look ? ceil_div(len, kTileKeys) : 0};
    const int oldest = len - a.q_len + 1;                  // its keys; less a window of almost 2^31 it would pass 32 bits
    const int first = oldest > a.window ? (oldest - a.window) / kTileKeys : 0, head = ceil_div(min(a.sinks, len), kTileKeys);
    return {head, max(first - head, 0), 0};
}

// Lanes x and 32 + x hold the position of key x: one register to a tile.  (The compiler has page and place of both halves, which a lane picks
// by its number, in LDS: 12 to 16 KB in every form that may ask for positions.)
template <int DTYPE, int D>
struct RuleTile : Tile32<DTYPE, D> {
    int kp;
    __device__ __forceinline__ void load_position(const RuleArgs &a, const int (&page)[2], const int (&place)[2], int h, int lane)
    {
        if (!a.k_pos) return;
        const int u = lane >> 4 & 1;
        const int64_t first = ((((int64_t)max(u ? page[1] : page[0], 0)) * a.h_kv + h) << a.page_log) + (u ? place[1] : place[0]);
        kp = a.k_pos[first + (lane & 15)];
    }
};

// The rule for the 16 NT rows of a wave's tile: lane (c, g) has rows 16 nt + c.  Positions of keys come from the lanes that hold them
// whenever they are asked for: the walk has no registers left for them.
template <int NT, int FORM>
struct RowRule {
    static constexpr bool kOn = true, kSeveral = (FORM & kAnything) != 0, kAsks = (FORM & (kWindow | kAnything)) != 0, kLook = (FORM & kLooks) != 0;
    const RuleArgs &a;
    int pos[NT], lo, hi;                                   // lo, hi: over all rows
    float slope2[NT];
    float *to;                                             // the first row's logits of the first tile
    int all, last;                                         // rows of a tile's logits; the last one, from the first
    int head;
    int64_t unit;

    __device__ __forceinline__ bool capped() const { return kAsks ? a.cap2 != 0.0f : (FORM & kCapped) != 0; }
    __device__ __forceinline__ bool biased() const { return kAsks ? a.slope != nullptr : (FORM & kBiased) != 0; }
    __device__ __forceinline__ bool windowed() const { return kAsks && a.window > 0; }

    __device__ __forceinline__ RowRule(const RuleArgs &args, int token0, int len, int rows, int row0, int h, int c) : a(args)
    {
        if constexpr ((FORM & kKept) != 0) {
            to = a.logits + ((int64_t)(token0 / a.q_len) * a.h_kv + h) * a.logit_tiles * rows * kTileKeys + row0 * kTileKeys;
            all = rows;
            last = rows - row0 - 1;
        }
        if constexpr (kLook) {
            head = h;
            unit = (int64_t)(token0 / a.q_len) * a.units + row0 / (16 * NT) * a.h_kv + h;
        }
        lo = 0x7fffffff;
        hi = -0x7fffffff - 1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int rc = min(row0 + 16 * nt + c, rows - 1), t = kSeveral ? rc / a.r : 0;
            if (biased()) slope2[nt] = a.slope[h * a.r + rc - t * a.r] * kLog2e;
            if (!kAsks && !biased()) continue;
            pos[nt] = a.k_pos ? a.q_pos[token0 + t] : len - a.q_len + t;
            if constexpr (!kSeveral) pos[nt] = __builtin_amdgcn_readfirstlane(pos[nt]);
            lo = min(lo, pos[nt]);
            hi = max(hi, pos[nt]);
        }
        if constexpr (kSeveral) {
            if (a.window > 0) {
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) {
                    lo = min(lo, __shfl_xor(lo, o, 64));
                    hi = max(hi, __shfl_xor(hi, o, 64));
                }
                lo = __builtin_amdgcn_readfirstlane(lo);
                hi = __builtin_amdgcn_readfirstlane(hi);
            }
        }
    }
    // of the lane's keys 4 g .. 4 g + 3 of both halves of a tile
    __device__ __forceinline__ void positions(int (&kp)[8], int held, int key0) const
    {
        int first = lane_here() >> 4 << 2;
        if (a.k_pos) {
#pragma unroll
            for (int e = 0; e < 8; ++e) kp[e] = __builtin_amdgcn_ds_bpermute(4 * first + 4 * (16 * (e >> 2) + (e & 3)), held);
        } else {
            first += key0;
#pragma unroll
            for (int e = 0; e < 8; ++e) kp[e] = first + 16 * (e >> 2) + (e & 3);
        }
    }
    __device__ __forceinline__ bool near(int kp, int nt) const
    {
        return a.window == 0 || distance(pos[nt], kp) < (uint32_t)a.window || kp < a.sinks;
    }
    __device__ __forceinline__ bool far(int kp) const
    {
        return max(distance(lo, kp), distance(hi, kp)) >= (uint32_t)a.window && kp >= a.sinks;
    }
    // of the tile's keys, a lane to a key; places are asked of its first and last key alone where that says all
    __device__ __forceinline__ uint32_t far_from_some(int held, int key0) const
    {
        if (!a.k_pos) {
            if (max(distance(hi, key0), distance(lo, key0 + kTileKeys - 1)) < (uint32_t)a.window && key0 <= lo) return 0;
            return (uint32_t)__ballot(far(key0 + (lane_here() & 31)));
        }
        return (uint32_t)__ballot(far(held));
    }
    __device__ __forceinline__ void shape(float (&y)[8], const int (&kp)[8], int nt) const
    {
        if (capped()) cap_scores<8>(y, a.cap2);
        if (biased()) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(-slope2[nt], (float)distance(pos[nt], kp[e]), y[e]);
        }
    }
    __device__ __forceinline__ bool looks(int tiles) const { return tiles > kFewTiles; }
    __device__ __forceinline__ bool seen_by_some(int kp) const { return kp < a.sinks || ((int)((uint32_t)lo - (uint32_t)kp) < a.window && (int)((uint32_t)kp - (uint32_t)hi) < a.window); }
    // Bit x: tile first + x has a key that some query may see; held: the group's pages.
    __device__ __forceinline__ uint32_t live_tiles(int held, const Listed &list, int first, int lane) const
    {
        const int half = lane >> 4 & 1, in_page = (1 << a.page_log) - 1;
        uint32_t live = 0;
#pragma unroll 1
        for (int x = 0; x < kHeldTiles; x += 8) {
            int kp[4];
            bool there[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int tile = x + 2 * y + (lane >> 5), page = __builtin_amdgcn_ds_bpermute(4 * (2 * tile + half), held);
                there[y] = page >= 0;
                kp[y] = a.k_pos[((((int64_t)max(page, 0)) * a.h_kv + head) << a.page_log) + ((list.tile(first + tile) * kTileKeys + 16 * half) & in_page) + (lane & 15)];
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const unsigned long long some = __ballot(there[y] && seen_by_some(kp[y]));
                live |= ((uint32_t)some != 0 ? 1u : 0u) << (x + 2 * y) | ((some >> 32) != 0 ? 2u : 0u) << (x + 2 * y);
            }
        }
        return live;
    }
    __device__ __forceinline__ void note(uint32_t live, int first, int tiles) const
    {
        if constexpr ((FORM & kKept) != 0) {
            const int lane = lane_here();
            if (a.live && lane < kHeldTiles && lane < tiles) a.live[unit * a.logit_tiles + first + lane] = live >> lane & 1;
        }
    }
    // Lanes of rows behind the last one store outside the descriptor's range, which is dropped: there is no branch.  (Where one may pass
    // the stores by, the wait for the next tile is a wait for them.)
    __device__ __forceinline__ void keep(const float (&y)[8], int nt, int listed) const
    {
        if constexpr ((FORM & kKept) != 0) {
            const int lane = lane_here();
            const __amdgpu_buffer_rsrc_t tile = __builtin_amdgcn_make_buffer_rsrc(to + (int64_t)listed * all * kTileKeys, 0, (last + 1) * kTileKeys * 4, 0x00020000);
            const int at = (16 * nt + (lane & 15)) * kTileKeys * 4 + 16 * (lane >> 4);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, floatx4{y[0], y[1], y[2], y[3]}), tile, at, 0, 2);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, floatx4{y[4], y[5], y[6], y[7]}), tile, at + 64, 0, 2);
        }
    }
    // whether multiply_tile has left the values of this key (row `at` of the cache) out that are not finite, and the query sees it
    __device__ __forceinline__ bool left_out_but_seen(int key, int64_t at, int all, int nt) const
    {
        const int kp = a.k_pos ? a.k_pos[at] : key;
        return near(kp, nt) && (key >= all || (a.window > 0 && far(kp)));
    }
};

struct RulePlan : DecodePlan {
    RuleArgs rule;
    long long chunks;                                      // of 2048 keys, of a (sequence, kv head); 0: no weights
    size_t logits, own_lse, live, need;
};

template <int DTYPE, int D, int NT, int FORM>
pbs_status launch_form(const RulePlan &plan, hipStream_t s)
{
    FormArgs<FORM> a;
    static_cast<RuleArgs &>(a) = plan.rule;
    constexpr bool several = (FORM & kAnything) != 0;      // queries that see different keys
    auto kernel = decode_own_kernel<DTYPE, D, NT, several, false, FormArgs<FORM>>;
    if constexpr ((FORM & kLooks) == 0)                    // (those that look have many tiles)
        if (plan.whole) kernel = decode_own_kernel<DTYPE, D, NT, several, true, FormArgs<FORM>>;
    return launch(kernel, dim3((unsigned)plan.grid), dim3(kDecThreads), 0, s, a);
}

template <int DTYPE, int D, int KEPT>
pbs_status launch_kept(const RulePlan &plan, hipStream_t s)
{
    const RuleArgs &a = plan.rule;
    if (a.look) {
        if (plan.nt == 2) return launch_form<DTYPE, D, 2, kAnything | kLooks | KEPT>(plan, s);
        return a.q_len > 1 ? launch_form<DTYPE, D, 1, kAnything | kLooks | KEPT>(plan, s) : launch_form<DTYPE, D, 1, kWindow | kLooks | KEPT>(plan, s);
    }
    if (plan.nt == 2) return launch_form<DTYPE, D, 2, kAnything | KEPT>(plan, s);
    if (a.q_len > 1) return launch_form<DTYPE, D, 1, kAnything | KEPT>(plan, s);
    if (a.window > 0) return launch_form<DTYPE, D, 1, kWindow | KEPT>(plan, s);
    if (a.slope) return a.cap2 != 0.0f ? launch_form<DTYPE, D, 1, kCapped | kBiased | KEPT>(plan, s) : launch_form<DTYPE, D, 1, kBiased | KEPT>(plan, s);
    return a.cap2 != 0.0f ? launch_form<DTYPE, D, 1, kCapped | KEPT>(plan, s) : launch_form<DTYPE, D, 1, KEPT>(plan, s);
}

// The walk over the keys of a cache of a type.
template <int DTYPE>
pbs_status launch_walk(const RulePlan &plan, int d, hipStream_t s);
#define PBS_WALK_OF(DTYPE)                                                                                        \
    template <>                                                                                                   \
    pbs_status launch_walk<DTYPE>(const RulePlan &plan, int d, hipStream_t s)                                     \
    {                                                                                                             \
        if (d == 128) return plan.chunks > 0 ? launch_kept<DTYPE, 128, kKept>(plan, s) : launch_kept<DTYPE, 128, 0>(plan, s); \
        return plan.chunks > 0 ? launch_kept<DTYPE, 64, kKept>(plan, s) : launch_kept<DTYPE, 64, 0>(plan, s);     \
    }

}  // namespace pbs
