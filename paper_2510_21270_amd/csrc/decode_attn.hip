// pbs_decode_attn: attention of each sequence's newest tokens over a paged cache, with a prefix that all sequences share.
//
// The softmax of one pass: a wave keeps, per query, the running maximum m, the sum l and O^T, all fp32.  Everything is
// transposed, so that a lane owns one query and nothing but the maximum crosses lanes:
//     S^T = K Q^T       A = rows of K (keys), B = Q^T, v_mfma_f32_16x16x32_bf16: lane (c, g) gets query c, keys 4g .. 4g + 3
//     O^T += V^T P^T    B = P^T: the probabilities as they lie in the lane after two tiles of 16 keys, A = V^T
// The contraction may run over the keys in any order if both operands agree: a lane's eight probabilities belong to keys
// {4g + i} of both tiles, so it loads these eight rows of V, 8 (d = 64: 4) features of each, and turns the little square with
// byte moves.  Nothing goes through LDS: each wave streams its own keys from memory into registers, a tile of 32 keys ahead
// of the one it multiplies.  8-bit values become bf16 exactly; a key's factor is applied to its logit, a value row's
// to its probability.  A probability enters the product as two terms in bf16 (its rounding alone would be off by 2^-8 of it, as much as O's
// own): the matrix units wait for the keys.  Measured, one term / two: 8 sequences of 131072 keys in bf16 719 / 717 us, 64 of 7 .. 16000
// in e4m3 58.5 / 58.6, in int8 60.0 / 60.5, of 64 features in int8 38.2 / 39.6, 2 of 9000 in int8 with 8 new tokens 28.3 / 29.2.
//
// The bytes of the cache bound it, and a batch's lengths differ by orders of magnitude, known to the device alone.  The tiles of
// all (sequence, kv head) units lie one behind the other in thought, and every wave takes an equal share of that row of
// tiles: the end of one unit, a few whole ones, the start of the next.  A piece of a unit leaves O^T, m and l in the
// workspace and a second launch joins the pieces; a unit that lies in one share whole is stored at once.  The prefix is
// cut into parts of its keys, and its rows are the queries of the whole batch: its keys are read for 16 or 32 rows at a time (or
// 128, prefix_attn.hip).  Measured, 32 query heads on 8 of 128, replayed: 8 sequences of 131072 keys in bf16 717 us (6.0 TB/s), 64 of
// 7 .. 16000 in e4m3 59 us (5.0 TB/s), one of 1000 keys 9.4 us (two launches, latency).
#include <type_traits>

#include "decode.h"

namespace pbs {

constexpr int kDecWaves = 4;
constexpr int kDecThreads = 64 * kDecWaves;
constexpr int kTileKeys = 32;
constexpr int kMostChunk = 4096;                           // keys of a part of the prefix
constexpr int kHeldTiles = 32;                             // tiles whose pages (two each) a wave's lanes hold
constexpr int kUnitCost = 2;                               // tiles, for 16 rows
constexpr int kMostQueries = 16;
constexpr int kFewPieces = 8;                              // of a row that one wave joins

// own keys of sequence i
__device__ __forceinline__ int own_len(const DecodeArgs &a, int i)
{
    const int most = (int)min((int64_t)a.max_len, (int64_t)a.max_pages << a.page_log);
    return min(max(a.lens[i], 0), most);
}

template <int DTYPE, int D>
struct Tile32 {
    static constexpr int ES = DTYPE == PBS_BF16 ? 2 : 1;
    static constexpr int KL = D * ES / 64;                 // 16-byte pieces of a key's row to a lane
    static constexpr int VW = D * ES / 64;                 // 4-byte words of a value row to a lane
    typedef uint32_t vword __attribute__((ext_vector_type(VW)));
    uintx4 k[2][KL];
    vword v[8];
    floatx4 kf[2], vf[2];
    bool ok[2];
};
template <>
struct Tile32<PBS_E4M3, 64> {
    static constexpr int ES = 1, KL = 1, VW = 1;
    struct vword { uint32_t x; __device__ uint32_t operator[](int) const { return x; } };
    uintx4 k[2][1];
    vword v[8];
    floatx4 kf[2], vf[2];
    bool ok[2];
};
template <>
struct Tile32<PBS_I8, 64> : Tile32<PBS_E4M3, 64> {};

// The 16 rows of sub-tile u start at row `first` of the cache's rows (a head's rows of a page are consecutive).
template <int DTYPE, int D>
__device__ __forceinline__ void load_tile(Tile32<DTYPE, D> &t, const DecodeArgs &a, const int (&page)[2], const int (&place)[2],
                                          int h, int c, int g)
{
    typedef Tile32<DTYPE, D> T;
    constexpr int RB = D * T::ES;                          // bytes of a row
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        t.ok[u] = page[u] >= 0;
        const int64_t first = ((((int64_t)max(page[u], 0)) * a.h_kv + h) << a.page_log) + place[u];
        const uint8_t *kr = a.K + (first + c) * RB + 16 * g;
#pragma unroll
        for (int s = 0; s < T::KL; ++s) t.k[u][s] = *reinterpret_cast<const uintx4 *>(kr + 64 * s);
        const uint8_t *vr = a.V + (first + 4 * g) * RB + c * (RB / 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) t.v[4 * u + i] = *reinterpret_cast<const typename T::vword *>(vr + i * RB);
        if constexpr (DTYPE != PBS_BF16) {
            t.kf[u] = *reinterpret_cast<const floatx4 *>(a.kf + first + 4 * g);
            t.vf[u] = *reinterpret_cast<const floatx4 *>(a.vf + first + 4 * g);
        }
    }
}

template <int D, int NT>
struct DecodeState {
    floatx4 o[D / 16][NT];                                 // O^T: lane (c, g), value i of tile j: feature (4g + i) * D/16 + j
    float m[NT], l[NT];                                    // m in log2 units, the same in a query's four lanes; l: this lane's keys
};

// the pair without what is not finite
__device__ __forceinline__ uint32_t finite_part(uint32_t pair)
{
    const uint32_t lo = (pair & 0x7f80u) == 0x7f80u ? 0u : pair & 0xffffu, hi = (pair & 0x7f800000u) == 0x7f800000u ? 0u : pair & 0xffff0000u;
    return lo | hi;
}

// One tile of 32 keys, the first of them key0.  Keys below sees[nt] are visible to the lane's query, keys below `all` to every
// query of the call, keys at or above `none` to no query.  SEVERAL: sees differs between queries; what is not finite in rows
// that some of them see is left out (a hidden row's weight is zero, but 0 * inf is NaN), and `dropped` says so.
// A weight enters the second product as two terms in bf16, itself rounded and what that leaves, 2^-16 of it at most being lost.  ODD: the
// values may not be finite; the rest, which has any sign or is zero, takes the finite ones only.
template <int DTYPE, int D, int NT, bool SEVERAL, bool ODD>
__device__ __forceinline__ void multiply_tile(DecodeState<D, NT> &st, const Tile32<DTYPE, D> &t, const bf16x8 (&q)[D / 32][NT],
                                              const int (&sees)[NT], int key0, int all, int none, float c2, int g, bool &dropped)
{
    constexpr int NJ = D / 16;
    floatx4 s[2][NT];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            bf16x8 ka;
            if constexpr (DTYPE == PBS_BF16) {
                ka = __builtin_bit_cast(bf16x8, t.k[u][x]);
            } else {
                const uintx2 lo = widen4<DTYPE>(t.k[u][x >> 1][2 * (x & 1)]), hi = widen4<DTYPE>(t.k[u][x >> 1][2 * (x & 1) + 1]);
                ka = __builtin_bit_cast(bf16x8, uintx4{lo[0], lo[1], hi[0], hi[1]});
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                s[u][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, q[x][nt], x == 0 ? floatx4{0} : s[u][nt], 0, 0, 0);
        }
    const bool masked = key0 + kTileKeys > all || !t.ok[0] || !t.ok[1];      // uniform
    bf16x8 p[NT], rest[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float y[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = s[e >> 2][nt][e & 3] * (DTYPE == PBS_BF16 ? c2 : t.kf[e >> 2][e & 3] * c2);
            if (masked && !(t.ok[e >> 2] && key0 + 16 * (e >> 2) + 4 * g + (e & 3) < (SEVERAL ? sees[nt] : none))) y[e] = -INFINITY;
            top = fmaxf(top, y[e]);
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m = fmaxf(st.m[nt], top);
        const float ref = m == -INFINITY ? 0.0f : m;       // nothing visible so far: every probability is exp2(-inf) = 0
        const float alpha = __builtin_amdgcn_exp2f(st.m[nt] - ref);
        st.m[nt] = m;
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float w = __builtin_amdgcn_exp2f(y[e] - ref);
            sum += w;
            if constexpr (DTYPE != PBS_BF16) {
                const float f = t.vf[e >> 2][e & 3];
                w = masked && y[e] == -INFINITY ? 0.0f : w * f;   // the factor of a hidden row may be NaN
            }
            p[nt][e] = (bf16_t)w;
            rest[nt][e] = (bf16_t)(w - (float)p[nt][e]);
        }
        st.l[nt] = st.l[nt] * alpha + sum;
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[j][nt][i] *= alpha;
        }
    }

    // rows of V as pairs of bf16: w[e][x] holds features 2x, 2x + 1 of the lane's NJ features of key e
    uint32_t w[8][NJ / 2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (DTYPE == PBS_BF16) {
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x) w[e][x] = t.v[e][x];
        } else {
#pragma unroll
            for (int x = 0; x < NJ / 4; ++x) {
                const uintx2 b = widen4<DTYPE>(t.v[e][x]);
                w[e][2 * x] = b[0];
                w[e][2 * x + 1] = b[1];
            }
        }
        // rows that no query sees may hold anything; their probabilities are zero, and 0 * NaN is not
        if (masked && !(t.ok[e >> 2] && key0 + 16 * (e >> 2) + 4 * g + (e & 3) < none)) {
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x) w[e][x] = 0;
        }
        if (SEVERAL && masked && key0 + 16 * (e >> 2) + 4 * g + (e & 3) >= all) {
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x) {
                const uint32_t f = finite_part(w[e][x]);
                dropped = dropped || f != w[e][x];
                w[e][x] = f;
            }
        }
    }
    auto turned = [&](int j) {                             // feature j of the lane's: its eight keys
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
        return uintx4{__builtin_amdgcn_perm(w[1][j >> 1], w[0][j >> 1], sel), __builtin_amdgcn_perm(w[3][j >> 1], w[2][j >> 1], sel),
                      __builtin_amdgcn_perm(w[5][j >> 1], w[4][j >> 1], sel), __builtin_amdgcn_perm(w[7][j >> 1], w[6][j >> 1], sel)};
    };
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const bf16x8 va = __builtin_bit_cast(bf16x8, turned(j));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            st.o[j][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p[nt], st.o[j][nt], 0, 0, 0);
            if (!ODD) st.o[j][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, rest[nt], st.o[j][nt], 0, 0, 0);
        }
    }
    if constexpr (ODD) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x) w[e][x] = finite_part(w[e][x]);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const bf16x8 va = __builtin_bit_cast(bf16x8, turned(j));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                st.o[j][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, rest[nt], st.o[j][nt], 0, 0, 0);
        }
    }
}

// What a wave does: rows row0 .. row0 + 16 NT - 1 of `rows` (row x: token token0 + x / r, head h * r + x % r) against tiles first,
// first + STEP, ... of keys 0 .. end - 1 of the list `table` (of len keys).
template <int DTYPE, int D, int NT, bool SEVERAL, bool OWN, int STEP>
__device__ __forceinline__ void walk_keys(DecodeState<D, NT> &st, const DecodeArgs &a, const int32_t *table, int len, int first,
                                          int end, int token0, int rows, int row0, int h)
{
    constexpr int NJ = D / 16;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    // lane x holds the page of 16 keys x of this wave's tiles
    const int tiles = ceil_div(end, kTileKeys);
    const int mine = tiles > first ? (tiles - first + STEP - 1) / STEP : 0;
    int held = -1;
    auto hold = [&](int from) __attribute__((always_inline)) {
        const int it = from + (lane >> 1), key = (first + STEP * it) * kTileKeys + 16 * (lane & 1);
        held = -1;
        if (it < mine && key < end) {
            held = table[key >> a.page_log];
            if (held >= a.pages) held = -1;
        }
    };
    auto fetch = [&](Tile32<DTYPE, D> &t, int it) __attribute__((always_inline)) {
        const int key0 = (first + STEP * it) * kTileKeys, at = 2 * (it & (kHeldTiles - 1));
        const int page[2] = {__builtin_amdgcn_readlane(held, at), __builtin_amdgcn_readlane(held, at + 1)};
        const int in_page = (1 << a.page_log) - 1;
        const int place[2] = {key0 & in_page, (key0 + 16) & in_page};
        load_tile<DTYPE, D>(t, a, page, place, h, c, g);
    };
    hold(0);
    bf16x8 q[D / 32][NT];
    int sees[NT];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            st.m[nt] = -INFINITY;
            st.l[nt] = 0.0f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) st.o[j][nt] = floatx4{0};
        }
    };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int rc = min(row0 + 16 * nt + c, rows - 1), t = rc / a.r;
        const bf16_t *src = a.Q + (int64_t)(token0 + t) * a.q.token + (int64_t)(h * a.r + rc - t * a.r) * a.q.head;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
            q[x][nt] = *reinterpret_cast<const bf16x8 *>(src + (DTYPE == PBS_BF16 ? 32 * x + 8 * g : 64 * (x >> 1) + 16 * g + 8 * (x & 1)));
        sees[nt] = OWN ? len - a.q_len + t + 1 : len;
    }
    clear();
    const int all = OWN ? len - a.q_len + 1 : len;

    Tile32<DTYPE, D> ta, tb;
    bool dropped = false;
    auto use = [&](const Tile32<DTYPE, D> &t, int it) __attribute__((always_inline)) {
        multiply_tile<DTYPE, D, NT, SEVERAL, false>(st, t, q, sees, (first + STEP * it) * kTileKeys, all, len, a.c2, g, dropped);
    };
    if (mine > 0) fetch(ta, 0);
    for (int it = 0; it < mine; it += 2) {
        if (it + 1 < mine) fetch(tb, it + 1);
        use(ta, it);
        if (it + 1 < mine) {
            if (it + 2 < mine) {
                if (((it + 2) & (kHeldTiles - 1)) == 0) hold(it + 2);
                fetch(ta, it + 2);
            }
            use(tb, it + 1);
        }
    }
    if constexpr (DTYPE != PBS_I8) {                       // (int8 values are finite)
        // values that are not finite show in O^T: such a wave goes over its keys again
        float zero = 0.0f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) zero = __builtin_fmaf(st.o[j][nt][i], 0.0f, zero);
        if (__builtin_expect(__any(zero != 0.0f), 0)) {
            clear();
            for (int it = 0; it < mine; ++it) {
                if ((it & (kHeldTiles - 1)) == 0) hold(it);
                fetch(ta, it);
                multiply_tile<DTYPE, D, NT, SEVERAL, true>(st, ta, q, sees, (first + STEP * it) * kTileKeys, all, len, a.c2, g, dropped);
            }
        }
    }
    if constexpr (SEVERAL && DTYPE != PBS_I8) {
        // what was left out, for the queries that see it: infinities and NaN come through any weight
        if (__builtin_expect(__any(dropped), 0)) {
            for (int key = max(all, first * kTileKeys); key < end; ++key) {
                if ((key / kTileKeys - first) % STEP != 0) continue;
                const int page = table[key >> a.page_log];
                if (page < 0 || page >= a.pages) continue;
                constexpr int ES = Tile32<DTYPE, D>::ES;
                const uint8_t *row = a.V + (((((int64_t)page * a.h_kv + h) << a.page_log) + (key & ((1 << a.page_log) - 1))) * D) * ES;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const int f = (4 * g + i) * NJ + j;
                        const bool odd = DTYPE == PBS_BF16 ? (reinterpret_cast<const uint16_t *>(row)[f] & 0x7f80) == 0x7f80 : (row[f] & 0x7f) == 0x7f;
                        const float v = DTYPE == PBS_BF16 ? (float)reinterpret_cast<const bf16_t *>(row)[f] : __uint_as_float(0x7fc00000u);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            if (odd && key < sees[nt]) st.o[j][nt][i] += v;
                    }
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        st.l[nt] += __shfl_xor(st.l[nt], 16, 64);
        st.l[nt] += __shfl_xor(st.l[nt], 32, 64);
    }
}

// A sum of zero, not a maximum of -inf, says that a query has met no key: NaN logits have no maximum.
template <int N>
__device__ __forceinline__ void store_output(const DecodeArgs &a, int token, int head, int f, const float (&o)[N], float m, float l)
{
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bf16_t *dst = a.O + (int64_t)token * a.o.token + (int64_t)head * a.o.head + f;
#pragma unroll
    for (int y = 0; y < N; y += 4) {
        const floatx4 v = floatx4{o[y], o[y + 1], o[y + 2], o[y + 3]} * inv;
        *reinterpret_cast<bf16x4 *>(dst + y) = __builtin_convertvector(v, bf16x4);
    }
    if (a.lse && f == 0) a.lse[(int64_t)token * a.h_q + head] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

__device__ __forceinline__ int tiles_of(const DecodeArgs &a, int i) { return ceil_div(own_len(a, i), kTileKeys); }
// What a unit of n tiles counts as: its start and its end cost a wave about as much as kUnitCost tiles.  Measured with 0 / 1 / 2 / 4 / 8:
// 64 sequences of 7 .. 16000 keys in e4m3, 8 kv heads, 77 / 63 / 62 / 63 / 65 us; 100 of 10 .. 600 21.5 / 21.2 / 21.1 / 21.9 / 24.1;
// two tiles of rows to a wave, 16 sequences of 10 .. 5000: 30.5 / 29.2 / 28.9 / 25.7 / 25.7.
template <int NT>
__device__ __forceinline__ int cost_of(int n) { return n > 0 ? n + kUnitCost * NT : 0; }

// of numbers that are not negative; most have 32 bits, whose division takes a third of the instructions
__device__ __forceinline__ int64_t quotient64(int64_t x, int64_t y)
{
    if (((x | y) >> 32) == 0) return (uint32_t)x / (uint32_t)y;
    return x / y;
}

// Sum over the workgroup, and in `before` the sum over the threads in front of this one.
__device__ __forceinline__ int scan_group(int v, int &before, int *sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int other = __shfl_up(sum, o, 64);
        if (lane >= o) sum += other;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    int total = 0;
    before = sum - v;
#pragma unroll
    for (int w = 0; w < kDecWaves; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    return total;
}

// One piece of a unit (sequence i, unit k of it), tiles first .. last - 1, by one wave.  direct: it is the whole unit, and no prefix.
template <int DTYPE, int D, int NT, bool SEVERAL>
__device__ __forceinline__ void own_piece(const DecodeArgs &a, int i, int k, int len, int first, int last, int64_t slot, bool direct)
{
    constexpr int NJ = D / 16;
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int tile = k / a.h_kv, h = k - tile * a.h_kv, rows = a.q_len * a.r, row0 = tile * 16 * NT;
    DecodeState<D, NT> st;
    walk_keys<DTYPE, D, NT, SEVERAL, true, 1>(st, a, a.table + (int64_t)i * a.max_pages, len, first, min(last * kTileKeys, len),
                                              i * a.q_len, rows, row0, h);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int x = 16 * nt + c, row = row0 + x;
        if (row >= rows) continue;
        const int t = row / a.r, head = h * a.r + row - t * a.r;
        const int64_t at = slot * a.slot_rows + x;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            float o[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[j] = st.o[j][nt][y];
            const int f = (4 * g + y) * NJ;
            if (direct) {
                store_output(a, i * a.q_len + t, head, f, o, st.m[nt], st.l[nt]);
            } else {
#pragma unroll
                for (int j = 0; j < NJ; j += 4)
                    *reinterpret_cast<floatx4 *>(a.piece_o + at * D + f + j) = floatx4{o[j], o[j + 1], o[j + 2], o[j + 3]};
            }
        }
        if (!direct && g == 0) {
            a.piece_ml[2 * at] = st.m[nt];
            a.piece_ml[2 * at + 1] = st.l[nt];
        }
    }
}

// WHOLE: a wave to a unit; otherwise an equal share of all tiles to a wave.
template <int DTYPE, int D, int NT, bool SEVERAL, bool WHOLE>
__global__ __launch_bounds__(kDecThreads, NT == 1 ? 2 : 1) void decode_own_kernel(DecodeArgs a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = blockIdx.x * kDecWaves + wave;
    if constexpr (WHOLE) {
        const int i = w / a.units, len = i < a.n_seq ? own_len(a, i) : 0;
        if (i < a.n_seq)
            own_piece<DTYPE, D, NT, SEVERAL>(a, i, w - i * a.units, len, 0, ceil_div(len, kTileKeys), 0, true);
        return;
    }
    int64_t total = 0, share, all, at, front;
    int i, len;
    if (a.n_seq <= 64) {                                   // every wave for itself, a lane to a sequence
        const int lane = threadIdx.x & 63, mine = lane < a.n_seq ? own_len(a, lane) : 0, v = cost_of<NT>(ceil_div(mine, kTileKeys));
        int sum = v;
        for (int o = 1; o < a.n_seq; o <<= 1) {
            const int other = __shfl_up(sum, o, 64);
            if (lane >= o) sum += other;
        }
        total = __builtin_amdgcn_readlane(sum, a.n_seq - 1);
        all = total * a.units;
        share = max(quotient64(all + a.shares - 1, a.shares), (int64_t)1);
        at = w * share;
        if (at >= all) return;
        i = __builtin_ctzll(__ballot(lane < a.n_seq && at < (int64_t)sum * a.units));
        len = __builtin_amdgcn_readlane(mine, i);
        front = (int64_t)__builtin_amdgcn_readlane(sum - v, i) * a.units;
    } else {
        __shared__ int sums[kDecWaves], found[kDecWaves];
        __shared__ int64_t found_front[kDecWaves];
        int before;
        for (int base = 0; base < a.n_seq; base += kDecThreads) {
            const int x = base + threadIdx.x;
            total += scan_group(x < a.n_seq ? cost_of<NT>(tiles_of(a, x)) : 0, before, sums);
        }
        all = total * a.units;
        share = max(quotient64(all + a.shares - 1, a.shares), (int64_t)1);
        // the sequence that each wave's share begins in, and the cost of those in front of it
        front = 0;
        for (int base = 0; base < a.n_seq; base += kDecThreads) {
            const int x = base + threadIdx.x, n = x < a.n_seq ? cost_of<NT>(tiles_of(a, x)) : 0;
            const int sum = scan_group(n, before, sums);
            const int64_t mine = (front + before) * a.units;
#pragma unroll
            for (int y = 0; y < kDecWaves; ++y) {
                const int64_t begin = (int64_t)(blockIdx.x * kDecWaves + y) * share;
                if (mine <= begin && begin < mine + (int64_t)n * a.units) {
                    found[y] = x;
                    found_front[y] = mine;
                }
            }
            front += sum;
        }
        __syncthreads();
        at = w * share;
        if (at >= all) return;
        i = __builtin_amdgcn_readfirstlane(found[wave]);
        len = __builtin_amdgcn_readfirstlane(own_len(a, i));
        front = found_front[wave];
    }
    const int64_t stop = min(at + share, all);
    int n = ceil_div(len, kTileKeys), cost = cost_of<NT>(n);
    const int64_t inside = at - front;                     // of the sequence's units, in tiles
    int k = __builtin_amdgcn_readfirstlane((int)quotient64(inside, cost)), off = __builtin_amdgcn_readfirstlane((int)(inside - (int64_t)k * cost));
    while (true) {
        const int take = (int)min((int64_t)(cost - off), stop - at);
        const int first = max(off - kUnitCost * NT, 0), last = off + take - kUnitCost * NT;             // tiles
        const int64_t unit = (int64_t)i * a.units + k, slot = w + unit;       // one of the two moves on with every piece
        if (last > first) {
            if (first == 0 && (threadIdx.x & 63) == 0)
                a.pieces[unit] = make_int2(w, (int)quotient64(at - off + cost - 1, share) - w + 1);
            own_piece<DTYPE, D, NT, SEVERAL>(a, i, k, len, first, last, slot, first == 0 && last == n && a.p_parts == 0);
        }
        at += take;
        if (at >= stop) break;
        off = 0;
        if (++k == a.units) {
            k = 0;
            do {
                len = own_len(a, ++i);
            } while (len == 0);                            // tiles are left, so there is a sequence with some
            len = __builtin_amdgcn_readfirstlane(len);
            n = ceil_div(len, kTileKeys);
            cost = cost_of<NT>(n);
        }
    }
}

template <int DTYPE, int D, int NT>
__global__ __launch_bounds__(kDecThreads, NT == 1 ? 2 : 1) void decode_prefix_kernel(DecodeArgs a, bool single)
{
    constexpr int NJ = D / 16;
    __shared__ __align__(16) float sum_o[kDecWaves][16][D + 4];
    __shared__ float sum_m[kDecWaves][NT * 16], sum_l[kDecWaves][NT * 16];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x, row0 = blockIdx.y * 16 * NT, part = blockIdx.z;
    const int begin = part * a.p_chunk, rows = a.n_seq * a.q_len * a.r;
    DecodeState<D, NT> st;
    walk_keys<DTYPE, D, NT, false, false, kDecWaves>(st, a, a.prefix, a.prefix_len, begin / kTileKeys + wave,
                                                     min(begin + a.p_chunk, a.prefix_len), 0, rows, row0, h);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
        if (g == 0) {
            sum_m[wave][16 * nt + c] = st.m[nt];
            sum_l[wave][16 * nt + c] = st.l[nt];
        }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecWaves; ++w) m = fmaxf(m, sum_m[w][16 * nt + c]);
        const float ref = m == -INFINITY ? 0.0f : m;
        const float mine_w = __builtin_amdgcn_exp2f(st.m[nt] - ref);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int y = 0; y < NJ / 4; ++y) {
                const floatx4 v = {st.o[4 * y][nt][i], st.o[4 * y + 1][nt][i], st.o[4 * y + 2][nt][i], st.o[4 * y + 3][nt][i]};
                *reinterpret_cast<floatx4 *>(&sum_o[wave][c][(4 * g + i) * NJ + 4 * y]) = st.l[nt] == 0.0f ? floatx4{0} : v * mine_w;
            }
        __syncthreads();
        const int x = tid >> 4, f = (tid & 15) * NJ, row = row0 + 16 * nt + x;
        if (row < rows) {
            float top = -INFINITY, l = 0.0f, o[NJ];
#pragma unroll
            for (int w = 0; w < kDecWaves; ++w) top = fmaxf(top, sum_m[w][16 * nt + x]);
            const float r0 = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int y = 0; y < NJ; ++y) o[y] = 0.0f;
#pragma unroll
            for (int w = 0; w < kDecWaves; ++w) {
                l += sum_l[w][16 * nt + x] * __builtin_amdgcn_exp2f(sum_m[w][16 * nt + x] - r0);
#pragma unroll
                for (int y = 0; y < NJ; ++y) o[y] += sum_o[w][x][f + y];
            }
            const int t = row / a.r, head = h * a.r + row - t * a.r;
            if (single) {
                store_output(a, t, head, f, o, top, l);
            } else {
                const int64_t at = (int64_t)part * a.n_seq * a.q_len * a.h_q + (int64_t)t * a.h_q + head;
#pragma unroll
                for (int y = 0; y < NJ; y += 4)
                    *reinterpret_cast<floatx4 *>(a.part_o + at * D + f + y) = floatx4{o[y], o[y + 1], o[y + 2], o[y + 3]};
                if (f == 0) {
                    a.part_ml[2 * at] = top;
                    a.part_ml[2 * at + 1] = l;
                }
            }
        }
        __syncthreads();
    }
}

// What lies of a row in the workspace: the prefix's parts, the pieces of its unit's own keys.
struct JoinRow {
    int64_t row, all_rows, slot;
    int token, head, parts, all, in_unit;
    bool done;                                             // stored where it was computed
};
__device__ __forceinline__ JoinRow join_row(const DecodeArgs &a, int64_t row, int rows_of_unit)
{
    JoinRow j;
    j.row = row;
    j.all_rows = (int64_t)a.n_seq * a.q_len * a.h_q;
    j.token = (int)((uint32_t)row / (uint32_t)a.h_q);      // fewer than 2^31 rows
    j.head = (int)row - j.token * a.h_q;
    const int i = j.token / a.q_len, h = j.head / a.r, in_seq = (j.token - i * a.q_len) * a.r + j.head - h * a.r;
    const int tile = in_seq / rows_of_unit;
    const int64_t unit = (int64_t)i * a.units + tile * a.h_kv + h;
    int2 own = make_int2(0, 0);
    if (a.shares > 0) own = a.pieces[unit];                // undefined where there are no keys
    if (a.shares > 0 && own_len(a, i) == 0) own = make_int2(0, 0);
    j.slot = own.x + unit;
    j.parts = a.p_parts;
    j.all = a.p_parts + own.y;
    j.in_unit = in_seq - tile * rows_of_unit;
    j.done = a.p_parts == 0 && own.y == 1;
    return j;
}
__device__ __forceinline__ int64_t place_of(const DecodeArgs &a, const JoinRow &j, int p)
{
    return p < j.parts ? p * j.all_rows + j.row : (j.slot + p - j.parts) * a.slot_rows + j.in_unit;
}
// m, l and features 4 x .. 4 x + 3 of every STEP-th piece from `first` on: four at a time, maxima and sums read together
template <int D, int STEP>
__device__ __forceinline__ void add_pieces(const DecodeArgs &a, const JoinRow &j, int first, int x, float &m, float &l, floatx4 &o)
{
    m = -INFINITY;
    l = 0.0f;
    o = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = first; p < j.all; p += 4 * STEP) {
        floatx2 ml[4];
        floatx4 po[4];
        float top = m;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int q = min(p + y * STEP, j.all - 1);
            const int64_t at = place_of(a, j, q);
            ml[y] = *reinterpret_cast<const floatx2 *>((q < j.parts ? a.part_ml : a.piece_ml) + 2 * at);
            po[y] = *reinterpret_cast<const floatx4 *>((q < j.parts ? a.part_o : a.piece_o) + at * D + 4 * x);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if (p + y * STEP >= j.all) ml[y] = floatx2{-INFINITY, 0.0f};
            top = fmaxf(top, ml[y][0]);
        }
        const float keep = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        l *= keep;
        o *= keep;
        m = top;
#pragma unroll
        for (int y = 0; y < 4; ++y)
            if (ml[y][1] != 0.0f) {                        // (NaN sums go through)
                const float f = __builtin_amdgcn_exp2f(ml[y][0] - m);
                l += ml[y][1] * f;
                o += po[y] * f;
            }
    }
}
// two of these, into the first; nothing is a sum of zero
__device__ __forceinline__ void add_sums(float &m, float &l, floatx4 &o, float m2, float l2, floatx4 o2)
{
    const float top = fmaxf(m, m2);
    const float f = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m - top), f2 = l2 == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m2 - top);
    l = l * f + l2 * f2;
    o = o * f + o2 * f2;
    m = top;
}

// Joins parts and pieces: ROWS rows to a workgroup, D / 4 threads to a piece.  With four rows a wave joins one by itself, unless one
// of the four has more than kFewPieces; those four, and a single row, are taken by the whole workgroup one after the other.
// Four rows are for many units, which have two or three pieces each: 300 sequences of 10 .. 256 keys, 8 kv heads, 38 -> 32 us;
// 1000 of 10 .. 1000 230 -> 211 us.  With 26 pieces to each of 1344 rows they are slower (39 -> 56 us).  rows_of_unit: 16 NT.
template <int D, int ROWS>
__global__ __launch_bounds__(kDecThreads) void decode_join_kernel(DecodeArgs a, int rows_of_unit)
{
    constexpr int L = D / 4, G = kDecThreads / L;
    __shared__ __align__(16) float so[G][D];
    __shared__ float sl[G], sm[G];
    __shared__ int many;
    const int64_t all_rows = (int64_t)a.n_seq * a.q_len * a.h_q;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (ROWS == kDecWaves) {
        if (threadIdx.x == 0) many = 0;
        __syncthreads();
        const int64_t row = (int64_t)blockIdx.x * ROWS + wave;
        JoinRow j = join_row(a, min(row, all_rows - 1), rows_of_unit);
        if (row >= all_rows) j.done = true;
        if (!j.done && j.all > kFewPieces && lane == 0) many = 1;
        __syncthreads();
        if (many == 0) {
            if (j.done) return;
            float m, l;
            floatx4 o;
            add_pieces<D, 64 / L>(a, j, lane / L, lane % L, m, l, o);
#pragma unroll
            for (int x = L; x < 64; x <<= 1) {
                const float m2 = __shfl_xor(m, x, 64), l2 = __shfl_xor(l, x, 64);
                floatx4 o2;
#pragma unroll
                for (int y = 0; y < 4; ++y) o2[y] = __shfl_xor(o[y], x, 64);
                add_sums(m, l, o, m2, l2, o2);
            }
            const float out[4] = {o[0], o[1], o[2], o[3]};
            if (lane < L) store_output(a, j.token, j.head, 4 * lane, out, m, l);
            return;
        }
    }
    for (int y = 0; y < ROWS; ++y) {
        const int64_t row = (int64_t)blockIdx.x * ROWS + y;
        if (row >= all_rows) return;
        const JoinRow j = join_row(a, row, rows_of_unit);
        if (j.done) continue;
        float m, l;
        floatx4 o;
        const int group = threadIdx.x / L, x = threadIdx.x % L;
        add_pieces<D, G>(a, j, group, x, m, l, o);
        *reinterpret_cast<floatx4 *>(&so[group][4 * x]) = o;
        if (x == 0) {
            sl[group] = l;
            sm[group] = m;
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int w = 1; w < G; ++w) add_sums(m, l, o, sm[w], sl[w], *reinterpret_cast<const floatx4 *>(&so[w][4 * x]));
            const float out[4] = {o[0], o[1], o[2], o[3]};
            store_output(a, j.token, j.head, 4 * x, out, m, l);
        }
        if constexpr (ROWS > 1) __syncthreads();
    }
}

// Keys of a part of the prefix, for decode_prefix_kernel: one workgroup to a compute unit, or as few rounds of them as parts of
// kMostChunk keys allow, and no more than 64 parts for fewer rounds' sake: the join reads them all.  Measured, whole call, d = 128,
// 8 kv heads: 128 / 256 / 512 workgroups take 33 / 28 / 33 us for 64 rows of 8000 keys in bf16 and 76 / 50 / 56 us for 32000 in
// e4m3; 2 kv heads, 16 rows, 32000 keys: 64 parts 25 us, 128 parts 29 us.
inline int part_keys(int64_t units, int64_t keys)
{
    if (units < 1 || keys < 1) return kMostChunk;
    const int64_t least = (keys + kMostChunk - 1) / kMostChunk, rounds = (least * units + 255) / 256;
    int64_t parts = rounds * 256 / units;
    if (parts > 64) parts = 64;
    if (parts < least) parts = least;
    const int64_t chunk = ((keys + parts - 1) / parts + 127) / 128 * 128;
    return chunk > kMostChunk ? kMostChunk : chunk < 128 ? 128 : (int)chunk;
}

// Whether decode_prefix_kernel, 16 or 32 rows to a workgroup, reads the prefix, or, from more rows on, the kernel of
// prefix_attn.hip, 128 rows to a workgroup.  The latter multiplies faster but starts and ends slower, and it wants 8-bit values
// written out as bf16, which costs as much as four passes of the former over them.  Measured, replayed, us, this kernel / that, 8 kv
// heads: bf16, 8000 keys: 64 rows 26 / 28, 128 rows 34 / 34, 160 rows 40 / 33, 256 rows 51 / 38; 2000 keys, 256 rows 28 / 33;
// 32000 keys, 96 rows 65 / 43.  e4m3: 8000 keys, 128 rows 34 / 44, 256 rows 52 / 48; 32000 keys, 128 rows 81 / 79, 256 rows
// 149 / 94.  Where they are equal it is the former, whose probabilities have two terms.
inline int prefix_tiles(int64_t rows, int h_kv, int64_t keys, int dtype)
{
    if (rows <= 16) return 1;
    const int64_t tiles = (rows + 31) / 32, work = tiles * h_kv * keys;
    if (rows <= 32) return 2;
    return dtype == PBS_BF16 ? (work <= 1 << 18 ? 2 : 0) : (tiles <= 4 || work <= 1 << 19 ? 2 : 0);
}

struct DecodePlan {
    DecodeArgs a;
    int nt, p_nt;
    bool whole, join;
    int join_rows;                                         // of a workgroup of the join
    long long grid, join_grid;                             // workgroups of the own keys (0: there are none), of the join
    size_t bytes;                                          // of the workspace, and where in it:
    size_t part_o, part_ml, piece_o, piece_ml, pieces, line_k, line_v, line_kf, line_vf;
};

inline pbs_status plan_decode(const pbs_decode_problem *p, const pbs_cache *c, DecodePlan &plan)
{
    if (!p) return PBS_ERR_NULL;
    const pbs_status st = check_cache(c);
    if (st != PBS_OK) return st;
    if (p->n_seq < 0 || p->q_len < 1 || p->h_q < 1 || p->h_q % c->h_kv != 0 || p->max_pages < 0 || p->max_len < 0 ||
        p->prefix_len < 0)
        return PBS_ERR_SHAPE;
    if (!(p->scale >= 0.0f) || isinf(p->scale)) return PBS_ERR_SHAPE;
    if (p->dtype != PBS_BF16 || p->q_len > kMostQueries) return PBS_ERR_UNSUPPORTED;
    if ((long long)p->n_seq * p->q_len * p->h_q > 0x7fffffffLL || (long long)p->n_seq * p->max_pages > 0x7fffffffLL)
        return PBS_ERR_UNSUPPORTED;
    if (p->max_len > 1 << 27 || p->prefix_len > 1 << 25) return PBS_ERR_UNSUPPORTED;         // sums of tiles and rows of parts are ints
    DecodeArgs &a = plan.a;
    a.n_seq = p->n_seq; a.q_len = p->q_len; a.h_q = p->h_q; a.h_kv = c->h_kv; a.r = p->h_q / c->h_kv;
    a.page_log = log2_of(c->page); a.pages = c->pages; a.max_pages = p->max_pages;
    const long long in_pages = (long long)p->max_pages * c->page;
    a.max_len = p->max_len < in_pages ? p->max_len : (int)in_pages;
    a.prefix_len = p->prefix_len;
    a.c2 = (p->scale > 0.0f ? p->scale : (float)(1.0 / sqrt((double)c->d))) * 1.4426950408889634f;
    a.q = p->q; a.o = p->o;
    const int64_t rows = (int64_t)a.q_len * a.r, p_rows = rows * a.n_seq;
    // Rows of a wave's tile: 32 where there are more than 16, which reads the keys once for both halves, with all of a SIMD's registers.
    // With 16 instead, 16 sequences of 10 .. 5000 keys, 8 new tokens, 32 / 8 heads: bf16 29 -> 34 us, e4m3 30 -> 29; 4 of 4000 .. 9000
    // with 16 new tokens 44 -> 70 us.
    plan.nt = rows <= 16 ? 1 : 2;
    plan.p_nt = prefix_tiles(p_rows, c->h_kv, a.prefix_len, c->dtype);     // 0: the kernel for many rows
    a.row_tiles = (int)((rows + 16 * plan.nt - 1) / (16 * plan.nt));
    a.units = a.h_kv * a.row_tiles;
    a.slot_rows = (int)(rows < 16 * plan.nt ? rows : 16 * plan.nt);
    const int64_t p_tile = plan.p_nt ? 16 * plan.p_nt : kPrefixRows;
    a.p_row_tiles = (int)((p_rows + p_tile - 1) / p_tile);
    if (plan.p_nt) {
        a.p_chunk = part_keys((int64_t)a.h_kv * a.p_row_tiles, a.prefix_len);
    } else {
        // Two workgroups to a compute unit, whole turns of the loop, pages of a part in a wave's lanes.  48 answers, 28 / 4 heads,
        // 32768 keys: 444 workgroups 53 us, 516, a second round for four of them, 65 us.
        const int64_t units = (int64_t)a.h_kv * a.p_row_tiles, parts = units < 512 ? 512 / units : 1;
        a.p_chunk = (int)(((a.prefix_len + parts - 1) / parts + 127) / 128 * 128);
        if (a.p_chunk > 1024) a.p_chunk = 1024;
        if (a.p_chunk < 128) a.p_chunk = 128;
    }
    const int64_t p_parts = ((int64_t)a.prefix_len + a.p_chunk - 1) / a.p_chunk;
    if (p_parts > 65535 || (p_parts > 0 && a.p_row_tiles > 65535)) return PBS_ERR_UNSUPPORTED;
    a.p_parts = (int)p_parts;
    const long long units = (long long)a.n_seq * a.units, tiles = ((long long)a.max_len + kTileKeys - 1) / kTileKeys;
    if (p->n_seq > 65535 || units > 0x7fffffffLL - 4096) return PBS_ERR_UNSUPPORTED;
    // Lengths up to which a unit has a wave to itself and nothing is joined.  Measured, 8 kv heads, d = 128, bf16, cut to shares / whole:
    // 64 sequences of 128 keys 16.6 / 10.2 us; of 250 keys, one 10.5 / 13.3, 300 of them 75 / 57; 1000 of 500 keys 408 / 361, but
    // 300 of 10 .. 500 41 / 44 and 1000 of 10 .. 2000 329 / 346.
    const int whole = units >= 4096 ? 512 : units >= 512 ? 256 : 128;
    plan.whole = a.p_parts == 0 && a.max_len <= whole;
    // what the chip holds at a time: two workgroups to a compute unit, one where they take all registers
    const long long most = units * (tiles + kUnitCost * plan.nt);
    a.shares = (plan.nt == 1 ? 512 : 256) * kDecWaves;
    if (a.shares > most) a.shares = (int)most;
    plan.grid = ((plan.whole ? units : a.max_len > 0 ? a.shares : 0) + kDecWaves - 1) / kDecWaves;
    a.shares = (int)(plan.whole ? 0 : plan.grid * kDecWaves);
    plan.join = !plan.whole && !(plan.grid == 0 && a.p_parts == 1 && plan.p_nt > 0);
    plan.join_rows = a.p_parts > 0 || a.shares > 2 * (int64_t)units ? 1 : kDecWaves;
    plan.join_grid = plan.join ? ((long long)a.n_seq * a.q_len * a.h_q + plan.join_rows - 1) / plan.join_rows : 0;
    if (!fits_grid(plan.grid, kDecThreads) || !fits_grid(plan.join_grid, kDecThreads)) return PBS_ERR_UNSUPPORTED;
    const size_t all = plan.join ? (size_t)a.n_seq * a.q_len * a.h_q * (size_t)a.p_parts : 0;
    const size_t slots = plan.join && plan.grid ? (size_t)(units + a.shares) * a.slot_rows : 0;
    size_t at = 0;
    auto room = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, kWsAlign); return here; };
    plan.part_o = room(all * c->d * 4);
    plan.piece_o = room(slots * c->d * 4);
    plan.part_ml = room(all * 8);
    plan.piece_ml = room(slots * 8);
    plan.pieces = room(slots ? (size_t)units * 8 : 0);
    const bool line = a.p_parts > 0 && plan.p_nt == 0 && c->dtype != PBS_BF16;
    a.p_room = line ? (a.prefix_len + 127) / 128 * 128 : 0;
    const size_t line_rows = (size_t)a.h_kv * a.p_room;
    plan.line_k = room(line_rows * c->d * 2);
    plan.line_v = room(line_rows * c->d * 2);
    plan.line_kf = room(line_rows * 4);
    plan.line_vf = room(line_rows * 4);
    plan.bytes = at;
    return PBS_OK;
}

template <int DTYPE, int D, bool SEVERAL, bool WHOLE>
pbs_status launch_own(const DecodePlan &plan, hipStream_t s)
{
    auto kernel = plan.nt == 1 ? decode_own_kernel<DTYPE, D, 1, SEVERAL, WHOLE> : decode_own_kernel<DTYPE, D, 2, SEVERAL, WHOLE>;
    return launch(kernel, dim3((unsigned)plan.grid), dim3(kDecThreads), 0, s, plan.a);
}

template <int DTYPE, int D>
pbs_status launch_decode(const DecodePlan &plan, hipStream_t s)
{
    const DecodeArgs &a = plan.a;
    pbs_status st = PBS_OK;
    if (a.p_parts > 0 && plan.p_nt == 0) {
        st = launch_prefix(a, DTYPE, D, s);
    } else if (a.p_parts > 0) {
        auto kernel = plan.p_nt == 1 ? decode_prefix_kernel<DTYPE, D, 1> : decode_prefix_kernel<DTYPE, D, 2>;
        st = launch(kernel, dim3(a.h_kv, a.p_row_tiles, a.p_parts), dim3(kDecThreads), 0, s, a, !plan.join);
    }
    if (st == PBS_OK && plan.grid > 0)
        st = a.q_len == 1 ? (plan.whole ? launch_own<DTYPE, D, false, true>(plan, s) : launch_own<DTYPE, D, false, false>(plan, s))
                          : (plan.whole ? launch_own<DTYPE, D, true, true>(plan, s) : launch_own<DTYPE, D, true, false>(plan, s));
    if (st != PBS_OK || !plan.join) return st;
    return launch(plan.join_rows == 1 ? decode_join_kernel<D, 1> : decode_join_kernel<D, kDecWaves>, dim3((unsigned)plan.join_grid),
                  dim3(kDecThreads), 0, s, a, 16 * plan.nt);
}

}  // namespace pbs

extern "C" size_t pbs_decode_workspace_bytes(const pbs_decode_problem *p, const pbs_cache *c)
{
    pbs::DecodePlan plan;
    return pbs::plan_decode(p, c, plan) == PBS_OK ? plan.bytes : 0;
}

extern "C" pbs_status pbs_decode_attn(const pbs_decode_problem *p, const pbs_cache *c, const void *Q,
                                      const int32_t *page_table, const int32_t *lens, const int32_t *prefix_pages, void *O,
                                      float *lse, void *ws, size_t ws_bytes, void *stream)
{
    using namespace pbs;
    DecodePlan plan;
    const pbs_status st = plan_decode(p, c, plan);
    if (st != PBS_OK) return st;
    if (p->n_seq == 0) return PBS_OK;
    if (!Q || !O || !lens || (p->max_pages > 0 && !page_table) || (p->prefix_len > 0 && !prefix_pages)) return PBS_ERR_NULL;
    if (!good_input(Q, p->q, 2) || !good_output(O, p->o, (long long)p->n_seq * p->q_len, p->h_q, c->d, 2)) return PBS_ERR_SHAPE;
    if (((reinterpret_cast<uintptr_t>(page_table) | reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(prefix_pages) |
          reinterpret_cast<uintptr_t>(lse)) & 3u) != 0)
        return PBS_ERR_SHAPE;
    // a wave stores where it has read its own queries; with other strides it would store over another's (an axis of one has no stride)
    if (Q == O && ((p->q.head != p->o.head && p->h_q > 1) || (p->q.token != p->o.token && (long long)p->n_seq * p->q_len > 1))) return PBS_ERR_SHAPE;
    if (plan.bytes > 0) {
        if (!ws) return PBS_ERR_NULL;
        if ((reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)) != 0 || ws_bytes < plan.bytes) return PBS_ERR_WORKSPACE;
    }
    DecodeArgs &a = plan.a;
    a.Q = static_cast<const bf16_t *>(Q);
    a.K = static_cast<const uint8_t *>(c->K);
    a.V = static_cast<const uint8_t *>(c->V);
    a.kf = c->k_scale;
    a.vf = c->v_scale;
    a.table = page_table;
    a.lens = lens;
    a.prefix = prefix_pages;
    a.O = static_cast<bf16_t *>(O);
    a.lse = lse;
    uint8_t *room = static_cast<uint8_t *>(ws);
    a.part_o = reinterpret_cast<float *>(room + plan.part_o);
    a.part_ml = reinterpret_cast<float *>(room + plan.part_ml);
    a.piece_o = reinterpret_cast<float *>(room + plan.piece_o);
    a.piece_ml = reinterpret_cast<float *>(room + plan.piece_ml);
    a.pieces = reinterpret_cast<int2 *>(room + plan.pieces);
    a.line_k = reinterpret_cast<bf16_t *>(room + plan.line_k);
    a.line_v = reinterpret_cast<bf16_t *>(room + plan.line_v);
    a.line_kf = reinterpret_cast<float *>(room + plan.line_kf);
    a.line_vf = reinterpret_cast<float *>(room + plan.line_vf);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->d == 128)
        return c->dtype == PBS_BF16 ? launch_decode<PBS_BF16, 128>(plan, s)
               : c->dtype == PBS_E4M3 ? launch_decode<PBS_E4M3, 128>(plan, s) : launch_decode<PBS_I8, 128>(plan, s);
    return c->dtype == PBS_BF16 ? launch_decode<PBS_BF16, 64>(plan, s)
           : c->dtype == PBS_E4M3 ? launch_decode<PBS_E4M3, 64>(plan, s) : launch_decode<PBS_I8, 64>(plan, s);
}
