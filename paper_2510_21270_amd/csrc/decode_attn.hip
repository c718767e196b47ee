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
// to its probability.
//
// The bytes of the cache bound it.  A call has few queries, so each (sequence, kv head) is cut into parts of the key axis that
// leave O^T, m and l in the workspace, and a second launch joins them.  The prefix is cut in the same way, but its rows are the
// queries of the whole batch: its keys are read once.
#include "pbs_host.h"
#include "serving.h"

namespace pbs {

constexpr int kDecWaves = 4;
constexpr int kDecThreads = 64 * kDecWaves;
constexpr int kTileKeys = 32;
constexpr int kMostChunk = 4096;                           // keys of a part: a wave's pages fit its 64 lanes
constexpr int kMostQueries = 16;

struct DecodeArgs {
    int n_seq, q_len, h_q, h_kv, r;
    int page_log, pages, max_pages, max_len, prefix_len;
    int chunk, parts;                                      // keys of a part (own keys), most parts of a sequence
    int row_tiles;                                         // of a sequence's q_len * r rows
    int p_chunk, p_parts, p_row_tiles;                     // the same of the prefix
    float c2;                                              // scale * log2(e)
    pbs_strides q, o;
    const bf16_t *Q;
    const uint8_t *K, *V;
    const float *kf, *vf;
    const int32_t *table, *lens, *prefix;
    bf16_t *O;
    float *lse, *part_o, *part_ml;
};

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

// V^T with the values that are not finite taken out, and where they were.
__device__ __forceinline__ bool not_finite(uint32_t pair)
{
    return (pair & 0x7f80u) == 0x7f80u || (pair & 0x7f800000u) == 0x7f800000u;
}
// kind 0: finite values, 1: +inf, 2: -inf, 3: NaN; the latter three as ones
__device__ __forceinline__ uint32_t pick_kind(uint32_t pair, int kind)
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

// One tile of 32 keys, the first of them key0.  `sees[nt]`: keys below it are visible to the lane's query; `all`: keys
// below it are visible to every query of the wave, keys at or above `none` to no query.
template <int DTYPE, int D, int NT>
__device__ __forceinline__ void multiply_tile(DecodeState<D, NT> &st, const Tile32<DTYPE, D> &t, const bf16x8 (&q)[D / 32][NT],
                                              const int (&sees)[NT], int key0, int all, int none, float c2, int g)
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
    bf16x8 p[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float y[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = s[e >> 2][nt][e & 3] * (DTYPE == PBS_BF16 ? c2 : t.kf[e >> 2][e & 3] * c2);
            if (masked && !(t.ok[e >> 2] && key0 + 16 * (e >> 2) + 4 * g + (e & 3) < sees[nt])) y[e] = -INFINITY;
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
    }
    auto turned = [&](int j) {                             // feature j of the lane's: its eight keys
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
        return uintx4{__builtin_amdgcn_perm(w[1][j >> 1], w[0][j >> 1], sel), __builtin_amdgcn_perm(w[3][j >> 1], w[2][j >> 1], sel),
                      __builtin_amdgcn_perm(w[5][j >> 1], w[4][j >> 1], sel), __builtin_amdgcn_perm(w[7][j >> 1], w[6][j >> 1], sel)};
    };
    bool odd = false;                                      // some query does not see a row that another does, with inf or NaN
    if (masked && all < none) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int x = 0; x < NJ / 2; ++x) odd = odd || not_finite(w[e][x]);
    }
    if (__any(odd)) {
        // finite values by their probabilities; of the others only which kind a query sees counts
        const bf16_t one = (bf16_t)1.0f, zero = (bf16_t)0.0f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uintx4 v = turned(j);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                bf16x8 seen;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    seen[e] = t.ok[e >> 2] && key0 + 16 * (e >> 2) + 4 * g + (e & 3) < sees[nt] ? one : zero;
#pragma unroll
                for (int kind = 0; kind < 4; ++kind) {
                    uintx4 k;
#pragma unroll
                    for (int x = 0; x < 4; ++x) k[x] = pick_kind(v[x], kind);
                    const bf16x8 ka = __builtin_bit_cast(bf16x8, k);
                    if (kind == 0) {
                        st.o[j][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, p[nt], st.o[j][nt], 0, 0, 0);
                    } else {
                        const floatx4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, seen, floatx4{0}, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (n[i] > 0.0f)
                                st.o[j][nt][i] += kind == 1 ? INFINITY : kind == 2 ? -INFINITY : __uint_as_float(0x7fc00000u);
                    }
                }
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const bf16x8 va = __builtin_bit_cast(bf16x8, turned(j));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            st.o[j][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p[nt], st.o[j][nt], 0, 0, 0);
    }
}

// Rows row0 .. row0 + 16 NT - 1 of `rows` (row x: token token0 + x / r, head h * r + x % r) against keys begin .. end - 1 of the
// list `table` (len keys), left in part `part` of the workspace, or in O where the call has a single part.
template <int DTYPE, int D, int NT>
__device__ __forceinline__ void decode_part(const DecodeArgs &a, const int32_t *table, int len, int begin, int end, bool own,
                                            int token0, int rows, int row0, int h, int part, bool single)
{
    constexpr int NJ = D / 16;
    __shared__ __align__(16) float sum_o[kDecWaves][16][D + 4];
    __shared__ float sum_m[kDecWaves][NT * 16], sum_l[kDecWaves][NT * 16];
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    bf16x8 q[D / 32][NT];
    int sees[NT];
    DecodeState<D, NT> st;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = row0 + 16 * nt + c;
        const bool there = row < rows;
        const int rc = there ? row : rows - 1;
        const int t = rc / a.r;
        const bf16_t *src = a.Q + (int64_t)(token0 + t) * a.q.token + (int64_t)(h * a.r + rc - t * a.r) * a.q.head;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
            q[x][nt] = *reinterpret_cast<const bf16x8 *>(src + (DTYPE == PBS_BF16 ? 32 * x + 8 * g : 64 * (x >> 1) + 16 * g + 8 * (x & 1)));
        sees[nt] = own ? len - a.q_len + t + 1 : len;
        st.m[nt] = -INFINITY;
        st.l[nt] = 0.0f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) st.o[j][nt] = floatx4{0};
    }
    const int all = own ? len - a.q_len + 1 : len;

    // this wave's tiles: wave, wave + 4, ...; lane x holds the page of 16 keys x of them
    const int tiles = ceil_div(end - begin, kTileKeys);
    const int mine = tiles > wave ? (tiles - wave + kDecWaves - 1) / kDecWaves : 0;
    int held = -1;
    {
        const int key = begin + (wave + kDecWaves * (lane >> 1)) * kTileKeys + 16 * (lane & 1);
        if ((lane >> 1) < mine && key < end) {
            held = table[key >> a.page_log];
            if (held >= a.pages) held = -1;
        }
    }
    auto fetch = [&](Tile32<DTYPE, D> &t, int it) {
        const int key0 = begin + (wave + kDecWaves * it) * kTileKeys;
        const int page[2] = {__builtin_amdgcn_readlane(held, 2 * it), __builtin_amdgcn_readlane(held, 2 * it + 1)};
        const int in_page = (1 << a.page_log) - 1;
        const int place[2] = {key0 & in_page, (key0 + 16) & in_page};
        load_tile<DTYPE, D>(t, a, page, place, h, c, g);
    };
    auto use = [&](const Tile32<DTYPE, D> &t, int it) {
        multiply_tile<DTYPE, D, NT>(st, t, q, sees, begin + (wave + kDecWaves * it) * kTileKeys, all, len, a.c2, g);
    };
    Tile32<DTYPE, D> ta, tb;
    if (mine > 0) fetch(ta, 0);
    for (int it = 0; it < mine; it += 2) {
        if (it + 1 < mine) fetch(tb, it + 1);
        use(ta, it);
        if (it + 1 < mine) {
            if (it + 2 < mine) fetch(ta, it + 2);
            use(tb, it + 1);
        }
    }

    // join the four waves; a sum of zero, not a maximum of -inf, says that a query has met no key: NaN logits have no maximum
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        st.l[nt] += __shfl_xor(st.l[nt], 16, 64);
        st.l[nt] += __shfl_xor(st.l[nt], 32, 64);
        if (g == 0) {
            sum_m[wave][16 * nt + c] = st.m[nt];
            sum_l[wave][16 * nt + c] = st.l[nt];
        }
    }
    __syncthreads();
    const int64_t all_rows = (int64_t)a.n_seq * a.q_len * a.h_q;
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
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                bf16_t *dst = a.O + (int64_t)(token0 + t) * a.o.token + (int64_t)head * a.o.head + f;
#pragma unroll
                for (int y = 0; y < NJ; y += 4) {
                    const floatx4 v = floatx4{o[y], o[y + 1], o[y + 2], o[y + 3]} * inv;
                    *reinterpret_cast<bf16x4 *>(dst + y) = __builtin_convertvector(v, bf16x4);
                }
                if (a.lse && (tid & 15) == 0)
                    a.lse[(int64_t)(token0 + t) * a.h_q + head] = l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
            } else {
                const int64_t at = part * all_rows + (int64_t)(token0 + t) * a.h_q + head;
#pragma unroll
                for (int y = 0; y < NJ; y += 4)
                    *reinterpret_cast<floatx4 *>(a.part_o + at * D + f + y) = floatx4{o[y], o[y + 1], o[y + 2], o[y + 3]};
                if ((tid & 15) == 0) {
                    a.part_ml[2 * at] = top;
                    a.part_ml[2 * at + 1] = l;
                }
            }
        }
        __syncthreads();
    }
}

// grid: x = kv head (consecutive workgroups, so that the XCDs share no page of a head), y = part * row tiles, z = sequence
template <int DTYPE, int D, int NT>
__global__ __launch_bounds__(kDecThreads, NT == 4 ? 1 : 2) void decode_own_kernel(DecodeArgs a, bool single)
{
    const int h = blockIdx.x, i = blockIdx.z;
    const int part = blockIdx.y / a.row_tiles, tile = blockIdx.y - part * a.row_tiles;
    const int len = own_len(a, i);
    const int begin = part * a.chunk;
    if (begin >= len && !single) return;                   // the joining launch knows which parts there are
    decode_part<DTYPE, D, NT>(a, a.table + (int64_t)i * a.max_pages, len, min(begin, len), min(begin + a.chunk, len), true,
                              i * a.q_len, a.q_len * a.r, tile * 16 * NT, h, a.p_parts + part, single);
}

template <int DTYPE, int D, int NT>
__global__ __launch_bounds__(kDecThreads, NT == 4 ? 1 : 2) void decode_prefix_kernel(DecodeArgs a, bool single)
{
    const int h = blockIdx.x, tile = blockIdx.y, part = blockIdx.z;
    const int begin = part * a.p_chunk;
    decode_part<DTYPE, D, NT>(a, a.prefix, a.prefix_len, begin, min(begin + a.p_chunk, a.prefix_len), false, 0,
                              a.n_seq * a.q_len * a.r, tile * 16 * NT, h, part, single);
}

// One workgroup of 4 x 32 threads (d = 64: 4 x 16) per row: every quarter takes every fourth part.
template <int D>
__global__ __launch_bounds__(D) void decode_join_kernel(DecodeArgs a)
{
    constexpr int L = D / 4;
    __shared__ __align__(16) float so[4][D];
    __shared__ float sm[4], sl[4];
    const int64_t row = blockIdx.x, all_rows = (int64_t)a.n_seq * a.q_len * a.h_q;
    const int token = (int)(row / a.h_q), head = (int)(row - (int64_t)token * a.h_q);
    const int quarter = threadIdx.x / L, x = threadIdx.x % L;
    const int parts = a.p_parts + ceil_div(own_len(a, token / a.q_len), a.chunk);
    float m = -INFINITY, l = 0.0f;
    floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = quarter; p < parts; p += 4) {
        const int64_t at = p * all_rows + row;
        const float pm = a.part_ml[2 * at], pl = a.part_ml[2 * at + 1];
        const floatx4 po = *reinterpret_cast<const floatx4 *>(a.part_o + at * D + 4 * x);
        if (pl == 0.0f) continue;
        const float top = fmaxf(m, pm);
        const float was = __builtin_amdgcn_exp2f(m - top), now = __builtin_amdgcn_exp2f(pm - top);
        o = o * was + po * now;
        l = l * was + pl * now;
        m = top;
    }
    *reinterpret_cast<floatx4 *>(&so[quarter][4 * x]) = o;
    if (x == 0) { sm[quarter] = m; sl[quarter] = l; }
    __syncthreads();
    if (quarter != 0) return;
    const float top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    l = 0.0f;
    o = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (sl[w] == 0.0f) continue;
        const float f = __builtin_amdgcn_exp2f(sm[w] - top);
        l += sl[w] * f;
        o += *reinterpret_cast<const floatx4 *>(&so[w][4 * x]) * f;
    }
    if (l != 0.0f) o *= 1.0f / l;
    *reinterpret_cast<bf16x4 *>(a.O + (int64_t)token * a.o.token + (int64_t)head * a.o.head + 4 * x) = __builtin_convertvector(o, bf16x4);
    if (a.lse && x == 0) a.lse[row] = l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Tiles of 16 queries to a wave: enough for the rows where few.
inline int tiles_for(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

// Keys of a part: the longest of 128, 256, ... 4096 with which the call has `wanted` workgroups.
inline int part_keys(int64_t units, int64_t keys, int64_t wanted)
{
    int chunk = kMostChunk;
    while (chunk > 128 && units * ((keys + chunk - 1) / chunk) < wanted) chunk >>= 1;
    return chunk;
}

struct DecodePlan {
    DecodeArgs a;
    int nt, p_nt;
    bool single;
    size_t bytes, ml_at;
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
    if (p->n_seq > 65535) return PBS_ERR_UNSUPPORTED;
    DecodeArgs &a = plan.a;
    a.n_seq = p->n_seq; a.q_len = p->q_len; a.h_q = p->h_q; a.h_kv = c->h_kv; a.r = p->h_q / c->h_kv;
    a.page_log = log2_of(c->page); a.pages = c->pages; a.max_pages = p->max_pages;
    a.max_len = (int)fmin((double)p->max_len, (double)p->max_pages * c->page);
    a.prefix_len = p->prefix_len;
    a.c2 = (p->scale > 0.0f ? p->scale : (float)(1.0 / sqrt((double)c->d))) * 1.4426950408889634f;
    a.q = p->q; a.o = p->o;
    const int64_t rows = (int64_t)a.q_len * a.r, p_rows = rows * a.n_seq;
    plan.nt = tiles_for(rows);
    plan.p_nt = tiles_for(p_rows);
    a.row_tiles = (int)((rows + 16 * plan.nt - 1) / (16 * plan.nt));
    a.p_row_tiles = (int)((p_rows + 16 * plan.p_nt - 1) / (16 * plan.p_nt));
    a.chunk = part_keys((int64_t)a.n_seq * a.h_kv * a.row_tiles, a.max_len, 1024);
    const int64_t parts = ((int64_t)a.max_len + a.chunk - 1) / a.chunk;
    a.p_chunk = part_keys((int64_t)a.h_kv * a.p_row_tiles, a.prefix_len, 1024);
    const int64_t p_parts = ((int64_t)a.prefix_len + a.p_chunk - 1) / a.p_chunk;
    if (parts * a.row_tiles > 65535 || p_parts > 65535 || a.p_row_tiles > 65535) return PBS_ERR_UNSUPPORTED;
    a.parts = (int)parts;
    a.p_parts = (int)p_parts;
    plan.single = a.parts + a.p_parts <= 1;
    const size_t all = (size_t)a.n_seq * a.q_len * a.h_q * (size_t)(a.parts + a.p_parts);
    plan.ml_at = align_up(all * c->d * 4, kWsAlign);
    plan.bytes = plan.single ? 0 : plan.ml_at + align_up(all * 8, kWsAlign);
    return PBS_OK;
}

template <int DTYPE, int D>
pbs_status launch_decode(const DecodePlan &plan, hipStream_t s)
{
    const DecodeArgs &a = plan.a;
    if (a.p_parts > 0) {
        auto kernel = plan.p_nt == 1 ? decode_prefix_kernel<DTYPE, D, 1>
                      : plan.p_nt == 2 ? decode_prefix_kernel<DTYPE, D, 2> : decode_prefix_kernel<DTYPE, D, 4>;
        const pbs_status st = launch(kernel, dim3(a.h_kv, a.p_row_tiles, a.p_parts), dim3(kDecThreads), 0, s, a, plan.single);
        if (st != PBS_OK) return st;
    }
    if (a.parts > 0 || plan.single) {
        if (!(plan.single && a.p_parts > 0)) {
            auto kernel = plan.nt == 1 ? decode_own_kernel<DTYPE, D, 1>
                          : plan.nt == 2 ? decode_own_kernel<DTYPE, D, 2> : decode_own_kernel<DTYPE, D, 4>;
            const int parts = a.parts > 0 ? a.parts : 1;
            const pbs_status st = launch(kernel, dim3(a.h_kv, parts * a.row_tiles, a.n_seq), dim3(kDecThreads), 0, s, a, plan.single);
            if (st != PBS_OK) return st;
        }
    }
    if (plan.single) return PBS_OK;
    return launch(decode_join_kernel<D>, dim3((unsigned)((int64_t)a.n_seq * a.q_len * a.h_q)), dim3(D), 0, s, a);
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
    a.part_o = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + plan.ml_at);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c->d == 128)
        return c->dtype == PBS_BF16 ? launch_decode<PBS_BF16, 128>(plan, s)
               : c->dtype == PBS_E4M3 ? launch_decode<PBS_E4M3, 128>(plan, s) : launch_decode<PBS_I8, 128>(plan, s);
    return c->dtype == PBS_BF16 ? launch_decode<PBS_BF16, 64>(plan, s)
           : c->dtype == PBS_E4M3 ? launch_decode<PBS_E4M3, 64>(plan, s) : launch_decode<PBS_I8, 64>(plan, s);
}
