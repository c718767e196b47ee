// pbs_cache_evict: every (sequence, kv head) keeps the keys of the largest weights, in its first places.
//
// Which ones stay is one number to a unit, the m-th largest of its keys' 32-bit ranks (protected rows above all, then the
// weights: the bits of floats that are not negative are in their order), and how many of the rows of that very rank do.  It is found
// digit by digit from the top (11, 11 and 10 bits), by counts of the digits in LDS.  Nothing is sorted and hardly anything moves: of the first m
// places those that are not kept are filled, in order, with the kept rows behind them, whatever their order was, because
// rows are marked with their positions.  Sources lie at m and behind, destinations in front: the moves do not touch each other.
//
// Up to 8192 keys a workgroup has a unit, its ranks in registers, and does it in one launch; the moves, as wide loads of whole rows, are
// another.  With more keys workgroups have 8192 of a unit each, and what one needs of the others (the newest position, counts of digits,
// how many stay in front of it) goes through the workspace from launch to launch: seven of them, of a few microseconds each (32768 keys by
// one workgroup, eight quads to a thread, took 65 us instead of 36: the counts in LDS have one compute unit).  Counts are
// integers: their order does not matter.  The selection reads 8 bytes a key and is bound by latency, the moves by the bytes.  Measured, us: 64
// sequences of 1040 keys, 8 kv heads, 16 rows out, selection 12 (15 with sums over a wave by LDS shuffles) and moves 4; 131072 keys in
// bf16, half of them out, selection 31 in six launches, moves 52 (5.1 TB/s).  max_len decides, the lengths being known to the device alone: the
// 64 sequences of 1040 keys, without their marks, take 15 under a bound of 1040, 70 under one of 16384, 208 under 65536.
#include <type_traits>

#include "pbs_host.h"
#include "serving.h"

namespace pbs {

typedef int intx4 __attribute__((ext_vector_type(4)));

constexpr int kBins = 2048;
constexpr int kMostWaves = 16;
constexpr int kHeld = 2;                                   // quads of ranks to a thread
constexpr int kPart = 64 * kMostWaves * 4 * kHeld;         // keys of a workgroup
constexpr int kMoveThreads = 256;
constexpr int kMoveEach = 4;                               // rows to a group of lanes

struct EvictArgs {
    int n_seq, h_kv, page_log, pages, max_pages, max_len, budget, sinks, recent, row_bytes;
    int room;                                              // moves of a unit at most
    int64_t rank_room;
    const int32_t *table, *lens;
    int32_t *new_lens;
    uint8_t *K, *V;
    float *kf, *vf, *weight;
    int32_t *position, *count, *to, *from;
    // of units with several workgroups: ranks, counts of three digits, the digits found and what is left to find, the newest
    // position and the counts of what stays of every workgroup
    int parts;
    uint32_t *ranks, *bins, *found;
    int32_t *newest;
    int4 *stays;
};

__device__ __forceinline__ int evict_len(const EvictArgs &a, int i)
{
    return min(max(a.lens[i], 0), (int)min((int64_t)a.max_len, (int64_t)a.max_pages << a.page_log));
}
// row of a place, or -1
__device__ __forceinline__ int64_t row_at(const EvictArgs &a, int i, int h, int place)
{
    const int page = a.table[(int64_t)i * a.max_pages + (place >> a.page_log)];
    if (page < 0 || page >= a.pages) return -1;
    return (((int64_t)page * a.h_kv + h) << a.page_log) + (place & ((1 << a.page_log) - 1));
}

// One to a bin's count, of every active lane; lanes that agree add once.
__device__ __forceinline__ void count_digit(uint32_t *bins, uint32_t digit)
{
    const unsigned long long all = __ballot(1);
    if (__ballot(digit == (uint32_t)__builtin_amdgcn_readfirstlane((int)digit)) == all) {
        if ((threadIdx.x & 63) == __builtin_ctzll(all)) atomicAdd(&bins[digit], (uint32_t)__builtin_popcountll(all));
    } else {
        atomicAdd(&bins[digit], 1u);
    }
}

// The highest digit from which on upwards `need` keys lie, and how many of the digit's own are among them.  By one wave: its lanes sum up a
// share of the bins each, the highest to lane 0, then the bins of the share that has it.
__device__ __forceinline__ uint32_t sum_upto(uint32_t v)
{
    // sums over the lanes up to each of a row of 16, then the rows in front; every lane of the wave is active
    auto from = [](uint32_t x, auto control, auto rows) __attribute__((always_inline)) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(control)::value, decltype(rows)::value, 0xf, false);
    };
    typedef std::integral_constant<int, 0xf> All;
    v += from(v, std::integral_constant<int, 0x111>(), All());                                   // lane - 1, - 2, - 4, - 8 of the row
    v += from(v, std::integral_constant<int, 0x112>(), All());
    v += from(v, std::integral_constant<int, 0x114>(), All());
    v += from(v, std::integral_constant<int, 0x118>(), All());
    v += from(v, std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());      // the last lane of row 0 to row 1, 2 to 3
    v += from(v, std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());      // lane 31 to rows 2 and 3
    return v;
}
template <int BINS>
__device__ __forceinline__ void find_digit(const uint32_t *bins, uint32_t need, uint32_t *found)
{
    constexpr int kEach = BINS / 64;
    const int lane = threadIdx.x & 63, top = BINS - kEach * (lane + 1);
    uint32_t mine = 0;
#pragma unroll
    for (int x = 0; x < kEach; ++x) mine += bins[top + ((x + lane) & (kEach - 1))];
    const uint32_t upto = sum_upto(mine);
    const int share = __builtin_ctzll(__ballot(upto >= need) | 1ull << 63);
    const uint32_t left = need - (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), share);
    const int first = BINS - kEach * share - 1;            // downwards
    const uint32_t n = lane < kEach ? bins[first - lane] : 0;
    const uint32_t all = sum_upto(n);
    if (all >= left && all - n < left) {
        found[0] = (uint32_t)(first - lane);
        found[1] = left - (all - n);
    }
}

// A workgroup's part of a unit: quad y of thread x is quad part * kHeld * threads + y * threads + x of the unit's places.  Four
// consecutive places lie in one page.
struct Unit {
    int unit, i, h, len, m, first;                         // first: quad of the thread's first one
    __device__ __forceinline__ Unit(const EvictArgs &a, int which, int part)
    {
        unit = which;
        i = unit / a.h_kv;
        h = unit - i * a.h_kv;
        len = evict_len(a, i);
        m = min(len, a.budget);
        first = part * kHeld * blockDim.x + threadIdx.x;
    }
    __device__ __forceinline__ bool moves() const { return len > m && m > 0; }
    __device__ __forceinline__ int place(int y, int e) const { return 4 * (first + y * (int)blockDim.x) + e; }
};

__device__ __forceinline__ void find_rows(int64_t (&row)[kHeld], const EvictArgs &a, const Unit &u)
{
#pragma unroll
    for (int y = 0; y < kHeld; ++y) row[y] = u.place(y, 0) < u.len ? row_at(a, u.i, u.h, u.place(y, 0)) : -1;
}

// largest of a value over the workgroup
__device__ __forceinline__ int group_max(int v, int *of_waves)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
    if ((threadIdx.x & 63) == 0) of_waves[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) v = max(v, of_waves[w]);
    return v;
}

__device__ __forceinline__ int newest_of(const Unit &u, const int64_t (&row)[kHeld], const intx4 (&p)[kHeld])
{
    int newest = -0x7fffffff - 1;
#pragma unroll
    for (int y = 0; y < kHeld; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (row[y] >= 0 && u.place(y, e) < u.len) newest = max(newest, p[y][e]);
    return newest;
}

__device__ __forceinline__ void rank_rows(uintx4 (&r)[kHeld], const EvictArgs &a, const Unit &u, const int64_t (&row)[kHeld],
                                          const floatx4 (&w)[kHeld], const intx4 (&p)[kHeld], int newest)
{
#pragma unroll
    for (int y = 0; y < kHeld; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool safe = p[y][e] < a.sinks || (uint32_t)newest - (uint32_t)p[y][e] < (uint32_t)a.recent;
            r[y][e] = safe ? 0xffffffffu : w[y][e] > 0.0f ? __float_as_uint(w[y][e]) : 0u;
            if (row[y] < 0) r[y][e] = u.place(y, e) < u.m ? 0xffffffffu : 0u;  // of no page: it stays where it is, or goes
        }
}

// Counts the digit of BITS bits at SHIFT of the ranks that begin with `prefix`.
template <int SHIFT, int BITS>
__device__ __forceinline__ void count_digits(uint32_t *bins, const Unit &u, const uintx4 (&r)[kHeld], uint32_t prefix)
{
#pragma unroll
    for (int y = 0; y < kHeld; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (u.place(y, e) < u.len && (SHIFT + BITS == 32 || r[y][e] >> (SHIFT + BITS & 31) == prefix))
                count_digit(bins, r[y][e] >> SHIFT & ((1u << BITS) - 1));
}
__device__ __forceinline__ void clear_bins(uint32_t *bins)
{
    for (int x = threadIdx.x; x < kBins; x += blockDim.x) bins[x] = 0;
}

// What stays of places, in front of place m and behind: those above the last rank, and of that rank itself.
struct Stays { int above, equal, above_behind, equal_behind; };
__device__ __forceinline__ int wave_upto(int v) { return (int)sum_upto((uint32_t)v); }

// Of the thread's quad y, and summed up over the lanes of its wave up to this one.
__device__ __forceinline__ Stays stays_of(const Unit &u, const uintx4 &r, int y, uint32_t last)
{
    Stays n = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int place = u.place(y, e);
        const bool there = place < u.len, front = place < u.m;
        n.above += there && front && r[e] > last;
        n.equal += there && front && r[e] == last;
        n.above_behind += there && !front && r[e] > last;
        n.equal_behind += there && !front && r[e] == last;
    }
    return n;
}
// The sums over the wave, for `counts`, one for each quad and wave.
__device__ __forceinline__ void count_stays(int4 *counts, const Unit &u, const uintx4 (&r)[kHeld], uint32_t last)
{
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
#pragma unroll
    for (int y = 0; y < kHeld; ++y) {
        const Stays n = stays_of(u, r[y], y, last);
        // (256 at most of each: two to a word)
        const uint32_t front = sum_upto((uint32_t)n.above << 16 | n.equal), behind = sum_upto((uint32_t)n.above_behind << 16 | n.equal_behind);
        if ((threadIdx.x & 63) == 63)
            counts[y * waves + wave] = make_int4((int)(front >> 16), (int)(front & 0xffff), (int)(behind >> 16), (int)(behind & 0xffff));
    }
}
// Ties of the last rank, free places and rows to move in front of some place.
struct Before { int ties, holes, sources; };
// In front of piece `upto` (uniform) of what lies behind b: counts_of(x), and places_of(x) in front of place m, of piece x; a lane to a piece.
template <class COUNTS, class PLACES>
__device__ __forceinline__ Before before(Before b, int upto, int need, COUNTS counts_of, PLACES places_of)
{
    for (int base = 0; base < upto; base += 64) {
        const int x = base + (threadIdx.x & 63);
        int4 n = make_int4(0, 0, 0, 0);
        int places = 0;
        if (x < upto) {
            n = counts_of(x);
            places = places_of(x);
        }
        const int equal = n.y + n.w, ties = wave_upto(equal), left = need - b.ties - (ties - equal);      // for this piece
        const int holes = wave_upto(places - n.x - min(max(left, 0), n.y)), sources = wave_upto(n.z + min(max(left - n.y, 0), n.w));
        b.ties += __builtin_amdgcn_readlane(ties, 63);
        b.holes += __builtin_amdgcn_readlane(holes, 63);
        b.sources += __builtin_amdgcn_readlane(sources, 63);
    }
    return b;
}
// Writes the moves of a workgroup's places; counts as count_stays left them, b: before the workgroup's first place.
__device__ __forceinline__ void list_moves(const EvictArgs &a, const Unit &u, const uintx4 (&r)[kHeld], const int4 *counts, uint32_t last,
                                           int need, Before b0)
{
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int base = 4 * (u.first - (int)threadIdx.x);     // the workgroup's first place
    int32_t *const to = a.to + (int64_t)u.unit * a.room, *const from = a.from + (int64_t)u.unit * a.room;
    const int front = min(u.m, u.len);
    auto in_front = [&](int upto) {
        return before(b0, upto, need, [&](int x) { return counts[x]; }, [&](int x) { return min(max(front - (base + 256 * x), 0), 256); });
    };
#pragma unroll 1
    for (int y = 0; y < kHeld; ++y) {
        const Before b = in_front(__builtin_amdgcn_readfirstlane(y * waves + wave));
        uintx4 ry = r[0];
#pragma unroll
        for (int x = 1; x < kHeld; ++x) ry = y == x ? r[x] : ry;
        const Stays n = stays_of(u, ry, y, last);
        int ties = b.ties + wave_upto(n.equal + n.equal_behind) - n.equal - n.equal_behind;
        uint32_t hole = 0, source = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int place = u.place(y, e);
            const bool stays = ry[e] > last || (ry[e] == last && ties < need);
            ties += place < u.len && ry[e] == last;
            hole |= place < u.len && place < u.m && !stays ? 1u << e : 0u;
            source |= place < u.len && place >= u.m && stays ? 1u << e : 0u;
        }
        const int holes = __builtin_popcount(hole), sources = __builtin_popcount(source);
        const uint32_t upto = sum_upto((uint32_t)holes << 16 | sources);
        int h = b.holes + (int)(upto >> 16) - holes, s = b.sources + (int)(upto & 0xffff) - sources;
        // (as many of one as of the other, and room for all of them)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (hole >> e & 1) to[h++] = u.place(y, e);
            if (source >> e & 1) from[s++] = u.place(y, e);
        }
    }
    if (wave == waves - 1) {                               // behind the workgroup's last place
        const Before all = in_front(kHeld * waves);
        if (lane == 0 && base + 256 * kHeld * waves >= u.len) a.count[u.unit] = all.sources;
    }
}

// A unit to a workgroup.
__global__ __launch_bounds__(64 * kMostWaves) void evict_select_kernel(EvictArgs a)
{
    __shared__ uint32_t bins[kBins], found[2];
    __shared__ int4 counts[kHeld * kMostWaves];
    __shared__ int most[kMostWaves];
    const Unit u(a, blockIdx.x, 0);
    if (!u.moves()) {
        if (threadIdx.x == 0) a.count[u.unit] = 0;
        return;
    }
    int64_t row[kHeld];
    floatx4 w[kHeld];
    intx4 p[kHeld];
    find_rows(row, a, u);
#pragma unroll
    for (int y = 0; y < kHeld; ++y) {
        w[y] = *reinterpret_cast<const floatx4 *>(a.weight + max(row[y], (int64_t)0));
        p[y] = *reinterpret_cast<const intx4 *>(a.position + max(row[y], (int64_t)0));
    }
    clear_bins(bins);
    const int newest = group_max(newest_of(u, row, p), most);
    uintx4 r[kHeld];
    rank_rows(r, a, u, row, w, p, newest);
    count_digits<21, 11>(bins, u, r, 0);
    __syncthreads();
    if (threadIdx.x < 64) find_digit<2048>(bins, u.m, found);
    __syncthreads();
    uint32_t prefix = found[0], need = found[1];
    clear_bins(bins);
    __syncthreads();
    count_digits<10, 11>(bins, u, r, prefix);
    __syncthreads();
    if (threadIdx.x < 64) find_digit<2048>(bins, need, found);
    __syncthreads();
    prefix = prefix << 11 | found[0];
    need = found[1];
    clear_bins(bins);
    __syncthreads();
    count_digits<0, 10>(bins, u, r, prefix);
    __syncthreads();
    if (threadIdx.x < 64) find_digit<1024>(bins, need, found);
    __syncthreads();
    prefix = prefix << 10 | found[0];                      // ranks above it stay, and of this one the first `need`
    need = found[1];
    count_stays(counts, u, r, prefix);
    __syncthreads();
    list_moves(a, u, r, counts, prefix, (int)need, Before{0, 0, 0});
}

// The same by `parts` workgroups to a unit, a launch to a phase: 0 the newest position, 1 ranks and the first digit, 2 the second, 3 the
// third, 4 what stays of every workgroup's places, 5 the moves.
template <int PHASE>
__global__ __launch_bounds__(64 * kMostWaves) void evict_phase_kernel(EvictArgs a)
{
    __shared__ uint32_t bins[kBins], found[2];
    __shared__ int4 counts[kHeld * kMostWaves];
    __shared__ int most[kMostWaves];
    const int part = blockIdx.x % a.parts;
    const Unit u(a, blockIdx.x / a.parts, part);
    const int tid = threadIdx.x, threads = blockDim.x;
    if (!u.moves()) {
        if (PHASE == 0 && part == 0 && tid == 0) a.count[u.unit] = 0;
        return;
    }
    const bool empty = part * kPart >= u.len;
    uint32_t *const unit_bins = a.bins + (int64_t)u.unit * 3 * kBins, *const unit_found = a.found + 8ll * u.unit;
    uintx4 *const ranks = reinterpret_cast<uintx4 *>(a.ranks + u.unit * a.rank_room);
    if constexpr (PHASE == 0)
        for (int x = part * threads + tid; x < 3 * kBins; x += a.parts * threads) unit_bins[x] = 0;
    int64_t row[kHeld];
    floatx4 w[kHeld];
    intx4 p[kHeld];
    uintx4 r[kHeld];
    if constexpr (PHASE <= 1) {
        find_rows(row, a, u);
#pragma unroll
        for (int y = 0; y < kHeld; ++y) {
            if (PHASE == 1) w[y] = *reinterpret_cast<const floatx4 *>(a.weight + max(row[y], (int64_t)0));
            p[y] = *reinterpret_cast<const intx4 *>(a.position + max(row[y], (int64_t)0));
        }
    } else {
#pragma unroll
        for (int y = 0; y < kHeld; ++y) r[y] = u.place(y, 0) < u.len ? ranks[u.place(y, 0) >> 2] : uintx4{0, 0, 0, 0};
    }
    if constexpr (PHASE == 0) {
        const int newest = group_max(newest_of(u, row, p), most);
        if (tid == 0) a.newest[(int64_t)u.unit * a.parts + part] = newest;
        return;
    }
    if constexpr (PHASE == 1) {
        int newest = -0x7fffffff - 1;
        for (int x = tid; x < a.parts; x += threads) newest = max(newest, a.newest[(int64_t)u.unit * a.parts + x]);
        newest = group_max(newest, most);
        rank_rows(r, a, u, row, w, p, newest);
#pragma unroll
        for (int y = 0; y < kHeld; ++y)
            if (u.place(y, 0) < u.len) ranks[u.place(y, 0) >> 2] = r[y];
    }
    if (empty && PHASE < 4) return;
    // what has been found so far; the digit of the launch before is found here, by every workgroup for itself
    uint32_t prefix = 0, need = u.m;
    if constexpr (PHASE >= 2) {
        if constexpr (PHASE > 2) {
            prefix = unit_found[2 * (PHASE == 3 ? 0 : 1)];
            need = unit_found[2 * (PHASE == 3 ? 0 : 1) + 1];
        }
        if constexpr (PHASE <= 4) {
            constexpr int kDigit = PHASE - 2;
            for (int x = tid; x < kBins; x += threads) bins[x] = unit_bins[kDigit * kBins + x];
            __syncthreads();
            if (tid < 64) find_digit<kDigit == 2 ? 1024 : 2048>(bins, need, found);
            __syncthreads();
            prefix = prefix << (kDigit == 2 ? 10 : 11) | found[0];
            need = found[1];
            if (part == 0 && tid == 0) {
                unit_found[2 * kDigit] = prefix;
                unit_found[2 * kDigit + 1] = need;
            }
        } else {
            prefix = unit_found[4];
            need = unit_found[5];
        }
    }
    if constexpr (PHASE >= 1 && PHASE <= 3) {
        clear_bins(bins);
        __syncthreads();
        if constexpr (PHASE == 1) count_digits<21, 11>(bins, u, r, 0);
        if constexpr (PHASE == 2) count_digits<10, 11>(bins, u, r, prefix);
        if constexpr (PHASE == 3) count_digits<0, 10>(bins, u, r, prefix);
        __syncthreads();
        for (int x = tid; x < kBins; x += threads)
            if (bins[x] != 0) atomicAdd(&unit_bins[(PHASE - 1) * kBins + x], bins[x]);
    } else {
        count_stays(counts, u, r, prefix);
        __syncthreads();
        int4 *const of_parts = a.stays + (int64_t)u.unit * a.parts;
        if constexpr (PHASE == 4) {
            if (tid < 64) {
                const int4 n = tid < kHeld * kMostWaves ? counts[tid] : make_int4(0, 0, 0, 0);
                const int4 all = make_int4(wave_upto(n.x), wave_upto(n.y), wave_upto(n.z), wave_upto(n.w));
                if (tid == 63) of_parts[part] = all;
            }
        } else {
            const Before b = before(Before{0, 0, 0}, part, (int)need, [&](int x) { return of_parts[x]; },
                                    [&](int x) { return min(max(u.m - x * kPart, 0), kPart); });
            if (!empty) list_moves(a, u, r, counts, prefix, (int)need, b);
        }
    }
}

// LANES (a power of two) lanes of 16 bytes to a row; `parts` workgroups to a unit.  The first workgroups also write the lengths, which
// the selection has read.
template <int LANES>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, unsigned parts)
{
    constexpr int kGroups = kMoveThreads / LANES;
    const int64_t x = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x;
    if (x < a.n_seq) a.new_lens[x] = min(evict_len(a, (int)x), a.budget);
    const unsigned unit = blockIdx.x / parts;
    if (a.room == 0 || unit >= (unsigned)(a.n_seq * a.h_kv)) return;
    const int i = unit / a.h_kv, h = unit - i * a.h_kv, lane = threadIdx.x % LANES;
    const int first = (blockIdx.x - unit * parts) * kGroups * kMoveEach + threadIdx.x / LANES, count = a.count[unit];
    const int32_t *const to = a.to + (int64_t)unit * a.room, *const from = a.from + (int64_t)unit * a.room;
    int64_t src[kMoveEach], dst[kMoveEach];
    uintx4 k[kMoveEach], v[kMoveEach];
    uint32_t one[kMoveEach];
    // the first lanes of a row also have its weight, its position and its factors
    uint32_t *const mark = reinterpret_cast<uint32_t *>(lane == 0 ? a.weight : lane == 1 ? reinterpret_cast<float *>(a.position)
                                                        : lane == 2 ? a.kf : lane == 3 ? a.vf : nullptr);
#pragma unroll
    for (int y = 0; y < kMoveEach; ++y) {
        const int at = first + y * kGroups;
        src[y] = dst[y] = -1;
        if (at < count) {
            src[y] = row_at(a, i, h, from[at]);
            dst[y] = row_at(a, i, h, to[at]);
        }
    }
#pragma unroll
    for (int y = 0; y < kMoveEach; ++y)
        if (src[y] >= 0) {
            k[y] = *reinterpret_cast<const uintx4 *>(a.K + src[y] * a.row_bytes + 16 * lane);
            v[y] = *reinterpret_cast<const uintx4 *>(a.V + src[y] * a.row_bytes + 16 * lane);
            if (mark) one[y] = mark[src[y]];
        }
#pragma unroll
    for (int y = 0; y < kMoveEach; ++y)
        if (src[y] >= 0 && dst[y] >= 0) {
            *reinterpret_cast<uintx4 *>(a.K + dst[y] * a.row_bytes + 16 * lane) = k[y];
            *reinterpret_cast<uintx4 *>(a.V + dst[y] * a.row_bytes + 16 * lane) = v[y];
            if (mark) mark[dst[y]] = one[y];
        }
}

struct EvictPlan {
    EvictArgs a;
    int waves;
    long long units, parts, grid;                          // of the moves
    size_t bytes, count, to, from, ranks, bins, found, newest, stays;
};

inline pbs_status plan_evict(const pbs_evict_problem *p, const pbs_cache *c, EvictPlan &plan)
{
    if (!p) return PBS_ERR_NULL;
    const pbs_status st = check_cache(c);
    if (st != PBS_OK) return st;
    if (p->n_seq < 0 || p->max_pages < 0 || p->max_len < 0 || p->budget < 0 || p->sinks < 0 || p->recent < 0 ||
        (long long)p->sinks + p->recent > p->budget)
        return PBS_ERR_SHAPE;
    if (p->n_seq > 65535 || p->max_len > 1 << 27 || (long long)p->n_seq * p->max_pages > 0x7fffffffLL) return PBS_ERR_UNSUPPORTED;
    EvictArgs &a = plan.a;
    a = {};
    a.n_seq = p->n_seq; a.h_kv = c->h_kv; a.page_log = log2_of(c->page); a.pages = c->pages; a.max_pages = p->max_pages;
    const long long in_pages = (long long)p->max_pages * c->page;
    a.max_len = p->max_len < in_pages ? p->max_len : (int)in_pages;
    a.budget = p->budget; a.sinks = p->sinks; a.recent = p->recent;
    a.row_bytes = c->d * (c->dtype == PBS_BF16 ? 2 : 1);
    const int over = a.max_len > a.budget ? a.max_len - a.budget : 0;
    a.room = over < a.budget ? over : a.budget;
    plan.waves = a.max_len <= kPart / 4 ? kMostWaves / 4 : kMostWaves;
    a.parts = a.max_len <= kPart ? 1 : (a.max_len + kPart - 1) / kPart;
    a.rank_room = ((int64_t)a.max_len + 3) / 4 * 4;
    plan.units = (long long)a.n_seq * a.h_kv;
    const int rows = kMoveThreads / (a.row_bytes / 16) * kMoveEach;
    plan.parts = ((long long)a.room + rows - 1) / rows;
    const long long lens = ((long long)a.n_seq + kMoveThreads - 1) / kMoveThreads;
    plan.grid = plan.parts * plan.units > lens ? plan.parts * plan.units : lens;
    if (!fits_grid(plan.units * a.parts, 64 * plan.waves) || plan.units * a.parts > 0x7fffffffLL || !fits_grid(plan.grid, kMoveThreads)) return PBS_ERR_UNSUPPORTED;
    size_t at = 0;
    auto room = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, kWsAlign); return here; };
    const bool any = a.room > 0;                           // otherwise nothing can move
    plan.count = room(any ? (size_t)plan.units * 4 : 0);
    plan.to = room((size_t)plan.units * a.room * 4);
    plan.from = room((size_t)plan.units * a.room * 4);
    const size_t apart = any && a.parts > 1 ? (size_t)plan.units : 0;
    plan.ranks = room(apart * a.rank_room * 4);
    plan.bins = room(apart * 3 * kBins * 4);
    plan.found = room(apart * 8 * 4);
    plan.newest = room(apart * a.parts * 4);
    plan.stays = room(apart * a.parts * 16);
    plan.bytes = at;
    return PBS_OK;
}

inline pbs_status launch_evict(const EvictPlan &plan, hipStream_t s)
{
    const EvictArgs &a = plan.a;
    if (a.room > 0) {
        const dim3 grid((unsigned)(plan.units * a.parts)), block(64 * plan.waves);
        void (*const phases[])(EvictArgs) = {evict_phase_kernel<0>, evict_phase_kernel<1>, evict_phase_kernel<2>,
                                             evict_phase_kernel<3>, evict_phase_kernel<4>, evict_phase_kernel<5>};
        pbs_status st = a.parts == 1 ? launch(evict_select_kernel, grid, block, 0, s, a) : PBS_OK;
        for (int x = 0; x < 6 && a.parts > 1 && st == PBS_OK; ++x) st = launch(phases[x], grid, block, 0, s, a);
        if (st != PBS_OK) return st;
    }
    const unsigned parts = plan.parts > 0 ? (unsigned)plan.parts : 1;
    auto kernel = a.row_bytes == 256 ? evict_move_kernel<16> : a.row_bytes == 128 ? evict_move_kernel<8> : evict_move_kernel<4>;
    return launch(kernel, dim3((unsigned)plan.grid), dim3(kMoveThreads), 0, s, a, parts);
}

}  // namespace pbs

extern "C" size_t pbs_evict_workspace_bytes(const pbs_evict_problem *p, const pbs_cache *c)
{
    pbs::EvictPlan plan;
    return pbs::plan_evict(p, c, plan) == PBS_OK ? plan.bytes : 0;
}

extern "C" pbs_status pbs_cache_evict(const pbs_evict_problem *p, const pbs_cache *c, const pbs_cache_marks *marks,
                                      const int32_t *page_table, const int32_t *lens, int32_t *new_lens, void *ws, size_t ws_bytes,
                                      void *stream)
{
    using namespace pbs;
    EvictPlan plan;
    const pbs_status st = plan_evict(p, c, plan);
    if (st != PBS_OK) return st;
    if (!marks || !marks->weight || !marks->position) return PBS_ERR_NULL;
    if (!aligned16(marks->weight) || !aligned16(marks->position)) return PBS_ERR_SHAPE;
    if (p->n_seq == 0) return PBS_OK;
    if (!lens || !new_lens || (p->max_pages > 0 && !page_table)) return PBS_ERR_NULL;
    if (((reinterpret_cast<uintptr_t>(page_table) | reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(new_lens)) & 3u) != 0)
        return PBS_ERR_SHAPE;
    if (plan.bytes > 0) {
        if (!ws) return PBS_ERR_NULL;
        if ((reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)) != 0 || ws_bytes < plan.bytes) return PBS_ERR_WORKSPACE;
    }
    EvictArgs &a = plan.a;
    a.table = page_table; a.lens = lens; a.new_lens = new_lens;
    a.K = static_cast<uint8_t *>(c->K);
    a.V = static_cast<uint8_t *>(c->V);
    a.kf = c->dtype == PBS_BF16 ? nullptr : c->k_scale;
    a.vf = c->dtype == PBS_BF16 ? nullptr : c->v_scale;
    a.weight = marks->weight;
    a.position = marks->position;
    uint8_t *room = static_cast<uint8_t *>(ws);
    a.count = reinterpret_cast<int32_t *>(room + plan.count);
    a.to = reinterpret_cast<int32_t *>(room + plan.to);
    a.from = reinterpret_cast<int32_t *>(room + plan.from);
    a.ranks = reinterpret_cast<uint32_t *>(room + plan.ranks);
    a.bins = reinterpret_cast<uint32_t *>(room + plan.bins);
    a.found = reinterpret_cast<uint32_t *>(room + plan.found);
    a.newest = reinterpret_cast<int32_t *>(room + plan.newest);
    a.stays = reinterpret_cast<int4 *>(room + plan.stays);
    return launch_evict(plan, static_cast<hipStream_t>(stream));
}
