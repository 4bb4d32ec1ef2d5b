// verify_shared.hip -- paged attention of a batch whose requests begin with the same
// tokens: the keys of a common prefix are read once for all rows that see them.
//
// A segment is a run of packed query rows and a run of KV blocks that they see:
//   prefix k   all rows of the requests of group k, the blocks of its prefix;
//   own i      the rows of request i, its blocks behind the prefix.
// A row's softmax runs over its prefix segment and its own one.  Both parts leave the
// running maximum m (of the scores times scale log2 e), l = sum 2^(s - m) and the
// output sum 2^(s - m) v, unnormalised and in fp32, and a last pass joins them:
//     out = sum_k 2^(m_k - M) o_k / (sum_k 2^(m_k - M) l_k + 2^(sink log2 e - M)).
//
// Work.  A pair is (segment, KV head, row tile), a unit 128 keys of a pair (fp32: 64).  The workgroups
// are all resident at once.  Some take the prefixes: each pair's keys are cut into parts
// of the same length, an item is one part of one pair, and the items of a part's tiles
// follow each other.  The others take the own units, numbered segment by segment, then
// head, tile and key, in equal ranges.  A range's piece of pair p in workgroup w leaves
// its partial result in slot p + w, which no other piece has, since one of the two grows
// from each piece to the next; an item's slot is its number.
//
// Matrix products, per 16-row tile and 32 keys (two blocks), lane = 16 lg + l16:
//   S^T = K Q^T    v_mfma_f32_16x16x32_bf16, A = K: row m of product t is key
//                  8 ((m >> 2) & 1) + 4 t + (m & 3) of block m >> 3, so that lane lg's
//                  results of both products are its eight keys 8 lg .. 8 lg + 7 of 32;
//   O^T += V^T P^T the same instruction, A = V^T: a lane's 16 bytes are the eight keys
//                  8 lg .. 8 lg + 7 of dim l16, B = P^T as the scores left it.
// Nothing but the operands of several wavefronts goes through LDS.  bf16's weights enter the
// second product in bf16, as verify_attention's do; maxima, sums and outputs are in fp32, and
// the sum is that of the unrounded weights.  The rounding takes the output's error from
// the 0.0017 of its norm that the store alone leaves to 0.0022-0.0023.  A second product with
// what the rounding takes off leaves 0.0017 and costs a third more where the matrix units count: 288
// rows behind 65536 keys 297 -> 391 us, 32 requests of nine rows 87 -> 100, 64 single rows 52.6 ->
// 54.9 (fp32 inputs have fp32 weights and products).
//
// Few rows (flat): the four wavefronts of a workgroup take 32 of a unit's 128 keys each,
// with all rows, straight from memory into operand registers, the next unit's keys
// asked for as soon as this one's scores are done.  Bound by memory: 64 requests of
// one row, 8192 keys of their own, 2.1 GB in 372 to 415 us by what ran before (5.8 to 5.2 TB/s).
// Many rows (tall): the wavefronts take the rows, and the keys pass through a ring of
// LDS stages that all of them read.  Bound by the matrix units, the exponentials and the
// latencies between them: 288 rows behind 65536 common keys, 309 GFLOP in 303 us.
// Both at once: 32 requests of nine rows, 512 to 4096 keys behind 8192 common ones, 86 us
// (the walk 77, of which each kind of work alone would take about 45).
#include <type_traits>

#include "common.h"

// m0 is set inside the global->LDS load sequence (see dma16_run); the compiler
// reloads m0 before each of its own uses, so clobbering it there is safe.
#pragma clang diagnostic ignored "-Winline-asm"

namespace averify {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr float kLog2e = 1.4426950408889634f;
// KV blocks of a unit: two for each wavefront in bf16, one in fp32, whose products take
// eight times as long (two requests of three rows, 130 keys behind 64 common ones: 14.5 us,
// with two 16.3).
constexpr int unit_shift(bool f32) { return f32 ? 2 : 3; }
constexpr int kUnitBlocks = 1 << unit_shift(false);
static_assert(kUnitBlocks == 2 * kWaves && 1 << unit_shift(true) == kWaves, "the flat walks' blocks");
// What a pair costs beside its blocks (its rows, the first blocks' latency, the join of
// the wavefronts, the partial result), in units: it counts so many units more, without
// blocks, in front of its own.
constexpr int kPairUnits = 1;
constexpr int kInlineSegs = 256;    // segments whose units every workgroup counts itself
// A prefix's unit of 128 rows beside one of few rows: 3.5 us where 4.3 (the one fills the
// matrix units, the other waits for 64 KiB; 32 requests of nine rows, 8192 common keys).
constexpr float kTallUnit = 0.8f;
constexpr int kStages = 4;          // of the tall walk's ring
// Keys of a short request, and of all tiles of a workgroup's share of them, at most (see
// shared_short).
constexpr int short_keys(bool f32, int d) { return f32 ? d == 64 ? 704 : 448 : d == 64 ? 4096 : 2048; }
constexpr int short_share(bool f32, int d) { return f32 ? 896 : d == 64 ? 2560 : 2048; }
constexpr float kNoMax = -3.0e38f;  // a maximum over no key
// Softmax weights may exceed 1 by up to this factor (log2) before a row's maximum is
// raised: with a maximum that need not be exact the raise is rare.
constexpr float kSlackLog2 = 8.f;
// 16-row tiles of a flat walk at most.  In bf16 two of them and the keys under way do not
// fit 256 registers, and the ring serves 32 rows as well (5.2 TB/s; flat, with 16 rows, 5.6;
// with Q in LDS three fit, but 32 requests of nine rows take 71 us instead of 65).  In fp32
// more rows read the keys less often: 288 rows behind 65536 common keys, 309 GFLOP, take
// 2.55 ms (121 TFLOP/s) with three tiles, 2.81 with two.
constexpr int flat_tiles(bool f32, int d) { return !f32 ? 1 : d == 64 ? 4 : 3; }
constexpr int tall_tiles(int d) { return d == 64 ? 3 : 2; }  // per wavefront

// The lane's number, of which the compiler does not know that it is the same in every
// piece of a workgroup: what a walk derives from it is computed in that walk, instead of
// taking registers from all others.
__device__ __forceinline__ int own_lane() {
    int lane = threadIdx.x % kWave;
    asm volatile("" : "+v"(lane));
    return lane;
}

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
// callers' tensors need only be aligned to an element
typedef uint32_t u32x4h_t __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));

// Where a row's partial results lie.
struct __attribute__((aligned(16))) RowParts {
    int64_t unit0;  // own: the segment's first unit, and pair
    int pair0, real, tiles, height, e0;  // units of a pair (0: none), tiles, rows of a tile, the row's first place
    int item0, parts, prefix_tiles, prefix_height, prefix_e0;  // of a prefix: likewise (parts 0: none)
};
static_assert(sizeof(RowParts) == 48, "three loads");

struct SharedArgs {
    const void* q;
    const uint8_t* kc;
    const uint8_t* vc;
    const float* sinks;
    void* out;
    float* part_o;    // [slots][tile rows][D]
    float2* part_ml;  // [slots][tile rows] maximum and sum
    RowParts* rows;  // [total_q]
    struct Share* share;
    struct Segment* segments;  // where a workgroup does not count them itself
    struct Items* items;
    int num_seqs, num_groups, hq, hkv, group, max_blocks, num_blocks, max_seq_len, max_prefix, total_q;
    int nwg;
    int tile_a, tile_b;    // rows of a tile at most: prefix and own segments
    int unit_shift;        // KV blocks of a unit, log2
    int weighted;          // own units are counted by the rows of their tiles
    int64_t slots_a, slots_b;
    float scale_log2;
};

struct Index {  // device arrays that nothing writes
    const int32_t* __restrict__ tables;
    const int32_t* __restrict__ lens;
    const int32_t* __restrict__ q_start;
    const int32_t* __restrict__ group_start;
    const int32_t* __restrict__ prefix;
};

struct __attribute__((aligned(16))) Segment {
    int64_t unit0;   // number of its first unit
    int pair0;       // own: of its first pair; prefix: pairs
    int q0, rows;    // first packed row, packed rows times query heads per KV head
    int b_lo, b_hi;  // blocks
    int table;       // the request whose block table lists the blocks
    int S;           // keys from S on are not the request's
    int pos0;        // own: position of the first row; prefix: whether a row stands inside
    int group;       // own: the request's group, or -1
};

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return max(lo, min(v, hi)); }

__device__ __forceinline__ int clamped_len(const SharedArgs& a, const Index& x, int i) {
    return clamp_to(x.lens[i], 0, min(a.max_seq_len, a.max_blocks * kBlockTokens));
}

// Whole blocks of group k's prefix, as far as its first request has cached them: their ids
// are read from that request's row.
__device__ __forceinline__ int prefix_blocks(const SharedArgs& a, const Index& x, int k) {
    const int cached = clamped_len(a, x, clamp_to(x.group_start[k], 0, a.num_seqs - 1));
    return clamp_to(x.prefix[k], 0, min(a.max_prefix, cached)) / kBlockTokens;
}

// The group of request i: the last one that begins at or before it, if it holds i.
__device__ __forceinline__ int group_of(const SharedArgs& a, const Index& x, int i) {
    int lo = 0, hi = a.num_groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (x.group_start[mid] <= i) lo = mid; else hi = mid - 1;
    }
    return x.group_start[lo] <= i && i < x.group_start[lo + 1] ? lo : -1;
}

// Segment s, but for its first unit and pair.
__device__ __forceinline__ Segment segment_of(const SharedArgs& a, const Index& x, int s) {
    Segment g;
    const bool first = s < a.num_groups;
    if (first) {
        const int r0 = clamp_to(x.group_start[s], 0, a.num_seqs), r1 = clamp_to(x.group_start[s + 1], r0, a.num_seqs);
        g.q0 = clamp_to(x.q_start[r0], 0, a.total_q);
        g.rows = (clamp_to(x.q_start[r1], g.q0, a.total_q) - g.q0) * a.group;
        g.b_lo = 0;
        g.b_hi = prefix_blocks(a, x, s);
        g.table = min(r0, a.num_seqs - 1);
        g.S = g.b_hi * kBlockTokens;
        g.pos0 = 0;
        g.group = s;
    } else {
        const int i = s - a.num_groups;
        g.q0 = clamp_to(x.q_start[i], 0, a.total_q);
        const int n = clamp_to(x.q_start[i + 1], g.q0, a.total_q) - g.q0;
        g.rows = n * a.group;
        g.group = group_of(a, x, i);
        g.S = clamped_len(a, x, i);
        g.b_lo = g.group >= 0 ? prefix_blocks(a, x, g.group) : 0;
        g.b_hi = max(g.b_lo, (g.S + kBlockTokens - 1) / kBlockTokens);
        g.table = i;
        g.pos0 = g.S - n;
    }
    return g;
}

// A segment's rows divided evenly over as few tiles of at most `most` rows as there need
// be: their number, and the rows of one.
__device__ __forceinline__ int tiles_of(const Segment& g, int most) {
    // most is a power of two, or three times one
    const uint32_t n = (uint32_t)(g.rows + most - 1) >> __builtin_ctz(most);
    return most % 3 == 0 ? __umulhi(n, 0xaaaaaaabu) >> 1 : n;
}
__device__ __forceinline__ int tile_rows(const Segment& g, int tiles) {
    if (tiles <= 1) return max(16, (g.rows + 15) / 16 * 16);
    return ((uint32_t)(g.rows + tiles - 1) / (uint32_t)tiles + 15) / 16 * 16;
}

__device__ __forceinline__ int units_of(const SharedArgs& a, const Segment& g) {
    return g.b_hi > g.b_lo ? (g.b_hi - g.b_lo + (1 << a.unit_shift) - 1) >> a.unit_shift : 0;
}

// Where the requests' rows may differ by several 16-row tiles per wavefront, a unit does
// not cost the same in all of them (128 keys of head dim 64 take a workgroup 3.1 us with
// 16 rows, 3.7 with 64, 4.3 with 128, 5.9 with 192): a unit then counts `each` and a
// pair `extra` more; otherwise 1 and kPairUnits.
constexpr int kMostEach = 6;
struct Cost {
    int extra, each;
};
__device__ __forceinline__ Cost cost_of(const SharedArgs& a, int height) {
    return a.weighted ? Cost{4 * kPairUnits, height <= 16 ? 3 : height <= 128 ? 4 : kMostEach} : Cost{kPairUnits, 1};
}

// v of the lanes up to this one, summed.
__device__ __forceinline__ int scan_lanes(int v) {
    auto add = [&](auto ctrl, auto rows) {
        v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    };
    using std::integral_constant;
    add(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // the lane 1, 2, 4, 8 before it in its row of 16
    add(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // the last lane of the row before
    add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // the last lane of the first half
    return v;
}
__device__ __forceinline__ int64_t scan_lanes(int64_t v) {
    for (int o = 1; o < kWave; o <<= 1) {
        const int64_t w = __shfl_up(v, o);
        if ((int)threadIdx.x % kWave >= o) v += w;
    }
    return v;
}

// Maximum and sum over lanes l, l ^ 16, l ^ 32, l ^ 48, which hold one row's keys.
__device__ __forceinline__ float rows_max(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float m = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float rows_sum(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float m = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// a / b rounded down, 0 <= a < 2^52: a quotient in binary64 is not rounded up to the next
// whole number.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) { return (int64_t)((double)a / (double)b); }

// How the workgroups are divided: na of them take the prefixes' items, the others the ub
// own units behind unit ua.  Where there are fewer of these than workgroups, cb of them
// have one.
struct __attribute__((aligned(16))) Share {
    int64_t ua, ub;
    int items, na, cb;
};

// A prefix's items: the first one, and the parts that each of its pairs is cut into.
struct Items {
    int first, parts;
};

// What a part of a prefix costs beside its units, in units, with its way through the join.
__device__ __forceinline__ float item_units(const SharedArgs& a) {
    return a.unit_shift == unit_shift(true) && a.tile_a > 16 ? 1.f : 2.f;
}

// Counts the units and pairs of all segments and cuts the prefixes' pairs into items, by
// one workgroup of THREADS threads.  Count: of all units.
template <int THREADS, typename Count>
__device__ __forceinline__ Share count_units(const SharedArgs& a, const Index& x, Segment* segments, Items* items) {
    __shared__ Count s_units[THREADS / kWave];
    __shared__ int s_pairs[THREADS / kWave];
    const int tid = threadIdx.x, lane = tid % kWave, segs = a.num_groups + a.num_seqs;
    Count units = 0;
    int pairs = 0;
    for (int base = 0; base < segs; base += THREADS) {
        const int s = base + tid;
        Segment g;
        int p = 0, each = 0;
        if (s < segs) {
            g = segment_of(a, x, s);
            const int tiles = tiles_of(g, s < a.num_groups ? a.tile_a : a.tile_b), real = units_of(a, g);
            const Cost c = s >= a.num_groups && a.weighted ? cost_of(a, tile_rows(g, tiles)) : Cost{kPairUnits, 1};
            each = real > 0 ? c.extra + real * c.each : 0;
            p = each > 0 ? tiles * a.hkv : 0;
        }
        const Count u = (Count)p * each, u_lanes = scan_lanes(u);
        const int own = s < a.num_groups ? 0 : p;  // prefixes' pairs have slots of their own
        const int p_lanes = scan_lanes(own);
        if (lane == kWave - 1) s_units[tid / kWave] = u_lanes, s_pairs[tid / kWave] = p_lanes;
        __syncthreads();
        Count u_all = 0, u_before = units + u_lanes - u;
        int p_all = 0, p_before = pairs + p_lanes - own;
#pragma unroll
        for (int w = 0; w < THREADS / kWave; ++w) {
            if (w < tid / kWave) u_before += s_units[w], p_before += s_pairs[w];
            u_all += s_units[w];
            p_all += s_pairs[w];
        }
        if (s < segs) {
            g.unit0 = u_before;
            g.pair0 = s < a.num_groups ? p : p_before;
            segments[s] = g;
        }
        units += u_all;
        pairs += p_all;
        __syncthreads();
    }
    Share h;
    h.ua = a.num_seqs > 0 ? segments[a.num_groups].unit0 : units;
    h.ub = units - h.ua;
    // a row that stands in front of its prefix's last key sees a part of it
    for (int i = tid; i < a.num_seqs; i += THREADS) {
        const Segment& g = segments[a.num_groups + i];
        if (g.group >= 0 && g.rows > 0 && g.pos0 < g.b_lo * kBlockTokens - 1) segments[g.group].pos0 = 1;
    }
    h.na = h.items = 0;
    if (h.ua > 0) {
        // The parts' length and the number of workgroups with which the last of all is
        // done first: 64 lengths between an eighth of a workgroup's mean share and four
        // times it, one to a lane, each with as many workgroups as there are items, with
        // a half and a third of that, and with their share of the work.  Every wavefront
        // does it for itself.
        const float unit = a.tile_a >= 128 ? kTallUnit : 1.f, own = (float)h.ub * (a.weighted ? 0.25f : 1.f);
        const float mean = fmaxf(1.f, ((float)h.ua * unit + own) * __builtin_amdgcn_rcpf(unit * a.nwg));
        auto length = [&](int c) { return fminf(1.0e9f, ceilf(mean * 0.125f * __builtin_amdgcn_exp2f(5.f / 63 * c))); };
        auto parts_of = [&](int units, float cost) {
            return max(1, (int)ceilf((float)units * __builtin_amdgcn_rcpf(cost) - 0.001f));
        };
        const float cost = length(lane);
        float all = 0.f;
        int longest = 0;
        for (int base = 0; base < a.num_groups; base += kWave) {
            // a group to a lane, handed to all lanes one after the other
            const Segment* mine = segments + min(base + lane, a.num_groups - 1);
            const int my_units = units_of(a, *mine), my_pairs = mine->pair0;
            for (int k = 0; k < min(kWave, a.num_groups - base); ++k) {
                const int units = __builtin_amdgcn_readlane(my_units, k), pairs = __builtin_amdgcn_readlane(my_pairs, k);
                const int parts = parts_of(units, cost);
                all += (float)pairs * (float)parts;
                longest = max(longest, pairs ? (int)ceilf((float)units * __builtin_amdgcn_rcpf((float)parts) - 0.001f) : 0);
            }
        }
        // the workgroups of this length, eight at least for each kind of work
        const float most = h.ub > 0 ? a.nwg - 8 : a.nwg;
        const float share = (float)h.ua * unit * a.nwg * __builtin_amdgcn_rcpf((float)h.ua * unit + own);
        float time = INFINITY, na = 0.f;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const float want = ceilf((n == 3 ? share : all * (n == 2 ? 1.f / 3 : n == 1 ? 0.5f : 1.f)) * 0.125f - 0.001f) * 8.f;
            const float wgs = fminf(fmaxf(want, 8.f), most);
            const float rounds = ceilf(all * __builtin_amdgcn_rcpf(wgs) - 0.001f);
            const float t = fmaxf(rounds * ((float)longest + item_units(a)) * unit, own * __builtin_amdgcn_rcpf(fmaxf(a.nwg - wgs, 1.f)));
            na = t <= time ? wgs : na;
            time = fminf(t, time);
        }
        // (rounded sums: items that would not fit are cut off well before the last slot)
        if (!(all < 0.99f * (float)a.slots_a)) time = INFINITY;
        float best = time;  // over all lanes: rows of 16 by rotations, then their four results
        auto least = [&](auto ctrl) {
            best = fminf(best, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(best), decltype(ctrl)::value, 0xf, 0xf, true)));
        };
        least(std::integral_constant<int, 0x121>{});
        least(std::integral_constant<int, 0x122>{});
        least(std::integral_constant<int, 0x124>{});
        least(std::integral_constant<int, 0x128>{});
        best = -rows_max(-best);
        // the longest parts of equal candidates; whole prefixes always fit
        const uint64_t equal = __ballot(time == best);
        const int winner = 63 - __clzll((long long)equal);
        const bool fits = best < INFINITY;
        const float chosen = fits ? length(winner) : 1.0e9f;
        h.na = fits ? __builtin_amdgcn_readlane((int)na, winner) : h.ub > 0 ? a.nwg / 2 : a.nwg;
        for (int base = 0; base < a.num_groups; base += kWave) {
            const int k = base + lane;
            const Segment* g = segments + min(k, a.num_groups - 1);
            const int parts = k < a.num_groups && g->pair0 > 0 ? parts_of(units_of(a, *g), chosen) : 0;
            const int here = scan_lanes(parts * g->pair0);
            if (tid < kWave && k < a.num_groups) items[k] = Items{h.items + here - parts * g->pair0, parts};
            h.items += __builtin_amdgcn_readlane(here, kWave - 1);
        }
    }
    // (weighted: a range that lies within a pair holds a unit's beginning)
    h.cb = (int)min((int64_t)(a.nwg - h.na), a.weighted && h.ub > 0 ? max((int64_t)1, h.ub / kMostEach) : h.ub);
    __syncthreads();
    return h;
}

constexpr int kScheduleGroups = 2048;  // that a schedule's workgroup keeps in LDS
__global__ __launch_bounds__(1024) void shared_schedule(SharedArgs a, Index x) {
    // every request looks for its group among them
    __shared__ int32_t s_start[kScheduleGroups + 1], s_prefix[kScheduleGroups];
    if (a.num_groups <= kScheduleGroups) {
        for (int k = threadIdx.x; k <= a.num_groups; k += 1024) {
            s_start[k] = x.group_start[k];
            if (k < a.num_groups) s_prefix[k] = x.prefix[k];
        }
        __syncthreads();
        x.group_start = s_start;
        x.prefix = s_prefix;
    }
    const Share h = count_units<1024, int64_t>(a, x, a.segments, a.items);
    if (threadIdx.x == 0) *a.share = h;
}

// The last k in lo .. hi with begin(k) <= at (begin(lo) is), by a whole wavefront: 64 places
// at once, so that thousands of entries in memory are two latencies deep.
template <typename Begin, typename At>
__device__ __forceinline__ int find_last(Begin begin, int lo, int hi, At at) {
    const int lane = threadIdx.x % kWave;
    for (;;) {
        const int step = (hi - lo) / kWave + 1;
        const int k = lo + lane * step;
        const int found = __popcll(__ballot(k <= hi && begin(min(k, hi)) <= at));
        lo += max(0, found - 1) * step;
        if (step == 1) return lo;
        hi = min(hi, lo + step - 1);
    }
}

// The request of a packed row: the last one that begins at or before it.
__device__ __forceinline__ int request_of(const int32_t* q_start, int num_seqs, int row) {
    int lo = 0, hi = num_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (q_start[mid] <= row) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// The rows' records for the pass that joins: a row to a thread of the launch where the
// descriptor is in LDS, to a wavefront where it is in memory.
template <bool INLINE>
__device__ __forceinline__ void describe_rows(const SharedArgs& a, const Index& x, const Segment* segments, const Items* items,
                                              int64_t ua) {
    constexpr int kRows = INLINE ? kThreads : kWaves;  // of a workgroup at a time
    const int mine = INLINE ? threadIdx.x : threadIdx.x / kWave;
    for (int64_t row = (int64_t)blockIdx.x * kRows + mine; row < a.total_q; row += (int64_t)a.nwg * kRows) {
        const int i = INLINE ? request_of(x.q_start, a.num_seqs, (int)row)
                             : find_last([&](int k) { return x.q_start[k]; }, 0, a.num_seqs - 1, (int)row);
        RowParts r{};
        r.e0 = -1;  // a row of no request
        if (x.q_start[i] <= row && row < x.q_start[i + 1]) {
            const Segment own = segments[a.num_groups + i];
            r.unit0 = own.unit0 - ua;
            r.pair0 = own.pair0;
            r.real = units_of(a, own);
            r.tiles = tiles_of(own, a.tile_b);
            r.height = tile_rows(own, r.tiles);
            r.e0 = max(0, (int)row - own.q0) * a.group;
            if (own.group >= 0) {
                const Segment common = segments[own.group];
                r.item0 = items[own.group].first;
                r.parts = common.pair0 > 0 ? items[own.group].parts : 0;
                r.prefix_tiles = tiles_of(common, a.tile_a);
                r.prefix_height = tile_rows(common, r.prefix_tiles);
                r.prefix_e0 = max(0, (int)row - common.q0) * a.group;
            }
        }
        a.rows[row] = r;
    }
}

// One workgroup's piece of a pair.
struct Piece {
    int q0, row0, rows;  // the segment's first packed row; the tile's first row and rows
    int head;
    int b_lo, b_hi;      // the segment's blocks
    int u0, u1;          // units
    int min_pos, S;      // lowest position of a row; keys from S on are not the request's
    int pos0;            // own: position of the segment's first row
    bool prefix, masked; // of a prefix, in which some row stands
    const int32_t* table;
    int64_t slot_row;    // first row of the partial result
};

// The position of the tile's row r; rows behind its last one see no key.
__device__ __forceinline__ int row_position(const SharedArgs& a, const Index& x, const Piece& p, int r) {
    if (r >= p.rows) return -1;
    const int at = (p.row0 + r) / a.group;
    if (!p.prefix) return p.pos0 + at;
    if (!p.masked) return INT32_MAX;
    const int row = p.q0 + at, i = request_of(x.q_start, a.num_seqs, row);
    return clamped_len(a, x, i) - (x.q_start[i + 1] - row);
}

template <typename T, int D>
__device__ __forceinline__ const T* query_row(const SharedArgs& a, const Piece& p, int r) {
    const int e = p.row0 + min(r, p.rows - 1);
    return static_cast<const T*>(a.q) + ((int64_t)(p.q0 + e / a.group) * a.hq + p.head * a.group + e % a.group) * D;
}

// The scores of a lane's N keys of one row become weights 2^(scale s - m), whose sum joins
// l.  Where a weight would exceed the slack the maximum is raised first, and what has
// been summed is rescaled.
template <int N, int DT>
__device__ __forceinline__ void weigh(float* s, float scale, float& m, float& l, f32x4_t* o) {
    float t[N];
#pragma unroll
    for (int e = 0; e < N; ++e) t[e] = fmaf(s[e], scale, -m);
    float top = t[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, t[e]);
    if (__any(top > kSlackLog2)) {
        float high = s[0];
#pragma unroll
        for (int e = 1; e < N; ++e) high = fmaxf(high, s[e]);
        const float next = fmaxf(m, rows_max(high * scale)), f = __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= f;
#pragma unroll
        for (int e = 0; e < N; ++e) t[e] = fmaf(s[e], scale, -m);
    }
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        s[e] = __builtin_amdgcn_exp2f(t[e]);
        sum += s[e];
    }
    l += sum;
}

// V^T of keys from `left` on (of the lane's eight) becomes zero: what a slot behind the
// last key holds may be no number.
__device__ __forceinline__ uint4 first_keys(uint4 v, int left) {
    const uint32_t m[4] = {left > 1 ? ~0u : left > 0 ? 0xffffu : 0u, left > 3 ? ~0u : left > 2 ? 0xffffu : 0u,
                           left > 5 ? ~0u : left > 4 ? 0xffffu : 0u, left > 7 ? ~0u : left > 6 ? 0xffffu : 0u};
    return make_uint4(v.x & m[0], v.y & m[1], v.z & m[2], v.w & m[3]);
}

__device__ __forceinline__ bf16x8_t as_bf16x8(const uint4& v) { return __builtin_bit_cast(bf16x8_t, v); }

// One step of 32 keys from block b0 on for RT row tiles.  load_k(t, c) and load_v(dt)
// give the operands; EDGE: some row does not see some key, or a block is not mapped
// (ok: whether the lane's keys' is).
template <int D, int RT, bool EDGE, typename LoadK, typename AfterK, typename LoadV>
__device__ __forceinline__ void step32(const Piece& p, int lg, int b0, bool ok, float scale, const bf16x8_t (*q)[D / 32],
                                       const int* pos, float* m, float* l, f32x4_t (*o)[D / 16], LoadK load_k,
                                       AfterK after_k, LoadV load_v) {
    f32x4_t s[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bf16x8_t k = load_k(t, c);
#pragma unroll
            for (int r = 0; r < RT; ++r) s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[r][c], s[r][t], 0, 0, 0);
        }
    after_k();
    const int key0 = b0 * kBlockTokens + 8 * lg;
    bf16x8_t w[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float e8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            e8[e] = s[r][e / 4][e % 4];
            if (EDGE && (!ok || key0 + e > pos[r])) e8[e] = -INFINITY;
        }
        weigh<8, D / 16>(e8, scale, m[r], l[r], o[r]);
        w[r] = as_bf16x8(make_uint4(pack_bf16x2(e8[0], e8[1]), pack_bf16x2(e8[2], e8[3]), pack_bf16x2(e8[4], e8[5]),
                                    pack_bf16x2(e8[6], e8[7])));
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
        uint4 v = load_v(t);
        if (EDGE) v = first_keys(v, ok ? p.S - key0 : 0);
#pragma unroll
        for (int r = 0; r < RT; ++r) o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v), w[r], o[r][t], 0, 0, 0);
    }
}

// Row r's dims 16 t + 4 lg .. + 3 of the partial result, and its maximum and sum.
template <int D>
__device__ __forceinline__ void store_partial(const SharedArgs& a, const Piece& p, int lg, int r, int t, const f32x4_t& v) {
    if (r < p.rows) *reinterpret_cast<f32x4_t*>(a.part_o + (p.slot_row + r) * D + 16 * t + 4 * lg) = v;
}

// A row's output: its sum joined by its sink, which adds to nothing else.  A row without
// keys is zero.
template <typename T>
__device__ __forceinline__ void store_out(const SharedArgs& a, int64_t row, int h, int D, int d, float top, float sum,
                                          const f32x4_t& acc) {
    const float den = a.sinks ? sum + exp2f(fmaf(a.sinks[h], kLog2e, -top)) : sum;
    const f32x4_t y = sum == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc / den;
    T* to = static_cast<T*>(a.out) + (row * a.hq + h) * D + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) Storage<T>::store(to, e, y[e]);
}

// The W wavefronts' states of the same rows, joined and stored: as a partial result, or
// where the piece is all that its rows see (WHOLE) as the output.  smem: W D / 16 KiB.
template <typename T, int D, int RT, bool WHOLE, int W>
__device__ __forceinline__ void join_waves(const SharedArgs& a, const Piece& p, float* m, float* l, f32x4_t (*o)[D / 16],
                                           uint8_t* smem) {
    constexpr int DT = D / 16;
    __shared__ float s_ml[2][W][16];
    const int wave = threadIdx.x / kWave, lane = own_lane(), l16 = lane % 16;
    f32x4_t* part = reinterpret_cast<f32x4_t*>(smem);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float sum = rows_sum(l[r]);
        if (lane < 16) s_ml[0][wave][l16] = m[r], s_ml[1][wave][l16] = sum;
#pragma unroll
        for (int t = 0; t < DT; ++t) part[(wave * DT + t) * kWave + lane] = o[r][t];
        __syncthreads();
        float top = s_ml[0][0][l16];
#pragma unroll
        for (int w = 1; w < W; ++w) top = fmaxf(top, s_ml[0][w][l16]);
        float f[W], all = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            f[w] = __builtin_amdgcn_exp2f(s_ml[0][w][l16] - top);
            all = fmaf(s_ml[1][w][l16], f[w], all);
        }
#pragma unroll
        for (int t0 = 0; t0 < DT; t0 += W) {
            const int t = t0 + wave;
            if (DT % W != 0 && t >= DT) break;
            f32x4_t v = part[t * kWave + lane] * f[0];
#pragma unroll
            for (int w = 1; w < W; ++w) v += part[(w * DT + t) * kWave + lane] * f[w];
            if constexpr (WHOLE) {
                const int e = p.row0 + r * 16 + l16;
                if (r * 16 + l16 < p.rows)
                    store_out<T>(a, p.q0 + e / a.group, p.head * a.group + e % a.group, D, 16 * t + 4 * (lane / 16), top, all, v);
            } else {
                store_partial<D>(a, p, lane / 16, r * 16 + l16, t, v);
            }
        }
        if (!WHOLE && threadIdx.x < 16 && r * 16 + l16 < p.rows) a.part_ml[p.slot_row + r * 16 + l16] = make_float2(top, all);
        __syncthreads();
    }
}

// Few rows, bf16.
template <int D, bool WHOLE = false, int W = kWaves>
__device__ void walk_flat(const SharedArgs& a, const Index& x, const Piece& p, uint8_t* smem) {
    constexpr int RT = 1, DT = D / 16, C = D / 32;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = own_lane(), l16 = lane % 16,
              lg = lane / 16;
    bf16x8_t q[RT][C];
    f32x4_t o[RT][DT];
    float m[RT], l[RT];
    int pos[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const uint16_t* row = query_row<uint16_t, D>(a, p, r * 16 + l16);
#pragma unroll
        for (int c = 0; c < C; ++c)
            q[r][c] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4h_t*>(row + 32 * c + 8 * lg));
        pos[r] = row_position(a, x, p, r * 16 + l16);
        m[r] = kNoMax;
        l[r] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[r][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int64_t kTile = (int64_t)D * kBlockTokens * 2;  // bytes of a block's keys of one head
    // This wavefront's two blocks of a unit.  The ids of 32 units lie in the lanes of a
    // register, -1 where a block is unmapped or behind the last one.
    auto first = [&](int u) { return p.b_lo + 2 * (u * W + wave); };
    auto read_ids = [&](int u) {
        const int b = first(u + lane / 2) + lane % 2;
        const int id = u + lane / 2 < p.u1 && b < p.b_hi ? p.table[b] : -1;
        return id >= 0 && id < a.num_blocks ? id : -1;
    };
    uint4 k[2][C], v[DT];
    const int k_at = (l16 & 3) * 16 + ((l16 >> 2) & 1) * 128 + lg * 256, v_at = l16 * 32 + (lg & 1) * 16;
    auto load_k = [&](int id0, int id1) {
        const uint8_t* from = a.kc + ((int64_t)max(l16 >> 3 ? id1 : id0, 0) * a.hkv + p.head) * kTile + k_at;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t) k[t][c] = ld16(from + c * 1024 + t * 64);
    };
    auto load_v = [&](int id0, int id1) {
        const uint8_t* from = a.vc + ((int64_t)max(lg >> 1 ? id1 : id0, 0) * a.hkv + p.head) * kTile + v_at;
#pragma unroll
        for (int t = 0; t < DT; ++t) v[t] = ld16(from + t * 512);
    };
    int ids = read_ids(p.u0);
    int id0 = __builtin_amdgcn_readlane(ids, 0), id1 = __builtin_amdgcn_readlane(ids, 1);
    if (id0 >= 0 || id1 >= 0) {
        load_k(id0, id1);
        load_v(id0, id1);
    }
    for (int u = p.u0; u < p.u1; ++u) {
        const int b0 = first(u), at = (u + 1 - p.u0) % 32;
        if (at == 0) ids = read_ids(u + 1);
        const int next0 = __builtin_amdgcn_readlane(ids, 2 * at), next1 = __builtin_amdgcn_readlane(ids, 2 * at + 1);
        const bool more = next0 >= 0 || next1 >= 0;
        if (id0 >= 0 || id1 >= 0) {
            const bool edge = (b0 + 2) * kBlockTokens - 1 > p.min_pos || id0 < 0 || id1 < 0;
            const bool ok = (lg >> 1 ? id1 : id0) >= 0;
            auto step = [&](auto is_edge) {
                step32<D, RT, decltype(is_edge)::value>(
                    p, lg, b0, ok, a.scale_log2, q, pos, m, l, o, [&](int t, int c) { return as_bf16x8(k[t][c]); },
                    [&]() { if (more) load_k(next0, next1); }, [&](int t) { return v[t]; });
            };
            if (edge) step(std::true_type{});
            else step(std::false_type{});
        } else if (more) {
            load_k(next0, next1);
        }
        if (more) load_v(next0, next1);
        id0 = next0;
        id1 = next1;
    }
    join_waves<uint16_t, D, RT, WHOLE, W>(a, p, m, l, o, smem);
}

// Few rows, fp32: fp32 products (v_mfma_f32_16x16x4_f32), a block of 16 keys at a time.
// Lane 16 lg + l16 takes the 16-byte chunks lg, lg + 4, ... of key l16; product i of a
// chunk multiplies its i-th dim.  A lane's 16 bytes of V^T are its keys 4 lg .. 4 lg + 3.
// Bound by the matrix units where there are several tiles, by memory with one.
template <int D, int RT, bool WHOLE = false, int W = kWaves>
__device__ void walk_flat_f32(const SharedArgs& a, const Index& x, const Piece& p, uint8_t* smem) {
    constexpr int DT = D / 16, C = D / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = own_lane(), l16 = lane % 16,
              lg = lane / 16;
    // Q as its operands: of one tile in registers, of more in LDS
    constexpr bool kInLds = RT > 1;
    f32x4_t q[kInLds ? 1 : C], o[RT][DT];
    f32x4_t* s_q = reinterpret_cast<f32x4_t*>(smem);
    float m[RT], l[RT];
    int pos[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float* row = query_row<float, D>(a, p, r * 16 + l16) + 4 * lg;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (!kInLds) q[c] = *reinterpret_cast<const f32x4u_t*>(row + 16 * c);
            else if (c % W == wave) s_q[(r * C + c) * kWave + lane] = *reinterpret_cast<const f32x4u_t*>(row + 16 * c);
        }
        pos[r] = row_position(a, x, p, r * 16 + l16);
        m[r] = kNoMax;
        l[r] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[r][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int64_t kTile = (int64_t)D * kBlockTokens * 4;
    const int blocks = p.u1 - p.u0;  // of this wavefront: one of every unit
    auto block = [&](int e) { return p.b_lo + (p.u0 + e) * W + wave; };
    // the ids of 64 of them in the lanes of a register, as in walk_flat
    auto read_ids = [&](int e) {
        const int b = block(e + lane), id = e + lane < blocks && b < p.b_hi ? p.table[b] : -1;
        return id >= 0 && id < a.num_blocks ? id : -1;
    };
    int ids = read_ids(0);
    f32x4_t k[C], v[DT];
    auto load_k = [&](int id) {
        const uint8_t* from = a.kc + ((int64_t)id * a.hkv + p.head) * kTile + l16 * 16 + lg * 256;
#pragma unroll
        for (int c = 0; c < C; ++c) k[c] = *reinterpret_cast<const f32x4_t*>(from + c * 1024);
    };
    auto load_v = [&](int id) {
        const uint8_t* from = a.vc + ((int64_t)id * a.hkv + p.head) * kTile + l16 * 64 + lg * 16;
#pragma unroll
        for (int t = 0; t < DT; ++t) v[t] = *reinterpret_cast<const f32x4_t*>(from + t * 1024);
    };
    int id = __builtin_amdgcn_readlane(ids, 0);
    if (id >= 0) {
        load_k(id);
        load_v(id);
    }
    if (kInLds) __syncthreads();
    for (int e = 0; e < blocks; ++e) {
        if ((e + 1) % kWave == 0) ids = read_ids(e + 1);
        const int next = __builtin_amdgcn_readlane(ids, (e + 1) % kWave);
        if (id >= 0) {
            const int key0 = block(e) * kBlockTokens + 4 * lg;
            const bool edge = block(e) * kBlockTokens + kBlockTokens - 1 > p.min_pos;
            // several chains of products: none waits for the one before it
            constexpr int kChains = RT > 1 ? 1 : 2;
            f32x4_t s[RT * kChains];
#pragma unroll
            for (int r = 0; r < RT * kChains; ++r) s[r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const f32x4_t y = kInLds ? s_q[(r * C + c) * kWave + lane] : q[c];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        f32x4_t& sum = s[r * kChains + i % kChains];
                        sum = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][i], y[i], sum, 0, 0, 0);
                    }
                }
            if (kChains > 1) s[0] += s[1];
            if (next >= 0) load_k(next);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + i > pos[r]) s[r][i] = -INFINITY;
                }
                float w[4] = {s[r][0], s[r][1], s[r][2], s[r][3]};
                weigh<4, DT>(w, a.scale_log2, m[r], l[r], o[r]);
                s[r] = f32x4_t{w[0], w[1], w[2], w[3]};
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + i >= p.S) v[t][i] = 0.f;
                }
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[r][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][i], s[r][i], o[r][t], 0, 0, 0);
            }
        } else if (next >= 0) {
            load_k(next);
        }
        if (next >= 0) load_v(next);
        id = next;
    }
    if (kInLds) __syncthreads();  // Q is used up
    join_waves<float, D, RT, WHOLE, W>(a, p, m, l, o, smem);
}

// Many rows, bf16: wavefront w has the rows' tiles w, w + 4, ...; the ring's stages hold two
// blocks each, K and then V.  While a step's scores become weights on the vector units,
// the next step's are on the matrix units, so that a wavefront keeps both at work.
template <int D, int RT>
__device__ void walk_tall(const SharedArgs& a, const Index& x, const Piece& p, uint8_t* smem) {
    constexpr int DT = D / 16, C = D / 32;
    constexpr int kTile = D * kBlockTokens * 2;  // bytes of a block's keys of one head
    constexpr int kStage = 4 * kTile, kRun = kTile / 1024;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = own_lane(), l16 = lane % 16,
              lg = lane / 16;
    bf16x8_t q[RT][C];
    f32x4_t o[RT][DT];
    float m[RT], l[RT];
    int pos[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row_at = (r * kWaves + wave) * 16 + l16;
        const uint16_t* row = query_row<uint16_t, D>(a, p, row_at);
#pragma unroll
        for (int c = 0; c < C; ++c)
            q[r][c] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4h_t*>(row + 32 * c + 8 * lg));
        pos[r] = row_position(a, x, p, row_at);
        m[r] = kNoMax;
        l[r] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[r][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int b_first = p.b_lo + p.u0 * kUnitBlocks, b_end = min(p.b_hi, p.b_lo + p.u1 * kUnitBlocks);
    const int steps = max(0, (b_end - b_first + 1) / 2);
    // The ids of 64 blocks lie in the lanes of a register, two runs of them in turn; -1
    // where a block is unmapped or behind the last one.  Each read is waited for where
    // it is made: left pending, the compiler would have to wait in every step, for the
    // ring's loads too.
    auto read_ids = [&](int from) {
        const int b = b_first + from + lane;
        const int id = b < b_end ? p.table[b] : -1;
        __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
        return id >= 0 && id < a.num_blocks ? id : -1;
    };
    int even = read_ids(0), odd = steps > 32 ? read_ids(64) : -1;
    auto id_of = [&](int at) { return __builtin_amdgcn_readlane(at & 64 ? odd : even, at & 63); };
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)smem;
    // wavefronts 0 and 1 fetch the K tiles of a step's two blocks, 2 and 3 the V tiles
    auto fetch = [&](int e) {
        const int id = max(0, id_of(2 * e + (wave & 1)));
        const uint8_t* from = (wave < 2 ? a.kc : a.vc) + ((int64_t)id * a.hkv + p.head) * kTile;
        dma16_run<kRun>(ring + (e % kStages) * kStage + wave * kTile, from, lane * 16);
    };
    // (K's reads take twice the cycles they would with the second block's keys 0-3 and 4-7
    // exchanged between the two products; putting the weights back in order before the
    // second contraction then costs more than LDS, a third busy, gains: 295 -> 304 us.)
    const int k_at = (l16 >> 3) * kTile + (l16 & 3) * 16 + ((l16 >> 2) & 1) * 128 + lg * 256;
    const int v_at = 2 * kTile + (lg >> 1) * kTile + l16 * 32 + (lg & 1) * 16;
    f32x4_t s[RT][2];
    uint4 k[C][2];
    auto read_k = [&](int e) {
        const uint8_t* stage = smem + (e % kStages) * kStage + k_at;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t) k[c][t] = ld16(stage + c * 1024 + t * 64);
    };
    auto products = [&]() {
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k[c][t]), q[r][c], s[r][t], 0, 0, 0);
    };
    // the loads of Q are done before the ring's are counted
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
#pragma unroll
    for (int e = 0; e < kStages - 1; ++e)
        if (e < steps) fetch(e);
    if (steps >= kStages - 1) wait_vmcnt<(kStages - 2) * kRun>();
    else wait_vmcnt<0>();
    lds_barrier();
    const bool works = wave * 16 < p.rows;  // a wavefront without rows fetches and waits
    if (works) {
        read_k(0);
        products();
    }
    for (int e = 0; e < steps; ++e) {
        // this wavefront's loads of stage e + 2 may be under way
        if (e + 2 < steps) wait_vmcnt<kRun>();
        else wait_vmcnt<0>();
        // behind it stage e + 1 is whole, and nobody reads stage e - 1 any more
        lds_barrier();
        // the run of ids before this step's is used up
        if (e % 32 == 0 && e > 0 && 2 * e + 64 < 2 * steps) (e & 32 ? even : odd) = read_ids(2 * e + 64);
        if (e + kStages - 1 < steps) fetch(e + kStages - 1);
        uint8_t* stage = smem + (e % kStages) * kStage;
        const int b0 = b_first + 2 * e, id0 = id_of(2 * e), id1 = id_of(2 * e + 1);
        if ((b0 + 2) * kBlockTokens - 1 > p.min_pos || id0 < 0 || id1 < 0) {
            // some row does not see some key, or a block is not mapped
            const int key0 = b0 * kBlockTokens + 8 * lg;
            const bool ok = (lg >> 1 ? id1 : id0) >= 0;
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    if (!ok || key0 + n > pos[r]) s[r][n / 4][n % 4] = -INFINITY;
            // what a slot without a key holds may be no number: it becomes zero in V
            if ((b0 + 2) * kBlockTokens > p.S || id0 < 0 || id1 < 0) {
                const int block = threadIdx.x / D, left = p.S - (b0 + block) * kBlockTokens;
                if (block < 2) {
                    uint4* v = reinterpret_cast<uint4*>(stage + (2 + block) * kTile + threadIdx.x % D * 32);
                    const bool mapped = (block ? id1 : id0) >= 0;
                    v[0] = first_keys(v[0], mapped ? left : 0);
                    v[1] = first_keys(v[1], mapped ? left - 8 : 0);
                }
                lds_barrier();
            }
        }
        if (!works) continue;
        read_k(e + 1);  // behind the last step: what lies there, for nothing
        // the weights' exponents; where one exceeds the slack its row's maximum is raised
        float t[RT][8];
        bool high = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = kNoMax;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                t[r][n] = fmaf(s[r][n / 4][n % 4], a.scale_log2, -m[r]);
                top = fmaxf(top, t[r][n]);
            }
            high |= top > kSlackLog2;
        }
        if (__any(high)) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float top = kNoMax;
#pragma unroll
                for (int n = 0; n < 8; ++n) top = fmaxf(top, s[r][n / 4][n % 4] * a.scale_log2);
                const float next = fmaxf(m[r], rows_max(top)), f = __builtin_amdgcn_exp2f(m[r] - next);
                m[r] = next;
                l[r] *= f;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[r][d] *= f;
#pragma unroll
                for (int n = 0; n < 8; ++n) t[r][n] = fmaf(s[r][n / 4][n % 4], a.scale_log2, -m[r]);
            }
        }
        uint4 v[DT];
#pragma unroll
        for (int d = 0; d < DT / 2; ++d) v[d] = ld16(stage + v_at + d * 512);
        // whoever has products to issue goes before the other wavefront of the SIMD
        // (309 GFLOP of 288 rows: 320 -> 312 us)
        __builtin_amdgcn_s_setprio(1);
        products();
        bf16x8_t w[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                t[r][n] = __builtin_amdgcn_exp2f(t[r][n]);
                sum += t[r][n];
            }
            l[r] += sum;
            w[r] = as_bf16x8(make_uint4(pack_bf16x2(t[r][0], t[r][1]), pack_bf16x2(t[r][2], t[r][3]),
                                        pack_bf16x2(t[r][4], t[r][5]), pack_bf16x2(t[r][6], t[r][7])));
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (d >= DT / 2) v[d] = ld16(stage + v_at + d * 512);
#pragma unroll
            for (int r = 0; r < RT; ++r)
                o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v[d]), w[r], o[r][d], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row_at = (r * kWaves + wave) * 16 + l16;
        const float sum = rows_sum(l[r]);
#pragma unroll
        for (int t = 0; t < DT; ++t) store_partial<D>(a, p, lg, row_at, t, o[r][t]);
        if (lg == 0 && row_at < p.rows) a.part_ml[p.slot_row + row_at] = make_float2(m[r], sum);
    }
    __syncthreads();  // the ring is free
}

template <typename T, int D>
constexpr int smem_bytes() {
    const int joined = kWaves * (D / 16) * 1024;  // or fp32's Q
    static_assert(sizeof(T) == 2 || flat_tiles(true, D) * 16 * D * 4 <= joined, "Q");
    const int ring = sizeof(T) == 2 ? kStages * 4 * D * kBlockTokens * 2 : 0;
    return joined > ring ? joined : ring;
}

template <typename T, int D, bool INLINE>
__global__ __launch_bounds__(kThreads, 2) void shared_walk(SharedArgs a, Index x) {
    __shared__ __attribute__((aligned(16))) uint8_t smem[smem_bytes<T, D>()];
    __shared__ Segment s_segments[INLINE ? kInlineSegs : 1];
    __shared__ Items s_items[INLINE ? kInlineSegs : 1];
    const Segment* segments = INLINE ? s_segments : a.segments;
    const Items* prefix_items = INLINE ? s_items : a.items;
    Share h;
    const int segs = a.num_groups + a.num_seqs;
    if constexpr (INLINE) {
        // the descriptor in LDS first, where the ring will be: one latency instead of one
        // for each array that another one's entry leads to
        int32_t* s_start = reinterpret_cast<int32_t*>(smem);
        int32_t* s_lens = s_start + kInlineSegs + 1;
        int32_t* s_groups = s_lens + kInlineSegs;
        int32_t* s_prefix = s_groups + kInlineSegs + 1;
        for (int i = threadIdx.x; i <= max(a.num_seqs, a.num_groups); i += kThreads) {
            // all four on their way before the first is waited for (places behind an
            // array's last entry take that again)
            const int seq = min(i, a.num_seqs), group = min(i, a.num_groups);
            const int start = x.q_start[seq], len = x.lens[min(i, a.num_seqs - 1)];
            const int begin = x.group_start[group], prefix = x.prefix[min(i, a.num_groups - 1)];
            s_start[seq] = start;
            s_lens[min(i, a.num_seqs - 1)] = len;
            s_groups[group] = begin;
            s_prefix[min(i, a.num_groups - 1)] = prefix;
        }
        __syncthreads();
        const Index y{x.tables, s_lens, s_start, s_groups, s_prefix};
        h = count_units<kThreads, int>(a, y, s_segments, s_items);
        describe_rows<INLINE>(a, y, s_segments, s_items, h.ua);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.share = h;  // for the pass that joins
        __syncthreads();
    } else {
        h = *a.share;
        describe_rows<INLINE>(a, x, a.segments, a.items, h.ua);
    }
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int na = same(h.na), b = blockIdx.x;
    const bool first = b < na;
    // Workgroups go round the eight XCDs.  Each XCD takes a run of the items, its workgroups
    // one after the other: the tiles of one part of the keys follow each other, so that
    // they are walked at the same time and the keys come out of the XCD's L2.
    const int xcd = b % 8, step = first ? na / 8 : 0;
    int item = first ? (int)((int64_t)same(h.items) * xcd / 8) + b / 8 : 0;
    const int items = first ? (int)((int64_t)same(h.items) * (xcd + 1) / 8) : 0;
    const int w = b - na, count = same(h.cb);
    int64_t u = 0, u_end = 0;
    if (!first) {
        if (w >= count) return;
        u = quotient(h.ub * w, count);
        u_end = quotient(h.ub * (w + 1), count);
    }
    while (first ? item < items : u < u_end) {
        const int64_t at = first ? item : h.ua + u;
        auto begin = [&](int k) { return first ? (int64_t)prefix_items[k].first : segments[k].unit0; };
        // the last segment that begins at or before it
        const int lo = find_last(begin, first ? 0 : a.num_groups, (first ? a.num_groups : segs) - 1, at);
        const Segment& g = segments[lo];
        const int real = same(units_of(a, g)), tiles = same(tiles_of(g, first ? a.tile_a : a.tile_b));
        const int tile_height = same(tile_rows(g, tiles));
        const int64_t local = at - begin(lo);
        int tile;
        int64_t slot;
        Piece p;
        if (first) {
            // item = (head * parts + part) * tiles + tile
            const uint32_t parts = same(prefix_items[lo].parts), e = same((int)local), row = e / (uint32_t)tiles;
            p.head = row / parts;
            const uint32_t part = row - p.head * parts;
            tile = e - row * tiles;
            p.u0 = (int)quotient((int64_t)real * part, parts);
            p.u1 = (int)quotient((int64_t)real * (part + 1), parts);
            slot = item;
            item += step;
        } else {
            const Cost c = cost_of(a, tile_height);
            const int each = c.extra + real * c.each, pair = same((int)quotient(local, each));
            p.head = (uint32_t)pair / (uint32_t)tiles;
            tile = pair - p.head * tiles;
            const int from = same((int)(local - (int64_t)pair * each)), to = same((int)min((int64_t)each, from + (u_end - u)));
            u += to - from;
            // the units that begin in this range
            p.u0 = (int)((uint32_t)(max(0, from - c.extra) + c.each - 1) / (uint32_t)c.each);
            p.u1 = (int)((uint32_t)(max(0, to - c.extra) + c.each - 1) / (uint32_t)c.each);
            if (p.u1 <= p.u0) continue;
            slot = same(g.pair0) + pair + w;
        }
        p.q0 = same(g.q0);
        p.row0 = tile * tile_height;
        p.rows = max(0, min(tile_height, same(g.rows) - p.row0));
        p.b_lo = same(g.b_lo);
        p.b_hi = same(g.b_hi);
        p.S = same(g.S);
        p.table = x.tables + (int64_t)same(g.table) * a.max_blocks;
        p.prefix = first;
        p.pos0 = same(g.pos0);
        p.masked = first && p.pos0;
        p.min_pos = first ? (p.masked ? -1 : INT32_MAX) : p.pos0 + p.row0 / a.group;
        if (slot >= (first ? a.slots_a : a.slots_b) || p.rows == 0) continue;
        p.slot_row = first ? slot * a.tile_a : a.slots_a * a.tile_a + slot * a.tile_b;
        // keys that none of the tile's rows sees
        if (!first) {
            const int seen = p.pos0 + (p.row0 + p.rows - 1) / a.group + 1 - p.b_lo * kBlockTokens;
            p.u1 = max(p.u0, min(p.u1, (max(0, seen) + (kBlockTokens << a.unit_shift) - 1) / kBlockTokens >> a.unit_shift));
        }
        const int tiles16 = (p.rows + 15) / 16;
        if constexpr (sizeof(T) == 4) {
            if (tiles16 == 1) walk_flat_f32<D, 1>(a, x, p, smem);
            else if (tiles16 == 2) walk_flat_f32<D, 2>(a, x, p, smem);
            else if (tiles16 == 3) walk_flat_f32<D, 3>(a, x, p, smem);
            else walk_flat_f32<D, flat_tiles(true, D)>(a, x, p, smem);
        } else {
            constexpr int RT = tall_tiles(D);
            if (tiles16 == 1) walk_flat<D>(a, x, p, smem);
            else if (tiles16 <= 4) walk_tall<D, 1>(a, x, p, smem);
            else if (tiles16 <= 8) walk_tall<D, 2>(a, x, p, smem);
            else walk_tall<D, RT>(a, x, p, smem);
        }
    }
}

// Few and short requests: a workgroup walks all that 16 rows of a request and head see, the
// prefix as the request's own table names it, with nothing to divide before and nothing to
// join behind it; eight wavefronts in bf16 where every tile has a compute unit of its own.
// Bound by the chain of lengths, block ids and keys, then by 0.6 us per unit of bf16, 1.0
// of fp32, and with many requests by the keys, prefixes out of L2.  Replayed, divided and
// like this, head dim 128: 8 requests of a row and 128 keys 10.4 and 4.2 us, of 2000 keys,
// 1000 of them common, 16.2 and 14.6 (of 3000 19.4 and 19.7); head dim 64, 2 requests of 4000
// keys 13.1 and 12.3.  fp32, 8 of 256 keys 14.2 and 9.1; two of 440 keys, half of them common,
// 11.8 and 12.8, three quarters common 13.5 and 12.8; two of 512 13.8 and 15.4, but eight of nine
// rows and 520 keys 29.8 and 16.4: with more tiles the division takes longer, which the limit
// on keys alone leaves out; head dim 64, two of 700 keys 12.4 and 11.8.  All tiles' keys together: 64 requests of eight heads, 2000 keys,
// 250 of them common, 94 and 83, 1750 common 25.5 and 27.4; head dim 64, 2200 keys 43 and 34,
// 20 and 19, 3000 keys 52 and 48, 21 and 25.  With several tiles in bf16, which read the same
// keys again: 20 requests of nine rows and 2000 keys 35 and 30, but more tiles than fit at
// once, 64 such requests, 256 keys 31 and 28, 512 keys 37 and 52.
//
// Workgroup (head, request, tile).
template <typename T, int D, int W>
__global__ __launch_bounds__(W * kWave, 2) void shared_short(SharedArgs a, Index x) {
    __shared__ __attribute__((aligned(16))) uint8_t smem[W * (D / 16) * 1024];
    const int i = blockIdx.y;
    const int q0 = clamp_to(x.q_start[i], 0, a.total_q), n = clamp_to(x.q_start[i + 1], q0, a.total_q) - q0;
    Piece p{};
    p.q0 = q0;
    p.head = blockIdx.x;
    p.S = clamped_len(a, x, i);
    p.b_hi = (p.S + kBlockTokens - 1) / kBlockTokens;
    p.pos0 = p.S - n;
    p.table = x.tables + (int64_t)i * a.max_blocks;
    const int rows = n * a.group;
    for (p.row0 = blockIdx.z * 16; p.row0 < rows; p.row0 += gridDim.z * 16) {
        p.rows = min(16, rows - p.row0);
        p.min_pos = p.pos0 + p.row0 / a.group;
        const int seen = p.pos0 + (p.row0 + p.rows - 1) / a.group + 1;
        constexpr int kUnit = W * kBlockTokens * (sizeof(T) == 2 ? 2 : 1);
        p.u1 = (max(0, seen) + kUnit - 1) / kUnit;
        if constexpr (sizeof(T) == 2) walk_flat<D, true, W>(a, x, p, smem);
        else walk_flat_f32<D, 1, true, W>(a, x, p, smem);
    }
}

// A row's parts joined: kLanes lanes for the dims of a (row, query head), SPLIT groups of
// them for its pieces, a workgroup per row and run of heads.
template <typename T, int D, int SPLIT>
__global__ __launch_bounds__(kThreads) void shared_join(SharedArgs a) {
    constexpr int kLanes = D / 4, kGroups = kThreads / kLanes, kHeads = kGroups / SPLIT, kBatch = 8;
    __shared__ f32x4_t s_acc[SPLIT > 1 ? kThreads : 1];
    __shared__ float2 s_ml[SPLIT > 1 ? kGroups : 1];
    const int row = blockIdx.x, tid = threadIdx.x;
    const RowParts r = a.rows[row];
    const Share sh = *a.share;
    if (r.e0 < 0) return;
    const int unit = tid / kLanes, part_of = unit % SPLIT, d = tid % kLanes * 4;
    const int h = min((int)blockIdx.y * kHeads + unit / SPLIT, a.hq - 1);
    const int head = h / a.group, in_group = h % a.group;
    // pieces of the two pairs, one after the other: the first one's row among the partial
    // rows, and the distance to the next one's
    int pieces[2] = {0, 0};
    int64_t at[2] = {0, 0}, next_at[2] = {0, a.tile_b};
    if (r.parts > 0) {
        const int e = r.prefix_e0 + in_group, tile = r.prefix_tiles > 1 ? (uint32_t)e / (uint32_t)r.prefix_height : 0;
        const int64_t slot = r.item0 + (int64_t)head * r.parts * r.prefix_tiles + tile;
        pieces[0] = slot + (int64_t)(r.parts - 1) * r.prefix_tiles < a.slots_a ? r.parts : 0;
        at[0] = slot * a.tile_a + e - tile * r.prefix_height;
        next_at[0] = (int64_t)r.prefix_tiles * a.tile_a;
    }
    if (r.real > 0) {
        const int e = r.e0 + in_group, tile = r.tiles > 1 ? (uint32_t)e / (uint32_t)r.height : 0, pair = head * r.tiles + tile;
        const Cost c = cost_of(a, r.height);
        const int64_t u0 = r.unit0 + (int64_t)pair * (c.extra + r.real * c.each) + c.extra;  // where its first unit begins
        // workgroup w owns units [ub w / cb, ub (w + 1) / cb)
        const int w0 = (int)quotient((u0 + 1) * sh.cb - 1, sh.ub);
        const int w1 = (int)quotient((u0 + (r.real - 1) * c.each + 1) * sh.cb - 1, sh.ub);
        const int64_t slot = r.pair0 + pair + w0;
        pieces[1] = (int)max((int64_t)0, min((int64_t)(w1 - w0 + 1), a.slots_b - slot));
        at[1] = a.slots_a * a.tile_a + slot * a.tile_b + e - tile * r.height;
    }
    float top = kNoMax, sum = 0.f;
    f32x4_t acc{0.f, 0.f, 0.f, 0.f};
    const int all = pieces[0] + pieces[1];
    for (int base = part_of; base < all; base += SPLIT * kBatch) {
        float2 ml[kBatch];
        f32x4_t o[kBatch];
#pragma unroll
        for (int z = 0; z < kBatch; ++z) {
            const int e = min(base + z * SPLIT, all - 1), k = e < pieces[0] ? 0 : 1;
            const int64_t from = at[k] + (k ? e - pieces[0] : e) * next_at[k];
            ml[z] = a.part_ml[from];
            o[z] = *reinterpret_cast<const f32x4_t*>(a.part_o + from * D + d);
        }
#pragma unroll
        for (int z = 0; z < kBatch; ++z) {
            if (base + z * SPLIT >= all) break;
            const float next = fmaxf(top, ml[z].x);
            const float f0 = exp2f(top - next), f1 = exp2f(ml[z].x - next);
            top = next;
            sum = fmaf(sum, f0, ml[z].y * f1);
            acc = acc * f0 + o[z] * f1;
        }
    }
    if constexpr (SPLIT > 1) {
        s_acc[tid] = acc;
        if (d == 0) s_ml[unit] = make_float2(top, sum);
        __syncthreads();
        if (part_of != 0) return;
#pragma unroll
        for (int z = 1; z < SPLIT; ++z) {
            const float2 ml = s_ml[unit + z];
            const float next = fmaxf(top, ml.x);
            const float f0 = exp2f(top - next), f1 = exp2f(ml.x - next);
            top = next;
            sum = fmaf(sum, f0, ml.y * f1);
            acc = acc * f0 + s_acc[tid + z * kLanes] * f1;
        }
    }
    if ((int)blockIdx.y * kHeads + unit / SPLIT >= a.hq) return;
    store_out<T>(a, row, h, D, d, top, sum, acc);
}

// ------------------------------------------------------------------ host side

struct SharedPlan {
    int nwg, tile_a, tile_b;
    int64_t slots_a, slots_b, segs;
    bool inlined, weighted;
    int short_tiles, short_waves;  // row tiles of a request where all are short (shared_short), or 0
    int split;  // groups of threads that share a row's pieces in the pass that joins
    size_t o_bytes, ml_bytes, total;
};

// Row tiles and partial results.  A tile holds at most the rows that its segment may
// have: few of them (flat) or 64 tall_tiles.
int plan_shared(const verify_attn_params* p, int32_t total_q, int32_t max_q_len, int32_t max_seq_len, int32_t num_groups,
                int32_t max_prefix_len, SharedPlan& s) {
    const int group = p->num_q_heads / p->num_kv_heads, D = p->head_dim;
    const bool f32 = p->dtype == VERIFY_F32;
    auto tile = [&](int64_t rows) {
        const int flat = 16 * flat_tiles(f32, D);
        if (!f32 && rows > flat) return 64 * tall_tiles(D);
        return rows <= 16 ? 16 : rows <= 32 ? 32 : flat;
    };
    const int64_t rows = (int64_t)total_q * group;
    s.nwg = 2 * device_cus() / 8 * 8;
    s.tile_a = tile(rows);
    const int64_t own_rows = std::min<int64_t>(rows, (int64_t)max_q_len * group);
    s.tile_b = tile(own_rows);
    s.weighted = own_rows > 128 && s.tile_b > 128;
    // (rounded up, so that fewer rows in smaller tiles never need more)
    const int64_t keys = std::min<int64_t>(max_seq_len, (int64_t)p->max_blocks_per_seq * kBlockTokens);
    const int64_t tiles16 = (own_rows + 15) / 16, pairs16 = tiles16 * p->num_seqs * p->num_kv_heads;
    const int64_t share = short_share(f32, D) / (!f32 && tiles16 > 1 && pairs16 > s.nwg ? 2 : 1);
    s.short_tiles = keys <= short_keys(f32, D) && pairs16 * keys <= s.nwg * share && p->num_seqs <= 65535 ? (int)tiles16 : 0;
    if (s.short_tiles) {
        s.short_waves = !f32 && 2 * pairs16 <= s.nwg ? 8 : kWaves;
        s.total = 0;
        return VERIFY_OK;
    }
    const int64_t pairs_a = ((rows + s.tile_a - 1) / s.tile_a + num_groups) * p->num_kv_heads;
    const int64_t pairs_b = ((rows + s.tile_b - 1) / s.tile_b + p->num_seqs) * p->num_kv_heads;
    if (pairs_a + pairs_b >= (1 << 30)) return VERIFY_EUNSUPPORTED;
    s.slots_a = pairs_a + 4 * s.nwg;
    s.slots_b = pairs_b + s.nwg;
    s.segs = (int64_t)num_groups + p->num_seqs;
    const int64_t part_rows = s.slots_a * s.tile_a + s.slots_b * s.tile_b;
    s.o_bytes = (size_t)part_rows * D * 4;
    s.ml_bytes = align_up((size_t)part_rows * 8, 16);
    s.total = s.o_bytes + s.ml_bytes + (size_t)total_q * sizeof(RowParts) + sizeof(Share) +
              (size_t)s.segs * sizeof(Segment) + (size_t)num_groups * sizeof(Items);
    // the units of all pairs in 32 bits: then every workgroup can count them itself
    const int64_t most_units = std::min<int64_t>(std::max(max_seq_len, max_prefix_len), (int64_t)p->max_blocks_per_seq * kBlockTokens) /
                                   (kBlockTokens << unit_shift(f32)) + 2 + kPairUnits;  // times kMostEach
    s.inlined = s.segs <= kInlineSegs && (pairs_a + pairs_b) * most_units * kMostEach < (1LL << 31) && s.slots_a < (1LL << 30);

    s.split = s.nwg >= 24 * pairs_a ? 8 : s.nwg >= 8 * pairs_a ? 4 : 1;
    return VERIFY_OK;
}

int check_shared(const verify_attn_params* p, int32_t total_q, int32_t max_q_len, int32_t max_seq_len, int32_t num_groups,
                 int32_t max_prefix_len) {
    const int rc = validate(p, total_q, max_q_len, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    if (num_groups < 0 || max_prefix_len < 0) return VERIFY_EINVAL;
    if (p->sliding_window > 0 || p->kv_split_blocks > 0) return VERIFY_EUNSUPPORTED;
    if (num_groups > 65535) return VERIFY_EUNSUPPORTED;
    const int64_t group = p->num_q_heads / p->num_kv_heads;
    if ((int64_t)total_q * group >= (1 << 30)) return VERIFY_EUNSUPPORTED;
    // the launch that joins: fewer than 2^32 threads in x, 65536 workgroups in y
    if (total_q >= (1 << 24) || p->num_q_heads > 65535) return VERIFY_EUNSUPPORTED;
    if (p->max_blocks_per_seq > (1 << 26)) return VERIFY_EUNSUPPORTED;
    return VERIFY_OK;
}

// Nothing to share: the call is verify_attention.
bool is_plain(const verify_attn_params* p, int32_t num_groups, int32_t max_prefix_len) {
    return num_groups == 0 || max_prefix_len < kBlockTokens || p->num_blocks == 0;
}

template <typename T, int D>
void launch_shared(const SharedArgs& a, const Index& x, const SharedPlan& plan, hipStream_t stream) {
    if (plan.short_tiles) {
        // 65535 in z at most: a workgroup takes every gridDim.z-th tile
        const dim3 grid(a.hkv, a.num_seqs, std::min(plan.short_tiles, 65535));
        if constexpr (sizeof(T) == 2) {
            if (plan.short_waves == 8) {
                hipLaunchKernelGGL((shared_short<T, D, 8>), grid, dim3(8 * kWave), 0, stream, a, x);
                return;
            }
        }
        hipLaunchKernelGGL((shared_short<T, D, kWaves>), grid, dim3(kThreads), 0, stream, a, x);
        return;
    }
    const int split = plan.split;
    if (plan.inlined) {
        hipLaunchKernelGGL((shared_walk<T, D, true>), dim3(a.nwg), dim3(kThreads), 0, stream, a, x);
    } else {
        hipLaunchKernelGGL(shared_schedule, dim3(1), dim3(1024), 0, stream, a, x);
        hipLaunchKernelGGL((shared_walk<T, D, false>), dim3(a.nwg), dim3(kThreads), 0, stream, a, x);
    }
    auto join = [&](auto n) {
        constexpr int kHeads = kThreads / (D / 4) / decltype(n)::value;
        hipLaunchKernelGGL((shared_join<T, D, decltype(n)::value>), dim3(a.total_q, (a.hq + kHeads - 1) / kHeads),
                           dim3(kThreads), 0, stream, a);
    };
    if (split == 8) join(std::integral_constant<int, 8>{});
    else if (split == 4) join(std::integral_constant<int, 4>{});
    else join(std::integral_constant<int, 1>{});
}

// two workgroups per compute unit
static_assert(sizeof(Segment) == 48 && smem_bytes<uint16_t, 128>() + (48 + 8) * kInlineSegs + 1024 <= 80 * 1024 &&
              sizeof(Share) % 16 == 0, "LDS and workspace");

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_attention_shared_workspace_size(const verify_attn_params* params, int32_t total_q,
                                                      int32_t max_q_len, int32_t max_seq_len, int32_t num_groups,
                                                      int32_t max_prefix_len, size_t* bytes) {
    int rc = check_shared(params, total_q, max_q_len, max_seq_len, num_groups, max_prefix_len);
    if (rc != VERIFY_OK) return rc;
    if (!bytes) return VERIFY_EINVAL;
    *bytes = 0;
    if (params->num_seqs == 0 || total_q == 0) return VERIFY_OK;
    if (is_plain(params, num_groups, max_prefix_len))
        return verify_attention_workspace_size(params, total_q, max_q_len, max_seq_len, bytes);
    SharedPlan s{};
    rc = plan_shared(params, total_q, max_q_len, max_seq_len, num_groups, max_prefix_len, s);
    if (rc == VERIFY_OK) *bytes = s.total;
    return rc;
}

extern "C" int verify_attention_shared(const verify_attn_params* params, int32_t total_q, int32_t max_q_len,
                                       int32_t max_seq_len, int32_t num_groups, int32_t max_prefix_len,
                                       const void* q, const void* k_cache, const void* v_cache,
                                       const int32_t* block_tables, const int32_t* seq_lens, const int32_t* q_start,
                                       const int32_t* group_start, const int32_t* prefix_lens, const float* sinks,
                                       void* out, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    int rc = check_shared(params, total_q, max_q_len, max_seq_len, num_groups, max_prefix_len);
    if (rc != VERIFY_OK) return rc;
    if (is_plain(params, num_groups, max_prefix_len))
        return verify_attention(params, total_q, max_q_len, max_seq_len, q, k_cache, v_cache, block_tables, seq_lens,
                                q_start, sinks, out, workspace, workspace_bytes, stream);
    if (params->num_seqs == 0 || total_q == 0) return VERIFY_OK;
    if (!q || !k_cache || !v_cache || !block_tables || !seq_lens || !q_start || !group_start || !prefix_lens || !out)
        return VERIFY_EINVAL;
    if (((uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)workspace) & 15) return VERIFY_EINVAL;
    SharedPlan s{};
    rc = plan_shared(params, total_q, max_q_len, max_seq_len, num_groups, max_prefix_len, s);
    if (rc != VERIFY_OK) return rc;
    if (s.total > 0 && (!workspace || workspace_bytes < s.total)) return VERIFY_EWORKSPACE;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    SharedArgs a{};
    a.q = q;
    a.kc = static_cast<const uint8_t*>(k_cache);
    a.vc = static_cast<const uint8_t*>(v_cache);
    a.sinks = sinks;
    a.out = out;
    a.part_o = reinterpret_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(ws + s.o_bytes);
    a.rows = reinterpret_cast<RowParts*>(ws + s.o_bytes + s.ml_bytes);
    a.share = reinterpret_cast<Share*>(a.rows + total_q);
    a.segments = reinterpret_cast<Segment*>(a.share + 1);
    a.items = reinterpret_cast<Items*>(a.segments + s.segs);
    a.num_seqs = params->num_seqs;
    a.num_groups = num_groups;
    a.hq = params->num_q_heads;
    a.hkv = params->num_kv_heads;
    a.group = a.hq / a.hkv;
    a.max_blocks = params->max_blocks_per_seq;
    a.num_blocks = params->num_blocks;
    a.max_seq_len = max_seq_len;
    a.max_prefix = max_prefix_len;
    a.total_q = total_q;
    a.nwg = s.nwg;
    a.tile_a = s.tile_a;
    a.tile_b = s.tile_b;
    a.weighted = s.weighted;
    a.unit_shift = unit_shift(params->dtype == VERIFY_F32);
    a.slots_a = s.slots_a;
    a.slots_b = s.slots_b;
    const float scale = params->scale > 0.f ? params->scale : 1.f / sqrtf((float)params->head_dim);
    a.scale_log2 = scale * kLog2e;
    const Index x{block_tables, seq_lens, q_start, group_start, prefix_lens};
    if (params->dtype == VERIFY_BF16)
        params->head_dim == 128 ? launch_shared<uint16_t, 128>(a, x, s, stream)
                                : launch_shared<uint16_t, 64>(a, x, s, stream);
    else
        params->head_dim == 128 ? launch_shared<float, 128>(a, x, s, stream)
                                : launch_shared<float, 64>(a, x, s, stream);
    return check_launch();
}
