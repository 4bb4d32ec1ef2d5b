// verify_evict.hip -- the keys that a bounded cache keeps, and their moves.
//
// The plan.  For each (request, KV head): the c-th largest of the S slots' sort keys
// by a radix select (digits of 11, 11 and 10 bits, histograms in LDS), then the kept
// slots in slot order, the holes among the first c and the kept slots behind them.  A
// slot's sort key is one 32-bit word: the order key of its weight, above all of them
// 0xffffffff for what is always kept, 0 for what never is.  At least c keys are not 0
// (every slot below c has one), so a key of 0 counts nowhere.
//   evict_plan    caches of up to 16384 slots: one workgroup, one launch, the keys in
//                 registers, 4, 8 or 16 per thread, from the first pass to the last (one
//                 request of 1024 slots, eight heads: 11.7 us with 16, 6.3 with 4;
//                 of 8192: 12.3 with 16, 9.6 with 8);
//   evict_hist (three launches), evict_lists, evict_join
//                 longer caches: a workgroup per chunk of them, the sort keys, histograms
//                 and lists in the workspace between the launches (a single workgroup
//                 took 543 us for 131072 slots; the five 46 when each read the table,
//                 the weights and the ordinals again, in chunks of 16384 slots; 30 now).
// What bounds it: a cache's workgroup, half vector instructions and half waits (32 caches
// to 16384 slots: the vector units are active 51 % of the time that a compute unit has
// one), and the launches of a long cache, each 1 to 3 us of work.  What it reads is 8
// bytes per slot, in pieces of 64 contiguous bytes; four lanes take a block's four
// quarters, so that a load touches 16 lines (a block per lane: 64, and the keys' arrival
// took 9 us of a plan of 16384's 40).
//
// The moves.
//   kv_compact    one wavefront per 16-slot block that keys move into.
#include "common.h"

namespace averify {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
// Slots of a thread, and of a workgroup: all of a cache in one, or a chunk of a longer
// one (131072 slots, eight heads: 46 us in chunks of 16 per thread, 36 of 8, 39 of 4).
constexpr int kSlots = 16, kAlone = kPlanThreads * kSlots;
constexpr int kPart = 8, kChunk = kPlanThreads * kPart;
constexpr int kDigitBits = 11;
constexpr int kBins = 1 << kDigitBits;
constexpr int kMaxChunks = 2048;                // of a request
constexpr uint32_t kAlways = 0xffffffffu;
typedef int32_t i32x4u_t __attribute__((ext_vector_type(4), aligned(4)));

struct PlanArgs {
    const float* key_weights;
    const int32_t* key_order;
    const int32_t* block_tables;
    const int32_t* seq_lens;
    const int32_t* num_tokens;
    int32_t* source;
    int32_t* new_lens;
    // long caches:
    uint4* keys;      // [pairs][chunks] sort keys, see stored_keys
    int32_t* hist;    // [2][pairs][hists][kBins]: the chunks', and their sum where evict_sum forms it
    uint16_t* lists;  // [pairs][chunks][kChunk]: holes from the front, movers from the back
    int2* counts;     // [pairs][chunks] holes and movers
    uint2* state;     // [pairs][2] digits found and keys still needed, after one and two passes
    int64_t pairs;
    int hkv, chunks, hists, max_blocks, num_blocks, max_seq_len, max_keys, keep_first, keep_recent;
};

struct PlanGeom {
    int i, g, S, c;
    int64_t pair, recent;  // ordinals from `recent` on are always kept
};

__device__ __forceinline__ PlanGeom plan_geom(const PlanArgs& a, int g, int i) {
    PlanGeom p;
    p.i = i;
    p.g = g;
    p.S = (int)max((int64_t)0, min((int64_t)a.seq_lens[i], min((int64_t)a.max_seq_len, (int64_t)a.max_blocks * kBlockTokens)));
    p.c = min(p.S, a.max_keys);
    p.pair = (int64_t)i * a.hkv + g;
    p.recent = (int64_t)(a.num_tokens ? a.num_tokens[i] : p.S) - a.keep_recent;
    return p;
}

// First slot of this thread's quarter k of a chunk: wavefront, quarter, lane in order.
template <int N>
__device__ __forceinline__ int slot_of(int chunk, int k) {
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    return (chunk * kPlanWaves + wv) * (kWave * N) + (16 * k + lane / 4) * kBlockTokens + lane % 4 * 4;
}

// Sort keys of this thread's slots: key[4 k + e] that of slot_of(k) + e.
template <int N>
__device__ __forceinline__ void load_keys(const PlanArgs& a, const PlanGeom& p, int chunk, uint32_t (&key)[N]) {
    const int32_t* table = a.block_tables + (int64_t)p.i * a.max_blocks;
    const int blocks = (p.S + kBlockTokens - 1) / kBlockTokens;
    int id[N / 4];
    float4 w[N / 4];
    int4 o[N / 4];
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const int b = slot_of<N>(chunk, k) / kBlockTokens;
        id[k] = b < blocks ? table[b] : -1;
    }
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const bool mapped = id[k] >= 0 && id[k] < a.num_blocks;
        const int64_t at = ((int64_t)(mapped ? id[k] : 0) * a.hkv + p.g) * kBlockTokens + threadIdx.x % 4 * 4;
        if (!mapped) continue;
        w[k] = *reinterpret_cast<const float4*>(a.key_weights + at);
        if (a.key_order) o[k] = *reinterpret_cast<const int4*>(a.key_order + at);
    }
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const bool mapped = id[k] >= 0 && id[k] < a.num_blocks;
        const int s0 = slot_of<N>(chunk, k);
        const float wk[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        const int ok[4] = {o[k].x, o[k].y, o[k].z, o[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int s = s0 + e, ord = a.key_order ? ok[e] : s;
            uint32_t v = min(order_key(__float_as_uint(wk[e])), kAlways - 1);
            if (ord < a.keep_first || ord >= p.recent) v = kAlways;
            if (!mapped) v = s < p.c ? kAlways : 0u;
            key[4 * k + e] = s < p.S ? v : 0u;
        }
    }
}

// Inclusive prefix sum over the wavefront.
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// Lanes below this one whose bit of `mask` is set.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// A pass of the select: the digits found so far are in prefix, under the mask known.
struct Digits {
    uint32_t prefix, known;
    int need;  // of the keys that share them, this many are among the c largest
    __device__ uint32_t mask(int pass) const { return pass == 0 ? 0xffe00000u : pass == 1 ? 0x001ffc00u : 0x000003ffu; }
    __device__ int shift(int pass) const { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
};

// Adds the thread's keys that share the digits to the histogram of the next one.  The
// lanes that agree with the first of them go as one addition: weights that are equal
// (zeros, what is always kept) would otherwise wait for each other.
template <int N>
__device__ __forceinline__ void add_keys(const Digits& d, int pass, const uint32_t (&key)[N], int* hist) {
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const bool in = key[e] != 0 && (key[e] & d.known) == d.prefix;
        const uint64_t mask = __ballot(in);
        if (mask == 0) continue;
        const int bin = (int)((key[e] & d.mask(pass)) >> d.shift(pass));
        const int leader = __builtin_ctzll(mask);
        const bool same = in && bin == __builtin_amdgcn_readlane(bin, leader);
        const uint64_t agree = __ballot(same);
        if (lane == leader) atomicAdd(&hist[bin], __popcll(agree));
        if (in && !same) atomicAdd(&hist[bin], 1);
    }
}

struct PlanShared {
    int hist[kBins];
    int sums[kPlanWaves];
    int digit, above, count;
};

// Sum of sh.sums over the wavefronts before this one; over all of them in `total`.
__device__ __forceinline__ int sums_before(const PlanShared& sh, int& total) {
    const int lane = threadIdx.x & (kWave - 1);
    const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int x = wave_scan(lane < kPlanWaves ? sh.sums[lane] : 0);
    total = __builtin_amdgcn_readlane(x, kPlanWaves - 1);
    return wv > 0 ? __builtin_amdgcn_readlane(x, wv - 1) : 0;
}

__device__ __forceinline__ void clear_hist(PlanShared& sh) {
    for (int e = threadIdx.x; e < kBins; e += kPlanThreads) sh.hist[e] = 0;
    __syncthreads();
}

// The digit of the c-th largest key, from the whole histogram (every thread's
// additions done), added to d.  Returns the keys that share all digits now.
__device__ __forceinline__ int find_digit(PlanShared& sh, Digits& d, int pass) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    __syncthreads();
    // two bins per thread, the highest first
    const int top = kBins - 1 - 2 * tid;
    const int h1 = sh.hist[top], h0 = sh.hist[top - 1];
    const int x = wave_scan(h1 + h0);
    if (lane == kWave - 1) sh.sums[wv] = x;
    __syncthreads();
    int all;
    const int above = sums_before(sh, all) + x - h1 - h0;
    const bool hi = above < d.need && d.need <= above + h1;
    const bool lo = above + h1 < d.need && d.need <= above + h1 + h0;
    if (hi || lo) {
        sh.digit = hi ? top : top - 1;
        sh.above = hi ? above : above + h1;
        sh.count = hi ? h1 : h0;
    }
    __syncthreads();
    d.prefix |= (uint32_t)sh.digit << d.shift(pass);
    d.known |= d.mask(pass);
    d.need -= sh.above;
    return sh.count;
}

// Which of the thread's keys are kept: those above the c-th largest, and of those
// equal to it the first d.need in slot order, of `count` in all and `before` in
// earlier chunks.
template <int N>
__device__ __forceinline__ uint32_t kept_bits(PlanShared& sh, const Digits& d, const uint32_t (&key)[N], int count,
                                              int before) {
    uint32_t kept = 0, equal = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        kept |= (uint32_t)(key[e] > d.prefix) << e;
        equal |= (uint32_t)(key[e] == d.prefix) << e;
    }
    if (count == d.need) return kept | equal;
    // ranks among the equal ones: wavefronts, quarters, lanes, elements in order
    int rank[N / 4], total = 0;
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        rank[k] = total;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t m = __ballot((equal >> (4 * k + e)) & 1u);
            rank[k] += lanes_below(m);
            total += __popcll(m);
        }
    }
    const int wv = threadIdx.x / kWave;
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) sh.sums[wv] = total;
    __syncthreads();
    int all;
    before += sums_before(sh, all);
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        int r = before + rank[k];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if ((equal >> (4 * k + e)) & 1u) kept |= (uint32_t)(r++ < d.need) << (4 * k + e);
    }
    return kept;
}

// Writes the plan of the kept slots that stay, and lists the holes below c and the
// kept slots from c on in slot order: hole(n, slot), mover(n, slot) for the n-th of
// each.  Returns their numbers.
template <int N, typename Hole, typename Mover>
__device__ __forceinline__ int2 list_slots(PlanShared& sh, const PlanGeom& p, int chunk, uint32_t kept, int32_t* source,
                                           Hole hole, Mover mover) {
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    uint32_t front = 0, inside = 0;
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        const int s0 = slot_of<N>(chunk, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            front |= (uint32_t)(s0 + e < p.c) << (4 * k + e);
            inside |= (uint32_t)(s0 + e < p.S) << (4 * k + e);
        }
        // holes are written over after a barrier, by whoever fills them
        const int four = (front >> (4 * k)) & 0xf;
        if (four == 0xf) {
            *reinterpret_cast<i32x4u_t*>(source + s0) = i32x4u_t{s0, s0 + 1, s0 + 2, s0 + 3};
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if ((four >> e) & 1) source[s0 + e] = s0 + e;
        }
    }
    const uint32_t bits[2] = {front & ~kept, inside & kept & ~front};
    int rank[2][N / 4], total[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const bool some = __any(bits[j] != 0);
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            rank[j][k] = total[j];
            if (!some) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint64_t m = __ballot((bits[j] >> (4 * k + e)) & 1u);
                rank[j][k] += lanes_below(m);
                total[j] += __popcll(m);
            }
        }
    }
    __syncthreads();
    // both in one word: a chunk has 2^14 slots
    if (lane == 0) sh.sums[wv] = total[0] | total[1] << 16;
    __syncthreads();
    int all;
    const int before = sums_before(sh, all);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (total[j] == 0) continue;
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            const int s0 = slot_of<N>(chunk, k);
            int n = (j == 0 ? before & 0xffff : before >> 16) + rank[j][k];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((bits[j] >> (4 * k + e)) & 1u) {
                    if (j == 0) hole(n++, s0 + e);
                    else mover(n++, s0 + e);
                }
        }
    }
    return make_int2(all & 0xffff, all >> 16);
}

// What a plan needs whoever is kept; true where that is all of it.
__device__ __forceinline__ bool plan_ends(const PlanArgs& a, const PlanGeom& p, int32_t* source) {
    if (p.g == 0 && threadIdx.x == 0) a.new_lens[p.i] = p.c;
    for (int d = p.c + threadIdx.x; d < a.max_keys; d += kPlanThreads) source[d] = -1;
    if (p.S != p.c) return false;
    for (int d = threadIdx.x; d < p.c; d += kPlanThreads) source[d] = d;
    return true;
}

// Grid (requests, KV heads), caches of up to N slots per thread.  Workgroups go round the
// eight XCDs: where the requests are a multiple of eight, a request's heads meet in one,
// whose L2 then serves the lines that hold two heads' slots (32 requests of 16384 slots,
// eight heads: 24 us with the heads first, 20; of 4096: 9.9 and 8.4).
template <int N>
__global__ __launch_bounds__(kPlanThreads) void evict_plan(PlanArgs a) {
    __shared__ PlanShared sh;
    __shared__ uint16_t s_hole[kPlanThreads * N / 2], s_mover[kPlanThreads * N / 2];  // at most min(c, S - c) each
    const PlanGeom p = plan_geom(a, blockIdx.y, blockIdx.x);
    int32_t* source = a.source + p.pair * a.max_keys;
    if (plan_ends(a, p, source)) return;
    uint32_t key[N];
    load_keys(a, p, 0, key);
    Digits d{0, 0, p.c};
    int count = 0;
    for (int pass = 0; pass < 3; ++pass) {
        clear_hist(sh);
        add_keys(d, pass, key, sh.hist);
        count = find_digit(sh, d, pass);
    }
    const uint32_t kept = kept_bits(sh, d, key, count, 0);
    const int2 n = list_slots<N>(
        sh, p, 0, kept, source, [&](int k, int s) { s_hole[k] = (uint16_t)s; }, [&](int k, int s) { s_mover[k] = (uint16_t)s; });
    __syncthreads();
    for (int u = threadIdx.x; u < n.x; u += kPlanThreads) source[s_hole[u]] = s_mover[u];
}

// The histograms of a pass.
__device__ __forceinline__ int32_t* chunk_hists(const PlanArgs& a, const PlanGeom& p, int pass) {
    return a.hist + ((pass & 1) * a.pairs + p.pair) * a.hists * kBins;
}

// Their sum over a request of many chunks, which every chunk's workgroup would form for
// itself.  Grid (KV heads x pieces of 64 bins, requests), 16 wavefronts for the chunks.
__global__ __launch_bounds__(kPlanThreads) void evict_sum(PlanArgs a, int pass) {
    __shared__ int s_sum[kPlanWaves][kWave];
    const PlanGeom p = plan_geom(a, blockIdx.x % a.hkv, blockIdx.y);
    if (p.S == p.c) return;
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int bin = blockIdx.x / a.hkv * kWave + lane, chunks = (p.S + kChunk - 1) / kChunk;
    int32_t* h = chunk_hists(a, p, pass) + bin;
    int v = 0;
#pragma unroll 8
    for (int k = wv; k < chunks; k += kPlanWaves) v += h[(int64_t)k * kBins];
    s_sum[wv][lane] = v;
    __syncthreads();
    if (wv > 0) return;
#pragma unroll
    for (int k = 1; k < kPlanWaves; ++k) v += s_sum[k][lane];
    h[(int64_t)a.chunks * kBins] = v;
}

__device__ __forceinline__ void sum_hists(const PlanArgs& a, const PlanGeom& p, int pass, PlanShared& sh) {
    const bool summed = a.hists > a.chunks;
    const int32_t* h = chunk_hists(a, p, pass) + (summed ? (int64_t)a.chunks * kBins : 0);
    const int chunks = summed ? 1 : (p.S + kChunk - 1) / kChunk;
    int v[kBins / kPlanThreads] = {};
#pragma unroll 8
    for (int k = 0; k < chunks; ++k)
#pragma unroll
        for (int e = 0; e < kBins / kPlanThreads; ++e) v[e] += h[(int64_t)k * kBins + e * kPlanThreads + threadIdx.x];
#pragma unroll
    for (int e = 0; e < kBins / kPlanThreads; ++e) sh.hist[e * kPlanThreads + threadIdx.x] = v[e];
}
// The digits after `pass` passes: those before from the state, the last one's from the
// histograms.
__device__ __forceinline__ int digits_after(const PlanArgs& a, const PlanGeom& p, int passes, PlanShared& sh, Digits& d) {
    d = Digits{0, 0, p.c};
    if (passes > 1) {
        const uint2 s = a.state[p.pair * 2 + passes - 2];
        d.prefix = s.x;
        d.need = (int)s.y;
        d.known = passes == 2 ? d.mask(0) : d.mask(0) | d.mask(1);
    }
    sum_hists(a, p, passes - 1, sh);
    return find_digit(sh, d, passes - 1);
}

// This thread's sort keys as the first pass leaves them for the others: they then need
// neither the table nor the ordinals, and arrive while the histograms are added up.
__device__ __forceinline__ uint4* stored_keys(const PlanArgs& a, const PlanGeom& p, int chunk) {
    return a.keys + ((p.pair * a.chunks + chunk) * (kPart / 4)) * kPlanThreads + threadIdx.x;
}
__device__ __forceinline__ void fetch_keys(const PlanArgs& a, const PlanGeom& p, int chunk, uint32_t (&key)[kPart]) {
    const uint4* from = stored_keys(a, p, chunk);
#pragma unroll
    for (int k = 0; k < kPart / 4; ++k) {
        const uint4 v = from[k * kPlanThreads];
        key[4 * k] = v.x, key[4 * k + 1] = v.y, key[4 * k + 2] = v.z, key[4 * k + 3] = v.w;
    }
}

// Grid (KV heads x chunks, requests), as the two kernels after it.
template <int PASS>
__global__ __launch_bounds__(kPlanThreads) void evict_hist(PlanArgs a) {
    __shared__ PlanShared sh;
    const PlanGeom p = plan_geom(a, blockIdx.x % a.hkv, blockIdx.y);
    const int chunk = blockIdx.x / a.hkv;
    if (p.S == p.c || (int64_t)chunk * kChunk >= p.S) return;
    uint32_t key[kPart];
    if constexpr (PASS == 0) {
        load_keys(a, p, chunk, key);
        uint4* to = stored_keys(a, p, chunk);
#pragma unroll
        for (int k = 0; k < kPart / 4; ++k)
            to[k * kPlanThreads] = make_uint4(key[4 * k], key[4 * k + 1], key[4 * k + 2], key[4 * k + 3]);
    } else {
        fetch_keys(a, p, chunk, key);
    }
    Digits d{0, 0, p.c};
    if (PASS > 0) {
        digits_after(a, p, PASS, sh, d);
        if (chunk == 0 && threadIdx.x == 0) a.state[p.pair * 2 + PASS - 1] = make_uint2(d.prefix, (uint32_t)d.need);
        __syncthreads();
    }
    clear_hist(sh);
    add_keys(d, PASS, key, sh.hist);
    __syncthreads();
    int32_t* out = chunk_hists(a, p, PASS) + (int64_t)chunk * kBins;
    for (int e = threadIdx.x; e < kBins; e += kPlanThreads) out[e] = sh.hist[e];
}

__global__ __launch_bounds__(kPlanThreads) void evict_lists(PlanArgs a) {
    __shared__ PlanShared sh;
    const PlanGeom p = plan_geom(a, blockIdx.x % a.hkv, blockIdx.y);
    const int chunk = blockIdx.x / a.hkv;
    int32_t* source = a.source + p.pair * a.max_keys;
    if (chunk == 0 && plan_ends(a, p, source)) return;
    if (p.S == p.c || (int64_t)chunk * kChunk >= p.S) return;
    uint32_t key[kPart];
    fetch_keys(a, p, chunk, key);
    Digits d;
    const int count = digits_after(a, p, 3, sh, d);
    int before = 0;
    if (count != d.need) {  // a lane per earlier chunk
        const int32_t* h = chunk_hists(a, p, 2) + (d.prefix & d.mask(2));
        for (int k = threadIdx.x & (kWave - 1); k < chunk; k += kWave) before += h[(int64_t)k * kBins];
        before = __builtin_amdgcn_readlane(wave_scan(before), kWave - 1);
    }
    const uint32_t kept = kept_bits(sh, d, key, count, before);
    uint16_t* list = a.lists + (p.pair * a.chunks + chunk) * kChunk;
    const int s0 = chunk * kChunk;
    const int2 n = list_slots<kPart>(
        sh, p, chunk, kept, source, [&](int k, int s) { list[k] = (uint16_t)(s - s0); },
        [&](int k, int s) { list[kChunk - 1 - k] = (uint16_t)(s - s0); });
    if (threadIdx.x == 0) a.counts[p.pair * a.chunks + chunk] = n;
}

// The n-th hole of the request takes its n-th mover.
__global__ __launch_bounds__(kPlanThreads) void evict_join(PlanArgs a) {
    __shared__ int s_movers[kMaxChunks];  // before and in each chunk
    __shared__ int s_holes;
    const PlanGeom p = plan_geom(a, blockIdx.x % a.hkv, blockIdx.y);
    const int chunk = blockIdx.x / a.hkv, chunks = (p.S + kChunk - 1) / kChunk;
    if (p.S == p.c || chunk >= chunks) return;
    const int2* counts = a.counts + p.pair * a.chunks;
    const int holes = counts[chunk].x;
    if (holes == 0) return;
    if (threadIdx.x < kWave) {
        int holes_before = 0, sum = 0;
        for (int base = 0; base < chunks; base += kWave) {
            const int k = base + threadIdx.x;
            const int2 n = k < chunks ? counts[k] : make_int2(0, 0);
            const int x = wave_scan(n.y), y = wave_scan(k < chunk ? n.x : 0);
            if (k < chunks) s_movers[k] = sum + x;
            sum += __builtin_amdgcn_readlane(x, kWave - 1);
            holes_before += __builtin_amdgcn_readlane(y, kWave - 1);
        }
        if (threadIdx.x == 0) s_holes = holes_before;
    }
    __syncthreads();
    const uint16_t* lists = a.lists + p.pair * a.chunks * kChunk;
    int32_t* source = a.source + p.pair * a.max_keys;
    for (int u = threadIdx.x; u < holes; u += kPlanThreads) {
        const int n = s_holes + u;
        int k = 0, top = chunks - 1;  // the first chunk with more than n movers up to its end
        while (k < top) {
            const int mid = (k + top) / 2;
            if (s_movers[mid] <= n) k = mid + 1;
            else top = mid;
        }
        const int m = n - (k > 0 ? s_movers[k - 1] : 0);
        source[chunk * kChunk + lists[(int64_t)chunk * kChunk + u]] = k * kChunk + lists[(int64_t)k * kChunk + kChunk - 1 - m];
    }
}

struct CompactArgs {
    const int32_t* block_tables;
    const int32_t* source;
    const int32_t* new_lens;
    void* kc;
    void* vc;
    float* key_weights;
    int32_t* key_order;
    int hkv, max_blocks, num_blocks, max_keys, blocks;
};

constexpr int kCompactWaves = 4;

__device__ __forceinline__ uint32_t bits_of(float x) { return __float_as_uint(x); }
__device__ __forceinline__ uint32_t bits_of(uint16_t x) { return x; }
__device__ __forceinline__ float of_bits(uint32_t x, float) { return __uint_as_float(x); }
__device__ __forceinline__ uint16_t of_bits(uint32_t x, uint16_t) { return (uint16_t)x; }

// A block that many keys move into is written whole, the keys that stay as they are
// included.  Lines that are written in part are read back and merged at the memory,
// which costs as much as reading them here: 16 caches of 8 to 16 thousand keys brought
// to 4096 took 242 us with partial writes, 217 with whole ones (1.05 GB at the rate of
// a copy: a moved key's value lies in D 32-byte pieces of 16 keys, so all of the blocks
// it leaves and enters passes by).  A block with few moves writes those alone (32 caches
// with nine moves per head: 12 us, whole 19; the same with 2, 3 and 4 blocks per
// wavefront, and the long moves slower).  Between them, 16 caches of 4096 slots in which
// every block has the same number of moves, in part and whole: one 132 and 152 us, two
// 163 and 165, three 180 and 170, four 189 and 173, five 192 and 169, eight 187 and 170.
// From three on the step with nine moves takes 13.4 us instead of 12.3.
constexpr int kWholeMoves = 5;

// Grid (KV heads x groups of blocks, requests), a wavefront per block, a lane per slot
// and quarter of the dims.
template <typename T, int D>
__global__ __launch_bounds__(kCompactWaves * kWave) void kv_compact(CompactArgs a) {
    constexpr int N = 16 / (int)sizeof(T);
    constexpr int64_t TILE = (int64_t)D * kBlockTokens;
    const int i = blockIdx.y, g = blockIdx.x % a.hkv;
    const int lane = threadIdx.x & (kWave - 1), t = lane & 15, part = lane >> 4;
    const int b = blockIdx.x / a.hkv * kCompactWaves + threadIdx.x / kWave;
    if (b >= a.blocks) return;
    const int d = b * kBlockTokens + t;
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    int s = d;
    if (d < a.max_keys && d < a.new_lens[i]) s = a.source[((int64_t)i * a.hkv + g) * a.max_keys + d];
    const int to = table[b];
    int from = -1;
    if (s != d && s >= 0 && s / kBlockTokens < a.max_blocks) from = table[s / kBlockTokens];
    const bool moved = from >= 0 && from < a.num_blocks && to >= 0 && to < a.num_blocks;
    const int moves = __popcll(__ballot(moved)) / 4;
    if (moves == 0 || (!moved && moves < kWholeMoves)) return;
    const int slot = moved ? s % kBlockTokens : t;
    const int64_t src = (int64_t)(moved ? from : to) * a.hkv + g, dst = (int64_t)to * a.hkv + g;
    const u32x4* ks = reinterpret_cast<const u32x4*>(static_cast<const T*>(a.kc) + src * TILE) + slot;
    u32x4* kd = reinterpret_cast<u32x4*>(static_cast<T*>(a.kc) + dst * TILE) + t;
    const T* vs = static_cast<const T*>(a.vc) + src * TILE + slot;
    T* vd = static_cast<T*>(a.vc) + dst * TILE + t;
    u32x4 k[D / N / 4];
    uint32_t v[D / 4];
#pragma unroll
    for (int x = 0; x < D / N / 4; ++x) k[x] = ks[(4 * x + part) * kBlockTokens];
#pragma unroll
    for (int x = 0; x < D / 4; ++x) v[x] = bits_of(vs[(4 * x + part) * kBlockTokens]);
#pragma unroll
    for (int x = 0; x < D / N / 4; ++x) kd[(4 * x + part) * kBlockTokens] = k[x];
#pragma unroll
    for (int x = 0; x < D / 4; ++x) vd[(4 * x + part) * kBlockTokens] = of_bits(v[x], T{});
    if (!moved) return;
    if (part == 0 && a.key_weights) a.key_weights[dst * kBlockTokens + t] = a.key_weights[src * kBlockTokens + slot];
    if (part == 1 && a.key_order) a.key_order[dst * kBlockTokens + t] = a.key_order[src * kBlockTokens + slot];
}

int check(const verify_attn_params* p, int32_t max_seq_len, int32_t max_keys) {
    const int rc = validate(p, 0, 0, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    if (p->sliding_window > 0) return VERIFY_EUNSUPPORTED;
    return max_keys < 1 ? VERIFY_EINVAL : VERIFY_OK;
}

// Chunks of the longest request; 1: evict_plan alone, without a workspace.
int64_t plan_chunks(const verify_attn_params& p, int32_t max_seq_len) {
    const int64_t longest = std::min<int64_t>(max_seq_len, (int64_t)p.max_blocks_per_seq * kBlockTokens);
    return longest <= kAlone ? 1 : (longest + kChunk - 1) / kChunk;
}

// Histograms of a request: evict_sum adds up those of more than 20 chunks (eight heads,
// each workgroup adding them up for itself and with evict_sum: 131072 slots 30 and 35 us,
// 196608 40 and 39, a million 183 and 88).
size_t plan_hists(int64_t chunks) { return chunks + (chunks > 20); }

// A grid's first dimension holds fewer than 2^32 threads, those of the chunks and of
// evict_sum; its second fewer than 2^16 workgroups, evict_plan's heads.
bool plan_fits(const verify_attn_params& p, int64_t chunks) {
    return chunks <= kMaxChunks && p.num_kv_heads < (1 << 16) && std::max<int64_t>(chunks, kBins / kWave) * p.num_kv_heads < (1 << 22);
}

struct PlanSpace {
    size_t hist, lists, counts, state, total;  // offsets behind the sort keys
};

PlanSpace plan_space(const verify_attn_params& p, int32_t max_seq_len, int32_t max_keys) {
    PlanSpace w{};
    const size_t chunks = (size_t)plan_chunks(p, max_seq_len), pairs = (size_t)p.num_seqs * p.num_kv_heads;
    if (chunks == 1 || max_keys >= max_seq_len) return w;
    w.hist = pairs * chunks * kChunk * sizeof(uint32_t);
    w.lists = w.hist + align_up(2 * pairs * plan_hists(chunks) * kBins * sizeof(int32_t), 256);
    w.counts = w.lists + align_up(pairs * chunks * kChunk * sizeof(uint16_t), 256);
    w.state = w.counts + align_up(pairs * chunks * sizeof(int2), 256);
    w.total = w.state + align_up(pairs * 2 * sizeof(uint2), 256);
    return w;
}

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_evict_plan_workspace_size(const verify_attn_params* params, int32_t max_seq_len,
                                                int32_t max_keys, size_t* bytes) {
    if (!bytes) return VERIFY_EINVAL;
    const int rc = check(params, max_seq_len, max_keys);
    if (rc != VERIFY_OK) return rc;
    if (!plan_fits(*params, plan_chunks(*params, max_seq_len))) return VERIFY_EUNSUPPORTED;
    *bytes = plan_space(*params, max_seq_len, max_keys).total;
    return VERIFY_OK;
}

extern "C" int verify_evict_plan(const verify_attn_params* params, int32_t max_seq_len, int32_t max_keys,
                                 int32_t keep_first, int32_t keep_recent, const float* key_weights,
                                 const int32_t* key_order, const int32_t* block_tables, const int32_t* seq_lens,
                                 const int32_t* num_tokens, int32_t* source, int32_t* new_lens, void* workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    const int rc = check(params, max_seq_len, max_keys);
    if (rc != VERIFY_OK) return rc;
    const verify_attn_params& p = *params;
    if (keep_first < 0 || keep_recent < 0 || (int64_t)keep_first + keep_recent > max_keys) return VERIFY_EINVAL;
    if (p.num_seqs > 0 && (!block_tables || !seq_lens || !source || !new_lens)) return VERIFY_EINVAL;
    if (p.num_seqs > 0 && p.num_blocks > 0 && !key_weights) return VERIFY_EINVAL;
    if (((uintptr_t)key_weights | (uintptr_t)key_order | (uintptr_t)workspace) & 15) return VERIFY_EINVAL;
    const int64_t chunks = plan_chunks(p, max_seq_len);
    if (!plan_fits(p, chunks)) return VERIFY_EUNSUPPORTED;
    const PlanSpace space = plan_space(p, max_seq_len, max_keys);
    if (workspace_bytes < space.total || (space.total > 0 && !workspace)) return VERIFY_EWORKSPACE;
    if (p.num_seqs == 0) return VERIFY_OK;
    PlanArgs a{};
    a.key_weights = key_weights;
    a.key_order = key_order;
    a.block_tables = block_tables;
    a.seq_lens = seq_lens;
    a.num_tokens = num_tokens;
    a.source = source;
    a.new_lens = new_lens;
    a.pairs = (int64_t)p.num_seqs * p.num_kv_heads;
    a.chunks = (int)chunks;
    a.hists = (int)plan_hists(chunks);
    a.hkv = p.num_kv_heads;
    a.max_blocks = p.max_blocks_per_seq;
    a.num_blocks = p.num_blocks;
    a.max_seq_len = max_seq_len;
    a.max_keys = max_keys;
    a.keep_first = keep_first;
    a.keep_recent = keep_recent;
    if (space.total == 0) {  // (also where no request can exceed max_keys)
        const dim3 grid((unsigned)p.num_seqs, (unsigned)p.num_kv_heads);
        const int64_t longest = std::min<int64_t>(max_seq_len, (int64_t)p.max_blocks_per_seq * kBlockTokens);
        if (longest <= 4 * kPlanThreads) hipLaunchKernelGGL(evict_plan<4>, grid, dim3(kPlanThreads), 0, stream, a);
        else if (longest <= 8 * kPlanThreads) hipLaunchKernelGGL(evict_plan<8>, grid, dim3(kPlanThreads), 0, stream, a);
        else hipLaunchKernelGGL(evict_plan<kSlots>, grid, dim3(kPlanThreads), 0, stream, a);
        return check_launch();
    }
    char* ws = static_cast<char*>(workspace);
    a.keys = reinterpret_cast<uint4*>(ws);
    a.hist = reinterpret_cast<int32_t*>(ws + space.hist);
    a.lists = reinterpret_cast<uint16_t*>(ws + space.lists);
    a.counts = reinterpret_cast<int2*>(ws + space.counts);
    a.state = reinterpret_cast<uint2*>(ws + space.state);
    const dim3 grid((unsigned)(p.num_kv_heads * chunks), (unsigned)p.num_seqs);
    const dim3 sums((unsigned)(p.num_kv_heads * (kBins / kWave)), (unsigned)p.num_seqs);
    auto sum = [&](int pass) {
        if (a.hists > a.chunks) hipLaunchKernelGGL(evict_sum, sums, dim3(kPlanThreads), 0, stream, a, pass);
    };
    hipLaunchKernelGGL(evict_hist<0>, grid, dim3(kPlanThreads), 0, stream, a);
    sum(0);
    hipLaunchKernelGGL(evict_hist<1>, grid, dim3(kPlanThreads), 0, stream, a);
    sum(1);
    hipLaunchKernelGGL(evict_hist<2>, grid, dim3(kPlanThreads), 0, stream, a);
    sum(2);
    hipLaunchKernelGGL(evict_lists, grid, dim3(kPlanThreads), 0, stream, a);
    hipLaunchKernelGGL(evict_join, grid, dim3(kPlanThreads), 0, stream, a);
    return check_launch();
}

extern "C" int verify_kv_compact(const verify_attn_params* params, int32_t max_keys, const int32_t* block_tables,
                                 const int32_t* source, const int32_t* new_lens, void* k_cache, void* v_cache,
                                 float* key_weights, int32_t* key_order, hipStream_t stream) {
    const int rc = check(params, 0, max_keys);
    if (rc != VERIFY_OK) return rc;
    const verify_attn_params& p = *params;
    if (p.num_seqs > 0 && (!block_tables || !source || !new_lens)) return VERIFY_EINVAL;
    if (p.num_seqs > 0 && p.num_blocks > 0 && (!k_cache || !v_cache)) return VERIFY_EINVAL;
    if (((uintptr_t)k_cache | (uintptr_t)v_cache) & 15) return VERIFY_EINVAL;
    if (p.num_seqs == 0 || p.num_blocks == 0) return VERIFY_OK;
    CompactArgs a{};
    a.block_tables = block_tables;
    a.source = source;
    a.new_lens = new_lens;
    a.kc = k_cache;
    a.vc = v_cache;
    a.key_weights = key_weights;
    a.key_order = key_order;
    a.hkv = p.num_kv_heads;
    a.max_blocks = p.max_blocks_per_seq;
    a.num_blocks = p.num_blocks;
    a.max_keys = max_keys;
    a.blocks = (int)std::min<int64_t>(((int64_t)max_keys + kBlockTokens - 1) / kBlockTokens, p.max_blocks_per_seq);
    const int64_t groups = ((int64_t)a.blocks + kCompactWaves - 1) / kCompactWaves;
    if (groups * a.hkv >= (1 << 24)) return VERIFY_EUNSUPPORTED;
    const dim3 grid((unsigned)(groups * a.hkv), (unsigned)p.num_seqs), threads(kCompactWaves * kWave);
    const bool wide = p.head_dim == 128;
    auto* kernel = p.dtype == VERIFY_BF16 ? (wide ? kv_compact<uint16_t, 128> : kv_compact<uint16_t, 64>)
                                          : (wide ? kv_compact<float, 128> : kv_compact<float, 64>);
    hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a);
    return check_launch();
}
