// verify_evict.hip -- the keys that a bounded cache keeps, and their moves.
//
//   evict_plan   one workgroup per (request, KV head): the c-th largest sort key of
//                the request's S slots by a radix select (three digits, histograms in
//                LDS), then one sweep in slot order that finds the kept slots, the
//                holes among the first c and the kept slots behind them.  A thread
//                takes a 16-slot block at a time, 64 contiguous bytes of each array.
//   kv_compact   one wavefront per 16-slot block that keys move into.
//
// A slot's sort key is one 32-bit word: the order key of its weight, above all of
// them 0xffffffff for what is always kept, 0 for what never is.
#include "common.h"

namespace averify {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kDigitBits = 11;
constexpr int kBins = 1 << kDigitBits;

struct PlanArgs {
    const float* key_weights;
    const int32_t* key_order;
    const int32_t* block_tables;
    const int32_t* seq_lens;
    const int32_t* num_tokens;
    int32_t* source;
    int32_t* new_lens;
    int32_t* lists;  // [pairs][2][list_len]: holes, and kept slots behind c
    int64_t list_len;
    int hkv, max_blocks, num_blocks, max_seq_len, max_keys, keep_first, keep_recent;
};

// Exclusive prefix sum over the workgroup; the total in `total`.
__device__ __forceinline__ int scan_exclusive(int v, int* wave_sums, int& total) {
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    int x = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();  // the sums of the scan before are read
    if (lane == kWave - 1) wave_sums[wv] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int s = wave_sums[w];
        before += w < wv ? s : 0;
        all += s;
    }
    total = all;
    return before + x - v;
}

__global__ __launch_bounds__(kPlanThreads) void evict_plan(PlanArgs a) {
    __shared__ int hist[kBins];
    __shared__ int wave_sums[kPlanWaves];
    __shared__ int s_digit, s_above;
    const int g = blockIdx.x, i = blockIdx.y, tid = threadIdx.x;
    const int S = (int)max((int64_t)0, min((int64_t)a.seq_lens[i], min((int64_t)a.max_seq_len, (int64_t)a.max_blocks * kBlockTokens)));
    const int c = min(S, a.max_keys);
    const int64_t pair = (int64_t)i * a.hkv + g;
    int32_t* source = a.source + pair * a.max_keys;
    if (g == 0 && tid == 0) a.new_lens[i] = c;
    if (S == c) {
        for (int d = tid; d < a.max_keys; d += kPlanThreads) source[d] = d < c ? d : -1;
        return;
    }
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    const int64_t recent = (int64_t)(a.num_tokens ? a.num_tokens[i] : S) - a.keep_recent;
    const int blocks = (S + kBlockTokens - 1) / kBlockTokens;
    const int rounds = (blocks + kPlanThreads - 1) / kPlanThreads;

    // the sort keys of this thread's block of a round, and how many of them count
    uint32_t key[kBlockTokens];
    int cnt = 0;
    auto load = [&](int round) {
        const int b = round * kPlanThreads + tid, s0 = b * kBlockTokens;
        cnt = b < blocks ? min(kBlockTokens, S - s0) : 0;
        if (cnt == 0) return;
        const int id = table[b];
        if (id < 0 || id >= a.num_blocks) {
#pragma unroll
            for (int e = 0; e < kBlockTokens; ++e) key[e] = s0 + e < c ? 0xffffffffu : 0u;
            return;
        }
        const int64_t at = ((int64_t)id * a.hkv + g) * kBlockTokens;
#pragma unroll
        for (int e = 0; e < kBlockTokens; ++e) {
            const uint32_t k = min(order_key(__float_as_uint(a.key_weights[at + e])), 0xfffffffeu);
            const int o = a.key_order ? a.key_order[at + e] : s0 + e;
            key[e] = o < a.keep_first || o >= recent ? 0xffffffffu : k;
        }
    };

    // the c-th largest key: its digits from the top, `need` of the keys that share the
    // digits so far being among the c largest
    uint32_t prefix = 0, known = 0;  // known: mask of the digits found
    int need = c;
    if (rounds == 1) load(0);
    for (int shift = 32 - kDigitBits; ; shift = max(0, shift - kDigitBits)) {
        const uint32_t digits = ~known & (0xffffffffu << shift);  // of this pass
        for (int e = tid; e < kBins; e += kPlanThreads) hist[e] = 0;
        __syncthreads();
        for (int round = 0; round < rounds; ++round) {
            if (rounds > 1) load(round);
#pragma unroll
            for (int e = 0; e < kBlockTokens; ++e)
                if (e < cnt && (key[e] & known) == prefix) atomicAdd(&hist[(key[e] & digits) >> shift], 1);
        }
        __syncthreads();
        // two bins per thread, the highest first
        const int top = kBins - 1 - 2 * tid;
        const int h1 = hist[top], h0 = hist[top - 1];
        int total;
        const int above = scan_exclusive(h1 + h0, wave_sums, total);
        if (above < need && need <= above + h1) {
            s_digit = top;
            s_above = above;
        } else if (above + h1 < need && need <= above + h1 + h0) {
            s_digit = top - 1;
            s_above = above + h1;
        }
        __syncthreads();
        prefix |= (uint32_t)s_digit << shift;
        need -= s_above;
        known |= digits;
        __syncthreads();
        if (shift == 0) break;
    }

    // slots in order: kept are the keys above prefix and the first `need` equal to it
    int32_t* holes = a.lists + pair * 2 * a.list_len;
    int32_t* movers = holes + a.list_len;
    int ties = 0, nholes = 0, nmovers = 0;
    for (int round = 0; round < rounds; ++round) {
        if (rounds > 1) load(round);
        const int s0 = (round * kPlanThreads + tid) * kBlockTokens;
        int eq = 0, total;
#pragma unroll
        for (int e = 0; e < kBlockTokens; ++e) eq += e < cnt && key[e] == prefix;
        int rank = ties + scan_exclusive(eq, wave_sums, total);
        ties += total;
        uint32_t hole = 0, mover = 0;
#pragma unroll
        for (int e = 0; e < kBlockTokens; ++e) {
            if (e >= cnt) continue;
            bool kept = key[e] > prefix;
            if (key[e] == prefix) kept = rank++ < need;
            if (s0 + e < c) {
                if (kept) source[s0 + e] = s0 + e;
                else hole |= 1u << e;
            } else if (kept) {
                mover |= 1u << e;
            }
        }
        // both counts in one scan: a round has 2^14 slots
        const int mine = __popc(hole) | (__popc(mover) << 16);
        const int before = scan_exclusive(mine, wave_sums, total);
        int h = nholes + (before & 0xffff), m = nmovers + (before >> 16);
#pragma unroll
        for (int e = 0; e < kBlockTokens; ++e) {
            if ((hole >> e) & 1u) holes[h++] = s0 + e;
            if ((mover >> e) & 1u) movers[m++] = s0 + e;
        }
        nholes += total & 0xffff;
        nmovers += total >> 16;
    }
    __syncthreads();
    for (int u = tid; u < nholes; u += kPlanThreads) source[holes[u]] = movers[u];
    for (int d = c + tid; d < a.max_keys; d += kPlanThreads) source[d] = -1;
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

// Grid (KV heads x groups of blocks, requests), a wavefront per block.
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
    const bool move = from >= 0 && from < a.num_blocks && to >= 0 && to < a.num_blocks;
    if (!move) return;
    const int slot = s % kBlockTokens;
    const int64_t src = (int64_t)from * a.hkv + g, dst = (int64_t)to * a.hkv + g;
    const uint4* ks = reinterpret_cast<const uint4*>(static_cast<const T*>(a.kc) + src * TILE) + slot;
    uint4* kd = reinterpret_cast<uint4*>(static_cast<T*>(a.kc) + dst * TILE) + t;
    uint4 k[D / N / 4];
#pragma unroll
    for (int x = 0; x < D / N / 4; ++x) k[x] = ks[(4 * x + part) * kBlockTokens];
#pragma unroll
    for (int x = 0; x < D / N / 4; ++x) kd[(4 * x + part) * kBlockTokens] = k[x];
    const T* vs = static_cast<const T*>(a.vc) + src * TILE + slot;
    T* vd = static_cast<T*>(a.vc) + dst * TILE + t;
    for (int x0 = 0; x0 < D / 4; x0 += 16) {
        T v[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] = vs[(4 * (x0 + x) + part) * kBlockTokens];
#pragma unroll
        for (int x = 0; x < 16; ++x) vd[(4 * (x0 + x) + part) * kBlockTokens] = v[x];
    }
    if (part == 0 && a.key_weights) a.key_weights[dst * kBlockTokens + t] = a.key_weights[src * kBlockTokens + slot];
    if (part == 1 && a.key_order) a.key_order[dst * kBlockTokens + t] = a.key_order[src * kBlockTokens + slot];
}

int check(const verify_attn_params* p, int32_t max_seq_len, int32_t max_keys) {
    const int rc = validate(p, 0, 0, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    if (p->sliding_window > 0) return VERIFY_EUNSUPPORTED;
    return max_keys < 1 ? VERIFY_EINVAL : VERIFY_OK;
}

// Holes of a (request, KV head) at most.
int64_t list_len(const verify_attn_params& p, int32_t max_seq_len, int32_t max_keys) {
    const int64_t longest = std::min<int64_t>(max_seq_len, (int64_t)p.max_blocks_per_seq * kBlockTokens);
    return std::max<int64_t>(0, std::min<int64_t>(max_keys, longest - max_keys));
}

size_t plan_bytes(const verify_attn_params& p, int32_t max_seq_len, int32_t max_keys) {
    return align_up((size_t)p.num_seqs * p.num_kv_heads * 2 * (size_t)list_len(p, max_seq_len, max_keys) * sizeof(int32_t), 256);
}

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_evict_plan_workspace_size(const verify_attn_params* params, int32_t max_seq_len,
                                                int32_t max_keys, size_t* bytes) {
    if (!bytes) return VERIFY_EINVAL;
    const int rc = check(params, max_seq_len, max_keys);
    if (rc == VERIFY_OK) *bytes = plan_bytes(*params, max_seq_len, max_keys);
    return rc;
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
    const size_t need = plan_bytes(p, max_seq_len, max_keys);
    if (workspace_bytes < need || (need > 0 && !workspace)) return VERIFY_EWORKSPACE;
    if (p.num_seqs == 0) return VERIFY_OK;
    PlanArgs a{};
    a.key_weights = key_weights;
    a.key_order = key_order;
    a.block_tables = block_tables;
    a.seq_lens = seq_lens;
    a.num_tokens = num_tokens;
    a.source = source;
    a.new_lens = new_lens;
    a.lists = static_cast<int32_t*>(workspace);
    a.list_len = list_len(p, max_seq_len, max_keys);
    a.hkv = p.num_kv_heads;
    a.max_blocks = p.max_blocks_per_seq;
    a.num_blocks = p.num_blocks;
    a.max_seq_len = max_seq_len;
    a.max_keys = max_keys;
    a.keep_first = keep_first;
    a.keep_recent = keep_recent;
    hipLaunchKernelGGL(evict_plan, dim3((unsigned)p.num_kv_heads, (unsigned)p.num_seqs), dim3(kPlanThreads), 0, stream, a);
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
