// verify_key_weights.hip -- the attention weight that every cached key gathers from a
// step's rows, summed over the rows and the query heads of its KV head.
//
//   w[t] = sum_r 2^(s_rt - m_r) / l_r,   l_r = sum_t' 2^(s_rt' - m_r),  s in log2 units
//
// r runs over the (row, head of the group) pairs of a (request, KV head), m_r is about
// the row's maximum.  A key's weight needs every row's l_r, so the keys are read
// twice, in two launches:
//   weight_stats  rows stay, keys stream past: each lane keeps a running maximum and
//                 sum per row over the keys of its own columns, joined at the end of
//                 a split of the keys into one (maximum, sum) per row and split;
//   weight_sums   keys stay in registers, rows stream past from LDS: a key's weights
//                 are added up within its lane; the splits' sums are joined into m_r
//                 and 1 / l_r as the rows are staged.
// (A row's logarithm log2 l_r + m_r in the place of the two would be rounded at the
// size of the scores, and every weight of the row with it.)
// Scores are MFMA products, the queries the first operand and 16 keys the second, so
// that a lane holds one key (column) and four rows of every product.  A block's K tile
// lies in memory as the operand wants it: 16 bytes per lane, 1 KiB per load, no LDS.
#include <type_traits>

#include "common.h"

namespace averify {
namespace {

constexpr int kWgtWaves = 4;
constexpr int kWgtThreads = kWgtWaves * kWave;
constexpr float kWgtLog2e = 1.4426950408889634f;
// 16-row tiles of a weight_stats workgroup at most
constexpr int stat_tiles(bool bf16) { return bf16 ? 8 : 4; }

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
// queries are aligned to their elements only
typedef uint32_t u32x4u_t __attribute__((ext_vector_type(4), aligned(2)));

struct WgtArgs {
    const void* q;
    const void* kc;
    const int32_t* block_tables;
    const int32_t* seq_lens;
    const int32_t* q_start;
    const int32_t* num_rows;
    const int32_t* num_tokens;
    const float* sinks;
    float* key_weights;
    int32_t* key_order;
    float2* part;  // [total_q][Hq][splits] (maximum, sum relative to it) of each split
    int num_seqs, total_q, hq, hkv, group, max_blocks, num_blocks, max_seq_len;
    float scale_log2, decay;
    int splits, split_blocks;    // of weight_stats
    int chunks;                  // row chunks in its grid
    int sum_blocks;              // blocks of a weight_sums workgroup
    int lds_tiles;               // row tiles that weight_sums holds in LDS
};

struct WgtGeom {
    int q0, n, S, rows, blocks;  // rows: counted rows times the group
};

__device__ __forceinline__ WgtGeom wgt_geom(const WgtArgs& a, int i) {
    WgtGeom g;
    g.q0 = min(max(a.q_start[i], 0), a.total_q);
    g.n = max(min(a.q_start[i + 1], a.total_q) - g.q0, 0);
    g.S = (int)max((int64_t)0, min((int64_t)a.seq_lens[i], min((int64_t)a.max_seq_len, (int64_t)a.max_blocks * kBlockTokens)));
    const int counted = a.num_rows ? min(max(a.num_rows[i], 0), g.n) : g.n;
    g.rows = counted * a.group;
    g.blocks = (g.S + kBlockTokens - 1) / kBlockTokens;
    return g;
}

// Operands of 16 rows or keys over the head dim: NC 16-byte chunks per lane, chunk c
// of lane l the dims of 16-byte chunk 4 c + l / 16 of row or key l % 16.
template <typename T, int D>
struct Operand {
    static constexpr int NC = D * kBlockTokens * (int)sizeof(T) / 1024;
    uint4 v[NC];
};

// scores of 16 rows against 16 keys: lane l has key l % 16 of rows 4 (l / 16) + 0 .. 3
template <int D>
__device__ __forceinline__ f32x4_t product(const uint4* q, const uint4* k, uint16_t) {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < Operand<uint16_t, D>::NC; ++c)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q[c]), __builtin_bit_cast(bf16x8_t, k[c]),
                                                      acc, 0, 0, 0);
    return acc;
}
template <int D>
__device__ __forceinline__ f32x4_t product(const uint4* q, const uint4* k, float) {
    // two sums, so that consecutive products do not wait for each other
    f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < Operand<float, D>::NC; ++c) {
        const f32x4_t x = __builtin_bit_cast(f32x4_t, q[c]), y = __builtin_bit_cast(f32x4_t, k[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc[e & 1], 0, 0, 0);
    }
    return acc[0] + acc[1];
}

// Stages rows [first, first + 16 tiles) of (request, KV head) in LDS in operand
// order.  Places behind the last row repeat the chunk's first row: their products are
// finite wherever that row's are, so what is multiplied by zero later stays zero.
// `pos` receives the rows' positions (-1 without a row).
template <typename T, int D>
__device__ __forceinline__ void stage_rows(const WgtArgs& a, const WgtGeom& geo, int g, int first, int tiles, uint4* lds,
                                           int* pos) {
    constexpr int NC = Operand<T, D>::NC;
    for (int e = threadIdx.x; e < tiles * NC * kWave; e += kWgtThreads) {
        const int lane = e % kWave, c = e / kWave % NC, tile = e / kWave / NC;
        int r = first + tile * 16 + lane % 16;
        if (r >= geo.rows) r = first;
        const int j = r / a.group, h = r - j * a.group;
        const T* src = static_cast<const T*>(a.q) + ((int64_t)(geo.q0 + j) * a.hq + g * a.group + h) * D +
                       (4 * c + lane / 16) * (16 / (int)sizeof(T));
        const u32x4u_t v = *reinterpret_cast<const u32x4u_t*>(src);
        lds[e] = make_uint4(v.x, v.y, v.z, v.w);
    }
    for (int t = threadIdx.x; t < tiles * 16; t += kWgtThreads)
        pos[t] = first + t < geo.rows ? geo.S - geo.n + (first + t) / a.group : -1;
}

// K tile of block `phys`, KV head g.
template <typename T, int D>
__device__ __forceinline__ void load_keys(const WgtArgs& a, int g, int phys, Operand<T, D>& k) {
    const uint4* src = static_cast<const uint4*>(a.kc) + ((int64_t)phys * a.hkv + g) * (Operand<T, D>::NC * kWave) +
                       (threadIdx.x & (kWave - 1));
#pragma unroll
    for (int c = 0; c < Operand<T, D>::NC; ++c) k.v[c] = src[c * kWave];
}

// Blocks of a wavefront's step: 8 to 16 KiB of keys in flight.
constexpr int step_blocks(int d, bool bf16) { return d == 128 && !bf16 ? 2 : 4; }

// Row slack: a row's sum is kept relative to a maximum that may be exceeded by this
// many powers of two before the sum is rescaled (rarely, then).
constexpr float kSlackLog2 = 8.f;

// Grid (row chunks x KV heads x splits, requests).
template <typename T, int D, int RT>
__global__ __launch_bounds__(kWgtThreads) void weight_stats(WgtArgs a) {
    constexpr int NB = step_blocks(D, sizeof(T) == 2), NC = Operand<T, D>::NC;
    __shared__ uint4 s_q[RT * NC * kWave];
    __shared__ float s_m[kWgtWaves][RT * 16], s_l[kWgtWaves][RT * 16];
    __shared__ __attribute__((aligned(16))) int s_pos[RT * 16];
    const int i = blockIdx.y;
    const int g = blockIdx.x % a.hkv;
    const int chunk0 = blockIdx.x / a.hkv % a.chunks, split = blockIdx.x / a.hkv / a.chunks;
    const WgtGeom geo = wgt_geom(a, i);
    const int b_lo = split * a.split_blocks;
    if (b_lo >= geo.blocks) return;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), l16 = lane & 15, lg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    const int p0 = geo.S - geo.n;  // position of row 0
    for (int first = chunk0 * (RT * 16); first < geo.rows; first += a.chunks * (RT * 16)) {
        const int tiles = min(RT, (geo.rows - first + 15) / 16);
        __syncthreads();
        stage_rows<T, D>(a, geo, g, first, tiles, s_q, s_pos);
        __syncthreads();
        const int p_first = p0 + first / a.group;
        const int p_last = p0 + (min(first + RT * 16, geo.rows) - 1) / a.group;
        // blocks that a row of the chunk sees
        const int b_hi = min(min(b_lo + a.split_blocks, geo.blocks), p_last < 0 ? 0 : p_last / kBlockTokens + 1);
        float m[RT][4], l[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[r][e] = -INFINITY;
                l[r][e] = 0.f;
            }
        for (int b = b_lo + w * NB; b < b_hi; b += kWgtWaves * NB) {
            const int id = lane < NB && b + lane < b_hi ? table[b + lane] : -1;
            const bool valid = id >= 0 && id < a.num_blocks;
            const uint32_t ok = (uint32_t)__ballot(valid);
            if (ok == 0) continue;
            Operand<T, D> k[NB];
#pragma unroll
            for (int x = 0; x < NB; ++x) load_keys<T, D>(a, g, __builtin_amdgcn_readlane(valid ? id : 0, x), k[x]);
            const bool masked = ok != (1u << NB) - 1 || (b + NB) * kBlockTokens - 1 > p_first;
            // keeps the query operands in LDS: hoisted out of the loop they would take
            // D / 8 (bf16) or D / 4 registers per tile
            int ql = lane;
            asm volatile("" : "+v"(ql));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (r >= tiles) break;
                uint4 qv[NC];
#pragma unroll
                for (int c = 0; c < NC; ++c) qv[c] = s_q[(r * NC + c) * kWave + ql];
                f32x4_t s[NB];
#pragma unroll
                for (int x = 0; x < NB; ++x) s[x] = product<D>(qv, k[x].v, T{});
                if (masked) {
                    const i32x4_t pos = *reinterpret_cast<const i32x4_t*>(s_pos + r * 16 + (ql >> 4) * 4);
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const int t = ((ok >> x) & 1u) ? (b + x) * kBlockTokens + l16 : INT32_MAX;
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[x][e] = t <= pos[e] ? s[x][e] : -INFINITY;
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float top = s[0][e];
#pragma unroll
                    for (int x = 1; x < NB; ++x) top = fmaxf(top, s[x][e]);
                    top *= a.scale_log2;
                    if (__any(top > m[r][e] + kSlackLog2)) {
                        const float mn = fmaxf(m[r][e], top);
                        l[r][e] *= m[r][e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r][e] - mn);
                        m[r][e] = mn;
                    }
                    const float ref = m[r][e] == -INFINITY ? 0.f : m[r][e];
#pragma unroll
                    for (int x = 0; x < NB; ++x) l[r][e] += __builtin_amdgcn_exp2f(fmaf(s[x][e], a.scale_log2, -ref));
                }
            }
        }
        // join the 16 columns, then the wavefronts
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float M = wave_max_xor(m[r][e], 16);
                const float L = wave_sum_xor(m[r][e] == -INFINITY ? l[r][e] : l[r][e] * __builtin_amdgcn_exp2f(m[r][e] - M), 16);
                if (l16 == 0) {
                    s_m[w][r * 16 + lg * 4 + e] = M;
                    s_l[w][r * 16 + lg * 4 + e] = L;
                }
            }
        __syncthreads();
        const int r = first + tid;
        if (tid < RT * 16 && r < geo.rows) {
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int x = 0; x < kWgtWaves; ++x) M = fmaxf(M, s_m[x][tid]);
#pragma unroll
            for (int x = 0; x < kWgtWaves; ++x)
                L += s_m[x][tid] == -INFINITY ? s_l[x][tid] : s_l[x][tid] * __builtin_amdgcn_exp2f(s_m[x][tid] - M);
            const int j = r / a.group, h = r - j * a.group;
            a.part[((int64_t)(geo.q0 + j) * a.hq + g * a.group + h) * a.splits + split] = make_float2(M, L);
        }
    }
}

// Grid (KV heads x ranges of sum_blocks blocks, requests).  Where the request's
// counted rows fit the LDS tiles they are staged once; otherwise every step of the
// keys stages them in turn.
template <typename T, int D, int NB>
__global__ __launch_bounds__(kWgtThreads) void weight_sums(WgtArgs a) {
    constexpr int NC = Operand<T, D>::NC;
    extern __shared__ uint4 s_dyn[];  // the row tiles, then their rows' m, 1 / l and positions
    uint4* s_q = s_dyn;
    float* s_m = reinterpret_cast<float*>(s_dyn + a.lds_tiles * NC * kWave);
    float* s_inv = s_m + a.lds_tiles * 16;
    int* s_pos = reinterpret_cast<int*>(s_inv + a.lds_tiles * 16);
    const int i = blockIdx.y;
    const int g = blockIdx.x % a.hkv, range = blockIdx.x / a.hkv;
    const WgtGeom geo = wgt_geom(a, i);
    const int b_lo = range * a.sum_blocks;
    if (b_lo >= geo.blocks) return;
    const int b_hi = min(b_lo + a.sum_blocks, geo.blocks);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), l16 = lane & 15, lg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    const int p0 = geo.S - geo.n;
    const int nsplit = (geo.blocks + a.split_blocks - 1) / a.split_blocks;
    auto stage = [&](int first, int tiles) {
        stage_rows<T, D>(a, geo, g, first, tiles, s_q, s_pos);
        for (int t = tid; t < tiles * 16; t += kWgtThreads) {
            // a place without a row, a row without a key: 2^(s - inf) * 0
            float m = INFINITY, inv = 0.f;
            const int r = first + t;
            if (r < geo.rows) {
                const int j = r / a.group, h = g * a.group + r - j * a.group;
                const float2* part = a.part + ((int64_t)(geo.q0 + j) * a.hq + h) * a.splits;
                float M = -INFINITY, L = 0.f;
                for (int s = 0; s < nsplit; ++s) {
                    const float2 p = part[s];
                    const float mn = fmaxf(M, p.x);
                    if (mn == -INFINITY) {
                        L += p.y;  // 0, or a NaN
                    } else {
                        L = L * __builtin_amdgcn_exp2f(M - mn) + p.y * __builtin_amdgcn_exp2f(p.x - mn);
                        M = mn;
                    }
                }
                if (a.sinks && M != -INFINITY) L += exp2f(a.sinks[h] * kWgtLog2e - M);
                if (M != -INFINITY) {
                    m = M;
                    inv = 1.f / L;
                } else if (L != 0.f) {  // every score was NaN
                    m = L;
                }
            }
            s_m[t] = m;
            s_inv[t] = inv;
        }
    };
    const int all_tiles = (geo.rows + 15) / 16;
    const bool once = all_tiles <= a.lds_tiles;
    if (once) {
        stage(0, all_tiles);
        __syncthreads();
    }
    for (int b0 = b_lo; b0 < b_hi; b0 += kWgtWaves * NB) {
        const int b = b0 + w * NB;
        const int id = lane < NB && b + lane < b_hi ? table[b + lane] : -1;
        const bool valid = id >= 0 && id < a.num_blocks;
        const uint32_t ok = (uint32_t)__ballot(valid);
        Operand<T, D> k[NB];
        float sum[NB];
#pragma unroll
        for (int x = 0; x < NB; ++x) sum[x] = 0.f;
        if (ok) {
#pragma unroll
            for (int x = 0; x < NB; ++x) load_keys<T, D>(a, g, __builtin_amdgcn_readlane(valid ? id : 0, x), k[x]);
        }
        auto add_tiles = [&](int first, int tiles) {
            for (int r = 0; r < tiles; ++r) {
                const int row = r * 16;
                const int p_lo = __builtin_amdgcn_readfirstlane(s_pos[row]);
                const int p_hi = __builtin_amdgcn_readfirstlane(s_pos[min(row + 16, geo.rows - first) - 1]);
                if (p_hi < b * kBlockTokens) continue;  // none of its rows sees the step's keys
                uint4 qv[NC];
#pragma unroll
                for (int c = 0; c < NC; ++c) qv[c] = s_q[(r * NC + c) * kWave + lane];
                const f32x4_t m = *reinterpret_cast<const f32x4_t*>(s_m + r * 16 + lg * 4);
                const f32x4_t inv = *reinterpret_cast<const f32x4_t*>(s_inv + r * 16 + lg * 4);
                if ((b + NB) * kBlockTokens - 1 > p_lo) {
                    // keys that some of the rows do not see
                    const i32x4_t pos = *reinterpret_cast<const i32x4_t*>(s_pos + r * 16 + lg * 4);
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const f32x4_t s = product<D>(qv, k[x].v, T{});
                        const int t = (b + x) * kBlockTokens + l16;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float p = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, -m[e])) * inv[e];
                            sum[x] += t <= pos[e] ? p : 0.f;
                        }
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const f32x4_t s = product<D>(qv, k[x].v, T{});
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            sum[x] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, -m[e])), inv[e], sum[x]);
                    }
                }
            }
        };
        if (once) {
            if (ok) add_tiles(0, all_tiles);
        } else {
            // from the first row that sees the step's first key
            const int64_t skip = max((int64_t)0, (int64_t)b0 * kBlockTokens - p0) * a.group;
            for (int64_t f = skip / 16 * 16; f < geo.rows; f += a.lds_tiles * 16) {
                const int first = (int)f, tiles = min(a.lds_tiles, (geo.rows - first + 15) / 16);
                __syncthreads();
                stage(first, tiles);
                __syncthreads();
                if (ok) add_tiles(first, tiles);
            }
        }
        if (!ok) continue;
        // four lane groups hold different rows of the same 16 keys; afterwards lane
        // group lg stores the blocks x with x % 4 == lg
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            sum[x] += __shfl_xor(sum[x], 16);
            sum[x] += __shfl_xor(sum[x], 32);
            const int phys = __builtin_amdgcn_readlane(valid ? id : 0, x);
            const int t = (b + x) * kBlockTokens + l16;
            if (lg == x % 4 && ((ok >> x) & 1u) && t < geo.S) {
                const int64_t at = ((int64_t)phys * a.hkv + g) * kBlockTokens + l16;
                float v = sum[x];
                if (t >= p0) a.key_order[at] = (a.num_tokens ? a.num_tokens[i] : geo.S) - geo.S + t;
                else if (a.decay != 0.f) v += a.decay * a.key_weights[at];
                a.key_weights[at] = v;
            }
        }
    }
}

// ------------------------------------------------------------------ host side

struct WgtPlan {
    int chunks, stat_tiles;  // weight_stats: row chunks, tiles per chunk
    int splits, split_blocks;
    int lds_tiles, sum_blocks, ranges;
    bool once;
    size_t bytes, cover;
};

int64_t tile_bytes(const verify_attn_params& p) {
    return 16 * (int64_t)p.head_dim * (p.dtype == VERIFY_BF16 ? 2 : 4);
}

int make_plan(const verify_attn_params& p, int32_t total_q, int32_t max_q_len, int32_t max_seq_len, WgtPlan* out) {
    WgtPlan pl{};
    const int64_t G = p.num_q_heads / p.num_kv_heads;
    const int64_t tiles = (G * std::max(1, max_q_len) + 15) / 16;
    const int64_t blocks = std::max<int64_t>(
        1, std::min<int64_t>(((int64_t)max_seq_len + kBlockTokens - 1) / kBlockTokens, p.max_blocks_per_seq));
    const bool bf16 = p.dtype == VERIFY_BF16;
    const int64_t step = kWgtWaves * step_blocks(p.head_dim, bf16);  // blocks of a workgroup's step
    const int most_tiles = stat_tiles(bf16);
    pl.stat_tiles = (int)std::min<int64_t>(tiles, most_tiles);
    pl.chunks = (int)std::min<int64_t>((tiles + most_tiles - 1) / most_tiles, 4096);
    // a split has at most 128 blocks, and at least a step, towards four workgroups per
    // compute unit
    const int64_t want = 4 * 256, most = (blocks + step - 1) / step, least = (blocks + 127) / 128;
    const int64_t wgs = (int64_t)p.num_kv_heads * pl.chunks;
    auto splits = [&](int64_t seqs) { return std::max(least, std::min(most, (want + seqs * wgs - 1) / (seqs * wgs))); };
    const int64_t ns = splits(std::max(1, p.num_seqs));
    pl.split_blocks = (int)(((blocks + ns - 1) / ns + step - 1) / step * step);
    pl.splits = (int)((blocks + pl.split_blocks - 1) / pl.split_blocks);
    pl.once = tiles * tile_bytes(p) <= 56 * 1024;
    if (pl.once) {
        pl.lds_tiles = (int)tiles;
        pl.sum_blocks = pl.split_blocks;
    } else {
        pl.lds_tiles = (int)(16 * 1024 / tile_bytes(p));
        pl.sum_blocks = kWgtWaves;
    }
    // a grid dimension holds fewer than 2^32 threads
    const int64_t ranges = (blocks + pl.sum_blocks - 1) / pl.sum_blocks;
    pl.ranges = (int)ranges;
    if (std::max<int64_t>(pl.splits * wgs, ranges * p.num_kv_heads) >= (1 << 24)) return VERIFY_EUNSUPPORTED;
    const size_t row = (size_t)p.num_q_heads * sizeof(float2);
    pl.bytes = align_up(row * total_q * pl.splits, 256);
    // Any batch of fewer requests: b of them have at most b max_q_len rows and
    // want / (b wgs) + 1 splits, or `least`.
    const int64_t few = ((int64_t)std::max(1, max_q_len) * want + wgs - 1) / wgs + total_q;
    pl.cover = std::max(pl.bytes, align_up(row * (size_t)std::max(std::min(few, (int64_t)total_q * most), (int64_t)total_q * least), 256));
    *out = pl;
    return VERIFY_OK;
}

template <typename T, int D>
void launch(const WgtArgs& a, const WgtPlan& pl, int seqs, hipStream_t stream) {
    const dim3 stats((unsigned)((int64_t)a.hkv * pl.chunks * pl.splits), (unsigned)seqs);
    auto run = [&](auto rt) {
        hipLaunchKernelGGL((weight_stats<T, D, decltype(rt)::value>), stats, dim3(kWgtThreads), 0, stream, a);
    };
    switch (pl.stat_tiles) {
        case 1: run(std::integral_constant<int, 1>{}); break;
        case 2: run(std::integral_constant<int, 2>{}); break;
        case 3: run(std::integral_constant<int, 3>{}); break;
        case 4: run(std::integral_constant<int, 4>{}); break;
        default:
            if constexpr (sizeof(T) == 2) {
                if (pl.stat_tiles <= 6) run(std::integral_constant<int, 6>{});
                else run(std::integral_constant<int, 8>{});
            }
    }
    const dim3 sums((unsigned)pl.ranges * a.hkv, (unsigned)seqs);
    const size_t lds = (size_t)pl.lds_tiles * (Operand<T, D>::NC * kWave * sizeof(uint4) + 3 * 16 * sizeof(float));
    if (pl.once) hipLaunchKernelGGL((weight_sums<T, D, step_blocks(D, sizeof(T) == 2)>), sums, dim3(kWgtThreads), lds, stream, a);
    else hipLaunchKernelGGL((weight_sums<T, D, 1>), sums, dim3(kWgtThreads), lds, stream, a);
}

int check(const verify_attn_params* p, int32_t total_q, int32_t max_q_len, int32_t max_seq_len) {
    const int rc = validate(p, total_q, max_q_len, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    if (p->sliding_window > 0) return VERIFY_EUNSUPPORTED;
    return VERIFY_OK;
}

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_key_weights_workspace_size(const verify_attn_params* params, int32_t total_q, int32_t max_q_len,
                                                 int32_t max_seq_len, size_t* bytes) {
    if (!bytes) return VERIFY_EINVAL;
    const int rc = check(params, total_q, max_q_len, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    WgtPlan pl;
    const int fits = make_plan(*params, total_q, max_q_len, max_seq_len, &pl);
    if (fits == VERIFY_OK) *bytes = pl.cover;
    return fits;
}

extern "C" int verify_key_weights(const verify_attn_params* params, int32_t total_q, int32_t max_q_len,
                                  int32_t max_seq_len, const void* q, const void* k_cache,
                                  const int32_t* block_tables, const int32_t* seq_lens, const int32_t* q_start,
                                  const int32_t* num_rows, const int32_t* num_tokens, const float* sinks, float decay,
                                  float* key_weights, int32_t* key_order, void* workspace, size_t workspace_bytes,
                                  hipStream_t stream) {
    int rc = check(params, total_q, max_q_len, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    const verify_attn_params& p = *params;
    if (!(decay >= 0.f) || decay > 3.0e38f) return VERIFY_EINVAL;
    if (p.num_seqs > 0 && (!block_tables || !seq_lens || !q_start)) return VERIFY_EINVAL;
    if (p.num_blocks > 0 && p.num_seqs > 0 && (!k_cache || !key_weights || !key_order)) return VERIFY_EINVAL;
    if (total_q > 0 && !q) return VERIFY_EINVAL;
    if ((uintptr_t)k_cache & 15) return VERIFY_EINVAL;
    WgtPlan pl;
    rc = make_plan(p, total_q, max_q_len, max_seq_len, &pl);
    if (rc != VERIFY_OK) return rc;
    if (workspace_bytes < pl.bytes || (pl.bytes > 0 && !workspace)) return VERIFY_EWORKSPACE;
    if (p.num_seqs == 0 || p.num_blocks == 0 || max_seq_len == 0) return VERIFY_OK;
    WgtArgs a{};
    a.q = q;
    a.kc = k_cache;
    a.block_tables = block_tables;
    a.seq_lens = seq_lens;
    a.q_start = q_start;
    a.num_rows = num_rows;
    a.num_tokens = num_tokens;
    a.sinks = sinks;
    a.key_weights = key_weights;
    a.key_order = key_order;
    a.part = static_cast<float2*>(workspace);
    a.num_seqs = p.num_seqs;
    a.total_q = total_q;
    a.hq = p.num_q_heads;
    a.hkv = p.num_kv_heads;
    a.group = p.num_q_heads / p.num_kv_heads;
    a.max_blocks = p.max_blocks_per_seq;
    a.num_blocks = p.num_blocks;
    a.max_seq_len = max_seq_len;
    a.scale_log2 = (p.scale > 0.f ? p.scale : 1.0f / sqrtf((float)p.head_dim)) * kWgtLog2e;
    a.decay = decay;
    a.splits = pl.splits;
    a.split_blocks = pl.split_blocks;
    a.chunks = pl.chunks;
    a.sum_blocks = pl.sum_blocks;
    a.lds_tiles = pl.lds_tiles;
    if (p.dtype == VERIFY_BF16)
        p.head_dim == 128 ? launch<uint16_t, 128>(a, pl, p.num_seqs, stream) : launch<uint16_t, 64>(a, pl, p.num_seqs, stream);
    else
        p.head_dim == 128 ? launch<float, 128>(a, pl, p.num_seqs, stream) : launch<float, 64>(a, pl, p.num_seqs, stream);
    return check_launch();
}
