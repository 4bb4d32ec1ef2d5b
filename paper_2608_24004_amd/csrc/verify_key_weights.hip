// verify_key_weights.hip -- the attention weight that every cached key gathers from a
// step's rows, summed over the rows and the query heads of its KV head.
//
//   w[t] = sum_r 2^(s_rt - m_r) / l_r,   l_r = sum_t' 2^(s_rt' - m_r),  s in log2 units
//
// r runs over the (row, head of the group) pairs of a (request, KV head), m_r is about
// the row's maximum.  A key's weight needs every row's l_r, so the keys are read
// twice, in two launches:
//   weight_stats  each lane keeps a running maximum and sum per row over the keys of
//                 its own columns, joined at the end of a split of the keys into one
//                 (maximum, sum) per row and split;
//   weight_sums   a key's weights are added up within its lane; the splits' parts are
//                 joined into m_r and 1 / l_r as the rows are staged in LDS.
// In both the rows stay and the keys stream past, the next step's loads in flight.
// Where the scores themselves are few (a decoding step) weight_stats stores them and
// weight_sums reads those instead.  With more rows than LDS holds the second becomes
//   weight_join, weight_sums_rows, weight_store   the parts joined once, then keys
//                 stay in registers and the rows stream past through LDS.
// What bounds it: few rows, the keys' bytes (32 requests of 475 MB of keys, 36 rows each:
// 179 us for two passes that both read them, 5.3 TB/s, the rate of a copy); many rows, in
// the first pass the vector instructions, an exponential per row and key among them, in the
// second uneven rows and waits as much (the prompts named at weight_sums_rows' segments: 65
// and 74 us, in which a compute unit has work for 50 and 46, its vector units then active
// 77 and 53 % of the time; the matrix instructions take 14 us of each).
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
constexpr int kStatTiles = 8;

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
    float2* part;  // (maximum, sum relative to it) of each row and split, see part_of
    float2* rows;  // (maximum, 1 / sum) of each row: [request][KV head][row]
    int num_seqs, total_q, hq, hkv, group, max_blocks, num_blocks, max_seq_len;
    float scale_log2, decay;
    uint32_t group_magic;        // ceil(2^32 / group)
    int splits, split_blocks;    // of weight_stats
    int chunks;                  // row chunks in its grid
    int sum_blocks;              // blocks of a weight_sums workgroup
    int segments, segment_tiles; // of weight_sums_rows
    int64_t sum_keys;            // keys of a segment's sums
    float* sums;                 // [requests][Hkv][segments][sum_keys]
    f32x4_t* scores;             // [requests][Hkv][score_blocks], see scores_of
    int score_rows, score_blocks;
    int lds_tiles;               // row tiles that weight_sums holds in LDS
};

// r / group: exact where r (group - 1) < 2^32, which the host checks.
__device__ __forceinline__ int by_group(const WgtArgs& a, int r) {
    return a.group == 1 ? r : (int)__umulhi((uint32_t)r, a.group_magic);
}

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

// The parts of row r of KV head g: [request][KV head][row][splits].
__device__ __forceinline__ float2* part_of(const WgtArgs& a, const WgtGeom& geo, int g, int r) {
    return a.part + ((int64_t)geo.q0 * a.hq + (int64_t)g * geo.rows + r) * a.splits;
}

__device__ __forceinline__ float2* rows_of(const WgtArgs& a, const WgtGeom& geo, int g) {
    return a.rows + (int64_t)geo.q0 * a.hq + (int64_t)g * geo.rows;
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
// order.  Places behind the last row repeat it.  Where no row of a tile is masked, their
// products are multiplied by zero, which leaves a NaN of a row or key that is not finite:
// the last row sees every key that any row of its tile sees, so that such a key's weight
// is NaN by that row itself.  `pos` receives the rows' positions (-1 without a row).
template <typename T, int D>
__device__ __forceinline__ void stage_rows(const WgtArgs& a, const WgtGeom& geo, int g, int first, int tiles, uint4* lds,
                                           int* pos) {
    constexpr int NC = Operand<T, D>::NC;
    for (int e = threadIdx.x; e < tiles * NC * kWave; e += kWgtThreads) {
        const int lane = e % kWave, c = e / kWave % NC, tile = e / kWave / NC;
        int r = first + tile * 16 + lane % 16;
        if (r >= geo.rows) r = geo.rows - 1;
        if (geo.rows == 0) {
            lds[e] = make_uint4(0, 0, 0, 0);
            continue;
        }
        const int j = by_group(a, r), h = r - j * a.group;
        const T* src = static_cast<const T*>(a.q) + ((int64_t)(geo.q0 + j) * a.hq + g * a.group + h) * D +
                       (4 * c + lane / 16) * (16 / (int)sizeof(T));
        const u32x4u_t v = *reinterpret_cast<const u32x4u_t*>(src);
        lds[e] = make_uint4(v.x, v.y, v.z, v.w);
    }
    for (int t = threadIdx.x; t < tiles * 16; t += kWgtThreads)
        pos[t] = first + t < geo.rows ? geo.S - geo.n + by_group(a, first + t) : -1;
}

// op over the 16 lanes of a row, by rotations of it within the vector unit (shuffles
// go through LDS, one latency each).
template <typename Op>
__device__ __forceinline__ float of_16_lanes(float x, Op op) {
    auto turn = [](float x, auto n) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x120 + decltype(n)::value, 0xf, 0xf, false));
    };
    x = op(x, turn(x, std::integral_constant<int, 8>{}));
    x = op(x, turn(x, std::integral_constant<int, 4>{}));
    x = op(x, turn(x, std::integral_constant<int, 2>{}));
    return op(x, turn(x, std::integral_constant<int, 1>{}));
}

// The sum over the four rows of 16 lanes.
__device__ __forceinline__ float of_4_rows(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);  // rows 0 + 1 twice, 2 + 3 twice
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// K tile of block `phys`, KV head g.  ONCE: read for the last time in the call, and kept
// out of the way of what is read again (the second pass of the 32 requests above: 187 ->
// 181 us for both; the only one of a decoding step, 32 requests of 4097 keys: 70 -> 63).
template <typename T, int D, bool ONCE>
__device__ __forceinline__ void load_keys(const WgtArgs& a, int g, int phys, Operand<T, D>& k) {
    const uint4* src = static_cast<const uint4*>(a.kc) + ((int64_t)phys * a.hkv + g) * (Operand<T, D>::NC * kWave) +
                       (threadIdx.x & (kWave - 1));
#pragma unroll
    for (int c = 0; c < Operand<T, D>::NC; ++c) k.v[c] = ONCE ? ld16_stream(src + c * kWave) : src[c * kWave];
}

// Blocks of a wavefront's step where keys stream past (two such steps are in
// registers, 8 or 16 KiB of loads in flight), and where they stay.
constexpr int step_blocks(int d, bool bf16) { return d == 128 && !bf16 ? 1 : 2; }
constexpr int held_blocks(int d, bool bf16) { return d == 128 && !bf16 ? 2 : 4; }
// Row tiles that then go by together: 16 KiB.
constexpr int row_tiles(int d, bool bf16) { return 16 * 1024 / (16 * d * (bf16 ? 2 : 4)); }

// Row slack: a row's sum is kept relative to a maximum that may be exceeded by this
// many powers of two before the sum is rescaled (rarely, then).
constexpr float kSlackLog2 = 8.f;
// The maximum of no score: finite, so that it needs no case of its own (2^(-inf - m)
// is 0, 2^(m - m) is 1, and any score exceeds it).
constexpr float kNoScore = -3.0e38f;

// The blocks of a wavefront, NB at a time and kWgtWaves * NB apart, their ids read 64
// at a time (one per lane) and their K tiles a step ahead of their use.
template <typename T, int D, int NB, bool ONCE = false>
struct Walk {
    const WgtArgs& a;
    const int32_t* table;
    int g, b, b_hi;   // next blocks to load: [b, b + NB), below b_hi
    int ids, at;      // ids of the wavefront's next blocks from lane `at` on

    __device__ Walk(const WgtArgs& a, const int32_t* table, int g, int b, int b_hi)
        : a(a), table(table), g(g), b(b), b_hi(b_hi), ids(-1), at(kWave) {}

    // The blocks' bits in the result: valid ids.  `phys` receives the ids, and K tiles
    // are loaded from those it then holds: the loads are the same in number whatever
    // is valid, so that a wait for the step before need not wait for them.
    __device__ __forceinline__ uint32_t load(Operand<T, D> (&k)[NB], int (&phys)[NB]) {
        uint32_t ok = 0;
        if (b < b_hi) {
            if (at >= kWave) {
                const int lane = threadIdx.x & (kWave - 1);
                const int bl = b + lane / NB * (kWgtWaves * NB) + lane % NB;
                ids = bl < b_hi ? table[bl] : -1;
                // settled here, every 64 blocks: otherwise the compiler waits for it, and
                // with it for the keys in flight, at every step's reading of the ids
                __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
                at = 0;
            }
#pragma unroll
            for (int x = 0; x < NB; ++x) {
                const int id = __builtin_amdgcn_readlane(ids, at + x);
                const bool valid = id >= 0 && id < a.num_blocks;
                ok |= (uint32_t)valid << x;
                phys[x] = valid ? id : 0;
            }
            at += NB;
            b += kWgtWaves * NB;
        }
#pragma unroll
        for (int x = 0; x < NB; ++x) load_keys<T, D, ONCE>(a, g, phys[x], k[x]);
        return ok;
    }
};

// Scores of block b that weight_stats leaves for weight_sums: [row / 4][key][row % 4],
// the four rows that a lane holds of a product.
__device__ __forceinline__ f32x4_t* scores_of(const WgtArgs& a, int i, int g, int b) {
    return a.scores + (((int64_t)i * a.hkv + g) * a.score_blocks + b) * (a.score_rows / 4) * kBlockTokens;
}

// Grid (row chunks x KV heads x splits, requests).  SCORES: the products are stored.
template <typename T, int D, int RT, bool SCORES = false>
__global__ __launch_bounds__(kWgtThreads) void weight_stats(WgtArgs a) {
    constexpr int NB = step_blocks(D, sizeof(T) == 2), NC = Operand<T, D>::NC;
    __shared__ uint4 s_q[RT * NC * kWave];
    __shared__ float s_m[kWgtWaves][RT * 16], s_l[kWgtWaves][RT * 16];
    __shared__ __attribute__((aligned(16))) int s_pos[RT * 16];
    const int i = blockIdx.y;
    const int g = blockIdx.x % a.hkv;
    // the last rows first: a prompt's see the most keys
    const int chunk0 = a.chunks - 1 - blockIdx.x / a.hkv % a.chunks, split = blockIdx.x / a.hkv / a.chunks;
    const WgtGeom geo = wgt_geom(a, i);
    const int b_lo = split * a.split_blocks;
    if (b_lo >= geo.blocks) return;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), l16 = lane & 15, lg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    const int p0 = geo.S - geo.n;  // position of row 0
    for (int first = chunk0 * (RT * 16); first < geo.rows; first += a.chunks * (RT * 16)) {
        const int tiles = min(RT, (geo.rows - first + 15) / 16);
        const int p_first = p0 + by_group(a, first);
        const int p_last = p0 + by_group(a, min(first + RT * 16, geo.rows) - 1);
        // blocks that a row of the chunk sees
        const int b_hi = min(min(b_lo + a.split_blocks, geo.blocks), p_last < 0 ? 0 : p_last / kBlockTokens + 1);
        float m[RT][4], l[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[r][e] = kNoScore;
                l[r][e] = 0.f;
            }
        // (also of a step without a valid block, and with no test before the first tile: if
        // there is a way past their use, keys are waited for before their registers are
        // loaded again, and the next step's with them)
        auto compute = [&](const Operand<T, D> (&k)[NB], uint32_t ok, int b) {
            const bool masked = ok != (1u << NB) - 1 || (b + NB) * kBlockTokens - 1 > p_first;
            // keeps the query operands in LDS: hoisted out of the loop they would take
            // D / 8 (bf16) or D / 4 registers per tile
            int ql = lane;
            asm volatile("" : "+v"(ql));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (r > 0 && r >= tiles) break;
                uint4 qv[NC];
#pragma unroll
                for (int c = 0; c < NC; ++c) qv[c] = s_q[(r * NC + c) * kWave + ql];
                f32x4_t s[NB];
#pragma unroll
                for (int x = 0; x < NB; ++x) s[x] = product<D>(qv, k[x].v, T{});
                if constexpr (SCORES) {
#pragma unroll
                    for (int x = 0; x < NB; ++x)
                        if (((ok >> x) & 1u) && lg * 4 < geo.rows && geo.rows <= a.score_rows)
                            scores_of(a, i, g, b + x)[lane] = s[x];
                }
                if (masked) {
                    const i32x4_t pos = *reinterpret_cast<const i32x4_t*>(s_pos + r * 16 + (ql >> 4) * 4);
#pragma unroll
                    for (int x = 0; x < NB; ++x) {
                        const int t = ((ok >> x) & 1u) ? (b + x) * kBlockTokens + l16 : INT32_MAX;
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[x][e] = t <= pos[e] ? s[x][e] : -INFINITY;
                    }
                }
                // the scores as they enter the exponentials; one test for all of them
                float top = -INFINITY;
                auto relative = [&](int e, int x) { return fmaf(s[x][e], a.scale_log2, -m[r][e]); };
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int x = 0; x < NB; ++x) top = fmaxf(top, relative(e, x));
                if (__any(top > kSlackLog2)) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float mn = s[0][e];
#pragma unroll
                        for (int x = 1; x < NB; ++x) mn = fmaxf(mn, s[x][e]);
                        mn = fmaxf(m[r][e], mn * a.scale_log2);
                        l[r][e] *= __builtin_amdgcn_exp2f(m[r][e] - mn);
                        m[r][e] = mn;
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int x = 0; x < NB; ++x) l[r][e] += __builtin_amdgcn_exp2f(relative(e, x));
            }
        };
        Walk<T, D, NB, SCORES> walk(a, table, g, b_lo + w * NB, b_hi);
        Operand<T, D> k0[NB], k1[NB];
        int phys[NB] = {}, b = walk.b;
        uint32_t ok0 = walk.load(k0, phys), ok1;
        __syncthreads();  // the chunk before is done with the rows
        stage_rows<T, D>(a, geo, g, first, tiles, s_q, s_pos);
        __syncthreads();
        // in pairs of steps, without a way out between a step's loads and their use
        constexpr int STEP = kWgtWaves * NB;
        int steps = b < b_hi ? (b_hi - b + STEP - 1) / STEP : 0;
        for (; steps > 1; steps -= 2) {
            ok1 = walk.load(k1, phys);
            compute(k0, ok0, b);
            ok0 = walk.load(k0, phys);
            compute(k1, ok1, b + STEP);
            b += 2 * STEP;
        }
        if (steps > 0) compute(k0, ok0, b);
        // join the 16 columns, then the wavefronts
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float M = of_16_lanes(m[r][e], [](float x, float y) { return fmaxf(x, y); });
                const float L = of_16_lanes(l[r][e] * __builtin_amdgcn_exp2f(m[r][e] - M), [](float x, float y) { return x + y; });
                if (l16 == 0) {
                    s_m[w][r * 16 + lg * 4 + e] = M;
                    s_l[w][r * 16 + lg * 4 + e] = L;
                }
            }
        __syncthreads();
        const int r = first + tid;
        if (tid < RT * 16 && r < geo.rows) {
            float M = kNoScore, L = 0.f;
#pragma unroll
            for (int x = 0; x < kWgtWaves; ++x) M = fmaxf(M, s_m[x][tid]);
#pragma unroll
            for (int x = 0; x < kWgtWaves; ++x) L += s_l[x][tid] * __builtin_amdgcn_exp2f(s_m[x][tid] - M);
            part_of(a, geo, g, r)[split] = make_float2(M, L);
        }
    }
}

// A row's (m, 1 / l) from its splits' parts, and its head's sink.  A row without a
// key has (inf, 0), and so has a place without a row: 2^(s - inf) * 0.
__device__ __forceinline__ float2 join_parts(const WgtArgs& a, const float2* part, int nsplit, int h) {
    constexpr int kRound = 8;  // loads in flight: one by one each cost a memory latency
    float M = kNoScore, L = 0.f;
    for (int s0 = 0; s0 < nsplit; s0 += kRound) {
        float2 p[kRound];
#pragma unroll
        for (int x = 0; x < kRound; ++x) p[x] = part[min(s0 + x, nsplit - 1)];
        float mn = M;
#pragma unroll
        for (int x = 0; x < kRound; ++x) mn = fmaxf(mn, p[x].x);
        L *= __builtin_amdgcn_exp2f(M - mn);
#pragma unroll
        for (int x = 0; x < kRound; ++x) L += s0 + x < nsplit ? p[x].y * __builtin_amdgcn_exp2f(p[x].x - mn) : 0.f;
        M = mn;
    }
    if (M == kNoScore) return make_float2(L == 0.f ? INFINITY : L, 0.f);  // (or every score was NaN)
    if (a.sinks) L += exp2f(a.sinks[h] * kWgtLog2e - M);
    return make_float2(M, 1.f / L);
}

// Adds the weights of 16 rows to sum[x], key l16 of block b + x; `pos` are the four
// rows' positions (-1: none), read where some row does not see some key.
template <typename T, int D, int NB>
__device__ __forceinline__ void add_tile(const WgtArgs& a, const uint4* qv, const Operand<T, D> (&k)[NB], const f32x4_t& m,
                                         const f32x4_t& inv, bool masked, const i32x4_t& pos, int b, float (&sum)[NB]) {
    const int l16 = threadIdx.x & 15;
    if (masked) {
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

// Writes the sums of key t: added to `old` (its decayed sum), or a new key's first.
__device__ __forceinline__ void store_weight(const WgtArgs& a, const WgtGeom& geo, int i, int64_t at, int t, float sum,
                                             float old) {
    const bool fresh = t >= geo.S - geo.n;
    if (fresh) a.key_order[at] = (a.num_tokens ? a.num_tokens[i] : geo.S) - geo.S + t;
    a.key_weights[at] = fresh || a.decay == 0.f ? sum : sum + a.decay * old;
}

// Few rows: grid (KV heads x ranges of sum_blocks blocks, requests).  The request's
// row tiles stay in LDS, its keys stream past.  SCORES: where the rows are no more than
// score_rows, the scores that weight_stats stored are read in the keys' place, a thread
// per key.
template <typename T, int D, bool SCORES>
__global__ __launch_bounds__(kWgtThreads) void weight_sums(WgtArgs a) {
    constexpr int NB = step_blocks(D, sizeof(T) == 2), NC = Operand<T, D>::NC;
    extern __shared__ uint4 s_dyn[];  // the row tiles, then their rows' m, 1 / l and positions
    uint4* s_q = s_dyn;
    float* s_m = reinterpret_cast<float*>(s_dyn + a.lds_tiles * NC * kWave);
    float* s_inv = s_m + a.lds_tiles * 16;
    int* s_pos = reinterpret_cast<int*>(s_inv + a.lds_tiles * 16);
    // backwards: the keys that weight_stats read last are still in the last-level cache
    // (32 requests of 475 MB: 112 -> 97 us)
    const int i = a.num_seqs - 1 - blockIdx.y;
    const int g = blockIdx.x % a.hkv, range = blockIdx.x / a.hkv;
    const WgtGeom geo = wgt_geom(a, i);
    const int b_lo = range * a.sum_blocks;
    if (b_lo >= geo.blocks) return;
    const int b_hi = min(b_lo + a.sum_blocks, geo.blocks);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), l16 = lane & 15, lg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    const int nsplit = (geo.blocks + a.split_blocks - 1) / a.split_blocks;
    if (SCORES && geo.rows <= a.score_rows) {
        if (tid < geo.rows) {
            const float2 mi = join_parts(a, part_of(a, geo, g, tid), nsplit, g * a.group + tid - by_group(a, tid) * a.group);
            s_m[tid] = mi.x;
            s_inv[tid] = mi.y;
            s_pos[tid] = geo.S - geo.n + by_group(a, tid);
        }
        __syncthreads();
        for (int t = b_lo * kBlockTokens + tid; t < min(b_hi * kBlockTokens, geo.S); t += kWgtThreads) {
            const int id = table[t / kBlockTokens];
            if (id < 0 || id >= a.num_blocks) continue;
            const int64_t at = ((int64_t)id * a.hkv + g) * kBlockTokens + t % kBlockTokens;
            const float old = t < geo.S - geo.n && a.decay != 0.f ? a.key_weights[at] : 0.f;
            const f32x4_t* scores = scores_of(a, i, g, t / kBlockTokens) + t % kBlockTokens;
            float sum = 0.f;
            for (int r0 = 0; r0 < geo.rows; r0 += 4) {
                const f32x4_t x = scores[r0 / 4 * kBlockTokens];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (r0 + r >= geo.rows) break;
                    // (a key that no row sees has no scores, and is not asked for them)
                    const float p = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale_log2, -s_m[r0 + r])) * s_inv[r0 + r];
                    sum += t <= s_pos[r0 + r] ? p : 0.f;
                }
            }
            store_weight(a, geo, i, at, t, sum, old);
        }
        return;
    }
    const int all_tiles = max(1, (geo.rows + 15) / 16);
    Walk<T, D, NB, true> walk(a, table, g, b_lo + w * NB, b_hi);
    // lane group lg holds the weights of block x = lg of a step
    auto load_old = [&](uint32_t ok, const int (&phys)[NB], int b) {
        float old = 0.f;
#pragma unroll
        for (int x = 0; x < NB; ++x)
            if (lg == x && ((ok >> x) & 1u) && (b + x) * kBlockTokens + l16 < geo.S - geo.n)
                old = a.key_weights[((int64_t)phys[x] * a.hkv + g) * kBlockTokens + l16];
        return old;
    };
    // rows beyond the LDS tiles (a request with more rows than announced) go by in
    // further rounds over the keys, which add to what the first has written
    for (int first = 0; first == 0 || first < all_tiles; first += a.lds_tiles) {
        const int tiles = min(a.lds_tiles, all_tiles - first);
        Walk<T, D, NB, true> go = walk;
        Operand<T, D> k0[NB], k1[NB];
        int phys0[NB] = {}, phys1[NB] = {}, b = go.b;
        uint32_t ok0 = go.load(k0, phys0), ok1;
        if (first > 0) __syncthreads();
        stage_rows<T, D>(a, geo, g, first * 16, tiles, s_q, s_pos);
        for (int t = tid; t < tiles * 16; t += kWgtThreads) {
            float2 mi = make_float2(INFINITY, 0.f);
            const int r = first * 16 + t;
            if (r < geo.rows) {
                mi = join_parts(a, part_of(a, geo, g, r), nsplit, g * a.group + r - by_group(a, r) * a.group);
            }
            s_m[t] = mi.x;
            s_inv[t] = mi.y;
        }
        __syncthreads();
        auto step = [&](const Operand<T, D> (&k)[NB], const int (&phys)[NB], uint32_t ok, int b) {
            const float old = first == 0 ? load_old(ok, phys, b) : 0.f;
            float sum[NB];
#pragma unroll
            for (int x = 0; x < NB; ++x) sum[x] = 0.f;
            // (one tile at least, whatever there is: see weight_stats)
            for (int r = 0; r == 0 || r < tiles; ++r) {
                const bool masked = (b + NB) * kBlockTokens - 1 > __builtin_amdgcn_readfirstlane(s_pos[r * 16]);
                uint4 qv[NC];
#pragma unroll
                for (int c = 0; c < NC; ++c) qv[c] = s_q[(r * NC + c) * kWave + lane];
                const f32x4_t m = *reinterpret_cast<const f32x4_t*>(s_m + r * 16 + lg * 4);
                const f32x4_t inv = *reinterpret_cast<const f32x4_t*>(s_inv + r * 16 + lg * 4);
                const i32x4_t pos = *reinterpret_cast<const i32x4_t*>(s_pos + r * 16 + lg * 4);
                add_tile<T, D, NB>(a, qv, k, m, inv, masked, pos, b, sum);
            }
            // the four lane groups hold different rows of the same 16 keys
            float mine = 0.f;
            int block = 0;
            bool store = false;
#pragma unroll
            for (int x = 0; x < NB; ++x) {
                sum[x] = of_4_rows(sum[x]);
                if (lg == x) {
                    mine = sum[x];
                    block = phys[x];
                    store = (ok >> x) & 1u;
                }
            }
            const int t = (b + lg) * kBlockTokens + l16;
            if (store && t < geo.S) {
                const int64_t at = ((int64_t)block * a.hkv + g) * kBlockTokens + l16;
                if (first == 0) store_weight(a, geo, i, at, t, mine, old);
                else a.key_weights[at] += mine;
            }
        };
        constexpr int STEP = kWgtWaves * NB;
        int steps = b < b_hi ? (b_hi - b + STEP - 1) / STEP : 0;
        for (; steps > 1; steps -= 2) {
            ok1 = go.load(k1, phys1);
            step(k0, phys0, ok0, b);
            ok0 = go.load(k0, phys0);
            step(k1, phys1, ok1, b + STEP);
            b += 2 * STEP;
        }
        if (steps > 0) step(k0, phys0, ok0, b);
    }
}

// Many rows: the parts of every row joined, once.
__global__ __launch_bounds__(kWgtThreads) void weight_join(WgtArgs a) {
    const int i = blockIdx.y;
    const WgtGeom geo = wgt_geom(a, i);
    const int nsplit = (geo.blocks + a.split_blocks - 1) / a.split_blocks;
    const int g = blockIdx.x % a.hkv;
    for (int r = blockIdx.x / a.hkv * kWgtThreads + threadIdx.x; r < geo.rows; r += gridDim.x / a.hkv * kWgtThreads)
        rows_of(a, geo, g)[r] = join_parts(a, part_of(a, geo, g, r), nsplit, g * a.group + r - by_group(a, r) * a.group);
}

// Many rows: grid (KV heads x segments of the rows x ranges of sum_blocks blocks,
// requests).  Every wavefront holds keys of its own, and the segment's rows go by in
// LDS, 16 KiB at a time, the next ones in flight: read by every wavefront for itself
// (eight on the same 64 keys) they cost 92 us of the prompts' pass, since a KV head's
// query rows lie 1 KiB in 8 and meet in a quarter of the second level cache.
// Prompts are cut into segments because the rows are uneven work: the first keys are
// seen by all of them, the last by few.  weight_store adds the segments' sums.
template <typename T, int D>
__global__ __launch_bounds__(kWgtThreads) void weight_sums_rows(WgtArgs a) {
    constexpr int NB = held_blocks(D, sizeof(T) == 2), NC = Operand<T, D>::NC;
    constexpr int CT = row_tiles(D, sizeof(T) == 2);       // tiles of a chunk
    constexpr int LD = CT * NC * kWave / kWgtThreads;      // 16-byte pieces of it per thread
    constexpr int ROWS = CT * 16;
    __shared__ uint4 s_q[2][CT * NC * kWave];
    __shared__ __attribute__((aligned(16))) float2 s_mi[2][ROWS];  // the rows' m and 1 / l
    const int i = blockIdx.y;
    const int g = blockIdx.x % a.hkv, segment = blockIdx.x / a.hkv % a.segments;
    const int b_lo = blockIdx.x / a.hkv / a.segments * a.sum_blocks;
    const WgtGeom geo = wgt_geom(a, i);
    if (b_lo >= geo.blocks) return;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), l16 = lane & 15, lg = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int32_t* table = a.block_tables + (int64_t)i * a.max_blocks;
    const int p0 = geo.S - geo.n, b = b_lo + w * NB;
    Walk<T, D, NB> walk(a, table, g, b, geo.blocks);
    Operand<T, D> k[NB];
    int phys[NB] = {};
    const uint32_t ok = walk.load(k, phys);
    float sum[NB];
#pragma unroll
    for (int x = 0; x < NB; ++x) sum[x] = 0.f;

    // the segment's tiles, from that of the first row that sees the range's first key
    const int64_t skip = max((int64_t)0, (int64_t)b_lo * kBlockTokens - p0) * a.group;
    const int64_t first = max(skip / 16, (int64_t)segment * a.segment_tiles);
    // (the last segment takes the rows past those announced, too)
    const int all = (geo.rows + 15) / 16;
    const int last = segment == a.segments - 1 ? all : (int)min((int64_t)all, (int64_t)(segment + 1) * a.segment_tiles);
    const int chunks = first < last ? ((int)(last - first) + CT - 1) / CT : 0;
    const float2* stats = rows_of(a, geo, g);
    uint4 qr[LD];
    float2 mr;
    auto load = [&](int chunk) {
        const int row0 = ((int)first + chunk * CT) * 16;
#pragma unroll
        for (int x = 0; x < LD; ++x) {
            const int e = x * kWgtThreads + tid, ln = e % kWave, c = e / kWave % NC, tile = e / kWave / NC;
            const int r = min(row0 + tile * 16 + ln % 16, geo.rows - 1);  // (a place without a row: the last one)
            const int j = by_group(a, r), h = r - j * a.group;
            const T* src = static_cast<const T*>(a.q) + ((int64_t)(geo.q0 + j) * a.hq + g * a.group + h) * D +
                           (4 * c + ln / 16) * (16 / (int)sizeof(T));
            const u32x4u_t v = *reinterpret_cast<const u32x4u_t*>(src);
            qr[x] = make_uint4(v.x, v.y, v.z, v.w);
        }
        mr = stats[min(row0 + tid % ROWS, geo.rows - 1)];
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int x = 0; x < LD; ++x) s_q[buf][x * kWgtThreads + tid] = qr[x];
        if (tid < ROWS) s_mi[buf][tid] = mr;
    };
    if (chunks > 0) {
        load(0);
        put(0);
    }
    __syncthreads();
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int buf = chunk & 1;
        load(min(chunk + 1, chunks - 1));
        for (int t = 0; t < CT; ++t) {
            const int row = ((int)first + chunk * CT + t) * 16;
            if (row >= last * 16 || row >= geo.rows) break;
            const int p_lo = p0 + by_group(a, row), p_hi = p0 + by_group(a, min(row + 16, geo.rows) - 1);
            if (p_hi < b * kBlockTokens) continue;  // none of its rows sees the wavefront's keys
            const bool masked = (b + NB) * kBlockTokens - 1 > p_lo || row + 16 > geo.rows;
            i32x4_t pos = {};
            if (masked) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int rr = row + lg * 4 + e;
                    pos[e] = rr < geo.rows ? p0 + by_group(a, rr) : -1;
                }
            }
            uint4 qv[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) qv[c] = s_q[buf][(t * NC + c) * kWave + lane];
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(&s_mi[buf][t * 16 + lg * 4]);
            const f32x4_t y = *reinterpret_cast<const f32x4_t*>(&s_mi[buf][t * 16 + lg * 4 + 2]);
            add_tile<T, D, NB>(a, qv, k, f32x4_t{x[0], x[2], y[0], y[2]}, f32x4_t{x[1], x[3], y[1], y[3]}, masked, pos, b, sum);
        }
        put(buf ^ 1);
        __syncthreads();
    }
    // the four lane groups hold different rows of the same 16 keys
    float mine = 0.f;
    int block = 0;
    bool store = false;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
        sum[x] = of_4_rows(sum[x]);
        if (lg == x) {
            mine = sum[x];
            block = phys[x];
            store = (ok >> x) & 1u;
        }
    }
    const int t = (b + lg) * kBlockTokens + l16;
    if (!store || t >= geo.S) return;
    if (a.segments > 1) {
        a.sums[(((int64_t)i * a.hkv + g) * a.segments + segment) * a.sum_keys + t] = mine;
        return;
    }
    const int64_t at = ((int64_t)block * a.hkv + g) * kBlockTokens + l16;
    store_weight(a, geo, i, at, t, mine, t < p0 && a.decay != 0.f ? a.key_weights[at] : 0.f);
}

// Grid (KV heads x 256 keys, requests).
__global__ __launch_bounds__(kWgtThreads) void weight_store(WgtArgs a) {
    const int i = blockIdx.y, g = blockIdx.x % a.hkv, t = blockIdx.x / a.hkv * kWgtThreads + threadIdx.x;
    const WgtGeom geo = wgt_geom(a, i);
    if (t >= geo.S) return;
    const int id = a.block_tables[(int64_t)i * a.max_blocks + t / kBlockTokens];
    if (id < 0 || id >= a.num_blocks) return;
    const float* sums = a.sums + ((int64_t)i * a.hkv + g) * a.segments * a.sum_keys + t;
    float v = 0.f;
#pragma unroll 4
    for (int x = 0; x < a.segments; ++x) v += sums[(int64_t)x * a.sum_keys];
    const int64_t at = ((int64_t)id * a.hkv + g) * kBlockTokens + t % kBlockTokens;
    store_weight(a, geo, i, at, t, v, a.decay != 0.f && t < geo.S - geo.n ? a.key_weights[at] : 0.f);
}

// ------------------------------------------------------------------ host side

struct WgtPlan {
    int chunks, stat_tiles;  // weight_stats: row chunks, tiles per chunk
    int splits, split_blocks;
    int lds_tiles, sum_blocks, ranges;
    int stat_rows;           // rows times the group of a request, about
    bool once;
    int segments, segment_tiles;
    int score_rows, score_blocks;  // 0: the keys are read twice
    int64_t sum_keys;
    size_t rows_at, sums_at, bytes, cover;
};

int64_t tile_bytes(const verify_attn_params& p) {
    return 16 * (int64_t)p.head_dim * (p.dtype == VERIFY_BF16 ? 2 : 4);
}

constexpr int64_t kSumWgs = 2048;  // (request, KV head, range, segment)s that segments are made towards

int make_plan(const verify_attn_params& p, int32_t total_q, int32_t max_q_len, int32_t max_seq_len, WgtPlan* out) {
    WgtPlan pl{};
    const int64_t G = p.num_q_heads / p.num_kv_heads;
    const int64_t tiles = (G * std::max(1, max_q_len) + 15) / 16;
    const int64_t blocks = std::max<int64_t>(
        1, std::min<int64_t>(((int64_t)max_seq_len + kBlockTokens - 1) / kBlockTokens, p.max_blocks_per_seq));
    const bool bf16 = p.dtype == VERIFY_BF16;
    const int64_t step = kWgtWaves * step_blocks(p.head_dim, bf16);  // blocks of a workgroup's step
    // Every row chunk reads the keys again: as few as hold the tiles, evenly (64 requests
    // of 72 rows, head dim 64: 418 us with four tiles each, 294 with all five).  A
    // prompt's keys come from the cache, and it is better off with more wavefronts in a
    // compute unit (133 us with four tiles each, 146 with eight).
    const int64_t parts = tiles > 32 ? (tiles + 3) / 4 : (tiles + kStatTiles - 1) / kStatTiles;
    pl.stat_tiles = (int)((tiles + parts - 1) / parts);
    pl.chunks = (int)std::min<int64_t>(parts, 4096);
    // A split has at least a step, and at most 128 blocks, towards two workgroups per
    // compute unit in bf16 (eight requests of 2000 to 4096 keys, 36 rows: 28 us with 512
    // workgroups, 33 with 1024: each stages the rows and joins their parts) and eight in
    // fp32 (six requests of 500 to 4100 keys, 40 rows, head dim 64: 36 us with 1024, 27
    // with 2048; the products are 2.5 us of each pass, the rest those starts and ends).
    const int64_t want = bf16 ? 512 : 2048, most = (blocks + step - 1) / step, least = pl.chunks > 1 ? (blocks + 1023) / 1024 : (blocks + 127) / 128;
    const int64_t wgs = (int64_t)p.num_kv_heads * pl.chunks;
    auto split_of = [&](int64_t seqs) {  // its blocks, in a batch of `seqs` requests
        const int64_t ns = std::max(least, std::min(most, (want + seqs * wgs - 1) / (seqs * wgs)));
        return ((blocks + ns - 1) / ns + step - 1) / step * step;
    };
    pl.split_blocks = (int)split_of(std::max(1, p.num_seqs));
    pl.splits = (int)((blocks + pl.split_blocks - 1) / pl.split_blocks);
    pl.once = tiles * tile_bytes(p) <= 56 * 1024;
    if (pl.once) {
        pl.lds_tiles = (int)tiles;
        pl.sum_blocks = pl.split_blocks;
    } else {
        pl.sum_blocks = kWgtWaves * held_blocks(p.head_dim, bf16);
        pl.stat_rows = (int)std::min<int64_t>(tiles * 16, 1 << 20);
        // segments of 16 tiles at least, towards eight workgroups per compute unit (of a
        // prompt's half have nothing to do): two prompts of 2531 and 1300 rows, four heads
        // per KV head, 96 us in 6 segments, 76 in 12 and 16, 74 in 48, but then 14 instead
        // of 5 to add them
        const int64_t whole = std::max<int64_t>(1, p.num_seqs) * p.num_kv_heads * ((blocks + pl.sum_blocks - 1) / pl.sum_blocks);
        pl.segments = (int)std::max<int64_t>(1, std::min<int64_t>({16, tiles / 16, kSumWgs / whole}));
        pl.segment_tiles = (int)std::min<int64_t>((tiles + pl.segments - 1) / pl.segments, 1 << 27);
    }
    // a grid dimension holds fewer than 2^32 threads
    const int64_t ranges = (blocks + pl.sum_blocks - 1) / pl.sum_blocks * std::max(1, pl.segments);
    pl.ranges = (int)ranges;
    if (std::max<int64_t>(pl.splits * wgs, ranges * p.num_kv_heads) >= (1 << 24)) return VERIFY_EUNSUPPORTED;
    const size_t row = (size_t)p.num_q_heads * sizeof(float2);
    // the parts, and with many rows what they join into
    pl.rows_at = align_up(row * total_q * pl.splits, 256);
    const size_t joined = pl.once ? 0 : align_up(row * total_q, 256);
    pl.sum_keys = blocks * kBlockTokens;
    const size_t sums = pl.segments > 1 ? align_up((size_t)p.num_seqs * p.num_kv_heads * pl.segments * pl.sum_keys * sizeof(float), 256) : 0;
    // A row tile whose scores are at most a quarter of the keys' bytes to write and read:
    // 32 requests of 4097 keys, 4 rows, head dim 128: 94 us reading the keys twice, 63;
    // 16 requests of 2000 to 8000, 8 rows: 59 and 52; the same in fp32, 16 rows: 65 and 52;
    // where they are half, 8 rows at head dim 64: 59 and 60; 15 rows, four heads: 31 and 37.
    // Not where the requests' bounds exceed the cache twice over, and the scores with them.
    size_t scores = 0;
    const int64_t rows = align_up(G * std::max(1, max_q_len), 4), bounds = blocks * p.num_seqs, room = 2 * (int64_t)p.num_blocks;
    if (rows <= 16 && 4 * (2 * rows * kBlockTokens * (int64_t)sizeof(float)) <= tile_bytes(p)) {
        scores = (size_t)std::min(bounds, room) * p.num_kv_heads * rows * kBlockTokens * sizeof(float);
        if (bounds <= room) {
            pl.score_rows = (int)rows;
            pl.score_blocks = (int)blocks;
        }
    }
    pl.sums_at = pl.rows_at + joined;
    pl.bytes = pl.sums_at + sums + scores;
    // Any batch of fewer requests and rows: one request alone is cut into the most splits,
    // and all total_q rows may be its own, whatever max_q_len says.  Fewer requests may also
    // have more segments: kSumWgs of them at most in all.
    const size_t most_parts = row * total_q * (size_t)((blocks + split_of(1) - 1) / split_of(1));
    const int64_t key_ranges = (blocks + pl.sum_blocks - 1) / pl.sum_blocks;
    const size_t most_sums = pl.once ? 0 : align_up((size_t)(kSumWgs / key_ranges) * pl.sum_keys * sizeof(float), 256);
    pl.cover = align_up(most_parts, 256) + joined + std::max(sums, most_sums) + scores;
    *out = pl;
    return VERIFY_OK;
}

template <typename T, int D>
void launch(const WgtArgs& a, const WgtPlan& pl, hipStream_t stream) {
    const unsigned seqs = (unsigned)a.num_seqs;
    const dim3 stats((unsigned)((int64_t)a.hkv * pl.chunks * pl.splits), seqs), sums((unsigned)pl.ranges * a.hkv, seqs);
    auto run = [&](auto rt) {
        hipLaunchKernelGGL((weight_stats<T, D, decltype(rt)::value>), stats, dim3(kWgtThreads), 0, stream, a);
    };
    if (pl.score_rows > 0) {
        hipLaunchKernelGGL((weight_stats<T, D, 1, true>), stats, dim3(kWgtThreads), 0, stream, a);
    } else switch (pl.stat_tiles) {
        case 1: run(std::integral_constant<int, 1>{}); break;
        case 2: run(std::integral_constant<int, 2>{}); break;
        case 3: run(std::integral_constant<int, 3>{}); break;
        case 4: run(std::integral_constant<int, 4>{}); break;
        case 5: case 6: run(std::integral_constant<int, 6>{}); break;
        default: run(std::integral_constant<int, kStatTiles>{});
    }
    if (pl.once) {
        const size_t lds = (size_t)pl.lds_tiles * (Operand<T, D>::NC * kWave * sizeof(uint4) + 3 * 16 * sizeof(float));
        if (pl.score_rows > 0) hipLaunchKernelGGL((weight_sums<T, D, true>), sums, dim3(kWgtThreads), lds, stream, a);
        else hipLaunchKernelGGL((weight_sums<T, D, false>), sums, dim3(kWgtThreads), lds, stream, a);
        return;
    }
    const dim3 join((unsigned)((pl.stat_rows + kWgtThreads - 1) / kWgtThreads * a.hkv), seqs);
    hipLaunchKernelGGL(weight_join, join, dim3(kWgtThreads), 0, stream, a);
    hipLaunchKernelGGL((weight_sums_rows<T, D>), sums, dim3(kWgtThreads), 0, stream, a);
    const dim3 store((unsigned)((pl.sum_keys + kWgtThreads - 1) / kWgtThreads * a.hkv), seqs);
    if (a.segments > 1) hipLaunchKernelGGL(weight_store, store, dim3(kWgtThreads), 0, stream, a);
}

int check(const verify_attn_params* p, int32_t total_q, int32_t max_q_len, int32_t max_seq_len) {
    const int rc = validate(p, total_q, max_q_len, max_seq_len);
    if (rc != VERIFY_OK) return rc;
    if (p->sliding_window > 0) return VERIFY_EUNSUPPORTED;
    const int64_t group = p->num_q_heads / p->num_kv_heads;
    const int64_t rows = ((int64_t)total_q + 1) * group;  // see by_group
    if (rows >= (1 << 30) || rows * (group - 1) >= ((int64_t)1 << 32)) return VERIFY_EUNSUPPORTED;
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
    if (((uintptr_t)k_cache | (uintptr_t)workspace) & 15) return VERIFY_EINVAL;
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
    a.rows = reinterpret_cast<float2*>(static_cast<char*>(workspace) + pl.rows_at);
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
    a.group_magic = (uint32_t)((((uint64_t)1 << 32) + a.group - 1) / a.group);
    a.splits = pl.splits;
    a.split_blocks = pl.split_blocks;
    a.chunks = pl.chunks;
    a.sum_blocks = pl.sum_blocks;
    a.lds_tiles = pl.lds_tiles;
    a.segments = pl.segments;
    a.segment_tiles = pl.segment_tiles;
    a.sum_keys = pl.sum_keys;
    a.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.sums_at);
    a.scores = reinterpret_cast<f32x4_t*>(a.sums);  // (either, never both)
    a.score_rows = pl.score_rows;
    a.score_blocks = pl.score_blocks;
    if (p.dtype == VERIFY_BF16)
        p.head_dim == 128 ? launch<uint16_t, 128>(a, pl, stream) : launch<uint16_t, 64>(a, pl, stream);
    else
        p.head_dim == 128 ? launch<float, 128>(a, pl, stream) : launch<float, 64>(a, pl, stream);
    return check_launch();
}
