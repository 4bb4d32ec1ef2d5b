// verify_rotary.hip -- rotary positions on one or several axes, of the scored rows'
// queries and keys, alone or with the append to the paged cache.
//
// A pair (a, b) of a head's dims is multiplied by e^(i x), x = position * inv_freq.
// Every head of a row turns by the same R / 2 angles, so a workgroup takes a tile of
// kTile packed rows and some of the heads: it computes the tile's sines and cosines
// once into LDS and then streams the heads past them, 16 bytes per thread and load.
//
// The angle.  Only the fraction of a turn of position * inv_freq / 2 pi matters, and
// a product in fp32 has lost it at positions of a few ten thousands.  It is taken in
// binary64, its integer part is removed there, and sine and cosine are evaluated in
// fp32 on a half turn at most.
//
// The append.  K goes to its slots in the 16-byte chunks that the cache keeps
// together; V, which the cache keeps transposed, passes through LDS.  Threads run
// over a tile's rows first, so that the consecutive slots of a prompt's rows leave in
// whole cache lines.
#include <type_traits>

#include "common.h"

namespace averify {
namespace {

constexpr int kRotThreads = 256;
constexpr int kTile = 16;           // packed rows of a workgroup
constexpr int kMaxFreqs = 64;       // head_dim 128 rotated whole
constexpr int kSearchEntries = 1024; // of q_start, kept in LDS to find the rows' requests

struct RotArgs {
    const void* q;
    const void* k;
    const void* v;
    const int32_t* positions;
    const double* inv_freq;
    void* q_out;
    void* k_out;  // rotated keys, or with APPEND the key cache
    void* v_out;  // APPEND: the value cache
    const int32_t* block_tables;
    const int32_t* seq_lens;
    const int32_t* q_start;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    int total_q, hq, hkv, num_axes, freqs, heads_per_wg;
    int num_seqs, max_blocks, num_blocks;
    float scale;
    uint8_t axis[kMaxFreqs];
};

// A row's place in the cache: block id (-1: not stored) and slot.
struct Place {
    int32_t block, slot;
};

// The places of the tile's rows.  A row's request is the last with q_start <= row:
// the first entries of q_start, or evenly spaced ones of a larger batch, are searched
// in LDS (a dependent read of global memory per step of a binary search would cost
// several times the rest of a small call), the entries between two of them in memory.
__device__ __forceinline__ void find_places(const RotArgs& a, int row0, int rows, int32_t* s_start, Place* place) {
    const int tid = threadIdx.x;
    const int every = (a.num_seqs + kSearchEntries - 1) / kSearchEntries;
    const int entries = (a.num_seqs + every - 1) / every;
    for (int e = tid; e < entries; e += kRotThreads) s_start[e] = a.q_start[e * every];
    __syncthreads();
    if (tid < rows) {
        const int row = row0 + tid;
        int lo = 0, hi = entries - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s_start[mid] <= row) lo = mid; else hi = mid - 1;
        }
        int i = lo * every, end = min(i + every, a.num_seqs) - 1;
        while (i < end) {
            const int mid = (i + end + 1) >> 1;
            if (a.q_start[mid] <= row) i = mid; else end = mid - 1;
        }
        const int q0 = a.q_start[i], q1 = a.q_start[i + 1];
        Place p{-1, 0};
        const int64_t pos = (int64_t)a.seq_lens[i] - ((int64_t)q1 - row);
        if (q0 <= row && row < q1 && pos >= 0 && pos / kBlockTokens < a.max_blocks) {
            const int id = a.block_tables[(int64_t)i * a.max_blocks + pos / kBlockTokens];
            p.block = id >= 0 && id < a.num_blocks ? id : -1;
            p.slot = (int)(pos % kBlockTokens);
        }
        place[tid] = p;
    }
}

template <typename T> struct Vec;  // 16 bytes of storage elements
template <> struct Vec<uint16_t> {
    static constexpr int N = 8;
    static __device__ uint4 pack(const float* f) {
        return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                          pack_bf16x2(f[6], f[7]));
    }
};
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

__device__ __forceinline__ void turn(float& x, float& y, const float2& cs) {
    // explicit, so that every layout's code rounds alike
    const float a = x, b = y;
    x = fmaf(-b, cs.y, a * cs.x);
    y = fmaf(b, cs.x, a * cs.y);
}

// WIDE: all rows and pair halves are 16-byte aligned; otherwise element by element.
// INTER: the pair of frequency f is (2f, 2f + 1).
template <typename T, int D, bool APPEND, bool WIDE, bool INTER>
__global__ __launch_bounds__(kRotThreads) void rotate_rows(RotArgs a) {
    constexpr int N = Vec<T>::N;
    constexpr int CH = D / N;  // 16-byte chunks of a head
    __shared__ float2 cs[kTile][kMaxFreqs];
    __shared__ Place place[kTile];
    // the search's entries, then the values of one head
    __shared__ uint4 scratch[kTile * (CH + 1) > kSearchEntries / 4 ? kTile * (CH + 1) : kSearchEntries / 4];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const int row0 = blockIdx.x * kTile;
    const int rows = min(kTile, a.total_q - row0);
    // heads in the order K, V, Q: the first two have the longer way
    const int kv_heads = APPEND ? 2 * a.hkv : a.hkv;
    const int h_lo = blockIdx.y * a.heads_per_wg;
    const int h_hi = min(h_lo + a.heads_per_wg, kv_heads + a.hq);

    // angles: a wavefront per row, a frequency per lane
    if (lane < a.freqs) {
        const double turns_per = a.inv_freq[lane] * 0.15915494309189533577;  // 1 / 2 pi
        const int32_t* pos = a.positions + (int64_t)a.axis[lane] * a.total_q + row0;
        for (int r = wv; r < rows; r += kRotThreads / kWave) {
            const double t = (double)pos[r] * turns_per;
            float sn, cn;
            sincospif(2.f * (float)(t - rint(t)), &sn, &cn);
            cs[r][lane] = make_float2(cn * a.scale, sn * a.scale);
        }
    }
    if constexpr (APPEND) {
        if (h_lo < kv_heads) find_places(a, row0, rows, reinterpret_cast<int32_t*>(scratch), place);
    }
    __syncthreads();

    const int half = a.freqs;  // the distance of a pair's dims, unless INTER
    if constexpr (WIDE) {
        // An item is what one thread turns: a chunk (INTER), or a chunk of first
        // dims with the chunk of their partners; then the chunks that pass through.
        const int turned = INTER ? 2 * half / N : half / N;
        const int items = turned + (CH - 2 * half / N);
        auto item_chunks = [&](int it, int& c0, int& c1) {
            c0 = it;
            c1 = !INTER && it < turned ? it + half / N : -1;
            if (it >= turned) c0 = 2 * half / N + (it - turned);
        };
        auto turn_item = [&](int it, int r, uint4& v0, uint4& v1) {
            if (it >= turned) return;
            float x[N], y[N];
            unpack16(v0, x, T{});
            if constexpr (INTER) {
#pragma unroll
                for (int e = 0; e < N; e += 2) turn(x[e], x[e + 1], cs[r][it * (N / 2) + e / 2]);
            } else {
                unpack16(v1, y, T{});
#pragma unroll
                for (int e = 0; e < N; ++e) turn(x[e], y[e], cs[r][it * N + e]);
                v1 = Vec<T>::pack(y);
            }
            v0 = Vec<T>::pack(x);
        };
        // heads [lo, hi) of rows, row to row: items fastest
        auto rotate_heads = [&](const T* in, int64_t in_stride, T* out, int64_t out_stride, int lo, int hi) {
            int sh = 0;
            while ((1 << sh) < items) ++sh;
            const int it = tid & ((1 << sh) - 1);
            if (it >= items) return;
            int c0, c1;
            item_chunks(it, c0, c1);
            for (int u = tid >> sh; u < (hi - lo) * kTile; u += kRotThreads >> sh) {
                const int r = u % kTile, h = lo + u / kTile;
                if (r >= rows) continue;
                const T* src = in + (row0 + r) * in_stride + (int64_t)h * D;
                uint4 v0 = ld16(src + c0 * N), v1 = make_uint4(0, 0, 0, 0);
                if (c1 >= 0) v1 = ld16(src + c1 * N);
                turn_item(it, r, v0, v1);
                T* dst = out + (row0 + r) * out_stride + (int64_t)h * D;
                *reinterpret_cast<uint4*>(dst + c0 * N) = v0;
                if (c1 >= 0) *reinterpret_cast<uint4*>(dst + c1 * N) = v1;
            }
        };
        const int r = tid % kTile;
        if constexpr (APPEND) {
            const T* kin = static_cast<const T*>(a.k) + (row0 + r) * a.k_stride;
            const int64_t tile = (int64_t)D * kBlockTokens;
            const bool store = r < rows && place[r].block >= 0;
            const Place p = store ? place[r] : Place{0, 0};
            for (int h = h_lo; h < min(h_hi, a.hkv); ++h) {
                T* to = static_cast<T*>(a.k_out) + ((int64_t)p.block * a.hkv + h) * tile + p.slot * N;
                for (int it = tid / kTile; it < items && store; it += kRotThreads / kTile) {
                    int c0, c1;
                    item_chunks(it, c0, c1);
                    uint4 v0 = ld16(kin + h * D + c0 * N), v1 = make_uint4(0, 0, 0, 0);
                    if (c1 >= 0) v1 = ld16(kin + h * D + c1 * N);
                    turn_item(it, r, v0, v1);
                    *reinterpret_cast<uint4*>(to + c0 * (kBlockTokens * N)) = v0;
                    if (c1 >= 0) *reinterpret_cast<uint4*>(to + c1 * (kBlockTokens * N)) = v1;
                }
            }
            for (int h = max(h_lo, a.hkv) - a.hkv; h < min(h_hi, kv_heads) - a.hkv; ++h) {
                __syncthreads();  // the search, or the head before, is done with scratch
                for (int e = tid; e < rows * CH; e += kRotThreads)
                    scratch[e / CH * (CH + 1) + e % CH] =
                        ld16(static_cast<const T*>(a.v) + (row0 + e / CH) * a.v_stride + h * D + e % CH * N);
                __syncthreads();
                T* to = static_cast<T*>(a.v_out) + ((int64_t)p.block * a.hkv + h) * tile + p.slot;
                const T* from = reinterpret_cast<const T*>(scratch + r * (CH + 1));
                if (store)
                    for (int d = tid / kTile; d < D; d += kRotThreads / kTile) to[d * kBlockTokens] = from[d];
            }
        } else if (a.k) {
            rotate_heads(static_cast<const T*>(a.k), a.k_stride, static_cast<T*>(a.k_out), a.k_out_stride, h_lo,
                         min(h_hi, a.hkv));
        }
        rotate_heads(static_cast<const T*>(a.q), a.q_stride, static_cast<T*>(a.q_out), a.q_out_stride,
                     max(h_lo, kv_heads) - kv_heads, h_hi - kv_heads);
    } else {
        // an item is a pair, or two neighbouring dims that pass through
        for (int u = tid; u < (h_hi - h_lo) * kTile * (D / 2); u += kRotThreads) {
            const int it = u % (D / 2), r = u / (D / 2) % kTile, hh = h_lo + u / (D / 2) / kTile;
            if (r >= rows) continue;
            const bool key = hh < a.hkv, value = !key && hh < kv_heads;
            const int h = key ? hh : value ? hh - a.hkv : hh - kv_heads;
            const bool turned = it < half && !value;
            const int d0 = turned && !INTER ? it : 2 * it, d1 = turned && !INTER ? it + half : 2 * it + 1;
            const T* src = static_cast<const T*>(key ? a.k : value ? a.v : a.q) +
                           (row0 + r) * (key ? a.k_stride : value ? a.v_stride : a.q_stride) + (int64_t)h * D;
            T x = src[d0], y = src[d1];  // bits, kept as they are unless turned
            if (turned) {
                float fx = Storage<T>::load(&x, 0), fy = Storage<T>::load(&y, 0);
                turn(fx, fy, cs[r][it]);
                Storage<T>::store(&x, 0, fx);
                Storage<T>::store(&y, 0, fy);
            }
            if (APPEND && (key || value)) {
                const Place p = place[r];
                if (p.block < 0) continue;
                T* to = static_cast<T*>(key ? a.k_out : a.v_out) + ((int64_t)p.block * a.hkv + h) * D * kBlockTokens;
                auto at = [&](int d) { return key ? (d / N * kBlockTokens + p.slot) * N + d % N : d * kBlockTokens + p.slot; };
                to[at(d0)] = x;
                to[at(d1)] = y;
            } else {
                T* dst = static_cast<T*>(key ? a.k_out : a.q_out) +
                         (row0 + r) * (key ? a.k_out_stride : a.q_out_stride) + (int64_t)h * D;
                dst[d0] = x;
                dst[d1] = y;
            }
        }
    }
}

int check_params(const verify_rotary_params* p, int32_t total_q, int32_t hq, int32_t hkv) {
    if (!p) return VERIFY_EINVAL;
    if (p->dtype != VERIFY_F32 && p->dtype != VERIFY_BF16) return VERIFY_EUNSUPPORTED;
    if (p->head_dim != 64 && p->head_dim != 128) return VERIFY_EUNSUPPORTED;
    if (p->rotary_dim < 2 || p->rotary_dim > p->head_dim || p->rotary_dim % 2) return VERIFY_EINVAL;
    if (p->num_axes < 1 || p->num_axes > VERIFY_ROTARY_MAX_AXES) return VERIFY_EINVAL;
    if (p->interleaved != 0 && p->interleaved != 1) return VERIFY_EINVAL;
    if (!(p->scale >= 0.f) || p->scale > 3.0e38f) return VERIFY_EINVAL;
    for (int f = 0; f < p->rotary_dim / 2; ++f)
        if (p->axis[f] >= p->num_axes) return VERIFY_EINVAL;
    if (total_q < 0 || hq < 1 || hkv < 0) return VERIFY_EINVAL;
    if (hq > 32768 || hkv > 16384) return VERIFY_EUNSUPPORTED;  // grid y
    return VERIFY_OK;
}

template <typename T, int D, bool APPEND>
void launch(const RotArgs& a, const verify_rotary_params& p, bool wide, hipStream_t stream) {
    const int heads = a.hq + (APPEND ? 2 : 1) * a.hkv;
    const dim3 grid((unsigned)(((int64_t)a.total_q + kTile - 1) / kTile),
                    (unsigned)((heads + a.heads_per_wg - 1) / a.heads_per_wg));
    auto run = [&](auto w, auto inter) {
        hipLaunchKernelGGL((rotate_rows<T, D, APPEND, decltype(w)::value, decltype(inter)::value>), grid,
                           dim3(kRotThreads), 0, stream, a);
    };
    if (p.interleaved) wide ? run(std::true_type{}, std::true_type{}) : run(std::false_type{}, std::true_type{});
    else wide ? run(std::true_type{}, std::false_type{}) : run(std::false_type{}, std::false_type{});
}

// Fills in what both calls share and launches.
template <bool APPEND>
int rotary_call(RotArgs& a, const verify_rotary_params& p, hipStream_t stream) {
    a.num_axes = p.num_axes;
    a.freqs = p.rotary_dim / 2;
    a.scale = p.scale > 0.f ? p.scale : 1.f;
    for (int f = 0; f < a.freqs; ++f) a.axis[f] = p.axis[f];
    // Heads per workgroup: two where the rows are few (more workgroups, each done
    // sooner), as many as leave four workgroups per compute unit otherwise (every
    // workgroup computes its tile's angles).
    const int heads = a.hq + (APPEND ? 2 : 1) * a.hkv;
    const int64_t tiles = ((int64_t)a.total_q + kTile - 1) / kTile;
    const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>((heads + 1) / 2, 4 * device_cus() / tiles));
    a.heads_per_wg = (int)((heads + chunks - 1) / chunks);
    const int esize = p.dtype == VERIFY_BF16 ? 2 : 4, n = 16 / esize;
    uint64_t bits = (uint64_t)(uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.q_out | (uintptr_t)a.k_out;
    const int64_t strides = a.q_stride | a.k_stride | a.v_stride | a.q_out_stride | a.k_out_stride;
    const int step = p.interleaved ? p.rotary_dim : a.freqs;
    const bool wide = (bits & 15) == 0 && strides % n == 0 && step % n == 0;
    if (p.dtype == VERIFY_BF16)
        p.head_dim == 128 ? launch<uint16_t, 128, APPEND>(a, p, wide, stream) : launch<uint16_t, 64, APPEND>(a, p, wide, stream);
    else
        p.head_dim == 128 ? launch<float, 128, APPEND>(a, p, wide, stream) : launch<float, 64, APPEND>(a, p, wide, stream);
    return check_launch();
}

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_rotary(const verify_rotary_params* params, int32_t total_q, int32_t num_q_heads,
                             int32_t num_kv_heads, const void* q, int64_t q_stride, const void* k,
                             int64_t k_stride, const int32_t* positions, const double* inv_freq,
                             void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                             hipStream_t stream) {
    const int rc = check_params(params, total_q, num_q_heads, num_kv_heads);
    if (rc != VERIFY_OK) return rc;
    const int64_t wq = (int64_t)num_q_heads * params->head_dim, wk = (int64_t)num_kv_heads * params->head_dim;
    if (q_stride < wq || q_out_stride < wq || (num_kv_heads > 0 && (k_stride < wk || k_out_stride < wk)))
        return VERIFY_EINVAL;
    if (total_q == 0) return VERIFY_OK;
    if (!q || !q_out || !positions || !inv_freq) return VERIFY_EINVAL;
    if ((num_kv_heads > 0) != (k != nullptr) || (num_kv_heads > 0) != (k_out != nullptr)) return VERIFY_EINVAL;
    if ((q == q_out && q_stride != q_out_stride) || (k && k == k_out && k_stride != k_out_stride))
        return VERIFY_EINVAL;
    RotArgs a{};
    a.q = q;
    a.k = k;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.k_out = k_out;
    a.q_stride = q_stride;
    a.q_out_stride = q_out_stride;
    if (k) {
        a.k_stride = k_stride;
        a.k_out_stride = k_out_stride;
    }
    a.total_q = total_q;
    a.hq = num_q_heads;
    a.hkv = num_kv_heads;
    return rotary_call<false>(a, *params, stream);
}

extern "C" int verify_rotary_append(const verify_attn_params* attn, const verify_rotary_params* params,
                                    int32_t total_q, const void* q, int64_t q_stride, const void* k_new,
                                    int64_t k_stride, const void* v_new, int64_t v_stride,
                                    const int32_t* positions, const double* inv_freq,
                                    const int32_t* block_tables, const int32_t* seq_lens,
                                    const int32_t* q_start, void* q_out, int64_t q_out_stride,
                                    void* k_cache, void* v_cache, hipStream_t stream) {
    int rc = validate(attn, total_q, 0, 0);
    if (rc == VERIFY_OK) rc = check_params(params, total_q, attn->num_q_heads, attn->num_kv_heads);
    if (rc != VERIFY_OK) return rc;
    if (params->head_dim != attn->head_dim || params->dtype != attn->dtype) return VERIFY_EINVAL;
    const int64_t wq = (int64_t)attn->num_q_heads * attn->head_dim, wk = (int64_t)attn->num_kv_heads * attn->head_dim;
    if (q_stride < wq || q_out_stride < wq || k_stride < wk || v_stride < wk) return VERIFY_EINVAL;
    if (total_q == 0) return VERIFY_OK;
    if (attn->num_seqs == 0)  // rows of no request: the queries alone
        return verify_rotary(params, total_q, attn->num_q_heads, 0, q, q_stride, nullptr, 0, positions, inv_freq,
                             q_out, q_out_stride, nullptr, 0, stream);
    if (!q || !q_out || !positions || !inv_freq || !k_new || !v_new || !block_tables || !seq_lens || !q_start ||
        !k_cache || !v_cache)
        return VERIFY_EINVAL;
    if ((uintptr_t)k_cache & 15) return VERIFY_EINVAL;
    if (q == q_out && q_stride != q_out_stride) return VERIFY_EINVAL;
    RotArgs a{};
    a.q = q;
    a.k = k_new;
    a.v = v_new;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.k_out = k_cache;
    a.v_out = v_cache;
    a.block_tables = block_tables;
    a.seq_lens = seq_lens;
    a.q_start = q_start;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out_stride = q_out_stride;
    a.total_q = total_q;
    a.hq = attn->num_q_heads;
    a.hkv = attn->num_kv_heads;
    a.num_seqs = attn->num_seqs;
    a.max_blocks = attn->max_blocks_per_seq;
    a.num_blocks = attn->num_blocks;
    return rotary_call<true>(a, *params, stream);
}
