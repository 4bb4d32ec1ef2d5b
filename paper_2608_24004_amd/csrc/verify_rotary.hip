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
// What bounds it: memory, above a few thousand rows (5461 rows of 40 heads of 128, 112
// MB: 27 us, 4.2 TB/s); below, a launch and the latencies of positions, rows and, for
// the append, of q_start, the request's length and its block ids.
//
// The append.  K goes to its slots in the 16-byte chunks that the cache keeps
// together; V, which the cache keeps transposed, passes through LDS.  Threads run
// over a tile's rows first, so that the consecutive slots of a prompt's rows leave in
// whole cache lines.
#include <type_traits>

#include "rotary.h"

namespace averify {
namespace {

// Heads of K that a workgroup takes (their chunks pass through registers, all loads
// before the first store).
constexpr int kKeyHeads = 4;
// Of Q at most: 5461 rows of 32 heads 26.9 us with 8 or fewer, 28.8 with 16, 30.7 with 24.
constexpr int kQueryHeads = 8;
constexpr int batch(bool inter) { return inter ? 4 : 1; }  // query items of a thread in flight

// Workgroup (tile, y): y below key_wgs takes keys, below key_wgs + value_wgs values,
// the others queries.  Keys and values come first: theirs is the longer way.
// WIDE: all rows and pair halves are 16-byte aligned; otherwise element by element.
// INTER: the pair of frequency f is (2f, 2f + 1).
template <typename T, int D, bool APPEND, bool WIDE, bool INTER>
__global__ __launch_bounds__(kRotThreads) void rotate_rows(RotArgs a) {
    constexpr int N = Vec<T>::N;
    constexpr int CH = D / N;  // 16-byte chunks of a head
    constexpr int VH = value_heads((int)sizeof(T)), kBatch = batch(INTER);
    constexpr int PLACE = APPEND ? kSearchEntries / 4 : 0, VALUES = APPEND && WIDE ? VH * kTile * (CH + 1) : 0;
    __shared__ float2 cs[kTile][kMaxFreqs];
    __shared__ Place place[kTile];
    __shared__ uint4 s_start[PLACE ? PLACE : 1];
    __shared__ uint4 s_val[VALUES ? VALUES : 1];
    const int tid = threadIdx.x;
    // Workgroups go round the eight XCDs: each takes neighbouring tiles, whose rows share
    // cache lines of the paged cache (six prompts of 12 thousand rows in all: 60 -> 56 us).
    const int xq = gridDim.x / 8, xr = gridDim.x % 8, xcd = blockIdx.x % 8;
    const int row0 = (xcd * xq + min(xcd, xr) + (int)(blockIdx.x / 8)) * kTile;
    const int rows = min(kTile, a.total_q - row0);
    const int y = blockIdx.y;
    const bool key = y < a.key_wgs, value = !key && y < a.key_wgs + a.value_wgs;
    const int per = key ? kKeyHeads : value ? VH : a.heads_per_wg;
    const int h_lo = (key ? y : value ? y - a.key_wgs : y - a.key_wgs - a.value_wgs) * per;
    const int h_hi = min(h_lo + per, key || value ? a.hkv : a.hq);

    // angles: a frequency per lane; with 32 or fewer of them two rows per wavefront
    const int fsh = a.freqs <= 32 ? 5 : 6;
    auto angles = [&]() {
        const int f = tid & ((1 << fsh) - 1), r0 = tid >> fsh, step = kRotThreads >> fsh;
        if (f >= a.freqs) return;
        const double turns_per = a.inv_freq[f] * 0.15915494309189533577;  // 1 / 2 pi
        const int32_t* pos = a.positions + (int64_t)a.axis[f] * a.total_q + row0;
        for (int r = r0; r < rows; r += step) cs[r][f] = unit_circle((double)pos[r] * turns_per, a.scale);
    };

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
        auto load_item = [&](const T* head, int c0, int c1, u32x4& v0, u32x4& v1) {
            v0 = *reinterpret_cast<const u32x4*>(head + c0 * N);
            if (!INTER) v1 = *reinterpret_cast<const u32x4*>(head + (c1 >= 0 ? c1 : c0) * N);
        };
        auto turn_item = [&](int it, int r, u32x4& v0, u32x4& v1) {
            if (it >= turned) return;
            float x[N], y[N];
            unpack16(make_uint4(v0.x, v0.y, v0.z, v0.w), x, T{});
            if constexpr (INTER) {
#pragma unroll
                for (int e = 0; e < N; e += 2) turn(x[e], x[e + 1], cs[r][it * (N / 2) + e / 2]);
            } else {
                unpack16(make_uint4(v1.x, v1.y, v1.z, v1.w), y, T{});
#pragma unroll
                for (int e = 0; e < N; ++e) turn(x[e], y[e], cs[r][it * N + e]);
                const uint4 w = Vec<T>::pack(y);
                v1 = u32x4{w.x, w.y, w.z, w.w};
            }
            const uint4 w = Vec<T>::pack(x);
            v0 = u32x4{w.x, w.y, w.z, w.w};
        };
        if (APPEND && key) {
            // a thread per row and item, its chunks of every head of the workgroup
            const int r = tid % kTile, it = tid / kTile;
            const T* in = static_cast<const T*>(a.k) + (row0 + min(r, rows - 1)) * a.k_stride;
            for (int base = it; base - it < items; base += kRotThreads / kTile) {
                const int my = min(base, items - 1);
                int c0, c1;
                item_chunks(my, c0, c1);
                u32x4 v0[kKeyHeads], v1[kKeyHeads];
#pragma unroll
                for (int x = 0; x < kKeyHeads; ++x) load_item(in + min(h_lo + x, h_hi - 1) * D, c0, c1, v0[x], v1[x]);
                if (base == it) {
                    angles();
                    find_places(a, row0, rows, reinterpret_cast<int32_t*>(s_start), place);
                    __syncthreads();
                }
                const Place p = r < rows ? place[r] : Place{-1, 0};
                if (p.block < 0 || base >= items) continue;
#pragma unroll
                for (int x = 0; x < kKeyHeads; ++x) {
                    if (h_lo + x >= h_hi) break;
                    turn_item(my, r, v0[x], v1[x]);
                    T* to = static_cast<T*>(a.k_out) + ((int64_t)p.block * a.hkv + h_lo + x) * (D * kBlockTokens) + p.slot * N;
                    *reinterpret_cast<u32x4*>(to + c0 * (kBlockTokens * N)) = v0[x];
                    if (c1 >= 0) *reinterpret_cast<u32x4*>(to + c1 * (kBlockTokens * N)) = v1[x];
                }
            }
        } else if (APPEND && value) {
            store_values<T, D>(a, row0, rows, h_lo, h_hi, reinterpret_cast<int32_t*>(s_start), place, s_val);
        } else {
            // row to row: items fastest, kBatch of a thread in flight (every thread's loads
            // are made, of the last row and item past the end: with a test before each the
            // prompts of append took 60 us, 56 without)
            const T* in = static_cast<const T*>(key ? a.k : a.q);
            T* out = static_cast<T*>(key ? a.k_out : a.q_out);
            const int64_t in_stride = key ? a.k_stride : a.q_stride, out_stride = key ? a.k_out_stride : a.q_out_stride;
            int sh = 0;
            while ((1 << sh) < items) ++sh;
            const int my = tid & ((1 << sh) - 1), it = min(my, items - 1);
            int c0, c1;
            item_chunks(it, c0, c1);
            const int step = kRotThreads >> sh, all = (h_hi - h_lo) * kTile;
            angles();
            __syncthreads();
            for (int base = 0; base < all; base += kBatch * step) {
                const int u0 = base + (tid >> sh);
                u32x4 v0[kBatch], v1[kBatch];
#pragma unroll
                for (int x = 0; x < kBatch; ++x) {
                    const int u = min(u0 + x * step, all - 1);
                    load_item(in + (row0 + min(u % kTile, rows - 1)) * in_stride + (int64_t)(h_lo + u / kTile) * D, c0, c1,
                              v0[x], v1[x]);
                }
#pragma unroll
                for (int x = 0; x < kBatch; ++x) {
                    const int u = u0 + x * step, r = u % kTile;
                    if (my >= items || u >= all || r >= rows) continue;
                    turn_item(it, r, v0[x], v1[x]);
                    T* dst = out + (row0 + r) * out_stride + (int64_t)(h_lo + u / kTile) * D;
                    *reinterpret_cast<u32x4*>(dst + c0 * N) = v0[x];
                    if (c1 >= 0) *reinterpret_cast<u32x4*>(dst + c1 * N) = v1[x];
                }
            }
        }
    } else {
        if (!value) angles();
        if (APPEND && (key || value)) find_places(a, row0, rows, reinterpret_cast<int32_t*>(s_start), place);
        __syncthreads();
        // an item is a pair, or two neighbouring dims that pass through
        for (int u = tid; u < (h_hi - h_lo) * kTile * (D / 2); u += kRotThreads) {
            const int it = u % (D / 2), r = u / (D / 2) % kTile, h = h_lo + u / (D / 2) / kTile;
            if (r >= rows) continue;
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

template <typename T, int D, bool APPEND>
void launch(const RotArgs& a, const verify_rotary_params& p, bool wide, hipStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)a.total_q + kTile - 1) / kTile),
                    (unsigned)(a.key_wgs + a.value_wgs + (a.hq + a.heads_per_wg - 1) / a.heads_per_wg));
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
    a.freqs = p.rotary_dim / 2;
    a.scale = p.scale > 0.f ? p.scale : 1.f;
    for (int f = 0; f < a.freqs; ++f) a.axis[f] = p.axis[f];
    // Query heads per workgroup: two where the rows are few (more workgroups, each done
    // sooner), up to kQueryHeads otherwise (every workgroup computes its tile's angles).
    const int64_t tiles = ((int64_t)a.total_q + kTile - 1) / kTile;
    const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>((a.hq + 1) / 2, 8 * device_cus() / tiles));
    a.heads_per_wg = (int)std::min<int64_t>((a.hq + chunks - 1) / chunks, kQueryHeads);
    a.key_wgs = (a.hkv + kKeyHeads - 1) / kKeyHeads;
    const int esize = p.dtype == VERIFY_BF16 ? 2 : 4, n = 16 / esize;
    if (APPEND) a.value_wgs = (a.hkv + value_heads(esize) - 1) / value_heads(esize);
    const uint64_t bits = (uint64_t)(uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.q_out | (uintptr_t)a.k_out;
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
