// verify_norm_rotary.hip -- queries and keys brought to one length per head and turned to
// their positions, alone or with the append to the paged cache.
//
// A head x of D dims becomes x * rsqrt(mean(x^2) + eps) * weight, then its pairs are
// multiplied by e^(i position inv_freq) as verify_rotary does.  Sums, norm and rotation
// are in fp32, with one rounding at the store: a norm and a rotation in calls of their
// own would round twice and move every byte twice.
//
// The threads of a head are neighbours in a wavefront, each with a chunk of 16 bytes and
// the chunk of its dims' partners, so that a head's sum of squares takes a few exchanges
// between lanes and no memory.  A thread keeps the weights of its dims for all the heads
// that it takes, multiplied into the sine and cosine of its row: a matrix per pair that
// is the same for all heads.  Loads leave before the angles are computed.
//
// What bounds it: memory above a few thousand rows (5461 rows of 40 heads of 128, 112 MB:
// 29.6 us, 3.8 TB/s; with the weights' and the rotation's products apart, eight-way bank
// conflicts on the angles and 128 bytes of a thread under way 36); below, a launch and
// the latencies of positions, rows and, for the append, of q_start, the request's length
// and block ids.
#include <type_traits>

#include "rotary.h"

namespace averify {
namespace {

struct NormArgs {
    RotArgs r;
    const float* q_weight;  // [D] or null: all ones
    const float* k_weight;
    float eps;
};

// v summed over the 2^sh neighbouring lanes of a group (sh <= 6), the same sum in all.
__device__ __forceinline__ float group_sum(float v, int sh) {
    auto dpp = [&](auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if (sh > 0) v += dpp(std::integral_constant<int, 0xB1>{});   // lane ^ 1
    if (sh > 1) v += dpp(std::integral_constant<int, 0x4E>{});   // lane ^ 2
    if (sh > 2) v += dpp(std::integral_constant<int, 0x141>{});  // the other four of eight
    if (sh > 3) v += dpp(std::integral_constant<int, 0x140>{});  // the other eight of sixteen
    if (sh > 4) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if (sh > 5) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// Query or key heads of a workgroup at most (six prompts of 12 thousand rows in all: 54.3 us
// with 16, 56.8 with 8).
constexpr int kNormHeads = 16;
// Workgroups of a compute unit that the choice of heads counts with.  A unit holds, wide,
// by registers five with pairs of halves (fp32 heads of 64 dims seven), eight of
// neighbouring pairs without and, by the values' LDS, five (128 dims) or seven (64) with the
// append.  Counting with those instead is not faster on the average of 16 lengths, 700 to
// 8000 rows of 40 heads: neighbouring pairs with the append, fp32 of 128 dims, 1.8 % slower,
// of 64 dims, bf16 and fp32, 3.1 % slower and the same; halves, fp32 of 64 dims, 2.3 % slower,
// with the append the same.  For bf16 of 128 dims five instead of six are 2.9 % faster (1000
// rows 10.2 and 13.2 us).
constexpr int resident(bool append, bool wide, bool inter, bool f32, int d) {
    if (!wide || (inter && !append)) return 8;
    return inter && (f32 || d == 64) ? 6 : 5;
}
// (row, head) units of a thread in flight, 64 bytes.
constexpr int units(bool inter) { return inter ? 4 : 2; }

// Workgroup (tile, y): y below key_wgs takes keys, below key_wgs + value_wgs values,
// the others queries.  WIDE: all rows and pair halves are 16-byte aligned; otherwise
// element by element, a pair per lane.  INTER: the pair of frequency f is (2f, 2f + 1).
template <typename T, int D, bool APPEND, bool WIDE, bool INTER>
__global__ __launch_bounds__(kRotThreads) void norm_rotate_rows(NormArgs na) {
    constexpr int N = Vec<T>::N;
    constexpr int CH = D / N;  // 16-byte chunks of a head
    constexpr int VH = value_heads((int)sizeof(T));
    constexpr int PLACE = APPEND ? kSearchEntries : 1, VALUES = APPEND && WIDE ? VH * kTile * (CH + 1) : 1;
    // rows four banks apart: a wavefront reads eight rows at once, 16 bytes per lane
    __shared__ __attribute__((aligned(16))) float s_cos[kTile][kMaxFreqs + 4];
    __shared__ __attribute__((aligned(16))) float s_sin[kTile][kMaxFreqs + 4];
    __shared__ Place place[kTile];
    __shared__ int32_t s_start[PLACE];
    __shared__ uint4 s_val[VALUES];
    const RotArgs& a = na.r;
    const int tid = threadIdx.x;
    // neighbouring tiles on one XCD: their rows share cache lines of the paged cache
    const int xq = gridDim.x / 8, xr = gridDim.x % 8, xcd = blockIdx.x % 8;
    const int row0 = (xcd * xq + min(xcd, xr) + (int)(blockIdx.x / 8)) * kTile;
    const int rows = min(kTile, a.total_q - row0);
    const int y = blockIdx.y;
    const bool key = y < a.key_wgs, value = !key && y < a.key_wgs + a.value_wgs;
    const int per = value ? VH : a.heads_per_wg;
    const int h_lo = (key ? y : value ? y - a.key_wgs : y - a.key_wgs - a.value_wgs) * per;
    const int h_hi = min(h_lo + per, key || value ? a.hkv : a.hq);
    const int half = a.freqs;  // the distance of a pair's dims, unless INTER
    const T* in = static_cast<const T*>(key ? a.k : a.q);
    const int64_t in_stride = key ? a.k_stride : a.q_stride;
    const float* weight = key ? na.k_weight : na.q_weight;

    // angles: a frequency per lane; with 32 or fewer of them two rows per wavefront
    const int fsh = a.freqs <= 32 ? 5 : 6;
    auto angles = [&]() {
        const int f = tid & ((1 << fsh) - 1), r0 = tid >> fsh, step = kRotThreads >> fsh;
        if (f >= a.freqs) return;
        const double turns_per = a.inv_freq[f] * 0.15915494309189533577;  // 1 / 2 pi
        const int32_t* pos = a.positions + (int64_t)a.axis[f] * a.total_q + row0;
        for (int r = r0; r < rows; r += step) {
            const float2 cs = unit_circle((double)pos[r] * turns_per, a.scale);
            s_cos[r][f] = cs.x;
            s_sin[r][f] = cs.y;
        }
    };
    // where row r's head h_lo goes (null: nowhere), and the distance of its chunks there
    auto target = [&](int r) -> T* {
        if (APPEND && key) {
            const Place p = place[r];
            if (p.block < 0) return nullptr;
            return static_cast<T*>(a.k_out) + ((int64_t)p.block * a.hkv + h_lo) * (D * kBlockTokens) + p.slot * N;
        }
        return static_cast<T*>(key ? a.k_out : a.q_out) + (row0 + r) * (key ? a.k_out_stride : a.q_out_stride) + (int64_t)h_lo * D;
    };
    const int chunk_step = APPEND && key ? kBlockTokens * N : N;

    if constexpr (WIDE) {
        if (APPEND && value) {
            store_values<T, D>(a, row0, rows, h_lo, h_hi, s_start, place, s_val);
            return;
        }
        // An item is what one thread turns: a chunk (INTER), or a chunk of first dims
        // with the chunk of their partners; then the chunks that pass through unturned.
        const int turned = INTER ? 2 * half / N : half / N;
        const int items = turned + (CH - 2 * half / N);
        int sh = 0;
        while ((1 << sh) < items) ++sh;
        const int lane = tid & ((1 << sh) - 1), it = min(lane, items - 1);
        const bool pair = !INTER && it < turned, works = lane < items;
        const int c0 = it < turned ? it : 2 * half / N + (it - turned);
        const int c1 = pair ? it + half / N : c0;
        const int step = kRotThreads >> sh, all = (h_hi - h_lo) * kTile;
        // A thread's units: their rows alternate between kSets (32 threads to a head), or are
        // all the same one.
        constexpr int kUnits = units(INTER), kSets = CH == 32 ? 2 : 1;
        const int u0 = tid >> sh;
        const T* from[kSets];
#pragma unroll
        for (int z = 0; z < kSets; ++z) from[z] = in + (row0 + min((u0 + z * step) % kTile, rows - 1)) * in_stride + h_lo * D;
        u32x4 v0[kUnits], v1[kUnits];
        auto load = [&](int base) {
#pragma unroll
            for (int x = 0; x < kUnits; ++x) {
                const T* head = from[x % kSets] + min(base + u0 + x * step, all - 1) / kTile * D;
                v0[x] = *reinterpret_cast<const u32x4*>(head + c0 * N);
                if constexpr (!INTER) v1[x] = *reinterpret_cast<const u32x4*>(head + c1 * N);
            }
        };
        load(0);
        float w0[N], w1[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            w0[e] = weight ? weight[c0 * N + e] : 1.f;
            if constexpr (!INTER) w1[e] = weight ? weight[c1 * N + e] : 1.f;
        }
        angles();
        if (APPEND && key) find_places(a, row0, rows, s_start, place);
        __syncthreads();
        // Weights, sine and cosine as one matrix per pair (a, b), the same for all heads of
        // a row: a' = rs (aa a + ab b), b' = rs (ba a + bb b).
        constexpr int F = INTER ? N / 2 : N;
        float aa[kSets][F], ab[kSets][F], ba[kSets][F], bb[kSets][F];
        T* to[kSets];
#pragma unroll
        for (int z = 0; z < kSets; ++z) {
            const int r = (u0 + z * step) % kTile;
            float cn[F], sn[F];
            const int f0 = it < turned ? it * F : 0;
            __builtin_memcpy(cn, __builtin_assume_aligned(&s_cos[r][f0], F * 4 > 16 ? 16 : F * 4), sizeof(cn));
            __builtin_memcpy(sn, __builtin_assume_aligned(&s_sin[r][f0], F * 4 > 16 ? 16 : F * 4), sizeof(sn));
#pragma unroll
            for (int e = 0; e < F; ++e) {
                const float wa = w0[INTER ? 2 * e : e], wb = INTER ? w0[2 * e + 1] : w1[e];
                const float c = it < turned ? cn[e] : 1.f, d = it < turned ? sn[e] : 0.f;
                aa[z][e] = wa * c;
                ab[z][e] = -wb * d;
                ba[z][e] = wa * d;
                bb[z][e] = wb * c;
            }
            to[z] = works && r < rows ? target(r) : nullptr;
        }
        const int head_step = APPEND && key ? D * kBlockTokens : D;
        for (int base = 0; base < all; base += kUnits * step) {
            if (base) load(base);
#pragma unroll
            for (int x = 0; x < kUnits; ++x) {
                const int u = base + u0 + x * step, z = x % kSets;
                float p[N], q[N], ss = 0.f;  // with INTER q stays unused
                unpack16(make_uint4(v0[x].x, v0[x].y, v0[x].z, v0[x].w), p, T{});
#pragma unroll
                for (int e = 0; e < N; ++e) ss = fmaf(p[e], p[e], ss);
                if constexpr (!INTER) {
                    unpack16(make_uint4(v1[x].x, v1[x].y, v1[x].z, v1[x].w), q, T{});
                    float s1 = 0.f;
#pragma unroll
                    for (int e = 0; e < N; ++e) s1 = fmaf(q[e], q[e], s1);
                    ss += pair ? s1 : 0.f;
                }
                const float rs = rsqrtf(fmaf(group_sum(works ? ss : 0.f, sh), 1.f / D, na.eps));
                if (u >= all || !to[z]) continue;
                float ya[F], yb[F];
#pragma unroll
                for (int e = 0; e < F; ++e) {
                    const float xa = p[INTER ? 2 * e : e], xb = INTER ? p[2 * e + 1] : q[e];
                    ya[e] = rs * fmaf(ab[z][e], xb, aa[z][e] * xa);
                    yb[e] = rs * fmaf(bb[z][e], xb, ba[z][e] * xa);
                }
                T* head = to[z] + u / kTile * head_step;
                if constexpr (INTER) {
#pragma unroll
                    for (int e = 0; e < F; ++e) p[2 * e] = ya[e], p[2 * e + 1] = yb[e];
                    const uint4 y = Vec<T>::pack(p);
                    *reinterpret_cast<u32x4*>(head + c0 * chunk_step) = u32x4{y.x, y.y, y.z, y.w};
                } else {
                    const uint4 y0 = Vec<T>::pack(ya);
                    *reinterpret_cast<u32x4*>(head + c0 * chunk_step) = u32x4{y0.x, y0.y, y0.z, y0.w};
                    if (pair) {
                        const uint4 y1 = Vec<T>::pack(yb);
                        *reinterpret_cast<u32x4*>(head + c1 * chunk_step) = u32x4{y1.x, y1.y, y1.z, y1.w};
                    }
                }
            }
        }
    } else {
        if (!value) angles();
        if (APPEND && (key || value)) find_places(a, row0, rows, s_start, place);
        __syncthreads();
        if (value) {
            for (int u = tid; u < (h_hi - h_lo) * kTile * D; u += kRotThreads) {
                const int d = u % D, r = u / D % kTile, h = h_lo + u / D / kTile;
                if (r >= rows || place[r].block < 0) continue;
                static_cast<T*>(a.v_out)[(((int64_t)place[r].block * a.hkv + h) * D + d) * kBlockTokens + place[r].slot] =
                    static_cast<const T*>(a.v)[(row0 + r) * a.v_stride + (int64_t)h * D + d];
            }
            return;
        }
        // an item is a pair, or two neighbouring dims that pass through unturned; the
        // D / 2 lanes of a head are neighbours, and all of them stay to the end
        constexpr int kSh = D == 128 ? 6 : 5;
        const int it = tid & (D / 2 - 1);
        const bool turned = it < half;
        const int d0 = turned && !INTER ? it : 2 * it, d1 = turned && !INTER ? it + half : 2 * it + 1;
        const float w0 = weight ? weight[d0] : 1.f, w1 = weight ? weight[d1] : 1.f;
        for (int u = tid >> kSh; u < (h_hi - h_lo) * kTile; u += kRotThreads >> kSh) {
            const int r = u % kTile, h = h_lo + u / kTile;
            const T* head = in + (row0 + min(r, rows - 1)) * in_stride + (int64_t)h * D;
            float p = Storage<T>::load(head, d0), q = Storage<T>::load(head, d1);
            const float rs = rsqrtf(fmaf(group_sum(fmaf(p, p, q * q), kSh), 1.f / D, na.eps));
            if (r >= rows) continue;
            p *= rs * w0;
            q *= rs * w1;
            if (turned) turn(p, q, make_float2(s_cos[r][it], s_sin[r][it]));
            T* to = target(r);
            if (!to) continue;
            to += (h - h_lo) * (APPEND && key ? D * kBlockTokens : D);
            Storage<T>::store(to, d0 / N * chunk_step + d0 % N, p);
            Storage<T>::store(to, d1 / N * chunk_step + d1 % N, q);
        }
    }
}

template <typename T, int D, bool APPEND>
void launch_norm(const NormArgs& a, const verify_rotary_params& p, bool wide, hipStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)a.r.total_q + kTile - 1) / kTile),
                    (unsigned)(a.r.key_wgs + a.r.value_wgs + (a.r.hq + a.r.heads_per_wg - 1) / a.r.heads_per_wg));
    auto run = [&](auto w, auto inter) {
        hipLaunchKernelGGL((norm_rotate_rows<T, D, APPEND, decltype(w)::value, decltype(inter)::value>), grid,
                           dim3(kRotThreads), 0, stream, a);
    };
    if (p.interleaved) wide ? run(std::true_type{}, std::true_type{}) : run(std::false_type{}, std::true_type{});
    else wide ? run(std::true_type{}, std::false_type{}) : run(std::false_type{}, std::false_type{});
}

// Fills in what both calls share and launches.
template <bool APPEND>
int norm_call(NormArgs& na, const verify_rotary_params& p, hipStream_t stream) {
    RotArgs& a = na.r;
    a.freqs = p.rotary_dim / 2;
    a.scale = p.scale > 0.f ? p.scale : 1.f;
    for (int f = 0; f < a.freqs; ++f) a.axis[f] = p.axis[f];
    const int esize = p.dtype == VERIFY_BF16 ? 2 : 4, n = 16 / esize;
    if (APPEND) a.value_wgs = (a.hkv + value_heads(esize) - 1) / value_heads(esize);
    const uint64_t bits = (uint64_t)(uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.q_out | (uintptr_t)a.k_out;
    const int64_t strides = a.q_stride | a.k_stride | a.v_stride | a.q_out_stride | a.k_out_stride;
    const int step = p.interleaved ? p.rotary_dim : a.freqs;
    const bool wide = (bits & 15) == 0 && strides % n == 0 && step % n == 0;
    // Heads per workgroup, two at least.  Each costs its heads and some four more for its
    // tile's angles; what counts is the mean of all of them and of the rounds that they
    // take (2500 rows of 40 heads: eight, in one round, 14.0 us; three, in not quite two, 18.2;
    // 8000 rows: eight, in two, 39.4; 16, in one and a sixth, 41.5).  Of long inputs all
    // that a workgroup takes.
    const int64_t tiles = ((int64_t)a.total_q + kTile - 1) / kTile,
                  fit = (int64_t)resident(APPEND, wide, p.interleaved, esize == 4, p.head_dim) * device_cus();
    auto groups = [&](int64_t heads, int h) { return (heads + h - 1) / h; };
    auto wgs = [&](int h) { return tiles * (groups(a.hq, h) + groups(a.hkv, h) + a.value_wgs); };
    auto cost = [&](int h) { return ((wgs(h) + fit - 1) / fit * fit + wgs(h)) * (h + 4); };
    a.heads_per_wg = std::min(std::max(a.hq, a.hkv), kNormHeads);
    if (wgs(kNormHeads) <= 2 * fit)
        for (int h = a.heads_per_wg - 1; h >= 2; --h)
            if (cost(h) < cost(a.heads_per_wg)) a.heads_per_wg = h;
    a.key_wgs = (int)groups(a.hkv, a.heads_per_wg);
    if (p.dtype == VERIFY_BF16)
        p.head_dim == 128 ? launch_norm<uint16_t, 128, APPEND>(na, p, wide, stream)
                          : launch_norm<uint16_t, 64, APPEND>(na, p, wide, stream);
    else
        p.head_dim == 128 ? launch_norm<float, 128, APPEND>(na, p, wide, stream)
                          : launch_norm<float, 64, APPEND>(na, p, wide, stream);
    return check_launch();
}

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_norm_rotary(const verify_rotary_params* params, int32_t total_q, int32_t num_q_heads,
                                  int32_t num_kv_heads, const void* q, int64_t q_stride, const void* k,
                                  int64_t k_stride, const float* q_weight, const float* k_weight, float eps,
                                  const int32_t* positions, const double* inv_freq, void* q_out,
                                  int64_t q_out_stride, void* k_out, int64_t k_out_stride, hipStream_t stream) {
    const int rc = check_params(params, total_q, num_q_heads, num_kv_heads);
    if (rc != VERIFY_OK) return rc;
    if (!(eps >= 0.f) || eps > 3.0e38f) return VERIFY_EINVAL;
    const int64_t wq = (int64_t)num_q_heads * params->head_dim, wk = (int64_t)num_kv_heads * params->head_dim;
    if (q_stride < wq || q_out_stride < wq || (num_kv_heads > 0 && (k_stride < wk || k_out_stride < wk)))
        return VERIFY_EINVAL;
    if (total_q == 0) return VERIFY_OK;
    if (!q || !q_out || !positions || !inv_freq) return VERIFY_EINVAL;
    if ((num_kv_heads > 0) != (k != nullptr) || (num_kv_heads > 0) != (k_out != nullptr)) return VERIFY_EINVAL;
    if ((q == q_out && q_stride != q_out_stride) || (k && k == k_out && k_stride != k_out_stride))
        return VERIFY_EINVAL;
    NormArgs na{};
    RotArgs& a = na.r;
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
    na.q_weight = q_weight;
    na.k_weight = k_weight;
    na.eps = eps;
    return norm_call<false>(na, *params, stream);
}

extern "C" int verify_norm_rotary_append(const verify_attn_params* attn, const verify_rotary_params* params,
                                         int32_t total_q, const void* q, int64_t q_stride, const void* k_new,
                                         int64_t k_stride, const void* v_new, int64_t v_stride,
                                         const float* q_weight, const float* k_weight, float eps,
                                         const int32_t* positions, const double* inv_freq,
                                         const int32_t* block_tables, const int32_t* seq_lens,
                                         const int32_t* q_start, void* q_out, int64_t q_out_stride,
                                         void* k_cache, void* v_cache, hipStream_t stream) {
    int rc = validate(attn, total_q, 0, 0);
    if (rc == VERIFY_OK) rc = check_params(params, total_q, attn->num_q_heads, attn->num_kv_heads);
    if (rc != VERIFY_OK) return rc;
    if (params->head_dim != attn->head_dim || params->dtype != attn->dtype) return VERIFY_EINVAL;
    if (!(eps >= 0.f) || eps > 3.0e38f) return VERIFY_EINVAL;
    const int64_t wq = (int64_t)attn->num_q_heads * attn->head_dim, wk = (int64_t)attn->num_kv_heads * attn->head_dim;
    if (q_stride < wq || q_out_stride < wq || k_stride < wk || v_stride < wk) return VERIFY_EINVAL;
    if (total_q == 0) return VERIFY_OK;
    if (attn->num_seqs == 0)  // rows of no request: the queries alone
        return verify_norm_rotary(params, total_q, attn->num_q_heads, 0, q, q_stride, nullptr, 0, q_weight, nullptr,
                                  eps, positions, inv_freq, q_out, q_out_stride, nullptr, 0, stream);
    if (!q || !q_out || !positions || !inv_freq || !k_new || !v_new || !block_tables || !seq_lens || !q_start ||
        !k_cache || !v_cache)
        return VERIFY_EINVAL;
    if ((uintptr_t)k_cache & 15) return VERIFY_EINVAL;
    if (q == q_out && q_stride != q_out_stride) return VERIFY_EINVAL;
    NormArgs na{};
    RotArgs& a = na.r;
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
    na.q_weight = q_weight;
    na.k_weight = k_weight;
    na.eps = eps;
    return norm_call<true>(na, *params, stream);
}
