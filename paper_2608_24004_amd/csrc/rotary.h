// rotary.h -- what the calls that turn queries and keys to their positions share: the
// rows' places in the paged cache, the angles, the values' way into the cache and the
// checks of the parameters.
#pragma once

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
    int total_q, hq, hkv, freqs;
    int key_wgs, value_wgs, heads_per_wg;
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

// scale (cos, sin) of t turns: their fraction, in binary64, then fp32.
__device__ __forceinline__ float2 unit_circle(double t, float scale) {
    float sn, cn;
    sincospif(2.f * (float)(t - rint(t)), &sn, &cn);
    return make_float2(scale * cn, scale * sn);
}

__device__ __forceinline__ void turn(float& x, float& y, const float2& cs) {
    // explicit, so that every layout's code rounds alike
    const float a = x, b = y;
    x = fmaf(-b, cs.y, a * cs.x);
    y = fmaf(b, cs.x, a * cs.y);
}

// Heads of V that a workgroup takes (through LDS).
constexpr int value_heads(int esize) { return esize == 2 ? 4 : 2; }

// Values of the tile's rows and heads h_lo .. h_hi - 1 into the cache, which keeps them
// transposed: through s_val, value_heads * kTile * (CH + 1) chunks, so that the threads
// that store run over the rows.
template <typename T, int D>
__device__ __forceinline__ void store_values(const RotArgs& a, int row0, int rows, int h_lo, int h_hi, int32_t* s_start,
                                             Place* place, uint4* s_val) {
    constexpr int N = Vec<T>::N, CH = D / N, VH = value_heads((int)sizeof(T));
    const int tid = threadIdx.x;
    u32x4 v[VH * kTile * CH / kRotThreads];
#pragma unroll
    for (int x = 0; x < VH * kTile * CH / kRotThreads; ++x) {
        const int e = x * kRotThreads + tid, c = e % CH, r = e / CH % kTile, h = e / CH / kTile;
        v[x] = *reinterpret_cast<const u32x4*>(static_cast<const T*>(a.v) + (row0 + min(r, rows - 1)) * a.v_stride +
                                               min(h_lo + h, h_hi - 1) * D + c * N);
    }
    find_places(a, row0, rows, s_start, place);
#pragma unroll
    for (int x = 0; x < VH * kTile * CH / kRotThreads; ++x) {
        const int e = x * kRotThreads + tid, c = e % CH;
        s_val[e / CH * (CH + 1) + c] = make_uint4(v[x].x, v[x].y, v[x].z, v[x].w);
    }
    __syncthreads();
    // threads over the rows first: neighbouring slots of a dim are neighbours
    const int r = tid % kTile;
    const Place p = r < rows ? place[r] : Place{-1, 0};
    if (p.block < 0) return;
    for (int h = h_lo; h < h_hi; ++h) {
        const T* from = reinterpret_cast<const T*>(s_val + ((h - h_lo) * kTile + r) * (CH + 1));
        T* to = static_cast<T*>(a.v_out) + ((int64_t)p.block * a.hkv + h) * (D * kBlockTokens) + p.slot;
#pragma unroll
        for (int d = 0; d < D; d += kRotThreads / kTile) to[(d + tid / kTile) * kBlockTokens] = from[d + tid / kTile];
    }
}

inline int check_params(const verify_rotary_params* p, int32_t total_q, int32_t hq, int32_t hkv) {
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
    if (((int64_t)total_q + kTile - 1) / kTile >= (1 << 24)) return VERIFY_EUNSUPPORTED;  // fewer than 2^32 threads in x
    return VERIFY_OK;
}

}  // namespace
}  // namespace averify
