// verify_logits.hip -- logits changed before tokens are accepted from them: penalties
// for tokens that a request has had, biases and grammar masks; and the counts of
// tokens that the penalties read.
//
// Row j of a request stands behind its drafts 1 .. j, so a token's count there is the
// stored one and those of these drafts.  With h[v] whether v was in the prompt or has
// a count c[v] > 0:
//     x *= x > 0 ? 1 / repetition : repetition   where h[v]
//     x += bias[v] - frequency c[v] - presence [c[v] > 0]
//     x  = -inf                                  where the row's mask lacks v
//
// What bounds it: memory, 2 V bytes in and out per row (288 rows of 151936 with all changes
// 36.4 us, a copy 37), and with single rows the latencies that lead to a span's logits
// (256 of them 61 to 64 us, a copy 32).  The request's state is small
// beside them: a bit per token tells whether a count need be read at all, so V / 4
// bytes of bits and the counts of the few tokens that were had.  A workgroup takes
// kSpan tokens of one request and all of its rows: state and biases become a bit and a
// summand per token in registers, eight tokens to a thread; a draft changes those of
// one token on the way to the next row.  What hides the memory's latency is the number
// of wavefronts, seven per SIMD in bf16 (by LDS) and six in fp32 (by registers): counts and
// biases, which only a draft needs again, lie in LDS (with them and the next rows in registers,
// four wavefronts, the 288 rows took 60 us; in a loop over spans that reads a request's
// parameters once, six, 40).  Wavefronts whose tokens nothing changes move bits.
#include <type_traits>

#include "common.h"

namespace averify {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                  // tokens of a thread
constexpr int kSpan = kThreads * kPer;   // tokens of a workgroup
constexpr int kRows = 4;                 // rows in flight

struct AdjustArgs {
    const void* logits;
    void* out;
    const int32_t* tokens;
    const int32_t* q_start;
    const float* repetition;
    const float* frequency;
    const float* presence;
    const int32_t* counts;
    const uint8_t* seen;
    const int32_t* slots;
    const int32_t* bias_start;
    const int32_t* bias_tokens;
    const float* bias_values;
    const uint8_t* mask;
    const int32_t* mask_rows;
    int64_t row_stride, out_stride;
    int vocab, words, total_q, num_slots, num_biases, num_masks;
    int penal;
};

// A thread's eight logits, neighbours, in 16-byte accesses that need only be aligned to
// an element (rows of an odd vocabulary).
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct Group {
    using Vec = std::conditional_t<sizeof(T) == 2, u32x4_2, u32x4_4>;
    static constexpr int kVecs = kPer * (int)sizeof(T) / 16, kIn = 16 / (int)sizeof(T);
    uint4 v[kVecs];

    // `room` of the eight are in the vocabulary
    __device__ __forceinline__ void load(const T* at, int room) {
        if (room >= kPer) {
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const Vec x = __builtin_nontemporal_load(reinterpret_cast<const Vec*>(at + k * kIn));
                v[k] = make_uint4(x.x, x.y, x.z, x.w);
            }
        } else {
            T t[kPer] = {};
#pragma unroll
            for (int e = 0; e < kPer; ++e) if (e < room) t[e] = at[e];
            __builtin_memcpy(v, t, sizeof(t));
        }
    }
    __device__ __forceinline__ void store(T* at, int room) const {
        if (room >= kPer) {
#pragma unroll
            for (int k = 0; k < kVecs; ++k) *reinterpret_cast<Vec*>(at + k * kIn) = Vec{v[k].x, v[k].y, v[k].z, v[k].w};
        } else {
            T t[kPer];
            __builtin_memcpy(t, v, sizeof(t));
#pragma unroll
            for (int e = 0; e < kPer; ++e) if (e < room) at[e] = t[e];
        }
    }
    __device__ __forceinline__ void get(float* x) const {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) unpack16(v[k], x + k * kIn, T{});
    }
    __device__ __forceinline__ void set(const float* x) {
        if constexpr (sizeof(T) == 2)
            v[0] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                              pack_bf16x2(x[6], x[7]));
        else
            __builtin_memcpy(v, x, kPer * sizeof(float));
    }
};

// -inf where a bit of `allowed` is 0, the others' bits as they are.
__device__ __forceinline__ void mask_bits(Group<uint16_t>& g, uint32_t allowed) {
    auto all = [&](int e) { return (uint32_t)((int32_t)(allowed << (31 - e)) >> 31); };
    auto pair = [&](uint32_t w, int e) {
        const uint32_t m = (all(e) & 0xffffu) | (all(e + 1) & 0xffff0000u);
        return (w & m) | (0xff80ff80u & ~m);
    };
    g.v[0] = make_uint4(pair(g.v[0].x, 0), pair(g.v[0].y, 2), pair(g.v[0].z, 4), pair(g.v[0].w, 6));
}
__device__ __forceinline__ void mask_bits(Group<float>& g, uint32_t allowed) {
    float v[kPer];
    g.get(v);
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e] = allowed >> e & 1u ? v[e] : -INFINITY;
    g.set(v);
}

// Workgroup (x, i, z): tokens x kSpan .. of request i, the z-th part of its rows.
template <typename T, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void adjust_rows(AdjustArgs a) {
    __shared__ int s_token[kThreads];
    __shared__ float s_value[kThreads];
    __shared__ int s_found[kThreads / kWave];
    __shared__ int s_draft[kThreads];
    __shared__ int s_mask[kThreads];
    __shared__ int s_count[kPer][kThreads];
    __shared__ float s_bias[kPer][kThreads];
    const int tid = threadIdx.x, i = blockIdx.y;
    const bool penal = a.penal;
    const int slot = penal ? a.slots ? a.slots[i] : i : -1;
    const float rep = a.repetition ? a.repetition[i] : 1.f, freq = a.frequency ? a.frequency[i] : 0.f,
                pres = a.presence ? a.presence[i] : 0.f;
    const int b0 = a.bias_start ? max(0, min(a.bias_start[i], a.num_biases)) : 0;
    const int b1 = a.bias_start ? min(a.bias_start[i + 1], a.num_biases) : 0;
    const int q0 = max(0, min(a.q_start[i], a.total_q)), n = max(0, min(a.q_start[i + 1], a.total_q) - q0);
    const int part = (n + (int)gridDim.z - 1) / (int)gridDim.z;
    const int j0 = min(n, (int)blockIdx.z * part), j1 = min(n, j0 + part);
    if (j0 >= j1) return;
    // the rows' drafts and masks, kThreads of them at a time
    auto read_rows = [&](int from) {
        const int j = from + tid;
        s_draft[tid] = penal && j > 0 && j < n ? a.tokens[q0 + j] : -1;
        s_mask[tid] = a.mask_rows && j < n ? a.mask_rows[q0 + j] : -1;
    };
    int rows0 = j0;  // the row of the first entry in s_draft
    read_rows(rows0);
    __syncthreads();
    const float inv = 1.f / rep;
    const int span0 = blockIdx.x * kSpan;
    const int tok0 = span0 + tid * kPer, room = a.vocab - tok0;
    const bool live = room > 0;
    // the eight bits of a bit array
    auto bits_of = [&](const uint8_t* bits) -> uint32_t { return live ? bits[tok0 >> 3] : 0; };

    const T* in = static_cast<const T*>(a.logits) + (int64_t)q0 * a.row_stride;
    T* to = static_cast<T*>(a.out) + (int64_t)q0 * a.out_stride;
    // The next rows' masks and logits.  What a mask lacks whole need not be read; in
    // place, neither need what nothing changes (`touched`, a bit per row).
    Group<T> g[kRows];
    uint32_t allowed[kRows];
    auto load_masks = [&](int base) {
#pragma unroll
        for (int x = 0; x < kRows; ++x) {
            allowed[x] = 0xffu;
            if (a.mask_rows && base + x < j1) {
                const int m = s_mask[base + x - rows0];
                if (m >= 0 && m < a.num_masks) allowed[x] = bits_of(a.mask + (int64_t)m * a.words * 4);
            }
        }
    };
    auto load_rows = [&](int base, uint32_t touched) {
#pragma unroll
        for (int x = 0; x < kRows; ++x)
            if (base + x < j1 && live && allowed[x] && (!IN_PLACE || (touched >> x & 1u) || allowed[x] != 0xffu))
                g[x].load(in + (int64_t)(base + x) * a.row_stride + tok0, room);
    };
    // The state's bits and the first masks, then out of place the first rows, are under way
    // before anything is waited for that does not lead to them.
    uint32_t prompt = 0, out = 0;
    const int32_t* counts = nullptr;
    if (penal && slot >= 0 && slot < a.num_slots) {
        const uint8_t* seen = a.seen + (int64_t)slot * 2 * a.words * 4;
        counts = a.counts + (int64_t)slot * a.vocab;
        prompt = bits_of(seen);
        out = bits_of(seen + (int64_t)a.words * 4);
    }
    load_masks(j0);
    if (!IN_PLACE) load_rows(j0, 0);
    int c[kPer] = {};
    if (out) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) c[e] = (out >> e & 1u) && e < room ? counts[tok0 + e] : 0;
    }

    // a token of this span: its thread, and its place among that thread's
    auto owner = [&](int d) { return (d - span0) / kPer; };
    auto place = [&](int d) { return (d - span0) % kPer; };
    // the request's state: tokens had (a bit each), their counts, biases
    uint32_t had = 0, biased = 0;
    float add[kPer];  // -0: a sum's neutral element
#pragma unroll
    for (int e = 0; e < kPer; ++e) add[e] = -0.f;
    if (b1 > b0) {
        bool found = false;
        // the list's entries of this span, kThreads of the list at a time, in its order
        for (int base = b0; base < b1; base += kThreads) {
            const int at = base + tid, tok = at < b1 ? a.bias_tokens[at] : -1;
            const bool here = tok >= span0 && tok - span0 < kSpan && tok < a.vocab;
            if (!__syncthreads_or(here)) continue;
            if (!found) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) s_bias[e][tid] = -0.f;
                found = true;
            }
            const uint64_t vote = __ballot(here);
            if (tid % kWave == 0) s_found[tid / kWave] = __popcll(vote);
            __syncthreads();
            int before = 0, all = 0;
#pragma unroll
            for (int w = 0; w < kThreads / kWave; ++w) {
                before += w < tid / kWave ? s_found[w] : 0;
                all += s_found[w];
            }
            if (here) {
                const int p = before + __popcll(vote & ((1ull << (tid % kWave)) - 1));
                s_token[p] = tok;
                s_value[p] = a.bias_values[at];
            }
            __syncthreads();
            for (int p = 0; p < all; ++p) {
                const int d = s_token[p];
                if (owner(d) == tid) s_bias[place(d)][tid] += s_value[p], biased |= 1u << place(d);
            }
        }
        if (biased) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) add[e] = s_bias[e][tid];
        }
    }
    if (penal) {
        had = prompt;
        if (out) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                c[e] = max(0, c[e]);
                had |= (uint32_t)(c[e] > 0) << e;
                if (c[e] > 0) add[e] -= fmaf(freq, (float)c[e], pres);
            }
        }
        if (n > 1) {  // there are drafts
#pragma unroll
            for (int e = 0; e < kPer; ++e) s_count[e][tid] = c[e];
        }
    }
    // the draft that row j stands behind, or -1 where it is none of this span's tokens
    auto in_span = [&](int d) { return d >= span0 && d - span0 < kSpan && d < a.vocab ? d : -1; };
    auto draft_of = [&](int j) {
        const int d = __builtin_amdgcn_readfirstlane(j < j1 ? s_draft[j - rows0] : -1);
        return in_span(d);
    };
    auto count_draft = [&](int d) {
        if (d < 0 || owner(d) != tid) return;
        const int e = place(d), c = ++s_count[e][tid];
        const float bias = biased >> e & 1u ? s_bias[e][tid] : -0.f, sum = bias - fmaf(freq, (float)c, pres);
        had |= 1u << e;
#pragma unroll
        for (int n = 0; n < kPer; ++n) add[n] = n == e ? sum : add[n];
    };
    if (penal) {
        // the drafts in front of this part's rows
        for (int from = 1; from < j0; from += kThreads) {
            const int d = from + tid < j0 ? a.tokens[q0 + from + tid] : -1;
            __syncthreads();
            s_token[tid] = d;
            __syncthreads();
            for (int j = 0; j < min(kThreads, j0 - from); ++j) count_draft(in_span(s_token[j]));
        }
    }

    for (int base = j0; base < j1; base += kRows) {
        int draft[kRows];
#pragma unroll
        for (int x = 0; x < kRows; ++x) draft[x] = draft_of(base + x);
        if (IN_PLACE || base > j0) {
            uint32_t touched = had | biased ? ~0u : 0u, mine = 0;
#pragma unroll
            for (int x = 0; x < kRows; ++x) {
                if (IN_PLACE && draft[x] >= 0) mine |= owner(draft[x]) == tid;
                touched |= mine << x;
            }
            load_rows(base, touched);
        }
#pragma unroll
        for (int x = 0; x < kRows; ++x) {
            const int j = base + x;
            if (j >= j1) break;
            count_draft(draft[x]);
            const bool change = had || biased, masked = allowed[x] != 0xffu;
            if (__any(change)) {
                if (change && allowed[x]) {
                    float v[kPer];
                    g[x].get(v);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const float f = v[e] > 0.f ? inv : rep;
                        v[e] = fmaf(v[e], had >> e & 1u ? f : 1.f, add[e]);
                    }
                    g[x].set(v);
                }
            }
            if (masked) mask_bits(g[x], allowed[x]);
            if (live && (!IN_PLACE || change || masked)) g[x].store(to + (int64_t)j * a.out_stride + tok0, room);
        }
        if (base + kRows >= j1) break;
        if (base + 2 * kRows > rows0 + kThreads) {  // the next rows' entries are not all here
            __syncthreads();
            rows0 = base + kRows;
            read_rows(rows0);
            __syncthreads();
        }
        load_masks(base + kRows);
    }
}

struct CountArgs {
    int32_t* counts;
    uint32_t* seen;
    const int32_t* tokens;
    const int32_t* start;
    const int32_t* num;
    const int32_t* slots;
    int vocab, words, total, num_slots, prompt;
};

// Integer sums and bits: the order in which they arrive changes nothing.
//
// Workgroup (x, i): request i's tokens, kThreads at a time.
__global__ __launch_bounds__(kThreads) void count_tokens(CountArgs a) {
    const int i = blockIdx.y;
    const int slot = a.slots ? a.slots[i] : i;
    if (slot < 0 || slot >= a.num_slots) return;
    const int t0 = max(0, min(a.start[i], a.total));
    int n = max(0, min(a.start[i + 1], a.total) - t0);
    if (a.num) n = min(n, a.num[i]);
    uint32_t* seen = a.seen + ((int64_t)slot * 2 + (a.prompt ? 0 : 1)) * a.words;
    int32_t* counts = a.counts + (int64_t)slot * a.vocab;
    for (int64_t j = blockIdx.x * kThreads + threadIdx.x; j < n; j += (int64_t)gridDim.x * kThreads) {
        const int tok = a.tokens[t0 + j];
        if (tok < 0 || tok >= a.vocab) continue;
        if (!a.prompt) atomicAdd(counts + tok, 1);
        atomicOr(seen + (tok >> 5), 1u << (tok & 31));
    }
}

// The same for many tokens of a request, kPart at a time: text has the same few words of
// bits again and again, and thousands of atomic operations on one word of memory come
// one after the other (64 thousand tokens of eight prompts: 58 us).  So the bits are
// gathered in LDS, where a set bit costs a read, and each word that got some leaves once.
constexpr int kManyThreads = 512;
constexpr int kPart = 4096;
constexpr int kManyWords = 16384;  // LDS: a vocabulary of 524288
__global__ __launch_bounds__(kManyThreads) void count_many(CountArgs a) {
    extern __shared__ uint32_t s_bits[];
    const int i = blockIdx.y, tid = threadIdx.x;
    const int slot = a.slots ? a.slots[i] : i;
    const int t0 = max(0, min(a.start[i], a.total));
    int n = max(0, min(a.start[i + 1], a.total) - t0);
    if (a.num) n = min(n, a.num[i]);
    if (slot < 0 || slot >= a.num_slots || (int64_t)blockIdx.x * kPart >= n) return;
    for (int w = tid; w < a.words; w += kManyThreads) s_bits[w] = 0;
    __syncthreads();
    int32_t* counts = a.counts + (int64_t)slot * a.vocab;
    for (int64_t part = (int64_t)blockIdx.x * kPart; part < n; part += (int64_t)gridDim.x * kPart) {
        int tok[kPart / kManyThreads];
#pragma unroll
        for (int x = 0; x < kPart / kManyThreads; ++x) {
            const int64_t j = part + x * kManyThreads + tid;
            tok[x] = j < n ? a.tokens[t0 + j] : -1;
        }
#pragma unroll
        for (int x = 0; x < kPart / kManyThreads; ++x) {
            if (tok[x] < 0 || tok[x] >= a.vocab) continue;
            if (!a.prompt) atomicAdd(counts + tok[x], 1);
            const uint32_t bit = 1u << (tok[x] & 31);
            volatile uint32_t* word = s_bits + (tok[x] >> 5);
            if (!(*word & bit)) atomicOr(s_bits + (tok[x] >> 5), bit);
        }
    }
    __syncthreads();
    uint32_t* seen = a.seen + ((int64_t)slot * 2 + (a.prompt ? 0 : 1)) * a.words;
    for (int w = tid; w < a.words; w += kManyThreads)
        if (s_bits[w]) atomicOr(seen + w, s_bits[w]);
}

template <typename T>
void launch_adjust(const AdjustArgs& a, const dim3& grid, hipStream_t stream) {
    if (a.logits == a.out) hipLaunchKernelGGL((adjust_rows<T, true>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((adjust_rows<T, false>), grid, dim3(kThreads), 0, stream, a);
}

}  // namespace
}  // namespace averify

using namespace averify;

extern "C" int verify_adjust_logits(int32_t num_seqs, int32_t total_q, int64_t vocab, int64_t row_stride,
                                    int32_t logits_dtype, const void* logits, const int32_t* tokens,
                                    const int32_t* q_start, const verify_adjust_params* params, void* out,
                                    int64_t out_stride, hipStream_t stream) {
    if (!params || num_seqs < 0 || total_q < 0 || vocab < 1) return VERIFY_EINVAL;
    if (logits_dtype != VERIFY_F32 && logits_dtype != VERIFY_BF16) return VERIFY_EUNSUPPORTED;
    // a span's tokens and a part's rows are counted in 32 bits
    if (vocab >= (int64_t)INT32_MAX - kSpan || total_q >= (1 << 30) || num_seqs > 65535) return VERIFY_EUNSUPPORTED;
    if (row_stride == 0) row_stride = vocab;
    if (out_stride == 0) out_stride = vocab;
    if (row_stride < vocab || out_stride < vocab) return VERIFY_EINVAL;
    const bool penal = params->repetition || params->frequency || params->presence;
    const bool biases = params->bias_start, masks = params->mask_rows;
    if (penal && (!params->counts || !params->seen || !tokens)) return VERIFY_EINVAL;
    if (biases && ((!params->bias_tokens || !params->bias_values) && params->num_biases > 0)) return VERIFY_EINVAL;
    if (masks && !params->mask && params->num_masks > 0) return VERIFY_EINVAL;
    if (params->num_slots < 0 || params->num_biases < 0 || params->num_masks < 0) return VERIFY_EINVAL;
    if (num_seqs == 0 || total_q == 0) return VERIFY_OK;
    if (!logits || !out || !q_start) return VERIFY_EINVAL;
    if (logits == out && row_stride != out_stride) return VERIFY_EINVAL;
    AdjustArgs a{};
    a.logits = logits;
    a.out = out;
    a.tokens = tokens;
    a.q_start = q_start;
    if (penal) {
        a.penal = 1;
        a.repetition = params->repetition;
        a.frequency = params->frequency;
        a.presence = params->presence;
        a.counts = params->counts;
        a.seen = reinterpret_cast<const uint8_t*>(params->seen);
        a.slots = params->slots;
        a.num_slots = params->num_slots;
    }
    if (biases && params->num_biases > 0) {
        a.bias_start = params->bias_start;
        a.bias_tokens = params->bias_tokens;
        a.bias_values = params->bias_values;
        a.num_biases = params->num_biases;
    }
    if (masks && params->num_masks > 0) {
        a.mask = reinterpret_cast<const uint8_t*>(params->mask);
        a.mask_rows = params->mask_rows;
        a.num_masks = params->num_masks;
    }
    a.row_stride = row_stride;
    a.out_stride = out_stride;
    a.vocab = (int)vocab;
    a.words = (int)((vocab + 31) / 32);
    a.total_q = total_q;
    // a request's rows are divided where there would be few workgroups otherwise
    const int64_t spans = (vocab + kSpan - 1) / kSpan, wgs = spans * num_seqs, rows = ((int64_t)total_q + num_seqs - 1) / num_seqs;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({(1024 + wgs - 1) / wgs, rows, 65535}));
    const dim3 grid((unsigned)spans, (unsigned)num_seqs, (unsigned)parts);
    if (logits_dtype == VERIFY_BF16) launch_adjust<uint16_t>(a, grid, stream);
    else launch_adjust<float>(a, grid, stream);
    return check_launch();
}

extern "C" int verify_count_tokens(int32_t num_seqs, int32_t total_tokens, int64_t vocab, int32_t num_slots,
                                   const int32_t* tokens, const int32_t* token_start, const int32_t* num_tokens,
                                   const int32_t* slots, int32_t prompt, int32_t* counts, uint32_t* seen,
                                   hipStream_t stream) {
    if (num_seqs < 0 || total_tokens < 0 || num_slots < 0 || vocab < 1 || (prompt != 0 && prompt != 1)) return VERIFY_EINVAL;
    if (vocab >= INT32_MAX - 31 || num_seqs > 65535) return VERIFY_EUNSUPPORTED;
    if (num_seqs == 0 || total_tokens == 0 || num_slots == 0) return VERIFY_OK;
    if (!tokens || !token_start || !seen || (!prompt && !counts)) return VERIFY_EINVAL;
    const CountArgs a{counts, seen, tokens, token_start, num_tokens, slots, (int)vocab, (int)((vocab + 31) / 32),
                      total_tokens, num_slots, prompt};
    const int64_t per = ((int64_t)total_tokens + num_seqs - 1) / num_seqs;
    // from where clearing and reading the words costs less than the atomic operations
    if (per >= 512 && a.words <= kManyWords) {
        const dim3 grid((unsigned)std::min<int64_t>(((int64_t)total_tokens + kPart - 1) / kPart, std::max(1, 1024 / num_seqs)),
                        (unsigned)num_seqs);
        hipLaunchKernelGGL(count_many, grid, dim3(kManyThreads), a.words * 4, stream, a);
    } else {
        const dim3 grid((unsigned)std::min<int64_t>((per + kThreads - 1) / kThreads, 256), (unsigned)num_seqs);
        hipLaunchKernelGGL(count_tokens, grid, dim3(kThreads), 0, stream, a);
    }
    return check_launch();
}
