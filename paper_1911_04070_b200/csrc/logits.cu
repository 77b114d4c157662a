// What a decoding step does to its logits before a token is taken: penalties for tokens that stand in the history, biases, masks.
// See bpt_adjust_logits in include/bpt.h.
//
// Bound by memory for a large batch, by latency for a small one.  One launch, one pass over the logits: a CTA takes a piece of
// one row's vocabulary, asks for its logits, and while they are on their way goes through the row's history and counts, in shared
// memory, the ids that fall into its piece.  Counts are whole numbers, so the order of the atomics does not show.  The history is read
// once per piece, from L2 after the first; a table of counts in global memory would have to be cleared, filled and read by a launch each.
//
// Rows may start anywhere (an odd vocabulary, a slice of a larger tensor): a row's elements are taken in groups of 8 that lie on
// 16-byte boundaries of the logits, whatever their index.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <cstdlib>

#include "bpt_internal.cuh"

namespace bpt {
namespace {

constexpr int kLgStep = 2048;       // no piece of a row is smaller

struct LgParams {
    const void* logits;
    void* out;
    const void* history;
    const int32_t *lengths, *prompts;
    const float *repetition, *presence, *frequency;     // per row, or null: the values below
    const void* bias;
    const void* bias_ids;
    const float* bias_values;
    const uint32_t* allowed;
    long long vocab, logits_stride, out_stride, history_stride, bias_stride, allowed_stride;
    long long bias_count;
    int history_len, history64, bias_ids64, bias_bf16, pieces, count;   // count: there is a history that matters
    float rep, pres, freq;
};

__device__ __forceinline__ float elem(float x) { return x; }
__device__ __forceinline__ float elem(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float x, float* y) { *y = x; }
__device__ __forceinline__ void put(float x, __nv_bfloat16* y) { *y = __float2bfloat16(x); }

template <typename T>
__device__ __forceinline__ void read8(const T* at, float (&x)[8]) {     // 16-byte aligned
    constexpr int per = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 8 / per; ++j) {
        const uint4 q = *((const uint4*)at + j);
        T e[per];
        memcpy(e, &q, 16);
#pragma unroll
        for (int i = 0; i < per; ++i) x[j * per + i] = elem(e[i]);
    }
}
template <typename T>
__device__ __forceinline__ void write8(T* at, const float (&x)[8]) {
    constexpr int per = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 8 / per; ++j) {
        T e[per];
#pragma unroll
        for (int i = 0; i < per; ++i) put(x[j * per + i], e + i);
        uint4 q;
        memcpy(&q, e, 16);
        *((uint4*)at + j) = q;
    }
}
__device__ __forceinline__ long long id_at(const void* ids, int is64, long long i) {
    return is64 ? __ldg((const long long*)ids + i) : (long long)__ldg((const int*)ids + i);
}

constexpr unsigned kLgPrompt = 0x80000000u;     // of an id's word: it stands in the prompt; the other bits count the places behind it
constexpr int kLgAhead = 4;                     // ids of the history a thread asks for at once

// The 8 values of a bias from `at` on, of which `before` values lie before it in its row and `behind` from it on: wherever that starts, in
// whole 16-byte pieces around it while those lie in the row.
__device__ __forceinline__ void bias8(const float* at, long long before, long long behind, float (&z)[8]) {
    const int s = (int)((uintptr_t)at & 15) / 4;
    if (before >= s && behind >= 12) {
        unsigned w[12];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const uint4 q = __ldg((const uint4*)(at - s) + j);
            w[4 * j] = q.x; w[4 * j + 1] = q.y; w[4 * j + 2] = q.z; w[4 * j + 3] = q.w;
        }
#pragma unroll
        for (int j = 0; j < 11; ++j) w[j] = s & 1 ? w[j + 1] : w[j];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(s & 2 ? w[j + 2] : w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = j < behind && -j <= before ? __ldg(at + j) : 0.f;
    }
}
__device__ __forceinline__ void bias8(const __nv_bfloat16* at, long long before, long long behind, float (&z)[8]) {
    const int s = (int)((uintptr_t)at & 15) / 2;
    if (before >= s && behind >= 16) {
        unsigned w[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint4 q = __ldg((const uint4*)(at - s) + j);
            w[4 * j] = q.x; w[4 * j + 1] = q.y; w[4 * j + 2] = q.z; w[4 * j + 3] = q.w;
        }
#pragma unroll
        for (int j = 0; j < 7; ++j) w[j] = s & 2 ? w[j + 1] : w[j];
#pragma unroll
        for (int j = 0; j < 5; ++j) w[j] = s & 4 ? w[j + 2] : w[j];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned two = s & 1 ? __funnelshift_r(w[j], w[j + 1], 16) : w[j];
            z[2 * j] = __uint_as_float(two << 16);
            z[2 * j + 1] = __uint_as_float(two & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = j < behind && -j <= before ? elem(at[j]) : 0.f;
    }
}

__device__ __forceinline__ float bias_at(const LgParams& p, long long row, int i) {
    const long long b = row * p.bias_stride + i;
    return p.bias_bf16 ? __bfloat162float(__ldg((const __nv_bfloat16*)p.bias + b)) : __ldg((const float*)p.bias + b);
}

template <typename TL, typename TO, int THREADS, int GROUPS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) adjust_logits_kernel(const __grid_constant__ LgParams p) {
    extern __shared__ uint4 lg_smem[];
    __shared__ int listed;
    constexpr unsigned step = THREADS * 8, piece = step * GROUPS;
    // seen: of each id of the piece how often it is in the history, then, for an id of the list, the value it ends with
    unsigned* seen = (unsigned*)lg_smem;                            // [piece]
    unsigned short* list = (unsigned short*)(seen + piece);         // [piece]: ids that are in the history or in the row's list of biases
    int* biased = (int*)(list + piece);                             // [piece] if bias_count: 1 + which entry of that list
    const long long row = blockIdx.x / p.pieces;
    const int k = (int)(blockIdx.x - row * p.pieces);
    const TL* in = (const TL*)p.logits + row * p.logits_stride;
    TO* out = (TO*)p.out + row * p.out_stride;
    const int vocab = (int)p.vocab;
    const int lead = (int)(((uintptr_t)in & 15) / sizeof(TL));
    const int first = k * (int)piece - lead;                        // index of the piece's first element; below 0: none
    const int tid = threadIdx.x;
    const bool sparse = p.count || p.bias_count;

    // what does not depend on anything is asked for first: the first ids of the history (where they are behind the length they are
    // dropped), the settings, the logits
    const long long base = row * p.history_stride;
    long long ids[kLgAhead];
    int len = p.history_len, prompt = 0;
    if (p.count) {
#pragma unroll
        for (int j = 0; j < kLgAhead; ++j) {
            const int t = tid + j * THREADS;
            ids[j] = t < p.history_len ? id_at(p.history, p.history64, base + t) : -1;
        }
        if (p.lengths) len = min(max(__ldg(p.lengths + row), 0), len);
        if (p.prompts) prompt = min(max(__ldg(p.prompts + row), 0), len);
    }
    uint4 raw[GROUPS][sizeof(TL) / 2];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int i = first + (int)(g * step) + tid * 8;
        if (i >= 0 && i <= vocab - 8)
#pragma unroll
            for (int j = 0; j < (int)sizeof(TL) / 2; ++j) raw[g][j] = *((const uint4*)(in + i) + j);
    }
    if (sparse) {
        for (unsigned i = tid; i < piece / 4; i += THREADS) lg_smem[i] = make_uint4(0, 0, 0, 0);
        if (p.bias_count)
            for (unsigned i = tid; i < piece / 4; i += THREADS) ((uint4*)biased)[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) listed = 0;
        __syncthreads();
        // Position of an id in the piece, or >= piece.  An id from 2^32 - lead on would come out below lead, where no element is.
        const auto place = [&](long long id) { return (unsigned)((unsigned long long)id >> 32) ? piece : (unsigned)id - (unsigned)first; };
        const auto is_element = [&](unsigned at) { return at < piece && (unsigned)(first + (int)at) < (unsigned)vocab; };
        const auto count = [&](long long id, int t) {
            const unsigned at = place(id);
            if (!is_element(at)) return;
            const unsigned old = t < prompt ? atomicOr(seen + at, kLgPrompt) : atomicAdd(seen + at, 1u);
            if (!old) list[atomicAdd(&listed, 1)] = (unsigned short)at;     // in any order: each id of the list is dealt with by itself
        };
        if (p.count) {
#pragma unroll
            for (int j = 0; j < kLgAhead; ++j)
                if (tid + j * THREADS < len) count(ids[j], tid + j * THREADS);
            for (int t0 = tid + kLgAhead * THREADS; t0 < len; t0 += kLgAhead * THREADS) {
#pragma unroll
                for (int j = 0; j < kLgAhead; ++j) ids[j] = t0 + j * THREADS < len ? id_at(p.history, p.history64, base + t0 + j * THREADS) : -1;
#pragma unroll
                for (int j = 0; j < kLgAhead; ++j)
                    if (t0 + j * THREADS < len) count(ids[j], t0 + j * THREADS);
            }
            __syncthreads();
        }
        if (p.bias_count) {
            for (int t = tid; t < (int)p.bias_count; t += THREADS) {
                const unsigned at = place(id_at(p.bias_ids, p.bias_ids64, row * p.bias_count + t));
                if (!is_element(at)) continue;
                const int old = atomicMax(biased + at, t + 1);              // given twice: the later one
                if (!old && !seen[at]) list[atomicAdd(&listed, 1)] = (unsigned short)at;
            }
            __syncthreads();
        }
        const float rep = p.repetition ? __ldg(p.repetition + row) : p.rep, pres = p.presence ? __ldg(p.presence + row) : p.pres,
                    freq = p.frequency ? __ldg(p.frequency + row) : p.freq;
        for (int e = tid; e < listed; e += THREADS) {
            const unsigned at = list[e], w = seen[at];
            const int i = first + (int)at;
            float v = elem(in[i]);
            if (w) {
                const unsigned n = w & ~kLgPrompt;
                v = v > 0.f ? v / rep : v * rep;
                if (n) v -= fmaf(freq, (float)n, pres);
            }
            if (p.bias) v += bias_at(p, row, i);
            if (p.bias_count && biased[at]) v += __ldg(p.bias_values + row * p.bias_count + biased[at] - 1);
            seen[at] = v == 0.f ? 0x80000000u : __float_as_uint(v);         // 0 is for ids that are not in the list
        }
        __syncthreads();
    }
    const uint32_t* allowed = p.allowed ? p.allowed + row * p.allowed_stride : nullptr;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int at = g * (int)step + tid * 8, i = first + at;
        if (i >= 0 && i <= vocab - 8) {
            float x[8];
            read8((const TL*)raw[g], x);
            if (p.bias) {
                float z[8];
                const long long b = row * p.bias_stride + i;
                if (p.bias_bf16) bias8((const __nv_bfloat16*)p.bias + b, i, vocab - i, z);
                else bias8((const float*)p.bias + b, i, vocab - i, z);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += z[j];
            }
            if (sparse) {
                unsigned w[8];
                *(uint4*)w = *(const uint4*)(seen + at);
                *(uint4*)(w + 4) = *(const uint4*)(seen + at + 4);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = w[j] ? __uint_as_float(w[j]) : x[j];
            }
            if (allowed) {              // bits i .. i + 7, of one word or two
                const int w0 = i >> 5, w1 = (i + 7) >> 5;
                const unsigned a = __ldg(allowed + w0), bits = __funnelshift_r(a, w1 > w0 ? __ldg(allowed + w1) : a, (unsigned)i & 31u);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (bits >> j) & 1 ? x[j] : -INFINITY;
            }
            if (((uintptr_t)(out + i) & 15) == 0) {
                write8(out + i, x);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) put(x[j], out + i + j);
            }
        } else {                        // a group that hangs over an end of the row, or lies behind it
            for (int j = max(0, -i); j < 8 && i + j < vocab; ++j) {
                float v = elem(in[i + j]);
                if (p.bias) v += bias_at(p, row, i + j);
                if (sparse && seen[at + j]) v = __uint_as_float(seen[at + j]);
                if (allowed && !((__ldg(allowed + ((i + j) >> 5)) >> ((i + j) & 31)) & 1)) v = -INFINITY;
                put(v, out + i + j);
            }
        }
    }
}

int bytes_of(bpt_dtype t) { return t == BPT_F32 ? 4 : 2; }
bool on_element(const void* q, int bytes) { return ((uintptr_t)q & (bytes - 1)) == 0; }
bool is_type(bpt_dtype t) { return t == BPT_F32 || t == BPT_BF16; }

bpt_status check_logits(const bpt_logits_args* a) {
    if (!a || a->rows < 0 || a->vocab < 1 || !is_type(a->dtype) || !is_type(a->out_dtype)) return BPT_ERR_INVALID_ARG;
    if (a->history_len < 0 || a->bias_count < 0) return BPT_ERR_INVALID_ARG;
    if (a->rows == 0) return BPT_OK;                // empty tensors may have no address
    if (a->rows > 1 && (a->logits_stride < a->vocab || a->out_stride < a->vocab)) return BPT_ERR_INVALID_ARG;
    if (a->history_len > 0) {
        if ((a->history_bytes != 4 && a->history_bytes != 8) || !a->history || !on_element(a->history, a->history_bytes)) return BPT_ERR_INVALID_ARG;
        if (a->history_stride < 0) return BPT_ERR_INVALID_ARG;
        if (!on_element(a->lengths, 4) || !on_element(a->prompt_lengths, 4)) return BPT_ERR_INVALID_ARG;
        if (!a->repetition_rows && !(a->repetition > 0.f && std::isfinite(a->repetition))) return BPT_ERR_INVALID_ARG;
        if (!a->presence_rows && !std::isfinite(a->presence)) return BPT_ERR_INVALID_ARG;
        if (!a->frequency_rows && !std::isfinite(a->frequency)) return BPT_ERR_INVALID_ARG;
        if (!on_element(a->repetition_rows, 4) || !on_element(a->presence_rows, 4) || !on_element(a->frequency_rows, 4)) return BPT_ERR_INVALID_ARG;
    }
    if (a->bias && (!is_type(a->bias_dtype) || !on_element(a->bias, bytes_of(a->bias_dtype)) || (a->bias_stride && a->bias_stride < a->vocab)))
        return BPT_ERR_INVALID_ARG;
    if (a->bias_count > 0 && ((a->bias_id_bytes != 4 && a->bias_id_bytes != 8) || !a->bias_ids || !a->bias_values ||
                              !on_element(a->bias_ids, a->bias_id_bytes) || !on_element(a->bias_values, 4)))
        return BPT_ERR_INVALID_ARG;
    if (a->allowed && (!on_element(a->allowed, 4) || (a->allowed_stride && a->allowed_stride < (a->vocab + 31) / 32))) return BPT_ERR_INVALID_ARG;
    if (a->vocab > 0x3fffffffll || a->history_len > 0x3fffffffll || a->bias_count > 0x3fffffffll || a->rows > 0x3fffffffll) return BPT_ERR_UNSUPPORTED;
    if (a->rows * ((a->vocab + kLgStep) / kLgStep + 1) > 0x7fffffffll) return BPT_ERR_UNSUPPORTED;
    return BPT_OK;
}

template <typename TL, typename TO, int THREADS, int GROUPS>
bpt_status run(LgParams p, long long rows, cudaStream_t st) {
    constexpr int piece = THREADS * 8 * GROUPS;
    p.pieces = (int)((p.vocab + 16 / sizeof(TL) - 1 + piece - 1) / piece);       // wherever the row starts
    const size_t smem = (size_t)piece * (p.bias_count ? 10 : p.count ? 6 : 0);
    if (smem > 40 * 1024 &&     // with the static part, 48 KB is the limit without asking
        cudaFuncSetAttribute(adjust_logits_kernel<TL, TO, THREADS, GROUPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
        return BPT_ERR_CUDA;
    adjust_logits_kernel<TL, TO, THREADS, GROUPS><<<(unsigned)(rows * p.pieces), THREADS, smem, st>>>(p);
    const bool ok = cudaGetLastError() == cudaSuccess;
    trace_mark(st, "adjust_logits");
    return ok ? BPT_OK : BPT_ERR_CUDA;
}
template <typename TL, typename TO>
bpt_status pick(const LgParams& p, long long rows, cudaStream_t st) {
#ifdef LG_VARIANT
    if (getenv("LG_VARIANT")) switch (atoi(getenv("LG_VARIANT"))) {
        case 0: return run<TL, TO, 1024, 1>(p, rows, st);
        case 1: return run<TL, TO, 512, 1>(p, rows, st);
        case 2: return run<TL, TO, 512, 2>(p, rows, st);
        case 3: return run<TL, TO, 256, 1>(p, rows, st);
        case 4: return run<TL, TO, 256, 2>(p, rows, st);
        case 5: return run<TL, TO, 256, 4>(p, rows, st);
        case 6: return run<TL, TO, 1024, 2>(p, rows, st);
    }
#endif
    return run<TL, TO, 1024, 1>(p, rows, st);
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" bpt_status bpt_adjust_logits(const bpt_logits_args* a, void* out, void* cuda_stream) {
    const bpt_status s = check_logits(a);
    if (s != BPT_OK) return s;
    if (a->rows == 0) return BPT_OK;
    if (!a->logits || !out || !on_element(a->logits, bytes_of(a->dtype)) || !on_element(out, bytes_of(a->out_dtype))) return BPT_ERR_INVALID_ARG;
    LgParams p{};
    p.logits = a->logits; p.out = out; p.history = a->history;
    p.lengths = a->lengths; p.prompts = a->prompt_lengths;
    p.repetition = a->repetition_rows; p.presence = a->presence_rows; p.frequency = a->frequency_rows;
    p.rep = a->repetition; p.pres = a->presence; p.freq = a->frequency;
    p.bias = a->bias; p.bias_ids = a->bias_ids; p.bias_values = a->bias_values; p.allowed = reinterpret_cast<const uint32_t*>(a->allowed);
    p.vocab = a->vocab; p.logits_stride = a->logits_stride; p.out_stride = a->out_stride; p.history_stride = a->history_stride;
    p.bias_stride = a->bias_stride; p.allowed_stride = a->allowed_stride;
    p.bias_count = a->bias_count;
    p.history_len = (int)a->history_len; p.history64 = a->history_bytes == 8; p.bias_ids64 = a->bias_id_bytes == 8; p.bias_bf16 = a->bias_dtype == BPT_BF16;
    // settings that change nothing need no history
    p.count = a->history_len > 0 && (a->repetition_rows || a->presence_rows || a->frequency_rows || a->repetition != 1.f || a->presence != 0.f || a->frequency != 0.f);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    typedef __nv_bfloat16 bf;
    if (a->dtype == BPT_F32) return a->out_dtype == BPT_F32 ? pick<float, float>(p, a->rows, st) : pick<float, bf>(p, a->rows, st);
    return a->out_dtype == BPT_F32 ? pick<bf, float>(p, a->rows, st) : pick<bf, bf>(p, a->rows, st);
}
