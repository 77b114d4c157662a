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

#include "bpt_internal.cuh"

namespace bpt {
namespace {

constexpr int kLgSms = 148;
constexpr int kLgThreads = 256;
constexpr int kLgStep = kLgThreads * 8;     // elements per CTA and group of 8 per thread

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

template <typename TL, typename TO, int GROUPS>
__global__ void __launch_bounds__(kLgThreads) adjust_logits_kernel(const __grid_constant__ LgParams p) {
    extern __shared__ unsigned lg_smem[];
    constexpr int piece = kLgStep * GROUPS;
    unsigned* seen = lg_smem;                                   // [piece] if count
    int* biased = (int*)(lg_smem + (p.count ? piece : 0));      // [piece] if bias_count: 1 + which entry of the row's list
    const long long row = blockIdx.x / p.pieces;
    const int k = (int)(blockIdx.x - row * p.pieces);
    const TL* in = (const TL*)p.logits + row * p.logits_stride;
    TO* out = (TO*)p.out + row * p.out_stride;
    const int lead = (int)(((uintptr_t)in & 15) / sizeof(TL));
    const long long first = (long long)k * piece - lead;        // index of the piece's first element; below 0: none
    const int tid = threadIdx.x;

    float x[GROUPS][8];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const long long i = first + g * kLgStep + tid * 8;
        if (i >= 0 && i + 8 <= p.vocab) {
            read8(in + i, x[g]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[g][j] = i + j >= 0 && i + j < p.vocab ? elem(in[i + j]) : 0.f;
        }
    }
    if (p.count)
        for (int i = tid; i < piece; i += kLgThreads) seen[i] = 0;
    if (p.bias_count)
        for (int i = tid; i < piece; i += kLgThreads) biased[i] = 0;
    if (p.count || p.bias_count) __syncthreads();
    float rep = p.rep, pres = p.pres, freq = p.freq;
    if (p.count) {
        if (p.repetition) rep = __ldg(p.repetition + row);
        if (p.presence) pres = __ldg(p.presence + row);
        if (p.frequency) freq = __ldg(p.frequency + row);
        int len = p.history_len, prompt = 0;
        if (p.lengths) len = min(max(__ldg(p.lengths + row), 0), len);
        if (p.prompts) prompt = min(max(__ldg(p.prompts + row), 0), len);
        const long long base = row * p.history_stride;
#pragma unroll 8
        for (int t = tid; t < len; t += kLgThreads) {
            const unsigned long long at = (unsigned long long)id_at(p.history, p.history64, base + t) - (unsigned long long)first;
            if (at < piece) {                       // of this piece; ids outside the vocabulary are in no piece's elements
                if (t < prompt) atomicOr(seen + at, kLgPrompt);
                else atomicAdd(seen + at, 1u);
            }
        }
    }
    for (long long t = tid; t < p.bias_count; t += kLgThreads) {
        const unsigned long long at = (unsigned long long)id_at(p.bias_ids, p.bias_ids64, row * p.bias_count + t) - (unsigned long long)first;
        if (at < piece) atomicMax(biased + at, (int)t + 1);      // given twice: the later one
    }
    if (p.count || p.bias_count) __syncthreads();
    const uint32_t* allowed = p.allowed ? p.allowed + row * p.allowed_stride : nullptr;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int at = g * kLgStep + tid * 8;
        const long long i = first + at;
        if (i + 8 <= 0 || i >= p.vocab) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i + j < 0 || i + j >= p.vocab) continue;
            float v = x[g][j];
            if (p.count) {
                const unsigned w = seen[at + j];
                if (w) {
                    const unsigned n = w & ~kLgPrompt;
                    v = v > 0.f ? v / rep : v * rep;
                    if (n) v -= fmaf(freq, (float)n, pres);
                }
            }
            if (p.bias) {
                const long long b = row * p.bias_stride + i + j;
                v += p.bias_bf16 ? __bfloat162float(((const __nv_bfloat16*)p.bias)[b]) : ((const float*)p.bias)[b];
            }
            if (p.bias_count) {
                const int e = biased[at + j];
                if (e) v += __ldg(p.bias_values + row * p.bias_count + e - 1);
            }
            if (allowed && !((__ldg(allowed + ((i + j) >> 5)) >> ((i + j) & 31)) & 1)) v = -INFINITY;
            x[g][j] = v;
        }
        if (i >= 0 && i + 8 <= p.vocab && ((uintptr_t)(out + i) & 15) == 0) {
            write8(out + i, x[g]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j >= 0 && i + j < p.vocab) put(x[g][j], out + i + j);
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

template <typename TL, typename TO, int GROUPS>
bpt_status run(LgParams p, long long rows, cudaStream_t st) {
    constexpr int piece = kLgStep * GROUPS;
    p.pieces = (int)((p.vocab + 16 / sizeof(TL) - 1 + piece - 1) / piece);       // wherever the row starts
    const size_t smem = (size_t)piece * 4 * ((p.count ? 1 : 0) + (p.bias_count ? 1 : 0));
    if (smem > 48 * 1024 && cudaFuncSetAttribute(adjust_logits_kernel<TL, TO, GROUPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
        return BPT_ERR_CUDA;
    adjust_logits_kernel<TL, TO, GROUPS><<<(unsigned)(rows * p.pieces), kLgThreads, smem, st>>>(p);
    const bool ok = cudaGetLastError() == cudaSuccess;
    trace_mark(st, "adjust_logits");
    return ok ? BPT_OK : BPT_ERR_CUDA;
}
template <typename TL, typename TO>
bpt_status pick(const LgParams& p, long long rows, cudaStream_t st) {
    const long long steps = rows * ((p.vocab + kLgStep - 1) / kLgStep);
    // larger pieces read the history less often, once there are CTAs enough
    return steps >= 8 * kLgSms ? run<TL, TO, 4>(p, rows, st) : run<TL, TO, 1>(p, rows, st);
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
