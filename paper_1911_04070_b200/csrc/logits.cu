// What a decoding step does to its logits before a token is taken: penalties for tokens that stand in the history, biases, masks.
// See bpt_adjust_logits in include/bpt.h.
//
// Bound by memory for a large batch, by latency for a small one.  Few ids of a vocabulary stand in a history: one pass computes
// allowed ? logits + bias : -inf for every element, as if there were none, and the ids that stand there or in the row's own list of biases are found,
// once each, and written once more.  Counts are whole numbers in shared memory, so the order of the atomics does not show.
// Two ways, by the rule at plan(): in one launch, each CTA finding the ids of its own piece of the row while its other threads pass over that
// (one sequence, 256 ids, history of 8192: 5.5 us; 32 rows of 32000, histories of 4096: 6.6 us); or, for many pieces, a launch that lists each
// row's ids by a hash table beside the pass, and one that writes them behind it (256 rows of 128001 in bf16 with bias and mask: the pass
// 34 us without a history, 3.9 TB/s, where PyTorch's copy_ of the logits takes 28 and its neg 24; 48 us with histories of 2048, of which listing leaves
// the pass fewer SMs at first and the last launch is the tail.  With the ids found by every piece for itself 95 us).  In place the pass waits
// for the listing before it writes: with a mask and such histories 53 us against 49 (fp32 77 against 71); 32 rows of 32000 in one launch 10.2
// against 8.2, since the logits of a piece's ids are read before it is written.
//
// Rows may start anywhere (an odd vocabulary, a slice of a larger tensor): a row's elements are taken in groups of 8 that lie on
// 16-byte boundaries of the logits, whatever their index.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "any8.cuh"
#include "bpt_internal.cuh"

namespace bpt {
namespace {

constexpr int kLgSms = 148;
// Threads that pass over a piece, 16 elements each, where that is all a CTA does; where it also goes through the history, and
// then the threads that do that.
constexpr int kLgStream = 256, kLgStreamToo = 512, kLgSparse = 512;
constexpr int kLgPiece = kLgStream * 16, kLgPieceToo = kLgStreamToo * 16;

struct LgListed { unsigned id; float value; };
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
    int history_len, history64, bias_ids64, bias_bf16, pieces, count, in_place;   // count: there is a history that matters
    float rep, pres, freq;
    LgListed* listed;           // [rows][listed_stride], or null
    int* n_listed;              // [rows]
    long long listed_stride;
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

struct NoBias {};

__device__ __forceinline__ float bias_at(const LgParams& p, long long row, int i) {
    const long long b = row * p.bias_stride + i;
    return p.bias_bf16 ? __bfloat162float(__ldg((const __nv_bfloat16*)p.bias + b)) : __ldg((const float*)p.bias + b);
}
__device__ __forceinline__ bool is_allowed(const uint32_t* allowed, int i) { return !allowed || ((__ldg(allowed + (i >> 5)) >> (i & 31)) & 1); }

// What a listed id ends with.  w: its word of the counts; e: 1 + its entry of the row's own list of biases, or 0.
__device__ __forceinline__ float listed_value(const LgParams& p, long long row, int i, float v, unsigned w, int e, float rep, float pres, float freq,
                                              const uint32_t* allowed) {
    if (w) {
        const unsigned n = w & ~kLgPrompt;
        v = v > 0.f ? v / rep : v * rep;
        if (n) v -= fmaf(freq, (float)n, pres);
    }
    if (p.bias) v += bias_at(p, row, i);
    if (e) v += __ldg(p.bias_values + row * p.bias_count + e - 1);
    return is_allowed(allowed, i) ? v : -INFINITY;
}

// What needs no history, for this thread's two groups of 8 elements of a piece, STEP elements apart: out = allowed ? logits + bias : -inf.
// All loads are on their way together, before `ready` is called, where all of those lie in the row.
template <typename TL, typename TO, typename B, bool MASK, int STEP, typename F>
__device__ __forceinline__ void stream(const LgParams& p, long long row, const TL* in, TO* out, const B* bias, const uint32_t* allowed, int ia, F&& ready) {
    constexpr bool BIAS = !std::is_same_v<B, NoBias>;
    constexpr int pieces = sizeof(TL) / 2;      // of 16 bytes
    const int vocab = (int)p.vocab, ib = ia + STEP;
    const bool inside = ia >= 16 && ib <= vocab - 24;
    uint4 raw[2][pieces];
    Any8<std::conditional_t<BIAS, B, float>> z[2];
    unsigned lo[2], hi[2];
    if (inside) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int j = 0; j < pieces; ++j) raw[g][j] = *((const uint4*)(in + (g ? ib : ia)) + j);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int i = g ? ib : ia;
            if constexpr (BIAS) z[g].load(bias + i);
            if constexpr (MASK) {
                lo[g] = __ldg(allowed + (i >> 5));
                hi[g] = __ldg(allowed + ((i + 7) >> 5));
            }
        }
    }
    ready();        // all threads together: there may be a barrier in it
    if (inside) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int i = g ? ib : ia;
            float x[8];
            read8((const TL*)raw[g], x);
            if constexpr (BIAS) {
                float b[8];
                z[g].get(b);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += b[j];
            }
            if constexpr (MASK) {       // bits i .. i + 7, of one word or two
                const unsigned bits = __funnelshift_r(lo[g], hi[g], (unsigned)i & 31u);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (bits >> j) & 1 ? x[j] : -INFINITY;
            }
            if (((uintptr_t)(out + i) & 15) == 0) {
                write8(out + i, x);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) put(x[j], out + i + j);
            }
        }
    } else {                            // near an end of the row, over it or behind it
#pragma unroll 1
        for (int i = ia; i <= ib; i += STEP)
#pragma unroll 1
            for (int j = max(0, -i); j < 8 && i + j < vocab; ++j) {
                const float v = elem(in[i + j]) + (BIAS ? bias_at(p, row, i + j) : 0.f);
                put(is_allowed(allowed, i + j) ? v : -INFINITY, out + i + j);
            }
    }
}

// A row's ids that are in its history or its own list of biases, once each, with the values that they end with: an open hash table in shared
// memory, one CTA per row.  Runs beside the pass over the vocabulary, behind which put_listed_kernel writes the values.
constexpr int kLgSlots = 16384, kLgMostIds = kLgSlots * 3 / 4, kLgHashThreads = 1024;

template <typename TL>
__global__ void __launch_bounds__(kLgHashThreads) list_ids_kernel(const __grid_constant__ LgParams p, int slots) {
    extern __shared__ uint4 lg_smem[];
    __shared__ int listed;
    volatile unsigned* key = (volatile unsigned*)lg_smem;       // [slots]: 1 + id, or 0
    unsigned* seen = (unsigned*)lg_smem + slots;                // [slots]: as in adjust_logits_kernel
    int* biased = (int*)(seen + slots);                         // [slots] if bias_count
    const long long row = blockIdx.x;
    const TL* in = (const TL*)p.logits + row * p.logits_stride;
    const int vocab = (int)p.vocab, tid = threadIdx.x;
    const uint32_t* allowed = p.allowed ? p.allowed + row * p.allowed_stride : nullptr;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long base = row * p.history_stride;
    long long ids[kLgAhead];
    int len = p.history_len, prompt = 0;
    if (p.count) {
#pragma unroll
        for (int j = 0; j < kLgAhead; ++j) {
            const int t = tid + j * kLgHashThreads;
            ids[j] = t < p.history_len ? id_at(p.history, p.history64, base + t) : -1;
        }
        if (p.lengths) len = min(max(__ldg(p.lengths + row), 0), len);
        if (p.prompts) prompt = min(max(__ldg(p.prompts + row), 0), len);
    }
    for (int i = tid; i < slots / 4 * (p.bias_count ? 3 : 2); i += kLgHashThreads) lg_smem[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) listed = 0;
    __syncthreads();
    // The slot of an id; there are more slots than ids, so one is found.  Most ids of a text are there already: looked at before they are claimed.
    const auto slot_of = [&](unsigned id) {
        unsigned s = (id * 2654435761u) >> 7 & (unsigned)(slots - 1);
        for (;; s = (s + 1) & (unsigned)(slots - 1)) {
            unsigned old = key[s];
            if (!old) old = atomicCAS((unsigned*)key + s, 0u, id + 1);
            if (!old || old == id + 1) return s;
        }
    };
    const auto count = [&](long long id, int t) {
        if ((unsigned long long)id >= (unsigned long long)vocab) return;
        const unsigned s = slot_of((unsigned)id);
        if (t < prompt) atomicOr(seen + s, kLgPrompt);
        else atomicAdd(seen + s, 1u);
    };
    if (p.count) {
#pragma unroll
        for (int j = 0; j < kLgAhead; ++j)
            if (tid + j * kLgHashThreads < len) count(ids[j], tid + j * kLgHashThreads);
        for (int t = tid + kLgAhead * kLgHashThreads; t < len; t += kLgHashThreads) count(id_at(p.history, p.history64, base + t), t);
    }
    for (int t = tid; t < (int)p.bias_count; t += kLgHashThreads) {
        const long long id = id_at(p.bias_ids, p.bias_ids64, row * p.bias_count + t);
        if ((unsigned long long)id < (unsigned long long)vocab) atomicMax(biased + slot_of((unsigned)id), t + 1);    // given twice: the later one
    }
    __syncthreads();
    const float rep = p.repetition ? __ldg(p.repetition + row) : p.rep, pres = p.presence ? __ldg(p.presence + row) : p.pres,
                freq = p.frequency ? __ldg(p.frequency + row) : p.freq;
    LgListed* to = p.listed + row * p.listed_stride;
    for (int s0 = tid; s0 < slots; s0 += kLgAhead * kLgHashThreads) {
        int id[kLgAhead];
        float v[kLgAhead];
#pragma unroll
        for (int j = 0; j < kLgAhead; ++j) {        // the logits of several on their way at once
            const int s = s0 + j * kLgHashThreads;
            id[j] = s < slots ? (int)key[s] - 1 : -1;
            v[j] = id[j] >= 0 ? elem(in[id[j]]) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kLgAhead; ++j) {
            if (id[j] < 0) continue;
            const int s = s0 + j * kLgHashThreads;
            to[atomicAdd(&listed, 1)] = LgListed{(unsigned)id[j], listed_value(p, row, id[j], v[j], seen[s], p.bias_count ? biased[s] : 0, rep, pres, freq, allowed)};
        }
    }
    __syncthreads();
    if (tid == 0) p.n_listed[row] = listed;
}

template <typename TO>
__global__ void __launch_bounds__(kLgHashThreads) put_listed_kernel(const __grid_constant__ LgParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long row = blockIdx.x;
    const int n = p.n_listed[row];
    for (int e = threadIdx.x; e < n; e += kLgHashThreads) {
        const LgListed one = p.listed[row * p.listed_stride + e];
        put(one.value, (TO*)p.out + row * p.out_stride + one.id);
    }
}

// The first STREAM threads of a CTA pass over its piece of a row.  The others, if there are any, go through the row's history and its own list
// of biases meanwhile, and write the ids that stand there once more, behind the others; in place, the others wait until the logits
// of those ids are read.  Where there are no others, list_ids_kernel may be at work on those ids: in place its end is waited for.
template <typename TL, typename TO, int STREAM, int SPARSE>
__global__ void __launch_bounds__(STREAM + SPARSE, SPARSE ? 1 : 4) adjust_logits_kernel(const __grid_constant__ LgParams p) {
    extern __shared__ uint4 lg_smem[];
    __shared__ int listed;
    if (SPARSE == 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int step = STREAM * 8;
    constexpr unsigned piece = 2 * step;
    const unsigned row = blockIdx.x / (unsigned)p.pieces;
    const int k = (int)(blockIdx.x - row * (unsigned)p.pieces);
    const TL* in = (const TL*)p.logits + row * p.logits_stride;
    TO* out = (TO*)p.out + row * p.out_stride;
    const uint32_t* allowed = p.allowed ? p.allowed + row * p.allowed_stride : nullptr;
    const int vocab = (int)p.vocab;
    const int lead = (int)(((uintptr_t)in & 15) / sizeof(TL));
    const int first = k * (int)piece - lead;                        // index of the piece's first element; below 0: none
    if (SPARSE == 0 || threadIdx.x < STREAM) {
        const int i0 = first + (int)threadIdx.x * 8;
        const auto ready = [&] {
            if (SPARSE && p.in_place) __syncthreads();
            if (SPARSE == 0 && p.listed && p.in_place) asm volatile("griddepcontrol.wait;" ::: "memory");
        };
        const long long b = row * p.bias_stride;
        if (!p.bias && allowed) stream<TL, TO, NoBias, true, step>(p, row, in, out, (const NoBias*)nullptr, allowed, i0, ready);
        else if (!p.bias) stream<TL, TO, NoBias, false, step>(p, row, in, out, (const NoBias*)nullptr, nullptr, i0, ready);
        else if (p.bias_bf16 && allowed) stream<TL, TO, __nv_bfloat16, true, step>(p, row, in, out, (const __nv_bfloat16*)p.bias + b, allowed, i0, ready);
        else if (p.bias_bf16) stream<TL, TO, __nv_bfloat16, false, step>(p, row, in, out, (const __nv_bfloat16*)p.bias + b, nullptr, i0, ready);
        else if (allowed) stream<TL, TO, float, true, step>(p, row, in, out, (const float*)p.bias + b, allowed, i0, ready);
        else stream<TL, TO, float, false, step>(p, row, in, out, (const float*)p.bias + b, nullptr, i0, ready);
        if (SPARSE) __syncthreads();
        // the kernel that then writes the listed ids waits for this one to end, and so for the listing, too
        if (SPARSE == 0 && p.listed && !p.in_place && blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    if constexpr (SPARSE > 0) {
        // seen: how often each id of the piece is in the history, then, for a listed id, the value that it ends with
        unsigned* seen = (unsigned*)lg_smem;                            // [piece]
        int* biased = (int*)(seen + piece);                             // [piece] if bias_count: 1 + which entry of the row's list of biases
        unsigned short* list = (unsigned short*)(biased + (p.bias_count ? piece : 0));      // [listed_most]: ids that stand in the history or in that list
        const int tid = (int)threadIdx.x - STREAM;
        const auto join = [&] { __syncwarp(); asm volatile("bar.sync 1, %0;" :: "n"(SPARSE) : "memory"); };
        // the first ids are asked for before their number is known; those behind the length are dropped
        const long long base = row * p.history_stride;
        long long ids[kLgAhead];
        int len = p.history_len, prompt = 0;
        if (p.count) {
#pragma unroll
            for (int j = 0; j < kLgAhead; ++j) {
                const int t = tid + j * SPARSE;
                ids[j] = t < p.history_len ? id_at(p.history, p.history64, base + t) : -1;
            }
            if (p.lengths) len = min(max(__ldg(p.lengths + row), 0), len);
            if (p.prompts) prompt = min(max(__ldg(p.prompts + row), 0), len);
        }
        for (unsigned i = tid; i < piece / 4 * (p.bias_count ? 2 : 1); i += SPARSE) lg_smem[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) listed = 0;
        join();
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
                if (tid + j * SPARSE < len) count(ids[j], tid + j * SPARSE);
            for (int t0 = tid + kLgAhead * SPARSE; t0 < len; t0 += kLgAhead * SPARSE) {
#pragma unroll
                for (int j = 0; j < kLgAhead; ++j) ids[j] = t0 + j * SPARSE < len ? id_at(p.history, p.history64, base + t0 + j * SPARSE) : -1;
#pragma unroll
                for (int j = 0; j < kLgAhead; ++j)
                    if (t0 + j * SPARSE < len) count(ids[j], t0 + j * SPARSE);
            }
            join();
        }
        if (p.bias_count) {
            for (int t = tid; t < (int)p.bias_count; t += SPARSE) {
                const unsigned at = place(id_at(p.bias_ids, p.bias_ids64, row * p.bias_count + t));
                if (!is_element(at)) continue;
                const int old = atomicMax(biased + at, t + 1);              // given twice: the later one
                if (!old && !seen[at]) list[atomicAdd(&listed, 1)] = (unsigned short)at;
            }
            join();
        }
        const float rep = p.repetition ? __ldg(p.repetition + row) : p.rep, pres = p.presence ? __ldg(p.presence + row) : p.pres,
                    freq = p.frequency ? __ldg(p.frequency + row) : p.freq;
        const int n_listed = listed;
        for (int e = tid; e < n_listed; e += SPARSE) {
            const unsigned at = list[e];
            const int i = first + (int)at;
            seen[at] = __float_as_uint(listed_value(p, row, i, elem(in[i]), seen[at], p.bias_count ? biased[at] : 0, rep, pres, freq, allowed));
        }
        if (p.in_place) __syncthreads();        // the logits of the list are read
        __syncthreads();                        // the piece is written
        for (int e = tid; e < n_listed; e += SPARSE) put(__uint_as_float(seen[list[e]]), out + first + list[e]);
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
    if (a->rows * (a->vocab / kLgPiece + 2) > 0x7fffffffll) return BPT_ERR_UNSUPPORTED;
    return BPT_OK;
}

struct LgPlan {
    bool sparse, list;      // ids of a history or of the rows' own lists count; they are listed by a launch of their own
    int pieces, slots;
    long long stride;       // listed ids per row, at most
    size_t bytes;
};
bool counts(const bpt_logits_args& a) {     // settings that change nothing need no history
    return a.history_len > 0 && (a.repetition_rows || a.presence_rows || a.frequency_rows || a.repetition != 1.f || a.presence != 0.f || a.frequency != 0.f);
}
LgPlan plan(const bpt_logits_args& a) {
    LgPlan q{};
    const long long most = (counts(a) ? a.history_len : 0) + a.bias_count;
    q.sparse = most > 0;
    const auto pieces = [&](int piece) { return (int)((a.vocab + 16 / bytes_of(a.dtype) - 1 + piece - 1) / piece); };     // wherever the row starts
    q.stride = std::min(most, (long long)a.vocab);
    // Every CTA of a row going through all of its history is the shorter way while there are few CTAs to a row or to an SM.  B200, bf16 with a mask,
    // microseconds of one launch | of listing apart: 32 rows of 32000, histories of 8000 10 | 23; 128 rows of 32000, 2000 14 | 14; 32 rows of 128000,
    // 8000 21 | 27; 256 rows of 32000, 1000 23 | 16; 64 rows of 128000, 500 21 | 12, 8000 33 | 29; 512 rows of 5000, 2000 19 | 23.
    q.list = q.sparse && pieces(kLgPieceToo) >= 4 && a.rows * pieces(kLgPieceToo) > 5 * kLgSms && most <= kLgMostIds;
    q.pieces = pieces(q.sparse && !q.list ? kLgPieceToo : kLgPiece);
    q.slots = 1024;
    while (q.slots < kLgSlots && q.slots < 2 * most) q.slots *= 2;
    q.bytes = q.list ? (size_t)a.rows * (q.stride * sizeof(LgListed) + 4) : 0;
    return q;
}

template <typename K>
bool start(K kernel, unsigned grid, int threads, size_t smem, bool dependent, cudaStream_t st, const LgParams& p) {
    cudaLaunchAttribute attr[1] = {};       // its launch overlaps the kernel before
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = dependent ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess) return true;
    cudaGetLastError();     // reported by this status, not by the next call of somebody else
    return false;
}
template <typename TL, typename TO, int STREAM, int SPARSE>
bool run(const LgParams& p, long long rows, size_t smem, bool dependent, cudaStream_t st) {
    if (smem > 40 * 1024 &&     // with the static part, 48 KB is the limit without asking
        cudaFuncSetAttribute(adjust_logits_kernel<TL, TO, STREAM, SPARSE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLgPieceToo * 10) != cudaSuccess) {
        cudaGetLastError();     // reported by this status, not by the next call of somebody else
        return false;
    }
    const bool ok = start(adjust_logits_kernel<TL, TO, STREAM, SPARSE>, (unsigned)(rows * p.pieces), STREAM + SPARSE, smem, dependent, st, p);
    trace_mark(st, "adjust_logits");
    return ok;
}
template <typename TL>
bool run_list(const LgParams& p, long long rows, int slots, cudaStream_t st) {
    const size_t smem = (size_t)slots * (p.bias_count ? 12 : 8);
    if (smem > 40 * 1024 &&
        cudaFuncSetAttribute(list_ids_kernel<TL>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLgSlots * 12) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    list_ids_kernel<TL><<<(unsigned)rows, kLgHashThreads, smem, st>>>(p, slots);
    const bool ok = cudaGetLastError() == cudaSuccess;
    trace_mark(st, "list_ids");
    return ok;
}
template <typename TL, typename TO>
bpt_status launch(const LgParams& p, const LgPlan& q, long long rows, cudaStream_t st) {
    bool ok;
    if (!q.sparse) {
        ok = run<TL, TO, kLgStream, 0>(p, rows, 0, false, st);
    } else if (q.list) {
        ok = run_list<TL>(p, rows, q.slots, st) && run<TL, TO, kLgStream, 0>(p, rows, 0, true, st) &&
             start(put_listed_kernel<TO>, (unsigned)rows, kLgHashThreads, 0, true, st, p);
        trace_mark(st, "put_listed");
    } else {
        const size_t list = (size_t)std::min<long long>(kLgPieceToo, q.stride) * 2;
        ok = run<TL, TO, kLgStreamToo, kLgSparse>(p, rows, (size_t)kLgPieceToo * (p.bias_count ? 8 : 4) + (list + 15) / 16 * 16, false, st);
    }
    return ok ? BPT_OK : BPT_ERR_CUDA;
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" size_t bpt_adjust_logits_workspace_bytes(const bpt_logits_args* a) {
    return check_logits(a) == BPT_OK && a->rows > 0 ? plan(*a).bytes : 0;
}

extern "C" bpt_status bpt_adjust_logits(const bpt_logits_args* a, void* out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const bpt_status s = check_logits(a);
    if (s != BPT_OK) return s;
    if (a->rows == 0) return BPT_OK;
    if (!a->logits || !out || !on_element(a->logits, bytes_of(a->dtype)) || !on_element(out, bytes_of(a->out_dtype))) return BPT_ERR_INVALID_ARG;
    if (a->logits == out && (a->dtype != a->out_dtype || (a->rows > 1 && a->logits_stride != a->out_stride))) return BPT_ERR_INVALID_ARG;
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
    p.in_place = a->logits == out;
    p.count = counts(*a);
    const LgPlan q = plan(*a);
    p.pieces = q.pieces;
    if (q.list) {
        if (!workspace || workspace_bytes < q.bytes) return BPT_ERR_WORKSPACE;
        if ((uintptr_t)workspace & 15) return BPT_ERR_INVALID_ARG;
        p.listed = static_cast<LgListed*>(workspace);
        p.n_listed = reinterpret_cast<int*>(p.listed + a->rows * q.stride);
        p.listed_stride = q.stride;
    }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    typedef __nv_bfloat16 bf;
    if (a->dtype == BPT_F32) return a->out_dtype == BPT_F32 ? launch<float, float>(p, q, a->rows, st) : launch<float, bf>(p, q, a->rows, st);
    return a->out_dtype == BPT_F32 ? launch<bf, float>(p, q, a->rows, st) : launch<bf, bf>(p, q, a->rows, st);
}
