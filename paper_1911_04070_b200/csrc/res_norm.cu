// The seam between two blocks of a layer (arXiv 1911.04070, Algorithm 2 of Sec. 3.3 has Z = norm(H + GSA(H)) and
// H' = norm(Z + FFN(Z)); this is that step with the scaled residual, gate and second norm that deeper stacks use):
//     n = post(b),   r = alpha h + gate n,   y = norm(r),        row by row over D channels,
// post and norm each absent, layer normalisation or root-mean-square normalisation, and its backward.
//
// Both directions are bound by HBM: a row is read once, lives in registers as fp32 (variance about the mean, in a
// second sweep over the registers), and every result is rounded once to the tensors' type when it is stored.  The forward
// leaves mean and reciprocal deviation of both norms (16 bytes a row) for the backward, which recomputes everything else
// from h and b.
//
// A row belongs to TPR threads, NE channels each: one warp (in the backward above 256 channels two, whose column sums would
// not leave registers for enough warps otherwise) as far as registers go, a whole CTA above.  What remains to be bound by is instructions: the arithmetic is written
// on pairs (fma.rn.f32x2 and the like, two channels an instruction), and weights, biases and gate are turned to fp32 once per
// CTA and kept in shared memory in the order in which the threads read them.  The backward's CTAs each take a fixed,
// contiguous share of the rows and keep the column sums of the parameter gradients in registers; the shares are added by
// a second kernel in a fixed order, so results are bit-reproducible.  Backward rows are fetched two rows ahead into
// shared memory by asynchronous copies; every thread reads back only what it copied itself, so no barrier is needed for them.
#include <algorithm>

#include "bpt_internal.cuh"
#include "mma_tools.cuh"

namespace bpt {
namespace {

constexpr int kRnSms = 148;
constexpr int kRnMaxD = 8192;
// Rows of a thread group in flight (the current one and those ahead), as far as shared memory goes; below two there is no staging.
__host__ __device__ constexpr int cta_threads(int tpr) { return tpr < 128 ? 256 : tpr; }
template <typename T, int VEC, int NE, int TPR>
__host__ __device__ constexpr int bwd_stages() {
    constexpr size_t one = 4 * NE * sizeof(T) * cta_threads(TPR), room = 224 * 1024 - 4 * NE * 4 * TPR;
    return sizeof(T) * VEC < 4 || 2 * one > room ? 1 : 3 * one > room ? 2 : 3;
}

struct RnParams {
    const void *h, *b, *dy, *dr;
    const void *weight, *bias, *post_weight, *post_bias, *gate;
    void *y, *r, *dh, *db, *d_gate;
    float4* stats_out;      // [rows]: mean and 1 / deviation of the post norm, of the norm
    const float4* stats;
    float *part;            // [grid][4][D]: weight, bias, post weight, post bias
    float *gate_part;       // [units][D]
    long long rows, group_rows;
    int D, norm, post, splits, units;
    bool param_bf16, gate_bf16, gate_rows;   // gate_rows: a gate row per row
    bool gate_each;         // forward: the gate's row depends on the row (read from memory, not kept in shared memory)
    float alpha, eps;
};

// Two channels per instruction, kept as 64-bit values so that they stay in register pairs.
typedef unsigned long long pair_t;
__device__ __forceinline__ pair_t mk(float x, float y) { pair_t d; asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y)); return d; }
__device__ __forceinline__ float2 un(pair_t a) { float2 d; asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(a)); return d; }
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) { pair_t d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) { pair_t d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) { pair_t d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ pair_t both(float a) { return mk(a, a); }
__device__ __forceinline__ float elem(const pair_t* x, int e) { const float2 f = un(x[e / 2]); return e & 1 ? f.y : f.x; }

// A thread's NE elements: chunk v is VEC consecutive channels of type T at at(v), or zeros where live(v) is false.
template <typename T, int VEC, int NE, typename At, typename Live>
__device__ __forceinline__ void load_row(pair_t* x, At at, Live live) {
    if constexpr (VEC == 1) {
        auto one = [&](int v) {
            if (!live(v)) return 0.f;
            if constexpr (sizeof(T) == 4) return *reinterpret_cast<const float*>(at(v));
            else return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(at(v)));
        };
#pragma unroll
        for (int i = 0; i < NE / 2; ++i) { const float a = one(2 * i), b = one(2 * i + 1); x[i] = mk(a, b); }
    } else {
#pragma unroll
        for (int v = 0; v < NE / VEC; ++v) {
            if constexpr (sizeof(T) == 4) {
                const ulonglong2 w = live(v) ? *reinterpret_cast<const ulonglong2*>(at(v)) : make_ulonglong2(0, 0);
                x[v * 2] = w.x;
                x[v * 2 + 1] = w.y;
            } else {
                const uint4 q = live(v) ? *reinterpret_cast<const uint4*>(at(v)) : make_uint4(0, 0, 0, 0);
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) x[v * 4 + i] = mk(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
            }
        }
    }
}
// Chunk v of a thread's elements to p
template <typename T, int VEC>
__device__ __forceinline__ void pack(void* p, const pair_t* x, int v) {
    if constexpr (VEC == 1) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float*>(p) = elem(x, v);
        else *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(elem(x, v));
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(x[v * 2], x[v * 2 + 1]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 f = un(x[v * 4 + i]); w[i] = pack_bf16(f.x, f.y); }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
// A parameter of channel c.  Plain loads: __ldg of a bf16 is inline assembly that the compiler may move above a test for a null pointer.
__device__ __forceinline__ float param(const void* p, bool bf16, long long c) {
    if (bf16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[c]);
    return reinterpret_cast<const float*>(p)[c];
}

// Channel of element e of thread t
template <int VEC, int TPR>
__device__ __forceinline__ int channel(int e, int t) { return (e / VEC * TPR + t) * VEC + e % VEC; }
// One parameter row as fp32 in shared memory, four elements of a thread together; `missing` where there is none, zeros past D.
template <int VEC, int NE, int TPR, int RPC>
__device__ __forceinline__ void fill(float4* dst, const void* p, bool bf16, long long off, float missing, int D, int t, int sub) {
    for (int q = sub; q < NE / 4; q += RPC) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = channel<VEC, TPR>(4 * q + i, t);
            f[i] = c >= D ? 0.f : p ? param(p, bf16, off + c) : missing;
        }
        dst[q * TPR + t] = make_float4(f[0], f[1], f[2], f[3]);
    }
}

// Sum of a pair over the TPR threads of a row, the same bits in every thread.  The first exchange leaves v.x with the warp's lower
// half and v.y with its upper half, so that the other four serve both.  slots: for each row group of the CTA two buffers of
// TPR / 32 pairs, used in turn, so that one barrier (of the group's threads) per sum is enough.
template <int TPR> __host__ __device__ constexpr int slot_count() { return TPR > 32 ? cta_threads(TPR) / 16 : 1; }
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float2 v, float2* slots, int& turn) {
    const int lane = threadIdx.x & 31;
    const bool upper = lane & 16;
    float a = (upper ? v.y : v.x) + __shfl_xor_sync(0xffffffffu, upper ? v.x : v.y, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    if constexpr (TPR > 32) {
        float2* s = slots + (threadIdx.x / TPR * 2 + turn) * (TPR / 32);
        turn ^= 1;
        if ((lane & 15) == 0) reinterpret_cast<float*>(s + (threadIdx.x % TPR >> 5))[lane >> 4] = a;
        if constexpr (TPR == cta_threads(TPR)) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
        v = s[0];
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w) { v.x += s[w].x; v.y += s[w].y; }
        return v;
    } else {
        return make_float2(__shfl_sync(0xffffffffu, a, 0), __shfl_sync(0xffffffffu, a, 16));
    }
}
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float2* slots, int& turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        static_assert(TPR == cta_threads(TPR), "the whole CTA");
        float2* s = slots + turn * (TPR / 32);
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5].x = v;
        __syncthreads();
        v = s[0].x;
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w) v += s[w].x;
    }
    return v;
}

// Mean (0 for rms) and reciprocal deviation of the row held in x; channels past D hold zeros (live: chunk inside D).
template <int TPR, int NE, int VEC, typename Live>
__device__ __forceinline__ float2 row_stats(const pair_t* x, int kind, float inv_d, float eps, Live live, float2* slots, int& turn) {
    float mean = 0.f;
    if (kind == BPT_NORM_LAYER) {
        pair_t s = 0;
#pragma unroll
        for (int i = 0; i < NE / 2; ++i) s = add2(s, x[i]);
        mean = row_sum<TPR>(un(s).x + un(s).y, slots, turn) * inv_d;
    }
    pair_t q = 0;
#pragma unroll
    for (int i = 0; i < NE / 2; ++i) {
        const pair_t m = VEC == 1 ? mk(live(2 * i) ? -mean : 0.f, live(2 * i + 1) ? -mean : 0.f) : both(live(2 * i / VEC) ? -mean : 0.f);
        const pair_t c = add2(x[i], m);
        q = fma2(c, c, q);
    }
    return make_float2(mean, rsqrtf(row_sum<TPR>(un(q).x + un(q).y, slots, turn) * inv_d + eps));
}

template <typename T, int VEC, int NE, int TPR>
__global__ void __launch_bounds__(cta_threads(TPR), NE <= 16 ? 1024 / cta_threads(TPR) : 1) res_norm_fwd_kernel(const RnParams p) {
    constexpr int NV = NE / VEC, NP = NE / 2, RPC = cta_threads(TPR) / TPR;
    extern __shared__ __align__(16) float4 prm[];       // [weight, bias if norm; post weight, post bias if post; gate if kept][NE / 4][TPR]
    __shared__ float2 slots[slot_count<TPR>()];
    int turn = 0;
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int D = p.D;
    const float inv_d = 1.f / (float)D;
    auto chan = [&](int v) { return (v * TPR + t) * VEC; };
    auto live = [&](int v) { return chan(v) < D; };
    constexpr int kRow = NE / 4 * TPR;
    const int k_post = p.norm ? 2 : 0, k_gate = k_post + (p.post ? 2 : 0);
    if (p.norm) {
        fill<VEC, NE, TPR, RPC>(prm, p.weight, p.param_bf16, 0, 1.f, D, t, sub);
        fill<VEC, NE, TPR, RPC>(prm + kRow, p.bias, p.param_bf16, 0, 0.f, D, t, sub);
    }
    if (p.post) {
        fill<VEC, NE, TPR, RPC>(prm + k_post * kRow, p.post_weight, p.param_bf16, 0, 1.f, D, t, sub);
        fill<VEC, NE, TPR, RPC>(prm + (k_post + 1) * kRow, p.post_bias, p.param_bf16, 0, 0.f, D, t, sub);
    }
    if (p.gate && !p.gate_each) fill<VEC, NE, TPR, RPC>(prm + k_gate * kRow, p.gate, p.gate_bf16, 0, 1.f, D, t, sub);
    __syncthreads();
    // pairs 2 q and 2 q + 1 of parameter row k
    auto get = [&](int k, int q, pair_t* f) {
        const ulonglong2 w = reinterpret_cast<const ulonglong2*>(prm)[k * kRow + q * TPR + t];
        f[0] = w.x;
        f[1] = w.y;
    };
    for (long long row = (long long)blockIdx.x * RPC + sub; row < p.rows; row += (long long)gridDim.x * RPC) {
        const long long off = row * D;
        pair_t n[NP], r[NP];
        float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
        load_row<T, VEC, NE>(r, [&](int v) { return reinterpret_cast<const T*>(p.h) + off + chan(v); }, live);
        load_row<T, VEC, NE>(n, [&](int v) { return reinterpret_cast<const T*>(p.b) + off + chan(v); }, [&](int v) { return p.b && live(v); });
        if (p.post) {
            const float2 s = row_stats<TPR, NE, VEC>(n, p.post, inv_d, p.eps, live, slots, turn);
            st.x = s.x; st.y = s.y;
            const pair_t scale = both(s.y), minus = both(-s.x);
#pragma unroll
            for (int q = 0; q < NE / 4; ++q) {
                pair_t w[2], c[2];
                get(k_post, q, w);
                get(k_post + 1, q, c);
#pragma unroll
                for (int i = 0; i < 2; ++i) n[2 * q + i] = fma2(mul2(add2(n[2 * q + i], minus), scale), w[i], c[i]);
            }
        }
        if (p.gate) {
            if (p.gate_each) {
                const long long goff = (row / p.group_rows) * D;
                auto g = [&](int e) {
                    const int c = channel<VEC, TPR>(e, t);
                    return c < D ? param(p.gate, p.gate_bf16, goff + c) : 0.f;
                };
#pragma unroll
                for (int i = 0; i < NP; ++i) n[i] = mul2(n[i], mk(g(2 * i), g(2 * i + 1)));
            } else {
#pragma unroll
                for (int q = 0; q < NE / 4; ++q) {
                    pair_t w[2];
                    get(k_gate, q, w);
                    n[2 * q] = mul2(n[2 * q], w[0]);
                    n[2 * q + 1] = mul2(n[2 * q + 1], w[1]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) r[i] = fma2(both(p.alpha), r[i], n[i]);
        if (p.r)
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (live(v)) pack<T, VEC>(reinterpret_cast<T*>(p.r) + off + chan(v), r, v);
        if (p.norm) {
            const float2 s = row_stats<TPR, NE, VEC>(r, p.norm, inv_d, p.eps, live, slots, turn);
            st.z = s.x; st.w = s.y;
            const pair_t scale = both(s.y), minus = both(-s.x);
#pragma unroll
            for (int q = 0; q < NE / 4; ++q) {
                pair_t w[2], c[2];
                get(0, q, w);
                get(1, q, c);
#pragma unroll
                for (int i = 0; i < 2; ++i) r[2 * q + i] = fma2(mul2(add2(r[2 * q + i], minus), scale), w[i], c[i]);
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (live(v)) pack<T, VEC>(reinterpret_cast<T*>(p.y) + off + chan(v), r, v);
        }
        if (p.stats_out && t == 0) p.stats_out[row] = st;
    }
}

// One piece (VEC elements) of a row into shared memory; pieces of two bytes have no asynchronous copy and are not staged.
// The staged pieces are read back by plain loads, so copy and wait are ordered against memory accesses for the compiler.
template <int BYTES>
__device__ __forceinline__ void stage_copy(uint32_t dst, const void* src) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
template <int N> __device__ __forceinline__ void stage_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Shared memory of the backward: four parameter rows, then the staged pieces, or the exchange of the column sums
template <typename T, int VEC, int NE, int TPR>
__host__ __device__ constexpr size_t bwd_smem() {
    constexpr int threads = cta_threads(TPR);
    constexpr int stages = bwd_stages<T, VEC, NE, TPR>();
    const size_t stage = stages > 1 ? (size_t)stages * 4 * NE * sizeof(T) * threads : 0;
    const size_t xch = TPR < threads ? (size_t)threads * NE * 4 : 0;
    return (size_t)4 * NE * 4 * TPR + (stage > xch ? stage : xch);
}

template <typename T, int VEC, int NE, int TPR, bool POST>
__global__ void __launch_bounds__(cta_threads(TPR), cta_threads(TPR) <= 256 ? 512 / cta_threads(TPR) : 1) res_norm_bwd_kernel(const RnParams p) {
    constexpr int NV = NE / VEC, NP = NE / 2, THREADS = cta_threads(TPR), RPC = THREADS / TPR;
    constexpr int PIECE = VEC * (int)sizeof(T);
    constexpr int STAGES = bwd_stages<T, VEC, NE, TPR>();
    constexpr bool STAGED = STAGES > 1;
    extern __shared__ __align__(16) float4 prm[];       // [weight, post weight, post bias, gate][NE / 4][TPR]
    constexpr int kRow = NE / 4 * TPR;
    unsigned char* const smem = reinterpret_cast<unsigned char*>(prm + 4 * kRow);
    __shared__ float2 slots[slot_count<TPR>()];
    int turn = 0;
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int D = p.D;
    const float inv_d = 1.f / (float)D;
    auto chan = [&](int v) { return (v * TPR + t) * VEC; };
    auto live = [&](int v) { return chan(v) < D; };
    const uint32_t mine = smem_u32(smem) + threadIdx.x * PIECE;
    const void* src[4] = {p.h, p.b, p.norm ? p.dy : nullptr, p.dr};
    auto slot = [&](int stage, int a, int v) { return (uint32_t)(((stage * 4 + a) * NV + v) * THREADS * PIECE); };
    auto fetch = [&](long long row, long long off, long long end, int stage) {     // off: row * D
        if constexpr (STAGED) {
            if (row < end) {
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    if (src[a])
#pragma unroll
                        for (int v = 0; v < NV; ++v)
                            if (live(v)) stage_copy<PIECE>(mine + slot(stage, a, v), reinterpret_cast<const T*>(src[a]) + off + chan(v));
            }
            cp_async_commit();
        }
    };
    // Staged: what has no source (a missing tensor, channels past D) holds zeros from the start, so every read is unconditional.
    auto take = [&](long long off, int stage, int a, pair_t* x) {
        if constexpr (STAGED) load_row<T, VEC, NE>(x, [&](int v) { return smem + threadIdx.x * PIECE + slot(stage, a, v); }, [](int) { return true; });
        else load_row<T, VEC, NE>(x, [&](int v) { return reinterpret_cast<const T*>(src[a]) + off + chan(v); }, [&](int v) { return src[a] && live(v); });
    };
    auto clear_stages = [&] {
        if constexpr (STAGED)
#pragma unroll 1
            for (int stage = 0; stage < STAGES; ++stage)
#pragma unroll
                for (int a = 0; a < 4; ++a)
#pragma unroll
                    for (int v = 0; v < NV; ++v)
                        if (!src[a] || !live(v))
#pragma unroll
                            for (int i = 0; i < PIECE / 4; ++i) *reinterpret_cast<uint32_t*>(smem + threadIdx.x * PIECE + slot(stage, a, v) + 4 * i) = 0;
    };
    auto get = [&](int k, int q, pair_t* f) {
        const ulonglong2 w = reinterpret_cast<const ulonglong2*>(prm)[k * kRow + q * TPR + t];
        f[0] = w.x;
        f[1] = w.y;
    };

    pair_t s_w[NP], s_b[NP], s_g[NP], s_pw[POST ? NP : 1], s_pb[POST ? NP : 1];   // this thread's column sums
#pragma unroll
    for (int i = 0; i < NP; ++i) s_w[i] = s_b[i] = s_g[i] = 0;
    if constexpr (POST) {
#pragma unroll
        for (int i = 0; i < NP; ++i) s_pw[i] = s_pb[i] = 0;
    }
    // Adds s over the CTA's thread groups and stores it to out[0 .. D) as fp32 (or bf16); barriers before and after.
    auto flush = [&](const pair_t* s, void* out, bool bf16) {
        auto put = [&](int c, float a) {
            if (bf16) reinterpret_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(a);
            else reinterpret_cast<float*>(out)[c] = a;
        };
        if constexpr (RPC > 1) {
            float* x = reinterpret_cast<float*>(smem);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const int c = channel<VEC, TPR>(e, t);
                if (c < D) x[sub * (NE * TPR) + c] = elem(s, e);
            }
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += THREADS) {
                float a = 0.f;
#pragma unroll
                for (int w = 0; w < RPC; ++w) a += x[w * (NE * TPR) + c];
                put(c, a);
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const int c = channel<VEC, TPR>(e, t);
                if (c < D) put(c, elem(s, e));
            }
        }
    };

    fill<VEC, NE, TPR, RPC>(prm, p.weight, p.param_bf16, 0, 1.f, D, t, sub);
    if constexpr (POST) {
        fill<VEC, NE, TPR, RPC>(prm + kRow, p.post_weight, p.param_bf16, 0, 1.f, D, t, sub);
        fill<VEC, NE, TPR, RPC>(prm + 2 * kRow, p.post_bias, p.param_bf16, 0, 0.f, D, t, sub);
    }
    for (int unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const long long g = unit / p.splits, s = unit % p.splits;
        const long long lo = g * p.group_rows + p.group_rows * s / p.splits, hi = g * p.group_rows + p.group_rows * (s + 1) / p.splits;
        clear_stages();         // the sums of the unit before went through the same memory
        for (int k = 0; k < STAGES - 1; ++k) fetch(lo + sub + (long long)k * RPC, (lo + sub + (long long)k * RPC) * D, hi, k);
        __syncthreads();        // the unit before is past its gate
        if (!p.gate_rows) fill<VEC, NE, TPR, RPC>(prm + 3 * kRow, p.gate, p.gate_bf16, g * D, 1.f, D, t, sub);
        __syncthreads();
        int stage = 0;
        const float4 none = make_float4(0.f, 1.f, 0.f, 1.f);
        float4 st = none, st_next = p.stats && lo + sub < hi ? p.stats[lo + sub] : none;
        const long long ahead = (long long)(STAGES - 1) * RPC * D;
        long long off = (lo + sub) * D;
        for (long long row = lo + sub; row < hi; row += RPC, off += (long long)RPC * D) {
            st = st_next;
            if (p.stats && row + RPC < hi) st_next = p.stats[row + RPC];
            if constexpr (STAGED) stage_wait<STAGED ? STAGES - 2 : 0>();
            pair_t n[NP], x[NP], d[NP];   // n: post(b) before scale and shift; x: norm(r) before scale and shift; d: the running gradient
            take(off, stage, 1, n);
            if constexpr (POST) {
                const pair_t scale = both(st.y), minus = both(-st.x);
#pragma unroll
                for (int i = 0; i < NP; ++i) n[i] = mul2(add2(n[i], minus), scale);
            }
            pair_t gate[NP];
            if (p.gate_rows) {
                auto w = [&](int e) {
                    const int c = channel<VEC, TPR>(e, t);
                    return c < D ? param(p.gate, p.gate_bf16, off + c) : 0.f;
                };
#pragma unroll
                for (int i = 0; i < NP; ++i) gate[i] = mk(w(2 * i), w(2 * i + 1));
            } else {
#pragma unroll
                for (int q = 0; q < NE / 4; ++q) get(3, q, gate + 2 * q);
            }
            // the branch as it enters the sum, before the gate: pairs 2 q, 2 q + 1
            auto branch = [&](int q, pair_t* f) {
                f[0] = n[2 * q];
                f[1] = n[2 * q + 1];
                if constexpr (POST) {
                    pair_t w[2], c[2];
                    get(1, q, w);
                    get(2, q, c);
                    f[0] = fma2(f[0], w[0], c[0]);
                    f[1] = fma2(f[1], w[1], c[1]);
                }
            };
            if (src[2]) {
                take(off, stage, 0, x);
                take(off, stage, 2, d);
                const pair_t scale = both(st.w), minus = both(-st.z);
                pair_t mx = 0, my = 0;
#pragma unroll
                for (int q = 0; q < NE / 4; ++q) {
                    pair_t f[2], w[2];
                    branch(q, f);
                    get(0, q, w);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int i = 2 * q + j;
                        const pair_t r = fma2(both(p.alpha), x[i], mul2(gate[i], f[j]));
                        x[i] = mul2(add2(r, minus), scale);
                        s_w[i] = fma2(d[i], x[i], s_w[i]);
                        s_b[i] = add2(s_b[i], d[i]);
                        d[i] = mul2(d[i], w[j]);
                        mx = add2(mx, d[i]);
                        my = fma2(d[i], x[i], my);
                    }
                }
                const float2 m = row_sum2<TPR>(make_float2(un(mx).x + un(mx).y, un(my).x + un(my).y), slots, turn);
                const pair_t m1 = both(p.norm == BPT_NORM_LAYER ? -m.x * inv_d : 0.f), m2 = both(-m.y * inv_d);
#pragma unroll
                for (int i = 0; i < NP; ++i) d[i] = mul2(scale, add2(d[i], fma2(x[i], m2, m1)));
                if (src[3]) {
                    take(off, stage, 3, x);
#pragma unroll
                    for (int i = 0; i < NP; ++i) d[i] = add2(d[i], x[i]);
                }
            } else {
                take(off, stage, 3, d);
            }
            if (p.dh) {
#pragma unroll
                for (int i = 0; i < NP; ++i) x[i] = mul2(both(p.alpha), d[i]);
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    if (live(v)) pack<T, VEC>(reinterpret_cast<T*>(p.dh) + off + chan(v), x, v);
            }
            pair_t mx = 0, my = 0;
#pragma unroll
            for (int q = 0; q < NE / 4; ++q) {
                pair_t f[2];
                branch(q, f);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int i = 2 * q + j;
                    if (p.gate_rows) x[i] = mul2(d[i], f[j]);
                    else s_g[i] = fma2(d[i], f[j], s_g[i]);
                    d[i] = mul2(d[i], gate[i]);
                }
                if constexpr (POST) {
                    pair_t w[2];
                    get(1, q, w);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int i = 2 * q + j;
                        s_pw[i] = fma2(d[i], n[i], s_pw[i]);
                        s_pb[i] = add2(s_pb[i], d[i]);
                        d[i] = mul2(d[i], w[j]);
                        mx = add2(mx, d[i]);
                        my = fma2(d[i], n[i], my);
                    }
                }
            }
            if (p.gate_rows && p.d_gate) {
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    const int c = channel<VEC, TPR>(e, t);
                    const float a = elem(x, e);
                    if (c >= D) continue;
                    if (p.gate_bf16) reinterpret_cast<__nv_bfloat16*>(p.d_gate)[off + c] = __float2bfloat16_rn(a);
                    else reinterpret_cast<float*>(p.d_gate)[off + c] = a;
                }
            }
            if constexpr (POST) {
                const float2 m = row_sum2<TPR>(make_float2(un(mx).x + un(mx).y, un(my).x + un(my).y), slots, turn);
                const pair_t scale = both(st.y), m1 = both(p.post == BPT_NORM_LAYER ? -m.x * inv_d : 0.f), m2 = both(-m.y * inv_d);
#pragma unroll
                for (int i = 0; i < NP; ++i) d[i] = mul2(scale, add2(d[i], fma2(n[i], m2, m1)));
            }
            if (p.db)
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    if (live(v)) pack<T, VEC>(reinterpret_cast<T*>(p.db) + off + chan(v), d, v);
            fetch(row + (STAGES - 1) * RPC, off + ahead, hi, stage == 0 ? STAGES - 1 : stage - 1);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
        if constexpr (STAGED) stage_wait<0>();
        if (p.d_gate && !p.gate_rows) {
            if (p.splits == 1) flush(s_g, reinterpret_cast<char*>(p.d_gate) + g * D * (p.gate_bf16 ? 2 : 4), p.gate_bf16);
            else flush(s_g, p.gate_part + (long long)unit * D, false);
#pragma unroll
            for (int i = 0; i < NP; ++i) s_g[i] = 0;
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float* part = p.part + (long long)blockIdx.x * 4 * D;
    if (p.norm) {
        flush(s_w, part, false);
        flush(s_b, part + D, false);
    }
    if constexpr (POST) {
        flush(s_pw, part + 2 * D, false);
        flush(s_pb, part + 3 * D, false);
    }
}

// Adds the shares: out[c] = sum over `count` rows of `part`, in a fixed order: 32 interleaved partial sums, then their sum.  A
// block has 32 channels of the output that blockIdx.y picks, a warp for each partial sum.
struct RnFinish {
    const float *part, *gate_part;
    void *d_weight, *d_bias, *d_post_weight, *d_post_bias, *d_gate;
    long long groups;
    int D, grid, splits;
    bool param_bf16, gate_bf16;
};
__global__ void __launch_bounds__(1024) res_norm_finish_kernel(const RnFinish f) {
    __shared__ float x[32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");      // the shares are there
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    for (long long o = blockIdx.y; o < 4 + f.groups; o += gridDim.y) {
        const float* part = o < 4 ? f.part + o * f.D : f.gate_part + (o - 4) * f.splits * f.D;
        void* out = o == 0 ? f.d_weight : o == 1 ? f.d_bias : o == 2 ? f.d_post_weight : o == 3 ? f.d_post_bias : f.d_gate;
        if (!out) continue;
        const int count = o < 4 ? f.grid : f.splits;
        const long long stride = o < 4 ? 4ll * f.D : f.D;
        const bool bf16 = o < 4 ? f.param_bf16 : f.gate_bf16;
        float a = 0.f;
        if (c < f.D)
#pragma unroll 10
            for (int k = w; k < count; k += 32) a += part[k * stride + c];
        x[w][lane] = a;
        __syncthreads();
        // warp w sums channel w of the block
        a = x[lane][w];
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) a += __shfl_xor_sync(0xffffffffu, a, s);
        const int ch = blockIdx.x * 32 + w;
        if (lane == 0 && ch < f.D) {
            const long long at = o < 4 ? ch : (o - 4) * f.D + ch;
            if (bf16) reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(a);
            else reinterpret_cast<float*>(out)[at] = a;
        }
        __syncthreads();
    }
}

// Shares of the backward: `grid` CTAs over `units` = groups x splits row ranges.
struct RnPlan { int grid, splits, units; long long groups, group_rows; bool gate_rows; };
RnPlan plan_bwd(const bpt_res_norm_args& a) {
    RnPlan q{};
    const int rpc = a.D <= 256 ? 8 : a.D <= 512 ? 4 : 1;
    q.gate_rows = a.gate && a.gate_groups == a.rows && a.rows > 1;
    q.groups = a.gate && !q.gate_rows ? a.gate_groups : 1;
    q.group_rows = q.groups ? a.rows / q.groups : 0;
    const long long per_group = (q.group_rows + rpc - 1) / rpc;   // no split smaller than one pass of the CTA's warps
    const long long cap = kRnSms * (a.D <= 512 ? 2 : a.D <= 1024 ? 4 : a.D <= 2048 ? 2 : 1);   // 512 threads of 128 registers per SM, in CTAs of 256, 128, 256 or 512
    q.splits = (int)std::max<long long>(1, std::min<long long>(per_group, cap / std::max<long long>(1, q.groups)));
    q.units = (int)std::min<long long>(q.groups * q.splits, 0x7fffffff);
    q.grid = (int)std::min<long long>(q.units, cap);
    return q;
}

bpt_status check_res_norm(const bpt_res_norm_args* a) {
    if (!a || a->rows < 0 || a->D < 1 || !(a->eps >= 0.f)) return BPT_ERR_INVALID_ARG;
    if (a->dtype != BPT_F32 && a->dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    if (a->param_dtype != BPT_F32 && a->param_dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    if (a->gate_dtype != BPT_F32 && a->gate_dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    if (a->norm < 0 || a->norm > BPT_NORM_RMS || a->post_norm < 0 || a->post_norm > BPT_NORM_RMS) return BPT_ERR_INVALID_ARG;
    if (!a->b && a->rows > 0 && (a->post_norm || a->gate)) return BPT_ERR_INVALID_ARG;   // an empty tensor may have no address
    if ((a->weight || a->bias) && !a->norm) return BPT_ERR_INVALID_ARG;
    if ((a->post_weight || a->post_bias) && !a->post_norm) return BPT_ERR_INVALID_ARG;
    if (a->gate && (a->gate_groups < 1 || a->rows % a->gate_groups)) return BPT_ERR_INVALID_ARG;
    if (a->D > kRnMaxD || a->rows > 0x7fffffffll) return BPT_ERR_UNSUPPORTED;
    return BPT_OK;
}
RnParams make_params(const bpt_res_norm_args& a) {
    RnParams p{};
    p.h = a.h; p.b = a.b;
    p.weight = a.weight; p.bias = a.bias; p.post_weight = a.post_weight; p.post_bias = a.post_bias; p.gate = a.gate;
    p.rows = a.rows; p.D = a.D; p.norm = a.norm; p.post = a.post_norm;
    p.group_rows = a.gate ? std::max<long long>(1, a.rows / a.gate_groups) : std::max<long long>(1, a.rows);
    p.param_bf16 = a.param_dtype == BPT_BF16; p.gate_bf16 = a.gate_dtype == BPT_BF16;
    p.alpha = a.alpha; p.eps = a.eps;
    return p;
}
bool aligned16(std::initializer_list<const void*> ptrs) {
    for (const void* q : ptrs)
        if ((uintptr_t)q & 15) return false;
    return true;
}
bool element_aligned(std::initializer_list<const void*> ptrs, bpt_dtype t) {
    for (const void* q : ptrs)
        if ((uintptr_t)q & (t == BPT_F32 ? 3 : 1)) return false;
    return true;
}

template <typename T, int VEC, int NE, int TPR>
bpt_status run_fwd(const RnParams& p, cudaStream_t st) {
    constexpr int threads = cta_threads(TPR), rpc = threads / TPR;
    constexpr size_t all = (size_t)5 * NE * 4 * TPR;
    const size_t smem = (size_t)((p.norm ? 2 : 0) + (p.post ? 2 : 0) + (p.gate && !p.gate_each ? 1 : 0)) * NE * 4 * TPR;
    if (smem > 32 * 1024 &&     // with the static part, 48 KB is the limit without asking
        cudaFuncSetAttribute(res_norm_fwd_kernel<T, VEC, NE, TPR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)all) != cudaSuccess)
        return BPT_ERR_CUDA;
    // as many CTAs as run at once: each turns the parameters to fp32 once
    const long long grid = std::min<long long>((p.rows + rpc - 1) / rpc, kRnSms * std::max(1, 1024 / threads));
    res_norm_fwd_kernel<T, VEC, NE, TPR><<<(unsigned)grid, threads, smem, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}
template <typename T, int VEC>
bpt_status pick_fwd(const RnParams& p, cudaStream_t st) {
    if (p.D <= 256) return run_fwd<T, VEC, 8, 32>(p, st);
    if (p.D <= 512) return run_fwd<T, VEC, 16, 32>(p, st);
    if (p.D <= 1024) return run_fwd<T, VEC, 32, 32>(p, st);
    if (p.D <= 2048) return run_fwd<T, VEC, 16, 128>(p, st);
    if (p.D <= 4096) return run_fwd<T, VEC, 16, 256>(p, st);
    return run_fwd<T, VEC, 16, 512>(p, st);
}

template <typename T, int VEC, int NE, int TPR, bool POST>
bpt_status run_bwd(const RnParams& p, int grid, cudaStream_t st) {
    constexpr size_t smem = bwd_smem<T, VEC, NE, TPR>();
    if (smem > 32 * 1024 &&   // with the static part, 48 KB is the limit without asking
        cudaFuncSetAttribute(res_norm_bwd_kernel<T, VEC, NE, TPR, POST>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
        return BPT_ERR_CUDA;
    res_norm_bwd_kernel<T, VEC, NE, TPR, POST><<<grid, cta_threads(TPR), smem, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}
template <typename T, int VEC, int NE, int TPR>
bpt_status run_bwd(const RnParams& p, int grid, cudaStream_t st) {
    return p.post ? run_bwd<T, VEC, NE, TPR, true>(p, grid, st) : run_bwd<T, VEC, NE, TPR, false>(p, grid, st);
}
template <typename T, int VEC>
bpt_status pick_bwd(const RnParams& p, int grid, cudaStream_t st) {
    if (p.D <= 256) return run_bwd<T, VEC, 8, 32>(p, grid, st);
    if (p.D <= 512) return run_bwd<T, VEC, 8, 64>(p, grid, st);
    if (p.D <= 1024) return run_bwd<T, VEC, 8, 128>(p, grid, st);
    if (p.D <= 2048) return run_bwd<T, VEC, 8, 256>(p, grid, st);
    if (p.D <= 4096) return run_bwd<T, VEC, 8, 512>(p, grid, st);
    return run_bwd<T, VEC, 16, 512>(p, grid, st);
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" bpt_status bpt_res_norm_fwd(const bpt_res_norm_args* a, void* y, void* r, float* stats, void* cuda_stream) {
    const bpt_status s = check_res_norm(a);
    if (s != BPT_OK) return s;
    if (a->rows == 0) return BPT_OK;
    if ((a->norm != BPT_NORM_NONE) != (y != nullptr) || (!y && !r)) return BPT_ERR_INVALID_ARG;
    if (!a->h) return BPT_ERR_INVALID_ARG;
    if (!aligned16({stats})) return BPT_ERR_INVALID_ARG;
    if (!element_aligned({a->h, a->b, y, r}, a->dtype) || !element_aligned({a->weight, a->bias, a->post_weight, a->post_bias}, a->param_dtype) ||
        !element_aligned({a->gate}, a->gate_dtype))
        return BPT_ERR_INVALID_ARG;
    RnParams p = make_params(*a);
    p.y = y; p.r = r; p.stats_out = reinterpret_cast<float4*>(stats);
    p.gate_each = a->gate && a->gate_groups > 1;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    // 16-byte accesses need whole 16-byte pieces per row; other widths and addresses go element by element
    const bool vec = a->D % (a->dtype == BPT_F32 ? 4 : 8) == 0 && aligned16({a->h, a->b, y, r});
    bpt_status e;
    if (a->dtype == BPT_F32) e = vec ? pick_fwd<float, 4>(p, st) : pick_fwd<float, 1>(p, st);
    else e = vec ? pick_fwd<__nv_bfloat16, 8>(p, st) : pick_fwd<__nv_bfloat16, 1>(p, st);
    trace_mark(st, "res_norm_fwd");
    return e;
}

extern "C" size_t bpt_res_norm_bwd_workspace_bytes(const bpt_res_norm_args* a) {
    if (check_res_norm(a) != BPT_OK) return 0;
    const RnPlan q = plan_bwd(*a);
    return ((size_t)q.grid * 4 + (a->gate && !q.gate_rows && q.splits > 1 ? (size_t)q.units : 0)) * a->D * 4;
}

extern "C" bpt_status bpt_res_norm_bwd(const bpt_res_norm_args* a, const float* stats, const void* dy, const void* dr, void* dh, void* db, void* d_weight,
                                       void* d_bias, void* d_post_weight, void* d_post_bias, void* d_gate, void* workspace,
                                       size_t workspace_bytes, void* cuda_stream) {
    const bpt_status s = check_res_norm(a);
    if (s != BPT_OK) return s;
    if ((dy && !a->norm) || (db && !a->b) || (d_weight && !a->weight) || (d_bias && !a->bias) || (d_post_weight && !a->post_weight) ||
        (d_post_bias && !a->post_bias) || (d_gate && !a->gate))
        return BPT_ERR_INVALID_ARG;
    if (a->rows > 0 && (!a->h || (!stats && (a->norm || a->post_norm)) || !aligned16({stats}))) return BPT_ERR_INVALID_ARG;
    if (!element_aligned({a->h, a->b, dy, dr, dh, db}, a->dtype) ||
        !element_aligned({a->weight, a->bias, a->post_weight, a->post_bias, d_weight, d_bias, d_post_weight, d_post_bias}, a->param_dtype) ||
        !element_aligned({a->gate, d_gate}, a->gate_dtype))
        return BPT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < bpt_res_norm_bwd_workspace_bytes(a)) return BPT_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return BPT_ERR_INVALID_ARG;
    const RnPlan q = plan_bwd(*a);
    RnParams p = make_params(*a);
    p.stats = reinterpret_cast<const float4*>(stats);
    p.dy = dy; p.dr = dr; p.dh = dh; p.db = db; p.d_gate = d_gate;
    p.part = static_cast<float*>(workspace);
    p.gate_part = p.part + (size_t)q.grid * 4 * a->D;
    p.splits = q.splits; p.units = q.units; p.gate_rows = q.gate_rows;
    p.group_rows = q.group_rows;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool vec = a->D % (a->dtype == BPT_F32 ? 4 : 8) == 0 && aligned16({a->h, a->b, dy, dr, dh, db});
    if (a->rows > 0) {
        bpt_status e;
        if (a->dtype == BPT_F32) e = vec ? pick_bwd<float, 4>(p, q.grid, st) : pick_bwd<float, 1>(p, q.grid, st);
        else e = vec ? pick_bwd<__nv_bfloat16, 8>(p, q.grid, st) : pick_bwd<__nv_bfloat16, 1>(p, q.grid, st);
        if (e != BPT_OK) return e;
        trace_mark(st, "res_norm_bwd");
    }
    RnFinish f{};
    f.part = p.part;
    f.d_weight = d_weight; f.d_bias = d_bias; f.d_post_weight = d_post_weight; f.d_post_bias = d_post_bias;
    f.D = a->D; f.grid = a->rows > 0 ? q.grid : 0; f.splits = a->rows > 0 ? q.splits : 0;
    f.param_bf16 = p.param_bf16; f.gate_bf16 = p.gate_bf16;
    // one split per group: the rows of d_gate are complete already (with no rows at all they are zeros)
    const bool gate_sums = d_gate && !q.gate_rows && (q.splits > 1 || a->rows == 0);
    f.gate_part = p.gate_part; f.d_gate = gate_sums ? d_gate : nullptr; f.groups = gate_sums ? q.groups : 0;
    if (d_weight || d_bias || d_post_weight || d_post_bias || gate_sums) {
        const dim3 grid((a->D + 31) / 32, (unsigned)std::min<long long>(4 + f.groups, 65535));
        cudaLaunchAttribute attr[1] = {};       // launched while the shares are still being summed, where there is room
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = grid;
        cfg.blockDim = dim3(1024);
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = a->rows > 0 ? 1 : 0;
        if (cudaLaunchKernelEx(&cfg, res_norm_finish_kernel, f) != cudaSuccess) {
            cudaGetLastError();     // reported by this status, not by the next call of somebody else
            return BPT_ERR_CUDA;
        }
        trace_mark(st, "res_norm_finish");
    }
    return BPT_OK;
}
