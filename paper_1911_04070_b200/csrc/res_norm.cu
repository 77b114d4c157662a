// The seam between two blocks of a layer (arXiv 1911.04070, Algorithm 2 of Sec. 3.3 has Z = norm(H + GSA(H)) and
// H' = norm(Z + FFN(Z)); this is that step with the scaled residual, gate and second norm that deeper stacks use):
//     n = post(b),   r = alpha h + gate n,   y = norm(r),        row by row over D channels,
// post and norm each absent, layer normalisation or root-mean-square normalisation, and its backward.
//
// Both directions are bound by HBM: a row is read once, lives in registers as fp32 (statistics about the mean in a
// second sweep over the registers), and every result is rounded once to the tensors' type when it is stored.  The
// backward recomputes n, r and the statistics from h and b instead of reading saved ones.
//
// A row belongs to TPR threads, NE channels each: one warp up to 512 (backward) / 1024 (forward) channels, so that
// the row sums are shuffles, a whole CTA above.  The backward's CTAs each take a fixed, contiguous share of the rows
// and keep the column sums of the parameter gradients in registers; the shares are added by a second kernel in a
// fixed order, so results are bit-reproducible.  Backward rows are fetched two rows ahead into shared memory by
// asynchronous copies; every thread reads back only what it copied itself, so no barrier is needed for them.
#include <algorithm>

#include "bpt_internal.cuh"
#include "mma_tools.cuh"

namespace bpt {
namespace {

constexpr int kRnSms = 148;
constexpr int kRnMaxD = 8192;
// Rows of a thread group in flight (the current one and those ahead), as far as shared memory goes; below two there is no staging.
template <typename T, int VEC, int NE, int TPR>
__host__ __device__ constexpr int bwd_stages() {
    constexpr size_t one = 4 * NE * sizeof(T) * (TPR == 32 ? 256 : TPR);
    return sizeof(T) * VEC < 4 || 2 * one > 200 * 1024 ? 1 : 3 * one > 200 * 1024 ? 2 : 3;
}

struct RnParams {
    const void *h, *b, *dy, *dr;
    const void *weight, *bias, *post_weight, *post_bias, *gate;
    void *y, *r, *dh, *db, *d_gate;
    float *part;            // [grid][4][D]: weight, bias, post weight, post bias
    float *gate_part;       // [units][D]
    long long rows, group_rows;
    int D, norm, post, splits, units;
    bool param_bf16, gate_bf16, gate_rows;   // gate_rows: a gate row per row
    float alpha, eps;
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// VEC consecutive elements of type T <-> fp32
template <typename T, int VEC>
__device__ __forceinline__ void unpack(const void* p, float* f) {
    if constexpr (VEC == 1) {
        f[0] = to_f(*reinterpret_cast<const T*>(p));
    } else if constexpr (sizeof(T) == 4) {
        static_assert(VEC == 4, "16 bytes");
        const float4 v = *reinterpret_cast<const float4*>(p);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
        static_assert(VEC == 8, "16 bytes");
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void pack(void* p, const float* f) {
    if constexpr (VEC == 1) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float*>(p) = f[0];
        else *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(f[0]);
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
}
// VEC parameters from channel c on (their type is a run-time choice of the whole grid)
template <int VEC>
__device__ __forceinline__ void load_param(const void* p, bool bf16, long long c, float* f) {
    if constexpr (VEC == 1) {
        // plain loads: __ldg of a bf16 is inline assembly that the compiler may move above the caller's test for a null pointer
        if (bf16) f[0] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[c]);
        else f[0] = reinterpret_cast<const float*>(p)[c];
    } else if (bf16) {
        if constexpr (VEC == 8) {
            unpack<__nv_bfloat16, 8>(reinterpret_cast<const __nv_bfloat16*>(p) + c, f);
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(p) + c);
            f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
            f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) unpack<float, 4>(reinterpret_cast<const float*>(p) + c + 4 * i, f + 4 * i);
    }
}

// Sum of a pair over the TPR threads of a row, the same bits in every thread.  slots: two buffers of TPR / 32 pairs,
// used in turn, so that one barrier per sum is enough.
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float2 v, float2* slots, int& turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if constexpr (TPR > 32) {
        float2* s = slots + turn * (TPR / 32);
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w) { v.x += s[w].x; v.y += s[w].y; }
    }
    return v;
}

// Mean (0 for rms) and reciprocal deviation of the row held in x; channels past D hold zeros and are left out by `live`.
template <int TPR, int NE, int VEC, typename Live>
__device__ __forceinline__ float2 row_stats(const float (&x)[NE], int kind, int D, float eps, Live live, float2* slots, int& turn) {
    float mean = 0.f;
    if (kind == BPT_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NE; ++i) s += x[i];
        mean = row_sum2<TPR>(make_float2(s, 0.f), slots, turn).x / (float)D;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const float c = live(i / VEC) ? x[i] - mean : 0.f;
        q = fmaf(c, c, q);
    }
    q = row_sum2<TPR>(make_float2(q, 0.f), slots, turn).x;
    return make_float2(mean, rsqrtf(q / (float)D + eps));
}

template <typename T, int VEC, int NE, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) res_norm_fwd_kernel(const RnParams p) {
    constexpr int NV = NE / VEC, RPC = TPR == 32 ? 8 : 1;
    __shared__ float2 slots[TPR > 32 ? 2 * (TPR / 32) : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const int D = p.D;
    auto chan = [&](int v) { return (v * TPR + t) * VEC; };
    auto live = [&](int v) { return chan(v) < D; };
    for (long long row = (long long)blockIdx.x * RPC + threadIdx.x / TPR; row < p.rows; row += (long long)gridDim.x * RPC) {
        const long long off = row * D;
        float n[NE], r[NE];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) n[v * VEC + i] = r[v * VEC + i] = 0.f;
            if (live(v)) {
                unpack<T, VEC>(reinterpret_cast<const T*>(p.h) + off + chan(v), &r[v * VEC]);
                if (p.b) unpack<T, VEC>(reinterpret_cast<const T*>(p.b) + off + chan(v), &n[v * VEC]);
            }
        }
        if (p.post) {
            const float2 st = row_stats<TPR, NE, VEC>(n, p.post, D, p.eps, live, slots, turn);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!live(v)) continue;
                float w[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) n[v * VEC + i] = (n[v * VEC + i] - st.x) * st.y;
                if (p.post_weight) {
                    load_param<VEC>(p.post_weight, p.param_bf16, chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) n[v * VEC + i] *= w[i];
                }
                if (p.post_bias) {
                    load_param<VEC>(p.post_bias, p.param_bf16, chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) n[v * VEC + i] += w[i];
                }
            }
        }
        const long long goff = p.gate ? (row / p.group_rows) * D : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (!live(v)) continue;
            if (p.gate) {
                float w[VEC];
                load_param<VEC>(p.gate, p.gate_bf16, goff + chan(v), w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) n[v * VEC + i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) r[v * VEC + i] = fmaf(p.alpha, r[v * VEC + i], n[v * VEC + i]);
            if (p.r) pack<T, VEC>(reinterpret_cast<T*>(p.r) + off + chan(v), &r[v * VEC]);
        }
        if (p.norm) {
            const float2 st = row_stats<TPR, NE, VEC>(r, p.norm, D, p.eps, live, slots, turn);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!live(v)) continue;
                float w[VEC], y[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) y[i] = (r[v * VEC + i] - st.x) * st.y;
                if (p.weight) {
                    load_param<VEC>(p.weight, p.param_bf16, chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) y[i] *= w[i];
                }
                if (p.bias) {
                    load_param<VEC>(p.bias, p.param_bf16, chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) y[i] += w[i];
                }
                pack<T, VEC>(reinterpret_cast<T*>(p.y) + off + chan(v), y);
            }
        }
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

// Bytes of shared memory of the backward: the staged pieces, or the exchange of the column sums at the end
template <typename T, int VEC, int NE, int TPR>
__host__ __device__ constexpr size_t bwd_smem() {
    constexpr int threads = TPR == 32 ? 256 : TPR;
    constexpr int stages = bwd_stages<T, VEC, NE, TPR>();
    const size_t stage = stages > 1 ? (size_t)stages * 4 * NE * sizeof(T) * threads : 0;
    const size_t xch = TPR == 32 ? (size_t)8 * NE * 32 * 4 : 0;
    return stage > xch ? stage : xch;
}

template <typename T, int VEC, int NE, int TPR, bool POST>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR) res_norm_bwd_kernel(const RnParams p) {
    constexpr int NV = NE / VEC, THREADS = TPR == 32 ? 256 : TPR, RPC = THREADS / TPR;
    constexpr int PIECE = VEC * (int)sizeof(T);
    constexpr int STAGES = bwd_stages<T, VEC, NE, TPR>();
    constexpr bool STAGED = STAGES > 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float2 slots[TPR > 32 ? 2 * (TPR / 32) : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int D = p.D;
    const float inv_d = 1.f / (float)D;
    auto chan = [&](int v) { return (v * TPR + t) * VEC; };
    auto live = [&](int v) { return chan(v) < D; };
    const uint32_t mine = smem_u32(smem) + threadIdx.x * PIECE;
    const void* src[4] = {p.h, p.b, p.dy, p.dr};
    auto slot = [&](int stage, int a, int v) { return (uint32_t)(((stage * 4 + a) * NV + v) * THREADS * PIECE); };
    auto fetch = [&](long long row, long long end, int stage) {
        if constexpr (STAGED) {
            if (row < end) {
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    if (src[a])
#pragma unroll
                        for (int v = 0; v < NV; ++v)
                            if (live(v)) stage_copy<PIECE>(mine + slot(stage, a, v), reinterpret_cast<const T*>(src[a]) + row * D + chan(v));
            }
            cp_async_commit();
        }
    };
    auto take = [&](long long row, int stage, int a, int v, float* f) {
        if constexpr (STAGED) unpack<T, VEC>(smem + threadIdx.x * PIECE + slot(stage, a, v), f);
        else unpack<T, VEC>(reinterpret_cast<const T*>(src[a]) + row * D + chan(v), f);
    };

    float s_w[NE], s_b[NE], s_g[NE], s_pw[POST ? NE : 1], s_pb[POST ? NE : 1];   // this thread's column sums
#pragma unroll
    for (int i = 0; i < NE; ++i) s_w[i] = s_b[i] = s_g[i] = 0.f;
    if constexpr (POST) {
#pragma unroll
        for (int i = 0; i < NE; ++i) s_pw[i] = s_pb[i] = 0.f;
    }
    // Adds s over the CTA's thread groups and stores it to out[0 .. D) as fp32 (or bf16): ends with every thread past its reads.
    auto flush = [&](const float* s, void* out, bool bf16) {
        if constexpr (RPC > 1) {
            float* x = reinterpret_cast<float*>(smem);
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (live(v)) x[sub * (NE * 32) + chan(v) + i] = s[v * VEC + i];
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += THREADS) {
                float a = 0.f;
#pragma unroll
                for (int w = 0; w < RPC; ++w) a += x[w * (NE * 32) + c];
                if (bf16) reinterpret_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(a);
                else reinterpret_cast<float*>(out)[c] = a;
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (live(v)) {
                        if (bf16) reinterpret_cast<__nv_bfloat16*>(out)[chan(v) + i] = __float2bfloat16_rn(s[v * VEC + i]);
                        else reinterpret_cast<float*>(out)[chan(v) + i] = s[v * VEC + i];
                    }
        }
    };

    for (int unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
        const long long g = unit / p.splits, s = unit % p.splits;
        const long long lo = g * p.group_rows + p.group_rows * s / p.splits, hi = g * p.group_rows + p.group_rows * (s + 1) / p.splits;
        for (int k = 0; k < STAGES - 1; ++k) fetch(lo + sub + (long long)k * RPC, hi, k);
        int stage = 0;
        for (long long row = lo + sub; row < hi; row += RPC) {
            if constexpr (STAGED) stage_wait<STAGED ? STAGES - 2 : 0>();
            const long long off = row * D, goff = p.gate_rows ? off : g * D;
            float n[NE], x[NE], d[NE];   // n: post(b) before scale and shift; x: r, then norm(r) before scale and shift; d: the running gradient
            float2 st1 = make_float2(0.f, 1.f), st2 = make_float2(0.f, 1.f);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) n[v * VEC + i] = x[v * VEC + i] = d[v * VEC + i] = 0.f;
                if (live(v)) {
                    take(row, stage, 0, v, &x[v * VEC]);
                    if (p.b) take(row, stage, 1, v, &n[v * VEC]);
                }
            }
            if constexpr (POST) {
                st1 = row_stats<TPR, NE, VEC>(n, p.post, D, p.eps, live, slots, turn);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) n[v * VEC + i] = live(v) ? (n[v * VEC + i] - st1.x) * st1.y : 0.f;
            }
            // the branch as it enters the sum, before the gate
            auto branch = [&](int v, float* f) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[i] = n[v * VEC + i];
                if constexpr (POST) {
                    float w[VEC];
                    if (p.post_weight) {
                        load_param<VEC>(p.post_weight, p.param_bf16, chan(v), w);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) f[i] *= w[i];
                    }
                    if (p.post_bias) {
                        load_param<VEC>(p.post_bias, p.param_bf16, chan(v), w);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) f[i] += w[i];
                    }
                }
            };
            if (p.norm && p.dy) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if (!live(v)) continue;
                    float f[VEC];
                    branch(v, f);
                    if (p.gate) {
                        float w[VEC];
                        load_param<VEC>(p.gate, p.gate_bf16, goff + chan(v), w);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) f[i] *= w[i];
                    }
#pragma unroll
                    for (int i = 0; i < VEC; ++i) x[v * VEC + i] = fmaf(p.alpha, x[v * VEC + i], f[i]);
                }
                st2 = row_stats<TPR, NE, VEC>(x, p.norm, D, p.eps, live, slots, turn);
                float2 m = make_float2(0.f, 0.f);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if (!live(v)) continue;
                    float dy[VEC], w[VEC];
                    take(row, stage, 2, v, dy);
                    if (p.weight) load_param<VEC>(p.weight, p.param_bf16, chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const int e = v * VEC + i;
                        x[e] = (x[e] - st2.x) * st2.y;
                        s_w[e] = fmaf(dy[i], x[e], s_w[e]);
                        s_b[e] += dy[i];
                        d[e] = p.weight ? dy[i] * w[i] : dy[i];
                        m.x += d[e];
                        m.y = fmaf(d[e], x[e], m.y);
                    }
                }
                m = row_sum2<TPR>(m, slots, turn);
                const float m1 = p.norm == BPT_NORM_LAYER ? m.x * inv_d : 0.f, m2 = m.y * inv_d;
#pragma unroll
                for (int i = 0; i < NE; ++i) d[i] = st2.y * (d[i] - m1 - x[i] * m2);
            }
            float2 m = make_float2(0.f, 0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!live(v)) continue;
                float w[VEC];
                if (p.dr) {
                    take(row, stage, 3, v, w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[v * VEC + i] += w[i];
                }
                if (p.dh) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) w[i] = p.alpha * d[v * VEC + i];
                    pack<T, VEC>(reinterpret_cast<T*>(p.dh) + off + chan(v), w);
                }
                if (p.gate) {
                    float f[VEC];
                    branch(v, f);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) f[i] *= d[v * VEC + i];
                    if (p.gate_rows) {
                        if (p.d_gate) {
                            if (p.gate_bf16)
#pragma unroll
                                for (int i = 0; i < VEC; ++i) reinterpret_cast<__nv_bfloat16*>(p.d_gate)[off + chan(v) + i] = __float2bfloat16_rn(f[i]);
                            else
#pragma unroll
                                for (int i = 0; i < VEC; ++i) reinterpret_cast<float*>(p.d_gate)[off + chan(v) + i] = f[i];
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < VEC; ++i) s_g[v * VEC + i] += f[i];
                    }
                    load_param<VEC>(p.gate, p.gate_bf16, goff + chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[v * VEC + i] *= w[i];
                }
                if constexpr (POST) {
                    if (p.post_weight) load_param<VEC>(p.post_weight, p.param_bf16, chan(v), w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const int e = v * VEC + i;
                        s_pw[e] = fmaf(d[e], n[e], s_pw[e]);
                        s_pb[e] += d[e];
                        if (p.post_weight) d[e] *= w[i];
                        m.x += d[e];
                        m.y = fmaf(d[e], n[e], m.y);
                    }
                } else if (p.db) {
                    pack<T, VEC>(reinterpret_cast<T*>(p.db) + off + chan(v), &d[v * VEC]);
                }
            }
            if constexpr (POST) {
                m = row_sum2<TPR>(m, slots, turn);
                const float m1 = p.post == BPT_NORM_LAYER ? m.x * inv_d : 0.f, m2 = m.y * inv_d;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if (!live(v) || !p.db) continue;
                    float w[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) w[i] = st1.y * (d[v * VEC + i] - m1 - n[v * VEC + i] * m2);
                    pack<T, VEC>(reinterpret_cast<T*>(p.db) + off + chan(v), w);
                }
            }
            fetch(row + (long long)(STAGES - 1) * RPC, hi, (stage + STAGES - 1) % STAGES);
            stage = (stage + 1) % STAGES;
        }
        if constexpr (STAGED) stage_wait<0>();
        if (p.d_gate && !p.gate_rows) {
            if (p.splits == 1) flush(s_g, reinterpret_cast<char*>(p.d_gate) + g * D * (p.gate_bf16 ? 2 : 4), p.gate_bf16);
            else flush(s_g, p.gate_part + (long long)unit * D, false);
#pragma unroll
            for (int i = 0; i < NE; ++i) s_g[i] = 0.f;
        }
    }
    float* part = p.part + (long long)blockIdx.x * 4 * D;
    flush(s_w, part, false);
    flush(s_b, part + D, false);
    if constexpr (POST) {
        flush(s_pw, part + 2 * D, false);
        flush(s_pb, part + 3 * D, false);
    }
}

// Adds the shares: out[c] = sum over `count` rows of `part`, in the order of the rows: eight interleaved partial sums, then
// their sum.  Blocks cover 32 channels; blockIdx.y picks the output.
struct RnFinish {
    const float *part, *gate_part;
    void *d_weight, *d_bias, *d_post_weight, *d_post_bias, *d_gate;
    long long groups;
    int D, grid, splits;
    bool param_bf16, gate_bf16;
};
__global__ void __launch_bounds__(256) res_norm_finish_kernel(const RnFinish f) {
    __shared__ float x[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    for (long long o = blockIdx.y; o < 4 + f.groups; o += gridDim.y) {
        const float* part = o < 4 ? f.part + o * f.D : f.gate_part + (o - 4) * f.splits * f.D;
        void* out = o == 0 ? f.d_weight : o == 1 ? f.d_bias : o == 2 ? f.d_post_weight : o == 3 ? f.d_post_bias : f.d_gate;
        if (!out) continue;
        const int count = o < 4 ? f.grid : f.splits;
        const long long stride = o < 4 ? 4ll * f.D : f.D;
        const bool bf16 = o < 4 ? f.param_bf16 : f.gate_bf16;
        const long long at = o < 4 ? c : (o - 4) * f.D + c;
        float a = 0.f;
        if (c < f.D)
#pragma unroll 4
            for (int k = w; k < count; k += 8) a += part[k * stride + c];
        x[w][threadIdx.x & 31] = a;
        __syncthreads();
        if (w == 0 && c < f.D) {
#pragma unroll
            for (int k = 1; k < 8; ++k) a += x[k][threadIdx.x];
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
    const int rpc = a.D <= 512 ? 8 : 1;
    q.gate_rows = a.gate && a.gate_groups == a.rows && a.rows > 1;
    q.groups = a.gate && !q.gate_rows ? a.gate_groups : 1;
    q.group_rows = q.groups ? a.rows / q.groups : 0;
    const long long per_group = (q.group_rows + rpc - 1) / rpc;   // no split smaller than one pass of the CTA's warps
    const long long cap = kRnSms * (a.D <= 256 ? 2 : a.D <= 512 ? 1 : a.D <= 1024 ? 4 : a.D <= 2048 ? 2 : 1);   // CTAs that fit by registers
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
    constexpr int rpc = TPR == 32 ? 8 : 1;
    const long long grid = std::min<long long>((p.rows + rpc - 1) / rpc, kRnSms * 16);
    res_norm_fwd_kernel<T, VEC, NE, TPR><<<(unsigned)grid, TPR == 32 ? 256 : TPR, 0, st>>>(p);
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
    res_norm_bwd_kernel<T, VEC, NE, TPR, POST><<<grid, TPR == 32 ? 256 : TPR, smem, st>>>(p);
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}
template <typename T, int VEC, int NE, int TPR>
bpt_status run_bwd(const RnParams& p, int grid, cudaStream_t st) {
    return p.post ? run_bwd<T, VEC, NE, TPR, true>(p, grid, st) : run_bwd<T, VEC, NE, TPR, false>(p, grid, st);
}
template <typename T, int VEC>
bpt_status pick_bwd(const RnParams& p, int grid, cudaStream_t st) {
    if (p.D <= 256) return run_bwd<T, VEC, 8, 32>(p, grid, st);
    if (p.D <= 512) return run_bwd<T, VEC, 16, 32>(p, grid, st);
    if (p.D <= 1024) return run_bwd<T, VEC, 8, 128>(p, grid, st);
    if (p.D <= 2048) return run_bwd<T, VEC, 8, 256>(p, grid, st);
    if (p.D <= 4096) return run_bwd<T, VEC, 8, 512>(p, grid, st);
    return run_bwd<T, VEC, 16, 512>(p, grid, st);
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" bpt_status bpt_res_norm_fwd(const bpt_res_norm_args* a, void* y, void* r, void* cuda_stream) {
    const bpt_status s = check_res_norm(a);
    if (s != BPT_OK) return s;
    if (a->rows == 0) return BPT_OK;
    if ((a->norm != BPT_NORM_NONE) != (y != nullptr) || (!y && !r)) return BPT_ERR_INVALID_ARG;
    if (!a->h) return BPT_ERR_INVALID_ARG;
    if (!element_aligned({a->h, a->b, y, r}, a->dtype) || !element_aligned({a->weight, a->bias, a->post_weight, a->post_bias}, a->param_dtype) ||
        !element_aligned({a->gate}, a->gate_dtype))
        return BPT_ERR_INVALID_ARG;
    RnParams p = make_params(*a);
    p.y = y; p.r = r;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    // 16-byte accesses need whole 16-byte pieces per row; other widths and addresses go element by element
    const bool vec = a->D % (a->dtype == BPT_F32 ? 4 : 8) == 0 &&
                     aligned16({a->h, a->b, y, r, a->weight, a->bias, a->post_weight, a->post_bias, a->gate});
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

extern "C" bpt_status bpt_res_norm_bwd(const bpt_res_norm_args* a, const void* dy, const void* dr, void* dh, void* db, void* d_weight,
                                       void* d_bias, void* d_post_weight, void* d_post_bias, void* d_gate, void* workspace,
                                       size_t workspace_bytes, void* cuda_stream) {
    const bpt_status s = check_res_norm(a);
    if (s != BPT_OK) return s;
    if ((dy && !a->norm) || (db && !a->b) || (d_weight && !a->weight) || (d_bias && !a->bias) || (d_post_weight && !a->post_weight) ||
        (d_post_bias && !a->post_bias) || (d_gate && !a->gate))
        return BPT_ERR_INVALID_ARG;
    if (a->rows > 0 && !a->h) return BPT_ERR_INVALID_ARG;
    if (!element_aligned({a->h, a->b, dy, dr, dh, db}, a->dtype) ||
        !element_aligned({a->weight, a->bias, a->post_weight, a->post_bias, d_weight, d_bias, d_post_weight, d_post_bias}, a->param_dtype) ||
        !element_aligned({a->gate, d_gate}, a->gate_dtype))
        return BPT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < bpt_res_norm_bwd_workspace_bytes(a)) return BPT_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return BPT_ERR_INVALID_ARG;
    const RnPlan q = plan_bwd(*a);
    RnParams p = make_params(*a);
    p.dy = dy; p.dr = dr; p.dh = dh; p.db = db; p.d_gate = d_gate;
    p.part = static_cast<float*>(workspace);
    p.gate_part = p.part + (size_t)q.grid * 4 * a->D;
    p.splits = q.splits; p.units = q.units; p.gate_rows = q.gate_rows;
    p.group_rows = q.group_rows;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool vec = a->D % (a->dtype == BPT_F32 ? 4 : 8) == 0 &&
                     aligned16({a->h, a->b, dy, dr, dh, db, a->weight, a->bias, a->post_weight, a->post_bias, a->gate});
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
        res_norm_finish_kernel<<<grid, 256, 0, st>>>(f);
        trace_mark(st, "res_norm_finish");
    }
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}
