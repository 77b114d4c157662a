// Gated feed-forward block for a few rows -- decoding: one token and its ancestors in the partition tree (Sec. 3.2.1 of
// arXiv 1911.04070), times the sequences that step together:  h = act(x Wg^T) * (x Wu^T),  y = h Wd^T.
//
// With so few rows the block is a pass over the weights, and its time is latency: what counts is that all SMs have their
// share of the weights in flight at once, and the two launches.  So the weights are the M operand of mma.sync m16n8k16 (16
// weight rows, 8 tokens), loaded straight from memory into fragments, 16 bytes a lane: a fragment's k indices may be any
// 16 columns as long as both operands take the same ones, so lane t of a row takes columns 8 t .. 8 t + 7 of a 32-column
// chunk, half of them for each of two products.  No shared memory, no barrier stands between memory and the tensor cores.
//   kernel 1: a CTA has 16 rows of Wg and of Wu, its eight warps share out the columns, their sums meet in shared memory, where
//             the activation and the product follow; h is stored as two bf16 terms, h = hi + lo, so that it is not rounded to
//             bf16 at all (16 bits are left) and kernel 2 has its operand ready.
//   kernel 2: a cluster of CTAs has 16 rows of Wd and shares out its F columns, the sums of its CTAs meet through distributed
//             shared memory in rank order.  It is launched early (programmatic dependent launch) and has its first weights in
//             registers when kernel 1 ends.
// Sums run in a fixed order: bit-reproducible.
#include <algorithm>

#include "bpt_internal.cuh"
#include "ff_act.cuh"
#include "gated_ff_rows.cuh"
#include "mma_tools.cuh"

namespace bpt {
namespace {

constexpr int kFrWarps = 8;
constexpr int kFrThreads = kFrWarps * 32;

__device__ __forceinline__ uint4 ld16(const void* p, bool live) { return live ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0); }
// Weights and inputs do not change while a kernel runs: read-only loads, kept out of the first-level cache where they are used once.
__device__ __forceinline__ uint4 ld16_once(const void* p, bool live) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (live) asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// 32 columns: the low halves of every lane's eight, then the high halves
__device__ __forceinline__ void mma32(float (&c)[4], const uint4& lo_row, const uint4& hi_row, const uint4& b) {
    const uint32_t a0[4] = {lo_row.x, hi_row.x, lo_row.y, hi_row.y}, a1[4] = {lo_row.z, hi_row.z, lo_row.w, hi_row.w};
    mma_bf16(c, a0, b.x, b.y);
    mma_bf16(c, a1, b.z, b.w);
}

template <int ACT, int NT>
__global__ void __launch_bounds__(kFrThreads, 2) gated_ff_rows_in_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ wg,
                                                                      const __nv_bfloat16* __restrict__ wu, __nv_bfloat16* __restrict__ h,
                                                                      int* __restrict__ status, int rows, int D, int F) {
    extern __shared__ float red[];      // [warp][gate, up][NT * 128]
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) status[threadIdx.x] = 0;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int f0 = blockIdx.x * 16, r0 = blockIdx.y * (8 * NT);
    const bool lo = f0 + g < F, hi = f0 + g + 8 < F;
    const size_t at_lo = (size_t)(f0 + g) * D + 8 * t, at_hi = at_lo + (size_t)8 * D, at_x = (size_t)(r0 + g) * D + 8 * t;
    float cg[NT][4], cu[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) cg[n][i] = cu[n][i] = 0.f;
    const int chunks = (D + 31) / 32;
#pragma unroll 2
    for (int c = w; c < chunks; c += kFrWarps) {
        const bool in = c * 32 + 8 * t < D;
        const uint4 g0 = ld16_once(wg + at_lo + c * 32, in && lo), g1 = ld16_once(wg + at_hi + c * 32, in && hi);
        const uint4 u0 = ld16_once(wu + at_lo + c * 32, in && lo), u1 = ld16_once(wu + at_hi + c * 32, in && hi);
        uint4 b[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) b[n] = ld16(x + at_x + (size_t)n * 8 * D + c * 32, in && r0 + n * 8 + g < rows);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            mma32(cg[n], g0, g1, b[n]);
            mma32(cu[n], u0, u1, b[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        *reinterpret_cast<float4*>(red + ((w * 2 + 0) * NT + n) * 128 + lane * 4) = make_float4(cg[n][0], cg[n][1], cg[n][2], cg[n][3]);
        *reinterpret_cast<float4*>(red + ((w * 2 + 1) * NT + n) * 128 + lane * 4) = make_float4(cu[n][0], cu[n][1], cu[n][2], cu[n][3]);
    }
    __syncthreads();
    for (int s = threadIdx.x; s < NT * 128; s += kFrThreads) {
        float gv = 0.f, uv = 0.f, unused;
#pragma unroll
        for (int k = 0; k < kFrWarps; ++k) {
            gv += red[(k * 2 + 0) * NT * 128 + s];
            uv += red[(k * 2 + 1) * NT * 128 + s];
        }
        const int l = (s & 127) >> 2, f = f0 + (l >> 2) + (s & 2) * 4, row = r0 + (s >> 7) * 8 + (l & 3) * 2 + (s & 1);
        if (f < F && row < rows) {
            const float v = ff_act<ACT, false>(gv, unused) * uv;
            const __nv_bfloat16 t = __float2bfloat16_rn(v);
            const float r = __bfloat162float(t);
            h[(size_t)row * F + f] = t;
            h[(size_t)(rows + row) * F + f] = __float2bfloat16_rn(isinf(r) ? 0.f : v - r);      // an infinite value has no second term
        }
    }
}

template <int NT>
__global__ void __launch_bounds__(kFrThreads, 2) gated_ff_rows_out_kernel(const __nv_bfloat16* h, const __nv_bfloat16* __restrict__ wd,
                                                                       __nv_bfloat16* y, int rows, int D, int F, int parts) {
    extern __shared__ float red[];      // [warp][NT * 128], then this CTA's sums [NT * 128]
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int part = blockIdx.x % parts, d0 = blockIdx.x / parts * 16, r0 = blockIdx.y * (8 * NT);
    const bool lo = d0 + g < D, hi = d0 + g + 8 < D;
    const size_t at_lo = (size_t)(d0 + g) * F + 8 * t, at_hi = at_lo + (size_t)8 * F, at_h = (size_t)(r0 + g) * F + 8 * t;
    const size_t second = (size_t)rows * F;
    const int chunks = (F + 31) / 32, step = kFrWarps * parts, c_first = part * kFrWarps + w;
    auto weights = [&](int c, uint4& a, uint4& b) {
        const bool in = c < chunks && c * 32 + 8 * t < F;
        a = ld16_once(wd + at_lo + (size_t)c * 32, in && lo);
        b = ld16_once(wd + at_hi + (size_t)c * 32, in && hi);
    };
    uint4 a0[2], a1[2];                 // two chunks ahead
#pragma unroll
    for (int i = 0; i < 2; ++i) weights(c_first + i * step, a0[i], a1[i]);
    asm volatile("griddepcontrol.wait;" ::: "memory");      // kernel 1 has ended and its h is visible (h is not __restrict__: no load of it may move up)
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
    for (int c = c_first; c < chunks; c += 2 * step) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int cc = c + i * step;
            const bool in = cc < chunks && cc * 32 + 8 * t < F;
            const uint4 w0 = a0[i], w1 = a1[i];
            weights(cc + 2 * step, a0[i], a1[i]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const bool live = in && r0 + n * 8 + g < rows;
                const __nv_bfloat16* src = h + at_h + (size_t)n * 8 * F + (size_t)cc * 32;
                const uint4 bh = ld16(src, live), bl = ld16(src + second, live);
                mma32(acc[n], w0, w1, bh);
                mma32(acc[n], w0, w1, bl);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
        *reinterpret_cast<float4*>(red + (w * NT + n) * 128 + lane * 4) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
    __syncthreads();
    float* sums = red + kFrWarps * NT * 128;
    for (int s = threadIdx.x; s < NT * 128; s += kFrThreads) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kFrWarps; ++k) v += red[k * NT * 128 + s];
        sums[s] = v;
    }
    if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
    // the cluster's CTAs share out the results
    const uint32_t sums_u = smem_u32(sums);
    for (int s = part * kFrThreads + threadIdx.x; s < NT * 128; s += parts * kFrThreads) {
        float v = 0.f;
        if (parts == 1) {
            v = sums[s];
        } else {
            for (int k = 0; k < parts; ++k) {
                uint32_t at;
                float q;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(sums_u + 4u * s), "r"(k));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(q) : "r"(at) : "memory");
                v += q;
            }
        }
        const int l = (s & 127) >> 2, d = d0 + (l >> 2) + (s & 2) * 4, row = r0 + (s >> 7) * 8 + (l & 3) * 2 + (s & 1);
        if (d < D && row < rows) y[(size_t)row * D + d] = __float2bfloat16_rn(v);
    }
    if (parts > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");   // nobody reads an ended CTA's memory
}

template <int ACT, int NT>
bpt_status run_in(const GatedFfRows& p, cudaStream_t st) {
    constexpr size_t smem = (size_t)kFrWarps * 2 * NT * 128 * 4;
    if (smem > 48 * 1024 &&
        cudaFuncSetAttribute(gated_ff_rows_in_kernel<ACT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
        return BPT_ERR_CUDA;
    const dim3 grid((p.F + 15) / 16, (p.rows + 8 * NT - 1) / (8 * NT));
    gated_ff_rows_in_kernel<ACT, NT><<<grid, kFrThreads, smem, st>>>(p.x, p.w_gate, p.w_up, p.h, p.status, p.rows, p.D, p.F);
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}
template <int NT>
bpt_status run_out(const GatedFfRows& p, cudaStream_t st) {
    constexpr size_t smem = (size_t)(kFrWarps + 1) * NT * 128 * 4;
    const int tiles = (p.D + 15) / 16, row_groups = (p.rows + 8 * NT - 1) / (8 * NT);
    // CTAs per cluster: as many as there are SMs for, with at least a chunk of 32 columns for every warp
    int parts = 1;
    while (parts < 8 && tiles * row_groups * parts * 2 <= 148 && (p.F + 31) / 32 >= kFrWarps * parts * 2) parts *= 2;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = parts; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * parts, row_groups);
    cfg.blockDim = dim3(kFrThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, gated_ff_rows_out_kernel<NT>, (const __nv_bfloat16*)p.h, p.w_down, p.y, p.rows, p.D, p.F, parts) == cudaSuccess) return BPT_OK;
    cudaGetLastError();     // reported by this status, not by the next call of somebody else
    return BPT_ERR_CUDA;
}
template <int NT>
bpt_status run(const GatedFfRows& p, cudaStream_t st) {
    const bpt_status e = p.act == BPT_ACT_RELU ? run_in<BPT_ACT_RELU, NT>(p, st) : p.act == BPT_ACT_SILU ? run_in<BPT_ACT_SILU, NT>(p, st)
                                                                                                        : run_in<BPT_ACT_GELU, NT>(p, st);
    if (e != BPT_OK) return e;
    trace_mark(st, "gated_ff_rows_in");
    const bpt_status f = run_out<NT>(p, st);
    trace_mark(st, "gated_ff_rows_out");
    return f;
}

}  // namespace

bpt_status launch_gated_ff_rows(const GatedFfRows& p, cudaStream_t st) {
    return p.rows <= 8 ? run<1>(p, st) : p.rows <= 16 ? run<2>(p, st) : p.rows <= 32 ? run<4>(p, st) : run<8>(p, st);
}

}  // namespace bpt
