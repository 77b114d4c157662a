// The norm over all gradients of a model, and clipping.  See bpt_grad_norm / bpt_clip_grads in include/bpt.h.
//
// Bound by memory: every gradient is read once for the norm, and once more and written where it is scaled; between the two lies one number.
// Two launches whatever the number of tensors (up to what a launch's arguments hold): the list of tensors travels in the arguments, so
// nothing is copied and the calls can be captured.  All tensors together are cut into units of 2048 elements, and each CTA takes a
// contiguous share of the units, so that a few large and many small tensors balance.  The second kernel walks a CTA's share backwards:
// what the first one read last is still in L2.
//
// B200, on the GPU: 9 tensors of 0.26 million values 6.2 to 7.3 us (two short launches; one launch of a cluster of 16 CTAs took 8 to 10).  50 MB of
// bf16 in 54 tensors: the norm alone 16.4 us, below the limit 17, of which grad_norm is 12.3 (4.1 TB/s; a reduction of 67 MB of PyTorch's takes
// 24) and the launch behind it the rest; cut in place 31; cut into fp32 41 (150 MB read and written once are 23, the norm's own read
// comes on top).  1.2 GB in 432 tensors scaled into bf16 608 us (norm 6.2 TB/s, scaling 5.6).  Eight groups of 8 elements on their way per thread
// instead of four: 25 (below the limit) / 53 (into fp32) / 597 where four took 17.8 / 41 / 608; units dealt out in turn instead of in one range
// per CTA: 20 / 44 / 595.
//
// Squares are summed in fp32 over 8 elements and then in fp64, which costs one addition per 16 or 32 bytes; where a sum of 8 squares
// leaves the range in which fp32 loses nothing, those 8 are squared in fp64: no gradient is too large or too small for its norm.  Where that
// norm or the factor leaves fp32's normal range, the factor is taken from the norm as it was summed and applied in two steps (factor_of).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>

#include "bpt_internal.cuh"

namespace bpt {
namespace {

constexpr int kGcSms = 148;
constexpr int kGcUnit = 2048;       // elements; 8 per thread
constexpr int kGcThreads = 256;
constexpr int kGcMost = 960;        // tensors per launch: 32 bytes each, in at most 32 KB of arguments

struct GcTensor {
    const void* grad;
    void* out;              // null: in place
    long long numel;
    unsigned first_unit;    // in this launch
    unsigned flags;
};
// kGcLead: flags / kGcLead is how many elements lie between the boundary of 8 elements (16 bytes of bf16, 32 of fp32) before the tensor and its start
enum : unsigned { kGcGradBf16 = 1, kGcOutBf16 = 2, kGcSameStart = 4, kGcLead = 8 };

template <int N>
struct GcList {
    GcTensor t[N];
};
struct GcParams {
    double* parts;          // one per CTA of all launches
    float* norm;
    unsigned units, ctas;   // of this launch
    int n, first_part, all_parts;
    float max_norm, eps;
    int inf, write_norm, into;      // into: some tensor has a result of its own
};

// Calls body(tensor, first and last unit of this CTA's share in it) tensor by tensor, forwards or backwards.
template <int N, bool BACK, typename F>
__device__ __forceinline__ void walk(const GcList<N>& list, const GcParams& p, F&& body) {
    const unsigned lo = (unsigned)((unsigned long long)p.units * blockIdx.x / p.ctas), hi = (unsigned)((unsigned long long)p.units * (blockIdx.x + 1) / p.ctas);
    if (lo == hi) return;
    int a = 0, b = p.n - 1;     // the last tensor whose first unit is not behind the share's first (or last) one
    const unsigned want = BACK ? hi - 1 : lo;
    while (a < b) {
        const int mid = (a + b + 1) >> 1;
        if (list.t[mid].first_unit <= want) a = mid;
        else b = mid - 1;
    }
    for (unsigned u = BACK ? hi : lo; BACK ? u > lo : u < hi;) {
        const unsigned first = list.t[a].first_unit, next = a + 1 < p.n ? list.t[a + 1].first_unit : p.units;
        if (BACK) {
            const unsigned start = max(first, lo);
            body(list.t[a--], start - first, u - first);
            u = start;
        } else {
            const unsigned end = min(next, hi);
            body(list.t[a++], u - first, end - first);
            u = end;
        }
    }
}

__device__ __forceinline__ int lead_of(const GcTensor& t) { return (int)(t.flags / kGcLead); }

// 8 elements as they lie: 16 bytes of bf16, 32 of fp32.
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 q;
    __device__ __forceinline__ void load(const void* at) { asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(at)); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[2 * j] = __uint_as_float(w[j] << 16);
            x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
};
template <> struct Raw8<float> {
    float f[8];
    __device__ __forceinline__ void load(const void* at) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(at));
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = f[j];
    }
};
__device__ __forceinline__ float elem(float x) { return x; }
__device__ __forceinline__ float elem(__nv_bfloat16 x) { return __bfloat162float(x); }

// This thread's groups of 8 elements in units u0 .. u1 of a tensor: body(index of the group's first element, its values, whether all 8
// belong to the tensor; those that do not are 0).  kGcAhead groups are on their way at a time.
constexpr int kGcAhead = 4;
template <typename T, bool BACK, typename F>
__device__ __forceinline__ void groups_of(const GcTensor& t, unsigned u0, unsigned u1, F&& body) {
    const int lead = lead_of(t);
    const T* base = (const T*)t.grad - lead;            // on a boundary of 8 elements
    const long long g0 = (long long)u0 * (kGcUnit / 8), g1 = (long long)u1 * (kGcUnit / 8);
    const long long whole0 = lead ? 1 : 0, whole1 = (t.numel + lead) / 8;       // groups that lie in the tensor as a whole
    const long long f0 = max(g0, whole0), f1 = min(g1, whole1);
    const auto part = [&](long long g) {
        float x[8];
        const long long i = g * 8 - lead;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = i + j >= 0 && i + j < t.numel ? elem(((const T*)t.grad)[i + j]) : 0.f;
        body(i, x, false);
    };
    // the two ends, each by a warp of its own
    if (threadIdx.x == 0 && g0 < whole0) part(0);
    if (threadIdx.x == 32 && f1 >= whole0 && whole1 < g1 && whole1 * 8 < t.numel + lead) part(whole1);
    const long long n = f1 - f0, step = kGcThreads;
    long long k = threadIdx.x;
    const auto at = [&](long long i) { return BACK ? f1 - 1 - i : f0 + i; };
    for (; k + (kGcAhead - 1) * step < n; k += kGcAhead * step) {
        Raw8<T> r[kGcAhead];
#pragma unroll
        for (int j = 0; j < kGcAhead; ++j) r[j].load(base + at(k + j * step) * 8);
#pragma unroll
        for (int j = 0; j < kGcAhead; ++j) {
            float x[8];
            r[j].get(x);
            body(at(k + j * step) * 8 - lead, x, true);
        }
    }
    for (; k < n; k += step) {
        Raw8<T> r;
        r.load(base + at(k) * 8);
        float x[8];
        r.get(x);
        body(at(k) * 8 - lead, x, true);
    }
}
template <bool BACK, typename F>
__device__ __forceinline__ void groups(const GcTensor& t, unsigned u0, unsigned u1, F&& body) {
    if (t.flags & kGcGradBf16) groups_of<__nv_bfloat16, BACK>(t, u0, u1, body);
    else groups_of<float, BACK>(t, u0, u1, body);
}

template <int N>
__global__ void __launch_bounds__(kGcThreads) grad_norm_kernel(const __grid_constant__ GcList<N> list, const __grid_constant__ GcParams p) {
    __shared__ double share[kGcThreads / 32];
    __shared__ unsigned largest[kGcThreads / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    double sum = 0;
    unsigned most = 0;      // bits of |x|, which order as the values do, NaN above infinity
    if (p.inf) {
        walk<N, false>(list, p, [&](const GcTensor& t, unsigned u0, unsigned u1) {
            groups<false>(t, u0, u1, [&](long long, const float (&x)[8], bool) {
#pragma unroll
                for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);
            });
        });
    } else {
        walk<N, false>(list, p, [&](const GcTensor& t, unsigned u0, unsigned u1) {
            groups<false>(t, u0, u1, [&](long long, const float (&x)[8], bool) {
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(x[j], x[j], s);
                if (s >= 0x1p-80f && s <= 0x1p120f) {       // what underflowed is below 2^-46 of the sum
                    sum += (double)s;
                } else {
                    unsigned any = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) any |= __float_as_uint(x[j]) & 0x7fffffffu;
                    if (any) {                              // zeros are common: a table's gradient is mostly zeros
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum = fma((double)x[j], (double)x[j], sum);
                    }
                }
            });
        });
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, o);
        most = max(most, __shfl_xor_sync(~0u, most, o));
    }
    if (lane == 0) { share[warp] = sum; largest[warp] = most; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kGcThreads / 32; ++w) { sum += share[w]; most = max(most, largest[w]); }
        p.parts[p.first_part + blockIdx.x] = p.inf ? (double)__uint_as_float(most) : sum;
    }
}

// The norm from the shares, the same in every CTA: thread by thread, then over the warps, in one order.
__device__ double whole_norm(const GcParams& p) {
    __shared__ double share[kGcThreads / 32];
    double v = 0;
    if (p.inf) {
        for (int i = threadIdx.x; i < p.all_parts; i += kGcThreads) { const double q = p.parts[i]; v = q > v || q != q ? q : v; }
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < p.all_parts; i += kGcThreads) v += p.parts[i];
    }
    const auto join = [&](double a, double b) { return p.inf ? (a != a || a > b ? a : b) : a + b; };
#pragma unroll
    for (int o = 16; o; o >>= 1) v = join(v, __shfl_xor_sync(~0u, v, o));
    if ((threadIdx.x & 31) == 0) share[threadIdx.x >> 5] = v;
    __syncthreads();
    v = share[0];
    for (int w = 1; w < kGcThreads / 32; ++w) v = join(v, share[w]);
    return p.inf ? v : sqrt(v);
}

__device__ __forceinline__ void store8(float* at, const float (&x)[8]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(at), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* at, const float (&x)[8]) {
    __nv_bfloat162 q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
    uint4 w;
    memcpy(&w, q, 16);
    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" :: "l"(at), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
}
__device__ __forceinline__ void put(float x, float* y) { *y = x; }
__device__ __forceinline__ void put(float x, __nv_bfloat16* y) { *y = __float2bfloat16(x); }

// The factor as two, whose product it is: (g * step) * c.  step is 1 but for factors below fp32's normal numbers.
struct GcFactor {
    float c, step;
};
// max_norm / (norm + eps) where fp32 holds the norm and the quotient as normal numbers, which is as good as always; in fp64 otherwise.  A quotient q
// below 2^-126 is taken in two steps that lose nothing: what is left of a gradient at all, at least 2^-150 of it, was at least 2^-150 / q,
// which is 2^-24 (2^70 for q below 2^-220) and with the step 2^-124 (2^-79); and q / step is normal down to q = 2^-275, below which
// results are at most a few of the smallest numbers.
__device__ __forceinline__ GcFactor factor_of(const GcParams& p, double norm) {
    if (p.max_norm > FLT_MAX) return {1.f, 1.f};        // no limit: not infinity / infinity
    const float norm32 = (float)norm, c = p.max_norm / (norm32 + p.eps);
    if (norm32 >= FLT_MIN && norm32 <= FLT_MAX && c >= FLT_MIN) return {c, 1.f};
    const double q = (double)p.max_norm / (norm + (double)p.eps);
    const float step = q < 0x1p-220 ? 0x1p-149f : q < 0x1p-126 ? 0x1p-100f : 1.f;
    return {(float)(q / (double)step), step};
}

// c * the elements of units u0 .. u1 into a result of type T
template <typename T>
__device__ __forceinline__ void scale_units(const GcTensor& t, unsigned u0, unsigned u1, const GcFactor& by) {
    T* out = (T*)(t.out ? t.out : const_cast<void*>(t.grad));
    const bool same_start = t.flags & kGcSameStart;
    groups<true>(t, u0, u1, [&](long long i, float (&x)[8], bool whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * by.step * by.c;
        if (whole && same_start) {
            store8(out + i, x);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j >= 0 && i + j < t.numel) put(x[j], out + i + j);
        }
    });
}

template <int N>
__global__ void __launch_bounds__(kGcThreads) grad_scale_kernel(const __grid_constant__ GcList<N> list, const __grid_constant__ GcParams p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const double norm = whole_norm(p);
    if (p.write_norm && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = (float)norm;
    GcFactor by = factor_of(p, norm);
    const bool cut = by.step < 1.f || !(by.c >= 1.f);       // NaN cuts, too: a NaN norm leaves no gradient that looks sound
    if (!cut) by.c = 1.f;                                   // times 1 changes no value
    if (!cut && !p.into) return;
    walk<N, true>(list, p, [&](const GcTensor& t, unsigned u0, unsigned u1) {
        if (!cut && !t.out) return;
        if (t.flags & kGcOutBf16) scale_units<__nv_bfloat16>(t, u0, u1, by);
        else scale_units<float>(t, u0, u1, by);
    });
}

__global__ void __launch_bounds__(kGcThreads) grad_norm_finish_kernel(const __grid_constant__ GcParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float norm = (float)whole_norm(p);
    if (threadIdx.x == 0) *p.norm = norm;
}

int bytes_of(bpt_dtype t) { return t == BPT_F32 ? 4 : 2; }
bool on_element(const void* q, int bytes) { return ((uintptr_t)q & (bytes - 1)) == 0; }
long long units_of(const bpt_grad& g) {
    const int e = bytes_of(g.dtype), lead = (int)(((uintptr_t)g.grad & (8 * e - 1)) / e);
    return (g.numel + lead + kGcUnit - 1) / kGcUnit;
}

bpt_status check_grads(const bpt_grad* g, int32_t n, int32_t norm, bool clip) {
    if (n < 0 || (n && !g) || (norm != BPT_GRAD_NORM_L2 && norm != BPT_GRAD_NORM_MAX)) return BPT_ERR_INVALID_ARG;
    long long units = 0;
    for (int i = 0; i < n; ++i) {
        if (g[i].numel < 0 || (g[i].dtype != BPT_F32 && g[i].dtype != BPT_BF16)) return BPT_ERR_INVALID_ARG;
        if (g[i].numel && (!g[i].grad || !on_element(g[i].grad, bytes_of(g[i].dtype)))) return BPT_ERR_INVALID_ARG;
        if (clip && g[i].out && ((g[i].out_dtype != BPT_F32 && g[i].out_dtype != BPT_BF16) || !on_element(g[i].out, bytes_of(g[i].out_dtype))))
            return BPT_ERR_INVALID_ARG;
        if (g[i].numel > (1ll << 40)) return BPT_ERR_UNSUPPORTED;
        units += units_of(g[i]);
    }
    return units >> 31 ? BPT_ERR_UNSUPPORTED : BPT_OK;
}

// What is written must be written by one CTA and read by no other: no two results may overlap, nor a result another's gradient.
// The same tensor twice is such an overlap.
bpt_status check_overlaps(const bpt_grad* g, int32_t n) {
    struct Span { uintptr_t from, to; int who; bool write; };
    Span* s = new (std::nothrow) Span[2 * (size_t)n + 1];
    if (!s) return BPT_ERR_INVALID_ARG;
    int m = 0;
    for (int i = 0; i < n; ++i) {
        if (!g[i].numel) continue;
        const uintptr_t a = (uintptr_t)g[i].grad, b = (uintptr_t)g[i].out;
        s[m++] = {a, a + (uintptr_t)g[i].numel * bytes_of(g[i].dtype), i, !b || b == a};
        if (b && b != a) s[m++] = {b, b + (uintptr_t)g[i].numel * bytes_of(g[i].out_dtype), i, true};
        if (b == a && g[i].out_dtype != g[i].dtype) { delete[] s; return BPT_ERR_INVALID_ARG; }
    }
    std::sort(s, s + m, [](const Span& x, const Span& y) { return x.from < y.from; });
    bool ok = true;
    uintptr_t end = 0, written = 0;     // how far spans so far reach, and those that are written
    for (int i = 0; i < m && ok; ++i) {
        ok = s[i].from >= (s[i].write ? end : written);
        end = std::max(end, s[i].to);
        if (s[i].write) written = std::max(written, s[i].to);
    }
    delete[] s;
    return ok ? BPT_OK : BPT_ERR_INVALID_ARG;
}

struct GcPlan {
    unsigned units, ctas;
    int n, next;        // tensors of this launch, the first of the next one
};
// Launch by launch: what fits one list, as many CTAs as run at once.
GcPlan next_launch(const bpt_grad* g, int32_t n, int from) {
    GcPlan q{0, 0, 0, from};
    long long units = 0;
    for (; q.next < n && q.n < kGcMost; ++q.next) {
        if (!g[q.next].numel) continue;
        units += units_of(g[q.next]);
        ++q.n;
    }
    q.units = (unsigned)units;
    q.ctas = (unsigned)std::min<long long>(units, kGcSms * 4);
    return q;
}

template <typename K, typename... A>
bool start(K kernel, unsigned grid, bool dependent, cudaStream_t st, const A&... args) {
    cudaLaunchAttribute attr[1] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kGcThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = dependent ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return true;
    cudaGetLastError();     // reported by this status, not by the next call of somebody else
    return false;
}

template <int N>
bool launch(const bpt_grad* g, int from, const GcPlan& q, GcParams p, bool scale, bool dependent, cudaStream_t st) {
    GcList<N> list;
    unsigned unit = 0;
    int k = 0;
    for (int i = from; i < q.next; ++i) {
        if (!g[i].numel) continue;
        const int e = bytes_of(g[i].dtype), oe = g[i].out ? bytes_of(g[i].out_dtype) : e;
        const unsigned lead = (unsigned)(((uintptr_t)g[i].grad & (8 * e - 1)) / e);
        // whole groups of 8 can be stored in one piece where they start on a boundary in the result, too
        const bool same = !g[i].out || (((uintptr_t)g[i].out - (uintptr_t)lead * oe) & (8 * oe - 1)) == 0;
        list.t[k++] = {g[i].grad, g[i].out, g[i].numel, unit,
                       (e == 2 ? kGcGradBf16 : 0u) | ((g[i].out ? oe : e) == 2 ? kGcOutBf16 : 0u) | (same ? kGcSameStart : 0u) | lead * kGcLead};
        unit += (unsigned)units_of(g[i]);
    }
    p.units = q.units; p.ctas = q.ctas; p.n = q.n;
    const bool ok = scale ? start(grad_scale_kernel<N>, q.ctas, dependent, st, list, p) : start(grad_norm_kernel<N>, q.ctas, dependent, st, list, p);
    trace_mark(st, scale ? "grad_scale" : "grad_norm");
    return ok;
}
bool launch(const bpt_grad* g, int from, const GcPlan& q, const GcParams& p, bool scale, bool dependent, cudaStream_t st) {
    // a launch's arguments are copied: 9 tensors in the long list 12.8 us a call, in the short one 9.8 (one of 24 entries: 9.9); 117 tensors 26 and 23
    if (q.n <= 120) return launch<120>(g, from, q, p, scale, dependent, st);
    return launch<kGcMost>(g, from, q, p, scale, dependent, st);
}

size_t workspace_bytes(const bpt_grad* g, int32_t n) {
    size_t parts = 0;
    for (int from = 0; from < n;) {
        const GcPlan q = next_launch(g, n, from);
        parts += q.ctas;
        from = q.next;
    }
    return std::max<size_t>(16, parts * sizeof(double));
}

bpt_status run(const bpt_grad* g, int32_t n, int32_t norm_type, bool clip, float max_norm, float eps, float* norm, void* workspace, size_t workspace_n,
               cudaStream_t st) {
    const bpt_status s = check_grads(g, n, norm_type, clip);
    if (s != BPT_OK) return s;
    if (!norm || !on_element(norm, 4)) return BPT_ERR_INVALID_ARG;
    if (clip && (!(max_norm >= 0.f) || !(eps >= 0.f))) return BPT_ERR_INVALID_ARG;
    if (clip && check_overlaps(g, n) != BPT_OK) return BPT_ERR_INVALID_ARG;
    const size_t need = workspace_bytes(g, n);
    if (!workspace || workspace_n < need) return BPT_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return BPT_ERR_INVALID_ARG;
    GcParams p{};
    p.parts = static_cast<double*>(workspace);
    p.norm = norm;
    p.max_norm = max_norm; p.eps = eps; p.inf = norm_type == BPT_GRAD_NORM_MAX;
    int launches = 0, parts = 0;
    for (int from = 0; from < n;) {
        const GcPlan q = next_launch(g, n, from);
        if (q.n) {
            p.first_part = parts;
            if (!launch(g, from, q, p, false, false, st)) return BPT_ERR_CUDA;
            parts += (int)q.ctas;
            ++launches;
        }
        from = q.next;
    }
    p.all_parts = parts;
    // a list of one launch may begin while the norm is still being summed; several must all be through: the wait covers the last one only
    const bool dependent = launches == 1;
    if (!clip || parts == 0) {
        if (!start(grad_norm_finish_kernel, 1, dependent, st, p)) return BPT_ERR_CUDA;
        trace_mark(st, "grad_norm_finish");
        return BPT_OK;
    }
    p.write_norm = 1;
    for (int i = 0; i < n; ++i) p.into |= g[i].out != nullptr && g[i].numel > 0;
    for (int from = 0; from < n;) {
        const GcPlan q = next_launch(g, n, from);
        if (q.n) {
            if (!launch(g, from, q, p, true, dependent, st)) return BPT_ERR_CUDA;
            p.write_norm = 0;
        }
        from = q.next;
    }
    return BPT_OK;
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" size_t bpt_grad_norm_workspace_bytes(const bpt_grad* grads, int32_t n) {
    return check_grads(grads, n, BPT_GRAD_NORM_L2, false) == BPT_OK ? workspace_bytes(grads, n) : 0;
}

extern "C" bpt_status bpt_grad_norm(const bpt_grad* grads, int32_t n, int32_t norm_type, float* norm, void* workspace, size_t workspace_n, void* cuda_stream) {
    return run(grads, n, norm_type, false, 0.f, 0.f, norm, workspace, workspace_n, (cudaStream_t)cuda_stream);
}

extern "C" bpt_status bpt_clip_grads(const bpt_grad* grads, int32_t n, int32_t norm_type, float max_norm, float eps, float* norm, void* workspace,
                                     size_t workspace_n, void* cuda_stream) {
    return run(grads, n, norm_type, true, max_norm, eps, norm, workspace, workspace_n, (cudaStream_t)cuda_stream);
}
