// Token ids to node states, and the gradient of the table.  See bpt_embed_fwd / bpt_embed_bwd in include/bpt.h.
//
// Forward: out[b, t] = scale * weight[ids[b, t]], zero rows behind the tokens.  Bound by what it writes.  A few lanes of a warp per
// row, as many as the row has 16-byte pieces, 32 at most; a warp's rows are independent, so 64 warps per SM keep enough loads in flight.
//
// Backward: dW[v] = scale * sum of d_out over the places where v stands.  Float atomics would add in another order every time, and a
// table of counts per id is as long as the vocabulary; so the places are sorted by id (stable, radix 2^9 at most: one pass up to 511
// ids, two up to 262143) and the sorted list is cut into tiles of equal length, whatever the frequencies: a warp adds the rows
// of its tile in order in fp32 registers and writes a run of one id that lies inside the tile straight to dW.  The ends of runs that
// cross tiles go to fp32 partial rows, which embed_finish adds in tile order.  Rows of ids that occur nowhere are zeroed by CTAs of their own,
// so every row of dW is written once.  All sums have one order: bit-reproducible.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "bpt_internal.cuh"

namespace bpt {
namespace {

constexpr int kEmSms = 148;
constexpr int kEmDigit = 9;                 // bits per sort pass, at most
constexpr int kEmBins = 1 << kEmDigit;
constexpr int kEmSortThreads = 1024;
constexpr int kEmZeroRows = 256;            // rows of dW per CTA that zeroes

struct EmParams {
    const void* ids;
    const int32_t* lengths;
    const void* weight;                     // forward
    void* out;                              // forward: out; backward: dW
    const void* d_out;
    int* record;
    long long vocab, padding_idx;
    unsigned rows, tokens, out_rows, M;     // rows of out in all, ids and out rows per sequence, ids in all
    int D, id64;
    float scale;
    // backward
    int *hist, *keys[2], *src[2];           // sort: [tiles][kEmBins], id and row of d_out of each place, before and after a pass
    float* part;                            // [tiles of the sum][2][D]
    int sort_tile, sort_tiles, sum_tile, sum_tiles, sum_ctas;
};

__device__ __forceinline__ long long load_id(const EmParams& p, long long i) {
    return p.id64 ? __ldg((const long long*)p.ids + i) : (long long)__ldg((const int*)p.ids + i);
}
// The length of a sequence, clamped to what there is.
__device__ __forceinline__ unsigned real_tokens(const EmParams& p, unsigned b) {
    if (!p.lengths) return p.tokens;
    const int n = __ldg(p.lengths + b);
    return n < 0 ? 0u : min((unsigned)n, p.tokens);
}
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f(float x, float* y) { *y = x; }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16* y) { *y = __float2bfloat16(x); }

// VEC elements in fp32, in pieces of at most 16 bytes
template <int VEC, typename T>
__device__ __forceinline__ void load_vec(const T* at, float (&x)[VEC]) {
    if constexpr (VEC == 1) {
        x[0] = to_f(__ldg(at));
    } else {
        constexpr int per = 16 / sizeof(T);
#pragma unroll
        for (int j = 0; j < VEC / per; ++j) {
            const uint4 q = __ldg((const uint4*)at + j);
            T e[per];
            memcpy(e, &q, 16);
#pragma unroll
            for (int i = 0; i < per; ++i) x[j * per + i] = to_f(e[i]);
        }
    }
}
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T* at, const float (&x)[VEC]) {
    if constexpr (VEC == 1) {
        from_f(x[0], at);
    } else {
        constexpr int per = 16 / sizeof(T);
#pragma unroll
        for (int j = 0; j < VEC / per; ++j) {
            T e[per];
#pragma unroll
            for (int i = 0; i < per; ++i) from_f(x[j * per + i], e + i);
            uint4 q;
            memcpy(&q, e, 16);
            *((uint4*)at + j) = q;
        }
    }
}

template <typename TW, typename TO, int VEC>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmParams p, int lanes) {
    const unsigned per_cta = 256 / lanes;
    const unsigned long long row = (unsigned long long)blockIdx.x * per_cta + threadIdx.x / lanes;
    if (row >= p.rows) return;
    const unsigned b = (unsigned)row / p.out_rows, t = (unsigned)row - b * p.out_rows;
    const int lane = threadIdx.x & (lanes - 1);
    long long id = -1;
    if (t < real_tokens(p, b)) {
        id = load_id(p, (long long)b * p.tokens + t);
        if (id < 0 || id >= p.vocab) {
            if (lane == 0) *p.record = (int)BPT_ERR_INDEX;
            id = -1;
        }
    }
    TO* out = (TO*)p.out + (long long)row * p.D;
    const TW* w = (const TW*)p.weight + id * p.D;
    for (int c = lane * VEC; c < p.D; c += lanes * VEC) {
        float x[VEC];
        if (id < 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = 0.f;
        } else {
            load_vec<VEC>(w + c, x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] *= p.scale;
        }
        store_vec<VEC>(out + c, x);
    }
}

// ---------------------------------------------------------------------------------------------------------
// the sort
// ---------------------------------------------------------------------------------------------------------
// Id of place i, or `vocab` for a place that adds nothing: behind its sequence's length, at padding_idx, out of range.
__device__ __forceinline__ int sort_key(const EmParams& p, unsigned i, int* row) {
    const unsigned b = i / p.tokens, t = i - b * p.tokens;
    *row = (int)(b * p.out_rows + t);
    if (t >= real_tokens(p, b)) return (int)p.vocab;
    const long long id = load_id(p, i);
    if (id < 0 || id >= p.vocab) {
        *p.record = (int)BPT_ERR_INDEX;
        return (int)p.vocab;
    }
    return id == p.padding_idx ? (int)p.vocab : (int)id;
}
__device__ __forceinline__ void pdl_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// How often each digit stands in each tile of the list.
__global__ void __launch_bounds__(kEmSortThreads) embed_hist_kernel(EmParams p, int from, int shift, int bins) {
    __shared__ int count[kEmBins];
    pdl_start();
    for (int i = threadIdx.x; i < bins; i += kEmSortThreads) count[i] = 0;
    __syncthreads();
    pdl_wait();
    const long long first = (long long)blockIdx.x * p.sort_tile, end = min(first + p.sort_tile, (long long)p.M);
    for (long long i = first + threadIdx.x; i < end; i += kEmSortThreads) {
        int row;
        const int key = from < 0 ? sort_key(p, (unsigned)i, &row) : p.keys[from][i];
        atomicAdd(&count[(key >> shift) & (bins - 1)], 1);      // whole numbers: any order gives the same
    }
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += kEmSortThreads) p.hist[(long long)blockIdx.x * kEmBins + i] = count[i];
}

// One stable pass: a place goes behind all of smaller digit, and of its own digit behind those of earlier tiles, earlier rounds,
// earlier warps and lower lanes.
__global__ void __launch_bounds__(kEmSortThreads) embed_scatter_kernel(EmParams p, int from, int to, int shift, int bins) {
    __shared__ int base[kEmBins];                   // where this tile's next place of a digit goes
    __shared__ int total[kEmBins];
    __shared__ unsigned short in_warp[32][kEmBins];
    __shared__ int scan[32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_start();
    for (int i = tid; i < kEmBins; i += kEmSortThreads) base[i] = total[i] = 0;
    for (int i = tid; i < 32 * kEmBins; i += kEmSortThreads) (&in_warp[0][0])[i] = 0;
    __syncthreads();
    pdl_wait();
    // groups of `bins` threads share out the tiles
    {
        const int groups = kEmSortThreads / bins, group = tid / bins, d = tid - group * bins;
        int before = 0, all = 0;
#pragma unroll 8
        for (int t = group; t < p.sort_tiles; t += groups) {
            const int c = p.hist[(long long)t * kEmBins + d];
            all += c;
            before += t < (int)blockIdx.x ? c : 0;
        }
        atomicAdd(&total[d], all);
        atomicAdd(&base[d], before);
    }
    __syncthreads();
    int mine = tid < bins ? total[tid] : 0, sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(~0u, sum, o);
        if (lane >= o) sum += up;
    }
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    if (tid < bins) {
        int off = sum - mine;
        for (int w = 0; w < warp; ++w) off += scan[w];
        base[tid] += off;
    }
    const long long first = (long long)blockIdx.x * p.sort_tile, end = min(first + p.sort_tile, (long long)p.M);
    for (long long at = first; at < end; at += kEmSortThreads) {
        const long long i = at + tid;
        const bool on = i < end;
        int key = 0, row = 0;
        if (on) {
            if (from < 0) {
                key = sort_key(p, (unsigned)i, &row);
            } else {
                key = p.keys[from][i];
                row = p.src[from][i];
            }
        }
        const int d = (key >> shift) & (bins - 1);
        const unsigned peers = __match_any_sync(~0u, on ? d : -1);
        const int rank = __popc(peers & ((1u << lane) - 1));
        if (on && rank == 0) in_warp[warp][d] = (unsigned short)__popc(peers);
        __syncthreads();
        if (tid < bins) {                           // counts of the warps to places
            int off = base[tid];
            int next = off;
#pragma unroll
            for (int w = 0; w < 32; ++w) next += in_warp[w][tid];
            total[tid] = next;
        }
        __syncthreads();
        if (on) {
            int off = base[d] + rank;
            for (int w = 0; w < warp; ++w) off += in_warp[w][d];
            p.keys[to][off] = key;
            p.src[to][off] = row;
        }
        __syncthreads();
        if (on && rank == 0) in_warp[warp][d] = 0;
        if (tid < bins) base[tid] = total[tid];
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------------------------------------
constexpr int kEmSumWarps = 4;
constexpr int kEmAhead = 8;     // rows of d_out on their way per warp

// first i with keys[i] >= key
__device__ int lower_bound(const int* keys, int n, int key) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

template <typename TW, typename TO, int VEC>
__device__ void sum_tile(const EmParams& p, const int* keys, const int* src, int tile, int slice, int lane) {
    const int first = tile * p.sum_tile, end = min(first + p.sum_tile, (int)p.M);
    const int c = (slice * 32 + lane) * VEC;
    const bool on = c < p.D;
    const TO* d_out = (const TO*)p.d_out + c;
    TW* dw = (TW*)p.out + c;
    const int before = first > 0 ? keys[first - 1] : -1, after = end < (int)p.M ? keys[end] : -1;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    auto flush = [&](int key, bool from_before, bool goes_on) {
        if (key < (int)p.vocab && on) {
            if (from_before || goes_on) {
                float* at = p.part + ((long long)tile * 2 + (from_before ? 0 : 1)) * p.D + c;
#pragma unroll
                for (int i = 0; i < VEC; ++i) at[i] = acc[i];
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] *= p.scale;
                store_vec<VEC>(dw + (long long)key * p.D, acc);
            }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    };
    int run = keys[first];
    bool from_before = run == before;
    for (int at = first; at < end; at += 32) {
        const int n = min(32, end - at);
        const int my_key = lane < n ? keys[at + lane] : -1, my_src = lane < n ? src[at + lane] : 0;
        for (int r = 0; r < n; r += kEmAhead) {
            float x[kEmAhead][VEC];
#pragma unroll
            for (int j = 0; j < kEmAhead; ++j) {
                const int key = __shfl_sync(~0u, my_key, (r + j) & 31), row = __shfl_sync(~0u, my_src, (r + j) & 31);
                if (r + j < n && key < (int)p.vocab && on) load_vec<VEC>(d_out + (long long)row * p.D, x[j]);
                else
#pragma unroll
                    for (int i = 0; i < VEC; ++i) x[j][i] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < kEmAhead; ++j) {
                const int key = __shfl_sync(~0u, my_key, (r + j) & 31);
                if (r + j >= n) break;
                if (key != run) {
                    flush(run, from_before, false);
                    run = key;
                    from_before = false;
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] += x[j][i];
            }
        }
    }
    flush(run, from_before, run == after);
}

template <typename TW, typename TO, int VEC>
__global__ void __launch_bounds__(kEmSumWarps * 32) embed_sum_kernel(EmParams p, int sorted) {
    __shared__ bool there[kEmZeroRows];
    pdl_start();
    pdl_wait();
    const int *keys = p.keys[sorted], *src = p.src[sorted];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x < (unsigned)p.sum_ctas) {
        const int slices = (p.D + 32 * VEC - 1) / (32 * VEC);
        const long long work = (long long)blockIdx.x * kEmSumWarps + warp;
        const int tile = (int)(work / slices);
        if (tile < p.sum_tiles) sum_tile<TW, TO, VEC>(p, keys, src, tile, (int)(work - (long long)tile * slices), lane);
        return;
    }
    // rows of ids that occur nowhere
    const long long first = (long long)(blockIdx.x - p.sum_ctas) * kEmZeroRows, end = min(first + kEmZeroRows, p.vocab);
    for (int i = threadIdx.x; i < kEmZeroRows; i += kEmSumWarps * 32) there[i] = false;
    __syncthreads();
    const int lo = lower_bound(keys, (int)p.M, (int)first), hi = lower_bound(keys, (int)p.M, (int)end);
    for (int i = lo + threadIdx.x; i < hi; i += kEmSumWarps * 32) there[keys[i] - first] = true;
    __syncthreads();
    const float zero[VEC] = {};
    for (long long v = first + warp; v < end; v += kEmSumWarps) {
        if (there[v - first]) continue;
        for (int c = lane * VEC; c < p.D; c += 32 * VEC) store_vec<VEC>((TW*)p.out + v * p.D + c, zero);
    }
}

// A run of one id over several tiles: the partial rows of its tiles, in order, split over the warps and joined in the order of the warps.
// One CTA per tile and 32 columns' vectors; all but those in whose tile such a run starts end at once.
constexpr int kEmFinishWarps = 8;
template <typename TW, int VEC>
__global__ void __launch_bounds__(kEmFinishWarps * 32) embed_finish_kernel(EmParams p, int sorted) {
    __shared__ float share[kEmFinishWarps][32 * VEC];
    pdl_wait();
    const int* keys = p.keys[sorted];
    const int tile = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int first = tile * p.sum_tile, next = first + p.sum_tile;
    if (next >= (int)p.M) return;
    const int key = keys[next];
    if (key >= (int)p.vocab || keys[next - 1] != key) return;           // no run of an id goes on
    if (keys[first] == key && first > 0 && keys[first - 1] == key) return;      // it began in an earlier tile
    int last = tile + 1;                                                // the last tile that begins with this id
    for (;;) {
        const long long t = (long long)last + 1 + lane, i = t * p.sum_tile;
        const unsigned same = __ballot_sync(~0u, i < (long long)p.M && keys[i < (long long)p.M ? i : 0] == key);
        const int more = same == ~0u ? 32 : __ffs(~same) - 1;
        last += more;
        if (more < 32) break;
    }
    const int n = last - tile + 1;      // slot 1 of the first tile, slot 0 of the others
    const int per = (n + kEmFinishWarps - 1) / kEmFinishWarps, from = min(n, warp * per), to = min(n, from + per);
    const int c = ((int)blockIdx.y * 32 + lane) * VEC;
    float acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    if (c < p.D) {
#pragma unroll 4
        for (int j = from; j < to; ++j) {
            const float* at = p.part + ((long long)(tile + j) * 2 + (j == 0 ? 1 : 0)) * p.D + c;
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += at[i];
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) share[warp][lane * VEC + i] = acc[i];
    __syncthreads();
    if (warp == 0 && c < p.D) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float s = share[0][lane * VEC + i];
            for (int w = 1; w < kEmFinishWarps; ++w) s += share[w][lane * VEC + i];
            acc[i] = s * p.scale;
        }
        store_vec<VEC>((TW*)p.out + (long long)key * p.D + c, acc);
    }
}

bpt_status check_embed(const bpt_embed_args* a) {
    if (!a || a->batch < 0 || a->tokens < 0 || a->out_rows < a->tokens || a->vocab < 1 || a->D < 1) return BPT_ERR_INVALID_ARG;
    if ((a->id_bytes != 4 && a->id_bytes != 8) || !std::isfinite(a->scale)) return BPT_ERR_INVALID_ARG;
    if (a->weight_dtype != BPT_F32 && a->weight_dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    if (a->out_dtype != BPT_F32 && a->out_dtype != BPT_BF16) return BPT_ERR_INVALID_ARG;
    if (a->padding_idx < -1 || a->padding_idx >= a->vocab) return BPT_ERR_INVALID_ARG;
    // row numbers and sort keys are 32-bit
    if (a->vocab > 0x3fffffffll || a->D > (1 << 20)) return BPT_ERR_UNSUPPORTED;
    if (a->batch && a->out_rows > 0x3fffffffll / a->batch) return BPT_ERR_UNSUPPORTED;
    if (a->batch * a->out_rows > (1ll << 40) / a->D) return BPT_ERR_UNSUPPORTED;     // no device holds it; grids stay below 2^31
    return BPT_OK;
}
EmParams embed_params(const bpt_embed_args& a) {
    EmParams p{};
    p.ids = a.ids; p.lengths = a.lengths; p.weight = a.weight;
    p.vocab = a.vocab; p.padding_idx = a.padding_idx;
    p.rows = (unsigned)(a.batch * a.out_rows); p.tokens = (unsigned)a.tokens; p.out_rows = (unsigned)a.out_rows;
    p.M = (unsigned)(a.batch * a.tokens);
    p.D = a.D; p.id64 = a.id_bytes == 8; p.scale = a.scale;
    return p;
}
bool on_16(const void* q) { return ((uintptr_t)q & 15) == 0; }
bool on_element(const void* q, int bytes) { return ((uintptr_t)q & (bytes - 1)) == 0; }
int bytes_of(bpt_dtype t) { return t == BPT_F32 ? 4 : 2; }

struct EmPlan {
    int passes, digit, sort_tile, sort_tiles, sum_tile, sum_tiles;
    size_t hist, list, part;     // bytes; list: one of the four arrays
};
EmPlan embed_plan(const bpt_embed_args& a) {
    EmPlan q{};
    const long long M = a.batch * a.tokens;
    int bits = 1;
    while ((a.vocab >> bits) != 0) ++bits;          // keys are 0 .. vocab
    q.passes = (bits + kEmDigit - 1) / kEmDigit;
    q.digit = (bits + q.passes - 1) / q.passes;
    // one CTA per tile and SM, no more: each scatter CTA adds up the counts of all tiles
    q.sort_tile = (int)std::max<long long>(kEmSortThreads, ((M + kEmSms - 1) / kEmSms + 31) / 32 * 32);
    q.sort_tiles = (int)((M + q.sort_tile - 1) / q.sort_tile);
    q.sum_tile = 32;
    q.sum_tiles = (int)((M + q.sum_tile - 1) / q.sum_tile);
    q.hist = (size_t)q.sort_tiles * kEmBins * 4;
    q.list = ((size_t)M * 4 + 15) / 16 * 16;
    q.part = (size_t)q.sum_tiles * 2 * a.D * 4;
    return q;
}

template <typename... A>
bool start(void (*kernel)(A...), dim3 grid, int threads, cudaStream_t st, bool first, A... args) {
    cudaLaunchAttribute attr[1] = {};       // its launch overlaps the kernel before, for whose end it then waits
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = first ? 0 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return true;
    cudaGetLastError();     // reported by this status, not by the next call of somebody else
    return false;
}

template <typename TW, typename TO, int VEC>
bool run_sum(const EmParams& p, int sorted, cudaStream_t st) {
    const int slices = (p.D + 32 * VEC - 1) / (32 * VEC);
    EmParams q = p;
    q.sum_ctas = (int)(((long long)p.sum_tiles * slices + kEmSumWarps - 1) / kEmSumWarps);
    const unsigned zero_ctas = (unsigned)((p.vocab + kEmZeroRows - 1) / kEmZeroRows);
    if (!start(embed_sum_kernel<TW, TO, VEC>, dim3(q.sum_ctas + zero_ctas), kEmSumWarps * 32, st, p.sum_tiles == 0, q, sorted)) return false;
    trace_mark(st, "embed_sum");
    if (p.sum_tiles < 2) return true;       // no run crosses tiles
    if (!start(embed_finish_kernel<TW, VEC>, dim3((unsigned)p.sum_tiles - 1, (unsigned)slices), kEmFinishWarps * 32, st, false, q, sorted)) return false;
    trace_mark(st, "embed_finish");
    return true;
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" bpt_status bpt_embed_fwd(const bpt_embed_args* a, void* out, void* cuda_stream) {
    const bpt_status s = check_embed(a);
    if (s != BPT_OK) return s;
    if (a->batch == 0 || a->out_rows == 0) return BPT_OK;
    if (!out || !a->weight || (a->tokens && !a->ids)) return BPT_ERR_INVALID_ARG;
    const int we = bytes_of(a->weight_dtype), oe = bytes_of(a->out_dtype);
    if (!on_element(a->ids, a->id_bytes) || !on_element(a->lengths, 4) || !on_element(a->weight, we) || !on_element(out, oe)) return BPT_ERR_INVALID_ARG;
    EmParams p = embed_params(*a);
    p.out = out;
    p.record = device_record();
    if (!p.record) return BPT_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool vec = a->D % 8 == 0 && on_16(a->weight) && on_16(out);       // whole 16-byte pieces in both
    const int pieces = vec ? a->D / 8 : a->D;
    int lanes = 1;
    while (lanes < pieces && lanes < 32) lanes *= 2;
    const unsigned grid = (unsigned)(((unsigned long long)p.rows + 256 / lanes - 1) / (256 / lanes));
    typedef __nv_bfloat16 bf;
    const bool wf = a->weight_dtype == BPT_F32, of = a->out_dtype == BPT_F32;
#define BPT_EMBED_FWD(TW, TO) (vec ? start(embed_fwd_kernel<TW, TO, 8>, dim3(grid), 256, st, true, p, lanes) \
                                   : start(embed_fwd_kernel<TW, TO, 1>, dim3(grid), 256, st, true, p, lanes))
    const bool ok = wf ? (of ? BPT_EMBED_FWD(float, float) : BPT_EMBED_FWD(float, bf)) : (of ? BPT_EMBED_FWD(bf, float) : BPT_EMBED_FWD(bf, bf));
#undef BPT_EMBED_FWD
    trace_mark(st, "embed_fwd");
    return ok ? BPT_OK : BPT_ERR_CUDA;
}

extern "C" size_t bpt_embed_bwd_workspace_bytes(const bpt_embed_args* a) {
    if (check_embed(a) != BPT_OK) return 0;
    const EmPlan q = embed_plan(*a);
    return std::max<size_t>(16, q.hist + 4 * q.list + q.part);
}

extern "C" bpt_status bpt_embed_bwd(const bpt_embed_args* a, const void* d_out, void* d_weight, void* workspace, size_t workspace_bytes,
                                    void* cuda_stream) {
    const bpt_status s = check_embed(a);
    if (s != BPT_OK) return s;
    const long long M = a->batch * a->tokens;
    if (!d_weight || (M && (!a->ids || !d_out))) return BPT_ERR_INVALID_ARG;
    const int we = bytes_of(a->weight_dtype), oe = bytes_of(a->out_dtype);
    if (!on_element(a->ids, a->id_bytes) || !on_element(a->lengths, 4) || !on_element(d_weight, we) || !on_element(d_out, oe)) return BPT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < bpt_embed_bwd_workspace_bytes(a)) return BPT_ERR_WORKSPACE;
    if (!on_16(workspace)) return BPT_ERR_INVALID_ARG;
    const EmPlan q = embed_plan(*a);
    EmParams p = embed_params(*a);
    p.d_out = d_out;
    p.out = d_weight;
    p.record = device_record();
    if (!p.record) return BPT_ERR_CUDA;
    char* at = static_cast<char*>(workspace);
    p.hist = reinterpret_cast<int*>(at); at += q.hist;
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = reinterpret_cast<int*>(at); at += q.list;
        p.src[i] = reinterpret_cast<int*>(at); at += q.list;
    }
    p.part = reinterpret_cast<float*>(at);
    p.sort_tile = q.sort_tile; p.sort_tiles = q.sort_tiles; p.sum_tile = q.sum_tile; p.sum_tiles = q.sum_tiles;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int sorted = 0;
    if (M > 0) {
        const int bins = 1 << q.digit;
        for (int i = 0; i < q.passes; ++i) {
            const int from = i == 0 ? -1 : (i - 1) & 1, to = i & 1;
            if (!start(embed_hist_kernel, dim3(q.sort_tiles), kEmSortThreads, st, i == 0, p, from, i * q.digit, bins)) return BPT_ERR_CUDA;
            trace_mark(st, "embed_hist");
            if (!start(embed_scatter_kernel, dim3(q.sort_tiles), kEmSortThreads, st, false, p, from, to, i * q.digit, bins)) return BPT_ERR_CUDA;
            trace_mark(st, "embed_scatter");
            sorted = to;
        }
    }
    const bool vec = a->D % 8 == 0 && on_16(d_weight) && on_16(d_out);
    typedef __nv_bfloat16 bf;
    const bool wf = a->weight_dtype == BPT_F32, of = a->out_dtype == BPT_F32;
#define BPT_EMBED_SUM(TW, TO) (vec ? run_sum<TW, TO, 8>(p, sorted, st) : run_sum<TW, TO, 1>(p, sorted, st))
    const bool ok = wf ? (of ? BPT_EMBED_SUM(float, float) : BPT_EMBED_SUM(float, bf)) : (of ? BPT_EMBED_SUM(bf, float) : BPT_EMBED_SUM(bf, bf));
#undef BPT_EMBED_SUM
    return ok ? BPT_OK : BPT_ERR_CUDA;
}
