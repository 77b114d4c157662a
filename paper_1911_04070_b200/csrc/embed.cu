// Token ids to node states, and the gradient of the table.  See bpt_embed_fwd / bpt_embed_bwd in include/bpt.h.
//
// Forward: out[b, t] = scale * weight[ids[b, t]], zero rows behind the tokens.  It mostly writes: 67 MB (4 x 16383 rows of 512 in bf16, 8192
// tokens each) in 16.4 us, 4.1 TB/s, and 268 MB in 47 (8 x 8192 ids of 256, 2048 wide) or 69 (of 131072, drawn as words are, whose rows it reads from
// memory).  Timed the same way PyTorch's fill_ and zero_ of 67 MB take 20.5 us, of 268 MB 72.
//
// Backward: dW[v] = scale * sum of d_out over the places where v stands.  Float atomics would add in another order every time, and a
// table of counts per id is as long as the vocabulary; so the places are sorted by id (stable, digits of at most 9 bits: one pass up to 511
// ids, two up to 262143), by one launch of one cluster up to 131072 places and by two launches a pass beyond.  The sorted list is cut into
// tiles of equal length, whatever the frequencies: a warp adds the rows of its tile in order in fp32 registers and writes a run of one id that
// lies inside the tile straight to dW; the ends of runs that cross warps are joined in shared memory, of those that cross CTAs in
// embed_finish, both in the order of the list.  Rows of ids that occur nowhere are zeroed by CTAs of their own between those that sum, so
// every row of dW is written once.  All sums have one order: bit-reproducible.
// B200, forward + backward on the GPU: 4 x 8192 ids of 256, 512 wide, 42 us (forward 16, sort 9.5, sums and zeros about 10, finish about 6);
// 16 x 512 ids of 32001 x 201 in fp32 31 us (forward 8, sort 9.5); 8 x 8192 ids of 131072 x 2048 240 us (forward 68, sort 22, sums and zeros of
// 268 MB read and 537 MB written about 135).  What it took: sorting by two launches a pass and tiles per warp only 57 / 45 / 300; zeroing all of dW beside
// the sort 289 for the last (a kernel that only zeroes is the slower way: 3.9 TB/s); CTAs that zero 32 KB instead of 128 KB there 290, and 128 KB
// instead of a share of the table's size 37 instead of 31 for the second.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cooperative_groups.h>
#include <cstring>

#include "any8.cuh"
#include "bpt_internal.cuh"

namespace bpt {
namespace {

constexpr int kEmSms = 148;
constexpr int kEmDigit = 9;                 // bits per sort pass, at most
constexpr int kEmBins = 1 << kEmDigit;
constexpr int kEmSortThreads = 1024;

// n / d of n < 2^31 by a multiplication, after Granlund and Montgomery, Division by Invariant Integers using Multiplication (1994): with
// s = ceil(log2 d) and m = floor(2^32 (2^s - d) / d) + 1 it is (floor(m n / 2^32) + n) >> s.
struct FastDiv {
    unsigned d, m, s;
    FastDiv(unsigned by = 1) : d(by), m(1), s(0) {
        while ((1ull << s) < by) ++s;
        m = (unsigned)(((1ull << 32) * ((1ull << s) - by)) / by + 1);
    }
    __device__ __forceinline__ unsigned div(unsigned n) const { return (__umulhi(m, n) + n) >> s; }
};

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
    int* hist;                              // sort: [tiles][kEmBins]
    int2* list[2];                          // id and row of d_out of each place, before and after a pass
    float* part;                            // [sum_tiles][2][D]
    int sort_tile, sort_tiles, sum_tiles, warp_tile, slices, zero_rows, sorted;      // sorted: which of the lists is
    unsigned zero_ctas;
    FastDiv by_D, by_tokens, by_out_rows;
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

// 8 elements in fp32, in whole 16-byte pieces
template <typename T>
__device__ __forceinline__ void load8(const T* at, float (&x)[8]) {
    constexpr int per = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 8 / per; ++j) {
        const uint4 q = __ldg((const uint4*)at + j);
        T e[per];
        memcpy(e, &q, 16);
#pragma unroll
        for (int i = 0; i < per; ++i) x[j * per + i] = to_f(e[i]);
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* at, const float (&x)[8]) {
    constexpr int per = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 8 / per; ++j) {
        T e[per];
#pragma unroll
        for (int i = 0; i < per; ++i) from_f(x[j * per + i], e + i);
        uint4 q;
        memcpy(&q, e, 16);
        *((uint4*)at + j) = q;
    }
}

// The id of a row of out, or -1 for a row of zeros.
__device__ __forceinline__ long long id_of_row(const EmParams& p, unsigned row) {
    const unsigned b = p.by_out_rows.div(row), t = row - b * p.out_rows;
    if (t >= real_tokens(p, b)) return -1;
    const long long id = load_id(p, (long long)b * p.tokens + t);
    if (id >= 0 && id < p.vocab) return id;
    atomicOr(p.record, kRecordIndex);
    return -1;
}

// Rows of whole 16-byte pieces: `lanes` threads per row, kEmRows rows one after another per thread, with the ids and then the pieces of all
// of them on their way at once.
constexpr int kEmRows = 4;
template <typename TW, typename TO>
__global__ void __launch_bounds__(256) embed_fwd_kernel(EmParams p, int lanes) {
    const unsigned groups = 256 / lanes;
    const unsigned first = (blockIdx.x * groups + threadIdx.x / lanes) * kEmRows;
    const int lane = threadIdx.x & (lanes - 1);
    long long id[kEmRows];
#pragma unroll
    for (int r = 0; r < kEmRows; ++r) id[r] = first + r < p.rows ? id_of_row(p, first + r) : -1;
    for (int c = lane * 8; c < p.D; c += lanes * 8) {
        float x[kEmRows][8];
#pragma unroll
        for (int r = 0; r < kEmRows; ++r) {
            if (id[r] >= 0) {
                load8((const TW*)p.weight + id[r] * p.D + c, x[r]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[r][i] = 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < kEmRows; ++r) {
            if (first + r >= p.rows) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[r][i] = id[r] >= 0 ? x[r][i] * p.scale : 0.f;
            store8((TO*)p.out + (long long)(first + r) * p.D + c, x[r]);
        }
    }
}

// scale * 8 elements from column c on of an id's row, which may begin before the row or end behind it; zeros without an id.
template <typename TW>
__device__ __forceinline__ void scaled8(const EmParams& p, long long id, int c, float (&x)[8]) {
    if (id < 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
        return;
    }
    const TW* w = (const TW*)p.weight + id * p.D + c;
    if (any8_inside(w, (const TW*)p.weight, p.vocab * p.D)) {
        Any8<TW> raw;
        raw.load(w);
        raw.get(x);
    } else {                                    // at the ends of the table
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
            const long long at = id * p.D + c + j;
            const float v = at >= 0 && at < p.vocab * p.D ? to_f(__ldg(w + j)) : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = k == j ? v : x[k];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= p.scale;
}
// Any width from 8 on and any start: out as one list of elements, 8 of them that lie on a 16-byte boundary per thread, out of one row or the ends of two.
template <typename TW, typename TO>
__global__ void __launch_bounds__(256) embed_fwd_flat_kernel(EmParams p) {
    const int lead = (int)(((uintptr_t)p.out & 15) / sizeof(TO));
    const long long total = (long long)p.rows * p.D, i0 = ((long long)blockIdx.x * 256 + threadIdx.x) * 8 - lead;
    if (i0 >= total) return;
    const long long from = i0 < 0 ? 0 : i0;
    const unsigned row = total <= 0x7fffffffll ? p.by_D.div((unsigned)from) : (unsigned)(from / p.D);
    const int c = (int)(from - (long long)row * p.D), n = (int)(min(i0 + 8, total) - from), left = p.D - c;
    float x[8];
    scaled8<TW>(p, id_of_row(p, row), c, x);
    if (left < n) {
        float y[8];
        scaled8<TW>(p, id_of_row(p, row + 1), -left, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < left ? x[j] : y[j];
    }
    TO* out = (TO*)p.out + from;
    if (n == 8) {                       // then i0 >= 0, and a whole piece or two of out
        store8(out, x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) from_f(x[j], out + j);
    }
}
// Narrower than that: an element per thread.
template <typename TW, typename TO>
__global__ void __launch_bounds__(256) embed_fwd_narrow_kernel(EmParams p) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long long)p.rows * p.D) return;
    const unsigned row = (unsigned)(i / p.D);
    const long long id = id_of_row(p, row);
    from_f(id >= 0 ? to_f(__ldg((const TW*)p.weight + id * p.D + (i - (long long)row * p.D))) * p.scale : 0.f, (TO*)p.out + i);
}

// ---------------------------------------------------------------------------------------------------------
// the sort
// ---------------------------------------------------------------------------------------------------------
// Place i of the list as the sort begins with it: its id, or `vocab` for a place that adds nothing (behind its sequence's length, at padding_idx,
// out of range), and its row of d_out.
__device__ __forceinline__ int2 place_of(const EmParams& p, unsigned i, long long id) {
    const unsigned b = p.by_tokens.div(i), t = i - b * p.tokens;
    const bool real = t < real_tokens(p, b), in = id >= 0 && id < p.vocab;
    if (real && !in) atomicOr(p.record, kRecordIndex);
    return make_int2(real && in && id != p.padding_idx ? (int)id : (int)p.vocab, (int)(b * p.out_rows + t));
}
__device__ __forceinline__ void pdl_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The lanes of the warp with the same d, of `bits` bits, among the lanes of `on`.  One vote a bit: match.any takes longer.
__device__ __forceinline__ unsigned same_digit(int d, int bits, unsigned on) {
    unsigned peers = on;
#pragma unroll
    for (int b = 0; b < kEmDigit; ++b) {
        if (b >= bits) break;
        const unsigned ones = __ballot_sync(~0u, (d >> b) & 1);
        peers &= (d >> b) & 1 ? ones : ~ones;
    }
    return peers;
}

// How often each digit stands in each tile of the list.
__global__ void __launch_bounds__(kEmSortThreads) embed_hist_kernel(EmParams p, int from, int shift, int bins) {
    __shared__ int count[kEmBins];
    pdl_start();
    for (int i = threadIdx.x; i < bins; i += kEmSortThreads) count[i] = 0;
    __syncthreads();
    pdl_wait();
    const long long first = (long long)blockIdx.x * p.sort_tile, end = min(first + p.sort_tile, (long long)p.M);
    for (long long i = first + threadIdx.x; i < end; i += kEmSortThreads) {
        int key;
        if (from < 0) {
            key = place_of(p, (unsigned)i, load_id(p, i)).x;
        } else {
            key = p.list[from][i].x;
        }
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
        int2 entry = make_int2(0, 0);
        if (on) {
            if (from < 0) {
                entry = place_of(p, (unsigned)i, load_id(p, i));
            } else {
                entry = p.list[from][i];
            }
        }
        const int d = (entry.x >> shift) & (bins - 1);
        const unsigned peers = same_digit(d, 31 - __clz(bins), __ballot_sync(~0u, on));
        const int rank = __popc(peers & ((1u << lane) - 1));
        if (on && rank == 0) in_warp[warp][d] = (unsigned short)__popc(peers);
        __syncthreads();
        if (tid < bins) {                           // counts of the warps to places
            int next = base[tid];
#pragma unroll
            for (int w = 0; w < 32; ++w) next += in_warp[w][tid];
            total[tid] = next;
        }
        __syncthreads();
        if (on) {
            int off = base[d] + rank;
            for (int w = 0; w < warp; ++w) off += in_warp[w][d];
            p.list[to][off] = entry;
        }
        __syncthreads();
        if (on && rank == 0) in_warp[warp][d] = 0;
        if (tid < bins) base[tid] = total[tid];
        __syncthreads();
    }
}

// The whole sort of up to 131072 places (16 CTAs of 512 threads, 16 places each) in one launch: one cluster, a slice of the list per CTA, in registers.  A warp counts the digits
// of its own part of the slice, 32 places at a time; counts are added up over the warps, and over the cluster through distributed
// shared memory.  Between two passes the list goes through global memory (L2): scattered 8-byte stores to the other CTAs' shared memory
// took three times as long.
constexpr int kEmClusterThreads = 512, kEmRounds = 16, kEmClusterCtas = 16;
__global__ void __launch_bounds__(kEmClusterThreads) embed_sort_kernel(EmParams p, int passes, int digit, int rounds) {
    namespace cg = cooperative_groups;
    constexpr int warps = kEmClusterThreads / 32;
    __shared__ int total[kEmBins], base[kEmBins], scan[warps];         // this CTA's counts; where its first place of a digit goes
    __shared__ __align__(16) unsigned short in_warp[warps * kEmBins];   // [warps][bins]; cleared two at a time
    const cg::cluster_group cluster = cg::this_cluster();
    const int slice = rounds * kEmClusterThreads, bins = 1 << digit, me = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, first = me * slice + warp * rounds * 32 + lane, M = (int)p.M;
    pdl_start();
    int2 entry[kEmRounds];
    {
        long long id[kEmRounds];        // all on their way before one is looked at
#pragma unroll
        for (int r = 0; r < kEmRounds; ++r)
            if (r < rounds && first + r * 32 < M) id[r] = load_id(p, first + r * 32);
#pragma unroll
        for (int r = 0; r < kEmRounds; ++r)
            if (r < rounds && first + r * 32 < M) entry[r] = place_of(p, (unsigned)(first + r * 32), id[r]);
    }
    unsigned short* mine = in_warp + warp * bins;
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * digit;
        for (int i = lane; i < bins / 2; i += 32) ((unsigned*)mine)[i] = 0;
        if (pass > 0) {
#pragma unroll
            for (int r = 0; r < kEmRounds; ++r)
                if (r < rounds && first + r * 32 < M) entry[r] = __ldcg(&p.list[(pass + 1) & 1][first + r * 32]);
        }
        __syncwarp();
        int rank[kEmRounds];
#pragma unroll
        for (int r = 0; r < kEmRounds; ++r) {
            if (r >= rounds) break;
            const bool on = first + r * 32 < M;
            const int d = on ? (entry[r].x >> shift) & (bins - 1) : 0;
            const unsigned peers = same_digit(d, digit, __ballot_sync(~0u, on));
            const int before = mine[d], lower = __popc(peers & ((1u << lane) - 1));
            __syncwarp();
            if (on && lower == 0) mine[d] = (unsigned short)(before + __popc(peers));
            __syncwarp();
            rank[r] = before + lower;
        }
        __syncthreads();
        if (tid < bins) {
            unsigned short c[warps];
#pragma unroll
            for (int w = 0; w < warps; ++w) c[w] = in_warp[w * bins + tid];
            int sum = 0;
#pragma unroll
            for (int w = 0; w < warps; ++w) {
                in_warp[w * bins + tid] = (unsigned short)sum;              // places of the digit in the warps before: at most 2^13
                sum += c[w];
            }
            total[tid] = sum;
        }
        cluster.sync();
        int all = 0, before = 0;
        if (tid < bins)
#pragma unroll
            for (int c = 0; c < kEmClusterCtas; ++c) {
                const int n = c < ctas ? cluster.map_shared_rank(total, c)[tid] : 0;
                all += n;
                before += c < me ? n : 0;
            }
        int sum = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) scan[warp] = sum;
        __syncthreads();
        if (tid < bins) {
            int off = sum - all + before;
#pragma unroll
            for (int w = 0; w < warps; ++w) off += w < warp ? scan[w] : 0;
            base[tid] = off;
        }
        __syncthreads();
        int2* to = p.list[pass & 1];
#pragma unroll
        for (int r = 0; r < kEmRounds; ++r) {
            if (r >= rounds) break;
            if (first + r * 32 >= M) continue;
            const int d = (entry[r].x >> shift) & (bins - 1);
            to[base[d] + mine[d] + rank[r]] = entry[r];
        }
        // nobody reads this CTA's counts any more; between two passes the list is written
        if (ctas > 1 || pass + 1 < passes) cluster.sync();
    }
}

// ---------------------------------------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------------------------------------
constexpr int kEmSumWarps = 8;
constexpr int kEmSlice = 256;           // columns per CTA, 8 per lane
constexpr int kEmZeroBytes = 131072, kEmZeroLeast = 4096;       // of dW per CTA that zeroes, about: at most, at least

// A lane's 8 columns of a row of d_out, 8 * lane and on, as they lie: in whole 16-byte pieces, or anywhere.  Lanes behind the last column take the
// first ones, which nobody looks at.
template <typename T, bool VEC> struct EmRow {
    uint4 q[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* row, int lane, int columns, bool) {
        const T* at = row + (lane * 8 < columns ? lane * 8 : 0);
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) q[j] = __ldg((const uint4*)at + j);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        T e[8];
        memcpy(e, q, sizeof(e));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f(e[i]);
    }
};
template <typename T> struct EmRow<T, false> {
    Any8<T> raw;
    // inner: whatever lies around a row's elements belongs to the tensor
    __device__ __forceinline__ void load(const T* row, int lane, int columns, bool inner) {
        const int c = lane * 8 < columns ? lane * 8 : 0;
        if (inner) {
            raw.load(row + c);
        } else {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c + i < columns ? __ldg(row + c + i) : T(0.f);
            memcpy(raw.q, e, sizeof(e));
            raw.s = 0;
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const { raw.get(x); }
};

// A row of dW from a warp's columns, 8 to a lane.  One that starts anywhere is written in whole 16-byte pieces, too, put together from a lane's
// own values and the last ones of the lane before; element by element at its ends.
template <typename T, bool VEC>
__device__ __forceinline__ void put_row(T* at, int lane, int columns, const float (&x)[8], float scale) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * scale;
    if constexpr (VEC) {
        if (lane * 8 < columns) store8(at + lane * 8, y);
        return;
    }
    const int s = (int)((uintptr_t)at & 15) / (int)sizeof(T);       // column c of this lane goes to the pieces that begin at column 8 * lane - s
    T e[8];                                                         // columns 8 * lane - s and on
    if constexpr (sizeof(T) == 2) {
        unsigned w[9];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 two = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
            memcpy(&w[4 + i], &two, 4);
            w[i] = __shfl_up_sync(~0u, w[4 + i], 1);
        }
        w[8] = 0;
        const int from = 8 - s;             // of the 16 values: 1 .. 8
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = from & 2 ? w[i + 1] : w[i];
#pragma unroll
        for (int i = 0; i < 7; ++i) w[i] = from & 4 ? w[i + 2] : w[i];
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = from & 8 ? w[i + 4] : w[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = from & 1 ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
        memcpy(e, w, sizeof(e));
    } else {
        float z[11];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[3 + i] = y[i];
#pragma unroll
        for (int i = 0; i < 3; ++i) z[i] = __shfl_up_sync(~0u, y[5 + i], 1);
        const int from = 3 - s;             // of the 11 values: 0 .. 3
#pragma unroll
        for (int i = 0; i < 10; ++i) z[i] = from & 1 ? z[i + 1] : z[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = from & 2 ? z[i + 2] : z[i];
        memcpy(e, z, sizeof(e));
    }
    const int c = lane * 8 - s;
    constexpr int per = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 8; j += per) {
        if (c + j >= 0 && c + j + per <= columns) {
            uint4 q;
            memcpy(&q, e + j, 16);
            *(uint4*)(at + c + j) = q;
        } else {
#pragma unroll
            for (int i = j; i < j + per; ++i)
                if (c + i >= 0 && c + i < columns) at[c + i] = e[i];
        }
    }
    if (lane == 31)                         // what is left behind the last pieces
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (8 - i <= s && lane * 8 + i < columns) from_f(y[i], at + lane * 8 + i);
}

// What a warp leaves of the runs at the ends of its tile: the ids, and whether the places before and behind the tile belong to them.
struct EmEnds { int first, last; bool before, behind; };

template <typename TW, typename TO, bool VEC>
__global__ void __launch_bounds__(kEmSumWarps * 32, sizeof(TO) == 4 ? 2 : VEC ? 4 : 3) embed_sum_kernel(EmParams p) {
    __shared__ float part[kEmSumWarps][2][kEmSlice];        // sums of runs that go on before the warp's tile, and of those that begin in it and go on behind
    __shared__ EmEnds ends[kEmSumWarps];
    constexpr int kEmAhead = 4;             // rows of d_out on their way per warp
    pdl_start();
    pdl_wait();
    const int2* list = p.list[p.sorted];        // written while this kernel may have started: never through the read-only path (__ldg)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, M = (int)p.M, vocab = (int)p.vocab;
    // the CTAs that zero stand evenly between those that sum: reading and writing at the same time is the faster way
    const unsigned zero_before = (unsigned)((unsigned long long)blockIdx.x * p.zero_ctas / gridDim.x);
    const bool zero = (unsigned long long)(blockIdx.x + 1) * p.zero_ctas / gridDim.x > zero_before;
    if (!zero) {
        const unsigned work = blockIdx.x - zero_before;
        const int tile = (int)(work / (unsigned)p.slices), c0 = (int)(work - (unsigned)tile * p.slices) * kEmSlice, columns = min(kEmSlice, p.D - c0);
        const TO* d_out = (const TO*)p.d_out + c0;
        TW* dw = (TW*)p.out + c0;
        const bool wide = p.D >= 16;            // a row before and one behind hold the pieces around a row's ends
        const int a = (tile * kEmSumWarps + warp) * p.warp_tile, n = min(p.warp_tile, M - a);
        EmEnds me{vocab, vocab, false, false};
        if (n > 0) {
            const int2 mine = lane < n ? list[a + lane] : make_int2(vocab, 0);
            const int my_key = mine.x, my_src = mine.y;
            const int prev = a > 0 ? list[a - 1].x : -1, next = a + n < M ? list[a + n].x : -1;
            me.first = __shfl_sync(~0u, my_key, 0);
            me.last = __shfl_sync(~0u, my_key, n - 1);
            me.before = me.first < vocab && prev == me.first;
            me.behind = me.last < vocab && next == me.last;
            if (me.first < vocab) {
                const int real = __popc(__ballot_sync(~0u, my_key < vocab));        // places that count come first
                float acc[8] = {};
                int run = me.first;
                bool open = me.before;              // the run began before the tile
                const auto keep = [&](int slot) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) part[warp][slot][lane * 8 + i] = acc[i];
                };
                for (int r = 0; r < real; r += kEmAhead) {
                    EmRow<TO, VEC> x[kEmAhead];
#pragma unroll
                    for (int j = 0; j < kEmAhead; ++j) {
                        const int row = __shfl_sync(~0u, my_src, r + j < real ? r + j : 0);
                        x[j].load(d_out + (long long)row * p.D, lane, columns, wide && row > 0 && row + 1 < (int)p.rows);
                    }
#pragma unroll
                    for (int j = 0; j < kEmAhead; ++j) {
                        const int key = __shfl_sync(~0u, my_key, (r + j) & 31);
                        if (r + j >= real) break;
                        if (key != run) {
                            if (open) keep(0);
                            else put_row<TW, VEC>(dw + (long long)run * p.D, lane, columns, acc, p.scale);
                            open = false;
                            run = key;
#pragma unroll
                            for (int i = 0; i < 8; ++i) acc[i] = 0.f;
                        }
                        float v[8];
                        x[j].get(v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[i] += v[i];
                    }
                }
                if (open) keep(0);
                else if (me.behind) keep(1);
                else put_row<TW, VEC>(dw + (long long)run * p.D, lane, columns, acc, p.scale);
            }
        }
        if (lane == 0) ends[warp] = me;
        __syncthreads();
        // runs over several warps, in the warps' order: a column per thread
        const int c = threadIdx.x;
        float sum = 0.f;
        bool from_before = false, open = false;
        for (int w = 0; w < kEmSumWarps; ++w) {
            const EmEnds e = ends[w];
            const bool one = e.first == e.last;
            if (e.before) {
                if (w == 0) from_before = true;
                sum += part[w][0][c];
                open = one && e.behind;
                if (!open) {
                    if (c < columns) {
                        if (from_before) p.part[(long long)tile * 2 * p.D + c0 + c] = sum;
                        else from_f(sum * p.scale, dw + (long long)e.first * p.D + c);
                    }
                    from_before = false;
                    sum = 0.f;
                }
            }
            if (e.behind && !(one && e.before)) {
                sum = part[w][1][c];
                open = true;
            }
        }
        if (open && c < columns) p.part[((long long)tile * 2 + (from_before ? 0 : 1)) * p.D + c0 + c] = sum;
        return;
    }
    // rows of ids that occur nowhere, in 16-byte pieces of dW as one list of elements, whatever its rows' length
    bool* there = (bool*)part;                              // [zero_rows]
    __shared__ int found[2];
    const long long first = (long long)zero_before * p.zero_rows, end = min(first + p.zero_rows, p.vocab);
    for (int i = threadIdx.x; i < p.zero_rows; i += kEmSumWarps * 32) there[i] = false;
    // the places of these ids in the list: its first place with an id from `first` on, and from `end` on, among 256 probes at a time
    int lo[2] = {0, 0}, hi[2] = {M, M};
    while (lo[0] < hi[0] || lo[1] < hi[1]) {
        __syncthreads();
        if (threadIdx.x < 2) found[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int step = (hi[k] - lo[k] + 255) / 256, i = lo[k] + (int)threadIdx.x * step;
            const unsigned less = __ballot_sync(~0u, i < hi[k] && list[i].x < (k ? end : first));
            if (lane == 0) atomicAdd(&found[k], __popc(less));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {       // the last probe that is less lies before the place, the next one not
            const int step = (hi[k] - lo[k] + 255) / 256, n = found[k];
            hi[k] = min(hi[k], lo[k] + n * step);
            lo[k] = n ? lo[k] + (n - 1) * step + 1 : hi[k];
            if (!n) hi[k] = lo[k] = min(lo[k], hi[k]);
        }
    }
    constexpr int threads = kEmSumWarps * 32;
    const int rows = (int)(end - first), places = lo[1] - lo[0];
    if (places < rows * 128) {          // each place marks its row, 8 loads on their way at once
        for (int i = lo[0] + (int)threadIdx.x; i < lo[1]; i += 8 * threads) {
            int id[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) id[j] = i + j * threads < lo[1] ? list[i + j * threads].x : -1;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (id[j] >= 0) there[id[j] - first] = true;
        }
    } else {                            // few ids in many places: each row looks for one of its own
        for (int r = threadIdx.x; r < rows; r += threads) {
            int a = lo[0], b = lo[1];
            while (a < b) {
                const int mid = (a + b) >> 1;
                if (list[mid].x < first + r) a = mid + 1;
                else b = mid;
            }
            there[r] = a < lo[1] && list[a].x == first + r;
        }
    }
    __syncthreads();
    TW* from = (TW*)p.out + first * p.D;
    constexpr int per = 16 / sizeof(TW);
    const int lead = (int)(((uintptr_t)from & 15) / sizeof(TW)), total = rows * p.D;        // zero_rows * D is below 2^31
    const int row_step = threads * per / p.D, col_step = threads * per - row_step * p.D;
    int i = (int)threadIdx.x * per - lead, row = max(i, 0) / p.D, c = max(i, 0) - row * p.D;
    if (i < 0) {                        // over the start: the elements that are there
        for (int k = 0; k < i + per && k < total; ++k)
            if (!there[k / p.D]) from_f(0.f, from + k);
        i += threads * per;
        row = i / p.D;
        c = i - row * p.D;
    }
    while (i < total) {
        bool none = !there[row], all = !none;           // the rows that the piece lies in: none or all of them have a token
        for (int kr = row + 1, kc = c + per - p.D; kc > 0 && kr < rows; ++kr, kc -= p.D) {
            none = none && !there[kr];
            all = all && there[kr];
        }
        if (none && i + per <= total) {
            *(uint4*)(from + i) = make_uint4(0, 0, 0, 0);
        } else if (!all) {
            for (int k = i, kr = row, kc = c; k < i + per && k < total; ++k, ++kc) {
                while (kc >= p.D) { kc -= p.D; ++kr; }
                if (!there[kr]) from_f(0.f, from + k);
            }
        }
        i += threads * per;
        row += row_step;
        c += col_step;
        if (c >= p.D) { c -= p.D; ++row; }
    }
}

// A run of one id over several CTAs' tiles: the partial rows of its tiles, in order.  One CTA per tile and slice of the columns; all but those
// in whose tile such a run begins end at once.  Four groups of threads take a quarter of the partial rows each.
constexpr int kEmFinishGroups = 4;
template <typename TW>
__global__ void __launch_bounds__(kEmFinishGroups * kEmSlice) embed_finish_kernel(EmParams p) {
    __shared__ float share[kEmFinishGroups][kEmSlice];
    __shared__ int stop;
    pdl_wait();
    const int2* list = p.list[p.sorted];
    const int cta_tile = kEmSumWarps * p.warp_tile, tile = blockIdx.x, first = tile * cta_tile, next = first + cta_tile, M = (int)p.M;
    if (next >= M) return;
    const int key = list[next].x, last_here = list[next - 1].x, first_here = list[first].x, prev = first > 0 ? list[first - 1].x : -1;
    if (key >= (int)p.vocab || last_here != key) return;            // no run of an id goes on
    if (first_here == key && prev == key) return;                   // it began in an earlier tile
    // the first tile behind that does not begin with this id
    int n_tiles = p.sum_tiles;
    for (int t0 = tile + 2; t0 < p.sum_tiles; t0 += kEmFinishGroups * kEmSlice) {
        __syncthreads();
        if (threadIdx.x == 0) stop = p.sum_tiles;
        __syncthreads();
        const int t = t0 + (int)threadIdx.x;
        if (t < p.sum_tiles && list[t * cta_tile].x != key) atomicMin(&stop, t);
        __syncthreads();
        n_tiles = stop;
        if (n_tiles < p.sum_tiles) break;
    }
    const int n = n_tiles - tile;       // slot 1 of the first tile, slot 0 of the others
    const int group = threadIdx.x / kEmSlice, in_slice = threadIdx.x % kEmSlice, c = (int)blockIdx.y * kEmSlice + in_slice;
    const int per = (n + kEmFinishGroups - 1) / kEmFinishGroups, from = min(n, group * per), to = min(n, from + per);
    float sum = 0.f;
    if (c < p.D) {
#pragma unroll 8
        for (int j = from; j < to; ++j) sum += p.part[((long long)(tile + j) * 2 + (j == 0 ? 1 : 0)) * p.D + c];
    }
    share[group][in_slice] = sum;
    __syncthreads();
    if (group == 0 && c < p.D) {
        for (int g = 1; g < kEmFinishGroups; ++g) sum += share[g][in_slice];
        from_f(sum * p.scale, (TW*)p.out + (long long)key * p.D + c);
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
    p.by_D = FastDiv((unsigned)a.D); p.by_tokens = FastDiv((unsigned)std::max<long long>(1, a.tokens)); p.by_out_rows = FastDiv((unsigned)std::max<long long>(1, a.out_rows));
    p.D = a.D; p.id64 = a.id_bytes == 8; p.scale = a.scale;
    return p;
}
bool on_16(const void* q) { return ((uintptr_t)q & 15) == 0; }
bool on_element(const void* q, int bytes) { return ((uintptr_t)q & (bytes - 1)) == 0; }
int bytes_of(bpt_dtype t) { return t == BPT_F32 ? 4 : 2; }

// Whether the current device can run a cluster of 16 CTAs of the sort (8 always fit): asked once per device.
bool wide_clusters() {
    static std::atomic<int> known[64];      // by device ordinal: 0 not asked yet, 1 no, 2 yes
    int device;
    if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); return true; }     // a size query without a device
    if (device < 64 && known[device].load(std::memory_order_acquire)) return known[device].load(std::memory_order_acquire) == 2;
    cudaLaunchAttribute attr[1] = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)kEmClusterCtas, 1, 1};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)kEmClusterCtas);
    cfg.blockDim = dim3(kEmClusterThreads);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    const bool yes = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                     cudaOccupancyMaxActiveClusters(&n, embed_sort_kernel, &cfg) == cudaSuccess && n > 0;
    if (!yes) cudaGetLastError();
    if (device < 64) known[device].store(yes ? 2 : 1, std::memory_order_release);
    return yes;
}

struct EmPlan {
    int passes, digit, sort_tile, sort_tiles, sum_tiles, warp_tile;
    int ctas, rounds;            // of the sort in one launch; 0: it takes a launch or two a pass
    size_t hist, list, part;     // bytes; list: one of two
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
    // places per warp: long tiles leave fewer partial rows, short ones more CTAs to share the work
    const long long slices = (a.D + kEmSlice - 1) / kEmSlice;
    q.warp_tile = 32;
    while (q.warp_tile > 8 && M * slices < kEmSms * kEmSumWarps * q.warp_tile) q.warp_tile /= 2;
    q.sum_tiles = (int)((M + kEmSumWarps * q.warp_tile - 1) / (kEmSumWarps * q.warp_tile));
    const int most_ctas = M > 8 * kEmClusterThreads && wide_clusters() ? kEmClusterCtas : 8;
    if (M > 0 && M <= most_ctas * kEmRounds * kEmClusterThreads) {
        q.ctas = 1;
        while (q.ctas < most_ctas && q.ctas * kEmClusterThreads < M) q.ctas *= 2;
        q.rounds = (int)((M + q.ctas * kEmClusterThreads - 1) / (q.ctas * kEmClusterThreads));
    }
    q.hist = q.ctas ? 0 : (size_t)q.sort_tiles * kEmBins * 4;
    q.list = ((size_t)M * 8 + 15) / 16 * 16;
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

template <typename TW, typename TO, bool VEC>
bool run_sum(EmParams p, cudaStream_t st) {
    p.slices = (p.D + kEmSlice - 1) / kEmSlice;
    // rows per CTA that zeroes: enough to write, and few enough that their marks fit where the sums would be
    const long long row = (long long)sizeof(TW) * p.D, share = p.vocab * row / (2 * kEmSms);
    p.zero_rows = (int)std::min<long long>(4096, std::max<long long>(1, std::min<long long>(kEmZeroBytes, std::max<long long>(kEmZeroLeast, share)) / row));
    p.zero_ctas = (unsigned)((p.vocab + p.zero_rows - 1) / p.zero_rows);
    if (!start(embed_sum_kernel<TW, TO, VEC>, dim3((unsigned)(p.sum_tiles * p.slices) + p.zero_ctas), kEmSumWarps * 32, st, p.sum_tiles == 0, p)) return false;
    trace_mark(st, "embed_sum");
    if (p.sum_tiles < 2) return true;       // no run crosses tiles
    if (!start(embed_finish_kernel<TW>, dim3((unsigned)p.sum_tiles - 1, (unsigned)p.slices), kEmFinishGroups * kEmSlice, st, false, p)) return false;
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
    int lanes = 1;
    while (lanes < a->D / 8 && lanes < 32) lanes *= 2;
    const int rows_per_cta = 256 / lanes * kEmRows;
    const unsigned grid = vec ? (unsigned)(((unsigned long long)p.rows + rows_per_cta - 1) / rows_per_cta)
                         : a->D >= 8 ? (unsigned)(((unsigned long long)p.rows * p.D + 7 + 8 * 256 - 1) / (8 * 256))        // wherever out starts
                                     : (unsigned)(((unsigned long long)p.rows * p.D + 255) / 256);
    typedef __nv_bfloat16 bf;
    const bool wf = a->weight_dtype == BPT_F32, of = a->out_dtype == BPT_F32;
#define BPT_EMBED_FWD(TW, TO) (vec ? start(embed_fwd_kernel<TW, TO>, dim3(grid), 256, st, true, p, lanes) \
                         : a->D >= 8 ? start(embed_fwd_flat_kernel<TW, TO>, dim3(grid), 256, st, true, p) \
                                     : start(embed_fwd_narrow_kernel<TW, TO>, dim3(grid), 256, st, true, p))
    const bool ok = wf ? (of ? BPT_EMBED_FWD(float, float) : BPT_EMBED_FWD(float, bf)) : (of ? BPT_EMBED_FWD(bf, float) : BPT_EMBED_FWD(bf, bf));
#undef BPT_EMBED_FWD
    trace_mark(st, "embed_fwd");
    return ok ? BPT_OK : BPT_ERR_CUDA;
}

extern "C" size_t bpt_embed_bwd_workspace_bytes(const bpt_embed_args* a) {
    if (check_embed(a) != BPT_OK) return 0;
    const EmPlan q = embed_plan(*a);
    return std::max<size_t>(16, q.hist + 2 * q.list + q.part);
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
        p.list[i] = reinterpret_cast<int2*>(at); at += q.list;
    }
    p.part = reinterpret_cast<float*>(at);
    p.sort_tile = q.sort_tile; p.sort_tiles = q.sort_tiles; p.sum_tiles = q.sum_tiles; p.warp_tile = q.warp_tile;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (M > 0 && q.ctas) {
        cudaLaunchAttribute attr[1] = {};
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {(unsigned)q.ctas, 1, 1};
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)q.ctas);
        cfg.blockDim = dim3(kEmClusterThreads);
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, embed_sort_kernel, p, q.passes, q.digit, q.rounds) != cudaSuccess) {
            cudaGetLastError();
            return BPT_ERR_CUDA;
        }
        trace_mark(st, "embed_sort");
        p.sorted = (q.passes - 1) & 1;
    } else if (M > 0) {
        const int bins = 1 << q.digit;
        for (int i = 0; i < q.passes; ++i) {
            const int from = i == 0 ? -1 : (i - 1) & 1, to = i & 1;
            if (!start(embed_hist_kernel, dim3(q.sort_tiles), kEmSortThreads, st, i == 0, p, from, i * q.digit, bins)) return BPT_ERR_CUDA;
            trace_mark(st, "embed_hist");
            if (!start(embed_scatter_kernel, dim3(q.sort_tiles), kEmSortThreads, st, false, p, from, to, i * q.digit, bins)) return BPT_ERR_CUDA;
            trace_mark(st, "embed_scatter");
            p.sorted = to;
        }
    }
    const bool vec = a->D % 8 == 0 && on_16(d_weight) && on_16(d_out);
    typedef __nv_bfloat16 bf;
    const bool wf = a->weight_dtype == BPT_F32, of = a->out_dtype == BPT_F32;
#define BPT_EMBED_SUM(TW, TO) (vec ? run_sum<TW, TO, true>(p, st) : run_sum<TW, TO, false>(p, st))
    const bool ok = wf ? (of ? BPT_EMBED_SUM(float, float) : BPT_EMBED_SUM(float, bf)) : (of ? BPT_EMBED_SUM(bf, float) : BPT_EMBED_SUM(bf, bf));
#undef BPT_EMBED_SUM
    return ok ? BPT_OK : BPT_ERR_CUDA;
}
