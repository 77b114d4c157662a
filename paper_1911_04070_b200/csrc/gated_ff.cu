// Gated feed-forward block (the position-wise half of Algorithm 2, Sec. 3.3 of arXiv 1911.04070, with the gated inner layer
// of current language models in the place of relu):
//     h = act(x Wg^T) * (x Wu^T),    y = h Wd^T,        x [M, D], Wg, Wu [F, D], Wd [D, F], bf16, fp32 accumulation,
// and its backward from x and dy alone:
//     G = x Wg^T, U = x Wu^T, dH = dy Wd            (one kernel: three accumulators, G and U are never stored)
//     dG = dH U act'(G), dU = dH act(G), h = act(G) U
//     dx = dG Wg + dU Wu,   dWg = dG^T x,  dWu = dU^T x,  dWd = dy^T h.
//
// All five products run in one kernel template on pairs of CTAs (pair_tools.cuh): a load warp per CTA brings 64-deep
// slices of both operands in with TMA, one thread of the pair issues tcgen05 products of 256 rows x up to 256 columns,
// eight epilogue warps per CTA take finished accumulators out of tensor memory while the next tile's products run (two
// accumulators of 256 columns; in the three-accumulator kernel dH is double and G | U single, and a tile's dH products
// cover the epilogue of the tile before).  Operands that a product needs transposed are read as they lie: the matrix
// descriptors take either axis as the contiguous one, so no transposed copy exists anywhere.  Ragged edges are TMA's: what lies outside a tensor reads
// as zero and is not written.  Every wait is bounded; a give-up is reported through the status word.
#include <algorithm>

#include "bpt_internal.cuh"
#include "mma_tools.cuh"
#include "pair_tools.cuh"
#include "tc5_host.cuh"

namespace bpt {
namespace {

enum FfKernel { kFfIn, kFfOut, kFfBwdIn, kFfDx, kFfDw };

constexpr int kFfPairs = 74;                  // 148 SMs
constexpr int kFfEpiWarps = 8;
constexpr int kFfThreads = (4 + kFfEpiWarps) * 32;   // load warp, product warp, two idle warps (tensor-memory lane groups start at a multiple of four), epilogue
constexpr int kFfStageBytes = 32 * 1024;      // 128 x 64 of A and up to 128 x 64 of B per CTA
constexpr int kFfK = 64;

template <int KERNEL> struct FfShape {
    static constexpr int stages = KERNEL == kFfBwdIn ? 4 : 5;
    static constexpr int staging = KERNEL == kFfBwdIn ? 3 : 2;      // 4 KB output tiles per epilogue warp
    static constexpr int out_off = stages * kFfStageBytes;
    static constexpr int bar_off = out_off + kFfEpiWarps * staging * 4096;
    static constexpr size_t bytes = bar_off + 256 + 1024;
};

struct FfParams {
    CUtensorMap a0, a1, a2, b0, b1, b2, c0, c1, c2;
    int* status;
    int rows, D, F, splits, tiles;
};

// act(g) and, for the backward, its derivative
template <int ACT, bool GRAD>
__device__ __forceinline__ float ff_act(float g, float& da) {
    if (ACT == BPT_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        if (GRAD) da = s * fmaf(g, 1.f - s, 1.f);
        return g * s;
    }
    if (ACT == BPT_ACT_GELU) {
        const float c = fmaf(0.5f, erff(g * 0.70710678118654752f), 0.5f);
        if (GRAD) da = fmaf(g * 0.39894228040143268f, __expf(-0.5f * g * g), c);
        return g * c;
    }
    if (GRAD) da = g > 0.f ? 1.f : 0.f;
    return g < 0.f ? 0.f : g;
}

// ACT: a choice of the whole launch, where the kernel has an activation.  BN: accumulator columns of a tile (kFfOut, kFfDx; 256 in the others: 128 of G and 128 of U)
template <int KERNEL, int BN, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFfThreads, 1) gated_ff_kernel(const __grid_constant__ FfParams p) {
    using S = FfShape<KERNEL>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // the same offset in both CTAs
    const uint32_t s_u = smem_u32(smem), bar_u = s_u + S::bar_off;
    auto full = [&](int i) { return bar_u + 8u * (uint32_t)i; };
    auto empty = [&](int i) { return bar_u + 8u * (uint32_t)(S::stages + i); };
    auto tfull = [&](int i) { return bar_u + 8u * (uint32_t)(2 * S::stages + i); };
    auto tempty = [&](int i) { return bar_u + 8u * (uint32_t)(2 * S::stages + 2 + i); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::bar_off + 8 * (2 * S::stages + 4));
    volatile int* abort_s = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int rank = (int)pair::cta_rank(), pair_id = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

    if (tid == 0) {
        for (int i = 0; i < 2 * S::stages + 2; ++i) tc5::mbar_init(bar_u + 8u * i, 1);
        for (int i = 0; i < 2; ++i) tc5::mbar_init(tempty(i), 2 * kFfEpiWarps);
        tc5::mbar_init_fence();
        *abort_s = 0;
    }
    __syncwarp();
    if (w == 1) pair::tmem_alloc(smem_u32(tmem_slot), 512);
    tc5::fence_before_sync();
    pair::cluster_sync();
    tc5::fence_after_sync();
    const uint32_t tbase = *tmem_slot;

    const int kd = (p.D + kFfK - 1) / kFfK, kf = (p.F + kFfK - 1) / kFfK, km = (p.rows + kFfK - 1) / kFfK;
    const int n_tiles = KERNEL == kFfOut || KERNEL == kFfDx ? (p.D + BN - 1) / BN : (p.F + 127) / 128;   // along the output's columns
    const int dw_n0 = (p.D + 255) / 256, dw_n1 = (p.F + 255) / 256, dw_tiles = dw_n0 * dw_n1;             // weight gradients, each of the three
    struct Tile { int m, n, k0, k1, job, split; };
    auto tile_of = [&](int t) {
        Tile q{};
        if constexpr (KERNEL == kFfDw) {
            q.split = t / (3 * dw_tiles);
            const int u = t % (3 * dw_tiles), v = u % dw_tiles;
            q.job = u / dw_tiles;
            const int nn = q.job < 2 ? dw_n0 : dw_n1;
            q.m = v / nn * 256; q.n = v % nn * 256;
            q.k0 = (int)((long long)km * q.split / p.splits); q.k1 = (int)((long long)km * (q.split + 1) / p.splits);
        } else {
            q.m = t / n_tiles * 256;
            q.n = t % n_tiles * (KERNEL == kFfOut || KERNEL == kFfDx ? BN : 128);
            q.k1 = KERNEL == kFfIn ? kd : KERNEL == kFfOut ? kf : KERNEL == kFfBwdIn ? 2 * kd : 2 * kf;
        }
        return q;
    };

    if (w == 0 && lane == 0) {
        // =============== load thread ===============
        int it = 0;
        for (int t = pair_id; t < p.tiles && !*abort_s; t += n_pairs) {
            const Tile q = tile_of(t);
            const int m = q.m + rank * 128;
            for (int k = q.k0; k < q.k1; ++k, ++it) {
                const int st = it % S::stages, use = it / S::stages;
                if (use > 0 && !tc5::mbar_wait_idle(empty(st), (use - 1) & 1)) { *abort_s = 1; break; }
                const uint32_t a = s_u + st * kFfStageBytes, b = a + 16384;
                const uint32_t bar = pair::in_first(full(st));
                if constexpr (KERNEL == kFfIn) {
                    if (rank == 0) tc5::mbar_expect_tx(full(st), 2 * 32768);
                    pair::load_2d(a, &p.a0, k * kFfK, m, bar);
                    pair::load_2d(b, rank ? &p.b1 : &p.b0, k * kFfK, q.n, bar);
                } else if constexpr (KERNEL == kFfOut) {
                    if (rank == 0) tc5::mbar_expect_tx(full(st), 2 * (16384 + BN * 64));
                    pair::load_2d(a, &p.a0, k * kFfK, m, bar);
                    pair::load_2d(b, &p.b0, k * kFfK, q.n + rank * (BN / 2), bar);
                } else if constexpr (KERNEL == kFfBwdIn) {
                    if (k < kd) {       // dH: dy rows, Wd with its F axis contiguous
                        if (rank == 0) tc5::mbar_expect_tx(full(st), 2 * 24576);
                        pair::load_2d(a, &p.a1, k * kFfK, m, bar);
                        pair::load_2d(b, &p.b2, q.n + rank * 64, k * kFfK, bar);
                    } else {
                        if (rank == 0) tc5::mbar_expect_tx(full(st), 2 * 32768);
                        pair::load_2d(a, &p.a0, (k - kd) * kFfK, m, bar);
                        pair::load_2d(b, rank ? &p.b1 : &p.b0, (k - kd) * kFfK, q.n, bar);
                    }
                } else if constexpr (KERNEL == kFfDx) {
                    if (rank == 0) tc5::mbar_expect_tx(full(st), 2 * (16384 + BN * 64));
                    const bool second = k >= kf;
                    const int kk = (second ? k - kf : k) * kFfK;
                    pair::load_2d(a, second ? &p.a1 : &p.a0, kk, m, bar);
#pragma unroll
                    for (int j = 0; j < BN / 128; ++j) pair::load_2d(b + j * 8192, second ? &p.b1 : &p.b0, q.n + rank * (BN / 2) + j * 64, kk, bar);
                } else {
                    if (rank == 0) tc5::mbar_expect_tx(full(st), 2 * 32768);
                    const CUtensorMap* ma = q.job == 0 ? &p.a0 : q.job == 1 ? &p.a1 : &p.a2;
                    const CUtensorMap* mb = q.job < 2 ? &p.b0 : &p.b1;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        pair::load_2d(a + j * 8192, ma, m + j * 64, k * kFfK, bar);
                        pair::load_2d(b + j * 8192, mb, q.n + rank * 128 + j * 64, k * kFfK, bar);
                    }
                }
            }
        }
        // the releases of the last slices still arrive in this CTA's shared memory: see them in before it ends
        for (int j = it > S::stages ? it - S::stages : 0; j < it && !*abort_s; ++j)
            if (!tc5::mbar_wait_idle(empty(j % S::stages), (j / S::stages) & 1)) *abort_s = 1;
        if (*abort_s) {   // copies still in flight land before the CTA ends (their barrier may be the other CTA's: give them time)
            const long long start = clock64();
            while (clock64() - start < (1ll << 22)) {}
        }
    } else if (w == 1 && lane == 0 && rank == 0) {
        // =============== product thread ===============
        constexpr bool a_mn = KERNEL == kFfDw, b_mn = KERNEL == kFfDw || KERNEL == kFfDx;
        const uint32_t idesc = tc5::instr_desc(256, BN, a_mn, b_mn), idesc_dh = tc5::instr_desc(256, 128, 0, 1);
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (*abort_s) return;
            if (!pair::wait_cluster(bar, parity)) *abort_s = 1;
        };
        int it = 0, i = 0;
        for (int t = pair_id; t < p.tiles && !*abort_s; t += n_pairs, ++i) {
            const Tile q = tile_of(t);
            // an accumulator is free again when the epilogue of the tile two before has taken it out
            if (i >= 2) wait(tempty(i & 1), (i / 2 - 1) & 1);
            tc5::fence_after_sync();
            uint32_t acc = tbase + (KERNEL == kFfBwdIn ? 256u + (i & 1) * 128u : (i & 1) * 256u);
            for (int k = q.k0; k < q.k1; ++k, ++it) {
                const int st = it % S::stages;
                if constexpr (KERNEL == kFfBwdIn) {
                    if (k == kd) {      // G | U have one place: the tile before has to be out
                        if (i >= 1) wait(tempty((i - 1) & 1), ((i - 1) / 2) & 1);
                        tc5::fence_after_sync();
                        acc = tbase;
                    }
                }
                wait(full(st), (it / S::stages) & 1);
                if (*abort_s) break;
                tc5::fence_after_sync();
                const uint32_t a = s_u + st * kFfStageBytes, b = a + 16384;
                const bool dh = KERNEL == kFfBwdIn && k < kd;
                const uint32_t a_lo = a_mn ? pair::desc_lo_mn(a) : tc5::desc_lo_k_major(a);
                const uint32_t b_lo = b_mn || dh ? pair::desc_lo_mn(b) : tc5::desc_lo_k_major(b);
                const uint32_t b_step = b_mn || dh ? 2048 / 16 : 2, a_step = a_mn ? 2048 / 16 : 2;
                const bool first = k == q.k0 || (KERNEL == kFfBwdIn && k == kd);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    pair::mma(acc, a_lo + ks * a_step, b_lo + ks * b_step, dh ? idesc_dh : idesc, (first && ks == 0) ? 0u : 1u);
                pair::commit_both(empty(st));
            }
            if (*abort_s) break;
            pair::commit_both(tfull(i & 1));
        }
    } else if (w >= 4) {
        // =============== epilogue warps: 32 rows (tensor-memory lanes) x half of the tile's columns each ===============
        const int quad = w & 3, half = (w - 4) >> 2;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        unsigned char* stg = smem + S::out_off + (w - 4) * S::staging * 4096;
        const uint32_t stg_u = smem_u32(stg), release[2] = {pair::in_first(tempty(0)), pair::in_first(tempty(1))};
        // 16 bytes of this thread's row of staging tile `buf`
        auto put = [&](int buf, int chunk, uint32_t x, uint32_t y, uint32_t z, uint32_t v) {
            *reinterpret_cast<uint4*>(stg + buf * 4096 + tile_off(lane, chunk)) = make_uint4(x, y, z, v);
        };
        int i = 0;
        for (int t = pair_id; t < p.tiles; t += n_pairs, ++i) {
            const Tile q = tile_of(t);
            const bool ok = !*abort_s && tc5::mbar_wait_fast(tfull(i & 1), (i / 2) & 1);
            if (!__all_sync(0xffffffffu, ok)) { *abort_s = 1; break; }      // the whole warp together
            tc5::fence_after_sync();
            const int row = q.m + rank * 128 + quad * 32;
            auto done = [&] {           // this warp has taken the accumulator out
                tc5::fence_before_sync();
                __syncwarp();
                if (lane == 0) pair::arrive_cluster(release[i & 1]);
            };
            auto send = [&](const CUtensorMap* map, int buf, int col, int limit_cols, int limit_rows) {
                tc5::fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (col < limit_cols && row < limit_rows) {
                        if constexpr (KERNEL == kFfDw) pair::store_3d(map, col, row, q.job == 1 ? p.splits + q.split : q.split, stg_u + buf * 4096);
                        else pair::store_2d(map, col, row, stg_u + buf * 4096);
                    }
                    pair::store_commit();
                }
            };
            if constexpr (KERNEL == kFfIn) {
                const uint32_t src = tbase + lane_base + (i & 1) * 256 + half * 64;
                if (lane == 0) pair::store_wait_read<1>();
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
                    uint32_t g[32], u[32];
                    tc5::tmem_ld32(src + c, g);
                    tc5::tmem_ld32(src + 128 + c, u);
                    tc5::tmem_ld_wait();
                    if (c == 32) done();
                    float unused;
#pragma unroll
                    for (int j = 0; j < 32; ++j) g[j] = __float_as_uint(ff_act<ACT, false>(__uint_as_float(g[j]), unused) * __uint_as_float(u[j]));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t x[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y) x[y] = pack_bf16(__uint_as_float(g[j * 8 + 2 * y]), __uint_as_float(g[j * 8 + 2 * y + 1]));
                        put(i & 1, c / 8 + j, x[0], x[1], x[2], x[3]);
                    }
                }
                send(&p.c0, i & 1, q.n + half * 64, p.F, p.rows);
            } else if constexpr (KERNEL == kFfBwdIn) {
                const uint32_t src = tbase + lane_base + half * 64, src_dh = src + 256 + (i & 1) * 128;
                if (lane == 0) pair::store_wait_read<0>();
                __syncwarp();
#pragma unroll 1
                for (int c = 0; c < 64; c += 16) {
                    uint32_t g[16], u[16], dh[16];
                    tc5::tmem_ld16(src + c, g);
                    tc5::tmem_ld16(src + 128 + c, u);
                    tc5::tmem_ld16(src_dh + c, dh);
                    tc5::tmem_ld_wait();
                    if (c == 48) done();
                    uint32_t og[8], ou[8], oh[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float r[3][2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float gv = __uint_as_float(g[2 * j + e]), uv = __uint_as_float(u[2 * j + e]), dv = __uint_as_float(dh[2 * j + e]);
                            float da;
                            const float a = ff_act<ACT, true>(gv, da);
                            r[0][e] = dv * uv * da;
                            r[1][e] = dv * a;
                            r[2][e] = a * uv;
                        }
                        og[j] = pack_bf16(r[0][0], r[0][1]);
                        ou[j] = pack_bf16(r[1][0], r[1][1]);
                        oh[j] = pack_bf16(r[2][0], r[2][1]);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        put(0, c / 8 + j, og[4 * j], og[4 * j + 1], og[4 * j + 2], og[4 * j + 3]);
                        put(1, c / 8 + j, ou[4 * j], ou[4 * j + 1], ou[4 * j + 2], ou[4 * j + 3]);
                        put(2, c / 8 + j, oh[4 * j], oh[4 * j + 1], oh[4 * j + 2], oh[4 * j + 3]);
                    }
                }
                send(&p.c0, 0, q.n + half * 64, p.F, p.rows);
                send(&p.c1, 1, q.n + half * 64, p.F, p.rows);
                send(&p.c2, 2, q.n + half * 64, p.F, p.rows);
            } else if constexpr (KERNEL == kFfDw) {
                const uint32_t src = tbase + lane_base + (i & 1) * 256 + half * 128;
                const CUtensorMap* map = q.job < 2 ? &p.c0 : &p.c1;
                const int limit_cols = q.job < 2 ? p.D : p.F, limit_rows = q.job < 2 ? p.F : p.D;
#pragma unroll
                for (int c = 0; c < 128; c += 32) {
                    uint32_t x[32];
                    tc5::tmem_ld32(src + c, x);
                    tc5::tmem_ld_wait();
                    if (c == 96) done();
                    if (lane == 0) pair::store_wait_read<1>();
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) put((c / 32) & 1, j, x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                    send(map, (c / 32) & 1, q.n + half * 128 + c, limit_cols, limit_rows);
                }
            } else {
                constexpr int W = BN / 2 < 64 ? BN / 2 : 64;      // columns per stored tile
                const uint32_t src = tbase + lane_base + (i & 1) * 256 + half * (BN / 2);
#pragma unroll
                for (int c = 0; c < BN / 2; c += 32) {
                    uint32_t x[32];
                    tc5::tmem_ld32(src + c, x);
                    tc5::tmem_ld_wait();
                    if (c + 32 == BN / 2) done();
                    const int buf = (i * (BN / 2 / W) + c / W) & 1;
                    if (c % W == 0) {
                        if (lane == 0) pair::store_wait_read<1>();
                        __syncwarp();
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = pack_bf16(__uint_as_float(x[j * 8 + 2 * e]), __uint_as_float(x[j * 8 + 2 * e + 1]));
                        if constexpr (W == 64) put(buf, (c & 32) / 8 + j, y[0], y[1], y[2], y[3]);
                        else *reinterpret_cast<uint4*>(stg + buf * 4096 + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                    if (c % W + 32 == W) send(&p.c0, buf, q.n + half * (BN / 2) + c / W * W, p.D, p.rows);
                }
            }
        }
        if (lane == 0) pair::store_wait<0>();
    }

    __syncwarp();
    tc5::fence_before_sync();
    pair::cluster_sync();      // both CTAs are past their last product, load and barrier use
    if (tid == 0 && *abort_s && p.status) p.status[0] = (int)BPT_ERR_TIMEOUT;
    if (w == 1) pair::tmem_free(tbase, 512);
}

// Weight gradients: the fp32 sums of the row ranges, added in order, rounded once.
__global__ void __launch_bounds__(256) gated_ff_dw_sum_kernel(const float* __restrict__ part, __nv_bfloat16* __restrict__ dwg,
                                                              __nv_bfloat16* __restrict__ dwu, __nv_bfloat16* __restrict__ dwd, long long n, int splits) {
    const long long n8 = n / 8;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < 3 * n8; i += gridDim.x * 256ll) {
        const int job = (int)(i / n8);
        const long long e = (i % n8) * 8;
        const float* src = part + (long long)job * splits * n + e;
        float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
        for (int s = 1; s < splits; ++s) {
            const float4 c = *reinterpret_cast<const float4*>(src + s * n), d = *reinterpret_cast<const float4*>(src + s * n + 4);
            a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
            b.x += d.x; b.y += d.y; b.z += d.z; b.w += d.w;
        }
        __nv_bfloat16* out = (job == 0 ? dwg : job == 1 ? dwu : dwd) + e;
        *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
    }
}

// 2-D map over a row-major [n_rows, n_cols] bf16 matrix, boxes of box_rows x box_cols.
bool bf16_map(CUtensorMap* m, const void* base, long long n_rows, int n_cols, int box_rows, int box_cols = 64) {
    const cuuint64_t dims[2] = {(cuuint64_t)n_cols, (cuuint64_t)n_rows};
    const cuuint64_t strides[1] = {(cuuint64_t)n_cols * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return tc5::encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 3-D map over [n_mats, n_rows, n_cols] fp32, boxes of 32 x 32.
bool part_map(CUtensorMap* m, void* base, int n_mats, int n_rows, int n_cols) {
    const cuuint64_t dims[3] = {(cuuint64_t)n_cols, (cuuint64_t)n_rows, (cuuint64_t)n_mats};
    const cuuint64_t strides[2] = {(cuuint64_t)n_cols * 4, (cuuint64_t)n_rows * n_cols * 4};
    const cuuint32_t box[3] = {32, 32, 1}, estr[3] = {1, 1, 1};
    return tc5::encode_tiled()(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KERNEL, int BN, int ACT = BPT_ACT_RELU>
bpt_status run(const FfParams& p, cudaStream_t st, const char* name) {
    constexpr size_t smem = FfShape<KERNEL>::bytes;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    if (cudaFuncSetAttribute(gated_ff_kernel<KERNEL, BN, ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return BPT_ERR_CUDA;
    gated_ff_kernel<KERNEL, BN, ACT><<<2 * std::min(p.tiles, kFfPairs), kFfThreads, smem, st>>>(p);
    trace_mark(st, name);
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}

template <int KERNEL>
bpt_status run_act(const FfParams& p, int act, cudaStream_t st, const char* name) {
    return act == BPT_ACT_RELU ? run<KERNEL, 256, BPT_ACT_RELU>(p, st, name) : act == BPT_ACT_SILU ? run<KERNEL, 256, BPT_ACT_SILU>(p, st, name)
                                                                                                  : run<KERNEL, 256, BPT_ACT_GELU>(p, st, name);
}

constexpr size_t kStatusBytes = 256;
size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Row ranges of the weight-gradient products: as many as make whole rounds of the pairs, each at least eight slices deep.
int dw_splits(long long rows, int D, int F) {
    const long long tiles = 3ll * ((D + 255) / 256) * ((F + 255) / 256), km = (rows + kFfK - 1) / kFfK;
    int best = 1;
    double cost = 1e30;
    for (int s = 1; s <= 16 && (s == 1 || km / s >= 8); ++s) {
        const double rounds = (double)((tiles * s + kFfPairs - 1) / kFfPairs);
        const double c = rounds * ((double)km / s + 6.0) + 0.35 * tiles * s / kFfPairs;   // slices per pair, a tile's fixed cost, and the sums written
        if (c < cost - 1e-9) { cost = c; best = s; }
    }
    return best;
}

bpt_status check_ff(int64_t rows, int32_t D, int32_t F, int32_t act) {
    if (rows < 0 || D < 1 || F < 1 || act < BPT_ACT_RELU || act > BPT_ACT_GELU) return BPT_ERR_INVALID_ARG;
    if (D % 8 || F % 8 || rows > (1 << 26) || D > 32768 || F > 131072) return BPT_ERR_UNSUPPORTED;
    return BPT_OK;
}
bool aligned16(std::initializer_list<const void*> ptrs) {
    for (const void* q : ptrs)
        if ((uintptr_t)q & 15) return false;
    return true;
}
// Tiles of `bn` columns: fewer columns per tile while the pairs have less than one tile each.
int out_columns(long long rows, int D, int least) {
    int bn = 256;
    while (bn > least && (rows + 255) / 256 * ((D + bn - 1) / bn) * 2 <= kFfPairs) bn /= 2;
    return bn;
}

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" size_t bpt_gated_ff_workspace_bytes(int64_t rows, int32_t D, int32_t F, int backward) {
    if (check_ff(rows, D, F, BPT_ACT_RELU) != BPT_OK || rows == 0) return 0;
    const size_t hidden = round256((size_t)rows * F * 2);
    if (!backward) return hidden;
    return 3 * hidden + (size_t)3 * dw_splits(rows, D, F) * D * F * 4;
}

extern "C" bpt_status bpt_gated_ff_fwd(const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y, int64_t rows,
                                       int32_t D, int32_t F, int32_t act, void* status, void* workspace, size_t workspace_bytes,
                                       void* cuda_stream) {
    const bpt_status s = check_ff(rows, D, F, act);
    if (s != BPT_OK) return s;
    if (rows == 0) return !status || cudaMemsetAsync(status, 0, kStatusBytes, (cudaStream_t)cuda_stream) == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
    if (!x || !w_gate || !w_up || !w_down || !y || !aligned16({x, w_gate, w_up, w_down, y})) return BPT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < bpt_gated_ff_workspace_bytes(rows, D, F, 0)) return BPT_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255) return BPT_ERR_INVALID_ARG;
    if (!tc5::encode_tiled()) return BPT_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (status && cudaMemsetAsync(status, 0, kStatusBytes, st) != cudaSuccess) return BPT_ERR_CUDA;
    void* h = workspace;
    FfParams p{};
    p.status = static_cast<int*>(status);
    p.rows = (int)rows; p.D = D; p.F = F;
    if (!bf16_map(&p.a0, x, rows, D, 128) || !bf16_map(&p.b0, w_gate, F, D, 128) || !bf16_map(&p.b1, w_up, F, D, 128) ||
        !bf16_map(&p.c0, h, rows, F, 32))
        return BPT_ERR_CUDA;
    const int mt = (int)((rows + 255) / 256);
    p.tiles = mt * ((F + 127) / 128);
    bpt_status e = run_act<kFfIn>(p, act, st, "gated_ff_in");
    if (e != BPT_OK) return e;
    const int bn = out_columns(rows, D, 64);
    if (!bf16_map(&p.a0, h, rows, F, 128) || !bf16_map(&p.b0, w_down, D, F, bn / 2) || !bf16_map(&p.c0, y, rows, D, 32, bn == 64 ? 32 : 64))
        return BPT_ERR_CUDA;
    p.tiles = mt * ((D + bn - 1) / bn);
    return bn == 256 ? run<kFfOut, 256>(p, st, "gated_ff_out") : bn == 128 ? run<kFfOut, 128>(p, st, "gated_ff_out") : run<kFfOut, 64>(p, st, "gated_ff_out");
}

extern "C" bpt_status bpt_gated_ff_bwd(const void* x, const void* w_gate, const void* w_up, const void* w_down, const void* dy, void* dx,
                                       void* dw_gate, void* dw_up, void* dw_down, int64_t rows, int32_t D, int32_t F, int32_t act,
                                       void* status, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const bpt_status s = check_ff(rows, D, F, act);
    if (s != BPT_OK) return s;
    const bool weights = dw_gate || dw_up || dw_down;
    if (weights && !(dw_gate && dw_up && dw_down)) return BPT_ERR_INVALID_ARG;
    if (!aligned16({x, w_gate, w_up, w_down, dy, dx, dw_gate, dw_up, dw_down})) return BPT_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) {
        if (status && cudaMemsetAsync(status, 0, kStatusBytes, st) != cudaSuccess) return BPT_ERR_CUDA;
        if (weights)
            for (void* q : {dw_gate, dw_up, dw_down})
                if (cudaMemsetAsync(q, 0, (size_t)D * F * 2, st) != cudaSuccess) return BPT_ERR_CUDA;
        return BPT_OK;
    }
    if (!x || !w_gate || !w_up || !w_down || !dy || (!dx && !weights)) return BPT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < bpt_gated_ff_workspace_bytes(rows, D, F, 1)) return BPT_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255) return BPT_ERR_INVALID_ARG;
    if (!tc5::encode_tiled()) return BPT_ERR_CUDA;
    if (status && cudaMemsetAsync(status, 0, kStatusBytes, st) != cudaSuccess) return BPT_ERR_CUDA;
    const size_t hidden = round256((size_t)rows * F * 2);
    char* dg = static_cast<char*>(workspace);
    char *du = dg + hidden, *h = du + hidden;
    float* part = reinterpret_cast<float*>(h + hidden);
    const int mt = (int)((rows + 255) / 256);
    FfParams p{};
    p.status = static_cast<int*>(status);
    p.rows = (int)rows; p.D = D; p.F = F;
    if (!bf16_map(&p.a0, x, rows, D, 128) || !bf16_map(&p.a1, dy, rows, D, 128) || !bf16_map(&p.b0, w_gate, F, D, 128) ||
        !bf16_map(&p.b1, w_up, F, D, 128) || !bf16_map(&p.b2, w_down, D, F, 64) || !bf16_map(&p.c0, dg, rows, F, 32) ||
        !bf16_map(&p.c1, du, rows, F, 32) || !bf16_map(&p.c2, h, rows, F, 32))
        return BPT_ERR_CUDA;
    p.tiles = mt * ((F + 127) / 128);
    bpt_status e = run_act<kFfBwdIn>(p, act, st, "gated_ff_bwd_in");
    if (e != BPT_OK) return e;
    if (dx) {
        const int bn = out_columns(rows, D, 128);
        if (!bf16_map(&p.a0, dg, rows, F, 128) || !bf16_map(&p.a1, du, rows, F, 128) || !bf16_map(&p.b0, w_gate, F, D, 64) ||
            !bf16_map(&p.b1, w_up, F, D, 64) || !bf16_map(&p.c0, dx, rows, D, 32))
            return BPT_ERR_CUDA;
        p.tiles = mt * ((D + bn - 1) / bn);
        e = bn == 256 ? run<kFfDx, 256>(p, st, "gated_ff_dx") : run<kFfDx, 128>(p, st, "gated_ff_dx");
        if (e != BPT_OK) return e;
    }
    if (weights) {
        p.splits = dw_splits(rows, D, F);
        if (!bf16_map(&p.a0, dg, rows, F, 64) || !bf16_map(&p.a1, du, rows, F, 64) || !bf16_map(&p.a2, dy, rows, D, 64) ||
            !bf16_map(&p.b0, x, rows, D, 64) || !bf16_map(&p.b1, h, rows, F, 64) || !part_map(&p.c0, part, 2 * p.splits, F, D) ||
            !part_map(&p.c1, part + (size_t)2 * p.splits * D * F, p.splits, D, F))
            return BPT_ERR_CUDA;
        p.tiles = 3 * ((D + 255) / 256) * ((F + 255) / 256) * p.splits;
        e = run<kFfDw, 256>(p, st, "gated_ff_dw");
        if (e != BPT_OK) return e;
        const long long n = (long long)D * F;
        gated_ff_dw_sum_kernel<<<(unsigned)std::min<long long>((3 * n / 8 + 255) / 256, 148 * 8), 256, 0, st>>>(
            part, (__nv_bfloat16*)dw_gate, (__nv_bfloat16*)dw_up, (__nv_bfloat16*)dw_down, n, p.splits);
        trace_mark(st, "gated_ff_dw_sum");
    }
    return cudaGetLastError() == cudaSuccess ? BPT_OK : BPT_ERR_CUDA;
}
