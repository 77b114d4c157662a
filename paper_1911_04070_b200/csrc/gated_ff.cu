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
// eight or sixteen epilogue warps per CTA take finished accumulators out of tensor memory while the next tile's products run: two
// accumulators of 256 columns, in the three-accumulator kernel one for G | U of 128 columns and one for dH of 256 (a tile is
// G | U of its first half, dH, G | U of its second half).  Operands that a product needs transposed are read as they lie: the matrix
// descriptors take either axis as the contiguous one, so no transposed copy exists anywhere.  Ragged edges are TMA's: what lies
// outside a tensor reads as zero and is not written.  Every wait is bounded; a give-up is reported through the call's status word,
// if there is one, and the device's record (bpt_check_device), which a backward pass run by autograd has to rely on.
#include <algorithm>

#include "bpt_internal.cuh"
#include "ff_act.cuh"
#include "gated_ff_rows.cuh"
#include "mma_tools.cuh"
#include "pair_tools.cuh"
#include "tc5_host.cuh"

namespace bpt {
namespace {

// ..Split: the sum's range shared out, fp32 results.  kFfBwdInTwo: for few rows, results as two bf16 terms (value and remainder,
// the remainders kFfTwoRows rows further on), which the products after it take one after the other.
enum FfKernel { kFfIn, kFfOut, kFfBwdIn, kFfDx, kFfDw, kFfOutSplit, kFfDxSplit, kFfBwdInTwo };
constexpr int kFfTwoRows = 64;                // one slice of the weight gradients

constexpr int kFfPairs = 74;                  // 148 SMs
constexpr int kFfStageBytes = 32 * 1024;      // 128 x 64 of A and up to 128 x 64 of B per CTA
constexpr int kFfK = 64;

// The kernels with an activation have sixteen epilogue warps (four per 32 rows, 32 columns each): a warp takes its share of
// G and U into registers at once and gives the accumulator back before it computes.  The others have eight.  All results
// leave through small staged tiles and TMA stores; storing the inner rows straight from registers (a 32-byte sector per
// thread) freed shared memory for two more stages but held the warps longer: 232 against 214 us in the first kernel,
// 441 against 418 us in the three-accumulator one (65532 x 512, F = 2048, silu).
template <int KERNEL> struct FfShape {
    static constexpr bool act = KERNEL == kFfIn || KERNEL == kFfBwdIn || KERNEL == kFfBwdInTwo;
    static constexpr int epi_warps = act ? 16 : 8;
    static constexpr int threads = (2 + epi_warps) * 32;            // load warp, product warp, epilogue warps
    static constexpr int stages = 5;
    static constexpr int tile_bytes = act ? 2048 : 4096;            // a staged output tile: 32 rows of 64 or 128 bytes
    static constexpr int staging = 2;                               // staged tiles per epilogue warp
    static constexpr int out_off = stages * kFfStageBytes;
    static constexpr int bar_off = out_off + epi_warps * staging * tile_bytes;
    static constexpr size_t bytes = bar_off + 256 + 1024;
};

struct FfParams {
    CUtensorMap a0, a1, a2, b0, b1, b2, c0, c1, c2;
    int *status, *record;
    int rows, D, F, splits, tiles;
    int step;               // kFfBwdIn: columns of a tile, 256 or 128 (its first half only)
    bool clear;             // the call's first kernel clears the status block
    bool two;               // dG, dU and h are two terms
};

// The load thread of a CTA and the product thread of a pair go through the same slices: 64 deep, `STAGES` places in shared
// memory, A first, B 16 KB behind it.  What they do per slice is on the critical path (one slice is 512 cycles of products, and the
// warps next to them are busy), hence no divisions and no shared flags in here.
template <int STAGES> struct FfLoader {
    uint32_t s_u, full_first, full_own, empty_own;      // barriers of place 0; full_first: the pair's first CTA's, cluster address
    bool lead;
    int st = 0;
    uint32_t ph = 0;
    bool ok = true;

    // Slices [k0, k1) of this CTA's 128 rows (columns, if *_MN: the matrix lies with that axis contiguous) from row am of A, and of
    // its B_BYTES / 128 rows from row bn of B.  a_k, b_k: from one slice to the next (0: the same slice each time).
    template <bool A_MN, bool B_MN, int B_BYTES>
    __device__ __forceinline__ void slices(int k0, int k1, const CUtensorMap* ma, int am, const CUtensorMap* mb, int bn, int a_k = kFfK, int b_k = kFfK) {
        for (int k = k0; k < k1; ++k) {
            if (!ok || !tc5::mbar_wait_fast(empty_own + 8u * st, ph ^ 1)) { ok = false; return; }     // the first round passes at once
            const uint32_t a = s_u + st * kFfStageBytes, b = a + 16384, bar = full_first + 8u * st;
            if (lead) tc5::mbar_expect_tx(full_own + 8u * st, 2 * (16384 + B_BYTES));
            if constexpr (A_MN) {
#pragma unroll
                for (int j = 0; j < 2; ++j) pair::load_2d(a + j * 8192, ma, am + j * 64, k * a_k, bar);
            } else {
                pair::load_2d(a, ma, k * a_k, am, bar);
            }
            if constexpr (B_MN) {
#pragma unroll
                for (int j = 0; j < B_BYTES / 8192; ++j) pair::load_2d(b + j * 8192, mb, bn + j * 64, k * b_k, bar);
            } else {
                pair::load_2d(b, mb, k * b_k, bn, bar);
            }
            if (++st == STAGES) { st = 0; ph ^= 1; }
        }
    }
    // Waits until every slice that was loaded has been used.
    __device__ __forceinline__ void drain() {
        for (int j = 0; j < STAGES && ok; ++j) {
            ok = tc5::mbar_wait_fast(empty_own + 8u * st, ph ^ 1);
            if (++st == STAGES) { st = 0; ph ^= 1; }
        }
    }
};
template <int STAGES> struct FfProducts {
    uint32_t s_u, full_own, empty_own;
    int st = 0;
    uint32_t ph = 0;
    bool ok = true;

    __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity) {
        ok = ok && pair::wait_cluster(bar, parity);
        tc5::fence_after_sync();
    }
    template <bool A_MN, bool B_MN>
    __device__ __forceinline__ void slices(int n, uint32_t acc, uint32_t idesc) {
        const uint32_t a0 = A_MN ? pair::desc_lo_mn(s_u) : tc5::desc_lo_k_major(s_u);
        const uint32_t b0 = B_MN ? pair::desc_lo_mn(s_u + 16384) : tc5::desc_lo_k_major(s_u + 16384);
        constexpr uint32_t a_step = A_MN ? 2048 / 16 : 2, b_step = B_MN ? 2048 / 16 : 2;      // 16 of the 64 k
        uint32_t more = 0;
        for (int k = 0; k < n; ++k) {
            wait(full_own + 8u * st, ph);
            if (!ok) return;
            const uint32_t a = a0 + st * (kFfStageBytes / 16), b = b0 + st * (kFfStageBytes / 16);
            pair::mma(acc, a, b, idesc, more);
#pragma unroll
            for (int ks = 1; ks < 4; ++ks) pair::mma(acc, a + ks * a_step, b + ks * b_step, idesc, 1);
            more = 1;
            pair::commit_both(empty_own + 8u * st);
            if (++st == STAGES) { st = 0; ph ^= 1; }
        }
    }
};

// What two fp32 values lose in their bf16 pair, as a bf16 pair; an infinite value has no remainder.
__device__ __forceinline__ uint32_t remainder_bf16(float a, float b, uint32_t pair) {
    const float ha = __uint_as_float(pair << 16), hb = __uint_as_float(pair & 0xffff0000u);
    return pack_bf16(isinf(ha) ? 0.f : a - ha, isinf(hb) ? 0.f : b - hb);
}

// ACT: a choice of the whole launch, where the kernel has an activation.  BN: accumulator columns of a tile (kFfOut, kFfDx; 256 in the others: 128 of G and 128 of U)
template <int KERNEL, int BN, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(FfShape<KERNEL>::threads, 1) gated_ff_kernel(const __grid_constant__ FfParams p) {
    using S = FfShape<KERNEL>;
    constexpr bool kOut = KERNEL == kFfOut || KERNEL == kFfOutSplit, kDx = KERNEL == kFfDx || KERNEL == kFfDxSplit;
    constexpr bool kBwdIn = KERNEL == kFfBwdIn || KERNEL == kFfBwdInTwo, kTwo = KERNEL == kFfBwdInTwo;
    constexpr bool kPart = KERNEL == kFfDw || KERNEL == kFfOutSplit || KERNEL == kFfDxSplit;      // writes fp32 sums of part of the range
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // the same offset in both CTAs
    const uint32_t s_u = smem_u32(smem), bar_u = s_u + S::bar_off;
    auto full = [&](int i) { return bar_u + 8u * (uint32_t)i; };
    auto empty = [&](int i) { return bar_u + 8u * (uint32_t)(S::stages + i); };
    auto tfull = [&](int i) { return bar_u + 8u * (uint32_t)(2 * S::stages + i); };
    auto tempty = [&](int i) { return bar_u + 8u * (uint32_t)(2 * S::stages + 2 + i); };
    // G, U and dH: pair 0 of tfull / tempty belongs to G | U, pair 1 to dH
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + S::bar_off + 8 * (2 * S::stages + 4));
    volatile int* abort_s = reinterpret_cast<volatile int*>(tmem_slot + 1);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int rank = (int)pair::cta_rank(), pair_id = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

    if (p.clear && p.status && blockIdx.x == 0 && tid < 64) p.status[tid] = 0;      // a give-up is a second away
    if (tid == 0) {
        for (int i = 0; i < 2 * S::stages + 2; ++i) tc5::mbar_init(bar_u + 8u * i, 1);
        for (int i = 0; i < 2; ++i) tc5::mbar_init(tempty(i), 2 * S::epi_warps);
        tc5::mbar_init_fence();
        *abort_s = 0;
    }
    __syncwarp();
    if (w == 1) pair::tmem_alloc(smem_u32(tmem_slot), 512);
    tc5::fence_before_sync();
    pair::cluster_sync();
    tc5::fence_after_sync();
    const uint32_t tbase = *tmem_slot;
    // From here on the kernel before has ended and its results are visible; every thread waits, so that no bounded wait below
    // counts that kernel's time.
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int kd = (p.D + kFfK - 1) / kFfK, kf = (p.F + kFfK - 1) / kFfK, km = p.two ? 2 : (p.rows + kFfK - 1) / kFfK;
    const int n_tiles = kOut || kDx ? (p.D + BN - 1) / BN : kBwdIn ? (p.F + p.step - 1) / p.step : (p.F + 127) / 128;   // along the output's columns
    const int dw_n0 = (p.D + 255) / 256, dw_n1 = (p.F + 255) / 256, dw_tiles = dw_n0 * dw_n1;             // weight gradients, each of the three
    struct Tile { int m, n, k0, k1, job, split, halves; };      // corner, slices, and which product
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
            q.k1 = KERNEL == kFfIn ? kd : kOut ? kf : p.two ? 4 * kf : 2 * kf;
            if constexpr (kPart) {
                const int per = p.tiles / p.splits, all = q.k1;
                q.split = t / per;
                t %= per;
                q.k0 = all * q.split / p.splits; q.k1 = all * (q.split + 1) / p.splits;
            }
            q.m = t / n_tiles * 256;
            q.n = t % n_tiles * (kOut || kDx ? BN : kBwdIn ? p.step : 128);
            q.halves = p.step == 256 && p.F - q.n > 128 ? 2 : 1;         // of G | U
        }
        return q;
    };

    // The pairs stride over the tiles together: what runs at one time shares rows of A (a contiguous range of tiles per pair
    // read every row of A once per pair and was 17 % slower in the long products).
    if (w == 0 && lane == 0) {
        // =============== load thread ===============
        FfLoader<S::stages> ld{s_u, pair::in_first(full(0)), full(0), empty(0), rank == 0};
        const bool one = rank == 0;
        for (int t = pair_id; t < p.tiles && ld.ok; t += n_pairs) {
            const Tile q = tile_of(t);
            const int m = q.m + rank * 128, n = q.n + rank * (BN / 2);
            if constexpr (KERNEL == kFfIn) {
                ld.template slices<false, false, 16384>(0, kd, &p.a0, m, one ? &p.b0 : &p.b1, q.n);
            } else if constexpr (kOut) {
                ld.template slices<false, false, BN * 64>(q.k0, q.k1, &p.a0, m, &p.b0, n);
            } else if constexpr (kBwdIn) {      // dH: dy rows, Wd with its F axis contiguous
                ld.template slices<false, false, 16384>(0, kd, &p.a0, m, one ? &p.b0 : &p.b1, q.n);
                ld.template slices<false, true, 16384>(0, kd, &p.a1, m, &p.b2, n);
                if (q.halves == 2) ld.template slices<false, false, 16384>(0, kd, &p.a0, m, one ? &p.b0 : &p.b1, q.n + 128);
            } else if constexpr (kDx) {         // dG Wg, then dU Wu; with two terms the same for the remainders
                for (int seg = 0; seg < (p.two ? 4 : 2); ++seg) {
                    const int lo = q.k0 - seg * kf, hi = q.k1 - seg * kf;
                    ld.template slices<false, true, BN * 64>(lo < 0 ? 0 : lo, hi < kf ? hi : kf, seg & 1 ? &p.a1 : &p.a0, m + (seg >> 1) * kFfTwoRows,
                                                             seg & 1 ? &p.b1 : &p.b0, n);
                }
            } else {
                // with two terms x and dy meet both slices of the other operand
                ld.template slices<true, true, 16384>(q.k0, q.k1, q.job == 0 ? &p.a0 : q.job == 1 ? &p.a1 : &p.a2, m, q.job < 2 ? &p.b0 : &p.b1, n,
                                                      p.two && q.job == 2 ? 0 : kFfK, p.two && q.job < 2 ? 0 : kFfK);
            }
        }
        // the releases of the last slices still arrive in this CTA's shared memory: see them in before it ends
        ld.drain();
        if (!ld.ok) {   // copies still in flight land before the CTA ends (their barrier may be the other CTA's: give them time)
            *abort_s = 1;
            const long long start = clock64();
            while (clock64() - start < (1ll << 22)) {}
        }
    } else if (w == 1 && lane == 0 && rank == 0) {
        // =============== product thread ===============
        constexpr bool a_mn = KERNEL == kFfDw, b_mn = KERNEL == kFfDw || kDx;
        const uint32_t idesc = tc5::instr_desc(256, BN, a_mn, b_mn);
        FfProducts<S::stages> mm{s_u, full(0), empty(0)};
        int i = 0, gu = 0;      // tiles, G | U accumulators so far
        for (int t = pair_id; t < p.tiles && mm.ok; t += n_pairs, ++i) {
            const Tile q = tile_of(t);
            if constexpr (kBwdIn) {     // each accumulator has one place: what was there before has to be out
                for (int phase = 0; phase < 1 + q.halves && mm.ok; ++phase) {
                    if (phase == 1) {
                        if (i > 0) mm.wait(tempty(1), (i - 1) & 1);
                        mm.template slices<false, true>(kd, tbase + 256, tc5::instr_desc(256, 256, 0, 1));
                        if (mm.ok) pair::commit_both(tfull(1));
                    } else {
                        if (gu > 0) mm.wait(tempty(0), (gu - 1) & 1);
                        mm.template slices<false, false>(kd, tbase, idesc);
                        if (mm.ok) pair::commit_both(tfull(0));
                        ++gu;
                    }
                }
            } else {
                // an accumulator is free again when the epilogue of the tile two before has taken it out
                if (i >= 2) mm.wait(tempty(i & 1), (i / 2 - 1) & 1);
                mm.template slices<a_mn, b_mn>(q.k1 - q.k0, tbase + (i & 1) * 256u, idesc);
                if (mm.ok) pair::commit_both(tfull(i & 1));
            }
        }
        if (!mm.ok) *abort_s = 1;
    } else if (w >= 2) {
        // =============== epilogue warps: 32 rows (tensor-memory lanes) x a half or quarter of the tile's columns each ===============
        const int quad = w & 3, part = (w - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        unsigned char* stg = smem + S::out_off + (w - 2) * S::staging * S::tile_bytes;
        const uint32_t stg_u = smem_u32(stg), release0 = pair::in_first(tempty(0)), release1 = pair::in_first(tempty(1));
        // 16 bytes of this thread's row of staging tile `buf`: rows of 128 bytes, or of 64, in the store's swizzle
        auto put = [&](int buf, int chunk, uint32_t x, uint32_t y, uint32_t z, uint32_t v) {
            *reinterpret_cast<uint4*>(stg + buf * S::tile_bytes + tile_off(lane, chunk)) = make_uint4(x, y, z, v);
        };
        auto put64 = [&](int buf, int chunk, uint32_t x, uint32_t y, uint32_t z, uint32_t v) {
            *reinterpret_cast<uint4*>(stg + buf * S::tile_bytes + lane * 64 + ((chunk ^ ((lane >> 1) & 3)) << 4)) = make_uint4(x, y, z, v);
        };
        int i = 0, gu = 0;
        for (int t = pair_id; t < p.tiles; t += n_pairs, ++i) {
            const Tile q = tile_of(t);
            auto ready = [&](int which, uint32_t parity) {      // the whole warp together
                const bool ok = !*abort_s && tc5::mbar_wait_fast(tfull(which), parity);
                if (!__all_sync(0xffffffffu, ok)) { *abort_s = 1; return false; }
                tc5::fence_after_sync();
                return true;
            };
            if (!kBwdIn && !ready(i & 1, (i / 2) & 1)) break;
            const int row = q.m + rank * 128 + quad * 32;
            auto done = [&](uint32_t bar) {           // this warp has taken (its part of) an accumulator out
                tc5::fence_before_sync();
                __syncwarp();
                if (lane == 0) pair::arrive_cluster(bar);
            };
            auto send = [&](const CUtensorMap* map, int buf, int col, int limit_cols, int limit_rows) {
                tc5::fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (col < limit_cols && row < limit_rows) {
                        if constexpr (kPart) pair::store_3d(map, col, row, q.job == 1 ? p.splits + q.split : q.split, stg_u + buf * S::tile_bytes);
                        else pair::store_2d(map, col, row, stg_u + buf * S::tile_bytes);
                    }
                    pair::store_commit();
                }
            };
            if constexpr (KERNEL == kFfIn) {
                const uint32_t src = tbase + lane_base + (i & 1) * 256 + part * 32;
                uint32_t g[32], u[32];
                tc5::tmem_ld32(src, g);
                tc5::tmem_ld32(src + 128, u);
                tc5::tmem_ld_wait();
                done((i & 1) ? release1 : release0);
                if (lane == 0) pair::store_wait_read<1>();
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t x[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        float r[2], unused;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int k = j * 8 + 2 * y + e;
                            r[e] = ff_act<ACT, false>(__uint_as_float(g[k]), unused) * __uint_as_float(u[k]);
                        }
                        // rounded once: the second product's operands are bf16, and a second term would double that product
                        x[y] = pack_bf16(r[0], r[1]);
                    }
                    put64(i & 1, j, x[0], x[1], x[2], x[3]);
                }
                send(&p.c0, i & 1, q.n + part * 32, p.F, p.rows);
            } else if constexpr (kBwdIn) {
                const uint32_t src = tbase + lane_base + part * 32;
#pragma unroll 1
                for (int half = 0; half < q.halves; ++half, ++gu) {
                    const uint32_t src_dh = src + 256 + half * 128;
                    if (!ready(0, gu & 1)) break;
                    uint32_t g[32], u[32];
                    tc5::tmem_ld32(src, g);
                    tc5::tmem_ld32(src + 128, u);
                    tc5::tmem_ld_wait();
                    done(release0);
                    // What does not need dH comes first, and the inner row with it: the first half's dH is still being summed then,
                    // and the second half's products must not wait for this.  g becomes act(g), u becomes u act'(g).
                    const int col = q.n + half * 128 + part * 32;
                    const bool inside = col < p.F && row < (kTwo ? kFfTwoRows : p.rows);
                    // Two terms: the rows between the last one and kFfTwoRows are summed over too and hold zeros, whatever the weights.
                    const bool real = !kTwo || row + lane < p.rows;
                    uint32_t rem[kTwo ? 32 : 1];        // remainders: of h, then of dG and dU
                    if (lane == 0) pair::store_wait_read<0>();
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t x[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            float r[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int k = j * 8 + 2 * y + e;
                                const float uv = __uint_as_float(u[k]);
                                float da;
                                const float a = ff_act<ACT, true>(__uint_as_float(g[k]), da);
                                r[e] = a * uv;
                                g[k] = __float_as_uint(a);
                                u[k] = __float_as_uint(uv * da);
                            }
                            x[y] = real ? pack_bf16(r[0], r[1]) : 0;
                            if constexpr (kTwo) rem[j * 4 + y] = real ? remainder_bf16(r[0], r[1], x[y]) : 0;
                        }
                        put64(0, j, x[0], x[1], x[2], x[3]);
                        if constexpr (kTwo) put64(1, j, rem[j * 4], rem[j * 4 + 1], rem[j * 4 + 2], rem[j * 4 + 3]);
                    }
                    tc5::fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (inside) {
                            pair::store_2d(&p.c2, col, row, stg_u);
                            if (kTwo) pair::store_2d(&p.c2, col, row + kFfTwoRows, stg_u + S::tile_bytes);
                        }
                        pair::store_commit();
                    }
                    if (half == 0 && !ready(1, i & 1)) break;
                    if (lane == 0) pair::store_wait_read<0>();      // the inner row has left its tile
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 32; c += 16) {
                        uint32_t dh[16];
                        tc5::tmem_ld16(src_dh + c, dh);
                        tc5::tmem_ld_wait();
                        if (c == 16 && half == q.halves - 1) done(release1);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t o[2][4];
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const int k = c + j * 8 + 2 * y;
                                const float d0 = __uint_as_float(dh[j * 8 + 2 * y]), d1 = __uint_as_float(dh[j * 8 + 2 * y + 1]);
                                const float r[2][2] = {{d0 * __uint_as_float(u[k]), d1 * __uint_as_float(u[k + 1])},
                                                       {d0 * __uint_as_float(g[k]), d1 * __uint_as_float(g[k + 1])}};
#pragma unroll
                                for (int m = 0; m < 2; ++m) {
                                    o[m][y] = real ? pack_bf16(r[m][0], r[m][1]) : 0;
                                    if constexpr (kTwo) rem[m * 16 + k / 2] = real ? remainder_bf16(r[m][0], r[m][1], o[m][y]) : 0;
                                }
                            }
#pragma unroll
                            for (int m = 0; m < 2; ++m) put64(m, c / 8 + j, o[m][0], o[m][1], o[m][2], o[m][3]);
                        }
                    }
                    tc5::fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (inside) {
                            pair::store_2d(&p.c0, col, row, stg_u);
                            pair::store_2d(&p.c1, col, row, stg_u + S::tile_bytes);
                        }
                        pair::store_commit();
                    }
                    if constexpr (kTwo) {
                        if (lane == 0) pair::store_wait_read<0>();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 8; ++j) put64(j / 4, j % 4, rem[j * 4], rem[j * 4 + 1], rem[j * 4 + 2], rem[j * 4 + 3]);
                        tc5::fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            if (inside) {
                                pair::store_2d(&p.c0, col, row + kFfTwoRows, stg_u);
                                pair::store_2d(&p.c1, col, row + kFfTwoRows, stg_u + S::tile_bytes);
                            }
                            pair::store_commit();
                        }
                    }
                }
            } else if constexpr (kPart) {
                const uint32_t src = tbase + lane_base + (i & 1) * 256 + part * 128;
                const CUtensorMap* map = q.job < 2 ? &p.c0 : &p.c1;
                const int limit_cols = q.job < 2 ? p.D : p.F, limit_rows = KERNEL != kFfDw ? p.rows : q.job < 2 ? p.F : p.D;
#pragma unroll
                for (int c = 0; c < 128; c += 32) {
                    uint32_t x[32];
                    tc5::tmem_ld32(src + c, x);
                    tc5::tmem_ld_wait();
                    if (c == 96) done((i & 1) ? release1 : release0);
                    if (lane == 0) pair::store_wait_read<1>();
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) put((c / 32) & 1, j, x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                    send(map, (c / 32) & 1, q.n + part * 128 + c, limit_cols, limit_rows);
                }
            } else {
                constexpr int W = 64;       // columns per stored tile
                const uint32_t src = tbase + lane_base + (i & 1) * 256 + part * (BN / 2);
#pragma unroll
                for (int c = 0; c < BN / 2; c += 32) {
                    uint32_t x[32];
                    tc5::tmem_ld32(src + c, x);
                    tc5::tmem_ld_wait();
                    if (c + 32 == BN / 2) done((i & 1) ? release1 : release0);
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
                        put(buf, (c & 32) / 8 + j, y[0], y[1], y[2], y[3]);
                    }
                    if (c % W + 32 == W) send(&p.c0, buf, q.n + part * (BN / 2) + c / W * W, p.D, p.rows);
                }
            }
        }
        if (lane == 0) pair::store_wait<0>();
    }

    __syncwarp();
    tc5::fence_before_sync();
    pair::cluster_sync();      // both CTAs are past their last product, load and barrier use
    if (tid == 0 && *abort_s) report_timeout(p.status, p.record);
    if (w == 1) pair::tmem_free(tbase, 512);
}

// Results [jobs][n] from the fp32 sums of the ranges, part [jobs][splits][n]: added in order, rounded once.
__global__ void __launch_bounds__(256) gated_ff_sum_kernel(const float* part, __nv_bfloat16* out0, __nv_bfloat16* out1, __nv_bfloat16* out2,
                                                           long long n, int splits, int jobs) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long n8 = n / 8;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < jobs * n8; i += gridDim.x * 256ll) {
        const int job = (int)(i / n8);
        const long long e = (i % n8) * 8;
        const float* src = part + (long long)job * splits * n + e;
        float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
#pragma unroll 4
        for (int s = 1; s < splits; ++s) {
            const float4 c = *reinterpret_cast<const float4*>(src + s * n), d = *reinterpret_cast<const float4*>(src + s * n + 4);
            a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
            b.x += d.x; b.y += d.y; b.z += d.z; b.w += d.w;
        }
        __nv_bfloat16* out = (job == 0 ? out0 : job == 1 ? out1 : out2) + e;
        *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
    }
}
// 2-D map over a row-major [n_rows, n_cols] bf16 matrix, rows `ld` elements apart (0: n_cols), boxes of box_rows x box_cols.
bool bf16_map(CUtensorMap* m, const void* base, long long n_rows, int n_cols, int box_rows, int box_cols = 64, int ld = 0) {
    const cuuint64_t dims[2] = {(cuuint64_t)n_cols, (cuuint64_t)n_rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(ld ? ld : n_cols) * 2};
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

// Launches a kernel so that its CTAs may start (where they find room) while the kernel before it in the call still runs; both
// go on to what depends on it only once that one has ended (griddepcontrol.wait).  first: nothing of this call is before it.
template <typename... Params, typename... Args>
bool launch(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, bool first, Args... args) {
    cudaLaunchAttribute attr[1] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = first ? 0 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return true;
    cudaGetLastError();     // reported by the caller's status, not by the next call of somebody else
    return false;
}
template <int KERNEL, int BN, int ACT = BPT_ACT_RELU>
bpt_status run(const FfParams& p, cudaStream_t st, const char* name) {
    constexpr size_t smem = FfShape<KERNEL>::bytes;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    if (cudaFuncSetAttribute(gated_ff_kernel<KERNEL, BN, ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return BPT_ERR_CUDA;
    if (!launch(gated_ff_kernel<KERNEL, BN, ACT>, dim3(2 * std::min(p.tiles, kFfPairs)), FfShape<KERNEL>::threads, smem, st, p.clear, p)) return BPT_ERR_CUDA;
    trace_mark(st, name);
    return BPT_OK;
}

bpt_status sum_parts(const float* part, void* out0, void* out1, void* out2, long long n, int splits, int jobs, cudaStream_t st, const char* name) {
    if (!launch(gated_ff_sum_kernel, dim3((unsigned)std::min<long long>((jobs * n / 8 + 255) / 256, 148 * 8)), 256, 0, st, false, part,
                (__nv_bfloat16*)out0, (__nv_bfloat16*)out1, (__nv_bfloat16*)out2, n, splits, jobs))
        return BPT_ERR_CUDA;
    trace_mark(st, name);
    return BPT_OK;
}

template <int KERNEL>
bpt_status run_act(const FfParams& p, int act, cudaStream_t st, const char* name) {
    return act == BPT_ACT_RELU ? run<KERNEL, 256, BPT_ACT_RELU>(p, st, name) : act == BPT_ACT_SILU ? run<KERNEL, 256, BPT_ACT_SILU>(p, st, name)
                                                                                                  : run<KERNEL, 256, BPT_ACT_GELU>(p, st, name);
}

constexpr size_t kStatusBytes = 256;
// Inner rows start on 128-byte boundaries, whatever F is; what lies between F and there is neither written nor read.
int inner_ld(int F) { return (F + 63) / 64 * 64; }
size_t inner_bytes(long long rows, int F) { return ((size_t)rows * inner_ld(F) * 2 + 255) & ~(size_t)255; }

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
// y and dx, [rows, D] with `slices` slices to sum over.  While tiles of 256 columns leave half of the pairs idle, their sums are
// shared out: ranges of at least eight slices, eight at most.  Shorter and more ranges cost as much in fp32 partial sums as they
// save in products (y and dx at 512 x 2048, graph replay of the whole call, us: ranges of 4 slices, up to 16: 22.8 and 30.0 at 1023
// rows; of 8, up to 8: 20.0 and 28.5; at 1024 x 4096 and 2046 rows two ranges 48.6 and 76.4 against 51.7 and 88.1 of tiles of 128
// columns, whose products run at 0.6 of the rate).
struct OutPlan { int bn, splits; };
OutPlan plan_out(long long rows, int D, int slices) {
    const long long tiles = (rows + 255) / 256 * ((D + 255) / 256);
    const int splits = (int)std::min<long long>(std::min<long long>(kFfPairs / tiles, slices / 8), 8);
    if (splits > 1) return {256, splits};
    return {tiles * 2 <= kFfPairs ? 128 : 256, 1};
}
size_t part_bytes(long long rows, int D, int slices) {
    const OutPlan q = plan_out(rows, D, slices);
    return q.splits > 1 ? (size_t)q.splits * rows * D * 4 : 0;
}
// The backward's inner results: few rows keep two bf16 terms each, which costs nothing next to the launches and leaves the
// results' own rounding the only one that shows; more rows keep one (a third of the memory traffic, half of the products).
int bwd_terms(long long rows) { return rows <= kFfTwoRows ? 2 : 1; }
long long bwd_inner_rows(long long rows) { return bwd_terms(rows) == 2 ? 2 * kFfTwoRows : rows; }
int slices_of(int n) { return (n + kFfK - 1) / kFfK; }

}  // namespace
}  // namespace bpt

using namespace bpt;

extern "C" int32_t bpt_gated_ff_few_rows(int64_t rows, int32_t D, int32_t F) {
    return check_ff(rows, D, F, BPT_ACT_RELU) == BPT_OK && gated_ff_few_rows(rows, D, F);
}

extern "C" size_t bpt_gated_ff_workspace_bytes(int64_t rows, int32_t D, int32_t F, int backward) {
    if (check_ff(rows, D, F, BPT_ACT_RELU) != BPT_OK || rows == 0) return 0;
    if (!backward) return gated_ff_few_rows(rows, D, F) ? (size_t)rows * F * 4 : inner_bytes(rows, F) + part_bytes(rows, D, slices_of(F));
    // the partial sums of dx and of the weight gradients share their place
    return 3 * inner_bytes(bwd_inner_rows(rows), F) +
           std::max((size_t)3 * dw_splits(rows, D, F) * D * F * 4, part_bytes(rows, D, bwd_terms(rows) * 2 * slices_of(F)));
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
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (gated_ff_few_rows(rows, D, F)) {
        const GatedFfRows q{static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(w_gate), static_cast<const __nv_bfloat16*>(w_up),
                            static_cast<const __nv_bfloat16*>(w_down), static_cast<__nv_bfloat16*>(y), static_cast<__nv_bfloat16*>(workspace),
                            static_cast<int*>(status), (int)rows, D, F, act};
        return launch_gated_ff_rows(q, st);
    }
    if (!tc5::encode_tiled() || !tc5::context_current()) return BPT_ERR_CUDA;
    FfParams p{};
    p.status = static_cast<int*>(status);
    p.record = device_record();
    if (!p.record) return BPT_ERR_CUDA;
    p.clear = true;
    p.rows = (int)rows; p.D = D; p.F = F;
    const int ld = inner_ld(F);
    if (!bf16_map(&p.a0, x, rows, D, 128) || !bf16_map(&p.b0, w_gate, F, D, 128) || !bf16_map(&p.b1, w_up, F, D, 128) ||
        !bf16_map(&p.c0, workspace, rows, F, 32, 32, ld))
        return BPT_ERR_CUDA;
    const int mt = (int)((rows + 255) / 256);
    p.tiles = mt * ((F + 127) / 128);
    bpt_status e = run_act<kFfIn>(p, act, st, "gated_ff_in");
    if (e != BPT_OK) return e;
    p.clear = false;
    const OutPlan o = plan_out(rows, D, slices_of(F));
    float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + inner_bytes(rows, F));
    if (!bf16_map(&p.a0, workspace, rows, F, 128, 64, ld) || !bf16_map(&p.b0, w_down, D, F, o.bn / 2) ||
        !(o.splits > 1 ? part_map(&p.c0, part, o.splits, (int)rows, D) : bf16_map(&p.c0, y, rows, D, 32)))
        return BPT_ERR_CUDA;
    p.splits = o.splits;
    p.tiles = mt * ((D + o.bn - 1) / o.bn) * o.splits;
    if (o.splits == 1) return o.bn == 256 ? run<kFfOut, 256>(p, st, "gated_ff_out") : run<kFfOut, 128>(p, st, "gated_ff_out");
    e = run<kFfOutSplit, 256>(p, st, "gated_ff_out");
    if (e != BPT_OK) return e;
    return sum_parts(part, y, nullptr, nullptr, rows * (long long)D, o.splits, 1, st, "gated_ff_out_sum");
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
    if (!tc5::encode_tiled() || !tc5::context_current()) return BPT_ERR_CUDA;
    const long long inner = bwd_inner_rows(rows);
    const size_t hidden = inner_bytes(inner, F);
    char *dg = static_cast<char*>(workspace), *du = dg + hidden, *h = du + hidden;
    float* part = reinterpret_cast<float*>(h + hidden);
    const int mt = (int)((rows + 255) / 256);
    FfParams p{};
    p.status = static_cast<int*>(status);
    p.record = device_record();
    if (!p.record) return BPT_ERR_CUDA;
    p.clear = true;
    p.rows = (int)rows; p.D = D; p.F = F;
    const int ld = inner_ld(F);
    if (!bf16_map(&p.a0, x, rows, D, 128) || !bf16_map(&p.a1, dy, rows, D, 128) || !bf16_map(&p.b0, w_gate, F, D, 128) ||
        !bf16_map(&p.b1, w_up, F, D, 128) || !bf16_map(&p.b2, w_down, D, F, 64) ||
        !bf16_map(&p.c0, dg, inner, F, 32, 32, ld) || !bf16_map(&p.c1, du, inner, F, 32, 32, ld) || !bf16_map(&p.c2, h, inner, F, 32, 32, ld))
        return BPT_ERR_CUDA;
    // tiles of one half while whole ones leave half of the pairs idle: 16 slices of products one after the other instead of 24
    p.step = mt * ((F + 255) / 256) * 2 <= kFfPairs ? 128 : 256;
    p.tiles = mt * ((F + p.step - 1) / p.step);
    p.two = bwd_terms(rows) == 2;
    bpt_status e = p.two ? run_act<kFfBwdInTwo>(p, act, st, "gated_ff_bwd_in") : run_act<kFfBwdIn>(p, act, st, "gated_ff_bwd_in");
    if (e != BPT_OK) return e;
    p.clear = false;
    if (dx) {
        const OutPlan o = plan_out(rows, D, bwd_terms(rows) * 2 * slices_of(F));
        if (!bf16_map(&p.a0, dg, inner, F, 128, 64, ld) || !bf16_map(&p.a1, du, inner, F, 128, 64, ld) || !bf16_map(&p.b0, w_gate, F, D, 64) ||
            !bf16_map(&p.b1, w_up, F, D, 64) ||
            !(o.splits > 1 ? part_map(&p.c0, part, o.splits, (int)rows, D) : bf16_map(&p.c0, dx, rows, D, 32)))
            return BPT_ERR_CUDA;
        p.splits = o.splits;
        p.tiles = mt * ((D + o.bn - 1) / o.bn) * o.splits;
        e = o.splits > 1 ? run<kFfDxSplit, 256>(p, st, "gated_ff_dx")
                         : o.bn == 256 ? run<kFfDx, 256>(p, st, "gated_ff_dx") : run<kFfDx, 128>(p, st, "gated_ff_dx");
        if (e != BPT_OK) return e;
        if (o.splits > 1) e = sum_parts(part, dx, nullptr, nullptr, rows * (long long)D, o.splits, 1, st, "gated_ff_dx_sum");
        if (e != BPT_OK) return e;
    }
    if (weights) {
        p.splits = dw_splits(rows, D, F);
        if (!bf16_map(&p.a0, dg, inner, F, 64, 64, ld) || !bf16_map(&p.a1, du, inner, F, 64, 64, ld) || !bf16_map(&p.a2, dy, rows, D, 64) ||
            !bf16_map(&p.b0, x, rows, D, 64) || !bf16_map(&p.b1, h, inner, F, 64, 64, ld) || !part_map(&p.c0, part, 2 * p.splits, F, D) ||
            !part_map(&p.c1, part + (size_t)2 * p.splits * D * F, p.splits, D, F))
            return BPT_ERR_CUDA;
        p.tiles = 3 * ((D + 255) / 256) * ((F + 255) / 256) * p.splits;
        e = run<kFfDw, 256>(p, st, "gated_ff_dw");
        if (e != BPT_OK) return e;
        e = sum_parts(part, dw_gate, dw_up, dw_down, (long long)D * F, p.splits, 3, st, "gated_ff_dw_sum");
    }
    return e;
}
