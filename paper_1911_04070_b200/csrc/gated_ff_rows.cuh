// The gated feed-forward block for a few rows (gated_ff_rows.cu): what its launcher takes, and when it is the one to use.
#pragma once
#include "bpt_internal.cuh"

namespace bpt {

struct GatedFfRows {
    const __nv_bfloat16 *x, *w_gate, *w_up, *w_down;
    __nv_bfloat16* y;
    __nv_bfloat16* h;       // [2][rows, F]: the inner rows' two terms
    int* status;            // 256 bytes, cleared; or nullptr
    int rows, D, F, act;
};
bpt_status launch_gated_ff_rows(const GatedFfRows& p, cudaStream_t st);

// Whether a forward call runs here or on the tensor-memory kernels (gated_ff.cu).  A pass over the weights serves 8, 16, 32 or 64
// rows, and its time grows with rows x weights once it is no longer the memory that it waits for.  Measured (graph replay, us, here /
// there): 512 x 2048: 4.9 / 15.0 at 1 row, 10.7 / 16.4 at 64, 15.7 / 17.7 at 128, 22.6 / 18.0 at 192; 1024 x 4096: 14.5 / 20.9 at 32,
// 23.3 / 21.7 at 64; 256 x 1024: 11.9 / 15.7 at 256, 16.8 / 15.9 at 512; 128 x 512: 10.3 / 12.1 at 512, 13.1 / 12.3 at 1024;
// 2048 x 5632: 23.2 / 28.2 at 16, 35.1 / 28.5 at 32; 4096 x 11008: 49.7 / 88.6 at 1, 62.3 / 74.5 at 16, 88.6 / 75.9 at 32.
// The limit of 384 rows leaves to the tensor-memory kernels what the narrowest weights would still gain above it (1.8 us at 128 x 512).
inline bool gated_ff_few_rows(long long rows, int D, int F) {
    const long long served = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : (rows + 63) / 64 * 64;
    return rows <= 384 && (served <= 16 || served * D * F <= 135000000);
}

}  // namespace bpt
