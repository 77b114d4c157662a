// The gated feed-forward block for a few rows (gated_ff_rows.cu): what its launcher takes, and when it is the one to use.
#pragma once
#include "bpt_internal.cuh"

namespace bpt {

struct GatedFfRows {
    const __nv_bfloat16 *x, *w_gate, *w_up, *w_down;
    __nv_bfloat16* y;
    float* h;               // [rows, F]
    int* status;            // 256 bytes, cleared; or nullptr
    int rows, D, F, act;
};
bpt_status launch_gated_ff_rows(const GatedFfRows& p, cudaStream_t st);

// Whether a forward call runs here or on the tensor-memory kernels (gated_ff.cu).  A pass over the weights serves 8, 16, 32 or 64
// rows, and its time grows with rows x weights: mma.sync keeps up with memory for 8 rows only.  Measured (graph replay, us, here /
// there): 512 x 2048: 5.7 / 15.0 at 1 row, 12.0 / 16.4 at 64, 19.4 / 17.7 at 128; 1024 x 4096: 13.3 / 20.6 at 16, 22.0 / 20.9 at 32,
// 31.7 / 21.7 at 64; 256 x 1024: 13.4 / 15.7 at 256, 21.7 / 15.9 at 512; 128 x 512: 10.1 / 12.1 at 256, 15.5 / 12.3 at 1024;
// 2048 x 5632: 24.8 / 29.2 at 8, 33.4 / 28.2 at 16; 4096 x 11008: 73 / 79 at 8.
inline bool gated_ff_few_rows(long long rows, int D, int F) {
    const long long served = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : (rows + 63) / 64 * 64;
    return rows <= 256 && (served == 8 || served * D * F <= 80000000);
}

}  // namespace bpt
