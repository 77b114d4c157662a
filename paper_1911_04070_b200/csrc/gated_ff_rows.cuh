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

// One pass over the weights serves 64 rows.  Measured (graph replay, 512 x 2048): 5.5 us at one row, 6.6 at 14, 11.9 at 64,
// 18.4 at 65 against 23 us of the tensor-memory kernels at any of them; 1024 x 4096: 10.0, 13.3, 31.7, 52.0 against 36 us.
constexpr int kGatedFfFewRows = BPT_GATED_FF_FEW_ROWS;

}  // namespace bpt
