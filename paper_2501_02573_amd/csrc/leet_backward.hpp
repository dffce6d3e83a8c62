// Arguments of the kernels of the attention's backward pass (leet_bwd_16bit.hip, leet_bwd_f32.hip).
#pragma once

#include <hip/hip_runtime.h>

namespace leet {

// One walk over the tokens, from the first to the last or (reversed) from the last to the first:
//     out_i = sum over the tokens j passed so far, i's own included, of gamma^|i-j| (x_i . y_j) z_j, and what the state gives.
struct BwdRole {
    const void *x, *y;          // [BH][N][D]
    const void* z;              // [BH][N][DV]
    void* out;                  // [BH][N][DV], the input type
    // The state is [D][DV]: element (dk, c) of a sequence's entering state lies at dk*enter_row + c*enter_col, in a slot
    // at dk*slot_row + c*slot_col, and the leaving state is written as [D][DV].
    const float* enter;         // [BH] states or null: the state before the first token passed
    float* leave;               // [BH] states or null: the state behind the last one
    float* slots;               // [BH][nseg - 1] states: what entered segments 1 .. nseg - 1 left there, without `enter`
    int enter_row, enter_col, slot_row, slot_col;
    int reversed;
};

struct BwdParams {
    BwdRole role[3];
    int roles;
    const float* gamma;         // [H]; null: gamma is 1
    int BH, H, N;
    int nseg, seg_chunks;       // segments a sequence, in the order of the walk; chunks of all but the last
};

// D: width of the rows of x and y, DV of z and out.  fine: the leaving states are wanted to fp32's precision.
hipError_t launch_bwd_16bit_states(const BwdParams& p, int D, int DV, bool f16, bool fine, hipStream_t stream);
hipError_t launch_bwd_16bit_walk(const BwdParams& p, int D, int DV, bool f16, bool fine, hipStream_t stream);
// the same for both widths 128, a compute unit a sequence
hipError_t launch_bwd_16bit_tiles(const BwdParams& p, bool f16, bool fine, hipStream_t stream);
hipError_t launch_bwd_f32_states(const BwdParams& p, int D, hipStream_t stream);
hipError_t launch_bwd_f32_walk(const BwdParams& p, int D, hipStream_t stream);

}  // namespace leet
