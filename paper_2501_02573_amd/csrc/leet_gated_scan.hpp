// Arguments of the gated linear recurrence's kernels (leet_gated_scan.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

namespace leet {

struct RowsIn {
    const char* data;
    long long batch, token;  // strides in elements
};
struct RowsOut {
    char* data;
    long long batch, token;
};

struct GatedScanParams {
    RowsIn x, gate, h, dh;         // h, dh: backward
    RowsOut out, dx, dgate;        // out: forward; dx, dgate: backward
    const float* state_in;         // [S][C] or null
    float* state_out;              // forward: [S][C] or null
    const float* dstate_out;       // backward: [S][C] or null
    float* dstate_in;              // backward: [S][C] or null
    const int* offsets;            // [S + 1] or null: S = B sequences of N tokens
    int sequences;                 // S
    int B, N, C;
    int vector;                    // step: channels a thread takes, 1 or 4
    int columns;                   // column blocks of a batch entry
    int waves;                     // waves of a workgroup
    int tiles;                     // of a column block's N tokens
    void* workspace;               // more than one tile: gated_scan_workspace bytes
    int groups;                    // of column blocks, each with a ticket counter of its own
};

// Bytes of workspace for these sizes; 0: none is needed.
size_t gated_scan_workspace(int B, int N, int C, bool backward);
// Threads that a launch of these sizes has.
long long gated_scan_threads(int B, int N, int C, bool backward);

// elem, gate_elem: 0 = fp32, 1 = bf16, 2 = fp16; gate_elem is elem or 0.  mode: a leet_gate_mode
hipError_t launch_gated_scan(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream);
hipError_t launch_gated_scan_backward(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream);
// one token; rows through x, gate, out, the state through state_out (in place)
hipError_t launch_gated_step(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream);

}  // namespace leet
