// Arguments of the kernels that norm rows of a residual stream (leet_norm.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "leet_gated_scan.hpp"  // RowsIn, RowsOut

namespace leet {

constexpr int kNormChannels = 16384;  // a row lies in registers of 1024 threads at most

struct NormParams {
    RowsIn x;              // forward: x; backward: the gradient of the output
    RowsIn stream;         // forward: the residual; backward: the sum that was normed
    RowsIn grad;           // backward: the gradient that comes along the stream
    RowsOut out;           // forward: the normed row, or its 8-bit values; backward: the gradient in x's type
    RowsOut sum;           // forward: x + residual; backward: the gradient in the stream's type
    const void* weight;    // [C] or null
    void* weight_grad;     // [C] or null
    float* scales;         // 8 bits: [rows][C / group]
    float* partial;        // backward: [workgroups][C], sums of the weight's gradient
    float eps;
    int weight_f32;
    int C, N, rows;        // rows = B N
    int group;             // 8 bits: channels that share a scale
    int far;               // the rows exceed the last-level cache: nontemporal loads and stores
    int groups;            // backward: workgroups
};

// elem, stream_elem: 0 = fp32, 1 = bf16, 2 = fp16; stream_elem is elem or 0
hipError_t launch_norm(const NormParams& p, int elem, int stream_elem, bool q8, hipStream_t stream);
hipError_t launch_norm_backward(const NormParams& p, int elem, int stream_elem, hipStream_t stream);
// the weight's gradient from the sums that the backward kernel left in p.partial (zero where there are no rows)
hipError_t launch_norm_weight(const NormParams& p, int elem, hipStream_t stream);

// Workgroups of the backward kernel
int norm_groups(int rows, int C);
// Rows a workgroup takes at once
int norm_rows_at_once(int C);

}  // namespace leet
