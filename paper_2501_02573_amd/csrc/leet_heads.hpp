// Arguments of the kernels that rotate and normalise rows of heads (leet_heads.hip).
#pragma once

#include <hip/hip_runtime.h>

namespace leet {

// One of queries and keys.  Strides in elements.
struct HeadRows {
    const char* in;                      // x
    const char* grad;                    // backward: dy
    char* out;                           // y; backward: dx
    long long in_b, in_h, in_n;
    long long grad_b, grad_h, grad_n;
    long long out_b, out_h, out_n;
    const void* weight;                  // [d] or null
    void* weight_grad;                   // [d] or null
    int H;
};

struct HeadsParams {
    HeadRows q, k;                // k.H = 0: no keys
    const double* freq;           // [rot/2]
    const long long* positions;   // or null
    long long positions_batch, pos0;
    float scale, eps;
    int rot, d, N;
    int tokens;                   // B N
    int weight_f32;               // weights are fp32 whatever the elements are
    int transposed;
    int vector;                   // rows can be cut into pieces of four elements (else of one)
    int stream;                   // the rows exceed the last-level cache: nontemporal loads and stores
    int heads_per_wave, units_q, units;  // a wave takes so many heads of a token; waves a token needs
    int groups;                   // backward: workgroups a unit's tokens are spread over
    float* partial;               // backward: [groups * units][d]: sums of weight gradients, one row a workgroup
};

// elem: 0 = fp32, 1 = bf16, 2 = fp16
hipError_t launch_heads(const HeadsParams& p, int elem, int layout, bool norm, hipStream_t stream);
hipError_t launch_heads_backward(const HeadsParams& p, int elem, int layout, hipStream_t stream);
// the weight gradients from the sums that the backward kernel left in p.partial
hipError_t launch_heads_weights(const HeadsParams& p, int elem, hipStream_t stream);

// How the rows are spread over waves and workgroups: heads_per_wave, units, and for the backward kernel groups.
void plan_heads(HeadsParams* p, bool backward);

}  // namespace leet
