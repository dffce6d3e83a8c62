// Arguments of the kernels that take the norm over many tensors and clip them to it (leet_clip.hip).
#pragma once

#include <hip/hip_runtime.h>

namespace leet {

constexpr int kClipTensors = 64;    // of a launch
constexpr int kClipTile = 16384;    // elements that a workgroup takes at once
constexpr int kClipParts = 1024;    // sums of squares that the tensors are cut into, one a workgroup

struct ClipParams {
    const char* data[kClipTensors];
    char* out[kClipTensors];
    long long count[kClipTensors];
    int first[kClipTensors + 1];    // the tile that a tensor begins with; of the last + 1, all tiles
    unsigned char elem[kClipTensors];  // 0 = fp32, 1 = bf16, 2 = fp16
    int tensors;
    int far;                        // clip: all tensors together exceed the last-level cache
    int add;                        // squares: to the sums that launches before left
    double* parts;                  // [kClipParts]
    float* norm;                    // clip: where the norm goes, or null
    float limit;
};

hipError_t launch_clip_squares(const ClipParams& p, hipStream_t stream);
// the norm from the sums, and data times min(1, limit / norm) into out (p.tensors = 0: the norm alone)
hipError_t launch_clip(const ClipParams& p, hipStream_t stream);

}  // namespace leet
