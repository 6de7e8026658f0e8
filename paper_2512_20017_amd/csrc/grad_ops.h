// What api.hip hands to grad_ops.hip: the tensors of a list as the kernels see them.
#pragma once
#include "pbdr_internal.h"

namespace pbdr {

enum { kGradF32 = 0, kGradF16 = 1, kGradBF16 = 2 };

constexpr int kGradBlock = 256;
constexpr int kDenseVecs = 4;
constexpr int kAdamVecs = 1;
constexpr uint32_t kMaskPlanes = 8;
// Planes of a masked unit: Adam reads four vectors a plane, all of a unit before the first is used. At 8M points, a quarter of
// them used, 3 planes take 914 us with the norm, 4 take 919, 6 take 943, 8 in pairs 926; attributes have 1, 2, 3, 4 or 3K planes.
constexpr uint32_t kAdamPlanes = 3;
constexpr uint32_t kGradBlocks = 2048;            // workgroups of a launch that sums or scales (and one more per tensor at most)
constexpr uint32_t kAdamBlocks = 1u << 20;        // enough for a unit each: 2,048 workgroups that take several took 10 % longer
constexpr int kGradTableTensors = 64;             // tensors of one launch: the table is a kernel argument
constexpr int kAdamTableTensors = 32;
constexpr int kGradMaxTensors = 1024;             // of a call

struct GradTensorDev {
    const void* data;          // [planes][n]
    void* out;
    const uint8_t* visible;    // [n], or null: all
    uint64_t n, count;         // count = planes * n
    uint32_t planes, units;
    int32_t dtype;
};
struct GradTable {
    int count;
    uint32_t first[kGradTableTensors + 1];        // first workgroup of each tensor, and their number
    GradTensorDev t[kGradTableTensors];
};

struct AdamTensorDev {
    float *param, *grad, *m, *v;
    const uint8_t* visible;
    uint64_t n, count;
    uint32_t planes, units;
    float step_size;
};
struct AdamTable {
    int count;
    uint32_t first[kAdamTableTensors + 1];
    AdamDev adam;              // of every tensor but for step_size
    AdamTensorDev t[kAdamTableTensors];
};

// workspace: the running total, then a slot per workgroup
constexpr size_t kGradSlotsAt = 256;
constexpr size_t kGradWorkspace = kGradSlotsAt + (kGradBlocks + kGradTableTensors) * sizeof(double);

hipError_t launch_grad_norm(int count, const GradTensorDev* list, float max_norm, float* result, char* ws, hipStream_t s);
hipError_t launch_grad_scale(int count, const GradTensorDev* list, const float* result, hipStream_t s);
hipError_t launch_adam_list(int count, const AdamTensorDev* list, const AdamDev& adam, const float* result, hipStream_t s);

}  // namespace pbdr
