// What api.hip hands to grad_ops.hip: the tensors of a list as the kernels see them.
#pragma once
#include "pbdr_internal.h"

namespace pbdr {

enum { kGradF32 = 0, kGradF16 = 1, kGradBF16 = 2 };

constexpr int kGradBlock = 256;
constexpr int kDenseVecs = 2;                     // vectors of a lane in a unit of a tensor without mask (2, 4, 8: the same within 2 %)
// Planes of a masked unit, all of which are read before the first is used. Sums and scaling: 4 (8M points, a quarter used: norm
// 97 us, clipped into buffers of their own 386; 8 planes 98 and 425, 6 between). Adam reads four vectors a plane: 2 (8M points, a
// quarter used, with the norm: 736 us; 1 plane 766, 3 planes 740, 4 750; 1M points 207 each; 200,003 surfels 56, 3 and 4 planes 57).
constexpr uint32_t kMaskPlanes = 4;
constexpr uint32_t kAdamPlanes = 2;
// Workgroups of a launch that sums, eight per compute unit: units that need no reading leave gaps in masked tensors (8M points, a
// quarter used: norm 99 us; 1,024 workgroups 113, 512 168; 4,096 103). Tensors without mask take half as many for their units, and
// stream better so (1M points: norm 43.7 us against 45.8).
constexpr uint32_t kGradBlocks = 2048;
constexpr uint32_t kLineFloats = 32;              // of a cache line
constexpr uint32_t kMostBlocks = 1u << 23;        // of a launch: fewer than 2^32 threads
// Tensors of one launch: their table is a kernel argument, of 4 KB at most. A model's own tensors fit the short one, whose launch
// costs the host less (4,096 points: clipped 10.8 us with the long table, 10.1 with the short; norm and Adam 14.3 and 13.7).
constexpr uint32_t kGradTableTensors = 88, kAdamTableTensors = 48, kShortTable = 8;
constexpr int kGradMaxTensors = 1024;             // of a call

struct GradTensorDev {
    const void* data;          // [planes][n]
    void* out;
    const uint8_t* visible;    // [n], or null: all
    uint64_t n;
    uint32_t planes : 24, dtype : 8;
    uint32_t units;
};
template <uint32_t kMost>
struct GradTable {
    static constexpr uint32_t kTensors = kMost;
    uint32_t count, blocks;
    uint32_t first[kMost + 1];                    // first workgroup of each tensor, and their number
    GradTensorDev t[kMost];
};

struct AdamTensorDev {
    float *param, *grad, *m, *v;
    const uint8_t* visible;
    uint64_t n;
    uint32_t planes, units;
    float step_size;
};
template <uint32_t kMost>
struct AdamTable {
    static constexpr uint32_t kTensors = kMost;
    uint32_t count, blocks;
    uint32_t first[kMost + 1];
    AdamDev adam;              // of every tensor but for step_size
    AdamTensorDev t[kMost];
};

// a slot per workgroup that sums: a table has kGradBlocks of them at most, and one more per tensor whose units do not come out even
constexpr uint32_t kGradSlots = kGradBlocks + kGradTableTensors;
// Workgroups up to which one launch sums and finishes: 32 to 128 workgroups 8.3 us a call, 11 with a launch of its own for the
// end; 250 workgroups 10.5 and 10.3; 500 15.3 and 10.5.
constexpr uint32_t kAloneSlots = 128;
// Workgroups up to which every workgroup that scales adds the slots up itself: 128 to 500 workgroups 11.9 us a call, 13.2 to 15.7
// with a launch between; 1,000 workgroups 12.1 and 15.7; 2,000 16.3 and 15.9.
constexpr uint32_t kInlineSlots = 1024;
struct GradWorkspace {
    uint32_t done;             // workgroups of the running launch that have stored their sum; zero between launches
    double total;              // of the tables before the running one
    double slot[kGradSlots];
};

hipError_t launch_grad(int count, const GradTensorDev* list, float max_norm, float* result, GradWorkspace* ws, bool clip, hipStream_t s);
hipError_t launch_adam_list(int count, const AdamTensorDev* list, const AdamDev& adam, const float* result, hipStream_t s);

}  // namespace pbdr
