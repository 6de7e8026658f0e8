// What api.hip hands to grad_ops.hip: the tensors of a list as the kernels see them.
#pragma once
#include "pbdr_internal.h"

namespace pbdr {

enum { kGradF32 = 0, kGradF16 = 1, kGradBF16 = 2 };

constexpr int kGradBlock = 256;
// Vectors of a lane in a unit of a tensor without mask: 1M points' norm 42.4 us, clipped 109; 4 vectors 43.3 and 116.
constexpr int kDenseVecs = 2;
// Planes of a masked unit that sums or scales, all of which are read before the first is used (8M points, a quarter used: norm 97 us;
// 2 planes 136, 3 planes 97, 8 planes 100, where scaling runs out of registers).
constexpr uint32_t kMaskPlanes = 4;
// A workgroup that finds nothing to do still costs half a nanosecond of the launch, and large scenes are seen in small part: many planes
// a unit pay where little is used, few where much is, since workgroups then end more evenly. The used share is not known on the
// host, so the number of points decides, where the gain of the one has come to outweigh the loss of the other. Norm and Adam, SH3, us:
//   points      5 % used, 1 / 4 / 8 planes     25 % used              60 % used
//   200,000       24 /  21 /  25                30 /  31 /  35         48 /  50 /  54
//   300,000       31 /  24 /  29                40 /  39 /  43         69 /  71 /  73
//   600,000       51 /  33 /  36                69 /  66 /  67        129 / 132 / 130
//   1,500,000    111 /  59 /  54               154 / 141 / 143        301 / 311 / 317
//   3,500,000      - / 118 / 102                 - / 320 / 323          - / 759 / 776
//   4,500,000      - / 149 / 130                 - / 411 / 413          - / 999 / 999
//   8,000,000      - / 253 / 217                 - / 735 / 748
// Scaling takes runs of kScaleRun units of a masked tensor from kManyPoints on: clipped with runs of one and of four, 3.5M points 79
// and 56 us at 5 %, 372 and 378 at 60 %; 4.5M points 99 and 72, 478 and 487; 8M points 172 and 131, 377 and 377 at 25 %. Smaller
// scenes keep the form that is better for what a batch usually sees of them (1.5M points: 41 and 34, 157 and 161).
constexpr uint64_t kFewPoints = 400000, kManyPoints = 4000000;
constexpr uint32_t kScaleRun = 4;
// Workgroups of a launch that sums, eight per compute unit: units that need no reading leave gaps in masked tensors (8M points, a
// quarter used: norm 97.5 us; 1,024 workgroups 113; 4,096 96.5, but 1M points without mask 45.9 instead of 42.4). Tensors without
// mask take half as many for their units, and stream better so (1M points 43.7 us against 45.8).
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
    uint32_t count, blocks, each;                 // each: factor on the units that a workgroup takes in a row
    uint32_t first[kMost + 1];                    // first workgroup of each tensor, and their number
    GradTensorDev t[kMost];
};

struct AdamTensorDev {
    float *param, *grad, *m, *v;
    const uint8_t* visible;
    uint64_t n;
    uint32_t planes, units;
    uint32_t unit;             // planes of a unit of a masked tensor
    float step_size;
};
template <uint32_t kMost>
struct AdamTable {
    static constexpr uint32_t kTensors = kMost;
    uint32_t count, blocks, each;
    uint32_t first[kMost + 1];
    AdamDev adam;              // of every tensor but for step_size
    AdamTensorDev t[kMost];
};

// a slot per workgroup that sums: a table has kGradBlocks of them at most, and one more per tensor whose units do not come out even
constexpr uint32_t kGradSlots = kGradBlocks + kGradTableTensors;
// Workgroups up to which one launch sums and finishes: up to 64 workgroups 6.1 us a call, 130 6.7, 250 8.8, 500 13.4; with a launch of
// its own for the end 9.2 to 9.5.
constexpr uint32_t kAloneSlots = 256;
// Workgroups up to which every workgroup that scales adds the slots up itself: 130 to 500 workgroups 9.7 us a call, 1,000 10.1, 2,000
// 13.6; with a launch between 13.0 to 14.0.
constexpr uint32_t kInlineSlots = 1024;
struct GradWorkspace {
    uint32_t done;             // workgroups of the running launch that have stored their sum; zero between launches
    double total;              // of the tables before the running one
    double slot[kGradSlots];
};

hipError_t launch_grad(int count, const GradTensorDev* list, float max_norm, float* result, GradWorkspace* ws, bool clip, hipStream_t s);
hipError_t launch_adam_list(int count, const AdamTensorDev* list, const AdamDev& adam, const float* result, hipStream_t s);

}  // namespace pbdr
