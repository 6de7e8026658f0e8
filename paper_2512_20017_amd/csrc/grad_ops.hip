// Between the backward pass and the update: the global norm of the gradient over a list of tensors, its clipping, and selective
// Adam over a list with the clipping factor applied on the way (train_ops.hip has Adam for one tensor).
//
//   norm = sqrt(sum of g^2 over the used entries of all tensors);  scale = max_norm / norm where norm > max_norm, else 1
//
// All three are bound by HBM: two to sixteen operations per value read, no reuse. Squares are summed in fp64: a gradient of a mean
// over 6M values lies around 1e-7, and squares of fp32 numbers (1e-90 to 1e77) leave the range of fp32 on both sides. The fp64 adds
// cost no time beside the loads. No atomics on numbers: every workgroup has a fixed part of one tensor and a slot for its sum, and
// the slots are added in a fixed order, so the result is the same from run to run.
//
// A tensor is cut into units. Without a mask it is one row of planes * n values, and a unit is kDenseVecs vectors of 16 bytes per
// lane. With a mask a unit is one vector of points per lane and up to kMaskPlanes planes: the mask is read once for all of them,
// and a lane that has no used point reads nothing else. A lane that has one reads whole vectors, all planes of the unit at once.
// A device copy moves 5.4 TB/s here (read + written), a fill 7.
#include "grad_ops.h"
#include "wave_ops.h"

#include <cmath>

namespace pbdr {

template <int kDtype> struct GradType;
template <> struct GradType<kGradF32> { using T = float; };
template <> struct GradType<kGradF16> { using T = _Float16; };
template <> struct GradType<kGradBF16> { using T = __bf16; };

// 16 bytes of values; rows of a masked tensor begin at any multiple of a value's size
template <class T> struct GradVec {
    static constexpr int kN = 16 / sizeof(T);
    typedef T V __attribute__((ext_vector_type(kN), aligned(sizeof(T))));
};

// The end of a row: values at and after `at`, zero beyond its n values. One round trip: what lies beyond reads the last value.
template <class T>
__device__ __forceinline__ typename GradVec<T>::V load_end(const T* row, uint64_t at, uint64_t n)
{
    typename GradVec<T>::V v;
#pragma unroll
    for (int k = 0; k < GradVec<T>::kN; ++k) v[k] = row[min(at + k, n - 1)];
#pragma unroll
    for (int k = 0; k < GradVec<T>::kN; ++k) v[k] = at + k < n ? (T)v[k] : (T)0.f;
    return v;
}

// the bytes of the mask for kN consecutive points, zero beyond the last point
template <int kN> struct MaskOf;
template <> struct MaskOf<4> { using T = uint32_t; };
template <> struct MaskOf<8> { using T = uint64_t; };
template <int kN>
__device__ __forceinline__ typename MaskOf<kN>::T mask_bytes(const uint8_t* __restrict__ visible, uint64_t at, uint64_t n)
{
    using M = typename MaskOf<kN>::T;
    if (at + kN <= n) return *reinterpret_cast<const M*>(visible + at);
    if (at >= n) return 0;
    uint8_t byte[kN];
#pragma unroll
    for (int k = 0; k < kN; ++k) byte[k] = visible[min(at + k, n - 1)];
    M m = 0;
#pragma unroll
    for (int k = 0; k < kN; ++k) m |= at + k < n ? (M)byte[k] << (8 * k) : (M)0;
    return m;
}
template <int kN>
__device__ __forceinline__ bool used(typename MaskOf<kN>::T mask, int k)
{
    return ((uint32_t)(mask >> (8 * k)) & 0xffu) != 0u;
}

// a unit of a masked tensor: this lane's points and the planes
struct MaskedUnit {
    uint64_t at;
    uint32_t p0, p1;
};
template <int kN>
__device__ __forceinline__ MaskedUnit masked_unit(uint32_t u, uint32_t planes)
{
    const uint32_t groups = (planes + kMaskPlanes - 1) / kMaskPlanes, seg = u / groups, p0 = (u - seg * groups) * kMaskPlanes;
    return MaskedUnit{((uint64_t)seg * kGradBlock + threadIdx.x) * kN, p0, min(p0 + kMaskPlanes, planes)};
}

template <int kN>
__device__ __forceinline__ typename MaskOf<kN>::T unit_mask(const GradTensorDev& t, uint32_t u)
{
    if (u >= t.units) return 0;
    return mask_bytes<kN>(t.visible, masked_unit<kN>(u, t.planes).at, t.n);
}

template <class T>
__device__ __forceinline__ void add_square(double& acc, T v)
{
    const double d = (double)(float)v;
    acc = fma(d, d, acc);
}

template <int kDtype>
__device__ double sum_squares(const GradTensorDev& t, uint32_t first, uint32_t step)
{
    using T = typename GradType<kDtype>::T;
    using Vec = typename GradVec<T>::V;
    constexpr int kN = GradVec<T>::kN;
    const T* __restrict__ data = static_cast<const T*>(t.data);
    const uint64_t count = t.n * t.planes;
    double acc[4] = {0., 0., 0., 0.};
    if (t.visible == nullptr) {
        constexpr uint32_t kUnit = kGradBlock * kN * kDenseVecs;
        for (uint32_t u = first; u < t.units; u += step) {
            const uint64_t base = (uint64_t)u * kUnit + threadIdx.x * kN;
            Vec v[kDenseVecs];
            if ((uint64_t)(u + 1) * kUnit <= count) {
#pragma unroll
                for (int j = 0; j < kDenseVecs; ++j) v[j] = *reinterpret_cast<const Vec*>(data + base + j * kGradBlock * kN);
            } else {
#pragma unroll
                for (int j = 0; j < kDenseVecs; ++j) v[j] = load_end(data, base + j * kGradBlock * kN, count);
            }
#pragma unroll
            for (int j = 0; j < kDenseVecs; ++j)
#pragma unroll
                for (int k = 0; k < kN; ++k) add_square(acc[k & 3], (T)v[j][k]);
        }
    } else {
        typename MaskOf<kN>::T next = unit_mask<kN>(t, first);
        for (uint32_t u = first; u < t.units; u += step) {
            const typename MaskOf<kN>::T mask = next;
            next = unit_mask<kN>(t, u + step);      // on its way while this unit's values are
            if (mask == 0) continue;
            const MaskedUnit w = masked_unit<kN>(u, t.planes);
            const T* row = data + (uint64_t)w.p0 * t.n;
            Vec v[kMaskPlanes];
            if (w.at + kN <= t.n) {
#pragma unroll
                for (uint32_t i = 0; i < kMaskPlanes; ++i)
                    if (w.p0 + i < w.p1) v[i] = *reinterpret_cast<const Vec*>(row + i * t.n + w.at);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < kMaskPlanes; ++i)
                    if (w.p0 + i < w.p1) v[i] = load_end(row + i * t.n, w.at, t.n);
            }
#pragma unroll
            for (uint32_t i = 0; i < kMaskPlanes; ++i)
                if (w.p0 + i < w.p1) {
#pragma unroll
                    for (int k = 0; k < kN; ++k) add_square(acc[k & 3], used<kN>(mask, k) ? (T)v[i][k] : (T)0.f);
                }
        }
    }
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

// the tensor whose workgroups include `block`
template <class Table>
__device__ __forceinline__ uint32_t find_tensor(const Table& tab, uint32_t block)
{
    uint32_t lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) >> 1;
        if (tab.first[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// what the end of a sum needs
struct GradEnd {
    GradWorkspace* ws;
    float* result;
    float* norms;              // of the table's tensors
    float max_norm;
    int first_table, last_table;
};

// One workgroup of kThreads: adds the slots of each tensor of the table, and the tensors to the total of the tables before it;
// returns the factor. All slots are on their way before the first is waited for (one by one they took 8 us instead of 5).
// The order of the additions depends on the table alone. kAgent: the slots were stored by the running launch.
template <int kThreads, int kSlots, bool kAgent, class Table>
__device__ __forceinline__ float finish(const Table& tab, const GradEnd& end, bool write)
{
    __shared__ double sSlot[kSlots];
    __shared__ double sTensor[Table::kTensors];
    __shared__ uint32_t sFirst[Table::kTensors + 1];
    __shared__ float sScale;
    static_assert(kThreads > Table::kTensors, "");
    constexpr int kEach = (kSlots + kThreads - 1) / kThreads;
    const uint32_t count = tab.count, blocks = tab.blocks, lane = threadIdx.x & 63;
    double mine[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t i = j * kThreads + threadIdx.x;
        mine[j] = i >= blocks ? 0. : kAgent ? __hip_atomic_load(&end.ws->slot[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : end.ws->slot[i];
    }
    if (threadIdx.x <= count) sFirst[threadIdx.x] = tab.first[threadIdx.x];
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j * kThreads + threadIdx.x < kSlots) sSlot[j * kThreads + threadIdx.x] = mine[j];
    __syncthreads();
    // tensors of few slots: sixteen lanes each
    for (uint32_t t = threadIdx.x >> 4; t < count; t += kThreads / 16) {
        const uint32_t from = sFirst[t], to = sFirst[t + 1];
        if (to - from > 64) continue;
        double s = 0.;
        for (uint32_t i = from + (lane & 15); i < to; i += 16) s += sSlot[i];
        s = row_sum(s);
        if ((lane & 15) == 15) sTensor[t] = s;
    }
    for (uint32_t t = threadIdx.x >> 6; t < count; t += kThreads / 64) {
        const uint32_t from = sFirst[t], to = sFirst[t + 1];
        if (to - from <= 64) continue;
        double s = 0.;
#pragma unroll 4
        for (uint32_t i = from + lane; i < to; i += 64) s += sSlot[i];
        s = wave_sum(s);
        if (lane == 0) sTensor[t] = s;
    }
    __syncthreads();
    if (write && threadIdx.x < count) end.norms[threadIdx.x] = (float)sqrt(sTensor[threadIdx.x]);
    if (threadIdx.x < 64) {
        double s = 0.;
        for (uint32_t t = lane; t < count; t += 64) s += sTensor[t];
        s = wave_sum(s);
        if (lane == 0) {
            if (!end.first_table) s += end.ws->total;
            const double norm = sqrt(s);
            const float scale = !(norm <= 1.7976931348623157e308) ? 0.f : norm > (double)end.max_norm ? (float)((double)end.max_norm / norm) : 1.f;
            sScale = scale;
            if (write && end.last_table) {
                end.result[0] = (float)norm;
                end.result[1] = scale;
            } else if (write) {
                end.ws->total = s;
            }
        }
    }
    __syncthreads();
    return sScale;
}

template <class Table>
__global__ __launch_bounds__(1024) void k_grad_finish(GradEnd end, Table tab)
{
    finish<1024, kGradSlots, false>(tab, end, true);
}

// Every workgroup sums its part into a slot. 1M points SH3 (236 MB): 39 us, 6.0 TB/s; 8M points of which a quarter is used (466 MB):
// 95 us, 4.9 TB/s; the counters say 574 MB, since each of a stretch's sixteen units asks for the mask (128 MB in all, part of it from the
// caches) and runs of used points end inside lines.
// Masks that come several units early, units of more planes and 4,096 workgroups made the latter 3 to 40 % slower.
// kAlone: the last workgroup to be done finishes in the same launch: slots go past the caches of the eight dies (agent scope), and
// the counter is left at zero for the next launch.
template <bool kAlone, class Table>
__global__ __launch_bounds__(kGradBlock, 8) void k_grad_squares(GradEnd end, Table tab)
{
    __shared__ double sWave[kGradBlock / 64];
    __shared__ bool sLast;
    if (!kAlone || tab.blocks) {      // else one workgroup has come to write the norm of nothing
        const uint32_t ti = find_tensor(tab, blockIdx.x);
        const GradTensorDev& t = tab.t[ti];
        const uint32_t first = blockIdx.x - tab.first[ti], step = tab.first[ti + 1] - tab.first[ti];
        double s;
        if (t.dtype == kGradF32) s = sum_squares<kGradF32>(t, first, step);
        else if (t.dtype == kGradF16) s = sum_squares<kGradF16>(t, first, step);
        else s = sum_squares<kGradBF16>(t, first, step);
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) sWave[threadIdx.x >> 6] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double r = sWave[0];
        for (int w = 1; w < kGradBlock / 64; ++w) r += sWave[w];
        if (kAlone) {
            __hip_atomic_store(&end.ws->slot[blockIdx.x], r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sLast = __hip_atomic_fetch_add(&end.ws->done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
        } else {
            end.ws->slot[blockIdx.x] = r;
        }
    }
    if (!kAlone) return;
    __syncthreads();
    if (!sLast) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    finish<kGradBlock, kAloneSlots, true>(tab, end, true);
    if (threadIdx.x == 0) __hip_atomic_store(&end.ws->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// scale * g in fp32, rounded once more to the tensor's type; a factor of zero makes zeros of everything, NaN and infinities included
template <class T>
__device__ __forceinline__ T scaled(T g, float scale)
{
    return scale == 0.f ? (T)0.f : (T)((float)g * scale);
}

// what is written is not read again here: it leaves the last-level cache to the gradient
template <class Vec, class T>
__device__ __forceinline__ void store_vec(Vec v, T* to)
{
    __builtin_nontemporal_store(v, reinterpret_cast<Vec*>(to));
}

// units that a workgroup which scales takes in a row
__host__ __device__ __forceinline__ uint32_t scale_run(const GradTensorDev& t) { return t.visible && t.n >= kManyPoints ? kScaleRun : 1; }

template <int kDtype>
__device__ void write_scaled(const GradTensorDev& t, float scale, uint32_t begin, uint32_t end)
{
    using T = typename GradType<kDtype>::T;
    using Vec = typename GradVec<T>::V;
    constexpr int kN = GradVec<T>::kN;
    const T* data = static_cast<const T*>(t.data);      // may be the output
    T* out = static_cast<T*>(t.out);
    const bool apart = out != data;
    const uint64_t count = t.n * t.planes;
    if (t.visible == nullptr) {
        constexpr uint32_t kUnit = kGradBlock * kN * kDenseVecs;
        for (uint32_t u = begin; u < end; ++u) {
            const uint64_t base = (uint64_t)u * kUnit + threadIdx.x * kN;
            Vec v[kDenseVecs];
            if ((uint64_t)(u + 1) * kUnit <= count) {
#pragma unroll
                for (int j = 0; j < kDenseVecs; ++j) v[j] = *reinterpret_cast<const Vec*>(data + base + j * kGradBlock * kN);
#pragma unroll
                for (int j = 0; j < kDenseVecs; ++j) {
#pragma unroll
                    for (int k = 0; k < kN; ++k) v[j][k] = scaled((T)v[j][k], scale);
                    store_vec(v[j], out + base + j * kGradBlock * kN);
                }
            } else {
#pragma unroll
                for (int j = 0; j < kDenseVecs; ++j) v[j] = load_end(data, base + j * kGradBlock * kN, count);
#pragma unroll
                for (int j = 0; j < kDenseVecs; ++j)
#pragma unroll
                    for (int k = 0; k < kN; ++k)
                        if (base + j * kGradBlock * kN + k < count) out[base + j * kGradBlock * kN + k] = scaled((T)v[j][k], scale);
            }
        }
    } else {
        for (uint32_t u = begin; u < end; ++u) {
            const MaskedUnit w = masked_unit<kN>(u, t.planes);
            const typename MaskOf<kN>::T mask = mask_bytes<kN>(t.visible, w.at, t.n);
            if (mask == 0) continue;
            const uint64_t o = (uint64_t)w.p0 * t.n + w.at;
            if (w.at + kN <= t.n) {
                bool all = true;
#pragma unroll
                for (int k = 0; k < kN; ++k) all = all && used<kN>(mask, k);
                Vec v[kMaskPlanes], old[kMaskPlanes] = {};      // old: of the lanes that need it, on its way together with v
#pragma unroll
                for (uint32_t j = 0; j < kMaskPlanes; ++j)
                    if (w.p0 + j < w.p1) v[j] = *reinterpret_cast<const Vec*>(data + o + (uint64_t)j * t.n);
                // an unused entry among used ones is read and written back: stores that leave holes in a line cost the memory more
                if (!all && apart) {
#pragma unroll
                    for (uint32_t j = 0; j < kMaskPlanes; ++j)
                        if (w.p0 + j < w.p1) old[j] = *reinterpret_cast<const Vec*>(out + o + (uint64_t)j * t.n);
                }
#pragma unroll
                for (uint32_t j = 0; j < kMaskPlanes; ++j)
                    if (w.p0 + j < w.p1) {
#pragma unroll
                        for (int k = 0; k < kN; ++k) v[j][k] = used<kN>(mask, k) ? scaled((T)v[j][k], scale) : apart ? (T)old[j][k] : (T)v[j][k];
                        store_vec(v[j], out + o + (uint64_t)j * t.n);
                    }
            } else {
                Vec v[kMaskPlanes];
#pragma unroll
                for (uint32_t j = 0; j < kMaskPlanes; ++j)
                    if (w.p0 + j < w.p1) v[j] = load_end(data + (uint64_t)(w.p0 + j) * t.n, w.at, t.n);
#pragma unroll
                for (uint32_t j = 0; j < kMaskPlanes; ++j)
#pragma unroll
                    for (int k = 0; k < kN; ++k)
                        if (w.p0 + j < w.p1 && used<kN>(mask, k)) out[o + (uint64_t)j * t.n + k] = scaled((T)v[j][k], scale);
            }
        }
    }
}

// One unit per workgroup (2,048 workgroups that walk over the units took 4 to 10 % longer), four of a masked tensor of many points.
// 1M points SH3: 66 us for 236 MB read and written, 7.2 TB/s: most of what is read is still in the last-level cache, since nothing
// else of the two passes goes there. 2M surfels, twice what it holds: 148 us, 6.5 TB/s. 8M points of which a quarter is used: 234 us
// into another buffer, of which it reads the lines that are used in part, 0.32 GB, 178 us in place. kFinish: every workgroup adds the
// slots up for itself, one writes the result: for small lists, whose sums then need no ending.
template <bool kFinish, class Table>
__global__ __launch_bounds__(kGradBlock, 8) void k_grad_scale(GradEnd end, Table tab)
{
    const uint32_t block = gridDim.x - 1 - blockIdx.x;      // backwards: the end of the gradient was read last
    const uint32_t ti = find_tensor(tab, block);
    const GradTensorDev& t = tab.t[ti];
    const float scale = kFinish ? finish<kGradBlock, kInlineSlots, false>(tab, end, blockIdx.x == 0) : end.result[1];
    if (scale == 1.f && t.out == t.data) return;      // nothing would change
    const uint32_t run = tab.each * scale_run(t), begin = (block - tab.first[ti]) * run, stop = min(begin + run, t.units);
    if (t.dtype == kGradF32) write_scaled<kGradF32>(t, scale, begin, stop);
    else if (t.dtype == kGradF16) write_scaled<kGradF16>(t, scale, begin, stop);
    else write_scaled<kGradBF16>(t, scale, begin, stop);
}

// Adam, a unit per workgroup: 28 bytes an entry, the gradient's four among them (32 with zero_grad). 1M points SH3, 60 % used: 172 us for
// 0.96 GB, 5.6 TB/s, part of the gradient from the last-level cache; 8M points, a quarter used: 647 us for 3.2 GB, 5.0 TB/s (3.46 GB and
// 5.35 TB/s by the counters). With ordinary loads and stores of parameters and moments 203 us at 1M points, forwards 680 us at 8M.
// A lane takes four entries of a row, and a workgroup's stretch of a row begins on a cache line of the moments, wherever the row
// begins: lines that two wavefronts write in part cost 12 % of the whole (with the norm 200,003 surfels 64 us, 200,000 surfels 57). So
// lanes may stand before the row's begin, and the mask is read at the plane's own offset. The vectors of parameter, gradient and
// moments lie on 16 bytes each.
struct AdamVec {
    GradVec<float>::V p, g, m, v;
};

// the bytes of the mask of four points from `at` on, or ones without a mask; zero outside the row
template <bool kMasked>
__device__ __forceinline__ uint32_t adam_mask(const uint8_t* __restrict__ visible, int64_t at, int64_t n)
{
    struct __attribute__((packed)) Any { uint32_t bytes; };
    if (at >= 0 && at + 4 <= n) return kMasked ? reinterpret_cast<const Any*>(visible + at)->bytes : ~0u;
    if (at >= n || at <= -4) return 0;
    uint8_t byte[4] = {1, 1, 1, 1};
    if (kMasked) {
#pragma unroll
        for (int k = 0; k < 4; ++k) byte[k] = visible[max((int64_t)0, min(at + k, n - 1))];
    }
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) m |= at + k >= 0 && at + k < n ? (uint32_t)byte[k] << (8 * k) : 0u;
    return m;
}
__device__ __forceinline__ GradVec<float>::V load_near(const float* row, int64_t at, int64_t n)      // at an end of the row
{
    GradVec<float>::V v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = row[max((int64_t)0, min(at + k, n - 1))];
    return v;
}
__device__ __forceinline__ AdamVec adam_load(const AdamTensorDev& t, uint64_t row, int64_t at, int64_t n)
{
    using Vec = GradVec<float>::V;
    if (at < 0 || at + 4 > n) return AdamVec{load_near(t.param + row, at, n), load_near(t.grad + row, at, n), load_near(t.m + row, at, n), load_near(t.v + row, at, n)};
    // parameters and moments pass by the last-level cache, which holds part of the gradient that the norm has just read
    return AdamVec{__builtin_nontemporal_load(reinterpret_cast<const Vec*>(t.param + row + at)), *reinterpret_cast<const Vec*>(t.grad + row + at),
                   __builtin_nontemporal_load(reinterpret_cast<const Vec*>(t.m + row + at)), __builtin_nontemporal_load(reinterpret_cast<const Vec*>(t.v + row + at))};
}
// g * scale is rounded to fp32 as a clipped gradient in memory would be; entries with a zero in the mask keep their bits
__device__ __forceinline__ void adam_step(const AdamDev& c, float scale, uint32_t mask, AdamVec& x)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a = x.p[k], b = x.m[k], d = x.v[k];
        adam_one(c, a, scaled((float)x.g[k], scale), b, d);
        if (used<4>(mask, k)) {
            x.p[k] = a; x.m[k] = b; x.v[k] = d; x.g[k] = 0.f;
        }
    }
}
__device__ __forceinline__ void adam_store(const AdamDev& c, uint32_t mask, const AdamTensorDev& t, uint64_t row, int64_t at, int64_t n, const AdamVec& x)
{
    using Vec = GradVec<float>::V;
    if (at >= 0 && at + 4 <= n) {
        __builtin_nontemporal_store(x.p, reinterpret_cast<Vec*>(t.param + row + at));
        __builtin_nontemporal_store(x.m, reinterpret_cast<Vec*>(t.m + row + at));
        __builtin_nontemporal_store(x.v, reinterpret_cast<Vec*>(t.v + row + at));
        if (c.zero_grad) *reinterpret_cast<Vec*>(t.grad + row + at) = x.g;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (used<4>(mask, k)) {
                const uint64_t i = row + at + k;
                t.param[i] = x.p[k]; t.m[i] = x.m[k]; t.v[i] = x.v[k];
                if (c.zero_grad) t.grad[i] = 0.f;
            }
    }
}

// Without a mask the tensor is one row. With one a unit is t.unit planes of a stretch, taken one at a time.
template <bool kMasked>
__device__ __forceinline__ void adam_tensor(const AdamTensorDev& t, const AdamDev& c, float scale, uint32_t begin, uint32_t end)
{
    const uint32_t rows = kMasked ? t.planes : 1, unit = kMasked ? t.unit : 1, groups = (rows + unit - 1) / unit;
    const int64_t n = (int64_t)(kMasked ? t.n : t.n * t.planes);
    for (uint32_t u = begin; u < end; ++u) {
        const uint32_t seg = u / groups, p0 = (u - seg * groups) * unit, p1 = min(p0 + unit, rows);
        const int64_t at0 = ((int64_t)seg * kGradBlock + threadIdx.x) * 4;
        if (kMasked && unit > 1) {      // leave at once if no lane will have a used point, wherever the planes begin on a line
            const uint32_t before = threadIdx.x < kLineFloats / 4 ? adam_mask<true>(t.visible, at0 - (int64_t)kLineFloats, n) : 0u;
            if (!__syncthreads_or((int)(adam_mask<true>(t.visible, at0, n) | before))) continue;
        }
#pragma unroll 1
        for (uint32_t p = p0; p < p1; ++p) {
            const uint64_t row = (uint64_t)p * n;
            const int64_t at = at0 - (int64_t)((reinterpret_cast<uintptr_t>(t.m + row) >> 2) & (kLineFloats - 1));
            const uint32_t mask = adam_mask<kMasked>(t.visible, at, n);
            if (mask == 0) continue;
            AdamVec x = adam_load(t, row, at, n);
            adam_step(c, scale, mask, x);
            adam_store(c, mask, t, row, at, n, x);
        }
    }
}

template <class Table>
__global__ __launch_bounds__(kGradBlock) void k_adam_list(Table tab, const float* __restrict__ result)
{
    const uint32_t block = gridDim.x - 1 - blockIdx.x;      // backwards: the norm has read the end of the gradient last
    const uint32_t ti = find_tensor(tab, block);
    const AdamTensorDev& t = tab.t[ti];
    const float scale = result ? result[1] : 1.f;
    AdamDev c = tab.adam;
    c.step_size = t.step_size;
    const uint32_t begin = (block - tab.first[ti]) * tab.each, end = min(begin + tab.each, t.units);
    if (t.visible) adam_tensor<true>(t, c, scale, begin, end);
    else adam_tensor<false>(t, c, scale, begin, end);
}

static uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

static uint32_t units_of(const GradTensorDev& t)
{
    const uint64_t vec = t.dtype == kGradF32 ? 4 : 8;
    if (t.n == 0 || t.planes == 0) return 0;
    if (t.visible == nullptr) return (uint32_t)ceil_div(t.n * t.planes, kGradBlock * vec * kDenseVecs);
    return (uint32_t)(ceil_div(t.n, kGradBlock * vec) * ceil_div(t.planes, kMaskPlanes));
}
static uint32_t adam_unit(const AdamTensorDev& t) { return t.n < kFewPoints ? 1 : t.n < kManyPoints ? 4 : 8; }
static uint32_t units_of(const AdamTensorDev& t)      // lanes may stand before the begin of a row by a line less one
{
    if (t.n == 0 || t.planes == 0) return 0;
    if (t.visible == nullptr) return (uint32_t)ceil_div(t.n * t.planes + kLineFloats - 1, kGradBlock * 4);
    return (uint32_t)(ceil_div(t.n + kLineFloats - 1, kGradBlock * 4) * ceil_div(t.planes, t.unit));
}

// The workgroups that sum a table: one per unit, or, with more than kGradBlocks units, that many and each as many units.
template <class Table>
static uint32_t cut_sums(Table& tab, uint64_t units)
{
    const uint64_t each = units > kGradBlocks ? ceil_div(units, kGradBlocks) : 1;
    uint32_t at = 0;
    for (uint32_t i = 0; i < tab.count; ++i) {
        tab.first[i] = at;
        at += (uint32_t)ceil_div(tab.t[i].units, tab.t[i].visible || each == 1 ? each : 2 * each);
    }
    tab.each = 1;
    return tab.blocks = tab.first[tab.count] = at;
}

// The workgroups that scale or update a table: one per run of units, and longer runs only where a launch could not have as many.
template <class Table, class Run>
static uint32_t cut_runs(Table& tab, uint64_t units, Run run)
{
    tab.each = (uint32_t)ceil_div(units + 1, kMostBlocks);
    uint32_t at = 0;
    for (uint32_t i = 0; i < tab.count; ++i) {
        tab.first[i] = at;
        at += (uint32_t)ceil_div(tab.t[i].units, (uint64_t)tab.each * run(tab.t[i]));
    }
    return tab.blocks = tab.first[tab.count] = at;
}

// As many tensors of a list as the table holds; tensors without entries keep their place and get no unit.
template <class Table>
static uint64_t fill_table(Table& tab, const GradTensorDev* list, uint32_t count)
{
    uint64_t units = 0;
    tab.count = count < Table::kTensors ? count : Table::kTensors;
    for (uint32_t i = 0; i < tab.count; ++i) {
        tab.t[i] = list[i];
        units += tab.t[i].units = units_of(list[i]);
    }
    return units;
}

static_assert(sizeof(GradTable<kGradTableTensors>) + sizeof(GradEnd) <= 4096 && sizeof(AdamTable<kAdamTableTensors>) + sizeof(void*) <= 4096, "");

template <class Table>
static void grad_launches(uint32_t count, const GradTensorDev* list, float max_norm, float* result, GradWorkspace* ws, bool clip, hipStream_t s)
{
    Table tab;
    bool scaled = !clip;
    uint32_t at = 0;
    do {
        const uint64_t units = fill_table(tab, list + at, count - at);
        const uint32_t blocks = cut_sums(tab, units);
        const GradEnd end{ws, result, result + 2 + at, max_norm, at == 0, at + tab.count == count};
        const dim3 grid(blocks ? blocks : 1), block(kGradBlock);
        const bool alone = blocks <= kAloneSlots;
        const bool inlined = blocks && blocks <= kInlineSlots && units <= kGradBlocks && clip && end.first_table && end.last_table;      // a workgroup per unit
        {
            ProfScope prof(kKGradNorm, s);
            if (alone && !inlined) hipLaunchKernelGGL((k_grad_squares<true, Table>), grid, block, 0, s, end, tab);
            else hipLaunchKernelGGL((k_grad_squares<false, Table>), grid, block, 0, s, end, tab);
        }
        if (inlined) {
            ProfScope prof(kKGradScale, s);
            hipLaunchKernelGGL((k_grad_scale<true, Table>), grid, block, 0, s, end, tab);
            scaled = true;
        } else if (!alone) {
            ProfScope prof(kKGradFinish, s);
            hipLaunchKernelGGL(k_grad_finish<Table>, dim3(1), dim3(1024), 0, s, end, tab);
        }
        at += tab.count;
    } while (at < count);
    if (scaled) return;
    for (at = 0; at < count; at += tab.count) {
        const uint64_t units = fill_table(tab, list + at, count - at);
        const uint32_t blocks = cut_runs(tab, units, scale_run);
        if (blocks == 0) continue;
        const GradEnd end{ws, result, result + 2 + at, max_norm, 0, 0};
        ProfScope prof(kKGradScale, s);
        hipLaunchKernelGGL((k_grad_scale<false, Table>), dim3(blocks), dim3(kGradBlock), 0, s, end, tab);
    }
}

hipError_t launch_grad(int count, const GradTensorDev* list, float max_norm, float* result, GradWorkspace* ws, bool clip, hipStream_t s)
{
    if ((uint32_t)count <= kShortTable) grad_launches<GradTable<kShortTable>>(count, list, max_norm, result, ws, clip, s);
    else grad_launches<GradTable<kGradTableTensors>>(count, list, max_norm, result, ws, clip, s);
    return hipGetLastError();
}

template <class Table>
static void adam_launches(uint32_t count, const AdamTensorDev* list, const AdamDev& adam, const float* result, hipStream_t s)
{
    Table tab;
    tab.adam = adam;
    for (uint32_t at = 0; at < count; at += tab.count) {
        uint64_t units = 0;
        tab.count = count - at < Table::kTensors ? count - at : Table::kTensors;
        for (uint32_t i = 0; i < tab.count; ++i) {
            tab.t[i] = list[at + i];
            tab.t[i].unit = adam_unit(tab.t[i]);
            units += tab.t[i].units = units_of(tab.t[i]);
        }
        const uint32_t blocks = cut_runs(tab, units, [](const AdamTensorDev&) { return 1u; });
        if (blocks == 0) continue;
        ProfScope prof(kKAdamList, s);
        hipLaunchKernelGGL(k_adam_list<Table>, dim3(blocks), dim3(kGradBlock), 0, s, tab, result);
    }
}

hipError_t launch_adam_list(int count, const AdamTensorDev* list, const AdamDev& adam, const float* result, hipStream_t s)
{
    if ((uint32_t)count <= kShortTable) adam_launches<AdamTable<kShortTable>>(count, list, adam, result, s);
    else adam_launches<AdamTable<kAdamTableTensors>>(count, list, adam, result, s);
    return hipGetLastError();
}

}  // namespace pbdr
