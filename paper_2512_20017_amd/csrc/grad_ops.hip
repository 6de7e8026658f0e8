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
#include "grad_ops.h"

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

// the bytes of the mask for kN consecutive points, zero beyond the last point
template <int kN>
__device__ __forceinline__ uint64_t mask_bytes(const uint8_t* __restrict__ visible, uint64_t at, uint64_t n)
{
    if (at + kN <= n) return kN == 4 ? *reinterpret_cast<const uint32_t*>(visible + at) : *reinterpret_cast<const uint64_t*>(visible + at);
    uint64_t m = 0;
    for (int k = 0; k < kN; ++k)
        if (at + k < n) m |= (uint64_t)visible[at + k] << (8 * k);
    return m;
}
template <int kN>
__device__ __forceinline__ bool used(uint64_t mask, int k)
{
    return ((kN == 4 ? (uint32_t)mask >> (8 * k) : (uint32_t)(mask >> (8 * k))) & 0xffu) != 0u;
}

// a unit of a masked tensor: this lane's points and the planes
struct MaskedUnit {
    uint64_t at;
    uint32_t p0, p1;
};
template <int kN, uint32_t kPlanes>
__device__ __forceinline__ MaskedUnit masked_unit(uint32_t u, uint32_t planes)
{
    const uint32_t groups = (planes + kPlanes - 1) / kPlanes;
    const uint32_t seg = u / groups, p0 = (u - seg * groups) * kPlanes;
    return MaskedUnit{((uint64_t)seg * kGradBlock + threadIdx.x) * kN, p0, min(p0 + kPlanes, planes)};
}

template <class T>
__device__ __forceinline__ void add_square(double& acc, T v)
{
    const double d = (double)(float)v;
    acc = fma(d, d, acc);
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

template <int kDtype>
__device__ double sum_squares(const GradTensorDev& t, uint32_t first, uint32_t step)
{
    using T = typename GradType<kDtype>::T;
    using Vec = typename GradVec<T>::V;
    constexpr int kN = GradVec<T>::kN;
    const T* __restrict__ data = static_cast<const T*>(t.data);
    double acc[4] = {0., 0., 0., 0.};
    if (t.visible == nullptr) {
        constexpr uint32_t kUnit = kGradBlock * kN * kDenseVecs;
        for (uint32_t u = first; u < t.units; u += step) {
            const uint64_t base = (uint64_t)u * kUnit + threadIdx.x * kN;
#pragma unroll
            for (int j = 0; j < kDenseVecs; ++j) {
                const uint64_t at = base + (uint64_t)j * kGradBlock * kN;
                if (at + kN <= t.count) {
                    const Vec v = *reinterpret_cast<const Vec*>(data + at);
#pragma unroll
                    for (int k = 0; k < kN; ++k) add_square(acc[k & 3], v[k]);
                } else {
                    for (uint64_t i = at; i < t.count; ++i) add_square(acc[0], data[i]);
                }
            }
        }
    } else {
        if (first >= t.units) return 0.;
        MaskedUnit w = masked_unit<kN, kMaskPlanes>(first, t.planes);
        uint64_t mask = mask_bytes<kN>(t.visible, w.at, t.n);
        for (uint32_t u = first;;) {
            // the next unit's mask is on its way while this unit's values come
            const bool more = u + step < t.units;
            MaskedUnit w1 = w;
            uint64_t mask1 = 0;
            if (more) {
                w1 = masked_unit<kN, kMaskPlanes>(u + step, t.planes);
                mask1 = mask_bytes<kN>(t.visible, w1.at, t.n);
            }
            if (mask != 0) {
                const T* row = data + (uint64_t)w.p0 * t.n + w.at;
                if (w.at + kN <= t.n) {
                    Vec v[kMaskPlanes];
#pragma unroll
                    for (uint32_t j = 0; j < kMaskPlanes; ++j)
                        if (w.p0 + j < w.p1) v[j] = *reinterpret_cast<const Vec*>(row + (uint64_t)j * t.n);
#pragma unroll
                    for (uint32_t j = 0; j < kMaskPlanes; ++j)
                        if (w.p0 + j < w.p1) {
#pragma unroll
                            for (int k = 0; k < kN; ++k) add_square(acc[k & 3], used<kN>(mask, k) ? (T)v[j][k] : (T)0.f);
                        }
                } else {
                    for (uint32_t p = w.p0; p < w.p1; ++p, row += t.n)
                        for (int k = 0; k < kN; ++k)
                            if (used<kN>(mask, k)) add_square(acc[0], row[k]);
                }
            }
            if (!more) break;
            u += step;
            w = w1;
            mask = mask1;
        }
    }
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

// the tensor whose workgroups include `block`
__device__ __forceinline__ int find_tensor(const GradTable& tab, uint32_t block)
{
    int lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.first[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__global__ __launch_bounds__(kGradBlock) void k_grad_squares(GradTable tab, double* __restrict__ slots)
{
    __shared__ double sWave[kGradBlock / 64];
    const int ti = find_tensor(tab, blockIdx.x);
    const GradTensorDev& t = tab.t[ti];
    const uint32_t first = blockIdx.x - tab.first[ti], step = tab.first[ti + 1] - tab.first[ti];
    double s;
    if (t.dtype == kGradF32) s = sum_squares<kGradF32>(t, first, step);
    else if (t.dtype == kGradF16) s = sum_squares<kGradF16>(t, first, step);
    else s = sum_squares<kGradBF16>(t, first, step);
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) sWave[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double r = sWave[0];
        for (int w = 1; w < kGradBlock / 64; ++w) r += sWave[w];
        slots[blockIdx.x] = r;
    }
}

// One workgroup: adds the slots of each tensor of the table, and the tensors to the total of the tables before it.
__global__ __launch_bounds__(1024) void k_grad_finish(GradTable tab, const double* __restrict__ slots, double* __restrict__ total, int first_table,
                                                      int last_table, float max_norm, float* __restrict__ result, float* __restrict__ norms)
{
    __shared__ double sTensor[kGradTableTensors];
    for (int t = threadIdx.x >> 6; t < tab.count; t += 16) {
        double s = 0.;
        for (uint32_t i = tab.first[t] + (threadIdx.x & 63); i < tab.first[t + 1]; i += 64) s += slots[i];
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) {
            sTensor[t] = s;
            norms[t] = (float)sqrt(s);
        }
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    double sum = first_table ? 0. : *total;
    for (int t = 0; t < tab.count; ++t) sum += sTensor[t];
    *total = sum;
    if (!last_table) return;
    const double norm = sqrt(sum);
    result[0] = (float)norm;
    result[1] = !(norm <= 1.7976931348623157e308) ? 0.f : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.f;
}

// scale * g in fp32, rounded once more to the tensor's type; a factor of zero makes zeros of everything, NaN and infinities included
template <class T>
__device__ __forceinline__ T scaled(T g, float scale)
{
    return scale == 0.f ? (T)0.f : (T)((float)g * scale);
}

template <int kDtype>
__device__ void write_scaled(const GradTensorDev& t, float scale, uint32_t first, uint32_t step)
{
    using T = typename GradType<kDtype>::T;
    using Vec = typename GradVec<T>::V;
    constexpr int kN = GradVec<T>::kN;
    const T* data = static_cast<const T*>(t.data);      // may be the output
    T* out = static_cast<T*>(t.out);
    if (t.visible == nullptr) {
        constexpr uint32_t kUnit = kGradBlock * kN * kDenseVecs;
        for (uint32_t u = first; u < t.units; u += step) {
            const uint64_t base = (uint64_t)u * kUnit + threadIdx.x * kN;
#pragma unroll
            for (int j = 0; j < kDenseVecs; ++j) {
                const uint64_t at = base + (uint64_t)j * kGradBlock * kN;
                if (at + kN <= t.count) {
                    Vec v = *reinterpret_cast<const Vec*>(data + at);
#pragma unroll
                    for (int k = 0; k < kN; ++k) v[k] = scaled((T)v[k], scale);
                    *reinterpret_cast<Vec*>(out + at) = v;
                } else {
                    for (uint64_t i = at; i < t.count; ++i) out[i] = scaled(data[i], scale);
                }
            }
        }
    } else {
        for (uint32_t u = first; u < t.units; u += step) {
            const MaskedUnit w = masked_unit<kN, kMaskPlanes>(u, t.planes);
            const uint64_t mask = mask_bytes<kN>(t.visible, w.at, t.n);
            if (mask == 0) continue;
            bool all = true;
#pragma unroll
            for (int k = 0; k < kN; ++k) all = all && used<kN>(mask, k);
            const uint64_t o = (uint64_t)w.p0 * t.n + w.at;
            if (w.at + kN <= t.n) {
                Vec v[kMaskPlanes];
#pragma unroll
                for (uint32_t j = 0; j < kMaskPlanes; ++j)
                    if (w.p0 + j < w.p1) v[j] = *reinterpret_cast<const Vec*>(data + o + (uint64_t)j * t.n);
#pragma unroll
                for (uint32_t j = 0; j < kMaskPlanes; ++j)
                    if (w.p0 + j < w.p1) {
                        T* to = out + o + (uint64_t)j * t.n;
#pragma unroll
                        for (int k = 0; k < kN; ++k) v[j][k] = scaled((T)v[j][k], scale);
                        if (all) *reinterpret_cast<Vec*>(to) = v[j];
                        else
#pragma unroll
                            for (int k = 0; k < kN; ++k)
                                if (used<kN>(mask, k)) to[k] = v[j][k];
                    }
            } else {
                for (uint32_t p = w.p0; p < w.p1; ++p)
                    for (int k = 0; k < kN; ++k) {
                        const uint64_t a = (uint64_t)p * t.n + w.at + k;
                        if (used<kN>(mask, k)) out[a] = scaled(data[a], scale);
                    }
            }
        }
    }
}

__global__ __launch_bounds__(kGradBlock) void k_grad_scale(GradTable tab, const float* __restrict__ result)
{
    const int ti = find_tensor(tab, blockIdx.x);
    const GradTensorDev& t = tab.t[ti];
    const float scale = result[1];
    if (scale == 1.f && t.out == t.data) return;      // nothing would change
    const uint32_t first = blockIdx.x - tab.first[ti], step = tab.first[ti + 1] - tab.first[ti];
    if (t.dtype == kGradF32) write_scaled<kGradF32>(t, scale, first, step);
    else if (t.dtype == kGradF16) write_scaled<kGradF16>(t, scale, first, step);
    else write_scaled<kGradBF16>(t, scale, first, step);
}

// one used entry: Adam with the clipped gradient, g * scale rounded to fp32 as a clipped gradient in memory would be
__device__ __forceinline__ void adam_clipped(const AdamDev& c, float scale, float* p, float* g, float* m, float* v)
{
    float x = *p, mm = *m, vv = *v;
    adam_one(c, x, scaled(*g, scale), mm, vv);
    *p = x; *m = mm; *v = vv;
    if (c.zero_grad) *g = 0.f;
}

// four entries, of which those with a zero in the mask get their own bits back
struct AdamVec {
    GradVec<float>::V p, g, m, v;
};
__device__ __forceinline__ AdamVec adam_load(const AdamTensorDev& t, uint64_t at)
{
    using Vec = GradVec<float>::V;
    return AdamVec{*reinterpret_cast<const Vec*>(t.param + at), *reinterpret_cast<const Vec*>(t.grad + at), *reinterpret_cast<const Vec*>(t.m + at),
                   *reinterpret_cast<const Vec*>(t.v + at)};
}
__device__ __forceinline__ void adam_store(const AdamDev& c, float scale, uint32_t mask, const AdamTensorDev& t, uint64_t at, AdamVec x)
{
    using Vec = GradVec<float>::V;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a = x.p[k], b = x.m[k], d = x.v[k];
        adam_one(c, a, scaled((float)x.g[k], scale), b, d);
        if (used<4>(mask, k)) {
            x.p[k] = a; x.m[k] = b; x.v[k] = d; x.g[k] = 0.f;
        }
    }
    *reinterpret_cast<Vec*>(t.param + at) = x.p;
    *reinterpret_cast<Vec*>(t.m + at) = x.m;
    *reinterpret_cast<Vec*>(t.v + at) = x.v;
    if (c.zero_grad) *reinterpret_cast<Vec*>(t.grad + at) = x.g;
}

__global__ __launch_bounds__(kGradBlock) void k_adam_list(AdamTable tab, const float* __restrict__ result)
{
    int lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const AdamTensorDev& t = tab.t[lo];
    const float scale = result ? result[1] : 1.f;
    AdamDev c = tab.adam;
    c.step_size = t.step_size;
    const uint32_t first = blockIdx.x - tab.first[lo], step = tab.first[lo + 1] - tab.first[lo];
    if (t.visible == nullptr) {
        constexpr uint32_t kUnit = kGradBlock * 4 * kAdamVecs;
        for (uint32_t u = first; u < t.units; u += step) {
            const uint64_t base = (uint64_t)u * kUnit + threadIdx.x * 4;
#pragma unroll
            for (int j = 0; j < kAdamVecs; ++j) {
                const uint64_t at = base + (uint64_t)j * kGradBlock * 4;
                if (at + 4 <= t.count) adam_store(c, scale, ~0u, t, at, adam_load(t, at));
                else
                    for (uint64_t i = at; i < t.count; ++i) adam_clipped(c, scale, t.param + i, t.grad + i, t.m + i, t.v + i);
            }
        }
    } else {
        for (uint32_t u = first; u < t.units; u += step) {
            const MaskedUnit w = masked_unit<4, kAdamPlanes>(u, t.planes);
            const uint32_t mask = (uint32_t)mask_bytes<4>(t.visible, w.at, t.n);
            if (mask == 0) continue;
            uint64_t at = (uint64_t)w.p0 * t.n + w.at;
            if (w.at + 4 <= t.n) {
                AdamVec x[kAdamPlanes];
#pragma unroll
                for (uint32_t j = 0; j < kAdamPlanes; ++j)
                    if (w.p0 + j < w.p1) x[j] = adam_load(t, at + j * t.n);
#pragma unroll
                for (uint32_t j = 0; j < kAdamPlanes; ++j)
                    if (w.p0 + j < w.p1) adam_store(c, scale, mask, t, at + j * t.n, x[j]);
            } else {
                for (uint32_t p = w.p0; p < w.p1; ++p, at += t.n)
                    for (int k = 0; k < 4; ++k)
                        if (used<4>(mask, k)) adam_clipped(c, scale, t.param + at + k, t.grad + at + k, t.m + at + k, t.v + at + k);
            }
        }
    }
}

// Units of a tensor, and how many workgroups share the units of a table: one unit each up to kGradBlocks of them, then equal runs.
template <class T>
static void cut_units(T& t, int value_bytes, int dense_vecs, uint32_t planes)
{
    const uint64_t vec = 16 / value_bytes;
    if (t.count == 0) t.units = 0;
    else if (t.visible == nullptr) t.units = (uint32_t)((t.count + kGradBlock * vec * dense_vecs - 1) / (kGradBlock * vec * dense_vecs));
    else t.units = (uint32_t)((t.n + kGradBlock * vec - 1) / (kGradBlock * vec)) * ((t.planes + planes - 1) / planes);
}

template <class Table>
static uint32_t cut_blocks(Table& tab, uint32_t most)
{
    uint64_t units = 0;
    for (int i = 0; i < tab.count; ++i) units += tab.t[i].units;
    const uint64_t each = units > most ? (units + most - 1) / most : 1;
    uint32_t at = 0;
    for (int i = 0; i < tab.count; ++i) {
        tab.first[i] = at;
        at += (uint32_t)((tab.t[i].units + each - 1) / each);
    }
    tab.first[tab.count] = at;
    return at;
}

// A table of up to kGradTableTensors of the list; tensors without entries keep their place and get no workgroup.
static uint32_t fill_table(GradTable& tab, const GradTensorDev* list, int count)
{
    tab.count = count;
    for (int i = 0; i < count; ++i) {
        tab.t[i] = list[i];
        cut_units(tab.t[i], list[i].dtype == kGradF32 ? 4 : 2, kDenseVecs, kMaskPlanes);
    }
    return cut_blocks(tab, kGradBlocks);
}

hipError_t launch_grad_norm(int count, const GradTensorDev* list, float max_norm, float* result, char* ws, hipStream_t s)
{
    double* total = reinterpret_cast<double*>(ws);
    double* slots = reinterpret_cast<double*>(ws + kGradSlotsAt);
    int at = 0;
    ProfScope prof(kKGradNorm, s);
    do {
        GradTable tab;
        const int part = count - at < kGradTableTensors ? count - at : kGradTableTensors;
        const uint32_t blocks = fill_table(tab, list + at, part);
        if (blocks) hipLaunchKernelGGL(k_grad_squares, dim3(blocks), dim3(kGradBlock), 0, s, tab, slots);
        hipLaunchKernelGGL(k_grad_finish, dim3(1), dim3(1024), 0, s, tab, slots, total, at == 0, at + part == count, max_norm, result, result + 2 + at);
        at += part;
    } while (at < count);
    return hipGetLastError();
}

hipError_t launch_grad_scale(int count, const GradTensorDev* list, const float* result, hipStream_t s)
{
    ProfScope prof(kKGradScale, s);
    for (int at = 0; at < count; at += kGradTableTensors) {
        GradTable tab;
        const uint32_t blocks = fill_table(tab, list + at, count - at < kGradTableTensors ? count - at : kGradTableTensors);
        if (blocks) hipLaunchKernelGGL(k_grad_scale, dim3(blocks), dim3(kGradBlock), 0, s, tab, result);
    }
    return hipGetLastError();
}

hipError_t launch_adam_list(int count, const AdamTensorDev* list, const AdamDev& adam, const float* result, hipStream_t s)
{
    ProfScope prof(kKAdamList, s);
    for (int at = 0; at < count; at += kAdamTableTensors) {
        AdamTable tab;
        tab.adam = adam;
        tab.count = count - at < kAdamTableTensors ? count - at : kAdamTableTensors;
        for (int i = 0; i < tab.count; ++i) {
            tab.t[i] = list[at + i];
            cut_units(tab.t[i], 4, kAdamVecs, kAdamPlanes);
        }
        const uint32_t blocks = cut_blocks(tab, kAdamBlocks);
        if (blocks) hipLaunchKernelGGL(k_adam_list, dim3(blocks), dim3(kGradBlock), 0, s, tab, result);
    }
    return hipGetLastError();
}

}  // namespace pbdr
