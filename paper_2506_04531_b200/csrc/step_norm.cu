// Root-mean-square norms with the residual's addition, in 8 bits with scales if asked for, and their gradient.
#include "step_vector.cuh"

#include <cuda_fp8.h>
#include <math.h>

namespace halos_step {
namespace {

constexpr int kThreads = 256;
constexpr float kLargest8 = 448.f, kLeastScale = 0x1p-126f;

struct NormParams {
    const char *x, *residual, *weight, *dy, *dsummed;
    char *summed, *y, *dx, *dweight;
    float *scales, *rstd, *partial;
    uint32_t rows, dim, inner, middle, even;  // the inner two of up to three outer sizes; even: there is one at most
    uint32_t weight_type, group, groups;   // group > 0: elements to a scale
    uint32_t splits;                       // partial sums of dweight
    float eps;
    int64_t x_stride[3], residual_stride[3], summed_stride[3], y_stride[3], dy_stride[3], dsummed_stride[3], dx_stride[3];  // in elements, from the innermost outer size on
};

// Where a row begins, in elements.
__device__ __forceinline__ int64_t start_of(const NormParams& P, const int64_t (&stride)[3], uint32_t row) {
    if (P.even) return row * stride[0];
    const uint32_t outer = row / P.inner, k = row - outer * P.inner, i = outer / P.middle, j = outer - i * P.middle;
    return i * stride[2] + j * stride[1] + k * stride[0];
}

__device__ __forceinline__ float weight_at(const NormParams& P, uint32_t c) {
    if (P.weight_type == HALOS_F32) return reinterpret_cast<const float*>(P.weight)[c];
    if (P.weight_type == HALOS_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(P.weight)[c]);
    return __half2float(reinterpret_cast<const __half*>(P.weight)[c]);
}

// Sums and maxima over the CTA, the same in every thread.
__device__ __forceinline__ float cta_sum(float v) {
    __shared__ float s[kThreads / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) sum += s[w];
    return sum;
}
// Of bits of non-negative floats, among which a NaN is the largest.
__device__ __forceinline__ uint32_t cta_max(uint32_t v) {
    __shared__ uint32_t s[kThreads / 32];
    v = __reduce_max_sync(~0u, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = max(top, s[w]);
    return top;
}

__device__ __forceinline__ uint32_t size_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Elements of a row are taken as they are while their squares are neither infinite nor, beside an eps that is not there to hide it, lost: up to 2^48
// and from 2^-50 on.  Beyond, the row is taken times a power of two that makes its largest about 1.
constexpr uint32_t kMost = 0x57800000u;        // bits of 2^48: 2^30 squares still have a sum
constexpr uint32_t kLeast = 0x26800000u;       // of 2^-50
constexpr float kHides = 0x1p-80f;             // an eps from here on does
__device__ __forceinline__ bool out_of_range(uint32_t top, float eps) { return top > kMost || (top < kLeast && top && eps < kHides); }
// Infinities and NaN count as 2^100: they stay what they are.
__device__ __forceinline__ float step_for(uint32_t top) {
    const int e = min(max((int)(top >> 23) - 127, -100), 100);
    return __uint_as_float((uint32_t)(127 - e) << 23);
}
__device__ __forceinline__ float root_of(float sum, float step, const NormParams& P) { return step * rsqrtf(sum / (float)P.dim + P.eps * step * step); }

__device__ __forceinline__ float scale_of(uint32_t top) {
    const float s = __uint_as_float(top) / kLargest8;
    return s < kLeastScale ? kLeastScale : s;  // a NaN stays one
}
__device__ __forceinline__ uint8_t to_8_bits(float v) { return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

// ------------------------------------------------------------------------------------------------ rows of any size and alignment

template <typename T>
__device__ __forceinline__ float sum_at(const T* x, const T* r, uint32_t c) { return to_f32<T>(x[c]) + (r ? to_f32<T>(r[c]) : 0.f); }

constexpr uint32_t kTile = 4096;               // elements whose scales are found at a time; every group divides it

// A CTA to a row, which is read twice (three times in 8 bits), but for the first from the caches.
template <typename T>
__global__ void __launch_bounds__(kThreads) rms_norm_any_kernel(const __grid_constant__ NormParams P, bool quantized) {
    __shared__ uint32_t s_top[kTile / 32];
    const uint32_t row = blockIdx.x;
    const T* x = reinterpret_cast<const T*>(P.x) + start_of(P, P.x_stride, row);
    const T* r = P.residual ? reinterpret_cast<const T*>(P.residual) + start_of(P, P.residual_stride, row) : nullptr;
    T* out = P.residual ? reinterpret_cast<T*>(P.summed) + start_of(P, P.summed_stride, row) : nullptr;
    float sum = 0.f, step = 1.f;
    uint32_t top = 0;
    for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) {
        const float v = sum_at<T>(x, r, c);
        sum = fmaf(v, v, sum), top = max(top, size_bits(v));
    }
    sum = cta_sum(sum), top = cta_max(top);
    if (out_of_range(top, P.eps)) {
        step = step_for(top), sum = 0.f;
        for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) {
            const float v = sum_at<T>(x, r, c) * step;
            sum = fmaf(v, v, sum);
        }
        sum = cta_sum(sum);
    }
    const float rstd = root_of(sum, step, P);
    if (threadIdx.x == 0) P.rstd[row] = rstd;
    uint32_t whole = 0;
    if (quantized && P.group == P.dim) {
        for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) whole = max(whole, size_bits(sum_at<T>(x, r, c) * rstd * weight_at(P, c)));
        whole = cta_max(whole);
        if (threadIdx.x == 0) P.scales[row] = scale_of(whole);
    }
    const int64_t y0 = start_of(P, P.y_stride, row);
    for (uint32_t tile = 0; tile < P.dim; tile += kTile) {
        const uint32_t end = min(P.dim, tile + kTile);
        const bool grouped = quantized && P.group != P.dim;
        if (grouped) {
            __syncthreads();
            for (uint32_t g = threadIdx.x; g < kTile / 32; g += kThreads) s_top[g] = 0;
            __syncthreads();
            for (uint32_t c = tile + threadIdx.x; c < end; c += kThreads) atomicMax(&s_top[(c - tile) / P.group], size_bits(sum_at<T>(x, r, c) * rstd * weight_at(P, c)));
            __syncthreads();
            for (uint32_t g = threadIdx.x; g * P.group < end - tile; g += kThreads) P.scales[(int64_t)row * P.groups + tile / P.group + g] = scale_of(s_top[g]);
        }
        for (uint32_t c = tile + threadIdx.x; c < end; c += kThreads) {
            const float v = sum_at<T>(x, r, c), y = v * rstd * weight_at(P, c);
            if (out) out[c] = from_f32<T>(v);
            if (!quantized) reinterpret_cast<T*>(P.y)[y0 + c] = from_f32<T>(y);
            else reinterpret_cast<uint8_t*>(P.y)[y0 + c] = to_8_bits(y * (1.f / scale_of(grouped ? s_top[(c - tile) / P.group] : whole)));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) rms_norm_any_dx_kernel(const __grid_constant__ NormParams P) {
    const uint32_t row = blockIdx.x;
    const T* s = reinterpret_cast<const T*>(P.summed) + start_of(P, P.summed_stride, row);
    const T* dy = reinterpret_cast<const T*>(P.dy) + start_of(P, P.dy_stride, row);
    const T* ds = P.dsummed ? reinterpret_cast<const T*>(P.dsummed) + start_of(P, P.dsummed_stride, row) : nullptr;
    T* dx = reinterpret_cast<T*>(P.dx) + start_of(P, P.dx_stride, row);
    const float rstd = P.rstd[row];
    float dot = 0.f;
    for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) dot = fmaf(to_f32<T>(dy[c]) * weight_at(P, c), to_f32<T>(s[c]) * rstd, dot);
    const float mean = cta_sum(dot) / (float)P.dim;
    for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) {
        const float g = to_f32<T>(dy[c]) * weight_at(P, c), u = to_f32<T>(s[c]) * rstd;
        dx[c] = from_f32<T>(fmaf(rstd, fmaf(-u, mean, g), ds ? to_f32<T>(ds[c]) : 0.f));
    }
}

// A thread to a column; the rows are split into as many runs as fill the GPU.
template <typename T>
__global__ void __launch_bounds__(kThreads) rms_norm_any_dweight_kernel(const __grid_constant__ NormParams P) {
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= P.dim) return;
    const uint32_t from = (uint32_t)((uint64_t)P.rows * blockIdx.y / P.splits), to = (uint32_t)((uint64_t)P.rows * (blockIdx.y + 1) / P.splits);
    float sum = 0.f;
    for (uint32_t row = from; row < to; ++row)
        sum = fmaf(to_f32<T>(reinterpret_cast<const T*>(P.dy)[start_of(P, P.dy_stride, row) + c]),
                   to_f32<T>(reinterpret_cast<const T*>(P.summed)[start_of(P, P.summed_stride, row) + c]) * P.rstd[row], sum);
    P.partial[(int64_t)blockIdx.y * P.dim + c] = sum;
}

constexpr int kJoinColumns = 32, kJoinRows = 16;
__global__ void __launch_bounds__(kJoinColumns * kJoinRows) rms_norm_join_kernel(const __grid_constant__ NormParams P) {
    __shared__ float s[kJoinRows][kJoinColumns];
    const uint32_t x = threadIdx.x % kJoinColumns, y = threadIdx.x / kJoinColumns, c = blockIdx.x * kJoinColumns + x;
    float sum = 0.f;
    if (c < P.dim)
        for (uint32_t i = y; i < P.splits; i += kJoinRows) sum += P.partial[(int64_t)i * P.dim + c];
    s[y][x] = sum;
    __syncthreads();
    if (y || c >= P.dim) return;
#pragma unroll
    for (int i = 1; i < kJoinRows; ++i) sum += s[i][x];
    if (P.weight_type == HALOS_F32) reinterpret_cast<float*>(P.dweight)[c] = sum;
    else if (P.weight_type == HALOS_BF16) reinterpret_cast<__nv_bfloat16*>(P.dweight)[c] = __float2bfloat16_rn(sum);
    else reinterpret_cast<__half*>(P.dweight)[c] = __float2half_rn(sum);
}

// ------------------------------------------------------------------------------------------------ host

uint32_t splits_of(uint32_t rows, uint32_t dim, int32_t device) {
    const uint32_t columns = (dim + kThreads - 1) / kThreads, want = (uint32_t)sm_count(device) * 8 / columns;
    const uint32_t most = (rows + 15) / 16;      // runs of 16 rows or more
    return want < 1 ? 1 : want > most ? (most ? most : 1) : want;
}

int check(const halos_rms_norm_args* a) {
    if (!a || a->struct_size != sizeof(halos_rms_norm_args)) return fail(HALOS_ERR_INVALID_ARG, "norm: args missing or of another size");
    if (!is_type(a->dtype) || !is_type(a->weight_dtype)) return fail(HALOS_ERR_INVALID_ARG, "norm: dtype");
    int64_t rows = 1;
    for (int i = 0; i < 3; ++i) {
        if (a->size[i] < 0) return fail(HALOS_ERR_INVALID_ARG, "norm: size");
        if (a->size[i] > 0x7fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "norm: over 2^31 - 1 rows");
    }
    for (int i = 0; i < 3; ++i) {
        rows *= a->size[i];
        if (rows > 0x7fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "norm: over 2^31 - 1 rows");
    }
    if (a->dim == 0) return fail(HALOS_ERR_INVALID_ARG, "norm: rows of no elements");
    if (a->dim >= 1u << 30) return fail(HALOS_ERR_UNSUPPORTED, "norm: dim of 2^30 or more");
    return HALOS_OK;
}

// The outer sizes, from the innermost on, those taken together that every one of these tensors goes through in even steps.
void set_rows(NormParams& P, const halos_rms_norm_args* a, int64_t (*const* strides)[3], int tensors) {
    int64_t n[3] = {1, 1, 1};
    int inner[3] = {2, 1, 0}, last = -1;
    for (int i = 2; i >= 0; --i) {
        if (a->size[i] == 1) continue;
        bool even = last >= 0;
        for (int t = 0; even && t < tensors; ++t) even = (*strides[t])[i] == n[last] * (*strides[t])[inner[last]];
        if (even) n[last] *= a->size[i];
        else n[++last] = a->size[i], inner[last] = i;
    }
    for (int t = 0; t < tensors; ++t) {
        const int64_t was[3] = {(*strides[t])[0], (*strides[t])[1], (*strides[t])[2]};
        for (int k = 0; k < 3; ++k) (*strides[t])[k] = k <= last ? was[inner[k]] : 0;
    }
    P.rows = (uint32_t)(n[0] * n[1] * n[2]), P.inner = (uint32_t)n[0], P.middle = (uint32_t)n[1], P.even = last <= 0;
}

int fill(const halos_rms_norm_args* a, NormParams& P) {
    P.dim = a->dim;
    P.weight_type = a->weight_dtype, P.eps = a->eps, P.rstd = a->rstd, P.weight = (const char*)a->weight;
    P.summed = (char*)a->summed;
    if (((uintptr_t)a->weight | (uintptr_t)a->dweight) % size_of(a->weight_dtype) || (uintptr_t)a->rstd % 4) return fail(HALOS_ERR_INVALID_ARG, "norm: tensor not aligned to its elements");
    for (int i = 0; i < 3; ++i) {
        P.x_stride[i] = a->x_stride[i], P.residual_stride[i] = a->residual_stride[i], P.summed_stride[i] = a->summed_stride[i], P.y_stride[i] = a->y_stride[i];
        P.dy_stride[i] = a->dy_stride[i], P.dsummed_stride[i] = a->dsummed_stride[i], P.dx_stride[i] = a->dx_stride[i];
    }
    return HALOS_OK;
}

template <typename F>
int by_type(uint32_t type, F f) {
    if (type == HALOS_F32) return f(float());
    if (type == HALOS_BF16) return f(__nv_bfloat16());
    return f(__half());
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_rms_norm_fwd(const halos_rms_norm_args* a) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    if (!(a->eps >= 0.f) || !isfinite(a->eps)) return fail(HALOS_ERR_INVALID_ARG, "norm: eps must be finite and not negative");
    if (a->quantized && a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128) return fail(HALOS_ERR_UNSUPPORTED, "norm: group must be 0, 32, 64 or 128");
    NormParams P{};
    if (int rc = fill(a, P)) return rc;
    int64_t(*const here[])[3] = {&P.x_stride, &P.y_stride, &P.residual_stride, &P.summed_stride};
    set_rows(P, a, here, a->residual ? 4 : 2);
    if (P.rows == 0) return HALOS_OK;
    if (!a->x || !a->y || !a->rstd || !a->weight || (a->residual && !a->summed) || (a->quantized && !a->scales)) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    const uint32_t size = size_of(a->dtype);
    if (((uintptr_t)a->x | (uintptr_t)a->residual | (a->residual ? (uintptr_t)a->summed : 0) | (a->quantized ? 0 : (uintptr_t)a->y)) % size || (a->quantized && (uintptr_t)a->scales % 4))
        return fail(HALOS_ERR_INVALID_ARG, "norm: tensor not aligned to its elements");
    P.x = (const char*)a->x, P.residual = (const char*)a->residual, P.y = (char*)a->y, P.scales = a->scales;
    P.group = a->group && a->group < a->dim ? a->group : a->dim, P.groups = (a->dim + P.group - 1) / P.group;
    if (int rc = enter(a->device)) return rc;
    cudaStream_t st = (cudaStream_t)a->stream;
    return by_type(a->dtype, [&](auto t) {
        using T = decltype(t);
        rms_norm_any_kernel<T><<<P.rows, kThreads, 0, st>>>(P, a->quantized != 0);
        return cuda_status(cudaGetLastError(), "norm launch");
    });
}

extern "C" int halos_rms_norm_workspace(const halos_rms_norm_args* a, uint64_t* bytes) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    if (!bytes) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    if (int rc = enter(a->device)) return rc;
    *bytes = (uint64_t)splits_of((uint32_t)(a->size[0] * a->size[1] * a->size[2]), a->dim, a->device) * a->dim * sizeof(float);
    return HALOS_OK;
}

extern "C" int halos_rms_norm_bwd(const halos_rms_norm_args* a) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    NormParams P{};
    if (int rc = fill(a, P)) return rc;
    int64_t(*const here[])[3] = {&P.summed_stride, &P.dy_stride, &P.dx_stride, &P.dsummed_stride};
    set_rows(P, a, here, a->dsummed ? 4 : 3);
    if (!a->weight || !a->dweight || (P.rows && (!a->summed || !a->rstd || !a->dy || !a->dx))) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    if (((uintptr_t)a->summed | (uintptr_t)a->dy | (uintptr_t)a->dsummed | (uintptr_t)a->dx) % size_of(a->dtype)) return fail(HALOS_ERR_INVALID_ARG, "norm: tensor not aligned to its elements");
    if (int rc = enter(a->device)) return rc;
    P.splits = splits_of(P.rows, P.dim, a->device);
    if (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < (uint64_t)P.splits * P.dim * sizeof(float))
        return fail(HALOS_ERR_INVALID_ARG, "norm: workspace missing, not aligned or too small");
    P.dy = (const char*)a->dy, P.dsummed = (const char*)a->dsummed, P.dx = (char*)a->dx, P.dweight = (char*)a->dweight, P.partial = (float*)a->workspace;
    cudaStream_t st = (cudaStream_t)a->stream;
    const uint32_t columns = (P.dim + kThreads - 1) / kThreads;
    return by_type(a->dtype, [&](auto t) -> int {
        using T = decltype(t);
        if (P.rows) {
            rms_norm_any_dx_kernel<T><<<P.rows, kThreads, 0, st>>>(P);
            if (int rc = cuda_status(cudaGetLastError(), "norm launch")) return rc;
        }
        rms_norm_any_dweight_kernel<T><<<dim3(columns, P.splits), kThreads, 0, st>>>(P);
        if (int rc = cuda_status(cudaGetLastError(), "norm launch")) return rc;
        rms_norm_join_kernel<<<(P.dim + kJoinColumns - 1) / kJoinColumns, kJoinColumns * kJoinRows, 0, st>>>(P);
        return cuda_status(cudaGetLastError(), "norm launch");
    });
}
