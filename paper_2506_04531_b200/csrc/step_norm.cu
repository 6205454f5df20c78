// Root-mean-square norms with the residual's addition, in 8 bits with scales if asked for, and their gradient.
#include "step_vector.cuh"

#include <cuda_fp8.h>
#include <math.h>
#include <type_traits>

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
    uint32_t lanes, row_blocks;            // threads to a row; CTAs' rows
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

// ------------------------------------------------------------------------------------------------ rows that registers hold

// Threads of a row (a power of two, within a warp or of several) hold it in registers, N accesses of 16 bytes each, so that it is read once.  Rows need not begin
// on 16 bytes as long as all tensors' rows begin equally far behind such a boundary: then whole accesses lie inside and the ends are taken element by
// element (SHIFTED; the other form has neither ends nor the comparisons for them).
template <typename T> constexpr int kVector = 16 / (int)sizeof(T);

// The first element of a thread's access j; the row is shifted by `off` elements.
template <typename T>
__device__ __forceinline__ int column_of(uint32_t lane, uint32_t lanes, int j, int off) { return (int)(lane + lanes * j) * kVector<T> - off; }

template <typename T, bool SHIFTED>
__device__ __forceinline__ Words<T, kVector<T>> load_part(const T* row, int c, int dim, bool here) {
    constexpr int V = kVector<T>;
    if (here && c >= 0 && c + V <= dim) return load_words<T, V>(row + c);
    Words<T, V> r = no_words<T, V>();
    if constexpr (SHIFTED) {
        if (here && c < dim) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e >= 0 && c + e < dim) put_element<T, V>(r, e, row[c + e]);
        }
    }
    return r;
}
template <typename T, bool SHIFTED>
__device__ __forceinline__ void store_part(T* row, int c, int dim, bool here, const float (&v)[kVector<T>]) {
    constexpr int V = kVector<T>;
    if (here && c >= 0 && c + V <= dim) store_words<T, V>(row + c, narrow<T, V>(v));
    else if (SHIFTED && here && c < dim) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e >= 0 && c + e < dim) row[c + e] = from_f32<T>(v[e]);
    }
}

// The weights of an access: from memory, or (SHIFTED, where they would lie anywhere) from a copy in shared memory, spread so that neighbouring threads' are
// in different banks.
template <int V> __device__ __forceinline__ int spread(int c) { return c + c / V; }
template <int V>
__device__ __forceinline__ void load_weights(const NormParams& P, int c, float (&w)[V]) {
    if (c + V > (int)P.dim) {
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = 0.f;
    } else if (P.weight_type == HALOS_F32) widen<float, V>(load_words<float, V>(reinterpret_cast<const float*>(P.weight) + c), w);
    else if (P.weight_type == HALOS_BF16) widen<__nv_bfloat16, V>(load_words<__nv_bfloat16, V>(reinterpret_cast<const __nv_bfloat16*>(P.weight) + c), w);
    else widen<__half, V>(load_words<__half, V>(reinterpret_cast<const __half*>(P.weight) + c), w);
}

// Sums and maxima over the threads of a row.
struct RowSums {
    uint32_t lanes;
    float* s_sum;                          // [warps]
    uint32_t* s_top;
    __device__ __forceinline__ float sum(float v, bool& any) const {   // any: over the warp, or the CTA where rows are of several
        if (lanes <= 32) {
            for (uint32_t o = lanes / 2; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
            any = __any_sync(~0u, any);
            return v;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
        if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = v;
        any = __syncthreads_or(any);
        const uint32_t first = threadIdx.x / lanes * (lanes / 32);
        v = 0.f;
        for (uint32_t w = 0; w < lanes / 32; ++w) v += s_sum[first + w];
        __syncthreads();                   // before the places are used again
        return v;
    }
    __device__ __forceinline__ uint32_t top(uint32_t v) const {
        if (lanes <= 32) {
            for (uint32_t o = lanes / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
            return v;
        }
        v = __reduce_max_sync(~0u, v);
        if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = v;
        __syncthreads();
        const uint32_t first = threadIdx.x / lanes * (lanes / 32);
        for (uint32_t w = 0; w < lanes / 32; ++w) v = max(v, s_top[first + w]);
        __syncthreads();
        return v;
    }
};

template <typename T>
__device__ __forceinline__ int shift_of(const T* row) { return (int)((uintptr_t)row / sizeof(T) % kVector<T>); }

constexpr int kMostThreads = 512;
constexpr uint32_t kMostElements = 32;           // of a row to a thread

template <typename T, int N, bool SHIFTED, bool QUANTIZED>
__global__ void __launch_bounds__(kMostThreads, 2) rms_norm_kernel(const __grid_constant__ NormParams P) {
    constexpr int V = kVector<T>;
    extern __shared__ uint32_t s_dynamic[];
    __shared__ float s_sum[kMostThreads / 32];
    __shared__ uint32_t s_top[kMostThreads / 32];
    const uint32_t lanes = P.lanes, slot = threadIdx.x / lanes, lane = threadIdx.x % lanes, per = blockDim.x / lanes;
    const RowSums S{lanes, s_sum, s_top};
    uint32_t* s_group = s_dynamic;                                     // [rows of the CTA, groups]
    float* s_weight = reinterpret_cast<float*>(s_dynamic + (QUANTIZED ? per * P.groups : 0));
    if (QUANTIZED)
        for (uint32_t g = threadIdx.x; g < per * P.groups; g += blockDim.x) s_group[g] = 0;
    if (SHIFTED)
        for (uint32_t c = threadIdx.x; c < P.dim; c += blockDim.x) s_weight[spread<V>(c)] = weight_at(P, c);
    if (QUANTIZED || SHIFTED) __syncthreads();
    const int dim = (int)P.dim;

    for (uint32_t block = blockIdx.x; block < P.row_blocks; block += gridDim.x) {
        const uint32_t row = block * per + slot;
        const bool here = row < P.rows;
        const T* x = reinterpret_cast<const T*>(P.x) + (here ? start_of(P, P.x_stride, row) : 0);
        const int off = SHIFTED ? shift_of(x) : 0;
        Words<T, V> xw[N], rw[N];
#pragma unroll
        for (int j = 0; j < N; ++j) xw[j] = load_part<T, SHIFTED>(x, column_of<T>(lane, lanes, j, off), dim, here);
        if (P.residual) {
            const T* r = reinterpret_cast<const T*>(P.residual) + (here ? start_of(P, P.residual_stride, row) : 0);
#pragma unroll
            for (int j = 0; j < N; ++j) rw[j] = load_part<T, SHIFTED>(r, column_of<T>(lane, lanes, j, off), dim, here);
        }
        float v[N][V], sum = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) widen<T, V>(xw[j], v[j]);
        if (P.residual) {
            T* out = reinterpret_cast<T*>(P.summed) + (here ? start_of(P, P.summed_stride, row) : 0);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float r[V];
                widen<T, V>(rw[j], r);
#pragma unroll
                for (int e = 0; e < V; ++e) v[j][e] += r[e];
                store_part<T, SHIFTED>(out, column_of<T>(lane, lanes, j, off), dim, here, v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) sum = fmaf(v[j][e], v[j][e], sum);
        // A thread's sum below 2^96 has no element above 2^48.
        bool odd = !(sum <= 0x1p96f) || (P.eps < kHides && sum < 0x1p-100f);
        float step = 1.f, total = S.sum(sum, odd);
        if (odd) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) top = max(top, size_bits(v[j][e]));
            top = S.top(top);
            if (out_of_range(top, P.eps)) step = step_for(top);
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float t = v[j][e] * step;
                    sum = fmaf(t, t, sum);
                }
            total = S.sum(sum, odd);
        }
        const float rstd = root_of(total, step, P);
        if (here && lane == 0) P.rstd[row] = rstd;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int c = column_of<T>(lane, lanes, j, off);
            float w[V];
            if (!SHIFTED) load_weights<V>(P, c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (SHIFTED) w[e] = c + e >= 0 && c + e < dim ? s_weight[spread<V>(c + e)] : 0.f;
                v[j][e] = v[j][e] * rstd * w[e];
            }
        }
        const int64_t y0 = here ? start_of(P, P.y_stride, row) : 0;
        if constexpr (!QUANTIZED) {
#pragma unroll
            for (int j = 0; j < N; ++j) store_part<T, SHIFTED>(reinterpret_cast<T*>(P.y) + y0, column_of<T>(lane, lanes, j, off), dim, here, v[j]);
        } else {
            uint32_t* mine = s_group + slot * P.groups;
            const uint32_t group = P.group;
            if (group == P.dim) {
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (!SHIFTED || (column_of<T>(lane, lanes, j, off) + e >= 0 && column_of<T>(lane, lanes, j, off) + e < dim)) top = max(top, size_bits(v[j][e]));
                for (uint32_t o = min(lanes, 32u) / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
                if (here && lane % 32 == 0) atomicMax(mine, top);
            } else {
                const uint32_t run = min(min(group / V, lanes), 32u);   // threads whose accesses lie in one group
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int c = column_of<T>(lane, lanes, j, off);
                    uint32_t first = 0, second = 0;
                    const int border = SHIFTED ? (int)((uint32_t)max(c, 0) / group + 1) * (int)group : 0;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if (!SHIFTED || (c + e < border && c + e >= 0 && c + e < dim)) first = max(first, size_bits(v[j][e]));
                        else if (c + e >= border && c + e < dim) second = max(second, size_bits(v[j][e]));
                    }
                    if constexpr (!SHIFTED) {
                        for (uint32_t o = run / 2; o; o >>= 1) first = max(first, __shfl_xor_sync(~0u, first, o));
                        if (here && c < dim && lane % run == 0) atomicMax(&mine[(uint32_t)c / group], first);
                    } else if (here && c < dim) {
                        atomicMax(&mine[(uint32_t)max(c, 0) / group], first);
                        if (border < c + V && border < dim) atomicMax(&mine[(uint32_t)border / group], second);
                    }
                }
            }
            __syncthreads();
            for (uint32_t g = lane; here && g < P.groups; g += lanes) P.scales[(int64_t)row * P.groups + g] = scale_of(mine[g]);
            uint8_t* y = reinterpret_cast<uint8_t*>(P.y) + y0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int c = column_of<T>(lane, lanes, j, off);
                if (!here || c >= dim) continue;
                const uint32_t g = (uint32_t)max(c, 0) / group;
                const int border = SHIFTED ? (int)(g + 1) * (int)group : dim;
                const float first = 1.f / scale_of(mine[g]), second = SHIFTED && border < c + V && border < dim ? 1.f / scale_of(mine[g + 1]) : 0.f;
                float t[V];
#pragma unroll
                for (int e = 0; e < V; ++e) t[e] = v[j][e] * (!SHIFTED || c + e < border ? first : second);
                if (c >= 0 && c + V <= dim) {
#pragma unroll
                    for (int q = 0; q < V / 4; ++q) {
                        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(t[4 * q], t[4 * q + 1]), __NV_SATFINITE, __NV_E4M3);
                        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(t[4 * q + 2], t[4 * q + 3]), __NV_SATFINITE, __NV_E4M3);
                        reinterpret_cast<uint32_t*>(y + c)[q] = lo | hi << 16;
                    }
                } else if (SHIFTED) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (c + e >= 0 && c + e < dim) y[c + e] = to_8_bits(t[e]);
                }
            }
            if (block + gridDim.x < P.row_blocks) {
                __syncthreads();
                for (uint32_t g = threadIdx.x; g < per * P.groups; g += blockDim.x) s_group[g] = 0;
                __syncthreads();
            }
        }
    }
}

// The gradient.  A row's threads take rows in steps that keep the shift (a multiple of V), so that a thread has the same columns all along and adds up
// its part of dweight in registers; a CTA's rows are added in shared memory, and CTAs' by the kernel that joins.
template <typename T, int N, bool SHIFTED>
__global__ void __launch_bounds__(kMostThreads) rms_norm_back_kernel(const __grid_constant__ NormParams P) {
    constexpr int V = kVector<T>;
    extern __shared__ uint32_t s_dynamic[];
    __shared__ float s_sum[kMostThreads / 32];
    const uint32_t lanes = P.lanes, slot = threadIdx.x / lanes, lane = threadIdx.x % lanes, per = blockDim.x / lanes;
    const RowSums S{lanes, s_sum, nullptr};
    const int dim = (int)P.dim;
    // Rows of one warp are as many apart as the CTA has warps, 8: they have one shift, and their parts of dweight are added by shuffles.
    const uint32_t own = lanes < 32 ? threadIdx.x % 32 / lanes * (blockDim.x / 32) + threadIdx.x / 32 : slot;
    const uint32_t begin = blockIdx.x * per + own;
    float* s_weight = reinterpret_cast<float*>(s_dynamic);
    if (SHIFTED) {
        for (uint32_t c = threadIdx.x; c < P.dim; c += blockDim.x) s_weight[spread<V>(c)] = weight_at(P, c);
        __syncthreads();
    }
    const int off = SHIFTED ? shift_of(reinterpret_cast<const T*>(P.summed) + (int64_t)begin * P.summed_stride[0]) : 0;  // of rows that are not there, too
    float dw[N][V];
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.f;
    const auto weights = [&](int c, float (&w)[V]) {
        if (!SHIFTED) load_weights<V>(P, c, w);
        else {
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = c + e >= 0 && c + e < dim ? s_weight[spread<V>(c + e)] : 0.f;
        }
    };
    for (uint32_t block = blockIdx.x; block < P.row_blocks; block += gridDim.x) {
        const uint32_t row = block * per + own;
        const bool here = row < P.rows;
        const T* s = reinterpret_cast<const T*>(P.summed) + (here ? start_of(P, P.summed_stride, row) : 0);
        const T* dy = reinterpret_cast<const T*>(P.dy) + (here ? start_of(P, P.dy_stride, row) : 0);
        Words<T, V> sw[N], dyw[N], dsw[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int c = column_of<T>(lane, lanes, j, off);
            sw[j] = load_part<T, SHIFTED>(s, c, dim, here), dyw[j] = load_part<T, SHIFTED>(dy, c, dim, here);
        }
        if (P.dsummed) {
            const T* ds = reinterpret_cast<const T*>(P.dsummed) + (here ? start_of(P, P.dsummed_stride, row) : 0);
#pragma unroll
            for (int j = 0; j < N; ++j) dsw[j] = load_part<T, SHIFTED>(ds, column_of<T>(lane, lanes, j, off), dim, here);
        }
        const float rstd = here ? P.rstd[row] : 0.f;
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float a[V], b[V], w[V];
            widen<T, V>(dyw[j], a), widen<T, V>(sw[j], b), weights(column_of<T>(lane, lanes, j, off), w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float u = b[e] * rstd;
                dw[j][e] = fmaf(a[e], u, dw[j][e]);
                dot = fmaf(a[e] * w[e], u, dot);
            }
        }
        bool none = false;
        const float mean = S.sum(dot, none) / (float)P.dim;
        T* dx = reinterpret_cast<T*>(P.dx) + (here ? start_of(P, P.dx_stride, row) : 0);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float a[V], b[V], d[V], w[V];
            widen<T, V>(dyw[j], a), widen<T, V>(sw[j], b), weights(column_of<T>(lane, lanes, j, off), w);
            if (P.dsummed) widen<T, V>(dsw[j], d);
#pragma unroll
            for (int e = 0; e < V; ++e) a[e] = fmaf(rstd, fmaf(-(b[e] * rstd), mean, a[e] * w[e]), P.dsummed ? d[e] : 0.f);
            store_part<T, SHIFTED>(dx, column_of<T>(lane, lanes, j, off), dim, here, a);
        }
    }
    float* s_dw = s_weight;                                             // [dim], spread
    __syncthreads();
    for (uint32_t o = lanes; o < 32; o *= 2)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) dw[j][e] += __shfl_xor_sync(~0u, dw[j][e], o);
    const uint32_t turns = min(per, blockDim.x / 32), turn = lanes < 32 ? (threadIdx.x % 32 < lanes ? threadIdx.x / 32 : turns) : slot;
    for (uint32_t k = 0; k < turns; ++k) {
        if (turn == k) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int c = column_of<T>(lane, lanes, j, off);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (c + e >= 0 && c + e < dim) {
                        float& to = s_dw[spread<V>(c + e)];
                        to = k ? to + dw[j][e] : dw[j][e];
                    }
            }
        }
        __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < P.dim; c += blockDim.x) P.partial[(int64_t)blockIdx.x * P.dim + c] = s_dw[spread<V>(c)];
}

// ------------------------------------------------------------------------------------------------ host

// How rows are spread over threads: N accesses of 16 bytes to each of `lanes` threads, as few left over as possible, and several rows to a CTA
// where they are short.  N = 0: registers do not hold such rows.
struct Shape { uint32_t n, lanes, threads; };
Shape shape_of(uint32_t vectors, uint32_t size) {
    Shape best{0, 0, 0};
    for (uint32_t most : {kMostElements * 3 / 4, kMostElements}) {
        for (uint32_t n = most * size / 16; n >= 1; n = n > 4 ? n - 2 : n - 1)        // 8, 6 and 4 to 1
            for (uint32_t lanes = 4; lanes <= kMostThreads; lanes *= 2)
                if (lanes * n >= vectors && (!best.n || lanes * n < best.lanes * best.n)) best = Shape{n, lanes, lanes < kThreads ? kThreads : lanes};
        if (best.n) break;
    }
    return best;
}

// Whether rows of these tensors begin equally far behind 16 bytes (2), on them and in whole accesses (1), or neither (0).
struct Tensor { const void* at; const int64_t (*stride)[3]; uint32_t size; };
int alignment_of(const NormParams& P, uint32_t size, const Tensor* tensors, int n) {
    const uint32_t v = 16 / size;
    bool whole = P.dim % v == 0, alike = true;
    const uint64_t base = (uintptr_t)tensors[0].at / tensors[0].size % v;
    for (int t = 0; t < n; ++t) {
        const uint64_t at = (uintptr_t)tensors[t].at / tensors[t].size;
        whole &= at % v == 0, alike &= at % v == base;
        for (int k = 0; k < 3; ++k) {
            const uint64_t step = (uint64_t)(*tensors[t].stride)[k] % v;
            whole &= step == 0, alike &= step == (uint64_t)(*tensors[0].stride)[k] % v;
        }
    }
    return whole ? 1 : alike ? 2 : 0;
}

template <typename T, typename F>
int by_accesses(uint32_t n, bool shifted, F f) {
    const auto with = [&](auto s) -> int {
        if constexpr (sizeof(T) == 4) {
            if (n == 8) return f(std::integral_constant<int, 8>(), s);
            if (n == 6) return f(std::integral_constant<int, 6>(), s);
        }
        switch (n) {
            case 1: return f(std::integral_constant<int, 1>(), s);
            case 2: return f(std::integral_constant<int, 2>(), s);
            case 3: return f(std::integral_constant<int, 3>(), s);
            default: return f(std::integral_constant<int, 4>(), s);
        }
    };
    return shifted ? with(std::true_type()) : with(std::false_type());
}

// Accesses of 16 bytes that a row may need, wherever it begins.
uint32_t vectors_of(uint32_t dim, uint32_t size, bool shifted) {
    const uint32_t v = 16 / size;
    return shifted ? (dim + 2 * v - 2) / v : dim / v;
}

uint32_t spread_size(uint32_t dim, uint32_t size) { return dim + dim / (16 / size) + 1; }

uint32_t splits_of(uint32_t rows, uint32_t dim, int32_t device) {
    const uint32_t columns = (dim + kThreads - 1) / kThreads, want = (uint32_t)sm_count(device) * 8 / columns;
    const uint32_t most = (rows + 15) / 16;      // runs of 16 rows or more
    return want < 1 ? 1 : want > most ? (most ? most : 1) : want;
}

// CTAs of the gradient's kernel: a multiple of 8, so that steps of as many rows keep every shift.
uint32_t back_grid(uint32_t rows, const Shape& s, int32_t device) {
    const uint32_t blocks = (rows + s.threads / s.lanes - 1) / (s.threads / s.lanes), most = (uint32_t)sm_count(device) * (s.threads <= 512 ? 512 / s.threads : 1) / 8 * 8;
    return blocks >= most ? most : (blocks + 7) / 8 * 8;
}
// Partial sums of dweight, at most.
uint64_t most_splits(uint32_t rows, uint32_t dim, int32_t device) {
    const uint64_t few = splits_of(rows, dim, device), most = (uint64_t)sm_count(device) * 2 / 8 * 8, blocks = ((uint64_t)rows + 7) / 8 * 8;
    return few > (most < blocks ? most : blocks) ? few : most < blocks ? most : blocks;
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
        const uint32_t out = a->quantized ? 1 : size;
        const Tensor tensors[] = {{a->x, &P.x_stride, size}, {a->y, &P.y_stride, out}, {a->residual, &P.residual_stride, size}, {a->summed, &P.summed_stride, size}};
        const int aligned = alignment_of(P, size, tensors, a->residual ? 4 : 2);
        const bool weights = ((uintptr_t)a->weight) % 16 == 0;
        const bool shifted = aligned != 1 || !weights;
        const Shape s = shape_of(vectors_of(P.dim, size, shifted), size);
        if (aligned && s.n) {
            P.lanes = s.lanes;
            const uint32_t per = s.threads / s.lanes;
            P.row_blocks = (P.rows + per - 1) / per;
            const int shared = (int)((a->quantized ? per * P.groups * 4 : 0) + (shifted ? spread_size(P.dim, size) * 4 : 0));
            return by_accesses<T>(s.n, shifted, [&](auto n, auto sh) -> int {
                const auto launch = [&](auto* kernel, Allowed& allowed) -> int {
                    if (int rc = allow_smem(kernel, shared, allowed)) return rc;
                    const uint32_t resident = 2048 / s.threads, most = (uint32_t)sm_count(a->device) * resident;
                    // a copy of the weights is made once for many rows
                    const uint32_t grid = shifted && P.row_blocks > most ? most : P.row_blocks;
                    kernel<<<grid, s.threads, shared, st>>>(P);
                    return cuda_status(cudaGetLastError(), "norm launch");
                };
                static Allowed plain, quantized;
                return a->quantized ? launch(rms_norm_kernel<T, decltype(n)::value, decltype(sh)::value, true>, quantized)
                                    : launch(rms_norm_kernel<T, decltype(n)::value, decltype(sh)::value, false>, plain);
            });
        }
        rms_norm_any_kernel<T><<<P.rows, kThreads, 0, st>>>(P, a->quantized != 0);
        return cuda_status(cudaGetLastError(), "norm launch");
    });
}

extern "C" int halos_rms_norm_workspace(const halos_rms_norm_args* a, uint64_t* bytes) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    if (!bytes) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    if (int rc = enter(a->device)) return rc;
    *bytes = most_splits((uint32_t)(a->size[0] * a->size[1] * a->size[2]), a->dim, a->device) * a->dim * sizeof(float);
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
    if (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < most_splits(P.rows, P.dim, a->device) * P.dim * sizeof(float))
        return fail(HALOS_ERR_INVALID_ARG, "norm: workspace missing, not aligned or too small");
    P.dy = (const char*)a->dy, P.dsummed = (const char*)a->dsummed, P.dx = (char*)a->dx, P.dweight = (char*)a->dweight, P.partial = (float*)a->workspace;
    cudaStream_t st = (cudaStream_t)a->stream;
    const uint32_t columns = (P.dim + kThreads - 1) / kThreads;
    return by_type(a->dtype, [&](auto t) -> int {
        using T = decltype(t);
        const uint32_t size = sizeof(T);
        const Tensor tensors[] = {{a->summed, &P.summed_stride, size}, {a->dy, &P.dy_stride, size}, {a->dx, &P.dx_stride, size}, {a->dsummed, &P.dsummed_stride, size}};
        const int aligned = alignment_of(P, size, tensors, a->dsummed ? 4 : 3);
        const bool shifted = aligned != 1 || (uintptr_t)a->weight % 16;
        const Shape s = shape_of(vectors_of(P.dim, size, shifted), size);
        if (P.rows && s.n && (aligned == 1 || (aligned == 2 && P.even))) {
            P.lanes = s.lanes;
            const uint32_t per = s.threads / s.lanes;
            P.row_blocks = (P.rows + per - 1) / per;
            P.splits = back_grid(P.rows, s, a->device);
            const int shared = (int)(spread_size(P.dim, size) * 4);
            if (int rc = by_accesses<T>(s.n, shifted, [&](auto n, auto sh) -> int {
                    static Allowed allowed;
                    auto* kernel = rms_norm_back_kernel<T, decltype(n)::value, decltype(sh)::value>;
                    if (int rc = allow_smem(kernel, shared, allowed)) return rc;
                    kernel<<<P.splits, s.threads, shared, st>>>(P);
                    return cuda_status(cudaGetLastError(), "norm launch");
                }))
                return rc;
            rms_norm_join_kernel<<<(P.dim + kJoinColumns - 1) / kJoinColumns, kJoinColumns * kJoinRows, 0, st>>>(P);
            return cuda_status(cudaGetLastError(), "norm launch");
        }
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
