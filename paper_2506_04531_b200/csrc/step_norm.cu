// Root-mean-square norms with the residual's addition, in 8 bits with scales if asked for.
//
// y = s rstd w, s = x + residual, rstd = 1 / sqrt(mean s^2 + eps): five operations an element beside four accesses to memory, which bound it.  A row is read once: its threads
// hold it in registers, add up the squares by shuffles (and, where a row takes several warps, at a barrier of their own), and in 8 bits find the
// groups' largest by shuffles, too.  Rows come through shared memory, one or two ahead of their turn; arithmetic goes by pairs of 32-bit floats, since what is left of
// the instructions is what keeps the shorter cases from the memory's rate.  y is formed from the 32-bit sum, not from `summed`, which is rounded; in 8 bits it is
// rounded once, from 32.
//
// Measured (a pass among others; floor by bytes at the copy rate): 65536 x 768 bf16 with residual 67 us (92%), 16384 x 2048 bf16 with residual 46.5 us (88%), the same in 8 bits with
// a scale for 128 elements 49 us (73%), 32768 x 1021 bf16 with residual 75 us (54%: rows off every boundary, a third of the threads' places unused; f32, 16384 of them, 50 us, 82%),
// 262144 heads of 128 bf16 with residual 46 us (89%), 65536 x 768 f32 with residual 131 us (94%).  The kernel that goes over rows in loops: 16384 x 5120 f32 with residual 250 us (82%).
#include "step_norm.cuh"

#include <cuda_fp8.h>

namespace halos_step {
namespace norm {

constexpr float kLargest8 = 448.f, kLeastScale = 0x1p-126f;

// The largest over the CTA of bits of non-negative floats, among which a NaN is the largest.
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
__device__ __forceinline__ float root_of(float sum, float step, const Params& P, float lift = 1.f) { return step / lift * rsqrtf(sum * P.inverse_dim + P.eps * step * step); }
// Rows that are not all zeros and still so small that 32 bits do not hold one over their root: it is formed divided by kLift, and the products with it are taken times that.
constexpr float kLift = 0x1p64f;
__device__ __forceinline__ bool to_be_lifted(float rstd, float sum) { return isinf(rstd) && sum > 0.f; }

__device__ __forceinline__ float scale_of(uint32_t top) {
    const float s = __uint_as_float(top) * (1.f / kLargest8);
    return s < kLeastScale ? kLeastScale : s;  // a NaN stays one
}
// A scale and its reciprocal as the sum of two floats, which is off by 2^-46 of itself: the reciprocal's approximation is off by 2^-23, `left` is what it leaves of 1, exactly, and
// `low` is off by 2^-23 of itself.  A product with it that is rounded once is the quotient rounded once, as far as 8 bits can show it: a quotient that is the middle between two 8-bit
// values comes out as that, and only one within 2^-24 of the middle without being it may go to either side, as if it had been divided in 32 bits.
struct Scale {
    float scale, high, low;
    __device__ __forceinline__ explicit Scale(uint32_t top) : scale(scale_of(top)) {
        asm("rcp.approx.f32 %0, %1;" : "=f"(high) : "f"(scale));
        const float left = fmaf(-scale, high, 1.f);
        low = scale <= 0x1p127f ? left * high : 0.f;   // an infinite scale has a reciprocal of 0, of which nothing is left
    }
};
// Two elements over the scales that are theirs.
__device__ __forceinline__ float2 over(float2 v, const Scale& a, const Scale& b) { return fma2(v, make_float2(a.high, b.high), mul2(v, make_float2(a.low, b.low))); }
__device__ __forceinline__ uint8_t to_8_bits(float v) { return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }
template <int V>
__device__ __forceinline__ void store_8_bits(uint8_t* to, const float2 (&v)[V / 2]) {
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(v[2 * q], __NV_SATFINITE, __NV_E4M3), hi = __nv_cvt_float2_to_fp8x2(v[2 * q + 1], __NV_SATFINITE, __NV_E4M3);
        reinterpret_cast<uint32_t*>(to)[q] = lo | hi << 16;
    }
}
// The largest size among them, as bits; a NaN is the largest.
template <int V>
__device__ __forceinline__ uint32_t largest(const float2 (&v)[V / 2]) {
    float m = fabsf(v[0].x);
    const auto with = [&](float x) { asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(x))); };
    with(v[0].y);
#pragma unroll
    for (int i = 1; i < V / 2; ++i) with(v[i].x), with(v[i].y);
    return __float_as_uint(m);
}

// ------------------------------------------------------------------------------------------------ rows of any size and alignment

template <typename T>
__device__ __forceinline__ float sum_at(const T* x, const T* r, uint32_t c) { return to_f32<T>(x[c]) + (r ? to_f32<T>(r[c]) : 0.f); }

constexpr uint32_t kTile = 4096;               // elements whose scales are found at a time; every group divides it

// A CTA to a row, which is read twice (three times in 8 bits), but for the first from the caches.
template <typename T>
__global__ void __launch_bounds__(kThreads) rms_norm_any_kernel(const __grid_constant__ Params P, bool quantized) {
    __shared__ uint32_t s_top[kTile / 32];
    const uint32_t row = blockIdx.x;
    const T* x = row_at<const T>(P, P.in[0], row);
    const T* r = P.arrays > 1 ? row_at<const T>(P, P.in[1], row) : nullptr;
    T* out = P.arrays > 1 ? row_at<T>(P, P.out[1], row) : nullptr;
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
    const float rstd = root_of(sum, step, P), lift = to_be_lifted(rstd, sum) ? kLift : 1.f, root = root_of(sum, step, P, lift);
    if (threadIdx.x == 0) P.rstd[row] = rstd;
    const auto y_of = [&](float v, uint32_t c) { return v * root * lift * weight_at(P, c); };
    uint32_t whole = 0;
    if (quantized && P.group == P.dim) {
        for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) whole = max(whole, size_bits(y_of(sum_at<T>(x, r, c), c)));
        whole = cta_max(whole);
        if (threadIdx.x == 0) P.scales[row] = scale_of(whole);
    }
    const float scale_of_row = scale_of(whole);
    const int64_t y0 = start_of(P, P.out[0], row);
    for (uint32_t tile = 0; tile < P.dim; tile += kTile) {
        const uint32_t end = min(P.dim, tile + kTile);
        const bool grouped = quantized && P.group != P.dim;
        if (grouped) {
            __syncthreads();
            for (uint32_t g = threadIdx.x; g < kTile / 32; g += kThreads) s_top[g] = 0;
            __syncthreads();
            for (uint32_t c = tile + threadIdx.x; c < end; c += kThreads) atomicMax(&s_top[(c - tile) / P.group], size_bits(y_of(sum_at<T>(x, r, c), c)));
            __syncthreads();
            for (uint32_t g = threadIdx.x; g * P.group < end - tile; g += kThreads) P.scales[(int64_t)row * P.groups + tile / P.group + g] = scale_of(s_top[g]);
        }
        for (uint32_t c = tile + threadIdx.x; c < end; c += kThreads) {
            const float v = sum_at<T>(x, r, c), y = y_of(v, c);
            if (out) out[c] = from_f32<T>(v);
            if (!quantized) reinterpret_cast<T*>(P.out[0].at)[y0 + c] = from_f32<T>(y);
            else reinterpret_cast<uint8_t*>(P.out[0].at)[y0 + c] = to_8_bits(y / (grouped ? scale_of(s_top[(c - tile) / P.group]) : scale_of_row));
        }
    }
}

// ------------------------------------------------------------------------------------------------ rows that a CTA holds

template <typename T, int N, int L, Mode M, bool QUANTIZED, int ARRAYS>
__global__ void __launch_bounds__(kWide<T, N, M> ? kMostThreads : kThreads, kWide<T, N, M> ? 1 : 4) rms_norm_kernel(const __grid_constant__ Params P) {
    using A = Threads<T, N, L, M, kWide<T, N, M> ? kMostThreads : kThreads, ARRAYS>;
    constexpr int V = A::V, H = A::H;
    extern __shared__ __align__(16) char s_dynamic[];
    __shared__ uint32_t s_part[2 * kMostThreads / 32];
    const A t(P, s_dynamic, false);
    RowSums<(N > 1 && L == 32)> S(t.lanes, s_part);
    const int stages = (int)P.stages, dim = t.dim;
    constexpr bool added = ARRAYS > 1;
    for (int k = 0; k < stages - 1; ++k) t.fetch(k, k, false);
    uint32_t* s_group = reinterpret_cast<uint32_t*>(t.behind()) + t.own * P.groups;      // [rows of the CTA][groups], where not kWhole
    if (QUANTIZED && M != kWhole)
        for (uint32_t g = threadIdx.x % t.lanes; g < P.groups; g += t.lanes) s_group[g] = 0;
    t.load_weights();

    int stage = 0;
    for (uint32_t i = 0; i < P.run; ++i) {
        if (stages == 1) t.fetch(i, 0, false);
        wait_copies(stages == 3);
        if (stages > 1) t.fetch(i + stages - 1, stage ? stage - 1 : stages - 1, false);   // where the row before this was
        const uint32_t row = t.row_of(i);
        const bool here = row < P.rows;
        float2 v[N][H], sums = both(0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            t.arrived(stage, 0, j, here, v[j]);
            if (!added) keep_own<V, M>(v[j], t.column(j), dim);
        }
        if (added) {
            T* out = here ? row_at<T>(P, P.out[1], row) : nullptr;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float2 r[H];
                t.arrived(stage, 1, j, here, r);
#pragma unroll
                for (int i = 0; i < H; ++i) v[j][i] = add2(v[j][i], r[i]);
                keep_own<V, M>(v[j], t.column(j), dim);
                if (here) store_part<T, V, M>(out, t.column(j), dim, v[j]);
            }
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < H; ++i) sums = fma2(v[j][i], v[j][i], sums);
        float sum = sums.x + sums.y;
        // A thread's sum below 2^96 has no element above 2^48.
        bool odd = !(sum <= 0x1p96f) || (P.eps < kHides && sum < 0x1p-100f);
        float step = 1.f, total = S.sum(sum, odd);
        if (odd) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) top = max(top, largest<V>(v[j]));
            top = S.top(top);
            if (out_of_range(top, P.eps)) step = step_for(top);
            sums = both(0.f);
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    const float2 u = mul2(v[j][i], both(step));
                    sums = fma2(u, u, sums);
                }
            total = S.sum(sums.x + sums.y);
        }
        float rstd = root_of(total, step, P);
        if (here && t.leads()) P.rstd[row] = rstd;
        const bool lifted = to_be_lifted(rstd, total);
        if (lifted) rstd = root_of(total, step, P, kLift);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float2 w[H];
            t.weights(j, w);
#pragma unroll
            for (int i = 0; i < H; ++i) v[j][i] = mul2(v[j][i], both(rstd));
            if (lifted)
#pragma unroll
                for (int i = 0; i < H; ++i) v[j][i] = mul2(v[j][i], both(kLift));
#pragma unroll
            for (int i = 0; i < H; ++i) v[j][i] = mul2(v[j][i], w[i]);
        }
        const int64_t y0 = here ? start_of(P, P.out[0], row) : 0;
        if constexpr (!QUANTIZED) {
            if (here) {
#pragma unroll
                for (int j = 0; j < N; ++j) store_part<T, V, M>(reinterpret_cast<T*>(P.out[0].at) + y0, t.column(j), dim, v[j]);
            }
        } else {
            uint8_t* y = reinterpret_cast<uint8_t*>(P.out[0].at) + y0;
            float* scales = P.scales + (int64_t)row * P.groups;
            const uint32_t group = P.group;
            if constexpr (M == kWhole) {   // the threads of a group are neighbours in a warp, or the group is the row
                uint32_t top[N];
#pragma unroll
                for (int j = 0; j < N; ++j) top[j] = largest<V>(v[j]);
                if (group == P.dim) {
#pragma unroll
                    for (int j = 1; j < N; ++j) top[0] = max(top[0], top[j]);
                    top[0] = S.top(top[0]);
#pragma unroll
                    for (int j = 1; j < N; ++j) top[j] = top[0];
                    if (here && t.leads()) scales[0] = scale_of(top[0]);
                } else {
#pragma unroll
                    for (uint32_t o = 128 / V / 2; o; o >>= 1)
                        if (o * V < group)
#pragma unroll
                            for (int j = 0; j < N; ++j) top[j] = max(top[j], __shfl_xor_sync(~0u, top[j], o));
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int c = t.column(j);
                    if (!here || c >= dim) continue;
                    const Scale scale(top[j]);
                    if (group != P.dim && ((uint32_t)c & (group - 1)) == 0) scales[(uint32_t)c >> P.group_bits] = scale.scale;
#pragma unroll
                    for (int i = 0; i < H; ++i) v[j][i] = over(v[j][i], scale, scale);
                    store_8_bits<V>(y + c, v[j]);
                }
            } else {
                const auto meet = [&] {
                    if (t.lanes > 32) asm volatile("barrier.cta.sync %0, %1;" ::"r"(t.own + 1), "r"(t.lanes) : "memory");
                    else __syncwarp();
                };
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int c = t.column(j);
                    if (!here || c >= dim) continue;
                    // an access lies in one group or on the border of two
                    const uint32_t g = group == P.dim ? 0 : (uint32_t)max(c, 0) >> P.group_bits;
                    const int border = group == P.dim ? dim : (int)(g + 1) << P.group_bits;
                    uint32_t first = 0, second = 0;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const uint32_t bits = size_bits(e % 2 ? v[j][e / 2].y : v[j][e / 2].x);
                        if (c + e < border) first = max(first, bits);   // what is not the row's is 0
                        else second = max(second, bits);
                    }
                    atomicMax(&s_group[g], first);
                    if (border < c + V && border < dim) atomicMax(&s_group[g + 1], second);
                }
                meet();
                for (uint32_t g = threadIdx.x % t.lanes; here && g < P.groups; g += t.lanes) scales[g] = scale_of(s_group[g]);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int c = t.column(j);
                    if (!here || c >= dim) continue;
                    const uint32_t g = group == P.dim ? 0 : (uint32_t)max(c, 0) >> P.group_bits;
                    const int border = group == P.dim ? dim : (int)(g + 1) << P.group_bits;
                    const Scale first(s_group[g]), second(border < c + V && border < dim ? s_group[g + 1] : 0);
#pragma unroll
                    for (int i = 0; i < H; ++i) v[j][i] = over(v[j][i], c + 2 * i < border ? first : second, c + 2 * i + 1 < border ? first : second);
                    if (M == kShifted && c >= 0 && c + V <= dim) store_8_bits<V>(y + c, v[j]);
                    else {
#pragma unroll
                        for (int i = 0; i < H; ++i) {
                            if (owned<V>(c, 2 * i, dim)) y[c + 2 * i] = to_8_bits(v[j][i].x);
                            if (owned<V>(c, 2 * i + 1, dim)) y[c + 2 * i + 1] = to_8_bits(v[j][i].y);
                        }
                    }
                }
                meet();
                for (uint32_t g = threadIdx.x % t.lanes; g < P.groups; g += t.lanes) s_group[g] = 0;
                meet();
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ host

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
static void set_rows(Params& P, const int64_t (&size)[3], uint32_t outs) {
    Rows* every[5];
    uint32_t n = 0;
    for (uint32_t i = 0; i < P.arrays; ++i) every[n++] = &P.in[i];
    for (uint32_t i = 0; i < outs; ++i) every[n++] = &P.out[i];
    int64_t sizes[3] = {1, 1, 1};
    int inner[3] = {2, 1, 0}, last = -1;
    for (int i = 2; i >= 0; --i) {
        if (size[i] == 1) continue;
        bool even = last >= 0;
        for (uint32_t t = 0; even && t < n; ++t) even = every[t]->stride[i] == sizes[last] * every[t]->stride[inner[last]];
        if (even) sizes[last] *= size[i];
        else sizes[++last] = size[i], inner[last] = i;
    }
    for (uint32_t t = 0; t < n; ++t) {
        const int64_t was[3] = {every[t]->stride[0], every[t]->stride[1], every[t]->stride[2]};
        for (int k = 0; k < 3; ++k) every[t]->stride[k] = k <= last ? was[inner[k]] : 0;
    }
    P.rows = (uint32_t)(sizes[0] * sizes[1] * sizes[2]), P.inner = (uint32_t)sizes[0], P.middle = (uint32_t)sizes[1], P.even = last <= 0;
}

int fill(const halos_rms_norm_args* a, Params& P, uint32_t outs) {
    const uint32_t size = size_of(a->dtype);
    P.dim = a->dim, P.inverse_dim = 1.f / (float)a->dim, P.weight_type = a->weight_dtype, P.eps = a->eps, P.rstd = a->rstd, P.weight = (const char*)a->weight;
    if (((uintptr_t)a->weight | (uintptr_t)a->dweight) % size_of(a->weight_dtype) || (uintptr_t)a->rstd % 4) return fail(HALOS_ERR_INVALID_ARG, "norm: tensor not aligned to its elements");
    for (uint32_t t = 0; t < P.arrays; ++t) {      // the memory that its rows lie in
        int64_t low = 0, high = 0;
        for (int i = 0; i < 3; ++i) {
            const int64_t far = (a->size[i] - 1) * P.in[t].stride[i];
            if (far < 0) low += far;
            else high += far;
        }
        P.in[t].span[0] = P.in[t].at + low * size, P.in[t].span[1] = P.in[t].at + (high + a->dim) * size;
    }
    set_rows(P, a->size, outs);
    return HALOS_OK;
}

Mode mode_of(const Params& P, uint32_t size, uint32_t outs, uint32_t out_size) {
    const uint32_t v = 16 / size;
    const uint64_t base = (uintptr_t)P.in[0].at / size % v;
    bool whole = P.dim % v == 0, alike = P.even;
    const auto look = [&](const Rows& R, uint32_t bytes) {
        const uint64_t at = (uintptr_t)R.at / bytes;
        whole &= at % v == 0, alike &= at % v == base;
        for (int k = 0; k < 3; ++k) whole &= (uint64_t)R.stride[k] % v == 0, alike &= (uint64_t)R.stride[k] % v == (uint64_t)P.in[0].stride[k] % v;
    };
    for (uint32_t t = 0; t < P.arrays; ++t) look(P.in[t], size);
    for (uint32_t t = 0; t < outs; ++t) look(P.out[t], t ? size : out_size);
    return whole ? kWhole : alike ? kShifted : kLoose;
}

static Shape shape_of(const Params& P, uint32_t size, Mode mode, uint32_t groups, uint32_t least) {
    const uint32_t v = mode == kLoose ? 2 : 16 / size, accesses = accesses_of(P.dim, v, mode);
    Shape s{};
    spread_over(s, v, mode, accesses, least);
    if (!s.n) return s;
    const bool wide = s.n * v > kFew;
    s.threads = wide ? kMostThreads : kThreads, s.resident = wide ? 1 : 4;
    const uint32_t room = kSharedPerSM / s.resident - 1024 - 512, stage = P.arrays * s.n * s.threads * v * size;
    const uint32_t fixed = s.n * v * 4 * (mode == kShifted ? s.threads : s.lanes) + groups * s.per() * 4;
    if (fixed + stage > room) return Shape{};
    s.stages = mode == kLoose ? 1 : (room - fixed) / stage;
    if (s.stages > kMostStages) s.stages = kMostStages;
    s.shared = fixed + s.stages * stage;
    return s;
}

}  // namespace norm
}  // namespace halos_step

extern "C" int halos_rms_norm_fwd(const halos_rms_norm_args* a) {
    using namespace halos_step;
    using namespace halos_step::norm;
    if (int rc = check(a)) return rc;
    if (!(a->eps >= 0.f) || !isfinite(a->eps)) return fail(HALOS_ERR_INVALID_ARG, "norm: eps must be finite and not negative");
    if (a->quantized && a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128) return fail(HALOS_ERR_UNSUPPORTED, "norm: group must be 0, 32, 64 or 128");
    Params P{};
    P.arrays = a->residual ? 2 : 1;
    set(P.in[0], a->x, a->x_stride), set(P.in[1], a->residual, a->residual_stride), set(P.out[0], a->y, a->y_stride), set(P.out[1], a->summed, a->summed_stride);
    if (int rc = fill(a, P, P.arrays)) return rc;
    if (P.rows == 0) return HALOS_OK;
    if (!a->x || !a->y || !a->rstd || !a->weight || (a->residual && !a->summed) || (a->quantized && !a->scales)) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    const uint32_t size = size_of(a->dtype);
    if (((uintptr_t)a->x | (uintptr_t)a->residual | (a->residual ? (uintptr_t)a->summed : 0) | (a->quantized ? 0 : (uintptr_t)a->y)) % size || (a->quantized && (uintptr_t)a->scales % 4))
        return fail(HALOS_ERR_INVALID_ARG, "norm: tensor not aligned to its elements");
    P.scales = a->scales;
    P.group = a->group && a->group < a->dim ? a->group : a->dim, P.groups = (a->dim + P.group - 1) / P.group, P.group_bits = a->group == 32 ? 5 : a->group == 64 ? 6 : 7;
    if (int rc = enter(a->device)) return rc;
    cudaStream_t st = (cudaStream_t)a->stream;
    const Mode mode = mode_of(P, size, P.arrays, a->quantized ? 1 : size);
    const Shape s = shape_of(P, size, mode, a->quantized && mode != kWhole ? P.groups : 0, a->quantized && P.group < P.dim ? P.group * size / 16 : 1);
    return by_type(a->dtype, [&](auto t) -> int {
        using T = decltype(t);
        if (!s.n) {
            rms_norm_any_kernel<T><<<P.rows, kThreads, 0, st>>>(P, a->quantized != 0);
            return cuda_status(cudaGetLastError(), "norm launch");
        }
        P.lanes = s.lanes, P.stages = s.stages, P.row_blocks = (P.rows + s.per() - 1) / s.per();
        // CTAs take short runs of neighbouring rows, in the order in which they are started: the rows that are under way then lie close together in memory,
        // and that is worth more than few CTAs (65536 x 768: as many CTAs as there is room for, in even steps, 74 us; runs of 4 67 us).
        const uint32_t room = (uint32_t)sm_count(a->device) * s.resident, once = (P.row_blocks + room - 1) / room, long_run = (uint32_t)((uint64_t)P.row_blocks * 2 / (room * 7));
        P.apart = mode == kShifted && s.per() < 8 ? 8 / s.per() : 1, P.run = long_run > 4 ? long_run : once < 4 ? once : 4;
        const uint32_t grid = (P.row_blocks + P.apart * P.run - 1) / (P.apart * P.run) * P.apart;
        return by_accesses<T>(s.n, s.apart, mode, [&](auto n, auto l, auto m) -> int {
            const auto launch = [&](auto* kernel, Allowed& allowed) -> int {
                if (int rc = allow_smem(kernel, (int)s.shared, allowed)) return rc;
                kernel<<<grid, s.threads, s.shared, st>>>(P);
                return cuda_status(cudaGetLastError(), "norm launch");
            };
            static Allowed allowed[4];
            constexpr int N = decltype(n)::value, L = decltype(l)::value;
            constexpr Mode M = decltype(m)::value;
            if (P.arrays > 1) return a->quantized ? launch(rms_norm_kernel<T, N, L, M, true, 2>, allowed[0]) : launch(rms_norm_kernel<T, N, L, M, false, 2>, allowed[1]);
            return a->quantized ? launch(rms_norm_kernel<T, N, L, M, true, 1>, allowed[2]) : launch(rms_norm_kernel<T, N, L, M, false, 1>, allowed[3]);
        });
    });
}
