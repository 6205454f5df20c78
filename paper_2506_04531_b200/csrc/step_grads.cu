// The norm of many gradients at once, clipping by it, and the step of plain descent.
//
// Bound by memory: the norm reads every gradient once; clipping and the step read it again, since the factor is not known before, and write (and for
// the step read) as much.  A launch takes a table of up to 960 tensors as its argument; every CTA takes chunks of 32 KB from all of them in turn.
//
// Sums.  Eight neighbours' squares are added in 32 bits, which is exact to 2^-21, and groups are added in 64.  A group whose sum 32 bits would not hold
// (some |g| above 2^60, or nothing but |g| under 2^-48) is formed in 64 bits instead, so that no finite gradients have an infinite norm or one of 0.
// CTAs leave one partial sum each, and who needs the norm adds those up in their order: the same bits every time, without atomics.
//
// Measured: 148 tensors of 162M f32 gradients: the norm 94 us (6.9 TB/s), the clipped step on f32 parameters behind it 292 us (6.7 TB/s), both 402 to 411 us; 76 tensors of 70M bf16 gradients
// clipped into f32 110 us.  What is read a second time comes from the L2 cache as far as that holds it.  Small sets are bound by what Python asks of each tensor, 0.5 to 1 us.
#include "step_vector.cuh"

#include <algorithm>
#include <math.h>
#include <new>
#include <type_traits>

namespace halos_step {
namespace {

constexpr int kThreads = 256, kResident = 4;        // CTAs to an SM
constexpr int kWaves = 4;                           // of CTAs, at most: partial sums have an end
constexpr uint32_t kChunkBytes = 32768;             // of gradients
constexpr int kMostPieces = 960;                    // what a launch's 32764 bytes of arguments hold
enum Mode { kClip, kStep };

struct Piece {
    const void* in;
    void* out;
    int64_t n;
    uint32_t first;                                 // chunk
    uint16_t in_type, out_type;
};
template <int N>
struct Table {
    uint32_t pieces, chunks, run;                   // run: chunks to a CTA
    const double* partial;                          // of the norm; NULL: the factor is 1
    uint32_t partials;
    float max_norm, rate;
    float* norm;
    Piece piece[N];
};

// The piece that chunk `c` belongs to.
template <int N>
__device__ __forceinline__ int piece_of(const Table<N>& t, uint32_t c) {
    int lo = 0, hi = (int)t.pieces;                 // piece[lo].first <= c < piece[hi].first
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.piece[mid].first <= c) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double squares_of(const float (&v)[8]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
    if (s >= 0x1p-96f && s <= 0x1p120f) return (double)s;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) any |= __float_as_uint(v[i]);
    if (!(any << 1)) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) d = fma((double)v[i], (double)v[i], d);
    return d;
}

// The sum over the CTA, the same in every thread.
__device__ __forceinline__ double sum_of_all(double v) {
    __shared__ double s_sum[kThreads / 32];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) sum += s_sum[w];
    return sum;
}

template <typename T>
__device__ __forceinline__ double squares_of_chunk(const T* x, int n) {
    constexpr int kUnits = kChunkBytes / sizeof(T) / 8 / kThreads;
    double sum = 0.0;
    if (n == kChunkBytes / sizeof(T) && (uintptr_t)x % 16 == 0) {
        Words<T, 8> w[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u) w[u] = load_words<T, 8>(x + 8 * (threadIdx.x + kThreads * u));
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            float v[8];
            widen<T, 8>(w[u], v);
            sum += squares_of(v);
        }
        return sum;
    }
    for (int at = threadIdx.x; at < n; at += 8 * kThreads) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at + kThreads * i < n ? to_f32<T>(x[at + kThreads * i]) : 0.f;
        sum += squares_of(v);
    }
    return sum;
}

template <int N>
__global__ void __launch_bounds__(kThreads, kResident) grads_squares_kernel(const __grid_constant__ Table<N> t, double* partial) {
    double sum = 0.0;
    const uint32_t end = min(t.chunks, (blockIdx.x + 1) * t.run);
    for (uint32_t c = blockIdx.x * t.run; c < end; ++c) {
        const Piece& p = t.piece[piece_of(t, c)];
        const uint32_t size = p.in_type == HALOS_F32 ? 4 : 2;
        const int64_t at = (int64_t)(c - p.first) * (kChunkBytes / size), left = p.n - at;
        const int n = (int)(left < kChunkBytes / size ? left : kChunkBytes / size);
        if (p.in_type == HALOS_F32) sum += squares_of_chunk((const float*)p.in + at, n);
        else if (p.in_type == HALOS_BF16) sum += squares_of_chunk((const __nv_bfloat16*)p.in + at, n);
        else sum += squares_of_chunk((const __half*)p.in + at, n);
    }
    sum = sum_of_all(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of(const double* partial, uint32_t n) {
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) sum += partial[i];
    return sqrt(sum_of_all(sum));
}

__global__ void __launch_bounds__(kThreads) grads_norm_kernel(const double* partial, uint32_t n, float* norm) {
    after_previous();
    const double d = norm_of(partial, n);
    if (threadIdx.x == 0) *norm = (float)d;
}

// Whether 32 bits hold the factor to their last one.
__device__ __forceinline__ bool held_in_32_bits(double f) { return f == (double)(float)f || !(fabs(f) < 0x1p-126); }

template <Mode M, typename A, typename B>
__device__ __forceinline__ void apply_to_chunk(const A* x, B* y, int n, float f) {
    constexpr int kUnits = kChunkBytes / sizeof(A) / 8 / kThreads, kAtOnce = 2;
    if (n == kChunkBytes / sizeof(A) && ((uintptr_t)x | (uintptr_t)y) % 16 == 0) {
#pragma unroll
        for (int u = 0; u < kUnits; u += kAtOnce) {
            Words<A, 8> w[kAtOnce];
            Words<B, 8> o[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                w[k] = load_words<A, 8>(x + 8 * (threadIdx.x + kThreads * (u + k)));
                if (M == kStep) o[k] = load_words<B, 8>(y + 8 * (threadIdx.x + kThreads * (u + k)));
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                float g[8], p[8];
                widen<A, 8>(w[k], g);
                if (M == kStep) widen<B, 8>(o[k], p);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = M == kStep ? fmaf(-f, g[i], p[i]) : f * g[i];
                store_words<B, 8>(y + 8 * (threadIdx.x + kThreads * (u + k)), narrow<B, 8>(p));
            }
        }
        return;
    }
    for (int at = threadIdx.x; at < n; at += 8 * kThreads) {
        float g[8], p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = at + kThreads * i;
            g[i] = c < n ? to_f32<A>(x[c]) : 0.f;
            if (M == kStep) p[i] = c < n ? to_f32<B>(y[c]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + kThreads * i < n) y[at + kThreads * i] = from_f32<B>(M == kStep ? fmaf(-f, g[i], p[i]) : f * g[i]);
    }
}

// The same where 32 bits do not hold the factor, in 64: gradients so large that the norm is 2^126 times what they are clipped to, or more.
template <Mode M, typename A, typename B>
__device__ __noinline__ void apply_in_64_bits(const A* x, B* y, int n, double f) {
    for (int c = threadIdx.x; c < n; c += kThreads) {
        const double g = f * (double)to_f32<A>(x[c]);
        y[c] = from_f32<B>((float)(M == kStep ? (double)to_f32<B>(y[c]) - g : g));
    }
}

template <Mode M, typename A, typename B>
__device__ __forceinline__ void apply_to_chunk(const A* x, B* y, int n, double f) {
    if (held_in_32_bits(f)) apply_to_chunk<M>(x, y, n, (float)f);
    else apply_in_64_bits<M>(x, y, n, f);
}

template <Mode M, typename A>
__device__ __forceinline__ void apply_by_out(const Piece& p, int64_t at, int n, double f) {
    const A* x = (const A*)p.in + at;
    if (p.out_type == HALOS_F32) apply_to_chunk<M>(x, (float*)p.out + at, n, f);
    else if (p.out_type == HALOS_BF16) apply_to_chunk<M>(x, (__nv_bfloat16*)p.out + at, n, f);
    else apply_to_chunk<M>(x, (__half*)p.out + at, n, f);
}

// The chunks are taken from the last one on: what the pass for the norm read last is still in the L2 cache.
template <Mode M, int N>
__global__ void __launch_bounds__(kThreads, kResident) grads_apply_kernel(const __grid_constant__ Table<N> t) {
    double f = 1.0;
    after_previous();
    if (t.partial) {
        const double n = norm_of(t.partial, t.partials);
        if (n > (double)t.max_norm) f = (double)t.max_norm / n;
        if (t.norm && blockIdx.x == 0 && threadIdx.x == 0) *t.norm = (float)n;
    }
    const double factor = M == kStep ? (double)t.rate * f : f;
    const uint32_t end = min(t.chunks, (blockIdx.x + 1) * t.run);
    for (uint32_t c = blockIdx.x * t.run; c < end; ++c) {
        const uint32_t chunk = t.chunks - 1 - c;
        const Piece& p = t.piece[piece_of(t, chunk)];
        if (M == kClip && p.in == p.out && (float)factor == 1.f) continue;
        const uint32_t size = p.in_type == HALOS_F32 ? 4 : 2;
        const int64_t at = (int64_t)(chunk - p.first) * (kChunkBytes / size), left = p.n - at;
        const int n = (int)(left < kChunkBytes / size ? left : kChunkBytes / size);
        if (p.in_type == HALOS_F32) apply_by_out<M, float>(p, at, n, factor);
        else if (p.in_type == HALOS_BF16) apply_by_out<M, __nv_bfloat16>(p, at, n, factor);
        else apply_by_out<M, __half>(p, at, n, factor);
    }
}

// ------------------------------------------------------------------------------------------------ host

struct Range { uintptr_t from, to; uint64_t index; };

// Written tensors against one another and against the gradients.  A gradient may be its own output.
int check_overlap(const halos_grads_args* a) {
    Range* r = new (std::nothrow) Range[a->count];
    if (!r) return fail(HALOS_ERR_OOM, "gradients: host memory");
    uint64_t n = 0;
    for (uint64_t i = 0; i < a->count; ++i)
        if (a->numel[i]) r[n++] = Range{(uintptr_t)a->outs[i], (uintptr_t)a->outs[i] + (uintptr_t)a->numel[i] * size_of(a->out_dtypes[i]), i};
    std::sort(r, r + n, [](const Range& x, const Range& y) { return x.from < y.from; });
    bool bad = false;
    for (uint64_t i = 1; i < n; ++i) bad |= r[i].from < r[i - 1].to;
    for (uint64_t i = 0; i < a->count && !bad; ++i) {
        if (!a->numel[i]) continue;
        const uintptr_t from = (uintptr_t)a->grads[i], to = from + (uintptr_t)a->numel[i] * size_of(a->grad_dtypes[i]);
        // The written ranges are in order and apart: the first that ends after `from` is the only one that could be the gradient itself.
        const Range* at = std::upper_bound(r, r + n, from, [](uintptr_t v, const Range& y) { return v < y.to; });
        if (at == r + n || at->from >= to) continue;
        const bool same = at->index == i && at->from == from && a->out_dtypes[i] == a->grad_dtypes[i];
        bad |= !same || (at + 1 < r + n && at[1].from < to);
    }
    delete[] r;
    return bad ? fail(HALOS_ERR_INVALID_ARG, "gradients: a tensor that is written overlaps another") : HALOS_OK;
}

int check(const halos_grads_args* a, bool outs, bool norm) {
    if (!a || a->struct_size != sizeof(halos_grads_args)) return fail(HALOS_ERR_INVALID_ARG, "gradients: args missing or of another size");
    if (a->count && (!a->grads || !a->numel || !a->grad_dtypes || (outs && (!a->outs || !a->out_dtypes)))) return fail(HALOS_ERR_INVALID_ARG, "gradients: null array");
    if (a->count > 0xffffffull) return fail(HALOS_ERR_UNSUPPORTED, "gradients: over 2^24 - 1 tensors");
    for (uint64_t i = 0; i < a->count; ++i) {
        if (!is_type(a->grad_dtypes[i]) || (outs && !is_type(a->out_dtypes[i]))) return fail(HALOS_ERR_INVALID_ARG, "gradients: dtype");
        if (a->numel[i] < 0) return fail(HALOS_ERR_INVALID_ARG, "gradients: numel");
        if (a->numel[i] >= 1ll << 40) return fail(HALOS_ERR_UNSUPPORTED, "gradients: a tensor of 2^40 elements or more");
        if (!a->numel[i]) continue;
        if (!a->grads[i] || (outs && !a->outs[i])) return fail(HALOS_ERR_INVALID_ARG, "gradients: null pointer");
        if ((uintptr_t)a->grads[i] % size_of(a->grad_dtypes[i]) || (outs && (uintptr_t)a->outs[i] % size_of(a->out_dtypes[i])))
            return fail(HALOS_ERR_INVALID_ARG, "gradients: a tensor is not aligned to its elements");
    }
    if (norm && !(a->max_norm >= 0.f)) return fail(HALOS_ERR_INVALID_ARG, "gradients: max_norm must not be negative");
    return HALOS_OK;
}

uint64_t grid_limit(int32_t device) { return (uint64_t)sm_count(device) * kResident * kWaves; }

// Calls `launch` with tables of as many tensors as fit one; the number of CTAs goes by the chunks and is `limit` at most.
template <int N, typename F>
int in_tables(const halos_grads_args* a, bool outs, uint64_t limit, F launch) {
    uint64_t i = 0;
    for (;;) {
        Table<N> t{};
        uint64_t chunks = 0;
        for (; i < a->count && t.pieces < N; ++i) {
            if (!a->numel[i]) continue;
            const uint64_t here = ((uint64_t)a->numel[i] * size_of(a->grad_dtypes[i]) + kChunkBytes - 1) / kChunkBytes;
            if (chunks + here > 0xffffffffull) {
                if (!chunks) return fail(HALOS_ERR_UNSUPPORTED, "gradients: a tensor too large");
                break;
            }
            t.piece[t.pieces++] = Piece{a->grads[i], outs ? a->outs[i] : nullptr, a->numel[i], (uint32_t)chunks, a->grad_dtypes[i], (uint16_t)(outs ? a->out_dtypes[i] : 0)};
            chunks += here;
        }
        t.chunks = (uint32_t)chunks;
        t.run = (uint32_t)((chunks + limit - 1) / limit);
        if (t.pieces)
            if (int rc = launch(t, (unsigned)((chunks + t.run - 1) / t.run))) return rc;
        if (i == a->count) return HALOS_OK;
    }
}

// Small tables for few tensors: the arguments are copied with every launch.
template <typename F>
int by_count(uint64_t count, F f) {
    if (count <= 32) return f(std::integral_constant<int, 32>());
    if (count <= 320) return f(std::integral_constant<int, 320>());
    return f(std::integral_constant<int, kMostPieces>());
}

uint64_t most_partials(uint64_t count, int32_t device) { return grid_limit(device) * (1 + count / kMostPieces); }

int run(const halos_grads_args* a, bool apply, Mode mode) {
    const bool with_norm = a->norm != nullptr;
    if (int rc = enter(a->device)) return rc;
    const uint64_t limit = grid_limit(a->device);
    if (with_norm && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < most_partials(a->count, a->device) * sizeof(double)))
        return fail(HALOS_ERR_INVALID_ARG, "gradients: workspace missing, not aligned or too small");
    cudaStream_t st = (cudaStream_t)a->stream;
    double* partial = (double*)a->workspace;
    uint32_t partials = 0;
    return by_count(a->count, [&](auto size) -> int {
        constexpr int N = decltype(size)::value;
        if (with_norm) {
            const uint64_t room = a->workspace_bytes / sizeof(double);
            if (int rc = in_tables<N>(a, false, limit, [&](const Table<N>& t, unsigned grid) {
                    if (partials + (uint64_t)grid > room) return fail(HALOS_ERR_INVALID_ARG, "gradients: workspace too small");
                    grads_squares_kernel<N><<<grid, kThreads, 0, st>>>(t, partial + partials);
                    partials += grid;
                    return cuda_status(cudaGetLastError(), "gradient norm launch");
                }))
                return rc;
        }
        bool first = true;
        if (apply) {
            if (int rc = in_tables<N>(a, true, limit, [&](Table<N>& t, unsigned grid) {
                    t.partial = with_norm ? partial : nullptr, t.partials = partials, t.max_norm = a->max_norm, t.rate = a->rate;
                    t.norm = first ? a->norm : nullptr, first = false;
                    return launch_after(mode == kStep ? grads_apply_kernel<kStep, N> : grads_apply_kernel<kClip, N>, grid, kThreads, 0, st, "gradient launch", t);
                }))
                return rc;
        }
        if (with_norm && first) {  // nobody has written the norm
            return launch_after(grads_norm_kernel, 1, kThreads, 0, st, "gradient norm launch", (const double*)partial, partials, a->norm);
        }
        return HALOS_OK;
    });
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_grads_workspace(const halos_grads_args* a, uint64_t* bytes) {
    using namespace halos_step;
    if (!a || a->struct_size != sizeof(halos_grads_args) || !bytes) return fail(HALOS_ERR_INVALID_ARG, "gradients: args missing or of another size");
    if (a->count > 0xffffffull) return fail(HALOS_ERR_UNSUPPORTED, "gradients: over 2^24 - 1 tensors");
    if (int rc = enter(a->device)) return rc;
    *bytes = most_partials(a->count, a->device) * sizeof(double);
    return HALOS_OK;
}

extern "C" int halos_grad_norm(const halos_grads_args* a) {
    using namespace halos_step;
    if (int rc = check(a, false, false)) return rc;
    if (!a->norm) return fail(HALOS_ERR_INVALID_ARG, "gradients: null pointer");
    return run(a, false, kClip);
}

extern "C" int halos_clip_grads(const halos_grads_args* a) {
    using namespace halos_step;
    if (int rc = check(a, true, true)) return rc;
    if (!a->norm) return fail(HALOS_ERR_INVALID_ARG, "gradients: null pointer");
    if (int rc = check_overlap(a)) return rc;
    return run(a, true, kClip);
}

extern "C" int halos_sgd_step(const halos_grads_args* a) {
    using namespace halos_step;
    if (int rc = check(a, true, a && a->norm)) return rc;
    if (!isfinite(a->rate)) return fail(HALOS_ERR_INVALID_ARG, "gradients: rate must be finite");
    if (int rc = check_overlap(a)) return rc;
    return run(a, true, kStep);
}
