// What the norms' two directions share: rows and their strides, the threads that hold a row, and copies that run ahead.
#pragma once
#include "step_vector.cuh"

#include <math.h>
#include <string.h>
#include <type_traits>

namespace halos_step {
namespace norm {

constexpr int kThreads = 256, kMostThreads = 512;

struct Rows {
    char* at;
    const char* span[2];                   // first byte of any row, and the one behind the last
    int64_t stride[3];                     // in elements, from the innermost outer size on
};
struct Params {
    Rows in[3];                            // x, residual; back: summed, dy, dsummed
    Rows out[2];                           // y, summed; back: dx
    const char* weight;
    char* dweight;
    float *scales, *rstd, *partial;
    uint32_t rows, dim, inner, middle, even;  // the inner two of up to three outer sizes; even: there is one at most
    uint32_t arrays;                       // of `in` that there are
    uint32_t weight_type, group, group_bits, groups;   // elements to a scale, as a power of two where it is not the row, and scales to a row
    uint32_t splits;                       // partial sums of dweight
    uint32_t lanes, stages;                // threads to a row; rows of a thread on their way or being worked on
    uint32_t row_blocks, run, apart;       // rows of CTAs at a time; how many of those a CTA takes, how far apart
    float eps, inverse_dim;
};

// Where a row begins, in elements.
__device__ __forceinline__ int64_t start_of(const Params& P, const Rows& R, uint32_t row) {
    if (P.even) return row * R.stride[0];
    const uint32_t outer = row / P.inner, k = row - outer * P.inner, i = outer / P.middle, j = outer - i * P.middle;
    return i * R.stride[2] + j * R.stride[1] + k * R.stride[0];
}
template <typename T>
__device__ __forceinline__ T* row_at(const Params& P, const Rows& R, uint32_t row) { return reinterpret_cast<T*>(R.at) + start_of(P, R, row); }

__device__ __forceinline__ float weight_at(const Params& P, uint32_t c) {
    if (P.weight_type == HALOS_F32) return reinterpret_cast<const float*>(P.weight)[c];
    if (P.weight_type == HALOS_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(P.weight)[c]);
    return __half2float(reinterpret_cast<const __half*>(P.weight)[c]);
}

// The sum over a CTA of kThreads, the same in every thread.
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

// ------------------------------------------------------------------------------------------------ rows that a CTA holds

// `lanes` threads (a power of two, within a warp or of several) go through a row together, N accesses of V elements each.
//   kWhole    rows begin on 16 bytes and consist of whole accesses of 16 bytes
//   kShifted  rows of all tensors begin equally far behind such a boundary: whole accesses inside, the ends element by element where they are written.  A
//             thread's rows have one shift, so that it has the same columns in all of them
//   kLoose    neither: pairs of elements, each on its own
enum Mode { kWhole, kShifted, kLoose };
template <typename T, Mode M> constexpr int kVector = M == kLoose ? 2 : 16 / (int)sizeof(T);

template <int V> __device__ __forceinline__ bool owned(int c, int e, int dim) { return c + e >= 0 && c + e < dim; }

// The row's elements of an access, one by one, and 0 in the others' places.
template <typename T, int V>
__device__ __forceinline__ Words<T, V> pick(const T* row, int c, int dim) {
    Words<T, V> r = no_words<T, V>();
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (owned<V>(c, e, dim)) put_element<T, V>(r, e, row[c + e]);
    return r;
}
// What is not the row's counts as 0: an access at its end brings what lies beside it in memory.
template <int V, Mode M>
__device__ __forceinline__ void keep_own(float2 (&v)[V / 2], int c, int dim) {
    if (M == kShifted && (c < 0 || c + V > dim)) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) v[i] = make_float2(owned<V>(c, 2 * i, dim) ? v[i].x : 0.f, owned<V>(c, 2 * i + 1, dim) ? v[i].y : 0.f);
    }
}
template <typename T, int V, Mode M>
__device__ __forceinline__ void store_part(T* row, int c, int dim, const float2 (&v)[V / 2]) {
    if (c >= dim) return;
    if (M == kWhole || (M == kShifted && c >= 0 && c + V <= dim)) store_words<T, V>(row + c, narrow<T, V>(v));
    else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if (owned<V>(c, 2 * i, dim)) row[c + 2 * i] = from_f32<T>(v[i].x);
            if (owned<V>(c, 2 * i + 1, dim)) row[c + 2 * i + 1] = from_f32<T>(v[i].y);
        }
    }
}

constexpr uint32_t kMostStages = 3;

// A thread's part of rows.  What it will need is copied to places of its own in shared memory while it works on the rows before: registers would hold
// half of what has to be on its way.  A thread's N accesses are L apart, so that all addresses but a row's first are constants: rows of whole warps have
// L = 32, short ones L = 4 or 8 threads (or, with N = 1, any number).
template <typename T, int N, int L, Mode M, int THREADS, int ARRAYS>
struct Threads {
    static constexpr int V = kVector<T, M>, H = V / 2, kAccess = V * (int)sizeof(T);
    static constexpr int kArray = N * THREADS * kAccess, kStage = ARRAYS * kArray;          // bytes
    static constexpr int kPart = V >= 4 ? 4 : 2, kParts = V / kPart;                        // of an access's weights
    const Params& P;
    uint32_t lanes, own, per, from;
    int first, off, dim;                   // column of the first access; shift
    char* mine;                            // [stages][arrays][N] accesses of this thread
    float* rstd;                           // [stages] of this thread; back
    float* weight;                         // of this thread's first access
    uint32_t weight_step;                  // floats from one part of an access to the next; kShifted: of all accesses

    __device__ __forceinline__ Threads(const Params& P, char* shared, bool back) : P(P) {
        lanes = P.lanes, per = THREADS / lanes, dim = (int)P.dim;
        const uint32_t lane = threadIdx.x % lanes;
        // Rows of one warp are as many apart as the CTA has warps, 8: they have one shift.
        own = lanes < 32 ? threadIdx.x % 32 / lanes * (THREADS / 32) + threadIdx.x / 32 : threadIdx.x / lanes;
        from = blockIdx.x / P.apart * P.apart * P.run + blockIdx.x % P.apart;
        off = M == kShifted ? (int)((uintptr_t)(reinterpret_cast<T*>(P.in[0].at) + (int64_t)row_of(0) * P.in[0].stride[0]) / sizeof(T) % V) : 0;  // of rows that are not there, too
        first = (int)(lane / L * N * L + lane % L) * V - off;
        mine = shared + threadIdx.x * kAccess;
        float* behind = reinterpret_cast<float*>(shared + P.stages * kStage);
        rstd = behind + threadIdx.x;
        if (back) behind += P.stages * THREADS;
        weight_step = M == kShifted ? THREADS * kPart : (lanes * N) * kPart;
        weight = behind + (M == kShifted ? threadIdx.x * kPart : first / V * kPart);
    }
    __device__ __forceinline__ bool leads() const { return threadIdx.x % lanes == 0; }
    __device__ __forceinline__ int column(int j) const { return first + j * L * V; }

    // kShifted: [N][parts][threads] of kPart floats; else [parts][accesses], for all rows
    __device__ __forceinline__ float* weight_at_part(int j, int p) const { return M == kShifted ? weight + (j * kParts + p) * THREADS * kPart : weight + p * weight_step + j * L * kPart; }
    __device__ __forceinline__ void load_weights() const {
        if (M == kShifted || threadIdx.x < lanes) {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) weight_at_part(j, e / kPart)[e % kPart] = owned<V>(column(j), e, dim) ? weight_at(P, column(j) + e) : 0.f;
        }
        __syncthreads();
    }
    __device__ __forceinline__ void weights(int j, float2 (&w)[H]) const {
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            float2 part[kPart / 2];
            widen<float, kPart>(load_words<float, kPart>(weight_at_part(j, p)), part);
#pragma unroll
            for (int i = 0; i < kPart / 2; ++i) w[p * kPart / 2 + i] = part[i];
        }
    }
    __device__ __forceinline__ char* behind() const { return reinterpret_cast<char*>((weight - (M == kShifted ? threadIdx.x * kPart : first / V * kPart)) + (M == kShifted ? N * kParts * THREADS * kPart : kParts * weight_step)); }
    __device__ __forceinline__ uint32_t row_of(uint32_t turn) const { return (from + turn * P.apart) * per + own; }

    __device__ __forceinline__ void fetch(uint32_t turn, int stage, bool back) const {
        const uint32_t row = row_of(turn);
        if (turn < P.run && row < P.rows) {
            char* to = mine + stage * kStage;
#pragma unroll
            for (int array = 0; array < ARRAYS; ++array) {
                const Rows& R = P.in[array];
                const T* from = row_at<const T>(P, R, row);
                const T* at = from + first;
                // accesses at the ends of all rows but the tensor's first and last stay within it
                const bool inside = M == kWhole || (M == kShifted && reinterpret_cast<const char*>(from) >= R.span[0] + 16 && reinterpret_cast<const char*>(from + dim) + 16 <= R.span[1]);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    char* t = to + array * kArray + j * THREADS * kAccess;
                    if (column(j) >= dim) continue;
                    if (inside) copy_16(t, at + j * L * V);
                    else *reinterpret_cast<Words<T, V>*>(t) = pick<T, V>(from, column(j), dim);
                }
            }
            if (back) copy_4(rstd + stage * THREADS, P.rstd + row);
        }
        copies_end();
    }
    // An access that has arrived, as floats; 0 where there is none.  At a row's ends it holds what lies beside it.
    __device__ __forceinline__ void arrived(int stage, int array, int j, bool here, float2 (&v)[H]) const {
        Words<T, V> w = no_words<T, V>();
        if (here && column(j) < dim) w = load_words<T, V>(reinterpret_cast<const T*>(mine + stage * kStage + array * kArray + j * THREADS * kAccess));
        widen<T, V>(w, v);
    }
};

// Sums and maxima over the threads of a row: within a warp (its 32 threads where WHOLE), or of whole warps, which then meet at a barrier of their own.  Two sets
// of places in turn: whoever writes to one again has met, at the barrier in between, all who read it.
template <bool WHOLE>
struct RowSums {
    uint32_t lanes;
    uint32_t* s_part;                      // [2][warps]
    uint32_t turn;
    __device__ __forceinline__ RowSums(uint32_t lanes, uint32_t* s_part) : lanes(lanes), s_part(s_part), turn(0) {}
    template <typename A, typename F>
    __device__ __forceinline__ A within(A v, F join) const {
#pragma unroll
        for (uint32_t o = 16; o; o >>= 1)
            if (WHOLE || o < lanes) v = join(v, __shfl_xor_sync(~0u, v, o));
        return v;
    }
    template <typename A, typename F>
    __device__ __forceinline__ A over_warps(A v, bool& any, F join) {
        uint32_t* s = s_part + turn;
        turn ^= kMostThreads / 32;
        if (threadIdx.x % 32 == 0) memcpy(&s[threadIdx.x / 32], &v, 4);
        const uint32_t slot = threadIdx.x / lanes;
        int met;
        asm volatile("{\n .reg .pred p, q;\n setp.ne.s32 q, %1, 0;\n barrier.cta.red.or.aligned.pred p, %2, %3, q;\n selp.s32 %0, 1, 0, p;\n}" : "=r"(met) : "r"((int)any), "r"(slot + 1), "r"(lanes) : "memory");
        any = met;
        s += slot * (lanes / 32);
        memcpy(&v, &s[0], 4);
        for (uint32_t w = 1; w < lanes / 32; ++w) {
            A part;
            memcpy(&part, &s[w], 4);
            v = join(v, part);
        }
        return v;
    }
    __device__ __forceinline__ float sum(float v) {
        const auto add = [](float a, float b) { return a + b; };
        v = within(v, add);
        bool any = false;
        return lanes <= 32 ? v : over_warps(v, any, add);
    }
    __device__ __forceinline__ float sum(float v, bool& any) {   // any: over the warp, or the row where it is of several
        const auto add = [](float a, float b) { return a + b; };
        v = within(v, add), any = __any_sync(~0u, any);
        return lanes <= 32 ? v : over_warps(v, any, add);
    }
    __device__ __forceinline__ uint32_t top(uint32_t v) {
        const auto larger = [](uint32_t a, uint32_t b) { return max(a, b); };
        v = within(v, larger);
        bool any = false;
        return lanes <= 32 ? v : over_warps(v, any, larger);
    }
};

// ------------------------------------------------------------------------------------------------ host

// How rows are spread over threads, and how many of the CTAs an SM holds.  n = 0: no CTA holds such rows, for want of registers (over 16384 elements or a little less), or of shared
// memory for one row of each input to every thread under the spread that registers alone have chosen (f32 with two or three inputs: widths of 510 to 768, of 4094 to 6144, and backward
// with dsummed from 8193, off 16 bytes from 4094, on).  Kernels with loops take them.
struct Shape {
    uint32_t n, lanes, apart, threads, resident, stages, shared;   // apart: a thread's accesses
    uint32_t per() const { return threads / lanes; }
};

int check(const halos_rms_norm_args* a);
// Rows, weights and what goes with them; the tensors of `in` and `out` that are there are set beforehand.
int fill(const halos_rms_norm_args* a, Params& P, uint32_t outs);
Mode mode_of(const Params& P, uint32_t size, uint32_t outs, uint32_t out_size);
inline void set(Rows& R, const void* at, const int64_t (&stride)[3]) {
    R.at = (char*)at;
    for (int i = 0; i < 3; ++i) R.stride[i] = stride[i];
}

// Rows of many accesses take whole warps with N accesses to a thread, few first.
inline void spread_over(Shape& s, uint32_t accesses, uint32_t v, Mode mode, uint32_t elements, uint32_t most_lanes, uint32_t above) {
    if (s.n) return;
    s.apart = 32;
    for (uint32_t n : {2u, 3u, 1u, 4u, 6u, 8u, 16u})   // of equals the first
        if (n * v <= elements && n * v > above && !(mode == kLoose && (n == 6 || n == 3)))
            for (uint32_t lanes = 32; lanes <= most_lanes; lanes *= 2)
                if (lanes * n >= accesses && (!s.n || lanes * n < s.lanes * s.n)) s.n = n, s.lanes = lanes;
}
// Rows of up to 32 accesses: 4 or 8 threads with two or three each where rows are whole (what a row costs beside its accesses then falls on few threads: 410000 rows of
// 56 f32 in 8 bits 70 us with a thread to an access, 55 us with eight of them), else a thread to an access.  `least` threads stay neighbours.
inline void spread_short(Shape& s, uint32_t accesses, Mode mode, uint32_t least) {
    if (mode == kWhole)
        for (uint32_t lanes : {4u, 8u})
            for (uint32_t n : {2u, 3u})
                if (lanes >= least && lanes * n >= accesses && lanes < accesses && (!s.n || lanes * n < s.lanes * s.n)) s.n = n, s.lanes = s.apart = lanes;
    if (s.n) return;
    for (s.n = 1, s.apart = 32, s.lanes = 4; s.lanes < accesses;) s.lanes *= 2;
}

// One warp to a row where that takes kFew elements to a thread at most, else warps with few accesses to a thread: what they cost at the barrier is
// less than what long threads cost in registers (2048 bf16: two accesses to each of 128 threads 47 us, eight to each of 32 51 us).
constexpr uint32_t kFew = 24;
inline void spread_over(Shape& s, uint32_t v, Mode mode, uint32_t accesses, uint32_t least) {
    if (accesses <= 32) return spread_short(s, accesses, mode, least);
    spread_over(s, accesses, v, mode, kFew, 32, 0);
    spread_over(s, accesses, v, mode, (mode == kLoose ? 8 : 3) * v, kThreads, 0);
    spread_over(s, accesses, v, mode, kFew, kThreads, 0);
    spread_over(s, accesses, v, mode, 32, kMostThreads, kFew);
}
template <typename T, int N, Mode M> constexpr bool kWide = N * kVector<T, M> > (int)kFew;   // a CTA has 512 threads, and 128 registers to each of them
inline uint32_t accesses_of(uint32_t dim, uint32_t v, Mode mode) { return mode == kShifted ? (dim + 2 * v - 2) / v : (dim + v - 1) / v; }

template <typename F>
int by_type(uint32_t type, F f) {
    if (type == HALOS_F32) return f(float());
    if (type == HALOS_BF16) return f(__nv_bfloat16());
    return f(__half());
}
// Numbers of accesses that there are kernels for; 32 elements to a thread at most.
template <typename T, typename F>
int by_accesses(uint32_t n, uint32_t apart, Mode mode, F f) {
    if (apart < 32) {
        constexpr std::integral_constant<Mode, kWhole> whole;
        const auto counts = [&](auto l) { return n == 2 ? f(std::integral_constant<int, 2>(), l, whole) : f(std::integral_constant<int, 3>(), l, whole); };
        return apart == 4 ? counts(std::integral_constant<int, 4>()) : counts(std::integral_constant<int, 8>());
    }
    constexpr std::integral_constant<int, 32> l;
    const auto counts = [&](auto m) -> int {
        constexpr Mode M = decltype(m)::value;
        constexpr int kMost = 32 / kVector<T, M>;
        if constexpr (kMost >= 16)
            if (n == 16) return f(std::integral_constant<int, 16>(), l, m);
        if constexpr (kMost >= 8)
            if (n == 8) return f(std::integral_constant<int, 8>(), l, m);
        if constexpr (kMost >= 8 && M != kLoose)
            if (n == 6) return f(std::integral_constant<int, 6>(), l, m);
        if constexpr (M != kLoose)
            if (n == 3) return f(std::integral_constant<int, 3>(), l, m);
        if (n == 4) return f(std::integral_constant<int, 4>(), l, m);
        if (n == 2) return f(std::integral_constant<int, 2>(), l, m);
        return f(std::integral_constant<int, 1>(), l, m);
    };
    if (mode == kWhole) return counts(std::integral_constant<Mode, kWhole>());
    if (mode == kShifted) return counts(std::integral_constant<Mode, kShifted>());
    return counts(std::integral_constant<Mode, kLoose>());
}

}  // namespace norm
}  // namespace halos_step
