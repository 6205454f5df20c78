// Distillation from a teacher's top logits mixed with cross-entropy: loss, gradient, or both.
//
// Bound by memory: a forward pass reads the logits once, a backward pass reads and writes them once, and the two together
// read and write them once.  The second constraint is the exponential (16 per clock and SM): with a temperature a
// logit needs exp(z) and exp(z/T), in the statistics and again in the gradient.  Where T is 1, 2 or 4 the
// first is the second to the power T, which costs multiplications instead (kSquarings).
//
// Measured: 8192 x 50304 bf16 logits, 64 entries, T = 2, loss with gradient 352 to 365 us (4.7 to 4.5 TB/s, floor 256 us; the exponential
// unit and the issue slots are both 58% busy); gradient alone of 2048 x 32003 f16, T = 1: 58 us (4.6 TB/s).
#include "step_tcgen05.cuh"

namespace halos_step {
namespace {

constexpr int kMaxTeacher = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
enum Mode { kForward = 0, kBackward = 1, kBoth = 2 };

struct DistillParams {
    const char* z;
    char* dz;
    const void *labels, *index;
    const char* t;
    float *loss, *stats;
    const float* dloss;
    int64_t z_stride, dz_stride, index_stride, t_stride;  // in elements
    int64_t vocab, ignore_index;
    uint32_t k, labels_64, index_64, teacher_dtype;
    float temperature, mix;
};

__device__ __forceinline__ float teacher_at(const DistillParams& P, int64_t at) {
    if (P.teacher_dtype == HALOS_F32) return reinterpret_cast<const float*>(P.t)[at];
    if (P.teacher_dtype == HALOS_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(P.t)[at]);
    return __half2float(reinterpret_cast<const __half*>(P.t)[at]);
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// ------------------------------------------------------------------------------------------------ rows held in shared memory

// A CTA of kThreads + 32 walks rows, one held in shared memory at a time, in chunks.  Its last warp copies: as soon as the
// gradient of a chunk has been formed the next row's chunk is fetched over it, and meanwhile that warp works out the
// teacher's side of the next row.  The other warps go over the row twice, for the statistics and for the gradient,
// which they store from registers.  So the logits cross HBM once; several CTAs to an SM fill each other's gaps.
// A wait that runs out is marked and ends every later one at once; the loops and their barriers still run to the end.
template <int kThreads> struct Held {
    static constexpr int kWarps = kThreads / 32, kUnroll = 4, kChunk = kThreads * kUnroll;  // vectors
    static constexpr int kPerSM = kThreads == 128 ? 6 : kThreads == 256 ? 3 : 1;
    static constexpr int kMostChunks = 32;
};

struct Slot {  // what the last warp says of a row beside the entries themselves
    float plogp, pz, label_z, lse1, lseT, g;
    int label, ignored, bad, any;
};

// Splits a row at the 16-byte boundaries: elements [0, head) and [tail, V) singly, `vectors` whole vectors between.
template <typename T> struct Cut {
    int head, vectors, tail, singles;
    __device__ __forceinline__ Cut(const T* z, int V) {
        constexpr int N = 16 / sizeof(T);
        head = (int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(T);
        if (head > V) head = V;
        vectors = (V - head) / N;
        tail = head + vectors * N;
        singles = head + V - tail;
    }
    __device__ __forceinline__ int single(int i) const { return i < head ? i : i - head + tail; }
};

// A 32-bit word of a row (one element of 32 bits or two of 16): -infinity throughout, the larger of two, the largest in one.
template <typename T> __device__ __forceinline__ uint32_t low_word();
template <> __device__ __forceinline__ uint32_t low_word<float>() { return 0xff800000u; }
template <> __device__ __forceinline__ uint32_t low_word<__nv_bfloat16>() { return 0xff80ff80u; }
template <> __device__ __forceinline__ uint32_t low_word<__half>() { return 0xfc00fc00u; }
template <typename T> __device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max_words<float>(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
template <> __device__ __forceinline__ uint32_t max_words<__nv_bfloat16>(uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
}
template <> __device__ __forceinline__ uint32_t max_words<__half>(uint32_t a, uint32_t b) {
    const __half2 m = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
}
template <typename T> __device__ __forceinline__ float max_in_word(uint32_t w) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w);
    else {
        const float2 f = unpack2<T>(w);
        return fmaxf(f.x, f.y);
    }
}
// The pairs of a vector, in order, and back.
template <typename T> struct Pairs {
    static constexpr int kCount = sizeof(T) == 4 ? 2 : 4;
    __device__ static __forceinline__ float2 get(const uint4& v, int i) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        else return unpack2<T>(w[i]);
    }
    __device__ static __forceinline__ uint4 join(const float2* f) {
        if constexpr (sizeof(T) == 4)
            return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
        else return make_uint4(pack2<T>(f[0].x, f[0].y), pack2<T>(f[1].x, f[1].y), pack2<T>(f[2].x, f[2].y), pack2<T>(f[3].x, f[3].y));
    }
};

// The last warp's work on a row: label, teacher's probabilities, logits at their places.
template <typename T>
__device__ void describe_row(const DistillParams& P, const T* z, int64_t row, bool back, float* p, float* zk, int* idx, Slot& S) {
    const int lane = threadIdx.x & 31;
    int64_t label = 0;
    int ignored = 0, bad = 0;
    float label_z = 0.f;
    if (P.labels) {
        label = P.labels_64 ? static_cast<const int64_t*>(P.labels)[row] : (int64_t)static_cast<const int32_t*>(P.labels)[row];
        ignored = label == P.ignore_index;
        bad = !ignored && (label < 0 || label >= P.vocab);
        if (lane == 0 && !ignored && !bad) label_z = to_f32<T>(z[label]);
    }
    const float invT = 1.f / P.temperature;
    float top = -INFINITY;
    for (uint32_t first = 0; first < P.k; first += 128) {
        int64_t j[4];
        float t[4], at_z[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t i = first + u * 32 + lane;
            j[u] = -1, t[u] = 0.f;
            if (i < P.k) {
                const int64_t at = row * P.index_stride + i;
                j[u] = P.index_64 ? static_cast<const int64_t*>(P.index)[at] : (int64_t)static_cast<const int32_t*>(P.index)[at];
                t[u] = teacher_at(P, row * P.t_stride + i) * invT;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool in = j[u] >= 0 && j[u] < P.vocab;
            if (!in && j[u] != -1) bad = 1;
            at_z[u] = in && !ignored ? to_f32<T>(z[j[u]]) : 0.f;
            if (!in) j[u] = -1, t[u] = -INFINITY;
            top = fmaxf(top, t[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t i = first + u * 32 + lane;
            if (i < P.k) p[i] = t[u], zk[i] = at_z[u], idx[i] = (int)j[u];
        }
    }
    top = warp_max(top);
    float sum = 0.f;
    for (uint32_t i = lane; i < P.k; i += 32)
        if (p[i] != -INFINITY) sum += fast_exp2((p[i] - top) * kLog2e);
    sum = warp_sum(sum);
    const float log_sum = logf(sum);
    float plogp = 0.f, pz = 0.f;
    for (uint32_t i = lane; i < P.k; i += 32) {
        const float t = p[i];
        float q = 0.f;
        if (t != -INFINITY) {
            const float logp = t - top - log_sum;
            q = fast_exp2(logp * kLog2e);
            if (!(q == 0.f)) plogp += q * logp, pz += q * zk[i];  // 0 log 0 = 0, whatever the logit there; a NaN stays one
        }
        p[i] = q;
    }
    plogp = warp_sum(plogp);
    pz = warp_sum(pz);
    bad = __any_sync(~0u, bad);
    if (lane == 0) {
        S.plogp = plogp, S.pz = pz, S.any = !(sum == 0.f), S.label = bad ? -1 : (int)label, S.ignored = ignored, S.bad = bad, S.label_z = label_z;
        if (P.dloss) S.g = P.dloss[row];
        if (back) S.lse1 = P.stats[2 * row], S.lseT = P.stats[2 * row + 1];
    }
}

// exp2 of d cT, and of d c1 (a power of the first where the temperature allows).
template <int kSquarings> struct Exponentials {
    float2 cT, c1;
    __device__ __forceinline__ explicit Exponentials(float temperature) : cT(both(kLog2e / temperature)), c1(both(kLog2e)) {}
    __device__ __forceinline__ void operator()(float2 dT, float2 d1, float2& eT, float2& e1) const {
        eT = exp2_both(mul2(dT, cT));
        if constexpr (kSquarings >= 0) {
            e1 = eT;
#pragma unroll
            for (int i = 0; i < kSquarings; ++i) e1 = mul2(e1, e1);
        } else {
            e1 = exp2_both(mul2(d1, c1));
        }
    }
};

// a q1 + b qT of a row; where T = 2^n, q1 = qT^T exp(T lseT - lse1).
template <int kSquarings> struct Gradient {
    const Exponentials<kSquarings>& form;
    float a, b;
    float2 minusT, minus1, aa, bb, ab;
    __device__ __forceinline__ Gradient(const Exponentials<kSquarings>& e, const DistillParams& P, const Slot& S, float lse1, float lseT) : form(e) {
        const float g = S.bad ? NAN : S.g, LT = P.temperature * lseT;
        a = P.labels ? g * (1.f - P.mix) : 0.f, b = S.any || S.bad ? g * P.mix * P.temperature : 0.f;
        aa = both(kSquarings >= 0 ? a * fast_exp2((LT - lse1) * kLog2e) : a), bb = both(b), ab = add2(aa, bb);
        minusT = both(-LT), minus1 = both(-lse1);
    }
    __device__ __forceinline__ float2 operator()(float2 z) const {
        float2 qT, q1;
        form(add2(z, minusT), kSquarings >= 0 ? z : add2(z, minus1), qT, q1);
        return kSquarings == 0 ? mul2(ab, qT) : fma2(aa, q1, mul2(bb, qT));
    }
};

__device__ __forceinline__ void write_loss(const DistillParams& P, int64_t row, const Slot& S, float lse1, float lseT) {
    if (P.stats) P.stats[2 * row] = lse1, P.stats[2 * row + 1] = lseT;
    float loss = 0.f;
    if (!S.ignored) {
        if (P.labels) loss += (1.f - P.mix) * (lse1 - S.label_z);
        if (S.any) loss += P.mix * P.temperature * P.temperature * (S.plogp - S.pz / P.temperature + lseT);
        if (S.bad) loss = NAN;
    }
    P.loss[row] = loss;
}

// The row's own entries (the teacher's and the label) are formed once more, whole, and rounded once, over what is there already.
// `threads` threads, this one `at`; four to an entry look for its doubles and for the label.
template <typename T, int kSquarings>
__device__ __forceinline__ void write_entries(const DistillParams& P, T* dz, const Gradient<kSquarings>& gradient, const Slot& S, const float* p, const float* zk, const int* idx, int at,
                                              int threads) {
    for (uint32_t first = 0; first < P.k; first += threads / 4) {
        const uint32_t i = first + at / 4;
        const int j = i < P.k ? idx[i] : -1;
        float same = 0.f;
        if (j >= 0)
            for (uint32_t o = at & 3; o < P.k; o += 4) same += idx[o] == j ? p[o] : 0.f;
        same += __shfl_xor_sync(~0u, same, 1);
        same += __shfl_xor_sync(~0u, same, 2);
        if (j >= 0 && (at & 3) == 0) dz[j] = from_f32<T>(gradient(both(zk[i])).x - gradient.b * same - (P.labels && j == S.label ? gradient.a : 0.f));
    }
    if (at < 32 && P.labels && !S.bad) {
        int there = 0;
        for (uint32_t i = at; i < P.k; i += 32) there |= idx[i] == S.label;
        if (!__any_sync(~0u, there) && at == 0) dz[S.label] = from_f32<T>(gradient(both(S.label_z)).x - gradient.a);
    }
}

// A row to a warp, in registers, for rows of kShort bytes at most: everything that the row needs is asked for at once, and what a
// CTA per row spends on barriers and on waiting for its teacher falls away.
constexpr int kShort = 4096, kShortWarps = 4;
template <typename T, int kSquarings>
__global__ void __launch_bounds__(32 * kShortWarps) distill_short_kernel(const __grid_constant__ DistillParams P, int rows, int mode) {
    constexpr int kVectors = kShort / 512, kPairs = Pairs<T>::kCount;
    extern __shared__ __align__(128) char smem[];
    __shared__ Slot slots[kShortWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, V = (int)P.vocab;
    const int64_t row = (int64_t)blockIdx.x * kShortWarps + warp;
    if (row >= rows) return;
    const T* z = reinterpret_cast<const T*>(P.z) + row * P.z_stride;
    const Cut<T> c(z, V);
    const uint4* in = reinterpret_cast<const uint4*>(z + c.head);
    const uint32_t low = low_word<T>();
    uint4 x[kVectors];
#pragma unroll
    for (int u = 0; u < kVectors; ++u) x[u] = u * 32 + lane < c.vectors ? in[u * 32 + lane] : make_uint4(low, low, low, low);
    const float extra = lane < c.singles ? to_f32<T>(z[c.single(lane)]) : -INFINITY;
    float* p = reinterpret_cast<float*>(smem) + warp * 3 * P.k;
    float* zk = p + P.k;
    int* idx = reinterpret_cast<int*>(zk + P.k);
    describe_row<T>(P, z, row, mode == kBackward, p, zk, idx, slots[warp]);
    __syncwarp();
    const Slot S = slots[warp];
    const Exponentials<kSquarings> form(P.temperature);
    float lse1 = S.lse1, lseT = S.lseT;
    if (mode != kBackward) {
        uint32_t top = low;
#pragma unroll
        for (int u = 0; u < kVectors; ++u) top = max_words<T>(top, max_words<T>(max_words<T>(x[u].x, x[u].y), max_words<T>(x[u].z, x[u].w)));
        const float m = warp_max(fmaxf(max_in_word<T>(top), extra));
        const float2 minus = both(m == -INFINITY ? 0.f : -m);
        float2 sT = both(0.f), s1 = sT;
        const auto add = [&](float2 f) {  // the difference before the factor, as above
            const float2 d = add2(f, minus);
            float2 eT, e1;
            form(d, d, eT, e1);
            sT = add2(sT, eT), s1 = add2(s1, e1);
        };
        add(make_float2(extra, -INFINITY));
#pragma unroll
        for (int u = 0; u < kVectors; ++u)
            if (u * 32 < c.vectors)
#pragma unroll
                for (int q = 0; q < kPairs; ++q) add(Pairs<T>::get(x[u], q));
        lse1 = m + log2f(warp_sum(s1.x + s1.y)) * kLn2;
        lseT = m / P.temperature + log2f(warp_sum(sT.x + sT.y)) * kLn2;
        if (lane == 0) write_loss(P, row, S, lse1, lseT);
    }
    if (mode == kForward) return;
    const Gradient<kSquarings> gradient(form, P, S, lse1, lseT);
    T* dz = reinterpret_cast<T*>(P.dz) + row * P.dz_stride;
    uint4* out = reinterpret_cast<uint4*>(dz + c.head);
#pragma unroll
    for (int u = 0; u < kVectors; ++u)
        if (u * 32 + lane < c.vectors) {
            float2 f[kPairs];
#pragma unroll
            for (int q = 0; q < kPairs; ++q) f[q] = gradient(Pairs<T>::get(x[u], q));
            out[u * 32 + lane] = S.ignored ? make_uint4(0, 0, 0, 0) : Pairs<T>::join(f);
        }
    if (lane < c.singles) dz[c.single(lane)] = from_f32<T>(S.ignored ? 0.f : gradient(both(extra)).x);
    __syncwarp();  // orders the stores above before those below
    if (!S.ignored) write_entries<T, kSquarings>(P, dz, gradient, S, p, zk, idx, lane, 32);
}

// kSquarings: T = 1, 2, 4 as 0, 1, 2, where exp(z) = exp(z/T)^T; any other T as -1.
// kHeld false: a row that shared memory does not hold is read from global memory both times, the second time from the L2 cache; and
// a gradient whose rows lie off the logits' 16-byte boundaries is stored by elements.
template <typename T, int kSquarings, int kThreads, bool kHeld>
__global__ void __launch_bounds__(kThreads + 32, Held<kThreads>::kPerSM)
distill_kernel(const __grid_constant__ DistillParams P, int rows, int mode, int* fault) {
    using H = Held<kThreads>;
    constexpr int N = 16 / sizeof(T), kPairs = Pairs<T>::kCount, U = H::kUnroll;
    extern __shared__ __align__(128) char smem[];  // a row's whole vectors, then two sets of the teacher's entries
    __shared__ uint64_t bars[2 * H::kMostChunks + 4];  // full and free of each chunk, described[2], used[2]
    __shared__ Slot slots[2];
    __shared__ float part[2][3][32];
    __shared__ int gave_up;
    const int V = (int)P.vocab, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row_bytes = kHeld ? V / N * 16 : 0, chunks = (V / N + H::kChunk - 1) / H::kChunk;
    char* entries = smem + row_bytes;
    const uint32_t full = smem_u32(bars), free_ = full + 8 * H::kMostChunks, described = free_ + 8 * H::kMostChunks, used = described + 16;
    const Waits W{&gave_up, fault};
    if (threadIdx.x == 0) {
        for (int i = 0; kHeld && i < chunks; ++i) bar_init(full + 8 * i, 1), bar_init(free_ + 8 * i, H::kWarps);
        for (int i = 0; i < 2; ++i) bar_init(described + 8 * i, 1), bar_init(used + 8 * i, H::kWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        gave_up = 0;
    }
    __syncthreads();
    const bool want_stats = mode != kBackward, want_gradient = mode != kForward;

    if (warp == H::kWarps) {
        int it = 0;
        const auto copy = [&](int64_t row, int n) {  // the n-th row of this CTA
            const T* z = reinterpret_cast<const T*>(P.z) + row * P.z_stride;
            const Cut<T> c(z, V);
            for (int i = 0; kHeld && i < chunks; ++i) {
                if (n) W.wait_warp(free_ + 8 * i, (n - 1) & 1);
                const int bytes = min(H::kChunk, c.vectors - i * H::kChunk) * 16;
                if (lane == 0) {
                    if (gave_up || bytes <= 0) bar_arrive(full + 8 * i);
                    else {
                        bar_expect(full + 8 * i, bytes);
                        bulk_load(smem_u32(smem) + i * H::kChunk * 16, reinterpret_cast<const char*>(z + c.head) + i * H::kChunk * 16, bytes, full + 8 * i);
                    }
                }
            }
        };
        copy(blockIdx.x, 0);
        for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, ++it) {
            const int s = it & 1;
            if (it >= 2) W.wait_warp(used + 8 * s, (it / 2 - 1) & 1);
            float* p = reinterpret_cast<float*>(entries) + s * 3 * P.k;
            describe_row<T>(P, reinterpret_cast<const T*>(P.z) + row * P.z_stride, row, mode == kBackward, p, p + P.k, reinterpret_cast<int*>(p + 2 * P.k), slots[s]);
            __syncwarp();
            if (lane == 0) bar_arrive(described + 8 * s);
            if (row + gridDim.x < rows) copy(row + gridDim.x, it + 1);
        }
        if (kHeld && gave_up && lane == 0)  // copies in flight still write to shared memory
            for (int i = 0; i < chunks; ++i) W.drain(full + 8 * i, (it - 1) & 1);
        return;
    }

    const float c1 = kLog2e, cT = kLog2e / P.temperature;
    const Exponentials<kSquarings> exponentials(P.temperature);
    int it = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, ++it) {
        const T* z = reinterpret_cast<const T*>(P.z) + row * P.z_stride;
        const Cut<T> c(z, V);
        const int s = it & 1;
        const uint4* held = kHeld ? reinterpret_cast<const uint4*>(smem) : reinterpret_cast<const uint4*>(z + c.head);
        float extra = -INFINITY;
        if (threadIdx.x < c.singles) extra = to_f32<T>(z[c.single(threadIdx.x)]);

        float lse1, lseT;
        if (want_stats) {
            // A thread's sums are relative to the largest it has seen so far, which after the first few vectors hardly moves.
            // The difference comes before the factor: the type's lowest value times log2(e) would be -infinity.
            float m = extra;
            float2 sT = make_float2(0.f, 0.f), s1 = sT, minus = make_float2(m == -INFINITY ? 0.f : -m, m == -INFINITY ? 0.f : -m);
            const auto add = [&](float2 f) {
                const float2 d = add2(f, minus);
                float2 eT, e1;
                exponentials(d, d, eT, e1);
                sT = add2(sT, eT);
                if (kSquarings != 0) s1 = add2(s1, e1);
            };
            add(make_float2(extra, -INFINITY));
            for (int k = 0; k < chunks; ++k) {
                if (kHeld) W.wait_warp(full + 8 * k, it & 1);
                uint4 x[U];
                uint32_t tops[U];
                const uint4* from = held + k * H::kChunk + threadIdx.x;
                if ((k + 1) * H::kChunk <= c.vectors) {
#pragma unroll
                    for (int u = 0; u < U; ++u) x[u] = from[u * kThreads];
                } else {
                    const uint32_t low = low_word<T>();
#pragma unroll
                    for (int u = 0; u < U; ++u) x[u] = k * H::kChunk + u * kThreads + threadIdx.x < c.vectors ? from[u * kThreads] : make_uint4(low, low, low, low);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) tops[u] = max_words<T>(max_words<T>(x[u].x, x[u].y), max_words<T>(x[u].z, x[u].w));
#pragma unroll
                for (int u = 1; u < U; ++u) tops[0] = max_words<T>(tops[0], tops[u]);
                const float top = max_in_word<T>(tops[0]);
                if (top > m) {
                    const float fT = m == -INFINITY ? 0.f : fast_exp2((m - top) * cT), f1 = m == -INFINITY ? 0.f : fast_exp2((m - top) * c1);
                    sT = mul2(sT, make_float2(fT, fT)), s1 = mul2(s1, make_float2(f1, f1));  // s1 stays 0 where T = 1
                    m = top, minus = make_float2(-m, -m);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int q = 0; q < kPairs; ++q) add(Pairs<T>::get(x[u], q));
                if (kHeld && !want_gradient) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(free_ + 8 * k);
                }
            }
            if (kSquarings == 0) s1 = sT;
            float M = warp_max(m);
            const float d = m == -INFINITY ? 0.f : m - M;  // who has nothing has sums of 0, or a NaN
            float S1 = warp_sum((s1.x + s1.y) * fast_exp2(d * c1)), ST = warp_sum((sT.x + sT.y) * fast_exp2(d * cT));
            {
                if (lane == 0) part[s][0][warp] = M, part[s][1][warp] = S1, part[s][2][warp] = ST;
                asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
                const float wm = lane < H::kWarps ? part[s][0][lane] : -INFINITY;
                M = warp_max(wm);
                const float e = wm == -INFINITY ? 0.f : wm - M;
                S1 = warp_sum(lane < H::kWarps ? part[s][1][lane] * fast_exp2(e * c1) : 0.f);
                ST = warp_sum(lane < H::kWarps ? part[s][2][lane] * fast_exp2(e * cT) : 0.f);
            }
            lse1 = M + log2f(S1) * kLn2;
            lseT = M / P.temperature + log2f(ST) * kLn2;
        }
        W.wait_warp(described + 8 * s, (it / 2) & 1);
        const Slot S = slots[s];
        if (!want_stats) lse1 = S.lse1, lseT = S.lseT;
        else if (threadIdx.x == 0) write_loss(P, row, S, lse1, lseT);
        if (want_gradient) {
            // An ignored row's gradient is 0 whatever it holds.
            const Gradient<kSquarings> gradient(exponentials, P, S, lse1, lseT);
            T* dz = reinterpret_cast<T*>(P.dz) + row * P.dz_stride;
            uint4* out = reinterpret_cast<uint4*>(dz + c.head);
            for (int k = 0; k < chunks; ++k) {
                if (kHeld && !want_stats) W.wait_warp(full + 8 * k, it & 1);
                uint4 x[U];
                const uint4* from = held + k * H::kChunk + threadIdx.x;
                uint4* to = out + k * H::kChunk + threadIdx.x;
                const bool whole = (k + 1) * H::kChunk <= c.vectors;
                const auto inside = [&](int u) { return whole || k * H::kChunk + u * kThreads + threadIdx.x < c.vectors; };
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (inside(u)) x[u] = from[u * kThreads];
                if (kHeld) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(free_ + 8 * k);
                }
                const auto store = [&](int u, uint4 y) {
                    if (kHeld || ((reinterpret_cast<uintptr_t>(to) & 15) == 0)) {
                        __stcs(to + u * kThreads, y);
                    } else {
                        const T* e = reinterpret_cast<const T*>(&y);
#pragma unroll
                        for (int i = 0; i < N; ++i) reinterpret_cast<T*>(to + u * kThreads)[i] = e[i];
                    }
                };
                if (S.ignored) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (inside(u)) store(u, make_uint4(0, 0, 0, 0));
                    continue;
                }
                const auto form = [&](int u) {
                    float2 f[kPairs];
#pragma unroll
                    for (int q = 0; q < kPairs; ++q) f[q] = gradient(Pairs<T>::get(x[u], q));
                    store(u, Pairs<T>::join(f));
                };
                if (whole) {
#pragma unroll
                    for (int u = 0; u < U; ++u) form(u);
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (inside(u)) form(u);
                }
            }
            if (threadIdx.x < c.singles) dz[c.single(threadIdx.x)] = from_f32<T>(S.ignored ? 0.f : gradient(make_float2(extra, extra)).x);
            // The row's own entries lie in what other threads have written.
            asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
            if (!S.ignored) {
                const float* p = reinterpret_cast<const float*>(entries) + s * 3 * P.k;
                write_entries<T, kSquarings>(P, dz, gradient, S, p, p + P.k, reinterpret_cast<const int*>(p + 2 * P.k), threadIdx.x, kThreads);
            }
        }
        __syncwarp();
        if (lane == 0) bar_arrive(used + 8 * s);
    }
}

template <typename T>
int held_bytes(const DistillParams& P) { return (int)(P.vocab * sizeof(T) / 16 * 16 + P.k * 24); }
constexpr int kMostHeld = 225 * 1024;  // of 227 KB to a CTA, beside what the kernel declares itself

template <typename T, int kSquarings, int kThreads, bool kHeld = true>
int launch_rows(const DistillParams& P, int64_t rows, int mode, int sms, int* fault, cudaStream_t st) {
    using H = Held<kThreads>;
    auto* kernel = distill_kernel<T, kSquarings, kThreads, kHeld>;
    const int bytes = kHeld ? held_bytes<T>(P) : (int)P.k * 24;
    static Allowed allowed;
    if (int rc = allow_smem(kernel, bytes, allowed)) return rc;
    constexpr int kBeside = 3 * 1024;  // static shared memory of a CTA, and the 1 KB that the hardware keeps
    const int fit = kSharedPerSM / (bytes + kBeside), per_sm = fit < 1 ? 1 : fit < H::kPerSM ? fit : H::kPerSM;
    const int64_t most = (int64_t)sms * per_sm;
    kernel<<<(unsigned)(rows < most ? rows : most), kThreads + 32, bytes, st>>>(P, (int)rows, mode, fault);
    return cuda_status(cudaGetLastError(), "distill launch");
}

// Small CTAs (or single warps) for short rows: many of them hide each other's latencies, and a row's fixed cost (a reduction, two
// barriers) falls on fewer threads.  From half of an SM's shared memory on there is one CTA to an SM, which then needs all the threads.
template <typename T, int kSquarings>
int by_length(const DistillParams& P, int64_t rows, int mode, int sms, int* fault, cudaStream_t st) {
    const int64_t bytes = P.vocab * (int64_t)sizeof(T);
    const bool lies_like = mode == kForward || ((((uintptr_t)P.z ^ (uintptr_t)P.dz) & 15) == 0 && (rows == 1 || (P.z_stride - P.dz_stride) * (int64_t)sizeof(T) % 16 == 0));
    if (!lies_like || bytes > kMostHeld || held_bytes<T>(P) > kMostHeld) return launch_rows<T, kSquarings, 512, false>(P, rows, mode, sms, fault, st);
    if (bytes <= kShort) {
        static Allowed allowed;
        const int shared = kShortWarps * (int)P.k * 12;
        if (int rc = allow_smem(distill_short_kernel<T, kSquarings>, shared, allowed)) return rc;
        distill_short_kernel<T, kSquarings><<<(unsigned)((rows + kShortWarps - 1) / kShortWarps), 32 * kShortWarps, shared, st>>>(P, (int)rows, mode);
        return cuda_status(cudaGetLastError(), "distill launch");
    }
    // From 32 to 48 KB the smaller CTA is 4 to 8% faster over 4000 rows, the larger one 10% over 1000, where each CTA has two or three.
    if (bytes <= 32768 || (bytes <= 49152 && rows > 12 * sms)) return launch_rows<T, kSquarings, 128>(P, rows, mode, sms, fault, st);
    if (bytes <= 110 * 1024) return launch_rows<T, kSquarings, 256>(P, rows, mode, sms, fault, st);
    return launch_rows<T, kSquarings, 512>(P, rows, mode, sms, fault, st);
}

template <typename T>
int by_temperature(const DistillParams& P, int64_t rows, int mode, int32_t device, cudaStream_t st) {
    int* fault = nullptr;
    if (int rc = fault_mark(&fault)) return rc;
    const int sms = sm_count(device);
    if (P.temperature == 1.f) return by_length<T, 0>(P, rows, mode, sms, fault, st);
    if (P.temperature == 2.f) return by_length<T, 1>(P, rows, mode, sms, fault, st);
    if (P.temperature == 4.f) return by_length<T, 2>(P, rows, mode, sms, fault, st);
    return by_length<T, -1>(P, rows, mode, sms, fault, st);
}

template <Mode kMode>
int distill(const halos_distill_args* a) {
    if (!a || a->struct_size != sizeof(halos_distill_args)) return fail(HALOS_ERR_INVALID_ARG, "distill: args missing or of another size");
    if (!is_type(a->dtype) || (a->k && !is_type(a->teacher_dtype))) return fail(HALOS_ERR_INVALID_ARG, "distill: dtype");
    if (a->rows < 0 || a->vocab < 0) return fail(HALOS_ERR_INVALID_ARG, "distill: rows or vocab");
    if (!(a->temperature > 0.f) || !(a->temperature < INFINITY)) return fail(HALOS_ERR_INVALID_ARG, "distill: temperature must be positive");
    if (!(a->mix >= 0.f && a->mix <= 1.f)) return fail(HALOS_ERR_INVALID_ARG, "distill: mix must lie in [0, 1]");
    if (a->k > kMaxTeacher) return fail(HALOS_ERR_UNSUPPORTED, "distill: over 1024 teacher entries");
    if (a->rows > 0x7fffffffll || a->vocab > 0x7fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "distill: rows or vocab over 2^31 - 1");
    if (a->rows == 0) return HALOS_OK;
    if (a->vocab == 0) return fail(HALOS_ERR_INVALID_ARG, "distill: empty vocabulary");
    const uint32_t size = a->dtype == HALOS_F32 ? 4 : 2;
    if (!a->logits || (a->k && (!a->teacher_index || !a->teacher_logits))) return fail(HALOS_ERR_INVALID_ARG, "distill: null pointer");
    if (kMode != kBackward && !a->loss) return fail(HALOS_ERR_INVALID_ARG, "distill: null pointer");
    if (kMode != kForward && (!a->dloss || !a->dlogits)) return fail(HALOS_ERR_INVALID_ARG, "distill: null pointer");
    if (kMode != kBoth && !a->stats) return fail(HALOS_ERR_INVALID_ARG, "distill: null pointer");
    if ((uintptr_t)a->logits % size || (kMode != kForward && (uintptr_t)a->dlogits % size))
        return fail(HALOS_ERR_INVALID_ARG, "distill: tensor not aligned to its elements");
    if (kMode != kForward && a->rows > 1 && a->dlogits_stride < a->vocab) return fail(HALOS_ERR_INVALID_ARG, "distill: rows of dlogits overlap");
    if (kMode != kForward && a->rows > 1 && a->dlogits == a->logits && a->dlogits_stride != a->logits_stride)
        return fail(HALOS_ERR_INVALID_ARG, "distill: over the logits themselves dlogits must have their stride");
    if (int rc = enter(a->device)) return rc;
    DistillParams P{};
    P.z = (const char*)a->logits, P.dz = (char*)a->dlogits, P.labels = a->labels, P.index = a->teacher_index, P.t = (const char*)a->teacher_logits;
    P.loss = a->loss, P.stats = a->stats, P.dloss = a->dloss;
    P.z_stride = a->logits_stride, P.dz_stride = a->dlogits_stride, P.index_stride = a->teacher_index_stride, P.t_stride = a->teacher_logits_stride;
    P.vocab = a->vocab, P.ignore_index = a->ignore_index, P.k = a->k, P.labels_64 = a->labels_64, P.index_64 = a->index_64;
    P.teacher_dtype = a->teacher_dtype, P.temperature = a->temperature, P.mix = a->mix;
    cudaStream_t st = (cudaStream_t)a->stream;
    if (a->dtype == HALOS_F32) return by_temperature<float>(P, a->rows, kMode, a->device, st);
    if (a->dtype == HALOS_BF16) return by_temperature<__nv_bfloat16>(P, a->rows, kMode, a->device, st);
    return by_temperature<__half>(P, a->rows, kMode, a->device, st);
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_distill_fwd(const halos_distill_args* a) { return halos_step::distill<halos_step::kForward>(a); }
extern "C" int halos_distill_bwd(const halos_distill_args* a) { return halos_step::distill<halos_step::kBackward>(a); }
extern "C" int halos_distill_fwd_bwd(const halos_distill_args* a) { return halos_step::distill<halos_step::kBoth>(a); }
