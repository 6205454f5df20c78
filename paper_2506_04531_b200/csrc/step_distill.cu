// Distillation from a teacher's top logits mixed with cross-entropy: loss, gradient, or both, one CTA per row.
//
// Bound by memory: a forward pass reads the logits once, a backward pass reads and writes them once, and the two together
// read and write them once.  The second constraint is the exponential (16 per clock and SM): with a temperature a
// logit needs exp(z) and exp(z/T), in the statistics and again in the gradient.  Where T is 1, 2 or 4 the
// first is the second to the power T, which costs multiplications instead (kSquarings).
//
// Statistics are kept online: a thread holds the largest logit it has seen and the two sums relative to it, and
// rescales them when a larger one comes up, which after the first few vectors is rare.
#include "step_common.cuh"

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

// What warp 0 finds out about a row's teacher and label, for everybody.
struct RowShared {
    float p[kMaxTeacher], z[kMaxTeacher];   // teacher's probabilities and the row's logits at its entries
    int32_t idx[kMaxTeacher];
    float warp_m[32], warp_s1[32], warp_sT[32];
    float plogp, label_z, pz;               // sum p log p; z at the label; sum p z
    int64_t label;
    int ignored, bad, any;                  // label is ignore_index; something points outside; the teacher sent something
};

template <typename T>
__device__ void read_teacher(const DistillParams& P, const T* z, int64_t row, RowShared& S) {
    const int lane = threadIdx.x & 31;
    int64_t label = 0;
    int ignored = 0, bad = 0;
    if (P.labels) {
        label = P.labels_64 ? static_cast<const int64_t*>(P.labels)[row] : (int64_t)static_cast<const int32_t*>(P.labels)[row];
        ignored = label == P.ignore_index;
        bad = !ignored && (label < 0 || label >= P.vocab);
    }
    const float invT = 1.f / P.temperature;
    float top = -INFINITY;
    for (uint32_t i = lane; i < P.k; i += 32) {
        const int64_t at = row * P.index_stride + i;
        const int64_t j = P.index_64 ? static_cast<const int64_t*>(P.index)[at] : (int64_t)static_cast<const int32_t*>(P.index)[at];
        const bool in = j >= 0 && j < P.vocab;
        if (!in && j != -1) bad = 1;
        S.idx[i] = in ? (int32_t)j : -1;
        S.z[i] = in && !ignored ? to_f32<T>(z[j]) : 0.f;
        const float t = in ? teacher_at(P, row * P.t_stride + i) * invT : -INFINITY;
        S.p[i] = t;
        top = fmaxf(top, t);
    }
    top = warp_max(top);
    float sum = 0.f;
    for (uint32_t i = lane; i < P.k; i += 32)
        if (S.p[i] != -INFINITY) sum += exp2f((S.p[i] - top) * kLog2e);
    sum = warp_sum(sum);
    const float log_sum = logf(sum);
    float plogp = 0.f, pz = 0.f;
    for (uint32_t i = lane; i < P.k; i += 32) {
        const float t = S.p[i];
        float p = 0.f;
        if (t != -INFINITY) {
            const float logp = t - top - log_sum;
            p = expf(logp);
            if (p > 0.f) plogp += p * logp, pz += p * S.z[i];  // 0 log 0 = 0, whatever the logit there
        }
        S.p[i] = p;
    }
    plogp = warp_sum(plogp);
    pz = warp_sum(pz);
    bad = __any_sync(~0u, bad);
    if (lane == 0) {
        S.plogp = plogp;
        S.pz = pz;
        S.any = sum > 0.f;
        S.label = label;
        S.ignored = ignored;
        S.bad = bad;
        S.label_z = P.labels && !ignored && !bad ? to_f32<T>(z[label]) : 0.f;
    }
}

// x^T for T = 2^n by n squarings
template <int n> __device__ __forceinline__ float squared(float x) {
#pragma unroll
    for (int i = 0; i < n; ++i) x *= x;
    return x;
}

// kSquarings: T = 1, 2, 4 as 0, 1, 2; any other T as -1.
template <int kSquarings>
struct Online {
    float m = -INFINITY, s1 = 0.f, sT = 0.f;
    __device__ __forceinline__ void rescale(float to, float c1, float cT) {
        const float d = m - to;
        const float fT = m == -INFINITY ? 0.f : exp2f(d * cT);
        s1 *= kSquarings >= 0 ? squared<kSquarings < 0 ? 0 : kSquarings>(fT) : (m == -INFINITY ? 0.f : exp2f(d * c1));
        sT *= fT;
        m = to;
    }
    // The difference comes before the factor: a logit of the type's lowest value times log2(e) would be -infinity, and
    // -infinity minus itself no number.
    __device__ __forceinline__ void add(float z, float c1, float cT) {
        const float d = z - m;
        const float eT = exp2f(d * cT);
        sT += eT;
        s1 += kSquarings >= 0 ? squared<kSquarings < 0 ? 0 : kSquarings>(eT) : exp2f(d * c1);
    }
    template <int N> __device__ __forceinline__ void add_vector(const float (&z)[N], float c1, float cT) {
        float top = z[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, z[i]);
        if (top > m) rescale(top, c1, cT);
        if (m == -INFINITY) {  // nothing but -infinity so far (or a NaN, which has to come through)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (z[i] != z[i]) s1 = sT = z[i];
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) add(z[i], c1, cT);
    }
};

template <typename T, Mode kMode, int kSquarings, int kThreads>
__global__ void __launch_bounds__(kThreads) distill_kernel(const __grid_constant__ DistillParams P) {
    constexpr int N = 16 / sizeof(T), U = 4;
    __shared__ RowShared S;
    const int64_t row = blockIdx.x;
    const T* z = reinterpret_cast<const T*>(P.z) + row * P.z_stride;
    T* dz = reinterpret_cast<T*>(P.dz) + row * P.dz_stride;
    const int64_t V = P.vocab;
    const float c1 = kLog2e, cT = kLog2e / P.temperature;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    // [0, head) and [head + N vectors, V) singly, the rest in 16-byte vectors
    int64_t head = (int64_t)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(T);
    const bool wide = kMode == kForward || ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
    if (!wide || head > V) head = V;
    const int64_t vectors = (V - head) / N, tail = head + vectors * N;

    if (warp == 0) read_teacher<T>(P, z, row, S);

    float lse1, lseT;
    if (kMode == kBackward) {
        lse1 = P.stats[2 * row];
        lseT = P.stats[2 * row + 1];
        __syncthreads();
    } else {
        Online<kSquarings> acc;
        for (int64_t v0 = threadIdx.x; v0 < vectors; v0 += U * kThreads) {
            Vec<T, N> w[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v0 + u * kThreads < vectors) w[u] = *reinterpret_cast<const Vec<T, N>*>(z + head + (v0 + u * kThreads) * N);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v0 + u * kThreads < vectors) {
                    float f[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) f[i] = to_f32<T>(w[u].v[i]);
                    acc.template add_vector<N>(f, c1, cT);
                }
        }
        for (int64_t j = threadIdx.x; j < head + (V - tail); j += kThreads) {
            float f[1] = {to_f32<T>(z[j < head ? j : j - head + tail])};
            acc.template add_vector<1>(f, c1, cT);
        }
        const float wm = warp_max(acc.m);
        acc.rescale(wm, c1, cT);
        const float w1 = warp_sum(acc.s1), wT = warp_sum(acc.sT);
        if (lane == 0) S.warp_m[warp] = wm, S.warp_s1[warp] = w1, S.warp_sT[warp] = wT;
        __syncthreads();
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, S.warp_m[i]);
        float s1 = 0.f, sT = 0.f;
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) {
            const float d = S.warp_m[i] - m;
            const bool none = S.warp_m[i] == -INFINITY;
            s1 += none ? S.warp_s1[i] : S.warp_s1[i] * exp2f(d * c1);
            sT += none ? S.warp_sT[i] : S.warp_sT[i] * exp2f(d * cT);
        }
        lse1 = m + log2f(s1) * kLn2;
        lseT = m / P.temperature + log2f(sT) * kLn2;
        if (threadIdx.x == 0) {
            if (P.stats) P.stats[2 * row] = lse1, P.stats[2 * row + 1] = lseT;
            float loss = 0.f;
            if (!S.ignored) {
                if (P.labels) loss += (1.f - P.mix) * (lse1 - S.label_z);
                if (S.any) loss += P.mix * P.temperature * P.temperature * (S.plogp - S.pz / P.temperature + lseT);
                if (S.bad) loss = NAN;
            }
            P.loss[row] = loss;
        }
    }
    if (kMode == kForward) return;

    // a q1 + b qT, then the rows' own entries
    const bool ignored = S.ignored;
    const float g = S.bad ? NAN : P.dloss[row];
    const float a = P.labels ? g * (1.f - P.mix) : 0.f, b = S.any ? g * P.mix * P.temperature : 0.f;
    // Where T = 2^n, q1 = qT^T exp(T lseT - lse1).
    const float ratio = kSquarings > 0 ? exp2f((P.temperature * lseT - lse1) * kLog2e) : 1.f;
    const float LT = P.temperature * lseT, aR = a * ratio;
    const auto grad = [&](float x) -> float {
        if (kSquarings == 0) return (a + b) * exp2f((x - lse1) * c1);
        const float qT = exp2f((x - LT) * cT);
        if (kSquarings > 0) return fmaf(aR, squared<kSquarings < 0 ? 0 : kSquarings>(qT), b * qT);
        return fmaf(a, exp2f((x - lse1) * c1), b * qT);
    };
    if (ignored) {
        for (int64_t v = threadIdx.x; v < vectors; v += kThreads) {
            Vec<T, N> w;
#pragma unroll
            for (int i = 0; i < N; ++i) w.v[i] = from_f32<T>(0.f);
            *reinterpret_cast<Vec<T, N>*>(dz + head + v * N) = w;
        }
        for (int64_t j = threadIdx.x; j < head + (V - tail); j += kThreads) dz[j < head ? j : j - head + tail] = from_f32<T>(0.f);
        return;
    }
    for (int64_t v0 = threadIdx.x; v0 < vectors; v0 += U * kThreads) {
        Vec<T, N> w[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * kThreads < vectors) w[u] = *reinterpret_cast<const Vec<T, N>*>(z + head + (v0 + u * kThreads) * N);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (v0 + u * kThreads < vectors) {
#pragma unroll
                for (int i = 0; i < N; ++i) w[u].v[i] = from_f32<T>(grad(to_f32<T>(w[u].v[i])));
                *reinterpret_cast<Vec<T, N>*>(dz + head + (v0 + u * kThreads) * N) = w[u];
            }
    }
    for (int64_t j = threadIdx.x; j < head + (V - tail); j += kThreads) {
        const int64_t at = j < head ? j : j - head + tail;
        dz[at] = from_f32<T>(grad(to_f32<T>(z[at])));
    }
    __syncthreads();  // the entries below were written above by other threads of this CTA
    // Each entry is formed once more, whole, from the logit read at the start (dz may lie on z) and rounded once.
    for (uint32_t i = threadIdx.x; i < P.k; i += kThreads) {
        const int32_t j = S.idx[i];
        if (j < 0) continue;
        float p = 0.f;
        for (uint32_t o = 0; o < P.k; ++o) p += S.idx[o] == j ? S.p[o] : 0.f;
        dz[j] = from_f32<T>(grad(S.z[i]) - b * p - (P.labels && j == S.label ? a : 0.f));
    }
    if (warp == 0 && P.labels && !S.bad) {
        int there = 0;
        for (uint32_t i = lane; i < P.k; i += 32) there |= S.idx[i] == S.label;
        if (!__any_sync(~0u, there) && lane == 0) dz[S.label] = from_f32<T>(grad(S.label_z) - a);
    }
}

template <typename T, Mode kMode, int kSquarings>
int launch(const DistillParams& P, int64_t rows, cudaStream_t st) {
    if (P.vocab <= 4096) distill_kernel<T, kMode, kSquarings, 128><<<(unsigned)rows, 128, 0, st>>>(P);
    else distill_kernel<T, kMode, kSquarings, 512><<<(unsigned)rows, 512, 0, st>>>(P);
    return cuda_status(cudaGetLastError(), "distill launch");
}

template <typename T, Mode kMode>
int by_temperature(const DistillParams& P, int64_t rows, cudaStream_t st) {
    if (P.temperature == 1.f) return launch<T, kMode, 0>(P, rows, st);
    if (P.temperature == 2.f) return launch<T, kMode, 1>(P, rows, st);
    if (P.temperature == 4.f) return launch<T, kMode, 2>(P, rows, st);
    return launch<T, kMode, -1>(P, rows, st);
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
    if (int rc = enter(a->device)) return rc;
    DistillParams P{};
    P.z = (const char*)a->logits, P.dz = (char*)a->dlogits, P.labels = a->labels, P.index = a->teacher_index, P.t = (const char*)a->teacher_logits;
    P.loss = a->loss, P.stats = a->stats, P.dloss = a->dloss;
    P.z_stride = a->logits_stride, P.dz_stride = a->dlogits_stride, P.index_stride = a->teacher_index_stride, P.t_stride = a->teacher_logits_stride;
    P.vocab = a->vocab, P.ignore_index = a->ignore_index, P.k = a->k, P.labels_64 = a->labels_64, P.index_64 = a->index_64;
    P.teacher_dtype = a->teacher_dtype, P.temperature = a->temperature, P.mix = a->mix;
    cudaStream_t st = (cudaStream_t)a->stream;
    if (a->dtype == HALOS_F32) return by_temperature<float, kMode>(P, a->rows, st);
    if (a->dtype == HALOS_BF16) return by_temperature<__nv_bfloat16, kMode>(P, a->rows, st);
    return by_temperature<__half, kMode>(P, a->rows, st);
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_distill_fwd(const halos_distill_args* a) { return halos_step::distill<halos_step::kForward>(a); }
extern "C" int halos_distill_bwd(const halos_distill_args* a) { return halos_step::distill<halos_step::kBackward>(a); }
extern "C" int halos_distill_fwd_bwd(const halos_distill_args* a) { return halos_step::distill<halos_step::kBoth>(a); }
