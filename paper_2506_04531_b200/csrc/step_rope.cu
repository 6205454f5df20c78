// Rotary positions on queries and keys in one launch.
//
// Bound by memory: every element is read once and written once, 3 flops each.  What could cost more than that is the
// sine and cosine, so a block forms those of its tokens once, evenly over its threads, and keeps them in shared memory
// for all heads.
//
// Angles.  position * frequency in 32 bits is wrong by 2^-24 of the angle, 0.004 radians at position 65536.  A turn is
// therefore taken as 2^64: the frequency becomes a 64-bit fraction of a turn, the product with the position wraps
// by itself, and its top 32 bits are the angle.  The fraction is formed to its last bit or two, from a product of twice 64-bit floats' width, so that
// the angle is off by 2^-31 of a turn up to position 2^31, and by 2^-62 of a turn for each position beyond.
//
// Measured: 65536 tokens of 12 + 12 heads of 64, a quarter rotated, bf16, strided views of a projection: 70 us, 5.7 TB/s.  16411
// tokens of 16 + 4 heads of 128, all rotated, f16: 43 us, 3.9 TB/s; there sines and reading them back weigh a third.
#include "step_common.cuh"

namespace halos_step {
namespace {

constexpr int kThreads = 256;
// 1 / (2 pi) as the nearest 64-bit float and what that leaves out
constexpr double kTurnsPerRadian = 0.15915494309189535, kTurnsPerRadianRest = -9.839338337591243e-18;

struct RopeTensor {                  // q, then k
    const char* in;
    char* out;
    int64_t in_stride[3], out_stride[3];  // in elements
    uint32_t heads, head_groups;     // threads that share a token's column
    uint32_t tokens_per_block, blocks;
};
struct RopeParams {
    RopeTensor x[2];
    const double* freqs;
    const void* positions;
    int64_t position_stride[2], position_offset;
    uint32_t tokens, seq, head_dim, rot_dim;
    uint32_t rot_cols, cols;         // columns of two pieces per head: rotated ones first, then copied ones
    uint32_t positions_64, inverse;
    float magnitude;
};

// N neighbouring elements as they lie in memory, in one access and in whole registers.
template <int kBytes> struct Raw;
template <> struct Raw<16> { uint4 v; };
template <> struct Raw<8> { uint2 v; };
template <> struct Raw<4> { uint32_t v; };
template <> struct Raw<2> { uint16_t v; };
__device__ __forceinline__ void words_of(uint32_t (&w)[4], uint4 v) { w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w; }
__device__ __forceinline__ void words_of(uint32_t (&w)[2], uint2 v) { w[0] = v.x, w[1] = v.y; }
__device__ __forceinline__ void words_of(uint32_t (&w)[1], uint32_t v) { w[0] = v; }
__device__ __forceinline__ void words_of(uint32_t (&w)[1], uint16_t v) { w[0] = v; }
__device__ __forceinline__ void of_words(uint4& v, const uint32_t (&w)[4]) { v = make_uint4(w[0], w[1], w[2], w[3]); }
__device__ __forceinline__ void of_words(uint2& v, const uint32_t (&w)[2]) { v = make_uint2(w[0], w[1]); }
__device__ __forceinline__ void of_words(uint32_t& v, const uint32_t (&w)[1]) { v = w[0]; }
__device__ __forceinline__ void of_words(uint16_t& v, const uint32_t (&w)[1]) { v = (uint16_t)w[0]; }

template <typename T, int N>
__device__ __forceinline__ void widen(float (&f)[N], const Raw<N * sizeof(T)>& r) {
    uint32_t w[(N * sizeof(T) + 3) / 4];
    words_of(w, r.v);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = __uint_as_float(w[i]);
    } else if constexpr (N == 1) {
        f[0] = unpack2<T>(w[0]).x;
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 p = unpack2<T>(w[i]);
            f[2 * i] = p.x, f[2 * i + 1] = p.y;
        }
    }
}
template <typename T, int N>
__device__ __forceinline__ Raw<N * sizeof(T)> rounded(const float (&f)[N]) {
    uint32_t w[(N * sizeof(T) + 3) / 4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
    } else if constexpr (N == 1) {
        w[0] = pack2<T>(f[0], 0.f);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = pack2<T>(f[2 * i], f[2 * i + 1]);
    }
    Raw<N * sizeof(T)> r;
    of_words(r.v, w);
    return r;
}

// A column is two pieces of N neighbouring elements: (x0 of N pairs, x1 of the same pairs) in the half layout, 2N
// neighbours in the interleaved one.  The copied rest is cut in two halves of whole pieces, so that neighbouring threads
// take neighbouring pieces there too.  U heads are in flight at a time.
template <typename T, int N, bool kInterleaved, int U>
__global__ void __launch_bounds__(kThreads, 4) rope_kernel(const __grid_constant__ RopeParams P) {
    __shared__ uint64_t turn[128];                       // of each pair per position; a whole turn is 2^64
    __shared__ __align__(16) float2 cos_sin[kThreads * N];  // [token][pair]
    const RopeTensor& X = P.x[blockIdx.x >= P.x[0].blocks];
    const uint32_t token0 = (blockIdx.x >= P.x[0].blocks ? blockIdx.x - P.x[0].blocks : blockIdx.x) * X.tokens_per_block;
    const uint32_t pairs = P.rot_dim / 2;
    for (uint32_t p = threadIdx.x; p < pairs; p += kThreads) {
        const double f = P.freqs[p], product = f * kTurnsPerRadian;
        const double rest = fma(f, kTurnsPerRadian, -product) + f * kTurnsPerRadianRest;  // of the product's rounding and the constant's
        const uint64_t whole = (uint64_t)((product - floor(product)) * 18446744073709551616.0);  // saturates just below a whole turn
        turn[p] = whole + (uint64_t)llrint(rest * 18446744073709551616.0);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < X.tokens_per_block * pairs; i += kThreads) {
        const uint32_t sub = i / pairs, p = i - sub * pairs, token = token0 + sub;
        if (token >= P.tokens) break;
        const uint32_t b = token / P.seq, s = token - b * P.seq;
        int64_t t = P.position_offset + s;
        if (P.positions) {
            const int64_t at = b * P.position_stride[0] + s * P.position_stride[1];
            t = P.positions_64 ? static_cast<const int64_t*>(P.positions)[at] : (int64_t)static_cast<const int32_t*>(P.positions)[at];
        }
        const int32_t angle = (int32_t)(((uint64_t)t * turn[p]) >> 32);
        float sn, c;
        sincospif((float)angle * 4.656612873077393e-10f, &sn, &c);  // 2^-31 half turns
        cos_sin[i] = make_float2(c * P.magnitude, sn * (P.inverse ? -P.magnitude : P.magnitude));
    }
    __syncthreads();

    const uint32_t per_token = P.cols * X.head_groups, sub = threadIdx.x / per_token, token = token0 + sub;
    if (sub >= X.tokens_per_block || token >= P.tokens) return;
    const uint32_t r = threadIdx.x - sub * per_token, group = r / P.cols, col = r - group * P.cols;
    const uint32_t b = token / P.seq, s = token - b * P.seq;

    const bool rotated = col < P.rot_cols;
    uint32_t at0, at1;
    bool two = true;
    if (rotated) {
        at0 = kInterleaved ? col * 2 * N : col * N;
        at1 = kInterleaved ? at0 + N : at0 + pairs;
        if (kInterleaved) two = at1 < P.rot_dim;
    } else {
        at0 = P.rot_dim + (col - P.rot_cols) * N;
        at1 = at0 + (P.cols - P.rot_cols) * N;
        two = at1 < P.head_dim;
    }
    const float2* cs = cos_sin + sub * pairs + col * N;
    const int64_t in_step = X.in_stride[2] * X.head_groups, out_step = X.out_stride[2] * X.head_groups;
    const T* x = reinterpret_cast<const T*>(X.in) + b * X.in_stride[0] + s * X.in_stride[1] + group * X.in_stride[2] + at0;
    T* y = reinterpret_cast<T*>(X.out) + b * X.out_stride[0] + s * X.out_stride[1] + group * X.out_stride[2] + at0;
    const uint32_t apart = at1 - at0;
    using Piece = Raw<N * sizeof(T)>;
    for (uint32_t first = group; first < X.heads; first += U * X.head_groups, x += U * in_step, y += U * out_step) {
        Piece w0[U], w1[U];  // in flight as they lie in memory; widened one head at a time
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u * X.head_groups < X.heads) {
                w0[u] = *reinterpret_cast<const Piece*>(x + u * in_step);
                if (two) w1[u] = *reinterpret_cast<const Piece*>(x + u * in_step + apart);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (first + u * X.head_groups >= X.heads) break;
            if (rotated) {
                float x0[N], x1[N];
                widen<T, N>(x0, w0[u]);
                widen<T, N>(x1, w1[u]);  // of no meaning, and not stored, where there is no second piece
                if (!kInterleaved || N == 1) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float a = x0[i], d = x1[i];
                        x0[i] = fmaf(a, cs[i].x, -(d * cs[i].y));
                        x1[i] = fmaf(d, cs[i].x, a * cs[i].y);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; i += 2) {
                        const int j = i + 1 < N ? i + 1 : i;
                        const float a = x0[i], d = x0[j];
                        x0[i] = fmaf(a, cs[i / 2].x, -(d * cs[i / 2].y));
                        x0[j] = fmaf(d, cs[i / 2].x, a * cs[i / 2].y);
                        const float e = x1[i], g = x1[j];
                        const float2 v = two ? cs[N / 2 + i / 2] : make_float2(1.f, 0.f);
                        x1[i] = fmaf(e, v.x, -(g * v.y));
                        x1[j] = fmaf(g, v.x, e * v.y);
                    }
                }
                w0[u] = rounded<T, N>(x0);
                w1[u] = rounded<T, N>(x1);
            }
            *reinterpret_cast<Piece*>(y + u * out_step) = w0[u];
            if (two) *reinterpret_cast<Piece*>(y + u * out_step + apart) = w1[u];
        }
    }
}

template <typename T, int N, bool I>
int launch(const RopeParams& P, cudaStream_t st) {
    rope_kernel<T, N, I, (N * sizeof(T) >= 8 ? 4 : 8)><<<P.x[0].blocks + P.x[1].blocks, kThreads, 0, st>>>(P);
    return cuda_status(cudaGetLastError(), "rope launch");
}

template <typename T, bool I>
int pick(RopeParams& P, uint32_t n, cudaStream_t st) {
    if constexpr (sizeof(T) == 2) {
        if (n == 8) return launch<T, 8, I>(P, st);
    }
    if (n >= 4) return launch<T, 4, I>(P, st);
    if (n == 2) return launch<T, 2, I>(P, st);
    return launch<T, 1, I>(P, st);
}

template <typename T>
int by_layout(RopeParams& P, uint32_t n, uint32_t layout, cudaStream_t st) {
    return layout == HALOS_ROPE_INTERLEAVED ? pick<T, true>(P, n, st) : pick<T, false>(P, n, st);
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_rope(const halos_rope_args* a) {
    using namespace halos_step;
    if (!a || a->struct_size != sizeof(halos_rope_args)) return fail(HALOS_ERR_INVALID_ARG, "rope: args missing or of another size");
    if (!is_type(a->dtype)) return fail(HALOS_ERR_INVALID_ARG, "rope: dtype");
    if (a->layout > HALOS_ROPE_INTERLEAVED) return fail(HALOS_ERR_INVALID_ARG, "rope: layout");
    if (a->batch < 0 || a->seq < 0 || a->seq > 0x7fffffffll || a->batch > 0x7fffffffll) return fail(HALOS_ERR_INVALID_ARG, "rope: batch or seq");
    if (a->head_dim == 0 || a->rot_dim > a->head_dim || a->rot_dim % 2) return fail(HALOS_ERR_INVALID_ARG, "rope: rot_dim must be even and at most head_dim");
    if (a->head_dim > 256 || a->n_q > 65535 || a->n_k > 65535) return fail(HALOS_ERR_UNSUPPORTED, "rope: head_dim over 256 or too many heads");
    const int64_t tokens = a->batch * a->seq;
    const uint32_t heads = a->n_q + a->n_k;
    if (tokens == 0 || heads == 0) return HALOS_OK;
    if (tokens > 0x7fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "rope: over 2^31 - 1 tokens");
    if ((a->n_q && (!a->q_in || !a->q_out)) || (a->n_k && (!a->k_in || !a->k_out)) || (a->rot_dim && !a->freqs))
        return fail(HALOS_ERR_INVALID_ARG, "rope: null pointer");
    const int64_t q_size[3] = {a->batch, a->seq, a->n_q}, k_size[3] = {a->batch, a->seq, a->n_k};
    for (int i = 0; i < 3; ++i)
        if ((a->n_q && a->q_in == a->q_out && q_size[i] > 1 && a->q_in_stride[i] != a->q_out_stride[i]) ||
            (a->n_k && a->k_in == a->k_out && k_size[i] > 1 && a->k_in_stride[i] != a->k_out_stride[i]))
            return fail(HALOS_ERR_INVALID_ARG, "rope: in place the strides must be the same");
    const uint32_t size = a->dtype == HALOS_F32 ? 4 : 2;
    // Widest access (16 bytes) that divides the head, the pairs and every address.
    uint64_t all = a->head_dim | (a->layout == HALOS_ROPE_HALF ? a->rot_dim / 2 : a->rot_dim);
    uint64_t base = 0;
    for (int i = 0; i < 3; ++i) {
        if (a->n_q) all |= (uint64_t)a->q_in_stride[i] | (uint64_t)a->q_out_stride[i];
        if (a->n_k) all |= (uint64_t)a->k_in_stride[i] | (uint64_t)a->k_out_stride[i];
    }
    if (a->n_q) base |= (uintptr_t)a->q_in | (uintptr_t)a->q_out;
    if (a->n_k) base |= (uintptr_t)a->k_in | (uintptr_t)a->k_out;
    if (base % size) return fail(HALOS_ERR_INVALID_ARG, "rope: tensor not aligned to its elements");
    all = all * size | base;
    uint32_t n = 16 / size;
    while (n > 1 && all % (n * size)) n /= 2;
    if (int rc = enter(a->device)) return rc;

    RopeParams P{};
    P.x[0].in = (const char*)a->q_in, P.x[0].out = (char*)a->q_out, P.x[1].in = (const char*)a->k_in, P.x[1].out = (char*)a->k_out;
    P.freqs = a->freqs, P.positions = a->positions;
    for (int i = 0; i < 3; ++i) {
        P.x[0].in_stride[i] = a->q_in_stride[i], P.x[0].out_stride[i] = a->q_out_stride[i];
        P.x[1].in_stride[i] = a->k_in_stride[i], P.x[1].out_stride[i] = a->k_out_stride[i];
    }
    P.position_stride[0] = a->position_stride[0], P.position_stride[1] = a->position_stride[1];
    P.position_offset = a->position_offset;
    P.tokens = (uint32_t)tokens, P.seq = (uint32_t)a->seq, P.head_dim = a->head_dim, P.rot_dim = a->rot_dim;
    P.positions_64 = a->positions_64, P.inverse = a->inverse, P.magnitude = a->magnitude;
    P.rot_cols = (a->rot_dim + 2 * n - 1) / (2 * n);
    const bool in_place = (!a->n_q || a->q_in == a->q_out) && (!a->n_k || a->k_in == a->k_out);
    P.cols = P.rot_cols + (in_place ? 0 : (a->head_dim - a->rot_dim + 2 * n - 1) / (2 * n));
    if (P.cols == 0) return HALOS_OK;
    // As few threads per token as still fill the GPU: their fixed cost then falls on more heads.
    const int64_t want = ((int64_t)sm_count(a->device) * 1024 + tokens * P.cols - 1) / (tokens * P.cols);
    for (int i = 0; i < 2; ++i) {
        RopeTensor& X = P.x[i];
        X.heads = i ? a->n_k : a->n_q;
        if (!X.heads) continue;
        const uint32_t most = kThreads / P.cols < X.heads ? kThreads / P.cols : X.heads;
        uint32_t least = (X.heads + 7) / 8;
        if (least > most) least = most;
        X.head_groups = want > most ? most : want < least ? least : (uint32_t)want;
        X.tokens_per_block = kThreads / (P.cols * X.head_groups);
        const int64_t blocks = (tokens + X.tokens_per_block - 1) / X.tokens_per_block;
        if (blocks > 0x3fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "rope: too many tokens");
        X.blocks = (uint32_t)blocks;
    }
    cudaStream_t st = (cudaStream_t)a->stream;
    if (a->dtype == HALOS_F32) return by_layout<float>(P, n, a->layout, st);
    if (a->dtype == HALOS_BF16) return by_layout<__nv_bfloat16>(P, n, a->layout, st);
    return by_layout<__half>(P, n, a->layout, st);
}
