// Rotary positions on queries and keys in one launch.
//
// Bound by memory: every element is read once and written once, 3 flops each.  What could cost more than that is the
// sine and cosine, so a block forms those of its tokens once, evenly over its threads, and keeps them in shared memory
// for all heads.
//
// Angles.  position * frequency in 32 bits is wrong by 2^-24 of the angle, 0.004 radians at position 65536.  A turn is
// therefore taken as 2^64: the frequency becomes a 64-bit fraction of a turn, the product with the position wraps
// by itself, and its top 32 bits are the angle, off by 2^-32 of a turn, at any position.
#include "step_common.cuh"

namespace halos_step {
namespace {

constexpr int kThreads = 256;
constexpr double kTurnsPerRadian = 0.15915494309189533577;  // 1 / (2 pi)

struct RopeParams {
    const char *q_in, *k_in;
    char *q_out, *k_out;
    const double* freqs;
    const void* positions;
    int64_t q_in_stride[3], k_in_stride[3], q_out_stride[3], k_out_stride[3];  // in elements
    int64_t position_stride[2], position_offset, tokens;
    uint32_t seq, n_q, heads, head_dim, rot_dim;
    uint32_t rot_cols, cols;         // columns of two pieces per head: rotated ones first, then copied ones
    uint32_t head_groups;            // threads that share a token's column
    uint32_t tokens_per_block;
    uint32_t positions_64, inverse;
    float magnitude;
};

template <typename T, int N>
__device__ __forceinline__ void load_piece(float (&f)[N], const T* p) {
    const Vec<T, N> w = *reinterpret_cast<const Vec<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f32<T>(w.v[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_piece(T* p, const float (&f)[N]) {
    Vec<T, N> w;
#pragma unroll
    for (int i = 0; i < N; ++i) w.v[i] = from_f32<T>(f[i]);
    *reinterpret_cast<Vec<T, N>*>(p) = w;
}

// A column is two pieces of N neighbouring elements: (x0 of N pairs, x1 of the same pairs) in the half layout, 2N
// neighbours in the interleaved one.  The copied rest is cut in two halves of whole pieces, so that neighbouring threads
// take neighbouring pieces there too.  U heads are in flight at a time.
template <typename T, int N, bool kInterleaved, int U>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeParams P) {
    __shared__ uint64_t turn[128];              // of each pair per position; a whole turn is 2^64
    __shared__ float2 cos_sin[kThreads * N];    // [token][pair]
    const int64_t token0 = (int64_t)blockIdx.x * P.tokens_per_block;
    const uint32_t pairs = P.rot_dim / 2;
    for (uint32_t p = threadIdx.x; p < pairs; p += kThreads) {
        double turns = P.freqs[p] * kTurnsPerRadian;
        turns -= floor(turns);
        turn[p] = (uint64_t)(turns * 18446744073709551616.0);  // saturates just below a whole turn
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < P.tokens_per_block * pairs; i += kThreads) {
        const uint32_t sub = i / pairs, p = i - sub * pairs;
        const int64_t token = token0 + sub;
        if (token >= P.tokens) break;
        const int64_t b = token / P.seq, s = token - b * P.seq;
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

    const uint32_t per_token = P.cols * P.head_groups;
    const uint32_t sub = threadIdx.x / per_token;
    const int64_t token = token0 + sub;
    if (sub >= P.tokens_per_block || token >= P.tokens) return;
    const uint32_t r = threadIdx.x - sub * per_token;
    const uint32_t group = r / P.cols, col = r - group * P.cols;
    const int64_t b = token / P.seq, s = token - b * P.seq;

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
    float c[N], sn[N];
    if (rotated) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t pair = col * N + i;
            const float2 v = pair < pairs ? cos_sin[sub * pairs + pair] : make_float2(1.f, 0.f);
            c[i] = v.x, sn[i] = v.y;
        }
    }
    const T* q = reinterpret_cast<const T*>(P.q_in) + b * P.q_in_stride[0] + s * P.q_in_stride[1];
    const T* k = reinterpret_cast<const T*>(P.k_in) + b * P.k_in_stride[0] + s * P.k_in_stride[1] - P.n_q * P.k_in_stride[2];
    T* qo = reinterpret_cast<T*>(P.q_out) + b * P.q_out_stride[0] + s * P.q_out_stride[1];
    T* ko = reinterpret_cast<T*>(P.k_out) + b * P.k_out_stride[0] + s * P.k_out_stride[1] - P.n_q * P.k_out_stride[2];
    for (uint32_t first = group; first < P.heads; first += U * P.head_groups) {
        float x0[U][N], x1[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t h = first + u * P.head_groups;
            if (h < P.heads) {
                const T* x = h < P.n_q ? q + h * P.q_in_stride[2] : k + h * P.k_in_stride[2];
                load_piece<T, N>(x0[u], x + at0);
                if (two) load_piece<T, N>(x1[u], x + at1);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t h = first + u * P.head_groups;
            if (h >= P.heads) continue;
            T* y = h < P.n_q ? qo + h * P.q_out_stride[2] : ko + h * P.k_out_stride[2];
            if (rotated) {
                if (!kInterleaved || N == 1) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float a = x0[u][i], d = x1[u][i];
                        x0[u][i] = fmaf(a, c[i], -(d * sn[i]));
                        x1[u][i] = fmaf(d, c[i], a * sn[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; i += 2) {
                        const int j = i + 1 < N ? i + 1 : i;
                        const float a = x0[u][i], d = x0[u][j];
                        x0[u][i] = fmaf(a, c[i / 2], -(d * sn[i / 2]));
                        x0[u][j] = fmaf(d, c[i / 2], a * sn[i / 2]);
                        if (two) {
                            const float e = x1[u][i], g = x1[u][j];
                            x1[u][i] = fmaf(e, c[N / 2 + i / 2], -(g * sn[N / 2 + i / 2]));
                            x1[u][j] = fmaf(g, c[N / 2 + i / 2], e * sn[N / 2 + i / 2]);
                        }
                    }
                }
            }
            store_piece<T, N>(y + at0, x0[u]);
            if (two) store_piece<T, N>(y + at1, x1[u]);
        }
    }
}

template <typename T, int N, bool I>
int launch(const RopeParams& P, cudaStream_t st) {
    const int64_t blocks = (P.tokens + P.tokens_per_block - 1) / P.tokens_per_block;
    if (blocks > 0x7fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "rope: too many tokens");
    rope_kernel<T, N, I, (N * sizeof(T) >= 8 ? 4 : 8)><<<(unsigned)blocks, kThreads, 0, st>>>(P);
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
    if ((a->n_q && (!a->q_in || !a->q_out)) || (a->n_k && (!a->k_in || !a->k_out)) || (a->rot_dim && !a->freqs))
        return fail(HALOS_ERR_INVALID_ARG, "rope: null pointer");
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
    P.q_in = (const char*)a->q_in, P.k_in = (const char*)a->k_in, P.q_out = (char*)a->q_out, P.k_out = (char*)a->k_out;
    P.freqs = a->freqs, P.positions = a->positions;
    for (int i = 0; i < 3; ++i)
        P.q_in_stride[i] = a->q_in_stride[i], P.k_in_stride[i] = a->k_in_stride[i], P.q_out_stride[i] = a->q_out_stride[i], P.k_out_stride[i] = a->k_out_stride[i];
    P.position_stride[0] = a->position_stride[0], P.position_stride[1] = a->position_stride[1];
    P.position_offset = a->position_offset;
    P.tokens = tokens, P.seq = (uint32_t)a->seq, P.n_q = a->n_q, P.heads = heads, P.head_dim = a->head_dim, P.rot_dim = a->rot_dim;
    P.positions_64 = a->positions_64, P.inverse = a->inverse, P.magnitude = a->magnitude;
    P.rot_cols = (a->rot_dim + 2 * n - 1) / (2 * n);
    const bool in_place = (!a->n_q || a->q_in == a->q_out) && (!a->n_k || a->k_in == a->k_out);
    P.cols = P.rot_cols + (in_place ? 0 : (a->head_dim - a->rot_dim + 2 * n - 1) / (2 * n));
    if (P.cols == 0) return HALOS_OK;
    // As few threads per token as still fill the GPU: their fixed cost then falls on more heads.
    const uint32_t most = kThreads / P.cols < heads ? kThreads / P.cols : heads;
    const int64_t want = ((int64_t)sm_count(a->device) * 1024 + tokens * P.cols - 1) / (tokens * P.cols);
    uint32_t least = (heads + 7) / 8;
    if (least > most) least = most;
    P.head_groups = want > most ? most : want < least ? least : (uint32_t)want;
    P.tokens_per_block = kThreads / (P.cols * P.head_groups);
    cudaStream_t st = (cudaStream_t)a->stream;
    if (a->dtype == HALOS_F32) return by_layout<float>(P, n, a->layout, st);
    if (a->dtype == HALOS_BF16) return by_layout<__nv_bfloat16>(P, n, a->layout, st);
    return by_layout<__half>(P, n, a->layout, st);
}
