// The embedding with scaling, and its gradient by sorted tokens.
//
// The gradient's row for a token is the sum of the rows of dout where it stands.  Places are sorted by token, stably, with a radix sort of up to
// 9 bits a pass; then a warp takes 32 places in that order and 256 columns, and adds up what belongs together.  A token whose places go on
// into the next warps' is added up from those warps' sums, in order, by a kernel of its own.  So sums of a token's rows are in a fixed order, and no
// token, however frequent, waits for one warp.
#include "step_vector.cuh"

#include <math.h>
#include <type_traits>

namespace halos_step {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 32;             // sorted places to a warp
constexpr int kMostBits = 9;           // of a radix pass
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;

struct EmbedParams {
    const char *weight, *dout, *token;
    char *out, *dweight;
    int64_t weight_stride, out_stride, dout_stride, dweight_stride;  // in elements
    uint32_t tokens, vocab, dim, tokens_64, accumulate;
    float scale;
    uint32_t *key[2], *place[2];       // [tokens] each: sorted so far, and where they stood
    uint32_t *counts;                  // [bins, sort blocks]
    uint32_t *met;                     // a bit for each token of the vocabulary
    float *head, *tail;                // [chunks, dim]: sums of places that go on from the chunk before, or into the next
    uint32_t chunks, sort_blocks, span;
};

// The token at place t; vocab where it is none.
__device__ __forceinline__ uint32_t token_at(const EmbedParams& P, uint32_t t) {
    const int64_t v = P.tokens_64 ? reinterpret_cast<const int64_t*>(P.token)[t] : (int64_t) reinterpret_cast<const int32_t*>(P.token)[t];
    return v < 0 || v >= (int64_t)P.vocab ? P.vocab : (uint32_t)v;
}

template <typename A, typename W>
__global__ void __launch_bounds__(kThreads) embedding_kernel(const __grid_constant__ EmbedParams P) {
    const uint32_t t = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (t >= P.tokens) return;
    const uint32_t v = token_at(P, t);
    A* out = reinterpret_cast<A*>(P.out) + t * P.out_stride;
    const W* row = reinterpret_cast<const W*>(P.weight) + v * P.weight_stride;
    for (uint32_t c = threadIdx.x % 32; c < P.dim; c += 32) out[c] = from_f32<A>(v == P.vocab ? NAN : P.scale * to_f32<W>(row[c]));
}

// ------------------------------------------------------------------------------------------------ sort

// How often each digit comes in each block's span.
__global__ void __launch_bounds__(kSortThreads) embedding_count_kernel(const __grid_constant__ EmbedParams P, int pass, int shift, int bits) {
    __shared__ uint32_t s_count[1 << kMostBits];
    const uint32_t bins = 1u << bits, from = blockIdx.x * P.span, to = min(P.tokens, from + P.span);
    for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) s_count[b] = 0;
    __syncthreads();
    for (uint32_t i = from + threadIdx.x; i < to; i += kSortThreads) {
        const uint32_t key = pass ? P.key[pass & 1][i] : token_at(P, i);
        if (!pass && key < P.vocab) atomicOr(&P.met[key / 32], 1u << key % 32);
        atomicAdd(&s_count[key >> shift & (bins - 1)], 1u);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kSortThreads) P.counts[b * P.sort_blocks + blockIdx.x] = s_count[b];
}

// Moves a block's span to where its digits belong.
__global__ void __launch_bounds__(kSortThreads) embedding_place_kernel(const __grid_constant__ EmbedParams P, int pass, int shift, int bits) {
    __shared__ uint32_t s_base[1 << kMostBits], s_warp[kSortWarps];
    __shared__ uint16_t s_count[kSortWarps][1 << kMostBits];
    const uint32_t bins = 1u << bits, from = blockIdx.x * P.span, to = min(P.tokens, from + P.span), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t total = 0, before = 0;
    if (threadIdx.x < bins)
        for (uint32_t b = 0; b < P.sort_blocks; ++b) {
            const uint32_t n = P.counts[threadIdx.x * P.sort_blocks + b];
            total += n;
            if (b < blockIdx.x) before += n;
        }
    uint32_t upto = total;                                   // of the digits up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t n = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += n;
    }
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    for (uint32_t w = 0; w < warp; ++w) upto += s_warp[w];
    if (threadIdx.x < bins) s_base[threadIdx.x] = upto - total + before;
    for (uint32_t at = from; at < to; at += kSortThreads) {
        for (uint32_t i = threadIdx.x; i < kSortWarps << kMostBits; i += kSortThreads) (&s_count[0][0])[i] = 0;
        __syncthreads();
        const uint32_t i = at + threadIdx.x;
        const bool here = i < to;
        const uint32_t key = !here ? 0 : pass ? P.key[pass & 1][i] : token_at(P, i), digit = key >> shift & (bins - 1);
        const uint32_t same = __match_any_sync(~0u, here ? digit : bins), rank = __popc(same & ((1u << lane) - 1));
        if (here && rank == 0) s_count[warp][digit] = (uint16_t)__popc(same);
        __syncthreads();
        if (threadIdx.x < bins) {
            uint32_t sum = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t n = s_count[w][threadIdx.x];
                s_count[w][threadIdx.x] = (uint16_t)sum;
                sum += n;
            }
            total = sum;
        }
        __syncthreads();
        if (here) {
            const uint32_t to_place = s_base[digit] + s_count[warp][digit] + rank;
            P.key[(pass + 1) & 1][to_place] = key;
            P.place[(pass + 1) & 1][to_place] = pass ? P.place[pass & 1][i] : i;
        }
        __syncthreads();
        if (threadIdx.x < bins) s_base[threadIdx.x] += total;
    }
}

// ------------------------------------------------------------------------------------------------ sums

// Where V columns of T begin that a lane takes, for slab s; V divides the row.
template <typename W, int V>
__device__ __forceinline__ void write_row(const EmbedParams& P, uint32_t v, uint32_t c, const float (&sum)[V]) {
    W* to = reinterpret_cast<W*>(P.dweight) + v * P.dweight_stride + c;
    float r[V];
    if (P.accumulate) {
        widen<W, V>(load_words<W, V>(to), r);
#pragma unroll
        for (int e = 0; e < V; ++e) r[e] = fmaf(P.scale, sum[e], r[e]);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) r[e] = P.scale * sum[e];
    }
    store_words<W, V>(to, narrow<W, V>(r));
}

template <int V>
__device__ __forceinline__ void write_floats(float* to, const float (&v)[V]) { store_words<float, V>(to, narrow<float, V>(v)); }

template <typename A, typename W, int V>
__global__ void __launch_bounds__(kThreads) embedding_sum_kernel(const __grid_constant__ EmbedParams P, const uint32_t* key, const uint32_t* place, uint32_t slabs) {
    const uint32_t job = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, lane = threadIdx.x % 32, chunk = job / slabs, c = ((job - chunk * slabs) * 32 + lane) * V;
    if (chunk >= P.chunks) return;
    const uint32_t from = chunk * kChunk, n = min((uint32_t)kChunk, P.tokens - from);
    const uint32_t my_key = lane < n ? key[from + lane] : P.vocab, my_place = lane < n ? place[from + lane] : 0;
    const uint32_t key_before = from ? key[from - 1] : P.vocab, key_after = from + n < P.tokens ? key[from + n] : P.vocab;
    const bool mine = c < P.dim;
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    constexpr int kAhead = 8;
    bool began_before = __shfl_sync(~0u, my_key, 0) == key_before;
    for (uint32_t i0 = 0; i0 < n; i0 += kAhead) {
        Words<A, V> w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t k = __shfl_sync(~0u, my_key, i0 + i), t = __shfl_sync(~0u, my_place, i0 + i);
            w[i] = mine && k < P.vocab ? load_words<A, V>(reinterpret_cast<const A*>(P.dout) + t * P.dout_stride + c) : no_words<A, V>();
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t at = i0 + i;
            if (at >= n) break;
            const uint32_t k = __shfl_sync(~0u, my_key, at), next = at + 1 < n ? __shfl_sync(~0u, my_key, at + 1) : key_after;
            if (k >= P.vocab) break;                    // no tokens: they come last
            float v[V];
            widen<A, V>(w[i], v);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += v[e];
            const bool ends = at + 1 == n;
            if (next != k || ends) {
                if (mine) {
                    if (began_before) write_floats<V>(P.head + (int64_t)chunk * P.dim + c, sum);
                    else if (next == k) write_floats<V>(P.tail + (int64_t)chunk * P.dim + c, sum);
                    else write_row<W, V>(P, k, c, sum);
                }
                began_before = false;
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = 0.f;
            }
        }
    }
}

// The tokens whose places go on from one chunk into the next: the chunk where they begin adds up.
template <typename W, int V>
__global__ void __launch_bounds__(kThreads) embedding_join_kernel(const __grid_constant__ EmbedParams P, const uint32_t* key, uint32_t slabs) {
    const uint32_t job = blockIdx.x * (kThreads / 32) + threadIdx.x / 32, lane = threadIdx.x % 32, chunk = job / slabs, c = ((job - chunk * slabs) * 32 + lane) * V;
    if (chunk + 1 >= P.chunks) return;
    const uint32_t from = chunk * kChunk, k = key[from + kChunk - 1];
    if (k >= P.vocab || key[from + kChunk] != k || (from && key[from] == k && key[from - 1] == k)) return;
    if (c >= P.dim) return;
    float sum[V];
    widen<float, V>(load_words<float, V>(P.tail + (int64_t)chunk * P.dim + c), sum);
    for (uint32_t i = chunk + 1; i < P.chunks && key[i * kChunk] == k; ++i) {
        float v[V];
        widen<float, V>(load_words<float, V>(P.head + (int64_t)i * P.dim + c), v);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += v[e];
    }
    write_row<W, V>(P, k, c, sum);
}

template <typename W, int V>
__global__ void __launch_bounds__(kThreads) embedding_zero_kernel(const __grid_constant__ EmbedParams P) {
    const uint32_t v = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (v >= P.vocab || (P.tokens && P.met[v / 32] >> v % 32 & 1)) return;
    W* row = reinterpret_cast<W*>(P.dweight) + v * P.dweight_stride;
    for (uint32_t c = threadIdx.x % 32 * V; c < P.dim; c += 32 * V) store_words<W, V>(row + c, no_words<W, V>());
}

// ------------------------------------------------------------------------------------------------ host

int check(const halos_embedding_args* a) {
    if (!a || a->struct_size != sizeof(halos_embedding_args)) return fail(HALOS_ERR_INVALID_ARG, "embedding: args missing or of another size");
    if (!is_type(a->dtype) || !is_type(a->weight_dtype)) return fail(HALOS_ERR_INVALID_ARG, "embedding: dtype");
    if (a->tokens < 0 || a->vocab <= 0 || a->dim == 0) return fail(HALOS_ERR_INVALID_ARG, "embedding: tokens, vocab or dim");
    if (a->tokens > 0x7fffffffll || a->vocab >= 0x7fffffffll || a->dim >= 1u << 30) return fail(HALOS_ERR_UNSUPPORTED, "embedding: 2^31 - 1 tokens or rows, or 2^30 columns, or more");
    return HALOS_OK;
}

struct Sizes {
    uint32_t bits, passes, blocks, span, chunks;
    uint64_t arrays, counts, met, sums, all;   // bytes
};
uint64_t rounded_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
Sizes sizes_of(const halos_embedding_args* a, int32_t device) {
    Sizes s{};
    while ((uint64_t)a->vocab >> s.bits) ++s.bits;
    s.passes = (s.bits + kMostBits - 1) / kMostBits;
    const uint64_t most = sm_count(device);
    s.blocks = (uint32_t)((a->tokens + kSortThreads - 1) / kSortThreads);
    if (s.blocks > most) s.blocks = (uint32_t)most;
    if (s.blocks == 0) s.blocks = 1;
    s.span = (uint32_t)rounded_up((a->tokens + s.blocks - 1) / s.blocks, kSortThreads);
    s.chunks = (uint32_t)((a->tokens + kChunk - 1) / kChunk);
    s.arrays = rounded_up((uint64_t)a->tokens * 4, 16);
    s.counts = ((uint64_t)s.blocks << kMostBits) * 4;
    s.met = rounded_up(((uint64_t)a->vocab + 31) / 32 * 4, 16);
    s.sums = rounded_up((uint64_t)s.chunks * a->dim * 4, 16);
    s.all = 4 * s.arrays + s.counts + s.met + 2 * s.sums;
    return s;
}

template <typename F>
int by_type(uint32_t type, F f) {
    if (type == HALOS_F32) return f(float());
    if (type == HALOS_BF16) return f(__nv_bfloat16());
    return f(__half());
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_embedding_fwd(const halos_embedding_args* a) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    if (a->tokens == 0) return HALOS_OK;
    if (!a->token || !a->weight || !a->out) return fail(HALOS_ERR_INVALID_ARG, "embedding: null pointer");
    if ((uintptr_t)a->weight % size_of(a->weight_dtype) || (uintptr_t)a->out % size_of(a->dtype) || (uintptr_t)a->token % (a->tokens_64 ? 8 : 4))
        return fail(HALOS_ERR_INVALID_ARG, "embedding: tensor not aligned to its elements");
    if (int rc = enter(a->device)) return rc;
    EmbedParams P{};
    P.weight = (const char*)a->weight, P.out = (char*)a->out, P.token = (const char*)a->token, P.weight_stride = a->weight_stride, P.out_stride = a->out_stride;
    P.tokens = (uint32_t)a->tokens, P.vocab = (uint32_t)a->vocab, P.dim = a->dim, P.tokens_64 = a->tokens_64, P.scale = a->scale;
    cudaStream_t st = (cudaStream_t)a->stream;
    return by_type(a->dtype, [&](auto x) {
        return by_type(a->weight_dtype, [&](auto w) {
            embedding_kernel<decltype(x), decltype(w)><<<(P.tokens + kThreads / 32 - 1) / (kThreads / 32), kThreads, 0, st>>>(P);
            return cuda_status(cudaGetLastError(), "embedding launch");
        });
    });
}

extern "C" int halos_embedding_workspace(const halos_embedding_args* a, uint64_t* bytes) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    if (!bytes) return fail(HALOS_ERR_INVALID_ARG, "embedding: null pointer");
    if (int rc = enter(a->device)) return rc;
    *bytes = sizes_of(a, a->device).all;
    return HALOS_OK;
}

extern "C" int halos_embedding_bwd(const halos_embedding_args* a) {
    using namespace halos_step;
    if (int rc = check(a)) return rc;
    if (!a->dweight || (a->tokens && (!a->token || !a->dout))) return fail(HALOS_ERR_INVALID_ARG, "embedding: null pointer");
    const uint32_t size = size_of(a->dtype), wsize = size_of(a->weight_dtype);
    if ((uintptr_t)a->dweight % wsize || (uintptr_t)a->dout % size || (uintptr_t)a->token % (a->tokens_64 ? 8 : 4))
        return fail(HALOS_ERR_INVALID_ARG, "embedding: tensor not aligned to its elements");
    if (int rc = enter(a->device)) return rc;
    const Sizes s = sizes_of(a, a->device);
    if (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < s.all) return fail(HALOS_ERR_INVALID_ARG, "embedding: workspace missing, not aligned or too small");
    EmbedParams P{};
    P.dout = (const char*)a->dout, P.dweight = (char*)a->dweight, P.token = (const char*)a->token, P.dout_stride = a->dout_stride, P.dweight_stride = a->dweight_stride;
    P.tokens = (uint32_t)a->tokens, P.vocab = (uint32_t)a->vocab, P.dim = a->dim, P.tokens_64 = a->tokens_64, P.accumulate = a->accumulate, P.scale = a->scale;
    char* at = (char*)a->workspace;
    for (int i = 0; i < 2; ++i) P.key[i] = (uint32_t*)at, at += s.arrays, P.place[i] = (uint32_t*)at, at += s.arrays;
    P.counts = (uint32_t*)at, at += s.counts;
    P.met = (uint32_t*)at, at += s.met;
    P.head = (float*)at, at += s.sums;
    P.tail = (float*)at;
    P.chunks = s.chunks, P.sort_blocks = s.blocks, P.span = s.span;
    cudaStream_t st = (cudaStream_t)a->stream;
    // Widest access of 16 bytes at most that divides the rows and every address.
    uint32_t v = 8;
    const auto divides = [&](uint32_t n) {
        const auto fits = [&](const void* p, int64_t stride, uint32_t bytes) { return ((uintptr_t)p | (uint64_t)stride * bytes) % (n * bytes < 16 ? n * bytes : 16) == 0; };
        return a->dim % n == 0 && n * size <= 16 && fits(a->dweight, a->dweight_stride, wsize) && (!a->tokens || fits(a->dout, a->dout_stride, size));
    };
    while (v > 1 && !divides(v)) v /= 2;
    const auto by_width = [&](auto f) -> int {
        switch (v) {
            case 8: return f(std::integral_constant<int, 8>());
            case 4: return f(std::integral_constant<int, 4>());
            case 2: return f(std::integral_constant<int, 2>());
            default: return f(std::integral_constant<int, 1>());
        }
    };
    if ((uint64_t)P.chunks * ((P.dim + 32 * v - 1) / (32 * v)) > 0xffffff00ull) return fail(HALOS_ERR_UNSUPPORTED, "embedding: too many sums");
    if (P.tokens) {
        if (int rc = cuda_status(cudaMemsetAsync(P.met, 0, s.met, st), "embedding workspace")) return rc;
        for (uint32_t pass = 0, shift = 0; pass < s.passes; ++pass) {
            const int bits = (int)((s.bits - shift + s.passes - pass - 1) / (s.passes - pass));
            embedding_count_kernel<<<P.sort_blocks, kSortThreads, 0, st>>>(P, (int)pass, (int)shift, bits);
            embedding_place_kernel<<<P.sort_blocks, kSortThreads, 0, st>>>(P, (int)pass, (int)shift, bits);
            if (int rc = cuda_status(cudaGetLastError(), "embedding launch")) return rc;
            shift += bits;
        }
    }
    return by_type(a->weight_dtype, [&](auto wt) -> int {
        using W = decltype(wt);
        return by_width([&](auto n) -> int {
            constexpr int V = decltype(n)::value;
            const uint32_t slabs = (P.dim + 32 * V - 1) / (32 * V), per = kThreads / 32;
            if (!P.accumulate) embedding_zero_kernel<W, V><<<(P.vocab + per - 1) / per, kThreads, 0, st>>>(P);
            if (!P.tokens) return cuda_status(cudaGetLastError(), "embedding launch");
            const uint64_t jobs = (uint64_t)P.chunks * slabs;
            const uint32_t* key = P.key[s.passes & 1];
            const uint32_t* place = P.place[s.passes & 1];
            const unsigned grid = (unsigned)((jobs + per - 1) / per);
            const int rc = by_type(a->dtype, [&](auto x) {
                if constexpr (V * sizeof(x) <= 16) embedding_sum_kernel<decltype(x), W, V><<<grid, kThreads, 0, st>>>(P, key, place, slabs);
                return cuda_status(cudaGetLastError(), "embedding launch");
            });
            if (rc) return rc;
            embedding_join_kernel<W, V><<<grid, kThreads, 0, st>>>(P, key, slabs);
            return cuda_status(cudaGetLastError(), "embedding launch");
        });
    });
}
