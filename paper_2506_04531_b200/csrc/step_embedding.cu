// The embedding with scaling, and its gradient by sorted tokens.
//
// Both are bound by memory: the forward reads the rows that are asked for and writes as many as there are tokens; the gradient reads dout and writes every row
// of the table, most of them zeros.
//
// The gradient's row for a token is the sum of the rows of dout where it stands.  Up to 65536 places are sorted by token by one cluster of CTAs, in its shared memory, while
// the launch's other CTAs clear the rows that no token names; more are sorted by a radix sort over the GPU, and rows are cleared by a kernel of their own.  Both sorts
// are stable.  Then warps take equal runs of places in that order and 256 columns, and add up what belongs together; what goes on from warp to warp is joined in
// shared memory, and what goes on from CTA to CTA by the one that comes last, part by part in their order.  So the sums of a token's rows are in a fixed order, and no
// token, however frequent, waits for one warp.
//
// Measured: 65536 tokens x 768, bf16 from a table of 50304 in f32: forward 32 us (72% of the copy rate), gradient 69 us (56%): the sort takes 27 us, a third of them ranking places
// within a warp by ballots and a third moving them, in which 117 MB of rows are cleared (20 us alone); the sums, 36 us, read dout at 5 TB/s while the cleared rows leave the L2 cache.
// 7147 tokens x 1021 f16, half of them one token: 31 us.  With the sort over the GPU: 65537 x 768 99 us (40%), 131072 169 us (32%), 262144 254 us (34%).
#include "step_vector.cuh"

#include <atomic>
#include <math.h>
#include <type_traits>

namespace halos_step {
namespace {

constexpr int kThreads = 256;
constexpr int kMostBits = 9;           // of a radix pass
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;

struct EmbedParams {
    const char *weight, *dout, *token;
    char *out, *dweight;
    const char* dout_span[2];          // first byte of any row, and the one behind the last
    int64_t weight_stride, out_stride, dout_stride, dweight_stride;  // in elements
    uint32_t tokens, vocab, dim, tokens_64, accumulate;
    float scale;
    uint32_t *key[2], *place[2];       // [tokens] each: sorted so far, and where they stood
    uint32_t *counts;                  // [bins, sort blocks]
    uint32_t *met;                     // a bit for each token of the vocabulary
    float *head, *tail;                // [CTAs, dim]: sums of places that go on from the CTA before, or into the next
    uint32_t *arrived;                 // [CTAs, slabs]: how many have left their part of what begins in this one
    uint32_t chunk, slabs, jobs;       // places to a warp; runs of 256 columns; CTAs times slabs
    uint32_t sort_blocks, span;
};

// The token at place t; vocab where it is none.
__device__ __forceinline__ uint32_t token_at(const EmbedParams& P, uint32_t t) {
    const int64_t v = P.tokens_64 ? reinterpret_cast<const int64_t*>(P.token)[t] : (int64_t) reinterpret_cast<const int32_t*>(P.token)[t];
    return v < 0 || v >= (int64_t)P.vocab ? P.vocab : (uint32_t)v;
}

constexpr int kSlab = 256, kWarps = kThreads / 32;             // columns of a warp, eight to a lane

// A warp takes `AT_ONCE` tokens and 256 columns, with all loads under way before the first of them is used.
template <typename A, typename W, int V, int AT_ONCE>
__global__ void __launch_bounds__(kThreads) embedding_kernel(const __grid_constant__ EmbedParams P) {
    constexpr int J = kSlab / 32 / V;
    const uint32_t slab = blockIdx.x % P.slabs, first = (blockIdx.x / P.slabs * kWarps + threadIdx.x / 32) * AT_ONCE, lane = threadIdx.x % 32;
    if (first >= P.tokens) return;
    const auto column = [&](int j) { return slab * kSlab + (j * 32 + lane) * V; };
    uint32_t token[AT_ONCE];
    Words<W, V> w[AT_ONCE][J];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) token[i] = first + i < P.tokens ? token_at(P, first + i) : P.vocab;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j)
            w[i][j] = token[i] < P.vocab && column(j) < P.dim ? load_words<W, V>(reinterpret_cast<const W*>(P.weight) + token[i] * P.weight_stride + column(j)) : no_words<W, V>();
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        if (first + i >= P.tokens) break;
        A* out = reinterpret_cast<A*>(P.out) + (first + i) * P.out_stride;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float v[V];
            widen<W, V>(w[i][j], v);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = token[i] < P.vocab ? P.scale * v[e] : NAN;
            if (column(j) < P.dim) store_words<A, V>(out + column(j), narrow<A, V>(v));
        }
    }
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

// ------------------------------------------------------------------------------------------------ sort of up to 65536 places

// One cluster of CTAs sorts in its shared memory, a pass to a digit: threads rank their places within their warp, CTAs scan their warps' counts and exchange totals
// through the cluster, and places move to where they belong.  All other CTAs of the launch meanwhile write zeros to the rows that no token names, which
// they find out by going through the tokens themselves: the sort leaves the memory idle, and needs no other kernel's result.
constexpr uint32_t kMostInCluster = 8, kMostItems = 8, kMostClustered = kMostInCluster * kMostItems * kSortThreads;
constexpr uint32_t kMetWords = 4096;                         // of the vocabulary that a CTA looks at at a time

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet() { asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t address_in(const void* shared, uint32_t rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(shared)), "r"(rank));
    return a;
}

// Writes zeros to a row wherever it begins.
template <typename W>
__device__ __forceinline__ void clear_row(W* row, uint32_t dim, uint32_t lane, uint32_t lanes) {
    constexpr uint32_t kPer = 16 / sizeof(W);
    const uint32_t head = min(dim, (uint32_t)((16 - (uintptr_t)row % 16) % 16 / sizeof(W))), whole = (dim - head) / kPer, rest = head + whole * kPer;
    for (uint32_t c = lane; c < head; c += lanes) row[c] = from_f32<W>(0.f);
    for (uint32_t v = lane; v < whole; v += lanes) reinterpret_cast<uint4*>(row + head)[v] = make_uint4(0, 0, 0, 0);
    for (uint32_t c = rest + lane; c < dim; c += lanes) row[c] = from_f32<W>(0.f);
}

template <typename W>
__device__ __forceinline__ void clear_rows_not_met(const EmbedParams& P, uint32_t mine, uint32_t many, uint32_t* s_met) {
    const uint32_t words = (P.vocab + 31) / 32, warp = threadIdx.x / 32;
    // short rows take part of a warp each
    uint32_t lanes = 32;
    while (lanes > 8 && lanes * 16 / 2 >= P.dim * sizeof(W)) lanes /= 2;
    const uint32_t lane = threadIdx.x % lanes, sub = threadIdx.x % 32 / lanes;
    for (uint32_t first = 0; (uint64_t)first * many + mine < words; first += kMetWords) {       // word i of this CTA is word i * many + mine of all
        for (uint32_t i = threadIdx.x; i < kMetWords; i += kSortThreads) s_met[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (uint32_t t = threadIdx.x; t < P.tokens; t += kSortThreads) {
            const uint32_t v = token_at(P, t), word = v / 32, i = word / many;
            if (v < P.vocab && word - i * many == mine && i - first < kMetWords) atomicOr(&s_met[i - first], 1u << v % 32);
        }
        __syncthreads();
        for (uint32_t part = warp; part < kMetWords * 8; part += kSortWarps) {   // four rows at a time
            const uint32_t i = part / 8, four = part % 8 * 4;
            const uint64_t word = (uint64_t)(first + i) * many + mine;
            if (word >= words) break;
            const uint32_t met = s_met[i];
            for (uint32_t r = four + sub; r < four + 4; r += 32 / lanes) {
                const uint32_t v = (uint32_t)word * 32 + r;
                if (v < P.vocab && !(met >> r & 1)) clear_row(reinterpret_cast<W*>(P.dweight) + v * P.dweight_stride, P.dim, lane, lanes);
            }
        }
        __syncthreads();
    }
}

// The threads of the warp with this one's digit, among those where `is`: by its bits, which costs less than to look for equal values at once (31 us a sort of
// 65536 places with __match_any_sync).
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits, bool is) {
    uint32_t same = __ballot_sync(~0u, is);
#pragma unroll
    for (int b = 0; b < kMostBits; ++b)
        if (b < bits) {
            const uint32_t set = __ballot_sync(~0u, digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
    return same;
}

// The sum of the threads' values up to each; s_warp: [warps].
__device__ __forceinline__ uint32_t sum_up_to(uint32_t v, uint32_t* s_warp) {
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const auto within = [&](uint32_t x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t n = __shfl_up_sync(~0u, x, o);
            if (lane >= o) x += n;
        }
        return x;
    };
    v = within(v);
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    if (warp == 0) s_warp[lane] = within(s_warp[lane]);
    __syncthreads();
    return warp ? v + s_warp[warp - 1] : v;
}

template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads, 1) embedding_sort_kernel(const __grid_constant__ EmbedParams P, int passes, int bits_of_all, int in_cluster, uint32_t weight_type) {
    extern __shared__ __align__(16) uint64_t s_item[];         // [span]: key << 32 | place, as the cluster has sorted them; [span]: as this CTA has
    __shared__ __align__(16) uint16_t s_count[kSortWarps][1 << kMostBits];   // cleared by accesses of 16 bytes
    __shared__ uint32_t s_total[1 << kMostBits], s_base[1 << kMostBits], s_warp[kSortWarps];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if ((int)blockIdx.x >= in_cluster) {
        uint32_t* s_met = reinterpret_cast<uint32_t*>(&s_count[0][0]);
        const uint32_t mine = blockIdx.x - in_cluster, many = gridDim.x - in_cluster;
        if (weight_type == HALOS_F32) clear_rows_not_met<float>(P, mine, many, s_met);
        else clear_rows_not_met<__half>(P, mine, many, s_met);   // zero is the same in both
        return;
    }
    constexpr uint32_t span = ITEMS * kSortThreads;
    uint64_t* s_local = s_item + span;
    const uint32_t rank = cluster_rank(), begin = rank * span, here = begin >= P.tokens ? 0 : min(span, P.tokens - begin);
    uint64_t item[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const uint32_t local = (warp * ITEMS + k) * 32 + lane;
        item[k] = local < here ? (uint64_t)token_at(P, begin + local) << 32 | (begin + local) : 0;
    }
    for (uint32_t i = begin / ITEMS + threadIdx.x; i < P.jobs; i += in_cluster * kSortThreads) P.arrived[i] = 0;
    int shift = 0;
    for (int pass = 0; pass < passes; ++pass) {
        const int bits = (bits_of_all - shift + passes - pass - 1) / (passes - pass);
        const uint32_t bins = 1u << bits;
        uint32_t at[ITEMS];
        for (uint32_t i = threadIdx.x; i < sizeof s_count / 16; i += kSortThreads) reinterpret_cast<uint4*>(&s_count[0][0])[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const bool is = (warp * ITEMS + k) * 32 + lane < here;
            const uint32_t digit = (uint32_t)(item[k] >> 32) >> shift & (bins - 1);
            const uint32_t same = same_digit(digit, bits, is), before = __popc(same & ((1u << lane) - 1));
            const uint32_t had = is ? s_count[warp][digit] : 0;
            __syncwarp();
            if (is && before == 0) s_count[warp][digit] = (uint16_t)(had + __popc(same));
            __syncwarp();
            at[k] = had + before;
        }
        __syncthreads();
        uint32_t own = 0;                                      // of this thread's digit
        if (threadIdx.x < bins) {
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t n = s_count[w][threadIdx.x];
                s_count[w][threadIdx.x] = (uint16_t)own;
                own += n;
            }
            s_total[threadIdx.x] = own;
        }
        const uint32_t local_base = sum_up_to(own, s_warp) - own;
        if (threadIdx.x < bins) s_base[threadIdx.x] = local_base;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
            if ((warp * ITEMS + k) * 32 + lane < here) {
                const uint32_t digit = (uint32_t)(item[k] >> 32) >> shift & (bins - 1);
                s_local[s_base[digit] + s_count[warp][digit] + at[k]] = item[k];
            }
        cluster_meet();                                        // totals are there, and nobody needs what is in s_item
        uint32_t total = 0, before = 0;
        if (threadIdx.x < bins) {
            uint32_t n[kMostInCluster];
#pragma unroll
            for (uint32_t c = 0; c < kMostInCluster; ++c) {
                n[c] = 0;
                if (c < (uint32_t)in_cluster) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n[c]) : "r"(address_in(&s_total[threadIdx.x], c)) : "memory");
            }
#pragma unroll
            for (uint32_t c = 0; c < kMostInCluster; ++c) total += n[c], before += c < rank ? n[c] : 0;
        }
        const uint32_t base = sum_up_to(total, s_warp) - total + before;
        if (threadIdx.x < bins) s_base[threadIdx.x] = base - local_base;   // from the local order to the cluster's
        __syncthreads();
        // neighbours of one digit go to neighbouring places
        const bool last = pass + 1 == passes;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const uint32_t i = k * kSortThreads + threadIdx.x;
            if (i >= here) break;
            const uint64_t v = s_local[i];
            const uint32_t to = s_base[(uint32_t)(v >> 32) >> shift & (bins - 1)] + i;
            if (last) P.key[0][to] = (uint32_t)(v >> 32), P.place[0][to] = (uint32_t)v;
            else asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(address_in(&s_item[to % span], to / span)), "l"(v) : "memory");
        }
        cluster_meet();                                        // places have moved, totals have been read
        if (!last) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) item[k] = s_item[(warp * ITEMS + k) * 32 + lane];
        }
        shift += bits;
    }
}

// ------------------------------------------------------------------------------------------------ sums

template <typename W, int V>
__device__ __forceinline__ void write_part(const EmbedParams& P, uint32_t v, uint32_t c, const float* sum) {
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

// A few places, onto a table that is there: nothing is sorted or cleared.  A CTA to each place and 256 columns, which returns where an earlier place has the same token;
// the token's rows go round the warps, whose sums are joined in their order.  One launch: 8 to 100 places take 2.1 to 2.5 us and 9.6 of the host, sorted and then summed 10.8 to 13.4 and
// 12.  More places than threads would be looked through in turns by every CTA; they are sorted.
constexpr uint32_t kFewPlaces = kThreads;
template <typename A, typename W>
__global__ void __launch_bounds__(kThreads) embedding_few_kernel(const __grid_constant__ EmbedParams P) {
    constexpr int J = kSlab / 32;
    __shared__ uint32_t s_same[kWarps], s_place[kFewPlaces];
    __shared__ float s_sum[kWarps][kSlab];
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, place = blockIdx.y, key = token_at(P, place);
    const bool same = threadIdx.x < P.tokens && token_at(P, threadIdx.x) == key;
    const uint32_t in_warp = __ballot_sync(~0u, same);
    if (lane == 0) s_same[warp] = in_warp;
    if (__syncthreads_or((same && threadIdx.x < place) || key >= P.vocab)) return;
    uint32_t before = 0, many = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) {
        const uint32_t n = __popc(s_same[w]);
        before += w < warp ? n : 0, many += n;
    }
    if (same) s_place[before + __popc(in_warp & ((1u << lane) - 1))] = threadIdx.x;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSlab + lane;
    float sum[J];
#pragma unroll
    for (int j = 0; j < J; ++j) sum[j] = 0.f;
#pragma unroll 4
    for (uint32_t k = warp; k < many; k += kWarps) {
        const A* row = reinterpret_cast<const A*>(P.dout) + s_place[k] * P.dout_stride;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (first + j * 32 < P.dim) sum[j] += to_f32<A>(row[first + j * 32]);
    }
#pragma unroll
    for (int j = 0; j < J; ++j) s_sum[warp][j * 32 + lane] = sum[j];
    __syncthreads();
    const uint32_t column = blockIdx.x * kSlab + threadIdx.x;
    if (column >= P.dim) return;
    float all = s_sum[0][threadIdx.x];
    for (uint32_t w = 1; w < min(many, (uint32_t)kWarps); ++w) all += s_sum[w][threadIdx.x];
    write_part<W, 1>(P, key, column, &all);
}

constexpr int kAhead = 4096;                                   // bytes of dout that a warp has on their way

// A CTA takes 8 `chunk` neighbouring places in the sorted order and 256 columns, a warp `chunk` of the places, whose keys it holds 32 at a time.  Rows of dout are copied into shared memory
// ahead of their turn, in pieces of 16 bytes wherever the row begins; lanes have the columns of whole accesses where rows allow (V = 16 bytes), else every 32nd.
// A token whose places lie in one warp's chunk is written there.  What goes on from warp to warp is joined in shared memory; what goes on from CTA to
// CTA is left in memory, and the CTA that comes last, whichever it is, adds up the parts, in their order.
template <typename A, typename W, int V>
__global__ void __launch_bounds__(kThreads) embedding_sum_kernel(const __grid_constant__ EmbedParams P, const uint32_t* key, const uint32_t* place) {
    constexpr int J = kSlab / 32 / V, kRow = kSlab * (int)sizeof(A) + (V == 1 ? 16 : 0), kRing = kAhead / (kSlab * (int)sizeof(A));
    extern __shared__ __align__(16) char s_rows[];             // [warps][ring] rows
    __shared__ __align__(16) float s_head[kWarps][kSlab], s_tail[kWarps][kSlab];   // of V floats to an access
    static_assert(__alignof__(s_head) == 16 && __alignof__(s_tail) == 16, "the attribute is every declarator's");
    __shared__ uint32_t s_through[kWarps], s_goes[kWarps], s_last, s_ends, s_comes, s_key[2];   // keys of the run that comes from the CTA before, that goes on into the next
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, slab = blockIdx.x % P.slabs, block = blockIdx.x / P.slabs;
    const uint32_t span = P.chunk * kWarps, cta_from = block * span, from = min(P.tokens, cta_from + warp * P.chunk), n = min(P.chunk, P.tokens - from), blocks = P.jobs / P.slabs;
    const auto column = [&](int j) { return slab * kSlab + (j * 32 + lane) * V; };
    char* rows = s_rows + warp * kRing * kRow;
    after_previous();
    // Of 32 places and of the next 32 a lane has the key of one each, and where its row's columns begin.  Places of no token come last; `limit` is how many there
    // are before them, from `base` on, as far as is known: 64 at most.
    const A* here = reinterpret_cast<const A*>(P.dout) + slab * kSlab;
    const uint32_t columns = min((uint32_t)kSlab, P.dim - slab * kSlab);
    uint32_t base = 0, my_key, next_key, limit;
    const A *my_row, *next_row;
    const auto load = [&](uint32_t i, uint32_t& k, const A*& row) {
        k = i < n ? key[from + i] : P.vocab;
        row = here + (i < n ? place[from + i] : 0) * P.dout_stride;
    };
    const auto known = [&] {
        const uint32_t first = __ballot_sync(~0u, my_key < P.vocab), second = __ballot_sync(~0u, next_key < P.vocab);
        return ~first ? __popc(first) : 32 + __popc(second);
    };
    load(lane, my_key, my_row), load(lane + 32, next_key, next_row);
    const uint32_t key_before = from && n ? key[from - 1] : P.vocab, key_after = from + n < P.tokens ? key[from + n] : P.vocab;
    limit = known();
    const auto row_of = [&](uint32_t i) {                       // i: from `base` on
        return reinterpret_cast<const A*>(__shfl_sync(~0u, reinterpret_cast<uintptr_t>(i < 32 ? my_row : next_row), i % 32));
    };
    const auto fetch = [&](uint32_t i) {
        if (i < limit) {
            const A* row = row_of(i);
            char* to = rows + i % kRing * kRow;
            if constexpr (V > 1) {                              // each lane its own columns
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (column(j) < P.dim) copy_16(to + (j * 32 + lane) * 16, row + (j * 32 + lane) * V);
            } else {                                            // pieces of 16 bytes that cover the columns; the first begins up to 15 bytes before them
                const char* first = reinterpret_cast<const char*>((uintptr_t)row & ~(uintptr_t)15);
                const uint32_t bytes = (uint32_t)(reinterpret_cast<const char*>(row + columns) - first);
#pragma unroll
                for (int q = 0; q < (kRow + 511) / 512; ++q) {
                    const uint32_t at = (q * 32 + lane) * 16;
                    if (at >= bytes) break;
                    const char* p = first + at;
                    if (p >= P.dout_span[0] && p + 16 <= P.dout_span[1]) copy_16(to + at, p);
                    else {                                      // the tensor's own ends
#pragma unroll
                        for (int e = 0; e < 16 / (int)sizeof(A); ++e) {
                            const A* one = reinterpret_cast<const A*>(p) + e;
                            if (one >= row && one < row + columns) reinterpret_cast<A*>(to + at)[e] = *one;
                        }
                    }
                }
            }
        }
        copies_end();
    };
    float sum[J][V];
    const auto clear = [&] {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[j][e] = 0.f;
    };
    const auto keep = [&](float* s) {                           // [256], in the columns' order
#pragma unroll
        for (int j = 0; j < J; ++j) store_words<float, V>(s + (j * 32 + lane) * V, narrow<float, V>(sum[j]));
    };
    const auto add = [&](const float* s) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float v[V];
            widen<float, V>(load_words<float, V>(s + (j * 32 + lane) * V), v);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[j][e] += v[e];
        }
    };
    const auto write = [&](uint32_t k) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (column(j) < P.dim) write_part<W, V>(P, k, column(j), sum[j]);
    };
    const auto leave = [&](float* parts) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (column(j) < P.dim) store_words<float, V>(parts + (int64_t)block * P.dim + column(j), narrow<float, V>(sum[j]));
    };
    clear();
    bool began_before = n && __shfl_sync(~0u, my_key, 0) == key_before && key_before < P.vocab;
    bool through = false, tail = false;
    if (threadIdx.x == 0) s_comes = began_before, s_key[0] = my_key;
    for (uint32_t i = 0; i < kRing; ++i) fetch(i);
    for (;;) {
        // a bit for each of the first 31 places that is its token's last in this chunk; the 32nd's neighbour may still be on its way
        const uint32_t behind = __shfl_down_sync(~0u, my_key, 1), ends = __ballot_sync(~0u, base + lane + 1 >= n || behind != my_key), many = min(limit, 32u);
#pragma unroll 1
        for (uint32_t i = 0; i < many; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
            const char* slot = rows + i % kRing * kRow;
            if constexpr (V > 1) {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    float2 v[V / 2];
                    if (column(j) < P.dim) {
                        widen<A, V>(load_words<A, V>(reinterpret_cast<const A*>(slot) + (j * 32 + lane) * V), v);
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) {
                            const float2 t = add2(make_float2(sum[j][2 * e], sum[j][2 * e + 1]), v[e]);
                            sum[j][2 * e] = t.x, sum[j][2 * e + 1] = t.y;
                        }
                    }
                }
            } else {
                __syncwarp();                                   // pieces are other lanes' columns
                const A* row = reinterpret_cast<const A*>(slot + ((uintptr_t)row_of(i) & 15));
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (j * 32 < columns) sum[j][0] += to_f32<A>(row[j * 32 + lane]);
                __syncwarp();
            }
            fetch(i + kRing);
            if (i < 31 ? ends >> i & 1 : base + 32 >= n || __shfl_sync(~0u, next_key, 0) != __shfl_sync(~0u, my_key, 31)) {
                const uint32_t k = __shfl_sync(~0u, my_key, i);
                const bool on = base + i + 1 == n && key_after == k;    // goes on behind the chunk
                if (began_before) keep(s_head[warp]), through = on;
                else if (on) keep(s_tail[warp]), tail = true;
                else write(k);
                began_before = false;
                clear();
            }
        }
        if (limit <= 32) break;
        base += 32, my_key = next_key, my_row = next_row;
        load(base + 32 + lane, next_key, next_row), limit = known();
    }
    wait_copies(false);
    if (lane == 0) {
        s_through[warp] = through;
        s_goes[warp] = (through || tail) && from + n == min(P.tokens, cta_from + span);
        if (s_goes[warp]) s_key[1] = key_after;
    }
    __syncthreads();
    // From warp to warp.  The run that comes from the CTA before is warp 0's, any other that of the warp where it begins.
    bool goes = false;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) goes |= s_goes[w];
    const bool comes = s_comes;
    if (warp == 0 && comes) {
        clear(), add(s_head[0]);
        for (uint32_t w = 0; s_through[w] && w + 1 < kWarps;) add(s_head[++w]);
        leave(P.head);
    }
    if (tail) {
        clear(), add(s_tail[warp]);
        uint32_t w = warp + 1;
        for (; w < kWarps; ++w) {
            add(s_head[w]);
            if (!s_through[w]) break;
        }
        if (w < kWarps) write(key_after);
        else leave(P.tail);
    }
    if (!comes && !goes) return;
    // From CTA to CTA: up to two runs, or one that goes all the way through.
    __syncthreads();
    const bool one = comes && goes && s_key[0] == s_key[1];
    for (int r = 0; r < 2; ++r) {
        if (r == 0 ? !comes : !goes || one) continue;
        const uint32_t k = s_key[r];
        if (warp == 0) {
            uint32_t begins = block, ends = block;
            if (r == 0)
                for (bool more = true; more;) {                 // CTAs before this whose last place is k's
                    const bool is = lane < begins && key[(begins - lane) * span - 1] == k;
                    const uint32_t run = __ffs(~__ballot_sync(~0u, is)) - 1u;   // 2^32 - 1 where all are
                    begins -= run < 32 ? run : 32, more = run >= 32;
                }
            if (r == 1 || one)
                for (bool more = true; more;) {                 // CTAs behind it whose first place is k's
                    const uint32_t i = ends + 1 + lane;
                    const bool is = i < blocks && key[i * span] == k;
                    const uint32_t run = __ffs(~__ballot_sync(~0u, is)) - 1u;
                    ends += run < 32 ? run : 32, more = run >= 32;
                }
            if (lane == 0) {
                __threadfence();
                s_last = atomicAdd(&P.arrived[begins * P.slabs + slab], 1u) == ends - begins ? begins + 1 : 0;
                s_ends = ends;
                __threadfence();
            }
        }
        __syncthreads();
        const uint32_t begins = s_last - 1, ends = s_ends;
        if (s_last) {                                           // parts begins .. ends, in eight runs of neighbours
            const uint32_t parts = ends - begins + 1, per = (parts + kWarps - 1) / kWarps, lo = min(parts, warp * per), hi = min(parts, lo + per);
            clear();
#pragma unroll 4
            for (uint32_t i = lo; i < hi; ++i) {
                const float* part = (i ? P.head : P.tail) + (int64_t)(begins + i) * P.dim;
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (column(j) < P.dim) {
#pragma unroll
                        for (int e = 0; e < V; ++e) sum[j][e] += __ldcg(part + column(j) + e);
                    }
            }
            keep(s_head[warp]);
            __syncthreads();
            if (warp == 0) {
                for (uint32_t w = 1; w < kWarps && w * per < parts; ++w) add(s_head[w]);
                write(k);
            }
        }
        __syncthreads();
    }
}

template <typename W>
__global__ void __launch_bounds__(kThreads) embedding_zero_kernel(const __grid_constant__ EmbedParams P) {
    const uint32_t v = blockIdx.x * kWarps + threadIdx.x / 32;
    if (v >= P.vocab || (P.tokens && P.met[v / 32] >> v % 32 & 1)) return;
    clear_row(reinterpret_cast<W*>(P.dweight) + v * P.dweight_stride, P.dim, threadIdx.x % 32, 32);
}

// ------------------------------------------------------------------------------------------------ host

int check(const halos_embedding_args* a) {
    if (!a || a->struct_size != sizeof(halos_embedding_args)) return fail(HALOS_ERR_INVALID_ARG, "embedding: args missing or of another size");
    if (!is_type(a->dtype) || !is_type(a->weight_dtype)) return fail(HALOS_ERR_INVALID_ARG, "embedding: dtype");
    if (a->tokens < 0 || a->vocab <= 0 || a->dim == 0) return fail(HALOS_ERR_INVALID_ARG, "embedding: tokens, vocab or dim");
    if (a->tokens > 0x7fffffffll || a->vocab >= 0x7fffffffll || a->dim >= 1u << 30) return fail(HALOS_ERR_UNSUPPORTED, "embedding: 2^31 - 1 tokens or rows, or 2^30 columns, or more");
    return HALOS_OK;
}

// Widest access of 16 bytes at most that divides rows of these two tensors and every address; 32-bit tensors may take two of them.
uint32_t width_of(uint32_t dim, const void* a, int64_t a_stride, uint32_t a_size, const void* b, int64_t b_stride, uint32_t b_size) {
    const auto fits = [&](const void* p, int64_t stride, uint32_t size, uint32_t n) { return ((uintptr_t)p | (uint64_t)stride * size) % (n * size < 16 ? n * size : 16) == 0; };
    uint32_t v = 8;
    while (v > 1 && (dim % v || !fits(a, a_stride, a_size, v) || !fits(b, b_stride, b_size, v))) v /= 2;
    return v;
}
template <typename F>
int by_width(uint32_t v, F f) {
    switch (v) {
        case 8: return f(std::integral_constant<int, 8>());
        case 4: return f(std::integral_constant<int, 4>());
        case 2: return f(std::integral_constant<int, 2>());
        default: return f(std::integral_constant<int, 1>());
    }
}

struct Sizes {
    uint32_t bits, passes, blocks, span, chunk, slabs, ctas;
    uint64_t arrays, counts, met, arrived, sums, all;   // bytes
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
    s.slabs = (a->dim + kSlab - 1) / kSlab;
    // As many places to a warp as fill the SMs once with four CTAs each, 8 at least; where these are over 96, as often as it takes.
    const uint64_t jobs = (uint64_t)a->tokens * s.slabs, at_once = most * 4 * kWarps, times = (jobs + at_once * 96 - 1) / (at_once * 96);
    const uint64_t chunk = times ? (jobs + at_once * times - 1) / (at_once * times) : 0;
    s.chunk = chunk < 8 ? 8 : (uint32_t)chunk;
    s.ctas = (uint32_t)((a->tokens + s.chunk * kWarps - 1) / (s.chunk * kWarps));
    s.arrays = rounded_up((uint64_t)a->tokens * 4, 16);
    s.counts = ((uint64_t)s.blocks << kMostBits) * 4;
    s.met = rounded_up(((uint64_t)a->vocab + 31) / 32 * 4, 16);
    s.arrived = rounded_up((uint64_t)s.ctas * s.slabs * 4, 16);
    s.sums = rounded_up((uint64_t)s.ctas * a->dim * 4, 16);
    s.all = 4 * s.arrays + s.counts + s.met + s.arrived + 2 * s.sums;
    return s;
}

// How many clusters of the sort's kernel the device runs at the same time: asked for once for each size of a cluster (larger ones come with the most
// shared memory, which an SM has once in any case).
int clusters_at_once(int32_t device, const void* kernel, const cudaLaunchConfig_t& config, uint32_t in_cluster, int* clusters) {
    static std::atomic<int> known[64][kMostInCluster + 1];
    *clusters = known[device][in_cluster].load(std::memory_order_relaxed);
    if (*clusters) return HALOS_OK;
    if (int rc = cuda_status(cudaOccupancyMaxActiveClusters(clusters, kernel, &config), "embedding clusters")) return rc;
    if (*clusters < 1) *clusters = 1;
    known[device][in_cluster].store(*clusters, std::memory_order_relaxed);
    return HALOS_OK;
}

template <int ITEMS>
int sort(const EmbedParams& P, const Sizes& s, const halos_embedding_args* a) {
    uint32_t in_cluster = 1;
    while (in_cluster * ITEMS * kSortThreads < P.tokens) in_cluster *= 2;
    const uint32_t shared = 2 * ITEMS * kSortThreads * 8;
    static Allowed allowed;
    if (int rc = allow_smem(embedding_sort_kernel<ITEMS>, (int)shared, allowed)) return rc;
    cudaLaunchAttribute cluster{};
    cluster.id = cudaLaunchAttributeClusterDimension, cluster.val.clusterDim.x = in_cluster, cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = in_cluster, config.blockDim = kSortThreads, config.dynamicSmemBytes = shared, config.stream = (cudaStream_t)a->stream, config.attrs = &cluster, config.numAttrs = 1;
    if (!P.accumulate) {                               // as many more as run at the same time; a word of 32 rows to each at least
        int clusters = 0;
        if (int rc = clusters_at_once(a->device, (const void*)embedding_sort_kernel<ITEMS>, config, in_cluster, &clusters)) return rc;
        const uint32_t words = (P.vocab + 31) / 32, wanted = 1 + (words + in_cluster - 1) / in_cluster;
        config.gridDim = in_cluster * (clusters < 2 ? 2 : (uint32_t)clusters < wanted ? (uint32_t)clusters : wanted);
    }
    return cuda_status(cudaLaunchKernelEx(&config, embedding_sort_kernel<ITEMS>, P, (int)s.passes, (int)s.bits, (int)in_cluster, a->weight_dtype), "embedding launch");
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
    P.slabs = (P.dim + kSlab - 1) / kSlab;
    cudaStream_t st = (cudaStream_t)a->stream;
    // Four tokens to a warp, or one where that gives no SM eight warps.
    const bool few = (uint64_t)P.tokens * P.slabs < (uint64_t)sm_count(a->device) * 32;
    const uint64_t jobs = ((uint64_t)P.tokens + kWarps * (few ? 1 : 4) - 1) / (kWarps * (few ? 1 : 4)) * P.slabs;
    if (jobs > 0x7fffffffull) return fail(HALOS_ERR_UNSUPPORTED, "embedding: too many rows");
    return by_width(width_of(P.dim, a->weight, a->weight_stride, size_of(a->weight_dtype), a->out, a->out_stride, size_of(a->dtype)), [&](auto n) {
        return by_type(a->dtype, [&](auto x) {
            return by_type(a->weight_dtype, [&](auto w) {
                constexpr int V = decltype(n)::value;
                if (few) embedding_kernel<decltype(x), decltype(w), V, 1><<<(unsigned)jobs, kThreads, 0, st>>>(P);
                else embedding_kernel<decltype(x), decltype(w), V, 4><<<(unsigned)jobs, kThreads, 0, st>>>(P);
                return cuda_status(cudaGetLastError(), "embedding launch");
            });
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
    P.arrived = (uint32_t*)at, at += s.arrived;
    P.head = (float*)at, at += s.sums;
    P.tail = (float*)at;
    if ((uint64_t)s.ctas * s.slabs > 0x7fffffffull) return fail(HALOS_ERR_UNSUPPORTED, "embedding: too many sums");
    P.chunk = s.chunk, P.slabs = s.slabs, P.jobs = s.ctas * s.slabs, P.sort_blocks = s.blocks, P.span = s.span;
    cudaStream_t st = (cudaStream_t)a->stream;
    const bool whole = width_of(P.dim, a->dweight, a->dweight_stride, wsize, P.tokens ? a->dout : a->dweight, P.tokens ? a->dout_stride : a->dweight_stride, P.tokens ? size : wsize) >= 16 / size;
    const int64_t far = P.tokens ? (int64_t)(P.tokens - 1) * a->dout_stride : 0;
    P.dout_span[0] = P.dout + (far < 0 ? far : 0) * (int64_t)size, P.dout_span[1] = P.dout + ((far > 0 ? far : 0) + a->dim) * (int64_t)size;
    if (P.accumulate && P.tokens && P.tokens <= kFewPlaces)
        return by_type(a->weight_dtype, [&](auto wt) -> int {
            return by_type(a->dtype, [&](auto x) -> int {
                embedding_few_kernel<decltype(x), decltype(wt)><<<dim3(P.slabs, P.tokens), kThreads, 0, st>>>(P);
                return cuda_status(cudaGetLastError(), "embedding launch");
            });
        });
    int sorted = 0;                                    // which of the two arrays holds the sorted places
    if (P.tokens && P.tokens <= kMostClustered) {
        // eight CTAs as soon as there is work for them
        const uint32_t each = (P.tokens + kMostInCluster * kSortThreads - 1) / (kMostInCluster * kSortThreads);
        if (int rc = each <= 1 ? sort<1>(P, s, a) : each <= 2 ? sort<2>(P, s, a) : each <= 4 ? sort<4>(P, s, a) : sort<8>(P, s, a)) return rc;
    } else if (P.tokens) {
        if (int rc = cuda_status(cudaMemsetAsync(P.met, 0, s.met + s.arrived, st), "embedding workspace")) return rc;
        for (uint32_t pass = 0, shift = 0; pass < s.passes; ++pass) {
            const int bits = (int)((s.bits - shift + s.passes - pass - 1) / (s.passes - pass));
            embedding_count_kernel<<<P.sort_blocks, kSortThreads, 0, st>>>(P, (int)pass, (int)shift, bits);
            embedding_place_kernel<<<P.sort_blocks, kSortThreads, 0, st>>>(P, (int)pass, (int)shift, bits);
            if (int rc = cuda_status(cudaGetLastError(), "embedding launch")) return rc;
            shift += bits;
        }
        sorted = s.passes & 1;
    }
    return by_type(a->weight_dtype, [&](auto wt) -> int {
        using W = decltype(wt);
        if (!P.accumulate && (!P.tokens || P.tokens > kMostClustered)) {
            embedding_zero_kernel<W><<<(P.vocab + kWarps - 1) / kWarps, kThreads, 0, st>>>(P);
            if (int rc = cuda_status(cudaGetLastError(), "embedding launch")) return rc;
        }
        if (!P.tokens) return HALOS_OK;
        return by_type(a->dtype, [&](auto x) -> int {
            using A = decltype(x);
            const auto launch = [&](auto* kernel, uint32_t row, Allowed& allowed) -> int {
                const uint32_t shared = kWarps * (kAhead / (kSlab * (uint32_t)sizeof(A))) * row;
                if (int rc = allow_smem(kernel, (int)shared, allowed)) return rc;
                return launch_after(kernel, P.jobs, kThreads, shared, st, "embedding launch", P, (const uint32_t*)P.key[sorted], (const uint32_t*)P.place[sorted]);
            };
            static Allowed allowed[2];
            constexpr int V = 16 / sizeof(A);
            constexpr uint32_t row = kSlab * sizeof(A);
            return whole ? launch(embedding_sum_kernel<A, W, V>, row, allowed[0]) : launch(embedding_sum_kernel<A, W, 1>, row + 16, allowed[1]);
        });
    });
}
