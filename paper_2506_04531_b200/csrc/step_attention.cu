// Attention and its backward pass on the fifth-generation tensor cores.
//
// Forward, one CTA per 128 queries of a head: S = Q K^T into tensor memory, a thread per query takes its row through
// the online softmax, P goes back into tensor memory as the left operand of O += P V.  The running maximum is moved (and O rescaled)
// only when the probabilities of a tile add up to more than 2^10 without: a single one stays within both 16-bit types.
//
// Backward, two kernels without atomics, so that gradients are the same bits every time:
//   dK, dV: a CTA keeps 128 keys and walks the queries of its group's heads, 64 at a time.  It works on the transposes,
//           S^T = K Q^T and dP^T = V dO^T, so that P^T and dS^T are left operands in tensor memory: nothing is staged
//           in shared memory between the products.
//   dQ:     a CTA keeps 128 queries and walks the keys, 64 at a time: S, dP, and dQ += dS K with dS in tensor memory.
// That is 7 products per pair of tiles where adding dQ up by atomics would take 5; what it saves is the 32-bit dQ
// in memory, its clearing and conversion, and the order of its sums.
//
// Roles in a CTA: warps of 4 take the rows (thread = tensor memory lane), one warp issues the bulk copies, one the products.
//
// Measured, causal, 2048 tokens, bf16: 16 x 12 heads of 64 forward 196 us (525 TFLOP/s of visible pairs), backward 568 us (454);
// 4 x 16 heads of 128 forward 97 us (708).  Under way, a tile of 64 keys takes 0.76 us in each of an SM's two CTAs, of which the
// exponential unit is busy 74%; a quarter of a CTA's time is its beginning and end, which the other CTA only partly
// fills.  dK, dV: 1.1 us for 64 queries, bound by the products (63%); dQ: 0.76 us for 64 keys.
//
// p and ds are rounded to the inputs' type where they become operands (that is what the tensor cores take), and D comes from an o that was rounded
// to it (the forward pass returns no other); every sum, statistic and accumulator is in 32 bits, and each result is rounded once.
#include "step_tcgen05.cuh"

#include <limits.h>
#include <math.h>
#include <type_traits>

namespace halos_step {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRecord = 64;   // queries to a record
// Of 64 probabilities relative to a maximum that may be an old one.  Any bound that keeps a single one within 16-bit floats would do.
constexpr float kMostSum = 1024.f;
// Largest maximum, times scale log2(e), that is rounded to one number and taken off inside the multiply-add: the exponent of the maximum itself
// is then off by 2^-9 at most. At 2^28 it would be off by 16, and no probability relative to such a number stays small.
constexpr float kNear = 65536.f;

// What the backward pass knows of 64 queries of a head before it starts.  A query that sees nothing, or is none, has
// minus_lse2 = -infinity: its probabilities are 0.
struct Record {
    float minus_lse2[kRecord];   // - log2 of the sum of exponentials
    float minus_delta[kRecord];  // - dout . o
    int lo[kRecord], hi[kRecord];
};
static_assert(sizeof(Record) == 1024, "one bulk copy");
// The keys that a batch row's 64 queries see, in four numbers: some of them see [min_lo, max_hi), all of them see
// [max_lo, min_hi).  max_lo = INT_MAX: one of them sees nothing.
struct Reach { int min_lo, max_hi, max_lo, min_hi; };
// Largest squared lengths of dout of the queries and of v of the keys that take part, as bits of non-negative floats.
struct Lengths { uint32_t dout, v; };

// Floats with 5 bits of exponent hold neither a small p (under 2^-14 they lose digits) nor a ds of any size: it is as small as p times
// dout, and may be as large as the loss scale that dout carries. There p is taken 2^kRaised times and ds ds_steps times (a power of two that
// goes by the lengths of dout and v, |ds| <= 2 |dout| |v|), and what they add up to is divided again.  The lengths take a kernel of their own, 8 us
// of 440 (8197 tokens, 16/4 heads of 128).  bfloat16 has the exponents of 32-bit floats.
constexpr int kRaised = 10;
template <typename T> constexpr bool kNarrow = std::is_same<T, __half>::value;
template <typename T> __host__ __device__ constexpr float raised() { return kNarrow<T> ? (float)(1 << kRaised) : 1.f; }
// The power of two by which ds is taken: 2 |dout| |v| times it is 2^15 at most, of 65504.
template <typename T>
__device__ __forceinline__ float ds_steps(const Lengths* lengths) {
    if constexpr (!kNarrow<T>) return 1.f;
    const float square = __uint_as_float(lengths->dout) * __uint_as_float(lengths->v);
    if (!(square > 0.f)) return 1.f;                                   // then ds is 0
    const int e = (int)(__float_as_uint(square) >> 23) - 127;          // square < 2^(e + 1), so the product of the lengths < 2^((e + 2) >> 1)
    return __uint_as_float((uint32_t)(14 - ((e + 2) >> 1) + 127) << 23);
}

struct AttentionParams {
    int sq, sk, head_dim, n_q, group, batch, causal, q_tiles, k_tiles, records;
    int section;                      // key heads whose tiles are done side by side
    float scale, scale2;              // scale2 = scale log2(e)
    const int32_t *doc_start, *lens;
    const char *q, *k, *v, *o_in, *dout;
    char *o, *dq, *dk, *dv;
    float* lse;
    Record* record;                   // [batch, n_q, records]
    Reach* reach;                     // [batch, records]
    Lengths* lengths;                 // [batch, key heads], for kNarrow types
    float* dout_square;               // [batch, n_q, records], for kNarrow types: of a record's queries
    int* fault;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3], dout_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];  // in elements
};

// The keys [lo, hi) that query i of batch row b sees; lo = INT_MAX, hi = 0 if none.
__device__ __forceinline__ void seen_by(const AttentionParams& P, int b, int i, int& lo, int& hi) {
    lo = INT_MAX, hi = 0;
    if (i >= P.sq) return;
    const int t = i + P.sk - P.sq;
    int n = P.sk;
    if (P.lens) n = min(max(P.lens[b], 0), P.sk);
    if (t >= n) return;
    const int h = P.causal ? min(n, t + 1) : n;
    const int l = P.doc_start ? max(P.doc_start[(int64_t)b * P.sq + i], 0) : 0;
    if (l < h) lo = l, hi = h;
}

// Which tile of which head a CTA takes.  CTAs are numbered so that the longest come first where the mask is causal, and so that the
// heads whose keys and values are being read at a time fit the L2 cache: sections of heads, within a section tile by tile.
struct Place { int tile, b, h; };
__device__ __forceinline__ Place place_of(const AttentionParams& P, int tiles, int heads_per_batch, int section, bool last_first) {
    const int heads = P.batch * heads_per_batch, whole = section * tiles, sec = blockIdx.x / whole, at = blockIdx.x - sec * whole;
    const int here = min(section, heads - sec * section), rank = at / here, bh = sec * section + at - rank * here, b = bh / heads_per_batch;
    return Place{last_first ? tiles - 1 - rank : rank, b, bh - b * heads_per_batch};
}

template <typename T>
__device__ __forceinline__ void store_row(char* base, int64_t at, int head_dim, const uint32_t* words, int first) {
    // `words`: 16 packed pairs, elements first .. first + 32 of the row at element `at`
    T* row = reinterpret_cast<T*>(base) + at;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (first + 8 * i < head_dim)
            *reinterpret_cast<uint4*>(row + first + 8 * i) = make_uint4(words[4 * i], words[4 * i + 1], words[4 * i + 2], words[4 * i + 3]);
}

// Zeroes rows of a tile in shared memory (the bulk copy's layout) that nobody sees: their probabilities are zero, but
// zero times what may lie there need not be.  `threads` threads, thread `at`.
template <int DP>
__device__ __forceinline__ void clear_row(char* tile, int rows, int row) {
#pragma unroll
    for (int sub = 0; sub < DP / 64; ++sub)
#pragma unroll
        for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(tile + sub * rows * 128 + row * 128 + c * 16) = make_uint4(0, 0, 0, 0);
}

// ------------------------------------------------------------------------------------------------ forward

// Two CTAs to an SM, each with half of its tensor memory: beside O there is room for S of 64 keys three times (heads of 64) or
// twice (of 128).  The products run that far ahead, so that the softmax, which is what bounds this kernel (16
// exponentials per clock), finds its next S done.  P lies over its S.
template <int DP> struct Forward {
    static constexpr int kRing = DP == 64 ? 3 : 2;
    static constexpr int kStages = DP == 64 ? 4 : 2;
    static constexpr int kTileQ = 128 * DP * 2, kTileK = 64 * DP * 2;
    static constexpr int kSmem = 1024 + kTileQ + 2 * kStages * kTileK;
    static constexpr int kColO = 64 * kRing, kColumns = 256;
    static constexpr int kThreads = 192;
    static_assert(kColO + DP <= kColumns, "tensor memory");
};

template <typename T, int DP>
__global__ void __launch_bounds__(192, 2)
attention_fwd_kernel(const __grid_constant__ AttentionParams P, const __grid_constant__ CUtensorMap map_q,
                     const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using F = Forward<DP>;
    extern __shared__ char smem_raw[];
    char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    char* tile_q = smem;
    char* tile_k = smem + F::kTileQ;
    char* tile_v = tile_k + F::kStages * F::kTileK;
    __shared__ uint64_t bars[2 + 3 * F::kRing + 4 * F::kStages];
    __shared__ uint32_t s_tmem;
    __shared__ int s_gave_up, s_lo[4], s_hi[4];
    const uint32_t q_full = smem_u32(bars), left = q_full + 8, s_full = q_full + 16, p_full = s_full + 8 * F::kRing, pv_done = p_full + 8 * F::kRing;
    const uint32_t k_full = pv_done + 8 * F::kRing, v_full = k_full + 8 * F::kStages, k_free = v_full + 8 * F::kStages, v_free = k_free + 8 * F::kStages;
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;

    const Place place = place_of(P, P.q_tiles, P.n_q, P.section * P.group, P.causal);
    const int tile = place.tile, b = place.b, h = place.h, hk = h / P.group;

    if (threadIdx.x == 0) {
        bar_init(q_full, 1), bar_init(left, 1);
        for (int r = 0; r < F::kRing; ++r) bar_init(s_full + 8 * r, 1), bar_init(p_full + 8 * r, 128), bar_init(pv_done + 8 * r, 1);
        for (int s = 0; s < F::kStages; ++s) bar_init(k_full + 8 * s, 1), bar_init(v_full + 8 * s, 1), bar_init(k_free + 8 * s, 1), bar_init(v_free + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_gave_up = 0;
    }
    if (warp == 4) tmem_alloc<F::kColumns>(smem_u32(&s_tmem));
    int lo = INT_MAX, hi = 0;
    if (warp < 4) {
        seen_by(P, b, tile * 128 + threadIdx.x, lo, hi);
        int l = lo, g = hi;
#pragma unroll
        for (int o = 16; o; o >>= 1) l = min(l, __shfl_xor_sync(~0u, l, o)), g = max(g, __shfl_xor_sync(~0u, g, o));
        if (lane == 0) s_lo[warp] = l, s_hi[warp] = g;
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = uniform(s_tmem);
    const int min_lo = min(min(s_lo[0], s_lo[1]), min(s_lo[2], s_lo[3])), max_hi = max(max(s_hi[0], s_hi[1]), max(s_hi[2], s_hi[3]));
    const int first = uniform(max_hi ? min_lo / 64 : 0), n = uniform(max_hi ? (max_hi + 63) / 64 - first : 0);
    const Waits W{&s_gave_up, P.fault};

    if (warp == 5) {
        if (n) {
            const bool issuer = elected();
            const auto load = [&](const CUtensorMap* map, uint32_t tile_at, uint32_t bar, int row, int head, int rows) {
                if (!issuer) return;
                bar_expect(bar, rows * DP * 2);
                for (int d = 0; d < DP / 64; ++d) tma_load(tile_at + d * rows * 128, map, bar, d * 64, row, head, b);
            };
            load(&map_q, smem_u32(tile_q), q_full, tile * 128, h, 128);
            for (int j = 0, s = 0, use = 1; j < n; ++j) {
                if (j >= F::kStages) W.wait_warp(k_free + 8 * s, use);
                load(&map_k, smem_u32(tile_k) + s * F::kTileK, k_full + 8 * s, (first + j) * 64, hk, 64);
                if (j >= F::kStages) W.wait_warp(v_free + 8 * s, use);
                load(&map_v, smem_u32(tile_v) + s * F::kTileK, v_full + 8 * s, (first + j) * 64, hk, 64);
                if (++s == F::kStages) s = 0, use ^= 1;
            }
            if (*W.gave_up) {
                W.drain(q_full, 0);
                for (int j = max(0, n - F::kStages); j < n; ++j) W.drain(k_full + 8 * (j % F::kStages), (j / F::kStages) & 1), W.drain(v_full + 8 * (j % F::kStages), (j / F::kStages) & 1);
            }
        }
    } else if (warp == 4) {
        if (n) {
            const bool issuer = elected();
            int ks = 0, k_use = 0, vs = 0, v_use = 0, r = 0, use = 0;  // stage, place in the ring, and how often they came round
            const auto scores = [&](int place) {
                W.wait_warp(k_full + 8 * ks, k_use);
                tc_after_sync();
                if (issuer) {
                    product_ss<T, 64, DP, 128, 64>(tmem + 64 * place, smem_u32(tile_q), smem_u32(tile_k) + ks * F::kTileK);
                    mma_commit(s_full + 8 * place);
                    mma_commit(k_free + 8 * ks);
                }
                if (++ks == F::kStages) ks = 0, k_use ^= 1;
            };
            W.wait_warp(q_full, 0);
            for (int j = 0; j < F::kRing && j < n; ++j) scores(j);
            for (int j = 0; j < n; ++j) {
                W.wait_warp(v_full + 8 * vs, v_use);
                W.wait_warp(p_full + 8 * r, use);
                tc_after_sync();
                if (issuer) {
                    product_ts<T, DP, 64, 16>(tmem + F::kColO, tmem + 64 * r, smem_u32(tile_v) + vs * F::kTileK, j > 0);
                    mma_commit(pv_done + 8 * r);
                    mma_commit(v_free + 8 * vs);
                }
                if (j + F::kRing < n) scores(r);
                if (++vs == F::kStages) vs = 0, v_use ^= 1;
                if (++r == F::kRing) r = 0, use ^= 1;
            }
            if (*W.gave_up) {
                if (issuer) mma_commit(left);
                W.drain(left, 0);
            }
        }
    } else {
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        const int i = tile * 128 + threadIdx.x;
        const float2 factor = both(P.scale2);
        float m = -INFINITY, l = 0.f;  // m: of the scores before they are scaled
        int r = 0, use = 0, before = 0, before_use = 0;
        uint32_t x[64];
        // Probabilities are exp2((x - shift) scale2 - base). Up to kNear shift is 0, which costs one instruction less for each; beyond, the difference
        // comes before the factor and is exact where it matters, so that no exponent is above 0 once the maximum has moved.
        const auto reference = [&](float top, float& shift, float& base) {
            const float scaled = top * P.scale2;
            const bool near = fabsf(scaled) <= kNear;
            base = near ? scaled : 0.f, shift = near || top == -INFINITY ? 0.f : top;
        };
        const auto fetch = [&](uint32_t* to, int from) {
            tmem_load32(to, lanes + 64 * from);
            tmem_load32(to + 32, lanes + 64 * from + 32);
        };
        for (int j = 0; j < n; ++j) {
            const int key0 = (first + j) * 64;
            W.wait_warp(s_full + 8 * r, use);
            tc_after_sync();
            fetch(x, r);
            tmem_wait_loads32(x);
            tmem_hold32(x + 32);
            if (!__all_sync(~0u, lo <= key0 && hi >= key0 + 64)) {
#pragma unroll
                for (int c = 0; c < 64; ++c)
                    if (key0 + c < lo || key0 + c >= hi) x[c] = 0xff800000u;
            }
            // The maximum is not looked for as long as the probabilities stay small without: it was right for the first keys,
            // and where later ones are much larger the sum shows it.  Once to a tile: what comes after a move is added up as it is.
            float2 minus = both(-(m * P.scale2));
            const auto move_maximum = [&] {
                float tops[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) tops[c] = __uint_as_float(x[c]);
#pragma unroll
                for (int c = 4; c < 64; ++c) tops[c & 3] = fmaxf(tops[c & 3], __uint_as_float(x[c]));
                const float to = fmaxf(m, fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
                float old_shift, old_base, shift, base;
                reference(m, old_shift, old_base), reference(to, shift, base);
                const float f = m == -INFINITY ? 0.f : fast_exp2(fmaf(old_shift - shift, P.scale2, old_base - base));
                m = to, minus = both(-base);
                l *= f;
                if (__any_sync(~0u, shift != 0.f)) {
#pragma unroll
                    for (int c = 0; c < 64; ++c) x[c] = __float_as_uint(__uint_as_float(x[c]) - shift);
                }
                if (j) {  // every product so far is in O
                    W.wait_warp(pv_done + 8 * before, before_use);
                    tc_after_sync();
#pragma unroll
                    for (int c = 0; c < DP / 16; ++c) {
                        uint32_t o[16];
                        tmem_load16(o, lanes + F::kColO + 16 * c);
                        tmem_wait_loads16(o);
#pragma unroll
                        for (int q = 0; q < 16; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * f);
                        tmem_store16(lanes + F::kColO + 16 * c, o);
                    }
                    tmem_wait_stores();
                }
            };
            bool moved = __any_sync(~0u, !(fabsf(m * P.scale2) <= kNear));  // none yet, or beyond: always looked for
            if (moved) move_maximum();
            float sum;
            for (;;) {  // twice at most
                float2 sums[2] = {both(0.f), both(0.f)};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t words[16];
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        const float2 p = exp2_both(fma2(make_float2(__uint_as_float(x[32 * c + 2 * q]), __uint_as_float(x[32 * c + 2 * q + 1])), factor, minus));
                        sums[q & 1] = add2(sums[q & 1], p);
                        words[q] = pack2<T>(p.x, p.y);
                    }
                    tmem_store16(lanes + 64 * r + 16 * c, words);
                }
                const float2 pair = add2(sums[0], sums[1]);
                sum = pair.x + pair.y;
                if (moved || !__any_sync(~0u, sum > kMostSum)) break;
                moved = true;
                tmem_wait_stores();  // before the same places are written again
                move_maximum();
            }
            l += sum;
            if (key0 < min_lo || (key0 + 64 > max_hi && max_hi < P.sk)) {
                const int s = j % F::kStages, key = key0 + threadIdx.x;
                W.wait_warp(v_full + 8 * s, (j / F::kStages) & 1);
                if (threadIdx.x < 64 && (key < min_lo || key >= max_hi)) clear_row<DP>(tile_v + s * F::kTileK, 64, threadIdx.x);
                fence_async_shared();
            }
            tmem_wait_stores();
            tc_before_sync();
            bar_arrive(p_full + 8 * r);
            before = r, before_use = use;
            if (++r == F::kRing) r = 0, use ^= 1;
        }
        if (n) {
            W.wait_warp(pv_done + 8 * before, before_use);
            tc_after_sync();
        }
        {
            const float inv = l > 0.f ? 1.f / l : l;  // a NaN stays one
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                uint32_t o[32];
                if (n) {
                    tmem_load32(o, lanes + F::kColO + 32 * c);
                    tmem_wait_loads32(o);
                }
                if (i < P.sq) {
                    const bool none = hi == 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        o[e] = none ? 0u : pack2<T>(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
                    store_row<T>(P.o, b * P.o_stride[0] + i * P.o_stride[1] + h * P.o_stride[2], P.head_dim, o, 32 * c);
                }
            }
            float shift, base;
            reference(m, shift, base);
            if (i < P.sq) P.lse[((int64_t)b * P.n_q + h) * P.sq + i] = hi == 0 ? -INFINITY : (fmaf(shift, P.scale2, base) + log2f(l)) * kLn2;
        }
    }
    tc_before_sync();
    __syncthreads();
    if (warp == 4) tmem_free<F::kColumns>(tmem);
}

// ------------------------------------------------------------------------------------------------ backward

template <typename T>
__device__ __forceinline__ const T* row_of(const char* base, const int64_t* stride, int b, int64_t s, int h) {
    return reinterpret_cast<const T*>(base) + b * stride[0] + s * stride[1] + h * stride[2];
}

template <typename T>
__device__ __forceinline__ float dot8(uint4 a, uint4 b, float sum) {
    const uint32_t as[4] = {a.x, a.y, a.z, a.w}, bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 p = unpack2<T>(as[e]), q = unpack2<T>(bs[e]);
        sum = fmaf(p.x, q.x, fmaf(p.y, q.y, sum));
    }
    return sum;
}
template <typename T>
__device__ __forceinline__ float dot(const T* x, const T* y, int head_dim) {
    float sum = 0.f;
#pragma unroll 4
    for (int c = 0; c < head_dim; c += 8) sum = dot8<T>(*reinterpret_cast<const uint4*>(x + c), *reinterpret_cast<const uint4*>(y + c), sum);
    return sum;
}
// D = dout . o is off by the rounding of o to 16 bits, and ds = p (dp - D) by as much whatever its own size.  Against the sum over
// many keys that is little; a query with few keys, whose dp and D nearly cancel, would lose half of its digits to it.
// Its D is formed from sum p dp instead, in 32 bits.
constexpr int kFewKeys = 16;

// Records of 64 queries of a head, and once per batch row their reach.  Four threads to a query: with eight most instructions were
// addresses, with one the loads of a warp lay too far apart.
template <typename T>
__global__ void __launch_bounds__(4 * kRecord) attention_record_kernel(const __grid_constant__ AttentionParams P) {
    const int rec = blockIdx.x, h = blockIdx.y, b = blockIdx.z, r = threadIdx.x >> 2, part = threadIdx.x & 3, i = rec * kRecord + r;
    Record* R = P.record + ((int64_t)b * P.n_q + h) * P.records + rec;
    __shared__ Reach s_reach[8];
    __shared__ int s_lo[kRecord], s_hi[kRecord];
    __shared__ float s_lse2[kRecord], s_term[kRecord][kFewKeys + 1], s_square[8];
    float delta = 0.f, lse2 = 0.f, square = 0.f;
    if (i < P.sq) {  // rows that see nothing are read too; what comes of it is not used
        const T* o = row_of<T>(P.o_in, P.o_stride, b, i, h) + 8 * part;
        const T* d = row_of<T>(P.dout, P.dout_stride, b, i, h) + 8 * part;
        uint4 x[4], y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (8 * part + 32 * c < P.head_dim) x[c] = *reinterpret_cast<const uint4*>(o + 32 * c), y[c] = *reinterpret_cast<const uint4*>(d + 32 * c);
        lse2 = P.lse[((int64_t)b * P.n_q + h) * P.sq + i] * kLog2e;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (8 * part + 32 * c < P.head_dim) {
                delta = dot8<T>(x[c], y[c], delta);
                if (kNarrow<T>) square = dot8<T>(y[c], y[c], square);
            }
    }
    delta += __shfl_xor_sync(~0u, delta, 1);
    delta += __shfl_xor_sync(~0u, delta, 2);
    int lo, hi;
    seen_by(P, b, i, lo, hi);
    if constexpr (kNarrow<T>) {
        square += __shfl_xor_sync(~0u, square, 1);
        square += __shfl_xor_sync(~0u, square, 2);
        if (hi == 0) square = 0.f;
#pragma unroll
        for (int o = 16; o >= 4; o >>= 1) square = fmaxf(square, __shfl_xor_sync(~0u, square, o));
        if ((threadIdx.x & 31) == 0) s_square[threadIdx.x >> 5] = square;
    }
    // The queries with few keys, a thread to a query and a key; the terms are added in the order of the keys.
    const bool few = hi && hi - lo <= kFewKeys;
    if (part == 0) s_lse2[r] = lse2, s_lo[r] = lo, s_hi[r] = few ? hi : 0;
    if (__syncthreads_or(few)) {
        for (int p = threadIdx.x; p < kRecord * kFewKeys; p += 4 * kRecord) {
            const int q = p / kFewKeys, k = p % kFewKeys, query = rec * kRecord + q;
            if (s_lo[q] + k < s_hi[q] && s_hi[q]) {
                const int j = s_lo[q] + k;
                const float s = dot<T>(row_of<T>(P.q, P.q_stride, b, query, h), row_of<T>(P.k, P.k_stride, b, j, h / P.group), P.head_dim);
                const float dp = dot<T>(row_of<T>(P.dout, P.dout_stride, b, query, h), row_of<T>(P.v, P.v_stride, b, j, h / P.group), P.head_dim);
                s_term[q][k] = fast_exp2(fmaf(s, P.scale2, -s_lse2[q])) * dp;
            }
        }
        __syncthreads();
        if (few) {
            delta = 0.f;
            for (int k = 0; k < hi - lo; ++k) delta += s_term[r][k];
        }
    }
    if (part == 0) {
        R->minus_lse2[r] = hi ? (kNarrow<T> ? kRaised - lse2 : -lse2) : -INFINITY;
        R->minus_delta[r] = hi ? -delta : 0.f;
        R->lo[r] = lo;
        R->hi[r] = hi;
    }
    if (kNarrow<T> && threadIdx.x == 0) {  // written before the barrier that all threads have gone through
        for (int w = 1; w < 8; ++w) square = fmaxf(square, s_square[w]);
        P.dout_square[((int64_t)b * P.n_q + h) * P.records + rec] = square;
        if (rec == 0 && h % P.group == 0) P.lengths[(int64_t)b * (P.n_q / P.group) + h / P.group] = Lengths{0, 0};
    }
    if (h == 0) {
        Reach a{INT_MAX, 0, 0, INT_MAX};
        if (i < P.sq) a = Reach{lo, hi, lo, hi};  // rows past the end are zeros and need no mask
#pragma unroll
        for (int s = 16; s >= 4; s >>= 1) {
            a.min_lo = min(a.min_lo, __shfl_xor_sync(~0u, a.min_lo, s));
            a.max_hi = max(a.max_hi, __shfl_xor_sync(~0u, a.max_hi, s));
            a.max_lo = max(a.max_lo, __shfl_xor_sync(~0u, a.max_lo, s));
            a.min_hi = min(a.min_hi, __shfl_xor_sync(~0u, a.min_hi, s));
        }
        if ((threadIdx.x & 31) == 0) s_reach[threadIdx.x >> 5] = a;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 8; ++w) {
                const Reach c = s_reach[w];
                a = Reach{min(a.min_lo, c.min_lo), max(a.max_hi, c.max_hi), max(a.max_lo, c.max_lo), min(a.min_hi, c.min_hi)};
            }
            P.reach[(int64_t)b * P.records + rec] = a;
        }
    }
}

// The lengths that ds_steps goes by: a block takes its share of a key head's keys, eight threads to a key, and of its heads' records.  The
// first keys are under way while the block finds out which of them some query sees.
constexpr int kLengthsThreads = 256, kLengthsKeys = kLengthsThreads / 8, kLengthsAhead = 4;
template <typename T>
__global__ void __launch_bounds__(kLengthsThreads) attention_lengths_kernel(const __grid_constant__ AttentionParams P) {
    const int hk = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31, part = threadIdx.x & 7;
    __shared__ int s_lo, s_hi;
    __shared__ uint32_t s_v, s_d;
    if (threadIdx.x == 0) s_lo = INT_MAX, s_hi = 0, s_v = s_d = 0;
    __syncthreads();
    float v = 0.f, d = 0.f;
    bool known = false;
    const int64_t apart = (int64_t)gridDim.x * kLengthsKeys;
    for (int64_t first = (int64_t)blockIdx.x * kLengthsKeys + (threadIdx.x >> 3), done = 0; done < P.sk; done += apart * kLengthsAhead, first += apart * kLengthsAhead) {
        uint4 w[kLengthsAhead][2];
#pragma unroll
        for (int u = 0; u < kLengthsAhead; ++u)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int64_t j = first + u * apart;
                w[u][c] = make_uint4(0, 0, 0, 0);
                if (j < P.sk && 8 * part + 64 * c < P.head_dim) w[u][c] = *reinterpret_cast<const uint4*>(row_of<T>(P.v, P.v_stride, b, j, hk) + 8 * part + 64 * c);
            }
        if (!known) {
            int lo = INT_MAX, hi = 0;
            for (int r = threadIdx.x; r < P.records; r += kLengthsThreads) {
                const Reach a = P.reach[(int64_t)b * P.records + r];
                lo = min(lo, a.min_lo), hi = max(hi, a.max_hi);
            }
            if (hi) atomicMin(&s_lo, lo), atomicMax(&s_hi, hi);
            __syncthreads();
            known = true;
        }
#pragma unroll
        for (int u = 0; u < kLengthsAhead; ++u) {
            const int64_t j = first + u * apart;
            float square = dot8<T>(w[u][1], w[u][1], dot8<T>(w[u][0], w[u][0], 0.f));
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) square += __shfl_xor_sync(~0u, square, o);
            if (j >= s_lo && j < s_hi) v = fmaxf(v, square);
        }
    }
    for (int64_t r = (int64_t)blockIdx.x * kLengthsThreads + threadIdx.x; r < (int64_t)P.group * P.records; r += (int64_t)gridDim.x * kLengthsThreads)
        d = fmaxf(d, P.dout_square[((int64_t)b * P.n_q + hk * P.group) * P.records + r]);
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o)), d = fmaxf(d, __shfl_xor_sync(~0u, d, o));
    if (lane == 0) atomicMax(&s_v, __float_as_uint(v)), atomicMax(&s_d, __float_as_uint(d));
    __syncthreads();
    if (threadIdx.x == 0) {  // a maximum does not depend on the order
        Lengths& L = P.lengths[(int64_t)b * (P.n_q / P.group) + hk];
        atomicMax(&L.v, s_v), atomicMax(&L.dout, s_d);
    }
}

// dK and dV of 128 keys.  kSlots sets of 8 warps take the query tiles in turn, each with its own S^T and dP^T; four warps of a set take the
// first 32 queries, four the others.
template <int DP, int kSlots> struct Keys {
    static constexpr int kTileK = 128 * DP * 2, kTileQ = 64 * DP * 2;
    static constexpr int kStages = 3;
    static constexpr int kStageBytes = 2 * kTileQ + 1024;
    static constexpr int kSmem = 1024 + 2 * kTileK + kStages * kStageBytes;
    static constexpr int kColDV = kSlots * 128, kColDK = kColDV + DP, kColumns = kColDK + DP <= 256 ? 256 : 512;
    static constexpr int kThreads = kSlots * 256 + 64;
    static constexpr int kPerSM = kColumns == 256 ? 2 : 1;
    static_assert(kColDK + DP <= 512, "tensor memory");
};

template <typename T, int DP, int kSlots>
__global__ void __launch_bounds__(Keys<DP, kSlots>::kThreads, Keys<DP, kSlots>::kPerSM)
attention_keys_kernel(const __grid_constant__ AttentionParams P, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do) {
    using F = Keys<DP, kSlots>;
    extern __shared__ char smem_raw[];
    char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    char* tile_k = smem;
    char* tile_v = smem + F::kTileK;
    char* stages = smem + 2 * F::kTileK;  // each: Q, dO, record
    __shared__ uint64_t bars[2 + 2 * F::kStages + 4 * kSlots];
    __shared__ uint32_t s_tmem;
    __shared__ int s_gave_up, s_first, s_end;
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t kv_full = bar0, done = bar0 + 8, full = bar0 + 16, free_ = full + 8 * F::kStages, s_full = free_ + 8 * F::kStages, ds_full = s_full + 8 * kSlots,
                   dp_full = ds_full + 8 * kSlots, s_read = dp_full + 8 * kSlots;
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    constexpr int kCopyWarp = 8 * kSlots, kMmaWarp = kCopyWarp + 1;

    const Place place = place_of(P, P.k_tiles, P.n_q / P.group, P.section, false);  // under a causal mask the first keys have the most queries
    const int tile = place.tile, b = place.b, hk = place.h;
    const int key0 = tile * 128;

    if (threadIdx.x == 0) {
        bar_init(kv_full, 1), bar_init(done, 1);
        for (int s = 0; s < F::kStages; ++s) bar_init(full + 8 * s, 1), bar_init(free_ + 8 * s, 1);
        for (int s = 0; s < kSlots; ++s) bar_init(s_full + 8 * s, 1), bar_init(ds_full + 8 * s, 256), bar_init(dp_full + 8 * s, 1), bar_init(s_read + 8 * s, 256);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_gave_up = 0, s_first = INT_MAX, s_end = 0;
    }
    if (warp == kMmaWarp) tmem_alloc<F::kColumns>(smem_u32(&s_tmem));
    __syncthreads();
    const Reach* reach = P.reach + (int64_t)b * P.records;
    int begin = INT_MAX, end = 0;
    for (int r = threadIdx.x; r < P.records; r += F::kThreads) {
        const Reach a = reach[r];
        if (a.min_lo < key0 + 128 && a.max_hi > key0) begin = min(begin, r), end = max(end, r + 1);
    }
    if (end) atomicMin(&s_first, begin), atomicMax(&s_end, end);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = uniform(s_tmem);
    const int first = uniform(s_first), per_head = uniform(s_end ? s_end - first : 0), n = per_head * P.group;
    const Waits W{&s_gave_up, P.fault};

    if (warp == kCopyWarp) {
        if (n) {
            const bool issuer = elected();
            if (issuer) {
                bar_expect(kv_full, 2 * F::kTileK);
                for (int d = 0; d < DP / 64; ++d) {
                    tma_load(smem_u32(tile_k) + d * 128 * 128, &map_k, kv_full, d * 64, key0, hk, b);
                    tma_load(smem_u32(tile_v) + d * 128 * 128, &map_v, kv_full, d * 64, key0, hk, b);
                }
            }
            int it = 0, s = 0, use = 1, r = 0, h = hk * P.group;
            const Record* records = P.record + ((int64_t)b * P.n_q + h) * P.records + first;
            for (; it < n; ++it) {
                if (it >= F::kStages) W.wait_warp(free_ + 8 * s, use);
                if (issuer) {
                    const uint32_t at = smem_u32(stages) + s * F::kStageBytes, bar = full + 8 * s;
                    bar_expect(bar, F::kStageBytes);
                    for (int d = 0; d < DP / 64; ++d) {
                        tma_load(at + d * 64 * 128, &map_q, bar, d * 64, (first + r) * 64, h, b);
                        tma_load(at + F::kTileQ + d * 64 * 128, &map_do, bar, d * 64, (first + r) * 64, h, b);
                    }
                    bulk_load(at + 2 * F::kTileQ, records + r, 1024, bar);
                }
                if (++s == F::kStages) s = 0, use ^= 1;
                if (++r == per_head) r = 0, ++h, records += P.records;
            }
            if (*W.gave_up) {
                W.drain(kv_full, 0);
                for (int i = max(0, n - F::kStages); i < n; ++i) W.drain(full + 8 * (i % F::kStages), (i / F::kStages) & 1);
            }
        }
    } else if (warp == kMmaWarp) {
        if (n) {
            const bool issuer = elected();
            // stages of the tile whose scores come next, whose dP comes next, and which is being used up
            int s1 = 0, use1 = 0, s2 = 0, s3 = 0, slot = 0, use = 0;
            const auto tile_at = [&](int s) { return smem_u32(stages) + s * F::kStageBytes; };
            const auto next = [](int& s) { s = s + 1 == F::kStages ? 0 : s + 1; };
            const auto scores = [&](int slot) {
                W.wait_warp(full + 8 * s1, use1);
                tc_after_sync();
                if (issuer) {
                    product_ss<T, 64, DP, 128, 64>(tmem + slot * 128, smem_u32(tile_k), tile_at(s1));
                    mma_commit(s_full + 8 * slot);
                }
                next(s1);
                use1 ^= s1 == 0;
            };
            const auto dp = [&](int slot) {
                if (issuer) {
                    product_ss<T, 64, DP, 128, 64>(tmem + slot * 128 + 64, smem_u32(tile_v), tile_at(s2) + F::kTileQ);
                    mma_commit(dp_full + 8 * slot);
                }
                next(s2);
            };
            W.wait_warp(kv_full, 0);
            for (int it = 0; it < kSlots && it < n; ++it) scores(it), dp(it);
            for (int it = 0; it < n; ++it) {
                // S of the next tile in this slot can follow once this one has been read; dP only when P and dS, which lie over it, are used up
                if (it + kSlots < n) {
                    W.wait_warp(s_read + 8 * slot, use);
                    scores(slot);
                }
                W.wait_warp(ds_full + 8 * slot, use);
                tc_after_sync();
                if (issuer) {
                    const uint32_t q = tile_at(s3), at = tmem + slot * 128 + 64;
                    product_ts<T, DP, 64, 32>(tmem + F::kColDV, at, q + F::kTileQ, it > 0);
                    product_ts<T, DP, 64, 32>(tmem + F::kColDK, at + 16, q, it > 0);
                    mma_commit(free_ + 8 * s3);
                }
                next(s3);
                if (it + kSlots < n) dp(slot);
                if (++slot == kSlots) slot = 0, use ^= 1;
            }
            if (issuer) mma_commit(done);
            if (*W.gave_up) W.drain(done, 0);
        }
    } else {
        const int slot = warp >> 3, part = (warp >> 2) & 1, row = threadIdx.x & 127, key = key0 + row;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), at = lanes + slot * 128 + part * 32;
        int s = slot % F::kStages, use = slot / F::kStages, s_use = 0, rec = per_head ? slot % per_head : 0;
        const float steps = n ? ds_steps<T>(P.lengths + (int64_t)b * (P.n_q / P.group) + hk) : 1.f;
        const float2 step = both(steps / raised<T>());
        for (int it = slot; it < n; it += kSlots) {
            const Reach a = reach[first + rec];
            W.wait(full + 8 * s, use);
            W.wait_warp(s_full + 8 * slot, s_use);
            tc_after_sync();
            char* stage = stages + s * F::kStageBytes;
            const Record& R = *reinterpret_cast<const Record*>(stage + 2 * F::kTileQ);
            // A thread takes 4 keys by 8 queries: what belongs to a query is then read from shared memory for four keys at once, and shared
            // memory, which the products read their operands from, is what this loop runs short of.
            uint32_t x[32], y[32];
            tmem_load_16x32(x, at);
            tmem_load_16x32(x + 16, at + (16 << 16));
            tmem_wait_loads32(x);
            tc_before_sync();
            bar_arrive(s_read + 8 * slot);
            const int column = part * 32 + 2 * (lane & 3), key_of_lane = key0 + (warp & 3) * 32 + (lane >> 2);
            const bool masked = a.max_lo > key0 || a.min_hi < key0 + 128;
            const float2 factor = both(P.scale2);
            // P first, while the product dP may still be under way
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 ml = *reinterpret_cast<const float2*>(R.minus_lse2 + column + 8 * k);
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // keys key_of_lane + 8 i
                    uint32_t* e = x + 16 * (i >> 1) + 4 * k + 2 * (i & 1);
                    const float2 p = exp2_both(fma2(make_float2(__uint_as_float(e[0]), __uint_as_float(e[1])), factor, ml));
                    e[0] = __float_as_uint(p.x), e[1] = __float_as_uint(p.y);
                }
            }
            W.wait_warp(dp_full + 8 * slot, s_use);
            tc_after_sync();
            tmem_load_16x32(y, at + 64);
            tmem_load_16x32(y + 16, at + 64 + (16 << 16));
            tmem_wait_loads32(y);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float2 md = *reinterpret_cast<const float2*>(R.minus_delta + column + 8 * k);
                if (kNarrow<T>) md = mul2(md, step);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at_e = 16 * (i >> 1) + 4 * k + 2 * (i & 1);
                    const float2 dp = make_float2(__uint_as_float(y[at_e]), __uint_as_float(y[at_e + 1]));
                    const float2 ds = mul2(make_float2(__uint_as_float(x[at_e]), __uint_as_float(x[at_e + 1])), kNarrow<T> ? fma2(dp, step, md) : add2(dp, md));
                    y[at_e] = __float_as_uint(ds.x), y[at_e + 1] = __float_as_uint(ds.y);
                }
            }
            if (masked) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int2 lo = *reinterpret_cast<const int2*>(R.lo + column + 8 * k), hi = *reinterpret_cast<const int2*>(R.hi + column + 8 * k);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at_e = 16 * (i >> 1) + 4 * k + 2 * (i & 1), key = key_of_lane + 8 * i;
                        const auto hide = [&](int l, int h, uint32_t& p, uint32_t& ds) {
                            if (key < l || key >= h) p = ds = 0;
                            if (h - l == 1) ds = 0;  // a softmax of one term is constant
                        };
                        hide(lo.x, hi.x, x[at_e], y[at_e]), hide(lo.y, hi.y, x[at_e + 1], y[at_e + 1]);
                    }
                }
            }
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                uint32_t words[16];  // 16 columns of P, then 16 of dS
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int at_e = 16 * hh + 4 * k + 2 * i;
                        words[2 * k + i] = pack2<T>(__uint_as_float(x[at_e]), __uint_as_float(x[at_e + 1]));
                        words[8 + 2 * k + i] = pack2<T>(__uint_as_float(y[at_e]), __uint_as_float(y[at_e + 1]));
                    }
                tmem_store_16x32(at + 64 + (hh * 16 << 16), words);
            }
            tmem_wait_stores();
            if (a.max_lo == INT_MAX && part == 0) {  // a query that sees nothing may hold anything
                if (row < 64 ? R.hi[row] == 0 : R.hi[row - 64] == 0) clear_row<DP>(stage + (row < 64 ? 0 : F::kTileQ), 64, row & 63);
                fence_async_shared();
            }
            tc_before_sync();
            bar_arrive(ds_full + 8 * slot);
            s_use ^= 1;
            for (int step = 0; step < kSlots; ++step) {
                if (++s == F::kStages) s = 0, use ^= 1;
                if (++rec == per_head) rec = 0;
            }
        }
        if (n) W.wait_warp(done, 0);
        tc_after_sync();
        if (slot == 0) {  // four warps store dV, four dK
            {
                const int what = part;
                const float f = what ? P.scale / steps : 1.f / raised<T>();
                const int64_t* st = what ? P.dk_stride : P.dv_stride;
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) {
                    uint32_t o[32];
                    if (n) {
                        tmem_load32(o, lanes + (what ? F::kColDK : F::kColDV) + 32 * c);
                        tmem_wait_loads32(o);
                    }
                    if (key < P.sk) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = n ? pack2<T>(__uint_as_float(o[2 * e]) * f, __uint_as_float(o[2 * e + 1]) * f) : 0u;
                        store_row<T>(what ? P.dk : P.dv, b * st[0] + key * st[1] + hk * st[2], P.head_dim, o, 32 * c);
                    }
                }
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_free<F::kColumns>(tmem);
}

// dQ of 128 queries, two CTAs to an SM, the keys 64 at a time; four warps take the first 32 keys of a tile, four the others.
// K of a tile is needed from S to dQ, V only for dP: heads of 128, whose tiles fill shared memory to the last KB, have two
// places for K and one for V.
template <int DP> struct Queries {
    static constexpr int kTileQ = 128 * DP * 2, kTileK = 64 * DP * 2;
    static constexpr int kDPs = DP == 64 ? 2 : 1;                 // places for dP, and dS over it, beside one for S
    static constexpr int kStagesK = DP == 64 ? 4 : 2, kStagesV = DP == 64 ? 4 : 1;
    static constexpr int kColDP = 64, kColDQ = 64 + 64 * kDPs, kColumns = 256;
    static constexpr int kThreads = 256 + 64;
    struct Control {
        uint64_t bars[4 + 2 * kDPs + 2 * kStagesK + 2 * kStagesV];
        uint32_t tmem;
        int gave_up, lo[4], hi[4];
    };
    static constexpr int kTiles = 2 * kTileQ + (kStagesK + kStagesV) * kTileK, kSmem = kTiles + sizeof(Control);
    static_assert(kColDQ + DP <= kColumns, "tensor memory");
    static_assert(2 * (kSmem + 1024) <= kSharedPerSM, "two CTAs to an SM");
};

template <typename T, int DP>
__global__ void __launch_bounds__(Queries<DP>::kThreads, 2)
attention_queries_kernel(const __grid_constant__ AttentionParams P, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                         const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do) {
    using F = Queries<DP>;
    extern __shared__ __align__(1024) char smem[];  // all of it dynamic, so that it begins where the tiles have to
    char* tile_q = smem;
    char* tile_do = smem + F::kTileQ;
    char* tiles_k = smem + 2 * F::kTileQ;
    char* tiles_v = tiles_k + F::kStagesK * F::kTileK;
    typename F::Control& C = *reinterpret_cast<typename F::Control*>(smem + F::kTiles);
    const uint32_t q_full = smem_u32(C.bars), done = q_full + 8, s_full = q_full + 16, s_read = q_full + 24, dp_full = q_full + 32, ds_full = dp_full + 8 * F::kDPs,
                   k_full = ds_full + 8 * F::kDPs, k_free = k_full + 8 * F::kStagesK, v_full = k_free + 8 * F::kStagesK, v_free = v_full + 8 * F::kStagesV;
    if (smem_u32(smem) & 1023) {  // then no tile would lie as its descriptors say
        if (threadIdx.x == 0) say_fault(P.fault);
        return;
    }
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    constexpr int kCopyWarp = 8, kMmaWarp = kCopyWarp + 1;
    const Place place = place_of(P, P.q_tiles, P.n_q, P.section * P.group, P.causal);
    const int tile = place.tile, b = place.b, h = place.h, hk = h / P.group;

    if (threadIdx.x == 0) {
        bar_init(q_full, 1), bar_init(done, 1);
        for (int s = 0; s < F::kStagesK; ++s) bar_init(k_full + 8 * s, 1), bar_init(k_free + 8 * s, 1);
        for (int s = 0; s < F::kStagesV; ++s) bar_init(v_full + 8 * s, 1), bar_init(v_free + 8 * s, 1);
        bar_init(s_full, 1), bar_init(s_read, 256);
        // A warp may be done with dS of a tile while another is still at the one before: each place has its own count.
        for (int s = 0; s < F::kDPs; ++s) bar_init(dp_full + 8 * s, 1), bar_init(ds_full + 8 * s, 256);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        C.gave_up = 0;
    }
    if (warp == kMmaWarp) tmem_alloc<F::kColumns>(smem_u32(&C.tmem));
    const int row = threadIdx.x & 127, i = tile * 128 + row;
    int lo = INT_MAX, hi = 0;
    float minus_lse2 = -INFINITY, minus_delta = 0.f;
    if (warp < 8) {
        if (i < P.sq) {
            const Record& R = P.record[((int64_t)b * P.n_q + h) * P.records + i / kRecord];
            minus_lse2 = R.minus_lse2[i % kRecord], minus_delta = R.minus_delta[i % kRecord], lo = R.lo[i % kRecord], hi = R.hi[i % kRecord];
        }
        int l = lo, g = hi;
#pragma unroll
        for (int o = 16; o; o >>= 1) l = min(l, __shfl_xor_sync(~0u, l, o)), g = max(g, __shfl_xor_sync(~0u, g, o));
        if (lane == 0 && warp < 4) C.lo[warp] = l, C.hi[warp] = g;
    }
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = uniform(C.tmem);
    const int min_lo = min(min(C.lo[0], C.lo[1]), min(C.lo[2], C.lo[3])), max_hi = max(max(C.hi[0], C.hi[1]), max(C.hi[2], C.hi[3]));
    const int first = uniform(max_hi ? min_lo / 64 : 0), n = uniform(max_hi ? (max_hi + 63) / 64 - first : 0);
    const Waits W{&C.gave_up, P.fault};

    if (warp == kCopyWarp) {
        if (n) {
            const bool issuer = elected();
            if (issuer) {
                bar_expect(q_full, 2 * F::kTileQ);
                for (int d = 0; d < DP / 64; ++d) {
                    tma_load(smem_u32(tile_q) + d * 128 * 128, &map_q, q_full, d * 64, tile * 128, h, b);
                    tma_load(smem_u32(tile_do) + d * 128 * 128, &map_do, q_full, d * 64, tile * 128, h, b);
                }
            }
            int s = 0, use = 1, sv = 0, use_v = 1;
            const auto load = [&](const CUtensorMap* map, uint32_t at, uint32_t bar, int row) {
                if (!issuer) return;
                bar_expect(bar, F::kTileK);
                for (int d = 0; d < DP / 64; ++d) tma_load(at + d * 64 * 128, map, bar, d * 64, row, hk, b);
            };
            for (int j = 0; j < n; ++j) {
                if (j >= F::kStagesK) W.wait_warp(k_free + 8 * s, use);
                load(&map_k, smem_u32(tiles_k) + s * F::kTileK, k_full + 8 * s, (first + j) * 64);
                if (j >= F::kStagesV) W.wait_warp(v_free + 8 * sv, use_v);
                load(&map_v, smem_u32(tiles_v) + sv * F::kTileK, v_full + 8 * sv, (first + j) * 64);
                if (++s == F::kStagesK) s = 0, use ^= 1;
                if (++sv == F::kStagesV) sv = 0, use_v ^= 1;
            }
            if (*W.gave_up) {
                W.drain(q_full, 0);
                for (int i = max(0, n - F::kStagesK); i < n; ++i) W.drain(k_full + 8 * (i % F::kStagesK), (i / F::kStagesK) & 1);
                for (int i = max(0, n - F::kStagesV); i < n; ++i) W.drain(v_full + 8 * (i % F::kStagesV), (i / F::kStagesV) & 1);
            }
        }
    } else if (warp == kMmaWarp) {
        if (n) {
            const bool issuer = elected();
            // places: of K whose scores come next, of V, of K being used up, of dP coming next, of dS being used up
            int s1 = 0, use1 = 0, s2 = 0, use2 = 0, s3 = 0, d2 = 0, d3 = 0;
            const auto next = [](int& s, int of) { s = s + 1 == of ? 0 : s + 1; };
            const auto scores = [&] {
                W.wait_warp(k_full + 8 * s1, use1);
                tc_after_sync();
                if (issuer) {
                    product_ss<T, 64, DP, 128, 64>(tmem, smem_u32(tile_q), smem_u32(tiles_k) + s1 * F::kTileK);
                    mma_commit(s_full);
                }
                next(s1, F::kStagesK);
                use1 ^= s1 == 0;
            };
            const auto dp = [&] {
                W.wait_warp(v_full + 8 * s2, use2);
                tc_after_sync();
                if (issuer) {
                    product_ss<T, 64, DP, 128, 64>(tmem + F::kColDP + d2 * 64, smem_u32(tile_do), smem_u32(tiles_v) + s2 * F::kTileK);
                    mma_commit(dp_full + 8 * d2);
                    mma_commit(v_free + 8 * s2);
                }
                next(s2, F::kStagesV), next(d2, F::kDPs);
                use2 ^= s2 == 0;
            };
            W.wait_warp(q_full, 0);
            scores(), dp();
            for (int j = 0; j < n; ++j) {
                // the next S can follow once this one has been read, the next dP too where it has a place of its own
                if (j + 1 < n) {
                    W.wait_warp(s_read, j & 1);
                    scores();
                    if (F::kDPs > 1) dp();
                }
                W.wait_warp(ds_full + 8 * d3, (j / F::kDPs) & 1);
                tc_after_sync();
                if (issuer) {
                    product_ts<T, DP, 64, 32>(tmem + F::kColDQ, tmem + F::kColDP + d3 * 64, smem_u32(tiles_k) + s3 * F::kTileK, j > 0);
                    mma_commit(k_free + 8 * s3);
                }
                next(s3, F::kStagesK), next(d3, F::kDPs);
                if (F::kDPs == 1 && j + 1 < n) dp();
            }
            if (issuer) mma_commit(done);
            if (*W.gave_up) W.drain(done, 0);
        }
    } else {
        const int part = (warp >> 2) & 1;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float steps = n ? ds_steps<T>(P.lengths + (int64_t)b * (P.n_q / P.group) + hk) : 1.f;
        const float2 factor = both(P.scale2), ml = both(minus_lse2), step = both(steps / raised<T>()), md = both(minus_delta * step.x);
        const bool one = hi - lo == 1;  // a softmax of one term is constant
        for (int j = 0; j < n; ++j) {
            const int s = j % F::kStagesK, tile0 = (first + j) * 64, key0 = tile0 + part * 32;
            const uint32_t at_dp = lanes + F::kColDP + (j % F::kDPs) * 64 + part * 32;
            W.wait_warp(s_full, j & 1);
            tc_after_sync();
            uint32_t x[32], y[32];
            tmem_load32(x, lanes + part * 32);
            tmem_wait_loads32(x);
            tc_before_sync();
            bar_arrive(s_read);
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
                const float2 p = exp2_both(fma2(make_float2(__uint_as_float(x[c]), __uint_as_float(x[c + 1])), factor, ml));
                x[c] = __float_as_uint(p.x), x[c + 1] = __float_as_uint(p.y);
            }
            W.wait_warp(dp_full + 8 * (j % F::kDPs), (j / F::kDPs) & 1);
            tc_after_sync();
            tmem_load32(y, at_dp);
            tmem_wait_loads32(y);
            const bool masked = !__all_sync(~0u, lo <= key0 && hi >= key0 + 32);
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
                const float2 dp = make_float2(__uint_as_float(y[c]), __uint_as_float(y[c + 1]));
                const float2 ds = mul2(make_float2(__uint_as_float(x[c]), __uint_as_float(x[c + 1])), kNarrow<T> ? fma2(dp, step, md) : add2(dp, md));
                x[c] = __float_as_uint(ds.x), x[c + 1] = __float_as_uint(ds.y);
            }
            if (masked) {
#pragma unroll
                for (int c = 0; c < 32; ++c)
                    if (key0 + c < lo || key0 + c >= hi || one) x[c] = 0;
            }
            uint32_t words[16];
#pragma unroll
            for (int c = 0; c < 32; c += 2) words[c / 2] = pack2<T>(__uint_as_float(x[c]), __uint_as_float(x[c + 1]));
            tmem_store16(at_dp, words);
            tmem_wait_stores();
            if (part == 0 && (tile0 < min_lo || (tile0 + 64 > max_hi && max_hi < P.sk))) {
                // the copy's writes become visible through its own barrier
                W.wait_warp(k_full + 8 * s, (j / F::kStagesK) & 1);
                if (row < 64 && (tile0 + row < min_lo || tile0 + row >= max_hi)) clear_row<DP>(tiles_k + s * F::kTileK, 64, row);
                fence_async_shared();
            }
            tc_before_sync();
            bar_arrive(ds_full + 8 * (j % F::kDPs));
        }
        if (n) W.wait_warp(done, 0);
        tc_after_sync();
        {
#pragma unroll
            for (int c2 = 0; c2 < DP / 64; ++c2) {
                const int c = 2 * c2 + part;
                uint32_t o[32];
                if (n) {
                    tmem_load32(o, lanes + F::kColDQ + 32 * c);
                    tmem_wait_loads32(o);
                }
                if (i < P.sq) {
                    const float f = P.scale / steps;
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = hi ? pack2<T>(__uint_as_float(o[2 * e]) * f, __uint_as_float(o[2 * e + 1]) * f) : 0u;
                    store_row<T>(P.dq, b * P.dq_stride[0] + i * P.dq_stride[1] + h * P.dq_stride[2], P.head_dim, o, 32 * c);
                }
            }
        }
    }
    tc_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) tmem_free<F::kColumns>(tmem);
}

// ------------------------------------------------------------------------------------------------ host

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
    static Encode f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<Encode>(p);
    }();
    return f;
}

bool usable(const void* p, const int64_t* stride, const int64_t* size, uint32_t d) {
    if ((uintptr_t)p % 16) return false;
    for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (stride[i] % 8 || stride[i] < d || stride[i] >= (1ll << 38))) return false;
    return true;
}

// [batch, s, heads, head_dim] by boxes of `rows` tokens and 64 elements; what lies outside reads as zero.
int make_map(CUtensorMap* map, const halos_attention_args* a, const void* p, int64_t s, int64_t heads, const int64_t* stride, int rows) {
    const cuuint64_t dims[4] = {a->head_dim, (cuuint64_t)s, (cuuint64_t)heads, (cuuint64_t)a->batch};
    const auto bytes = [&](int64_t n, int64_t st) { return (cuuint64_t)(n > 1 ? st * 2 : a->head_dim * 2); };  // of a dimension of 1 it is never used
    const cuuint64_t strides[3] = {bytes(s, stride[1]), bytes(heads, stride[2]), bytes(a->batch, stride[0])};
    const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, ones[4] = {1, 1, 1, 1};
    Encode f = encoder();
    if (!f) return fail(HALOS_ERR_CUDA, "attention: the driver has no tensor maps");
    const CUresult r = f(map, a->dtype == HALOS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(p), dims, strides, box, ones,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? HALOS_OK : fail(HALOS_ERR_UNSUPPORTED, "attention: a tensor that no tensor map describes");
}

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

int check(const halos_attention_args* a, bool back) {
    if (!a || a->struct_size != sizeof(halos_attention_args)) return fail(HALOS_ERR_INVALID_ARG, "attention: args missing or of another size");
    if (!is_type(a->dtype)) return fail(HALOS_ERR_INVALID_ARG, "attention: dtype");
    if (a->dtype == HALOS_F32) return fail(HALOS_ERR_UNSUPPORTED, "attention: 16-bit types only");
    if (a->batch < 0 || a->sq < 0 || a->sk < 0) return fail(HALOS_ERR_INVALID_ARG, "attention: negative size");
    if (a->n_q == 0 || a->n_kv == 0 || a->n_q % a->n_kv) return fail(HALOS_ERR_INVALID_ARG, "attention: query heads must be a multiple of key heads");
    if (a->head_dim == 0 || a->head_dim % 8 || a->head_dim > 128) return fail(HALOS_ERR_UNSUPPORTED, "attention: head_dim must be a multiple of 8, at most 128");
    if (!(a->scale > 0.f) || !(a->scale * kLog2e < INFINITY)) return fail(HALOS_ERR_INVALID_ARG, "attention: scale must be positive, and finite times log2(e)");
    if (a->sq > (1 << 30) || a->sk > (1 << 30) || a->batch > 65535 || a->n_q > 65535) return fail(HALOS_ERR_UNSUPPORTED, "attention: over 2^30 tokens, 65535 heads or sequences");
    const int64_t tiles = (a->sq > a->sk ? a->sq : a->sk) / 128 + 1;
    if (tiles * a->batch * a->n_q > 0x7fffffffll) return fail(HALOS_ERR_UNSUPPORTED, "attention: too many tiles");
    if (a->batch == 0 || (a->sq == 0 && (!back || a->sk == 0))) return HALOS_OK;
    if ((a->sq && (!a->q || !a->o || !a->lse)) || (a->sk && (!a->k || !a->v))) return fail(HALOS_ERR_INVALID_ARG, "attention: null pointer");
    if (back && ((a->sq && (!a->dout || !a->dq)) || (a->sk && (!a->dk || !a->dv)))) return fail(HALOS_ERR_INVALID_ARG, "attention: null pointer");
    const int64_t q_size[3] = {a->batch, a->sq, a->n_q}, k_size[3] = {a->batch, a->sk, a->n_kv};
    bool ok = a->sq == 0 || (usable(a->q, a->q_stride, q_size, a->head_dim) && usable(a->o, a->o_stride, q_size, a->head_dim));
    ok = ok && (a->sk == 0 || (usable(a->k, a->k_stride, k_size, a->head_dim) && usable(a->v, a->v_stride, k_size, a->head_dim)));
    if (back) {
        ok = ok && (a->sq == 0 || (usable(a->dout, a->dout_stride, q_size, a->head_dim) && usable(a->dq, a->dq_stride, q_size, a->head_dim)));
        ok = ok && (a->sk == 0 || (usable(a->dk, a->dk_stride, k_size, a->head_dim) && usable(a->dv, a->dv_stride, k_size, a->head_dim)));
    }
    if (!ok) return fail(HALOS_ERR_UNSUPPORTED, "attention: bases and strides must be multiples of 16 bytes and rows apart");
    return HALOS_OK;
}

int params(const halos_attention_args* a, AttentionParams& P) {
    P.sq = (int)a->sq, P.sk = (int)a->sk, P.head_dim = a->head_dim, P.n_q = a->n_q, P.group = a->n_q / a->n_kv, P.batch = (int)a->batch;
    P.causal = a->causal != 0, P.q_tiles = (P.sq + 127) / 128, P.k_tiles = (P.sk + 127) / 128, P.records = (int)(round_up(a->sq, 128) / kRecord);
    // Keys and values of the heads of a section: 40 MB of the 126 MB L2 cache at most, one head at least.
    const int64_t head_bytes = (a->sk > 0 ? a->sk : 1) * 4 * (a->head_dim <= 64 ? 64 : 128), heads = a->batch * a->n_kv;
    P.section = (int)(heads < 40000000 / head_bytes ? heads : head_bytes < 40000000 ? 40000000 / head_bytes : 1);
    P.scale = a->scale, P.scale2 = a->scale * kLog2e, P.doc_start = a->doc_start, P.lens = a->lens;
    P.q = (const char*)a->q, P.k = (const char*)a->k, P.v = (const char*)a->v;
    P.o_in = P.o = (char*)a->o, P.dout = (const char*)a->dout, P.dq = (char*)a->dq, P.dk = (char*)a->dk, P.dv = (char*)a->dv, P.lse = a->lse;
    for (int i = 0; i < 3; ++i)
        P.q_stride[i] = a->q_stride[i], P.k_stride[i] = a->k_stride[i], P.v_stride[i] = a->v_stride[i], P.o_stride[i] = a->o_stride[i], P.dout_stride[i] = a->dout_stride[i], P.dq_stride[i] = a->dq_stride[i], P.dk_stride[i] = a->dk_stride[i], P.dv_stride[i] = a->dv_stride[i];
    return fault_mark(&P.fault);
}

template <typename T, int DP>
int forward(const halos_attention_args* a) {
    using F = Forward<DP>;
    AttentionParams P{};
    if (int rc = params(a, P)) return rc;
    CUtensorMap q, k{}, v{};
    if (int rc = make_map(&q, a, a->q, a->sq, a->n_q, a->q_stride, 128)) return rc;
    if (a->sk) {
        if (int rc = make_map(&k, a, a->k, a->sk, a->n_kv, a->k_stride, 64)) return rc;
        if (int rc = make_map(&v, a, a->v, a->sk, a->n_kv, a->v_stride, 64)) return rc;
    }
    static Allowed allowed;
    if (int rc = allow_smem(attention_fwd_kernel<T, DP>, F::kSmem, allowed)) return rc;
    attention_fwd_kernel<T, DP><<<P.q_tiles * P.batch * P.n_q, F::kThreads, F::kSmem, (cudaStream_t)a->stream>>>(P, q, k, v);
    return cuda_status(cudaGetLastError(), "attention launch");
}

uint64_t workspace(const halos_attention_args* a) {
    const uint64_t records = (uint64_t)(round_up(a->sq, 128) / kRecord);
    uint64_t bytes = a->batch * records * (a->n_q * sizeof(Record) + sizeof(Reach));
    if (a->dtype == HALOS_F16) bytes += a->batch * (a->n_kv * sizeof(Lengths) + a->n_q * records * sizeof(float));
    return bytes;
}

template <typename T, int DP, int kKeySlots>
int backward(const halos_attention_args* a) {
    AttentionParams P{};
    if (int rc = params(a, P)) return rc;
    P.record = (Record*)a->workspace;
    P.reach = (Reach*)(P.record + (int64_t)P.batch * P.n_q * P.records);
    P.lengths = (Lengths*)(P.reach + (int64_t)P.batch * P.records);
    P.dout_square = (float*)(P.lengths + (int64_t)P.batch * a->n_kv);
    cudaStream_t st = (cudaStream_t)a->stream;
    CUtensorMap q{}, d{}, k{}, v{};
    using K = Keys<DP, kKeySlots>;
    using Q = Queries<DP>;
    static Allowed allowed_keys, allowed_queries;
    if (int rc = allow_smem(attention_keys_kernel<T, DP, kKeySlots>, K::kSmem, allowed_keys)) return rc;
    if (int rc = allow_smem(attention_queries_kernel<T, DP>, Q::kSmem, allowed_queries)) return rc;
    if (P.sq) {
        attention_record_kernel<T><<<dim3(P.records, P.n_q, P.batch), 4 * kRecord, 0, st>>>(P);
        if (int rc = cuda_status(cudaGetLastError(), "attention launch")) return rc;
    }
    if constexpr (kNarrow<T>) {
        if (P.sq && P.sk) {
            // Four blocks to an SM over all heads at most: each goes over the reaches of its batch row once.
            const int64_t heads = (int64_t)P.batch * a->n_kv, most = (P.sk + kLengthsKeys - 1) / kLengthsKeys, want = (4 * (int64_t)sm_count(a->device) + heads - 1) / heads;
            attention_lengths_kernel<T><<<dim3((unsigned)(most < want ? most : want), a->n_kv, P.batch), kLengthsThreads, 0, st>>>(P);
            if (int rc = cuda_status(cudaGetLastError(), "attention launch")) return rc;
        }
    }
    if (P.sk) {
        if (P.sq) {
            if (int rc = make_map(&q, a, a->q, a->sq, a->n_q, a->q_stride, 64)) return rc;
            if (int rc = make_map(&d, a, a->dout, a->sq, a->n_q, a->dout_stride, 64)) return rc;
        }
        if (int rc = make_map(&k, a, a->k, a->sk, a->n_kv, a->k_stride, 128)) return rc;
        if (int rc = make_map(&v, a, a->v, a->sk, a->n_kv, a->v_stride, 128)) return rc;
        attention_keys_kernel<T, DP, kKeySlots><<<P.k_tiles * P.batch * (int)a->n_kv, K::kThreads, K::kSmem, st>>>(P, q, k, v, d);
        if (int rc = cuda_status(cudaGetLastError(), "attention launch")) return rc;
    }
    if (P.sq) {
        if (P.sk) {
            if (int rc = make_map(&k, a, a->k, a->sk, a->n_kv, a->k_stride, 64)) return rc;
            if (int rc = make_map(&v, a, a->v, a->sk, a->n_kv, a->v_stride, 64)) return rc;
        }
        if (int rc = make_map(&q, a, a->q, a->sq, a->n_q, a->q_stride, 128)) return rc;
        if (int rc = make_map(&d, a, a->dout, a->sq, a->n_q, a->dout_stride, 128)) return rc;
        attention_queries_kernel<T, DP><<<P.q_tiles * P.batch * P.n_q, Q::kThreads, Q::kSmem, st>>>(P, q, k, v, d);
        if (int rc = cuda_status(cudaGetLastError(), "attention launch")) return rc;
    }
    return HALOS_OK;
}

}  // namespace
}  // namespace halos_step

extern "C" int halos_attention_fwd(const halos_attention_args* a) {
    using namespace halos_step;
    if (int rc = check(a, false)) return rc;
    if (a->batch == 0 || a->sq == 0) return HALOS_OK;
    if (int rc = enter(a->device)) return rc;
    if (a->dtype == HALOS_BF16) return a->head_dim <= 64 ? forward<__nv_bfloat16, 64>(a) : forward<__nv_bfloat16, 128>(a);
    return a->head_dim <= 64 ? forward<__half, 64>(a) : forward<__half, 128>(a);
}

extern "C" int halos_attention_workspace(const halos_attention_args* a, uint64_t* bytes) {
    using namespace halos_step;
    if (!a || a->struct_size != sizeof(halos_attention_args) || !bytes || a->batch < 0 || a->sq < 0)
        return fail(HALOS_ERR_INVALID_ARG, "attention: args missing or of another size");
    *bytes = workspace(a);
    return HALOS_OK;
}

extern "C" int halos_attention_bwd(const halos_attention_args* a) {
    using namespace halos_step;
    if (int rc = check(a, true)) return rc;
    if (a->batch == 0 || (a->sq == 0 && a->sk == 0)) return HALOS_OK;
    if (workspace(a) && (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < workspace(a)))
        return fail(HALOS_ERR_INVALID_ARG, "attention: workspace missing, unaligned or too small");
    if (int rc = enter(a->device)) return rc;
    if (a->dtype == HALOS_BF16) return a->head_dim <= 64 ? backward<__nv_bfloat16, 64, 1>(a) : backward<__nv_bfloat16, 128, 2>(a);
    return a->head_dim <= 64 ? backward<__half, 64, 1>(a) : backward<__half, 128, 2>(a);
}
