// The gradient of root-mean-square norms.
//
// dx = rstd (g - u mean(g u)) + dsummed and dweight = sum over rows of dy u, with u = s rstd and g = dy w: three tensors read and one written.  A row goes through once; between the
// two passes over its threads' parts, which lie in shared memory, there is one sum.  dweight is added up in registers over all rows that a thread sees, then over the CTA's
// threads, and a second kernel adds up the CTAs' parts, in their order: no atomics, the same bits every time.
//
// Measured (by bytes at the copy rate), with dsummed: 16384 x 2048 bf16 55 us among other passes (74%), 52 by itself (the second kernel and its start take 4 of them), 65536 x 768 bf16
// 76 us (81%), 16384 x 1024 f32 48 us (85%), 8192 x 8192 f32 174 us (94%), 32768 x 1021 bf16 80 us (51%), 16384 x 1021 f32 54 us (76%); without: 4096 x 16384 f32 150 us (82%), 180560 heads of 80
// f16 33 us (40%), 3063 x 10 heads of 80 f32, strided, 16 us, of which the call takes 14.  The kernels that go over rows in loops, which read summed and dy twice: 24576 x 768 f32 with dsummed
// 122 us (38%), 13107 x 5120 342 us (48%), 4096 x 16384 409 us (40%).
#include "step_norm.cuh"


namespace halos_step {
namespace norm {

// ------------------------------------------------------------------------------------------------ rows of any size and alignment

template <typename T>
__global__ void __launch_bounds__(kThreads) rms_norm_any_dx_kernel(const __grid_constant__ Params P) {
    const uint32_t row = blockIdx.x;
    const T* s = row_at<const T>(P, P.in[0], row);
    const T* dy = row_at<const T>(P, P.in[1], row);
    const T* ds = P.arrays > 2 ? row_at<const T>(P, P.in[2], row) : nullptr;
    T* dx = row_at<T>(P, P.out[0], row);
    const float rstd = P.rstd[row];
    float dot = 0.f;
    for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) dot = fmaf(to_f32<T>(dy[c]) * weight_at(P, c), to_f32<T>(s[c]) * rstd, dot);
    const float mean = cta_sum(dot) * P.inverse_dim;
    for (uint32_t c = threadIdx.x; c < P.dim; c += kThreads) {
        const float g = to_f32<T>(dy[c]) * weight_at(P, c), u = to_f32<T>(s[c]) * rstd;
        dx[c] = from_f32<T>(fmaf(rstd, fmaf(-u, mean, g), ds ? to_f32<T>(ds[c]) : 0.f));
    }
}

// A thread to a column; the rows are split into as many runs as fill the GPU.
template <typename T>
__global__ void __launch_bounds__(kThreads) rms_norm_any_dweight_kernel(const __grid_constant__ Params P) {
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= P.dim) return;
    const uint32_t from = (uint32_t)((uint64_t)P.rows * blockIdx.y / P.splits), to = (uint32_t)((uint64_t)P.rows * (blockIdx.y + 1) / P.splits);
    float sum = 0.f;
    for (uint32_t row = from; row < to; ++row)
        sum = fmaf(to_f32<T>(row_at<const T>(P, P.in[1], row)[c]), to_f32<T>(row_at<const T>(P, P.in[0], row)[c]) * P.rstd[row], sum);
    P.partial[(int64_t)blockIdx.y * P.dim + c] = sum;
}

__device__ __forceinline__ void write_dweight(const Params& P, uint32_t c, float sum) {
    if (P.weight_type == HALOS_F32) reinterpret_cast<float*>(P.dweight)[c] = sum;
    else if (P.weight_type == HALOS_BF16) reinterpret_cast<__nv_bfloat16*>(P.dweight)[c] = __float2bfloat16_rn(sum);
    else reinterpret_cast<__half*>(P.dweight)[c] = __float2half_rn(sum);
}

constexpr int kJoinColumns = 32, kJoinRows = 32;
__global__ void __launch_bounds__(kJoinColumns * kJoinRows) rms_norm_join_kernel(const __grid_constant__ Params P) {
    __shared__ float s[kJoinRows][kJoinColumns];
    const uint32_t x = threadIdx.x % kJoinColumns, y = threadIdx.x / kJoinColumns, c = blockIdx.x * kJoinColumns + x;
    float sum = 0.f;
    after_previous();
    if (c < P.dim)
#pragma unroll 4
        for (uint32_t i = y; i < P.splits; i += kJoinRows) sum += P.partial[(int64_t)i * P.dim + c];
    s[y][x] = sum;
    __syncthreads();
    if (y || c >= P.dim) return;
#pragma unroll
    for (int i = 1; i < kJoinRows; ++i) sum += s[i][x];
    write_dweight(P, c, sum);
}

// ------------------------------------------------------------------------------------------------ rows that a CTA holds

// Places of a column in shared memory, so that threads that write neighbouring accesses meet different banks.
template <int V> __device__ __forceinline__ int spread(int c) { return c + c / V; }

// A thread has the same columns in all its rows and adds up its part of dweight in registers; a CTA's rows are added in shared memory, and CTAs' by
// the kernel that joins.
template <typename T, int N, int L, Mode M, int ARRAYS>
__global__ void __launch_bounds__(kWide<T, N, M> ? kMostThreads : kThreads, kWide<T, N, M> ? 1 : 3) rms_norm_back_kernel(const __grid_constant__ Params P) {
    constexpr int THREADS = kWide<T, N, M> ? kMostThreads : kThreads;
    using A = Threads<T, N, L, M, THREADS, ARRAYS>;
    constexpr int V = A::V, H = A::H;
    extern __shared__ __align__(16) char s_dynamic[];
    __shared__ uint32_t s_part[2 * kMostThreads / 32];
    const A t(P, s_dynamic, true);
    RowSums<(N > 1 && L == 32)> S(t.lanes, s_part);
    const int stages = (int)P.stages, dim = t.dim;
    for (int k = 0; k < stages - 1; ++k) t.fetch(k, k, true);
    t.load_weights();
    float2 dw[N][H];
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < H; ++i) dw[j][i] = both(0.f);

    int stage = 0;
    for (uint32_t i = 0; i < P.run; ++i) {
        if (stages == 1) t.fetch(i, 0, true);
        wait_copies(stages == 3);
        if (stages > 1) t.fetch(i + stages - 1, stage ? stage - 1 : stages - 1, true);   // where the row before this was
        const uint32_t row = t.row_of(i);
        const bool here = row < P.rows;
        const float rstd = here ? t.rstd[stage * THREADS] : 0.f;
        float2 dots = both(0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float2 u[H], a[H], w[H];
            t.arrived(stage, 0, j, here, u), t.arrived(stage, 1, j, here, a), t.weights(j, w);
#pragma unroll
            for (int i = 0; i < H; ++i) a[i] = mul2(a[i], mul2(u[i], both(rstd)));
            keep_own<V, M>(a, t.column(j), dim);
#pragma unroll
            for (int i = 0; i < H; ++i) dw[j][i] = add2(dw[j][i], a[i]), dots = fma2(a[i], w[i], dots);
        }
        const float mean = S.sum(dots.x + dots.y) * P.inverse_dim;
        T* dx = here ? row_at<T>(P, P.out[0], row) : nullptr;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float2 u[H], a[H], w[H], d[H];
            // from shared memory once more: registers would be too many
            t.arrived(stage, 0, j, here, u), t.arrived(stage, 1, j, here, a), t.weights(j, w);
            if (ARRAYS > 2) t.arrived(stage, 2, j, here, d);
            else {
#pragma unroll
                for (int i = 0; i < H; ++i) d[i] = both(0.f);
            }
#pragma unroll
            for (int i = 0; i < H; ++i) a[i] = fma2(both(rstd), fma2(a[i], w[i], mul2(mul2(u[i], both(rstd)), both(-mean))), d[i]);
            if (here) store_part<T, V, M>(dx, t.column(j), dim, a);
        }
        stage = stage + 1 == stages ? 0 : stage + 1;
    }
    for (uint32_t o = t.lanes; o < 32; o *= 2)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < H; ++i) dw[j][i] = add2(dw[j][i], make_float2(__shfl_xor_sync(~0u, dw[j][i].x, o), __shfl_xor_sync(~0u, dw[j][i].y, o)));
    float* s_dw = reinterpret_cast<float*>(s_dynamic);                  // [dim], spread; nothing else is needed any more
    wait_copies(false);
    __syncthreads();
    const uint32_t turns = min(t.per, THREADS / 32u), turn = t.lanes < 32 ? (threadIdx.x % 32 < t.lanes ? threadIdx.x / 32 : turns) : t.own;
    for (uint32_t k = 0; k < turns; ++k) {
        if (turn == k) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int c = t.column(j);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (owned<V>(c, e, dim)) {
                        float& to = s_dw[spread<V>(c + e)];
                        const float part = e % 2 ? dw[j][e / 2].y : dw[j][e / 2].x;
                        to = k ? to + part : part;
                    }
            }
        }
        __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < P.dim; c += blockDim.x) {
        const float sum = s_dw[spread<V>(c)];
        if (gridDim.x == 1) write_dweight(P, c, sum);
        else P.partial[(int64_t)blockIdx.x * P.dim + c] = sum;
    }
}

// ------------------------------------------------------------------------------------------------ host

static Shape back_shape_of(const Params& P, uint32_t size, Mode mode) {
    const uint32_t v = mode == kLoose ? 2 : 16 / size, accesses = accesses_of(P.dim, v, mode);
    Shape s{};
    spread_over(s, v, mode, accesses, 1);
    if (!s.n) return s;
    const bool wide = s.n * v > kFew;
    s.threads = wide ? kMostThreads : kThreads, s.resident = wide ? 1 : 3;
    const uint32_t room = kSharedPerSM / s.resident - 1024 - 256, stage = s.threads * (P.arrays * s.n * v * size + 4);
    const uint32_t fixed = s.n * v * 4 * (mode == kShifted ? s.threads : s.lanes), end = (P.dim + P.dim / v + 1) * 4;
    if (fixed + stage > room || end > room) return Shape{};
    s.stages = mode == kLoose ? 1 : (room - fixed) / stage;
    if (s.stages > kMostStages) s.stages = kMostStages;
    s.shared = fixed + s.stages * stage > end ? fixed + s.stages * stage : end;
    return s;
}

static uint32_t splits_of(uint32_t rows, uint32_t dim, int32_t device) {
    const uint32_t columns = (dim + kThreads - 1) / kThreads, want = (uint32_t)sm_count(device) * 8 / columns;
    const uint32_t most = (rows + 15) / 16;      // runs of 16 rows or more
    return want < 1 ? 1 : want > most ? (most ? most : 1) : want;
}

// Partial sums of dweight, at most.
static uint64_t most_splits(uint32_t rows, uint32_t dim, int32_t device) {
    const uint64_t few = splits_of(rows, dim, device), most = (uint64_t)sm_count(device) * 3 / 8 * 8, blocks = ((uint64_t)rows + 7) / 8 * 8;
    return few > (most < blocks ? most : blocks) ? few : most < blocks ? most : blocks;
}

}  // namespace norm
}  // namespace halos_step

extern "C" int halos_rms_norm_workspace(const halos_rms_norm_args* a, uint64_t* bytes) {
    using namespace halos_step;
    using namespace halos_step::norm;
    if (int rc = check(a)) return rc;
    if (!bytes) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    if (int rc = enter(a->device)) return rc;
    *bytes = most_splits((uint32_t)(a->size[0] * a->size[1] * a->size[2]), a->dim, a->device) * a->dim * sizeof(float);
    return HALOS_OK;
}

extern "C" int halos_rms_norm_bwd(const halos_rms_norm_args* a) {
    using namespace halos_step;
    using namespace halos_step::norm;
    if (int rc = check(a)) return rc;
    Params P{};
    P.arrays = a->dsummed ? 3 : 2;
    set(P.in[0], a->summed, a->summed_stride), set(P.in[1], a->dy, a->dy_stride), set(P.in[2], a->dsummed, a->dsummed_stride), set(P.out[0], a->dx, a->dx_stride);
    if (int rc = fill(a, P, 1)) return rc;
    if (!a->weight || !a->dweight || (P.rows && (!a->summed || !a->rstd || !a->dy || !a->dx))) return fail(HALOS_ERR_INVALID_ARG, "norm: null pointer");
    const uint32_t size = size_of(a->dtype);
    if (((uintptr_t)a->summed | (uintptr_t)a->dy | (uintptr_t)a->dsummed | (uintptr_t)a->dx) % size) return fail(HALOS_ERR_INVALID_ARG, "norm: tensor not aligned to its elements");
    if (int rc = enter(a->device)) return rc;
    if (!a->workspace || (uintptr_t)a->workspace % 16 || a->workspace_bytes < most_splits(P.rows, P.dim, a->device) * P.dim * sizeof(float))
        return fail(HALOS_ERR_INVALID_ARG, "norm: workspace missing, not aligned or too small");
    P.dweight = (char*)a->dweight, P.partial = (float*)a->workspace, P.splits = splits_of(P.rows, P.dim, a->device);
    cudaStream_t st = (cudaStream_t)a->stream;
    const Mode mode = mode_of(P, size, 1, size);
    const Shape s = P.rows ? back_shape_of(P, size, mode) : Shape{};
    const int rc = by_type(a->dtype, [&](auto t) -> int {
        using T = decltype(t);
        if (!s.n) {
            if (P.rows) {
                rms_norm_any_dx_kernel<T><<<P.rows, kThreads, 0, st>>>(P);
                if (int rc = cuda_status(cudaGetLastError(), "norm launch")) return rc;
            }
            rms_norm_any_dweight_kernel<T><<<dim3((P.dim + kThreads - 1) / kThreads, P.splits), kThreads, 0, st>>>(P);
            return cuda_status(cudaGetLastError(), "norm launch");
        }
        P.lanes = s.lanes, P.stages = s.stages, P.row_blocks = (P.rows + s.per() - 1) / s.per();
        // a multiple of 8, so that steps of as many rows keep every shift
        const uint32_t most = (uint32_t)sm_count(a->device) * s.resident / 8 * 8;
        P.splits = P.row_blocks < most ? (P.row_blocks + 7) / 8 * 8 : most;
        // A few rows are one CTA's, which needs no other kernel to join its sums.
        if (P.row_blocks <= 4 && (mode != kShifted || s.per() >= 8)) P.splits = 1;
        P.apart = P.splits, P.run = (P.row_blocks + P.splits - 1) / P.splits;
        return by_accesses<T>(s.n, s.apart, mode, [&](auto n, auto l, auto m) -> int {
            const auto launch = [&](auto* kernel, Allowed& allowed) -> int {
                if (int rc = allow_smem(kernel, (int)s.shared, allowed)) return rc;
                kernel<<<P.splits, s.threads, s.shared, st>>>(P);
                return cuda_status(cudaGetLastError(), "norm launch");
            };
            static Allowed allowed[2];
            constexpr int N = decltype(n)::value, L = decltype(l)::value;
            constexpr Mode M = decltype(m)::value;
            return P.arrays > 2 ? launch(rms_norm_back_kernel<T, N, L, M, 3>, allowed[0]) : launch(rms_norm_back_kernel<T, N, L, M, 2>, allowed[1]);
        });
    });
    if (rc || (s.n && P.splits == 1)) return rc;
    return launch_after(rms_norm_join_kernel, (P.dim + kJoinColumns - 1) / kJoinColumns, kJoinColumns * kJoinRows, 0, st, "norm launch", P);
}
