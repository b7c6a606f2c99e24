// The batched product with a low-rank adapter of its own for every request beside the shared matrix:
//   Y[b, :] = W X[b, :] + s_a up_a (down_a X[b, :]),  a = which[b].
// The shared product is csb_spmm's.  The adapters' part is two kernels around it: csb_adapter_down_kernel takes
// down_a X[b, :] into the workspace, csb_adapter_up_kernel adds up_a times that to Y.  Requests of one adapter are taken
// eight at a time (the eight columns of a tensor-core tile), found by every CTA for itself from `which`: nothing is sorted
// and no order of atomics enters.  Both kernels are bound by reading the adapters once; the arithmetic is in two tf32
// halves of the fp32 operand (22 bits; 16-bit adapters are one such half exactly, fp32 adapters two), fp32 sums.
#include <algorithm>

#include "csb_host.hpp"
#include "csb_device.cuh"
#include "csb_values.cuh"

namespace csb {

constexpr int kGroup = 8;               // requests of one adapter that a CTA takes together
constexpr int kDownThreads = 256, kUpThreads = 256;
constexpr int kMaxRank = 256;
constexpr int kScan = 4;                // entries of `which` that a thread looks at between two barriers

struct AdapterArgs {
    const float* X; float* Y;
    const void *down, *up;
    const int32_t *which, *ranks;
    const float* scales;
    float* part;                        // [splits][batch][rank_pad]
    long long ldx, ldy;
    int batch, count, rank, rank_pad, rows, cols, splits, split_cols;
};

struct Group {
    int32_t seen[kScan * (kDownThreads / 32)];
    int32_t rank_of_b;
    int32_t member[kGroup];
};

// The requests that CTA `b` works for: none unless b's place among the requests of its adapter is a multiple of kGroup,
// else b and up to kGroup - 1 that follow it.  Returns their number; all threads of the block take part.
template <int NT>
__device__ int find_group(const AdapterArgs& a, int b, Group& G) {
    const int mine = a.which[b];
    if (mine < 0 || mine >= a.count) return 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int before = 0, first = -1, found = 0;
    for (int base = 0; base < a.batch; base += NT * kScan) {
        uint32_t same[kScan];
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const int j = base + i * NT + (int)threadIdx.x;
            same[i] = __ballot_sync(0xffffffffu, j < a.batch && a.which[j] == mine);
            if (lane == 0) G.seen[i * (NT / 32) + warp] = __popc(same[i]);
        }
        __syncthreads();
        int at[kScan], total = before;
#pragma unroll
        for (int i = 0; i < kScan; ++i)
            for (int w = 0; w < NT / 32; ++w) {
                if (w == warp) at[i] = total + __popc(same[i] & ((1u << lane) - 1u));
                total += G.seen[i * (NT / 32) + w];
            }
        before = total;
        if (b >= base + NT * kScan) { __syncthreads(); continue; }
        if (b >= base) {
#pragma unroll
            for (int i = 0; i < kScan; ++i)
                if (base + i * NT + (int)threadIdx.x == b) G.rank_of_b = at[i];
            __syncthreads();
            first = G.rank_of_b;
            if (first % kGroup) return 0;
        }
#pragma unroll
        for (int i = 0; i < kScan; ++i) {
            const int j = base + i * NT + (int)threadIdx.x;
            if (j >= b && (same[i] >> lane & 1u) && at[i] - first < kGroup) G.member[at[i] - first] = j;
        }
        found = min(before - first, kGroup);
        __syncthreads();
        if (found == kGroup) break;
    }
    return found;
}

__device__ __forceinline__ int rank_of(const AdapterArgs& a, int which) {
    return a.ranks ? min(max(a.ranks[which], 0), a.rank) : a.rank;
}

// Eight values of a row of `size` from element c on, zeros behind its end.
template <bool VEC, typename T>
__device__ __forceinline__ void eight(const T* row, int c, int size, bool there, float (&v)[8]) {
    if (VEC) {
        if (there && c < size) { load_values(row + c, v); return; }            // (size is a multiple of 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = there && c + i < size ? to_float(row[c + i]) : 0.f;
    }
}

// part[split][b][:] = down_a X[b, columns of the split].  A warp takes 32 columns at a time: lane 4g + t has columns
// 8t .. 8t + 7 of ranks g and g + 8 and of request g, which are its operands of four steps of eight columns when those are
// counted in another order, so that every operand comes by wide loads straight from global memory.
template <typename T, int MT, bool VEC>
__global__ void __launch_bounds__(kDownThreads) csb_adapter_down_kernel(const AdapterArgs a) {
    __shared__ Group G;
    __shared__ float sum[kDownThreads / 32][MT * 16 * kGroup];
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x, n = find_group<kDownThreads>(a, b, G);
    if (!n) return;
    const int which = a.which[b], rank = rank_of(a, which), r0 = (int)blockIdx.z * MT * 16;
    if (r0 >= rank) return;                                      // (the other kernel reads no such part)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const T* down = static_cast<const T*>(a.down) + (size_t)which * a.rank * a.cols;
    const float* x = g < n ? a.X + (long long)G.member[g] * a.ldx : a.X;
    float d[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m) d[m][0] = d[m][1] = d[m][2] = d[m][3] = 0.f;
    const int c_end = min(a.cols, ((int)blockIdx.y + 1) * a.split_cols);
    for (int c0 = (int)blockIdx.y * a.split_cols + warp * 32; c0 < c_end; c0 += kDownThreads) {
        const int c = c0 + t * 8;
        float xv[8];
        uint32_t hi[8], lo[8];
        eight<VEC>(x, c, c_end, g < n, xv);
#pragma unroll
        for (int i = 0; i < 8; ++i) split_tf32(xv[i], hi[i], lo[i]);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int r = r0 + m * 16 + g;
            float u[8], v[8];
            eight<VEC>(down + (size_t)r * a.cols, c, c_end, r < rank, u);
            eight<VEC>(down + (size_t)(r + 8) * a.cols, c, c_end, r + 8 < rank, v);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                uint32_t w[4] = {__float_as_uint(u[i]), __float_as_uint(v[i]), __float_as_uint(u[i + 1]), __float_as_uint(v[i + 1])};
                if (sizeof(T) == 4) {
                    uint32_t wl[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) split_tf32(__uint_as_float(w[k]), w[k], wl[k]);
                    mma_tf32(d[m], wl, hi[i], hi[i + 1]);
                }
                mma_tf32(d[m], w, lo[i], lo[i + 1]);
                mma_tf32(d[m], w, hi[i], hi[i + 1]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[warp][(2 * t + (k & 1)) * MT * 16 + m * 16 + g + (k >> 1) * 8] = d[m][k];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 16 * n; i += kDownThreads) {
        const int r = r0 + i % (MT * 16);
        if (r >= a.rank_pad) continue;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kDownThreads / 32; ++w) s += sum[w][i];
        a.part[((size_t)blockIdx.y * a.batch + G.member[i / (MT * 16)]) * a.rank_pad + r] = s;
    }
}

// Y[b, rows] += s_a up_a (sum of the parts).  A warp takes 16 rows at a time; lane 4g + t has ranks 4t .. 4t + 3 of every
// 16 of rows g and g + 8 (again two steps in an order of their own).
template <typename T, bool VEC>
__global__ void __launch_bounds__(kUpThreads) csb_adapter_up_kernel(const AdapterArgs a, int rows_a_cta) {
    __shared__ Group G;
    __shared__ __align__(16) uint32_t hi[kGroup][kMaxRank + 16], lo[kGroup][kMaxRank + 16];
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x, n = find_group<kUpThreads>(a, b, G);
    if (!n) return;
    const int which = a.which[b], rank = rank_of(a, which);
    if (rank == 0) return;
    const float scale = a.scales ? a.scales[which] : 1.f;
    for (int i = threadIdx.x; i < kGroup * a.rank_pad; i += kUpThreads) {
        const int j = i / a.rank_pad, r = i % a.rank_pad;
        float s = 0.f;
        if (j < n && r < rank)
            for (int p = 0; p < a.splits; ++p) s += a.part[((size_t)p * a.batch + G.member[j]) * a.rank_pad + r];
        split_tf32(s * scale, hi[j][r], lo[j][r]);
    }
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const T* up = static_cast<const T*>(a.up) + (size_t)which * a.rank * a.rows;
    const int end = min(a.rows, ((int)blockIdx.y + 1) * rows_a_cta);
    for (int i0 = (int)blockIdx.y * rows_a_cta + warp * 16; i0 < end; i0 += kUpThreads / 2) {
        float d[4] = {0.f, 0.f, 0.f, 0.f};
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = i0 + g + (k >> 1) * 8, j = 2 * t + (k & 1);
            y[k] = row < end && j < n ? a.Y[(long long)G.member[j] * a.ldy + row] : 0.f;
        }
        for (int r0 = 0; r0 < rank; r0 += 16) {
            const int r = r0 + 4 * t;
            float u[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int row = i0 + g + 8 * k;
                const T* p = up + (size_t)row * a.rank + r;
                if (VEC && row < end && r + 4 <= rank) load_values(p, u[k]);
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[k][i] = row < end && r + i < rank ? to_float(p[i]) : 0.f;
                }
            }
            const uint4 h = *reinterpret_cast<const uint4*>(&hi[g][r]), l = *reinterpret_cast<const uint4*>(&lo[g][r]);
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                uint32_t w[4] = {__float_as_uint(u[0][i]), __float_as_uint(u[1][i]), __float_as_uint(u[0][i + 1]), __float_as_uint(u[1][i + 1])};
                const uint32_t h0 = i ? h.z : h.x, h1 = i ? h.w : h.y, l0 = i ? l.z : l.x, l1 = i ? l.w : l.y;
                if (sizeof(T) == 4) {
                    uint32_t wl[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) split_tf32(__uint_as_float(w[k]), w[k], wl[k]);
                    mma_tf32(d, wl, h0, h1);
                }
                mma_tf32(d, w, l0, l1);
                mma_tf32(d, w, h0, h1);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = i0 + g + (k >> 1) * 8, j = 2 * t + (k & 1);
            if (row < end && j < n) a.Y[(long long)G.member[j] * a.ldy + row] = y[k] + d[k];
        }
    }
}

#define CSB_CUDA(call)                                                                     \
    do {                                                                                   \
        cudaError_t e_ = (call);                                                           \
        if (e_ != cudaSuccess) {                                                           \
            set_error("%s failed: %s", #call, cudaGetErrorString(e_));                     \
            return e_ == cudaErrorMemoryAllocation ? CSB_ERR_ALLOC : CSB_ERR_CUDA;         \
        }                                                                                  \
    } while (0)

static int rank_pad(int rank) { return (rank + 15) / 16 * 16; }
// Columns of a split, a multiple of what a CTA takes in one turn: as many splits as give some CTAs to every SM even where
// all requests of a group of four share an adapter.
static int split_columns(int64_t cols, int batch) {
    const int64_t turns = (cols + kDownThreads - 1) / kDownThreads;
    const int64_t want = std::min<int64_t>(turns, std::max<int64_t>(1, 592 / ((batch + 3) / 4)));
    return (int)((turns + want - 1) / want * kDownThreads);
}
static int64_t workspace_bytes(int64_t cols, int batch, int rank) {
    const int64_t w = split_columns(cols, batch);
    return (cols + w - 1) / w * batch * rank_pad(rank) * 4;
}

template <typename... Args>
static cudaError_t launch(void (*kernel)(Args...), dim3 grid, int threads, void* stream, Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid; cfg.blockDim = dim3((unsigned)threads); cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename T, bool VEC>
static cudaError_t launch_down(const AdapterArgs& a, void* stream) {
    const unsigned tiles = (unsigned)(a.rank_pad / 16);
    if (tiles == 1) return launch<const AdapterArgs>(csb_adapter_down_kernel<T, 1, VEC>, dim3((unsigned)a.batch, (unsigned)a.splits), kDownThreads, stream, a);
    if (tiles == 2) return launch<const AdapterArgs>(csb_adapter_down_kernel<T, 2, VEC>, dim3((unsigned)a.batch, (unsigned)a.splits), kDownThreads, stream, a);
    return launch<const AdapterArgs>(csb_adapter_down_kernel<T, 4, VEC>, dim3((unsigned)a.batch, (unsigned)a.splits, (tiles + 3) / 4), kDownThreads, stream, a);
}

template <typename T>
static int adapters_on_device(const csb_matrix* A, AdapterArgs a, void* stream) {
    auto aligned = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
    const bool down_vec = a.cols % 8 == 0 && aligned(a.down, 16) && a.ldx % 4 == 0 && aligned(a.X, 16);
    const bool up_vec = a.rank % 4 == 0 && aligned(a.up, 4 * sizeof(T));
    CSB_CUDA((down_vec ? launch_down<T, true>(a, stream) : launch_down<T, false>(a, stream)));
    const int rc = guarded([&] { return product_any(A, a.X, a.ldx, a.batch, a.Y, a.ldy, stream); });
    if (rc != CSB_OK) return rc;
    // rows of a CTA: fewer where there are few requests, a multiple of what it takes in one turn
    int rows = kUpThreads / 2;
    while ((int64_t)a.batch * ((a.rows + rows - 1) / rows) > 8 * 592 && rows < 1024) rows *= 2;
    while ((a.rows + rows - 1) / rows > 65535) rows *= 2;
    const dim3 grid((unsigned)a.batch, (unsigned)((a.rows + rows - 1) / rows));
    CSB_CUDA((up_vec ? launch<const AdapterArgs, int>(csb_adapter_up_kernel<T, true>, grid, kUpThreads, stream, a, rows)
                    : launch<const AdapterArgs, int>(csb_adapter_up_kernel<T, false>, grid, kUpThreads, stream, a, rows)));
    return CSB_OK;
}

}  // namespace csb

using namespace csb;

extern "C" {

int64_t csb_adapters_workspace_bytes(const csb_matrix_t* A, int batch, int rank) {
    if (!A || batch <= 0 || rank < 1 || rank > kMaxRank) return 0;
    return workspace_bytes(A->cols, batch, rank);
}

int csb_spmm_adapters(const csb_matrix_t* A, const float* X, int64_t ldx, int batch, float* Y, int64_t ldy, int dtype, int count, int rank,
                      const void* down, const void* up, const int32_t* which, const int32_t* ranks, const float* scales,
                      void* workspace, int64_t workspace_size, void* stream) {
    clear_error();
    if (!A) { set_error("A is NULL"); return CSB_ERR_INVALID_ARG; }
    if (batch < 0 || count < 0 || rank < 1) { set_error("batch %d, count %d, rank %d", batch, count, rank); return CSB_ERR_INVALID_ARG; }
    if (dtype != CSB_F32 && dtype != CSB_F16 && dtype != CSB_BF16) { set_error("dtype %d of the adapters", dtype); return CSB_ERR_DTYPE; }
    if (rank > kMaxRank) { set_error("rank %d, at most %d", rank, kMaxRank); return CSB_ERR_UNSUPPORTED; }
    if (batch == 0) return CSB_OK;
    if (!X || !Y || !which) { set_error("X, Y or which is NULL"); return CSB_ERR_INVALID_ARG; }
    if (count > 0 && (!down || !up || !workspace)) { set_error("down, up or workspace is NULL"); return CSB_ERR_INVALID_ARG; }
    if (ldx < A->cols || ldy < A->rows) { set_error("ldx=%lld < cols or ldy=%lld < rows", (long long)ldx, (long long)ldy); return CSB_ERR_SHAPE; }
    const int64_t need = csb::workspace_bytes(A->cols, batch, rank);
    if (count > 0 && workspace_size < need) { set_error("workspace of %lld bytes, %lld needed", (long long)workspace_size, (long long)need); return CSB_ERR_INVALID_ARG; }
    if (A->device < 0) { set_error("matrix was encoded host-only (device = -1)"); return CSB_ERR_UNSUPPORTED; }
    if (A->val_dtype == CSB_Q16) { set_error("fixed-point handles serve csb_spmm_q16 only"); return CSB_ERR_UNSUPPORTED; }
    int current = -1;
    CSB_CUDA(cudaGetDevice(&current));
    if (current != A->device) { set_error("the matrix is on device %d, the current device is %d", A->device, current); return CSB_ERR_INVALID_ARG; }
    if (count == 0) return guarded([&] { return product_any(A, X, ldx, batch, Y, ldy, stream); });
    AdapterArgs a{};
    a.X = X; a.Y = Y; a.down = down; a.up = up; a.which = which; a.ranks = ranks; a.scales = scales; a.part = static_cast<float*>(workspace);
    a.ldx = ldx; a.ldy = ldy; a.batch = batch; a.count = count; a.rank = rank; a.rank_pad = rank_pad(rank); a.rows = (int)A->rows; a.cols = (int)A->cols;
    a.split_cols = split_columns(A->cols, batch); a.splits = (a.cols + a.split_cols - 1) / a.split_cols;
    return dtype == CSB_F32 ? adapters_on_device<float>(A, a, stream) : dtype == CSB_F16 ? adapters_on_device<__half>(A, a, stream)
                                                                                      : adapters_on_device<__nv_bfloat16>(A, a, stream);
}

}  // extern "C"
