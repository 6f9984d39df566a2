// tdq_layer_norm_backward: the gradients of the norm.
//
//   g = dy w,  h = (x - mean) rstd;   dx = rstd (g - 1/C sum g - h 1/C sum g h) + add;   dw = sum_m dy h;   db = sum_m dy
//
// Bound by HBM: dy, x and add are read once and dx is written once.  One thread block per SM goes through rows with its threads on the same channels
// all the while, so that the column sums of dw and db stay in registers too; the groups of a block meet in shared memory, the blocks in the
// workspace, one row of sums each, which a second kernel adds in order.  No atomics: the same call gives the same bits.  All sums are binary32.
#include "tdq_rows.cuh"

namespace tdq {
namespace {

constexpr int kBackThreads = 512;              // of a block
constexpr int kSumLanes = 16;                  // threads that share a column of the last sum

struct NormBackArgs {
    const void *x, *dy, *add;
    void* dx;
    const float *w, *mean, *rstd;
    float* part;                               // [blocks][2][C]
    int64_t M, x_stride, dy_stride, add_stride, dx_stride;   // strides in elements
    int32_t C;
};

// T threads a row, V vectors each; VEC: rows on the 16-byte grid.
template <int DT, int T, int V, bool VEC>
__global__ void __launch_bounds__(kBackThreads, 1) layer_norm_back_kernel(const NormBackArgs a) {
    using E = typename Elem<DT>::T;
    constexpr int P = kPerVec<DT>, kGroups = kBackThreads / T;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float room[kGroups][2][2 * (T > 32 ? T / 32 : 1)];
    pdl_wait();
    pdl_trigger();
    const int group = (int)threadIdx.x / T, t = (int)threadIdx.x % T, n = a.C;
    uint4* stage = reinterpret_cast<uint4*>(smem_raw) + (VEC ? 0 : group * kStageVecs<T, V>);
    const float inv = __fdiv_rn(1.f, (float)n);
    float dw[V * P], db[V * P];
#pragma unroll
    for (int i = 0; i < V * P; ++i) dw[i] = db[i] = 0.f;
    int turn = 0;
#pragma unroll 1
    for (int64_t m = (int64_t)blockIdx.x * kGroups + group; m < a.M; m += (int64_t)gridDim.x * kGroups, turn ^= 1) {
        uint4 xv[V], dv[V], av[V];
        const E *x = reinterpret_cast<const E*>(a.x) + m * a.x_stride, *dy = reinterpret_cast<const E*>(a.dy) + m * a.dy_stride;
        const E* add = reinterpret_cast<const E*>(a.add) + m * a.add_stride;
        if constexpr (VEC) {
            load_row<DT, T, V>(x, n, t, xv);
            load_row<DT, T, V>(dy, n, t, dv);
            if (a.add) load_row<DT, T, V>(add, n, t, av);
        } else {
            load_row_ragged<DT, T, V>(x, n, t, group, stage, xv);
            load_row_ragged<DT, T, V>(dy, n, t, group, stage, dv);
            if (a.add) load_row_ragged<DT, T, V>(add, n, t, group, stage, av);
        }
        const float mean = __ldg(a.mean + m), rstd = __ldg(a.rstd + m);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int first = (t + T * i) * P;
            float xf[P], df[P], w[P];
            widen_vec<DT>(xv[i], xf);
            widen_vec<DT>(dv[i], df);
            load_weights<P, VEC>(a.w, first, n, 1.f, w);
#pragma unroll
            for (int q = 0; q < P; ++q) {                    // behind the row dy is 0, so whatever h is there adds nothing
                const float h = (xf[q] - mean) * rstd, g = df[q] * w[q];
                s[0] += g;
                s[1] = fmaf(g, h, s[1]);
                if (VEC || first + q < n) dw[i * P + q] = fmaf(df[q], h, dw[i * P + q]);
                db[i * P + q] += df[q];
            }
        }
        group_sum<T, 2>(s, room[group][turn], group, t);
        const float c0 = s[0] * inv, c1 = s[1] * inv;
        E* dx = reinterpret_cast<E*>(a.dx) + m * a.dx_stride;
        uint4 out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int first = (t + T * i) * P;
            float xf[P], df[P], w[P];
            widen_vec<DT>(xv[i], xf);
            widen_vec<DT>(dv[i], df);
            load_weights<P, VEC>(a.w, first, n, 1.f, w);
            float r[P];
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const float h = (xf[q] - mean) * rstd, g = df[q] * w[q];
                r[q] = rstd * (g - c0 - h * c1);
            }
            if (a.add) {
                float af[P];
                widen_vec<DT>(av[i], af);
#pragma unroll
                for (int q = 0; q < P; ++q) r[q] += af[q];
            }
            out[i] = narrow_vec<DT>(r);
            if (VEC && first < n) reinterpret_cast<uint4*>(dx)[t + T * i] = out[i];
        }
        if constexpr (!VEC) store_row_ragged<DT, T, V>(dx, n, t, group, stage, out);
    }
    // the groups' sums, a channel's next to one another
    float* part = a.part + (int64_t)blockIdx.x * 2 * n;
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const int c = (t + T * i) * P + q;
                if (c < n) { part[c] = dw[i * P + q]; part[n + c] = db[i * P + q]; }
            }
    } else {
        constexpr int kCols = T * V * P;
        float* sums = reinterpret_cast<float*>(smem_raw);    // [groups][kCols]
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int q = 0; q < P; q += 4) {
                    const float* d = (which ? db : dw) + i * P + q;
                    *reinterpret_cast<float4*>(sums + group * kCols + (t + T * i) * P + q) = make_float4(d[0], d[1], d[2], d[3]);
                }
            __syncthreads();
            for (int c = (int)threadIdx.x; c < n; c += kBackThreads) {
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < kGroups; ++g) v += sums[g * kCols + c];
                part[which * n + c] = v;
            }
        }
    }
}

// out[c] = sum over `blocks` rows of part[.][c], in order within each of kSumLanes threads, then theirs
__global__ void __launch_bounds__(32 * kSumLanes) column_sums_kernel(const float* __restrict__ part, int blocks, int C, float* __restrict__ dw, float* __restrict__ db) {
    __shared__ float sums[kSumLanes][33];
    pdl_wait();
    pdl_trigger();
    const int lane = (int)threadIdx.x & 31, y = (int)threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane, n2 = 2 * (int64_t)C;
    float s = 0.f;
    if (c < n2) {
#pragma unroll 4
        for (int p = y; p < blocks; p += kSumLanes) s += part[p * n2 + c];
    }
    sums[y][lane] = s;
    __syncthreads();
    if (y == 0 && c < n2) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < kSumLanes; ++i) s += sums[i][lane];
        float* out = c < C ? dw : db;
        if (out) out[c < C ? c : c - C] = s;
    }
}

template <int DT, int T, int V, bool VEC>
cudaError_t launch_back(const NormBackArgs& a, unsigned blocks, int dev, cudaStream_t st) {
    constexpr int kGroups = kBackThreads / T;
    const int stage = VEC ? 0 : kGroups * kStageVecs<T, V> * 16, sums = kGroups > 1 ? kGroups * T * V * kPerVec<DT> * 4 : 0;
    const int smem = stage > sums ? stage : sums;
    auto* kernel = layer_norm_back_kernel<DT, T, V, VEC>;
    static std::atomic<uint64_t> done{0};
    if (smem > 40 * 1024) {
        const cudaError_t e = allow_smem(kernel, smem, done, dev);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3(blocks), dim3(kBackThreads), smem, st, a);
}
template <int DT, bool VEC>
cudaError_t pick_back(const NormBackArgs& a, RowShape s, unsigned blocks, int dev, cudaStream_t st) {
#define TDQ_SHAPE(T, V) if (s.t == T && s.v == V) return launch_back<DT, T, V, VEC>(a, blocks, dev, st)
    TDQ_SHAPE(32, 1); TDQ_SHAPE(32, 2); TDQ_SHAPE(32, 4);
    TDQ_SHAPE(128, 1); TDQ_SHAPE(128, 2); TDQ_SHAPE(128, 4);
    TDQ_SHAPE(256, 1); TDQ_SHAPE(256, 4); TDQ_SHAPE(512, 1); TDQ_SHAPE(512, 4);
    if constexpr (VEC) { TDQ_SHAPE(32, 3); TDQ_SHAPE(128, 3); }
    if constexpr (DT == TDQ_F32) TDQ_SHAPE(512, 8);
#undef TDQ_SHAPE
    return cudaErrorInvalidValue;
}
template <int DT>
cudaError_t backward(const NormBackArgs& a, bool vec, unsigned blocks, int n_sm, int dev, cudaStream_t st) {
    const RowShape s = row_shape((a.C + kPerVec<DT> - 1) / kPerVec<DT>, a.M, n_sm, 512, vec);
    return vec ? pick_back<DT, true>(a, s, blocks, dev, st) : pick_back<DT, false>(a, s, blocks, dev, st);
}
int64_t back_blocks(int64_t M, int n_sm) { return M < n_sm ? M : n_sm; }

}  // namespace
}  // namespace tdq

using namespace tdq;

extern "C" size_t tdq_layer_norm_backward_workspace_bytes(int64_t M, int64_t C) {
    const int n_sm = current_device_sm_count();
    if (M <= 0 || C <= 0 || C > kMaxRow) return 0;
    return (size_t)back_blocks(M, n_sm > 0 ? n_sm : 148) * 2 * (size_t)C * 4;
}

extern "C" tdq_status tdq_layer_norm_backward(const void* dy, int64_t dy_row_stride, const void* x, int64_t x_row_stride, tdq_dtype dtype, int64_t M, int64_t C,
                                              const float* mean, const float* rstd, const float* weight, const void* add, int64_t add_row_stride, void* dx,
                                              int64_t dx_row_stride, float* dweight, float* dbias, void* workspace, size_t workspace_bytes,
                                              void* cuda_stream) {
    if (!known_dtype(dtype) || M < 0 || C <= 0 || dy_row_stride < C || x_row_stride < C || dx_row_stride < C || (add && add_row_stride < C)) return TDQ_ERR_INVALID_ARG;
    const uintptr_t esz = dtype == TDQ_F32 ? 4 : 2;
    if (M > 0 && (!dy || !x || !mean || !rstd || !dx)) return TDQ_ERR_INVALID_ARG;
    if (off_grid(dy, esz) || off_grid(x, esz) || off_grid(dx, esz) || off_grid(add, esz) || off_grid(mean, 4) || off_grid(rstd, 4) || off_grid(weight, 4) || off_grid(dweight, 4) || off_grid(dbias, 4) ||
        off_grid(workspace, 16))
        return TDQ_ERR_ALIGNMENT;
    if (C > kMaxRow || M > INT32_MAX) return TDQ_ERR_UNSUPPORTED;
    if (M == 0 && !dweight && !dbias) return TDQ_OK;
    int dev = 0;
    const int n_sm = current_device_sm_count(&dev);
    if (n_sm <= 0) return TDQ_ERR_CUDA;
    const int64_t blocks = back_blocks(M, n_sm);
    if (M > 0 && (!workspace || workspace_bytes < (size_t)blocks * 2 * (size_t)C * 4)) return TDQ_ERR_WORKSPACE;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (M > 0) {
        NormBackArgs a = {};
        a.x = x; a.dy = dy; a.add = add; a.dx = dx; a.w = weight; a.mean = mean; a.rstd = rstd; a.part = reinterpret_cast<float*>(workspace);
        a.M = M; a.x_stride = x_row_stride; a.dy_stride = dy_row_stride; a.add_stride = add_row_stride; a.dx_stride = dx_row_stride; a.C = (int32_t)C;
        const bool vec = C * (int64_t)esz % 16 == 0 && on_grid(x, x_row_stride, M, esz) && on_grid(dy, dy_row_stride, M, esz) && on_grid(dx, dx_row_stride, M, esz) &&
                         (!add || on_grid(add, add_row_stride, M, esz)) && !off_grid(weight, 16);
        const unsigned b = (unsigned)blocks;
        const cudaError_t e = dtype == TDQ_F32 ? backward<TDQ_F32>(a, vec, b, n_sm, dev, st) : dtype == TDQ_BF16 ? backward<TDQ_BF16>(a, vec, b, n_sm, dev, st)
                                                                                                         : backward<TDQ_F16>(a, vec, b, n_sm, dev, st);
        if (e != cudaSuccess) return cuda_status(e);
        g_launch_count.fetch_add(1, std::memory_order_relaxed);
    }
    if (dweight || dbias) {                                  // without rows: zeros
        const cudaError_t e = launch_pdl(column_sums_kernel, dim3((unsigned)((2 * C + 31) / 32)), dim3(32 * kSumLanes), 0, st,
                                         (const float*)workspace, (int)blocks, (int)C, dweight, dbias);
        if (e != cudaSuccess) return cuda_status(e);
        g_launch_count.fetch_add(1, std::memory_order_relaxed);
    }
    return TDQ_OK;
}
