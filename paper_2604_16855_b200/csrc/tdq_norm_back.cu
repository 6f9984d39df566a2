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

constexpr int kSumLanes = 16;                  // threads that share a column of the last sum

struct NormBackArgs {
    const void *x, *dy, *add;
    void* dx;
    const float *w, *mean, *rstd;
    float* part;                               // [blocks][2][C]
    int64_t M, x_stride, dy_stride, add_stride, dx_stride;   // strides in elements
    int32_t C;
    bool w_vec;                                // weights on the 16-byte grid
};

// Threads of a block: as many whole groups as 80 registers a thread allow (128 for rows off the grid; 64 where a row takes more threads; binary32 with 64 for all: 9000 x 768
// 16.4 us for 15.5).  Whether the next row is on its way while one is worked on.
template <int T, bool VEC> constexpr int kBackThreads = T > 384 ? T : (VEC ? 768 : 512) / T * T;
template <int T, int V> constexpr int kBackAhead = V == 1 && T <= 768 ? 1 : 0;

// T threads a row, V vectors each; VEC: rows on the 16-byte grid.
template <int DT, int T, int V, bool VEC>
__global__ void __launch_bounds__(kBackThreads<T, VEC>, 1) layer_norm_back_kernel(const NormBackArgs a) {
    using E = typename Elem<DT>::T;
    constexpr int P = kPerVec<DT>, kThreads = kBackThreads<T, VEC>, kGroups = kThreads / T, D = kBackAhead<T, V>;
    constexpr bool KEEP = V == 1;                            // weights in registers
    static_assert(T <= 32 || kGroups <= kMaxGroups, "barriers");
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ __align__(8) float room[kGroups][2][2 * (T > 32 ? T / 32 : 1)];
    pdl_wait();
    pdl_trigger();
    const int group = (int)threadIdx.x / T, t = (int)threadIdx.x % T, n = a.C;
    uint4* stage = reinterpret_cast<uint4*>(smem_raw) + (VEC ? 0 : group * 3 * kStageVecs<T, V>);   // x, dy, add; the output takes the first
    constexpr int H = P / 2;                                 // pairs of a vector
    const float inv = __fdiv_rn(1.f, (float)n);
    float2 dw[V * H], db[V * H];
#pragma unroll
    for (int i = 0; i < V * H; ++i) dw[i] = db[i] = two(0.f);
    float2 w[KEEP ? V * H : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < V; ++i) load_weight_pairs<P>(a.w, a.w_vec, (t + T * i) * P, n, 1.f, w + i * H);
    }
    // rows are counted in 32 bits, and addresses made anew from them: kept, they take twenty registers
    const uint32_t M = (uint32_t)a.M, step = gridDim.x * kGroups, in_warp = T >= 32 ? 0u : (uint32_t)group % (32 / T);
    uint32_t m = blockIdx.x * kGroups + (uint32_t)group;     // groups of a warp go on together, until the first one's rows end
    struct Item {
        Row<DT, T, V, VEC> x, dy;
        float mean, rstd;
    } ring[D + 1];
    Row<DT, T, V, VEC> ar;
    const auto fetch = [&](Item& r, uint32_t at) {
        const bool on = at < M;
        r.x.fetch(reinterpret_cast<const E*>(a.x) + (int64_t)at * a.x_stride, n, t, on);
        r.dy.fetch(reinterpret_cast<const E*>(a.dy) + (int64_t)at * a.dy_stride, n, t, on);
        r.mean = on ? __ldg(a.mean + at) : 0.f;
        r.rstd = on ? __ldg(a.rstd + at) : 0.f;
    };
    if constexpr (D > 0) fetch(ring[0], m);
    int turn = 0;
    const auto work = [&](Item& row, Item& then) {
        const bool on = m < M;
        fetch(then, m + D * step);                           // D == 0: this row
        if (a.add) ar.fetch(reinterpret_cast<const E*>(a.add) + (int64_t)m * a.add_stride, n, t, on);
        uint4 xv[V], dv[V], av[V];
        if constexpr (!VEC) {
            group_sync<T>(group);
            row.x.put(stage, t);
            row.dy.put(stage + kStageVecs<T, V>, t);
            group_sync<T>(group);
        }
        row.x.take(stage, n, t, xv);
        row.dy.take(stage + (VEC ? 0 : kStageVecs<T, V>), n, t, dv);
        const float2 mu = two(-row.mean), rs = two(row.rstd);
        float2 s0 = two(0.f), s1 = two(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int first = (t + T * i) * P;
            float2 xf[H], df[H], wl[H];
            widen_pairs<DT>(xv[i], xf);
            widen_pairs<DT>(dv[i], df);
            if constexpr (!KEEP) load_weight_pairs<P>(a.w, a.w_vec, first, n, 1.f, wl);
#pragma unroll
            for (int q = 0; q < H; ++q) {                    // behind the row dy is 0, and h is kept out of what it could make NaN
                float2 h = __fmul2_rn(__fadd2_rn(xf[q], mu), rs);
                if (VEC ? first >= n : first + 2 * q >= n) h = two(0.f);
                else if (!VEC && first + 2 * q + 1 >= n) h.y = 0.f;
                const float2 g = __fmul2_rn(df[q], KEEP ? w[KEEP ? i * H + q : 0] : wl[q]);
                s0 = __fadd2_rn(s0, g);
                s1 = __ffma2_rn(g, h, s1);
                dw[i * H + q] = __ffma2_rn(df[q], h, dw[i * H + q]);
                db[i * H + q] = __fadd2_rn(db[i * H + q], df[q]);
            }
        }
        const float2 s = group_sum2<T>(make_float2(s0.x + s0.y, s1.x + s1.y), room[group][turn], group, t);
        turn ^= 1;
        const float2 c0 = two(-s.x * inv), c1 = two(-s.y * inv);
        if (a.add) {
            if constexpr (!VEC) {
                ar.put(stage + 2 * kStageVecs<T, V>, t);     // read again only behind the next row's meeting
                group_sync<T>(group);
            }
            ar.take(stage + (VEC ? 0 : 2 * kStageVecs<T, V>), n, t, av);
        }
        E* dx = reinterpret_cast<E*>(a.dx) + (int64_t)m * a.dx_stride;
        uint4 out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int first = (t + T * i) * P;
            float2 xf[H], df[H], wl[H], r[H];
            forget(xv[i]);                                   // made again: held, what the first pass made of the row leaves too few registers
            forget(dv[i]);
            widen_pairs<DT>(xv[i], xf);
            widen_pairs<DT>(dv[i], df);
            if constexpr (!KEEP) load_weight_pairs<P>(a.w, a.w_vec, first, n, 1.f, wl);
#pragma unroll
            for (int q = 0; q < H; ++q) {
                const float2 h = __fmul2_rn(__fadd2_rn(xf[q], mu), rs), g = __fmul2_rn(df[q], KEEP ? w[KEEP ? i * H + q : 0] : wl[q]);
                r[q] = __fmul2_rn(rs, __ffma2_rn(h, c1, __fadd2_rn(g, c0)));
            }
            if (a.add) {
                float2 af[H];
                widen_pairs<DT>(av[i], af);
#pragma unroll
                for (int q = 0; q < H; ++q) r[q] = __fadd2_rn(r[q], af[q]);
            }
            out[i] = narrow_pairs<DT>(r);
            if (VEC && first < n && on) reinterpret_cast<uint4*>(dx)[t + T * i] = out[i];
        }
        if constexpr (!VEC) store_row_ragged<DT, T, V>(dx, n, t, group, stage, out, on);
        m += step;
    };
    while (m - in_warp < M) {
        work(ring[0], ring[D]);
        if constexpr (D > 0) {
            if (m - in_warp >= M) break;
            work(ring[1], ring[0]);
        }
    }
    // the groups' sums, a channel's next to one another
    float* part = a.part + (int64_t)blockIdx.x * 2 * n;
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const int c = (t + T * i) * P + q;
                const float2 u = dw[i * H + q / 2], v = db[i * H + q / 2];
                if (c < n) { part[c] = q & 1 ? u.y : u.x; part[n + c] = q & 1 ? v.y : v.x; }
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
                    const float2* d = (which ? db : dw) + i * H + q / 2;
                    *reinterpret_cast<float4*>(sums + group * kCols + (t + T * i) * P + q) = make_float4(d[0].x, d[0].y, d[1].x, d[1].y);
                }
            __syncthreads();
            for (int c = (int)threadIdx.x; c < n; c += kThreads) {
                float v = 0.f;
#pragma unroll 16
                for (int g = 0; g < kGroups; ++g) v += sums[g * kCols + c];
                part[which * n + c] = v;
            }
        }
    }
}

// out[c] = sum over `blocks` rows of part[.][c], in order within each of kSumLanes threads, then theirs in pairs (one after another the rounding error of 1021 x 2000 is
// 1.10e-7 instead of 0.96e-7 of a column's sum)
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
        float v[kSumLanes];
#pragma unroll
        for (int i = 0; i < kSumLanes; ++i) v[i] = sums[i][lane];
#pragma unroll
        for (int d = 1; d < kSumLanes; d *= 2)
#pragma unroll
            for (int i = 0; i < kSumLanes; i += 2 * d) v[i] += v[i + d];
        float* out = c < C ? dw : db;
        if (out) out[c < C ? c : c - C] = v[0];
    }
}

template <int DT, int T, int V, bool VEC>
cudaError_t launch_back(const NormBackArgs& a, unsigned blocks, int dev, cudaStream_t st) {
    constexpr int kThreads = kBackThreads<T, VEC>, kGroups = kThreads / T;
    constexpr int kStage = VEC ? 0 : kGroups * 3 * kStageVecs<T, V> * 16, kSums = kGroups > 1 ? kGroups * T * V * kPerVec<DT> * 4 : 0, kSmem = kStage > kSums ? kStage : kSums;
    auto* kernel = layer_norm_back_kernel<DT, T, V, VEC>;
    static std::atomic<uint64_t> done{0};
    if (kSmem > 40 * 1024) {
        const cudaError_t e = allow_smem(kernel, kSmem, done, dev);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3(blocks), dim3(kThreads), kSmem, st, a);
}
template <int DT, bool VEC>
cudaError_t pick_back(const NormBackArgs& a, RowShape s, unsigned blocks, int dev, cudaStream_t st) {
#define TDQ_SHAPE(T, V) if (s.t == T && s.v == V) return launch_back<DT, T, V, VEC>(a, blocks, dev, st)
    TDQ_SHAPE(8, 1); TDQ_SHAPE(16, 1); TDQ_SHAPE(32, 1); TDQ_SHAPE(64, 1); TDQ_SHAPE(96, 1); TDQ_SHAPE(128, 1); TDQ_SHAPE(192, 1); TDQ_SHAPE(256, 1);
    TDQ_SHAPE(384, 1); TDQ_SHAPE(512, 1); TDQ_SHAPE(768, 1); TDQ_SHAPE(1024, 1); TDQ_SHAPE(1024, 2);
    if constexpr (DT == TDQ_F32) TDQ_SHAPE(1024, 4);
#undef TDQ_SHAPE
    return cudaErrorInvalidValue;
}
template <int DT>
cudaError_t backward(const NormBackArgs& a, bool vec, unsigned blocks, int dev, cudaStream_t st) {
    // A vector a thread: the column sums of more would leave no registers for the next row, and two or three in 384 or 512 threads an SM took longer (18464 x 768 bf16
    // with an addend 39 us, now 28), as rows by asynchronous copies through shared memory did (29).
    static const int threads[] = {8, 16, 32, 64, 96, 128, 192, 256, 384, 512, 768, 1024};
    const int64_t vecs = (a.C + kPerVec<DT> - 1) / kPerVec<DT>;
    RowShape s = {1024, vecs <= 1024 ? 1 : vecs <= 2048 ? 2 : 4};
    for (int t : threads)
        if (t >= vecs) { s.t = t; break; }
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
        a.w_vec = !off_grid(weight, 16);
        const bool vec = C * (int64_t)esz % 16 == 0 && on_grid(x, x_row_stride, M, esz) && on_grid(dy, dy_row_stride, M, esz) && on_grid(dx, dx_row_stride, M, esz) &&
                         (!add || on_grid(add, add_row_stride, M, esz));
        const unsigned b = (unsigned)blocks;
        const cudaError_t e = dtype == TDQ_F32 ? backward<TDQ_F32>(a, vec, b, dev, st) : dtype == TDQ_BF16 ? backward<TDQ_BF16>(a, vec, b, dev, st)
                                                                                                         : backward<TDQ_F16>(a, vec, b, dev, st);
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
