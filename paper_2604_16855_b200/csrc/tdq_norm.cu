// tdq_layer_norm: the norm in front of a layer, in the input's type or straight to the E4M3 codes that the 8-bit layer takes.
//
//   mean = 1/C sum x;   rstd = 1 / sqrt(1/C sum (x - mean)^2 + eps);   y = (x - mean) rstd w + b
//
// Bound by HBM: the input is read once and the output written once.  Blocks stay and go through rows, the next two already on their way (one, or none, where a row's
// vectors or threads are many: kAhead), with the weights in registers (one row a group of a block that ends with it: 16384 x 2048 bf16 38 us, now 26).  To codes it is bound by
// latency: 16 warps an SM, at 128 registers a thread, behind a row's two sums, its blocks' maxima and their quotients (56 % of the issue slots; 18464 x 768 bf16 13 us where the
// bytes take 7).  A row stays in the registers of the threads that share it, as binary32 between its passes: sum, then sum of squares about the mean (not
// sum x^2 - C mean^2, which loses what a far mean leaves), then the outputs.  Sums are binary32: lane by lane, then a butterfly, in the same order every time.
// Rows off the 16-byte grid pass through shared memory: aligned vectors in, words shifted out, and the other way round for the output.
#include "tdq_rows.cuh"

namespace tdq {
namespace {

struct NormArgs {
    const void* x;
    void* y;
    const float *w, *b;
    uint8_t* codes;
    float *scale, *mean, *rstd;
    int64_t M, x_stride, y_stride;             // strides in elements
    int32_t C, Kb;                             // channels, blocks of 128
    float eps;
    bool pow2, w_vec;                          // weights on the 16-byte grid
};

template <int T> constexpr int kNormThreads = T < 256 ? 256 : T;
// Rows on their way while one is worked on (none where T is for few rows), and whether the weights stay in registers.
template <int T, int V, bool CODES, bool VEC> constexpr int kAhead = T == 1024 ? 0 : V <= 2 || (VEC && !CODES) ? 2 : 1;
template <int T, int V> constexpr bool kKeepWeights = T < 1024 && V <= 3;

// Blocks go through rows, 1 / T of a block a row.  CODES: E4M3 codes and scales instead of y.
template <int DT, int T, int V, bool CODES, bool VEC>
__global__ void __launch_bounds__(kNormThreads<T>, T > 256 ? 1 : V == 1 ? (VEC ? 4 : 3) : 2) layer_norm_kernel(const NormArgs a) {
    using E = typename Elem<DT>::T;
    constexpr int P = kPerVec<DT>, kGroups = kNormThreads<T> / T, D = kAhead<T, V, CODES, VEC>;
    constexpr bool KEEP = kKeepWeights<T, V>;
    static_assert(T <= 32 || kGroups <= kMaxGroups, "barriers");
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float room[kGroups][2][T > 32 ? T / 32 : 1];
    pdl_wait();
    pdl_trigger();
    const int group = (int)threadIdx.x / T, t = (int)threadIdx.x % T, n = a.C;
    uint4* stage = reinterpret_cast<uint4*>(smem_raw) + (VEC ? 0 : group * kStageVecs<T, V>);
    constexpr int H = P / 2;                                 // pairs of a vector
    const uint32_t M = (uint32_t)a.M, step = gridDim.x * kGroups, in_warp = T >= 32 ? 0u : (uint32_t)group % (32 / T);
    uint32_t m = blockIdx.x * kGroups + (uint32_t)group;     // groups of a warp go on together, until the first one's rows end
    Row<DT, T, V, VEC> ring[D + 1];
    const auto fetch = [&](Row<DT, T, V, VEC>& r, uint32_t at) { r.fetch(reinterpret_cast<const E*>(a.x) + (int64_t)at * a.x_stride, n, t, at < M); };
#pragma unroll
    for (int i = 0; i <= D; ++i) fetch(ring[i], m + i * step);
    float2 w[KEEP ? V * H : 1], b[KEEP ? V * H : 1];
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            load_weight_pairs<P>(a.w, a.w_vec, (t + T * i) * P, n, 1.f, w + i * H);
            load_weight_pairs<P>(a.b, a.w_vec, (t + T * i) * P, n, 0.f, b + i * H);
        }
    }
    const float inv = __fdiv_rn(1.f, (float)n);
    const auto work = [&](Row<DT, T, V, VEC>& row) {
        const bool on = m < M;
        float2 f[V * H];
        {
            uint4 v[V];
            if constexpr (!VEC) {
                group_sync<T>(group);
                row.put(stage, t);
                group_sync<T>(group);
            }
            row.take(stage, n, t, v);
#pragma unroll
            for (int i = 0; i < V; ++i) widen_pairs<DT>(v[i], f + i * H);
        }
        fetch(row, m + (D + 1) * step);
        float2 sum = f[0];
#pragma unroll
        for (int i = 1; i < V * H; ++i) sum = __fadd2_rn(sum, f[i]);
        const float mean = group_sum<T>(sum.x + sum.y, room[group][0], group, t) * inv;
        sum = two(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int first = (t + T * i) * P;
#pragma unroll
            for (int q = 0; q < H; ++q) {
                float2& d = f[i * H + q];
                d = __fadd2_rn(d, two(-mean));
                // behind the row there are no deviations; on the grid a vector lies in the row or behind it, else it may end inside
                if (VEC ? first >= n : first + 2 * q >= n) d = two(0.f);
                else if (!VEC && first + 2 * q + 1 >= n) d.y = 0.f;
                sum = __ffma2_rn(d, d, sum);
            }
        }
        const float rstd = __frcp_rn(__fsqrt_rn(fmaf(group_sum<T>(sum.x + sum.y, room[group][1], group, t), inv, a.eps)));
        if (t == 0 && on) {
            if (a.mean) a.mean[m] = mean;
            if (a.rstd) a.rstd[m] = rstd;
        }
        uint32_t mx[V];
        uint4 out[V];
        E* const y_row = reinterpret_cast<E*>(a.y) + (int64_t)m * a.y_stride;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int idx = t + T * i, first = idx * P;
            float2 wl[H], bl[H], *y = f + i * H;
            if constexpr (!KEEP) {
                load_weight_pairs<P>(a.w, a.w_vec, first, n, 1.f, wl);
                load_weight_pairs<P>(a.b, a.w_vec, first, n, 0.f, bl);
            }
            mx[i] = 0;
#pragma unroll
            for (int q = 0; q < H; ++q) {
                y[q] = __ffma2_rn(__fmul2_rn(y[q], two(rstd)), KEEP ? w[KEEP ? i * H + q : 0] : wl[q], KEEP ? b[KEEP ? i * H + q : 0] : bl[q]);
                if constexpr (CODES) mx[i] = max(mx[i], max(__float_as_uint(y[q].x) & 0x7fffffffu, __float_as_uint(y[q].y) & 0x7fffffffu));
            }
            if constexpr (!CODES) {
                out[i] = narrow_pairs<DT>(y);
                if (VEC && first < n && on) reinterpret_cast<uint4*>(y_row)[idx] = out[i];
            }
        }
        if constexpr (CODES) {
            // 128 channels are kTeam neighbouring threads; behind the row weights are 1, biases and deviations 0 (or all NaN with the row), so y is 0.  The i-th thread of
            // a team works out the scale of its i-th block, once for all, and the others take it from there.
            constexpr int kTeam = 128 / P;
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int d = 1; d < kTeam; d <<= 1) mx[i] = max(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], d));
                if ((t & (kTeam - 1)) == i) mine = mx[i];
            }
            float scale, inverse;
            if (a.pow2) block_scale<true>(mine, scale, inverse);
            else block_scale<false>(mine, scale, inverse);
            const int block = t / kTeam + (t & (kTeam - 1)) * (T / kTeam);   // of the scale
            if (on && (t & (kTeam - 1)) < V && block < a.Kb) a.scale[(int64_t)m * a.Kb + block] = scale;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int idx = t + T * i;
                const float r = __shfl_sync(0xffffffffu, inverse, i, kTeam);
                const float2* y = f + i * H;
                if (on && idx < a.Kb * kTeam) {
                    uint8_t* dst = a.codes + ((int64_t)m * a.Kb * 128 + idx * P);
                    const uint32_t c0 = cvt4(y[0].x, y[0].y, y[1].x, y[1].y, r);
                    if constexpr (P == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(c0, cvt4(y[2].x, y[2].y, y[3].x, y[3].y, r));
                    else *reinterpret_cast<uint32_t*>(dst) = c0;
                }
            }
        }
        if constexpr (!CODES && !VEC) store_row_ragged<DT, T, V>(y_row, n, t, group, stage, out, on);
        m += step;
    };
    while (true) {
#pragma unroll
        for (int i = 0; i <= D; ++i) {
            if (m - in_warp >= M) return;
            work(ring[i]);
        }
    }
}

template <int DT, int T, int V, bool CODES, bool VEC>
cudaError_t launch_forward(const NormArgs& a, int n_sm, int dev, cudaStream_t st) {
    constexpr int kThreads = kNormThreads<T>, kGroups = kThreads / T, kSmem = VEC ? 0 : kGroups * kStageVecs<T, V> * 16;
    auto* kernel = layer_norm_kernel<DT, T, V, CODES, VEC>;
    static std::atomic<uint64_t> done{0};
    static std::atomic<int> per_sm[kMaxDevices];
    if (kSmem > 40 * 1024) {
        const cudaError_t e = allow_smem(kernel, kSmem, done, dev);
        if (e != cudaSuccess) return e;
    }
    const int64_t most = (int64_t)n_sm * blocks_per_sm(kernel, kThreads, kSmem, per_sm, dev), need = (a.M + kGroups - 1) / kGroups;
    return launch_pdl(kernel, dim3((unsigned)(need < most ? need : most)), dim3(kThreads), kSmem, st, a);
}
template <int DT, bool CODES, bool VEC>
cudaError_t pick_forward(const NormArgs& a, RowShape s, int n_sm, int dev, cudaStream_t st) {
#define TDQ_SHAPE(T, V) if (s.t == T && s.v == V) return launch_forward<DT, T, V, CODES, VEC>(a, n_sm, dev, st)
    if constexpr (!CODES) TDQ_SHAPE(8, 1);
    if constexpr (!CODES || DT != TDQ_F32) TDQ_SHAPE(16, 1);
    TDQ_SHAPE(32, 1); TDQ_SHAPE(32, 2); TDQ_SHAPE(32, 3); TDQ_SHAPE(64, 1); TDQ_SHAPE(64, 2); TDQ_SHAPE(64, 3);
    TDQ_SHAPE(128, 1); TDQ_SHAPE(128, 2); TDQ_SHAPE(128, 3); TDQ_SHAPE(256, 1); TDQ_SHAPE(256, 2);
    TDQ_SHAPE(512, 1); TDQ_SHAPE(512, 2); TDQ_SHAPE(1024, 1); TDQ_SHAPE(1024, 2); TDQ_SHAPE(1024, 3); TDQ_SHAPE(1024, 4);
#undef TDQ_SHAPE
    return cudaErrorInvalidValue;
}
template <int DT>
cudaError_t forward(const NormArgs& a, bool vec, int n_sm, int dev, cudaStream_t st) {
    const int64_t n = a.codes ? (int64_t)a.Kb * 128 : a.C;   // codes behind C are written too
    const RowShape s = row_shape((n + kPerVec<DT> - 1) / kPerVec<DT>, a.M, n_sm, a.codes ? 128 / kPerVec<DT> : 8, 1024);
    if (a.codes) return vec ? pick_forward<DT, true, true>(a, s, n_sm, dev, st) : pick_forward<DT, true, false>(a, s, n_sm, dev, st);
    return vec ? pick_forward<DT, false, true>(a, s, n_sm, dev, st) : pick_forward<DT, false, false>(a, s, n_sm, dev, st);
}

}  // namespace
}  // namespace tdq

using namespace tdq;

extern "C" tdq_status tdq_layer_norm(const void* x, tdq_dtype dtype, int64_t M, int64_t C, int64_t x_row_stride, const float* weight, const float* bias,
                                     float eps, uint32_t flags, void* y, int64_t y_row_stride, uint8_t* codes, float* scale, float* mean, float* rstd,
                                     void* cuda_stream) {
    if (!known_dtype(dtype) || M < 0 || C <= 0 || x_row_stride < C || !(eps >= 0.f) || (flags & ~TDQ_NORM_POW2)) return TDQ_ERR_INVALID_ARG;
    if (y ? y_row_stride < C || codes || scale || flags : M > 0 && (!codes || !scale)) return TDQ_ERR_INVALID_ARG;
    if (M == 0) return TDQ_OK;
    if (!x) return TDQ_ERR_INVALID_ARG;
    const uintptr_t esz = dtype == TDQ_F32 ? 4 : 2;
    if (off_grid(x, esz) || off_grid(y, esz) || off_grid(weight, 4) || off_grid(bias, 4) || off_grid(codes, 16) || off_grid(scale, 4) || off_grid(mean, 4) || off_grid(rstd, 4)) return TDQ_ERR_ALIGNMENT;
    if (C > kMaxRow || M > INT32_MAX) return TDQ_ERR_UNSUPPORTED;
    int dev = 0;
    const int n_sm = current_device_sm_count(&dev);
    if (n_sm <= 0) return TDQ_ERR_CUDA;
    NormArgs a = {};
    a.x = x; a.y = y; a.w = weight; a.b = bias; a.codes = codes; a.scale = scale; a.mean = mean; a.rstd = rstd;
    a.M = M; a.x_stride = x_row_stride; a.y_stride = y_row_stride; a.C = (int32_t)C; a.Kb = (int32_t)fp8_blocks(C); a.eps = eps; a.pow2 = (flags & TDQ_NORM_POW2) != 0; a.w_vec = !off_grid(weight, 16) && !off_grid(bias, 16);
    const bool vec = C * (int64_t)esz % 16 == 0 && on_grid(x, x_row_stride, M, esz) && (!y || on_grid(y, y_row_stride, M, esz));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dtype == TDQ_F32 ? forward<TDQ_F32>(a, vec, n_sm, dev, st) : dtype == TDQ_BF16 ? forward<TDQ_BF16>(a, vec, n_sm, dev, st)
                                                                                                        : forward<TDQ_F16>(a, vec, n_sm, dev, st);
    if (e == cudaSuccess) g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(e);
}
