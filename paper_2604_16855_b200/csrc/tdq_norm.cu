// tdq_layer_norm: the norm in front of a layer, in the input's type or straight to the E4M3 codes that the 8-bit layer takes.
//
//   mean = 1/C sum x;   rstd = 1 / sqrt(1/C sum (x - mean)^2 + eps);   y = (x - mean) rstd w + b
//
// Bound by HBM: the input is read once and the output written once.  A row stays in the registers of the threads that share it (a warp up to 1024
// channels of 16 bits, then 128 to 1024 threads), as binary32 between its passes: sum, then sum of squares about the mean (not sum x^2 - C mean^2,
// which loses what a far mean leaves), then the outputs.  Sums are binary32: lane by lane, then a butterfly, in the same order every time.
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
    bool pow2;
};

// Forward.  R rows at a time in a group (of warps only), which share the loads of w and b.  CODES: E4M3 codes and scales instead of y.
template <int DT, int T, int V, int R, bool CODES, bool VEC>
__global__ void __launch_bounds__(T < 256 ? 256 : T) layer_norm_kernel(const NormArgs a) {
    using E = typename Elem<DT>::T;
    constexpr int P = kPerVec<DT>, kThreads = T < 256 ? 256 : T, kGroups = kThreads / T;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ float room[kGroups][2][T > 32 ? T / 32 : 1];
    pdl_wait();
    pdl_trigger();
    const int group = (int)threadIdx.x / T, t = (int)threadIdx.x % T;
    uint4* stage = reinterpret_cast<uint4*>(smem_raw) + (VEC ? 0 : group * kStageVecs<T, V>);
    const int64_t row0 = ((int64_t)blockIdx.x * kGroups + group) * R;
    if (row0 >= a.M) return;                                 // the whole group
    const int n = a.C;
    float f[R][V * P], mean[R], rstd[R];
    {
        uint4 v[R][V];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t m = row0 + r < a.M ? row0 + r : a.M - 1;   // a row past the end: the last one once more, not stored
            const E* src = reinterpret_cast<const E*>(a.x) + m * a.x_stride;
            if constexpr (VEC) load_row<DT, T, V>(src, n, t, v[r]);
            else load_row_ragged<DT, T, V>(src, n, t, group, stage, v[r]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) widen_vec<DT>(v[r][i], f[r] + i * P);
    }
    const float inv = __fdiv_rn(1.f, (float)n);
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        s[r] = 0.f;
#pragma unroll
        for (int i = 0; i < V * P; ++i) s[r] += f[r][i];
    }
    group_sum<T, R>(s, room[group][0], group, t);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        mean[r] = s[r] * inv;
        s[r] = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int first = (t + T * i) * P;
#pragma unroll
            for (int q = 0; q < P; ++q) {
                f[r][i * P + q] -= mean[r];
                // a vector lies in the row or behind it, where rows are on the grid; else it may end inside
                if (VEC ? first < n : first + q < n) s[r] = fmaf(f[r][i * P + q], f[r][i * P + q], s[r]);
            }
        }
    }
    group_sum<T, R>(s, room[group][1], group, t);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        rstd[r] = __frcp_rn(__fsqrt_rn(fmaf(s[r], inv, a.eps)));
        if (t == 0 && row0 + r < a.M) {
            if (a.mean) a.mean[row0 + r] = mean[r];
            if (a.rstd) a.rstd[row0 + r] = rstd[r];
        }
    }
    uint4 out[R][V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int idx = t + T * i, first = idx * P;
        float w[P], b[P];
        load_weights<P, VEC>(a.w, first, n, 1.f, w);
        load_weights<P, VEC>(a.b, first, n, 0.f, b);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float* y = f[r] + i * P;
#pragma unroll
            for (int q = 0; q < P; ++q) y[q] = fmaf(y[q] * rstd[r], w[q], b[q]);
            if constexpr (!CODES) {
                if constexpr (VEC) {
                    if (first < n && row0 + r < a.M)
                        reinterpret_cast<uint4*>(reinterpret_cast<E*>(a.y) + (row0 + r) * a.y_stride)[idx] = narrow_vec<DT>(y);
                } else {
                    out[r][i] = narrow_vec<DT>(y);
                }
            } else {
                // 128 channels are 128 / P neighbouring threads of the group
                uint32_t mx = 0;
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    if (VEC ? first >= n : first + q >= n) y[q] = 0.f;
                    mx = max(mx, __float_as_uint(y[q]) & 0x7fffffffu);
                }
#pragma unroll
                for (int d = 1; d < 128 / P; d <<= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                float scale, inv_scale;
                if (a.pow2) block_scale<true>(mx, scale, inv_scale);
                else block_scale<false>(mx, scale, inv_scale);
                if (idx < a.Kb * (128 / P) && row0 + r < a.M) {
                    uint8_t* dst = a.codes + ((row0 + r) * a.Kb * 128 + first);
                    const uint32_t c0 = cvt4(y[0], y[1], y[2], y[3], inv_scale);
                    if constexpr (P == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(c0, cvt4(y[4], y[5], y[6], y[7], inv_scale));
                    else *reinterpret_cast<uint32_t*>(dst) = c0;
                    if ((idx & (128 / P - 1)) == 0) a.scale[(row0 + r) * a.Kb + idx / (128 / P)] = scale;
                }
            }
        }
    }
    if constexpr (!CODES && !VEC) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (row0 + r < a.M)                              // the whole group
                store_row_ragged<DT, T, V>(reinterpret_cast<E*>(a.y) + (row0 + r) * a.y_stride, n, t, group, stage, out[r]);
    }
}

template <int DT, int T, int V, bool CODES, bool VEC>
cudaError_t launch_forward(const NormArgs& a, int dev, cudaStream_t st) {
    constexpr int R = T == 32 ? 2 : 1, kThreads = T < 256 ? 256 : T, kGroups = kThreads / T;
    const int smem = VEC ? 0 : kGroups * kStageVecs<T, V> * 16;
    auto* kernel = layer_norm_kernel<DT, T, V, R, CODES, VEC>;
    static std::atomic<uint64_t> done{0};
    if (smem > 48 * 1024) {
        const cudaError_t e = allow_smem(kernel, smem, done, dev);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(kernel, dim3((unsigned)((a.M + kGroups * R - 1) / (kGroups * R))), dim3(kThreads), smem, st, a);
}
template <int DT, bool CODES, bool VEC>
cudaError_t pick_forward(const NormArgs& a, RowShape s, int dev, cudaStream_t st) {
#define TDQ_SHAPE(T, V) if (s.t == T && s.v == V) return launch_forward<DT, T, V, CODES, VEC>(a, dev, st)
    TDQ_SHAPE(32, 1); TDQ_SHAPE(32, 2); TDQ_SHAPE(32, 4);
    TDQ_SHAPE(128, 1); TDQ_SHAPE(128, 2); TDQ_SHAPE(128, 4);
    TDQ_SHAPE(256, 1); TDQ_SHAPE(256, 4); TDQ_SHAPE(512, 1); TDQ_SHAPE(512, 4); TDQ_SHAPE(1024, 1); TDQ_SHAPE(1024, 4);
    if constexpr (VEC) { TDQ_SHAPE(32, 3); TDQ_SHAPE(128, 3); }
#undef TDQ_SHAPE
    return cudaErrorInvalidValue;
}
template <int DT>
cudaError_t forward(const NormArgs& a, bool vec, int n_sm, int dev, cudaStream_t st) {
    const int64_t n = a.codes ? (int64_t)a.Kb * 128 : a.C;   // codes behind C are written too
    const RowShape s = row_shape((n + kPerVec<DT> - 1) / kPerVec<DT>, a.M, n_sm, 1024, vec);
    if (a.codes) return vec ? pick_forward<DT, true, true>(a, s, dev, st) : pick_forward<DT, true, false>(a, s, dev, st);
    return vec ? pick_forward<DT, false, true>(a, s, dev, st) : pick_forward<DT, false, false>(a, s, dev, st);
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
    a.M = M; a.x_stride = x_row_stride; a.y_stride = y_row_stride; a.C = (int32_t)C; a.Kb = (int32_t)fp8_blocks(C); a.eps = eps; a.pow2 = (flags & TDQ_NORM_POW2) != 0;
    const bool vec = C * (int64_t)esz % 16 == 0 && on_grid(x, x_row_stride, M, esz) && (!y || on_grid(y, y_row_stride, M, esz)) && !off_grid(weight, 16) && !off_grid(bias, 16);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dtype == TDQ_F32 ? forward<TDQ_F32>(a, vec, n_sm, dev, st) : dtype == TDQ_BF16 ? forward<TDQ_BF16>(a, vec, n_sm, dev, st)
                                                                                                        : forward<TDQ_F16>(a, vec, n_sm, dev, st);
    if (e == cudaSuccess) g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(e);
}
