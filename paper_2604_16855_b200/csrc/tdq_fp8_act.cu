// tdq_activation_backward_fp8: dz = dh activation'(z), z = code x scale kept in 8 bits.
//
// Bound by HBM: dh, a byte of z and dz an element; of 16 bits GELU's slope is bound by instructions as well (16384 x 4096 bf16 59 us, SiLU 51, ReLU 50; float32 GELU 88).  A vector of 16 bytes is
// eight or four channels, neighbouring lanes have neighbouring vectors, and a thread has two or four of them, 32 lanes apart.  Sixteen channels in a row a thread, whose
// accesses leave gaps: 62, 53, 50 and 102 us; blocks that stay and load ahead: 65, 54, 54 and 96.  Rows of dh or dz off the 16-byte grid go element by element,
// lanes along the row: twice the time in 16 bits (16384 x 4096 with a pitch of 4097 bf16 GELU 99 us, SiLU 85, float32 GELU 106).
#include "tdq_activation.cuh"
#include "tdq_rows.cuh"

namespace tdq {
namespace {

constexpr int kActThreads = 256;

struct ActArgs {
    const void* dh;
    void* dz;
    const uint8_t* codes;
    const float* scale;
    int64_t dh_stride, dz_stride;
    uint32_t n_blocks, Kb;
    int32_t C;
};

// two codes (low half of the word) as binary32
__device__ __forceinline__ float2 widen_codes(uint32_t two) {
    uint32_t h;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(h) : "r"(two));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// A block's scale, for the tanh form and SiLU 2^30 at most: with more every code but 0 has |z| >= 2^21, where the slopes are 0 or 1 whatever z is, and what they multiply on
// the way would pass binary32's range (from |z| = 1.2e13 on; code x scale itself does where the block's maximum is 248 x 2^120 or more).  An infinite scale counts as NaN.
// Once a vector; clamping z instead took 54.4 us for 52.3 (16384 x 4096 bf16, tanh form).
template <int ACT>
__device__ __forceinline__ float near_scale(float scale) {
    if constexpr (ACT == TDQ_ACT_GELU_TANH || ACT == TDQ_ACT_SILU) return fmaf(scale, 0.f, fmaxf(fminf(scale, 0x1p30f), -0x1p30f));
    return scale;
}

template <int DT> constexpr int kActVecs = DT == TDQ_F32 ? 2 : 4;   // a thread's (4 and 2: float32 88 us for 88, bf16 62 for 59)

template <int DT, int ACT>
__global__ void __launch_bounds__(kActThreads) act_back_kernel(const ActArgs a) {
    using E = typename Elem<DT>::T;
    constexpr int P = kPerVec<DT>, kLanes = 128 / P, V = kActVecs<DT>;         // lanes of a block
    pdl_wait();
    pdl_trigger();
    const uint32_t b0 = (blockIdx.x * (kActThreads / 32) + (threadIdx.x >> 5)) * (V * 32 / kLanes) + (threadIdx.x & 31) / kLanes, lane = threadIdx.x % kLanes;
    uint32_t m = b0 / a.Kb, k = b0 - m * a.Kb;
    uint4 v[V], *dst[V];
    uint32_t code[V][P / 4];
    float scale[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t b = b0 + i * (32 / kLanes);
        const int c = (int)(k * 128 + lane * P);
        dst[i] = nullptr;
        v[i] = make_uint4(0, 0, 0, 0);
        scale[i] = 0.f;
#pragma unroll
        for (int j = 0; j < P / 4; ++j) code[i][j] = 0;
        if (b < a.n_blocks && c < a.C) {
            v[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const E*>(a.dh) + (int64_t)m * a.dh_stride + c);
            dst[i] = reinterpret_cast<uint4*>(reinterpret_cast<E*>(a.dz) + (int64_t)m * a.dz_stride + c);
            const uint8_t* from = a.codes + (int64_t)b * 128 + lane * P;
            if constexpr (P == 8) {
                const uint2 r = __ldg(reinterpret_cast<const uint2*>(from));
                code[i][0] = r.x;
                code[i][P / 4 - 1] = r.y;
            } else code[i][0] = __ldg(reinterpret_cast<const uint32_t*>(from));
            scale[i] = __ldg(a.scale + b);
        }
        for (k += 32 / kLanes; k >= a.Kb; k -= a.Kb) ++m;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float f[P];
        widen_vec<DT>(v[i], f);
        const float near = near_scale<ACT>(scale[i]);
#pragma unroll
        for (int j = 0; j < P; j += 2) {
            const float2 z = __fmul2_rn(widen_codes(code[i][j >> 2] >> (8 * (j & 3))), both(near));
            const float2 d = __fmul2_rn(make_float2(f[j], f[j + 1]), slope<ACT>(z));
            f[j] = d.x;
            f[j + 1] = d.y;
        }
        if (dst[i]) *dst[i] = narrow_vec<DT>(f);
    }
}

// a warp for a block of 128
template <int DT, int ACT>
__global__ void __launch_bounds__(kActThreads) act_back_ragged_kernel(const ActArgs a) {
    using E = typename Elem<DT>::T;
    pdl_wait();
    pdl_trigger();
    const uint32_t b = blockIdx.x * (kActThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (b >= a.n_blocks) return;
    const uint32_t m = b / a.Kb, k = b - m * a.Kb;
    const int c0 = (int)k * 128 + (int)lane;
    const E* src = reinterpret_cast<const E*>(a.dh) + (int64_t)m * a.dh_stride + c0;
    E* dst = reinterpret_cast<E*>(a.dz) + (int64_t)m * a.dz_stride + c0;
    const uint8_t* code = a.codes + (int64_t)b * 128 + lane;
    const float scale = __ldg(a.scale + b);
    E v[4];
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool on = c0 + 32 * j < a.C;
        v[j] = on ? src[32 * j] : E(0);
        c[j] = on ? __ldg(code + 32 * j) : 0u;
    }
    const float near = near_scale<ACT>(scale);
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        const float2 z = __fmul2_rn(widen_codes(c[j] | c[j + 1] << 8), both(near));
        const float2 d = __fmul2_rn(make_float2(widen<DT>(v[j]), widen<DT>(v[j + 1])), slope<ACT>(z));
        const float r[2] = {d.x, d.y};
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (c0 + 32 * (j + q) < a.C) {
                if constexpr (DT == TDQ_F32) dst[32 * (j + q)] = r[q];
                else dst[32 * (j + q)] = (uint16_t)narrow2<DT>(r[q], 0.f);
            }
    }
}

template <int DT, int ACT>
cudaError_t launch_act(const ActArgs& a, bool vec, cudaStream_t st) {
    const uint32_t per = vec ? kActThreads / 32 * (kActVecs<DT> * 32 * kPerVec<DT> / 128) : kActThreads / 32;
    return launch_pdl(vec ? act_back_kernel<DT, ACT> : act_back_ragged_kernel<DT, ACT>, dim3((a.n_blocks + per - 1) / per), dim3(kActThreads), 0, st, a);
}
template <int DT>
cudaError_t pick_act(const ActArgs& a, int act, bool vec, cudaStream_t st) {
    switch (act) {
        case TDQ_ACT_RELU: return launch_act<DT, TDQ_ACT_RELU>(a, vec, st);
        case TDQ_ACT_GELU: return launch_act<DT, TDQ_ACT_GELU>(a, vec, st);
        case TDQ_ACT_GELU_TANH: return launch_act<DT, TDQ_ACT_GELU_TANH>(a, vec, st);
        case TDQ_ACT_SILU: return launch_act<DT, TDQ_ACT_SILU>(a, vec, st);
        default: return launch_act<DT, TDQ_ACT_NONE>(a, vec, st);
    }
}

}  // namespace
}  // namespace tdq

using namespace tdq;

extern "C" tdq_status tdq_activation_backward_fp8(const void* dh, tdq_dtype dtype, int64_t M, int64_t C, int64_t dh_row_stride, const uint8_t* zcodes,
                                                  const float* zscale, int32_t activation, void* dz, int64_t dz_row_stride, void* cuda_stream) {
    if (!known_dtype(dtype) || M < 0 || C <= 0 || C > INT32_MAX - 256 || dh_row_stride < C || dz_row_stride < C || activation < TDQ_ACT_NONE || activation > TDQ_ACT_SILU)
        return TDQ_ERR_INVALID_ARG;
    if (M == 0) return TDQ_OK;
    if (!dh || !zcodes || !zscale || !dz) return TDQ_ERR_INVALID_ARG;
    const uintptr_t esz = dtype == TDQ_F32 ? 4 : 2;
    if (off_grid(dh, esz) || off_grid(dz, esz) || off_grid(zcodes, 16) || off_grid(zscale, 4)) return TDQ_ERR_ALIGNMENT;
    const int64_t Kb = fp8_blocks(C);
    if (M > ((1 << 29) - 1024) / Kb) return TDQ_ERR_UNSUPPORTED;
    ActArgs a = {dh, dz, zcodes, zscale, dh_row_stride, dz_row_stride, (uint32_t)(M * Kb), (uint32_t)Kb, (int32_t)C};
    const bool vec = C * (int64_t)esz % 16 == 0 && on_grid(dh, dh_row_stride, M, (int64_t)esz) && on_grid(dz, dz_row_stride, M, (int64_t)esz);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dtype == TDQ_F32 ? pick_act<TDQ_F32>(a, activation, vec, st) : dtype == TDQ_BF16 ? pick_act<TDQ_BF16>(a, activation, vec, st)
                                                                                                     : pick_act<TDQ_F16>(a, activation, vec, st);
    if (e == cudaSuccess) g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(e);
}
