// Shared by the kernels of the block-scaled 8-bit floating point layer (tdq_fp8_quantize.cu, tdq_fp8_linear.cu, tdq_fp8_pair.cu)
// and by what stands around it (tdq_norm.cu, tdq_fp8_grad.cu).
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>

#include "tdq_common.cuh"

namespace tdq {

constexpr int64_t kFp8Block = 128;          // channels that share a scale (and output channels, for weights)
constexpr float kFp8Max = 448.0f;           // largest E4M3 value
constexpr float kFp8Smallest = 0x1p-64f;    // smallest maximum a scale is taken from
inline int64_t fp8_blocks(int64_t n) { return (n + kFp8Block - 1) / kFp8Block; }

struct Fp8Args {
    const float* xscale;       // [M][K]
    const float* wscale;       // [tiles of 128 output channels][K]
    const float* bias;         // [O] or null
    void* y;
    int64_t M, O, y_stride;
    int32_t K;                 // blocks of 128 channels
    int32_t tiles_m, tiles_n;  // of the kernel's own tile
    int32_t y_type;            // tdq_dtype
    int32_t y_vec;             // rows of y on the 16-byte grid
    int32_t n_stages, split;
    uint32_t* status;
};

// What follows the layer (tdq_fp8_linear_epilogue); the kernels without it have instances of their own.
struct Fp8Epilogue {
    int32_t activation;        // tdq_activation
    int32_t residual_vec, pre_vec;   // rows on the 16-byte grid
    const void* residual;      // [M][O] of y's type, or null
    void* pre;                 // likewise
    int64_t residual_stride, pre_stride;
    bool any() const { return activation != TDQ_ACT_NONE || residual || pre; }
};

// Tensor map of a [rows][cols] byte matrix read in boxes of box_rows x 128 bytes, 128-byte swizzle (K-major operand of the
// tensor core); false when the driver's encoder is missing or refuses.
bool fp8_operand_map(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int box_rows);
// Two CTAs on a tile of 256 tokens and 256 or 128 columns (tdq_fp8_pair.cu); xmap with boxes of 128 rows, wmap of half the columns.
tdq_status launch_fp8_pair(Fp8Args a, Fp8Epilogue e, int columns, const CUtensorMap& xmap, const CUtensorMap& wmap, int n_sm, int dev, cudaStream_t stream);

#ifdef __CUDACC__
namespace {

template <int DT> struct Elem { using T = uint16_t; };   // DT: tdq_dtype
template <> struct Elem<TDQ_F32> { using T = float; };

template <int DT>
__device__ __forceinline__ float widen(typename Elem<DT>::T v) {
    if constexpr (DT == TDQ_F32) return v;
    else if constexpr (DT == TDQ_BF16) return __uint_as_float((uint32_t)v << 16);
    else return __half2float(__ushort_as_half(v));
}
// bit pattern of the larger magnitude of two words' elements, and of a word's own (as binary32)
template <int DT>
__device__ __forceinline__ uint32_t max_abs(uint32_t m, uint32_t w) {
    if constexpr (DT == TDQ_F32) return max(m, w & 0x7fffffffu);
    else return __vmaxu2(m, w & 0x7fff7fffu);
}
template <int DT>
__device__ __forceinline__ uint32_t max_bits(uint32_t m) {
    if constexpr (DT == TDQ_F32) return m;
    else return __float_as_uint(widen<DT>((uint16_t)max(m & 0xffffu, m >> 16)));
}
// Scale and reciprocal of a block whose largest magnitude has this pattern.  POW2: the smallest power of two 2^s with a <= 448 2^s; with a = m 2^e,
// 1 <= m < 2, and 448 = 1.75 2^8 that is s = e - 8, one more where m > 1.75: the carry of 0x1fffff added to the pattern.
template <bool POW2>
__device__ __forceinline__ void block_scale(uint32_t bits, float& scale, float& r) {
    const float a = fmaxf(__uint_as_float(bits), kFp8Smallest);
    if constexpr (POW2) {
        const uint32_t e = (__float_as_uint(a) + 0x1fffffu) >> 23;
        scale = __uint_as_float((e - 8u) << 23);
        r = __uint_as_float((262u - e) << 23);
    } else {
        scale = __fdiv_rn(a, kFp8Max);
        r = __fdiv_rn(kFp8Max, a);
    }
    if (bits >= 0x7f800000u) scale = r = __uint_as_float(0x7fffffffu);
}
// two elements' codes, the first in the low byte
__device__ __forceinline__ uint32_t cvt2(float lo, float hi) {
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(hi), "f"(lo));
    return v;
}
__device__ __forceinline__ uint32_t cvt4(float a, float b, float c, float d, float r) {
    return cvt2(__fmul_rn(a, r), __fmul_rn(b, r)) | cvt2(__fmul_rn(c, r), __fmul_rn(d, r)) << 16;
}
template <int DT>
__device__ __forceinline__ void widen2(uint32_t w, float& lo, float& hi) {
    if constexpr (DT == TDQ_BF16) {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xffff0000u);
    } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        lo = f.x;
        hi = f.y;
    }
}
// the first n elements of a 16-byte vector, the rest zero
template <int DT>
__device__ __forceinline__ uint4 keep_first(const uint4& v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == TDQ_F32) w[i] = i < n ? w[i] : 0u;
        else w[i] = 2 * i >= n ? 0u : 2 * i + 1 >= n ? w[i] & 0xffffu : w[i];
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void copy4_async(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
// K-major operand rows of 128 bytes with the 128-byte swizzle: bands of eight rows follow each other every 1024 bytes; 32 more
// channels are 32 bytes further on (the hardware applies the swizzle to the address that results).
constexpr uint32_t kSwDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint64_t sw_desc(uint32_t saddr) {
    return ((uint64_t)kSwDescHi << 32) | ((saddr & 0x3FFFFu) >> 4) | (1u << 16);
}
__device__ __forceinline__ float4 lds_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds_u4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t fp8_cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void fp8_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// for the kernels that include tdq_tc.cuh first
#ifdef TDQ_TC_CUH_
__device__ __forceinline__ bool fp8_try(uint32_t bar_s, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar_s), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait of a warp on a barrier of its CTA.  try_wait without a time hint: the hardware holds the warp for a while at a time, where the hinted form
// comes back every 40 clocks (counted: half of all instructions of the pair kernel were the waiting warps').  Each lane asks for itself, and the caller
// brings them together (__syncwarp, which costs nothing that shows) before the warp-wide instructions that follow; lanes that vote in the loop instead
// took 1 % of a short layer's time (1 x 4096 -> 4096 bf16 5.14 -> 5.21 us, 576 x 384 -> 960 fp32 4.46 -> 4.51).
__device__ __forceinline__ void fp8_wait_more(uint32_t bar_s, uint32_t parity, Ctrl* c, uint32_t* status, uint32_t code,
                                              uint32_t limit = (uint32_t)kTimeoutCycles) {
    const uint32_t t0 = (uint32_t)clock();
#pragma unroll 1
    while (!fp8_try(bar_s, parity)) {
        if (c->abort_flag) return;
        if ((uint32_t)clock() - t0 > limit) {
            atomicCAS(status, 0u, code | ((uint32_t)blockIdx.x << 8));
            c->abort_flag = 1;
            return;
        }
    }
}
__device__ __forceinline__ void fp8_wait(uint32_t bar_s, uint32_t parity, Ctrl* c, uint32_t* status, uint32_t code) {
    if (!fp8_try(bar_s, parity)) fp8_wait_more(bar_s, parity, c, status, code);
    __syncwarp();
}
#endif
__device__ __forceinline__ uint32_t map_to_cta(uint32_t saddr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
    return r;
}

}  // namespace
#endif
}  // namespace tdq
