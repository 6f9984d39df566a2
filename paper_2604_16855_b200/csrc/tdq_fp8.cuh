// Shared by the kernels of the block-scaled 8-bit floating point layer (tdq_fp8_quantize.cu, tdq_fp8_linear.cu, tdq_fp8_pair.cu).
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

// Tensor map of a [rows][cols] byte matrix read in boxes of box_rows x 128 bytes, 128-byte swizzle (K-major operand of the
// tensor core); false when the driver's encoder is missing or refuses.
bool fp8_operand_map(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int box_rows);
// Two CTAs on a tile of 256 tokens and 256 or 128 columns (tdq_fp8_pair.cu); xmap with boxes of 128 rows, wmap of half the columns.
tdq_status launch_fp8_pair(Fp8Args a, int columns, const CUtensorMap& xmap, const CUtensorMap& wmap, int n_sm, int dev, cudaStream_t stream);

#ifdef __CUDACC__
namespace {

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
