// Shared by the kernels of tdq_fp8_weight_grad (tdq_fp8_grad.cu for large layers, tdq_fp8_grad_small.cu for little work).
#pragma once
#include "tdq_rows.cuh"

namespace tdq {

constexpr int kSmallSplitMax = 8;          // thread blocks that share a tile's tokens
constexpr int kSmallSteps = 16;            // of 32 tokens that one of them adds at most

struct GradSmallArgs {
    const uint8_t* xcodes;     // [M][Kb * 128]
    const float* xscale;       // [M][Kb]
    const void* dy;
    void* dw;
    float* db;                 // or null
    int64_t M, O, I, dy_stride, dw_stride;
    int32_t Kb, dw_type, dw_vec;
    uint32_t split;
    uint32_t* status;          // set to 0
};
// An estimate of that kernel's time in clocks, comparable with the other's, and in how many parts the tokens go; INT64_MAX where it cannot be taken.  vec: dy's rows on the
// 16-byte grid, O a multiple of eight; esz: bytes of its elements.
int64_t grad_small_cost(int64_t M, int64_t O, int64_t Kb, bool vec, int esz, int n_sm, uint32_t* split);
tdq_status launch_grad_small(GradSmallArgs a, tdq_dtype dy_dtype, bool vec, cudaStream_t st);

#ifdef __CUDACC__
namespace {

// four codes times their scale as four bf16, nearest even
__device__ __forceinline__ void restore4(uint32_t codes, float scale, uint32_t& lo, uint32_t& hi) {
    uint32_t h0, h1;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(h0), "=r"(h1) : "r"(codes));
    const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
    const float2 p0 = __fmul2_rn(f0, make_float2(scale, scale)), p1 = __fmul2_rn(f1, make_float2(scale, scale));
    lo = narrow2<TDQ_BF16>(p0.x, p0.y);
    hi = narrow2<TDQ_BF16>(p1.x, p1.y);
}
// The next bf16 addend of eight values, of PARTS that make them up: the leading eight bits of what is left, cut off; exact.  A value without a number goes to its first addend
// alone (a NaN keeps a bit of its mantissa that bf16 has).  f is left with the rest.
template <int PARTS>
__device__ __forceinline__ void grad_addend(float* f, uint32_t* r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t lead[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t v = __float_as_uint(f[2 * j + q]);
            lead[q] = v & 0xffff0000u;
            if constexpr (PARTS > 1) {
                lead[q] |= (v & 0x7fffffffu) > 0x7f800000u ? 0x00400000u : 0u;
                f[2 * j + q] = (v & 0x7f800000u) == 0x7f800000u ? 0.f : f[2 * j + q] - __uint_as_float(lead[q]);
            }
        }
        r[j] = __byte_perm(lead[0], lead[1], 0x7632);
    }
}

}  // namespace
#endif
}  // namespace tdq
