// tdq_quantize_act_fp8, tdq_quantize_weight_fp8: E4M3 codes with a binary32 scale for each block of 128 channels of a token, or of
// 128 x 128 of a weight matrix.
//
//   a = max(max |x|, 2^-64);   scale = fl(a / 448);   r = fl(448 / a);   code = E4M3(fl(x r)), nearest, ties to even
//
// Both quotients are IEEE divisions, one of each per block; an element costs one product, so that codes are those of the
// formula bit for bit.  |x r| <= 448 (1 + 2^-23) rounds to 448 at most.  The floor 2^-64 keeps scale and r normal numbers.
// A block with a NaN or an infinity gets scale NaN and codes NaN (0x7F): patterns of magnitudes compare as unsigned
// numbers, with NaN above infinity above everything finite, so the maximum carries them along.
//
// Bound by HBM: 2 (4) bytes in and 1 out an element, the input read once.  A block of a token is eight threads of sixteen
// channels each (16-byte loads, a 16-byte store, three shuffles for the maximum); rows off the 16-byte grid pass through
// shared memory word by word.  A weight block stays in the registers of 512 threads between its maximum and its codes (of fp32 vectors, 32 words a thread
// beside 40 registers, some go to local memory and back: 76 bytes a thread, which the first-level cache holds).
#include "tdq_fp8.cuh"

namespace tdq {
namespace {

constexpr int kThreadsA = 256;
constexpr int kThreadsW = 512;

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
// scale and reciprocal of a block whose largest magnitude has this pattern
__device__ __forceinline__ void block_scale(uint32_t bits, float& scale, float& r) {
    const float a = fmaxf(__uint_as_float(bits), kFp8Smallest);
    scale = __fdiv_rn(a, kFp8Max);
    r = __fdiv_rn(kFp8Max, a);
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
// the codes of a 16-byte vector: one word (four binary32) or two (eight 16-bit elements)
template <int DT>
__device__ __forceinline__ void codes_of(const uint4& v, float r, uint32_t* out) {
    if constexpr (DT == TDQ_F32) {
        out[0] = cvt4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w), r);
    } else {
        float a, b, c, d;
        widen2<DT>(v.x, a, b);
        widen2<DT>(v.y, c, d);
        out[0] = cvt4(a, b, c, d, r);
        widen2<DT>(v.z, a, b);
        widen2<DT>(v.w, c, d);
        out[1] = cvt4(a, b, c, d, r);
    }
}
// Elements [0, n) of a 16-byte vector one by one, the rest zero; n <= 0: nothing is read.
template <int DT>
__device__ __forceinline__ uint4 load_part(const typename Elem<DT>::T* p, int64_t n) {
    constexpr int kPer = 16 / (int)sizeof(typename Elem<DT>::T);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < n) {
            if constexpr (DT == TDQ_F32) w[i] = __float_as_uint(p[i]);
            else w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
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
// Sixteen channels a thread, eight neighbouring threads a block: scale and codes.  All lanes of the warp take part, `on` or not.
template <int DT>
__device__ __forceinline__ void quantize16(const uint4* v, bool on, uint4* codes, float* scale, bool first) {
    constexpr int kVecs = (int)sizeof(typename Elem<DT>::T);
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        mx = max_abs<DT>(mx, v[i].x);
        mx = max_abs<DT>(mx, v[i].y);
        mx = max_abs<DT>(mx, v[i].z);
        mx = max_abs<DT>(mx, v[i].w);
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) mx = max_abs<DT>(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    if (!on) return;
    float s, r;
    block_scale(max_bits<DT>(mx), s, r);
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) codes_of<DT>(v[i], r, out + i * (4 / kVecs));
    *codes = make_uint4(out[0], out[1], out[2], out[3]);
    if (first) *scale = s;
}

// Rows on the 16-byte grid: a thread holds sixteen consecutive channels, eight threads a block of 128.
template <int DT>
__global__ void __launch_bounds__(kThreadsA) act_fp8_kernel(const typename Elem<DT>::T* __restrict__ x, uint32_t n_blocks, uint32_t K,
                                                            int64_t C, int64_t stride, uint4* __restrict__ codes, float* __restrict__ scale) {
    using T = typename Elem<DT>::T;
    constexpr int kVecs = (int)sizeof(T);                  // 16-byte vectors a thread reads: 16 elements
    constexpr int kPer = 16 / (int)sizeof(T);
    pdl_wait();
    pdl_trigger();
    const uint32_t t = blockIdx.x * kThreadsA + threadIdx.x;
    const uint32_t b = t >> 3;                             // block of 128
    const bool on = b < n_blocks;
    const uint32_t m = on ? b / K : 0u, k = on ? b - m * K : 0u;
    const int64_t c0 = (int64_t)k * kFp8Block + (threadIdx.x & 7) * 16;
    const T* src = x + (int64_t)m * stride + c0;
    uint4 v[kVecs];
    if (on && c0 + 16 <= C) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = __ldg(reinterpret_cast<const uint4*>(src) + i);
    } else {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = load_part<DT>(src + i * kPer, on ? C - c0 - i * kPer : 0);
    }
    quantize16<DT>(v, on, codes + t, scale + b, (threadIdx.x & 7) == 0);   // rows of C_pad codes follow each other without a gap
}

// Rows anywhere: eight lanes per block of a row, KB consecutive blocks of it at a time, pass their aligned words through shared memory, coalesced, and read
// them back as the kernel above holds them, sixteen channels a thread, shifted by an element where the row of 16-bit elements starts in the
// middle of a word.  A word that holds an element of the row is read whole; what lies beside the row in it is not used.  Bound by instructions: a
// warp per block, whose quotients every lane then computes, took 112 a block (4097 x 1000 fp16 5.0 us, 18464 x 768 bf16 14.3), four blocks of any rows 80
// (4.7 and 11.8); this one 3.5 and 11.5.
template <int DT, int KB>
__global__ void __launch_bounds__(kThreadsA) act_fp8_ragged_kernel(const typename Elem<DT>::T* __restrict__ x, uint32_t n_chunks, uint32_t chunks, uint32_t K,
                                                                   int32_t C, int64_t stride, uint4* __restrict__ codes,
                                                                   float* __restrict__ scale) {
    using T = typename Elem<DT>::T;
    constexpr int kChunk = KB * (int)kFp8Block, kWords = kChunk * (int)sizeof(T) / 4, kLanes = 8 * KB;
    constexpr int kEach = kWords / kLanes, kPitch = kEach + 4;   // words of a thread, four apart from the next one's: no bank is met twice
    constexpr int kRoom = kLanes * kPitch + 4;             // a word more where the row is shifted
    __shared__ __align__(16) uint32_t words[kThreadsA / kLanes][kRoom];
    pdl_wait();
    pdl_trigger();
    const int lane = (int)threadIdx.x % kLanes, group = (int)threadIdx.x / kLanes;
    const uint32_t item = blockIdx.x * (kThreadsA / kLanes) + group;
    const bool on = item < n_chunks;
    const uint32_t m = on ? item / chunks : 0u, c = on ? item - m * chunks : 0u;
    const int n = on ? min(kChunk, C - (int)c * kChunk) : 0;   // channels
    const uintptr_t src = reinterpret_cast<uintptr_t>(x + (int64_t)m * stride + (int64_t)c * kChunk);
    const int off = (int)(src >> 1) & 1;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(src & ~(uintptr_t)3) + lane;
    uint32_t w[kEach + 1];
    const int n_words = sizeof(T) == 4 ? n : n ? (n + off + 1) / 2 : 0;
    if (n_words >= kWords) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) w[j] = __ldg(from + kLanes * j);
    } else {
#pragma unroll
        for (int j = 0; j < kEach; ++j) w[j] = lane + kLanes * j < n_words ? __ldg(from + kLanes * j) : 0u;
    }
    w[kEach] = n_words > kWords && lane == 0 ? __ldg(from + kWords) : 0u;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = lane + kLanes * j, owner = kEach <= kLanes ? lane / kEach + kLanes / kEach * j : i / kEach;
        words[group][i + 4 * owner] = w[j];
    }
    if (lane == 0) words[group][kLanes * kPitch] = w[kEach];
    __syncwarp();
    constexpr int kVecs = (int)sizeof(T);
    const uint4* mine = reinterpret_cast<const uint4*>(&words[group][lane * kPitch]);
    uint4 v[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) v[i] = mine[i];
    if (sizeof(T) == 2 && off) {
        const uint32_t next = words[group][(lane + 1) * kPitch];
        v[0] = make_uint4(__funnelshift_r(v[0].x, v[0].y, 16), __funnelshift_r(v[0].y, v[0].z, 16), __funnelshift_r(v[0].z, v[0].w, 16), __funnelshift_r(v[0].w, v[1].x, 16));
        v[1] = make_uint4(__funnelshift_r(v[1].x, v[1].y, 16), __funnelshift_r(v[1].y, v[1].z, 16), __funnelshift_r(v[1].z, v[1].w, 16), __funnelshift_r(v[1].w, next, 16));
    }
    const int valid = n - lane * 16;                       // of the thread's sixteen channels
    if (valid < 16) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = keep_first<DT>(v[i], valid - i * (16 / kVecs));
    }
    const uint32_t b = m * K + c * KB;
    quantize16<DT>(v, on && c * KB + (lane >> 3) < K, codes + (int64_t)b * 8 + lane, scale + b + (lane >> 3), (lane & 7) == 0);
}

// One block of 128 x 128 weights in registers; VEC: rows on the 16-byte grid, and three thread blocks per SM (4096 x 4096 fp32 16.0 us, bf16 10.0; 256
// threads with twice the registers, two per SM: 17.7 and 11.0).
template <int DT, bool VEC>
__global__ void __launch_bounds__(kThreadsW, VEC ? 3 : 1) weight_fp8_kernel(const typename Elem<DT>::T* __restrict__ w, int64_t O, int64_t I, int64_t I_pad,
                                                               uint8_t* __restrict__ codes, float* __restrict__ scale) {
    using T = typename Elem<DT>::T;
    constexpr int kPer = 16 / (int)sizeof(T);              // elements of a vector
    constexpr int kAcross = kFp8Block / kPer;              // vectors of a row of the block
    constexpr int kRows = kThreadsW / kAcross;             // rows per pass of the thread block
    constexpr int kPasses = kFp8Block / kRows;
    __shared__ uint32_t warp_max[kThreadsW / 32];
    pdl_wait();
    pdl_trigger();
    const int64_t col = (int64_t)blockIdx.x * kFp8Block + (threadIdx.x % kAcross) * kPer;
    const int64_t row0 = (int64_t)blockIdx.y * kFp8Block + threadIdx.x / kAcross;
    uint4 v[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int64_t row = row0 + i * kRows;
        const T* src = w + row * I + col;
        const int64_t n = row < O ? I - col : 0;
        if (VEC && n >= kPer) v[i] = __ldg(reinterpret_cast<const uint4*>(src));
        else v[i] = load_part<DT>(src, n);
    }
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        mx = max_abs<DT>(mx, v[i].x);
        mx = max_abs<DT>(mx, v[i].y);
        mx = max_abs<DT>(mx, v[i].z);
        mx = max_abs<DT>(mx, v[i].w);
    }
    mx = __reduce_max_sync(0xffffffffu, max_bits<DT>(mx));
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreadsW / 32; ++i) mx = max(mx, warp_max[i]);
    float s, r;
    block_scale(mx, s, r);
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int64_t row = row0 + i * kRows;
        if (row >= O) break;
        uint32_t out[2];
        codes_of<DT>(v[i], r, out);
        uint8_t* dst = codes + row * I_pad + col;
        if constexpr (DT == TDQ_F32) *reinterpret_cast<uint32_t*>(dst) = out[0];
        else *reinterpret_cast<uint2*>(dst) = make_uint2(out[0], out[1]);
    }
    if (threadIdx.x == 0) scale[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

template <int DT>
cudaError_t launch_act(const void* x, uint32_t n_blocks, uint32_t K, int64_t C, int64_t stride, uint8_t* codes, float* scale, cudaStream_t st) {
    using T = typename Elem<DT>::T;
    const T* p = reinterpret_cast<const T*>(x);
    if (reinterpret_cast<uintptr_t>(x) % 16 == 0 && (stride * (int64_t)sizeof(T)) % 16 == 0)
        return launch_pdl(act_fp8_kernel<DT>, dim3((n_blocks + kThreadsA / 8 - 1) / (kThreadsA / 8)), dim3(kThreadsA), 0, st, p, n_blocks, K, C, stride,
                          reinterpret_cast<uint4*>(codes), scale);
    // One block of a row at a time for rows of one block, two where four would leave half a warp idle at a row's end, else four (us on 25037 rows of bf16
    // with one, two and four: 70 channels 3.8, 4.9, 8.7; 147 5.2, 5.1, 8.8; 767 14.7, 13.9, 15.6; 1023 17.9, 17.6, 16.5).
    const auto ragged = [&](auto kernel, uint32_t kb) {
        const uint32_t chunks = (K + kb - 1) / kb, n_chunks = n_blocks / K * chunks, per = kThreadsA / (8 * kb);
        return launch_pdl(kernel, dim3((n_chunks + per - 1) / per), dim3(kThreadsA), 0, st, p, n_chunks, chunks, K, (int32_t)C, stride, reinterpret_cast<uint4*>(codes), scale);
    };
    if (K == 1) return ragged(act_fp8_ragged_kernel<DT, 1>, 1);
    if ((K & 3) == 1 || (K & 3) == 2) return ragged(act_fp8_ragged_kernel<DT, 2>, 2);
    return ragged(act_fp8_ragged_kernel<DT, 4>, 4);
}
template <int DT>
cudaError_t launch_weight(const void* w, int64_t O, int64_t I, uint8_t* codes, float* scale, cudaStream_t st) {
    using T = typename Elem<DT>::T;
    const T* p = reinterpret_cast<const T*>(w);
    const int64_t I_pad = fp8_blocks(I) * kFp8Block;
    const dim3 grid((unsigned)fp8_blocks(I), (unsigned)fp8_blocks(O));
    if (reinterpret_cast<uintptr_t>(w) % 16 == 0 && (I * (int64_t)sizeof(T)) % 16 == 0)
        return launch_pdl(weight_fp8_kernel<DT, true>, grid, dim3(kThreadsW), 0, st, p, O, I, I_pad, codes, scale);
    return launch_pdl(weight_fp8_kernel<DT, false>, grid, dim3(kThreadsW), 0, st, p, O, I, I_pad, codes, scale);
}
bool known_dtype(tdq_dtype t) { return t == TDQ_F32 || t == TDQ_BF16 || t == TDQ_F16; }

}  // namespace
}  // namespace tdq

using namespace tdq;

extern "C" tdq_status tdq_quantize_act_fp8(const void* x, tdq_dtype x_dtype, int64_t B, int64_t N, int64_t C, int64_t row_stride_elems,
                                           uint8_t* codes, float* scale, void* cuda_stream) {
    if (!known_dtype(x_dtype) || B < 0 || N < 0 || C <= 0 || row_stride_elems < C) return TDQ_ERR_INVALID_ARG;
    if (C > INT32_MAX || (N > 0 && B > INT64_MAX / N)) return TDQ_ERR_INVALID_ARG;
    const int64_t M = B * N, K = fp8_blocks(C);
    if (M == 0) return TDQ_OK;
    if (!x || !codes || !scale) return TDQ_ERR_INVALID_ARG;
    const uintptr_t esz = x_dtype == TDQ_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(x) % esz || reinterpret_cast<uintptr_t>(codes) % 16 || reinterpret_cast<uintptr_t>(scale) % 4) return TDQ_ERR_ALIGNMENT;
    if (M > ((1 << 29) - 1024) / K) return TDQ_ERR_UNSUPPORTED;   // 2^36 elements; the kernels count their threads in 32 bits
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const uint32_t n = (uint32_t)(M * K);
    cudaError_t e;
    if (x_dtype == TDQ_F32) e = launch_act<TDQ_F32>(x, n, (uint32_t)K, C, row_stride_elems, codes, scale, st);
    else if (x_dtype == TDQ_BF16) e = launch_act<TDQ_BF16>(x, n, (uint32_t)K, C, row_stride_elems, codes, scale, st);
    else e = launch_act<TDQ_F16>(x, n, (uint32_t)K, C, row_stride_elems, codes, scale, st);
    if (e == cudaSuccess) g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(e);
}

extern "C" tdq_status tdq_quantize_weight_fp8(const void* w, tdq_dtype w_dtype, int64_t O, int64_t I, uint8_t* wcodes, float* wscale,
                                              void* cuda_stream) {
    if (!known_dtype(w_dtype) || O < 0 || I <= 0) return TDQ_ERR_INVALID_ARG;
    if (O == 0) return TDQ_OK;
    if (!w || !wcodes || !wscale) return TDQ_ERR_INVALID_ARG;
    const uintptr_t esz = w_dtype == TDQ_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(w) % esz || reinterpret_cast<uintptr_t>(wcodes) % 16 || reinterpret_cast<uintptr_t>(wscale) % 4) return TDQ_ERR_ALIGNMENT;
    if (O > (int64_t)65535 * kFp8Block || I > INT32_MAX) return TDQ_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (w_dtype == TDQ_F32) e = launch_weight<TDQ_F32>(w, O, I, wcodes, wscale, st);
    else if (w_dtype == TDQ_BF16) e = launch_weight<TDQ_BF16>(w, O, I, wcodes, wscale, st);
    else e = launch_weight<TDQ_F16>(w, O, I, wcodes, wscale, st);
    if (e == cudaSuccess) g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(e);
}
