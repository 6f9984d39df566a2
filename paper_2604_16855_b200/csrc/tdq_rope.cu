// tdq_qk_norm_rope: root-mean-square norm of every query and key head and the rotation by the token's positions, in one pass.
//
//   r = 1 / sqrt(mean_i x_i^2 + eps);  n_i = x_i (r w_i);   for pair i < R/2:  t = pos[m, axis_i] freq_i,
//   (n_a, n_b) -> (n_a cos t - n_b sin t,  n_b cos t + n_a sin t);   channels from R on: n_i
//
// Angles.  t reaches 10^6 and more, where binary32 has lost the fraction of a turn.  A pair's turns per position are a fraction in units of 2^-64, right to
// half a unit (once a thread); its product with the position, modulo 2^64, is the fraction of a turn to position x 2^-65, no worse than the rounding to
// binary32 for sincospif up to positions of 2^40.  freq / 2 pi in binary64 alone is off by 2^-53 of itself, which the position multiplies: 9e-5 radians at 2^40,
// binary32's own step from 2^28 on.  In binary64 (product, turns, fraction for every token) 29386 x 2 x 256 bf16 took 32.6 us for 28.2.  Sum of
// squares, norm and rotation are binary32; one rounding at the store.
//
// Bound by HBM: every head is read and written once.  A thread owns the two vectors (16 bytes, or 8) of a head whose elements form pairs (halves:
// one from either half; adjacent: neighbours), so that a head is a power of two of lanes, its sum of squares a few shuffles, and
// no element passes through another thread: in place is safe.  A thread block takes some tokens with all their heads; a warp keeps to a
// group of heads and goes through the tokens with the next two's loads in flight.  The weights and the block's cosines and
// sines, computed once, are in shared memory, laid out so that the lanes of a head read consecutive 16-byte pieces: with a thread's
// eight pairs in one piece, four lanes met in every bank and shared memory was busy for 77 % of the time (88 us on 16384 tokens x 40 heads x 128
// bf16).  A warp per token with cosines times weights in 32 registers had too few loads in flight (95 us).
#include <cuda_fp16.h>

#include <algorithm>

#include "tdq_common.cuh"

namespace tdq {
namespace {

constexpr int kRopeWarps = 8;
constexpr int kSmSharedBytes = 227 * 1024;
constexpr size_t kTableMax = 32 * 1024;     // bytes of cosines and sines of a block (16 KB for eight tokens of 256 pairs)

struct RopeArgs {
    tdq_rope_heads q, k;
    const void* any;           // readable and 16-byte aligned
    const int64_t* pos;
    const double* freq;
    const int32_t* axis;
    int64_t M;
    int32_t Hq, H;             // query heads, all heads
    int32_t D, half, n_axes;   // half = R / 2
    int32_t norm, adjacent;
    float eps, inv_dim;        // inv_dim = 1 / D
    int32_t tokens, groups;    // of a block; of a token's heads, one for a warp at a time
    int32_t warps_across;      // warps of a block that share a token's groups
    int32_t lanes_log2;        // lanes of a head
};

template <int DT> struct Bits { using T = uint16_t; };
template <> struct Bits<TDQ_F32> { using T = float; };
template <int DT>
__device__ __forceinline__ float to_f(typename Bits<DT>::T v) {
    if constexpr (DT == TDQ_F32) return v;
    else if constexpr (DT == TDQ_BF16) return __uint_as_float((uint32_t)v << 16);
    else return __half2float(__ushort_as_half(v));
}
template <int DT>
__device__ __forceinline__ typename Bits<DT>::T from_f(float v) {
    if constexpr (DT == TDQ_F32) return v;
    else if constexpr (DT == TDQ_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    else return __half_as_ushort(__float2half_rn(v));
}
template <int VB> struct Bytes { using T = uint4; };      // a vector of VB bytes
template <> struct Bytes<8> { using T = uint2; };
template <int DT, int VB>
__device__ __forceinline__ void unpack(const typename Bytes<VB>::T& v, float* f) {
    const uint32_t* w = &v.x;
#pragma unroll
    for (int i = 0; i < VB / 4; ++i) {
        if constexpr (DT == TDQ_F32) {
            f[i] = __uint_as_float(w[i]);
        } else if constexpr (DT == TDQ_BF16) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = h.x;
            f[2 * i + 1] = h.y;
        }
    }
}
template <int DT, int VB>
__device__ __forceinline__ typename Bytes<VB>::T pack(const float* f) {
    typename Bytes<VB>::T v;
    uint32_t* w = &v.x;
#pragma unroll
    for (int i = 0; i < VB / 4; ++i) {
        if constexpr (DT == TDQ_F32) {
            w[i] = __float_as_uint(f[i]);
        } else if constexpr (DT == TDQ_BF16) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
            const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return v;
}

// a vector to shared memory, asynchronously; zeros if not `there`
template <int VB>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool there) {
    if constexpr (VB == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(there ? 8 : 0) : "memory");
}
template <int VB>
__device__ __forceinline__ typename Bytes<VB>::T lds_vec(uint32_t addr) {
    typename Bytes<VB>::T v;
    if constexpr (VB == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    else asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
// The turns a pair makes per position: the fraction of freq / 2 pi to the nearest 2^-64 (whole turns of it stay whole turns at every position).
// 1 / 2 pi is taken as the sum of two binary64 numbers, right to 2^-109, and the first product with its rounding error, so nothing above that is lost
// for frequencies up to 2^40.  Added to 1.5 x 2^20, a number's multiple of 2^-32 stands in the low half of the sum's bits (modulo a turn), and what
// that leaves is counted in units of 2^-64 the same way: with conversions to integers the general kernel takes 283 us for 277 (18432 x 32 x 72
// bf16; 266 with the binary64 quotient alone).
struct Speed { int64_t step; float bad; };                 // bad: NaN where freq is not finite, else 0
__device__ __forceinline__ Speed speed_of(double freq) {
    constexpr double kInv2Pi = 0x1.45f306dc9c883p-3, kInv2PiLow = -0x1.6b01ec5417056p-57, kHigh = 0x1.8p20, kLow = 0x1.8p-12;
    const double turns = __dmul_rn(freq, kInv2Pi), g = fma(freq, kInv2PiLow, fma(freq, kInv2Pi, -turns));
    const double f = turns - rint(turns);                  // the fraction is f + g
    const double high = f + g + kHigh, low = f - (high - kHigh) + g + kLow;
    const uint64_t step = ((uint64_t)__double_as_longlong(high) << 32) + (uint64_t)(__double_as_longlong(low) - __double_as_longlong(kLow));
    return {(int64_t)step, (float)(f - f)};
}
// cosine and sine at a position; the product's 64 low bits are its fraction of a turn, of which 32 are rounded to binary32
__device__ __forceinline__ float2 turn_at(const Speed& v, int64_t pos) {
    const int32_t frac = (int32_t)(((uint64_t)pos * (uint64_t)v.step) >> 32);
    float s, c;
    sincospif(fmaf((float)frac, 4.6566128730773926e-10f, v.bad), &s, &c);   // 2^-31: half turns
    return make_float2(c, s);
}
__device__ __forceinline__ uint32_t axis_of(const RopeArgs& a, int i) {   // an axis outside the positions counts as their last
    return min((uint32_t)__ldg(a.axis + i), (uint32_t)a.n_axes - 1u);
}

// Registers a thread, and with them warps an SM.  16 bits, 28 warps of 72: with 78 registers only 24 fit, and 2949 x 20 x 96 bf16 takes 10.6 us
// for 7.8; 20 warps 18432 x 24 x 64 fp16 29.8 us for 24.8, 32 warps of 64 25.9.  binary32, 32 warps of 64: 8192 x 32 x 80 39, 24 warps 47.
template <int DT> constexpr int rope_ahead = 2;
template <int DT, int VB> constexpr int rope_ring = DT == TDQ_F32 ? 0 : rope_ahead<DT> * 2 * VB;   // bytes of shared memory a thread
template <int DT> constexpr int rope_regs = DT == TDQ_F32 ? 64 : 72;
template <int DT> constexpr int rope_warps_per_sm = DT == TDQ_F32 ? 32 : 28;
template <int DT, bool ADJ, int VB>
__global__ void __maxnreg__(rope_regs<DT>) rope_kernel(const RopeArgs a) {
    using T = typename Bits<DT>::T;
    using Vec = typename Bytes<VB>::T;
    constexpr int V = VB / (int)sizeof(T);                 // elements of a vector, pairs of a thread
    constexpr bool kAsync = DT != TDQ_F32;
    constexpr int kAhead = rope_ahead<DT>;                 // tokens whose loads are in flight
    extern __shared__ float4 shared[];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t m0 = (int64_t)blockIdx.x * a.tokens;
    const int n_tok = (int)min((int64_t)a.tokens, a.M - m0);
    const int L = 1 << a.lanes_log2, unit = lane & (L - 1), units = a.half / V, all_units = a.D / (2 * V);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(shared) + VB * threadIdx.x;   // [tokens ahead][2][threads] vectors
    float4* const weights = shared + (kAsync ? kAhead * 2 * blockDim.x * VB / 16 : 0);   // [queries, keys][V / 2][units of a head]: four weights
    float4* const table = weights + (a.norm ? V * all_units : 0);   // [tokens][V / 2][turned units]: two pairs' cosines, then their sines
    const int row = warp / a.warps_across, across = warp - row * a.warps_across;   // the warp's first token and head group
    const int rows = (int)(blockDim.x >> 5) / a.warps_across;
    const bool has = unit < all_units, turns = unit < units;   // a unit of the turned channels (R is a multiple of 2 V)
    // element offsets of a unit's two vectors in a head
    const auto first_of = [&](int u) { return ADJ || u >= units ? 2 * u * V : u * V; };
    const auto second_of = [&](int u) { return ADJ || u >= units ? (2 * u + 1) * V : a.half + u * V; };
    const int e0 = first_of(unit), e1 = second_of(unit);
    bool have_table = false;                               // all warps make the same passes
    for (int first = blockIdx.y * a.warps_across; first < a.groups; first += gridDim.y * a.warps_across) {
        const int group = first + across;                  // behind the last one: no heads
        const int head = (group << (5 - a.lanes_log2)) + (lane >> a.lanes_log2);
        const bool mine = has && head < a.H, is_q = head < a.Hq;
        const int64_t in_step = rows * (is_q ? a.q.row_stride : a.k.row_stride), out_step = rows * (is_q ? a.q.out_row_stride : a.k.out_row_stride);
        const T* src = is_q ? reinterpret_cast<const T*>(a.q.x) + head * a.q.head_stride + (m0 + row) * a.q.row_stride
                            : reinterpret_cast<const T*>(a.k.x) + (head - a.Hq) * a.k.head_stride + (m0 + row) * a.k.row_stride;
        T* dst = is_q ? reinterpret_cast<T*>(a.q.out) + head * a.q.out_head_stride + (m0 + row) * a.q.out_row_stride
                      : reinterpret_cast<T*>(a.k.out) + (head - a.Hq) * a.k.out_head_stride + (m0 + row) * a.k.out_row_stride;
        // The thread's two vectors of the next tokens, zeros where it has none: 16 bits on their way to its own pieces of shared memory (16384 x
        // 40 x 128 bf16 62.1 -> 56.3 us; four tokens ahead 55.5, but 18432 x 24 x 64 fp16 24.7 instead of 22.6), binary32 in registers (8192 x 32 x 80: 39,
        // through shared memory 45).
        uint32_t next = 0;
        Vec held[kAhead][2];
        const auto load = [&](Vec* to_regs, int t) {
            const bool there = mine && t < n_tok;
            if constexpr (kAsync) {
                const uint32_t to = ring + (next % kAhead) * 2u * VB * blockDim.x;
                copy_async<VB>(to, there ? src + e0 : reinterpret_cast<const T*>(a.any), there);
                copy_async<VB>(to + VB * blockDim.x, there ? src + e1 : reinterpret_cast<const T*>(a.any), there);
                asm volatile("cp.async.commit_group;" ::: "memory");
                ++next;
            } else {
                to_regs[0] = to_regs[1] = Vec{};
                if (there) {
                    to_regs[0] = *reinterpret_cast<const Vec*>(src + e0);
                    to_regs[1] = *reinterpret_cast<const Vec*>(src + e1);
                }
            }
            src += in_step;
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(held[i], row + i * rows);
        if (!have_table) {                                 // meanwhile
            if (a.norm)
                for (int i = threadIdx.x; i < V * all_units; i += blockDim.x) {
                    const int k = i / all_units, u = i - k * all_units, c = k % (V / 2);
                    const float* w = k >= V / 2 ? a.k.weight : a.q.weight;
                    const int e = c < V / 4 ? first_of(u) + 4 * c : second_of(u) + 4 * (c - V / 4);
                    weights[i] = w ? __ldg(reinterpret_cast<const float4*>(w + e)) : make_float4(1.f, 1.f, 1.f, 1.f);
                }
            // a pair of every so many tokens for a thread
            const int wide = min(a.half, (int)blockDim.x), skip = wide ? (int)blockDim.x / wide : 1;
            for (int pair = wide ? (int)threadIdx.x % wide : a.half, t0 = wide ? (int)threadIdx.x / wide : 0; pair < a.half && t0 < skip; pair += wide) {
                const Speed v = speed_of(__ldg(a.freq + pair));
                const long long* pos = reinterpret_cast<const long long*>(a.pos) + (m0 + t0) * a.n_axes + axis_of(a, pair);
                const int u = pair / V, j = pair - u * V;
                float* to = reinterpret_cast<float*>(table + (t0 * (V / 2) + (j >> 1)) * units + u) + (j & 1);
                for (int t = t0; t < n_tok; t += skip, pos += (int64_t)skip * a.n_axes, to += skip * (V / 2) * units * 4) {
                    const float2 cs = turn_at(v, __ldg(pos));
                    to[0] = cs.x;
                    to[2] = cs.y;
                }
            }
            __syncthreads();
            have_table = true;
        }
        const float4* const wt = weights + (is_q ? 0 : V / 2 * all_units) + unit;
        for (int t = row; t < n_tok; t += rows) {
            Vec v0 = held[0][0], v1 = held[0][1];
            if constexpr (kAsync) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
                const uint32_t from = ring + (next % kAhead) * 2u * VB * blockDim.x;   // the oldest
                v0 = lds_vec<VB>(from);
                v1 = lds_vec<VB>(from + VB * blockDim.x);
            } else {
#pragma unroll
                for (int i = 0; i + 1 < kAhead; ++i) {
                    held[i][0] = held[i + 1][0];
                    held[i][1] = held[i + 1][1];
                }
            }
            // two elements an instruction: the kernel issues close to what the schedulers take (250 of them a warp and token, 309 with single elements, 18432 x 24 x 64 fp16)
            float2 x[V / 2], y[V / 2];
            unpack<DT, VB>(v0, reinterpret_cast<float*>(x));
            unpack<DT, VB>(v1, reinterpret_cast<float*>(y));
            load(held[kAhead - 1], t + kAhead * rows);
            if (a.norm) {
                float2 sx = make_float2(0.f, 0.f), sy = sx;
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    sx = __ffma2_rn(x[j], x[j], sx);
                    sy = __ffma2_rn(y[j], y[j], sy);
                }
                float ss = (sx.x + sx.y) + (sy.x + sy.y);
                for (int d = 1; d < L; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
                const float r = rsqrtf(fmaf(ss, a.inv_dim, a.eps));
                if (mine) {
                    const float2 rr = make_float2(r, r);
#pragma unroll
                    for (int c = 0; c < V / 4; ++c) {
                        const float4 p = wt[c * all_units], q = wt[(c + V / 4) * all_units];
                        x[2 * c] = __fmul2_rn(x[2 * c], __fmul2_rn(rr, make_float2(p.x, p.y)));
                        x[2 * c + 1] = __fmul2_rn(x[2 * c + 1], __fmul2_rn(rr, make_float2(p.z, p.w)));
                        y[2 * c] = __fmul2_rn(y[2 * c], __fmul2_rn(rr, make_float2(q.x, q.y)));
                        y[2 * c + 1] = __fmul2_rn(y[2 * c + 1], __fmul2_rn(rr, make_float2(q.z, q.w)));
                    }
                }
            }
            if (mine) {
                if (turns) {
                    const float4* cs = table + t * (V / 2) * units + unit;
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        const float4 two = cs[i * units];
                        if constexpr (ADJ) {               // pairs 2 i and 2 i + 1: neighbours in x, then in y
                            float2 &p = i < V / 4 ? x[2 * i] : y[2 * i - V / 2], &q = i < V / 4 ? x[2 * i + 1] : y[2 * i + 1 - V / 2];
                            p = make_float2(p.x * two.x - p.y * two.z, p.y * two.x + p.x * two.z);
                            q = make_float2(q.x * two.y - q.y * two.w, q.y * two.y + q.x * two.w);
                        } else {                           // x[i] and y[i]
                            const float2 c = make_float2(two.x, two.y), n = make_float2(two.z, two.w), x0 = x[i], y0 = y[i];
                            x[i] = __ffma2_rn(__fmul2_rn(y0, make_float2(-1.f, -1.f)), n, __fmul2_rn(x0, c));
                            y[i] = __ffma2_rn(x0, n, __fmul2_rn(y0, c));
                        }
                    }
                }
                *reinterpret_cast<Vec*>(dst + e0) = pack<DT, VB>(reinterpret_cast<const float*>(x));
                *reinterpret_cast<Vec*>(dst + e1) = pack<DT, VB>(reinterpret_cast<const float*>(y));
            }
            dst += out_step;
        }
        if constexpr (kAsync) asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
}

// Any head size, stride and alignment: a warp per head, a lane per pair.
template <int DT>
__global__ void __launch_bounds__(256) rope_any_kernel(const RopeArgs a) {
    using T = typename Bits<DT>::T;
    pdl_wait();
    pdl_trigger();
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    const int64_t m = item / a.H;
    if (m >= a.M) return;
    const int head = (int)(item - m * a.H);
    const bool is_q = head < a.Hq;
    const tdq_rope_heads& s = is_q ? a.q : a.k;
    const int hh = is_q ? head : head - a.Hq;
    const T* x = reinterpret_cast<const T*>(s.x) + m * s.row_stride + hh * s.head_stride;
    T* out = reinterpret_cast<T*>(s.out) + m * s.out_row_stride + hh * s.out_head_stride;
    float r = 1.f;
    if (a.norm) {
        float ss = 0.f;
        for (int i = lane; i < a.D; i += 32) {
            const float f = to_f<DT>(x[i]);
            ss = fmaf(f, f, ss);
        }
        for (int d = 1; d < 32; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        r = rsqrtf(fmaf(ss, a.inv_dim, a.eps));
    }
    const float* w = a.norm ? s.weight : nullptr;
    for (int i = lane; i < a.half; i += 32) {
        const int ia = a.adjacent ? 2 * i : i, ib = a.adjacent ? 2 * i + 1 : a.half + i;
        const float na = to_f<DT>(x[ia]) * (w ? r * __ldg(w + ia) : r), nb = to_f<DT>(x[ib]) * (w ? r * __ldg(w + ib) : r);
        const float2 t = turn_at(speed_of(__ldg(a.freq + i)), __ldg(reinterpret_cast<const long long*>(a.pos) + m * a.n_axes + axis_of(a, i)));
        out[ia] = from_f<DT>(na * t.x - nb * t.y);
        out[ib] = from_f<DT>(nb * t.x + na * t.y);
    }
    for (int i = 2 * a.half + lane; i < a.D; i += 32) out[i] = from_f<DT>(to_f<DT>(x[i]) * (w ? r * __ldg(w + i) : r));
}

// vectors of VB bytes everywhere, a head of at most 32 lanes, whole vectors on either side of the rotated channels' middle and end
template <int DT, int VB>
bool rope_fits(const RopeArgs& a) {
    constexpr int V = VB / (int)sizeof(typename Bits<DT>::T);
    const auto side = [&](const tdq_rope_heads& s) {
        return s.heads == 0 || (reinterpret_cast<uintptr_t>(s.x) % VB == 0 && reinterpret_cast<uintptr_t>(s.out) % VB == 0 && reinterpret_cast<uintptr_t>(s.weight) % 16 == 0 &&
                                s.row_stride % V == 0 && s.head_stride % V == 0 && s.out_row_stride % V == 0 && s.out_head_stride % V == 0);
    };
    return a.D % (2 * V) == 0 && a.half % V == 0 && a.D <= 64 * V && side(a.q) && side(a.k);
}

template <int DT, int VB>
cudaError_t launch_vec(RopeArgs a, int n_sm, int dev, cudaStream_t st) {
    constexpr int V = VB / (int)sizeof(typename Bits<DT>::T);
    a.lanes_log2 = 0;
    while ((2 * V << a.lanes_log2) < a.D) ++a.lanes_log2;
    const int per_warp = 32 >> a.lanes_log2, groups = (a.H + per_warp - 1) / per_warp;
    // about eight warps: all of a token's head groups side by side where there are no more, several tokens where there are few
    a.groups = groups;
    a.warps_across = groups < kRopeWarps ? groups : (groups + (groups + kRopeWarps - 1) / kRopeWarps - 1) / ((groups + kRopeWarps - 1) / kRopeWarps);
    const int rows = kRopeWarps / a.warps_across;
    const int warps = rows * a.warps_across, passes = (groups + a.warps_across - 1) / a.warps_across;
    const size_t per_block = (a.norm ? 2 * a.D * sizeof(float) : 0) + (size_t)rope_ring<DT, VB> * warps * 32, per_token = (size_t)a.half * sizeof(float2);
    const int table_deep = per_token ? (int)(kTableMax / (per_token * rows)) : 8;
    // Tokens a warp goes through (`deep`, eight at most: sixteen 16384 x 40 x 128 65 us for 57), and a token's groups of heads in one thread block after
    // another or in as many blocks: the least of rounds of resident blocks x (tokens x groups of a warp + 1), and blocks of an SM x warps / 16.
    // Against as many tokens as leave four blocks an SM, whatever fits at once: 2619 x 72 x 128 bf16 23.7 -> 18.8 us, 3272 x 6 x 128 6.0 -> 4.6, 314 x
    // 20 x 256 fp32 6.5 -> 4.7; 227 x 60 x 128, the worst of 23 sizes, 4.7 -> 4.9.
    uint64_t least = UINT64_MAX;
    int across = 1;
    for (int deep = 1; deep <= 8 && (deep == 1 || (deep <= table_deep && rows * (deep - 1) < a.M)); ++deep) {
        const uint32_t blocks = ((uint32_t)a.M + rows * deep - 1) / (rows * deep);
        const uint32_t fit = std::min<uint32_t>(rope_warps_per_sm<DT> / warps, (uint32_t)((size_t)kSmSharedBytes / (per_block + per_token * rows * deep + 1024)));
        for (int y = 1; y <= passes; y += passes > 1 ? passes - 1 : 1) {
            const uint64_t n = (uint64_t)blocks * y;
            if (n > INT32_MAX) break;
            const uint32_t held = fit * n_sm, rounds = ((uint32_t)n + held - 1) / held, an_sm = ((uint32_t)n + n_sm - 1) / n_sm;
            const uint64_t cost = 16ull * rounds * (1 + deep * (passes / y)) + (uint64_t)an_sm * warps;
            if (cost < least) { least = cost; a.tokens = rows * deep; across = y; }
        }
    }
    const size_t smem = per_block + per_token * a.tokens;
    a.any = a.q.heads ? a.q.x : a.k.x;
    const int64_t blocks = (a.M + a.tokens - 1) / a.tokens;
    void (*const kernel)(RopeArgs) = a.adjacent ? rope_kernel<DT, true, VB> : rope_kernel<DT, false, VB>;
    static std::atomic<uint64_t> smem_done[2];
    const cudaError_t e = allow_smem(kernel, (int)(kTableMax + rope_ring<DT, VB> * 32 * kRopeWarps + 2 * 64 * V * sizeof(float)), smem_done[a.adjacent], dev);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3((unsigned)blocks, (unsigned)across), dim3(rows * a.warps_across * 32), smem, st, a);
}

template <int DT>
tdq_status launch(RopeArgs a, cudaStream_t st) {
    int dev = 0;
    const int n_sm = current_device_sm_count(&dev);
    if (n_sm <= 0) return TDQ_ERR_CUDA;
    cudaError_t e = cudaErrorInvalidValue;
    // Heads of 72 or 80 channels whose halves are no whole vectors of 16 bytes, and rows on the 8-byte grid: vectors of 8 bytes (18432 x 32 x 72 bf16
    // 277 us with the general kernel, 61 so).
    if (rope_fits<DT, 16>(a)) {
        e = launch_vec<DT, 16>(a, n_sm, dev, st);
    } else if (DT != TDQ_F32 && rope_fits<DT, 8>(a)) {
        if constexpr (DT != TDQ_F32) e = launch_vec<DT, 8>(a, n_sm, dev, st);
    } else {
        const int64_t blocks = (a.M * a.H + 7) / 8;
        if (blocks > INT32_MAX) return TDQ_ERR_UNSUPPORTED;
        e = launch_pdl(rope_any_kernel<DT>, dim3((unsigned)blocks), dim3(256), 0, st, a);
    }
    if (e == cudaSuccess) g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return cuda_status(e);
}

// null pointers, sizes and element alignment of one side; TDQ_OK when it has no heads
tdq_status check_heads(const tdq_rope_heads& s, int64_t M, int64_t D, uintptr_t esz) {
    if (s.heads < 0) return TDQ_ERR_INVALID_ARG;
    if (s.heads == 0 || M == 0) return TDQ_OK;
    if (!s.x || !s.out) return TDQ_ERR_INVALID_ARG;
    if (s.heads > 65536) return TDQ_ERR_UNSUPPORTED;
    // strides such that no offset passes 63 bits
    const int64_t limit = (int64_t)1 << 40;
    const auto wild = [&](int64_t v) { return v < 0 || v > limit; };
    if (wild(s.row_stride) || wild(s.head_stride) || wild(s.out_row_stride) || wild(s.out_head_stride)) return TDQ_ERR_INVALID_ARG;
    // heads and rows of the output must not overlap one another
    const bool many_h = s.heads > 1, many_m = M > 1;
    if ((many_h && s.out_head_stride < D) || (many_m && s.out_row_stride < D)) return TDQ_ERR_INVALID_ARG;
    if (many_h && many_m && s.out_row_stride < (s.heads - 1) * s.out_head_stride + D &&
        (double)s.out_head_stride < (double)(M - 1) * (double)s.out_row_stride + (double)D)
        return TDQ_ERR_INVALID_ARG;
    if (s.x == s.out && ((many_m && s.row_stride != s.out_row_stride) || (many_h && s.head_stride != s.out_head_stride))) return TDQ_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(s.x) % esz || reinterpret_cast<uintptr_t>(s.out) % esz || reinterpret_cast<uintptr_t>(s.weight) % 4) return TDQ_ERR_ALIGNMENT;
    return TDQ_OK;
}

}  // namespace
}  // namespace tdq

using namespace tdq;

extern "C" tdq_status tdq_qk_norm_rope(const tdq_rope_heads* q, const tdq_rope_heads* k, tdq_dtype dtype, int64_t M, const tdq_rope_params* p,
                                       const int64_t* positions, const double* freq, const int32_t* axis, void* cuda_stream) {
    if (!p || (!q && !k) || M < 0) return TDQ_ERR_INVALID_ARG;
    if (dtype != TDQ_F32 && dtype != TDQ_BF16 && dtype != TDQ_F16) return TDQ_ERR_INVALID_ARG;
    if (p->head_dim <= 0 || p->rotary_dim < 0 || p->rotary_dim > p->head_dim || p->rotary_dim % 2) return TDQ_ERR_INVALID_ARG;
    if (p->flags & ~(uint32_t)(TDQ_ROPE_NORM | TDQ_ROPE_ADJACENT)) return TDQ_ERR_INVALID_ARG;
    if ((p->flags & TDQ_ROPE_NORM) && !(p->eps >= 0.f)) return TDQ_ERR_INVALID_ARG;
    if (p->rotary_dim > 0 && p->n_axes <= 0) return TDQ_ERR_INVALID_ARG;
    if (M > INT32_MAX || p->head_dim > 65536) return TDQ_ERR_UNSUPPORTED;
    const uintptr_t esz = dtype == TDQ_F32 ? 4 : 2;
    RopeArgs a = {};
    for (int i = 0; i < 2; ++i) {
        const tdq_rope_heads* s = i ? k : q;
        if (!s) continue;
        const tdq_status st = check_heads(*s, M, p->head_dim, esz);
        if (st != TDQ_OK) return st;
        (i ? a.k : a.q) = *s;
    }
    if (M == 0 || a.q.heads + a.k.heads == 0) return TDQ_OK;
    // one tensor passed for both sides and written: a head would be read after it was turned
    if (a.q.heads && a.k.heads && (a.q.out == a.k.out || a.q.out == a.k.x || a.k.out == a.q.x)) return TDQ_ERR_INVALID_ARG;
    if (p->rotary_dim > 0 && (!positions || !freq || !axis)) return TDQ_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(positions) % 8 || reinterpret_cast<uintptr_t>(freq) % 8 || reinterpret_cast<uintptr_t>(axis) % 4) return TDQ_ERR_ALIGNMENT;
    a.pos = positions;
    a.freq = freq;
    a.axis = axis;
    a.M = M;
    a.Hq = (int32_t)a.q.heads;
    a.H = (int32_t)(a.q.heads + a.k.heads);
    a.D = p->head_dim;
    a.half = p->rotary_dim / 2;
    a.n_axes = p->n_axes;
    a.norm = (p->flags & TDQ_ROPE_NORM) != 0;
    a.adjacent = (p->flags & TDQ_ROPE_ADJACENT) != 0;
    a.eps = p->eps;
    a.inv_dim = 1.f / (float)p->head_dim;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    return dtype == TDQ_F32 ? launch<TDQ_F32>(a, st) : dtype == TDQ_BF16 ? launch<TDQ_BF16>(a, st) : launch<TDQ_F16>(a, st);
}
