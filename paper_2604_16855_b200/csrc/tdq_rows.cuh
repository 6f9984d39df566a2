// Rows in registers, for the kernels of the norm (tdq_norm.cu, tdq_norm_back.cu): a group of threads holds a row in 16-byte vectors t, t + T, .., on the
// 16-byte grid or off it, and adds over it.
#pragma once
#include "tdq_fp8.cuh"

namespace tdq {
namespace {

constexpr int64_t kMaxRow = 16384;            // channels of the longest row

template <int DT> constexpr int kPerVec = 16 / (int)sizeof(typename Elem<DT>::T);

// T threads that share a row: a warp, or warps that meet at a barrier of their own.
template <int T>
__device__ __forceinline__ void group_sync(int group) {
    if constexpr (T == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(T) : "memory");
}
// N sums over the group's threads, all at once; `room` holds N floats per warp, and another use of it follows a barrier.
template <int T, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* room, int group, int t) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    if constexpr (T > 32) {
        constexpr int kWarps = T / 32;
        if ((t & 31) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) room[i * kWarps + (t >> 5)] = v[i];
        group_sync<T>(group);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = (t & 31) < kWarps ? room[i * kWarps + (t & 31)] : 0.f;
#pragma unroll
            for (int d = kWarps / 2; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            v[i] = __shfl_sync(0xffffffffu, s, 0);
        }
    }
}

template <int DT>
__device__ __forceinline__ void widen_vec(const uint4& v, float* f) {
    if constexpr (DT == TDQ_F32) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    } else {
        widen2<DT>(v.x, f[0], f[1]);
        widen2<DT>(v.y, f[2], f[3]);
        widen2<DT>(v.z, f[4], f[5]);
        widen2<DT>(v.w, f[6], f[7]);
    }
}
template <int DT>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {
    uint32_t r;
    if constexpr (DT == TDQ_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int DT>
__device__ __forceinline__ uint4 narrow_vec(const float* f) {
    if constexpr (DT == TDQ_F32) return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    else return make_uint4(narrow2<DT>(f[0], f[1]), narrow2<DT>(f[2], f[3]), narrow2<DT>(f[4], f[5]), narrow2<DT>(f[6], f[7]));
}
// Vectors t, t + T, .. of a row of n channels on the 16-byte grid, zeros behind it.
template <int DT, int T, int V>
__device__ __forceinline__ void load_row(const typename Elem<DT>::T* row, int n, int t, uint4* v) {
#pragma unroll
    for (int i = 0; i < V; ++i)
        v[i] = (t + T * i) * kPerVec<DT> < n ? __ldg(reinterpret_cast<const uint4*>(row) + t + T * i) : make_uint4(0, 0, 0, 0);
}
// The same of a row anywhere: its aligned vectors (one that holds an element of the row is read whole; what lies beside the row in it is not used)
// pass through `stage`, from which a thread reads five words of its vector and shifts.  Elements behind n are zero.
template <int DT, int T, int V>
__device__ __forceinline__ void load_row_ragged(const typename Elem<DT>::T* row, int n, int t, int group, uint4* stage, uint4* v) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(row);
    const int off = (int)(at & 15), n_vec = (off + n * (int)sizeof(typename Elem<DT>::T) + 15) >> 4;
    const uint4* src = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
    group_sync<T>(group);                                    // what was in `stage` has been read
#pragma unroll
    for (int i = 0; i < V + 1; ++i)
        if (t + T * i < n_vec) stage[t + T * i] = __ldg(src + t + T * i);
    group_sync<T>(group);
    const uint32_t* words = reinterpret_cast<const uint32_t*>(stage) + (off >> 2);
    const int shift = (off & 3) * 8;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int first = (t + T * i) * kPerVec<DT>;
        v[i] = make_uint4(0, 0, 0, 0);
        if (first >= n) continue;
        const uint32_t* p = words + 4 * (t + T * i);
        uint32_t a = p[0], b = p[1], c = p[2], d = p[3];
        if (sizeof(typename Elem<DT>::T) == 2 && shift) {
            const uint32_t e = p[4];
            a = __funnelshift_r(a, b, 16); b = __funnelshift_r(b, c, 16); c = __funnelshift_r(c, d, 16); d = __funnelshift_r(d, e, 16);
        }
        v[i] = keep_first<DT>(make_uint4(a, b, c, d), n - first);
    }
}
// The way back: vectors to a row anywhere, whole ones where the row's grid has them, elements at its ends.
template <int DT, int T, int V>
__device__ __forceinline__ void store_row_ragged(typename Elem<DT>::T* row, int n, int t, int group, uint4* stage, const uint4* v) {
    using E = typename Elem<DT>::T;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row);
    const int off = (int)(at & 15), bytes = n * (int)sizeof(E), n_vec = (off + bytes + 15) >> 4;
    group_sync<T>(group);
#pragma unroll
    for (int i = 0; i < V; ++i)
        if ((t + T * i) * kPerVec<DT> < n) stage[t + T * i] = v[i];
    group_sync<T>(group);
    uint4* dst = reinterpret_cast<uint4*>(at & ~(uintptr_t)15);
#pragma unroll
    for (int i = 0; i < V + 1; ++i) {
        const int j = t + T * i, first = 16 * j - off;       // byte of the row that the vector starts with
        if (j >= n_vec) continue;
        if (first >= 0 && first + 16 <= bytes) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(stage) + (first >> 2);
            uint32_t a = p[0], b = p[1], c = p[2], d = p[3];
            if (sizeof(E) == 2 && (first & 2)) {
                const uint32_t e = p[4];
                a = __funnelshift_r(a, b, 16); b = __funnelshift_r(b, c, 16); c = __funnelshift_r(c, d, 16); d = __funnelshift_r(d, e, 16);
            }
            dst[j] = make_uint4(a, b, c, d);
        } else {
            const E* p = reinterpret_cast<const E*>(stage);
#pragma unroll
            for (int q = 0; q < kPerVec<DT>; ++q) {
                const int e = first / (int)sizeof(E) + q;
                if (e >= 0 && e < n) row[e] = p[e];
            }
        }
    }
}
// kPer consecutive weights, `otherwise` where there are none or behind n
template <int PER, bool VEC>
__device__ __forceinline__ void load_weights(const float* w, int first, int n, float otherwise, float* f) {
    if (VEC && w && first < n) {
#pragma unroll
        for (int q = 0; q < PER; q += 4) {
            const float4 u = __ldg(reinterpret_cast<const float4*>(w + first + q));
            f[q] = u.x; f[q + 1] = u.y; f[q + 2] = u.z; f[q + 3] = u.w;
        }
    } else {
#pragma unroll
        for (int q = 0; q < PER; ++q) f[q] = w && first + q < n ? __ldg(w + first + q) : otherwise;
    }
}

// bytes of a group's stage: the longest row, its offset, and the word behind that a shift reads
template <int T, int V> constexpr int kStageVecs = T * V + 2;

// Threads and vectors a row: the fewest threads from a warp on that hold it in four vectors each, or, where rows are too few to fill the GPU, as many
// as leave each with one (4 x 4096 bf16: 512 threads).  EXACT: three vectors where three are enough (the rows on the grid, whose kernels are cheap).
struct RowShape { int t, v; };
inline RowShape row_shape(int64_t vecs, int64_t M, int n_sm, int most, bool exact) {
    int t = 32;
    const int wide = M < 4 * (int64_t)n_sm ? 1 : 4;
    while (t < most && (int64_t)t * wide < vecs) t = t == 32 ? 128 : 2 * t;
    const int v = (int)((vecs + t - 1) / t);
    if (v <= 1) return {t, 1};
    if (t <= 128 && v == 2) return {t, 2};
    if (t <= 128 && v == 3 && exact) return {t, 3};
    return {t, v <= 4 ? 4 : 8};
}
inline bool on_grid(const void* p, int64_t stride, int64_t M, int64_t esz) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (M <= 1 || stride * esz % 16 == 0);
}
inline bool known_dtype(tdq_dtype t) { return t == TDQ_F32 || t == TDQ_BF16 || t == TDQ_F16; }
inline bool off_grid(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

}  // namespace
}  // namespace tdq
