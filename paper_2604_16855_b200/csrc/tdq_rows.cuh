// Rows in registers, for the kernels of the norm (tdq_norm.cu, tdq_norm_back.cu): a group of T threads holds a row in 16-byte vectors t, t + T, .., on the
// 16-byte grid or off it, and adds over it.  Several groups share a warp, or several warps are a group.
#pragma once
#include "tdq_fp8.cuh"

namespace tdq {
namespace {

constexpr int64_t kMaxRow = 16384;            // channels of the longest row
constexpr int kMaxGroups = 15;                // of several warps in a block: it has barriers 0 (of all its threads) to 15

template <int DT> constexpr int kPerVec = 16 / (int)sizeof(typename Elem<DT>::T);

// Threads that share a row meet: within a warp, or warps at a barrier of their own.
template <int T>
__device__ __forceinline__ void group_sync(int group) {
    if constexpr (T <= 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(T) : "memory");
}
// The sum over the group's threads; `room` holds a float for each of the group's warps, and another use of it follows a barrier.
template <int T>
__device__ __forceinline__ float group_sum(float v, float* room, int group, int t) {
#pragma unroll
    for (int d = (T < 32 ? T : 32) / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if constexpr (T > 32) {
        constexpr int kWarps = T / 32;
        if ((t & 31) == 0) room[t >> 5] = v;
        group_sync<T>(group);
        if constexpr (kWarps <= 4) {
            v = room[0];
#pragma unroll
            for (int k = 1; k < kWarps; ++k) v += room[k];
        } else {
            v = (t & 31) < kWarps ? room[t & 31] : 0.f;
#pragma unroll
            for (int d = 16; d; d >>= 1)
                if (d < kWarps) v += __shfl_xor_sync(0xffffffffu, v, d);
            v = __shfl_sync(0xffffffffu, v, 0);
        }
    }
    return v;
}
// Two sums at a time: the first exchange leaves the lower half of the threads with one, the upper half with the other.  `room` holds two floats for each warp.
template <int T>
__device__ __forceinline__ float2 group_sum2(float2 v, float* room, int group, int t) {
    constexpr int W = T < 32 ? T : 32;
    const bool upper = t & (W / 2);
    float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xffffffffu, upper ? v.x : v.y, W / 2);
#pragma unroll
    for (int d = W / 4; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if constexpr (T <= 32) {
        const float o = __shfl_xor_sync(0xffffffffu, s, W / 2);
        return upper ? make_float2(o, s) : make_float2(s, o);
    } else {
        constexpr int kWarps = T / 32;
        if ((t & 15) == 0) room[(t >> 5) * 2 + (upper ? 1 : 0)] = s;
        group_sync<T>(group);
        if constexpr (kWarps <= 4) {
            float2 r = *reinterpret_cast<const float2*>(room);
#pragma unroll
            for (int k = 1; k < kWarps; ++k) r = __fadd2_rn(r, *reinterpret_cast<const float2*>(room + 2 * k));
            return r;
        } else {
            float2 r = (t & 31) < kWarps ? *reinterpret_cast<const float2*>(room + 2 * (t & 31)) : make_float2(0.f, 0.f);
            s = (upper ? r.y : r.x) + __shfl_xor_sync(0xffffffffu, upper ? r.x : r.y, 16);
#pragma unroll
            for (int d = 8; d; d >>= 1)
                if (d < kWarps) s += __shfl_xor_sync(0xffffffffu, s, d);
            return make_float2(__shfl_sync(0xffffffffu, s, 0), __shfl_sync(0xffffffffu, s, 16));
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
// the same as pairs, for packed arithmetic
template <int DT>
__device__ __forceinline__ void widen_pairs(const uint4& v, float2* f) {
    float g[kPerVec<DT>];
    widen_vec<DT>(v, g);
#pragma unroll
    for (int i = 0; i < kPerVec<DT> / 2; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
}
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }
// Keeps the compiler from holding on to what it has made of a vector: made again later, it needs no registers meanwhile.
__device__ __forceinline__ void forget(uint4& v) { asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)); }
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

template <int DT>
__device__ __forceinline__ uint4 narrow_pairs(const float2* f) {
    if constexpr (DT == TDQ_F32) return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    else return make_uint4(narrow2<DT>(f[0].x, f[0].y), narrow2<DT>(f[1].x, f[1].y), narrow2<DT>(f[2].x, f[2].y), narrow2<DT>(f[3].x, f[3].y));
}

// 16-byte vectors of a group's stage in shared memory: the longest row, its offset, and the word behind it that a shift reads
template <int T, int V> constexpr int kStageVecs = T * V + 2;

// Vectors t, t + T, .. of a row of n channels that lies `off` bytes into the stage, zeros behind it.
template <int DT, int T, int V>
__device__ __forceinline__ void take_ragged(const uint4* stage, int off, int n, int t, uint4* v) {
    const uint32_t* words = reinterpret_cast<const uint32_t*>(stage) + (off >> 2);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int first = (t + T * i) * kPerVec<DT>;
        v[i] = make_uint4(0, 0, 0, 0);
        if (first >= n) continue;
        const uint32_t* p = words + 4 * (t + T * i);
        uint32_t a = p[0], b = p[1], c = p[2], d = p[3];
        if (sizeof(typename Elem<DT>::T) == 2 && (off & 2)) {
            const uint32_t e = p[4];
            a = __funnelshift_r(a, b, 16); b = __funnelshift_r(b, c, 16); c = __funnelshift_r(c, d, 16); d = __funnelshift_r(d, e, 16);
        }
        v[i] = keep_first<DT>(make_uint4(a, b, c, d), n - first);
    }
}
// A row on its way.  fetch() starts the loads, take() gives vectors t, t + T, .. of the row, zeros behind its n channels.  Off the grid (!VEC) a row's aligned vectors (one that
// holds an element of the row is read whole; what lies beside the row in it is not used) pass through the group's stage: put() between two group_syncs, the first
// of which says that what was there has been read.  Plain loads: the output may be an input, and the read-only path is for what nobody writes meanwhile.
template <int DT, int T, int V, bool VEC>
struct Row {
    using E = typename Elem<DT>::T;
    static constexpr int P = kPerVec<DT>, N = V + (VEC ? 0 : 1);
    uint4 raw[N];
    int off;
    __device__ __forceinline__ void fetch(const E* row, int n, int t, bool on) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                raw[i] = on && (t + T * i) * P < n ? reinterpret_cast<const uint4*>(row)[t + T * i] : make_uint4(0, 0, 0, 0);
        } else {
            const uintptr_t at = reinterpret_cast<uintptr_t>(row);
            off = (int)(at & 15);
            const int n_vec = on ? (off + n * (int)sizeof(E) + 15) >> 4 : 0;
            const uint4* src = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
#pragma unroll
            for (int i = 0; i < N; ++i) raw[i] = t + T * i < n_vec ? src[t + T * i] : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void put(uint4* stage, int t) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < V || t < 2) stage[t + T * i] = raw[i];   // a row has at most one vector more than it has on the grid
    }
    __device__ __forceinline__ void take(const uint4* stage, int n, int t, uint4* v) const {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = raw[i];
        } else {
            take_ragged<DT, T, V>(stage, off, n, t, v);
        }
    }
};
// The way back: vectors to a row anywhere, whole ones where the row's grid has them, elements at its ends.  All threads of the group; a row that is not there (!on)
// is not stored.
template <int DT, int T, int V>
__device__ __forceinline__ void store_row_ragged(typename Elem<DT>::T* row, int n, int t, int group, uint4* stage, const uint4* v, bool on) {
    using E = typename Elem<DT>::T;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row);
    const int off = (int)(at & 15), bytes = n * (int)sizeof(E), n_vec = on ? (off + bytes + 15) >> 4 : 0;
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
// PER consecutive weights, `otherwise` where there are none or behind n; vec: w is on the 16-byte grid
template <int PER>
__device__ __forceinline__ void load_weights(const float* w, bool vec, int first, int n, float otherwise, float* f) {
    if (w && vec && first + PER <= n) {
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
template <int PER>
__device__ __forceinline__ void load_weight_pairs(const float* w, bool vec, int first, int n, float otherwise, float2* f) {
    float g[PER];
    load_weights<PER>(w, vec, first, n, otherwise, g);
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
}

// Threads and vectors a row.  Few rows: as many threads as leave each with one vector (4 x 4096 bf16: 512 threads).  Else the fewest threads that leave each with at most three
// (two from 256 threads on), whose registers then have room for the next row on its way; a row that fills less than a warp shares it.
struct RowShape { int t, v; };
inline RowShape row_shape(int64_t vecs, int64_t M, int n_sm, int least, int most) {
    int t = least;
    const bool few = M < 2 * (int64_t)n_sm;
    while (t < most && vecs > (int64_t)t * (few || t < 32 ? 1 : t < 256 ? 3 : 2)) t *= 2;
    return {t, (int)((vecs + t - 1) / t)};
}
inline bool on_grid(const void* p, int64_t stride, int64_t M, int64_t esz) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (M <= 1 || stride * esz % 16 == 0);
}
inline bool known_dtype(tdq_dtype t) { return t == TDQ_F32 || t == TDQ_BF16 || t == TDQ_F16; }
inline bool off_grid(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
// Blocks of a kernel that an SM holds, asked once per kernel and device.  `known` is a static of the caller, one per kernel.
template <typename F>
inline int blocks_per_sm(F* kernel, int threads, int smem, std::atomic<int> (&known)[kMaxDevices], int dev) {
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) n = 1;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace
}  // namespace tdq
