// tdq_fp8_weight_grad for little work: dw[o,i] = sum_m dy[m,o] x[m,i], db[o] = sum_m dy[m,o] in one kernel; of the workspace only the status word.
//
// What counts is the way from launch to result: the kernel for large layers (tdq_fp8_grad.cu) sets up tensor memory and copy engine and, for a dy that is not bf16, for cut
// tiles and for db, needs a second and a third kernel.  Here a thread block of eight warps has 64 outputs x one block of 128 channels in its registers (mma.sync, 32 x 32
// a warp), 32 tokens at a time from global memory through registers, cut into bf16 addends and restored on the way to shared memory; the thread blocks of a cluster share a
// tile's tokens, at most 512 each, and add their sums in order over distributed shared memory.
// Bound by the chain of a step (loads, conversion, shared memory, instructions: 1700 clocks, with two steps on their way as well).  From a graph, db included, against the other
// kernel: 64 x 256 -> 256 bf16 5.7 us for 8.3, 247 x 370 -> 37 fp32 5.0 for 12.2, 1000 x 300 -> 300 bf16 7.4 for 12.7, 1 x 1073 -> 208 fp16 6.0 for 10.9.
#include <type_traits>

#include "tdq_fp8_grad.cuh"

namespace tdq {
namespace {

constexpr int kSmallO = 64, kSmallTok = 32, kSmallThreads = 256;
constexpr uint32_t kSmallDy = kSmallTok * kSmallO * 2;    // bytes of an addend: rows of 64 outputs, 128 bytes, 16-byte columns exchanged by the row's number
constexpr uint32_t kSmallX = kSmallTok * 256;             // rows of 128 channels
template <int PARTS> constexpr uint32_t kSmallBuffer = PARTS * kSmallDy + kSmallX;

__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, const uint32_t* b) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void sts4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// DT: dy's type; VEC: its rows on the 16-byte grid, O a multiple of eight.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kSmallThreads, 2) fp8_grad_small_kernel(const GradSmallArgs a) {
    using E = typename Elem<DT>::T;
    constexpr int PARTS = DT == TDQ_BF16 ? 1 : DT == TDQ_F16 ? 2 : 3;
    constexpr uint32_t kBuffer = kSmallBuffer<PARTS>;
    constexpr int kPitch = 132;                              // floats of a row of the sums
    constexpr uint32_t kRoom = 2 * kBuffer > kSmallO * kPitch * 4 ? 2 * kBuffer : kSmallO * kPitch * 4;
    __shared__ __align__(128) uint8_t room[kRoom];           // two buffers; then the tile's sums
    __shared__ float db_sum[kSmallO];
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0u;
    const uint32_t room_s = (uint32_t)__cvta_generic_to_shared(room);
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t split = a.split, rank = split > 1 ? fp8_cluster_rank() : 0u, tile = blockIdx.x / split;
    const int32_t to = (int32_t)(tile / (uint32_t)a.Kb), ti = (int32_t)(tile - (uint32_t)to * (uint32_t)a.Kb);
    const int32_t steps = (int32_t)((a.M + kSmallTok - 1) / kSmallTok);
    const int32_t s0 = (int32_t)((int64_t)steps * rank / split), s1 = (int32_t)((int64_t)steps * (rank + 1) / split);

    // a thread's share of a step: eight outputs and sixteen codes of one token
    const int tok = tid >> 3, col = tid & 7;
    const int64_t o0 = (int64_t)to * kSmallO + col * 8;
    float f[8], sum[8], scale;
    uint4 code;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
    const auto load = [&](int32_t s) {
        const int64_t m = (int64_t)s * kSmallTok + tok;
        const bool on = s < s1 && m < a.M;
        code = make_uint4(0, 0, 0, 0);
        scale = 0.f;
        if (on) {
            code = __ldg(reinterpret_cast<const uint4*>(a.xcodes + (m * a.Kb + ti) * 128) + col);
            scale = __ldg(a.xscale + m * a.Kb + ti);
        }
        const E* src = reinterpret_cast<const E*>(a.dy) + (on ? m * a.dy_stride + o0 : 0);
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 8; j += kPerVec<DT>) widen_vec<DT>(on && o0 < a.O ? __ldg(reinterpret_cast<const uint4*>(src + j)) : make_uint4(0, 0, 0, 0), f + j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = on && o0 + j < a.O ? widen<DT>(src[j]) : 0.f;
        }
    };
    const auto store = [&](uint32_t buffer) {
        const uint32_t to_s = room_s + buffer * kBuffer + (uint32_t)tok * 128u + (((uint32_t)col ^ ((uint32_t)tok & 7u)) << 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += f[j];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            uint32_t r[4];
            grad_addend<PARTS>(f, r);
            sts4(to_s + p * kSmallDy, r[0], r[1], r[2], r[3]);
        }
        const uint32_t x_s = room_s + buffer * kBuffer + PARTS * kSmallDy + (uint32_t)tok * 256u;
        uint32_t r[8];
        restore4(code.x, scale, r[0], r[1]);
        restore4(code.y, scale, r[2], r[3]);
        restore4(code.z, scale, r[4], r[5]);
        restore4(code.w, scale, r[6], r[7]);
        sts4(x_s + (((2u * (uint32_t)col) ^ ((uint32_t)tok & 7u)) << 4), r[0], r[1], r[2], r[3]);
        sts4(x_s + (((2u * (uint32_t)col + 1u) ^ ((uint32_t)tok & 7u)) << 4), r[4], r[5], r[6], r[7]);
    };

    // a warp: 32 outputs x 32 channels.  Both operands lie with the tokens as rows, so both are turned on the way to registers
    const uint32_t wo = (uint32_t)(warp & 1) * 32u, wi = (uint32_t)(warp >> 1) * 32u, j8 = (uint32_t)lane >> 3, r8 = (uint32_t)lane & 7u;
    float acc[2][4][4];
#pragma unroll
    for (int x = 0; x < 32; ++x) acc[x >> 4][(x >> 2) & 3][x & 3] = 0.f;
    load(s0);
    for (int32_t s = s0; s < s1; ++s) {
        const uint32_t buffer = (uint32_t)(s - s0) & 1u, base = room_s + buffer * kBuffer;
        store(buffer);
        load(s + 1);
        __syncthreads();                                     // the step is there; and the one before has been read when the next is written over it, behind the next meeting
#pragma unroll
        for (uint32_t k = 0; k < kSmallTok / 16; ++k) {
            uint32_t b[2][4];                                // 16 channels each: two instructions' operands
#pragma unroll
            for (uint32_t n = 0; n < 2; ++n) {
                const uint32_t row = k * 16u + (j8 & 1u) * 8u + r8, c16 = (wi >> 3) + n * 2u + (j8 >> 1);
                ldmatrix4t(base + PARTS * kSmallDy + row * 256u + ((c16 ^ (row & 7u)) << 4), b[n]);
            }
#pragma unroll
            for (uint32_t p = 0; p < PARTS; ++p)
#pragma unroll
                for (uint32_t m = 0; m < 2; ++m) {
                    uint32_t x[4];
                    const uint32_t row = k * 16u + (j8 >> 1) * 8u + r8, c16 = (wo >> 3) + m * 2u + (j8 & 1u);
                    ldmatrix4t(base + p * kSmallDy + row * 128u + ((c16 ^ (row & 7u)) << 4), x);
#pragma unroll
                    for (uint32_t n = 0; n < 4; ++n) mma16816(acc[m][n], x, b[n >> 1] + 2 * (n & 1u));
                }
        }
    }
    __syncthreads();
    // the tile's sums to shared memory, row by row
    float* sums = reinterpret_cast<float*>(room);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2*>(sums + (wo + m * 16 + h * 8 + (lane >> 2)) * kPitch + wi + n * 8 + 2 * (lane & 3)) = make_float2(acc[m][n][2 * h], acc[m][n][2 * h + 1]);
    const bool adds = a.db && ti == 0;
    if (adds) {                                              // the outputs' sums: 4 tokens a warp by exchange, then eight warps through what is left of the room's places
        __shared__ float warp_sum[8][kSmallO];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 8);
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 16);
            if (lane < 8) warp_sum[warp][lane * 8 + j] = sum[j];
        }
        __syncthreads();
        if (tid < kSmallO) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) v += warp_sum[w][tid];
            db_sum[tid] = v;
        }
    }
    __syncthreads();
    if (split > 1) fp8_cluster_sync();                       // all parts' sums are there
    // this block's rows of the tile, all parts in order
    const int r0 = (int)(kSmallO * rank / split), r1 = (int)(kSmallO * (rank + 1) / split);
    const int64_t i = (int64_t)ti * 128 + 4 * lane;
    const int left = (int)min((int64_t)4, a.I - i);
    for (int r = r0 + warp; r < r1; r += 8) {
        const int64_t o = (int64_t)to * kSmallO + r;
        if (o >= a.O) break;
        const uint32_t at = room_s + (uint32_t)(r * kPitch + 4 * lane) * 4u;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (uint32_t p = 0; p < split; ++p) {
            float4 q;
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(map_to_cta(at, p)) : "memory");
            v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
        }
        if (left > 0) {
            if (a.dw_type == TDQ_F32) {
                float* dw = reinterpret_cast<float*>(a.dw) + o * a.dw_stride + i;
                if (a.dw_vec && left == 4) *reinterpret_cast<float4*>(dw) = make_float4(v[0], v[1], v[2], v[3]);
                else
                    for (int j = 0; j < left; ++j) dw[j] = v[j];
            } else {
                uint16_t* dw = reinterpret_cast<uint16_t*>(a.dw) + o * a.dw_stride + i;
                const uint32_t lo = a.dw_type == TDQ_BF16 ? narrow2<TDQ_BF16>(v[0], v[1]) : narrow2<TDQ_F16>(v[0], v[1]);
                const uint32_t hi = a.dw_type == TDQ_BF16 ? narrow2<TDQ_BF16>(v[2], v[3]) : narrow2<TDQ_F16>(v[2], v[3]);
                if (a.dw_vec && left == 4) *reinterpret_cast<uint2*>(dw) = make_uint2(lo, hi);
                else
                    for (int j = 0; j < left; ++j) dw[j] = (uint16_t)((j & 2 ? hi : lo) >> (16 * (j & 1)));
            }
        }
        if (adds && lane == 0) {
            float d = 0.f;
            const uint32_t db_s = (uint32_t)__cvta_generic_to_shared(db_sum + r);
            for (uint32_t p = 0; p < split; ++p) {
                float q;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(q) : "r"(map_to_cta(db_s, p)) : "memory");
                d += q;
            }
            a.db[o] = d;
        }
    }
    // No block leaves while another reads from it.  The lanes meet first: the barrier's instruction is the whole warp's, and the rows' loops are not.  Relaxed: what a warp has read from
    // other blocks is there by then, as it has gone into a store (a row's first lane has a channel, so that every load of the warp has been waited for); an
    // arrival that releases waits for those stores themselves (64 x 256 -> 256 bf16 6.1 us for 5.7).
    if (split > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

template <int DT, bool VEC>
cudaError_t launch_small(const GradSmallArgs& a, int64_t tiles, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.split));
    cfg.blockDim = dim3(kSmallThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = a.split;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, fp8_grad_small_kernel<DT, VEC>, a);
}

}  // namespace

int64_t grad_small_cost(int64_t M, int64_t O, int64_t Kb, bool vec, int esz, int n_sm, uint32_t* split) {
    const int64_t tiles = (O + kSmallO - 1) / kSmallO * Kb, steps = (M + kSmallTok - 1) / kSmallTok;
    if (tiles > INT32_MAX / kSmallSplitMax || steps > kSmallSteps * kSmallSplitMax) return INT64_MAX;
    // as many parts as keep the thread blocks on the GPU at once, and as many as their tokens want
    int64_t s = (steps + kSmallSteps - 1) / kSmallSteps;
    while (s < kSmallSplitMax && s < steps && tiles * (s + 1) <= n_sm) ++s;
    *split = (uint32_t)s;
    // Fitted to 44 layers of 1 to 7000 tokens, 64 to 4096 -> 32 to 6000 channels: the choice between the two kernels takes 2 % longer than the better one in the mean, on these layers, 34 % at
    // worst (497 tokens, 4040 -> 78 float32, 18.5 us for 13.8: float32 rows off the grid are charged too much there).  A step is
    // a chain of latencies, so that of two thread blocks on an SM each takes half.
    const int64_t rounds = (tiles * s + n_sm - 1) / n_sm, step = (steps + s - 1) / s * (vec ? 1700 : esz == 4 ? 3500 : 2600);
    return 5500 + (rounds == 1 ? step : rounds * (3100 + step / 2));
}

tdq_status launch_grad_small(GradSmallArgs a, tdq_dtype dy_dtype, bool vec, cudaStream_t st) {
    const int64_t tiles = (a.O + kSmallO - 1) / kSmallO * a.Kb;
    const cudaError_t e = dy_dtype == TDQ_F32    ? vec ? launch_small<TDQ_F32, true>(a, tiles, st) : launch_small<TDQ_F32, false>(a, tiles, st)
                          : dy_dtype == TDQ_BF16 ? vec ? launch_small<TDQ_BF16, true>(a, tiles, st) : launch_small<TDQ_BF16, false>(a, tiles, st)
                          : vec                  ? launch_small<TDQ_F16, true>(a, tiles, st)
                                                 : launch_small<TDQ_F16, false>(a, tiles, st);
    if (e != cudaSuccess) return TDQ_ERR_CUDA;
    g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return TDQ_OK;
}

}  // namespace tdq
