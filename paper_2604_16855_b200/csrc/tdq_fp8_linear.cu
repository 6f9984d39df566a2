// tdq_fp8_linear: y[m,o] = bias[o] + sum_k xs[m,k] ws[o/128,k] sum_{i in block k} x[m,i] w[o,i] on E4M3 codes.
//
// The sum of a block of 128 channels is four tensor-core instructions (kind::f8f6f4, binary32 accumulator in TMEM); its two scales
// change from block to block, so each block's sums are taken out of TMEM and added, scaled, to binary32 registers.
// Two kernels: tiles of 256 x 256 or 256 x 128 by pairs of CTAs (tdq_fp8_pair.cu) for layers with enough of them, and here the one for few tokens.
//
// fp8_split_kernel.  Few tokens: the time is that of reading the weights once, so all SMs have to read, however few rows the output
// has.  128 output channels are the instruction's 128 rows and NT tokens (16 .. 128) its columns; the contraction is cut in up to eight
// parts, one CTA of a cluster each, whose sums meet in distributed shared memory and are added in rank order: no atomics, no
// workspace, the same bits every time.  Up to 32 tokens the parts send their sums (st.async, counted by a barrier of the channel's owner): read between
// two cluster barriers that order memory they took 3100 of 9500 clocks on 1 x 4096 -> 4096, as much as the loads (6.2 -> 5.4 us).
// More sums than that are read by their owners all the same (128 tokens: 10.1 us, sent 11.3), since the room that they need where they are sent
// is two ring stages, and an owner of channels stores narrower pieces than an owner of tokens.
// Warps 0 and 2 load (tensor maps, 16 KB of weights and the tokens' 128 bytes a stage), warp 1 issues, warp 3 lays out the tokens' factors
// xs * ws of a block in shared memory, the others scale and add: a thread has one output channel and up to 32 tokens.
// Measured, from a graph: 1 x 4096 -> 4096 bf16 5.1 us with the weights in L2, 6.9 from memory (floor 2.6), 1 x 8192 -> 8192 14.7 (10.3), 576 x 384 -> 960 4.5.
// The tensor copies bring 38 bytes a clock to an SM, whatever their size (stages of two blocks: no gain); the rest is the chain from launch to
// first tile (1500 clocks), through the last tile, and the meeting.  Not kept: the weights prefetched to L2 ahead of the wait for the kernel
// before (a layer behind its quantizer 6.5 -> 7.0 us, 1 x 8192 -> 8192 14.7 -> 19.9).
#include <algorithm>

#include "tdq_tc.cuh"
#include "tdq_fp8.cuh"
#include "tdq_activation.cuh"

namespace tdq {

bool fp8_operand_map(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int box_rows) {
    static const TensorMapEncodeFn encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &res) != cudaSuccess || res != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return reinterpret_cast<TensorMapEncodeFn>(fn);
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)cols};
    const cuuint32_t box[2] = {(cuuint32_t)kFp8Block, (cuuint32_t)box_rows};
    const cuuint32_t elem_strides[2] = {1u, 1u};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

constexpr int64_t kFp8MaxExtent = INT32_MAX - 256;   // coordinates of the copies are 32-bit
constexpr int kSplitMaxStages = 12;
constexpr int kSplitMax = 8;                 // CTAs of a cluster
constexpr int kSplitSlots = 4;               // accumulators in TMEM
constexpr uint32_t kSplitCtrl = 1024;
constexpr uint32_t kWBytes = 128 * 128;      // a stage's weights
constexpr int kFactorChunk = 8;              // blocks whose factors are handed over at a time; two chunks' places
constexpr int kFactorSlots = 2 * kFactorChunk;
constexpr int kSplitWarp0 = 4;               // first adding warp

template <int NT> struct SplitShape {
    static constexpr int kCols = NT < 32 ? NT : 32;          // tokens per adding thread
    static constexpr int kWarps = 4 * (NT / kCols);
    static constexpr int kThreads = (kSplitWarp0 + kWarps) * 32;
    static constexpr uint32_t kStage = kWBytes + NT * 128;
    static constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    static constexpr uint32_t kSumStride = (NT + 4) * 4;     // bytes of a channel's sums, one part
    static constexpr bool kSend = NT <= 32;                  // sums are sent, not read
    static constexpr uint32_t kFixed = kSplitCtrl + 1024 + kFactorSlots * NT * 4 + (kSend ? (128 + kSplitMax) * kSumStride : 0);
};

struct SplitCtrl {
    uint64_t full[kSplitMaxStages], empty[kSplitMaxStages];
    uint64_t tfull[kSplitSlots], tempty[kSplitSlots];
    uint64_t factors[kFactorSlots];              // a block's factors are there
    uint64_t taken[2];                           // a chunk's factors have been read
    uint64_t sums;                               // all parts' sums of this CTA's channels have arrived
};
static_assert(sizeof(Ctrl) + sizeof(SplitCtrl) <= kSplitCtrl, "control block outgrew its reservation");

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}
// N consecutive columns of this warp's 32 TMEM lanes, waited for: lane i receives row i
template <int N>
__device__ __forceinline__ void tmem_ld_wait(uint32_t taddr, uint32_t* v) {
    static_assert(N == 16 || N == 32, "columns");
    if constexpr (N == 16)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
                     "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                       "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                     : "r"(taddr)
                     : "memory");
    else
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
                     "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                     "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                       "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                       "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                       "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                     : "r"(taddr)
                     : "memory");
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// The arrival that orders nothing: one that does waits for the thread's stores, about 2000 clocks behind those of y.
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// sixteen bytes to another CTA's shared memory, counted by a barrier there
__device__ __forceinline__ void send16(uint32_t addr_c, float2 a, float2 b, uint32_t bar_c) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(addr_c), "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "r"(bar_c) : "memory");
}

// An output with what follows the layer: z, stored where it is kept, then activation(z) + residual.
__device__ __forceinline__ float load_as(const void* p, int64_t at, int type) {
    if (type == TDQ_F32) return reinterpret_cast<const float*>(p)[at];
    const uint16_t v = reinterpret_cast<const uint16_t*>(p)[at];
    return type == TDQ_BF16 ? widen<TDQ_BF16>(v) : widen<TDQ_F16>(v);
}
__device__ __forceinline__ float finish(const Fp8Epilogue& e, int type, int64_t m, int64_t o, float z) {
    if (e.pre) {
        const int64_t at = m * e.pre_stride + o;
        if (type == TDQ_F32) reinterpret_cast<float*>(e.pre)[at] = z;
        else reinterpret_cast<uint16_t*>(e.pre)[at] = (uint16_t)pack16(z, 0.f, type == TDQ_F16);
    }
    z = activate_by(e.activation, z);
    return e.residual ? z + load_as(e.residual, m * e.residual_stride + o, type) : z;
}
struct Nothing {};

// EPI: with what follows the layer, in kernels of their own.
template <int NT, bool EPI>
__device__ __forceinline__ void split_body(const Fp8Args& a, const std::conditional_t<EPI, Fp8Epilogue, Nothing>& e, const CUtensorMap& xmap, const CUtensorMap& wmap) {
    using Sh = SplitShape<NT>;
    constexpr int CW = Sh::kCols;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    Ctrl* c = reinterpret_cast<Ctrl*>(smem_raw);             // its abort flag and TMEM address; the barriers are g's
    SplitCtrl* g = reinterpret_cast<SplitCtrl*>(smem_raw + sizeof(Ctrl));
    const uint32_t sm_s = smem_u32(smem_raw);
    const uint32_t ring_s = (sm_s + kSplitCtrl + 1023u) & ~1023u;
    const uint32_t n_stages = (uint32_t)a.n_stages;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kSplitMaxStages; ++i) { mbar_init(&g->full[i], 2); mbar_init(&g->empty[i], 1); }
        for (int i = 0; i < kSplitSlots; ++i) { mbar_init(&g->tfull[i], 1); mbar_init(&g->tempty[i], Sh::kWarps); }
        for (int i = 0; i < kFactorSlots; ++i) mbar_init(&g->factors[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&g->taken[i], Sh::kWarps);
        mbar_init(&g->sums, 1);
        c->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&wmap)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&xmap)) : "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem_base)), "n"(kSplitSlots * NT) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const uint32_t split = (uint32_t)a.split, rank = split > 1 ? fp8_cluster_rank() : 0u;
    tc_fence_before();
    __syncthreads();
    if (split > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // this CTA's barriers are initialised
    tc_fence_after();
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0u;
    const uint32_t tmem_base = c->tmem_base;
    const uint32_t tile = blockIdx.x / split;                // token tiles of an output tile follow each other: its weights stay in L2
    const int ot = (int)(tile / (uint32_t)a.tiles_m), tt = (int)(tile - (uint32_t)ot * (uint32_t)a.tiles_m);
    const uint32_t factors_s = ring_s + n_stages * Sh::kStage, sums_s = factors_s + kFactorSlots * NT * 4;
    const int n_tok = (int)min((int64_t)NT, a.M - (int64_t)tt * NT);
    // channels [mine, mine + n_mine) of the tile are finished here
    const uint32_t per = (128u + split - 1u) / split, mine = rank * per, n_mine = min(per, 128u - mine);
    if (Sh::kSend && split > 1 && threadIdx.x == 0) mbar_expect_tx(&g->sums, n_mine * split * (((uint32_t)n_tok + 3u) & ~3u) * 4u);
    const int kb0 = (int)((int64_t)a.K * rank / split), n_kb = (int)((int64_t)a.K * (rank + 1) / split) - kb0;

    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------ loads: weights by warp 0, tokens by warp 2
        const bool is_w = warp == 0;
        const uint32_t bytes = is_w ? kWBytes : NT * 128, dst = ring_s + (is_w ? 0u : kWBytes);
        const int row = is_w ? ot * 128 : tt * NT;
        uint32_t s = 0, ph = 0;
#pragma unroll 1
        for (int i = 0; i < n_kb; ++i) {
            if (i >= (int)n_stages) fp8_wait(smem_u32(&g->empty[s]), ph, c, a.status, 5u);
            if (c->abort_flag) break;
            if (elect_one()) {
                mbar_expect_tx(&g->full[s], bytes);
                tma_load_2d(dst + s * Sh::kStage, is_w ? &wmap : &xmap, (kb0 + i) * (int)kFp8Block, row, &g->full[s]);
            }
            __syncwarp();
            if (++s == n_stages) { s = 0; ph ^= (uint32_t)(i >= (int)n_stages); }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issue
        uint32_t s = 0, ph = 0;
        for (int i = 0; i < n_kb; ++i) {
            const uint32_t slot = (uint32_t)i % kSplitSlots;
            fp8_wait(smem_u32(&g->tempty[slot]), (((uint32_t)i / kSplitSlots) & 1u) ^ 1u, c, a.status, 3u);
            fp8_wait(smem_u32(&g->full[s]), ph, c, a.status, 4u);
            if (c->abort_flag) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t wd = sw_desc(ring_s + s * Sh::kStage), xd = sw_desc(ring_s + s * Sh::kStage + kWBytes);
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_f8(tmem_base + slot * NT, wd + 2 * k, xd + 2 * k, Sh::kIdesc, k ? 1u : 0u);
                mma_commit(smem_u32(&g->empty[s]));
                mma_commit(smem_u32(&g->tfull[slot]));
            }
            __syncwarp();
            if (++s == n_stages) { s = 0; ph ^= 1; }
        }
    } else if (warp == 3) {
        // ------------------------------------------------------------ factors
        constexpr int kTok = (NT + 31) / 32;                 // tokens per lane
        const float* ws = a.wscale + (int64_t)ot * a.K + kb0;
        const float* xs[kTok];
#pragma unroll
        for (int i = 0; i < kTok; ++i) xs[i] = a.xscale + min((int64_t)tt * NT + lane + 32 * i, a.M - 1) * a.K + kb0;   // past the end: never stored
        float f[kFactorChunk][kTok];
        const auto load = [&](int c0) {
#pragma unroll
            for (int q = 0; q < kFactorChunk; ++q) {
                const int kb = min(c0 + q, n_kb - 1);
                const float w = __ldg(ws + kb);
#pragma unroll
                for (int i = 0; i < kTok; ++i) f[q][i] = __ldg(xs[i] + kb) * w;
            }
        };
        load(0);
        for (int c0 = 0; c0 < n_kb && !c->abort_flag; c0 += kFactorChunk) {
            const int half = (c0 / kFactorChunk) & 1;
            if (c0 >= kFactorSlots) fp8_wait(smem_u32(&g->taken[half]), (uint32_t)(c0 / kFactorSlots + 1) & 1u, c, a.status, 6u);
#pragma unroll
            for (int q = 0; q < kFactorChunk; ++q) {
                const uint32_t place = (uint32_t)(half * kFactorChunk + q), at = factors_s + (place * NT + lane) * 4u;
                if (c0 + q < n_kb) {
#pragma unroll
                    for (int j = 0; j < kTok; ++j)
                        if (NT >= 32 || lane < NT) sts32(at + j * 128, __float_as_uint(f[q][j]));
                    __syncwarp();
                    mbar_arrive_lane0_s(smem_u32(&g->factors[place]), lane);
                }
            }
            if (c0 + kFactorChunk < n_kb) load(c0 + kFactorChunk);
        }
    } else if (warp >= kSplitWarp0) {
        // ------------------------------------------------------------ scaled sums
        const int pw = warp - kSplitWarp0, quarter = warp & 3, cg = pw >> 2;
        float2 acc[CW / 2];
#pragma unroll
        for (int j = 0; j < CW / 2; ++j) acc[j] = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int i = 0; i < n_kb; ++i) {
            const uint32_t slot = (uint32_t)i % kSplitSlots, place = (uint32_t)i % kFactorSlots;
            fp8_wait(smem_u32(&g->factors[place]), ((uint32_t)i / kFactorSlots) & 1u, c, a.status, 7u);
            fp8_wait(smem_u32(&g->tfull[slot]), ((uint32_t)i / kSplitSlots) & 1u, c, a.status, 2u);
            if (c->abort_flag) break;
            tc_fence_after();
            uint32_t v[CW];
            tmem_ld_wait<CW>(tmem_base + ((uint32_t)(quarter * 32) << 16) + slot * NT + cg * CW, v);
            tc_fence_before();
            __syncwarp();
            mbar_arrive_lane0_s(smem_u32(&g->tempty[slot]), lane);
            const uint32_t f_s = factors_s + (place * NT + cg * CW) * 4u;
#pragma unroll
            for (int j = 0; j < CW / 4; ++j) {
                const float4 f = lds_f4(f_s + 16u * j);
                acc[2 * j] = __ffma2_rn(make_float2(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1])), make_float2(f.x, f.y), acc[2 * j]);
                acc[2 * j + 1] = __ffma2_rn(make_float2(__uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])), make_float2(f.z, f.w), acc[2 * j + 1]);
            }
            if (i % kFactorChunk == kFactorChunk - 1) {
                __syncwarp();
                mbar_arrive_lane0_s(smem_u32(&g->taken[(i / kFactorChunk) & 1]), lane);
            }
        }
        if (split > 1) cluster_wait();                       // all CTAs' barriers are initialised
        if constexpr (Sh::kSend) {
            const uint32_t ch = (uint32_t)(quarter * 32 + lane), owner = ch / per;
            const uint32_t to = sums_s + (rank * per + ch - owner * per) * Sh::kSumStride + cg * CW * 4u;
            const uint32_t to_c = map_to_cta(to, split > 1 ? owner : 0u), bar_c = map_to_cta(smem_u32(&g->sums), split > 1 ? owner : 0u);
#pragma unroll
            for (int j = 0; j < CW / 4; ++j) {
                if (cg * CW + 4 * j >= n_tok) break;
                if (split > 1) send16(to_c + 16u * j, acc[2 * j], acc[2 * j + 1], bar_c);
                else sts128(to + 16u * j, __float_as_uint(acc[2 * j].x), __float_as_uint(acc[2 * j].y), __float_as_uint(acc[2 * j + 1].x), __float_as_uint(acc[2 * j + 1].y));
            }
        } else {
            // the last instruction has read the ring; the sums take its place, token by token
#pragma unroll
            for (int j = 0; j < CW / 2; ++j) {
                const uint32_t at = ring_s + ((uint32_t)(cg * CW + 2 * j) * 128u + (uint32_t)(quarter * 32 + lane)) * 4u;
                sts32(at, __float_as_uint(acc[j].x));
                sts32(at + 512u, __float_as_uint(acc[j].y));
            }
        }
    }
    if (split > 1 && warp < kSplitWarp0) cluster_wait();
    tc_fence_before();
    if constexpr (Sh::kSend) {
        if (split > 1) cluster_arrive_relaxed();                 // nothing more is sent
        __syncthreads();
        if (split > 1) fp8_wait(smem_u32(&g->sums), 0u, c, a.status, 8u);
        // four tokens of a channel a thread: lanes store neighbouring channels
        const int64_t o0 = (int64_t)ot * 128 + mine;
        for (uint32_t u = threadIdx.x; u < n_mine * (((uint32_t)n_tok + 3u) / 4u); u += Sh::kThreads) {
            const uint32_t quad = u / n_mine, ch = u - quad * n_mine;
            const int64_t o = o0 + ch;
            if (o >= a.O) continue;
            const float b = a.bias ? __ldg(a.bias + o) : 0.f;
            float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (uint32_t p = 0; p < split; ++p) {
                const float4 q = lds_f4(sums_s + (p * per + ch) * Sh::kSumStride + quad * 16u);
                r[0] += q.x; r[1] += q.y; r[2] += q.z; r[3] += q.w;
            }
            const int64_t at = ((int64_t)tt * NT + quad * 4) * a.y_stride + o;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((int)(quad * 4) + j >= n_tok) break;
                float v = r[j] + b;
                if constexpr (EPI) v = finish(e, a.y_type, (int64_t)tt * NT + quad * 4 + j, o, v);
                if (a.y_type == TDQ_F32) reinterpret_cast<float*>(a.y)[at + j * a.y_stride] = v;
                else reinterpret_cast<uint16_t*>(a.y)[at + j * a.y_stride] = (uint16_t)pack16(v, 0.f, a.y_type == TDQ_F16);
            }
        }
    } else {
        __syncthreads();
        if (split > 1) fp8_cluster_sync();                       // all CTAs' sums are there
        const int64_t o0 = (int64_t)ot * 128;
        for (uint32_t u = rank * Sh::kThreads + threadIdx.x; u < (uint32_t)n_tok * 32u; u += split * Sh::kThreads) {
            const int64_t o = o0 + (u & 31u) * 4;
            if (o >= a.O) continue;
            float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (uint32_t p = 0; p < split; ++p) {
                const float4 q = ld_cluster4(map_to_cta(ring_s + u * 16u, p));
                r[0] += q.x; r[1] += q.y; r[2] += q.z; r[3] += q.w;
            }
            const int left = (int)min((int64_t)4, a.O - o);
            if (a.bias) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < left) r[j] += __ldg(a.bias + o + j);
            }
            if constexpr (EPI) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < left) r[j] = finish(e, a.y_type, (int64_t)tt * NT + (u >> 5), o + j, r[j]);
            }
            const int64_t at = ((int64_t)tt * NT + (u >> 5)) * a.y_stride + o;
            if (a.y_type == TDQ_F32) {
                float* y = reinterpret_cast<float*>(a.y) + at;
                if (a.y_vec && left == 4) *reinterpret_cast<float4*>(y) = make_float4(r[0], r[1], r[2], r[3]);
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < left) y[j] = r[j];
            } else {
                uint16_t* y = reinterpret_cast<uint16_t*>(a.y) + at;
                const uint32_t w0 = pack16(r[0], r[1], a.y_type == TDQ_F16), w1 = pack16(r[2], r[3], a.y_type == TDQ_F16);
                if (a.y_vec && left == 4) *reinterpret_cast<uint2*>(y) = make_uint2(w0, w1);
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < left) y[j] = (uint16_t)((j & 2 ? w1 : w0) >> (16 * (j & 1)));
            }
        }
        __syncwarp();
        if (split > 1) cluster_arrive_relaxed();                 // nothing more is read
    }
    if (c->abort_flag) __nanosleep(1000000);                 // a wait gave up: give copies and tensor core a moment
    __syncwarp();                                            // out of the loops over outputs: what follows is the whole warp's
    if (split > 1) cluster_wait();                           // no CTA leaves while another sends to it or reads from it
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(kSplitSlots * NT) : "memory");
}

template <int NT>
__global__ void __launch_bounds__(SplitShape<NT>::kThreads, NT == 128 ? 1 : 2)
fp8_split_kernel(const Fp8Args a, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap) {
    split_body<NT, false>(a, Nothing{}, xmap, wmap);
}
template <int NT>
__global__ void __launch_bounds__(SplitShape<NT>::kThreads, NT == 128 ? 1 : 2)
fp8_split_epilogue_kernel(const Fp8Args a, const Fp8Epilogue e, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap) {
    split_body<NT, true>(a, e, xmap, wmap);
}

// Which kernel, and in how many parts: the least of these estimates in units of 10 ns, fitted to layers of 1 to 9000 tokens, 384 to 7040
// -> 48 to 8192 channels with every kernel and number of parts, from a graph.  On 70 others the choice costs 1.7 % more than the best one in the mean, 23 % at
// worst (591 x 6317 -> 54 bf16 7.95 us for 6.47).
//   NT tokens, s parts:  start x rounds + block x (blocks of a part) x (CTAs an SM runs) + meet x s (s > 1);  a round is as many clusters of s
//                        CTAs as the GPU holds, two CTAs per SM, one of NT = 128
//   pairs of CTAs:       start + block x K x rounds + end x (rounds - 1);  a round is a tile of 256 tokens and 256 or 128 channels for every
//                        pair of SMs
// Above 64 tokens, from as many 256 x 256 tiles as SMs on (two rounds) those are taken without an estimate, which charges a further round of them too
// much.  Measured with 256 x 128 instead: 148 tiles of 6 and 32 blocks 11.9 -> 13.2 and 36.5 -> 46 us, 152 of 16 and 32 25.4 -> 25.8 and 43.5 -> 45.5, 240
// to 640 of 6 5 to 12 % slower; faster only just above two rounds of a short contraction (2000 x 768 -> 4712 13.8 -> 13.3, 2048 x 768 -> 5120 fp32 21.3 -> 19.4).
// A cluster lies in one group of SMs, so fewer of them fit than SMs / s: with rounds counted in CTAs 2259 x 5113 -> 45 waited for two of
// eighteen clusters of eight (14.2 us; now 8.9).  Against 128 tokens a tile throughout: 576 x 384 -> 960 6.9 -> 4.7 us, 256 x 1024 -> 1024 6.9 -> 5.4.
struct Way { int nt, split; };                             // nt == 256: pairs, split the tile's columns
Way choose_way(int64_t M, int64_t O, int K, int n_sm) {
    // Clusters of 1 .. 8 CTAs that a B200 of 148 SMs holds, one CTA and two per SM, as the runtime reports them.  Constants, not a question to the GPU
    // at hand: which SMs form a group differs from one to the next, and the bits of a sum would with it.
    static const int holds[2][kSplitMax] = {{148, 74, 45, 33, 26, 22, 15, 15}, {296, 148, 93, 71, 56, 45, 37, 33}};
    static const struct { int nt, start, block, meet; } kinds[4] = {{16, 305, 22, 3}, {32, 350, 32, 2}, {64, 354, 35, 10}, {128, 480, 36, 0}};
    const int64_t tiles_n = fp8_blocks(O), pair_tiles = ((M + 255) / 256) * ((O + 255) / 256);
    if (M > 64 && pair_tiles >= n_sm) return {256, 256};
    Way best = {256, 256};
    const int64_t pairs = n_sm / 2 > 0 ? n_sm / 2 : 1, pair_rounds = (pair_tiles + pairs - 1) / pairs;
    int64_t least = INT64_MAX;
    if (M > 64) {
        const int64_t narrow_rounds = ((M + 255) / 256 * tiles_n + pairs - 1) / pairs;
        const int64_t wide = 475 + 34 * K * pair_rounds + 380 * (pair_rounds - 1), narrow = 360 + 27 * K * narrow_rounds + 160 * (narrow_rounds - 1);
        least = std::min(wide, narrow);
        if (narrow < wide) best.split = 128;
    }
    for (const auto& k : kinds) {
        if (k.nt > 16 && k.nt / 2 >= M) break;             // more than half of the tile would be empty
        const int64_t tiles = tiles_n * ((M + k.nt - 1) / k.nt);
        for (int s = 1; s <= kSplitMax && s <= K; ++s) {
            const int two = k.nt != 128;
            const int64_t at_once = std::max<int64_t>(1, (int64_t)holds[two][s - 1] * n_sm / 148), rounds = (tiles + at_once - 1) / at_once;
            const int64_t per_sm = std::max<int64_t>((tiles * s + n_sm - 1) / n_sm, two ? 2 * rounds - 1 : rounds);
            const int64_t cost = k.start * rounds + (int64_t)k.block * ((K + s - 1) / s) * per_sm + (s > 1 ? k.meet * s : 0);
            if (cost < least) { least = cost; best = {k.nt, s}; }
        }
    }
    return best;
}

template <int NT, bool EPI>
tdq_status launch_split_as(Fp8Args a, const std::conditional_t<EPI, Fp8Epilogue, Nothing>& e, int split, const uint8_t* xcodes, const CUtensorMap& wmap, int n_sm, int dev, cudaStream_t stream) {
    using Sh = SplitShape<NT>;
    CUtensorMap xmap;
    if (!fp8_operand_map(&xmap, xcodes, a.M, (int64_t)a.K * kFp8Block, NT)) return TDQ_ERR_CUDA;
    const int64_t tiles_m = (a.M + NT - 1) / NT, tiles_n = fp8_blocks(a.O), tiles = tiles_m * tiles_n;
    if (tiles > (int64_t)INT32_MAX / kSplitMax) return TDQ_ERR_UNSUPPORTED;
    a.split = split;
    a.tiles_m = (int32_t)tiles_m;
    a.tiles_n = (int32_t)tiles_n;
    // Two CTAs per SM, so that the next call's set themselves up while this one's end (a ring as deep as one CTA could have: 5.4 against 5.1 us on
    // 1 x 4096 -> 4096).  Two CTAs of clusters that wait for each other must both get their TMEM columns (512 in all): at least
    // 77 KB a CTA leaves room for two, and the 512 columns of NT = 128 come with so much shared memory that no other of these CTAs
    // fits beside them.
    const int per_cta = NT == 128 ? kSmemLimit : 113 * 1024;
    const int per = (a.K + a.split - 1) / a.split;
    const int least = ((NT == 128 ? 152 : 77) * 1024 - (int)Sh::kFixed + (int)Sh::kStage - 1) / (int)Sh::kStage;
    int stages = (per_cta - (int)Sh::kFixed) / (int)Sh::kStage;
    stages = stages > kSplitMaxStages ? kSplitMaxStages : stages;
    a.n_stages = stages < per ? stages : per > least ? per : least;
    const uint32_t smem = Sh::kFixed + (uint32_t)a.n_stages * Sh::kStage;
    static std::atomic<uint64_t> smem_done{0};
    if constexpr (EPI) {
        if (allow_smem(fp8_split_epilogue_kernel<NT>, kSmemLimit, smem_done, dev) != cudaSuccess) return TDQ_ERR_CUDA;
    } else {
        if (allow_smem(fp8_split_kernel<NT>, kSmemLimit, smem_done, dev) != cudaSuccess) return TDQ_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.split));
    cfg.blockDim = dim3(Sh::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)a.split;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    cudaError_t err;
    if constexpr (EPI) err = cudaLaunchKernelEx(&cfg, fp8_split_epilogue_kernel<NT>, a, e, xmap, wmap);
    else err = cudaLaunchKernelEx(&cfg, fp8_split_kernel<NT>, a, xmap, wmap);
    if (err != cudaSuccess) return TDQ_ERR_CUDA;
    g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return TDQ_OK;
}
template <int NT>
tdq_status launch_split(const Fp8Args& a, const Fp8Epilogue& e, int split, const uint8_t* xcodes, const CUtensorMap& wmap, int n_sm, int dev, cudaStream_t stream) {
    if (e.any()) return launch_split_as<NT, true>(a, e, split, xcodes, wmap, n_sm, dev, stream);
    return launch_split_as<NT, false>(a, {}, split, xcodes, wmap, n_sm, dev, stream);
}

// One warp: a fresh barrier with one expected arrival that never comes, waited on with the two kernels' own routine and a short limit.  Nothing is
// in flight when the warp leaves.
__global__ void __launch_bounds__(32) fp8_wait_selftest_kernel(uint32_t* status, uint32_t limit) {
    __shared__ Ctrl c;
    if (threadIdx.x == 0) {
        mbar_init(&c.full[0], 1);
        c.abort_flag = 0;
    }
    __syncwarp();
    fp8_wait_more(smem_u32(&c.full[0]), 0u, &c, status, 13u, limit);
}

}  // namespace

tdq_status fp8_wait_selftest(long long limit_cycles, uint32_t* status, cudaStream_t stream) {
    fp8_wait_selftest_kernel<<<1, 32, 0, stream>>>(status, (uint32_t)limit_cycles);
    return cuda_status(cudaGetLastError());
}

}  // namespace tdq

using namespace tdq;

extern "C" size_t tdq_fp8_linear_workspace_bytes(int64_t, int64_t, int64_t) { return kWorkspaceHeader; }

extern "C" tdq_status tdq_fp8_linear_tiles(int64_t M, int64_t I_pad, int64_t O, int32_t sm_count, int32_t* tokens, int32_t* channels, int32_t* parts) {
    if (M < 0 || O < 0 || I_pad <= 0 || I_pad % kFp8Block || sm_count <= 0 || !tokens || !channels || !parts) return TDQ_ERR_INVALID_ARG;
    if (M > kFp8MaxExtent || O > kFp8MaxExtent || I_pad > kFp8MaxExtent) return TDQ_ERR_UNSUPPORTED;
    *tokens = *channels = *parts = 0;
    if (M == 0 || O == 0) return TDQ_OK;
    const Way way = choose_way(M, O, (int)(I_pad / kFp8Block), sm_count);
    *tokens = way.nt;
    *channels = way.nt == 256 ? way.split : 128;
    *parts = way.nt == 256 ? 1 : way.split;
    return TDQ_OK;
}

namespace {
tdq_status fp8_linear(const uint8_t* xcodes, const float* xscale, const uint8_t* wcodes, const float* wscale, const float* bias, int64_t M, int64_t I_pad,
                      int64_t O, const Fp8Epilogue& e, void* y, tdq_dtype y_dtype, int64_t y_row_stride, void* workspace, size_t workspace_bytes,
                      void* cuda_stream) {
    if (M < 0 || O < 0 || I_pad <= 0 || I_pad % kFp8Block || y_row_stride < O) return TDQ_ERR_INVALID_ARG;
    if (y_dtype != TDQ_F32 && y_dtype != TDQ_BF16 && y_dtype != TDQ_F16) return TDQ_ERR_INVALID_ARG;
    if (M == 0 || O == 0) return TDQ_OK;
    if (!xcodes || !xscale || !wcodes || !wscale || !y) return TDQ_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < kWorkspaceHeader) return TDQ_ERR_WORKSPACE;
    const uintptr_t esz = y_dtype == TDQ_F32 ? 4 : 2;
    const auto off = [](const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; };
    if (off(xcodes, 16) || off(wcodes, 16) || off(workspace, 16) || off(xscale, 4) || off(wscale, 4) || off(bias, 4) || off(y, esz) ||
        off(e.residual, esz) || off(e.pre, esz))
        return TDQ_ERR_ALIGNMENT;
    if (M > kFp8MaxExtent || O > kFp8MaxExtent || I_pad > kFp8MaxExtent) return TDQ_ERR_UNSUPPORTED;
    int dev = 0;
    const int n_sm = current_device_sm_count(&dev);
    if (n_sm <= 0) return TDQ_ERR_CUDA;
    Fp8Args a = {};
    a.xscale = xscale;
    a.wscale = wscale;
    a.bias = bias;
    a.y = y;
    a.M = M;
    a.O = O;
    a.y_stride = y_row_stride;
    a.K = (int32_t)(I_pad / kFp8Block);
    a.y_type = y_dtype;
    a.y_vec = !off(y, 16) && (y_row_stride * (int64_t)esz) % 16 == 0;
    a.status = reinterpret_cast<uint32_t*>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    Fp8Epilogue f = e;
    f.residual_vec = !off(e.residual, 16) && (e.residual_stride * (int64_t)esz) % 16 == 0;
    f.pre_vec = !off(e.pre, 16) && (e.pre_stride * (int64_t)esz) % 16 == 0;
    const Way way = choose_way(M, O, a.K, n_sm);
    CUtensorMap wmap;
    if (!fp8_operand_map(&wmap, wcodes, O, I_pad, way.nt == 256 ? way.split / 2 : 128)) return TDQ_ERR_CUDA;
    if (way.nt == 16) return launch_split<16>(a, f, way.split, xcodes, wmap, n_sm, dev, st);
    if (way.nt == 32) return launch_split<32>(a, f, way.split, xcodes, wmap, n_sm, dev, st);
    if (way.nt == 64) return launch_split<64>(a, f, way.split, xcodes, wmap, n_sm, dev, st);
    if (way.nt == 128) return launch_split<128>(a, f, way.split, xcodes, wmap, n_sm, dev, st);
    CUtensorMap xmap;
    if (!fp8_operand_map(&xmap, xcodes, M, I_pad, 128)) return TDQ_ERR_CUDA;
    return launch_fp8_pair(a, f, way.split, xmap, wmap, n_sm, dev, st);
}
}  // namespace

extern "C" tdq_status tdq_fp8_linear(const uint8_t* xcodes, const float* xscale, const uint8_t* wcodes, const float* wscale, const float* bias,
                                     int64_t M, int64_t I_pad, int64_t O, void* y, tdq_dtype y_dtype, int64_t y_row_stride, void* workspace,
                                     size_t workspace_bytes, void* cuda_stream) {
    return fp8_linear(xcodes, xscale, wcodes, wscale, bias, M, I_pad, O, Fp8Epilogue{}, y, y_dtype, y_row_stride, workspace, workspace_bytes, cuda_stream);
}

extern "C" tdq_status tdq_fp8_linear_epilogue(const uint8_t* xcodes, const float* xscale, const uint8_t* wcodes, const float* wscale, const float* bias,
                                              int64_t M, int64_t I_pad, int64_t O, const tdq_fp8_epilogue* e, void* y, tdq_dtype y_dtype,
                                              int64_t y_row_stride, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!e || e->activation < TDQ_ACT_NONE || e->activation > TDQ_ACT_SILU || (e->residual && e->residual_row_stride < O) || (e->pre && e->pre_row_stride < O) ||
        (e->pre && e->pre == y))
        return TDQ_ERR_INVALID_ARG;
    if (e->pre && e->residual) return TDQ_ERR_UNSUPPORTED;
    Fp8Epilogue f = {};
    f.activation = e->activation;
    f.residual = e->residual;
    f.residual_stride = e->residual_row_stride;
    f.pre = e->pre;
    f.pre_stride = e->pre_row_stride;
    return fp8_linear(xcodes, xscale, wcodes, wscale, bias, M, I_pad, O, f, y, y_dtype, y_row_stride, workspace, workspace_bytes, cuda_stream);
}
