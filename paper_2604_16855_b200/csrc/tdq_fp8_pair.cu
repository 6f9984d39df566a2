// tdq_fp8_linear for layers with many tiles: two CTAs of a cluster on a tile of 256 tokens x 256 output channels.
//
// What bounds it.  A block of 128 channels is 512 clocks of tensor time per 256 x 256 tile; the 32 KB of operands that it uses in each
// CTA are written to shared memory meanwhile (64 bytes of the 128 a clock).  The sums of a block have scales of their own, so
// all 32768 of a CTA leave TMEM and are added to registers in the same time: 64 a clock of the 128 that the FMA pipe takes.  What must not
// happen is that tensor core and adders wait for each other: the tile's columns are two halves with two accumulators each (all 512
// TMEM columns), filled and drained in turn, so that three quarters of TMEM are in the tensor core's hands while one is read.
//
//   warps 0, 3  loads of this CTA's 128 token rows and 128 weight rows (tensor maps, 128-byte swizzle, 16 KB each a stage), signalled to
//               CTA 0's barrier
//   warp 1      CTA 0: issues the instructions (cta_group::2, 256 x 128 x 32), commits to both CTAs' barriers
//   warp 2      allocates TMEM
//   warps 4-11  scale and add: 32 token rows x 128 columns each in registers (so 232 registers a thread, 40 for the others), then bias,
//               rounding and the store through a swizzled strip of 4 KB
//
// Half h is columns 64 h .. 64 h + 63 of each CTA's 128 weight rows: with cta_group::2 either CTA brings half of the columns.
#include "tdq_fp8.cuh"
#include "tdq_tc.cuh"

namespace tdq {
namespace {

constexpr int kPairMaxStages = 6;
constexpr uint32_t kPairOperand = 128 * 128;             // bytes of a stage's rows of either operand
constexpr uint32_t kPairStage = 2 * kPairOperand;
constexpr uint32_t kPairCtrl = 1024;
constexpr int kAddWarp0 = 4, kAddWarps = 8;
constexpr int kPairThreads = (kAddWarp0 + kAddWarps) * 32;
constexpr uint32_t kStrip = 32 * 128;                    // 32 rows of 128 bytes
constexpr uint32_t kBiasBytes = 128 * 4;                 // a warp's columns
constexpr uint32_t kPairIdesc = (1u << 4) | ((128u >> 3) << 17) | ((256u >> 4) << 24);
constexpr int kRegsLoad = 40, kRegsAdd = 232;            // 128 * 40 + 256 * 232 <= 384 * 168

struct PairCtrl {
    uint64_t full[kPairMaxStages];                       // CTA 0: both CTAs' operands of the stage have landed
    uint64_t empty[kPairMaxStages];
    uint64_t tfull[4], tempty[4];                        // accumulator 2 (block & 1) + half (tempty: CTA 0 only)
};

__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma_f8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(kPairIdesc), "r"(accumulate) : "memory");
}
// arrives on the barrier of this address in both CTAs once this thread's instructions so far have completed
__device__ __forceinline__ void commit_pair(uint32_t bar_s) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar_s), "h"((uint16_t)3) : "memory");
}
// lane 0 of a converged warp arrives on a barrier of either CTA, given by its cluster address
__device__ __forceinline__ void arrive_cluster_lane0(uint32_t bar_c, int lane) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}"
                 ::"r"(bar_c), "r"(lane) : "memory");
}
__device__ __forceinline__ void scale_add32(uint64_t* acc, const uint32_t* v, uint64_t d) {
#pragma unroll
    for (int j = 0; j < 16; ++j) fma2(acc[j], pack2(v[2 * j], v[2 * j + 1]), d);
}

// Y16: y has 16-bit elements.
template <bool Y16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
fp8_pair_kernel(const Fp8Args a, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap,
                const __grid_constant__ CUtensorMap ymap) {
    extern __shared__ __align__(128) uint8_t smem_raw[];
    Ctrl* c = reinterpret_cast<Ctrl*>(smem_raw);             // its abort flag and TMEM address; the barriers are g's
    PairCtrl* g = reinterpret_cast<PairCtrl*>(smem_raw + sizeof(Ctrl));
    static_assert(sizeof(Ctrl) + sizeof(PairCtrl) <= kPairCtrl, "control block outgrew its reservation");
    const uint32_t sm_s = smem_u32(smem_raw);
    const uint32_t ring_s = (sm_s + kPairCtrl + 1023u) & ~1023u;   // the same offset in both CTAs
    const uint32_t n_stages = (uint32_t)a.n_stages;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t rank = fp8_cluster_rank();

    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairMaxStages; ++i) { mbar_init(&g->full[i], 2); mbar_init(&g->empty[i], 1); }
        for (int i = 0; i < 4; ++i) { mbar_init(&g->tfull[i], 1); mbar_init(&g->tempty[i], kAddWarps); }
        c->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem_base)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    fp8_cluster_sync();                                      // both CTAs' barriers are initialised
    tc_fence_after();
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0u;
    const uint32_t tmem_base = c->tmem_base;
    const int n_tiles = a.tiles_m * a.tiles_n, n_clusters = (int)gridDim.x / 2, first = (int)blockIdx.x / 2;
    const int K = a.K;

    if (warp < kAddWarp0) {
        setmaxnreg_dec<kRegsLoad>();
        if (warp == 0 || warp == 3) {
            // -------------------------------------------------------- loads: tokens by warp 0, weights by warp 3
            const bool is_x = warp == 0;
            const uint32_t dst0 = ring_s + (is_x ? 0u : kPairOperand);
            const uint32_t full0 = map_to_cta(smem_u32(&g->full[0]), 0), empty_s = smem_u32(&g->empty[0]);
            uint32_t s = 0, ph = 1;
            for (int tile = first; tile < n_tiles && !c->abort_flag; tile += n_clusters) {
                const int mt = tile / a.tiles_n, nt = tile - mt * a.tiles_n;
                const int row = (is_x ? mt : nt) * 256 + (int)rank * 128;   // past the end: the map fills with zeros
#pragma unroll 1
                for (int kb = 0; kb < K; ++kb) {
                    wait_hot(empty_s + s * 8, ph, c, a.status, 5u);
                    if (c->abort_flag) break;
                    if (elect_one()) {
                        if (rank == 0) mbar_expect_tx(&g->full[s], 2 * kPairOperand);   // this operand, both CTAs
                        tma_load_pair(dst0 + s * kPairStage, is_x ? &xmap : &wmap, kb * (int)kFp8Block, row, full0 + s * 8);
                    }
                    __syncwarp();
                    if (++s == n_stages) { s = 0; ph ^= 1; }
                }
            }
        } else if (warp == 1 && rank == 0) {
            // -------------------------------------------------------- MMA issue
            const uint32_t full_s = smem_u32(&g->full[0]), empty_s = smem_u32(&g->empty[0]);
            const uint32_t tfull_s = smem_u32(&g->tfull[0]), tempty_s = smem_u32(&g->tempty[0]);
            const uint64_t xd0 = sw_desc(ring_s), wd0 = sw_desc(ring_s + kPairOperand);
            uint32_t s = 0, ph = 0, n = 0;
            for (int tile = first; tile < n_tiles && !c->abort_flag; tile += n_clusters)
#pragma unroll 1
                for (int kb = 0; kb < K; ++kb, ++n) {
                    const uint32_t slot0 = (n & 1u) * 2, par = ((n >> 1) & 1u) ^ 1u;
                    wait_hot(full_s + s * 8, ph, c, a.status, 4u);
                    const uint64_t xd = xd0 + s * (kPairStage >> 4), wd = wd0 + s * (kPairStage >> 4);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        wait_hot(tempty_s + (slot0 + h) * 8, par, c, a.status, 3u);
                        if (c->abort_flag) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mma_f8_pair(tmem_base + (slot0 + h) * 128, xd + 2 * k, wd + h * (64 * 128 >> 4) + 2 * k, k ? 1u : 0u);
                            if (h == 1) commit_pair(empty_s + s * 8);
                            commit_pair(tfull_s + (slot0 + h) * 8);
                        }
                        __syncwarp();
                    }
                    if (c->abort_flag) break;
                    if (++s == n_stages) { s = 0; ph ^= 1; }
                }
        }
    } else {
        // ------------------------------------------------------------ scaled sums and epilogue
        setmaxnreg_inc<kRegsAdd>();
        const int aw = warp - kAddWarp0, quarter = warp & 3, h = aw >> 2;
        const uint32_t after_s = ring_s + n_stages * kPairStage;
        const uint32_t strip_s = after_s + (uint32_t)aw * kStrip, bias_s = after_s + kAddWarps * kStrip + (uint32_t)aw * kBiasBytes;
        const uint32_t tfull_s = smem_u32(&g->tfull[h]), tempty_c = map_to_cta(smem_u32(&g->tempty[h]), 0);
        const uint32_t tm0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + h * 128;
        uint32_t va[32], vb[32];
#pragma unroll
        for (int q = 0; q < 32; ++q) { va[q] = 0u; vb[q] = 0u; }
        uint32_t n = 0;
        for (int tile = first; tile < n_tiles && !c->abort_flag; tile += n_clusters) {
            const int mt = tile / a.tiles_n, nt = tile - mt * a.tiles_n;
            const int64_t m0 = (int64_t)mt * 256 + rank * 128 + quarter * 32;
            const int64_t n0 = (int64_t)nt * 256 + h * 64;       // columns n0 + 0..63 and n0 + 128 + 0..63
            const int64_t row = m0 + lane < a.M ? m0 + lane : a.M - 1;
            const float* xs = a.xscale + row * K;
            const int last = (int)((a.O - 1) >> 7);
            const float* ws0 = a.wscale + (int64_t)min(2 * nt, last) * K;
            const float* ws1 = a.wscale + (int64_t)min(2 * nt + 1, last) * K;
            uint64_t acc[64];
#pragma unroll
            for (int j = 0; j < 64; ++j) acc[j] = 0ull;
            __syncwarp();                                        // the last tile's biases have been read
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t col = n0 + (i >> 1) * 128 + (i & 1) * 32 + lane;
                sts32(bias_s + (uint32_t)(i * 32 + lane) * 4u, (a.bias && col < a.O) ? __float_as_uint(__ldg(a.bias + col)) : 0u);
            }
            float fx = __ldg(xs), f0 = __ldg(ws0), f1 = __ldg(ws1);
#pragma unroll 1
            for (int kb = 0; kb < K; ++kb, ++n) {
                const float d0f = fx * f0, d1f = fx * f1;
                const int next = min(kb + 1, K - 1);
                fx = __ldg(xs + next);
                f0 = __ldg(ws0 + next);
                f1 = __ldg(ws1 + next);
                const uint64_t d0 = pack2(__float_as_uint(d0f), __float_as_uint(d0f)), d1 = pack2(__float_as_uint(d1f), __float_as_uint(d1f));
                const uint32_t so = (n & 1u) * 2;
                wait_hot(tfull_s + so * 8, (n >> 1) & 1u, c, a.status, 2u);
                if (c->abort_flag) break;
                tc_fence_after();
                const uint32_t tm = tm0 + so * 128;
                tmem_ld32(tm, va);
                tmem_ld_wait_on(va);
                tmem_ld32(tm + 32, vb);
                scale_add32(acc, va, d0);
                tmem_ld_wait_on(vb);
                tmem_ld32(tm + 64, va);
                scale_add32(acc + 16, vb, d0);
                tmem_ld_wait_on(va);
                tmem_ld32(tm + 96, vb);
                scale_add32(acc + 32, va, d1);
                tmem_ld_wait_on(vb);
                tc_fence_before();
                __syncwarp();
                arrive_cluster_lane0(tempty_c + so * 8, lane);
                scale_add32(acc + 48, vb, d1);
            }
            if (c->abort_flag) break;
            // 32 rows x 128 bytes at a time: 32 columns of binary32 or 64 of 16 bits
            constexpr int kStripCols = Y16 ? 64 : 32;
            __syncwarp();
#pragma unroll
            for (int piece = 0; piece < 128 / kStripCols; ++piece) {
                const int c0 = piece * kStripCols;
                const int64_t col0 = n0 + (c0 >> 6) * 128 + (c0 & 63);
                if (lane == 0) bulk_wait_group_read0();          // the strip has been read
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j) {                    // 16 bytes each
                    constexpr int kPer = Y16 ? 8 : 4;
                    float o[kPer];
#pragma unroll
                    for (int q = 0; q < kPer; q += 4) {
                        uint64_t b0, b1;
                        float bl, bh;
                        lds128(bias_s + (uint32_t)(c0 + j * kPer + q) * 4u, b0, b1);
                        unpack2(acc[(c0 + j * kPer + q) / 2], o[q], o[q + 1]);
                        unpack2(acc[(c0 + j * kPer + q) / 2 + 1], o[q + 2], o[q + 3]);
                        unpack2(b0, bl, bh);
                        o[q] += bl; o[q + 1] += bh;
                        unpack2(b1, bl, bh);
                        o[q + 2] += bl; o[q + 3] += bh;
                    }
                    const uint32_t at = strip_s + (uint32_t)lane * 128u + (((uint32_t)j ^ ((uint32_t)lane & 7u)) << 4);
                    if constexpr (Y16)
                        sts128(at, pack16(o[0], o[1], a.y_type == TDQ_F16), pack16(o[2], o[3], a.y_type == TDQ_F16),
                               pack16(o[4], o[5], a.y_type == TDQ_F16), pack16(o[6], o[7], a.y_type == TDQ_F16));
                    else
                        sts128(at, __float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3]));
                }
                if (a.y_vec) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // generic writes before the engine's reads
                    __syncwarp();
                    if (lane == 0) {
                        if (m0 < a.M && col0 < a.O) tma_store_2d(&ymap, strip_s, (int32_t)col0, (int32_t)m0);
                        bulk_commit_group();
                    }
                } else {                                         // rows off the 16-byte grid: element by element, a row at a time
                    __syncwarp();
#pragma unroll 1
                    for (int r = 0; r < 32 && m0 + r < a.M; ++r)
#pragma unroll 1
                        for (int q = lane; q < kStripCols && col0 + q < a.O; q += 32) {
                            const uint32_t b = (uint32_t)q * (Y16 ? 2u : 4u);
                            const uint32_t at = strip_s + (uint32_t)r * 128u + ((((b >> 4) ^ ((uint32_t)r & 7u)) << 4) | (b & 15u));
                            if constexpr (Y16) reinterpret_cast<uint16_t*>(a.y)[(m0 + r) * a.y_stride + col0 + q] = (uint16_t)lds16(at);
                            else reinterpret_cast<uint32_t*>(a.y)[(m0 + r) * a.y_stride + col0 + q] = lds32(at);
                        }
                    __syncwarp();
                }
            }
        }
        tmem_ld_wait();
        if (lane == 0) bulk_wait_group0();                       // no store may still be reading this CTA's shared memory at exit
    }

    tc_fence_before();
    __syncthreads();
    if (c->abort_flag) __nanosleep(1000000);                     // a wait gave up: give copies and tensor core a moment
    fp8_cluster_sync();                                          // neither CTA leaves while the other may still signal it
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(512) : "memory");
}

}  // namespace

tdq_status launch_fp8_pair(Fp8Args a, const CUtensorMap& xmap, const CUtensorMap& wmap, int n_sm, int dev, cudaStream_t stream) {
    const bool y16 = a.y_type != TDQ_F32;
    CUtensorMap ymap;
    memset(&ymap, 0, sizeof ymap);
    if (a.y_vec && !encode_y_map(&ymap, a.y, y16, a.M, a.O, a.y_stride, y16 ? 64 : 32, 32, a.y_type == TDQ_F16)) a.y_vec = 0;
    a.tiles_m = (int32_t)((a.M + 255) / 256);
    a.tiles_n = (int32_t)((a.O + 255) / 256);
    constexpr uint32_t fixed = kPairCtrl + 1024 + kAddWarps * (kStrip + kBiasBytes);
    a.n_stages = (kSmemLimit - (int)fixed) / (int)kPairStage;
    if (a.n_stages > kPairMaxStages) a.n_stages = kPairMaxStages;
    const uint32_t smem = fixed + (uint32_t)a.n_stages * kPairStage;
    static std::atomic<uint64_t> smem_done[2];
    void (*const kernels[2])(Fp8Args, CUtensorMap, CUtensorMap, CUtensorMap) = {fp8_pair_kernel<false>, fp8_pair_kernel<true>};
    if (allow_smem(kernels[y16], kSmemLimit, smem_done[y16], dev) != cudaSuccess) return TDQ_ERR_CUDA;
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    if (tiles > INT32_MAX / 2) return TDQ_ERR_UNSUPPORTED;
    const unsigned clusters = (unsigned)(tiles < n_sm / 2 ? tiles : n_sm / 2);
    if (launch_pdl(kernels[y16], dim3(2 * clusters), dim3(kPairThreads), smem, stream, a, xmap, wmap, ymap) != cudaSuccess) return TDQ_ERR_CUDA;
    g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return TDQ_OK;
}

}  // namespace tdq
