// tdq_fp8_linear for layers with many tiles: two CTAs of a cluster on a tile of 256 tokens x 256 (or 128) output channels.
//
// What bounds it.  A block of 128 channels is 512 clocks of tensor time per 256 x 256 tile; the 32 KB of operands that it uses in each
// CTA are written to shared memory meanwhile (64 bytes of the 128 a clock).  The sums of a block have scales of their own, so
// all 32768 of a CTA leave TMEM and are added to registers in the same time: 64 a clock of the 128 that the FMA pipe takes.  What must not
// happen is that tensor core and adders wait for each other: the tile's columns are two halves with two accumulators each (all 512
// TMEM columns), filled and drained in turn, so that three quarters of TMEM are in the tensor core's hands while one is read.  An accumulator's
// way there and back (commit, notice, 128 columns taken in two steps, arrival at CTA 0, issue) is what a block costs: 600 to 650 clocks.
// Measured: 16384 x 4096 -> 4096 bf16 224 us in a burst (2.45 PFLOP/s), 259 sustained, where the 1000 W limit holds the clock at 1.2 GHz (cuBLAS
// on the same codes without block scales, 208 and 214); tensor pipe 71 % busy.  18464 x 768 -> 2304 bf16 38 and 44 us (cuBLAS 38 and 41): a tile's
// six blocks are 3700 of 6400 clocks, the rest its epilogue.
// Not kept: one issuing warp (8 % slower); instructions of 256 columns and two accumulators (388 k clocks for 363 k); each half's sums taken by all eight
// warps, 64 columns each (393 k); landing registers reused from load to load, which the compiler copies (up to 96 moves a block); the next
// accumulator's first load ahead of this one's last additions (422 k).
//
// Where 256 x 256 tiles would leave SMs empty, tiles of 256 x 128 (TN = 128): every accumulator is the whole tile's, four blocks in turn, issued by the two
// warps alternately, so that token rows are read once a block (with halves of 64 columns they would be read twice, more than shared memory gives).
// 24 KB a block and CTA instead of 32, and half of the epilogue: 512 x 4096 -> 4096 bf16 16.6 -> 14.3 us, 512 x 768 -> 2304 6.9 -> 5.5, 1500 x 640 -> 300
// 7.4 -> 5.3, 9000 x 2816 -> 200 13.1 -> 11.4; several rounds lose (2048 x 4096 -> 4096 32.5, 45.5).  Bound by its loads, 45 to 50 bytes a clock.
//
//   warps 0, 3  loads of this CTA's 128 token rows and 128 weight rows (tensor maps, 128-byte swizzle, 16 KB each a stage), signalled to
//               CTA 0's barrier; warp 0 the block's scales too (asynchronous copies: as loads of the adding warps, first-level cache or not,
//               they cost a quarter of the kernel's time)
//   warps 1, 2  CTA 0: issue the instructions (cta_group::2, 256 x 128 x 32) of one half each (of every other block), commit to both CTAs' barriers
//   warps 4-11  scale and add: 32 token rows x 128 (64) columns each in registers (so 232 registers a thread, 40 for the others), then bias,
//               rounding and the store through two swizzled strips of 4 KB
//
// Half h is columns 64 h .. 64 h + 63 of each CTA's 128 weight rows: with cta_group::2 either CTA brings half of the columns.
#include <type_traits>

#include "tdq_tc.cuh"
#include "tdq_fp8.cuh"

namespace tdq {
namespace {

constexpr uint32_t kPairOperand = 128 * 128;             // bytes of a stage's token rows, and of its weight rows with TN = 256
constexpr uint32_t kPairCtrl = 1024;                     // the ring behind it is on the 1 KB grid that the swizzles need, as the block's shared memory is
constexpr int kAddWarp0 = 4, kAddWarps = 8;
constexpr int kPairThreads = (kAddWarp0 + kAddWarps) * 32;
constexpr uint32_t kStrip = 32 * 128;                    // 32 rows of 128 bytes
constexpr uint32_t kBiasBytes = 128 * 4;                 // of a warp's 128 columns
constexpr int kStrips = 2;                               // of a warp: 128 columns of 16 bits, so that no store is waited for in a tile
// Scales of a block: 128 token rows', then two weight blocks'.  No barrier hands their places back.  Block n's are copied once its stage is free: the
// instructions of block n - stages have completed, and those were issued after the sums that their accumulator held before had been taken, at most
// kReuse blocks further back (256: two, or one or three where a tile of an odd number of blocks ends in between; 128: four).  Sums are taken in order, so
// the scales of all blocks up to n - stages - kReuse have been read: as many places as stages + kReuse are enough.
constexpr uint32_t kScaleBytes = 128 * 4 + 16;
constexpr uint32_t kPairIdesc = (1u << 4) | ((128u >> 3) << 17) | ((256u >> 4) << 24);
constexpr int kRegsLoad = 40, kRegsAdd = 232;            // 128 * 40 + 256 * 232 <= 384 * 168

template <int TN> struct PairShape {                     // TN: the tile's columns
    static constexpr int kStages = TN == 256 ? 4 : 6;    // 256: five leave no room for the second strip and gain nothing
    static constexpr int kScaleSlots = TN == 256 ? 8 : 16;
    static constexpr int kReuse = TN == 256 ? 3 : 4;
    static_assert(kScaleSlots >= kStages + kReuse, "a block's scales would be overwritten before they are read");
    static constexpr uint32_t kWeights = TN / 2 * 128;
    static constexpr uint32_t kStage = kPairOperand + kWeights;
    static constexpr uint32_t kSmem = kPairCtrl + kStages * kStage + kAddWarps * (kStrips * kStrip + kBiasBytes) + kScaleSlots * kScaleBytes;
};
struct PairCtrl {
    uint64_t full[6];                                    // CTA 0: both CTAs' operands of the stage have landed
    uint64_t empty[6];
    uint64_t scales[16];                                 // a block's scales have landed in this CTA
    uint64_t tfull[4], tempty[4];                        // TN = 256: accumulator 2 (a tile's block & 1) + half; 128: a block's & 3 (tempty: CTA 0 only)
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
__device__ __forceinline__ void bulk_wait_group_read1() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
// 64 consecutive columns of this warp's 32 TMEM lanes, waited for: lane i receives row i.  The other adding warp of the scheduler works meanwhile.
__device__ __forceinline__ void tmem_ld64_wait(uint32_t taddr, uint32_t* v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
                 "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
                 "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
                 "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]),
                   "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]),
                   "=r"(v[40]), "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]),
                   "=r"(v[48]), "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]),
                   "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
                 : "r"(taddr)
                 : "memory");
}
// acc += d v, two columns an instruction.  The empty statement makes the compiler have the sums before it goes on to the next load: moved behind
// it, they need registers of their own for v.
__device__ __forceinline__ void scale_add64(float2* acc, const uint32_t* v, float d) {
#pragma unroll
    for (int j = 0; j < 32; ++j) acc[j] = __ffma2_rn(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), make_float2(d, d), acc[j]);
#pragma unroll
    for (int j = 0; j < 32; j += 8)
        asm volatile("" ::"f"(acc[j].x), "f"(acc[j + 1].x), "f"(acc[j + 2].x), "f"(acc[j + 3].x), "f"(acc[j + 4].x), "f"(acc[j + 5].x), "f"(acc[j + 6].x),
                     "f"(acc[j + 7].x));
}
// arrives on the barrier when this thread's copies so far have landed
__device__ __forceinline__ void copies_arrive(uint32_t bar_s) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_s) : "memory");
}

// DT: y's tdq_dtype.
template <int DT, int TN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
fp8_pair_kernel(const Fp8Args a, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap,
                const __grid_constant__ CUtensorMap ymap) {
    constexpr bool Y16 = DT != TDQ_F32;
    using Sh = PairShape<TN>;
    constexpr int kPairStages = Sh::kStages, kScaleSlots = Sh::kScaleSlots;
    constexpr uint32_t kPairStage = Sh::kStage;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Ctrl* c = reinterpret_cast<Ctrl*>(smem_raw);             // its abort flag and TMEM address; the barriers are g's
    PairCtrl* g = reinterpret_cast<PairCtrl*>(smem_raw + sizeof(Ctrl));
    static_assert(sizeof(Ctrl) + sizeof(PairCtrl) <= kPairCtrl, "control block outgrew its reservation");
    const uint32_t sm_s = smem_u32(smem_raw);
    const uint32_t ring_s = sm_s + kPairCtrl;                // the same offset in both CTAs
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t rank = fp8_cluster_rank();

    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) { mbar_init(&g->full[i], 2); mbar_init(&g->empty[i], TN == 256 ? 2 : 1); }
        for (int i = 0; i < kScaleSlots; ++i) mbar_init(&g->scales[i], 32);
        for (int i = 0; i < 4; ++i) { mbar_init(&g->tfull[i], 1); mbar_init(&g->tempty[i], TN == 256 ? kAddWarps : 2 * kAddWarps); }
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

    const uint32_t strips0_s = ring_s + kPairStages * kPairStage, biases_s = strips0_s + kAddWarps * kStrips * kStrip;
    const uint32_t scales_s = biases_s + kAddWarps * kBiasBytes;

    if (warp < kAddWarp0) {
        setmaxnreg_dec<kRegsLoad>();
        if (warp == 0 || warp == 3) {
            // -------------------------------------------------------- loads: tokens by warp 0, weights by warp 3
            const bool is_x = warp == 0;
            const uint32_t dst0 = ring_s + (is_x ? 0u : kPairOperand);
            const uint32_t full0 = map_to_cta(smem_u32(&g->full[0]), 0), empty_s = smem_u32(&g->empty[0]);
            uint32_t s = 0, ph = 1, n = 0;
            for (int tile = first; tile < n_tiles && !c->abort_flag; tile += n_clusters) {
                const int mt = tile / a.tiles_n, nt = tile - mt * a.tiles_n;
                const int row = is_x ? mt * 256 + (int)rank * 128 : nt * TN + (int)rank * (TN / 2);   // past the end: the map fills with zeros
                // scales: rows lane, lane + 32, .. of xscale and, in lanes 0 and 1, the tile's two rows of wscale; the last row for those past the end
                const float* xs[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) xs[i] = a.xscale + min((int64_t)row + lane + 32 * i, a.M - 1) * K;
                const float* ws = a.wscale + min(TN == 256 ? (int64_t)2 * nt + (lane & 1) : (int64_t)nt, (a.O - 1) >> 7) * K;
#pragma unroll 1
                for (int kb = 0; kb < K; ++kb, ++n) {
                    fp8_wait(empty_s + s * 8, ph, c, a.status, 5u);
                    if (c->abort_flag) break;
                    if (elect_one()) {
                        if (rank == 0) mbar_expect_tx(&g->full[s], is_x ? 2 * kPairOperand : 2 * Sh::kWeights);   // this operand, both CTAs
                        tma_load_pair(dst0 + s * kPairStage, is_x ? &xmap : &wmap, kb * (int)kFp8Block, row, full0 + s * 8);
                    }
                    __syncwarp();
                    if (is_x) {
                        const uint32_t at = scales_s + (n % kScaleSlots) * kScaleBytes + (uint32_t)lane * 4u;
#pragma unroll
                        for (int i = 0; i < 4; ++i) copy4_async(at + i * 128, xs[i] + kb);
                        if (lane < 2) copy4_async(at + 512, ws + kb);
                        copies_arrive(smem_u32(&g->scales[0]) + (n % kScaleSlots) * 8);
                    }
                    if (++s == kPairStages) { s = 0; ph ^= 1; }
                }
            }
        } else if (TN == 128 && rank == 0) {
            // -------------------------------------------------------- MMA issue, every other block
            const uint32_t full_s = smem_u32(&g->full[0]), empty_s = smem_u32(&g->empty[0]), tfull_s = smem_u32(&g->tfull[0]), tempty_s = smem_u32(&g->tempty[0]);
            const uint32_t xd0 = (uint32_t)sw_desc(ring_s), wd0 = (uint32_t)sw_desc(ring_s + kPairOperand);
            const int64_t total = first < n_tiles ? (int64_t)((n_tiles - first + n_clusters - 1) / n_clusters) * K : 0;
            uint32_t s = (uint32_t)warp - 1u, ph = 0;
            for (int64_t n = warp - 1; n < total; n += 2) {
                const uint32_t slot = (uint32_t)n & 3u;
                fp8_wait(full_s + s * 8, ph, c, a.status, 4u);
                fp8_wait(tempty_s + slot * 8, ((uint32_t)(n >> 2) & 1u) ^ 1u, c, a.status, 3u);
                if (c->abort_flag) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t xd = (uint64_t)kSwDescHi << 32 | (xd0 + s * (kPairStage >> 4)), wd = (uint64_t)kSwDescHi << 32 | (wd0 + s * (kPairStage >> 4));
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_f8_pair(tmem_base + slot * 128, xd + 2 * k, wd + 2 * k, k ? 1u : 0u);
                    commit_pair(tfull_s + slot * 8);
                    commit_pair(empty_s + s * 8);
                }
                __syncwarp();
                if ((s += 2) >= kPairStages) { s -= kPairStages; ph ^= 1; }
            }
        } else if (TN == 256 && rank == 0) {
            // -------------------------------------------------------- MMA issue, half h of every block
            const uint32_t h = (uint32_t)warp - 1u;
            const uint32_t full_s = smem_u32(&g->full[0]), empty_s = smem_u32(&g->empty[0]);
            const uint32_t tfull_s = smem_u32(&g->tfull[0]) + h * 8, tempty_s = smem_u32(&g->tempty[0]) + h * 8;
            const uint32_t xd0 = (uint32_t)sw_desc(ring_s), wd0 = (uint32_t)sw_desc(ring_s + kPairOperand) + h * (64 * 128 >> 4);
            const uint32_t d0 = tmem_base + h * 128;
            uint32_t s = 0, ph = 0, par[2] = {1, 1};
            bool landed = false;                                 // the stage's barrier, asked while the last block's instructions were issued
            const auto block = [&](const int slot) {
                if (!landed) fp8_wait(full_s + s * 8, ph, c, a.status, 4u);
                fp8_wait(tempty_s + slot * 16, par[slot], c, a.status, 3u);
                if (c->abort_flag) return false;
                par[slot] ^= 1u;
                const uint32_t now = s;
                if (++s == kPairStages) { s = 0; ph ^= 1; }
                landed = mbar_test_s(full_s + s * 8, ph);
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t xd = (uint64_t)kSwDescHi << 32 | (xd0 + now * (kPairStage >> 4)), wd = (uint64_t)kSwDescHi << 32 | (wd0 + now * (kPairStage >> 4));
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_f8_pair(d0 + slot * 256, xd + 2 * k, wd + 2 * k, k ? 1u : 0u);
                    commit_pair(tfull_s + slot * 16);
                    commit_pair(empty_s + now * 8);
                }
                __syncwarp();
                return true;
            };
            bool on = true;
            for (int tile = first; tile < n_tiles && on; tile += n_clusters) {
#pragma unroll 1
                for (int kb = 0; kb + 1 < K && on; kb += 2) on = block(0) && block(1);
                if ((K & 1) && on) on = block(0);
            }
        }
    } else {
        // ------------------------------------------------------------ scaled sums and epilogue
        setmaxnreg_inc<kRegsAdd>();
        const int aw = warp - kAddWarp0, quarter = warp & 3, h = aw >> 2;
        const uint32_t strips_s = strips0_s + (uint32_t)aw * (kStrips * kStrip), bias_s = biases_s + (uint32_t)aw * kBiasBytes;
        const uint32_t x_s = scales_s + (uint32_t)(quarter * 32 + lane) * 4u, sfull_s = smem_u32(&g->scales[0]);
        const uint32_t tfull_s = smem_u32(&g->tfull[TN == 256 ? h : 0]), tempty_c = map_to_cta(smem_u32(&g->tempty[TN == 256 ? h : 0]), 0);
        const uint32_t tm0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + h * (TN / 2);
        uint32_t par = 0, n = 0;                                 // phase bits of the half's two accumulators; blocks so far
        const bool ragged = a.O % (Y16 ? 8 : 4) != 0;
        bool full = false, scaled = false;                       // the next block's barriers, asked ahead of their use
        for (int tile = first; tile < n_tiles && !c->abort_flag; tile += n_clusters) {
            const int mt = tile / a.tiles_n, nt = tile - mt * a.tiles_n;
            const int64_t m0 = (int64_t)mt * 256 + rank * 128 + quarter * 32;
            const int64_t n0 = (int64_t)nt * TN + h * 64;        // columns n0 + 0..63 and, with TN = 256, n0 + 128 + 0..63
            __syncwarp();                                        // the last tile's biases have been read
#pragma unroll
            for (int i = 0; i < TN / 64; ++i) {
                const int64_t col = n0 + (i >> 1) * 128 + (i & 1) * 32 + lane;
                sts32(bias_s + (uint32_t)(i * 32 + lane) * 4u, a.bias && col < a.O ? __float_as_uint(__ldg(a.bias + col)) : 0u);
            }
            // the tensor core has run ahead during the last tile's epilogue
            full = TN == 256 ? mbar_test_s(tfull_s, par & 1u) : mbar_test_s(tfull_s + (n & 3u) * 8, (n >> 2) & 1u);
            scaled = mbar_test_s(sfull_s + n % kScaleSlots * 8, (n / kScaleSlots) & 1u);
            float2 acc[TN / 4];
#pragma unroll
            for (int j = 0; j < TN / 4; ++j) acc[j] = make_float2(0.f, 0.f);
            if constexpr (TN == 256) {
                const auto block = [&](const int slot, uint32_t then) {
                    const uint32_t at = n % kScaleSlots;
                    if (!full) fp8_wait_more(tfull_s + slot * 16, (par >> slot) & 1u, c, a.status, 2u);
                    if (!scaled) fp8_wait_more(sfull_s + at * 8, (n / kScaleSlots) & 1u, c, a.status, 6u);
                    __syncwarp();
                    par ^= 1u << slot;
                    ++n;
                    tc_fence_after();
                    const float x = __uint_as_float(lds32(x_s + at * kScaleBytes));
                    const float w0 = __uint_as_float(lds32(scales_s + at * kScaleBytes + 512)), w1 = __uint_as_float(lds32(scales_s + at * kScaleBytes + 516));
                    uint32_t v[64];
                    tmem_ld64_wait(tm0 + slot * 256, v);
                    scale_add64(acc, v, x * w0);
                    tmem_ld64_wait(tm0 + slot * 256 + 64, v);
                    tc_fence_before();
                    __syncwarp();
                    arrive_cluster_lane0(tempty_c + slot * 16, lane);
                    full = mbar_test_s(tfull_s + then * 16, (par >> then) & 1u);
                    scaled = mbar_test_s(sfull_s + n % kScaleSlots * 8, (n / kScaleSlots) & 1u);
                    scale_add64(acc + 32, v, x * w1);
                };
#pragma unroll 1
                for (int kb = 0; kb + 1 < K; kb += 2) {
                    block(0, 1u);
                    block(1, 0u);
                    if (c->abort_flag) break;
                }
                if (K & 1) block(0, 0u);
            } else {
#pragma unroll 1
                for (int kb = 0; kb < K && !c->abort_flag; ++kb) {   // 64 columns of the block's accumulator
                    const uint32_t slot = n & 3u, at = n % kScaleSlots;
                    if (!full) fp8_wait_more(tfull_s + slot * 8, (n >> 2) & 1u, c, a.status, 2u);
                    if (!scaled) fp8_wait_more(sfull_s + at * 8, (n / kScaleSlots) & 1u, c, a.status, 6u);
                    __syncwarp();
                    ++n;
                    tc_fence_after();
                    const float d = __uint_as_float(lds32(x_s + at * kScaleBytes)) * __uint_as_float(lds32(scales_s + at * kScaleBytes + 512));
                    uint32_t v[64];
                    tmem_ld64_wait(tm0 + slot * 128, v);
                    tc_fence_before();
                    __syncwarp();
                    arrive_cluster_lane0(tempty_c + slot * 8, lane);
                    full = mbar_test_s(tfull_s + (n & 3u) * 8, (n >> 2) & 1u);
                    scaled = mbar_test_s(sfull_s + n % kScaleSlots * 8, (n / kScaleSlots) & 1u);
                    scale_add64(acc, v, d);
                }
            }
            if (c->abort_flag) break;
            // 32 rows x 128 bytes at a time: 32 columns of binary32 or 64 of 16 bits
            constexpr int kStripCols = Y16 ? 64 : 32;
            __syncwarp();
#pragma unroll
            for (int piece = 0; piece < TN / 2 / kStripCols; ++piece) {
                const int c0 = piece * kStripCols;
                const int64_t col0 = n0 + (c0 >> 6) * 128 + (c0 & 63);
                const uint32_t strip_s = strips_s + (uint32_t)(piece & 1) * kStrip;
                if (lane == 0) {                                 // the strip has been read: the last tile's stores, then but the last one
                    if (piece == 0) bulk_wait_group_read0();
                    else if (piece > 1) bulk_wait_group_read1();
                }
                __syncwarp();
                // biases first, all of them: behind a store to the strip every load of them waited out its latency
                float4 b[kStripCols / 4];
#pragma unroll
                for (int j = 0; j < kStripCols / 4; ++j) b[j] = lds_f4(bias_s + (uint32_t)(c0 + 4 * j) * 4u);
#pragma unroll
                for (int j = 0; j < 8; ++j) {                    // 16 bytes each
                    constexpr int kPer = Y16 ? 8 : 4;
                    float o[kPer];
#pragma unroll
                    for (int q = 0; q < kPer; q += 4) {
                        const float4 t = b[(j * kPer + q) / 4];
                        const float2 r0 = __fadd2_rn(acc[(c0 + j * kPer + q) / 2], make_float2(t.x, t.y));
                        const float2 r1 = __fadd2_rn(acc[(c0 + j * kPer + q) / 2 + 1], make_float2(t.z, t.w));
                        o[q] = r0.x; o[q + 1] = r0.y; o[q + 2] = r1.x; o[q + 3] = r1.y;
                    }
                    const uint32_t at = strip_s + (uint32_t)lane * 128u + (((uint32_t)j ^ ((uint32_t)lane & 7u)) << 4);
                    if constexpr (Y16)
                        sts128(at, pack16(o[0], o[1], DT == TDQ_F16), pack16(o[2], o[3], DT == TDQ_F16),
                               pack16(o[4], o[5], DT == TDQ_F16), pack16(o[6], o[7], DT == TDQ_F16));
                    else
                        sts128(at, __float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3]));
                }
                // the engine writes 16 bytes at a time: a last piece of columns that ends within them is stored by element
                if (a.y_vec && (!ragged || col0 + kStripCols <= a.O)) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // generic writes before the engine's reads
                    __syncwarp();
                    if (lane == 0) {
                        if (m0 < a.M && col0 < a.O) tma_store_2d(&ymap, strip_s, (int32_t)col0, (int32_t)m0);
                        bulk_commit_group();
                    }
                } else {
                    // Rows off the 16-byte grid: element by element, lanes along a row, eight rows in flight (one at a time 1717 x 1464 -> 4862 bf16
                    // took 33.5 us, 477 x 4009 -> 2809 fp32 23.6; now 18.2 and 18.1, on the grid 15.7 and 16.6).
                    using U = std::conditional_t<Y16, uint16_t, uint32_t>;
                    constexpr int kAcross = kStripCols / 32;
                    __syncwarp();
                    U* y = reinterpret_cast<U*>(a.y) + m0 * a.y_stride + col0 + lane;
                    const int rows = (int)max((int64_t)0, min((int64_t)32, a.M - m0));
                    const int64_t cols = a.O - col0 - lane;
#pragma unroll 1
                    for (int r0 = 0; r0 < rows; r0 += 8) {
                        U v[8][kAcross];
#pragma unroll
                        for (int r = 0; r < 8; ++r)
#pragma unroll
                            for (int q = 0; q < kAcross; ++q) {
                                const uint32_t b = (uint32_t)(lane + 32 * q) * (uint32_t)sizeof(U);
                                const uint32_t at = strip_s + (uint32_t)(r0 + r) * 128u + ((((b >> 4) ^ (uint32_t)r) << 4) | (b & 15u));
                                if constexpr (Y16) v[r][q] = (uint16_t)lds16(at);
                                else v[r][q] = lds32(at);
                            }
#pragma unroll
                        for (int r = 0; r < 8; ++r)
#pragma unroll
                            for (int q = 0; q < kAcross; ++q)
                                if (r0 + r < rows && 32 * q < cols) y[r * a.y_stride + 32 * q] = v[r][q];
                        y += 8 * a.y_stride;
                    }
                    if (lane == 0) bulk_commit_group();          // an empty one: a strip's turn is counted in groups
                    __syncwarp();
                }
            }
        }
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

tdq_status launch_fp8_pair(Fp8Args a, int columns, const CUtensorMap& xmap, const CUtensorMap& wmap, int n_sm, int dev, cudaStream_t stream) {
    const bool y16 = a.y_type != TDQ_F32, f16 = a.y_type == TDQ_F16;
    CUtensorMap ymap;
    memset(&ymap, 0, sizeof ymap);
    if (a.y_vec && !encode_y_map(&ymap, a.y, y16, a.M, a.O, a.y_stride, y16 ? 64 : 32, 32, f16)) a.y_vec = 0;
    a.tiles_m = (int32_t)((a.M + 255) / 256);
    a.tiles_n = (int32_t)((a.O + columns - 1) / columns);
    static_assert(PairShape<256>::kSmem <= (uint32_t)kSmemLimit && PairShape<128>::kSmem <= (uint32_t)kSmemLimit, "shared memory");
    static std::atomic<uint64_t> smem_done[2][3];
    void (*const kernels[2][3])(Fp8Args, CUtensorMap, CUtensorMap, CUtensorMap) = {
        {fp8_pair_kernel<TDQ_F32, 256>, fp8_pair_kernel<TDQ_BF16, 256>, fp8_pair_kernel<TDQ_F16, 256>},
        {fp8_pair_kernel<TDQ_F32, 128>, fp8_pair_kernel<TDQ_BF16, 128>, fp8_pair_kernel<TDQ_F16, 128>}};
    const int narrow = columns == 128;
    const uint32_t smem = narrow ? PairShape<128>::kSmem : PairShape<256>::kSmem;
    if (allow_smem(kernels[narrow][a.y_type], (int)smem, smem_done[narrow][a.y_type], dev) != cudaSuccess) return TDQ_ERR_CUDA;
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    if (tiles > INT32_MAX / 2) return TDQ_ERR_UNSUPPORTED;
    const unsigned clusters = (unsigned)(tiles < n_sm / 2 ? tiles : n_sm / 2);
    if (launch_pdl(kernels[narrow][a.y_type], dim3(2 * clusters), dim3(kPairThreads), smem, stream, a, xmap, wmap, ymap) != cudaSuccess) return TDQ_ERR_CUDA;
    g_launch_count.fetch_add(1, std::memory_order_relaxed);
    return TDQ_OK;
}

}  // namespace tdq
