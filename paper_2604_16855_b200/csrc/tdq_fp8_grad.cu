// tdq_fp8_weight_grad: dw[o,i] = sum_m dy[m,o] x[m,i], db[o] = sum_m dy[m,o], with x = code x scale kept in 8 bits.
//
// The scale of x changes along the sum (a token's block of 128 channels has its own), so it cannot be taken out of the product: the codes are restored to
// bf16 on their way to the tensor core, which with scales that are powers of two is exact.  The restored matrix is never in memory.
//
//   tile        256 outputs x 256 input channels by two CTAs (cta_group::2): each brings 128 outputs of dy (copied by the engine as they lie in memory,
//               64 tokens x 64 outputs a box, an operand whose slow axis is the sum's) and one block of 128 channels, written in the same layout by the
//               restoring warps.  64 tokens a stage: 16 KB of each.
//   sum         binary32 accumulators in TMEM (two of 256 columns), taken to binary32 registers every kGroup stages: the tensor core drops what it adds below
//               the accumulator's last place (32768 tokens in one: off by 5.3e-7 of the result, of a float32 dy 2.5e-6; so 1.6e-7 and 1.9e-7, like a product in binary32).
//   work        whole tiles, or all stages of all tiles in one row, cut in pieces for the pairs of SMs; a tile that is cut goes to the workspace in parts, which a second kernel
//               adds in order (several vectors a thread there: no gain).  No atomics: the same call gives the same bits.
//   dy          bf16 on the 16-byte grid is read in place; fp16 and float32 are cut into two and three bf16 addends (exact) and rows off the grid copied,
//               into the workspace, and the sum goes over all addends.
//
//   warps 0, 1  copies of dy; the instructions (CTA 0)      warp 3  copies of codes      warps 4-11  sums and output      warps 12-19  restore x, sum db
//
// Bound by the restoring warps' chain (codes, conversion, shared memory, notice: 580 clocks a stage, the tensor core's share 512) and by power: 16384 tokens, 1024 -> 4096 bf16
// 122 us from a graph at 1.6 GHz (the library's product of the restored matrices, which then are in memory, 94 to 107).  Little work goes to another kernel
// (tdq_fp8_grad_small.cu).  Not kept: arrivals that release at cluster scope (5000 clocks a stage), loads of codes and scales by the restoring warps themselves (150 us for 139 with all
// else the same), a longer stay in the accumulator (3 % faster).
#include <algorithm>
#include <numeric>

#include "tdq_tc.cuh"
#include "tdq_fp8_grad.cuh"

namespace tdq {
namespace {

constexpr int kTok = 64;                                  // tokens a stage
constexpr int kGradStages = 5;
constexpr int kGroup = 8;                                 // stages whose products an accumulator adds
constexpr uint32_t kGradOperand = kTok * 128 * 2;         // bytes: two halves of 64 columns, 128 bytes a token
constexpr uint32_t kGradHalf = kTok * 128;
constexpr uint32_t kGradStage = 2 * kGradOperand;
constexpr uint32_t kGradCtrl = 1024;
constexpr uint32_t kGradStrip = 32 * 128;
constexpr int kSumWarp0 = 4, kSumWarps = 8, kFillWarp0 = 12, kFillWarps = 8;
constexpr int kGradThreads = (kFillWarp0 + kFillWarps) * 32;
constexpr int kFillPairs = kFillWarps / 2;               // two warps fill a stage, every fourth one
constexpr uint32_t kGradCodes = kTok * 128;                // bytes of a stage's codes
constexpr uint32_t kGradSmem = kGradCtrl + kGradStages * kGradStage + kFillPairs * kGradCodes + kSumWarps * kGradStrip;
static_assert(kGradSmem <= (uint32_t)kSmemLimit, "shared memory");
constexpr int kGradRegsLoad = 32, kGradRegsSum = 160, kGradRegsFill = 64;   // 128 * 32 + 256 * 160 + 256 * 64 <= 640 * 96
// D binary32, both operands bf16 with the sum's axis slow, 256 columns x 256 rows
constexpr uint32_t kGradIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
constexpr uint32_t kGradDescLo = (kGradHalf >> 4) << 16;  // the next 64 columns; eight tokens further on are 1024 bytes (kSwDescHi)

// The row of all tiles' stages, in `clusters` pieces of whole units (of a stage, or of a tile's stages where tiles are not cut).
struct Cut {
    int32_t units, unit, clusters;
    // the first stage that cluster w adds
    __host__ __device__ int32_t begin(int32_t w) const { return unit * (units / clusters * w + min(w, units % clusters)); }
    // the cluster that adds stage s
    __host__ __device__ int32_t owner(int32_t s) const {
        const int32_t u = s / unit, q = units / clusters, r = units % clusters, longer = r * (q + 1);
        return u < longer ? u / (q + 1) : r + (u - longer) / q;
    }
};
struct GradArgs {
    const uint8_t* xcodes;     // [M][Kb * 128]
    const float* xscale;       // [M][Kb]
    const uint16_t* dy;        // bf16 [parts * rows_part][dy_stride]
    void* dw;
    float* db;                 // or null
    float* dbpart;             // [2 clusters + tiles][pairs of warps][256]: cut tiles' parts, whole tiles'
    float4* part;              // [2 clusters][2 CTAs][8 warps][32 quads of columns][32 rows]
    int64_t M, O, I, dy_stride, dw_stride, rows_part;
    int32_t Kb, tiles_o, tiles_i, stages_part, parts;   // stages of an addend, addends
    Cut cut;
    int32_t dw_vec;            // rows of dw on the 16-byte grid
    uint32_t* status;
};
struct GradCtrl {
    uint64_t landed[kGradStages];                            // this CTA's dy
    uint64_t full[kGradStages];                              // CTA 0: both CTAs' operands
    uint64_t empty[kGradStages];
    uint64_t codes[kFillPairs], taken[kFillPairs];            // a pair's codes have landed; have been read
    uint64_t tfull[2], tempty[2];
};
static_assert(sizeof(Ctrl) + sizeof(GradCtrl) <= kGradCtrl, "control block outgrew its reservation");

// A cluster's stages, tile by tile, in the order in which it adds them: the tile at its end first, which begins with the first tokens, then the rest, which begins in the
// middle of a tile.  So all clusters go through the tokens at about the same time, and what several tiles read is read from memory once (from the piece's
// begin on instead: 16384 tokens, 1024 -> 4096 bf16 135 us for 122, 2048 -> 4096 264 for 235).
struct Piece {
    int32_t per_tile, begin, end, last;                      // last: where its last tile's stages begin, if it has more than one tile; else its end
    __device__ Piece(int32_t per_tile_, const Cut& cut, int32_t w) : per_tile(per_tile_), begin(cut.begin(w)), end(cut.begin(w + 1)) {
        const int32_t t = (end - 1) / per_tile * per_tile;
        last = t > begin ? t : end;
    }
    __device__ int32_t stages() const { return end - begin; }
    // the k-th stage that is added
    __device__ int32_t stage(int32_t k) const { return k < end - last ? last + k : begin + k - (end - last); }
};
// the stages of one tile: k .. k + len - 1 of the piece's order, from stage `at` of the tile on
struct Stretch {
    int32_t tile, at, len;
    int32_t to, ti;                                          // the tile's outputs and channels, in tiles
    bool whole;
    int32_t slot;                                            // of the cluster's two places for parts
    __device__ Stretch(const Piece& p, int32_t k, int32_t tiles_i) {
        const int32_t s = p.stage(k);
        tile = s / p.per_tile;
        at = s - tile * p.per_tile;
        to = tile / tiles_i;
        ti = tile - to * tiles_i;
        len = min(p.per_tile - at, (k < p.end - p.last ? p.end : p.last) - s);
        whole = len == p.per_tile;
        slot = s == p.begin ? 0 : 1;
    }
};

__device__ __forceinline__ void grad_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void grad_mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(kGradIdesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void grad_commit(uint32_t bar_s) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar_s), "h"((uint16_t)3) : "memory");
}
// Lane 0 of a converged warp arrives on a barrier of either CTA, given by its cluster address.  Not with release at cluster scope, which waits for all
// that the thread has in flight (5000 clocks a stage instead of 700): what a restoring warp wrote is in its own CTA's shared memory, ordered by the proxy fence.
__device__ __forceinline__ void grad_arrive(uint32_t bar_c, int lane) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}"
                 ::"r"(bar_c), "r"(lane) : "memory");
}
// sixteen consecutive columns of this warp's 32 TMEM lanes, waited for: lane i receives row i
__device__ __forceinline__ void tmem_ld16_wait(uint32_t taddr, uint32_t* v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
                 "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr)
                 : "memory");
}
// DT: dw's tdq_dtype
template <int DT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGradThreads, 1)
fp8_grad_kernel(const GradArgs a, const __grid_constant__ CUtensorMap dymap, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap dwmap) {
    constexpr bool W16 = DT != TDQ_F32;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Ctrl* c = reinterpret_cast<Ctrl*>(smem_raw);             // its abort flag and TMEM address; the barriers are g's
    GradCtrl* g = reinterpret_cast<GradCtrl*>(smem_raw + sizeof(Ctrl));
    const uint32_t sm_s = smem_u32(smem_raw), ring_s = sm_s + kGradCtrl;
    const uint32_t codes_s = ring_s + kGradStages * kGradStage, strips_s = codes_s + kFillPairs * kGradCodes;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t rank = fp8_cluster_rank();
    // Where this cluster's work lies: a dozen quotients, ahead of the wait for the kernel before (behind it they took 2000 clocks to the first copy).
    const int32_t w = (int32_t)blockIdx.x / 2, per_tile = a.stages_part * a.parts;
    const Piece piece(per_tile, a.cut, w);
    const int32_t n_stages = piece.stages();
    const Stretch first(piece, 0, a.tiles_i);

    if (threadIdx.x == 0) {
        for (int i = 0; i < kGradStages; ++i) { mbar_init(&g->landed[i], 1); mbar_init(&g->full[i], 4); mbar_init(&g->empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&g->tfull[i], 1); mbar_init(&g->tempty[i], 2 * kSumWarps); }
        for (int i = 0; i < kFillPairs; ++i) { mbar_init(&g->codes[i], 1); mbar_init(&g->taken[i], 2); }
        c->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&dymap)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&xmap)) : "memory");
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

    if (warp < kSumWarp0) {
        setmaxnreg_dec<kGradRegsLoad>();
        if (warp == 0) {
            // -------------------------------------------------------- copies of dy
            const uint32_t landed_s = smem_u32(&g->landed[0]), empty_s = smem_u32(&g->empty[0]);
            uint32_t s = 0, ph = 1;
            for (int32_t k = 0; k < n_stages && !c->abort_flag;) {
                const Stretch t = k ? Stretch(piece, k, a.tiles_i) : first;
                const int32_t o = t.to * 256 + (int32_t)rank * 128;   // past the end: the map fills with zeros
                int32_t part = t.at / a.stages_part, tok = t.at - part * a.stages_part;
#pragma unroll 1
                for (int32_t i = 0; i < t.len; ++i) {
                    fp8_wait(empty_s + s * 8, ph, c, a.status, 5u);
                    if (c->abort_flag) break;
                    if (elect_one()) {
                        mbar_expect_tx(&g->landed[s], kGradOperand);
                        const int32_t row = (int32_t)(part * a.rows_part) + tok * kTok;
                        grad_load(ring_s + s * kGradStage, &dymap, o, row, landed_s + s * 8);
                        grad_load(ring_s + s * kGradStage + kGradHalf, &dymap, o + 64, row, landed_s + s * 8);
                    }
                    __syncwarp();
                    if (++s == kGradStages) { s = 0; ph ^= 1; }
                    if (++tok == a.stages_part) { tok = 0; ++part; }
                }
                k += t.len;
            }
            // the last stages' commits reach this CTA too: waited for, so that none is under way when it leaves
#pragma unroll 1
            for (int i = 0; i < kGradStages; ++i) {
                fp8_wait(empty_s + s * 8, ph, c, a.status, 5u);
                if (++s == kGradStages) { s = 0; ph ^= 1; }
            }
        } else if (warp == 3) {
            // -------------------------------------------------------- copies of codes, a slot for each pair of restoring warps
            const uint32_t codes_bar = smem_u32(&g->codes[0]), taken_s = smem_u32(&g->taken[0]);
            for (int32_t k = 0; k < n_stages && !c->abort_flag;) {
                const Stretch t = k ? Stretch(piece, k, a.tiles_i) : first;
                const int32_t x = (2 * t.ti + (int32_t)rank) * 128;   // past the end: the map fills with zeros
                int32_t tok = t.at % a.stages_part;
#pragma unroll 1
                for (const int32_t end = k + t.len; k < end; ++k) {
                    const uint32_t slot = (uint32_t)k % kFillPairs;
                    fp8_wait(taken_s + slot * 8, ((uint32_t)(k / kFillPairs) & 1u) ^ 1u, c, a.status, 9u);
                    if (c->abort_flag) break;
                    if (elect_one()) {
                        mbar_expect_tx(&g->codes[slot], kGradCodes);
                        grad_load(codes_s + slot * kGradCodes, &xmap, x, tok * kTok, codes_bar + slot * 8);
                    }
                    __syncwarp();
                    if (++tok == a.stages_part) tok = 0;
                }
            }
        } else if (warp == 1 && rank == 0) {
            // -------------------------------------------------------- instructions
            const uint32_t full_s = smem_u32(&g->full[0]), empty_s = smem_u32(&g->empty[0]), tfull_s = smem_u32(&g->tfull[0]), tempty_s = smem_u32(&g->tempty[0]);
            const uint32_t xd0 = kGradDescLo | ((ring_s & 0x3FFFFu) >> 4);
            uint32_t s = 0, ph = 0, group = 0;
            bool on = true;
            for (int32_t k = 0; k < n_stages && on;) {
                const Stretch t = k ? Stretch(piece, k, a.tiles_i) : first;
                for (int32_t i = 0; i < t.len && on; ++group) {
                    const int32_t len = min(kGroup, t.len - i);
                    const uint32_t slot = group & 1u;
                    fp8_wait(tempty_s + slot * 8, ((group >> 1) & 1u) ^ 1u, c, a.status, 3u);
#pragma unroll 1
                    for (int32_t j = 0; j < len; ++j) {
                        fp8_wait(full_s + s * 8, ph, c, a.status, 4u);
                        if (c->abort_flag) { on = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t lo = xd0 + s * (kGradStage >> 4);
                            const uint64_t ad = (uint64_t)kSwDescHi << 32 | lo, bd = (uint64_t)kSwDescHi << 32 | (lo + (kGradOperand >> 4));
#pragma unroll
                            for (int q = 0; q < kTok / 16; ++q) grad_mma(tmem_base + slot * 256, ad + q * (2048 >> 4), bd + q * (2048 >> 4), j || q ? 1u : 0u);
                            grad_commit(empty_s + s * 8);
                            if (j == len - 1) grad_commit(tfull_s + slot * 8);
                        }
                        __syncwarp();
                        if (++s == kGradStages) { s = 0; ph ^= 1; }
                    }
                    i += len;
                }
                k += t.len;
            }
            // and so do the other CTA's arrivals, of the last two accumulators' readers
#pragma unroll 1
            for (int i = 0; i < 2; ++i, ++group) fp8_wait(tempty_s + (group & 1u) * 8, ((group >> 1) & 1u) ^ 1u, c, a.status, 3u);
        }
    } else if (warp < kFillWarp0) {
        // ------------------------------------------------------------ sums and output
        setmaxnreg_inc<kGradRegsSum>();
        const int sw = warp - kSumWarp0, quarter = warp & 3, h = sw >> 2;
        const uint32_t strip_s = strips_s + (uint32_t)sw * kGradStrip;
        const uint32_t tfull_s = smem_u32(&g->tfull[0]), tempty_c = map_to_cta(smem_u32(&g->tempty[0]), 0);
        const uint32_t tm0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + h * 128;
        uint32_t group = 0;
        for (int32_t k = 0; k < n_stages && !c->abort_flag;) {
            const Stretch stretch = k ? Stretch(piece, k, a.tiles_i) : first;
            float2 acc[64];
#pragma unroll
            for (int j = 0; j < 64; ++j) acc[j] = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int32_t done = 0; done < stretch.len; done += kGroup, ++group) {
                const uint32_t slot = group & 1u;
                fp8_wait(tfull_s + slot * 8, (group >> 1) & 1u, c, a.status, 2u);
                if (c->abort_flag) break;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    uint32_t v[16];
                    tmem_ld16_wait(tm0 + slot * 256 + q * 16, v);
                    if (q == 7) {
                        tc_fence_before();
                        __syncwarp();
                        grad_arrive(tempty_c + slot * 8, lane);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        acc[q * 8 + j] = __fadd2_rn(acc[q * 8 + j], make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
                }
            }
            if (c->abort_flag) break;
            const int to = stretch.to, ti = stretch.ti;
            const bool whole = stretch.whole;
            const int32_t slot = 2 * w + stretch.slot;
            const int64_t o0 = (int64_t)to * 256 + rank * 128 + quarter * 32, i0 = (int64_t)ti * 256 + h * 128;
            if (!whole) {
                // a part, as it lies in the registers: 512 bytes an instruction
                float4* dst = a.part + ((((int64_t)slot * 2 + rank) * kSumWarps + sw) * 32) * 32 + lane;
#pragma unroll
                for (int j = 0; j < 32; ++j) dst[j * 32] = make_float4(acc[2 * j].x, acc[2 * j].y, acc[2 * j + 1].x, acc[2 * j + 1].y);
            } else if (!W16) {
#pragma unroll
                for (int piece = 0; piece < 4; ++piece) {
                    if (lane == 0) bulk_wait_group_read0();          // the strip has been read
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float2 u = acc[piece * 16 + 2 * j], v = acc[piece * 16 + 2 * j + 1];
                        sts128(strip_s + (uint32_t)lane * 128u + (((uint32_t)j ^ ((uint32_t)lane & 7u)) << 4), __float_as_uint(u.x), __float_as_uint(u.y),
                               __float_as_uint(v.x), __float_as_uint(v.y));
                    }
                    const int64_t col = i0 + piece * 32;
                    if (a.dw_vec && (a.I % 4 == 0 || col + 32 <= a.I)) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            if (o0 < a.O && col < a.I) tma_store_2d(&dwmap, strip_s, (int32_t)col, (int32_t)o0);
                            bulk_commit_group();
                        }
                    } else {
                        __syncwarp();
                        float* dw = reinterpret_cast<float*>(a.dw) + o0 * a.dw_stride + col + lane;
                        const int rows = (int)max((int64_t)0, min((int64_t)32, a.O - o0));
                        if (col + lane < a.I)
#pragma unroll 8
                            for (int r = 0; r < rows; ++r)
                                dw[r * a.dw_stride] = __uint_as_float(lds32(strip_s + (uint32_t)r * 128u + ((((uint32_t)lane >> 2) ^ ((uint32_t)r & 7u)) << 4) + ((uint32_t)lane & 3u) * 4u));
                        __syncwarp();
                    }
                }
            } else {
                if constexpr (W16) {
#pragma unroll
                    for (int piece = 0; piece < 2; ++piece) {
                        if (lane == 0) bulk_wait_group_read0();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float2* u = acc + piece * 32 + 4 * j;
                            sts128(strip_s + (uint32_t)lane * 128u + (((uint32_t)j ^ ((uint32_t)lane & 7u)) << 4), narrow2<DT>(u[0].x, u[0].y), narrow2<DT>(u[1].x, u[1].y),
                                   narrow2<DT>(u[2].x, u[2].y), narrow2<DT>(u[3].x, u[3].y));
                        }
                        const int64_t col = i0 + piece * 64;
                        if (a.dw_vec && (a.I % 8 == 0 || col + 64 <= a.I)) {
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                            __syncwarp();
                            if (lane == 0) {
                                if (o0 < a.O && col < a.I) tma_store_2d(&dwmap, strip_s, (int32_t)col, (int32_t)o0);
                                bulk_commit_group();
                            }
                        } else {
                            __syncwarp();
                            uint16_t* dw = reinterpret_cast<uint16_t*>(a.dw) + o0 * a.dw_stride + col + lane;
                            const int rows = (int)max((int64_t)0, min((int64_t)32, a.O - o0));
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const uint32_t b = (uint32_t)(lane + 32 * q) * 2u;
                                if (col + lane + 32 * q < a.I)
#pragma unroll 8
                                    for (int r = 0; r < rows; ++r)
                                        dw[r * a.dw_stride + 32 * q] = (uint16_t)lds16(strip_s + (uint32_t)r * 128u + (((b >> 4) ^ ((uint32_t)r & 7u)) << 4) + (b & 15u));
                            }
                            __syncwarp();
                        }
                    }
                }
            }
            k += stretch.len;
        }
        if (lane == 0) bulk_wait_group0();                   // no store may still be reading this CTA's shared memory at exit
    } else {
        // ------------------------------------------------------------ restored operand, sums of dy
        setmaxnreg_dec<kGradRegsFill>();
        const int fw = warp - kFillWarp0, pair = fw >> 1, side = fw & 1;   // a warp restores 32 tokens and sums 64 outputs of every fourth stage
        const uint32_t full0 = map_to_cta(smem_u32(&g->full[0]), 0), empty_s = smem_u32(&g->empty[0]), landed_s = smem_u32(&g->landed[0]);
        const uint32_t codes_bar = smem_u32(&g->codes[pair]), taken_bar = smem_u32(&g->taken[pair]);
        // Sixteen codes a lane and token, channels 16 (lane & 7) ..: of token 4 q + lane / 8, the upper 64 channels of its neighbour, so that eight lanes
        // read, and write, eight different 16-byte columns (the swizzle moves a row's by its number: odd and even rows never meet).
        const uint32_t ch = (uint32_t)lane & 7u, half = ch >> 2, tok0 = ((uint32_t)lane >> 3) ^ half;
        const uint32_t from_s = codes_s + (uint32_t)pair * kGradCodes + ((uint32_t)side * 32u + tok0) * 128u;
        const uint32_t to_s = ring_s + kGradOperand + half * kGradHalf + ((uint32_t)side * 32u + tok0) * 128u;
        uint32_t from[2], to[2][2];                          // of even and odd q
#pragma unroll
        for (uint32_t q = 0; q < 2; ++q) {
            from[q] = from_s + ((ch ^ (tok0 + 4u * q)) << 4);
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) to[q][j] = to_s + (((2u * (ch & 3u) + j) ^ (tok0 + 4u * q)) << 4);
        }
        float scale;                                         // of token side * 32 + lane of the next stage; 0 where there is none
        const auto scale_at = [&](int32_t block, int32_t tok) {
            const int64_t m = (int64_t)tok * kTok + side * 32 + lane;
            return block < a.Kb && m < a.M ? __ldg(a.xscale + m * a.Kb + block) : 0.f;
        };
        const auto scale_of = [&](int32_t k) {               // of any stage
            if (k >= n_stages) return 0.f;
            const int32_t st = piece.stage(k), tile = st / per_tile;
            return scale_at(2 * (tile % a.tiles_i) + (int32_t)rank, (st - tile * per_tile) % a.stages_part);
        };
        int32_t mine = pair;                                 // this warp's stage, in the piece's order
        uint32_t s = (uint32_t)pair, ph = 0;                 // its place in the ring
        uint32_t cph = 0;
        scale = scale_of(mine);
        for (int32_t k = 0; k < n_stages && !c->abort_flag;) {
            const Stretch t = k ? Stretch(piece, k, a.tiles_i) : first;
            // the tiles of the same outputs take turns at the column sums
            int32_t turn = a.db ? (t.at + mine - k) % a.tiles_i : -1, tok = (t.at + mine - k) % a.stages_part;   // of this warp's stage
            const int32_t block = 2 * t.ti + (int32_t)rank;
            float2 sum[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = make_float2(0.f, 0.f);
#pragma unroll 1
            for (; mine < k + t.len; mine += kFillPairs) {
                const float now = scale;
                tok += kFillPairs;
                while (tok >= a.stages_part) tok -= a.stages_part;
                scale = mine + kFillPairs < k + t.len ? scale_at(block, tok) : scale_of(mine + kFillPairs);
                fp8_wait(codes_bar, cph, c, a.status, 10u);
                cph ^= 1u;
                uint4 code[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) code[q] = lds_u4(from[q & 1] + q * 512u);
                __syncwarp();
                mbar_arrive_lane0_s(taken_bar, lane);
                fp8_wait(empty_s + s * 8, ph ^ 1u, c, a.status, 6u);
                if (c->abort_flag) break;
                const uint32_t d = s * kGradStage;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float f = __shfl_sync(0xffffffffu, now, 4 * q + (int)tok0);
                    uint32_t r[8];
                    restore4(code[q].x, f, r[0], r[1]);
                    restore4(code[q].y, f, r[2], r[3]);
                    restore4(code[q].z, f, r[4], r[5]);
                    restore4(code[q].w, f, r[6], r[7]);
                    sts128(to[q & 1][0] + d + q * 512u, r[0], r[1], r[2], r[3]);
                    sts128(to[q & 1][1] + d + q * 512u, r[4], r[5], r[6], r[7]);
                }
                fp8_wait(landed_s + s * 8, ph, c, a.status, 8u);
                if (c->abort_flag) break;
                if (turn == t.ti) {                          // 8 outputs x 16 tokens a lane; rows behind dy's end are zero
                    const uint32_t at = ring_s + d + (uint32_t)side * kGradHalf + ((uint32_t)lane >> 3) * 128u;
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        const uint4 u = lds_u4(at + q * 512u + ((ch ^ (((uint32_t)lane >> 3) + 4u * (q & 1))) << 4));
                        const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            sum[j] = __fadd2_rn(sum[j], make_float2(__uint_as_float(v[j] << 16), __uint_as_float(v[j] & 0xffff0000u)));
                    }
                }
                if (a.db) {
                    turn += kFillPairs;
                    while (turn >= a.tiles_i) turn -= a.tiles_i;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                grad_arrive(full0 + s * 8, lane);
                s += kFillPairs;
                if (s >= kGradStages) { s -= kGradStages; ph ^= 1u; }
            }
            if (c->abort_flag) break;
            if (a.db) {                                      // this stretch's column sums, this warp's
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int x = 8; x <= 16; x <<= 1)
                        sum[j] = __fadd2_rn(sum[j], make_float2(__shfl_xor_sync(0xffffffffu, sum[j].x, x), __shfl_xor_sync(0xffffffffu, sum[j].y, x)));
                if (lane < 8) {
                    float* to = a.dbpart + ((int64_t)(t.whole ? 2 * a.cut.clusters + t.tile : 2 * w + t.slot) * kFillPairs + pair) * 256 + rank * 128 + side * 64 + 8 * lane;
#pragma unroll
                    for (int j = 0; j < 4; j += 2) *reinterpret_cast<float4*>(to + 2 * j) = make_float4(sum[j].x, sum[j].y, sum[j + 1].x, sum[j + 1].y);
                }
            }
            k += t.len;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (c->abort_flag) __nanosleep(1000000);                 // a wait gave up: give copies and tensor core a moment
    // Neither CTA leaves while the tensor core may still read its operands; signals from the other have been waited for, each by one of the warps above.  Relaxed: an arrival
    // that releases waits for the thread's stores to memory (1400 clocks).
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(512) : "memory");
}

// Adds the parts of the tiles that were cut, in order of the sum: a thread block for 32 rows x 32 columns, which it turns to rows in shared memory.
// The blocks behind those add db, 32 outputs each.
template <int DT>
__global__ void __launch_bounds__(256) grad_parts_kernel(const GradArgs a, int32_t tile_blocks) {
    constexpr int kPitch = 36;                               // floats of a row of the turned block
    __shared__ __align__(16) float room[32 * kPitch];
    pdl_wait();
    pdl_trigger();
    const int32_t per_tile = a.stages_part * a.parts;
    if ((int32_t)blockIdx.x >= tile_blocks) {
        const int lane = (int)threadIdx.x & 31, y = (int)threadIdx.x >> 5;
        const int64_t o = ((int64_t)blockIdx.x - tile_blocks) * 32 + lane;
        const int to = (int)(o >> 8), col = (int)(o & 255);
        float s = 0.f;
        if (a.cut.unit != 1) {
            if (to < a.tiles_o) {
                const float* from = a.dbpart + (2 * a.cut.clusters + (int64_t)to * a.tiles_i) * (kFillPairs * 256) + (int64_t)(y & 1) * 512 + col;
#pragma unroll 8
                for (int t = y >> 1; t < a.tiles_i; t += 4) s += from[(int64_t)t * (kFillPairs * 256)] + from[(int64_t)t * (kFillPairs * 256) + 256];
            }
        } else if (to < a.tiles_o)
            for (int t = y >> 1; t < a.tiles_i; t += 4) {        // two threads a tile, two pairs of warps each
                const int32_t tile = to * a.tiles_i + t, first = tile * per_tile;
                const int32_t w0 = a.cut.owner(first), w1 = a.cut.owner(first + per_tile - 1);
                const float* from = a.dbpart + (int64_t)(y & 1) * 512 + col;
#pragma unroll 4
                for (int32_t w = w0; w <= w1; ++w) {
                    const int64_t slot = w0 == w1 ? 2 * a.cut.clusters + tile : 2 * w + (w == w0 && a.cut.begin(w) < first ? 1 : 0);
                    s += from[slot * (kFillPairs * 256)] + from[slot * (kFillPairs * 256) + 256];
                }
            }
        room[y * 32 + lane] = s;
        __syncthreads();
        if (y == 0 && o < a.O) {
#pragma unroll
            for (int i = 1; i < 8; ++i) s += room[i * 32 + lane];
            a.db[o] = s;
        }
        return;
    }
    const int tile = (int)blockIdx.x >> 6, unit = ((int)blockIdx.x >> 2) & 15, lane = (int)threadIdx.x & 31, g = (int)threadIdx.x >> 5;
    const int32_t first = tile * per_tile, w0 = a.cut.owner(first), w1 = a.cut.owner(first + per_tile - 1);
    if (w0 == w1) return;                                    // stored by the one that added it
    const int to = tile / a.tiles_i, ti = tile - to * a.tiles_i, sw = unit & 7, quarter = (int)blockIdx.x & 3;
    const int64_t o0 = (int64_t)to * 256 + (unit >> 3) * 128 + (sw & 3) * 32, i0 = (int64_t)ti * 256 + (sw >> 2) * 128 + quarter * 32;
    if (o0 >= a.O || i0 >= a.I) return;
    // the tile is the first of its clusters' pieces, but for the one whose piece begins before it
    const float4* from = a.part + (int64_t)unit * 1024 + quarter * 256 + g * 32 + lane;
    float4 s = from[(int64_t)(2 * w0 + (a.cut.begin(w0) < first ? 1 : 0)) * 16384];
    from += (int64_t)(w0 + 1) * 2 * 16384;
    for (int32_t left = w1 - w0; left > 0; left -= 8, from += 8 * 2 * 16384) {   // eight at a time in flight
        float4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? from[(int64_t)j * 2 * 16384] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) { s.x += v[j].x; s.y += v[j].y; s.z += v[j].z; s.w += v[j].w; }
    }
    *reinterpret_cast<float4*>(room + lane * kPitch + g * 4) = s;
    __syncthreads();
    const int r = (int)threadIdx.x >> 3, c = ((int)threadIdx.x & 7) * 4;
    const int64_t i = i0 + c, o = o0 + r;
    const int left = (int)min((int64_t)4, a.I - i);
    if (left <= 0 || o >= a.O) return;
    const float4 v = *reinterpret_cast<const float4*>(room + r * kPitch + c);
    const float f[4] = {v.x, v.y, v.z, v.w};
    if constexpr (DT == TDQ_F32) {
        float* dw = reinterpret_cast<float*>(a.dw) + o * a.dw_stride + i;
        if (a.dw_vec && left == 4) *reinterpret_cast<float4*>(dw) = v;
        else
            for (int j = 0; j < left; ++j) dw[j] = f[j];
    } else {
        uint16_t* dw = reinterpret_cast<uint16_t*>(a.dw) + o * a.dw_stride + i;
        const uint32_t lo = narrow2<DT>(f[0], f[1]), hi = narrow2<DT>(f[2], f[3]);
        if (a.dw_vec && left == 4) *reinterpret_cast<uint2*>(dw) = make_uint2(lo, hi);
        else
            for (int j = 0; j < left; ++j) dw[j] = (uint16_t)((j & 2 ? hi : lo) >> (16 * (j & 1)));
    }
}

// dy as `PARTS` bf16 addends, [PARTS][rows_part][stride], rows behind M zero
template <int DT, int PARTS, bool VEC>
__global__ void __launch_bounds__(256) grad_addends_kernel(const void* dy, int64_t M, int64_t O, int64_t stride, uint16_t* __restrict__ out, int64_t rows_part, int64_t out_stride) {
    using E = typename Elem<DT>::T;
    pdl_wait();
    pdl_trigger();
    const int64_t vecs = out_stride / 8, n = rows_part * vecs;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < n; u += (int64_t)gridDim.x * 256) {
        const int64_t m = u / vecs, o = (u - m * vecs) * 8;
        const E* src = reinterpret_cast<const E*>(dy) + m * stride + o;
        float f[8];
        if constexpr (VEC) {                                 // rows on the 16-byte grid, whole vectors
#pragma unroll
            for (int j = 0; j < 8; j += kPerVec<DT>) widen_vec<DT>(m < M ? __ldg(reinterpret_cast<const uint4*>(src + j)) : make_uint4(0, 0, 0, 0), f + j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = m < M && o + j < O ? widen<DT>(src[j]) : 0.f;
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            uint32_t r[4];
            grad_addend<PARTS>(f, r);
            *reinterpret_cast<uint4*>(out + (p * rows_part + m) * out_stride + o) = make_uint4(r[0], r[1], r[2], r[3]);
        }
    }
}

// dy [rows][cols] bf16 in boxes of 64 tokens x 64 outputs, 128-byte swizzle
bool grad_operand_map(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t stride) {
    return encode_y_map(map, const_cast<void*>(p), true, rows, cols, stride, 64, kTok, false);
}

struct GradPlan {
    int parts;                 // addends of dy
    bool copied;               // dy passes through the workspace
    int64_t rows_part, dy_stride, stages_part, tiles_o, tiles_i, total;
    int32_t clusters;
    int64_t unit;              // stages that stay together
    bool cut;                  // some tile is added by more than one cluster
    bool small;                // the kernel for little work instead
    uint32_t split;            // its parts of the tokens
    size_t dy_bytes, part_bytes, db_bytes, bytes;
};
// How the work is cut, and the room that takes: the status word, parts of tiles and of db, dy's addends.
GradPlan grad_plan(const void* dy, tdq_dtype dtype, int64_t dy_stride, int64_t M, int64_t O, int64_t I, int n_sm) {
    GradPlan p = {};
    p.parts = dtype == TDQ_BF16 ? 1 : dtype == TDQ_F16 ? 2 : 3;
    p.copied = dtype != TDQ_BF16 || reinterpret_cast<uintptr_t>(dy) % 16 || (M > 1 && dy_stride % 8);
    p.stages_part = (M + kTok - 1) / kTok;
    p.rows_part = p.stages_part * kTok;
    p.dy_stride = p.copied || M <= 1 ? (O + 7) / 8 * 8 : dy_stride;
    p.tiles_o = (O + 255) / 256;
    p.tiles_i = (I + 255) / 256;
    const int64_t tiles = p.tiles_o * p.tiles_i, per_tile = p.stages_part * p.parts;
    p.total = tiles * per_tile;
    // Whole tiles, or pieces of any length: the least of these estimates in clocks.  A stage is 580, a tile's store hides behind the next tile's stages
    // if there are enough.  Pieces pay for the second kernel and for every part, written once and read once; so fewer clusters than the GPU holds may be faster.
    const int32_t pairs = std::max(1, n_sm / 2);
    p.clusters = (int32_t)std::min<int64_t>(pairs, tiles);
    p.unit = per_tile;
    int64_t least = (tiles + p.clusters - 1) / p.clusters * std::max<int64_t>(580 * per_tile, 3000) + 2500;
    const auto consider = [&](int64_t w) {
        const int64_t cuts = w - std::gcd<int64_t>(w, tiles), parts = cuts + std::min(cuts, tiles);
        const int64_t cost = 580 * ((p.total + w - 1) / w) + 4500 + 120 * parts;
        if (cuts > 0 && cost < least) { least = cost; p.clusters = (int32_t)w; p.unit = 1; }
    };
    const int64_t most = std::min<int64_t>(pairs, p.total);
    for (int64_t w = most; w > 1; w -= w > 32 ? 6 : w > 16 ? 3 : 1) consider(w);
    for (int64_t w = 2 * tiles; w <= most; w += tiles) consider(w);   // equal parts of every tile: the fewest
    p.cut = p.unit == 1 && per_tile > 1;
    // against the kernel for little work: launch, tensor memory and the way to the first sums, dy's addends, and the second kernel that db needs anyway
    const int esz = dtype == TDQ_F32 ? 4 : 2;
    p.small = grad_small_cost(M, O, fp8_blocks(I), O % 8 == 0 && on_grid(dy, dy_stride, M, esz), esz, n_sm, &p.split) < least + 7000 + (p.copied ? 5000 : 0) + (p.cut ? 0 : 4000);
    if (p.small) {
        p.bytes = kWorkspaceHeader;
        return p;
    }
    p.dy_bytes = p.copied ? (size_t)(p.parts * p.rows_part * p.dy_stride) * 2 : 0;
    p.part_bytes = p.cut ? (size_t)2 * p.clusters * 256 * 256 * 4 : 0;
    p.db_bytes = (size_t)(2 * p.clusters + tiles) * kFillPairs * 256 * 4;
    p.bytes = kWorkspaceHeader + p.part_bytes + p.db_bytes + p.dy_bytes;
    return p;
}

template <int DT>
tdq_status launch_grad(const GradArgs& a, const GradPlan& p, const CUtensorMap& dymap, const CUtensorMap& xmap, const CUtensorMap& dwmap, int dev, cudaStream_t st) {
    static std::atomic<uint64_t> smem_done{0};
    if (allow_smem(fp8_grad_kernel<DT>, (int)kGradSmem, smem_done, dev) != cudaSuccess) return TDQ_ERR_CUDA;
    if (launch_pdl(fp8_grad_kernel<DT>, dim3(2 * (unsigned)p.clusters), dim3(kGradThreads), kGradSmem, st, a, dymap, xmap, dwmap) != cudaSuccess) return TDQ_ERR_CUDA;
    g_launch_count.fetch_add(1, std::memory_order_relaxed);
    if (p.cut || a.db) {
        const int32_t tile_blocks = p.cut ? (int32_t)(p.tiles_o * p.tiles_i * 64) : 0, db_blocks = a.db ? (int32_t)((a.O + 31) / 32) : 0;
        if (launch_pdl(grad_parts_kernel<DT>, dim3((unsigned)(tile_blocks + db_blocks)), dim3(256), 0, st, a, tile_blocks) != cudaSuccess) return TDQ_ERR_CUDA;
        g_launch_count.fetch_add(1, std::memory_order_relaxed);
    }
    return TDQ_OK;
}
template <int DT, int PARTS>
cudaError_t launch_addends(const void* dy, int64_t M, int64_t O, int64_t stride, uint16_t* out, const GradPlan& p, int n_sm, cudaStream_t st) {
    const int64_t blocks = (p.rows_part * (p.dy_stride / 8) + 255) / 256;
    const bool vec = O % 8 == 0 && on_grid(dy, stride, M, sizeof(typename Elem<DT>::T));
    return launch_pdl(vec ? grad_addends_kernel<DT, PARTS, true> : grad_addends_kernel<DT, PARTS, false>, dim3((unsigned)std::min<int64_t>(blocks, 16 * n_sm)), dim3(256), 0, st, dy, M, O, stride, out, p.rows_part, p.dy_stride);
}
constexpr int64_t kGradMax = INT32_MAX - 512;               // coordinates of the copies are 32-bit

}  // namespace
}  // namespace tdq

using namespace tdq;

extern "C" size_t tdq_fp8_weight_grad_workspace_bytes(const void* dy, tdq_dtype dy_dtype, int64_t dy_row_stride, int64_t M, int64_t O, int64_t I) {
    if (!known_dtype(dy_dtype) || M < 0 || O < 0 || I <= 0 || M > kGradMax / 3 || O > kGradMax || I > kGradMax) return 0;
    if (M == 0 || O == 0) return kWorkspaceHeader;
    const int n_sm = current_device_sm_count();
    return grad_plan(dy, dy_dtype, dy_row_stride, M, O, I, n_sm > 0 ? n_sm : 148).bytes;
}

extern "C" tdq_status tdq_fp8_weight_grad(const void* dy, tdq_dtype dy_dtype, int64_t dy_row_stride, const uint8_t* xcodes, const float* xscale, int64_t M,
                                          int64_t O, int64_t I, void* dw, tdq_dtype dw_dtype, int64_t dw_row_stride, float* db, void* workspace,
                                          size_t workspace_bytes, void* cuda_stream) {
    if (!known_dtype(dy_dtype) || !known_dtype(dw_dtype) || M < 0 || O < 0 || I <= 0 || dy_row_stride < O || dw_row_stride < I) return TDQ_ERR_INVALID_ARG;
    if (O == 0) return TDQ_OK;
    if (!dw || (M > 0 && (!dy || !xcodes || !xscale))) return TDQ_ERR_INVALID_ARG;
    const uintptr_t ysz = dy_dtype == TDQ_F32 ? 4 : 2, wsz = dw_dtype == TDQ_F32 ? 4 : 2;
    if (off_grid(dy, ysz) || off_grid(xcodes, 16) || off_grid(xscale, 4) || off_grid(dw, wsz) || off_grid(db, 4) || off_grid(workspace, 16)) return TDQ_ERR_ALIGNMENT;
    if (M > kGradMax / 3 || O > kGradMax || I > kGradMax || dy_row_stride > INT64_MAX / 8 || dw_row_stride > INT64_MAX / 8) return TDQ_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (M == 0) {
        if (cudaMemset2DAsync(dw, (size_t)dw_row_stride * wsz, 0, (size_t)I * wsz, (size_t)O, st) != cudaSuccess) return TDQ_ERR_CUDA;
        if (db && cudaMemsetAsync(db, 0, (size_t)O * 4, st) != cudaSuccess) return TDQ_ERR_CUDA;
        return TDQ_OK;
    }
    int dev = 0;
    const int n_sm = current_device_sm_count(&dev);
    if (n_sm <= 0) return TDQ_ERR_CUDA;
    const GradPlan p = grad_plan(dy, dy_dtype, dy_row_stride, M, O, I, n_sm);
    if (!p.small && (p.tiles_o * p.tiles_i > INT32_MAX / 128 || p.parts * p.rows_part > kGradMax || p.total > INT32_MAX)) return TDQ_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < p.bytes) return TDQ_ERR_WORKSPACE;
    if (p.small) {
        GradSmallArgs g = {xcodes, xscale, dy, dw, db, M, O, I, dy_row_stride, dw_row_stride, (int32_t)fp8_blocks(I), (int32_t)dw_dtype,
                           on_grid(dw, dw_row_stride, O, (int64_t)wsz) && I % 4 == 0, p.split,
                           reinterpret_cast<uint32_t*>(workspace)};
        return launch_grad_small(g, dy_dtype, O % 8 == 0 && on_grid(dy, dy_row_stride, M, (int64_t)ysz), st);
    }
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
    GradArgs a = {};
    a.xcodes = xcodes; a.xscale = xscale; a.dw = dw; a.db = db; a.M = M; a.O = O; a.I = I;
    a.status = reinterpret_cast<uint32_t*>(ws);
    a.part = reinterpret_cast<float4*>(ws + kWorkspaceHeader);
    a.dbpart = reinterpret_cast<float*>(ws + kWorkspaceHeader + p.part_bytes);
    a.dy_stride = p.dy_stride; a.dw_stride = dw_row_stride; a.rows_part = p.rows_part;
    a.Kb = (int32_t)fp8_blocks(I); a.tiles_o = (int32_t)p.tiles_o; a.tiles_i = (int32_t)p.tiles_i; a.stages_part = (int32_t)p.stages_part; a.parts = p.parts;
    a.cut = {(int32_t)(p.total / p.unit), (int32_t)p.unit, p.clusters};
    a.dw_vec = on_grid(dw, dw_row_stride, O, (int64_t)wsz);
    a.dy = reinterpret_cast<const uint16_t*>(dy);
    if (p.copied) {
        uint16_t* out = reinterpret_cast<uint16_t*>(ws + kWorkspaceHeader + p.part_bytes + p.db_bytes);
        a.dy = out;
        const cudaError_t e = dy_dtype == TDQ_BF16 ? launch_addends<TDQ_BF16, 1>(dy, M, O, dy_row_stride, out, p, n_sm, st)
                            : dy_dtype == TDQ_F16  ? launch_addends<TDQ_F16, 2>(dy, M, O, dy_row_stride, out, p, n_sm, st)
                                                   : launch_addends<TDQ_F32, 3>(dy, M, O, dy_row_stride, out, p, n_sm, st);
        if (e != cudaSuccess) return TDQ_ERR_CUDA;
        g_launch_count.fetch_add(1, std::memory_order_relaxed);
    }
    CUtensorMap dymap, xmap, dwmap;
    memset(&dwmap, 0, sizeof dwmap);
    if (!grad_operand_map(&dymap, a.dy, p.copied ? p.parts * p.rows_part : M, p.copied ? p.dy_stride : O, p.dy_stride)) return TDQ_ERR_CUDA;
    if (!fp8_operand_map(&xmap, xcodes, M, (int64_t)a.Kb * kFp8Block, kTok)) return TDQ_ERR_CUDA;
    const int64_t w_stride = O > 1 ? dw_row_stride : (I + 7) / 8 * 8;
    if (a.dw_vec && !encode_y_map(&dwmap, dw, wsz == 2, O, I, w_stride, wsz == 2 ? 64 : 32, 32, dw_dtype == TDQ_F16)) a.dw_vec = 0;
    return dw_dtype == TDQ_F32 ? launch_grad<TDQ_F32>(a, p, dymap, xmap, dwmap, dev, st)
         : dw_dtype == TDQ_BF16 ? launch_grad<TDQ_BF16>(a, p, dymap, xmap, dwmap, dev, st)
                                : launch_grad<TDQ_F16>(a, p, dymap, xmap, dwmap, dev, st);
}
