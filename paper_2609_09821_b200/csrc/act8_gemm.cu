// Weight gradient from an 8-bit checkpoint: C[n][k] = sum over rows r of A[r][n] H[r][k], A bf16 (the gradient at a layer's
// pre-activation), H restored from im_act8: code 2^e, or bf16(act(gamma code 2^e + beta)).  fp32 accumulation and output.
//
// 28 warps: 0 fetches A's tiles by TMA (64 rows x 64-column blocks, 128B-swizzled), 1 issues tcgen05.mma, 2 fetches H's codes
// (64 x 128, by TMA) and with 3 its scales (through registers, any alignment), 4..19 restore H's tile from shared memory into
// the layout that a swizzled TMA load of bf16 would leave, 20..27 take finished accumulators out of tensor memory.  Both
// operands are M/N-major; H is the M operand, so that a thread of the epilogue holds one k and its warp stores 32 neighbouring
// k of a row of C.
//
// PAIR: two CTAs of a cluster compute 256 k x 256 n together (cta_group::2), each restoring its own 128 columns of H and
// fetching half of A's columns: per k-block an SM takes in 16 KB of A and 8 KB of codes in place of 32 + 8 on a 128 x 256 tile of
// its own, which is all that L2 delivers.
//
// A code has at most 7 significant bits (act8.cuh) and the values under gamma, beta and ReLU are bf16 by definition, so bf16 operands lose
// nothing.  The tensor cores
// cut off what their accumulator does not hold rather than rounding it, an error that grows with the number of additions:
// after kChainBlocks k-blocks the epilogue adds the accumulator to the part's sum, which lies in tensor memory too, and the next chain
// starts from zero.
//
// 131072 x 1024 x 1024 from int8 under gamma, beta and ReLU: 237 us, 1160 TFLOP/s (in a long run, at the power limit, 285);
// 16000 x 512 x 1024 28 us, of which 12 are products; 65536 x 69 x 512 21 us, x 28 x 512 20.  What bounds the large product is the restoring warps,
// which take two thirds of the issue slots, and the stop at each chain's end.
//
// Work is cut along the rows where there are fewer output tiles than SMs (act8_split.cuh).  Each tile's rows are shared out to
// `slices` workers (a CTA or a pair) in equal ranges, so that workers of different tiles walk the same rows at the same time and share
// them in L2; where that pays, workers left over take the last rows of all tiles, in a row.  Partial tiles go to the workspace and a
// second kernel adds them in a fixed order.
#include <cstring>

#include "act8.cuh"
#include "act8_split.cuh"
#include "im_internal.h"
#include "mlp.h"
#include "tc_ptx.cuh"

namespace im {

namespace {

constexpr int kScaleWarps = 2, kDecodeWarps = 16, kGroupWarps = 8, kEpiWarps = 8;   // restoring warps: two groups, k-blocks in turn
constexpr int kFirstDecode = 2 + kScaleWarps, kFirstEpi = kFirstDecode + kDecodeWarps;
constexpr int kThreads = 32 * (kFirstEpi + kEpiWarps);
constexpr int kMaxCtas = 160;              // (the workspace is sized for so many)
constexpr int kChainBlocks = 20;           // k-blocks accumulated in tensor memory before they are added in fp32: the error of a
                                           // product is 6e-7 (2-norm) with 16, 9e-7 with 20, 1.3e-6 with 28, and 131072 x 1024 x 1024
                                           // takes 1 % longer with 16 and 2 % less with 28
// Slots for codes and scales.  Even, so that a slot always belongs to the same one of the two groups of restoring warps: copies
// complete in any order, and a group that waited for a slot's next phase while the one before, the other group's, was still
// incomplete would take that one's parity for its own.  (The stages' `empty` barriers may change hands: MMAs complete in order, and a
// group's wait for one follows its own wait for a later one of the round before.)
constexpr int kRaw = 6;
static_assert(kRaw % 2 == 0, "a slot belongs to one group");
constexpr int kRawBytes = kBlockRows * kTileK, kScaleBytes = kBlockRows * (kTileK / kActBlock);
constexpr int kMaxCols = 65536;            // of either operand
constexpr int kMaxRows = 0x7fff0000;       // row numbers (a k-block beyond the last) in 32 bits
constexpr int64_t kMaxStrideBytes = 1ll << 40;       // a tensor map's row strides are below
constexpr size_t kSmemLimit = 232448;

struct Act8GemmParams {
    Act8View h;
    const float *gamma, *beta;             // or null: 1, 0
    int R, Mo, No;                         // rows, columns of A, columns of H
    int tiles_k, tiles, kb;                // tiles along H's columns, all tiles, k-blocks of a tile
    int workers;                           // CTAs or pairs
    int slices, slice_kb, helpers;         // workers per tile and their k-blocks, and workers left over (act8_split.cuh)
    float *C;
    long long ldc;
    float *partial;                        // [slot][tile rows (n)][tile columns (k)]; null: every part is a whole tile and goes to C
    uint32_t *status;
};

template <int BLOCK_N, bool PAIR>
struct Plan {
    static constexpr int kCols = PAIR ? 2 * kTileK : kTileK;                     // columns of H per tile
    static constexpr int kACols = PAIR ? BLOCK_N / 2 : BLOCK_N;                  // columns of A that a CTA fetches
    static constexpr int kHBytes = kTileK * kBlockRows * 2, kABytes = kACols * kBlockRows * 2, kStageBytes = kHBytes + kABytes;    // (and codes and scales elsewhere)
    static constexpr int kStages = BLOCK_N == 64 ? 6 : 5;
    static constexpr int kAccs = PAIR ? 1 : 2;                                   // accumulators; behind them the sum of finished chains
    static constexpr int kTmemCols = BLOCK_N == 64 ? 256 : 512;                  // at least (kAccs + 1) BLOCK_N, a power of two
    static constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + (size_t)kRaw * (kRawBytes + kScaleBytes) + 512;
    static_assert(kSmemBytes <= kSmemLimit && (2 * kStages + 2 * kRaw + 2 * kAccs + 1) * 8 <= 512, "shared memory plan");
};

// Eight codes of one row to bf16.  MODE 0: code 2^e;  1: gamma code 2^e + beta;  2: the same under a ReLU.
template <int FORM, int MODE>
__device__ __forceinline__ void restore8(const uint2 &w, float scale, const F2 *ga, const F2 *be, uint32_t (&out)[4])
{
    const F2 s = f2(scale);
    F2 v[4];
    act8_decode4<FORM>(w.x, v[0], v[1]);
    act8_decode4<FORM>(w.y, v[2], v[3]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = mul2(v[j], s);
        if (MODE) v[j] = fma2(ga[j], v[j], be[j]);
        out[j] = bf16x2<MODE == 2>(v[j]);
    }
}

// The scale bytes of the 128 columns from block b0 of a row on, as one word (blocks behind the last: 0).  Loads that keep their
// place: the compiler would move them down to their first use.
__device__ __forceinline__ uint32_t load_scales(const uint8_t *p, int blocks, bool word)
{
    uint32_t w = 0u;
    if (word) {
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(w) : "l"(p));
        return w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < blocks) {
            uint32_t b;
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(b) : "l"(p + i));
            w |= b << (8 * i);
        }
    return w;
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&v)[32])
{
    const uint32_t *r = reinterpret_cast<const uint32_t *>(v);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                   "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                   "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, float (&v)[16])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr));
}
// Bounded wait of a whole warp (the same answer in every lane): false when the limit ran out or another role gave up.  The hint lets
// the hardware hold the warp for up to 20 us at a time: warps that spin take issue slots from those that restore.
// FROM_PEER: threads of the other CTA of the pair arrive on the barrier too, so what it hands over is acquired at cluster scope.
template <bool FROM_PEER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    const auto try_once = [&]() {
        uint32_t ok;
        if (FROM_PEER)
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tvote.sync.all.pred p, p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
        else
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tvote.sync.all.pred p, p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
        return ok != 0;
    };
    if (try_once()) return true;
    const unsigned long long t0 = global_ns();
    for (;;) {
        if (try_once()) return true;
        const bool late = global_ns() - t0 > g_wait_limit_ns;
        if (late) *abort_flag = 1;
        if (__any_sync(0xffffffffu, late || *abort_flag)) return false;
    }
}
// One lane of a converged warp, the same every time.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// Arrives on a barrier of the pair's leader (map_to_rank), whose MMA warp acquires at cluster scope: a release at cluster scope of
// shared memory alone.  Restored tiles need no more: they lie in this CTA's shared memory, fence.proxy.async has ordered them before the
// tensor core's reads, and the other lanes' share is ordered by the __syncwarp before this lane's release.  Nor do emptied accumulators:
// the loads from tensor memory are complete (tcgen05.wait::ld) and ordered before the arrive by tcgen05.fence, as the MMAs that
// overwrite them are behind the wait.  An arrive.release.cluster releases global memory too and waits for all of it, about 1 us:
// 131072 x 1024 x 1024 410 us with it for the tiles (450 by one warp for all of a k-block) and 260 for the accumulators alone, 249 with this.
__device__ __forceinline__ void mbar_arrive_shared_to_peer(uint32_t cluster_addr)
{
    asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory");
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void mbar_arrive_addr(uint32_t addr) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(addr) : "memory"); }

template <int BLOCK_N, bool PAIR, int FORM, int MODE>
__device__ __forceinline__ void act8_tn_body(const CUtensorMap &map_a, const CUtensorMap &map_h, const Act8GemmParams &P)
{
    using PL = Plan<BLOCK_N, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *raw = tiles + (size_t)PL::kStages * PL::kStageBytes, *scales = raw + (size_t)kRaw * kRawBytes;
    uint64_t *full = reinterpret_cast<uint64_t *>(scales + (size_t)kRaw * kScaleBytes);
    uint64_t *empty = full + PL::kStages, *raw_full = empty + PL::kStages, *raw_empty = raw_full + kRaw, *acc_full = raw_empty + kRaw, *acc_empty = acc_full + PL::kAccs;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + PL::kAccs);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int worker = PAIR ? (int)blockIdx.x >> 1 : (int)blockIdx.x;
    constexpr int kCtas = PAIR ? 2 : 1;

    // full, acc_empty: of the pair's leader (rank 0), whose MMA warp waits on them; the others: each CTA's own
    if (threadIdx.x == 0) {
        for (int s = 0; s < PL::kStages; ++s) { mbar_init(&full[s], 1 + kCtas * kGroupWarps); mbar_init(&empty[s], 1); }
        for (int s = 0; s < kRaw; ++s) { mbar_init(&raw_full[s], 1 + kScaleWarps); mbar_init(&raw_empty[s], kGroupWarps); }
        for (int a = 0; a < PL::kAccs; ++a) { mbar_init(&acc_full[a], 1); mbar_init(&acc_empty[a], kCtas * kEpiWarps); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR) tmem_alloc_pair(tmem_slot, PL::kTmemCols);
        else tmem_alloc(tmem_slot, PL::kTmemCols);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();                            // both CTAs' barriers exist before anyone signals them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (PAIR && threadIdx.x == 0 && rank == 1) {
        // the pair's MMAs address the accumulator at the same tensor-memory address in both CTAs
        uint32_t leader_base;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(leader_base) : "r"(map_to_rank(smem_u32(tmem_slot), 0)) : "memory");
        if (leader_base != tmem_base) *abort_flag = 1;
    }
    if (PAIR) __syncthreads();

    after_previous_kernel();                                 // nothing before this line touches global memory

    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    Part part;
    // The loops of the producer and of the MMA issuer are run by their whole warps, which keeps addresses and descriptors in
    // uniform registers; an elected lane issues.
    if (warp == 0) {
        const bool one = elect_one();
        const uint32_t full0 = PAIR ? map_to_rank(smem_u32(full), 0) : 0u;
        if (!g_skip_loads)
            for (int j = 0; ok && part_at(P, worker, j, part); ++j) {
                const int n0 = part.tile / P.tiles_k * BLOCK_N + (int)rank * PL::kACols;
                int row = part.k0 * kBlockRows;
                for (int i = 0; i < part.n; ++i, row += kBlockRows) {
                    if (!(ok = warp_wait(smem_u32(&empty[stage]), phase ^ 1u, abort_flag))) break;
                    uint8_t *sb = tiles + (size_t)stage * PL::kStageBytes + PL::kHBytes;
                    if (one) {
                        if (rank == 0) mbar_arrive_expect_tx(&full[stage], kCtas * PL::kABytes);
#pragma unroll
                        for (int b = 0; b < PL::kACols / 64; ++b) {
                            if (PAIR) tma_load_2d_pair(sb + b * 8192, &map_a, full0 + (uint32_t)(stage * 8), n0 + 64 * b, row);
                            else tma_load_2d(sb + b * 8192, &map_a, &full[stage], n0 + 64 * b, row);
                        }
                    }
                    __syncwarp();
                    if (++stage == PL::kStages) { stage = 0; phase ^= 1u; }
                }
            }
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc = instr_desc_bf16_mn(kCtas * kTileK, BLOCK_N);
            const bool one = elect_one();
            const uint64_t dh0 = smem_desc_mn_major_sw128(smem_u32(tiles), 8192u), da0 = smem_desc_mn_major_sw128(smem_u32(tiles) + PL::kHBytes, 8192u);
            for (int j = 0; ok && part_at(P, worker, j, part); ++j) {
                int in_chain = 0;
                for (int i = 0; i < part.n; ++i) {
                    if (in_chain == 0) {
                        if (!(ok = warp_wait<PAIR>(smem_u32(&acc_empty[acc]), acc_phase ^ 1u, abort_flag))) break;
                    }
                    if (!(ok = warp_wait<PAIR>(smem_u32(&full[stage]), phase, abort_flag))) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + (uint32_t)(acc * BLOCK_N);
                    const uint64_t step = (uint64_t)(uint32_t)(stage * (PL::kStageBytes >> 4)), dh = dh0 + step, da = da0 + step;
                    const bool last = in_chain == kChainBlocks - 1 || i == part.n - 1;
                    if (one) {
#pragma unroll
                        for (int k = 0; k < kBlockRows / 16; ++k) {
                            const uint32_t more = (in_chain | k) != 0 ? 1u : 0u;
                            if (PAIR) umma_bf16_pair(d, dh + (uint64_t)(128 * k), da + (uint64_t)(128 * k), idesc, more);
                            else umma_bf16(d, dh + (uint64_t)(128 * k), da + (uint64_t)(128 * k), idesc, more);
                        }
                        if (PAIR) umma_commit_pair(&empty[stage]);
                        else umma_commit(&empty[stage]);
                        if (last) {
                            if (PAIR) umma_commit_pair(&acc_full[acc]);
                            else umma_commit(&acc_full[acc]);
                        }
                    }
                    __syncwarp();
                    if (++stage == PL::kStages) { stage = 0; phase ^= 1u; }
                    ++in_chain;
                    if (last) {
                        in_chain = 0;
                        if (++acc == PL::kAccs) { acc = 0; acc_phase ^= 1u; }
                    }
                }
            }
        }
    } else if (warp < kFirstDecode) {
        // codes (warp 2) and scales (a row per lane; words are asked for kLead k-blocks ahead)
        constexpr int kLead = 4;
        const bool one = warp == 2 && elect_one();
        const int r = (warp - 2) * 32 + lane;
        int slot = 0;
        if (!g_skip_loads)
            for (int j = 0; ok && part_at(P, worker, j, part); ++j) {
                const int col = (part.tile % P.tiles_k) * PL::kCols + (int)rank * kTileK, blocks = (P.No - col + kActBlock - 1) / kActBlock;
                const bool word = blocks >= 4 && ((reinterpret_cast<uintptr_t>(P.h.scale) | (uintptr_t)P.h.ld_scale) & 3u) == 0;
                const uint8_t *p = P.h.scale + (col >> 5);
                int row = part.k0 * kBlockRows + r;                              // of the next word asked for
                uint32_t w[kLead];
                const auto ask = [&](uint32_t &to) {
                    to = row < P.R ? load_scales(p + (long long)row * P.h.ld_scale, blocks, word) : 0u;
                    row += kBlockRows;
                };
#pragma unroll
                for (int d = 0; d < kLead; ++d) ask(w[d]);
                for (int i0 = 0; ok && i0 < part.n; i0 += kLead) {
#pragma unroll
                    for (int d = 0; d < kLead; ++d) {
                        if (i0 + d >= part.n) break;
                        if (!(ok = warp_wait(smem_u32(&raw_empty[slot]), phase ^ 1u, abort_flag))) break;
                        if (one) {
                            mbar_arrive_expect_tx(&raw_full[slot], kRawBytes);
                            tma_load_2d(raw + (size_t)slot * kRawBytes, &map_h, &raw_full[slot], col, (part.k0 + i0 + d) * kBlockRows);
                        }
                        reinterpret_cast<uint32_t *>(scales + (size_t)slot * kScaleBytes)[r] = w[d];
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&raw_full[slot]);
                        ask(w[d]);
                        if (++slot == kRaw) { slot = 0; phase ^= 1u; }
                    }
                }
            }
    } else if (warp < kFirstEpi) {
        // Two groups of warps take the k-blocks in turn: the latencies of one's barriers, loads and fence lie under the other's work.
        // thread: 8 neighbouring columns of rows r, r + 16, r + 32 and r + 48.  Eight lanes cover the 64 columns of a swizzled block
        // row, so that a 16-byte store phase meets all banks; the four rows of a warp are b, b + 4, b + 1, b + 5, so that the two
        // rows of a half warp lie in different halves of the codes' swizzle.
        const int group = (warp - kFirstDecode) / kGroupWarps, w8 = (warp - kFirstDecode) % kGroupWarps;
        const int half = w8 >> 2, cq = lane & 7, l4 = lane >> 3;
        const int r = ((w8 >> 1) & 1) * 8 + (w8 & 1) * 2 + (l4 & 1) * 4 + (l4 >> 1);
        const uint32_t tile0 = smem_u32(tiles) + (uint32_t)(half * 8192 + r * 128) + (uint32_t)((cq ^ (r & 7)) << 4);
        const uint32_t raw0 = smem_u32(raw) + (uint32_t)(r * 128) + (uint32_t)(((half * 4 + (cq >> 1)) ^ (r & 7)) << 4) + (uint32_t)((cq & 1) * 8);
        const uint32_t scale0 = smem_u32(scales) + (uint32_t)(r * 4 + half * 2 + (cq >> 2));
        const uint32_t full0 = PAIR && rank == 1 ? map_to_rank(smem_u32(full), 0) : smem_u32(full), raw_full0 = smem_u32(raw_full), raw_empty0 = smem_u32(raw_empty), empty0 = smem_u32(empty);
        int taken = 0, slot = group;
        uint32_t raw_phase = 0;
        stage = group;
        for (int j = 0; ok && part_at(P, worker, j, part); ++j) {
            const int col = (part.tile % P.tiles_k) * PL::kCols + (int)rank * kTileK + half * 64 + cq * 8;
            F2 ga[MODE ? 4 : 1], be[MODE ? 4 : 1];
            if (MODE) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const auto at_col = [&](const float *p, int k, float other) { return p && k < P.No ? p[k] : other; };
                    ga[c] = f2(at_col(P.gamma, col + 2 * c, 1.0f), at_col(P.gamma, col + 2 * c + 1, 1.0f));
                    be[c] = f2(at_col(P.beta, col + 2 * c, 0.0f), at_col(P.beta, col + 2 * c + 1, 0.0f));
                }
            }
            // (taken: k-blocks of earlier parts; slot, stage and their phases: of this group's next one)
            for (int i = (taken + group) & 1; i < part.n; i += 2) {
                if (!(ok = warp_wait(raw_full0 + (uint32_t)(slot * 8), raw_phase, abort_flag))) break;
                const uint32_t from = raw0 + (uint32_t)(slot * kRawBytes), from_scale = scale0 + (uint32_t)(slot * kScaleBytes);
                uint2 w[4];
                uint32_t byte[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[q].x), "=r"(w[q].y) : "r"(from + q * 2048) : "memory");
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte[q]) : "r"(from_scale + q * 64) : "memory");
                }
                if (!(ok = warp_wait(empty0 + (uint32_t)(stage * 8), phase ^ 1u, abort_flag))) break;
                const uint32_t to = tile0 + (uint32_t)(stage * PL::kStageBytes);
                const int rows_left = P.R - (part.k0 + i) * kBlockRows;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t o[4];
                    restore8<FORM, MODE>(w[q], act8_scale(byte[q]), ga, be, o);
                    if (MODE && rows_left < kBlockRows && r + 16 * q >= rows_left) o[0] = o[1] = o[2] = o[3] = 0u;   // behind the last row: zeros, not beta
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + q * 2048), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_addr(raw_empty0 + (uint32_t)(slot * 8));
                    if (PAIR && rank == 1) mbar_arrive_shared_to_peer(full0 + (uint32_t)(stage * 8));
                    else mbar_arrive_addr(full0 + (uint32_t)(stage * 8));
                }
                stage += 2;
                if (stage >= PL::kStages) { stage -= PL::kStages; phase ^= 1u; }
                slot += 2;
                if (slot >= kRaw) { slot -= kRaw; raw_phase ^= 1u; }
            }
            taken += part.n;
        }
    } else {
        // two warps per quadrant of tensor memory (lanes 32 quad .. 32 quad + 31), each with one half of the tile's columns
        const int quad = warp & 3, c_first = ((warp - kFirstEpi) >> 2) * (BLOCK_N / 2);
        for (int j = 0; ok && part_at(P, worker, j, part); ++j) {
            const int n0 = part.tile / P.tiles_k * BLOCK_N, in_tile = (int)rank * kTileK + quad * 32 + lane;
            const int k = (part.tile % P.tiles_k) * PL::kCols + in_tile;
            // where this thread's column goes, and how far apart its rows are
            float *dst = P.partial ? P.partial + (long long)part.slot * (BLOCK_N * PL::kCols) + in_tile : P.C + (long long)n0 * P.ldc + k;
            const long long ld = P.partial ? PL::kCols : P.ldc;
            const int rows = k < P.No ? min(BLOCK_N, P.Mo - n0) : 0;
            for (int i0 = 0; i0 < part.n; i0 += kChainBlocks) {
                if (!(ok = warp_wait(smem_u32(&acc_full[acc]), acc_phase, abort_flag))) break;
                tc_fence_after();
                const uint32_t t_quad = tmem_base + ((uint32_t)(quad * 32) << 16), t_row = t_quad + (uint32_t)(acc * BLOCK_N), t_sum = t_quad + (uint32_t)(PL::kAccs * BLOCK_N);
                // 32 columns at a time: the accumulator plus the sum so far, back into the sum, or out if it is the last chain.  (c0 is hidden
                // from the compiler: where there is one step, on 64-column tiles, it would form all 32 addresses before the first chain
                // and spill 216 bytes next to registers that tensor-memory loads are writing.)
                const bool first = i0 == 0, last = i0 + kChainBlocks >= part.n;
#pragma unroll 1
                for (int c0 = c_first; c0 < c_first + BLOCK_N / 2; c0 += 32) {
                    asm volatile("" : "+r"(c0));
                    float v[32];
                    tmem_ld32_issue(t_row + (uint32_t)c0, v);
                    if (!first) {
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
                            float sum[16];
                            tmem_ld16_issue(t_sum + (uint32_t)(c0 + h), sum);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < 16; ++c) v[h + c] += sum[c];
                        }
                    } else tmem_ld_wait();
                    if (!last) tmem_st32(t_sum + (uint32_t)c0, v);
                    else {
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (c0 + c < rows) dst[(long long)(c0 + c) * ld] = v[c];
                    }
                }
                if (!last) asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR && rank == 1) mbar_arrive_shared_to_peer(map_to_rank(smem_u32(&acc_empty[acc]), 0));
                    else mbar_arrive(&acc_empty[acc]);
                }
                if (++acc == PL::kAccs) { acc = 0; acc_phase ^= 1u; }
            }
        }
    }
    // everyone meets (in a pair, so that shared memory and barriers outlive the peer's use of them); the allocating warp frees tensor memory
    if (*abort_flag && lane == 0) {
        // a wait ran out: copies and MMAs in flight get time to land (bounded)
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 200000ull) { }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) atomicOr(P.status, IM_DEV_WAIT_TIMEOUT);
    if (PAIR) cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) tmem_dealloc_pair(tmem_base, PL::kTmemCols);
        else tmem_dealloc(tmem_base, PL::kTmemCols);
    }
}
template <int BLOCK_N, int FORM, int MODE>
__global__ void __launch_bounds__(kThreads, 1) act8_tn_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_h,
                                                              const Act8GemmParams P)
{
    act8_tn_body<BLOCK_N, false, FORM, MODE>(map_a, map_h, P);
}
template <int FORM, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) act8_tn_pair_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                                            const __grid_constant__ CUtensorMap map_h, const Act8GemmParams P)
{
    act8_tn_body<256, true, FORM, MODE>(map_a, map_h, P);
}

// C = the partial tiles, added in a fixed order (slices, then helpers).  A warp has 128 columns of a row; with SPLIT the eight warps of a
// CTA share one row's parts, every eighth each, and their sums are added in order: few tiles have many parts.
// Launched early (programmatically): it waits for the products, and reads what they wrote by plain loads.
// slices from which it pays: 16000 x 300 x 700 (12 slices) 29.9 us and 30.9 without, x 69 x 512 (37) 13.0 and 20.7, x 512 x 1024 (9) 30.5 and 27.7
constexpr int kSplitFrom = 12;
template <int BLOCK_N, bool PAIR, bool SPLIT>
__global__ void __launch_bounds__(256) act8_tn_finish_kernel(const Act8GemmParams P)
{
    after_previous_kernel();
    using PL = Plan<BLOCK_N, PAIR>;
    constexpr long long kSlot = (long long)BLOCK_N * PL::kCols;
    __shared__ float4 s_part[SPLIT ? 8 : 1][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = SPLIT ? (int)blockIdx.y : (int)blockIdx.y * 8 + warp, k = (int)blockIdx.x * 128 + lane * 4;
    if (n >= P.Mo) return;
    const int tile = n / BLOCK_N * P.tiles_k + k / PL::kCols;
    const float *src = P.partial + (long long)(n % BLOCK_N) * PL::kCols + k % PL::kCols;
    const auto at = [&](long long slot) { return __ldcg(reinterpret_cast<const float4 *>(src + slot * kSlot)); };
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](const float4 &v) { sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w; };
#pragma unroll 4
    for (int s = SPLIT ? warp : 0; s < P.slices; s += SPLIT ? 8 : 1) add(at((long long)tile * P.slices + s));
    if (SPLIT) {
        s_part[warp][lane] = sum;
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int w = 1; w < 8; ++w) add(s_part[w][lane]);
    }
    if (P.helpers) {
        const int rest = P.kb - P.slices * P.slice_kb;
        const long long units = (long long)P.tiles * rest, u0 = (long long)tile * rest, u1 = u0 + rest;
        for (int h = (int)(u0 * P.helpers / units); h < P.helpers; ++h) {              // helpers with units in [u0, u1)
            const long long b = (long long)h * units / P.helpers, e = (long long)(h + 1) * units / P.helpers;
            if (b >= u1) break;
            if (e > u0 && e > b) add(at((long long)P.tiles * P.slices + h + tile));
        }
    }
    float *dst = P.C + (long long)n * P.ldc + k;
    if (k < P.No) dst[0] = sum.x;
    if (k + 1 < P.No) dst[1] = sum.y;
    if (k + 2 < P.No) dst[2] = sum.z;
    if (k + 3 < P.No) dst[3] = sum.w;
}
template <int BLOCK_N, bool PAIR>
cudaError_t launch_finish(const Act8GemmParams &p, cudaStream_t st)
{
    const unsigned gx = (unsigned)((p.No + 127) / 128);
    if (p.slices >= kSplitFrom) return launch_pdl(act8_tn_finish_kernel<BLOCK_N, PAIR, true>, dim3(gx, (unsigned)p.Mo), dim3(256), 0, st, 0, p);
    return launch_pdl(act8_tn_finish_kernel<BLOCK_N, PAIR, false>, dim3(gx, (unsigned)((p.Mo + 7) / 8)), dim3(256), 0, st, 0, p);
}

template <int FORM, int MODE>
cudaError_t launch_product(const Split &s, const CUtensorMap &map, const CUtensorMap &map_h, const Act8GemmParams &p, int grid, cudaStream_t st)
{
    static DeviceOnce once;
    const auto k64 = act8_tn_kernel<64, FORM, MODE>, k128 = act8_tn_kernel<128, FORM, MODE>, kpair = act8_tn_pair_kernel<FORM, MODE>;
    const cudaError_t e = once.run([&] {
        cudaError_t r = cudaFuncSetAttribute(k64, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan<64, false>::kSmemBytes);
        if (r == cudaSuccess) r = cudaFuncSetAttribute(k128, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan<128, false>::kSmemBytes);
        if (r == cudaSuccess) r = cudaFuncSetAttribute(kpair, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan<256, true>::kSmemBytes);
        return r;
    });
    if (e != cudaSuccess) return e;
    if (s.pair) return launch_pdl(kpair, dim3(grid), dim3(kThreads), Plan<256, true>::kSmemBytes, st, 0, map, map_h, p);
    if (s.block_n == 64) return launch_pdl(k64, dim3(grid), dim3(kThreads), Plan<64, false>::kSmemBytes, st, 0, map, map_h, p);
    return launch_pdl(k128, dim3(grid), dim3(kThreads), Plan<128, false>::kSmemBytes, st, 0, map, map_h, p);
}
template <int FORM>
cudaError_t launch_product(const Split &s, const CUtensorMap &map, const CUtensorMap &map_h, const Act8GemmParams &p, int mode, int grid, cudaStream_t st)
{
    return mode == 0 ? launch_product<FORM, 0>(s, map, map_h, p, grid, st)
         : mode == 1 ? launch_product<FORM, 1>(s, map, map_h, p, grid, st) : launch_product<FORM, 2>(s, map, map_h, p, grid, st);
}

}  // namespace

cudaError_t act8_set_wait_debug(unsigned long long limit_ns, int skip_loads)
{
    cudaError_t e = cudaMemcpyToSymbol(g_wait_limit_ns, &limit_ns, sizeof(limit_ns));
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_skip_loads, &skip_loads, sizeof(skip_loads));
    return e;
}

}  // namespace im

extern "C" {

size_t im_gemm_act8_tn_workspace_bytes(int32_t R, int32_t Mo, int32_t No)
{
    using namespace im;
    if (R < 1 || Mo < 1 || No < 1) return 0;
    // for as many SMs as there may be: a slot per worker, and one more per tile for helpers whose range crosses tiles
    const Split s = split_for(R, Mo, No, kMaxCtas);
    if (s.tiles >= s.workers || s.kb < 2 * kLeastBlocks) return 0;
    return (size_t)(s.workers + s.tiles) * s.slot_bytes();
}

im_status im_gemm_act8_tn(const uint16_t *A, int64_t lda, const im_act8 *H, float *C, int64_t ldc, int32_t R, int32_t Mo, int32_t No, const float *gamma,
                          const float *beta, int32_t relu, void *workspace, size_t workspace_bytes, uint32_t *status, void *cuda_stream)
{
    using namespace im;
    if (!A || !C || !status || R < 1 || Mo < 1 || No < 1 || lda < Mo || ldc < No || (lda & 7) || !aligned_to(A, 16) || !words(C, gamma, beta, status)) return IM_ERR_INVALID_ARG;
    if (!act8_valid(H, No) || (H->ld_code & 15) || !aligned_to(H->code, 16)) return IM_ERR_INVALID_ARG;
    if (Mo > kMaxCols || No > kMaxCols || R > kMaxRows || lda >= kMaxStrideBytes / 2 || H->ld_code >= kMaxStrideBytes) return IM_ERR_UNSUPPORTED;
    const size_t need = im_gemm_act8_tn_workspace_bytes(R, Mo, No);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16))) return IM_ERR_INVALID_ARG;
    int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    n_sm = n_sm < kMaxCtas ? n_sm : kMaxCtas;
    CUtensorMap map, map_h;
    if (!make_map(&map, A, (uint64_t)R, (uint64_t)Mo, (uint64_t)lda, kBlockRows) ||
        !make_map_bytes(&map_h, H->code, (uint64_t)R, (uint64_t)No, (uint64_t)H->ld_code, kBlockRows))
        return IM_ERR_CUDA;
    const Split s = split_for(R, Mo, No, n_sm);
    Act8GemmParams p;
    std::memset(&p, 0, sizeof(p));
    p.h = act8_view(H); p.gamma = gamma; p.beta = beta;
    p.R = R; p.Mo = Mo; p.No = No; p.tiles_k = s.tiles_k; p.tiles = s.tiles; p.kb = s.kb;
    p.workers = s.workers; p.slices = s.slices; p.slice_kb = s.slice_kb; p.helpers = s.helpers;
    p.C = C; p.ldc = ldc; p.partial = s.whole() ? nullptr : static_cast<float *>(workspace); p.status = status;
    const int mode = relu ? 2 : gamma || beta ? 1 : 0;
    const int busy = s.helpers || s.tiles * s.slices >= s.workers ? s.workers : s.tiles * s.slices;
    const int grid = s.pair ? 2 * busy : busy;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = H->form == IM_ACT8_INT8 ? launch_product<IM_ACT8_INT8>(s, map, map_h, p, mode, grid, st) : launch_product<IM_ACT8_E4M3>(s, map, map_h, p, mode, grid, st);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess && p.partial) {
        e = s.pair ? launch_finish<256, true>(p, st) : s.block_n == 64 ? launch_finish<64, false>(p, st) : launch_finish<128, false>(p, st);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    return e == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

}  // extern "C"
