// Weight gradient from an 8-bit checkpoint: C[n][k] = sum over rows r of A[r][n] H[r][k], A bf16 (the gradient at a layer's
// pre-activation), H restored from im_act8: code 2^e, or bf16(act(gamma code 2^e + beta)).  fp32 accumulation and output.
//
// One CTA per SM: warp 0 fetches A's tiles by TMA (64 rows x BLOCK_N columns, 128B-swizzled), warps 2..9 restore H's tile
// (64 rows x 128 columns) from global memory through registers into the layout that a swizzled TMA load would leave,
// warp 1 issues tcgen05.mma on both as M/N-major operands, warps 10..13 take finished accumulators out of tensor memory.
// H is the M operand, so that a thread of the epilogue holds one k and its warp stores 32 neighbouring k of a row of C.
//
// A restored value has at most 8 significant bits (act8.cuh), so bf16 operands lose nothing of the codes.  Tensor memory
// accumulates kChainBlocks k-blocks at a time; the epilogue adds such chains in fp32 in registers' rounding, which keeps the
// error of long sums independent of the number of rows.
//
// Work is cut along the rows where there are fewer output tiles than SMs: every tile's rows are shared out to the same
// number of CTAs in equal ranges, so that CTAs of different tiles walk the same rows at the same time and share them in L2;
// partial results go to the workspace and a second kernel adds them in a fixed order.
#include <cstring>

#include "act8.cuh"
#include "im_internal.h"
#include "mlp.h"
#include "tc_ptx.cuh"

namespace im {

namespace {

constexpr int kTileK = 128;                // columns of H per tile: the M of the instruction
constexpr int kBlockRows = 64;             // rows of a k-block
constexpr int kDecodeWarps = 8, kEpiWarps = 4;
constexpr int kThreads = 32 * (2 + kDecodeWarps + kEpiWarps);
constexpr int kMaxCtas = 160;              // (the workspace is sized for so many)
constexpr int kChainBlocks = 32;           // k-blocks accumulated in tensor memory before they are added in fp32
constexpr int kMaxCols = 65536;            // of either operand
constexpr size_t kSmemLimit = 232448;

struct Act8GemmParams {
    Act8View h;
    const float *gamma, *beta;             // or null: 1, 0
    int relu;
    int R, Mo, No;                         // rows, columns of A, columns of H
    int tiles_k, tiles, kb;                // tiles along H's columns, all tiles, k-blocks of a tile
    int slices;                            // CTAs sharing a tile
    float *C;
    long long ldc;
    float *partial;                        // [tile * slices + slice][BLOCK_N][128]
    uint32_t *status;
};

template <int BLOCK_N>
struct Plan {
    static constexpr int kABytes = kTileK * kBlockRows * 2, kBBytes = BLOCK_N * kBlockRows * 2, kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = (int)((kSmemLimit - 2048) / kStageBytes) > 8 ? 8 : (int)((kSmemLimit - 2048) / kStageBytes);
    static constexpr int kTmemCols = 2 * BLOCK_N;
    static constexpr size_t kSmemBytes = 1024 + (size_t)kStages * kStageBytes + 512;
};

// The rows of a CTA's part of a tile, in k-blocks.
__device__ __forceinline__ void part_blocks(const Act8GemmParams &P, int slice, int &k0, int &n)
{
    k0 = (int)((long long)slice * P.kb / P.slices);
    n = (int)((long long)(slice + 1) * P.kb / P.slices) - k0;
}

// Sixteen codes of one row to bf16, x16 columns of the swizzled tile: two 16-byte chunks.
template <bool AFFINE>
__device__ __forceinline__ void restore16(const uint4 &w, float s, int form, const float *ga, const float *be, bool relu, uint32_t (&out)[8])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float v[4];
        act8_decode4(u[q], form, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] *= s;
            if (AFFINE) {
                v[j] = __fmaf_rn(ga[4 * q + j], v[j], be[4 * q + j]);
                if (relu) v[j] = v[j] < 0.0f ? 0.0f : v[j];               // (a NaN stays)
            }
        }
        __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]);
        out[2 * q] = *reinterpret_cast<const uint32_t *>(&h);
        h = __floats2bfloat162_rn(v[2], v[3]);
        out[2 * q + 1] = *reinterpret_cast<const uint32_t *>(&h);
    }
}

template <int BLOCK_N, bool AFFINE>
__global__ void __launch_bounds__(kThreads, 1) act8_tn_kernel(const __grid_constant__ CUtensorMap map_a, const Act8GemmParams P)
{
    using PL = Plan<BLOCK_N>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *tiles = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t *full = reinterpret_cast<uint64_t *>(tiles + (size_t)PL::kStages * PL::kStageBytes);
    uint64_t *empty = full + PL::kStages, *acc_full = empty + PL::kStages, *acc_empty = acc_full + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < PL::kStages; ++s) { mbar_init(&full[s], 1 + kDecodeWarps); mbar_init(&empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&acc_full[a], 1); mbar_init(&acc_empty[a], kEpiWarps); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(tmem_slot, PL::kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const int parts = P.tiles * P.slices;
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    if (warp == 0) {
        if (lane == 0 && !g_skip_loads)
            for (int part = blockIdx.x; part < parts; part += gridDim.x) {
                const int slice = part / P.tiles, tile = part - slice * P.tiles;
                const int n0 = tile / P.tiles_k * BLOCK_N;
                int k0, n;
                part_blocks(P, slice, k0, n);
                bool ok = true;
                for (int i = 0; i < n && ok; ++i) {
                    if (!(ok = mbar_wait(&empty[stage], phase ^ 1u, abort_flag))) break;
                    uint8_t *sb = tiles + (size_t)stage * PL::kStageBytes + PL::kABytes;
                    mbar_arrive_expect_tx(&full[stage], PL::kBBytes);
#pragma unroll
                    for (int b = 0; b < BLOCK_N / 64; ++b) tma_load_2d(sb + b * 8192, &map_a, &full[stage], n0 + 64 * b, (k0 + i) * kBlockRows);
                    if (++stage == PL::kStages) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
            }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = instr_desc_bf16_mn(kTileK, BLOCK_N);
            bool ok = true;
            for (int part = blockIdx.x; part < parts && ok; part += gridDim.x) {
                int k0, n;
                part_blocks(P, part / P.tiles, k0, n);
                for (int i = 0; i < n && ok; ++i) {
                    const int in_chain = i % kChainBlocks;
                    if (in_chain == 0) {
                        if (!(ok = mbar_wait(&acc_empty[acc], acc_phase ^ 1u, abort_flag))) break;
                        tc_fence_after();
                    }
                    if (!(ok = mbar_wait(&full[stage], phase, abort_flag))) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(tiles + (size_t)stage * PL::kStageBytes);
                    const uint64_t da = smem_desc_mn_major_sw128(sa, 8192u), db = smem_desc_mn_major_sw128(sa + PL::kABytes, 8192u);
#pragma unroll
                    for (int k = 0; k < kBlockRows / 16; ++k)
                        umma_bf16(tmem_base + (uint32_t)(acc * BLOCK_N), da + (uint64_t)(128 * k), db + (uint64_t)(128 * k), idesc, (in_chain | k) != 0 ? 1u : 0u);
                    umma_commit(&empty[stage]);
                    if (++stage == PL::kStages) { stage = 0; phase ^= 1u; }
                    if (in_chain == kChainBlocks - 1 || i == n - 1) {
                        umma_commit(&acc_full[acc]);
                        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
                    }
                }
            }
        }
    } else if (warp < 2 + kDecodeWarps) {
        // thread: 16 neighbouring columns (cq) of rows r and r + 32 of every k-block; eight threads cover a row of the tile
        const int tid = (warp - 2) * 32 + lane, cq = tid & 7, r = tid >> 3;
        const bool relu = P.relu != 0;
        bool ok = true;
        for (int part = blockIdx.x; part < parts && ok; part += gridDim.x) {
            const int slice = part / P.tiles, tile = part - slice * P.tiles;
            const int col = (tile % P.tiles_k) * kTileK + cq * 16;
            int k0, n;
            part_blocks(P, slice, k0, n);
            float ga[16], be[16];
            if (AFFINE) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    ga[j] = P.gamma && col + j < P.No ? __ldg(P.gamma + col + j) : 1.0f;
                    be[j] = P.beta && col + j < P.No ? __ldg(P.beta + col + j) : 0.0f;
                }
            }
            const bool in_cols = col < P.No;               // (rows are padded to 16 codes, so a chunk is readable as a whole)
            uint4 w[2], w_next[2];
            uint32_t byte[2], byte_next[2];
            const auto fetch = [&](int i) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const long long row = (long long)(k0 + i) * kBlockRows + r + 32 * q;
                    const bool in = in_cols && i < n && row < P.R;
                    w_next[q] = in ? __ldg(reinterpret_cast<const uint4 *>(P.h.code + row * P.h.ld_code + col)) : make_uint4(0u, 0u, 0u, 0u);
                    byte_next[q] = in ? __ldg(P.h.scale + row * P.h.ld_scale + (col >> 5)) : 256u;      // 256: nothing there, zeros
                }
            };
            fetch(0);
            for (int i = 0; i < n; ++i) {
#pragma unroll
                for (int q = 0; q < 2; ++q) { w[q] = w_next[q]; byte[q] = byte_next[q]; }
                fetch(i + 1);
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&empty[stage], phase ^ 1u, abort_flag)))) break;
                const uint32_t sa = smem_u32(tiles + (size_t)stage * PL::kStageBytes) + (uint32_t)((cq >> 2) * 8192);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint32_t o[8];
                    restore16<AFFINE>(w[q], act8_scale(byte[q]), P.h.form, ga, be, relu, o);
                    if (byte[q] == 256u) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = 0u;
                    }
                    const int row = r + 32 * q;
                    // lanes 4..7 of a row write the other 64-column half: in the opposite order, so that eight lanes meet all banks
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const int c = p ^ (cq >> 2);
                        const uint32_t dst = sa + (uint32_t)(row * 128) + (uint32_t)((((cq & 3) * 2 + c) ^ (row & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(c ? o[4] : o[0]), "r"(c ? o[5] : o[1]), "r"(c ? o[6] : o[2]),
                                     "r"(c ? o[7] : o[3]) : "memory");
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&full[stage]);
                if (++stage == PL::kStages) { stage = 0; phase ^= 1u; }
            }
        }
    } else {
        const int quad = warp & 3;                         // tensor-memory lanes 32 quad .. 32 quad + 31
        bool ok = true;
        for (int part = blockIdx.x; part < parts && ok; part += gridDim.x) {
            const int slice = part / P.tiles, tile = part - slice * P.tiles;
            const int n0 = tile / P.tiles_k * BLOCK_N, k = (tile % P.tiles_k) * kTileK + quad * 32 + lane;
            int k0, n;
            part_blocks(P, slice, k0, n);
            // where this thread's column goes, and how far apart its rows are
            float *dst;
            long long ld;
            int rows = BLOCK_N;
            bool in = true;
            if (P.slices == 1) {
                dst = P.C + (long long)n0 * P.ldc + k;
                ld = P.ldc;
                rows = min(BLOCK_N, P.Mo - n0);
                in = k < P.No;
            } else {
                dst = P.partial + ((long long)tile * P.slices + slice) * (BLOCK_N * kTileK) + quad * 32 + lane;
                ld = kTileK;
            }
            for (int i0 = 0; i0 < n; i0 += kChainBlocks) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[acc], acc_phase, abort_flag)))) break;
                tc_fence_after();
                const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * BLOCK_N);
#pragma unroll 1
                for (int c0 = 0; c0 < BLOCK_N; c0 += 32) {
                    float v[32];
                    tmem_ld32_issue(t_row + (uint32_t)c0, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        if (!in || c0 + j >= rows) continue;
                        float *p = dst + (long long)(c0 + j) * ld;
                        *p = i0 == 0 ? v[j] : *p + v[j];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[acc]);
                if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
            }
        }
    }
    // everyone meets; the allocating warp frees tensor memory
    if (*abort_flag && lane == 0) {
        // a wait ran out: copies and MMAs in flight get time to land (bounded)
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 200000ull) { }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) atomicOr(P.status, IM_DEV_WAIT_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, PL::kTmemCols);
    }
}

// C = the slices' partial tiles, added in order: a warp per 32 x 4 columns of one row.
__global__ void __launch_bounds__(256) act8_tn_finish_kernel(const Act8GemmParams P, int block_n)
{
    const int lane = threadIdx.x & 31;
    const int n = (int)blockIdx.y * 8 + (threadIdx.x >> 5), kt = blockIdx.x;
    if (n >= P.Mo) return;
    const int tile = n / block_n * P.tiles_k + kt, row = n % block_n;
    const float4 *src = reinterpret_cast<const float4 *>(P.partial + (long long)tile * P.slices * (block_n * kTileK) + row * kTileK) + lane;
    float4 sum = src[0];
    for (int s = 1; s < P.slices; ++s) {
        const float4 v = src[(long long)s * (block_n * kTileK / 4)];
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    const int k = kt * kTileK + lane * 4;
    float *dst = P.C + (long long)n * P.ldc + k;
    if (k < P.No) dst[0] = sum.x;
    if (k + 1 < P.No) dst[1] = sum.y;
    if (k + 2 < P.No) dst[2] = sum.z;
    if (k + 3 < P.No) dst[3] = sum.w;
}

int block_n_for(int Mo) { return Mo <= 64 ? 64 : Mo <= 128 ? 128 : 256; }

struct Split {
    int block_n, tiles_k, tiles, kb, slices;
};
Split split_for(int R, int Mo, int No, int ctas)
{
    Split s;
    s.block_n = block_n_for(Mo);
    s.tiles_k = (No + kTileK - 1) / kTileK;
    s.tiles = s.tiles_k * ((Mo + s.block_n - 1) / s.block_n);
    s.kb = (R + kBlockRows - 1) / kBlockRows;
    s.slices = ctas / s.tiles;
    const int most = (s.kb + 3) / 4;                        // four k-blocks at least
    s.slices = s.slices < most ? s.slices : most;
    s.slices = s.slices < 1 ? 1 : s.slices;
    return s;
}
size_t partial_bytes(const Split &s) { return s.slices == 1 ? 0 : (size_t)s.tiles * s.slices * s.block_n * kTileK * sizeof(float); }

template <int BLOCK_N, bool AFFINE>
cudaError_t launch_product(const CUtensorMap &map, const Act8GemmParams &p, int grid, cudaStream_t st)
{
    static DeviceOnce once;
    const cudaError_t e = once.run([] {
        return cudaFuncSetAttribute(act8_tn_kernel<BLOCK_N, AFFINE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Plan<BLOCK_N>::kSmemBytes);
    });
    if (e != cudaSuccess) return e;
    act8_tn_kernel<BLOCK_N, AFFINE><<<grid, kThreads, Plan<BLOCK_N>::kSmemBytes, st>>>(map, p);
    return cudaGetLastError();
}
template <int BLOCK_N>
cudaError_t launch_product(const CUtensorMap &map, const Act8GemmParams &p, bool affine, int grid, cudaStream_t st)
{
    return affine ? launch_product<BLOCK_N, true>(map, p, grid, st) : launch_product<BLOCK_N, false>(map, p, grid, st);
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
    return partial_bytes(split_for(R, Mo, No, kMaxCtas));
}

im_status im_gemm_act8_tn(const uint16_t *A, int64_t lda, const im_act8 *H, float *C, int64_t ldc, int32_t R, int32_t Mo, int32_t No, const float *gamma,
                          const float *beta, int32_t relu, void *workspace, size_t workspace_bytes, uint32_t *status, void *cuda_stream)
{
    using namespace im;
    if (!A || !C || !status || R < 1 || Mo < 1 || No < 1 || lda < Mo || ldc < No || (lda & 7) || !aligned_to(A, 16) || !aligned_to(C, 4)) return IM_ERR_INVALID_ARG;
    if (!act8_valid(H, No) || (H->ld_code & 15) || !aligned_to(H->code, 16)) return IM_ERR_INVALID_ARG;
    if (Mo > kMaxCols || No > kMaxCols) return IM_ERR_UNSUPPORTED;
    const size_t need = im_gemm_act8_tn_workspace_bytes(R, Mo, No);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16))) return IM_ERR_INVALID_ARG;
    int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    n_sm = n_sm < kMaxCtas ? n_sm : kMaxCtas;
    CUtensorMap map;
    if (!make_map(&map, A, (uint64_t)R, (uint64_t)Mo, (uint64_t)lda, kBlockRows)) return IM_ERR_CUDA;
    const Split s = split_for(R, Mo, No, n_sm);
    Act8GemmParams p;
    std::memset(&p, 0, sizeof(p));
    p.h = act8_view(H); p.gamma = gamma; p.beta = beta; p.relu = relu != 0;
    p.R = R; p.Mo = Mo; p.No = No; p.tiles_k = s.tiles_k; p.tiles = s.tiles; p.kb = s.kb; p.slices = s.slices;
    p.C = C; p.ldc = ldc; p.partial = static_cast<float *>(workspace); p.status = status;
    const bool affine = gamma || beta || relu;
    const int parts = s.tiles * s.slices, grid = parts < n_sm ? parts : n_sm;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = s.block_n == 64 ? launch_product<64>(map, p, affine, grid, st)
                  : s.block_n == 128 ? launch_product<128>(map, p, affine, grid, st) : launch_product<256>(map, p, affine, grid, st);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess && s.slices > 1) {
        act8_tn_finish_kernel<<<dim3((unsigned)s.tiles_k, (unsigned)((Mo + 7) / 8)), 256, 0, st>>>(p, s.block_n);
        g_launches.fetch_add(1, std::memory_order_relaxed);
        e = cudaGetLastError();
    }
    return e == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

}  // extern "C"
