// Activations stored in 8 bits between the forward and the backward pass, and restored (the form: act8.cuh).
#include "act8.cuh"
#include "im_internal.h"

namespace im {

namespace {

constexpr int kThreads = 256;
constexpr int kStride = 32;                // columns between a thread's eight values where rows start anywhere

// A CTA covers 2^tx_bits groups of eight columns by the other threads' rows.  VEC: a thread's eight columns are neighbours, and a block
// of 32 columns is four neighbouring threads; else (tx_bits 5) they lie 32 apart, a block is a warp, and a warp's accesses to single
// elements are side by side (a row of eight neighbours a thread by single stores: 19 us for 9001 x 361 in place of 4).
// Both kernels do a few operations per byte: what bounds them is HBM, hence 16-byte loads and several rows in flight per thread
// (131072 x 1024 bf16 to int8 75 us, back 69: 5.4 and 5.9 TB/s; the maxima row by row: 78 us).
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) pack_kernel(const T *x, long long ldx, int M, int N, const Act8View out, int tx_bits)
{
    constexpr int kRows = !VEC ? 1 : sizeof(T) == 4 ? 2 : 4;              // in flight
    const int tx = threadIdx.x & ((1 << tx_bits) - 1), ty = threadIdx.x >> tx_bits, rows_per_cta = kThreads >> tx_bits;
    const int col = VEC ? (((int)blockIdx.x << tx_bits) + tx) * 8 : (int)blockIdx.x * 8 * kStride + tx;
    const long long row_step = (long long)gridDim.y * rows_per_cta;
    after_previous_kernel();
    // (whole warps run together: the maximum is taken across the lanes of a row)
    for (long long r0 = (long long)blockIdx.y * rows_per_cta; r0 < M; r0 += row_step * kRows) {
        Eight<T> raw[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const long long r = min(r0 + ty + i * row_step, (long long)M - 1);
            raw[i] = load8<VEC>(x + r * ldx, col, kStride, N);
        }
        uint32_t amax[kRows];
        if (VEC) {
            // (step by step over all rows: the exchanges of one hide under those of the others)
#pragma unroll
            for (int i = 0; i < kRows; ++i) amax[i] = largest8(raw[i]);
#pragma unroll
            for (int i = 0; i < kRows; ++i) amax[i] = max(amax[i], __shfl_xor_sync(0xffffffffu, amax[i], 1));
#pragma unroll
            for (int i = 0; i < kRows; ++i) amax[i] = max(amax[i], __shfl_xor_sync(0xffffffffu, amax[i], 2));
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const long long r = r0 + ty + i * row_step;
            F2 v[4];
            unpack8(raw[i], v);
            if (VEC) keep_side8(out, r < M, r, col, N, v, amax[i]);
            else keep8<kStride>(out, r < M, r, col, N, v);
        }
    }
}

template <typename T, bool VEC, bool AFFINE>
__global__ void __launch_bounds__(kThreads, 4) unpack_kernel(const Act8View in, int M, int N, const float *gamma, const float *beta, int relu, T *out,
                                                             long long ld_out, int tx_bits)
{
    constexpr int kRows = AFFINE || !VEC ? 2 : 4, kStep = VEC ? 1 : kStride;
    const int tx = threadIdx.x & ((1 << tx_bits) - 1), ty = threadIdx.x >> tx_bits, rows_per_cta = kThreads >> tx_bits;
    const int col = VEC ? (((int)blockIdx.x << tx_bits) + tx) * 8 : (int)blockIdx.x * 8 * kStride + tx;
    const long long row_step = (long long)gridDim.y * rows_per_cta;
    after_previous_kernel();
    F2 g[4], b[4];
    if (AFFINE) {
        const auto at = [&](const float *p, int k, float other) { return p && k < N ? p[k] : other; };
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = col + 2 * j * kStep;
            g[j] = f2(at(gamma, k, 1.0f), at(gamma, k + kStep, 1.0f));
            b[j] = f2(at(beta, k, 0.0f), at(beta, k + kStep, 0.0f));
        }
    }
    if (col >= N) return;
    for (long long r0 = (long long)blockIdx.y * rows_per_cta + ty; r0 < M; r0 += row_step * kRows) {
        uint2 raw[kRows];
        uint32_t byte[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const long long r = min(r0 + i * row_step, (long long)M - 1);
            raw[i] = load_codes8<VEC>(in.code + r * in.ld_code, col, kStride, N);
            if (VEC) byte[i] = in.scale[r * in.ld_scale + (col >> 5)];
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const long long r = r0 + i * row_step;
            if (r >= M) break;
            F2 v[4];
            if (VEC) act8_restore8(raw[i], byte[i], in.form, v);
            else {
                act8_restore8(raw[i], 127u, in.form, v);
                const uint8_t *ps = in.scale + r * in.ld_scale + (col >> 5);                 // (a value's block is the warp's j-th)
                const auto scale = [&](int j) { return act8_scale(col + j * kStride < N ? ps[j] : 0u); };
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = mul2(v[j], f2(scale(2 * j), scale(2 * j + 1)));
            }
            if (AFFINE) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fma2(g[j], v[j], b[j]);
            }
            if (AFFINE && relu) store8<VEC, true>(out + r * ld_out, col, kStride, N, v);
            else store8<VEC, false>(out + r * ld_out, col, kStride, N, v);
        }
    }
}

// Threads along a row: the most of 32, 16 and 8 that leave the fewest idle; and the grid.
int row_threads_bits(int N, bool vec)
{
    if (!vec) return 5;
    int best = 5;
    long long cover = -1;
    for (int bits = 5; bits >= 3; --bits) {
        const long long w = 8ll << bits, c = (N + w - 1) / w * w;
        if (cover < 0 || c < cover) { best = bits; cover = c; }
    }
    return best;
}
dim3 grid_for(int M, int N, int tx_bits, int rows_at_once, int n_sm)
{
    const int rows_per_cta = kThreads >> tx_bits;
    const unsigned gx = (unsigned)(((long long)N + (8 << tx_bits) - 1) / (8 << tx_bits));     // (so many that no thread's columns pass 2^31 - 1)
    long long gy = ((long long)M + rows_per_cta * rows_at_once - 1) / (rows_per_cta * rows_at_once);
    const long long most = ((long long)n_sm * 16 + gx - 1) / gx;         // beyond that each thread walks more rows
    gy = gy < most ? gy : most;
    return dim3(gx, (unsigned)(gy > 65535 ? 65535 : gy));
}

}  // namespace

}  // namespace im

extern "C" {

im_status im_act8_pack(int32_t M, int32_t N, const void *x, int64_t ldx, int32_t x_dtype, const im_act8 *out, void *cuda_stream)
{
    using namespace im;
    if (!x || M < 1 || N < 1 || ldx < N || !float_dtype(x_dtype) || !aligned_to(x, dtype_size(x_dtype)) || !act8_valid(out, N)) return IM_ERR_INVALID_ARG;
    const int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    const Act8View v = act8_view(out);
    const bool vec = rows_aligned16(x, ldx, x_dtype) && codes_aligned8(v);
    const int bits = row_threads_bits(N, vec);
    const dim3 grid = grid_for(M, N, bits, x_dtype == IM_DTYPE_F32 ? 2 : 4, n_sm);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    const float *xf = static_cast<const float *>(x);
    const __nv_bfloat16 *xb = static_cast<const __nv_bfloat16 *>(x);
    if (x_dtype == IM_DTYPE_F32) {
        if (vec) e = launch_pdl(pack_kernel<float, true>, grid, dim3(kThreads), 0, st, 0, xf, (long long)ldx, M, N, v, bits);
        else e = launch_pdl(pack_kernel<float, false>, grid, dim3(kThreads), 0, st, 0, xf, (long long)ldx, M, N, v, bits);
    } else {
        if (vec) e = launch_pdl(pack_kernel<__nv_bfloat16, true>, grid, dim3(kThreads), 0, st, 0, xb, (long long)ldx, M, N, v, bits);
        else e = launch_pdl(pack_kernel<__nv_bfloat16, false>, grid, dim3(kThreads), 0, st, 0, xb, (long long)ldx, M, N, v, bits);
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

im_status im_act8_unpack(int32_t M, int32_t N, const im_act8 *in, const float *gamma, const float *beta, int32_t relu, void *out, int64_t ld_out,
                         int32_t out_dtype, void *cuda_stream)
{
    using namespace im;
    if (!out || M < 1 || N < 1 || ld_out < N || !float_dtype(out_dtype) || !aligned_to(out, dtype_size(out_dtype)) || !words(gamma, beta) || !act8_valid(in, N)) return IM_ERR_INVALID_ARG;
    const int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    const Act8View v = act8_view(in);
    const bool vec = rows_aligned16(out, ld_out, out_dtype) && codes_aligned8(v), affine = gamma || beta || relu;
    const int bits = row_threads_bits(N, vec);
    const dim3 grid = grid_for(M, N, bits, 4, n_sm);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
#define IM_UNPACK(T, VEC)                                                                                                                     \
    do {                                                                                                                                      \
        if (affine) e = launch_pdl(unpack_kernel<T, VEC, true>, grid, dim3(kThreads), 0, st, 0, v, M, N, gamma, beta, relu, static_cast<T *>(out), (long long)ld_out, bits); \
        else e = launch_pdl(unpack_kernel<T, VEC, false>, grid, dim3(kThreads), 0, st, 0, v, M, N, (const float *)nullptr, (const float *)nullptr, 0, static_cast<T *>(out), (long long)ld_out, bits); \
    } while (0)
    if (out_dtype == IM_DTYPE_F32) {
        if (vec) IM_UNPACK(float, true);
        else IM_UNPACK(float, false);
    } else {
        if (vec) IM_UNPACK(__nv_bfloat16, true);
        else IM_UNPACK(__nv_bfloat16, false);
    }
#undef IM_UNPACK
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

}  // extern "C"
