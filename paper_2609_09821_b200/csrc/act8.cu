// Activations stored in 8 bits between the forward and the backward pass, and restored (the form: act8.cuh).
#include "act8.cuh"
#include "im_internal.h"

namespace im {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsAtOnce = 4;             // a thread's rows in flight

// A CTA covers 2^tx_bits groups of eight columns by the other threads' rows; a block of 32 columns is four neighbouring threads.
// Both kernels do a few operations per byte: what bounds them is HBM, hence 16-byte loads, four rows in flight per thread.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) pack_kernel(const T *x, long long ldx, int M, int N, const Act8View out, int tx_bits)
{
    const int tx = threadIdx.x & ((1 << tx_bits) - 1), ty = threadIdx.x >> tx_bits, rows_per_cta = kThreads >> tx_bits;
    const int col = (((int)blockIdx.x << tx_bits) + tx) * 8;
    const long long row_step = (long long)gridDim.y * rows_per_cta;
    // (whole warps run together: the maximum below is taken across four lanes of a row)
    for (long long r0 = (long long)blockIdx.y * rows_per_cta; r0 < M; r0 += row_step * kRowsAtOnce) {
        Eight<T> raw[kRowsAtOnce];
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
            const long long r = r0 + ty + i * row_step;
            raw[i] = r < M ? load8<VEC>(x + r * ldx, col, 1, N) : zero8(x);
        }
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
            const long long r = r0 + ty + i * row_step;
            F2 v[4];
            unpack8(raw[i], v);
            keep8<true, VEC, 1>(out, r < M, r, col, N, v);
        }
    }
}

template <typename T, bool VEC, bool AFFINE>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const Act8View in, int M, int N, const float *gamma, const float *beta, int relu, T *out,
                                                          long long ld_out, int tx_bits)
{
    const int tx = threadIdx.x & ((1 << tx_bits) - 1), ty = threadIdx.x >> tx_bits, rows_per_cta = kThreads >> tx_bits;
    const int col = (((int)blockIdx.x << tx_bits) + tx) * 8;
    const long long row_step = (long long)gridDim.y * rows_per_cta;
    F2 g[4], b[4];
    if (AFFINE) {
        const auto at = [&](const float *p, int k, float other) { return p && k < N ? __ldg(p + k) : other; };
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            g[j] = f2(at(gamma, col + 2 * j, 1.0f), at(gamma, col + 2 * j + 1, 1.0f));
            b[j] = f2(at(beta, col + 2 * j, 0.0f), at(beta, col + 2 * j + 1, 0.0f));
        }
    }
    if (col >= N) return;
    for (long long r0 = (long long)blockIdx.y * rows_per_cta + ty; r0 < M; r0 += row_step * kRowsAtOnce) {
        uint2 raw[kRowsAtOnce];
        uint32_t byte[kRowsAtOnce];
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
            const long long r = r0 + i * row_step;
            raw[i] = r < M ? load_codes8<VEC>(in.code + r * in.ld_code, col, 1, N) : make_uint2(0u, 0u);
            byte[i] = r < M ? in.scale[r * in.ld_scale + (col >> 5)] : 0u;
        }
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
            const long long r = r0 + i * row_step;
            if (r >= M) break;
            F2 v[4];
            act8_restore8(raw[i], byte[i], in.form, v);
            if (AFFINE) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fma2(g[j], v[j], b[j]);
            }
            if (AFFINE && relu) store8<VEC, true>(out + r * ld_out, col, 1, N, v);
            else store8<VEC, false>(out + r * ld_out, col, 1, N, v);
        }
    }
}

// Threads along a row: as many groups of eight columns as the row has, up to a warp's 32; and the grid over rows.
int row_threads_bits(int N) { return N <= 64 ? 3 : N <= 128 ? 4 : 5; }
dim3 grid_for(int M, int N, int tx_bits, int n_sm)
{
    const int rows_per_cta = kThreads >> tx_bits;
    const unsigned gx = (unsigned)((N + (8 << tx_bits) - 1) / (8 << tx_bits));
    long long gy = ((long long)M + rows_per_cta * kRowsAtOnce - 1) / (rows_per_cta * kRowsAtOnce);
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
    const int bits = row_threads_bits(N);
    const dim3 grid = grid_for(M, N, bits, n_sm);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const float *xf = static_cast<const float *>(x);
    const __nv_bfloat16 *xb = static_cast<const __nv_bfloat16 *>(x);
    if (x_dtype == IM_DTYPE_F32) {
        if (vec) pack_kernel<float, true><<<grid, kThreads, 0, st>>>(xf, ldx, M, N, v, bits);
        else pack_kernel<float, false><<<grid, kThreads, 0, st>>>(xf, ldx, M, N, v, bits);
    } else {
        if (vec) pack_kernel<__nv_bfloat16, true><<<grid, kThreads, 0, st>>>(xb, ldx, M, N, v, bits);
        else pack_kernel<__nv_bfloat16, false><<<grid, kThreads, 0, st>>>(xb, ldx, M, N, v, bits);
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

im_status im_act8_unpack(int32_t M, int32_t N, const im_act8 *in, const float *gamma, const float *beta, int32_t relu, void *out, int64_t ld_out,
                         int32_t out_dtype, void *cuda_stream)
{
    using namespace im;
    if (!out || M < 1 || N < 1 || ld_out < N || !float_dtype(out_dtype) || !aligned_to(out, dtype_size(out_dtype)) || !act8_valid(in, N)) return IM_ERR_INVALID_ARG;
    const int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    const Act8View v = act8_view(in);
    const bool vec = rows_aligned16(out, ld_out, out_dtype) && codes_aligned8(v), affine = gamma || beta || relu;
    const int bits = row_threads_bits(N);
    const dim3 grid = grid_for(M, N, bits, n_sm);
    cudaStream_t st = (cudaStream_t)cuda_stream;
#define IM_UNPACK(T, VEC)                                                                                                                     \
    do {                                                                                                                                      \
        if (affine) unpack_kernel<T, VEC, true><<<grid, kThreads, 0, st>>>(v, M, N, gamma, beta, relu, static_cast<T *>(out), ld_out, bits);   \
        else unpack_kernel<T, VEC, false><<<grid, kThreads, 0, st>>>(v, M, N, nullptr, nullptr, 0, static_cast<T *>(out), ld_out, bits);       \
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
    return cudaGetLastError() == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

}  // extern "C"
