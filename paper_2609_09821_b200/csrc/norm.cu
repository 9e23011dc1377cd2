// Layer norm of activation rows, forward, and the entry points of both passes.
//
//   mean = sum x / N,  rstd = 1 / sqrt(sum (x - mean)^2 / N + eps),  xh = (x - mean) rstd,  y = act(gamma xh + beta)
//
// A row is read once: it stays in the registers of 8 to 256 threads while its mean and then the squares about that mean are
// summed (two passes over registers, so an offset much larger than the spread costs no digits), fp32 throughout.
// What bounds it is HBM: every byte of x and y moves once (131072 x 1024 bf16: 91 us, 5.9 TB/s where a copy reaches 6.5; with the
// 8-bit checkpoint 32768 x 2048: 70 us, 4.8 TB/s, by then issue slots).
#include <cmath>

#include "im_internal.h"
#include "norm.h"

namespace im {

namespace {

constexpr int kThreads = 256;

// The sum of v over the T threads of a row; more than a warp's meet at the row group's own barrier.
template <int T>
__device__ __forceinline__ float row_sum(float v, float *shared, int group)
{
#pragma unroll
    for (int o = (T < 32 ? T : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (T > 32) {
        if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(T) : "memory");
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 32; ++w) v += shared[group * (T / 32) + w];
    }
    return v;
}

// T threads share a row, each holding C groups of eight values: VEC neighbours, else every T-th column.
// gamma and beta lie in shared memory, in the order in which the threads read them (16 bytes a lane side by side): in registers
// they would take twice the row's own share, and read from L1 anew for every row they cost 8 loads per group.
template <typename TX, typename TY, bool VEC, int T, int C>
__global__ void __launch_bounds__(kThreads) norm_forward_kernel(const NormForward P)
{
    constexpr int kGroups = kThreads / T;                         // rows of a CTA at a time
    __shared__ float s_sum[2][kThreads / 32];
    extern __shared__ float4 s_affine[];                          // [gamma, beta][C][2][T]
    const int t = threadIdx.x & (T - 1), g = threadIdx.x / T, N = P.N;
    const TX *x = static_cast<const TX *>(P.x);
    TY *y = static_cast<TY *>(P.y);
    const auto first = [&](int c) { return VEC ? (c * T + t) * 8 : c * 8 * T + t; };
    constexpr int kStep = VEC ? 1 : T;                            // between a group's columns
    const float n = (float)N;
    after_previous_kernel();

    for (int i = threadIdx.x; i < 8 * C * T; i += kThreads) {
        // element i of the layout: group c, half h, thread tt, position p of four
        const int p = i & 3, tt = (i >> 2) & (T - 1), h = (i >> 2) / T & 1, c = (i >> 2) / (2 * T);
        const int col = VEC ? (c * T + tt) * 8 + h * 4 + p : c * 8 * T + (h * 4 + p) * T + tt;
        reinterpret_cast<float *>(s_affine)[i] = P.gamma && col < N ? P.gamma[col] : 1.0f;
        reinterpret_cast<float *>(s_affine)[8 * C * T + i] = P.beta && col < N ? P.beta[col] : 0.0f;
    }
    Eight<TX> raw[C];
    const auto load_row = [&](long long r) {
#pragma unroll
        for (int c = 0; c < C; ++c) raw[c] = r < P.M ? load8<VEC>(x + r * P.ldx, first(c), T, N) : zero8(x);
    };
    const long long step = (long long)gridDim.x * kGroups;
    load_row((long long)blockIdx.x * kGroups + g);
    __syncthreads();
    for (long long base = (long long)blockIdx.x * kGroups; base < P.M; base += step) {       // (the whole CTA together)
        const long long r = base + g;
        F2 v[4 * C];
#pragma unroll
        for (int c = 0; c < C; ++c) unpack8(raw[c], v + 4 * c);
        if (base + step < P.M) load_row(r + step);
        F2 s = v[0];
#pragma unroll
        for (int i = 1; i < 4 * C; ++i) s = add2(s, v[i]);
        const float mean = row_sum<T>(lo(s) + hi(s), s_sum[0], g) / n;
        const F2 minus = f2(-mean);
        s = f2(0.0f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * c + i] = add2(v[4 * c + i], minus);
            if (first(c) + 7 * kStep >= N) {                       // columns behind the last
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[4 * c + i] = f2(first(c) + 2 * i * kStep < N ? lo(v[4 * c + i]) : 0.0f, first(c) + (2 * i + 1) * kStep < N ? hi(v[4 * c + i]) : 0.0f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s = fma2(v[4 * c + i], v[4 * c + i], s);
        }
        const float rstd = 1.0f / sqrtf(row_sum<T>(lo(s) + hi(s), s_sum[1], g) / n + P.eps);
        if (r < P.M && t == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
        const F2 scale = f2(rstd);
#pragma unroll
        for (int i = 0; i < 4 * C; ++i) v[i] = mul2(v[i], scale);      // xh, by the operations that the backward pass repeats
        if (P.keep.code) {
            if (VEC) {
                // (step by step over all groups: the exchanges of one hide under those of the others)
                uint32_t amax[C];
#pragma unroll
                for (int c = 0; c < C; ++c) amax[c] = abs_bits_max8(v + 4 * c);
#pragma unroll
                for (int c = 0; c < C; ++c) amax[c] = max(amax[c], __shfl_xor_sync(0xffffffffu, amax[c], 1));
#pragma unroll
                for (int c = 0; c < C; ++c) amax[c] = max(amax[c], __shfl_xor_sync(0xffffffffu, amax[c], 2));
#pragma unroll
                for (int c = 0; c < C; ++c) keep_side8(P.keep, r < P.M, r, first(c), N, v + 4 * c, amax[c]);
            } else {
#pragma unroll
                for (int c = 0; c < C; ++c) keep8<T>(P.keep, r < P.M, r, first(c), N, v + 4 * c);
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = first(c);
            F2 *e = v + 4 * c;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 ga = s_affine[(2 * c + h) * T + t], be = s_affine[(2 * (C + c) + h) * T + t];
                e[2 * h] = fma2(f2(ga.x, ga.y), e[2 * h], f2(be.x, be.y));
                e[2 * h + 1] = fma2(f2(ga.z, ga.w), e[2 * h + 1], f2(be.z, be.w));
            }
            if (r < P.M) {
                if (P.relu) store8<VEC, true>(y + r * P.ldy, col, T, N, e);
                else store8<VEC, false>(y + r * P.ldy, col, T, N, e);
            }
        }
    }
}

// Column sums of the backward pass: the partial rows in fp64, 32 threads a column with their loads in flight together, added in a
// fixed order.  Launched early (programmatically): it waits for the backward kernel, and reads what that wrote by plain loads.
constexpr int kFinishParts = 32;
__global__ void __launch_bounds__(32 * kFinishParts) norm_finish_kernel(const float *partial, int n_partials, int N, float *dgamma, float *dbeta)
{
    after_previous_kernel();
    __shared__ double part[kFinishParts][33];
    const int c = blockIdx.x * 32 + threadIdx.x;                          // of [dgamma | dbeta]
    double s = 0.0;
    if (c < 2 * N)
#pragma unroll 4
        for (int i = threadIdx.y; i < n_partials; i += kFinishParts) s += (double)__ldcg(partial + (long long)i * 2 * N + c);
    part[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && c < 2 * N) {
        double sum = 0.0;
#pragma unroll
        for (int p = 0; p < kFinishParts; ++p) sum += part[p][threadIdx.x];
        float *out = c < N ? dgamma : dbeta;
        if (out) out[c < N ? c : c - N] = (float)sum;
    }
}

template <typename TX, typename TY, bool VEC, int T, int C>
cudaError_t launch_forward(const NormForward &a, int n_sm, cudaStream_t stream)
{
    constexpr int kGroups = kThreads / T;
    constexpr size_t kSmem = (size_t)2 * 8 * C * T * sizeof(float);
    const auto kernel = norm_forward_kernel<TX, TY, VEC, T, C>;
    static DeviceOnce once;
    static std::atomic<int> per_sm[kMaxDevices];                  // CTAs that fit an SM
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = once.run([&] {
        cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
        int fit = 0;
        if (r == cudaSuccess) r = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, kernel, kThreads, kSmem);
        per_sm[dev].store(fit < 1 ? 1 : fit);
        return r;
    });
    if (e != cudaSuccess) return e;
    const long long want = ((long long)a.M + kGroups - 1) / kGroups, most = (long long)n_sm * per_sm[dev].load();
    return launch_pdl(kernel, dim3((unsigned)(want < most ? want : most)), dim3(kThreads), kSmem, stream, 0, a);
}
template <typename TX, typename TY>
cudaError_t dispatch_forward(const NormForward &a, bool vec, int n_sm, cudaStream_t st)
{
    const int N = a.N;
    if (!vec) {
        if (N <= 256) return launch_forward<TX, TY, false, 32, 1>(a, n_sm, st);
        if (N <= 512) return launch_forward<TX, TY, false, 32, 2>(a, n_sm, st);
        if (N <= 768) return launch_forward<TX, TY, false, 32, 3>(a, n_sm, st);
        if (N <= 1024) return launch_forward<TX, TY, false, 32, 4>(a, n_sm, st);
        return launch_forward<TX, TY, false, 256, 4>(a, n_sm, st);
    }
    if (N <= 64) return launch_forward<TX, TY, true, 8, 1>(a, n_sm, st);
    if (N <= 128) return launch_forward<TX, TY, true, 16, 1>(a, n_sm, st);
    if (N <= 256) return launch_forward<TX, TY, true, 32, 1>(a, n_sm, st);
    if (N <= 512) return launch_forward<TX, TY, true, 32, 2>(a, n_sm, st);
    if (N <= 768) return launch_forward<TX, TY, true, 32, 3>(a, n_sm, st);
    if (N <= 1024) return launch_forward<TX, TY, true, 32, 4>(a, n_sm, st);
    if (N <= 2048) return launch_forward<TX, TY, true, 64, 4>(a, n_sm, st);
    if (N <= 4096) return launch_forward<TX, TY, true, 128, 4>(a, n_sm, st);
    return launch_forward<TX, TY, true, 256, 4>(a, n_sm, st);
}

}  // namespace

cudaError_t launch_norm_forward(const NormForward &a, int x_dtype, int y_dtype, int n_sm, cudaStream_t stream)
{
    const bool vec = rows_aligned16(a.x, a.ldx, x_dtype) && rows_aligned16(a.y, a.ldy, y_dtype) && (!a.keep.code || codes_aligned8(a.keep));
    if (x_dtype == IM_DTYPE_F32)
        return y_dtype == IM_DTYPE_F32 ? dispatch_forward<float, float>(a, vec, n_sm, stream) : dispatch_forward<float, __nv_bfloat16>(a, vec, n_sm, stream);
    return y_dtype == IM_DTYPE_F32 ? dispatch_forward<__nv_bfloat16, float>(a, vec, n_sm, stream)
                                   : dispatch_forward<__nv_bfloat16, __nv_bfloat16>(a, vec, n_sm, stream);
}

}  // namespace im

extern "C" {

im_status im_layer_norm_forward(int32_t M, int32_t N, const void *x, int64_t ldx, int32_t x_dtype, const float *gamma, const float *beta, float eps,
                                int32_t relu, void *y, int64_t ldy, int32_t y_dtype, float *mean, float *rstd, const im_act8 *keep, void *cuda_stream)
{
    using namespace im;
    if (!x || !y || M < 1 || N < 1 || ldx < N || ldy < N || !float_dtype(x_dtype) || !float_dtype(y_dtype) || !(eps > 0.0f) || std::isinf(eps)) return IM_ERR_INVALID_ARG;
    if (!aligned_to(x, dtype_size(x_dtype)) || !aligned_to(y, dtype_size(y_dtype)) || !words(gamma, beta, mean, rstd)) return IM_ERR_INVALID_ARG;
    if (keep && !act8_valid(keep, N)) return IM_ERR_INVALID_ARG;
    if (N > kNormMaxCols) return IM_ERR_UNSUPPORTED;
    const int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    NormForward a;
    a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.M = M; a.N = N; a.relu = relu != 0;
    a.gamma = gamma; a.beta = beta; a.eps = eps; a.mean = mean; a.rstd = rstd; a.keep = act8_view(keep);
    const cudaError_t e = launch_norm_forward(a, x_dtype, y_dtype, n_sm, (cudaStream_t)cuda_stream);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

size_t im_layer_norm_workspace_bytes(int32_t M, int32_t N)
{
    using namespace im;
    if (M < 1 || N < 1) return 0;
    return (size_t)(M < kNormMaxPartials ? M : kNormMaxPartials) * 2 * (size_t)N * sizeof(float);
}

im_status im_layer_norm_backward(int32_t M, int32_t N, const void *dy, int64_t ld_dy, int32_t dy_dtype, const void *x, int64_t ldx, int32_t x_dtype,
                                 const float *mean, const float *rstd, const im_act8 *kept, const float *gamma, const float *beta, int32_t relu, void *dx,
                                 int64_t ld_dx, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace im;
    const bool sums = dgamma || dbeta;
    if (!dy || !rstd || M < 1 || N < 1 || ld_dy < N || !float_dtype(x_dtype) || !float_dtype(dy_dtype) || (!dx && !sums)) return IM_ERR_INVALID_ARG;
    if (!x == !kept || (x && (!mean || ldx < N)) || (kept && !act8_valid(kept, N)) || (dx && ld_dx < N)) return IM_ERR_INVALID_ARG;
    if (!aligned_to(dy, dtype_size(dy_dtype)) || !aligned_to(x, dtype_size(x_dtype)) || !aligned_to(dx, dtype_size(x_dtype))) return IM_ERR_INVALID_ARG;
    if (!words(mean, rstd, gamma, beta, dgamma, dbeta)) return IM_ERR_INVALID_ARG;
    if (sums && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < im_layer_norm_workspace_bytes(M, N))) return IM_ERR_INVALID_ARG;
    if (N > kNormMaxCols) return IM_ERR_UNSUPPORTED;
    const int n_sm = device_sm_count();
    if (n_sm <= 0) return IM_ERR_UNSUPPORTED;
    NormBackward a;
    a.dy = dy; a.x = x; a.dx = dx; a.ld_dy = ld_dy; a.ldx = ldx; a.ld_dx = ld_dx; a.M = M; a.N = N; a.relu = relu != 0;
    a.mean = mean; a.rstd = rstd; a.gamma = gamma; a.beta = beta; a.kept = act8_view(kept);
    a.partial = sums ? static_cast<float *>(workspace) : nullptr;
    a.dgamma = dgamma; a.dbeta = dbeta; a.finish = 0;
    int n_partials = 0;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = launch_norm_backward(a, x_dtype, dy_dtype, n_sm, &n_partials, st);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess && n_partials > 0) {
        e = launch_pdl(norm_finish_kernel, dim3((unsigned)((2 * N + 31) / 32)), dim3(32, kFinishParts), 0, st, 0, (const float *)a.partial, n_partials, N, dgamma, dbeta);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    return e == cudaSuccess ? IM_OK : IM_ERR_CUDA;
}

}  // extern "C"
