// Layer norm of activation rows, backward.  With xh the normalised row, h = dy where the ReLU passed (gamma xh + beta > 0) and
// g = gamma h:
//
//   dx = rstd (g - mean_n g - xh mean_n (g xh)),   dgamma = sum over rows of h xh,   dbeta = sum over rows of h
//
// xh comes from the forward's input and statistics, fl32(fl32(x - mean) rstd), which is bit for bit what the forward pass
// normalised to, so the ReLU opens the same elements; or from an 8-bit checkpoint of it.
// A thread owns eight columns for the whole launch: their share of dgamma and dbeta stays in registers over all rows that
// the CTA walks, and is written once, as one row of partial sums per CTA (summed in fp64 in a fixed order by a second
// kernel, so results are bit-reproducible).  The two row means are sums over the 8 to 1024 threads of a row.
// What bounds it is HBM: x (or its codes) and dy are read once, dx is written once.
#include "im_internal.h"
#include "norm.h"

namespace im {

namespace {

constexpr __host__ __device__ int cta_threads(int T) { return T > 256 ? T : 256; }

template <typename TX, typename TY, bool VEC, int T, int R, bool KEPT>
__global__ void __launch_bounds__(cta_threads(T)) norm_backward_kernel(const NormBackward P)
{
    constexpr int kCta = cta_threads(T), kGroups = kCta / T;
    constexpr int kWarps = T / 32;                                       // of a row (0: less than one)
    __shared__ float s_red[2][kGroups][kWarps > 0 ? kWarps : 1][2 * R];
    __shared__ float s_col[kGroups > 1 ? kCta * 16 : 1];
    const int t = threadIdx.x & (T - 1), g = threadIdx.x / T, N = P.N;
    const int col = VEC ? t * 8 : t;
    const TX *x = static_cast<const TX *>(P.x);
    TX *dx = static_cast<TX *>(P.dx);
    const TY *dy = static_cast<const TY *>(P.dy);
    float ga[8], be[8], acc_g[8], acc_b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int k = VEC ? col + j : col + j * T;
        ga[j] = P.gamma && k < N ? __ldg(P.gamma + k) : (k < N ? 1.0f : 0.0f);
        be[j] = P.beta && k < N ? __ldg(P.beta + k) : 0.0f;
        acc_g[j] = acc_b[j] = 0.0f;
    }
    const float inv_n = 1.0f / (float)N;
    int buf = 0;
    const long long step = (long long)gridDim.x * kGroups * R;
    for (long long base = (long long)blockIdx.x * kGroups * R; base < P.M; base += step) {     // (the whole CTA together)
        Eight<TX> rx[R];
        Eight<TY> ry[R];
        uint2 code[R];
        uint32_t byte[R];
        float mean[R], rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = base + (long long)i * kGroups + g;
            const bool in = r < P.M;
            ry[i] = in ? load8<VEC>(dy + r * P.ld_dy, col, T, N) : zero8(dy);
            rstd[i] = in ? P.rstd[r] : 0.0f;
            if (KEPT) {
                code[i] = in ? load_codes8<VEC>(P.kept.code + r * P.kept.ld_code, col, T, N) : make_uint2(0u, 0u);
                if (VEC) byte[i] = in && col < N ? P.kept.scale[r * P.kept.ld_scale + (col >> 5)] : 0u;
            } else {
                rx[i] = in ? load8<VEC>(x + r * P.ldx, col, T, N) : zero8(x);
                mean[i] = in ? P.mean[r] : 0.0f;
            }
        }
        float xh[R][8], h[R][8], s[2 * R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = base + (long long)i * kGroups + g;
            unpack8(ry[i], h[i]);
            if (KEPT) {
                act8_decode4(code[i].x, P.kept.form, *reinterpret_cast<float(*)[4]>(xh[i]));
                act8_decode4(code[i].y, P.kept.form, *reinterpret_cast<float(*)[4]>(xh[i] + 4));
                if (VEC) {
                    const float sc = act8_scale(byte[i]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) xh[i][j] = col + j < N ? xh[i][j] * sc : 0.0f;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int k = col + j * T;
                        xh[i][j] = r < P.M && k < N ? xh[i][j] * act8_scale(P.kept.scale[r * P.kept.ld_scale + (k >> 5)]) : 0.0f;
                    }
                }
            } else {
                unpack8(rx[i], xh[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int k = VEC ? col + j : col + j * T;
                    xh[i][j] = k < N ? __fmul_rn(__fsub_rn(xh[i][j], mean[i]), rstd[i]) : 0.0f;
                }
            }
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (P.relu && !(__fmaf_rn(ga[j], xh[i][j], be[j]) > 0.0f)) h[i][j] = 0.0f;
                const float gh = ga[j] * h[i][j];
                s1 += gh;
                s2 = fmaf(gh, xh[i][j], s2);
                acc_b[j] += h[i][j];
                acc_g[j] = fmaf(h[i][j], xh[i][j], acc_g[j]);
            }
            s[2 * i] = s1;
            s[2 * i + 1] = s2;
        }
#pragma unroll
        for (int k = 0; k < 2 * R; ++k)
#pragma unroll
            for (int o = (T < 32 ? T : 32) / 2; o > 0; o >>= 1) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
        if (T > 32) {
            if ((threadIdx.x & 31) == 0) {
#pragma unroll
                for (int k = 0; k < 2 * R; ++k) s_red[buf][g][t >> 5][k] = s[k];
            }
            __syncthreads();                    // (two buffers: nobody still reads the one that is written next)
#pragma unroll
            for (int k = 0; k < 2 * R; ++k) {
                s[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) s[k] += s_red[buf][g][w][k];
            }
            buf ^= 1;
        }
        if (dx) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const long long r = base + (long long)i * kGroups + g;
                const float c1 = s[2 * i] * inv_n, c2 = s[2 * i + 1] * inv_n;
                float out[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) out[j] = rstd[i] * (fmaf(ga[j], h[i][j], -c1) - xh[i][j] * c2);
                if (r < P.M) store8<VEC>(dx + r * P.ld_dx, col, T, N, out);
            }
        }
    }
    if (!P.partial) return;
    float *row = P.partial + (long long)blockIdx.x * 2 * N;
    if (kGroups > 1) {
        // one slot per column and kind: columns of a thread lie kCta / kGroups apart, so that lanes meet no bank twice
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s_col[(j * 2 + 0) * kCta + g * T + t] = acc_g[j];
            s_col[(j * 2 + 1) * kCta + g * T + t] = acc_b[j];
        }
        __syncthreads();
        if (g == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc_g[j] = acc_b[j] = 0.0f;
                for (int k = 0; k < kGroups; ++k) {
                    acc_g[j] += s_col[(j * 2 + 0) * kCta + k * T + t];
                    acc_b[j] += s_col[(j * 2 + 1) * kCta + k * T + t];
                }
            }
        }
    }
    if (g == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = VEC ? col + j : col + j * T;
            if (k < N) {
                row[k] = acc_g[j];
                row[N + k] = acc_b[j];
            }
        }
    }
}

template <typename TX, typename TY, bool VEC, int T, int R, bool KEPT>
cudaError_t launch_backward(const NormBackward &a, int n_sm, int *n_partials, cudaStream_t stream)
{
    constexpr int kGroups = cta_threads(T) / T;
    const long long want = ((long long)a.M + kGroups * R - 1) / (kGroups * R);
    long long most = (long long)n_sm * (cta_threads(T) > 256 ? 1 : 4);
    most = most < kNormMaxPartials ? most : kNormMaxPartials;
    const int grid = (int)(want < most ? want : most);
    norm_backward_kernel<TX, TY, VEC, T, R, KEPT><<<grid, cta_threads(T), 0, stream>>>(a);
    *n_partials = grid;
    return cudaGetLastError();
}
template <typename TX, typename TY, bool KEPT>
cudaError_t dispatch_width(const NormBackward &a, bool vec, int n_sm, int *n, cudaStream_t st)
{
    const int N = a.N;
    if (!vec) {
        if (N <= 256) return launch_backward<TX, TY, false, 32, 2, KEPT>(a, n_sm, n, st);
        if (N <= 1024) return launch_backward<TX, TY, false, 128, 2, KEPT>(a, n_sm, n, st);
        return launch_backward<TX, TY, false, 1024, 1, KEPT>(a, n_sm, n, st);
    }
    if (N <= 64) return launch_backward<TX, TY, true, 8, 2, KEPT>(a, n_sm, n, st);
    if (N <= 128) return launch_backward<TX, TY, true, 16, 2, KEPT>(a, n_sm, n, st);
    if (N <= 256) return launch_backward<TX, TY, true, 32, 2, KEPT>(a, n_sm, n, st);
    if (N <= 512) return launch_backward<TX, TY, true, 64, 2, KEPT>(a, n_sm, n, st);
    if (N <= 1024) return launch_backward<TX, TY, true, 128, 2, KEPT>(a, n_sm, n, st);
    if (N <= 2048) return launch_backward<TX, TY, true, 256, 2, KEPT>(a, n_sm, n, st);
    if (N <= 4096) return launch_backward<TX, TY, true, 512, 2, KEPT>(a, n_sm, n, st);
    return launch_backward<TX, TY, true, 1024, 1, KEPT>(a, n_sm, n, st);
}
template <typename TX, typename TY>
cudaError_t dispatch_source(const NormBackward &a, bool vec, int n_sm, int *n, cudaStream_t st)
{
    return a.x ? dispatch_width<TX, TY, false>(a, vec, n_sm, n, st) : dispatch_width<TX, TY, true>(a, vec, n_sm, n, st);
}

}  // namespace

cudaError_t launch_norm_backward(const NormBackward &a, int x_dtype, int dy_dtype, int n_sm, int *n_partials, cudaStream_t stream)
{
    const bool vec = rows_aligned16(a.dy, a.ld_dy, dy_dtype) && (!a.dx || rows_aligned16(a.dx, a.ld_dx, x_dtype)) &&
                     (a.x ? rows_aligned16(a.x, a.ldx, x_dtype) : codes_aligned8(a.kept));
    if (x_dtype == IM_DTYPE_F32)
        return dy_dtype == IM_DTYPE_F32 ? dispatch_source<float, float>(a, vec, n_sm, n_partials, stream)
                                        : dispatch_source<float, __nv_bfloat16>(a, vec, n_sm, n_partials, stream);
    return dy_dtype == IM_DTYPE_F32 ? dispatch_source<__nv_bfloat16, float>(a, vec, n_sm, n_partials, stream)
                                    : dispatch_source<__nv_bfloat16, __nv_bfloat16>(a, vec, n_sm, n_partials, stream);
}

}  // namespace im
