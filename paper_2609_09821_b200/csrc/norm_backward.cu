// Layer norm of activation rows, backward.  With xh the normalised row, h = dy where the ReLU passed (gamma xh + beta > 0) and
// g = gamma h:
//
//   dx = rstd (g - mean_n g - xh mean_n (g xh)),   dgamma = sum over rows of h xh,   dbeta = sum over rows of h
//
// xh comes from the forward's input and statistics, fl32(fl32(x - mean) rstd), which is bit for bit what the forward pass
// normalised to, so the ReLU opens the same elements; or from an 8-bit checkpoint of it.
// A thread owns eight columns for the whole launch: their share of dgamma and dbeta stays in registers over all rows that
// the CTA walks, and is written once, as one row of partial sums per CTA (summed in fp64 in a fixed order by a second
// kernel, or by the CTAs themselves where few hold all rows, so results are bit-reproducible).  The two row means are sums over the 8 to 512 threads of a row.
// x (or its codes) and dy are read once, dx is written once.  131072 x 1024 from int8, dy and dx bf16: 142 us, 4.7 TB/s; what bounds it is
// issue slots (62 %) between the barriers of two rows.  One row per barrier 193 us, four (spilled) 288, a warp per row with 32
// columns a lane 236.
#include "im_internal.h"
#include "norm.h"

namespace im {

namespace {

// Where eight CTAs hold all rows at once, they are one cluster and finish the column sums themselves.  What that saves is the second
// kernel's launch, 2 us of a call's 11.8; in a graph the cluster's barrier is worth about as much as a second kernel.  In a graph, with the
// second kernel and with the cluster: 16 x 256 bf16 3.8 us and 3.0, 64 x 512 fp32 4.3 and 4.2, 32 x 1024 fp32 4.9 and 5.2 (calls 11.9 and
// 9.9).  Not for wider rows (16 x 2048: 5.9 and 6.9), nor for two batches of rows a CTA (128 x 512: 4.5 and 5.1).
constexpr int kCluster = 8;

constexpr __host__ __device__ int cta_threads(int T) { return T > 256 ? T : 256; }

// The sums of K values (a power of two, at most 4) over the T lanes of a row (T < 32: in every lane), or over a warp: value
// lane_value(lane) of them, in every lane.
template <int T, int K>
__device__ __forceinline__ float lane_sums(float (&s)[K])
{
    constexpr unsigned kAll = 0xffffffffu;
    if (T < 32) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int o = T / 2; o > 0; o >>= 1) s[k] += __shfl_xor_sync(kAll, s[k], o);
        return 0.0f;
    }
    // each half of the lanes goes on with one half of the values: 6 exchanges for 4 values in place of 20
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int n = K / 2, o = 16; n > 0; n /= 2, o /= 2) {
        const bool up = lane & o;
#pragma unroll
        for (int k = 0; k < n; ++k) {
            const float mine = up ? s[n + k] : s[k], other = up ? s[k] : s[n + k];
            s[k] = mine + __shfl_xor_sync(kAll, other, o);
        }
    }
    float one = s[0];
#pragma unroll
    for (int o = 16 / K; o > 0; o >>= 1) one += __shfl_xor_sync(kAll, one, o);
    return one;
}
template <int K>
__device__ __forceinline__ int lane_value(int lane) { return lane / (32 / K); }
template <int K>
__device__ __forceinline__ bool lane_speaks(int lane) { return lane % (32 / K) == 0; }

// T threads share a row; each owns C groups of eight columns: VEC neighbours, else every T-th.  A group of T threads takes R rows
// at a time.
template <typename TX, typename TY, bool VEC, int T, int C, int R, bool KEPT, bool RELU>
__global__ void __launch_bounds__(cta_threads(T), 512 / cta_threads(T)) norm_backward_kernel(const NormBackward P)
{
    constexpr int kCta = cta_threads(T), kGroups = kCta / T, E = 4 * C;
    constexpr int kWarps = T / 32;                                       // of a row (0: less than one)
    __shared__ __align__(16) float s_red[2][kGroups][kWarps > 0 ? kWarps : 1][2 * R];
    __shared__ float s_col[kGroups > 1 ? kCta * 16 : 1];
    const int t = threadIdx.x & (T - 1), g = threadIdx.x / T, N = P.N;
    const auto first = [&](int c) { return VEC ? (c * T + t) * 8 : c * 8 * T + t; };
    constexpr int kStep = VEC ? 1 : T;
    after_previous_kernel();
    const TX *x = static_cast<const TX *>(P.x);
    TX *dx = static_cast<TX *>(P.dx);
    const TY *dy = static_cast<const TY *>(P.dy);
    F2 ga[E], be[RELU ? E : 1], acc_g[E], acc_b[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int k = first(i >> 2) + 2 * (i & 3) * kStep;
        const auto at = [&](const float *p, int c, float other) { return c >= N ? 0.0f : p ? p[c] : other; };
        ga[i] = f2(at(P.gamma, k, 1.0f), at(P.gamma, k + kStep, 1.0f));
        if (RELU) be[i] = f2(at(P.beta, k, 0.0f), at(P.beta, k + kStep, 0.0f));
        acc_g[i] = acc_b[i] = f2(0.0f);
    }
    const float inv_n = 1.0f / (float)N;
    int buf = 0;
    // what a batch of rows needs from memory; columns behind the last are zeros there, and so are their shares of all sums
    struct Batch {
        Eight<TX> x[KEPT ? 1 : R][C];
        Eight<TY> y[R][C];
        uint2 code[KEPT ? R : 1][C];
        uint32_t byte[KEPT ? R : 1][C];
        float mean[R], rstd[R];
    } raw;
    // Nothing is asked for under a condition (a load under one would be waited for where the branches meet): rows behind the last are
    // the last one again, columns behind the last (VEC: whole groups of them) the first, and neither enters a sum or an output.
    const auto load = [&](long long base) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const long long r = min(base + (long long)i * kGroups + g, (long long)P.M - 1);
            const TY *py = dy + r * P.ld_dy;
            const TX *px = x + r * P.ldx;
            const uint8_t *pc = P.kept.code + r * P.kept.ld_code, *ps = P.kept.scale + r * P.kept.ld_scale;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (VEC) {
                    const int col = first(c) < N ? first(c) : 0;
                    raw.y[i][c] = full8(py + col);
                    if (KEPT) {
                        raw.code[i][c] = __ldcs(reinterpret_cast<const uint2 *>(pc + col));
                        raw.byte[i][c] = ps[col >> 5];
                    } else raw.x[i][c] = full8(px + col);
                } else {
                    raw.y[i][c] = load8<false>(py, first(c), T, N);
                    if (KEPT) raw.code[i][c] = load_codes8<false>(pc, first(c), T, N);
                    else raw.x[i][c] = load8<false>(px, first(c), T, N);
                }
            }
            raw.rstd[i] = P.rstd[r];
            if (!KEPT) raw.mean[i] = P.mean[r];
        }
    };
    const long long step = (long long)gridDim.x * kGroups * R;
    load((long long)blockIdx.x * kGroups * R);
    for (long long base = (long long)blockIdx.x * kGroups * R; base < P.M; base += step) {     // (the whole CTA together)
        F2 xh[R][E], h[R][E];
        float s[2 * R], rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rstd[i] = raw.rstd[i];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                unpack8(raw.y[i][c], h[i] + 4 * c);
                if (!KEPT) {
                    unpack8(raw.x[i][c], xh[i] + 4 * c);
                    const F2 minus = f2(-raw.mean[i]), scale = f2(raw.rstd[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) xh[i][4 * c + j] = mul2(add2(xh[i][4 * c + j], minus), scale);
                } else if (VEC) {
                    act8_restore8(raw.code[i][c], raw.byte[i][c], P.kept.form, xh[i] + 4 * c);
                } else {
                    const long long r = base + (long long)i * kGroups + g;
                    act8_restore8(raw.code[i][c], 127u, P.kept.form, xh[i] + 4 * c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int k = first(c) + 2 * j * kStep;
                        const auto scale = [&](int col) { return r < P.M && col < N ? act8_scale(P.kept.scale[r * P.kept.ld_scale + (col >> 5)]) : 0.0f; };
                        xh[i][4 * c + j] = mul2(xh[i][4 * c + j], f2(scale(k), scale(k + kStep)));
                    }
                }
            }
        }
        load(base + step);
        if (base + kGroups * R > P.M) {                                   // the last batch: rows that are none
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (base + (long long)i * kGroups + g >= P.M) {
#pragma unroll
                    for (int e = 0; e < E; ++e) h[i][e] = xh[i][e] = f2(0.0f);
                }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            F2 s1 = f2(0.0f), s2 = f2(0.0f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (VEC && C > 1 && e % 4 == 0 && first(e / 4) >= N) break;
                if (RELU) {
                    const F2 y = fma2(ga[e], xh[i][e], be[e]);
                    h[i][e] = f2(lo(y) > 0.0f ? lo(h[i][e]) : 0.0f, hi(y) > 0.0f ? hi(h[i][e]) : 0.0f);
                }
                const F2 gh = mul2(ga[e], h[i][e]);
                s1 = add2(s1, gh);
                s2 = fma2(gh, xh[i][e], s2);
                acc_b[e] = add2(acc_b[e], h[i][e]);
                acc_g[e] = fma2(h[i][e], xh[i][e], acc_g[e]);
            }
            // (VEC: a thread behind the last column holds the first ones again, which may be infinite)
            const bool counts = !VEC || C > 1 || first(0) < N;
            s[2 * i] = counts ? lo(s1) + hi(s1) : 0.0f;
            s[2 * i + 1] = counts ? lo(s2) + hi(s2) : 0.0f;
        }
        const float one = lane_sums<T>(s);
        if (T == 32) {
#pragma unroll
            for (int k = 0; k < 2 * R; ++k) s[k] = __shfl_sync(0xffffffffu, one, k * (16 / R));
        }
        if (T > 32) {
            const int lane = threadIdx.x & 31;
            if (lane_speaks<2 * R>(lane)) s_red[buf][g][t >> 5][lane_value<2 * R>(lane)] = one;
            // the row group's own barrier (two buffers: nobody still reads the one that is written next)
            asm volatile("bar.sync %0, %1;" ::"r"(1 + g), "n"(T) : "memory");
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                float v[2 * R];
                if (R == 2) {
                    const float4 q = *reinterpret_cast<const float4 *>(s_red[buf][g][w]);
                    v[0] = q.x; v[1] = q.y; v[2 * R - 2] = q.z; v[2 * R - 1] = q.w;
                } else {
                    const float2 q = *reinterpret_cast<const float2 *>(s_red[buf][g][w]);
                    v[0] = q.x; v[1] = q.y;
                }
#pragma unroll
                for (int k = 0; k < 2 * R; ++k) s[k] = w == 0 ? v[k] : s[k] + v[k];
            }
            buf ^= 1;
        }
        if (dx) {
            const long long r0 = base + g;
            TX *pd = dx + r0 * P.ld_dx;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const F2 minus_c1 = f2(-(s[2 * i] * inv_n)), minus_c2 = f2(-(s[2 * i + 1] * inv_n)), scale = f2(rstd[i]);
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    F2 out[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int e = 4 * c + j;
                        out[j] = mul2(scale, fma2(xh[i][e], minus_c2, fma2(ga[e], h[i][e], minus_c1)));
                    }
                    if (r0 + (long long)i * kGroups < P.M && first(c) < N) {
                        if (VEC) full_store8<false>(pd + first(c), out);
                        else store8<false, false>(pd, first(c), T, N, out);
                    }
                }
                pd += kGroups * P.ld_dx;
            }
        }
    }
    if (!P.partial) return;
    float *row = P.partial + (long long)blockIdx.x * 2 * N;
    if (kGroups > 1) {
        // one slot per column and kind; neighbouring threads' slots lie side by side
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s_col[(4 * e + 0) * kCta + threadIdx.x] = lo(acc_g[e]);
            s_col[(4 * e + 1) * kCta + threadIdx.x] = hi(acc_g[e]);
            s_col[(4 * e + 2) * kCta + threadIdx.x] = lo(acc_b[e]);
            s_col[(4 * e + 3) * kCta + threadIdx.x] = hi(acc_b[e]);
        }
        __syncthreads();
        if (g == 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                acc_g[e] = acc_b[e] = f2(0.0f);
                for (int k = 0; k < kGroups; ++k) {
                    const float *p = s_col + k * T + t;
                    acc_g[e] = add2(acc_g[e], f2(p[(4 * e + 0) * kCta], p[(4 * e + 1) * kCta]));
                    acc_b[e] = add2(acc_b[e], f2(p[(4 * e + 2) * kCta], p[(4 * e + 3) * kCta]));
                }
            }
        }
    }
    if (g == 0 && (!P.finish || (int)blockIdx.x < P.finish)) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int k = first(e >> 2) + (2 * (e & 3) + u) * kStep;
                if (k < N) {
                    row[k] = u ? hi(acc_g[e]) : lo(acc_g[e]);
                    row[N + k] = u ? hi(acc_b[e]) : lo(acc_b[e]);
                }
            }
    }
    if (!P.finish) return;
    // (CTAs without rows have come here too: they take their share of the columns)
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    for (int k = (int)blockIdx.x * kCta + threadIdx.x; k < 2 * N; k += (int)gridDim.x * kCta) {
        float v[kCluster];
#pragma unroll
        for (int i = 0; i < kCluster; ++i) v[i] = i < P.finish ? __ldcg(P.partial + (long long)i * 2 * N + k) : 0.0f;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < kCluster; ++i) s += (double)v[i];
        float *out = k < N ? P.dgamma : P.dbeta;
        if (out) out[k < N ? k : k - N] = (float)s;
    }
}

template <typename TX, typename TY, bool VEC, int T, int C, int R, bool KEPT, bool RELU>
cudaError_t launch_backward(const NormBackward &a, int n_sm, int *n_partials, cudaStream_t stream)
{
    constexpr int kGroups = cta_threads(T) / T;
    const long long want = ((long long)a.M + kGroups * R - 1) / (kGroups * R);
    if (a.partial && want <= kCluster && T <= 128) {
        NormBackward b = a;
        b.finish = (int)want;
        *n_partials = 0;
        return launch_pdl(norm_backward_kernel<TX, TY, VEC, T, C, R, KEPT, RELU>, dim3(kCluster), dim3(cta_threads(T)), 0, stream, kCluster, b);
    }
    long long most = (long long)n_sm * (512 / cta_threads(T));
    most = most < kNormMaxPartials ? most : kNormMaxPartials;
    const int grid = (int)(want < most ? want : most);
    *n_partials = a.partial ? grid : 0;
    return launch_pdl(norm_backward_kernel<TX, TY, VEC, T, C, R, KEPT, RELU>, dim3((unsigned)grid), dim3(cta_threads(T)), 0, stream, 0, a);
}
template <typename TX, typename TY, bool KEPT, bool RELU>
cudaError_t dispatch_width(const NormBackward &a, bool vec, int n_sm, int *n, cudaStream_t st)
{
    const int N = a.N;
    if (!vec) {
        if (N <= 256) return launch_backward<TX, TY, false, 32, 1, 2, KEPT, RELU>(a, n_sm, n, st);
        if (N <= 1024) return launch_backward<TX, TY, false, 128, 1, 2, KEPT, RELU>(a, n_sm, n, st);
        return launch_backward<TX, TY, false, 512, 2, 1, KEPT, RELU>(a, n_sm, n, st);
    }
    if (N <= 64) return launch_backward<TX, TY, true, 8, 1, 2, KEPT, RELU>(a, n_sm, n, st);
    if (N <= 256) return launch_backward<TX, TY, true, 32, 1, 2, KEPT, RELU>(a, n_sm, n, st);
    if (N <= 512) return launch_backward<TX, TY, true, 64, 1, 2, KEPT, RELU>(a, n_sm, n, st);
    if (N <= 1024) return launch_backward<TX, TY, true, 128, 1, 2, KEPT, RELU>(a, n_sm, n, st);
    if (N <= 2048) return launch_backward<TX, TY, true, 256, 1, 2, KEPT, RELU>(a, n_sm, n, st);
    if (N <= 4096) return launch_backward<TX, TY, true, 512, 1, 1, KEPT, RELU>(a, n_sm, n, st);
    return launch_backward<TX, TY, true, 512, 2, 1, KEPT, RELU>(a, n_sm, n, st);
}
template <typename TX, typename TY>
cudaError_t dispatch_source(const NormBackward &a, bool vec, int n_sm, int *n, cudaStream_t st)
{
    if (a.relu) return a.x ? dispatch_width<TX, TY, false, true>(a, vec, n_sm, n, st) : dispatch_width<TX, TY, true, true>(a, vec, n_sm, n, st);
    return a.x ? dispatch_width<TX, TY, false, false>(a, vec, n_sm, n, st) : dispatch_width<TX, TY, true, false>(a, vec, n_sm, n, st);
}

}  // namespace

cudaError_t launch_norm_backward(const NormBackward &a, int x_dtype, int dy_dtype, int n_sm, int *n_partials, cudaStream_t stream)
{
    const bool vec = a.N % 8 == 0 && rows_aligned16(a.dy, a.ld_dy, dy_dtype) && (!a.dx || rows_aligned16(a.dx, a.ld_dx, x_dtype)) &&
                     (a.x ? rows_aligned16(a.x, a.ldx, x_dtype) : codes_aligned8(a.kept));
    if (x_dtype == IM_DTYPE_F32)
        return dy_dtype == IM_DTYPE_F32 ? dispatch_source<float, float>(a, vec, n_sm, n_partials, stream)
                                        : dispatch_source<float, __nv_bfloat16>(a, vec, n_sm, n_partials, stream);
    return dy_dtype == IM_DTYPE_F32 ? dispatch_source<__nv_bfloat16, float>(a, vec, n_sm, n_partials, stream)
                                    : dispatch_source<__nv_bfloat16, __nv_bfloat16>(a, vec, n_sm, n_partials, stream);
}

}  // namespace im
