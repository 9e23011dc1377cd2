// The 8-bit form of activations (im_act8): 32 consecutive columns of a row share a power of two 2^e, the least with
// e >= -100 for which the largest magnitude among them fits the code (127 as int8, 448 as e4m3); a code is the value over
// 2^e, rounded to nearest, ties to even.  A code has at most 7 significant bits, so a restored value is exact in bf16.
// The scale byte is e + 127 (27 .. 249, the last for int8 blocks with the largest fp32 numbers); 255 marks a block that held an infinity or a NaN and is restored as NaN.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/im.h"

namespace im {

constexpr int kActBlock = 32;

struct Act8View {                          // im_act8 as the kernels take it
    uint8_t *code, *scale;
    long long ld_code, ld_scale;
    int form;                              // IM_ACT8_*
};

// Whether `a` describes storage for rows of `cols` columns.
inline bool act8_valid(const im_act8 *a, int cols)
{
    return a && a->code && a->scale && (a->form == IM_ACT8_INT8 || a->form == IM_ACT8_E4M3) && a->ld_code >= cols &&
           a->ld_scale >= ((int64_t)cols + kActBlock - 1) / kActBlock;
}
inline Act8View act8_view(const im_act8 *a)
{
    Act8View v = {};
    if (a) { v.code = a->code; v.scale = a->scale; v.ld_code = a->ld_code; v.ld_scale = a->ld_scale; v.form = a->form; }
    return v;
}

// ------------------------------------------------------------------ two fp32 values in one register pair
// Each operation rounds both halves as its scalar form does; the packed forms take one issue slot for two results.
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float lo, float hi)
{
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(x, x); }
__device__ __forceinline__ float lo(F2 a) { return __uint_as_float((uint32_t)a.v); }
__device__ __forceinline__ float hi(F2 a) { return __uint_as_float((uint32_t)(a.v >> 32)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// bf16 of both halves, the low one in the low bits; RELU: negative values become 0, a NaN stays one.
template <bool RELU>
__device__ __forceinline__ uint32_t bf16x2(F2 a)
{
    uint32_t r;
    if (RELU) asm("cvt.rn.relu.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi(a)), "f"(lo(a)));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi(a)), "f"(lo(a)));
    return r;
}

// Scale byte of a block whose largest |value| has the bits `amax` (as an integer a NaN is larger than infinity, and that
// larger than any number, so one integer maximum finds both).
__device__ __forceinline__ uint32_t act8_scale_byte(uint32_t amax, int form)
{
    if (amax >= 0x7f800000u) return 255u;
    const bool i8 = form == IM_ACT8_INT8;
    // 127 = 1.984375 x 2^6, 448 = 1.75 x 2^8
    int b = (int)(amax >> 23) - (i8 ? 6 : 8) + ((amax & 0x7fffffu) > (i8 ? 0x7e0000u : 0x600000u) ? 1 : 0);
    return (uint32_t)(b < 27 ? 27 : b);
}
// 2^e; infinite for a marked block (255), whose codes are 0: NaN
__device__ __forceinline__ float act8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// 1 / 2^e, for byte != 255
__device__ __forceinline__ float act8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t abs_bits_max8(const F2 *v)
{
    uint32_t m = __vimax3_u32(abs_bits(lo(v[0])), abs_bits(hi(v[0])), abs_bits(lo(v[1])));
    m = __vimax3_u32(m, abs_bits(hi(v[1])), abs_bits(lo(v[2])));
    m = __vimax3_u32(m, abs_bits(hi(v[2])), abs_bits(lo(v[3])));
    return max(m, abs_bits(hi(v[3])));
}

// Codes of eight values, lowest byte first, under the scale byte that is theirs.
__device__ __forceinline__ uint2 act8_encode8(const F2 *v, uint32_t byte, int form)
{
    const F2 inv = f2(act8_inverse(byte));
    uint2 w;
    if (form == IM_ACT8_INT8) {
        // 1.5 x 2^23 + value / 2^e (one rounding, the division is exact): the sum's low byte is the nearest integer, in two's complement
        F2 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = fma2(v[i], inv, f2(12582912.0f));
        const auto pack = [](F2 a, F2 b) {
            return __byte_perm(__byte_perm(__float_as_uint(lo(a)), __float_as_uint(hi(a)), 0x0040), __byte_perm(__float_as_uint(lo(b)), __float_as_uint(hi(b)), 0x0040), 0x5410);
        };
        w = make_uint2(pack(q[0], q[1]), pack(q[2], q[3]));
    } else {
        uint16_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 q = mul2(v[i], inv);
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h[i]) : "f"(hi(q)), "f"(lo(q)));
        }
        w = make_uint2((uint32_t)h[0] | ((uint32_t)h[1] << 16), (uint32_t)h[2] | ((uint32_t)h[3] << 16));
    }
    return byte == 255u ? make_uint2(0u, 0u) : w;
}
// The numbers that four codes stand for, without their scale.
template <int FORM>
__device__ __forceinline__ void act8_decode4(uint32_t w, F2 &a, F2 &b)
{
    if (FORM == IM_ACT8_INT8) {
        // 2^23 + (code + 128) by its bits, minus 2^23 + 128: exact
        const uint32_t u = w ^ 0x80808080u;
        const F2 off = f2(-8388736.0f);
        a = add2(f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441))), off);
        b = add2(f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443))), off);
        return;
    }
    float v[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w >> (16 * i))));
        asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}" : "=f"(v[2 * i]), "=f"(v[2 * i + 1]) : "r"(h));
    }
    a = f2(v[0], v[1]);
    b = f2(v[2], v[3]);
}
// Eight values, with their scale.
__device__ __forceinline__ void act8_restore8(const uint2 &w, uint32_t byte, int form, F2 *v)
{
    if (form == IM_ACT8_INT8) {
        act8_decode4<IM_ACT8_INT8>(w.x, v[0], v[1]);
        act8_decode4<IM_ACT8_INT8>(w.y, v[2], v[3]);
    } else {
        act8_decode4<IM_ACT8_E4M3>(w.x, v[0], v[1]);
        act8_decode4<IM_ACT8_E4M3>(w.y, v[2], v[3]);
    }
    const F2 s = f2(act8_scale(byte));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], s);
}

// ------------------------------------------------------------------ rows of fp32 or bf16 values
// A thread's eight values of a row: VEC: eight neighbours, column col .. col + 7, by 16-byte accesses (the row's start allows
// them; a group that crosses the row's end goes element by element); else columns col, col + step, .. .
// Loads go past L1 for good (.cs) and are coherent: outputs may lie where inputs lie.
template <typename T> struct Eight;
template <> struct Eight<float> { float4 a, b; };
template <> struct Eight<__nv_bfloat16> { uint4 a; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void store_as(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_as(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ void set_element(Eight<float> &e, int j, float x) { reinterpret_cast<float *>(&e)[j] = x; }
__device__ __forceinline__ void set_element(Eight<__nv_bfloat16> &e, int j, __nv_bfloat16 x) { reinterpret_cast<__nv_bfloat16 *>(&e)[j] = x; }
__device__ __forceinline__ Eight<float> zero8(const float *) { return {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}; }
__device__ __forceinline__ Eight<__nv_bfloat16> zero8(const __nv_bfloat16 *) { return {make_uint4(0u, 0u, 0u, 0u)}; }
__device__ __forceinline__ Eight<float> full8(const float *p)
{
    return {__ldcs(reinterpret_cast<const float4 *>(p)), __ldcs(reinterpret_cast<const float4 *>(p) + 1)};
}
__device__ __forceinline__ Eight<__nv_bfloat16> full8(const __nv_bfloat16 *p) { return {__ldcs(reinterpret_cast<const uint4 *>(p))}; }

template <bool VEC, typename T>
__device__ __forceinline__ Eight<T> load8(const T *row, int col, int step, int cols)
{
    if (VEC && col <= cols - 8) return full8(row + col);
    Eight<T> e = zero8(row);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = VEC ? col + j : col + j * step;
        if (c < cols) set_element(e, j, row[c]);
    }
    return e;
}
__device__ __forceinline__ void unpack8(const Eight<float> &e, F2 *v)
{
    v[0] = f2(e.a.x, e.a.y); v[1] = f2(e.a.z, e.a.w);
    v[2] = f2(e.b.x, e.b.y); v[3] = f2(e.b.z, e.b.w);
}
__device__ __forceinline__ void unpack8(const Eight<__nv_bfloat16> &e, F2 *v)
{
    const uint32_t w[4] = {e.a.x, e.a.y, e.a.z, e.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
// RELU: negative values become 0, a NaN stays one.
template <bool RELU>
__device__ __forceinline__ float floored(float x) { return RELU && x < 0.0f ? 0.0f : x; }
template <bool RELU>
__device__ __forceinline__ void full_store8(float *p, const F2 *v)
{
    float4 a = make_float4(floored<RELU>(lo(v[0])), floored<RELU>(hi(v[0])), floored<RELU>(lo(v[1])), floored<RELU>(hi(v[1])));
    float4 b = make_float4(floored<RELU>(lo(v[2])), floored<RELU>(hi(v[2])), floored<RELU>(lo(v[3])), floored<RELU>(hi(v[3])));
    if ((reinterpret_cast<uintptr_t>(p) & 31) == 0) {
        // a whole sector by one instruction (131072 x 1024 restored as fp32: 111 us, by two stores of half a sector each 143)
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w), "f"(b.x), "f"(b.y),
                     "f"(b.z), "f"(b.w) : "memory");
        return;
    }
    reinterpret_cast<float4 *>(p)[0] = a;
    reinterpret_cast<float4 *>(p)[1] = b;
}
template <bool RELU>
__device__ __forceinline__ void full_store8(__nv_bfloat16 *p, const F2 *v)
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(bf16x2<RELU>(v[0]), bf16x2<RELU>(v[1]), bf16x2<RELU>(v[2]), bf16x2<RELU>(v[3]));
}
template <bool VEC, bool RELU, typename T>
__device__ __forceinline__ void store8(T *row, int col, int step, int cols, const F2 *v)
{
    if (VEC && col <= cols - 8) {
        full_store8<RELU>(row + col, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = VEC ? col + j : col + j * step;
        if (c < cols) store_as(row + c, floored<RELU>(j & 1 ? hi(v[j >> 1]) : lo(v[j >> 1])));
    }
}
// The largest magnitude among a thread's eight values, as fp32 bits (bf16: two at a time, by their own bits).
__device__ __forceinline__ uint32_t largest8(const Eight<float> &e)
{
    F2 v[4];
    unpack8(e, v);
    return abs_bits_max8(v);
}
__device__ __forceinline__ uint32_t largest8(const Eight<__nv_bfloat16> &e)
{
    constexpr uint32_t kAbs = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vimax3_u16x2(e.a.x & kAbs, e.a.y & kAbs, e.a.z & kAbs), e.a.w & kAbs);
    return max(m << 16, m & 0xffff0000u);
}
// Eight codes of a row, in the same two arrangements.
template <bool VEC>
__device__ __forceinline__ uint2 load_codes8(const uint8_t *row, int col, int step, int cols)
{
    if (VEC && col <= cols - 8) return __ldcs(reinterpret_cast<const uint2 *>(row + col));
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = VEC ? col + j : col + j * step;
        if (c < cols) w[j >> 2] |= (uint32_t)row[c] << (8 * (j & 3));
    }
    return make_uint2(w[0], w[1]);
}
template <bool VEC>
__device__ __forceinline__ void store_codes8(uint8_t *row, int col, int step, int cols, uint2 w)
{
    if (VEC && col <= cols - 8) {
        *reinterpret_cast<uint2 *>(row + col) = w;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = VEC ? col + j : col + j * step;
        if (c < cols) row[c] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
}

// Scale byte and codes of eight neighbouring values, given the largest magnitude of their block.  in: the row exists.
__device__ __forceinline__ void keep_side8(const Act8View &k, bool in, long long row, int col, int cols, const F2 *v, uint32_t amax)
{
    const uint32_t byte = act8_scale_byte(amax, k.form);
    const uint2 w = act8_encode8(v, byte, k.form);
    if (!in || col >= cols) return;
    if ((col & 31) == 0) k.scale[row * k.ld_scale + (col >> 5)] = (uint8_t)byte;
    store_codes8<true>(k.code + row * k.ld_code, col, 1, cols, w);
}

// Scale byte and codes of a thread's eight values of a row that lie T columns apart: a block is one value of each lane.  Whole warps.
template <int T>
__device__ __forceinline__ void keep8(const Act8View &k, bool in, long long row, int col, int cols, const F2 *v)
{
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = col + j * T;
        const float x = j & 1 ? hi(v[j >> 1]) : lo(v[j >> 1]);
        const uint32_t byte = act8_scale_byte(__reduce_max_sync(0xffffffffu, abs_bits(x)), k.form);
        if (in && (c & 31) == 0 && c < cols) k.scale[row * k.ld_scale + (c >> 5)] = (uint8_t)byte;
        const F2 one[4] = {f2(x, 0.0f), f2(0.0f), f2(0.0f), f2(0.0f)};
        w[j >> 2] |= (act8_encode8(one, byte, k.form).x & 255u) << (8 * (j & 3));
    }
    if (in) store_codes8<false>(k.code + row * k.ld_code, col, T, cols, make_uint2(w[0], w[1]));
}

// For kernels launched programmatically: they may start while the kernel before them in the stream ends, and wait here for what that
// writes; the kernel behind them may start in turn.
__device__ __forceinline__ void after_previous_kernel()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

inline bool aligned_to(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
// Whether all of these (any of them null) may hold 32-bit values.
template <typename... P>
inline bool words(const P *...p) { return (aligned_to(p, 4) && ...); }
inline size_t dtype_size(int dtype) { return dtype == IM_DTYPE_F32 ? 4 : 2; }
inline bool float_dtype(int dtype) { return dtype == IM_DTYPE_F32 || dtype == IM_DTYPE_BF16; }
// Whether every row of [.][ld] starts on 16 bytes.
inline bool rows_aligned16(const void *p, int64_t ld, int dtype) { return aligned_to(p, 16) && (ld * (int64_t)dtype_size(dtype)) % 16 == 0; }
inline bool codes_aligned8(const Act8View &v) { return aligned_to(v.code, 8) && v.ld_code % 8 == 0; }

}  // namespace im
