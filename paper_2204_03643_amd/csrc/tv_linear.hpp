// Channel products (y = act(x W^T + b) + r and its gradients): types, activations, the 8-bit blocks and the
// epilogue that the product kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tvl {

using bf16 = __bf16;
typedef bf16     bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16     bf16x8 __attribute__((ext_vector_type(8)));
typedef float    f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int16_t  s16x4 __attribute__((ext_vector_type(4)));

enum Act : int { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };
// how z is held for the backward call
enum Held : int { kHeldNone = 0, kHeldPlain = 1, kHeldBits = 2, kHeld8 = 3 };

constexpr int kBlock = 32;            // samples that share a step in an 8-bit checkpoint

template <class T> struct Elems { static constexpr int kPer16 = 16 / (int)sizeof(T); };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return (float)v; }
template <class T> __device__ __forceinline__ T narrow(float v) { return (T)v; }      // to nearest even

// Activations and their slopes.  A NaN goes through all of them (ReLU is zero where z <= 0, which a NaN is not);
// at -infinity gelu and silu are infinity times zero, a NaN.  Results that are kept in 32 bits take erff and expf
// of the device library.  Results that are rounded to bf16 (2^-8) take the normal distribution's tail as
// Q(|z|) = p(t) exp(-z^2/2) / 2, t = 1 / (1 + 0.3275911 |z| / sqrt 2), p the polynomial 7.1.26 of Abramowitz and
// Stegun (off by at most 1.5e-7), and the hardware's exp2 and reciprocal: 16 instructions in place of about 50.
struct Gauss { float cdf, bell; };          // Phi(z), exp(-z^2/2)
template <bool FAST> __device__ __forceinline__ Gauss gauss(float z)
{
    if constexpr (FAST) {
        const float bell = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.23164190f, 1.0f));
        const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float q = 0.5f * p * bell;
        return {z < 0.0f ? q : 1.0f - q, bell};
    } else {
        return {0.5f * (1.0f + erff(z * 0.70710678f)), expf(-0.5f * z * z)};
    }
}
template <bool FAST> __device__ __forceinline__ float logistic(float z)
{
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
    else return 1.0f / (1.0f + expf(-z));
}

template <bool FAST> __device__ __forceinline__ float act_of(float z, int act)
{
    if (act == kRelu) return z <= 0.0f ? 0.0f : z;
    if (act == kGelu) return z * gauss<FAST>(z).cdf;
    if (act == kSilu) return z * logistic<FAST>(z);
    return z;
}

template <bool FAST> __device__ __forceinline__ float slope_of(float z, int act)
{
    if (act == kRelu) return z <= 0.0f ? 0.0f : 1.0f;
    if (act == kGelu) {
        const Gauss g = gauss<FAST>(z);
        return g.cdf + z * g.bell * 0.39894228f;
    }
    if (act == kSilu) {
        const float s = logistic<FAST>(z);
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

// ---- 8-bit blocks.  The step is 2^(e - 6), 2^e the power of two at or below the block's largest finite magnitude
// (2^-120 at least, so that the step is a normal number): the exponent field of that magnitude, less six, is the byte
// that is kept, and everything is exact but the one rounding of x / step to a whole number.
constexpr uint32_t kLeastMagnitude = 7u << 23;      // 2^-120

__device__ __forceinline__ uint32_t finite_magnitude(float v)
{
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t step_byte(uint32_t magnitude)
{
    return (max(magnitude, kLeastMagnitude) >> 23) - 6u;
}
// the code of v for the step 2^(byte - 127); v / step < 128, so the product below cannot overflow
__device__ __forceinline__ int code_of(float v, uint32_t byte)
{
    const float inverse = __uint_as_float((254u - byte) << 23);
    const float q = fminf(fmaxf(rintf(v * inverse), -127.0f), 127.0f);
    return finite_magnitude(v) == 0u && (__float_as_uint(v) & 0x7fffffffu) != 0u ? -128 : (int)q;
}
__device__ __forceinline__ float value_of(int code, uint32_t byte)
{
    return code == -128 ? __uint_as_float(0x7fc00000u) : (float)code * __uint_as_float(byte << 23);
}

// ---- the epilogue of y = act(x W^T + b) + r
struct Epilogue {
    const void *bias;        // [n] or null
    const void *res;         // [m, n] rows of ldr elements, or null
    void       *y;           // [m, n] rows of ldy elements
    void       *held;        // z as it is, packed [m, n]; a bit a sample, 32 to a word; or codes, packed [m, n]
    uint8_t    *exps;        // [m, ceil(n / 32)] step bytes (kHeld8)
    int64_t     ldr, ldy;
    int32_t     act, kind;
};

// 16 bytes at any address that suits T (the hardware takes them in one access wherever they lie), and eight codes.
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_at1 __attribute__((ext_vector_type(2), aligned(1)));
template <class T> __device__ __forceinline__ u32x4 get16(const T *p)
{
    if constexpr (sizeof(T) == 4) return *(const u32x4_at4 *)p;
    else return *(const u32x4_at2 *)p;
}
template <class T> __device__ __forceinline__ void put16(T *p, u32x4 v)
{
    if constexpr (sizeof(T) == 4) *(u32x4_at4 *)p = v;
    else *(u32x4_at2 *)p = v;
}

// Adds the eight values of T that lie in v.
template <class T> __device__ __forceinline__ void add8(float (&p)[8], const u32x4 (&v)[sizeof(T) / 2])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2)       // a bf16 is the upper half of the f32
            p[i] += __uint_as_float(i & 1 ? v[0][i >> 1] & 0xffff0000u : v[0][i >> 1] << 16);
        else
            p[i] += __uint_as_float(v[i >> 2][i & 3]);
    }
}

// Eight consecutive values from p on, the first `have` of them (zeros for the others); and the way back.
template <class T> __device__ __forceinline__ void load8(float (&v)[8], const T *p, int have)
{
    if (have == 8) {
        u32x4 raw[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = get16(p + i * (16 / (int)sizeof(T)));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        add8<T>(v, raw);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < have ? widen(p[i]) : 0.0f;
    }
}
template <class T> __device__ __forceinline__ void store8(T *p, const float (&v)[8], int have)
{
    if (have == 8) {
        if constexpr (sizeof(T) == 2) {
            bf16x8 h;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = narrow<bf16>(v[i]);
            put16(p, __builtin_bit_cast(u32x4, h));
        } else {
            put16(p, __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}));
            put16(p + 4, __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = narrow<T>(v[i]);
    }
}
// Eight codes, four to a word, the first `have` of them.
__device__ __forceinline__ void store_codes(int8_t *p, u32x2 c, int have)
{
    if (have == 8) *(u32x2_at1 *)p = c;
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = (int8_t)(c[i >> 2] >> (8 * (i & 3)));
}

template <bool FAST> __device__ __forceinline__ void act8(float (&p)[8], int act)
{
    if (act == kRelu)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = act_of<FAST>(p[i], kRelu);
    else if (act == kGelu)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = act_of<FAST>(p[i], kGelu);
    else if (act == kSilu)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = act_of<FAST>(p[i], kSilu);
}

// Writes down z of (m, n .. n + 7), of which `have` exist, as e.kind says; four neighbouring lanes hold a block of 32
// columns of one row, and all lanes take part in the exchanges.  kHeldPlain keeps z in the call's dtype: in bf16, half the
// bytes of 32 bits for slopes that are off by 5.5e-4 (2-norm; beside 1.7e-3 of the gradients' own rounding).
template <class T>
__device__ __forceinline__ void hold8(const float (&p)[8], int64_t m, int n, int N, int have, const Epilogue &e)
{
    if (e.kind == kHeldPlain) {
        if (have) store8((T *)e.held + m * N + n, p, have);
    } else if (e.kind == kHeldBits) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have && !(p[i] <= 0.0f)) w |= 1u << ((n & 31) + i);
        w |= __shfl_xor(w, 1);
        w |= __shfl_xor(w, 2);
        if (have && (n & 31) == 0) ((uint32_t *)e.held)[m * ((N + 31) / 32) + n / 32] = w;
    } else if (e.kind == kHeld8) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) top = max(top, finite_magnitude(p[i]));
        top = max(top, (uint32_t)__shfl_xor(top, 1));
        top = max(top, (uint32_t)__shfl_xor(top, 2));
        const uint32_t byte = step_byte(top);
        u32x2 c = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i >> 2] |= ((uint32_t)code_of(p[i], byte) & 255u) << (8 * (i & 3));
        if (have && (n & 31) == 0) e.exps[m * ((N + 31) / 32) + n / 32] = (uint8_t)byte;
        store_codes((int8_t *)e.held + m * N + n, c, have);
    }
}

// p: the sums of products for outputs (m, n .. n + 7), n a multiple of eight.  row: whether this lane has a row at all (it
// takes part in its block's exchanges either way).
template <class T>
__device__ __forceinline__ void finish8(float (&p)[8], int64_t m, int n, int N, bool row, const Epilogue &e)
{
    const int have = row ? max(0, min(8, N - n)) : 0;
    float v[8];
    if (e.bias) {
        load8(v, (const T *)e.bias + n, have);
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] += v[i];
    }
    hold8<T>(p, m, n, N, have, e);
    if (!have) return;
    act8<sizeof(T) == 2>(p, e.act);
    if (e.res) {
        load8(v, (const T *)e.res + m * e.ldr + n, have);
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] += v[i];
    }
    store8((T *)e.y + m * e.ldy + n, p, have);
}

}  // namespace tvl
