// Byte checkpoints: activations held with eight bits per value and one power-of-two scale per group of
// 32, 64 or 128 consecutive columns (the layout and the rule for the exponent are stated in the public header).
//
// Why the scale is a power of two: x * 2^-e and code * 2^e are then exact, so the only rounding is that of the
// code itself, and a restored value has at most eight significant bits (int8: seven and a sign; e4m3: four),
// which makes it a bf16 number.  The matrix instructions take it as it is: a weight gradient from a checkpoint
// has no error beyond the code's own and that of the fp32 sums.  A scale of amax / 127 would use the codes
// better by at most one bit (half a bit on average) and would round every restored value a second time.
#pragma once

#include "cmpz_internal.h"

namespace cmpz {

constexpr uint32_t kTypeF32 = 0, kTypeF16 = 1, kTypeBF16 = 2;
constexpr uint32_t kByteInt8 = 0, kByteE4M3 = 1;
constexpr uint32_t kActNone = 0, kActRelu = 1, kActSilu = 2;

typedef __bf16   bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16   bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8  __attribute__((ext_vector_type(8)));
typedef float    f32x2  __attribute__((ext_vector_type(2)));
typedef float    f32x4  __attribute__((ext_vector_type(4)));
typedef float    f32x8  __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2  __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4  __attribute__((ext_vector_type(4)));

template <uint32_t T> struct ElemOf;
template <> struct ElemOf<kTypeF32>  { typedef float type; };
template <> struct ElemOf<kTypeF16>  { typedef _Float16 type; };
template <> struct ElemOf<kTypeBF16> { typedef __bf16 type; };

__host__ __device__ constexpr uint32_t type_bytes(uint32_t type) { return type == kTypeF32 ? 4u : 2u; }

// Where the parts of a checkpoint lie.
struct ByteLayout {
    uint64_t pitch;      // bytes of a row of codes: cols rounded up to 16, so that every row takes 128-bit accesses
    uint64_t ngroups;    // exponent bytes of a row
    uint64_t off_exps;   // exponents behind the codes
    uint64_t used;       // end of the exponents
    uint64_t total;      // rounded up to 16
};
inline ByteLayout byte_layout(uint64_t rows, uint64_t cols, uint32_t group)
{
    ByteLayout l;
    l.pitch = (cols + 15) & ~15ull;
    l.ngroups = (cols + group - 1) / group;
    l.off_exps = rows * l.pitch;
    l.used = l.off_exps + rows * l.ngroups;
    l.total = (l.used + 15) & ~15ull;
    return l;
}

// Eight values from p, of which the first n exist (the others read as zero and are not touched).  p has the
// alignment of its type only: 128-bit accesses may start anywhere on this hardware.
template <uint32_t T>
__device__ __forceinline__ f32x8 load8(const typename ElemOf<T>::type *p, int n)
{
    f32x8 v;
    if (n >= 8) {
        if constexpr (T == kTypeF32) {
            __builtin_memcpy(&v, p, 32);
        } else if constexpr (T == kTypeF16) {
            f16x8 h;
            __builtin_memcpy(&h, p, 16);
            v = __builtin_convertvector(h, f32x8);
        } else {
            bf16x8 h;
            __builtin_memcpy(&h, p, 16);
            v = __builtin_convertvector(h, f32x8);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < n ? (float)p[k] : 0.0f;
    }
    return v;
}

// Rounded to nearest even (values beyond fp16's range become infinities, as a cast has it).
template <uint32_t T>
__device__ __forceinline__ void store8(typename ElemOf<T>::type *p, f32x8 v, int n)
{
    typedef typename ElemOf<T>::type E;
    if (n >= 8) {
        if constexpr (T == kTypeF32) {
            __builtin_memcpy(p, &v, 32);
        } else if constexpr (T == kTypeF16) {
            const f16x8 h = __builtin_convertvector(v, f16x8);
            __builtin_memcpy(p, &h, 16);
        } else {
            const bf16x8 h = __builtin_convertvector(v, bf16x8);
            __builtin_memcpy(p, &h, 16);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) p[k] = (E)v[k];
    }
}

// Bit pattern of the largest finite magnitude of eight values (magnitudes order like their patterns).
__device__ __forceinline__ uint32_t amax8(f32x8 v, uint32_t m)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t a = __float_as_uint(v[k]) & 0x7fffffffu;
        const uint32_t f = a < 0x7f800000u ? a : 0u;
        m = f > m ? f : m;
    }
    return m;
}

// Largest of 2^steps neighbouring lanes (steps <= 4); all lanes of the wave take part.
__device__ __forceinline__ uint32_t lanes_max(uint32_t m, uint32_t steps)
{
    auto take = [&m](uint32_t o) { m = o > m ? o : m; };
    if (steps >= 1) take((uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));    // quad: 1 0 3 2
    if (steps >= 2) take((uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));    // quad: 2 3 0 1
    if (steps >= 3) take((uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, true));   // mirrored in 8
    if (steps >= 4) take((uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xf, 0xf, true));   // mirrored in 16
    return m;
}

// Biased exponent e + 127 of a group from the bit pattern of its largest magnitude: adding to the pattern
// carries into the exponent field exactly where the magnitude would round past the largest code
// (127.5 / 64 = 1.9921875: mantissa above 0x7f0000; 448 / 256 = 1.75: above 0x600000).  The lower bound keeps
// every restored value and its products normal, the upper one keeps them finite.
template <uint32_t F>
__device__ __forceinline__ uint32_t group_exponent(uint32_t amax_bits)
{
    int e = F == kByteInt8 ? (int)((amax_bits + 0x00ffffu) >> 23) - 6 : (int)((amax_bits + 0x1fffffu) >> 23) - 8;
    const int top = F == kByteInt8 ? 121 + 127 : 119 + 127;
    e = e < 17 ? 17 : e > top ? top : e;
    return (uint32_t)e;
}
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }
__device__ __forceinline__ float inverse_scale_of(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// Eight codes, the first in the lowest byte.
template <uint32_t F>
__device__ __forceinline__ u32x2 encode8(f32x8 v, float inv)
{
    u32x2 r;
    if constexpr (F == kByteInt8) {
        uint32_t b[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // adding 1.5 * 2^23 rounds to an integer, to nearest even, and leaves it in the low byte
            const float t = __builtin_amdgcn_fmed3f(v[k] * inv, -127.0f, 127.0f) + 12582912.0f;
            b[k] = (__float_as_uint(v[k]) & 0x7fffffffu) < 0x7f800000u ? __float_as_uint(t) : 0x80u;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t lo = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400u);
            const uint32_t hi = __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x04000c0cu);
            r[h] = lo | hi;
        }
    } else {
        float t[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float c = __builtin_amdgcn_fmed3f(v[k] * inv, -448.0f, 448.0f);
            t[k] = (__float_as_uint(v[k]) & 0x7fffffffu) < 0x7f800000u ? c : __uint_as_float(0x7fc00000u);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * h], t[4 * h + 1], 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * h + 2], t[4 * h + 3], w, true);
            r[h] = (uint32_t)w;
        }
    }
    return r;
}

// The four values of a word of codes.
template <uint32_t F>
__device__ __forceinline__ f32x4 decode4(uint32_t w, float s)
{
    f32x4 v;
    if constexpr (F == kByteInt8) {
        const float m = -128.0f * s;
        v[0] = (float)(int8_t)w * s;
        v[1] = (float)(int8_t)(w >> 8) * s;
        v[2] = (float)(int8_t)(w >> 16) * s;
        v[3] = (float)(int8_t)(w >> 24) * s;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (v[k] == m) v[k] = __uint_as_float(0x7fc00000u);   // code -128
    } else {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        v[0] = a[0] * s; v[1] = a[1] * s; v[2] = b[0] * s; v[3] = b[1] * s;
    }
    return v;
}

template <uint32_t F>
__device__ __forceinline__ f32x8 decode8(u32x2 w, float s)
{
    const f32x4 a = decode4<F>(w[0], s), b = decode4<F>(w[1], s);
    f32x8 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[k] = a[k]; v[4 + k] = b[k]; }
    return v;
}

struct ByteArgs {
    void          *x;          // the tensor: read by the store, written by the load
    uint64_t       ld;         // its row stride in elements
    uint8_t       *codes, *exps;
    uint64_t       pitch, ngroups;
    uint64_t       tail_from, tail_to;      // zero bytes behind the exponents, from the start of `codes`
    uint32_t       rows, cols;
    uint32_t       type, format, gshift;    // group = 1 << gshift
};
void launch_byte_store(const ByteArgs &a, hipStream_t st);
void launch_byte_load(const ByteArgs &a, hipStream_t st);

struct LinearGradArgs {
    const uint8_t *codes, *exps;
    uint64_t       pitch, ngroups;
    const void    *dy;
    uint64_t       ld_dy;
    void          *dw, *db;                 // db may be null
    float         *work;
    uint32_t       rows, cols, outs;
    uint32_t       type, out_type, format, gshift, accumulate;
};
uint64_t linear_grad_work(uint64_t rows, uint64_t cols, uint64_t outs, uint32_t type);
void launch_linear_grad(const LinearGradArgs &a, hipStream_t st);

struct NormArgs {
    const void    *x;                       // input, or null in a backward pass from codes
    const void    *dy;
    void          *y;                       // output, or the input's gradient
    const float   *gamma, *beta;            // either may be null: ones, zeros
    float         *dgamma, *dbeta;          // either may be null
    double        *stats;                   // [batch][groups][2]: mean, 1 / deviation
    uint8_t       *codes, *exps;            // null: no checkpoint
    uint64_t       pitch, ngroups, tail_from, tail_to;
    void          *work;
    uint64_t       batch;
    uint32_t       spatial, channels, groups, type, act, format, gshift;
    double         eps;
};
uint64_t group_norm_work(const NormArgs &a);                               // enough for either direction in any of its forms
uint64_t group_norm_forward_work(const NormArgs &a, uint32_t group);       // columns of a scale of the checkpoint, 0: none
uint64_t group_norm_grad_work(const NormArgs &a, bool params);
void launch_group_norm(const NormArgs &a, hipStream_t st);
void launch_group_norm_grad(const NormArgs &a, hipStream_t st);

}  // namespace cmpz
