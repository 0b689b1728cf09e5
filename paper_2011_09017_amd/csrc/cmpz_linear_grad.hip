// Weight gradient of a linear layer whose input is held as a byte checkpoint:
//   dW[n][k] = sum over m of dY[m][n] * X'[m][k],   db[n] = sum over m of dY[m][n].
//
// The codes are expanded to bf16 on their way into LDS, which is exact (the scales are powers of two), and the sums
// run in fp32 in the matrix units.  dY in bf16 enters as it is; fp16 and fp32 are split by truncation into two
// or three bf16 terms that add up to the value exactly, at two or three times the matrix work.
#include "cmpz_byte.h"

namespace cmpz {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;

constexpr int kTile = 128, kStep = 32, kThreads = 256;
constexpr int kRow = kTile * 2 + 32;          // bytes of a row in LDS: four rows of a transposed read lie in different banks

template <uint32_t T> constexpr int kTerms = T == kTypeBF16 ? 1 : T == kTypeF16 ? 2 : 3;

// The high halves of two fp32 patterns: two bf16 numbers, truncated.
__device__ __forceinline__ uint32_t high_halves(float a, float b)
{
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// Sixteen codes as bf16.
template <uint32_t F>
__device__ __forceinline__ void expand16(u32x4 w, float s, u32x4 *lo, u32x4 *hi)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t p0, p1;
        if constexpr (F == kByteInt8) {
            const f32x4 v = decode4<kByteInt8>(w[q], s);
            p0 = high_halves(v[0], v[1]);
            p1 = high_halves(v[2], v[3]);
        } else {
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[q], s, false);
            const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[q], s, true);
            __builtin_memcpy(&p0, &a, 4);
            __builtin_memcpy(&p1, &b, 4);
        }
        u32x4 &o = q < 2 ? *lo : *hi;
        o[2 * (q & 1)] = p0;
        o[2 * (q & 1) + 1] = p1;
    }
}

// Eight values as the terms of their split: term t of all eight in out[t].
template <uint32_t T>
__device__ __forceinline__ void split8(f32x8 v, u32x4 *out)
{
#pragma unroll
    for (int t = 0; t < kTerms<T>; ++t) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            out[t][h] = high_halves(v[2 * h], v[2 * h + 1]);
            if (t + 1 < kTerms<T>) {
#pragma unroll
                for (int q = 2 * h; q < 2 * h + 2; ++q) {
                    const float top = __uint_as_float(__float_as_uint(v[q]) & 0xffff0000u);
                    // an infinity is all in its first term
                    v[q] = fabsf(v[q]) == __builtin_inff() ? 0.0f : v[q] - top;
                }
            }
        }
    }
}

// Eight reduction rows of a column, as a matrix operand: lane l holds column l % 16, rows 8 * (l / 16) .. + 7.
// `at`: the lane's address of row 8 * (l / 16) + (l % 16) / 4, column 4 * (l % 4); a group of 16 lanes reads four rows of
// sixteen columns, which arrive transposed.
__device__ __forceinline__ bf16x8 transposed(const uint8_t *at)
{
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * kRow));
    bf16x8 r;
    __builtin_memcpy(&r, &a, 8);
    __builtin_memcpy(reinterpret_cast<char *>(&r) + 8, &b, 8);
    return r;
}

__device__ __forceinline__ void put(void *p, uint64_t i, uint32_t type, float v, uint32_t accumulate)
{
    if (type == kTypeF32) {
        float *q = static_cast<float *>(p) + i;
        *q = accumulate ? *q + v : v;
    } else if (type == kTypeF16) {
        _Float16 *q = static_cast<_Float16 *>(p) + i;
        *q = (_Float16)(accumulate ? (float)*q + v : v);
    } else {
        __bf16 *q = static_cast<__bf16 *>(p) + i;
        *q = (__bf16)(accumulate ? (float)*q + v : v);
    }
}

struct Plan { uint32_t tiles_n, tiles_k, splits, rows_per; };

template <uint32_t T, uint32_t F>
__global__ __launch_bounds__(kThreads) void k_linear_grad(LinearGradArgs a, Plan p)
{
    typedef typename ElemOf<T>::type E;
    constexpr int TERMS = kTerms<T>;
    __shared__ __align__(16) uint8_t s_y[TERMS][kStep * kRow];
    __shared__ __align__(16) uint8_t s_x[kStep * kRow];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    uint32_t b = blockIdx.x;
    const uint32_t tn = b % p.tiles_n; b /= p.tiles_n;
    const uint32_t tk = b % p.tiles_k, split = b / p.tiles_k;
    const uint32_t n0 = tn * kTile, k0 = tk * kTile;
    const uint32_t m_beg = split * p.rows_per;
    const uint32_t m_end = a.rows - m_beg < p.rows_per ? a.rows : m_beg + p.rows_per;
    const bool with_db = a.db && tk == 0;

    f32x4 acc[4][4], accb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        accb[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    }
    const uint32_t wk = (wave & 1u) * 64u, wn = (wave >> 1) * 64u;
    const uint32_t frag = ((lane >> 4) * 8u + ((lane & 15u) >> 2)) * kRow + (lane & 3u) * 8u;
    bf16x8 ones;
#pragma unroll
    for (int k = 0; k < 8; ++k) ones[k] = (__bf16)1.0f;

    for (uint32_t m0 = m_beg; m0 < m_end; m0 += kStep) {
        // dY: rows of 16 vectors of eight; codes: rows of eight times sixteen
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t r = (tid >> 4) + 16u * q, c = (tid & 15u) * 8u, m = m0 + r;
            const int n = m < m_end && n0 + c < a.outs ? (int)(a.outs - n0 - c) : 0;
            const E *src = static_cast<const E *>(a.dy) + (n > 0 ? (uint64_t)m * a.ld_dy + n0 + c : 0);
            u32x4 t[TERMS];
            split8<T>(load8<T>(src, n), t);
#pragma unroll
            for (int k = 0; k < TERMS; ++k) *reinterpret_cast<u32x4 *>(&s_y[k][r * kRow + c * 2u]) = t[k];
        }
        {
            const uint32_t r = tid >> 3, c = (tid & 7u) * 16u, m = m0 + r;
            u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
            if (m < m_end && k0 + c < a.cols) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(a.codes + (uint64_t)m * a.pitch + k0 + c);
                expand16<F>(w, scale_of(a.exps[(uint64_t)m * a.ngroups + ((k0 + c) >> a.gshift)]), &lo, &hi);
            }
            *reinterpret_cast<u32x4 *>(&s_x[r * kRow + c * 2u]) = lo;
            *reinterpret_cast<u32x4 *>(&s_x[r * kRow + c * 2u + 16u]) = hi;
        }
        __syncthreads();
        bf16x8 fx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) fx[i] = transposed(s_x + frag + (wk + 16u * i) * 2u);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 fy = transposed(s_y[t] + frag + (wn + 16u * j) * 2u);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[i], fy, acc[i][j], 0, 0, 0);
                if (with_db) accb[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fy, accb[j], 0, 0, 0);
            }
        }
        __syncthreads();
    }

    // lane: output row n = lane % 16, four consecutive k
    float *part = p.splits > 1 ? a.work + (uint64_t)split * a.outs * a.cols : nullptr;
    float *part_b = p.splits > 1 ? a.work + (uint64_t)p.splits * a.outs * a.cols + (uint64_t)split * a.outs : nullptr;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t n = n0 + wn + 16u * j + (lane & 15u);
        if (n >= a.outs) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t k = k0 + wk + 16u * i + (lane >> 4) * 4u;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (k + q >= a.cols) continue;
                if (part) part[(uint64_t)n * a.cols + k + q] = acc[i][j][q];
                else put(a.dw, (uint64_t)n * a.cols + k + q, a.out_type, acc[i][j][q], a.accumulate);
            }
        }
        if (with_db && wk == 0 && lane < 16u) {
            if (part) part_b[n] = accb[j][0];
            else put(a.db, n, a.out_type, accb[j][0], a.accumulate);
        }
    }
}

// Joins the partial sums of the ranges of rows, in their order.
__global__ __launch_bounds__(kThreads) void k_linear_grad_join(LinearGradArgs a, uint32_t splits, uint64_t values)
{
    const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i < values) {
        float s = 0.0f;
        for (uint32_t k = 0; k < splits; ++k) s += a.work[(uint64_t)k * values + i];
        put(a.dw, i, a.out_type, s, a.accumulate);
    } else if (a.db && i - values < a.outs) {
        float s = 0.0f;
        for (uint32_t k = 0; k < splits; ++k) s += a.work[(uint64_t)splits * values + (uint64_t)k * a.outs + (i - values)];
        put(a.db, i - values, a.out_type, s, a.accumulate);
    }
}

Plan make_plan(uint64_t rows, uint64_t cols, uint64_t outs)
{
    Plan p;
    p.tiles_n = outs ? (uint32_t)((outs + kTile - 1) / kTile) : 1;
    p.tiles_k = cols ? (uint32_t)((cols + kTile - 1) / kTile) : 1;         // without columns the bias gradient is left
    const uint64_t tiles = (uint64_t)p.tiles_n * p.tiles_k;
    uint64_t splits = tiles >= 512 ? 1 : 512 / tiles;
    const uint64_t steps = (rows + kStep - 1) / kStep;
    if (splits > (steps + 7) / 8) splits = (steps + 7) / 8;                // no fewer than eight steps each
    if (splits < 1) splits = 1;
    p.rows_per = (uint32_t)((steps + splits - 1) / splits * kStep);
    if (p.rows_per == 0) p.rows_per = kStep;
    p.splits = (uint32_t)((rows + p.rows_per - 1) / p.rows_per);
    if (p.splits < 1) p.splits = 1;
    return p;
}

template <uint32_t T>
void launch_as(const LinearGradArgs &a, const Plan &p, hipStream_t st)
{
    const dim3 grid(p.tiles_n * p.tiles_k * p.splits);
    if (a.format == kByteInt8) hipLaunchKernelGGL((k_linear_grad<T, kByteInt8>), grid, dim3(kThreads), 0, st, a, p);
    else hipLaunchKernelGGL((k_linear_grad<T, kByteE4M3>), grid, dim3(kThreads), 0, st, a, p);
}

}  // namespace

uint64_t linear_grad_work(uint64_t rows, uint64_t cols, uint64_t outs, uint32_t type)
{
    const Plan p = make_plan(rows, cols, outs);
    return p.splits > 1 ? 4ull * p.splits * (outs * cols + outs) : 0;
}

void launch_linear_grad(const LinearGradArgs &a, hipStream_t st)
{
    const Plan p = make_plan(a.rows, a.cols, a.outs);
    if (a.type == kTypeF32) launch_as<kTypeF32>(a, p, st);
    else if (a.type == kTypeF16) launch_as<kTypeF16>(a, p, st);
    else launch_as<kTypeBF16>(a, p, st);
    if (p.splits > 1) {
        const uint64_t values = (uint64_t)a.outs * a.cols;
        hipLaunchKernelGGL(k_linear_grad_join, dim3((uint32_t)((values + a.outs + kThreads - 1) / kThreads)), dim3(kThreads),
                           0, st, a, p.splits, values);
    }
}

}  // namespace cmpz
