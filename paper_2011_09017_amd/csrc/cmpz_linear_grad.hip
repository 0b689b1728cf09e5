// Weight gradient of a linear layer whose input is held as a byte checkpoint:
//   dW[n][k] = sum over m of dY[m][n] * X'[m][k],   db[n] = sum over m of dY[m][n].
//
// The codes are expanded to bf16 on their way into LDS, which is exact (the scales are powers of two), and the sums
// run in fp32 in the matrix units.  dY in bf16 enters as it is; fp16 and fp32 are split by truncation into two
// or three bf16 terms that add up to the value exactly, at two or three times the matrix work.
//
// Both operands are reduced along their rows, so both are read transposed from LDS.  Measured, rows x cols x outs of
// 8192 x 4096 x 4096 on random values: int8 with bf16 252 us (1.09 PFLOP/s), e4m3 226, fp16 450 and fp32 660 (two and three
// terms); 16384 x 4096 x 8192 e4m3 877 us (1.25 PFLOP/s); 8192^3 as A^T B from bf16 in memory the library reaches 1.12.
// A stage of 32 rows takes 0.98 us at 256 x 256.  Counters of 8192 x 4096 x 4096 (int8, e4m3): matrix units busy for 50 and 59 % of
// the clock cycles, LDS for 39 and 45 (a sixth of that are bank conflicts), so neither is the bound: all eight waves pass one
// barrier a stage and are in the same phase together, and the two units work in turn.  Beside them lie the expansion (int8: 12 %
// over e4m3) and 3.4 reads of the operands through eight L2 caches (340 MB, 1.35 TB/s: no bound).  Operands of zeros take 219 us:
// part of the rest is power.  fp16 could do with one product to a value (x' is an fp16 number too but in groups of extreme
// exponents), at half of its matrix work; the split is the one that needs no look at the exponents.
#include "cmpz_byte.h"

#include <cmath>
#include <type_traits>

namespace cmpz {
namespace {

typedef float    f32x16 __attribute__((ext_vector_type(16)));
typedef short    s16x4  __attribute__((ext_vector_type(4)));
typedef __bf16   bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4  __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;

constexpr uint32_t kStep = 32;                 // rows of a stage: the reduction of two matrix instructions
constexpr uint32_t kThreads = 256;             // four waves (the largest tile: eight)
constexpr uint32_t kPad = 64;                  // behind a row in LDS: the four rows of a transposed read of 32 columns lie in
                                               // different banks

template <uint32_t T> constexpr int kTerms = T == kTypeBF16 ? 1 : T == kTypeF16 ? 2 : 3;

// The high halves of two fp32 patterns: two bf16 numbers, truncated.
__device__ __forceinline__ uint32_t high_halves(float a, float b)
{
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// Sixteen codes as bf16, at a quarter of their value (`s`: a quarter of their scale), which keeps 128 * s finite.
// int8: the code -128, which stands for NaN, comes out as -128 * s; `found` collects whether there was one.
constexpr float kShrink = 0.25f;
template <uint32_t F>
__device__ __forceinline__ void expand16(u32x4 w, float s, u32x4 *lo, u32x4 *hi, uint32_t *found)
{
    const float m = -128.0f * s;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t p0, p1;
        if constexpr (F == kByteInt8) {
            const uint32_t u = w[q] ^ 0x80808080u;                        // code + 128
            *found |= (u - 0x01010101u) & ~u;                             // a byte of zero leaves its highest bit
            // exact: (code + 128) * s - 128 * s
            p0 = high_halves(__builtin_fmaf((float)(u & 0xffu), s, m), __builtin_fmaf((float)((u >> 8) & 0xffu), s, m));
            p1 = high_halves(__builtin_fmaf((float)((u >> 16) & 0xffu), s, m), __builtin_fmaf((float)(u >> 24), s, m));
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

// Eight reduction rows of a column, as a matrix operand: lane l holds column l % 32, rows 8 * (l / 32) .. + 7.
// `at`: the lane's address of row 8 * (l / 32) + (l % 16) / 4, column 16 * (l / 16 % 2) + 4 * (l % 4); a group of 16 lanes
// reads four rows of sixteen columns, which arrive transposed.
template <uint32_t PITCH>
__device__ __forceinline__ bf16x8 transposed(const uint8_t *at)
{
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * PITCH));
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

// Four neighbouring results, of which `left` exist.
__device__ __forceinline__ void put4(void *p, uint64_t i, uint32_t type, f32x4 v, uint32_t accumulate, int left)
{
    if (left == 4 && !accumulate) {
        if (type == kTypeF32) {
            __builtin_memcpy(static_cast<float *>(p) + i, &v, 16);
        } else if (type == kTypeF16) {
            const f16x4 h = __builtin_convertvector(v, f16x4);
            __builtin_memcpy(static_cast<_Float16 *>(p) + i, &h, 8);
        } else {
            const bf16x4 h = __builtin_convertvector(v, bf16x4);
            __builtin_memcpy(static_cast<__bf16 *>(p) + i, &h, 8);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < left) put(p, i + k, type, v[k], accumulate);
}

// sharers: tiles that share a range's sum of db; parts_b: its parts; few_log: for few outputs, log2 of the threads of a row
struct Plan { uint32_t tiles_n, tiles_k, splits, rows_per, sharers, parts_b, few_log; };

// Eight values of dY as they lie in memory.
template <uint32_t T> struct Raw { u32x4 w[T == kTypeF32 ? 2 : 1]; };
template <uint32_t T>
__device__ __forceinline__ f32x8 values_of(const Raw<T> &r)
{
    f32x8 v;
    if constexpr (T == kTypeF32) {
        __builtin_memcpy(&v, &r, 32);
    } else if constexpr (T == kTypeF16) {
        f16x8 h;
        __builtin_memcpy(&h, &r, 16);
        v = __builtin_convertvector(h, f32x8);
    } else {
        bf16x8 h;
        __builtin_memcpy(&h, &r, 16);
        v = __builtin_convertvector(h, f32x8);
    }
    return v;
}

// A workgroup computes TN x TK results over a range of rows, 32 rows (a stage) at a time.  WN x WK waves take FN x FK
// results of 32 x 32 each.  Two stages lie in LDS.  A stage is worked on in units: 16 of its rows, one term of dY.  While
// the matrix units work on the operands of one unit, which are in registers, a wave reads those of the next; in the last
// unit of stage t it also stores stage t + 2 over stage t (which every wave has read when it passes the one barrier
// of the stage) and loads stage t + 4 from memory.  The number of stages is even, so that the registers of the loads and
// the LDS slots alternate by a compile-time index; rows of zeros before the first fill the first two.
// SETS of two: the waves come twice, each set with LDS of its own and one half of the rows, and their sums meet at the end:
// as many waves as two workgroups have, with half of their partial sums in memory.
template <uint32_t T, uint32_t F, int FN, int FK, int WN, int WK, int SETS>
__global__ __launch_bounds__(64 * WN * WK * SETS, 2) void k_linear_grad(LinearGradArgs a, Plan p)
{
    constexpr uint32_t kWaves = WN * WK, kThreads = 64 * kWaves;          // of a set
    constexpr int TERMS = kTerms<T>;
    constexpr uint32_t ES = type_bytes(T);
    constexpr uint32_t TN = FN * 32 * WN, TK = FK * 32 * WK;
    constexpr uint32_t PY = TN * 2 + kPad, PX = TK * 2 + kPad;            // bytes of a row in LDS
    constexpr uint32_t VY = TN / 8, VX = TK / 16;                         // vectors of a row
    constexpr uint32_t YV = VY * kStep / kThreads, XV = VX * kStep >= kThreads ? VX * kStep / kThreads : 1;
    constexpr uint32_t RY = kThreads / VY, RX = kThreads / VX;            // rows between a thread's vectors
    static_assert(YV >= 1, "every thread brings a part of dY");
    // one block of LDS: two stages of dY's terms, two of x', and at the end the rows of the results
    constexpr uint32_t SY = kStep * PY, SX = kStep * PX, RW = FK * 32 + 4, RV = FK * 8;
    constexpr uint32_t kStages = 2 * TERMS * SY + 2 * SX, kRows = kWaves * 32 * RW * 4;
    __shared__ __align__(16) uint8_t s_all[SETS * (kStages > kRows ? kStages : kRows)];
    const uint32_t set = SETS > 1 ? threadIdx.x / kThreads : 0u;
    uint8_t *s_set = s_all + set * kStages;
    auto s_y = [&](int slot, int term) -> uint8_t * { return s_set + (slot * TERMS + term) * SY; };
    auto s_x = [&](int slot) -> uint8_t * { return s_set + 2 * TERMS * SY + slot * SX; };

    const uint32_t tid = threadIdx.x - set * kThreads, lane = tid & 63u, wave = tid >> 6;
    uint32_t b = blockIdx.x;
    const uint32_t tn = b % p.tiles_n; b /= p.tiles_n;
    const uint32_t tk = b % p.tiles_k, split = b / p.tiles_k;
    const uint32_t n_first = tn * TN, k0 = tk * TK;
    // a last tile of fewer than eight columns starts earlier, so that a vector of its columns fits (they are stored once)
    const uint32_t n0 = a.outs - n_first < 8 ? a.outs - 8 : n_first;
    uint32_t m_beg = split * p.rows_per, m_end = a.rows - m_beg < p.rows_per ? a.rows : m_beg + p.rows_per;
    // the first set has the odd row, and every set as many stages as that one
    const uint32_t most = SETS > 1 ? (m_end - m_beg + 1) / 2 : m_end - m_beg;
    if (SETS > 1) {
        if (set) m_beg += most;
        else m_end = m_beg + most;
    }
    const uint32_t stages = ((most + kStep - 1) / kStep + 1) & ~1u;
    const int64_t m_zero = (int64_t)m_end - (int64_t)stages * kStep;      // first row of stage 0: m_beg, or up to 64 before it

    // ---- what this thread brings from memory: YV vectors of dY and XV of codes ----
    const uint32_t ry = tid / VY, cy = (tid % VY) * 8u;
    // the vector that crosses the last column moves back into the row, here and in LDS; those behind it, and codes
    // behind the last column, read anything: their results are not stored
    const uint32_t ny = n0 + cy + 8 > a.outs ? a.outs - 8 : n0 + cy;
    const uint32_t dst_y = n0 + cy < a.outs ? ny - n0 : cy;
    const uint32_t rx = (tid / VX) & (kStep - 1u), cx = (tid % VX) * 16u; // (small tiles: several threads bring the same codes)
    const uint32_t kx = k0 + cx < a.cols ? k0 + cx : (uint32_t)a.pitch - 16u;
    const uint8_t *dy = static_cast<const uint8_t *>(a.dy);
    const uint64_t row_y = a.ld_dy * ES;
    // offsets from the first row of a stage: rows are at most 2^24 values apart
    uint32_t off_y[YV], off_x[XV], off_e[XV];
#pragma unroll
    for (uint32_t q = 0; q < YV; ++q) off_y[q] = (ry + q * RY) * (uint32_t)row_y + ny * ES;
#pragma unroll
    for (uint32_t q = 0; q < XV; ++q) {
        off_x[q] = (rx + q * RX) * (uint32_t)a.pitch + kx;
        off_e[q] = (rx + q * RX) * (uint32_t)a.ngroups + (kx >> a.gshift);
    }
    struct Fetched { Raw<T> y[YV]; u32x4 x[XV]; uint32_t e[XV]; } got[2];
    auto load = [&](Fetched &g, uint32_t s) {                             // stage 2 or later: all its rows exist
        const uint64_t m0 = (uint64_t)(m_zero + (int64_t)s * kStep);
        const uint8_t *y = dy + m0 * row_y, *x = a.codes + m0 * a.pitch, *e = a.exps + m0 * a.ngroups;
#pragma unroll
        for (uint32_t q = 0; q < YV; ++q) __builtin_memcpy(&g.y[q], y + off_y[q], sizeof(g.y[q]));
#pragma unroll
        for (uint32_t q = 0; q < XV; ++q) {
            g.x[q] = *reinterpret_cast<const u32x4 *>(x + off_x[q]);
            g.e[q] = e[off_e[q]];
        }
    };
    auto load_first = [&](Fetched &g, uint32_t s) {                       // stage 0 or 1: rows before m_beg are zero in both operands
        const int64_t m0 = m_zero + (int64_t)s * kStep;
#pragma unroll
        for (uint32_t q = 0; q < YV; ++q) {
            const int64_t m = m0 + ry + q * RY;
            g.y[q] = Raw<T>{};
            if (m >= (int64_t)m_beg) __builtin_memcpy(&g.y[q], dy + (uint64_t)m * row_y + (uint64_t)ny * ES, sizeof(g.y[q]));
        }
#pragma unroll
        for (uint32_t q = 0; q < XV; ++q) {
            const int64_t m = m0 + rx + q * RX;
            g.x[q] = u32x4{0, 0, 0, 0};
            g.e[q] = 127;
            if (m >= (int64_t)m_beg) {
                g.x[q] = *reinterpret_cast<const u32x4 *>(a.codes + (uint64_t)m * a.pitch + kx);
                g.e[q] = a.exps[(uint64_t)m * a.ngroups + (kx >> a.gshift)];
            }
        }
    };
    // into LDS; returns a word with one of the bits 0x80808080 set where a code stands for NaN
    auto store = [&](const Fetched &g, int slot) -> uint32_t {
#pragma unroll
        for (uint32_t q = 0; q < YV; ++q) {
            const uint32_t at = (ry + q * RY) * PY + dst_y * 2u;
            if constexpr (T == kTypeBF16) {
                *reinterpret_cast<u32x4 *>(s_y(slot, 0) + at) = g.y[q].w[0];
            } else {
                u32x4 t[TERMS];
                split8<T>(values_of<T>(g.y[q]), t);
#pragma unroll
                for (int k = 0; k < TERMS; ++k) *reinterpret_cast<u32x4 *>(s_y(slot, k) + at) = t[k];
            }
        }
        uint32_t found = 0;
#pragma unroll
        for (uint32_t q = 0; q < XV; ++q) {
            u32x4 lo, hi;
            expand16<F>(g.x[q], scale_of(g.e[q]) * kShrink, &lo, &hi, &found);
            uint8_t *at = s_x(slot) + (rx + q * RX) * PX + cx * 2u;
            *reinterpret_cast<u32x4 *>(at) = lo;
            *reinterpret_cast<u32x4 *>(at + 16) = hi;
        }
        return found;
    };
    auto mark_nan = [&](const Fetched &g, int slot) {
#pragma unroll 1
        for (uint32_t k = 0; k < 16u * XV; ++k) {
            const uint32_t q = k >> 4, c = k & 15u;
            uint32_t w = 0;
#pragma unroll
            for (uint32_t i = 0; i < XV; ++i)
#pragma unroll
                for (uint32_t h = 0; h < 4; ++h)
                    if (i == q && h == c >> 2) w = g.x[i][h];
            if (((w >> (8u * (c & 3u))) & 0xffu) == 0x80u)
                *reinterpret_cast<uint16_t *>(s_x(slot) + (rx + q * RX) * PX + (cx + c) * 2u) = 0x7fc0u;
        }
    };
    // the bias gradient's share of this workgroup: every stage, or those of its turn among the tiles that share it
    float sum_b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum_b[k] = 0.0f;
    uint32_t next_b = a.db && tk < p.sharers ? tk : 0xffffffffu;
    auto sum_bias = [&](const Fetched &g, uint32_t s) {
        if (s != next_b || s >= stages) return;
        next_b += p.sharers;
#pragma unroll
        for (uint32_t q = 0; q < YV; ++q) {
            const f32x8 v = values_of<T>(g.y[q]);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum_b[k] += v[k];
        }
    };

    // ---- operands and results of this wave ----
    const uint32_t wk = (wave % WK) * (FK * 32u), wn = (wave / WK) * (FN * 32u);
    const uint32_t frag_row = (lane >> 5) * 8u + ((lane & 15u) >> 2), frag_col = ((lane >> 4) & 1u) * 32u + (lane & 3u) * 8u;
    const uint32_t at_y = frag_row * PY + frag_col + wn * 2u, at_x = frag_row * PX + frag_col + wk * 2u;
    f32x16 acc[FK][FN];
#pragma unroll
    for (int i = 0; i < FK; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x16{};
    bf16x8 fy[2][FN], fx[2][FK];
    auto read_y = [&](int buffer, int slot, int term, int half) {
#pragma unroll
        for (int j = 0; j < FN; ++j) fy[buffer][j] = transposed<PY>(s_y(slot, term) + at_y + half * 16u * PY + 64u * j);
    };
    auto read_x = [&](int slot, int half) {
#pragma unroll
        for (int i = 0; i < FK; ++i) fx[half][i] = transposed<PX>(s_x(slot) + at_x + half * 16u * PX + 64u * i);
    };
    auto multiply = [&](int half, int buffer) {
#pragma unroll
        for (int i = 0; i < FK; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[half][i], fy[buffer][j], acc[i][j], 0, 0, 0);
    };

    // bf16: one region of the last half of stage t and the first of stage t + 1, all of whose operands it reads, so that
    // the expansion can lie between any of its products.  With several terms the split is spread better by the
    // units, one after the other; the barrier stands before the last.
    auto step = [&](auto parity, auto more, auto last, uint32_t t) {
        constexpr int P = decltype(parity)::value;
        constexpr int UNITS = 2 * TERMS;                                  // unit u: half u / TERMS, term u % TERMS
        uint32_t found = 0;
        // behind the barrier every wave has the operands of stage t in registers, and stage t + 1 is stored
        if constexpr (TERMS == 1) {
            __syncthreads();
            read_y(0, P ^ 1, 0, 0);
            read_x(P ^ 1, 0);
            found = store(got[P], P);
            multiply(1, 1);
            read_y(1, P ^ 1, 0, 1);
            read_x(P ^ 1, 1);
            if constexpr (!decltype(last)::value) multiply(0, 0);
#pragma unroll
            for (int k = 0; k < 2 * FN * FK; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);        // a matrix instruction
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);        // LDS reads
                __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);        // vector arithmetic
                if (k & 1) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);   // an LDS write
            }
        } else {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int next = (u + 1) % UNITS, slot = u + 1 < UNITS ? P : P ^ 1;
                if (u + 1 == UNITS) __syncthreads();
                read_y(next & 1, slot, next % TERMS, next / TERMS);
                if (next % TERMS == 0) read_x(slot, next / TERMS);
                if (u + 1 == UNITS) found = store(got[P], P);
                multiply(u / TERMS, u & 1);
#pragma unroll
                for (int k = 0; k < FN * FK; ++k) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (F == kByteInt8 && (found & 0x80808080u)) mark_nan(got[P], P);
        sum_bias(got[P], t + 2);
        if constexpr (decltype(more)::value) load(got[P], t + 4);
    };

    if (stages > 0) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            load_first(got[s], s);
            if (store(got[s], s) & 0x80808080u) mark_nan(got[s], s);
            sum_bias(got[s], s);
            if (stages > 2) load(got[s], s + 2);
        }
        __syncthreads();
        read_y(0, 0, 0, 0);
        read_x(0, 0);
        if constexpr (TERMS == 1) {                                       // stage 0 but its last unit
            multiply(0, 0);
            read_y(1, 0, 0, 1);
            read_x(0, 1);
        }
    }
    // The loads of the loop are unconditional: behind a branch the wait for a stage would be one for all loads under way.
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    const std::true_type yes;
    const std::false_type no;
    uint32_t t = 0;
#pragma unroll 1
    for (; t + 4 < stages; t += 2) {
        step(even, yes, no, t);
        step(odd, yes, no, t + 1);
    }
    if (t + 2 < stages) {
        step(even, no, no, t);
        step(odd, no, no, t + 1);
        t += 2;
    }
    if (t < stages) {
        step(even, no, no, t);
        step(odd, no, yes, t + 1);
    }

    // ---- results: a lane holds row n = lane % 32 of dW and four times four consecutive k of every 32 x 32; 32 rows at a time
    // go through LDS, so that a row is stored by neighbouring lanes ----
    __syncthreads();
    float *rows = reinterpret_cast<float *>(s_all) + wave * (32u * RW);   // RW floats a row, RV vectors of four in it
    constexpr uint32_t kOther = kWaves * 32u * RW;                        // from a wave's rows to those of its like in the second set
    void *out = p.splits > 1 ? static_cast<void *>(a.work + (uint64_t)split * a.outs * a.cols) : a.dw;
    const uint32_t out_type = p.splits > 1 ? kTypeF32 : a.out_type, accumulate = p.splits > 1 ? 0u : a.accumulate;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
#pragma unroll
        for (int i = 0; i < FK; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 *>(rows + set * kOther + (lane & 31u) * RW + 32u * i + 8u * q + (lane >> 5) * 4u) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]} * (1.0f / kShrink);
        const uint32_t n_row = n0 + wn + 32u * j;
        if (SETS > 1) __syncthreads();
#pragma unroll 1
        for (uint32_t v = lane + 64u * set; v < 32u * RV; v += 64u * SETS) {      // the sets store in turn
            const uint32_t r = v / RV, c = (v % RV) * 4u, n = n_row + r, k = k0 + wk + c;
            f32x4 t = *reinterpret_cast<const f32x4 *>(rows + r * RW + c);
            if (SETS > 1) t += *reinterpret_cast<const f32x4 *>(rows + kOther + r * RW + c);
            if (n >= n_first && n < a.outs && k < a.cols)
                put4(out, (uint64_t)n * a.cols + k, out_type, t, accumulate, a.cols - k < 4 ? (int)(a.cols - k) : 4);
        }
        if (SETS > 1) __syncthreads();
    }
    if (a.db && tk < p.sharers) {                                         // columns of the threads with the same vector
        float *s = reinterpret_cast<float *>(s_all);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) s[threadIdx.x * 8u + k] = sum_b[k];
        __syncthreads();
        float *part_b = a.work + (p.splits > 1 ? (uint64_t)p.splits * a.outs * a.cols : 0) + (uint64_t)(split * p.sharers + tk) * a.outs;
        static_assert(SETS * kThreads >= TN, "a thread for every column");
        if (threadIdx.x < TN) {                                           // a column each: vector threadIdx.x / 8 of the row
            const uint32_t from = n0 + (threadIdx.x & ~7u), n = (from + 8 > a.outs ? a.outs - 8 : from) + (threadIdx.x & 7u);
            // a vector moved back shares columns with the one before it, a last tile that starts earlier with the tile before
            if (from < a.outs && n >= from && n >= n_first) {
                float v = 0.0f;
#pragma unroll 8
                for (uint32_t r = 0; r < SETS * kThreads / VY; ++r) v += s[r * TN + threadIdx.x];
                if (p.parts_b > 1) part_b[n] = v;
                else put(a.db, n, a.out_type, v, a.accumulate);
            }
        }
    }
}

// Fewer than eight outputs (a gate, a small head), or no columns at all: too narrow for the matrix tiles.  A thread takes
// four columns and NO outputs of every parts-th row of a range, in fp32; a row takes 2^few_log threads, and the parts meet in LDS.
// Loads are unconditional (what does not exist repeats its neighbour), so that those of four rows are under way at once:
// 8192 x 4096 x 1 bf16 with db 20 us, 500000 x 8 x 2 fp32 28 (with a thread to four columns of all rows of a range, and loads
// behind branches, 54 and 356); latency and the join, the codes alone are 6.6 us of reading.
template <uint32_t T, uint32_t F, int NO>
__global__ __launch_bounds__(kThreads) void k_linear_grad_few(LinearGradArgs a, Plan p)
{
    typedef typename ElemOf<T>::type E;
    __shared__ f32x4 s[kThreads];
    uint32_t b = blockIdx.x;
    const uint32_t tn = b % p.tiles_n; b /= p.tiles_n;
    const uint32_t tk = b % p.tiles_k, split = b / p.tiles_k;
    const uint32_t wide = 1u << p.few_log, parts = kThreads >> p.few_log, slot = threadIdx.x & (wide - 1u), part = threadIdx.x >> p.few_log;
    const uint32_t n0 = tn * NO, k0 = (tk * wide + slot) * 4u;
    const uint32_t m_beg = split * p.rows_per, m_end = a.rows - m_beg < p.rows_per ? a.rows : m_beg + p.rows_per;
    const int n = a.outs - n0 < NO ? (int)(a.outs - n0) : NO;
    const bool mine = k0 < a.cols && part == 0;
    const uint32_t k_read = k0 < a.cols ? k0 : 0u;
    f32x4 acc[NO];
    float sum[NO];
#pragma unroll
    for (int j = 0; j < NO; ++j) {
        acc[j] = f32x4{0, 0, 0, 0};
        sum[j] = 0.0f;
    }
    const E *dy = static_cast<const E *>(a.dy) + n0;
    auto values = [&](uint32_t m, float (&y)[NO]) {
#pragma unroll
        for (int j = 0; j < NO; ++j) {
            y[j] = (float)dy[(uint64_t)m * a.ld_dy + (j < n ? j : n - 1)];
            sum[j] += y[j];
        }
    };
    if (a.cols) {
#pragma unroll 4
        for (uint32_t m = m_beg + part; m < m_end; m += parts) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(a.codes + (uint64_t)m * a.pitch + k_read);
            const uint32_t e = a.exps[(uint64_t)m * a.ngroups + (k_read >> a.gshift)];
            float y[NO];
            values(m, y);
            const f32x4 x = decode4<F>(w, scale_of(e));
#pragma unroll
            for (int j = 0; j < NO; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[j][q] = __builtin_fmaf(y[j], x[q], acc[j][q]);
        }
    } else {
#pragma unroll 4
        for (uint32_t m = m_beg + part; m < m_end; m += parts) {
            float y[NO];
            values(m, y);
        }
    }
    void *out = p.splits > 1 ? static_cast<void *>(a.work + (uint64_t)split * a.outs * a.cols) : a.dw;
    float *part_b = a.work + (uint64_t)p.splits * a.outs * a.cols + (uint64_t)split * a.outs;
    const bool with_db = a.db && tk == 0;                                 // uniform
#pragma unroll
    for (int j = 0; j < NO; ++j) {
        if (j >= n) break;
        if (parts > 1 && a.cols) {
            __syncthreads();
            s[threadIdx.x] = acc[j];
            __syncthreads();
            if (part == 0) {
#pragma unroll 4
                for (uint32_t r = 1; r < parts; ++r) acc[j] += s[r * wide + slot];
            }
        }
        if (mine)
            put4(out, (uint64_t)(n0 + j) * a.cols + k0, p.splits > 1 ? kTypeF32 : a.out_type, acc[j], p.splits > 1 ? 0u : a.accumulate,
                 a.cols - k0 < 4 ? (int)(a.cols - k0) : 4);
    }
    if (with_db) {
        float *sb = reinterpret_cast<float *>(s);
#pragma unroll
        for (int j = 0; j < NO; ++j) {
            if (j >= n) break;
            if (parts > 1) {
                __syncthreads();
                if (slot == 0) sb[part] = sum[j];
                __syncthreads();
            }
            if (threadIdx.x == 0) {
#pragma unroll 8
                for (uint32_t r = 1; r < parts; ++r) sum[j] += sb[r];
                if (p.splits > 1) part_b[n0 + j] = sum[j];
                else put(a.db, n0 + j, a.out_type, sum[j], a.accumulate);
            }
        }
    }
}

// Joins the partial sums of the ranges of rows: `count` rows of `n` values each to one row of results, dW's and db's in one
// launch.  A thread takes four values of every parts-th row, then the sums of the parts are added up in order: with
// many ranges and few results there would be too few loads in flight otherwise (251 ranges of 64 x 256: 7.0 us with 16 parts, 5.4 with 32).
struct JoinJob { const float *w; void *out; uint64_t n; uint32_t count, parts_log, blocks; };

__global__ __launch_bounds__(kThreads) void k_linear_grad_join(JoinJob a, JoinJob b, uint32_t type, uint32_t accumulate)
{
    __shared__ f32x4 s[kThreads];
    const bool first = blockIdx.x < a.blocks;
    const JoinJob j = first ? a : b;
    const uint32_t block = first ? blockIdx.x : blockIdx.x - a.blocks, parts = 1u << j.parts_log;
    const uint32_t slots = kThreads >> j.parts_log, slot = threadIdx.x & (slots - 1u), part = threadIdx.x / slots;
    const uint64_t i = ((uint64_t)block * slots + slot) * 4u;
    const int left = i < j.n ? (j.n - i < 4 ? (int)(j.n - i) : 4) : 0;
    f32x4 t = {0, 0, 0, 0};
    if (left == 4) {
#pragma unroll 4
        for (uint32_t k = part; k < j.count; k += parts) {
            f32x4 v;
            __builtin_memcpy(&v, j.w + k * j.n + i, 16);
            t += v;
        }
    } else {
        for (uint32_t k = part; k < j.count; k += parts)
            for (int q = 0; q < 4; ++q)
                if (q < left) t[q] += j.w[k * j.n + i + q];
    }
    if (parts > 1) {
        s[threadIdx.x] = t;
        __syncthreads();
        if (part) return;
        for (uint32_t k = 1; k < parts; ++k) t += s[threadIdx.x + k * slots];
    }
    if (left > 0) put4(j.out, i, type, t, accumulate, left);
}

JoinJob join_job(const float *w, uint32_t count, uint64_t n, void *out)
{
    JoinJob j{w, out, n, count, count >= 128 ? 5u : count >= 32 ? 4u : count >= 8 ? 2u : 0u, 0};
    const uint32_t values = 4u * (kThreads >> j.parts_log);
    j.blocks = (uint32_t)((n + values - 1) / values);
    return j;
}

// Tiles of dW that a workgroup may take, its sets of waves, how many such workgroups a CU holds (with three terms of dY one
// of any tile: the smallest takes 96 KB of LDS then), and what a stage (32 rows
// of each set) takes with w of them on it, in ns, for t terms: a0 + a1 * t + (b0 + b1 * t) * w.  Fitted to 8192 and 16384 rows, all
// CUs busy (ns measured / fitted for bf16, fp16, fp32): 256 x 256: 980 / 975, 1740 / 1760, 2550 / 2545; 128 x 128: 707 / 707, 1205 /
// 1199, 1692 / 1691; 64 x 256: 884 / 882, 1210 / 1254, 1631 / 1626; 64 x 64, two of them: 801 / 800, 1120 / 1120, one: 564 / 560, fp32
// 818 / 820.  With one set, two workgroups to a CU, the middle two take 4 to 15 % longer and leave twice the partial sums
// (8192 x 1024 x 1024 bf16: 42 us where this takes 38; 200704 x 256 x 64 fp32: 43 and 37).
struct Tile { uint32_t n, k, sets, resident; double a0, a1, b0, b1; };
constexpr Tile kTiles[] = {{256, 256, 1, 1, 190, 785, 0, 0}, {128, 128, 2, 1, 215, 492, 0, 0}, {64, 256, 2, 1, 510, 372, 0, 0},
                           {64, 64, 2, 2, 380, -60, 50, 190}};
constexpr int kTileCount = 4, kFewOutputs = kTileCount;

uint32_t resident_of(const Tile &t, uint32_t type) { return type == kTypeF32 ? 1u : t.resident; }
bool few_outputs(uint64_t cols, uint64_t outs) { return outs < 8 || cols == 0; }

// Time of the launches in ns, roughly: what the choice between tiles and numbers of ranges goes by.
double cost_of(const Tile &t, uint64_t rows, uint64_t cols, uint64_t outs, uint32_t type, uint64_t splits)
{
    const double terms = type == kTypeBF16 ? 1 : type == kTypeF16 ? 2 : 3;
    const double tiles = (double)((outs + t.n - 1) / t.n) * (double)((cols + t.k - 1) / t.k);
    const double per_cu = std::ceil(tiles * (double)splits / 256.0);
    const double resident = resident_of(t, type), full = std::floor(per_cu / resident), rest = per_cu - full * resident;
    auto stage = [&](double w) { return w > 0 ? t.a0 + t.a1 * terms + (t.b0 + t.b1 * terms) * w : 0.0; };
    const double stages = std::ceil((double)rows / kStep / (double)(splits * t.sets)) + 3;        // and what a workgroup begins with
    const double body = stages * (full * stage(resident) + stage(rest));
    const double memory = (double)rows * ((double)outs * type_bytes(type) + (double)cols) / 5000.0;    // at 5 TB/s
    const double results = (double)t.n * t.k * (splits > 1 ? 4 : 2) * per_cu / 40.0;                   // stores at 40 B/ns per CU
    return (body > memory ? body : memory) + results + (splits > 1 ? 3000.0 + (double)splits * outs * cols * 4.0 / 5000.0 : 0.0);
}

struct Choice { int tile; Plan plan; };

Choice choose(uint64_t rows, uint64_t cols, uint64_t outs, uint32_t type)
{
    const uint64_t steps = (rows + kStep - 1) / kStep;
    Choice c{kFewOutputs, {}};
    uint64_t splits = 1;
    uint32_t tile_n = 8, tile_k = 4;
    c.plan.few_log = 0;
    if (few_outputs(cols, outs)) {
        for (; tile_k < 256 && tile_k < cols; tile_k *= 2) ++c.plan.few_log;
        const uint64_t tiles = ((outs + 7) / 8) * ((cols + tile_k - 1) / tile_k + (cols == 0));
        splits = tiles && tiles < 1024 ? 1024 / tiles : 1;
        if (splits > (steps + 1) / 2) splits = (steps + 1) / 2;           // no fewer than two stages each
    } else {
        double best = 0;
        for (int i = 0; i < kTileCount; ++i) {
            const uint64_t tiles = ((outs + kTiles[i].n - 1) / kTiles[i].n) * ((cols + kTiles[i].k - 1) / kTiles[i].k);
            if (tiles > (1u << 22)) continue;                             // threads of a launch are counted with 32 bits
            // one range, and as many as fill a quarter of the CUs, half of them, all of them once and, where two fit, twice
            for (uint64_t fill : {0ull, 64ull, 128ull, 256ull, 512ull}) {
                uint64_t k = fill / tiles;
                if (fill && (k < 2 || fill > 256ull * resident_of(kTiles[i], type))) continue;
                if (k > steps / (4 * kTiles[i].sets)) k = steps / (4 * kTiles[i].sets);   // no fewer than four stages each
                if (k < 1) k = 1;
                const double t = cost_of(kTiles[i], rows, cols, outs, type, k);
                if (best == 0 || t < best) { best = t; c.tile = i; splits = k; }
            }
        }
        tile_n = kTiles[c.tile].n;
        tile_k = kTiles[c.tile].k;
    }
    if (splits < 1) splits = 1;
    Plan &p = c.plan;
    p.tiles_n = outs ? (uint32_t)((outs + tile_n - 1) / tile_n) : 1;
    p.tiles_k = cols ? (uint32_t)((cols + tile_k - 1) / tile_k) : 1;       // without columns the bias gradient is left
    p.rows_per = steps ? (uint32_t)((steps + splits - 1) / splits * kStep) : kStep;
    p.splits = rows ? (uint32_t)((rows + p.rows_per - 1) / p.rows_per) : 1;
    // Where no ranges have to be joined, a short sum of db is left to the first tile: adding up a stage takes about 40 ns there,
    // a launch to join the tiles' shares 4 us (256 x 512 x 1000 fp32 with db: 16.1 us with it, 12.3 without).
    p.sharers = c.tile == kFewOutputs || (p.splits == 1 && steps <= 64) ? 1 : p.tiles_k;
    p.parts_b = p.splits * p.sharers;
    return c;
}

template <uint32_t T, uint32_t F>
void launch_as(const LinearGradArgs &a, const Choice &c, hipStream_t st)
{
    const Plan &p = c.plan;
    const dim3 grid(p.tiles_n * p.tiles_k * p.splits);
    switch (c.tile) {
    case 0: hipLaunchKernelGGL((k_linear_grad<T, F, 4, 2, 2, 4, 1>), grid, dim3(512), 0, st, a, p); break;
    case 1: hipLaunchKernelGGL((k_linear_grad<T, F, 2, 2, 2, 2, 2>), grid, dim3(512), 0, st, a, p); break;
    case 2: hipLaunchKernelGGL((k_linear_grad<T, F, 2, 2, 1, 4, 2>), grid, dim3(512), 0, st, a, p); break;
    case 3: hipLaunchKernelGGL((k_linear_grad<T, F, 1, 1, 2, 2, 2>), grid, dim3(512), 0, st, a, p); break;
    default:
        if (a.outs == 1) hipLaunchKernelGGL((k_linear_grad_few<T, F, 1>), grid, dim3(kThreads), 0, st, a, p);
        else if (a.outs == 2) hipLaunchKernelGGL((k_linear_grad_few<T, F, 2>), grid, dim3(kThreads), 0, st, a, p);
        else if (a.outs <= 4) hipLaunchKernelGGL((k_linear_grad_few<T, F, 4>), grid, dim3(kThreads), 0, st, a, p);
        else hipLaunchKernelGGL((k_linear_grad_few<T, F, 8>), grid, dim3(kThreads), 0, st, a, p);
    }
}

template <uint32_t T>
void launch_of(const LinearGradArgs &a, const Choice &c, hipStream_t st)
{
    if (a.format == kByteInt8) launch_as<T, kByteInt8>(a, c, st);
    else launch_as<T, kByteE4M3>(a, c, st);
}

}  // namespace

uint64_t linear_grad_work(uint64_t rows, uint64_t cols, uint64_t outs, uint32_t type)
{
    const Plan p = choose(rows, cols, outs, type).plan;
    return 4ull * ((p.splits > 1 ? p.splits * outs * cols : 0) + (p.parts_b > 1 ? p.parts_b * outs : 0));
}

void launch_linear_grad(const LinearGradArgs &a, hipStream_t st)
{
    const Choice c = choose(a.rows, a.cols, a.outs, a.type);
    const Plan &p = c.plan;
    if (a.type == kTypeF32) launch_of<kTypeF32>(a, c, st);
    else if (a.type == kTypeF16) launch_of<kTypeF16>(a, c, st);
    else launch_of<kTypeBF16>(a, c, st);
    const uint64_t values = (uint64_t)a.outs * a.cols;
    const JoinJob none{};
    const JoinJob w = p.splits > 1 && values ? join_job(a.work, p.splits, values, a.dw) : none;
    const JoinJob b = a.db && p.parts_b > 1 ? join_job(a.work + (p.splits > 1 ? p.splits * values : 0), p.parts_b, a.outs, a.db) : none;
    if (w.blocks + b.blocks)
        hipLaunchKernelGGL(k_linear_grad_join, dim3(w.blocks + b.blocks), dim3(kThreads), 0, st, w, b, a.out_type, a.accumulate);
}

}  // namespace cmpz
