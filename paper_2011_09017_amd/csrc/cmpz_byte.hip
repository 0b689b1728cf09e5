// Storing and loading byte checkpoints: streaming kernels, bound by memory (bf16: 3.02 B per value in either
// direction with groups of 64; fp32: 5.02).
//
// A thread takes 16 consecutive columns of a row: 128-bit accesses on both sides, and the group's largest
// magnitude needs two, four or eight neighbouring lanes (DPP, no LDS).  Rows are dealt to threads in units of whole
// groups, so that a group never crosses a wave.  Measured (a copy of 1 GiB reaches 5.16 TB/s): bf16 8192 x 8192
// stored in 41.5 us (4.9 TB/s) and loaded in 32.6 (both tensors then fit the memory-side cache), fp32 387200 x 96 in
// 35 to 38 us and 28.5; one row of 4096 in 2.0 and 1.8 us.
#include "cmpz_byte.h"

namespace cmpz {
namespace {

constexpr int kThreads = 256;

template <uint32_t T, uint32_t F>
__global__ __launch_bounds__(kThreads) void k_byte_store(ByteArgs a, uint64_t row0, uint32_t units, uint32_t steps,
                                                         FastDiv div_units)
{
    typedef typename ElemOf<T>::type E;
    const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t r = div_units.div(at), c = (at - r * units) * 16u;
    const uint64_t row = row0 + r;
    const bool in = row < a.rows && c < a.cols;
    const int n = in ? (int)(a.cols - c) : 0;                             // columns that exist from c on
    const E *p = static_cast<const E *>(a.x) + (in ? row * a.ld + c : 0);
    const f32x8 v0 = load8<T>(p, n), v1 = load8<T>(p + 8, n - 8);
    const uint32_t e = group_exponent<F>(lanes_max(amax8(v1, amax8(v0, 0u)), steps));
    if (blockIdx.x == 0 && row0 == 0 && threadIdx.x < a.tail_to - a.tail_from) a.codes[a.tail_from + threadIdx.x] = 0;
    if (!in) return;
    const float inv = inverse_scale_of(e);
    const u32x2 lo = encode8<F>(v0, inv), hi = encode8<F>(v1, inv);       // columns that do not exist: zeros
    u32x4 w = {lo[0], lo[1], hi[0], hi[1]};
    *reinterpret_cast<u32x4 *>(a.codes + row * a.pitch + c) = w;
    if ((c & ((1u << a.gshift) - 1u)) == 0) a.exps[row * a.ngroups + (c >> a.gshift)] = (uint8_t)e;
}

// Values beyond the output type's largest finite value (fp16 only: a code may round up past 65504) become that value.
template <uint32_t T, uint32_t F>
__global__ __launch_bounds__(kThreads) void k_byte_load(ByteArgs a, uint64_t row0, uint32_t units, FastDiv div_units)
{
    typedef typename ElemOf<T>::type E;
    const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t r = div_units.div(at), c = (at - r * units) * 16u;
    const uint64_t row = row0 + r;
    if (row >= a.rows) return;
    const u32x4 w = *reinterpret_cast<const u32x4 *>(a.codes + row * a.pitch + c);
    const float s = scale_of(a.exps[row * a.ngroups + (c >> a.gshift)]);
    f32x8 v0 = decode8<F>(u32x2{w[0], w[1]}, s), v1 = decode8<F>(u32x2{w[2], w[3]}, s);
    if constexpr (T == kTypeF16) {
        auto held = [](float f) { return fabsf(f) > 65504.0f ? copysignf(65504.0f, f) : f; };   // NaN stays
#pragma unroll
        for (int k = 0; k < 8; ++k) { v0[k] = held(v0[k]); v1[k] = held(v1[k]); }
    }
    const int n = (int)(a.cols - c);
    E *p = static_cast<E *>(a.x) + row * a.ld + c;
    store8<T>(p, v0, n);
    store8<T>(p + 8, v1, n - 8);
}

// fp32: four codes a thread, so that neighbouring lanes store neighbouring 16 bytes (with sixteen codes a lane's four
// stores lie 64 bytes apart from the next lane's: 52 us for 387200 x 96 where this takes 28); four of them per thread.
template <uint32_t F>
__global__ __launch_bounds__(kThreads) void k_byte_load_wide(ByteArgs a, uint64_t row0, uint32_t units, FastDiv div_units)
{
    constexpr uint32_t kUnits = 4;
    uint32_t w[kUnits], e[kUnits], c[kUnits];
    uint64_t row[kUnits];
#pragma unroll
    for (uint32_t k = 0; k < kUnits; ++k) {
        const uint32_t at = (blockIdx.x * kUnits + k) * kThreads + threadIdx.x, r = div_units.div(at);
        c[k] = (at - r * units) * 4u;
        row[k] = row0 + r;
        w[k] = e[k] = 0;
        if (row[k] < a.rows) {
            w[k] = *reinterpret_cast<const uint32_t *>(a.codes + row[k] * a.pitch + c[k]);
            e[k] = a.exps[row[k] * a.ngroups + (c[k] >> a.gshift)];
        }
    }
#pragma unroll
    for (uint32_t k = 0; k < kUnits; ++k) {
        if (row[k] >= a.rows) continue;
        const f32x4 v = decode4<F>(w[k], scale_of(e[k]));
        float *p = static_cast<float *>(a.x) + row[k] * a.ld + c[k];
        if (a.cols - c[k] >= 4) {
            __builtin_memcpy(p, &v, 16);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (c[k] + i < a.cols) p[i] = v[i];
        }
    }
}

// Launches over ranges of rows whose units can be counted with 31 bits.
template <class LAUNCH>
void by_rows(uint64_t rows, uint32_t units, uint32_t per_thread, LAUNCH go)
{
    const uint64_t most = (1ull << 31) / units, block = (uint64_t)kThreads * per_thread;
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t n = rows - r < most ? rows - r : most;
        go(r, (uint32_t)((n * units + block - 1) / block));
    }
}

template <uint32_t T, uint32_t F>
void store_as(const ByteArgs &a, hipStream_t st)
{
    const uint32_t steps = a.gshift - 4, lanes = 1u << steps;
    const uint32_t units = (uint32_t)((a.pitch / 16 + lanes - 1) / lanes * lanes);
    const FastDiv d = FastDiv::make(units);
    by_rows(a.rows, units, 1, [&](uint64_t r, uint32_t grid) {
        hipLaunchKernelGGL((k_byte_store<T, F>), dim3(grid), dim3(kThreads), 0, st, a, r, units, steps, d);
    });
}

template <uint32_t T, uint32_t F>
void load_as(const ByteArgs &a, hipStream_t st)
{
    if constexpr (T == kTypeF32) {
        const uint32_t units = (a.cols + 3) / 4;
        const FastDiv d = FastDiv::make(units);
        by_rows(a.rows, units, 4, [&](uint64_t r, uint32_t grid) {
            hipLaunchKernelGGL((k_byte_load_wide<F>), dim3(grid), dim3(kThreads), 0, st, a, r, units, d);
        });
    } else {
        const uint32_t units = (uint32_t)(a.pitch / 16);
        const FastDiv d = FastDiv::make(units);
        by_rows(a.rows, units, 1, [&](uint64_t r, uint32_t grid) {
            hipLaunchKernelGGL((k_byte_load<T, F>), dim3(grid), dim3(kThreads), 0, st, a, r, units, d);
        });
    }
}

}  // namespace

void launch_byte_store(const ByteArgs &a, hipStream_t st)
{
    const bool i8 = a.format == kByteInt8;
    if (a.type == kTypeF32) i8 ? store_as<kTypeF32, kByteInt8>(a, st) : store_as<kTypeF32, kByteE4M3>(a, st);
    else if (a.type == kTypeF16) i8 ? store_as<kTypeF16, kByteInt8>(a, st) : store_as<kTypeF16, kByteE4M3>(a, st);
    else i8 ? store_as<kTypeBF16, kByteInt8>(a, st) : store_as<kTypeBF16, kByteE4M3>(a, st);
}

void launch_byte_load(const ByteArgs &a, hipStream_t st)
{
    const bool i8 = a.format == kByteInt8;
    if (a.type == kTypeF32) i8 ? load_as<kTypeF32, kByteInt8>(a, st) : load_as<kTypeF32, kByteE4M3>(a, st);
    else if (a.type == kTypeF16) i8 ? load_as<kTypeF16, kByteInt8>(a, st) : load_as<kTypeF16, kByteE4M3>(a, st);
    else i8 ? load_as<kTypeBF16, kByteInt8>(a, st) : load_as<kTypeBF16, kByteE4M3>(a, st);
}

}  // namespace cmpz
