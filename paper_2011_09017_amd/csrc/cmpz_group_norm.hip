// Group norm with an activation, channels last: x[batch][spatial][channels], statistics over the spatial positions
// and the channels of a group.
//   forward   h = (x - mean) * r, r = 1 / sqrt(var + eps);  u = h * gamma + beta;  y = act(u); the input can be kept as
//             a byte checkpoint in the same pass
//   backward  x' from the input or from its checkpoint, h and u as above from x' and the forward pass's mean and r;
//             du = dy * act'(u);  dbeta = sum du, dgamma = sum du * h over batch and positions;
//             A = sum du * gamma, B = sum du * gamma * h over a group;  dx = r * (du * gamma - (A + h * B) / count)
//
// Two passes each: the sums need all of a sample before the first output.  A workgroup takes a range of positions
// with all their channels, a thread eight neighbouring channels (128-bit accesses whatever a group's width is) of
// every rp-th position; sums are kept per channel and thread and joined per channel, then per group, in LDS.
#include "cmpz_byte.h"

namespace cmpz {
namespace {

constexpr uint32_t kMaxThreads = 1024;
constexpr uint32_t kPlain = 2;                 // source of the input: not codes

struct Plan {
    uint32_t nv;          // threads of a position: vectors of eight channels, in whole quantisation groups
    uint32_t rp;          // positions side by side
    uint32_t threads;
    uint32_t chunks;      // workgroups of a sample
    uint32_t rows_per;    // positions of a workgroup
    FastDiv  div_nv, div_chunks, div_per;
};

Plan make_plan(const NormArgs &a, uint32_t lanes)
{
    Plan p;
    p.nv = ((a.channels + 7) / 8 + lanes - 1) / lanes * lanes;
    p.rp = p.nv >= 512 ? 1 : 512 / p.nv;
    if (p.rp > a.spatial) p.rp = a.spatial ? a.spatial : 1;
    p.threads = (p.nv * p.rp + 63) / 64 * 64;
    const uint64_t want = a.batch ? (1024 + a.batch - 1) / a.batch : 1;
    uint64_t chunks = (a.spatial + p.rp * 4ull - 1) / (p.rp * 4ull);
    if (chunks > want) chunks = want;
    if (chunks < 1) chunks = 1;
    p.rows_per = (uint32_t)(((a.spatial + chunks - 1) / chunks + p.rp - 1) / p.rp * p.rp);
    if (p.rows_per < 1) p.rows_per = 1;
    p.chunks = (a.spatial + p.rows_per - 1) / p.rows_per;
    if (p.chunks < 1) p.chunks = 1;
    p.div_nv = FastDiv::make(p.nv);
    p.div_chunks = FastDiv::make(p.chunks);
    p.div_per = FastDiv::make(a.channels / a.groups);
    return p;
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) v += __shfl_xor(v, k);
    return v;
}

__device__ __forceinline__ float sigmoid(float u)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u));
}

// The place of a thread: its vector of eight channels and its first position, and those of its workgroup.
struct Place { uint32_t n, chunk, v, r, row_beg, row_end; int valid; };
__device__ __forceinline__ Place place(const NormArgs &a, const Plan &p, uint32_t block)
{
    Place q;
    q.n = p.div_chunks.div(block);
    q.chunk = block - q.n * p.chunks;
    q.r = p.div_nv.div(threadIdx.x);
    q.v = threadIdx.x - q.r * p.nv;
    q.row_beg = q.chunk * p.rows_per;
    q.row_end = a.spatial - q.row_beg < p.rows_per ? a.spatial : q.row_beg + p.rows_per;
    // channels that exist from this vector on; threads behind the last position's have none
    q.valid = q.r < p.rp && 8u * q.v < a.channels ? (int)(a.channels - 8u * q.v) : 0;
    return q;
}

// Sums over the workgroup's threads of eight values per thread: over the rp positions for every channel, into s[c].
template <class V>
__device__ __forceinline__ void join_channels(V *s, const V (&v)[8], const Plan &p)
{
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) s[threadIdx.x * 8u + k] = v[k];
    __syncthreads();
    const uint32_t width = p.nv * 8u;
    for (uint32_t c = threadIdx.x; c < width; c += blockDim.x) {
        double t = 0.0;
        for (uint32_t r = 0; r < p.rp; ++r) t += (double)s[r * width + c];
        s[c] = (V)t;
    }
    __syncthreads();
}

// Sum over a group's channels of f(c), by one wave.
template <class FN>
__device__ __forceinline__ double group_total(uint32_t g, uint32_t per, FN f)
{
    double t = 0.0;
    for (uint32_t c = threadIdx.x & 63u; c < per; c += 64u) t += f(g * per + c);
    return wave_sum(t);
}

// ---- forward ------------------------------------------------------------------------------------------

// Sums and sums of squares in fp64, which the vector units add at the rate of fp32: no cancellation however far
// the mean lies from zero, and no second pass over the data for the variance.
template <uint32_t T>
__global__ __launch_bounds__(kMaxThreads) void k_norm_sums(NormArgs a, Plan p)
{
    extern __shared__ double s_sum[];
    typedef typename ElemOf<T>::type E;
    const Place q = place(a, p, blockIdx.x);
    double s1[8], s2[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) s1[k] = s2[k] = 0.0;
    if (q.valid > 0) {
        const E *x = static_cast<const E *>(a.x) + (uint64_t)q.n * a.spatial * a.channels + 8u * q.v;
        for (uint32_t r = q.row_beg + q.r; r < q.row_end; r += p.rp) {
            const f32x8 v = load8<T>(x + (uint64_t)r * a.channels, q.valid);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double d = (double)v[k];
                s1[k] += d;
                s2[k] = __builtin_fma(d, d, s2[k]);
            }
        }
    }
    const uint32_t per = a.channels / a.groups, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    double *part = static_cast<double *>(a.work);
    for (int which = 0; which < 2; ++which) {
        join_channels(s_sum, which ? s2 : s1, p);
        for (uint32_t g = wave; g < a.groups; g += waves) {
            const double t = group_total(g, per, [&](uint32_t c) { return s_sum[c]; });
            if ((threadIdx.x & 63u) == 0) part[(((uint64_t)q.n * a.groups + g) * p.chunks + q.chunk) * 2 + which] = t;
        }
    }
}

// Two totals over the workgroups of a sample, for every group, into s[2 * g], s[2 * g + 1].
__device__ __forceinline__ void join_chunks(double *s, const double *part, uint32_t n, const NormArgs &a, const Plan &p)
{
    const uint32_t wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63u;
    for (uint32_t g = wave; g < a.groups; g += waves) {
        const double *at = part + ((uint64_t)n * a.groups + g) * p.chunks * 2;
        double t1 = 0.0, t2 = 0.0;
        for (uint32_t c = lane; c < p.chunks; c += 64u) { t1 += at[2 * c]; t2 += at[2 * c + 1]; }
        t1 = wave_sum(t1);
        t2 = wave_sum(t2);
        if (lane == 0) { s[2 * g] = t1; s[2 * g + 1] = t2; }
    }
    __syncthreads();
}

__device__ __forceinline__ float activate(float u, uint32_t act)
{
    return act == kActSilu ? u * sigmoid(u) : act == kActRelu ? (u > 0.0f ? u : u != u ? u : 0.0f) : u;
}

template <uint32_t T, uint32_t F>
__global__ __launch_bounds__(kMaxThreads) void k_norm_apply(NormArgs a, Plan p)
{
    extern __shared__ double s_sum[];
    typedef typename ElemOf<T>::type E;
    const Place q = place(a, p, blockIdx.x);
    join_chunks(s_sum, static_cast<const double *>(a.work), q.n, a, p);
    const double count = (double)a.spatial * (double)(a.channels / a.groups);
    for (uint32_t g = threadIdx.x; g < a.groups; g += blockDim.x) {
        const double mean = s_sum[2 * g] / count;
        double var = s_sum[2 * g + 1] / count - mean * mean;
        if (var < 0.0) var = 0.0;
        const double rstd = 1.0 / sqrt(var + a.eps);
        s_sum[2 * g] = mean;
        s_sum[2 * g + 1] = rstd;
        if (q.chunk == 0 && a.stats) {
            a.stats[((uint64_t)q.n * a.groups + g) * 2] = mean;
            a.stats[((uint64_t)q.n * a.groups + g) * 2 + 1] = rstd;
        }
    }
    __syncthreads();
    float mean[8], mul[8], add[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t c = 8u * q.v + k;
        mean[k] = mul[k] = add[k] = 0.0f;
        if (k < q.valid) {
            const uint32_t g = p.div_per.div(c);
            mean[k] = (float)s_sum[2 * g];
            mul[k] = (float)s_sum[2 * g + 1] * (a.gamma ? a.gamma[c] : 1.0f);
            add[k] = a.beta ? a.beta[c] : 0.0f;
        }
    }
    if (F != kPlain && blockIdx.x == 0 && threadIdx.x < a.tail_to - a.tail_from) a.codes[a.tail_from + threadIdx.x] = 0;
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    // every thread of the workgroup goes round as often: the lanes of a quantisation group meet in lanes_max
    for (uint32_t base = q.row_beg; base < q.row_end; base += p.rp) {
        const uint32_t r = base + q.r;
        const bool in = r < q.row_end && q.r < p.rp;
        const int n = in ? q.valid : 0;
        const uint64_t row = row0 + r;
        const f32x8 x = load8<T>(static_cast<const E *>(a.x) + (n > 0 ? row * a.channels + 8u * q.v : 0), n);
        f32x8 y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = activate(__builtin_fmaf(x[k] - mean[k], mul[k], add[k]), a.act);
        store8<T>(static_cast<E *>(a.y) + (n > 0 ? row * a.channels + 8u * q.v : 0), y, n);
        if constexpr (F != kPlain) {
            const uint32_t e = group_exponent<F>(lanes_max(amax8(x, 0u), a.gshift - 3));
            if (in && 8u * q.v < a.pitch) {
                *reinterpret_cast<u32x2 *>(a.codes + row * a.pitch + 8u * q.v) = encode8<F>(x, inverse_scale_of(e));
                if (n > 0 && ((8u * q.v) & ((1u << a.gshift) - 1u)) == 0)
                    a.exps[row * a.ngroups + ((8u * q.v) >> a.gshift)] = (uint8_t)e;
            }
        }
    }
}

// ---- backward -----------------------------------------------------------------------------------------

template <uint32_t T, uint32_t S>
__device__ __forceinline__ f32x8 source8(const NormArgs &a, uint64_t row, uint32_t v, int n)
{
    typedef typename ElemOf<T>::type E;
    if constexpr (S == kPlain) {
        return load8<T>(static_cast<const E *>(a.x) + (n > 0 ? row * a.channels + 8u * v : 0), n);
    } else {
        if (n <= 0) return f32x8{0, 0, 0, 0, 0, 0, 0, 0};
        const u32x2 w = *reinterpret_cast<const u32x2 *>(a.codes + row * a.pitch + 8u * v);
        return decode8<S>(w, scale_of(a.exps[row * a.ngroups + ((8u * v) >> a.gshift)]));
    }
}

// A thread's eight channels.
struct Channels { float mean[8], rstd[8], gamma[8], beta[8]; };
__device__ __forceinline__ Channels channels_of(const NormArgs &a, const Plan &p, const Place &q)
{
    Channels c;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t ch = 8u * q.v + k;
        c.mean[k] = c.rstd[k] = c.gamma[k] = c.beta[k] = 0.0f;
        if (k < q.valid) {
            const double *st = a.stats + ((uint64_t)q.n * a.groups + p.div_per.div(ch)) * 2;
            c.mean[k] = (float)st[0];
            c.rstd[k] = (float)st[1];
            c.gamma[k] = a.gamma ? a.gamma[ch] : 1.0f;
            c.beta[k] = a.beta ? a.beta[ch] : 0.0f;
        }
    }
    return c;
}

// du = dy * act'(u) and h of eight channels.
__device__ __forceinline__ void gradient8(const NormArgs &a, const Plan &p, const Place &q, const Channels &c, f32x8 x, f32x8 dy,
                                          f32x8 *du, f32x8 *h)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float hk = (x[k] - c.mean[k]) * c.rstd[k], u = __builtin_fmaf(hk, c.gamma[k], c.beta[k]);
        (*h)[k] = hk;
        if (a.act == kActSilu) {
            const float g = sigmoid(u);
            (*du)[k] = dy[k] * (g * __builtin_fmaf(u, 1.0f - g, 1.0f));
        } else if (a.act == kActRelu) {
            bool positive = u > 0.0f;
            // where fp32 cannot tell the side of the border (its error is below eight roundings of these terms), fp64 does
            const float terms = __builtin_fmaf(fabsf(c.gamma[k] * c.rstd[k]), fabsf(x[k]) + fabsf(c.mean[k]), fabsf(c.beta[k]));
            if (fabsf(u) < 0x1p-20f * terms && k < q.valid) {
                const double *st = a.stats + ((uint64_t)q.n * a.groups + p.div_per.div(8u * q.v + k)) * 2;
                positive = ((double)x[k] - st[0]) * st[1] * (double)c.gamma[k] + (double)c.beta[k] > 0.0;
            }
            (*du)[k] = positive ? dy[k] : u != u ? u : 0.0f;
        } else {
            (*du)[k] = dy[k];
        }
    }
}

template <uint32_t T, uint32_t S>
__global__ __launch_bounds__(kMaxThreads) void k_norm_grad_sums(NormArgs a, Plan p)
{
    extern __shared__ double s_sum[];
    typedef typename ElemOf<T>::type E;
    float *s = reinterpret_cast<float *>(s_sum);
    const Place q = place(a, p, blockIdx.x);
    const Channels ch = channels_of(a, p, q);
    float sp[8], sq[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sp[k] = sq[k] = 0.0f;
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    if (q.valid > 0) {
        for (uint32_t r = q.row_beg + q.r; r < q.row_end; r += p.rp) {
            const uint64_t row = row0 + r;
            const f32x8 dy = load8<T>(static_cast<const E *>(a.dy) + row * a.channels + 8u * q.v, q.valid);
            f32x8 du, h;
            gradient8(a, p, q, ch, source8<T, S>(a, row, q.v, q.valid), dy, &du, &h);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sp[k] += du[k];
                sq[k] = __builtin_fmaf(du[k], h[k], sq[k]);
            }
        }
    }
    const uint32_t per = a.channels / a.groups, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    double *part = static_cast<double *>(a.work);
    float *chan = reinterpret_cast<float *>(part + 2ull * a.batch * a.groups * p.chunks) + 2ull * blockIdx.x * a.channels;
    for (int which = 0; which < 2; ++which) {
        join_channels(s, which ? sq : sp, p);
        for (uint32_t c = threadIdx.x; c < a.channels; c += blockDim.x) chan[(uint64_t)which * a.channels + c] = s[c];
        for (uint32_t g = wave; g < a.groups; g += waves) {
            const double t = group_total(g, per, [&](uint32_t c) { return (double)s[c] * (double)(a.gamma ? a.gamma[c] : 1.0f); });
            if ((threadIdx.x & 63u) == 0) part[(((uint64_t)q.n * a.groups + g) * p.chunks + q.chunk) * 2 + which] = t;
        }
    }
}

// dbeta and dgamma of sixteen channels: the sums of the first pass's workgroups, in a fixed order.
__device__ __forceinline__ void join_parameters(double *s, const NormArgs &a, const Plan &p, uint32_t block)
{
    const uint64_t records = a.spatial ? a.batch * p.chunks : 0;
    const float *chan = reinterpret_cast<const float *>(static_cast<const double *>(a.work) + 2ull * a.batch * a.groups * p.chunks);
    const uint32_t c = block * 16u + (threadIdx.x & 15u), parts = blockDim.x >> 4;
    double t[2] = {0.0, 0.0};
    if (c < a.channels) {
        for (uint64_t k = threadIdx.x >> 4; k < records; k += parts) {
            t[0] += (double)chan[2 * k * a.channels + c];
            t[1] += (double)chan[(2 * k + 1) * a.channels + c];
        }
    }
    for (int which = 0; which < 2; ++which) {
        float *out = which ? a.dgamma : a.dbeta;
        __syncthreads();
        s[threadIdx.x] = t[which];
        __syncthreads();
        if (threadIdx.x < 16u && c < a.channels && out) {
            double sum = 0.0;
            for (uint32_t k = 0; k < parts; ++k) sum += s[16u * k + threadIdx.x];
            out[c] = (float)sum;
        }
    }
}

template <uint32_t T, uint32_t S>
__global__ __launch_bounds__(kMaxThreads) void k_norm_grad_apply(NormArgs a, Plan p, uint32_t param_blocks)
{
    extern __shared__ double s_sum[];
    typedef typename ElemOf<T>::type E;
    if (blockIdx.x < param_blocks) { join_parameters(s_sum, a, p, blockIdx.x); return; }
    const Place q = place(a, p, blockIdx.x - param_blocks);
    join_chunks(s_sum, static_cast<const double *>(a.work), q.n, a, p);
    const Channels ch = channels_of(a, p, q);
    const double count = (double)a.spatial * (double)(a.channels / a.groups);
    float ga[8], gb[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        ga[k] = gb[k] = 0.0f;
        if (k < q.valid) {
            const uint32_t g = p.div_per.div(8u * q.v + k);
            ga[k] = (float)(s_sum[2 * g] / count);
            gb[k] = (float)(s_sum[2 * g + 1] / count);
        }
    }
    if (q.valid <= 0) return;
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    for (uint32_t r = q.row_beg + q.r; r < q.row_end; r += p.rp) {
        const uint64_t row = row0 + r;
        const f32x8 dy = load8<T>(static_cast<const E *>(a.dy) + row * a.channels + 8u * q.v, q.valid);
        f32x8 du, h, dx;
        gradient8(a, p, q, ch, source8<T, S>(a, row, q.v, q.valid), dy, &du, &h);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            dx[k] = ch.rstd[k] * (__builtin_fmaf(du[k], ch.gamma[k], -ga[k]) - h[k] * gb[k]);
        store8<T>(static_cast<E *>(a.y) + row * a.channels + 8u * q.v, dx, q.valid);
    }
}

size_t lds_bytes(const NormArgs &a, const Plan &p, uint32_t per_thread)
{
    const size_t joined = (size_t)p.threads * per_thread, groups = 16ull * a.groups;
    return joined > groups ? joined : groups;
}

template <uint32_t T>
void forward_as(const NormArgs &a, hipStream_t st)
{
    const uint32_t lanes = a.codes ? 1u << (a.gshift - 3) : 1u;
    const Plan p = make_plan(a, lanes);
    const dim3 grid((uint32_t)(a.batch * p.chunks)), block(p.threads);
    hipLaunchKernelGGL((k_norm_sums<T>), grid, block, lds_bytes(a, p, 64), st, a, p);
    const size_t lds = 16ull * a.groups;
    if (!a.codes) hipLaunchKernelGGL((k_norm_apply<T, kPlain>), grid, block, lds, st, a, p);
    else if (a.format == kByteInt8) hipLaunchKernelGGL((k_norm_apply<T, kByteInt8>), grid, block, lds, st, a, p);
    else hipLaunchKernelGGL((k_norm_apply<T, kByteE4M3>), grid, block, lds, st, a, p);
}

template <uint32_t T, uint32_t S>
void backward_as(const NormArgs &a, hipStream_t st)
{
    const Plan p = make_plan(a, 1);
    const uint32_t work = a.spatial ? (uint32_t)(a.batch * p.chunks) : 0;
    const uint32_t params = a.dgamma || a.dbeta ? (a.channels + 15) / 16 : 0;
    if (work) hipLaunchKernelGGL((k_norm_grad_sums<T, S>), dim3(work), dim3(p.threads), lds_bytes(a, p, 32), st, a, p);
    if (work + params)
        hipLaunchKernelGGL((k_norm_grad_apply<T, S>), dim3(work + params), dim3(p.threads), lds_bytes(a, p, 8), st, a, p, params);
}

template <uint32_t T>
void backward_of(const NormArgs &a, hipStream_t st)
{
    if (!a.codes) backward_as<T, kPlain>(a, st);
    else if (a.format == kByteInt8) backward_as<T, kByteInt8>(a, st);
    else backward_as<T, kByteE4M3>(a, st);
}

}  // namespace

// One figure for a forward and a backward pass, with a checkpoint or without (the plans differ with the threads that a
// position takes).
uint64_t group_norm_work(const NormArgs &a)
{
    uint64_t most = 0;
    for (uint32_t lanes : {1u, 4u, 8u, 16u}) {
        const uint64_t records = a.batch * make_plan(a, lanes).chunks;
        const uint64_t bytes = records * (16ull * a.groups + (lanes == 1u ? 8ull * a.channels : 0ull));
        if (bytes > most) most = bytes;
    }
    return most;
}

void launch_group_norm(const NormArgs &a, hipStream_t st)
{
    if (a.type == kTypeF32) forward_as<kTypeF32>(a, st);
    else if (a.type == kTypeF16) forward_as<kTypeF16>(a, st);
    else forward_as<kTypeBF16>(a, st);
}

void launch_group_norm_grad(const NormArgs &a, hipStream_t st)
{
    if (a.type == kTypeF32) backward_of<kTypeF32>(a, st);
    else if (a.type == kTypeF16) backward_of<kTypeF16>(a, st);
    else backward_of<kTypeBF16>(a, st);
}

}  // namespace cmpz
