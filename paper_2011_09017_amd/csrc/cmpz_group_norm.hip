// Group norm with an activation, channels last: x[batch][spatial][channels], statistics over the spatial positions
// and the channels of a group.
//   forward   h = (x - mean) * r, r = 1 / sqrt(var + eps);  u = h * gamma + beta;  y = act(u); the input can be kept as
//             a byte checkpoint in the same pass
//   backward  x' from the input or from its checkpoint, h and u as above from x' and the forward pass's mean and r;
//             du = dy * act'(u);  dbeta = sum du, dgamma = sum du * h over batch and positions;
//             A = sum du * gamma, B = sum du * gamma * h over a group;  dx = r * (du * gamma - (A + h * B) / count)
//
// The sums need all of a sample before the first output.  Where a sample's channels can be cut into segments of whole
// groups that fit the registers of one workgroup, that workgroup reads its segment once and does everything (k_norm_slab,
// k_norm_grad_slab).  Otherwise there are two passes: a workgroup takes a range of positions with all their channels.
// In both a thread takes eight neighbouring channels (128-bit accesses whatever a group's width is) of every rp-th
// position; sums are kept per channel and thread and joined per channel, then per group, in LDS.
//
// Measured on bf16 with int8 codes, SiLU: 256 x 12544 x 64 in 8 groups (411 MB a tensor, copies run at 5.16 TB/s): forward sums
// 103 us (4.0 TB/s), apply 222 (1031 MB in all, 4.6); backward sums 179 (3.5: the sigmoid and the codes' expansion on 16
// values a lane beside 48 bytes of loads), apply 203 (5.1); counters show no byte read twice.  One pass, 256 x 49 x 512 fp32:
// 18.0 and 22.2 us (3.3 and 2.6 TB/s): all its workgroups are on the chip at once, loading, adding and storing at the same
// time; one sample of 49 x 512 bf16: 6.3 us, latency.
//
// All are compiled for 1024 threads, so for 128 registers.  One-pass backward kernels of vectors that cross groups (ONE false) spill
// up to 54 of them (ReLU), 22 (SiLU) and 14 (none): 256 x 49 x 480 in 32 groups, ReLU fp32 with int8 codes, takes 40.3 us
// backward where 512 channels take 26.0.
#include "cmpz_byte.h"

#include <type_traits>

namespace cmpz {
namespace {

constexpr uint32_t kMaxThreads = 1024;
constexpr uint32_t kPlain = 2;                 // source of the input: not codes
constexpr uint32_t kSlabRows = 4;              // positions that a thread of a slab keeps in registers

struct Plan {
    uint32_t nv;          // threads of a position: vectors of eight channels (two passes: in whole quantisation groups)
    uint32_t rp;          // positions side by side
    uint32_t threads;
    uint32_t chunks;      // workgroups of a sample: ranges of positions, or segments of channels
    uint32_t rows_per;    // positions of a workgroup
    uint32_t per;         // channels of a group
    double   share;       // 1 / (positions * per)
    FastDiv  div_nv, div_chunks, div_per;
};

void finish_plan(Plan *p, const NormArgs &a)
{
    p->threads = (p->nv * p->rp + 63) / 64 * 64;
    p->per = a.channels / a.groups;
    p->share = a.spatial ? 1.0 / ((double)a.spatial * (double)p->per) : 0.0;
    p->div_nv = FastDiv::make(p->nv);
    p->div_chunks = FastDiv::make(p->chunks);
    p->div_per = FastDiv::make(p->per);
}

// About 512 workgroups of 512 threads, two to a CU: each has parameters, statistics and the joining of its sums to pay for
// (8 x 16384 x 320 bf16 forward: 60 us, with 1024 of them 68; 64 x 3136 x 256: 76 and 88; 256 x 12544 x 64: 335 and 331).
Plan two_pass_plan(const NormArgs &a, uint32_t lanes)
{
    Plan p{};
    p.nv = ((a.channels + 7) / 8 + lanes - 1) / lanes * lanes;
    p.rp = p.nv >= 512 ? 1 : 512 / p.nv;
    if (p.rp > a.spatial) p.rp = a.spatial ? a.spatial : 1;
    const uint64_t want = a.batch ? (512 + a.batch - 1) / a.batch : 1;
    uint64_t chunks = (a.spatial + p.rp * 4ull - 1) / (p.rp * 4ull);
    if (chunks > want) chunks = want;
    if (chunks < 1) chunks = 1;
    p.rows_per = (uint32_t)(((a.spatial + chunks - 1) / chunks + p.rp - 1) / p.rp * p.rp);
    if (p.rows_per < 1) p.rows_per = 1;
    p.chunks = (a.spatial + p.rows_per - 1) / p.rows_per;
    if (p.chunks < 1) p.chunks = 1;
    finish_plan(&p, a);
    return p;
}

uint32_t lcm(uint32_t x, uint32_t y)
{
    uint32_t g = x, h = y;
    while (h) { const uint32_t t = g % h; g = h; h = t; }
    return x / g * y;
}

// The smallest segment is a multiple of eight channels, of a group and, where codes are written, of a quantisation group
// (or all channels).  It grows to 128 bytes of a position, and below that there is no slab: with 64 bytes the backward
// pass of 128 x 784 x 512 bf16 took 192 us where two passes take 93.  It grows to 192 vectors too, three full waves: 4096 x 16 x
// 512 bf16 took 75 and 103 us with 128 and 54 and 85 with 256, but 256 x 49 x 512 fp32 backward 25 with 196 and 32 with 392.  Small segments, down to a single wave, keep
// all of a CU's registers busy with loads (256 x 7 x 7 x 512 fp32, both directions: 42 us, with 1024 vectors to a segment 80).
bool slab_plan(Plan *out, const NormArgs &a, uint32_t lanes)
{
    if (a.spatial == 0) return false;
    Plan p{};
    const uint32_t all = (a.channels + 7) / 8;
    uint32_t unit = lcm(8u * lanes, a.channels / a.groups) / 8;
    if (unit >= all) unit = (all + lanes - 1) / lanes * lanes;
    const uint64_t most = (uint64_t)kMaxThreads * kSlabRows;
    auto fits = [&](uint32_t nv) { return (uint64_t)nv * a.spatial <= most && nv <= kMaxThreads; };
    if (!fits(unit)) return false;
    p.nv = unit;
    while (p.nv + unit <= all && fits(p.nv + unit) && (p.nv * 8 * type_bytes(a.type) < 128 || (uint64_t)p.nv * a.spatial < 192)) p.nv += unit;
    if (p.nv < all && p.nv * 8 * type_bytes(a.type) < 128) return false;
    p.chunks = (all + p.nv - 1) / p.nv;
    // Positions per thread: as many as it can hold, so that a CU has most bytes in flight; one where all threads fit the
    // chip at once and only the time of a single workgroup counts.
    const uint64_t vectors = (uint64_t)p.nv * a.spatial;
    uint32_t rows = (uint32_t)((vectors + kMaxThreads - 1) / kMaxThreads);
    if (a.batch * p.chunks * vectors > 256ull * kMaxThreads && rows < kSlabRows) rows = kSlabRows;
    p.rp = (a.spatial + rows - 1) / rows;
    while ((uint64_t)p.rp * p.nv > kMaxThreads) {
        ++rows;
        p.rp = (a.spatial + rows - 1) / rows;
    }
    if (rows > kSlabRows) return false;
    p.rows_per = a.spatial;
    finish_plan(&p, a);
    if (a.batch * p.chunks * p.threads > 1ull << 31) return false;        // a launch counts its threads with 32 bits
    *out = p;
    return true;
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

__device__ __forceinline__ float activate(float u, uint32_t act)
{
    return act == kActSilu ? u * sigmoid(u) : act == kActRelu ? (u > 0.0f ? u : u != u ? u : 0.0f) : u;
}

// The place of a thread: its sample, its first channel, how many of its eight channels exist, its first position.
struct Place { uint32_t n, chunk, c, v, r; int valid; };
__device__ __forceinline__ Place place(const Plan &p, uint32_t block, uint32_t first_channel, uint32_t end_channel)
{
    Place q;
    q.n = p.div_chunks.div(block);
    q.chunk = block - q.n * p.chunks;
    q.r = p.div_nv.div(threadIdx.x);
    q.v = threadIdx.x - q.r * p.nv;
    q.c = first_channel + 8u * q.v;
    // threads behind the last position's have no channels
    q.valid = q.r < p.rp && q.c < end_channel ? (int)(end_channel - q.c) : 0;
    return q;
}

// Sums over the workgroup's threads of eight values per thread and channel: over the rp positions for every channel, into
// s[channel of the segment].  Two sums at once, the second behind the first's threads * 8 values.  The loops over LDS are
// unrolled by hand, here and in join_parameters: else every read waits for the one before it (256 x 49 x 512 fp32
// backward: 28.9 us, unrolled 25.8).
template <class V>
__device__ __forceinline__ void join_channels(V *s, const V (&v)[8], const V (&w)[8], const Plan &p)
{
    V *s2 = s + blockDim.x * 8u;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) { s[threadIdx.x * 8u + k] = v[k]; s2[threadIdx.x * 8u + k] = w[k]; }
    __syncthreads();
    const uint32_t width = p.nv * 8u;
    for (uint32_t c = threadIdx.x; c < 2u * width; c += blockDim.x) {
        V *q = c < width ? s + c : s2 + (c - width);
        double t = 0.0;
#pragma unroll 8
        for (uint32_t r = 0; r < p.rp; ++r) t += (double)q[r * width];
        *q = (V)t;
    }
    __syncthreads();
}

// Lanes that add up `items` values: a whole wave, or for few a power of two of it, so that a wave takes several groups at once
// (65536 x 1 x 512 in 32 groups, forward: 880 us with a wave to a group, 139 so; 64 x 3136 x 256 in 256: 117 and 83).
__device__ __forceinline__ uint32_t lanes_of(uint32_t items)
{
    uint32_t w = 64u;
    while (w > 1u && w / 2u >= items) w >>= 1;
    return w;
}
__device__ __forceinline__ double lanes_sum(double v, uint32_t w)
{
    if (w == 64u) return wave_sum(v);
    for (uint32_t k = w >> 1; k; k >>= 1) v += __shfl_xor(v, (int)k);
    return v;
}

// For each of `groups` groups, w lanes to one: take(group, lane of the w, mine).  Lanes behind the last group take it once more
// (take's sums cross lanes); `mine`: this lane has the group's result.
template <class FN>
__device__ __forceinline__ void each_group(uint32_t groups, uint32_t w, FN take)
{
    const uint32_t at_once = 64u / w, lane = threadIdx.x & 63u;
    for (uint32_t g0 = (threadIdx.x >> 6) * at_once; g0 < groups; g0 += (blockDim.x >> 6) * at_once) {
        const uint32_t g = g0 + lane / w;
        take(g < groups ? g : groups - 1u, lane & (w - 1u), g < groups && (lane & (w - 1u)) == 0);
    }
}

// Sum over a group's channels of f(channel of the segment), by w lanes; g counts from the segment's first group.
template <class FN>
__device__ __forceinline__ double group_total(uint32_t g, uint32_t per, uint32_t sub, uint32_t w, FN f)
{
    double t = 0.0;
    for (uint32_t c = sub; c < per; c += w) t += f(g * per + c);
    return lanes_sum(t, w);
}

// ---- forward ------------------------------------------------------------------------------------------

// Sums and sums of squares in fp64, which the vector units add at the rate of fp32, and no second pass over the data for the
// variance E[x^2] - E[x]^2 while that is at least kUnsure of E[x^2]: with 2^-53 to a rounding it is right to 2^-26 then.  Where
// it is less (a mean some 256 deviations from zero), the workgroup adds up its values a second time, less a value near
// their mean: they are in registers or caches (256 x 49 x 512 fp32: 13.8 us, so 18.9; 64 x 3136 x 256: 127 and 149).  All
// values less the first of their group, at once, would cost everyone 8 to 10 % (256 x 49 x 512 fp32 with codes: 18.6 us and 19.9).
constexpr double kUnsure = 0x1p-16;
template <bool ABOUT>
__device__ __forceinline__ void add_moments(f32x8 v, const float (&at)[8], double (&s1)[8], double (&s2)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const double d = ABOUT ? (double)v[k] - (double)at[k] : (double)v[k];
        s1[k] += d;
        s2[k] = __builtin_fma(d, d, s2[k]);
    }
}

// Totals of the workgroup for each of `groups` groups of its segment: give(g, sum, sum of squares) by one lane.  Groups of eight channels and more: a vector lies in one or two of them, and its channels are added up to
// these before LDS (32 bytes a thread instead of 128, which would leave a CU two workgroups).
template <class FN>
__device__ __forceinline__ void join_moments(double *s, double (&s1)[8], double (&s2)[8], uint32_t groups, const Plan &p, const Place &q,
                                             uint32_t first, FN give)
{
    if (p.per >= 8) {
        const uint32_t c0 = q.c - first, g0 = p.div_per.div(c0), cut = (g0 + 1u) * p.per - c0;   // channels in the first of the two
        double t1 = 0.0, t2 = 0.0, u1 = 0.0, u2 = 0.0;
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            if (k < cut) { t1 += s1[k]; t2 += s2[k]; }
            else { u1 += s1[k]; u2 += s2[k]; }
        }
        double *o = s + 4u * threadIdx.x;
        o[0] = t1; o[1] = t2; o[2] = u1; o[3] = u2;
        __syncthreads();
        const uint32_t w = lanes_of((p.per / 8u + 2u) * p.rp);
        each_group(groups, w, [&](uint32_t g, uint32_t sub, bool mine) {
            const uint32_t v0 = g * p.per / 8u, nv = ((g + 1u) * p.per - 1u) / 8u - v0 + 1u, items = nv * p.rp;
            double a1 = 0.0, a2 = 0.0;
            for (uint32_t i = sub; i < items; i += w) {
                const uint32_t r = i / nv, v = v0 + (i - r * nv);
                const double *in = s + 4u * (r * p.nv + v) + (8u * v < g * p.per ? 2u : 0u);
                a1 += in[0];
                a2 += in[1];
            }
            a1 = lanes_sum(a1, w);
            a2 = lanes_sum(a2, w);
            if (mine) give(g, a1, a2);
        });
    } else {
        join_channels(s, s1, s2, p);
        const double *u = s + blockDim.x * 8u;
        const uint32_t w = lanes_of(p.per);
        each_group(groups, w, [&](uint32_t g, uint32_t sub, bool mine) {
            const double a1 = group_total(g, p.per, sub, w, [&](uint32_t c) { return s[c]; });
            const double a2 = group_total(g, p.per, sub, w, [&](uint32_t c) { return u[c]; });
            if (mine) give(g, a1, a2);
        });
    }
}

// From the sums about `at`.  unsure: kUnsure.
struct Moments { double mean, rstd; bool unsure; };
__device__ __forceinline__ Moments moments_of(const NormArgs &a, const Plan &p, double at, double s1, double s2)
{
    const double off = s1 * p.share, square = s2 * p.share;
    double var = square - off * off;
    if (var < 0.0) var = 0.0;
    var += a.eps;
    const bool unsure = var < kUnsure * square;
    // an approximation of 26 bits and two steps of Newton's method: a division and a square root take four times as long
    double r = __builtin_amdgcn_rsq(var);
    r = r * __builtin_fma(-0.5 * var * r, r, 1.5);
    r = r * __builtin_fma(-0.5 * var * r, r, 1.5);
    // a mean that is an fp32 number but for the roundings of its division is one: that of equal values is their value
    double mean = at + off;
    const double near = (double)(float)mean;
    if (fabs(mean - near) <= 0x1p-48 * fabs(mean)) mean = near;
    return {mean, r, unsure};
}

// u = (x - mean) * mul + add of a thread's channels (a group of equal values gives exactly beta): what the mean loses in
// its rounding to fp32 is in `add`.
struct __align__(16) Group { float mean, lost; double rstd; };            // mean + lost: the mean
__device__ __forceinline__ Group group_of(double mean, double rstd)
{
    const float near = (float)mean;
    return {near, (float)(mean - (double)near), rstd};
}
struct Line { float mean[8], mul[8], add[8]; };
__device__ __forceinline__ Line parameters_of(const NormArgs &a, const Place &q)
{
    Line l;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        l.mean[k] = l.mul[k] = l.add[k] = 0.0f;
        if (k < q.valid) {
            l.mul[k] = a.gamma ? a.gamma[q.c + k] : 1.0f;
            l.add[k] = a.beta ? a.beta[q.c + k] : 0.0f;
        }
    }
    return l;
}
template <class FN>
__device__ __forceinline__ void apply_moments(Line *l, const Plan &p, const Place &q, uint32_t first, FN of_group)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (k < q.valid) {
            const Group m = of_group(p.div_per.div(q.c + k - first));
            l->mean[k] = m.mean;
            l->mul[k] = (float)(m.rstd * (double)l->mul[k]);
            l->add[k] = __builtin_fmaf(-m.lost, l->mul[k], l->add[k]);
        }
    }
}

// y and codes of one vector; all lanes of a quantisation group come here together.  `in`: its position exists.
template <uint32_t T, uint32_t F, bool EVEN>
__device__ __forceinline__ void put_outputs(const NormArgs &a, const Place &q, const Line &l, f32x8 x, uint64_t row, bool in)
{
    typedef typename ElemOf<T>::type E;
    const int n = in ? q.valid : 0;
    f32x8 y;
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = activate(__builtin_fmaf(x[k] - l.mean[k], l.mul[k], l.add[k]), a.act);
    if (n > 0) store8<T>(static_cast<E *>(a.y) + row * a.channels + q.c, y, EVEN ? 8 : n);
    if constexpr (F != kPlain) {
        const uint32_t e = group_exponent<F>(lanes_max(amax8(x, 0u), a.gshift - 3));
        if (in && q.c < a.pitch) {
            *reinterpret_cast<u32x2 *>(a.codes + row * a.pitch + q.c) = encode8<F>(x, inverse_scale_of(e));
            if (n > 0 && (q.c & ((1u << a.gshift) - 1u)) == 0) a.exps[row * a.ngroups + (q.c >> a.gshift)] = (uint8_t)e;
        }
    }
}

// load8 where either all eight values exist or none (EVEN: channels are a multiple of eight).
template <uint32_t T, bool EVEN>
__device__ __forceinline__ f32x8 load_vector(const typename ElemOf<T>::type *p, int n)
{
    if constexpr (EVEN) {
        f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (n > 0) v = load8<T>(p, 8);
        return v;
    } else {
        return load8<T>(p, n);
    }
}

__device__ __forceinline__ void put_tail(const NormArgs &a)
{
    if (blockIdx.x == 0 && threadIdx.x < a.tail_to - a.tail_from) a.codes[a.tail_from + threadIdx.x] = 0;
}

template <uint32_t T, uint32_t F, bool EVEN>
__global__ __launch_bounds__(kMaxThreads) void k_norm_slab(NormArgs a, Plan p)
{
    extern __shared__ __align__(16) double s_sum[];
    __shared__ uint32_t s_unsure;
    typedef typename ElemOf<T>::type E;
    Place q = place(p, blockIdx.x, 0, 0);
    const uint32_t first = q.chunk * p.nv * 8u, end = a.channels - first < p.nv * 8u ? a.channels : first + p.nv * 8u;
    q = place(p, blockIdx.x, first, end);
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    if (threadIdx.x == 0) s_unsure = 0;                                   // (barriers lie between this and what sets it)
    f32x8 x[kSlabRows];
    float at[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    double s1[8], s2[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) s1[k] = s2[k] = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < kSlabRows; ++i) {
        const uint32_t r = q.r + i * p.rp;
        const int n = r < a.spatial ? q.valid : 0;
        x[i] = load_vector<T, EVEN>(static_cast<const E *>(a.x) + (n > 0 ? (row0 + r) * a.channels + q.c : 0), n);
    }
    Line l = parameters_of(a, q);
#pragma unroll
    for (uint32_t i = 0; i < kSlabRows; ++i) add_moments<false>(x[i], at, s1, s2);
    const uint32_t groups = (end - first) / p.per;
    Group *m = reinterpret_cast<Group *>(s_sum + (p.per < 8u ? 16u : 4u) * blockDim.x);
    auto give = [&](uint32_t g, const Moments &v) {
        m[g] = group_of(v.mean, v.rstd);
        if (a.stats) {
            double *st = a.stats + ((uint64_t)q.n * a.groups + p.div_per.div(first) + g) * 2;
            st[0] = v.mean;
            st[1] = v.rstd;
        }
    };
    join_moments(s_sum, s1, s2, groups, p, q, first, [&](uint32_t g, double t1, double t2) {
        const Moments v = moments_of(a, p, 0.0, t1, t2);
        if (v.unsure) s_unsure = 1;
        give(g, v);
    });
    __syncthreads();
    if (s_unsure) {                                                       // (uniform) about the means as they are so far
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s1[k] = s2[k] = 0.0;
            if (k < q.valid) at[k] = m[p.div_per.div(q.c + k - first)].mean;
        }
#pragma unroll
        for (uint32_t i = 0; i < kSlabRows; ++i) {
            f32x8 v;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float f = q.r + i * p.rp < a.spatial ? x[i][k] : at[k];
                asm volatile("" : "+v"(f));                               // else the fp64 forms of all values are kept from above
                v[k] = f;
            }
            add_moments<true>(v, at, s1, s2);
        }
        join_moments(s_sum, s1, s2, groups, p, q, first, [&](uint32_t g, double t1, double t2) {
            give(g, moments_of(a, p, (double)m[g].mean, t1, t2));
        });
        __syncthreads();
    }
    apply_moments(&l, p, q, first, [&](uint32_t g) { return m[g]; });
    if (F != kPlain) put_tail(a);
#pragma unroll
    for (uint32_t i = 0; i < kSlabRows; ++i) {
        if (i * p.rp >= a.spatial) break;                                 // (uniform)
        const uint32_t r = q.r + i * p.rp;
        put_outputs<T, F, EVEN>(a, q, l, x[i], row0 + r, r < a.spatial && q.r < p.rp);
    }
}

// A workgroup's record of a group: the mean of its values, and the sum of the squares of their distances from it.
template <uint32_t T, bool EVEN>
__global__ __launch_bounds__(kMaxThreads) void k_norm_sums(NormArgs a, Plan p)
{
    extern __shared__ __align__(16) double s_sum[];
    __shared__ uint32_t s_unsure;
    typedef typename ElemOf<T>::type E;
    const Place q = place(p, blockIdx.x, 0, a.channels);
    const uint32_t beg = q.chunk * p.rows_per, end = a.spatial - beg < p.rows_per ? a.spatial : beg + p.rows_per;
    if (threadIdx.x == 0) s_unsure = 0;                                   // (barriers lie between this and what sets it)
    const E *row0 = static_cast<const E *>(a.x) + ((uint64_t)q.n * a.spatial + beg) * a.channels;
    float at[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    double s1[8], s2[8];
    auto add_up = [&](auto about) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s1[k] = s2[k] = 0.0;
        if (q.valid <= 0) return;
        const E *x = row0 + (uint64_t)q.r * a.channels + q.c;
        const uint64_t step = (uint64_t)p.rp * a.channels;
        const int n = EVEN ? 8 : q.valid;
        uint32_t left = end - beg > q.r ? (end - beg - q.r + p.rp - 1) / p.rp : 0;      // positions of this thread
        for (; left >= 4; left -= 4, x += 4 * step) {                     // four loads in flight
            f32x8 v[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) v[i] = load8<T>(x + i * step, n);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) add_moments<decltype(about)::value>(v[i], at, s1, s2);
        }
        for (; left; --left, x += step) add_moments<decltype(about)::value>(load8<T>(x, n), at, s1, s2);
    };
    const double count = (double)(end - beg) * (double)p.per, share = 1.0 / count;
    auto give = [&](uint32_t g, double mean, double squares) {
        double *o = static_cast<double *>(a.work) + (((uint64_t)q.n * a.groups + g) * p.chunks + q.chunk) * 2;
        o[0] = mean;
        o[1] = squares < 0.0 ? 0.0 : squares;
    };
    add_up(std::false_type{});
    join_moments(s_sum, s1, s2, a.groups, p, q, 0, [&](uint32_t g, double t1, double t2) {
        const double mean = t1 * share, squares = t2 - t1 * mean;
        if (squares + a.eps * count < kUnsure * t2) s_unsure = 1;
        give(g, mean, squares);
    });
    __syncthreads();
    if (s_unsure == 0) return;                                            // (uniform) about the groups' first values here
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < q.valid) at[k] = (float)row0[p.div_per.div(q.c + k) * p.per];
    add_up(std::true_type{});
    join_moments(s_sum, s1, s2, a.groups, p, q, 0, [&](uint32_t g, double t1, double t2) {
        const double off = t1 * share;
        give(g, (double)row0[g * p.per] + off, t2 - t1 * off);
    });
}

// Two totals over the workgroups of a sample and group, by one wave.
struct Totals { double t1, t2; };
__device__ __forceinline__ Totals join_chunks(const double *part, uint64_t sample_and_group, const Plan &p)
{
    const double *at = part + sample_and_group * p.chunks * 2;
    double t1 = 0.0, t2 = 0.0;
#pragma unroll 4
    for (uint32_t c = threadIdx.x & 63u; c < p.chunks; c += 64u) { t1 += at[2 * c]; t2 += at[2 * c + 1]; }
    return {wave_sum(t1), wave_sum(t2)};
}

// Mean and 1 / deviation of every sample and group, between the two passes, from the workgroups' records about the first one's
// mean.  A launch of its own costs 3 us; with this in the prologue of the second pass's workgroups, each of them reads all of
// its sample's records: one sample of 65536 x 128 takes 41.6 us so where the three launches take 33.8, but 64 samples of 3136 x
// 256 take 72 where they take 76.  The launch is taken always; the line between the two has not been drawn.
__global__ __launch_bounds__(kMaxThreads) void k_norm_join(NormArgs a, Plan p, double *stats)
{
    const double full = (double)p.rows_per * (double)p.per, last = (double)(a.spatial - (p.chunks - 1u) * p.rows_per) * (double)p.per;
    for (uint64_t i = blockIdx.x * 16ull + (threadIdx.x >> 6); i < a.batch * a.groups; i += gridDim.x * 16ull) {
        const double *at = static_cast<const double *>(a.work) + i * p.chunks * 2, near = at[0];
        double t1 = 0.0, t2 = 0.0;
#pragma unroll 4
        for (uint32_t c = threadIdx.x & 63u; c < p.chunks; c += 64u) {
            const double off = at[2 * c] - near, sum = (c + 1u < p.chunks ? full : last) * off;
            t1 += sum;
            t2 += __builtin_fma(sum, off, at[2 * c + 1]);
        }
        const Moments v = moments_of(a, p, near, wave_sum(t1), wave_sum(t2));
        if ((threadIdx.x & 63u) == 0) {
            stats[2 * i] = v.mean;
            stats[2 * i + 1] = v.rstd;
        }
    }
}

template <uint32_t T, uint32_t F, bool EVEN>
__global__ __launch_bounds__(kMaxThreads) void k_norm_apply(NormArgs a, Plan p, const double *stats)
{
    typedef typename ElemOf<T>::type E;
    const Place q = place(p, blockIdx.x, 0, a.channels);
    const uint32_t beg = q.chunk * p.rows_per, end = a.spatial - beg < p.rows_per ? a.spatial : beg + p.rows_per;
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    const E *src = static_cast<const E *>(a.x) + (q.valid > 0 ? q.c : 0);
    auto fetch = [&](uint32_t base) {
        const uint32_t r = base + q.r;
        const int n = r < end ? q.valid : 0;
        return load_vector<T, EVEN>(src + (n > 0 ? (row0 + r) * a.channels : 0), n);
    };
    Line l = parameters_of(a, q);
    apply_moments(&l, p, q, 0, [&](uint32_t g) {
        const double *st = stats + ((uint64_t)q.n * a.groups + g) * 2;
        return group_of(st[0], st[1]);
    });
    if (F != kPlain) put_tail(a);
    // every thread of the workgroup goes round as often: the lanes of a quantisation group meet in put_outputs
    f32x8 next = fetch(beg);
    for (uint32_t base = beg; base < end; base += p.rp) {
        const f32x8 x = next;
        next = fetch(base + p.rp);                                        // behind the end: nothing
        const uint32_t r = base + q.r;
        put_outputs<T, F, EVEN>(a, q, l, x, row0 + r, r < end && q.r < p.rp);
    }
}

// ---- backward -----------------------------------------------------------------------------------------

// Eight values of the input as `v` * `s`: codes and their scale, or the values themselves and 1.
struct Source { f32x8 v; float s; };
template <uint32_t T, uint32_t S> struct Held {                           // as they lie in memory
    u32x4 w[T == kTypeF32 ? 2 : 1];
    // EVEN: eight values or none
    template <bool EVEN>
    __device__ __forceinline__ void load(const void *x, const NormArgs &a, uint64_t row, uint32_t c, int n)
    {
        typedef typename ElemOf<T>::type E;
        const E *p = static_cast<const E *>(x) + (n > 0 ? row * a.channels + c : 0);
        if constexpr (EVEN) {
#pragma unroll
            for (int k = 0; k < (int)(sizeof(w) / 16); ++k) w[k] = u32x4{0, 0, 0, 0};
            if (n > 0) __builtin_memcpy(w, p, sizeof(w));
            return;
        }
        if (n >= 8) { __builtin_memcpy(w, p, sizeof(w)); return; }
        E e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = k < n ? p[k] : (E)0.0f;
        __builtin_memcpy(w, e, sizeof(w));
    }
    __device__ __forceinline__ Source values() const
    {
        typename ElemOf<T>::type e[8];
        __builtin_memcpy(e, w, sizeof(w));
        Source r;
        r.s = 1.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) r.v[k] = (float)e[k];
        return r;
    }
};
template <uint32_t S> struct HeldCodes {
    u32x2 w;
    uint32_t e;
    template <bool>
    __device__ __forceinline__ void load(const void *, const NormArgs &a, uint64_t row, uint32_t c, int n)
    {
        w = u32x2{0, 0};
        e = 127;
        if (n > 0) {
            w = *reinterpret_cast<const u32x2 *>(a.codes + row * a.pitch + c);
            e = a.exps[row * a.ngroups + (c >> a.gshift)];
        }
    }
    __device__ __forceinline__ Source values() const
    {
        Source r;
        r.s = scale_of(e);
        if constexpr (S == kByteInt8) {
            uint32_t found = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t u = w[h] ^ 0x80808080u;                    // code + 128
                found |= (u - 0x01010101u) & ~u;                          // a byte of zero leaves its highest bit
#pragma unroll
                for (int k = 0; k < 4; ++k) r.v[4 * h + k] = (float)(int8_t)(w[h] >> (8 * k));
            }
            if (found & 0x80808080u) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (r.v[k] == -128.0f) r.v[k] = __uint_as_float(0x7fc00000u);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), q = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
                r.v[4 * h] = p[0]; r.v[4 * h + 1] = p[1]; r.v[4 * h + 2] = q[0]; r.v[4 * h + 3] = q[1];
            }
        }
        return r;
    }
};
template <uint32_t T, uint32_t S> using HeldAs = typename std::conditional<S == kPlain, Held<T, S>, HeldCodes<S>>::type;

// h' = (x - mean) * hr of a thread's channels, with the mean rounded to fp32.  What that rounding loses, hm = h - h', is the same
// for all of a group: it is put where the values are summed or used, so that nothing grows with the distance of the
// mean from zero and no value pays for it.  u = h' * gamma + beta, with hm * gamma in beta; B = B' + hm * A, and h B = h' B + hm B,
// of which the second part is put to A.  ONE: all of a vector's channels are in one group.
template <bool ONE> struct Channels { float mean[ONE ? 1 : 8], hr[ONE ? 1 : 8], gamma[8], beta[8]; };
__device__ __forceinline__ double lost_of(const double *st) { return ((double)(float)st[0] - st[0]) * st[1]; }
template <bool ONE>
__device__ __forceinline__ Channels<ONE> channels_of(const NormArgs &a, const Plan &p, const Place &q, float (&hm)[ONE ? 1 : 8])
{
    Channels<ONE> c;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        c.gamma[k] = c.beta[k] = 0.0f;
        if (k < q.valid) {
            c.gamma[k] = a.gamma ? a.gamma[q.c + k] : 1.0f;
            c.beta[k] = a.beta ? a.beta[q.c + k] : 0.0f;
        }
        if (k < (ONE ? 1 : 8)) {
            c.mean[k] = c.hr[k] = hm[k] = 0.0f;
            if (k < q.valid) {
                const double *st = a.stats + ((uint64_t)q.n * a.groups + p.div_per.div(q.c + k)) * 2;
                c.mean[k] = (float)st[0];
                c.hr[k] = (float)st[1];
                hm[k] = (float)lost_of(st);
            }
        }
        c.beta[k] = __builtin_fmaf(hm[ONE ? 0 : k], c.gamma[k], c.beta[k]);
    }
    return c;
}

// du = dy * act'(u) and h' of eight channels.  in: the position exists; h' of the zero that stands for one may be infinite.
template <uint32_t ACT, bool ONE>
__device__ __forceinline__ void gradient8(const NormArgs &a, const Plan &p, const Place &q, const Channels<ONE> &c, const Source &x,
                                          f32x8 dy, f32x8 *du, f32x8 *h, bool in = true)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float hk = __builtin_fmaf(x.v[k], x.s, -c.mean[ONE ? 0 : k]) * (in ? c.hr[ONE ? 0 : k] : 0.0f);
        (*h)[k] = hk;
        if constexpr (ACT == kActNone) {
            (*du)[k] = dy[k];
        } else {
            const float u = __builtin_fmaf(hk, c.gamma[k], c.beta[k]);
            if constexpr (ACT == kActSilu) {
                const float g = sigmoid(u);
                (*du)[k] = dy[k] * (g * __builtin_fmaf(u, 1.0f - g, 1.0f));
            } else {
                bool positive = u > 0.0f;
                // where fp32 cannot tell the side of the border (its error is below four roundings of these terms), fp64 does
                const float terms = __builtin_fmaf(fabsf(c.gamma[k]), fabsf(hk), fabsf(c.beta[k]));
                if (fabsf(u) < 0x1p-20f * terms && k < q.valid) {
                    uint32_t ch = q.c + k;
                    asm volatile("" : "+v"(ch));                           // rare: nothing of this is worth registers outside
                    const double *st = a.stats + ((uint64_t)q.n * a.groups + p.div_per.div(ch)) * 2;
                    const double v = ((double)x.v[k] * (double)x.s - st[0]) * st[1];
                    positive = v * (a.gamma ? (double)a.gamma[ch] : 1.0) + (a.beta ? (double)a.beta[ch] : 0.0) > 0.0;
                }
                (*du)[k] = positive ? dy[k] : u != u ? u : 0.0f;
            }
        }
    }
}

// gamma and hm of the segment's channels in LDS, for the waves that add up groups (a barrier follows).  ONE: hm once per vector,
// whose threads put hm * A to their own sums; eight registers for it in the others spill.
template <bool ONE> struct Shared {
    const float *gamma, *lost;
    __device__ __forceinline__ float hm(uint32_t c) const { return lost[ONE ? c >> 3 : c]; }
};
template <bool ONE>
__device__ __forceinline__ Shared<ONE> put_channels(float *s, const Plan &p, const Channels<ONE> &c, const float (&hm)[ONE ? 1 : 8])
{
    if (threadIdx.x < p.nv) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s[8u * threadIdx.x + k] = c.gamma[k];
            if (!ONE) s[8u * (p.nv + threadIdx.x) + k] = hm[ONE ? 0 : k];
        }
        if (ONE) s[8u * p.nv + threadIdx.x] = hm[0];
    }
    return {s, s + 8u * p.nv};
}

__device__ __forceinline__ void add_sums(f32x8 du, f32x8 h, float (&sp)[8], float (&sq)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        sp[k] += du[k];
        sq[k] = __builtin_fmaf(du[k], h[k], sq[k]);
    }
}

// dx = hr * (du * gamma - (A + h * B)); ga, gb: A + hm B and B of the channels' groups, divided by the count; h: h'.
template <bool ONE>
__device__ __forceinline__ f32x8 input_gradient(const Channels<ONE> &c, f32x8 du, f32x8 h, const float (&ga)[ONE ? 1 : 8],
                                                const float (&gb)[ONE ? 1 : 8])
{
    f32x8 dx;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float t = __builtin_fmaf(du[k], c.gamma[k], -ga[ONE ? 0 : k]);
        dx[k] = c.hr[ONE ? 0 : k] * __builtin_fmaf(-h[k], gb[ONE ? 0 : k], t);
    }
    return dx;
}

// A + hm B and B over the count, for a thread's channels, from s[2 * g], s[2 * g + 1]; channel `first` is the first group's.
template <bool ONE>
__device__ __forceinline__ void pick_totals(const double *s, const NormArgs &a, const Plan &p, const Place &q, uint32_t first,
                                            float (&ga)[ONE ? 1 : 8], float (&gb)[ONE ? 1 : 8])
{
#pragma unroll
    for (int k = 0; k < (ONE ? 1 : 8); ++k) {
        ga[k] = gb[k] = 0.0f;
        if (k < q.valid) {
            const uint32_t g = p.div_per.div(q.c + k - first);
            ga[k] = (float)(s[2 * g] * p.share);
            gb[k] = (float)(s[2 * g + 1] * p.share);
        }
    }
}

// dbeta and dgamma of sixteen channels: the sums of `records` workgroups or samples, in a fixed order.
__device__ __forceinline__ void join_parameters(double *s, const NormArgs &a, const float *chan, uint64_t records, uint32_t block,
                                                float *dbeta, float *dgamma)
{
    const uint32_t c = block * 16u + (threadIdx.x & 15u), parts = blockDim.x >> 4;
    double t[2] = {0.0, 0.0};
    if (c < a.channels) {
#pragma unroll 4
        for (uint64_t k = threadIdx.x >> 4; k < records; k += parts) {
            t[0] += (double)chan[2 * k * a.channels + c];
            t[1] += (double)chan[(2 * k + 1) * a.channels + c];
        }
    }
    for (int which = 0; which < 2; ++which) {
        float *out = which ? dgamma : dbeta;
        __syncthreads();
        s[threadIdx.x] = t[which];
        __syncthreads();
        if (threadIdx.x < 16u && c < a.channels && out) {
            double sum = 0.0;
#pragma unroll 16
            for (uint32_t k = 0; k < parts; ++k) sum += s[16u * k + threadIdx.x];
            out[c] = (float)sum;
        }
    }
}

// blocks: workgroups for all channels.  With `to` a workgroup joins one of several ranges of records to a record there.
__global__ __launch_bounds__(kMaxThreads) void k_norm_parameters(NormArgs a, const float *chan, uint64_t records, uint64_t range,
                                                                 uint32_t blocks, float *to)
{
    extern __shared__ __align__(16) double s_sum[];
    const uint32_t r = blockIdx.x / blocks, block = blockIdx.x - r * blocks;
    const uint64_t beg = r * range, n = records - beg < range ? records - beg : range;
    float *out = to + 2ull * r * a.channels;
    join_parameters(s_sum, a, chan + 2 * beg * a.channels, n, block, to ? out : a.dbeta, to ? out + a.channels : a.dgamma);
}

// Ranges that the records of many samples are joined in first, so that more than the few workgroups of the channels
// read them (100000 x 1 x 40, backward: 634 us with one step, 136 with two; 3000 x 9 x 256: 39.9 and 28.6); 1: a second launch would cost more.
uint32_t parameter_ranges(const NormArgs &a, uint64_t records)
{
    const uint32_t blocks = (a.channels + 15) / 16;
    return records < 2048 || blocks >= 256 ? 1 : 512 / blocks;
}

template <uint32_t T, uint32_t S, uint32_t ACT, bool ONE>
__global__ __launch_bounds__(kMaxThreads) void k_norm_grad_slab(NormArgs a, Plan p)
{
    extern __shared__ __align__(16) double s_sum[];
    typedef typename ElemOf<T>::type E;
    Place q = place(p, blockIdx.x, 0, 0);
    const uint32_t first = q.chunk * p.nv * 8u, end = a.channels - first < p.nv * 8u ? a.channels : first + p.nv * 8u;
    q = place(p, blockIdx.x, first, end);
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    float *s = reinterpret_cast<float *>(s_sum);
    float hm[ONE ? 1 : 8];
    const Channels<ONE> ch = channels_of<ONE>(a, p, q, hm);
    Held<T, kPlain> dy[kSlabRows];
    HeldAs<T, S> x[kSlabRows];
#pragma unroll
    for (uint32_t i = 0; i < kSlabRows; ++i) {
        const uint32_t r = q.r + i * p.rp;
        const int n = r < a.spatial ? q.valid : 0;
        dy[i].template load<ONE>(a.dy, a, row0 + r, q.c, n);
        x[i].template load<ONE>(a.x, a, row0 + r, q.c, n);
    }
    const Shared<ONE> sc = put_channels<ONE>(s + blockDim.x * 16u, p, ch, hm);
    float sp[8], sq[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sp[k] = sq[k] = 0.0f;
    f32x8 du, h;
#pragma unroll
    for (uint32_t i = 0; i < kSlabRows; ++i) {
        if (i * p.rp >= a.spatial) break;                                 // (uniform)
        gradient8<ACT, ONE>(a, p, q, ch, x[i].values(), dy[i].values().v, &du, &h, q.r + i * p.rp < a.spatial);
        add_sums(du, h, sp, sq);
    }
    double *tot = s_sum + 8u * blockDim.x + 8u * p.nv;
    const float *s2 = s + blockDim.x * 8u;
    auto sum_h = [&](uint32_t c) { return ONE ? s2[c] : __builtin_fmaf(sc.hm(c), s[c], s2[c]); };   // of du * h
    if (ONE) {
#pragma unroll
        for (int k = 0; k < 8; ++k) sq[k] = __builtin_fmaf(hm[0], sp[k], sq[k]);
    }
    join_channels(s, sp, sq, p);
    const uint32_t groups = (end - first) / p.per, w = lanes_of(p.per);
    const bool params = a.dbeta || a.dgamma;
    for (uint32_t c = threadIdx.x; params && c < end - first; c += blockDim.x) {
        if (a.batch == 1) {
            if (a.dbeta) a.dbeta[first + c] = s[c];
            if (a.dgamma) a.dgamma[first + c] = sum_h(c);
        } else {
            float *chan = static_cast<float *>(a.work) + 2ull * q.n * a.channels + first + c;
            chan[0] = s[c];
            chan[a.channels] = sum_h(c);
        }
    }
    each_group(groups, w, [&](uint32_t g, uint32_t sub, bool mine) {
        const double t1 = group_total(g, p.per, sub, w, [&](uint32_t c) { return (double)s[c] * (double)sc.gamma[c]; });
        const double t2 = group_total(g, p.per, sub, w, [&](uint32_t c) { return (double)sum_h(c) * (double)sc.gamma[c]; });
        if (mine) { tot[2 * g] = t1 + (double)sc.hm(g * p.per) * t2; tot[2 * g + 1] = t2; }
    });
    __syncthreads();
    float ga[ONE ? 1 : 8], gb[ONE ? 1 : 8];
    pick_totals<ONE>(tot, a, p, q, first, ga, gb);
#pragma unroll
    for (uint32_t i = 0; i < kSlabRows; ++i) {
        const uint32_t r = q.r + i * p.rp;
        if (r >= a.spatial || q.valid <= 0) break;
        gradient8<ACT, ONE>(a, p, q, ch, x[i].values(), dy[i].values().v, &du, &h);
        store8<T>(static_cast<E *>(a.y) + (row0 + r) * a.channels + q.c, input_gradient<ONE>(ch, du, h, ga, gb), q.valid);
    }
}

// Two positions of a thread at a time, all their loads in flight: take(position, du, h).
template <uint32_t T, uint32_t S, uint32_t ACT, bool ONE, class FN>
__device__ __forceinline__ void each_gradient(const NormArgs &a, const Plan &p, const Place &q, const Channels<ONE> &ch, FN take)
{
    const uint32_t beg = q.chunk * p.rows_per, end = a.spatial - beg < p.rows_per ? a.spatial : beg + p.rows_per;
    const uint64_t row0 = (uint64_t)q.n * a.spatial;
    if (q.valid <= 0 || q.r >= end - beg) return;
    uint32_t left = (end - beg - q.r + p.rp - 1) / p.rp;                  // positions of this thread
    uint64_t row = row0 + beg + q.r;
    const int n = ONE ? 8 : q.valid;
    auto one = [&](const Held<T, kPlain> &dy, const HeldAs<T, S> &x, uint64_t at) {
        f32x8 du, h;
        gradient8<ACT, ONE>(a, p, q, ch, x.values(), dy.values().v, &du, &h);
        take(at, du, h);
    };
    for (; left >= 2; left -= 2, row += 2 * p.rp) {
        Held<T, kPlain> dy[2];
        HeldAs<T, S> x[2];
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            dy[i].template load<false>(a.dy, a, row + i * p.rp, q.c, n);
            x[i].template load<false>(a.x, a, row + i * p.rp, q.c, n);
        }
        one(dy[0], x[0], row);
        one(dy[1], x[1], row + p.rp);
    }
    if (left) {
        Held<T, kPlain> dy;
        HeldAs<T, S> x;
        dy.template load<false>(a.dy, a, row, q.c, n);
        x.template load<false>(a.x, a, row, q.c, n);
        one(dy, x, row);
    }
}

template <uint32_t T, uint32_t S, uint32_t ACT, bool ONE>
__global__ __launch_bounds__(kMaxThreads) void k_norm_grad_sums(NormArgs a, Plan p)
{
    extern __shared__ __align__(16) double s_sum[];
    const Place q = place(p, blockIdx.x, 0, a.channels);
    float *s = reinterpret_cast<float *>(s_sum);
    float hm[ONE ? 1 : 8];
    const Channels<ONE> ch = channels_of<ONE>(a, p, q, hm);
    const Shared<ONE> sc = put_channels<ONE>(s + blockDim.x * 16u, p, ch, hm);
    float sp[8], sq[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sp[k] = sq[k] = 0.0f;
    each_gradient<T, S, ACT, ONE>(a, p, q, ch, [&](uint64_t, f32x8 du, f32x8 h) { add_sums(du, h, sp, sq); });
    const float *s2 = s + blockDim.x * 8u;
    auto sum_h = [&](uint32_t c) { return ONE ? s2[c] : __builtin_fmaf(sc.hm(c), s[c], s2[c]); };   // of du * h
    if (ONE) {
#pragma unroll
        for (int k = 0; k < 8; ++k) sq[k] = __builtin_fmaf(hm[0], sp[k], sq[k]);
    }
    join_channels(s, sp, sq, p);
    const uint32_t w = lanes_of(p.per);
    double *part = static_cast<double *>(a.work);
    float *chan = reinterpret_cast<float *>(part + 2ull * a.batch * a.groups * p.chunks) + 2ull * blockIdx.x * a.channels;
    const bool params = a.dbeta || a.dgamma;
    for (uint32_t c = threadIdx.x; params && c < a.channels; c += blockDim.x) {
        chan[c] = s[c];
        chan[a.channels + c] = sum_h(c);
    }
    each_group(a.groups, w, [&](uint32_t g, uint32_t sub, bool mine) {
        const double t1 = group_total(g, p.per, sub, w, [&](uint32_t c) { return (double)s[c] * (double)sc.gamma[c]; });
        const double t2 = group_total(g, p.per, sub, w, [&](uint32_t c) { return (double)sum_h(c) * (double)sc.gamma[c]; });
        double *o = part + (((uint64_t)q.n * a.groups + g) * p.chunks + q.chunk) * 2;
        if (mine) { o[0] = t1; o[1] = t2; }
    });
}

// Between the two passes: the totals A + hm B and B of every sample and group, and the parameters' gradients.
__global__ __launch_bounds__(kMaxThreads) void k_norm_grad_join(NormArgs a, Plan p, double *totals, uint32_t param_blocks)
{
    extern __shared__ __align__(16) double s_sum[];
    const double *part = static_cast<const double *>(a.work);
    if (blockIdx.x < param_blocks) {
        join_parameters(s_sum, a, reinterpret_cast<const float *>(part + 2ull * a.batch * a.groups * p.chunks),
                        a.spatial ? a.batch * p.chunks : 0, blockIdx.x, a.dbeta, a.dgamma);
        return;
    }
    const uint64_t step = (gridDim.x - param_blocks) * 16ull;
    for (uint64_t i = (blockIdx.x - param_blocks) * 16ull + (threadIdx.x >> 6); i < a.batch * a.groups; i += step) {
        const Totals t = join_chunks(part, i, p);
        if ((threadIdx.x & 63u) == 0) {
            totals[2 * i] = t.t1 + lost_of(a.stats + 2 * i) * t.t2;
            totals[2 * i + 1] = t.t2;
        }
    }
}

template <uint32_t T, uint32_t S, uint32_t ACT, bool ONE>
__global__ __launch_bounds__(kMaxThreads) void k_norm_grad_apply(NormArgs a, Plan p, const double *totals)
{
    typedef typename ElemOf<T>::type E;
    const Place q = place(p, blockIdx.x, 0, a.channels);
    float hm[ONE ? 1 : 8];
    const Channels<ONE> ch = channels_of<ONE>(a, p, q, hm);
    float ga[ONE ? 1 : 8], gb[ONE ? 1 : 8];
    pick_totals<ONE>(totals + 2ull * q.n * a.groups, a, p, q, 0, ga, gb);
    each_gradient<T, S, ACT, ONE>(a, p, q, ch, [&](uint64_t row, f32x8 du, f32x8 h) {
        store8<T>(static_cast<E *>(a.y) + row * a.channels + q.c, input_gradient<ONE>(ch, du, h, ga, gb), q.valid);
    });
}

// ---- launches -----------------------------------------------------------------------------------------

// LDS of a workgroup: `per_thread` bytes for each of its threads, and two doubles per group (behind them, or instead).
size_t lds_bytes(const Plan &p, size_t per_thread, size_t groups, bool both)
{
    const size_t joined = p.threads * per_thread, totals = 16 * groups;
    return both ? joined + totals : joined > totals ? joined : totals;
}
uint32_t join_blocks(const NormArgs &a)                                   // sixteen waves, a sample and group each
{
    const uint64_t n = (a.batch * a.groups + kMaxThreads / 64 - 1) / (kMaxThreads / 64);
    return (uint32_t)(n < 65536 ? n : 65536);
}
// What the first pass leaves in the workspace: two totals per sample, range and group; for the parameters' gradients two sums
// per channel behind them.
uint64_t records_bytes(const NormArgs &a, const Plan &p, bool params)
{
    const uint64_t records = a.batch * p.chunks;
    return (records * (16ull * a.groups + (params ? 8ull * a.channels : 0ull)) + 15) & ~15ull;
}
uint32_t lanes_of_group(uint32_t group) { return group ? group / 8u : 1u; }   // threads of a position that share a scale
size_t moment_bytes(const Plan &p) { return p.per < 8u ? 128 : 32; }

template <uint32_t T, uint32_t F, bool EVEN>
void forward_as(const NormArgs &a, hipStream_t st)
{
    const uint32_t lanes = lanes_of_group(F != kPlain ? 1u << a.gshift : 0u);
    Plan p;
    if (slab_plan(&p, a, lanes)) {
        hipLaunchKernelGGL((k_norm_slab<T, F, EVEN>), dim3((uint32_t)(a.batch * p.chunks)), dim3(p.threads),
                           lds_bytes(p, moment_bytes(p), p.nv * 8u / p.per, true), st, a, p);
        return;
    }
    p = two_pass_plan(a, lanes);
    const dim3 grid((uint32_t)(a.batch * p.chunks)), block(p.threads);
    hipLaunchKernelGGL((k_norm_sums<T, EVEN>), grid, block, lds_bytes(p, moment_bytes(p), 0, false), st, a, p);
    double *stats = a.stats ? a.stats : static_cast<double *>(a.work) + 2ull * a.batch * a.groups * p.chunks;
    hipLaunchKernelGGL(k_norm_join, dim3(join_blocks(a)), dim3(kMaxThreads), 0, st, a, p, stats);
    hipLaunchKernelGGL((k_norm_apply<T, F, EVEN>), grid, block, 0, st, a, p, stats);
}

template <uint32_t T, uint32_t S, uint32_t ACT, bool ONE>
void backward_as(const NormArgs &a, hipStream_t st)
{
    const uint32_t params = a.dgamma || a.dbeta ? (a.channels + 15) / 16 : 0;
    Plan p;
    if (a.batch && slab_plan(&p, a, 1)) {
        hipLaunchKernelGGL((k_norm_grad_slab<T, S, ACT, ONE>), dim3((uint32_t)(a.batch * p.chunks)), dim3(p.threads),
                           lds_bytes(p, 64, p.nv * 8u / p.per, true) + 64 * p.nv, st, a, p);
        if (!params || a.batch == 1) return;
        const float *chan = static_cast<const float *>(a.work);
        uint64_t records = a.batch;
        const uint32_t ranges = parameter_ranges(a, records);
        if (ranges > 1) {
            const uint64_t range = (records + ranges - 1) / ranges, used = (records + range - 1) / range;
            float *to = static_cast<float *>(a.work) + 2 * records * a.channels;
            hipLaunchKernelGGL(k_norm_parameters, dim3((uint32_t)used * params), dim3(kMaxThreads), 8 * kMaxThreads, st, a, chan, records, range,
                               params, to);
            chan = to;
            records = used;
        }
        hipLaunchKernelGGL(k_norm_parameters, dim3(params), dim3(kMaxThreads), 8 * kMaxThreads, st, a, chan, records, records, params,
                           static_cast<float *>(nullptr));
        return;
    }
    p = two_pass_plan(a, 1);
    const uint32_t work = a.spatial ? (uint32_t)(a.batch * p.chunks) : 0;
    double *totals = reinterpret_cast<double *>(static_cast<uint8_t *>(a.work) + records_bytes(a, p, params != 0));
    const uint32_t joins = work ? join_blocks(a) : 0;
    if (work)
        hipLaunchKernelGGL((k_norm_grad_sums<T, S, ACT, ONE>), dim3(work), dim3(p.threads), lds_bytes(p, 64, 0, false) + 64 * p.nv, st, a, p);
    if (params + joins)
        hipLaunchKernelGGL(k_norm_grad_join, dim3(params + joins), dim3(kMaxThreads), 8 * kMaxThreads, st, a, p, totals, params);
    if (work) hipLaunchKernelGGL((k_norm_grad_apply<T, S, ACT, ONE>), dim3(work), dim3(p.threads), 0, st, a, p, totals);
}

template <uint32_t T, uint32_t S, uint32_t ACT>
void backward_act(const NormArgs &a, hipStream_t st)
{
    if (a.channels / a.groups % 8 == 0) backward_as<T, S, ACT, true>(a, st);
    else backward_as<T, S, ACT, false>(a, st);
}

template <uint32_t T, uint32_t S>
void backward_from(const NormArgs &a, hipStream_t st)
{
    if (a.act == kActSilu) backward_act<T, S, kActSilu>(a, st);
    else if (a.act == kActRelu) backward_act<T, S, kActRelu>(a, st);
    else backward_act<T, S, kActNone>(a, st);
}

template <uint32_t T>
void backward_of(const NormArgs &a, hipStream_t st)
{
    if (!a.codes) backward_from<T, kPlain>(a, st);
    else if (a.format == kByteInt8) backward_from<T, kByteInt8>(a, st);
    else backward_from<T, kByteE4M3>(a, st);
}

template <uint32_t T, bool EVEN>
void forward_to(const NormArgs &a, hipStream_t st)
{
    if (!a.codes) forward_as<T, kPlain, EVEN>(a, st);
    else if (a.format == kByteInt8) forward_as<T, kByteInt8, EVEN>(a, st);
    else forward_as<T, kByteE4M3, EVEN>(a, st);
}

template <uint32_t T>
void forward_of(const NormArgs &a, hipStream_t st)
{
    if (a.channels % 8 == 0) forward_to<T, true>(a, st);
    else forward_to<T, false>(a, st);
}

}  // namespace

uint64_t group_norm_forward_work(const NormArgs &a, uint32_t group)
{
    const uint32_t lanes = lanes_of_group(group);
    Plan p;
    if (slab_plan(&p, a, lanes)) return 0;
    return records_bytes(a, two_pass_plan(a, lanes), false) + 16ull * a.batch * a.groups;   // and mean and deviation, if nobody wants them
}

uint64_t group_norm_grad_work(const NormArgs &a, bool params)
{
    Plan p;
    if (slab_plan(&p, a, 1)) return params && a.batch > 1 ? 8ull * (a.batch + parameter_ranges(a, a.batch)) * a.channels : 0;   // sums of every sample
    return records_bytes(a, two_pass_plan(a, 1), params) + 16ull * a.batch * a.groups;
}

uint64_t group_norm_work(const NormArgs &a)
{
    uint64_t most = group_norm_grad_work(a, true);
    for (uint32_t group : {0u, 32u, 64u, 128u}) {
        const uint64_t bytes = group_norm_forward_work(a, group);
        if (bytes > most) most = bytes;
    }
    return most;
}

void launch_group_norm(const NormArgs &a, hipStream_t st)
{
    if (a.type == kTypeF32) forward_of<kTypeF32>(a, st);
    else if (a.type == kTypeF16) forward_of<kTypeF16>(a, st);
    else forward_of<kTypeBF16>(a, st);
}

void launch_group_norm_grad(const NormArgs &a, hipStream_t st)
{
    if (a.type == kTypeF32) backward_of<kTypeF32>(a, st);
    else if (a.type == kTypeF16) backward_of<kTypeF16>(a, st);
    else backward_of<kTypeBF16>(a, st);
}

}  // namespace cmpz
