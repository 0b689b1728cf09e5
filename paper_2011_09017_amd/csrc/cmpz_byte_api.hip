// C entry points of the byte checkpoints and of the operators that read and write them: argument checks and
// launches; nothing here allocates, waits or keeps anything between calls.
#include "../../include/cmpz.h"
#include "cmpz_byte.h"

#include <cmath>

using namespace cmpz;

namespace {

constexpr uint64_t kMost = (1ull << 31) - 1;           // rows, columns, positions
constexpr uint64_t kMostWide = 1ull << 24;             // a product's columns and rows of dY: offsets within 32 rows are kept in 32 bits

struct DeviceGuard {
    int prev = -1;
    int rc = CMP_OK;
    explicit DeviceGuard(int dev)
    {
        if (dev < 0) { rc = CMP_E_ARG; return; }
        if (hipGetDevice(&prev) != hipSuccess) { prev = -1; rc = CMP_E_HIP; return; }
        if (prev == dev) { prev = -1; return; }
        const hipError_t e = hipSetDevice(dev);
        if (e == hipSuccess) return;
        (void)hipGetLastError();                                          // it would come back from the next call that asks
        rc = e == hipErrorInvalidDevice ? CMP_E_ARG : CMP_E_HIP;
        prev = -1;
    }
    ~DeviceGuard() { if (prev >= 0) (void)hipSetDevice(prev); }
};

int launched() { return hipGetLastError() == hipSuccess ? CMP_OK : CMP_E_HIP; }

bool misaligned(const void *p, uint32_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1u)) != 0; }

bool shape_ok(const cmp_byte_shape *s)
{
    return s && s->rows <= kMost && s->cols <= kMost && (s->format == CMP_BYTE_INT || s->format == CMP_BYTE_FLOAT) &&
           (s->group == 32 || s->group == 64 || s->group == 128);
}

// Workgroups of a product are counted by a launch.
bool product_ok(const cmp_byte_shape &s, uint64_t outs)
{
    return s.cols <= kMostWide && outs <= kMostWide && outs * s.cols <= 1ull << 36;
}

uint32_t gshift_of(uint32_t group) { return group == 32 ? 5u : group == 64 ? 6u : 7u; }

// The parts of a checkpoint in `buf`; CMP_E_ARG / `small` where there is none or it is too small.
template <class ARGS>
int place_checkpoint(ARGS *a, const cmp_byte_shape &s, const void *buf, uint64_t bytes, int small)
{
    const ByteLayout l = byte_layout(s.rows, s.cols, s.group);
    if (bytes < l.total) return small;
    if (l.total && (!buf || misaligned(buf, 16))) return CMP_E_ARG;
    uint8_t *p = static_cast<uint8_t *>(const_cast<void *>(buf));
    a->codes = p;
    a->exps = p ? p + l.off_exps : nullptr;
    a->pitch = l.pitch;
    a->ngroups = l.ngroups;
    a->format = s.format;
    a->gshift = gshift_of(s.group);
    return CMP_OK;
}

int byte_args(ByteArgs *a, const cmp_byte_shape *s, const void *x, uint32_t type, uint64_t ld, const void *buf, uint64_t bytes,
              int small)
{
    if (!shape_ok(s) || type > CMP_TYPE_BF || ld < s->cols) return CMP_E_ARG;
    const bool empty = s->rows == 0 || s->cols == 0;
    if (!empty && (!x || misaligned(x, type_bytes(type)))) return CMP_E_ARG;
    const int rc = place_checkpoint(a, *s, buf, bytes, small);
    if (rc != CMP_OK) return rc;
    const ByteLayout l = byte_layout(s->rows, s->cols, s->group);
    a->x = const_cast<void *>(x);
    a->ld = ld;
    a->tail_from = l.used;
    a->tail_to = l.total;
    a->rows = (uint32_t)s->rows;
    a->cols = (uint32_t)s->cols;
    a->type = type;
    return CMP_OK;
}

int norm_args(NormArgs *a, const cmp_norm_shape *s)
{
    if (!s || s->spatial > kMost || s->batch > CMP_NORM_MAX_BATCH || s->batch * s->spatial > kMost) return CMP_E_ARG;
    if (s->channels < 1 || s->channels > CMP_NORM_MAX_CHANNELS || s->groups < 1 || s->groups > CMP_NORM_MAX_GROUPS) return CMP_E_ARG;
    if (s->channels % s->groups || s->type > CMP_TYPE_BF || s->act > CMP_ACT_SILU) return CMP_E_ARG;
    if (!(s->eps > 0.0) || !std::isfinite(s->eps)) return CMP_E_ARG;
    *a = NormArgs{};
    a->batch = s->batch;
    a->spatial = (uint32_t)s->spatial;
    a->channels = s->channels;
    a->groups = s->groups;
    a->type = s->type;
    a->act = s->act;
    a->eps = s->eps;
    a->gshift = 3;
    return CMP_OK;
}

// The checkpoint of a norm's input: one row per position.
int norm_checkpoint(NormArgs *a, const cmp_norm_shape &s, uint32_t format, uint32_t group, const void *buf, uint64_t bytes, int small)
{
    const cmp_byte_shape b{s.batch * s.spatial, s.channels, format, group};
    if (!shape_ok(&b)) return CMP_E_ARG;
    const int rc = place_checkpoint(a, b, buf, bytes, small);
    const ByteLayout l = byte_layout(b.rows, b.cols, b.group);
    a->tail_from = l.used;
    a->tail_to = l.total;
    return rc;
}

int norm_forward(int device, const cmp_norm_shape *shape, const void *d_x, const float *d_gamma, const float *d_beta, void *d_y,
                 double *d_stats, uint32_t format, uint32_t group, void *d_ck, size_t cap, void *d_work, size_t work_bytes,
                 void *stream, bool either)
{
    NormArgs a;
    int rc = norm_args(&a, shape);
    if (rc != CMP_OK) return rc;
    const bool empty = shape->batch == 0 || shape->spatial == 0;
    const uint32_t es = type_bytes(shape->type);
    if (!empty && (!d_x || !d_y || misaligned(d_x, es) || misaligned(d_y, es))) return CMP_E_ARG;
    if (misaligned(d_gamma, 4) || misaligned(d_beta, 4) || misaligned(d_stats, 8)) return CMP_E_ARG;
    if (d_ck && (rc = norm_checkpoint(&a, *shape, format, group, d_ck, cap, CMP_E_NOSPACE)) != CMP_OK) return rc;
    const uint64_t need = empty ? 0 : either ? group_norm_work(a) : group_norm_forward_work(a, d_ck ? group : 0);
    if (work_bytes < need) return CMP_E_NOSPACE;
    if (need && (!d_work || misaligned(d_work, 16))) return CMP_E_ARG;
    DeviceGuard guard(device);
    if (guard.rc != CMP_OK) return guard.rc;
    if (empty) return CMP_OK;
    a.x = d_x;
    a.y = d_y;
    a.gamma = d_gamma;
    a.beta = d_beta;
    a.stats = d_stats;
    a.work = d_work;
    launch_group_norm(a, static_cast<hipStream_t>(stream));
    return launched();
}

}  // namespace

extern "C" {

size_t cmp_byte_bytes(const cmp_byte_shape *shape)
{
    return shape_ok(shape) ? (size_t)byte_layout(shape->rows, shape->cols, shape->group).total : 0;
}

int cmp_byte_store(int device, const cmp_byte_shape *shape, const void *d_x, uint32_t type, uint64_t ld, void *d_ck, size_t cap,
                   void *stream)
{
    ByteArgs a{};
    const int rc = byte_args(&a, shape, d_x, type, ld, d_ck, cap, CMP_E_NOSPACE);
    if (rc != CMP_OK) return rc;
    DeviceGuard guard(device);
    if (guard.rc != CMP_OK) return guard.rc;
    if (a.rows == 0 || a.cols == 0) return CMP_OK;
    launch_byte_store(a, static_cast<hipStream_t>(stream));
    return launched();
}

int cmp_byte_load(int device, const cmp_byte_shape *shape, const void *d_ck, size_t bytes, void *d_out, uint32_t type, uint64_t ld,
                  void *stream)
{
    ByteArgs a{};
    const int rc = byte_args(&a, shape, d_out, type, ld, d_ck, bytes, CMP_E_FORMAT);
    if (rc != CMP_OK) return rc;
    DeviceGuard guard(device);
    if (guard.rc != CMP_OK) return guard.rc;
    if (a.rows == 0 || a.cols == 0) return CMP_OK;
    launch_byte_load(a, static_cast<hipStream_t>(stream));
    return launched();
}

size_t cmp_byte_linear_grad_work(const cmp_byte_shape *shape, uint64_t outs, uint32_t type)
{
    if (!shape_ok(shape) || !product_ok(*shape, outs) || type > CMP_TYPE_BF) return 0;
    return (size_t)linear_grad_work(shape->rows, shape->cols, outs, type);
}

int cmp_byte_linear_grad(int device, const cmp_byte_shape *shape, const void *d_ck, size_t bytes, const void *d_dy, uint32_t type,
                         uint64_t outs, uint64_t ld_dy, void *d_dw, void *d_db, uint32_t out_type, int accumulate, void *d_work,
                         size_t work_bytes, void *stream)
{
    LinearGradArgs a{};
    if (!shape_ok(shape) || !product_ok(*shape, outs) || ld_dy < outs || ld_dy > kMostWide || type > CMP_TYPE_BF) return CMP_E_ARG;
    if (out_type != type && out_type != CMP_TYPE_F) return CMP_E_ARG;
    const uint32_t es = type_bytes(type), os = type_bytes(out_type);
    if (shape->rows && outs && (!d_dy || misaligned(d_dy, es))) return CMP_E_ARG;
    if (shape->cols && outs && (!d_dw || misaligned(d_dw, os))) return CMP_E_ARG;
    if (d_db && misaligned(d_db, os)) return CMP_E_ARG;
    const int rc = place_checkpoint(&a, *shape, d_ck, bytes, CMP_E_FORMAT);
    if (rc != CMP_OK) return rc;
    const uint64_t need = linear_grad_work(shape->rows, shape->cols, outs, type);
    if (work_bytes < need) return CMP_E_NOSPACE;
    if (need && (!d_work || misaligned(d_work, 16))) return CMP_E_ARG;
    DeviceGuard guard(device);
    if (guard.rc != CMP_OK) return guard.rc;
    if (outs == 0 || (shape->cols == 0 && !d_db)) return CMP_OK;
    a.dy = d_dy;
    a.ld_dy = ld_dy;
    a.dw = d_dw;
    a.db = d_db;
    a.work = static_cast<float *>(d_work);
    a.rows = (uint32_t)shape->rows;
    a.cols = (uint32_t)shape->cols;
    a.outs = (uint32_t)outs;
    a.type = type;
    a.out_type = out_type;
    a.accumulate = accumulate ? 1u : 0u;
    launch_linear_grad(a, static_cast<hipStream_t>(stream));
    return launched();
}

size_t cmp_group_norm_work(const cmp_norm_shape *shape)
{
    NormArgs a;
    if (norm_args(&a, shape) != CMP_OK) return 0;
    return a.batch && a.spatial ? (size_t)group_norm_work(a) : 0;
}

size_t cmp_group_norm_forward_work(const cmp_norm_shape *shape, uint32_t group)
{
    NormArgs a;
    if (norm_args(&a, shape) != CMP_OK || (group != 0 && group != 32 && group != 64 && group != 128)) return 0;
    return a.batch && a.spatial ? (size_t)group_norm_forward_work(a, group) : 0;
}

size_t cmp_group_norm_grad_work(const cmp_norm_shape *shape, int params)
{
    NormArgs a;
    if (norm_args(&a, shape) != CMP_OK) return 0;
    return a.batch && a.spatial ? (size_t)group_norm_grad_work(a, params != 0) : 0;
}

int cmp_group_norm(int device, const cmp_norm_shape *shape, const void *d_x, const float *d_gamma, const float *d_beta, void *d_y,
                   double *d_stats, uint32_t format, uint32_t group, void *d_ck, size_t cap, void *d_work, size_t work_bytes,
                   void *stream)
{
    return norm_forward(device, shape, d_x, d_gamma, d_beta, d_y, d_stats, format, group, d_ck, cap, d_work, work_bytes, stream, true);
}

int cmp_group_norm_forward(int device, const cmp_norm_shape *shape, const void *d_x, const float *d_gamma, const float *d_beta, void *d_y,
                           double *d_stats, uint32_t format, uint32_t group, void *d_ck, size_t cap, void *d_work, size_t work_bytes,
                           void *stream)
{
    return norm_forward(device, shape, d_x, d_gamma, d_beta, d_y, d_stats, format, group, d_ck, cap, d_work, work_bytes, stream, false);
}

int cmp_group_norm_grad(int device, const cmp_norm_shape *shape, const void *d_dy, const void *d_x, uint32_t format, uint32_t group,
                        const void *d_ck, size_t bytes, const float *d_gamma, const float *d_beta, const double *d_stats, void *d_dx,
                        float *d_dgamma, float *d_dbeta, void *d_work, size_t work_bytes, void *stream)
{
    NormArgs a;
    int rc = norm_args(&a, shape);
    if (rc != CMP_OK) return rc;
    const bool empty = shape->batch == 0 || shape->spatial == 0;
    const uint32_t es = type_bytes(shape->type);
    if (!empty && (!d_dy || !d_dx || !d_stats || misaligned(d_dy, es) || misaligned(d_dx, es))) return CMP_E_ARG;
    if (!empty && !d_x == !d_ck) return CMP_E_ARG;                        // the input or its checkpoint, not both
    if (misaligned(d_x, es) || misaligned(d_gamma, 4) || misaligned(d_beta, 4) || misaligned(d_stats, 8) || misaligned(d_dgamma, 4) ||
        misaligned(d_dbeta, 4))
        return CMP_E_ARG;
    if (d_ck && (rc = norm_checkpoint(&a, *shape, format, group, d_ck, bytes, CMP_E_FORMAT)) != CMP_OK) return rc;
    const uint64_t need = empty ? 0 : group_norm_grad_work(a, d_dgamma || d_dbeta);
    if (work_bytes < need) return CMP_E_NOSPACE;
    if (need && (!d_work || misaligned(d_work, 16))) return CMP_E_ARG;
    DeviceGuard guard(device);
    if (guard.rc != CMP_OK) return guard.rc;
    a.x = d_x;
    a.dy = d_dy;
    a.y = d_dx;
    a.gamma = d_gamma;
    a.beta = d_beta;
    a.dgamma = d_dgamma;
    a.dbeta = d_dbeta;
    a.stats = const_cast<double *>(d_stats);
    a.work = d_work;
    launch_group_norm_grad(a, static_cast<hipStream_t>(stream));
    return launched();
}

}  // extern "C"
