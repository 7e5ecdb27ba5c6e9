// What the entry points check their arguments with, on the host, before any HIP call (api.hip, layers_api.hip).
#pragma once

#include <cstddef>
#include <cstdint>

#include "ssmv.h"

namespace ssmv {

// The status `code`, its text kept for ssmv_last_error of this thread (api.hip).
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(int hip_code, const char *what);

inline size_t io_bytes(int io) { return io == SSMV_BF16 ? 2 : 4; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_ptr(const void *p, const char *name)
{
    if (!p) return fail(SSMV_EINVAL, "%s is NULL", name);
    if (!aligned16(p)) return fail(SSMV_EALIGN, "%s (%p) is not 16-byte aligned", name, p);
    return SSMV_OK;
}

inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// a tensor of the I/O type that needs only its elements' alignment
inline int check_io(const void *p, int io, const char *name)
{
    if (!p) return fail(SSMV_EINVAL, "%s is NULL", name);
    if (!aligned_to(p, io_bytes(io))) return fail(SSMV_EALIGN, "%s (%p) is not aligned to its elements", name, p);
    return SSMV_OK;
}

inline int check_f32(const void *p, const char *name)
{
    if (!p) return fail(SSMV_EINVAL, "%s is NULL", name);
    if (!aligned_to(p, 4)) return fail(SSMV_EALIGN, "%s (%p) is not 4-byte aligned", name, p);
    return SSMV_OK;
}

// 0 = packed
inline int check_stride(int64_t *stride, long packed, const char *name)
{
    if (*stride == 0) *stride = packed;
    if (*stride < packed || *stride > (int64_t)1 << 40)
        return fail(SSMV_EINVAL, "%s %lld: rows of %ld elements would overlap, or it is beyond 2^40", name, (long long)*stride, packed);
    return SSMV_OK;
}

inline int check_io_type(int io)
{
    return io == SSMV_F32 || io == SSMV_BF16 ? SSMV_OK : fail(SSMV_EINVAL, "io_dtype %d unknown", io);
}

inline int check_rows(int32_t *rows_in, int rows, const int32_t *src_row)
{
    if (*rows_in == 0) *rows_in = rows;
    if (*rows_in < 0) return fail(SSMV_EINVAL, "rows_in %d < 0", *rows_in);
    if (!src_row && *rows_in < rows) return fail(SSMV_EINVAL, "rows_in %d < %d rows that go out, and no src_row", *rows_in, rows);
    if (!aligned_to(src_row, 4)) return fail(SSMV_EALIGN, "src_row is not 4-byte aligned");
    return SSMV_OK;
}

#define TRY(call) do { const int rc_ = (call); if (rc_ != SSMV_OK) return rc_; } while (0)

}  // namespace ssmv
