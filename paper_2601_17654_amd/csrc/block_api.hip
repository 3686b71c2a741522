// C ABI of the transformer-block operators: argument checks, workspace layout and launch
// order.  Declarations and contracts: include/kareus.h.
#include <cmath>

#include "kr_block.h"

using namespace kr;

namespace {

constexpr int64_t kWidthMost = 1 << 30;

bool type_ok(int32_t t) { return t == KR_F32 || t == KR_F16 || t == KR_BF16; }

kr_status said(hipError_t e) { return e == hipSuccess ? KR_OK : KR_EHIP; }

// A matrix argument: rows `ld` elements apart, aligned to its elements.
bool matrix_ok(const void *p, int64_t ld, int64_t width, size_t size)
{
    return p && (uintptr_t)p % size == 0 && ld >= width;
}

size_t size_of(int32_t t) { return t == KR_F32 ? 4 : 2; }

kr_status norm_checked(bool held, int32_t type, int64_t rows, int64_t width, const void *x,
                       int64_t ldx, const void *res, int64_t ldr, const void *w, float eps,
                       void *sum, int64_t lds, void *out, int64_t ldo, float *scale, float *rstd,
                       void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || !(eps >= 0.0f) || std::isinf(eps))
        return KR_EINVAL;
    if (width > kWidthMost) return KR_EUNSUPPORTED;
    if (rows == 0) return KR_OK;
    const size_t es = size_of(type);
    if (!matrix_ok(x, ldx, width, es) || (res && !matrix_ok(res, ldr, width, es)) || !w ||
        (uintptr_t)w % es || (sum && !matrix_ok(sum, lds, width, es)) ||
        !matrix_ok(out, ldo, width, held ? 1 : es) || (held && !scale))
        return KR_EINVAL;
    const NormArgs a{rows, (int)width, x, res, w, ldx, ldr, eps, sum, out, lds, ldo, rstd, scale};
    return said(launch_norm(type, held, a, (hipStream_t)stream));
}

}  // namespace

extern "C" kr_status kr_add_rms_norm(int32_t type, int64_t rows, int64_t width, const void *x,
                                     int64_t ldx, const void *residual, int64_t ldr,
                                     const void *weight, float eps, void *sum, int64_t lds,
                                     void *out, int64_t ldo, float *rstd, void *stream)
{
    return norm_checked(false, type, rows, width, x, ldx, residual, ldr, weight, eps, sum, lds, out,
                        ldo, nullptr, rstd, stream);
}

extern "C" kr_status kr_add_rms_norm_bytes(int32_t type, int64_t rows, int64_t width, const void *x,
                                           int64_t ldx, const void *residual, int64_t ldr,
                                           const void *weight, float eps, void *sum, int64_t lds,
                                           int8_t *q, int64_t ldq, float *scale, float *rstd,
                                           void *stream)
{
    return norm_checked(true, type, rows, width, x, ldx, residual, ldr, weight, eps, sum, lds, q,
                        ldq, scale, rstd, stream);
}

extern "C" size_t kr_add_rms_norm_backward_workspace(int32_t type, int64_t rows, int64_t width)
{
    if (!type_ok(type) || rows < 0 || width < 1 || width > kWidthMost) return 0;
    return (size_t)norm_back_slots(type, rows, (int)width) * (size_t)width * sizeof(float);
}

extern "C" kr_status kr_add_rms_norm_backward(int32_t type, int64_t rows, int64_t width,
                                              const void *dout, int64_t ldo, const void *sum,
                                              int64_t lds, const void *weight, const float *rstd,
                                              const void *dsum, int64_t ldd, void *dx, int64_t ldx,
                                              float *dweight, void *ws, size_t ws_bytes,
                                              void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || !dweight) return KR_EINVAL;
    if (width > kWidthMost) return KR_EUNSUPPORTED;
    const size_t es = size_of(type);
    if (rows > 0 &&
        (!matrix_ok(dout, ldo, width, es) || !matrix_ok(sum, lds, width, es) || !weight ||
         (uintptr_t)weight % es || !rstd || (dsum && !matrix_ok(dsum, ldd, width, es)) ||
         !matrix_ok(dx, ldx, width, es)))
        return KR_EINVAL;
    const size_t need = kr_add_rms_norm_backward_workspace(type, rows, width);
    if (ws_bytes < need || (need && !ws)) return KR_ECAPACITY;
    if ((uintptr_t)ws % sizeof(float)) return KR_EINVAL;
    const NormBackArgs a{rows, (int)width, sum, weight, dout, dsum, lds, ldo, ldd, rstd,
                         dx, ldx, dweight, (float *)ws};
    return said(launch_norm_back(type, a, (hipStream_t)stream));
}
