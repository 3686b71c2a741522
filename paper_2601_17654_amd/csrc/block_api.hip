// C ABI of the transformer-block operators: argument checks, workspace layout and launch
// order.  Declarations and contracts: include/kareus.h.
#include <cmath>

#include "kr_gated.h"

using namespace kr;

namespace {

constexpr int64_t kWidthMost = 1 << 24;

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

// ---- projections --------------------------------------------------------------------------

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kLdMost = 1 << 22;    // bytes between rows that the tiles' 32-bit offsets take
constexpr int64_t kRowMost = 1 << 21;   // bytes of a row: with two rows side by side, that
constexpr int64_t kRowsMost = 0x7FFFFFFF;
constexpr int64_t kChannelsMost = 1 << 27;
constexpr int64_t kTilesMost = 1 << 23;  // a grid has fewer than 2^32 threads, 256 a block
constexpr int64_t kBytesMost = 131071;  // 2^14 times this is below 2^31: sums cannot overflow

// Bump allocator over the caller's workspace (or a size query when base is null).
struct Carve {
    char *base;
    size_t used = 0;
    char *take(int64_t n)
    {
        used = (used + kAlign - 1) / kAlign * kAlign;
        char *p = base ? base + used : nullptr;
        used += (size_t)n;
        return p;
    }
};

// Whether a grid holds the smaller tiles of rows x columns outputs (two planes: half as wide).
bool tiles_fit(int64_t rows, int64_t columns)
{
    return ((rows + 127) / 128) * ((columns + 63) / 64) <= kTilesMost;
}

int64_t padded(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// A matrix as the tiles take it: itself, or a copy with rows of a multiple of 16 bytes.
struct Laid {
    Operand op;
    const void *from;
    int64_t from_ld, bytes;
    bool copy;
    Laid(const void *p, int64_t ld, int64_t rows, int64_t bytes_, Carve &c, bool always = false)
        : from(p), from_ld(rows > 1 ? ld : padded(bytes_)), bytes(bytes_)
    {
        copy = always || (uintptr_t)p % 16 || from_ld % 16 || bytes % 16 || from_ld > kLdMost;
        if (copy) {
            const int64_t to = padded(bytes);
            op = Operand{c.take(rows * to), to, rows, to};
        } else {
            op = Operand{(const char *)p, from_ld, rows, bytes};
        }
    }
    void add_to(PadArgs &a) const
    {
        if (copy)
            a.m[a.count++] = {(const char *)from, from_ld, op.rows, bytes, (char *)op.p, op.ld};
    }
};

bool gated_ok(const kr_gated *g)
{
    return g && (g->type == KR_F16 || g->type == KR_BF16) && (g->act == KR_SILU || g->act == KR_GELU) &&
           g->rows >= 0 && g->width >= 1 && g->hidden >= 1 &&
           (g->rows == 0 || matrix_ok(g->x, g->ldx, g->width, 2)) &&
           matrix_ok(g->wg, g->ldg, g->width, 2) && matrix_ok(g->wu, g->ldu, g->width, 2);
}

bool gated_fits(const kr_gated *g)
{
    return g->rows <= kRowsMost && g->width <= kRowMost / 2 && g->hidden <= kRowMost / 2 &&
           tiles_fit(g->rows, g->hidden > g->width ? g->hidden : g->width);
}

// The backward pass puts both weights' gradients in one product besides.
bool gated_back_fits(const kr_gated *g)
{
    return gated_fits(g) && tiles_fit(2 * ((g->hidden + 7) / 8 * 8), g->width);
}

struct GatedLaid {
    Laid x, wg, wu;
    // one_ld: both weights' rows the same distance apart (one sum over both takes them)
    GatedLaid(const kr_gated *g, Carve &c, bool one_ld)
        : x(g->x, g->ldx * 2, g->rows, g->width * 2, c),
          wg(g->wg, g->ldg * 2, g->hidden, g->width * 2, c, one_ld && g->ldg != g->ldu),
          wu(g->wu, g->ldu * 2, g->hidden, g->width * 2, c, one_ld && (wg.copy || g->ldg != g->ldu))
    {
        if (one_ld && wu.copy && !wg.copy)
            wg = Laid(g->wg, g->ldg * 2, g->hidden, g->width * 2, c, true);
    }
    GatedArgs args(const kr_gated *g) const
    {
        GatedArgs a{};
        a.type = g->type;
        a.act = g->act;
        a.m = g->rows;
        a.n = g->hidden;
        a.k_bytes = padded(g->width * 2);
        a.x = x.op;
        a.wg = wg.op;
        a.wu = wu.op;
        return a;
    }
    hipError_t fill(hipStream_t st) const
    {
        PadArgs a{};
        x.add_to(a);
        wg.add_to(a);
        wu.add_to(a);
        return launch_pad(a, st);
    }
};

// A matrix as it is.
Operand as_is(const void *p, int64_t ld, int64_t rows, int64_t bytes)
{
    return {(const char *)p, ld, rows, bytes};
}

kr_status gated_run(const kr_gated *g, void *out, int64_t ldo, Carve &c, hipStream_t st)
{
    if (g->rows <= kFewRows) {
        if (!out) return KR_OK;
        GatedArgs a{};
        a.type = g->type;
        a.act = g->act;
        a.m = g->rows;
        a.n = g->hidden;
        a.x = as_is(g->x, g->ldx * 2, g->rows, g->width * 2);
        a.wg = as_is(g->wg, g->ldg * 2, g->hidden, g->width * 2);
        a.wu = as_is(g->wu, g->ldu * 2, g->hidden, g->width * 2);
        a.out = out;
        a.ldo = ldo;
        return said(launch_gated_few(a, st));
    }
    const GatedLaid l(g, c, false);
    GatedArgs a = l.args(g);
    a.out = out;
    a.ldo = ldo;
    a.part = c.take((int64_t)gated_part(a.m, a.n, a.k_bytes));
    if (!out) return KR_OK;
    const hipError_t e = l.fill(st);
    return said(e == hipSuccess ? launch_gated(a, st) : e);
}

kr_status gated_back_run(const kr_gated *g, GatedBackArgs &b, Carve &c, hipStream_t st)
{
    const GatedLaid l(g, c, true);
    b.f = l.args(g);
    b.width = g->width;
    b.n_pad = (g->hidden + 7) / 8 * 8;
    b.d = c.take(g->rows * 4 * b.n_pad);
    const int64_t tops = (int64_t)gated_back_tops(g->type);
    b.tops = tops ? c.take(tops) : nullptr;
    b.f.part = c.take((int64_t)gated_back_part(b.f.m, b.f.n, b.n_pad, b.width, b.f.k_bytes));
    if (!b.dwg) return KR_OK;
    const hipError_t e = l.fill(st);
    return said(e == hipSuccess ? launch_gated_back(b, st) : e);
}

bool bytes_ok(const kr_bytes *p)
{
    return p && p->m >= 0 && p->n >= 1 && p->k >= 1 && (p->m == 0 || matrix_ok(p->a, p->lda, p->k, 1)) &&
           matrix_ok(p->b, p->ldb, p->k, 1) && (p->m == 0 || p->sa) && p->sb;
}

bool bytes_fits(const kr_bytes *p)
{
    return p->m <= kRowsMost && p->n <= kChannelsMost && p->k <= kBytesMost && tiles_fit(p->m, p->n);
}

kr_status bytes_run(const kr_bytes *p, int32_t type, void *out, int64_t ldo, Carve &c, hipStream_t st)
{
    if (p->m <= kFewRows) {
        if (!out) return KR_OK;
        const BytesArgs x{type, p->m, p->n, p->k, as_is(p->a, p->lda, p->m, p->k),
                          as_is(p->b, p->ldb, p->n, p->k), p->sa, p->sb, out, ldo, nullptr};
        return said(launch_bytes_few(x, st));
    }
    const Laid a(p->a, p->lda, p->m, p->k, c), b(p->b, p->ldb, p->n, p->k, c);
    BytesArgs x{};
    x.out_type = type;
    x.m = p->m;
    x.n = p->n;
    x.k_bytes = padded(p->k);
    x.a = a.op;
    x.b = b.op;
    x.sa = p->sa;
    x.sb = p->sb;
    x.out = out;
    x.ldo = ldo;
    x.part = c.take((int64_t)bytes_part(x.m, x.n, x.k_bytes));
    if (!out) return KR_OK;
    PadArgs pads{};
    a.add_to(pads);
    b.add_to(pads);
    const hipError_t e = launch_pad(pads, st);
    return said(e == hipSuccess ? launch_bytes(x, st) : e);
}

bool ws_ok(const void *ws, size_t bytes, size_t need) { return bytes >= need && (ws || !need); }

}  // namespace

extern "C" size_t kr_gated_projection_workspace(const kr_gated *g)
{
    if (!gated_ok(g) || !gated_fits(g) || g->rows == 0) return 0;
    Carve c{nullptr};
    gated_run(g, nullptr, 0, c, nullptr);
    return c.used;
}

extern "C" kr_status kr_gated_projection(const kr_gated *g, void *out, int64_t ldo, void *ws,
                                         size_t ws_bytes, void *stream)
{
    if (!gated_ok(g)) return KR_EINVAL;
    if (!gated_fits(g)) return KR_EUNSUPPORTED;
    if (g->rows == 0) return KR_OK;
    if (!matrix_ok(out, ldo, g->hidden, 2) || (uintptr_t)ws % 16) return KR_EINVAL;
    if (!ws_ok(ws, ws_bytes, kr_gated_projection_workspace(g))) return KR_ECAPACITY;
    Carve c{(char *)ws};
    return gated_run(g, out, ldo, c, (hipStream_t)stream);
}

extern "C" size_t kr_gated_projection_backward_workspace(const kr_gated *g)
{
    if (!gated_ok(g) || !gated_back_fits(g)) return 0;
    Carve c{nullptr};
    GatedBackArgs b{};
    gated_back_run(g, b, c, nullptr);
    return c.used;
}

extern "C" kr_status kr_gated_projection_backward(const kr_gated *g, const void *dh, int64_t ldh,
                                                  void *dx, int64_t lddx, void *dwg, int64_t lddg,
                                                  void *dwu, int64_t lddu, void *ws,
                                                  size_t ws_bytes, void *stream)
{
    if (!gated_ok(g)) return KR_EINVAL;
    if (!gated_back_fits(g)) return KR_EUNSUPPORTED;
    if ((g->rows > 0 && (!matrix_ok(dh, ldh, g->hidden, 2) || !matrix_ok(dx, lddx, g->width, 2))) ||
        !matrix_ok(dwg, lddg, g->width, 2) || !matrix_ok(dwu, lddu, g->width, 2) || (uintptr_t)ws % 16)
        return KR_EINVAL;
    if (!ws_ok(ws, ws_bytes, kr_gated_projection_backward_workspace(g))) return KR_ECAPACITY;
    Carve c{(char *)ws};
    GatedBackArgs b{};
    b.dh = dh;
    b.ldh = ldh;
    b.dx = dx;
    b.lddx = lddx;
    b.dwg = dwg;
    b.lddg = lddg;
    b.dwu = dwu;
    b.lddu = lddu;
    return gated_back_run(g, b, c, (hipStream_t)stream);
}

extern "C" size_t kr_byte_matmul_workspace(const kr_bytes *p)
{
    if (!bytes_ok(p) || !bytes_fits(p) || p->m == 0) return 0;
    Carve c{nullptr};
    bytes_run(p, KR_F32, nullptr, 0, c, nullptr);
    return c.used;
}

extern "C" kr_status kr_byte_matmul(const kr_bytes *p, int32_t type, void *out, int64_t ldo, void *ws,
                                    size_t ws_bytes, void *stream)
{
    if (!bytes_ok(p) || !type_ok(type)) return KR_EINVAL;
    if (!bytes_fits(p)) return KR_EUNSUPPORTED;
    if (p->m == 0) return KR_OK;
    if (!matrix_ok(out, ldo, p->n, size_of(type)) || (uintptr_t)ws % 16) return KR_EINVAL;
    if (!ws_ok(ws, ws_bytes, kr_byte_matmul_workspace(p))) return KR_ECAPACITY;
    Carve c{(char *)ws};
    return bytes_run(p, type, out, ldo, c, (hipStream_t)stream);
}
