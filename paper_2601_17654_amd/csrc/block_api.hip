// C ABI of the transformer-block operators: argument checks, workspace layout and launch
// order.  Declarations and contracts: include/kareus.h.
#include <algorithm>
#include <cmath>

#include "kr_drop.h"
#include "kr_gated.h"
#include "kr_scaled.h"

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

// ---- dropout and layer norm -----------------------------------------------------------------

namespace {

constexpr int64_t kDropWidthMost = 1 << 30;
constexpr int64_t kDropRowsMost = (int64_t)1 << 32;  // a row's number is one word of the counter

bool drop_ok(const kr_drop *d)
{
    return !d || (d->p >= 0.0 && d->p <= 1.0 && (uintptr_t)d->seed_at % 8 == 0);
}

}  // namespace

extern "C" kr_status kr_dropout(int32_t type, int64_t rows, int64_t width, const void *x, int64_t ldx,
                                const void *residual, int64_t ldr, const kr_drop *drop, void *out,
                                int64_t ldo, void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || !drop || !drop_ok(drop)) return KR_EINVAL;
    if (width > kDropWidthMost || rows > kDropRowsMost) return KR_EUNSUPPORTED;
    if (rows == 0) return KR_OK;
    const size_t es = size_of(type);
    if (!matrix_ok(x, ldx, width, es) || (residual && !matrix_ok(residual, ldr, width, es)) ||
        !matrix_ok(out, ldo, width, es))
        return KR_EINVAL;
    const DropoutArgs a{rows, width, x, residual, out, ldx, ldr, ldo, 0, drop_of(drop)};
    return said(launch_dropout(type, a, (hipStream_t)stream));
}

extern "C" kr_status kr_add_layer_norm(int32_t type, int64_t rows, int64_t width, const void *x,
                                       int64_t ldx, const void *residual, int64_t ldr,
                                       const void *weight, const void *bias, float eps,
                                       const kr_drop *drop, void *sum, int64_t lds, void *out,
                                       int64_t ldo, float *mean, float *rstd, void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || !(eps >= 0.0f) || std::isinf(eps) || !drop_ok(drop))
        return KR_EINVAL;
    if (width > kWidthMost || (drop && rows > kDropRowsMost)) return KR_EUNSUPPORTED;
    if (rows == 0) return KR_OK;
    const size_t es = size_of(type);
    if (!matrix_ok(x, ldx, width, es) || (residual && !matrix_ok(residual, ldr, width, es)) ||
        !weight || (uintptr_t)weight % es || (uintptr_t)bias % es ||
        (sum && !matrix_ok(sum, lds, width, es)) || !matrix_ok(out, ldo, width, es))
        return KR_EINVAL;
    const LayerNormArgs a{rows, (int)width, x, residual, weight, bias, ldx, ldr, eps,
                          sum, out, lds, ldo, mean, rstd, 0, drop_of(drop)};
    return said(launch_layer_norm(type, a, (hipStream_t)stream));
}

extern "C" size_t kr_add_layer_norm_backward_workspace(int32_t type, int64_t rows, int64_t width)
{
    if (!type_ok(type) || rows < 0 || width < 1 || width > kWidthMost) return 0;
    return (size_t)layer_norm_back_slots(rows, (int)width) * 2 * (size_t)width * sizeof(float);
}

extern "C" kr_status kr_add_layer_norm_backward(
    int32_t type, int64_t rows, int64_t width, const void *dout, int64_t ldo, const void *sum,
    int64_t lds, const void *weight, const float *mean, const float *rstd, const void *dsum,
    int64_t ldd, const kr_drop *drop, void *dresidual, int64_t ldr, void *dx, int64_t ldx,
    float *dweight, float *dbias, void *ws, size_t ws_bytes, void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || !dweight || !drop_ok(drop)) return KR_EINVAL;
    if (width > kWidthMost || (drop && rows > kDropRowsMost)) return KR_EUNSUPPORTED;
    const size_t es = size_of(type);
    const Drop d = drop_of(drop);
    if (rows > 0 &&
        (!matrix_ok(dout, ldo, width, es) || !matrix_ok(sum, lds, width, es) || !weight ||
         (uintptr_t)weight % es || !mean || !rstd || (dsum && !matrix_ok(dsum, ldd, width, es)) ||
         !matrix_ok(dresidual, ldr, width, es) || (d.cut && !dx) ||
         (dx && (dx == dresidual || !matrix_ok(dx, ldx, width, es)))))
        return KR_EINVAL;
    const size_t need = kr_add_layer_norm_backward_workspace(type, rows, width);
    if (ws_bytes < need || (need && !ws)) return KR_ECAPACITY;
    if ((uintptr_t)ws % sizeof(float)) return KR_EINVAL;
    const LayerNormBackArgs a{rows, (int)width, sum, weight, dout, dsum, lds, ldo, ldd, mean, rstd,
                              dresidual, dx, ldr, ldx, dweight, dbias, (float *)ws, 0, d};
    return said(launch_layer_norm_back(type, a, (hipStream_t)stream));
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

// ---- products of values held in 8-bit floating point ----------------------------------------

namespace {

constexpr int64_t kHeldMost = 1 << 30;  // rows and columns of a held matrix

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// A held matrix of rows x width as an argument.
bool held_ok(const kr_scaled *h, int64_t rows, int64_t width)
{
    return h && (rows == 0 || (h->q && h->ld >= h->room && h->room >= width && h->scale &&
                               (uintptr_t)h->scale % 4 == 0 && h->lds % 4 == 0 &&
                               h->lds >= up(rows, kScaled)));
}

HeldMatrix held(const kr_scaled *h)
{
    return {(char *)h->q, h->ld, h->room, (uint8_t *)h->scale, h->lds};
}

bool scaled_ok(const kr_scaled_product *p)
{
    return p && p->m >= 0 && p->n >= 1 && p->k >= 1 && held_ok(&p->a, p->m, p->k) &&
           held_ok(&p->b, p->n, p->k);
}

bool product_fits(int64_t m, int64_t n, int64_t k)
{
    return m <= kRowsMost && n <= kChannelsMost && k <= kRowMost && tiles_fit(m, n);
}

bool scaled_fits(const kr_scaled_product *p) { return product_fits(p->m, p->n, p->k); }

bool hold_fits(int64_t rows, int64_t width)
{
    return rows <= kHeldMost && width <= kHeldMost &&
           up(rows, kScaled) / kScaled * (up(width, kScaled) / kScaled) <= kHoldTilesMost;
}

// A product's arguments: its part in the workspace, and operands that are laid out anew.
struct ScaledLaid {
    ScaledArgs x;
    bool few;
    Laid a, b;
    ScaledLaid(const kr_scaled_product *p, int32_t type, void *out, int64_t ldo, Carve &c)
        : x{type, p->m, p->n, p->k, held(&p->a), held(&p->b), out, ldo, nullptr},
          few(p->m <= kScaledFew),
          // rows to a multiple of 16 bytes: theirs, where they have that room
          a(p->a.q, p->a.ld, few ? 0 : p->m, room_of(p->a, p->k), c),
          b(p->b.q, p->b.ld, few ? 0 : p->n, room_of(p->b, p->k), c)
    {
        if (few) return;
        x.part = c.take((int64_t)scaled_part(type, p->m, p->n, p->k));
        set(x.a, a);
        set(x.b, b);
    }
    static int64_t room_of(const kr_scaled &h, int64_t k) { return h.room >= padded(k) ? padded(k) : k; }
    static void set(HeldMatrix &h, const Laid &l)
    {
        h.q = (char *)l.op.p;
        h.ld = l.op.ld;
        h.bytes = l.op.bytes;
    }
    kr_status fill(hipStream_t st) const
    {
        if (few) return KR_OK;
        PadArgs pads{};
        a.add_to(pads);
        b.add_to(pads);
        return said(launch_pad(pads, st));
    }
};

kr_status scaled_run(const kr_scaled_product *p, int32_t type, void *out, int64_t ldo, Carve &c,
                     hipStream_t st)
{
    const ScaledLaid l(p, type, out, ldo, c);
    if (!out) return KR_OK;
    const kr_status s = l.fill(st);
    if (s != KR_OK) return s;
    return said(l.few ? launch_scaled_few(l.x, st) : launch_scaled(l.x, st));
}

}  // namespace

extern "C" kr_status kr_scaled_hold(int32_t type, int64_t rows, int64_t width, const void *x,
                                    int64_t ldx, int32_t square, const kr_scaled *plain,
                                    const kr_scaled *crossed, void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || (square != 0 && square != 1) || (!plain && !crossed))
        return KR_EINVAL;
    if (!hold_fits(rows, width)) return KR_EUNSUPPORTED;
    if (rows == 0) return KR_OK;
    if (!matrix_ok(x, ldx, width, size_of(type)) ||
        (plain && (!held_ok(plain, rows, width) || plain->room > up(width, kScaled))) ||
        (crossed && (!held_ok(crossed, width, rows) || crossed->room > up(rows, kScaled))))
        return KR_EINVAL;
    HoldArgs a{rows, width, x, ldx, {}, {}, up(width, kScaled) / kScaled};
    if (plain) a.plain = held(plain);
    if (crossed) a.crossed = held(crossed);
    return said(launch_hold(type, square != 0, a, (hipStream_t)stream));
}

extern "C" kr_status kr_scaled_values(int32_t type, int64_t rows, int64_t width, const kr_scaled *h,
                                      void *out, int64_t ldo, void *stream)
{
    if (!type_ok(type) || rows < 0 || width < 1 || !held_ok(h, rows, width)) return KR_EINVAL;
    if (rows > kHeldMost || width > kHeldMost) return KR_EUNSUPPORTED;
    if (rows == 0) return KR_OK;
    if (!matrix_ok(out, ldo, width, size_of(type))) return KR_EINVAL;
    const HeldValuesArgs a{rows, width, held(h), out, ldo, 0};
    return said(launch_held_values(type, a, (hipStream_t)stream));
}

extern "C" size_t kr_scaled_matmul_workspace(const kr_scaled_product *p)
{
    if (!scaled_ok(p) || !scaled_fits(p) || p->m == 0) return 0;
    size_t most = 0;
    for (const int32_t type : {KR_F32, KR_BF16}) {
        Carve c{nullptr};
        scaled_run(p, type, nullptr, 0, c, nullptr);
        most = std::max(most, c.used);
    }
    return most;
}

extern "C" kr_status kr_scaled_matmul(const kr_scaled_product *p, int32_t type, void *out, int64_t ldo,
                                      void *ws, size_t ws_bytes, void *stream)
{
    if (!scaled_ok(p) || !type_ok(type)) return KR_EINVAL;
    if (!scaled_fits(p)) return KR_EUNSUPPORTED;
    if (p->m == 0) return KR_OK;
    if (!matrix_ok(out, ldo, p->n, size_of(type)) || (uintptr_t)ws % 16) return KR_EINVAL;
    if (!ws_ok(ws, ws_bytes, kr_scaled_matmul_workspace(p))) return KR_ECAPACITY;
    Carve c{(char *)ws};
    return scaled_run(p, type, out, ldo, c, (hipStream_t)stream);
}

namespace {

bool linear_ok(const kr_linear *l)
{
    return l && type_ok(l->type) && l->rows >= 0 && l->width >= 1 && l->hidden >= 1 &&
           (l->rows == 0 || matrix_ok(l->x, l->ldx, l->width, size_of(l->type))) &&
           matrix_ok(l->w, l->ldw, l->width, size_of(l->type));
}

bool linear_fits(const kr_linear *l)
{
    return product_fits(l->rows, l->hidden, l->width) && hold_fits(l->rows, l->width) &&
           hold_fits(l->hidden, l->width);
}

bool linear_back_fits(const kr_linear *l)
{
    return linear_fits(l) && product_fits(l->rows, l->width, l->hidden) &&
           product_fits(l->hidden, l->width, l->rows) && hold_fits(l->rows, l->hidden);
}

// Room for a held matrix, rows of a multiple of 16 bytes, in a workspace.
kr_scaled held_room(int64_t rows, int64_t width, Carve &c)
{
    const int64_t room = padded(width), lds = up(rows, kScaled);
    kr_scaled h{};
    h.ld = h.room = room;
    h.lds = lds;
    h.q = c.take(rows * room);
    h.scale = c.take(up(width, kScaled) / kScaled * lds);
    return h;
}

HoldArgs hold_args(int64_t rows, int64_t width, const void *x, int64_t ldx, const kr_scaled *plain,
                   const kr_scaled *crossed)
{
    HoldArgs a{rows, width, x, ldx, {}, {}, up(width, kScaled) / kScaled};
    if (plain) a.plain = held(plain);
    if (crossed) a.crossed = held(crossed);
    return a;
}

// c.base null: sizes alone.
kr_status linear_run(const kr_linear *l, void *out, int64_t ldo, Carve &c, hipStream_t st)
{
    const kr_scaled x = held_room(l->rows, l->width, c), w = held_room(l->hidden, l->width, c);
    const kr_scaled_product p{l->rows, l->hidden, l->width, x, w};
    if (c.base) {
        const hipError_t e = launch_hold_linear(
            l->type, hold_args(l->rows, l->width, l->x, l->ldx, &x, nullptr),
            hold_args(l->hidden, l->width, l->w, l->ldw, &w, nullptr), st);
        if (e != hipSuccess) return said(e);
    }
    return scaled_run(&p, l->type, c.base ? out : nullptr, ldo, c, st);
}

kr_status linear_back_run(const kr_linear *l, const void *dout, int64_t ldd, void *dx, int64_t lddx,
                          void *dw, int64_t lddw, Carve &c, hipStream_t st)
{
    const bool for_x = !c.base || dx, for_w = !c.base || dw;
    kr_scaled d{}, dt{}, wt{}, xt{};
    if (for_x) {
        d = held_room(l->rows, l->hidden, c);
        wt = held_room(l->width, l->hidden, c);
    }
    if (for_w) {
        dt = held_room(l->hidden, l->rows, c);
        xt = held_room(l->width, l->rows, c);
    }
    const kr_scaled_product px{l->rows, l->width, l->hidden, d, wt}, pw{l->hidden, l->width, l->rows, dt, xt};
    if (c.base) {
        const hipError_t e = launch_hold_linear_back(
            l->type, hold_args(l->rows, l->hidden, dout, ldd, for_x ? &d : nullptr, for_w ? &dt : nullptr),
            hold_args(l->hidden, l->width, l->w, l->ldw, nullptr, &wt),
            hold_args(l->rows, l->width, l->x, l->ldx, nullptr, &xt), st);
        if (e != hipSuccess) return said(e);
    }
    if (!for_x || !for_w) {
        return for_x ? scaled_run(&px, l->type, dx, lddx, c, st) : scaled_run(&pw, l->type, dw, lddw, c, st);
    }
    // (held_room's rows need no laying out anew)
    const ScaledLaid x(&px, l->type, dx, lddx, c), w(&pw, l->type, dw, lddw, c);
    if (!c.base) return KR_OK;
    if (!x.few && !w.few) return said(launch_scaled_pair(x.x, w.x, st));
    const hipError_t e = x.few ? launch_scaled_few(x.x, st) : launch_scaled(x.x, st);
    return said(e != hipSuccess ? e : w.few ? launch_scaled_few(w.x, st) : launch_scaled(w.x, st));
}

}  // namespace

extern "C" size_t kr_scaled_linear_workspace(const kr_linear *l)
{
    if (!linear_ok(l) || !linear_fits(l) || l->rows == 0) return 0;
    Carve c{nullptr};
    linear_run(l, nullptr, 0, c, nullptr);
    return c.used;
}

extern "C" kr_status kr_scaled_linear(const kr_linear *l, void *out, int64_t ldo, void *ws,
                                      size_t ws_bytes, void *stream)
{
    if (!linear_ok(l)) return KR_EINVAL;
    if (!linear_fits(l)) return KR_EUNSUPPORTED;
    if (l->rows == 0) return KR_OK;
    if (!matrix_ok(out, ldo, l->hidden, size_of(l->type)) || (uintptr_t)ws % 16) return KR_EINVAL;
    if (!ws_ok(ws, ws_bytes, kr_scaled_linear_workspace(l))) return KR_ECAPACITY;
    Carve c{(char *)ws};
    return linear_run(l, out, ldo, c, (hipStream_t)stream);
}

extern "C" size_t kr_scaled_linear_backward_workspace(const kr_linear *l)
{
    if (!linear_ok(l) || !linear_back_fits(l) || l->rows == 0) return 0;
    Carve c{nullptr};
    linear_back_run(l, nullptr, 0, nullptr, 0, nullptr, 0, c, nullptr);
    return c.used;
}

extern "C" kr_status kr_scaled_linear_backward(const kr_linear *l, const void *dout, int64_t lddo, void *dx,
                                               int64_t lddx, void *dw, int64_t lddw, void *ws,
                                               size_t ws_bytes, void *stream)
{
    if (!linear_ok(l)) return KR_EINVAL;
    if (!linear_back_fits(l)) return KR_EUNSUPPORTED;
    const size_t es = size_of(l->type);
    if ((l->rows > 0 && (!matrix_ok(dout, lddo, l->hidden, es) || (dx && !matrix_ok(dx, lddx, l->width, es)))) ||
        (dw && !matrix_ok(dw, lddw, l->width, es)) || (uintptr_t)ws % 16)
        return KR_EINVAL;
    if (l->rows == 0) return dw ? said(launch_zeros(dw, lddw * es, l->hidden, l->width * es, (hipStream_t)stream))
                               : KR_OK;
    if (!dx && !dw) return KR_OK;
    if (!ws_ok(ws, ws_bytes, kr_scaled_linear_backward_workspace(l))) return KR_ECAPACITY;
    Carve c{(char *)ws};
    return linear_back_run(l, dout, lddo, dx, lddx, dw, lddw, c, (hipStream_t)stream);
}
