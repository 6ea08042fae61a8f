// C ABI of the feed-forward operators (include/isc.h): argument validation on
// the host, then the launches.
#include "expert.hpp"
#include "orthogonalize.hpp"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <limits>

namespace {

constexpr int64_t kI32Max = std::numeric_limits<int32_t>::max();
constexpr int64_t kI64Room = int64_t{1} << 56;  // elements a strided tensor may span
constexpr size_t kAlign = 256;
constexpr int32_t kMaxNorm = 65536, kMaxNormBwd = 16384, kMaxExperts = 1024, kMaxSlots = 64, kMaxTokens = 1 << 20;
constexpr int32_t kMaxRouted = (1 << 28) - 64;  // 64 tokens for every workgroup of 1024 threads of a launch

bool element_type(int32_t t) { return t == ISC_F32 || t == ISC_F16 || t == ISC_BF16; }
size_t type_bytes(int32_t t) { return t == ISC_F32 ? 4 : t == ISC_MX8 ? 1 : 2; }
bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// A rows x cols tensor of a call: `rows` rows `ld` elements apart.
struct Span {
    const void *p;
    int64_t rows, cols, ld;
    size_t size;  // of an element
    size_t bytes() const { return rows < 1 ? 0 : size * static_cast<size_t>((rows - 1) * ld + cols); }
    bool shape_ok() const { return !p || (ld >= cols && (rows < 1 || ld <= kI64Room / rows)); }
};

bool overlap(const Span &a, const Span &b) {
    if (!a.p || !b.p) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x < y + b.bytes() && y < x + a.bytes();
}
// The same rows, written in place of what was read there.
bool in_place(const Span &a, const Span &b) {
    return a.p == b.p && a.cols == b.cols && a.size == b.size && (a.ld == b.ld || a.rows < 2);
}

int hip_status(hipError_t e) { return e == hipSuccess ? ISC_OK : ISC_ERR_HIP; }

int check_w4(const isc_w4_desc *d, isc::W4Shape *w) {
    if (!d) return ISC_ERR_NULL;
    if (d->E < 1 || d->N < 1 || d->K < 1) return ISC_ERR_SHAPE;
    if (d->layout != ISC_W4_TILES && d->layout != ISC_W4_ROWS) return ISC_ERR_ARG;
    // an input's offsets in a matrix stay in 32 bits, the experts' in 64
    if (d->E > kMaxExperts || d->K > (1 << 24) || d->N > (1 << 24) ||
        static_cast<int64_t>(d->N + 127) * (d->K + 511) > int64_t{1} << 36)
        return ISC_ERR_LIMIT;
    *w = isc::W4Shape{d->E, d->N, d->K};
    return ISC_OK;
}

// The largest N and K of the experts' matrices, whose rows' bytes stay in 32 bits.
constexpr int32_t kMaxWidth = 1 << 20;

// A call on experts: what holds for it whatever it computes.
int check_expert(const isc_expert_desc *d, int32_t T) {
    if (!d) return ISC_ERR_NULL;
    if (d->E < 1 || d->N < 1 || d->K < 1 || d->slots < 1 || T < 0) return ISC_ERR_SHAPE;
    if (!element_type(d->type)) return ISC_ERR_ARG;
    if (d->E > kMaxExperts || d->slots > kMaxSlots || d->N > kMaxWidth || d->K > kMaxWidth || T > kMaxTokens)
        return ISC_ERR_LIMIT;
    return isc::expert_launches_fit(static_cast<int64_t>(T) * d->slots, d->E, d->N, d->K, d->type) ? ISC_OK
                                                                                                  : ISC_ERR_LIMIT;
}

// The largest magnitude of a s + b s^3 + c s^5 over [0, r]: at an end, or where the
// slope a + 3 b s^2 + 5 c s^4 is 0.
double most_of(double a, double b, double c, double r) {
    const auto at = [=](double s) { return std::fabs(s * (a + s * s * (b + c * s * s))); };
    double most = at(r);
    const auto look = [&](double square) {
        if (square > 0.0 && square < r * r) most = std::max(most, at(std::sqrt(square)));
    };
    // the slope's roots by the sum that does not cancel, so that a small c loses neither
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
        const double t = -(3.0 * b + std::copysign(std::sqrt(d), b));
        look(t / (10.0 * c));
        look(2.0 * a / t);
    }
    return most;
}

Span flat(const void *p, int64_t n, size_t size) { return Span{p, 1, n, n, size}; }

}  // namespace

extern "C" {

int isc_rmsnorm(int32_t T, int32_t D, int32_t type, const void *x, int64_t ldx, const void *r, int64_t ldr,
                const void *w, int32_t w_type, float eps, void *h, int64_t ldh, void *y, int64_t ldy, void *q,
                int64_t ldq, void *scales, int64_t lds, float *rstd, void *stream) {
    if (T < 0 || D < 1) return ISC_ERR_SHAPE;
    if (!element_type(type) || !element_type(w_type) || !(eps >= 0.0f) || std::isinf(eps)) return ISC_ERR_ARG;
    if (D > kMaxNorm) return ISC_ERR_LIMIT;
    const size_t b = type_bytes(type);
    const int64_t groups = (D + 31) / 32;
    const Span in[3] = {{x, T, D, ldx, b}, {r, T, D, ldr, b}, {w, 1, D, D, type_bytes(w_type)}};
    const Span out[5] = {{h, T, D, ldh, b}, {y, T, D, ldy, b}, {q, T, D, ldq, 1}, {scales, T, groups, lds, 1},
                         flat(rstd, T, 4)};
    if (T == 0) return ISC_OK;
    if (!x || !w || (!h && !y && !q && !rstd) || !q != !scales) return ISC_ERR_NULL;
    for (const Span &s : in)
        if (!s.shape_ok()) return ISC_ERR_SHAPE;
    for (const Span &s : out)
        if (!s.shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(x, b) || !aligned(r, b) || !aligned(w, type_bytes(w_type)) || !aligned(h, b) || !aligned(y, b) ||
        !aligned(rstd, 4))
        return ISC_ERR_ALIGN;
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < 3; ++j)
            if (overlap(out[i], in[j]) && !(i < 2 && j < 2 && in_place(out[i], in[j]))) return ISC_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ISC_ERR_ALIAS;
    }
    if (const int st = isc::require_gfx950()) return st;
    const isc::NormArgs a{x, r, w, h, y, q, scales, rstd, ldx, ldr, ldh, ldy, ldq, lds, T, D, type, w_type, eps};
    return hip_status(isc::launch_rmsnorm(a, static_cast<hipStream_t>(stream)));
}

int isc_rmsnorm_bwd_workspace_size(int32_t T, int32_t D, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    if (T < 0 || D < 1) return ISC_ERR_SHAPE;
    if (D > kMaxNormBwd) return ISC_ERR_LIMIT;
    *bytes = sizeof(float) * static_cast<size_t>(isc::norm_bwd_blocks(T, D)) * static_cast<size_t>(D);
    return ISC_OK;
}

int isc_rmsnorm_bwd(int32_t T, int32_t D, int32_t type, const void *dy, int64_t ldy, const void *h, int64_t ldh,
                    const void *w, int32_t w_type, const float *rstd, const void *dh, int64_t ldd, void *dx,
                    int64_t ldx, float *dw, void *ws, size_t ws_bytes, void *stream) {
    size_t need = 0;
    if (const int st = isc_rmsnorm_bwd_workspace_size(T, D, &need)) return st;
    if (!element_type(type) || !element_type(w_type)) return ISC_ERR_ARG;
    const size_t b = type_bytes(type);
    if (!dw || !ws || (T > 0 && (!dy || !h || !w || !rstd || !dx))) return ISC_ERR_NULL;
    const Span in[5] = {{dy, T, D, ldy, b}, {h, T, D, ldh, b}, {dh, T, D, ldd, b}, {w, 1, D, D, type_bytes(w_type)},
                        flat(rstd, T, 4)};
    const Span out[3] = {{dx, T, D, ldx, b}, flat(dw, D, 4), flat(ws, static_cast<int64_t>(need), 1)};
    for (const Span &s : in)
        if (T > 0 && !s.shape_ok()) return ISC_ERR_SHAPE;
    if (T > 0 && !out[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(dy, b) || !aligned(h, b) || !aligned(dh, b) || !aligned(w, type_bytes(w_type)) || !aligned(rstd, 4) ||
        !aligned(dx, b) || !aligned(dw, 4) || !aligned(ws, kAlign))
        return ISC_ERR_ALIGN;
    if (ws_bytes < need) return ISC_ERR_WORKSPACE;
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 5; ++j)
            if (overlap(out[i], in[j]) && !(i == 0 && j < 3 && in_place(out[i], in[j]))) return ISC_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ISC_ERR_ALIAS;
    }
    if (const int st = isc::require_gfx950()) return st;
    const isc::NormBwdArgs a{dy, h, w, dh, rstd, dx, dw, static_cast<float *>(ws), ldy, ldh, ldd, ldx, T, D, type,
                             w_type};
    return hip_status(isc::launch_rmsnorm_bwd(a, static_cast<hipStream_t>(stream)));
}

int isc_route_workspace_size(int32_t T, int32_t E, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    if (T < 0 || E < 1) return ISC_ERR_SHAPE;
    if (E > kMaxExperts || T > kMaxRouted) return ISC_ERR_LIMIT;
    *bytes = isc::route_count_bytes(T, E);
    return ISC_OK;
}

int isc_route(int32_t T, int32_t E, int32_t k, int32_t type, const void *logits, int64_t ld, const float *bias,
              int32_t score, int32_t groups, int32_t keep_groups, int32_t renorm, float scale, int32_t *ids,
              float *weights, int32_t *offsets, int32_t *order, void *ws, size_t ws_bytes, void *stream) {
    size_t need = 0;
    if (const int st = isc_route_workspace_size(T, E, &need)) return st;
    if (k < 1 || k > E || groups < 1 || E % groups != 0 || keep_groups < 1 || keep_groups > groups)
        return ISC_ERR_SHAPE;
    if (!element_type(type) || (score != ISC_SCORE_SOFTMAX && score != ISC_SCORE_SIGMOID) || std::isnan(scale))
        return ISC_ERR_ARG;
    if (k > kMaxSlots || groups > 64 || static_cast<int64_t>(T) * k > kI32Max) return ISC_ERR_LIMIT;
    if (!offsets != !order || (T > 0 && (!logits || !ids || !weights))) return ISC_ERR_NULL;
    if (!order) need = 0;
    const int64_t pairs = static_cast<int64_t>(T) * k;
    const Span in[2] = {{logits, T, E, ld, type_bytes(type)}, flat(bias, E, 4)};
    const Span out[5] = {flat(ids, pairs, 4), flat(weights, pairs, 4), flat(offsets, E + 1, 4), flat(order, pairs, 4),
                         flat(need ? ws : nullptr, static_cast<int64_t>(need), 1)};
    if (T > 0 && !in[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(logits, type_bytes(type)) || !aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4) ||
        !aligned(offsets, 4) || !aligned(order, 4) || (need && !aligned(ws, kAlign)))
        return ISC_ERR_ALIGN;
    if (need && (!ws || ws_bytes < need)) return ws ? ISC_ERR_WORKSPACE : ISC_ERR_NULL;
    for (int i = 0; i < 5; ++i) {
        for (const Span &s : in)
            if (overlap(out[i], s)) return ISC_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return ISC_ERR_ALIAS;
    }
    if (const int st = isc::require_gfx950()) return st;
    if (T == 0 && !order) return ISC_OK;
    const isc::RouteArgs a{logits, bias, ld, T, E, k, type, score == ISC_SCORE_SIGMOID, groups, keep_groups, renorm != 0,
                           scale, ids, weights, offsets, order, static_cast<uint16_t *>(ws)};
    return hip_status(isc::launch_route(a, static_cast<hipStream_t>(stream)));
}

int isc_route_bwd(int32_t T, int32_t E, int32_t k, int32_t type, const float *dweights, const void *logits, int64_t ld,
                  const int32_t *ids, int32_t score, int32_t renorm, float scale, void *dlogits, int64_t ldd,
                  void *stream) {
    if (T < 0 || E < 1 || k < 1 || k > E) return ISC_ERR_SHAPE;
    if (!element_type(type) || (score != ISC_SCORE_SOFTMAX && score != ISC_SCORE_SIGMOID) || std::isnan(scale))
        return ISC_ERR_ARG;
    if (E > kMaxExperts || k > kMaxSlots) return ISC_ERR_LIMIT;
    if (T == 0) return ISC_OK;
    if (!dweights || !logits || !ids || !dlogits) return ISC_ERR_NULL;
    const size_t b = type_bytes(type);
    const int64_t pairs = static_cast<int64_t>(T) * k;
    const Span in[3] = {{logits, T, E, ld, b}, flat(dweights, pairs, 4), flat(ids, pairs, 4)};
    const Span out = {dlogits, T, E, ldd, b};
    if (!in[0].shape_ok() || !out.shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(logits, b) || !aligned(dweights, 4) || !aligned(ids, 4) || !aligned(dlogits, b)) return ISC_ERR_ALIGN;
    for (const Span &s : in)
        if (overlap(out, s) && !in_place(out, s)) return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    const isc::RouteBwdArgs a{dweights, logits, ids, dlogits, ld, ldd, T, E, k, type, score == ISC_SCORE_SIGMOID,
                              renorm != 0, scale};
    return hip_status(isc::launch_route_bwd(a, static_cast<hipStream_t>(stream)));
}

int isc_w4_size(const isc_w4_desc *d, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    isc::W4Shape w;
    if (const int st = check_w4(d, &w)) return st;
    *bytes = static_cast<size_t>(w.bytes(d->layout));
    return ISC_OK;
}

int isc_w4_quantize(const isc_w4_desc *d, const void *w, int32_t type, int64_t ld, uint8_t *codes, uint8_t *scales,
                    void *stream) {
    isc::W4Shape s;
    if (const int st = check_w4(d, &s)) return st;
    if (!element_type(type)) return ISC_ERR_ARG;
    if (!w || !codes || !scales) return ISC_ERR_NULL;
    const int64_t rows = static_cast<int64_t>(s.E) * s.N;
    const Span in = {w, rows, s.K, ld, type_bytes(type)};
    const Span c = flat(codes, rows * ((s.K + 1) / 2), 1), sc = flat(scales, rows * s.groups(), 1);
    if (!in.shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(w, type_bytes(type))) return ISC_ERR_ALIGN;
    if (overlap(c, in) || overlap(sc, in) || overlap(c, sc)) return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    return hip_status(isc::launch_w4_quantize(s, w, type, ld, codes, scales, static_cast<hipStream_t>(stream)));
}

int isc_w4_pack_codes(const isc_w4_desc *d, const uint8_t *codes, const uint8_t *scales, void *packed, void *stream) {
    isc::W4Shape s;
    if (const int st = check_w4(d, &s)) return st;
    if (!codes || !scales || !packed) return ISC_ERR_NULL;
    const int64_t rows = static_cast<int64_t>(s.E) * s.N;
    const Span c = flat(codes, rows * ((s.K + 1) / 2), 1), sc = flat(scales, rows * s.groups(), 1);
    const Span out = flat(packed, s.bytes(d->layout), 1);
    if (!aligned(packed, kAlign)) return ISC_ERR_ALIGN;
    if (overlap(out, c) || overlap(out, sc)) return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    return hip_status(isc::launch_w4_pack(s, d->layout, codes, scales, static_cast<uint8_t *>(packed),
                                          static_cast<hipStream_t>(stream)));
}

int isc_w4_linear_workspace_size(const isc_w4_desc *d, int32_t T, int32_t x_type, int32_t slots, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    isc::W4Shape w;
    if (const int st = check_w4(d, &w)) return st;
    if (T < 0 || slots < 0) return ISC_ERR_SHAPE;
    if (!element_type(x_type) && x_type != ISC_MX8) return ISC_ERR_ARG;
    if (T > kMaxTokens || slots > kMaxSlots) return ISC_ERR_LIMIT;
    *bytes = isc::w4_linear_column_bytes(w, T, x_type, slots);
    return ISC_OK;
}

int isc_w4_linear(const isc_w4_desc *d, const void *packed, int32_t T, const void *x, int32_t x_type, int64_t ldx,
                  const void *x_scales, int64_t ld_scales, int32_t slots, const int32_t *ids, const int32_t *offsets,
                  const int32_t *order, void *y, int32_t y_type, int64_t ldy, int32_t relu, void *ws, size_t ws_bytes,
                  void *stream) {
    size_t need = 0;
    if (const int st = isc_w4_linear_workspace_size(d, T, x_type, slots, &need)) return st;
    isc::W4Shape w;
    if (const int st = check_w4(d, &w)) return st;
    if (d->layout != ISC_W4_TILES || !element_type(y_type) || (slots == 0 && w.E != 1)) return ISC_ERR_ARG;
    if (T == 0) return ISC_OK;
    if (!packed || !x || !y || (x_type == ISC_MX8) != (x_scales != nullptr) ||
        (slots && (!ids || !offsets || !order)) || (need && !ws))
        return ISC_ERR_NULL;
    const int64_t rows = slots ? static_cast<int64_t>(T) * slots : T;
    const Span in[6] = {{x, T, w.K, ldx, type_bytes(x_type)},
                        {x_scales, T, w.groups(), ld_scales, 1},
                        flat(packed, w.bytes(d->layout), 1),
                        flat(slots ? ids : nullptr, rows, 4),
                        flat(slots ? offsets : nullptr, w.E + 1, 4),
                        flat(slots ? order : nullptr, rows, 4)};
    const Span out[2] = {{y, rows, w.N, ldy, type_bytes(y_type)},
                         flat(need ? ws : nullptr, static_cast<int64_t>(need), 1)};
    if (!in[0].shape_ok() || !in[1].shape_ok() || !out[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(x, type_bytes(x_type)) || !aligned(packed, kAlign) || !aligned(y, type_bytes(y_type)) ||
        (need && !aligned(ws, kAlign)) ||
        (slots && (!aligned(ids, 4) || !aligned(offsets, 4) || !aligned(order, 4))))
        return ISC_ERR_ALIGN;
    if (ws_bytes < need) return ISC_ERR_WORKSPACE;
    for (const Span &o : out)
        for (const Span &s : in)
            if (overlap(o, s)) return ISC_ERR_ALIAS;
    if (overlap(out[0], out[1])) return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    isc::W4Args a{};
    a.w = w;
    a.packed = static_cast<const uint8_t *>(packed);
    a.x = x, a.ldx = ldx, a.xtype = x_type;
    a.xs = static_cast<const uint8_t *>(x_scales), a.ldxs = ld_scales;
    a.T = T, a.slots = slots, a.ids = ids, a.offsets = offsets, a.order = order;
    a.y = y, a.ldy = ldy, a.ytype = y_type, a.relu = relu != 0;
    a.columns = static_cast<uint8_t *>(ws);
    return hip_status(isc::launch_w4_linear(a, static_cast<hipStream_t>(stream)));
}

int isc_w4_skip_workspace_size(const isc_w4_desc *d, int32_t T, int32_t slots, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    isc::W4Shape w;
    if (const int st = check_w4(d, &w)) return st;
    if (T < 0 || slots < 0) return ISC_ERR_SHAPE;
    if (T > kMaxTokens || slots > kMaxSlots) return ISC_ERR_LIMIT;
    const int ranges = isc::w4_skip_ranges(w, T, slots);
    *bytes = ranges > 1 ? sizeof(float) * static_cast<size_t>(ranges) * static_cast<size_t>(T) * w.N : 0;
    return ISC_OK;
}

int isc_w4_skip(const isc_w4_desc *d, const void *packed, int32_t T, const void *x, int32_t x_type, int64_t ldx,
                int32_t slots, const int32_t *ids, const float *weights, void *y, int32_t y_type, int64_t ldy, void *ws,
                size_t ws_bytes, void *stream) {
    size_t need = 0;
    if (const int st = isc_w4_skip_workspace_size(d, T, slots, &need)) return st;
    isc::W4Shape w;
    if (const int st = check_w4(d, &w)) return st;
    if (d->layout != ISC_W4_ROWS || !element_type(x_type) || !element_type(y_type) || (slots == 0 && w.E != 1))
        return ISC_ERR_ARG;
    if (T == 0) return ISC_OK;
    if (!packed || !x || !y || (slots && (!ids || !weights)) || (need && !ws)) return ISC_ERR_NULL;
    const int64_t rows = slots ? static_cast<int64_t>(T) * slots : T;
    const Span in[4] = {{x, rows, w.K, ldx, type_bytes(x_type)},
                        flat(packed, w.bytes(d->layout), 1),
                        flat(slots ? ids : nullptr, rows, 4),
                        flat(slots ? weights : nullptr, rows, 4)};
    const Span out[2] = {{y, T, w.N, ldy, type_bytes(y_type)},
                         flat(need ? ws : nullptr, static_cast<int64_t>(need), 1)};
    if (!in[0].shape_ok() || !out[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(x, type_bytes(x_type)) || !aligned(packed, kAlign) || !aligned(y, type_bytes(y_type)) ||
        (need && !aligned(ws, kAlign)) || (slots && (!aligned(ids, 4) || !aligned(weights, 4))))
        return ISC_ERR_ALIGN;
    if (ws_bytes < need) return ISC_ERR_WORKSPACE;
    for (const Span &o : out)
        for (const Span &s : in)
            if (overlap(o, s)) return ISC_ERR_ALIAS;
    if (overlap(out[0], out[1])) return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    isc::W4Args a{};
    a.w = w;
    a.packed = static_cast<const uint8_t *>(packed);
    a.x = x, a.ldx = ldx, a.xtype = x_type;
    a.T = T, a.slots = slots, a.ids = ids, a.weights = weights;
    a.y = y, a.ldy = ldy, a.ytype = y_type;
    a.part = static_cast<float *>(ws);
    return hip_status(isc::launch_w4_skip(a, static_cast<hipStream_t>(stream)));
}

int isc_expert_linear_workspace_size(const isc_expert_desc *d, int32_t T, int32_t combine, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    if (const int st = check_expert(d, T)) return st;
    const int64_t pairs = static_cast<int64_t>(T) * d->slots;
    *bytes = isc::expert_plan_bytes(pairs, d->E, d->type) +
             (combine ? sizeof(float) * static_cast<size_t>(pairs * isc::expert_ld(d->N)) : 0);
    return ISC_OK;
}

int isc_expert_linear(const isc_expert_desc *d, const void *w, int64_t ldw, int32_t T, const void *x, int64_t ldx,
                      const int32_t *ids, const float *weights, const int32_t *offsets, const int32_t *order, void *y,
                      int32_t y_type, int64_t ldy, int32_t relu, int32_t combine, void *ws, size_t ws_bytes,
                      void *stream) {
    size_t need = 0;
    if (const int st = isc_expert_linear_workspace_size(d, T, combine, &need)) return st;
    if (!element_type(y_type) || (relu && combine)) return ISC_ERR_ARG;
    if (T == 0) return ISC_OK;
    if (!w || !x || !ids || !offsets || !order || !y || !ws || (combine && !weights)) return ISC_ERR_NULL;
    const size_t b = type_bytes(d->type), yb = type_bytes(y_type);
    const int64_t pairs = static_cast<int64_t>(T) * d->slots;
    const Span in[6] = {{x, d->shared ? T : pairs, d->K, ldx, b}, {w, static_cast<int64_t>(d->E) * d->N, d->K, ldw, b},
                        flat(ids, pairs, 4), flat(combine ? weights : nullptr, pairs, 4), flat(offsets, d->E + 1, 4),
                        flat(order, pairs, 4)};
    const Span out[2] = {{y, combine ? T : pairs, d->N, ldy, yb}, flat(ws, static_cast<int64_t>(need), 1)};
    if (!in[0].shape_ok() || !in[1].shape_ok() || !out[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(w, b) || !aligned(x, b) || !aligned(y, yb) || !aligned(ids, 4) || !aligned(in[3].p, 4) ||
        !aligned(offsets, 4) || !aligned(order, 4) || !aligned(ws, kAlign))
        return ISC_ERR_ALIGN;
    if (ws_bytes < need) return ISC_ERR_WORKSPACE;
    for (const Span &o : out)
        for (const Span &s : in)
            if (overlap(o, s)) return ISC_ERR_ALIAS;
    if (overlap(out[0], out[1])) return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    isc::ExpertLinearArgs a{};
    a.a = {T, d->E, d->N, d->K, d->slots, d->type, d->shared != 0, x, w, ldx, ldw, ids, offsets, order, weights,
           isc::expert_plan_at(ws, pairs, d->E, d->type)};
    a.y = y;
    a.ldy = ldy;
    a.ytype = y_type;
    a.relu = relu != 0;
    a.combine = combine != 0;
    a.part = static_cast<float *>(isc::past(ws, static_cast<int64_t>(isc::expert_plan_bytes(pairs, d->E, d->type))));
    return hip_status(isc::launch_expert_linear(a, static_cast<hipStream_t>(stream)));
}

int isc_expert_linear_bwd_workspace_size(const isc_expert_desc *d, int32_t T, int32_t relu, int32_t combine,
                                         size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    if (const int st = check_expert(d, T)) return st;
    if (relu && combine) return ISC_ERR_ARG;
    *bytes = isc::expert_bwd_bytes(T, d->E, d->N, d->K, d->slots, d->type, d->shared != 0, relu != 0, combine != 0).all;
    return ISC_OK;
}

int isc_expert_linear_bwd(const isc_expert_desc *d, const void *w, int64_t ldw, int32_t T, const void *x, int64_t ldx,
                          const void *dy, int64_t lddy, const void *y, int64_t ldy, const int32_t *ids,
                          const float *weights, const int32_t *offsets, const int32_t *order, int32_t combine, void *dx,
                          int64_t lddx, void *dw, float *dweights, void *ws, size_t ws_bytes, void *stream) {
    size_t need = 0;
    if (const int st = isc_expert_linear_bwd_workspace_size(d, T, y != nullptr, combine, &need)) return st;
    if (dweights && !combine) return ISC_ERR_ARG;
    if (!dx && !dw && !dweights) return ISC_ERR_NULL;
    if (T == 0 && !dw) return ISC_OK;
    if (T > 0 && (!w || !x || !dy || !ids || !offsets || !order || !ws || (combine && !weights))) return ISC_ERR_NULL;
    const size_t b = type_bytes(d->type);
    const int64_t pairs = static_cast<int64_t>(T) * d->slots, xrows = d->shared ? T : pairs;
    const int64_t weightsn = static_cast<int64_t>(d->E) * d->N;
    const Span in[8] = {{x, xrows, d->K, ldx, b}, {w, weightsn, d->K, ldw, b}, {dy, combine ? T : pairs, d->N, lddy, b},
                        {y, pairs, d->N, ldy, b}, flat(ids, pairs, 4), flat(combine ? weights : nullptr, pairs, 4),
                        flat(offsets, d->E + 1, 4), flat(order, pairs, 4)};
    const Span out[4] = {{dx, xrows, d->K, lddx, b}, {dw, weightsn, d->K, d->K, b}, flat(dweights, pairs, 4),
                         flat(ws, static_cast<int64_t>(need), 1)};
    for (int i = 0; i < 4; ++i)
        if (T > 0 && !in[i].shape_ok()) return ISC_ERR_SHAPE;
    if (T > 0 && !out[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(w, b) || !aligned(x, b) || !aligned(dy, b) || !aligned(y, b) || !aligned(dx, b) || !aligned(dw, b) ||
        !aligned(ids, 4) || !aligned(in[5].p, 4) || !aligned(offsets, 4) || !aligned(order, 4) ||
        !aligned(dweights, 4) || !aligned(ws, kAlign))
        return ISC_ERR_ALIGN;
    if (T > 0 && ws_bytes < need) return ISC_ERR_WORKSPACE;
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; T > 0 && j < 8; ++j)
            if (overlap(out[i], in[j])) return ISC_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (T > 0 && overlap(out[i], out[j])) return ISC_ERR_ALIAS;
    }
    if (const int st = isc::require_gfx950()) return st;
    const isc::ExpertBwdBytes at =
        isc::expert_bwd_bytes(T, d->E, d->N, d->K, d->slots, d->type, d->shared != 0, y != nullptr, combine != 0);
    isc::ExpertBwdArgs a{};
    a.a = {T, d->E, d->N, d->K, d->slots, d->type, d->shared != 0, x, w, ldx, ldw, ids, offsets, order, weights,
           isc::expert_plan_at(ws, pairs, d->E, d->type)};
    a.dy = dy;
    a.y = y;
    a.lddy = lddy;
    a.ldy = ldy;
    a.combine = combine != 0;
    a.dx = dx;
    a.dw = dw;
    a.dweights = dweights;
    a.lddx = lddx;
    a.masked = isc::past(ws, static_cast<int64_t>(at.masked));
    a.part = static_cast<float *>(isc::past(ws, static_cast<int64_t>(at.part)));
    a.dots = static_cast<float *>(isc::past(ws, static_cast<int64_t>(at.dots)));
    return hip_status(isc::launch_expert_bwd(a, static_cast<hipStream_t>(stream)));
}

int isc_orthogonalize_workspace_size(int32_t B, int32_t M, int32_t N, size_t *bytes) {
    if (!bytes) return ISC_ERR_NULL;
    if (B < 0 || M < 1 || N < 1) return ISC_ERR_SHAPE;
    const isc::OrthShape s{B, M, N};
    if (B > 65535 || M > 65536 || N > 65536 || !isc::orth_launches_fit(s)) return ISC_ERR_LIMIT;
    *bytes = static_cast<size_t>(s.bytes());
    return ISC_OK;
}

int isc_orthogonalize(int32_t B, int32_t M, int32_t N, int32_t type, const void *g, int64_t ldg, int32_t steps,
                      const float *coefficients, float eps, void *o, int32_t o_type, int64_t ldo, void *ws,
                      size_t ws_bytes, void *stream) {
    size_t need = 0;
    if (const int st = isc_orthogonalize_workspace_size(B, M, N, &need)) return st;
    if (!element_type(type) || (o_type != ISC_F16 && o_type != ISC_BF16) || steps < 1 || steps > 64 ||
        !(eps >= 0.0f) || std::isinf(eps))
        return ISC_ERR_ARG;
    if (!coefficients) return ISC_ERR_NULL;
    double most = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double a = coefficients[3 * i], b = coefficients[3 * i + 1], c = coefficients[3 * i + 2];
        // b A + c A A is an fp16 operand too: 2^6 times it stays below 2^16
        if (!(std::fabs(b) * most * most + std::fabs(c) * std::pow(most, 4) <= 512.0)) return ISC_ERR_ARG;
        most = most_of(a, b, c, most);
        if (!(most <= 16.0)) return ISC_ERR_ARG;
    }
    if (B == 0) return ISC_OK;
    if (!g || !o || !ws) return ISC_ERR_NULL;
    const int64_t rows = static_cast<int64_t>(B) * M;
    const Span in{g, rows, N, ldg, type_bytes(type)};
    const Span out[2] = {{o, rows, N, ldo, 2}, flat(ws, static_cast<int64_t>(need), 1)};
    if (!in.shape_ok() || !out[0].shape_ok()) return ISC_ERR_SHAPE;
    if (!aligned(g, type_bytes(type)) || !aligned(o, 2) || !aligned(ws, kAlign)) return ISC_ERR_ALIGN;
    if (ws_bytes < need) return ISC_ERR_WORKSPACE;
    // g is read before o is written
    if ((overlap(out[0], in) && !in_place(out[0], in)) || overlap(out[1], in) || overlap(out[0], out[1]))
        return ISC_ERR_ALIAS;
    if (const int st = isc::require_gfx950()) return st;
    const isc::OrthArgs a{isc::OrthShape{B, M, N}, g, ldg, type, o_type, steps, coefficients, eps, o, ldo,
                          static_cast<char *>(ws)};
    return hip_status(isc::launch_orthogonalize(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
