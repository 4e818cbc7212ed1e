// tbn_api_ffn.cpp -- C ABI of the feed-forward operators (declared in include/tbn.h): the gated block of two-bit filters,
// Muon's step, products in 8-bit integers.  Argument validation, workspace layout and launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>

#include "tbn.h"
#include "tbn_checks.h"
#include "tbn_kernels.h"

using namespace tbn::checks;

namespace {

// ---- the gated block ---------------------------------------------------------------------
tbn_status check_glu(const tbn_glu_desc* d) {
    if (!d) return fail(TBN_ERR_NULL, "desc is NULL");
    if (d->rows <= 0 || d->c <= 0 || d->f <= 0) return fail(TBN_ERR_SHAPE, "every size must be positive");
    if (d->act != TBN_ACT_SILU && d->act != TBN_ACT_GELU && d->act != TBN_ACT_RELU) return fail(TBN_ERR_UNSUPPORTED, "unknown activation");
    const int64_t most = (int64_t)1 << 34;
    if (d->c > (1 << 20) || d->f > (1 << 24) || d->rows > (1 << 30) || d->rows > most / (d->c + 7) || d->rows > most / d->f)
        return fail(TBN_ERR_SHAPE, "tensor too large");
    if (tbn_packed_bytes(2 * (int64_t)d->f, d->c) >= (int64_t)1 << 31) return fail(TBN_ERR_SHAPE, "codes of 2 GiB and more");
    return TBN_OK;
}

int32_t padded(const tbn_glu_desc* d) { return (d->c + 7) / 8 * 8; }
int64_t glu_ws(const tbn_glu_desc* d) { return d->c % 8 ? d->rows * padded(d) * 2 : 0; }

// x with its rows padded where the kernels need it; null: a failed launch in *e.
const uint16_t* glu_input(const tbn_glu_desc* d, const void* x, void* ws, hipStream_t stream, hipError_t* e) {
    *e = hipSuccess;
    if (d->c % 8 == 0) return static_cast<const uint16_t*>(x);
    *e = tbn::launch_pad_channels(tbn::make_pad(x, d->rows, d->c, padded(d), ws), tbn::PadArgs{}, stream);
    return *e == hipSuccess ? static_cast<const uint16_t*>(ws) : nullptr;
}

// ---- Muon --------------------------------------------------------------------------------
tbn_status check_muon(const tbn_muon_tensor* t, int32_t n) {
    if (!t) return fail(TBN_ERR_NULL, "tensors is NULL");
    if (n <= 0 || n > (1 << 20)) return fail(TBN_ERR_SHAPE, "1 to 2^20 tensors");
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].rows <= 0 || t[i].cols <= 0) return fail(TBN_ERR_SHAPE, "every size must be positive");
        if (t[i].rows > (1 << 20) || t[i].cols > (1 << 20) || (int64_t)t[i].rows * t[i].cols >= (int64_t)1 << 31)
            return fail(TBN_ERR_SHAPE, "matrix too large");
    }
    return TBN_OK;
}

struct Span {
    uintptr_t begin, end;
    bool operator<(const Span& o) const { return begin < o.begin; }
};

Span span(const void* p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes}; }

// Whether arrays that are written overlap one another, or one that is read one of them.
tbn_status check_muon_overlap(const tbn_muon_tensor* t, int32_t n, int64_t g_size, const void* ws, int64_t ws_bytes, const void* lr) {
    const size_t count = (size_t)n * 2 + 1;
    const std::unique_ptr<Span[]> s(new (std::nothrow) Span[count]);
    if (!s) return fail(TBN_ERR_HIP, "out of host memory");
    for (int32_t i = 0; i < n; ++i) {
        s[2 * (size_t)i] = span(t[i].w, (int64_t)t[i].rows * t[i].cols * 4);
        s[2 * (size_t)i + 1] = span(t[i].m, (int64_t)t[i].rows * t[i].cols * 4);
    }
    s[count - 1] = span(ws, ws_bytes);
    std::sort(s.get(), s.get() + count);
    bool bad = false;
    for (size_t i = 1; i < count; ++i) bad |= s[i].begin < s[i - 1].end;
    auto meets = [&](const Span& g) {  // s is in order and apart: the last one that begins before g's end
        const Span* const next = std::lower_bound(s.get(), s.get() + count, Span{g.end, 0});
        return next != s.get() && g.begin < (next - 1)->end;
    };
    for (int32_t i = 0; i < n && !bad; ++i) bad = meets(span(t[i].g, (int64_t)t[i].rows * t[i].cols * g_size));
    if (bad || (lr && meets(span(lr, 4)))) return fail(TBN_ERR_SHAPE, "an array that is written, or the workspace, overlaps another");
    return TBN_OK;
}

int64_t muon_ws(const tbn_muon_tensor* t, int32_t n) {
    int64_t most = 0;
    for (int32_t at = 0; at < n;) {
        const int k = tbn::muon_group(t + at, n - at);
        most = std::max(most, tbn::muon_group_bytes(t + at, k));
        at += k;
    }
    return most;
}

// ---- products in 8-bit integers ----------------------------------------------------------
tbn_status check_rows(int64_t rows, int64_t c) {
    if (rows <= 0 || c <= 0) return fail(TBN_ERR_SHAPE, "every size must be positive");
    if (c > (1 << 24) || rows > (1 << 30) || rows > ((int64_t)1 << 34) / c) return fail(TBN_ERR_SHAPE, "tensor too large");
    return TBN_OK;
}

}  // namespace

extern "C" {

tbn_status tbn_glu_workspace_size(const tbn_glu_desc* desc, size_t* bytes) {
    if (!bytes) return fail(TBN_ERR_NULL, "bytes is NULL");
    const tbn_status st = check_glu(desc);
    if (st != TBN_OK) return st;
    *bytes = (size_t)glu_ws(desc);
    return TBN_OK;
}

tbn_status tbn_glu_fwd(const tbn_glu_desc* desc, const void* x, const uint32_t* codes, const float* alpha, void* h, tbn_dtype ht,
                       void* gu, void* ws, size_t ws_bytes, hipStream_t stream) {
    tbn_status st = check_glu(desc);
    if (st != TBN_OK) return st;
    if (!x || !codes || !alpha || !h) return fail(TBN_ERR_NULL, "x, codes, alpha and h are required");
    if (!known(ht)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (!aligned(x, 16) || !aligned(codes, 16) || !aligned(alpha, 4) || !aligned(h, 16) || !aligned(gu, 16))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const int64_t need = glu_ws(desc), rc = desc->rows * desc->c, rf = desc->rows * desc->f;
    if (need && (st = check_ws(ws, ws_bytes, need)) != TBN_OK) return st;
    if (overlap({{h, rf * size_of(ht)}, {gu, rf * 4}, {need ? ws : nullptr, need}},
                {{x, rc * 2}, {codes, tbn_packed_bytes(2 * (int64_t)desc->f, desc->c)}, {alpha, (int64_t)desc->f * 8}}))
        return fail(TBN_ERR_SHAPE, "an output or the workspace overlaps another operand");
    hipError_t e;
    tbn::GluArgs a = {};
    a.x = glu_input(desc, x, ws, stream, &e);
    if (e != hipSuccess) return done(e, "tbn_glu_fwd");
    a.codes = codes;
    a.alpha = alpha;
    a.h = h;
    a.gu = static_cast<uint16_t*>(gu);
    a.rows = desc->rows;
    a.c = padded(desc);
    a.f = desc->f;
    a.h_f32 = ht == TBN_F32;
    return done(tbn::launch_glu(a, nullptr, desc->act, stream), "tbn_glu_fwd");
}

tbn_status tbn_glu_bwd(const tbn_glu_desc* desc, const void* dh, const void* gu, const void* x, const uint32_t* codes,
                       const float* alpha, void* dgu, void* h, tbn_dtype ht, void* ws, size_t ws_bytes, hipStream_t stream) {
    tbn_status st = check_glu(desc);
    if (st != TBN_OK) return st;
    if (!dh || !dgu) return fail(TBN_ERR_NULL, "dh and dgu are required");
    if (!gu && (!x || !codes || !alpha)) return fail(TBN_ERR_NULL, "without gu, x, codes and alpha are required");
    if (!known(ht)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (gu) x = nullptr, codes = nullptr, alpha = nullptr;
    if (!aligned(dh, 16) || !aligned(gu, 16) || !aligned(x, 16) || !aligned(codes, 16) || !aligned(alpha, 4) || !aligned(dgu, 16) ||
        !aligned(h, 16))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const int64_t need = gu ? 0 : glu_ws(desc), rc = desc->rows * desc->c, rf = desc->rows * desc->f;
    if (need && (st = check_ws(ws, ws_bytes, need)) != TBN_OK) return st;
    if (overlap({{dgu, rf * 4}, {h, rf * size_of(ht)}, {need ? ws : nullptr, need}},
                {{dh, rf * 2}, {gu, rf * 4}, {x, rc * 2}, {codes, tbn_packed_bytes(2 * (int64_t)desc->f, desc->c)},
                 {alpha, (int64_t)desc->f * 8}}))
        return fail(TBN_ERR_SHAPE, "an output or the workspace overlaps another operand");
    tbn::GluArgs a = {};
    if (!gu) {
        hipError_t e;
        a.x = glu_input(desc, x, ws, stream, &e);
        if (e != hipSuccess) return done(e, "tbn_glu_bwd");
    }
    a.codes = codes;
    a.alpha = alpha;
    a.dh = static_cast<const uint16_t*>(dh);
    a.h = h;
    a.gu = static_cast<uint16_t*>(dgu);
    a.rows = desc->rows;
    a.c = padded(desc);
    a.f = desc->f;
    a.h_f32 = ht == TBN_F32;
    return done(tbn::launch_glu(a, static_cast<const uint16_t*>(gu), desc->act, stream), "tbn_glu_bwd");
}

tbn_status tbn_muon_workspace_size(const tbn_muon_tensor* tensors, int32_t n, size_t* bytes) {
    if (!bytes) return fail(TBN_ERR_NULL, "bytes is NULL");
    const tbn_status st = check_muon(tensors, n);
    if (st != TBN_OK) return st;
    *bytes = (size_t)muon_ws(tensors, n);
    return TBN_OK;
}

tbn_status tbn_muon_step(const tbn_muon_tensor* tensors, int32_t n, tbn_dtype gt, const tbn_muon_hyper* hyper, void* ws,
                         size_t ws_bytes, hipStream_t stream) {
    tbn_status st = check_muon(tensors, n);
    if (st != TBN_OK) return st;
    if (!hyper) return fail(TBN_ERR_NULL, "hyper is NULL");
    if (!known(gt)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    const int64_t g_size = size_of(gt);
    for (int32_t i = 0; i < n; ++i) {
        if (!tensors[i].w || !tensors[i].m || !tensors[i].g) return fail(TBN_ERR_NULL, "w, m and g are required");
        if (!aligned(tensors[i].w, 4) || !aligned(tensors[i].m, 4) || !aligned(tensors[i].g, (uintptr_t)g_size))
            return fail(TBN_ERR_ALIGN, "misaligned pointer");
        if (!std::isfinite(tensors[i].weight_decay) || !std::isfinite(tensors[i].scale))
            return fail(TBN_ERR_SHAPE, "weight_decay and scale have to be finite");
    }
    // (as the kernels take them, in fp32)
    if (!((float)hyper->momentum >= 0 && (float)hyper->momentum < 1)) return fail(TBN_ERR_SHAPE, "momentum has to be in [0, 1)");
    if (!(hyper->eps >= 1e-30 && hyper->eps <= 1)) return fail(TBN_ERR_SHAPE, "eps has to be in [1e-30, 1]");
    if (hyper->steps < 1 || hyper->steps > tbn::kMuonSteps) return fail(TBN_ERR_SHAPE, "1 to 32 steps");
    if (!hyper->lr_dev && !std::isfinite((float)hyper->lr)) return fail(TBN_ERR_SHAPE, "lr has to be finite");
    if (!aligned(hyper->lr_dev, 4)) return fail(TBN_ERR_ALIGN, "misaligned lr_dev");
    const int64_t need = muon_ws(tensors, n);
    if ((st = check_ws(ws, ws_bytes, need)) != TBN_OK) return st;
    if ((st = check_muon_overlap(tensors, n, g_size, ws, need, hyper->lr_dev)) != TBN_OK) return st;
    tbn::MuonHyper h = {};
    h.lr = (float)hyper->lr;
    h.lr_dev = hyper->lr_dev;
    h.momentum = (float)hyper->momentum;
    h.eps = (float)hyper->eps;
    h.steps = hyper->steps;
    h.nesterov = hyper->nesterov != 0;
    h.g_f32 = gt == TBN_F32;
    for (int32_t at = 0; at < n;) {
        const int k = tbn::muon_group(tensors + at, n - at);
        const hipError_t e = tbn::launch_muon_group(tensors + at, k, h, static_cast<uint8_t*>(ws), stream);
        if (e != hipSuccess) return done(e, "tbn_muon_step");
        at += k;
    }
    return TBN_OK;
}

tbn_status tbn_quantize_rows_i8(const void* x, tbn_dtype xt, int64_t rows, int32_t c, int8_t* q, float* scale, hipStream_t stream) {
    if (!x || !q || !scale) return fail(TBN_ERR_NULL, "x, q and scale are required");
    const tbn_status st = check_rows(rows, c);
    if (st != TBN_OK) return st;
    if (!known(xt)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4)) return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const int64_t pitch = ((int64_t)c + 15) / 16 * 16;
    if (overlap({{q, rows * pitch}, {scale, rows * 4}}, {{x, rows * c * size_of(xt)}}))
        return fail(TBN_ERR_SHAPE, "an output overlaps an input or another output");
    const int64_t most = 1 << 22;  // rows a launch: 2^30 threads
    for (int64_t r = 0; r < rows; r += most) {
        const hipError_t e = tbn::launch_rows_i8(static_cast<const uint8_t*>(x) + r * c * size_of(xt), xt == TBN_F32, std::min(most, rows - r), c,
                                                 q + r * pitch, scale + r, stream);
        if (e != hipSuccess) return done(e, "tbn_quantize_rows_i8");
    }
    return TBN_OK;
}

tbn_status tbn_matmul_i8(int64_t rows, int32_t n, int32_t c, const int8_t* q, const float* x_scale, const int8_t* w,
                         const float* w_scale, const tbn_epilogue* ep, void* y, tbn_dtype yt, hipStream_t stream) {
    if (!q || !x_scale || !w || !w_scale || !y) return fail(TBN_ERR_NULL, "q, w, their scales and y are required");
    tbn_status st = check_rows(rows, c);
    if (st != TBN_OK || (st = check_rows(rows, n)) != TBN_OK || (st = check_rows(n, c)) != TBN_OK) return st;
    if (c % 16 != 0) return fail(TBN_ERR_SHAPE, "rows are padded to a multiple of 16 values");
    if (c > 131056) return fail(TBN_ERR_SHAPE, "sums of more than 131056 products leave 32 bits");
    if (!known(yt)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    const tbn_epilogue none = {};
    if (!ep) ep = &none;
    if (!aligned(q, 16) || !aligned(w, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(y, 16) || !aligned(ep->scale, 4) ||
        !aligned(ep->bias, 4) || !aligned(ep->residual, 16))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const int64_t out = rows * n * size_of(yt), channels = (int64_t)n * 4;
    if (overlap({{y, out}}, {{q, rows * c}, {x_scale, rows * 4}, {w, (int64_t)n * c}, {w_scale, channels}, {ep->scale, channels},
                             {ep->bias, channels}, {ep->residual == y ? nullptr : ep->residual, out}}))
        return fail(TBN_ERR_SHAPE, "y overlaps an input");
    tbn::RowsI8Args a = {};
    a.x = q;
    a.w = w;
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.scale = ep->scale;
    a.bias = ep->bias;
    a.residual = ep->residual;
    a.relu = ep->relu;
    a.y = y;
    a.rows = rows;
    a.n = n;
    a.c = c;
    a.y_f32 = yt == TBN_F32;
    return done(tbn::launch_matmul_i8(a, stream), "tbn_matmul_i8");
}

}  // extern "C"
