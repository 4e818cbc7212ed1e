// tbn_api_finetune.cpp -- C ABI of what is trained and served beside the two-bit filters (declared in
// include/tbn.h): layer normalisation, AdamW over many tensors, low-rank adapters.  Argument validation, workspace
// layout and launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <string>
#include <vector>

#include "tbn.h"
#include "tbn_kernels.h"

namespace {

tbn_status fail(tbn_status s, const char* what) { return tbn::set_error(s, what); }

tbn_status done(hipError_t e, const char* where) {
    return e == hipSuccess ? TBN_OK : tbn::set_error(TBN_ERR_HIP, std::string(where) + ": " + hipGetErrorString(e));
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool known(tbn_dtype t) { return t == TBN_BF16 || t == TBN_F32; }
int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }
int64_t size_of(tbn_dtype t) { return t == TBN_F32 ? 4 : 2; }

tbn_status check_ws(const void* ws, size_t bytes, int64_t need) {
    if (!ws || bytes < (size_t)need) return fail(TBN_ERR_WORKSPACE, "workspace too small");
    if (!aligned(ws, 16)) return fail(TBN_ERR_ALIGN, "workspace must be 16-byte aligned");
    return TBN_OK;
}

// Whether an output shares a byte with an input or with another output (operands that are not given are NULL).
struct Operand {
    const void* p;
    int64_t bytes;
};
bool meet(const void* p, int64_t bytes, const void* q, int64_t qbytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + (uintptr_t)qbytes && b < a + (uintptr_t)bytes;
}
bool overlap(std::initializer_list<Operand> outputs, std::initializer_list<Operand> inputs) {
    for (const Operand* o = outputs.begin(); o != outputs.end(); ++o) {
        if (!o->p) continue;
        for (const Operand& i : inputs)
            if (i.p && meet(o->p, o->bytes, i.p, i.bytes)) return true;
        for (const Operand* k = outputs.begin(); k != o; ++k)
            if (k->p && meet(o->p, o->bytes, k->p, k->bytes)) return true;
    }
    return false;
}

// ---- layer normalisation -----------------------------------------------------------------
tbn_status check_ln(int64_t rows, int32_t c) {
    if (rows <= 0 || c <= 0) return fail(TBN_ERR_SHAPE, "sizes must be positive");
    if (c > (1 << 30) || rows > ((int64_t)1 << 40) / c) return fail(TBN_ERR_SHAPE, "tensor too large");
    return TBN_OK;
}

// ---- AdamW -------------------------------------------------------------------------------
struct Span {
    uintptr_t begin, end;
    bool operator<(const Span& o) const { return begin < o.begin; }
};

// Whether arrays that are written overlap one another, or a gradient one of them.
bool overlap(const tbn_adamw_tensor* t, int32_t n, bool eight, int64_t g_size) {
    std::vector<Span> s;
    s.reserve((size_t)n * (eight ? 5 : 3));
    auto span = [](const void* p, int64_t bytes) {
        return Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes};
    };
    for (int32_t i = 0; i < n; ++i) s.push_back(span(t[i].w, t[i].count * 4));
    for (int32_t i = 0; i < n; ++i) s.push_back(span(t[i].m, t[i].count * (eight ? 1 : 4)));
    for (int32_t i = 0; i < n; ++i) s.push_back(span(t[i].v, t[i].count * (eight ? 1 : 4)));
    for (int32_t i = 0; eight && i < n; ++i) {
        s.push_back(span(t[i].m_scale, (t[i].count + 255) / 256 * 4));
        s.push_back(span(t[i].v_scale, (t[i].count + 255) / 256 * 4));
    }
    std::sort(s.begin(), s.end());
    for (size_t i = 1; i < s.size(); ++i)
        if (s[i].begin < s[i - 1].end) return true;
    for (int32_t i = 0; i < n; ++i) {  // s is in order and apart: the last one that begins before the gradient's end
        const Span g = span(t[i].g, t[i].count * g_size);
        const auto next = std::lower_bound(s.begin(), s.end(), Span{g.end, 0});
        if (next != s.begin() && g.begin < (next - 1)->end) return true;
    }
    return false;
}

constexpr int64_t kMostBlocks = 1 << 23;  // of a launch: 2^31 threads

// ---- adapters ----------------------------------------------------------------------------
tbn_status check_adapter(const tbn_adapter_desc* d) {
    if (!d) return fail(TBN_ERR_NULL, "desc is NULL");
    if (d->rows <= 0 || d->c <= 0 || d->k <= 0 || d->rank <= 0 || d->adapters <= 0)
        return fail(TBN_ERR_SHAPE, "every size must be positive");
    if (d->rank > 128) return fail(TBN_ERR_UNSUPPORTED, "ranks up to 128");
    if (d->adapters > 65535) return fail(TBN_ERR_UNSUPPORTED, "up to 65535 adapters");
    const int64_t most = 0x7FFFFFFF, sr = (int64_t)d->adapters * d->rank;
    const int64_t wide = d->c > d->k ? d->c : d->k;
    if (d->rows > (1 << 27) || wide > (1 << 24) || sr * wide > most || d->rows > ((int64_t)1 << 35) / wide)
        return fail(TBN_ERR_SHAPE, "tensor too large");
    // ordering the rows by adapter reads the index once for each adapter: 0.3 s at this limit, 10 at the largest sizes
    if (d->rows * d->adapters > ((int64_t)1 << 38)) return fail(TBN_ERR_UNSUPPORTED, "rows times adapters up to 2^38");
    return TBN_OK;
}

// Workspace: the partial sums of t (of dt), behind them the sums; backward also the rows by adapter and the partial
// gradients.
struct AdapterWs {
    tbn::AdapterPlan plan;
    int64_t t_off, order_off, span_off, grad_off, total;
    int32_t grad_splits;
    bool sorted;
};

AdapterWs adapter_ws(const tbn_adapter_desc* d, bool backward) {
    AdapterWs w = {};
    const int64_t rr = d->rows * d->rank * 4;
    w.plan = tbn::plan_adapter_shrink(d->rows, backward ? d->k : d->c, d->rank, d->adapters);
    w.t_off = w.plan.splits > 1 ? round256(w.plan.splits * rr) : 0;
    w.total = w.t_off + round256(rr);
    w.sorted = tbn::adapter_sorted_rows(d->rows, d->adapters);
    if (backward || w.sorted) {
        w.order_off = w.total;
        w.span_off = w.order_off + round256(d->rows * 4);
        w.total = w.span_off + round256((int64_t)d->adapters * 8);
    }
    if (backward) {
        w.grad_off = w.total;
        w.grad_splits = tbn::adapter_outer_splits(d->rows, d->c, d->k, d->adapters);
        const int64_t grads = (int64_t)d->adapters * d->rank * ((int64_t)d->c + d->k) * 4;
        w.total = w.grad_off + (w.grad_splits > 1 ? round256(w.grad_splits * grads) : 0);
    }
    return w;
}

// Sizes of the operands: values of x and of y, of a bank's a and b; bytes of the others.
struct AdapterBytes {
    int64_t rc, rk, rank_c, rank_k, t, index, scale, a, b;
    AdapterBytes(const tbn_adapter_desc* d, tbn_dtype wt)
        : rc(d->rows * d->c), rk(d->rows * d->k), rank_c((int64_t)d->adapters * d->rank * d->c),
          rank_k((int64_t)d->adapters * d->rank * d->k), t(d->rows * d->rank * 4), index(d->rows * 4), scale((int64_t)d->adapters * 4),
          a(rank_c * size_of(wt)), b(rank_k * size_of(wt)) {}
};

// Whether the expanding kernel adds the partial sums itself, which saves few rows a launch of 2 us.
bool expand_sums(int32_t splits, const tbn_adapter_desc* d) {
    return splits > 1 && tbn::adapter_few_rows(d->rows, d->adapters);
}

tbn::AdapterArgs adapter_args(const tbn_adapter_desc* d, const int32_t* index, tbn_dtype wt) {
    tbn::AdapterArgs a = {};
    a.index = index;
    a.rows = d->rows;
    a.R = d->rank;
    a.S = d->adapters;
    a.splits = 1;
    a.w_f32 = wt == TBN_F32;
    return a;
}

}  // namespace

extern "C" {

tbn_status tbn_layernorm_fwd(const void* x, tbn_dtype xt, int64_t rows, int32_t c, const float* gamma, const float* beta,
                             float eps, void* y, tbn_dtype yt, float* mean, float* inv_std, hipStream_t stream) {
    if (!x || !y) return fail(TBN_ERR_NULL, "x and y are required");
    tbn_status st = check_ln(rows, c);
    if (st != TBN_OK) return st;
    if (!known(xt) || !known(yt)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (!(eps >= 0) || !std::isfinite(eps)) return fail(TBN_ERR_SHAPE, "eps has to be finite and not negative");
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) ||
        !aligned(inv_std, 4))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const int64_t stats = rows * 4, params = (int64_t)c * 4;
    if (overlap({{y, rows * c * size_of(yt)}, {mean, stats}, {inv_std, stats}},
                {{x, rows * c * size_of(xt)}, {gamma, params}, {beta, params}}))
        return fail(TBN_ERR_SHAPE, "an output overlaps an input or another output");
    tbn::LnArgs a = {};
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.inv_std = inv_std;
    a.rows = rows;
    a.C = c;
    a.eps = eps;
    a.x_f32 = xt == TBN_F32;
    a.y_f32 = yt == TBN_F32;
    return done(tbn::launch_layernorm_fwd(a, stream), "tbn_layernorm_fwd");
}

tbn_status tbn_layernorm_workspace_size(int64_t rows, int32_t c, size_t* bytes) {
    if (!bytes) return fail(TBN_ERR_NULL, "bytes is NULL");
    tbn_status st = check_ln(rows, c);
    if (st != TBN_OK) return st;
    *bytes = tbn::layernorm_bwd_bytes(rows, c);
    return TBN_OK;
}

tbn_status tbn_layernorm_bwd(const void* x, tbn_dtype xt, const void* dy, tbn_dtype yt, int64_t rows, int32_t c,
                             const float* mean, const float* inv_std, const float* gamma, void* dx, float* dgamma,
                             float* dbeta, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (!x || !dy || !mean || !inv_std || !dx || !dgamma || !dbeta) return fail(TBN_ERR_NULL, "missing pointer");
    size_t need;
    tbn_status st = tbn_layernorm_workspace_size(rows, c, &need);
    if (st != TBN_OK) return st;
    if (!known(xt) || !known(yt)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(mean, 4) || !aligned(inv_std, 4) ||
        !aligned(gamma, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    st = check_ws(ws, ws_bytes, (int64_t)need);
    if (st != TBN_OK) return st;
    const int64_t x_bytes = rows * c * size_of(xt), stats = rows * 4, params = (int64_t)c * 4;
    if (overlap({{dx, x_bytes}, {dgamma, params}, {dbeta, params}, {ws, (int64_t)need}},
                {{x, x_bytes}, {dy, rows * c * size_of(yt)}, {mean, stats}, {inv_std, stats}, {gamma, params}}))
        return fail(TBN_ERR_SHAPE, "an output or the workspace overlaps another operand");
    tbn::LnArgs a = {};
    a.x = x;
    a.dy = dy;
    a.dx = dx;
    a.gamma = gamma;
    a.mean = const_cast<float*>(mean);
    a.inv_std = const_cast<float*>(inv_std);
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.partial = reinterpret_cast<float*>(ws);
    a.rows = rows;
    a.C = c;
    a.x_f32 = xt == TBN_F32;
    a.y_f32 = yt == TBN_F32;
    return done(tbn::launch_layernorm_bwd(a, stream), "tbn_layernorm_bwd");
}

tbn_status tbn_adamw_step(const tbn_adamw_tensor* tensors, int32_t n, tbn_state state, tbn_dtype gt,
                          const tbn_adamw_hyper* h, hipStream_t stream) try {
    if (!tensors || !h) return fail(TBN_ERR_NULL, "tensors and hyper are required");
    if (n <= 0) return fail(TBN_ERR_SHAPE, "at least one tensor is required");
    if ((state != TBN_STATE_F32 && state != TBN_STATE_E4M3) || !known(gt))
        return fail(TBN_ERR_UNSUPPORTED, "unknown state or gradient type");
    if (!(h->beta1 >= 0 && h->beta1 < 1) || !(h->beta2 >= 0 && h->beta2 < 1) || !(h->eps >= 0) || !std::isfinite(h->eps) ||
        (!h->lr_dev && !std::isfinite(h->lr)) || (!h->step_dev && h->step < 1))
        return fail(TBN_ERR_SHAPE, "betas have to be in [0, 1), eps >= 0, lr finite and step >= 1");
    if (!aligned(h->step_dev, 4) || !aligned(h->lr_dev, 4)) return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const bool eight = state == TBN_STATE_E4M3;
    for (int32_t i = 0; i < n; ++i) {
        const tbn_adamw_tensor& t = tensors[i];
        if (!t.w || !t.m || !t.v || !t.g || (eight && (!t.m_scale || !t.v_scale)))
            return fail(TBN_ERR_NULL, "w, m, v, g and, for 8-bit states, the scales are required");
        if (t.count <= 0) return fail(TBN_ERR_SHAPE, "count must be positive");
        if (t.count > kMostBlocks * tbn::kAdamwRound) return fail(TBN_ERR_SHAPE, "count too large");
        if (!std::isfinite(t.weight_decay)) return fail(TBN_ERR_SHAPE, "weight_decay must be finite");
        const uintptr_t s = eight ? 1 : 4;
        if (!aligned(t.w, 4) || !aligned(t.m, s) || !aligned(t.v, s) || !aligned(t.g, gt == TBN_F32 ? 4 : 2) ||
            (eight && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
            return fail(TBN_ERR_ALIGN, "misaligned pointer");
    }
    if (overlap(tensors, n, eight, gt == TBN_F32 ? 4 : 2))
        return fail(TBN_ERR_SHAPE, "arrays that are written overlap (or a tensor is listed twice), or a gradient overlaps one");

    tbn::AdamwBatch b = {};
    b.step = (uint32_t)h->step;
    b.seed = h->seed;
    b.step_dev = h->step_dev;
    b.lr_dev = h->lr_dev;
    b.lr = h->lr;
    b.beta1 = h->beta1;
    b.beta2 = h->beta2;
    b.eps = h->eps;
    if (!h->step_dev) {
        b.c1 = -std::expm1(h->step * std::log(h->beta1));
        b.c2 = -std::expm1(h->step * std::log(h->beta2));
    }
    // A block takes four rounds, whose loads it issues together, unless that leaves CUs without a block: 100000 weights 3.3 us,
    // with four rounds 5.1 (8-bit states 4.2 and 6.9); 700000 5.5 and 6.6; 1500000 8.6 with four; 268 M with 8-bit
    // states 809 with four, 890 with one at a time.
    int64_t all = 0;
    for (int32_t i = 0; i < n; ++i) all += (tensors[i].count + tbn::kAdamwRound - 1) / tbn::kAdamwRound;
    b.rounds = all >= 1024 ? 4 : all >= 512 ? 2 : 1;
    const int64_t chunk = (int64_t)b.rounds * tbn::kAdamwRound;
    int64_t blocks = 0;
    auto flush = [&]() {
        if (b.n == 0) return hipSuccess;
        const hipError_t e = tbn::launch_adamw(b, blocks, gt == TBN_BF16, eight, stream);
        b.n = 0;
        blocks = 0;
        return e;
    };
    for (int32_t i = 0; i < n; ++i) {
        const tbn_adamw_tensor& t = tensors[i];
        const int64_t need = (t.count + chunk - 1) / chunk;
        if (b.n == tbn::kAdamwTensors || blocks + need > kMostBlocks) {
            const hipError_t e = flush();
            if (e != hipSuccess) return done(e, "tbn_adamw_step");
        }
        if (b.n == 0) b.first = i;
        b.t[b.n++] = {t.w, t.m, t.v, t.g, t.m_scale, t.v_scale, t.count, t.weight_decay, (int32_t)blocks};
        blocks += need;
    }
    return done(flush(), "tbn_adamw_step");
} catch (...) {
    return TBN_ERR_HIP;  // host memory ran out; nothing has been queued
}

tbn_status tbn_adapter_workspace_size(tbn_op op, const tbn_adapter_desc* desc, size_t* bytes) {
    tbn_status st = check_adapter(desc);
    if (st != TBN_OK) return st;
    if (!bytes) return fail(TBN_ERR_NULL, "bytes is NULL");
    if (op != TBN_OP_FWD && op != TBN_OP_BWD_DATA) return fail(TBN_ERR_UNSUPPORTED, "unknown op");
    *bytes = (size_t)adapter_ws(desc, op == TBN_OP_BWD_DATA).total;
    return TBN_OK;
}

tbn_status tbn_adapter_fwd(const tbn_adapter_desc* desc, const void* x, tbn_dtype xt, const int32_t* index, const void* a,
                           const void* b, tbn_dtype wt, const float* scale, const void* residual, void* y, tbn_dtype yt,
                           float* t, void* ws, size_t ws_bytes, hipStream_t stream) {
    tbn_status st = check_adapter(desc);
    if (st != TBN_OK) return st;
    if (!x || !index || !a || !b || !y) return fail(TBN_ERR_NULL, "x, index, a, b and y are required");
    if (!known(xt) || !known(wt) || !known(yt)) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (!aligned(x, 16) || !aligned(a, 16) || !aligned(b, 16) || !aligned(y, 16) || !aligned(residual, 16) ||
        !aligned(index, 4) || !aligned(scale, 4) || !aligned(t, 16))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const AdapterWs w = adapter_ws(desc, false);
    st = check_ws(ws, ws_bytes, w.total);
    if (st != TBN_OK) return st;
    const AdapterBytes n(desc, wt);
    const int64_t y_bytes = n.rk * size_of(yt);
    if (overlap({{y, y_bytes}, {t, n.t}, {ws, w.total}}, {{x, n.rc * size_of(xt)}, {index, n.index}, {a, n.a}, {b, n.b}, {scale, n.scale},
                                                           {residual == y ? nullptr : residual, y_bytes}}))
        return fail(TBN_ERR_SHAPE, "an output or the workspace overlaps another operand");
    float* part = reinterpret_cast<float*>(ws);
    float* sum = t ? t : reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + w.t_off);

    tbn::AdapterArgs s = adapter_args(desc, index, wt);
    s.x = x;
    s.x_f32 = xt == TBN_F32;
    s.w = a;
    s.C = desc->c;
    s.part = w.plan.splits > 1 ? part : sum;
    hipError_t e;
    if (w.sorted) {
        s.order = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(ws) + w.order_off);
        s.span = reinterpret_cast<int2*>(reinterpret_cast<char*>(ws) + w.span_off);
        s.sorted = s.order;
        e = tbn::launch_adapter_order(s, stream);
        if (e != hipSuccess) return done(e, "tbn_adapter_fwd (order)");
    }
    e = tbn::launch_adapter_shrink(s, w.plan, 0, stream);
    if (e != hipSuccess) return done(e, "tbn_adapter_fwd (shrink)");

    tbn::AdapterArgs p = adapter_args(desc, index, wt);
    p.sorted = s.sorted;
    p.w = b;
    p.scale = scale;
    p.residual = residual;
    p.y = y;
    p.y_f32 = yt == TBN_F32;
    p.C = desc->k;
    p.part = sum;
    if (w.plan.splits > 1) {
        if (expand_sums(w.plan.splits, desc)) {
            p.part = part;
            p.splits = w.plan.splits;
            p.t = t;
        } else {
            e = tbn::launch_adapter_finish(part, desc->rows * desc->rank, w.plan.splits, sum, stream);
            if (e != hipSuccess) return done(e, "tbn_adapter_fwd (sum)");
        }
    }
    return done(tbn::launch_adapter_expand(p, 0, stream), "tbn_adapter_fwd (expand)");
}

tbn_status tbn_adapter_bwd(const tbn_adapter_desc* desc, const void* x, tbn_dtype xt, const void* dy, tbn_dtype dyt,
                           const int32_t* index, const void* a, const void* b, tbn_dtype wt, const float* scale,
                           const float* t, const void* residual, void* dx, tbn_dtype dxt, float* da, float* db, void* ws,
                           size_t ws_bytes, hipStream_t stream) {
    tbn_status st = check_adapter(desc);
    if (st != TBN_OK) return st;
    if (!x || !dy || !index || !a || !b || !t) return fail(TBN_ERR_NULL, "x, dy, index, a, b and t are required");
    if (!dx && !da && !db) return fail(TBN_ERR_NULL, "one of dx, da and db is required");
    if (!known(xt) || !known(dyt) || !known(wt) || (dx && !known(dxt))) return fail(TBN_ERR_UNSUPPORTED, "unknown dtype");
    if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(a, 16) || !aligned(b, 16) || !aligned(dx, 16) ||
        !aligned(residual, 16) || !aligned(da, 16) || !aligned(db, 16) || !aligned(index, 4) || !aligned(scale, 4) ||
        !aligned(t, 16))
        return fail(TBN_ERR_ALIGN, "misaligned pointer");
    const AdapterWs w = adapter_ws(desc, true);
    st = check_ws(ws, ws_bytes, w.total);
    if (st != TBN_OK) return st;
    const AdapterBytes n(desc, wt);
    const int64_t dx_bytes = n.rc * size_of(dxt);
    if (overlap({{dx, dx_bytes}, {da, n.rank_c * 4}, {db, n.rank_k * 4}, {ws, w.total}},
                {{x, n.rc * size_of(xt)}, {dy, n.rk * size_of(dyt)}, {index, n.index}, {a, n.a}, {b, n.b}, {scale, n.scale}, {t, n.t},
                 {residual == dx || !dx ? nullptr : residual, dx_bytes}}))
        return fail(TBN_ERR_SHAPE, "an output or the workspace overlaps another operand");
    char* base = reinterpret_cast<char*>(ws);
    float* part = reinterpret_cast<float*>(base);
    float* dt = reinterpret_cast<float*>(base + w.t_off);
    int32_t* order = reinterpret_cast<int32_t*>(base + w.order_off);
    int2* span = reinterpret_cast<int2*>(base + w.span_off);
    hipError_t e;

    tbn::AdapterArgs s = adapter_args(desc, index, wt);
    s.order = da || db || w.sorted ? order : nullptr;
    s.span = span;
    if (w.sorted || !(dx || da)) {
        e = tbn::launch_adapter_order(s, stream);
        if (e != hipSuccess) return done(e, "tbn_adapter_bwd (order)");
        s.sorted = w.sorted ? order : nullptr;
    }
    bool summed = true;  // dt holds the sums
    if (dx || da) {
        s.x = dy;
        s.x_f32 = dyt == TBN_F32;
        s.w = b;
        s.scale = scale;
        s.C = desc->k;
        s.part = w.plan.splits > 1 ? part : dt;
        e = tbn::launch_adapter_shrink(s, w.plan, 1, stream);
        if (e != hipSuccess) return done(e, "tbn_adapter_bwd (shrink)");
        summed = w.plan.splits == 1;
        if (!summed && !(dx && expand_sums(w.plan.splits, desc))) {
            e = tbn::launch_adapter_finish(part, desc->rows * desc->rank, w.plan.splits, dt, stream);
            if (e != hipSuccess) return done(e, "tbn_adapter_bwd (sum)");
            summed = true;
        }
    }
    auto expand = [&]() -> tbn_status {
        if (!dx) return TBN_OK;
        tbn::AdapterArgs p = adapter_args(desc, index, wt);
        p.sorted = s.sorted;
        p.w = a;
        p.residual = residual;
        p.y = dx;
        p.y_f32 = dxt == TBN_F32;
        p.C = desc->c;
        p.part = summed ? dt : part;
        p.splits = summed ? 1 : w.plan.splits;
        p.t = summed ? nullptr : dt;
        return done(tbn::launch_adapter_expand(p, 1, stream), "tbn_adapter_bwd (expand)");
    };
    // The gradients first: they find the end of dy in the caches (unless dt is what the expansion sums).
    if (!summed || (!da && !db)) {
        st = expand();
        if (st != TBN_OK || (!da && !db)) return st;
    }

    const int64_t na = da ? n.rank_c : 0, nb = db ? n.rank_k : 0;
    float* grads = reinterpret_cast<float*>(base + w.grad_off);
    const bool split = w.grad_splits > 1;
    tbn::AdapterOuterJob jobs[2] = {{x, dt, nullptr, split ? grads : da, desc->c, 0},
                                    {dy, t, scale, split ? grads + na : db, desc->k, 1}};
    const int f32[2] = {xt == TBN_F32, dyt == TBN_F32};
    tbn::AdapterOuter o = {};
    o.order = order;
    o.span = span;
    o.split_stride = na + nb;
    o.R = desc->rank;
    const bool together = da && db && f32[0] == f32[1];
    for (int k = 0; k < 2; ++k) {
        if (!(k ? db : da) || (together && k)) continue;
        o.job[0] = jobs[k];
        o.job[1] = together ? jobs[1] : tbn::AdapterOuterJob{};
        o.blocks0 = (uint32_t)((jobs[k].C + 63) / 64);
        e = tbn::launch_adapter_outer(o, desc->adapters, w.grad_splits, f32[k], stream);
        if (e != hipSuccess) return done(e, "tbn_adapter_bwd (gradients)");
    }
    if (split) {
        e = tbn::launch_adapter_outer_sum(grads, w.grad_splits, na, nb, da, db, stream);
        if (e != hipSuccess) return done(e, "tbn_adapter_bwd (sum)");
    }
    return summed ? expand() : TBN_OK;
}

}  // extern "C"
