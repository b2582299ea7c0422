// C entry points of the memory core's operators (linear attention, block norms) and of the clip over many gradient
// tensors: argument validation on the host.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "../../include/cleanba_layers.h"
#include "blocknorm.h"
#include "gradclip.h"
#include "linattn.h"
#include "status.h"

using namespace cb;

namespace {

// An array of rows of `w` contiguous elements at three strided axes. Axes of one element have no stride.
struct Strided {
    const char* name;
    const void* p;
    int64_t n[3], s[3];
    int64_t w;
    int es;
    bool written;

    Strided(const char* name, const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2,
            int64_t w, int es, bool written)
        : name(name), p(p), n{n0, n1, n2}, s{s0, s1, s2}, w(w), es(es), written(written) {
        for (int i = 0; i < 3; ++i)
            if (n[i] <= 1) s[i] = 0;
    }
    double reach() const {   // elements from the first to the last, as a double: strides are the caller's
        double r = double(w);
        for (int i = 0; i < 3; ++i) r += double(n[i] - 1) * double(s[i]);
        return r;
    }
    bool empty() const { return n[0] == 0 || n[1] == 0 || n[2] == 0 || w == 0; }
    size_t bytes() const { return empty() ? 0 : size_t(reach()) * es; }
    // axis numbers by falling stride
    void order(int* ax) const {
        ax[0] = 0; ax[1] = 1; ax[2] = 2;
        std::sort(ax, ax + 3, [&](int a, int b) { return s[a] > s[b]; });
    }
    // No two elements in one place, each axis stepping over all that the smaller strides span.
    bool nested() const {
        int ax[3];
        order(ax);
        int64_t span = w;
        for (int k = 2; k >= 0; --k) {
            const int i = ax[k];
            if (n[i] <= 1) continue;
            if (s[i] < span) return false;
            span += (n[i] - 1) * s[i];
        }
        return true;
    }
};

// Whether some rows of a and b (same strides, nested) share an element when b starts `d` elements after a. An axis's step
// is larger than all that the later axes span, so only the two nearest multiples of it can bring rows together.
bool rows_meet(const Strided& a, const Strided& b, const int* ax, int level, int64_t d) {
    if (level == 3) return d < a.w && -d < b.w;
    const int i = ax[level];
    if (a.n[i] <= 1 || a.s[i] == 0) return rows_meet(a, b, ax, level + 1, d);
    const int64_t f = d >= 0 ? d / a.s[i] : -((-d + a.s[i] - 1) / a.s[i]);
    for (int64_t m = f; m <= f + 1; ++m)
        if (m > -a.n[i] && m < a.n[i] && rows_meet(a, b, ax, level + 1, d - m * a.s[i])) return true;
    return false;
}

bool arrays_meet(const Strided& a, const Strided& b) {
    if (!a.p || !b.p || !ranges_overlap(a.p, a.bytes(), b.p, b.bytes())) return false;
    if (a.es != b.es) return true;
    // An axis on which they step differently (the heads of parts of one buffer, where dk is not dv) becomes part of the row,
    // with all that it spans.
    Strided x = a, y = b;
    for (int i = 0; i < 3; ++i)
        if (a.n[i] != b.n[i] || a.s[i] != b.s[i])
            for (Strided* r : {&x, &y}) {
                r->w += (r->n[i] - 1) * r->s[i];
                r->n[i] = 1;
                r->s[i] = 0;
            }
    Strided wide = x;
    wide.w = std::max(x.w, y.w);
    const int64_t d = reinterpret_cast<intptr_t>(b.p) - reinterpret_cast<intptr_t>(a.p);
    if (!wide.nested() || d % a.es) return true;
    int ax[3];
    x.order(ax);
    return rows_meet(x, y, ax, 0, d / a.es);
}

// Strides and aliases of a call's arrays. Of the first `in_place` ones an output may be an input itself.
template <size_t N>
impala_status_t check_arrays(const char* fn, const Strided (&v)[N], size_t in_place = 0) {
    for (const Strided& x : v) {
        if (!x.p) continue;
        for (int i = 0; i < 3; ++i)
            if (x.s[i] < 0) return fail(IMPALA_EINVAL, "%s: %s has a negative stride", fn, x.name);
        if (!(x.reach() < std::ldexp(1.0, 60))) return fail(IMPALA_EINVAL, "%s: %s reaches too far", fn, x.name);
        if (reinterpret_cast<uintptr_t>(x.p) % x.es) return fail(IMPALA_EINVAL, "%s: %s is misaligned", fn, x.name);
        if (x.written && !x.empty() && !x.nested())
            return fail(IMPALA_EINVAL, "%s: %s has elements in one place", fn, x.name);
    }
    auto same = [&](const Strided& a, const Strided& b) {
        return a.written != b.written && a.p == b.p && a.es == b.es && a.w == b.w && a.n[0] == b.n[0] && a.s[0] == b.s[0];
    };
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < i; ++j)
            if (!(i < in_place && same(v[i], v[j])) && (v[i].written || v[j].written) && !v[i].empty() && !v[j].empty() && arrays_meet(v[i], v[j]))
                return fail(IMPALA_EINVAL, "%s: %s and %s overlap", fn, v[j].name, v[i].name);
    return IMPALA_OK;
}

impala_status_t check_linattn(const char* fn, const linattn_shape_t* c) {
    if (!c) return fail(IMPALA_EINVAL, "%s: argument 'shape' is NULL", fn);
    if (!valid_prec(c->prec)) return fail(IMPALA_EINVAL, "%s: bad prec", fn);
    if (c->T < 0 || c->E < 0 || c->heads < 1 || c->dk < 1 || c->dv < 1)
        return fail(IMPALA_EINVAL, "%s: shape out of range", fn);
    if (c->dk > kLaMaxDim || c->dv > kLaMaxDim)
        return fail(IMPALA_EUNSUPPORTED, "%s: heads of at most %d (got dk=%d dv=%d)", fn, kLaMaxDim, c->dk, c->dv);
    if (int64_t(c->E) * c->heads > (int64_t(1) << 21) || c->T > (1 << 30))
        return fail(IMPALA_EUNSUPPORTED, "%s: at most 2^21 states and 2^30 steps in a call", fn);
    return IMPALA_OK;
}

Strided la_array(const char* name, const void* p, const linattn_shape_t& c, const linattn_strides_t& s, int w, bool written) {
    return Strided(name, p, c.T, s.t, c.E, s.e, c.heads, s.h, w, c.prec == IMPALA_PREC_BF16 ? 2 : 4, written);
}
Strided la_state(const char* name, const float* p, const linattn_shape_t& c, bool written) {
    return Strided(name, p, 1, 0, 1, 0, 1, 0, int64_t(c.E) * c.heads * c.dk * c.dv, 4, written);
}
Strided la_dones(const uint8_t* p, const linattn_shape_t& c) {
    return Strided("dones", p, c.T, c.done_t, c.E, c.done_e, 1, 0, 1, 1, false);
}
Strided la_decay(const float* p, const linattn_shape_t& c) {
    return Strided("log_decay", p, 1, 0, 1, 0, 1, 0, c.heads, 4, false);
}
LaView la_view(const void* p, const linattn_strides_t& s) { return LaView{p, s.t, s.e, s.h}; }

LaArgs la_args(const linattn_shape_t& c, const float* log_decay, const uint8_t* dones) {
    LaArgs a{};
    a.log_decay = log_decay; a.dones = dones; a.d_t = c.done_t; a.d_e = c.done_e;
    a.T = c.T; a.E = c.E; a.H = c.heads;
    return a;
}

impala_status_t run_linattn(const char* fn, const linattn_shape_t& c, const LaArgs& a, void* ws, size_t ws_bytes,
                            hipStream_t stream) {
    const size_t need = linattn_ws_bytes(c.prec, c.T, c.E, c.heads, c.dk, c.dv, a.np);
    if (need > 0 && !ws) return fail(IMPALA_EINVAL, "%s: argument 'ws' is NULL", fn);
    if (ws_bytes < need) return fail(IMPALA_EWORKSPACE, "%s: workspace %zu < %zu bytes", fn, ws_bytes, need);
    if (need > 0 && reinterpret_cast<uintptr_t>(ws) % 16) return fail(IMPALA_EINVAL, "%s: ws must be 16-byte aligned", fn);
    return hip_status(linattn(c.prec, a, ws, stream), fn);
}

impala_status_t linattn_forward(const char* fn, const linattn_shape_t& c, const void* q, const void* k, const void* v,
                                const float* log_decay, const uint8_t* dones, const float* s0, void* o, float* s_out,
                                void* ws, size_t ws_bytes, hipStream_t stream) {
    if (c.E == 0) return ok();
    if (c.T > 0 && (!q || !k || !v || !o || !log_decay)) return fail(IMPALA_EINVAL, "%s: an array is NULL", fn);
    const Strided v_[] = {la_array("q", q, c, c.q, c.dk, false), la_array("k", k, c, c.k, c.dk, false),
                          la_array("v", v, c, c.v, c.dv, false), la_array("o", o, c, c.o, c.dv, true),
                          la_dones(dones, c), la_decay(log_decay, c),
                          // the state may go through in place, so s0 counts only where it is another
                          la_state("s0", s0 == s_out ? nullptr : s0, c, false), la_state("s_out", s_out, c, true)};
    const impala_status_t st = check_arrays(fn, v_);
    if (st) return st;
    LaArgs a = la_args(c, log_decay, dones);
    LaPass& p = a.pass[a.np++];
    p.q = la_view(q, c.q); p.k = la_view(k, c.k); p.v = la_view(v, c.v); p.o = la_view(o, c.o);
    p.x0 = s0; p.x1 = s_out; p.dk = c.dk; p.dv = c.dv; p.xk = c.dv; p.xn = 1;
    p.in = 1.f; p.out = c.scale;
    return run_linattn(fn, c, a, ws, ws_bytes, stream);
}

impala_status_t check_blocknorm(const char* fn, const blocknorm_shape_t* c) {
    if (!c) return fail(IMPALA_EINVAL, "%s: argument 'shape' is NULL", fn);
    if (!valid_prec(c->prec)) return fail(IMPALA_EINVAL, "%s: bad prec", fn);
    if (c->n < 0 || c->n > (int64_t(1) << 40) || c->C < 1 || c->groups < 1 || c->C % c->groups)
        return fail(IMPALA_EINVAL, "%s: shape out of range (groups must divide C)", fn);
    if (c->C > kBnMaxC) return fail(IMPALA_EUNSUPPORTED, "%s: at most %d channels (got %d)", fn, kBnMaxC, c->C);
    if (c->norm < IMPALA_NORM_NONE || c->norm > IMPALA_NORM_RMS || c->norm2 < IMPALA_NORM_NONE || c->norm2 > IMPALA_NORM_RMS)
        return fail(IMPALA_EINVAL, "%s: bad norm", fn);
    if (c->gate_act < IMPALA_GATE_LINEAR || c->gate_act > IMPALA_GATE_SIGMOID)
        return fail(IMPALA_EINVAL, "%s: bad gate_act %d", fn, c->gate_act);
    if (!(c->eps >= 0.f)) return fail(IMPALA_EINVAL, "%s: eps must be >= 0", fn);
    return IMPALA_OK;
}

Strided bn_rows(const char* name, const void* p, const blocknorm_shape_t& c, int64_t ld, bool written) {
    return Strided(name, p, c.n, ld, 1, 0, 1, 0, c.C, c.prec == IMPALA_PREC_BF16 ? 2 : 4, written);
}
Strided bn_cols(const char* name, const float* p, const blocknorm_shape_t& c, bool written) {
    return Strided(name, p, 1, 0, 1, 0, 1, 0, c.C, 4, written);
}

BnArgs bn_args(const blocknorm_shape_t& c) {
    BnArgs a{};
    a.n = c.n; a.C = c.C; a.G = c.groups; a.norm = c.norm; a.norm2 = c.norm2; a.act = c.gate_act; a.eps = c.eps;
    return a;
}
BnMat bn_mat(const void* p, int64_t ld) { return BnMat{const_cast<void*>(p), ld}; }

template <size_t N>
impala_status_t check_lds(const char* fn, const blocknorm_shape_t& c, const Strided (&v)[N], int rows) {
    for (int i = 0; i < rows; ++i)
        if (v[i].p && c.n > 1 && v[i].s[0] < c.C)
            return fail(IMPALA_EINVAL, "%s: the row stride of %s is below C", fn, v[i].name);
    return IMPALA_OK;
}

}  // namespace

extern "C" {

size_t impala_linattn_workspace_bytes(const linattn_shape_t* shape, int backward) {
    if (check_linattn(__func__, shape) != IMPALA_OK) return 0;
    ok();
    return linattn_ws_bytes(shape->prec, shape->T, shape->E, shape->heads, shape->dk, shape->dv, backward ? 3 : 1);
}

impala_status_t impala_linattn_fwd(const linattn_shape_t* shape, const void* q, const void* k, const void* v,
                                   const float* log_decay, const uint8_t* dones, const float* s0, void* o,
                                   float* s_out, void* ws, size_t ws_bytes, hipStream_t stream) {
    const impala_status_t st = check_linattn(__func__, shape);
    if (st) return st;
    return linattn_forward(__func__, *shape, q, k, v, log_decay, dones, s0, o, s_out, ws, ws_bytes, stream);
}

impala_status_t impala_linattn_step(const linattn_shape_t* shape, const void* q, const void* k, const void* v,
                                    const float* log_decay, const uint8_t* dones, const float* s_in, void* o,
                                    float* s_out, hipStream_t stream) {
    const impala_status_t st = check_linattn(__func__, shape);
    if (st) return st;
    if (shape->T != 1) return fail(IMPALA_EINVAL, "impala_linattn_step: T must be 1 (got %d)", shape->T);
    if (shape->E > 0) CHECK_PTR(s_out);
    return linattn_forward(__func__, *shape, q, k, v, log_decay, dones, s_in, o, s_out, nullptr, 0, stream);
}

impala_status_t impala_linattn_bwd(const linattn_shape_t* shape, const void* d_o, const void* q, const void* k,
                                   const void* v, const float* log_decay, const uint8_t* dones, const float* s0,
                                   const float* ds_out, void* dq, void* dk, void* dv, float* ds0, void* ws,
                                   size_t ws_bytes, hipStream_t stream) {
    const impala_status_t st = check_linattn(__func__, shape);
    if (st) return st;
    const linattn_shape_t& c = *shape;
    if (c.E == 0) return ok();
    if (c.T > 0) {
        CHECK_PTR(d_o); CHECK_PTR(q); CHECK_PTR(k); CHECK_PTR(v); CHECK_PTR(log_decay);
        CHECK_PTR(dq); CHECK_PTR(dk); CHECK_PTR(dv);
    }
    const Strided v_[] = {la_array("d_o", d_o, c, c.o, c.dv, false), la_array("q", q, c, c.q, c.dk, false),
                          la_array("k", k, c, c.k, c.dk, false), la_array("v", v, c, c.v, c.dv, false),
                          la_array("dq", dq, c, c.gq, c.dk, true), la_array("dk", dk, c, c.gk, c.dk, true),
                          la_array("dv", dv, c, c.gv, c.dv, true), la_dones(dones, c), la_decay(log_decay, c),
                          la_state("s0", s0, c, false), la_state("ds_out", ds_out, c, false),
                          la_state("ds0", ds0, c, true)};
    const impala_status_t sv = check_arrays(__func__, v_);
    if (sv) return sv;
    LaArgs a = la_args(c, log_decay, dones);
    // dq_t = scale S_t d_o_t: the forward pass with k and v exchanged and the transposed state
    LaPass& p = a.pass[a.np++];
    p.q = la_view(d_o, c.o); p.k = la_view(v, c.v); p.v = la_view(k, c.k); p.o = la_view(dq, c.gq);
    p.x0 = s0; p.dk = c.dv; p.dv = c.dk; p.xk = 1; p.xn = c.dv; p.in = 1.f; p.out = c.scale;
    // dk_t = G_t v_t and dv_t = G_t^T k_t, with G the sum of q d_o^T from the end on
    LaPass& r = a.pass[a.np++];
    r.q = la_view(v, c.v); r.k = la_view(d_o, c.o); r.v = la_view(q, c.q); r.o = la_view(dk, c.gk);
    r.x0 = ds_out; r.dk = c.dv; r.dv = c.dk; r.xk = 1; r.xn = c.dv; r.back = 1; r.in = c.scale; r.out = 1.f;
    LaPass& w = a.pass[a.np++];
    w.q = la_view(k, c.k); w.k = la_view(q, c.q); w.v = la_view(d_o, c.o); w.o = la_view(dv, c.gv);
    w.x0 = ds_out; w.x1 = ds0; w.dk = c.dk; w.dv = c.dv; w.xk = c.dv; w.xn = 1; w.back = 1; w.in = c.scale; w.out = 1.f;
    return run_linattn(__func__, c, a, ws, ws_bytes, stream);
}

impala_status_t impala_blocknorm_fwd(const blocknorm_shape_t* shape, const void* h, const float* gamma,
                                     const float* beta, const void* gate, const float* rscale, const void* res,
                                     void* out, const float* gamma2, const float* beta2, void* out2,
                                     hipStream_t stream) {
    impala_status_t st = check_blocknorm(__func__, shape);
    if (st) return st;
    const blocknorm_shape_t& c = *shape;
    if (out2 && c.groups != 1) return fail(IMPALA_EUNSUPPORTED, "%s: a second norm needs groups == 1", __func__);
    if (c.n == 0) return ok();
    CHECK_PTR(h); CHECK_PTR(out);
    const Strided v[] = {bn_rows("h", h, c, c.ld_h, false), bn_rows("gate", gate, c, c.ld_gate, false),
                         bn_rows("res", res, c, c.ld_res, false), bn_rows("out", out, c, c.ld_out, true),
                         bn_rows("out2", out2, c, c.ld_out2, true), bn_cols("gamma", gamma, c, false),
                         bn_cols("beta", beta, c, false), bn_cols("rscale", rscale, c, false),
                         bn_cols("gamma2", gamma2, c, false), bn_cols("beta2", beta2, c, false)};
    if ((st = check_lds(__func__, c, v, 5)) || (st = check_arrays(__func__, v, 5))) return st;
    BnArgs a = bn_args(c);
    a.h = bn_mat(h, c.ld_h); a.gate = bn_mat(gate, c.ld_gate); a.res = bn_mat(res, c.ld_res);
    a.out = bn_mat(out, c.ld_out); a.out2 = bn_mat(out2, c.ld_out2);
    a.gamma = gamma; a.beta = beta; a.rscale = rscale; a.gamma2 = gamma2; a.beta2 = beta2;
    return hip_status(blocknorm_fwd(c.prec, a, stream), __func__);
}

size_t impala_blocknorm_bwd_workspace_bytes(const blocknorm_shape_t* shape) {
    if (check_blocknorm(__func__, shape) != IMPALA_OK) return 0;
    ok();
    return blocknorm_bwd_ws_bytes(shape->prec, shape->n, shape->C, shape->groups, shape->groups == 1);
}

impala_status_t impala_blocknorm_bwd(const blocknorm_shape_t* shape, const void* dout, const void* dout2,
                                     const void* h, const float* gamma, const float* beta, const void* gate,
                                     const float* rscale, const void* out, const float* gamma2, void* dh,
                                     float* dgamma, float* dbeta, void* dgate, float* drscale, void* dres,
                                     float* dgamma2, float* dbeta2, void* ws, size_t ws_bytes,
                                     hipStream_t stream) {
    impala_status_t st = check_blocknorm(__func__, shape);
    if (st) return st;
    const blocknorm_shape_t& c = *shape;
    if (dout2 && c.groups != 1) return fail(IMPALA_EUNSUPPORTED, "%s: a second norm needs groups == 1", __func__);
    if (dgate && !gate) return fail(IMPALA_EINVAL, "%s: dgate without gate", __func__);
    if (c.n > 0) {
        if (!dout2 && (dgamma2 || dbeta2)) return fail(IMPALA_EINVAL, "%s: dgamma2 or dbeta2 without dout2", __func__);
        if (!dout2) CHECK_PTR(dout);
        CHECK_PTR(h); CHECK_PTR(dh); CHECK_PTR(ws);
        if (dout2) CHECK_PTR(out);
    }
    const bool rows = c.n > 0;
    const Strided v[] = {bn_rows("dout", dout, c, c.ld_dout, false), bn_rows("dout2", dout2, c, c.ld_dout2, false),
                         bn_rows("h", h, c, c.ld_h, false), bn_rows("gate", gate, c, c.ld_gate, false),
                         bn_rows("out", dout2 ? out : nullptr, c, c.ld_out, false), bn_rows("dh", dh, c, c.ld_dh, true),
                         bn_rows("dgate", dgate, c, c.ld_dgate, true), bn_rows("dres", dres, c, c.ld_dres, true),
                         bn_cols("gamma", gamma, c, false), bn_cols("beta", beta, c, false),
                         bn_cols("rscale", rscale, c, false), bn_cols("gamma2", gamma2, c, false),
                         bn_cols("dgamma", dgamma, c, true), bn_cols("dbeta", dbeta, c, true),
                         bn_cols("drscale", drscale, c, true), bn_cols("dgamma2", dgamma2, c, true),
                         bn_cols("dbeta2", dbeta2, c, true)};
    if (rows && (st = check_lds(__func__, c, v, 8))) return st;
    if ((st = check_arrays(__func__, v, 8))) return st;
    if (rows) {
        const size_t need = blocknorm_bwd_ws_bytes(c.prec, c.n, c.C, c.groups, dout2 != nullptr);
        if (ws_bytes < need) return fail(IMPALA_EWORKSPACE, "%s: workspace %zu < %zu bytes", __func__, ws_bytes, need);
        if (reinterpret_cast<uintptr_t>(ws) % 16) return fail(IMPALA_EINVAL, "%s: ws must be 16-byte aligned", __func__);
    }
    BnArgs a = bn_args(c);
    a.dout = bn_mat(dout, c.ld_dout); a.dout2 = bn_mat(dout2, c.ld_dout2); a.h = bn_mat(h, c.ld_h);
    a.gate = bn_mat(gate, c.ld_gate); a.out = bn_mat(out, c.ld_out); a.dh = bn_mat(dh, c.ld_dh);
    a.dgate = bn_mat(dgate, c.ld_dgate); a.dres = bn_mat(dres, c.ld_dres);
    a.gamma = gamma; a.beta = beta; a.rscale = rscale; a.gamma2 = gamma2;
    float* grads[5] = {dgamma, dbeta, drscale, dgamma2, dbeta2};
    for (int i = 0; i < 5; ++i) a.grads[i] = grads[i];
    return hip_status(blocknorm_bwd(c.prec, a, ws, stream), __func__);
}

static impala_status_t check_grad_tensors(const char* fn, const grad_tensor_t* t, int32_t n) {
    if (n < 0 || n > 65536) return fail(IMPALA_EINVAL, "%s: between 0 and 65536 tensors", fn);
    if (n > 0) CHECK_PTR(t);
    for (int i = 0; i < n; ++i)
        if (t[i].count < 0 || t[i].count > (int64_t(1) << 40))
            return fail(IMPALA_EINVAL, "%s: tensor %d has a bad count", fn, i);
    return IMPALA_OK;
}

size_t grad_clip_workspace_bytes(const grad_tensor_t* tensors, int32_t n_tensors) {
    if (check_grad_tensors(__func__, tensors, n_tensors) != IMPALA_OK) return 0;
    ok();
    return grad_clip_ws_bytes(tensors, n_tensors);
}

impala_status_t grad_clip(const grad_tensor_t* tensors, int32_t n_tensors, float max_grad_norm, float* stats,
                          void* ws, size_t ws_bytes, hipStream_t stream) try {
    const impala_status_t st = check_grad_tensors(__func__, tensors, n_tensors);
    if (st) return st;
    struct Range { uintptr_t a, b; bool write; };
    std::vector<Range> v;
    v.reserve(2 * size_t(n_tensors));
    for (int i = 0; i < n_tensors; ++i) {
        const grad_tensor_t& t = tensors[i];
        if (t.count == 0) continue;
        if (!valid_prec(t.src_prec) || (t.dst && !valid_prec(t.dst_prec)))
            return fail(IMPALA_EINVAL, "%s: tensor %d has a bad prec", __func__, i);
        if (!t.src) return fail(IMPALA_EINVAL, "%s: tensor %d has no src", __func__, i);
        const int es = t.src_prec == IMPALA_PREC_BF16 ? 2 : 4, ed = t.dst_prec == IMPALA_PREC_BF16 ? 2 : 4;
        const uintptr_t s = reinterpret_cast<uintptr_t>(t.src), d = reinterpret_cast<uintptr_t>(t.dst);
        if (s % es || (d && d % ed)) return fail(IMPALA_EINVAL, "%s: tensor %d is misaligned", __func__, i);
        if (s != d || es != ed) v.push_back({s, s + size_t(t.count) * es, false});
        if (d) v.push_back({d, d + size_t(t.count) * ed, true});
    }
    std::sort(v.begin(), v.end(), [](const Range& x, const Range& y) { return x.a < y.a; });
    uintptr_t read = 0, written = 0;   // the ends of what was read and written so far
    for (const Range& r : v) {
        if (r.a < written || (r.write && r.a < read)) return fail(IMPALA_EINVAL, "%s: a dst overlaps another array", __func__);
        (r.write ? written : read) = std::max(r.write ? written : read, r.b);
    }
    CHECK_PTR(ws);
    const size_t need = grad_clip_ws_bytes(tensors, n_tensors);
    if (ws_bytes < need) return fail(IMPALA_EWORKSPACE, "%s: workspace %zu < %zu bytes", __func__, ws_bytes, need);
    if (reinterpret_cast<uintptr_t>(ws) % 8) return fail(IMPALA_EINVAL, "%s: ws must be 8-byte aligned", __func__);
    return hip_status(grad_clip_run(tensors, n_tensors, max_grad_norm, stats, ws, stream), __func__);
} catch (const std::bad_alloc&) {
    return fail(IMPALA_EINVAL, "grad_clip: out of host memory");
}

}  // extern "C"
