// C entry points of the memory core's operators (linear attention, block norms): argument validation on the host.
#include <algorithm>
#include <cmath>

#include "../../include/cleanba_layers.h"
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
    for (int i = 0; i < 3; ++i)
        if (a.n[i] != b.n[i] || a.s[i] != b.s[i]) return true;
    Strided wide = a;
    wide.w = std::max(a.w, b.w);
    const int64_t d = reinterpret_cast<intptr_t>(b.p) - reinterpret_cast<intptr_t>(a.p);
    if (!wide.nested() || d % a.es) return true;
    int ax[3];
    a.order(ax);
    return rows_meet(a, b, ax, 0, d / a.es);
}

// Strides and aliases of a call's arrays; an error text, or "".
template <size_t N>
impala_status_t check_arrays(const char* fn, const Strided (&v)[N]) {
    for (const Strided& x : v) {
        if (!x.p) continue;
        for (int i = 0; i < 3; ++i)
            if (x.s[i] < 0) return fail(IMPALA_EINVAL, "%s: %s has a negative stride", fn, x.name);
        if (!(x.reach() < std::ldexp(1.0, 60))) return fail(IMPALA_EINVAL, "%s: %s reaches too far", fn, x.name);
        if (reinterpret_cast<uintptr_t>(x.p) % x.es) return fail(IMPALA_EINVAL, "%s: %s is misaligned", fn, x.name);
        if (x.written && !x.empty() && !x.nested())
            return fail(IMPALA_EINVAL, "%s: %s has elements in one place", fn, x.name);
    }
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < i; ++j)
            if ((v[i].written || v[j].written) && !v[i].empty() && !v[j].empty() && arrays_meet(v[i], v[j]))
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
    if (int64_t(c->E) * c->heads > (int64_t(1) << 21))
        return fail(IMPALA_EUNSUPPORTED, "%s: at most 2^21 states in a call", fn);
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

}  // extern "C"
