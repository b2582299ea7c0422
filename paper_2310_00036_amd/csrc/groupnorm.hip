// Group norm with an activation on channels-last activations, forward and backward.
//
// Per frame and group of C / G channels, over the N = H W C / G elements of the group:
//   mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) rstd,
//   z = xh gamma + beta, y = act(z);
// backward, with da = dy act'(z) and h = gamma da:
//   dbeta = sum da, dgamma = sum da xh, dx = rstd (h - mean(h) - xh mean(h xh)),
// where the group's sums of h and h xh are the gamma-weighted sums of the frame's per-channel sums
// of da and da xh, so the backward reduces per channel only.
//
// Both directions are HBM-bound (forward: x in, y out; backward: x and dy in, dx out). A workgroup
// holds its share of a frame (a chunk of whole pixels, all channels) in registers, so the statistics
// are two-pass (mean, then the squares about it) and x is still read once. A frame that fits one
// workgroup is done in one launch; a larger one is cut into chunks whose statistics are combined
// exactly (sums of squares about the chunks' own means, then about the common one) by a small second
// launch, and a third applies them.
//
// A thread keeps one column of V channels (16 bytes, or one channel where C or an address does not
// allow it) for all its pixels; columns are padded to a power of two per pixel so that the threads of
// a wave that share a column are found by their lane's high bits.
#include "common.h"
#include "kernels.h"

#include <algorithm>

namespace cb {

namespace {

template <class P, int V>
struct GnVec;
template <>
struct GnVec<PrecBF16, 8> {
    using Raw = uint4;
    static CB_DEV float get(const Raw& r, int e) {
        const uint32_t w = e < 2 ? r.x : e < 4 ? r.y : e < 6 ? r.z : r.w;
        return e & 1 ? bf_hi(w) : bf_lo(w);
    }
    static CB_DEV Raw put(const float (&v)[8]) {
        return make_uint4(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7]));
    }
};
template <>
struct GnVec<PrecBF16, 1> {
    using Raw = uint16_t;
    static CB_DEV float get(const Raw& r, int) { return bf2f(r); }
    static CB_DEV Raw put(const float (&v)[1]) { return f2bf(v[0]); }
};
template <>
struct GnVec<PrecF32, 4> {
    using Raw = float4;
    static CB_DEV float get(const Raw& r, int e) { return e == 0 ? r.x : e == 1 ? r.y : e == 2 ? r.z : r.w; }
    static CB_DEV Raw put(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <>
struct GnVec<PrecF32, 1> {
    using Raw = float;
    static CB_DEV float get(const Raw& r, int) { return r; }
    static CB_DEV Raw put(const float (&v)[1]) { return v[0]; }
};

enum { GN_NONE = 0, GN_RELU = 1, GN_SILU = 2 };

CB_DEV float gn_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

CB_DEV float gn_act(float z, int act) {
    if (act == GN_RELU) return relu_f(z);
    if (act == GN_SILU) return z * gn_sigmoid(z);
    return z;
}

// dy act'(z). The relu's decision next to its border is taken in 64 bits: with |z| within rounding
// of zero, 32 bits would decide by the order of their roundings (one element in 10^6 or so).
CB_DEV float gn_dact(float dy, float x, float mu, float rs, float ga, float be, float xh, int act) {
    if (act == GN_NONE) return dy;
    const float t = xh * ga, z = t + be;
    if (act == GN_RELU) {
        bool pos = z > 0.f;
        if (fabsf(z) <= 0x1p-20f * (fabsf(t) + fabsf(be)))
            pos = (double(x) - double(mu)) * double(rs) * double(ga) + double(be) > 0.0;
        return pos ? dy : 0.f;
    }
    const float s = gn_sigmoid(z);
    return dy * (s * (1.f + z * (1.f - s)));
}

// The wave's sum over the lanes that share the low bits below `from` (a power of two).
CB_DEV float gn_lanes(float v, int from) {
    for (int m = from; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// Sums of per-thread column values over the workgroup, by group: val[0..V) are this thread's channels
// (one value where `one`: the column lies in one group). The result for group g is left in out[g]
// times `scale`. red: NT * V floats. Ends with a barrier.
template <int V, int NT>
CB_DEV void gn_group_sums(const GnArgs& a, float (&val)[V], float scale, float* red, float* out) {
    const int t = threadIdx.x, lane = t & 63, col = t & (a.cvp - 1);
    const bool one = a.cg % V == 0;
    const int w = one ? a.cvp : a.cvp * V;
    if (one) {
#pragma unroll
        for (int e = 1; e < V; ++e) val[0] += val[e];
    }
    if (a.cvp < 64) {
        val[0] = gn_lanes(val[0], a.cvp);
        if (!one)
#pragma unroll
            for (int e = 1; e < V; ++e) val[e] = gn_lanes(val[e], a.cvp);
    }
    const int per = a.cvp < 64 ? 64 : a.cvp, row = t / per, R = NT / per;
    if (a.cvp >= 64 || lane < a.cvp) {
        if (one) red[row * w + col] = val[0];
        else
#pragma unroll
            for (int e = 0; e < V; ++e) red[row * w + col * V + e] = val[e];
    }
    __syncthreads();
    const int eg = one ? a.cg / V : a.cg;
    for (int g = t >> 6; g < a.G; g += NT / 64) {
        float s = 0.f;
        for (int i = lane; i < R * eg; i += 64) {
            const int r = i / eg;
            s += red[r * w + g * eg + (i - r * eg)];
        }
        s = gn_lanes(s, 1);
        if (lane == 0) out[g] = s * scale;
    }
    __syncthreads();
}

// Per-channel sums over the workgroup: out[c] for every channel. Ends with a barrier.
template <int V, int NT>
CB_DEV void gn_channel_sums(const GnArgs& a, float (&val)[V], float* red, float* out) {
    const int t = threadIdx.x, lane = t & 63, col = t & (a.cvp - 1);
    const int w = a.cvp * V;
    if (a.cvp < 64) {
#pragma unroll
        for (int e = 0; e < V; ++e) val[e] = gn_lanes(val[e], a.cvp);
    }
    const int per = a.cvp < 64 ? 64 : a.cvp, row = t / per, R = NT / per;
    if (a.cvp >= 64 || lane < a.cvp)
#pragma unroll
        for (int e = 0; e < V; ++e) red[row * w + col * V + e] = val[e];
    __syncthreads();
    for (int c = t; c < a.C; c += NT) {
        float s = 0.f;
        for (int r = 0; r < R; ++r) s += red[r * w + c];
        out[c] = s;
    }
    __syncthreads();
}

// This thread's pixels of chunk `ck` of frame `f`: rows row + j * rpp < rows.
template <int NT>
struct GnPos {
    int64_t base;     // first element of the chunk
    int rows, row, rpp, col;
    bool on;
    CB_DEV GnPos(const GnArgs& a, int64_t f, int ck) {
        const int t = threadIdx.x;
        col = t & (a.cvp - 1);
        row = t >> a.cvs;
        rpp = NT >> a.cvs;
        const int r0 = ck * a.crows;
        rows = min(a.crows, a.HW - r0);
        base = (f * a.HW + r0) * a.C;
        on = col < a.cv;
    }
};

template <class P, int V, int NV, int NT>
CB_DEV void gn_load(const void* src, const GnArgs& a, const GnPos<NT>& p, typename GnVec<P, V>::Raw (&raw)[NV]) {
    using Raw = typename GnVec<P, V>::Raw;
    const typename P::T* x = static_cast<const typename P::T*>(src) + p.base + p.col * V;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int r = p.row + j * p.rpp;
        raw[j] = Raw{};
        if (p.on && r < p.rows) raw[j] = *reinterpret_cast<const Raw*>(x + int64_t(r) * a.C);
    }
}

// The thread's V channels of a per-channel or (by group) per-group vector.
template <int V>
CB_DEV void gn_per_channel(const float* v, int c0, int C, float other, float (&out)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = v && c0 + e < C ? v[c0 + e] : other;
}
template <int V>
CB_DEV void gn_per_group(const float* v, int c0, int C, int cg, float (&out)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = c0 + e < C ? v[(c0 + e) / cg] : 0.f;
}

// Forward statistics of one chunk per workgroup, and (WHOLE: the chunk is the frame) the output.
// Chunks leave their mean and sum of squares about it in ws [n][chunks][2][G].
template <class P, int V, int NV, int NT, int WHOLE>
__global__ __launch_bounds__(NT) void gn_fwd_kernel(GnArgs a) {
    using Vec = GnVec<P, V>;
    __shared__ float red[NT * V];
    __shared__ float gmean[kGnMaxC], gm2[kGnMaxC];
    const int64_t f = WHOLE ? blockIdx.x : blockIdx.x / unsigned(a.chunks);
    const int ck = WHOLE ? 0 : int(blockIdx.x % unsigned(a.chunks));
    const GnPos<NT> p(a, f, ck);
    typename Vec::Raw raw[NV];
    gn_load<P, V, NV, NT>(a.x, a, p, raw);
    const int c0 = p.col * V;
    const float inv = 1.f / (float(p.rows) * float(a.cg));
    float s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)   // slots outside the chunk hold zeros
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] += Vec::get(raw[j], e);
    gn_group_sums<V, NT>(a, s, inv, red, gmean);
    float mu[V];
    gn_per_group<V>(gmean, c0, a.C, a.cg, mu);
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (p.on && p.row + j * p.rpp < p.rows)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = Vec::get(raw[j], e) - mu[e];
                s[e] += d * d;
            }
    gn_group_sums<V, NT>(a, s, 1.f, red, gm2);
    if constexpr (!WHOLE) {
        float* o = a.part + (f * a.chunks + ck) * 2 * a.G;
        for (int g = threadIdx.x; g < a.G; g += NT) {
            o[g] = gmean[g];
            o[a.G + g] = gm2[g];
        }
    } else {
        float ga[V], be[V], rs[V];
        gn_per_group<V>(gm2, c0, a.C, a.cg, rs);
#pragma unroll
        for (int e = 0; e < V; ++e) rs[e] = 1.f / sqrtf(rs[e] * inv + a.eps);
        for (int g = threadIdx.x; g < a.G; g += NT) {
            if (a.mean) a.mean[f * a.G + g] = gmean[g];
            if (a.rstd) a.rstd[f * a.G + g] = 1.f / sqrtf(gm2[g] * inv + a.eps);
        }
        gn_per_channel<V>(a.gamma, c0, a.C, 1.f, ga);
        gn_per_channel<V>(a.beta, c0, a.C, 0.f, be);
        typename P::T* y = static_cast<typename P::T*>(a.y) + p.base + c0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int r = p.row + j * p.rpp;
            if (!(p.on && r < p.rows)) continue;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[e] = gn_act((Vec::get(raw[j], e) - mu[e]) * rs[e] * ga[e] + be[e], a.act);
            *reinterpret_cast<typename Vec::Raw*>(y + int64_t(r) * a.C) = Vec::put(v);
        }
    }
}

// A frame's statistics from its chunks', one workgroup per frame, a wave per group in turn.
__global__ __launch_bounds__(256) void gn_stats_kernel(GnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t f = blockIdx.x;
    const float* part = a.part + f * a.chunks * 2 * a.G;
    for (int g = threadIdx.x >> 6; g < a.G; g += 4) {
        double s = 0.0;
        for (int k = lane; k < a.chunks; k += 64)
            s += double(part[int64_t(k) * 2 * a.G + g]) * min(a.crows, a.HW - k * a.crows);
        for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
        const double mean = s / a.HW;
        double q = 0.0;
        for (int k = lane; k < a.chunks; k += 64) {
            const float* o = part + int64_t(k) * 2 * a.G;
            const double d = double(o[g]) - mean;
            q += double(o[a.G + g]) + d * d * (double(min(a.crows, a.HW - k * a.crows)) * a.cg);
        }
        for (int m = 1; m < 64; m <<= 1) q += __shfl_xor(q, m);
        if (lane == 0) {
            const float mf = float(mean), rf = float(1.0 / sqrt(q / (double(a.HW) * a.cg) + double(a.eps)));
            a.smean[f * a.G + g] = mf;
            a.srstd[f * a.G + g] = rf;
            if (a.mean) a.mean[f * a.G + g] = mf;
            if (a.rstd) a.rstd[f * a.G + g] = rf;
        }
    }
}

template <class P, int V, int NV, int NT>
__global__ __launch_bounds__(NT) void gn_apply_kernel(GnArgs a) {
    using Vec = GnVec<P, V>;
    const int64_t f = blockIdx.x / unsigned(a.chunks);
    const GnPos<NT> p(a, f, int(blockIdx.x % unsigned(a.chunks)));
    typename Vec::Raw raw[NV];
    gn_load<P, V, NV, NT>(a.x, a, p, raw);
    const int c0 = p.col * V;
    float mu[V], rs[V], ga[V], be[V];
    gn_per_group<V>(a.smean + f * a.G, c0, a.C, a.cg, mu);
    gn_per_group<V>(a.srstd + f * a.G, c0, a.C, a.cg, rs);
    gn_per_channel<V>(a.gamma, c0, a.C, 1.f, ga);
    gn_per_channel<V>(a.beta, c0, a.C, 0.f, be);
    typename P::T* y = static_cast<typename P::T*>(a.y) + p.base + c0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int r = p.row + j * p.rpp;
        if (!(p.on && r < p.rows)) continue;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = gn_act((Vec::get(raw[j], e) - mu[e]) * rs[e] * ga[e] + be[e], a.act);
        *reinterpret_cast<typename Vec::Raw*>(y + int64_t(r) * a.C) = Vec::put(v);
    }
}

// Backward. STEP 0: the chunk is the frame: sums, then dx. STEP 1: the chunk's per-channel sums of da
// and da xh to part [n][chunks][2][C]. STEP 2: dx of the chunk from the frame's means of h and h xh.
// STEP 0 leaves the frame's channel sums in fsum [n][2][C].
template <class P, int V, int NV, int NT, int STEP>
__global__ __launch_bounds__(NT) void gn_bwd_kernel(GnArgs a) {
    using Vec = GnVec<P, V>;
    __shared__ float red[STEP == 2 ? 1 : NT * V];
    __shared__ float cb_[STEP == 2 ? 1 : kGnMaxC], cg_[STEP == 2 ? 1 : kGnMaxC];
    __shared__ float m1s[STEP == 0 ? kGnMaxC : 1], m2s[STEP == 0 ? kGnMaxC : 1];
    const int64_t f = STEP == 0 ? blockIdx.x : blockIdx.x / unsigned(a.chunks);
    const int ck = STEP == 0 ? 0 : int(blockIdx.x % unsigned(a.chunks));
    const GnPos<NT> p(a, f, ck);
    typename Vec::Raw rx[NV], rd[NV];
    gn_load<P, V, NV, NT>(a.x, a, p, rx);
    gn_load<P, V, NV, NT>(a.dy, a, p, rd);
    const int c0 = p.col * V;
    float mu[V], rs[V], ga[V], be[V];
    gn_per_group<V>(a.mean + f * a.G, c0, a.C, a.cg, mu);
    gn_per_group<V>(a.rstd + f * a.G, c0, a.C, a.cg, rs);
    gn_per_channel<V>(a.gamma, c0, a.C, 1.f, ga);
    gn_per_channel<V>(a.beta, c0, a.C, 0.f, be);
    const int t = threadIdx.x;
    if constexpr (STEP != 2) {
        float sb[V], sg[V];
#pragma unroll
        for (int e = 0; e < V; ++e) sb[e] = sg[e] = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (p.on && p.row + j * p.rpp < p.rows)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float x = Vec::get(rx[j], e), xh = (x - mu[e]) * rs[e];
                    const float da = gn_dact(Vec::get(rd[j], e), x, mu[e], rs[e], ga[e], be[e], xh, a.act);
                    sb[e] += da;
                    sg[e] += da * xh;
                }
        gn_channel_sums<V, NT>(a, sb, red, cb_);
        gn_channel_sums<V, NT>(a, sg, red, cg_);
        float* o = STEP == 0 ? a.fsum + f * 2 * a.C : a.part + (f * a.chunks + ck) * 2 * a.C;
        for (int c = t; c < a.C; c += NT) {
            o[c] = cb_[c];
            o[a.C + c] = cg_[c];
        }
    }
    if constexpr (STEP == 1) return;
    float m1[V], m2[V];
    if constexpr (STEP == 0) {
        const float inv = 1.f / (float(a.HW) * float(a.cg));
        for (int g = t >> 6; g < a.G; g += NT / 64) {
            float u = 0.f, v = 0.f;
            for (int c = g * a.cg + (t & 63); c < (g + 1) * a.cg; c += 64) {
                const float gm = a.gamma ? a.gamma[c] : 1.f;
                u += gm * cb_[c];
                v += gm * cg_[c];
            }
            u = gn_lanes(u, 1);
            v = gn_lanes(v, 1);
            if ((t & 63) == 0) {
                m1s[g] = u * inv;
                m2s[g] = v * inv;
            }
        }
        __syncthreads();
        gn_per_group<V>(m1s, c0, a.C, a.cg, m1);
        gn_per_group<V>(m2s, c0, a.C, a.cg, m2);
    } else {
        gn_per_group<V>(a.smean + f * a.G, c0, a.C, a.cg, m1);
        gn_per_group<V>(a.srstd + f * a.G, c0, a.C, a.cg, m2);
    }
    typename P::T* dx = static_cast<typename P::T*>(a.y) + p.base + c0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int r = p.row + j * p.rpp;
        if (!(p.on && r < p.rows)) continue;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float x = Vec::get(rx[j], e), xh = (x - mu[e]) * rs[e];
            const float da = gn_dact(Vec::get(rd[j], e), x, mu[e], rs[e], ga[e], be[e], xh, a.act);
            v[e] = rs[e] * (da * ga[e] - m1[e] - xh * m2[e]);
        }
        *reinterpret_cast<typename Vec::Raw*>(dx + int64_t(r) * a.C) = Vec::put(v);
    }
}

// A frame's channel sums from its chunks' (fsum [n][2][C]), and its means of h and h xh (smean, srstd
// [n][G]): one workgroup per frame.
__global__ __launch_bounds__(256) void gn_bwd_means_kernel(GnArgs a) {
    __shared__ float ch[2 * kGnMaxC];
    const int64_t f = blockIdx.x;
    const float* part = a.part + f * a.chunks * 2 * a.C;
    for (int c = threadIdx.x; c < 2 * a.C; c += 256) {
        double s = 0.0;
        for (int k = 0; k < a.chunks; ++k) s += part[int64_t(k) * 2 * a.C + c];
        ch[c] = float(s);
        a.fsum[f * 2 * a.C + c] = float(s);
    }
    __syncthreads();
    const double inv = 1.0 / (double(a.HW) * a.cg);
    for (int g = threadIdx.x; g < a.G; g += 256) {
        double u = 0.0, v = 0.0;
        for (int c = g * a.cg; c < (g + 1) * a.cg; ++c) {
            const double gm = a.gamma ? a.gamma[c] : 1.f;
            u += gm * ch[c];
            v += gm * ch[a.C + c];
        }
        a.smean[f * a.G + g] = float(u * inv);
        a.srstd[f * a.G + g] = float(v * inv);
    }
}

// dbeta and dgamma: the frames' channel sums added in a fixed order, in 64 bits. A workgroup takes 4
// columns in 64 slices of the frames.
__global__ __launch_bounds__(256) void gn_params_kernel(GnArgs a, float* dgamma, float* dbeta) {
    __shared__ double sh[256];
    const int c = blockIdx.x * 4 + (threadIdx.x & 3), sl = threadIdx.x >> 2;
    double s = 0.0;
    if (c < 2 * a.C)
        for (int64_t f = sl; f < a.n; f += 64) s += a.fsum[f * 2 * a.C + c];
    sh[threadIdx.x] = s;
    __syncthreads();
    for (int w = 32; w >= 1; w >>= 1) {
        if (sl < w) sh[threadIdx.x] += sh[threadIdx.x + 4 * w];
        __syncthreads();
    }
    if (sl == 0 && c < 2 * a.C) {
        float* o = c < a.C ? dbeta : dgamma;
        if (o) o[c < a.C ? c : c - a.C] = float(sh[threadIdx.x]);
    }
}

// Sizes of the register chunks: threads and vectors per thread. The smallest that holds the frame.
struct GnShape { int nt, nv; };
constexpr GnShape kGnShapes[] = {{256, 2}, {256, 8}, {512, 8}, {1024, 8}};
constexpr int kGnNumShapes = 4;
constexpr int kGnSplit = 1;   // the shape of the chunks of a frame that none of them holds

struct GnPlan {
    int shape, V, whole, chunks;
    size_t part, fsum, smean, srstd, total;   // byte offsets
};

size_t gn_align(size_t b) { return (b + 255) / 256 * 256; }

// v16: 16-byte columns are allowed (C and every address).
GnPlan gn_plan(int prec, int64_t n, int H, int W, int C, int G, int bwd, int v16, GnArgs* a) {
    GnPlan p{};
    const int V = v16 ? (prec == BF16 ? 8 : 4) : 1;
    const int64_t HW = int64_t(H) * W;
    const int cv = C / V;
    int cvp = 1, cvs = 0;
    while (cvp < cv) cvp *= 2, ++cvs;
    p.V = V;
    p.whole = 0;
    p.shape = kGnSplit;
    for (int k = 0; k < kGnNumShapes; ++k) {
        if (kGnShapes[k].nt < cvp) continue;
        if (HW <= int64_t(kGnShapes[k].nt / cvp) * kGnShapes[k].nv) {
            p.shape = k;
            p.whole = 1;
            break;
        }
    }
    while (kGnShapes[p.shape].nt < cvp) ++p.shape;
    const int crows = p.whole ? int(HW) : kGnShapes[p.shape].nt / cvp * kGnShapes[p.shape].nv;
    p.chunks = int((HW + crows - 1) / crows);
    size_t off = 0;
    auto take = [&](size_t floats) { const size_t o = off; off += gn_align(floats * sizeof(float)); return o; };
    p.part = take(p.whole ? 0 : size_t(n) * p.chunks * 2 * (bwd ? C : G));
    p.fsum = take(bwd ? size_t(n) * 2 * C : 0);
    p.smean = take(p.whole ? 0 : size_t(n) * G);
    p.srstd = take(p.whole ? 0 : size_t(n) * G);
    p.total = off;
    if (a) {
        a->n = n; a->HW = int(HW); a->C = C; a->G = G; a->cg = C / G;
        a->cv = cv; a->cvp = cvp; a->cvs = cvs; a->crows = crows; a->chunks = p.chunks;
    }
    return p;
}

bool gn_vec_ok(int prec, int C, std::initializer_list<const void*> ptrs) {
    if (C % (prec == BF16 ? 8 : 4)) return false;
    for (const void* q : ptrs)
        if (reinterpret_cast<uintptr_t>(q) & 15) return false;
    return true;
}

template <class P, int V>
void gn_fwd_launch(const GnPlan& p, const GnArgs& a, hipStream_t s) {
    const dim3 grid(unsigned(a.n * a.chunks));
#define GN_W(K, NT, NV) \
    if (p.whole && p.shape == K) hipLaunchKernelGGL((gn_fwd_kernel<P, V, NV, NT, 1>), grid, dim3(NT), 0, s, a);
    GN_W(0, 256, 2) GN_W(1, 256, 8) GN_W(2, 512, 8) GN_W(3, 1024, 8)
#undef GN_W
    if (p.whole) return;
#define GN_C(K, NT, NV)                                                                             \
    if (p.shape == K) {                                                                             \
        hipLaunchKernelGGL((gn_fwd_kernel<P, V, NV, NT, 0>), grid, dim3(NT), 0, s, a);              \
        hipLaunchKernelGGL(gn_stats_kernel, dim3(unsigned(a.n)), dim3(256), 0, s, a);               \
        hipLaunchKernelGGL((gn_apply_kernel<P, V, NV, NT>), grid, dim3(NT), 0, s, a);               \
    }
    GN_C(1, 256, 8)
    if constexpr (V == 1) { GN_C(2, 512, 8) GN_C(3, 1024, 8) }
#undef GN_C
}

template <class P, int V>
void gn_bwd_launch(const GnPlan& p, const GnArgs& a, hipStream_t s) {
    const dim3 grid(unsigned(a.n * a.chunks));
#define GN_W(K, NT, NV) \
    if (p.whole && p.shape == K) hipLaunchKernelGGL((gn_bwd_kernel<P, V, NV, NT, 0>), grid, dim3(NT), 0, s, a);
    GN_W(0, 256, 2) GN_W(1, 256, 8) GN_W(2, 512, 8) GN_W(3, 1024, 8)
#undef GN_W
    if (p.whole) return;
#define GN_C(K, NT, NV)                                                                             \
    if (p.shape == K) {                                                                             \
        hipLaunchKernelGGL((gn_bwd_kernel<P, V, NV, NT, 1>), grid, dim3(NT), 0, s, a);              \
        hipLaunchKernelGGL(gn_bwd_means_kernel, dim3(unsigned(a.n)), dim3(256), 0, s, a);           \
        hipLaunchKernelGGL((gn_bwd_kernel<P, V, NV, NT, 2>), grid, dim3(NT), 0, s, a);              \
    }
    GN_C(1, 256, 8)
    if constexpr (V == 1) { GN_C(2, 512, 8) GN_C(3, 1024, 8) }
#undef GN_C
}

std::string gn_key(const char* name, int prec, int H, int W, int C) {
    return cb_key(name, prec, cb_dims(H, W) + "x" + std::to_string(C));
}

}  // namespace

int64_t groupnorm_blocks(int prec, int64_t n, int H, int W, int C, int G) {
    return n * gn_plan(prec, n, H, W, C, G, 0, 0, nullptr).chunks;   // one-channel columns: the most chunks
}

size_t groupnorm_ws_bytes(int prec, int64_t n, int H, int W, int C, int G, int bwd) {
    const size_t a = gn_plan(prec, n, H, W, C, G, bwd, 0, nullptr).total;   // either column width
    return C % (prec == BF16 ? 8 : 4) ? a : std::max(a, gn_plan(prec, n, H, W, C, G, bwd, 1, nullptr).total);
}

hipError_t groupnorm_fwd(int prec, int H, int W, GnArgs a, void* ws, hipStream_t s) {
    const GnPlan p = gn_plan(prec, a.n, H, W, a.C, a.G, 0, gn_vec_ok(prec, a.C, {a.x, a.y}), &a);
    char* w = static_cast<char*>(ws);
    a.part = reinterpret_cast<float*>(w + p.part);
    a.smean = reinterpret_cast<float*>(w + p.smean);
    a.srstd = reinterpret_cast<float*>(w + p.srstd);
    ProfScope ps(s, [&] { return gn_key("groupnorm_fwd", prec, H, W, a.C); });
    if (prec == BF16) {
        if (p.V == 8) gn_fwd_launch<PrecBF16, 8>(p, a, s);
        else gn_fwd_launch<PrecBF16, 1>(p, a, s);
    } else {
        if (p.V == 4) gn_fwd_launch<PrecF32, 4>(p, a, s);
        else gn_fwd_launch<PrecF32, 1>(p, a, s);
    }
    return hipGetLastError();
}

hipError_t groupnorm_bwd(int prec, int H, int W, GnArgs a, float* dgamma, float* dbeta, void* ws, hipStream_t s) {
    const GnPlan p = gn_plan(prec, a.n, H, W, a.C, a.G, 1, gn_vec_ok(prec, a.C, {a.x, a.dy, a.y}), &a);
    char* w = static_cast<char*>(ws);
    a.part = reinterpret_cast<float*>(w + p.part);
    a.fsum = reinterpret_cast<float*>(w + p.fsum);
    a.smean = reinterpret_cast<float*>(w + p.smean);
    a.srstd = reinterpret_cast<float*>(w + p.srstd);
    if (a.n > 0) {
        ProfScope ps(s, [&] { return gn_key("groupnorm_bwd", prec, H, W, a.C); });
        if (prec == BF16) {
            if (p.V == 8) gn_bwd_launch<PrecBF16, 8>(p, a, s);
            else gn_bwd_launch<PrecBF16, 1>(p, a, s);
        } else {
            if (p.V == 4) gn_bwd_launch<PrecF32, 4>(p, a, s);
            else gn_bwd_launch<PrecF32, 1>(p, a, s);
        }
    }
    if (dgamma || dbeta) {
        ProfScope ps(s, [&] { return gn_key("groupnorm_params", prec, H, W, a.C); });
        hipLaunchKernelGGL(gn_params_kernel, dim3(unsigned((2 * a.C + 3) / 4)), dim3(256), 0, s, a, dgamma, dbeta);
    }
    return hipGetLastError();
}

}  // namespace cb
