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
// launch, and a third applies them. bf16 elements cost vector instructions before they cost bandwidth
// (57.8 M elements at 60 instructions are 88 us, their traffic 68), so an element's work is folded into
// per-channel constants: z = (x - mu) k + beta, dx = da k + (x - mu) c2 + c3.
//
// Sums of a chunk (at most 65536 elements, up to 8 in a row per thread, then pairwise) are float32; those
// over chunks and frames are 64 bits. The silu's sigmoid takes the hardware's exponential and reciprocal:
// the first is off by |z| 2^-24, which is what z's own rounding leaves of it, the second by 2^-23. In float32
// with silu y is off by 8.9e-8 and dx by 6.8e-8 of their norm (a plain evaluation in float32: 8.2e-8 and
// 7.7e-8), dgamma and dbeta by 1.2e-7 and 1.1e-7, a last place, from the chunks' sums (summed in 64 bits: 7.7e-8
// and 6.7e-8).
//
// Measured, against a copy's 5.1 TB/s: 2048 x 42x42x16 bf16 forward 44 us, 5.3 TB/s; 2048 x 21x21x64 bf16
// backward 102 us, 3.4 TB/s (two tensors in registers leave two workgroups a CU, whose loads, arithmetic and
// stores overlap only with each other's); 2048 x 42x42x32 bf16 forward 117 us, 4.0 TB/s (a workgroup of 1024
// threads fills a CU; held to 64 registers, so that two fit, it spills and is no faster); chunked, 3 x
// 333x517x48 float32 backward 37 + 56 us, 5.3 TB/s of its two passes; 8 x 11x11x32 forward 6.4 us, a launch,
// a trip to memory and two reductions. Stores past the caches take 10 to 25 % off the forward alone and give
// it all back in what reads y next (2048 x 42x42x16 forward and an elementwise reader: 83 against 89 us).
//
// A thread keeps one column of V channels (16 bytes, or one channel where C or an address does not
// allow it) for all its pixels; columns are padded to a power of two per pixel so that the threads of
// a wave that share a column are found by their lane's high bits.
#include "common.h"
#include "groupnorm.h"
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

template <int ACT>
CB_DEV float gn_act(float z, int act_) {
    const int act = ACT < 0 ? act_ : ACT;
    if (act == GN_RELU) return relu_f(z);
    if (act == GN_SILU) return z * gn_sigmoid(z);
    return z;
}

// A channel's constants: d = x - mu, xh = d rstd, z = d k + be with k = rstd gamma. The relu's decision
// z > 0 is x beyond t = mu - be / k on the side that k's sign says: s x > s t with s = +-1. It is taken
// against the largest float32 that is no larger than s t, formed in 64 bits once a channel, so it is
// the decision of the exact z for every x, where z itself in 32 bits would decide by its rounding (one
// element in 10^6); and the sign of s x - T is exact in one fma.
// bf16 activations (CEN = 0) take x for x - mu with mu in the constants: fewer registers and instructions,
// and what cancels, 2^-24 |mu| rstd, is far below the 2^-9 |mu| rstd that their own rounding leaves.
struct GnChannel { float mu, k, p, q; };   // relu: p = s, q = -T; silu: p = be (CEN) or be - mu k
// da = dy act'(z) of V channels, and d (x itself without CEN). ACT < 0: the activation is a.act.
template <class Vec, int V, int ACT, int CEN>
CB_DEV void gn_dact(const GnArgs& a, const typename Vec::Raw& rx, const typename Vec::Raw& rd,
                    const GnChannel (&ch)[V], float (&d)[V], float (&da)[V]) {
    const int act = ACT < 0 ? a.act : ACT;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float x = Vec::get(rx, e);
        d[e] = CEN ? x - ch[e].mu : x;
        da[e] = Vec::get(rd, e);
        if (act == GN_RELU) {
            da[e] = __builtin_fmaf(x, ch[e].p, ch[e].q) > 0.f ? da[e] : 0.f;
        } else if (act == GN_SILU) {
            const float z = __builtin_fmaf(d[e], ch[e].k, ch[e].p), s = gn_sigmoid(z);
            da[e] *= s * (1.f + z * (1.f - s));
        }
    }
}

// The wave's sum over the lanes that share the low bits below `from` (a power of two).
CB_DEV float gn_lanes(float v, int from) {
    for (int m = from; m < 64; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// ... of V values: their exchanges run together.
template <int V>
CB_DEV void gn_lanes_each(float (&v)[V], int from) {
    for (int m = from; m < 64; m <<= 1) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = __shfl_xor(v[e], m);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += o[e];
    }
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
        if (one) val[0] = gn_lanes(val[0], a.cvp);
        else gn_lanes_each<V>(val, a.cvp);
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
    if (a.cvp < 64) gn_lanes_each<V>(val, a.cvp);
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
    int g0, r0;       // group of the column's first channel, and its place in the group
    bool on;
    CB_DEV GnPos(const GnArgs& a, int64_t f, int ck) {
        const int t = threadIdx.x;
        col = t & (a.cvp - 1);
        row = t >> a.cvs;
        rpp = NT >> a.cvs;
        const int first = ck * a.crows;
        rows = min(a.crows, a.HW - first);
        base = (f * a.HW + first) * a.C;
        on = col < a.cv;
        const int c0 = on ? col * (a.C / a.cv) : 0;
        g0 = c0 / a.cg;
        r0 = c0 - g0 * a.cg;
    }
};

// After each vector of a pass: the next one's work does not start early (its registers would add up).
CB_DEV void gn_step() { __builtin_amdgcn_sched_barrier(0); }

// The chunk as a buffer resource: what lies past its end, or in a padding column, reads as zero and is not
// written, without a branch (one around each load would make the wave wait for each).
template <class Raw>
CB_DEV Raw gn_get(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    if constexpr (sizeof(Raw) == 16) return __builtin_bit_cast(Raw, buf_load16(r, off));
    else if constexpr (sizeof(Raw) == 4) return __builtin_bit_cast(Raw, __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
    else return __builtin_bit_cast(Raw, __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0));
}
template <class Raw>
CB_DEV void gn_put(__amdgpu_buffer_rsrc_t r, uint32_t off, Raw v) {
    if constexpr (sizeof(Raw) == 16) buf_store16(r, off, __builtin_bit_cast(uint4, v));
    else if constexpr (sizeof(Raw) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), r, off, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), r, off, 0, 0);
}
template <class P, int NT>
CB_DEV __amdgpu_buffer_rsrc_t gn_rsrc(const void* base, const GnArgs& a, const GnPos<NT>& p) {
    return buf_rsrc(static_cast<const typename P::T*>(base) + p.base, uint32_t(p.rows) * uint32_t(a.C) * sizeof(typename P::T));
}
template <class P, int V, int NV, int NT>
CB_DEV void gn_load(const void* src, const GnArgs& a, const GnPos<NT>& p, typename GnVec<P, V>::Raw (&raw)[NV]) {
    const auto rs = gn_rsrc<P, NT>(src, a, p);
    const uint32_t es = sizeof(typename P::T), step = uint32_t(p.rpp) * uint32_t(a.C) * es;
    const uint32_t off = p.on ? (uint32_t(p.row) * uint32_t(a.C) + uint32_t(p.col * V)) * es : kOOB;
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = gn_get<typename GnVec<P, V>::Raw>(rs, off + uint32_t(j) * step);
}
// f(j) -> the vector to store, for every slot that the chunk has.
template <class P, int V, int NV, int NT, class Fn>
CB_DEV void gn_store(void* dst, const GnArgs& a, const GnPos<NT>& p, Fn&& f) {
    const auto rs = gn_rsrc<P, NT>(dst, a, p);
    const uint32_t es = sizeof(typename P::T), step = uint32_t(p.rpp) * uint32_t(a.C) * es;
    const uint32_t off = p.on ? (uint32_t(p.row) * uint32_t(a.C) + uint32_t(p.col * V)) * es : kOOB;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (j * p.rpp < p.rows) {
            gn_put<typename GnVec<P, V>::Raw>(rs, off + uint32_t(j) * step, f(j));
            gn_step();
        }
}

// Before each pass over the register chunk: the values that follow are formed anew from the raw words, where
// the compiler would keep the floats of the pass before (twice the registers: one workgroup per CU
// instead of two).
template <class Raw, int NV>
CB_DEV void gn_again(Raw (&raw)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if constexpr (sizeof(Raw) == 16) {
            uint4 u = __builtin_bit_cast(uint4, raw[j]);
            asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));
            raw[j] = __builtin_bit_cast(Raw, u);
        }
    }
}

// The thread's V channels of a per-channel vector (NULL: `other`). A column that is on lies inside the
// channels whole.
template <int V, class Pos>
CB_DEV void gn_per_channel(const float* v, const Pos& p, float other, float (&out)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = other;
    if (!v || !p.on) return;
    if constexpr (V == 1) {
        out[0] = v[p.col];
    } else {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 q = load_f4(v + p.col * V + e);
            out[e] = q.x; out[e + 1] = q.y; out[e + 2] = q.z; out[e + 3] = q.w;
        }
    }
}
// ... and of a per-group vector: one group where the groups are whole columns, else counted on from the
// first channel's (a division per channel would be most of the kernel's instructions).
template <int V, class Pos>
CB_DEV void gn_per_group(const float* v, const GnArgs& a, const Pos& p, float (&out)[V]) {
    if (a.cg % V == 0) {
        const float q = v[p.g0];
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = q;
    } else {
        int g = p.g0, r = p.r0;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            out[e] = v[min(g, a.G - 1)];
            if (++r == a.cg) { r = 0; ++g; }
        }
    }
}

template <int V, int ACT, int CEN, class Pos>
CB_DEV void gn_channels(const GnArgs& a, int64_t f, const Pos& p, GnChannel (&ch)[V]) {
    const int act = ACT < 0 ? a.act : ACT;
    float mu[V], rs[V], ga[V], be[V];
    gn_per_group<V>(a.mean + f * a.G, a, p, mu);
    gn_per_group<V>(a.rstd + f * a.G, a, p, rs);
    gn_per_channel<V>(a.gamma, p, 1.f, ga);
    gn_per_channel<V>(a.beta, p, 0.f, be);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        ch[e].mu = mu[e];
        ch[e].k = rs[e] * ga[e];
        ch[e].p = CEN ? be[e] : __builtin_fmaf(-mu[e], ch[e].k, be[e]);
        ch[e].q = 0.f;
        if (act == GN_RELU) {
            const double k = double(rs[e]) * double(ga[e]);
            const double t = k == 0.0 ? (be[e] > 0.f ? -__builtin_inf() : __builtin_inf()) : double(mu[e]) - double(be[e]) / k;
            const double st = k < 0.0 ? -t : t;
            float T = float(st);
            if (double(T) > st) T = T > 0.f ? __uint_as_float(__float_as_uint(T) - 1)
                                    : T < 0.f ? __uint_as_float(__float_as_uint(T) + 1) : -0x1p-149f;
            ch[e].p = k < 0.0 ? -1.f : 1.f;
            ch[e].q = -T;
            gn_step();
        }
    }
}

// Forward statistics of one chunk per workgroup, and (WHOLE: the chunk is the frame) the output.
// Chunks leave their mean and sum of squares about it in ws [n][chunks][2][G].
template <class P, int V, int NV, int NT, int WHOLE, int ACT>
__global__ __launch_bounds__(NT) void gn_fwd_kernel(GnArgs a) {
    using Vec = GnVec<P, V>;
    __shared__ float red[NT * V];
    __shared__ float gmean[kGnMaxC], gm2[kGnMaxC];
    const int64_t f = WHOLE ? blockIdx.x : blockIdx.x / unsigned(a.chunks);
    const int ck = WHOLE ? 0 : int(blockIdx.x % unsigned(a.chunks));
    const GnPos<NT> p(a, f, ck);
    typename Vec::Raw raw[NV];
    gn_load<P, V, NV, NT>(a.x, a, p, raw);
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
    gn_per_group<V>(gmean, a, p, mu);
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = 0.f;
    gn_again(raw);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (p.on && p.row + j * p.rpp < p.rows)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = Vec::get(raw[j], e) - mu[e];
                s[e] = __builtin_fmaf(d, d, s[e]);
            }
        gn_step();
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
        gn_per_group<V>(gm2, a, p, rs);
#pragma unroll
        for (int e = 0; e < V; ++e) rs[e] = 1.f / sqrtf(rs[e] * inv + a.eps);
        for (int g = threadIdx.x; g < a.G; g += NT) {
            if (a.mean) a.mean[f * a.G + g] = gmean[g];
            if (a.rstd) a.rstd[f * a.G + g] = 1.f / sqrtf(gm2[g] * inv + a.eps);
        }
        gn_per_channel<V>(a.gamma, p, 1.f, ga);
        gn_per_channel<V>(a.beta, p, 0.f, be);
#pragma unroll
        for (int e = 0; e < V; ++e) rs[e] *= ga[e];
        gn_again(raw);
        gn_store<P, V, NV, NT>(a.y, a, p, [&](int j) CB_INLINE_LAMBDA {
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e)
                v[e] = gn_act<ACT>(__builtin_fmaf(Vec::get(raw[j], e) - mu[e], rs[e], be[e]), a.act);
            return Vec::put(v);
        });
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

template <class P, int V, int NV, int NT, int ACT>
__global__ __launch_bounds__(NT) void gn_apply_kernel(GnArgs a) {
    using Vec = GnVec<P, V>;
    const int64_t f = blockIdx.x / unsigned(a.chunks);
    const GnPos<NT> p(a, f, int(blockIdx.x % unsigned(a.chunks)));
    typename Vec::Raw raw[NV];
    gn_load<P, V, NV, NT>(a.x, a, p, raw);
    float mu[V], rs[V], ga[V], be[V];
    gn_per_group<V>(a.smean + f * a.G, a, p, mu);
    gn_per_group<V>(a.srstd + f * a.G, a, p, rs);
    gn_per_channel<V>(a.gamma, p, 1.f, ga);
    gn_per_channel<V>(a.beta, p, 0.f, be);
#pragma unroll
    for (int e = 0; e < V; ++e) rs[e] *= ga[e];
    gn_store<P, V, NV, NT>(a.y, a, p, [&](int j) CB_INLINE_LAMBDA {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = gn_act<ACT>(__builtin_fmaf(Vec::get(raw[j], e) - mu[e], rs[e], be[e]), a.act);
        return Vec::put(v);
    });
}

// Backward. STEP 0: the chunk is the frame: sums, then dx. STEP 1: the chunk's per-channel sums of da
// and da xh to part [n][chunks][2][C]. STEP 2: dx of the chunk. The frame's channel sums are in fsum
// [n][2][C] (left there by STEP 0, read by STEP 2); its means of h and h xh are formed from them.
template <class P, int V, int NV, int NT, int STEP, int ACT>
__global__ __launch_bounds__(NT, V == 8 && STEP == 0 ? 4 : 1) void gn_bwd_kernel(GnArgs a) {
    using Vec = GnVec<P, V>;
    constexpr int CEN = sizeof(typename P::T) == 4;
    __shared__ float red[STEP == 2 ? 1 : NT * V];
    __shared__ float sums[2 * kGnMaxC];
    __shared__ float m1s[STEP == 1 ? 1 : kGnMaxC], m2s[STEP == 1 ? 1 : kGnMaxC];
    const int64_t f = STEP == 0 ? blockIdx.x : blockIdx.x / unsigned(a.chunks);
    const int ck = STEP == 0 ? 0 : int(blockIdx.x % unsigned(a.chunks));
    const GnPos<NT> p(a, f, ck);
    typename Vec::Raw rx[NV], rd[NV];
    gn_load<P, V, NV, NT>(a.x, a, p, rx);
    gn_load<P, V, NV, NT>(a.dy, a, p, rd);
    GnChannel ch[V];
    gn_channels<V, ACT, CEN>(a, f, p, ch);
    const int t = threadIdx.x;
    if constexpr (STEP != 2) {
        float sb[V], sg[V];
#pragma unroll
        for (int e = 0; e < V; ++e) sb[e] = sg[e] = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j)   // (slots outside the chunk: dy = 0)
            if (j * p.rpp < p.rows) {
                float d[V], da[V];
                gn_dact<Vec, V, ACT, CEN>(a, rx[j], rd[j], ch, d, da);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    sb[e] += da[e];
                    sg[e] = __builtin_fmaf(da[e], d[e], sg[e]);
                }
                gn_step();
            }
        gn_again(rx);
        gn_again(rd);
        float rs[V];
        gn_per_group<V>(a.rstd + f * a.G, a, p, rs);
        if constexpr (!CEN) {
            float mu[V];
            gn_per_group<V>(a.mean + f * a.G, a, p, mu);
#pragma unroll
            for (int e = 0; e < V; ++e) sg[e] = __builtin_fmaf(-mu[e], sb[e], sg[e]);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) sg[e] *= rs[e];
        gn_channel_sums<V, NT>(a, sb, red, sums);
        gn_channel_sums<V, NT>(a, sg, red, sums + a.C);
        float* o = STEP == 0 ? a.fsum + f * 2 * a.C : a.part + (f * a.chunks + ck) * 2 * a.C;
        for (int c = t; c < 2 * a.C; c += NT) o[c] = sums[c];
    } else {
        for (int c = t; c < 2 * a.C; c += NT) sums[c] = a.fsum[f * 2 * a.C + c];
        __syncthreads();
    }
    if constexpr (STEP == 1) return;
    const float inv = 1.f / (float(a.HW) * float(a.cg));
    for (int g = t >> 6; g < a.G; g += NT / 64) {
        float u = 0.f, v = 0.f;
        for (int c = g * a.cg + (t & 63); c < (g + 1) * a.cg; c += 64) {
            const float gm = a.gamma ? a.gamma[c] : 1.f;
            u += gm * sums[c];
            v += gm * sums[a.C + c];
        }
        u = gn_lanes(u, 1);
        v = gn_lanes(v, 1);
        if ((t & 63) == 0) {
            m1s[g] = u * inv;
            m2s[g] = v * inv;
        }
    }
    __syncthreads();
    // dx = rs (da ga - m1 - xh m2) = da k + d c2 + c3; mu and k are read again rather than kept over the
    // first pass (kept, they spill, and the scratch memory's writes cost more than the loads)
    float c2[V], c3[V], k[V], rs[V];
    gn_per_group<V>(m1s, a, p, c3);
    gn_per_group<V>(m2s, a, p, c2);
    gn_per_group<V>(a.rstd + f * a.G, a, p, rs);
    gn_per_channel<V>(a.gamma, p, 1.f, k);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        c3[e] *= -rs[e];
        c2[e] *= -rs[e] * rs[e];
        k[e] *= rs[e];
    }
    if constexpr (!CEN) {
        float mu[V];
        gn_per_group<V>(a.mean + f * a.G, a, p, mu);
#pragma unroll
        for (int e = 0; e < V; ++e) c3[e] = __builtin_fmaf(-mu[e], c2[e], c3[e]);
    }
    gn_store<P, V, NV, NT>(a.y, a, p, [&](int j) CB_INLINE_LAMBDA {
        float d[V], da[V], v[V];
        gn_dact<Vec, V, ACT, CEN>(a, rx[j], rd[j], ch, d, da);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = __builtin_fmaf(da[e], k[e], __builtin_fmaf(d[e], c2[e], c3[e]));
        return Vec::put(v);
    });
}

// Column sums of x [sets][rows][cols] in a fixed order, in 64 bits: out [sets][cols]; with out2, the
// columns from `half` on go there. A workgroup takes 4 columns in 256 slices of the rows.
__global__ __launch_bounds__(1024) void gn_columns_kernel(const float* __restrict__ x, int64_t rows, int cols, int half,
                                                          float* out, float* out2) {
    __shared__ double sh[1024];
    const int blocks = (cols + 3) / 4, c = int(blockIdx.x % blocks) * 4 + (threadIdx.x & 3), sl = threadIdx.x >> 2;
    const int64_t set = blockIdx.x / blocks;
    double s = 0.0;
    if (c < cols) {
        const float* p = x + set * rows * cols + c;
        int64_t r = sl;
        for (; r + 7 * 256 < rows; r += 8 * 256) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p[(r + 256 * u) * cols];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += v[u];
        }
        for (; r < rows; r += 256) s += p[r * cols];
    }
    sh[threadIdx.x] = s;
    __syncthreads();
    for (int w = 128; w >= 1; w >>= 1) {
        if (sl < w) sh[threadIdx.x] += sh[threadIdx.x + 4 * w];
        __syncthreads();
    }
    if (sl == 0 && c < cols) {
        float* o = c < half ? out : out2;
        if (o) o[set * half + (c < half ? c : c - half)] = float(sh[threadIdx.x]);
    }
}

// Sizes of the register chunks: threads and vectors per thread. The smallest that holds the frame, since a
// whole frame saves a pass over x (and two over x and dy).
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

// ACT < 0 (the activation chosen in the kernel) for one-channel columns
template <class P, int V, int ACT>
void gn_fwd_launch(const GnPlan& p, const GnArgs& a, hipStream_t s) {
    const dim3 grid(unsigned(a.n * a.chunks));
#define GN_W(K, NT, NV) \
    if (p.whole && p.shape == K) hipLaunchKernelGGL((gn_fwd_kernel<P, V, NV, NT, 1, ACT>), grid, dim3(NT), 0, s, a);
    GN_W(0, 256, 2) GN_W(1, 256, 8) GN_W(2, 512, 8) GN_W(3, 1024, 8)
#undef GN_W
    if (p.whole) return;
#define GN_C(K, NT, NV)                                                                             \
    if (p.shape == K) {                                                                             \
        hipLaunchKernelGGL((gn_fwd_kernel<P, V, NV, NT, 0, -1>), grid, dim3(NT), 0, s, a);          \
        hipLaunchKernelGGL(gn_stats_kernel, dim3(unsigned(a.n)), dim3(256), 0, s, a);               \
        hipLaunchKernelGGL((gn_apply_kernel<P, V, NV, NT, ACT>), grid, dim3(NT), 0, s, a);          \
    }
    GN_C(1, 256, 8)
    if constexpr (V == 1) { GN_C(2, 512, 8) GN_C(3, 1024, 8) }
#undef GN_C
}

// Each frame's column sums over its chunks; a launch holds fewer than 2^32 threads.
void gn_frame_sums(const GnArgs& a, hipStream_t s) {
    const int64_t cols = 2 * int64_t(a.C), blocks = (cols + 3) / 4, most = (int64_t(1) << 21) / blocks;
    for (int64_t f = 0; f < a.n; f += most)
        hipLaunchKernelGGL(gn_columns_kernel, dim3(unsigned(std::min(most, a.n - f) * blocks)), dim3(1024), 0, s,
                           a.part + f * a.chunks * cols, int64_t(a.chunks), int(cols), int(cols), a.fsum + f * cols,
                           static_cast<float*>(nullptr));
}

template <class P, int V, int ACT>
void gn_bwd_launch(const GnPlan& p, const GnArgs& a, hipStream_t s) {
    const dim3 grid(unsigned(a.n * a.chunks));
#define GN_W(K, NT, NV) \
    if (p.whole && p.shape == K) hipLaunchKernelGGL((gn_bwd_kernel<P, V, NV, NT, 0, ACT>), grid, dim3(NT), 0, s, a);
    GN_W(0, 256, 2) GN_W(1, 256, 8) GN_W(2, 512, 8) GN_W(3, 1024, 8)
#undef GN_W
    if (p.whole) return;
#define GN_C(K, NT, NV)                                                                                  \
    if (p.shape == K) {                                                                                  \
        hipLaunchKernelGGL((gn_bwd_kernel<P, V, NV, NT, 1, ACT>), grid, dim3(NT), 0, s, a);              \
        gn_frame_sums(a, s);                                                                             \
        hipLaunchKernelGGL((gn_bwd_kernel<P, V, NV, NT, 2, ACT>), grid, dim3(NT), 0, s, a);              \
    }
    GN_C(1, 256, 8)
    if constexpr (V == 1) { GN_C(2, 512, 8) GN_C(3, 1024, 8) }
#undef GN_C
}

template <class P, int V>
void gn_launch(const GnPlan& p, const GnArgs& a, int bwd, hipStream_t s) {
    if constexpr (V == 1) {
        if (bwd) gn_bwd_launch<P, V, -1>(p, a, s);
        else gn_fwd_launch<P, V, -1>(p, a, s);
    } else {
#define GN_A(ACT)                                     \
    if (a.act == ACT) {                               \
        if (bwd) gn_bwd_launch<P, V, ACT>(p, a, s);   \
        else gn_fwd_launch<P, V, ACT>(p, a, s);       \
    }
        GN_A(GN_NONE) GN_A(GN_RELU) GN_A(GN_SILU)
#undef GN_A
    }
}

std::string gn_key(const char* name, int prec, int H, int W, int C) {
    return cb_key(name, prec, cb_dims(H, W) + "x" + std::to_string(C));
}

}  // namespace

int64_t groupnorm_threads(int prec, int64_t n, int H, int W, int C, int G) {
    const GnPlan p = gn_plan(prec, n, H, W, C, G, 0, 0, nullptr);   // one-channel columns: the most chunks
    return n * std::max<int64_t>(256, int64_t(p.chunks) * kGnShapes[p.shape].nt);
}

size_t groupnorm_ws_bytes(int prec, int64_t n, int H, int W, int C, int G, int bwd) {
    const size_t a = gn_plan(prec, n, H, W, C, G, bwd, 0, nullptr).total;   // either column width
    return C % (prec == BF16 ? 8 : 4) ? a : std::max(a, gn_plan(prec, n, H, W, C, G, bwd, 1, nullptr).total);
}

bool groupnorm_fwd_whole(int prec, int64_t n, int H, int W, int C, int G, const void* x, const void* y) {
    return gn_plan(prec, n, H, W, C, G, 0, gn_vec_ok(prec, C, {x, y}), nullptr).whole;
}

hipError_t groupnorm_fwd(int prec, int H, int W, GnArgs a, void* ws, hipStream_t s) {
    const GnPlan p = gn_plan(prec, a.n, H, W, a.C, a.G, 0, gn_vec_ok(prec, a.C, {a.x, a.y}), &a);
    char* w = static_cast<char*>(ws);
    a.part = reinterpret_cast<float*>(w + p.part);
    a.smean = reinterpret_cast<float*>(w + p.smean);
    a.srstd = reinterpret_cast<float*>(w + p.srstd);
    ProfScope ps(s, [&] { return gn_key("groupnorm_fwd", prec, H, W, a.C); });
    if (prec == BF16) {
        if (p.V == 8) gn_launch<PrecBF16, 8>(p, a, 0, s);
        else gn_launch<PrecBF16, 1>(p, a, 0, s);
    } else {
        if (p.V == 4) gn_launch<PrecF32, 4>(p, a, 0, s);
        else gn_launch<PrecF32, 1>(p, a, 0, s);
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
            if (p.V == 8) gn_launch<PrecBF16, 8>(p, a, 1, s);
            else gn_launch<PrecBF16, 1>(p, a, 1, s);
        } else {
            if (p.V == 4) gn_launch<PrecF32, 4>(p, a, 1, s);
            else gn_launch<PrecF32, 1>(p, a, 1, s);
        }
    }
    if (dgamma || dbeta) {
        ProfScope ps(s, [&] { return gn_key("groupnorm_params", prec, H, W, a.C); });
        hipLaunchKernelGGL(gn_columns_kernel, dim3(unsigned((2 * a.C + 3) / 4)), dim3(1024), 0, s, a.fsum, a.n, 2 * a.C,
                           a.C, dbeta, dgamma);
    }
    return hipGetLastError();
}

}  // namespace cb
