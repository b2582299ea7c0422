// A block's norm, gate, scale and residual sum, with the next block's norm of that sum, forward and backward, in one pass
// over the rows. HBM-bound: each array is read or written once, a row is held in registers from its statistics to its
// stores. A row (or a group of its channels) is taken by tpr neighbouring threads, V elements each, so that one row's sums
// are shuffles inside a wave up to 1024 channels.
#include <algorithm>
#include <type_traits>

#include "blocknorm.h"
#include "common.h"
#include "kernels.h"
#include "plan.h"

namespace cb {

namespace {

// 16 bytes at any alignment of an element: global memory takes them so.
typedef uint32_t bn_u32x4 __attribute__((ext_vector_type(4), aligned(2)));

template <class T>
struct BnVec {
    static constexpr int N = 16 / sizeof(T);
    static CB_DEV uint4 raw(const T* p, int left) {   // zeros behind `left` elements
        if (left >= N) {
            const bn_u32x4 v = *reinterpret_cast<const bn_u32x4*>(p);
            return make_uint4(v[0], v[1], v[2], v[3]);
        }
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) {
                if constexpr (sizeof(T) == 2) w[i / 2] |= uint32_t(p[i]) << (16 * (i & 1));
                else w[i] = __float_as_uint(p[i]);
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static CB_DEV void unpack(uint4 v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2) { x[2 * i] = bf_lo(w[i]); x[2 * i + 1] = bf_hi(w[i]); }
            else x[i] = __uint_as_float(w[i]);
        }
    }
    static CB_DEV void store(T* p, int left, const float* x) {
        if (left >= N) {
            bn_u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) v[i] = pack2bf(x[2 * i], x[2 * i + 1]);
                else v[i] = __float_as_uint(x[i]);
            }
            *reinterpret_cast<bn_u32x4*>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) {
                    if constexpr (sizeof(T) == 2) p[i] = f2bf(x[i]);
                    else p[i] = x[i];
                }
        }
    }
    static CB_DEV float round(float x) {
        if constexpr (sizeof(T) == 2) return bf2f(f2bf(x));
        else return x;
    }
};

// A thread's place: row slot and group of its workgroup, columns t N, t N + tpr N, ... of the group.
struct BnPlace {
    int slot, t, grp, width;   // width: channels of the group
    int64_t row, step;
    bool on;
    CB_DEV BnPlace(const BnArgs& a) {
        const int s = int(threadIdx.x) / a.tpr;
        t = int(threadIdx.x) - s * a.tpr;
        slot = s / a.gb;
        grp = blockIdx.y * a.gb + s % a.gb;
        on = slot < a.rb && grp < a.G;
        width = on ? a.cg : 0;
        row = int64_t(blockIdx.x) * a.rb + slot;
        step = int64_t(gridDim.x) * a.rb;
    }
};

// x plus that of the lane that `ctrl` names, by a data-parallel-primitive move.
template <int CTRL>
CB_DEV float dpp_add(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
typedef unsigned bn_u32x2 __attribute__((ext_vector_type(2)));

// Sums of K numbers over the tpr threads of a row, in every one of them, in a fixed order: neighbours, quads (mirrored
// halves once four lanes agree), rows of 16, of 32, the wave; then the row's waves through LDS, whose two halves the
// calls take in turn (`flip`), so that one barrier a call is enough.
template <int K>
CB_DEV void row_sum(float (&v)[K], int tpr, float* sh, int& flip) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (tpr >= 2) v[k] = dpp_add<0xB1>(v[k]);
        if (tpr >= 4) v[k] = dpp_add<0x4E>(v[k]);
        if (tpr >= 8) v[k] = dpp_add<0x141>(v[k]);
        if (tpr >= 16) v[k] = dpp_add<0x140>(v[k]);
        if (tpr >= 32) {
            const unsigned u = __float_as_uint(v[k]);
            const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            v[k] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
        if (tpr >= 64) {
            const unsigned u = __float_as_uint(v[k]);
            const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            v[k] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
    }
    if (tpr > 64) {
        const int wave = threadIdx.x >> 6, w = tpr >> 6, first = wave / w * w;
        float* h = sh + flip * 16 * 4;
        flip ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) h[wave * K + k] = v[k];
        lds_barrier();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = h[first * K + k];
            for (int i = 1; i < w; ++i) v[k] += h[(first + i) * K + k];
        }
    }
}

// 1 / (1 + exp(-x)) from the hardware's 2^t and reciprocal: the product's rounding error and log2(e)'s own are made good
// on the power, one Newton step on the reciprocal, so that it is off by about an ulp in a third of the instructions of
// expf and a division (65536 x 1024 bf16 backward, which they bound beside HBM). Beyond +-88 it is 0 or 1 to 32 bits;
// selections keep NaN.
CB_DEV float bn_sigmoid(float x) {
    constexpr float kL2E = 1.44269504f, kL2ELo = 1.92596300e-8f, kLn2 = 0.69314718f;
    float a = x < -88.f ? 88.f : -x;
    a = x > 88.f ? -88.f : a;
    const float t = a * kL2E, lo = fmaf(a, kL2ELo, fmaf(a, kL2E, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, lo * kLn2, e);
    const float d = 1.f + e, r = __builtin_amdgcn_rcpf(d);
    return fmaf(fmaf(-d, r, 1.f), r, r);
}

// 1 / sqrt(v), v >= 0, with one Newton step (none from 0 or infinity, where it would make NaN). The instruction takes
// denormal numbers, which are squares of rows about 1e-19, for zero: small numbers are scaled to it and back.
CB_DEV float bn_rsqrt(float v) {
    const bool small = v < 0x1p-100f;
    v = small ? v * 0x1p100f : v;
    const float r = __builtin_amdgcn_rsqf(v);
    const float y = r > 0.f && r < INFINITY ? fmaf(r * 0.5f, fmaf(-v * r, r, 1.f), r) : r;
    return small ? y * 0x1p50f : y;
}

// The columns that are the row's own: x, or zero.
template <int V, int N, class F>
CB_DEV void bn_own(float (&x)[V], int width, int t, int tpr, F&& f) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (i / N * tpr + t) * N + i % N < width ? f(x[i]) : 0.f;
}

// x <- (x - mean) rstd in place for M rows side by side (padding stays out of the sums by `width`); r: rstd. Two passes
// over the registers. MEAN: a norm of the kernel may be a layer norm; the kinds are told apart by selections. A slot behind
// the last row (width 0) has r = 1: with eps = 0 its zeros would make NaN of the column sums.
template <bool MEAN, int M, int V, int N>
CB_DEV void bn_normalise(float (*const (&x)[M])[V], const int (&kind)[M], float (&r)[M], int width, int t, int tpr, float inv,
                         float eps, float* sh, int& flip) {
    float s[M];
    if constexpr (MEAN) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            s[m] = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) s[m] += (*x[m])[i];
        }
        row_sum(s, tpr, sh, flip);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const float mean = kind[m] == 1 ? s[m] * inv : 0.f;
            bn_own<V, N>(*x[m], width, t, tpr, [&](float v) { return v - mean; });
        }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
        s[m] = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) s[m] += (*x[m])[i] * (*x[m])[i];
    }
    row_sum(s, tpr, sh, flip);
#pragma unroll
    for (int m = 0; m < M; ++m) {
        r[m] = kind[m] == 0 || width == 0 ? 1.f : bn_rsqrt(s[m] * inv + eps);
#pragma unroll
        for (int i = 0; i < V; ++i) (*x[m])[i] *= r[m];
    }
}

// Gradient at a norm's input from d at its normalised output xh: rstd (d - mean(d) - xh mean(d xh)).
template <int V>
CB_DEV void bn_back(float (&d)[V], const float (&xh)[V], float r, int kind, int tpr, float inv, float* sh, int& flip) {
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) { s[0] += d[i]; s[1] += d[i] * xh[i]; }
    row_sum(s, tpr, sh, flip);
    const float m = kind == 1 ? s[0] * inv : 0.f, mx = kind == 0 ? 0.f : s[1] * inv;
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = r * (d[i] - m - (kind == 0 ? 0.f : xh[i] * mx));
}

template <class T, int V>
struct BnRow {
    static constexpr int N = BnVec<T>::N;
    struct Raw { uint4 v[V / N]; };
    static CB_DEV Raw load(const BnMat& m, const BnArgs& a, const BnPlace& p, int64_t row, bool on) {
        Raw r;
        const T* q = static_cast<const T*>(m.p) + row * m.ld + int64_t(p.grp) * a.cg;
#pragma unroll
        for (int j = 0; j < V / N; ++j) {
            const int c = (j * a.tpr + p.t) * N;
            r.v[j] = BnVec<T>::raw(q + c, on ? p.width - c : 0);
        }
        return r;
    }
    static CB_DEV void unpack(const Raw& r, float (&x)[V]) {
#pragma unroll
        for (int j = 0; j < V / N; ++j) BnVec<T>::unpack(r.v[j], x + j * N);
    }
    static CB_DEV void store(const BnMat& m, const BnArgs& a, const BnPlace& p, int64_t row, const float (&x)[V]) {
        T* q = static_cast<T*>(m.p) + row * m.ld + int64_t(p.grp) * a.cg;
#pragma unroll
        for (int j = 0; j < V / N; ++j) {
            const int c = (j * a.tpr + p.t) * N;
            BnVec<T>::store(q + c, p.width - c, x + j * N);
        }
    }
    // a float vector over the channels, `other` where there is none; zero in the padding, where a layer norm's gradient
    // leaves its mean
    static CB_DEV void vec(const float* v, float other, const BnArgs& a, const BnPlace& p, float (&x)[V]) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const int c = (i / N * a.tpr + p.t) * N + i % N;
            const float* q = v ? v + int64_t(p.grp) * a.cg + c : nullptr;
            if (q && c + 4 <= p.width) {
                const float4 f = load_f4(q);
                x[i] = f.x; x[i + 1] = f.y; x[i + 2] = f.z; x[i + 3] = f.w;
            } else
#pragma unroll
                for (int u = 0; u < 4; ++u) x[i + u] = c + u >= p.width ? 0.f : q ? q[u] : other;
        }
    }
};

template <class T, int V, bool GATE, bool TWO, bool MEAN>
__global__ __launch_bounds__(512) void bn_fwd_kernel(BnArgs a) {
    using R = BnRow<T, V>;
    constexpr int N = BnVec<T>::N;
    constexpr bool AHEAD = V == 8;   // with 16 elements a thread the registers are the rows' at hand
    __shared__ float sh[2 * 16 * 4];
    const BnPlace p(a);
    const float inv = 1.f / float(a.cg);
    int flip = 0;
    float gamma[V], beta[V], rs[V], gamma2[V], beta2[V];
    R::vec(a.gamma, 1.f, a, p, gamma);
    R::vec(a.beta, 0.f, a, p, beta);
    R::vec(a.rscale, 1.f, a, p, rs);
    if (TWO) { R::vec(a.gamma2, 1.f, a, p, gamma2); R::vec(a.beta2, 0.f, a, p, beta2); }
    // whole workgroups go round together (row_sum has barriers), the next round's rows on their way
    int64_t base = int64_t(blockIdx.x) * a.rb;
    typename R::Raw rh, rg, rr;
    auto fetch = [&](int64_t base) {
        const int64_t row = base + p.slot;
        const bool on = row < a.n;
        rh = R::load(a.h, a, p, row, on);
        if (GATE) rg = R::load(a.gate, a, p, row, on);
        rr = R::load(a.res, a, p, row, on && a.res.p);
    };
    if (AHEAD) fetch(base);
    for (; base < a.n; base += p.step) {
        if (!AHEAD) fetch(base);
        const int64_t row = base + p.slot;
        BnPlace q = p;
        if (row >= a.n) q.width = 0;
        float x[V], y[V], gt[V];
        R::unpack(rh, x);
        R::unpack(rr, y);
        if (GATE) R::unpack(rg, gt);
        if (AHEAD && base + p.step < a.n) fetch(base + p.step);
        float r[1];
        bn_normalise<MEAN, 1, V, N>({&x}, {a.norm}, r, q.width, p.t, a.tpr, inv, a.eps, sh, flip);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float u = x[i] * gamma[i] + beta[i];
            if (GATE) u *= a.act == 0 ? gt[i] : a.act == 1 ? gt[i] * bn_sigmoid(gt[i]) : bn_sigmoid(gt[i]);
            y[i] = y[i] + u * rs[i];
        }
        R::store(a.out, a, q, row, y);
        if (TWO) {
            bn_own<V, N>(y, q.width, p.t, a.tpr, [](float v) { return BnVec<T>::round(v); });
            bn_normalise<MEAN, 1, V, N>({&y}, {a.norm2}, r, q.width, p.t, a.tpr, inv, a.eps, sh, flip);
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = y[i] * gamma2[i] + beta2[i];
            R::store(a.out2, a, q, row, y);
        }
    }
}

template <class T, int V, bool GATE, bool TWO, bool MEAN>
__global__ __launch_bounds__(512) void bn_bwd_kernel(BnArgs a) {
    using R = BnRow<T, V>;
    constexpr int N = BnVec<T>::N, Q = TWO ? 5 : 3;
    constexpr bool AHEAD = V == 8;
    __shared__ float sh[2 * 16 * 4];
    extern __shared__ float cols[];   // [threads][V]
    const BnPlace p(a);
    const float inv = 1.f / float(a.cg);
    int flip = 0;
    float gamma[V], beta[V], rs[V], gamma2[V];
    if (AHEAD) {
        R::vec(a.gamma, 1.f, a, p, gamma);
        R::vec(a.beta, 0.f, a, p, beta);
        R::vec(a.rscale, 1.f, a, p, rs);
        if (TWO) R::vec(a.gamma2, 1.f, a, p, gamma2);
    }
    float sum[Q][V];
#pragma unroll
    for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[k][i] = 0.f;
    int64_t base = int64_t(blockIdx.x) * a.rb;
    typename R::Raw rd, rh, rg, rd2, ro;
    auto fetch = [&](int64_t base) {
        const int64_t row = base + p.slot;
        const bool on = row < a.n;
        rh = R::load(a.h, a, p, row, on);
        if (TWO) {
            ro = R::load(a.out, a, p, row, on);
            rd2 = R::load(a.dout2, a, p, row, on);
        }
        rd = R::load(a.dout, a, p, row, on && a.dout.p);
        if (GATE) rg = R::load(a.gate, a, p, row, on);
    };
    if (AHEAD) fetch(base);
    for (; base < a.n; base += p.step) {
        if (!AHEAD) fetch(base);
        const int64_t row = base + p.slot;
        BnPlace q = p;
        if (row >= a.n) q.width = 0;
        float ds[V], x[V], gt[V], d[V], y[V], r[TWO ? 2 : 1];
        R::unpack(rh, x);
        R::unpack(rd, ds);
        if (GATE) R::unpack(rg, gt);
        if (TWO) { R::unpack(rd2, d); R::unpack(ro, y); }
        if (AHEAD && base + p.step < a.n) fetch(base + p.step);
        if constexpr (TWO) {
            bn_normalise<MEAN, 2, V, N>({&x, &y}, {a.norm, a.norm2}, r, q.width, p.t, a.tpr, inv, a.eps, sh, flip);
            if (!AHEAD) R::vec(a.gamma2, 1.f, a, p, gamma2);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sum[Q - 2][i] += d[i] * y[i];
                sum[Q - 1][i] += d[i];
                d[i] *= gamma2[i];
            }
            bn_back<V>(d, y, r[1], a.norm2, a.tpr, inv, sh, flip);
#pragma unroll
            for (int i = 0; i < V; ++i) ds[i] += d[i];
        } else {
            bn_normalise<MEAN, 1, V, N>({&x}, {a.norm}, r, q.width, p.t, a.tpr, inv, a.eps, sh, flip);
        }
        if (a.dres.p) R::store(a.dres, a, q, row, ds);
        if (!AHEAD) {   // held through the loop they would be in memory all the same
            R::vec(a.gamma, 1.f, a, p, gamma);
            R::vec(a.beta, 0.f, a, p, beta);
            R::vec(a.rscale, 1.f, a, p, rs);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float z = x[i] * gamma[i] + beta[i], du = ds[i] * rs[i];
            float act = 1.f;
            if (GATE) {
                float slope = 1.f;
                if (a.act == 0) act = gt[i];
                else {
                    const float s = bn_sigmoid(gt[i]);
                    act = a.act == 1 ? gt[i] * s : s;
                    slope = a.act == 1 ? s * (1.f + gt[i] * (1.f - s)) : s * (1.f - s);
                }
                gt[i] = du * z * slope;
            }
            sum[2][i] += ds[i] * (z * act);
            const float dz = du * act;
            sum[0][i] += dz * x[i];
            sum[1][i] += dz;
            ds[i] = dz * gamma[i];
        }
        if (GATE && a.dgate.p) R::store(a.dgate, a, q, row, gt);
        bn_back<V>(ds, x, r[0], a.norm, a.tpr, inv, sh, flip);
        R::store(a.dh, a, q, row, ds);
    }
    // the workgroup's column sums: over its row slots, then one partial row
#pragma unroll
    for (int k = 0; k < Q; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) cols[threadIdx.x * V + i] = sum[k][i];
        __syncthreads();
        if (p.slot == 0 && p.on)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i / N * a.tpr + p.t) * N + i % N;
                if (c >= a.cg) continue;
                float s = sum[k][i];
                for (int u = 1; u < a.rb; ++u) s += cols[(threadIdx.x + u * a.gb * a.tpr) * V + i];
                a.part[(int64_t(blockIdx.x) * Q + k) * a.C + p.grp * a.cg + c] = s;
            }
    }
}

// Column sums over the workgroups' partial rows: 32 columns a workgroup, 32 slices of the partials each, in 64 bits. (Within a
// workgroup, over n / 512 rows or so, they are float32 sums in a thread and over its row slots: 3001 x 1531 is off by 1.1e-7 from
// 64 bits, with 64-bit sums throughout by 1.0e-7.)
__global__ __launch_bounds__(1024) void bn_cols_kernel(BnArgs a, int blocks, int nq) {
    __shared__ double sh[32][33];
    const int k = blockIdx.y, lane = threadIdx.x & 31, sl = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float* out = a.grads[k];
    if (!out) return;
    double s = 0.0;
    if (c < a.C) {
        const float* p = a.part + int64_t(k) * a.C + c;
        const int64_t st = int64_t(nq) * a.C;
        int b = sl;
        for (; b + 7 * 32 < blocks; b += 8 * 32) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p[(b + 32 * u) * st];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += v[u];
        }
        for (; b < blocks; b += 32) s += p[b * st];
    }
    sh[sl][lane] = s;
    __syncthreads();
    if (sl == 0 && c < a.C) {
#pragma unroll
        for (int u = 1; u < 32; ++u) s += sh[u][lane];
        out[c] = float(s);
    }
}

struct BnPlan { int V, threads, tpr, gb, rb; int64_t blocks; int gy; };

constexpr int kBnFwdBlocks = 1024;
constexpr int kBnBlocks = 512;   // of a backward pass: each leaves a row of partial column sums

BnPlan bn_plan(int64_t n, int C, int G) {
    BnPlan p;
    const int cg = C / G;
    p.V = cg <= 4096 ? 8 : 16;
    p.tpr = 1;
    while (p.tpr * p.V < cg) p.tpr *= 2;
    p.threads = std::max(256, p.tpr);
    const int units = p.threads / p.tpr;
    p.gb = std::min(G, units);
    p.rb = units / p.gb;
    p.gy = (G + p.gb - 1) / p.gb;
    p.blocks = (n + p.rb - 1) / p.rb;
    return p;
}

template <class T, int V>
hipError_t bn_launch(const BnArgs& a, const BnPlan& p, bool bwd, hipStream_t s) {
    const dim3 grid(unsigned(p.blocks), unsigned(p.gy)), block(p.threads);
    auto go = [&](auto gate, auto two, auto mean) {
        constexpr bool GA = decltype(gate)::value, TW = decltype(two)::value, ME = decltype(mean)::value;
        if (bwd) hipLaunchKernelGGL((bn_bwd_kernel<T, V, GA, TW, ME>), grid, block, size_t(p.threads) * V * 4, s, a);
        else hipLaunchKernelGGL((bn_fwd_kernel<T, V, GA, TW, ME>), grid, block, 0, s, a);
    };
    const bool two = bwd ? a.dout2.p != nullptr : a.out2.p != nullptr;
    auto pick = [](bool b, auto f) { b ? f(std::true_type{}) : f(std::false_type{}); };
    pick(a.gate.p != nullptr, [&](auto gate) {
        pick(two, [&](auto tw) {
            pick(a.norm == 1 || (two && a.norm2 == 1), [&](auto mean) { go(gate, tw, mean); });
        });
    });
    return hipGetLastError();
}

hipError_t bn_run(int prec, BnArgs& a, const BnPlan& p, bool bwd, hipStream_t s) {
    a.cg = a.C / a.G; a.tpr = p.tpr; a.gb = p.gb; a.rb = p.rb;
    ProfScope ps(s, [&] {
        return cb_key(bwd ? "blocknorm_bwd" : "blocknorm_fwd", prec, std::to_string(a.n) + "x" + cb_dims(a.C, a.G));
    });
    if (prec == 0) return p.V == 8 ? bn_launch<uint16_t, 8>(a, p, bwd, s) : bn_launch<uint16_t, 16>(a, p, bwd, s);
    return p.V == 8 ? bn_launch<float, 8>(a, p, bwd, s) : bn_launch<float, 16>(a, p, bwd, s);
}

}  // namespace

size_t blocknorm_bwd_ws_bytes(int, int64_t n, int C, int G, bool two) {
    const int64_t blocks = std::min<int64_t>(bn_plan(n, C, G).blocks, kBnBlocks);
    return size_t(std::max<int64_t>(blocks, 1)) * (two ? 5 : 3) * C * 4;
}

hipError_t blocknorm_fwd(int prec, BnArgs a, hipStream_t s) {
    if (a.n == 0) return hipSuccess;
    BnPlan p = bn_plan(a.n, a.C, a.G);
    p.blocks = std::min<int64_t>(p.blocks, kBnFwdBlocks);
    return bn_run(prec, a, p, false, s);
}

hipError_t blocknorm_bwd(int prec, BnArgs a, void* ws, hipStream_t s) {
    const bool two = a.dout2.p;
    if (a.n == 0) {
        for (float* g : a.grads)
            if (g) {
                const hipError_t e = fill_zero(g, a.C, s);
                if (e != hipSuccess) return e;
            }
        return hipSuccess;
    }
    BnPlan p = bn_plan(a.n, a.C, a.G);
    p.blocks = std::min<int64_t>(p.blocks, kBnBlocks);
    a.part = static_cast<float*>(ws);
    const hipError_t e = bn_run(prec, a, p, true, s);
    if (e != hipSuccess) return e;
    const int nq = two ? 5 : 3;
    ProfScope ps(s, [&] { return "blocknorm_params/" + std::to_string(p.blocks) + "x" + cb_dims(a.C, nq); });
    hipLaunchKernelGGL(bn_cols_kernel, dim3(unsigned((a.C + 31) / 32), unsigned(nq)), dim3(1024), 0, s, a, int(p.blocks), nq);
    return hipGetLastError();
}

}  // namespace cb
