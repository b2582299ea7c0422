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
    static CB_DEV void load(const T* p, int left, float* x) {
        if (left >= N) {
            const bn_u32x4 v = *reinterpret_cast<const bn_u32x4*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) { x[2 * i] = bf_lo(v[i]); x[2 * i + 1] = bf_hi(v[i]); }
                else x[i] = __uint_as_float(v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (sizeof(T) == 2) x[i] = i < left ? bf2f(p[i]) : 0.f;
                else x[i] = i < left ? p[i] : 0.f;
            }
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

// Sums of K numbers over the tpr threads of a row, in every one of them, in a fixed order.
template <int K>
CB_DEV void row_sum(float (&v)[K], int tpr, float* sh) {
    for (int d = min(tpr, 64) / 2; d > 0; d >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], d);
    if (tpr > 64) {
        const int wave = threadIdx.x >> 6, w = tpr >> 6, first = wave / w * w;
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) sh[wave * K + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = sh[first * K + k];
            for (int i = 1; i < w; ++i) v[k] += sh[(first + i) * K + k];
        }
    }
}

// x <- (x - mean) rstd in place (padding stays out of the sums by `width`); returns rstd. Two passes over the registers.
// MEAN: a norm of the kernel may be a layer norm; the kinds are told apart by selections, not by branches around sums.
template <bool MEAN, int V, int N>
CB_DEV float bn_normalise(float (&x)[V], int kind, int width, int t, int tpr, float inv, float eps, float* sh) {
    float s[1] = {0.f};
    if constexpr (MEAN) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[0] += x[i];
        row_sum(s, tpr, sh);
        const float mean = kind == 1 ? s[0] * inv : 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (i / N * tpr + t) * N + i % N < width ? x[i] - mean : 0.f;
        s[0] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s[0] += x[i] * x[i];
    row_sum(s, tpr, sh);
    const float r = kind == 0 ? 1.f : 1.f / sqrtf(s[0] * inv + eps);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= r;
    return r;
}

// Gradient at a norm's input from d at its normalised output xh: rstd (d - mean(d) - xh mean(d xh)).
template <int V, int N>
CB_DEV void bn_back(float (&d)[V], const float (&xh)[V], float r, int kind, int tpr, float inv, float* sh) {
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) { s[0] += d[i]; s[1] += d[i] * xh[i]; }
    row_sum(s, tpr, sh);
    const float m = kind == 1 ? s[0] * inv : 0.f, mx = kind == 0 ? 0.f : s[1] * inv;
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = r * (d[i] - m - (kind == 0 ? 0.f : xh[i] * mx));
}

CB_DEV float bn_sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

template <class T, int V>
struct BnRow {
    static constexpr int N = BnVec<T>::N;
    static CB_DEV void load(const BnMat& m, const BnArgs& a, const BnPlace& p, int64_t row, float (&x)[V]) {
        const T* q = static_cast<const T*>(m.p) + row * m.ld + int64_t(p.grp) * a.cg;
#pragma unroll
        for (int j = 0; j < V / N; ++j) {
            const int c = (j * a.tpr + p.t) * N;
            BnVec<T>::load(q + c, p.width - c, x + j * N);
        }
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
        for (int i = 0; i < V; ++i) {
            const int c = (i / N * a.tpr + p.t) * N + i % N;
            x[i] = c >= p.width ? 0.f : v ? v[int64_t(p.grp) * a.cg + c] : other;
        }
    }
};

template <class T, int V, bool GATE, bool TWO, bool MEAN>
__global__ __launch_bounds__(V == 8 ? 256 : 512) void bn_fwd_kernel(BnArgs a) {
    using R = BnRow<T, V>;
    constexpr int N = BnVec<T>::N;
    __shared__ float sh[32];
    const BnPlace p(a);
    const float inv = 1.f / float(a.cg);
    float gamma[V], beta[V], rs[V], gamma2[V], beta2[V];
    R::vec(a.gamma, 1.f, a, p, gamma);
    R::vec(a.beta, 0.f, a, p, beta);
    R::vec(a.rscale, 1.f, a, p, rs);
    if (TWO) { R::vec(a.gamma2, 1.f, a, p, gamma2); R::vec(a.beta2, 0.f, a, p, beta2); }
    // whole workgroups go round together: row_sum has barriers
    for (int64_t base = int64_t(blockIdx.x) * a.rb; base < a.n; base += p.step) {
        const int64_t row = base + p.slot;
        BnPlace q = p;
        if (row >= a.n) q.width = 0;
        float x[V], y[V];
        R::load(a.h, a, q, row, x);
        float gt[V];
        if (GATE) R::load(a.gate, a, q, row, gt);
        if (a.res.p) R::load(a.res, a, q, row, y);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = 0.f;
        bn_normalise<MEAN, V, N>(x, a.norm, q.width, p.t, a.tpr, inv, a.eps, sh);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float u = x[i] * gamma[i] + beta[i];
            if (GATE) u *= a.act == 0 ? gt[i] : a.act == 1 ? gt[i] * bn_sigmoid(gt[i]) : bn_sigmoid(gt[i]);
            y[i] = y[i] + u * rs[i];
        }
        R::store(a.out, a, q, row, y);
        if (TWO) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i / N * a.tpr + p.t) * N + i % N;
                y[i] = c < q.width ? BnVec<T>::round(y[i]) : 0.f;
            }
            bn_normalise<MEAN, V, N>(y, a.norm2, q.width, p.t, a.tpr, inv, a.eps, sh);
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = y[i] * gamma2[i] + beta2[i];
            R::store(a.out2, a, q, row, y);
        }
    }
}

template <class T, int V, bool GATE, bool TWO, bool MEAN>
__global__ __launch_bounds__(V == 8 ? 256 : 512) void bn_bwd_kernel(BnArgs a) {
    using R = BnRow<T, V>;
    constexpr int N = BnVec<T>::N, Q = TWO ? 5 : 3;
    __shared__ float sh[32];
    extern __shared__ float cols[];   // [threads][V]
    const BnPlace p(a);
    const float inv = 1.f / float(a.cg);
    float gamma[V], beta[V], rs[V], gamma2[V];
    R::vec(a.gamma, 1.f, a, p, gamma);
    R::vec(a.beta, 0.f, a, p, beta);
    R::vec(a.rscale, 1.f, a, p, rs);
    if (TWO) R::vec(a.gamma2, 1.f, a, p, gamma2);
    float sum[Q][V];
#pragma unroll
    for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[k][i] = 0.f;
    for (int64_t base = int64_t(blockIdx.x) * a.rb; base < a.n; base += p.step) {
        const int64_t row = base + p.slot;
        BnPlace q = p;
        if (row >= a.n) q.width = 0;
        float ds[V], x[V], gt[V];
        if (a.dout.p) R::load(a.dout, a, q, row, ds);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) ds[i] = 0.f;
        R::load(a.h, a, q, row, x);
        if (GATE) R::load(a.gate, a, q, row, gt);
        if (TWO) {
            float d[V], y[V];
            R::load(a.dout2, a, q, row, d);
            R::load(a.out, a, q, row, y);
            const float r = bn_normalise<MEAN, V, N>(y, a.norm2, q.width, p.t, a.tpr, inv, a.eps, sh);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sum[Q - 2][i] += d[i] * y[i];
                sum[Q - 1][i] += d[i];
                d[i] *= gamma2[i];
            }
            bn_back<V, N>(d, y, r, a.norm2, a.tpr, inv, sh);
#pragma unroll
            for (int i = 0; i < V; ++i) ds[i] += d[i];
        }
        if (a.dres.p) R::store(a.dres, a, q, row, ds);
        const float r = bn_normalise<MEAN, V, N>(x, a.norm, q.width, p.t, a.tpr, inv, a.eps, sh);
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
        bn_back<V, N>(ds, x, r, a.norm, a.tpr, inv, sh);
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

// Column sums over the workgroups' partial rows: 32 columns a workgroup, 8 slices of the partials each.
__global__ __launch_bounds__(256) void bn_cols_kernel(BnArgs a, int blocks, int nq) {
    __shared__ double sh[8][33];
    const int k = blockIdx.y, lane = threadIdx.x & 31, sl = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float* out = a.grads[k];
    if (!out) return;
    double s = 0.0;
    if (c < a.C)
        for (int b = sl; b < blocks; b += 8) s += a.part[(int64_t(b) * nq + k) * a.C + c];
    sh[sl][lane] = s;
    __syncthreads();
    if (sl == 0 && c < a.C) {
#pragma unroll
        for (int u = 1; u < 8; ++u) s += sh[u][lane];
        out[c] = float(s);
    }
}

struct BnPlan { int V, threads, tpr, gb, rb; int64_t blocks; int gy; };

constexpr int kBnBlocks = 1024;   // of a backward pass: each leaves a row of partial column sums

BnPlan bn_plan(int64_t n, int C, int G) {
    BnPlan p;
    const int cg = C / G;
    p.V = cg <= 512 ? 8 : 16;
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
    p.blocks = std::min<int64_t>(p.blocks, 1 << 16);
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
    hipLaunchKernelGGL(bn_cols_kernel, dim3(unsigned((a.C + 31) / 32), unsigned(nq)), dim3(256), 0, s, a, int(p.blocks), nq);
    return hipGetLastError();
}

}  // namespace cb
