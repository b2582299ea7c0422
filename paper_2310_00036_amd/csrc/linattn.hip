// Linear attention with a decay per head over rollouts: R_p = keep_p R_{p-1} + k_p v_p^T, o_p = R_p^T q_p, forward for
// the outputs and the gradient of q (with the roles of k and v and of q and the output's gradient exchanged), backwards
// for those of k and v.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "linattn.h"

namespace cb {

namespace {

CB_DEV const void* la_at(const void* p, int64_t elems, int es) { return static_cast<const char*>(p) + elems * es; }

// The recurrence row by row: one wave for 64 columns of one env's and head's state, a column a lane, its dk numbers in
// registers.
template <class Pr, int DK>
__global__ __launch_bounds__(64) void la_steps_kernel(LaArgs a, int y0) {
    using T = typename Pr::T;
    constexpr int KL = (DK + 63) / 64;
    __shared__ float sq[DK], sk[DK];
    const LaPass& P = a.pass[y0 + blockIdx.y];
    const int lane = threadIdx.x;
    const int nbs = (P.dv + 63) / 64;
    const int64_t eh = blockIdx.x / nbs;
    const int n = int(blockIdx.x % nbs) * 64 + lane;
    const int64_t e = eh / a.H, h = eh % a.H;
    const bool on = n < P.dv;
    const float g = expf(a.log_decay[h]);
    const int64_t dir = P.back ? -1 : 1;
    int64_t t = P.back ? a.T - 1 : 0;
    const T* q = static_cast<const T*>(P.q.p) + e * P.q.e + h * P.q.h + t * P.q.t;
    const T* k = static_cast<const T*>(P.k.p) + e * P.k.e + h * P.k.h + t * P.k.t;
    const T* v = static_cast<const T*>(P.v.p) + e * P.v.e + h * P.v.h + t * P.v.t + n;
    T* o = static_cast<T*>(const_cast<void*>(P.o.p)) + e * P.o.e + h * P.o.h + t * P.o.t + n;
    auto keep_at = [&](int64_t td) { return a.dones && a.dones[td * a.d_t + e * a.d_e] ? 0.f : g; };
    float R[DK];
#pragma unroll
    for (int i = 0; i < DK; ++i) R[i] = 0.f;
    float keep = P.back ? 1.f : keep_at(0);
    if (P.x0 && keep != 0.f && on) {
        const float* x = P.x0 + eh * P.dk * P.dv + int64_t(n) * P.xn;
#pragma unroll
        for (int i = 0; i < DK; ++i)
            if (i < P.dk) R[i] = x[i * P.xk];
    }
    T nq[KL], nk[KL], nv = T(0);
    auto fetch = [&] {
#pragma unroll
        for (int u = 0; u < KL; ++u) {
            const int i = lane + 64 * u;
            nq[u] = i < P.dk ? q[i] : T(0);
            nk[u] = i < P.dk ? k[i] : T(0);
        }
        nv = on ? *v : T(0);
    };
    fetch();
    for (int p = 0; p < a.T; ++p) {
#pragma unroll
        for (int u = 0; u < KL; ++u)
            if (lane + 64 * u < DK) {
                sq[lane + 64 * u] = Pr::load(nq[u]);
                sk[lane + 64 * u] = Pr::load(nk[u]);
            }
        const float vn = Pr::load(nv) * P.in;
        __syncthreads();
        if (p + 1 < a.T) { q += dir * P.q.t; k += dir * P.k.t; v += dir * P.v.t; fetch(); }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < DK; ++i) {
            R[i] = (keep == 0.f ? 0.f : keep * R[i]) + sk[i] * vn;
            s += sq[i] * R[i];
        }
        if (on) *o = Pr::store(s * P.out);
        o += dir * P.o.t;
        // what lies between this row and the next: the later one's episode start
        if (P.back) keep = keep_at(t);
        else if (p + 1 < a.T) keep = keep_at(t + 1);
        t += dir;
        __syncthreads();
    }
    if (P.x1 && on) {
        if (!P.back) keep = 1.f;
        float* x = P.x1 + eh * P.dk * P.dv + int64_t(n) * P.xn;
#pragma unroll
        for (int i = 0; i < DK; ++i)
            if (i < P.dk) x[i * P.xk] = keep == 0.f ? 0.f : keep * R[i];
    }
}

template <class Pr>
hipError_t la_steps(const LaArgs& a, hipStream_t s) {
    for (int y = 0; y < a.np; ++y) {
        const LaPass& P = a.pass[y];
        const dim3 grid(unsigned(int64_t(a.E) * a.H * ((P.dv + 63) / 64)));
        if (P.dk <= 32) hipLaunchKernelGGL((la_steps_kernel<Pr, 32>), grid, dim3(64), 0, s, a, y);
        else if (P.dk <= 64) hipLaunchKernelGGL((la_steps_kernel<Pr, 64>), grid, dim3(64), 0, s, a, y);
        else hipLaunchKernelGGL((la_steps_kernel<Pr, 128>), grid, dim3(64), 0, s, a, y);
    }
    return hipGetLastError();
}

// No rows: the state goes through (a gradient too: nothing is between the two).
__global__ void la_empty_kernel(const float* x0, float* x1, int64_t n) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
        x1[i] = x0 ? x0[i] : 0.f;
}

}  // namespace

size_t linattn_ws_bytes(int, int, int, int, int, int, int) { return 0; }

hipError_t linattn(int prec, LaArgs a, void*, hipStream_t s) {
    if (int64_t(a.E) * a.H == 0) return hipSuccess;
    if (a.T == 0) {
        for (int y = 0; y < a.np; ++y) {
            const LaPass& P = a.pass[y];
            const int64_t n = int64_t(a.E) * a.H * P.dk * P.dv;
            if (!P.x1 || P.x1 == P.x0) continue;
            const int64_t blocks = std::min<int64_t>((n + 255) / 256, 4096);
            hipLaunchKernelGGL(la_empty_kernel, dim3(unsigned(blocks)), dim3(256), 0, s, P.x0, P.x1, n);
        }
        return hipGetLastError();
    }
    ProfScope ps(s, [&] {
        return cb_key("linattn", prec, std::to_string(a.T) + "x" + std::to_string(a.E) + "x" + std::to_string(a.H) + "x" +
                                           cb_dims(a.pass[0].dk, a.pass[0].dv) + (a.np > 1 ? "/bwd" : ""));
    });
    return prec == 0 ? la_steps<PrecBF16>(a, s) : la_steps<PrecF32>(a, s);
}

}  // namespace cb
