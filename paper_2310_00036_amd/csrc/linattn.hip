// Linear attention with a decay per head over rollouts: R_p = keep_p R_{p-1} + k_p v_p^T, o_p = R_p^T q_p, forward for
// the outputs and the gradient of q (with the roles of k and v and of q and the output's gradient exchanged), backwards
// for those of k and v.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "linattn.h"

namespace cb {

namespace {

// One step from state to state, HBM-bound: the state is read and written once. A workgroup has one state, a thread four
// neighbouring columns of every (NT / LR)th row, all loaded before anything waits (LR: the lanes of a row, a power of two).
// 4096 envs x 8 heads of 128 x 128: 4.3 GB in 0.86 ms, 5.0 TB/s. (A rollout of 4 steps of 512 envs x 8 heads of 64 takes 49 us
// as a chunk and took 31 row by row from registers: with one step, where the state is all there is to move, a chunk's
// set-up would cost more than the step. On 64 envs x 4 heads the chunk is the faster from 4 steps on, 8 us for 18.)
template <class Pr, int NT, int LR>
__global__ __launch_bounds__(NT) void la_step_kernel(LaArgs a) {
    using T = typename Pr::T;
    constexpr int RP = NT / LR;                      // rows at a time
    constexpr int UN = (kLaMaxDim + RP - 1) / RP;    // of them, at most
    __shared__ float sq[kLaMaxDim], sk[kLaMaxDim];
    __shared__ float4 red[NT / 64][LR];
    const LaPass& P = a.pass[0];
    const int tid = threadIdx.x, col = tid % LR * 4, r0 = tid / LR, dk = P.dk, dv = P.dv;
    const uint32_t eh = blockIdx.x, e = eh / uint32_t(a.H), h = eh - e * a.H;
    const bool cut = a.dones && a.dones[int64_t(e) * a.d_e];
    const int64_t base = int64_t(eh) * dk * dv;
    const bool whole = dv % 4 == 0;
    float4 x[UN];
    const float* px = P.x0 && !cut && col < dv ? P.x0 + base + col : nullptr;
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int kk = r0 + u * RP;
        x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (u * RP >= dk) break;
        if (px && kk < dk) {
            const float* p = px + kk * dv;
            if (whole) x[u] = load_f4(p);
            else {
                x[u].x = p[0];
                if (col + 1 < dv) x[u].y = p[1];
                if (col + 2 < dv) x[u].z = p[2];
                if (col + 3 < dv) x[u].w = p[3];
            }
        }
    }
    const T* v = static_cast<const T*>(P.v.p) + e * P.v.e + h * P.v.h;
    const T* q = static_cast<const T*>(P.q.p) + e * P.q.e + h * P.q.h;
    const T* k = static_cast<const T*>(P.k.p) + e * P.k.e + h * P.k.h;
    for (int i = tid; i < dk; i += NT) { sq[i] = Pr::load(q[i]); sk[i] = Pr::load(k[i]); }
    float vv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) vv[i] = col + i < dv ? Pr::load(v[col + i]) : 0.f;
    const float gd = float(exp(double(a.log_decay[h])));
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float* py = P.x1 ? P.x1 + base + col : nullptr;
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int kk = r0 + u * RP;
        if (u * RP >= dk) break;
        if (kk < dk && col < dv) {
            const float kf = sk[kk], qf = sq[kk];
            // (without a state before it there is nothing to decay: zero times a decay of infinity is none)
            x[u].x = (px ? gd * x[u].x : 0.f) + kf * vv[0];
            x[u].y = (px ? gd * x[u].y : 0.f) + kf * vv[1];
            x[u].z = (px ? gd * x[u].z : 0.f) + kf * vv[2];
            x[u].w = (px ? gd * x[u].w : 0.f) + kf * vv[3];
            o.x += qf * x[u].x; o.y += qf * x[u].y; o.z += qf * x[u].z; o.w += qf * x[u].w;
            if (py) {
                float* p = py + kk * dv;
                if (whole) *reinterpret_cast<cb_f32x4_a4*>(p) = cb_f32x4_a4{x[u].x, x[u].y, x[u].z, x[u].w};
                else {
                    p[0] = x[u].x;
                    if (col + 1 < dv) p[1] = x[u].y;
                    if (col + 2 < dv) p[2] = x[u].z;
                    if (col + 3 < dv) p[3] = x[u].w;
                }
            }
        }
    }
#pragma unroll
    for (int d = LR; d < 64; d *= 2) {
        o.x += __shfl_xor(o.x, d); o.y += __shfl_xor(o.y, d); o.z += __shfl_xor(o.z, d); o.w += __shfl_xor(o.w, d);
    }
    if ((tid & 63) < LR) red[tid >> 6][tid & 63] = o;
    __syncthreads();
    if (tid < LR && col < dv) {
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) {
            const float4 t = red[w][tid];
            o.x += t.x; o.y += t.y; o.z += t.z; o.w += t.w;
        }
        T* po = static_cast<T*>(const_cast<void*>(P.o.p)) + e * P.o.e + h * P.o.h + col;
        const float y[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < dv) po[i] = Pr::store(y[i] * P.out);
    }
}

template <class Pr>
hipError_t la_step(const LaArgs& a, hipStream_t s) {
    const LaPass& P = a.pass[0];
    const dim3 grid(unsigned(int64_t(a.E) * a.H));
    if (P.dv <= 32) hipLaunchKernelGGL((la_step_kernel<Pr, 64, 8>), grid, dim3(64), 0, s, a);
    else if (P.dv <= 64) hipLaunchKernelGGL((la_step_kernel<Pr, 256, 16>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((la_step_kernel<Pr, 256, 32>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------- chunks of 64 rows on the matrix cores
//
// Rows i of a chunk with the state X before it (c_i: episode starts up to row i, counting its own going forward and not
// going back; l = 1 forward, 0 back; n rows):
//   o_i = [c_i = 0] g^(i+l) X^T q_i + sum_{j <= i, c_j = c_i} g^(i-j) (q_i . k_j) v_j,
//   X  <- [c = 0] g^n X + sum_{j: c_j = c} g^(n-l-j) k_j v_j^T.
// A wave owns 16 columns of v, o and X. X stays in its registers as results of the matrix products, laid out so that they
// are, without moving between lanes, the operand of X^T q. The 64 x 64 products q_i . k_j are formed once by the waves
// together and handed round in LDS.
//
// 64 rows: the products on the diagonal grow with the chunk, the state's with its number, and a wave's lanes are the rows.
// A chunk of 64-wide heads is 32 KB in bf16 and takes a workgroup of four waves 2.9 us (7000 cycles, about 1150 of them in
// the matrix cores); two of them share a CU, 2048 x 256 envs x 4 heads take 279 us, 4.0 TB/s. Heads of 128: eight waves, alone on
// a CU, 5.6 us for 64 KB.

constexpr int kL = 64;
typedef uint32_t cb_u32x2 __attribute__((ext_vector_type(2)));
// words at any alignment of an element, which global memory takes
typedef uint32_t la_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t la_u32x4 __attribute__((ext_vector_type(4), aligned(2)));

// bf16: products of two bf16 numbers are exact; what is no bf16 number (the decayed products, X, the decayed v) goes into
// a product as three of them, each nearest to what the ones before leave: 24 bits, as float32 has. (Two for the decayed
// products and X, 16 bits, would show wherever a sum's terms cancel; they take 60 us for 65 in the backward pass of 128 x 128
// envs x 8 heads of 64, 128 for 136 in 16384 x 2 x 8 heads of 128 forward.)
struct LaB {
    using T = uint16_t;
    using Frag = uint4;
    static constexpr int KB = 32, KPL = 8;   // contraction per fragment, elements of it a lane holds (at KPL * group)
    static constexpr int NP = 3, NX = 3, NV = 3;
    static CB_DEV cb_f32x4 mma(Frag a, Frag b, cb_f32x4 c) { return PrecBF16::mma(a, b, c); }
    static CB_DEV float load(T v) { return bf2f(v); }
    static CB_DEV void unpack(Frag f, float* x) {
        x[0] = bf_lo(f.x); x[1] = bf_hi(f.x); x[2] = bf_lo(f.y); x[3] = bf_hi(f.y);
        x[4] = bf_lo(f.z); x[5] = bf_hi(f.z); x[6] = bf_lo(f.w); x[7] = bf_hi(f.w);
    }
    static CB_DEV uint32_t finite2(uint32_t u) {
        return ((u & 0x7f80u) == 0x7f80u ? 0u : u & 0xffffu) | ((u & 0x7f800000u) == 0x7f800000u ? 0u : u & 0xffff0000u);
    }
    static CB_DEV Frag finite(Frag f) { return make_uint4(finite2(f.x), finite2(f.y), finite2(f.z), finite2(f.w)); }
    // x as a sum of bf16 numbers, the first plane the nearest one, each further plane nearest to the rest
    template <int N>
    static CB_DEV void split(float* x, Frag (&f)[N]) {
#pragma unroll
        for (int p = 0; p < N; ++p) {
            f[p] = make_uint4(pack2bf(x[0], x[1]), pack2bf(x[2], x[3]), pack2bf(x[4], x[5]), pack2bf(x[6], x[7]));
            float y[8];
            unpack(f[p], y);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] -= y[i];
        }
    }
    // four neighbouring entries of a row of the decayed products, plane by plane
    static CB_DEV void store_p(unsigned char* p, int plane, cb_f32x4 x) {
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const uint2 v = make_uint2(pack2bf(x[0], x[1]), pack2bf(x[2], x[3]));
            *reinterpret_cast<uint2*>(p + u * plane) = v;
            x[0] -= bf_lo(v.x); x[1] -= bf_hi(v.x); x[2] -= bf_lo(v.y); x[3] -= bf_hi(v.y);
        }
    }
    // Fragment with the contraction along the tile's rows row0 .. row0+31, of 16 columns: operand row (or column) r is
    // column col + 4 (r / 4) CS + r % 4, so CS = 1 takes neighbours and CS = 2 skips every other four.
    template <int CS>
    static CB_DEV Frag cols(const unsigned char* tile, int rs, int row0, int col) {
        const int l = threadIdx.x & 63, g = l >> 4, c = l & 15;
        const unsigned char* p = tile + (row0 + 8 * g + (c >> 2)) * rs + (col + 4 * CS * (c & 3)) * 2;
        const uint2 a = lds_read_tr16(p), b = lds_read_tr16(p + 4 * rs);
        return make_uint4(a.x, a.y, b.x, b.y);
    }
    // X's 16 x 16 results: the row that result m has in lane group g as its r-th, so that two results are a fragment
    static CB_DEV int krow(int m, int g, int r) { return 32 * (m >> 1) + 8 * g + 4 * (m & 1) + r; }
    static CB_DEV Frag kcols(const unsigned char* tile, int rs, int row0, int m) {
        return cols<2>(tile, rs, row0, 32 * (m >> 1) + 4 * (m & 1));
    }
    template <int NT>
    static CB_DEV void xfrag(const cb_f32x4 (&X)[NT], int kb, Frag (&f)[NX]) {
        float x[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) { x[r] = X[2 * kb][r]; x[4 + r] = X[2 * kb + 1][r]; }
        split(x, f);
    }
    static CB_DEV void store4o(__amdgpu_buffer_rsrc_t r, uint32_t off, cb_f32x4 x) {
        __builtin_amdgcn_raw_buffer_store_b64(cb_u32x2{pack2bf(x[0], x[1]), pack2bf(x[2], x[3])}, r, off, 0, 0);
    }
    static CB_DEV void store1o(__amdgpu_buffer_rsrc_t r, uint32_t off, float x) {
        __builtin_amdgcn_raw_buffer_store_b16(f2bf(x), r, off, 0, 0);
    }
    static CB_DEV T store(float x) { return f2bf(x); }
    static CB_DEV void store4(T* p, cb_f32x4 x) {
        *reinterpret_cast<la_u32x2*>(p) = la_u32x2{pack2bf(x[0], x[1]), pack2bf(x[2], x[3])};
    }
};

struct LaF {
    using T = float;
    using Frag = float4;
    static constexpr int KB = 16, KPL = 4;
    static constexpr int NP = 1, NX = 1, NV = 1;
    static CB_DEV cb_f32x4 mma(Frag a, Frag b, cb_f32x4 c) {
        c = PrecF32::mma(a.x, b.x, c);
        c = PrecF32::mma(a.y, b.y, c);
        c = PrecF32::mma(a.z, b.z, c);
        return PrecF32::mma(a.w, b.w, c);
    }
    static CB_DEV float load(T v) { return v; }
    static CB_DEV void unpack(Frag f, float* x) { x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w; }
    static CB_DEV Frag finite(Frag f) {
        return make_float4(isfinite(f.x) ? f.x : 0.f, isfinite(f.y) ? f.y : 0.f, isfinite(f.z) ? f.z : 0.f,
                           isfinite(f.w) ? f.w : 0.f);
    }
    template <int N>
    static CB_DEV void split(float* x, Frag (&f)[N]) { f[0] = make_float4(x[0], x[1], x[2], x[3]); }
    static CB_DEV void store_p(unsigned char* p, int, cb_f32x4 x) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    }
    template <int CS>
    static CB_DEV Frag cols(const unsigned char* tile, int rs, int row0, int col) {
        const int l = threadIdx.x & 63, g = l >> 4, c = l & 15;
        const unsigned char* p = tile + (row0 + 4 * g) * rs + (col + c) * 4;
        return make_float4(*reinterpret_cast<const float*>(p), *reinterpret_cast<const float*>(p + rs),
                           *reinterpret_cast<const float*>(p + 2 * rs), *reinterpret_cast<const float*>(p + 3 * rs));
    }
    static CB_DEV int krow(int m, int g, int r) { return 16 * m + 4 * g + r; }
    static CB_DEV Frag kcols(const unsigned char* tile, int rs, int row0, int m) { return cols<1>(tile, rs, row0, 16 * m); }
    template <int NT>
    static CB_DEV void xfrag(const cb_f32x4 (&X)[NT], int kb, Frag (&f)[NX]) {
        f[0] = make_float4(X[kb][0], X[kb][1], X[kb][2], X[kb][3]);
    }
    static CB_DEV void store4o(__amdgpu_buffer_rsrc_t r, uint32_t off, cb_f32x4 x) {
        buf_store16(r, off, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                                       __float_as_uint(x[3])));
    }
    static CB_DEV void store1o(__amdgpu_buffer_rsrc_t r, uint32_t off, float x) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), r, off, 0, 0);
    }
    static CB_DEV T store(float x) { return x; }
    static CB_DEV void store4(T* p, cb_f32x4 x) { *reinterpret_cast<cb_f32x4_a4*>(p) = x; }
};

// Where a pass is cut along the rollout, each segment's own contribution to the state, then the states before them.
struct LaSegs {
    int segs, chunks;          // segments, chunks in each but the last
    float* state[kLaMaxPasses];    // [segs][E H][dk dv]
    float* factor[kLaMaxPasses];   // [segs][E H]: what a segment leaves of the state before it; -1: an episode starts in it
};

template <class Tr, int DK, int NW, bool STATE>
struct LaTile {   // STATE: without q and the products
    static constexpr int ES = sizeof(typename Tr::T);
    static constexpr int RSK = DK * ES + 16, RSV = 16 * NW * ES + 16;
    // The products' rows. Of 32-wide heads, rows 0 .. 31 have 32 columns (what is above the diagonal is not read), so that
    // four bf16 workgroups share a CU: 1024 x 64 envs x 16 heads of 32 forward 81 us, with square planes 96. (Wider heads are
    // no more in a CU with it and pay for the addresses: 2048 x 64 x 4 heads of 64 forward 93 us square, 95 so.)
    static constexpr int RSP = kL * ES + 16, RSP0 = DK == 32 ? kL / 2 * ES + 16 : RSP;
    static constexpr int Q = 0, K = STATE ? 0 : kL * RSK, V = K + kL * RSK, P = V + kL * RSV, PP = kL / 2 * (RSP0 + RSP);
    static CB_DEV int prow(int i) {
        return RSP0 == RSP ? i * RSP : i < kL / 2 ? i * RSP0 : kL / 2 * RSP0 + (i - kL / 2) * RSP;
    }
    // g^0 .. g^64, 16 zeros, in out g^0 .. in out g^64, X's and v's weights by row, the rows that start an episode
    static constexpr int TAB = STATE ? P : P + Tr::NP * PP;
    static constexpr int BYTES = TAB + (2 * 68 + 16 + 2 * kL + 2) * 4;
    static constexpr int UQ = DK * ES / 16 / NW > 0 ? DK * ES / 16 / NW : 1;   // 16-byte pieces of q and k a thread moves
    static constexpr int UV = ES;                                             // of v
};

// Rows of one array through a buffer resource that is moved from chunk to chunk, at 32-bit offsets: what lies behind the
// chunk's last row, or in columns behind the array's, reads zero and is not written. A row steps by st bytes; going back,
// st is negative and the resource starts at the chunk's last row, so offsets have -(n - 1) st added.
// With |st| <= 2^25 a resource ends below 2^31 = kOOB, and no offset comes round into it modulo 2^32: rows go to 127 (threads
// without a row in a chunk of 32-wide bf16 heads among 8 waves), so going forward offsets stay below 127 2^25 + 2^9 < 2^32, and
// going back that of a row r >= n is 2^32 - (r - n + 1) |st| or more, which is n |st| or more, behind (n - 1) |st| + bytes;
// in columns behind the array's, rows go to 63: kOOB +- 63 |st| lies within 2^25 and 2^32.
constexpr int64_t kLaReach = int64_t(1) << 25;
struct LaRows {
    const char* p;             // the chunk's first row
    int st, bytes;             // bytes: of a row
    CB_DEV __amdgpu_buffer_rsrc_t rsrc(int n) const {
        const int span = __builtin_amdgcn_readfirstlane((n - 1) * st);
        const uint64_t b = reinterpret_cast<uint64_t>(span < 0 ? p + span : p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(b)), hi = __builtin_amdgcn_readfirstlane(uint32_t(b >> 32));
        return buf_rsrc(reinterpret_cast<const void*>(uint64_t(hi) << 32 | lo),
                        __builtin_amdgcn_readfirstlane(abs(span) + bytes));
    }
    CB_DEV uint32_t first(int n) const { return uint32_t(max(0, -(n - 1) * st)); }
    CB_DEV uint32_t at(int row, int byte) const { return byte >= bytes ? kOOB : uint32_t(row) * uint32_t(st) + byte; }
    CB_DEV void next() { p += int64_t(kL) * st; }
};

// The piece's elements behind the row's last, which are the next ones' in memory, as zeros.
template <class T>
CB_DEV uint4 la_cut(uint4 v, int left) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) w[i] = 2 * i + 1 < left ? w[i] : 2 * i < left ? w[i] & 0xffffu : 0u;
        else w[i] = i < left ? w[i] : 0u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The same piece by its address, where the array's alignment or strides do not suit a buffer resource. The row's last piece
// goes element by element.
template <class T>
CB_DEV uint4 la_gather(const T* p, int left) {
    constexpr int VE = 16 / sizeof(T);
    if (left >= VE) {
        const la_u32x4 w = *reinterpret_cast<const la_u32x4*>(p);
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    T x[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) x[i] = i < left ? p[i] : T(0);
    uint4 v;
    __builtin_memcpy(&v, x, 16);
    return v;
}

// The same number, but for the compiler: what rare paths derive from it is not computed ahead of the main loop and kept in
// registers throughout (60 of them here).
CB_DEV int la_here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Row j's numbers from v's fragments at column col of the wave's 16: whichever lane holds it hands it over. j is the same
// in all lanes. (Selections instead of an index keep the fragments in registers.)
template <class Tr, int NJ>
CB_DEV float la_row_at(const typename Tr::Frag (&fv)[NJ], int j, int col) {
    float y = 0.f;
#pragma unroll
    for (int jb = 0; jb < NJ; ++jb) {
        float x[Tr::KPL];
        typename Tr::Frag f = fv[jb];
        asm volatile("" : "+v"(f.x), "+v"(f.y), "+v"(f.z), "+v"(f.w));   // unpacked here, not ahead of the rows' loop
        Tr::unpack(f, x);
#pragma unroll
        for (int u = 0; u < Tr::KPL; ++u) y = j / Tr::KB == jb && j % Tr::KPL == u ? x[u] : y;
    }
    return __shfl(y, j / Tr::KPL % 4 * 16 + col);
}

// Waves a SIMD is to hold: two of the whole pass's, four of the states' where their registers allow it without memory.
template <class Tr, int DK, bool STATE>
constexpr int la_simd_waves = STATE && DK <= 64 && sizeof(typename Tr::T) == 2 ? 4 : 2;

template <class Tr, int DK, int NW, bool STATE, bool FAST>
__global__ __launch_bounds__(64 * NW, (la_simd_waves<Tr, DK, STATE>)) void la_chunk_kernel(LaArgs a, LaSegs sg, int y0, int ny,
                                                                                          int blocks) {
    using T = typename Tr::T;
    using Frag = typename Tr::Frag;
    using L = LaTile<Tr, DK, NW, STATE>;
    constexpr int KB = Tr::KB, KPL = Tr::KPL, NT = DK / 16, NJ = kL / KB;
    // Float32 products of 16 contracted numbers take 128 cycles: those of padding only are passed over.
    constexpr bool SKIP = sizeof(T) == 4 && DK == 128;
    extern __shared__ __align__(16) unsigned char lds[];
    float* pw = reinterpret_cast<float*>(lds + L::TAB);
    float* pin = pw + 68 + 16;
    float* xw = pin + 68;      // [c_i = 0] out g^(i+l)
    float* vw = xw + kL;       // [c_j = c] in g^(n-l-j)
    uint64_t* starts = reinterpret_cast<uint64_t*>(vw + kL);   // bit i: an episode starts at row i

    // Workgroups go round the 8 XCDs one by one: those of the passes on one state, which read the same arrays, are 8 apart,
    // so they share an L2 at about the same time.
    // (Quotients come from vector instructions; as scalars again, what is addressed by them needs no loop over lanes.)
    auto quot = [](uint32_t x, uint32_t y) { return uint32_t(__builtin_amdgcn_readfirstlane(int(x / y))); };
    const uint32_t turn = blockIdx.x >> 3, turn_y = ny > 1 ? quot(turn, ny) : turn;
    const int y = y0 + int(turn - turn_y * ny);
    const uint32_t bid = turn_y * 8 + (blockIdx.x & 7);
    if (int(bid) >= blocks) return;
    const LaPass& P = a.pass[y];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;
    const uint32_t EH = uint32_t(a.E) * a.H;   // <= 2^21
    const int n0 = 16 * wave;                  // the wave's columns; the workgroup has all
    const int seg = sg.segs > 1 ? int(quot(bid, EH)) : 0;
    const uint32_t eh32 = bid - seg * EH, e32 = quot(eh32, a.H);
    const int64_t eh = eh32, e = e32, h = eh32 - e32 * a.H;
    const int p0 = seg * sg.chunks * kL;
    const int p1 = sg.segs == 1 ? a.T : int(min(int64_t(a.T), int64_t(p0) + int64_t(sg.chunks) * kL));

    const int64_t dir = P.back ? -1 : 1, t0 = P.back ? a.T - 1 - p0 : p0;
    const int dk = P.dk, dv = P.dv, back = P.back, vec = P.vec;
    const float out = P.out;
    auto rows = [&](const LaView& x, int d) {
        return LaRows{static_cast<const char*>(x.p) + (e * x.e + h * x.h + t0 * x.t) * L::ES, FAST ? int(dir * x.t) * L::ES : 0,
                      d * L::ES};
    };
    LaRows q = rows(P.q, dk), k = rows(P.k, dk), v = rows(P.v, dv), o = rows(P.o, dv);
    LaRows dn{reinterpret_cast<const char*>(a.dones + (a.dones ? e * a.d_e + t0 * a.d_t : 0)), a.dones ? int(dir * a.d_t) : 0,
              a.dones ? 1 : 0};
    const int later = back ? 0 : 1;

    // the chunk's q, k and v on their way to LDS: 16-byte pieces, 64 rows of CQ or CV of them
    constexpr int CQ = DK * L::ES / 16, CV = 16 * NW * L::ES / 16;
    uint4 rq[L::UQ], rk[L::UQ], rv[L::UV];
    uint32_t rd = 0;
    constexpr int RQ = 64 * NW / CQ, RV = 64 * NW / CV;   // rows from one of a thread's pieces to the next
    static_assert(RQ * CQ == 64 * NW && RV * CV == 64 * NW, "a thread's pieces lie in one column");
    const int rowq = tid / CQ, colq = tid % CQ * 16, rowv = tid / CV, colv = tid % CV * 16;
    const uint32_t atq = q.at(rowq, colq), atk = k.at(rowq, colq), atv = v.at(rowv, colv);
    auto fetch = [&](int n, int p) CB_INLINE_LAMBDA {   // rows p .. p + n - 1
        if (FAST) {
            const auto bq = q.rsrc(n), bk = k.rsrc(n), bv = v.rsrc(n);
#pragma unroll
            for (int u = 0; u < L::UQ; ++u) {
                if (!STATE) rq[u] = buf_load16(bq, atq + (q.first(n) + u * RQ * q.st));
                rk[u] = buf_load16(bk, atk + (k.first(n) + u * RQ * k.st));
            }
#pragma unroll
            for (int u = 0; u < L::UV; ++u) rv[u] = buf_load16(bv, atv + (v.first(n) + u * RV * v.st));
        } else {
            auto piece = [&](const LaView& x, int row, int col, int d) {
                const T* r = static_cast<const T*>(x.p) + e * x.e + h * x.h + (t0 + dir * (p - p0 + row)) * x.t + col;
                return la_gather<T>(r, row < n ? d - col : 0);
            };
#pragma unroll
            for (int u = 0; u < L::UQ; ++u) {
                if (!STATE) rq[u] = piece(P.q, rowq + RQ * u, colq / L::ES, dk);
                rk[u] = piece(P.k, rowq + RQ * u, colq / L::ES, dk);
            }
#pragma unroll
            for (int u = 0; u < L::UV; ++u) rv[u] = piece(P.v, rowv + RV * u, colv / L::ES, dv);
            if (wave == 0) rd = a.dones && lane < n ? a.dones[e * a.d_e + (t0 + dir * (p - p0 + lane)) * a.d_t] : 0;
        }
        // (Kept as it is loaded: a comparison here would wait for it and all loads before it.)
        if (FAST && wave == 0) rd = __builtin_amdgcn_raw_buffer_load_b8(dn.rsrc(n), uint32_t(lane * dn.st) + dn.first(n), 0, 0);
    };
    const bool tail = FAST && (vec & 2);
    const uint32_t ato = o.at(c, (n0 + 4 * g) * L::ES);
    const bool busy = n0 < dv;   // a wave behind the last column only moves rows and forms products
    fetch(min(kL, p1 - p0), p0);

    // X's numbers in a state: results m, rows krow(m, g, r), column n0 + c; what the state has not is zero, and not written.
    cb_f32x4 X[NT];
    const int xcol = n0 + c;
    auto state = [&](const float* x) {
        const uint64_t q = reinterpret_cast<uint64_t>(x + eh * dk * dv);
        return buf_rsrc(reinterpret_cast<const void*>(q), x ? uint32_t(dk * dv * 4) : 0u);
    };
    auto xat = [&](int kk, int xk, int xn) { return kk < dk && xcol < dv ? uint32_t(kk * xk + xcol * xn) * 4 : kOOB; };
    {
        const float* x = P.x0;
        int xk = P.xk, xn = P.xn;
        if (STATE) x = nullptr;
        else if (sg.segs > 1) { x = sg.state[y] + int64_t(seg) * EH * dk * dv; xk = dv; xn = 1; }
        const auto bx = state(x);
        if (xk == 1 && dk % 4 == 0) {
#pragma unroll
            for (int m = 0; m < NT; ++m) {
                const uint4 v = buf_load16(bx, xat(Tr::krow(m, g, 0), 1, xn));
                X[m] = cb_f32x4{__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
            }
        } else {
            // rows behind the last are behind the state's end where rows are its outer axis
            const uint32_t at = xat(Tr::krow(0, g, 0), xk, xn);
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t off = xk != dv ? xat(Tr::krow(m, g, r), xk, xn)
                                         : at == kOOB ? kOOB : at + Tr::krow(m, 0, r) * xk * 4;
                    X[m][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(bx, off, 0, 0));
                }
        }
    }

    if (tid < 16) pin[tid - 16] = 0.f;
    if (tid <= kL) {
        // exp(tid log g), the product's rounding error made good
        const float ld = a.log_decay[h], x = tid ? float(tid) * ld : 0.f, lo = fmaf(float(tid), ld, -x);
        float w = expf(x);
        w = tid && isfinite(x) ? fmaf(w, lo, w) : w;
        pw[tid] = w;
        pin[tid] = w * P.in * out;
    }
    if (!STATE && KB == 32) {   // products above the diagonal that a fragment of 32 rows takes along
        for (int u = tid; u < 2 * 16 * Tr::NP * 4; u += 64 * NW) {
            const int pl = u / (2 * 16 * 4), b = u / 64 % 2, i = u / 4 % 16, j = u % 4;
            *reinterpret_cast<uint2*>(lds + L::P + pl * L::PP + L::prow(32 * b + i) + (32 * b + 16 + 4 * j) * L::ES) =
                make_uint2(0, 0);
        }
    }

    lds_barrier();
    float factor = 1.f;
    for (int p = p0; p < p1; p += kL) {
        const int n = min(kL, p1 - p);
#pragma unroll
        for (int u = 0; u < L::UQ; ++u) {
            if (__builtin_expect(tail, 0)) {
                const int left = dk - la_here(colq) / L::ES;
                rq[u] = la_cut<T>(rq[u], left);
                rk[u] = la_cut<T>(rk[u], left);
            }
            if (rowq + RQ * u < kL) {
                if (!STATE) *reinterpret_cast<uint4*>(lds + L::Q + (rowq + RQ * u) * L::RSK + colq) = rq[u];
                *reinterpret_cast<uint4*>(lds + L::K + (rowq + RQ * u) * L::RSK + colq) = rk[u];
            }
        }
#pragma unroll
        for (int u = 0; u < L::UV; ++u) {
            if (__builtin_expect(tail, 0)) rv[u] = la_cut<T>(rv[u], dv - la_here(colv) / L::ES);
            *reinterpret_cast<uint4*>(lds + L::V + (rowv + RV * u) * L::RSV + colv) = rv[u];
        }
        // episode starts before what row i holds, of the chunk's starts m
        auto count_in = [&](uint64_t m, int i) {
            return __popcll(back ? m & ((uint64_t(1) << i) - 1) : m & (~uint64_t(0) >> (63 - i)));
        };
        if (wave == 0) {
            const uint64_t m = __ballot(rd != 0 && lane < n);
            const int ci = count_in(m, lane);
            xw[lane] = ci == 0 ? pw[lane + later] * out : 0.f;
            vw[lane] = lane < n && ci == __popcll(m) ? pw[n - later - lane] * P.in : 0.f;
            if (lane == 0) *starts = m;
        }
        const float over = pw[n];
        lds_barrier();
        const uint64_t ms = *starts;
        const uint64_t m = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(ms >> 32)))) << 32 |
                           uint32_t(__builtin_amdgcn_readfirstlane(int(ms)));
        auto count = [&](int i) { return count_in(m, i); };
        const int total = __popcll(m);
        if (STATE) factor = total || factor < 0.f ? -1.f : factor * over;
        q.next(); k.next(); v.next(); dn.next();
        if (p > p0) o.next();   // the chunk at hand's, to be written at its end
        if (p + kL < p1) fetch(min(kL, p1 - p - kL), p + kL);

        if (!STATE) {   // in out g^(i-j) q_i . k_j by tiles on and below the diagonal, a wave's few at once
            constexpr int MT = (10 + NW - 1) / NW;
            cb_f32x4 d[MT];
            float w[MT][4];
            int tb[MT], tt[MT];
#pragma unroll
            for (int y = 0; y < MT; ++y) {
                const int u = min(wave + NW * y, 9);
                tb[y] = u < 1 ? 0 : u < 3 ? 1 : u < 6 ? 2 : 3;
                tt[y] = u - tb[y] * (tb[y] + 1) / 2;
                d[y] = cb_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < 4; ++r) w[y][r] = pin[16 * (tb[y] - tt[y]) + c - 4 * g - r];   // zero above the diagonal
            }
#pragma unroll
            for (int kb = 0; kb < DK / KB; ++kb)
                if (!SKIP || kb * KB < dk)
#pragma unroll
                for (int y = 0; y < MT; ++y) {
                    const Frag fk = *reinterpret_cast<const Frag*>(lds + L::K + (16 * tt[y] + c) * L::RSK + kb * 64 + 16 * g);
                    const Frag fq = *reinterpret_cast<const Frag*>(lds + L::Q + (16 * tb[y] + c) * L::RSK + kb * 64 + 16 * g);
                    d[y] = Tr::mma(fk, fq, d[y]);
                }
#pragma unroll
            for (int y = 0; y < MT; ++y)
#pragma unroll
                for (int r = 0; r < 4; ++r) d[y][r] *= w[y][r];
            if (__builtin_expect(m != 0, 0)) {
#pragma unroll
                for (int y = 0; y < MT; ++y) {
                    const int ci = count(la_here(16 * tb[y] + c)), j0 = la_here(16 * tt[y] + 4 * g);
#pragma unroll
                    for (int r = 0; r < 4; ++r) d[y][r] = count(j0 + r) == ci ? d[y][r] : 0.f;
                }
            }
            // (Behind the tenth tile a wave repeats it: the same numbers in the same place.)
#pragma unroll
            for (int y = 0; y < MT; ++y)
                Tr::store_p(lds + L::P + L::prow(16 * tb[y] + c) + (16 * tt[y] + 4 * g) * L::ES, L::PP, d[y]);
        }

        __builtin_amdgcn_sched_barrier(0);
        if (!busy) { lds_barrier(); continue; }
        Frag fv[NJ];
#pragma unroll
        for (int jb = 0; jb < NJ; ++jb) fv[jb] = Tr::template cols<1>(lds + L::V, L::RSV, jb * KB, 16 * wave);

        cb_f32x4 O[4];
        if (!STATE) {   // X^T q, columns i
#pragma unroll
            for (int b = 0; b < 4; ++b) O[b] = cb_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < DK / KB; ++kb) {
                if (SKIP && kb * KB >= dk) break;
                Frag fx[Tr::NX], fq[4];
                Tr::xfrag(X, kb, fx);
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    fq[b] = *reinterpret_cast<const Frag*>(lds + L::Q + (16 * b + c) * L::RSK + kb * 64 + 16 * g);
                // (Neighbouring products go to different sums: one on another's result waits for it.)
#pragma unroll
                for (int u = 0; u < Tr::NX; ++u)
#pragma unroll
                    for (int b = 0; b < 4; ++b) O[b] = Tr::mma(fx[u], fq[b], O[b]);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) O[b] *= xw[16 * b + c];
            if (__builtin_expect(m != 0, 0)) {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (count(la_here(16 * b + c)) != 0) O[b] = cb_f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }

        __builtin_amdgcn_sched_barrier(0);
        {   // X <- over X + sum_j w_j k_j v_j^T
            cb_f32x4 U[NT];
            auto rows = [&](auto clean) CB_INLINE_LAMBDA {
#pragma unroll
                for (int t = 0; t < NT; ++t) U[t] = cb_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int jb = 0; jb < NJ; ++jb) {
                    float x[KPL];
                    Tr::unpack(clean(fv[jb]), x);
#pragma unroll
                    for (int u = 0; u < KPL; ++u) x[u] *= vw[jb * KB + KPL * g + u];
                    Frag fw[Tr::NV];
                    Tr::split(x, fw);
                    constexpr int TG = SKIP ? 2 : NT < 4 ? NT : 4;   // at a time
#pragma unroll
                    for (int t0 = 0; t0 < NT; t0 += TG) {
                        if (SKIP && t0 * 16 >= dk) break;
                        Frag fk[TG];
#pragma unroll
                        for (int t = 0; t < TG; ++t) fk[t] = clean(Tr::kcols(lds + L::K, L::RSK, jb * KB, t0 + t));
#pragma unroll
                        for (int u = Tr::NV - 1; u >= 0; --u)
#pragma unroll
                            for (int t = 0; t < TG; ++t) U[t0 + t] = Tr::mma(fk[t], fw[u], U[t0 + t]);
                    }
                }
            };
            rows([](Frag f) { return f; });
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) sum = fmaf(U[t][0], U[t][1], fmaf(U[t][2], U[t][3], sum));
            // A number that is not finite comes through a weight of zero as NaN. Then without all such, and theirs added
            // for the rows that the state sees.
            if (__builtin_expect(__any(sum != sum), 0)) {
                asm volatile("" ::: "memory");   // the fragments are read again, not kept for this
                rows([](Frag f) { return Tr::finite(f); });
                const int cc = la_here(c), gg = la_here(g);
#pragma unroll 1
                for (int j = 0; j < n; ++j) {
                    const float x = la_row_at<Tr>(fv, j, cc), w = vw[j] * x;
                    if (count(j) != total) continue;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float kk = Tr::load(*reinterpret_cast<const T*>(lds + L::K + j * L::RSK +
                                                                                  Tr::krow(t, gg, r) * L::ES));
                            if (!isfinite(x) || !isfinite(kk)) U[t][r] += w * kk;
                        }
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) X[t][r] = (total ? 0.f : over * X[t][r]) + U[t][r];
        }
        lds_barrier();

        if (!STATE) {   // sum over j of the products with v
            cb_f32x4 A[4];
            auto rows = [&](auto clean) CB_INLINE_LAMBDA {
#pragma unroll
                for (int b = 0; b < 4; ++b) A[b] = cb_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int jb = 0; jb < NJ; ++jb)
#pragma unroll
                    for (int u = Tr::NP - 1; u >= 0; --u) {
                        Frag fp[4];
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            if (jb * KB <= 16 * b + 15)
                                fp[b] = *reinterpret_cast<const Frag*>(lds + L::P + u * L::PP + L::prow(16 * b + c) +
                                                                       jb * 64 + 16 * g);
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            if (jb * KB <= 16 * b + 15) A[b] = Tr::mma(clean(fv[jb]), clean(fp[b]), A[b]);
                    }
            };
            rows([](Frag f) { return f; });
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < 4; ++b) sum = fmaf(A[b][0], A[b][1], fmaf(A[b][2], A[b][3], sum));
            if (__builtin_expect(__any(sum != sum), 0)) {   // as above: a later row's, or one's of another episode
                asm volatile("" ::: "memory");
                rows([](Frag f) { return Tr::finite(f); });
                const int cc = la_here(c), gg = la_here(g);
#pragma unroll 1
                for (int j = 0; j < n; ++j) {
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = la_row_at<Tr>(fv, j, 4 * gg + r);
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const int i = 16 * b + cc;
                        if (j > i || count(j) != count(i)) continue;
                        float w = 0.f;
#pragma unroll
                        for (int u = 0; u < Tr::NP; ++u)
                            w += Tr::load(*reinterpret_cast<const T*>(lds + L::P + u * L::PP + L::prow(i) + j * L::ES));
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (!isfinite(x[r]) || !isfinite(w)) A[b][r] += w * x[r];
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) O[b][r] += A[b][r];
            if constexpr (FAST) {
                const auto bo = o.rsrc(n);
                const uint32_t f = o.first(n);
                if (__builtin_expect(vec & 1, 1)) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) Tr::store4o(bo, ato + (f + 16 * b * o.st), O[b]);
                } else {
                    const int left = dv - la_here(n0 + 4 * g);
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            Tr::store1o(bo, r < left ? ato + (f + 16 * b * o.st + r * L::ES) : kOOB, O[b][r]);
                }
            } else {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int i = la_here(16 * b + c), col = la_here(n0 + 4 * g);
                    if (i >= n) continue;
                    T* po = static_cast<T*>(const_cast<void*>(P.o.p)) + e * P.o.e + h * P.o.h +
                            (t0 + dir * (p - p0 + i)) * P.o.t;
                    if (col + 4 <= dv) {
                        Tr::store4(po + col, O[b]);
                        continue;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (col + r < dv) po[col + r] = Tr::store(O[b][r]);
                }
            }
        }
    }

    float* x = STATE ? sg.state[y] + int64_t(seg) * EH * dk * dv : seg == sg.segs - 1 ? P.x1 : nullptr;
    if (x) {
        const int xk = STATE ? dv : P.xk, xn = STATE ? 1 : P.xn;
        const auto bx = state(x);
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(X[m][r]), bx, xat(Tr::krow(m, g, r), xk, xn), 0, 0);
    }
    if (STATE && tid == 0) sg.factor[y][int64_t(seg) * EH + eh] = factor;
}

// The states before the segments, in place of their contributions.
__global__ __launch_bounds__(256) void la_scan_kernel(LaArgs a, LaSegs sg) {
    const LaPass& P = a.pass[blockIdx.y];
    const int64_t EH = int64_t(a.E) * a.H, S = int64_t(P.dk) * P.dv, i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= EH * S) return;
    const int64_t eh = i / S;
    const int kn = int(i - eh * S);
    float x = P.x0 ? P.x0[eh * S + int64_t(kn / P.dv) * P.xk + int64_t(kn % P.dv) * P.xn] : 0.f;
    float* st = sg.state[blockIdx.y] + i;
    const float* f = sg.factor[blockIdx.y] + eh;
    for (int s = 0; s + 1 < sg.segs; ++s) {
        const float u = st[s * EH * S], w = f[s * EH];
        st[s * EH * S] = x;
        x = (w < 0.f ? 0.f : w * x) + u;
    }
    st[(sg.segs - 1) * EH * S] = x;
}

template <class Tr, int DK, int NW>
hipError_t la_chunks_launch(const LaArgs& a, const LaSegs& sg, int y0, int ny, bool state, hipStream_t s) {
    // A workgroup has a state of its own, all columns (16 NW >= dv, by la_waves), so a state may go through in place.
    const int blocks = int(int64_t(a.E) * a.H * (state ? sg.segs - 1 : sg.segs));
    const dim3 grid(unsigned((blocks + 7) / 8 * 8 * ny));
    bool fast = true;
    for (int y = y0; y < y0 + ny; ++y) fast &= a.pass[y].vec >> 2 & 1;
    const int lds = state ? LaTile<Tr, DK, NW, true>::BYTES : LaTile<Tr, DK, NW, false>::BYTES;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64 * NW), lds, s, a, sg, y0, ny, blocks); };
    if (state) fast ? go(la_chunk_kernel<Tr, DK, NW, true, true>) : go(la_chunk_kernel<Tr, DK, NW, true, false>);
    else fast ? go(la_chunk_kernel<Tr, DK, NW, false, true>) : go(la_chunk_kernel<Tr, DK, NW, false, false>);
    return hipGetLastError();
}

int la_dim(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }
// Waves of a workgroup, 16 columns each. Float32 rows of 128 take eight whatever the columns, to move the rows.
int la_waves(int prec, int dk, int dv) { return prec == 1 && la_dim(dk) == 128 ? 8 : la_dim(dv) / 16; }

template <class Tr, int DK>
hipError_t la_chunks_nw(const LaArgs& a, const LaSegs& sg, int y0, int ny, bool state, hipStream_t s) {
    if constexpr (!(sizeof(typename Tr::T) == 4 && DK == 128)) {
        switch (la_waves(sizeof(typename Tr::T) == 4, DK, a.pass[y0].dv)) {
            case 2: return la_chunks_launch<Tr, DK, 2>(a, sg, y0, ny, state, s);
            case 4: return la_chunks_launch<Tr, DK, 4>(a, sg, y0, ny, state, s);
        }
    }
    return la_chunks_launch<Tr, DK, 8>(a, sg, y0, ny, state, s);
}

// Passes whose kernels are the same go in one launch.
template <class Tr>
hipError_t la_chunks(const LaArgs& a, const LaSegs& sg, bool state, hipStream_t s) {
    for (int y = 0, ny; y < a.np; y += ny) {
        for (ny = 1; y + ny < a.np && la_dim(a.pass[y + ny].dk) == la_dim(a.pass[y].dk) &&
                     la_dim(a.pass[y + ny].dv) == la_dim(a.pass[y].dv); ++ny) {}
        hipError_t e;
        switch (la_dim(a.pass[y].dk)) {
            case 32: e = la_chunks_nw<Tr, 32>(a, sg, y, ny, state, s); break;
            case 64: e = la_chunks_nw<Tr, 64>(a, sg, y, ny, state, s); break;
            default: e = la_chunks_nw<Tr, 128>(a, sg, y, ny, state, s); break;
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Segments of the rollout that run at once: as many as fill the chip's places for workgroups once, of four chunks at
// least. Each segment's state has to be known first, which reads k and v again and takes two launches more: less than
// three segments gain nothing. (16384 x 2 envs x 8 heads of 128: 16 chains of 256 chunks, which take 5.6 us each;
// in 16 segments 138 us in all.)
int la_segs(int prec, int T, int64_t EH, int dk, int dv, int passes, int* chunks) {
    const int64_t nc = (int64_t(T) + kL - 1) / kL;
    *chunks = int(nc);
    if (EH == 0) return 1;
    // passes of a launch: of the backward's three, the two that contract over v's axis, or all where the kernels are one
    const int together = passes > 1 ? (la_dim(dk) == la_dim(dv) ? 3 : 2) : 1, out = passes > 1 ? dk : dv;
    const int waves = la_waves(prec, passes > 1 ? dv : dk, out);
    const int64_t chains = EH * together, places = 256 * (8 / waves);   // a CU holds 8 waves
    const int64_t want = std::min(places / chains, nc / 4);
    if (want < 3) return 1;
    *chunks = int((nc + want - 1) / want);
    return int((nc + *chunks - 1) / *chunks);
}

int64_t la_a256(int64_t b) { return (b + 255) / 256 * 256; }

// No rows: the state goes through (a gradient too: nothing is between the two).
__global__ void la_empty_kernel(const float* x0, float* x1, int64_t n) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
        x1[i] = x0 ? x0[i] : 0.f;
}

}  // namespace

size_t linattn_ws_bytes(int prec, int T, int E, int H, int dk, int dv, int passes) {
    int chunks;
    const int64_t EH = int64_t(E) * H, segs = la_segs(prec, T, EH, dk, dv, passes, &chunks);
    if (segs == 1) return 0;
    return size_t(passes * (la_a256(segs * EH * dk * dv * 4) + la_a256(segs * EH * 4)));
}

hipError_t linattn(int prec, LaArgs a, void* ws, hipStream_t s) {
    if (int64_t(a.E) * a.H == 0) return hipSuccess;
    if (a.T == 0) {
        for (int y = 0; y < a.np; ++y) {
            const LaPass& P = a.pass[y];
            const int64_t n = int64_t(a.E) * a.H * P.dk * P.dv;
            if (!P.x1 || P.x1 == P.x0) continue;
            const int64_t blocks = std::min<int64_t>((n + 255) / 256, 4096);
            ProfScope ps(s, [&] { return "linattn_state/" + std::to_string(n); });
            hipLaunchKernelGGL(la_empty_kernel, dim3(unsigned(blocks)), dim3(256), 0, s, P.x0, P.x1, n);
        }
        return hipGetLastError();
    }
    ProfScope ps(s, [&] {
        return cb_key("linattn", prec, std::to_string(a.T) + "x" + std::to_string(a.E) + "x" + std::to_string(a.H) + "x" +
                                           cb_dims(a.pass[0].dk, a.pass[0].dv) + (a.np > 1 ? "/bwd" : ""));
    });
    if (a.T == 1 && a.np == 1) return prec == 0 ? la_step<PrecBF16>(a, s) : la_step<PrecF32>(a, s);
    const int es = prec == 0 ? 2 : 4, ve = 16 / es;
    // Rows that a buffer resource reaches: of whole words (it ends with the last row's last one), each behind the last
    // one's end, not too far apart. (Others go by their addresses: 128 x 1024 envs x 8 heads of 64, bf16, in rows of 50 MB
    // forward 213 us, contiguous 211; 128 x 512 x 8 heads of 33 x 71 forward 287, backward 812, of 34 x 70 241 and 522.)
    auto reach = [&](const LaView& v, int d) {
        const int k = 4 / es;
        return reinterpret_cast<uintptr_t>(v.p) % 4 == 0 && d % k == 0 && v.t % k == 0 && v.e % k == 0 && v.h % k == 0 && v.t >= d &&
               v.t <= kLaReach / es;
    };
    LaSegs sg{};
    const int64_t EH = int64_t(a.E) * a.H;
    const LaPass& last = a.pass[a.np - 1];   // the one whose axes are k's and v's, in either direction
    sg.segs = la_segs(prec, a.T, EH, last.dk, last.dv, a.np, &sg.chunks);
    char* w = static_cast<char*>(ws);
    for (int y = 0; y < a.np; ++y) {
        LaPass& P = a.pass[y];
        P.vec = (P.dv % 4 == 0) | (P.dk % ve != 0 || P.dv % ve != 0) << 1 |
                (reach(P.q, P.dk) && reach(P.k, P.dk) && reach(P.v, P.dv) && reach(P.o, P.dv) && a.d_t <= kLaReach) << 2;
        if (sg.segs == 1) continue;
        sg.state[y] = reinterpret_cast<float*>(w);
        w += la_a256(sg.segs * EH * P.dk * P.dv * 4);
        sg.factor[y] = reinterpret_cast<float*>(w);
        w += la_a256(sg.segs * EH * 4);
    }
    auto run = [&](bool state) { return prec == 0 ? la_chunks<LaB>(a, sg, state, s) : la_chunks<LaF>(a, sg, state, s); };
    if (sg.segs > 1) {
        hipError_t e = run(true);
        if (e != hipSuccess) return e;
        const int64_t n = EH * a.pass[0].dk * a.pass[0].dv;
        hipLaunchKernelGGL(la_scan_kernel, dim3(unsigned((n + 255) / 256), unsigned(a.np)), dim3(256), 0, s, a, sg);
    }
    return run(false);
}

}  // namespace cb
