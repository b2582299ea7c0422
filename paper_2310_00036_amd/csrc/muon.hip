// Orthogonalised updates: Newton-Schulz products on gfx950 matrix cores, and the Muon step over the
// flat parameter buffer that they serve.
//
// One Newton-Schulz step is X <- (a I + b A + c A^2) X with A = X X^T on the smaller side m <= n. The
// factors of all steps are polynomials of the first Gram matrix, so a segment of L steps needs X twice:
//   A = X X^T;  per step  P = a I + b A + c A^2,  Q <- P Q,  A <- P A P;  then X <- Q X,
// 3 m^2 n + (4 L - 3) m^3 operations with the symmetric products computed by halves, against
// L (3 m^2 n + m^3) for the steps one by one. What bounds L is rounding: A squares the singular values
// and P A P grows what is small by a^2 a step, the rounding of A along with it. A's error is 2^-24 of
// its norm, so the next segment starts from a fresh Gram matrix. Five steps on gradient-like matrices
// (a few strong directions over noise) are off by 0.7e-6 to 2.8e-6 of their norm with segments of 2, 2 and 1
// steps (kSegF32: float32 matrices and muon_step), where the steps one by one in float32 are by 1e-6 to 2e-6
// (at most twice theirs on one matrix). With 3 and 2 (kSegBf16) they are off by 2e-6 to 14e-6, which bf16
// results, at 1.7e-3 from their own rounding, do not see; one segment of 5 is off by 2^-7 for singular values
// spread over six decades, more than bf16 resolves.
// On square matrices the operations are the same either way; on 15 : 1 they are 1 : 1.4.
//
// Every matrix is held as two f16 planes, v = hi + lo with lo = f16(v - hi): 22 bits and more under a
// power-of-two scale that keeps values in f16's normal range (at least 2^-40 of a matrix's bound is
// resolved). A product is hi hi + hi lo + lo hi in f16 MFMAs with float32 accumulation, at a third of
// the f16 rate, where float32 MFMAs are issued at a sixteenth (large library products: 0.153 of 1.49
// PFLOP/s, a tenth); what it drops, lo lo, is 2^-22 of a product at most. bf16 inputs take one plane: their
// 8 bits are exact under a power-of-two scale, but for elements below 2^-17 of the root mean square, which
// f16 holds to 2^-25 of it; so they need one product in the Gram matrix and two with Q.
// Sums of squares, norms and the clip are 64 bits.
//
// Launches of a pass: sums of squares; planes of X (for muon_step with the momentum update and Adam
// for the rest); and per segment the Gram product (split over k), its sum, the m x m products, and
// Q X, whose last form writes the result or the updated parameters. Matrices of up to 64 on the
// smaller side have their whole m x m part in one workgroup's LDS, in float32, inside the launch that
// sums the others' Gram partials. All matrices of a call go through the same launches. Small matrices
// of muon_orthogonalize do without all that: one launch, a workgroup each (ns_one_kernel).
//
// What bounds a call: up to m = 512 or so the latency of its 20 launches, 4 to 8 us each (3872 x 256
// float32 119 us, its bytes 2 us and its products 2 at the f16 rate; the base net's muon_step 137 us);
// from there on the tile product (4096 x 4096 bf16 3.55 ms, 390 TFLOP/s of the result's operations,
// 1.2 PFLOP/s of f16 products where a large library product of f16 matrices reaches 1.49).
#include "common.h"
#include "kernels.h"
#include "muon.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>
#include <vector>

namespace cb {

namespace {

constexpr int kSegF32 = 2, kSegBf16 = 3, kMaxSegs = kNsMaxSteps / 2;
// What the tile rules count workgroups against. Not the current device's number: the layout of a workspace
// follows from the rules, and its size is asked for without a device. On fewer they are slower, not wrong.
constexpr int kNsCus = 256;
constexpr float kNsDefault[3] = {3.4445f, -4.7750f, 2.0315f};

typedef _Float16 ns_f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 ns_f16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t ns_u32x4 __attribute__((ext_vector_type(4)));

CB_DEV cb_f32x4 ns_mma(uint4 a, uint4 b, cb_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(ns_f16x8, a), __builtin_bit_cast(ns_f16x8, b), c,
                                                  0, 0, 0);
}

// Four values to their planes. Each value is made final first: joined with the product that formed it,
// its conversion would round once where the difference takes the twice rounded hi, and the two planes
// would miss an f16 step of each other now and then.
CB_DEV void ns_split(const float (&v)[4], uint2& hi, uint2& lo) {
    ns_f16x4 h, l;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float x = v[r];
        asm("" : "+v"(x));
        h[r] = static_cast<_Float16>(x);
        l[r] = static_cast<_Float16>(x - static_cast<float>(h[r]));
    }
    hi = __builtin_bit_cast(uint2, h);
    lo = __builtin_bit_cast(uint2, l);
}
CB_DEV void ns_join(uint2 hi, uint2 lo, float (&v)[4]) {
    const ns_f16x4 h = __builtin_bit_cast(ns_f16x4, hi), l = __builtin_bit_cast(ns_f16x4, lo);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = static_cast<float>(h[r]) + static_cast<float>(l[r]);
}

// A matrix of two planes is stored in blocks of 32 columns: a row's 32 hi, then its 32 lo, so that what a
// tile loads of a row for one step of the products is one 128-byte line. ns_at: the byte offset of (row,
// col)'s hi; its lo is 64 bytes on. A matrix of one plane is row-major.
constexpr int kLo = 64;
CB_DEV int64_t ns_at(int row, int col, int ld) { return (int64_t(row) * ld + (col & ~31)) * 4 + (col & 31) * 2; }
// Four neighbours of a row (four-aligned), or one below the other.
CB_DEV void ns_store(char* d, int row, int col, int ld, uint2 hi, uint2 lo) {
    char* p = d + ns_at(row, col, ld);
    *reinterpret_cast<uint2*>(p) = hi;
    *reinterpret_cast<uint2*>(p + kLo) = lo;
}
CB_DEV void ns_store_across(char* d, int row, int col, int ld, uint2 hi, uint2 lo) {
    const uint16_t h[4] = {uint16_t(hi.x), uint16_t(hi.x >> 16), uint16_t(hi.y), uint16_t(hi.y >> 16)};
    const uint16_t l[4] = {uint16_t(lo.x), uint16_t(lo.x >> 16), uint16_t(lo.y), uint16_t(lo.y >> 16)};
    char* p = d + ns_at(row, col, ld);
#pragma unroll
    for (int r = 0; r < 4; ++r, p += int64_t(ld) * 4) {
        *reinterpret_cast<uint16_t*>(p) = h[r];
        *reinterpret_cast<uint16_t*>(p + kLo) = l[r];
    }
}

// This workgroup's group; blk becomes its index within the group.
CB_DEV int ns_group(const NsArgs& a, int& blk) {
    int g = 0;
    while (g + 1 < a.ng && blk >= a.start[g + 1]) ++g;
    blk -= a.start[g];
    return g;
}
CB_DEV int64_t ns_offset(const NsArgs& a, const NsGroup& G, int b) {
    return G.table ? a.off[G.table - 1 + b] : int64_t(b) * G.rows * G.cols;
}
// Tile t of the lower triangle, row by row.
CB_DEV void ns_tile(int t, int& ti, int& tj) {
    ti = 0;
    while (t > ti) { t -= ti + 1; ++ti; }
    tj = t;
}

// Workgroups go to the eight XCDs in turn. The one of n that works on item `blk` so that each XCD has its
// items in one run, and (ns_tile_near) neighbouring items share panels of the operands in its L2.
CB_DEV int ns_xcd(int blk, int n) {
    const int x = blk & 7, q = n >> 3, r = n & 7;
    return x * q + min(x, r) + (blk >> 3);
}
// Tile t of the lower triangle of T x T, in bands of kNear rows, column by column.
constexpr int kNear = 6, kWide = 8;
CB_DEV void ns_tile_near(int t, int T, int& ti, int& tj) {
    int r = 0, h;
    for (;; r += h) {
        h = min(kNear, T - r);
        const int count = h * r + h * (h + 1) / 2;
        if (t < count) break;
        t -= count;
    }
    if (t < h * r) {
        tj = t / h;
        ti = r + t % h;
        return;
    }
    t -= h * r;
    int d = 0;
    while (t >= h - d) t -= h - d++;
    tj = r + d;
    ti = tj + t;
}

// ------------------------------------------------------------------ the tile product
//
// acc += A B^T over k in [k0, k1) for a BT x BT tile, in NsWaves' waves. An operand is a padded matrix
// [rows][k] of NP planes, leading dimension ld elements; padding is zero, so there are no edges. Tiles go
// from memory into an LDS ring of ST stages by direct loads that stay in flight across barriers (one wait
// per stage, counted), in the layout they have in memory; 16-byte slots are permuted within a row so that
// a fragment read meets every bank. A product of 4224 x 4224 planes (253 tiles of 192, one a CU) takes 195
// us; on zeros, which draw less power, 160, and of these 142 without its loads, 139 without its matrix
// instructions: both pipes are near their ends, and finer interleaving of the two brought nothing.

// 16 bytes a lane to LDS at lds + 16 lane. Inline so that the compiler, which cannot tell a ring's
// stages apart, does not wait for every load in flight before an LDS read; the waits are written out.
// (The s_nop is the wait state between the write of m0 and its use. Nothing else here uses m0, which
// the compiler keeps out of its allocation.)
CB_DEV void ns_dma16(ns_u32x4 rsrc, uint32_t lds, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(off), "s"(rsrc) : "memory");
}
template <int N>
CB_DEV void ns_wait() {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
CB_DEV ns_u32x4 ns_rsrc(const char* base, int64_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    // (uniform, and said to be: it goes into scalar registers)
    return ns_u32x4{uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(p)))),
                    uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(p >> 32)))),
                    uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(bytes)))), 0x00020000u};
}
CB_DEV uint32_t ns_lds(const unsigned char* p) { return uint32_t(reinterpret_cast<uintptr_t>((lds_t*)(p))); }

// Waves of a tile: WM x WN of them, FM x FN fragments of 16 each. What a wave reads of LDS per product
// falls with its fragments: at 4 x 4 (tiles of 128) reads and the incoming loads take as long as the
// products, at 6 x 6 (tiles of 192, one workgroup a CU) two thirds of that.
template <int BT>
struct NsWaves {
    static constexpr int WM = 2, WN = 2, NW = WM * WN;
    static constexpr int FM = BT / WM / 16, FN = BT / WN / 16;
};

// The rows of a tile that fragment i, j of the two operands hold (r: 0 .. 15). Any order gives the same
// products; with this one a lane's results of two neighbouring fragments are eight neighbours along M, and
// two along N, so that it writes 16 bytes of a row at once and 4 of a mirrored one.
template <int BT>
CB_DEV int ns_row_a(int i, int r) { return BT == 32 ? r : i / 2 * 32 + (r >> 2) * 8 + (i & 1) * 4 + (r & 3); }
template <int BT>
CB_DEV int ns_row_b(int j, int r) { return BT == 32 ? r : j / 2 * 32 + r * 2 + (j & 1); }

template <int BT, int BK, int NP>
struct NsOperand {
    static constexpr int NW = NsWaves<BT>::NW;
    static constexpr int RB = BK * NP * 2;                 // bytes of a tile row
    static constexpr int BYTES = BT * RB;
    static constexpr int NI = BYTES / (1024 * NW);         // direct loads a wave
    static constexpr int SPR = RB / 16;                    // 16-byte slots per row
    static_assert(BYTES % (1024 * NW) == 0, "whole loads");
    static_assert(BT != 32 || RB != 64, "key would depend on r0");
    uint32_t base[NI];
    // Chunk c of row r is in slot c ^ key(r), or, where two rows share 128 bytes, half of them in the other's
    // place. key: eight lanes of a fragment read meet eight slots, with the rows that ns_row_a and ns_row_b give
    // them (of the bits r0 .. r4 of a row they vary r0, r1, r3 and r1, r2, r3; in tiles of 32 r0, r1, r2).
    static CB_DEV int key(int r) {
        const int hi = (RB == 64 ? 0 : r << 2) ^ r, lo = BT == 32 ? r >> 2 : r >> 3;
        return BT == 32 ? r & 7 : (hi & 4) | (r & 2) | (lo & 1);
    }
    static CB_DEV int slot(int r, int c) {   // in 16 bytes from the tile's start
        return RB == 64 ? (r >> 1) * 8 + ((((r & 1) << 2) | c) ^ key(r)) : r * SPR + (c ^ key(r));
    }
    CB_DEV NsOperand(int ld, int row0, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int s = (wave + NW * i) * 64 + lane;
            int r, c;
            if (RB == 64) {   // (key does not depend on r0)
                const int e = (s & 7) ^ key(s >> 3 << 1);
                r = (s >> 3 << 1) + (e >> 2);
                c = e & 3;
            } else {
                r = s / SPR;
                c = (s % SPR) ^ key(r);
            }
            base[i] = uint32_t(row0 + r) * uint32_t(ld) * (NP * 2u) + uint32_t(c * 16);
        }
    }
    // this wave's load i of a tile at k
    CB_DEV void issue(int i, ns_u32x4 rs, uint32_t lds, int k, bool live, int wave) const {
        ns_dma16(rs, lds + (wave + NW * i) * 1024, live ? base[i] + uint32_t(k) * (NP * 2u) : kOOB);
    }
    // plane p's 8 consecutive k (step ks of 32, lane group g) of tile row `row`
    static CB_DEV uint4 frag(const unsigned char* t, int p, int row, int ks, int lane) {
        return *reinterpret_cast<const uint4*>(t + slot(row, (ks * NP + p) * 4 + (lane >> 4)) * 16);
    }
};

template <int BT, int BK, int ST, int NA, int NB>
constexpr int ns_lds_bytes() { return ST * (NA + NB) * BT * BK * 2; }

template <int BT>
using NsAcc = cb_f32x4[NsWaves<BT>::FM][NsWaves<BT>::FN];

template <int BT>
CB_DEV void ns_clear(NsAcc<BT>& acc) {
#pragma unroll
    for (int i = 0; i < NsWaves<BT>::FM; ++i)
#pragma unroll
        for (int j = 0; j < NsWaves<BT>::FN; ++j) acc[i][j] = cb_f32x4{0.f, 0.f, 0.f, 0.f};
}

// CROSS: the products with a lo plane are summed apart from the hi hi ones and added at the end. The matrix
// cores seem to cut off what a sum cannot hold rather than round it (a model of sums so cut has the errors
// measured here, one of rounded sums a third of them), and so a third as many additions to the large sum leave
// less of that bias. It matters in the m x m chain, whose errors the later products multiply: ns_cross.
template <int BT, int BK, int ST, int NA, int NB, bool CROSS = false>
CB_DEV void ns_gemm(const char* A, int64_t abytes, int lda, int arow, const char* B, int64_t bbytes, int ldb, int brow,
                    int k0, int k1, unsigned char* smem, NsAcc<BT>& acc) {
    using W = NsWaves<BT>;
    constexpr int FM = W::FM, FN = W::FN, KS = BK / 32;
    using OA = NsOperand<BT, BK, NA>;
    using OB = NsOperand<BT, BK, NB>;
    constexpr int STAGE = OA::BYTES + OB::BYTES, LPS = OA::NI + OB::NI;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, wm = wave / W::WN, wn = wave % W::WN;
    const OA oa(lda, arow, wave, lane);
    const OB ob(ldb, brow, wave, lane);
    const ns_u32x4 ra = ns_rsrc(A, abytes), rb = ns_rsrc(B, bbytes);
    const uint32_t lds0 = ns_lds(smem);
    const int nb = (k1 - k0) / BK;
    // this wave's load d of stage `it`; past the end it is out of range (zeros), so every stage counts the same
    auto issue = [&](int it, int d) CB_INLINE_LAMBDA {
        const uint32_t l = lds0 + uint32_t(it % ST) * STAGE;
        if (d < OA::NI) oa.issue(d < OA::NI ? d : 0, ra, l, k0 + it * BK, it < nb, wave);
        else ob.issue(d < OA::NI ? 0 : d - OA::NI, rb, l + OA::BYTES, k0 + it * BK, it < nb, wave);
    };
    auto read_a = [&](int st, int p, int ks, int i) CB_INLINE_LAMBDA {
        return OA::frag(smem + (st % ST) * STAGE, p, wm * (FM * 16) + ns_row_a<BT>(i, r16), ks, lane);
    };
    auto read_b = [&](int st, int p, int ks, int j) CB_INLINE_LAMBDA {
        return OB::frag(smem + (st % ST) * STAGE + OA::BYTES, p, wn * (FN * 16) + ns_row_b<BT>(j, r16), ks, lane);
    };
    // x y row by row; with(ks, i) before row i of step ks: reads and loads go between the products, for
    // one block of either would hold the matrix core up
    auto mul = [&](NsAcc<BT>& sum, const uint4 (&x)[KS][FM], const uint4 (&y)[KS][FN], auto&& with) CB_INLINE_LAMBDA {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                with(ks, i);
#pragma unroll
                for (int j = 0; j < FN; ++j) sum[i][j] = ns_mma(x[ks][i], y[ks][j], sum[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    static_assert(FM == FN, "a row's reads are one fragment of each operand");
    // The barrier stands before a stage's last product, whose operands are in registers by then: after it
    // the stage's buffer is free, the next stage is in LDS, and its first fragments are read in the first
    // half of that product; the others are read during the products before. No product waits for LDS. The
    // freed buffer's loads are issued half in that product and half in the next stage's first one.
    constexpr int R = KS * FM, HALF = NA > 1 || NB > 1 ? LPS / 2 : LPS;
    NsAcc<BT> apart;
    if constexpr (CROSS) ns_clear<BT>(apart);
    NsAcc<BT>& cross = CROSS ? apart : acc;
    uint4 a0[KS][FM], b0[KS][FN], a1[KS][FM], b1[KS][FN], na[KS][FM], nbf[KS][FN];
    for (int s = 0; s < ST - 1; ++s)
#pragma unroll
        for (int d = 0; d < LPS; ++d) issue(s, d);
#pragma unroll
    for (int d = 0; d < HALF; ++d) issue(ST - 1, d);
    ns_wait<(ST - 2) * LPS + HALF>();   // this wave's loads of stage 0 are in LDS
    lds_barrier();                      // all waves' are
#pragma unroll
    for (int q = 0; q < R; ++q) {
        a0[q / FM][q % FM] = read_a(0, 0, q / FM, q % FM);
        b0[q / FM][q % FM] = read_b(0, 0, q / FM, q % FM);
    }
    auto stage = [&](int it, uint4 (&x0)[KS][FM], uint4 (&y0)[KS][FN], uint4 (&nx)[KS][FM], uint4 (&ny)[KS][FN]) CB_INLINE_LAMBDA {
        if constexpr (NA > 1 || NB > 1)
            mul(acc, x0, y0, [&](int ks, int i) CB_INLINE_LAMBDA {
                if constexpr (NB > 1) b1[ks][i] = read_b(it, 1, ks, i);
                else a1[ks][i] = read_a(it, 1, ks, i);
                const int at = ks * FM + i;
#pragma unroll
                for (int d = HALF + at * (LPS - HALF) / R; d < HALF + (at + 1) * (LPS - HALF) / R; ++d) issue(it + ST - 1, d);
            });
        if constexpr (NA > 1 && NB > 1)
            mul(cross, x0, b1, [&](int ks, int i) CB_INLINE_LAMBDA { a1[ks][i] = read_a(it, 1, ks, i); });
        ns_wait<(ST - 2) * LPS>();
        lds_barrier();
        mul(NA > 1 || NB > 1 ? cross : acc, NA > 1 ? a1 : x0, NA > 1 ? y0 : NB > 1 ? b1 : y0, [&](int ks, int i) CB_INLINE_LAMBDA {
            const int at = ks * FM + i;
#pragma unroll
            for (int q = 2 * at; q < 2 * at + 2; ++q)
                if (q < R) {
                    nx[q / FM][q % FM] = read_a(it + 1, 0, q / FM, q % FM);
                    ny[q / FM][q % FM] = read_b(it + 1, 0, q / FM, q % FM);
                }
#pragma unroll
            for (int d = at * HALF / R; d < (at + 1) * HALF / R; ++d) issue(it + ST, d);
        });
    };
    for (int it = 0; it < nb; ++it) {
        stage(it, a0, b0, NA > 1 && NB > 1 ? a0 : na, nbf);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if constexpr (!(NA > 1 && NB > 1)) a0[ks][i] = na[ks][i];
                b0[ks][i] = nbf[ks][i];
            }
    }
    ns_wait<0>();
    lds_barrier();
    if constexpr (CROSS)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] += apart[i][j][e];
}

// f(M, N, acc[i][j], i, j) for every group of four rows M .. M+3 of column N that this lane holds (local).
template <int BT, class Fn>
CB_DEV void ns_each(NsAcc<BT>& acc, Fn&& f) {
    using W = NsWaves<BT>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = lane >> 4, r16 = lane & 15, wm = wave / W::WN, wn = wave % W::WN;
#pragma unroll
    for (int i = 0; i < W::FM; ++i)
#pragma unroll
        for (int j = 0; j < W::FN; ++j)
            f(wm * (W::FM * 16) + ns_row_a<BT>(i, 4 * g), wn * (W::FN * 16) + ns_row_b<BT>(j, r16), acc[i][j], i, j);
}

// The planes of value(M, N, acc[i][j], i, j, w) (four rows M .. of column N), to d as the matrix [N][M] from
// (n0, m0) on, and with `mirror` to e as [M][N] from (m0, n0) on. Blocks of two by two fragments together.
template <int BT, class Fn>
CB_DEV void ns_emit(NsAcc<BT>& acc, char* d, int ld, int n0, int m0, bool mirror, char* e, int lde, Fn&& value) {
    using W = NsWaves<BT>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = lane >> 4, r16 = lane & 15, wm = wave / W::WN * (W::FM * 16), wn = wave % W::WN * (W::FN * 16);
    if constexpr (BT == 32) {
        const int M = wm + 4 * g, N = wn + r16;
        float w[4];
        value(M, N, acc[0][0], 0, 0, w);
        uint2 hi, lo;
        ns_split(w, hi, lo);
        ns_store(d, n0 + N, m0 + M, ld, hi, lo);
        if (mirror) ns_store_across(e, m0 + M, n0 + N, lde, hi, lo);
    } else {
#pragma unroll
        for (int i = 0; i < W::FM; i += 2)
#pragma unroll
            for (int j = 0; j < W::FN; j += 2) {
                const int M = wm + ns_row_a<BT>(i, 4 * g), N = wn + ns_row_b<BT>(j, r16);
                uint2 hi[2][2], lo[2][2];   // [N][M / 4]
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float w[4];
                        value(M + 4 * u, N + v, acc[i + u][j + v], i + u, j + v, w);
                        ns_split(w, hi[v][u], lo[v][u]);
                    }
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    char* p = d + ns_at(n0 + N + v, m0 + M, ld);
                    *reinterpret_cast<uint4*>(p) = make_uint4(hi[v][0].x, hi[v][0].y, hi[v][1].x, hi[v][1].y);
                    *reinterpret_cast<uint4*>(p + kLo) = make_uint4(lo[v][0].x, lo[v][0].y, lo[v][1].x, lo[v][1].y);
                }
                if (mirror) {
                    char* p = e + ns_at(m0 + M, n0 + N, lde);
#pragma unroll
                    for (int r = 0; r < 8; ++r, p += int64_t(lde) * 4) {
                        auto two = [&](const uint2 (&x)[2][2]) CB_INLINE_LAMBDA {
                            const uint32_t a = r & 2 ? x[0][r / 4].y : x[0][r / 4].x, b = r & 2 ? x[1][r / 4].y : x[1][r / 4].x;
                            return r & 1 ? (a >> 16) | (b & 0xffff0000u) : (a & 0xffffu) | (b << 16);
                        };
                        *reinterpret_cast<uint32_t*>(p) = two(hi);
                        *reinterpret_cast<uint32_t*>(p + kLo) = two(lo);
                    }
                }
            }
    }
}

// ------------------------------------------------------------------ Gram product

struct NsSeg {                 // one segment's polynomials and scales (host constants)
    int len;
    float c[kSegBf16][3];
    float sa, sp, st, sq;      // power-of-two scales of A, P, P A and Q
    float su, sv;              // and of P Q and b Q + c A' Q
    float alpha;               // the Gram matrix's scale where X's planes have a static one, else 0
};

// X is held as X / rho with rho = ||x|| / max(||x||, eps), so that it keeps its bits where eps is far above
// the norm; info[mat] = (what undoes the first planes' scale and divides by the norm, rho).
CB_DEV float2 ns_info(const NsArgs& a, int mat) { return reinterpret_cast<const float2*>(a.ws + a.info)[mat]; }
CB_DEV float ns_alpha(const NsArgs& a, const NsSeg& s, int mat) {
    const float2 i = ns_info(a, mat);
    const float f = s.alpha > 0.f ? i.y : i.x * i.y;
    return s.alpha > 0.f ? s.alpha * f * f : f * f;
}

// One tile of A = X X^T (smaller side), scaled; or, where k is split or the m x m part is done in LDS, the
// k range of one split of it to part [split][tile][N][M] float32. Only the lower triangle's tiles, so half
// the operations. Without the split 3872 x 256 would be 10 workgroups of 61 steps; with it 210 of 3, 8 us,
// of which the start and the end of a workgroup are most. 4096 x 4096: 243 us, 114 in one plane.
template <int BT, int BK, int ST, int NP>
__global__ __launch_bounds__(64 * NsWaves<BT>::NW) void ns_gram_kernel(NsArgs a, NsSeg s, int src) {
    extern __shared__ __align__(16) unsigned char smem[];
    int blk = blockIdx.x;
    const NsGroup& G = a.g[ns_group(a, blk)];
    if (BT >= 128) blk = ns_xcd(blk, G.batch * G.gtiles * G.splits);
    const int t = blk % G.gtiles, z = blk / G.gtiles % G.splits, b = blk / (G.splits * G.gtiles);
    int ti, tj;
    ns_tile(t, ti, tj);   // (where partials are summed, in this order)
    if (BT >= 128 && G.splits == 1) ns_tile_near(t, G.mp / BT, ti, tj);
    const char* X = a.ws + (G.tall ? G.xt : G.x)[src] + int64_t(b) * NP * (G.tall ? G.ts : G.xs);   // [m][n]
    const int k0 = z * G.kchunk, k1 = min(G.np, k0 + G.kchunk);
    NsAcc<BT> acc;
    ns_clear<BT>(acc);
    const int ld = G.tall ? G.ldt : G.ldx;
    const int64_t xs = NP * (G.tall ? G.ts : G.xs);
    ns_gemm<BT, BK, ST, NP, NP>(X, xs, ld, ti * BT, X, xs, ld, tj * BT, k0, k1, smem, acc);
    if (G.splits == 1 && !G.small) {
        char* D = a.ws + G.a + int64_t(b) * 2 * G.ms;
        const float f = ns_alpha(a, s, G.first + b) * s.sa;
        ns_emit<BT>(acc, D, G.ldm, tj * BT, ti * BT, ti != tj, D, G.ldm,
                    [&](int, int, cb_f32x4 v, int, int, float (&w)[4]) CB_INLINE_LAMBDA {
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[r] = v[r] * f;
                    });
        return;
    }
    float* part = reinterpret_cast<float*>(a.ws + G.part + int64_t(b) * G.ps) + (int64_t(z) * G.gtiles + t) * (BT * BT);
    ns_each<BT>(acc, [&](int M, int N, cb_f32x4 v, int, int) CB_INLINE_LAMBDA {
        *reinterpret_cast<float4*>(part + N * BT + M) = make_float4(v[0], v[1], v[2], v[3]);
    });
}

// ------------------------------------------------------------------ the m x m products

// A whole segment's m x m part of one matrix with m <= 64 in LDS, float32: five m x m buffers of pitch
// 68, which a fragment read of 16 bytes from each of 16 rows crosses without bank conflicts.
constexpr int kSmPitch = 68, kSmBuf = 64 * kSmPitch, kSmThreads = 1024;
constexpr int kSmLds = 5 * kSmBuf * int(sizeof(float));

// f(N, M, v, mirror): four rows M .. M+3 of column N of L R^T for symmetric L, R that commute: the lower
// triangle's tiles of 16 in turn over the waves, the others their mirror images. A lane group takes four
// neighbouring k of each 16 (any order of k is the same sum), so four products share a 16-byte read.
// back: from the last wave on, for the second of two products between the same barriers.
template <class Fn>
CB_DEV void ns_small_mul(const float* L, const float* R, int mt, int pitch, bool back, Fn&& f) {
    const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = back ? kSmThreads / 64 - 1 - (threadIdx.x >> 6) : threadIdx.x >> 6;
    for (int t = wave; t < mt * (mt + 1) / 2; t += kSmThreads / 64) {
        int i, j;
        ns_tile(t, i, j);
        const float* l = L + (i * 16 + r16) * pitch + 4 * g;
        const float* r = R + (j * 16 + r16) * pitch + 4 * g;
        float4 x[4], y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < mt) {
                x[k] = *reinterpret_cast<const float4*>(l + 16 * k);
                y[k] = *reinterpret_cast<const float4*>(r + 16 * k);
            }
        // two sums, so that a product does not wait for the one before
        cb_f32x4 acc{0.f, 0.f, 0.f, 0.f}, acc2{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < mt) {
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k].x, y[k].x, acc, 0, 0, 0);
                acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k].y, y[k].y, acc2, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k].z, y[k].z, acc, 0, 0, 0);
                acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[k].w, y[k].w, acc2, 0, 0, 0);
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += acc2[e];
        f(j * 16 + r16, i * 16 + 4 * g, acc, i != j);
    }
}
CB_DEV void ns_small_put(float* D, int pitch, int N, int M, float4 v, bool mirror) {
    *reinterpret_cast<float4*>(D + N * pitch + M) = v;
    if (mirror) {
        D[M * pitch + N] = v.x; D[(M + 1) * pitch + N] = v.y;
        D[(M + 2) * pitch + N] = v.z; D[(M + 3) * pitch + N] = v.w;
    }
}
// D = a I + b A + c A^2.
CB_DEV void ns_small_poly(const float* A, float* D, int mt, int pitch, float a, float b, float c) {
    ns_small_mul(A, A, mt, pitch, false, [&](int N, int M, cb_f32x4 v, bool mirror) CB_INLINE_LAMBDA {
        const float4 q = *reinterpret_cast<const float4*>(A + N * pitch + M);
        ns_small_put(D, pitch, N, M,
                     make_float4(b * q.x + c * v[0] + (N == M ? a : 0.f), b * q.y + c * v[1] + (N == M + 1 ? a : 0.f),
                                 b * q.z + c * v[2] + (N == M + 2 ? a : 0.f), b * q.w + c * v[3] + (N == M + 3 ? a : 0.f)),
                     mirror);
    });
}

// The sum of n float4, `step` floats apart, in order; eight loads in flight.
CB_DEV float4 ns_sum(const float* p, int n, int64_t step) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z = 0; z < n; z += 8) {
        float4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const float4*>(p + min(z + u, n - 1) * step);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (z + u < n) { s.x += v[u].x; s.y += v[u].y; s.z += v[u].z; s.w += v[u].w; }
    }
    return s;
}

CB_DEV void ns_small(const NsArgs& a, const NsGroup& G, const NsSeg& s, int b, float* sm) {
    float *A = sm, *T = sm + kSmBuf, *P = sm + 2 * kSmBuf, *Q = sm + 3 * kSmBuf, *Q2 = sm + 4 * kSmBuf;
    const int mt = (G.m + 15) / 16;
    const float alpha = ns_alpha(a, s, G.first + b);
    const float* part = reinterpret_cast<const float*>(a.ws + G.part + int64_t(b) * G.ps);
    for (int e = threadIdx.x * 4; e < 64 * 64; e += 4 * kSmThreads) {
        const float4 v = ns_sum(part + e, G.splits, 4096);
        *reinterpret_cast<float4*>(A + (e >> 6) * kSmPitch + (e & 63)) =
            make_float4(v.x * alpha, v.y * alpha, v.z * alpha, v.w * alpha);
    }
    __syncthreads();
    auto put = [&](float* D) {
        return [=](int N, int M, cb_f32x4 v, bool mirror) CB_INLINE_LAMBDA {
            ns_small_put(D, kSmPitch, N, M, make_float4(v[0], v[1], v[2], v[3]), mirror);
        };
    };
    for (int t = 0; t < s.len; ++t) {
        float* D = t == 0 ? Q : P;
        ns_small_poly(A, D, mt, kSmPitch, s.c[t][0], s.c[t][1], s.c[t][2]);
        __syncthreads();
        if (t > 0) {
            ns_small_mul(P, Q, mt, kSmPitch, false, put(Q2));
            float* w = Q; Q = Q2; Q2 = w;
        }
        if (t + 1 < s.len) {
            const float* F = t == 0 ? Q : P;   // the first P is Q
            ns_small_mul(F, A, mt, kSmPitch, t > 0, put(T));
            __syncthreads();
            ns_small_mul(T, F, mt, kSmPitch, false, put(A));
        }
        __syncthreads();
    }
    char* q = a.ws + G.q[0] + int64_t(b) * 2 * G.ms;
    for (int e = threadIdx.x * 4; e < 64 * 64; e += 4 * kSmThreads) {
        const int N = e >> 6, M = e & 63;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = N < G.m && M + r < G.m ? Q[N * kSmPitch + M + r] * s.sq : 0.f;
        uint2 hi, lo;
        ns_split(v, hi, lo);
        ns_store(q, N, M, G.ldm, hi, lo);
    }
}

// Sums the Gram partials in split order. m <= 64: and goes on to Q. Else A's planes, 16 columns of a
// tile a workgroup, with the mirror image of an off-diagonal tile. Two steps at m = 64: 11 us on 16 waves
// (17 on 4), a product of 64 x 64 taking 0.5 us of a CU's float32 matrix rate; 256 x 256 in 20 splits: 6 us.
template <int NT>
__global__ __launch_bounds__(NT) void ns_reduce_kernel(NsArgs a, NsSeg s) {
    extern __shared__ __align__(16) unsigned char smem[];
    int blk = blockIdx.x;
    const NsGroup& G = a.g[ns_group(a, blk)];
    if constexpr (NT == kSmThreads)
        if (G.small) {
            ns_small(a, G, s, blk, reinterpret_cast<float*>(smem));
            return;
        }
    float* sh = reinterpret_cast<float*>(smem);   // [BT][17]
    const int bt = G.bg, strips = bt / 16;
    const int n0 = (blk % strips) * 16, t = blk / strips % G.gtiles, b = blk / (strips * G.gtiles);
    int ti, tj;
    ns_tile(t, ti, tj);
    const float alpha = ns_alpha(a, s, G.first + b) * s.sa;
    const float* part = reinterpret_cast<const float*>(a.ws + G.part + int64_t(b) * G.ps) + int64_t(t) * bt * bt;
    char* A = a.ws + G.a + int64_t(b) * 2 * G.ms;
    for (int e = threadIdx.x * 4; e < 16 * bt; e += 4 * NT) {
        const int N = n0 + e / bt, M = e % bt;
        const float4 q = ns_sum(part + N * bt + M, G.splits, int64_t(G.gtiles) * bt * bt);
        float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] *= alpha;
            sh[(M + r) * 17 + e / bt] = v[r];
        }
        uint2 hi, lo;
        ns_split(v, hi, lo);
        ns_store(A, tj * bt + N, ti * bt + M, G.ldm, hi, lo);
    }
    if (ti == tj) return;
    __syncthreads();
    for (int e = threadIdx.x * 4; e < 16 * bt; e += 4 * NT) {
        const int M = e / 16, q = e % 16;
        const float v[4] = {sh[M * 17 + q], sh[M * 17 + q + 1], sh[M * 17 + q + 2], sh[M * 17 + q + 3]};
        uint2 hi, lo;
        ns_split(v, hi, lo);
        ns_store(A, ti * bt + M, tj * bt + n0 + q, G.ldm, hi, lo);
    }
}

// The products of symmetric matrices that commute: tiles of the lower triangle and their mirror images, one
// or two products a launch. m = 256: 5 us (36 tiles of 32), a launch and eight trips to memory in turn;
// 1001 x 2: 30 us for one product or two (72 or 144 tiles of 128; tiles of 64, 272 or 544, took 24 and 38);
// 4096: 195 us, 1.21 PFLOP/s.
enum { NS_A = 0, NS_T, NS_P, NS_V, NS_Q0, NS_Q1 };
struct NsJob {                 // dst = diag I + fa add + f lhs rhs (scales included)
    int lhs, rhs, dst, add;
    float f, fa, diag;
};
struct NsJobs { int n; NsJob j[2]; };

CB_DEV char* ns_buf(const NsArgs& a, const NsGroup& G, int id, int b) {
    const int64_t o = id == NS_A ? G.a : id == NS_T ? G.t : id == NS_P ? G.p : id == NS_V ? G.v : id == NS_Q0 ? G.q[0] : G.q[1];
    return a.ws + o + int64_t(b) * 2 * G.ms;
}

// With tiles of 32 and 64, where a launch is a row of latencies, `add` is read before the product.
template <int BT, int BK, int ST, bool CROSS>
__global__ __launch_bounds__(64 * NsWaves<BT>::NW) void ns_prod_kernel(NsArgs a, NsJobs jobs) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr bool EARLY = BT <= 64;
    using W = NsWaves<BT>;
    int blk = blockIdx.x;
    const NsGroup& G = a.g[ns_group(a, blk)];
    if (BT >= 128) blk = ns_xcd(blk, G.batch * G.tiles * jobs.n);
    const NsJob& J = jobs.j[blk / G.tiles % jobs.n];
    const int b = blk / (jobs.n * G.tiles);
    int ti, tj;
    if (BT >= 128) ns_tile_near(blk % G.tiles, G.mp / BT, ti, tj);
    else ns_tile(blk % G.tiles, ti, tj);
    const char* add = ns_buf(a, G, J.add, b);
    uint4 early[EARLY ? W::FM : 1][EARLY ? W::FN : 1];
    NsAcc<BT> acc;
    ns_clear<BT>(acc);
    if (EARLY && (J.fa != 0.f || J.diag != 0.f))
        ns_each<BT>(acc, [&](int M, int N, cb_f32x4, int i, int j) CB_INLINE_LAMBDA {
            const char* p = add + ns_at(tj * BT + N, ti * BT + M, G.ldm);
            const uint2 h = *reinterpret_cast<const uint2*>(p), l = *reinterpret_cast<const uint2*>(p + kLo);
            early[i][j] = make_uint4(h.x, h.y, l.x, l.y);
        });
    ns_gemm<BT, BK, ST, 2, 2, CROSS>(ns_buf(a, G, J.lhs, b), 2 * G.ms, G.ldm, ti * BT, ns_buf(a, G, J.rhs, b), 2 * G.ms, G.ldm,
                                     tj * BT, 0, G.mp, smem, acc);
    char* D = ns_buf(a, G, J.dst, b);
    const float f = J.f, fa = J.fa, diag = J.diag;
    ns_emit<BT>(acc, D, G.ldm, tj * BT, ti * BT, ti != tj, D, G.ldm,
                [&](int M, int N, cb_f32x4 v, int i, int j, float (&w)[4]) CB_INLINE_LAMBDA {
        const int m = ti * BT + M, n = tj * BT + N;
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = f * v[r];
        if (fa != 0.f || diag != 0.f) {
            uint4 e;
            if constexpr (EARLY) {
                e = early[i][j];
            } else {
                const char* p = add + ns_at(n, m, G.ldm);
                const uint2 h = *reinterpret_cast<const uint2*>(p), l = *reinterpret_cast<const uint2*>(p + kLo);
                e = make_uint4(h.x, h.y, l.x, l.y);
            }
            float q[4];
            ns_join(make_uint2(e.x, e.y), make_uint2(e.z, e.w), q);
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] += fa * q[r] + (m + r == n ? diag : 0.f);
        }
    });
}

// ------------------------------------------------------------------ Q X

// A tile of Q X: the next segment's planes of X and of its transpose, the result, or the parameters, so that
// the result of muon_step is never written. 3872 x 256: 9 us (244 tiles of 64), where k = 256 is four steps of
// the ring and the start, the writes and the launch are most; 7744 x 512: 19 us; 4096 x 4096: 360 us.
enum { NS_OUT_MID = 0, NS_OUT_F32, NS_OUT_BF16, NS_OUT_STEP };
struct NsApply {
    int out, src, dst, q;      // X buffer read, X buffer written (MID), Q buffer of the large groups
    float f;                   // 1 / (scale of Q, of X where static), times the new scale (MID)
    int use_inv;               // X carries its matrix's own scale (info)
    void* y;
    float* p;                  // parameters (STEP)
    float decay, lr;
    uint16_t* mir; int64_t mir_off, mir_len;
};

template <int BT, int BK, int ST, int NP>
__global__ __launch_bounds__(64 * NsWaves<BT>::NW) void ns_apply_kernel(NsArgs a, NsApply ap) {
    extern __shared__ __align__(16) unsigned char smem[];
    int blk = blockIdx.x;
    const NsGroup& G = a.g[ns_group(a, blk)];
    const int tn = G.rp / BT, tm = G.cp / BT;   // N over the rows, M over the columns
    int jt = blk % tn, it = blk / tn % tm, b = blk / (tn * tm);
    if (BT >= 128) {   // bands of kWide rows, column by column
        blk = ns_xcd(blk, G.batch * tn * tm);
        b = blk / (tn * tm);
        blk %= tn * tm;
        const int r = blk / (kWide * tm) * kWide, h = min(kWide, tn - r);
        blk -= r * tm;
        jt = r + blk % h;
        it = blk / h;
    }
    const int ld = G.tall ? G.ldx : G.ldt;
    const int64_t xs = NP * (G.tall ? G.xs : G.ts);
    const char* X = a.ws + (G.tall ? G.x : G.xt)[ap.src] + b * xs;   // [n][m]
    const char* Q = a.ws + (G.small ? G.q[0] : G.q[ap.q]) + int64_t(b) * 2 * G.ms;
    NsAcc<BT> acc;
    ns_clear<BT>(acc);
    // the result's rows are X's where it is tall (M, the contiguous index, over Q's) and Q's where it is wide
    if constexpr (NP == 2) {
        const bool tall = G.tall;
        ns_gemm<BT, BK, ST, 2, 2>(tall ? Q : X, tall ? 2 * G.ms : xs, tall ? G.ldm : ld, it * BT, tall ? X : Q,
                                  tall ? xs : 2 * G.ms, tall ? ld : G.ldm, jt * BT, 0, G.mp, smem, acc);
    } else if (G.tall) {
        ns_gemm<BT, BK, ST, 2, NP>(Q, 2 * G.ms, G.ldm, it * BT, X, xs, ld, jt * BT, 0, G.mp, smem, acc);
    } else {
        ns_gemm<BT, BK, ST, NP, 2>(X, xs, ld, it * BT, Q, 2 * G.ms, G.ldm, jt * BT, 0, G.mp, smem, acc);
    }
    float f = ap.f;
    const float2 info = ns_info(a, G.first + b);
    if (ap.use_inv) f *= info.x;
    if (ap.out != NS_OUT_MID) f *= info.y;
    if (ap.out == NS_OUT_MID) {
        char* D = a.ws + G.x[ap.dst] + int64_t(b) * 2 * G.xs;
        char* T = a.ws + G.xt[ap.dst] + int64_t(b) * 2 * G.ts;
        ns_emit<BT>(acc, D, G.ldx, jt * BT, it * BT, true, T, G.ldt,
                    [&](int, int, cb_f32x4 v, int, int, float (&w)[4]) CB_INLINE_LAMBDA {
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[r] = v[r] * f;
                    });
        return;
    }
    const int64_t off = ns_offset(a, G, b);
    const int rows = G.rows, cols = G.cols;
    if (ap.out == NS_OUT_BF16) {
        uint16_t* y = static_cast<uint16_t*>(ap.y) + off;
        const bool vec = cols % 4 == 0 && (reinterpret_cast<uintptr_t>(y) & 7) == 0;
        ns_each<BT>(acc, [&](int M, int N, cb_f32x4 v, int, int) CB_INLINE_LAMBDA {
            const int r = jt * BT + N, c = it * BT + M;
            if (r >= rows) return;
            uint16_t* o = y + int64_t(r) * cols + c;
            if (vec && c < cols) store4(o, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < cols) o[e] = f2bf(v[e] * f);
        });
        return;
    }
    if (ap.out == NS_OUT_F32) {
        float* y = static_cast<float*>(ap.y) + off;
        ns_each<BT>(acc, [&](int M, int N, cb_f32x4 v, int, int) CB_INLINE_LAMBDA {
            const int r = jt * BT + N, c = it * BT + M;
            if (r >= rows) return;
            float* o = y + int64_t(r) * cols + c;
            if (c + 4 <= cols) {
                *reinterpret_cast<cb_f32x4_a4*>(o) = cb_f32x4_a4{v[0] * f, v[1] * f, v[2] * f, v[3] * f};
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < cols) o[e] = v[e] * f;
            }
        });
        return;
    }
    // the parameters: p <- decay p - lr scale O
    f *= ap.lr * G.scale;
    ns_each<BT>(acc, [&](int M, int N, cb_f32x4 v, int, int) CB_INLINE_LAMBDA {
        const int r = jt * BT + N, c = it * BT + M;
        if (r >= rows || c >= cols) return;
        const int64_t o = off + int64_t(r) * cols + c;
        const int k = min(4, cols - c);
        float w[4];
        if (k == 4) {
            const float4 p = load_f4(ap.p + o);
            w[0] = ap.decay * p.x - f * v[0]; w[1] = ap.decay * p.y - f * v[1];
            w[2] = ap.decay * p.z - f * v[2]; w[3] = ap.decay * p.w - f * v[3];
            *reinterpret_cast<cb_f32x4_a4*>(ap.p + o) = cb_f32x4_a4{w[0], w[1], w[2], w[3]};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < k) {
                    w[e] = ap.decay * ap.p[o + e] - f * v[e];
                    ap.p[o + e] = w[e];
                }
        }
        if (ap.mir)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t d = o + e - ap.mir_off;
                if (e < k && d >= 0 && d < ap.mir_len) ap.mir[d] = f2bf(w[e]);
            }
    });
}

// ------------------------------------------------------------------ sums of squares, planes

enum { NS_SRC_F32 = 0, NS_SRC_BF16, NS_SRC_STEP };

// The workgroup's sums of N values of each of 256 threads, in a fixed order. Ends with a barrier.
template <int N>
CB_DEV void ns_sum256(double (&v)[N], double* sh) {
    for (int m = 1; m < 64; m <<= 1) {
        double o[N];
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = __shfl_xor(v[k], m);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += o[k];
    }
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) sh[(threadIdx.x >> 6) * N + k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (sh[k] + sh[N + k]) + (sh[2 * N + k] + sh[3 * N + k]);
    __syncthreads();
}

// Blocks [0, start[ng]) sum a matrix's elements in G.nsum shares; (STEP) those after them the gaps'.
// Memory-bound where it is long (the wide net's 35 MB of g and m: 11 us), else latency: 5 to 7 us.
// Three doubles a block: sum g^2, sum g m, sum m^2 (others: sum x^2, 0, 0).
template <int SRC>
__global__ __launch_bounds__(256) void ns_sums_kernel(NsArgs a, MuonElem e, const void* src, int block0) {
    __shared__ double sh[12];
    int64_t at, len;
    int blk = blockIdx.x;
    bool both = SRC == NS_SRC_STEP;
    if (SRC != NS_SRC_STEP || blk < a.start[a.ng]) {
        const NsGroup& G = a.g[ns_group(a, blk)];
        const int b = blk / G.nsum, k = blk % G.nsum;
        const int64_t tot = int64_t(G.rows) * G.cols, per = ((tot + G.nsum - 1) / G.nsum + 3) / 4 * 4;
        at = ns_offset(a, G, b) + k * per;
        len = min(per, tot - k * per);
    } else {
        blk -= a.start[a.ng];
        int i = 0;
        while (i + 1 < e.ngaps && blk >= e.gap_start[i + 1]) ++i;
        const int nb = e.gap_start[i + 1] - e.gap_start[i], k = blk - e.gap_start[i];
        const int64_t per = ((e.gap_len[i] + nb - 1) / nb + 3) / 4 * 4;
        at = e.gap[i] + k * per;
        len = min(per, e.gap_len[i] - k * per);
        both = false;
    }
    double gg = 0.0, gm = 0.0, mm = 0.0;
    auto add = [&](float g, float m) CB_INLINE_LAMBDA {
        gg += double(g) * g;
        if (SRC == NS_SRC_STEP && both) {
            gm += double(g) * m;
            mm += double(m) * m;
        }
    };
    if (SRC == NS_SRC_BF16) {
        const uint16_t* x = static_cast<const uint16_t*>(src) + at;
        if ((reinterpret_cast<uintptr_t>(x) & 7) == 0) {
            for (int64_t i = threadIdx.x * 4; i < len; i += 1024) {
                float v[4] = {0.f, 0.f, 0.f, 0.f};
                if (i + 4 <= len) load4(x + i, v);
                else
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (i + q < len) v[q] = bf2f(x[i + q]);
#pragma unroll
                for (int q = 0; q < 4; ++q) add(v[q], 0.f);
            }
        } else {
            for (int64_t i = threadIdx.x; i < len; i += 256) add(bf2f(x[i]), 0.f);
        }
    } else {
        const float* x = (SRC == NS_SRC_STEP ? e.g : static_cast<const float*>(src)) + at;
        const float* m = e.m + at;
        for (int64_t i = threadIdx.x * 4; i < len; i += 1024) {
            if (i + 4 <= len) {
                const float4 v = load_f4(x + i);
                float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
                if (SRC == NS_SRC_STEP && both) w = load_f4(m + i);
                add(v.x, w.x); add(v.y, w.y); add(v.z, w.z); add(v.w, w.w);
            } else {
                for (int64_t q = i; q < len; ++q) add(x[q], SRC == NS_SRC_STEP && both ? m[q] : 0.f);
            }
        }
    }
    double t[3] = {gg, gm, mm};
    ns_sum256(t, sh);
    if (threadIdx.x == 0) {
        double* o = reinterpret_cast<double*>(a.ws + a.sums) + int64_t(3) * (block0 + blockIdx.x);
        o[0] = t[0]; o[1] = t[1]; o[2] = t[2];
    }
}

// Workgroups of the planes: tiles of 64 x 64 of the padded shape.
__host__ __device__ inline int ns_plane_blocks(const NsGroup& G) { return (G.rp / 64) * (G.cp / 64); }

// The power of two that brings a matrix of this norm to a root mean square in [1, 2): elements stay below
// 2 sqrt(2^28) in f16's range. By exponents: the double logarithm and power of a few threads would be most of
// the launch's time where it is short.
CB_DEV float ns_scale(double norm, double elems) {
    int k = 0;
    if (norm > 0.0 && isfinite(norm)) k = -(ilogb(norm * norm / elems) >> 1);
    return ldexpf(1.f, k < -126 ? -126 : k > 126 ? 126 : k);
}
// ... and info as ns_info. A zero matrix: (1, 0).
CB_DEV float2 ns_norms(double norm, double f, float eps) {
    if (norm == 0.0) return make_float2(1.f, 0.f);
    return make_float2(float(1.0 / (norm * f)), float(norm / (norm > double(eps) || norm != norm ? norm : double(eps))));
}

CB_DEV float ns_adam(float p, float g, float& m, float& v, const MuonElem& e) {
    m = e.b1 * m + e.omb1 * g;
    v = e.b2 * v + e.omb2 * g * g;
    const float mh = m / e.bc1, vh = v / e.bc2;
    return p - e.alr * mh / (sqrtf(vh) + e.aeps);
}

// Four neighbours of a row as they are in memory, n of them inside.
template <class T>
CB_DEV void ns_load4(const T* x, int n, float (&w)[4]) {
    if (sizeof(T) == 4) {
        if (n == 4) {
            const float4 v = load_f4(reinterpret_cast<const float*>(x));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            return;
        }
    } else if (n == 4 && (reinterpret_cast<uintptr_t>(x) & 7) == 0) {
        load4(reinterpret_cast<const uint16_t*>(x), w);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = i >= n ? 0.f : sizeof(T) == 4 ? reinterpret_cast<const float*>(x)[i] : bf2f(reinterpret_cast<const uint16_t*>(x)[i]);
}

// X's planes from the source (STEP: u from the clipped gradient and the momentum, which is updated),
// padded with zeros; blocks after the matrices' (STEP): Adam on what no matrix covers. The elements are
// loaded before the norms are formed, which takes as long as they do to arrive. A workgroup takes 64 x 64
// through LDS, so that both forms are written by rows. 3872 x 256: 11 us for 12 MB, latency; the wide net's
// 1101 tiles: 24 us, 87 MB at 3.6 TB/s.
template <int SRC, int NP>
__global__ __launch_bounds__(256) void ns_planes_kernel(NsArgs a, MuonElem e, const void* src, float eps, int block0) {
    using T = std::conditional_t<SRC == NS_SRC_BF16, uint16_t, float>;
    __shared__ double sh[16];
    __shared__ float tile[64 * 65];
    const double* sums = reinterpret_cast<const double*>(a.ws + a.sums);
    int blk = blockIdx.x;
    const bool gap = SRC == NS_SRC_STEP && blk >= a.start[a.ng];
    const int gi = gap ? 0 : ns_group(a, blk);
    const NsGroup& G = a.g[gi];
    const int per = ns_plane_blocks(G), b = gap ? 0 : blk / per, k = gap ? 0 : blk % per;
    const int64_t off = ns_offset(a, G, b);
    const int tc = max(1, G.cp / 64), r0 = k / tc * 64, q0 = k % tc * 64;   // (no group at all: gaps only)
    float x[4][4], mv[4][4];
    if (!gap)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q = threadIdx.x + 256 * i, r = r0 + (q >> 4), c = q0 + (q & 15) * 4;
            const int n = r < G.rows ? min(4, G.cols - c) : 0;
            const int64_t o = off + int64_t(r) * G.cols + c;
            ns_load4((SRC == NS_SRC_STEP ? reinterpret_cast<const T*>(e.g) : static_cast<const T*>(src)) + o, n, x[i]);
            if (SRC == NS_SRC_STEP) ns_load4(reinterpret_cast<const T*>(e.m) + o, n, mv[i]);
        }
    double t[4] = {0.0, 0.0, 0.0, 0.0};   // the call's g^2; the matrix's g^2, g m, m^2
    if (SRC == NS_SRC_STEP)
        for (int i = threadIdx.x; i < e.nblocks; i += 256) t[0] += sums[3 * i];
    if (!gap) {
        const double* ms = sums + int64_t(3) * (G.part0 + b * G.nsum);
        for (int i = threadIdx.x; i < G.nsum; i += 256) {
            t[1] += ms[3 * i]; t[2] += ms[3 * i + 1]; t[3] += ms[3 * i + 2];
        }
    }
    ns_sum256(t, sh);
    float clip = 1.f;
    if (SRC == NS_SRC_STEP) {
        const double norm = sqrt(t[0]);
        if (blockIdx.x == 0 && block0 == 0 && threadIdx.x == 0 && e.stats) {
            e.stats[0] = float(norm);
            e.stats[1] = isfinite(norm) ? 0.f : 1.f;
        }
        clip = (e.max_norm > 0.f && norm > double(e.max_norm)) ? float(double(e.max_norm) / norm) : 1.f;
    }
    if (gap) {
        blk -= a.start[a.ng];
        int i = 0;
        while (i + 1 < e.ngaps && blk >= e.gap_start[i + 1]) ++i;
        const int nb = e.gap_start[i + 1] - e.gap_start[i], z = blk - e.gap_start[i];
        for (int64_t q = int64_t(z) * 256 + threadIdx.x; q < e.gap_len[i]; q += int64_t(nb) * 256) {
            const int64_t o = e.gap[i] + q;
            float m = e.m[o], v = e.v[o];
            const float p = ns_adam(e.p[o], e.g[o] * clip, m, v, e);
            e.p[o] = p; e.m[o] = m; e.v[o] = v;
            if (e.mir && o >= e.mir_off && o < e.mir_off + e.mir_len) e.mir[o - e.mir_off] = f2bf(p);
        }
        return;
    }
    double norm = sqrt(t[1]);
    if (SRC == NS_SRC_STEP) {
        // ||c1 g + c2 m|| from the three sums; where the two all but cancel what is left of it is
        // their rounding, and a norm no smaller than that keeps the singular values below one
        const double c1 = double(e.c1) * clip, c2 = e.c2;
        const double est = c1 * c1 * t[1] + 2.0 * c1 * c2 * t[2] + c2 * c2 * t[3];
        const double least = 0x1p-21 * (fabs(c1) * sqrt(t[1]) + fabs(c2) * sqrt(t[3]));
        norm = est < least * least ? least : sqrt(est);
        eps = e.eps;
    }
    const float f = ns_scale(norm, double(G.rows) * G.cols);
    if (k == 0 && threadIdx.x == 0) reinterpret_cast<float2*>(a.ws + a.info)[G.first + b] = ns_norms(norm, f, eps);
    char* X = a.ws + G.x[0] + int64_t(b) * NP * G.xs;
    char* Xt = a.ws + G.xt[0] + int64_t(b) * NP * G.ts;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int q = threadIdx.x + 256 * i, lr = q >> 4, lc = (q & 15) * 4, r = r0 + lr, c = q0 + lc;
        const int n = r < G.rows ? min(4, G.cols - c) : 0;
        float (&w)[4] = x[i];
        if (SRC == NS_SRC_STEP) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float gs = e.omu * (w[u] * clip);
                mv[i][u] = e.mu * mv[i][u] + gs;
                w[u] = e.nesterov ? e.mu * mv[i][u] + gs : mv[i][u];
            }
            float* m = e.m + off + int64_t(r) * G.cols + c;
            if (n == 4) {
                *reinterpret_cast<cb_f32x4_a4*>(m) = cb_f32x4_a4{mv[i][0], mv[i][1], mv[i][2], mv[i][3]};
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (u < n) m[u] = mv[i][u];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = u < n ? w[u] * f : 0.f;
        uint2 hi, lo;
        ns_split(w, hi, lo);
        if (NP > 1) ns_store(X, r, c, G.ldx, hi, lo);
        else *reinterpret_cast<uint2*>(X + (int64_t(r) * G.ldx + c) * 2) = hi;
#pragma unroll
        for (int u = 0; u < 4; ++u) tile[(lc + u) * 65 + lr] = w[u];
    }
    __syncthreads();
    for (int q = threadIdx.x; q < 1024; q += 256) {   // the transpose
        const int lc = q >> 4, lr = (q & 15) * 4;
        const float w[4] = {tile[lc * 65 + lr], tile[lc * 65 + lr + 1], tile[lc * 65 + lr + 2], tile[lc * 65 + lr + 3]};
        uint2 hi, lo;
        ns_split(w, hi, lo);
        if (NP > 1) ns_store(Xt, q0 + lc, r0 + lr, G.ldt, hi, lo);
        else *reinterpret_cast<uint2*>(Xt + (int64_t(q0 + lc) * G.ldt + r0 + lr) * 2) = hi;
    }
}

// ------------------------------------------------------------------ small matrices: all of it in one launch
//
// A matrix of at most 64 on its smaller side that fits one CU's LDS in float32 takes one workgroup and no
// workspace: its steps one by one, as they are written, from LDS in float32 MFMAs. What bounds it is the
// latency of each of its products and, at m = 64, the float32 matrix rate of one CU; the launches of the
// other way are 5 us each. 4 x 144x16: 15 us (61 the other way), 4 x 288x32: 28, 8 x 288x64: 66, 300 x
// 144x32: 40. Float32 products also keep it at half the error, 5e-7 of the norm where the planes have 1e-6.

struct NsOne { int rows, cols, steps; float eps; float c[kNsMaxSteps][3]; };

constexpr int kOnePart = 16 * 256;   // the Gram product's shares, and the doubles of the norm's sum
__host__ __device__ inline int ns_one_pitch(int v) { return (v + 15) / 16 * 16 + 4; }   // 4 x odd: rows meet all banks
__host__ __device__ inline int64_t ns_one_lds(int rows, int cols) {
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows, mp = (m + 15) / 16 * 16;
    return (int64_t(mp) * ns_one_pitch(n) + 2 * int64_t(mp) * ns_one_pitch(m) + kOnePart) * 4;
}

// f(row, col, element) over a rows x cols matrix: a group of lanes along a row, so that memory is read
// and written in order.
template <class Fn>
CB_DEV void ns_one_each(int rows, int cols, Fn&& f) {
    const int sh = cols <= 8 ? 3 : cols <= 16 ? 4 : cols <= 32 ? 5 : 6;
#pragma unroll 4
    for (int r = threadIdx.x >> sh; r < rows; r += kSmThreads >> sh)
#pragma unroll 2
        for (int c = threadIdx.x & ((1 << sh) - 1); c < cols; c += 1 << sh) f(r, c, r * cols + c);
}

template <bool BF>
__global__ __launch_bounds__(kSmThreads) void ns_one_kernel(const void* src, void* dst, NsOne o) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int rows = o.rows, cols = o.cols;
    const bool tall = rows > cols;
    const int m = tall ? cols : rows, n = tall ? rows : cols;
    const int mt = (m + 15) / 16, nt = (n + 15) / 16, pm = mt * 16 + 4, pn = nt * 16 + 4;
    float* part = reinterpret_cast<float*>(smem);
    float* A = part + kOnePart;
    float* P = A + mt * 16 * pm;
    float* X = P + mt * 16 * pm;   // [m][n]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r16 = lane & 15;
    constexpr int NW = kSmThreads / 64;
    const int64_t base = int64_t(blockIdx.x) * rows * cols;

    for (int i = threadIdx.x; i < mt * 16 * pn; i += kSmThreads) X[i] = 0.f;
    __syncthreads();
    double gg = 0.0;
    ns_one_each(rows, cols, [&](int r, int c, int e) CB_INLINE_LAMBDA {
        const float v = BF ? bf2f(static_cast<const uint16_t*>(src)[base + e]) : static_cast<const float*>(src)[base + e];
        X[tall ? c * pn + r : r * pn + c] = v;
        gg += double(v) * v;
    });
    const double norm = sqrt(block_sum<kSmThreads>(gg, reinterpret_cast<double*>(smem)));
    // X = rho x / norm with the factor rho beside it: an eps far above the norm does not underflow X
    const double inv = norm == 0.0 ? 1.0 : 1.0 / norm;
    float rho = norm == 0.0 ? 0.f : float(norm / (norm > double(o.eps) || norm != norm ? norm : double(o.eps)));
    for (int i = threadIdx.x; i < mt * 16 * pn; i += kSmThreads) X[i] = float(X[i] * inv);
    __syncthreads();

    const int tiles = mt * (mt + 1) / 2, split = NW / tiles;
    for (int t = 0; t < o.steps; ++t) {
        // A = X X^T: the lower triangle's tiles over the waves, k in `split` shares; the sum in their order
        if (wave < tiles * split) {
            const int z = wave / tiles;
            int i, j;
            ns_tile(wave - z * tiles, i, j);
            const float* l = X + (i * 16 + r16) * pn + 4 * g;
            const float* r = X + (j * 16 + r16) * pn + 4 * g;
            cb_f32x4 acc{0.f, 0.f, 0.f, 0.f}, acc2{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int k = z; k < nt; k += split) {
                const float4 x = *reinterpret_cast<const float4*>(l + 16 * k), y = *reinterpret_cast<const float4*>(r + 16 * k);
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, y.x, acc, 0, 0, 0);
                acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, y.y, acc2, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, y.z, acc, 0, 0, 0);
                acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, y.w, acc2, 0, 0, 0);
            }
            *reinterpret_cast<float4*>(part + wave * 256 + r16 * 16 + 4 * g) =
                make_float4(acc[0] + acc2[0], acc[1] + acc2[1], acc[2] + acc2[2], acc[3] + acc2[3]);
        }
        __syncthreads();
        for (int e = threadIdx.x * 4; e < tiles * 256; e += 4 * kSmThreads) {
            const int q = e >> 8, N = (e >> 4) & 15, M = e & 15;
            int i, j;
            ns_tile(q, i, j);
            float4 v = *reinterpret_cast<const float4*>(part + e);
            for (int z = 1; z < split; ++z) {
                const float4 w = *reinterpret_cast<const float4*>(part + z * tiles * 256 + e);
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
            const float f = t == 0 ? rho * rho : 1.f;
            v.x *= f; v.y *= f; v.z *= f; v.w *= f;
            ns_small_put(A, pm, j * 16 + N, i * 16 + M, v, i != j);
        }
        __syncthreads();
        ns_small_poly(A, P, mt, pm, o.c[t][0], o.c[t][1], o.c[t][2]);
        __syncthreads();
        // X <- P X in place: a wave owns 16 columns, and has read them before it writes
        const float f = t == 0 ? rho : 1.f;
        for (int cb = wave; cb < nt; cb += NW) {
            float x[16];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < mt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[k * 4 + r] = X[(16 * k + 4 * g + r) * pn + cb * 16 + r16];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < mt) {
                    cb_f32x4 acc{0.f, 0.f, 0.f, 0.f}, acc2{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < mt) {
                            const float4 p = *reinterpret_cast<const float4*>(P + (i * 16 + r16) * pm + 16 * k + 4 * g);
                            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(p.x, x[k * 4], acc, 0, 0, 0);
                            acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(p.y, x[k * 4 + 1], acc2, 0, 0, 0);
                            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(p.z, x[k * 4 + 2], acc, 0, 0, 0);
                            acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(p.w, x[k * 4 + 3], acc2, 0, 0, 0);
                        }
#pragma unroll
                    for (int r = 0; r < 4; ++r) X[(i * 16 + 4 * g + r) * pn + cb * 16 + r16] = f * (acc[r] + acc2[r]);
                }
        }
        __syncthreads();
    }
    ns_one_each(rows, cols, [&](int r, int c, int e) CB_INLINE_LAMBDA {
        const float v = X[tall ? c * pn + r : r * pn + c];
        if (BF) static_cast<uint16_t*>(dst)[base + e] = f2bf(v);
        else static_cast<float*>(dst)[base + e] = v;
    });
}

// ------------------------------------------------------------------ host: shapes, layout, launches


int64_t up(int64_t v, int64_t k) { return (v + k - 1) / k * k; }
int64_t a256(int64_t v) { return up(v, 256); }

// Which way a batch goes: the one launch where it fits, unless few matrices have so much work that the other
// way, which spreads one over several CUs, is the faster (8 x 320x64: 69 against 73 us, 8 x 432x64: 88 against
// 73, 64 x 432x64: 90 against 95; 4 x 144x16: 15 against 61).
bool ns_one(int64_t batch, int rows, int cols) {
    const int64_t m = up(std::min(rows, cols), 16), n = up(std::max(rows, cols), 16);
    return m <= 64 && ns_one_lds(rows, cols) <= 160 * 1024 && (batch >= 64 || m * m * n <= 64 * 64 * 320);
}

// Tiles of the m x m products: the smallest whose workgroups do not outnumber the CUs, one a CU (of 32: two).
// Measured, one product: m = 256, tiles of 32 and 64: 4.9 and 7.3 us; 768 (300 and 78 tiles): 8.6 and 11.2,
// two matrices (600 and 156): 15.3 and 13.1; 1024, tiles of 64 and 128: 13.7 and 24.9, two matrices (272 and
// 72): 24 and 25; 2816, 128 and 192 (253 and 120): 66 and 106; 4096 (561 and 253): 192 a fifth faster. Sides
// below 1024 would be padded too far by 192.
int ns_bt(int m, int64_t batch) {
    auto tiles = [&](int bt) { const int64_t t = (m + bt - 1) / bt; return batch * t * (t + 1) / 2; };
    return tiles(32) <= 2 * kNsCus ? 32 : tiles(64) <= kNsCus ? 64 : tiles(128) <= kNsCus || m < 1024 ? 128 : 192;
}

void ns_shape(NsGroup& G, int rows, int cols, int batch) {
    G.rows = rows; G.cols = cols; G.batch = batch;
    G.tall = rows > cols;
    G.m = std::min(rows, cols); G.n = std::max(rows, cols);
    G.small = G.m <= 64;
    G.bt = G.small ? 64 : ns_bt(G.m, batch);
    G.bg = std::max(G.bt, 64);
    // tiles of Q X: the same rule on their own number
    const int64_t wide = int64_t(batch) * ((rows + 63) / 64) * ((cols + 63) / 64);
    G.ba = G.bt == 192 ? 192 : G.small || (wide <= kNsCus && G.bt <= 64) ? 64 : 128;
    const int pad = std::max(G.bg, G.ba);
    G.rp = int(up(rows, pad)); G.cp = int(up(cols, pad));
    G.mp = std::min(G.rp, G.cp); G.np = std::max(G.rp, G.cp);
    auto triangle = [](int t) { return t * (t + 1) / 2; };
    G.tiles = triangle(G.mp / G.bt);
    G.gtiles = triangle(G.mp / G.bg);
    // the Gram product's k in splits of at least two 64-blocks, towards what the CUs hold
    const int nb = G.np / 64;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(std::max(1, nb / 2),
                                                                kNsCus / (int64_t(batch) * G.gtiles)));
    const int each = int((nb + want - 1) / want);
    G.kchunk = each * 64;
    G.splits = (nb + each - 1) / each;
    // blocks of the sums: 8192 elements each, at most 1024 in all and 4 a thread of what adds them up
    G.nsum = int(std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1, 1024 / batch), int64_t(rows) * cols / 8192)));
    G.ldx = G.cp; G.ldt = G.rp; G.ldm = G.mp;
    G.xs = int64_t(G.rp) * G.ldx * 2;
    G.ts = int64_t(G.cp) * G.ldt * 2;
    G.ms = int64_t(G.mp) * G.ldm * 2;
    G.ps = int64_t(G.splits) * G.gtiles * G.bg * G.bg * 4;
    G.scale = 1.f;
}

// Steps in one segment at most.
int ns_most(int prec) { return prec == BF16 ? kSegBf16 : kSegF32; }

// Lays the group's buffers out from `at`; np0: planes of X as it comes; two: a second X buffer.
int64_t ns_layout(NsGroup& G, int64_t at, int np0, bool two) {
    auto take = [&](int64_t bytes) { const int64_t o = at; at += a256(bytes); return o; };
    const bool big = !G.small;
    for (int k = 0; k < 2; ++k) {
        int64_t* x = k ? G.xt : G.x;
        const int64_t plane = G.batch * (k ? G.ts : G.xs);
        x[0] = take(plane * (two ? 2 : np0));   // a later segment may write it with both planes
        x[1] = take(two ? plane * 2 : 0);
    }
    G.part = take(G.batch * G.ps);
    const int64_t mm = G.batch * G.ms * 2;
    G.q[0] = take(mm);
    G.q[1] = take(big ? mm : 0);
    G.a = take(big ? mm : 0);
    G.t = take(big ? mm : 0);
    G.p = take(big ? mm : 0);
    G.v = take(big ? mm : 0);
    return at;
}

struct NsProgram {
    int nseg;
    NsSeg seg[kMaxSegs];
    double xscale[kMaxSegs];   // scale of X after segment i
};

double pow2_scale(double bound, int most) {   // the largest power of two (at most 2^most) with bound * it <= 2^15
    const double e = std::floor(15.0 - std::log2(std::max(bound, 1e-30)));
    return std::exp2(std::min<double>(e, most));
}

// The segments of `steps` steps and the scales of their matrices, from bounds on the singular values:
// they start at one at most, and a step maps them by s -> s (a + b s^2 + c s^4). False, and P is not to be
// run, where they could grow past 2^10 (planes would no longer resolve them), or a segment's product of
// polynomials past 10^15, or where they shrink what the planes hold too far. Which steps share a segment
// depends on `most`, so what one length accepts another may not.
bool ns_program(int steps, const float* coeffs, int most, NsProgram& P) {
    P.nseg = (steps + most - 1) / most;
    double s = 1.0 + 0x1p-10;
    int at = 0;
    for (int k = 0; k < P.nseg; ++k) {
        NsSeg& g = P.seg[k];
        std::memset(&g, 0, sizeof(g));
        g.len = (steps - at + P.nseg - k - 1) / (P.nseg - k);
        double amax = s * s, pmax = 0, tmax = 0, q = 1, qmax = 0;
        double av[kSegBf16], pv[kSegBf16], qv[kSegBf16];   // each step's bounds on A, P and Q
        const int first = at;
        for (int t = 0; t < g.len; ++t, ++at) {
            const float* c = coeffs ? coeffs + 3 * at : kNsDefault;
            const double a = c[0], b = c[1], cc = c[2], lam = s * s;
            for (int i = 0; i < 3; ++i) g.c[t][i] = c[i];
            auto poly = [&](double l) { return std::fabs(a + b * l + cc * l * l); };
            double p = std::max(poly(0), poly(lam));
            if (cc != 0) {
                const double v = -b / (2 * cc);
                if (v > 0 && v < lam) p = std::max(p, poly(v));
            }
            // extrema of s (a + b s^2 + c s^4): a + 3 b l + 5 c l^2 = 0 with l = s^2
            double ns = s * poly(lam);
            auto extremum = [&](double l) { if (l > 0 && l < lam) ns = std::max(ns, std::sqrt(l) * poly(l)); };
            const double d = 9 * b * b - 20 * cc * a;
            if (cc != 0 && d >= 0) {
                extremum((-3 * b + std::sqrt(d)) / (10 * cc));
                extremum((-3 * b - std::sqrt(d)) / (10 * cc));
            } else if (cc == 0 && b != 0) {
                extremum(-a / (3 * b));
            }
            q *= p;
            av[at - first] = lam; pv[at - first] = p; qv[at - first] = q;
            pmax = std::max(pmax, p); qmax = std::max(qmax, q); tmax = std::max(tmax, lam * p);
            s = ns * (1 + 0x1p-10);
            if (!(s <= 1024.0) || !(qmax <= 1e15)) return false;
            if (t + 1 < g.len) amax = std::max(amax, s * s);
        }
        g.sa = float(pow2_scale(amax, 14));
        g.sp = float(pow2_scale(pmax, 14));
        g.st = float(pow2_scale(tmax, 14));
        g.sq = float(pow2_scale(qmax, 14));
        double v = 0;
        for (int t = 1; t < g.len; ++t) v = std::max(v, double(std::fabs(g.c[t][1])) + std::fabs(g.c[t][2]) * amax);
        g.su = float(pow2_scale(pmax * qmax, 14));
        g.sv = float(pow2_scale(qmax * v, 14));
        P.xscale[k] = pow2_scale(s, 12);
        // Planes hold 22 bits of what is 2^-3 or more under its scale (f16's smallest step is 2^-24). Every
        // matrix of the segment has one scale for all steps, so a step that shrinks it too far is refused; of V
        // = b Q + c A' Q it is what A' V adds to the next Q that counts.
        auto held = [](double bound, double scale) { return bound * scale >= 0x1p-3; };
        for (int t = 0; t < g.len; ++t) {
            const bool more = t + 1 < g.len;
            if (!held(av[t], g.sa) || !held(pv[t], g.sp) || !held(qv[t], g.sq) || (t > 0 && !held(qv[t], g.sv / amax)) ||
                (more && (!held(av[t] * pv[t], g.st) || !held(pv[t] * qv[t], g.su))))
                return false;
        }
        if (at < steps && !held(s, P.xscale[k])) return false;
        g.alpha = k == 0 ? 0.f : float(1.0 / (P.xscale[k - 1] * P.xscale[k - 1]));
    }
    return true;
}

// The groups of `a` that `take` accepts, with `blocks` workgroups each.
template <class Take, class Blocks>
NsArgs ns_select(const NsArgs& a, Take&& take, Blocks&& blocks, int& total) {
    NsArgs r = a;
    r.ng = 0;
    total = 0;
    for (int g = 0; g < a.ng; ++g)
        if (take(a.g[g])) {
            r.g[r.ng] = a.g[g];
            r.start[r.ng++] = total;
            total += blocks(a.g[g]);
        }
    r.start[r.ng] = total;
    return r;
}

#define NS_LAUNCH(K, N, LDS, ...) hipLaunchKernelGGL(K, dim3(unsigned(N)), dim3(256), LDS, s, __VA_ARGS__)
#define NS_TILES(K, N, LDS, ...) hipLaunchKernelGGL(K, dim3(unsigned(N)), dim3(64 * NsWaves<BT>::NW), LDS, s, __VA_ARGS__)

template <int BT, int BK, int ST>
void ns_gram(const NsArgs& a, const NsSeg& g, int src, int np, hipStream_t s) {
    int n;
    const NsArgs r = ns_select(a, [](const NsGroup& G) { return G.bg == BT; },
                               [](const NsGroup& G) { return G.batch * G.gtiles * G.splits; }, n);
    if (!n) return;
    if (np == 1) NS_TILES((ns_gram_kernel<BT, 64, ST, 1>), n, (ns_lds_bytes<BT, 64, ST, 1, 1>()), r, g, src);
    else NS_TILES((ns_gram_kernel<BT, BK, ST, 2>), n, (ns_lds_bytes<BT, BK, ST, 2, 2>()), r, g, src);
}

// Whether a group of a float32 call sums its chain's cross products apart (ns_gemm). Below m = 512 the plain
// sums are off by more than a float32 evaluation of the steps, from there on by less, as its own sums get longer:
// 3872 x 256 1.31 to 1.5 times as much as that (1.07 with CROSS, 1 % slower), 70 x 200x260 1.35 (1.08, 4 %),
// 12 x 400x2000 1.11 (0.81, 3 %); 512 x 512 0.94 (0.70, 2 %), 2 x 1001x1531 0.85 (0.63, 6 %), 3000 x 2000 0.77
// (0.61, 6 %).
bool ns_cross(const NsGroup& G) { return G.m < 512; }

template <int BT, int BK, int ST, bool CROSS>
void ns_prod(const NsArgs& a, const NsJobs& jobs, bool f32, hipStream_t s) {
    int n;
    const NsArgs r = ns_select(a, [&](const NsGroup& G) { return G.bt == BT && !G.small && (f32 && ns_cross(G)) == CROSS; },
                               [&](const NsGroup& G) { return G.batch * G.tiles * jobs.n; }, n);
    if (n) NS_TILES((ns_prod_kernel<BT, BK, ST, CROSS>), n, (ns_lds_bytes<BT, BK, ST, 2, 2>()), r, jobs);
}

template <int BT, int BK, int ST>
void ns_apply(const NsArgs& a, const NsApply& ap, int np, hipStream_t s) {
    int n;
    const NsArgs r = ns_select(a, [](const NsGroup& G) { return G.ba == BT; },
                               [](const NsGroup& G) { return G.batch * (G.rp / BT) * (G.cp / BT); }, n);
    if (!n) return;
    if constexpr (BT == 64 && ST > 2)
        // More tiles than CUs: two stages, so that a CU holds two of them and there is no second round (the base
        // net's 305: 14 -> 11 us; the 244 of 3872 x 256 take 0.4 us longer with two).
        if (n > kNsCus) {
            ns_apply<BT, BK, 2>(a, ap, np, s);
            return;
        }
    if (np == 1) NS_TILES((ns_apply_kernel<BT, BK, ST, 1>), n, (ns_lds_bytes<BT, BK, ST, 2, 1>()), r, ap);
    else NS_TILES((ns_apply_kernel<BT, BK, ST, 2>), n, (ns_lds_bytes<BT, BK, ST, 2, 2>()), r, ap);
}

// The m x m products of a segment; returns which Q buffer holds Q. f32: of a float32 call.
int ns_chain(const NsArgs& a, const NsSeg& g, bool f32, hipStream_t s) {
    auto run = [&](const NsJobs& j) {
        ns_prod<32, 64, 4, false>(a, j, f32, s);
        ns_prod<32, 64, 4, true>(a, j, f32, s);
        ns_prod<64, 64, 4, false>(a, j, f32, s);
        ns_prod<64, 64, 4, true>(a, j, f32, s);
        ns_prod<128, 32, 4, false>(a, j, f32, s);
        ns_prod<128, 32, 4, true>(a, j, f32, s);
        ns_prod<192, 32, 3, false>(a, j, f32, s);   // (m >= 1024)
    };
    // the first P is Q
    run({1, {{NS_A, NS_A, NS_Q0, NS_A, g.sq * g.c[0][2] / (g.sa * g.sa), g.sq * g.c[0][1] / g.sa, g.sq * g.c[0][0]}}});
    // The chip holds two products at once (m = 256: two cost 5.2 us, one 5.1; at m = 512, 272 tiles, 8.1 and
    // 6.4, and both ways take the same time).
    bool wide = true;
    for (int i = 0; i < a.ng; ++i) wide = wide && (a.g[i].small || 2 * int64_t(a.g[i].batch) * a.g[i].tiles <= kNsCus);
    if (wide) {
        // A step more in three launches of two products each, where the other way takes four: with R = P A and
        // U = P Q the next A is A' = R P, and the next Q = P' Q = a Q + A' (b Q + c A' Q), A' Q = R U; the P'
        // of a step after that goes with it. What was read last is written next; A' takes A's place.
        int q = NS_Q0, p = NS_Q0, r = NS_Q1, u = NS_T, v = NS_P;
        float sp = g.sq;
        for (int t = 1; t < g.len; ++t) {
            const float ca = g.c[t][0], cb = g.c[t][1], cc = g.c[t][2];
            run({2, {{p, q, u, NS_A, g.su / (sp * g.sq), 0.f, 0.f}, {p, NS_A, r, NS_A, g.st / (sp * g.sa), 0.f, 0.f}}});
            run({2, {{r, p, NS_A, NS_A, g.sa / (g.st * sp), 0.f, 0.f},
                     {r, u, v, q, cc * g.sv / (g.st * g.su), cb * g.sv / g.sq, 0.f}}});
            run({t + 1 < g.len ? 2 : 1, {{NS_A, v, r, q, g.sq / (g.sa * g.sv), ca, 0.f},
                                         {NS_A, NS_A, u, NS_A, g.sp * cc / (g.sa * g.sa), g.sp * cb / g.sa, g.sp * ca}}});
            const int q0 = q, u0 = v;
            q = r; p = u; r = q0; u = t == 1 ? u0 : u == NS_T ? NS_P : NS_T; v = NS_V;
            sp = g.sp;
        }
        return q == NS_Q1;
    }
    int q = 0;
    for (int t = 0; t < g.len; ++t) {
        const float sd = t == 0 ? g.sq : g.sp;
        const int p = t == 0 ? NS_Q0 : NS_P;
        if (t > 0)
            run({1, {{NS_A, NS_A, p, NS_A, sd * g.c[t][2] / (g.sa * g.sa), sd * g.c[t][1] / g.sa, sd * g.c[t][0]}}});
        NsJobs j{};
        if (t > 0) {
            j.j[j.n++] = {NS_P, q ? NS_Q1 : NS_Q0, q ? NS_Q0 : NS_Q1, NS_A, 1.f / g.sp, 0.f, 0.f};
            q ^= 1;
        }
        if (t + 1 < g.len) j.j[j.n++] = {p, NS_A, NS_T, NS_A, g.st / (sd * g.sa), 0.f, 0.f};
        if (j.n) run(j);
        if (t + 1 < g.len) run({1, {{NS_T, p, NS_A, NS_A, g.sa / (g.st * sd), 0.f, 0.f}}});
    }
    return q;
}

// All segments of one pass, X's planes (np of them) in place; `last` describes the final output.
hipError_t ns_run(const NsArgs& a, const NsProgram& P, int np, NsApply last, hipStream_t s) {
    int src = 0;
    for (int k = 0; k < P.nseg; ++k) {
        const NsSeg& g = P.seg[k];
        ns_gram<64, 64, 4>(a, g, src, np, s);
        ns_gram<128, 32, 4>(a, g, src, np, s);
        ns_gram<192, 32, 3>(a, g, src, np, s);
        int n;
        const NsArgs r = ns_select(a, [](const NsGroup& G) { return G.small || G.splits > 1; }, [](const NsGroup& G) {
            return G.small ? G.batch : G.batch * G.gtiles * (G.bg / 16);
        }, n);
        bool small = false;
        for (int i = 0; i < a.ng; ++i) small = small || a.g[i].small;
        if (n && small) hipLaunchKernelGGL(ns_reduce_kernel<kSmThreads>, dim3(unsigned(n)), dim3(kSmThreads), kSmLds, s, r, g);
        else if (n) NS_LAUNCH(ns_reduce_kernel<256>, n, 256 * 17 * int(sizeof(float)), r, g);
        const int q = ns_chain(a, g, last.out != NS_OUT_BF16, s);
        const bool end = k + 1 == P.nseg;
        NsApply ap = last;
        if (!end) ap.out = NS_OUT_MID;
        ap.src = src; ap.dst = src ^ 1; ap.q = q;
        ap.use_inv = k == 0;
        ap.f = float((end ? 1.0 : P.xscale[k]) / (double(g.sq) * (k == 0 ? 1.0 : P.xscale[k - 1])));
        ns_apply<64, 64, 4>(a, ap, np, s);
        ns_apply<128, 32, 4>(a, ap, np, s);
        ns_apply<192, 32, 3>(a, ap, np, s);
        src ^= 1;
        np = 2;
    }
    return hipGetLastError();
}

int64_t orth_layout(int prec, int64_t batch, int rows, int cols, int steps, NsArgs& a) {
    std::memset(&a, 0, sizeof(a));
    a.ng = 1;
    NsGroup& G = a.g[0];
    ns_shape(G, rows, cols, int(batch));
    a.info = 0;
    a.sums = a256(batch * 8);
    return ns_layout(G, a.sums + a256(batch * G.nsum * 24), prec == BF16 ? 1 : 2, steps > ns_most(prec));
}

}  // namespace

bool muon_coeffs_ok(int prec, int steps, const float* coeffs) {
    NsProgram P{};
    return ns_program(steps, coeffs, ns_most(prec), P);
}

bool muon_orth_small(int64_t batch, int rows, int cols) { return ns_one(batch, rows, cols); }

size_t muon_orth_ws_bytes(int prec, int64_t batch, int rows, int cols, int steps) {
    if (ns_one(batch, rows, cols)) return 256;   // nothing; but zero stands for a refusal
    NsArgs a;
    return size_t(orth_layout(prec, batch, rows, cols, steps, a));
}

hipError_t muon_orth(int prec, int64_t batch, int rows, int cols, const void* x, int steps, const float* coeffs,
                     float eps, void* y, void* ws, hipStream_t s) {
    ProfScope ps(s, [&] { return cb_key("muon_orthogonalize", prec, cb_dims(rows, cols) + "x" + std::to_string(batch)); });
    if (ns_one(batch, rows, cols)) {
        NsOne o{rows, cols, steps, eps, {}};
        for (int t = 0; t < steps; ++t)
            for (int i = 0; i < 3; ++i) o.c[t][i] = coeffs ? coeffs[3 * t + i] : kNsDefault[i];
        const unsigned lds = unsigned(ns_one_lds(rows, cols));
        if (prec == BF16) hipLaunchKernelGGL(ns_one_kernel<true>, dim3(unsigned(batch)), dim3(kSmThreads), lds, s, x, y, o);
        else hipLaunchKernelGGL(ns_one_kernel<false>, dim3(unsigned(batch)), dim3(kSmThreads), lds, s, x, y, o);
        return hipGetLastError();
    }
    NsArgs a;
    orth_layout(prec, batch, rows, cols, steps, a);
    a.ws = static_cast<char*>(ws);
    NsProgram P{};
    if (!ns_program(steps, coeffs, ns_most(prec), P)) return hipErrorInvalidValue;
    const NsGroup& G = a.g[0];
    MuonElem e{};
    const int64_t sums = batch * G.nsum, planes = batch * int64_t(ns_plane_blocks(G));
    if (prec == BF16) {
        NS_LAUNCH((ns_sums_kernel<NS_SRC_BF16>), sums, 0, a, e, x, 0);
        NS_LAUNCH((ns_planes_kernel<NS_SRC_BF16, 1>), planes, 0, a, e, x, eps, 0);
    } else {
        NS_LAUNCH((ns_sums_kernel<NS_SRC_F32>), sums, 0, a, e, x, 0);
        NS_LAUNCH((ns_planes_kernel<NS_SRC_F32, 2>), planes, 0, a, e, x, eps, 0);
    }
    NsApply ap{};
    ap.out = prec == BF16 ? NS_OUT_BF16 : NS_OUT_F32;
    ap.y = y;
    return ns_run(a, P, prec == BF16 ? 1 : 2, ap, s);
}

// ------------------------------------------------------------------ the step over the flat buffer

namespace {

struct MuonPlan {
    struct Pass { NsArgs a; MuonElem e; int block0, sums, planes; };
    std::vector<Pass> pass;
    int nblocks = 0;
    int64_t total = 0;
};

// Passes of at most kNsMats matrices in kNsGroups shapes; each also has the gaps that lie before its
// matrices in the buffer (the last one those after). `mats` sorted by offset.
MuonPlan muon_plan(int64_t n_params, const std::vector<MuonMat>& mats, int steps, int scale_mode) {
    MuonPlan plan;
    int64_t at = 0;
    size_t i = 0;
    int first = 0;
    do {
        MuonPlan::Pass P;
        std::memset(&P, 0, sizeof(P));
        struct Shape { int rows, cols; std::vector<int64_t> off; };
        std::vector<Shape> shapes;
        auto gap = [&](int64_t to) {
            if (to > at) {
                P.e.gap[P.e.ngaps] = at;
                P.e.gap_len[P.e.ngaps++] = to - at;
            }
        };
        int count = 0;
        for (; i < mats.size() && count < kNsMats; ++i, ++count) {
            size_t k = 0;
            while (k < shapes.size() && !(shapes[k].rows == mats[i].rows && shapes[k].cols == mats[i].cols)) ++k;
            if (k == shapes.size()) {
                if (k == size_t(kNsGroups)) break;
                shapes.push_back({mats[i].rows, mats[i].cols, {}});
            }
            shapes[k].off.push_back(mats[i].offset);
            gap(mats[i].offset);
            at = mats[i].offset + int64_t(mats[i].rows) * mats[i].cols;
        }
        if (i == mats.size()) {
            gap(n_params);
            at = n_params;
        }
        P.block0 = plan.nblocks;
        int o = 0;
        for (const Shape& sh : shapes) {
            NsGroup& G = P.a.g[P.a.ng];
            ns_shape(G, sh.rows, sh.cols, int(sh.off.size()));
            G.first = first + o;
            G.table = 1 + o;
            for (int64_t f : sh.off) P.a.off[o++] = f;
            // the spectral norm that keeps a layer's output as large as its input, or the root mean
            // square of an Adam update
            const double fi = sh.rows, fo = sh.cols;
            G.scale = float(scale_mode == 0 ? std::sqrt(std::max(1.0, fo / fi)) : 0.2 * std::sqrt(std::max(fi, fo)));
            P.a.start[P.a.ng++] = P.sums;
            G.part0 = P.block0 + P.sums;
            P.sums += G.batch * G.nsum;
            P.planes += G.batch * ns_plane_blocks(G);
        }
        P.a.start[P.a.ng] = P.sums;
        first += o;
        for (int k = 0; k < P.e.ngaps; ++k) {   // 4096 elements a block, at most 256 a gap
            P.e.gap_start[k + 1] =
                P.e.gap_start[k] + int(std::max<int64_t>(1, std::min<int64_t>(256, (P.e.gap_len[k] + 4095) / 4096)));
        }
        P.sums += P.e.gap_start[P.e.ngaps];
        P.planes += P.e.gap_start[P.e.ngaps];
        plan.nblocks += P.sums;
        plan.pass.push_back(P);
    } while (i < mats.size());
    const int64_t sums = a256(int64_t(first) * 8), base = sums + a256(int64_t(plan.nblocks) * 24);
    for (MuonPlan::Pass& P : plan.pass) {
        P.a.info = 0;
        P.a.sums = sums;
        int64_t end = base;   // passes follow each other in the same memory
        for (int g = 0; g < P.a.ng; ++g) end = ns_layout(P.a.g[g], end, 2, steps > kSegF32);
        plan.total = std::max(plan.total, end);
        P.e.nblocks = plan.nblocks;
    }
    return plan;
}

}  // namespace

size_t muon_step_ws_bytes(int64_t n_params, const std::vector<MuonMat>& mats, int steps) {
    return size_t(muon_plan(n_params, mats, steps, 0).total);
}

hipError_t muon_update(const MuonStep& m, const std::vector<MuonMat>& mats, void* ws, hipStream_t s) {
    if (m.n <= 0) return hipSuccess;
    MuonPlan plan = muon_plan(m.n, mats, m.steps, m.scale_mode);
    NsProgram P{};
    if (!ns_program(m.steps, m.coeffs, kSegF32, P)) return hipErrorInvalidValue;
    ProfScope ps(s, [&] { return "muon/" + std::to_string(m.n); });
    for (MuonPlan::Pass& p : plan.pass) {
        p.a.ws = static_cast<char*>(ws);
        MuonElem& e = p.e;
        const OptArgs& o = m.adam;
        e.p = o.p; e.g = o.g; e.m = o.m; e.v = o.v;
        e.mu = m.momentum; e.omu = m.omu; e.nesterov = m.nesterov;
        e.c1 = m.nesterov ? m.omu * (1.f + m.momentum) : m.omu;
        e.c2 = m.nesterov ? m.momentum * m.momentum : m.momentum;
        e.b1 = o.b1; e.b2 = o.b2; e.omb1 = o.omb1; e.omb2 = o.omb2; e.bc1 = o.bc1; e.bc2 = o.bc2;
        e.alr = o.lr; e.aeps = o.eps; e.max_norm = o.max_norm; e.eps = m.eps;
        e.stats = m.stats; e.mir = o.mir; e.mir_off = o.mir_off; e.mir_len = o.mir_len;
        NS_LAUNCH((ns_sums_kernel<NS_SRC_STEP>), p.sums, 0, p.a, e, nullptr, p.block0);
    }
    for (const MuonPlan::Pass& p : plan.pass) {
        // the planes' blocks by group, then the gaps' (counted from start[ng])
        int n;
        const NsArgs r = ns_select(p.a, [](const NsGroup&) { return true; }, [](const NsGroup& G) {
            return G.batch * ns_plane_blocks(G);
        }, n);
        NS_LAUNCH((ns_planes_kernel<NS_SRC_STEP, 2>), p.planes, 0, r, p.e, nullptr, 0.f, p.block0);
        if (p.a.ng == 0) continue;
        NsApply ap{};
        ap.out = NS_OUT_STEP;
        ap.p = m.adam.p;
        ap.decay = m.decay; ap.lr = m.lr;
        ap.mir = m.adam.mir; ap.mir_off = m.adam.mir_off; ap.mir_len = m.adam.mir_len;
        const hipError_t err = ns_run(p.a, P, 2, ap, s);
        if (err != hipSuccess) return err;
    }
    return hipGetLastError();
}

}  // namespace cb
