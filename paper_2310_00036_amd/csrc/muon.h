// Internal interface of the orthogonalised updates (muon.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "kernels.h"

namespace cb {

// Orthogonalised updates (Newton-Schulz products) and the Muon step:
// steps in [1, 16]; coeffs: host [steps][3] or NULL (the default quintic in every step)
// Whether singular values and the products of a segment's polynomials stay bounded (muon_update: as float32).
bool muon_coeffs_ok(int prec, int steps, const float* coeffs);
bool muon_orth_small(int64_t batch, int rows, int cols);   // one launch, no workspace
size_t muon_orth_ws_bytes(int prec, int64_t batch, int rows, int cols, int steps);
hipError_t muon_orth(int prec, int64_t batch, int rows, int cols, const void* x, int steps, const float* coeffs,
                     float eps, void* y, void* ws, hipStream_t s);
struct MuonMat { int64_t offset; int rows, cols; };   // a matrix of the flat buffer
struct MuonStep {
    int64_t n;
    OptArgs adam;             // buffers, the clip, Adam's constants for what no matrix covers, the mirror
    float lr, decay;          // p <- decay p - lr scale O
    float momentum, omu;      // momentum, 1 - momentum (formed in double)
    int nesterov, steps, scale_mode;
    float eps;
    const float* coeffs;
    float* stats;
};
size_t muon_step_ws_bytes(int64_t n_params, const std::vector<MuonMat>& mats, int steps);
// mats sorted by offset, disjoint.
hipError_t muon_update(const MuonStep& m, const std::vector<MuonMat>& mats, void* ws, hipStream_t s);

constexpr int kNsGroups = 8;       // shapes per pass
constexpr int kNsMats = 64;        // matrices with offsets of their own per pass
constexpr int kNsMaxSteps = 16;

// Matrices of one shape. rp x cp: the shape padded to whole tiles; m <= n the sides, mp and np padded.
struct NsGroup {
    int rows, cols, rp, cp, m, n, mp, np, tall;   // tall: rows > cols
    int batch, first;                 // first: index of its first matrix in the call
    int small;                        // m <= 64: the m x m part in one workgroup
    int bt, bg, ba;                   // tiles of the m x m products (32 to 192), of the Gram product, of Q X
    int tiles, gtiles, splits, kchunk;   // tiles of symmetric m x m products; the Gram product's k split
    int table, nsum, part0;           // 1 + its first offset in NsArgs::off (0: b * rows * cols); its blocks of the sums
    float scale;                      // the update's factor (muon_step)
    int64_t x[2], xt[2], part, a, t, p, v, q[2];   // workspace byte offsets of the first matrix (xt: X transposed)
    int ldx, ldt, ldm;                   // leading dimensions of X, its transpose and the m x m matrices
    int64_t xs, ts, ms, ps;              // bytes of one plane of each, and of one matrix's partials
};

struct NsArgs {
    NsGroup g[kNsGroups];
    int64_t off[kNsMats];             // element offsets of matrices with a table
    int ng;
    int start[kNsGroups + 1];         // workgroups of this launch by group
    char* ws;
    int64_t info, sums;               // workspace byte offsets: two floats a matrix; 3 doubles a block of the sums
};

struct MuonElem {                     // the elementwise part of muon_step
    float* p; const float* g; float* m; float* v;
    float mu, omu, c1, c2;            // momentum, 1 - momentum; u = c1 s g + c2 m
    int nesterov;
    float b1, b2, omb1, omb2, bc1, bc2, alr, aeps;   // Adam for the rest
    float max_norm, eps;
    float* stats;
    uint16_t* mir; int64_t mir_off, mir_len;
    int nblocks;                      // blocks of the sums in the whole call
    int64_t gap[kNsMats + 1], gap_len[kNsMats + 1];   // what no matrix covers
    int ngaps, gap_start[kNsMats + 2];
};

}  // namespace cb
