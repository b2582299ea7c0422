// Internal interface of the group norm (groupnorm.hip). A header of its own, like muon.h: the sources of the
// learner path's kernels, by whose digest their counter figures are current, do not include it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cb {

// Group norm with an activation, channels last; x, y, dy [n, HW, C] in the storage type
constexpr int kGnMaxC = 1024;
struct GnArgs {
    const void* x; const void* dy; void* y;        // backward: y is dx
    const float* gamma; const float* beta;         // [C] or NULL (1, 0)
    float* mean; float* rstd;                      // [n, G]; forward: may be NULL
    float eps;
    int act;                                       // 0 none, 1 relu, 2 silu
    int64_t n;
    int HW, C, G, cg;                              // cg = C / G channels per group
    // filled by the launcher: columns of V channels per pixel, padded to cvp = 2^cvs; pixels and
    // number of a frame's chunks; workspace
    int cv, cvp, cvs, crows, chunks;
    float* part; float* fsum; float* smean; float* srstd;
};
size_t groupnorm_ws_bytes(int prec, int64_t n, int H, int W, int C, int G, int bwd);   // at any alignment
// Whether a forward on these addresses takes a frame a workgroup, and so no workspace.
bool groupnorm_fwd_whole(int prec, int64_t n, int H, int W, int C, int G, const void* x, const void* y);
int64_t groupnorm_threads(int prec, int64_t n, int H, int W, int C, int G);   // of a launch, at most
hipError_t groupnorm_fwd(int prec, int H, int W, GnArgs a, void* ws, hipStream_t s);
// n == 0: dgamma and dbeta are cleared. Either may be NULL.
hipError_t groupnorm_bwd(int prec, int H, int W, GnArgs a, float* dgamma, float* dbeta, void* ws, hipStream_t s);

}  // namespace cb
