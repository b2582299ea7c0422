// Internal interface of the block norms (blocknorm.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cb {

// out = res + rscale (norm(h) gamma + beta) act(gate), out2 = norm2(out) gamma2 + beta2; n rows of C channels, the first
// norm over groups of cg = C / G of them. Every array has its own row stride, in elements.
constexpr int kBnMaxC = 8192;
struct BnMat { void* p; int64_t ld; };
struct BnArgs {
    BnMat h, gate, res, out, out2;            // NULL: gate 1, res 0, no second norm
    BnMat dout, dout2, dh, dgate, dres;       // backward; dout, dgate, dres may be NULL
    const float* gamma; const float* beta; const float* rscale;   // [C]; NULL: 1, 0, 1
    const float* gamma2; const float* beta2;
    float* grads[5];                          // dgamma, dbeta, drscale, dgamma2, dbeta2 [C], or NULL
    int64_t n;
    int C, G, cg;
    int norm, norm2, act;                     // 0 none, 1 layer, 2 rms; act 0 linear, 1 silu, 2 sigmoid
    float eps;
    // filled by the launcher
    int tpr, gb, rb;                          // threads a row (or group) takes; groups and rows a workgroup takes
    float* part;                              // [blocks][5 or 3][C]
};
size_t blocknorm_bwd_ws_bytes(int prec, int64_t n, int C, int G, bool two);
hipError_t blocknorm_fwd(int prec, BnArgs a, hipStream_t s);
hipError_t blocknorm_bwd(int prec, BnArgs a, void* ws, hipStream_t s);   // n == 0: the column sums are cleared

}  // namespace cb
