// Internal interface of the linear attention with a decay per head (linattn.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cb {

// One pass of the recurrence  R_p = keep_p R_{p-1} + in k_p v_p^T,  o_p = out R_p^T q_p  over the rows p = 0 .. T-1 of a
// rollout: in its order (p = t), or backwards (p = T-1-t), which is what the gradients are. An episode start at t cuts
// between t-1 and t, whichever way the rows run. q, k [T, E, H, dk], v, o [T, E, H, dv], element strides for step, env
// and head.
struct LaView { const void* p; int64_t t, e, h; };
struct LaPass {
    LaView q, k, v;
    LaView o;                  // written
    const float* x0;           // [E, H, dk, dv] or NULL (zeros): R before the first row; backwards: added to its R
    float* x1;                 // or NULL: R of the last row; backwards: keep R as it leaves the rollout
    int dk, dv, back;
    int xk, xn;                // element strides of a state's two axes
    float in, out;
    int vec;                   // bit 0: o has whole fours of columns; 1: rows end inside a 16-byte piece; 2: all rows are in
                               // a buffer resource's reach
};
constexpr int kLaMaxPasses = 3;
constexpr int kLaMaxDim = 128;
struct LaArgs {
    LaPass pass[kLaMaxPasses];
    int np;
    const float* log_decay;    // [H]
    const uint8_t* dones;      // element strides d_t, d_e; or NULL (no episode starts)
    int64_t d_t, d_e;
    int T, E, H;
};
size_t linattn_ws_bytes(int prec, int T, int E, int H, int dk, int dv, int passes);
// The passes' vec bits are filled in here. ws: linattn_ws_bytes, 16-byte aligned, or NULL where that is zero.
hipError_t linattn(int prec, LaArgs a, void* ws, hipStream_t s);

}  // namespace cb
