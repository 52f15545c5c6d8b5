// The gated layer of channel-last tensors and its backward pass: shapes, plan, launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "wino_norm.h"

namespace wino {

// y[m][f] = act(x w0^T + b0) * (x w1^T + b1); x [M][C], w [2][K][C], b [2][K].
struct GatedShape {
    int64_t M;
    int C, K;
    Io io;
    Act act;
};
struct GatedArgs {
    const void *dy, *x, *w;
    const float* bias;                       // or null
    void *y, *dx, *dw;                       // dx, dw, dbias: null if not wanted
    float* dbias;
};
struct GatedPlan {
    bool fits;
    int first, dx, dw;                       // tile shapes of the products
    int dx_splits, dw_splits;                // parts of the sums over units and over tokens
    size_t dz, dbias, px, pw, tops, need;    // workspace: bytes of each region
};
GatedPlan gated_plan(const GatedShape& s, bool backward);
int gated_results(int shape);                // of a workgroup's tile
bool gated_few(const GatedShape& s);         // forward: a wave for each unit
hipError_t launch_gated(const GatedArgs& a, const GatedShape& s, const GatedPlan& p, hipStream_t st);
hipError_t launch_gated_backward(const GatedArgs& a, const GatedShape& s, const GatedPlan& p, void* ws, hipStream_t st);

}  // namespace wino
