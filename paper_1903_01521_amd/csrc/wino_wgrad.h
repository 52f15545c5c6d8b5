// Weight gradient of the 3x3 stride-1 layer on channel-last tensors: launchers.
#pragma once

#include "wino_norm.h"

namespace wino {

struct WgradShape {
    int N, C, H, W, K, pad, Ho, Wo;
    Io io;                                   // of dy, and of x
    // the layer's input is act(norm(x)) of G groups; norm false: x itself
    bool norm, x8;
    int G, D;
    Act act;
};

struct WgradArgs {
    const void *x, *dy;
    const int8_t* codes;                     // in place of x, with rows
    const float *rows, *stats, *gamma, *beta;
    float* dg;                               // [K][C][3][3]
};

bool wgrad_fits(const WgradShape& s);        // offsets and counts that the kernel handles
size_t wgrad_workspace(const WgradShape& s);
hipError_t launch_wgrad(const WgradArgs& a, const WgradShape& s, void* ws, hipStream_t st);

}  // namespace wino
