// Norm of each head of queries and keys with the position rotation, and its backward
// pass: shapes, plan and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "wino_norm.h"

namespace wino {

// One of the two tensors: [N][L][heads][D], tokens ld elements apart.
struct QkSide {
    const void *x, *dy;
    const float* gamma;                      // [D] or null
    const int* pos;                          // [N][L] rows of the table, or null: token t is at t
    void* y;                                 // forward, [N][L][heads][D]
    void* dx;                                // backward, as x
    float* dgamma;                           // [D] or null
    int L, heads, ld;
};
struct QkShape {
    int N, D, R, T;                          // R channels rotated, by a table of T rows
    bool pairs;                              // channels 2i, 2i+1 turn together, else i, i + R/2
    float eps;
    const float* rot;                        // [T][R/2][2] of cos, sin
    Io io;
};

// A team of `team` lanes has a token's vectors of `heads` heads, in turn, `vp` pairs of
// channels a lane.
struct QkPlan {
    bool fits;
    int vp, team, blocks[2];                 // workgroups of each tensor
    int64_t items[2];
    size_t need;
};
QkPlan qk_plan(const QkShape& s, const QkSide (&t)[2], bool backward);
hipError_t launch_qk_norm(const QkShape& s, const QkSide (&t)[2], const QkPlan& p, hipStream_t st);
hipError_t launch_qk_norm_backward(const QkShape& s, const QkSide (&t)[2], const QkPlan& p, void* ws, hipStream_t st);

}  // namespace wino
