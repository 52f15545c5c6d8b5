// Cross attention of channel-last tokens to an encoder's states, forward and
// backward: shapes, plans and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "wino_norm.h"

namespace wino {

// q [N][Lq][Hq][D], k and v [N][Lk][Hk][D], tokens ld* elements apart; query head h
// reads key head h / rep.  The rows of a (image, key head) pair are its rep * Lq
// query vectors, row t * rep + g being head g of the group at token t.
struct AttnShape {
    int N, Lq, Lk, Hq, Hk, D, rep;
    int64_t rows;                            // of a pair
    int ldq, ldk, ldv;
    float scale;
    Io io;
};

struct AttnArgs {
    const void *q, *k, *v;
    const int* klen;                         // keys of an image, or null
    const uint8_t* mask;                     // [N][Lk], 0: left out; or null
    void* y;                                 // [N][Lq][Hq][D]
    float* lse;                              // [N][Hq][Lq] or null
};

struct AttnBwd {
    const void *dy, *q, *k, *v, *y;
    const float* lse;
    const int* klen;
    const uint8_t* mask;
    void *dq, *dk, *dv;
};

// How a launch is cut: workgroups of `rows` rows (or keys), the other axis in
// `splits` parts whose results another launch joins.
struct AttnCut {
    int64_t tiles;
    int splits;
};
struct AttnPlan {
    bool fits;
    bool few;                                // forward: a workgroup of one wave, 32 rows
    AttnCut rows, keys;                      // of the launch over rows, and backward over keys
    size_t delta, part, stat, need;          // workspace: bytes of each region (16-byte aligned)
};
AttnPlan attn_plan(const AttnShape& s, bool backward);
hipError_t launch_attn(const AttnArgs& a, const AttnShape& s, const AttnPlan& p, void* ws, hipStream_t st);
hipError_t launch_attn_backward(const AttnBwd& a, const AttnShape& s, const AttnPlan& p, void* ws, hipStream_t st);

}  // namespace wino
