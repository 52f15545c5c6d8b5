// Group norm with an activation, its backward pass and the 8-bit activation
// checkpoint, on channel-last tensors: plan and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace wino {

enum class Io { F32, F16, BF16 };            // element type of the activations
inline int io_size(Io t) { return t == Io::F32 ? 4 : 2; }
enum class Act { None, Relu, Silu };

// A tensor [N][P][C] (P = H*W pixels) in G groups of D = C/G channels.
struct NormShape {
    int N, C, G, D;
    int64_t P;
    Io io;
    Act act;
};

// 8-bit checkpoint of such a tensor: int8 codes [N][P][C], padded to 16 bytes,
// then float rows [N][C][2] of centre and step.
inline size_t act8_rows_at(const NormShape& s) { return ((size_t)s.N * s.P * s.C + 15) / 16 * 16; }
inline size_t act8_size(const NormShape& s) { return act8_rows_at(s) + (size_t)s.N * s.C * 8; }

// How a pass over the tensor is cut.  A workgroup holds `px` pixels of `cb`
// channels in registers, up to `nv` vectors of `vec` channels a thread; its
// threads are `rows` pixels of cv = cb/vec columns (wrows, parts: see Cut).  one:
// px is the whole image and cb whole groups, so that the statistics never leave
// the workgroup; else the image is cut into `chunks` and the statistics are
// joined by a launch in between.
struct NormPlan {
    bool one, fits;                          // fits: below 2^30 workgroups' items
    int vec, nv, threads, cb, cv, rows, wrows, parts, chunks;
    int64_t px;
    size_t lds, need;                        // dynamic LDS, workspace bytes
};

// backward: dy and x are held.  aligned: the tensors are on 16-byte addresses.
NormPlan norm_plan(const NormShape& s, bool backward, bool aligned);

struct NormFwd {
    const void* x;
    const float *gamma, *beta;               // null: 1 and 0
    void* y;                                 // null: only the checkpoint
    float* stats;                            // [N][G][2] of mean and rstd, or null
    int8_t* codes;                           // checkpoint, or null
    float* rows;
    float eps;
};
hipError_t launch_norm(const NormFwd& a, const NormShape& s, const NormPlan& p, void* ws, hipStream_t st);

// y from x (or from a checkpoint: codes and rows) and the statistics; null
// statistics: the values themselves.
struct NormApply {
    const void* x;
    const int8_t* codes;
    const float *rows, *stats, *gamma, *beta;
    void* y;
};
hipError_t launch_norm_apply(const NormApply& a, const NormShape& s, bool aligned, hipStream_t st);

struct NormBwd {
    const void *dy, *x;
    const int8_t* codes;                     // in place of x, with rows
    const float *rows, *stats, *gamma, *beta;
    void* dx;
    float *dgamma, *dbeta;
};
hipError_t launch_norm_backward(const NormBwd& a, const NormShape& s, const NormPlan& p, void* ws, hipStream_t st);

}  // namespace wino
