// Arguments of the kernels between two blocks (block_norm.inc), and how a backward pass is dealt to workgroups.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_plan.hpp"
#include "philox.hpp"

namespace lrd {

constexpr int64_t BN_MOST_WIDTH = 16384;       // a row in the registers of 1024 threads, 16 columns each

struct BlockNormFwd {
    const void *F, *X;              // F null: Y is X, and not written
    const float *w_post, *b_post, *gate, *w_pre, *b_pre;
    void *Y, *N;
    DropRng rng;
    int64_t T, gate_rows;
    int d;
    bool layer;
    float eps, alpha, beta;
};

struct BlockNormBwd {
    const void *dY, *dN, *F, *Y;    // dY or dN may be null
    const float *w_post, *b_post, *gate, *w_pre;
    void *dX, *dF;                  // nullable
    float *dgate, *gate_partial, *partial;
    bool sums[BN_SUMS];             // which parameters' gradients are wanted
    DropRng rng;
    int64_t T, gate_rows, units, parts, part_rows, workgroups;
    int d;
    bool layer, by_slot, branch, out;
    float eps, alpha, beta;
};

hipError_t block_norm_fwd_bf16(const BlockNormFwd& g, hipStream_t st);
hipError_t block_norm_fwd_f32(const BlockNormFwd& g, hipStream_t st);
hipError_t block_norm_bwd_bf16(const BlockNormBwd& g, hipStream_t st);
hipError_t block_norm_bwd_f32(const BlockNormBwd& g, hipStream_t st);
// Sums of the partial rows: outs[s] (nullable) from partial [workgroups][BN_SUMS][d]; dgate from gate_partial [groups * parts][d].
hipError_t block_norm_sums(const BlockNormBwd& g, float* const (&outs)[BN_SUMS], hipStream_t st);

}  // namespace lrd
