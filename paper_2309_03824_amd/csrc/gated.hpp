// The second products of a gated pair and what joins them (gated.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrd {

// Zg = Hg.Ug^T + bg, Zu = Hu.Uu^T + bu from H = [Hg | Hu] [T x 2 r], U [2][out x r], bias [2][out] or null;
// forward (dA null): A = act(Zg) * Zu;  backward: dZ[0] = dA * Zu * act'(Zg), dZ[1] = dA * act(Zg).
struct GatedOp {
    const void *H, *U;
    const float* bias;
    const void* dA;
    void *A, *dZ;               // dZ [2][T x out]
    int64_t T, out, r;
    int act;                    // lrd.h's LRD_ACT_*
    bool bf16;
};
hipError_t run_gated(const GatedOp& op, hipStream_t st);

}  // namespace lrd
