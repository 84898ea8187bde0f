// The second products of a gated pair and what joins them (gated.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrd {

// Zg = Hg.Ug^T + bg, Zu = Hu.Uu^T + bu from H = [Hg | Hu] [T x 2 r], U [2][out x r], bias [2][out] or null;
// forward (dA null): A = act(Zg) * Zu;  backward: dZ[0] = dA * Zu * act'(Zg), dZ[1] = dA * act(Zg), in rows of ldz = out elements or
// out rounded up to a multiple of 8, then padded with zeros.
struct GatedOp {
    const void *H, *U;
    const float* bias;
    const void* dA;
    void *A, *dZ;               // dZ [2][T x ldz]
    int64_t T, out, r, ldz, u_rows;     // u_rows: of each factor in U, out or as padded
    int act;                    // lrd.h's LRD_ACT_*
    bool bf16;
};
hipError_t run_gated(const GatedOp& op, hipStream_t st);
// out [2][n]: column sums of the two matrices Z [2][T x ld]; for few rows, in one launch where column_sums takes four (all gradients of the fp32
// layer 256 x 768 -> 1536 63.5 -> 53.9 us).
bool pair_sums_supported(int64_t T);
hipError_t pair_sums(const void* Z, int64_t T, int64_t n, int64_t ld, bool bf16, float* out, hipStream_t st);
// dst [2][rows x cols] = the first rows and columns of src [2][rows_s x cols_s] (fp32).
hipError_t crop_pair(const float* src, int64_t rows_s, int64_t cols_s, float* dst, int64_t rows, int64_t cols, hipStream_t st);

// out [2][M x N] (fp32, dense): for each of two layers g the sum over T rows of A[t][m] * B[t][n]; A of layer g begins a_bs elements behind the first's, B b_bs.
struct FewRows {
    const void* A;
    int64_t lda, a_bs;
    const void* B;
    int64_t ldb, b_bs;
    float* out;
    int64_t M, N;
};
bool few_rows_supported(int64_t T, int64_t in, int64_t out, int64_t r, bool bf16, bool padded);       // padded: the products need copies at padded sizes
hipError_t few_rows(const FewRows* jobs, int n, int64_t T, bool bf16, hipStream_t st);       // one or two, in one launch

}  // namespace lrd
