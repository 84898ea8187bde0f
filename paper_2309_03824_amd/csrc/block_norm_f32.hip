// fp32 rows of block_norm.inc, and the sums of both types' partial rows.
#include "lrd_device.hpp"
#define ELEM float
#include "block_norm.inc"

hipError_t block_norm_fwd_f32(const BlockNormFwd& g, hipStream_t st) { return dispatch(g, st); }
hipError_t block_norm_bwd_f32(const BlockNormBwd& g, hipStream_t st) { return dispatch(g, st); }

namespace {

// out[c] = sum over k of src[k][c], a fixed order: sixteen lanes of rows, then their sums in order.  (Four lanes took 11 us for 512 rows of 1024.)
struct SumRows { const float* src; float* out; int64_t ld, rows, group_stride, out_stride; };
struct SumRowsArgs { SumRows job[BN_SUMS + 1]; int64_t first_block[BN_SUMS + 2]; int64_t col_blocks; int d, jobs; };
__global__ __launch_bounds__(1024) void sum_rows_kernel(SumRowsArgs a)
{
    __shared__ float part[16][64];
    int j = 0;
    while (j + 1 < a.jobs && (int64_t)blockIdx.x >= a.first_block[j + 1]) ++j;
    const SumRows& s = a.job[j];
    const int64_t b = blockIdx.x - a.first_block[j], group = b / a.col_blocks;
    const int c = (int)(b - group * a.col_blocks) * 64 + (threadIdx.x & 63), l = threadIdx.x >> 6;
    float v = 0.f;
    if (c < a.d) {
        const float* at = s.src + group * s.group_stride + c;
#pragma unroll 8
        for (int64_t k = l; k < s.rows; k += 16) v += at[k * s.ld];
    }
    part[l][threadIdx.x & 63] = v;
    __syncthreads();
    if (l == 0 && c < a.d) {
#pragma unroll
        for (int k = 1; k < 16; ++k) v += part[k][threadIdx.x];
        s.out[group * s.out_stride + c] = v;
    }
}

}  // namespace

hipError_t block_norm_sums(const BlockNormBwd& g, float* const (&outs)[BN_SUMS], hipStream_t st)
{
    SumRowsArgs a;
    a.d = g.d; a.jobs = 0; a.col_blocks = ceil_div(g.d, 64);
    int64_t blocks = 0;
    auto add = [&](const SumRows& s, int64_t groups) {
        a.job[a.jobs] = s;
        a.first_block[a.jobs++] = blocks;
        blocks += groups * a.col_blocks;
    };
    for (int s = 0; s < BN_SUMS; ++s)
        if (g.sums[s]) add({g.partial + (int64_t)s * g.d, outs[s], (int64_t)BN_SUMS * g.d, g.workgroups, 0, 0}, 1);
    if (g.dgate && g.parts > 1) add({g.gate_partial, g.dgate, g.d, g.parts, g.parts * g.d, g.d}, g.units / g.parts);
    if (!a.jobs) return hipSuccess;
    hipLaunchKernelGGL(sum_rows_kernel, dim3((unsigned)blocks), dim3(1024), 0, st, a);
    return hipGetLastError();
}

}  // namespace lrd
