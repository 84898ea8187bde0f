// The second products of a gated pair, Zg = Hg.Ug^T and Zu = Hu.Uu^T, and what joins them: A = act(Zg) * Zu, or, backward, dZg and dZu
// from dA.  Zg and Zu never leave the registers: over a rank they cost less to compute again than to store and load (2 r
// multiplications against 4 bytes written and read an element).
#include <algorithm>
#include <cstdio>
#include <string>

#include "gated.hpp"
#include "lrd.h"
#include "lrd_internal.hpp"
#include "lrd_measure.h"

namespace lrd {
namespace {

// act(z) and act'(z).  bf16: the polynomials of the library's other GELU epilogues, and the hardware's reciprocal.
template <int ACT, bool BF16>
__device__ __forceinline__ void act_terms(float z, float& a, float& da)
{
    if constexpr (ACT == LRD_ACT_NONE) {
        a = z;
        da = 1.f;
    } else if constexpr (ACT == LRD_ACT_GELU) {
        if constexpr (BF16) {
            a = gelu_bf16_f(z);
            da = gelu_grad_bf16_f(z);
        } else {
            float Phi, phi;
            gelu_terms(z, Phi, phi);
            a = z * Phi;
            da = fmaf(z, phi, Phi);
        }
    } else {
        const float e = __expf(-z);
        const float s = BF16 ? __builtin_amdgcn_rcpf(1.f + e) : 1.f / (1.f + e);
        a = z * s;
        da = fmaf(a, 1.f - s, s);
    }
}

template <class T>
struct GatedArgs {
    const T *H, *U;
    const float* bias;
    const T* dA;
    T *A, *dZ;
    int64_t rows, out, r, row_tiles, col_tiles;
};

// Any sizes and alignments: 64 x 64 results of both products a workgroup, operands through LDS in steps of 64 bytes of k.
// Four waves, 32 x 32 results each, in blocks of 16 x 16 whose operands are swapped: a lane holds four columns of a row.
template <class T, int ACT, bool BACK, bool ALIGNED>
__global__ __launch_bounds__(256) void gated_tile_kernel(GatedArgs<T> g)
{
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int VEC = 16 / sizeof(T), STEP = 4 * VEC, LD = STEP + VEC;      // a row of 64 bytes and 16 of padding
    typedef T TV __attribute__((ext_vector_type(VEC)));
    __shared__ __align__(16) T tile[4][64 * LD];                              // Hg, Hu, Ug, Uu
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4, r16 = lane & 15;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    for (int64_t at = blockIdx.x; at < g.row_tiles * g.col_tiles; at += gridDim.x) {
        const int64_t m0 = at / g.col_tiles * 64, n0 = at % g.col_tiles * 64;
        f32x4 acc[2][2][2];
#pragma unroll
        for (int p = 0; p < 8; ++p) acc[p >> 2][p >> 1 & 1][p & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int lr = tid >> 2, lc = tid & 3;                                // row and 16-byte chunk that this thread loads
        for (int64_t k0 = 0; k0 < g.r; k0 += STEP) {
            TV v[4];
            const int64_t k = k0 + lc * VEC;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const bool there = p < 2 ? m0 + lr < g.rows : n0 + lr < g.out;
                const T* row = p < 2 ? g.H + (m0 + lr) * 2 * g.r + p * g.r : g.U + ((p - 2) * g.out + n0 + lr) * g.r;
                if constexpr (ALIGNED) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[p][e] = (T)0.f;
                    if (there && k < g.r) v[p] = *reinterpret_cast<const TV*>(row + k);
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[p][e] = there && k + e < g.r ? row[k + e] : (T)0.f;
                }
            }
            __syncthreads();
#pragma unroll
            for (int p = 0; p < 4; ++p) *reinterpret_cast<TV*>(&tile[p][lr * LD + lc * VEC]) = v[p];
            __syncthreads();
            TV a[2][2], b[2][2];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    a[p][i] = *reinterpret_cast<const TV*>(&tile[p][(wm + i * 16 + r16) * LD + q * VEC]);
                    b[p][i] = *reinterpret_cast<const TV*>(&tile[2 + p][(wn + i * 16 + r16) * LD + q * VEC]);
                }
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if constexpr (BF16) {
                            acc[p][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[p][j], a[p][i], acc[p][i][j], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int c = 0; c < 4; ++c) acc[p][i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[p][j][c], a[p][i][c], acc[p][i][j], 0, 0, 0);
                        }
                    }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t m = m0 + wm + i * 16 + r16, n = n0 + wn + j * 16 + q * 4 + e;
                    if (m >= g.rows || n >= g.out) continue;
                    const float zg = acc[0][i][j][e] + (g.bias ? g.bias[n] : 0.f), zu = acc[1][i][j][e] + (g.bias ? g.bias[g.out + n] : 0.f);
                    float a, da;
                    act_terms<ACT, BF16>(zg, a, da);
                    const int64_t o = m * g.out + n;
                    if constexpr (BACK) {
                        const float d = to_f32(g.dA[o]);
                        g.dZ[o] = from_f32<T>(d * zu * da);
                        g.dZ[g.rows * g.out + o] = from_f32<T>(d * a);
                    } else {
                        g.A[o] = from_f32<T>(a * zu);
                    }
                }
    }
}

template <class T, int ACT, bool BACK>
hipError_t launch(const GatedOp& op, hipStream_t st)
{
    GatedArgs<T> g;
    g.H = (const T*)op.H; g.U = (const T*)op.U; g.bias = op.bias; g.dA = (const T*)op.dA; g.A = (T*)op.A; g.dZ = (T*)op.dZ;
    g.rows = op.T; g.out = op.out; g.r = op.r;
    g.row_tiles = ceil_div(op.T, 64); g.col_tiles = ceil_div(op.out, 64);
    const dim3 grid((unsigned)std::min<int64_t>(g.row_tiles * g.col_tiles, 1 << 20));
    note_kernel("gated_tile_kernel");
    if (op.r % (16 / sizeof(T)) == 0) hipLaunchKernelGGL((gated_tile_kernel<T, ACT, BACK, true>), grid, dim3(256), 0, st, g);
    else hipLaunchKernelGGL((gated_tile_kernel<T, ACT, BACK, false>), grid, dim3(256), 0, st, g);
    return hipGetLastError();
}

template <int ACT, bool BACK>
hipError_t by_type(const GatedOp& op, hipStream_t st)
{
    return op.bf16 ? launch<bf16_t, ACT, BACK>(op, st) : launch<float, ACT, BACK>(op, st);
}
template <bool BACK>
hipError_t by_act(const GatedOp& op, hipStream_t st)
{
    if (op.act == LRD_ACT_GELU) return by_type<LRD_ACT_GELU, BACK>(op, st);
    if (op.act == LRD_ACT_SILU) return by_type<LRD_ACT_SILU, BACK>(op, st);
    return by_type<LRD_ACT_NONE, BACK>(op, st);
}

}  // namespace

hipError_t run_gated(const GatedOp& op, hipStream_t st)
{
    hipEvent_t ev0 = nullptr, ev1 = nullptr;
    const int logged = log_begin(&ev0, &ev1);
    if (logged >= 0) (void)hipEventRecord(ev0, st);
    const hipError_t e = op.dA ? by_act<true>(op, st) : by_act<false>(op, st);
    if (logged >= 0) {
        (void)hipEventRecord(ev1, st);
        log_end(logged, op.dA ? LRD_ROLE_NONE : LRD_ROLE_FWD_UP, 0, 0, 1, op.T, op.out, op.r, 2);
    }
    return e;
}

}  // namespace lrd
