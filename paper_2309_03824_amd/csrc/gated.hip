// The second products of a gated pair, Zg = Hg.Ug^T and Zu = Hu.Uu^T, and what joins them: A = act(Zg) * Zu, or, backward, dZg and dZu
// from dA.  Zg and Zu never leave the registers: over a rank they cost less to compute again than to store and load (2 r
// multiplications against 4 bytes written and read an element).
#include <algorithm>

#include "gated.hpp"
#include "gated_plan.hpp"
#include "lds_load.hpp"
#include "lrd.h"
#include "lrd_internal.hpp"
#include "lrd_measure.h"
#include "wide_plan.hpp"

namespace lrd {
namespace {

// Phi(z) and phi(z) of the normal distribution, relative to their value also where they run into 0: with t = 1 / (1 + 0.3 |z|),
//     Phi(-|z|) = exp(-z^2 / 2) g(t),  g(t) = t (c1 + .. + c8 t^7) ~ erfcx(|z| / sqrt 2) / 2,
// the polynomial of least greatest relative error over |z| <= 14.5 (1.7e-7; evaluated in fp32 5e-7).  The other GELU epilogues' polynomial, 1.2e-4
// absolute, is 1.6 % off at z = -2.5 and has the wrong sign from -4 on, where Zu multiplies it; their erf form is 0.16 % off at -5.
// (Forward of 8192 x 4096 x 256 in bf16: the call 62 us, with that polynomial 54.)
__device__ __forceinline__ void normal_terms(float z, float& Phi, float& phi)
{
    const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * (z * z));
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.f));
    float g = fmaf(3.542372492e-02f, t, -1.561583627e-01f);
    g = fmaf(g, t, 2.045565620e-01f);
    g = fmaf(g, t, -5.203374174e-02f);
    g = fmaf(g, t, 1.276915914e-01f);
    g = fmaf(g, t, 1.001760114e-01f);
    g = fmaf(g, t, 1.207121250e-01f);
    g = fmaf(g, t, 1.196320080e-01f);
    const float tail = g * t * e;
    Phi = z >= 0.f ? 1.f - tail : tail;
    phi = 0.39894228040143268f * e;
}

// act(z), and backward act'(z): the same functions in both directions and types, so that a gradient is that of the value.
template <int ACT, bool BF16>
__device__ __forceinline__ void act_terms(float z, float& a, float& da)
{
    if constexpr (ACT == LRD_ACT_NONE) {
        a = z;
        da = 1.f;
    } else if constexpr (ACT == LRD_ACT_GELU) {
        float Phi, phi;
        normal_terms(z, Phi, phi);
        a = z * Phi;
        da = fmaf(z, phi, Phi);
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
    int64_t rows, out, r, ldz, u_rows, row_tiles, col_tiles;
};

// Four columns of a row from their two sums, as many as there are; backward also the zeros that a row of dZ is padded with.
template <class T, int ACT, bool BACK>
__device__ __forceinline__ void store_four(const GatedArgs<T>& g, int64_t m, int64_t n, f32x4 zg, f32x4 zu)
{
    typedef T T4 __attribute__((ext_vector_type(4)));
    constexpr bool BF16 = sizeof(T) == 2;
    const int64_t o = m * g.out + n, left = g.out - n;
    const bool quads = g.out % 4 == 0;
    if (g.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) { zg[e] += g.bias[n + e]; zu[e] += g.bias[g.out + n + e]; }
    }
    T4 d, x, y;
    if constexpr (BACK) {
        if (quads && left > 0) d = *reinterpret_cast<const T4*>(g.dA + o);
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) d[e] = e < left ? g.dA[o + e] : (T)0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, da;
        act_terms<ACT, BF16>(zg[e], a, da);
        if constexpr (BACK) {
            x[e] = e < left ? from_f32<T>(to_f32((T)d[e]) * zu[e] * da) : (T)0.f;
            y[e] = e < left ? from_f32<T>(to_f32((T)d[e]) * a) : (T)0.f;
        } else x[e] = y[e] = from_f32<T>(a * zu[e]);
    }
    const int64_t width = BACK ? g.ldz : g.out;
#pragma unroll
    for (int w = 0; w < (BACK ? 2 : 1); ++w) {
        T* to = BACK ? g.dZ + (w * g.rows + m) * g.ldz + n : g.A + o;
        const T4 v = w ? y : x;
        if (width % 4 == 0) *reinterpret_cast<T4*>(to) = v;
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < width) to[e] = v[e];
        }
    }
}

// Any sizes and alignments: 64 x 64 results of both products a workgroup, operands through LDS in steps of 64 bytes of k.
// Four waves, 32 x 32 results each, in blocks of 16 x 16 whose operands are swapped: a lane holds four columns of a row.
template <class T, int ACT, bool BACK>
__global__ __launch_bounds__(256) void gated_tile_kernel(GatedArgs<T> g)
{
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int VEC = 16 / sizeof(T), STEP = 4 * VEC, LD = STEP + VEC;      // a row of 64 bytes and 16 of padding
    typedef T TV __attribute__((ext_vector_type(VEC)));
    typedef TV TU __attribute__((aligned(sizeof(T))));                        // a vector at any element
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
                const T* row = p < 2 ? g.H + (m0 + lr) * 2 * g.r + p * g.r : g.U + ((p - 2) * g.u_rows + n0 + lr) * g.r;
                if (there && k + VEC <= g.r) {
                    v[p] = *reinterpret_cast<const TU*>(row + k);
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
            for (int j = 0; j < 2; ++j) {
                const int64_t m = m0 + wm + i * 16 + r16, n = n0 + wn + j * 16 + q * 4;
                if (m < g.rows && n < (BACK ? g.ldz : g.out)) store_four<T, ACT, BACK>(g, m, n, acc[0][i][j], acc[1][i][j]);
            }
    }
}

// Few results, and all of fp32: blocks of 16 TB x 16 TB of both products, r cut over the KS waves of a workgroup in steps of 64 bytes, fragments
// straight from memory (L2), up to DEPTH - 1 steps ahead; there is no barrier before the waves' sums meet.  Such calls are bound by latency and by
// how many compute units get work.  Any sizes: rows past the end repeat the last one (their results are not stored), and k past r is zero.
template <class T, int ACT, bool BACK, int TB, int KS>
__global__ __launch_bounds__(64 * KS) void gated_direct_kernel(GatedArgs<T> g)
{
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int VEC = 16 / sizeof(T), STEP = 4 * VEC, E = 16 * TB, LDT = E + 4, DEPTH = TB == 1 ? 4 : 2;
    typedef T TV __attribute__((ext_vector_type(VEC)));
    typedef TV TU __attribute__((aligned(sizeof(T))));          // a vector at any element
    __shared__ float sums[KS][2][E * LDT];
    const int tid = threadIdx.x, lane = tid & 63, ks = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, r16 = lane & 15;
    const int64_t m0 = blockIdx.x / (uint32_t)g.col_tiles * (int64_t)E, n0 = blockIdx.x % (uint32_t)g.col_tiles * (int64_t)E;
    const int r = (int)g.r, whole = r / STEP;
    const T *a[TB], *b[TB];
#pragma unroll
    for (int i = 0; i < TB; ++i) {
        a[i] = g.H + min(m0 + i * 16 + r16, g.rows - 1) * 2 * g.r + q * VEC;
        b[i] = g.U + min(n0 + i * 16 + r16, g.out - 1) * g.r + q * VEC;
    }
    const int64_t other = g.u_rows * g.r;
    f32x4 acc[2][TB][TB];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < TB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[p][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    TV av[DEPTH][2][TB], bv[DEPTH][2][TB];
    auto fetch = [&](int step, int at) {
        const int k = step * STEP;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                av[at][p][i] = *reinterpret_cast<const TU*>(a[i] + p * g.r + k);
                bv[at][p][i] = *reinterpret_cast<const TU*>(b[i] + p * other + k);
            }
    };
    auto multiply = [&](int at) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < TB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    if constexpr (BF16) {
                        acc[p][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bv[at][p][j], av[at][p][i], acc[p][i][j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[p][i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(bv[at][p][j][c], av[at][p][i][c], acc[p][i][j], 0, 0, 0);
                    }
                }
    };
    const int mine = whole > ks ? (whole - ks + KS - 1) / KS : 0;
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
        if (d < mine) fetch(ks + d * KS, d);
    for (int s = 0; s < mine; s += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (s + d + DEPTH - 1 < mine) fetch(ks + (s + d + DEPTH - 1) * KS, (d + DEPTH - 1) % DEPTH);
            if (s + d < mine) multiply(d);
        }
    }
    if (whole * STEP < r && whole % KS == ks) {
        const int k = whole * STEP;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < TB; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const bool there = k + q * VEC + e < r;
                    av[0][p][i][e] = there ? a[i][p * g.r + k + e] : (T)0.f;
                    bv[0][p][i][e] = there ? b[i][p * other + k + e] : (T)0.f;
                }
        multiply(0);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < TB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) *reinterpret_cast<f32x4*>(&sums[ks][p][(i * 16 + r16) * LDT + j * 16 + q * 4]) = acc[p][i][j];
    __syncthreads();
    for (int x = tid; x < E * E; x += 64 * KS) {
        const int ml = x / E, nl = x % E;
        const int64_t m = m0 + ml, n = n0 + nl;
        if (m >= g.rows || n >= (BACK ? g.ldz : g.out)) continue;
        float zg = sums[0][0][ml * LDT + nl], zu = sums[0][1][ml * LDT + nl];
#pragma unroll
        for (int z = 1; z < KS; ++z) { zg += sums[z][0][ml * LDT + nl]; zu += sums[z][1][ml * LDT + nl]; }
        const bool there = !BACK || n < g.out;
        if (g.bias && there) { zg += g.bias[n]; zu += g.bias[g.out + n]; }
        float av1, da;
        act_terms<ACT, BF16>(zg, av1, da);
        if constexpr (BACK) {
            const float d = there ? to_f32(g.dA[m * g.out + n]) : 0.f;
            g.dZ[m * g.ldz + n] = there ? from_f32<T>(d * zu * da) : (T)0.f;
            g.dZ[(g.rows + m) * g.ldz + n] = there ? from_f32<T>(d * av1) : (T)0.f;
        } else {
            g.A[m * g.out + n] = from_f32<T>(av1 * zu);
        }
    }
}

// Ranks past the registers of the kernel above, and results whose columns are no whole 16 bytes (bf16, r a multiple of 8): 128 x 128 results of both
// products a workgroup of eight waves (64 x 32 each), H and U in steps of 64 k through two LDS stages.
template <int ACT, bool BACK>
__global__ __launch_bounds__(512, 2) void gated_deep_kernel(GatedArgs<bf16_t> g)
{
    constexpr int MAT = 128 * 128, STAGE = 4 * MAT;           // bytes of 64 k of 128 rows; Hg, Hu, Ug, Uu
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = (int)uni(threadIdx.x >> 6), q = lane >> 4, r16 = lane & 15;
    // each die takes a run of row tiles, whose column tiles follow one another
    const uint32_t total = gridDim.x, f = blockIdx.x, die = f & 7u, per = total >> 3, more = total & 7u;
    const uint32_t t = die * per + min(die, more) + (f >> 3);
    const int64_t m0 = t / (uint32_t)g.col_tiles * (int64_t)128, n0 = t % (uint32_t)g.col_tiles * (int64_t)128;
    const int rows = (int)min(g.rows - m0, (int64_t)128), cols = (int)min(g.out - n0, (int64_t)128);

    // a wave loads 64 rows of one of the four
    const int mat = wave >> 1;
    const uint32_t r = uni((uint32_t)g.r), ld = mat < 2 ? 2 * r : r;
    const int there = mat < 2 ? rows : cols;
    const char* base = uni_ptr(mat < 2 ? g.H + m0 * 2 * g.r + mat * g.r : g.U + ((mat - 2) * g.u_rows + n0) * g.r);
    uint32_t span = ((uint32_t)(there - 1) * ld + r) * 2u;
    settle(base, span);
    uint32_t voff[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int row = (wave & 1) * 64 + p * 8 + (lane >> 3);
        voff[p] = row < there ? ((uint32_t)row * ld + ((lane & 7) ^ kc_swz(row)) * 8) * 2u : BUF_OOB;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const int steps = (g.r + 63) / 64;
    auto load = [&](int step) {
        const uint32_t to = lds0 + (step & 1) * STAGE + wave * 8192, k0 = step * 64;
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int row = (wave & 1) * 64 + p * 8 + (lane >> 3);
            const uint32_t k = k0 + ((lane & 7) ^ kc_swz(row)) * 8;
            load_to_lds(to + p * 1024, base + k0 * 2, span - k0 * 2, k < r ? voff[p] : BUF_OOB);
        }
    };
    load(0);
    const int wm = (wave >> 2) * 64, wn = (wave & 3) * 32;
    f32x4 acc[2][4][2];
#pragma unroll
    for (int p = 0; p < 16; ++p) acc[p >> 3][(p >> 1) & 3][p & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int step = 0; step < steps; ++step) {
        wait_vm<0>();
        lds_barrier();
        if (step + 1 < steps) load(step + 1);
        const char* at = reinterpret_cast<const char*>(smem) + (step & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                bf16x8 a[4], b[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = wm + i * 16 + r16;
                    a[i] = *reinterpret_cast<const bf16x8*>(at + p * MAT + row * 128 + (((kk * 4 + q) ^ kc_swz(row)) << 4));
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = wn + j * 16 + r16;
                    b[j] = *reinterpret_cast<const bf16x8*>(at + (2 + p) * MAT + row * 128 + (((kk * 4 + q) ^ kc_swz(row)) << 4));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[p][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[p][i][j], 0, 0, 0);
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t m = m0 + wm + i * 16 + r16, n = n0 + wn + j * 16 + q * 4;
            if (m < g.rows && n < (BACK ? g.ldz : g.out)) store_four<bf16_t, ACT, BACK>(g, m, n, acc[0][i][j], acc[1][i][j]);
        }
}

template <int ACT, bool BACK>
hipError_t launch_deep(const GatedOp& op, hipStream_t st)
{
    constexpr int lds_bytes = 2 * 4 * 128 * 128;
    auto kern = gated_deep_kernel<ACT, BACK>;
    static OncePerDevice lds_allowed;
    const hipError_t e = allow_lds(kern, lds_bytes, lds_allowed);
    if (e != hipSuccess) return e;
    note_kernel("gated_deep_kernel");
    GatedArgs<bf16_t> g;
    g.H = (const bf16_t*)op.H; g.U = (const bf16_t*)op.U; g.bias = op.bias; g.dA = (const bf16_t*)op.dA; g.A = (bf16_t*)op.A; g.dZ = (bf16_t*)op.dZ;
    g.rows = op.T; g.out = op.out; g.r = op.r; g.ldz = op.ldz; g.u_rows = op.u_rows;
    g.row_tiles = ceil_div(op.T, 128); g.col_tiles = ceil_div(op.out, 128);
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.row_tiles * g.col_tiles)), dim3(512), lds_bytes, st, g);
    return hipGetLastError();
}

template <class T, int ACT, bool BACK>
hipError_t launch(const GatedOp& op, GatedRoute how, hipStream_t st)
{
    GatedArgs<T> g;
    g.H = (const T*)op.H; g.U = (const T*)op.U; g.bias = op.bias; g.dA = (const T*)op.dA; g.A = (T*)op.A; g.dZ = (T*)op.dZ;
    g.rows = op.T; g.out = op.out; g.r = op.r; g.ldz = op.ldz; g.u_rows = op.u_rows;
    if (how == DIRECT_16) {
        g.row_tiles = ceil_div(op.T, 16); g.col_tiles = ceil_div(op.out, 16);
        note_kernel("gated_direct_kernel<16>");
        hipLaunchKernelGGL((gated_direct_kernel<T, ACT, BACK, 1, 8>), dim3((unsigned)(g.row_tiles * g.col_tiles)), dim3(512), 0, st, g);
        return hipGetLastError();
    }
    if (how == DIRECT_32) {
        g.row_tiles = ceil_div(op.T, 32); g.col_tiles = ceil_div(op.out, 32);
        note_kernel("gated_direct_kernel<32>");
        hipLaunchKernelGGL((gated_direct_kernel<T, ACT, BACK, 2, 4>), dim3((unsigned)(g.row_tiles * g.col_tiles)), dim3(256), 0, st, g);
        return hipGetLastError();
    }
    g.row_tiles = ceil_div(op.T, 64); g.col_tiles = ceil_div(op.out, 64);
    const dim3 grid((unsigned)std::min<int64_t>(g.row_tiles * g.col_tiles, 1 << 20));
    note_kernel("gated_tile_kernel");
    hipLaunchKernelGGL((gated_tile_kernel<T, ACT, BACK>), grid, dim3(256), 0, st, g);
    return hipGetLastError();
}

// Long batches (bf16, r a multiple of 8 up to 512): a wave keeps 32 rows of Hg and of Hu in registers, all of r, and its workgroup of
// four walks along the columns in chunks of 64, Ug's and Uu's in turn through two LDS buffers (one is multiplied while the other
// loads).  Results leave as whole 128-byte lines by way of 4 KB of LDS of each wave's own, where dA of the chunk has been loaded
// in the backward: a lane takes its dA from there, puts dZg in its place and dZu there after dZg has left.
constexpr int COLS = 64;             // columns of a chunk
constexpr int ROWS = 32;             // rows of a wave
constexpr int SUB = COLS * 64 * 2;   // LDS bytes of 64 k of a chunk of one factor
constexpr int WAVES = 4;
static_assert(ROWS * WAVES == GATED_WIDE_ROWS && COLS == GATED_WIDE_COLS && 64 * WAVES == GATED_WIDE_THREADS, "as planned");
constexpr int AUX_NT = 2;            // non-temporal: results are too many for the caches

struct GatedWideArgs {
    const bf16_t *H, *U, *dA;
    bf16_t* out[2];                  // A; or dZg, dZu
    const float* bias;
    int64_t rows;
    int n, r;                        // columns (of each factor), rank
    int inner, chunks;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const void* base, uint32_t span)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)span, (int)BUF_FLAGS);
}

// Element E of the lane's quad.
template <int E>
__device__ __forceinline__ float quad(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), E * 0x55, 0xf, 0xf, true));
}

// KS = ceil(r / 64).
template <int KS, int ACT, bool BACK, bool BIAS>
__global__ __launch_bounds__(64 * WAVES, KS <= 4 ? 2 : 1) void gated_wide_kernel(GatedWideArgs g)
{
    constexpr int CHUNK = KS * SUB, PER = 8 / WAVES;      // bytes of a factor's chunk, loads per wave of 64 k of it
    constexpr int STORES = BACK ? 8 : 4;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = (int)uni(threadIdx.x >> 6);
    // each die takes a run of row blocks, whose ranges of columns follow one another
    const uint32_t total = gridDim.x, f = blockIdx.x, die = f & 7u, per = total >> 3, more = total & 7u;
    const uint32_t t = die * per + min(die, more) + (f >> 3);
    const int range = (int)(t % (uint32_t)g.inner);
    const int64_t row0 = (int64_t)(t / (uint32_t)g.inner) * (ROWS * WAVES) + wave * ROWS;
    const int rows = (int)max((int64_t)0, min(g.rows - row0, (int64_t)ROWS));
    const int first = range * g.chunks, n_chunks = min(g.chunks, (g.n + COLS - 1) / COLS - first);

    const uint32_t r = uni((uint32_t)g.r);
    const char* u0 = uni_ptr(g.U + (int64_t)first * COLS * g.r);
    int64_t other = uni64((int64_t)g.n * g.r * 2);       // from Ug to Uu
    int left0 = (int)uni((uint32_t)(g.n - first * COLS));
    settle(u0, other, left0);
    uint32_t voff[PER], vtail[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int row = (p * WAVES + wave) * 8 + (lane >> 3), k = ((lane & 7) ^ kc_swz(row)) * 8;
        voff[p] = ((uint32_t)row * r + k) * 2u;
        vtail[p] = (KS - 1) * 64 + k < g.r ? voff[p] : BUF_OOB;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
    // 64 columns of a factor to its buffer; columns past the last are past the descriptor
    auto load_chunk = [&](int c, int which) {
        const char* at = u0 + (int64_t)c * (COLS * 2) * r + (which ? other : 0);
        const uint32_t span = ((uint32_t)(min(left0 - c * COLS, COLS) - 1) * r + r) * 2u;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int p = 0; p < PER; ++p)
                load_to_lds(lds0 + which * CHUNK + s * SUB + (p * WAVES + wave) * 1024, at + s * 128, span - s * 128u, s == KS - 1 ? vtail[p] : voff[p]);
    };
    // H in the layout of the MFMA operand: lane l holds row (l & 15), k = 8 * (l >> 4) + 0..7 of each group of 32
    const int q = lane >> 4, r16 = lane & 15;
    bf16x8 h[2][2][KS * 2];
    {
        const int64_t ldh = 2 * (int64_t)g.r;
        const char* base = uni_ptr(g.H + row0 * ldh);
        const __amdgpu_buffer_rsrc_t rh = descriptor(base, uni(rows > 0 ? (uint32_t)(rows * ldh * 2) : 0u));
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int kk = 0; kk < KS * 2; ++kk) {
                    const int k = kk * 32 + q * 8, row = i * 16 + r16;
                    const uint32_t off = k < g.r && row < rows ? ((uint32_t)row * 2u * r + w * r + k) * 2u : BUF_OOB;
                    h[w][i][kk] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rh, off, 0, 0));
                }
    }

    const __amdgpu_buffer_rsrc_t rb = descriptor(uni_ptr(g.bias), BIAS ? uni((uint32_t)g.n * 8u) : 0u);
    // The sums begin with the biases: lane l holds that of column 16 j + 4 (l >> 4) + (l & 3) for each j, from where its quad has the
    // four that it needs.  Loaded half a chunk early, ahead of the loads that the chunk waits for.  (Loaded where they are added, behind
    // load_chunk, the compiler's wait for them took in that chunk: 52 us instead of 43 for 8192 x 4096 x 256; fetched from other
    // lanes through LDS 52; as the accumulators' registers, where they come late, 48.)
    float bias[2][4];
    auto load_bias = [&](int c, int w) {
        if constexpr (BIAS) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t col = (uint32_t)((first + c) * COLS + j * 16 + q * 4 + (r16 & 3));
                bias[w][j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rb, col < (uint32_t)g.n ? (col + w * (uint32_t)g.n) * 4u : BUF_OOB, 0, 0));
            }
            asm volatile("" ::: "memory");
        }
    };
    load_bias(0, 0);
    load_chunk(0, 0);

    const uint32_t f0 = r16 * 128 + ((q ^ kc_swz(r16)) << 4);
    f32x4 acc[2][2][4];
    auto start = [&](int w) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x4 from{0.f, 0.f, 0.f, 0.f};
            if constexpr (BIAS) {
                asm volatile("" : "+v"(bias[w][j]));           // (there by the wait before)
                from = f32x4{quad<0>(bias[w][j]), quad<1>(bias[w][j]), quad<2>(bias[w][j]), quad<3>(bias[w][j])};
            }
            acc[w][0][j] = acc[w][1][j] = from;
        }
    };
    auto multiply = [&](int w) {
        const char* at = reinterpret_cast<const char*>(smem) + w * CHUNK;
#pragma unroll
        for (int kk = 0; kk < KS * 2; ++kk) {
            bf16x8 b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const bf16x8*>(at + (kk >> 1) * SUB + j * 2048 + ((kk & 1) ? f0 ^ 64 : f0));
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[w][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], h[w][i][kk], acc[w][i][j], 0, 0, 0);
        }
    };

    // this wave's 32 rows of 128 bytes, chunks of a row permuted
    char* const stage = reinterpret_cast<char*>(smem) + 2 * CHUNK + wave * (ROWS * 128);
    const uint32_t stage_lds = lds0 + 2 * CHUNK + wave * (ROWS * 128);
    const int wr = r16 * 128 + (q & 1) * 8, srow = lane >> 3, scol = lane & 7;
    const int64_t at0 = row0 * g.n;
    uint32_t row_span = uni(rows > 0 ? (uint32_t)(((int64_t)rows * g.n) * 2) : 0u);
    const char* d0 = BACK ? uni_ptr(g.dA + at0) : nullptr;
    if constexpr (BACK) settle(d0, row_span);
    const __amdgpu_buffer_rsrc_t rc0 = descriptor(uni_ptr(g.out[0] + at0), row_span), rc1 = BACK ? descriptor(uni_ptr(g.out[1] + at0), row_span) : rc0;
    // (rows and columns that do not exist are past the descriptors: every wave issues the operations that the waits count)
    auto place = [&](int row, int col) { return row < rows && col < g.n ? ((uint32_t)row * (uint32_t)g.n + col) * 2u : BUF_OOB; };

    for (int c = 0; c < n_chunks; ++c) {
        const int col0 = (first + c) * COLS;
        if (c == 0) wait_vm<0>();
        else wait_vm<STORES>();           // (Ug's loads are older than the last chunk's stores)
        lds_barrier();
        if constexpr (BACK) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = e * 8 + srow;
                load_to_lds(stage_lds + e * 1024, d0, row_span, place(row, col0 + (scol ^ kc_swz(row)) * 8));
            }
        }
        start(0);
        load_bias(c, 1);
        load_chunk(c, 1);
        __builtin_amdgcn_s_setprio(1);       // (multiplying before another workgroup's epilogue: 2 % of 43 us)
        multiply(0);
        wait_vm<0>();
        lds_barrier();
        start(1);
        if (c + 1 < n_chunks) load_chunk(c + 1, 0);
        multiply(1);
        __builtin_amdgcn_s_setprio(0);
        load_bias(c + 1, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            u32x2 held[4];
            char* const at = stage + i * 2048;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 zg = acc[0][i][j], zu = acc[1][i][j];
                char* const mine = at + wr + (((j * 2 + (q >> 1)) ^ kc_swz(r16)) << 4);
                f32x4 x, y;
                if constexpr (BACK) {
                    const bf16x4 d = *reinterpret_cast<const bf16x4*>(mine);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float a, da;
                        act_terms<ACT, true>(zg[e], a, da);
                        x[e] = (float)d[e] * zu[e] * da;
                        y[e] = (float)d[e] * a;
                    }
                    held[j] = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float a, da;
                        act_terms<ACT, true>(zg[e], a, da);
                        x[e] = a * zu[e];
                    }
                }
                *reinterpret_cast<u32x2*>(mine) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
            }
            asm volatile("" ::: "memory");      // (a wave's LDS operations complete in order: its reads see its writes)
#pragma unroll
            for (int w = 0; w < (BACK ? 2 : 1); ++w) {
                if (w) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x2*>(at + wr + (((j * 2 + (q >> 1)) ^ kc_swz(r16)) << 4)) = held[j];
                    asm volatile("" ::: "memory");
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int sr = e * 8 + srow;
                    const u32x4 v = *reinterpret_cast<const u32x4*>(at + sr * 128 + ((scol ^ kc_swz(sr)) << 4));
                    __builtin_amdgcn_raw_buffer_store_b128(v, w ? rc1 : rc0, place(i * 16 + sr, col0 + scol * 8), 0, AUX_NT);
                }
                asm volatile("" ::: "memory");
            }
        }
    }
}

template <int KS, int ACT, bool BACK, bool BIAS>
hipError_t launch_wide(const GatedOp& op, hipStream_t st)
{
    constexpr int PER_CU = KS <= 4 ? 2 : 1;
    constexpr int lds_bytes = 2 * KS * SUB + WAVES * ROWS * 128;
    static_assert(PER_CU * lds_bytes <= 160 * 1024, "LDS of a compute unit");
    auto kern = gated_wide_kernel<KS, ACT, BACK, BIAS>;
    static OncePerDevice lds_allowed;
    const hipError_t e = allow_lds(kern, lds_bytes, lds_allowed);
    if (e != hipSuccess) return e;
    note_kernel(BACK ? "gated_wide_kernel,grad" : "gated_wide_kernel");
    GatedWideArgs g;
    g.H = (const bf16_t*)op.H; g.U = (const bf16_t*)op.U; g.dA = (const bf16_t*)op.dA; g.bias = op.bias;
    g.out[0] = (bf16_t*)(BACK ? op.dZ : op.A);
    g.out[1] = BACK ? (bf16_t*)op.dZ + op.T * op.out : nullptr;
    g.rows = op.T; g.n = (int)op.out; g.r = (int)op.r;
    const int64_t row_blocks = ceil_div(op.T, ROWS * WAVES);
    const int all = (int)ceil_div(op.out, COLS);
    g.chunks = wide_chunks(row_blocks, all, 256 * PER_CU);
    g.inner = (int)ceil_div(all, g.chunks);
    hipLaunchKernelGGL(kern, dim3((unsigned)(row_blocks * g.inner)), dim3(64 * WAVES), lds_bytes, st, g);
    return hipGetLastError();
}

template <int ACT, bool BACK, bool BIAS>
hipError_t wide_by_depth(const GatedOp& op, hipStream_t st)
{
    switch (ceil_div(op.r, 64)) {
    case 1: return launch_wide<1, ACT, BACK, BIAS>(op, st);
    case 2: return launch_wide<2, ACT, BACK, BIAS>(op, st);
    case 3: return launch_wide<3, ACT, BACK, BIAS>(op, st);
    case 4: return launch_wide<4, ACT, BACK, BIAS>(op, st);
    case 5: return launch_wide<5, ACT, BACK, BIAS>(op, st);
    case 6: return launch_wide<6, ACT, BACK, BIAS>(op, st);
    case 7: return launch_wide<7, ACT, BACK, BIAS>(op, st);
    default: return launch_wide<8, ACT, BACK, BIAS>(op, st);
    }
}

template <int ACT, bool BACK>
hipError_t by_type(const GatedOp& op, hipStream_t st)
{
    const GatedRoute how = gated_route(op.T, op.out, op.r, op.ldz != op.out, op.bf16, BUF_MAX_LD);
    if (how == WIDE) return op.bias ? wide_by_depth<ACT, BACK, true>(op, st) : wide_by_depth<ACT, BACK, false>(op, st);
    if (how == DEEP) return launch_deep<ACT, BACK>(op, st);
    return op.bf16 ? launch<bf16_t, ACT, BACK>(op, how, st) : launch<float, ACT, BACK>(op, how, st);
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

namespace {
__global__ __launch_bounds__(256) void crop_pair_kernel(const float* __restrict__ src, int64_t rows_s, int64_t cols_s, float* __restrict__ dst, int64_t rows, int64_t cols)
{
    const int64_t each = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < 2 * each; i += (int64_t)gridDim.x * 256) {
        const int64_t k = i < each ? i : i - each, row = (uint32_t)k / (uint32_t)cols;
        dst[i] = src[((i < each ? 0 : rows_s) + row) * cols_s + (k - row * cols)];
    }
}
}  // namespace

namespace {
// out[g][c] = sum over t of Z[g][t][c] for two matrices, rows in sixteen lanes, then their sums in order.
template <class T>
__global__ __launch_bounds__(1024) void pair_sums_kernel(const T* __restrict__ Z, int64_t rows, int64_t n, int64_t ld, float* __restrict__ out)
{
    __shared__ float part[16][64];
    const int l = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const T* from = Z + blockIdx.y * rows * ld + c;
    float s = 0.f;
    if (c < n) {
#pragma unroll 8
        for (int64_t t = l; t < rows; t += 16) s += to_f32(from[t * ld]);
    }
    part[l][threadIdx.x & 63] = s;
    __syncthreads();
    if (l == 0 && c < n) {
#pragma unroll
        for (int k = 1; k < 16; ++k) s += part[k][threadIdx.x];
        out[blockIdx.y * n + c] = s;
    }
}
}  // namespace

bool pair_sums_supported(int64_t T) { return T <= 1024; }

hipError_t pair_sums(const void* Z, int64_t T, int64_t n, int64_t ld, bool bf16, float* out, hipStream_t st)
{
    const dim3 grid((unsigned)ceil_div(n, 64), 2);
    if (bf16) hipLaunchKernelGGL(pair_sums_kernel<bf16_t>, grid, dim3(1024), 0, st, (const bf16_t*)Z, T, n, ld, out);
    else hipLaunchKernelGGL(pair_sums_kernel<float>, grid, dim3(1024), 0, st, (const float*)Z, T, n, ld, out);
    return hipGetLastError();
}

hipError_t crop_pair(const float* src, int64_t rows_s, int64_t cols_s, float* dst, int64_t rows, int64_t cols, hipStream_t st)
{
    if (rows * cols >= (int64_t(1) << 32)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(2 * rows * cols, 256), 4096));
    hipLaunchKernelGGL(crop_pair_kernel, grid, dim3(256), 0, st, src, rows_s, cols_s, dst, rows, cols);
    return hipGetLastError();
}

namespace {
// Weight gradients over few tokens are bound by their store: 64 x 64 of a result in a workgroup, 4 x 4 a thread, the operands' rows through LDS
// sixteen at a time in 32 bits; tokens are added in order.  Any sizes and alignments, so that neither operands nor results need padded copies.
struct FewRowsArgs { FewRows job[2]; uint32_t cols[2], each[2], first; int64_t T; };      // blocks along N, of a layer, of the first job
template <class T>
__global__ __launch_bounds__(256) void few_rows_kernel(FewRowsArgs g)
{
    constexpr int STEP = 16;
    __shared__ __align__(16) float a[STEP][64], b[STEP][64];
    const int k = blockIdx.x >= g.first;
    const FewRows& j = g.job[k];
    const uint32_t at = blockIdx.x - (k ? g.first : 0u), layer = at >= g.each[k], tile = at - layer * g.each[k];
    const int64_t m0 = tile / g.cols[k] * (int64_t)64, n0 = tile % g.cols[k] * (int64_t)64;
    const T* const A = (const T*)j.A + layer * j.a_bs;
    const T* const B = (const T*)j.B + layer * j.b_bs;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, col = threadIdx.x & 63, row = threadIdx.x >> 6;
    const bool am = m0 + col < j.M, bn = n0 + col < j.N;
    f32x4 acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int64_t t0 = 0; t0 < g.T; t0 += STEP) {
        float x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + i * 4 + row;
            x[i] = t < g.T && am ? to_f32(A[t * j.lda + m0 + col]) : 0.f;
            y[i] = t < g.T && bn ? to_f32(B[t * j.ldb + n0 + col]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i * 4 + row][col] = x[i]; b[i * 4 + row][col] = y[i]; }
        __syncthreads();
        const int there = (int)min(g.T - t0, (int64_t)STEP);
        for (int t = 0; t < there; ++t) {
            const f32x4 u = *reinterpret_cast<const f32x4*>(&a[t][ty * 4]), v = *reinterpret_cast<const f32x4*>(&b[t][tx * 4]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(u[i], v[e], acc[i][e]);
        }
    }
    const int64_t n = n0 + tx * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + ty * 4 + i;
        if (m >= j.M || n >= j.N) continue;
        float* const to = j.out + (layer * j.M + m) * j.N + n;
        if (j.N % 4 == 0) *reinterpret_cast<f32x4*>(to) = acc[i];
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < j.N) to[e] = acc[i][e];
        }
    }
}
int64_t few_rows_blocks(int64_t M, int64_t N) { return ceil_div(M, 64) * ceil_div(N, 64); }
}  // namespace

// As many tokens as this is the faster way for at every size measured (us, all gradients, in = 1024, this way and by the engines): bf16 16 tokens
// -> 4096 at rank 384 32.4 and 33.6 (one token 29.0 and 40.7), 32 37.2 and 35.1; with padded copies for those 32 tokens -> 2730 at rank 193 36.3 and
// 41.2, 64 47.8 and 46.9; fp32 64 tokens -> 4096 at rank 384 66.4 and 70.6, at rank 193 62.1 and 61.3.
bool few_rows_supported(int64_t T, int64_t in, int64_t out, int64_t r, bool bf16, bool padded)
{
    return T <= (!bf16 ? 64 : padded ? 32 : 16) && few_rows_blocks(out, r) + few_rows_blocks(r, in) < (int64_t(1) << 23);      // (threads of both layers: 32 bits)
}

hipError_t few_rows(const FewRows* jobs, int n, int64_t T, bool bf16, hipStream_t st)
{
    FewRowsArgs g{};
    g.T = T;
    int64_t blocks = 0;
    for (int k = 0; k < n; ++k) {
        g.job[k] = jobs[k];
        g.cols[k] = (uint32_t)ceil_div(jobs[k].N, 64);
        g.each[k] = (uint32_t)few_rows_blocks(jobs[k].M, jobs[k].N);
        blocks += 2 * (int64_t)g.each[k];
        if (k == 0) g.first = (uint32_t)blocks;
    }
    if (bf16) hipLaunchKernelGGL(few_rows_kernel<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, st, g);
    else hipLaunchKernelGGL(few_rows_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, st, g);
    return hipGetLastError();
}

}  // namespace lrd
