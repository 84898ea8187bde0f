// Dropout: Y = X / (1 - p) where the generator keeps an element, else 0.  The mask is nowhere stored; the gradient is the same
// call on dY.
//
// Bound by the traffic of X and Y; a thread takes the eight elements that one generator call serves.
#include <algorithm>

#include "lrd_internal.hpp"

namespace lrd {
namespace {

template <class T, bool DROP>
__global__ __launch_bounds__(256) void dropout_kernel(const T* X, T* Y, int64_t n, DropRng rng)      // Y may be X
{
    typedef T Eight __attribute__((ext_vector_type(8)));
    typedef Eight T8 __attribute__((aligned(16)));          // (what the call asks of X and Y; eight of fp32 would be taken to begin on 32 bytes)
    const int64_t groups = n / 8, stride = (int64_t)gridDim.x * 256;
    DropKey key;
    if constexpr (DROP) key = DropKey(rng.state);
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += stride) {
        T8 v = *reinterpret_cast<const T8*>(X + g * 8);
        if constexpr (DROP) {
            const Words4 w = key.eight((uint64_t)g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = drop_bits(w, e) >= rng.below ? (T)((float)v[e] * rng.scale) : (T)0.f;
        }
        *reinterpret_cast<T8*>(Y + g * 8) = v;
    }
    if (blockIdx.x == 0 && threadIdx.x < n - groups * 8) {
        const int64_t i = groups * 8 + threadIdx.x;
        if constexpr (DROP) {
            const Words4 w = key.eight((uint64_t)groups);
            Y[i] = drop_bits(w, threadIdx.x) >= rng.below ? (T)((float)X[i] * rng.scale) : (T)0.f;
        } else Y[i] = X[i];
    }
}

template <class T>
hipError_t launch(const void* X, void* Y, int64_t n, const DropRng& rng, hipStream_t st)
{
    const dim3 grid((unsigned)std::min<int64_t>(std::max<int64_t>(1, ceil_div(n / 8, 256)), 1 << 16));
    if (rng.below) hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, st, (const T*)X, (T*)Y, n, rng);
    else hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, st, (const T*)X, (T*)Y, n, rng);
    return hipGetLastError();
}

}  // namespace

hipError_t dropout(const void* X, void* Y, int64_t n, bool bf16, const DropRng& rng, hipStream_t st)
{
    if (n <= 0) return hipSuccess;
    return bf16 ? launch<bf16_t>(X, Y, n, rng, st) : launch<float>(X, Y, n, rng, st);
}

}  // namespace lrd
