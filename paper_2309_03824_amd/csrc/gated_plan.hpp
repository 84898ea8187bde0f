// Which kernel computes the second products of a gated pair (see gated.hip).
#pragma once
#include <cstdint>

namespace lrd {

enum GatedRoute { DIRECT_16, DIRECT_32, WIDE, DEEP, TILES };
constexpr int GATED_WIDE_ROWS = 128, GATED_WIDE_COLS = 64, GATED_WIDE_THREADS = 256;      // of a workgroup; columns at a time
constexpr int GATED_DEEP_TILE = 128, GATED_DEEP_THREADS = 512;

// By the number of workgroups that a kernel gives work (us a call by itself, T x out x r with SiLU, forward):
//   16 x 16 blocks up to 512 of them (64 x 1024 x 256 6.2, in 32 x 32 ones 6.8, wide 8.4; 64 x 4096 8.8, 7.1, 8.5; fp32 64 x 1024 6.7, 9.6, in tiles 24.0);
//   32 x 32 blocks up to 512 of them, or 1024 where the wide kernel does not take the call (512 x 1024 x 256 9.0, wide 9.8; 256 x 4096 12.8, 10.0;
//   256 x 2730 11.0, deep 13.4, in tiles 11.9; 506 x 2730 x 416 19.8, 17.8, 24.2; fp32 512 x 2048 25.2, in tiles 25.7, 1024 x 2048 45.0, 35.3);
//   then wide, else deep (8192 x 4096 x 256 43, deep 73, in tiles 80; x 1024 deep 226, in tiles 307), else tiles.
// padded: rows of dZ are longer than out.  most_ld: the longest rows that the wide kernel addresses.
inline GatedRoute gated_route(int64_t T, int64_t out, int64_t r, bool padded, bool bf16, int64_t most_ld)
{
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    auto tiles = [&](int64_t e) { return up(T, e) * up(out, e); };
    // a launch counts its threads in 32 bits (the tiles' workgroups walk, and need no more than there are)
    auto launches = [](int64_t workgroups, int threads) { return workgroups < (int64_t(1) << 32) / threads; };
    // (32-bit byte offsets within 32 rows of a result and 64 columns of a factor; within 128 rows of H or U)
    const bool wide = bf16 && r % 8 == 0 && r <= 512 && out % 8 == 0 && !padded && out <= most_ld &&
                      launches(up(T, GATED_WIDE_ROWS) * up(out, GATED_WIDE_COLS), GATED_WIDE_THREADS);
    const bool deep = bf16 && r % 8 == 0 && r <= (int64_t(1) << 21) && launches(tiles(GATED_DEEP_TILE), GATED_DEEP_THREADS);
    if (tiles(16) <= 512) return DIRECT_16;
    if (tiles(32) <= (wide ? 512 : 1024)) return DIRECT_32;
    return wide ? WIDE : deep ? DEEP : TILES;
}

}  // namespace lrd
