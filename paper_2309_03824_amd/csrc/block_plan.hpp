// How the rows of a block norm's backward pass are dealt to workgroups (see block_norm.inc).
#pragma once
#include <algorithm>
#include <cstdint>

namespace lrd {

enum { BN_W_PRE, BN_B_PRE, BN_W_POST, BN_B_POST, BN_SUMS, BN_GATE = BN_SUMS };     // partial rows of a workgroup, and the gate's of a unit
#define BN_BIT(SUM) (1 << lrd::BN_##SUM)

// Units of rows, none across two rows of the gate: `by_slot`, a group of gate_rows rows each, for one of a workgroup's slots;
// else `parts` of part_rows rows in each group (the last ones of the last group may be empty), for a workgroup.
struct BlockNormPlan {
    int64_t gate_rows, units, parts, part_rows, workgroups;
    bool by_slot;
};

// Workgroups of a forward pass, a row or a few each, in two dimensions: a launch counts the threads of one in 32 bits (2^26 rows of a wave each, 2^24
// of 256 threads).  The last row of the grid may be longer than what is left.
struct RowsGrid { uint32_t x, y; };
inline RowsGrid rows_grid(int64_t workgroups, int threads)
{
    const int64_t most = ((int64_t(1) << 32) - 1) / threads, y = (workgroups + most - 1) / most;
    return {(uint32_t)((workgroups + y - 1) / y), (uint32_t)y};
}

// Threads of a row: the fewest whose registers hold it, 16 columns each.  (8 for rows that are no whole groups of 16 bytes: 8192 x 4095 194 us against
// 169, 2048 x 8003 175 against 109.)
inline int block_norm_threads(int64_t d) { return d <= 1024 ? 64 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024; }
inline int64_t block_norm_slots(int threads) { return threads == 64 ? 8 : 1; }      // rows that a workgroup works on at once
// Workgroups that run at a time: eight waves a compute unit, or sixteen of those that have 128 registers.  (Twice as many for 8192 x 1024: as many
// partial rows more, and each workgroup too few rows to load ahead.)
inline int64_t block_norm_resident(int threads) { return threads == 256 ? 512 : 256; }

inline BlockNormPlan block_norm_plan(int64_t T, int64_t d, int64_t gate_rows)
{
    auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    const int threads = block_norm_threads(d);
    const int64_t slots = block_norm_slots(threads), most = block_norm_resident(threads);
    BlockNormPlan p;
    p.gate_rows = gate_rows > 0 && gate_rows < T ? gate_rows : T;
    const int64_t groups = up(T, p.gate_rows);
    p.by_slot = groups > 1 && p.gate_rows <= 16;
    if (p.by_slot) {
        p.units = groups; p.parts = 1; p.part_rows = p.gate_rows;
        p.workgroups = std::min(most, up(groups, slots));
        return p;
    }
    // parts of a group so that there is a unit for each workgroup, and no smaller than a round of its slots
    const int64_t wanted = up(std::min(most, up(T, slots)), groups);
    p.part_rows = std::max(slots, up(p.gate_rows, wanted));
    p.parts = up(p.gate_rows, p.part_rows);
    p.units = groups * p.parts;
    p.workgroups = std::min(most, p.units);
    return p;
}

// Most workgroups and gate units over every gate for T tokens or fewer: partial rows that a workspace has room for.
inline int64_t block_norm_most_workgroups(int64_t T) { return std::min<int64_t>(512, 2 * T); }
inline int64_t block_norm_most_units(int64_t T) { return std::min<int64_t>(1024, 2 * T); }

}  // namespace lrd
