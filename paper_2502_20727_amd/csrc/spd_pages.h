// Paged KV cache: the handle, the plan of a step as host and kernels read it, and the layout of a page.
#pragma once

#include "spd_internal.h"
#include "spd_q8.h"

struct spd_pages {
    spd_pages_config cfg;
    int group;              // query heads per KV head
    int row_bytes;          // of a position's keys or values: codes and scales
    int shift;              // log2 of the 16-position blocks per page
    size_t head_bytes;      // of one head's share of a page
    size_t page_bytes;
};

// ------------------------------------------------------------------------------------------
// A page and head: 16-position blocks of keys, the same of values, key scales, value scales.  A block is a sequence of
// 1 KiB chunks, 16 bytes for each lane of a wavefront, lane = 16 g + r.
// Keys: lane (g, r) holds position r, features 4 E c + E g .. + E - 1 of chunk c (E = elements in 16 bytes).  As the contraction of
// the scores runs over features in any order that queries share, a lane's 16 bytes are whole operands of the matrix cores.
// Values: lane (g, r) holds positions 4 g .. 4 g + 3 of features r + 16 t, t = (E / 4) c .. (E / 4) (c + 1) - 1: what the second
// contraction takes beside probabilities as they leave the score tiles (four consecutive keys per lane).
// 4-bit codes: a block is D / 8 bytes for each lane.  Keys: lane (g, r) holds features D / 4 g .. D / 4 (g + 1) - 1 of position r, two to a byte.  Values: byte
// 4 u + j of lane (g, r) holds features r + 32 u (low half) and r + 32 u + 16 of position 4 g + j: two that share a scale, as the instruction that
// widens them takes one.  The scales are a byte for each position and group of 32 features, group after group, the keys' and then the values'.
// ------------------------------------------------------------------------------------------
SPD_HD int spd_page_value_off(int r, int f, int E) {
    const int t = f / 16;
    return (((t / (E / 4)) * 4 + r / 4) * 16 + f % 16) * E + (t % (E / 4)) * 4 + r % 4;
}

// ------------------------------------------------------------------------------------------
// The plan.  Attention sees the visible positions of a piece of work as a list of 16-position blocks: the first `sink_blocks`
// of the sequence, then those from block0 on.
// ------------------------------------------------------------------------------------------
constexpr uint32_t SPD_PLAN_MAGIC = 0x53504731u;
constexpr int SPD_COUNTERS = 16384;      // 32-bit, at the start of the workspace: items done of rows x head, zero between calls
constexpr int SPD_SMALL_WAVES = 8;       // of a workgroup of the kernel for few rows
constexpr int SPD_SMALL_ROWS = 16;       // rows (token x query head of the KV group) of an item of the kernel for few of them
constexpr int SPD_LARGE_ROWS = 128;      // ... and of the kernel for many

struct spd_plan_seq {
    int32_t pos, q_len, tok0, table;     // first new position, new tokens, row of the first, first entry in the plan's page table
    int64_t held0;                       // row of position 0 in spd_pages_read()'s output
    int32_t end, pad;                    // pos + q_len
};
// (Work carries a copy of its sequence: a kernel is a load from its first address, not two.)
struct spd_plan_item {                   // rows x blocks of one sequence, for every KV head
    spd_plan_seq s;
    int32_t row0;                        // first row
    int32_t sink_blocks, block0;
    int32_t first, count;                // blocks of the list
    int32_t slot;                        // where its partial result goes, or -1: it is the whole result
    int32_t slot0, parts;                // the rows' partial results: slots slot0 .. slot0 + parts - 1
    int32_t group;                       // number of the rows among those cut into items
    int32_t pad[3];
};
struct spd_plan_merge {                  // rows whose partial results lie in slots slot0 .. slot0 + parts - 1
    spd_plan_seq s;
    int32_t row0, rows, slot0, parts;
};
struct spd_plan_block {                  // a 16-position block that receives new tokens
    spd_plan_seq s;
    int32_t block, pad[3];
};
struct spd_plan_header {
    uint32_t magic;
    int32_t batch, tokens, window, sinks;
    int32_t n_small, n_large, n_merge, n_write;
    int64_t held;
    spd_pages_config cfg;                // of the handle that made the plan
    int32_t seqs, table, small, large, merge, write;            // byte offsets
    int32_t merge_rows, max_end;         // most rows of a merge, most positions of a sequence
    size_t bytes, part_small, part_large, workspace;             // of the plan; byte offsets into the workspace (counters at 0); its size
};

// partial results: per slot and KV head `rows` x (d outputs, then maximum and sum), fp32
inline size_t spd_part_floats(int rows, int d) { return (size_t)rows * (d + 2); }
