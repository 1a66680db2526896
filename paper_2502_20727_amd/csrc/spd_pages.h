// Paged KV cache: the handle, the plan of a step as host and kernels read it, and the layout of a page.
#pragma once

#include <cmath>

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

// ------------------------------------------------------------------------------------------
// How work is cut, on the host and on the device alike: a step has the same items, and the same results, whoever planned it.
// ------------------------------------------------------------------------------------------
// The chip holds this many workgroups of the kernel for few rows at once (one of eight waves per compute unit: 48 sequences of up to 16000
// 31.0 us, two of four waves 33 to 38), two per compute unit of the one for many.
constexpr int SPD_SMALL_TARGET = 256, SPD_COMPUTE_UNITS = 256;
constexpr int SPD_LARGE_MIN_BLOCKS = 8;
// Of the kernel for few rows over 4-bit pages two fit on a compute unit.  It is cut for them where there are pieces (times KV heads) enough that
// half as many would be uneven: us a call (means of three draws of lengths), cut for 256 / 512 workgroups: 136 sequences of up to 8000 22.4 / 19.8, 200 34.4 / 26.4, 300 44.3 / 37.2, 24 on
// 8 heads 32.3 / 26.0, 64 on 8 53.0 / 53.1; short ones gain nothing, 192 of up to 2000 12.0 / 12.4.  Of fewer pieces more parts are more to join: 48 of up to 16000 15.4 / 16.2 (though
// 100 of up to 8000 17.5 / 16.7, 40 on 5 heads, which are more, 34.6 / 26.8).
SPD_HD int spd_small_target(int cache_dtype, int64_t pieces) { return cache_dtype == SPD_E2M1 && pieces > SPD_SMALL_TARGET / 2 ? 2 * SPD_SMALL_TARGET : SPD_SMALL_TARGET; }

// the visible blocks of rows row0 .. row0 + rows - 1 of a sequence whose first new position is `pos`
struct spd_piece {
    int32_t sink_blocks, block0, total;
};
SPD_HD spd_piece spd_piece_between(int first, int last, int window, int sinks) {      // to queries at positions first .. last
    spd_piece w;
    const int low = window && first >= window ? (first - window + 1) / 16 : 0;      // first block of the first row's window
    w.sink_blocks = (int)(((int64_t)(sinks < last + 1 ? sinks : last + 1) + 15) / 16);
    w.block0 = low;
    if (w.sink_blocks >= low) w.sink_blocks = w.block0 = 0;
    w.total = w.sink_blocks + last / 16 + 1 - w.block0;
    return w;
}
SPD_HD spd_piece spd_piece_of(int group, int pos, int row0, int rows, int window, int sinks) {
    return spd_piece_between(pos + row0 / group, pos + (row0 + rows - 1) / group, window, sinks);
}

// Pieces are cut into items of at most `chunk` blocks, first what each of `target` workgroups would have of them; `unit` blocks go together.
SPD_HD int64_t spd_first_chunk(int64_t total, int kv, int target, int unit) {
    const int64_t c = ((total * kv + target - 1) / target + unit - 1) / unit * unit;
    return c > unit ? c : unit;
}
// what lengths leave over after whole chunks makes more items than the target: longer chunks, SPD_LONGER times at most, while cutting is what makes them
constexpr int SPD_LONGER = 16;
SPD_HD int64_t spd_next_chunk(int64_t chunk, int unit) { return (chunk + chunk / 16 + unit) / unit * unit; }
SPD_HD int spd_parts(int total, int64_t chunk, int most) {
    const int64_t n = (total + chunk - 1) / chunk;
    return n < most ? (int)n : most;
}
// the most items a piece is cut into.  Many rows:
SPD_HD int spd_most_large(int blocks) { return blocks / SPD_LARGE_MIN_BLOCKS > 1 ? blocks / SPD_LARGE_MIN_BLOCKS : 1; }
// Rows whose blocks go round a workgroup's waves three times or less are not cut.  Beyond that a turn of a wave (a pair of blocks) takes
// about as long as 0.15 of the join of a part by one of `sets` sets of threads, which gives the number of parts that ends first when
// there is room for all of them.  (us a call, 0.05 / 0.1 / 0.3: 16 sequences of 4096 11.5 / 11.0 / 11.5, one of 32000 17.9 / 15.8 / 14.6; 64
// of 500: 6.8 uncut, 8.4 in two parts)
SPD_HD int spd_sets(int group) { return group > 8 ? 1 : group > 4 ? 2 : group > 2 ? 4 : group > 1 ? 8 : 16; }
SPD_HD int spd_most_small(int blocks, int sets) {
    if (blocks <= 3 * 2 * SPD_SMALL_WAVES) return 1;
    const int square = 3 * blocks * sets / 20;      // (blocks: 2^23 at most)
    int n = (int)sqrtf((float)square);
    while (n * n > square) --n;
    while ((n + 1) * (n + 1) <= square) ++n;
    return n < blocks / 8 ? n : blocks / 8;
}
// Many rows: cut so that a workgroup per compute unit has work, or one and a half, or two (halves = 2, 3, 4), whichever is estimated to end first: the time
// in ns of `items` whose longest has `longest` blocks, `slots` of them parts; in whole numbers, since floating-point products are rounded differently on the host
// and on the device, and of two cuts that take as long (in one of eighty such pairs) the one would choose the first and the other the second.  A tile of four
// blocks takes a workgroup 1.65 us by itself and 2.35 beside another; a join costs a launch and its partial results twice (66 KB each, 0.018 us).
// us a call, cut for 256 / 384 / 512 workgroups: three windowed chunks of 333 tokens, 5 heads 23.2 / 26.3 / 26.1, without the window 38.8 / 37.2 / 35.4, the
// same over e4m3 41.3 / 37.8 / 34.6, d 64 28.7 / 27.2 / 27.9, two of 333 behind 16000 64.3 / 62.1 / 55.7, one of 300 behind 2000, 8 heads of 8 63.3 / 49.1 /
// 41.9.  Of 200 calls of all types and widths that the three cut differently this picks cuts that are 1 % slower than the best of them on average, 15 % at
// most (with a part at 0.04 us: 3 % and 39 %).
SPD_HD int64_t spd_estimate_large(int longest, int64_t items, int64_t slots, int kv) {
    const int64_t groups = items * kv, tiles = (longest + 3) / 4, rounds = (groups + 2 * SPD_COMPUTE_UNITS - 1) / (2 * SPD_COMPUTE_UNITS);
    return tiles * (groups <= SPD_COMPUTE_UNITS ? 1650 : 2350 * rounds) + (slots ? 3000 + 18 * slots * kv : 0);
}
// blocks of the i-th of `parts` items of a piece of `total` blocks
SPD_HD int spd_item_first(int total, int unit, int parts, int i) {      // i * units / parts whole units (parts: some hundred at most)
    const unsigned units = (total + unit - 1) / unit, n = parts;
    return (int)(i * (units / n) + i * (units % n) / n) * unit;
}
SPD_HD int spd_item_count(int total, int unit, int parts, int i) {
    const int end = spd_item_first(total, unit, parts, i + 1);
    return (end < total ? end : total) - spd_item_first(total, unit, parts, i);
}

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
    // A plan that is made on the device: on the host the n_* are the most there can be (and so many workgroups are launched), on the device those of the step.
    int32_t on_device;
    int32_t q_len, entries;              // limits: new tokens of a request, entries of its row of the page table
    int32_t reqs, cuts, backs, order;           // byte offsets of what the first of its kernels leaves for the second
    size_t device_bytes;
    int32_t rows, free0, top, n_backs;   // of the step: rows in use, free pages before it, and with those that came back; requests that gave some back
    int32_t sorted;                      // pieces of few rows begin at the items that `order` says
};
// what is known of a request, and of a piece of 128 of its rows, between the two kernels
struct spd_plan_req {
    int32_t pos, q_len, tok0, state;     // first position, rows, the first row; 0: fine, 1: pages come back, else why it is not served
    int32_t need0, back0, back, few;     // new pages, pages that come back: of those before it, its own; number of its piece of few rows
    int32_t item0, parts, slot0, group;  // few rows
    int32_t piece0, pieces;              // many
    int32_t write0, writes;              // 16-position blocks that receive new tokens
};
struct spd_plan_cut {
    int32_t item0, parts, slot0, merge;
};
struct spd_plan_back {                   // a request whose pages come back: pages that come back before its own
    int32_t back0, req;
};
constexpr int SPD_BUILD_BATCH = 4096, SPD_BUILD_PIECES = 8192;      // most requests, pieces of 128 rows, of a plan made on the device

// partial results: per slot and KV head `rows` x (d outputs, then maximum and sum), fp32
inline size_t spd_part_floats(int rows, int d) { return (size_t)rows * (d + 2); }
