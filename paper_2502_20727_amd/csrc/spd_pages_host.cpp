// Host side of the paged KV cache: the handle, the rotary table and the plan of a step.
// Nothing in this file touches a device.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "spd_pages.h"

namespace {

// The chip holds SMALL_TARGET workgroups of the kernel for few rows at once (one of eight waves per compute unit: 48 sequences of up to 16000
// 31.0 us, two of four waves 33 to 38), two per compute unit of the one for many.
constexpr int SMALL_TARGET = 256, COMPUTE_UNITS = 256;
constexpr int LARGE_MIN_BLOCKS = 8;

struct Piece {
    int seq, row0, rows, sink_blocks, block0, total;
};

// the visible blocks of rows row0 .. row0 + rows - 1
Piece piece_of(const spd_pages *P, int seq, int pos, int row0, int rows, int window, int sinks) {
    Piece w;
    w.seq = seq;
    w.row0 = row0;
    w.rows = rows;
    const int first = pos + row0 / P->group, last = pos + (row0 + rows - 1) / P->group;
    const int low = window && first >= window ? (first - window + 1) / 16 : 0;      // first block of the first row's window
    w.sink_blocks = (int)(((int64_t)std::min(sinks, last + 1) + 15) / 16);
    w.block0 = low;
    if (w.sink_blocks >= low) w.sink_blocks = w.block0 = 0;
    w.total = w.sink_blocks + last / 16 + 1 - w.block0;
    return w;
}

// Cuts pieces into items of at most `chunk` blocks, what each of `target` workgroups would have of them (0: not at all), into no more than `target`
// items where the pieces are fewer; `unit` blocks go together.  most(blocks): the most items a piece is cut into.
template <class Most>
void cut(const std::vector<Piece> &pieces, const std::vector<spd_plan_seq> &seqs, int kv, int target, int unit, Most most,
         std::vector<spd_plan_item> &items, std::vector<spd_plan_merge> &merges, int &slots) {
    int64_t total = 0;
    for (const Piece &w : pieces) total += w.total;
    int64_t chunk = target ? std::max<int64_t>(unit, ((total * kv + target - 1) / target + unit - 1) / unit * unit) : 0;
    auto parts_of = [&](const Piece &w) { return chunk ? (int)std::min<int64_t>(most(w.total), (w.total + chunk - 1) / chunk) : 1; };
    // (what lengths leave over after whole chunks makes more items than the target: longer chunks, while cutting is what makes them)
    for (int i = 0; i < 16 && chunk; ++i) {
        int64_t n = 0;
        for (const Piece &w : pieces) n += parts_of(w);
        if (n * kv <= target || n == (int64_t)pieces.size()) break;
        chunk = (chunk + chunk / 16 + unit) / unit * unit;
    }
    for (const Piece &w : pieces) {
        const int units = (w.total + unit - 1) / unit;
        const int parts = std::min(units, parts_of(w));
        for (int i = 0; i < parts; ++i) {
            spd_plan_item it;
            it.s = seqs[w.seq];
            it.row0 = w.row0;
            it.sink_blocks = w.sink_blocks;
            it.block0 = w.block0;
            it.first = (int)((int64_t)i * units / parts) * unit;
            it.count = std::min((int)((int64_t)(i + 1) * units / parts) * unit, w.total) - it.first;
            it.slot = parts > 1 ? slots + i : -1;
            it.slot0 = slots;
            it.parts = parts;
            it.group = (int)merges.size();
            it.pad[0] = it.pad[1] = it.pad[2] = 0;
            items.push_back(it);
        }
        if (parts > 1) {
            merges.push_back(spd_plan_merge{seqs[w.seq], w.row0, w.rows, slots, parts});
            slots += parts;
        }
    }
    // the longest first, so that none of them starts when the rest is done
    std::stable_sort(items.begin(), items.end(), [](const spd_plan_item &a, const spd_plan_item &b) { return a.count > b.count; });
}

// Many rows: cut so that a workgroup per compute unit has work, or one and a half, or two, whichever is estimated to end first.  A tile of four
// blocks takes a workgroup 1.65 us by itself and 2.35 beside another; a join costs a launch and its partial results twice (66 KB each, 0.018 us).
// us a call, cut for 256 / 384 / 512 workgroups: three windowed chunks of 333 tokens, 5 heads 23.2 / 26.3 / 26.1, without the window 38.8 / 37.2 / 35.4, the
// same over e4m3 41.3 / 37.8 / 34.6, d 64 28.7 / 27.2 / 27.9, two of 333 behind 16000 64.3 / 62.1 / 55.7, one of 300 behind 2000, 8 heads of 8 63.3 / 49.1 /
// 41.9.  Of 200 calls of all types and widths that the three cut differently this picks cuts that are 1 % slower than the best of them on average, 15 % at
// most (with a part at 0.04 us: 3 % and 39 %).
void cut_large(const std::vector<Piece> &pieces, const std::vector<spd_plan_seq> &seqs, int kv, std::vector<spd_plan_item> &items,
               std::vector<spd_plan_merge> &merges, int &slots) {
    if (pieces.empty()) return;
    double least = 0.0;
    for (int halves = 2; halves <= 4; ++halves) {
        std::vector<spd_plan_item> i;
        std::vector<spd_plan_merge> m;
        int n = 0;
        cut(pieces, seqs, kv, COMPUTE_UNITS * halves / 2, 4, [](int blocks) { return std::max(1, blocks / LARGE_MIN_BLOCKS); }, i, m, n);
        const int64_t groups = (int64_t)i.size() * kv;
        const double tiles = (i[0].count + 3) / 4, rounds = (double)((groups + 2 * COMPUTE_UNITS - 1) / (2 * COMPUTE_UNITS));
        const double us = tiles * (groups <= COMPUTE_UNITS ? 1.65 : 2.35 * rounds) + (n ? 3.0 + 0.018 * n * kv : 0.0);
        if (halves == 2 || us < least) {
            least = us;
            items.swap(i);
            merges.swap(m);
            slots = n;
        }
    }
}

template <class T>
int place(size_t &at, const std::vector<T> &v) {
    at = (at + 15) & ~(size_t)15;
    const int here = (int)at;
    at += v.size() * sizeof(T);
    return here;
}
template <class T>
void put(char *plan, int at, const std::vector<T> &v) {
    if (!v.empty()) std::memcpy(plan + at, v.data(), v.size() * sizeof(T));
}

int plan_impl(const spd_pages *P, int32_t batch, const int32_t *positions, const int32_t *q_lens, const int32_t *page_table, int32_t ld_table,
              int32_t window, int32_t sinks, void *plan_host, size_t capacity, size_t *bytes) {
    const spd_pages_config &c = P->cfg;
    if (!bytes || batch < 0 || batch > 65535 || window < 0 || sinks < 0 || (sinks && !window) || ld_table < 0) return SPD_EINVAL;
    if (batch && (!positions || !q_lens || !page_table)) return SPD_EINVAL;
    spd_plan_header h;
    std::memset(&h, 0, sizeof(h));
    int64_t tokens = 0, held = 0, entries = 0;
    for (int b = 0; b < batch; ++b) {
        if (positions[b] < 0 || q_lens[b] < 0 || (int64_t)positions[b] + q_lens[b] > c.max_ctx) return SPD_EINVAL;
        const int end = positions[b] + q_lens[b];
        if ((end + c.page_size - 1) / c.page_size > ld_table) return SPD_EINVAL;
        tokens += q_lens[b];
        held += end;
        entries += (end + c.page_size - 1) / c.page_size;
    }
    if (tokens > (1 << 24) || entries > (1 << 28)) return SPD_EINVAL;

    std::vector<spd_plan_seq> seqs(batch);
    std::vector<int32_t> table;
    table.reserve((size_t)entries);
    std::vector<uint8_t> uses((size_t)c.n_pages, 0);
    int tok0 = 0;
    int64_t held0 = 0;
    for (int b = 0; b < batch; ++b) {
        spd_plan_seq &s = seqs[b];
        s.pos = positions[b];
        s.q_len = q_lens[b];
        s.end = s.pos + s.q_len;
        s.pad = 0;
        s.tok0 = tok0;
        s.table = (int)table.size();
        s.held0 = held0;
        tok0 += s.q_len;
        held0 += s.end;
        h.max_end = std::max(h.max_end, s.end);
        for (int i = 0; i < (s.end + c.page_size - 1) / c.page_size; ++i) {
            const int32_t page = page_table[(size_t)b * ld_table + i];
            if (page < 0 || page >= c.n_pages) return SPD_EINVAL;
            if (uses[page] < 2) ++uses[page];
            table.push_back(page);
        }
    }
    std::vector<spd_plan_block> writes;
    for (int b = 0; b < batch; ++b) {
        const spd_plan_seq &s = seqs[b];
        if (!s.q_len) continue;
        for (int i = s.pos / c.page_size; i <= (s.end - 1) / c.page_size; ++i)
            if (uses[table[s.table + i]] != 1) return SPD_EINVAL;      // written here and in use elsewhere
        for (int blk = s.pos / 16; blk <= (s.end - 1) / 16; ++blk) writes.push_back(spd_plan_block{s, blk, {0, 0, 0}});
    }

    std::vector<Piece> few, many;
    for (int b = 0; b < batch; ++b) {
        const int64_t rows = (int64_t)seqs[b].q_len * P->group;
        if (rows == 0) continue;
        if (rows <= SPD_SMALL_ROWS) {
            few.push_back(piece_of(P, b, seqs[b].pos, 0, (int)rows, window, sinks));
            continue;
        }
        for (int64_t r = 0; r < rows; r += SPD_LARGE_ROWS)
            many.push_back(piece_of(P, b, seqs[b].pos, (int)r, (int)std::min<int64_t>(SPD_LARGE_ROWS, rows - r), window, sinks));
    }
    std::vector<spd_plan_item> small, large;
    std::vector<spd_plan_merge> joined, merges;      // (the rows of the kernel for few are joined by the last of their items)
    int small_slots = 0, large_slots = 0;
    const bool counted = (int64_t)few.size() * c.n_kv_heads <= SPD_COUNTERS;
    // Rows whose blocks go round a workgroup's waves three times or less are not cut.  Beyond that a turn of a wave (a pair of blocks) takes
    // about as long as 0.15 of the join of a part by one of `sets` sets of threads, which gives the number of parts that ends first when
    // there is room for all of them.  (us a call, 0.05 / 0.1 / 0.3: 16 sequences of 4096 11.5 / 11.0 / 11.5, one of 32000 17.9 / 15.8 / 14.6; 64
    // of 500: 6.8 uncut, 8.4 in two parts)
    const int sets = P->group > 8 ? 1 : P->group > 4 ? 2 : P->group > 2 ? 4 : P->group > 1 ? 8 : 16;
    auto most_small = [&](int blocks) { return blocks <= 3 * 2 * SPD_SMALL_WAVES ? 1 : (int)std::min(std::sqrt(0.15 * blocks * sets), blocks / 8.0); };
    cut(few, seqs, c.n_kv_heads, counted ? SMALL_TARGET : 0, 2, most_small, small, joined, small_slots);
    cut_large(many, seqs, c.n_kv_heads, large, merges, large_slots);
    for (const spd_plan_merge &m : merges) h.merge_rows = std::max(h.merge_rows, m.rows);

    h.magic = SPD_PLAN_MAGIC;
    h.batch = batch;
    h.tokens = (int)tokens;
    h.window = window;
    h.sinks = sinks;
    h.n_small = (int)small.size();
    h.n_large = (int)large.size();
    h.n_merge = (int)merges.size();
    h.n_write = (int)writes.size();
    h.held = held;
    h.cfg = c;
    size_t at = sizeof(h);
    h.seqs = place(at, seqs);
    h.table = place(at, table);
    h.small = place(at, small);
    h.large = place(at, large);
    h.merge = place(at, merges);
    h.write = place(at, writes);
    at = (at + 15) & ~(size_t)15;
    if (at > 0x7fffffffull) return SPD_EINVAL;
    h.bytes = at;
    // (the counters' place is kept wherever there is a workspace: another plan may use it next, and finds them at zero)
    h.part_small = small_slots || large_slots ? SPD_COUNTERS * 4 : 0;
    h.part_large = h.part_small + spd_align256((size_t)small_slots * c.n_kv_heads * spd_part_floats(SPD_SMALL_ROWS, c.head_dim) * 4);
    h.workspace = h.part_large + spd_align256((size_t)large_slots * c.n_kv_heads * spd_part_floats(SPD_LARGE_ROWS, c.head_dim) * 4);
    *bytes = h.bytes;
    if (!plan_host) return SPD_OK;
    if (capacity < h.bytes) return SPD_EINVAL;
    char *plan = (char *)plan_host;
    std::memset(plan, 0, h.bytes);
    std::memcpy(plan, &h, sizeof(h));
    put(plan, h.seqs, seqs);
    put(plan, h.table, table);
    put(plan, h.small, small);
    put(plan, h.large, large);
    put(plan, h.merge, merges);
    put(plan, h.write, writes);
    return SPD_OK;
}

}  // namespace

extern "C" {

int spd_pages_create(const spd_pages_config *cfg, spd_pages **out) {
    if (!cfg || !out) return SPD_EINVAL;
    *out = nullptr;
    const spd_pages_config &c = *cfg;
    if (c.n_q_heads <= 0 || c.n_kv_heads <= 0 || c.head_dim <= 0 || c.page_size <= 0 || c.n_pages <= 0 || c.max_ctx <= 0) return SPD_EINVAL;
    if (c.n_q_heads % c.n_kv_heads) return SPD_EINVAL;
    if (!(c.rope_base > 0.f) || !std::isfinite(c.rope_base)) return SPD_EINVAL;
    if ((c.dtype != SPD_BF16 && c.dtype != SPD_F16) || (c.cache_dtype != SPD_E4M3 && c.cache_dtype != SPD_BF16 && c.cache_dtype != SPD_F16))
        return SPD_EINVAL;
    if (c.cache_dtype != SPD_E4M3 && c.cache_dtype != c.dtype) return SPD_EUNSUPPORTED;
    if (c.head_dim != 64 && c.head_dim != 128) return SPD_EUNSUPPORTED;
    if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128 && c.page_size != 256) return SPD_EUNSUPPORTED;
    if (c.n_q_heads / c.n_kv_heads > 16 || c.n_q_heads > 1024) return SPD_EUNSUPPORTED;
    if (c.max_ctx > (1 << 26)) return SPD_EUNSUPPORTED;       // row numbers (token x head of the group) are 32-bit
    spd_pages *p = new (std::nothrow) spd_pages();
    if (!p) return SPD_EINVAL;
    p->cfg = c;
    p->group = c.n_q_heads / c.n_kv_heads;
    p->width = c.cache_dtype == SPD_E4M3 ? 1 : 2;
    p->shift = 0;
    while ((16 << p->shift) < c.page_size) ++p->shift;
    p->head_bytes = (size_t)c.page_size * (2 * (size_t)c.head_dim * p->width + 8);
    p->page_bytes = p->head_bytes * c.n_kv_heads;
    *out = p;
    return SPD_OK;
}

void spd_pages_destroy(spd_pages *pages) { delete pages; }

int spd_pages_get_sizes(const spd_pages *pages, spd_pages_sizes *out) {
    if (!pages || !out) return SPD_EINVAL;
    out->pool_bytes = pages->page_bytes * (size_t)pages->cfg.n_pages;
    out->rope_bytes = (size_t)pages->cfg.max_ctx * pages->cfg.head_dim * 4;
    return SPD_OK;
}

int spd_pages_rope_table(const spd_pages *pages, float *host) {
    if (!pages || !host) return SPD_EINVAL;
    try {
        const int half = pages->cfg.head_dim / 2;
        std::vector<double> theta(half);
        for (int j = 0; j < half; ++j) theta[j] = std::pow((double)pages->cfg.rope_base, -(double)j / half);
        const int n = pages->cfg.max_ctx, span = 1024;
        spd_parallel_for((n + span - 1) / span, [&](int k) {
            for (int p = k * span; p < std::min(n, (k + 1) * span); ++p)
                for (int j = 0; j < half; ++j) {
                    host[((size_t)p * half + j) * 2] = (float)std::cos(p * theta[j]);
                    host[((size_t)p * half + j) * 2 + 1] = (float)std::sin(p * theta[j]);
                }
        });
    } catch (...) {      // (no memory, no thread)
        return SPD_EINVAL;
    }
    return SPD_OK;
}

int spd_pages_plan(const spd_pages *pages, int32_t batch, const int32_t *positions, const int32_t *q_lens, const int32_t *page_table,
                   int32_t ld_table, int32_t window, int32_t sinks, void *plan_host, size_t capacity, size_t *bytes) {
    if (!pages) return SPD_EINVAL;
    try {
        return plan_impl(pages, batch, positions, q_lens, page_table, ld_table, window, sinks, plan_host, capacity, bytes);
    } catch (...) {      // (no memory)
        return SPD_EINVAL;
    }
}

int spd_pages_plan_get_info(const spd_pages *pages, const void *plan_host, spd_pages_plan_info *out) {
    if (!pages || !plan_host || !out) return SPD_EINVAL;
    spd_plan_header h;
    std::memcpy(&h, plan_host, sizeof(h));
    if (h.magic != SPD_PLAN_MAGIC || std::memcmp(&h.cfg, &pages->cfg, sizeof(h.cfg))) return SPD_EINVAL;
    out->batch = h.batch;
    out->tokens = h.tokens;
    out->held = h.held;
    out->workspace_bytes = h.workspace;
    return SPD_OK;
}

}  // extern "C"
