// Host side of the paged KV cache: the handle, the rotary table and the plan of a step.
// Nothing in this file touches a device.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "spd_pages.h"

namespace {

struct Piece : spd_piece {
    int seq, row0, rows;
};

Piece piece_of(const spd_pages *P, int seq, int pos, int row0, int rows, int window, int sinks) {
    Piece w;
    (spd_piece &)w = spd_piece_of(P->group, pos, row0, rows, window, sinks);
    w.seq = seq;
    w.row0 = row0;
    w.rows = rows;
    return w;
}

// Cuts pieces into items for `target` workgroups (0: not at all), into no more than so many where the pieces are fewer.  most(blocks): the most items a
// piece is cut into.
template <class Most>
void cut(const std::vector<Piece> &pieces, const std::vector<spd_plan_seq> &seqs, int kv, int target, int unit, Most most,
         std::vector<spd_plan_item> &items, std::vector<spd_plan_merge> &merges, int &slots) {
    int64_t total = 0;
    for (const Piece &w : pieces) total += w.total;
    int64_t chunk = target ? spd_first_chunk(total, kv, target, unit) : 0;
    auto parts_of = [&](const Piece &w) { return chunk ? spd_parts(w.total, chunk, most(w.total)) : 1; };
    for (int i = 0; i < SPD_LONGER && chunk; ++i) {
        int64_t n = 0;
        for (const Piece &w : pieces) n += parts_of(w);
        if (n * kv <= target || n == (int64_t)pieces.size()) break;
        chunk = spd_next_chunk(chunk, unit);
    }
    for (const Piece &w : pieces) {
        const int parts = std::min((w.total + unit - 1) / unit, parts_of(w));
        for (int i = 0; i < parts; ++i) {
            spd_plan_item it;
            it.s = seqs[w.seq];
            it.row0 = w.row0;
            it.sink_blocks = w.sink_blocks;
            it.block0 = w.block0;
            it.first = spd_item_first(w.total, unit, parts, i);
            it.count = spd_item_count(w.total, unit, parts, i);
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

void cut_large(const std::vector<Piece> &pieces, const std::vector<spd_plan_seq> &seqs, int kv, std::vector<spd_plan_item> &items,
               std::vector<spd_plan_merge> &merges, int &slots) {
    if (pieces.empty()) return;
    int64_t least = 0;
    for (int halves = 2; halves <= 4; ++halves) {
        std::vector<spd_plan_item> i;
        std::vector<spd_plan_merge> m;
        int n = 0;
        cut(pieces, seqs, kv, SPD_COMPUTE_UNITS * halves / 2, 4, spd_most_large, i, m, n);
        const int64_t ns = spd_estimate_large(i[0].count, (int64_t)i.size(), n, kv);
        if (halves == 2 || ns < least) {
            least = ns;
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
    const int sets = spd_sets(P->group);
    auto most_small = [&](int blocks) { return spd_most_small(blocks, sets); };
    cut(few, seqs, c.n_kv_heads, counted ? spd_small_target(c.cache_dtype, (int64_t)few.size() * c.n_kv_heads) : 0, 2, most_small, small, joined, small_slots);
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
    const bool coded = c.cache_dtype == SPD_E4M3 || c.cache_dtype == SPD_E2M1;
    if ((c.dtype != SPD_BF16 && c.dtype != SPD_F16) || (!coded && c.cache_dtype != SPD_BF16 && c.cache_dtype != SPD_F16)) return SPD_EINVAL;
    if (!coded && c.cache_dtype != c.dtype) return SPD_EUNSUPPORTED;
    if (c.head_dim != 64 && c.head_dim != 128) return SPD_EUNSUPPORTED;
    if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128 && c.page_size != 256) return SPD_EUNSUPPORTED;
    if (c.n_q_heads / c.n_kv_heads > 16 || c.n_q_heads > 1024) return SPD_EUNSUPPORTED;
    if (c.max_ctx > (1 << 26)) return SPD_EUNSUPPORTED;       // row numbers (token x head of the group) are 32-bit
    spd_pages *p = new (std::nothrow) spd_pages();
    if (!p) return SPD_EINVAL;
    p->cfg = c;
    p->group = c.n_q_heads / c.n_kv_heads;
    p->row_bytes = c.cache_dtype == SPD_E2M1 ? c.head_dim / 2 + c.head_dim / 32 : c.head_dim * (c.cache_dtype == SPD_E4M3 ? 1 : 2) + 4;
    p->shift = 0;
    while ((16 << p->shift) < c.page_size) ++p->shift;
    p->head_bytes = (size_t)c.page_size * 2 * p->row_bytes;
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

int64_t spd_pages_estimate(int32_t longest, int32_t items, int32_t slots, int32_t n_kv_heads) {
    if (longest <= 0 || items <= 0 || slots < 0 || n_kv_heads <= 0) return SPD_EINVAL;
    return spd_estimate_large(longest, items, slots, n_kv_heads);
}

int spd_pages_reserve(const spd_pages *pages, const spd_pages_limits *limits, void *plan_host, size_t capacity, size_t *bytes, size_t *device_bytes) {
    if (!pages || !limits || !bytes || !device_bytes) return SPD_EINVAL;
    const spd_pages_config &c = pages->cfg;
    const spd_pages_limits &l = *limits;
    if (l.batch <= 0 || l.tokens <= 0 || l.q_len <= 0 || l.q_len > l.tokens || l.entries <= 0 || l.window < 0 || l.sinks < 0 || (l.sinks && !l.window)) return SPD_EINVAL;
    if (l.batch > SPD_BUILD_BATCH || l.tokens > (1 << 24) || (int64_t)l.batch * l.entries > (1 << 28)) return SPD_EUNSUPPORTED;
    const int64_t rows = (int64_t)l.tokens * pages->group, kv = c.n_kv_heads;
    const int64_t most_few = std::min(l.batch, l.tokens);
    int64_t pieces = 0;      // of many rows
    if ((int64_t)l.q_len * pages->group > SPD_SMALL_ROWS) pieces = rows / SPD_LARGE_ROWS + std::min<int64_t>(l.batch, rows / (SPD_SMALL_ROWS + 1));
    if (pieces > SPD_BUILD_PIECES) return SPD_EUNSUPPORTED;
    // Items, and those of them that are parts: with no more items than the target no more parts than that; with chunks made longer SPD_LONGER times, 2.6 times
    // what a workgroup would have, a piece that is longer than that has less than twice its length's worth of them.
    const int64_t small_slots = spd_small_target(c.cache_dtype, most_few * kv) / kv, large_slots = pieces ? 2 * SPD_COMPUTE_UNITS / kv : 0;
    spd_plan_header h;
    std::memset(&h, 0, sizeof(h));
    h.magic = SPD_PLAN_MAGIC;
    h.batch = l.batch;
    h.tokens = l.tokens;
    h.window = l.window;
    h.sinks = l.sinks;
    h.n_small = (int)(most_few + small_slots);
    h.n_large = (int)(pieces + large_slots);
    h.n_merge = (int)std::min<int64_t>(pieces, large_slots / 2);
    h.n_write = (int)std::min<int64_t>(l.tokens, l.tokens / 16 + 2 * most_few);
    h.cfg = c;
    h.merge_rows = SPD_LARGE_ROWS;
    h.on_device = 1;
    h.q_len = l.q_len;
    h.entries = l.entries;
    size_t at = sizeof(h);
    auto room = [&](size_t n, size_t size) {
        at = (at + 15) & ~(size_t)15;
        const size_t here = at;
        at += n * size;
        return (int)here;
    };
    h.seqs = room(l.batch, sizeof(spd_plan_seq));
    h.reqs = room(l.batch, sizeof(spd_plan_req));
    h.cuts = room(pieces, sizeof(spd_plan_cut));
    h.backs = room(l.batch, sizeof(spd_plan_back));
    h.order = room(most_few, 4);
    h.small = room(h.n_small, sizeof(spd_plan_item));
    h.large = room(h.n_large, sizeof(spd_plan_item));
    h.merge = room(h.n_merge, sizeof(spd_plan_merge));
    h.write = room(h.n_write, sizeof(spd_plan_block));
    h.table = room((size_t)l.batch * l.entries, 4);
    at = spd_align256(at);
    if (at > 0x7fffffffull) return SPD_EUNSUPPORTED;
    *bytes = (sizeof(h) + 15) & ~(size_t)15;
    *device_bytes = h.device_bytes = at;
    h.bytes = *bytes;
    h.part_small = small_slots || large_slots ? SPD_COUNTERS * 4 : 0;
    h.part_large = h.part_small + spd_align256((size_t)(small_slots * kv) * spd_part_floats(SPD_SMALL_ROWS, c.head_dim) * 4);
    h.workspace = h.part_large + spd_align256((size_t)(large_slots * kv) * spd_part_floats(SPD_LARGE_ROWS, c.head_dim) * 4);
    if (!plan_host) return SPD_OK;
    if (capacity < h.bytes) return SPD_EINVAL;
    std::memset(plan_host, 0, h.bytes);
    std::memcpy(plan_host, &h, sizeof(h));
    return SPD_OK;
}

}  // extern "C"
