// The plan of a step made on the device, from request lengths that are there: pages taken from the free list and given back, the page table's new
// entries, rows and slots of the new tokens, and the work of spd_pages_write() and spd_pages_attention() in the form that the host's plan has it.
//
// Two kernels.  The first, a single workgroup, adds up: everything that one request has to know of the others is a prefix sum over them (rows, pages
// needed, pages that come back, blocks written, items), and the chunk that work is cut into is a search over sums, as on the host
// (spd_pages.h).  The second has a workgroup per request, checks its pages and writes what is the request's.  A request whose pages are not of
// the pool is found out there and leaves its items empty.
#include <algorithm>
#include <cstring>

#include "spd_pages.h"

namespace {

struct BuildArgs {
    const int32_t *positions, *q_lens, *n_free;
    int32_t *page_table, *free_pages, *n_free_out;
    int32_t *positions_out, *served, *first_row, *row_seq, *row_pos;
    int64_t *row_slot;
    char *plan;
    int64_t ld_table;
    int batch, tokens, q_len, entries, window, sinks;      // limits
    int page_size, n_pages, kv, group, most_end;           // most_end: positions a request may have
    int seqs, reqs, cuts, small, large, merge, write, table;      // byte offsets
    int tails;                                             // workgroups of the second kernel for rows behind the last request
};

constexpr int THREADS = 1024, WAVES = THREADS / 64;

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Exclusive prefix sums over the workgroup of N numbers a thread, and their totals.  `lds`: WAVES * N.
template <int N>
__device__ __forceinline__ void scan(int (&v)[N], int (&total)[N], int *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int mine[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int x = v[n];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(x, d, 64);
            x += lane >= d ? y : 0;
        }
        mine[n] = x - v[n];
        if (lane == 63) lds[wave * N + n] = x;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int x = lds[w * N + n];
            before += w < wave ? x : 0;
            all += x;
        }
        v[n] = before + mine[n];
        total[n] = all;
    }
    __syncthreads();
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_xor(x, d, 64);
        x = y > x ? y : x;
    }
    return x;
}

// The first kernel.  PER requests, and as many pieces of 128 rows as are needed, in a thread, one after the other.
template <int PER>
__global__ void __launch_bounds__(THREADS) k_build_sums(BuildArgs A) {
    __shared__ int lds[WAVES * 4];
    __shared__ int few_total[PER * THREADS], many_total[SPD_BUILD_PIECES];
    __shared__ unsigned short few_most[PER * THREADS];
    __shared__ unsigned long long sums[2];                 // blocks of the pieces of few rows, of many
    __shared__ int fits[4][WAVES];                         // does a chunk make few enough items?  few rows; many, for 2, 3 and 4 halves
    __shared__ double us[3];
    __shared__ int bucket[2][256], longest[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    spd_plan_header &H = *(spd_plan_header *)A.plan;
    if (tid < 2) {
        sums[tid] = 0;
        longest[tid] = 1;
    }
    for (int i = tid; i < 512; i += THREADS) bucket[i >> 8][i & 255] = 0;
    const int free_now = A.n_free ? *A.n_free : 0, free0 = free_now < 0 ? 0 : free_now > A.n_pages ? A.n_pages : free_now;
    int pos[PER], q[PER], rows[PER];
    // rows
    int v1[1] = {0}, t1[1];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = tid * PER + k;
        pos[k] = b < A.batch ? A.positions[b] : 0;
        q[k] = b < A.batch ? A.q_lens[b] : 0;
        rows[k] = q[k] > 0 && q[k] <= A.q_len ? q[k] : 0;
    }
    const int most_rows = A.tokens + 1;          // (where their sums stop, lest they overflow)
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        v1[0] += rows[k];
        v1[0] = v1[0] < most_rows ? v1[0] : most_rows;
    }
    {
        // as scan(), of sums that stop
        int x = v1[0];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(x, d, 64);
            x += lane >= d ? y : 0;
            x = x < most_rows ? x : most_rows;
        }
        const int up = __shfl_up(x, 1, 64);
        if (lane == 63) lds[wave] = x;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) before = all;
            all += lds[w];
            all = all < most_rows ? all : most_rows;
        }
        before += lane ? up : 0;
        v1[0] = before < most_rows ? before : most_rows;
        t1[0] = all;
        __syncthreads();
    }
    // pages that come back, pages that are needed
    int tok0[PER], back[PER], need[PER];
    bool fine[PER];
    int v2[2] = {0, 0}, t2[2];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        tok0[k] = v1[0] < A.tokens ? v1[0] : A.tokens;
        v1[0] += rows[k];
        fine[k] = pos[k] >= 0 && q[k] >= SPD_STEP_RELEASE && q[k] <= A.q_len && pos[k] <= A.most_end - (q[k] > 0 ? q[k] : 0) && v1[0] <= A.tokens;
        v1[0] = v1[0] < most_rows ? v1[0] : most_rows;
        back[k] = need[k] = 0;
        if (fine[k] && A.free_pages) {
            const int held = ceil_div(pos[k], A.page_size);
            if (q[k] > 0) need[k] = ceil_div(pos[k] + q[k], A.page_size) - held;
            if (q[k] < 0) back[k] = held;
        }
        v2[0] += back[k];
        v2[1] += need[k];
    }
    scan(v2, t2, lds);
    const int top = t2[0] < A.n_pages - free0 ? free0 + t2[0] : A.n_pages;
    // pieces
    int back0[PER], need0[PER], few[PER], pieces[PER], writes[PER];
    int v4[4] = {0, 0, 0, 0}, t4[4];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        back0[k] = v2[0];
        need0[k] = v2[1];
        v2[0] += back[k];
        v2[1] += need[k];
        few[k] = pieces[k] = writes[k] = 0;
        const bool got = fine[k] && (need[k] == 0 || v2[1] <= top);
        if (got && q[k] > 0) {
            const int n = q[k] * A.group;
            few[k] = n <= SPD_SMALL_ROWS;
            pieces[k] = few[k] ? 0 : ceil_div(n, SPD_LARGE_ROWS);
            writes[k] = (pos[k] + q[k] - 1) / 16 - pos[k] / 16 + 1;
        }
        if (!fine[k]) need[k] = SPD_STEP_LENGTHS;          // (from here on: why not)
        else if (!got) need[k] = SPD_STEP_NO_PAGES;
        v4[0] += few[k];
        v4[1] += pieces[k];
        v4[2] += writes[k];
        v4[3] += got ? need[k] : 0;
    }
    scan(v4, t4, lds);
    const int n_few = t4[0], n_many = t4[1];
    const int sets = spd_sets(A.group);
    int few0[PER], piece0[PER], write0[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        few0[k] = v4[0];
        piece0[k] = v4[1];
        write0[k] = v4[2];
        v4[0] += few[k];
        v4[1] += pieces[k];
        v4[2] += writes[k];
        int total = 0;
        if (few[k]) {
            total = spd_piece_of(A.group, pos[k], 0, q[k] * A.group, A.window, A.sinks).total;
            few_total[few0[k]] = total;
            const int most = spd_most_small(total, sets);
            few_most[few0[k]] = (unsigned short)(most < 65535 ? most : 65535);
        }
        if (n_few) {
            total = wave_sum(total);                       // (at most 64 * 2^23)
            if (lane == 0 && total) atomicAdd(&sums[0], (unsigned long long)total);
        }
        // a wave together for each of its requests of many rows
        unsigned long long todo = __builtin_amdgcn_ballot_w64(pieces[k] > 0);
        while (todo) {
            const int from = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int p = __builtin_amdgcn_readlane(pos[k], from), n = __builtin_amdgcn_readlane(q[k], from) * A.group,
                      at = __builtin_amdgcn_readlane(piece0[k], from);
            unsigned long long all = 0;
            for (int i = lane; i * SPD_LARGE_ROWS < n; i += 64) {
                const int row0 = i * SPD_LARGE_ROWS, left = n - row0;
                const int blocks = spd_piece_of(A.group, p, row0, left < SPD_LARGE_ROWS ? left : SPD_LARGE_ROWS, A.window, A.sinks).total;
                many_total[at + i] = blocks;
                all += blocks;
            }
            atomicAdd(&sums[1], all);
        }
    }
    __syncthreads();
    // The chunks: every wave tries the one that is `wave` times longer than the first
    const bool cut_few = n_few && (int64_t)n_few * A.kv <= SPD_COUNTERS;
    auto longer = [](int64_t chunk, int times, int unit) {
        for (int i = 0; i < times; ++i) chunk = spd_next_chunk(chunk, unit);
        return chunk;
    };
    const int64_t first_few = spd_first_chunk((int64_t)sums[0], A.kv, SPD_SMALL_TARGET, 2);
    auto first_many = [&](int h) { return spd_first_chunk((int64_t)sums[1], A.kv, SPD_COMPUTE_UNITS * (h + 2) / 2, 4); };
    // (chunks and pieces are less than 2^31 blocks, so that 32 bits divide: a chunk that is longer than any piece is as good as the longest of 2^30)
    auto short_of = [](int64_t chunk) { return (int)(chunk < 1 << 30 ? chunk : 1 << 30); };
    if (cut_few) {
        const int chunk = short_of(longer(first_few, wave, 2));
        int n = 0;
        for (int i = lane; i < n_few; i += 64) {
            const int parts = ceil_div(few_total[i], chunk), most = few_most[i];
            n += parts < most ? parts : most;
        }
        n = wave_sum(n);
        if (lane == 0) fits[0][wave] = (int64_t)n * A.kv <= SPD_SMALL_TARGET || n == n_few;
    }
    if (n_many) {
#pragma unroll
        for (int h = 0; h < 3; ++h) {
            const int chunk = short_of(longer(first_many(h), wave, 4));
            int n = 0;
            for (int i = lane; i < n_many; i += 64) {
                const int parts = ceil_div(many_total[i], chunk), most = spd_most_large(many_total[i]);
                n += parts < most ? parts : most;
            }
            n = wave_sum(n);
            if (lane == 0) fits[h + 1][wave] = (int64_t)n * A.kv <= SPD_COMPUTE_UNITS * (h + 2) / 2 || n == n_many;
        }
    }
    __syncthreads();
    auto chosen = [&](int which, int64_t first, int unit) {
        int times = 0;
        while (times < SPD_LONGER && !fits[which][times]) ++times;
        return short_of(longer(first, times, unit));
    };
    static_assert(WAVES == SPD_LONGER, "a wave for each chunk that is tried");
    const int few_chunk = cut_few ? chosen(0, first_few, 2) : 0;
    auto parts_few = [&](int i) {
        if (!few_chunk) return 1;
        const int parts = ceil_div(few_total[i], few_chunk), most = few_most[i], units = ceil_div(few_total[i], 2);
        const int n = parts < most ? parts : most;
        return n < units ? n : units;
    };
    auto parts_many = [&](int i, int chunk) {
        const int parts = ceil_div(many_total[i], chunk), most = spd_most_large(many_total[i]), units = ceil_div(many_total[i], 4);
        const int n = parts < most ? parts : most;
        return n < units ? n : units;
    };
    int many_chunk = 1 << 30;
    if (n_many) {
        if (wave < 3) {
            const int chunk = chosen(wave + 1, first_many(wave), 4);
            int n = 0, slots = 0, most = 0;
            for (int i = lane; i < n_many; i += 64) {
                const int parts = parts_many(i, chunk);
                n += parts;
                slots += parts > 1 ? parts : 0;
                // the longest of a piece's items is its last, or (as the last may have less than four blocks in its last unit) the one before
                for (int k = parts > 2 ? parts - 2 : 0; k < parts; ++k) {
                    const int c = spd_item_count(many_total[i], 4, parts, k);
                    most = c > most ? c : most;
                }
                if (parts > 2) {                           // an earlier one has all of the units that the last has where two or more have one more
                    const int units = ceil_div(many_total[i], 4), c = units % parts >= 2 ? ceil_div(units, parts) * 4 : 0;
                    most = c > most ? c : most;
                }
            }
            n = wave_sum(n);
            slots = wave_sum(slots);
            most = wave_max(most);
            if (lane == 0) us[wave] = spd_estimate_large(most, n, slots, A.kv);
        }
        __syncthreads();
        int h = 0;
        if (us[1] < us[0]) h = 1;
        if (us[2] < us[h]) h = 2;
        many_chunk = chosen(h + 1, first_many(h), 4);
    }
    // Items: those of a piece one after the other, the pieces with the longest items first, by 256 lengths
    int parts[PER], v3[3] = {0, 0, 0}, t3[3];
    int longest_few = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        parts[k] = few[k] ? parts_few(few0[k]) : 0;
        v3[0] += parts[k];
        v3[1] += parts[k] > 1 ? parts[k] : 0;
        v3[2] += parts[k] > 1;
        const int c = few[k] ? ceil_div(few_total[few0[k]], parts[k]) : 0;
        longest_few = c > longest_few ? c : longest_few;
    }
    scan(v3, t3, lds);
    const int n_small = t3[0];
    const int per = ceil_div(n_many, THREADS);             // pieces a thread
    int m3[3] = {0, 0, 0}, tm[3] = {0, 0, 0};
    int longest_many = 0;
    if (n_many) {
        for (int k = 0; k < per; ++k) {
            const int i = tid * per + k;
            if (i >= n_many) break;
            const int n = parts_many(i, many_chunk), c = ceil_div(many_total[i], n);
            m3[0] += n;
            m3[1] += n > 1 ? n : 0;
            m3[2] += n > 1;
            longest_many = c > longest_many ? c : longest_many;
        }
        scan(m3, tm, lds);
    }
    longest_few = wave_max(longest_few);
    longest_many = wave_max(longest_many);
    if (lane == 0) {
        atomicMax(&longest[0], longest_few);
        atomicMax(&longest[1], longest_many);
    }
    __syncthreads();
    auto bucket_of = [&](int which, int total, int n) { return 255 - (int)((int64_t)ceil_div(total, n) * 255 / longest[which]); };
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (few[k]) atomicAdd(&bucket[0][bucket_of(0, few_total[few0[k]], parts[k])], parts[k]);
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i >= n_many) break;
        const int n = parts_many(i, many_chunk);
        atomicAdd(&bucket[1][bucket_of(1, many_total[i], n)], n);
    }
    __syncthreads();
    if (wave < 2) {
        int x[4], all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = bucket[wave][lane * 4 + i];
            all += x[i];
        }
        int sum = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(sum, d, 64);
            sum += lane >= d ? y : 0;
        }
        sum -= all;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bucket[wave][lane * 4 + i] = sum;
            sum += x[i];
        }
    }
    __syncthreads();
    // (which of the pieces of one length comes first is left to chance: it is the order they are started in, and nothing else)
    spd_plan_req *reqs = (spd_plan_req *)(A.plan + A.reqs);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = tid * PER + k;
        if (b >= A.batch) break;
        spd_plan_req r;
        r.pos = pos[k];
        r.q_len = rows[k];
        r.tok0 = tok0[k];
        r.state = need[k] < 0 ? need[k] : q[k] < 0 ? 1 : 0;
        r.need0 = need0[k];
        r.back0 = back0[k];
        r.back = back[k];
        r.item0 = few[k] ? atomicAdd(&bucket[0][bucket_of(0, few_total[few0[k]], parts[k])], parts[k]) : 0;
        r.parts = parts[k];
        r.slot0 = v3[1];
        r.group = v3[2];
        v3[1] += parts[k] > 1 ? parts[k] : 0;
        v3[2] += parts[k] > 1;
        r.piece0 = piece0[k];
        r.pieces = pieces[k];
        r.write0 = write0[k];
        r.writes = writes[k];
        r.pad = 0;
        reqs[b] = r;
        if (A.first_row) {
            A.first_row[b] = tok0[k];
            if (b == A.batch - 1) A.first_row[A.batch] = t1[0] < A.tokens ? t1[0] : A.tokens;
        }
    }
    spd_plan_cut *cuts = (spd_plan_cut *)(A.plan + A.cuts);
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i >= n_many) break;
        spd_plan_cut c;
        c.parts = parts_many(i, many_chunk);
        c.item0 = atomicAdd(&bucket[1][bucket_of(1, many_total[i], c.parts)], c.parts);
        c.slot0 = m3[1];
        c.merge = m3[2];
        m3[1] += c.parts > 1 ? c.parts : 0;
        m3[2] += c.parts > 1;
        cuts[i] = c;
    }
    if (tid == 0) {
        H.n_small = n_small;
        H.n_large = tm[0];
        H.n_merge = tm[2];
        H.n_write = t4[2];
        H.rows = t1[0] < A.tokens ? t1[0] : A.tokens;
        H.free0 = free0;
        H.top = top;
        if (A.n_free_out) *A.n_free_out = top - t4[3];
    }
}

// The k-th of the pages that are handed out: from the top of the free ones, where those that came back lie.
__device__ __forceinline__ int new_page(const BuildArgs &A, const spd_plan_req *reqs, int free0, int top, int k) {
    const int at = top - 1 - k;
    if (at < free0) return A.free_pages[at];
    // (it is being put there by another workgroup: the last request with no more than so many before it has it)
    const int j = at - free0;
    int lo = 0, hi = A.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (reqs[mid].back0 <= j) lo = mid;
        else hi = mid;
    }
    return A.page_table[lo * A.ld_table + (j - reqs[lo].back0)];
}

constexpr int CHUNK_ROWS = 2048, CHUNK_PAGES = CHUNK_ROWS / 16 + 1;

// The second kernel: a workgroup per request and 2048 of its rows.
__global__ void __launch_bounds__(256) k_build_requests(BuildArgs A) {
    const spd_plan_header &H = *(const spd_plan_header *)A.plan;
    const int tid = threadIdx.x, chunk = blockIdx.y;
    auto no_row = [&](int row) {
        if (A.row_seq) A.row_seq[row] = -1;
        if (A.row_pos) A.row_pos[row] = -1;
        if (A.row_slot) A.row_slot[row] = -1;
    };
    if ((int)blockIdx.x >= A.batch) {            // rows behind the last request
        const int n = gridDim.y * A.tails;
        for (int row = H.rows + ((blockIdx.x - A.batch) * gridDim.y + chunk) * 256 + tid; row < A.tokens; row += n * 256) no_row(row);
        return;
    }
    const int b = blockIdx.x, free0 = H.free0, top = H.top;
    const spd_plan_req *reqs = (const spd_plan_req *)(A.plan + A.reqs);
    const spd_plan_req r = reqs[b];
    int32_t *row = A.page_table + b * A.ld_table;
    const bool first = chunk == 0;
    if (r.state == 1) {                          // its pages come back
        if (!first) return;
        for (int i = tid; i < r.back; i += 256)
            if (free0 + r.back0 + i < A.n_pages) A.free_pages[free0 + r.back0 + i] = row[i];
        if (tid == 0) {
            if (A.positions_out) A.positions_out[b] = 0;
            if (A.served) A.served[b] = 0;
            ((spd_plan_seq *)(A.plan + A.seqs))[b] = spd_plan_seq{0, 0, r.tok0, b * A.entries, 0, 0, 0};
        }
        return;
    }
    const int row0 = chunk * CHUNK_ROWS, rows = r.q_len - row0 < CHUNK_ROWS ? r.q_len - row0 : CHUNK_ROWS;      // of the chunk
    if (!first && rows <= 0) return;
    // the pages, as the plan has them; those of the chunk's rows are kept
    __shared__ int pages[CHUNK_PAGES];
    const int end = r.pos + r.q_len;
    bool bad = false;
    if (r.state == 0 && r.q_len > 0) {
        const int n = ceil_div(end, A.page_size), held = A.free_pages ? ceil_div(r.pos, A.page_size) : n, from = (r.pos + row0) / A.page_size;
        int32_t *table = (int32_t *)(A.plan + A.table) + (size_t)b * A.entries;
        for (int i = tid; i < n; i += 256) {
            const int page = i < held ? row[i] : new_page(A, reqs, free0, top, r.need0 + i - held);
            const bool none = (unsigned)page >= (unsigned)A.n_pages;
            bad |= none;
            if (first) {
                if (i >= held) row[i] = page;
                table[i] = none ? 0 : page;
            }
            if (i >= from && i - from < CHUNK_PAGES) pages[i - from] = page;
        }
    }
    bad = __syncthreads_or(bad);
    const bool served = r.state == 0 && !bad;
    if (A.row_seq || A.row_pos || A.row_slot)
        for (int i = tid; i < rows; i += 256) {
            const int at = r.tok0 + row0 + i, p = r.pos + row0 + i;
            if (at >= A.tokens) break;
            if (!served) {
                no_row(at);
                continue;
            }
            if (A.row_seq) A.row_seq[at] = b;
            if (A.row_pos) A.row_pos[at] = p;
            if (A.row_slot) A.row_slot[at] = (int64_t)pages[p / A.page_size - (r.pos + row0) / A.page_size] * A.page_size + p % A.page_size;
        }
    if (!first) return;
    if (tid == 0) {
        if (A.positions_out) A.positions_out[b] = served ? end : r.pos;
        if (A.served) A.served[b] = served ? r.q_len : r.state < 0 ? r.state : SPD_STEP_PAGE;
    }
    const spd_plan_seq s = {r.pos, served ? r.q_len : 0, r.tok0, b * A.entries, 0, served ? end : r.pos, 0};
    if (tid == 0) ((spd_plan_seq *)(A.plan + A.seqs))[b] = s;
    for (int i = tid; i < r.writes; i += 256)
        ((spd_plan_block *)(A.plan + A.write))[r.write0 + i] = spd_plan_block{s, served ? r.pos / 16 + i : -1, {0, 0, 0}};
    auto item = [&](spd_plan_item *to, const spd_piece &w, int first_row, int unit, int parts, int i, int slot0, int group) {
        spd_plan_item it;
        it.s = s;
        it.row0 = first_row;
        it.sink_blocks = w.sink_blocks;
        it.block0 = w.block0;
        it.first = spd_item_first(w.total, unit, parts, i);
        it.count = served ? spd_item_count(w.total, unit, parts, i) : 0;
        it.slot = parts > 1 ? slot0 + i : -1;
        it.slot0 = slot0;
        it.parts = parts;
        it.group = group;
        it.pad[0] = it.pad[1] = it.pad[2] = 0;
        *to = it;
    };
    const int n = r.q_len * A.group;
    if (r.parts) {
        const spd_piece w = spd_piece_of(A.group, r.pos, 0, n, A.window, A.sinks);
        for (int i = tid; i < r.parts; i += 256) item((spd_plan_item *)(A.plan + A.small) + r.item0 + i, w, 0, 2, r.parts, i, r.slot0, r.group);
    }
    for (int k = tid; k < r.pieces; k += 256) {
        const spd_plan_cut c = ((const spd_plan_cut *)(A.plan + A.cuts))[r.piece0 + k];
        const int first_row = k * SPD_LARGE_ROWS, left = n - first_row, mine = left < SPD_LARGE_ROWS ? left : SPD_LARGE_ROWS;
        const spd_piece w = spd_piece_of(A.group, r.pos, first_row, mine, A.window, A.sinks);
        for (int i = 0; i < c.parts; ++i) item((spd_plan_item *)(A.plan + A.large) + c.item0 + i, w, first_row, 4, c.parts, i, c.slot0, c.merge);
        if (c.parts > 1) ((spd_plan_merge *)(A.plan + A.merge))[c.merge] = spd_plan_merge{s, first_row, served ? mine : 0, c.slot0, c.parts};
    }
}

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

extern "C" int spd_pages_build(const spd_pages *pages, const void *plan_host, void *plan_dev, const spd_pages_step *step, void *stream) {
    if (!pages || !plan_host || !step || !plan_dev || !aligned(plan_dev, 16)) return SPD_EINVAL;
    spd_plan_header h;
    std::memcpy(&h, plan_host, sizeof(h));
    if (h.magic != SPD_PLAN_MAGIC || std::memcmp(&h.cfg, &pages->cfg, sizeof(h.cfg)) || !h.on_device) return SPD_EINVAL;
    const spd_pages_step &t = *step;
    const spd_pages_config &c = pages->cfg;
    if (!t.positions || !t.q_lens || !t.page_table || t.ld_table < h.entries) return SPD_EINVAL;
    if (!t.free_pages != !t.n_free || !t.free_pages != !t.n_free_out) return SPD_EINVAL;
    // what is read and written, each apart from the others but for what may be brought up to date in place
    const struct {
        const void *at;
        int64_t rows, width, pitch;
        int size;
    } all[] = {{t.positions, 1, 4ll * h.batch, 0, 4}, {t.q_lens, 1, 4ll * h.batch, 0, 4}, {t.n_free, 1, 4, 0, 4},
               {t.page_table, h.batch, 4ll * h.entries, 4 * t.ld_table, 4}, {t.free_pages, 1, 4ll * c.n_pages, 0, 4}, {t.n_free_out, 1, 4, 0, 4},
               {t.positions_out, 1, 4ll * h.batch, 0, 4}, {t.served, 1, 4ll * h.batch, 0, 4}, {t.first_row, 1, 4ll * h.batch + 4, 0, 4},
               {t.row_seq, 1, 4ll * h.tokens, 0, 4}, {t.row_pos, 1, 4ll * h.tokens, 0, 4}, {t.row_slot, 1, 8ll * h.tokens, 0, 8},
               {plan_dev, 1, (int64_t)h.device_bytes, 0, 16}};
    constexpr int N = sizeof(all) / sizeof(all[0]), READ = 3;      // (the first three are only read)
    for (int i = 0; i < N; ++i) {
        if (!aligned(all[i].at, all[i].size)) return SPD_EINVAL;
        for (int j = i + 1 > READ ? i + 1 : READ; j < N; ++j) {
            if (all[i].at == all[j].at && ((i == 0 && all[j].at == t.positions_out && j == 6) || (i == 2 && j == 5))) continue;
            const int64_t pi = all[i].pitch ? all[i].pitch : all[i].width, pj = all[j].pitch ? all[j].pitch : all[j].width;
            if (spd_share_memory({all[i].at, all[i].rows, all[i].width, pi}, {all[j].at, all[j].rows, all[j].width, pj})) return SPD_EINVAL;
        }
    }
    (void)hipGetLastError();
    BuildArgs A;
    A.positions = t.positions;
    A.q_lens = t.q_lens;
    A.n_free = t.n_free;
    A.page_table = t.page_table;
    A.free_pages = t.free_pages;
    A.n_free_out = t.n_free_out;
    A.positions_out = t.positions_out;
    A.served = t.served;
    A.first_row = t.first_row;
    A.row_seq = t.row_seq;
    A.row_pos = t.row_pos;
    A.row_slot = t.row_slot;
    A.plan = (char *)plan_dev;
    A.ld_table = t.ld_table;
    A.batch = h.batch;
    A.tokens = h.tokens;
    A.q_len = h.q_len;
    A.entries = h.entries;
    A.window = h.window;
    A.sinks = h.sinks;
    A.page_size = c.page_size;
    A.n_pages = c.n_pages;
    A.kv = c.n_kv_heads;
    A.group = pages->group;
    A.most_end = (int)std::min<int64_t>(c.max_ctx, (int64_t)h.entries * c.page_size);
    A.seqs = h.seqs;
    A.reqs = h.reqs;
    A.cuts = h.cuts;
    A.small = h.small;
    A.large = h.large;
    A.merge = h.merge;
    A.write = h.write;
    A.table = h.table;
    const bool by_row = t.row_seq || t.row_pos || t.row_slot;
    A.tails = by_row ? std::min(64, (h.tokens + 255) / 256) : 0;
    hipStream_t s = (hipStream_t)stream;
    if (h.batch <= THREADS) hipLaunchKernelGGL((k_build_sums<1>), dim3(1), dim3(THREADS), 0, s, A);
    else if (h.batch <= 2 * THREADS) hipLaunchKernelGGL((k_build_sums<2>), dim3(1), dim3(THREADS), 0, s, A);
    else hipLaunchKernelGGL((k_build_sums<4>), dim3(1), dim3(THREADS), 0, s, A);
    SPD_HIP(hipGetLastError());
    hipLaunchKernelGGL(k_build_requests, dim3(h.batch + A.tails, by_row ? (h.q_len + CHUNK_ROWS - 1) / CHUNK_ROWS : 1), dim3(256), 0, s, A);
    SPD_HIP(hipGetLastError());
    return SPD_OK;
}
