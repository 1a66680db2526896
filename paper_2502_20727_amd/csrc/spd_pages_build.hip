// The plan of a step made on the device, from request lengths that are there: pages taken from the free list and given back, the page table's new
// entries, rows and slots of the new tokens, and the work of spd_pages_write() and spd_pages_attention() in the form that the host's plan has it.
//
// Two kernels.  The first, a single workgroup, adds up: everything that one request has to know of the others is a prefix sum over them (rows, pages
// needed, pages that come back, blocks written, items), and the chunk that work is cut into is a search over sums, as on the host
// (spd_pages.h).  The second has a workgroup per request, checks its pages and writes what is the request's.  A request whose pages are not of
// the pool is found out there and leaves its items empty.  (A single request of few rows takes both in one launch.)
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
    unsigned by_group;                                     // 2^32 / group, rounded up
    int cache_dtype, page_size, page_shift, n_pages, kv, group, most_end;      // most_end: positions a request may have
    int seqs, reqs, cuts, backs, order, small, large, merge, write, table;      // byte offsets
    int tails;                                             // workgroups of the second kernel for rows behind the last request
};

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 1024, WAVES = THREADS / 64;      // of the first kernel, at most

__device__ __forceinline__ int ceil_div(int a, int b) { return (int)((unsigned)(a + b - 1) / (unsigned)b); }

// a row's token: rows are below 2^28 and by_group is 2^32 / group rounded up, so that this divides by the group, 16 at most
__device__ __forceinline__ int token_of(const BuildArgs &A, int row) { return A.group == 1 ? row : (int)__umulhi(row, A.by_group); }

// Sums stop at 2^30: what goes beyond any limit does not come round to within it.
__device__ __forceinline__ unsigned add(unsigned a, unsigned b) {
    const unsigned c = a + b;
    return c < 1u << 30 ? c : 1u << 30;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned shifted(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false); }
// inclusive prefix sums over rows of 16 lanes, over the wave
__device__ __forceinline__ unsigned row_sums(unsigned x) {
    x = add(x, shifted<0x111, 0xf>(x));
    x = add(x, shifted<0x112, 0xf>(x));
    x = add(x, shifted<0x114, 0xf>(x));
    return add(x, shifted<0x118, 0xf>(x));
}
__device__ __forceinline__ unsigned wave_sums(unsigned x) {
    x = row_sums(x);
    x = add(x, shifted<0x142, 0xa>(x));          // the last lane of rows 0 and 2 into rows 1 and 3
    return add(x, shifted<0x143, 0xc>(x));       // ... of the lower half into the upper
}
__device__ __forceinline__ unsigned last_lane(unsigned x) { return (unsigned)__builtin_amdgcn_readlane((int)x, 63); }

// Exclusive prefix sums over the workgroup of N numbers a thread, and their totals.  `lds`: WAVES * N, which nobody reads any more.
template <int N>
__device__ __forceinline__ void scan(unsigned (&v)[N], unsigned (&total)[N], unsigned *lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    unsigned mine[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const unsigned x = wave_sums(v[n]);
        mine[n] = x - v[n];
        if (lane == 63) lds[wave * N + n] = x;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const unsigned x = row_sums(lane < waves ? lds[lane * N + n] : 0);
        const unsigned before = wave ? (unsigned)__builtin_amdgcn_readlane((int)x, wave - 1) : 0;
        total[n] = (unsigned)__builtin_amdgcn_readlane((int)x, 15);
        v[n] = add(before, mine[n]);
    }
}

// n / d rounded up, less one, of whole numbers in floats, `inverse` = 1 / d rounded to the nearest.  (n - 0.5) / d is 0.5 / d from a whole number at least, and the
// result less than n / d * 2^-23 off: exact for n up to 2^22, which is the blocks of the longest sequence.
__device__ __forceinline__ float times_less_one(float n, float inverse) { return floorf(fmaf(n, inverse, -0.5f * inverse)); }

// The first kernel.  PER requests a thread, one after the other.  Bound by how long one thing waits for another: loads, about six
// sums over the workgroup, barriers, and the fetching of its own instructions, which is why little of it is unrolled or divides in 64 bits.  us, one
// request / 256 with four chunks of prompts / 2048 with 64: 4.8 / 13.8 / 25.3, both launches 11.4 / 19.5 / 34.0 (chunks tried one after the other by the whole workgroup, dividing in 64
// bits: 32.0 / 57.1 / 119.8).
struct Sums {
    int rows, free0, top, n_backs, sorted;      // as in the header
};
template <int PER>
__device__ __forceinline__ Sums build_sums(const BuildArgs &A) {
    __shared__ unsigned lds[3][WAVES * 8];
    __shared__ int many_pos[PER * THREADS], many_rows[PER * THREADS], many_first[PER * THREADS];      // requests of many rows: position, rows, first piece
    // Of the pieces of few rows, of many: blocks; the most items that each may be cut into, later those that it is, less one.  Whole numbers in floats, which
    // divide faster.
    __shared__ float2 few_pieces[PER * THREADS], many_pieces[SPD_BUILD_PIECES];
    __shared__ unsigned long long sums[2];                 // blocks of the pieces of few rows, of many
    // few rows; many, for 2, 3 and 4 halves: the chunks that are tried, and does one make few enough items?
    __shared__ int chunks[4][SPD_LONGER], fits[4][SPD_LONGER];
    __shared__ int counts[3][3];                           // items, those that are parts, blocks of the longest, as many rows might be cut
    __shared__ int buckets[2][256];
    __shared__ unsigned took;                              // pages, where there are not enough
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    spd_plan_header &H = *(spd_plan_header *)A.plan;
    const int free_now = A.n_free ? *A.n_free : 0, free0 = free_now < 0 ? 0 : free_now > A.n_pages ? A.n_pages : free_now;
    int pos[PER], q[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int b = tid * PER + k;
        pos[k] = b < A.batch ? A.positions[b] : 0;
        q[k] = b < A.batch ? A.q_lens[b] : 0;
    }
    if (tid < 2) sums[tid] = took = 0;
    if (tid < 9) counts[tid / 3][tid % 3] = 0;
    if (tid < 64) fits[tid / SPD_LONGER][tid % SPD_LONGER] = 0;
    for (int i = tid; i < 512; i += blockDim.x) buckets[i >> 8][i & 255] = 0;
    bool fine[PER], got[PER], stuck[PER];                  // its lengths are within the limits; there are pages for it; it has a page that is none, and new ones already
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        fine[k] = pos[k] >= 0 && q[k] >= SPD_STEP_RELEASE && q[k] <= A.q_len && pos[k] <= A.most_end - (q[k] > 0 ? q[k] : 0);
        stuck[k] = false;
    }
    auto rows_of = [&](int k) { return q[k] > 0 && q[k] <= A.q_len ? q[k] : 0; };
    auto held_of = [&](int k) { return (pos[k] + A.page_size - 1) >> A.page_shift; };
    auto back_of = [&](int k) { return A.free_pages && fine[k] && q[k] < 0 ? held_of(k) : 0; };
    auto need_of = [&](int k) { return A.free_pages && fine[k] && !stuck[k] && q[k] > 0 ? ((pos[k] + q[k] + A.page_size - 1) >> A.page_shift) - held_of(k) : 0; };
    auto few_of = [&](int k) { return got[k] && q[k] > 0 && q[k] * A.group <= SPD_SMALL_ROWS; };
    auto pieces_of = [&](int k) { return got[k] && q[k] > 0 && q[k] * A.group > SPD_SMALL_ROWS ? (q[k] * A.group + SPD_LARGE_ROWS - 1) / SPD_LARGE_ROWS : 0; };
    auto writes_of = [&](int k) { return got[k] && q[k] > 0 ? (pos[k] + q[k] - 1) / 16 - pos[k] / 16 + 1 : 0; };
    // A request that has a page that is none is refused by the second kernel, when new pages are in its row already.  Its positions stay, so that the next step would hand
    // it others and the first would be nobody's: where a page lies in the first new place it is refused here and takes none.  Each wave looks by itself, through the entries of
    // those of its requests that want pages (in most steps few do), sixteen lanes a request: of 1 / 64 / 256 / 2048 requests 0 / 0.7 / 1.7 / 2.7 us a plan.
    {
        auto a_page = [&](int page) { return (unsigned)page < (unsigned)A.n_pages; };
        int *mine = many_first + wave * 64 * PER, *held = many_rows + wave * 64 * PER, *found = many_pos + wave * 64 * PER;      // request, its entries, is it so?
        int n = 0, at[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const bool asks = need_of(k) && held_of(k);
            const unsigned long long who = __builtin_amdgcn_ballot_w64(asks);
            at[k] = asks ? n + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0)) : -1;
            if (asks) {
                mine[at[k]] = tid * PER + k;
                held[at[k]] = held_of(k);
                found[at[k]] = 0;
            }
            n += __builtin_popcountll(who);
        }
        if (n) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int i = lane >> 4; i < n; i += 4) {
                const int32_t *row = A.page_table + mine[i] * A.ld_table;
                const int h = held[i], next = row[h];
                bool bad = false;
                constexpr int N = 16;            // asked for at a time (those behind the last are the last)
#pragma unroll 1
                for (int e = lane & 15; e < h; e += 16 * N) {
                    int page[N];
#pragma unroll
                    for (int u = 0; u < N; ++u) page[u] = row[e + 16 * u < h ? e + 16 * u : h - 1];
#pragma unroll
                    for (int u = 0; u < N; ++u) bad |= !a_page(page[u]);
                }
                if (bad && a_page(next)) found[i] = 1;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (at[k] >= 0) stuck[k] = found[at[k]];
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) got[k] = fine[k] && !stuck[k];
    // Rows, pages that come back, those of whom; pages needed; pieces of few rows, of many, blocks written; requests of many rows.  Who has no rows or no pages left is found by
    // sums of those before it, after which there are new ones to be taken: in most steps nobody is.
    unsigned v[8], t[8];
    int top;
    bool short_of_rows = false, short_of_pages = false;
    for (int turn = 0;; ++turn) {
#pragma unroll
        for (int n = 0; n < 8; ++n) v[n] = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            v[0] += rows_of(k);
            v[1] += back_of(k);
            v[2] += back_of(k) > 0;
            v[3] += need_of(k);
            v[4] += few_of(k);
            v[5] += pieces_of(k);
            v[6] += writes_of(k);
            v[7] += pieces_of(k) > 0;
        }
        scan(v, t, lds[turn]);
        top = (int)t[1] < A.n_pages - free0 ? free0 + (int)t[1] : A.n_pages;
        if (!short_of_rows && (int)t[0] > A.tokens) {
            short_of_rows = true;
            unsigned r = v[0];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                r = add(r, rows_of(k));
                if ((int)r > A.tokens) fine[k] = got[k] = false;
            }
        } else if (!short_of_pages && (int)t[3] > top) {
            short_of_pages = short_of_rows = true;
            unsigned n = v[3];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                n = add(n, need_of(k));
                if (need_of(k) && (int)n > top) got[k] = false;
            }
        } else break;
    }
    const int n_few = t[4], n_many = t[5], n_long = t[7];
    spd_plan_req *reqs = (spd_plan_req *)(A.plan + A.reqs);
    // what is known of each so far is put away, and the pieces are measured
    int few0 = v[4];
    unsigned taken = 0;
    {
        unsigned row = v[0], back = v[1], backs = v[2], need = v[3];
        int few = few0, piece = v[5], write = v[6], many = v[7];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int b = tid * PER + k, tok0 = (int)row < A.tokens ? (int)row : A.tokens;
            if (b < A.batch) {
                spd_plan_req &r = reqs[b];
                *(i32x4 *)&r.pos = (i32x4){pos[k], rows_of(k), tok0, !fine[k] ? SPD_STEP_LENGTHS : stuck[k] ? SPD_STEP_PAGE : !got[k] ? SPD_STEP_NO_PAGES : q[k] < 0 ? 1 : 0};
                *(i32x4 *)&r.need0 = (i32x4){(int)need, (int)back, back_of(k), few};
                *(i32x4 *)&r.piece0 = (i32x4){piece, pieces_of(k), write, writes_of(k)};
                if (back_of(k)) ((spd_plan_back *)(A.plan + A.backs))[backs] = spd_plan_back{(int)back, b};
                if (A.first_row) A.first_row[b] = tok0;
            }
            if (few_of(k)) few_pieces[few].x = (float)spd_piece_between(pos[k], pos[k] + q[k] - 1, A.window, A.sinks).total;
            if (pieces_of(k)) {
                many_pos[many] = pos[k];
                many_rows[many] = q[k] * A.group;
                many_first[many++] = piece;
            }
            row = add(row, rows_of(k));
            back += back_of(k);
            backs += back_of(k) > 0;
            need = add(need, need_of(k));
            taken += got[k] ? need_of(k) : 0;
            few += few_of(k);
            piece += pieces_of(k);
            write += writes_of(k);
        }
    }
    __syncthreads();
    const int sets = spd_sets(A.group);
#pragma unroll 1
    for (int i = tid; i - lane < n_few; i += blockDim.x) {
        const int total = i < n_few ? (int)few_pieces[i].x : 0;
        const unsigned all = last_lane(wave_sums(total));  // (64 * 2^22 at most)
        if (lane == 0) atomicAdd(&sums[0], (unsigned long long)all);
        if (i < n_few) few_pieces[i].y = (float)(spd_most_small(total, sets) - 1);
    }
#pragma unroll 1
    for (int i = tid; i - lane < n_many; i += blockDim.x) {
        int total = 0;
        if (i < n_many) {
            int lo = 0, hi = n_long;                       // its request: the last that begins no later
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2, first = many_first[mid];
                lo = first <= i ? mid : lo;
                hi = first <= i ? hi : mid;
            }
            const int row0 = (i - many_first[lo]) * SPD_LARGE_ROWS, left = many_rows[lo] - row0, row1 = row0 + (left < SPD_LARGE_ROWS ? left : SPD_LARGE_ROWS) - 1;
            auto token = [&](int row) { return token_of(A, row); };
            total = spd_piece_between(many_pos[lo] + token(row0), many_pos[lo] + token(row1), A.window, A.sinks).total;
            many_pieces[i] = make_float2((float)total, (float)(spd_most_large(total) - 1));
        }
        const unsigned all = last_lane(wave_sums(total));
        if (lane == 0) atomicAdd(&sums[1], (unsigned long long)all);
    }
    __syncthreads();
    // The chunks: of those tried the first that makes few enough items.  Each wave tries one, of few rows or of many for one of three numbers of workgroups, and
    // others after it if that is too short.
    const bool cut_few = n_few && (int64_t)n_few * A.kv <= SPD_COUNTERS;
    {
        const int which = n_many ? wave & 3 : 0, c0 = n_many ? wave >> 2 : wave, step = n_many ? WAVES / 4 : waves;
        const int n = which ? n_many : n_few, unit = which ? 4 : 2;
        const int target = which == 0 ? spd_small_target(A.cache_dtype, (int64_t)n_few * A.kv) : SPD_COMPUTE_UNITS / 2 * (which + 1);
        const float2 *pieces = which ? many_pieces : few_pieces;
        if (which || cut_few) {
            // spd_first_chunk(), in 32 bits: no piece has more than 2^22 blocks, and 2^29 does for all that is more
            static_assert(SPD_SMALL_TARGET == 256 && SPD_COMPUTE_UNITS == 256, "targets are 128 times 2, 3 or 4");
            const unsigned long long share = (sums[which ? 1 : 0] * A.kv + 127) >> 7;
            const unsigned y = share < 1u << 31 ? (unsigned)share : 1u << 31;
            const unsigned first = ((target == 384 ? (y + 2) / 3 : target == 512 ? (y + 3) / 4 : (y + 1) / 2) + unit - 1) & -unit;
            int chunk = first < (unsigned)unit ? unit : first < 1u << 29 ? (int)first : 1 << 29;
            auto next = [&]() {                            // spd_next_chunk(): units are powers of two
                chunk = (chunk + chunk / 16 + unit) & -unit;
                chunk = chunk < 1 << 29 ? chunk : 1 << 29;
            };
            auto skip = [&](int times) {
#pragma unroll 1
                for (int i = 0; i < times; ++i) next();
            };
            skip(c0);
#pragma unroll 1
            for (int c = c0; c < SPD_LONGER; c += step, skip(step)) {
                const float inverse = 1.f / (float)chunk;
                float more = 0.f;                          // items beyond one for each piece
#pragma unroll 4
                for (int i = lane; i < n; i += 64) more += fminf(times_less_one(pieces[i].x, inverse), pieces[i].y);
                const unsigned items = n + last_lane(wave_sums((unsigned)more));
                const bool fit = (int64_t)items * A.kv <= target || (int)items == n;
                if (lane == 0) {
                    fits[which][c] = fit;
                    chunks[which][c] = chunk;
                }
                if (fit) break;                            // (a wave's later ones are not asked for)
            }
        }
    }
    __syncthreads();
    auto chosen = [&](int which) {                         // 1 / the chunk
        const unsigned long long fit = __builtin_amdgcn_ballot_w64(lane < SPD_LONGER && fits[which][lane < SPD_LONGER ? lane : 0]);
        int chunk = chunks[which][fit ? __builtin_ctzll(fit) : SPD_LONGER - 1];
        const int unit = which ? 4 : 2;
        if (!fit) chunk = (chunk + chunk / 16 + unit) & -unit;
        return 1.f / (float)chunk;
    };
    int halves = 0;
    // items of a piece, less one: no more than whole units
    auto parts_less_one = [&](float2 p, float inverse, float by_unit) { return fminf(fminf(times_less_one(p.x, inverse), p.y), times_less_one(p.x, by_unit)); };
    if (n_many) {
        // (where there are many rows there are sixteen waves: five for each number of halves)
        if (wave < 15) {
            const int h = wave % 3;
            const float inverse = chosen(h + 1);
            unsigned items = 0, slots = 0;
            int most = 0;
#pragma unroll 1
            for (int i = wave / 3 * 64 + lane; i < n_many; i += 5 * 64) {
                const float2 p = many_pieces[i];
                const int total = (int)p.x, parts = (int)parts_less_one(p, inverse, 0.25f) + 1, units = (total + 3) / 4;
                items += parts;
                slots += parts > 1 ? parts : 0;
                // The longest of its items has units / parts of them, rounded up: the last, which the last unit may leave shorter, and an earlier one if
                // as many as two have one more than the others (or none has)
                const int each = (int)times_less_one((float)units, 1.f / (float)parts) + 1, c = each * 4, more = units - (each - 1) * parts;
                const int last = total - (units - each) * 4;
                const int longest_here = (more == 1 || parts == 1) ? (last > c - 4 ? last : c - 4) : c;
                most = longest_here > most ? longest_here : most;
            }
            items = last_lane(wave_sums(items));
            slots = last_lane(wave_sums(slots));
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int y = __shfl_xor(most, d, 64);
                most = y > most ? y : most;
            }
            if (lane == 0) {
                atomicAdd(&counts[h][0], (int)items);
                atomicAdd(&counts[h][1], (int)slots);
                atomicMax(&counts[h][2], most);
            }
        }
        __syncthreads();
        const int h = lane < 3 ? lane : 0;
        const long long ns = spd_estimate_large(counts[h][2], counts[h][0], counts[h][1], A.kv), ns0 = __shfl(ns, 0), ns1 = __shfl(ns, 1), ns2 = __shfl(ns, 2);
        halves = ns1 < ns0 ? ns2 < ns1 ? 2 : 1 : ns2 < ns0 ? 2 : 0;
    }
    {
        const float few_inverse = cut_few ? chosen(0) : 0.f, many_inverse = n_many ? chosen(halves + 1) : 0.f;      // (few rows: uncut where there are not enough counters)
#pragma unroll 1
        for (int i = tid; i < n_few; i += blockDim.x) few_pieces[i].y = cut_few ? parts_less_one(few_pieces[i], few_inverse, 0.5f) : 0.f;
#pragma unroll 1
        for (int i = tid; i < n_many; i += blockDim.x) many_pieces[i].y = parts_less_one(many_pieces[i], many_inverse, 0.25f);
        __syncthreads();
    }
    // Items, those of a piece one after the other.  Where a compute unit has more than one, the pieces with the longest items come first, by lengths that are 1/16 of
    // a power of two apart; which of one length is first is left to chance: it is the order they are started in, and nothing else.  In order / as they come, us a
    // call of attention: 64 sequences of up to 8000 on 8 heads 68.8 / 78.8, 200 on one head 32.1 / 33.3, 600 of up to 4000 43.7 / 50.9, 6 chunks of 700 tokens on 8 heads
    // 278 / 297; 48 of up to 16000 on one head 20.3 / 20.4.
    auto place = [&](int *bucket, int n_pieces, const float2 *pieces, int *to, int step) {
        auto bucket_of = [&](int i) {
            const int n = (__float_as_int(pieces[i].x * __builtin_amdgcn_rcpf(pieces[i].y + 1.f)) >> 19) - (127 << 4);      // of its items' blocks, about
            return 255 - (n < 0 ? 0 : n < 255 ? n : 255);
        };
#pragma unroll 1
        for (int i = tid; i < n_pieces; i += blockDim.x) atomicAdd(&bucket[bucket_of(i)], (int)pieces[i].y + 1);
        __syncthreads();
        if (wave == 0) {
            unsigned x[4], all = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) all += x[i] = bucket[lane * 4 + i];
            unsigned sum = wave_sums(all) - all;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bucket[lane * 4 + i] = sum;
                sum += x[i];
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < n_pieces; i += blockDim.x) to[i * step] = atomicAdd(&bucket[bucket_of(i)], (int)pieces[i].y + 1);
        __syncthreads();
    };
    int n_small, n_large = 0, n_merge = 0;
    {
        unsigned s[3] = {0, 0, 0}, all[3];
        int few = few0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int parts = few_of(k) ? (int)few_pieces[few].y + 1 : 0;
            few += few_of(k);
            s[0] += parts;
            s[1] += parts > 1 ? parts : 0;
            s[2] += parts > 1;
        }
        scan(s, all, lds[1]);
        n_small = all[0];
        few = few0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int b = tid * PER + k, parts = few_of(k) ? (int)few_pieces[few].y + 1 : 0;
            if (b < A.batch) *(i32x4 *)&reqs[b].item0 = (i32x4){(int)s[0], parts, (int)s[1], (int)s[2]};
            few += few_of(k);
            s[0] += parts;
            s[1] += parts > 1 ? parts : 0;
            s[2] += parts > 1;
        }
    }
    const bool sorted = n_small * A.kv > SPD_COMPUTE_UNITS;      // (few rows: the first items are then those in `order`)
    if (sorted) place(buckets[0], n_few, few_pieces, (int *)(A.plan + A.order), 1);
    if (n_many) {
        spd_plan_cut *cuts = (spd_plan_cut *)(A.plan + A.cuts);
        const int per = ceil_div(n_many, blockDim.x);
        unsigned s[3] = {0, 0, 0}, all[3];
#pragma unroll 1
        for (int i = tid * per; i < n_many && i < (tid + 1) * per; ++i) {
            const int n = (int)many_pieces[i].y + 1;
            s[0] += n;
            s[1] += n > 1 ? n : 0;
            s[2] += n > 1;
        }
        scan(s, all, lds[2]);
#pragma unroll 1
        for (int i = tid * per; i < n_many && i < (tid + 1) * per; ++i) {
            const int n = (int)many_pieces[i].y + 1;
            *(i32x4 *)&cuts[i] = (i32x4){(int)s[0], n, (int)s[1], (int)s[2]};
            s[0] += n;
            s[1] += n > 1 ? n : 0;
            s[2] += n > 1;
        }
        n_large = all[0];
        n_merge = all[2];
        __syncthreads();
        if (n_large * A.kv > SPD_COMPUTE_UNITS) place(buckets[1], n_many, many_pieces, &cuts[0].item0, sizeof(spd_plan_cut) / 4);
    }
    if (short_of_pages) {
        __syncthreads();
        taken = last_lane(wave_sums(taken));
        if (lane == 0) atomicAdd(&took, taken);
        __syncthreads();
    }
    const Sums now = {(int)t[0] < A.tokens ? (int)t[0] : A.tokens, free0, top, (int)t[2], sorted};
    if (tid == 0) {
        H.n_small = n_small;
        H.n_large = n_large;
        H.n_merge = n_merge;
        H.n_write = t[6];
        H.rows = now.rows;
        H.free0 = free0;
        H.top = top;
        H.n_backs = now.n_backs;
        H.sorted = sorted;
        if (A.n_free_out) *A.n_free_out = top - (int)(short_of_pages ? took : t[3]);
        if (A.first_row) A.first_row[A.batch] = now.rows;
    }
    return now;
}
template <int PER>
__global__ void __launch_bounds__(THREADS) k_build_sums(BuildArgs A) { build_sums<PER>(A); }

constexpr int CHUNK_ROWS = 2048, CHUNK_PAGES = CHUNK_ROWS / 16 + 1;

// rows behind the last request: the i-th of n workgroups
__device__ __forceinline__ void no_row(const BuildArgs &A, int row) {
    if (A.row_seq) A.row_seq[row] = -1;
    if (A.row_pos) A.row_pos[row] = -1;
    if (A.row_slot) A.row_slot[row] = -1;
}
__device__ __forceinline__ void build_tail(const BuildArgs &A, int rows, int i, int n) {
    for (int row = rows + i * 256 + threadIdx.x; row < A.tokens; row += n * 256) no_row(A, row);
}

// A request and 2048 of its rows, by 256 threads.
__device__ __forceinline__ void build_request(const BuildArgs &A, const Sums &H, int b, int chunk) {
    const int tid = threadIdx.x, free0 = H.free0, top = H.top;
    const spd_plan_req *reqs = (const spd_plan_req *)(A.plan + A.reqs);
    const spd_plan_back *backs = (const spd_plan_back *)(A.plan + A.backs);
    int32_t *row = A.page_table + b * A.ld_table;
    // (what a thread will most likely want is asked for before it is known that it does: one wait for memory instead of three)
    constexpr int EARLY = 4;
    int early[EARLY];
#pragma unroll
    for (int k = 0; k < EARLY; ++k) early[k] = tid + 256 * k < A.entries ? row[tid + 256 * k] : 0;
    const int early_back = tid < A.batch ? backs[tid].back0 : 0;
    const spd_plan_req r = reqs[b];
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
        // New pages come from the top of the free ones, where those that came back lie (put there by other workgroups, at this moment: they are taken
        // from their requests' rows of the table).  `giver`: the last of these that has the first of them, the next are its or the ones' before it.
        const int top_new = top - 1 - r.need0;
        int giver = 0;
        if (n > held && top_new >= free0) {
            giver = __syncthreads_count(tid < H.n_backs && early_back <= top_new - free0) - 1;
            for (int i = tid + 256; i - tid < H.n_backs; i += 256) giver += __syncthreads_count(i < H.n_backs && backs[i].back0 <= top_new - free0);
        }
        auto new_page = [&](int k) {
            const int j = top_new - k - free0;
            if (j < 0) return A.free_pages[top_new - k];
            int g = giver;
            while (backs[g].back0 > j) --g;
            return A.page_table[backs[g].req * A.ld_table + (j - backs[g].back0)];
        };
        auto enter = [&](int i, int page) {
            const bool none = (unsigned)page >= (unsigned)A.n_pages;
            bad |= none;
            if (first) {
                if (i >= held) row[i] = page;
                table[i] = none ? 0 : page;
            }
            if (i >= from && i - from < CHUNK_PAGES) pages[i - from] = page;
        };
#pragma unroll
        for (int k = 0; k < EARLY; ++k)
            if (tid + 256 * k < n) enter(tid + 256 * k, tid + 256 * k < held ? early[k] : new_page(tid + 256 * k - held));
        for (int i = tid + 256 * EARLY; i < n; i += 256) enter(i, i < held ? row[i] : new_page(i - held));
    }
    bad = __syncthreads_or(bad);
    const bool served = r.state == 0 && !bad;
    if (A.row_seq || A.row_pos || A.row_slot)
        for (int i = tid; i < rows; i += 256) {
            const int at = r.tok0 + row0 + i, p = r.pos + row0 + i;
            if (at >= A.tokens) break;
            if (!served) {
                no_row(A, at);
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
        const spd_piece w = spd_piece_between(r.pos, end - 1, A.window, A.sinks);
        const int item0 = H.sorted ? ((const int *)(A.plan + A.order))[r.few] : r.item0;
        for (int i = tid; i < r.parts; i += 256) item((spd_plan_item *)(A.plan + A.small) + item0 + i, w, 0, 2, r.parts, i, r.slot0, r.group);
    }
    for (int k = tid >> 3; k < r.pieces; k += 32) {        // eight threads a piece
        const spd_plan_cut c = ((const spd_plan_cut *)(A.plan + A.cuts))[r.piece0 + k];
        const int first_row = k * SPD_LARGE_ROWS, left = n - first_row, mine = left < SPD_LARGE_ROWS ? left : SPD_LARGE_ROWS;
        const spd_piece w = spd_piece_between(r.pos + token_of(A, first_row), r.pos + token_of(A, first_row + mine - 1), A.window, A.sinks);
        for (int i = tid & 7; i < c.parts; i += 8) item((spd_plan_item *)(A.plan + A.large) + c.item0 + i, w, first_row, 4, c.parts, i, c.slot0, c.merge);
        if (c.parts > 1 && (tid & 7) == 0) ((spd_plan_merge *)(A.plan + A.merge))[c.merge] = spd_plan_merge{s, first_row, served ? mine : 0, c.slot0, c.parts};
    }
}

// The second kernel: a workgroup per request and 2048 of its rows, and some for the rows behind.  Three loads that wait for each other (request, page, the rows of those
// whose pages came back): us, one request / 256 / 2048 of up to 2000 positions 3.7 / 5.7 / 8.9.
__global__ void __launch_bounds__(256) k_build_requests(BuildArgs A) {
    const spd_plan_header &h = *(const spd_plan_header *)A.plan;
    const Sums H = {h.rows, h.free0, h.top, h.n_backs, h.sorted};
    if ((int)blockIdx.x < A.batch) return build_request(A, H, blockIdx.x, blockIdx.y);
    build_tail(A, H.rows, (blockIdx.x - A.batch) * gridDim.y + blockIdx.y, gridDim.y * A.tails);
}

// Both for a single request of few rows (interactive decoding): a launch less, whose enqueuing is what a call outside of a graph waits for.  us a call, this / two
// kernels: 9.0 / 11.4, in a graph 7.6 / 8.1; a second request would have to wait for the first: 10.6 / 11.0, 10.6 / 8.6.
__global__ void __launch_bounds__(256) k_build_one(BuildArgs A) {
    const Sums H = build_sums<1>(A);
    __syncthreads();
    build_request(A, H, 0, 0);
    if (A.tails) build_tail(A, H.rows, 0, 1);
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
    A.cache_dtype = c.cache_dtype;
    A.page_size = c.page_size;
    A.page_shift = pages->shift + 4;
    A.n_pages = c.n_pages;
    A.kv = c.n_kv_heads;
    A.group = pages->group;
    A.by_group = (unsigned)(((1ull << 32) + pages->group - 1) / pages->group);
    A.most_end = (int)std::min<int64_t>(c.max_ctx, (int64_t)h.entries * c.page_size);
    A.seqs = h.seqs;
    A.reqs = h.reqs;
    A.cuts = h.cuts;
    A.backs = h.backs;
    A.order = h.order;
    A.small = h.small;
    A.large = h.large;
    A.merge = h.merge;
    A.write = h.write;
    A.table = h.table;
    const bool by_row = t.row_seq || t.row_pos || t.row_slot;
    A.tails = by_row ? std::min(64, (h.tokens + 255) / 256) : 0;
    hipStream_t s = (hipStream_t)stream;
    if (!h.n_large && h.batch == 1) {
        hipLaunchKernelGGL(k_build_one, dim3(1), dim3(256), 0, s, A);
        SPD_HIP(hipGetLastError());
        return SPD_OK;
    }
    const int threads = h.n_large ? THREADS : std::min(THREADS, (h.batch + 63) / 64 * 64);
    if (h.batch <= THREADS) hipLaunchKernelGGL((k_build_sums<1>), dim3(1), dim3(threads), 0, s, A);
    else hipLaunchKernelGGL((k_build_sums<SPD_BUILD_BATCH / THREADS>), dim3(1), dim3(THREADS), 0, s, A);
    SPD_HIP(hipGetLastError());
    hipLaunchKernelGGL(k_build_requests, dim3(h.batch + A.tails, by_row ? (h.q_len + CHUNK_ROWS - 1) / CHUNK_ROWS : 1), dim3(256), 0, s, A);
    SPD_HIP(hipGetLastError());
    return SPD_OK;
}
