// Pages that requests share: forks, truncations and ends of requests whose pages others may hold, pages moved to the front of a
// cache, and the copies of pages that both ask for.  Tables and stacks as in cache.hip; a page of either cache is a row of bytes here.
#include <limits.h>

#include <type_traits>

#include "launch.hpp"
#include "pages.hpp"

namespace ea {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// ---- forks ----------------------------------------------------------------------------------------------------------
// Request r becomes the first new_lens[r] tokens of what request parents[r] held, all at once.  shares[page] counts the holders of a page beyond
// the first.  Every entry that a request takes over adds a holder and every one that it leaves takes one away; integer
// atomics, whose order does not matter.  A page that comes out below zero has no holder: its last entry among those that are
// left (of the last request, its last page) claims it by an atomic minimum on the count itself, and a sum over the claims gives it its
// place on the stack.  A page that ends a request in its middle will be written to, so if others hold it, too, the request gets a copy; one
// of those it ends may keep it unless somebody holds it whole.
// Bound: latency, of the chain lengths -> entries -> counts -> claims -> stack -> tails.  Up to FORK_ONE entries in the tables one work-group
// does all of it, for its steps to be a barrier apart and not a launch.  More are FORK_GROUPS work-groups' work where it counts, since a
// compute unit handles about one address a clock where they are all different: there are four launches then, by FORK_STEP.
// 64 requests, 56 of them new with 1700 pages of 8 prompts: 12 us in one launch, 16 in four (with the ending and the copies 31.1 us a pass and 51.0);
// 1020 with 45000 pages of 60 prompts: 130 us in one, 22 in four, and their end 162 and 34.

constexpr int FORK_THREADS = 1024;
constexpr int FORK_MAX_REQUESTS = 4096;
constexpr int FORK_AT_ONCE = 8;         // entries a thread has on their way

struct ForkParams {
    const int32_t* lens; const int32_t* parents; const int32_t* new_lens;
    int32_t* table;            // [R][blocks]
    int32_t* free_pages; int32_t* free_count;
    int32_t* shares;           // [n_pages]
    int32_t* lens_out;         // [R]
    int32_t* moves;            // [R][2]
    int32_t* status;           // [4]
    int32_t* taken; int32_t* left;      // [R * blocks] each (workspace): pages taken over, pages left
    int32_t* lists;            // [6][FORK_LIST] (workspace): what the launches hand on of the requests
    int R, blocks, page_shift, n_pages;
};

enum FORK_STEP { FORK_ALL, FORK_LENGTHS, FORK_COUNT, FORK_CLAIM, FORK_FINISH };
// (R * max_blocks: how many pages there are the host does not know.  A fork of 8 or 128 prompts to all requests and its end, replayed / from Python, us in one
// launch and in four: 64 requests of 256 blocks with full tables 65 / 65 and 28 / 35, 1024 of 16 74 / 74 and 31 / 36; with tables 1/64 full 20 / 20 and 23 / 35,
// 29 / 29 and 27 / 38.  At 65536 entries, full: 251 to 278 and 40 to 45; 1/64 full: 21 to 29 and 24 to 36.  The border is drawn for tables with room
// to grow, where one launch saves the host three; full tables of 16384 entries are twice as fast in four.)
constexpr long FORK_ONE = 16384;
constexpr int FORK_GROUPS = 256, FORK_LIST = FORK_MAX_REQUESTS + 8;

// (one work-group's scope will do for its own counts: across the card's L2s atomics take several times as long)
template <FORK_STEP STEP> struct Counts {
    static constexpr int SCOPE = STEP == FORK_COUNT || STEP == FORK_CLAIM ? __HIP_MEMORY_SCOPE_AGENT : __HIP_MEMORY_SCOPE_WORKGROUP;
    static EA_DEV int get(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, SCOPE); }
    static EA_DEV void set(int32_t* p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, SCOPE); }
    static EA_DEV void add(int32_t* p, int v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, SCOPE); }
    static EA_DEV void min(int32_t* p, int v) { __hip_atomic_fetch_min(p, v, __ATOMIC_RELAXED, SCOPE); }
};

// Sum of v over the threads below this one; total: over all.  Every thread calls it.
template <int NW> EA_DEV int group_scan(int v, int (*sums)[NW], int turn, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = wave_scan(v);
    if (lane == 63) sums[turn][wave] = at;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) { const int s = sums[turn][w]; if (w < wave) before += s; total += s; }
    return before + at - v;
}

template <FORK_STEP STEP>
__global__ __launch_bounds__(FORK_THREADS) void cache_fork_kernel(ForkParams p) {
    using C = Counts<STEP>;
    constexpr bool ALL = STEP == FORK_ALL;
    constexpr int T = FORK_THREADS, NW = T / 64, U = STEP == FORK_COUNT || STEP == FORK_CLAIM ? 1 : FORK_AT_ONCE, MAX = FORK_MAX_REQUESTS, SLOTS = 2 * MAX;
    __shared__ int32_t have[MAX], next[MAX], tail[MAX];         // lengths before and after; the page in whose middle a request comes to end, or -1
    __shared__ int32_t prefix[2][MAX + 1];                      // entries taken over and left by the requests in front
    __shared__ uint16_t from[MAX];
    __shared__ unsigned int ends[MAX], best[MAX];
    // claims a thread looks at at a time, their counts per lane (45000 claims, the last launch: 22.6 us with 4, 20.0 with 8, 18.6 with 16, 21.7 with 32)
    constexpr int S = ALL ? 64 / NW : 256 / NW, PER = NW * S / 64;
    __shared__ int sums[2][NW], claims[2][NW * S];
    __shared__ int invalid, strange;
    int32_t* const take = prefix[0];
    int32_t* const leave = prefix[1];
    const int tid = threadIdx.x, R = p.R, shift = p.page_shift, most = p.blocks << shift;
    int turn = 0;
    auto scan = [&](int v, int& total) { turn ^= 1; return group_scan<NW>(v, sums, turn, total); };
    auto ok_page = [&](int page) { return (unsigned)page < (unsigned)p.n_pages; };
    auto tail_of = [&](int parent, int len) {
        if (!(len & ((1 << shift) - 1))) return -1;
        const int page = p.table[(long)parent * p.blocks + (len >> shift)];
        return ok_page(page) ? page : -1;
    };
    int takes = 0, leaves = 0;
    if constexpr (ALL || STEP == FORK_LENGTHS) {
        if (tid == 0) { invalid = strange = 0; take[0] = leave[0] = 0; }
        for (int r = tid; r < R; r += T) have[r] = p.lens[r];
        for (int r0 = 0; r0 < R; r0 += T) {
            const int r = r0 + tid;
            int a = 0, b = 0;                             // entries taken over, left
            int parent = r < R ? p.parents[r] : 0, len = r < R ? p.new_lens[r] : 0;
            if (r0 == 0) __syncthreads();
            if (r < R) {
                // a request whose lengths or parent are out of range stays as it is, its last page among those that are held whole (and one whose
                // own length is takes part in nothing)
                const bool mine = have[r] >= 0 && have[r] <= most;
                const int theirs = have[min(max(parent, 0), R - 1)];
                const bool stays = !(mine && (unsigned)parent < (unsigned)R && theirs <= most && len >= 0 && len <= theirs);
                if (stays) {
                    parent = r;
                    len = mine ? have[r] : 0;
                    atomicAdd(&invalid, 1);
                }
                from[r] = (uint16_t)parent;
                next[r] = len;
                tail[r] = stays ? -1 : tail_of(parent, len);
                const int old = mine ? pages_of(have[r], shift) : 0, now = pages_of(len, shift);
                a = parent == r ? 0 : now;
                b = !mine ? 0 : parent == r ? old - now : old;
            }
            int ta, tb;
            a += scan(a, ta);
            b += scan(b, tb);
            if (r < R) { take[r + 1] = takes + a; leave[r + 1] = leaves + b; }
            takes += ta; leaves += tb;
        }
        __syncthreads();
    }
    int32_t* const kept[6] = {p.lists, p.lists + FORK_LIST, p.lists + 2 * FORK_LIST, p.lists + 3 * FORK_LIST, p.lists + 4 * FORK_LIST, p.lists + 5 * FORK_LIST};
    if constexpr (STEP == FORK_LENGTHS) {
        for (int r = tid; r < R; r += T) { kept[0][r] = have[r]; kept[1][r] = next[r]; kept[2][r] = tail[r]; kept[3][r] = from[r]; }
        for (int r = tid; r <= R; r += T) { kept[4][r] = take[r]; kept[5][r] = leave[r]; }
        if (tid == 0) { p.status[2] = invalid; p.status[3] = 0; }
        return;
    } else if constexpr (!ALL) {
        for (int r = tid; r < R; r += T) { have[r] = kept[0][r]; next[r] = kept[1][r]; tail[r] = kept[2][r]; from[r] = (uint16_t)kept[3][r]; }
        for (int r = tid; r <= R; r += T) { take[r] = kept[4][r]; leave[r] = kept[5][r]; }
        if (tid == 0) invalid = strange = 0;
        __syncthreads();
        takes = take[R]; leaves = leave[R];
    }
    const int first = (ALL ? 0 : blockIdx.x * (T * U)) + tid, stride = (ALL ? 1 : FORK_GROUPS) * T * U;
    // the requests that have entries i0 + u T, U searches side by side
    const int top_step = R > 1 ? 1 << (31 - __clz(R - 1)) : 0;
    auto owners = [&](const int32_t* pref, int i0, int (&r)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = 0;
        for (int step = top_step; step; step >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (r[u] + step < R && pref[r[u] + step] <= i0 + u * T) r[u] += step;
    };
    if constexpr (ALL || STEP == FORK_COUNT) {
        int odd = 0;
        // of two lists of entries, each by its own rule: read, noted, counted
        auto count_all = [&](const int32_t* pref, int n, int32_t* note, int by, auto entry) {
            for (int i0 = first; i0 < n; i0 += stride) {
                int r[U], page[U];
                owners(pref, i0, r);
#pragma unroll
                for (int u = 0; u < U; ++u) page[u] = i0 + u * T < n ? p.table[entry(r[u], i0 + u * T - pref[r[u]])] : 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (i0 + u * T >= n) break;
                    note[i0 + u * T] = page[u];
                    if (ok_page(page[u])) C::add(&p.shares[page[u]], by); else ++odd;
                }
            }
        };
        count_all(take, takes, p.taken, 1, [&](int r, int k) { return (long)from[r] * p.blocks + k; });
        count_all(leave, leaves, p.left, -1, [&](int r, int k) { return (long)r * p.blocks + (from[r] == r ? pages_of(next[r], shift) : 0) + k; });
        if (odd) atomicAdd(ALL ? &strange : &p.status[3], odd);
        if constexpr (ALL) { __threadfence_block(); __syncthreads(); }
    }
    if constexpr (ALL || STEP == FORK_CLAIM) {
        // the tables of the forks
        for (int i0 = first; i0 < takes; i0 += stride) {
            int r[U];
            owners(take, i0, r);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * T;
                if (i < takes) p.table[(long)r[u] * p.blocks + (i - take[r[u]])] = p.taken[i];
            }
        }
        // claims: the count becomes -2 - i for the last entry i of a page without a holder; other entries are struck off
        for (int i0 = first; i0 < leaves; i0 += stride) {
            int page[U], held[U];
#pragma unroll
            for (int u = 0; u < U; ++u) page[u] = i0 + u * T < leaves ? p.left[i0 + u * T] : -1;
#pragma unroll
            for (int u = 0; u < U; ++u) held[u] = ok_page(page[u]) ? C::get(&p.shares[page[u]]) : 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (held[u] < 0) C::min(&p.shares[page[u]], -2 - (i0 + u * T));
                else if (i0 + u * T < leaves) p.left[i0 + u * T] = -1;
            }
        }
        if constexpr (ALL) { __threadfence_block(); __syncthreads(); }
    }
    if constexpr (ALL || STEP == FORK_FINISH) {
        const int count = min(max(*p.free_count, 0), p.n_pages);
        // the stack: claims from the last entry to the first, S of a thread's at a time and the next on their way
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        int back = 0, page[S], ahead[S];
        auto left_from = [&](int i0, int (&x)[S]) {
#pragma unroll
            for (int u = 0; u < S; ++u) { const int i = leaves - 1 - (i0 + u * T + tid); x[u] = i >= 0 ? p.left[i] : -1; }
        };
        left_from(0, ahead);
        for (int i0 = 0; i0 < leaves; i0 += T * S) {
            unsigned long long in[S];
            turn ^= 1;
#pragma unroll
            for (int u = 0; u < S; ++u) page[u] = ahead[u];
            left_from(i0 + T * S, ahead);
#pragma unroll
            for (int u = 0; u < S; ++u) {
                const bool mine = ok_page(page[u]) && C::get(&p.shares[page[u]]) == -2 - (leaves - 1 - (i0 + u * T + tid));
                in[u] = __ballot(mine);
                if (lane == 0) claims[turn][u * NW + wave] = __popcll(in[u]);
            }
            __syncthreads();
            int n = 0, at_wave = 0;                       // of the lane's counts; of those in front of its one of this wave
#pragma unroll
            for (int k = 0; k < PER; ++k) { const int c = claims[turn][PER * lane + k]; n += c; if (k < wave % PER) at_wave += c; }
            const int up_to = wave_scan(n);
#pragma unroll
            for (int u = 0; u < S; ++u) {
                const int at = count + back + __builtin_amdgcn_readlane(up_to - n + at_wave, (u * NW + wave) / PER) + __popcll(in[u] & ((1ull << lane) - 1ull));
                if (in[u] >> lane & 1) {
                    if (at < p.n_pages) p.free_pages[at] = page[u];
                    else atomicAdd(&strange, 1);          // (the stack was full: its count was none of free pages)
                    C::set(&p.shares[page[u]], 0);
                }
            }
            back += __builtin_amdgcn_readlane(up_to, 63);
        }
        const int top = min(count + back, p.n_pages);
        // tails: how many requests end in a page, and which of them may keep it, by a table of those pages that others hold too
        int32_t* const slots = prefix[0];                 // (SLOTS of them; the sums are no longer needed)
        static_assert(SLOTS <= 2 * (MAX + 1) && (SLOTS & (SLOTS - 1)) == 0, "the table has a mask and lies over the sums");
        __syncthreads();
        for (int i = tid; i < SLOTS; i += T) slots[i] = -1;
        for (int r = tid; r < R; r += T) { ends[r] = 0; best[r] = 2 * MAX; }
        __syncthreads();
        // the request that stands for all with this page: the first that came upon its place
        auto stands_for = [&](int page, int r) {
            for (unsigned int h = (unsigned int)page * 2654435761u >> 19;; h = (h + 1) & (SLOTS - 1)) {
                int k = slots[h];
                if (k < 0) { k = atomicCAS(&slots[h], -1, r); if (k < 0) k = r; }
                if (tail[k] == page) return k;
            }
        };
        auto rank = [&](int r) { return (unsigned int)(from[r] == r ? r : MAX + r); };
        constexpr int EACH = MAX / T;                     // requests of a thread
        int stand[EACH], holders[EACH], which[EACH];      // which: a copy's number among all
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int r = e * T + tid;
            stand[e] = which[e] = -1;
            holders[e] = r < R && tail[r] >= 0 ? C::get(&p.shares[tail[r]]) + 1 : 0;
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int r = e * T + tid;
            if (holders[e] <= 1) continue;
            stand[e] = stands_for(tail[r], r);
            atomicAdd(&ends[stand[e]], 1u);
            atomicMin(&best[stand[e]], rank(r));
        }
        __threadfence_block();                            // (the stack, for its readers below)
        __syncthreads();
        int copies = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int r = e * T + tid;
            if (e * T >= R) break;
            const bool copy = stand[e] >= 0 && (holders[e] > (int)ends[stand[e]] || best[stand[e]] != rank(r));
            int total;
            const int at = copies + scan(copy, total);
            if (copy) which[e] = at;
            copies += total;
        }
        const int granted = min(copies, top);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int r = e * T + tid;
            if (r >= R) break;
            const int len = next[r];
            const bool mine = have[r] >= 0 && have[r] <= most;
            // (where no page is left the request ends before its tail)
            p.lens_out[r] = !mine ? have[r] : which[e] >= granted ? len & -(1 << shift) : len;
            if (which[e] >= 0) {
                C::add(&p.shares[tail[r]], -1);
                if (which[e] < granted) {
                    const int to = p.free_pages[top - 1 - which[e]];
                    if (!ok_page(to)) atomicAdd(&strange, 1);
                    p.table[(long)r * p.blocks + (len >> shift)] = to;
                    *(i32x2*)(p.moves + 2 * which[e]) = i32x2{tail[r], to};
                }
            }
            if (r >= granted) *(i32x2*)(p.moves + 2 * r) = i32x2{-1, -1};
        }
        __syncthreads();
        if (tid == 0) {
            *p.free_count = top - granted;
            p.status[0] = granted; p.status[1] = copies - granted;
            if constexpr (ALL) { p.status[2] = invalid; p.status[3] = strange; }
            else p.status[3] += strange;
        }
    }
}

// ---- compaction -----------------------------------------------------------------------------------------------------
// Of n_pages, `used` are not on the stack of free ones.  The i-th free page below `used` (a hole) takes what the i-th page in use from
// `used` on holds; there are as many of one as of the other.  A bit per page, set for the free ones, and the number of set bits in
// front of each word give either's rank.
// One work-group makes bits, sums and the list of holes; a thread for each page and each entry of the tables then makes moves and tables of
// it.  Bound: latency, of two launches: 4.7 and 4.8 us for 9000 pages (five launches, each for all pages: 16 us in all).

constexpr int COMPACT_THREADS = 256;
constexpr int COMPACT_WORDS = 1 << 14;      // of 32 pages, up to which the bits are made in LDS

struct CompactParams {
    const int32_t* lens; const int32_t* table; const int32_t* free_pages; const int32_t* free_count; const int32_t* shares;
    int32_t* table_out; int32_t* free_out; int32_t* shares_out; int32_t* moves; int32_t* status;
    uint32_t* bits;            // [words + 1]: a page's bit is set if it is free
    int32_t* before;           // [words + 1]: set bits in the words in front
    int32_t* holes;            // [n_pages / 2]: free pages below `used`, in order
    int R, blocks, page_shift, n_pages, words;
};

EA_DEV int compact_free(const CompactParams& p) { return min(max(*p.free_count, 0), p.n_pages); }
EA_DEV bool bit_of(const CompactParams& p, int page) { return p.bits[page >> 5] >> (page & 31) & 1; }
// free pages in front of `page`
EA_DEV int free_before(const CompactParams& p, int page) { return p.before[page >> 5] + __popc(p.bits[page >> 5] & ((1u << (page & 31)) - 1u)); }

template <bool IN_LDS>
__global__ __launch_bounds__(1024) void compact_index_kernel(CompactParams p) {
    constexpr int T = 1024, NW = T / 64, U = 8;
    __shared__ int sums[2][NW];
    __shared__ uint32_t local[IN_LDS ? COMPACT_WORDS : 1];
    __shared__ int strange;
    const int tid = threadIdx.x, free = compact_free(p);
    uint32_t* const bits = IN_LDS ? local : p.bits;
    if (tid == 0) strange = 0;
    for (int w = tid; w < p.words; w += T) bits[w] = 0u;
    __threadfence_block();
    __syncthreads();
    int odd = 0;
    for (int i0 = tid; i0 < free; i0 += T * U) {
        int page[U];
#pragma unroll
        for (int u = 0; u < U; ++u) page[u] = i0 + u * T < free ? p.free_pages[i0 + u * T] : 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * T >= free) break;
            const unsigned int bit = 1u << (page[u] & 31);
            const bool fresh = (unsigned)page[u] < (unsigned)p.n_pages &&
                               !(__hip_atomic_fetch_or(&bits[page[u] >> 5], bit, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) & bit);
            odd += !fresh;                                // (out of range, or on the stack twice)
        }
    }
    if (odd) atomicAdd(&strange, odd);
    __threadfence_block();
    __syncthreads();
    int at = 0, turn = 0;
    for (int w0 = 0; w0 <= p.words; w0 += T) {
        const int w = w0 + tid, n = w < p.words ? __popc(__hip_atomic_load(&bits[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)) : 0;
        int total;
        turn ^= 1;
        const int first = at + group_scan<NW>(n, sums, turn, total);
        if (w <= p.words) p.before[w] = first;
        at += total;
    }
    const int used = p.n_pages - at;
    for (int w = tid; w <= p.words; w += T) {             // (each thread its own sums again)
        uint32_t x = w < p.words ? __hip_atomic_load(&bits[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0u;
        if (IN_LDS) p.bits[w] = x;
        int rank = p.before[w];
        for (; x; x &= x - 1) {
            const int page = 32 * w + __ffs((int)x) - 1;
            if (page < used) p.holes[rank++] = page;
        }
    }
    if (tid < 4) p.status[tid] = tid == 1 ? used : tid == 3 ? strange : 0;
}
// One thread for each page, then one for each entry of the tables
__global__ __launch_bounds__(COMPACT_THREADS) void compact_move_kernel(CompactParams p) {
    const long id = (long)blockIdx.x * COMPACT_THREADS + threadIdx.x;
    const int used = p.n_pages - p.before[p.words];
    auto place = [&](int page) {                          // where page `page`, which is in use, goes
        // (rank among the pages in use from `used` on)
        return page < used ? page : p.holes[(page - used) - (free_before(p, page) - free_before(p, used))];
    };
    if (id < p.n_pages) {
        const int page = (int)id, holes = used < p.n_pages ? free_before(p, used) : 0;
        // entries of the stack, and how many of them are no page or one that is on it already: -1 in their place, taken last of all
        const int stack = compact_free(p), empty = stack - p.before[p.words];
        if (page < p.n_pages / 2 && page >= holes) *(i32x2*)(p.moves + 2 * page) = i32x2{-1, -1};
        p.free_out[page] = page < empty ? -1 : page < stack ? p.n_pages - 1 - (page - empty) : p.free_pages[page];
        if (p.shares) {
            // (a page's count is read and written by one thread, and a moved one's by the page that it moves from)
            if (page >= used) {
                if (!bit_of(p, page)) { p.shares_out[place(page)] = p.shares[page]; }
                p.shares_out[page] = 0;
            } else if (!bit_of(p, page)) p.shares_out[page] = p.shares[page];
        }
        if (page >= used && !bit_of(p, page)) {
            const int rank = (page - used) - (free_before(p, page) - holes);
            *(i32x2*)(p.moves + 2 * rank) = i32x2{page, p.holes[rank]};
        }
        if (page == 0) p.status[0] = holes;
        return;
    }
    const long i = id - p.n_pages;
    if (i >= (long)p.R * p.blocks) return;
    const int r = (int)(i / p.blocks), b = (int)(i - (long)r * p.blocks), len = p.lens[r];
    int page = p.table[i];
    const bool ok = len >= 0 && len <= p.blocks << p.page_shift;
    if (!ok && b == 0) atomicAdd(&p.status[2], 1);
    if (ok && b < pages_of(len, p.page_shift)) {
        // (an entry that is no page in use stays as it is)
        if ((unsigned)page >= (unsigned)p.n_pages || bit_of(p, page)) atomicAdd(&p.status[3], 1);
        else page = place(page);
    }
    p.table_out[i] = page;
}

// ---- copies ---------------------------------------------------------------------------------------------------------
// moves[i] = (from, to), the first `count` of them.  Bound: HBM, twice the pages' bytes.  A work-group copies 16 KB at a time, four
// loads of 16 bytes a thread on their way together (eight: no faster).  Copies of more than COPY_FAR bytes in all bypass the caches: 2230 pages of
// 132 KB, 589 MB read and written, take 118 us, 5.0 TB/s, for 127; 110 of them 7.9 us for 7.1.  Around the border, pages of a cache of 3 GB: 61 MiB 27.1
// past the caches and 27.1 through them, 121 MiB 52.9 and 54.9, 30 MiB 14.4 and 12.9.

constexpr int COPY_U = 4, COPY_PIECE = 256 * COPY_U;      // of 16 bytes
constexpr long COPY_FAR = 64l << 20;

__global__ __launch_bounds__(256) void cache_copy_kernel(const i32x4* src, i32x4* dst, const int32_t* moves, const int32_t* count, int most,
                                                         int units, int src_pages, int dst_pages) {
    const int n = min(max(*count, 0), most), pieces = (units + COPY_PIECE - 1) / COPY_PIECE;
    const long all = (long)n * pieces;
    auto copy = [&](auto far) {
        for (long w = blockIdx.x; w < all; w += gridDim.x) {
            const int i = (int)(w / pieces), piece = (int)(w - (long)i * pieces);
            const int from = moves[2l * i], to = moves[2l * i + 1];
            if ((unsigned)from >= (unsigned)src_pages || (unsigned)to >= (unsigned)dst_pages) continue;
            const i32x4* const a = src + (long)from * units;
            i32x4* const b = dst + (long)to * units;
            i32x4 v[COPY_U];
#pragma unroll
            for (int u = 0; u < COPY_U; ++u) { const int k = piece * COPY_PIECE + u * 256 + threadIdx.x; if (k < units) v[u] = __builtin_nontemporal_load(a + k); }
#pragma unroll
            for (int u = 0; u < COPY_U; ++u) {
                const int k = piece * COPY_PIECE + u * 256 + threadIdx.x;
                if (k >= units) continue;
                if constexpr (decltype(far)::value) __builtin_nontemporal_store(v[u], b + k); else b[k] = v[u];
            }
        }
    };
    if ((long)n * units * 16 > COPY_FAR) copy(std::true_type{}); else copy(std::false_type{});
}

}  // namespace ea

namespace {
using namespace ea;

bool tables_shape_ok(int R, int blocks, int page, int n_pages) {
    return R > 0 && R <= FORK_MAX_REQUESTS && blocks > 0 && cache_page_ok(page) && n_pages > 0 && (long)blocks * page <= (1l << 22) &&
           (long)n_pages * page <= (long)INT_MAX;
}
size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
bool workspace_ok(const void* ws, size_t have, size_t need) { return ws && !((uintptr_t)ws & 255) && have >= need; }
int compact_words(int n_pages) { return (n_pages + 31) / 32; }

}  // namespace

extern "C" {

size_t entmax_attn_cache_fork_workspace_bytes(int R, int max_blocks) {
    if (!tables_shape_ok(R, max_blocks, 16, 1)) return 0;
    return 2 * round256((size_t)R * max_blocks * 4) + round256(6 * FORK_LIST * 4);
}

int entmax_attn_cache_fork(const int32_t* lens, const int32_t* parents, const int32_t* new_lens, int32_t* block_table, int32_t* free_pages,
                           int32_t* free_count, int32_t* shares, int32_t* lens_out, int32_t* moves, int32_t* status,
                           int R, int max_blocks, int page_size, int n_pages, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!lens || !parents || !new_lens || !block_table || !free_pages || !free_count || !shares || !lens_out || !moves || !status) return EA_ERR_NULL;
    if (!tables_shape_ok(R, max_blocks, page_size, n_pages)) return EA_ERR_SHAPE;
    if (lens_out == new_lens || lens_out == parents || ((uintptr_t)moves & 7)) return EA_ERR_LAYOUT;
    if (!workspace_ok(workspace, workspace_bytes, entmax_attn_cache_fork_workspace_bytes(R, max_blocks))) return EA_ERR_WORKSPACE;
    ForkParams p{lens, parents, new_lens, block_table, free_pages, free_count, shares, lens_out, moves, status};
    const size_t entries = round256((size_t)R * max_blocks * 4);
    p.taken = (int32_t*)workspace; p.left = (int32_t*)((char*)workspace + entries); p.lists = (int32_t*)((char*)workspace + 2 * entries);
    p.R = R; p.blocks = max_blocks; p.page_shift = cache_page_shift(page_size); p.n_pages = n_pages;
    hipStream_t s = (hipStream_t)hip_stream;
    const dim3 block(FORK_THREADS);
    if ((long)R * max_blocks <= FORK_ONE) {
        hipLaunchKernelGGL(cache_fork_kernel<FORK_ALL>, dim3(1), block, 0, s, p);
    } else {
        hipLaunchKernelGGL(cache_fork_kernel<FORK_LENGTHS>, dim3(1), block, 0, s, p);
        hipLaunchKernelGGL(cache_fork_kernel<FORK_COUNT>, dim3(FORK_GROUPS), block, 0, s, p);
        hipLaunchKernelGGL(cache_fork_kernel<FORK_CLAIM>, dim3(FORK_GROUPS), block, 0, s, p);
        hipLaunchKernelGGL(cache_fork_kernel<FORK_FINISH>, dim3(1), block, 0, s, p);
    }
    return launched();
}

size_t entmax_attn_cache_compact_workspace_bytes(int n_pages) {
    if (n_pages <= 0 || n_pages > (1 << 27)) return 0;
    return 2 * round256(((size_t)compact_words(n_pages) + 1) * 4) + round256(((size_t)n_pages / 2 + 1) * 4);
}

int entmax_attn_cache_compact(const int32_t* lens, const int32_t* block_table, const int32_t* free_pages, const int32_t* free_count,
                              const int32_t* shares, int32_t* table_out, int32_t* free_out, int32_t* shares_out, int32_t* moves, int32_t* status,
                              int R, int max_blocks, int page_size, int n_pages, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!lens || !block_table || !free_pages || !free_count || !table_out || !free_out || (n_pages > 1 && !moves) || !status || !shares != !shares_out)
        return EA_ERR_NULL;
    if (!tables_shape_ok(R, max_blocks, page_size, n_pages)) return EA_ERR_SHAPE;
    if ((uintptr_t)moves & 7) return EA_ERR_LAYOUT;
    if (!workspace_ok(workspace, workspace_bytes, entmax_attn_cache_compact_workspace_bytes(n_pages))) return EA_ERR_WORKSPACE;
    CompactParams p{lens, block_table, free_pages, free_count, shares, table_out, free_out, shares_out, moves, status};
    p.R = R; p.blocks = max_blocks; p.page_shift = cache_page_shift(page_size); p.n_pages = n_pages; p.words = compact_words(n_pages);
    char* ws = (char*)workspace;
    p.bits = (uint32_t*)ws; ws += round256(((size_t)p.words + 1) * 4);
    p.before = (int32_t*)ws; ws += round256(((size_t)p.words + 1) * 4);
    p.holes = (int32_t*)ws;
    hipStream_t s = (hipStream_t)hip_stream;
    if (p.words <= COMPACT_WORDS) hipLaunchKernelGGL(compact_index_kernel<true>, dim3(1), dim3(1024), 0, s, p);
    else hipLaunchKernelGGL(compact_index_kernel<false>, dim3(1), dim3(1024), 0, s, p);
    const long items = n_pages + (long)R * max_blocks;
    hipLaunchKernelGGL(compact_move_kernel, dim3((unsigned int)((items + COMPACT_THREADS - 1) / COMPACT_THREADS)), dim3(COMPACT_THREADS), 0, s, p);
    return launched();
}

int entmax_attn_cache_copy(const void* src, void* dst, const int32_t* moves, const int32_t* count, int max_moves, size_t page_bytes,
                           int src_pages, int dst_pages, void* hip_stream) {
    if (!src || !dst || !count || (max_moves > 0 && !moves)) return EA_ERR_NULL;
    if (max_moves < 0 || src_pages <= 0 || dst_pages <= 0 || page_bytes == 0 || page_bytes / 16 > (size_t)(INT_MAX - COPY_PIECE)) return EA_ERR_SHAPE;
    if (page_bytes % 16 || !aligned16(src) || !aligned16(dst)) return EA_ERR_LAYOUT;
    if (max_moves == 0) return EA_OK;
    const int units = (int)(page_bytes / 16);
    const long work = (long)max_moves * ((units + COPY_PIECE - 1) / COPY_PIECE);
    hipLaunchKernelGGL(cache_copy_kernel, dim3((unsigned int)(work < 4096 ? work : 4096)), dim3(256), 0, (hipStream_t)hip_stream,
                       (const i32x4*)src, (i32x4*)dst, moves, count, max_moves, units, src_pages, dst_pages);
    return launched();
}

}  // extern "C"
