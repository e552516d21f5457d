// Pages that requests share: forks, truncations and ends of requests whose pages others may hold, pages moved to the front of a
// cache, and the copies of pages that both ask for.  Tables and stacks as in cache.hip; a page of either cache is a row of bytes here.
#include <limits.h>

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
// Bound: latency, of the chain lengths -> entries -> counts -> claims -> stack -> tails.  One work-group does all of it, for its steps to
// be a barrier apart and not a launch.

constexpr int FORK_THREADS = 1024;
constexpr int FORK_MAX_REQUESTS = 4096;
constexpr int FORK_AT_ONCE = 4;         // entries a thread has on their way

struct ForkParams {
    const int32_t* lens; const int32_t* parents; const int32_t* new_lens;
    int32_t* table;            // [R][blocks]
    int32_t* free_pages; int32_t* free_count;
    int32_t* shares;           // [n_pages]
    int32_t* lens_out;         // [R]
    int32_t* moves;            // [R][2]
    int32_t* status;           // [4]
    int32_t* taken; int32_t* left;      // [R * blocks] each (workspace): pages taken over, pages left
    int R, blocks, page_shift, n_pages;
};

EA_DEV int count_of(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
EA_DEV void count_add(int32_t* p, int v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Sum of v over the threads below this one; total: over all.  Every thread calls it.
template <int NW> EA_DEV int group_scan(int v, int (*sums)[NW], int turn, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int at = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) { const int o = __shfl_up(at, off); if (lane >= off) at += o; }
    if (lane == 63) sums[turn][wave] = at;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) { const int s = sums[turn][w]; if (w < wave) before += s; total += s; }
    return before + at - v;
}
__global__ __launch_bounds__(FORK_THREADS) void cache_fork_kernel(ForkParams p) {
    constexpr int T = FORK_THREADS, NW = T / 64, U = FORK_AT_ONCE, MAX = FORK_MAX_REQUESTS;
    __shared__ int32_t have[MAX], next[MAX], take[MAX + 1], leave[MAX + 1];       // lengths; prefix sums of entries taken over and left
    __shared__ uint16_t from[MAX];
    __shared__ int sums[2][NW];
    __shared__ int invalid, strange;
    const int tid = threadIdx.x, R = p.R, shift = p.page_shift, most = p.blocks << shift;
    const int count = min(max(*p.free_count, 0), p.n_pages);
    int turn = 0;
    auto scan = [&](int v, int& total) { turn ^= 1; return group_scan<NW>(v, sums, turn, total); };
    if (tid == 0) { invalid = strange = 0; take[0] = leave[0] = 0; }
    for (int r = tid; r < R; r += T) have[r] = p.lens[r];
    __syncthreads();
    int takes = 0, leaves = 0;
    for (int r0 = 0; r0 < R; r0 += T) {
        const int r = r0 + tid;
        int a = 0, b = 0;                                 // entries taken over, left
        if (r < R) {
            // a request whose lengths or parent are out of range stays as it is (and one whose own length is takes part in nothing)
            int parent = p.parents[r], len = p.new_lens[r];
            const bool mine = have[r] >= 0 && have[r] <= most;
            const bool ok = mine && (unsigned)parent < (unsigned)R && len >= 0 && len <= have[min(max(parent, 0), R - 1)] &&
                            have[min(max(parent, 0), R - 1)] <= most;
            if (!ok) { parent = r; len = mine ? have[r] : 0; atomicAdd(&invalid, 1); }
            from[r] = (uint16_t)parent;
            next[r] = len;
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
    // entry k of what request r leaves is its page base + k
    auto left_at = [&](int i, int r) { return (from[r] == r ? pages_of(next[r], shift) : 0) + (i - leave[r]); };
    auto ok_page = [&](int page) { return (unsigned)page < (unsigned)p.n_pages; };
    int odd = 0;
    for (int i0 = tid; i0 < takes; i0 += T * U) {
        int page[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * T;
            page[u] = -1;
            if (i < takes) { const int r = owner(take, R, i); page[u] = p.table[(long)from[r] * p.blocks + (i - take[r])]; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * T;
            if (i >= takes) break;
            p.taken[i] = page[u];
            if (ok_page(page[u])) count_add(&p.shares[page[u]], 1); else ++odd;
        }
    }
    for (int i0 = tid; i0 < leaves; i0 += T * U) {
        int page[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * T;
            page[u] = -1;
            if (i < leaves) { const int r = owner(leave, R, i); page[u] = p.table[(long)r * p.blocks + left_at(i, r)]; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * T;
            if (i >= leaves) break;
            p.left[i] = page[u];
            if (ok_page(page[u])) count_add(&p.shares[page[u]], -1); else ++odd;
        }
    }
    if (odd) atomicAdd(&strange, odd);
    __threadfence();
    __syncthreads();
    // the tables of the forks; claims: the count becomes -2 - i for the last entry i of a page without a holder
    for (int i0 = tid; i0 < takes; i0 += T * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * T;
            if (i < takes) { const int r = owner(take, R, i); p.table[(long)r * p.blocks + (i - take[r])] = p.taken[i]; }
        }
    }
    for (int i0 = tid; i0 < leaves; i0 += T * U) {
        int page[U], held[U];
#pragma unroll
        for (int u = 0; u < U; ++u) page[u] = i0 + u * T < leaves ? p.left[i0 + u * T] : -1;
#pragma unroll
        for (int u = 0; u < U; ++u) held[u] = ok_page(page[u]) ? count_of(&p.shares[page[u]]) : 0;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (held[u] < 0) __hip_atomic_fetch_min(&p.shares[page[u]], -2 - (i0 + u * T), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __threadfence();
    __syncthreads();
    // the stack: claims from the last entry to the first
    int back = 0;
    for (int i0 = 0; i0 < leaves; i0 += T * U) {
        int page[U], n = 0;
        bool mine[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = leaves - 1 - (i0 + tid * U + u);
            page[u] = i >= 0 ? p.left[i] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = leaves - 1 - (i0 + tid * U + u);
            mine[u] = ok_page(page[u]) && count_of(&p.shares[page[u]]) == -2 - i;
            n += mine[u];
        }
        int total, at = count + back + scan(n, total);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (mine[u]) {
                if (at < p.n_pages) p.free_pages[at] = page[u];
                ++at;
                __hip_atomic_store(&p.shares[page[u]], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        back += total;
    }
    __threadfence();
    __syncthreads();
    const int top = min(count + back, p.n_pages);
    // tails: the page in whose middle a request ends
    int32_t* const tail = take;                           // (no longer needed)
    for (int r = tid; r < R; r += T) {
        const int len = next[r];
        int page = -1;
        if (len & ((1 << shift) - 1)) {
            page = p.table[(long)r * p.blocks + (len >> shift)];
            if (!ok_page(page)) page = -1;
        }
        tail[r] = page;
    }
    __syncthreads();
    int copies = 0, granted = 0;
    for (int r0 = 0; r0 < R; r0 += T) {
        const int r = r0 + tid;
        const int page = r < R ? tail[r] : -1;
        bool copy = false;
        if (page >= 0) {
            const int holders = count_of(&p.shares[page]) + 1;
            if (holders > 1) {
                int ends = 0, best = 2 * MAX;
                for (int k = 0; k < R; ++k)
                    if (tail[k] == page) { ++ends; best = min(best, from[k] == k ? k : MAX + k); }
                copy = holders > ends || best != (from[r] == r ? r : MAX + r);
            }
        }
        int total;
        const int at = copies + scan(copy, total);
        const bool got = copy && at < top;
        if (r < R) {
            const int len = next[r];
            p.lens_out[r] = have[r] < 0 || have[r] > most ? have[r] : copy && !got ? len & -(1 << shift) : len;
        }
        if (copy) leave[r] = got ? at : -2 - at;          // (no longer needed: which copy it is, counted over the requests)
        else if (r < R) leave[r] = -1;
        copies += total;
    }
    __syncthreads();                                      // (all counts have been read)
    granted = min(copies, top);
    for (int r = tid; r < R; r += T) {
        const int at = leave[r];
        if (at == -1) continue;
        count_add(&p.shares[tail[r]], -1);
        if (at < 0) continue;                             // no page left: the request ends before its tail
        const int to = p.free_pages[top - 1 - at];
        if (!ok_page(to)) { atomicAdd(&strange, 1); }
        p.table[(long)r * p.blocks + (next[r] >> shift)] = to;
        *(i32x2*)(p.moves + 2 * at) = i32x2{tail[r], to};
    }
    for (int i = granted + tid; i < R; i += T) *(i32x2*)(p.moves + 2 * i) = i32x2{-1, -1};
    __syncthreads();
    if (tid == 0) {
        *p.free_count = top - granted;
        p.status[0] = granted; p.status[1] = copies - granted; p.status[2] = invalid; p.status[3] = strange;
    }
}

// ---- compaction -----------------------------------------------------------------------------------------------------
// Of n_pages, `used` are not on the stack of free ones.  The i-th free page below `used` (a hole) takes what the i-th page in use from
// `used` on holds; there are as many of one as of the other.  A bit per page, set for the free ones, and the number of set bits in
// front of each word give either's rank.
// Four launches: bits cleared and set, words summed (one work-group), ranks turned into moves and the tables rewritten.  Bound: latency of the launches.

constexpr int COMPACT_THREADS = 256;

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

__global__ __launch_bounds__(COMPACT_THREADS) void compact_clear_kernel(CompactParams p) {
    const int i = blockIdx.x * COMPACT_THREADS + threadIdx.x;
    if (i <= p.words) p.bits[i] = 0u;
    if (i < 4) p.status[i] = 0;
}
__global__ __launch_bounds__(COMPACT_THREADS) void compact_mark_kernel(CompactParams p) {
    const int i = blockIdx.x * COMPACT_THREADS + threadIdx.x;
    if (i >= compact_free(p)) return;
    const int page = p.free_pages[i];
    const bool fresh = (unsigned)page < (unsigned)p.n_pages && !(atomicOr(&p.bits[page >> 5], 1u << (page & 31)) >> (page & 31) & 1u);
    if (!fresh) atomicAdd(&p.status[3], 1);               // (out of range, or on the stack twice)
}
__global__ __launch_bounds__(1024) void compact_sum_kernel(CompactParams p) {
    constexpr int T = 1024, NW = T / 64, U = 8;
    __shared__ int sums[2][NW];
    int at = 0, turn = 0;
    for (int w0 = 0; w0 <= p.words; w0 += T * U) {
        int n[U], mine = 0, total;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int w = w0 + threadIdx.x * U + u;
            n[u] = w < p.words ? __popc(p.bits[w]) : 0;
            mine += n[u];
        }
        turn ^= 1;
        int first = at + group_scan<NW>(mine, sums, turn, total);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int w = w0 + threadIdx.x * U + u;
            if (w <= p.words) p.before[w] = first;
            first += n[u];
        }
        at += total;
    }
}
__global__ __launch_bounds__(COMPACT_THREADS) void compact_holes_kernel(CompactParams p) {
    const int page = blockIdx.x * COMPACT_THREADS + threadIdx.x;
    const int used = p.n_pages - p.before[p.words];
    if (page >= used || !bit_of(p, page)) return;
    p.holes[free_before(p, page)] = page;
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
        const int page = (int)id, holes = used < p.n_pages ? free_before(p, used) : 0, free = p.before[p.words];
        if (page < p.n_pages / 2 && page >= holes) *(i32x2*)(p.moves + 2 * page) = i32x2{-1, -1};
        p.free_out[page] = page < free ? p.n_pages - 1 - page : p.free_pages[page];
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
        if (page == 0) { p.status[0] = holes; p.status[1] = used; }
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
// loads of 16 bytes a thread on their way together.

constexpr int COPY_U = 4, COPY_PIECE = 256 * COPY_U;      // of 16 bytes

__global__ __launch_bounds__(256) void cache_copy_kernel(const i32x4* src, i32x4* dst, const int32_t* moves, const int32_t* count, int most,
                                                         int units, int src_pages, int dst_pages) {
    const int n = min(max(*count, 0), most), pieces = (units + COPY_PIECE - 1) / COPY_PIECE;
    const long all = (long)n * pieces;
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
        for (int u = 0; u < COPY_U; ++u) { const int k = piece * COPY_PIECE + u * 256 + threadIdx.x; if (k < units) b[k] = v[u]; }
    }
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
    return 2 * round256((size_t)R * max_blocks * 4);
}

int entmax_attn_cache_fork(const int32_t* lens, const int32_t* parents, const int32_t* new_lens, int32_t* block_table, int32_t* free_pages,
                           int32_t* free_count, int32_t* shares, int32_t* lens_out, int32_t* moves, int32_t* status,
                           int R, int max_blocks, int page_size, int n_pages, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!lens || !parents || !new_lens || !block_table || !free_pages || !free_count || !shares || !lens_out || !moves || !status) return EA_ERR_NULL;
    if (!tables_shape_ok(R, max_blocks, page_size, n_pages)) return EA_ERR_SHAPE;
    if (lens_out == new_lens || lens_out == parents || ((uintptr_t)moves & 7)) return EA_ERR_LAYOUT;
    if (!workspace_ok(workspace, workspace_bytes, entmax_attn_cache_fork_workspace_bytes(R, max_blocks))) return EA_ERR_WORKSPACE;
    ForkParams p{lens, parents, new_lens, block_table, free_pages, free_count, shares, lens_out, moves, status,
                 (int32_t*)workspace, (int32_t*)((char*)workspace + round256((size_t)R * max_blocks * 4)), R, max_blocks, cache_page_shift(page_size), n_pages};
    hipLaunchKernelGGL(cache_fork_kernel, dim3(1), dim3(FORK_THREADS), 0, (hipStream_t)hip_stream, p);
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
    auto groups = [](long n) { return dim3((unsigned int)((n + COMPACT_THREADS - 1) / COMPACT_THREADS)); };
    const dim3 block(COMPACT_THREADS);
    hipLaunchKernelGGL(compact_clear_kernel, groups(p.words + 4), block, 0, s, p);
    hipLaunchKernelGGL(compact_mark_kernel, groups(n_pages), block, 0, s, p);
    hipLaunchKernelGGL(compact_sum_kernel, dim3(1), dim3(1024), 0, s, p);
    hipLaunchKernelGGL(compact_holes_kernel, groups(n_pages), block, 0, s, p);
    hipLaunchKernelGGL(compact_move_kernel, groups(n_pages + (long)R * max_blocks), block, 0, s, p);
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
