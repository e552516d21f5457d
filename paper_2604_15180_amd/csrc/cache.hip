// The paged caches of a serving program: block tables and slots made on the GPU, rows written to their slots and
// read back (layouts: cache4.hpp, cache8.hpp).
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "cache4.hpp"
#include "cache8.hpp"
#include "common.hpp"
#include "launch.hpp"

namespace ea {

// ---- block tables ---------------------------------------------------------------------------------------------------
// One step of a scheduler: request r goes from lens[r] cached tokens to new_lens[r].  Pages that shrinking requests leave
// go back to the top of the stack of free pages, the last request's last page first; growing requests then take theirs
// from its top in their order.  A step taken back thus leaves the stack as it was.
// Three prefix sums over the requests (pages left, pages wanted, new tokens) turn the work into independent items - a
// page, a token row - that find their request by bisection.  Bound: latency, of the chain lengths -> sums -> stack ->
// table -> slots; one work-group does all of it, so that its steps are a barrier apart and not a launch; the rows of a
// long prompt are left to a second kernel.  64 requests with a token each: 3.7 us; 1000 requests of which 150 end, start or go
// back, with 61000 rows: 10.2 and 3.6 us (four pages a thread at once: 11.5).

constexpr int TABLE_MAX_REQUESTS = 4096;
constexpr int TABLE_SLOTS_THREADS = 1024;
constexpr int TABLE_ROWS_INSIDE = 4096;         // token rows up to which the work-group of the tables makes the slots as well

struct TableParams {
    const int32_t* lens; const int32_t* new_lens;
    int32_t* table;            // [R][blocks]
    int32_t* free_pages;       // [n_pages]
    int32_t* free_count;       // [1]
    int32_t* lens_out;         // [R]
    int32_t* start;            // [R + 1]
    int32_t* slots; int32_t* positions;     // [rows]
    int32_t* status;           // [4]
    int R, blocks, page_shift, n_pages, rows;
};

// position and slot of token row t of request r (the table is final)
EA_DEV void table_row(const TableParams& p, int t, int r, int start, int end, bool granted) {
    const int position = p.new_lens[r] - (end - start) + (t - start);
    int slot = -1;
    if (granted) {
        const int page = p.table[(long)r * p.blocks + (position >> p.page_shift)];
        if ((unsigned)page < (unsigned)p.n_pages) slot = (page << p.page_shift) + (position & ((1 << p.page_shift) - 1));
    }
    p.slots[t] = slot;
    p.positions[t] = position;
}

__global__ __launch_bounds__(1024) void cache_tables_kernel(TableParams p) {
    constexpr int T = 1024, NW = T / 64;
    __shared__ int32_t left[TABLE_MAX_REQUESTS + 1], want[TABLE_MAX_REQUESTS + 1], start[TABLE_MAX_REQUESTS + 1];   // exclusive prefix sums
    __shared__ int32_t wsum[NW][4];
    __shared__ int refused, invalid, strange, given;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, R = p.R;
    const int most = p.blocks << p.page_shift;           // (at most 2^22)
    const int count = min(max(*p.free_count, 0), p.n_pages);
    if (tid == 0) { refused = invalid = strange = given = 0; left[0] = want[0] = start[0] = 0; }
    // a request whose lengths are out of range takes part in nothing
    auto lengths = [&](int r, int& a, int& b) {
        a = p.lens[r]; b = p.new_lens[r];
        const bool ok = a >= 0 && b >= 0 && a <= most && b <= most;
        if (!ok) a = b = 0;
        return ok;
    };
    int a = 0, b = 0;                                     // of the thread's last request
    bool ok = true;
    long long tokens = 0;
    int back = 0, wanted = 0;
    for (int r0 = 0; r0 < R; r0 += T) {
        const int r = r0 + tid;
        a = b = 0;
        ok = r >= R || lengths(r, a, b);
        const int have = pages_of(a, p.page_shift), need = pages_of(b, p.page_shift);
        // sums over a wave: pages below 2^24, tokens below 2^28
        int v[3] = {wave_scan(max(have - need, 0)), wave_scan(max(need - have, 0)), wave_scan(max(b - a, 0))};
        __syncthreads();                                  // (of the round before: the sums have been read)
        if (lane == 63) { wsum[wave][0] = v[0]; wsum[wave][1] = v[1]; wsum[wave][2] = v[2]; }
        if (!ok) atomicAdd(&invalid, 1);
        __syncthreads();
        long long at = tokens + v[2];
        v[0] += back; v[1] += wanted;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int s0 = wsum[w][0], s1 = wsum[w][1], s2 = wsum[w][2];
            if (w < wave) { v[0] += s0; v[1] += s1; at += s2; }
            back += s0; wanted += s1; tokens += s2;
        }
        // (tokens: what does not fit 31 bits fits no list of rows either)
        if (r < R) { left[r + 1] = v[0]; want[r + 1] = v[1]; start[r + 1] = (int)min(at, (long long)INT_MAX); }
    }
    __syncthreads();
    const int top = min(count + back, p.n_pages);
    // request r is granted what it wants (both conditions only grow with r: the requests that get pages are the first that want any)
    auto granted = [&](int r, bool grows) { return (want[r + 1] == want[r] || want[r + 1] <= top) && (!grows || start[r + 1] <= p.rows); };
    for (int r = tid; r < R; r += T) {
        if (R > T) ok = lengths(r, a, b);                 // (else still there)
        const bool fits = granted(r, b > a);
        if (!fits) atomicAdd(&refused, 1);
        else if (want[r + 1] > want[r]) atomicMax(&given, want[r + 1]);
        p.start[r + 1] = start[r + 1];
        p.lens_out[r] = !ok ? p.lens[r] : fits ? b : a;   // (lens may be lens_out: each thread reads its own)
    }
    if (tid == 0) p.start[0] = 0;
    for (int i = tid; i < back; i += T) {
        const int r = owner(left, R, i);
        const int k = pages_of(p.new_lens[r], p.page_shift) + (i - left[r]);
        const int at = count + (back - 1 - i), page = p.table[(long)r * p.blocks + k];
        if (at < p.n_pages) p.free_pages[at] = page;
        if (at >= p.n_pages || (unsigned)page >= (unsigned)p.n_pages) atomicAdd(&strange, 1);
    }
    __syncthreads();
    const int g = given;
    for (int i = tid; i < g; i += T) {
        const int r = owner(want, R, i);
        const int page = p.free_pages[top - 1 - i];
        const int old = p.new_lens[r] - (start[r + 1] - start[r]);
        if ((unsigned)page >= (unsigned)p.n_pages) atomicAdd(&strange, 1);
        p.table[(long)r * p.blocks + pages_of(old, p.page_shift) + (i - want[r])] = page;
    }
    if (tid == 0) *p.free_count = top - g;
    __syncthreads();
    if (tid == 0) { p.status[0] = min(start[R], p.rows); p.status[1] = refused; p.status[2] = invalid; p.status[3] = strange; }
    if (p.rows > TABLE_ROWS_INSIDE) return;               // (cache_slots_kernel)
    for (int t = tid; t < p.rows; t += T) {
        if (t < start[R]) { const int r = owner(start, R, t); table_row(p, t, r, start[r], start[r + 1], granted(r, true)); }
        else { p.slots[t] = -1; p.positions[t] = 0; }
    }
}

// (the starts are copied to LDS first: searched in global memory each step is a round trip to the L2, 4.5 us in place of 3.6 for
// 61000 rows of 1000 requests)
__global__ __launch_bounds__(TABLE_SLOTS_THREADS) void cache_slots_kernel(TableParams p) {
    constexpr int T = TABLE_SLOTS_THREADS;
    __shared__ int32_t start[TABLE_MAX_REQUESTS + 1];
    for (int r = threadIdx.x; r <= p.R; r += T) start[r] = p.start[r];
    __syncthreads();
    const int t = blockIdx.x * T + threadIdx.x;
    if (t >= p.rows) return;
    if (t < start[p.R]) {
        const int r = owner(start, p.R, t);
        table_row(p, t, r, start[r], start[r + 1], p.lens_out[r] == p.new_lens[r]);
    } else { p.slots[t] = -1; p.positions[t] = 0; }
}

// ---- rows in 4 bits -------------------------------------------------------------------------------------------------
// A block of 32 values is four lanes with eight each.  Scale 2^s with s = floor(log2 max|x|) - 2, one more where
// max|x| > 7 * 2^s: then no value is further from its level than half the distance of two levels, 6 and the
// next power of two among them (with s alone, values up to 8 * 2^s would be cut to 6 * 2^s).  The scale is a power of two, so
// x / 2^s is exact and the rounding to a level, ties to the even code, is the only one.
// Bound: HBM, 2 bytes (bf16) and 17/32 byte a value: 16001 tokens of 16 rows of 128 values are written in 17.2 us and read back in
// 17.0, 4.9 TB/s of reads and writes together (one item a thread: 18.0 and 19.5; 64 tokens 2.8 us, with four items a thread 4.1).

struct RowParams {
    const void* src[2]; void* dst[2];       // K, V (write: src, read: dst), strides st
    long st[2][2];                          // token, head
    unsigned char* cache;
    const int32_t* slots;
    int T, Hk, page_shift, n_pages;
};

constexpr unsigned int ROWS_MANY = 1u << 18;       // items from which a thread takes four (1024 work-groups of single ones)

// An item is eight neighbouring values of a row; items of a token follow each other (K's heads, then V's).  Of a large batch each
// thread takes U, a work-group's width apart, so that their loads are on their way together.
struct RowItem { int t, which, h, sub, slot; bool on; };
template <int D> EA_DEV RowItem row_item(const RowParams& p, unsigned int item, unsigned int items) {
    constexpr unsigned int LPR = D / 8;
    RowItem r;
    const unsigned int id = min(item, items - 1) / LPR, per = 2u * p.Hk;
    r.sub = (int)(item % LPR);
    r.t = (int)(id / per);
    const int i = (int)(id - r.t * per);
    r.which = i >= p.Hk;
    r.h = i - (r.which ? p.Hk : 0);
    r.slot = p.slots[r.t];
    r.on = item < items && r.slot >= 0 && (r.slot >> p.page_shift) < p.n_pages;
    return r;
}
// Where the item's codes and its scale byte lie (the first page's for an item that takes no part)
template <int D> EA_DEV void row_place(const RowParams& p, const RowItem& r, unsigned char*& codes, unsigned char*& scale) {
    const int slot = r.on ? r.slot : 0;
    const int row = slot & ((1 << p.page_shift) - 1);
    const long head = (long)(slot >> p.page_shift) * p.Hk + r.h;
    unsigned char* const base = p.cache + ((head * (2 * (D / 2 + D / 32)) + r.which * (D / 2 + D / 32)) << p.page_shift);
    codes = base + row * (D / 2) + 4 * r.sub;
    scale = base + ((D / 2) << p.page_shift) + row * (D / 32) + (r.sub >> 2);
}

template <class E, int D, int U>
__global__ __launch_bounds__(256) void cache4_write_kernel(RowParams p, unsigned int items) {
    using elem = typename E::elem;
    typedef elem vec __attribute__((ext_vector_type(8)));
    const unsigned int first = blockIdx.x * (256u * U) + threadIdx.x;
    RowItem r[U];
    vec x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = row_item<D>(p, first + 256u * u, items);
#pragma unroll
    for (int u = 0; u < U; ++u)
        x[u] = *(const vec*)((const elem*)p.src[r[u].which] + r[u].t * p.st[r[u].which][0] + r[u].h * p.st[r[u].which][1] + 8 * r[u].sub);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        // magnitudes as integers: they order like the values, and infinities and NaN stay above all others
        unsigned int top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint((float)x[u][e]) & 0x7fffffffu);
        top = max(top, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));     // over the block's four lanes
        top = max(top, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));
        int byte = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u);                // (7 * 2^s has the fraction 0.75)
        byte = min(max(byte, 1), 252);
        const float scale = __uint_as_float((unsigned int)byte << 23);
        unsigned int codes = 0;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, (float)x[u][0], (float)x[u][1], scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, (float)x[u][2], (float)x[u][3], scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, (float)x[u][4], (float)x[u][5], scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, (float)x[u][6], (float)x[u][7], scale, 3);
        if (top >= 0x7f800000u) { byte = 255; codes = 0; }
        unsigned char *to, *to_scale;
        row_place<D>(p, r[u], to, to_scale);
        if (r[u].on) {
            *(unsigned int*)to = codes;
            if ((r[u].sub & 3) == 0) *to_scale = (unsigned char)byte;
        }
    }
}

template <class E, int D, int U>
__global__ __launch_bounds__(256) void cache4_read_kernel(RowParams p, unsigned int items) {
    using elem = typename E::elem;
    typedef elem vec __attribute__((ext_vector_type(8)));
    const unsigned int first = blockIdx.x * (256u * U) + threadIdx.x;
    RowItem r[U];
    unsigned int codes[U], byte[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = row_item<D>(p, first + 256u * u, items);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        unsigned char *from, *from_scale;
        row_place<D>(p, r[u], from, from_scale);
        codes[u] = *(const unsigned int*)from;
        byte[u] = *from_scale;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float scale = cache4_scale(byte[u]);
        const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 1);
        const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 3);
        const float v[8] = {v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
        vec y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (elem)(v[e] * scale);
        if (r[u].on) *(vec*)((elem*)p.dst[r[u].which] + r[u].t * p.st[r[u].which][0] + r[u].h * p.st[r[u].which][1] + 8 * r[u].sub) = y;
    }
}

// ---- rows in 8 bits -------------------------------------------------------------------------------------------------
// A block is 16 tokens of a head's keys or values with one scale s = max|x| / 127, rounded to float32; a code is the integer nearest to
// x / s, ties to the even one.  Rows are appended: those of a call that stand next to each other and go to one block are one run, which a wave
// takes as a whole for one head's keys or values.  The rows in front of a run's first keep their codes, unless the run's own scale is
// larger than the block's: then it becomes the block's, and they are rounded once more.  A run that begins with row 0
// begins its block.
// Bound: HBM for a prompt: 16001 tokens of 16 rows of 128 values are written in 22.2 us, 4.4 TB/s of reads and writes together, and read back in 18.5,
// 5.3 TB/s; 64 tokens 4.5 and 3.2 us, chains slots -> rows, scale and kept codes -> codes.
// The nearest integer n is that of x times 1 / s, which is off by up to 2^-16; the remainder x - n s, exact in one fused
// multiply-add, then tells whether n is the one (halves are exact, too).  It hardly ever is not, nor is a value: both are looked at
// for all of a lane's values at once, and put right in a branch of their own.  Kept codes: c s_old = p + e with two floats, and
// likewise.

// Tokens whose runs a wave looks after: 1 up to C8_FEW (tokens x heads of keys and values), 4 up to C8_MANY, 16 above.  One each keeps the
// waves short, but of a prompt's only each sixteenth finds a run.  us with 1 / 4 / 16 tokens, 8 key heads of 128: 1400 requests with a token each
// (22400) 16.7 / 16.2 / 25.3, 4000 (64000) 47.3 / 38.6 / 40.0; 8 chunks of 512 (50000) 22.0 / 13.4 / 10.4; chunks of 127, 5 heads of 64 (23000)
// 7.4 / 6.0 / 6.0.  Around C8_FEW, 1 / 4: 8 key heads of 128, requests with a token each, 128 (2048) 4.3 / 7.2, 256 (4096) 5.0 / 7.8, 512 (8192) 7.6 / 8.8, 1024 (16384)
// 11.8 / 11.7; one chunk of as many tokens 6.8 / 6.2, 7.9 / 6.4, 8.7 / 7.0 and 12.9 / 8.6: at 4096 tokens apart gain more than a chunk loses, at 8192 less.
constexpr int C8_FEW = 1 << 12, C8_MANY = 1 << 15;

// The float whose lowest byte is the nearest integer to x * inv, |x * inv| < 2^22; less C8_MAGIC it is that integer
constexpr float C8_MAGIC = 12582912.f;          // 1.5 * 2^23
EA_DEV float c8_near(float x, float inv) { return fmaf(x, inv, C8_MAGIC); }
// The lowest bytes of four, in order
EA_DEV unsigned int c8_bytes(const float* m) {
    const unsigned int lo = __builtin_amdgcn_perm(__float_as_uint(m[1]), __float_as_uint(m[0]), 0x0c0c0400u);
    const unsigned int hi = __builtin_amdgcn_perm(__float_as_uint(m[3]), __float_as_uint(m[2]), 0x0c0c0400u);
    return hi << 16 | lo;
}
// n, an integer one of the two next to x / s, where x = p + e (e far below s): the nearest, ties to the even one
EA_DEV float c8_put_right(float n, float p, float e, float s) {
    const float rest = fmaf(-n, s, p), side = copysignf(1.f, rest);
    // 2 |x - n s| - s: both sums are exact next to zero and have the right sign elsewhere
    const float over = fmaf(2.f * side, e, 2.f * fabsf(rest) - s);
    if (over > 0.f || (over == 0.f && ((int)n & 1))) n += side;
    return fminf(fmaxf(n, -127.f), 127.f);
}

template <class E, int D, int ROWS>
__global__ __launch_bounds__(256) void cache8_write_kernel(RowParams p, unsigned int waves) {
    using elem = typename E::elem;
    typedef elem vec __attribute__((ext_vector_type(8)));
    constexpr int LPR = D / 8, AT_ONCE = 64 / LPR, STEPS = C8_BLOCK / AT_ONCE;
    const unsigned int id = blockIdx.x * 4u + (unsigned int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per = 2u * p.Hk;
    if (id >= waves) return;
    const int lane = threadIdx.x & 63, sub = lane % LPR, rsel = lane / LPR;
    const int t0 = (int)(id / per) * ROWS, which = id % per >= (unsigned int)p.Hk, h = (int)(id % per) - (which ? p.Hk : 0);
    // lane k: row t0 + k.  Runs begin where the block changes (or the call does).
    const int shift = p.page_shift, t = t0 + lane;
    auto slot_of = [&](int row) {
        const int slot = row >= 0 && row < p.T ? p.slots[row] : -1;
        return slot >= 0 && (slot >> shift) < p.n_pages ? slot : -1;
    };
    const int slot = lane <= ROWS + C8_BLOCK ? slot_of(t) : -1;
    const int before = __shfl_up(slot, 1), at_first = t0 > 0 ? slot_of(t0 - 1) : -1;
    const unsigned long long changes = __ballot((lane == 0 ? at_first : before) >> 4 != slot >> 4);     // (-1 >> 4 is no block)
    unsigned long long todo = changes & __ballot(slot >= 0 && lane < ROWS);
    const elem* const src = (const elem*)p.src[which] + h * p.st[which][1] + 8 * sub;
    while (todo) {
        const int r0 = __ffsll((long long)todo) - 1;
        todo &= todo - 1;
        const unsigned long long behind = changes >> r0 >> 1;
        const int rows = min(behind ? __ffsll((long long)behind) : 64, C8_BLOCK);           // of this run (more: slots that differ not)
        vec x[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int k = min(i * AT_ONCE + rsel, rows - 1);                                // (a row once more in place of one that is not there)
            x[i] = *(const vec*)(src + (t0 + r0 + k) * p.st[which][0]);
        }
        const int s0 = __builtin_amdgcn_readlane(slot, r0);
        unsigned char* const part = p.cache + ((long)(s0 >> shift) * p.Hk + h) * cache8_part_bytes(D, shift);
        const int block = (s0 & ((1 << shift) - 1)) / C8_BLOCK;
        float* const scale_at = cache8_scale(part, D, shift, which, block);
        unsigned char* const codes = part + ((which * D) << shift) + block * C8_BLOCK * D + 8 * sub;
        // the lowest of the run's rows in the block, bit by bit
        unsigned long long low = __ballot(lane >= r0 && lane < r0 + rows);
        int first = 0;
#pragma unroll
        for (int bit = 3; bit >= 0; --bit) {
            const unsigned long long zero = __ballot(!(slot >> bit & 1)) & low;
            if (zero) low = zero; else first |= 1 << bit;
        }
        // (asked for with the rows, whether they will be rounded again or not: 64 requests with a token each 1 us less)
        float was = 0.f;
        uint2 kept[STEPS];
        if (first) {
            was = *scale_at;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) kept[i] = *(const uint2*)(codes + min(i * AT_ONCE + rsel, first - 1) * D);
        }
        unsigned int bits = 0;                                                              // (of positive floats order like them)
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) bits = max(bits, __float_as_uint((float)x[i][e]) & 0x7fffffffu);
        bits = (unsigned int)wave_max((int)bits);
        const bool odd = bits >= 0x7f800000u;                                               // some value is not finite
        if (odd) {
            bits = 0;
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned int a = __float_as_uint((float)x[i][e]) & 0x7fffffffu;
                    bits = max(bits, a < 0x7f800000u ? a : 0u);
                }
            bits = (unsigned int)wave_max((int)bits);
        }
        const float old = fabsf(was), need = bits ? fmaxf(__uint_as_float(bits) / 127.f, 0x1p-126f) : 0.f;
        const bool grown = !(old >= need && old < INFINITY), strange = odd || __float_as_uint(was) >> 31;
        const float s = grown ? need : old, inv = s > 0.f ? 1.f / s : 0.f;
        if (grown && first) {
            // (scales below 1 are taken up, so that no part of c s_old is lost where it counts)
            const float up = s < 1.f ? 0x1p60f : 1.f, so = (old < INFINITY ? old : 0.f) * up, sn = s * up, in = 1.f / sn;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (i * AT_ONCE >= first) break;
                const int k = i * AT_ONCE + rsel;
                float m[8], far = 0.f;
                auto code = [&](int e) { return (float)(signed char)((e >> 2 ? kept[i].y : kept[i].x) >> (8 * (e & 3))); };
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    m[e] = c8_near(code(e) * so, in);
                    far = fmaxf(far, fabsf(fmaf(C8_MAGIC - m[e], sn, code(e) * so)));
                }
                // (the products, up to 127 sn, are rounded by up to 2^-17 sn)
                if (__any(2.f * far >= sn * (1.f - 0x1p-14f) || cache8_odd(kept[i].x) || cache8_odd(kept[i].y))) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float c = code(e), q = c * so;
                        m[e] = (c == -128.f ? c : c8_put_right(m[e] - C8_MAGIC, q, fmaf(c, so, -q), sn)) + C8_MAGIC;
                    }
                }
                if (k < first) *(uint2*)(codes + k * D) = uint2{c8_bytes(m), c8_bytes(m + 4)};
            }
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (i * AT_ONCE >= rows) break;
            const int k = i * AT_ONCE + rsel;
            float m[8], far = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m[e] = c8_near((float)x[i][e], inv);
                far = fmaxf(far, fabsf(fmaf(C8_MAGIC - m[e], s, (float)x[i][e])));
            }
            if (odd || __any(2.f * far >= s)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = (float)x[i][e];
                    m[e] = (fabsf(v) < INFINITY ? c8_put_right(m[e] - C8_MAGIC, v, 0.f, s) : -128.f) + C8_MAGIC;
                }
            }
            const int row = __shfl(slot, r0 + min(k, rows - 1)) & (C8_BLOCK - 1);
            if (k < rows) *(uint2*)(codes + row * D) = uint2{c8_bytes(m), c8_bytes(m + 4)};
        }
        if (lane == 0 && (grown || !first || strange)) *scale_at = strange ? -s : s;
    }
}

template <class E, int D, int U>
__global__ __launch_bounds__(256) void cache8_read_kernel(RowParams p, unsigned int items) {
    using elem = typename E::elem;
    typedef elem vec __attribute__((ext_vector_type(8)));
    const unsigned int first = blockIdx.x * (256u * U) + threadIdx.x;
    RowItem r[U];
    uint2 codes[U];
    float scale[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = row_item<D>(p, first + 256u * u, items);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int slot = r[u].on ? r[u].slot : 0, row = slot & ((1 << p.page_shift) - 1);
        const unsigned char* const part = p.cache + ((long)(slot >> p.page_shift) * p.Hk + r[u].h) * cache8_part_bytes(D, p.page_shift);
        codes[u] = *(const uint2*)(part + ((r[u].which * D) << p.page_shift) + row * D + 8 * r[u].sub);
        scale[u] = *cache8_scale(part, D, p.page_shift, r[u].which, row / C8_BLOCK);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float v[8];
        cache8_expand(codes[u], __float_as_uint(scale[u]) >> 31, v);
        vec y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (elem)(v[e] * fabsf(scale[u]));
        if (r[u].on) *(vec*)((elem*)p.dst[r[u].which] + r[u].t * p.st[r[u].which][0] + r[u].h * p.st[r[u].which][1] + 8 * r[u].sub) = y;
    }
}

}  // namespace ea

namespace {
using namespace ea;

bool cache_shape_ok(int Hk, int d, int page, long n_pages) {
    return Hk > 0 && Hk <= 65535 && (d == 64 || d == 128) && cache_page_ok(page) && n_pages > 0 && n_pages * page <= (long)INT_MAX;
}

int rows_check(const void* k, const void* v, const int64_t* ks, const int64_t* vs, const int32_t* slots, const void* cache,
               int T, int Hk, int d, int t, int n_pages, int page, bool writes_rows) {
    if (!cache || !ks || !vs || (T > 0 && (!k || !v || !slots))) return EA_ERR_NULL;
    if (t != EA_F32 && t != EA_BF16) return EA_ERR_DTYPE;
    if (T < 0 || !cache_shape_ok(Hk, d, page, n_pages) || (long)T * 2 * Hk * (d / 8) > 0xffffff00l) return EA_ERR_SHAPE;   // (a launch holds 2^32 threads)
    const int size = t == EA_BF16 ? 2 : 4;
    if (!aligned16(k) || !aligned16(v) || !aligned16(cache)) return EA_ERR_LAYOUT;
    const int64_t* both[2] = {ks, vs};
    for (const int64_t* st : both) {
        if (st[0] < 0 || st[1] < 0 || (st[0] * size) % 16 || (st[1] * size) % 16) return EA_ERR_LAYOUT;
        if (!writes_rows) continue;
        // rows that are written must not overlap
        const int64_t a = st[0], b = st[1];
        const bool ok = (T <= 1 || a >= (b < a && Hk > 1 ? b * (Hk - 1) + d : d)) && (Hk == 1 || b >= (a <= b && T > 1 ? a * (T - 1) + d : d));
        if (!ok) return EA_ERR_LAYOUT;
    }
    return EA_OK;
}

RowParams row_params(void* cache, const int32_t* slots, const int64_t* ks, const int64_t* vs, int T, int Hk, int page, int n_pages) {
    RowParams p{};
    p.cache = (unsigned char*)cache; p.slots = slots;
    for (int i = 0; i < 2; ++i) { p.st[0][i] = ks[i]; p.st[1][i] = vs[i]; }
    p.T = T; p.Hk = Hk; p.page_shift = cache_page_shift(page); p.n_pages = n_pages;
    return p;
}
enum RowsCall { WRITE4, READ4, READ8 };
template <RowsCall CALL, class E, int D, int U> void rows_launch(const RowParams& p, unsigned int items, hipStream_t s) {
    const dim3 grid((unsigned int)(((long)items + 256 * U - 1) / (256 * U)));
    if constexpr (CALL == WRITE4) hipLaunchKernelGGL((cache4_write_kernel<E, D, U>), grid, dim3(256), 0, s, p, items);
    else if constexpr (CALL == READ4) hipLaunchKernelGGL((cache4_read_kernel<E, D, U>), grid, dim3(256), 0, s, p, items);
    else hipLaunchKernelGGL((cache8_read_kernel<E, D, U>), grid, dim3(256), 0, s, p, items);
}
template <RowsCall CALL> int rows_run(const RowParams& p, int d, int dtype, hipStream_t s) {
    const unsigned int items = (unsigned int)((long)p.T * 2 * p.Hk * (d / 8));
    const bool many = items >= ROWS_MANY;
    auto pick = [&](auto e) {
        using E = decltype(e);
        if (d == 64) { if (many) rows_launch<CALL, E, 64, 4>(p, items, s); else rows_launch<CALL, E, 64, 1>(p, items, s); }
        else { if (many) rows_launch<CALL, E, 128, 4>(p, items, s); else rows_launch<CALL, E, 128, 1>(p, items, s); }
    };
    if (dtype == EA_BF16) pick(Bf16{}); else pick(F32{});
    return launched();
}
template <class E, int D, int ROWS> void write8_launch(const RowParams& p, hipStream_t s) {
    const unsigned int waves = (unsigned int)(((long)p.T + ROWS - 1) / ROWS * 2 * p.Hk);
    hipLaunchKernelGGL((cache8_write_kernel<E, D, ROWS>), dim3(waves / 4 + (waves % 4 != 0)), dim3(256), 0, s, p, waves);
}

}  // namespace

extern "C" {

int entmax_attn_cache_tables(const int32_t* lens, const int32_t* new_lens, int32_t* block_table, int32_t* free_pages,
                             int32_t* free_count, int32_t* lens_out, int32_t* token_start, int32_t* slots, int32_t* positions,
                             int32_t* status, int R, int max_blocks, int page_size, int n_pages, int max_tokens, void* hip_stream) {
    if (!lens || !new_lens || !block_table || !free_pages || !free_count || !lens_out || !token_start || !status) return EA_ERR_NULL;
    if (max_tokens > 0 && (!slots || !positions)) return EA_ERR_NULL;
    if (R <= 0 || R > TABLE_MAX_REQUESTS || max_blocks <= 0 || !cache_page_ok(page_size) || n_pages <= 0 || max_tokens < 0 || max_tokens > (1 << 30))
        return EA_ERR_SHAPE;
    if ((long)max_blocks * page_size > (1l << 22) || (long)n_pages * page_size > (long)INT_MAX) return EA_ERR_SHAPE;
    if (lens_out == new_lens) return EA_ERR_LAYOUT;
    TableParams p{lens, new_lens, block_table, free_pages, free_count, lens_out, token_start, slots, positions, status,
                  R, max_blocks, cache_page_shift(page_size), n_pages, max_tokens};
    hipStream_t s = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(cache_tables_kernel, dim3(1), dim3(1024), 0, s, p);
    if (max_tokens > TABLE_ROWS_INSIDE) hipLaunchKernelGGL(cache_slots_kernel, dim3((max_tokens + TABLE_SLOTS_THREADS - 1) / TABLE_SLOTS_THREADS),
                                                           dim3(TABLE_SLOTS_THREADS), 0, s, p);
    return launched();
}

size_t entmax_attn_cache4_page_bytes(int Hk, int d, int page_size) {
    if (!cache_shape_ok(Hk, d, page_size, 1)) return 0;
    return (size_t)Hk * cache_page_bytes(d, page_size);
}

int entmax_attn_cache4_write(const void* K, const void* V, const int64_t* k_strides, const int64_t* v_strides, const int32_t* slots,
                             void* cache, int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream) {
    const int rc = rows_check(K, V, k_strides, v_strides, slots, cache, T, Hk, d, dtype, n_pages, page_size, false);
    if (rc) return rc;
    if (T == 0) return EA_OK;
    RowParams p = row_params(cache, slots, k_strides, v_strides, T, Hk, page_size, n_pages);
    p.src[0] = K; p.src[1] = V;
    return rows_run<WRITE4>(p, d, dtype, (hipStream_t)hip_stream);
}

int entmax_attn_cache4_read(const void* cache, const int32_t* slots, void* K, void* V, const int64_t* k_strides, const int64_t* v_strides,
                            int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream) {
    const int rc = rows_check(K, V, k_strides, v_strides, slots, cache, T, Hk, d, dtype, n_pages, page_size, true);
    if (rc) return rc;
    if (T == 0) return EA_OK;
    RowParams p = row_params(const_cast<void*>(cache), slots, k_strides, v_strides, T, Hk, page_size, n_pages);
    p.dst[0] = K; p.dst[1] = V;
    return rows_run<READ4>(p, d, dtype, (hipStream_t)hip_stream);
}

size_t entmax_attn_cache8_page_bytes(int Hk, int d, int page_size) {
    if (!cache_shape_ok(Hk, d, page_size, 1)) return 0;
    return (size_t)Hk * cache8_part_bytes(d, cache_page_shift(page_size));
}

int entmax_attn_cache8_write(const void* K, const void* V, const int64_t* k_strides, const int64_t* v_strides, const int32_t* slots,
                             void* cache, int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream) {
    const int rc = rows_check(K, V, k_strides, v_strides, slots, cache, T, Hk, d, dtype, n_pages, page_size, false);
    if (rc) return rc;
    if (T == 0) return EA_OK;
    RowParams p = row_params(cache, slots, k_strides, v_strides, T, Hk, page_size, n_pages);
    p.src[0] = K; p.src[1] = V;
    hipStream_t s = (hipStream_t)hip_stream;
    const long heads = (long)T * 2 * Hk;
    auto pick = [&](auto e, auto rows) {
        using E = decltype(e);
        if (d == 64) write8_launch<E, 64, decltype(rows)::value>(p, s); else write8_launch<E, 128, decltype(rows)::value>(p, s);
    };
    auto rows = [&](auto e) {
        if (heads <= C8_FEW) pick(e, std::integral_constant<int, 1>{});
        else if (heads <= C8_MANY) pick(e, std::integral_constant<int, 4>{});
        else pick(e, std::integral_constant<int, 16>{});
    };
    if (dtype == EA_BF16) rows(Bf16{}); else rows(F32{});
    return launched();
}

int entmax_attn_cache8_read(const void* cache, const int32_t* slots, void* K, void* V, const int64_t* k_strides, const int64_t* v_strides,
                            int T, int Hk, int d, int dtype, int n_pages, int page_size, void* hip_stream) {
    const int rc = rows_check(K, V, k_strides, v_strides, slots, cache, T, Hk, d, dtype, n_pages, page_size, true);
    if (rc) return rc;
    if (T == 0) return EA_OK;
    RowParams p = row_params(const_cast<void*>(cache), slots, k_strides, v_strides, T, Hk, page_size, n_pages);
    p.dst[0] = K; p.dst[1] = V;
    return rows_run<READ8>(p, d, dtype, (hipStream_t)hip_stream);
}

}  // extern "C"
