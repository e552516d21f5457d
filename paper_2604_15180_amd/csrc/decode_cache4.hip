// One query per head and request against the paged 4-bit cache (cache4.hpp): entmax_attn_decode for a serving program.
//   cache4_scores_kernel : s_j = <q, k_j> for a part of a request's keys and up to 16 query heads that share a key head, on
//                          the matrix cores: key codes are an operand as they lie in memory, their scale bytes the operand's scales.
//                          By Eq. 5 only scores within sqrt(d) / (alpha - 1) of the head's maximum can be in the support, and
//                          a running maximum is a lower bound of the final one: of each 64 keys the maximum per head is written,
//                          and the scores where one of them is within that window of the largest the wave knows.
//   cache4_entmax_kernel : per head, tau from the scores of the blocks whose maximum is in the window, and o = sum p_j v_j over
//                          the support.
// The queries: q = 2^e (t_0 + 2^-5 t_1 + 2^-10 t_2 + ...) with e4m3 terms t_i up to 2, each the rounding of what the terms before it
// left.  Of each eight neighbouring products the matrix cores keep what lies within 2^-13 of the largest sum of an operand pair's
// exponents (measured: at 2^-14 a product is lost, at any place of the eight; beyond the eight, and for the scales, the sum is fp32's),
// which a small element's last bits would miss.  The terms lie where e4m3 has the same step, 2^-9, for all small values (below 2^-6 its
// values are subnormal): codes are multiples of 1/2 up to 6, exponents go up to 2 + 1, and no product has bits below 2^-10.  A term takes
// five bits off a value's 8 or 24 (four significant ones, and the rest has a sign): four terms hold a bf16 value exactly down to 2^-17
// of the row's largest, and below that to 2^-25 of it, five an fp32 value down to 2^-6 and to 2^-30: less than fp32's own rounding of the
// score.  (Three terms, 2^-12 and 2^-20, were 1 to 3 % faster - one request of 131072 keys 50.8 us, four terms 51.6; 48 requests up to
// 32768 keys 41.6 and 42.5 - but where one channel of the query is 128 times the others the scores were ten times further off than
// in fp32.  Two terms reaching up to 2^8, so with
// smaller last bits beside them, were off by 2e-5 in tau; terms up to 4 by 1e-4 now and then; as they are, the sums are exact up to
// their one rounding for each term.)
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "cache4.hpp"
#include "common.hpp"
#include "launch.hpp"

namespace ea {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int C4_WAVES = 4;             // waves per work-group of the score kernel
constexpr int C4_BLOCK = 64;            // keys per maximum
constexpr int C4_MAX_PART = 512;        // keys per wave of the score kernel, at most

struct Cache4Params {
    const void* q; const unsigned char* cache; const int32_t* table; const int32_t* lens;
    float* O; float* tau; int32_t* support;
    float* scores;            // [R][Hq][stride]: s_j, where a block's maximum was in the window (else whatever stood there)
    float* bmax;              // [R][Hq][stride / 64]: maximum of 64 keys; +inf also where a score is not a number or a page id out of range
    long stride;              // keys a head has room for (cache4_stride)
    int part;                 // keys per wave of the score kernel, a multiple of 64
    int R, Hq, Hk, G, colgroups;        // G = Hq / Hk query heads per key head, in colgroups of up to 16
    int blocks, n_pages, page_shift, max_len;
    float c;                  // (alpha - 1) / sqrt(d)
    double c64;
    float alpha, r, win;      // win: the window of Eq. 5 in units of s, slightly widened
};

// sums and maxima over lanes by ALU instructions: in a chain of exchanges through LDS each waits for the one before (the entmax
// kernel for one request of 1000 keys and 32 heads 8.9 us with them, 7.3 without)
template <int CTRL> EA_DEV float dpp_move(float v) { return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false)); }
EA_DEV float across16(float v) {        // over the lanes n, n + 16, n + 32, n + 48
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
EA_DEV float across16_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
EA_DEV float whole_wave_max(float v) {
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    return across16_max(fmaxf(v, dpp_move<0x140>(v)));
}
EA_DEV float whole_wave_sum(float v) { return across16(group_sum<16>(v)); }

// Terms of the row's values as operand registers of the 16x16x128 instruction: lane (n, g) = (lane % 16, lane / 16) supplies,
// of column n, the contraction indices 16 g .. 16 g + 15 and 64 + 16 g .. in the e4m3 format (D = 64: both the same; a 4-bit operand:
// 32 g .. 32 g + 31, whose scale byte is the lane's own; the scale of a column's block b is that of lane (n, b)).
template <int NT> struct QTerms { i32x8 t[NT]; int scale[NT]; };   // scale: bytes

// What a lane reads of its head's row: a wave's quarter of the sixteen elements of each 64.
template <class E, int D> struct QRow {
    using elem = typename E::elem;
    typedef elem vec __attribute__((ext_vector_type(4)));
    vec v[D / 64];
    EA_DEV void load(const void* q, long head, bool live, int wave) {
        const int g = __lane_id() >> 4;
#pragma unroll
        for (int run = 0; run < D / 64; ++run) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[run][e] = (elem)0.f;
            if (live) v[run] = *(const vec*)((const elem*)q + head * D + 64 * run + 16 * g + 4 * wave);
        }
    }
};
// The waves of a work-group convert their quarters and hand them round through LDS.  Every thread calls this.  Returns the scale byte
// of keys from which a score of the lane's row may pass 2^120; odd: that row holds an infinity or a NaN.
template <class E, int D, int NT>
EA_DEV int query_terms(const QRow<E, D>& row, int wave, int (*words)[8][64], float (*tops)[16], QTerms<NT>& out, bool& odd) {
    constexpr int RUNS = D / 64;
    const int lane = __lane_id();
    float top = 0.f, x[RUNS][4];
#pragma unroll
    for (int run = 0; run < RUNS; ++run)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[run][e] = (float)row.v[run][e];
            const float a = fabsf(x[run][e]);
            top = a < INFINITY ? fmaxf(top, a) : INFINITY;             // (a NaN counts as infinite)
        }
    top = across16_max(top);
    if (lane < 16) tops[wave][lane] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0][lane & 15], tops[1][lane & 15]), fmaxf(tops[2][lane & 15], tops[3][lane & 15]));
    // the largest value below 2; rows below 2^-100 lose what is below that
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 127);
#pragma unroll
    for (int run = 0; run < RUNS; ++run) {
        float* v = x[run];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ldexpf(v[i], -e);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            int bits = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
            bits = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], bits, true);
            words[t][4 * run + wave][lane] = bits;
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(bits, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(bits, true);
            v[0] = (v[0] - lo[0]) * 32.f; v[1] = (v[1] - lo[1]) * 32.f;
            v[2] = (v[2] - hi[0]) * 32.f; v[3] = (v[3] - hi[1]) * 32.f;
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        out.scale[t] = 127 + e - 5 * t;
#pragma unroll
        for (int w = 0; w < 8; ++w) out.t[t][w] = words[t][RUNS == 1 ? w & 3 : w][lane];
    }
    // |score| < D * 6 * 2^(byte - 127) * 2^(1 + e) <= 2^(byte - 116 + e)
    odd = !(top < INFINITY);
    return odd ? 255 : min(255, 236 - e);
}

EA_DEV unsigned int c4_ordered(float f) {
    const unsigned int u = __float_as_uint(f);
    return (u & 0x80000000u) ? ~u : (u ^ 0x80000000u);
}
EA_DEV float c4_from_ordered(unsigned int u) { return __uint_as_float((u & 0x80000000u) ? (u ^ 0x80000000u) : ~u); }

// Tiles: at D = 128 sixteen keys, one instruction per term; at D = 64 two sets of sixteen keys, the lower half of the lanes
// (contraction indices 0 .. 63 of the operand) one, the upper half the other.  Then (PAIR) up to eight query heads stand in columns 0 .. 7
// with their terms in the lower indices, for the first set, and once more in columns 8 .. 15 in the upper ones, for the second,
// with zeros elsewhere: both sets in one instruction per term.  More heads have their terms in both halves, and the keys are worked on
// one set at a time, with zeros in place of the other's (32 heads x 131072 keys, one head a key head: 38 us, PAIR 32; fp32 queries 40 and 32).
// Result: lane (n, g) holds column n's scores with keys 4 g .. 4 g + 3 of a set.  A wave keeps two blocks of 64 keys on their way: as soon as
// the matrix cores have taken a tile, the same tile of the block after the next is requested.  The addresses of all its keys are
// formed at once, a lane for each sixteen.
template <class E, int D, bool PAIR>
__global__ __launch_bounds__(64 * C4_WAVES) void cache4_scores_kernel(Cache4Params p) {
    constexpr int NT = sizeof(typename E::elem) == 2 ? 4 : 5, SETS = 128 / D, TK = 16 * SETS, U = C4_BLOCK / TK;
    constexpr int PASSES = PAIR ? 1 : SETS, COLS = PAIR ? 8 : 16;         // instructions of a tile and term; query heads side by side
    static_assert(!PAIR || SETS == 2, "two sets to a tile");
    constexpr int ROW = D / 2, SROW = D / 32;
    __shared__ unsigned int smax[16];                       // ordered bits of the work-group's running maxima
    __shared__ int words[NT][8][64];
    __shared__ float tops[C4_WAVES][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4, col = n % COLS;
    const int set0 = PAIR ? n / COLS : 0;                   // the set the lane's column is for
    // Short requests have few parts, and the work-groups that find nothing to do must not fall on some of the XCDs, or some of the 32
    // CUs of each, to which consecutive work-groups are dealt in turn.  So the part is the slowest index (as the fastest one 48
    // requests of 64 .. 32768 tokens took 98 us in place of 50: all their first parts stood on one XCD), and the requests move
    // on by one CU from part to part (50 -> 41 us).
    const int kvh = blockIdx.x / p.colgroups, cg = blockIdx.x - kvh * p.colgroups, chunk = blockIdx.z;
    const int req = (int)((blockIdx.y + (unsigned int)((p.R - 1) & 31) * chunk) % (unsigned int)p.R);
    const int shift = p.page_shift, in_page = (1 << shift) - 1;
    // the waves take the work-group's blocks in turn, so that a request shorter than its part of the keys is all four waves' work
    const int c0 = chunk * C4_WAVES * p.part;
    auto block_key = [&](int i) { return c0 + (i * C4_WAVES + wave) * C4_BLOCK; };        // first key of the wave's block i
    const bool live = cg * 16 + col < p.G;                  // (else a column without a head: zeros, nothing is written)
    const long head = (long)req * p.Hq + kvh * p.G + (live ? cg * 16 + col : 0);
    // length, pages and query are asked for together, and the first keys before the query is worked on.  Lane 4 i + j: the sixteen
    // keys j of block i (C4_MAX_PART: at most eight blocks).
    const int len = p.lens[req];
    const int key16 = block_key(lane >> 2) + 16 * (lane & 3);
    int id = p.table[(long)req * p.blocks + min(key16 >> shift, p.blocks - 1)];
    QRow<E, D> qrow;
    qrow.load(p.q, head, live, wave);
    if (len < 0 || len > p.max_len || c0 >= len) return;
    const int k1 = min(len, c0 + C4_WAVES * p.part);
    const int mine = ((k1 - c0 + C4_BLOCK - 1) / C4_BLOCK - wave + C4_WAVES - 1) / C4_WAVES;       // the wave's blocks
    if (threadIdx.x < 16) smax[threadIdx.x] = c4_ordered(-INFINITY);
    const bool strange = (unsigned)id >= (unsigned)p.n_pages;
    const bool bad = __any(strange && key16 < k1);
    if (strange) id = 0;
    const long page_bytes = (long)(2 * (ROW + SROW)) << shift;
    const unsigned char* const page = p.cache + ((long)id * p.Hk + kvh) * page_bytes;
    const uint64_t rows16 = (uint64_t)(page + (key16 & in_page) * ROW), scales16 = (uint64_t)(page + (ROW << shift) + (key16 & in_page) * SROW);
    float* const scores = p.scores + head * p.stride;
    float* const bmax = p.bmax + head * (p.stride / C4_BLOCK);
    // what the lane loads of sixteen rows
    const unsigned int lrow = n * ROW + 16 * (SETS == 2 ? g & 1 : g), lsrow = n * SROW + (SETS == 2 ? g & 1 : g);
    struct Batch { i32x4 a[U]; int sc[U]; };
    typedef const unsigned char __attribute__((address_space(1)))* global_bytes;       // (a pointer from two integers is not known to be global)
    typedef const i32x4 __attribute__((address_space(1)))* global_codes;
    auto from_lane = [](uint64_t v, int l) {
        return (global_bytes)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, l));
    };
    auto load = [&](Batch& x, int i, int u) {               // (past the end the rows of some page are loaded)
        const int l = 4 * i + SETS * u;
        global_bytes rows = from_lane(rows16, l), scales = from_lane(scales16, l);
        if constexpr (SETS == 2) {                          // the upper lanes' keys may lie in another page (of 16)
            const global_bytes rows1 = from_lane(rows16, l + 1), scales1 = from_lane(scales16, l + 1);
            if (g >> 1) { rows = rows1; scales = scales1; }
        }
        x.a[u] = __builtin_nontemporal_load((global_codes)(rows + lrow));
        x.sc[u] = scales[lsrow];
    };
    QTerms<NT> q;
    int limit, lowest;                                      // scale bytes from which the lane's, some lane's score may not be finite
    bool odd;                                               // the lane's query is not
    float lmax = -INFINITY;
    auto compute = [&](auto more, Batch& x, int i) {
        const int t0 = block_key(i);
        const bool part_of = t0 + C4_BLOCK > k1;
        f32x4 s[U][PASSES];
        float best = -INFINITY;
        int top = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (what lies behind the end may be anything, also a scale that is not a number)
            if (part_of && t0 + u * TK + (SETS == 2 ? 16 * (g >> 1) : 0) + n >= k1) { x.a[u] = i32x4{0, 0, 0, 0}; x.sc[u] = 1; }
            top = max(top, x.sc[u]);
#pragma unroll
            for (int set = 0; set < PASSES; ++set) {
                i32x8 av = {x.a[u][0], x.a[u][1], x.a[u][2], x.a[u][3], 0, 0, 0, 0};
                int sc = x.sc[u];
                if (PASSES == 2 && (g >> 1) != set) { av = i32x8{0, 0, 0, 0, 0, 0, 0, 0}; sc = 1; }
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = NT - 1; t >= 0; --t)
                    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, q.t[t], acc, 4, 0, 0, sc, 0, q.scale[t]);
                s[u][set] = acc;
            }
            if constexpr (decltype(more)::value) load(x, i + 2, u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int set = 0; set < PASSES; ++set)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (part_of && t0 + u * TK + 16 * (set0 + set) + 4 * g + k >= k1) s[u][set][k] = -INFINITY;
                    best = fmaxf(best, s[u][set][k]);
                }
        if constexpr (PAIR) best = fmaxf(best, dpp_move<0x128>(best));          // (row_ror 8: the head's other column)
        best = across16_max(best);
        if (bad || odd) best = INFINITY;
        if (__any(top >= lowest)) { if (wave_max(top) >= limit) best = INFINITY; }     // (hardly ever: a head goes by its own query alone)
        if (!live) best = -INFINITY;
        const float shared_max = c4_from_ordered(__hip_atomic_load(&smax[col], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        lmax = fmaxf(lmax, best);
        const float m = fmaxf(lmax, shared_max);
        if (live && g == 0) bmax[t0 / C4_BLOCK] = best;
        // (a maximum that is infinite: NaN, nothing is kept, nor is anything needed)
        const bool keep = best >= m - p.win - 1e-6f * fabsf(m) && live;
        if (!__any(keep)) return;
        if (g == 0 && best > shared_max) atomicMax(&smax[col], c4_ordered(best));
        if (keep) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int set = 0; set < PASSES; ++set) *(f32x4*)(scores + t0 + u * TK + 16 * (set0 + set) + 4 * g) = s[u][set];
        }
    };
    constexpr auto more = std::true_type{};
    constexpr auto no_more = std::false_type{};
    Batch x0, x1;
#pragma unroll
    for (int u = 0; u < U; ++u) if (mine > 0) load(x0, 0, u);
#pragma unroll
    for (int u = 0; u < U; ++u) if (mine > 1) load(x1, 1, u);
    limit = query_terms<E, D, NT>(qrow, wave, words, tops, q, odd);
    lowest = -wave_max(-limit);
    if constexpr (PAIR) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w) { if (set0) q.t[t][w] = 0; else q.t[t][4 + w] = 0; }
    }
    int i = 0;
    for (; i + 3 < mine; i += 2) { compute(more, x0, i); compute(more, x1, i + 1); }
    if (i + 2 < mine) { compute(more, x0, i); compute(no_more, x1, i + 1); compute(no_more, x0, i + 2); }
    else {
        if (i < mine) compute(no_more, x0, i);
        if (i + 1 < mine) compute(no_more, x1, i + 1);
    }
}

// A wave takes a part of the head's blocks, in order, and keeps its candidates to itself: the waves meet only in the sums of an
// evaluation and of the output.  SPLIT work-groups do the same for a head, each for a part of the output's elements: with few heads the
// card is empty, and what one CU can have on its way limits how fast the rows of a long support are read (32 heads of 131072 keys, 8 key heads, at
// alpha 1.05: 1620 us with one, 522 with four; flat heads at alpha 1.5: 203 and 149; short supports the same; the choice: cache4_run).
template <int D, int AM, int NW, int SPLIT>
__global__ __launch_bounds__(64 * NW) void cache4_entmax_kernel(Cache4Params p) {
    constexpr int SEG = 512, ROW = D / 2, SROW = D / 32, DS = D / SPLIT, LPR = DS / 8, AT_ONCE = 64 / LPR, U = 4;
    __shared__ float lx[NW][SEG];           // c (s - s_max), in the order of the keys; then the probabilities
    __shared__ int lj[NW][SEG];             // key; then its slot
    __shared__ float red[2][NW][2];
    __shared__ int ired[NW];
    __shared__ float osum[NW][DS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slice = blockIdx.z;             // elements DS * slice .. of the output
    const int h = blockIdx.x, req = blockIdx.y, kvh = h / p.G;
    const long head = (long)req * p.Hq + h;
    const int len = p.lens[req];
    const bool len_ok = len >= 0 && len <= p.max_len;
    const int nblocks = len_ok ? (len + C4_BLOCK - 1) / C4_BLOCK : 0, per = (nblocks + NW - 1) / NW;
    const int b0 = min(wave * per, nblocks), b1 = min(b0 + per, nblocks);
    const float* scores = p.scores + head * p.stride;
    const float* bmax = p.bmax + head * (p.stride / C4_BLOCK);
    const float r = p.r;

    float gm = -INFINITY;
    for (int b = b0 + lane; b < b1; b += 64) gm = fmaxf(gm, bmax[b]);
    gm = whole_wave_max(gm);
    if (lane == 0) red[0][wave][0] = gm;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) gm = fmaxf(gm, red[0][w][0]);
    float* O = p.O + head * D + slice * DS;
    if (len == 0 || !len_ok || !(fabsf(gm) < INFINITY)) {
        // no keys: zeros.  A length or page out of range, or a score that is infinite or not a number: not a number
        const float v = len == 0 ? 0.f : __builtin_nanf("");
        if (tid < DS) O[tid] = v;
        if (tid == 0 && slice == 0) { p.tau[head] = v; if (p.support) p.support[head] = len == 0 ? 0 : -1; }
        return;
    }
    // f(x, key) for the scores of the wave's blocks that reach into the window, in the order of their keys, a block at a time, four
    // such loads in flight, and then after(); every 64 blocks enough() may end it (asked after every load, 1 us more for 48 requests up
    // to 32768 keys).  (The score kernel has written these blocks: its window was this one or a lower one.)
    auto walk = [&](auto f, auto after, auto enough) {
        for (int c0 = b0; c0 < b1; c0 += 64) {
            unsigned long long todo = __ballot(c0 + lane < b1 && p.c * (bmax[min(c0 + lane, b1 - 1)] - gm) >= -1.f);
            while (todo) {
                float s[U];
                int key[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    key[u] = -1;
                    if (!todo) continue;
                    key[u] = (c0 + __ffsll((long long)todo) - 1) * C4_BLOCK;
                    todo &= todo - 1;
                    s[u] = scores[key[u] + lane];
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (key[u] >= 0) f(p.c * (s[u] - gm), key[u] + lane);       // (keys past the end were written as -inf)
                after();
            }
            if (enough()) return;
        }
    };
    // The same for sums alone: g(x) for all of them, 256 keys a load.
    auto stream = [&](auto g) {
        for (int c0 = b0; c0 < b1; c0 += 64) {
            const unsigned long long in = __ballot(c0 + lane < b1 && p.c * (bmax[min(c0 + lane, b1 - 1)] - gm) >= -1.f);
#pragma unroll 1
            for (int j = 0; j < 16; j += U) {
                f32x4 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    v[u] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    if (in >> (4 * (j + u) + (lane >> 4)) & 1) v[u] = *(const f32x4*)(scores + (c0 + 4 * (j + u)) * C4_BLOCK + 4 * lane);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) g(p.c * (v[u][e] - gm));
            }
        }
    };
    // Candidates in the order of their keys, whatever else the score kernel wrote: the sums below do not depend on when its
    // waves learned of each other's maxima.  Scores enter as differences to the maximum, which are exact where they are small.
    int total = 0;
    walk([&](float x, int j) {
        const unsigned long long in = __ballot(x >= -1.f);
        const int at = total + __popcll(in & ((1ull << lane) - 1ull));
        if (x >= -1.f && at < SEG) { lx[wave][at] = x; lj[wave][at] = j; }
        total += __popcll(in);
    }, [] {}, [&] { return total > SEG; });
    const bool over = total > SEG;          // then every evaluation of this wave streams its blocks instead
    // F = sum [x - tau]^r and G = sum [x - tau]^(r - 1) over the work-group, the same in every thread
    int turn = 0;
    auto eval = [&](float tau, float& F, float& G) {
        float f = 0.f, gs = 0.f;
        auto term = [&](float x) {
            const float y = x - tau;
            if (!(y > 0.f)) return;
            if (AM == ALPHA_GEN && r < 1.f) { f += pow_r<AM>(y, r); return; }       // (pow_r1 holds y at 1e-6 and above there; G is not asked for)
            const float y1 = pow_r1<AM>(y, r);
            gs += y1;
            f = fmaf(y1, y, f);
        };
        if (!over) for (int i = lane; i < total; i += 64) term(lx[wave][i]);
        else stream(term);
        f = whole_wave_sum(f);
        gs = whole_wave_sum(gs);
        turn ^= 1;                          // (two sets: a wave that is ahead writes the other one)
        if (lane == 0) { red[turn][wave][0] = f; red[turn][wave][1] = gs; }
        __syncthreads();
        F = G = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) { F += red[turn][w][0]; G += red[turn][w][1]; }
    };
    // tau in [-1, 0] (Eq. 5).  r >= 1: F^(1/r) is a norm of the [x - tau]_+, convex in tau, so Newton steps for F^(1/r) = 1 from the
    // left rise to the root; they end where a step no longer moves tau.  r < 1 (alpha > 2): bisection over the
    // floats from 2^-45 to 1 for -tau, by their bits, since N equal keys have tau = -N^(-1/r), down to 2^-44 (2^22 keys, r = 1/2), and
    // to be known relative to itself: 29 evaluations, and -tau is the first float at which F >= 1.
    float tau = -1.f;
    if (AM != ALPHA_GEN || r >= 1.f) {
        for (int it = 0; it < 40; ++it) {
            float F, G;
            eval(tau, F, G);
            // norm less 1; for alpha near 1 F^(1/r) is 1 but for a part in r, and is formed less 1 from the start (1.4 us more for 24
            // requests of 8192 keys at r = 4, where the difference is exact to fp32's last places)
            const float over1 = AM == ALPHA_15 ? sqrtf(F) - 1.f : AM == ALPHA_20 ? F - 1.f
                                : r <= 16.f    ? __builtin_amdgcn_exp2f(__builtin_amdgcn_logf(F) * (1.f / r)) - 1.f
                                               : expm1f(logf(F) / r);
            // (N keys: 1 = F <= N (-tau)^r, so that tau <= -2^-22 for the 2^22 keys there can be; rounding must not carry it to 0)
            const float next = fminf(tau + over1 * F / ((over1 + 1.f) * G), -0x1p-23f);
            // (a step from far left may be rounded past the root by some 1e-7: the next one goes back to its left, and what is left
            // of -tau, down to 2^-22, decides whether it is needed)
            const float step = next - tau;
            tau = next;
            if (step < 3e-8f && fabsf(step) <= -0x1p-12f * next) break;
        }
    } else {
        unsigned int lo = __float_as_uint(0x1p-45f), hi = __float_as_uint(1.f);     // F(-lo) < 1 <= F(-hi)
        while (hi - lo > 1) {
            float F, G;
            const unsigned int mid = (lo + hi) >> 1;
            eval(-__uint_as_float(mid), F, G);
            if (F >= 1.f) hi = mid; else lo = mid;
        }
        tau = -__uint_as_float(hi);
    }

    // o = sum over the support of p_j v_j.  The support is moved to the front of the wave's candidates, with slots in place
    // of keys; then a row's part of values is DS / 8 lanes with eight each, and a wave reads 64 / (DS / 8) rows at a time.
    const int32_t* pages = p.table + (long)req * p.blocks;
    const int shift = p.page_shift, in_page = (1 << shift) - 1, sub = lane % LPR, rsel = lane / LPR, eight = slice * LPR + sub;
    const long page_bytes = (long)(2 * (ROW + SROW)) << shift, stride = page_bytes * p.Hk;
    const unsigned char* const values = p.cache + kvh * page_bytes + ((long)(ROW + SROW) << shift);
    float acc[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = 0.f;
    int nsup = 0;
    float psum = 0.f;
    auto keep_support = [&](float x, int j, int& at) {
        const float y = x - tau;
        const float pj = y > 0.f ? pow_r<AM>(y, r) : 0.f;
        psum += pj;
        const unsigned long long in = __ballot(pj > 0.f);
        const int to = at + __popcll(in & ((1ull << lane) - 1ull));
        if (pj > 0.f) { lx[wave][to] = pj; lj[wave][to] = (pages[j >> shift] << shift) + (j & in_page); }
        at += __popcll(in);
    };
    auto add_rows = [&](int count) {
        constexpr int S = 4;
        for (int i0 = 0; i0 < count; i0 += S * AT_ONCE) {
            unsigned int codes[S];
            float ps[S];
#pragma unroll
            for (int u = 0; u < S; ++u) {
                const int i = i0 + u * AT_ONCE + rsel;
                codes[u] = 0u; ps[u] = 0.f;
                if (i < count) {
                    const int slot = lj[wave][i];
                    const unsigned char* vb = values + (slot >> shift) * stride;
                    const int row = slot & in_page;
                    codes[u] = *(const unsigned int*)(vb + row * ROW + 4 * eight);
                    const unsigned int byte = vb[(ROW << shift) + row * SROW + (eight >> 2)];
                    ps[u] = lx[wave][i] * cache4_scale(byte);
                }
            }
#pragma unroll
            for (int u = 0; u < S; ++u) {
                const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 1);
                const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], 1.f, 3);
                const float v[8] = {v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] = fmaf(ps[u], v[k], acc[k]);
            }
        }
        nsup += count;
    };
    int kept = 0;
    if (!over) {
        for (int i0 = 0; i0 < total; i0 += 64) {
            const bool in = i0 + lane < total;
            keep_support(in ? lx[wave][i0 + lane] : -2.f, in ? lj[wave][i0 + lane] : 0, kept);
        }
    } else {
        walk([&](float x, int j) { keep_support(x, j, kept); },
             [&] { if (kept > SEG - 64 * U) { add_rows(kept); kept = 0; } }, [] { return false; });
    }
    add_rows(kept);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if constexpr (LPR <= 8) acc[k] += dpp_move<0x128>(acc[k]);              // (row_ror 8, 4, 2)
        if constexpr (LPR <= 4) acc[k] += dpp_move<0x124>(acc[k]);
        if constexpr (LPR <= 2) acc[k] += dpp_move<0x122>(acc[k]);
        acc[k] = across16(acc[k]);
        if (rsel == 0) osum[wave][8 * sub + k] = acc[k];
    }
    psum = whole_wave_sum(psum);
    turn ^= 1;                              // (a wave may still be reading the last evaluation's sums)
    if (lane == 0) { ired[wave] = nsup; red[turn][wave][0] = psum; }
    __syncthreads();
    if (tid < DS) {
        float o = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) { o += osum[w][tid]; sum += red[turn][w][0]; }
        // the p add up to 1 but for tau's last place, r times over: what is left of it is common to all where r is large
        O[tid] = o / sum;
    }
    if (tid == 0 && slice == 0) {
        p.tau[head] = (float)(p.c64 * (double)gm + (double)tau);
        int sum = 0;
        for (int w = 0; w < NW; ++w) sum += ired[w];
        if (p.support) p.support[head] = sum;
    }
}

template <int D, int NW, int SPLIT> void cache4_entmax(const Cache4Params& p, hipStream_t s) {
    const dim3 grid(p.Hq, p.R, SPLIT), block(64 * NW);
    switch (p.alpha == 1.5f ? ALPHA_15 : p.alpha == 2.0f ? ALPHA_20 : ALPHA_GEN) {
        case ALPHA_15: hipLaunchKernelGGL((cache4_entmax_kernel<D, ALPHA_15, NW, SPLIT>), grid, block, 0, s, p); break;
        case ALPHA_20: hipLaunchKernelGGL((cache4_entmax_kernel<D, ALPHA_20, NW, SPLIT>), grid, block, 0, s, p); break;
        default: hipLaunchKernelGGL((cache4_entmax_kernel<D, ALPHA_GEN, NW, SPLIT>), grid, block, 0, s, p); break;
    }
}
template <class E, int D>
void cache4_run(const Cache4Params& p, hipStream_t s) {
    const int per_group = C4_WAVES * p.part;
    const dim3 grid(p.Hk * p.colgroups, p.R, (p.max_len + per_group - 1) / per_group), block(64 * C4_WAVES);
    if (D == 64 && p.G <= 8) hipLaunchKernelGGL((cache4_scores_kernel<E, D, D == 64>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((cache4_scores_kernel<E, D, false>), grid, block, 0, s, p);
    // Four work-groups per head up to 64 heads, one from 65 on; there eight waves below 512 heads, four from 512 on.  Both sides of the
    // borders, D = 128, us (alpha 1.5 with short supports at 1000 / 32768 keys; alpha 1.05 with supports of most keys, the same):
    //   64 heads: four work-groups 8.0 / 8.1, 10.3 / 146, one 7.6 / 8.0, 14.4 / 416;  96: four 9.3 / 9.0, 12.7 / 182, one 7.6 / 8.0, 14.7 / 417
    //   384 heads: eight waves 9.4 / 10.9, 23 / 556, four 7.6 / 12.6, 30 / 915;  512: eight 9.3 / 11.8, 24 / 599, four 7.8 / 14.0, 33 / 984;
    //   768: eight 11.2 / 13.5, 29 / 693, four 8.6 / 13.5, 36 / 1085
    // The host knows neither the lengths nor the supports: the borders lie where short supports, the rule, begin to lose.
    const long heads = (long)p.R * p.Hq;
    if (heads <= 64) cache4_entmax<D, 8, 4>(p, s);
    else if (heads < 512) cache4_entmax<D, 8, 1>(p, s);
    else cache4_entmax<D, 4, 1>(p, s);
}

}  // namespace ea

namespace {
using namespace ea;

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Keys per wave of the score kernel: few enough that the waves of all heads number about 4096 (sixteen per CU), where several requests are
// taken to be half as long as the longest, at least C4_BLOCK, and at most C4_MAX_PART: the longest request's keys are not to queue up
// behind few waves.  (24 requests up to 8192 keys, 8 key heads: 192 keys 10 us, 256 11, 512 12.5; 48 requests up to 32768: 41 to 42 us
// from 192 to 512; one of 131072, 32 key heads: 192 and 256 keys 55 us, 512 51.)
int cache4_part(int R, int Hq, int Hk, int max_len) {
    const long groups = (long)R * Hk * ((Hq / Hk + 15) / 16);
    const long part = ((long)max_len * groups / (R > 1 ? 8192 : 4096) + 63) / 64 * 64;
    return part < C4_BLOCK ? C4_BLOCK : part > C4_MAX_PART ? C4_MAX_PART : (int)part;
}
// (an odd number of blocks: heads a power of two apart would begin on the same memory channels)
long cache4_stride(int max_len) { return (((long)max_len + C4_BLOCK - 1) / C4_BLOCK | 1) * C4_BLOCK; }
bool cache4_decode_shape_ok(int R, int Hq, int Hk, int d, int max_len) {
    return R > 0 && R <= 65535 && Hk > 0 && Hq > 0 && Hq % Hk == 0 && Hq <= 65535 && (d == 64 || d == 128) && max_len > 0 &&
           max_len <= (1 << 22);
}

}  // namespace

extern "C" {

size_t entmax_attn_decode_cache4_workspace_bytes(int R, int Hq, int Hk, int d, int max_len) {
    if (!cache4_decode_shape_ok(R, Hq, Hk, d, max_len)) return 0;
    const size_t keys = (size_t)R * Hq * cache4_stride(max_len);
    return align256(keys * 4) + align256(keys / C4_BLOCK * 4);
}

int entmax_attn_decode_cache4(const void* q, const void* cache, const int32_t* block_table, const int32_t* lens,
                              float* O, float* tau, int32_t* support,
                              int R, int Hq, int Hk, int d, int dtype, int max_len, int max_blocks, int n_pages, int page_size,
                              float alpha, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!q || !cache || !block_table || !lens || !O || !tau) return EA_ERR_NULL;
    if (dtype != EA_F32 && dtype != EA_BF16) return EA_ERR_DTYPE;
    if (!cache4_decode_shape_ok(R, Hq, Hk, d, max_len) || !cache_page_ok(page_size) || n_pages <= 0 || max_blocks <= 0 ||
        (long)n_pages * page_size > (long)INT_MAX || (long)max_blocks * page_size < max_len)
        return EA_ERR_SHAPE;
    if (!isfinite(alpha) || !(alpha > 1.f) || alpha > EA_ALPHA_MAX) return EA_ERR_ALPHA;
    if (!aligned16(q) || !aligned16(cache)) return EA_ERR_LAYOUT;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < entmax_attn_decode_cache4_workspace_bytes(R, Hq, Hk, d, max_len))
        return EA_ERR_WORKSPACE;
    Cache4Params p{};
    p.q = q; p.cache = (const unsigned char*)cache; p.table = block_table; p.lens = lens;
    p.O = O; p.tau = tau; p.support = support;
    p.stride = cache4_stride(max_len);
    p.scores = (float*)workspace;
    p.bmax = (float*)((char*)workspace + align256((size_t)R * Hq * p.stride * 4));
    p.R = R; p.Hq = Hq; p.Hk = Hk; p.G = Hq / Hk; p.colgroups = (p.G + 15) / 16;
    p.blocks = max_blocks; p.n_pages = n_pages; p.page_shift = cache_page_shift(page_size); p.max_len = max_len;
    p.part = cache4_part(R, Hq, Hk, max_len);
    p.alpha = alpha; p.r = 1.f / (alpha - 1.f);
    p.c64 = ((double)alpha - 1.0) / sqrt((double)d);
    p.c = (float)p.c64;
    p.win = (1.f + 1e-5f) / p.c;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == EA_BF16) { if (d == 64) cache4_run<Bf16, 64>(p, s); else cache4_run<Bf16, 128>(p, s); }
    else { if (d == 64) cache4_run<F32, 64>(p, s); else cache4_run<F32, 128>(p, s); }
    return launched();
}

}  // extern "C"
