// One query per head and request against the paged 4-bit cache (cache4.hpp): entmax_attn_decode for a serving program.
//   cache4_scores_kernel : s_j = <q, k_j> for a part of a request's keys and up to 16 query heads that share a key head, on
//                          the matrix cores: key codes are an operand as they lie in memory, their scale bytes the operand's scales.
//                          By Eq. 5 only scores within sqrt(d) / (alpha - 1) of the head's maximum can be in the support, and
//                          a running maximum is a lower bound of the final one: of each 64 keys the maximum per head is written,
//                          and the scores where one of them is within that window of the largest the wave knows.
//   paged_entmax_kernel  : per head, tau from the scores of the blocks whose maximum is in the window, and o = sum p_j v_j over
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
#include <type_traits>

#include "cache4.hpp"
#include "paged_decode.hpp"

namespace ea {

// The cache as the kernel that gathers values takes it (paged_decode.hpp)
struct Cache4 {
    static constexpr bool WINDOWS = false, PACKED = false;
    struct Piece { unsigned int codes; float scale; };            // eight values
    static EA_DEV Piece none() { return {0u, 0.f}; }
    template <int D> static EA_DEV long part_bytes(int shift) { return (long)(2 * (D / 2 + D / 32)) << shift; }
    template <int D> static EA_DEV long values_at(int shift) { return (long)(D / 2 + D / 32) << shift; }
    template <int D> static EA_DEV Piece load(const unsigned char* vb, int row, int eight, int shift) {
        return {*(const unsigned int*)(vb + row * (D / 2) + 4 * eight), cache4_scale(vb[((D / 2) << shift) + row * (D / 32) + (eight >> 2)])};
    }
    static EA_DEV float scale(const Piece& x) { return x.scale; }
    static EA_DEV void expand(const Piece& x, float* v) {
        const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x.codes, 1.f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x.codes, 1.f, 1);
        const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x.codes, 1.f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x.codes, 1.f, 3);
        v[0] = v0[0]; v[1] = v0[1]; v[2] = v1[0]; v[3] = v1[1]; v[4] = v2[0]; v[5] = v2[1]; v[6] = v3[0]; v[7] = v3[1];
    }
};

// Terms of the row's values as operand registers of the 16x16x128 instruction: lane (n, g) = (lane % 16, lane / 16) supplies,
// of column n, the contraction indices 16 g .. 16 g + 15 and 64 + 16 g .. in the e4m3 format (D = 64: both the same; a 4-bit operand:
// 32 g .. 32 g + 31, whose scale byte is the lane's own; the scale of a column's block b is that of lane (n, b)).
template <int NT> struct QTerms { i32x8 t[NT]; int scale[NT]; };   // scale: bytes

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

// Tiles: at D = 128 sixteen keys, one instruction per term; at D = 64 two sets of sixteen keys, the lower half of the lanes
// (contraction indices 0 .. 63 of the operand) one, the upper half the other.  Then (PAIR) up to eight query heads stand in columns 0 .. 7
// with their terms in the lower indices, for the first set, and once more in columns 8 .. 15 in the upper ones, for the second,
// with zeros elsewhere: both sets in one instruction per term.  More heads have their terms in both halves, and the keys are worked on
// one set at a time, with zeros in place of the other's (32 heads x 131072 keys, one head a key head: 38 us, PAIR 32; fp32 queries 40 and 32).
// Result: lane (n, g) holds column n's scores with keys 4 g .. 4 g + 3 of a set.  A wave keeps two blocks of 64 keys on their way: as soon as
// the matrix cores have taken a tile, the same tile of the block after the next is requested.  The addresses of all its keys are
// formed at once, a lane for each sixteen.
template <class E, int D, bool PAIR>
__global__ __launch_bounds__(64 * PD_WAVES) void cache4_scores_kernel(PagedParams p) {
    constexpr int NT = sizeof(typename E::elem) == 2 ? 4 : 5, SETS = 128 / D, TK = 16 * SETS, U = PD_BLOCK / TK;
    constexpr int PASSES = PAIR ? 1 : SETS, COLS = PAIR ? 8 : 16;         // instructions of a tile and term; query heads side by side
    static_assert(!PAIR || SETS == 2, "two sets to a tile");
    constexpr int ROW = D / 2, SROW = D / 32;
    __shared__ unsigned int smax[16];                       // ordered bits of the work-group's running maxima
    __shared__ int words[NT][8][64];
    __shared__ float tops[PD_WAVES][16];
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
    const int c0 = chunk * PD_WAVES * p.part;
    auto block_key = [&](int i) { return c0 + (i * PD_WAVES + wave) * PD_BLOCK; };        // first key of the wave's block i
    const bool live = cg * 16 + col < p.G;                  // (else a column without a head: zeros, nothing is written)
    const long head = (long)req * p.Hq + kvh * p.G + (live ? cg * 16 + col : 0);
    // length, pages and query are asked for together, and the first keys before the query is worked on.  Lane 4 i + j: the sixteen
    // keys j of block i (PD_MAX_PART: at most eight blocks).
    const int len = p.lens[req];
    const int key16 = block_key(lane >> 2) + 16 * (lane & 3);
    int id = p.table[(long)req * p.blocks + min(key16 >> shift, p.blocks - 1)];
    QRow<E, D> qrow;
    qrow.load(p.q, head, live, wave);
    if (len < 0 || len > p.max_len || c0 >= len) return;
    const int k1 = min(len, c0 + PD_WAVES * p.part);
    const int mine = ((k1 - c0 + PD_BLOCK - 1) / PD_BLOCK - wave + PD_WAVES - 1) / PD_WAVES;       // the wave's blocks
    if (threadIdx.x < 16) smax[threadIdx.x] = ordered_bits(-INFINITY);
    const bool strange = (unsigned)id >= (unsigned)p.n_pages;
    const bool bad = __any(strange && key16 < k1);
    if (strange) id = 0;
    const long page_bytes = (long)(2 * (ROW + SROW)) << shift;
    const unsigned char* const page = p.cache + ((long)id * p.Hk + kvh) * page_bytes;
    const uint64_t rows16 = (uint64_t)(page + (key16 & in_page) * ROW), scales16 = (uint64_t)(page + (ROW << shift) + (key16 & in_page) * SROW);
    float* const scores = p.scores + head * p.stride;
    float* const bmax = p.bmax + head * (p.stride / PD_BLOCK);
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
        const bool part_of = t0 + PD_BLOCK > k1;
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
        const float shared_max = from_ordered_bits(__hip_atomic_load(&smax[col], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        lmax = fmaxf(lmax, best);
        const float m = fmaxf(lmax, shared_max);
        if (live && g == 0) bmax[t0 / PD_BLOCK] = best;
        // (a maximum that is infinite: NaN, nothing is kept, nor is anything needed)
        const bool keep = best >= m - p.win - 1e-6f * fabsf(m) && live;
        if (!__any(keep)) return;
        if (g == 0 && best > shared_max) atomicMax(&smax[col], ordered_bits(best));
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

template <class E, int D>
void cache4_run(const PagedParams& p, hipStream_t s) {
    const int per_group = PD_WAVES * p.part;
    const dim3 grid(p.Hk * p.colgroups, p.R, (p.max_len + per_group - 1) / per_group), block(64 * PD_WAVES);
    if (D == 64 && p.G <= 8) hipLaunchKernelGGL((cache4_scores_kernel<E, D, D == 64>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((cache4_scores_kernel<E, D, false>), grid, block, 0, s, p);
    paged_entmax<Cache4, D>(p, s);
}

}  // namespace ea

namespace {
using namespace ea;

bool cache4_decode_shape_ok(int R, int Hq, int Hk, int d, int max_len) {
    return R > 0 && R <= 65535 && Hk > 0 && Hq > 0 && Hq % Hk == 0 && Hq <= 65535 && (d == 64 || d == 128) && max_len > 0 &&
           max_len <= (1 << 22);
}

}  // namespace

extern "C" {

size_t entmax_attn_decode_cache4_workspace_bytes(int R, int Hq, int Hk, int d, int max_len) {
    if (!cache4_decode_shape_ok(R, Hq, Hk, d, max_len)) return 0;
    const size_t keys = (size_t)R * Hq * paged_stride(max_len);
    return align256(keys * 4) + align256(keys / PD_BLOCK * 4);
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
    PagedParams p{};
    p.q = q; p.cache = (const unsigned char*)cache; p.table = block_table; p.lens = lens;
    p.O = O; p.tau = tau; p.support = support;
    p.stride = paged_stride(max_len);
    p.scores = (float*)workspace;
    p.bmax = (float*)((char*)workspace + align256((size_t)R * Hq * p.stride * 4));
    p.R = R; p.Hq = Hq; p.Hk = Hk; p.G = Hq / Hk; p.colgroups = (p.G + 15) / 16;
    p.blocks = max_blocks; p.n_pages = n_pages; p.page_shift = cache_page_shift(page_size); p.max_len = p.span = max_len;
    p.part = paged_part(R, Hq, Hk, max_len);
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
