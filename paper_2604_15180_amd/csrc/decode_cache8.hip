// One query per head and request against the paged 8-bit cache (cache8.hpp), over all its tokens or a sliding window and the first few.
//   cache8_scores_kernel : s_j = <q, k_j> for a part of the keys that a request's query sees and up to 16 query heads that share a key
//                          head, on the matrix cores; of each 64 keys the maximum per head, and the scores where one of them is
//                          within the window of Eq. 5 of the largest the wave knows.
//   paged_entmax_kernel  : tau and the output (paged_decode.hpp).
// The queries: q = 2^(e - 6) (t_0 + 2^-7 t_1 + 2^-14 t_2 + ...) with integers t_i of eight bits, 2^e the power of two at or below the
// row's largest magnitude; each is the rounding of what those before it left (t_0 up to 127, and so t_1 where t_0 was cut from 128;
// the others up to 64).  Products with the codes and their sums over d are exact 32-bit integers, below 2^21 for d = 128; two
// neighbouring terms are put together as integers too, so that a score is one fused multiply-add of two numbers rounded to float32, times
// the tile's scale.  Three terms know a bf16 element to 2^-21 of the row's largest power of two (exactly down to 2^-13 of
// it), four an fp32 element to 2^-28: less than the rounding of the sum in float32.
#include <type_traits>

#include "cache8.hpp"
#include "paged_decode.hpp"

namespace ea {

// The cache as the kernel that gathers values takes it (paged_decode.hpp)
struct Cache8 {
    static constexpr bool WINDOWS = true, PACKED = true;
    struct Piece { uint2 codes; float scale; };                   // eight values
    static EA_DEV Piece none() { return {uint2{0u, 0u}, 0.f}; }
    template <int D> static EA_DEV long part_bytes(int shift) { return cache8_part_bytes(D, shift); }
    template <int D> static EA_DEV long values_at(int shift) { return (long)D << shift; }
    template <int D> static EA_DEV Piece load(const unsigned char* vb, int row, int eight, int shift) {
        return {*(const uint2*)(vb + row * D + 8 * eight), *cache8_scale(vb - ((long)D << shift), D, shift, 1, row / C8_BLOCK)};
    }
    static EA_DEV float scale(const Piece& x) { return fabsf(x.scale); }
    static EA_DEV void expand(const Piece& x, float* v) { cache8_expand(x.codes, __float_as_uint(x.scale) >> 31, v); }
};

// Terms of a row's values as operand registers of the 16x16x64 instruction: lane (n, g) = (lane % 16, lane / 16) supplies, of column n,
// the contraction indices 16 g .. 16 g + 15; one register set for each 64 of them.
template <int D, int NT> struct QDigits { i32x4 t[NT][D / 64]; float unit; };      // unit: of the last term
constexpr int Q8_LEAST = -90;           // rows whose largest magnitude is below 2^-90 lose what is below that

// The waves of a work-group convert their quarters and hand them round through LDS.  Every thread calls this.  odd: the lane's row
// holds an infinity or a NaN.
template <class E, int D, int NT>
EA_DEV void query_digits(const QRow<E, D>& row, int wave, int (*words)[8][64], float (*tops)[16], QDigits<D, NT>& out, bool& odd) {
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
    odd = !(top < INFINITY);
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, Q8_LEAST), 127);
#pragma unroll
    for (int run = 0; run < RUNS; ++run) {
        float* v = x[run];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = odd ? 0.f : ldexpf(v[i], 6 - e);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            int bits = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float n = fminf(fmaxf(rintf(v[i]), -127.f), 127.f);
                bits |= ((int)n & 255) << (8 * i);
                v[i] = (v[i] - n) * 128.f;                             // (both exact)
            }
            words[t][4 * run + wave][lane] = bits;
        }
    }
    __syncthreads();
    out.unit = ldexpf(1.f, e - 6 - 7 * (NT - 1));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int run = 0; run < RUNS; ++run)
#pragma unroll
            for (int w = 0; w < 4; ++w) out.t[t][run][w] = words[t][4 * run + w][lane];
}

// Tiles of sixteen keys, one instruction per term and 64 elements.  Result: lane (n, g) holds column n's scores with keys
// 4 g .. 4 g + 3.  A wave keeps a block of 64 keys on its way: as soon as the matrix cores have taken a tile, the same tile of the
// next block is requested.  The addresses and scales of all its tiles are formed and loaded at once, a lane for each.
// At D = 128 an operand is half a row, but a load is of eight whole rows (half lines cost 15 %): lane (n, g) loads of row n mod 8, then of row
// n mod 8 + 8, piece g, or piece 4 + g in the lanes n >= 8, and the two halves of sixteen lanes exchange what is the other's.
// Bound: HBM, for long requests: one of 131072 keys with 32 key heads takes 93 us, 5.8 TB/s of keys; 48 requests up to 32768 keys 63 us, 4.3 TB/s;
// 64 with a window of 4000, 34 us, 4.0 TB/s.  One block ahead leaves registers for three or four waves per SIMD (two blocks: two waves, 104
// us and 74 for 102 and 72 before the scores were packed).
template <class E, int D>
__global__ __launch_bounds__(64 * PD_WAVES, 3) void cache8_scores_kernel(PagedParams p) {
    constexpr int NT = sizeof(typename E::elem) == 2 ? 3 : 4, RUNS = D / 64, U = PD_BLOCK / 16;
    __shared__ unsigned int smax[16];                       // ordered bits of the work-group's running maxima
    __shared__ int words[NT][8][64];
    __shared__ float tops[PD_WAVES][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    // the part of the keys is the slowest index, and the requests move on by one CU from part to part: short requests have few
    // parts, and the work-groups that find nothing to do must not fall on some of the XCDs or CUs
    const int kvh = blockIdx.x / p.colgroups, cg = blockIdx.x - kvh * p.colgroups, chunk = blockIdx.z;
    const int req = (int)((blockIdx.y + (unsigned int)((p.R - 1) & 31) * chunk) % (unsigned int)p.R);
    const int shift = p.page_shift, in_page = (1 << shift) - 1;
    // (the waves take the work-group's blocks in turn, so that a request shorter than its part of the keys is all four waves' work)
    const int first = chunk * PD_WAVES * (p.part / PD_BLOCK);
    auto block_at = [&](int i) { return first + i * PD_WAVES + wave; };                   // the wave's block i
    const bool live = cg * 16 + n < p.G;                    // (else a column without a head: zeros, nothing is written)
    const long head = (long)req * p.Hq + kvh * p.G + (live ? cg * 16 + n : 0);
    const int len = p.lens[req];
    QRow<E, D> qrow;
    qrow.load(p.q, head, live, wave);
    if (len <= 0 || len > p.max_len) return;
    const Visible vis = visible_blocks(len, p.window, p.sinks);
    if (first >= vis.count) return;
    const int last = min(vis.count, first + PD_WAVES * (p.part / PD_BLOCK));
    const int mine = (last - first - wave + PD_WAVES - 1) / PD_WAVES;                     // the wave's blocks
    if (threadIdx.x < 16) smax[threadIdx.x] = ordered_bits(-INFINITY);
    auto first_key = [&](int b) { return (b + (b >= vis.head ? vis.jump : 0)) * PD_BLOCK; };
    auto seen = [&](int key) { return key < vis.sinks || (key >= vis.low && key < len); };
    // Lane 4 i + j: the sixteen keys j of block i (PD_MAX_PART: at most eight blocks)
    const int key16 = first_key(block_at(lane >> 2)) + 16 * (lane & 3);
    const bool wanted = (lane >> 2) < mine && (key16 < vis.sinks || (key16 + 15 >= vis.low && key16 < len));    // some key of it is seen
    int id = wanted ? p.table[(long)req * p.blocks + (key16 >> shift)] : 0;
    const bool strange = (unsigned)id >= (unsigned)p.n_pages;
    if (strange) id = 0;
    const int part_bytes = cache8_part_bytes(D, shift);
    const unsigned char* const page = p.cache + ((long)id * p.Hk + kvh) * part_bytes;
    const uint64_t rows16 = (uint64_t)(page + (key16 & in_page) * D);
    const float scale16 = wanted ? *cache8_scale(page, D, shift, 0, (key16 & in_page) / C8_BLOCK) : 0.f;
    float* const room = p.scores + head * p.stride + first * PD_BLOCK;
    PagedBlock* const found = p.found + head * (p.stride / PD_BLOCK);
    const unsigned int lrow = RUNS == 2 ? (n & 7) * D + 64 * (n >> 3) + 16 * g : n * D + 16 * g;
    struct Batch { i32x4 a[U][RUNS]; };
    typedef const unsigned char __attribute__((address_space(1)))* global_bytes;       // (a pointer from two integers is not known to be global)
    typedef const i32x4 __attribute__((address_space(1)))* global_codes;
    auto load = [&](Batch& x, int i, int u) {               // (rows of some page where no key is seen)
        const int l = 4 * i + u;
        const global_bytes rows = (global_bytes)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(rows16 >> 32), l) << 32 |
                                                 (uint32_t)__builtin_amdgcn_readlane((int)rows16, l));
#pragma unroll
        for (int run = 0; run < RUNS; ++run) x.a[u][run] = __builtin_nontemporal_load((global_codes)(rows + lrow + 1024 * run));
    };
    auto operands = [&](i32x4 (&a)[RUNS]) {               // (row_ror 8: from the lane n + 8 or n - 8 of the same sixteen)
        if constexpr (RUNS == 2) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int lo = a[0][w], hi = a[1][w];
                a[0][w] = __builtin_amdgcn_update_dpp(lo, hi, 0x128, 0xf, 0xc, false);
                a[1][w] = __builtin_amdgcn_update_dpp(hi, lo, 0x128, 0xf, 0x3, false);
            }
        }
    };
    QDigits<D, NT> q;
    bool odd, bad;                                          // the lane's query is not finite; a score may not be
    float lmax = -INFINITY;
    unsigned int kept = wave * paged_room(last - first);    // where the lane's head has its next four
    auto compute = [&](auto more, Batch& x, int i) {
        const int b = block_at(i), t0 = first_key(b);
        const bool whole = t0 + PD_BLOCK <= vis.sinks || (t0 >= vis.low && t0 + PD_BLOCK <= len);
        f32x4 s[U];
        float best = -INFINITY;
        bool nan = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float scale = __uint_as_float((unsigned int)__builtin_amdgcn_readlane((int)__float_as_uint(scale16), 4 * i + u));
            operands(x.a[u]);
            i32x4 acc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                acc[t] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int run = 0; run < RUNS; ++run) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x.a[u][run], q.t[t][run], acc[t], 0, 0, 0);
            }
            if (__float_as_uint(scale) >> 31) {             // (a sign bit: some code may stand for NaN)
                bool any = false;
#pragma unroll
                for (int run = 0; run < RUNS; ++run)
#pragma unroll
                    for (int w = 0; w < 4; ++w) any |= cache8_odd((unsigned int)x.a[u][run][w]);
                nan |= any && seen(t0 + 16 * u + n);
            }
            if constexpr (decltype(more)::value) load(x, i + 1, u);
            const float unit = fabsf(scale) * q.unit;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int hi = NT == 3 ? acc[0][k] : acc[0][k] * 128 + acc[1][k], lo = acc[NT - 2][k] * 128 + acc[NT - 1][k];
                s[u][k] = fmaf((float)hi, 16384.f, (float)lo) * unit;
            }
        }
        float quad[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!whole) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (!seen(t0 + 16 * u + 4 * g + k)) s[u][k] = -INFINITY;
            }
            quad[u] = fmaxf(fmaxf(s[u][0], s[u][1]), fmaxf(s[u][2], s[u][3]));
            best = fmaxf(best, quad[u]);
        }
        best = across16_max(best);
        if (bad || __any(nan)) best = INFINITY;
        if (!live) best = -INFINITY;
        const float shared_max = from_ordered_bits(__hip_atomic_load(&smax[n], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
        lmax = fmaxf(lmax, best);
        const float m = fmaxf(lmax, shared_max);
        // (a maximum that is infinite: NaN, nothing is kept, nor is anything needed)
        const float low = m - p.win - 1e-6f * fabsf(m);
        unsigned int fours = 0;
        const unsigned int before = kept;
        if (__any(best >= low && live)) {
            if (g == 0 && best > shared_max) atomicMax(&smax[n], ordered_bits(best));
#pragma unroll
            for (int u = 0; u < U; ++u) fours |= (quad[u] >= low && live) << (4 * u + g);
            fours = across16_or(fours);
            kept += __popc(fours);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned int k = before + __popc(fours & ((1u << (4 * u + g)) - 1u));
                if (quad[u] >= low && live) *(f32x4*)(room + 4 * k) = s[u];
            }
        }
        if (live && g == 0) found[b] = PagedBlock{best, (unsigned short)fours, (unsigned short)before};
    };
    constexpr auto more = std::true_type{};
    constexpr auto no_more = std::false_type{};
    Batch x0;
#pragma unroll
    for (int u = 0; u < U; ++u) if (mine > 0) load(x0, 0, u);
    query_digits<E, D, NT>(qrow, wave, words, tops, q, odd);
    // |score| < 2^21 * 2^14 (three terms; 2^28 * 2^14) * unit * scale, and unit holds 2^-14 (2^-21): at most 2^22 * 2^(e - 6) * scale
    const float most = whole_wave_max(wanted ? (fabsf(scale16) < INFINITY ? fabsf(scale16) : INFINITY) : 0.f);
    bad = odd || __any(strange) || !(most < INFINITY) || !(most * q.unit < (NT == 3 ? 0x1p84f : 0x1p77f));
    int i = 0;
    for (; i + 1 < mine; ++i) compute(more, x0, i);
    if (i < mine) compute(no_more, x0, i);
}

template <class E, int D>
void cache8_run(const PagedParams& p, hipStream_t s) {
    const int per_group = PD_WAVES * p.part;
    const dim3 grid(p.Hk * p.colgroups, p.R, (p.span + per_group - 1) / per_group), block(64 * PD_WAVES);
    hipLaunchKernelGGL((cache8_scores_kernel<E, D>), grid, block, 0, s, p);
    paged_entmax<Cache8, D>(p, s);
}

}  // namespace ea

namespace {
using namespace ea;

bool cache8_decode_shape_ok(int R, int Hq, int Hk, int d, int max_len, int window, int sinks) {
    return R > 0 && R <= 65535 && Hk > 0 && Hq > 0 && Hq % Hk == 0 && Hq <= 65535 && (d == 64 || d == 128) && max_len > 0 &&
           max_len <= (1 << 22) && window >= 0 && sinks >= 0;
}
// Keys of the blocks that hold a key that is seen, at most: the window may begin and end inside a block
int cache8_span(int max_len, int window, int sinks) {
    const long all = ((long)max_len + PD_BLOCK - 1) / PD_BLOCK;
    if (window == 0) return (int)all * PD_BLOCK;
    const long some = ((long)sinks + PD_BLOCK - 1) / PD_BLOCK + ((long)window + PD_BLOCK - 2) / PD_BLOCK + 1;
    return (int)(some < all ? some : all) * PD_BLOCK;
}

// (three blocks for the waves' quarters: paged_room)
long cache8_stride(int span) { return paged_stride(span + 3 * PD_BLOCK); }

}  // namespace

extern "C" {

size_t entmax_attn_decode_cache8_workspace_bytes(int R, int Hq, int Hk, int d, int max_len, int window, int sinks) {
    if (!cache8_decode_shape_ok(R, Hq, Hk, d, max_len, window, sinks)) return 0;
    const size_t keys = (size_t)R * Hq * cache8_stride(cache8_span(max_len, window, sinks));
    return align256(keys * 4) + align256(keys / PD_BLOCK * sizeof(PagedBlock));
}

int entmax_attn_decode_cache8(const void* q, const void* cache, const int32_t* block_table, const int32_t* lens,
                              float* O, float* tau, int32_t* support,
                              int R, int Hq, int Hk, int d, int dtype, int max_len, int max_blocks, int n_pages, int page_size,
                              int window, int sinks, float alpha, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!q || !cache || !block_table || !lens || !O || !tau) return EA_ERR_NULL;
    if (dtype != EA_F32 && dtype != EA_BF16) return EA_ERR_DTYPE;
    if (!cache8_decode_shape_ok(R, Hq, Hk, d, max_len, window, sinks) || !cache_page_ok(page_size) || n_pages <= 0 || max_blocks <= 0 ||
        (long)n_pages * page_size > (long)INT_MAX || (long)max_blocks * page_size < max_len)
        return EA_ERR_SHAPE;
    if (!isfinite(alpha) || !(alpha > 1.f) || alpha > EA_ALPHA_MAX) return EA_ERR_ALPHA;
    if (!aligned16(q) || !aligned16(cache)) return EA_ERR_LAYOUT;
    if (!workspace || ((uintptr_t)workspace & 255) ||
        workspace_bytes < entmax_attn_decode_cache8_workspace_bytes(R, Hq, Hk, d, max_len, window, sinks))
        return EA_ERR_WORKSPACE;
    PagedParams p{};
    p.q = q; p.cache = (const unsigned char*)cache; p.table = block_table; p.lens = lens;
    p.O = O; p.tau = tau; p.support = support;
    p.span = cache8_span(max_len, window, sinks);
    p.stride = cache8_stride(p.span);
    p.scores = (float*)workspace;
    p.found = (PagedBlock*)((char*)workspace + align256((size_t)R * Hq * p.stride * 4));
    p.R = R; p.Hq = Hq; p.Hk = Hk; p.G = Hq / Hk; p.colgroups = (p.G + 15) / 16;
    p.blocks = max_blocks; p.n_pages = n_pages; p.page_shift = cache_page_shift(page_size); p.max_len = max_len;
    p.window = window; p.sinks = sinks;
    p.part = paged_part(R, Hq, Hk, p.span);
    p.group = PD_WAVES * p.part / PD_BLOCK;
    p.by_group = (unsigned int)((1ull << 32) / p.group) + 1u;
    p.alpha = alpha; p.r = 1.f / (alpha - 1.f);
    p.c64 = ((double)alpha - 1.0) / sqrt((double)d);
    p.c = (float)p.c64;
    p.win = (1.f + 1e-5f) / p.c;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == EA_BF16) { if (d == 64) cache8_run<Bf16, 64>(p, s); else cache8_run<Bf16, 128>(p, s); }
    else { if (d == 64) cache8_run<F32, 64>(p, s); else cache8_run<F32, 128>(p, s); }
    return launched();
}

}  // extern "C"
