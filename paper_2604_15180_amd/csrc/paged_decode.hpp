// What the decodes from the paged caches (cache4.hpp, cache8.hpp) share: the parameters, sums over lanes, a query's row as the score
// kernels load it, and the second kernel, which solves tau and gathers the values.  A cache's own translation unit has its score kernel.
#pragma once
#include <limits.h>
#include <math.h>

#include "common.hpp"
#include "launch.hpp"

namespace ea {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int PD_WAVES = 4;             // waves per work-group of a score kernel
constexpr int PD_BLOCK = 64;            // keys per maximum
constexpr int PD_MAX_PART = 512;        // keys per wave of a score kernel, at most

// What a score kernel leaves of 64 keys and a head for the second kernel.
// The 4-bit cache's (not Cache::PACKED): their maximum in bmax (+inf also where a score is not a number or a page id out of range), and at
// their own places in scores all 64, where one of them was within the window of Eq. 5 under the largest score its wave knew.
// The 8-bit cache's (PACKED): the maximum, and a bit for each four neighbouring keys of which one was in that window.  The scores of these
// fours alone are written: each wave of a work-group packs those of a head, one behind the other, into a quarter (paged_room) of the
// room that the work-group's keys have; `before` lie in front of the block's, counted from the room's beginning.
// Keys in the window are few and far between, and a store costs the same whether it fills a line or not: with whole blocks the stores took 14 of
// 68 us for 48 requests up to 32768 keys, now 9 of 63, and 7 of 99 for one of 131072 with 32 key heads, now 1; unpacked fours were no faster
// than blocks.  The second kernel takes 0.5 to 1 us more, which is what the 4-bit cache would gain, whose keys are half the bytes.
struct alignas(8) PagedBlock { float max; unsigned short fours, before; };
// fours of a wave's quarter, of a work-group with so many blocks (together up to three blocks more than those)
EA_DEV unsigned int paged_room(int blocks) { return (blocks + PD_WAVES - 1) / PD_WAVES * (PD_BLOCK / 4); }

struct PagedParams {
    const void* q; const unsigned char* cache; const int32_t* table; const int32_t* lens;
    float* O; float* tau; int32_t* support;
    float* scores;            // [R][Hq][stride]
    float* bmax; PagedBlock* found;     // [R][Hq][stride / 64], one of them: see PagedBlock
    long stride;              // keys a head has room for (paged_stride)
    int part;                 // keys per wave of the score kernel, a multiple of 64
    int group; unsigned int by_group;   // (PACKED) blocks of its work-group; 2^32 / group, rounded up: the upper half of a block's number (below 2^17) times it is the group's
    int R, Hq, Hk, G, colgroups;        // G = Hq / Hk query heads per key head, in colgroups of up to 16
    int blocks, n_pages, page_shift, max_len;
    int window, sinks;        // (8-bit cache) keys a query sees: the last `window` and the first `sinks`; window 0: all
    int span;                 // keys of the blocks a request can have that hold one it sees
    float c;                  // (alpha - 1) / sqrt(d)
    double c64;
    float alpha, r, win;      // win: the window of Eq. 5 in units of s, slightly widened
};

// The blocks of 64 keys of a request that hold a key its query sees: the first `head` of the request, and those from
// block head + jump on.  A block's number among them is what scores and maxima are kept by.
struct Visible { int low, sinks, head, jump, count; };      // keys below `sinks` and from `low` on are seen
EA_DEV Visible visible_blocks(int len, int window, int sinks) {
    Visible v;
    v.low = window > 0 ? max(len - window, 0) : 0;
    v.sinks = min(sinks, v.low);
    v.head = (v.sinks + PD_BLOCK - 1) / PD_BLOCK;
    v.jump = max(v.low / PD_BLOCK - v.head, 0);
    v.count = (len + PD_BLOCK - 1) / PD_BLOCK - v.jump;
    return v;
}

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
EA_DEV unsigned int across16_or(unsigned int v) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = a[0] | a[1];
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return b[0] | b[1];
}
EA_DEV float whole_wave_max(float v) {
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    return across16_max(fmaxf(v, dpp_move<0x140>(v)));
}
EA_DEV float whole_wave_sum(float v) { return across16(group_sum<16>(v)); }

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
EA_DEV unsigned int ordered_bits(float f) {
    const unsigned int u = __float_as_uint(f);
    return (u & 0x80000000u) ? ~u : (u ^ 0x80000000u);
}
EA_DEV float from_ordered_bits(unsigned int u) { return __uint_as_float((u & 0x80000000u) ? (u ^ 0x80000000u) : ~u); }

// A wave takes a part of the head's blocks, in order, and keeps its candidates to itself: the waves meet only in the sums of an
// evaluation and of the output.  SPLIT work-groups do the same for a head, each for a part of the output's elements: with few heads the
// card is empty, and what one CU can have on its way limits how fast the rows of a long support are read (32 heads of 131072 keys, 8 key heads, at
// alpha 1.05: 1620 us with one, 522 with four; flat heads at alpha 1.5: 203 and 149; short supports the same; the choice: paged_entmax).
template <class C, int D, int AM, int NW, int SPLIT>
__global__ __launch_bounds__(64 * NW) void paged_entmax_kernel(PagedParams p) {
    constexpr int SEG = 512, DS = D / SPLIT, LPR = DS / 8, AT_ONCE = 64 / LPR, U = 4;
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
    Visible vis;                              // (a constant but for its count where the cache's decode has no window)
    if constexpr (C::WINDOWS) vis = visible_blocks(len_ok ? len : 0, p.window, p.sinks);
    else vis = Visible{0, 0, 0, 0, len_ok ? (len + PD_BLOCK - 1) / PD_BLOCK : 0};
    const int nblocks = vis.count, per = (nblocks + NW - 1) / NW;
    const int b0 = min(wave * per, nblocks), b1 = min(b0 + per, nblocks);
    const float* scores = p.scores + head * p.stride;
    auto block_max = [&](int b) {
        if constexpr (C::PACKED) return p.found[head * (p.stride / PD_BLOCK) + b].max;
        else return p.bmax[head * (p.stride / PD_BLOCK) + b];
    };
    const float r = p.r;

    float gm = -INFINITY;
    for (int b = b0 + lane; b < b1; b += 64) gm = fmaxf(gm, block_max(b));
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
    // A lane for each of 64 blocks from c0 on: whether it reaches into the window, and where what was left of its scores begins; of a
    // packed block's which fours
    struct Left { int at; unsigned int fours; bool in; };
    auto left_of = [&](int c0) {
        const int b = min(c0 + lane, b1 - 1);
        if constexpr (C::PACKED) {
            const PagedBlock x = p.found[head * (p.stride / PD_BLOCK) + b];
            const bool in = c0 + lane < b1 && p.c * (x.max - gm) >= -1.f;
            return Left{(int)__umulhi((unsigned int)b, p.by_group) * p.group * PD_BLOCK + 4 * x.before, in ? x.fours : 0u, in};
        } else {
            return Left{0, 0u, c0 + lane < b1 && p.c * (block_max(b) - gm) >= -1.f};
        }
    };
    // f(x, key) for the scores of the wave's blocks that reach into the window, in the order of their keys, a block at a time, four
    // such loads in flight, and then after(); every 64 blocks enough() may end it (asked after every load, 1 us more for 48 requests up
    // to 32768 keys).  (What the score kernel has not written is below the window: its own was this one or a lower one.)
    const unsigned int below = (1u << (lane >> 2)) - 1u;
    auto walk = [&](auto f, auto after, auto enough) {
        for (int c0 = b0; c0 < b1; c0 += 64) {
            const Left left = left_of(c0);
            unsigned long long todo = __ballot(left.in);
            while (todo) {
                float s[U];
                int key[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    key[u] = -1;
                    if constexpr (C::PACKED) s[u] = -INFINITY;
                    if (!todo) continue;
                    const int i = __ffsll((long long)todo) - 1;
                    key[u] = (c0 + i) * PD_BLOCK;
                    todo &= todo - 1;
                    if constexpr (C::PACKED) {
                        const unsigned int fours = (unsigned int)__builtin_amdgcn_readlane((int)left.fours, i);
                        const int at = __builtin_amdgcn_readlane(left.at, i);
                        // (the other lanes load nothing: with addresses of their own for no use 1 to 2 us more)
                        if (fours >> (lane >> 2) & 1) s[u] = scores[at + 4 * __popc(fours & below) + (lane & 3)];
                    } else {
                        s[u] = scores[key[u] + lane];
                    }
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
            const Left left = left_of(c0);
            const unsigned long long in = __ballot(left.in);
#pragma unroll 1
            for (int j = 0; j < 16; j += U) {
                f32x4 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    v[u] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    const int i = 4 * (j + u) + (lane >> 4);                    // (the lane's block)
                    if constexpr (C::PACKED) {
                        const unsigned int fours = __shfl(left.fours, i);
                        const int at = __shfl(left.at, i);
                        if (fours >> (lane & 15) & 1) v[u] = *(const f32x4*)(scores + at + 4 * __popc(fours & ((1u << (lane & 15)) - 1u)));
                    } else {
                        if (in >> i & 1) v[u] = *(const f32x4*)(scores + (c0 + 4 * (j + u)) * PD_BLOCK + 4 * lane);
                    }
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
    const long page_bytes = C::template part_bytes<D>(shift), stride = page_bytes * p.Hk;
    const unsigned char* const values = p.cache + kvh * page_bytes + C::template values_at<D>(shift);
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
        if (pj > 0.f) {
            lx[wave][to] = pj;
            if (C::WINDOWS && j >= vis.head * PD_BLOCK) j += vis.jump * PD_BLOCK;
            lj[wave][to] = (pages[j >> shift] << shift) + (j & in_page);
        }
        at += __popcll(in);
    };
    auto add_rows = [&](int count) {
        constexpr int S = 4;
        for (int i0 = 0; i0 < count; i0 += S * AT_ONCE) {
            typename C::Piece piece[S];
            float ps[S];
#pragma unroll
            for (int u = 0; u < S; ++u) {
                const int i = i0 + u * AT_ONCE + rsel;
                piece[u] = C::none(); ps[u] = 0.f;
                if (i < count) {
                    const int slot = lj[wave][i];
                    piece[u] = C::template load<D>(values + (slot >> shift) * stride, slot & in_page, eight, shift);
                    ps[u] = lx[wave][i] * C::scale(piece[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < S; ++u) {
                float v[8];
                C::expand(piece[u], v);
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

template <class C, int D, int NW, int SPLIT> void paged_entmax_launch(const PagedParams& p, hipStream_t s) {
    const dim3 grid(p.Hq, p.R, SPLIT), block(64 * NW);
    switch (p.alpha == 1.5f ? ALPHA_15 : p.alpha == 2.0f ? ALPHA_20 : ALPHA_GEN) {
        case ALPHA_15: hipLaunchKernelGGL((paged_entmax_kernel<C, D, ALPHA_15, NW, SPLIT>), grid, block, 0, s, p); break;
        case ALPHA_20: hipLaunchKernelGGL((paged_entmax_kernel<C, D, ALPHA_20, NW, SPLIT>), grid, block, 0, s, p); break;
        default: hipLaunchKernelGGL((paged_entmax_kernel<C, D, ALPHA_GEN, NW, SPLIT>), grid, block, 0, s, p); break;
    }
}
template <class C, int D> void paged_entmax(const PagedParams& p, hipStream_t s) {
    // Four work-groups per head up to 64 heads, one from 65 on; there eight waves below 512 heads, four from 512 on.  Both sides of the
    // borders, D = 128, us (alpha 1.5 with short supports at 1000 / 32768 keys; alpha 1.05 with supports of most keys, the same):
    //   64 heads: four work-groups 8.0 / 8.1, 10.3 / 146, one 7.6 / 8.0, 14.4 / 416;  96: four 9.3 / 9.0, 12.7 / 182, one 7.6 / 8.0, 14.7 / 417
    //   384 heads: eight waves 9.4 / 10.9, 23 / 556, four 7.6 / 12.6, 30 / 915;  512: eight 9.3 / 11.8, 24 / 599, four 7.8 / 14.0, 33 / 984;
    //   768: eight 11.2 / 13.5, 29 / 693, four 8.6 / 13.5, 36 / 1085
    // The host knows neither the lengths nor the supports: the borders lie where short supports, the rule, begin to lose.
    const long heads = (long)p.R * p.Hq;
    // (The 8-bit cache's values are twice the bytes: sixteen waves for long requests of few heads.  One of 131072 keys, 32 heads: with short supports
    // 12.8 us for 12.0 with eight, with flat scores 140 for 184, at alpha 1.05 459 for 728.  Around the border, both launches, 8 key heads, one request of normal
    // queries and keys, alpha 1.5, a third of the queries, alpha 1.05, sixteen / eight: 65536 keys, 32 heads 43.9 / 52.0, 89 / 105, 206 / 305; 64 heads 47.7 / 57.1, 93 / 107, 223 / 308;
    // 32768 keys, 32 heads 29.9 / 32.0, 65 / 65, 118 / 166: nearly alike but for long supports.)
    if constexpr (C::PACKED) {
        if (heads <= 64 && p.span >= 65536) return paged_entmax_launch<C, D, 16, 4>(p, s);
    }
    if (heads <= 64) paged_entmax_launch<C, D, 8, 4>(p, s);
    else if (heads < 512) paged_entmax_launch<C, D, 8, 1>(p, s);
    else {
        // Two waves for many heads with few keys each.  Packed scores (the 8-bit cache), us with four / two waves at 1000, 4000 and 8000 keys:
        //   640 heads 8.6 / 8.2, 10.0 / 11.0, 11.6 / 14.1;  1024: 9.2 / 8.5, 11.2 / 12.2, 12.7 / 14.0;  2048: 14.6 / 10.4, 17.3 / 14.0, 19.7 / 18.2
        if constexpr (C::PACKED) {
            if (2l * p.span <= 5 * heads) return paged_entmax_launch<C, D, 2, 1>(p, s);
        }
        paged_entmax_launch<C, D, 4, 1>(p, s);
    }
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Keys per wave of the score kernel: few enough that the waves of all heads number about 4096 (sixteen per CU), where several requests are
// taken to be half as long as the longest, at least PD_BLOCK, and at most PD_MAX_PART: the longest request's keys are not to queue up
// behind few waves.  (24 requests up to 8192 keys, 8 key heads: 192 keys 10 us, 256 11, 512 12.5; 48 requests up to 32768: 41 to 42 us
// from 192 to 512; one of 131072, 32 key heads: 192 and 256 keys 55 us, 512 51.)
inline int paged_part(int R, int Hq, int Hk, int max_len) {
    const long groups = (long)R * Hk * ((Hq / Hk + 15) / 16);
    const long part = ((long)max_len * groups / (R > 1 ? 8192 : 4096) + 63) / 64 * 64;
    return part < PD_BLOCK ? PD_BLOCK : part > PD_MAX_PART ? PD_MAX_PART : (int)part;
}
// (an odd number of blocks: heads a power of two apart would begin on the same memory channels)
inline long paged_stride(int max_len) { return (((long)max_len + PD_BLOCK - 1) / PD_BLOCK | 1) * PD_BLOCK; }

}  // namespace ea
