// One query per head and request against the paged 4-bit cache (cache4.hpp): entmax_attn_decode for a serving program.
//   cache4_scores_kernel : s_j = <q, k_j> for a part of a request's keys and up to 16 query heads that share a key head, on
//                          the matrix cores: key codes are an operand as they lie in memory, their scale bytes the operand's scales.
//                          By Eq. 5 only scores within sqrt(d) / (alpha - 1) of the head's maximum can be in the support, and
//                          a running maximum is a lower bound of the final one: a wave lists, per head, the scores within that window
//                          of the largest it knows, with their keys, in the order of the keys, and leaves their number and its maximum.
//   cache4_entmax_kernel : per head, tau from the listed scores and o = sum p_j v_j over the support.
// The queries: q = 2^e (t_0 + 2^-5 t_1 + 2^-10 t_2 + ...) with e4m3 terms t_i below 2^8, each the rounding of what the terms before it
// left.  Of each eight neighbouring products the matrix cores keep what lies within 2^-13 of the largest one's exponent (measured: a
// product 2^-14 of its neighbour is lost, at any place of the eight; beyond the eight and for the scales the sum is fp32's),
// which a small element's last bits would miss.  So the terms are multiples of 1/8: codes are multiples of 1/2 up to 6, exponents go up to
// 2 + 7, and no product has bits below 2^-4.  Three terms then hold a bf16 value exactly down to 2^-13 of the row's largest, and below that
// to 2^-21 of it; four hold an fp32 value to 2^-26.  (Two terms with e4m3's own last bits, 2^-9, were off by 2e-5 in
// tau; with the multiples of 1/8 the sums are exact up to their one rounding for each term.)
#include <limits.h>
#include <math.h>

#include "cache4.hpp"
#include "common.hpp"
#include "launch.hpp"

namespace ea {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int C4_MAX_LISTS = 1024;      // lists (waves of the score kernel) per head
constexpr int C4_WAVES = 4;             // waves per work-group of the score kernel

struct Cache4Params {
    const void* q; const unsigned char* cache; const int32_t* table; const int32_t* lens;
    float* O; float* tau; int32_t* support;
    uint2* cand;              // [R][Hq][lists][part] listed scores: (bits of s_j, j)
    int* ccnt;                // [R][Hq][lists] how many; -1: the request's length or a page of it is out of range
    float* gmax;              // [R][Hq][lists] maximum of the part; +inf also where a score is not a number
    int R, Hq, Hk, G, colgroups;        // G = Hq / Hk query heads per key head, in colgroups of up to 16
    int blocks, n_pages, page_shift, max_len;
    int part, lists;          // keys per wave, waves per head
    float c;                  // (alpha - 1) / sqrt(d)
    double c64;
    float alpha, r, win;      // win: the window of Eq. 5 in units of s, slightly widened
};

// Terms of the row's values as operand registers of the 16x16x128 instruction: lane (n, g) = (lane % 16, lane / 16) supplies,
// of column n, the contraction indices 16 g .. 16 g + 15 and 64 + 16 g .. in the e4m3 format (a 4-bit operand:
// 32 g .. 32 g + 31, whose scale byte is the lane's own; the scale of a column's block b is that of lane (n, b)).
template <int NT> struct QTerms { i32x8 t[NT]; int scale[NT]; };

template <class E, int D, int NT> EA_DEV void load_query(const Cache4Params& p, const void* q, long head, bool live, QTerms<NT>& out) {
    using elem = typename E::elem;
    typedef elem vec __attribute__((ext_vector_type(8)));
    constexpr int RUNS = D / 64;
    const int g = __lane_id() >> 4;
    float x[RUNS][16];
#pragma unroll
    for (int run = 0; run < RUNS; ++run)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            vec v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (elem)0.f;
            if (live) v = *(const vec*)((const elem*)q + head * D + 64 * run + 16 * g + 8 * half);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[run][8 * half + e] = (float)v[e];
        }
    float top = 0.f;
#pragma unroll
    for (int run = 0; run < RUNS; ++run)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(x[run][e]));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    // the largest term below 2^8; scales from 2^-122 up: rows below 2^-100 lose what is below that
    const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100) - 7;
#pragma unroll
    for (int run = 0; run < RUNS; ++run)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[run][i] = ldexpf(x[run][i], -e);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        out.scale[t] = 127 + e - 5 * t;
#pragma unroll
        for (int w = 0; w < 8; ++w) out.t[t][w] = 0;
#pragma unroll
        for (int run = 0; run < RUNS; ++run)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                float* v = &x[run][4 * w];
                constexpr float EIGHTHS = 1.5f * (1 << 20);          // added and taken off again: rounds to multiples of 1/8
                int bits = __builtin_amdgcn_cvt_pk_fp8_f32((v[0] + EIGHTHS) - EIGHTHS, (v[1] + EIGHTHS) - EIGHTHS, 0, false);
                bits = __builtin_amdgcn_cvt_pk_fp8_f32((v[2] + EIGHTHS) - EIGHTHS, (v[3] + EIGHTHS) - EIGHTHS, bits, true);
                out.t[t][4 * run + w] = bits;
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(bits, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(bits, true);
                v[0] = (v[0] - lo[0]) * 32.f; v[1] = (v[1] - lo[1]) * 32.f;
                v[2] = (v[2] - hi[0]) * 32.f; v[3] = (v[3] - hi[1]) * 32.f;
            }
    }
}

EA_DEV unsigned int c4_ordered(float f) {
    const unsigned int u = __float_as_uint(f);
    return (u & 0x80000000u) ? ~u : (u ^ 0x80000000u);
}
EA_DEV float c4_from_ordered(unsigned int u) { return __uint_as_float((u & 0x80000000u) ? (u ^ 0x80000000u) : ~u); }

// Tiles: at D = 128 sixteen keys, one instruction per term; at D = 64 two sets of sixteen keys, the lower half of the lanes
// (contraction indices 0 .. 63 of the operand) one, the upper half the other, and the query terms stand in one half of their operand
// with zeros in the other, once for each set.  Result: lane (n, g) holds head n's scores with keys 4 g .. 4 g + 3 of a set.
template <class E, int D>
__global__ __launch_bounds__(64 * C4_WAVES) void cache4_scores_kernel(Cache4Params p) {
    constexpr int NT = sizeof(typename E::elem) == 2 ? 3 : 4, SETS = 128 / D, TK = 16 * SETS, U = 4;
    constexpr int ROW = D / 2, SROW = D / 32;
    __shared__ unsigned int smax[16];                       // ordered bits of the work-group's running maxima
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int kvh = blockIdx.y / p.colgroups, cg = blockIdx.y - kvh * p.colgroups, req = blockIdx.z;
    const int len = p.lens[req];
    const int list = blockIdx.x * C4_WAVES + wave;
    const bool live = cg * 16 + n < p.G;
    const long head = (long)req * p.Hq + kvh * p.G + cg * 16 + n;      // (only where live)
    if (threadIdx.x < 16) smax[threadIdx.x] = c4_ordered(-INFINITY);
    __syncthreads();
    const bool len_ok = len >= 0 && len <= p.max_len;
    const int k0 = list * p.part, k1 = len_ok ? min(len, k0 + p.part) : k0;
    float lmax = -INFINITY;
    int count = 0;
    bool bad = !len_ok;
    if (k0 < k1) {
        QTerms<NT> q;
        load_query<E, D, NT>(p, p.q, head, live, q);
        uint2* const mine = p.cand + ((size_t)(live ? head : 0) * p.lists + list) * (size_t)p.part;
        const int32_t* pages = p.table + (long)req * p.blocks;
        const int in_page = (1 << p.page_shift) - 1;
        const int key_lane = (SETS == 2 ? 16 * (g >> 1) : 0) + n, block_lane = SETS == 2 ? g & 1 : g;   // the operand row and block this lane loads
        for (int t0 = k0; t0 < k1; t0 += TK * U) {
            i32x4 a[U];
            int sc[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // a lane's key decides its page: the sets of a tile may lie in two, and what lies behind the length in none
                const int key = t0 + u * TK + key_lane;
                const int first = min(key & ~15, k1 - 1);
                int page = pages[first >> p.page_shift];
                if ((unsigned)page >= (unsigned)p.n_pages) { bad = true; page = 0; }
                const unsigned char* base = p.cache + (((long)page * p.Hk + kvh) * (2 * (ROW + SROW)) << p.page_shift);
                const int row = key & in_page;
                a[u] = __builtin_nontemporal_load((const i32x4*)(base + row * ROW + 16 * block_lane));
                sc[u] = base[(ROW << p.page_shift) + row * SROW + block_lane];
                // what lies behind the end may be anything, also a scale that is not a number, which a zero term of the other
                // set's key in the same operand row would not hide
                if (key >= k1) { a[u] = i32x4{0, 0, 0, 0}; sc[u] = 127; }
            }
            float s[U][SETS][4];
            float best = -INFINITY;
            bool odd = false;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const i32x8 av = {a[u][0], a[u][1], a[u][2], a[u][3], 0, 0, 0, 0};
#pragma unroll
                for (int set = 0; set < SETS; ++set) {
                    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = NT - 1; t >= 0; --t) {
                        i32x8 b = q.t[t];
                        if constexpr (SETS == 2) {
                            const i32x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
                            if (set == 0) b = i32x8{b[0], b[1], b[2], b[3], z[0], z[0], z[0], z[0]};
                            else b = i32x8{z[0], z[0], z[0], z[0], b[0], b[1], b[2], b[3]};
                        }
                        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, b, acc, 4, 0, 0, sc[u], 0, q.scale[t]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = t0 + u * TK + 16 * set + 4 * g + i;
                        const float v = key < k1 && live ? acc[i] : -INFINITY;
                        odd = odd || (key < k1 && live && !(fabsf(acc[i]) < INFINITY));
                        s[u][set][i] = v;
                        best = fmaxf(best, v);
                    }
                }
            }
            if (odd) best = INFINITY;
            best = fmaxf(best, __shfl_xor(best, 16));
            best = fmaxf(best, __shfl_xor(best, 32));
            const float shared_max = c4_from_ordered(*(volatile unsigned int*)&smax[n]);
            lmax = fmaxf(lmax, best);
            const float m = fmaxf(lmax, shared_max), keep = m - p.win - 1e-6f * fabsf(m);
            if (!__any(best >= keep && best > -INFINITY)) continue;
            if (g == 0 && best > shared_max) atomicMax(&smax[n], c4_ordered(best));
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int set = 0; set < SETS; ++set) {
                    // the head's four lanes hold sixteen keys: lane g the keys 4 g .. 4 g + 3, in this order
                    int mask = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) mask |= (s[u][set][i] >= keep && s[u][set][i] > -INFINITY ? 1 : 0) << i;
                    if (!__any(mask)) continue;
                    int all = mask << (4 * g);
                    all |= __shfl_xor(all, 16);
                    all |= __shfl_xor(all, 32);
                    int at = count + __popc(all & ((1 << (4 * g)) - 1));
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (mask >> i & 1) mine[at++] = make_uint2(__float_as_uint(s[u][set][i]), (unsigned int)(t0 + u * TK + 16 * set + 4 * g + i));
                    count += __popc(all);
                }
        }
    }
    bad = __any(bad);
    if (live && g == 0) {
        p.ccnt[head * p.lists + list] = bad ? -1 : count;
        p.gmax[head * p.lists + list] = lmax;
    }
}

template <int D, int AM>
__global__ __launch_bounds__(256) void cache4_entmax_kernel(Cache4Params p) {
    constexpr int T = 256, NW = T / 64, CAP = 2048, ROW = D / 2, SROW = D / 32, DPL = D / 64;
    __shared__ float lx[CAP];               // c (s - s_max), in the order of the keys
    __shared__ int lj[CAP];
    __shared__ int pref[C4_MAX_LISTS + 1];
    __shared__ float red[NW][2];
    __shared__ int ired[NW][2];
    __shared__ float osum[NW][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x, req = blockIdx.y, kvh = h / p.G;
    const long head = (long)req * p.Hq + h;
    const uint2* cand = p.cand + (size_t)head * p.lists * (size_t)p.part;
    const float r = p.r;

    // the head's maximum, and the listed scores before each list
    float gm = -INFINITY;
    int bad = 0, base = 0;
    if (tid == 0) pref[0] = 0;
    for (int l0 = 0; l0 < p.lists; l0 += T) {
        const int l = l0 + tid;
        int cnt = l < p.lists ? p.ccnt[head * p.lists + l] : 0;
        if (l < p.lists) gm = fmaxf(gm, p.gmax[head * p.lists + l]);
        if (cnt < 0) { bad = 1; cnt = 0; }
        int incl = cnt;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(incl, off);
            if (lane >= off) incl += up;
        }
        __syncthreads();
        if (lane == 63) ired[wave][0] = incl;
        __syncthreads();
        int before = base;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            before += w < wave ? ired[w][0] : 0;
            base += ired[w][0];
        }
        if (l < p.lists) pref[l + 1] = before + incl;
    }
    gm = wave_max(gm);
    bad = __any(bad);
    if (lane == 0) { red[wave][0] = gm; ired[wave][1] = bad; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) { gm = fmaxf(gm, red[w][0]); bad |= ired[w][1]; }
    const int M = pref[p.lists];
    float* O = p.O + head * D;
    if (bad || !(fabsf(gm) < INFINITY)) {
        // no keys: zeros.  A length or page out of range, or a score that is infinite or not a number: not a number
        const bool none = !bad && gm == -INFINITY;
        const float v = none ? 0.f : __builtin_nanf("");
        for (int i = tid; i < D; i += T) O[i] = v;
        if (tid == 0) { p.tau[head] = v; if (p.support) p.support[head] = none ? 0 : -1; }
        return;
    }
    auto listed = [&](int i) {              // i < M
        int lo = 0, hi = p.lists;           // pref[lo] <= i < pref[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (pref[mid] <= i) lo = mid; else hi = mid;
        }
        return cand[(size_t)lo * p.part + (i - pref[lo])];
    };
    // Candidates in the order of their keys, whatever else the score kernel listed: the sums below do not depend on when its
    // waves learned of each other's maxima.  Scores enter as differences to the maximum, which are exact where they are small.
    int total = 0;
    for (int i0 = 0; i0 < M; i0 += T) {
        const int i = i0 + tid;
        float x = -2.f;
        int j = 0;
        if (i < M) { const uint2 e = listed(i); x = p.c * (__uint_as_float(e.x) - gm); j = (int)e.y; }
        const unsigned long long in = __ballot(x >= -1.f);
        __syncthreads();
        if (lane == 0) ired[wave][0] = __popcll(in);
        __syncthreads();
        int at = total + __popcll(in & ((1ull << lane) - 1ull));
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            at += w < wave ? ired[w][0] : 0;
            total += ired[w][0];
        }
        if (x >= -1.f && at < CAP) { lx[at] = x; lj[at] = j; }
    }
    __syncthreads();
    const bool over = total > CAP;          // then every evaluation streams the listed scores instead
    const int nsrc = over ? M : total;
    auto at = [&](int i, float& x, int& j) {
        if (over) { const uint2 e = listed(i); x = p.c * (__uint_as_float(e.x) - gm); j = (int)e.y; }
        else { x = lx[i]; j = lj[i]; }
    };
    // F = sum [x - tau]^r and G = sum [x - tau]^(r - 1) over the work-group, the same in every thread
    auto eval = [&](float tau, float& F, float& G) {
        F = 0.f; G = 0.f;
        for (int i = tid; i < nsrc; i += T) {
            float x; int j;
            at(i, x, j);
            const float y = x - tau;
            if (y > 0.f) { const float y1 = pow_r1<AM>(y, r); G += y1; F = fmaf(y1, y, F); }
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) { F += __shfl_xor(F, off); G += __shfl_xor(G, off); }
        __syncthreads();
        if (lane == 0) { red[wave][0] = F; red[wave][1] = G; }
        __syncthreads();
        F = G = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) { F += red[w][0]; G += red[w][1]; }
    };
    // tau in [-1, 0] (Eq. 5).  r >= 1: F^(1/r) is a norm of the [x - tau]_+, convex in tau, so Newton steps for F^(1/r) = 1 from the
    // left rise to the root and stay left of it; they end where a step no longer moves tau.  r < 1 (alpha > 2): bisection.
    float tau = -1.f;
    if (r >= 1.f) {
        for (int it = 0; it < 40; ++it) {
            float F, G;
            eval(tau, F, G);
            const float norm = AM == ALPHA_15 ? sqrtf(F) : AM == ALPHA_20 ? F : __builtin_amdgcn_exp2f(__builtin_amdgcn_logf(F) * (1.f / r));
            const float next = fminf(tau + (norm - 1.f) * F / (norm * G), 0.f);
            if (!(next > tau)) break;
            const bool small = next - tau < 3e-8f;
            tau = next;
            if (small) break;
        }
    } else {
        float lo = -1.f, hi = 0.f;
        for (int it = 0; it < 26; ++it) {
            float F, G;
            tau = 0.5f * (lo + hi);
            eval(tau, F, G);
            if (F >= 1.f) lo = tau; else hi = tau;
        }
        tau = 0.5f * (lo + hi);
    }

    // o = sum over the support of p_j v_j: a wave takes 64 candidates at a time and walks those with p > 0; its lanes
    // then read that key's row of codes
    float acc[DPL];
#pragma unroll
    for (int k = 0; k < DPL; ++k) acc[k] = 0.f;
    int nsup = 0;
    const int32_t* pages = p.table + (long)req * p.blocks;
    for (int b0 = wave * 64; b0 < nsrc; b0 += T) {
        float x = -2.f;
        int j = 0;
        if (b0 + lane < nsrc) at(b0 + lane, x, j);
        const float y = x - tau;
        const float pj = y > 0.f ? pow_r<AM>(y, r) : 0.f;
        unsigned long long todo = __ballot(pj > 0.f);
        nsup += __popcll(todo);
        while (todo) {
            const int src = __ffsll((long long)todo) - 1;
            todo &= todo - 1;
            const float pv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(pj), src));
            const int key = __builtin_amdgcn_readlane(j, src);
            const int page = pages[key >> p.page_shift], row = key & ((1 << p.page_shift) - 1);
            const unsigned char* vb = p.cache + ((((long)page * p.Hk + kvh) * (2 * (ROW + SROW)) + (ROW + SROW)) << p.page_shift);
            // lane: the values DPL lane ..
            const unsigned int byte = vb[(ROW << p.page_shift) + row * SROW + lane * DPL / 32];
            const float scale = byte == 255u ? __builtin_nanf("") : __uint_as_float(byte << 23);
            const unsigned int codes = vb[row * ROW + lane * DPL / 2] >> (DPL == 1 ? 4 * (lane & 1) : 0);
#pragma unroll
            for (int k = 0; k < DPL; ++k) {
                const unsigned int c = codes >> (4 * k), m = c & 7u;
                const float level = m < 2u ? 0.5f * (float)m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
                acc[k] = fmaf(pv, ((c & 8u) ? -level : level) * scale, acc[k]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < DPL; ++k) osum[wave][lane * DPL + k] = acc[k];
    if (lane == 0) ired[wave][1] = nsup;
    __syncthreads();
    if (tid < D) O[tid] = (osum[0][tid] + osum[1][tid]) + (osum[2][tid] + osum[3][tid]);
    if (tid == 0) {
        p.tau[head] = (float)(p.c64 * (double)gm + (double)tau);
        if (p.support) p.support[head] = (ired[0][1] + ired[1][1]) + (ired[2][1] + ired[3][1]);
    }
}

template <class E, int D>
void cache4_run(const Cache4Params& p, hipStream_t s) {
    hipLaunchKernelGGL((cache4_scores_kernel<E, D>), dim3(p.lists / C4_WAVES, p.Hk * p.colgroups, p.R), dim3(64 * C4_WAVES), 0, s, p);
    const dim3 grid(p.Hq, p.R);
    switch (p.alpha == 1.5f ? ALPHA_15 : p.alpha == 2.0f ? ALPHA_20 : ALPHA_GEN) {
        case ALPHA_15: hipLaunchKernelGGL((cache4_entmax_kernel<D, ALPHA_15>), grid, dim3(256), 0, s, p); break;
        case ALPHA_20: hipLaunchKernelGGL((cache4_entmax_kernel<D, ALPHA_20>), grid, dim3(256), 0, s, p); break;
        default: hipLaunchKernelGGL((cache4_entmax_kernel<D, ALPHA_GEN>), grid, dim3(256), 0, s, p); break;
    }
}

}  // namespace ea

namespace {
using namespace ea;

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Keys per wave of the score kernel: so many that the waves of all heads number about 4096 (sixteen per CU), at least 64, and
// so few lists per head that the second kernel holds their prefix sums.
struct Cache4Split { int part, lists; };
Cache4Split cache4_split(int R, int Hq, int Hk, int max_len) {
    const long groups = (long)R * Hk * ((Hq / Hk + 15) / 16);
    long waves = 4096 / groups;
    if (waves < C4_WAVES) waves = C4_WAVES;
    if (waves > C4_MAX_LISTS) waves = C4_MAX_LISTS;
    long part = (max_len + waves - 1) / waves;
    part = (part + 63) / 64 * 64;
    if (part < 64) part = 64;
    long lists = (max_len + part - 1) / part;
    lists = (lists + C4_WAVES - 1) / C4_WAVES * C4_WAVES;
    if (lists < C4_WAVES) lists = C4_WAVES;
    return {(int)part, (int)lists};
}
bool cache4_decode_shape_ok(int R, int Hq, int Hk, int d, int max_len) {
    return R > 0 && R <= 65535 && Hk > 0 && Hq > 0 && Hq % Hk == 0 && Hq <= 65535 && (d == 64 || d == 128) && max_len > 0 &&
           max_len <= (1 << 22);
}

}  // namespace

extern "C" {

size_t entmax_attn_decode_cache4_workspace_bytes(int R, int Hq, int Hk, int d, int max_len) {
    if (!cache4_decode_shape_ok(R, Hq, Hk, d, max_len)) return 0;
    const Cache4Split sp = cache4_split(R, Hq, Hk, max_len);
    const size_t lists = (size_t)R * Hq * sp.lists;
    return 2 * align256(lists * 4) + align256(lists * sp.part * 8);
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
    if (((uintptr_t)q & 15) || ((uintptr_t)cache & 15)) return EA_ERR_LAYOUT;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < entmax_attn_decode_cache4_workspace_bytes(R, Hq, Hk, d, max_len))
        return EA_ERR_WORKSPACE;
    const Cache4Split sp = cache4_split(R, Hq, Hk, max_len);
    Cache4Params p{};
    p.q = q; p.cache = (const unsigned char*)cache; p.table = block_table; p.lens = lens;
    p.O = O; p.tau = tau; p.support = support;
    const size_t lists = (size_t)R * Hq * sp.lists;
    p.gmax = (float*)workspace;
    p.ccnt = (int*)((char*)workspace + align256(lists * 4));
    p.cand = (uint2*)((char*)workspace + 2 * align256(lists * 4));
    p.R = R; p.Hq = Hq; p.Hk = Hk; p.G = Hq / Hk; p.colgroups = (p.G + 15) / 16;
    p.blocks = max_blocks; p.n_pages = n_pages; p.page_shift = cache_page_shift(page_size); p.max_len = max_len;
    p.part = sp.part; p.lists = sp.lists;
    p.alpha = alpha; p.r = 1.f / (alpha - 1.f);
    p.c64 = ((double)alpha - 1.0) / sqrt((double)d);
    p.c = (float)p.c64;
    p.win = (1.f + 1e-5f) / p.c;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == EA_BF16) { if (d == 64) cache4_run<Bf16, 64>(p, s); else cache4_run<Bf16, 128>(p, s); }
    else { if (d == 64) cache4_run<F32, 64>(p, s); else cache4_run<F32, 128>(p, s); }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_last_hip_error((int)e); return EA_ERR_HIP; }
    return EA_OK;
}

}  // extern "C"
