// Queries and keys as the attention calls take them: per-head RMS norm of what a layer's projections
// give, and the rotation by one or several position axes, in one pass; and the gradient of that.
//   y = w x / sqrt(mean x^2 + eps),   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position[axis(i)] * inv_freq[i]
// With R the rotation, xh = x / sqrt(mean x^2 + eps) and g = R^T dy:
//   dw = sum g xh,   dx = (g w - xh mean(g w xh)) / sqrt(mean x^2 + eps)
// Bound: HBM, each row is read once and written once.  A row (one head of one token) is D / 8 lanes, a lane
// holds four pairs, both members of each, so that the rotation needs no exchange between lanes; the angles
// of a token are formed once and serve all heads a lane walks through.
#include <math.h>

#include "common.hpp"
#include "launch.hpp"

namespace ea {

constexpr int MAX_AXES = 4;

struct PrepParams {
    const void* x[2];            // q, k (rows of `st` strides)
    void* y[2];                  // forward: [B][H][N][D] of E; backward: dx, strides `dst`
    const float* dy[2];          // backward: [B][H][N][D]
    const float* w[2];           // null: ones
    float* dw[2];                // null: not wanted
    float* part;                 // backward: [work-groups][2][D] sums of dw
    const int32_t* pos;          // [axes][B * N]
    const float* inv_freq;       // [rot / 2]
    long st[2][3], dst[2][3];    // strides of batch, token, head, in elements
    int H[2];
    int N, tokens, pairs, axes, heads_per_group;
    int end[MAX_AXES];           // pairs before end[a] (and not before end[a - 1]) turn with axis a
    float eps;
    int norm;
};

// the lane's four pairs: members a[4], b[4]
struct Pairs { float a[4], b[4]; };

// Where the lane's four pairs lie in a row: the first members at `a`, the second at `b` (neighbours: eight elements at
// `a`, members alternating).  Pairs past the rotated ones are laid over the rest of the row the same way.
template <int D, bool NEIGHBOURS> EA_DEV void pair_place(int sub, int pairs, int& a, int& b) {
    if constexpr (NEIGHBOURS) { a = 8 * sub; b = a + 4; }
    else {
        const int i = 4 * sub;
        const bool turned = i < pairs;
        a = turned ? i : i + pairs;                      // rot + (i - pairs)
        b = a + (turned ? pairs : D / 2 - pairs);
    }
}
template <bool NEIGHBOURS, class T> EA_DEV Pairs load_pairs(const T* row, int a, int b) {
    typedef T vec __attribute__((ext_vector_type(4)));
    const vec u = *(const vec*)(row + a), v = *(const vec*)(row + b);
    Pairs p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (NEIGHBOURS) { p.a[e] = (float)(e < 2 ? u[2 * e] : v[2 * e - 4]); p.b[e] = (float)(e < 2 ? u[2 * e + 1] : v[2 * e - 3]); }
        else { p.a[e] = (float)u[e]; p.b[e] = (float)v[e]; }
    }
    return p;
}
template <bool NEIGHBOURS, class T> EA_DEV void store_pairs(T* row, int a, int b, const Pairs& p) {
    typedef T vec __attribute__((ext_vector_type(4)));
    vec u, v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (NEIGHBOURS) { if (e < 2) { u[2 * e] = (T)p.a[e]; u[2 * e + 1] = (T)p.b[e]; } else { v[2 * e - 4] = (T)p.a[e]; v[2 * e - 3] = (T)p.b[e]; } }
        else { u[e] = (T)p.a[e]; v[e] = (T)p.b[e]; }
    }
    *(vec*)(row + a) = u;
    *(vec*)(row + b) = v;
}

// cos and sin of the lane's four angles for one token.  The product is formed in 64 bits and the nearest quarter turn is taken off
// there: at position 100000 an angle in 32 bits is off by up to 2^-8 of a radian.  What is left, at most pi / 4, goes to Taylor's series
// up to its 9th and 10th power (the next terms are below 2e-9 and 2e-10), so that both are known to about a step of fp32 of their
// own.  (The hardware's sine and cosine of turns are off by 1.3e-7 of 1, and a half turn rounded to fp32 by 9e-8.  They took 4.5 us in
// place of 4.7 for eight tokens, 44.9 in place of 45.9 for 131072 tokens of three heads; the same for many heads.)
EA_DEV void angles(const PrepParams& p, int token, int sub, float (&c)[4], float (&s)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = 4 * sub + e;
        c[e] = 1.f; s[e] = 0.f;
        if (i < p.pairs) {
            int ax = 0;
#pragma unroll
            for (int k = 0; k < MAX_AXES - 1; ++k) ax += i >= p.end[k];
            const double quarters = (double)p.pos[(long)ax * p.tokens + token] * ((double)p.inv_freq[i] * 0.63661977236758134308);
            const double whole = __builtin_rint(quarters);
            const float t = (float)((quarters - whole) * 1.57079632679489661923), t2 = t * t;
            const float sn = fmaf(t * t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), t);
            const float cs = fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
            const int quadrant = (int)(long)whole & 3;
            const float x = quadrant & 1 ? sn : cs, y = quadrant & 1 ? cs : sn;
            c[e] = quadrant == 1 || quadrant == 2 ? -x : x;
            s[e] = quadrant & 2 ? -y : y;
        }
    }
}

// Several heads' rows are on their way at once (the compiler does not unroll a loop with cross-lane sums by itself, and one row
// at a time does not cover the memory's latency: 32768 tokens of 32 heads, D = 128, bf16, 123 -> 115 us; two rows 118, eight 114; 111 with
// the first ones asked for before the angles: 4.8 TB/s of reads and writes).
template <class E, int D, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_prep_kernel(PrepParams p) {
    using elem = typename E::elem;
    constexpr int LPR = D / 8, TPG = 256 / LPR, HB = 4;
    const int sub = threadIdx.x % LPR;
    const int token = blockIdx.x * TPG + threadIdx.x / LPR;
    if (token >= p.tokens) return;                       // (no exchange crosses the lanes of a row)
    const int b = token / p.N, n = token - b * p.N;
    int pa, pb;
    pair_place<D, NEIGHBOURS>(sub, p.pairs, pa, pb);
    const int h0 = blockIdx.y * p.heads_per_group, h1 = min(p.H[0] + p.H[1], h0 + p.heads_per_group);
    auto row = [&](int which, int h) { return (const elem*)p.x[which] + b * p.st[which][0] + n * p.st[which][1] + h * p.st[which][2]; };
    // heads first .. last - 1 of q (which = 0) or k are this work-group's
    auto heads_of = [&](int which, int& first, int& last) {
        const int base = which ? p.H[0] : 0;
        first = max(h0, base) - base;
        last = min(h1, base + p.H[which]) - base;
    };
    Pairs v[HB];
    auto load = [&](int which, int h, int last) {
#pragma unroll
        for (int k = 0; k < HB; ++k) v[k] = load_pairs<NEIGHBOURS>(row(which, min(h + k, last - 1)), pa, pb);
    };
    int first, last;
    const int start = h0 < p.H[0] ? 0 : 1;
    heads_of(start, first, last);
    load(start, first, last);                            // (on their way while the angles are formed)
    float c[4], s[4];
    angles(p, token, sub, c, s);
#pragma unroll 1
    for (int which = start; which < 2; ++which) {
        heads_of(which, first, last);
        if (first >= last) continue;
        Pairs w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.a[e] = w.b[e] = 1.f;
        if (p.w[which]) w = load_pairs<NEIGHBOURS>(p.w[which], pa, pb);
        elem* y = (elem*)p.y[which] + ((long)b * p.H[which] * p.N + n) * D;
        for (int h = first; h < last; h += HB) {
            if (which != start || h != first) load(which, h, last);
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                float rstd = 1.f;
                if (p.norm) {
                    float sq = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) sq = fmaf(v[k].a[e], v[k].a[e], fmaf(v[k].b[e], v[k].b[e], sq));
                    rstd = rsqrtf(group_sum<LPR>(sq) * (1.f / D) + p.eps);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = v[k].a[e] * rstd * w.a[e], bb = v[k].b[e] * rstd * w.b[e];
                    v[k].a[e] = a * c[e] - bb * s[e];
                    v[k].b[e] = a * s[e] + bb * c[e];
                }
                if (h + k < last) store_pairs<NEIGHBOURS>(y + (long)(h + k) * p.N * D, pa, pb, v[k]);
            }
        }
    }
}

// A work-group takes every gridDim.x-th set of tokens and a part of the heads, and leaves one row of sums of dw; qk_prep_dw_kernel adds
// the rows.  (16384 tokens of 32 heads, D = 64, bf16: 44 us, 6.1 TB/s; with one row at a time on its way 52.)
template <class E, int D, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void qk_prep_bwd_kernel(PrepParams p) {
    using elem = typename E::elem;
    constexpr int LPR = D / 8, TPG = 256 / LPR, HB = 2;
    __shared__ float sums[4][2][D];
    const int sub = threadIdx.x % LPR;
    int pa, pb;
    pair_place<D, NEIGHBOURS>(sub, p.pairs, pa, pb);
    Pairs dw[2];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[which].a[e] = dw[which].b[e] = 0.f;
    const int p0 = blockIdx.y * p.heads_per_group, p1 = min(p.H[0] + p.H[1], p0 + p.heads_per_group);
    for (long set = blockIdx.x; set * TPG < p.tokens; set += gridDim.x) {
        const int token = (int)(set * TPG) + threadIdx.x / LPR;
        if (token >= p.tokens) break;
        const int b = token / p.N, n = token - b * p.N;
        Pairs gr[HB], v[HB];
        auto load = [&](int which, int h0, int last) {
            const elem* x = (const elem*)p.x[which] + b * p.st[which][0] + n * p.st[which][1];
            const float* dy = p.dy[which] + ((long)b * p.H[which] * p.N + n) * D;
#pragma unroll
            for (int k = 0; k < HB; ++k) {
                const int h = min(h0 + k, last - 1);
                gr[k] = load_pairs<NEIGHBOURS>(dy + (long)h * p.N * D, pa, pb);
                v[k] = load_pairs<NEIGHBOURS>(x + h * p.st[which][2], pa, pb);
            }
        };
        const int start = p0 < p.H[0] ? 0 : 1;
        load(start, start ? p0 - p.H[0] : p0, start ? p1 - p.H[0] : min(p1, p.H[0]));        // (on their way while the angles are formed)
        float c[4], s[4];
        angles(p, token, sub, c, s);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            Pairs w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w.a[e] = w.b[e] = 1.f;
            if (p.w[which]) w = load_pairs<NEIGHBOURS>(p.w[which], pa, pb);
            elem* dx = (elem*)p.y[which] + b * p.dst[which][0] + n * p.dst[which][1];
            const int base = which ? p.H[0] : 0;
            const int first = max(p0, base) - base, last = min(p1, base + p.H[which]) - base;
            for (int h0 = first; h0 < last; h0 += HB) {
                if (which != start || h0 != first) load(which, h0, last);
#pragma unroll
                for (int k = 0; k < HB; ++k) {
                    if (h0 + k >= last) break;
                    Pairs& g = gr[k];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ga = g.a[e] * c[e] + g.b[e] * s[e];
                        g.b[e] = g.b[e] * c[e] - g.a[e] * s[e];
                        g.a[e] = ga;
                    }
                    if (p.norm) {
                        float sq = 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) sq = fmaf(v[k].a[e], v[k].a[e], fmaf(v[k].b[e], v[k].b[e], sq));
                        const float rstd = rsqrtf(group_sum<LPR>(sq) * (1.f / D) + p.eps);
                        float dot = 0.f;
                        Pairs xh;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            xh.a[e] = v[k].a[e] * rstd; xh.b[e] = v[k].b[e] * rstd;
                            dw[which].a[e] = fmaf(g.a[e], xh.a[e], dw[which].a[e]);
                            dw[which].b[e] = fmaf(g.b[e], xh.b[e], dw[which].b[e]);
                            g.a[e] *= w.a[e]; g.b[e] *= w.b[e];
                            dot = fmaf(g.a[e], xh.a[e], fmaf(g.b[e], xh.b[e], dot));
                        }
                        dot = group_sum<LPR>(dot) * (1.f / D);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            g.a[e] = rstd * (g.a[e] - xh.a[e] * dot);
                            g.b[e] = rstd * (g.b[e] - xh.b[e] * dot);
                        }
                    }
                    store_pairs<NEIGHBOURS>(dx + (h0 + k) * p.dst[which][2], pa, pb, g);
                }
            }
        }
    }
    if (!p.part) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int off = LPR; off < 64; off <<= 1) {
                dw[which].a[e] += __shfl_xor(dw[which].a[e], off);
                dw[which].b[e] += __shfl_xor(dw[which].b[e], off);
            }
        if (lane < LPR) store_pairs<NEIGHBOURS>(&sums[wave][which][0], pa, pb, dw[which]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += 256) {
        const float* s0 = &sums[0][0][0] + i;
        p.part[((long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * D + i] = (s0[0] + s0[2 * D]) + (s0[4 * D] + s0[6 * D]);
    }
}

// dw[which][i] = sum over the rows of `part`, in 64 bits: sixteen columns per work-group, 64 threads to a column (with 64 columns and
// sixteen threads a launch took 10 us for 1024 rows: each thread's 64 loads stood in a row)
__global__ __launch_bounds__(1024) void qk_prep_dw_kernel(const float* part, float* dwq, float* dwk, int rows, int D) {
    constexpr int COLS = 16, U = 4;
    __shared__ double sums[16][COLS];
    const int col = threadIdx.x % COLS, slice = threadIdx.x / COLS, i = blockIdx.x * COLS + col;
    double a = 0.0;
    for (int r0 = slice; r0 < rows; r0 += 64 * U) {
        float v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = r0 + 64 * u < rows ? part[(long)(r0 + 64 * u) * 2 * D + i] : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) a += (double)v[u];
    }
    a += __shfl_xor(a, 16);                 // a wave holds four slices of the sixteen columns
    a += __shfl_xor(a, 32);
    if ((threadIdx.x & 63) < COLS) sums[threadIdx.x >> 6][col] = a;
    __syncthreads();
    if (threadIdx.x < COLS) {
#pragma unroll
        for (int k = 1; k < 16; ++k) a += sums[k][col];
        float* out = i < D ? dwq : dwk;
        if (out) out[i < D ? i : i - D] = (float)a;
    }
}

}  // namespace ea

namespace {
using namespace ea;

constexpr int BWD_GROUPS = 1024;        // work-groups of the backward: four per CU, each leaves one row of sums

int tokens_per_group(int d) { return 256 / (d / 8); }

// strides in elements: rows of a tensor start at multiples of 16 bytes
bool strides_ok(const int64_t* st, int elem_bytes) {
    if (!st) return false;
    for (int k = 0; k < 3; ++k)
        if (st[k] < 0 || (st[k] * elem_bytes) % 16) return false;
    return true;
}
// An output's rows must not overlap: the strides, in whichever order, hold the extents below them.
bool rows_apart(const int64_t* st, const int (&extent)[3], int d) {
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (st[order[j]] < st[order[i]]) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
    int64_t reach = d;                  // elements from the first to behind the last of what lies below
    for (int k = 0; k < 3; ++k) {
        if (extent[order[k]] == 1) continue;
        if (st[order[k]] < reach) return false;
        reach += st[order[k]] * (int64_t)(extent[order[k]] - 1);
    }
    return true;
}

int prep_check(const void* q, const void* k, int B, int Hq, int Hk, int N, int d, int t, const int32_t* positions,
               const float* inv_freq, int rot, int n_axes, const int* sections, int norm, float eps,
               const float* wq, const float* wk) {
    if (!q || !k) return EA_ERR_NULL;
    if (t != EA_F32 && t != EA_BF16) return EA_ERR_DTYPE;
    if (B <= 0 || N <= 0 || Hq <= 0 || Hk <= 0 || Hq > 65535 || Hk > 65535 || (d != 64 && d != 128) || (long)B * N > (1l << 27)) return EA_ERR_SHAPE;
    if (rot < 0 || rot > d || rot % 8) return EA_ERR_SHAPE;
    if (rot > 0) {
        if (!positions || !inv_freq) return EA_ERR_NULL;
        if (n_axes < 1 || n_axes > MAX_AXES) return EA_ERR_SHAPE;
        if (!sections && n_axes > 1) return EA_ERR_NULL;
        long sum = 0;
        for (int a = 0; sections && a < n_axes; ++a) {
            if (sections[a] < 0) return EA_ERR_SHAPE;
            sum += sections[a];
        }
        if (sections && sum != rot / 2) return EA_ERR_SHAPE;
    }
    if (norm && !(isfinite(eps) && eps > 0.f)) return EA_ERR_SHAPE;
    if (!norm && (wq || wk)) return EA_ERR_SHAPE;
    if (!aligned16(wq) || !aligned16(wk)) return EA_ERR_LAYOUT;
    return EA_OK;
}

void prep_params(PrepParams& p, const void* q, const void* k, const float* wq, const float* wk, const int32_t* positions,
                 const float* inv_freq, int B, int Hq, int Hk, int N, int rot, int n_axes, const int* sections, int norm, float eps,
                 const int64_t* q_strides, const int64_t* k_strides) {
    p.x[0] = q; p.x[1] = k; p.w[0] = wq; p.w[1] = wk;
    p.pos = positions; p.inv_freq = inv_freq;
    for (int i = 0; i < 3; ++i) { p.st[0][i] = q_strides[i]; p.st[1][i] = k_strides[i]; }
    p.H[0] = Hq; p.H[1] = Hk; p.N = N; p.tokens = B * N; p.pairs = rot / 2; p.axes = n_axes;
    int end = 0;
    for (int a = 0; a < MAX_AXES; ++a) {
        if (rot > 0 && a < n_axes) end += sections ? sections[a] : rot / 2;
        p.end[a] = end;
    }
    for (int a = n_axes > 0 ? n_axes - 1 : 0; a < MAX_AXES; ++a) p.end[a] = rot / 2;     // the last axis takes what is left
    p.eps = eps; p.norm = norm;
}

// Work-groups: one for `sets` of tokens, and where these are fewer than `enough` one for each part of the heads as well.  (The angles of
// a token are formed once for each part.  Gradient of 16384 tokens of 32 heads: 512 work-groups 44 us, 1024 of half the heads 52; of
// 2174 tokens of 10 heads: 136 work-groups 11.0, 544 10.0.)
dim3 prep_grid(PrepParams& p, int sets, int enough) {
    const int heads = p.H[0] + p.H[1];
    int parts = 1;
    while (parts < heads && (long)sets * parts < enough) parts *= 2;
    p.heads_per_group = (heads + parts - 1) / parts;
    return dim3(sets, (heads + p.heads_per_group - 1) / p.heads_per_group);
}

template <class E, int D> void fwd_launch(const PrepParams& p, bool neighbours, dim3 grid, hipStream_t s) {
    if (neighbours) hipLaunchKernelGGL((qk_prep_kernel<E, D, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((qk_prep_kernel<E, D, false>), grid, dim3(256), 0, s, p);
}
template <class E, int D> void bwd_launch(const PrepParams& p, bool neighbours, dim3 grid, hipStream_t s) {
    if (neighbours) hipLaunchKernelGGL((qk_prep_bwd_kernel<E, D, true>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((qk_prep_bwd_kernel<E, D, false>), grid, dim3(256), 0, s, p);
}

}  // namespace

extern "C" {

int entmax_attn_qk_norm_rope_fwd(const void* q, const void* k, void* q_out, void* k_out,
                                 const int64_t* q_strides, const int64_t* k_strides,
                                 const float* q_weight, const float* k_weight, const int32_t* positions, const float* inv_freq,
                                 int B, int Hq, int Hk, int N, int d, int dtype,
                                 int rot, int n_axes, const int* sections, int interleaved, int norm, float eps, void* hip_stream) {
    const int rc = prep_check(q, k, B, Hq, Hk, N, d, dtype, positions, inv_freq, rot, n_axes, sections, norm, eps, q_weight, k_weight);
    if (rc) return rc;
    if (!q_out || !k_out || !q_strides || !k_strides) return EA_ERR_NULL;
    const int size = dtype == EA_BF16 ? 2 : 4;
    if (!strides_ok(q_strides, size) || !strides_ok(k_strides, size) || !aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out))
        return EA_ERR_LAYOUT;
    PrepParams p{};
    prep_params(p, q, k, q_weight, k_weight, positions, inv_freq, B, Hq, Hk, N, rot, n_axes, sections, norm, eps, q_strides, k_strides);
    p.y[0] = q_out; p.y[1] = k_out;
    const dim3 grid = prep_grid(p, (p.tokens + tokens_per_group(d) - 1) / tokens_per_group(d), 1024);
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == EA_BF16) { if (d == 64) fwd_launch<Bf16, 64>(p, interleaved, grid, s); else fwd_launch<Bf16, 128>(p, interleaved, grid, s); }
    else { if (d == 64) fwd_launch<F32, 64>(p, interleaved, grid, s); else fwd_launch<F32, 128>(p, interleaved, grid, s); }
    return launched();
}

size_t entmax_attn_qk_norm_rope_workspace_bytes(int d) {
    return d == 64 || d == 128 ? (size_t)BWD_GROUPS * 2 * d * sizeof(float) : 0;
}

int entmax_attn_qk_norm_rope_bwd(const void* q, const void* k, const float* dq_out, const float* dk_out, void* dq, void* dk,
                                 const int64_t* q_strides, const int64_t* k_strides, const int64_t* dq_strides, const int64_t* dk_strides,
                                 const float* q_weight, const float* k_weight, const int32_t* positions, const float* inv_freq,
                                 float* dq_weight, float* dk_weight,
                                 int B, int Hq, int Hk, int N, int d, int dtype,
                                 int rot, int n_axes, const int* sections, int interleaved, int norm, float eps,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = prep_check(q, k, B, Hq, Hk, N, d, dtype, positions, inv_freq, rot, n_axes, sections, norm, eps, q_weight, k_weight);
    if (rc) return rc;
    if (!dq_out || !dk_out || !dq || !dk || !q_strides || !k_strides || !dq_strides || !dk_strides) return EA_ERR_NULL;
    if (!norm && (dq_weight || dk_weight)) return EA_ERR_SHAPE;
    const int size = dtype == EA_BF16 ? 2 : 4;
    if (!strides_ok(q_strides, size) || !strides_ok(k_strides, size) || !strides_ok(dq_strides, size) || !strides_ok(dk_strides, size) ||
        !aligned16(q) || !aligned16(k) || !aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dq) || !aligned16(dk))
        return EA_ERR_LAYOUT;
    if (!rows_apart(dq_strides, {B, N, Hq}, d) || !rows_apart(dk_strides, {B, N, Hk}, d)) return EA_ERR_LAYOUT;
    const bool want_dw = dq_weight || dk_weight;
    if (want_dw && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < entmax_attn_qk_norm_rope_workspace_bytes(d)))
        return EA_ERR_WORKSPACE;
    PrepParams p{};
    prep_params(p, q, k, q_weight, k_weight, positions, inv_freq, B, Hq, Hk, N, rot, n_axes, sections, norm, eps, q_strides, k_strides);
    p.y[0] = dq; p.y[1] = dk; p.dy[0] = dq_out; p.dy[1] = dk_out;
    for (int i = 0; i < 3; ++i) { p.dst[0][i] = dq_strides[i]; p.dst[1][i] = dk_strides[i]; }
    p.part = want_dw ? (float*)workspace : nullptr;
    const int sets = (p.tokens + tokens_per_group(d) - 1) / tokens_per_group(d);
    dim3 grid = prep_grid(p, sets, 512);
    if (grid.x * grid.y > BWD_GROUPS) grid.x = BWD_GROUPS / grid.y;
    const int groups = grid.x * grid.y;
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == EA_BF16) { if (d == 64) bwd_launch<Bf16, 64>(p, interleaved, grid, s); else bwd_launch<Bf16, 128>(p, interleaved, grid, s); }
    else { if (d == 64) bwd_launch<F32, 64>(p, interleaved, grid, s); else bwd_launch<F32, 128>(p, interleaved, grid, s); }
    if (want_dw)
        hipLaunchKernelGGL(qk_prep_dw_kernel, dim3(2 * d / 16), dim3(1024), 0, s, p.part, dq_weight, dk_weight, groups, d);
    return launched();
}

}  // extern "C"
