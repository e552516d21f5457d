// Driver for the host-sanitizer build of the operators' boundary: every call must return before anything is enqueued.
#include <stdio.h>

#include "../../include/entmax_attn.h"

#define CHECK(cond) do { if (!(cond)) { printf("failed: %s (line %d)\n", #cond, __LINE__); return 1; } } while (0)

int main() {
    alignas(256) static float x[1024];
    alignas(256) static char ws[1024];
    static int32_t m[64], n[64];
    int64_t st[3] = {128, 64, 64}, zero[3] = {0, 64, 64};
    const int sections[2] = {16, 17};
    auto fwd = [&](int d, int dtype, int axes, const int* sec, const int64_t* s) {
        return entmax_attn_qk_norm_rope_fwd(x, x, x, x, s, st, nullptr, nullptr, m, x, 1, 1, 1, 2, d, dtype, 64, axes, sec, 0, 1, 1e-6f, nullptr);
    };
    CHECK(fwd(96, EA_F32, 1, nullptr, st) == EA_ERR_SHAPE);
    CHECK(fwd(64, 5, 1, nullptr, st) == EA_ERR_DTYPE);
    CHECK(fwd(64, EA_F32, 2, sections, st) == EA_ERR_SHAPE);
    CHECK(fwd(64, EA_F32, 2, nullptr, st) == EA_ERR_NULL);
    CHECK(fwd(64, EA_F32, 1, nullptr, nullptr) == EA_ERR_NULL);
    CHECK(entmax_attn_qk_norm_rope_bwd(x, x, x, x, x, x, st, st, zero, st, nullptr, nullptr, m, x, x, x, 2, 1, 1, 2, 64, EA_F32, 64, 1, nullptr, 0, 1,
                                       1e-6f, ws, sizeof ws, nullptr) == EA_ERR_LAYOUT);
    CHECK(entmax_attn_qk_norm_rope_bwd(x, x, x, x, x, x, st, st, st, st, nullptr, nullptr, m, x, x, x, 1, 1, 1, 2, 64, EA_F32, 64, 1, nullptr, 0, 1,
                                       1e-6f, ws, sizeof ws, nullptr) == EA_ERR_WORKSPACE);
    CHECK(entmax_attn_qk_norm_rope_workspace_bytes(64) > 0 && entmax_attn_qk_norm_rope_workspace_bytes(1) == 0);
    CHECK(entmax_attn_cache_tables(m, n, m, m, m, n, m, m, m, m, 1, 4, 16, 8, 4, nullptr) == EA_ERR_LAYOUT);
    CHECK(entmax_attn_cache_tables(m, n, m, m, m, m, m, m, m, m, 5000, 4, 16, 8, 4, nullptr) == EA_ERR_SHAPE);
    CHECK(entmax_attn_cache4_page_bytes(2, 64, 16) == 2 * 16 * 68 && entmax_attn_cache4_page_bytes(2, 64, 17) == 0);
    CHECK(entmax_attn_cache4_write(x, x, st, st, m, ws, 0, 1, 64, EA_F32, 1, 16, nullptr) == EA_OK);
    CHECK(entmax_attn_cache4_read(ws, m, x, x, zero, st, 2, 1, 64, EA_F32, 1, 16, nullptr) == EA_ERR_LAYOUT);
    CHECK(entmax_attn_decode_cache4_workspace_bytes(64, 32, 8, 128, 1 << 22) > 0);
    CHECK(entmax_attn_decode_cache4_workspace_bytes(1, 3, 2, 128, 64) == 0);
    CHECK(entmax_attn_decode_cache4(x, ws, m, m, x, x, nullptr, 1, 2, 1, 64, EA_F32, 64, 4, 1, 16, 1.f, ws, sizeof ws, nullptr) == EA_ERR_ALPHA);
    CHECK(entmax_attn_decode_cache4(x, ws, m, m, x, x, nullptr, 1, 2, 1, 64, EA_F32, 64, 4, 1, 16, 1.5f, ws, 16, nullptr) == EA_ERR_WORKSPACE);
    printf("ok\n");
    return 0;
}
