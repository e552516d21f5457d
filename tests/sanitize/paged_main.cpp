// Driver for the host-sanitizer build of the boundary of the 8-bit cache and of shared pages: every call must return before anything is
// enqueued.
#include <stdio.h>

#include "../../include/entmax_attn.h"

#define CHECK(cond) do { if (!(cond)) { printf("failed: %s (line %d)\n", #cond, __LINE__); return 1; } } while (0)

int main() {
    alignas(256) static float x[1024];
    alignas(256) static char ws[1024];
    alignas(16) static int32_t m[64], n[64];
    int64_t st[2] = {64, 64}, zero[2] = {0, 64};
    CHECK(entmax_attn_cache8_page_bytes(2, 64, 16) == 2 * (2 * 16 * 64 + 16) && entmax_attn_cache8_page_bytes(65535, 128, 256) > 0);
    CHECK(entmax_attn_cache8_page_bytes(2, 64, 17) == 0 && entmax_attn_cache8_page_bytes(65536, 64, 16) == 0);
    CHECK(entmax_attn_cache8_write(x, x, st, st, m, ws, 0, 1, 64, EA_F32, 1, 16, nullptr) == EA_OK);
    CHECK(entmax_attn_cache8_write(x, x, st, st, m, ws, 2147483647, 65535, 128, EA_BF16, 1, 16, nullptr) == EA_ERR_SHAPE);
    CHECK(entmax_attn_cache8_read(ws, m, x, x, zero, st, 2, 1, 64, EA_F32, 1, 16, nullptr) == EA_ERR_LAYOUT);
    for (int window : {0, 1, 63, 64, 65, 66, 1 << 22, 2147483647})
        for (int sinks : {0, 1, 64, 2147483647})
            CHECK(entmax_attn_decode_cache8_workspace_bytes(64, 32, 8, 128, 1 << 22, window, sinks) > 0);
    CHECK(entmax_attn_decode_cache8_workspace_bytes(65535, 65535, 1, 128, 1 << 22, 0, 0) > 0);
    CHECK(entmax_attn_decode_cache8_workspace_bytes(1, 3, 2, 128, 64, 0, 0) == 0);
    CHECK(entmax_attn_decode_cache8(x, ws, m, m, x, x, nullptr, 1, 2, 1, 64, EA_F32, 64, 4, 1, 16, 2147483647, 2147483647, 1.f, ws, sizeof ws, nullptr) == EA_ERR_ALPHA);
    CHECK(entmax_attn_decode_cache8(x, ws, m, m, x, x, nullptr, 1, 2, 1, 64, EA_F32, 64, 4, 1, 16, 1, 1, 1.5f, ws, 16, nullptr) == EA_ERR_WORKSPACE);
    CHECK(entmax_attn_cache_fork_workspace_bytes(4096, 1 << 18) > 0 && entmax_attn_cache_fork_workspace_bytes(4096, (1 << 18) + 1) == 0);
    CHECK(entmax_attn_cache_fork(m, m, m, m, m, m, m, n, m, m, 1, 4, 16, 8, ws, 16, nullptr) == EA_ERR_WORKSPACE);
    CHECK(entmax_attn_cache_fork(m, m, n, m, m, m, m, n, m, m, 1, 4, 16, 8, ws, sizeof ws, nullptr) == EA_ERR_LAYOUT);
    CHECK(entmax_attn_cache_compact_workspace_bytes(1 << 27) > 0 && entmax_attn_cache_compact_workspace_bytes((1 << 27) + 1) == 0);
    CHECK(entmax_attn_cache_compact(m, m, m, m, nullptr, m, m, n, m, m, 1, 4, 16, 8, ws, sizeof ws, nullptr) == EA_ERR_NULL);
    CHECK(entmax_attn_cache_compact(m, m, m, m, n, m, m, n, m, m, 1, 1 << 20, 16, 8, ws, sizeof ws, nullptr) == EA_ERR_SHAPE);
    CHECK(entmax_attn_cache_copy(ws, ws, m, n, 1, (size_t)-16, 4, 4, nullptr) == EA_ERR_SHAPE);
    CHECK(entmax_attn_cache_copy(ws, ws, m, n, 1, 8, 4, 4, nullptr) == EA_ERR_LAYOUT);
    CHECK(entmax_attn_cache_copy(ws, ws, nullptr, n, 0, 16, 4, 4, nullptr) == EA_OK);
    printf("ok\n");
    return 0;
}
