// Pages of a cache: sizes, slots, and the items (pages, token rows) of requests.
#pragma once
#include "tiles.hpp"

namespace ea {

// Slots are 32-bit: token `slot % page` of page `slot / page`.
inline bool cache_page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128 || page == 256; }
inline int cache_page_shift(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : 8; }

EA_DEV int pages_of(int len, int shift) { return (len + (1 << shift) - 1) >> shift; }

// largest r with pref[r] <= i, for i < pref[R] (so that request r has an item i)
EA_DEV int owner(const int32_t* pref, int R, int i) {
    int lo = 0, hi = R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pref[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

// inclusive sum over the lanes up to this one, by data-parallel-primitive adds (through LDS each of the six steps waits for its
// predecessor's round trip)
template <int CTRL, int ROWS> EA_DEV int scan_step(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
EA_DEV int wave_scan(int v) {
    v = scan_step<0x111, 0xf>(v);        // row_shr 1, 2, 4, 8: within sixteen lanes
    v = scan_step<0x112, 0xf>(v);
    v = scan_step<0x114, 0xf>(v);
    v = scan_step<0x118, 0xf>(v);
    v = scan_step<0x142, 0xa>(v);        // row_bcast 15: the row before, to the odd rows
    v = scan_step<0x143, 0xc>(v);        // row_bcast 31: the lower half, to the upper one
    return v;
}

}  // namespace ea
