// Layout of the 4-bit key/value cache, shared by the kernels that write, read and attend to it.
// A page holds `page` tokens of all Hk heads, [n_pages][Hk][page_bytes]; a head's part of a page is
//   key codes [page][d/2], key scales [page][d/32], value codes [page][d/2], value scales [page][d/32].
// 32 neighbouring values share the scale 2^(byte - 127) (byte 255: not finite); a code is a sign above the three bits of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6, the value with the lower index in the lower half of its byte.  These are the operand and
// scale formats of the gfx950 matrix instructions: a tile of key codes goes from memory to the matrix cores unchanged.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "tiles.hpp"

namespace ea {

// The scale of a byte.  (Byte 0, which no write leaves: 2^-127 is subnormal, the bit below the exponent's first.)
EA_DEV float cache4_scale(unsigned int byte) { return byte == 255u ? __builtin_nanf("") : __uint_as_float(byte ? byte << 23 : 1u << 22); }

constexpr int cache_page_bytes(int d, int page) { return page * 2 * (d / 2 + d / 32); }   // of one head's part

// Slots are 32-bit: token `slot % page` of page `slot / page`.
inline bool cache_page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128 || page == 256; }
inline int cache_page_shift(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : 8; }

}  // namespace ea
