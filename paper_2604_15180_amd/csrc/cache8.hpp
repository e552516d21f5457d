// Layout of the 8-bit key/value cache, shared by the kernels that write, read and attend to it.
// A page holds `page` tokens of all Hk heads, [n_pages][Hk][part bytes]; a head's part of a page is
//   key codes [page][d], value codes [page][d], key scales [page/16], value scales [page/16] (float32), unused up to a multiple of 16.
// The d values of 16 neighbouring tokens share a scale: value = code * |scale|, code -127 .. 127; code -128 is not a number, and the
// sign bit of a scale says that its block may hold such codes, so that nobody has to look for them elsewhere.  Sixteen tokens are
// the keys of one tile of the 16-column matrix instructions: a tile of codes goes from memory to the matrix cores unchanged, and its
// integer products are exact and have one factor.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "pages.hpp"
#include "tiles.hpp"

namespace ea {

constexpr int C8_BLOCK = 16;           // tokens per scale

constexpr int cache8_part_bytes(int d, int shift) { return ((2 * d) << shift) + (shift > 4 ? 8 << (shift - 4) : 16); }
// Scale `block` of the keys or the values (which) of a head's part
EA_DEV float* cache8_scale(unsigned char* part, int d, int shift, int which, int block) {
    return (float*)(part + ((2 * d) << shift) + 4 * ((which << (shift - 4)) + block));
}
EA_DEV const float* cache8_scale(const unsigned char* part, int d, int shift, int which, int block) {
    return cache8_scale(const_cast<unsigned char*>(part), d, shift, which, block);
}
// Whether one of four codes is -128
EA_DEV bool cache8_odd(unsigned int codes) {
    const unsigned int y = codes ^ 0x80808080u;
    return ((y - 0x01010101u) & ~y & 0x80808080u) != 0;
}
// Eight values in units of the scale; `strange`: codes -128 become NaN
EA_DEV void cache8_expand(uint2 codes, bool strange, float* v) {
    const int w[2] = {(int)codes.x, (int)codes.y};
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)(signed char)(w[k >> 2] >> (8 * (k & 3)));
    if (strange) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] == -128.f ? __builtin_nanf("") : v[k];
    }
}

}  // namespace ea
