// 16-byte units that two neighbouring ones make.
#pragma once

#include <cstdint>

namespace aloco {

// The 16 bytes that begin `bytes` (2..14, even) before the end of prev and go on
// into cur.
__device__ __forceinline__ uint4 join_units(const uint4 &prev, const uint4 &cur, int bytes) {
    const uint32_t c[8] = {prev.x, prev.y, prev.z, prev.w, cur.x, cur.y, cur.z, cur.w};
    const int words = bytes >> 2;
    uint32_t t[5];  // words 3 - words and on
#pragma unroll
    for (int i = 0; i < 5; ++i)
        t[i] = words & 2 ? (words & 1 ? c[i] : c[i + 1]) : (words & 1 ? c[i + 2] : c[i + 3]);
    const uint32_t pick = bytes & 2 ? 0x5432u : 0x7654u;
    return make_uint4(__byte_perm(t[0], t[1], pick), __byte_perm(t[1], t[2], pick),
                      __byte_perm(t[2], t[3], pick), __byte_perm(t[3], t[4], pick));
}

}  // namespace aloco
