// Which launches attention over a cache's rows (span_attn.hip) goes out as.  Arithmetic on sizes alone (no HIP), so that a
// test on the CPU can walk it.
#pragma once

#include <algorithm>
#include <cstdint>

namespace vitcop {

constexpr int SP_KEYS = 32, SP_WAVES = 4;            // keys a wavefront at a time, wavefronts that share a slice

// Query rows of a KV head are its tokens' heads, R = T * G of them.  A workgroup takes 16 `blocks` of them (wide: 128
// `blocks`, attn_wide_kernel) and one of `slices` of the keys.
struct SpanPlan {
    bool wide;
    int blocks, row_blocks, slices;
};
// keys: the most rows that a block of query rows looks at; fits: whether the wide kernel's offsets hold them
inline SpanPlan span_plan(int64_t B, int64_t Hkv, int64_t rows, int64_t keys, int d, bool fits) {
    SpanPlan p{};
    p.wide = fits && rows > 64;
    p.blocks = p.wide ? (d == 128 && rows >= 256 ? 2 : 1) : (rows <= 16 ? 1 : (rows <= 32 ? 2 : 4));
    const int unit = p.blocks * (p.wide ? 128 : 16), tile = p.wide ? 64 : SP_KEYS * SP_WAVES;
    p.row_blocks = (int)((rows + unit - 1) / unit);
    const int64_t wgs = B * Hkv * p.row_blocks, tiles = (keys + tile - 1) / tile;
    p.slices = (int)std::max<int64_t>(1, std::min<int64_t>((512 + wgs - 1) / std::max<int64_t>(wgs, 1), tiles / (p.wide ? 4 : 2)));
    return p;
}

}  // namespace vitcop
