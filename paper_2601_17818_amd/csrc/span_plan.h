// Which launches attention over a cache's rows (span_attn.hip) goes out as.  Arithmetic on sizes alone (no HIP), so that a
// test on the CPU can walk it.
#pragma once

#include <algorithm>
#include <cstdint>

namespace vitcop {

constexpr int SP_KEYS = 32, SP_WAVES = 4;            // keys a wavefront at a time, wavefronts that share a slice

// Query rows of a KV head are its tokens' heads, R = T * G of them; a workgroup takes 16 `blocks` of them and one of
// `slices` of the keys.
struct SpanPlan {
    int blocks, row_blocks, slices;
};
// keys: the most rows that a block of query rows looks at
inline SpanPlan span_plan(int64_t B, int64_t Hkv, int64_t rows, int64_t keys, int d) {
    (void)d;
    SpanPlan p;
    p.blocks = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    p.row_blocks = (int)((rows + 16 * p.blocks - 1) / (16 * p.blocks));
    const int64_t wgs = B * Hkv * p.row_blocks, tiles = (keys + SP_KEYS - 1) / SP_KEYS;
    p.slices = (int)std::max<int64_t>(1, std::min<int64_t>((512 + wgs - 1) / std::max<int64_t>(wgs, 1), tiles / (2 * SP_WAVES)));
    return p;
}

}  // namespace vitcop
