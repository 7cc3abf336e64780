// Which launches attention of tokens and drafts over a cache's rows (span_attn.hip) goes out as.  Arithmetic on sizes alone (no
// HIP), so that a test on the CPU can walk it.
#pragma once

#include <algorithm>
#include <cstdint>

namespace vitcop {

constexpr int SP_KEYS = 32, SP_WAVES = 4;            // span_attn_kernel: keys a wavefront at a time, wavefronts of a slice
constexpr int SP_FEW_ROWS = 32;                      // query rows that it takes at most, where the other one's offsets fit

// Query rows of a KV head are its tokens' heads, T * G of them.  A workgroup takes 16 `blocks` of them (wide: 128 `blocks`,
// attn_wide_kernel) and one of `slices` of the keys.
struct SpanPlan {
    bool wide;
    int blocks, row_blocks, slices;
};

// T tokens over `start` rows and their own (a tree's: the drafts), or a window of them and the sinks.
struct SpanSizes {
    int64_t B, Hkv, T, G, start, window, sinks;
    int d;
    bool tree, own;                                  // own: samples have lengths of their own
    // Their order and their slices go by those lengths, unless a window makes most of them alike.
    bool ragged() const { return own && B > 1 && (window == 0 || start < 2 * window); }
};

// The kernels are priced in us and the cheapest kind, number of blocks and of slices is taken.  What a launch streams costs its
// bytes at the chip's 5.8 (wide: 5.2) TB/s, or what the fullest CU has to do, whichever is more; slices cost their merge, 3 and
// its bytes, and 2 more for the second launch, which is what a program that captures nothing waits for where all this is short.
//
// Few rows, in steps of 128 keys of a workgroup.  A CU with a workgroup alone takes 1.55 us a step (d = 64: 0.85), 2.1 (1.1)
// where all CUs have one, and 2.5 (1.25) where some have more; measured, us by the number of slices (pairs of a sample and a KV
// head x keys, of 128): 32 x 300 1: 9.5, 4: 9.6; x 600 1: 11.8, 4: 10.6, 8: 10.6; x 1200 1: 17.0, 4: 12.9, 8: 11.8, 16: 12.1;
// x 16000 1: 206, 8: 53.1; 96 x 600 1: 11.9, 2: 13.7; x 4000 1: 61.5, 2: 44.6; 288 x 2000 1: 73.8, 2: 66.6, 4: 61.5; 320 x 4000
// 1: 145, 3: 121; 512 x 300 1: 20.2, 2: 24.4; x 3000 1: 136, 2: 141; 4 x 16000 of 7 query heads 16: 19.4, 64: 14.7, 128: 17.1;
// of 64: 4 x 600 1: 7.4, 4: 7.8; x 4000 1: 22.2, 32: 9.0; 64 x 300 1: 7.0, 2: 9.3; x 3000 1: 27.0, 4: 17.4.
//
// Many rows, in tiles of 64 keys: one block of 128 rows takes 0.88 us a tile where CUs are left over and 1.0 where not, and 7 to
// begin and end; two blocks 1.6 to 1.8 and 8, so that one is better where a workgroup has few tiles or all fit at once, two where
// there are rounds of workgroups.  (Drafts take one: with two the registers do not hold the masks, 2.0 us a tile even on an idle
// chip.  Those of d = 64 are priced like windows, three workgroups to a CU, though their 170 registers leave room for two.)
// Measured, us: 317 tokens of 7 query heads x 4 KV heads behind 16384 rows one block 3: 91.0, 7: 93.5, two 3: 132, 5: 89.6, 7: 81.9,
// 14: 98.4; 100 behind 8000 one 4: 38.8, 8: 29.0, 10: 30.4, two 7: 40.2, 21: 31.9; 2 x 8192 with a window of 2048 one 487, two 421;
// 2 x 2000 with one of 500 54.6, 53.3; 640 tokens of 32 heads 15.9, 24.8; 8 x 64 drafts x 28 / 4 heads behind 4096 1: 63.1, 2: 47.9,
// 3: 62.1; of 64: 4 x 64 x 16 / 4 behind 3000 1: 38.8, 4: 19.7, 8: 18.3, 16: 25.4.
// Samples of their own lengths: 64 x up to 16000 keys x 28 / 4 1: 263, 2: 211, 8: 224; 12 x 8000 x 16 1: 127, 2: 98.6, 4: 86.7;
// 40 x 8000 x 28 / 4 1: 116, 3: 75.9, 8: 80.4; 20 x 3000 x 32 1: 104, 2: 112; 8 x 700 tokens behind 3000 x 28 / 4 two blocks 1: 103,
// 2: 135.
inline SpanPlan span_plan(const SpanSizes& z, bool fits) {
    const int64_t rows = z.T * z.G, pairs = z.B * z.Hkv, all = z.start + z.T;
    SpanPlan best{};
    best.wide = fits && rows > SP_FEW_ROWS;
    float least = 0.f;
    auto price = [&](int blocks, int64_t slices, bool first) {
        SpanPlan p{best.wide, blocks, 0, (int)slices};
        const int64_t unit = blocks * (p.wide ? 128 : 16), in_block = std::min(z.T, unit / z.G + 2);   // tokens of a block
        p.row_blocks = (int)((rows + unit - 1) / unit);
        const int64_t wgs = pairs * p.row_blocks * slices, on_cu = (wgs + 255) / 256;
        // rows that a block looks at, the last one and, where workgroups take turns, the middle one
        const int64_t keys = z.window ? std::min(all, z.window + in_block + z.sinks) : all;
        const int64_t mean = z.tree || wgs <= 256 ? keys : std::min(keys, z.start + (z.T + 1) / 2 + in_block);
        const float bytes = (float)pairs * (float)std::min(all, z.window ? z.window + z.T + z.sinks : all) * (float)(4 * z.d);
        const int tile = p.wide ? 64 : SP_KEYS * SP_WAVES;
        const float steps = (float)(((mean + tile - 1) / tile + slices - 1) / slices);
        const bool d64 = z.d == 64;
        // samples of their own lengths: some 0.6 of the longest one's keys in the mean, and a CU that begins with a long one goes
        // on with a short one
        const float share = z.ragged() ? 0.6f : 1.f, load = z.ragged() && on_cu > 1 ? 0.62f : 1.f;
        float us;
        if (!p.wide) {
            const float step = wgs <= 128 ? (d64 ? 0.85f : 1.55f) : (wgs <= 256 ? (d64 ? 1.1f : 2.1f) : (d64 ? 1.25f : 2.5f));
            us = std::max(share * bytes / 5.8e6f, load * (float)on_cu * steps * step);
        } else {
            const float step = d64 ? 0.65f : (blocks == 2 ? (wgs <= 128 ? 1.6f : 1.8f) : (wgs <= 128 ? 0.88f : 1.0f));
            const float ends = blocks == 2 ? 8.f : 7.f, rounds = wgs > 512 ? (float)wgs / 256.f + 0.3f : (float)on_cu;
            us = std::max(share * bytes / 5.2e6f, std::max(1.f, load * rounds) * steps * step) +
                 (d64 ? (float)((wgs + 767) / 768) : rounds) * ends;
        }
        if (slices > 1) us += 5.f + (float)(pairs * rows * slices) * (float)(8 * z.d) / 6e6f;
        if (first || us < least) {
            least = us;
            best = p;
        }
    };
    const int few = rows <= 16 ? 1 : 2, most = best.wide && z.d == 128 && !z.tree ? 2 : 1;
    const int64_t keys = z.window ? std::min(all, z.window + z.T + z.sinks) : all;
    bool first = true;
    for (int i = 1; i <= most; ++i) {
        const int blocks = best.wide ? i : few, tile = best.wide ? 128 : SP_KEYS * SP_WAVES;          // (two tiles a slice)
        const int64_t unit = blocks * (best.wide ? 128 : 16), wgs = pairs * ((rows + unit - 1) / unit);
        const int64_t cap = std::max<int64_t>(1, std::min<int64_t>((keys + tile - 1) / tile, 1024 / std::max<int64_t>(wgs, 1)));
        for (const int64_t s : {(int64_t)1, (int64_t)2, (int64_t)3, (int64_t)4, (int64_t)6, 128 / wgs, 256 / wgs, 512 / wgs, cap})
            if (s >= 1 && s <= cap) {
                price(blocks, s, first);
                first = false;
            }
    }
    return best;
}

}  // namespace vitcop
