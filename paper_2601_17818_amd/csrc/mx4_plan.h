// Which launches the calls on 4-bit caches and matrices go out as.  Arithmetic on sizes alone (no HIP), so that a test on the CPU
// can walk it.
#pragma once

#include <algorithm>
#include <cstdint>

namespace vitcop {

// ---- attention over a cache (mx4_attn.hip) ----------------------------------------------------------------------

constexpr int MA_MAX_G = 16, MA_KEYS = 32;           // query heads a pass, keys a wavefront at a time

// the columns of a product that a part of the probabilities takes, by the number of products
constexpr int ma_columns(int products) { return products == 1 ? 5 : (products == 2 ? 8 : 16); }
constexpr int attn_products(int heads) { return heads <= ma_columns(1) ? 1 : (heads <= ma_columns(2) ? 2 : 3); }

// How many slices of the keys and wavefronts to a slice.  A workgroup costs some two microseconds before its first and after
// its last key, the merge of slices three to four; a CU draws 31 KB/us (rows of 64: 22) with eight wavefronts on it, the chip
// 6.2 TB/s, 24 KB/us a CU.  Measured, us a call of captured ones, over caches of 600 MB in turn (pairs of a sample and a KV head
// x keys, of 128 or of 64, one query head):
//  - up to 128 pairs, one slice for up to one_slice_keys (in one, in slices: 32 x 650 7.5, 7.7; 32 x 1000 8.9, 7.8; 128 x 801 8.3,
//    9.4; 128 x 1200 10.3, 10.6; 128 x 1500 11.6, 10.9; of 64 32 x 1000 7.0, 7.1; 128 x 1200 8.0, 8.9; 128 x 2000 10.5, 9.9); above,
//    slices of 256 to 512 keys take four wavefronts (32 x 1500 in six, with four and eight wavefronts 7.9, 8.1); longer ones, of
//    fewer than 32 pairs, eight, one workgroup to a CU (16 x 65536 in 32 with four and in 16 with eight 28.9, 28.5), and of more
//    pairs four, three to a CU, which come out even where 256 is no multiple of the pairs (96 x 15000 in two, eight wavefronts
//    45.5, in eight, four 38.2; 64 x 40000 60.9, 60.0; of 64 42.7, 39.2).
//  - up to 512 pairs, slices of four wavefronts where some CUs would have a workgroup more than others for long enough to pay
//    for the merge (one slice, the plan's: 132 x 1800 12.6, 12.6; x 7200 35.8, 29.2; 232 x 7200 40.7, 40.7 (in three 42.5); 280 x 3600
//    34.8, 31.6; 340 x 14400 131, 113 (in three 108); of 64 87, 68; 512 x 14400 157, 157).
//  - of one slice the more pairs there are, the fewer wavefronts, and the more keys, the more: two, four, eight 640 x 150 7.1, 7.5,
//    9.7; 640 x 650 16.5, 14.6, 16.4; 1500 x 300 16.0, 16.6, 19.4; 1500 x 650 27.9, 26.8, 29.5; 3000 x 450 35.9, 35.9, 44.0;
//    3000 x 1000 71.8, 68.2, 76.8; four, eight 280 x 900 12.9, 13.6; 420 x 7200 78.0, 71.1; of 64 760 x 7200 76.6, 69.9; and none
//    of them to be without a key.
inline int64_t one_slice_keys(int64_t pairs, int d) {
    return d == 64 ? 1000 + 4 * pairs : 750 + std::max<int64_t>(0, pairs - 60) * 15 / 2;
}
struct AttnPlan {
    int waves, keys_per_split, splits;
};
inline AttnPlan attn_plan(int B, int N, int Hkv, int d) {
    const int64_t pairs = (int64_t)B * Hkv;
    AttnPlan p{8, 0, 1};
    if (pairs <= 128) {
        if (N > one_slice_keys(pairs, d)) {
            p.waves = 4;
            p.splits = (int)std::min<int64_t>(512 / pairs, (N + 255) / 256);
            if ((N + p.splits - 1) / p.splits > 512)
                p = pairs < 32 ? AttnPlan{8, 0, (int)(256 / pairs)} : AttnPlan{4, 0, (int)(768 / pairs)};
        }
    } else if (pairs <= 512 && N > 800) {
        const float pair_us = (float)N * (float)(d * 17 / 16) / (d == 64 ? 22e3f : 31e3f);          // of a CU
        const float chip_us = (float)pairs * (float)N * (float)(d * 17 / 16) / 6.2e6f;
        float least = 1e30f;
        for (int s = 1; s <= 4; ++s) {
            const float us = std::max(chip_us, pair_us / s * (float)((pairs * s + 255) / 256)) + (s > 1 ? 4.f : 0.f);
            if (us < least) {
                least = us;
                p.splits = s;
            }
        }
        if (p.splits > 1) p.waves = 4;
    }
    if (p.splits == 1) {
        if (pairs > 256 && (N <= 1500 || pairs > (d == 64 ? 1024 : 512))) p.waves = 4;
        if ((pairs > 768 && N <= (pairs > 2048 ? 800 : 400)) || (pairs > 512 && N <= 160)) p.waves = 2;
        while (p.waves > 2 && (p.waves / 2) * MA_KEYS >= N) p.waves /= 2;
    }
    const int64_t unit = p.waves * MA_KEYS, keys = (N + p.splits - 1) / p.splits;
    p.keys_per_split = (int)std::min<int64_t>(std::max<int64_t>(1, (keys + unit - 1) / unit) * unit, INT32_MAX);
    p.splits = (int)std::max<int64_t>(1, ((int64_t)N + p.keys_per_split - 1) / p.keys_per_split);
    return p;
}

// ---- projections by a matrix (mx4_project.hip) ------------------------------------------------------------------

// At most sixteen rows of x.  A workgroup reads its rows of x whatever it takes of W, so of more than four rows it takes as many
// blocks of 16 rows of W, up to four, as give the CUs' rounds the least cost: one up to 256 blocks, two up to 512, three (11008
// rows) up to 768.  Up to four rows of x are cheap: two blocks where the CUs' rounds of one are even, so that half as many do.
// Eight wavefronts where a CU has one workgroup, columns enough for them and no more of x than of W.  Measured, us a call of
// captured ones, over matrices of 600 MB in turn, 16, 32, 48, 64 rows of W:
//  - 8 x 8192 x 8192 10.9, 9.7, 11.6, 13.0; 8 x 11008 x 4096 9.4, 9.5, 7.9, 8.5; 8 x 28672 x 4096 18.4, 15.9, 16.4, 15.1; 16 x 4096 x 4096
//    5.8, 6.9, 7.7, 8.4; 16 x 8192 x 4096 9.2, 7.5, 8.3, 8.9; 16 x 11008 x 4096 13.5, 11.3, 9.0, 9.5; 16 x 14336 x 4096 15.1, 11.1, 13.0, 9.9.
//  - 16 and 32: 1 x 11008 x 4096 7.0, 7.6; 1 x 16384 x 2048 6.0, 5.7; 1 x 20480 x 4096 10.5, 11.1; 1 x 14336 x 14336 23.5, 22.5; 2 x 12288 x
//    4096 7.2, 7.9; 2 x 14336 x 4096 8.4, 8.2; 2 x 28672 x 4096 13.2, 14.0; 4 x 14336 x 14336 27.9, 23.9; 4 x 57344 x 1024 9.3, 9.0; and with
//    three steps in flight 4 x 6144 x 4096 6.1, 5.7; 4 x 8192 x 8192 10.1, 9.6; 4 x 8192 x 2048 4.6, 4.5.
//  - four and eight wavefronts: 1 x 4096 x 1024 2.9, 3.0; x 2048 3.3, 3.4; x 4096 5.3, 4.5; x 8192 8.3, 6.3; 4 x 2048 x 1536 3.0, 3.0;
//    8 x 4096 x 2048 3.5, 3.5; x 14336 12.3, 10.3.
inline float few_us(int64_t tiles, int blocks, int K) {          // of the CUs' rounds: a workgroup's x, and its rows of W
    return (float)(((tiles + blocks - 1) / blocks + 255) / 256) * (0.234f * blocks + 0.27f) * (1e-3f * (float)K);
}
inline int few_blocks(int64_t tiles, int K) {                // of 16 rows of W, for more than four rows of x
    int best = 1;
    for (int blocks = 2; blocks <= (K <= 32768 ? 4 : 3); ++blocks)           // (the rows' exponents are in LDS, too)
        if (few_us(tiles, blocks, K) < few_us(tiles, best, K)) best = blocks;
    return best;
}

struct FewPlan {
    int blocks, x_loads, waves, depth;   // of 16 rows of W a workgroup, of four rows of x a step; steps in flight
};
inline FewPlan few_plan(int M, int N, int K) {
    const int tiles = N / 16;
    if (M <= 4) {
        if (tiles <= 256) return K <= 1024 ? FewPlan{1, 1, 4, 2} : FewPlan{1, 1, 8, 3};
        if (tiles <= 512 && K > 2048) return {2, 1, 4, 3};
        return tiles > 512 && (tiles + 255) / 256 % 2 == 0 ? FewPlan{2, 1, 4, 2} : FewPlan{1, 1, 4, 2};
    }
    const int blocks = few_blocks(tiles, K);
    if (M <= 8) {
        if (blocks == 1) return K <= 2048 ? FewPlan{1, 2, 4, 2} : FewPlan{1, 2, 8, 2};
        return {blocks, 2, 4, blocks == 2 ? 3 : 2};
    }
    return {blocks, 4, 4, blocks == 1 ? 3 : 2};
}

// Which launch: sixteen rows of x at a time, tiles of 32 mb with k in how many slices, or the matrix to bf16 and the bf16
// projection.  By estimated time, us, fitted to some 400 sizes of 17 to 5500 rows with weights from HBM, where it loses
// 0.7 % against the better of the three:
//  - sixteen rows at a time: 2.2, 0.5 for every 256 workgroups and for each of them a CU takes 0.5, 0.74 or 1.2 for a thousand
//    columns (16, 32 or 64 rows of W, few_us); W is read again for every sixteen rows of x;
//  - tiles: 2 + rt + 0.5 mb for the launch, the first loads and the end, then rounds of 256 workgroups over the slice's steps (a
//    CU holds two of the smallest, which overlap); a further round costs 1 + 0.4 mb rt, a MB of y 0.15, slices 3 for the kernel
//    that adds them up and 0.2 a MB;
//  - by way of bf16: 8.1 for two launches, for a million values of the matrix 0.27, of y 1.4, for a thousand columns 3.6, and
//    1.7 PFLOP/s.
// Measured, us a call of captured ones, over matrices of 600 MB in turn:
//  - sixteen at a time, tiles: 48 x 4096 x 4096 12.0, 13.4; 80 rows 17.4, 15.3; 24 x 4096 x 14336 20.0, 15.2; 48 x 11008 x 4096 17.4, 19.5;
//    64 x 8192 x 4096 15.8, 14.3; 80 x 4096 x 512 7.7, 5.2 (with 80 x 4096 x 4096 the worst choices found).
//  - tiles of 128 and of 256 rows of W: 317 x 3584 x 14336 48.8, 47.9; 128 x 4096 x 4096 17.3, 26.3; 640 x 4096 x 11008 70.0, 64.2;
//    1024 x 4096 x 4096 40.7, 44.7; x 11008 101, 90.2; 1536 x 4096 x 4096 88.4, 50.4; 1024 x 3584 x 14336 144, 109.
//  - slices: 64 x 4096 x 11008 in eight 17.6, in four 22.6; 64 x 11008 x 4096 in one 19.8, in two 20.6; 200 x 4096 x 4096 in one 19.1, in
//    two 21.1; 300 x 4096 x 4096 in four 24.4, in one 24.4, in two 31.7.
//  - tiles, bf16: 1024 x 4096 x 4096 40.7, 50.4; 2048 rows 62.7, 69.4; 2048 x 11008 x 4096 186, 159; 2251 x 6112 x 7968 233, 217.
struct MpKind {                          // of tiles: 32 mb rows of x by 64 rt rows of W, us a step of 128 columns
    int mb, rt;
    float step_us;
};
inline constexpr MpKind mp_kinds[] = {{1, 2, 0.46f}, {2, 2, 0.66f}, {3, 2, 0.93f}, {4, 2, 1.14f}, {5, 2, 1.34f},
                               {3, 4, 1.35f}, {4, 4, 1.72f}, {5, 4, 2.15f}};
struct MpPlan {
    int kind, slices, steps_per_slice;   // kind < 0: mx4_few_kernel
    bool unpack;                         // the matrix to bf16 first, if there is scratch for it
};
inline MpPlan mp_plan(int M, int N, int K) {
    MpPlan best{-1, 1, 0, false};
    if (M <= 16) return best;
    const int steps = (K + 127) / 128;
    const int few = few_blocks(N / 16, K);
    const int64_t few_groups = (int64_t)((N / 16 + few - 1) / few) * ((M + 15) / 16);
    float least = 2.24f + few_us(few_groups * few, few, K) + 0.544f * few_groups / 256;
    for (int kind = 0; kind < 8 && K >= 512; ++kind) {
        const int mb = mp_kinds[kind].mb, rt = mp_kinds[kind].rt;
        const int64_t tiles = (int64_t)((N + 64 * rt - 1) / (64 * rt)) * ((M + 32 * mb - 1) / (32 * mb));
        const float fixed = 2.f + rt + 0.5f * mb + 0.3e-6f * (float)M * (float)N;
        for (int want = 1, last = 0; want <= 16 && want <= steps / 4 && (want == 1 || tiles * want <= 1024); ++want) {
            const int per = (steps + want - 1) / want;
            if (per == last) continue;
            last = per;
            const int slices = (steps + per - 1) / per;                                        // (none of them empty)
            const int64_t rounds = (tiles * slices + 255) / 256;
            const float overlap = rounds > 1 && mb == 1 ? 0.84f : 1.f;
            float us = fixed + (float)rounds * overlap * per * mp_kinds[kind].step_us + (1.f + 0.4f * mb * rt) * (rounds - 1);
            if (slices > 1) us += 3.f + 0.8e-6f * slices * (float)M * (float)N;
            if (us < least) {
                least = us;
                best = {kind, slices, per, false};
            }
        }
    }
    const float m = (float)M, n = (float)N, k = (float)K;
    best.unpack = 8.1f + 0.274e-6f * n * k + 1.38e-6f * m * n + 3.55e-3f * k + 1.19e-9f * m * n * k < least;
    return best;
}

}  // namespace vitcop
