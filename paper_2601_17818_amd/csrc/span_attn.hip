// Attention of few or many tokens over the rows of a cache, o = softmax(scale q K^T) V of each, as two spans of rows: for a
// window the first rows (sinks), which all see, and the rows up to the tokens' own; for a tree of drafts the cache's rows,
// which all see, and the drafts.  Bound by the cache's bytes while a KV head's query rows are few, by the matrix cores and the
// vector pipe beside them from about a hundred on.
//
// The query rows of a KV head (its tokens' heads, token after token) share its K and V.  A workgroup takes 16 NB of these
// rows and a slice of the keys, a wavefront 32 keys at a time: scores S^T = K Q^T (16x16x32: a lane holds 4 keys of one
// row), the softmax with the lane's row as its only query, O^T += V^T P^T.
//  - K goes from memory straight into the product, V through the wavefront's own piece of LDS and back transposed
//    (ds_read_b64_tr_b16).  The key of element 4 t + r of a lane's 8 is 16 t + 4 (lane / 16) + r, where the scores are.
//  - A probability goes into the product as the sum of bf16: of three for up to 16 rows, 24 bits as in vitcop_decode_attn (us with
//    two and with three: 8 drafts x 32 heads x 384 keys 9.9, 10.2, 64 windows of 4096 x 28 / 4 heads 85, 85), of two for 32, where
//    the third would cost more (16 trees of 25 drafts 65, 69.5) and 16 bits are 2^-8 of what the output's rounding takes away.
//    Sums, references and outputs are fp32.
//  - The running reference of the softmax moves only when a score exceeds it by 2^8; until then no lane needs another's scores.
//  - Rows past a span's end are past its descriptor and read as zeros; what is masked is so by selection, so that neither
//    stale rows nor drafts that nobody sees reach a result, whatever they hold.
// span_merge_kernel combines the slices; a single slice is finished on the spot.
#include "vitcop_internal.h"
#include "device_utils.h"
#include "span_device.h"

#include <algorithm>
#include <type_traits>

namespace vitcop {

constexpr float SP_SLACK = 8.f;              // log2

__device__ __forceinline__ float span_quotient(float o, float l) { return l == 0.f ? 0.f : o / l; }
__device__ __forceinline__ float span_lse(float m, float l) {
    return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, int NB, bool TREE>
__global__ __launch_bounds__(64 * SP_WAVES, NB == 2 ? 2 : 3) void span_attn_kernel(const SpanArgs A) {
    constexpr int STEPS = D / 32, BLOCKS = D / 16, ROWS = 16 * NB, PARTS = NB == 1 ? 3 : 2;
    constexpr int VROW = 2 * D + 32;                                 // bytes of a V row in LDS: the pad keeps eight rows apart
    constexpr int LPR = D / 8, RPL = 64 / LPR, VL = SP_KEYS / RPL;   // V: lanes a row, rows a load, loads a tile
    static_assert(SP_KEYS * VROW >= 16 * D * 4, "the outputs take V's place at the end");
    __shared__ __attribute__((aligned(16))) char vt[SP_WAVES][SP_KEYS * VROW];
    __shared__ float sm[SP_WAVES][ROWS][2];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int hk = blockIdx.x, rb = blockIdx.y / (unsigned)A.slices, slice = blockIdx.y - rb * A.slices;
    int b = blockIdx.z;
    if (A.ragged) b = span_sample(A, b, 256 / (A.Hkv * A.slices * A.row_blocks));
    const int G = A.G, Hq = A.Hkv * G;
    const int n_tok = A.counts ? min(max(A.counts[b], 0), A.T) : A.T;
    const int start = A.starts ? min(max(A.starts[b], 0), A.start) : A.start;
    const int r0 = rb * ROWS, n_rows = min(ROWS, n_tok * G - r0);
    if (n_rows <= 0) return;

    // the two spans, and what this block of rows looks at
    const int t_first = r0 / G, t_last = (r0 + n_rows - 1) / G;
    int lo = 0, len_a, len_b;                                        // lo: the cache row that span b begins with
    uint64_t seen = 0;                                               // TREE: drafts that a token of the sample sees
    if constexpr (TREE) {
        len_a = start;
        len_b = n_tok;
        uint64_t w = lane < n_tok ? A.tree[b * A.tree_batch + lane] : 0;
        uint32_t w0 = (uint32_t)w, w1 = (uint32_t)(w >> 32);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            w0 |= __shfl_xor(w0, o, 64);
            w1 |= __shfl_xor(w1, o, 64);
        }
        seen = (uint64_t)w1 << 32 | w0;
    } else {
        const int p = start + t_first;
        lo = A.window ? max(0, p - A.window + 1) : 0;
        len_a = min(A.sinks, lo);
        len_b = start + t_last + 1 - lo;
    }
    const int tiles_a = (len_a + SP_KEYS - 1) / SP_KEYS, tiles = tiles_a + (len_b + SP_KEYS - 1) / SP_KEYS;
    const int per = tiles / A.slices, more = tiles - per * A.slices;
    const int tile_begin = slice * per + min(slice, more), tile_end = tile_begin + per + (slice < more ? 1 : 0);

    const int64_t kv_row = (int64_t)A.Hkv * D;
    const uint16_t* const ka = A.k + b * A.kv_batch + hk * D;
    const uint16_t* const va = A.v + b * A.kv_batch + hk * D;
    const uint16_t* const kb = TREE ? A.k2 + b * A.k2_batch + hk * D : ka + lo * kv_row;
    const uint16_t* const vb = TREE ? A.v2 + b * A.v2_batch + hk * D : va + lo * kv_row;

    u32x4 kr[2][STEPS], vr[VL];
    // a descriptor for each tile: 32 rows from a 64-bit address on, however long the cache is
    auto load = [&](int tile) __attribute__((always_inline)) {
        const bool in_b = tile >= tiles_a;
        const int row0 = (in_b ? tile - tiles_a : tile) * SP_KEYS, left = min(SP_KEYS, (in_b ? len_b : len_a) - row0);
        const int64_t k_row = TREE && in_b ? A.k2_row : kv_row, v_row = TREE && in_b ? A.v2_row : kv_row;
        const unsigned k_bytes = (unsigned)k_row * 2, v_bytes = (unsigned)v_row * 2;
        const auto k_desc = __builtin_amdgcn_make_buffer_rsrc((void*)((in_b ? kb : ka) + row0 * k_row), 0,
                                                              (left - 1) * k_bytes + 2 * D, 0x00020000);
        const auto v_desc = __builtin_amdgcn_make_buffer_rsrc((void*)((in_b ? vb : va) + row0 * v_row), 0,
                                                              (left - 1) * v_bytes + 2 * D, 0x00020000);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < STEPS; ++c)
                kr[t][c] = __builtin_amdgcn_raw_buffer_load_b128(k_desc, (16 * t + l16) * k_bytes + 16 * g4 + 64 * c, 0, 0);
#pragma unroll
        for (int i = 0; i < VL; ++i)
            vr[i] = __builtin_amdgcn_raw_buffer_load_b128(v_desc, (RPL * i + lane / LPR) * v_bytes + 16 * (lane % LPR), 0, 0);
    };
    const int first = tile_begin + wv;
    if (first < tile_end) load(first);

    bf16x8 qf[NB][STEPS];                                            // Q^T: 8 channels of a row a step (rows past the end: the last)
    int at[NB];                                                      // the cache row of each column's token
    uint64_t bits[NB];                                               // TREE: the drafts that it sees
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int r = r0 + min(16 * n + l16, n_rows - 1), t = r / G, g = r - t * G;
        const uint16_t* qp = A.q + b * A.q_batch + t * A.q_row + (int64_t)(hk * G + g) * D + 8 * g4;
#pragma unroll
        for (int c = 0; c < STEPS; ++c) qf[n][c] = *reinterpret_cast<const bf16x8*>(qp + 32 * c);
        at[n] = start + t;
        bits[n] = 0;
        if constexpr (TREE) bits[n] = A.tree[b * A.tree_batch + t];
    }
    f32x4 o[NB][BLOCKS];
    float m[NB], l[NB];                                              // of the column (m for all its keys, l over this lane's)
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        m[n] = -INFINITY;
        l[n] = 0.f;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((ext_vector_type(8))) short s16x8;
    char* const mine = vt[wv];
    const unsigned tr = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)mine +
                        (4 * g4 + ((lane >> 2) & 3)) * VROW + (lane & 3) * 8;
    for (int tile = first; tile < tile_end; tile += SP_WAVES) {
        const bool in_b = tile >= tiles_a;
        const int row0 = (in_b ? tile - tiles_a : tile) * SP_KEYS, left = min(SP_KEYS, (in_b ? len_b : len_a) - row0);
        f32x4 s[NB][2];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < STEPS; ++c)
                    s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[t][c]), qf[n][c], s[n][t],
                                                                      0, 0, 0);
            }
        if constexpr (TREE) {
            if (in_b)                                                // drafts that no token sees: zeros, whatever they hold
#pragma unroll
                for (int i = 0; i < VL; ++i)
                    if (!(seen >> (row0 + RPL * i + lane / LPR) & 1)) vr[i] = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int i = 0; i < VL; ++i)
            *reinterpret_cast<u32x4*>(mine + (RPL * i + lane / LPR) * VROW + lane % LPR * 16) = vr[i];
        if (tile + SP_WAVES < tile_end) load(tile + SP_WAVES);       // (uniform) in flight from here on
        // masks: none where every row of the block sees all 32 keys
        const int key0 = lo + row0;                                  // (span b of a window)
        const bool whole = left == SP_KEYS && (!in_b || (!TREE && key0 + SP_KEYS - 1 <= start + t_first &&
                                                         (A.window == 0 || key0 > start + t_last - A.window)));
        if (!whole) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int kk = 16 * (e >> 2) + 4 * g4 + (e & 3);
                    bool sees = kk < left;
                    if (in_b) {
                        if constexpr (TREE) {
                            sees = sees && (bits[n] >> (row0 + kk) & 1);
                        } else {
                            const int j = key0 + kk;
                            sees = sees && j <= at[n] && (A.window == 0 || j > at[n] - A.window || j < A.sinks);
                        }
                    }
                    s[n][e >> 2][e & 3] = sees ? s[n][e >> 2][e & 3] : -INFINITY;
                }
        }
        float top[NB];
        bool over = false;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            top[n] = fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])),
                           fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3]))) * A.scale_log2e;
            over |= top[n] > m[n] + SP_SLACK;
        }
        if (__builtin_amdgcn_ballot_w64(over) != 0) {
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                top[n] = fmaxf(top[n], __shfl_xor(top[n], 16, 64));
                top[n] = fmaxf(top[n], __shfl_xor(top[n], 32, 64));
                const float m_new = fmaxf(m[n], top[n]);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - m_new);
                m[n] = m_new;
                l[n] *= alpha;
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[n][i][r] *= alpha;
            }
        }
        u32x4 part[NB][PARTS];                                       // of each pair of probabilities, the rest of the rest last
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const float base = m[n] == -INFINITY ? 0.f : m[n];       // (nothing but -inf so far: 0, not NaN)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 1][2 * (e & 1)], A.scale_log2e, -base));
                const float c = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 1][2 * (e & 1) + 1], A.scale_log2e, -base));
                l[n] += a;
                l[n] += c;
                float ra = a, rc = c;
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {
                    const uint32_t w = pack_bf16(ra, rc);
                    part[n][k][e] = w;
                    ra -= bf16_lo(w);
                    rc -= bf16_hi(w);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();                             // (one wavefront's LDS accesses stay in order)
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(uintptr_t)(tr + i * 32));
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(uintptr_t)(tr + i * 32 + 16 * VROW));
            const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int k = 0; k < PARTS; ++k)
#pragma unroll
                for (int n = 0; n < NB; ++n)
                    o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, part[n][k]), o[n][i], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();                             // the next tile's rows replace these
    }

    // the wavefronts' states meet, 16 rows at a time, by threads (row, four channels)
    float (&so)[SP_WAVES][16][D] = *reinterpret_cast<float (*)[SP_WAVES][16][D]>(&vt[0][0]);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
        __syncthreads();                                             // all are done with V, or with the rows before
        if (g4 == 0) {
            sm[wv][16 * n + l16][0] = m[n];
            sm[wv][16 * n + l16][1] = l[n];
        }
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) *reinterpret_cast<f32x4*>(&so[wv][l16][16 * i + 4 * g4]) = o[n][i];
        __syncthreads();
        for (int idx = threadIdx.x; idx < 16 * (D / 4); idx += 64 * SP_WAVES) {
            const int row = idx / (D / 4), ch = idx % (D / 4) * 4, local = 16 * n + row;
            if (local >= n_rows) continue;
            float mn = -INFINITY;
#pragma unroll
            for (int w = 0; w < SP_WAVES; ++w) mn = fmaxf(mn, sm[w][local][0]);
            float lt = 0.f;
            f32x4 ot = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < SP_WAVES; ++w) {
                const float a = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(sm[w][local][0] - mn);
                lt += sm[w][local][1] * a;
                ot += *reinterpret_cast<const f32x4*>(&so[w][row][ch]) * a;
            }
            const int r = r0 + local;
            if (A.slices > 1) {
                const int64_t slot = (((int64_t)b * A.Hkv + hk) * A.T * G + r) * A.slices + slice;
                *reinterpret_cast<f32x4*>(A.part_o + slot * D + ch) = ot;
                if (ch == 0) {
                    A.part_ml[slot * 2] = mn;
                    A.part_ml[slot * 2 + 1] = lt;
                }
                continue;
            }
            const int t = r / G, h = hk * G + r - t * G;
            *reinterpret_cast<uint2*>(A.out + (((int64_t)b * A.T + t) * Hq + h) * D + ch) =
                make_uint2(pack_bf16(span_quotient(ot.x, lt), span_quotient(ot.y, lt)),
                           pack_bf16(span_quotient(ot.z, lt), span_quotient(ot.w, lt)));
            if (A.lse && ch == 0) A.lse[((int64_t)b * Hq + h) * A.T + t] = span_lse(mn, lt);
        }
    }
}

// The slices of a query row combined, by threads (slices, four channels) whose loads go out before the weights are known.
// GROUPS = 1: up to SM_FEW slices, all of a thread's, a workgroup taking as many rows as it has room for.  GROUPS = 8 (d = 64: 16):
// a thread takes every GROUPSth slice of one row, and the groups' sums meet in LDS in a fixed order.  (14336 rows of two slices
// 5.5 us, 8876 of seven 7.5; with a workgroup to each row 14336 of four took 17.4.)
constexpr int SM_THREADS = 256, SM_FEW = 8;
template <int D, int GROUPS>
__global__ __launch_bounds__(SM_THREADS) void span_merge_kernel(const SpanArgs A) {
    constexpr int QUADS = D / 4, ROWS = SM_THREADS / (QUADS * GROUPS), AHEAD = GROUPS == 1 ? SM_FEW : 4;
    __shared__ f32x4 sums[GROUPS][QUADS];
    __shared__ float total[GROUPS];
    const int rows = A.T * A.G, G = A.G, Hq = A.Hkv * G;
    const int c = threadIdx.x % QUADS, grp = GROUPS == 1 ? 0 : threadIdx.x / QUADS;
    const unsigned id = ROWS == 1 ? blockIdx.x : blockIdx.x * ROWS + threadIdx.x / QUADS;
    const unsigned pair = id / (unsigned)rows, r = id - pair * (unsigned)rows;
    const int b = pair / (unsigned)A.Hkv, hk = pair - b * A.Hkv;
    const int t = (int)r / G, h = hk * G + (int)r - t * G;
    if (b >= A.B || t >= (A.counts ? A.counts[b] : A.T)) return;         // (one row: for all of its threads)
    const float* po = A.part_o + (int64_t)id * A.slices * D + 4 * c;
    const float2* ml = reinterpret_cast<const float2*>(A.part_ml) + (int64_t)id * A.slices;
    f32x4 x[AHEAD];
    float2 w[AHEAD];
    auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int s = s0 + i * GROUPS;
            w[i] = float2{-INFINITY, 0.f};
            x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (s < A.slices) {
                x[i] = *reinterpret_cast<const f32x4*>(po + (int64_t)s * D);
                w[i] = ml[s];
            }
        }
    };
    request(grp);
    float mn = -INFINITY;
    if constexpr (GROUPS == 1) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) mn = fmaxf(mn, w[i].x);
    } else {
        for (int s = threadIdx.x & 63; s < A.slices; s += 64) mn = fmaxf(mn, ml[s].x);
        mn = wave_max(mn);
    }
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int s0 = grp; s0 < A.slices; s0 += AHEAD * GROUPS) {
        if (s0 != grp) request(s0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float a = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(w[i].x - mn);
            v += x[i] * a;
            l += w[i].y * a;
        }
    }
    if constexpr (GROUPS > 1) {
        sums[grp][c] = v;
        if (c == 0) total[grp] = l;
        __syncthreads();
        if (grp != 0) return;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) {
            v += sums[i][c];
            l += total[i];
        }
    }
    *reinterpret_cast<uint2*>(A.out + (((int64_t)b * A.T + t) * Hq + h) * D + 4 * c) =
        make_uint2(pack_bf16(span_quotient(v.x, l), span_quotient(v.y, l)), pack_bf16(span_quotient(v.z, l), span_quotient(v.w, l)));
    if (A.lse && c == 0) A.lse[((int64_t)b * Hq + h) * A.T + t] = span_lse(mn, l);
}

template <int D>
static int launch_span_merge(const SpanArgs& A, hipStream_t s) {
    const int64_t rows = (int64_t)A.B * A.T * A.G * A.Hkv;
    constexpr int GROUPS = SM_THREADS / (D / 4);
    if (A.slices <= SM_FEW)
        hipLaunchKernelGGL((span_merge_kernel<D, 1>), dim3((unsigned)((rows + GROUPS - 1) / GROUPS)), dim3(SM_THREADS), 0, s, A);
    else
        hipLaunchKernelGGL((span_merge_kernel<D, GROUPS>), dim3((unsigned)rows), dim3(SM_THREADS), 0, s, A);
    return launch_status("span_merge");
}

SpanChoice span_choice(int B, int T, int start, int Hq, int Hkv, int d, int window, int sinks, bool tree, bool own) {
    // the wide kernel addresses a span with 32 bits of bytes
    const int64_t all = (int64_t)start + T, keys = window == 0 ? all : std::min<int64_t>(all, (int64_t)window + T);
    const bool fits = (std::max<int64_t>(keys, sinks) + 256) * Hkv * d * 2 < ((int64_t)1 << 32);
    SpanSizes z{B, Hkv, T, Hq / Hkv, start, window, sinks, d, tree, own};
    SpanChoice c{span_plan(z, fits), z.ragged(), 0};
    size_t most = c.plan.slices;                             // (the same sizes with the other kind of lengths)
    z.own = !own;
    if (z.ragged() != c.ragged) most = std::max<size_t>(most, span_plan(z, fits).slices);
    if (most > 1) c.ws_bytes = up256((size_t)B * T * Hq * most * d * 4) + up256((size_t)B * T * Hq * most * 2 * 4);
    return c;
}

template <int D>
static int launch_span_d(SpanArgs A, const SpanPlan& p, int Hq, void* ws, hipStream_t s) {
    A.row_blocks = p.row_blocks;
    A.slices = p.slices;
    A.part_o = static_cast<float*>(ws);
    A.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + up256((size_t)A.B * A.T * Hq * p.slices * D * 4));
    int rc;
    if (p.wide) {
        rc = launch_attn_spans(A, D, p.blocks, s);
    } else {
        if ((int64_t)p.slices * p.row_blocks > 65535) return fail(VITCOP_EUNSUPPORTED, "attention over a cache: too many query rows");
        auto kernel = [&](auto tree) {
            constexpr bool TREE = decltype(tree)::value;
            return p.blocks == 1 ? span_attn_kernel<D, 1, TREE> : span_attn_kernel<D, 2, TREE>;
        };
        hipLaunchKernelGGL(A.tree ? kernel(std::true_type{}) : kernel(std::false_type{}),
                           dim3(A.Hkv, p.slices * p.row_blocks, A.B), dim3(64 * SP_WAVES), 0, s, A);
        rc = launch_status("span_attn");
    }
    return rc || p.slices == 1 ? rc : launch_span_merge<D>(A, s);
}

int launch_span_attn(const SpanCall& c, const vitcop_cache_t& C, int Hq, const SpanChoice& p, void* ws, hipStream_t s) {
    SpanArgs A{};
    A.q = c.q;
    A.q_row = c.q_row;
    A.q_batch = c.q_batch;
    A.k = C.k;
    A.v = C.v;
    A.kv_batch = (int64_t)C.capacity * C.Hkv * C.d;
    A.k2 = c.k;
    A.v2 = c.v;
    A.k2_row = c.k_row;
    A.k2_batch = c.k_batch;
    A.v2_row = c.v_row;
    A.v2_batch = c.v_batch;
    A.tree = c.tree;
    A.tree_batch = c.tree_batch;
    A.starts = c.start_samples;
    A.counts = c.n_samples;
    A.B = C.B;
    A.T = c.T;
    A.G = Hq / C.Hkv;
    A.Hkv = C.Hkv;
    A.start = c.start;
    A.window = c.window;
    A.sinks = c.sinks;
    A.scale_log2e = c.scale * 1.4426950408889634f;
    A.out = c.out;
    A.lse = c.lse;
    A.ragged = p.ragged;
    return C.d == 64 ? launch_span_d<64>(A, p.plan, Hq, ws, s) : launch_span_d<128>(A, p.plan, Hq, ws, s);
}

}  // namespace vitcop
