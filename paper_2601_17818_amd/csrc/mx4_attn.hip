// One decoding step over a KV cache held in 4 bits (format: mx4_device.h): o = softmax(scale K q) V for the new token of
// every sample.  Bound by the cache's bytes, 17/32 of one a value, each read once for every 16 query heads of a KV head.
//
// A workgroup takes one KV head of a sample and one slice of the keys, a wavefront 32 keys at a time: scores S^T = K Q^T
// (16x16x32: a lane holds 4 keys of one head), the softmax with the lane's head as its only query, O^T += V^T P^T.  The
// products are on the matrix cores also where a KV head has a single query head and 15 of 16 columns are idle: on the vector
// pipe a key's 2 d values would cost an FMA each and, before it, half a conversion; here the conversions alone remain.
//  - K goes from the conversion straight into the product: a lane's 16 (8) bytes of a row are 32 (16) neighbouring
//    channels, and the order of the channels in a sum is free as long as q is read in the same one.
//  - V has to be turned (a product's operand holds one channel of several keys): its bf16 rows go through LDS and come back
//    transposed (ds_read_b64_tr_b16).  The key of element 4 t + r of a lane's 8 is 16 t + 4 (lane / 16) + r, which is where
//    the scores are.
//  - The probabilities stay 32-bit: each is the sum of three bf16, its first, second and last eight bits.  Up to five heads have
//    them side by side in the columns of one product (heads in columns 0 to 4, 5 to 9 and 10 to 14, which otherwise would repeat
//    one), up to eight in those of two, more in one product for each; the columns' sums meet at the end.
//    (us, by this rule and with three products: 64 x 1536 keys x 32 heads 74.3, 88.9; 4 x 65536 x 28 / 4 31.3, 35.0; 4 x 60000 x 16
//    heads of 64 56.4, 66.5.)
//  - The running reference of the softmax moves only when a score exceeds it by 2^8, which is rare after the first tiles; until
//    then no lane needs to know another's scores.  Sums, references and outputs are fp32.
// mx4_merge_kernel combines the slices; a single slice is finished on the spot.
#include "vitcop_internal.h"
#include "mx4_device.h"
#include "mx4_plan.h"

#include <algorithm>

namespace vitcop {

constexpr float MA_SLACK = 8.f;              // log2

// The first eight bits of a positive number (those `kept`), the rest, and the first eight of two numbers as a pair of bf16.
__device__ __forceinline__ float ma_first(float x, uint32_t kept = 0xFFFF0000u) {
    return __uint_as_float(__float_as_uint(x) & kept);
}
__device__ __forceinline__ float ma_rest(float x) { return x - ma_first(x); }
__device__ __forceinline__ uint32_t ma_pair(float x, float y) {
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}
// x + the value of the lane COLUMNS to the right in the row of 16
template <int COLUMNS>
__device__ __forceinline__ float ma_plus(float x, float of) {
    return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(of), 0x100 + COLUMNS, 0xF, 0xF, true));      // row_shl
}

// what a head without any key gives: zeros, and minus infinity as the logarithm of its sum
__device__ __forceinline__ float mx4_quotient(float o, float l) { return l == 0.f ? 0.f : o / l; }
__device__ __forceinline__ float mx4_lse(float m, float l) {
    return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// WAVES wavefronts, 32 keys at a time each, share the slice (attn_plan: how many), PRODUCTS: of a tile's probabilities with V.
// Registers for three workgroups of four on a CU, two of eight.
template <int D, int WAVES, int PRODUCTS>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 ? 2 : 3) void mx4_attn_kernel(
    const uint16_t* __restrict__ q, const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_scales,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_scales, float* __restrict__ part_o,
    float* __restrict__ part_ml, int capacity, int N, int Hq, int Hkv, int g0, int G, float scale_log2e, int keys_per_split,
    int n_splits, const int32_t* __restrict__ n_samples, uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int STEPS = D / 32, BLOCKS = D / 16, COLUMNS = ma_columns(PRODUCTS);
    constexpr int ROW = D / 2, GROUPS = D / MX4_GROUP;               // bytes of a row of codes, of exponents
    constexpr int VROW = 2 * D + 32;                                 // bytes of a V row in LDS: the pad keeps eight rows apart
    constexpr int LPR = ROW / 16, RPL = 64 / LPR, VL = MA_KEYS / RPL;         // V: lanes a row, rows a load, loads a tile
    static_assert(MA_KEYS * VROW >= MA_MAX_G * D * 4, "the outputs take V's place at the end");
    __shared__ __attribute__((aligned(16))) char vt[WAVES][MA_KEYS * VROW];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
    const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int h0 = hk * (Hq / Hkv) + g0;                     // first query head of this pass
    const int key_begin = split * keys_per_split, slice_end = min(N, key_begin + keys_per_split);
    const int first = key_begin + wv * MA_KEYS;

    // Rows past the slice's end read as zeros: the descriptors end there.
    const int64_t head_row = ((int64_t)b * Hkv + hk) * capacity;
    const auto kc_desc = __builtin_amdgcn_make_buffer_rsrc((void*)(k_codes + head_row * ROW), 0, slice_end * ROW, 0x00020000);
    const auto ks_desc = __builtin_amdgcn_make_buffer_rsrc((void*)(k_scales + head_row * GROUPS), 0, slice_end * GROUPS, 0x00020000);
    const auto vc_desc = __builtin_amdgcn_make_buffer_rsrc((void*)(v_codes + head_row * ROW), 0, slice_end * ROW, 0x00020000);
    const auto vs_desc = __builtin_amdgcn_make_buffer_rsrc((void*)(v_scales + head_row * GROUPS), 0, slice_end * GROUPS, 0x00020000);
    constexpr int NT = 2;                                    // non-temporal
    typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
    u32x4 kr[2], vr[VL];                                     // (d = 64: two dwords of K)
    uint32_t ke[2], ve[VL];
    auto load = [&](int key0) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const unsigned row = (unsigned)(key0 + 16 * t + l16);
            if constexpr (D == 128) {
                kr[t] = __builtin_amdgcn_raw_buffer_load_b128(kc_desc, row * ROW + 16 * g4, 0, NT);
            } else {
                const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(kc_desc, row * ROW + 8 * g4, 0, NT);
                kr[t] = u32x4{w.x, w.y, 0u, 0u};
            }
            ke[t] = __builtin_amdgcn_raw_buffer_load_b8(ks_desc, row * GROUPS + g4 * GROUPS / 4, 0, NT);
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const unsigned row = (unsigned)(key0 + RPL * i + lane / LPR);
            vr[i] = __builtin_amdgcn_raw_buffer_load_b128(vc_desc, row * ROW + 16 * (lane % LPR), 0, NT);
            ve[i] = __builtin_amdgcn_raw_buffer_load_b8(vs_desc, row * GROUPS + lane % LPR, 0, NT);
        }
    };
    if (first < slice_end) load(first);                      // (before it is known how many rows the sample has)
    const int head = l16 % COLUMNS, part0 = l16 / COLUMNS;   // of this lane's column; the part of a probability it takes first
    const uint32_t past0 = part0 > 0 ? 0xFFFF0000u : 0u, past1 = part0 > 1 ? 0xFFFF0000u : 0u;
    bf16x8 qf[STEPS];                                        // Q^T of the head (heads past G: head G - 1), channels as K's
#pragma unroll
    for (int c = 0; c < STEPS; ++c)
        qf[c] = *reinterpret_cast<const bf16x8*>(q + ((int64_t)b * Hq + h0 + min(head, G - 1)) * D + D / 4 * g4 + 8 * c);
    const int key_end = n_samples ? min(slice_end, max(n_samples[b], 0)) : slice_end;
    f32x4 o[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;                            // of the head (m for all its keys, l over this lane's)
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((ext_vector_type(8))) short s16x8;
    char* const mine = vt[wv];
    const unsigned tr = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)mine +
                        (4 * g4 + ((lane >> 2) & 3)) * VROW + (lane & 3) * 8;
    for (int key0 = first; key0 < key_end; key0 += WAVES * MA_KEYS) {
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float e = mx4_scale(ke[t]);
#pragma unroll
            for (int c = 0; c < STEPS; ++c)
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, mx4_values(kr[t][c], e)), qf[c], s[t],
                                                               0, 0, 0);
        }
        if (key0 + MA_KEYS > key_end)                        // rows past the sample's: zeros, whatever they hold
#pragma unroll
            for (int i = 0; i < VL; ++i)
                if (key0 + RPL * i + lane / LPR >= key_end) {
                    vr[i] = u32x4{0u, 0u, 0u, 0u};
                    ve[i] = 0u;
                }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const float e = mx4_scale(ve[i]);
            u32x4* const row = reinterpret_cast<u32x4*>(mine + (RPL * i + lane / LPR) * VROW + lane % LPR * 64);
#pragma unroll
            for (int c = 0; c < 4; ++c) row[c] = mx4_values(vr[i][c], e);
        }
        if (key0 + WAVES * MA_KEYS < key_end) load(key0 + WAVES * MA_KEYS);        // (uniform) in flight from here on
        float p[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int key = key0 + 16 * (e >> 2) + 4 * g4 + (e & 3);
            p[e] = key < key_end ? s[e >> 2][e & 3] * scale_log2e : -INFINITY;
            top = fmaxf(top, p[e]);
        }
        if (__builtin_amdgcn_ballot_w64(top > m + MA_SLACK) != 0) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m, top);
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= alpha;
        }
        const float base = m == -INFINITY ? 0.f : m;         // (nothing but -inf so far: 0, not NaN)
        u32x4 part[PRODUCTS];                                // of each pair of probabilities
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = __builtin_amdgcn_exp2f(p[2 * e] - base), c = __builtin_amdgcn_exp2f(p[2 * e + 1] - base);
            l += a;
            l += c;
            const float a1 = ma_rest(a), c1 = ma_rest(c);
            if constexpr (PRODUCTS == 1) {
                const float ar = a - ma_first(a, past0), cr = c - ma_first(c, past0);
                part[0][e] = ma_pair(ar - ma_first(ar, past1), cr - ma_first(cr, past1));
            } else {
                part[0][e] = PRODUCTS == 2 && part0 ? ma_pair(a1, c1) : ma_pair(a, c);
                if constexpr (PRODUCTS == 3) part[1][e] = ma_pair(a1, c1);
                part[PRODUCTS - 1][e] = PRODUCTS == 2 && part0 ? 0u : ma_pair(ma_rest(a1), ma_rest(c1));
            }
        }
        __builtin_amdgcn_wave_barrier();                     // (one wavefront's LDS accesses stay in order)
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(uintptr_t)(tr + i * 32));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(uintptr_t)(tr + i * 32 + 16 * VROW));
            const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int n = 0; n < PRODUCTS; ++n)
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, part[n]), o[i], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();                     // the next tile's rows replace these
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if constexpr (PRODUCTS < 3) {                            // the parts' columns, least first
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                o[i][r] = PRODUCTS == 1 ? ma_plus<5>(o[i][r], ma_plus<5>(o[i][r], o[i][r])) : ma_plus<8>(o[i][r], o[i][r]);
    }
    __shared__ float sm[WAVES][MA_MAX_G][2];
    float (&so)[WAVES][MA_MAX_G][D] = *reinterpret_cast<float (*)[WAVES][MA_MAX_G][D]>(&vt[0][0]);
    __syncthreads();                                         // all are done with V
    if (l16 < G) {
        if (g4 == 0) {
            sm[wv][l16][0] = m;
            sm[wv][l16][1] = l;
        }
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) *reinterpret_cast<f32x4*>(&so[wv][l16][16 * i + 4 * g4]) = o[i];
    }
    __syncthreads();
    // the wavefronts' states combined by threads (head, four channels): this slice's partial, or with `out` the output
    for (int idx = threadIdx.x; idx < G * (D / 4); idx += 64 * WAVES) {
        const int g = idx / (D / 4), ch = idx % (D / 4) * 4;
        float mn = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mn = fmaxf(mn, sm[w][g][0]);
        float lt = 0.f;
        f32x4 ot = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float a = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(sm[w][g][0] - mn);
            lt += sm[w][g][1] * a;
            ot += *reinterpret_cast<const f32x4*>(&so[w][g][ch]) * a;
        }
        const int64_t bh = (int64_t)b * Hq + h0 + g;
        if (out != nullptr) {
            *reinterpret_cast<uint2*>(out + bh * D + ch) =
                make_uint2(pack_bf16(mx4_quotient(ot.x, lt), mx4_quotient(ot.y, lt)),
                           pack_bf16(mx4_quotient(ot.z, lt), mx4_quotient(ot.w, lt)));
            if (lse && ch == 0) lse[bh] = mx4_lse(mn, lt);
            continue;
        }
        const int64_t slot = bh * n_splits + split;
        *reinterpret_cast<f32x4*>(part_o + slot * D + ch) = ot;
        if (ch == 0) {
            part_ml[slot * 2] = mn;
            part_ml[slot * 2 + 1] = lt;
        }
    }
}

// The slices of a head combined: a thread takes four channels of every MM_GROUPSth slice, whose loads go out before the weights
// are known; the groups' sums meet in LDS in a fixed order.
constexpr int MM_THREADS = 256;
template <int D>
__global__ __launch_bounds__(MM_THREADS) void mx4_merge_kernel(const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                               int n_splits, uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int QUADS = D / 4, MM_GROUPS = MM_THREADS / QUADS, AHEAD = 4;
    __shared__ f32x4 sums[MM_GROUPS][QUADS];
    __shared__ float total[MM_GROUPS];
    const int64_t bh = blockIdx.x;
    const int c = threadIdx.x % QUADS, grp = threadIdx.x / QUADS;
    const float* po = part_o + bh * n_splits * D + 4 * c;
    const float2* ml = reinterpret_cast<const float2*>(part_ml) + bh * n_splits;
    f32x4 x[AHEAD];
    float2 w[AHEAD];
    auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) {
            const int s = s0 + t * MM_GROUPS;
            if (s < n_splits) {
                x[t] = *reinterpret_cast<const f32x4*>(po + (int64_t)s * D);
                w[t] = ml[s];
            }
        }
    };
    request(grp);
    float mn = -INFINITY;
    for (int s = threadIdx.x & 63; s < n_splits; s += 64) mn = fmaxf(mn, ml[s].x);
    mn = wave_max(mn);
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int s0 = grp; s0 < n_splits; s0 += AHEAD * MM_GROUPS) {
        if (s0 != grp) request(s0);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
            if (s0 + t * MM_GROUPS < n_splits) {
                const float a = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(w[t].x - mn);
                v += x[t] * a;
                l += w[t].y * a;
            }
    }
    sums[grp][c] = v;
    if (c == 0) total[grp] = l;
    __syncthreads();
    if (grp != 0) return;
#pragma unroll
    for (int i = 1; i < MM_GROUPS; ++i) {
        v += sums[i][c];
        l += total[i];
    }
    *reinterpret_cast<uint2*>(out + bh * D + 4 * c) = make_uint2(pack_bf16(mx4_quotient(v.x, l), mx4_quotient(v.y, l)),
                                                                 pack_bf16(mx4_quotient(v.z, l), mx4_quotient(v.w, l)));
    if (lse && c == 0) lse[bh] = mx4_lse(mn, l);
}

size_t decode_mx4_workspace_bytes(int B, int N, int Hq, int Hkv, int d) {
    const size_t s = attn_plan(B, N, Hkv, d).splits;
    return s == 1 ? 0 : up256((size_t)B * Hq * s * d * 4) + up256((size_t)B * Hq * s * 2 * 4);
}

template <int D, int PRODUCTS>
static auto* attn_kernel(int waves) {
    return waves == 8 ? mx4_attn_kernel<D, 8, PRODUCTS>
                      : (waves == 4 ? mx4_attn_kernel<D, 4, PRODUCTS> : mx4_attn_kernel<D, 2, PRODUCTS>);
}

template <int D>
static int launch_attn_d(const uint16_t* q, const vitcop_cache_mx4_t& C, uint16_t* out, float* lse, int N,
                         const int32_t* n_samples, int Hq, float scale, void* ws, hipStream_t s) {
    const int B = C.B, group = Hq / C.Hkv;
    const AttnPlan p = attn_plan(B, N, C.Hkv, D);
    float* po = static_cast<float*>(ws);
    float* pml = reinterpret_cast<float*>(static_cast<char*>(ws) + up256((size_t)B * Hq * p.splits * D * 4));
    for (int g0 = 0; g0 < group; g0 += MA_MAX_G) {
        const int G = std::min(MA_MAX_G, group - g0);
        const int products = attn_products(G);
        auto* kernel = products == 1 ? attn_kernel<D, 1>(p.waves)
                                     : (products == 2 ? attn_kernel<D, 2>(p.waves) : attn_kernel<D, 3>(p.waves));
        hipLaunchKernelGGL(kernel, dim3(p.splits, C.Hkv, B), dim3(64 * p.waves), 0, s, q, C.k_codes, C.k_scales, C.v_codes,
                           C.v_scales, po, pml, C.capacity, N, Hq, C.Hkv, g0, G,
                           scale * 1.4426950408889634f, p.keys_per_split, p.splits, n_samples, p.splits == 1 ? out : nullptr, lse);
        const int rc = launch_status("mx4_attn");
        if (rc) return rc;
    }
    if (p.splits == 1) return VITCOP_OK;
    hipLaunchKernelGGL((mx4_merge_kernel<D>), dim3((unsigned)(B * Hq)), dim3(MM_THREADS), 0, s, po, pml, p.splits, out, lse);
    return launch_status("mx4_merge");
}

int launch_decode_attn_mx4(const uint16_t* q, const vitcop_cache_mx4_t& C, uint16_t* out, float* lse, int N,
                           const int32_t* n_samples, int Hq, float scale, void* ws, hipStream_t s) {
    return C.d == 64 ? launch_attn_d<64>(q, C, out, lse, N, n_samples, Hq, scale, ws, s)
                     : launch_attn_d<128>(q, C, out, lse, N, n_samples, Hq, scale, ws, s);
}

}  // namespace vitcop
