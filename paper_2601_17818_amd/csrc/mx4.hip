// Rows of bf16 to 4 bits and back (format: mx4_device.h), as matrices (weights) and as the rows of a KV cache.  Single
// passes: 2 bytes a value on one side, 17/32 on the other, and a few instructions for eight values, so HBM-bound.
// Eight values to a thread, 16 bytes of bf16 and one dword of codes: a group is a quad of lanes.  The bf16 side, read or
// written once, goes past the caches: with rows from HBM a cache of 4 x 2944 x 32 x 128 (244 MB with its bf16 rows, K and V
// inside QKV rows) to 4 bits 42.8 us, 5.7 TB/s, through the caches 46.6; back 34.7, through them 45; a matrix of 11776 x 4096
// 20.8 and 17.9 us.
#include "vitcop_internal.h"
#include "mx4_device.h"

#include <algorithm>

namespace vitcop {

constexpr int MX_THREADS = 256, MX_UNROLL = 2;

// Units of eight values, `per_row` to a row of the bf16 side (rows `stride` elements apart); the 4-bit side is dense.
template <bool QUANTIZE>
__global__ __launch_bounds__(MX_THREADS) void mx4_rows_kernel(const uint16_t* __restrict__ x, uint16_t* __restrict__ y,
                                                              int64_t stride, uint32_t* codes, uint8_t* scales,
                                                              uint32_t units, uint32_t per_row) {
    const uint32_t first = blockIdx.x * (MX_THREADS * MX_UNROLL) + threadIdx.x;
    auto at = [&](uint32_t u) { return (int64_t)(u / per_row) * stride + (int64_t)(u % per_row) * 8; };
    if constexpr (QUANTIZE) {
        uint4 v[MX_UNROLL];
#pragma unroll
        for (int i = 0; i < MX_UNROLL; ++i) {
            const uint32_t u = first + i * MX_THREADS;
            v[i] = u < units ? ld_nt16(x + at(u)) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < MX_UNROLL; ++i) {
            const uint32_t u = first + i * MX_THREADS;
            uint32_t e;
            const uint32_t c = mx4_codes(v[i], e);           // (units is a multiple of four: whole quads)
            if (u < units) {
                codes[u] = c;
                if ((u & 3) == 0) scales[u >> 2] = (uint8_t)e;
            }
        }
    } else {
        uint32_t c[MX_UNROLL], e[MX_UNROLL];
#pragma unroll
        for (int i = 0; i < MX_UNROLL; ++i) {
            const uint32_t u = min(first + i * MX_THREADS, units - 1);
            c[i] = codes[u];
            e[i] = scales[u >> 2];
        }
#pragma unroll
        for (int i = 0; i < MX_UNROLL; ++i) {
            const uint32_t u = first + i * MX_THREADS;
            if (u < units) __builtin_nontemporal_store(mx4_values(c[i], mx4_scale(e[i])), reinterpret_cast<u32x4*>(y + at(u)));
        }
    }
}

static dim3 rows_grid(uint32_t units) {
    return dim3((unsigned)(((uint64_t)units + MX_THREADS * MX_UNROLL - 1) / (MX_THREADS * MX_UNROLL)));
}

int launch_mx4_quantize(const uint16_t* x, int64_t x_stride, int M, int K, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    const uint32_t units = (uint32_t)((int64_t)M * K / 8);
    hipLaunchKernelGGL((mx4_rows_kernel<true>), rows_grid(units), dim3(MX_THREADS), 0, s, x, nullptr, x_stride,
                       reinterpret_cast<uint32_t*>(codes), scales, units, (uint32_t)(K / 8));
    return launch_status("mx4_quantize");
}

int launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int M, int K, uint16_t* y, int64_t y_stride,
                          hipStream_t s) {
    const uint32_t units = (uint32_t)((int64_t)M * K / 8);
    hipLaunchKernelGGL((mx4_rows_kernel<false>), rows_grid(units), dim3(MX_THREADS), 0, s, nullptr, y, y_stride,
                       reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(codes)), const_cast<uint8_t*>(scales), units,
                       (uint32_t)(K / 8));
    return launch_status("mx4_dequantize");
}

// Rows of a cache.  The bf16 side is token-major, the cache head-major (an attention wavefront reads one head's rows one
// after the other), so a wavefront takes one head's rows of consecutive tokens: MC_ROWS loads of 16 bytes a lane in flight,
// pieces of a head's row (2 d bytes) on one side, one contiguous run on the other.
constexpr int MC_THREADS = 256, MC_ROWS = 2;

struct Mx4Side {                         // K or V
    const uint16_t* x;                   // rows to write, or
    uint16_t* y;                         // rows to read
    uint8_t* codes;
    uint8_t* scales;
};
struct Mx4Rows {
    Mx4Side side[2];
    int64_t row_stride, batch_stride;    // of x
    const int32_t* start_samples;
    const int32_t* n_samples;
    int T, Hkv, capacity, start, blocks; // blocks: of tokens, per sample and head
    uint32_t waves;
};

template <int D, bool WRITE>
__global__ __launch_bounds__(MC_THREADS) void mx4_cache_kernel(Mx4Rows a) {
    constexpr int LPR = D / 8, RPL = 64 / LPR;               // lanes a row, rows a load
    const int lane = threadIdx.x & 63, c = lane % LPR;
    const uint32_t wave = blockIdx.x * (MC_THREADS / 64) + (threadIdx.x >> 6);
    if (wave >= a.waves) return;
    const Mx4Side side = a.side[blockIdx.y];
    const uint32_t h = wave % a.Hkv, rest = wave / a.Hkv;
    const uint32_t tb = rest % a.blocks, b = rest / a.blocks;
    const int t0 = (int)tb * (RPL * MC_ROWS) + lane / LPR;
    const int64_t start = a.start_samples ? a.start_samples[b] : a.start;
    const int n = a.n_samples ? min(max(a.n_samples[b], 0), a.T) : a.T;
    const int64_t head = ((int64_t)b * a.Hkv + h) * a.capacity;
    auto row_of = [&](int t) { return head + start + t; };
    auto inside = [&](int t) { return start + t >= 0 && start + t < a.capacity; };
    if constexpr (WRITE) {
        const uint16_t* src = side.x + (int64_t)b * a.batch_stride + h * D + 8 * c;
        uint4 v[MC_ROWS];
#pragma unroll
        for (int i = 0; i < MC_ROWS; ++i) {
            const int t = t0 + i * RPL;
            v[i] = t < n ? ld_nt16(src + t * a.row_stride) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < MC_ROWS; ++i) {
            const int t = t0 + i * RPL;
            uint32_t e;
            const uint32_t w = mx4_codes(v[i], e);
            if (t >= n || !inside(t)) continue;
            *reinterpret_cast<uint32_t*>(side.codes + row_of(t) * (D / 2) + 4 * c) = w;
            if ((c & 3) == 0) side.scales[row_of(t) * (D / MX4_GROUP) + c / 4] = (uint8_t)e;
        }
    } else {
        uint32_t w[MC_ROWS], e[MC_ROWS];
#pragma unroll
        for (int i = 0; i < MC_ROWS; ++i) {
            const int t = t0 + i * RPL;
            const bool live = t < a.T && inside(t);
            w[i] = live ? *reinterpret_cast<const uint32_t*>(side.codes + row_of(t) * (D / 2) + 4 * c) : 0u;
            e[i] = live ? side.scales[row_of(t) * (D / MX4_GROUP) + c / 4] : 0u;
        }
#pragma unroll
        for (int i = 0; i < MC_ROWS; ++i) {
            const int t = t0 + i * RPL;
            if (t < a.T)
                __builtin_nontemporal_store(mx4_values(w[i], mx4_scale(e[i])),
                                            reinterpret_cast<u32x4*>(side.y + (((int64_t)b * a.T + t) * a.Hkv + h) * D + 8 * c));
        }
    }
}

// `a` apart from blocks and waves; one or two sides
static int launch_cache(Mx4Rows a, int sides, int B, int d, bool write, hipStream_t s) {
    const int per_wave = 64 / (d / 8) * MC_ROWS;
    a.blocks = (a.T + per_wave - 1) / per_wave;
    a.waves = (uint32_t)((int64_t)B * a.Hkv * a.blocks);
    auto* kernel = d == 64 ? (write ? mx4_cache_kernel<64, true> : mx4_cache_kernel<64, false>)
                           : (write ? mx4_cache_kernel<128, true> : mx4_cache_kernel<128, false>);
    hipLaunchKernelGGL(kernel, dim3((a.waves + 3) / 4, sides), dim3(MC_THREADS), 0, s, a);
    return launch_status(write ? "cache_mx4_write" : "cache_mx4_read");
}

int launch_cache_mx4_write(const vitcop_cache_mx4_t& C, const uint16_t* k, const uint16_t* v, int64_t row_stride,
                           int64_t batch_stride, int T, int start, const int32_t* start_samples,
                           const int32_t* n_samples, hipStream_t s) {
    Mx4Rows a{};
    int sides = 0;
    if (k) a.side[sides++] = Mx4Side{k, nullptr, C.k_codes, C.k_scales};
    if (v) a.side[sides++] = Mx4Side{v, nullptr, C.v_codes, C.v_scales};
    a.row_stride = row_stride;
    a.batch_stride = batch_stride;
    a.start_samples = start_samples;
    a.n_samples = n_samples;
    a.T = T;
    a.Hkv = C.Hkv;
    a.capacity = C.capacity;
    a.start = start;
    return launch_cache(a, sides, C.B, C.d, true, s);
}

int launch_cache_mx4_read(const vitcop_cache_mx4_t& C, uint16_t* k, uint16_t* v, int T, int start,
                          const int32_t* start_samples, hipStream_t s) {
    Mx4Rows a{};
    int sides = 0;
    if (k) a.side[sides++] = Mx4Side{nullptr, k, C.k_codes, C.k_scales};
    if (v) a.side[sides++] = Mx4Side{nullptr, v, C.v_codes, C.v_scales};
    a.start_samples = start_samples;
    a.T = T;
    a.Hkv = C.Hkv;
    a.capacity = C.capacity;
    a.start = start;
    return launch_cache(a, sides, C.B, C.d, false, s);
}

}  // namespace vitcop
