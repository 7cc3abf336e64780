// Rotary embedding with a position for each of several axes, on the way to a buffer of queries and the rows of a cache; and
// rows written to the caches of all layers.  Both move each byte once: HBM-bound, and a launch's latency where tokens are few.
#include "vitcop_internal.h"
#include "device_utils.h"

#include <algorithm>
#include <cmath>

namespace vitcop {

// theta^(-2i/d) / (2 pi) as a fraction of 2^64: position * fraction modulo 2^64 is the angle's part of a revolution, which a
// 32-bit product of a far position and a speed has lost (position 10^5, the fastest pair: 2^-8 of a radian), and costs two
// integer products instead of arithmetic in 64-bit floating point.
struct RopeAxesArgs {
    vitcop_rope_axes_t R;
    int slots;                          // threads that share a pair group's heads
    uint16_t axes[16];                  // two bits for each of a group's eight pairs
    uint64_t speed[128];
};

constexpr int RA_THREADS = 256;

// A thread turns eight pairs (16 bytes of a head's lower half and 16 of its upper one) of up to HEADS heads of a token: its
// sines and cosines serve them all, and their loads go out together.  The heads of v pass through.
template <int HEADS>
__global__ __launch_bounds__(RA_THREADS) void rope_axes_kernel(const RopeAxesArgs A) {
    const vitcop_rope_axes_t& R = A.R;
    const unsigned groups = (unsigned)R.d / 16, per_token = groups * A.slots;
    const unsigned id = blockIdx.x * RA_THREADS + threadIdx.x;
    const unsigned token = id / per_token, rest = id - token * per_token;
    if (token >= (unsigned)(R.B * R.T)) return;
    const unsigned b = token / (unsigned)R.T, slot = rest / groups, group = rest - slot * groups;
    const int t = (int)(token - b * (unsigned)R.T);
    const int n_q = R.q ? R.Hq : 0, n_k = R.k ? R.Hkv : 0, n_v = R.v ? R.Hkv : 0;
    const int half = R.d / 2, c0 = 8 * (int)group;
    const int64_t row = (int64_t)(R.start_samples ? R.start_samples[b] : R.start) + t;
    const bool live = t < (R.n_samples ? R.n_samples[b] : R.T);
    if (!live) return;
    const bool k_in_place = R.k_out == R.k, fits = k_in_place || (row >= 0 && row < R.capacity);
    const uint16_t* src[HEADS];
    uint16_t* dst[HEADS];
    uint4 lo[HEADS], hi[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        int h = (int)slot + i * A.slots;
        src[i] = nullptr;
        if (h < n_q) {
            src[i] = R.q + b * R.q_batch_stride + t * R.q_row_stride + (int64_t)h * R.d;
            dst[i] = R.q_out == R.q ? const_cast<uint16_t*>(src[i]) : R.q_out + ((int64_t)token * R.Hq + h) * R.d;
        } else if (fits && (h -= n_q) < n_k) {
            src[i] = R.k + b * R.k_batch_stride + t * R.k_row_stride + (int64_t)h * R.d;
            dst[i] = k_in_place ? const_cast<uint16_t*>(src[i])
                                : R.k_out + (((int64_t)b * R.capacity + row) * R.Hkv + h) * R.d;
        } else if (fits && (h -= n_k) < n_v) {
            src[i] = R.v + b * R.v_batch_stride + t * R.v_row_stride + (int64_t)h * R.d;
            dst[i] = R.v_out + (((int64_t)b * R.capacity + row) * R.Hkv + h) * R.d;
        }
        if (src[i]) {
            lo[i] = *reinterpret_cast<const uint4*>(src[i] + c0);
            hi[i] = *reinterpret_cast<const uint4*>(src[i] + half + c0);
        }
    }
    int pos[VITCOP_MAX_AXES];
#pragma unroll
    for (int a = 0; a < VITCOP_MAX_AXES; ++a)
        pos[a] = a < R.n_axes ? R.positions[((int64_t)a * R.B + b) * R.T + t] : 0;
    float sn[8], cs[8];
    const unsigned axes = A.axes[group];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned a = (axes >> (2 * i)) & 3;
        const int p = a < 2 ? (a == 0 ? pos[0] : pos[1]) : (a == 2 ? pos[2] : pos[3]);
        const uint64_t turn = (uint64_t)(int64_t)p * A.speed[c0 + i];
        sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sn[i], &cs[i]);        // (in half revolutions, [-1, 1])
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        if (!src[i]) continue;
        if ((int)slot + i * A.slots < n_q + n_k) {
            uint32_t* const l = reinterpret_cast<uint32_t*>(&lo[i]);
            uint32_t* const h = reinterpret_cast<uint32_t*>(&hi[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x0 = bf16_lo(l[j]), x1 = bf16_hi(l[j]), y0 = bf16_lo(h[j]), y1 = bf16_hi(h[j]);
                l[j] = pack_bf16(x0 * cs[2 * j] - y0 * sn[2 * j], x1 * cs[2 * j + 1] - y1 * sn[2 * j + 1]);
                h[j] = pack_bf16(y0 * cs[2 * j] + x0 * sn[2 * j], y1 * cs[2 * j + 1] + x1 * sn[2 * j + 1]);
            }
        }
        *reinterpret_cast<uint4*>(dst[i] + c0) = lo[i];
        *reinterpret_cast<uint4*>(dst[i] + half + c0) = hi[i];
    }
}

int launch_rope_axes(const vitcop_rope_axes_t& R, hipStream_t s) {
    RopeAxesArgs A{};
    A.R = R;
    const int pairs = R.d / 2, heads = (R.q ? R.Hq : 0) + (R.k ? R.Hkv : 0) + (R.v ? R.Hkv : 0);
    int left[VITCOP_MAX_AXES] = {}, a = 0;
    for (int i = 0; i < R.n_axes; ++i) left[i] = R.sections[i];
    for (int i = 0; i < pairs; ++i) {
        while (left[a] == 0) a = (a + 1) % R.n_axes;                     // (the sections' sum is `pairs`: one is left)
        --left[a];
        A.axes[i / 8] |= (uint16_t)(a << (2 * (i % 8)));
        if (R.interleaved) a = (a + 1) % R.n_axes;
    }
    // (one power and a product for each pair: 2^-64 of relative error a product, 128 of them)
    const long double step = powl((long double)R.theta, -2.0L / R.d);
    long double speed = 0x1p64L * 0.15915494309189533576888376337251436L;
    for (int i = 0; i < pairs; ++i, speed *= step) A.speed[i] = (uint64_t)(speed + 0.5L);
    const int64_t units = (int64_t)R.B * R.T * (R.d / 16) * heads;
    const int per_thread = units >= (1 << 20) ? 4 : (units >= (1 << 18) ? 2 : 1);
    A.slots = (heads + per_thread - 1) / per_thread;
    const int64_t threads = (int64_t)R.B * R.T * (R.d / 16) * A.slots;
    auto* kernel = per_thread == 4 ? rope_axes_kernel<4> : (per_thread == 2 ? rope_axes_kernel<2> : rope_axes_kernel<1>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((threads + RA_THREADS - 1) / RA_THREADS)), dim3(RA_THREADS), 0, s, A);
    return launch_status("rope_axes");
}

// Rows to the caches: 16 bytes a thread.
constexpr int CA_THREADS = 256, CA_LAYERS = 64;
struct CacheAppendArgs {
    vitcop_cache_append_t A;
    int first, sides;                       // layer; of k and v, those given
    uint16_t* cache[2][CA_LAYERS];          // of k, of v
    int start[CA_LAYERS];
};
__global__ __launch_bounds__(CA_THREADS) void cache_append_kernel(const CacheAppendArgs P) {
    const vitcop_cache_append_t& A = P.A;
    const int layer = blockIdx.z / P.sides, of_v = P.sides == 2 ? blockIdx.z & 1 : A.k == nullptr, b = blockIdx.y;
    const unsigned chunks = (unsigned)(A.Hkv * A.d) / 8, id = blockIdx.x * CA_THREADS + threadIdx.x;
    const int i = (int)(id / chunks), c = (int)(id - (unsigned)i * chunks);
    if (i >= (A.n_samples ? min(A.n_samples[b], A.rows) : A.rows)) return;
    const int from = A.idx ? A.idx[(int64_t)b * A.rows + i] : i;
    const int64_t to = (int64_t)(A.start_samples ? A.start_samples[(int64_t)(P.first + layer) * A.B + b] : P.start[layer]) + i;
    if (from < 0 || from >= A.T || to < 0 || to >= A.capacity) return;
    const uint16_t* src = of_v ? A.v + (P.first + layer) * A.v_layer_stride + b * A.v_batch_stride + from * A.v_row_stride
                               : A.k + (P.first + layer) * A.k_layer_stride + b * A.k_batch_stride + from * A.k_row_stride;
    uint16_t* dst = P.cache[of_v][layer] + ((int64_t)b * A.capacity + to) * A.Hkv * A.d;
    *reinterpret_cast<uint4*>(dst + 8 * c) = *reinterpret_cast<const uint4*>(src + 8 * c);
}

int launch_cache_append(const vitcop_cache_append_t& A, hipStream_t s) {
    const int64_t units = (int64_t)A.rows * A.Hkv * A.d / 8;
    for (int first = 0; first < A.n_layers; first += CA_LAYERS) {
        CacheAppendArgs P{};
        P.A = A;
        P.first = first;
        P.sides = (A.k != nullptr) + (A.v != nullptr);
        const int n = std::min(CA_LAYERS, A.n_layers - first);
        for (int l = 0; l < n; ++l) {
            if (A.k) P.cache[0][l] = A.k_cache[first + l];
            if (A.v) P.cache[1][l] = A.v_cache[first + l];
            P.start[l] = A.start_samples ? 0 : A.start[first + l];
        }
        hipLaunchKernelGGL(cache_append_kernel, dim3((unsigned)((units + CA_THREADS - 1) / CA_THREADS), A.B, P.sides * n),
                           dim3(CA_THREADS), 0, s, P);
        const int rc = launch_status("cache_append");
        if (rc) return rc;
    }
    return VITCOP_OK;
}

}  // namespace vitcop
