// Rotary embedding with a position for each of several axes, on the way to a buffer of queries and the rows of a cache; and
// rows written to the caches of all layers.  Both move each byte once: HBM-bound, and a launch's latency where tokens are few.
#include "vitcop_internal.h"
#include "device_utils.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace vitcop {

// theta^(-2i/d) / (2 pi) as a fraction of 2^64: position * fraction modulo 2^64 is the angle's part of a revolution, which a
// 32-bit product of a far position and a speed has lost (position 10^5, the fastest pair: 2^-8 of a radian), and costs two
// integer products instead of arithmetic in 64-bit floating point.  The host gives the speed of every eighth pair, each thread
// goes on from there by products with theta^(-2/d) (64 bits of each are kept: the eighth is off by less than 2^-60, the farthest
// position's angle by 2^-29 of a revolution), which keeps the launch's arguments short: all speeds of 128 channels and the caches'
// descriptor took 6.8 us of host time a call, this 4.1.
struct RopeAxesArgs {
    vitcop_rope_axes_t R;
    int slots;                          // threads that share a pair group's heads
    uint16_t axes[16];                  // two bits for each of a group's eight pairs
    uint64_t speed[16], step;
};

constexpr int RA_THREADS = 256;

// A thread turns eight pairs (16 bytes of a head's lower half and 16 of its upper one) of up to HEADS heads of a token: its
// sines and cosines serve them all, and their loads go out together.  The heads of v pass through.  Stores are non-temporal: us
// with ordinary and with these, inputs from memory, 2 x 6400 tokens of 28 + 2 x 4 heads 49.5, 45.5 (5.2 TB/s), 8 x 1500 of
// 3 x 32 110, 103.5, 4 x up to 640 of them 13.8, 13.1, 64 x up to 700 of 16 + 2 x 4 of 64 38.2, 32.7; non-temporal loads as well
// 43.4, 99.8, 13.5, 38.1 (what has just been projected is better left where it is).
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
    const bool k_in_place = R.k && R.k_out == R.k, fits = k_in_place || (row >= 0 && row < R.capacity);
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
    uint64_t speed = A.speed[group];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned a = (axes >> (2 * i)) & 3;
        const int p = a < 2 ? (a == 0 ? pos[0] : pos[1]) : (a == 2 ? pos[2] : pos[3]);
        const uint64_t turn = (uint64_t)(int64_t)p * speed;
        speed = __umul64hi(speed, A.step);
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
        st_nt16(dst[i] + c0, lo[i]);
        st_nt16(dst[i] + half + c0, hi[i]);
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
    const long double step = powl((long double)R.theta, -2.0L / R.d), two = step * step, eight = two * two * two * two;
    A.step = (uint64_t)(step * 0x1p64L + 0.5L);                          // (theta > 1: below 1)
    long double speed = 0x1p64L * 0.15915494309189533576888376337251436L;
    for (int i = 0; i < pairs / 8; ++i, speed *= eight) A.speed[i] = (uint64_t)(speed + 0.5L);
    const int64_t units = (int64_t)R.B * R.T * (R.d / 16) * heads;
    const int per_thread = units >= (1 << 20) ? 4 : (units >= (1 << 18) ? 2 : 1);
    A.slots = (heads + per_thread - 1) / per_thread;
    const int64_t threads = (int64_t)R.B * R.T * (R.d / 16) * A.slots;
    auto* kernel = per_thread == 4 ? rope_axes_kernel<4> : (per_thread == 2 ? rope_axes_kernel<2> : rope_axes_kernel<1>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((threads + RA_THREADS - 1) / RA_THREADS)), dim3(RA_THREADS), 0, s, A);
    return launch_status("rope_axes");
}

// Rows to the caches: 16 bytes a thread, with non-temporal stores (us with ordinary and with these, of 8 KB a row: 32 layers x 16
// samples x up to 8 of 16 rows 26.3, 19.3, 4 x 16 x 64 19.5, 14.4).  The caches of up to CA_LAYERS layers by a table, or, where
// they are one allocation, by the first one and their distance, which spares the call the table (32 layers, host time with the
// binding 14.0 -> 10.1 us).
constexpr int CA_THREADS = 256, CA_LAYERS = 64;
struct CacheTable {
    uint16_t* cache[2][CA_LAYERS];          // of k, of v
    int start[CA_LAYERS];
};
struct CacheStack {
    uint16_t* cache[2];
    int64_t stride;
};
template <typename CACHES>
struct CacheAppendArgs {
    vitcop_cache_append_t A;
    int first, sides;                       // layer; of k and v, those given
    CACHES caches;
};
template <typename CACHES>
__global__ __launch_bounds__(CA_THREADS) void cache_append_kernel(const CacheAppendArgs<CACHES> P) {
    const vitcop_cache_append_t& A = P.A;
    const int layer = blockIdx.z / P.sides, of_v = P.sides == 2 ? blockIdx.z & 1 : A.k == nullptr, b = blockIdx.y;
    const unsigned chunks = (unsigned)(A.Hkv * A.d) / 8, id = blockIdx.x * CA_THREADS + threadIdx.x;
    const int i = (int)(id / chunks), c = (int)(id - (unsigned)i * chunks);
    if (i >= (A.n_samples ? min(A.n_samples[b], A.rows) : A.rows)) return;
    const int from = A.idx ? A.idx[(int64_t)b * A.rows + i] : i;
    int64_t to;
    uint16_t* cache;
    if constexpr (std::is_same<CACHES, CacheTable>::value) {
        to = A.start_samples ? A.start_samples[(int64_t)(P.first + layer) * A.B + b] : P.caches.start[layer];
        cache = P.caches.cache[of_v][layer];
    } else {
        to = A.start_samples[(int64_t)layer * A.B + b];
        cache = P.caches.cache[of_v] + layer * P.caches.stride;
    }
    to += i;
    if (from < 0 || from >= A.T || to < 0 || to >= A.capacity) return;
    const uint16_t* src = of_v ? A.v + (P.first + layer) * A.v_layer_stride + b * A.v_batch_stride + from * A.v_row_stride
                               : A.k + (P.first + layer) * A.k_layer_stride + b * A.k_batch_stride + from * A.k_row_stride;
    uint16_t* dst = cache + ((int64_t)b * A.capacity + to) * A.Hkv * A.d;
    st_nt16(dst + 8 * c, *reinterpret_cast<const uint4*>(src + 8 * c));
}

int launch_cache_append(const vitcop_cache_append_t& A, hipStream_t s) {
    const int64_t units = (int64_t)A.rows * A.Hkv * A.d / 8;
    const int sides = (A.k != nullptr) + (A.v != nullptr);
    const unsigned wgs = (unsigned)((units + CA_THREADS - 1) / CA_THREADS);
    if (A.cache_layer_stride != 0 && A.start_samples && A.n_layers * sides <= 65535) {
        const CacheStack caches{{A.k ? A.k_cache[0] : nullptr, A.v ? A.v_cache[0] : nullptr}, A.cache_layer_stride};
        const CacheAppendArgs<CacheStack> P{A, 0, sides, caches};
        hipLaunchKernelGGL(cache_append_kernel<CacheStack>, dim3(wgs, A.B, sides * A.n_layers), dim3(CA_THREADS), 0, s, P);
        return launch_status("cache_append");
    }
    for (int first = 0; first < A.n_layers; first += CA_LAYERS) {
        CacheAppendArgs<CacheTable> P{A, first, sides, {}};
        const int n = std::min(CA_LAYERS, A.n_layers - first);
        for (int l = 0; l < n; ++l) {
            const int at = first + l;
            if (A.k) P.caches.cache[0][l] = A.cache_layer_stride ? A.k_cache[0] + at * A.cache_layer_stride : A.k_cache[at];
            if (A.v) P.caches.cache[1][l] = A.cache_layer_stride ? A.v_cache[0] + at * A.cache_layer_stride : A.v_cache[at];
            P.caches.start[l] = A.start_samples ? 0 : A.start[at];
        }
        hipLaunchKernelGGL(cache_append_kernel<CacheTable>, dim3(wgs, A.B, sides * n), dim3(CA_THREADS), 0, s, P);
        const int rc = launch_status("cache_append");
        if (rc) return rc;
    }
    return VITCOP_OK;
}

}  // namespace vitcop
