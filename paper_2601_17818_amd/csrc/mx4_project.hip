// Projections of few rows by a matrix held in 4 bits (format: mx4_device.h): y = x W^T (+ residual), the few rows of a
// decoding step's new tokens.  Bound by the matrix' bytes, 17/32 of one a value, each read once for every 64 rows of x.
//
// A workgroup takes 16 RT rows of W and its wavefronts take turns at their columns, 128 at a time: a lane's 16 bytes are one
// group of 32 columns of one row of W, which the conversion turns straight into operands of the product (16x16x32, W's rows
// as the product's rows, MB blocks of 16 rows of x as its columns); the order of the columns in a sum is free as long as x is
// read in the same one.  The wavefronts' sums meet in LDS and are added in a fixed order.
// Columns past K and rows past M read as zeros: their offsets lie past the descriptors' ends.
#include "vitcop_internal.h"
#include "mx4_device.h"

#include <algorithm>

namespace vitcop {

constexpr unsigned MP_OUTSIDE = 0x80000000u;         // every operand is smaller

struct MpArgs {
    const uint16_t* x;
    const uint8_t* codes;
    const uint8_t* scales;
    uint16_t* y;
    const uint16_t* res;
    int64_t x_stride, y_stride, res_stride;
    int M, N, K;
};

template <int MB, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_project_kernel(MpArgs a) {
    __shared__ f32x4 sums[WAVES][RT * MB][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
    const int n0 = blockIdx.x * (16 * RT), m0 = blockIdx.y * (16 * MB);
    const int groups = a.K / MX4_GROUP, chunks = (groups + 3) / 4;
    const auto c_desc = __builtin_amdgcn_make_buffer_rsrc((void*)a.codes, 0, (unsigned)((int64_t)a.N * a.K / 2), 0x00020000);
    const auto s_desc = __builtin_amdgcn_make_buffer_rsrc((void*)a.scales, 0, (unsigned)((int64_t)a.N * groups), 0x00020000);
    const auto x_desc = __builtin_amdgcn_make_buffer_rsrc((void*)a.x, 0, (unsigned)(((a.M - 1) * a.x_stride + a.K) * 2), 0x00020000);
    unsigned c_off[RT], s_off[RT], x_off[MB];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int n = n0 + 16 * r + l16;
        c_off[r] = n < a.N ? (unsigned)n * (unsigned)(a.K / 2) : MP_OUTSIDE;
        s_off[r] = n < a.N ? (unsigned)n * (unsigned)groups : MP_OUTSIDE;
    }
#pragma unroll
    for (int j = 0; j < MB; ++j) {
        const int m = m0 + 16 * j + l16;
        x_off[j] = m < a.M ? (unsigned)(m * a.x_stride * 2) : MP_OUTSIDE;
    }
    u32x4 cw[RT], xv[MB][4];
    uint32_t ce[RT];
    auto load = [&](int chunk) __attribute__((always_inline)) {
        const unsigned g = (unsigned)(4 * chunk + g4), outside = g < (unsigned)groups ? 0u : MP_OUTSIDE;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            cw[r] = __builtin_amdgcn_raw_buffer_load_b128(c_desc, (c_off[r] + 16 * g) | outside, 0, 0);
            ce[r] = __builtin_amdgcn_raw_buffer_load_b8(s_desc, (s_off[r] + g) | outside, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                xv[j][c] = __builtin_amdgcn_raw_buffer_load_b128(x_desc, (x_off[j] + 64 * g + 16 * c) | outside, 0, 0);
    };
    f32x4 acc[RT][MB];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MB; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (wv < chunks) load(wv);
    for (int chunk = wv; chunk < chunks; chunk += WAVES) {
        u32x4 cc[RT], xx[MB][4];
        uint32_t ee[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            cc[r] = cw[r];
            ee[r] = ce[r];
        }
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) xx[j][c] = xv[j][c];
        if (chunk + WAVES < chunks) load(chunk + WAVES);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bf16x8 w = __builtin_bit_cast(bf16x8, mx4_values(cc[r][c], mx4_scale(ee[r])));
#pragma unroll
                for (int j = 0; j < MB; ++j)
                    acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, xx[j][c]), acc[r][j], 0, 0, 0);
            }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MB; ++j) sums[wv][r * MB + j][lane] = acc[r][j];
    __syncthreads();
    // a thread adds up four neighbouring columns of a row of y
    for (int idx = threadIdx.x; idx < RT * MB * 64; idx += 64 * WAVES) {
        const int t = idx >> 6, r = t / MB, j = t - r * MB, ln = idx & 63;
        const int n = n0 + 16 * r + 4 * (ln >> 4), m = m0 + 16 * j + (ln & 15);
        if (n >= a.N || m >= a.M) continue;
        f32x4 v = sums[0][t][ln];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += sums[w][t][ln];
        if (a.res) {
            const uint2 u = *reinterpret_cast<const uint2*>(a.res + m * a.res_stride + n);
            v += f32x4{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
        }
        *reinterpret_cast<uint2*>(a.y + m * a.y_stride + n) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
}

template <int MB, int RT, int WAVES>
static int launch_rows(const MpArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((mx4_project_kernel<MB, RT, WAVES>), dim3((a.N + 16 * RT - 1) / (16 * RT), (a.M + 16 * MB - 1) / (16 * MB)),
                       dim3(64 * WAVES), 0, s, a);
    return launch_status("mx4_project");
}

size_t project_mx4_workspace_bytes(int M, int N, int K) { return 0; }

int launch_project_mx4(const uint16_t* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales, uint16_t* y,
                       int64_t y_stride, const uint16_t* res, int64_t res_stride, int M, int N, int K, void* ws,
                       size_t ws_bytes, hipStream_t s) {
    const MpArgs a{x, codes, scales, y, res, x_stride, y_stride, res_stride, M, N, K};
    if (M <= 16) return launch_rows<1, 1, 8>(a, s);
    if (M <= 32) return launch_rows<2, 2, 8>(a, s);
    return launch_rows<4, 2, 8>(a, s);
}

}  // namespace vitcop
