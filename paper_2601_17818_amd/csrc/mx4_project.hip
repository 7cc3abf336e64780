// Projections by a matrix held in 4 bits (format: mx4_device.h): y = x W^T (+ residual), for the few rows of a decoding step's
// new tokens and up to the rows that survive pruning (for thousands, see the choice of the launch below).  Bound by the matrix'
// bytes, 17/32 of one a value, until there are some ten rows; then by x, which every workgroup reads, and from some hundred
// rows on by the matrix cores.
//
// The codes go to LDS as they are, and only an operand of a product is turned into bf16 (one instruction for two values, the
// group's power of two included; W's rows are the product's rows, x's rows its columns, 16x16x32).  A lane's 16 bytes of
// codes are one group of 32 columns of one row, and since the order of the columns in a sum is free as long as x is read in
// the same one, they are the operands of four products.  Loads go straight to LDS, neighbouring lanes for neighbouring bytes:
// an operand's lanes hold a row each, and loads in that order cost a cycle for every lane (1 x 4096 x 11008: 10.0 us, now 6.3).
// LDS serves 16 lanes' 16 bytes at a time; the 16-byte pieces of a row are stored in an order in which 16 rows' same pieces
// lie in different banks.  Columns past K and rows past M or N read as zeros: their offsets lie past the descriptors' ends.
#include "vitcop_internal.h"
#include "mx4_device.h"
#include "mx4_plan.h"

#include <algorithm>
#include <atomic>

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
    float* part;                         // slices of K: [slices][M][N] sums, left to be added up; or nullptr
    int slices, steps_per_slice;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t mp_desc(const void* base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (unsigned)bytes, 0x00020000);
}

// 16 bytes a lane from memory to the 1024 bytes of LDS at `to`
__device__ __forceinline__ void mp_load(__amdgpu_buffer_rsrc_t from, char* to, unsigned offset) {
#ifdef __HIP_DEVICE_COMPILE__                 // (the host's pass does not know loads of 16 bytes)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
#endif
}

// More than 64 KB of dynamic LDS for a kernel, once for every device (`raised`: a bit for each, one such word an instantiation;
// a second thread that repeats the call does no harm).
static int mp_raise_lds(const void* kernel, int bytes, std::atomic<uint64_t>& raised) {
    int device = 0;
    int rc = hip_status(hipGetDevice(&device), "hipGetDevice");
    const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
    if (rc || (raised.load(std::memory_order_acquire) & bit)) return rc;
    rc = hip_status(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes),
                    "hipFuncSetAttribute(project_mx4)");
    if (rc == VITCOP_OK) raised.fetch_or(bit, std::memory_order_release);
    return rc;
}

// At most 16 rows of x (or any number, 16 at a time): a workgroup takes 16 R rows of W, and its wavefronts take turns at their
// columns, 128 at a time, each with DEPTH steps in flight in an LDS ring of its own; their sums meet at the end, in a fixed
// order.  XI: loads of four rows of x a step.  Measured with weights from HBM, us (of which 2.5 are the launch): 1 x 4096 x 4096
// 4.4, 1 x 11008 x 4096 7.0 (23.9 MB in 4.4 us: 5.4 TB/s), 8 x 11008 x 4096 7.9, 16 x 11008 x 4096 9.0.
template <int R, int XI, int WAVES, int DEPTH>
constexpr int mp_ring_bytes() { return WAVES * DEPTH * (R + XI) * 1024; }

template <int R, int XI, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void mx4_few_kernel(MpArgs a) {
    constexpr int NL = R + XI, SLOT = NL * 1024;             // loads a step, bytes of a step in the ring
    static_assert(R <= WAVES, "a wavefront for every 16 rows at the end");
    extern __shared__ __attribute__((aligned(16))) char mp_lds[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * (16 * R), m0 = blockIdx.y * 16;
    const int groups = a.K / MX4_GROUP, steps = (groups + 3) / 4, rows = min(16 * R, a.N - n0);
    const auto c_desc = mp_desc(a.codes + (int64_t)n0 * (a.K / 2), rows * (a.K / 2));
    const auto s_desc = mp_desc(a.scales + (int64_t)n0 * groups, rows * groups);
    const auto x_desc = mp_desc(a.x + m0 * a.x_stride, ((a.M - m0 - 1) * a.x_stride + a.K) * 2);
    char* const ring = mp_lds + wv * (DEPTH * SLOT);
    char* const exps = mp_lds + mp_ring_bytes<R, XI, WAVES, DEPTH>();
    // the epilogue's part of the first R wavefronts: four neighbouring columns of a row of y a lane
    const int n = n0 + 16 * wv + 4 * g4, m = m0 + l16;
    const bool mine = wv < R && n < a.N && m < a.M;
    uint2 res = make_uint2(0, 0);
    if (a.res && mine) res = *reinterpret_cast<const uint2*>(a.res + m * a.res_stride + n);
    // the exponents of these rows: one contiguous run
    for (int u = 64 * wv; u < R * groups; u += 64 * WAVES) mp_load(s_desc, exps + u * 16, (u + lane) * 16);
    // where this lane's 16 bytes of a load come from
    const int c_grp = lane % 4 ^ (lane >> 4);
    const unsigned c_off = (unsigned)(lane / 4) * (unsigned)(a.K / 2) + 16 * c_grp, c_next = 16 * (unsigned)(a.K / 2);
    unsigned x_off[XI];
    int x_slot[XI];
#pragma unroll
    for (int q = 0; q < XI; ++q) {
        const int row = 4 * q + lane / 16;
        x_slot[q] = lane % 16 ^ row;
        x_off[q] = m0 + row < a.M ? (unsigned)(row * a.x_stride * 2) + 16 * x_slot[q] : MP_OUTSIDE;
    }
    auto load = [&](int slot, int step) __attribute__((always_inline)) {
        char* const to = ring + slot * SLOT;
#pragma unroll
        for (int r = 0; r < R; ++r)
            mp_load(c_desc, to + r * 1024, (c_off + r * c_next + 64 * step) | (4 * step + c_grp < groups ? 0u : MP_OUTSIDE));
#pragma unroll
        for (int q = 0; q < XI; ++q)
            mp_load(x_desc, to + (R + q) * 1024,
                    (x_off[q] + 256 * step) | (4 * step + (x_slot[q] >> 2) < groups ? 0u : MP_OUTSIDE));
    };
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) load(i, wv + i * WAVES);         // (past the last step: nothing is fetched)
    f32x4 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(DEPTH * NL) : "memory");
    __builtin_amdgcn_s_barrier();                            // everybody's exponents are there
    asm volatile("" ::: "memory");
    int slot = 0;
    for (int step = wv; step < steps; step += WAVES) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * NL) : "memory");
        const char* const from = ring + slot * SLOT;
        const int row = min(l16, 4 * XI - 1);                // (rows past M: whatever the last loaded one gives, not stored)
        u32x4 cc[R], xx[4];
        uint32_t ee[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            cc[r] = *reinterpret_cast<const u32x4*>(from + r * 1024 + l16 * 64 + (g4 ^ (l16 >> 2)) * 16);
            ee[r] = *reinterpret_cast<const uint8_t*>(exps + (16 * r + l16) * groups + min(4 * step + g4, groups - 1));
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            xx[c] = *reinterpret_cast<const u32x4*>(from + R * 1024 + row * 256 + ((4 * g4 + c) ^ row) * 16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load(slot, step + DEPTH * WAVES);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int r = 0; r < R; ++r)
                acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, mx4_values(cc[r][c], mx4_scale(ee[r]))),
                                                                 __builtin_bit_cast(bf16x8, xx[c]), acc[r], 0, 0, 0);
        slot = slot + 1 == DEPTH ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");          // no load may outlive the ring
    __syncthreads();
    f32x4 (*sums)[R][64] = reinterpret_cast<f32x4 (*)[R][64]>(mp_lds);
#pragma unroll
    for (int r = 0; r < R; ++r) sums[wv][r][lane] = acc[r];
    __syncthreads();
    if (!mine) return;
    f32x4 v = sums[0][wv][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += sums[w][wv][lane];
    v += f32x4{bf16_lo(res.x), bf16_hi(res.x), bf16_lo(res.y), bf16_hi(res.y)};
    *reinterpret_cast<uint2*>(a.y + m * a.y_stride + n) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

template <int R, int XI, int WAVES, int DEPTH>
static int launch_few(const MpArgs& a, hipStream_t s) {
    constexpr int ring = mp_ring_bytes<R, XI, WAVES, DEPTH>(), most = ring + R * (R == 4 ? 16384 : 32768);
    static_assert(most <= 160 * 1024, "LDS of a CU: K = 2^16, and 2^15 with 64 rows of W");
    const size_t lds = ring + ((size_t)a.K / 2 * R + 1023) / 1024 * 1024;
    static std::atomic<uint64_t> raised{0};
    if (lds > 65536) {
        const int rc = mp_raise_lds(reinterpret_cast<const void*>(&mx4_few_kernel<R, XI, WAVES, DEPTH>), most, raised);
        if (rc) return rc;
    }
    hipLaunchKernelGGL((mx4_few_kernel<R, XI, WAVES, DEPTH>), dim3((a.N + 16 * R - 1) / (16 * R), (a.M + 15) / 16),
                       dim3(64 * WAVES), lds, s, a);
    return launch_status("mx4_few");
}

// the kernel of few_plan, which is one of these
template <int R, int XI, int WAVES, int DEPTH>
static bool launched(const FewPlan& p, const MpArgs& a, hipStream_t s, int& rc) {
    if (p.blocks != R || p.x_loads != XI || p.waves != WAVES || p.depth != DEPTH) return false;
    rc = launch_few<R, XI, WAVES, DEPTH>(a, s);
    return true;
}
static int launch_few_rows(const MpArgs& a, hipStream_t s) {
    const FewPlan p = few_plan(a.M, a.N, a.K);
    int rc = VITCOP_EUNSUPPORTED;
    launched<1, 1, 4, 2>(p, a, s, rc) || launched<1, 1, 8, 3>(p, a, s, rc) || launched<2, 1, 4, 3>(p, a, s, rc) ||
        launched<2, 1, 4, 2>(p, a, s, rc) || launched<1, 2, 4, 2>(p, a, s, rc) || launched<1, 2, 8, 2>(p, a, s, rc) ||
        launched<2, 2, 4, 3>(p, a, s, rc) || launched<3, 2, 4, 2>(p, a, s, rc) || launched<4, 2, 4, 2>(p, a, s, rc) ||
        launched<1, 4, 4, 3>(p, a, s, rc) || launched<2, 4, 4, 2>(p, a, s, rc) || launched<3, 4, 4, 2>(p, a, s, rc) ||
        launched<4, 4, 4, 2>(p, a, s, rc);
    return rc;
}

// More rows: eight wavefronts, MT_WM by MT_WN, take 32 MB rows of x and 64 RT rows of W over a slice of K, 128 columns at a time,
// both operands through a ring of NS steps in LDS that all of them read.  A step moves 8 (4 MB + RT) KB from LDS and 8 MB + 4 RT
// KB into it at 128 bytes a cycle (MB = 5, RT = 2: 1730 cycles) and multiplies 4 MB RT times a wavefront (1280 cycles a SIMD);
// without loads from memory it takes 2250, with them some 3000.  RT = 4 reads x half as often (MB = 4: 1630 and 2048 cycles) and
// reaches 1.02 PFLOP/s at 1024 x 4096 x 11008, where a large bf16 product reaches 1.5 to 1.6; without its reads of x, its loads, its
// conversions that took 8, 3 and 0 % less.  Tried and not kept (the kernel's own time at 64 x 4096 x 11008 and at 317 x 3584 x 14336):
// reading a step ahead into registers, between the products (+4, -1 %), four wavefronts with twice the columns each (+7, +12 %),
// different starts in k (+1, +11 %).  K >= 512; WHOLE: whole steps.  The slices' sums are added by mx4_sum_kernel.
constexpr int MT_WM = 2, MT_WN = 4, MT_WAVES = MT_WM * MT_WN;
template <int MB, int RT, int NS>
constexpr int mp_tile_bytes() { return NS * (16 * MB * MT_WM * 256 + 16 * RT * MT_WN * 64) + 3 * 16 * RT * MT_WN * 16; }

template <int MB, int RT, int NS, bool WHOLE>
__global__ __launch_bounds__(64 * MT_WAVES) void mx4_tile_kernel(MpArgs a) {
    constexpr int BM = 16 * MB * MT_WM, BN = 16 * RT * MT_WN, EXPS = BN * 16;                // (EXPS: bytes of a unit of exponents)
    // loads of x, of codes, of both a wavefront and step, bytes of a step
    constexpr int XL = BM / (4 * MT_WAVES), CL = BN / (16 * MT_WAVES), NL = XL + CL, SLOT = BM * 256 + BN * 64;
    static_assert(XL * 4 * MT_WAVES == BM && CL * 16 * MT_WAVES == BN, "whole loads for every wavefront");
    extern __shared__ __attribute__((aligned(16))) char mp_lds[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv % MT_WM, wn = wv / MT_WM;
    // an XCD takes an eighth of the tiles, one after the other, so that none has more than its CUs while others have fewer
    // (75 x 4272 x 9856, 34 columns of tiles and seven slices: 20.4 us; columns dealt out whole 31.5); those of the same rows
    // of W together, which share its L2, all slices of them: parts of rows a power of two apart would share its channels
    const unsigned tiles_m = (a.M + BM - 1) / BM;
    const unsigned id = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), col = id / tiles_m;
    const int slice = col % a.slices, n0 = col / a.slices * BN, m0 = id % tiles_m * BM;
    if (n0 >= a.N) return;
    const int groups = a.K / MX4_GROUP;
    const int first = slice * a.steps_per_slice, end = min((groups + 3) / 4, first + a.steps_per_slice);
    const int rows = min(BN, a.N - n0);
    const auto c_desc = mp_desc(a.codes + (int64_t)n0 * (a.K / 2), (int64_t)rows * (a.K / 2));
    const int s_bytes = (rows * groups + 3) & ~3;            // (whole words)
    const auto s_desc = mp_desc(a.scales + (int64_t)n0 * groups, s_bytes);
    const auto x_desc = mp_desc(a.x + m0 * a.x_stride, ((a.M - m0 - 1) * a.x_stride + a.K) * 2);
    const int c_grp = lane % 4 ^ (lane >> 4);
    const unsigned c_off = (unsigned)(16 * CL * wv + lane / 4) * (unsigned)(a.K / 2) + 16 * c_grp;
    const unsigned c_next = 16 * (unsigned)(a.K / 2);
    unsigned x_off[XL];
    int x_grp[XL];
#pragma unroll
    for (int q = 0; q < XL; ++q) {
        const int row = 4 * (XL * wv + q) + lane / 16, piece = lane % 16 ^ (row & 15);
        x_grp[q] = piece >> 2;
        x_off[q] = m0 + row < a.M ? (unsigned)(row * a.x_stride * 2) + 16 * piece : MP_OUTSIDE;
    }
    auto load = [&](int slot, int step) __attribute__((always_inline)) {
        char* const to = mp_lds + slot * SLOT;
        auto past = [&](int grp) __attribute__((always_inline)) {
            return step < end && (WHOLE || 4 * step + grp < groups) ? 0u : MP_OUTSIDE;
        };
#pragma unroll
        for (int i = 0; i < CL; ++i)
            mp_load(c_desc, to + BM * 256 + (CL * wv + i) * 1024, (c_off + i * c_next + 64 * step) | past(c_grp));
#pragma unroll
        for (int q = 0; q < XL; ++q) mp_load(x_desc, to + (XL * wv + q) * 1024, (x_off[q] + 256 * step) | past(x_grp[q]));
    };
    // Exponents come in units, 16 bytes of a row a lane: those of four steps, a row's last unit ending with it, or where rows
    // do not start at whole words of three, from the word on that holds the first.  Two are asked for here, and with every
    // step of a unit some rows of the one after the next.
    constexpr int UNIT = WHOLE ? 4 : 3, ROWS = (BN + UNIT * MT_WAVES - 1) / (UNIT * MT_WAVES);       // steps; rows a wavefront
    static_assert(2 * BN / 64 <= MT_WAVES && ROWS <= 64, "two units in one load each");
    char* const scales = mp_lds + NS * SLOT;
    auto unit_at = [&](int row, int unit) __attribute__((always_inline)) {
        return WHOLE ? row * groups + min(4 * first + 16 * unit, groups - 16)
                     : min((row * groups + 4 * first + 12 * unit) & ~3, s_bytes - 16);
    };
    if (wv < 2 * BN / 64) mp_load(s_desc, scales + wv * 1024, (unsigned)unit_at(wv % (BN / 64) * 64 + lane, wv / (BN / 64)));
    f32x4 acc[RT][MB];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MB; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) load(i, first + i);     // (past the last step: nothing is fetched)
    int slot = 0, ahead = NS - 1, unit = 0, exp_slot = 0, phase = 0;
    for (int step = first; step < end; ++step) {
        // everybody's loads for this step are there (at least NL for each later one were issued after them), and everybody has
        // read the slots that are filled next
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * NL) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const char* const from = mp_lds + slot * SLOT;
        const char* const exps = scales + exp_slot * EXPS;
        const int grp = WHOLE ? 4 * step + g4 : min(4 * step + g4, groups - 1);
        u32x4 cc[RT], xx[MB][4];
        uint32_t ee[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = 16 * (RT * wn + r) + l16;
            cc[r] = *reinterpret_cast<const u32x4*>(from + BM * 256 + row * 64 + (g4 ^ (l16 >> 2)) * 16);
            ee[r] = *reinterpret_cast<const uint8_t*>(exps + row * 16 + ((row * groups + grp - unit_at(row, unit)) & 15));
        }
#pragma unroll
        for (int j = 0; j < MB; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                xx[j][c] = *reinterpret_cast<const u32x4*>(from + (16 * (MB * wm + j) + l16) * 256 + ((4 * g4 + c) ^ l16) * 16);
        const int e_row = ROWS * (MT_WAVES * phase + wv);
        if (lane < ROWS && e_row + lane < BN)
            mp_load(s_desc, scales + (exp_slot == 0 ? 2 : exp_slot - 1) * EXPS + e_row * 16,
                    (unsigned)unit_at(e_row + lane, unit + 2));
        load(ahead, step + NS - 1);
        if (++phase == UNIT) {
            phase = 0;
            ++unit;
            exp_slot = exp_slot == 2 ? 0 : exp_slot + 1;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bf16x8 w = __builtin_bit_cast(bf16x8, mx4_values(cc[r][c], mx4_scale(ee[r])));
#pragma unroll
                for (int j = 0; j < MB; ++j)
                    acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, xx[j][c]), acc[r][j], 0, 0, 0);
            }
        slot = slot + 1 == NS ? 0 : slot + 1;
        ahead = ahead + 1 == NS ? 0 : ahead + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");          // no load may outlive the workgroup's LDS
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < MB; ++j) {
            const int n = n0 + 16 * (RT * wn + r) + 4 * g4, m = m0 + 16 * (MB * wm + j) + l16;
            if (n >= a.N || m >= a.M) continue;
            f32x4 v = acc[r][j];
            if (a.part) {
                *reinterpret_cast<f32x4*>(a.part + ((int64_t)slice * a.M + m) * a.N + n) = v;
                continue;
            }
            if (a.res) {
                const uint2 u = *reinterpret_cast<const uint2*>(a.res + m * a.res_stride + n);
                v += f32x4{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
            }
            *reinterpret_cast<uint2*>(a.y + m * a.y_stride + n) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        }
}

template <int MB, int RT, int NS, bool WHOLE>
static int launch_tiles_of(const MpArgs& a, hipStream_t s) {
    const int tiles = (a.N + 16 * RT * MT_WN - 1) / (16 * RT * MT_WN) * ((a.M + 32 * MB - 1) / (32 * MB)) * a.slices;
    constexpr int lds = mp_tile_bytes<MB, RT, NS>();
    static_assert(lds <= 160 * 1024, "LDS of a CU");
    static_assert(lds > 65536, "raised for all of them");
    static std::atomic<uint64_t> raised{0};
    const int rc = mp_raise_lds(reinterpret_cast<const void*>(&mx4_tile_kernel<MB, RT, NS, WHOLE>), lds, raised);
    if (rc) return rc;
    hipLaunchKernelGGL((mx4_tile_kernel<MB, RT, NS, WHOLE>), dim3((tiles + 7) / 8 * 8), dim3(64 * MT_WAVES), lds, s, a);
    return launch_status("mx4_tile");
}

template <int MB, int RT, int NS>
static int launch_tiles(const MpArgs& a, hipStream_t s) {
    return a.K % 128 == 0 ? launch_tiles_of<MB, RT, NS, true>(a, s) : launch_tiles_of<MB, RT, NS, false>(a, s);
}

// y = the slices' sums added up in their order (+ residual): four columns of a row a thread, eight slices' loads and the
// residual's in flight at once, since it is a chain of round trips and little else (both kernels of 64 x 4096 x 11008 in eight
// slices 17.3 us; with launch_partial_reduce, whose threads take eight columns and four slices at a time, 17.8).
__global__ __launch_bounds__(256) void mx4_sum_kernel(MpArgs a) {
    const int quads = a.N / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)a.M * quads) return;
    const int64_t m = id / quads, n = (id - m * quads) * 4, slice = (int64_t)a.M * a.N;
    const float* p = a.part + m * a.N + n;
    uint2 res = make_uint2(0, 0);
    if (a.res) res = *reinterpret_cast<const uint2*>(a.res + m * a.res_stride + n);
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < a.slices; s0 += 8) {
        f32x4 t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s0 + i < a.slices) t[i] = *reinterpret_cast<const f32x4*>(p + (s0 + i) * slice);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s0 + i < a.slices) v += t[i];
    }
    v += f32x4{bf16_lo(res.x), bf16_hi(res.x), bf16_lo(res.y), bf16_hi(res.y)};
    *reinterpret_cast<uint2*>(a.y + m * a.y_stride + n) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

static size_t plan_bytes(const MpPlan& p, int M, int N, int K) {
    if (p.unpack) return up256((size_t)N * K * 2) + gemm_workspace_bytes(M, N, K);
    return p.slices > 1 ? up256((size_t)p.slices * M * N * 4) : 0;
}
size_t project_mx4_workspace_bytes(int M, int N, int K) { return plan_bytes(mp_plan(M, N, K), M, N, K); }

int launch_project_mx4(const uint16_t* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales, uint16_t* y,
                       int64_t y_stride, const uint16_t* res, int64_t res_stride, int M, int N, int K, void* ws,
                       size_t ws_bytes, hipStream_t s) {
    MpArgs a{x, codes, scales, y, res, x_stride, y_stride, res_stride, M, N, K, nullptr, 1, 0};
    const MpPlan p = mp_plan(M, N, K);
    const bool scratch = ws_bytes >= plan_bytes(p, M, N, K);
    if (p.unpack && scratch) {
        uint16_t* w = static_cast<uint16_t*>(ws);
        const size_t own = up256((size_t)N * K * 2);
        const int rc = launch_mx4_dequantize(codes, scales, N, K, w, K, s);
        if (rc) return rc;
        return launch_gemm_ws(x, x_stride, w, y, y_stride, res, res_stride, M, N, K, nullptr,
                              ws_bytes > own ? static_cast<char*>(ws) + own : nullptr, ws_bytes - own, s);
    }
    if (p.kind < 0) return launch_few_rows(a, s);
    const bool cut = p.slices > 1 && scratch && !p.unpack;
    a.slices = cut ? p.slices : 1;
    a.steps_per_slice = cut ? p.steps_per_slice : (K + 127) / 128;
    if (cut) a.part = static_cast<float*>(ws);
    int rc = 0;
    switch (p.kind) {
        case 0: rc = launch_tiles<1, 2, 4>(a, s); break;
        case 1: rc = launch_tiles<2, 2, 4>(a, s); break;
        case 2: rc = launch_tiles<3, 2, 3>(a, s); break;
        case 3: rc = launch_tiles<4, 2, 3>(a, s); break;
        case 4: rc = launch_tiles<5, 2, 3>(a, s); break;
        case 5: rc = launch_tiles<3, 4, 3>(a, s); break;
        case 6: rc = launch_tiles<4, 4, 3>(a, s); break;
        default: rc = launch_tiles<5, 4, 2>(a, s); break;
    }
    if (rc || !cut) return rc;
    hipLaunchKernelGGL(mx4_sum_kernel, dim3((unsigned)(((int64_t)M * (N / 4) + 255) / 256)), dim3(256), 0, s, a);
    return launch_status("mx4_sum");
}

}  // namespace vitcop
