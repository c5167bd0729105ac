// C = A W^T: activations in 8 (E4M3) or 4 bits (E2M1) on weights in 4 bits, a power-of-two scale per 32 values on both sides.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 features x 128 values by 128 values x 16 rows and applies both scales itself: lane
// l = 16 q + c gives the scale of block q (32 values) of its feature or row c.  A 4-bit operand is 16 bytes a lane, block q of the
// row; an 8-bit one two pieces of 16 bytes, values 16 q .. and 64 + 16 q .. of the 128.  With weights as the first operand a lane ends
// up with four consecutive features of one row.
#include "sjd_mx.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// The unit adds eight neighbouring products in fixed point.  With E the largest sum of two operands' exponents among the eight it keeps what
// each product has from 2^(E - 13) up and cuts the rest towards zero (seen with a pair that cancels and a third product, for every code);
// other eights are added in fp32.  E4M3 spans 15 binades, so small values beside large ones are cut: 5e-6 of a result in the 2-norm of random
// rows, and up to 2^-13 of the largest product for each of the other seven, whatever is left of the sum.  A bf16 result (4e-3) takes
// that; for fp32 results the activations go in twice, the values from 2 on (codes with bit 0x40) and the others, each with the rest as
// zeros.  Nothing is cut then: products of the large ones have E <= 8 + 2 and are multiples of 2^-2 2^-1, those of the small ones E <= 0 + 2
// and 2^-9 2^-1.  E2M1 times E2M1: E <= 4, 2^-2.
__device__ __forceinline__ uint32_t mx_large(uint32_t w)        // 0xFF in the bytes with bit 0x40
{
    const uint32_t t = (w >> 6) & 0x01010101u;
    return (t << 8) - t;
}
__device__ __forceinline__ uint4 mx_and(const uint4 &a, const uint4 &m) { return make_uint4(a.x & m.x, a.y & m.y, a.z & m.z, a.w & m.w); }
__device__ __forceinline__ uint4 mx_andn(const uint4 &a, const uint4 &m) { return make_uint4(a.x & ~m.x, a.y & ~m.y, a.z & ~m.z, a.w & ~m.w); }
__device__ __forceinline__ uint4 mx_large4(const uint4 &a) { return make_uint4(mx_large(a.x), mx_large(a.y), mx_large(a.z), mx_large(a.w)); }

template <int FMT> __device__ __forceinline__ f32x4 mx_mfma(const uint4 &w, const uint4 &a0, const uint4 &a1, f32x4 acc, int ws, int as)
{
    const i32x8 W = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    const i32x8 A = {(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(W, A, acc, 4, FMT == SJD_MX8 ? 0 : 4, 0, ws, 0, as);
}

__device__ __forceinline__ void mx_store4(float *p, const f32x4 &v, int n, bool vec)
{
    if (vec && n >= 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else for (int i = 0; i < 4; ++i) if (i < n) p[i] = v[i];
}
__device__ __forceinline__ void mx_store4(bf16_t *p, const f32x4 &v, int n, bool vec)
{
    if (vec && n >= 4) *reinterpret_cast<uint2 *>(p) = make_uint2(f32_to_bf16(v[0]) | (uint32_t)f32_to_bf16(v[1]) << 16,
                                                                  f32_to_bf16(v[2]) | (uint32_t)f32_to_bf16(v[3]) << 16);
    else for (int i = 0; i < 4; ++i) if (i < n) p[i] = f32_to_bf16(v[i]);
}

// acc += W A^T for one step of 128 values
template <int FMT, bool EXACT> __device__ __forceinline__ f32x4 mx_step(const uint4 &w, uint4 a0, uint4 a1, f32x4 acc, int ws, int as)
{
    if (FMT == SJD_MX8 && EXACT) {
        const uint4 m0 = mx_large4(a0), m1 = mx_large4(a1);
        acc = mx_mfma<FMT>(w, mx_andn(a0, m0), mx_andn(a1, m1), acc, ws, as);
        a0 = mx_and(a0, m0); a1 = mx_and(a1, m1);
    }
    return mx_mfma<FMT>(w, a0, a1, acc, ws, as);
}

// ---- few rows -------------------------------------------------------------------------------
// A workgroup owns TN tiles of features and up to 16 MT rows; its waves take the records of a tile in turn, so K is split eight ways, and their
// sums meet in LDS in wave order.  A wave has one record of every tile (4 steps of 128 values) and its activations in flight: each
// step's registers are refilled as soon as its products are issued.
template <int FMT, int MT, int TN, typename T>
__global__ __launch_bounds__(512, 2) void mx_rows_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                         const uint8_t *__restrict__ packed, int M, int N, int Kp, int tiles, int groups,
                                                         T *__restrict__ C, int64_t ldc, int vec)
{
    constexpr int WK = 8, F = MT * TN, NA = FMT == SJD_MX8 ? 2 : 1;
    constexpr bool EXACT = sizeof(T) == 4;
    __shared__ f32x4 red[WK][F][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
    const int t0 = (int)blockIdx.x * TN, steps = Kp / 128, arow = FMT == SJD_MX8 ? Kp : Kp / 2, srow = Kp / 32;
    const int64_t row0 = (int64_t)blockIdx.y * (16 * MT);
    const int live = (int)min((int64_t)(16 * MT), M - row0);
    const auto wb = mx_buffer(packed + (size_t)t0 * groups * MX_REC, (size_t)min(TN, tiles - t0) * groups * MX_REC);
    const auto ab = mx_buffer(codes + (size_t)row0 * arow, (size_t)live * arow), sb = mx_buffer(scales + (size_t)row0 * srow, (size_t)live * srow);
    int va[MT], vs[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) { va[mt] = (mt * 16 + c) * arow + 16 * q; vs[mt] = (mt * 16 + c) * srow; }

    f32x4 acc[MT][TN];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < TN; ++t) acc[mt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    uint4 w[4][TN], a[4][MT][NA], as[MT], an[MT];
    int ws[TN], wn[TN];
    const int last = min(TN, tiles - t0) - 1;              // (tiles behind the last read it again, and are not written)
    auto load_scales = [&](int g) {
#pragma unroll
        for (int t = 0; t < TN; ++t) wn[t] = __builtin_amdgcn_raw_buffer_load_b32(wb, lane * 4, (min(t, last) * groups + g) * MX_REC + 4096, 0);
        // (a row's scales of four steps; a step at a time they would be as many lines as the activations themselves)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) an[mt] = mx_load16(sb, vs[mt], g * 16);
    };
    auto load_step = [&](int g, int s) {
        const bool in = g * 4 + s < steps;                 // (the last record has steps behind K)
        const int k = in ? g * 4 + s : 0, oob = in ? 0 : MX_OOB;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int i = 0; i < NA; ++i) a[s][mt][i] = mx_load16(ab, va[mt] + oob, k * (64 * NA) + 64 * i);
        }
#pragma unroll
        for (int t = 0; t < TN; ++t) w[s][t] = mx_load16(wb, lane * 16 + oob, (min(t, last) * groups + g) * MX_REC + s * 1024);
    };
    auto step = [&](int s) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int ax = (int)((s == 0 ? as[mt].x : s == 1 ? as[mt].y : s == 2 ? as[mt].z : as[mt].w) >> (8 * q));
            uint4 lo[NA], hi[NA];
            if (FMT == SJD_MX8 && EXACT) {
#pragma unroll
                for (int i = 0; i < NA; ++i) {
                    const uint4 m = mx_large4(a[s][mt][i]);
                    lo[i] = mx_andn(a[s][mt][i], m); hi[i] = mx_and(a[s][mt][i], m);
                }
#pragma unroll
                for (int t = 0; t < TN; ++t) acc[mt][t] = mx_mfma<FMT>(w[s][t], lo[0], lo[NA - 1], acc[mt][t], ws[t] >> (8 * s), ax);
            } else {
#pragma unroll
                for (int i = 0; i < NA; ++i) hi[i] = a[s][mt][i];
            }
#pragma unroll
            for (int t = 0; t < TN; ++t) acc[mt][t] = mx_mfma<FMT>(w[s][t], hi[0], NA == 2 ? hi[NA - 1] : make_uint4(0, 0, 0, 0), acc[mt][t], ws[t] >> (8 * s), ax);
        }
    };
    int g = wave;
    if (g < groups) {
        load_scales(g);
#pragma unroll
        for (int s = 0; s < 4; ++s) load_step(g, s);
        for (; g + WK < groups; g += WK) {
#pragma unroll
            for (int t = 0; t < TN; ++t) ws[t] = wn[t];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) as[mt] = an[mt];
            load_scales(g + WK);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                step(s);
                __builtin_amdgcn_sched_barrier(0);
                load_step(g + WK, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int t = 0; t < TN; ++t) ws[t] = wn[t];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {                      // (behind K lie the next row's, which may be NaN's)
            as[mt] = an[mt];
            if (g * 4 + 1 >= steps) as[mt].y = 0;
            if (g * 4 + 2 >= steps) as[mt].z = 0;
            if (g * 4 + 3 >= steps) as[mt].w = 0;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) step(s);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < TN; ++t) red[wave][mt * TN + t][lane] = acc[mt][t];
    __syncthreads();
    for (int f = wave; f < F; f += WK) {
        const int mt = f / TN, t = f % TN, n = (t0 + t) * 16 + 4 * q;
        f32x4 x = red[0][f][lane];
#pragma unroll
        for (int i = 1; i < WK; ++i) x += red[i][f][lane];
        const int64_t row = row0 + mt * 16 + c;
        if (row < M && n < N) mx_store4(C + row * ldc + n, x, N - n, vec);
    }
}

// ---- many rows ------------------------------------------------------------------------------
// A workgroup makes BM rows x BN features.  Its waves share the activations of a step (BM x 128 codes and their scales) through LDS: requested
// AHEAD steps ahead, parked in the other of two buffers when a step's products are done, one barrier a step.  Weights go straight to registers,
// as far ahead, in the order in which they are packed.  The 16-byte pieces of a row of LDS change places by the row's number, so that eight
// lanes that read the same piece of eight rows meet all banks once.
template <int FMT, int WM, int WN, int MT, int NT, int AHEAD, typename T>
__global__ __launch_bounds__(64 * WM * WN, 2) void mx_tile_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                                  const uint8_t *__restrict__ packed, int M, int N, int Kp, int tiles, int groups,
                                                                  int per, T *__restrict__ C, int64_t ldc, int vec, float *__restrict__ part)
{
    constexpr int W = WM * WN, BM = WM * MT * 16, NA = FMT == SJD_MX8 ? 2 : 1, ROW = 64 * NA, PC = ROW / 16;
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int LOADS = BM * PC / (64 * W);                  // 16-byte loads to LDS a thread makes a step
    static_assert(BM * PC % (64 * W) == 0 && LOADS >= 1, "");
    __shared__ uint4 a_lds[2][BM * PC], s_lds[2][BM];          // s_lds: a row's scales of four steps
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
    const int wm = wave / WN, wn = wave % WN;
    // Workgroups go to the eight XCDs in turn.  An XCD gets neighbouring tasks, rows first: the workgroups that read the same weights, and
    // as many as it runs at a time read few more activations than one of them, from its own L2.
    const int mb = (int)(((int64_t)M + BM - 1) / BM), all = (int)gridDim.x, each = all / 8, more = all % 8, x = (int)blockIdx.x % 8;
    const int task = x * each + min(x, more) + (int)blockIdx.x / 8;
    const int64_t row0 = (int64_t)(task % mb) * BM;
    const int t0 = (task / mb * WN + wn) * NT, tb = min(t0, tiles - 1), last = min(NT, tiles - tb) - 1;
    const int arow = FMT == SJD_MX8 ? Kp : Kp / 2, srow = Kp / 32, steps = Kp / 128;
    const int k_beg = (int)blockIdx.z * per, k_end = min(steps, k_beg + per);          // (per is a multiple of 4)
    const auto wb = mx_buffer(packed + (size_t)tb * groups * MX_REC, (size_t)(last + 1) * groups * MX_REC);   // (tiles behind the last read it again)
    const int live = (int)min((int64_t)BM, M - row0);
    const auto ab = mx_buffer(codes + (size_t)row0 * arow, (size_t)live * arow), sb = mx_buffer(scales + (size_t)row0 * srow, (size_t)live * srow);

    // what this thread copies: piece p of row r goes to place p ^ f(r)
    int src[LOADS];
    constexpr int RS = 64 * W / PC;                            // rows between a thread's pieces, a multiple of 8
    const int r0 = (int)threadIdx.x / PC, pc = (int)threadIdx.x % PC, dst = r0 * PC + (PC == 8 ? pc ^ (r0 & 7) : pc ^ ((r0 >> 1) & 3));
#pragma unroll
    for (int i = 0; i < LOADS; ++i) src[i] = (r0 + i * RS) * arow + pc * 16;           // (rows behind the last: zeros)
    const int srow0 = (int)threadIdx.x % BM;                   // (threads too many for the rows copy some twice)
    uint4 ga[AHEAD][LOADS], w[AHEAD][NT], gs;
    int ws[NT], wn4[NT];
    auto fetch = [&](int k, int set) {
#pragma unroll
        for (int t = 0; t < NT; ++t) w[set][t] = mx_load16(wb, lane * 16, (min(t, last) * groups + (k >> 2)) * MX_REC + (k & 3) * 1024);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) ga[set][i] = mx_load16(ab, src[i], k * ROW);
    };
    auto fetch_scales = [&](int k) {                           // of the four steps from k on
#pragma unroll
        for (int t = 0; t < NT; ++t) wn4[t] = __builtin_amdgcn_raw_buffer_load_b32(wb, lane * 4, (min(t, last) * groups + (k >> 2)) * MX_REC + 4096, 0);
        gs = mx_load16(sb, srow0 * srow, k * 4);
    };
    auto park = [&](int st, int set) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) a_lds[st][dst + i * RS * PC] = ga[set][i];
    };
    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[mt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    // where this lane reads: row c of the wave's first tile, its one or two pieces; the other tiles lie 16 rows on
    const int at = (wm * MT * 16 + c) * PC, p0 = at + (PC == 8 ? q ^ (c & 7) : q ^ ((c >> 1) & 3)), p1 = at + (PC == 8 ? (4 + q) ^ (c & 7) : 0);
    // Step k = 4 g + s, whose set of registers is s % AHEAD; step k + AHEAD is fetched into it.  LDS reads run two row tiles ahead of the
    // products (left alone the compiler takes one register pair and waits for every read).
    auto step = [&](int k, auto s_) {
        constexpr int s = s_.value, set = s % AHEAD, nx = (s + 1) % AHEAD, st = s & 1;
        uint4 wc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) { wc[t] = w[set][t]; if (s == 0) ws[t] = wn4[t]; }
        __syncthreads();                                       // step k is parked, step k - 1 has been read
        if (s == 0) fetch_scales(min(k + 4, (k_end - 1) & ~3));
        fetch(min(k + AHEAD, k_end - 1), set);                 // (behind the end the last step again: no branch around loads)
        __builtin_amdgcn_sched_barrier(0);
        const uint4 *la = a_lds[st];
        const uint8_t *ls = reinterpret_cast<const uint8_t *>(s_lds[(k >> 2) & 1]) + (wm * MT * 16 + c) * 16 + s * 4 + q;
        uint4 ring[2][NA];
        int as[2];
        auto read = [&](int mt) {
            as[mt & 1] = ls[mt * 256];
            ring[mt & 1][0] = la[p0 + mt * 16 * PC];
            if (NA == 2) ring[mt & 1][NA - 1] = la[p1 + mt * 16 * PC];
        };
        read(0);
        if (MT > 1) read(1);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            __builtin_amdgcn_sched_barrier(0);
            const uint4 a0 = ring[mt & 1][0], a1 = NA == 2 ? ring[mt & 1][NA - 1] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[mt][t] = mx_step<FMT, EXACT>(wc[t], a0, a1, acc[mt][t], (int)((uint32_t)ws[t] >> (8 * s)), as[mt & 1]);
            if (mt + 2 < MT) { __builtin_amdgcn_sched_barrier(0); read(mt + 2); }
        }
        __builtin_amdgcn_sched_barrier(0);
        park(st ^ 1, nx);
        if (s == 0) s_lds[((k >> 2) & 1) ^ 1][srow0] = gs;      // (last read in the group before this one)
    };
    fetch_scales(k_beg);
    fetch(k_beg, 0);
    if (AHEAD == 2) fetch(min(k_beg + 1, k_end - 1), AHEAD - 1);
    park(0, 0);
    s_lds[(k_beg >> 2) & 1][srow0] = gs;
    int k = k_beg;
    for (; k + 4 <= k_end; k += 4) {
        step(k, std::integral_constant<int, 0>());
        step(k + 1, std::integral_constant<int, 1>());
        step(k + 2, std::integral_constant<int, 2>());
        step(k + 3, std::integral_constant<int, 3>());
    }
    if (k < k_end) step(k, std::integral_constant<int, 0>());
    if (k + 1 < k_end) step(k + 1, std::integral_constant<int, 1>());
    if (k + 2 < k_end) step(k + 2, std::integral_constant<int, 2>());
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int64_t row = row0 + (wm * MT + mt) * 16 + c;
        if (row >= M) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int n = (t0 + t) * 16 + 4 * q;
            if (n >= N) continue;
            if (gridDim.z > 1) mx_store4(part + ((size_t)blockIdx.z * M + row) * mx_up(N, 4) + n, acc[mt][t], 4, true);
            else mx_store4(C + row * ldc + n, acc[mt][t], N - n, vec);
        }
    }
}

// adds the K-slices in their order
template <typename T>
__global__ __launch_bounds__(256) void mx_join_kernel(const float *__restrict__ part, int slices, int M, int N, T *__restrict__ C, int64_t ldc, int vec)
{
    const int Np = mx_up(N, 4);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, total = (int64_t)M * (Np / 4);
    if (i >= total) return;
    const float4 *p = reinterpret_cast<const float4 *>(part) + i;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < slices; ++s) {
        const float4 v = p[s * total];
        x += (f32x4){v.x, v.y, v.z, v.w};
    }
    const int64_t row = i / (Np / 4);
    const int n = (int)(i - row * (Np / 4)) * 4;
    mx_store4(C + row * ldc + n, x, N - n, vec);
}

// ---- which kernel ---------------------------------------------------------------------------
// Whichever is estimated to be done first.  A launch takes as long as its weights from memory or as the CU with most workgroups: something
// fixed and so many steps (records) times what one costs, fitted to measured times with cold weights in us, bf16 results, activations in 8 bits
// (within 5 % for most of 53 shapes of 100 to 2048 rows, K from 1536 to 11008):
//  - tiles: where a CU has one workgroup, and where it has several (below);
//  - few rows: 0.6 + (records / 8) (1.5 + 0.6 TN) for 16 rows, several workgroups on a CU a seventh less; for 32 rows 2 + 0.4 a workgroup +
//    (records / 8) (2.6 + 0.95 TN).
// Slices of K add their sums' way through memory and a launch.  What this takes is 0.7 % slower than the best of all over those shapes, 12 %
// at most.  Results of fp32 issue every product of 8 bits twice and rows of 4 bits read half the LDS, which the plan does not know: it may miss
// their best kernel by more (2048 x 22016 x 4096: 339 us fp32, 141 to 160 us from 4 bits).  us, measured, the kernel chosen and the next best ones:
//   16 rows    22016 x 4096   rows 6 tiles 11.1   3 tiles 11.7, 1 tile 17.0           (weights alone 7.5)
//   100        4096 x 4096    rows 4 tiles 8.4    64 x 64 in 2 slices 12.2, 64 x 64 14.2
//   100        8192 x 1536    64 x 64 7.7         rows 4 tiles 9.0, 64 x 128 9.1
//   100        4096 x 11008   64 x 128 in 4 slices 16.9   rows 4 tiles 17.0, in 2 slices 22.8
//   200        4096 x 4096    64 x 64 14.0        64 x 128 in 2 slices 14.9, rows 4 tiles 15.5
//   256        12288 x 4096   64 x 192 20.8       64 x 128 24.7, 128 x 128 25.0
//   512        4096 x 4096    64 x 128 17.0       64 x 64 18.0, 128 x 128 23.6
//   1024       8192 x 1536    128 x 256 19.2      128 x 128 20.4, 64 x 192 20.6
//   2048       12288 x 4096   128 x 192 97.6      128 x 256 107, 128 x 128 112
//   2048       22016 x 4096   128 x 192 181       256 x 256 188, 128 x 128 190      (in turn, medians of 40; another day 180 and 177)
struct MxTile { int bm, bn; struct { double fixed, step; } one, several; };
static const MxTile mx_tiles[] = {{64, 64, {3.4, 0.33}, {3.4, 0.226}}, {64, 128, {4.7, 0.364}, {4.5, 0.307}}, {64, 192, {5.9, 0.41}, {5.7, 0.38}},
                                  {128, 128, {7.1, 0.517}, {7.9, 0.51}}, {128, 192, {8.4, 0.77}, {9.5, 0.633}}, {128, 256, {7.8, 0.864}, {13.9, 0.933}},
                                  {256, 256, {12.3, 1.46}, {1.7, 1.82}}};
#define MX_NO_KERNEL -2
struct MxPlan { int kind, tn, mt, slices, per, wgs; };      // kind: -1 few rows, MX_NO_KERNEL: no grid holds the product, else the tile
static MxPlan mx_plan(int M, int N, int K)
{
    const int steps = mx_up(K, 128) / 128, groups = mx_groups(K);
    const double tiles = std::ceil(N / 16.0), stream = (double)N * K * 0.53 / 5.5e6;          // us from memory
    MxPlan best = {MX_NO_KERNEL, 0, 0, 1, 0, 0};
    double cost = 1e30;
    auto take = [&](double t, const MxPlan &p) { if (t < cost) { cost = t; best = p; } };
    const int mt = M <= 16 ? 1 : 2;
    for (int tn : {1, 2, 3, 4, 6}) {
        if ((mt == 2 && tn == 6) || M > 32 * 65535) continue;          // (what a grid holds)
        const double wgs = std::ceil(tiles / tn) * std::ceil(M / (16.0 * mt)), n = std::ceil(wgs / 256);
        const double records = std::max(groups / 8.0, 0.4);
        const double t = mt == 1 ? n * (0.6 + records * (1.5 + 0.6 * tn)) * (n > 1 ? 0.85 : 1) : 2 + n * (0.4 + records * (2.6 + 0.95 * tn));
        // (where memory bounds both: the one with less beside it)
        take(std::max(t, stream) + 0.01 * t, {-1, tn, mt, 1, 0, 0});
    }
    if (M > 32)
        for (int k = 0; k < 7; ++k) {
            const MxTile &x = mx_tiles[k];
            const int64_t wgs = (int64_t)((M + (int64_t)x.bm - 1) / x.bm) * ((N + (int64_t)x.bn - 1) / x.bn);
            if (wgs > INT32_MAX) continue;
            for (int sl = 1; sl <= 4 && (sl == 1 || steps >= 8 * sl); sl *= 2) {
                const int per = mx_up((steps + sl - 1) / sl, 4), slices = (steps + per - 1) / per;
                const double n = std::ceil((double)wgs * slices / 256), t = n > 1 ? x.several.fixed + per * n * x.several.step : x.one.fixed + per * x.one.step;
                const double join = slices > 1 ? 1 + 1.6e-6 * M * N * slices : 0;
                take(std::max(t, stream) + 0.01 * t + join, {k, 0, 0, slices, per, (int)wgs});
            }
        }
    return best;
}

static int mx_product_args(int32_t format, const uint8_t *codes, const uint8_t *scales, const uint8_t *packed, int32_t M, int32_t N, int32_t K,
                           int32_t dtype, void *C, int64_t ldc)
{
    if (!codes || !scales || !packed || !C || M < 1 || N < 1 || K < 1 || K > SJD_MX_MAX_K || ldc < N) return SJD_EINVAL;
    if ((format != SJD_MX8 && format != SJD_MX4) || (dtype != 0 && dtype != 1)) return SJD_EINVAL;
    return mx_aligned(codes) && mx_aligned(scales) && mx_aligned(packed) ? SJD_OK : SJD_EINVAL;
}
static int64_t mx_quads(int N) { return ((int64_t)N + 3) / 4; }
static size_t mx_product_bytes(const MxPlan &p, int M, int N) { return p.slices > 1 ? (size_t)p.slices * M * mx_quads(N) * sizeof(float4) : 0; }

extern "C" int sjd_mx_product_workspace(int32_t M, int32_t N, int32_t K, size_t *bytes)
{
    if (!bytes || M < 1 || N < 1 || K < 1 || K > SJD_MX_MAX_K) return SJD_EINVAL;
    const MxPlan p = mx_plan(M, N, K);
    *bytes = mx_product_bytes(p, M, N);
    return p.kind == MX_NO_KERNEL ? SJD_EINVAL : SJD_OK;
}

// The sums of C on the kernel that `p` names; arguments are checked
static int mx_product_on(const MxPlan &p, int32_t format, const uint8_t *codes, const uint8_t *scales, const uint8_t *packed, int M, int N, int K,
                         int32_t dtype, void *C, int64_t ldc, void *workspace, void *stream)
{
    const int Kp = mx_up(K, 128), tiles = (int)(((int64_t)N + 15) / 16), groups = mx_groups(K);
    if (p.kind == MX_NO_KERNEL || !mx_fits(p.kind < 0 ? ((int64_t)tiles + p.tn - 1) / p.tn : p.wgs, 512)) return SJD_EINVAL;
    const int64_t joins = ((int64_t)M * mx_quads(N) + 255) / 256;
    if (p.slices > 1 && !mx_fits(joins, 256)) return SJD_EINVAL;
    const int vec = (uintptr_t)C % (dtype ? 8 : 16) == 0 && ldc % 4 == 0;
    hipStream_t s = (hipStream_t)stream;
    float *part = (float *)workspace;
#define ROWS(F, MT, TN, T) SJD_LAUNCH((mx_rows_kernel<F, MT, TN, T>), dim3((tiles + TN - 1) / TN, (M + 16 * MT - 1) / (16 * MT)), dim3(512), 0, s, codes, scales, packed, M, N, Kp, tiles, groups, (T *)C, ldc, vec)
#define TILE(F, WM, WN, MT, NT, A, T) SJD_LAUNCH((mx_tile_kernel<F, WM, WN, MT, NT, A, T>), dim3((unsigned)p.wgs, 1, p.slices), \
                                                 dim3(64 * WM * WN), 0, s, codes, scales, packed, M, N, Kp, tiles, groups, p.per, (T *)C, ldc, vec, part)
#define GO(F, T) do { \
        if (p.kind == 0) TILE(F, 1, 4, 4, 1, 2, T); \
        else if (p.kind == 1) TILE(F, 1, 4, 4, 2, 2, T); \
        else if (p.kind == 2) TILE(F, 1, 4, 4, 3, 2, T); \
        else if (p.kind == 3) TILE(F, 1, 4, 8, 2, 2, T); \
        else if (p.kind == 4) TILE(F, 1, 4, 8, 3, 1, T); \
        else if (p.kind == 5) TILE(F, 1, 8, 8, 2, 1, T); \
        else if (p.kind == 6) TILE(F, 2, 4, 8, 4, 1, T); \
        else if (p.mt == 1) { \
            if (p.tn == 1) ROWS(F, 1, 1, T); else if (p.tn == 2) ROWS(F, 1, 2, T); else if (p.tn == 3) ROWS(F, 1, 3, T); else if (p.tn == 4) ROWS(F, 1, 4, T); else ROWS(F, 1, 6, T); \
        } else { \
            if (p.tn == 1) ROWS(F, 2, 1, T); else if (p.tn == 2) ROWS(F, 2, 2, T); else if (p.tn == 3) ROWS(F, 2, 3, T); else ROWS(F, 2, 4, T); \
        } } while (0)
    if (format == SJD_MX8) { if (dtype == 0) GO(SJD_MX8, float); else GO(SJD_MX8, bf16_t); }
    else { if (dtype == 0) GO(SJD_MX4, float); else GO(SJD_MX4, bf16_t); }
#undef GO
#undef TILE
#undef ROWS
    HIP_TRY(hipGetLastError());
    if (p.slices > 1) {
        const dim3 grid((unsigned)joins);
        if (dtype == 0) SJD_LAUNCH((mx_join_kernel<float>), grid, dim3(256), 0, s, (const float *)part, p.slices, M, N, (float *)C, ldc, vec);
        else SJD_LAUNCH((mx_join_kernel<bf16_t>), grid, dim3(256), 0, s, (const float *)part, p.slices, M, N, (bf16_t *)C, ldc, vec);
        HIP_TRY(hipGetLastError());
    }
    return SJD_OK;
}

extern "C" int sjd_mx_product(int32_t format, const uint8_t *codes, const uint8_t *scales, const uint8_t *packed, int32_t M, int32_t N,
                              int32_t K, int32_t dtype, void *C, int64_t ldc, void *workspace, size_t workspace_bytes, void *stream)
{
    SJD_TRY(mx_product_args(format, codes, scales, packed, M, N, K, dtype, C, ldc));
    const MxPlan p = mx_plan(M, N, K);
    const size_t need = mx_product_bytes(p, M, N);
    if (need && (!workspace || workspace_bytes < need || !mx_aligned(workspace))) return SJD_EINVAL;
    return mx_product_on(p, format, codes, scales, packed, M, N, K, dtype, C, ldc, workspace, stream);
}

extern "C" int sjd_mx_product_plan(int32_t M, int32_t N, int32_t K, int32_t *rows, int32_t *cols, int32_t *slices)
{
    if (!rows || !cols || !slices || M < 1 || N < 1 || K < 1 || K > SJD_MX_MAX_K) return SJD_EINVAL;
    const MxPlan p = mx_plan(M, N, K);
    if (p.kind == MX_NO_KERNEL) return SJD_EINVAL;
    *rows = p.kind < 0 ? 16 * p.mt : mx_tiles[p.kind].bm;
    *cols = p.kind < 0 ? 16 * p.tn : mx_tiles[p.kind].bn;
    *slices = p.slices;
    return SJD_OK;
}

extern "C" int sjd_mx_product_test(int32_t rows, int32_t cols, int32_t slices, int32_t format, const uint8_t *codes, const uint8_t *scales,
                                   const uint8_t *packed, int32_t M, int32_t N, int32_t K, int32_t dtype, void *C, int64_t ldc, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    SJD_TRY(mx_product_args(format, codes, scales, packed, M, N, K, dtype, C, ldc));
    MxPlan p = {MX_NO_KERNEL, 0, 0, 1, 0, 0};
    if (rows <= 32) {
        const int tn = cols / 16;
        if ((rows != 16 && rows != 32) || cols != 16 * tn || tn < 1 || tn > (rows == 16 ? 6 : 4) || tn == 5 || slices != 1 || M > 32 * 65535) return SJD_EINVAL;
        if ((rows == 16) != (M <= 16)) return SJD_EINVAL;      // (as the plan has it)
        p = {-1, tn, rows / 16, 1, 0, 0};
    }
    for (int k = 0; k < 7; ++k) {
        if (mx_tiles[k].bm != rows || mx_tiles[k].bn != cols || M <= 32 || (slices != 1 && slices != 2 && slices != 4)) continue;
        const int64_t wgs = (((int64_t)M + rows - 1) / rows) * (((int64_t)N + cols - 1) / cols);
        if (wgs > INT32_MAX) return SJD_EINVAL;
        const int steps = mx_up(K, 128) / 128, per = mx_up((steps + slices - 1) / slices, 4);
        p = {k, 0, 0, (steps + per - 1) / per, per, (int)wgs};
    }
    if (p.kind == MX_NO_KERNEL) return SJD_EINVAL;
    const size_t need = mx_product_bytes(p, M, N);
    if (need && (!workspace || workspace_bytes < need || !mx_aligned(workspace))) return SJD_EINVAL;
    return mx_product_on(p, format, codes, scales, packed, M, N, K, dtype, C, ldc, workspace, stream);
}
