// A cache of keys and values in 8 bits (E4M3) with a power-of-two scale per block of 32 positions and head: appending a window, and the
// window's attention over it.
//
// A block's record holds keys and values as v_mfma_f32_16x16x32_f16 takes them, two operands (8 codes each) to the 16 bytes of a lane,
// so a wave reads a record as contiguous KiB loads.  Codes become fp16 exactly; scales stay outside the products.
#include "sjd_mx.h"

#include <algorithm>

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

#define KV8_MAX_SEQS 32767
#define KV8_MAX_HEADS 65535

static bool kv8_sizes(int n_seqs, int L, int n_kv, int hd, int cap)
{
    if (n_seqs < 1 || n_seqs > KV8_MAX_SEQS || L < 1 || n_kv < 1 || n_kv > KV8_MAX_HEADS || cap < 1 || cap > INT32_MAX - 64 || L > cap) return false;
    return hd == 32 || hd == 64 || hd == 96 || hd == 128 || hd == 256;
}

// ---- append ---------------------------------------------------------------------------------
// A workgroup makes the keys (or the values) of one block: new rows and the codes that the block holds already meet in LDS as fp32,
// their largest magnitude gives the scale, and a thread then makes 16 bytes of the record.
// Windows of 16 for 8 sequences, 32 heads of 128, fp32: 5.9 us, three waits for memory one after the other (the length, the rows and codes, the
// stores' end) and the launch; 2000 bf16 rows of a prompt 11.4 us, 49 MB at 4.3 TB/s against a copy's 4.9.
template <int HD, int WHICH, typename T>
__device__ __forceinline__ void kv8_append_block(const T *__restrict__ src, int64_t ld, int held, int rows, int vec, uint8_t *__restrict__ rec,
                                                 uint8_t *__restrict__ scale, float *tile, uint32_t *top)
{
    constexpr int PITCH = HD + 4, KS = HD / 32, UNITS = HD / 8, W = 4 * (int)sizeof(T) / 8;      // W: uint4 in eight values, 1 or 2
    const int tid = threadIdx.x, lane = tid & 63, pair = __builtin_amdgcn_readfirstlane(tid >> 6);
    // code group of this thread: two operands of eight codes (2 HD threads)
    auto place = [&](int half, int e, int &p, int &d) {
        const int o = pair * 2 + half;
        if (WHICH) { d = o * 16 + (lane & 15); p = (e >> 2) * 16 + (lane >> 4) * 4 + (e & 3); }
        else { p = o / KS * 16 + (lane & 15); d = o % KS * 32 + (lane >> 4) * 8 + e; }
    };
    // everything is requested before anything is used: eight values of two rows of the block (zeros where they are not new), and the codes held
    uint4 raw[2][W], old;
    if (vec) {
        const auto from = mx_buffer((const uint8_t *)(src + held * ld), MX_OOB - 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = tid + i * 2 * HD, r = u / UNITS, c = u % UNITS * 8;
            const bool in = r >= held && r < rows;
#pragma unroll
            for (int w = 0; w < W; ++w) raw[i][w] = mx_load16(from, in ? ((r - held) * (int)ld + c) * (int)sizeof(T) + w * 16 : MX_OOB, 0);
        }
    }
    old = mx_load16(mx_buffer(rec, 32 * HD), held ? tid * 16 : MX_OOB, 0);
    const int was = held ? *scale : 0;
    __builtin_amdgcn_sched_barrier(0);
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int u = tid + i * 2 * HD, r = u / UNITS, c = u % UNITS * 8;
        float x[8];
        if (vec) mx_load8<T>(reinterpret_cast<const T *>(raw[i]), 0, 8, true, x);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
            if (r >= held && r < rows) mx_load8<T>(src + r * ld, c, HD, false, x);
        }
        if (r < held) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max(amax, mx_finite_bits(x[e]));
        float4 *dst = reinterpret_cast<float4 *>(tile + r * PITCH + c);
        dst[0] = make_float4(x[0], x[1], x[2], x[3]); dst[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
    if (held) {
        const float s = mx_pow2(was);
        // Code 256 with the largest scale, what values from 248 * 2^120 on were rounded to, is 2^128: the largest float below gives the same
        // scale and the same code again.
        const bool over = __builtin_amdgcn_readfirstlane(was) >= 247;
        const uint32_t w[4] = {old.x, old.y, old.z, old.w};
        float y[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
            y[4 * i] = lo.x * s; y[4 * i + 1] = lo.y * s; y[4 * i + 2] = hi.x * s; y[4 * i + 3] = hi.y * s;
        }
        if (over) {
#pragma unroll
            for (int e = 0; e < 16; ++e) if (isinf(y[e])) y[e] = copysignf(3.4028234664e38f, y[e]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            int p, d;
            place(e >> 3, e & 7, p, d);
            if (p < held) { tile[p * PITCH + d] = y[e]; amax = max(amax, mx_finite_bits(y[e])); }
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o));
    if (lane == 0) top[pair] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < HD / 32; ++w) amax = max(amax, top[w]);
    const int byte = mx_scale_byte<SJD_MX8>(amax);
    const float inv = mx_pow2(254 - byte);
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            int p, d;
            place(i >> 1, (i & 1) * 4 + j, p, d);
            y[j] = tile[p * PITCH + d];
        }
        out[i] = mx_e4m3x4(y[0], y[1], y[2], y[3], inv);
    }
    reinterpret_cast<uint4 *>(rec)[tid] = make_uint4(out[0], out[1], out[2], out[3]);
    if (tid == 0) *scale = (uint8_t)byte;
}
template <int HD, typename T>
__global__ __launch_bounds__(2 * HD) void kv8_append_kernel(const T *__restrict__ k, const T *__restrict__ v, int64_t ld,
                                                            const int32_t *__restrict__ len, int L, int cap, int nblk, int vec,
                                                            uint8_t *__restrict__ cache, uint8_t *__restrict__ scales)
{
    __shared__ __attribute__((aligned(16))) float tile[32 * (HD + 4)];
    __shared__ uint32_t top[HD / 32];
    const int which = blockIdx.z & 1, b = blockIdx.z >> 1, head = blockIdx.y;
    const int n = len[b];
    if (n < 0 || n > cap - L) return;
    const int blk = (n >> 5) + (int)blockIdx.x, p0 = blk * 32;
    if (p0 >= n + L) return;
    const int held = max(n - p0, 0), rows = n + L - p0;          // rows [held, rows) of the block are new
    const size_t at = ((size_t)b * gridDim.y + head) * nblk + blk;
    uint8_t *rec = cache + at * 64 * HD, *scale = scales + at * 2;
    const int64_t row = ((int64_t)b * L + (p0 - n)) * ld + (int64_t)head * HD;
    if (which) kv8_append_block<HD, 1, T>(v + row, ld, held, rows, vec, rec + 32 * HD, scale + 1, tile, top);
    else kv8_append_block<HD, 0, T>(k + row, ld, held, rows, vec, rec, scale, tile, top);
}

extern "C" int sjd_kv8_append(int32_t dtype, const void *k, const void *v, int64_t ld, const int32_t *len, int32_t n_seqs, int32_t L,
                              int32_t n_kv_heads, int32_t head_dim, int32_t cap, uint8_t *cache, uint8_t *scales, void *stream)
{
    if (!k || !v || !len || !cache || !scales || (dtype != 0 && dtype != 1)) return SJD_EINVAL;
    if (!kv8_sizes(n_seqs, L, n_kv_heads, head_dim, cap) || ld < (int64_t)n_kv_heads * head_dim || !mx_aligned(cache) || !mx_aligned(scales)) return SJD_EINVAL;
    const int64_t blocks = ((int64_t)L + 31) / 32 + 1;
    if (!mx_fits(blocks, 2 * head_dim)) return SJD_EINVAL;
    const dim3 grid((unsigned)blocks, n_kv_heads, n_seqs * 2);
    // (loads of 16 bytes: rows aligned, and a block's within 32-bit offsets)
    const int vec = mx_vec(k, ld, dtype) && mx_vec(v, ld, dtype) && ld <= MX_OOB / 256, nblk = (cap + 31) / 32;
    hipStream_t s = (hipStream_t)stream;
#define GO1(HD, T) SJD_LAUNCH((kv8_append_kernel<HD, T>), grid, dim3(2 * HD), 0, s, (const T *)k, (const T *)v, ld, len, L, cap, nblk, vec, cache, scales)
#define GO(HD) do { if (dtype == 0) GO1(HD, float); else GO1(HD, bf16_t); } while (0)
    switch (head_dim) {
        case 32: GO(32); break;
        case 64: GO(64); break;
        case 96: GO(96); break;
        case 128: GO(128); break;
        default: GO(256); break;
    }
#undef GO
#undef GO1
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}

// ---- attention ------------------------------------------------------------------------------
#define KV8_WAVES 8
#define KV8_ROWS 16
// Where every walk has up to this many blocks none is split, four blocks a wave, and nothing is joined.  Cut and joined against whole: 9.6 us
// against 6.6 (300 positions, one query, 32 heads), 10.1 against 8.4 (583, 16 queries); longer walks gain from the cut.
#define KV8_SHORT 32
#define KV8_SKEW 256     // blocks of a cache whose walks may differ by more than a second launch costs
#define KV8_LIFT 12.f    // a row's reference is its largest score less this: weights up to 2^KV8_TOP in fp16, 22 bits of hi + lo hold from
#define KV8_TOP 15.f     // 2^-14 on, and 2^-37 of the largest below
#define KV8_O_LIFT 14.f  // weights times value scales, where those differ: 22 bits hold from 2^-27 of the largest on
#define KV8_NONE -3.4028234664e38f        // reference of a row that has seen nothing: finite, so that differences need no cases
#define KV8_FAR 1048576.f        // references from here on: fp32 has 1/8 between scores

// The queries of one sequence that read one cache head, L * (heads per cache head) rows with a query's heads next to each other, are cut
// into groups of 16 rows.  A (sequence, group) pair walks the blocks that any of its queries sees, the sinks' first.  Where the pairs are too
// few for the chip their walks are cut into splits, all of about the same number of blocks: lengths live on the device, so the kernels work
// the cut out themselves, every workgroup the same.
// More rows to a workgroup read less from L2, but leave fewer waves on a CU.  Two tiles of rows a wave: 35.4 us against 38.8 at 32 queries x 4 heads a
// cache head and 16 k positions, where a head's records are read 8 times (15 TB/s), but 28.5 against 22.5 at 4 x 8 queries, 40.6 against 34.9 for
// a prompt of 1000; four to eight tiles over codes made fp16 once in LDS, 50 to 58 for the first.
struct Kv8Plan {
    const int32_t *len;
    int32_t n_seqs, L, group, qgroups;     // heads per cache head; row groups of KV8_ROWS rows per sequence
    int32_t group_shift, qgroups_shift;    // their logarithms, or -1 where they are no powers of two
    int32_t window, sinks, cap, nblk;
    int32_t slots, least;                      // splits to aim for per cache head, of so many blocks at least; 0: one per pair, none cut
};
__device__ __forceinline__ int kv8_div(int x, int d, int shift) { return shift >= 0 ? x >> shift : x / d; }     // (a division is 20 instructions in a row)
__device__ __forceinline__ int kv8_query(const Kv8Plan &pl, int row) { return kv8_div(row, pl.group, pl.group_shift); }
__device__ __forceinline__ int kv8_seq(const Kv8Plan &pl, int pair) { return kv8_div(pair, pl.qgroups, pl.qgroups_shift); }
struct Kv8Span { int32_t i0, i1, n, first, front, count; };    // queries, cached positions; block v is v < front ? v : first + v - front
__device__ __forceinline__ Kv8Span kv8_span(const Kv8Plan &pl, int pair)
{
    Kv8Span s;
    const int b = kv8_seq(pl, pair), r0 = (pair - b * pl.qgroups) * KV8_ROWS;
    s.n = pl.len[b];
    s.i0 = kv8_query(pl, r0);
    s.i1 = kv8_query(pl, min(r0 + KV8_ROWS - 1, pl.L * pl.group - 1));
    s.first = s.front = s.count = 0;
    if (s.n < 0 || s.n > pl.cap - pl.L) return s;
    const int last = s.n + s.i1;
    if (pl.window) {
        s.first = max(0, s.n + s.i0 - pl.window + 1) >> 5;
        s.front = min((min(pl.sinks, last + 1) + 31) >> 5, s.first);
    }
    s.count = s.front + (last >> 5) - s.first + 1;
    return s;
}
struct Kv8Part { int32_t pair, split, splits, per, base; };     // a slot's pair, its place among the pair's splits, blocks per split
// Lanes look at 64 pairs at a time; by_pair: the part that starts the given pair, else the part of the given slot.  With `per` blocks
// a split, per >= total / slots up to the rounding of fp32, the splits of all pairs are at most total / per + pairs (1 - 1 / per): never more
// than slots + pairs.
__device__ __forceinline__ bool kv8_part(const Kv8Plan &pl, int want, bool by_pair, Kv8Part &part)
{
    const int pairs = pl.n_seqs * pl.qgroups, lane = threadIdx.x & 63;
    const int c0 = lane < pairs ? kv8_span(pl, lane).count : 0;
    float total = 0.f;
    uint64_t cut = 0;                                                          // any walk long enough
    for (int p0 = 0; p0 < pairs; p0 += 64) {
        const int n = p0 == 0 ? c0 : p0 + lane < pairs ? kv8_span(pl, p0 + lane).count : 0;
        float c = (float)n;
        cut |= __ballot(n > KV8_SHORT);
        for (int o = 1; o < min(pairs, 64); o <<= 1) c += __shfl_xor(c, o);
        total += __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(c)));
    }
    part.per = cut ? max(pl.least, (int)ceilf(total / (float)pl.slots)) : KV8_SHORT;
    int base = 0;
    for (int p0 = 0; p0 < pairs; p0 += 64) {
        const int c = p0 == 0 ? c0 : p0 + lane < pairs ? kv8_span(pl, p0 + lane).count : 0;
        const int mine = (c + part.per - 1) / part.per;
        int incl = mine;
        for (int o = 1; o < min(pairs, 64); o <<= 1) { const int up = __shfl_up(incl, o); if (lane >= o) incl += up; }
        const int start = base + incl - mine;
        const uint64_t hit = by_pair ? __ballot(p0 + lane == want) : __ballot(want >= start && want < start + mine);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            part.pair = p0 + l;
            part.splits = __builtin_amdgcn_readlane(mine, l);
            part.base = __builtin_amdgcn_readlane(start, l);
            part.split = by_pair ? 0 : want - part.base;
            return true;
        }
        base += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

__device__ __forceinline__ f16x8 kv8_f16(uint32_t lo, uint32_t hi, float scale = 1.f)        // eight codes, times a power of two
{
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
    return (f16x8){a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// bytes 0x80 where a code is NaN (0x7F with any sign)
__device__ __forceinline__ uint32_t kv8_nan(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
// the largest over the four lanes of a column (l % 16)
__device__ __forceinline__ float kv8_across(float x)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float kv8_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// reference for a largest score: far ones have no room for the lift (it would be rounded to more than fp16 holds)
__device__ __forceinline__ float kv8_ref(float top) { return top - (fabsf(top) < KV8_FAR ? KV8_LIFT : 0.f); }
// log2 of a score's weight, s cs - m.  Far references are roundings of a product, and s cs itself may be many powers of two beside it: the
// product is rounded likewise before it is compared.
__device__ __forceinline__ float kv8_log(float s, float cs, float m)
{
    float p = s * cs;
    asm("" : "+v"(p));                             // (no fused multiply-add)
    return fabsf(m) >= KV8_FAR ? p - m : fmaf(s, cs, -m);
}

// 2^d as two factors: the exponential has no subnormal results, the product with the second one has.  The first stays normal when it is
// divided by a sum of weights (up to 2^15 for each of 2^31 positions).
__device__ __forceinline__ void kv8_scale(float d, float &big, float &small)
{
    const float b = fmaxf(d, -60.f);
    big = kv8_exp2(b); small = kv8_exp2(d - b);
}

// record of a split: O[KV8_ROWS][HD], then m, d and l of the rows; rows behind the last are not written
__host__ __device__ __forceinline__ size_t kv8_record(int hd) { return (size_t)KV8_ROWS * (hd + 3); }

__device__ __forceinline__ void kv8_out(float *p, const f32x4 &v, bool vec)
{
    if (vec) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else { p[0] = v[0]; p[1] = v[1]; p[2] = v[2]; p[3] = v[3]; }
}
__device__ __forceinline__ void kv8_out(bf16_t *p, const f32x4 &v, bool vec)
{
    if (vec) *reinterpret_cast<uint2 *>(p) = make_uint2(f32_to_bf16(v[0]) | (uint32_t)f32_to_bf16(v[1]) << 16,
                                                        f32_to_bf16(v[2]) | (uint32_t)f32_to_bf16(v[3]) << 16);
    else { p[0] = f32_to_bf16(v[0]); p[1] = f32_to_bf16(v[1]); p[2] = f32_to_bf16(v[2]); p[3] = f32_to_bf16(v[3]); }
}

// Per block of 32 positions, with the scales 2^ek and 2^ev of its keys and values:
//   S^T[key][row] = K codes . Q (Q scaled per row to 2^13 .. 2^14, hi + lo fp16)        s = S * 2^ek * 2^eq * log2(e) / sqrt(HD)
//   l = sum 2^(s - m),   O = sum 2^(s + ev - m - d) * V codes,   out = O * 2^d / l
// with a reference m that may be any number near the largest s, and a whole number d: O has one of its own because the blocks' scales differ, so
// that fp16 holds its largest contributions whatever the scales are.  d is relative to m, so that neither loses bits to the other.
// Most walks need less.  While the value scales are within a few powers of two of the wave's first one, the codes take the difference when they
// become fp16 (exactly: 2^-9 2^-5 .. 448 2^6), d is that first scale, and m stays until a score is 2^KV8_TOP above it: what is left of a block
// beside its conversions (64 codes a lane) is 8 exponentials, their sum and a comparison.  Against references that follow every block: 38.7 us
// against 43.8 (32 queries x 4 heads a cache head, 16 k positions), 15.2 against 16.3 (8 x 16 queries of 32 heads), 19.9 against 22.2
// (128 queries, 4 k positions); no difference where memory bounds, one query.
// The two score tiles of a block leave lane (g, c) with row c and the positions 16 h + 4 g + i: the order in which V's operands hold them.
template <int HD, typename T>
__global__ __launch_bounds__(64 * KV8_WAVES, HD <= 128 ? 4 : 2) void kv8_attention_kernel(const T *__restrict__ q, int64_t ldq, const uint8_t *__restrict__ cache,
                                                                          const uint8_t *__restrict__ scales, Kv8Plan pl, T *__restrict__ out,
                                                                          int64_t ldo, int vec, float *__restrict__ part)
{
    constexpr int KS = HD / 32, DT = HD / 16, RG = KV8_ROWS, PL = sizeof(T) == 4 ? 2 : 1, CH = DT < 8 ? DT : 8;
    __shared__ f16x8 q_lds[KS][PL][64];
    __shared__ float q_scale[RG];
    __shared__ float m_all[KV8_WAVES][RG], d_all[KV8_WAVES][RG], l_all[KV8_WAVES][RG];
    __shared__ f32x4 o_slot[KV8_WAVES][CH][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const int head = blockIdx.x, heads = gridDim.x;
    Kv8Part pt = {(int)blockIdx.y, 0, 1, 0, 0};
    if (pl.slots && !kv8_part(pl, (int)blockIdx.y, false, pt)) return;
    const Kv8Span sp = kv8_span(pl, pt.pair);
    if (!sp.count) return;
    const int per = pl.slots ? pt.per : sp.count;
    const int v_beg = pt.split * per, v_end = min(sp.count, v_beg + per);
    const int b = kv8_seq(pl, pt.pair), r0 = (pt.pair - b * pl.qgroups) * RG, rows = pl.L * pl.group;

    // The next block's keys are requested when this block's have left their registers, its values likewise.
    const size_t at0 = ((size_t)b * heads + head) * pl.nblk;
    uint4 ka[KS], va[KS];
    int sc = 0;
    auto place = [&](int v) { return v < sp.front ? v : sp.first + v - sp.front; };
    auto fetch_k = [&](int v) {                                    // (behind the end: nothing is read)
        const int blk = place(min(v, v_end - 1));
        const auto rec = mx_buffer(cache + (at0 + blk) * (64 * HD), v < v_end ? 64 * HD : 0);      // (a descriptor in scalars: one register of lane offsets)
#pragma unroll
        for (int p = 0; p < KS; ++p) ka[p] = mx_load16(rec, lane * 16 + p * 1024, 0);
        sc = *reinterpret_cast<const uint16_t *>(scales + (at0 + blk) * 2);
    };
    auto fetch_v = [&](int v) {
        const auto rec = mx_buffer(cache + (at0 + place(min(v, v_end - 1))) * (64 * HD), v < v_end ? 64 * HD : 0);
#pragma unroll
        for (int p = 0; p < KS; ++p) va[p] = mx_load16(rec, lane * 16 + (KS + p) * 1024, 0);
    };
    int v = v_beg + wave;
    // Q by wave 0: lane (g, c) has values 32 ks + 8 g .. of row c.  Requested first: loads return in order.
    float x[KS][8];
    if (wave == 0) {
        const int r = min(r0 + c, rows - 1);
        const int i = kv8_query(pl, r);
        const T *src = q + ((size_t)b * pl.L + i) * ldq + ((size_t)head * pl.group + (r - i * pl.group)) * HD;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) mx_load8<T>(src, ks * 32 + g * 8, HD, vec & 1, x[ks]);
    }
    __builtin_amdgcn_sched_barrier(0);
    fetch_k(v);
    fetch_v(v);
    __builtin_amdgcn_sched_barrier(0);

    if (wave == 0) {
        uint32_t top = 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, mx_finite_bits(x[ks][e]));
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int up = min(max(127 + 13 - (int)(top >> 23), -126), 127);        // 2^up * the largest is in 2^13 .. 2^14
        const float mul = mx_pow2(127 + up);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            f16x8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = x[ks][e] * mul;              // (exact)
                hi[e] = (_Float16)y;
                lo[e] = (_Float16)(y - (float)hi[e]);
            }
            q_lds[ks][0][lane] = hi;
            if (PL == 2) q_lds[ks][PL - 1][lane] = lo;
        }
        if (g == 0) q_scale[c] = mx_pow2(127 - up) * (1.4426950408889634f / sqrtf((float)HD));
    }
    __syncthreads();

    f32x4 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = KV8_NONE, d, l = 0.f;
    const float qs = q_scale[c];
    const int pos = sp.n + kv8_query(pl, min(r0 + c, rows - 1));
    // S = K codes . Q, then the next block's keys are requested; whole: no row's mask hides anything of the block
    f32x4 s[2];
    int k0 = 0, sb = 0;
    bool whole = true;
    auto scores = [&]() {
        k0 = place(v) * 32;
        whole = k0 + 31 <= sp.n + sp.i0 && (!pl.window || k0 > sp.n + sp.i1 - pl.window || k0 + 31 < pl.sinks);
        s[0] = s[1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int op = 0; op < 2 * KS; ++op) {
            const f16x8 k = (op & 1) ? kv8_f16(ka[op / 2].z, ka[op / 2].w) : kv8_f16(ka[op / 2].x, ka[op / 2].y);
#pragma unroll
            for (int p = PL - 1; p >= 0; --p) s[op / KS] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q_lds[op % KS][p][lane], s[op / KS], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        fetch_k(v + KV8_WAVES);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto sees = [&](int e) {
        const int key = k0 + (e >> 2) * 16 + g * 4 + (e & 3);
        return (key <= pos) & ((pl.window == 0) | (key > pos - pl.window) | (key < pl.sinks));
    };
    // O += V codes times `scale` . P, then the next block's values are requested
    auto weigh = [&](const f16x8 &ph, const f16x8 &plo, uint32_t seen, float scale) {
        if (!whole) {
            // Zero times NaN is NaN: where a mask may hide a NaN code from some row, the codes are taken out, and the rows that see one
            // get it by counting.
            uint32_t any = 0;
#pragma unroll
            for (int p = 0; p < KS; ++p) any |= kv8_nan(va[p].x) | kv8_nan(va[p].y) | kv8_nan(va[p].z) | kv8_nan(va[p].w);
            if (__ballot(any != 0)) {
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    uint32_t &w0 = (t & 1) ? va[t / 2].z : va[t / 2].x, &w1 = (t & 1) ? va[t / 2].w : va[t / 2].y;
                    const uint32_t n0 = kv8_nan(w0) >> 7, n1 = kv8_nan(w1) >> 7;        // 1 in the byte of a NaN
                    f16x8 ind, vis;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        ind[e] = (_Float16)(float)(((e < 4 ? n0 : n1) >> (8 * (e & 3))) & 1u);
                        vis[e] = (_Float16)(float)(seen >> e & 1u);
                    }
                    f32x4 hits = {0.f, 0.f, 0.f, 0.f};
                    hits = __builtin_amdgcn_mfma_f32_16x16x32_f16(ind, vis, hits, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (hits[i] != 0.f) o[t][i] = NAN;
                    w0 &= ~(n0 * 0xFFu); w1 &= ~(n1 * 0xFFu);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const f16x8 vv = (t & 1) ? kv8_f16(va[t / 2].z, va[t / 2].w, scale) : kv8_f16(va[t / 2].x, va[t / 2].y, scale);
            if (PL == 2) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, plo, o[t], 0, 0, 0);
            o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, ph, o[t], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        fetch_v(v + KV8_WAVES);
    };
    // ---- value scales near the first one ----
    sb = __builtin_amdgcn_readfirstlane(sc);
    const int base = sb >> 8;
    bool far = true;                             // any row of the wave has a far reference, or none yet
    for (; v < v_end; v += KV8_WAVES) {
        sb = __builtin_amdgcn_readfirstlane(sc);
        const int up = (sb >> 8) - base;
        if (up < -5 || up > 6) break;
        scores();
        const float cs = qs * mx_pow2(sb & 255);
        float bm;
        uint32_t seen = 0xFFu;
        if (whole) {
            bm = s[0][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) bm = fmaxf(bm, s[e >> 2][e & 3]);
            bm *= cs;
        } else {
            bm = -INFINITY;
            seen = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool see = sees(e);
                seen |= see ? 1u << e : 0u;
                bm = fmaxf(bm, see ? s[e >> 2][e & 3] * cs : -INFINITY);
            }
        }
        if (__ballot(bm - m > KV8_TOP)) {
            const float mn = fmaxf(m, kv8_ref(kv8_across(bm))), turn = kv8_exp2(m - mn);
            l *= turn;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= turn;
            m = mn;
            far = __ballot(fabsf(m) >= KV8_FAR) != 0;
        }
        float x[8];
        if (whole && !far) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = kv8_exp2(fmaf(s[e >> 2][e & 3], cs, -m));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = seen >> e & 1 ? kv8_exp2(kv8_log(s[e >> 2][e & 3], cs, m)) : 0.f;
        }
        f16x8 ph, plo = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            l += x[e];
            ph[e] = (_Float16)x[e];
            if (PL == 2) plo[e] = (_Float16)(x[e] - (float)ph[e]);
        }
        weigh(ph, plo, seen, mx_pow2(127 + up));
    }
    d = (float)(base - 127);
    // ---- the rest of a walk whose value scales differ by more ----
    for (; v < v_end; v += KV8_WAVES) {
        sb = __builtin_amdgcn_readfirstlane(sc);
        scores();
        const float cs = qs * mx_pow2(sb & 255), ev = (float)((sb >> 8) - 127);
        float bm = -INFINITY;
        uint32_t seen = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool see = whole || sees(e);
            seen |= see ? 1u << e : 0u;
            bm = fmaxf(bm, see ? s[e >> 2][e & 3] * cs : -INFINITY);
        }
        bm = kv8_across(bm);
        const float mn = fmaxf(m, kv8_ref(bm));
        const float down = m - mn, dn = rintf(fmaxf(d + down, bm - mn + ev - KV8_O_LIFT));
        const float so = kv8_exp2(down), turn = kv8_exp2(down + (d - dn));      // what the sums so far are rescaled by
        const float f = kv8_exp2(fminf(ev - dn, 120.f));
        float sum = 0.f;
        f16x8 ph, plo = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = seen >> e & 1 ? kv8_exp2(kv8_log(s[e >> 2][e & 3], cs, mn)) : 0.f;
            sum += x;
            float pf = x * f;
            if (PL == 2) asm("" : "+v"(pf));     // (the product in fp32 for both parts: fused into the conversion to fp16 it rounds otherwise now and then)
            ph[e] = (_Float16)pf;
            if (PL == 2) plo[e] = (_Float16)(pf - (float)ph[e]);
        }
        l = l * so + sum;
        m = mn; d = dn;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] *= turn;
        weigh(ph, plo, seen, 1.f);
    }

    // ---- the waves of a workgroup, in wave order ----
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) { m_all[wave][c] = m; d_all[wave][c] = d; l_all[wave][c] = l; }
    __syncthreads();
    float *dst = part + ((size_t)head * gridDim.y + blockIdx.y) * kv8_record(HD);
    float M = KV8_NONE, D = -INFINITY, den = 0.f;
#pragma unroll
    for (int w = 0; w < KV8_WAVES; ++w) M = fmaxf(M, m_all[w][c]);
#pragma unroll
    for (int w = 0; w < KV8_WAVES; ++w) {
        const float down = m_all[w][c] - M;
        den += kv8_exp2(down) * l_all[w][c];                             // (sums of nothing are zero, or NaN)
        D = fmaxf(D, d_all[w][c] + down);
    }
    D = rintf(D);
    const float mine = kv8_exp2(m - M + (d - D));
    float norm, tiny;
    kv8_scale(D, norm, tiny);
    norm /= den;
    const int r = r0 + c, i = kv8_query(pl, r);
#pragma unroll
    for (int t0 = 0; t0 < DT; t0 += CH) {
        if (t0) __syncthreads();
#pragma unroll
        for (int t = 0; t < CH; ++t) if (t0 + t < DT) o_slot[wave][t][lane] = o[t0 + t] * mine;
        __syncthreads();
        for (int t = wave; t < CH && t0 + t < DT; t += KV8_WAVES) {
            f32x4 a = o_slot[0][t][lane];
#pragma unroll
            for (int w = 1; w < KV8_WAVES; ++w) a += o_slot[w][t][lane];
            const int d = (t0 + t) * 16 + g * 4;
            if (r >= rows) continue;
            if (pt.splits > 1) *reinterpret_cast<float4 *>(dst + c * HD + d) = make_float4(a[0], a[1], a[2], a[3]);
            else kv8_out(out + ((size_t)b * pl.L + i) * ldo + ((size_t)head * pl.group + (r - i * pl.group)) * HD + d, a * norm * tiny, vec & 2);
        }
    }
    if (pt.splits > 1 && wave == 0 && g == 0 && r < rows) { dst[RG * HD + c] = M; dst[RG * HD + RG + c] = D; dst[RG * HD + 2 * RG + c] = den; }
}

// Joins the splits of a pair.  64 units (four values of a row) a workgroup, KV8_JOIN threads each: a thread takes every KV8_JOIN-th split,
// then they meet in LDS in order.
#define KV8_JOIN 4
template <typename T>
__global__ __launch_bounds__(64 * KV8_JOIN) void kv8_merge_kernel(const float *__restrict__ part, Kv8Plan pl, int hd, int slots_total, T *__restrict__ out,
                                                                  int64_t ldo, int vec)
{
    __shared__ float red[KV8_JOIN][3][64];
    __shared__ f32x4 acc[KV8_JOIN][64];
    Kv8Part pt;
    if (!kv8_part(pl, (int)blockIdx.y, true, pt) || pt.splits < 2) return;
    const int head = blockIdx.x, b = kv8_seq(pl, pt.pair), r0 = (pt.pair - b * pl.qgroups) * KV8_ROWS, rows = pl.L * pl.group;
    const size_t rec = kv8_record(hd);
    const float *src = part + ((size_t)head * slots_total + pt.base) * rec;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int u = (int)blockIdx.z * 64 + x, lr = u / (hd / 4), d = u % (hd / 4) * 4, r = r0 + lr;
    const bool live = lr < KV8_ROWS && r < rows;
    const float *e = src + KV8_ROWS * hd + lr;
    float M = KV8_NONE, D = 0.f, den = 0.f;
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float ms, float ds, float ls, const f32x4 &v) {
        const float Mn = fmaxf(M, ms), down = M - Mn, downs = ms - Mn, Dn = rintf(fmaxf(D + down, ds + downs));
        den = den * kv8_exp2(down) + ls * kv8_exp2(downs);
        a = a * kv8_exp2(down + (D - Dn)) + v * kv8_exp2(downs + (ds - Dn));
        M = Mn; D = Dn;
    };
    if (live) {
#pragma unroll 4
        for (int s = y; s < pt.splits; s += KV8_JOIN) {
            const float4 v = *reinterpret_cast<const float4 *>(src + s * rec + lr * hd + d);
            add(e[s * rec], e[s * rec + KV8_ROWS], e[s * rec + 2 * KV8_ROWS], (f32x4){v.x, v.y, v.z, v.w});
        }
    }
    red[y][0][x] = M; red[y][1][x] = D; red[y][2][x] = den;
    acc[y][x] = a;
    __syncthreads();
    if (y || !live) return;
#pragma unroll
    for (int i = 1; i < KV8_JOIN; ++i) add(red[i][0][x], red[i][1][x], red[i][2][x], acc[i][x]);
    const int i = kv8_query(pl, r);
    float norm, tiny;
    kv8_scale(D, norm, tiny);
    kv8_out(out + ((size_t)b * pl.L + i) * ldo + ((size_t)head * pl.group + (r - i * pl.group)) * hd + d, a * (norm / den) * tiny, vec & 2);
}

static int kv8_plan(int n_seqs, int L, int n_heads, int n_kv, int hd, int cap, Kv8Plan *pl, int *slots_total)
{
    if (!kv8_sizes(n_seqs, L, n_kv, hd, cap) || n_heads < n_kv || n_heads % n_kv || n_heads > KV8_MAX_HEADS) return SJD_EINVAL;
    const int64_t rows = (int64_t)L * (n_heads / n_kv);
    const int64_t pairs = n_seqs * ((rows + KV8_ROWS - 1) / KV8_ROWS);
    if (rows > INT32_MAX - KV8_ROWS || pairs > 65535) return SJD_EINVAL;
    pl->n_seqs = n_seqs; pl->L = L; pl->group = n_heads / n_kv; pl->qgroups = (int)((rows + KV8_ROWS - 1) / KV8_ROWS);
    auto shift = [](int d) { return d & (d - 1) ? -1 : __builtin_ctz(d); };
    pl->group_shift = shift(pl->group); pl->qgroups_shift = shift(pl->qgroups);
    pl->cap = cap; pl->nblk = (cap + 31) / 32;
    // Too few workgroups: splits for 256.  (512: 15.0 us against 13.7, one query, 4 k positions; splits up to 384 pairs and heads: 25.5 against 15.3,
    // 8 x 16 queries of 32 heads.)
    // Enough, but windows over long caches, of which one sequence may hold most: walks longer than 5/4 of the mean are cut.  One sequence of 30 k
    // positions and seven of 100, 32 heads: 45.6 us against 102; eight of 2000, where it only costs the second launch, 27.1 against 23.8.  (Prompts have
    // many groups of rows, which even out by themselves: 38 against 63; and every workgroup looks at all pairs.)
    const bool few = pairs * n_kv < 192, skew = pl->nblk > KV8_SKEW && rows <= 32 && pairs <= 256;
    pl->slots = pl->nblk <= KV8_SHORT ? 0 : few ? std::max(1, 256 / n_kv) : skew ? ((int)pairs * 4 + 4) / 5 : 0;
    pl->least = few ? KV8_WAVES : KV8_SHORT;
    *slots_total = (int)pairs + pl->slots;
    return SJD_OK;
}

extern "C" int sjd_kv8_attention_workspace(int32_t n_seqs, int32_t L, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t cap,
                                           size_t *bytes)
{
    if (!bytes) return SJD_EINVAL;
    Kv8Plan pl;
    int slots;
    SJD_TRY(kv8_plan(n_seqs, L, n_heads, n_kv_heads, head_dim, cap, &pl, &slots));
    *bytes = pl.slots ? (size_t)slots * n_kv_heads * kv8_record(head_dim) * sizeof(float) : 0;
    return SJD_OK;
}

extern "C" int sjd_kv8_attention(int32_t dtype, const void *q, int64_t ldq, const uint8_t *cache, const uint8_t *scales, const int32_t *len,
                                 int32_t n_seqs, int32_t L, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t cap, int32_t window,
                                 int32_t sinks, void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !cache || !scales || !len || !out || (dtype != 0 && dtype != 1) || window < 0 || sinks < 0) return SJD_EINVAL;
    if (!mx_aligned(cache) || !mx_aligned(scales)) return SJD_EINVAL;
    size_t need = 0;
    SJD_TRY(sjd_kv8_attention_workspace(n_seqs, L, n_heads, n_kv_heads, head_dim, cap, &need));
    if (need && (!workspace || workspace_bytes < need || !mx_aligned(workspace))) return SJD_EINVAL;
    if (ldq < (int64_t)n_heads * head_dim || ldo < (int64_t)n_heads * head_dim) return SJD_EINVAL;
    Kv8Plan pl;
    int slots;
    SJD_TRY(kv8_plan(n_seqs, L, n_heads, n_kv_heads, head_dim, cap, &pl, &slots));
    pl.len = len; pl.window = window; pl.sinks = sinks;
    const int vec = (mx_vec(q, ldq, dtype) ? 1 : 0) | ((uintptr_t)out % (dtype ? 8 : 16) == 0 && ldo % 4 == 0 ? 2 : 0);
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid(n_kv_heads, slots);
#define GO1(HD, T) SJD_LAUNCH((kv8_attention_kernel<HD, T>), grid, dim3(64 * KV8_WAVES), 0, s, (const T *)q, ldq, cache, scales, pl, (T *)out, ldo, vec, (float *)workspace)
#define GO(HD) do { if (dtype == 0) GO1(HD, float); else GO1(HD, bf16_t); } while (0)
    switch (head_dim) {
        case 32: GO(32); break;
        case 64: GO(64); break;
        case 96: GO(96); break;
        case 128: GO(128); break;
        default: GO(256); break;
    }
#undef GO
#undef GO1
    HIP_TRY(hipGetLastError());
    if (pl.slots) {
        const int join = 64 * KV8_JOIN, units = std::min<int64_t>(KV8_ROWS, (int64_t)pl.L * pl.group) * (head_dim / 4);
        const dim3 mgrid(n_kv_heads, pl.n_seqs * pl.qgroups, (units + 63) / 64);
        if (dtype == 0) SJD_LAUNCH((kv8_merge_kernel<float>), mgrid, dim3(join), 0, s, (const float *)workspace, pl, head_dim, slots, (float *)out, ldo, vec);
        else SJD_LAUNCH((kv8_merge_kernel<bf16_t>), mgrid, dim3(join), 0, s, (const float *)workspace, pl, head_dim, slots, (bf16_t *)out, ldo, vec);
        HIP_TRY(hipGetLastError());
    }
    return SJD_OK;
}
