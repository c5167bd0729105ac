// Paged caches of keys and values (see include/sjd.h): layout and helpers shared by the operators that write and read them.
#pragma once
#include "sjd_mx.h"

#define PAGE_MAX_SEQS 65535
#define PAGE_MAX_HEADS 4096
#define PAGE_MAX_ROWS (1 << 24)

// A pool of pages and the sequences that a call is about.  Rows start[b] .. start[b + 1] - 1 are the new tokens of sequence b, which stand at
// positions len[b] ..; entry p / page of its table row is the page of position p.  Everything device memory holds is taken as possibly
// wrong: starts are kept inside the rows, a sequence that does not fit its table sits out, pages outside the pool hold nothing.
struct PageSeqs {
    const int32_t *start, *len, *table;
    int32_t n_seqs, rows, width, page_shift, n_pages;
};
struct PageSeq { int32_t r0, m, n; };        // first row, new tokens (0: sits out), cached positions
__device__ __forceinline__ PageSeq page_seq(const PageSeqs &sq, int b)
{
    PageSeq s;
    s.r0 = min(max(sq.start[b], 0), sq.rows);
    s.m = min(max(sq.start[b + 1], s.r0), sq.rows) - s.r0;
    s.n = sq.len[b];
    if (s.n < 0 || (int64_t)s.n + s.m > (int64_t)sq.width << sq.page_shift) s.m = 0;
    return s;
}
// Record of block blk (32 positions) of a sequence, in records of one head from the pool's start on: -1 where the page is none of the pool's
__device__ __forceinline__ int64_t page_record(const PageSeqs &sq, const int32_t *row, int blk, int head, int heads)
{
    const int sh = sq.page_shift - 5, id = row[blk >> sh];
    return (uint32_t)id < (uint32_t)sq.n_pages ? (((int64_t)id * heads + head) << sh) + (blk & ((1 << sh) - 1)) : -1;
}

__device__ __forceinline__ int page_lane(int x, int l) { return __builtin_amdgcn_readlane(x, l); }
// The sum over this lane and those before it: inside rows of 16 lanes, then from row to row
template <int CTRL, int ROWS> __device__ __forceinline__ int page_from(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ float page_from(float x) { return __int_as_float(page_from<CTRL, ROWS>(__float_as_int(x))); }
template <typename N> __device__ __forceinline__ N page_sum_up(N x)
{
    x += page_from<0x111, 0xF>(x); x += page_from<0x112, 0xF>(x); x += page_from<0x114, 0xF>(x); x += page_from<0x118, 0xF>(x);
    x += page_from<0x142, 0xA>(x);
    x += page_from<0x143, 0xC>(x);
    return x;
}

static inline bool page_shape(const sjd_pages *p)
{
    if (!p || (p->dtype != 0 && p->dtype != 1) || p->n_kv_heads < 1 || p->n_kv_heads > PAGE_MAX_HEADS || p->n_pages < 1) return false;
    if (p->page < 32 || p->page > 1 << 16 || (p->page & (p->page - 1))) return false;
    const int hd = p->head_dim;
    return hd == 32 || hd == 64 || hd == 96 || hd == 128 || hd == 256;
}
static inline bool page_seqs(const sjd_pages *p, const int32_t *start, const int32_t *len, const int32_t *table, int width, int n_seqs, int rows, PageSeqs *sq)
{
    if (!start || !len || !table || n_seqs < 1 || n_seqs > PAGE_MAX_SEQS || rows < 1 || rows > PAGE_MAX_ROWS) return false;
    if (width < 1 || (int64_t)width * p->page > INT32_MAX - 64) return false;
    *sq = {start, len, table, n_seqs, rows, width, __builtin_ctz((unsigned)p->page), p->n_pages};
    return true;
}

// ---- rotary positions -----------------------------------------------------------------------
// A pair's angle at a position is position * frequency, modulo whole turns, in units of 2^-64 turns: exact in 64-bit whole numbers
// however far the position is.  The nearest quarter turn comes off; what is left, |r| <= pi / 4 to 2^-32 turns, goes into the Taylor
// series of sine and cosine, whose first terms left out are r^11 / 11! < 2e-9 and r^12 / 12! < 2e-10.
__device__ __forceinline__ void rope_angle(int pos, uint64_t turns, float magnitude, float &c, float &s)
{
    // the product's upper half, an eighth up, so that its top two bits round (a negative position is 2^32 too large where it is multiplied)
    const uint32_t p = (uint32_t)pos, lo = (uint32_t)turns, hi = (uint32_t)(turns >> 32);
    const uint32_t a = __umulhi(p, lo) + p * hi - (pos < 0 ? lo : 0u) + 0x20000000u;
    const int quarter = (int)(a >> 30);
    const float r = (float)((int)(a & 0x3FFFFFFFu) - 0x20000000) * 1.4629180792671596e-9f;        // 2 pi / 2^32
    const float z = r * r;
    const float sn = r * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -0.16666667f), 1.f);
    const float cn = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
    const float cs = (quarter & 1) ? sn : cn, ss = (quarter & 1) ? cn : sn;
    // cosines are negative in quarters 1 and 2, sines in 2 and 3
    c = __uint_as_float(__float_as_uint(cs) ^ ((a + 0x40000000u) & 0x80000000u)) * magnitude;
    s = __uint_as_float(__float_as_uint(ss) ^ (a & 0x80000000u)) * magnitude;
}
struct Rope { const uint64_t *turns; int32_t rot, interleaved; float magnitude, sign; };      // rot 0: nothing turns
// (the fields of a call, or nothing to turn)
static inline bool rope_fits(const uint64_t *turns, int rot, int interleaved, float magnitude, int hd)
{
    if (!turns) return rot == 0;
    return rot >= 2 && rot % 2 == 0 && rot <= hd && (interleaved == 0 || interleaved == 1) && magnitude == magnitude && fabsf(magnitude) <= 3.4e38f && (uintptr_t)turns % 8 == 0;
}

// Eight values as they are stored
template <typename T> struct Eight { uint4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ float eight_get(const Eight<T> &x, int e);
template <> __device__ __forceinline__ float eight_get<float>(const Eight<float> &x, int e) { return __uint_as_float((&x.w[e >> 2].x)[e & 3]); }
template <> __device__ __forceinline__ float eight_get<bf16_t>(const Eight<bf16_t> &x, int e)
{
    const uint32_t w = (&x.w[0].x)[e >> 1];
    return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
}
__device__ __forceinline__ void eight_set(Eight<float> &x, const float (&v)[8])
{
    x.w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    x.w[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
}
// Two values in bf16, to the nearest, ties to even, NaN stays NaN: one instruction
__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 b16x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, b16x2));
}
__device__ __forceinline__ void eight_set(Eight<bf16_t> &x, const float (&v)[8])
{
    x.w[0] = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}
template <typename T> __device__ __forceinline__ Eight<T> eight_load(const T *p)
{
    Eight<T> x;
#pragma unroll
    for (int w = 0; w < (int)sizeof(T) / 2; ++w) x.w[w] = reinterpret_cast<const uint4 *>(p)[w];
    return x;
}
template <typename T> __device__ __forceinline__ void eight_store(T *p, const Eight<T> &x)
{
#pragma unroll
    for (int w = 0; w < (int)sizeof(T) / 2; ++w) reinterpret_cast<uint4 *>(p)[w] = x.w[w];
}
template <typename T> __device__ __forceinline__ float one_get(T v);
template <> __device__ __forceinline__ float one_get<float>(float v) { return v; }
template <> __device__ __forceinline__ float one_get<bf16_t>(bf16_t v) { return bf16_to_f32(v); }
template <typename T> __device__ __forceinline__ T one_set(float v);
template <> __device__ __forceinline__ float one_set<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t one_set<bf16_t>(float v) { return (bf16_t)bf16_pair(v, v); }

// Unit u of a head's hd / 16: sixteen values in two eights, at eight_at(u, 0) and eight_at(u, 1).  Where rot is a multiple of 16 the first
// rot / 16 units hold both values of their pairs: the eights u and u + rot / 16 of the half layout, two neighbours of the interleaved one.
// Sixteen values that do not turn are two neighbours behind them.
__device__ __forceinline__ int eight_at(const Rope &ro, int u, int which)
{
    const int units = ro.rot >> 4;
    if (u < units && !ro.interleaved) return 8 * (u + which * units);
    return 16 * u + 8 * which;
}
struct UnitAngles { float c[8], s[8]; };
__device__ __forceinline__ void unit_angles(const Rope &ro, int u, int pos, UnitAngles &a)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        rope_angle(pos, ro.turns[8 * u + e], ro.magnitude, a.c[e], a.s[e]);
        a.s[e] *= ro.sign;
    }
}
template <typename T> __device__ __forceinline__ void unit_turn(const Rope &ro, const UnitAngles &a, Eight<T> &x, Eight<T> &y)
{
    float p[8], q[8];
    if (!ro.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = eight_get(x, e), v = eight_get(y, e);
            p[e] = fmaf(u, a.c[e], -v * a.s[e]); q[e] = fmaf(v, a.c[e], u * a.s[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = eight_get(x, 2 * e), v = eight_get(x, 2 * e + 1), w = eight_get(y, 2 * e), z = eight_get(y, 2 * e + 1);
            p[2 * e] = fmaf(u, a.c[e], -v * a.s[e]); p[2 * e + 1] = fmaf(v, a.c[e], u * a.s[e]);
            q[2 * e] = fmaf(w, a.c[e + 4], -z * a.s[e + 4]); q[2 * e + 1] = fmaf(z, a.c[e + 4], w * a.s[e + 4]);
        }
    }
    eight_set(x, p); eight_set(y, q);
}
// Pair i of the rot / 2 of a head: the places of its two values
__device__ __forceinline__ void pair_at(const Rope &ro, int i, int &a, int &b)
{
    if (ro.interleaved) { a = 2 * i; b = a + 1; }
    else { a = i; b = i + (ro.rot >> 1); }
}
