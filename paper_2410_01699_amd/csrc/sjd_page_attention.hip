// Attention of new tokens over a paged cache (see include/sjd.h for the records): causal, grouped heads, ragged, with a prefix that several
// sequences share computed once for all of them.
#include "sjd_page.h"

#include <algorithm>

typedef __attribute__((ext_vector_type(8))) __bf16 b16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

#define PA_WAVES 4
#define PA_ROWS 16
#define PA_TOP 16.f                       // a row's reference stays until a score is 2^PA_TOP above it
#define PA_NONE -3.4028234664e38f         // reference of a row that has seen nothing: finite, so that differences need no cases
#define PA_FAR 1048576.f                  // references from here on: fp32 has 1/8 between scores

// The work is cut three ways.  A segment is what queries and keys have in common: the queries of one sequence over its own positions, or those of
// a group of sequences over the prefix that they share.  A segment's (row, head) pairs, the heads of one cache head next to each
// other, are cut into tiles of PA_ROWS; where tiles are too few for the chip, their walks over the blocks of 32 positions are cut
// into splits.  Lengths live on the device, so every workgroup works the cut out for itself, all alike.
struct PaPlan {
    PageSeqs sq;
    const int32_t *groups, *prefix;
    int32_t n_groups;
    int32_t heads, group, group_shift;         // cache heads; query heads to one, and the logarithm of that or -1
    int32_t window, sinks;
    int32_t slots, least;                      // splits to aim for per cache head, of so many blocks at least; 0: none cut
    int32_t items;                             // (segment, tile, split) triples a launch has room for
};
__device__ __forceinline__ int pa_div(const PaPlan &pl, int x) { return pl.group_shift >= 0 ? x >> pl.group_shift : x / pl.group; }

// Blocks v < front are the sinks', then come those from first on, count in all
struct PaSeg { int32_t r0, m, n, seq, first, front, count; };      // n: position of row r0 (own), -1 (a prefix); seq: whose table is read
__device__ __forceinline__ int pa_group_of(const PaPlan &pl, int b)         // the group that holds sequence b, or -1
{
    int lo = 0, hi = pl.n_groups;                      // the last group that begins at or before b
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (pl.groups[mid] <= b) lo = mid + 1;
        else hi = mid;
    }
    return lo > 0 && b < pl.groups[lo] ? lo - 1 : -1;
}
// Blocks that the sequences of group g have in common, 0 where the group has fewer than two
__device__ __forceinline__ int pa_shared(const PaPlan &pl, int g)
{
    const int gs = max(pl.groups[g], 0), ge = min(pl.groups[g + 1], pl.sq.n_seqs);
    if (ge - gs < 2) return 0;
    return min(max(pl.prefix[g], 0), pl.sq.width << pl.sq.page_shift) >> 5;
}
__device__ __forceinline__ PaSeg pa_segment(const PaPlan &pl, int s)
{
    PaSeg sg = {0, 0, -1, 0, 0, 0, 0};
    if (s < pl.n_groups) {
        const int shared = pa_shared(pl, s);
        if (!shared) return sg;
        const int gs = max(pl.groups[s], 0), ge = min(pl.groups[s + 1], pl.sq.n_seqs);
        sg.r0 = min(max(pl.sq.start[gs], 0), pl.sq.rows);
        sg.m = min(max(pl.sq.start[ge], sg.r0), pl.sq.rows) - sg.r0;
        sg.seq = gs;
        sg.count = sg.m ? shared : 0;
        return sg;
    }
    const int b = s - pl.n_groups;
    const PageSeq q = page_seq(pl.sq, b);
    sg.r0 = q.r0; sg.m = q.m; sg.n = q.n; sg.seq = b;
    if (!q.m) return sg;
    const int last = (q.n + q.m - 1) >> 5;
    if (pl.window) {
        sg.first = max(0, q.n - pl.window + 1) >> 5;
        sg.front = min((min(pl.sinks, q.n + q.m) + 31) >> 5, sg.first);
    }
    if (pl.n_groups) {
        const int g = pa_group_of(pl, b);
        if (g >= 0) sg.first = min(pa_shared(pl, g), last + 1);
    }
    sg.count = sg.front + last + 1 - sg.first;
    return sg;
}

struct PaPart { int32_t seg, tile, split, splits, per, base; };
__device__ __forceinline__ int pa_tiles(const PaPlan &pl, const PaSeg &sg) { return (sg.m * pl.group + PA_ROWS - 1) / PA_ROWS; }
__device__ __forceinline__ int pa_per(const PaPlan &pl)
{
    if (!pl.slots) return 0x3FFFFFFF;
    const int n = pl.n_groups + pl.sq.n_seqs, lane = threadIdx.x & 63;
    float total = 0.f;
    for (int s0 = 0; s0 < n; s0 += 64) {
        float c = 0.f;
        if (s0 + lane < n) { const PaSeg sg = pa_segment(pl, s0 + lane); c = (float)sg.count * pa_tiles(pl, sg); }
        for (int o = 1; o < min(n, 64); o <<= 1) c += __shfl_xor(c, o);
        total += __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(c)));
    }
    return (int)fmaxf((float)pl.least, fminf(ceilf(total / (float)pl.slots), 1e9f));
}
// The part that a slot is, or (by_seg) the first one of a segment.  With per >= total / slots the splits of all tiles are at most slots + tiles.
__device__ __forceinline__ bool pa_part(const PaPlan &pl, int per, int want, bool by_seg, PaPart &part)
{
    const int n = pl.n_groups + pl.sq.n_seqs, lane = threadIdx.x & 63;
    int base = 0;
    for (int s0 = 0; s0 < n; s0 += 64) {
        int tiles = 0, splits = 0;
        if (s0 + lane < n) {
            const PaSeg sg = pa_segment(pl, s0 + lane);
            splits = (int)(((int64_t)sg.count + per - 1) / per);
            tiles = sg.count ? pa_tiles(pl, sg) : 0;
        }
        int incl = tiles * splits;
        const int mine = incl;
        for (int o = 1; o < min(n, 64); o <<= 1) { const int up = __shfl_up(incl, o); if (lane >= o) incl += up; }
        const int begin = base + incl - mine;
        const uint64_t hit = by_seg ? __ballot(s0 + lane == want) : __ballot(want >= begin && want < begin + mine);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            part.seg = s0 + l;
            part.splits = __builtin_amdgcn_readlane(splits, l);
            part.base = __builtin_amdgcn_readlane(begin, l);
            const int at = by_seg ? 0 : want - part.base;
            part.per = per;
            part.tile = part.splits ? at / part.splits : 0;
            part.split = part.splits ? at % part.splits : 0;
            return true;
        }
        base += __builtin_amdgcn_readlane(incl, min(n, 64) - 1);
    }
    return false;
}

// The sequence whose table a prefix is read from: the first of the group that does not sit out
__device__ __forceinline__ int pa_reader(const PaPlan &pl, int g)
{
    const int gs = max(pl.groups[g], 0), ge = min(pl.groups[g + 1], pl.sq.n_seqs);
    for (int b = gs; b < ge; ++b) if (page_seq(pl.sq, b).m) return b;
    return gs;
}
// Position of a row of group g, or -1 where its sequence sits out
__device__ __forceinline__ int pa_position(const PaPlan &pl, int g, int row)
{
    int lo = max(pl.groups[g], 0), hi = min(pl.groups[g + 1], pl.sq.n_seqs);        // the first sequence that ends behind the row
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (pl.sq.start[mid + 1] <= row) lo = mid + 1;
        else hi = mid;
    }
    if (lo >= pl.sq.n_seqs) return -1;
    const PageSeq q = page_seq(pl.sq, lo);
    return q.m && row >= q.r0 && row < q.r0 + q.m ? q.n + row - q.r0 : -1;
}

// ---- what a wave does with a block -------------------------------------------------------------
__device__ __forceinline__ float pa_across(float x)          // the largest over the four lanes of a column (l % 16)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pa_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Operands.  A block's scores come as two tiles S^T[position][row], whose results leave lane (g, c) = (l / 16, l % 16) with row c and four positions;
// the positions of a tile's rows are chosen so that these are the ones that a unit of 16 bytes of the values holds, so probabilities are the
// second product's operand where they are.
//   bf16: tile a, row r is position 16 (r / 8) + 4 (r / 4 % 2) + 8 a + r % 4; a lane's eight positions are those of unit g
//   fp32: tile a, row r is position 16 a + r; four of a lane's are those of unit 4 a + g
template <typename T> struct PaOps;
template <> struct PaOps<bf16_t> {
    __device__ static __forceinline__ int position(int a, int r) { return ((r >> 3) << 4) + ((r >> 2 & 1) << 2) + (a << 3) + (r & 3); }
};
template <> struct PaOps<float> {
    __device__ static __forceinline__ int position(int a, int r) { return 16 * a + r; }
};
__device__ __forceinline__ b16x8 as_b16(const uint4 &u) { return __builtin_bit_cast(b16x8, u); }
__device__ __forceinline__ float word(const uint4 &u, int i) { return __uint_as_float((&u.x)[i]); }

template <int HD, typename T> struct PaTile {
    static constexpr int B16 = sizeof(T) == 2;
    static constexpr int KS = B16 ? HD / 32 : HD / 16;         // 16-byte units of a row to a lane
    static constexpr int DT = HD / 16;
    static constexpr int VU = B16 ? 1 : 2;                     // units of values to a tile of 16 dimensions
    static constexpr int NK = 2 * KS, NV = DT * VU;            // loads a block
    // bytes into a record: what a lane adds, and what is the same for all
    __device__ static __forceinline__ int k_lane(int lane) { return 16 * ((lane >> 4) * 32 + PaOps<T>::position(0, lane & 15)); }
    static constexpr int k_at(int a, int ks) { return 16 * (128 * ks + (B16 ? 8 : 16) * a); }
    __device__ static __forceinline__ int v_lane(int lane) { return 16 * ((lane >> 4) * 32 + (lane & 15)); }
    static constexpr int v_at(int t, int a) { return 32 * HD * (int)sizeof(T) + 16 * ((t >> 1) * 32 * (B16 ? 4 : 8) + 128 * a + (t & 1) * 16); }
    __device__ static __forceinline__ f32x4 score(const uint4 &k, const uint4 &q, f32x4 s)
    {
        if constexpr (B16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(k), as_b16(q), s, 0, 0, 0);
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(word(k, i), word(q, i), s, 0, 0, 0);
            return s;
        }
    }
};
// The top bit of each value of a word that is an infinity or NaN
__device__ __forceinline__ uint32_t pa_wild(uint32_t w, bf16_t) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t pa_wild(uint32_t w, float) { return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u; }

__device__ __forceinline__ size_t pa_record(int hd) { return (size_t)PA_ROWS * (hd + 2); }      // O[PA_ROWS][hd], then m and l of the rows

template <typename T> __device__ __forceinline__ void pa_out(T *p, const f32x4 &v, bool vec);
template <> __device__ __forceinline__ void pa_out<float>(float *p, const f32x4 &v, bool vec)
{
    if (vec) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else { p[0] = v[0]; p[1] = v[1]; p[2] = v[2]; p[3] = v[3]; }
}
template <> __device__ __forceinline__ void pa_out<bf16_t>(bf16_t *p, const f32x4 &v, bool vec)
{
    if (vec) *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    else { p[0] = f32_to_bf16(v[0]); p[1] = f32_to_bf16(v[1]); p[2] = f32_to_bf16(v[2]); p[3] = f32_to_bf16(v[3]); }
}

// l = sum 2^(s - m), O = sum 2^(s - m) v, with s in powers of two and a reference m that is at most 2^PA_TOP below the largest s: while no score is
// above that, a block costs 8 exponentials a lane, their sum and a comparison beside its products.  bf16: probabilities go in as
// two bf16 (16 bits), which costs nothing where memory bounds.
template <int HD, typename T>
__global__ __launch_bounds__(64 * PA_WAVES, HD * (int)sizeof(T) < 512 ? 2 : 1) void page_attention_kernel(const T *__restrict__ q, int64_t ldq,
                                                                                                       const T *__restrict__ cache, PaPlan pl, float qk, T *__restrict__ out,
                                                                                                       int64_t ldo, int vec, float *__restrict__ part)
{
    using P = PaTile<HD, T>;
    constexpr int KS = P::KS, DT = P::DT, VU = P::VU, E = 16 / (int)sizeof(T), RECB = 64 * HD * (int)sizeof(T), CH = DT < 8 ? DT : 8;
    constexpr bool AHEAD = HD * (int)sizeof(T) <= 512;                // the next block is requested while this one is worked on, where registers hold both
    __shared__ float m_all[PA_WAVES][PA_ROWS], l_all[PA_WAVES][PA_ROWS];
    __shared__ f32x4 o_slot[PA_WAVES][CH][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const int head = blockIdx.x % (uint32_t)pl.heads, slot = blockIdx.x / (uint32_t)pl.heads;
    PaPart pt;
    if (!pa_part(pl, pa_per(pl), slot, false, pt)) return;
    const PaSeg sg = pa_segment(pl, pt.seg);
    const bool own = pt.seg >= pl.n_groups;
    const int seq = own ? sg.seq : pa_reader(pl, pt.seg);
    const int32_t *row_of_pages = pl.sq.table + (int64_t)seq * pl.sq.width;
    const int e0 = pt.tile * PA_ROWS, entries = sg.m * pl.group;        // (row, head) pairs of the segment
    const int entry = e0 + c, ec = min(entry, entries - 1);
    const int i = pa_div(pl, ec), h = ec - i * pl.group, row = sg.r0 + i;
    // what the tile's last query sees ends the walk
    const int tail = own ? sg.front + max(((sg.n + pa_div(pl, min(e0 + PA_ROWS, entries) - 1)) >> 5) + 1 - sg.first, 0) : sg.count;
    const int beg = pt.split * pt.per, end = min(min(sg.count, tail), beg + pt.per);
    auto place = [&](int v) { return v < sg.front ? v : sg.first + v - sg.front; };

    uint4 qa[KS];
    {
        const T *src = q + (int64_t)row * ldq + ((int64_t)head * pl.group + h) * HD;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = (4 * ks + g) * E;
            if (vec & 1) qa[ks] = *reinterpret_cast<const uint4 *>(src + d);
            else {
                T x[E];
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = src[d + e];
                qa[ks] = __builtin_bit_cast(uint4, x);
            }
        }
    }
    uint4 ka[2][KS], va[DT][VU];
    int64_t rec = -1;
    auto fetch = [&](int v) {           // record of block v, its keys requested; behind the end nothing is read
        rec = page_record(pl.sq, row_of_pages, place(min(v, end - 1)), head, pl.heads);
        const auto b = mx_buffer((const uint8_t *)(cache + max(rec, (int64_t)0) * (64 * HD)), RECB);
        const int at = v < end && rec >= 0 ? P::k_lane(lane) : MX_OOB;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) ka[a][ks] = mx_load16(b, at, P::k_at(a, ks));
    };
    auto fetch_v = [&](int64_t r, bool in) {
        const auto b = mx_buffer((const uint8_t *)(cache + max(r, (int64_t)0) * (64 * HD)), RECB);
        const int at = in && r >= 0 ? P::v_lane(lane) : MX_OOB;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int a = 0; a < VU; ++a) va[t][a] = mx_load16(b, at, P::v_at(t, a));
    };
    int v = beg + wave;
    if (AHEAD && beg < end) {
        fetch(v);
        fetch_v(rec, v < end);
    }
    const int pos = own ? sg.n + i : pa_position(pl, pt.seg, row);

    f32x4 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = PA_NONE, l = 0.f;
    bool far = false;
    for (; v < end; v += PA_WAVES) {
        const int k0 = place(v) * 32;
        if (!AHEAD) fetch(v);
        const int64_t now = rec;
        const bool held = now >= 0;
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int a = 0; a < 2; ++a) s[a] = P::score(ka[a][ks], qa[ks], s[a]);
        __builtin_amdgcn_sched_barrier(0);
        if (AHEAD) fetch(v + PA_WAVES);
        else fetch_v(now, true);
        __builtin_amdgcn_sched_barrier(0);
        // does every row of the tile see all of the block?
        const bool mine = held && k0 + 31 <= pos && (pl.window == 0 || k0 > pos - pl.window || k0 + 31 < pl.sinks);
        const bool whole = __ballot(!mine) == 0;
        uint32_t seen = 0xFFu;
        float bm;
        if (whole) {
            bm = s[0][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) bm = fmaxf(bm, s[e >> 2][e & 3]);
            bm *= qk;
        } else {
            seen = 0;
            bm = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = k0 + PaOps<T>::position(e >> 2, 4 * g + (e & 3));
                const bool see = held & (key <= pos) & ((pl.window == 0) | (key > pos - pl.window) | (key < pl.sinks));
                seen |= see ? 1u << e : 0u;
                bm = fmaxf(bm, see ? s[e >> 2][e & 3] * qk : -INFINITY);
            }
        }
        if (__ballot(bm - m > PA_TOP)) {
            const float mn = fmaxf(m, pa_across(bm)), turn = pa_exp2(m - mn);
            l *= turn;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= turn;
            m = mn;
            far = __ballot(fabsf(m) >= PA_FAR && m > PA_NONE) != 0;
        }
        float x[8];
        if (whole && !far) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = pa_exp2(fmaf(s[e >> 2][e & 3], qk, -m));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float w = s[e >> 2][e & 3] * qk;
                asm("" : "+v"(w));                  // (rounded as the reference was: no fused multiply-add)
                x[e] = seen >> e & 1 ? pa_exp2(w - m) : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) l += x[e];
        if (!whole) {
            // Zero times NaN is NaN: where a mask may hide an infinity or NaN from some row it is taken out, and the rows that see one get it by counting.
            uint32_t any = 0;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int a = 0; a < VU; ++a)
#pragma unroll
                    for (int w = 0; w < 4; ++w) any |= pa_wild((&va[t][a].x)[w], T());
            if (__ballot(any != 0)) {
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    f32x4 hits = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int a = 0; a < VU; ++a) {
                        uint4 ones, vis;
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            uint32_t &x = (&va[t][a].x)[w];
                            asm("" : "+v"(x));                  // (worked out here: kept from above the marks of all dimensions would not fit)
                            const uint32_t bad = pa_wild(x, T());
                            if constexpr (sizeof(T) == 2) {
                                (&ones.x)[w] = (bad >> 15) * 0x3F80u;
                                (&vis.x)[w] = ((seen >> (2 * w) & 1) | (seen >> (2 * w + 1) & 1) << 16) * 0x3F80u;
                                x &= ~((bad >> 15) * 0xFFFFu);
                            } else {
                                hits = __builtin_amdgcn_mfma_f32_16x16x4f32(bad ? 1.f : 0.f, seen >> (4 * a + w) & 1 ? 1.f : 0.f, hits, 0, 0, 0);
                                x = bad ? 0u : x;
                            }
                        }
                        if constexpr (sizeof(T) == 2) hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(ones), as_b16(vis), hits, 0, 0, 0);
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w) if (hits[w] != 0.f) o[t][w] = NAN;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if constexpr (sizeof(T) == 2) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                hi[w] = bf16_pair(x[2 * w], x[2 * w + 1]);
                lo[w] = bf16_pair(x[2 * w] - __uint_as_float(hi[w] << 16), x[2 * w + 1] - __uint_as_float(hi[w] & 0xFFFF0000u));
            }
            const b16x8 ph = as_b16(make_uint4(hi[0], hi[1], hi[2], hi[3])), plo = as_b16(make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(va[t][0]), plo, o[t], 0, 0, 0);
                o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(va[t][0]), ph, o[t], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int a = 0; a < VU; ++a)
#pragma unroll
                    for (int w = 0; w < 4; ++w) o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(word(va[t][a], w), x[4 * a + w], o[t], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (AHEAD) fetch_v(rec, v + PA_WAVES < end);
    }

    // ---- the waves of a workgroup, in wave order ----
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) { m_all[wave][c] = m; l_all[wave][c] = l; }
    __syncthreads();
    float M = PA_NONE, den = 0.f;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) M = fmaxf(M, m_all[w][c]);
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) den += pa_exp2(m_all[w][c] - M) * l_all[w][c];
    const float turn = pa_exp2(m - M);
    // the only part of its rows: no more than one split, and no prefix
    const bool alone = own && pt.splits == 1 && (!pl.n_groups || sg.first == 0 || pl.window);
    const float norm = den == 0.f ? 0.f : 1.f / den;
    float *dst = part + ((size_t)head * pl.items + slot) * pa_record(HD);
#pragma unroll
    for (int t0 = 0; t0 < DT; t0 += CH) {
        if (t0) __syncthreads();
#pragma unroll
        for (int t = 0; t < CH; ++t) if (t0 + t < DT) o_slot[wave][t][lane] = o[t0 + t] * turn;
        __syncthreads();
        for (int t = wave; t < CH && t0 + t < DT; t += PA_WAVES) {
            f32x4 a = o_slot[0][t][lane];
#pragma unroll
            for (int w = 1; w < PA_WAVES; ++w) a += o_slot[w][t][lane];
            const int d = (t0 + t) * 16 + g * 4;
            if (entry >= entries) continue;
            if (!alone) *reinterpret_cast<float4 *>(dst + c * HD + d) = make_float4(a[0], a[1], a[2], a[3]);
            else pa_out(out + (int64_t)row * ldo + ((int64_t)head * pl.group + h) * HD + d, a * norm, vec & 2);
        }
    }
    if (!alone && wave == 0 && g == 0 && entry < entries) { dst[PA_ROWS * HD + c] = M; dst[PA_ROWS * HD + PA_ROWS + c] = den; }
}

// Joins the parts of rows that have several: those of their sequence's tile, then those of the prefix.  A workgroup takes 64 units (four values of a
// row) of an own tile, PA_JOIN threads each: a thread takes every PA_JOIN-th part, then they meet in LDS in order.
#define PA_JOIN 4
template <typename T>
__global__ __launch_bounds__(64 * PA_JOIN) void page_merge_kernel(const float *__restrict__ part, PaPlan pl, int hd, int chunks, T *__restrict__ out, int64_t ldo, int vec)
{
    __shared__ float red[PA_JOIN][2][64];
    __shared__ f32x4 acc[PA_JOIN][64];
    const int head = blockIdx.x % (uint32_t)pl.heads, rest = blockIdx.x / (uint32_t)pl.heads, chunk = rest % chunks;
    // the own tile of this workgroup
    PaPlan tiles = pl;
    tiles.n_groups = 0;
    PaPart at;
    {
        // (counted as if nothing were cut or shared: one part a tile)
        const int n = pl.sq.n_seqs, lane = threadIdx.x & 63, want = rest / chunks;
        int base = 0, found = 0;
        for (int s0 = 0; s0 < n && !found; s0 += 64) {
            int t = 0;
            if (s0 + lane < n) t = (page_seq(pl.sq, s0 + lane).m * pl.group + PA_ROWS - 1) / PA_ROWS;
            int incl = t;
            for (int o = 1; o < min(n, 64); o <<= 1) { const int up = __shfl_up(incl, o); if (lane >= o) incl += up; }
            const uint64_t hit = __ballot(want >= base + incl - t && want < base + incl);
            if (hit) {
                const int l = __ffsll((unsigned long long)hit) - 1;
                at.seg = pl.n_groups + s0 + l;
                at.tile = want - base - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(t, l));
                found = 1;
            }
            base += __builtin_amdgcn_readlane(incl, min(n, 64) - 1);
        }
        if (!found) return;
    }
    const int per = pa_per(pl);
    PaPart mine, shared;
    pa_part(pl, per, at.seg, true, mine);
    const PaSeg sg = pa_segment(pl, at.seg);
    int g = -1;
    shared.splits = 0;
    if (pl.n_groups && !pl.window) {
        g = pa_group_of(pl, sg.seq);
        if (g >= 0) {
            if (!pa_shared(pl, g)) g = -1;
            else pa_part(pl, per, g, true, shared);
        }
    }
    if (g < 0 && mine.splits == 1) return;                  // (written already)
    const size_t rec = pa_record(hd);
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int u = chunk * 64 + x, lr = u / (hd / 4), d = u % (hd / 4) * 4, entry = at.tile * PA_ROWS + lr;
    const bool live = lr < PA_ROWS && entry < sg.m * pl.group;
    const int i = pa_div(pl, min(entry, sg.m * pl.group - 1)), h = entry - i * pl.group;
    const float *from = part + (size_t)head * pl.items * rec;
    const int e2 = g < 0 ? 0 : (sg.r0 + i - pa_segment(pl, g).r0) * pl.group + h;          // the row's place in the prefix's segment
    const int base1 = mine.base + at.tile * mine.splits, base2 = shared.base + e2 / PA_ROWS * shared.splits, lr2 = e2 % PA_ROWS;
    float M = PA_NONE, den = 0.f;
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float ms, float ls, const f32x4 &v) {
        const float Mn = fmaxf(M, ms), down = pa_exp2(M - Mn), downs = pa_exp2(ms - Mn);
        den = den * down + ls * downs;
        a = a * down + v * downs;
        M = Mn;
    };
    if (live) {
        const int parts = mine.splits + shared.splits;
#pragma unroll 4
        for (int s = y; s < parts; s += PA_JOIN) {
            const bool first = s < mine.splits;
            const int r = first ? lr : lr2;
            const float *src = from + (size_t)(first ? base1 + s : base2 + s - mine.splits) * rec;
            const float4 v = *reinterpret_cast<const float4 *>(src + r * hd + d);
            add(src[PA_ROWS * hd + r], src[PA_ROWS * hd + PA_ROWS + r], (f32x4){v.x, v.y, v.z, v.w});
        }
    }
    red[y][0][x] = M; red[y][1][x] = den;
    acc[y][x] = a;
    __syncthreads();
    if (y || !live) return;
#pragma unroll
    for (int w = 1; w < PA_JOIN; ++w) add(red[w][0][x], red[w][1][x], acc[w][x]);
    pa_out(out + (int64_t)(sg.r0 + i) * ldo + ((int64_t)head * pl.group + h) * hd + d, a * (den == 0.f ? 0.f : 1.f / den), vec & 2);
}

static int pa_plan(const sjd_pages *p, int rows, int n_seqs, int n_groups, int n_heads, int width, int window, PaPlan *pl)
{
    if (!page_shape(p) || rows < 1 || rows > PAGE_MAX_ROWS || n_seqs < 1 || n_seqs > PAGE_MAX_SEQS || n_groups < 0 || n_groups > n_seqs) return SJD_EINVAL;
    if (width < 1 || (int64_t)width * p->page > INT32_MAX - 64) return SJD_EINVAL;
    if (n_heads < p->n_kv_heads || n_heads % p->n_kv_heads || n_heads > PAGE_MAX_HEADS) return SJD_EINVAL;
    pl->heads = p->n_kv_heads; pl->group = n_heads / p->n_kv_heads;
    pl->group_shift = pl->group & (pl->group - 1) ? -1 : __builtin_ctz((unsigned)pl->group);
    const int64_t entries = (int64_t)rows * pl->group;
    if (entries > INT32_MAX / 2) return SJD_EINVAL;
    // Tiles: every segment has a last one that is not full.
    const int64_t own = entries / PA_ROWS + n_seqs, shared = n_groups ? entries / PA_ROWS + n_groups : 0;
    const int64_t nblk = ((int64_t)width * p->page + 31) / 32;
    const bool few = own * p->n_kv_heads < 512;
    pl->slots = nblk <= 32 || !few ? 0 : std::max(1, 512 / p->n_kv_heads);
    pl->least = 2 * PA_WAVES;
    pl->n_groups = n_groups;
    if ((own + shared + pl->slots) * p->n_kv_heads >= (int64_t)1 << 24) return SJD_EINVAL;
    pl->items = (int)(own + shared + pl->slots);
    pl->window = window;
    return SJD_OK;
}

extern "C" int sjd_page_attention_workspace(const sjd_pages *pages, int32_t rows, int32_t n_seqs, int32_t n_groups, int32_t n_heads, int32_t width, size_t *bytes)
{
    if (!bytes) return SJD_EINVAL;
    PaPlan pl;
    SJD_TRY(pa_plan(pages, rows, n_seqs, n_groups, n_heads, width, 0, &pl));
    *bytes = pl.slots || n_groups ? (size_t)pl.items * pl.heads * PA_ROWS * (pages->head_dim + 2) * sizeof(float) : 0;
    return SJD_OK;
}

extern "C" int sjd_page_attention(const sjd_pages *pages, const void *q, int64_t ldq, int32_t n_heads, int32_t rows, const int32_t *start, const int32_t *len, int32_t n_seqs,
                                  const int32_t *table, int32_t width, const int32_t *groups, const int32_t *prefix, int32_t n_groups, const void *cache, float scale,
                                  int32_t window, int32_t sinks, void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    PageSeqs sq;
    if (!page_shape(pages) || !page_seqs(pages, start, len, table, width, n_seqs, rows, &sq)) return SJD_EINVAL;
    if (!q || !cache || !out || !mx_aligned(cache) || window < 0 || sinks < 0 || !(scale > 0.f) || !(scale < 1e30f)) return SJD_EINVAL;
    if (n_groups < 0 || (n_groups > 0 && (!groups || !prefix))) return SJD_EINVAL;
    size_t need = 0;
    SJD_TRY(sjd_page_attention_workspace(pages, rows, n_seqs, n_groups, n_heads, width, &need));
    if (need && (!workspace || workspace_bytes < need || !mx_aligned(workspace))) return SJD_EINVAL;
    const int hd = pages->head_dim, dt = pages->dtype;
    if (ldq < (int64_t)n_heads * hd || ldo < (int64_t)n_heads * hd) return SJD_EINVAL;
    // (of a prefix little is left inside a window, and what a query sees of it is its own: a window's walks are the sequences' own)
    PaPlan pl;
    SJD_TRY(pa_plan(pages, rows, n_seqs, window ? 0 : n_groups, n_heads, width, window, &pl));
    pl.sq = sq; pl.groups = groups; pl.prefix = prefix; pl.sinks = sinks;
    const int vec = (mx_vec(q, ldq, dt) ? 1 : 0) | ((uintptr_t)out % (dt ? 8 : 16) == 0 && ldo % 4 == 0 ? 2 : 0);
    const float qk = scale * 1.4426950408889634f;
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)(pl.items * pl.heads));
#define GO1(HD, T) SJD_LAUNCH((page_attention_kernel<HD, T>), grid, dim3(64 * PA_WAVES), 0, s, (const T *)q, ldq, (const T *)cache, pl, qk, (T *)out, ldo, vec, (float *)workspace)
#define GO(HD) do { if (dt == 0) GO1(HD, float); else GO1(HD, bf16_t); } while (0)
    switch (hd) {
        case 32: GO(32); break;
        case 64: GO(64); break;
        case 96: GO(96); break;
        case 128: GO(128); break;
        default: GO(256); break;
    }
#undef GO
#undef GO1
    HIP_TRY(hipGetLastError());
    if (pl.slots || pl.n_groups) {
        const int chunks = (PA_ROWS * (hd / 4) + 63) / 64;
        const int64_t tiles = (int64_t)rows * pl.group / PA_ROWS + n_seqs;
        const dim3 mgrid((unsigned)(tiles * chunks * pl.heads));
        if (dt == 0) SJD_LAUNCH((page_merge_kernel<float>), mgrid, dim3(64 * PA_JOIN), 0, s, (const float *)workspace, pl, hd, chunks, (float *)out, ldo, vec);
        else SJD_LAUNCH((page_merge_kernel<bf16_t>), mgrid, dim3(64 * PA_JOIN), 0, s, (const float *)workspace, pl, hd, chunks, (bf16_t *)out, ldo, vec);
        HIP_TRY(hipGetLastError());
    }
    return SJD_OK;
}
