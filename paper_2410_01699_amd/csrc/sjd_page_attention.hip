// Attention of new tokens over a paged cache (see include/sjd.h for the records): causal, grouped heads, ragged, with a prefix that several
// sequences share computed once for all of them.
#include "sjd_page.h"

#include <algorithm>

typedef __attribute__((ext_vector_type(8))) __bf16 b16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

#define PA_WAVES 4
#define PA_TOP 16.f                       // a row's reference stays until a score is 2^PA_TOP above it
#define PA_NONE -3.4028234664e38f         // reference of a row that has seen nothing: finite, so that differences need no cases
#define PA_LOW -3.4028e38f               // least reference of a row that has seen something: what overflows downwards weighs nothing against it
#define PA_FAR 1048576.f                  // references from here on: fp32 has 1/8 between scores

// The work is cut three ways.  A segment is what queries and keys have in common: the queries of one sequence over its own positions, or those of
// a group of sequences over the prefix that they share.  A segment's (row, head) pairs, the heads of one cache head next to each
// other, are cut into tiles of `rows` (16, 32 or 128); where tiles are too few for the chip, their walks over the blocks of 32 positions are cut
// into splits.  Lengths live on the device, so every workgroup works the cut out for itself, all alike, and those of a tile's first split leave
// word of it for the kernel that joins the parts.
struct PaPlan {
    PageSeqs sq;
    const int32_t *groups, *prefix;
    int32_t n_groups;
    int32_t heads, group, group_shift;         // cache heads; query heads to one, and the logarithm of that or -1
    int32_t window, sinks;
    int32_t rows_shift;                        // logarithm of a tile's rows
    int32_t slots, least;                      // splits to aim for per cache head, of so many blocks at least; 0: none cut
    int32_t items, tiles;                      // (segment, tile, split) triples that a launch has room for, and own tiles
};
__device__ __forceinline__ int pa_div(const PaPlan &pl, int x) { return pl.group_shift >= 0 ? x >> pl.group_shift : x / pl.group; }

// r0, m: rows; n: position of row r0 (of an own segment); seq: whose table is read (a prefix: of the group's first sequence); g: the group whose prefix comes
// before an own segment's blocks, or -1.  Blocks v < front are the sinks', then come those from first on, count in all.
struct PaSeg { int32_t r0, m, n, seq, g, first, front, count; };       // (of a prefix: first, front: the group's sequences [front, front + first), walked from block 0 on)
__device__ __forceinline__ int pa_group_of(const PaPlan &pl, int b)         // the group that holds sequence b, or -1
{
    int lo = 0, hi = pl.n_groups;                      // groups that begin at or before b
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (pl.groups[mid] <= b) lo = mid + 1;
        else hi = mid;
    }
    return lo > 0 && b < pl.groups[lo] ? lo - 1 : -1;
}
// Blocks of the whole pages that the sequences of group g have in common, 0 where the group has fewer than two
__device__ __forceinline__ int pa_inside(const PaPlan &pl, int b) { return min(max(b, 0), pl.sq.n_seqs); }
__device__ __forceinline__ int pa_shared(const PaPlan &pl, int g)
{
    const int gs = pa_inside(pl, pl.groups[g]), ge = pa_inside(pl, pl.groups[g + 1]);
    if (ge - gs < 2) return 0;
    return min(max(pl.prefix[g], 0) >> pl.sq.page_shift, pl.sq.width) << (pl.sq.page_shift - 5);
}
// The blocks of an own segment behind `shared` ones of a prefix
__device__ __forceinline__ void pa_blocks(const PaPlan &pl, PaSeg &sg, int g, int shared)
{
    if (!sg.m) return;
    const int last = (sg.n + sg.m - 1) >> 5;
    if (pl.window) {
        sg.first = max(0, sg.n - pl.window + 1) >> 5;
        sg.front = min((min(pl.sinks, sg.n + sg.m) + 31) >> 5, sg.first);
    }
    if (shared) { sg.g = g; sg.first = min(shared, last + 1); }
    sg.count = sg.front + last + 1 - sg.first;
}
__device__ __forceinline__ PaSeg pa_segment(const PaPlan &pl, int s)
{
    PaSeg sg = {0, 0, 0, 0, -1, 0, 0, 0};
    if (s < pl.n_groups) {
        const int shared = pa_shared(pl, s), gs = pa_inside(pl, pl.groups[s]), ge = pa_inside(pl, pl.groups[s + 1]);
        if (!shared) return sg;
        sg.r0 = min(max(pl.sq.start[gs], 0), pl.sq.rows);
        sg.m = min(max(pl.sq.start[ge], sg.r0), pl.sq.rows) - sg.r0;
        sg.seq = sg.front = gs; sg.first = ge - gs;
        sg.count = sg.m ? shared : 0;
        return sg;
    }
    const int b = s - pl.n_groups;
    const PageSeq q = page_seq(pl.sq, b);
    sg.r0 = q.r0; sg.m = q.m; sg.n = q.n; sg.seq = b;
    const int g = pl.n_groups ? pa_group_of(pl, b) : -1;
    pa_blocks(pl, sg, g, g < 0 ? 0 : pa_shared(pl, g));
    return sg;
}
// Segment `lane` of the first 64.  Where these are all, everything is requested at once and goes from lane to lane: a trip to memory costs more than all that
// follows it.
__device__ __forceinline__ PaSeg pa_first(const PaPlan &pl, int lane)
{
    const int n = pl.n_groups + pl.sq.n_seqs;
    if (n > 64) return pa_segment(pl, lane);
    PaSeg sg = {0, 0, 0, 0, -1, 0, 0, 0};
    const int b = lane - pl.n_groups;
    int gs = 0, ge = 0, pre = 0, s0 = 0, s1 = 0;
    if (lane < pl.n_groups) { gs = pl.groups[lane]; ge = pl.groups[lane + 1]; pre = pl.prefix[lane]; }
    if (b >= 0 && lane < n) { s0 = pl.sq.start[b]; s1 = pl.sq.start[b + 1]; sg.n = pl.sq.len[b]; }
    gs = pa_inside(pl, gs); ge = pa_inside(pl, ge);
    sg.r0 = min(max(s0, 0), pl.sq.rows);
    const int r1 = min(max(s1, sg.r0), pl.sq.rows);
    sg.m = r1 - sg.r0;
    sg.seq = max(b, 0);
    if (sg.n < 0 || (int64_t)sg.n + sg.m > (int64_t)pl.sq.width << pl.sq.page_shift) sg.m = 0;
    int g = -1, shared = ge - gs < 2 ? 0 : min(max(pre, 0) >> pl.sq.page_shift, pl.sq.width) << (pl.sq.page_shift - 5);
    int mine = 0;
    for (int i = pl.n_groups - 1; i >= 0; --i) {            // (the first group that has the sequence)
        const int lo = page_lane(gs, i), hi = page_lane(ge, i), sh = page_lane(shared, i);
        if (b >= lo && b < hi) { g = i; mine = sh; }
        const int f = page_lane(sg.r0, min(pl.n_groups + lo, 63)), l = page_lane(r1, max(min(pl.n_groups + hi, 64) - 1, 0));
        if (lane == i && shared) { sg.r0 = f; sg.m = max(l - f, 0); sg.n = 0; sg.seq = sg.front = lo; sg.first = hi - lo; sg.count = sg.m ? shared : 0; }
    }
    if (b < 0 && !shared) sg.m = 0;
    if (b >= 0) pa_blocks(pl, sg, g, mine);
    return sg;
}
__device__ __forceinline__ int pa_tiles(const PaPlan &pl, const PaSeg &sg) { return (sg.m * pl.group + (1 << pl.rows_shift) - 1) >> pl.rows_shift; }

// What a slot is: its segment, tile and split, the first slot of the segment, and of own segments the number of its first tile among the own ones
struct PaPart { PaSeg sg; int32_t seg, tile, split, splits, per, base, own; };
// Lanes look at 64 segments at a time, c0: those of the first 64.  by_seg: the first slot of the given segment.  own_total: the own tiles whose first slot is launched, if
// the walk gets to its last 64.  With per >= total / slots the splits of all tiles are at most slots + tiles, so that these are all; starts or groups without sense can ask for
// more slots than there are, and the tiles behind them have no word (the join would take what an earlier call left for one) and do not count.  Counts stay below 2^31 there too: no segment's
// above 2^24, no sum before 64 of them above 2^29, both more than a launch has.
__device__ __forceinline__ bool pa_part(const PaPlan &pl, const PaSeg &c0, int per, int want, bool by_seg, PaPart &part, int &own_total)
{
    const int n = pl.n_groups + pl.sq.n_seqs, lane = threadIdx.x & 63;
    int base = 0, own = 0;
    for (int s0 = 0; s0 < n; s0 += 64) {
        const PaSeg sg = s0 == 0 ? c0 : s0 + lane < n ? pa_segment(pl, s0 + lane) : PaSeg{};
        const bool prefix = s0 + lane < pl.n_groups;
        const int splits = max((int)(((int64_t)sg.count + per - 1) / per), !prefix && sg.m ? 1 : 0);     // (of own segments one at least, which may be empty)
        const int tiles = splits ? pa_tiles(pl, sg) : 0, mine = (int)min((int64_t)tiles * splits, (int64_t)1 << 24);
        const int incl = page_sum_up(mine), begin = base + incl - mine;
        int mine_own = prefix ? 0 : tiles;
        if (mine_own && begin + mine > pl.items) mine_own = max(0, pl.items - begin + splits - 1) / splits;
        const int incl_own = page_sum_up(mine_own);
        const uint64_t hit = by_seg ? __ballot(s0 + lane == want) : __ballot(want >= begin && want < begin + mine);
        own_total = own + page_lane(incl_own, 63);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            part.sg = {page_lane(sg.r0, l), page_lane(sg.m, l), page_lane(sg.n, l), page_lane(sg.seq, l), page_lane(sg.g, l), page_lane(sg.first, l), page_lane(sg.front, l), page_lane(sg.count, l)};
            part.seg = s0 + l;
            part.splits = page_lane(splits, l);
            part.base = page_lane(begin, l);
            part.own = own + page_lane(incl_own - mine_own, l);
            part.per = per;
            const int at = by_seg ? 0 : want - part.base, d = max(part.splits, 1);
            part.tile = at / d;
            part.split = at - part.tile * d;
            return true;
        }
        base = min(base + page_lane(incl, 63), 1 << 29);
        own = own_total;
    }
    return false;
}
__device__ __forceinline__ int pa_per(const PaPlan &pl, const PaSeg &c0)
{
    if (!pl.slots) return 0x3FFFFFFF;
    const int n = pl.n_groups + pl.sq.n_seqs, lane = threadIdx.x & 63;
    float total = 0.f;
    for (int s0 = 0; s0 < n; s0 += 64) {
        const PaSeg sg = s0 == 0 ? c0 : s0 + lane < n ? pa_segment(pl, s0 + lane) : PaSeg{};
        const float c = page_sum_up((float)sg.count * pa_tiles(pl, sg));
        total += __int_as_float(page_lane(__float_as_int(c), 63));
    }
    return (int)fmaxf((float)pl.least, fminf(ceilf(total / (float)pl.slots), 1e9f));
}

// Word of an own tile for the kernel that joins its parts: its first row and entries, its tile, its first slot and splits, those of the prefix's first tile, and what its
// entries' numbers are higher there.  In front of all: the number of words.
struct PaWord { int32_t r0, entries, tile, base1, splits1, base2, splits2, above; };
__device__ __forceinline__ PaWord *pa_words(float *part) { return reinterpret_cast<PaWord *>(part) + 1; }

// Position of a row of the sequences lo .. hi - 1, or -1 where its sequence sits out: rows, tokens and positions of the first 64 segments are in LDS
__device__ __forceinline__ int pa_position(const PaPlan &pl, const int32_t (*known)[3], int lo, int hi, int row)
{
    const bool all = pl.n_groups + pl.sq.n_seqs <= 64;
    const int end = hi;
    while (lo < hi) {                           // the first sequence that ends behind the row
        const int mid = (lo + hi) >> 1;
        int last;
        if (all) last = known[pl.n_groups + mid][0] + known[pl.n_groups + mid][1];
        else { const PageSeq q = page_seq(pl.sq, mid); last = q.r0 + q.m; }
        if (last <= row) lo = mid + 1;
        else hi = mid;
    }
    if (lo >= end) return -1;
    PageSeq q;
    if (all) q = {known[pl.n_groups + lo][0], known[pl.n_groups + lo][1], known[pl.n_groups + lo][2]};
    else q = page_seq(pl.sq, lo);
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

// record of a part: O[rows][hd], then m and l of the rows
__device__ __forceinline__ size_t pa_record(int rows, int hd) { return (size_t)rows * (hd + 2); }

template <typename T> __device__ __forceinline__ void pa_out(T *p, const f32x4 &v, bool vec);
template <> __device__ __forceinline__ void pa_out<float>(float *p, const f32x4 &v, bool vec)
{
    if (vec) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else { p[0] = v[0]; p[1] = v[1]; p[2] = v[2]; p[3] = v[3]; }
}
template <> __device__ __forceinline__ void pa_out<bf16_t>(bf16_t *p, const f32x4 &v, bool vec)
{
    if (vec) *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    else { p[0] = one_set<bf16_t>(v[0]); p[1] = one_set<bf16_t>(v[1]); p[2] = one_set<bf16_t>(v[2]); p[3] = one_set<bf16_t>(v[3]); }
}

// What a workgroup is about.  own: a sequence's own positions; alone: the only part of its rows; [gs, ge): a group's sequences; entries e0 .. of the segment's, each a
// row and a head; blocks [beg, end) of the segment's; first: (of a prefix) no row stands before this position.
struct PaWork { PaSeg sg; int32_t own, alone, gs, ge, e0, entries, beg, end, first; };
__device__ __forceinline__ bool pa_work(const PaPlan &pl, int head, int slot, int32_t (*known)[3], float *part, PaWork &w)
{
    const int lane = threadIdx.x & 63, rows = 1 << pl.rows_shift, n = pl.n_groups + pl.sq.n_seqs;
    const PaSeg c0 = pa_first(pl, lane);
    const int per = pa_per(pl, c0);
    PaPart pt;
    int total;
    const bool some = pa_part(pl, c0, per, slot, false, pt, total);
    const bool writer = head == 0 && part && threadIdx.x < 64;
    if (slot == 0 && writer) {
        PaPart none;
        if (n > 64) pa_part(pl, c0, per, 0x7FFFFFFF, false, none, total);
        if (lane == 0) *reinterpret_cast<int32_t *>(part) = total;
    }
    if (!some) return false;
    w.sg = pt.sg;
    w.own = pt.seg >= pl.n_groups;
    w.alone = w.own && pt.splits == 1 && pt.sg.g < 0;
    if (w.own && writer && pt.split == 0) {
        PaWord word = {pt.sg.r0, pt.sg.m * pl.group, pt.tile, pt.base, pt.splits, 0, 0, 0};
        if (pt.sg.g >= 0) {
            PaPart before;
            pa_part(pl, c0, per, pt.sg.g, true, before, total);
            word.base2 = before.base; word.splits2 = before.splits; word.above = (pt.sg.r0 - before.sg.r0) * pl.group;
        }
        if (lane == 0 && pt.own + pt.tile < pl.tiles) pa_words(part)[pt.own + pt.tile] = word;      // (more than that: of starts without sense)
    }
    w.gs = w.ge = 0;
    w.first = -1;
    if (!w.own) {
        // the table of the first sequence that does not sit out
        w.gs = pt.sg.front; w.ge = pt.sg.front + pt.sg.first;
        w.sg.front = w.sg.first = 0;
        known[lane][0] = c0.r0; known[lane][1] = c0.m; known[lane][2] = c0.n;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (n <= 64) {
            const uint64_t in = __ballot(lane >= pl.n_groups + w.gs && lane < pl.n_groups + w.ge && c0.m > 0);
            if (in) w.sg.seq = __ffsll((unsigned long long)in) - 1 - pl.n_groups;
            if (!(in & __ballot(c0.n < pt.sg.count * 32)) && in == __ballot(lane >= pl.n_groups + w.gs && lane < pl.n_groups + w.ge)) w.first = pt.sg.count * 32;
        } else
            for (int b = w.gs; b < w.ge; ++b) if (page_seq(pl.sq, b).m) { w.sg.seq = b; break; }
    }
    w.e0 = pt.tile * rows; w.entries = pt.sg.m * pl.group;
    // what the tile's last query sees ends the walk
    const int tail = w.own ? pt.sg.front + max(((pt.sg.n + pa_div(pl, min(w.e0 + rows, w.entries) - 1)) >> 5) + 1 - pt.sg.first, 0) : pt.sg.count;
    w.beg = pt.split * pt.per; w.end = min(min(pt.sg.count, tail), w.beg + pt.per);
    return true;
}
// An entry of a table row by a scalar load (said so: taken for a vector load, it comes back behind all loads that are under way)
__device__ __forceinline__ int pa_page(const int32_t *row, int i)
{
    typedef const __attribute__((address_space(4))) int32_t *fixed;
    return ((fixed)(uintptr_t)row)[__builtin_amdgcn_readfirstlane(i)];
}
// The block that is v-th of a segment's
__device__ __forceinline__ int pa_place(const PaSeg &sg, int v) { return v < sg.front ? v : sg.first + v - sg.front; }

// Weights of a block's two score tiles for the row of this lane: x[e] = 2^(s qk - m), the reference and what is summed so far brought up to date.  whole: every
// row sees all of the block; else seen says which of the lane's eight positions its row sees.
template <typename T, int DT>
__device__ __forceinline__ void pa_weights(const PaPlan &pl, const f32x4 (&s)[2], float qk, int pos, int k0, bool held, bool whole, bool &far, float &m, float &l, f32x4 (&o)[DT],
                                           uint32_t &seen, float (&x)[8])
{
    const int g = (threadIdx.x & 63) >> 4;
    float bm;
    seen = 0xFFu;
    if (whole) {
        bm = fmaxf(fmaxf(s[0][0], s[0][1]), s[0][2]);
        bm = fmaxf(fmaxf(bm, s[0][3]), s[1][0]);
        bm = fmaxf(fmaxf(bm, s[1][1]), s[1][2]);
        bm = fmaxf(fmaxf(bm, s[1][3]) * qk, PA_LOW);
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
        bm = fmaxf(bm, seen ? PA_LOW : -INFINITY);
    }
    if (__ballot(bm - m > PA_TOP)) {
        const float mn = fmaxf(m, pa_across(bm)), turn = pa_exp2(m - mn);
        l *= turn;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] *= turn;
        m = mn;
        far |= __ballot(fabsf(mn) >= PA_FAR && mn > PA_LOW) != 0;
    }
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
}
// Weights as the second product's operand, two bf16: 16 bits
__device__ __forceinline__ void pa_pack(const float (&x)[8], uint4 &hi, uint4 &lo)
{
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t h = bf16_pair(x[2 * w], x[2 * w + 1]);
        (&hi.x)[w] = h;
        (&lo.x)[w] = bf16_pair(x[2 * w] - __uint_as_float(h << 16), x[2 * w + 1] - __uint_as_float(h & 0xFFFF0000u));
    }
}
// Zero times NaN is NaN: where a mask may hide an infinity or NaN from some row it is taken out of the values, and the rows that see one are counted.
// Takes them out of a unit; a bit for each.
__device__ __forceinline__ uint32_t pa_marks(uint4 &v, bf16_t)
{
    uint32_t marks = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t &u = (&v.x)[w];
        const uint32_t bad = pa_wild(u, bf16_t()) >> 15;
        u &= ~(bad * 0xFFFFu);
        marks |= ((bad | bad >> 15) & 3u) << (2 * w);
    }
    return marks;
}
__device__ __forceinline__ uint32_t pa_marks(uint4 &v, float)
{
    uint32_t marks = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t &u = (&v.x)[w];
        const uint32_t bad = pa_wild(u, float()) >> 31;
        u = bad ? 0u : u;
        marks |= bad << w;
    }
    return marks;
}
// What a row's sums are multiplied by: nothing where it has seen nothing, NaN where it has seen only scores that overflowed downwards
__device__ __forceinline__ float pa_norm(float m, float l) { return l != 0.f ? 1.f / l : m > PA_NONE ? NAN : 0.f; }
// NaN to the sums o (of a tile of dimensions whose units' marks are given) of the rows that see a marked value
template <typename T, int VU>
__device__ __forceinline__ void pa_taint(const uint32_t (&marks)[VU], uint32_t seen, f32x4 &o)
{
    f32x4 hits = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int a = 0; a < VU; ++a) {
        if constexpr (sizeof(T) == 2) {
            uint4 ones, vis;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                (&ones.x)[w] = ((marks[a] >> (2 * w) & 1) | (marks[a] >> (2 * w + 1) & 1) << 16) * 0x3F80u;
                (&vis.x)[w] = ((seen >> (2 * w) & 1) | (seen >> (2 * w + 1) & 1) << 16) * 0x3F80u;
            }
            hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(ones), as_b16(vis), hits, 0, 0, 0);
        } else {
#pragma unroll
            for (int w = 0; w < 4; ++w)
                hits = __builtin_amdgcn_mfma_f32_16x16x4f32(marks[a] >> w & 1 ? 1.f : 0.f, seen >> (4 * a + w) & 1 ? 1.f : 0.f, hits, 0, 0, 0);
        }
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) o[w] = hits[w] != 0.f ? NAN : o[w];
}
// A lane's units of a query
template <typename T, int KS> __device__ __forceinline__ void pa_query(const T *src, bool vec, uint4 (&qa)[KS])
{
    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = (4 * ks + ((threadIdx.x & 63) >> 4)) * E;
        if (vec) qa[ks] = *reinterpret_cast<const uint4 *>(src + d);
        else {
            T x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = src[d + e];
            qa[ks] = __builtin_bit_cast(uint4, x);
        }
    }
}

// l = sum 2^(s - m), O = sum 2^(s - m) v, with s in powers of two and a reference m that is at most 2^PA_TOP below the largest s: while no score is
// above that, a block costs 8 exponentials a lane and tile, their sum and a comparison beside its products.  bf16: probabilities go in as
// two bf16 (16 bits), which costs nothing where memory bounds.
// Up to 32 rows: a workgroup has 16 MT; its waves take the blocks in turn, each for all rows, so that a record goes straight to the registers of one wave.
// Memory bounds: 6.9 TB/s with every CU at it (8 x 16 queries of 32 heads of 128, fp32: 1 MB a workgroup in 37 us), but a workgroup's cut takes 2 us, its first records
// 2 to 3, its waves' sums 1 to 3: 29 us for 134 MB (one query, 4 k positions), 23 for 79 (16 queries behind a prefix of 14 k).
template <int HD, typename T, int MT>
__global__ __launch_bounds__(64 * PA_WAVES, HD <= 128 && HD * (int)sizeof(T) * MT <= 512 ? 2 : 1) void page_few_kernel(const T *__restrict__ q, int64_t ldq,
                                                                                                       const T *__restrict__ cache, PaPlan pl, float qk, T *__restrict__ out,
                                                                                                       int64_t ldo, int vec, float *__restrict__ part)
{
    using P = PaTile<HD, T>;
    constexpr int KS = P::KS, DT = P::DT, VU = P::VU, RECB = 64 * HD * (int)sizeof(T), CH = DT < 8 ? DT : 8, ROWS = 16 * MT;
    constexpr bool AHEAD = HD * (int)sizeof(T) * (MT + 3) <= 2048;       // the next block is requested while this one is worked on, where registers hold both
    __shared__ float m_all[PA_WAVES][MT][16], l_all[PA_WAVES][MT][16];
    __shared__ f32x4 o_slot[PA_WAVES][CH][64];
    __shared__ int32_t known[PA_WAVES][64][3];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const int head = blockIdx.x % (uint32_t)pl.heads, slot = blockIdx.x / (uint32_t)pl.heads;
    PaWork wk;
    if (!pa_work(pl, head, slot, known[wave], part, wk)) return;
    const PaSeg &sg = wk.sg;
    const bool own = wk.own, alone = wk.alone;
    const int32_t *pages_of = pl.sq.table + (int64_t)__builtin_amdgcn_readfirstlane(sg.seq) * pl.sq.width;
    const int e0 = wk.e0, entries = wk.entries, beg = wk.beg, end = wk.end, mts = (min(entries - e0, ROWS) + 15) >> 4;      // (tiles of 16 in use)
    auto place = [&](int v) { return pa_place(sg, v); };

    int at[MT], pos[MT];                                 // head of entry e0 + 16 mt + c, position of its row
    uint4 qa[MT][KS];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int e = min(e0 + 16 * mt + c, entries - 1), i = pa_div(pl, e), row = sg.r0 + i;
        at[mt] = e - i * pl.group;
        pos[mt] = own ? sg.n + i : row;
        pa_query<T, KS>(q + (int64_t)row * ldq + ((int64_t)head * pl.group + at[mt]) * HD, vec & 1, qa[mt]);
    }
    uint4 ka[2][KS], va[DT][VU];
    // The page of a block is looked up while the block before it is requested.
    const int sh = pl.sq.page_shift - 5;
    int64_t rec = -1;
    int id = 0;
    auto look = [&](int v) { id = pa_page(pages_of, place(min(v, end - 1)) >> sh); };
    auto fetch = [&](int v) {           // record of block v, its keys requested; behind the end nothing is read
        const int blk = place(min(v, end - 1));
        rec = (uint32_t)id < (uint32_t)pl.sq.n_pages ? (((int64_t)id * pl.heads + head) << sh) + (blk & ((1 << sh) - 1)) : -1;
        look(v + PA_WAVES);
        const auto b = mx_buffer((const uint8_t *)(cache + max(rec, (int64_t)0) * (64 * HD)), RECB);
        const int from = v < end && rec >= 0 ? P::k_lane(lane) : MX_OOB;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) ka[a][ks] = mx_load16(b, from, P::k_at(a, ks));
    };
    auto fetch_v = [&](int64_t r, bool in) {
        const auto b = mx_buffer((const uint8_t *)(cache + max(r, (int64_t)0) * (64 * HD)), RECB);
        const int from = in && r >= 0 ? P::v_lane(lane) : MX_OOB;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int a = 0; a < VU; ++a) va[t][a] = mx_load16(b, from, P::v_at(t, a));
    };
    int v = beg + wave;
    if (beg < end) look(v);
    if (AHEAD && beg < end) {
        fetch(v);
        fetch_v(rec, v < end);
    }
    int low = 0x7FFFFFFF;                       // the tile's first position
    if (!own) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) pos[mt] = pa_position(pl, known[wave], wk.gs, wk.ge, pos[mt]);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) low = min(low, pos[mt]);

    f32x4 o[MT][DT];
    float m[MT], l[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = PA_NONE; l[mt] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[mt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    bool far = false;
    for (; v < end; v += PA_WAVES) {
        const int k0 = place(v) * 32;
        if (!AHEAD) fetch(v);
        const int64_t now = rec;
        const bool held = now >= 0;
        f32x4 s[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            s[mt][0] = s[mt][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (mt && mt >= mts) continue;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int a = 0; a < 2; ++a) s[mt][a] = P::score(ka[a][ks], qa[mt][ks], s[mt][a]);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (AHEAD) fetch(v + PA_WAVES);
        else fetch_v(now, true);
        __builtin_amdgcn_sched_barrier(0);
        // does every row of the tile see all of the block?
        const bool whole = held && __ballot(!(k0 + 31 <= low)) == 0 && (pl.window == 0 || k0 + 31 < pl.sinks || (own && k0 > sg.n + pa_div(pl, min(e0 + ROWS, entries) - 1) - pl.window));
        uint4 ph[MT], plo[MT];
        f32x4 x32[MT][2];
        uint32_t seen[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            seen[mt] = 0u;
            if (mt && mt >= mts) continue;
            float x[8];
            pa_weights<T, DT>(pl, s[mt], qk, pos[mt], k0, held, whole, far, m[mt], l[mt], o[mt], seen[mt], x);
            if constexpr (sizeof(T) == 2) pa_pack(x, ph[mt], plo[mt]);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x32[mt][e >> 2][e & 3] = x[e];
            }
        }
        if (!whole) {
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
                    uint32_t marks[VU];
#pragma unroll
                    for (int a = 0; a < VU; ++a) {
                        asm("" : "+v"(va[t][a].x), "+v"(va[t][a].y), "+v"(va[t][a].z), "+v"(va[t][a].w));      // (worked out here: kept from above the marks of all would not fit)
                        marks[a] = pa_marks(va[t][a], T());
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) pa_taint<T, VU>(marks, seen[mt], o[mt][t]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt && mt >= mts) continue;
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    o[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(va[t][0]), as_b16(plo[mt]), o[mt][t], 0, 0, 0);
                    o[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(va[t][0]), as_b16(ph[mt]), o[mt][t], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int a = 0; a < VU; ++a)
#pragma unroll
                        for (int w = 0; w < 4; ++w) o[mt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(word(va[t][a], w), x32[mt][a][w], o[mt][t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (AHEAD) fetch_v(rec, v + PA_WAVES < end);
    }

    // ---- the waves of a workgroup, in wave order ----
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        l[mt] += __shfl_xor(l[mt], 16);
        l[mt] += __shfl_xor(l[mt], 32);
        if (g == 0) { m_all[wave][mt][c] = m[mt]; l_all[wave][mt][c] = l[mt]; }
    }
    __syncthreads();
    float *dst = part + 8 + 8 * (size_t)pl.tiles + ((size_t)head * pl.items + slot) * pa_record(ROWS, HD);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        if (mt && mt >= mts) break;
        float M = PA_NONE, den = 0.f;
#pragma unroll
        for (int w = 0; w < PA_WAVES; ++w) M = fmaxf(M, m_all[w][mt][c]);
#pragma unroll
        for (int w = 0; w < PA_WAVES; ++w) den += pa_exp2(m_all[w][mt][c] - M) * l_all[w][mt][c];
        const float turn = pa_exp2(m[mt] - M), norm = pa_norm(M, den);
        const int entry = e0 + 16 * mt + c, i = pa_div(pl, min(entry, entries - 1));
#pragma unroll
        for (int t0 = 0; t0 < DT; t0 += CH) {
            if (mt || t0) __syncthreads();
#pragma unroll
            for (int t = 0; t < CH; ++t) if (t0 + t < DT) o_slot[wave][t][lane] = o[mt][t0 + t] * turn;
            __syncthreads();
            for (int t = wave; t < CH && t0 + t < DT; t += PA_WAVES) {
                f32x4 a = o_slot[0][t][lane];
#pragma unroll
                for (int w = 1; w < PA_WAVES; ++w) a += o_slot[w][t][lane];
                const int d = (t0 + t) * 16 + g * 4;
                if (entry >= entries) continue;
                if (!alone) *reinterpret_cast<float4 *>(dst + (16 * mt + c) * HD + d) = make_float4(a[0], a[1], a[2], a[3]);
                else pa_out(out + (int64_t)(sg.r0 + i) * ldo + ((int64_t)head * pl.group + at[mt]) * HD + d, a * norm, vec & 2);
            }
        }
        if (!alone && wave == 0 && g == 0 && entry < entries) { dst[ROWS * HD + 16 * mt + c] = M; dst[ROWS * (HD + 1) + 16 * mt + c] = den; }
    }
}

// Many rows, bf16: a wave has 32 rows of its own, the four of a workgroup 128, and all four walk the same blocks, two at a time.  Records go from memory straight to LDS
// (no registers in between), each wave a quarter of each, while the step before is worked on; LDS holds two steps, so that one barrier a step is enough.
// K units of positions 16 .. 31 change places by 8 there: the sixteen lanes of a read then cover all 64 banks.  Here the products bound, so weights are one
// bf16 (8 bits, an error like that of the result's own rounding), and one more tile of values, all of them 1, gives their sums.
// Prompts of 2040 and 1446 tokens, 32/8 heads of 128: 63.6 us, 805 TFLOP/s of what the mask leaves; matrix units are busy 39 % of the time (two waves a SIMD hold 255
// registers each).  On the way (kernel under a tracer): records through registers 92 us (their copies to LDS, and spills whose reloads wait for the prefetches); a branch for each block's
// reference 80; without 74; 67 with this part first (see below).
template <int HD>
__global__ __launch_bounds__(64 * PA_WAVES, 2) void page_many_kernel(const bf16_t *__restrict__ q, int64_t ldq, const bf16_t *__restrict__ cache, PaPlan pl, float qk,
                                                                     bf16_t *__restrict__ out, int64_t ldo, int vec, float *__restrict__ part)
{
    typedef bf16_t T;
    using P = PaTile<HD, T>;
    constexpr int KS = P::KS, DT = P::DT, RECB = 64 * HD * 2, NL = RECB / (1024 * PA_WAVES), MT = 2, NB = 2, RW = 16 * MT, ROWS = RW * PA_WAVES;
    __shared__ __attribute__((aligned(16))) uint8_t even[NB * RECB], odd[NB * RECB];      // (two variables: a read of one does not wait for loads into the other)
    __shared__ uint8_t marks[2][NB][RECB / 32];             // of the values' units
    __shared__ int32_t wild[2][PA_WAVES];                   // a bit for each block: whether there are any
    __shared__ int32_t known[PA_WAVES][64][3];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    // (the last segments' last tiles first: of prompts these have the longest walks)
    const int head = blockIdx.x % (uint32_t)pl.heads, slot = pl.items - 1 - (int)(blockIdx.x / (uint32_t)pl.heads);
    PaWork wk;
    if (!pa_work(pl, head, slot, known[wave], part, wk)) return;
    const PaSeg &sg = wk.sg;
    const int32_t *pages_of = pl.sq.table + (int64_t)__builtin_amdgcn_readfirstlane(sg.seq) * pl.sq.width;
    const int e0 = wk.e0 + wave * RW, left = wk.entries - e0, beg = wk.beg, end = wk.end;       // (left <= 0: this wave only loads)
    const int high = sg.n + pa_div(pl, max(min(e0 + RW, wk.entries) - 1, 0)), first = wk.own ? sg.n + pa_div(pl, wk.e0) : wk.first;    // (own) the wave's last, the tile's first position

    // Steps n = 0, 1, .. have blocks beg + NB n ..; the pages of a step are looked up while the step before it is requested.
    const int sh = pl.sq.page_shift - 5, swap = wave < PA_WAVES / 2 ? (lane & 16) >> 1 : 0, from = wave * (RECB / PA_WAVES) + (lane ^ swap) * 16;
    const int steps = beg < end ? (end - beg + NB - 1) / NB : 0;
    int id[NB];
    uint32_t holds = 0;                         // bits NB (n % 2) ..: the blocks of step n that lie in the pool
    auto block = [&](int n, int i) { return pa_place(sg, min(beg + NB * n + i, end - 1)); };
    auto look = [&](int n) {
#pragma unroll
        for (int i = 0; i < NB; ++i) id[i] = pa_page(pages_of, block(n, i) >> sh);
    };
    auto request = [&](int n, uint8_t *to) {
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const bool ok = beg + NB * n + i < end && (uint32_t)id[i] < (uint32_t)pl.sq.n_pages;
            const int64_t rec = ok ? (((int64_t)id[i] * pl.heads + head) << sh) + (block(n, i) & ((1 << sh) - 1)) : 0;
            bits |= ok ? 1u << i : 0u;
            const auto b = mx_buffer((const uint8_t *)(cache + rec * (64 * HD)), RECB);
#pragma unroll
            for (int j = 0; j < NL; ++j)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void *)(to + i * RECB + wave * (RECB / PA_WAVES) + j * 1024), 16, from, j * 1024, 0, 0);
        }
        holds = (n & 1) ? (holds & 3u) | bits << NB : (holds & ~3u) | bits;
    };
    if (steps) {
        look(0);
        request(0, even);
        look(1);
    }
    int at[MT], pos[MT], low = 0x7FFFFFFF;
    uint4 qa[MT][KS];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int e = max(min(e0 + 16 * mt + c, wk.entries - 1), 0), i = pa_div(pl, e), row = sg.r0 + i;
        at[mt] = e - i * pl.group;
        pos[mt] = wk.own ? sg.n + i : pa_position(pl, known[wave], wk.gs, wk.ge, row);
        low = min(low, pos[mt]);
        pa_query<T, KS>(q + (int64_t)row * ldq + ((int64_t)head * pl.group + at[mt]) * HD, vec & 1, qa[mt]);
    }
    f32x4 o[MT][DT + 1];
    float m[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = PA_NONE;
#pragma unroll
        for (int t = 0; t <= DT; ++t) o[mt][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    bool far = false;
    // where a lane's units are in LDS
    const int k0at = 16 * (g * 32 + (PaOps<T>::position(0, c) ^ (c & 8))), k1at = k0at ^ 128, vat = P::v_lane(lane);
    // Steps that some row may not see all of: infinities and NaN leave the values, what is not in the pool becomes zeros
    auto clean = [&](int n, uint8_t *buf) {
        const uint32_t held = holds >> (NB * (n & 1)) & 3u;
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < NB; ++i)
            for (int u = wave * 64 + lane; u < RECB / 32; u += 64 * PA_WAVES) {
                uint4 *at = reinterpret_cast<uint4 *>(buf + i * RECB + RECB / 2) + u;
                uint4 x = *at;
                uint32_t mk = 0;
                if (held >> i & 1) mk = pa_marks(x, T());
                else x = make_uint4(0u, 0u, 0u, 0u);
                marks[n & 1][i][u] = (uint8_t)mk;
                if (mk || !(held >> i & 1)) *at = x;
                any |= __ballot(mk != 0) ? 1u << i : 0u;
            }
        wild[n & 1][wave] = any;
        __syncthreads();
    };
    auto work = [&](int n, const uint8_t *buf, bool edge) {           // edge: it has been cleaned
        int k0[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) k0[i] = block(n, i) * 32;
        const uint32_t held = holds >> (NB * (n & 1)) & 3u;
        // (blocks that none of the wave's rows sees are the last ones of a tile)
        if (left <= 0 || (wk.own && k0[0] > high)) return;
        f32x4 s[MT][2 * NB];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 2 * NB; ++i) s[mt][i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            uint4 ka[KS][2];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                ka[ks][0] = *reinterpret_cast<const uint4 *>(buf + i * RECB + k0at + P::k_at(0, ks));
                ka[ks][1] = *reinterpret_cast<const uint4 *>(buf + i * RECB + k1at + P::k_at(0, ks));
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    s[mt][2 * i] = P::score(ka[ks][0], qa[mt][ks], s[mt][2 * i]);
                    s[mt][2 * i + 1] = P::score(ka[ks][1], qa[mt][ks], s[mt][2 * i + 1]);
                }
        }
        uint4 va[DT];                           // of the first block; the second's are read during the first's products
#pragma unroll
        for (int t = 0; t < DT; ++t) va[t] = *reinterpret_cast<const uint4 *>(buf + vat + P::v_at(t, 0));
        const int last = k0[NB - 1] + 31;
        const bool whole = held == 3u && __ballot(!(last <= low)) == 0 && (pl.window == 0 || last < pl.sinks || (wk.own && k0[0] > high - pl.window));
        float least[MT] = {PA_LOW, PA_LOW};
        if (edge) {
            uint32_t seen[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                seen[mt] = 0xFFFFu;
                if (whole) continue;
                seen[mt] = 0;
#pragma unroll
                for (int e = 0; e < 8 * NB; ++e) {
                    const int key = k0[e >> 3] + PaOps<T>::position(e >> 2 & 1, 4 * g + (e & 3));
                    const bool see = ((held >> (e >> 3) & 1) != 0) & (key <= pos[mt]) & ((pl.window == 0) | (key > pos[mt] - pl.window) | (key < pl.sinks));
                    seen[mt] |= see ? 1u << e : 0u;
                    s[mt][e >> 2][e & 3] = see ? s[mt][e >> 2][e & 3] : -INFINITY;
                }
                least[mt] = seen[mt] ? PA_LOW : -INFINITY;
            }
            // (also where this wave's rows see all: the values were taken out for the others)
            if (wild[n & 1][0] | wild[n & 1][1] | wild[n & 1][2] | wild[n & 1][3]) {
                const int unit = P::v_lane(lane) >> 4;
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        uint32_t mk[1] = {marks[n & 1][i][unit + (P::v_at(t, 0) - RECB / 2) / 16]};
                        asm("" : "+v"(mk[0]));
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) pa_taint<T, 1>(mk, seen[mt] >> (8 * i), o[mt][t]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        }
        float bm[MT], ref[MT], mul = qk;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            bm[mt] = s[mt][0][0];
#pragma unroll
            for (int e = 1; e + 1 < 8 * NB; e += 2) bm[mt] = fmaxf(fmaxf(bm[mt], s[mt][e >> 2][e & 3]), s[mt][(e + 1) >> 2][(e + 1) & 3]);
            bm[mt] = fmaxf(fmaxf(bm[mt], s[mt][2 * NB - 1][3]) * qk, least[mt]);
        }
        if (__ballot((bm[0] - m[0] > PA_TOP) | (bm[1] - m[1] > PA_TOP))) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float mn = fmaxf(m[mt], pa_across(bm[mt])), turn = pa_exp2(m[mt] - mn);
#pragma unroll
                for (int t = 0; t <= DT; ++t) o[mt][t] *= turn;
                m[mt] = mn;
                far |= __ballot(fabsf(mn) >= PA_FAR && mn > PA_LOW) != 0;
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ref[mt] = m[mt];
        if (far) {                              // (scores rounded as the reference was: no fused multiply-add)
            mul = 1.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                ref[mt] = 0.f;
#pragma unroll
                for (int e = 0; e < 8 * NB; ++e) {
                    float w = s[mt][e >> 2][e & 3] * qk;
                    asm("" : "+v"(w));
                    s[mt][e >> 2][e & 3] = w - m[mt];
                }
            }
        }
        // No branches from here on: a block's weights are made while the products of the one before run.  This part goes before the other workgroup's loads and
        // scores on the same CU: 144 us against 153, 4000 tokens of 32 heads of 128.
        __builtin_amdgcn_s_setprio(1);
        const uint4 ones = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            uint4 ph[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = pa_exp2(fmaf(s[mt][2 * i + (e >> 2)][e & 3], mul, -ref[mt]));
#pragma unroll
                for (int w = 0; w < 4; ++w) (&ph[mt].x)[w] = bf16_pair(x[2 * w], x[2 * w + 1]);
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(va[t]), as_b16(ph[mt]), o[mt][t], 0, 0, 0);
                if (i + 1 < NB) va[t] = *reinterpret_cast<const uint4 *>(buf + (i + 1) * RECB + vat + P::v_at(t, 0));
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][DT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_b16(ones), as_b16(ph[mt]), o[mt][DT], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    auto step = [&](int n, uint8_t *now, uint8_t *next) {
        if (n + 1 < steps) {
            request(n + 1, next);
            look(n + 2);
        }
        const bool edge = pl.window || block(n, NB - 1) * 32 + 31 > first || (holds >> (NB * (n & 1)) & 3u) != 3u;
        if (edge) clean(n, now);
        work(n, now, edge);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // the loads into LDS
        __syncthreads();
    };
    if (steps) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        for (int n = 0; n < steps; n += 2) {
            step(n, even, odd);
            if (n + 1 < steps) step(n + 1, odd, even);
        }
    }
    float *dst = part + 8 + 8 * (size_t)pl.tiles + ((size_t)head * pl.items + slot) * pa_record(ROWS, HD);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const float l = o[mt][DT][0], norm = pa_norm(m[mt], l);
        const int r = wave * RW + 16 * mt + c, entry = wk.e0 + r;
        if (entry >= wk.entries) continue;
        if (wk.alone) {
            T *to = out + (int64_t)(sg.r0 + pa_div(pl, entry)) * ldo + ((int64_t)head * pl.group + at[mt]) * HD + 4 * g;
#pragma unroll
            for (int t = 0; t < DT; ++t) pa_out(to + 16 * t, o[mt][t] * norm, vec & 2);
        } else {
#pragma unroll
            for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4 *>(dst + r * HD + 16 * t + 4 * g) = o[mt][t];
            if (g == 0) { dst[ROWS * HD + r] = m[mt]; dst[ROWS * (HD + 1) + r] = l; }
        }
    }
}

// Joins the parts of rows that have several: those of their sequence's tile, then those of the prefix.  A workgroup takes 32 units (four values of a
// row) of an own tile at a time, PA_JOIN threads each: a thread takes every PA_JOIN-th part, then they meet in LDS in order.  4 us: a launch and three trips to memory in a row
// (8 to 11 where it worked the cut out again instead of reading the words).
#define PA_JOIN 8
#define PA_UNITS 32
template <typename T>
__global__ __launch_bounds__(PA_UNITS * PA_JOIN) void page_merge_kernel(const float *__restrict__ part, PaPlan pl, int hd, int chunks, T *__restrict__ out, int64_t ldo, int vec)
{
    __shared__ float red[PA_JOIN][2][PA_UNITS];
    __shared__ f32x4 acc[PA_JOIN][PA_UNITS];
    const int head = blockIdx.x % (uint32_t)pl.heads, rest = blockIdx.x / (uint32_t)pl.heads, own = rest / chunks;
    const PaWord w = (reinterpret_cast<const PaWord *>(part) + 1)[own];
    if (own >= *reinterpret_cast<const int32_t *>(part) || w.splits1 + w.splits2 < 2) return;                  // (no tile, or written already)
    const int rows = 1 << pl.rows_shift;
    const size_t rec = pa_record(rows, hd);
    const float *from = part + 8 + 8 * (size_t)pl.tiles + (size_t)head * pl.items * rec;
    const int x = threadIdx.x % PA_UNITS, y = threadIdx.x / PA_UNITS, units = min(rows, w.entries - w.tile * rows) * (hd / 4);
    const int base1 = w.base1 + w.tile * w.splits1, parts = w.splits1 + w.splits2;
    for (int u0 = rest % chunks * PA_UNITS; u0 < units; u0 += chunks * PA_UNITS) {
        const int u = u0 + x, lr = u / (hd / 4), d = u % (hd / 4) * 4, entry = w.tile * rows + lr;
        const bool live = u < units;
        const int e2 = entry + w.above, lr2 = e2 & (rows - 1), base2 = w.base2 + (e2 >> pl.rows_shift) * w.splits2;      // the entry's place in the prefix's segment
        float M = PA_NONE, den = 0.f;
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
        auto add = [&](float ms, float ls, const f32x4 &v) {
            const float Mn = fmaxf(M, ms), down = pa_exp2(M - Mn), downs = pa_exp2(ms - Mn);
            den = den * down + ls * downs;
            a = a * down + v * downs;
            M = Mn;
        };
        if (live) {
#pragma unroll 4
            for (int s = y; s < parts; s += PA_JOIN) {
                const bool first = s < w.splits1;
                const int r = first ? lr : lr2;
                const uint32_t slot = first ? base1 + s : base2 + s - w.splits1;
                if (slot >= (uint32_t)pl.items) continue;                   // (of starts or groups without sense)
                const float *src = from + (size_t)slot * rec;
                const float4 v = *reinterpret_cast<const float4 *>(src + r * hd + d);
                add(src[rows * hd + r], src[rows * (hd + 1) + r], (f32x4){v.x, v.y, v.z, v.w});
            }
        }
        red[y][0][x] = M; red[y][1][x] = den;
        acc[y][x] = a;
        __syncthreads();
        if (y == 0 && live) {
#pragma unroll
            for (int j = 1; j < PA_JOIN; ++j) add(red[j][0][x], red[j][1][x], acc[j][x]);
            const int i = pa_div(pl, entry), h = entry - i * pl.group;
            pa_out(out + (int64_t)(w.r0 + i) * ldo + ((int64_t)head * pl.group + h) * hd + d, a * pa_norm(M, den), vec & 2);
        }
        __syncthreads();
    }
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
    // Rows of a tile.  More rows read a record less often, fewer leave more workgroups; only token counts are known here, not lengths.  us in a graph, 16 / 32 / 128 rows:
    // 256 tokens of 32 heads 9.8 / 10.8 / 17.0; 512 tokens of 32/8 heads 17.8 / 16.1 / 20.7; 2 x 1000 tokens of 24 heads of 64
    // 37.7 / 32.5 / 30.8; prompts of 2040 and 1446, 32/8 heads 163 / 136 / 67.  A prefix is read by all rows of its group: 16 queries of 32/8 heads behind 14 k
    // positions 28 / 23 (16 / 32).
    const int64_t mean = (entries + n_seqs - 1) / n_seqs, most = n_groups ? std::max(mean, entries / n_groups) : mean;
    const int row = p->head_dim * (p->dtype ? 2 : 4);
    const bool many = p->dtype == 1 && p->head_dim <= 128 && most >= 64 && (entries >> 7) * p->n_kv_heads >= 256;
    const bool two = row <= 512 && ((n_groups && most > 16) || (entries >> 5) * p->n_kv_heads >= 384);
    pl->rows_shift = many ? 7 : two ? 5 : 4;
    // Splits where tiles are few, about as many as workgroups are resident (one query of 32 heads, 4 k positions, fp32: 32.7 with 512 splits, 35.4 with 384).  Whole tiles take part of
    // that room: 16 queries behind a prefix, tiles of 32 rows of heads of 128, bf16, of which 512 are resident too: 27.0 with 384, 31.5 with 512.  Windows of many rows lose by being cut:
    // 8 x 16 queries of 32 heads, 1.2 k positions, fp32 52 whole, 62 .. 68 cut.  Every segment has a last tile that is not full.  The bounds on tiles (320, 512) and the 8 blocks
    // of the shortest split stand on these alone.
    // Tables of up to 1024 positions are never cut, whatever the lengths: one sequence of 1 or 16 rows, 32 heads of 128, whole / cut: bf16 100 positions 6.1 / 7.9, 272 8.1 / 9.8, 688
    // 11.0 / 10.1, 1000 14.5 / 11.1; fp32 9.2 / 11.1, 14.5 / 14.3, 24.0 / 16.4, 29.6 / 17.6.  So whole walks of more than about 500 (bf16) or 300 positions lose.
    const int64_t own = (entries >> pl->rows_shift) + n_seqs, shared = n_groups ? (entries >> pl->rows_shift) + n_groups : 0;
    const int64_t nblk = ((int64_t)width * p->page + 31) / 32;
    const bool few = own * p->n_kv_heads < (mean > 64 ? 320 : 512);
    const int resident = row > 512 || p->head_dim > 128 || (row > 256 && pl->rows_shift == 5) ? 256 : row > 128 && pl->rows_shift == 5 ? 384 : 512;
    pl->slots = nblk <= 32 || !few ? 0 : std::max(1, resident / p->n_kv_heads);
    pl->least = 2 * PA_WAVES;
    pl->n_groups = n_groups;
    if ((own + shared + pl->slots) * p->n_kv_heads >= (int64_t)1 << 24) return SJD_EINVAL;
    pl->items = (int)(own + shared + pl->slots);
    pl->tiles = (int)own;
    pl->window = window;
    return SJD_OK;
}
static size_t pa_bytes(const PaPlan &pl, int hd)
{
    if (!pl.slots && !pl.n_groups) return 0;
    const size_t rows = (size_t)1 << pl.rows_shift;
    return (8 + 8 * (size_t)pl.tiles + (size_t)pl.items * pl.heads * rows * (hd + 2)) * sizeof(float);
}

template <int HD, typename T>
static void pa_launch(dim3 grid, hipStream_t s, const T *q, int64_t ldq, const T *cache, const PaPlan &pl, float qk, T *out, int64_t ldo, int vec, float *ws)
{
    if constexpr (sizeof(T) == 2 && HD <= 128) {
        if (pl.rows_shift == 7) {
            SJD_LAUNCH((page_many_kernel<HD>), grid, dim3(64 * PA_WAVES), 0, s, q, ldq, cache, pl, qk, out, ldo, vec, ws);
            return;
        }
    }
    constexpr int two = HD * (int)sizeof(T) <= 512 ? 2 : 1;
    if (pl.rows_shift == 4) SJD_LAUNCH((page_few_kernel<HD, T, 1>), grid, dim3(64 * PA_WAVES), 0, s, q, ldq, cache, pl, qk, out, ldo, vec, ws);
    else SJD_LAUNCH((page_few_kernel<HD, T, two>), grid, dim3(64 * PA_WAVES), 0, s, q, ldq, cache, pl, qk, out, ldo, vec, ws);
}

extern "C" int sjd_page_attention_workspace(const sjd_pages *pages, int32_t rows, int32_t n_seqs, int32_t n_groups, int32_t n_heads, int32_t width, size_t *bytes)
{
    if (!bytes) return SJD_EINVAL;
    PaPlan pl;
    SJD_TRY(pa_plan(pages, rows, n_seqs, n_groups, n_heads, width, 0, &pl));
    *bytes = pa_bytes(pl, pages->head_dim);
    if (n_groups) {                             // (with a window groups are not used)
        SJD_TRY(pa_plan(pages, rows, n_seqs, 0, n_heads, width, 0, &pl));
        *bytes = std::max(*bytes, pa_bytes(pl, pages->head_dim));
    }
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
    const bool join = pl.slots || pl.n_groups;
    const int vec = (mx_vec(q, ldq, dt) ? 1 : 0) | ((uintptr_t)out % (dt ? 8 : 16) == 0 && ldo % 4 == 0 ? 2 : 0);
    const float qk = scale * 1.4426950408889634f;
    float *ws = join ? (float *)workspace : nullptr;
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)(pl.items * pl.heads));
#define GO(HD) do { if (dt == 0) pa_launch<HD, float>(grid, s, (const float *)q, ldq, (const float *)cache, pl, qk, (float *)out, ldo, vec, ws); \
                    else pa_launch<HD, bf16_t>(grid, s, (const bf16_t *)q, ldq, (const bf16_t *)cache, pl, qk, (bf16_t *)out, ldo, vec, ws); } while (0)
    switch (hd) {
        case 32: GO(32); break;
        case 64: GO(64); break;
        case 96: GO(96); break;
        case 128: GO(128); break;
        default: GO(256); break;
    }
#undef GO
    HIP_TRY(hipGetLastError());
    if (join) {
        // (workgroups for tiles as full as they are on average: many hold one token)
        const int64_t full = std::min<int64_t>((int64_t)1 << pl.rows_shift, ((int64_t)rows * pl.group + n_seqs - 1) / n_seqs);
        const int64_t tiles = (int64_t)pl.tiles * pl.heads;
        const int chunks = (int)std::min((full * (hd / 4) + PA_UNITS - 1) / PA_UNITS, std::max<int64_t>(1, ((int64_t)1 << 23) / tiles));
        const dim3 mgrid((unsigned)(tiles * chunks));
        if (dt == 0) SJD_LAUNCH((page_merge_kernel<float>), mgrid, dim3(PA_UNITS * PA_JOIN), 0, s, (const float *)ws, pl, hd, chunks, (float *)out, ldo, vec);
        else SJD_LAUNCH((page_merge_kernel<bf16_t>), mgrid, dim3(PA_UNITS * PA_JOIN), 0, s, (const float *)ws, pl, hd, chunks, (bf16_t *)out, ldo, vec);
        HIP_TRY(hipGetLastError());
    }
    return SJD_OK;
}
