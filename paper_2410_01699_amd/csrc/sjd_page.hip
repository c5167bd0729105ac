// Rotary positions of rows of heads, and the append of new keys and values to a paged cache with the rotation on the way.
#include "sjd_page.h"

#include <algorithm>
#include <cmath>

// ---- frequencies (host) -----------------------------------------------------------------------
extern "C" int sjd_rope_turns(double theta, int32_t rot_dim, int32_t scaling, double factor, double original, double slow, double fast, uint64_t *turns)
{
    if (!turns || rot_dim < 2 || rot_dim % 2 || rot_dim > 256 || !(theta > 1.0) || !(theta <= 1e30)) return SJD_EINVAL;
    if (scaling < SJD_ROPE_PLAIN || scaling > SJD_ROPE_PARTS) return SJD_EINVAL;
    if (scaling != SJD_ROPE_PLAIN && (!(factor >= 1.0) || !(factor <= 1e6))) return SJD_EINVAL;
    if (scaling == SJD_ROPE_BASE && rot_dim == 2) return SJD_EINVAL;
    if (scaling == SJD_ROPE_PARTS && (!(original >= 1.0) || !(original <= 1e12) || !(slow > 0.0) || !(fast > slow) || !(fast <= 1e12))) return SJD_EINVAL;
    const double tau = 6.283185307179586476925;
    if (scaling == SJD_ROPE_BASE) theta *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(theta, -2.0 * i / rot_dim);
        if (scaling == SJD_ROPE_LINEAR) f /= factor;
        if (scaling == SJD_ROPE_PARTS) {
            const double keep = std::min(std::max((original * f / tau - slow) / (fast - slow), 0.0), 1.0);
            f = f * keep + f / factor * (1.0 - keep);
        }
        turns[i] = (uint64_t)std::nearbyint(std::ldexp(f / tau, 64));            // (f <= 1: below 2^62)
    }
    return SJD_OK;
}

// ---- rotation of rows ---------------------------------------------------------------------------
// A thread turns one unit (sixteen values, eight pairs) of NH heads of a row: angles are the same for all heads, so they are made once.  Memory bounds: 4001 rows of
// 40 heads of 128, 64 dimensions turned, bf16 16 us, 82 MB at a copy's 5.1 TB/s; one row 2.6 us, launch and latency.
template <typename T, int NH>
__global__ __launch_bounds__(256) void rope_kernel(const T *x, int64_t ldx, T *out, int64_t ldo, const int32_t *__restrict__ pos, uint32_t rows,
                                                   uint32_t heads, uint32_t hd, Rope ro)
{
    const uint32_t units = hd >> 4, sets = (heads + NH - 1) / NH, work = units * sets;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, row = id / work, at = id - row * work;
    if (row >= rows) return;
    const uint32_t h0 = at / units * NH, u = at % units;
    const int p = pos[row];
    const int ea = eight_at(ro, u, 0), eb = eight_at(ro, u, 1);
    const bool turns = (int)u < ro.rot >> 4;
    const T *src = x + row * ldx;
    Eight<T> a[NH], b[NH];
#pragma unroll
    for (int i = 0; i < NH; ++i) {
        const uint32_t h = min(h0 + i, heads - 1);
        a[i] = eight_load(src + h * hd + ea); b[i] = eight_load(src + h * hd + eb);
    }
    UnitAngles an;
    if (turns) unit_angles(ro, u, p, an);
    T *dst = out + row * ldo;
#pragma unroll
    for (int i = 0; i < NH; ++i) {
        if (h0 + i >= heads) break;
        if (turns) unit_turn(ro, an, a[i], b[i]);
        eight_store(dst + (h0 + i) * hd + ea, a[i]); eight_store(dst + (h0 + i) * hd + eb, b[i]);
    }
}
// Any rot and any alignment: a thread turns one pair of a row's heads, or copies two values that do not turn.
template <typename T>
__global__ __launch_bounds__(256) void rope_pairs_kernel(const T *x, int64_t ldx, T *out, int64_t ldo, const int32_t *__restrict__ pos, uint32_t rows,
                                                         uint32_t heads, uint32_t hd, Rope ro)
{
    const uint32_t half = hd >> 1, sets = (heads + 7) / 8, work = half * sets;
    const uint32_t id = blockIdx.x * 256 + threadIdx.x, row = id / work, at = id - row * work;
    if (row >= rows) return;
    const uint32_t h0 = at / half * 8, i = at % half;
    const bool turns = (int)i < ro.rot >> 1;
    int ea = 2 * i, eb = 2 * i + 1;
    float c = 1.f, s = 0.f;
    if (turns) {
        pair_at(ro, i, ea, eb);
        rope_angle(pos[row], ro.turns[i], ro.magnitude, c, s);
        s *= ro.sign;
    }
    const T *src = x + row * ldx;
    T *dst = out + row * ldo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t h = h0 + j;
        if (h >= heads) break;
        const T a = src[h * hd + ea], b = src[h * hd + eb];
        const float u = one_get(a), v = one_get(b);
        dst[h * hd + ea] = turns ? one_set<T>(fmaf(u, c, -v * s)) : a;
        dst[h * hd + eb] = turns ? one_set<T>(fmaf(v, c, u * s)) : b;
    }
}

extern "C" int sjd_rope(int32_t dtype, const void *x, int64_t ldx, void *out, int64_t ldo, const int32_t *pos, int32_t rows, int32_t n_heads, int32_t head_dim,
                        const uint64_t *turns, int32_t rot_dim, int32_t interleaved, float magnitude, int32_t inverse, void *stream)
{
    if (!x || !out || !pos || !turns || (dtype != 0 && dtype != 1) || rows < 1 || n_heads < 1 || n_heads > 2 * PAGE_MAX_HEADS) return SJD_EINVAL;
    if (head_dim < 2 || head_dim > 256 || head_dim % 2 || !rope_fits(turns, rot_dim, interleaved, magnitude, head_dim) || (inverse != 0 && inverse != 1)) return SJD_EINVAL;
    if (ldx < (int64_t)n_heads * head_dim || ldo < (int64_t)n_heads * head_dim) return SJD_EINVAL;
    const Rope ro = {turns, rot_dim, interleaved, magnitude, inverse ? -1.f : 1.f};
    const bool vec = mx_vec(x, ldx, dtype) && mx_vec(out, ldo, dtype) && rot_dim % 16 == 0 && head_dim % 16 == 0;
    const int64_t units = head_dim / 16;
    // (four heads a thread once there are threads enough for the chip)
    const bool many = vec && (int64_t)rows * n_heads * units >= 1 << 18;
    const int64_t threads = rows * (vec ? units * ((n_heads + (many ? 3 : 0)) / (many ? 4 : 1)) : (int64_t)head_dim / 2 * ((n_heads + 7) / 8));
    if (threads >= ((int64_t)1 << 32) - 256) return SJD_EINVAL;
    const dim3 grid((unsigned)((threads + 255) / 256));
    hipStream_t s = (hipStream_t)stream;
#define GO(T) do { \
        if (many) SJD_LAUNCH((rope_kernel<T, 4>), grid, dim3(256), 0, s, (const T *)x, ldx, (T *)out, ldo, pos, rows, n_heads, head_dim, ro); \
        else if (vec) SJD_LAUNCH((rope_kernel<T, 1>), grid, dim3(256), 0, s, (const T *)x, ldx, (T *)out, ldo, pos, rows, n_heads, head_dim, ro); \
        else SJD_LAUNCH((rope_pairs_kernel<T>), grid, dim3(256), 0, s, (const T *)x, ldx, (T *)out, ldo, pos, rows, n_heads, head_dim, ro); } while (0)
    if (dtype == 0) GO(float); else GO(bf16_t);
#undef GO
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}

// ---- append -----------------------------------------------------------------------------------
// The blocks of 32 positions that a call touches, sequence by sequence: item i is one of them.  Lanes look at 64 sequences at a time.
struct PageItem { PageSeq s; int32_t seq, blk; };
__device__ __forceinline__ bool page_item(const PageSeqs &sq, int want, PageItem &it)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < sq.n_seqs; b0 += 64) {
        const PageSeq s = b0 + lane < sq.n_seqs ? page_seq(sq, b0 + lane) : PageSeq{0, 0, 0};
        const int first = s.n >> 5, c = s.m ? ((s.n + s.m - 1) >> 5) - first + 1 : 0;
        const int incl = page_sum_up(c), begin = base + incl - c;
        const uint64_t hit = __ballot(want >= begin && want < begin + c);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            it.s = {page_lane(s.r0, l), page_lane(s.m, l), page_lane(s.n, l)};
            it.seq = b0 + l;
            it.blk = page_lane(first, l) + want - page_lane(begin, l);
            return true;
        }
        base += page_lane(incl, 63);
    }
    return false;
}

// A workgroup takes the new rows of one block of a sequence: of one cache head its keys (turned) and values, through LDS into the record's order,
// or of NH query heads the turned rows.  vec: rows of 16-byte units whose pairs lie in units; else values one by one.
// 4791 rows of prompts, 32/8 heads of 128, bf16: 27 us, 118 MB at 4.4 TB/s (a copy: 5.1); a workgroup loads, turns and stores one after the other.  Windows of 16 for 8
// sequences, 32 heads, fp32: 7 us, four trips to memory in a row (lengths, page, rows, records).
template <int HD, typename T, int NH>
__global__ __launch_bounds__(256) void page_append_kernel(PageSeqs sq, const T *q, int64_t ldq, T *q_out, int64_t ldqo, const T *__restrict__ k,
                                                          const T *__restrict__ v, int64_t ld, int heads, int kv, int sets, Rope ro, int vec, T *__restrict__ cache)
{
    constexpr int PITCH = HD + 16 / (int)sizeof(T), UNITS = HD / 16, E = 16 / (int)sizeof(T), WORK = 32 * UNITS;
    __shared__ __attribute__((aligned(16))) T tile[2][32 * PITCH];
    const int y = (int)(blockIdx.x % (uint32_t)sets);
    PageItem it;
    if (!page_item(sq, (int)(blockIdx.x / (uint32_t)sets), it)) return;
    const PageSeq s = it.s;
    const int p0 = it.blk * 32, lo = max(s.n - p0, 0), hi = min(s.n + s.m - p0, 32);       // positions [lo, hi) of the block are new
    const int64_t row0 = (int64_t)s.r0 + p0 - s.n;                                        // row of the block's first position (may lie before the rows)
    const int tid = threadIdx.x;
    if (y >= kv) {
        const int h0 = (y - kv) * NH;
        if (vec) {
            for (int w = lo * UNITS + tid; w < hi * UNITS; w += 256) {
                const int p = w / UNITS, u = w % UNITS, ea = eight_at(ro, u, 0), eb = eight_at(ro, u, 1);
                const T *src = q + (row0 + p) * ldq;
                T *dst = q_out + (row0 + p) * ldqo;
                Eight<T> a[NH], b[NH];
#pragma unroll
                for (int i = 0; i < NH; ++i) {
                    const int h = min(h0 + i, heads - 1);
                    a[i] = eight_load(src + h * HD + ea); b[i] = eight_load(src + h * HD + eb);
                }
                UnitAngles an;
                const bool turns = u < ro.rot >> 4;
                if (turns) unit_angles(ro, u, p0 + p, an);
#pragma unroll
                for (int i = 0; i < NH; ++i) {
                    if (h0 + i >= heads) break;
                    if (turns) unit_turn(ro, an, a[i], b[i]);
                    eight_store(dst + (h0 + i) * HD + ea, a[i]); eight_store(dst + (h0 + i) * HD + eb, b[i]);
                }
            }
        } else {
            // (four pairs' values are requested before the first is used)
            for (int w0 = lo * (HD / 2) + tid; w0 < hi * (HD / 2); w0 += 4 * 256) {
                T a[4][NH], b[4][NH];
                int ea[4], eb[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const int w = min(w0 + z * 256, hi * (HD / 2) - 1), p = w / (HD / 2), i = w % (HD / 2);
                    ea[z] = 2 * i; eb[z] = 2 * i + 1;
                    if (i < ro.rot >> 1) pair_at(ro, i, ea[z], eb[z]);
#pragma unroll
                    for (int j = 0; j < NH; ++j) {
                        const T *src = q + (row0 + p) * ldq + min(h0 + j, heads - 1) * HD;
                        a[z][j] = src[ea[z]]; b[z][j] = src[eb[z]];
                    }
                }
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const int w = w0 + z * 256, p = w / (HD / 2), i = w % (HD / 2);
                    if (w >= hi * (HD / 2)) break;
                    const bool turns = i < ro.rot >> 1;
                    float c = 1.f, sn = 0.f;
                    if (turns) rope_angle(p0 + p, ro.turns[i], ro.magnitude, c, sn);
#pragma unroll
                    for (int j = 0; j < NH; ++j) {
                        if (h0 + j >= heads) break;
                        T *dst = q_out + (row0 + p) * ldqo + (h0 + j) * HD;
                        const T x = a[z][j], y = b[z][j];
                        dst[ea[z]] = turns ? one_set<T>(fmaf(one_get(x), c, -one_get(y) * sn)) : x;
                        dst[eb[z]] = turns ? one_set<T>(fmaf(one_get(y), c, one_get(x) * sn)) : y;
                    }
                }
            }
        }
        return;
    }
    const int64_t rec = page_record(sq, sq.table + (int64_t)it.seq * sq.width, it.blk, y, kv);
    if (rec < 0) return;
    if (vec) {
#pragma unroll
        for (int w0 = 0; w0 < WORK; w0 += 256) {
            const int w = w0 + tid, p = w / UNITS, u = w % UNITS, ea = eight_at(ro, u, 0), eb = eight_at(ro, u, 1);
            if (p >= 32 || p < lo || p >= hi) continue;
            const T *ks = k + (row0 + p) * ld + y * HD, *vs = v + (row0 + p) * ld + y * HD;
            Eight<T> a = eight_load(ks + ea), b = eight_load(ks + eb);
            const Eight<T> c = eight_load(vs + 16 * u), d = eight_load(vs + 16 * u + 8);
            if (u < ro.rot >> 4) {
                UnitAngles an;
                unit_angles(ro, u, p0 + p, an);
                unit_turn(ro, an, a, b);
            }
            eight_store(&tile[0][p * PITCH + ea], a); eight_store(&tile[0][p * PITCH + eb], b);
            eight_store(&tile[1][p * PITCH + 16 * u], c); eight_store(&tile[1][p * PITCH + 16 * u + 8], d);
        }
    } else {
#pragma unroll 4
        for (int w = lo * (HD / 2) + tid; w < hi * (HD / 2); w += 256) {
            const int p = w / (HD / 2), i = w % (HD / 2);
            const T *ks = k + (row0 + p) * ld + y * HD, *vs = v + (row0 + p) * ld + y * HD;
            int ea = 2 * i, eb = 2 * i + 1;
            tile[1][p * PITCH + ea] = vs[ea]; tile[1][p * PITCH + eb] = vs[eb];
            T a, b;
            if (i < ro.rot >> 1) {
                pair_at(ro, i, ea, eb);
                float c, sn;
                rope_angle(p0 + p, ro.turns[i], ro.magnitude, c, sn);
                const float x = one_get(ks[ea]), z = one_get(ks[eb]);
                a = one_set<T>(fmaf(x, c, -z * sn)); b = one_set<T>(fmaf(z, c, x * sn));
            } else { a = ks[ea]; b = ks[eb]; }
            tile[0][p * PITCH + ea] = a; tile[0][p * PITCH + eb] = b;
        }
    }
    __syncthreads();
    T *dst = cache + rec * (64 * HD);
#pragma unroll
    for (int w = tid; w < 32 * HD / E; w += 256) {                     // keys: unit (w / 32, position w % 32)
        const int p = w & 31;
        if (p >= lo && p < hi) *reinterpret_cast<uint4 *>(dst + w * E) = *reinterpret_cast<const uint4 *>(&tile[0][p * PITCH + (w >> 5) * E]);
    }
#pragma unroll
    for (int w = tid; w < 32 * HD / E; w += 256) {                     // values: unit (dimension, E positions)
        const int d = (w / (32 * (32 / E))) * 32 + (w & 31), u = (w >> 5) & (32 / E - 1);
        T x[E];
        bool all = true;
        int at[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            at[e] = E == 8 ? (u >> 1) * 16 + (e >> 2) * 8 + (u & 1) * 4 + (e & 3) : u * 4 + e;
            all &= at[e] >= lo && at[e] < hi;
            x[e] = tile[1][at[e] * PITCH + d];
        }
        T *to = dst + 32 * HD + w * E;
        if (all) {
            uint4 o;
            if (E == 8) o = make_uint4((uint32_t)x[0] | (uint32_t)x[1] << 16, (uint32_t)x[2] | (uint32_t)x[3] << 16, (uint32_t)x[E - 4] | (uint32_t)x[E - 3] << 16,
                                       (uint32_t)x[E - 2] | (uint32_t)x[E - 1] << 16);
            else o = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
            *reinterpret_cast<uint4 *>(to) = o;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (at[e] >= lo && at[e] < hi) to[e] = x[e];
        }
    }
}

extern "C" int sjd_page_append(const sjd_pages *pages, const void *q, int64_t ldq, int32_t n_heads, void *q_out, int64_t ldqo, const void *k, const void *v, int64_t ld,
                               int32_t rows, const int32_t *start, const int32_t *len, int32_t n_seqs, const int32_t *table, int32_t width, const uint64_t *turns,
                               int32_t rot_dim, int32_t interleaved, float magnitude, void *cache, void *stream)
{
    PageSeqs sq;
    if (!page_shape(pages) || !page_seqs(pages, start, len, table, width, n_seqs, rows, &sq)) return SJD_EINVAL;
    const int hd = pages->head_dim, kv = pages->n_kv_heads, dt = pages->dtype;
    if (!k || !v || !cache || !mx_aligned(cache) || ld < (int64_t)kv * hd || !rope_fits(turns, rot_dim, interleaved, magnitude, hd)) return SJD_EINVAL;
    if ((q == nullptr) != (q_out == nullptr)) return SJD_EINVAL;
    if (q && (!turns || n_heads < 1 || n_heads > PAGE_MAX_HEADS || ldq < (int64_t)n_heads * hd || ldqo < (int64_t)n_heads * hd)) return SJD_EINVAL;
    const Rope ro = {turns, rot_dim, interleaved, magnitude, 1.f};
    const int vec = mx_vec(k, ld, dt) && mx_vec(v, ld, dt) && rot_dim % 16 == 0 && (!q || (mx_vec(q, ldq, dt) && mx_vec(q_out, ldqo, dt)));
    const int64_t items = (int64_t)rows / 32 + 2 * (int64_t)n_seqs;                 // (a sequence's new tokens touch at most m / 32 + 2 blocks)
    // (two query heads a workgroup, whose angles are made once, where there are workgroups enough for the chip: six prompts of up to 1000 tokens, 32 heads of 128,
    // 27.0 us, 28.9 with one and 29.8 with four)
    const bool many = q && items * n_heads >= 2048;
    const int sets = kv + (q ? (n_heads + (many ? 1 : 0)) / (many ? 2 : 1) : 0);
    if (!mx_fits(items * sets, 256)) return SJD_EINVAL;
    const dim3 grid((unsigned)(items * sets));
    hipStream_t s = (hipStream_t)stream;
#define GO2(HD, T, NH) SJD_LAUNCH((page_append_kernel<HD, T, NH>), grid, dim3(256), 0, s, sq, (const T *)q, ldq, (T *)q_out, ldqo, (const T *)k, (const T *)v, ld, n_heads, kv, sets, ro, vec, (T *)cache)
#define GO1(HD, T) do { if (many) GO2(HD, T, 2); else GO2(HD, T, 1); } while (0)
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
#undef GO2
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}
