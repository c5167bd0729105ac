// The norms between two blocks of a decoder with the gate and the residual scale between them (see include/sjd.h).
#include "sjd_page.h"

// A row to a workgroup, in registers from the first sum to the last: a thread has NE groups of eight values, zeros behind the row.
// Two sums over the row, of x^2 and of h^2, each over a wave's lanes and then over the waves through LDS.  Memory bounds: 2048 rows of 4096, a gate a row, bf16
// 22.1 us, 117 MB at a copy's 5.1 TB/s (resid partly stays in the memory-side cache); one row 4.1 us, launch and the two sums.
// 2048 rows of 4095: 37 us.
#define BN_THREADS 256
__device__ __forceinline__ float bn_sum(float v, float *red)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}
// Value e of group n of this thread's: VEC (rows of whole units of 16 bytes): eight neighbours; else every 256th, so that lanes read neighbours
template <bool VEC> __device__ __forceinline__ int bn_column(int n, int e) { return VEC ? 8 * ((int)threadIdx.x + BN_THREADS * n) + e : (int)threadIdx.x + BN_THREADS * (8 * n + e); }
template <bool VEC, typename T> __device__ __forceinline__ void bn_load(const T *row, int n, int d, float (&v)[8])
{
    if (VEC) {
        if (bn_column<true>(n, 0) < d) mx_load8<T>(row, bn_column<true>(n, 0), d, true, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = bn_column<false>(n, e) < d ? one_get(row[bn_column<false>(n, e)]) : 0.f;
}
template <bool VEC, typename T> __device__ __forceinline__ void bn_store(T *row, int n, int d, const float (&v)[8])
{
    if (VEC) {
        if (bn_column<true>(n, 0) >= d) return;
        Eight<T> o;
        eight_set(o, v);
        eight_store(row + bn_column<true>(n, 0), o);
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e) if (bn_column<false>(n, e) < d) row[bn_column<false>(n, e)] = one_set<T>(v[e]);
}
template <typename T, int NE, bool VEC>
__global__ __launch_bounds__(BN_THREADS) void block_norm_kernel(const T *x, int64_t ldx, const float *__restrict__ post, const T *__restrict__ gate, int64_t ldg,
                                                                float scale, float *__restrict__ resid, int64_t ldr, const float *__restrict__ pre, float eps, int d, T *out, int64_t ldo)
{
    __shared__ float red[2][4];
    const int64_t row = blockIdx.x;
    x += row * ldx; resid += row * ldr; out += row * ldo;
    if (gate) gate += row * ldg;
    float a[NE][8], h[NE][8], g[NE][8];
#pragma unroll
    for (int n = 0; n < NE; ++n) {
        bn_load<VEC, T>(x, n, d, a[n]);
        bn_load<VEC, float>(resid, n, d, h[n]);
        if (gate) bn_load<VEC, T>(gate, n, d, g[n]);
    }
    if (post) {
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NE; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(a[n][e], a[n][e], sum);
        const float r = 1.f / sqrtf(bn_sum(sum, red[0]) / (float)d + eps);
#pragma unroll
        for (int n = 0; n < NE; ++n) {
            float w[8];
            bn_load<VEC, float>(post, n, d, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) a[n][e] = a[n][e] * r * w[e];
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int n = 0; n < NE; ++n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[n][e] += scale * (gate ? g[n][e] * a[n][e] : a[n][e]);
            if (bn_column<VEC>(n, e) < d) sum = fmaf(h[n][e], h[n][e], sum);
        }
        bn_store<VEC, float>(resid, n, d, h[n]);
    }
    if (!pre) return;
    const float r = 1.f / sqrtf(bn_sum(sum, red[1]) / (float)d + eps);
#pragma unroll
    for (int n = 0; n < NE; ++n) {
        float w[8];
        bn_load<VEC, float>(pre, n, d, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = h[n][e] * r * w[e];
        bn_store<VEC, T>(out, n, d, w);
    }
}

extern "C" int sjd_block_norm(int32_t dtype, const void *x, int64_t ldx, const float *post, const void *gate, int64_t ldg, float scale, float *resid, int64_t ldr,
                              const float *pre, float eps, int32_t rows, int32_t d, void *out, int64_t ldo, void *stream)
{
    if (!x || !resid || (dtype != 0 && dtype != 1) || rows < 1 || d < 1 || d > SJD_NORM_MAX_D || ldx < d || ldr < d) return SJD_EINVAL;
    if ((pre == nullptr) != (out == nullptr) || (out && ldo < d) || (gate && ldg != 0 && ldg < d)) return SJD_EINVAL;
    if (!(eps >= 0.f) || !(eps < 1e30f) || !(fabsf(scale) < 1e30f) || !mx_fits(rows, BN_THREADS)) return SJD_EINVAL;
    const bool vec = d % 8 == 0 && mx_vec(x, ldx, dtype) && mx_vec(resid, ldr, 0) && (!gate || mx_vec(gate, ldg, dtype)) && (!out || mx_vec(out, ldo, dtype)) &&
                    (uintptr_t)post % 16 == 0 && (uintptr_t)pre % 16 == 0;
    hipStream_t s = (hipStream_t)stream;
#define GO2(T, NE, VEC) SJD_LAUNCH((block_norm_kernel<T, NE, VEC>), dim3(rows), dim3(BN_THREADS), 0, s, (const T *)x, ldx, post, (const T *)gate, ldg, scale, resid, ldr, pre, eps, d, (T *)out, ldo)
#define GO1(T, NE) do { if (vec) GO2(T, NE, true); else GO2(T, NE, false); } while (0)
#define GO(NE) do { if (dtype == 0) GO1(float, NE); else GO1(bf16_t, NE); } while (0)
    const int eights = (d + 8 * BN_THREADS - 1) / (8 * BN_THREADS);
    if (eights <= 1) GO(1);
    else if (eights <= 2) GO(2);
    else if (eights <= 4) GO(4);
    else GO(8);
#undef GO
#undef GO1
#undef GO2
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}
