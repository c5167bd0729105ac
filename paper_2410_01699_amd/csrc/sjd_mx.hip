// Writers of microscaled rows: quantisation (of x, or of SiLU(x) * up), RMSNorm with the residual's addition, weights.
//
// A quad of lanes holds a block of 32 values, eight each: two lane exchanges give the block's scale, a lane stores its own
// eight codes.  All three move bytes and nothing else: what bounds them is memory, or the latency of one pass where rows are few.
#include "sjd_mx.h"

#include <algorithm>

// ---- quantisation ---------------------------------------------------------------------------
// A thread has eight values of a row; rows shorter than 2048 share a workgroup.  SiLU(gate) * up of 128 fp32 rows of 11008: 4.7 us, 12.7 MB at
// 2.7 TB/s: the launch and the latency of its one pass.
template <typename T, int FMT, bool GATED>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T *__restrict__ x, const T *__restrict__ up, int64_t ld, int rows, int K,
                                                          int Kp, int tx, int vec, uint8_t *__restrict__ codes,
                                                          uint8_t *__restrict__ scales)
{
    const int ty = 256 / tx;
    const int64_t row = (int64_t)blockIdx.x * ty + threadIdx.x / tx;
    const int c = ((int)blockIdx.y * tx + threadIdx.x % tx) * 8;
    if (row >= rows || c >= Kp) return;            // (whole quads: tx and Kp / 8 are multiples of 16)
    float v[8];
    mx_load8<T>(x + row * ld, c, K, vec, v);
    if (GATED) {
        float u[8];
        mx_load8<T>(up + row * ld, c, K, vec, u);
        float low = v[0], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            low = fminf(low, v[i]);
            y[i] = v[i] / (1.f + expf(-v[i])) * u[i];
        }
        // Below -80 the sigmoid is e^v to fp32, which ends at -87 (-103 as a subnormal) though the product with u need not: its two halves go
        // to one factor each.
        if (low < -80.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] < -80.f) {
                    const float h = expf(0.5f * v[i]);
                    y[i] = v[i] * h * (h * u[i]);
                }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = y[i];
    }
    uint2 q;
    const int byte = mx_quantise8<FMT>(v, q);
    if (FMT == SJD_MX8) *reinterpret_cast<uint2 *>(codes + (size_t)row * Kp + c) = q;
    else *reinterpret_cast<uint32_t *>(codes + (size_t)row * (Kp / 2) + c / 2) = q.x;
    if ((threadIdx.x & 3) == 0) scales[(size_t)row * (Kp / 32) + c / 32] = (uint8_t)byte;
}

extern "C" int sjd_mx_quantize(int32_t format, int32_t dtype, const void *x, const void *up, int64_t ld, int32_t rows, int32_t K,
                               uint8_t *codes, uint8_t *scales, void *stream)
{
    if (!x || !codes || !scales || rows < 1 || K < 1 || K > SJD_MX_MAX_K || ld < K) return SJD_EINVAL;
    if ((format != SJD_MX8 && format != SJD_MX4) || (dtype != 0 && dtype != 1)) return SJD_EINVAL;
    if (!mx_aligned(codes) || !mx_aligned(scales)) return SJD_EINVAL;
    const int Kp = mx_up(K, 128);
    int tx = 16;
    while (tx < 256 && tx * 8 < Kp) tx *= 2;
    const int64_t groups = ((int64_t)rows + 256 / tx - 1) / (256 / tx);
    if (!mx_fits(groups, 256)) return SJD_EINVAL;
    const dim3 grid((unsigned)groups, (unsigned)((Kp / 8 + tx - 1) / tx));
    const int vec = mx_vec(x, ld, dtype) && (!up || mx_vec(up, ld, dtype));
    hipStream_t s = (hipStream_t)stream;
#define GO(T, F, G) SJD_LAUNCH((mx_quantize_kernel<T, F, G>), grid, dim3(256), 0, s, (const T *)x, (const T *)up, ld, rows, K, Kp, tx, vec, codes, scales)
#define GO2(T, F) do { if (up) GO(T, F, true); else GO(T, F, false); } while (0)
    if (dtype == 0) { if (format == SJD_MX8) GO2(float, SJD_MX8); else GO2(float, SJD_MX4); }
    else { if (format == SJD_MX8) GO2(bf16_t, SJD_MX8); else GO2(bf16_t, SJD_MX4); }
#undef GO2
#undef GO
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}

// ---- RMSNorm --------------------------------------------------------------------------------
// One workgroup per row; a thread holds its eight values of h from the sum of squares to the codes, and what rows of more than 8192 have
// beyond that is read again from where it was kept.
// One fp32 row of 4096 3 us, the launch and one pass' latency; 2048 bf16 rows 18.7 us, 92 MB at a copy's rate.
template <typename T, int FMT>
__global__ __launch_bounds__(1024) void mx_rmsnorm_kernel(const T *__restrict__ x, int64_t ldx, float *__restrict__ resid, int64_t ldr,
                                                          const float *__restrict__ gain, float eps, int d, int dp, int vx, int vr, int vg,
                                                          uint8_t *__restrict__ codes, uint8_t *__restrict__ scales)
{
    __shared__ float part[16];
    const int64_t row = blockIdx.x;
    const int step = blockDim.x * 8;
    const T *xr = x ? x + row * ldx : nullptr;
    float *rr = resid ? resid + row * ldr : nullptr;
    float h[8], ss = 0.f;
    auto fetch = [&](int c, float (&v)[8], bool keep) {
        if (rr) mx_load8<float>(rr, c, d, vr, v);
        if (xr && (keep || !rr)) {
            float a[8];
            mx_load8<T>(xr, c, d, vx, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = rr ? v[i] + a[i] : a[i];
            if (rr) {
                if (vr && c + 8 <= d) {
                    reinterpret_cast<float4 *>(rr + c)[0] = make_float4(v[0], v[1], v[2], v[3]);
                    reinterpret_cast<float4 *>(rr + c)[1] = make_float4(v[4], v[5], v[6], v[7]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (c + i < d) rr[c + i] = v[i];
                }
            }
        }
    };
    const int c0 = threadIdx.x * 8;
    if (c0 < dp) {
        fetch(c0, h, true);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(h[i], h[i], ss);
    }
    for (int c = c0 + step; c < dp; c += step) {
        float v[8];
        fetch(c, v, true);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) ss += __shfl_xor(ss, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
    __syncthreads();
    float sum = 0.f;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) sum += part[w];
    const float r = 1.f / sqrtf(sum / (float)d + eps);
    auto emit = [&](int c, const float (&v)[8]) {
        float y[8], gn[8];
        mx_load8<float>(gain, c, d, vg, gn);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[i] * r * gn[i];
        if (c + 8 > d) {                       // (what lies behind the row is zero whatever the row holds)
#pragma unroll
            for (int i = 0; i < 8; ++i) if (c + i >= d) y[i] = 0.f;
        }
        uint2 q;
        const int byte = mx_quantise8<FMT>(y, q);
        if (FMT == SJD_MX8) *reinterpret_cast<uint2 *>(codes + (size_t)row * dp + c) = q;
        else *reinterpret_cast<uint32_t *>(codes + (size_t)row * (dp / 2) + c / 2) = q.x;
        if ((threadIdx.x & 3) == 0) scales[(size_t)row * (dp / 32) + c / 32] = (uint8_t)byte;
    };
    if (c0 < dp) emit(c0, h);
    for (int c = c0 + step; c < dp; c += step) {
        float v[8];
        fetch(c, v, false);
        emit(c, v);
    }
}

extern "C" int sjd_mx_rmsnorm(int32_t format, int32_t dtype, const void *x, int64_t ldx, float *resid, int64_t ldr, const float *gain,
                              float eps, int32_t rows, int32_t d, uint8_t *codes, uint8_t *scales, void *stream)
{
    if ((!x && !resid) || !gain || !codes || !scales || rows < 1 || d < 1 || d > SJD_MX_MAX_K || !(eps >= 0.f)) return SJD_EINVAL;
    if ((x && ldx < d) || (resid && ldr < d)) return SJD_EINVAL;
    if ((format != SJD_MX8 && format != SJD_MX4) || (x && dtype != 0 && dtype != 1)) return SJD_EINVAL;
    if (!mx_aligned(codes) || !mx_aligned(scales)) return SJD_EINVAL;
    const int dp = mx_up(d, 128);
    const int threads = std::min(1024, mx_up(dp / 8, 64));
    if (!mx_fits(rows, threads)) return SJD_EINVAL;
    const int vx = x && mx_vec(x, ldx, dtype), vr = resid && mx_vec(resid, ldr, 0), vg = mx_aligned(gain);
    hipStream_t s = (hipStream_t)stream;
#define GO(T, F) SJD_LAUNCH((mx_rmsnorm_kernel<T, F>), dim3(rows), dim3(threads), 0, s, (const T *)x, ldx, resid, ldr, gain, eps, d, dp, vx, vr, vg, codes, scales)
    if (!x || dtype == 0) { if (format == SJD_MX8) GO(float, SJD_MX8); else GO(float, SJD_MX4); }
    else { if (format == SJD_MX8) GO(bf16_t, SJD_MX8); else GO(bf16_t, SJD_MX4); }
#undef GO
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}

// ---- weights --------------------------------------------------------------------------------
// A workgroup makes one record: a wave reads a feature's 512 values (eight a lane) at a time, the codes meet in LDS in the record's
// order and leave as whole lines.  22016 bf16 rows of 4096: 47 us, 228 MB at a copy's rate.
template <typename T>
__global__ __launch_bounds__(256) void mx_weights_kernel(const T *__restrict__ w, int64_t ld, int N, int K, int groups, int vec,
                                                         uint8_t *__restrict__ packed)
{
    __shared__ uint4 rec[MX_REC / 16];
    uint8_t *r = reinterpret_cast<uint8_t *>(rec);
    const int g = (int)(blockIdx.x % (unsigned)groups), t = (int)(blockIdx.x / (unsigned)groups);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t n = (int64_t)t * 16 + wave * 4 + i;
        if (n < N) mx_load8<T>(w + n * ld, g * MX_GROUP + lane * 8, K, vec, v[i]);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
    const int b = lane >> 2, s = b >> 2, q = b & 3;        // block of the lane inside the 512 values
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int f = wave * 4 + i;
        uint2 code;
        const int byte = mx_quantise8<SJD_MX4>(v[i], code);
        *reinterpret_cast<uint32_t *>(r + s * 1024 + (q * 16 + f) * 16 + (lane & 3) * 4) = code.x;
        if ((lane & 3) == 0) r[4096 + (q * 16 + f) * 4 + s] = (uint8_t)byte;
    }
    __syncthreads();
    uint4 *dst = reinterpret_cast<uint4 *>(packed + (size_t)blockIdx.x * MX_REC);
    for (int i = threadIdx.x; i < MX_REC / 16; i += 256) dst[i] = rec[i];
}

extern "C" int sjd_mx_weights_bytes(int32_t N, int32_t K, size_t *bytes)
{
    if (!bytes || N < 1 || K < 1 || K > SJD_MX_MAX_K) return SJD_EINVAL;
    *bytes = (size_t)(((int64_t)N + 15) / 16) * mx_groups(K) * MX_REC;
    return SJD_OK;
}

extern "C" int sjd_mx_weights(int32_t dtype, const void *W, int64_t ld, int32_t N, int32_t K, uint8_t *packed, void *stream)
{
    if (!W || !packed || N < 1 || K < 1 || K > SJD_MX_MAX_K || ld < K || (dtype != 0 && dtype != 1) || !mx_aligned(packed)) return SJD_EINVAL;
    const int64_t grid = (((int64_t)N + 15) / 16) * mx_groups(K);
    if (!mx_fits(grid, 256)) return SJD_EINVAL;
    const int vec = mx_vec(W, ld, dtype);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == 0) SJD_LAUNCH((mx_weights_kernel<float>), dim3((unsigned)grid), dim3(256), 0, s, (const float *)W, ld, N, K, mx_groups(K), vec, packed);
    else SJD_LAUNCH((mx_weights_kernel<bf16_t>), dim3((unsigned)grid), dim3(256), 0, s, (const bf16_t *)W, ld, N, K, mx_groups(K), vec, packed);
    HIP_TRY(hipGetLastError());
    return SJD_OK;
}
