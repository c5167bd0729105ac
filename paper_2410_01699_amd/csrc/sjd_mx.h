// Microscaled formats (see include/sjd.h): device helpers shared by the operators that write and read them.
#pragma once
#include "sjd_internal.h"

#define MX_REC 4352                      // bytes of a record of packed weights: 16 features x 512 values and their scales
#define MX_GROUP 512                     // values of a row in one record

__host__ __device__ __forceinline__ int mx_up(int n, int m) { return (int)(((int64_t)n + m - 1) / m * m); }
__host__ __device__ __forceinline__ int mx_groups(int K) { return (int)(((int64_t)K + MX_GROUP - 1) / MX_GROUP); }

// 2^(byte - 127); byte 0 is 2^-127, a subnormal
__device__ __forceinline__ float mx_pow2(int byte) { return __uint_as_float(byte > 0 ? (uint32_t)byte << 23 : 1u << 22); }

// Bits of |v| if v is finite, else 0: the largest of them gives a block's scale (order of bits = order of magnitudes).
__device__ __forceinline__ uint32_t mx_finite_bits(float v)
{
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}
// Scale byte from those bits.  448 = 1.75 * 2^8 and 6 = 1.5 * 2^2: the power of two follows from the exponent, one more where the
// mantissa is above the format's.  Subnormal magnitudes come out negative and take byte 0.
template <int FMT> __device__ __forceinline__ int mx_scale_byte(uint32_t amax)
{
    constexpr int top = FMT == SJD_MX8 ? 8 : 2;
    constexpr uint32_t mant = FMT == SJD_MX8 ? 0x600000u : 0x400000u;
    return max((int)(amax >> 23) - top + ((amax & 0x7FFFFFu) > mant ? 1 : 0), 0);
}
// E4M3 codes of four values times inv (= 2^(127 - byte), exact), non-finite values as 0x7F
__device__ __forceinline__ uint32_t mx_e4m3x4(float a, float b, float c, float d, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
    uint32_t u = (uint32_t)w;
    // (the conversion keeps a NaN's sign and takes infinities to 0x7F | sign or to 448, by a mode bit)
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((__float_as_uint(v[i]) & 0x7F800000u) == 0x7F800000u) u = (u & ~(0xFFu << (8 * i))) | (0x7Fu << (8 * i));
    return u;
}
// E2M1 codes of eight finite values over 2^(byte - 127)
__device__ __forceinline__ uint32_t mx_e2m1x8(const float (&v)[8], float scale)
{
    uint32_t u = 0;
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[0], v[1], scale, 0);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[2], v[3], scale, 1);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[4], v[5], scale, 2);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[6], v[7], scale, 3);
    return u;
}

// Eight consecutive values of a row of `K`, from column c (a multiple of 8), as fp32; behind K zeros.  vec: the rows are 16-byte aligned.
template <typename T> __device__ __forceinline__ void mx_load8(const T *row, int c, int K, bool vec, float (&v)[8]);
template <> __device__ __forceinline__ void mx_load8<float>(const float *row, int c, int K, bool vec, float (&v)[8])
{
    if (vec && c + 8 <= K) {
        const float4 a = reinterpret_cast<const float4 *>(row + c)[0], b = reinterpret_cast<const float4 *>(row + c)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < K ? row[c + i] : 0.f;
    }
}
template <> __device__ __forceinline__ void mx_load8<bf16_t>(const bf16_t *row, int c, int K, bool vec, float (&v)[8])
{
    if (vec && c + 8 <= K) {
        const uint4 a = *reinterpret_cast<const uint4 *>(row + c);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < K ? bf16_to_f32(row[c + i]) : 0.f;
    }
}
// Whether rows of `ld` elements from p on start at multiples of 16 bytes
static inline bool mx_vec(const void *p, int64_t ld, int dtype) { return (uintptr_t)p % 16 == 0 && ld * (dtype ? 2 : 4) % 16 == 0; }
// (what a launch holds: fewer than 2^32 threads in its first dimension)
static inline bool mx_fits(int64_t workgroups, int threads) { return workgroups * threads < (int64_t)1 << 32; }
static inline bool mx_aligned(const void *p) { return (uintptr_t)p % 16 == 0; }

// A block of 32 values lies in the 4 lanes of a quad, eight each: its scale byte, the same in all four.  bad: a value of the
// block is not finite.
template <int FMT> __device__ __forceinline__ int mx_quad_scale(const float (&v)[8], bool &bad)
{
    uint32_t m = 0, nf = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        m = max(m, mx_finite_bits(v[i]));
        if (FMT == SJD_MX4) nf |= (__float_as_uint(v[i]) & 0x7F800000u) == 0x7F800000u ? 1u : 0u;
    }
    m = max(m, (uint32_t)__shfl_xor((int)m, 1)); m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    if (FMT == SJD_MX4) { nf |= (uint32_t)__shfl_xor((int)nf, 1); nf |= (uint32_t)__shfl_xor((int)nf, 2); }
    bad = FMT == SJD_MX4 && nf;
    return mx_scale_byte<FMT>(m);
}
// Quantises a quad's block: this lane's eight codes to `codes` (8 bytes E4M3, 4 bytes E2M1); returns the scale byte
template <int FMT> __device__ __forceinline__ int mx_quantise8(const float (&v)[8], uint2 &codes)
{
    bool bad;
    const int byte = mx_quad_scale<FMT>(v, bad);
    if (FMT == SJD_MX8) {
        const float inv = mx_pow2(254 - byte);            // (byte is at most 247)
        codes = make_uint2(mx_e4m3x4(v[0], v[1], v[2], v[3], inv), mx_e4m3x4(v[4], v[5], v[6], v[7], inv));
        return byte;
    }
    codes = make_uint2(bad ? 0u : mx_e2m1x8(v, mx_pow2(byte)), 0u);
    return bad ? 255 : byte;
}

// Buffer descriptors: scalar offsets, and loads whose vector offset lies behind the end give zeros and cost no memory access (scalar offsets
// stay inside: the hardware takes them from the size before it compares).
#define MX_OOB 0x40000000        // behind every buffer here
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_buffer(const uint8_t *p, size_t bytes)
{
    // (uniform, and said so: else every load becomes a loop over the wave's descriptors)
    const uint64_t a = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
__device__ __forceinline__ uint4 mx_load16(__amdgpu_buffer_rsrc_t r, int v, int s)
{
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, v, s, 0);
    return make_uint4(x[0], x[1], x[2], x[3]);
}
