// What the serving operators' kernels share: 8-bit values and their scales, rows at any address.
#pragma once

#include "sconv_tokens_common.h"
#include "sconv_serving.h"

namespace sconv {

struct e4m3 { uint8_t b; };                            // a value in 8 bits (its scale is its block's)
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

inline int serving_type_size(int t) { return t == SCONV_E4M3 ? 1 : type_size(t); }

// Eight neighbouring elements of a row of which `have` are there (others: zeros), from any address that the type allows: the memory takes
// 16 bytes at any of them.  A row's last elements come one by one.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int have, float* v)
{
    if (have >= 8) {
        if constexpr (sizeof(T) == 2) {
            typedef bf16x8 any __attribute__((aligned(2)));
            const bf16x8 q = *(const any*)p;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)q[i];
        } else {
            typedef f32x4 any __attribute__((aligned(4)));
            const f32x4 a = *(const any*)p, b = *(const any*)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < have ? (float)p[i] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, int have, const float* v)
{
    if (have >= 8) {
        if constexpr (sizeof(T) == 2) {
            typedef bf16x8 any __attribute__((aligned(2)));
            bf16x8 q;
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = (bf16)v[i];
            *(any*)p = q;
        } else {
            typedef f32x4 any __attribute__((aligned(4)));
            *(any*)p = f32x4{v[0], v[1], v[2], v[3]};
            *(any*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < have) p[i] = (T)v[i];
    }
}

__device__ __forceinline__ void load8_typed(const void* p, int type, int64_t at, int have, float* v)
{
    if (type == SCONV_BF16) load8((const bf16*)p + at, have, v);
    else load8((const float*)p + at, have, v);
}

// The largest of a block's finite magnitudes, as its bits (which are ordered as the values are).
__device__ __forceinline__ uint32_t finite_top(const float* v, int n = 8)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const uint32_t u = __float_as_uint(v[i]) & 0x7fffffffu;
        top = u < 0x7f800000u && u > top ? u : top;
    }
    return top;
}

// The largest over aligned groups of 16 lanes (WIDE: 32).
template <bool WIDE>
__device__ __forceinline__ uint32_t lanes_top(uint32_t v)
{
#define SCONV_ROTATED(n) (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + n, 0xf, 0xf, false)
    v = max(v, SCONV_ROTATED(8));
    v = max(v, SCONV_ROTATED(4));
    v = max(v, SCONV_ROTATED(2));
    v = max(v, SCONV_ROTATED(1));
#undef SCONV_ROTATED
    if constexpr (WIDE) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(r[0], r[1]);
    }
    return v;
}

// The scale byte of a block whose largest finite magnitude has these bits: (1 + m) 2^x <= 1.75 * 2^8 * 2^e for the smallest e.
__device__ __forceinline__ int scale_byte(uint32_t top)
{
    const int s = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(s, 1);
}
__device__ __forceinline__ float scale_inverse(int s) { return __uint_as_float((uint32_t)(254 - s) << 23); }
// 2^(s - 127)
__device__ __forceinline__ float scale_of(int s) { return __uint_as_float((uint32_t)s << 23); }

// Eight values into 8 bits: the product with a power of two is exact (or far below the smallest step), the conversion rounds once.
__device__ __forceinline__ u32x2 to_e4m3(const float* v, float inverse)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inverse, v[5] * inverse, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inverse, v[7] * inverse, hi, true);
    return u32x2{(uint32_t)lo, (uint32_t)hi};
}
__device__ __forceinline__ void store8(e4m3* p, int have, u32x2 q)
{
    typedef u32x2 any __attribute__((aligned(1)));
    if (have >= 8) { *(any*)p = q; return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < have) p[i].b = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
}
// Eight values in 8 bits as they lie in memory, and as numbers.
__device__ __forceinline__ u32x2 load8_bytes(const e4m3* p, int have)
{
    typedef u32x2 any __attribute__((aligned(1)));
    if (have >= 8) return *(const any*)p;
    u32x2 q = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < have) q[i >> 2] |= (uint32_t)p[i].b << (8 * (i & 3));
    return q;
}
__device__ __forceinline__ void from_e4m3(u32x2 q, float scale, float* v)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true);
        v[4 * i] = a[0] * scale; v[4 * i + 1] = a[1] * scale; v[4 * i + 2] = b[0] * scale; v[4 * i + 3] = b[1] * scale;
    }
}

// Eight values in 8 bits as 16-bit ones, which hold them exactly, times a power of two.
__device__ __forceinline__ bf16x8 widened(uint32_t lo, uint32_t hi, float scale = 1.0f)
{
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Division of 0 .. 2^31 - 1 by a number of the same range by multiplication: m = ceil(2^(31 + l) / d) with 2^(l - 1) < d <= 2^l passes
// 2^(31 + l) / d by less than 2^l / d, so n * m / 2^(31 + l) stays below the next whole number.
struct Divide { uint32_t d, m; int l; };
inline Divide divide_by(uint32_t d)
{
    int l = 0;
    while ((uint64_t(1) << l) < d) ++l;
    return Divide{d, (uint32_t)(((uint64_t(1) << (31 + l)) + d - 1) / d), l};
}
__host__ __device__ __forceinline__ uint32_t divided(uint32_t n, const Divide& by) { return (uint32_t)(((uint64_t)n * by.m) >> (31 + by.l)); }

int launch_rmsnorm_forward(const sconv_rmsnorm_desc_t& d, const void* x, const void* residual, const void* w, void* y, uint8_t* scale,
                           void* total, float* rstd, hipStream_t stream);
size_t rmsnorm_workspace(const sconv_rmsnorm_desc_t& d);
int launch_rmsnorm_backward(const sconv_rmsnorm_desc_t& d, const void* dy, const void* total, const float* rstd, const void* w,
                            const void* dt, void* dx, void* dres, void* dw, void* ws, hipStream_t stream);
int launch_quant8(const sconv_quant8_desc_t& d, const void* x, void* q, uint8_t* scale, hipStream_t stream);
int launch_linear8(const sconv_linear8_desc_t& d, const void* x, const uint8_t* xs, const void* w, const uint8_t* ws, void* y, hipStream_t stream);
int launch_cache(const sconv_cache_desc_t& d, bool write, void* k, void* v, const int32_t* starts, const int32_t* counts,
                 const sconv_pages_dev_t& pages, hipStream_t stream);
size_t paged_workspace(const sconv_paged_desc_t& d);
int launch_paged(const sconv_paged_desc_t& d, const void* q, const sconv_pages_dev_t& pages, const float* lam, const int32_t* lengths,
                 void* out, void* ws, size_t ws_bytes, hipStream_t stream);

}  // namespace sconv
