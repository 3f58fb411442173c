// What the token operators' kernels share: types, vector loads and stores, reductions over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sconv_internal.h"
#include "sconv_tokens.h"

namespace sconv {

typedef __bf16 bf16;
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

inline int type_size(int t) { return t == SCONV_BF16 ? 2 : 4; }
inline bool type_known(int t) { return t == SCONV_F32 || t == SCONV_BF16; }

// V elements from an address aligned to them (at most 16 bytes at a time), as floats.
template <int V>
__device__ __forceinline__ void load_vec(const float* p, float* v)
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const f32x4 q = *(const f32x4*)(p + i);
            v[i] = q[0]; v[i + 1] = q[1]; v[i + 2] = q[2]; v[i + 3] = q[3];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = p[i];
    }
}

template <int V>
__device__ __forceinline__ void load_vec(const bf16* p, float* v)
{
    if constexpr (V == 8) {
        const bf16x8 q = *(const bf16x8*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)q[i];
    } else if constexpr (V == 4) {
        const bf16x4 q = *(const bf16x4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)q[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)p[i];
    }
}

template <int V>
__device__ __forceinline__ void store_vec(float* p, const float* v)
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *(f32x4*)(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = v[i];
    }
}

template <int V>
__device__ __forceinline__ void store_vec(bf16* p, const float* v)
{
    if constexpr (V == 8) {
        bf16x8 q;
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = (bf16)v[i];
        *(bf16x8*)p = q;
    } else if constexpr (V == 4) {
        *(bf16x4*)p = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = (bf16)v[i];
    }
}

// One element of an array whose type is known at run time only (weights).
__device__ __forceinline__ float load_typed(const void* p, int type, int64_t i)
{
    return type == SCONV_BF16 ? (float)((const bf16*)p)[i] : ((const float*)p)[i];
}

__device__ __forceinline__ void store_typed(void* p, int type, int64_t i, float v)
{
    if (type == SCONV_BF16) ((bf16*)p)[i] = (bf16)v;
    else ((float*)p)[i] = v;
}

// Sum over aligned groups of L lanes (16, 32 or 64); every lane has it, and the order is fixed.  Within 16 lanes the neighbours come by
// rotation as operands of the sums themselves, beyond by swaps of halves: no trip through LDS.
template <int L>
__device__ __forceinline__ float lanes_sum(float v)
{
    static_assert(L == 16 || L == 32 || L == 64, "whole rows of lanes");
#define SCONV_ROTATED(n) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + n, 0xf, 0xf, false))
    v += SCONV_ROTATED(8);
    v += SCONV_ROTATED(4);
    v += SCONV_ROTATED(2);
    v += SCONV_ROTATED(1);
#undef SCONV_ROTATED
    if constexpr (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (L == 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// V elements as they lie in memory, to be loaded ahead of their use.
template <typename T, int V>
struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Pack { T e[V]; };

// Whether the runtime takes a grid of so many workgroups of so many threads: threads are counted in 32 bits.
inline bool grid_fits(int64_t blocks, int threads) { return blocks * threads < (int64_t(1) << 32); }

inline bool aligned_to(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

int launch_layernorm_forward(const sconv_layernorm_desc_t& d, const void* x, const void* w, const void* b, void* y,
                             float* mean, float* rstd, hipStream_t stream);
size_t layernorm_workspace(const sconv_layernorm_desc_t& d);
int launch_layernorm_backward(const sconv_layernorm_desc_t& d, const void* dy, const void* x, const float* mean,
                              const float* rstd, const void* w, void* dx, void* dw, void* db, void* ws,
                              hipStream_t stream);
int launch_rotary(const sconv_rotary_desc_t& d, const void* q, const void* k, const int32_t* pos, const float* freq,
                  void* qo, void* ko, hipStream_t stream);
size_t diffattn_forward_workspace(const sconv_diffattn_desc_t& d);
size_t diffattn_backward_workspace(const sconv_diffattn_desc_t& d);
int launch_diffattn_forward(const sconv_diffattn_desc_t& d, const void* q, const void* k, const void* v, const float* lam,
                            const int32_t* lengths, const uint8_t* mask, void* out, void* second, float* lse, void* ws,
                            size_t ws_bytes, hipStream_t stream);
int launch_diffattn_backward(const sconv_diffattn_desc_t& d, const void* dout, const void* q, const void* k, const void* v,
                             const float* lam, const int32_t* lengths, const uint8_t* mask, const void* out,
                             const void* second, const float* lse, void* dq, void* dk, void* dv, float* dlam, void* ws,
                             hipStream_t stream);

}  // namespace sconv
