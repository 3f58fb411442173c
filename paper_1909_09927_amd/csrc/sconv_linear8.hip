// Product of 8-bit operands with block scales (formula in sconv_serving.h).
//
// Few rows (up to 64, single tokens): bound by the weights' read.  A workgroup takes 16 weight rows, its wavefronts share out the blocks of
// 128, read weights from memory straight into the product's registers and meet in LDS.  The 8-bit values become 16-bit ones, exactly, a
// block's product is exact to 32 bits and takes its scale as it joins the sum.
// Many rows: tiles of 64 x 64, operands from memory in the same way.
//
// Layout of the products: weights are A, tokens are B, so that a lane's results are neighbours of one token's row.  Which depths of a block a
// lane holds does not matter, as long as both operands have the same.
#include <algorithm>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct LinArgs {
    const uint8_t* x; const uint8_t* xs; const uint8_t* w; const uint8_t* ws; void* y;
    int M, N, K, KB, vec;
    int64_t x_m, w_n, y_m;
};

// 16 bytes of a row of which `have` are there, from any address.
__device__ __forceinline__ i32x4 bytes16(const uint8_t* p, int have)
{
    typedef i32x4 any __attribute__((aligned(1)));
    if (have >= 16) return *(const any*)p;
    union { i32x4 v; uint32_t u[4]; } r;
    r.v = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) if (i < have) r.u[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return r.v;
}

// Eight bytes as 16-bit values.
__device__ __forceinline__ bf16x8 widened(int lo, int hi)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <typename T>
__device__ __forceinline__ void store_row4(T* p, int have, bool vec, const float* v)
{
    if (vec && have >= 4) { store_vec<4>(p, v); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < have) p[i] = (T)v[i];
}

// Few rows: MT tiles of 16 tokens, NW wavefronts.  A lane has 32 bytes (l / 16) * 32.. of row l % 16 of both operands.
template <typename T, int MT, int NW>
__global__ __launch_bounds__(64 * NW) void linear_few(LinArgs a)
{
    __shared__ f32x4 part[NW][MT][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, c = l & 15, h = l >> 4, n0 = blockIdx.x * 16;
    const uint8_t* wr = a.w + (int64_t)min(n0 + c, a.N - 1) * a.w_n + 32 * h;
    const uint8_t* ws = a.ws + (int64_t)(n0 >> 7) * a.KB;
    const uint8_t* xr[MT];
    const uint8_t* xs[MT];
    f32x4 sum[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = min(16 * t + c, a.M - 1);
        xr[t] = a.x + m * a.x_m + 32 * h;
        xs[t] = a.xs + (int64_t)m * a.KB;
        sum[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    i32x4 wv[2], xv[MT][2];
    int we, xe[MT];
    const auto fetch = [&](int kb) {
        const int k = kb * 128, have = a.K - k - 32 * h;
        wv[0] = bytes16(wr + k, have);
        wv[1] = bytes16(wr + k + 16, have - 16);
        we = ws[kb];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            xv[t][0] = bytes16(xr[t] + k, have);
            xv[t][1] = bytes16(xr[t] + k + 16, have - 16);
            xe[t] = xs[t][kb];
        }
    };
    if (w < a.KB) fetch(w);
    for (int kb = w; kb < a.KB; kb += NW) {
        bf16x8 wf[4], xf[MT][4];
        int e[MT];
#pragma unroll
        for (int s = 0; s < 4; ++s) wf[s] = widened(wv[s >> 1][2 * (s & 1)], wv[s >> 1][2 * (s & 1) + 1]);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            e[t] = we + xe[t] - 254;
#pragma unroll
            for (int s = 0; s < 4; ++s) xf[t][s] = widened(xv[t][s >> 1][2 * (s & 1)], xv[t][s >> 1][2 * (s & 1) + 1]);
        }
        if (kb + NW < a.KB) fetch(kb + NW);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < 4; ++s) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[s], xf[t][s], p, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[t][i] += __builtin_ldexpf(p[i], e[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[w][t][l] = sum[t];
    __syncthreads();
    for (int t = w; t < MT; t += NW) {
        f32x4 v = part[0][t][l];
#pragma unroll
        for (int i = 1; i < NW; ++i) v += part[i][t][l];
        const int m = 16 * t + c, n = n0 + 4 * h;
        const float o[4] = {v[0], v[1], v[2], v[3]};
        if (m < a.M) store_row4((T*)a.y + m * a.y_m + n, a.N - n, a.vec, o);
    }
}

// Many rows, simple form: 64 x 64 results a workgroup, a wavefront 16 weight rows by 64 tokens, operands from memory.
template <typename T>
__global__ __launch_bounds__(256) void linear_tile(LinArgs a, int row_tiles)
{
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, c = l & 15, h = l >> 4;
    const int nt = blockIdx.x / row_tiles, n0 = nt * 64 + 16 * w, m0 = (blockIdx.x - nt * row_tiles) * 64;
    const uint8_t* wr = a.w + (int64_t)min(n0 + c, a.N - 1) * a.w_n + 32 * h;
    const uint8_t* ws = a.ws + (int64_t)(min(n0, a.N - 1) >> 7) * a.KB;
    f32x4 sum[4] = {};
    for (int kb = 0; kb < a.KB; ++kb) {
        const int k = kb * 128, have = a.K - k - 32 * h;
        const i32x4 w0 = bytes16(wr + k, have), w1 = bytes16(wr + k + 16, have - 16);
        const int we = ws[kb];
        bf16x8 wf[4] = {widened(w0[0], w0[1]), widened(w0[2], w0[3]), widened(w1[0], w1[1]), widened(w1[2], w1[3])};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int m = min(m0 + 16 * t + c, a.M - 1);
            const uint8_t* xr = a.x + m * a.x_m + 32 * h + k;
            const i32x4 x0 = bytes16(xr, have), x1 = bytes16(xr + 16, have - 16);
            const int e = we + a.xs[(int64_t)m * a.KB + kb] - 254;
            f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[0], widened(x0[0], x0[1]), p, 0, 0, 0);
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[1], widened(x0[2], x0[3]), p, 0, 0, 0);
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[2], widened(x1[0], x1[1]), p, 0, 0, 0);
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[3], widened(x1[2], x1[3]), p, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[t][i] += __builtin_ldexpf(p[i], e);
        }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int m = m0 + 16 * t + c, n = n0 + 4 * h;
        const float o[4] = {sum[t][0], sum[t][1], sum[t][2], sum[t][3]};
        if (m < a.M) store_row4((T*)a.y + m * a.y_m + n, a.N - n, a.vec, o);
    }
}

template <typename T>
int linear_run(const LinArgs& a, hipStream_t stream)
{
    if (a.M <= 64) {
        const int64_t grid = ((int64_t)a.N + 15) / 16;
        if (!grid_fits(grid, 512)) return SCONV_EUNSUPPORTED;
        const dim3 blocks((unsigned)grid), threads(512);
        if (a.M <= 16) hipLaunchKernelGGL((linear_few<T, 1, 8>), blocks, threads, 0, stream, a);
        else if (a.M <= 32) hipLaunchKernelGGL((linear_few<T, 2, 8>), blocks, threads, 0, stream, a);
        else hipLaunchKernelGGL((linear_few<T, 4, 8>), blocks, threads, 0, stream, a);
        return launch_status();
    }
    const int64_t row_tiles = ((int64_t)a.M + 63) / 64, grid = row_tiles * (((int64_t)a.N + 63) / 64);
    if (!grid_fits(grid, 256)) return SCONV_EUNSUPPORTED;
    hipLaunchKernelGGL((linear_tile<T>), dim3((unsigned)grid), dim3(256), 0, stream, a, (int)row_tiles);
    return launch_status();
}

}  // namespace

int launch_linear8(const sconv_linear8_desc_t& d, const void* x, const uint8_t* xs, const void* w, const uint8_t* ws, void* y, hipStream_t stream)
{
    LinArgs a = {};
    a.x = (const uint8_t*)x; a.xs = xs; a.w = (const uint8_t*)w; a.ws = ws; a.y = y;
    a.M = d.M; a.N = d.N; a.K = d.K; a.KB = (int)(((int64_t)d.K + 127) / 128);
    a.x_m = d.x_m; a.w_n = d.w_n; a.y_m = d.y_m;
    a.vec = d.y_m % 4 == 0 && aligned_to(y, 16);
    return d.y_type == SCONV_BF16 ? linear_run<bf16>(a, stream) : linear_run<float>(a, stream);
}

}  // namespace sconv
