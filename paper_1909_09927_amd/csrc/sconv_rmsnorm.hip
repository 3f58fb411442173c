// Root-mean-square norm with the residual's addition, forward and backward (formulas in sconv_serving.h).
//
// Bound by memory: forward reads x and residual and writes sum and result once, backward reads dy, the sum and its gradient and writes
// one or two gradients.  So a row stays in registers between its sum of squares and its result: LPR lanes hold NV chunks of eight channels
// each, from any address.  A block of 128 channels that shares a scale is 16 neighbouring lanes, whose largest value comes
// by rotation.  The weight's gradient sums over all rows: a workgroup walks many rows, keeps its sums in registers and writes one row of partial
// sums, which a second kernel adds in a fixed order.
// Measured, 16 bits, medians: forward 25088 x 512 with a residual 17.4 us (5.9 TB/s, in part from the caches); 64 x 2048 3.3 us, one latency chain.
// Gradient 25088 x 512 21.4 + 3.8 us (4.1 TB/s both), 25088 x 1024 39.9 (5.2 TB/s), 1568 x 16384 60 (3.4 TB/s: one row a workgroup, nothing ahead).
#include <algorithm>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

struct RmsArgs {
    const void* x; const void* res; const void* w; void* y; uint8_t* scale; void* total; float* rstd;
    const void* dy; const void* t; const float* rstd_in; const void* dt; void* dx; void* dres; float* part;
    int rows, C, blocks, w_type;         // blocks: of 128 channels
    int64_t x_r, res_r, t_r, y_r;
    float eps, inv_c;
};

// Sum over the LPR lanes of a row; where a row has several wavefronts they meet in LDS (red: not reused before the next barrier).
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* red)
{
    v = lanes_sum<(LPR < 64 ? LPR : 64)>(v);
    if constexpr (LPR > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < LPR / 64; ++i) v += red[i];
    }
    return v;
}

template <typename TX, typename TR, typename TY, int LPR, int NV>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR) void rms_fwd(RmsArgs a)
{
    constexpr int RPB = LPR < 256 ? 256 / LPR : 1;
    __shared__ float red[16];
    const int lane = threadIdx.x % LPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;
    const bool live = row < a.rows;
    const TX* x = (const TX*)a.x + row * a.x_r;
    const TR* res = (const TR*)a.res + row * a.res_r;
    float t[NV][8];
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * LPR + lane) * 8, have = live ? a.C - c : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t[j][i] = 0.0f;
        if (have > 0) {
            load8(x + c, have, t[j]);
            if (a.res) {
                float r[8];
                load8(res + c, have, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[j][i] += r[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(t[j][i], t[j][i], sum);
    }
    const float rstd = 1.0f / sqrtf(fmaf(row_sum<LPR>(sum, red), a.inv_c, a.eps));
    if (!live) return;
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * LPR + lane) * 8, have = a.C - c;
        if (have > 0 && a.res) store8((TR*)a.total + row * a.t_r + c, have, t[j]);
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.0f;
        if (have > 0 && a.w) load8_typed(a.w, a.w_type, c, have, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[j][i] *= rstd * w[i];
        if constexpr (sizeof(TY) == 1) {
            // (lanes behind the row hold zeros, or NaN of an infinite rstd, which a scale does not know of)
            const int s = scale_byte(lanes_top<false>(finite_top(t[j])));
            if (have > 0) {
                store8((e4m3*)a.y + row * a.y_r + c, have, to_e4m3(t[j], scale_inverse(s)));
                if ((lane & 15) == 0) a.scale[row * a.blocks + c / 128] = (uint8_t)s;
            }
        } else if (have > 0) {
            store8((TY*)a.y + row * a.y_r + c, have, t[j]);
        }
    }
}

// TG: dy; TR: the sum, its gradient and dres; TX: dx.
template <typename TG, typename TR, typename TX, int LPR, int NV>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR) void rms_bwd(RmsArgs a)
{
    constexpr int RPB = LPR < 256 ? 256 / LPR : 1;
    __shared__ float red[2][16];
    extern __shared__ float sums[];      // [RPB][C] (RPB > 1)
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    float dw[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    float w[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * LPR + lane) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[j][i] = 1.0f;
        if (a.w && c < a.C) load8_typed(a.w, a.w_type, c, a.C - c, w[j]);
    }
    // AHEAD: a row is read while the one before it is worked on (25088 x 512 25.9 -> 24.5 us).  Two chunks of it a lane have no room for that
    // (25088 x 1024 38.6 -> 50 us, 1568 x 16384 66 -> 185).
    constexpr bool AHEAD = NV == 1;
    float next_u[NV][8], next_g[NV][8], next_d[NV][8], next_rstd = 0.0f;
    const auto read = [&](int64_t row) __attribute__((always_inline)) {
        const bool live = row < a.rows;
        next_rstd = live ? a.rstd_in[row] : 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * 8, have = live ? a.C - c : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) next_u[j][i] = next_g[j][i] = next_d[j][i] = 0.0f;
            if (have <= 0) continue;
            load8((const TR*)a.t + row * a.t_r + c, have, next_u[j]);
            load8((const TG*)a.dy + row * a.y_r + c, have, next_g[j]);
            if (a.dt) load8((const TR*)a.dt + row * a.res_r + c, have, next_d[j]);
        }
    };
    int turn = 0;
    int64_t row = (int64_t)blockIdx.x * RPB + group;
    const int64_t step = (int64_t)gridDim.x * RPB;
    if (AHEAD) read(row);
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step, row += step, turn ^= 1) {
        const bool live = row < a.rows;
        if (!AHEAD) read(row);
        const float rstd = next_rstd;
        float u[NV][8], g[NV][8], d[NV][8];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[j][i] = next_u[j][i] * rstd;
                g[j][i] = next_g[j][i];
                d[j][i] = next_d[j][i];
                dw[j][i] = fmaf(g[j][i], u[j][i], dw[j][i]);
                g[j][i] *= w[j][i];
                sum = fmaf(g[j][i], u[j][i], sum);
            }
        if (AHEAD && r0 + step < a.rows) read(row + step);
        if (!a.dx && !a.dres) continue;
        const float mean = row_sum<LPR>(sum, red[turn]) * a.inv_c;
        if (!live) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * 8, have = a.C - c;
            if (have <= 0) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) d[j][i] = fmaf(rstd, fmaf(-u[j][i], mean, g[j][i]), d[j][i]);
            if (a.dx) store8((TX*)a.dx + row * a.C + c, have, d[j]);
            if (a.dres) store8((TR*)a.dres + row * a.C + c, have, d[j]);
        }
    }
    if (!a.part) return;
    float* out = a.part + (int64_t)blockIdx.x * a.C;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * 8;
            if (c < a.C) store8(out + c, a.C - c, dw[j]);
        }
    } else {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * 8;
            if (c < a.C) store8(sums + group * a.C + c, a.C - c, dw[j]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.C; c += 256) {
            float t = 0.0f;
            for (int g = 0; g < RPB; ++g) t += sums[g * a.C + c];
            out[c] = t;
        }
    }
}

// dw: 32 groups of lanes add every 32nd row of the partial sums of 32 columns, then the groups are added in their order.  Bound by latency: many
// rows are asked for at once.
__global__ __launch_bounds__(1024) void rms_dw_sum(const float* part, int blocks, int C, void* dw, int type)
{
    __shared__ float sums[32][33];
    const int l = threadIdx.x & 31, g = threadIdx.x >> 5, c = blockIdx.x * 32 + l;
    float v = 0.0f;
    if (c < C)
#pragma unroll 16
        for (int b = g; b < blocks; b += 32) v += part[(int64_t)b * C + c];
    sums[g][l] = v;
    __syncthreads();
    if (g == 0 && c < C) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sums[i][l];
        store_typed(dw, type, c, t);
    }
}

// Workgroups of a backward call at most: four a compute unit (25088 x 512: 512 28.3 us, 768 25.1, 1024 24.5, 1568 28.6).
constexpr int RMS_BLOCKS = 1024;

// Lanes a row and chunks a lane: the fewest lanes that hold a row in four chunks (backward: two), more where the rows are few and
// would leave most of the chip idle.
void rms_shape(int C, int rows, int most, int* lpr, int* nv)
{
    const int chunks = (C + 7) / 8;
    int l = 16;
    while (l < 1024 && chunks > l * (l == 16 ? 1 : most)) l *= 4;
    while (l < 256 && rows < 1024 && chunks > l) l *= 4;
    *lpr = l;
    int n = 1;
    while (l * n < chunks) n *= 2;
    *nv = n;
}

template <typename TX, typename TR, typename TY>
int fwd_run(const RmsArgs& a, hipStream_t stream)
{
    int lpr, nv;
    rms_shape(a.C, a.rows, 4, &lpr, &nv);
    const int rpb = lpr < 256 ? 256 / lpr : 1, threads = std::max(lpr, 256);
    const int64_t grid = ((int64_t)a.rows + rpb - 1) / rpb;
    if (!grid_fits(grid, threads)) return SCONV_EUNSUPPORTED;
#define SCONV_RMS(L, N)                                                                                                     \
    if (lpr == L && nv == N) {                                                                                              \
        hipLaunchKernelGGL((rms_fwd<TX, TR, TY, L, N>), dim3((unsigned)grid), dim3(threads), 0, stream, a);                 \
        return launch_status();                                                                                             \
    }
    SCONV_RMS(16, 1) SCONV_RMS(64, 1) SCONV_RMS(64, 2) SCONV_RMS(64, 4) SCONV_RMS(256, 1) SCONV_RMS(256, 2) SCONV_RMS(256, 4) SCONV_RMS(1024, 2)
#undef SCONV_RMS
    return SCONV_EUNSUPPORTED;
}

template <typename TG, typename TR, typename TX>
int bwd_run(const RmsArgs& a, int blocks, int lpr, int nv, hipStream_t stream)
{
    const int rpb = lpr < 256 ? 256 / lpr : 1, threads = std::max(lpr, 256);
    const size_t lds = rpb > 1 && a.part ? (size_t)rpb * a.C * sizeof(float) : 0;
#define SCONV_RMS(L, N)                                                                                                     \
    if (lpr == L && nv == N) {                                                                                              \
        hipLaunchKernelGGL((rms_bwd<TG, TR, TX, L, N>), dim3((unsigned)blocks), dim3(threads), lds, stream, a);             \
        return launch_status();                                                                                             \
    }
    SCONV_RMS(16, 1) SCONV_RMS(64, 1) SCONV_RMS(64, 2) SCONV_RMS(256, 1) SCONV_RMS(256, 2) SCONV_RMS(1024, 1) SCONV_RMS(1024, 2)
#undef SCONV_RMS
    return SCONV_EUNSUPPORTED;
}

RmsArgs rms_args(const sconv_rmsnorm_desc_t& d)
{
    RmsArgs a = {};
    a.rows = d.rows; a.C = d.C; a.blocks = (d.C + 127) / 128; a.w_type = d.w_type;
    a.x_r = d.x_r; a.res_r = d.res_r; a.t_r = d.t_r; a.y_r = d.y_r;
    a.eps = d.eps; a.inv_c = 1.0f / (float)d.C;
    return a;
}

}  // namespace

size_t rmsnorm_workspace(const sconv_rmsnorm_desc_t& d) { return (size_t)RMS_BLOCKS * d.C * sizeof(float); }

int launch_rmsnorm_forward(const sconv_rmsnorm_desc_t& d, const void* x, const void* residual, const void* w, void* y, uint8_t* scale,
                           void* total, float* rstd, hipStream_t stream)
{
    RmsArgs a = rms_args(d);
    a.x = x; a.res = residual; a.w = w; a.y = y; a.scale = scale; a.total = total; a.rstd = rstd;
    if (d.x_type == SCONV_F32) {
        if (d.y_type == SCONV_E4M3) return fwd_run<float, float, e4m3>(a, stream);
        return d.y_type == SCONV_BF16 ? fwd_run<float, float, bf16>(a, stream) : fwd_run<float, float, float>(a, stream);
    }
    if (d.t_type == SCONV_F32)
        return d.y_type == SCONV_E4M3 ? fwd_run<bf16, float, e4m3>(a, stream) : fwd_run<bf16, float, bf16>(a, stream);
    return d.y_type == SCONV_E4M3 ? fwd_run<bf16, bf16, e4m3>(a, stream) : fwd_run<bf16, bf16, bf16>(a, stream);
}

int launch_rmsnorm_backward(const sconv_rmsnorm_desc_t& d, const void* dy, const void* total, const float* rstd, const void* w,
                            const void* dt, void* dx, void* dres, void* dw, void* ws, hipStream_t stream)
{
    RmsArgs a = rms_args(d);
    a.dy = dy; a.t = total; a.rstd_in = rstd; a.w = w; a.dt = dt; a.dx = dx; a.dres = dres;
    a.part = dw ? (float*)ws : nullptr;
    int blocks = 0;
    if (d.rows > 0 && (dx || dres || dw)) {
        int lpr, nv;
        rms_shape(d.C, d.rows, 2, &lpr, &nv);
        const int rpb = lpr < 256 ? 256 / lpr : 1;
        blocks = (int)std::min<int64_t>(RMS_BLOCKS, ((int64_t)d.rows + rpb - 1) / rpb);
        const int rc = d.t_type == SCONV_BF16  ? bwd_run<bf16, bf16, bf16>(a, blocks, lpr, nv, stream)
                       : d.x_type == SCONV_BF16 ? bwd_run<bf16, float, bf16>(a, blocks, lpr, nv, stream)
                       : d.y_type == SCONV_BF16 ? bwd_run<bf16, float, float>(a, blocks, lpr, nv, stream)
                                                : bwd_run<float, float, float>(a, blocks, lpr, nv, stream);
        if (rc) return rc;
    }
    if (!dw) return SCONV_OK;
    hipLaunchKernelGGL(rms_dw_sum, dim3((unsigned)((d.C + 31) / 32)), dim3(1024), 0, stream, (const float*)ws, blocks, d.C, dw, d.w_type);
    return launch_status();
}

}  // namespace sconv
