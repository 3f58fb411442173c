// Layer norm over the channels of every place, forward and backward (formulas in sconv_tokens.h).
//
// Bound by memory: forward reads x and writes y once, backward reads dy and x and writes dx once.  So a row stays in registers
// between the statistics and the result: its sums are formed in two steps (mean, then squared distances from it), so that no
// large squares cancel where the mean is large against the spread, and that costs no second read.
//   tokens  a row of C contiguous channels belongs to 16, 64 or 256 lanes, which hold NV vectors each.
//   map     x[c][s] is contiguous along the places: a workgroup takes P places and all channels, lanes along the places read
//           whole segments of every channel, and tiles of 128 to 512 channels (backward: dy's of all channels) are turned in LDS so
//           that tokens are written (dy: read) in whole segments too.
// The weight's gradient sums over all places: every workgroup walks many rows, keeps the sums of its own in registers, and
// writes one row of partial sums, which a second kernel adds in a fixed order.
// Measured (kernels alone; a large copy moves 4.90 TB/s): forward, 25088 x 512 in 16 bits 12.0 us (4.3 TB/s), 6272 x 4096 19.6; rows that do not
// lie at whole vectors are read an element a lane (6272 x 4100 77 us); map 8 x 256 x 56 x 56 in 32 bits to 16-bit tokens 12.9 us (3.0 TB/s:
// reading and writing follow each other in a workgroup); backward, 25088 x 512 in 16 bits 17.3 us (4.5 TB/s) and 3.5 for the sums;
// backward, map 32 x 896 x 14 x 14 in 32 bits 27 us (2.5 TB/s: 416 workgroups, one round) and 5.3; 49 x 2048 3.3 us (latency).
#include <math.h>

#include <algorithm>

#include "sconv_tokens_common.h"

namespace sconv {

namespace {

struct LnArgs {
    const void* x; const void* dy; const void* w; const void* b; void* y; void* dx;
    float* mean; float* rstd;            // forward: written (or null)
    const float* mean_in; const float* rstd_in;
    float* part;                         // backward: [blocks][2][C], or null
    int64_t rows;                        // N * S
    int S, C, N, w_type;
    int v4;                              // map: four channels of a token, and of the weights, lie aligned
    int64_t x_n, x_s, y_n, y_s;
    float eps, inv_c;
};

// (image, place) of a row; S is the row count itself where rows lie at one stride.
__device__ __forceinline__ void place_of(const LnArgs& a, int64_t row, int& n, int& s)
{
    if (a.N == 1) { n = 0; s = (int)row; }
    else { n = (int)((uint32_t)row / (uint32_t)a.S); s = (int)((uint32_t)row - (uint32_t)n * (uint32_t)a.S); }
}

template <int V>
__device__ __forceinline__ void load_w(const void* w, int type, int c, float* v)
{
    if (type == SCONV_BF16) load_vec<V>((const bf16*)w + c, v);
    else load_vec<V>((const float*)w + c, v);
}

// Sum over the LPR lanes of a row; for LPR = 256 the four wavefronts meet in LDS (red: 4 floats a call, not reused before the
// next barrier).
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* red)
{
    v = lanes_sum<(LPR < 64 ? LPR : 64)>(v);
    if constexpr (LPR > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (red[0] + red[1]) + (red[2] + red[3]);
    }
    return v;
}

template <typename TX, typename TY, int V, int LPR, int NV>
__global__ __launch_bounds__(256) void ln_fwd(LnArgs a)
{
    __shared__ float red[2][4];
    const int lane = threadIdx.x % LPR;
    const int64_t row = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const bool live = row < a.rows;
    int n = 0, s = 0;
    if (live) place_of(a, row, n, s);
    const TX* x = (const TX*)a.x + n * a.x_n + s * a.x_s;
    TY* y = (TY*)a.y + n * a.y_n + s * a.y_s;
    float v[NV][V];
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * LPR + lane) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = 0.0f;
        if (live && c < a.C) load_vec<V>(x + c, v[j]);
#pragma unroll
        for (int i = 0; i < V; ++i) sum += v[j][i];
    }
    const float mean = row_sum<LPR>(sum, red[0]) * a.inv_c;
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if ((j * LPR + lane) * V < a.C)
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[j][i] - mean; sq = fmaf(d, d, sq); }
    }
    const float rstd = 1.0f / sqrtf(fmaf(row_sum<LPR>(sq, red[1]), a.inv_c, a.eps));
    if (!live) return;
    if (a.mean && lane == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * LPR + lane) * V;
        if (c >= a.C) continue;
        float w[V], b[V], o[V];
        if (a.w) load_w<V>(a.w, a.w_type, c, w);
        if (a.b) load_w<V>(a.b, a.w_type, c, b);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            o[i] = (v[j][i] - mean) * rstd;
            if (a.w) o[i] *= w[i];
            if (a.b) o[i] += b[i];
        }
        store_vec<V>(y + c, o);
    }
}

// Rows too long for registers (C over 8192) and maps that are not held (ln_map_held): one workgroup a place, x read three times (from
// the caches after the first).  xs_c: stride between channels.
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void ln_fwd_long(LnArgs a, int64_t xs_s, int64_t xs_c)
{
    __shared__ float red[2][4];
    const int64_t row = blockIdx.x;
    int n, s;
    place_of(a, row, n, s);
    const TX* x = (const TX*)a.x + n * a.x_n + s * xs_s;
    TY* y = (TY*)a.y + n * a.y_n + s * a.y_s;
    float sum = 0.0f, sq = 0.0f;
    for (int c = threadIdx.x; c < a.C; c += 256) sum += (float)x[c * xs_c];
    const float mean = row_sum<256>(sum, red[0]) * a.inv_c;
    for (int c = threadIdx.x; c < a.C; c += 256) { const float d = (float)x[c * xs_c] - mean; sq = fmaf(d, d, sq); }
    const float rstd = 1.0f / sqrtf(fmaf(row_sum<256>(sq, red[1]), a.inv_c, a.eps));
    if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
    for (int c = threadIdx.x; c < a.C; c += 256) {
        float o = ((float)x[c * xs_c] - mean) * rstd;
        if (a.w) o *= load_typed(a.w, a.w_type, c);
        if (a.b) o += load_typed(a.b, a.w_type, c);
        y[c] = (TY)o;
    }
}

// Map in, tokens out.  P places (lanes), CG = threads / P groups of channels; a thread holds channels cg + CG * j.  Tiles of 8 CG
// channels are turned in LDS, four channels of a place a thread.
template <typename TX, typename TY, int P, int THREADS, int NJ>
__global__ __launch_bounds__(THREADS) void ln_map_fwd(LnArgs a, int tiles)
{
    constexpr int CG = THREADS / P, CH = CG * 8;
    __shared__ __attribute__((aligned(16))) float tile[P][CH + 4];
    __shared__ float part[2][CG][P];
    const int p = threadIdx.x % P, cg = threadIdx.x / P;
    const int n = blockIdx.x / tiles, s0 = (blockIdx.x % tiles) * P;
    const int places = min(P, a.S - s0);
    const TX* x = (const TX*)a.x + n * a.x_n;          // (offsets within an image: 32 bits)
    const uint32_t xs = (uint32_t)a.x_s, at = cg * xs + s0 + min(p, places - 1);
    float v[NJ];
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) v[j] = cg + CG * j < a.C ? (float)x[at + CG * j * xs] : 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) sum += v[j];
    part[0][cg][p] = sum;
    __syncthreads();
    float mean = 0.0f;
#pragma unroll
    for (int g = 0; g < CG; ++g) mean += part[0][g][p];
    mean *= a.inv_c;
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        if (cg + CG * j < a.C) { const float d = v[j] - mean; sq = fmaf(d, d, sq); }
    part[1][cg][p] = sq;
    __syncthreads();
    float var = 0.0f;
#pragma unroll
    for (int g = 0; g < CG; ++g) var += part[1][g][p];
    const float rstd = 1.0f / sqrtf(fmaf(var, a.inv_c, a.eps));
    if (a.mean && cg == 0 && p < places) {
        a.mean[(int64_t)n * a.S + s0 + p] = mean;
        a.rstd[(int64_t)n * a.S + s0 + p] = rstd;
    }
    TY* y = (TY*)a.y + n * a.y_n + (int64_t)s0 * a.y_s;
#pragma unroll
    for (int jb = 0; jb < NJ / 8; ++jb) {
        if (jb * CH >= a.C) break;
        if (jb) __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[p][cg + CG * i] = (v[jb * 8 + i] - mean) * rstd;
        __syncthreads();
#pragma unroll
        for (int e0 = 0; e0 < P * CH / 4; e0 += THREADS) {
            const int e = e0 + threadIdx.x, q = e / (CH / 4), k = e % (CH / 4) * 4, c = jb * CH + k;
            if (q >= places || c >= a.C) continue;
            const f32x4 o = *(const f32x4*)&tile[q][k];
            float r[4] = {o[0], o[1], o[2], o[3]};
            if (a.v4) {
                float w[4], b[4];
                if (a.w) load_w<4>(a.w, a.w_type, c, w);
                if (a.b) load_w<4>(a.b, a.w_type, c, b);
#pragma unroll
                for (int i = 0; i < 4; ++i) { if (a.w) r[i] *= w[i]; if (a.b) r[i] += b[i]; }
                store_vec<4>(y + q * a.y_s + c, r);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (c + i >= a.C) break;
                    if (a.w) r[i] *= load_typed(a.w, a.w_type, c + i);
                    if (a.b) r[i] += load_typed(a.b, a.w_type, c + i);
                    y[q * a.y_s + c + i] = (TY)r[i];
                }
            }
        }
    }
}

// Backward, tokens: a workgroup walks rows blockIdx, blockIdx + gridDim, ... of its row groups.
template <typename TX, typename TY, int V, int LPR, int NV>
__global__ __launch_bounds__(256) void ln_bwd(LnArgs a)
{
    constexpr int RPB = 256 / LPR;
    __shared__ float red[4][4];
    extern __shared__ float sums[];      // [RPB][C] (RPB > 1)
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    float w[NV][V], aw[NV][V], ab[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * LPR + lane) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) { w[j][i] = 1.0f; aw[j][i] = ab[j][i] = 0.0f; }
        if (a.w && c < a.C) load_w<V>(a.w, a.w_type, c, w[j]);
    }
    // the next row is on its way while this one is summed
    Pack<TX, V> xp[NV];
    Pack<TY, V> gp[NV];
    float mean_next = 0.0f, rstd_next = 0.0f;
    const auto fetch = [&](int64_t row) {
        if (row >= a.rows) return;
        int n, s;
        place_of(a, row, n, s);
        const TX* x = (const TX*)a.x + n * a.x_n + s * a.x_s;
        const TY* dy = (const TY*)a.dy + n * a.y_n + s * a.y_s;
        mean_next = a.mean_in[row];
        rstd_next = a.rstd_in[row];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * V;
            if (c < a.C) { xp[j] = *(const Pack<TX, V>*)(x + c); gp[j] = *(const Pack<TY, V>*)(dy + c); }
        }
    };
    int turn = 0;
    fetch((int64_t)blockIdx.x * RPB + group);
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB, turn ^= 2) {
        const int64_t row = r0 + group;
        const bool live = row < a.rows;
        const float mean = mean_next, rstd = rstd_next;
        float u[NV][V], g[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) { u[j][i] = (float)xp[j].e[i]; g[j][i] = (float)gp[j].e[i]; }
        fetch(row + (int64_t)gridDim.x * RPB);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (live && (j * LPR + lane) * V < a.C) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    u[j][i] = (u[j][i] - mean) * rstd;
                    aw[j][i] = fmaf(g[j][i], u[j][i], aw[j][i]);
                    ab[j][i] += g[j][i];
                    g[j][i] *= w[j][i];
                    s1 += g[j][i];
                    s2 = fmaf(g[j][i], u[j][i], s2);
                }
            }
        }
        if (a.dx) {
            s1 = row_sum<LPR>(s1, red[turn]) * a.inv_c;
            s2 = row_sum<LPR>(s2, red[turn + 1]) * a.inv_c;
            if (live) {
                TX* dx = (TX*)a.dx + row * a.C;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int c = (j * LPR + lane) * V;
                    if (c >= a.C) continue;
                    float o[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] = rstd * (g[j][i] - s1 - u[j][i] * s2);
                    store_vec<V>(dx + c, o);
                }
            }
        }
    }
    if (!a.part) return;
    float* out = a.part + (int64_t)blockIdx.x * 2 * a.C;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * LPR + lane) * V;
            if (c >= a.C) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) { out[c + i] = aw[j][i]; out[a.C + c + i] = ab[j][i]; }
        }
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * LPR + lane) * V;
                if (c >= a.C) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) sums[group * a.C + c + i] = k ? ab[j][i] : aw[j][i];
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.C; c += 256) {
                float t = 0.0f;
                for (int g2 = 0; g2 < RPB; ++g2) t += sums[g2 * a.C + c];
                out[k * a.C + c] = t;
            }
        }
    }
}

// dx of rows too long for registers, and of maps that are not held.
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void ln_bwd_long(LnArgs a, int64_t xs_s, int64_t xs_c, int64_t ds_n, int64_t ds_s, int64_t ds_c)
{
    __shared__ float red[2][4];
    const int64_t row = blockIdx.x;
    int n, s;
    place_of(a, row, n, s);
    const TX* x = (const TX*)a.x + n * a.x_n + s * xs_s;
    const TY* dy = (const TY*)a.dy + n * a.y_n + s * a.y_s;
    TX* dx = (TX*)a.dx + n * ds_n + s * ds_s;
    const float mean = a.mean_in[row], rstd = a.rstd_in[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const float g = (float)dy[c] * (a.w ? load_typed(a.w, a.w_type, c) : 1.0f);
        s1 += g;
        s2 = fmaf(g, ((float)x[c * xs_c] - mean) * rstd, s2);
    }
    s1 = row_sum<256>(s1, red[0]) * a.inv_c;
    s2 = row_sum<256>(s2, red[1]) * a.inv_c;
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const float g = (float)dy[c] * (a.w ? load_typed(a.w, a.w_type, c) : 1.0f);
        dx[c * ds_c] = (TX)(rstd * (g - s1 - ((float)x[c * xs_c] - mean) * rstd * s2));
    }
}

// The weight's gradient for the same: workgroup (slab of rows, 64 channels), four wavefronts along the rows.
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void ln_dw_long(LnArgs a, int64_t xs_s, int64_t xs_c)
{
    __shared__ float t[2][4][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = blockIdx.y * 64 + lane;
    float aw = 0.0f, ab = 0.0f;
    if (c < a.C)
        for (int64_t row = (int64_t)blockIdx.x * 4 + wv; row < a.rows; row += (int64_t)gridDim.x * 4) {
            int n, s;
            place_of(a, row, n, s);
            const float d = (float)((const TY*)a.dy)[n * a.y_n + s * a.y_s + c];
            const float u = ((float)((const TX*)a.x)[n * a.x_n + s * xs_s + c * xs_c] - a.mean_in[row]) * a.rstd_in[row];
            aw = fmaf(d, u, aw);
            ab += d;
        }
    t[0][wv][lane] = aw;
    t[1][wv][lane] = ab;
    __syncthreads();
    if (threadIdx.x < 128) {
        const int k = threadIdx.x >> 6;
        if (c < a.C)
            a.part[((int64_t)blockIdx.x * 2 + k) * a.C + c] = (t[k][0][lane] + t[k][1][lane]) + (t[k][2][lane] + t[k][3][lane]);
    }
}

// Backward, map: dx (map) and the sums over the places of a workgroup's tiles.  x stays in registers (channels cg + CG * j of a
// place), dy of the whole tile in LDS, turned on the way in and read twice.  Lane p keeps the sums of the channels j with j % P == p of
// its channel group.
inline int map_row(int C) { const int quads = (C + 3) / 4; return 4 * (quads + (quads & 1 ? 2 : 1)); }   // 4 times an odd number

template <typename TX, typename TY, int P, int THREADS, int NJ>
__global__ __launch_bounds__(THREADS, 4) void ln_map_bwd(LnArgs a, int tiles, int64_t total, int row)
{
    constexpr int CG = THREADS / P, KEEP = (NJ + P - 1) / P;
    extern __shared__ __attribute__((aligned(16))) float tile[];   // [P][row], then the weights [CG * NJ]
    __shared__ float part[2][CG][P];
    float* ws = tile + P * row;
    const int p = threadIdx.x % P, cg = threadIdx.x / P, quads = (a.C + 3) / 4;
    for (int c = threadIdx.x; c < CG * NJ; c += THREADS) ws[c] = c >= a.C ? 0.0f : a.w ? load_typed(a.w, a.w_type, c) : 1.0f;
    float aw[KEEP], ab[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) aw[k] = ab[k] = 0.0f;
    // Workgroups go round the eight chiplets: neighbouring tiles go to one of them, whose cache joins the lines that both read and
    // write parts of (16 places of a channel in 32 bits are half a line): 32 x 896 x 14 x 14 36.5 -> 31.0 us, 64 x 1024 x 7 x 7 30.5 -> 24.9,
    // 8 x 256 x 56 x 56, whose tiles are whole lines, 28.0 -> 28.2.
    const int64_t chunk = (total + 7) / 8;
    for (int64_t k = blockIdx.x; k < 8 * chunk; k += gridDim.x) {
        const int64_t t = k % 8 * chunk + k / 8;
        if (t >= total) continue;
        const int n = (int)(t / tiles), s0 = (int)(t % tiles) * P;
        const int places = min(P, a.S - s0), at = min(p, places - 1);
        const bool live = p < places;
        const TX* x = (const TX*)a.x + n * a.x_n;      // (offsets within an image: 32 bits)
        const uint32_t xs = (uint32_t)a.x_s, first = cg * xs + s0 + at;
        const TY* dy = (const TY*)a.dy + n * a.y_n + (int64_t)s0 * a.y_s;
        const float mean = a.mean_in[(int64_t)n * a.S + s0 + at], rstd = a.rstd_in[(int64_t)n * a.S + s0 + at];
        float u[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) u[j] = cg + CG * j < a.C ? (float)x[first + CG * j * xs] : 0.0f;
        for (int e = threadIdx.x; e < P * quads; e += THREADS) {
            const int q = e / quads, c = (e - q * quads) * 4;
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (q < places) {
                if (a.v4) load_vec<4>(dy + q * a.y_s + c, d);
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c + i < a.C) d[i] = (float)dy[q * a.y_s + c + i];
                }
            }
            *(f32x4*)(tile + q * row + c) = f32x4{d[0], d[1], d[2], d[3]};
        }
        __syncthreads();
        const float* mine = tile + p * row + cg;
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            if (CG * j >= a.C) { u[j] = 0.0f; continue; }
            const bool there = live && cg + CG * j < a.C;
            const float d = there ? mine[CG * j] : 0.0f, w = ws[cg + CG * j];
            u[j] = there ? (u[j] - mean) * rstd : 0.0f;
            if (a.part) {
                const float sw = lanes_sum<P>(d * u[j]), sb = lanes_sum<P>(d);
                if (p == j % P) { aw[j / P] += sw; ab[j / P] += sb; }
            }
            s1 = fmaf(d, w, s1);
            s2 = fmaf(d * w, u[j], s2);
        }
        part[0][cg][p] = s1;
        part[1][cg][p] = s2;
        __syncthreads();
        if (a.dx) {
            s1 = s2 = 0.0f;
#pragma unroll
            for (int c = 0; c < CG; ++c) { s1 += part[0][c][p]; s2 += part[1][c][p]; }
            s1 *= a.inv_c;
            s2 *= a.inv_c;
            TX* dx = (TX*)a.dx + (int64_t)n * a.C * a.S;
            const uint32_t to = cg * a.S + s0 + p;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                if (live && cg + CG * j < a.C)
                    dx[to + (uint32_t)(CG * j) * a.S] = (TX)(rstd * (mine[CG * j] * ws[cg + CG * j] - s1 - u[j] * s2));
        }
        __syncthreads();                               // tile and part are written again
    }
    if (!a.part) return;
    float* out = a.part + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int c = cg + CG * j;
        if (p == j % P && c < a.C) { out[c] = aw[j / P]; out[a.C + c] = ab[j / P]; }
    }
}

// Partial sums [blocks][2][C] -> dw, db.  32 columns a workgroup, 32 groups of rows, whose loads do not wait for each other.
__global__ __launch_bounds__(1024) void ln_dw_sum(const float* part, int blocks, int C, void* dw, void* db, int type)
{
    __shared__ float t[32][33];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (e < 2 * C) {
#pragma unroll 16
        for (int k = group; k < blocks; k += 32) v += part[(int64_t)k * 2 * C + e];
    }
    t[group][lane] = v;
    __syncthreads();
    // (a wavefront half a column: the groups as lanes)
    v = lanes_sum<32>(t[lane][group]);
    const int column = blockIdx.x * 32 + group;
    if (lane == 0 && column < 2 * C) {
        if (column < C) store_typed(dw, type, column, v);
        else store_typed(db, type, column - C, v);
    }
}

LnArgs ln_args(const sconv_layernorm_desc_t& d)
{
    LnArgs a = {};
    a.N = d.N; a.S = d.S; a.C = d.C; a.w_type = d.w_type;
    a.rows = (int64_t)d.N * d.S;
    a.x_n = d.x_n; a.x_s = d.x_s; a.y_n = d.y_n; a.y_s = d.y_s;
    a.eps = d.eps;
    a.inv_c = 1.0f / (float)d.C;
    if (d.layout == SCONV_LAYOUT_TOKENS && d.x_n == d.S * d.x_s && d.y_n == d.S * d.y_s) { a.N = 1; a.S = (int)a.rows; }
    return a;
}

// Lanes a row and vectors a lane (0 vectors: too long for registers).  A row's own lanes as few as hold it in four
// vectors of eight; rows that do not fill the chip take a whole workgroup each.
void ln_shape(int C, int V, int64_t rows, int* lpr, int* nv)
{
    const int vecs = (C + V - 1) / V, most = 32 / V;   // vectors a lane: 32 elements at most
    *lpr = 256;
    if (vecs <= 16 * std::min(most, 2)) *lpr = 16;
    else if (vecs <= 64 * most && rows >= 1024) *lpr = 64;
    else if (vecs > 256 * most) { *nv = 0; return; }
    int n = 1;
    while (n * *lpr < vecs) n *= 2;
    *nv = n;
}

// Maps whose places stay in registers: 2048 channels at most, an image within 32 bits of bytes.
bool ln_map_held(const sconv_layernorm_desc_t& d)
{
    const int64_t most = int64_t(1) << 30;
    return d.layout == SCONV_LAYOUT_MAP && d.C <= 2048 && d.x_s * d.C < most - d.S && (int64_t)d.S * d.C < most;
}

// Places of a tile: whole 128-byte lines of a map in 32 bits, fewer where the channels would not fit the registers.  Backward over 128
// channels: half lines, whose smaller tiles of dy let more workgroups share a compute unit while neighbours share a cache (16 against 32
// places: 32 x 512 x 28 x 28 46.6 and 57.6 us, 8 x 256 x 56 x 56 25.3 and 28.1; 16 x 128 x 56 x 56 28.5 and 25.3, 16 x 64 x 112 x 112 78 and 53).
int ln_map_places(const sconv_layernorm_desc_t& d, bool backward) { return d.C <= (backward ? 128 : 1024) ? 32 : 16; }

template <typename K>
int ln_allow_lds(K kern, size_t bytes)
{
    // (beside the kernel's own arrays)
    return bytes <= 48 * 1024 || hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess
               ? SCONV_OK : SCONV_ELAUNCH;
}

// Most workgroups of a backward call, each with a row of partial sums: 512 fill the chip twice over; more would only
// add to the second kernel's work.
constexpr int LN_BLOCKS = 512;

// Elements a vector of a tokens call: 16 bytes of the narrower type where every row begins at such a place, else 1.
int ln_vector(const sconv_layernorm_desc_t& d, const LnArgs& a)
{
    const int V = d.y_type == SCONV_BF16 ? 8 : 4;
    const int64_t strides = a.x_s | a.y_s | (a.N > 1 ? a.x_n | a.y_n : 0) | d.C;
    const bool vec = strides % V == 0 && aligned_to(a.x, 16) && aligned_to(a.y, 16) && aligned_to(a.dy, 16) &&
                     aligned_to(a.dx, 16) && aligned_to(a.w, 16) && aligned_to(a.b, 16);
    return vec ? V : 1;
}

template <typename TX, typename TY, int V>
int ln_tokens(const LnArgs& a, bool backward, int blocks, hipStream_t stream)
{
    int lpr, nv;
    ln_shape(a.C, V, a.rows, &lpr, &nv);
    const int rpb = 256 / lpr;
    const unsigned grid = (unsigned)((a.rows + rpb - 1) / rpb);
    if (!backward && !grid_fits(grid, 256)) return SCONV_EUNSUPPORTED;
    const unsigned bgrid = (unsigned)std::min<int64_t>(blocks, grid);
    const size_t lds = rpb > 1 && a.part ? (size_t)rpb * a.C * 4 : 0;
#define SCONV_LN(L, M)                                                                                          \
    if (lpr == L && nv == M) {                                                                                  \
        if (backward) hipLaunchKernelGGL((ln_bwd<TX, TY, V, L, M>), dim3(bgrid), dim3(256), lds, stream, a);    \
        else hipLaunchKernelGGL((ln_fwd<TX, TY, V, L, M>), dim3(grid), dim3(256), 0, stream, a);                \
        return launch_status();                                                                                 \
    }
    SCONV_LN(16, 1) SCONV_LN(16, 2) SCONV_LN(64, 1) SCONV_LN(64, 2) SCONV_LN(64, 4)
    SCONV_LN(256, 1) SCONV_LN(256, 2) SCONV_LN(256, 4)
    if constexpr (V <= 4) { SCONV_LN(64, 8) SCONV_LN(256, 8) }
    if constexpr (V == 1) { SCONV_LN(64, 16) SCONV_LN(64, 32) SCONV_LN(256, 16) SCONV_LN(256, 32) }
#undef SCONV_LN
    return SCONV_EUNSUPPORTED;
}

template <typename TX, typename TY>
int ln_run(const sconv_layernorm_desc_t& d, LnArgs a, bool backward, hipStream_t stream)
{
    const int blocks = LN_BLOCKS;
    if (ln_map_held(d)) {
        a.v4 = (a.y_s | a.y_n | d.C) % 4 == 0 && aligned_to(a.y, 16) && aligned_to(a.dy, 16) && aligned_to(a.w, 16) && aligned_to(a.b, 16);
        const int P = ln_map_places(d, backward), tiles = (d.S + P - 1) / P;
        const int64_t total = (int64_t)tiles * d.N;
        if (backward) {
            const unsigned grid = (unsigned)std::min<int64_t>(blocks, (total + 7) / 8 * 8);
            const int row = map_row(d.C);
#define SCONV_LN_MAP(PP, TH, J)                                                                                     \
    {                                                                                                               \
        const size_t lds = ((size_t)PP * row + TH / PP * J) * sizeof(float);                                        \
        const int rc = ln_allow_lds(ln_map_bwd<TX, TY, PP, TH, J>, lds);                                            \
        if (rc) return rc;                                                                                          \
        hipLaunchKernelGGL((ln_map_bwd<TX, TY, PP, TH, J>), dim3(grid), dim3(TH), lds, stream, a, tiles, total, row); \
        return launch_status();                                                                                     \
    }
            if (d.C <= 128) SCONV_LN_MAP(32, 512, 8)
            // (a workgroup a compute unit at most: twice the threads on a tile, 64 x 1024 x 7 x 7 24.8 -> 22.0 us, 32 x 896 x 7 x 7
            // 19.3 -> 17.4; with more tiles they push out the second workgroup, 32 x 896 x 14 x 14 33.7 -> 37.4)
            if (total <= 256 && d.C > 256) {
                if (d.C <= 512) SCONV_LN_MAP(16, 1024, 8)
                if (d.C <= 1024) SCONV_LN_MAP(16, 1024, 16)
            }
            if (d.C <= 256) SCONV_LN_MAP(16, 512, 8)
            if (d.C <= 512) SCONV_LN_MAP(16, 512, 16)
            if (d.C <= 1024) SCONV_LN_MAP(16, 512, 32)
            SCONV_LN_MAP(16, 1024, 32)
#undef SCONV_LN_MAP
        }
#define SCONV_LN_MAP(PP, TH, J)                                                                                              \
    {                                                                                                                        \
        if (!grid_fits(total, TH)) return SCONV_EUNSUPPORTED;                                                                \
        hipLaunchKernelGGL((ln_map_fwd<TX, TY, PP, TH, J>), dim3((unsigned)total), dim3(TH), 0, stream, a, tiles);           \
        return launch_status();                                                                                              \
    }
        if (d.C <= 128) SCONV_LN_MAP(32, 512, 8)
        if (d.C <= 256) SCONV_LN_MAP(32, 512, 16)
        if (d.C <= 512) SCONV_LN_MAP(32, 1024, 16)
        if (d.C <= 1024) SCONV_LN_MAP(32, 1024, 32)
        SCONV_LN_MAP(16, 1024, 32)
#undef SCONV_LN_MAP
    }
    const bool map = d.layout == SCONV_LAYOUT_MAP;
    if (!map) {
        constexpr int V = sizeof(TY) == 2 ? 8 : 4;
        if (d.C <= 8192)
            return ln_vector(d, a) == V ? ln_tokens<TX, TY, V>(a, backward, blocks, stream)
                                        : ln_tokens<TX, TY, 1>(a, backward, blocks, stream);
    }
    const int64_t xs_s = map ? 1 : a.x_s, xs_c = map ? a.x_s : 1;
    if ((!backward || a.dx) && !grid_fits(a.rows, 256)) return SCONV_EUNSUPPORTED;
    if (!backward) {
        hipLaunchKernelGGL((ln_fwd_long<TX, TY>), dim3((unsigned)a.rows), dim3(256), 0, stream, a, xs_s, xs_c);
        return launch_status();
    }
    if (a.dx) {
        const int64_t SC = (int64_t)a.S * a.C;
        hipLaunchKernelGGL((ln_bwd_long<TX, TY>), dim3((unsigned)a.rows), dim3(256), 0, stream, a, xs_s, xs_c, SC,
                           map ? (int64_t)1 : (int64_t)a.C, map ? (int64_t)a.S : (int64_t)1);
        const int rc = launch_status();
        if (rc) return rc;
    }
    if (a.part) {
        hipLaunchKernelGGL((ln_dw_long<TX, TY>), dim3(64, (unsigned)((a.C + 63) / 64)), dim3(256), 0, stream, a, xs_s, xs_c);
        return launch_status();
    }
    return SCONV_OK;
}

// Workgroups that write partial sums in a backward call.
int ln_part_blocks(const sconv_layernorm_desc_t& d, const LnArgs& a)
{
    const int blocks = LN_BLOCKS;
    if (ln_map_held(d)) {
        const int P = ln_map_places(d, true);
        return (int)std::min<int64_t>(blocks, ((int64_t)((d.S + P - 1) / P) * d.N + 7) / 8 * 8);
    }
    if (d.layout == SCONV_LAYOUT_TOKENS && d.C <= 8192) {
        int lpr, nv;
        ln_shape(d.C, ln_vector(d, a), a.rows, &lpr, &nv);
        const int rpb = 256 / lpr;
        return (int)std::min<int64_t>(blocks, (a.rows + rpb - 1) / rpb);
    }
    return 64;
}

int ln_typed(const sconv_layernorm_desc_t& d, const LnArgs& a, bool backward, hipStream_t stream)
{
    if (d.x_type == SCONV_BF16) return ln_run<bf16, bf16>(d, a, backward, stream);
    if (d.y_type == SCONV_BF16) return ln_run<float, bf16>(d, a, backward, stream);
    return ln_run<float, float>(d, a, backward, stream);
}

}  // namespace

size_t layernorm_workspace(const sconv_layernorm_desc_t& d) { return (size_t)LN_BLOCKS * 2 * d.C * sizeof(float); }

int launch_layernorm_forward(const sconv_layernorm_desc_t& d, const void* x, const void* w, const void* b, void* y,
                             float* mean, float* rstd, hipStream_t stream)
{
    LnArgs a = ln_args(d);
    if (a.rows == 0) return SCONV_OK;
    a.x = x; a.w = w; a.b = b; a.y = y; a.mean = mean; a.rstd = rstd;
    return ln_typed(d, a, false, stream);
}

int launch_layernorm_backward(const sconv_layernorm_desc_t& d, const void* dy, const void* x, const float* mean,
                              const float* rstd, const void* w, void* dx, void* dw, void* db, void* ws,
                              hipStream_t stream)
{
    LnArgs a = ln_args(d);
    a.x = x; a.dy = dy; a.w = w; a.dx = dx; a.mean_in = mean; a.rstd_in = rstd;
    a.part = dw ? (float*)ws : nullptr;
    int blocks = 0;
    if (a.rows > 0 && (dx || dw)) {
        const int rc = ln_typed(d, a, true, stream);
        if (rc) return rc;
        blocks = ln_part_blocks(d, a);
    }
    if (!dw) return SCONV_OK;
    hipLaunchKernelGGL(ln_dw_sum, dim3((unsigned)((2 * d.C + 31) / 32)), dim3(1024), 0, stream, (const float*)ws, blocks, d.C, dw, db, d.w_type);
    return launch_status();
}

}  // namespace sconv
