// Rotary positions over several axes, queries and keys in one launch (formulas in sconv_tokens.h).
//
// Bound by memory: every element is read and written once.  The sine and cosine of a pair are the same for all heads of a
// token, so a workgroup takes whole tokens: it forms them once into LDS - the angle in 64 bits, reduced to an eighth of a turn
// there, then the two Taylor polynomials in 32 bits - and then turns the tokens' heads with them, 16 bytes a lane.
// Measured: 12544 tokens of 28 heads of 64 in 32 bits 29 us (6.1 TB/s, part of it from the last-level cache), 6272 tokens of 16 heads of 64
// in 16 bits 6.9 us (3.7 TB/s), 64 single tokens 3.6 us (latency).
#include <algorithm>

#include "sconv_tokens_common.h"

namespace sconv {

namespace {

struct RotArgs {
    const void* q; const void* k; void* qo; void* ko;
    const int32_t* pos; const float* freq;
    int64_t tokens;                      // B * S
    int S, Hq, Hk, D, pairs, axes, inverse;
    int64_t q_b, q_s, q_h, k_b, k_s, k_h, qo_b, qo_s, qo_h, ko_b, ko_s, ko_h, pos_b;
    uint8_t axis[SCONV_ROTARY_MAX_PAIRS];
};

// cos and sin of pos * freq.  |x| <= pi/4 after the reduction: the first terms left out are below 2e-9.
__device__ __forceinline__ void turn_of(int pos, float freq, float* c, float* s)
{
    const double quarters = (double)pos * (double)freq * 0.63661977236758134308;   // 2 / pi
    const double whole = rint(quarters);
    const float x = (float)((quarters - whole) * 1.57079632679489661923);
    const int k = (int)(whole - 4.0 * floor(whole * 0.25));
    const float z = x * x;
    const float sn = x + x * z * fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const float a = (k & 1) ? sn : cs, b = (k & 1) ? cs : sn;
    *c = (k == 1 || k == 2) ? -a : a;
    *s = (k >= 2) ? -b : b;
}

// V elements a lane (V = 1: any sizes, strides and addresses).  TT tokens a workgroup.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotArgs a, int TT)
{
    extern __shared__ __attribute__((aligned(16))) float cs[];   // [TT][pairs] cosines, then sines; then where the tokens' heads begin
    const uint32_t t0 = blockIdx.x * (uint32_t)TT;               // (tokens fit 31 bits)
    const int here = (int)min((uint32_t)TT, (uint32_t)a.tokens - t0);
    float* sn = cs + TT * a.pairs;
    int64_t* begin = (int64_t*)(sn + TT * a.pairs);              // [TT][4]: q, k, and the results
    if ((int)threadIdx.x < here) {
        const uint32_t tok = t0 + threadIdx.x, b = tok / (uint32_t)a.S, s = tok - b * (uint32_t)a.S;
        begin[4 * threadIdx.x] = b * a.q_b + s * a.q_s;
        begin[4 * threadIdx.x + 1] = b * a.k_b + s * a.k_s;
        begin[4 * threadIdx.x + 2] = b * a.qo_b + s * a.qo_s;
        begin[4 * threadIdx.x + 3] = b * a.ko_b + s * a.ko_s;
    }
    for (int e = threadIdx.x; e < here * a.pairs; e += 256) {
        const int t = e / a.pairs, p = e - t * a.pairs;
        const uint32_t tok = t0 + t, b = tok / (uint32_t)a.S, s = tok - b * (uint32_t)a.S;
        float c, v;
        turn_of(a.pos[b * a.pos_b + (int64_t)s * a.axes + a.axis[p]], a.freq[p], &c, &v);
        cs[e] = c;
        sn[e] = a.inverse ? -v : v;
    }
    __syncthreads();
    // units of a head: V pairs that turn (halves: two vectors; interleaved: 2V elements side by side), then the rest in Vs
    const int turning = a.pairs / V, rest = (a.D - 2 * a.pairs) / V, units = turning + rest;
    const int heads = a.Hq + a.Hk, per = heads * units, all = here * per;
    for (int e = threadIdx.x; e < all; e += 256) {
        const int t = (int)((uint32_t)e / (uint32_t)per), r = e - t * per, hh = (int)((uint32_t)r / (uint32_t)units), u = r - hh * units;
        const bool key = hh >= a.Hq;
        const T* x = key ? (const T*)a.k + begin[4 * t + 1] + (hh - a.Hq) * a.k_h : (const T*)a.q + begin[4 * t] + hh * a.q_h;
        T* y = key ? (T*)a.ko + begin[4 * t + 3] + (hh - a.Hq) * a.ko_h : (T*)a.qo + begin[4 * t + 2] + hh * a.qo_h;
        float v0[V], v1[V], o0[V], o1[V];
        if (u >= turning) {
            const int i = 2 * a.pairs + (u - turning) * V;
            load_vec<V>(x + i, v0);
            store_vec<V>(y + i, v0);
            continue;
        }
        const float* c = cs + t * a.pairs + u * V;
        const float* d = sn + t * a.pairs + u * V;
        if constexpr (INTER) {
            load_vec<V>(x + 2 * u * V, v0);
            load_vec<V>(x + 2 * u * V + V, v1);
            // v0, v1: the 2V elements in order; pair i is elements 2i, 2i + 1
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e0 = 2 * i, e1 = 2 * i + 1;
                const float p = e0 < V ? v0[e0 % V] : v1[e0 % V], q = e1 < V ? v0[e1 % V] : v1[e1 % V];
                const float r0 = p * c[i] - q * d[i], r1 = p * d[i] + q * c[i];
                if (e0 < V) o0[e0 % V] = r0; else o1[e0 % V] = r0;
                if (e1 < V) o0[e1 % V] = r1; else o1[e1 % V] = r1;
            }
            store_vec<V>(y + 2 * u * V, o0);
            store_vec<V>(y + 2 * u * V + V, o1);
        } else {
            load_vec<V>(x + u * V, v0);
            load_vec<V>(x + a.pairs + u * V, v1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                o0[i] = v0[i] * c[i] - v1[i] * d[i];
                o1[i] = v0[i] * d[i] + v1[i] * c[i];
            }
            store_vec<V>(y + u * V, o0);
            store_vec<V>(y + a.pairs + u * V, o1);
        }
    }
}

template <typename T>
int rotary_run(const RotArgs& a, bool inter, bool vec, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T);
    // about 2048 vectors a workgroup, and at least two workgroups a compute unit where there are so many tokens
    const int64_t per = std::max<int64_t>(1, (int64_t)(a.Hq + a.Hk) * a.D / (2 * (vec ? V : 1)));
    int64_t TT = std::max<int64_t>(1, std::min<int64_t>(2048 / per, a.tokens / 512));
    TT = std::min<int64_t>(std::min<int64_t>(TT, 4096 / a.pairs), 256);
    const unsigned grid = (unsigned)((a.tokens + TT - 1) / TT);
    if (!grid_fits(grid, 256)) return SCONV_EUNSUPPORTED;
    const size_t lds = (size_t)TT * (a.pairs * 2 * sizeof(float) + 4 * sizeof(int64_t));
    if (vec && inter) hipLaunchKernelGGL((rotary_kernel<T, V, true>), dim3(grid), dim3(256), lds, stream, a, (int)TT);
    else if (vec) hipLaunchKernelGGL((rotary_kernel<T, V, false>), dim3(grid), dim3(256), lds, stream, a, (int)TT);
    else if (inter) hipLaunchKernelGGL((rotary_kernel<T, 1, true>), dim3(grid), dim3(256), lds, stream, a, (int)TT);
    else hipLaunchKernelGGL((rotary_kernel<T, 1, false>), dim3(grid), dim3(256), lds, stream, a, (int)TT);
    return launch_status();
}

}  // namespace

int launch_rotary(const sconv_rotary_desc_t& d, const void* q, const void* k, const int32_t* pos, const float* freq,
                  void* qo, void* ko, hipStream_t stream)
{
    RotArgs a = {};
    a.q = q; a.k = k; a.qo = qo; a.ko = ko; a.pos = pos; a.freq = freq;
    a.tokens = (int64_t)d.B * d.S;
    a.S = d.S; a.Hq = d.Hq; a.Hk = d.Hk; a.D = d.D; a.pairs = d.pairs; a.axes = d.axes; a.inverse = d.inverse;
    a.q_b = d.q_b; a.q_s = d.q_s; a.q_h = d.q_h; a.k_b = d.k_b; a.k_s = d.k_s; a.k_h = d.k_h;
    a.qo_b = d.qo_b; a.qo_s = d.qo_s; a.qo_h = d.qo_h; a.ko_b = d.ko_b; a.ko_s = d.ko_s; a.ko_h = d.ko_h;
    a.pos_b = d.pos_b;
    for (int p = 0; p < d.pairs; ++p) a.axis[p] = d.axis[p];
    if (a.tokens == 0 || d.Hq + d.Hk == 0) return SCONV_OK;
    const int V = d.type == SCONV_BF16 ? 8 : 4;
    int64_t strides = d.q_b | d.q_s | d.q_h | d.qo_b | d.qo_s | d.qo_h | d.pairs | (d.D - 2 * d.pairs);
    if (d.Hk) strides |= d.k_b | d.k_s | d.k_h | d.ko_b | d.ko_s | d.ko_h;
    const bool vec = strides % V == 0 && aligned_to(q, 16) && aligned_to(k, 16) && aligned_to(qo, 16) && aligned_to(ko, 16);
    return d.type == SCONV_BF16 ? rotary_run<bf16>(a, d.interleaved, vec, stream) : rotary_run<float>(a, d.interleaved, vec, stream);
}

}  // namespace sconv
