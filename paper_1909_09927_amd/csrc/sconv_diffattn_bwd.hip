// Differential attention, backward (formulas in sconv_tokens.h, product layout in sconv_diffattn_common.h).
//
// The weights are formed again from the saved sums (lse), so nothing of Sq x Sk is ever stored.  The two maps share
// G = dout V^T, and dv needs one product with A_1 - lam A_2.  Three kernels:
//   delta   d_1, d_2 of every row, from the saved results.
//   rows    dq: a wavefront keeps 32 queries and walks the keys, as the forward kernel does; also sum_j A_2 G of every row, from
//           unrounded weights, for lam's gradient (d_2 itself stems from results that were rounded).
//   keys    dk, dv: a wavefront keeps 32 keys and walks the queries of every head that shares them, so the sum over heads
//           and queries has one order and needs no atomics.
// Measured in 16 bits, each kernel by itself under the profiler: 8 x 784 x 8 heads of 32 (values of 64): delta 6.5, keys 66, rows 51, dlam 4.7 us
// (bound by exp, a quarter-rate instruction, and by latency: 448 workgroups are 1.75 a compute unit; with the forward's 37 they add up
// to 166, a pass without the profiler takes 149); 2 x 3136 x 8 heads of 64 (128): dv 145, dk 271, rows 243 us (560, 600 and 660
// TFLOP/s with what is formed again).  Heads of 65 to 128 go over the keys three times, form the weights each time and spill (dq in 32 bits
// 1.5 KB a lane): 2 x 784 x 4 heads of 128 (256) 212 us forward and backward in 16 bits, 662 in 32.
// All sums are in 32 bits.  In 16 bits the weights are rounded to the operands' type for dv, as forward; dS goes as two 16-bit values,
// the second holding what the first's rounding left out: its rounding alone would be as large as that of the results, and what d_m
// carries over from rounded results comes on top (dq 2.6e-3 of its norm off against 1.7e-3 for 32 bits rounded once, now 1.9e-3; 13 - 16 % of
// the pass).
#include <math.h>

#include <algorithm>

#include "sconv_diffattn_common.h"

namespace sconv {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

// delta[0] = dout . (out + lam second), delta[1] = dout . second; 16 lanes a row.
template <typename T, int V>
__global__ __launch_bounds__(256) void attn_delta(AttnArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16, all = (int64_t)a.B * a.Sq * a.H;
    const int lane = threadIdx.x % 16;
    if (row >= all) return;                            // (whole groups of 16 lanes)
    const int64_t bi = row / a.H;
    const int head = (int)(row - bi * a.H), b = (int)(bi / a.Sq), i = (int)(bi - (int64_t)b * a.Sq);
    const T* g = (const T*)a.dout + row * a.Dv;
    const T* o = (const T*)a.out_in + row * a.Dv;
    const T* s = (const T*)a.second_in + row * a.Dv;
    float first = 0.0f, second = 0.0f;
    for (int d = lane * V; d < a.Dv; d += 16 * V) {
        float x[V], y[V], z[V];
        load_vec<V>(g + d, x);
        load_vec<V>(o + d, y);
        load_vec<V>(s + d, z);
#pragma unroll
        for (int e = 0; e < V; ++e) { first = fmaf(x[e], y[e], first); second = fmaf(x[e], z[e], second); }
    }
    first = lanes_sum<16>(first);
    second = lanes_sum<16>(second);
    if (lane == 0) {
        const int64_t at = ((int64_t)b * a.H + head) * a.Sq + i, half = (int64_t)a.B * a.H * a.Sq;
        const bool none = a.lse_in[at] == -INFINITY;   // (such a row's dout may be anything)
        a.delta[at] = none ? 0.0f : fmaf(a.lam[head], second, first);
        a.delta[half + at] = none ? 0.0f : second;
    }
}

// dlam[h] = -sum over requests and queries, in one order.
__global__ __launch_bounds__(1024) void attn_dlam(const float* part, int B, int H, int Sq, float* dlam)
{
    __shared__ float t[16];
    const int h = blockIdx.x;
    const int64_t all = (int64_t)B * Sq;
    float v = 0.0f;
#pragma unroll 8
    for (int64_t k = threadIdx.x; k < all; k += 1024) {
        const int b = (int)((uint32_t)k / (uint32_t)Sq), i = (int)((uint32_t)k - (uint32_t)b * (uint32_t)Sq);   // (B H Sq < 2^31)
        v += part[((int64_t)b * H + h) * Sq + i];
    }
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) t[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x < 64) {
        v = lanes_sum<16>(t[threadIdx.x & 15]);
        if (threadIdx.x == 0) dlam[h] = 0.0f - v;
    }
}

// The ends of the two kernels below: a lane's query or key.
template <typename T, int NT>
__device__ __forceinline__ void rows_end(const AttnArgs& a, int b, int i, int head, int mine, int h, int64_t stat, float spread,
                                         const f32x16 (&acc)[2][NT])
{
    spread = half_sum(spread);
    if (mine >= a.rows) return;
    const int64_t at = (((int64_t)b * a.Sq + i) * a.H + head) * 2 * a.D;
    if (a.row_splits > 1) {
        const int64_t split = blockIdx.y, all = (int64_t)a.B * a.Sq * a.H;
        if (h == 0) a.part_s[split * all + stat] = spread;
        float* to = a.part_q + split * all * 2 * a.D + at;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float x[4] = {acc[m][t][e], acc[m][t][e + 1], acc[m][t][e + 2], acc[m][t][e + 3]};
                    store4(to + m * a.D, 32 * t + 8 * (e >> 2) + 4 * h, a.D, a.D % 4 == 0, x);
                }
        return;
    }
    if (h == 0) a.dlam_part[stat] = spread;
    T* dq = (T*)a.dq + at;
    const bool v4 = a.ovec && a.D % 4 == 0;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                float x[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) x[z] = acc[m][t][e + z] * a.scale;
                store4(dq + m * a.D, 32 * t + 8 * (e >> 2) + 4 * h, a.D, v4, x);
            }
}

template <typename T, int NT, int VT, int WHAT>
__device__ __forceinline__ void keys_end(const AttnArgs& a, int b, int hk, int j, int h, const f32x16 (&dk)[2][NT], const f32x16 (&dv)[VT])
{
    if (j >= a.Sk) return;
    const int64_t row = ((int64_t)b * a.Sk + j) * a.Hkv + hk, all = (int64_t)a.B * a.Sk * a.Hkv, split = blockIdx.y;
    const bool parts = a.key_splits > 1;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        if (!(WHAT >> (m + 1) & 1)) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = 32 * t + 8 * (e >> 2) + 4 * h;
                const float f = parts ? 1.0f : a.scale;
                const float x[4] = {dk[m][t][e] * f, dk[m][t][e + 1] * f, dk[m][t][e + 2] * f, dk[m][t][e + 3] * f};
                if (parts) store4(a.part_k + (split * all + row) * 2 * a.D + m * a.D, d, a.D, a.D % 4 == 0, x);
                else store4((T*)a.dk + row * 2 * a.D + m * a.D, d, a.D, a.ovec && a.D % 4 == 0, x);
            }
    }
    if (WHAT & 1)
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = 32 * t + 8 * (e >> 2) + 4 * h;
                const float x[4] = {dv[t][e], dv[t][e + 1], dv[t][e + 2], dv[t][e + 3]};
                if (parts) store4(a.part_v + (split * all + row) * a.Dv, d, a.Dv, a.Dv % 4 == 0, x);
                else store4((T*)a.dv + row * a.Dv, d, a.Dv, a.ovec && a.Dv % 4 == 0, x);
            }
}

// Parts of dq, dk, dv and of dlam's rows, added in one order: one launch for up to four arrays.
struct PartSums { const float* from[4]; void* to[4]; int64_t n[4]; int splits[4], wide[4]; float scale[4]; };   // wide: 32-bit results
template <typename T>
__global__ __launch_bounds__(256) void attn_add_parts(PartSums p, int64_t all)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        int64_t k = i;
        int w = 0;
        while (w < 3 && k >= p.n[w]) k -= p.n[w++];
        float v = 0.0f;
#pragma unroll 4
        for (int s = 0; s < p.splits[w]; ++s) v += p.from[w][s * p.n[w] + k];
        v *= p.scale[w];
        if (p.wide[w]) ((float*)p.to[w])[k] = v;
        else ((T*)p.to[w])[k] = (T)v;
    }
}

template <typename T, bool VEC, int DT>
__global__ __launch_bounds__(256) void attn_bwd_rows(AttnArgs a)
{
    constexpr int NW = 4, TH = 256, BN = 32, DVT = 2 * DT;
    typedef Tile<T, BN, DVT> In;                       // (keys and values alike)
    constexpr int KS = DT / 16, VS = DVT / 16, NT = DT / 32;
    typedef typename Frag<T>::type frag;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    bf16* kt = (bf16*)lds;
    bf16* vt = kt + In::SIZE;
    uint32_t* words = (uint32_t*)(vt + In::SIZE);      // [2]

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int tile = a.row_tiles - 1 - blockIdx.x / bh_all;
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int mine = tile * 32 * NW + 32 * w + (l & 31), r = min(mine, a.rows - 1), i = r / a.G, g = r - i * a.G;
    const int head = hk * a.G + g, n = keys_of(a, b);
    const int64_t stat = ((int64_t)b * a.H + head) * a.Sq + i, half = (int64_t)a.B * a.H * a.Sq;
    const float lse0 = a.lse_in[stat] * LOG2E, lse1 = a.lse_in[half + stat] * LOG2E;
    const float d0 = a.delta[stat], d1 = a.delta[half + stat], lam = a.lam[head];
    const bool none = lse0 == -INFINITY;
    const int see = limit_of(a, i, n), lim = none ? 0 : see;
    // (limits of the rows rise; a row that the mask leaves empty only makes its wavefront test every key)
    const int wmin = __any(none) ? 0 : __builtin_amdgcn_readfirstlane(see), wmax = __builtin_amdgcn_readlane(see, 31);
    const int k0 = blockIdx.y * a.row_keys, k1 = min(limit_of(a, min(tile * 32 * NW + 32 * NW - 1, a.rows - 1) / a.G, n), k0 + a.row_keys);
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_b : nullptr;

    frag qf[2][KS], gf[VS];
    const T* q = (const T*)a.q + b * a.q_b + i * a.q_s + (int64_t)head * 2 * a.q_h;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[m][s] = global_frag<VEC>(q + m * a.q_h, 16 * s + 8 * h, a.D);
    const T* go = (const T*)a.dout + (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv;
#pragma unroll
    for (int s = 0; s < VS; ++s) gf[s] = global_frag<VEC>(go, 16 * s + 8 * h, a.Dv);

    f32x16 acc[2][NT];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][t][e] = 0.0f;
    float spread = 0.0f;                               // sum_j A_2 G

    const T* kb = (const T*)a.k + b * a.k_b + (int64_t)hk * 2 * a.k_h;
    const T* vb = (const T*)a.v + b * a.v_b + (int64_t)hk * a.v_h;
    Stage<T, VEC, BN, 2, DT, TH> ks;
    Stage<T, VEC, BN, 1, DVT, TH> vs;
    uint8_t seen = 1;
    const auto fetch = [&](int j0) {
        ks.load(kb, a.k_s, a.k_h, j0, n, a.D);
        vs.load(vb, a.v_s, 0, j0, n, a.Dv);
        if (mask && threadIdx.x < BN) seen = mask[min(j0 + (int)threadIdx.x, n - 1)];
    };
    if (k0 < k1) fetch(k0);
    const int kcol = col_lane<In::LD>();
    int turn = 0;
    for (int j0 = k0; j0 < k1; j0 += BN, turn ^= 1) {
        const bool whole = !mask && j0 + BN <= n;
        uint32_t* wd = words + turn;
        if (!whole && threadIdx.x < BN) {
            const uint64_t there = __ballot(j0 + (int)threadIdx.x < n && seen);
            if (l == 0) wd[0] = (uint32_t)there;
        }
        __syncthreads();
        ks.store(kt, whole ? nullptr : wd, a.D);
        vs.store(vt, whole ? nullptr : wd, a.Dv);
        __syncthreads();
        if (j0 + BN < k1) fetch(j0 + BN);
        if (j0 >= wmax) continue;
        f32x16 s0, s1, gt;
#pragma unroll
        for (int e = 0; e < 16; ++e) s0[e] = s1[e] = gt[e] = 0.0f;
        const bf16* krow = kt + (l & 31) * In::LD + 8 * h;
        const bf16* vrow = vt + (l & 31) * In::LD + 8 * h;
#pragma unroll
        for (int t = 0; t < KS; ++t) s0 = mma(s0, tile_row<T, In::PLANE>(krow + 16 * t), qf[0][t]);
#pragma unroll
        for (int t = 0; t < KS; ++t) s1 = mma(s1, tile_row<T, In::PLANE>(krow + DT + 16 * t), qf[1][t]);
#pragma unroll
        for (int t = 0; t < VS; ++t) gt = mma(gt, tile_row<T, In::PLANE>(vrow + 16 * t), gf[t]);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s0[e] = __builtin_amdgcn_exp2f(fmaf(s0[e], a.scale2, -lse0));
            s1[e] = __builtin_amdgcn_exp2f(fmaf(s1[e], a.scale2, -lse1));
        }
        const uint32_t word = whole ? ~0u : wd[0];
        if (j0 + 32 > wmin || (mask && word != ~0u)) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int j = 8 * (e >> 2) + 4 * h + (e & 3);
                const bool ok = j0 + j < lim && (word >> j & 1);
                s0[e] = ok ? s0[e] : 0.0f;
                s1[e] = ok ? s1[e] : 0.0f;
                gt[e] = ok ? gt[e] : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            spread = fmaf(s1[e], gt[e], spread);
            s0[e] *= gt[e] - d0;
            s1[e] *= -lam * (gt[e] - d1);
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                acc[0][t] = mma_fine<T, In>(acc[0][t], kt + kcol + 16 * st * In::LD + 32 * t, s0, st);
                acc[1][t] = mma_fine<T, In>(acc[1][t], kt + kcol + 16 * st * In::LD + DT + 32 * t, s1, st);
            }
        }
        settle();
    }
    rows_end<T, NT>(a, b, i, head, mine, h, stat, spread, acc);
}

// WHAT: 1: dv, 2: dk of the first map, 4: of the second (all three where their sums fit the registers).
template <typename T, bool VEC, int DT, int WHAT>
__global__ __launch_bounds__(256) void attn_bwd_keys(AttnArgs a)
{
    constexpr int NW = 4, TH = 256, BM = 32, DVT = 2 * DT;
    typedef Tile<T, BM, DVT> In;                       // (queries and dout alike)
    constexpr int KS = DT / 16, VS = DVT / 16, NT = DT / 32, VT = DVT / 32;
    constexpr bool DV = WHAT & 1, DK0 = WHAT & 2, DK1 = WHAT & 4, MAP0 = DV || DK0, MAP1 = DV || DK1, NEED_G = DK0 || DK1;
    typedef typename Frag<T>::type frag;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    bf16* qt = (bf16*)lds;
    bf16* gt = qt + In::SIZE;
    float* stats = (float*)(gt + In::SIZE);            // [2][4][32]: lse of both maps (log2), d of both
    uint32_t* words = (uint32_t*)(stats + 256);        // [2]

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int j0 = (int)(blockIdx.x / bh_all) * 32 * NW;
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int n = keys_of(a, b), j = j0 + 32 * w + (l & 31), in = min(j, a.Sk - 1);
    const bool ok = j < n && (!a.mask || a.mask[b * a.mask_b + in]);
    const bool all_ok = __all(ok);
    // the first query that sees a key, of this lane's key, the wavefront's and the workgroup's first one; the wavefront's last
    const int64_t off = (int64_t)a.Sq - n;
    const int seen_by = a.causal ? (int)std::max<int64_t>(0, j + off) : 0;
    const int wfirst = __builtin_amdgcn_readfirstlane(seen_by), wlast = __builtin_amdgcn_readlane(seen_by, 31);
    const int start = a.causal ? (int)std::max<int64_t>(0, j0 + off) / BM * BM : 0;

    frag kf[2][KS], vf[VS];
    const T* k = (const T*)a.k + b * a.k_b + in * a.k_s + (int64_t)hk * 2 * a.k_h;
    const T* v = (const T*)a.v + b * a.v_b + in * a.v_s + (int64_t)hk * a.v_h;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        if (MAP0) kf[0][s] = global_frag<VEC>(k, 16 * s + 8 * h, a.D);
        if (MAP1) kf[1][s] = global_frag<VEC>(k + a.k_h, 16 * s + 8 * h, a.D);
    }
    if (NEED_G)
#pragma unroll
        for (int s = 0; s < VS; ++s) vf[s] = global_frag<VEC>(v, 16 * s + 8 * h, a.Dv);

    f32x16 dk[2][NT], dv[VT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[0][t][e] = dk[1][t][e] = 0.0f;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) dv[t][e] = 0.0f;

    Stage<T, VEC, BM, 2, DT, TH> qs;
    Stage<T, VEC, BM, 1, DVT, TH> gs;
    float stat = 0.0f, sum = 0.0f;
    const int64_t half = (int64_t)a.B * a.H * a.Sq;
    const auto fetch = [&](int g, int i0) {
        const int head = hk * a.G + g;
        qs.load((const T*)a.q + b * a.q_b + (int64_t)head * 2 * a.q_h, a.q_s, a.q_h, i0, a.Sq, a.D);
        gs.load((const T*)a.dout + ((int64_t)b * a.Sq * a.H + head) * a.Dv, (int64_t)a.H * a.Dv, 0, i0, a.Sq, a.Dv);
        if (threadIdx.x < 128) {                       // thread: statistic x row
            const int i = min(i0 + (int)(threadIdx.x & 31), a.Sq - 1), what = threadIdx.x >> 5;
            const int64_t at = ((int64_t)b * a.H + head) * a.Sq + i;
            sum = a.lse_in[at];
            stat = what == 0 ? sum * LOG2E : what == 1 ? a.lse_in[half + at] * LOG2E : a.delta[at + (what == 3 ? half : 0)];
        }
    };
    // this part of the (head, tile of queries) pairs
    const int per = start < a.Sq && j0 < n ? (a.Sq - start + BM - 1) / BM : 0;
    const int64_t pairs = (int64_t)per * a.G;
    int64_t left = pairs * (blockIdx.y + 1) / a.key_splits;
    const int64_t from = pairs * blockIdx.y / a.key_splits;
    left -= from;
    int g = per ? (int)(from / per) : 0, i0 = per ? start + (int)(from % per) * BM : 0;
    if (left > 0) fetch(g, i0);
    const int col = col_lane<In::LD>();
    int turn = 0;
    for (; left > 0; turn ^= 1) {
        float* st = stats + 128 * turn;
        if (threadIdx.x < 128) {
            // a row that is not there, or sees nothing, is cleared: its weights, all 1 then, meet zeros
            const bool there = i0 + (int)(threadIdx.x & 31) < a.Sq && sum != -INFINITY;
            st[threadIdx.x] = there ? stat : 0.0f;
            const uint64_t bits = __ballot(there);
            if (threadIdx.x == 0) words[turn] = (uint32_t)bits;
        }
        __syncthreads();
        qs.store(qt, words + turn, a.D);
        gs.store(gt, words + turn, a.Dv);
        __syncthreads();
        const int at = i0;
        const float lam = a.lam[hk * a.G + g];
        i0 += BM;
        if (i0 >= a.Sq) { i0 = start; ++g; }
        if (--left > 0) fetch(g, i0);
        if (at + BM <= wfirst || j0 + 32 * w >= n) continue;
        f32x16 s0, s1, gg;
#pragma unroll
        for (int e = 0; e < 16; ++e) s0[e] = s1[e] = gg[e] = 0.0f;
        const bf16* qrow = qt + (l & 31) * In::LD + 8 * h;
        const bf16* grow = gt + (l & 31) * In::LD + 8 * h;
        if (MAP0)
#pragma unroll
            for (int t = 0; t < KS; ++t) s0 = mma(s0, tile_row<T, In::PLANE>(qrow + 16 * t), kf[0][t]);
        if (MAP1)
#pragma unroll
            for (int t = 0; t < KS; ++t) s1 = mma(s1, tile_row<T, In::PLANE>(qrow + DT + 16 * t), kf[1][t]);
        if (NEED_G)
#pragma unroll
            for (int t = 0; t < VS; ++t) gg = mma(gg, tile_row<T, In::PLANE>(grow + 16 * t), vf[t]);
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const f32x4 l0 = *(const f32x4*)(st + 2 * e + 4 * h), l1 = *(const f32x4*)(st + 32 + 2 * e + 4 * h);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                if (MAP0) s0[e + z] = __builtin_amdgcn_exp2f(fmaf(s0[e + z], a.scale2, -l0[z]));
                if (MAP1) s1[e + z] = __builtin_amdgcn_exp2f(fmaf(s1[e + z], a.scale2, -l1[z]));
            }
        }
        if (!all_ok || at < wlast) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool in_sum = ok && at + 8 * (e >> 2) + 4 * h + (e & 3) >= seen_by;
                s0[e] = in_sum ? s0[e] : 0.0f;
                s1[e] = in_sum ? s1[e] : 0.0f;
                gg[e] = in_sum ? gg[e] : 0.0f;
            }
        }
        if (DV) {
            f32x16 p;
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = fmaf(-lam, s1[e], s0[e]);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                frag f;
                to_frag(p, x, f);
#pragma unroll
                for (int t = 0; t < VT; ++t) dv[t] = mma(dv[t], tile_col<T, In::LD, In::PLANE>(gt + col + 16 * x * In::LD + 32 * t), f);
            }
        }
        if (NEED_G) {
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4 d0 = *(const f32x4*)(st + 64 + 2 * e + 4 * h), d1 = *(const f32x4*)(st + 96 + 2 * e + 4 * h);
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    s0[e + z] *= gg[e + z] - d0[z];
                    s1[e + z] *= -lam * (gg[e + z] - d1[z]);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if (DK0) dk[0][t] = mma_fine<T, In>(dk[0][t], qt + col + 16 * x * In::LD + 32 * t, s0, x);
                    if (DK1) dk[1][t] = mma_fine<T, In>(dk[1][t], qt + col + 16 * x * In::LD + DT + 32 * t, s1, x);
                }
            }
        }
        settle();
    }
    keys_end<T, NT, VT, WHAT>(a, b, hk, j, h, dk, dv);
}

// The same two in 16 bits, whole vectors everywhere, whose tiles go to LDS directly.
template <int DT>
__global__ __launch_bounds__(256, 2) void attn_rows_direct(AttnArgs a)
{
    constexpr int NW = 4, BN = 64, NB = BN / 32, DVT = 2 * DT, KS = DT / 16, VS = DVT / 16, NT = DT / 32, TILE = BN * 2 * DVT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    bf16* tiles = (bf16*)lds;
    uint32_t* words = (uint32_t*)(tiles + 2 * TILE);   // [3][NB]

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int tile = a.row_tiles - 1 - blockIdx.x / bh_all;
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int mine = tile * 32 * NW + 32 * w + (l & 31), r = min(mine, a.rows - 1), i = r / a.G, g = r - i * a.G;
    const int head = hk * a.G + g, n = keys_of(a, b);
    const int64_t stat = ((int64_t)b * a.H + head) * a.Sq + i, half = (int64_t)a.B * a.H * a.Sq;
    const float lse0 = a.lse_in[stat] * LOG2E, lse1 = a.lse_in[half + stat] * LOG2E;
    const float d0 = a.delta[stat], d1 = a.delta[half + stat], lam = a.lam[head];
    const bool none = lse0 == -INFINITY;
    const int see = limit_of(a, i, n), lim = none ? 0 : see;
    const int wmin = __any(none) ? 0 : __builtin_amdgcn_readfirstlane(see), wmax = __builtin_amdgcn_readlane(see, 31);
    const int k0 = blockIdx.y * a.row_keys, k1 = min(limit_of(a, min(tile * 32 * NW + 32 * NW - 1, a.rows - 1) / a.G, n), k0 + a.row_keys);
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_b : nullptr;

    bf16x8 qf[2][KS], gf[VS];
    const bf16* q = (const bf16*)a.q + b * a.q_b + i * a.q_s + (int64_t)head * 2 * a.q_h;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[m][s] = row_frag(q + m * a.q_h + 16 * s + 8 * h);
    const bf16* go = (const bf16*)a.dout + (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv;
#pragma unroll
    for (int s = 0; s < VS; ++s) gf[s] = row_frag(go + 16 * s + 8 * h);

    f32x16 acc[2][NT];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][t][e] = 0.0f;
    float spread = 0.0f;

    const bf16* kb = (const bf16*)a.k + b * a.k_b + (int64_t)hk * 2 * a.k_h;
    const bf16* vb = (const bf16*)a.v + b * a.v_b + (int64_t)hk * a.v_h;
    typedef Direct<BN, 2, DT, NW> Keys;
    typedef Direct<BN, 1, DVT, NW> Values;
    Keys kd;
    Values vd;
    kd.init(a.k_s, a.k_h);
    vd.init(a.v_s, 0);
    int row4[4], col2[2];                              // (both tiles' rows have 2 DT elements)
    Keys::row_lane(row4);
    Keys::col_lane(col2);
    uint8_t seen = 1;
    const auto fetch = [&](int j0, int turn) {
        bf16* kt = tiles + turn * TILE;
        kd.load(kb, a.k_s, a.k_h, j0, n, kt);
        vd.load(vb, a.v_s, 0, j0, n, kt + BN * DVT);
    };
    const auto fetch_mask = [&](int j0) { if (mask && threadIdx.x < BN) seen = mask[min(j0 + (int)threadIdx.x, n - 1)]; };
    const auto mark = [&](int j0, int slot) {
        if (mask && threadIdx.x < BN) {
            const uint64_t there = __ballot(j0 + (int)threadIdx.x < n && seen);
            if (threadIdx.x < NB) words[slot * NB + threadIdx.x] = (uint32_t)(threadIdx.x ? there >> 32 : there);
        }
    };
    const auto after = [](int slot) { return slot == 2 ? 0 : slot + 1; };
    int turn = 0, slot = 0;
    if (k0 < k1) {
        fetch(k0, 0);
        fetch_mask(k0);
        mark(k0, 0);
        if (k0 + BN < k1) { fetch_mask(k0 + BN); mark(k0 + BN, 1); }
    }
    for (int j0 = k0; j0 < k1; j0 += BN, turn ^= 1, slot = after(slot)) {
        Keys::arrived();
        __syncthreads();
        if (j0 + BN < k1) fetch(j0 + BN, turn ^ 1);
        if (j0 + 2 * BN < k1) fetch_mask(j0 + 2 * BN);
        bf16* kt = tiles + turn * TILE;
        bf16* vt = kt + BN * DVT;
        const uint32_t* wd = words + slot * NB;
        if (mask) {
            bool all = true;
#pragma unroll
            for (int x = 0; x < NB; ++x) all = all && wd[x] == ~0u;
            if (!all) {
                Keys::clear(kt, wd);
                Values::clear(vt, wd);
                __syncthreads();
            }
        }
#pragma unroll 1
        for (int x = 0; x < NB; ++x) {
            const int js = j0 + 32 * x;
            const uint32_t word = mask ? __builtin_amdgcn_readfirstlane(wd[x]) : ~0u;
            if (js >= wmax || word == 0) continue;
            const bf16* ks = kt + 32 * x * DVT;
            const bf16* vs = vt + 32 * x * DVT;
            f32x16 s0, s1, gt;
#pragma unroll
            for (int e = 0; e < 16; ++e) s0[e] = s1[e] = gt[e] = 0.0f;
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const int c0 = 16 * t, c1 = DT + 16 * t;
                s0 = mma(s0, row_frag(ks + row4[c0 / 16 % 4] + c0 / 64 * 64), qf[0][t]);
                s1 = mma(s1, row_frag(ks + row4[c1 / 16 % 4] + c1 / 64 * 64), qf[1][t]);
            }
#pragma unroll
            for (int t = 0; t < VS; ++t) gt = mma(gt, row_frag(vs + row4[t % 4] + t / 4 * 64), gf[t]);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s0[e] = __builtin_amdgcn_exp2f(fmaf(s0[e], a.scale2, -lse0));
                s1[e] = __builtin_amdgcn_exp2f(fmaf(s1[e], a.scale2, -lse1));
            }
            if (js + 32 > wmin || word != ~0u) {
                const uint32_t bits = seen_bits(js, lim, word) >> (4 * h);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int pos = 8 * (e >> 2) + (e & 3);
                    s0[e] = masked(s0[e], bits, pos, 0);
                    s1[e] = masked(s1[e], bits, pos, 0);
                    gt[e] = masked(gt[e], bits, pos, 0);
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float gv = gt[8 * st + e], p1 = s1[8 * st + e];
                        if (m) spread = fmaf(p1, gv, spread);
                        x[e] = m ? p1 * (-lam * (gv - d1)) : s0[8 * st + e] * (gv - d0);
                    }
                    bf16x8 f, rest;
                    to_frag(x, f);
                    rest_frag(x, f, rest);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int c = m * DT + 32 * t;
                        acc[m][t] = mma_fine<DVT>(acc[m][t], ks + col2[c / 32 % 2] + c / 64 * 64 + 16 * st * DVT, f, rest);
                    }
                }
            }
            settle();
        }
        if (j0 + 2 * BN < k1) mark(j0 + 2 * BN, after(after(slot)));
    }
    rows_end<bf16, NT>(a, b, i, head, mine, h, stat, spread, acc);
}

// (keys: WHAT as above.  At DT = 64 the sums and operands of all three leave room for one wavefront a SIMD only, which waits for
// each of its own products; dv and dk apart form the weights twice, and are done sooner with two: 345 against 404 us.)  SUB:
// tiles of 32 queries whose products stand in one straight line.
template <int DT, int WHAT, int SUB>
__global__ __launch_bounds__(256, 2) void attn_keys_direct(AttnArgs a)
{
    constexpr bool DV = WHAT & 1, DK = WHAT & 6;
    constexpr int NW = 4, BM = 64, MB = BM / 32, DVT = 2 * DT, KS = DT / 16, VS = DVT / 16, NT = DT / 32, VT = DVT / 32;
    constexpr int TILE = BM * 2 * DVT;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    bf16* tiles = (bf16*)lds;
    // [2][4][BM]: lse of both maps (log2) and d of both; lam's size is taken into the second lse - |lam| A_2 = exp2(S_2 - it) - and
    // its sign into the second d
    float* stats = (float*)(tiles + 2 * TILE);
    uint32_t* words = (uint32_t*)(stats + 8 * BM);     // [2][MB]

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int j0 = (int)(blockIdx.x / bh_all) * 32 * NW;
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int n = keys_of(a, b), j = j0 + 32 * w + (l & 31), in = min(j, a.Sk - 1);
    const bool ok = j < n && (!a.mask || a.mask[b * a.mask_b + in]);
    const bool all_ok = __all(ok), any_ok = __any(ok);
    const int64_t off = (int64_t)a.Sq - n;
    const int seen_by = a.causal ? (int)std::max<int64_t>(0, j + off) : 0;
    const int wfirst = __builtin_amdgcn_readfirstlane(seen_by), wlast = __builtin_amdgcn_readlane(seen_by, 31);
    const int start = a.causal ? (int)std::max<int64_t>(0, j0 + off) / BM * BM : 0;

    bf16x8 kf[2][KS], vf[VS];
    const bf16* k = (const bf16*)a.k + b * a.k_b + in * a.k_s + (int64_t)hk * 2 * a.k_h;
    const bf16* v = (const bf16*)a.v + b * a.v_b + in * a.v_s + (int64_t)hk * a.v_h;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        kf[0][s] = row_frag(k + 16 * s + 8 * h);
        kf[1][s] = row_frag(k + a.k_h + 16 * s + 8 * h);
    }
    if (DK)
#pragma unroll
    for (int s = 0; s < VS; ++s) vf[s] = row_frag(v + 16 * s + 8 * h);

    f32x16 dk[2][NT], dv[VT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[0][t][e] = dk[1][t][e] = 0.0f;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) dv[t][e] = 0.0f;

    typedef Direct<BM, 2, DT, NW> Queries;
    typedef Direct<BM, 1, DVT, NW> Grads;
    Queries qd;
    Grads gd;
    const int64_t g_s = (int64_t)a.H * a.Dv;
    qd.init(a.q_s, a.q_h);
    gd.init(g_s, 0);
    int row4[4], col2[2];
    Queries::row_lane(row4);
    Queries::col_lane(col2);
    float stat = 0.0f, sum = 0.0f;
    const int64_t half = (int64_t)a.B * a.H * a.Sq;
    const auto fetch = [&](int g, int i0, int turn) {
        const int head = hk * a.G + g;
        bf16* qt = tiles + turn * TILE;
        qd.load((const bf16*)a.q + b * a.q_b + (int64_t)head * 2 * a.q_h, a.q_s, a.q_h, i0, a.Sq, qt);
        gd.load((const bf16*)a.dout + ((int64_t)b * a.Sq * a.H + head) * a.Dv, g_s, 0, i0, a.Sq, qt + BM * DVT);
        // thread: statistic x row
        const int i = min(i0 + (int)(threadIdx.x % BM), a.Sq - 1), what = threadIdx.x / BM;
        const int64_t at = ((int64_t)b * a.H + head) * a.Sq + i;
        const float lam = a.lam[head];
        sum = a.lse_in[at];
        stat = what == 0 ? sum * LOG2E : what == 1 ? a.lse_in[half + at] * LOG2E - log2f(fabsf(lam)) : a.delta[at + (what == 3 ? half : 0)];
        if (what == 3) stat = copysignf(1.0f, lam) * stat;
    };
    const auto mark = [&](int i0, int turn) {
        const bool there = i0 + (int)(threadIdx.x % BM) < a.Sq && sum != -INFINITY;
        stats[turn * 4 * BM + threadIdx.x] = there ? stat : 0.0f;
        const uint64_t bits = __ballot(there);
        if (threadIdx.x < MB) words[turn * MB + threadIdx.x] = (uint32_t)(threadIdx.x ? bits >> 32 : bits);
    };
    // this part of the (head, tile of queries) pairs
    const int per = start < a.Sq && j0 < n ? (a.Sq - start + BM - 1) / BM : 0;
    const int64_t pairs = (int64_t)per * a.G;
    int64_t left = pairs * (blockIdx.y + 1) / a.key_splits;
    const int64_t from = pairs * blockIdx.y / a.key_splits;
    left -= from;
    int turn = 0, g = per ? (int)(from / per) : 0, i0 = per ? start + (int)(from % per) * BM : 0;
    if (left > 0) { fetch(g, i0, 0); mark(i0, 0); }
    while (left > 0) {
        Queries::arrived();
        __syncthreads();
        const int at = i0, was = g;
        i0 += BM;
        if (i0 >= a.Sq) { i0 = start; ++g; }
        if (--left > 0) fetch(g, i0, turn ^ 1);
        bf16* qt = tiles + turn * TILE;
        bf16* gt = qt + BM * DVT;
        bool whole = true;
#pragma unroll
        for (int x = 0; x < MB; ++x) whole = whole && words[turn * MB + x] == ~0u;
        if (!whole) {                                  // rows that see nothing may hold anything
            Queries::clear(qt, words + turn * MB);
            Grads::clear(gt, words + turn * MB);
            __syncthreads();
        }
        const float sign = -copysignf(1.0f, a.lam[hk * a.G + was]);   // of the second map
#pragma unroll 1
        for (int x0 = 0; x0 < MB; x0 += SUB) {
            const int is = at + 32 * x0;
            if (is + 32 * SUB <= wfirst || is >= a.Sq || !any_ok) continue;
            const float* st = stats + turn * 4 * BM + 32 * x0 + 4 * h;
            const bf16* qx = qt + 32 * x0 * DVT;
            const bf16* gx = gt + 32 * x0 * DVT;
            f32x16 s0[SUB], s1[SUB], gg[SUB];
#pragma unroll
            for (int x = 0; x < SUB; ++x) {
                const bf16* qs = qx + 32 * x * DVT;
                const bf16* gs = gx + 32 * x * DVT;
#pragma unroll
                for (int e = 0; e < 16; ++e) s0[x][e] = s1[x][e] = gg[x][e] = 0.0f;
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    const int c0 = 16 * t, c1 = DT + 16 * t;
                    s0[x] = mma(s0[x], row_frag(qs + row4[c0 / 16 % 4] + c0 / 64 * 64), kf[0][t]);
                    s1[x] = mma(s1[x], row_frag(qs + row4[c1 / 16 % 4] + c1 / 64 * 64), kf[1][t]);
                }
                if (DK)
#pragma unroll
                    for (int t = 0; t < VS; ++t) gg[x] = mma(gg[x], row_frag(gs + row4[t % 4] + t / 4 * 64), vf[t]);
            }
#pragma unroll
            for (int x = 0; x < SUB; ++x)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 l0 = *(const f32x4*)(st + 32 * x + 2 * e), l1 = *(const f32x4*)(st + 32 * x + BM + 2 * e);
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        s0[x][e + z] = __builtin_amdgcn_exp2f(fmaf(s0[x][e + z], a.scale2, -l0[z]));
                        s1[x][e + z] = __builtin_amdgcn_exp2f(fmaf(s1[x][e + z], a.scale2, -l1[z]));
                    }
                }
            if (!all_ok || is < wlast) {
#pragma unroll
                for (int x = 0; x < SUB; ++x) {
                    // rows from `from` on of this 32 see the lane's key
                    const int from = seen_by - is - 32 * x;
                    const uint32_t bits = (!ok || from >= 32 ? 0u : from <= 0 ? ~0u : ~0u << from) >> (4 * h);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int pos = 8 * (e >> 2) + (e & 3);
                        s0[x][e] = masked(s0[x][e], bits, pos, 0);
                        s1[x][e] = masked(s1[x][e], bits, pos, 0);
                        gg[x][e] = masked(gg[x][e], bits, pos, 0);
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < SUB; ++x) {
                const bf16* qs = qx + 32 * x * DVT;
                const bf16* gs = gx + 32 * x * DVT;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if (DV) {
                        bf16x8 f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = (bf16)fmaf(sign, s1[x][8 * y + e], s0[x][8 * y + e]);
#pragma unroll
                        for (int t = 0; t < VT; ++t)
                            dv[t] = mma(dv[t], col_frag<DVT>(gs + col2[t % 2] + t / 2 * 64 + 16 * y * DVT), f);
                    }
                    if (DK) {
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; e += 4) {
                                const f32x4 d = *(const f32x4*)(st + 32 * x + (2 + m) * BM + 2 * (8 * y + e));
#pragma unroll
                                for (int z = 0; z < 4; ++z) {
                                    const int u = 8 * y + e + z;
                                    v[e + z] = m ? s1[x][u] * fmaf(sign, gg[x][u], d[z]) : s0[x][u] * (gg[x][u] - d[z]);
                                }
                            }
                            bf16x8 f, rest;
                            to_frag(v, f);
                            rest_frag(v, f, rest);
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                const int c = m * DT + 32 * t;
                                dk[m][t] = mma_fine<DVT>(dk[m][t], qs + col2[c / 32 % 2] + c / 64 * 64 + 16 * y * DVT, f, rest);
                            }
                        }
                    }
                }
            }
            settle();
        }
        if (left > 0) mark(i0, turn ^ 1);
        turn ^= 1;
    }
    keys_end<bf16, NT, VT, WHAT>(a, b, hk, j, h, dk, dv);
}

template <typename T, bool VEC, int DT, int WHAT>
int keys_launch(const AttnArgs& a, hipStream_t stream)
{
    constexpr size_t lds = (size_t)2 * Tile<T, 32, 2 * DT>::SIZE * 2 + 256 * 4 + 8;
    const int rc = allow_lds(attn_bwd_keys<T, VEC, DT, WHAT>, lds);
    if (rc) return rc;
    const int64_t grid = (int64_t)((a.Sk + 127) / 128) * a.B * a.Hkv;
    hipLaunchKernelGGL((attn_bwd_keys<T, VEC, DT, WHAT>), dim3((unsigned)grid, (unsigned)a.key_splits), dim3(256), lds, stream, a);
    return launch_status();
}

template <int DT, int WHAT, int SUB>
int keys_direct_launch(const AttnArgs& a, hipStream_t stream)
{
    constexpr size_t lds = (size_t)2 * 64 * 4 * DT * sizeof(bf16) + 8 * 64 * 4 + 4 * 4;
    const int rc = allow_lds(attn_keys_direct<DT, WHAT, SUB>, lds);
    if (rc) return rc;
    hipLaunchKernelGGL((attn_keys_direct<DT, WHAT, SUB>), dim3((unsigned)((int64_t)((a.Sk + 127) / 128) * a.B * a.Hkv), (unsigned)a.key_splits),
                       dim3(256), lds, stream, a);
    return launch_status();
}

template <int DT>
int direct_main(const AttnArgs& a, hipStream_t stream)
{
    int rc;
    if constexpr (DT == 32) rc = keys_direct_launch<DT, 7, 1>(a, stream);
    else {
        rc = keys_direct_launch<DT, 1, 2>(a, stream);
        if (!rc) rc = keys_direct_launch<DT, 6, 1>(a, stream);
    }
    if (rc) return rc;
    constexpr size_t lds = (size_t)2 * 64 * 4 * DT * sizeof(bf16) + 3 * 2 * 4;
    rc = allow_lds(attn_rows_direct<DT>, lds);
    if (rc) return rc;
    hipLaunchKernelGGL((attn_rows_direct<DT>), dim3((unsigned)((int64_t)a.row_tiles * a.B * a.Hkv), (unsigned)a.row_splits), dim3(256), lds, stream, a);
    return launch_status();
}

template <typename T, bool VEC, int DT>
int bwd_main(const AttnArgs& a, hipStream_t stream)
{
    int rc = SCONV_OK;
    if constexpr (VEC && sizeof(T) == 2 && DT <= 64) {
        // (tiles' rows beside each other, and within what a buffer's offsets reach)
        const int64_t far = int64_t(1) << 22;
        if (a.Sq > 0 && a.Sk > 0 && a.D == DT && a.Dv == 2 * DT && a.k_h + DT <= a.k_s && a.q_h + DT <= a.q_s && a.v_s >= a.Dv &&
            a.k_s < far && a.q_s < far && a.v_s < far && (int64_t)a.H * a.Dv < far)
            return direct_main<DT>(a, stream);
    }
    if (a.Sk > 0) {
        if constexpr (DT <= 64) rc = keys_launch<T, VEC, DT, 7>(a, stream);
        else {
            // (the three sums of 128 columns and their operands do not fit a lane's registers together)
            rc = keys_launch<T, VEC, DT, 1>(a, stream);
            if (!rc) rc = keys_launch<T, VEC, DT, 2>(a, stream);
            if (!rc) rc = keys_launch<T, VEC, DT, 4>(a, stream);
        }
        if (rc) return rc;
    }
    if (a.Sq == 0) return rc;
    constexpr size_t lds = (size_t)2 * Tile<T, 32, 2 * DT>::SIZE * 2 + 8;
    rc = allow_lds(attn_bwd_rows<T, VEC, DT>, lds);
    if (rc) return rc;
    hipLaunchKernelGGL((attn_bwd_rows<T, VEC, DT>), dim3((unsigned)((int64_t)a.row_tiles * a.B * a.Hkv), (unsigned)a.row_splits), dim3(256), lds, stream, a);
    return launch_status();
}

template <typename T, bool VEC>
int bwd_run(const AttnArgs& a, float* dlam, hipStream_t stream)
{
    int rc;
    if (a.Sq > 0) {
        const dim3 grid((unsigned)(((int64_t)a.B * a.Sq * a.H + 15) / 16));
        if (a.Dv % 4 == 0 && aligned_to(a.dout, 16) && aligned_to(a.out_in, 16) && aligned_to(a.second_in, 16)) hipLaunchKernelGGL((attn_delta<T, 4>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((attn_delta<T, 1>), grid, dim3(256), 0, stream, a);
        rc = launch_status();
        if (rc) return rc;
    }
    const int most = std::max(a.D, (a.Dv + 1) / 2);
    if (most <= 32) rc = bwd_main<T, VEC, 32>(a, stream);
    else if (most <= 64) rc = bwd_main<T, VEC, 64>(a, stream);
    else rc = bwd_main<T, VEC, 128>(a, stream);
    if (rc) return rc;
    PartSums p = {};
    int64_t all = 0;
    const auto add = [&](int w, const float* from, void* to, int64_t n, int splits, float scale, bool wide) {
        if (splits < 2) return;
        p.from[w] = from; p.to[w] = to; p.n[w] = n; p.splits[w] = splits; p.scale[w] = scale; p.wide[w] = wide;
        all += n;
    };
    const int64_t queries = (int64_t)a.B * a.Sq * a.H, keys = (int64_t)a.B * a.Sk * a.Hkv;
    add(0, a.part_q, a.dq, queries * 2 * a.D, a.row_splits, a.scale, false);
    add(1, a.part_k, a.dk, keys * 2 * a.D, a.key_splits, a.scale, false);
    add(2, a.part_v, a.dv, keys * a.Dv, a.key_splits, 1.0f, false);
    add(3, a.part_s, a.dlam_part, queries, a.row_splits, 1.0f, true);
    if (all > 0) {
        hipLaunchKernelGGL((attn_add_parts<T>), dim3((unsigned)std::min<int64_t>((all + 255) / 256, 1 << 20)), dim3(256), 0, stream, p, all);
        rc = launch_status();
        if (rc) return rc;
    }
    hipLaunchKernelGGL(attn_dlam, dim3((unsigned)a.H), dim3(1024), 0, stream, a.dlam_part, a.B, a.H, a.Sq, dlam);
    return launch_status();
}

}  // namespace

namespace {

// Parts where the workgroups of a kernel do not fill the chip: of the keys for dq, of the (head, tile of queries) pairs for dk and dv; up to
// a workgroup a compute unit, two tiles a part at least.
struct BwdPlan { int row_splits, row_keys, key_splits; size_t rows, q, s, k, v; };

BwdPlan bwd_plan(const sconv_diffattn_desc_t& d)
{
    BwdPlan p = {1, d.Sk > 0 ? d.Sk : 1, 1, 0, 0, 0, 0, 0};
    const int64_t G = d.H / d.Hkv, bh = (int64_t)d.B * d.Hkv, queries = (int64_t)d.B * d.Sq * d.H, keys = bh * d.Sk;
    p.rows = (size_t)(3 * queries) * sizeof(float);
    if (queries == 0 || keys == 0) return p;
    const int64_t row_blocks = (d.Sq * G + 127) / 128 * bh, key_blocks = ((int64_t)d.Sk + 127) / 128 * bh;
    const int64_t row = std::min<int64_t>(256 / row_blocks, d.Sk / 128), key = std::min<int64_t>(256 / key_blocks, G * ((d.Sq + 63) / 64) / 2);
    if (row > 1) {
        p.row_keys = (int)((d.Sk + row - 1) / row + 63) / 64 * 64;
        p.row_splits = (d.Sk + p.row_keys - 1) / p.row_keys;
    }
    if (key > 1) p.key_splits = (int)key;
    const auto whole = [](int64_t floats) { return (size_t)((floats + 3) / 4 * 4) * sizeof(float); };    // (16-byte steps)
    p.rows = whole(3 * queries);
    if (p.row_splits > 1) { p.q = whole(p.row_splits * queries * 2 * d.D); p.s = whole(p.row_splits * queries); }
    if (p.key_splits > 1) { p.k = whole(p.key_splits * keys * 2 * d.D); p.v = whole(p.key_splits * keys * d.Dv); }
    return p;
}

}  // namespace

size_t diffattn_backward_workspace(const sconv_diffattn_desc_t& d)
{
    const BwdPlan p = bwd_plan(d);
    return p.rows + p.q + p.s + p.k + p.v;
}

int launch_diffattn_backward(const sconv_diffattn_desc_t& d, const void* dout, const void* q, const void* k, const void* v,
                             const float* lam, const int32_t* lengths, const uint8_t* mask, const void* out,
                             const void* second, const float* lse, void* dq, void* dk, void* dv, float* dlam, void* ws,
                             hipStream_t stream)
{
    AttnArgs a = attn_args(d, q, k, v, lam, lengths, mask);
    const bool vec = attn_vector(a, d.type) && aligned_to(dout, 16);
    a.dout = dout; a.out_in = out; a.second_in = second; a.lse_in = lse;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.ovec = aligned_to(dq, 16) && aligned_to(dk, 16) && aligned_to(dv, 16);
    a.delta = (float*)ws;
    a.dlam_part = a.delta + 2 * (int64_t)d.B * d.H * d.Sq;
    a.row_tiles = (a.rows + 127) / 128;
    const BwdPlan p = bwd_plan(d);
    a.row_splits = p.row_splits; a.row_keys = p.row_keys; a.key_splits = p.key_splits;
    char* at = (char*)ws + p.rows;
    a.part_q = (float*)at;
    a.part_s = (float*)(at += p.q);
    a.part_k = (float*)(at += p.s);
    a.part_v = (float*)(at += p.k);
    if (d.B == 0) a.Sq = a.Sk = 0;                     // nothing but lam's gradient to clear
    if (d.type == SCONV_BF16) return vec ? bwd_run<bf16, true>(a, dlam, stream) : bwd_run<bf16, false>(a, dlam, stream);
    return vec ? bwd_run<float, true>(a, dlam, stream) : bwd_run<float, false>(a, dlam, stream);
}

}  // namespace sconv
