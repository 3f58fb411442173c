// Differential attention, forward (formulas in sconv_tokens.h, product layout in sconv_diffattn_common.h).
//
// One pass over the keys with a running maximum and sum for each of the two maps.  The rows of a tile are (query, head of the
// group) pairs, so heads that share keys share their tiles, and a single token's heads fill one tile.  A key tile's values are
// read once for both maps.
//   wide   128 rows a workgroup, 32 a wavefront; every wavefront walks all keys of the tile.
//   few    32 rows a workgroup: its wavefronts take 32 keys each of a tile of 128, and join at the end.
// Either may split the keys over workgroups, whose parts a second kernel joins in a fixed order.
// Weights are rounded to the operands' type for their product with the values; the sums they are divided by are of the
// unrounded ones, in 32 bits.
#include <math.h>

#include <algorithm>

#include "sconv_diffattn_common.h"

namespace sconv {

namespace {

// One softmax over 32 more keys: s becomes the weights against the running maximum top (kept safe: 0 while nothing was seen),
// l the lane's part of the sum.  The maximum follows only when it has grown by 2^8: until then weights are at most 256, and
// sums stay exact to their 24 bits all the same.
template <int NT>
__device__ __forceinline__ void soften(f32x16& s, float scale2, float& top, float& safe, float& l, f32x16 (&o)[NT])
{
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = half_max(mx) * scale2;
    if (__any(mx > top + 8.0f)) {
        const float grown = fmaxf(top, mx);
        safe = grown == -INFINITY ? 0.0f : grown;
        const float f = __builtin_amdgcn_exp2f(top - safe);
        top = grown;
        l *= f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= f;
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale2, -safe));
        sum += s[i];
    }
    l += sum;
}


template <typename T, int DT, int DVT, int NW, bool FEW>
struct FwdShape {
    static constexpr int BN = FEW ? 32 * NW : 32;
    static constexpr int ROWS = FEW ? 32 : 32 * NW;
    static constexpr int BUFS = FEW ? 1 : 2;           // a wide workgroup writes one tile while it reads the other
    static constexpr int WAVES = !FEW && sizeof(T) == 2 && DT <= 64 ? 2 : 1;
    static constexpr int TILE = BN * (Tile<T, 2 * DT>::LD + Tile<T, DVT>::LD);
    static constexpr size_t LDS = (size_t)BUFS * TILE * sizeof(T) + 3 * (BN / 32) * 4;
};

template <typename T, bool VEC, int DT, int DVT, int NW, bool FEW>
__global__ __launch_bounds__(64 * NW, (FwdShape<T, DT, DVT, NW, FEW>::WAVES)) void attn_fwd(AttnArgs a)
{
    typedef FwdShape<T, DT, DVT, NW, FEW> Shape;
    constexpr int BN = Shape::BN, ROWS = Shape::ROWS;
    constexpr int KLD = Tile<T, 2 * DT>::LD, VLD = Tile<T, DVT>::LD, KS = DT / 16, NT = DVT / 32, TH = 64 * NW;
    typedef typename Frag<T>::type frag;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    T* tiles = (T*)lds;
    uint32_t* words = (uint32_t*)(tiles + Shape::BUFS * Shape::TILE);    // [3][BN / 32]: of the tile that is read, the next one and the one after

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int tile = a.row_tiles - 1 - blockIdx.x / bh_all;      // the rows that see most first
    const int split = blockIdx.y, dv0 = blockIdx.z * DVT, dvn = min(DVT, a.Dv - dv0);
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int first = tile * ROWS + (FEW ? 0 : 32 * w);
    const int mine = first + (l & 31), r = min(mine, a.rows - 1), i = r / a.G, g = r - i * a.G;
    const int n = keys_of(a, b);
    const int lim = limit_of(a, i, n);
    // limits rise with the rows: of this wavefront's first and last one, and of the workgroup's last one
    const int wmin = __builtin_amdgcn_readfirstlane(lim), wmax = __builtin_amdgcn_readlane(lim, 31);
    const int last = limit_of(a, min(tile * ROWS + ROWS - 1, a.rows - 1) / a.G, n);
    const int k0 = split * a.split_keys, k1 = (int)min((int64_t)last, (int64_t)k0 + a.split_keys);
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_b : nullptr;

    frag qf[2][KS];
    const T* q = (const T*)a.q + b * a.q_b + i * a.q_s + (int64_t)(hk * a.G + g) * 2 * a.q_h;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[m][s] = global_frag<VEC>(q + m * a.q_h, 16 * s + 8 * h, a.D);

    f32x16 o[2][NT];
    float top[2], safe[2], sum[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        top[m] = -INFINITY; safe[m] = 0.0f; sum[m] = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[m][t][e] = 0.0f;
    }

    const T* kb = (const T*)a.k + b * a.k_b + (int64_t)hk * 2 * a.k_h;
    const T* vb = (const T*)a.v + b * a.v_b + (int64_t)hk * a.v_h + dv0;
    Stage<T, VEC, BN, 2, DT, TH> ks;
    Stage<T, VEC, BN, 1, DVT, TH> vs;
    uint8_t seen = 1;
    const auto fetch = [&](int j0) {
        ks.load(kb, a.k_s, a.k_h, j0, n, a.D);
        vs.load(vb, a.v_s, 0, j0, n, dvn);
        if (mask && threadIdx.x < BN) seen = mask[min(j0 + (int)threadIdx.x, n - 1)];
    };
    // A tile on its way into LDS: which of its keys are there (words), then the rows.
    const auto mark = [&](int j0, int slot) {
        if ((mask || j0 + BN > n) && threadIdx.x < BN) {
            const uint64_t there = __ballot(j0 + (int)threadIdx.x < n && seen);
            uint32_t* wd = words + slot * (BN / 32);
            if (l == 0) wd[2 * w] = (uint32_t)there;
            if (l == 32) wd[2 * w + 1] = (uint32_t)(there >> 32);
        }
    };
    const auto put = [&](int j0, int turn, int slot) {
        T* kt = tiles + (Shape::BUFS > 1 ? turn : 0) * Shape::TILE;
        const uint32_t* wd = mask || j0 + BN > n ? words + slot * (BN / 32) : nullptr;
        ks.store(kt, wd, a.D);
        vs.store(kt + BN * KLD, wd, dvn);
    };
    const int vcol = col_lane<T, VLD>();
    const auto after = [](int slot) { return slot == 2 ? 0 : slot + 1; };
    int turn = 0, slot = 0;
    if (k0 < k1) {
        fetch(k0);
        mark(k0, 0);
        if (Shape::BUFS > 1) {
            if (mask || k0 + BN > n) __syncthreads();
            put(k0, 0, 0);
            if (k0 + BN < k1) { fetch(k0 + BN); mark(k0 + BN, 1); }
        }
    }
    for (int j0 = k0; j0 < k1; j0 += BN, turn ^= 1, slot = after(slot)) {
        const bool whole = !mask && j0 + BN <= n;
        const uint32_t* wd = words + slot * (BN / 32);
        __syncthreads();
        if (Shape::BUFS > 1) {
            // (this tile is there; the next one's keys were marked before the barrier)
            if (j0 + BN < k1) {
                put(j0 + BN, turn ^ 1, after(slot));
                if (j0 + 2 * BN < k1) fetch(j0 + 2 * BN);
            }
        } else {
            put(j0, 0, slot);
            __syncthreads();
            if (j0 + BN < k1) fetch(j0 + BN);
        }
        const T* kt = tiles + (Shape::BUFS > 1 ? turn : 0) * Shape::TILE;
        const T* vt = kt + BN * KLD;
#pragma unroll
        for (int sub = 0; sub < (FEW ? 1 : BN / 32); ++sub) {
            const int row0 = FEW ? 32 * w : 32 * sub, js = j0 + row0;
            if (js >= wmax) continue;
            f32x16 s[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[m][e] = 0.0f;
#pragma unroll
                for (int t = 0; t < KS; ++t)
                    s[m] = mma(s[m], row_frag(kt + (row0 + (l & 31)) * KLD + m * DT + 16 * t + 8 * h), qf[m][t]);
            }
            const uint32_t word = whole ? ~0u : wd[row0 >> 5];
            if (js + 32 > wmin || (mask && word != ~0u)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = 8 * (e >> 2) + 4 * h + (e & 3);
                    const bool ok = js + j < lim && (word >> j & 1);
                    s[0][e] = ok ? s[0][e] : -INFINITY;
                    s[1][e] = ok ? s[1][e] : -INFINITY;
                }
            }
            soften(s[0], a.scale2, top[0], safe[0], sum[0], o[0]);
            soften(s[1], a.scale2, top[1], safe[1], sum[1], o[1]);
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                frag p0, p1;
                to_frag(s[0], st, p0);
                to_frag(s[1], st, p1);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const frag vf = col_frag<VLD>(vt + vcol + (row0 + 16 * st) * VLD + 32 * t);
                    o[0][t] = mma(o[0][t], vf, p0);
                    o[1][t] = mma(o[1][t], vf, p1);
                }
            }
        }
        settle();
        if (Shape::BUFS > 1) { if (j0 + 2 * BN < k1) mark(j0 + 2 * BN, after(after(slot))); }
        else if (j0 + BN < k1) mark(j0 + BN, after(slot));
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) sum[m] = half_sum(sum[m]);

    if constexpr (FEW) {
        // the wavefronts' parts meet in LDS, over the tiles: statistics first, then the sums, halving the wavefronts
        __syncthreads();
        float* ml = (float*)lds;                       // [NW][2][2][32]
        float* acc = ml + NW * 128;                    // [NW / 2][2][DVT][32]
#pragma unroll
        for (int m = 0; m < 2; ++m)
            if (h == 0) { ml[(w * 4 + 2 * m) * 32 + l] = top[m]; ml[(w * 4 + 2 * m + 1) * 32 + l] = sum[m]; }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float most = -INFINITY;
#pragma unroll
            for (int k = 0; k < NW; ++k) most = fmaxf(most, ml[(k * 4 + 2 * m) * 32 + (l & 31)]);
            const float base = most == -INFINITY ? 0.0f : most;
            float all = 0.0f;
#pragma unroll
            for (int k = 0; k < NW; ++k)
                all += ml[(k * 4 + 2 * m + 1) * 32 + (l & 31)] * __builtin_amdgcn_exp2f(ml[(k * 4 + 2 * m) * 32 + (l & 31)] - base);
            const float f = __builtin_amdgcn_exp2f(top[m] - base);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[m][t][e] *= f;
            top[m] = most;
            sum[m] = all;
        }
#pragma unroll
        for (int half = NW / 2; half > 0; half /= 2) {
            if (w >= half && w < 2 * half) {
                float* to = acc + (w - half) * 2 * DVT * 32;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) to[((m * NT + t) * 16 + e) * 64 + l] = o[m][t][e];
            }
            __syncthreads();
            if (w < half) {
                const float* from = acc + w * 2 * DVT * 32;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[m][t][e] += from[((m * NT + t) * 16 + e) * 64 + l];
            }
            __syncthreads();
        }
        if (w != 0) return;
    }
    if (mine >= a.rows) return;

    if (a.splits > 1) {
        const int64_t at = ((int64_t)split * bh_all + bh) * a.rows + mine;
        if (blockIdx.z == 0 && h == 0) *(f32x4*)(a.part_ml + 4 * at) = f32x4{top[0], sum[0], top[1], sum[1]};
        const int wide = (a.Dv + 3) / 4 * 4;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            if (sum[m] == 0.0f) continue;              // the joining kernel does not read it either
            float* to = a.part + (at * 2 + m) * wide + dv0;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const int d = 32 * t + 8 * (e >> 2) + 4 * h;
                    if (dv0 + d < wide && d < DVT)
                        *(f32x4*)(to + d) = f32x4{o[m][t][e], o[m][t][e + 1], o[m][t][e + 2], o[m][t][e + 3]};
                }
        }
        return;
    }
    const int head = hk * a.G + g;
    const float inv0 = sum[0] == 0.0f ? 0.0f : 1.0f / sum[0], inv1 = sum[1] == 0.0f ? 0.0f : 1.0f / sum[1];
    const float lam = a.lam[head];
    const int64_t at = (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv + dv0;
    T* out = (T*)a.out + at;
    T* second = a.second ? (T*)a.second + at : nullptr;
    const bool v4 = a.ovec && a.Dv % 4 == 0;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            float x[4], y[4];
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                y[z] = o[1][t][e + z] * inv1;
                // (a query that sees nothing answers 0, whatever lam is)
                x[z] = sum[1] == 0.0f ? 0.0f : fmaf(-lam, y[z], o[0][t][e + z] * inv0);
            }
            const int d = 32 * t + 8 * (e >> 2) + 4 * h;
            store4(out, d, dvn, v4, x);
            if (second) store4(second, d, dvn, v4, y);
        }
    if (a.lse && blockIdx.z == 0 && h == 0) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
            a.lse[(((int64_t)m * a.B + b) * a.H + head) * a.Sq + i] =
                sum[m] == 0.0f ? -INFINITY : (top[m] + log2f(sum[m])) * 0.69314718055994530942f;
    }
}

// Joins the splits' parts: a workgroup a row, lanes along the values.
template <typename T>
__global__ __launch_bounds__(256) void attn_join(AttnArgs a)
{
    const int bh_all = a.B * a.Hkv;
    const int64_t row = blockIdx.x;                    // bh * rows + r
    const int bh = (int)(row / a.rows), r = (int)(row - (int64_t)bh * a.rows), b = bh / a.Hkv, hk = bh % a.Hkv;
    const int i = r / a.G, head = hk * a.G + r % a.G, wide = (a.Dv + 3) / 4 * 4, d = threadIdx.x;
    float val[2], lse[2];
    bool none = true;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        float most = -INFINITY;
        for (int s = 0; s < a.splits; ++s) most = fmaxf(most, a.part_ml[4 * ((int64_t)s * bh_all * a.rows + row) + 2 * m]);
        const float base = most == -INFINITY ? 0.0f : most;
        float all = 0.0f, sum = 0.0f;
        for (int s = 0; s < a.splits; ++s) {
            const int64_t at = (int64_t)s * bh_all * a.rows + row;
            const float l = a.part_ml[4 * at + 2 * m + 1];
            if (l == 0.0f) continue;
            const float f = __builtin_amdgcn_exp2f(a.part_ml[4 * at + 2 * m] - base);
            all += l * f;
            if (d < a.Dv) sum = fmaf(a.part[(at * 2 + m) * wide + d], f, sum);
        }
        val[m] = all == 0.0f ? 0.0f : sum / all;
        lse[m] = all == 0.0f ? -INFINITY : (most + log2f(all)) * 0.69314718055994530942f;
        none = all == 0.0f;
    }
    if (d < a.Dv) {
        const int64_t at = (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv + d;
        ((T*)a.out)[at] = (T)(none ? 0.0f : fmaf(-a.lam[head], val[1], val[0]));
        if (a.second) ((T*)a.second)[at] = (T)val[1];
    }
    if (a.lse && d < 2) a.lse[(((int64_t)d * a.B + b) * a.H + head) * a.Sq + i] = d ? lse[1] : lse[0];
}

struct FwdPlan { bool few; int rows_tile, row_tiles, chunks, splits, split_keys; size_t part, ml; };

int dim_tile(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

FwdPlan fwd_plan(const sconv_diffattn_desc_t& d, size_t ws_bytes)
{
    FwdPlan p = {};
    const int64_t G = d.H / d.Hkv, rows = d.Sq * G, bh = (int64_t)d.B * d.Hkv;
    const int DT = dim_tile(d.D), DVT = DT == 32 ? 64 : 128;
    p.few = rows <= 32;
    p.rows_tile = p.few ? 32 : 128;
    p.row_tiles = (int)((rows + p.rows_tile - 1) / p.rows_tile);
    p.chunks = (d.Dv + DVT - 1) / DVT;
    p.splits = 1;
    p.split_keys = d.Sk > 0 ? d.Sk : 1;
    // keys are split, at 512 a part or more, where wide workgroups fill half of the chip at most, and until few ones fill it four
    // times over (requests' lengths differ, and a workgroup without keys ends at once)
    const int64_t base = p.row_tiles * bh * p.chunks;
    if (base == 0) return p;
    int64_t splits = std::min<int64_t>(p.few ? (1024 + base - 1) / base : 512 / base, (d.Sk + 511) / 512);
    const int64_t wide = (d.Dv + 3) / 4 * 4, each = bh * rows * (2 * wide + 4) * (int64_t)sizeof(float);
    splits = std::min<int64_t>(splits, (int64_t)(ws_bytes / (size_t)each));
    if (splits > 1) {
        const int64_t keys = ((d.Sk + splits - 1) / splits + 127) / 128 * 128;
        p.split_keys = (int)keys;
        p.splits = (int)((d.Sk + keys - 1) / keys);
        p.part = (size_t)(p.splits * bh * rows * 2 * wide) * sizeof(float);
        p.ml = (size_t)(p.splits * bh * rows * 4) * sizeof(float);
    }
    return p;
}

template <typename T, bool VEC, int DT, int DVT, int NW, bool FEW>
int fwd_launch(const AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    constexpr size_t tiles = FwdShape<T, DT, DVT, NW, FEW>::LDS, join = (size_t)(NW * 128 + NW / 2 * 2 * DVT * 32) * 4;
    constexpr size_t lds = FEW && join > tiles ? join : tiles;
    const auto kern = attn_fwd<T, VEC, DT, DVT, NW, FEW>;
    const int rc = allow_lds(kern, lds);
    if (rc) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.row_tiles * a.B * a.Hkv), (unsigned)p.splits, (unsigned)p.chunks),
                       dim3(64 * NW), lds, stream, a);
    return launch_status();
}

template <typename T, bool VEC>
int fwd_run(AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    const int DT = dim_tile(a.D);
    int rc;
    if (p.few) {
        // (tiles of 128 wide rows in 32 bits do not fit a workgroup's LDS: two wavefronts of 32 keys)
        if (DT == 32) rc = fwd_launch<T, VEC, 32, 64, 4, true>(a, p, stream);
        else if (DT == 64) rc = fwd_launch<T, VEC, 64, 128, sizeof(T) == 2 ? 4 : 2, true>(a, p, stream);
        else rc = fwd_launch<T, VEC, 128, 128, sizeof(T) == 2 ? 4 : 2, true>(a, p, stream);
    } else {
        if (DT == 32) rc = fwd_launch<T, VEC, 32, 64, 4, false>(a, p, stream);
        else if (DT == 64) rc = fwd_launch<T, VEC, 64, 128, 4, false>(a, p, stream);
        else rc = fwd_launch<T, VEC, 128, 128, 4, false>(a, p, stream);
    }
    if (rc || p.splits == 1) return rc;
    hipLaunchKernelGGL((attn_join<T>), dim3((unsigned)((int64_t)a.B * a.Hkv * a.rows)), dim3(256), 0, stream, a);
    return launch_status();
}

}  // namespace

AttnArgs attn_args(const sconv_diffattn_desc_t& d, const void* q, const void* k, const void* v, const float* lam,
                   const int32_t* lengths, const uint8_t* mask)
{
    AttnArgs a = {};
    a.q = q; a.k = k; a.v = v; a.lam = lam; a.len = lengths; a.mask = mask;
    a.B = d.B; a.Sq = d.Sq; a.Sk = d.Sk; a.H = d.H; a.Hkv = d.Hkv; a.G = d.H / d.Hkv; a.D = d.D; a.Dv = d.Dv;
    a.causal = d.causal; a.rows = d.Sq * a.G;
    a.scale = d.scale; a.scale2 = d.scale * 1.44269504088896340736f;
    a.q_b = d.q_b; a.q_s = d.q_s; a.q_h = d.q_h; a.k_b = d.k_b; a.k_s = d.k_s; a.k_h = d.k_h;
    a.v_b = d.v_b; a.v_s = d.v_s; a.v_h = d.v_h; a.mask_b = d.mask_b;
    a.splits = 1;
    return a;
}

bool attn_vector(const AttnArgs& a, int type)
{
    const int64_t strides = a.q_b | a.q_s | a.q_h | a.k_b | a.k_s | a.k_h | a.v_b | a.v_s | a.v_h | a.D | a.Dv;
    return strides % (16 / type_size(type)) == 0 && aligned_to(a.q, 16) && aligned_to(a.k, 16) && aligned_to(a.v, 16);
}

size_t diffattn_forward_workspace(const sconv_diffattn_desc_t& d)
{
    const FwdPlan p = fwd_plan(d, ~(size_t)0 >> 1);
    return p.part + p.ml;
}

int launch_diffattn_forward(const sconv_diffattn_desc_t& d, const void* q, const void* k, const void* v, const float* lam,
                            const int32_t* lengths, const uint8_t* mask, void* out, void* second, float* lse, void* ws,
                            size_t ws_bytes, hipStream_t stream)
{
    AttnArgs a = attn_args(d, q, k, v, lam, lengths, mask);
    if (d.B == 0 || d.Sq == 0) return SCONV_OK;
    const FwdPlan p = fwd_plan(d, ws_bytes);
    a.out = out; a.second = second; a.lse = lse;
    a.ovec = aligned_to(out, 16) && aligned_to(second, 16);
    a.splits = p.splits; a.split_keys = p.split_keys; a.row_tiles = p.row_tiles;
    a.part = (float*)ws;
    a.part_ml = (float*)((char*)ws + p.part);
    const bool vec = attn_vector(a, d.type);
    if (d.type == SCONV_BF16) return vec ? fwd_run<bf16, true>(a, p, stream) : fwd_run<bf16, false>(a, p, stream);
    return vec ? fwd_run<float, true>(a, p, stream) : fwd_run<float, false>(a, p, stream);
}

}  // namespace sconv
