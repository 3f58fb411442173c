// Differential attention, forward (formulas in sconv_tokens.h, product layout in sconv_diffattn_common.h).
//
// One pass over the keys with a running maximum and sum for each of the two maps.  The rows of a tile are (query, head of the
// group) pairs, so heads that share keys share their tiles, and a single token's heads fill one tile.  A key tile's values are
// read once for both maps.
//   wide   128 rows a workgroup, 32 a wavefront; every wavefront walks all keys of the tile.
//   few    up to 32 rows a workgroup: its wavefronts walk keys of their own, and join at the end.
// Either may split the keys over workgroups, whose parts a second kernel joins in a fixed order.
// In 16 bits wide calls round their weights to the operands' type for the product with the values, which is two thirds of their matrix
// work: a second product with what the rounding leaves out would bring the result from 2.4e-3 of its norm off to its own rounding's
// 1.7e-3, and 12544 queries from 502 to 774 us, 2 x 3136 from 148 to 223, a training pass of 784 places from 155 to 177.  Few rows' wait
// for memory and take that second product (16 requests of up to 32768 keys 132.7 us
// without, 134.2 with, one of 32 rows 23.7 and 25.8).  The sums that weights are divided by are of the unrounded ones, in 32 bits.
// Measured, heads of 64 with values of 128: 12544 queries seeing what came before, 8 heads on 4, 16 bits 491 us = 984 TFLOP/s of seen pairs
// (a large 16-bit product reaches 1137, the pipe's power limit); 2 x 3136 x 8 unmasked 158 us; 32 bits, 8 x 196 x 7 heads 44 us
// (112 workgroups); one token of 16 requests over up to 32768 keys 130 us = 4.4 TB/s, and 5 for the join.
// Heads of 65 to 128 do not fit the registers everywhere: attn_wide spills 500 bytes a lane in 32 bits, attn_few up to 550.
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


template <typename T, int DT, int DVT>
struct WideShape {
    static constexpr int NW = 4, BN = 32, ROWS = 32 * NW;
    static constexpr int WAVES = sizeof(T) == 2 && DT <= 64 ? 2 : 1;
    typedef Tile<T, BN, 2 * DT> Keys;
    typedef Tile<T, BN, DVT> Values;
    static constexpr int TILE = Keys::SIZE + Values::SIZE;
    static constexpr size_t LDS = (size_t)2 * TILE * 2 + 3 * 4;    // (one tile is written while the other is read)
};

// A row's part of a call whose keys are split: unweighted sums and statistics, for the joining kernel.
struct RowPart {
    float* o; float* ml; int wide;
    __device__ __forceinline__ RowPart(const AttnArgs& a, int split, int bh, int row)
    {
        const int64_t at = ((int64_t)split * a.B * a.Hkv + bh) * a.rows + row;
        wide = (a.Dv + 3) / 4 * 4;
        o = a.part + at * 2 * wide;
        ml = a.part_ml + 4 * at;
    }
    __device__ __forceinline__ void stats(const float (&top)[2], const float (&sum)[2]) const { *(f32x4*)ml = f32x4{top[0], sum[0], top[1], sum[1]}; }
    // (the joining kernel does not read sums of nothing)
    __device__ __forceinline__ void store(int m, float sum, int dv0, int d, int most, float x, float y, float z, float w) const
    {
        if (sum != 0.0f && d < most && dv0 + d < wide) *(f32x4*)(o + m * wide + dv0 + d) = f32x4{x, y, z, w};
    }
};

// A row's results: values dv0 .. dv0 + dvn of a head.
template <typename T>
struct RowOut {
    T* out; T* second; int dvn, b, i, head; bool v4, none; float inv0, inv1, lam;
    __device__ __forceinline__ RowOut(const AttnArgs& a, int b_, int i_, int head_, int dv0, int dvn_, const float (&sum)[2])
    {
        b = b_; i = i_; head = head_; dvn = dvn_;
        const int64_t at = (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv + dv0;
        out = (T*)a.out + at;
        second = a.second ? (T*)a.second + at : nullptr;
        v4 = a.ovec && a.Dv % 4 == 0;
        none = sum[1] == 0.0f;
        inv0 = none ? 0.0f : 1.0f / sum[0];
        inv1 = none ? 0.0f : 1.0f / sum[1];
        lam = a.lam[head];
    }
    __device__ __forceinline__ void store(int d, const float (&o0)[4], const float (&o1)[4]) const
    {
        float x[4], y[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            y[z] = o1[z] * inv1;
            // (a query that sees nothing answers 0, whatever lam is)
            x[z] = none ? 0.0f : fmaf(-lam, y[z], o0[z] * inv0);
        }
        store4(out, d, dvn, v4, x);
        if (second) store4(second, d, dvn, v4, y);
    }
    __device__ __forceinline__ void stats(const AttnArgs& a, const float (&top)[2], const float (&sum)[2]) const
    {
        if (!a.lse) return;
#pragma unroll
        for (int m = 0; m < 2; ++m)
            a.lse[(((int64_t)m * a.B + b) * a.H + head) * a.Sq + i] =
                sum[m] == 0.0f ? -INFINITY : (top[m] + log2f(sum[m])) * 0.69314718055994530942f;
    }
};

// The end of a wide kernel: a lane's row, to the results or to its part of them.
template <typename T, int NT, int DVT>
__device__ __forceinline__ void wide_end(const AttnArgs& a, int b, int bh, int split, int dv0, int mine, int i, int head, int h,
                                         const f32x16 (&o)[2][NT], const float (&top)[2], float (&sum)[2])
{
#pragma unroll
    for (int m = 0; m < 2; ++m) sum[m] = half_sum(sum[m]);
    if (mine >= a.rows) return;
    if (a.splits > 1) {
        const RowPart part(a, split, bh, mine);
        if (dv0 == 0 && h == 0) part.stats(top, sum);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    part.store(m, sum[m], dv0, 32 * t + 8 * (e >> 2) + 4 * h, DVT, o[m][t][e], o[m][t][e + 1], o[m][t][e + 2], o[m][t][e + 3]);
        return;
    }
    const RowOut<T> row(a, b, i, head, dv0, min(DVT, a.Dv - dv0), sum);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const float x[4] = {o[0][t][e], o[0][t][e + 1], o[0][t][e + 2], o[0][t][e + 3]};
            const float y[4] = {o[1][t][e], o[1][t][e + 1], o[1][t][e + 2], o[1][t][e + 3]};
            row.store(32 * t + 8 * (e >> 2) + 4 * h, x, y);
        }
    if (dv0 == 0 && h == 0) row.stats(a, top, sum);
}

template <typename T, bool VEC, int DT, int DVT>
__global__ __launch_bounds__(256, (WideShape<T, DT, DVT>::WAVES)) void attn_wide(AttnArgs a)
{
    typedef WideShape<T, DT, DVT> Shape;
    constexpr int NW = Shape::NW, BN = Shape::BN, ROWS = Shape::ROWS;
    typedef typename Shape::Keys Keys;
    typedef typename Shape::Values Values;
    constexpr int KS = DT / 16, NT = DVT / 32, TH = 64 * NW;
    typedef typename Frag<T>::type frag;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    bf16* tiles = (bf16*)lds;
    uint32_t* words = (uint32_t*)(tiles + 2 * Shape::TILE);    // [3]: of the tile that is read, the next one and the one after

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int tile = a.row_tiles - 1 - blockIdx.x / bh_all;      // the rows that see most first
    const int split = blockIdx.y, dv0 = blockIdx.z * DVT, dvn = min(DVT, a.Dv - dv0);
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int mine = tile * ROWS + 32 * w + (l & 31), r = min(mine, a.rows - 1), i = r / a.G, g = r - i * a.G;
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
            if (threadIdx.x == 0) words[slot] = (uint32_t)there;
        }
    };
    const auto put = [&](int j0, int turn, int slot) {
        bf16* kt = tiles + turn * Shape::TILE;
        const uint32_t* wd = mask || j0 + BN > n ? words + slot : nullptr;
        ks.store(kt, wd, a.D);
        vs.store(kt + Keys::SIZE, wd, dvn);
    };
    const int vcol = col_lane<Values::LD>();
    const auto after = [](int slot) { return slot == 2 ? 0 : slot + 1; };
    int turn = 0, slot = 0;
    if (k0 < k1) {
        fetch(k0);
        mark(k0, 0);
        if (mask || k0 + BN > n) __syncthreads();
        put(k0, 0, 0);
        if (k0 + BN < k1) { fetch(k0 + BN); mark(k0 + BN, 1); }
    }
    for (int j0 = k0; j0 < k1; j0 += BN, turn ^= 1, slot = after(slot)) {
        __syncthreads();
        // (this tile is there; the next one's keys were marked before the barrier)
        if (j0 + BN < k1) {
            put(j0 + BN, turn ^ 1, after(slot));
            if (j0 + 2 * BN < k1) fetch(j0 + 2 * BN);
        }
        if (j0 < wmax) {
            const bf16* kt = tiles + turn * Shape::TILE;
            const bf16* vt = kt + Keys::SIZE;
            const bf16* krow = kt + (l & 31) * Keys::LD + 8 * h;
            f32x16 s[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[m][e] = 0.0f;
#pragma unroll
                for (int t = 0; t < KS; ++t) s[m] = mma(s[m], tile_row<T, Keys::PLANE>(krow + m * DT + 16 * t), qf[m][t]);
            }
            const uint32_t word = mask || j0 + BN > n ? words[slot] : ~0u;
            if (j0 + 32 > wmin || (mask && word != ~0u)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = 8 * (e >> 2) + 4 * h + (e & 3);
                    const bool ok = j0 + j < lim && (word >> j & 1);
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
                    const frag vf = tile_col<T, Values::LD, Values::PLANE>(vt + vcol + 16 * st * Values::LD + 32 * t);
                    o[0][t] = mma(o[0][t], vf, p0);
                    o[1][t] = mma(o[1][t], vf, p1);
                }
            }
            settle();
        }
        if (j0 + 2 * BN < k1) mark(j0 + 2 * BN, after(after(slot)));
    }
    wide_end<T, NT, DVT>(a, b, bh, split, dv0, mine, i, hk * a.G + g, h, o, top, sum);
}

// Wide rows in 16 bits, whole vectors everywhere: as attn_wide, with tiles of BN keys that go to LDS directly.
template <int DT, int DVT>
struct DirectShape {
    static constexpr int NW = 4, BN = 64, ROWS = 32 * NW;
    static constexpr int TILE = BN * (2 * DT + DVT);
    static constexpr size_t LDS = (size_t)2 * TILE * 2 + 3 * (BN / 32) * 4;
};

template <int DT, int DVT>
__global__ __launch_bounds__(256, (DT <= 64 ? 2 : 1)) void attn_direct(AttnArgs a)
{
    typedef DirectShape<DT, DVT> Shape;
    constexpr int NW = Shape::NW, BN = Shape::BN, ROWS = Shape::ROWS, KS = DT / 16, NT = DVT / 32, NB = BN / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    bf16* tiles = (bf16*)lds;
    uint32_t* words = (uint32_t*)(tiles + 2 * Shape::TILE);    // [3][NB]

    const int bh_all = a.B * a.Hkv, bh = blockIdx.x % bh_all, b = bh / a.Hkv, hk = bh % a.Hkv;
    const int tile = a.row_tiles - 1 - blockIdx.x / bh_all;      // the rows that see most first
    const int split = blockIdx.y, dv0 = blockIdx.z * DVT;
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, h = l >> 5;
    const int mine = tile * ROWS + 32 * w + (l & 31), r = min(mine, a.rows - 1), i = r / a.G, g = r - i * a.G;
    const int n = keys_of(a, b);
    const int lim = limit_of(a, i, n);
    const int wmin = __builtin_amdgcn_readfirstlane(lim), wmax = __builtin_amdgcn_readlane(lim, 31);
    const int last = limit_of(a, min(tile * ROWS + ROWS - 1, a.rows - 1) / a.G, n);
    const int k0 = split * a.split_keys, k1 = (int)min((int64_t)last, (int64_t)k0 + a.split_keys);
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_b : nullptr;

    bf16x8 qf[2][KS];
    const bf16* q = (const bf16*)a.q + b * a.q_b + i * a.q_s + (int64_t)(hk * a.G + g) * 2 * a.q_h;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[m][s] = row_frag(q + m * a.q_h + 16 * s + 8 * h);

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

    const bf16* kb = (const bf16*)a.k + b * a.k_b + (int64_t)hk * 2 * a.k_h;
    const bf16* vb = (const bf16*)a.v + b * a.v_b + (int64_t)hk * a.v_h + dv0;
    typedef Direct<BN, 2, DT, NW> Keys;
    typedef Direct<BN, 1, DVT, NW> Values;
    Keys kd;
    Values vd;
    kd.init(a.k_s, a.k_h);
    vd.init(a.v_s, 0);
    int krow[4], vcol[2];
    Keys::row_lane(krow);
    Values::col_lane(vcol);
    uint8_t seen = 1;
    const auto fetch = [&](int j0, int turn) {
        bf16* kt = tiles + turn * Shape::TILE;
        kd.load(kb, a.k_s, a.k_h, j0, n, kt);
        vd.load(vb, a.v_s, 0, j0, n, kt + BN * 2 * DT);
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
        __syncthreads();                               // this tile is there, the other one has been read
        if (j0 + BN < k1) fetch(j0 + BN, turn ^ 1);
        if (j0 + 2 * BN < k1) fetch_mask(j0 + 2 * BN);
        bf16* kt = tiles + turn * Shape::TILE;
        bf16* vt = kt + BN * 2 * DT;
        int stop = wmax;
        if (mask) {
            const uint32_t* wd = words + slot * NB;
            bool all = true, none = true;
#pragma unroll
            for (int x = 0; x < NB; ++x) { all = all && wd[x] == ~0u; none = none && wd[x] == 0; }
            if (none) stop = 0;                        // nothing to do here
            else if (!all) {                           // values that the mask leaves out may be anything
                Values::clear(vt, wd);
                __syncthreads();
            }
        }
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            const int js = j0 + 32 * x;
            if (js >= stop) continue;
            f32x16 s[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[m][e] = 0.0f;
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    const int c = m * DT + 16 * t;
                    s[m] = mma(s[m], row_frag(kt + krow[c / 16 % 4] + 32 * x * 2 * DT + c / 64 * 64), qf[m][t]);
                }
            }
            if (js + 32 > wmin || mask) {
                const uint32_t bits = seen_bits(js, lim, mask ? words[slot * NB + x] : ~0u) >> (4 * h);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[m][e] = masked(s[m][e], bits, 8 * (e >> 2) + (e & 3), 0xff800000u);
            }
            float mx[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                mx[m] = s[m][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mx[m] = fmaxf(mx[m], s[m][e]);
                mx[m] = half_max(mx[m]) * a.scale2;
            }
            if (__any(mx[0] > top[0] + 8.0f || mx[1] > top[1] + 8.0f)) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const float grown = fmaxf(top[m], mx[m]);
                    safe[m] = grown == -INFINITY ? 0.0f : grown;
                    const float f = __builtin_amdgcn_exp2f(top[m] - safe[m]);
                    top[m] = grown;
                    sum[m] *= f;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[m][t][e] *= f;
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                bf16x8 p[2];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float v = __builtin_amdgcn_exp2f(fmaf(s[m][8 * st + e], a.scale2, -safe[m]));
                        sum[m] += v;
                        p[m][e] = (bf16)v;
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const bf16x8 vf = col_frag<DVT>(vt + vcol[t % 2] + t / 2 * 64 + (32 * x + 16 * st) * DVT);
                    o[0][t] = mma(o[0][t], vf, p[0]);
                    o[1][t] = mma(o[1][t], vf, p[1]);
                }
            }
            settle();
        }
        if (j0 + 2 * BN < k1) mark(j0 + 2 * BN, after(after(slot)));
    }
    wide_end<bf16, NT, DVT>(a, b, bh, split, dv0, mine, i, hk * a.G + g, h, o, top, sum);
}

// Few rows: RT tiles of 16 to a wavefront, in products of 16 x 16.  A wavefront walks 32 keys at a time of its own, alone: its keys
// go from memory to registers as the product reads them, its values through LDS of its own (to be read down the keys), and no
// barrier stands between its loads.  The wavefronts join at the end.
template <typename T, int DVT>
struct FewShape {
    static constexpr int NW = 4, BN = 32;
    typedef Tile<T, BN, DVT> Values;                   // of a wavefront
};

template <typename T, bool VEC, int DT, int DVT, int RT>
__global__ __launch_bounds__(256, (sizeof(T) == 2 && DT <= 64 && RT == 1 ? 2 : 1)) void attn_few(AttnArgs a)
{
    typedef FewShape<T, DVT> Shape;
    typedef typename Shape::Values Values;
    constexpr int NW = Shape::NW, BN = Shape::BN, KS = DT / 32, NT = DVT / 16, E = 16 / sizeof(T);
    constexpr int NV = BN * DVT / E / 64, VPER = DVT / E;   // 16-byte vectors of a lane's and a row's share of the values
    typedef typename Frag<T>::type frag;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    // (a request's splits on different chiplets, whose blocks go round: requests' lengths differ)
    const int bh_all = a.B * a.Hkv, bh = (int)((blockIdx.x + blockIdx.y) % (uint32_t)bh_all), b = bh / a.Hkv, hk = bh % a.Hkv;
    const int first = (int)(blockIdx.x / bh_all) * 16 * RT;
    const int split = blockIdx.y, dv0 = blockIdx.z * DVT, dvn = min(DVT, a.Dv - dv0);
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, c = l & 15, h = l >> 4;
    bf16* vt = (bf16*)lds + w * Values::SIZE;
    const int n = keys_of(a, b);
    int lim[RT], wmin = n;
    frag qf[RT][2][KS];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = min(first + 16 * x + c, a.rows - 1), i = r / a.G, g = r - i * a.G;
        lim[x] = limit_of(a, i, n);
        const T* q = (const T*)a.q + b * a.q_b + i * a.q_s + (int64_t)(hk * a.G + g) * 2 * a.q_h;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[x][m][s] = global_frag<VEC>(q + m * a.q_h, 32 * s + 8 * h, a.D);
    }
    wmin = __builtin_amdgcn_readfirstlane(lim[0]);          // of the first row: limits rise
    const int last = limit_of(a, min(first + 16 * RT - 1, a.rows - 1) / a.G, n);
    const int k0 = split * a.split_keys, k1 = (int)min((int64_t)last, (int64_t)k0 + a.split_keys);
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_b : nullptr;

    f32x4 o[RT][2][NT];
    float top[RT][2], safe[RT][2], sum[RT][2];
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            top[x][m] = -INFINITY; safe[x][m] = 0.0f; sum[x][m] = 0.0f;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[x][m][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

    const T* kb = (const T*)a.k + b * a.k_b + (int64_t)hk * 2 * a.k_h;
    const T* vb = (const T*)a.v + b * a.v_b + (int64_t)hk * a.v_h + dv0;
    Raw<T> kr[2][2][KS];                               // [16 keys][map][depth]
    u32x4 vr[NV];
    uint8_t seen = 1;
    const auto fetch_keys = [&](int j0) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const T* row = kb + (int64_t)min(j0 + 16 * y + c, n - 1) * a.k_s;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int s = 0; s < KS; ++s) load_raw<VEC>(kr[y][m][s], row + m * a.k_h, 32 * s + 8 * h, a.D);
        }
    };
    const auto fetch_values = [&](int j0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int e = v * 64 + l;
            vr[v] = load16<VEC>(vb + (int64_t)min(j0 + e / VPER, n - 1) * a.v_s, e % VPER * E, dvn);
        }
        if (mask) seen = mask[min(j0 + (l & 31), n - 1)];
    };
    int j0 = k0 + BN * w;
    if (j0 < k1) { fetch_keys(j0); fetch_values(j0); }
    for (; j0 < k1; j0 += BN * NW) {
        const int next = j0 + BN * NW;
        f32x4 s[RT][2][2];                             // [rows][map][16 keys]
        const bool ragged = a.D < DT;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int x = 0; x < RT; ++x) s[x][m][y] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    const frag kf = raw_frag<VEC>(kr[y][m][t], 32 * t + 8 * h, a.D, ragged);
#pragma unroll
                    for (int x = 0; x < RT; ++x) s[x][m][y] = mma(s[x][m][y], kf, qf[x][m][t]);
                }
            }
        if (next < k1) fetch_keys(next);
        const uint32_t word = mask || j0 + BN > n ? (uint32_t)__ballot(j0 + (l & 31) < n && seen) : ~0u;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int e = v * 64 + l, row = e / VPER;
            const bool there = e % VPER * E < dvn && (word >> row & 1);
            put16<Values::PLANE>(vt + row * Values::LD + e % VPER * E, shift16<VEC, T>(vr[v], e % VPER * E, dvn), there, T());
        }
        if (next < k1) fetch_values(next);
        if (j0 + 32 > wmin || word != ~0u) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = 16 * y + 4 * h + e;
#pragma unroll
                    for (int x = 0; x < RT; ++x) {
                        const bool ok = j0 + j < lim[x] && (word >> j & 1);
                        s[x][0][y][e] = ok ? s[x][0][y][e] : -INFINITY;
                        s[x][1][y][e] = ok ? s[x][1][y][e] : -INFINITY;
                    }
                }
        }
        float p[RT][2][8];
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                f32x4 (&z)[2] = s[x][m];
                float mx = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
                mx = half_max(quarter_max(mx)) * a.scale2;
                if (__any(mx > top[x][m] + 8.0f)) {
                    const float grown = fmaxf(top[x][m], mx);
                    safe[x][m] = grown == -INFINITY ? 0.0f : grown;
                    const float f = __builtin_amdgcn_exp2f(top[x][m] - safe[x][m]);
                    top[x][m] = grown;
                    sum[x][m] *= f;
#pragma unroll
                    for (int t = 0; t < NT; ++t) o[x][m][t] *= f;
                }
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = __builtin_amdgcn_exp2f(fmaf(z[y][e], a.scale2, -safe[x][m]));
                        sum[x][m] += v;
                        p[x][m][4 * y + e] = v;
                    }
            }
        const int vcol = few_col_lane<Values::LD>();
        frag pf[RT][2], rest[RT][2];                   // (rest: 16 bits)
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                if constexpr (sizeof(T) == 2) weight_frags(p[x][m], pf[x][m], rest[x][m]);
                else to_frag(p[x][m], pf[x][m]);
            }
        wave_lds_fence();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const frag vf = tile_col<T, Values::LD, Values::PLANE, 16>(vt + vcol + 16 * t);
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                if constexpr (sizeof(T) == 2) {
                    o[x][0][t] = mma(o[x][0][t], vf, rest[x][0]);
                    o[x][1][t] = mma(o[x][1][t], vf, rest[x][1]);
                }
                o[x][0][t] = mma(o[x][0][t], vf, pf[x][0]);
                o[x][1][t] = mma(o[x][1][t], vf, pf[x][1]);
            }
        }
        wave_lds_fence();
        settle();
    }
    // the wavefronts' parts meet in LDS, over the tiles: statistics first, then the sums, halving the wavefronts
    __syncthreads();
    float* ml = (float*)lds;                           // [NW][RT][2][2][16]
    float* acc = ml + NW * RT * 64;                    // [NW / 2][RT * 2 * NT * 4][64]
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            sum[x][m] = half_sum(quarter_sum(sum[x][m]));
            if (h == 0) {
                float* at = ml + ((w * RT + x) * 2 + m) * 32 + c;
                at[0] = top[x][m];
                at[16] = sum[x][m];
            }
        }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float most = -INFINITY, all = 0.0f;
#pragma unroll
            for (int k = 0; k < NW; ++k) most = fmaxf(most, ml[((k * RT + x) * 2 + m) * 32 + c]);
            const float base = most == -INFINITY ? 0.0f : most;
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float* at = ml + ((k * RT + x) * 2 + m) * 32 + c;
                all = fmaf(at[16], __builtin_amdgcn_exp2f(at[0] - base), all);
            }
            const float f = __builtin_amdgcn_exp2f(top[x][m] - base);
#pragma unroll
            for (int t = 0; t < NT; ++t) o[x][m][t] *= f;
            top[x][m] = most;
            sum[x][m] = all;
        }
#pragma unroll
    for (int half = NW / 2; half > 0; half /= 2) {
        if (w >= half && w < 2 * half) {
            f32x4* to = (f32x4*)acc + (w - half) * RT * 2 * NT * 64 + l;
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int t = 0; t < NT; ++t) to[((x * 2 + m) * NT + t) * 64] = o[x][m][t];
        }
        __syncthreads();
        if (w < half) {
            const f32x4* from = (const f32x4*)acc + w * RT * 2 * NT * 64 + l;
#pragma unroll
            for (int x = 0; x < RT; ++x)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int t = 0; t < NT; ++t) o[x][m][t] += from[((x * 2 + m) * NT + t) * 64];
        }
        __syncthreads();
    }
    if (w != 0) return;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int mine = first + 16 * x + c, i = mine / a.G;
        if (mine >= a.rows) continue;
        if (a.splits > 1) {
            const RowPart part(a, split, bh, mine);
            if (blockIdx.z == 0 && h == 0) part.stats(top[x], sum[x]);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    part.store(m, sum[x][m], dv0, 16 * t + 4 * h, DVT, o[x][m][t][0], o[x][m][t][1], o[x][m][t][2], o[x][m][t][3]);
            continue;
        }
        const RowOut<T> row(a, b, i, hk * a.G + mine - i * a.G, dv0, dvn, sum[x]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float u[4] = {o[x][0][t][0], o[x][0][t][1], o[x][0][t][2], o[x][0][t][3]};
            const float v[4] = {o[x][1][t][0], o[x][1][t][1], o[x][1][t][2], o[x][1][t][3]};
            row.store(16 * t + 4 * h, u, v);
        }
        if (blockIdx.z == 0 && h == 0) row.stats(a, top[x], sum[x]);
    }
}

// Joins the splits' parts: a workgroup a row, lanes along the two maps' values, four groups of them along the splits.
constexpr int MAX_SPLITS = 128;
template <typename T>
__global__ __launch_bounds__(1024) void attn_join(AttnArgs a)
{
    __shared__ float f[2][MAX_SPLITS], val[4][512], total[2];
    const int bh_all = a.B * a.Hkv;
    const int64_t row = blockIdx.x, all_rows = (int64_t)bh_all * a.rows;   // row: bh * rows + r
    const int bh = (int)(row / a.rows), r = (int)(row - (int64_t)bh * a.rows), b = bh / a.Hkv, hk = bh % a.Hkv;
    const int i = r / a.G, head = hk * a.G + r % a.G, wide = (a.Dv + 3) / 4 * 4;
    // a wavefront a map: the parts' weights against the largest maximum, over the joined sum
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    if (w < 2) {
        float t[2], s[2], most = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int split = l + 64 * k;
            t[k] = -INFINITY; s[k] = 0.0f;
            if (split < a.splits) {
                const float* ml = a.part_ml + 4 * (split * all_rows + row) + 2 * w;
                t[k] = ml[0]; s[k] = ml[1];
            }
            most = fmaxf(most, t[k]);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        const float base = most == -INFINITY ? 0.0f : most;
#pragma unroll
        for (int k = 0; k < 2; ++k) t[k] = s[k] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(t[k] - base);
        const float sum = lanes_sum<64>(fmaf(s[0], t[0], s[1] * t[1])), inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        f[w][l] = t[0] * inv;
        f[w][l + 64] = t[1] * inv;
        if (l == 0) {
            total[w] = sum;
            if (a.lse) a.lse[(((int64_t)w * a.B + b) * a.H + head) * a.Sq + i] = sum == 0.0f ? -INFINITY : (most + log2f(sum)) * 0.69314718055994530942f;
        }
    }
    __syncthreads();
    const bool none = total[1] == 0.0f;
    const int group = threadIdx.x >> 8, lane = threadIdx.x & 255;
    for (int e = lane; e < 2 * a.Dv; e += 256) {
        const int m = e >= a.Dv, d = e - m * a.Dv;
        const float* from = a.part + (row * 2 + m) * wide + d;
        float v = 0.0f;
#pragma unroll 8
        for (int s = group; s < a.splits; s += 4) {
            // (parts of nothing were not written)
            const float x = from[s * all_rows * 2 * wide], g = f[m][s];
            v += g == 0.0f ? 0.0f : g * x;
        }
        val[group][e] = v;
    }
    __syncthreads();
    const int d = threadIdx.x;
    if (d < a.Dv) {
        const int e = d + a.Dv;
        const float x = (val[0][d] + val[1][d]) + (val[2][d] + val[3][d]), y = (val[0][e] + val[1][e]) + (val[2][e] + val[3][e]);
        const int64_t at = (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv + d;
        ((T*)a.out)[at] = (T)(none ? 0.0f : fmaf(-a.lam[head], y, x));
        if (a.second) ((T*)a.second)[at] = (T)y;
    }
}

// The same for the wide kernels' rows: a thread takes four values of a row and walks its parts, twice - a few as a rule; few rows over long
// caches have up to 32 in 16 bits (32768 keys) and 128 in 32 bits, which take the longer for it (40 rows over 32768 keys 52 us, 32 rows, which
// attn_few takes, 26).
template <typename T>
__global__ __launch_bounds__(256) void attn_join_wide(AttnArgs a)
{
    const int quads = (a.Dv + 3) / 4, wide = 4 * quads;
    const int64_t all_rows = (int64_t)a.B * a.Hkv * a.rows, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= all_rows * quads) return;
    const int64_t row = at / quads;
    const int d = (int)(at - row * quads) * 4;
    const int bh = (int)(row / a.rows), r = (int)(row - (int64_t)bh * a.rows), b = bh / a.Hkv, hk = bh % a.Hkv;
    const int i = r / a.G, head = hk * a.G + r % a.G;
    float most[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f}, o[2][4] = {};
    for (int s = 0; s < a.splits; ++s) {
        const f32x4 ml = *(const f32x4*)(a.part_ml + 4 * (s * all_rows + row));
        most[0] = fmaxf(most[0], ml[0]);
        most[1] = fmaxf(most[1], ml[2]);
    }
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const f32x4 ml = *(const f32x4*)(a.part_ml + 4 * (s * all_rows + row));
        const float* from = a.part + (s * all_rows + row) * 2 * wide + d;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const f32x4 x = *(const f32x4*)(from + m * wide);
            // (parts of nothing were not written)
            const bool some = ml[2 * m + 1] != 0.0f;
            const float f = some ? __builtin_amdgcn_exp2f(ml[2 * m] - most[m]) : 0.0f;
            sum[m] = fmaf(some ? ml[2 * m + 1] : 0.0f, f, sum[m]);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[m][e] = fmaf(some ? x[e] : 0.0f, f, o[m][e]);
        }
    }
    const RowOut<T> out(a, b, i, head, 0, a.Dv, sum);
    out.store(d, o[0], o[1]);
    if (d == 0) out.stats(a, most, sum);
}

struct FwdPlan { bool few; int rt, row_tiles, chunks, splits, split_keys; size_t part, ml; };

int dim_tile(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

FwdPlan fwd_plan(const sconv_diffattn_desc_t& d, bool lengths, size_t ws_bytes)
{
    FwdPlan p = {};
    const int64_t G = d.H / d.Hkv, rows = d.Sq * G, bh = (int64_t)d.B * d.Hkv;
    const int DVT = dim_tile(d.D) == 32 ? 64 : 128;
    // (32 rows at once: in 32 bits their pieces would not fit the registers)
    p.few = rows <= 32;
    p.rt = rows > 16 && d.type == SCONV_BF16 ? 2 : 1;
    const int tile = p.few ? 16 * p.rt : 128;
    p.row_tiles = (int)((rows + tile - 1) / tile);
    p.chunks = (d.Dv + DVT - 1) / DVT;
    p.splits = 1;
    p.split_keys = d.Sk > 0 ? d.Sk : 1;
    // Keys are split.  Few rows': until their workgroups fill the chip twice over at two a compute unit, at 512 keys a part or more;
    // four times over and 1024 where requests' lengths differ (16 requests of up to 32768 keys: 16 parts).  Wide ones':
    // where they fill half of the chip at most, at so many a part that the join, which reads 8 Dv bytes of every row and part,
    // stays behind what it saves: 1024 in 16 bits (50 workgroups over 3136 keys: 48 us, unsplit 103; 112 over 784: 31 us
    // unsplit, 38 in two), 256 in 32 (28 over 784: 90 us, unsplit 210).
    const int64_t base = p.row_tiles * bh * p.chunks;
    if (base == 0 || rows == 0) return p;
    const int64_t least = p.few ? (lengths ? 1024 : 512) : d.type == SCONV_BF16 ? 1024 : 256, most = lengths ? 1024 : 512;
    int64_t splits = std::min<int64_t>(p.few ? (most + base - 1) / base : 512 / base, (d.Sk + least - 1) / least);
    const int64_t wide = (d.Dv + 3) / 4 * 4, each = bh * rows * (2 * wide + 4) * (int64_t)sizeof(float);
    splits = std::min<int64_t>(std::min<int64_t>(splits, MAX_SPLITS), (int64_t)(ws_bytes / (size_t)each));
    if (splits > 1) {
        const int64_t keys = ((d.Sk + splits - 1) / splits + 127) / 128 * 128;
        p.split_keys = (int)keys;
        p.splits = (int)((d.Sk + keys - 1) / keys);
        p.part = (size_t)(p.splits * bh * rows * 2 * wide) * sizeof(float);
        p.ml = (size_t)(p.splits * bh * rows * 4) * sizeof(float);
    }
    return p;
}

template <typename T, bool VEC, int DT, int DVT>
int wide_launch(const AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    constexpr size_t lds = WideShape<T, DT, DVT>::LDS;
    const auto kern = attn_wide<T, VEC, DT, DVT>;
    const int rc = allow_lds(kern, lds);
    if (rc) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.row_tiles * a.B * a.Hkv), (unsigned)p.splits, (unsigned)p.chunks),
                       dim3(256), lds, stream, a);
    return launch_status();
}

template <int DT, int DVT>
int direct_launch(const AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    constexpr size_t lds = DirectShape<DT, DVT>::LDS;
    const auto kern = attn_direct<DT, DVT>;
    const int rc = allow_lds(kern, lds);
    if (rc) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.row_tiles * a.B * a.Hkv), (unsigned)p.splits, (unsigned)p.chunks),
                       dim3(256), lds, stream, a);
    return launch_status();
}

template <typename T, bool VEC, int DT, int DVT, int RT>
int few_launch(const AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    constexpr size_t tiles = (size_t)4 * FewShape<T, DVT>::Values::SIZE * 2, join = (size_t)(4 * RT * 64 + 2 * RT * 2 * DVT * 16) * 4;
    constexpr size_t lds = join > tiles ? join : tiles;
    const auto kern = attn_few<T, VEC, DT, DVT, RT>;
    const int rc = allow_lds(kern, lds);
    if (rc) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)((int64_t)a.row_tiles * a.B * a.Hkv), (unsigned)p.splits, (unsigned)p.chunks),
                       dim3(256), lds, stream, a);
    return launch_status();
}

template <typename T, bool VEC, int DT, int DVT>
int fwd_launch(const AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    if constexpr (VEC && sizeof(T) == 2) {
        // (a tile has to lie within what a buffer's offsets reach; values' rows beside each other)
        const int64_t far = int64_t(1) << 22;
        if (!p.few && a.D == DT && a.Dv % DVT == 0 && a.k_s < far && a.k_h < far * 128 && a.v_s >= DVT && a.v_s < far)
            return direct_launch<DT, DVT>(a, p, stream);
    }
    if (!p.few) return wide_launch<T, VEC, DT, DVT>(a, p, stream);
    if constexpr (sizeof(T) == 2)
        if (p.rt == 2) return few_launch<T, VEC, DT, DVT, 2>(a, p, stream);
    return few_launch<T, VEC, DT, DVT, 1>(a, p, stream);
}

template <typename T, bool VEC>
int fwd_run(AttnArgs& a, const FwdPlan& p, hipStream_t stream)
{
    const int DT = dim_tile(a.D);
    const int rc = DT == 32 ? fwd_launch<T, VEC, 32, 64>(a, p, stream)
                 : DT == 64 ? fwd_launch<T, VEC, 64, 128>(a, p, stream) : fwd_launch<T, VEC, 128, 128>(a, p, stream);
    if (rc || p.splits == 1) return rc;
    if (!p.few) {
        const int64_t threads = (int64_t)a.B * a.Hkv * a.rows * ((a.Dv + 3) / 4);
        hipLaunchKernelGGL((attn_join_wide<T>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
        return launch_status();
    }
    hipLaunchKernelGGL((attn_join<T>), dim3((unsigned)((int64_t)a.B * a.Hkv * a.rows)), dim3(1024), 0, stream, a);
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
    size_t most = 0;
    for (const bool lengths : {false, true}) {
        const FwdPlan p = fwd_plan(d, lengths, ~(size_t)0 >> 1);
        most = std::max(most, p.part + p.ml);
    }
    return most;
}

int launch_diffattn_forward(const sconv_diffattn_desc_t& d, const void* q, const void* k, const void* v, const float* lam,
                            const int32_t* lengths, const uint8_t* mask, void* out, void* second, float* lse, void* ws,
                            size_t ws_bytes, hipStream_t stream)
{
    AttnArgs a = attn_args(d, q, k, v, lam, lengths, mask);
    if (d.B == 0 || d.Sq == 0) return SCONV_OK;
    const FwdPlan p = fwd_plan(d, lengths != nullptr, ws_bytes);
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
