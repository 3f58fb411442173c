// Differential attention of new tokens over a paged cache (formulas in sconv_tokens.h, the cache in sconv_serving.h).
//
// Bound by the cache's read.  The keys of all requests, laid end to end in units of 32, are shared out among workgroups by their number, so
// that workgroups are alike whatever the requests' lengths: a workgroup walks its stretch, request after request; a request that
// lies within one is answered there, others leave parts, which a second kernel joins.  Where every request begins follows from the lengths, which
// each workgroup adds up itself.
// Within a stretch a wavefront walks units of its own, alone: keys go from memory to registers as the product reads them, values
// through LDS of its own (to be read down the keys), the next unit's on their way under this one's products.  8-bit values become 16-bit ones with
// their scale as they come, which is exact.  Scores are formed transposed - keys down, queries across -, so a softmax stays within a lane's
// quarter and the weights never leave the registers.  Weights go as two 16-bit values for their product with V (three pieces in 32 bits).
#include <algorithm>

#include "sconv_diffattn_common.h"
#include "sconv_serving_common.h"

namespace sconv {

namespace {

constexpr int NW = 4, BN = 32;           // wavefronts of a workgroup, keys of a unit
constexpr int LEAST = 8;                 // units of a stretch at least: two of every wavefront
constexpr int MAX_PARTS = 1024;

struct PagedArgs {
    const void* q; const void* k; const void* v; const uint8_t* kx; const uint8_t* vx; const int32_t* table; const float* lam;
    const int32_t* len; void* out;
    float* part; float* part_ml;         // [Hkv][parts][2][rows]: [2][wide], [4]
    int B, Sq, H, Hkv, G, D, Dv, causal, rows, pages, width, capacity, parts;   // rows = Sq * G: of one request and key head, r = i * G + g
    int ovec;
    float scale2;                        // scale * log2(e)
    int64_t q_b, q_s, q_h, k_p, k_s, k_h, v_p, v_s, v_h, kx_p, kx_s, kx_h, vx_p, vx_s, vx_h, table_b;
    Divide page;
};

// What the pages hold, as products take it: e4m3 and 16 bits one plane, 32 bits three.
template <typename P> struct Kept { typedef bf16 type; };
template <> struct Kept<float> { typedef float type; };

// 16-bit values against 32-bit ones in three pieces.
using sconv::mma;
template <typename C>
__device__ __forceinline__ C mma(C c, const bf16x8& a, const bf16x8x3& b)
{
    c = mma(c, a, b.p[2]);
    c = mma(c, a, b.p[1]);
    return mma(c, a, b.p[0]);
}

__device__ __forceinline__ int positions(const PagedArgs& a, int b) { return min(max(a.len[b], 0), a.capacity); }
__device__ __forceinline__ int units_of(int n) { return (n + BN - 1) / BN; }

// All requests' units, and those of requests before b: every wavefront adds them up for itself.
__device__ __forceinline__ int wave_total(int v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int units_before(const PagedArgs& a, int upto)
{
    const int l = threadIdx.x & 63;
    int v = 0;
    for (int b = l; b < upto; b += 64) v += units_of(positions(a, b));
    return wave_total(v);
}
// Units of a stretch.
__device__ __forceinline__ int stretch_of(const PagedArgs& a, int units) { return max((units + a.parts - 1) / a.parts, LEAST); }
// The request that unit u lies in, and the units before it.
__device__ __forceinline__ void request_of(const PagedArgs& a, int u, int& b, int& before)
{
    const int l = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0;; b0 += 64) {
        const int mine = b0 + l < a.B ? units_of(positions(a, b0 + l)) : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int t = __shfl_up(upto, d);
            if (l >= d) upto += t;
        }
        const uint64_t past = __ballot(base + upto > u);
        if (past || b0 + 64 >= a.B) {
            const int at = past ? __builtin_ctzll(past) : 63;
            b = __builtin_amdgcn_readfirstlane(b0 + at);
            before = __builtin_amdgcn_readfirstlane(base + __shfl(upto - mine, at));
            return;
        }
        base += __shfl(upto, 63);
    }
}

// How many of a request's n positions query i sees.
__device__ __forceinline__ int limit_of(const PagedArgs& a, int i, int n)
{
    if (!a.causal) return n;
    const int64_t lim = (int64_t)i + n - a.Sq + 1;
    return (int)(lim < 0 ? 0 : lim > n ? n : lim);
}

// 16 bytes of a row from element d on, of `have` elements: load16 and shift16 for bytes.
template <bool FULL>
__device__ __forceinline__ u32x4 load16_any(const uint8_t* row, int d, int have)
{
    typedef u32x4 any __attribute__((aligned(1)));
    if constexpr (FULL) return *(const any*)(row + d);
    if (have >= 16) return *(const any*)(row + min(d, have - 16));
    u32x4 r = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) if (d + i < have) r[i >> 2] |= (uint32_t)row[d + i] << (8 * (i & 3));
    return r;
}
template <bool FULL, typename T>
__device__ __forceinline__ u32x4 load16_any(const T* row, int d, int have)
{
    typedef u32x4 any __attribute__((aligned(2)));
    if constexpr (FULL) return *(const any*)(row + d);
    return load16<false>(row, d, have);
}

__device__ __forceinline__ bf16x8 widened(uint32_t lo, uint32_t hi, float scale)
{
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A key's row of one map as it lies in memory: the fragments of KS steps of 32.  In 8 bits a lane reads 16 bytes at once, which are eight
// depths of each of two steps (of one where there is one).
template <typename P, int KS> struct RawKey { Raw<P> r[KS]; };
template <int KS> struct RawKey<e4m3, KS> { u32x4 r[(KS + 1) / 2]; };
template <typename P, int KS>
__device__ __forceinline__ int depth_of(int s, int h)
{
    if constexpr (sizeof(P) == 1 && KS > 1) return 64 * (s / 2) + 16 * h + 8 * (s % 2);
    return 32 * s + 8 * h;
}
template <bool FULL, typename P, int KS>
__device__ __forceinline__ void load_key(RawKey<P, KS>& k, const P* row, int h, int have)
{
    if constexpr (sizeof(P) == 1) {
        const uint8_t* p = (const uint8_t*)row;
        if constexpr (KS == 1) {
            const u32x2 x = load8_bytes(row + 8 * h, FULL ? 8 : have - 8 * h);
            k.r[0] = u32x4{x[0], x[1], 0, 0};
        } else {
#pragma unroll
            for (int i = 0; i < KS / 2; ++i) k.r[i] = load16_any<FULL>(p, 64 * i + 16 * h, have);
        }
    } else {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < (int)sizeof(P) / 2; ++i) k.r[s].u[i] = load16_any<FULL>(row, 32 * s + 8 * h + 4 * i, have);
    }
}
template <bool FULL, typename P, int KS>
__device__ __forceinline__ typename Frag<typename Kept<P>::type>::type key_frag(const RawKey<P, KS>& k, int s, int h, int have, float scale)
{
    if constexpr (sizeof(P) == 1) {
        if constexpr (KS == 1) return widened(k.r[0][0], k.r[0][1], scale);
        else {
            const u32x4 x = shift16<FULL, uint8_t>(k.r[s / 2], 64 * (s / 2) + 16 * h, have);
            return widened(x[2 * (s % 2)], x[2 * (s % 2) + 1], scale);
        }
    } else {
        return raw_frag<FULL>(k.r[s], 32 * s + 8 * h, have, !FULL);
    }
}

// A row's weights for their product with the values.
template <typename T> struct Weights;
template <> struct Weights<bf16> {
    bf16x8 hi, lo;
    __device__ __forceinline__ void set(const float (&v)[8]) { weight_frags(v, hi, lo); }
    template <typename V> __device__ __forceinline__ f32x4 times(f32x4 c, const V& v) const { return mma(mma(c, v, lo), v, hi); }
};
template <> struct Weights<float> {
    bf16x8x3 p;
    __device__ __forceinline__ void set(const float (&v)[8]) { p = in_pieces<true>(v); }
    template <typename V> __device__ __forceinline__ f32x4 times(f32x4 c, const V& v) const { return mma(c, v, p); }
};

// T: queries and results; P: the pages.  FULL: heads are DT and values whole DVT wide.  ALIGNED: a page is whole 16 slots, so that half a
// unit lies on one page.  RT: tiles of 16 rows.
template <typename T, typename P, bool FULL, bool ALIGNED, int DT, int DVT, int RT>
__global__ __launch_bounds__(256, (sizeof(T) == 2 && DT <= 64 && RT == 1 ? 2 : 1)) void paged_attn(PagedArgs a)
{
    typedef typename Kept<P>::type KT;
    typedef Tile<KT, BN, DVT> Values;
    constexpr int KS = DT / 32, NT = DVT / 16, E = 16 / sizeof(P);
    constexpr int NV = BN * DVT / E / 64, VPER = DVT / E;        // 16-byte vectors of a lane's and a row's share of the values
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, c = l & 15, h = l >> 4;
    const int per_head = a.parts ? a.parts : a.B;
    const int at = blockIdx.x % per_head, rest = blockIdx.x / per_head, hk = rest % a.Hkv, first = rest / a.Hkv * 16 * RT;
    const int dv0 = blockIdx.z * DVT, dvn = min(DVT, a.Dv - dv0), wide = (a.Dv + 3) / 4 * 4;
    bf16* vt = (bf16*)lds + w * Values::SIZE;

    int b, begin, end;                                           // the request, the stretch in units from its first
    if (a.parts) {
        const int all = units_before(a, a.B), per = stretch_of(a, all);
        const int64_t from = (int64_t)at * per;
        if (from >= all) return;
        int before;
        request_of(a, (int)from, b, before);
        begin = (int)from - before;
        end = (int)min(from + per, (int64_t)all) - before;
    } else {
        b = at;
        begin = 0;
        end = units_of(positions(a, b));
    }

    for (;; ++b) {
        const int n = positions(a, b), units = units_of(n);
        if (a.parts && units == 0) continue;
        const int u1 = min(end, units);
        int lim[RT];
        typename Frag<T>::type qf[RT][2][KS];
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            const int r = min(first + 16 * x + c, a.rows - 1), i = r / a.G, g = r - i * a.G;
            lim[x] = limit_of(a, i, n);
            const T* q = (const T*)a.q + b * a.q_b + i * a.q_s + (int64_t)(hk * a.G + g) * 2 * a.q_h;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int s = 0; s < KS; ++s) qf[x][m][s] = global_frag<false>(q + m * a.q_h, depth_of<P, KS>(s, h), a.D);
        }
        const int least = __builtin_amdgcn_readfirstlane(lim[0]);    // of the first row: limits rise

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

        const P* kb = (const P*)a.k + (int64_t)hk * 2 * a.k_h;
        const P* vb = (const P*)a.v + (int64_t)hk * a.v_h + dv0;
        const uint8_t* kxb = a.kx + (int64_t)hk * 2 * a.kx_h;
        const uint8_t* vxb = a.vx + (int64_t)hk * a.vx_h;
        RawKey<P, KS> kr[2][2];                                  // [16 keys][map]
        uint8_t ke[2][2] = {}, ve[NV] = {};
        u32x4 vr[NV];
        uint32_t there = 0, there_next = 0;                      // keys of the unit that are there, as bits
        // the pages of a unit's halves (ALIGNED) or of key l % 32
        int page[2], slot[2];
        const auto look = [&](int u) {
            const int j0 = u * BN;
            there_next = 0;
#pragma unroll
            for (int y = 0; y < (ALIGNED ? 2 : 1); ++y) {
                const int j = ALIGNED ? j0 + 16 * y : j0 + (l & 31);
                const int e = (int)divided((uint32_t)j, a.page);
                int p = a.table[b * a.table_b + min(e, a.width - 1)];
                slot[y] = j - e * (int)a.page.d;
                const bool ok = j < n && p >= 0 && p < a.pages;
                if (!ok) p = slot[y] = 0;
                page[y] = p;
                if constexpr (ALIGNED) {
                    const int left = n - j;
                    if (ok) there_next |= (left >= 16 ? 0xffffu : (1u << left) - 1u) << (16 * y);
                } else {
                    there_next = (uint32_t)__ballot(ok);
                }
            }
        };
        const auto fetch_keys = [&]() {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int p = ALIGNED ? page[y] : __shfl(page[0], 16 * y + c), s = ALIGNED ? slot[y] + c : __shfl(slot[0], 16 * y + c);
                const P* row = kb + p * a.k_p + s * a.k_s;
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    load_key<FULL>(kr[y][m], row + m * a.k_h, h, a.D);
                    if constexpr (sizeof(P) == 1) ke[y][m] = kxb[p * a.kx_p + s * a.kx_s + m * a.kx_h];
                }
            }
        };
        const auto fetch_values = [&]() {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = v * 64 + l, row = e / VPER, y = v * (64 / VPER) / 16;
                const int p = ALIGNED ? page[y] : __shfl(page[0], row), s = ALIGNED ? slot[y] + (row & 15) : __shfl(slot[0], row);
                if constexpr (sizeof(P) == 1) {
                    vr[v] = load16_any<FULL>((const uint8_t*)vb + p * a.v_p + s * a.v_s, e % VPER * E, dvn);
                    ve[v] = vxb[p * a.vx_p + s * a.vx_s];
                } else {
                    vr[v] = load16_any<FULL>(vb + p * a.v_p + s * a.v_s, e % VPER * E, dvn);
                }
            }
        };
        int u = begin + w;
        if (u < u1) { look(u); fetch_keys(); fetch_values(); }
        for (; u < u1; u += NW) {
            const int j0 = u * BN;
            const bool more = u + NW < u1;
            there = there_next;
            if (more) look(u + NW);
            f32x4 s[RT][2][2];                                   // [rows][map][16 keys]
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
#pragma unroll
                    for (int x = 0; x < RT; ++x) s[x][m][y] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int t = 0; t < KS; ++t) {
                        const auto kf = key_frag<FULL>(kr[y][m], t, h, a.D, scale_of(ke[y][m]));
#pragma unroll
                        for (int x = 0; x < RT; ++x) s[x][m][y] = mma(s[x][m][y], kf, qf[x][m][t]);
                    }
                }
            if (more) fetch_keys();
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = v * 64 + l, row = e / VPER, d = e % VPER * E;
                const bool ok = d < dvn && (there >> row & 1);
                bf16* to = vt + row * Values::LD + d;
                if constexpr (sizeof(P) == 1) {
                    const u32x4 x = shift16<FULL, uint8_t>(vr[v], d, dvn);
                    const float f = scale_of(ve[v]);
                    const bf16x8 zero = {}, x0 = widened(x[0], x[1], f), x1 = widened(x[2], x[3], f);
                    *(bf16x8*)to = ok ? x0 : zero;
                    *(bf16x8*)(to + 8) = ok ? x1 : zero;
                } else {
                    put16<Values::PLANE>(to, shift16<FULL, P>(vr[v], d, dvn), ok, P());
                }
            }
            if (more) fetch_values();
            if (j0 + BN > least || there != ~0u) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = 16 * y + 4 * h + e;
#pragma unroll
                        for (int x = 0; x < RT; ++x) {
                            const bool ok = j0 + j < lim[x] && (there >> j & 1);
                            s[x][0][y][e] = ok ? s[x][0][y][e] : -INFINITY;
                            s[x][1][y][e] = ok ? s[x][1][y][e] : -INFINITY;
                        }
                    }
            }
            Weights<T> p[RT][2];
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
                    float v[8];
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[4 * y + e] = __builtin_amdgcn_exp2f(fmaf(z[y][e], a.scale2, -safe[x][m]));
                            sum[x][m] += v[4 * y + e];
                        }
                    p[x][m].set(v);
                }
            const int vcol = few_col_lane<Values::LD>();
            wave_lds_fence();
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const auto vf = tile_col<KT, Values::LD, Values::PLANE, 16>(vt + vcol + 16 * t);
#pragma unroll
                for (int x = 0; x < RT; ++x) {
                    o[x][0][t] = p[x][0].times(o[x][0][t], vf);
                    o[x][1][t] = p[x][1].times(o[x][1][t], vf);
                }
            }
            wave_lds_fence();
            settle();
        }
        // the wavefronts' parts meet in LDS, over the tiles: statistics first, then the sums, halving the wavefronts
        __syncthreads();
        float* ml = (float*)lds;                                 // [NW][RT][2][2][16]
        float* acc = ml + NW * RT * 64;                          // [NW / 2][RT * 2 * NT * 4][64]
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                sum[x][m] = half_sum(quarter_sum(sum[x][m]));
                if (h == 0) {
                    float* to = ml + ((w * RT + x) * 2 + m) * 32 + c;
                    to[0] = top[x][m];
                    to[16] = sum[x][m];
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
                    const float* from = ml + ((k * RT + x) * 2 + m) * 32 + c;
                    all = fmaf(from[16], __builtin_amdgcn_exp2f(from[0] - base), all);
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
        if (w == 0) {
            const bool whole = begin == 0 && u1 == units;
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                const int mine = first + 16 * x + c;
                if (mine >= a.rows) continue;
                if (whole) {
                    const int i = mine / a.G, head = hk * a.G + mine - i * a.G;
                    T* out = (T*)a.out + (((int64_t)b * a.Sq + i) * a.H + head) * a.Dv + dv0;
                    // (a query that sees nothing answers 0, whatever lam is)
                    const bool none = sum[x][1] == 0.0f;
                    const float i0 = none ? 0.0f : 1.0f / sum[x][0], i1 = none ? 0.0f : a.lam[head] / sum[x][1];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        float r[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) r[e] = none ? 0.0f : fmaf(o[x][0][t][e], i0, -o[x][1][t][e] * i1);
                        store4(out, 16 * t + 4 * h, dvn, a.ovec, r);
                    }
                } else {
                    const int64_t row = (((int64_t)hk * a.parts + at) * 2 + (begin == 0 ? 1 : 0)) * a.rows + mine;
                    if (blockIdx.z == 0 && h == 0) *(f32x4*)(a.part_ml + 4 * row) = f32x4{top[x][0], sum[x][0], top[x][1], sum[x][1]};
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const int d = 16 * t + 4 * h;
                            if (dv0 + d < wide) *(f32x4*)(a.part + (row * 2 + m) * wide + dv0 + d) = o[x][m][t];
                        }
                }
            }
        }
        if (!a.parts || end <= units) return;
        // the next request, from its first unit on
        end -= units;
        begin = 0;
        __syncthreads();
    }
}

// Joins a row's parts: a workgroup a row of (request, query, head), a thread a value of each map.
template <typename T>
__global__ __launch_bounds__(256) void paged_join(PagedArgs a)
{
    __shared__ float f[2][MAX_PARTS];
    __shared__ float total[2];
    const int64_t id = blockIdx.x;
    const int head = (int)(id % a.H), i = (int)(id / a.H % a.Sq), b = (int)(id / a.H / a.Sq);
    const int hk = head / a.G, r = i * a.G + head % a.G, wide = (a.Dv + 3) / 4 * 4;
    T* out = (T*)a.out + id * a.Dv;
    const int units = units_of(positions(a, b));
    if (units == 0) {
        for (int d = threadIdx.x; d < a.Dv; d += 256) out[d] = (T)0.0f;
        return;
    }
    const int per = stretch_of(a, units_before(a, a.B)), before = units_before(a, b);
    const int p0 = before / per, p1 = (before + units - 1) / per, count = p1 - p0 + 1;
    if (count == 1) return;                              // (answered where it was computed)
    const auto row_of = [&](int p) { return (((int64_t)hk * a.parts + p0 + p) * 2 + (p == 0 ? 1 : 0)) * a.rows + r; };
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    if (w < 2) {
        float most = -INFINITY, sum = 0.0f;
        for (int p = l; p < count; p += 64) most = fmaxf(most, a.part_ml[4 * row_of(p) + 2 * w]);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        const float base = most == -INFINITY ? 0.0f : most;
        for (int p = l; p < count; p += 64) {
            const float* ml = a.part_ml + 4 * row_of(p) + 2 * w;
            const float g = ml[1] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ml[0] - base);
            f[w][p] = g;
            sum = fmaf(ml[1], g, sum);
        }
        sum = lanes_sum<64>(sum);
        if (l == 0) total[w] = sum;
    }
    __syncthreads();
    const bool none = total[1] == 0.0f;
    const float i0 = none ? 0.0f : 1.0f / total[0], i1 = none ? 0.0f : a.lam[head] / total[1];
    for (int d = threadIdx.x; d < a.Dv; d += 256) {
        float x = 0.0f, y = 0.0f;
#pragma unroll 4
        for (int p = 0; p < count; ++p) {
            const float* from = a.part + row_of(p) * 2 * wide + d;
            // (a part whose keys were all hidden adds nothing)
            const float g0 = f[0][p], g1 = f[1][p], v0 = from[0], v1 = from[wide];
            x += g0 == 0.0f ? 0.0f : g0 * v0;
            y += g1 == 0.0f ? 0.0f : g1 * v1;
        }
        out[d] = (T)(none ? 0.0f : fmaf(x, i0, -y * i1));
    }
}

int dim_tile(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

struct PagedPlan { int rt, row_tiles, chunks, parts; size_t part, ml; };

PagedPlan paged_plan(const sconv_paged_desc_t& d, size_t ws_bytes)
{
    PagedPlan p = {};
    if (d.B == 0 || d.Sq == 0) return p;
    const int G = d.H / d.Hkv, rows = d.Sq * G, DVT = dim_tile(d.pages.D) == 32 ? 64 : 128;
    p.rt = rows > 16 && d.type == SCONV_BF16 ? 2 : 1;
    p.row_tiles = (rows + 16 * p.rt - 1) / (16 * p.rt);
    p.chunks = (d.pages.Dv + DVT - 1) / DVT;
    // as many stretches as fill the chip twice over, and no more than the caches can have
    const int64_t units = (int64_t)d.B * (((int64_t)d.pages.table_width * d.pages.page_size + BN - 1) / BN), base = (int64_t)d.Hkv * p.row_tiles * p.chunks;
    if (units >= (int64_t(1) << 31)) return p;
    int64_t parts = std::min<int64_t>(std::min<int64_t>((512 + base - 1) / base, (units + LEAST - 1) / LEAST), MAX_PARTS);
    const int64_t wide = (d.pages.Dv + 3) / 4 * 4, each = (int64_t)d.Hkv * 2 * rows * (2 * wide + 4) * (int64_t)sizeof(float);
    if ((size_t)(parts * each) > ws_bytes) return p;
    p.parts = (int)parts;
    p.part = (size_t)(parts * d.Hkv * 2 * rows * 2 * wide) * sizeof(float);
    p.ml = (size_t)(parts * d.Hkv * 2 * rows * 4) * sizeof(float);
    return p;
}

template <typename T, typename P, bool FULL, bool ALIGNED, int DT, int DVT, int RT>
int paged_launch(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    constexpr size_t tiles = (size_t)NW * Tile<typename Kept<P>::type, BN, DVT>::SIZE * 2, join = (size_t)(NW * RT * 64 + NW / 2 * RT * 2 * DVT * 16) * 4;
    constexpr size_t lds = join > tiles ? join : tiles;
    const auto kern = paged_attn<T, P, FULL, ALIGNED, DT, DVT, RT>;
    const int rc = allow_lds(kern, lds);
    if (rc) return rc;
    const int64_t grid = (int64_t)(p.parts ? p.parts : a.B) * a.Hkv * p.row_tiles;
    if (!grid_fits(grid, 256) || !grid_fits((int64_t)a.B * a.Sq * a.H, 256)) return SCONV_EUNSUPPORTED;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid, 1, (unsigned)p.chunks), dim3(256), lds, stream, a);
    return launch_status();
}

template <typename T, typename P, bool FULL, bool ALIGNED>
int paged_shape(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    const int DT = dim_tile(a.D);
    if constexpr (sizeof(T) == 2)
        if (p.rt == 2)
            return DT == 32 ? paged_launch<T, P, FULL, ALIGNED, 32, 64, 2>(a, p, stream)
                 : DT == 64 ? paged_launch<T, P, FULL, ALIGNED, 64, 128, 2>(a, p, stream) : paged_launch<T, P, FULL, ALIGNED, 128, 128, 2>(a, p, stream);
    return DT == 32 ? paged_launch<T, P, FULL, ALIGNED, 32, 64, 1>(a, p, stream)
         : DT == 64 ? paged_launch<T, P, FULL, ALIGNED, 64, 128, 1>(a, p, stream) : paged_launch<T, P, FULL, ALIGNED, 128, 128, 1>(a, p, stream);
}

template <typename T, typename P>
int paged_run(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    const int DT = dim_tile(a.D), DVT = DT == 32 ? 64 : 128;
    const bool full = a.D == DT && a.Dv % DVT == 0, aligned = a.page.d % 16 == 0;
    const int rc = full ? (aligned ? paged_shape<T, P, true, true>(a, p, stream) : paged_shape<T, P, true, false>(a, p, stream))
                        : (aligned ? paged_shape<T, P, false, true>(a, p, stream) : paged_shape<T, P, false, false>(a, p, stream));
    if (rc || p.parts == 0) return rc;
    hipLaunchKernelGGL((paged_join<T>), dim3((unsigned)((int64_t)a.B * a.Sq * a.H)), dim3(256), 0, stream, a);
    return launch_status();
}

}  // namespace

size_t paged_workspace(const sconv_paged_desc_t& d)
{
    const PagedPlan p = paged_plan(d, ~(size_t)0 >> 1);
    return p.part + p.ml;
}

int launch_paged(const sconv_paged_desc_t& d, const void* q, const sconv_pages_dev_t& pages, const float* lam, const int32_t* lengths,
                 void* out, void* ws, size_t ws_bytes, hipStream_t stream)
{
    const sconv_pages_t& g = d.pages;
    const PagedPlan p = paged_plan(d, ws_bytes);
    PagedArgs a = {};
    a.q = q; a.k = pages.k; a.v = pages.v; a.kx = pages.ks; a.vx = pages.vs; a.table = pages.table; a.lam = lam; a.len = lengths; a.out = out;
    a.B = d.B; a.Sq = d.Sq; a.H = d.H; a.Hkv = d.Hkv; a.G = d.H / d.Hkv; a.D = g.D; a.Dv = g.Dv; a.causal = d.causal; a.rows = d.Sq * a.G;
    a.pages = g.pages; a.width = g.table_width; a.capacity = g.pages > 0 ? g.table_width * g.page_size : 0; a.parts = p.parts;
    a.ovec = aligned_to(out, 16) && g.Dv % 4 == 0;
    a.scale2 = d.scale * 1.44269504088896340736f;
    a.q_b = d.q_b; a.q_s = d.q_s; a.q_h = d.q_h; a.k_p = g.k_p; a.k_s = g.k_s; a.k_h = g.k_h; a.v_p = g.v_p; a.v_s = g.v_s; a.v_h = g.v_h;
    a.kx_p = g.ks_p; a.kx_s = g.ks_s; a.kx_h = g.ks_h; a.vx_p = g.vs_p; a.vx_s = g.vs_s; a.vx_h = g.vs_h; a.table_b = g.table_b;
    a.page = divide_by((uint32_t)g.page_size);
    a.part = (float*)ws;
    a.part_ml = (float*)((char*)ws + p.part);
    if (d.type == SCONV_BF16) return g.type == SCONV_E4M3 ? paged_run<bf16, e4m3>(a, p, stream) : paged_run<bf16, bf16>(a, p, stream);
    return g.type == SCONV_E4M3 ? paged_run<float, e4m3>(a, p, stream) : paged_run<float, float>(a, p, stream);
}

}  // namespace sconv
