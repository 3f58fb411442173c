// Differential attention: what its kernels share.
//
// Layout of the matrix products.  A 32 x 32 product tile takes from each lane 8 elements of a row of A (row l % 32) and 8 of a
// column of B (column l % 32), both at depths 8 (l / 32) .. + 7 of a 16-deep step.  Of the result each lane holds column
// l % 32, rows 8 (r / 4) + 4 (l / 32) + r % 4 in registers r = 0..15.
// 32-bit operands go through the 16-bit matrix pipe as well, as three pieces that hold 8 bits of the value each (their sum is the
// value) and six of the nine products of pieces.  The three left out are within 2^-21 of the product and, as pieces are cut off, of its sign:
// a product comes out 0.63 * 2^-24 short on average, which is what a 32-bit rounding may do.  That is 192 cycles for what the 32-bit
// pipe does in 512.
// So a result can be the next product's B as it stands in its lane: registers 8s..8s+7 are the depths
//   16 s + 4 (l / 32) + {0, 1, 2, 3, 8, 9, 10, 11}
// of step s, provided that A's elements come in that order (col_frag below).  Scores are therefore formed transposed - keys down,
// queries across -: a query's softmax runs inside a lane and its partner, and the weights never leave the registers.
#pragma once

#include "sconv_tokens_common.h"

namespace sconv {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const void* q; const void* k; const void* v; const float* lam; const int32_t* len; const uint8_t* mask;
    void* out; void* second; float* lse;                     // forward: written
    const void* dout; const void* out_in; const void* second_in; const float* lse_in;   // backward
    void* dq; void* dk; void* dv;
    float* part; float* part_ml;                             // forward over several splits: [split][B Hkv][rows]..
    float* delta; float* dlam_part;                          // backward: [2][B][H][Sq], [B][H][Sq]
    float* part_q; float* part_s; float* part_k; float* part_v;   // parts of dq, dlam_part, dk, dv, in their layouts
    int row_splits, row_keys, key_splits;                    // keys a part of dq; parts of dk and dv
    int B, Sq, Sk, H, Hkv, G, D, Dv, causal, rows;           // rows = Sq * G: of one request and key head, r = i * G + g
    int splits, split_keys, row_tiles;
    int ovec;                                                // outputs can be written 16 bytes at a time
    float scale, scale2;                                     // scale2 = scale * log2(e)
    int64_t q_b, q_s, q_h, k_b, k_s, k_h, v_b, v_s, v_h, mask_b;
};

struct bf16x8x3 { bf16x8 p[3]; };
template <typename T> struct Frag;
template <> struct Frag<bf16> { typedef bf16x8 type; static constexpr int PLANES = 1; };
template <> struct Frag<float> { typedef bf16x8x3 type; static constexpr int PLANES = 3; };

__device__ __forceinline__ f32x16 mma(f32x16 c, bf16x8 a, bf16x8 b) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f32x4 c, bf16x8 a, bf16x8 b) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <typename C>
__device__ __forceinline__ C mma(C c, const bf16x8x3& a, const bf16x8x3& b)
{
    c = mma(c, a.p[2], b.p[0]);
    c = mma(c, a.p[0], b.p[2]);
    c = mma(c, a.p[1], b.p[1]);
    c = mma(c, a.p[1], b.p[0]);
    c = mma(c, a.p[0], b.p[1]);
    return mma(c, a.p[0], b.p[0]);
}

// Two values as pieces: the upper 16 bits of the value, of what is left, and of what is left then.  An Inf stands in the third piece alone,
// behind two of the type's largest value: the third meets the other operand's first only, which is 0 under a value of 0 alone, while the other
// operand's lower pieces are 0 wherever its bits are few, and Inf * 0 would be NaN for a product that is Inf.  NaN ends there too.  WEIGHT: a
// softmax weight, never Inf.
template <bool WEIGHT>
__device__ __forceinline__ float upper(float x)
{
    const float most = __uint_as_float(0x7f7f0000u);
    if constexpr (!WEIGHT) x = __builtin_amdgcn_fmed3f(x, -most, most);
    return __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}
template <bool WEIGHT>
__device__ __forceinline__ void pieces(float x, float y, uint32_t& hi, uint32_t& mid, uint32_t& lo)
{
    const float xh = upper<WEIGHT>(x), yh = upper<WEIGHT>(y), xr = x - xh, yr = y - yh;
    const float xm = upper<WEIGHT>(xr), ym = upper<WEIGHT>(yr), xl = xr - xm, yl = yr - ym;
    hi = __builtin_amdgcn_perm(__float_as_uint(yh), __float_as_uint(xh), 0x07060302u);
    mid = __builtin_amdgcn_perm(__float_as_uint(ym), __float_as_uint(xm), 0x07060302u);
    lo = __builtin_amdgcn_perm(__float_as_uint(yl), __float_as_uint(xl), 0x07060302u);
}
template <bool WEIGHT>
__device__ __forceinline__ bf16x8x3 in_pieces(const float (&v)[8])
{
    union { uint32_t u[4]; bf16x8 f; } p[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) pieces<WEIGHT>(v[2 * i], v[2 * i + 1], p[0].u[i], p[1].u[i], p[2].u[i]);
    return bf16x8x3{{p[0].f, p[1].f, p[2].f}};
}

// The same in tiles of 16 x 16 (32 deep): a lane has 8 elements at depths 8 (l / 16) .. + 7 of row or column l % 16, and of the result
// column l % 16, rows 4 (l / 16) + 0..3.  Two results of 16 keys are the next product's B at depths
//   4 (l / 16) + {0, 1, 2, 3, 16, 17, 18, 19}.

// Ends a loop's round of products.  The compiler keeps its distance between a product and whoever reads its result, except, seen in
// 32-bit code, where the first copy of a result stands behind the loop's exit branch: it then read registers a few
// cycles early.  18 wait states are what the longest product needs.
__device__ __forceinline__ void settle()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 3");
    __builtin_amdgcn_sched_barrier(0);
}

// A tile in LDS: rows of W 16-bit elements and 16 bytes of padding, so that lanes reading one column chunk of consecutive rows meet
// different banks; 32-bit values in three such planes.
template <typename T, int ROWS, int W>
struct Tile { static constexpr int LD = W + 8, PLANE = ROWS * LD, SIZE = Frag<T>::PLANES * PLANE; };

// 8 consecutive elements from an address aligned to 16 bytes.
__device__ __forceinline__ bf16x8 row_frag(const bf16* p) { return *(const bf16x8*)p; }
template <typename T, int PLANE>
__device__ __forceinline__ typename Frag<T>::type tile_row(const bf16* p)
{
    if constexpr (sizeof(T) == 2) return row_frag(p);
    else return bf16x8x3{{row_frag(p), row_frag(p + PLANE), row_frag(p + 2 * PLANE)}};
}

// The transposed tile's row fragment: column l % 32 of 32, depths (rows) 4 (l / 32) + {0..3} and SKIP more.  p: the tile at its first row
// and column, plus col_lane().
template <int LD, int SKIP = 8>
__device__ __forceinline__ bf16x8 col_frag(const bf16* p)
{
    typedef __attribute__((address_space(3))) s16x4 lds4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + SKIP * LD));
    union { s16x4 s[2]; bf16x8 v; } u;
    u.s[0] = a; u.s[1] = b;
    return u.v;
}
template <typename T, int LD, int PLANE, int SKIP = 8>
__device__ __forceinline__ typename Frag<T>::type tile_col(const bf16* p)
{
    if constexpr (sizeof(T) == 2) return col_frag<LD, SKIP>(p);
    else return bf16x8x3{{col_frag<LD, SKIP>(p), col_frag<LD, SKIP>(p + PLANE), col_frag<LD, SKIP>(p + 2 * PLANE)}};
}
// Where a lane reads (16 lanes of the transposing read take four rows of 16 columns; lane i has row i / 4, four columns).
template <int LD>
__device__ __forceinline__ int col_lane()
{
    const int l = threadIdx.x & 63;
    return (4 * (l >> 5) + ((l & 15) >> 2)) * LD + ((l >> 4) & 1) * 16 + (l & 3) * 4;
}
// For tiles of 16 x 16: column l % 16 of 16, depths 4 (l / 16) + {0..3, 16..19}.
template <int LD>
__device__ __forceinline__ int few_col_lane()
{
    const int l = threadIdx.x & 63;
    return (4 * (l >> 4) + ((l & 15) >> 2)) * LD + (l & 3) * 4;
}

// Registers 8s..8s+7 of a result as the next product's B.
__device__ __forceinline__ void to_frag(const float (&v)[8], bf16x8& f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (bf16)v[i];
}
__device__ __forceinline__ void to_frag(const float (&v)[8], bf16x8x3& f) { f = in_pieces<true>(v); }
template <typename F>
__device__ __forceinline__ void to_frag(const f32x16& p, int s, F& f)
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[8 * s + i];
    to_frag(v, f);
}

// What to_frag's rounding to 16 bits left out (32 bits: nothing).
__device__ __forceinline__ void rest_frag(const float (&v)[8], const bf16x8& f, bf16x8& rest)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = (bf16)(v[i] - (float)f[i]);
}
// Weights in two values, cut off and not rounded so that both are positive where the weight is: an Inf that meets them stays one.
__device__ __forceinline__ void weight_frags(const float (&v)[8], bf16x8& f, bf16x8& rest)
{
    union { uint32_t u[4]; bf16x8 f; } hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) hi.u[i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
    f = hi.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = (bf16)fmaxf(v[i] - upper<true>(v[i]), v[i] * 0x1p-17f);
}
// Products with values held twice as finely as 16 bits do: B = f + rest.
template <int LD>
__device__ __forceinline__ f32x16 mma_fine(f32x16 c, const bf16* a, const bf16x8& f, const bf16x8& rest)
{
    const bf16x8 x = col_frag<LD>(a);
    return mma(mma(c, x, rest), x, f);
}
template <typename T, typename Tl>
__device__ __forceinline__ f32x16 mma_fine(f32x16 c, const bf16* a, const f32x16& v, int s)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[8 * s + i];
    if constexpr (sizeof(T) == 4) return mma(c, tile_col<T, Tl::LD, Tl::PLANE>(a), in_pieces<false>(x));
    else {
        bf16x8 f, rest;
        to_frag(x, f);
        rest_frag(x, f, rest);
        return mma_fine<Tl::LD>(c, a, f, rest);
    }
}

// 16 bytes of a row in memory into a tile (rows that are not there: zeros).
template <int PLANE>
__device__ __forceinline__ void put16(bf16* to, u32x4 r, bool there, bf16)
{
    *(u32x4*)to = there ? r : u32x4{0, 0, 0, 0};
}
template <int PLANE>
__device__ __forceinline__ void put16(bf16* to, u32x4 r, bool there, float)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    if (!there) r = u32x4{0, 0, 0, 0};
    u32x2 p[3];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t hi, mid, lo;
        pieces<false>(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]), hi, mid, lo);
        p[0][i] = hi; p[1][i] = mid; p[2][i] = lo;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *(u32x2*)(to + k * PLANE) = p[k];
}

// 16 bytes of elements d.. of a row that has `have` of them, in two steps, so that nothing waits for the load before its use.  VEC: d
// and the row are aligned and `have` is whole 16 bytes; where d lies beyond, an address inside is read and the result is to be cleared.
// Otherwise 16 bytes at any address, the last ones of the row where 16 bytes from d would pass its end, which shift16 then moves down
// (clearing what lies beyond); rows shorter than 16 bytes come element by element.
template <bool VEC, typename T>
__device__ __forceinline__ u32x4 load16(const T* row, int d, int have)
{
    constexpr int E = 16 / sizeof(T);
    if constexpr (VEC) return *(const u32x4*)(row + (d < have ? d : 0));
    if (have >= E) {
        typedef u32x4 u32x4_any __attribute__((aligned(2)));
        return *(const u32x4_any*)(row + min(d, have - E));
    }
    union { u32x4 u; T e[E]; } r;
#pragma unroll
    for (int i = 0; i < E; ++i) r.e[i] = row[d + i < have ? d + i : 0];
#pragma unroll
    for (int i = 0; i < E; ++i) if (d + i >= have) r.e[i] = (T)0.0f;
    return r.u;
}
template <bool VEC, typename T>
__device__ __forceinline__ u32x4 shift16(u32x4 v, int d, int have)
{
    constexpr int E = 16 / sizeof(T);
    if (VEC || have < E) return v;
    const int drop = min(max(d - (have - E), 0), E);   // elements before d
    uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
    if (drop >= E / 2) { lo = hi; hi = 0; }
    const int bits = drop % (E / 2) * (int)sizeof(T) * 8;
    lo = bits ? lo >> bits | hi << (64 - bits) : lo;
    hi >>= bits;
    if (drop >= E) lo = 0;
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// A fragment of a row in memory as it is loaded, and as it is used (cleared beyond `have`): apart, so that nothing waits for the load
// before its use.
template <typename T> struct Raw { u32x4 u[sizeof(T) / 2]; };
template <bool VEC, typename T>
__device__ __forceinline__ void load_raw(Raw<T>& r, const T* row, int d, int have)
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = load16<VEC>(row, d + 4 * i, have);
}
template <bool VEC>
__device__ __forceinline__ bf16x8 raw_frag(const Raw<bf16>& r, int d, int have, bool ragged)
{
    union { u32x4 u; bf16x8 v; } x;
    x.u = shift16<VEC, bf16>(r.u[0], d, have);
    if (ragged && d >= have) x.u = u32x4{0, 0, 0, 0};
    return x.v;
}
template <bool VEC>
__device__ __forceinline__ bf16x8x3 raw_frag(const Raw<float>& r, int d, int have, bool ragged)
{
    union { u32x4 u[2]; float v[8]; } x;
    x.u[0] = shift16<VEC, float>(r.u[0], d, have);
    x.u[1] = shift16<VEC, float>(r.u[1], d + 4, have);
    if (ragged && d >= have) x.u[0] = u32x4{0, 0, 0, 0};
    if (ragged && d + 4 >= have) x.u[1] = u32x4{0, 0, 0, 0};
    return in_pieces<false>(x.v);
}
template <bool VEC, typename T>
__device__ __forceinline__ typename Frag<T>::type global_frag(const T* row, int d, int have)
{
    Raw<T> r;
    load_raw<VEC>(r, row, d, have);
    return raw_frag<VEC>(r, d, have, true);
}

// Four neighbouring results of a row (columns d..d+3 of `have`).
template <typename T>
__device__ __forceinline__ void store4(T* row, int d, int have, bool vec, const float* v)
{
    if (vec) {
        if (d < have) store_vec<4>(row + d, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < have) row[d + i] = (T)v[i];
    }
}

// The other half of the wavefront's value (lane l +- 32).
__device__ __forceinline__ float half_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The neighbouring 16 lanes' value (lane l ^ 16).
__device__ __forceinline__ float quarter_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quarter_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Which of 32 keys from js on a query sees that sees `lim` of them, as bits; and what the others' scores become.
__device__ __forceinline__ uint32_t seen_bits(int js, int lim, uint32_t word)
{
    const int left = lim - js;
    return left >= 32 ? word : left <= 0 ? 0u : word & ((1u << left) - 1u);
}
__device__ __forceinline__ float masked(float v, uint32_t bits, int pos, uint32_t other)
{
    const uint32_t m = (uint32_t)((int32_t)(bits << (31 - pos)) >> 31);      // all ones where bit pos is set
    return __uint_as_float((__float_as_uint(v) & m) | (other & ~m));
}

// Keys of request b that exist.
__device__ __forceinline__ int keys_of(const AttnArgs& a, int b) { return a.len ? min(max(a.len[b], 0), a.Sk) : a.Sk; }
// How many of its n keys query i sees, the mask aside.
__device__ __forceinline__ int limit_of(const AttnArgs& a, int i, int n)
{
    if (!a.causal) return n;
    const int64_t lim = (int64_t)i + n - a.Sq + 1;
    return (int)(lim < 0 ? 0 : lim > n ? n : lim);
}

// ROWS rows of a tile on their way from memory to LDS, through registers, so that the loads of one tile run under the products of
// the one before.  A row has PARTS rows of W elements of memory beside each other (the two keys of a head).
template <typename T, bool VEC, int ROWS, int PARTS, int W, int THREADS>
struct Stage {
    typedef Tile<T, ROWS, PARTS * W> To;
    static constexpr int E = 16 / sizeof(T), PER = PARTS * W / E, N = ROWS * PER / THREADS;
    static_assert(N * THREADS == ROWS * PER, "whole vectors for every thread");
    u32x4 r[N];

    // row j of the tile: base + (j0 + j) * stride, its part m at + m * part; rows from `rows` on are not there (one that is, is
    // read instead, and cleared by store).
    __device__ __forceinline__ void load(const T* base, int64_t stride, int64_t part, int j0, int rows, int have)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int e = n * THREADS + threadIdx.x, row = e / PER, c = e % PER, m = c / (W / E), d = (c % (W / E)) * E;
            r[n] = load16<VEC>(base + (int64_t)min(j0 + row, rows - 1) * stride + m * part, d, have);
        }
    }
    // words: a bit for every row that is there (LDS), null: all are
    __device__ __forceinline__ void store(bf16* tile, const uint32_t* words, int have) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int e = n * THREADS + threadIdx.x, row = e / PER, c = e % PER, d = (c % (W / E)) * E;
            const bool there = d < have && (!words || (words[row >> 5] >> (row & 31) & 1));
            put16<To::PLANE>(tile + row * To::LD + c * E, shift16<VEC, T>(r[n], d, have), there, T());
        }
    }
};

// The arguments both directions share.
AttnArgs attn_args(const sconv_diffattn_desc_t& d, const void* q, const void* k, const void* v, const float* lam,
                   const int32_t* lengths, const uint8_t* mask);

// Whether q, k and v can be read 16 bytes at a time.
bool attn_vector(const AttnArgs& a, int type);

// 16-bit tiles that go from memory to LDS directly: rows of W elements without padding, whose 16-byte chunks stand at chunk ^ turn(row)
// of every eight.  turn() differs over eight rows, for lanes that read one chunk of each, and by whole 32 bytes over four, for
// the transposing read of four rows, so that these lie in different banks (2.7 conflict cycles an LDS instruction are counted all the same
// over 12544 queries; which lanes the hardware takes together was not looked into).  A wavefront's load fills 1024
// bytes in a row; each lane chooses the chunk of memory that belongs where its 16 bytes come to lie.  The buffer ends with the last
// row's last part: with one part, and rows that do not overlap, rows that are not there come as zeros; with two parts they may come
// as what lies between the parts.
template <int ROWS, int PARTS, int W, int NW>
struct Direct {
    static constexpr int RW = PARTS * W, N = ROWS * RW * 2 / 1024 / NW;     // loads of a wavefront
    static_assert(N * NW * 1024 == ROWS * RW * 2, "whole loads for every wavefront");
    uint32_t off[N];
    __device__ __forceinline__ static int turn(int row) { return (row & 3) << 1 | (row >> 2 & 1); }
    __device__ __forceinline__ void init(int64_t stride, int64_t part)
    {
        const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = ((i * NW + w) * 64 + l) * 8, row = at / RW, chunk = at % RW / 8;
            const int from = chunk ^ turn(row), m = from / (W / 8), d = from % (W / 8) * 8;
            off[i] = (uint32_t)(row * stride + m * part + d) * 2;
        }
    }
    // rows j0 .. j0 + ROWS of base (uniform), of which `rows` exist
    __device__ __forceinline__ void load(const bf16* base, int64_t stride, int64_t part, int j0, int rows, bf16* tile) const
    {
#if defined(__HIP_DEVICE_COMPILE__)                    // (the host's compiler does not know buffer resources)
        typedef __attribute__((address_space(3))) void lds_t;
        const int64_t left = ((int64_t)(rows - j0 - 1) * stride + (PARTS - 1) * part + W) * 2, most = (int64_t)1 << 31;
        const uint64_t at = (uint64_t)(base + (int64_t)j0 * stride);
        const uint64_t p = ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, __builtin_amdgcn_readfirstlane((uint32_t)(left < most ? left : most)), 0x00027000);
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_t*)(tile + (i * NW + w) * 512), 16, off[i], 0, 0, 0);
#endif
    }
    // this wavefront's loads have come: before the barrier behind which others read them, as nothing in the language ties loads to LDS to it
    __device__ __forceinline__ static void arrived()
    {
#if defined(__HIP_DEVICE_COMPILE__)
        __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0)
#endif
    }
    // a row's fragment: row l % 32 of the tile, columns c .. c + 7 + 8 (l / 32): tile + at[c / 16 % 4] + c / 64 * 64
    __device__ __forceinline__ static void row_lane(int (&at)[4])
    {
        const int l = threadIdx.x & 63, row = l & 31, h = l >> 5;
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = row * RW + ((2 * i + h) ^ turn(row)) * 8;
    }
    // a column fragment (col_frag): columns 32 t.., rows from 16 s: tile + at[t % 2] + t / 2 * 64 + 16 s * RW
    __device__ __forceinline__ static void col_lane(int (&at)[2])
    {
        const int l = threadIdx.x & 63, row = 4 * (l >> 5) + ((l & 15) >> 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) at[i] = row * RW + (((4 * i + 2 * ((l >> 4) & 1) + ((l & 3) >> 1)) ^ turn(row)) * 8) + (l & 1) * 4;
    }
    // clears the rows whose bit is 0
    __device__ __forceinline__ static void clear(bf16* tile, const uint32_t* words)
    {
#pragma unroll
        for (int e = threadIdx.x; e < ROWS * RW / 8; e += 64 * NW) {
            const int row = e / (RW / 8);
            if (!(words[row >> 5] >> (row & 31) & 1)) *(u32x4*)(tile + e * 8) = u32x4{0, 0, 0, 0};
        }
    }
};

// Sets the dynamic LDS size a kernel may ask for, where it is above the default.
template <typename K>
inline int allow_lds(K kern, size_t bytes)
{
    if (bytes <= 64 * 1024) return SCONV_OK;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess
               ? SCONV_OK : SCONV_ELAUNCH;
}

}  // namespace sconv
