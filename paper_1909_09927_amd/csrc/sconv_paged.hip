// Differential attention of new tokens over a paged cache (formulas in sconv_tokens.h, the cache in sconv_serving.h).
//
// Bound by the cache's read.  The keys of all requests, laid end to end in units of 32, are shared out among wavefronts by their number, so
// that wavefronts are alike whatever the requests' lengths: each walks its stretch alone, request after request, without barriers; a request
// that lies within one stretch is answered there, others leave parts, which a second kernel joins.  Where every request begins follows from the
// lengths, which each wavefront adds up itself.
// DIRECT (heads as wide as the tile, 16-byte rows, pages of whole 16 slots): keys, values and their scales go from memory to LDS without
// registers, two units deep.  Otherwise keys go to registers as the product reads them and values through registers to LDS (to be read down
// the keys), the next unit's on their way under this one's products.  8-bit values become 16-bit ones, exactly, on their way to
// the products.  Scores are formed transposed - keys down, queries across -, so a softmax stays within a lane's quarter and the weights never
// leave the registers.  Weights go as three 16-bit values for their product with V.
#include <algorithm>

#include "sconv_diffattn_common.h"
#include "sconv_serving_common.h"

namespace sconv {

namespace {

constexpr int BN = 32;                   // keys of a unit
constexpr int PLACES = 1024;             // wavefronts: one to a SIMD.  (Two: 64 requests of up to 784 35 -> 38 us, 16 of up to 32768 68 -> 71.)
constexpr int MAX_PARTS = PLACES;

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
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <typename C>
__device__ __forceinline__ C mma(C c, const bf16x8& a, const bf16x8x3& b)
{
    c = mma(c, a, b.p[2]);
    c = mma(c, a, b.p[1]);
    return mma(c, a, b.p[0]);
}

__device__ __forceinline__ int positions(const PagedArgs& a, int b) { return min(max(a.len[b], 0), a.capacity); }
__device__ __forceinline__ int units_of(int n) { return (int)(((uint32_t)n + BN - 1) / BN); }      // (n up to 2^31 - 1)

// All requests' units, and those of requests before b: every wavefront adds them up for itself.
__device__ __forceinline__ int units_before(const PagedArgs& a, int upto)
{
    const int l = threadIdx.x & 63;
    int v = 0;
    for (int b = l; b < upto; b += 64) v += units_of(positions(a, b));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    return __builtin_amdgcn_readfirstlane(v);
}
// Units of a stretch.
__device__ __forceinline__ int stretch_of(const PagedArgs& a, int units) { return max((units + a.parts - 1) / a.parts, 1); }
// Of stretch `at`: its first unit, counted from request b's first, and its end, likewise, and b's positions; false: it has none.
__device__ __forceinline__ bool find_stretch(const PagedArgs& a, int at, int& b, int& begin, int& end, int& n)
{
    const int l = threadIdx.x & 63;
    int all, u = 0, per = 0, base = 0;
    if (a.B > 64) {
        all = units_before(a, a.B);
        per = stretch_of(a, all);
        u = (int)min((int64_t)at * per, (int64_t)all);
        if (u == all) return false;
    }
    for (int b0 = 0;; b0 += 64) {
        const int length = b0 + l < a.B ? positions(a, b0 + l) : 0, mine = units_of(length);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int t = __shfl_up(upto, d);
            if (l >= d) upto += t;
        }
        if (a.B <= 64) {
            all = __builtin_amdgcn_readlane(upto, 63);
            per = stretch_of(a, all);
            u = (int)min((int64_t)at * per, (int64_t)all);
            if (u == all) return false;
        }
        const uint64_t past = __ballot(base + upto > u);
        if (past) {
            const int lane = __builtin_ctzll(past);
            b = b0 + lane;
            const int before = base + __builtin_amdgcn_readlane(upto - mine, lane);
            begin = u - before;
            end = (int)min((int64_t)u + per, (int64_t)all) - before;
            n = __builtin_amdgcn_readlane(length, lane);
            return true;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
        if (b0 + 64 >= a.B) return false;                // (not reached: the units add up to more than u)
    }
}

// The arguments once more, from where the kernel got them: what is wanted between requests only need not lie in scalar registers, of which the
// loop over units has too few.
typedef __attribute__((address_space(4))) const PagedArgs* ArgsAgain;
__device__ __forceinline__ ArgsAgain again()
{
#if defined(__HIP_DEVICE_COMPILE__)
    ArgsAgain p = (ArgsAgain)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
#else
    return nullptr;
#endif
}

// How many of a request's n positions query i of Sq sees.
__device__ __forceinline__ int limit_of(int causal, int Sq, int i, int n)
{
    if (!causal) return n;
    const int64_t lim = (int64_t)i + n - Sq + 1;
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

// A row's weights for their product with the values: three 16-bit values that make up the weight's 32 bits.  16-bit values of the cache meet them as they
// are, an Inf among them, too, so each is positive where the weight is: the largest 16-bit value below the weight, the largest below what is left, and what is
// left then, which 16 bits hold.  (Two would leave 2^-16 of a weight out: where two keys cancel to 2^-11 that is 1 % of the answer.  16 requests of up to
// 32768, 8 bits 70.8 us with two, 70.1 with three; 64 of up to 784, 16 bits 34.7 and 35.0; 2048 short ones with 8 heads 91 and 97.)
template <typename T> struct Weights;
template <> struct Weights<bf16> {
    bf16x8 p[3];
    __device__ __forceinline__ static float below(float x) { return __uint_as_float(__builtin_elementwise_sub_sat(__float_as_uint(x), 1u) & 0xffff0000u); }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        union { uint32_t u[4]; bf16x8 f; } q[3];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[2] = {v[2 * i], v[2 * i + 1]};
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                const float a = n < 2 ? below(x[0]) : x[0], b = n < 2 ? below(x[1]) : x[1];
                q[n].u[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
                x[0] -= a;
                x[1] -= b;
            }
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) p[n] = q[n].f;
    }
    template <typename V> __device__ __forceinline__ f32x4 times(f32x4 c, const V& v) const { return mma(mma(mma(c, v, p[2]), v, p[1]), v, p[0]); }
};
template <> struct Weights<float> {
    bf16x8x3 p;
    __device__ __forceinline__ void set(const float (&v)[8]) { p = in_pieces<true>(v); }
    template <typename V> __device__ __forceinline__ f32x4 times(f32x4 c, const V& v) const { return mma(c, v, p); }
};

// Units in LDS (DIRECT).  A key's two rows stand beside each other, RK bytes, a value's RV; their 16-byte chunks stand at chunk ^ turn, so that
// the lanes that are served together meet different banks: 16 keys' rows of one chunk, and in the transposing read 8 (8 bits: 16) values' rows
// of one or two.  Behind them the dwords that hold the scales of every key (both maps) and value.
template <typename P, int DT, int DVT>
struct Unit {
    static constexpr int ES = sizeof(P), RK = 2 * DT * ES, RV = DVT * ES, CK = RK / 16, CV = RV / 16;
    static constexpr int K = BN * RK, V = BN * RV, SCALES = ES == 1 ? 256 : 0;       // bytes; SCALES: twice
    static constexpr int NK = K / 1024, NV = V / 1024, HK = NK / 2, HV = NV / 2;     // loads of a unit and of half of it
    static constexpr int KLOADS = NK + (ES == 1), VLOADS = NV + (ES == 1);
    static constexpr int SIZE = K + V + 2 * SCALES, STAGES = 2, LDS = STAGES * SIZE + (ES == 1 ? 3 * BN * 4 : 0);
    __device__ __forceinline__ static int turn_k(int key) { return RK >= 256 ? key & 15 : key / (256 / std::min(RK, 256)) & (CK - 1); }
    __device__ __forceinline__ static int turn_v(int key)
    {
        if (ES == 1) return RV == 128 ? (key >> 1 & 3) | (key >> 4 & 1) << 2 : (key >> 2 & 1) | (key >> 4 & 1) << 1;
        return RV == 256 ? (key & 7) << 1 : (key >> 1 & 3) << 1;
    }
};

// vmcnt(n): all but the n youngest of the wavefront's loads have come
template <int n>
__device__ __forceinline__ void loads_left()
{
    asm volatile("" ::: "memory");
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | (n >> 4) << 14);
#endif
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// Four reads of eight bytes a lane out of LDS, of which 16 lanes each take a tile turned: `b8` eight rows of 16 bytes' columns, else four rows of
// 16 two-byte columns.  They wait for themselves only: the compiler's would wait for every load to LDS under way.
template <bool b8, int apart>
__device__ __forceinline__ void columns(u32x2 (&r)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (b8)
        asm volatile("ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]) : "v"(a0), "v"(a1), "v"(a2), "v"(a3) : "memory");
    else
        asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:%6\n\tds_read_b64_tr_b16 %2, %5\n\tds_read_b64_tr_b16 %3, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]) : "v"(a0), "v"(a2), "n"(apart) : "memory");
#endif
}
__device__ __forceinline__ uint32_t lds_at(const void* p)
{
    typedef __attribute__((address_space(3))) const void lds_t;
    return (uint32_t)(uintptr_t)(lds_t*)p;
}
__device__ __forceinline__ void load_to_lds(const void* from, uint8_t* to, bool dword)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) void lds_t;
    typedef __attribute__((address_space(1))) const void mem_t;
    if (dword) __builtin_amdgcn_global_load_lds((mem_t*)from, (lds_t*)to, 4, 0, 0);
    else __builtin_amdgcn_global_load_lds((mem_t*)from, (lds_t*)to, 16, 0, 0);
#endif
}

// T: queries and results; P: the pages.  FULL: heads are DT and values whole DVT wide.  DIRECT: half a unit lies on one page, too (16 requests over
// 16384 positions, 8 bits 64 us, through registers 72; 64 over 400, 16 bits 27.1, 28.8).  A lane has one of 16 rows; PAIR, up to 8 rows: lanes
// c < 8 have the first map's, the others the second's, so that softmax and the products with the values are done once for both (64 us, as 16 rows
// 77; 27.1, 30.2).  More than 16 rows read the cache once for every 16 (two tiles of rows a wavefront: 32 rows, 8 requests over 8192, 16 bits
// 42 -> 57 us, two requests 27 -> 34).
template <typename T, typename P, bool FULL, bool DIRECT, int DT, int DVT, bool PAIR>
__global__ __launch_bounds__(64, (DIRECT && sizeof(T) == 2 && DT <= 64 ? 2 : 1)) void paged_attn(PagedArgs a)
{
    typedef typename Kept<P>::type KT;
    typedef Tile<KT, BN, DVT> Values;
    typedef Unit<P, DT, DVT> U;
    static_assert(!DIRECT || (FULL && sizeof(P) <= 2), "whole rows of whole pages");
    constexpr int M = PAIR ? 1 : 2;                              // maps of a lane
    constexpr int KS = DT / 32, NT = DVT / 16, E = 16 / sizeof(P), SC = sizeof(P) == 1;
    constexpr int NV = BN * DVT / E / 64, VPER = DVT / E;        // 16-byte vectors of a lane's and a row's share of the values
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int l = threadIdx.x, c = l & 15, h = l >> 4, own_m = PAIR ? c >> 3 : 0, own_c = PAIR ? c & 7 : c;
    const int per_head = a.parts ? a.parts : a.B;
    const int at = blockIdx.x % per_head, rest = blockIdx.x / per_head, hk = rest % a.Hkv, first = rest / a.Hkv * 16;
    const int dv0 = blockIdx.z * DVT, dvn = min(DVT, a.Dv - dv0);

    int b, begin, end, n;                                        // the request, the stretch in units from its first, the request's positions
    if (a.parts) {
        if (!find_stretch(a, at, b, begin, end, n)) return;
    } else {
        b = at;
        begin = 0;
        n = __builtin_amdgcn_readfirstlane(positions(a, b));
        end = units_of(n);
    }

    const P* kb = (const P*)a.k + (int64_t)hk * 2 * a.k_h;
    const P* vb = (const P*)a.v + (int64_t)hk * a.v_h + dv0;
    const uint8_t* kxb = a.kx + (int64_t)hk * 2 * a.kx_h;
    const uint8_t* vxb = a.vx + (int64_t)hk * a.vx_h;
    const int32_t* table = a.table + b * a.table_b;              // DIRECT: of the request whose units are asked for
    // Where a unit's keys are, in three steps of an iteration each: its pages are asked for, found, read from.  DIRECT: the pages of its two
    // halves, for the whole wavefront, and rows lie at 32-bit offsets from the halves' first; otherwise the page of key l % 32.
    typedef __attribute__((address_space(4))) const int32_t scalar_t;
    int entry[2] = {};
    int page = 0, slot = 0;
    uint32_t there_next = 0;                                 // keys of the unit that are there, as bits
    // (DIRECT: units are asked for in turn, from one request to the next.  Of the half that is next: its place in the table, its first slot, the
    // keys from it on; of its request: its units that have not been asked for)
    int asked_b = b, units_left = units_of(n) - begin, next_at = 0, next_slot = 0, next_left = n - begin * BN, asked_slot[2], asked_left[2];
    if constexpr (DIRECT) {
        next_at = (int)divided((uint32_t)(begin * BN), a.page);
        next_slot = begin * BN - next_at * (int)a.page.d;
    }
    const auto ask = [&](int u) {
        if constexpr (DIRECT) {
            if (__builtin_expect(units_left == 0, 0)) {
                const ArgsAgain z = again();
                do {
                    if (++asked_b >= z->B) break;        // (not reached: there are units to ask for)
                    next_left = min(max(((scalar_t*)z->len)[asked_b], 0), z->capacity);
                    units_left = units_of(next_left);
                } while (units_left == 0);
                table = z->table + asked_b * z->table_b;
                next_at = next_slot = 0;
            }
            --units_left;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                entry[y] = ((scalar_t*)table)[min(next_at, a.width - 1)];        // (no kernel writes it while this one runs)
                asked_slot[y] = next_slot;
                asked_left[y] = next_left;
                next_left -= 16;
                next_slot += 16;
                if (next_slot == (int)a.page.d) { next_slot = 0; ++next_at; }
            }
        } else {
            entry[0] = table[min((int)divided((uint32_t)(u * BN + (l & 31)), a.page), a.width - 1)];
        }
    };
    uint32_t page_of[2], slot_of[2];                             // DIRECT: the halves' pages and first slots
    const auto find = [&](int u) {
        if constexpr (DIRECT) {
            there_next = 0;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const bool ok = asked_left[y] > 0 && (uint32_t)entry[y] < (uint32_t)a.pages;
                page_of[y] = ok ? entry[y] : 0;
                slot_of[y] = ok ? asked_slot[y] : 0;
                const uint32_t keys = asked_left[y] >= 16 ? 0xffffu : (1u << asked_left[y]) - 1u;
                if (ok) there_next |= keys << (16 * y);
            }
        } else {
            const int j = u * BN + (l & 31), p = entry[0];
            const bool ok = j < n && p >= 0 && p < a.pages;
            page = ok ? p : 0;
            slot = ok ? j - (int)(divided((uint32_t)j, a.page) * a.page.d) : 0;
            there_next = (uint32_t)__ballot(ok);
        }
    };
    // straight to LDS: a load is 1024 bytes in a row; each lane chooses the chunk of memory that belongs where its 16 bytes come to lie
    uint32_t k_off[DIRECT ? U::HK : 1], v_off[DIRECT ? 2 : 1][DIRECT ? U::HV : 1];
    float* scales = (float*)(lds + U::STAGES * U::SIZE);     // [2 maps, values][BN]
    uint32_t there_of[2] = {}, low_k[2] = {}, low_v[2] = {};   // of this unit and the next: what is there, the low bits of its scales' addresses
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < U::HK; ++i) {
            const int key = (i * 64 + l) / U::CK, chunk = (l % U::CK) ^ U::turn_k(key), m = chunk / (U::CK / 2);
            k_off[i] = (uint32_t)(key * a.k_s + m * a.k_h) * U::ES + chunk % (U::CK / 2) * 16;
        }
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < U::HV; ++i) {
                const int key = (i * 64 + l) / U::CV, chunk = (l % U::CV) ^ U::turn_v(16 * y + key);
                v_off[y][i] = (uint32_t)(key * a.v_s) * U::ES + chunk * 16;
            }
    }
    // (a scale's dword: the four aligned bytes that its byte is one of)
    const uint32_t kx_lane = (uint32_t)(c * a.kx_s) + (l >= 32 ? (uint32_t)a.kx_h : 0u), vx_lane = (uint32_t)(c * a.vx_s);
    const auto scale_load = [&](const uint8_t* half0, const uint8_t* half1, uint32_t lane, uint8_t* to, uint32_t& low) {
        const uint64_t at = (uint64_t)(l & 16 ? half1 : half0) + lane;
        low = (uint32_t)at & 3;
        load_to_lds((const void*)(at - low), to, true);
    };
    const auto half = [&](int y, int64_t page_stride, int64_t slot_stride, int size) {
        return (uint64_t)page_of[y] * (uint32_t)(page_stride * size) + (uint64_t)slot_of[y] * (uint32_t)(slot_stride * size);
    };
    const auto send_keys = [&](int stage, uint32_t& low) {
        uint8_t* to = (uint8_t*)lds + stage * U::SIZE;
        if constexpr (SC) scale_load(kxb + half(0, a.kx_p, a.kx_s, 1), kxb + half(1, a.kx_p, a.kx_s, 1), kx_lane, to + U::K + U::V, low);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const char* from = (const char*)kb + half(y, a.k_p, a.k_s, sizeof(P));
#pragma unroll
            for (int i = 0; i < U::HK; ++i) load_to_lds(from + k_off[i], to + (y * U::HK + i) * 1024, false);
        }
    };
    const auto send_values = [&](int stage, uint32_t& low) {
        uint8_t* to = (uint8_t*)lds + stage * U::SIZE + U::K;
        if constexpr (SC) scale_load(vxb + half(0, a.vx_p, a.vx_s, 1), vxb + half(1, a.vx_p, a.vx_s, 1), vx_lane, to + U::V + U::SCALES, low);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const char* from = (const char*)vb + half(y, a.v_p, a.v_s, sizeof(P));
#pragma unroll
            for (int i = 0; i < U::HV; ++i) load_to_lds(from + v_off[y][i], to + (y * U::HV + i) * 1024, false);
        }
    };

    int left = end - begin, stage = 0;                           // DIRECT: the stretch's units that are not multiplied yet; where this one's are
    bool first_request = true;
    // a lane's rows: the same in every request.  DIRECT: a request's queries are read a request ahead.
    const int row0 = min(first + own_c, a.rows - 1), token = row0 / a.G, head0 = hk * a.G + row0 % a.G;
    const float lam = a.lam[head0];
    const T* q_row = (const T*)a.q + token * a.q_s + ((int64_t)head0 * 2 + own_m) * a.q_h;
    typename Frag<T>::type next_q[M][KS];
    const auto read_q = [&](int r) {
        const ArgsAgain z = again();
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int s = 0; s < KS; ++s) next_q[m][s] = global_frag<false>(q_row + r * z->q_b + m * z->q_h, depth_of<P, KS>(s, h), z->D);
    };
    if (DIRECT) read_q(b);
    for (int next_n;; ++b, n = __builtin_amdgcn_readfirstlane(next_n)) {
        const int units = units_of(n);
        const ArgsAgain z = again();
        next_n = b + 1 < z->B ? min(max(((scalar_t*)z->len)[b + 1], 0), z->capacity) : 0;
        if (z->parts && units == 0) {
            if (b + 1 >= z->B) return;                           // (not reached: the stretch goes on)
            if (DIRECT) read_q(b + 1);
            continue;
        }
        const int u1 = min(end, units);
        if (!DIRECT) read_q(b);
        typename Frag<T>::type qf[M][KS];
        const int lim = limit_of(z->causal, z->Sq, token, n);
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[m][s] = next_q[m][s];
        const int least = __builtin_amdgcn_readfirstlane(lim);    // of the first row: limits rise

        f32x4 o[M][NT];
        float top[M], safe[M], sum[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            top[m] = -INFINITY; safe[m] = 0.0f; sum[m] = 0.0f;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[m][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        f32x4 s[M][2];                                           // [map][16 keys]
        Weights<T> p[M];
        // scores of the keys that are not there, or not seen, go; then the weights, times their values' scales
        const auto soften = [&](int j0, uint32_t there, const float (&by)[8]) {
            if (__builtin_expect(j0 > least - BN || there != ~0u, 0)) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = 16 * y + 4 * h + e;
                        const bool ok = j0 + j < lim && (there >> j & 1);
#pragma unroll
                        for (int m = 0; m < M; ++m) s[m][y][e] = ok ? s[m][y][e] : -INFINITY;
                    }
            }
#pragma unroll
            for (int m = 0; m < M; ++m) {
                f32x4 (&z)[2] = s[m];
                float mx = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
                mx = half_max(quarter_max(mx)) * a.scale2;
                if (__builtin_expect(__any(mx > top[m] + 8.0f), 0)) {
                    const float grown = fmaxf(top[m], mx);
                    safe[m] = grown == -INFINITY ? 0.0f : grown;
                    const float f = __builtin_amdgcn_exp2f(top[m] - safe[m]);
                    top[m] = grown;
                    sum[m] *= f;
#pragma unroll
                    for (int t = 0; t < NT; ++t) o[m][t] *= f;
                }
                float v[8];
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float w = __builtin_amdgcn_exp2f(fmaf(z[y][e], a.scale2, -safe[m]));
                        sum[m] += w;
                        v[4 * y + e] = DIRECT && SC ? w * by[4 * y + e] : w;
                    }
                p[m].set(v);
            }
        };
        int u = begin;
        if constexpr (DIRECT) {
            // the first two units' loads; those of later requests go out under the products of the ones before
            if (first_request && left > 0) {
                ask(u);
                find(u);
                if (left > 1) ask(u + 1);
                there_of[0] = there_next;
                send_keys(0, low_k[0]);
                send_values(0, low_v[0]);
                if (left > 1) {
                    find(u + 1);
                    if (left > 2) ask(u + 2);
                    there_of[1] = there_next;
                    send_keys(1, low_k[1]);
                    send_values(1, low_v[1]);
                }
            }
            first_request = false;
            if (z->parts && end > units && b + 1 < z->B) read_q(b + 1);
            for (; u < u1; ++u, --left, stage ^= 1) {
                const int j0 = u * BN;
                const uint32_t there = there_of[0];
                uint8_t* kt = (uint8_t*)lds + stage * U::SIZE;
                uint8_t* vt = kt + U::K;
                // younger than this unit's keys: its values, the next unit
                if (left > 1) loads_left<U::VLOADS + U::KLOADS + U::VLOADS>();
                else loads_left<U::VLOADS>();
                float fk[2][2] = {};
                if constexpr (SC) {
                    // (lane l: map l / 32 of key l % 32)
                    const uint32_t d = *(const uint32_t*)(vt + U::V + 4 * l), low = low_k[0];
                    scales[l] = scale_of((int)(d >> (8 * low) & 255));
                    wave_lds_fence();
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int m = 0; m < 2; ++m) fk[y][m] = scales[32 * m + 16 * y + c];
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
                        const uint8_t* row = kt + (16 * y + c) * U::RK;
#pragma unroll
                        for (int t = 0; t < KS; ++t) {
                            bf16x8 kf;
                            if constexpr (!SC) {
                                kf = *(const bf16x8*)(row + ((m * (U::CK / 2) + 4 * t + h) ^ U::turn_k(c)) * 16);
                            } else if constexpr (KS == 1) {
                                const u32x2 x = *(const u32x2*)(row + ((m * (U::CK / 2) + (h >> 1)) ^ U::turn_k(c)) * 16 + 8 * (h & 1));
                                kf = widened(x[0], x[1], fk[y][m]);
                            } else {
                                // (16 bytes are two steps: depth_of)
                                const u32x4 x = *(const u32x4*)(row + ((m * (U::CK / 2) + 4 * (t / 2) + h) ^ U::turn_k(c)) * 16);
                                kf = widened(x[2 * (t % 2)], x[2 * (t % 2) + 1], fk[y][m]);
                            }
                            z = mma(z, kf, qf[PAIR ? 0 : m][t]);
                        }
                        // (both maps' keys meet every lane's query: a lane keeps its own map's)
                        f32x4& to = s[PAIR ? 0 : m][y];
                        if (PAIR && m == 1) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) to[e] = own_m ? z[e] : to[e];
                        } else {
                            to = z;
                        }
                    }
                const bool more = left > 2;
                uint32_t low_k_then = 0, low_v_then = 0;
                if (more) {
                    find(u + 2);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (of the products' reads)
                    send_keys(stage, low_k_then);
                    if (left > 3) ask(u + 3);
                    __builtin_amdgcn_sched_barrier(0);
                }
                // younger than this unit's values: the next unit, the keys of the one after it
                if (more) loads_left<U::KLOADS + U::VLOADS + U::KLOADS>();
                else if (left > 1) loads_left<U::KLOADS + U::VLOADS>();
                else loads_left<0>();
                float fv[8] = {}, apart = 1.0f;
                if constexpr (SC) {
                    const uint32_t d = *(const uint32_t*)(vt + U::V + U::SCALES + 4 * l), low = low_v[0];
                    // (what is not there counts as 1: nothing of it may reach a sum)
                    const bool has = there >> (l & 31) & 1;
                    const int byte = (int)(d >> (8 * low) & 255);
                    // (the weights take the scales: 2^32 goes between them and the values, so that neither leaves the range of 32 bits)
                    const bool far = __any(has && byte > 200);
                    apart = far ? 0x1p32f : 0x1p-32f;
                    if (l < 32) scales[64 + l] = has ? scale_of(byte) * (far ? 0x1p-32f : 0x1p32f) : 1.0f;
                    wave_lds_fence();
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const f32x4 g = *(const f32x4*)(scales + 64 + 16 * y + 4 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) fv[4 * y + e] = g[e];
                    }
                }
                if (__builtin_expect(there != ~0u, 0)) {
                    for (int e = l; e < BN * U::CV; e += 64)
                        if (!(there >> (e / U::CV) & 1)) *(u32x4*)(vt + e * 16) = u32x4{0, 0, 0, 0};
                    wave_lds_fence();
                }
                soften(j0, there, fv);
                // 8 bits: 16 lanes take eight keys of 16 columns, lane i the columns' half i % 2 of key i / 2 of {4 h .., 16 + 4 h ..}; 16 bits:
                // four keys, lane i four columns of key i / 4 of {4 h ..}, then of {16 + 4 h ..}.  (a row's chunks differ in its low bits only)
                const int r = SC ? (c >> 1 & 3) + 4 * h + (c >> 3) * 16 : 4 * h + (c >> 2);
                const uint32_t v0 = lds_at(vt) + r * U::RV + (SC ? U::turn_v(r) * 16 + 8 * (c & 1) : (U::turn_v(r) ^ (c >> 1 & 1)) * 16 + 8 * (c & 1));
                static_assert(U::SIZE % U::RV == 0 && U::K % U::RV == 0, "rows at whole rows' places");
#pragma unroll
                for (int t0 = 0; t0 < NT; t0 += SC ? 4 : 2) {
                    u32x2 x[4];
                    if constexpr (SC) columns<true, 0>(x, v0 ^ 16 * t0, v0 ^ 16 * (t0 + 1), v0 ^ 16 * (t0 + 2), v0 ^ 16 * (t0 + 3));
                    else columns<false, 16 * U::RV>(x, v0 ^ 32 * t0, 0, v0 ^ 32 * (t0 + 1), 0);
#pragma unroll
                    for (int t = t0; t < t0 + (SC ? 4 : 2); ++t) {
                        bf16x8 vf;
                        if constexpr (SC) {
                            vf = widened(x[t - t0][0], x[t - t0][1], apart);
                        } else {
                            union { u32x2 u[2]; bf16x8 v; } y = {{x[2 * (t - t0)], x[2 * (t - t0) + 1]}};
                            vf = y.v;
                        }
#pragma unroll
                        for (int m = 0; m < M; ++m) o[m][t] = p[m].times(o[m][t], vf);
                    }
                }
                if (more) {
                    send_values(stage, low_v_then);
                    __builtin_amdgcn_sched_barrier(0);
                }
                there_of[0] = there_of[1]; low_k[0] = low_k[1]; low_v[0] = low_v[1];
                there_of[1] = there_next; low_k[1] = low_k_then; low_v[1] = low_v_then;
                settle();
            }
        } else {
            RawKey<P, KS> kr[2][2];                                  // [16 keys][map]
            uint8_t ke[2][2] = {}, ve[NV] = {};
            u32x4 vr[NV];
            const auto fetch_keys = [&]() {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int64_t p = __shfl(page, 16 * y + c), s = __shfl(slot, 16 * y + c);
                    const P* row = kb + (p * a.k_p + s * a.k_s);
                    const uint8_t* x = SC ? kxb + (p * a.kx_p + s * a.kx_s) : nullptr;
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        load_key<FULL>(kr[y][m], row + m * a.k_h, h, a.D);
                        if constexpr (SC) ke[y][m] = x[m * a.kx_h];
                    }
                }
            };
            const auto fetch_values = [&]() {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int key = v * (64 / VPER) + l / VPER, d = l % VPER * E;
                    const int64_t p = __shfl(page, key), s = __shfl(slot, key);
                    const P* row = vb + (p * a.v_p + s * a.v_s);
                    if constexpr (SC) {
                        vr[v] = load16_any<FULL>((const uint8_t*)row, d, dvn);
                        ve[v] = vxb[p * a.vx_p + s * a.vx_s];
                    } else {
                        vr[v] = load16_any<FULL>(row, d, dvn);
                    }
                }
            };
            bf16* vt = (bf16*)lds;
            const float none[8] = {};
            table = a.table + b * a.table_b;
            if (u < u1) {
                ask(u);
                find(u);
                if (u + 1 < u1) ask(u + 1);
                fetch_keys();
                fetch_values();
            }
            for (; u < u1; ++u) {
                const bool more = u + 1 < u1;
                const uint32_t there = there_next;
                if (more) find(u + 1);
                if (u + 2 < u1) ask(u + 2);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int t = 0; t < KS; ++t) {
                            const auto kf = key_frag<FULL>(kr[y][m], t, h, a.D, scale_of(ke[y][m]));
                            z = mma(z, kf, qf[PAIR ? 0 : m][t]);
                        }
                        // (both maps' keys meet every lane's query: a lane keeps its own map's)
                        f32x4& to = s[PAIR ? 0 : m][y];
                        if (PAIR && m == 1) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) to[e] = own_m ? z[e] : to[e];
                        } else {
                            to = z;
                        }
                    }
                if (more) fetch_keys();
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int e = v * 64 + l, row = e / VPER, d = e % VPER * E;
                    const bool ok = d < dvn && (there >> row & 1);
                    bf16* to = vt + row * Values::LD + d;
                    if constexpr (SC) {
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
                soften(u * BN, there, none);
                const int vcol = few_col_lane<Values::LD>();
                wave_lds_fence();
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const auto vf = tile_col<KT, Values::LD, Values::PLANE, 16>(vt + vcol + 16 * t);
#pragma unroll
                    for (int m = 0; m < M; ++m) o[m][t] = p[m].times(o[m][t], vf);
                }
                wave_lds_fence();
                settle();
            }
        }
        const ArgsAgain f = again();
        const int wide = (f->Dv + 3) / 4 * 4;
        const bool whole = begin == 0 && u1 == units;
        const int mine = first + own_c;
#pragma unroll
        for (int m = 0; m < M; ++m) sum[m] = half_sum(quarter_sum(sum[m]));
        if (whole) {
            T* out = (T*)f->out + (((int64_t)b * f->Sq + token) * f->H + head0) * f->Dv + dv0;
            // (a query that sees nothing answers 0, whatever lam is)
            const float s0 = sum[0], s1 = PAIR ? __shfl_xor(s0, 8) : sum[M - 1];
            const bool none = own_m == 0 ? s1 == 0.0f : s0 == 0.0f;
            const float by0 = own_m ? lam / s0 : 1.0f / s0, by1 = PAIR ? 0.0f : lam / s1;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float r[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float other = PAIR ? __shfl_xor(o[0][t][e] * by0, 8) : o[M - 1][t][e] * by1;
                    r[e] = none ? 0.0f : fmaf(o[0][t][e], by0, -other);
                }
                if (own_m == 0 && mine < f->rows) store4(out, 16 * t + 4 * h, dvn, f->ovec, r);
            }
        } else if (mine < f->rows) {
            const int64_t row = (((int64_t)hk * f->parts + at) * 2 + (begin == 0 ? 1 : 0)) * f->rows + mine;
#pragma unroll
            for (int m = 0; m < M; ++m) {
                if (blockIdx.z == 0 && h == 0) *(f32x2*)(f->part_ml + 4 * row + 2 * (m + own_m)) = f32x2{top[m], sum[m]};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int d = 16 * t + 4 * h;
                    if (dv0 + d < wide) *(f32x4*)(f->part + (row * 2 + m + own_m) * wide + dv0 + d) = o[m][t];
                }
            }
        }
        if (!f->parts || end <= units || b + 1 >= f->B) return;
        // the next request, from its first unit on
        end -= units;
        begin = 0;
    }
}

// Joins a row's parts: a workgroup a row of (request, query, head); lanes along both maps' values, four at a time, groups of lanes along the parts.
template <typename T>
__global__ __launch_bounds__(256) void paged_join(PagedArgs a)
{
    __shared__ float f[2][MAX_PARTS], total[2];
    __shared__ f32x4 meet[256];
    __shared__ int counts[4][3];
    const int64_t id = blockIdx.x;
    const int head = (int)(id % a.H), i = (int)(id / a.H % a.Sq), b = (int)(id / a.H / a.Sq);
    const int hk = head / a.G, r = i * a.G + head % a.G, quads = (a.Dv + 3) / 4;
    T* out = (T*)a.out + id * a.Dv;
    // (the lanes share the requests out: 4096 of up to 512 positions, 16 heads, 16 bits 608 us the call, each wavefront for itself 886)
    int all = 0, before = 0, units = 0;
    for (int r = threadIdx.x; r < a.B; r += 256) {
        const int n = units_of(positions(a, r));
        all += n;
        before += r < b ? n : 0;
        units += r == b ? n : 0;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) { all += __shfl_xor(all, d); before += __shfl_xor(before, d); units += __shfl_xor(units, d); }
    if ((threadIdx.x & 63) == 0) {
        int* to = counts[threadIdx.x >> 6];
        to[0] = all; to[1] = before; to[2] = units;
    }
    __syncthreads();
    all = counts[0][0] + counts[1][0] + counts[2][0] + counts[3][0];
    before = counts[0][1] + counts[1][1] + counts[2][1] + counts[3][1];
    units = counts[0][2] + counts[1][2] + counts[2][2] + counts[3][2];
    if (units == 0) {
        for (int d = threadIdx.x; d < a.Dv; d += 256) out[d] = (T)0.0f;
        return;
    }
    const int per = stretch_of(a, all), p0 = min(before / per, a.parts - 1), p1 = min((before + units - 1) / per, a.parts - 1), count = p1 - p0 + 1;
    if (count == 1) return;                              // (answered where it was computed)
    // the first part is its wavefront's last request, the others are their wavefronts' first
    const int64_t row0 = ((int64_t)hk * a.parts + p0) * 2 * a.rows + r;
    const auto row_of = [&](int p) { return row0 + (int64_t)(2 * p + (p == 0 ? 1 : 0)) * a.rows; };
    // 2 * quads lanes a group (at most 128), as many groups as there are lanes for; a group's first parts are asked for at once
    constexpr int AHEAD = 4;
    const int wide = 2 * quads, groups = 256 / wide, group = threadIdx.x / wide, q = threadIdx.x - group * wide, m = q >= quads;
    f32x4 part[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) part[i] = *(const f32x4*)(a.part + (row_of(min(group + i * groups, count - 1)) * wide + q) * 4);
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
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    // (a part whose keys were all hidden adds nothing)
    const auto add = [&](int p, const f32x4& x) {
        const float g = f[m][p];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += g == 0.0f ? 0.0f : g * x[e];
    };
    if (group < groups) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) if (group + i * groups < count) add(group + i * groups, part[i]);
#pragma unroll 4
        for (int p = group + AHEAD * groups; p < count; p += groups) add(p, *(const f32x4*)(a.part + (row_of(p) * wide + q) * 4));
    }
    meet[threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.x >= quads) return;
    f32x4 x = meet[threadIdx.x], y = meet[quads + threadIdx.x];
    for (int g = 1; g < groups; ++g) { x += meet[g * wide + threadIdx.x]; y += meet[g * wide + quads + threadIdx.x]; }
    const bool none = total[1] == 0.0f;
    const float i0 = none ? 0.0f : 1.0f / total[0], i1 = none ? 0.0f : a.lam[head] / total[1];
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = none ? 0.0f : fmaf(x[e], i0, -y[e] * i1);
    store4(out, 4 * (int)threadIdx.x, a.Dv, a.ovec, o);
}

int dim_tile(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

struct PagedPlan { bool full, direct, pair; int row_tiles, chunks, parts; size_t part, ml; };

// What a call's operands allow (addresses apart from their low bits do not count: the workspace's size does not know them).
PagedPlan paged_plan(const sconv_paged_desc_t& d, const sconv_pages_dev_t* at, size_t ws_bytes)
{
    PagedPlan p = {};
    if (d.B == 0 || d.Sq == 0) return p;
    const sconv_pages_t& g = d.pages;
    const int G = d.H / d.Hkv, rows = d.Sq * G, DT = dim_tile(g.D), DVT = DT == 32 ? 64 : 128;
    p.pair = rows <= 8;
    p.row_tiles = (rows + 15) / 16;
    p.chunks = (g.Dv + DVT - 1) / DVT;
    // (16 rows of both maps within 32-bit offsets, strides of 32 bits)
    const int64_t far = int64_t(1) << 24;
    p.full = g.D == DT && g.Dv % DVT == 0;
    const bool aligned = g.page_size % 16 == 0 && std::max({g.k_s, g.v_s, g.ks_s, g.vs_s}) < far && std::max(g.k_h, g.ks_h) < 8 * far && std::max({g.k_p, g.v_p, g.ks_p, g.vs_p}) < 128 * far;
    const int size = serving_type_size(g.type);
    p.direct = p.full && aligned && size <= 2 && (g.k_p | g.k_s | g.k_h | g.v_p | g.v_s | g.v_h) % (16 / size) == 0;
    if (size == 1) {
        // a scale is read with the aligned dword around it: the last byte has to be the last of one
        const int64_t last_k = (g.pages - 1) * g.ks_p + (g.page_size - 1) * g.ks_s + (g.Hk - 1) * g.ks_h, last_v = (g.pages - 1) * g.vs_p + (g.page_size - 1) * g.vs_s + (g.Hv - 1) * g.vs_h;
        p.direct = p.direct && last_k % 4 == 3 && last_v % 4 == 3;
    }
    if (at) p.direct = p.direct && aligned_to(at->k, 16) && aligned_to(at->v, 16) && aligned_to(at->ks, 4) && aligned_to(at->vs, 4);
    // As many stretches as there are places for wavefronts (16-bit heads of more than 64 fill LDS with three: 16 requests over 16384, heads of 128
    // (256), 276 -> 190 us), no more than the caches can have units, or 64 MB hold parts.
    const int64_t units = (int64_t)d.B * (((int64_t)g.table_width * g.page_size + BN - 1) / BN), base = (int64_t)d.Hkv * p.row_tiles * p.chunks;
    if (units >= (int64_t(1) << 31)) return p;
    // Short caches, and more of them the more requests fill the chip: a wavefront a request, without parts or a second kernel (equal lengths, split
    // and so: one request of 128 positions 14 and 10 us, 64 with 8 heads 13.9 and 9.8, of 512 29 and 25; 512 with 8 heads, 8 bits, of 1024 253 and 215,
    // one of 1024 among others a quarter of it at most 80 and 75, 128 such 29 and 46).
    if ((int64_t)g.table_width * g.page_size <= 256 * std::max<int64_t>(1, d.B * base / PLACES)) return p;
    const int64_t places = DT == 128 && g.type == SCONV_BF16 ? PLACES * 3 / 4 : PLACES;
    const int64_t wide = (g.Dv + 3) / 4 * 4, each = (int64_t)d.Hkv * 2 * rows * (2 * wide + 4) * (int64_t)sizeof(float);
    int64_t parts = std::max<int64_t>(std::min<int64_t>(places / base, (int64_t(64) << 20) / each), 1);
    parts = std::min<int64_t>(std::min<int64_t>(parts, units), MAX_PARTS);
    // (one stretch: every request is a wavefront's, as without scratch)
    if (parts == 1 || (size_t)(parts * each) > ws_bytes) return p;
    p.parts = (int)parts;
    p.part = (size_t)(parts * d.Hkv * 2 * rows * 2 * wide) * sizeof(float);
    p.ml = (size_t)(parts * d.Hkv * 2 * rows * 4) * sizeof(float);
    return p;
}

template <typename T, typename P, bool FULL, bool DIRECT, int DT, int DVT, bool PAIR>
int paged_launch(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    size_t lds = (size_t)Tile<typename Kept<P>::type, BN, DVT>::SIZE * 2;
    if constexpr (DIRECT) lds = Unit<P, DT, DVT>::LDS;
    const auto kern = paged_attn<T, P, FULL, DIRECT, DT, DVT, PAIR>;
    const int rc = allow_lds(kern, lds);
    if (rc) return rc;
    const int64_t grid = (int64_t)(p.parts ? p.parts : a.B) * a.Hkv * p.row_tiles;
    if (!grid_fits(grid, 64) || !grid_fits((int64_t)a.B * a.Sq * a.H, 256)) return SCONV_EUNSUPPORTED;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid, 1, (unsigned)p.chunks), dim3(64), lds, stream, a);
    return launch_status();
}

template <typename T, typename P, bool FULL, bool DIRECT>
int paged_shape(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    const int DT = dim_tile(a.D);
    if (p.pair)
        return DT == 32 ? paged_launch<T, P, FULL, DIRECT, 32, 64, true>(a, p, stream)
             : DT == 64 ? paged_launch<T, P, FULL, DIRECT, 64, 128, true>(a, p, stream) : paged_launch<T, P, FULL, DIRECT, 128, 128, true>(a, p, stream);
    return DT == 32 ? paged_launch<T, P, FULL, DIRECT, 32, 64, false>(a, p, stream)
         : DT == 64 ? paged_launch<T, P, FULL, DIRECT, 64, 128, false>(a, p, stream) : paged_launch<T, P, FULL, DIRECT, 128, 128, false>(a, p, stream);
}

template <typename T, typename P>
int paged_run(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    int rc;
    if constexpr (sizeof(P) <= 2) rc = p.direct ? paged_shape<T, P, true, true>(a, p, stream) : p.full ? paged_shape<T, P, true, false>(a, p, stream) : paged_shape<T, P, false, false>(a, p, stream);
    else rc = p.full ? paged_shape<T, P, true, false>(a, p, stream) : paged_shape<T, P, false, false>(a, p, stream);
    if (rc || p.parts == 0) return rc;
    hipLaunchKernelGGL((paged_join<T>), dim3((unsigned)((int64_t)a.B * a.Sq * a.H)), dim3(256), 0, stream, a);
    return launch_status();
}

}  // namespace

size_t paged_workspace(const sconv_paged_desc_t& d)
{
    const PagedPlan p = paged_plan(d, nullptr, ~(size_t)0 >> 1);
    return p.part + p.ml;
}

int launch_paged(const sconv_paged_desc_t& d, const void* q, const sconv_pages_dev_t& pages, const float* lam, const int32_t* lengths,
                 void* out, void* ws, size_t ws_bytes, hipStream_t stream)
{
    const sconv_pages_t& g = d.pages;
    const PagedPlan p = paged_plan(d, &pages, ws_bytes);
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
