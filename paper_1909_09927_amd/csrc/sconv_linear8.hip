// Product of 8-bit operands with block scales (formula in sconv_serving.h).
//
// Few rows (up to 64, single tokens): bound by the weights' read, and by what every workgroup reads of the tokens.  A workgroup takes 16 or 32 weight
// rows, its eight wavefronts share out the blocks of 128, read operands from memory straight into the product's registers and meet in LDS.
// Many rows: tiles through LDS, bound by the matrix pipe, or by the results' write where the depth is small.
// Measured, 16-bit results, medians: 16 x 2048 to 8192 6.5 us (2.6 TB/s), 64 x 8192 to 8192 36; 12544 x 2048 to 8192 209 (2014 TFLOP/s; 201 cold, 221 to
// 278 where call follows call for milliseconds and the clock falls), 4096 x 8192 to 8192 220 (2495), 25088 x 512 to 2048 47 (1115), 6272 x 896 to 1000 14.9.
// A tile of 256 x 256 costs 4.3 us beside its depth, 13 us for 1000.  Depths of no whole 16 go through registers, in tiles of 128 x 128: 4096 x 1000 to
// 4096 53 us, x 1008 26; 4096 x 8200 to 8192 450.
// Up to 64 rows, in 32-bit results and with `exact` the 8-bit values become 16-bit ones, exactly, and products are exact to 32 bits.  Other 16-bit
// results take 8-bit products with the scales as operands, at nearly twice the rate (12544 x 2048 to 8192 209 us, with `exact` 341;
// 784 x 2048 to 2048 12.3 and 19.1).  The matrix pipe takes eight products at a time and cuts off what lies 2^-13 or more below the largest of
// them: of normal values 1.4e-5 of a result's norm at any depth, which rounding to 16 bits (1.7e-3) hides; where the largest products cancel it
// shows (two channels of 1000 times the rest with opposite signs, depth 256: 1.1e-2), so it is the caller's choice.
//
// Layout of the products: weights are A, tokens are B, so that a lane's results are neighbours of one token's row.  Which depths of a block a
// lane holds does not matter, as long as both operands have the same.
#include <algorithm>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

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

template <typename T>
__device__ __forceinline__ void store_row4(T* p, int have, bool vec, const float* v)
{
    if (vec && have >= 4) { store_vec<4>(p, v); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < have) p[i] = (T)v[i];
}

// Few rows: MT tiles of 16 tokens against NT tiles of 16 weight rows, NW wavefronts.  A lane has 32 bytes (l / 16) * 32.. of row l % 16 of both
// operands.  Products are 16-bit ones of the converted values, whatever the result's type: the memory is what they wait for (64 x 8192 to 8192
// 36.3 us, by 8-bit products 34.2; 64 x 2048 to 8192 11.0 and 10.1).
template <typename T, int MT, int NT, int NW>
__global__ __launch_bounds__(64 * NW) void linear_few(LinArgs a)
{
    __shared__ f32x4 part[NW][MT * NT][64];
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63, c = l & 15, h = l >> 4, n0 = blockIdx.x * 16 * NT;
    const uint8_t* wr[NT];
    const uint8_t* ws = a.ws + (int64_t)(n0 >> 7) * a.KB;          // (NT tiles lie within 128 rows)
    const uint8_t* xr[MT];
    const uint8_t* xs[MT];
    f32x4 sum[MT][NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) wr[n] = a.w + (int64_t)min(n0 + 16 * n + c, a.N - 1) * a.w_n + 32 * h;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = min(16 * t + c, a.M - 1);
        xr[t] = a.x + m * a.x_m + 32 * h;
        xs[t] = a.xs + (int64_t)m * a.KB;
#pragma unroll
        for (int n = 0; n < NT; ++n) sum[t][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    union Raw32 { i32x4 q[2]; i32x8 v; };
    Raw32 wv[NT], xv[MT];
    int we = 0, xe[MT] = {};
    const auto fetch = [&](int kb) {
        const int k = kb * 128, have = a.K - k - 32 * h;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            wv[n].q[0] = bytes16(wr[n] + k, have);
            wv[n].q[1] = bytes16(wr[n] + k + 16, have - 16);
        }
        we = ws[kb];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            xv[t].q[0] = bytes16(xr[t] + k, have);
            xv[t].q[1] = bytes16(xr[t] + k + 16, have - 16);
            xe[t] = xs[t][kb];
        }
    };
    if (w < a.KB) fetch(w);
    for (int kb = w; kb < a.KB; kb += NW) {
        const bool more = kb + NW < a.KB;
        bf16x8 wf[NT][4], xf[MT][4];
        int e[MT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int s = 0; s < 4; ++s) wf[n][s] = widened(wv[n].v[2 * s], wv[n].v[2 * s + 1]);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            e[t] = we + xe[t] - 254;
#pragma unroll
            for (int s = 0; s < 4; ++s) xf[t][s] = widened(xv[t].v[2 * s], xv[t].v[2 * s + 1]);
        }
        if (more) fetch(kb + NW);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < 4; ++s) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[n][s], xf[t][s], p, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[t][n][i] += __builtin_ldexpf(p[i], e[t]);
            }
        // (18 wait states are what the longest product needs: seen in another kernel, the compiler counts too few where a result's first
        // reader stands behind a loop's exit)
        asm volatile("s_nop 15\n\ts_nop 3");
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) part[w][t * NT + n][l] = sum[t][n];
    __syncthreads();
    for (int i = w; i < MT * NT; i += NW) {
        f32x4 v = part[0][i][l];
#pragma unroll
        for (int k = 1; k < NW; ++k) v += part[k][i][l];
        const int m = 16 * (i / NT) + c, n = n0 + 16 * (i % NT) + 4 * h;
        const float o[4] = {v[0], v[1], v[2], v[3]};
        if (m < a.M) store_row4((T*)a.y + m * a.y_m + n, a.N - n, a.vec, o);
    }
}

// Many rows.  WM x WN wavefronts, each 32 TM tokens by 32 TN weight rows, walk the depth in stages of 64, which pass through a ring of four
// buffers in LDS: beneath a stage's products three later ones' loads are under way and the next one's fragments go to registers, so that no
// product waits for memory.  (Two buffers of 128 wait for it at every block: 12544 x 2048 to 8192 317 us.)
// A row of a stage is four chunks of 16 bytes, which stand at chunk ^ turn(row), so that lanes that read one chunk of 16 consecutive rows meet
// different banks.  DIRECT: chunks go from memory to LDS without registers (rows at whole chunks); a chunk behind a row's end is asked
// for behind the buffer's and comes as zeros.  Results are turned in LDS, so that a token's are written in whole lines.
template <int WM, int WN, int TM, int TN>
struct RingShape {
    static constexpr int BM = WM * TM * 32, BN = WN * TN * 32, WAVES = WM * WN, THREADS = 64 * WAVES, STAGES = 4;
    static constexpr int ROWS = BN + BM, N = ROWS / 16 / WAVES;          // rows of a buffer (weights, then tokens), its loads by one wavefront
    static_assert(N * WAVES * 16 == ROWS && BN % (16 * WAVES) == 0, "whole loads of one operand each");
    static constexpr int OUT = 4096;                                     // of a wavefront's results on their way out, in the ring
    static constexpr int RING = STAGES * ROWS * 64, CHUNK = 120;         // blocks whose scales are in LDS: of the tokens, then of the weights
    static_assert(WAVES * OUT <= RING, "results go out through the ring");
    static constexpr size_t LDS = (size_t)RING + CHUNK * (BM + BN / 128) + WAVES;
};

// vmcnt(n) lgkmcnt(0): all loads but the n youngest have come, and all reads of LDS
template <int n>
__device__ __forceinline__ void loads_and_reads()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_waitcnt(0x0070 | (n & 15) | (n >> 4) << 14);
#endif
}
// A barrier that waits for none of this wavefront's loads (a fence would, for those to LDS).
__device__ __forceinline__ void bare_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a tile's scales may be.  PIPE: anything, 8-bit products take them as operands.  16-bit products: tokens take both operands' scales, 2^by.  Values
// are 2^-9 to 448, so with 2^-108 to 2^100 no token leaves the range of 16 bits, and no product or sum of products, a multiple of
// 2^(by - 18), that of normal numbers.  NEAR: scales of 2^-54 to 2^50, of which any two are such.  ZEROS: others too, but two that are beyond these
// ends belong to zeros (whose blocks have the smallest scale).  FAR: anything, a stage's sums take the scales.
// (4096 x 8192 to 8192, every other token zeros, 32-bit results: 388 us in ZEROS, which looks at the values, 365 where nobody does.  Looked for in
// every call: 411 us for ordinary scales, 400 this way.)
enum { PIPE, NEAR, ZEROS, FAR };

// The tile of which (m0, n0) is the first token and weight row.  false: nothing is written, its scales are others.
template <typename T, int SCALES, bool DIRECT, int WM, int WN, int TM, int TN>
__device__ __forceinline__ bool ring_tile(const LinArgs& a, uint8_t* lds, int m0, int n0)
{
    constexpr bool FAST = SCALES == PIPE;
    typedef RingShape<WM, WN, TM, TN> Shape;
    constexpr int N = Shape::N, WAVES = Shape::WAVES, NWL = Shape::BN / 16 / WAVES, STAGES = Shape::STAGES;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, c = l & 31, h = l >> 5;
    const int wm = w / WN, wn = w - wm * WN;

    // a load is 16 rows of four chunks; lane l writes chunk l % 4 of row l / 4
    const auto row_of = [&](int i) { return ((i < NWL ? i : i - NWL) * WAVES + w) * 16 + (l >> 2); };
    const int chunk = (l & 3) ^ (l >> 4);
    uint32_t off[DIRECT ? N : 1];
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < N; ++i) off[i] = (uint32_t)(row_of(i) * (i < NWL ? a.w_n : a.x_m) + 16 * chunk);
    }
    i32x4 held[DIRECT ? 1 : N];
    const auto slot = [&](int i, int buffer) {           // in bytes, of a load's first row
        return (buffer * Shape::ROWS + (i < NWL ? 0 : Shape::BN) + ((i < NWL ? i : i - NWL) * WAVES + w) * 16) * 64;
    };
    int f_buffer = 0, left = a.K;                        // of the stage to be loaded: its buffer, the depth from it on
    [[maybe_unused]] const uint32_t size_w = (uint32_t)((min(a.N - n0, Shape::BN) - 1) * a.w_n), size_x = (uint32_t)((min(a.M - m0, Shape::BM) - 1) * a.x_m);
    const uint8_t* from_w = a.w + n0 * a.w_n;
    const uint8_t* from_x = a.x + m0 * a.x_m;
    // (buffers end with the tile's last row's last byte: rows behind it, and a stage behind the depth, come as zeros)
    const auto load = [&](int i) __attribute__((always_inline)) {
        if constexpr (DIRECT) {
#if defined(__HIP_DEVICE_COMPILE__)
            typedef __attribute__((address_space(3))) void lds_t;
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(i < NWL ? from_w : from_x), 0, (i < NWL ? size_w : size_x) + max(left, 0), 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_t*)(lds + slot(i, f_buffer)), 16, 16 * chunk >= left ? 0x80000000u : off[i], 0, 0, 0);
#endif
        } else {
            const uint8_t* p = i < NWL ? from_w + min(row_of(i), a.N - 1 - n0) * a.w_n : from_x + min(row_of(i), a.M - 1 - m0) * a.x_m;
            held[i] = bytes16(p + 16 * chunk, left - 16 * chunk);
        }
    };
    const auto loaded = [&]() {
        f_buffer = (f_buffer + 1) % STAGES;
        left -= 64;
        from_w += 64;
        from_x += 64;
    };
    const auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < N; ++i) load(i);
        loaded();
    };
    const auto put = [&](int buffer) {
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < N; ++i) *(i32x4*)(lds + slot(i, buffer) + 16 * l) = held[i];
    };
    // The scales of a stretch of blocks, block after block, the tile's tokens beside each other: read from memory in the loop, a line for every
    // token and block, they cost more than the operands (4096 x 8192 to 8192 284 us, without them 219).
    uint8_t* x_scales = lds + Shape::RING;
    uint8_t* w_scales = x_scales + Shape::CHUNK * Shape::BM;
    // what a wavefront has to tell the others, behind a barrier
    uint8_t* told = w_scales + Shape::BN / 128 * Shape::CHUNK;
    const auto say = [&](bool yes) {
        if (l == 0) told[w] = yes;
    };
    const auto met = [&]() {
        int any = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) any |= told[i];
        return any != 0;
    };
    const auto stretch = [&](int kb0) {
        const int count = min(Shape::CHUNK, a.KB - kb0);
        [[maybe_unused]] bool odd = false;               // outside 2^-54 .. 2^50, of which any two make no sum that is far
        const auto look = [&](int byte) {
            if constexpr (SCALES == NEAR) odd = odd || (uint32_t)(byte - 73) > 177u - 73u;
        };
        for (int r = threadIdx.x; r < Shape::BM; r += Shape::THREADS) {
            const uint8_t* from = a.xs + (int64_t)min(m0 + r, a.M - 1) * a.KB + kb0;
            for (int k = 0; k < count; k += 16) {
                const i32x4 v = bytes16(from + k, count - k);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (k + i < count) {
                        const int byte = v[i >> 2] >> (8 * (i & 3)) & 255;
                        x_scales[(k + i) * Shape::BM + r] = (uint8_t)byte;
                        look(byte);
                    }
            }
        }
        for (int e = threadIdx.x; e < Shape::BN / 128 * count; e += Shape::THREADS) {
            const int n = e / count, k = e - n * count, byte = a.ws[(int64_t)min((n0 >> 7) + n, (a.N - 1) >> 7) * a.KB + kb0 + k];
            w_scales[n * Shape::CHUNK + k] = (uint8_t)byte;
            look(byte);
        }
        if constexpr (SCALES == NEAR) say(__any(odd));
    };
    int we = 0, xe[TM] = {}, we_next = 0, xe_next[TM] = {};
    const auto load_scales = [&](int k) {                // of block k of the stretch
        we_next = w_scales[wn * TN * 32 / 128 * Shape::CHUNK + k];
#pragma unroll
        for (int t = 0; t < TM; ++t) xe_next[t] = x_scales[k * Shape::BM + (wm * TM + t) * 32 + c];
    };
    const auto take_scales = [&]() {
        we = we_next;
#pragma unroll
        for (int t = 0; t < TM; ++t) xe[t] = xe_next[t];
    };
    f32x16 sum[TM][TN];
    // a lane's 32 bytes of a row: chunks 2 h and the next
    const uint8_t* mine[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) mine[i] = lds + c * 64 + 16 * ((2 * h + i) ^ (c >> 2 & 3));
    const auto frag = [&](int row) {
        union { i32x8 v; i32x4 q[2]; } r;
#pragma unroll
        for (int i = 0; i < 2; ++i) r.q[i] = *(const i32x4*)(mine[i] + row * 64);
        return r.v;
    };
    struct Frags { i32x8 w[TN], x[TM]; };
    static_assert(TM == TN && N % TM == 0, "loads, reads and products in TM equal steps");
    const auto read = [&](Frags& f, int buffer, int t) __attribute__((always_inline)) {
        const int first = buffer * Shape::ROWS;
        f.w[t] = frag(first + (wn * TN + t) * 32);
        f.x[t] = frag(first + Shape::BN + (wm * TM + t) * 32);
    };
    [[maybe_unused]] int far = 0;
    const auto multiply = [&](const Frags& f, int t) {
        if constexpr (FAST) {
#pragma unroll
            for (int n = 0; n < TN; ++n) sum[t][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.w[n], f.x[t], sum[t][n], 0, 0, 0, we, 0, xe[t]);
        } else if constexpr (SCALES == FAR) {
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                f32x16 p = {};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(f.w[n][2 * i], f.w[n][2 * i + 1]), widened(f.x[t][2 * i], f.x[t][2 * i + 1]), p, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[t][n][e] += __builtin_ldexpf(p[e], we + xe[t] - 254);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            int by = we + xe[t] - 254;
            if constexpr (SCALES == ZEROS) {
                const int said = by;
                uint32_t xb = 0, wb = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    xb |= (uint32_t)f.x[t][i];
#pragma unroll
                    for (int n = 0; n < TN; ++n) wb |= (uint32_t)f.w[n][i];
                }
                by = min(max(said, -108), 100);
                far |= (int)(__ballot(by != said && (xb & 0x7f7f7f7fu)) != 0) & (int)(__ballot((wb & 0x7f7f7f7fu) != 0) != 0);
            }
            const float e = __builtin_ldexpf(1.0f, by);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 xv = widened(f.x[t][2 * i], f.x[t][2 * i + 1], e);
#pragma unroll
                for (int n = 0; n < TN; ++n)
                    sum[t][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widened(f.w[n][2 * i], f.w[n][2 * i + 1]), xv, sum[t][n], 0, 0, 0);
            }
        }
    };
    // Where stage i is multiplied, stage i + 1 is read into registers and stage i + 4 asked for, into the buffer that stage i has left.  arrived: stage
    // i + 1's loads have come (others' behind the barrier); those of two stages are younger.
    int buffer = 0;                                      // of stage i
    const auto step = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto arrived = [&]() {
        step();
        if constexpr (DIRECT) {
            loads_and_reads<2 * N>();
            bare_barrier();
        } else {
            __syncthreads();
        }
        step();
    };
    // A stage's products; between them the next one's fragments are read and a later one's loads go out, a few at a time (all at once they hold
    // up the wavefront that issues them).  ahead: the block whose scales are read, or -1.
    const auto multiply_stage = [&](const Frags& now, Frags& next, int ahead) {
        if constexpr (!DIRECT) put((buffer + 2) % STAGES);
        const int following = (buffer + 1) % STAGES;
#pragma unroll
        for (int t = 0; t < TM; ++t) {
#pragma unroll
            for (int i = 0; i < N / TM; ++i) load(t * (N / TM) + i);
            read(next, following, t);
            if (t == TM - 1 && ahead >= 0) load_scales(ahead);
            multiply(now, t);
            if constexpr (FAST && DIRECT) {
#pragma unroll
                for (int n = 0; n < TN; ++n) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (n < TN / 2) __builtin_amdgcn_sched_group_barrier(0x010, 2 * N / TM / TN, 0);
                    else __builtin_amdgcn_sched_group_barrier(0x100, 8 / TN, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        loaded();
        buffer = following;
    };
    Frags even, odd;
    if (a.KB > 0) {
#pragma unroll
        for (int i = 0; i < (DIRECT ? 4 : 3); ++i) {
            fetch();
            if (!DIRECT && i < 2) put(i);
            step();
        }
    }
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[t][n][e] = 0.0f;
    for (int kb0 = 0; kb0 < a.KB; kb0 += Shape::CHUNK) {
        if (kb0) __syncthreads();
        stretch(kb0);
        if constexpr (DIRECT) loads_and_reads<2 * N>();       // (of the first stage, at the start)
        __syncthreads();
        if constexpr (SCALES == NEAR) {
            if (met()) {
                far = 1;
                break;
            }
        }
        load_scales(0);
        take_scales();
        if (kb0 == 0) {
#pragma unroll
            for (int t = 0; t < TM; ++t) read(even, 0, t);
        }
        const int count = min(Shape::CHUNK, a.KB - kb0);
        for (int k = 0; k < count; ++k) {
            arrived();
            multiply_stage(even, odd, min(k + 1, count - 1));
            arrived();
            multiply_stage(odd, even, -1);
            take_scales();
            // (18 wait states are what the longest product needs: seen in another kernel, the compiler counts too few where a result's first
            // reader stands behind a loop's exit)
            step();
            asm volatile("s_nop 15\n\ts_nop 3");
            step();
        }
    }
    // (stages behind the last have been asked for: none outlives its workgroup's LDS, or meets the results in it)
    step();
    if constexpr (DIRECT) loads_and_reads<0>();
    __syncthreads();
    step();
    if constexpr (SCALES == NEAR || SCALES == ZEROS) {
        say(far);
        __syncthreads();
        if (met()) {
            __syncthreads();
            return false;
        }
    }
    const int out_n = n0 + wn * TN * 32, out_m = m0 + wm * TM * 32;
    // 32 tokens by as many results as 4 KB hold, a row of 16-byte chunks turned by the token
    constexpr int WIDE = Shape::OUT / 32 / (int)sizeof(T) < TN * 32 ? Shape::OUT / 32 / (int)sizeof(T) : TN * 32, E = 16 / (int)sizeof(T), CH = WIDE / E;
    T* out = (T*)(lds + w * Shape::OUT);
    const bool whole = a.vec && a.y_m % E == 0;
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
        for (int n = 0; n < TN * 32; n += WIDE) {
#pragma unroll
            for (int q = 0; q < WIDE / 8; ++q) {
                const int at = 8 * q + 4 * h, e = 4 * (q & 3);
                const f32x16& s = sum[t][n / 32 + q / 4];
                const float o[4] = {s[e], s[e + 1], s[e + 2], s[e + 3]};
                store_vec<4>(out + c * WIDE + ((at / E) ^ (c & (CH - 1))) * E + at % E, o);
            }
            wave_lds_fence();
#pragma unroll
            for (int i = 0; i < 32 * CH / 64; ++i) {
                const int row = (i * 64 + l) / CH, at = (i * 64 + l) % CH, m = out_m + 32 * t + row, have = a.N - out_n - n - at * E;
                const i32x4 v = *(const i32x4*)(out + row * WIDE + (at ^ (row & (CH - 1))) * E);
                if (m >= a.M) continue;
                T* y = (T*)a.y + m * a.y_m + out_n + n + at * E;
                if (whole && have >= E) *(i32x4*)y = v;
                else {
                    union { i32x4 v; T e[E]; } r;
                    r.v = v;
#pragma unroll
                    for (int j = 0; j < E; ++j) if (j < have) y[j] = r.e[j];
                }
            }
            wave_lds_fence();
        }
    return true;
}

// rest: so many tiles, the last, come in quarters, of 32 TM / 2 tokens and 32 TN / 2 weight rows a wavefront; they go first, which also keeps the
// compute units from writing their results all at once (25088 x 512 to 2048 52 -> 48 us).
template <typename T, bool FAST, bool DIRECT, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN, TM * TN > 8 ? 1 : 2) void linear_ring(LinArgs a, int tiles_m, int tiles_n, int rest)
{
    typedef RingShape<WM, WN, TM, TN> Shape;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int whole = tiles_m * tiles_n - rest, id = (int)blockIdx.x - 4 * rest;
    // blocks go round the chiplets: each gets a stretch of tiles, in groups of eight tiles of tokens that share their weights
    const int each = whole / 8, more = whole % 8, chip = id % 8;
    const int lin = id >= 0 ? chip * each + min(chip, more) + id / 8 : whole + (int)blockIdx.x / 4;
    const int width = 8 * tiles_n, group = lin / width, in = lin - group * width, high = min(8, tiles_m - 8 * group), tn = in / high, tm = 8 * group + in - tn * high;
    const int m0 = tm * Shape::BM, n0 = tn * Shape::BN;
    constexpr int FIRST = FAST ? PIPE : NEAR;
    constexpr int SM = TM > 2 ? TM / 2 : TM, SN = TN > 2 ? TN / 2 : TN;      // FAR holds a stage's sums, too, for which larger tiles have no room
    const auto small = [&](int m, int n) __attribute__((always_inline)) {
        if (m >= a.M || n >= a.N || ring_tile<T, FIRST, DIRECT, WM, WN, SM, SN>(a, lds, m, n)) return;
        if constexpr (!FAST)
            if (!ring_tile<T, ZEROS, DIRECT, WM, WN, SM, SN>(a, lds, m, n)) ring_tile<T, FAR, DIRECT, WM, WN, SM, SN>(a, lds, m, n);
    };
    if constexpr (TM * TN > 8) {
        int part = (int)blockIdx.x % 4, parts = 1;
        if (id >= 0) {
            if (ring_tile<T, FIRST, DIRECT, WM, WN, TM, TN>(a, lds, m0, n0)) return;
            if constexpr (!FAST)
                if (ring_tile<T, ZEROS, DIRECT, WM, WN, TM, TN>(a, lds, m0, n0)) return;
            part = 0;
            parts = 4;
        }
        for (; parts > 0; --parts, ++part) {
            small(m0 + part / 2 * (Shape::BM / 2), n0 + part % 2 * (Shape::BN / 2));
            __syncthreads();
        }
    } else {
        small(m0, n0);
    }
}

template <typename T, bool FAST, bool DIRECT, int WM, int WN, int TM, int TN>
int ring_launch(const LinArgs& a, hipStream_t stream)
{
    typedef RingShape<WM, WN, TM, TN> Shape;
    const int64_t tiles_m = ((int64_t)a.M + Shape::BM - 1) / Shape::BM, tiles_n = ((int64_t)a.N + Shape::BN - 1) / Shape::BN;
    // Where whole tiles would leave half of the compute units or more without one in their last round, so many go in quarters.
    const int64_t last = tiles_m * tiles_n % 256, rest = TM * TN > 8 && last <= 128 ? last : 0, grid = tiles_m * tiles_n + 3 * rest;
    if (!grid_fits(grid, Shape::THREADS)) return SCONV_EUNSUPPORTED;
    const auto kern = linear_ring<T, FAST, DIRECT, WM, WN, TM, TN>;
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)Shape::LDS) != hipSuccess) return SCONV_ELAUNCH;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(Shape::THREADS), Shape::LDS, stream, a, (int)tiles_m, (int)tiles_n, (int)rest);
    return launch_status();
}

template <typename T, int MT, int NT, int NW>
int few_launch(const LinArgs& a, hipStream_t stream)
{
    const int64_t grid = ((int64_t)a.N + 16 * NT - 1) / (16 * NT);
    if (!grid_fits(grid, 64 * NW)) return SCONV_EUNSUPPORTED;
    hipLaunchKernelGGL((linear_few<T, MT, NT, NW>), dim3((unsigned)grid), dim3(64 * NW), 0, stream, a);
    return launch_status();
}

template <typename T, bool FAST>
int linear_run(const LinArgs& a, hipStream_t stream)
{
    // Two weight tiles a workgroup share what it reads of the tokens, where one fills the chip twice (16 tokens, 2048 to 8192: 7.7 -> 6.4 us, 64 tokens
    // by 8-bit products 15.3 -> 9.8); with fewer rows they leave compute units idle (2048 to 2048, 16 tokens: 5.0 -> 5.9).  Tiles through LDS take over where
    // they are ahead by and large (8-bit products: at 64 tokens 2048 to 8192 11.7 us against 9.8, 1024 to 16384 9.0 against 11.6, 8192 to 8192 47 against 34).
    const bool two = a.N >= 4096;
    if (a.M <= 16) return two ? few_launch<T, 1, 2, 8>(a, stream) : few_launch<T, 1, 1, 8>(a, stream);
    if (a.M <= 32) return two ? few_launch<T, 2, 2, 8>(a, stream) : few_launch<T, 2, 1, 8>(a, stream);
    if (a.M <= 64) return two ? few_launch<T, 4, 2, 8>(a, stream) : few_launch<T, 4, 1, 8>(a, stream);
    // (a tile has to lie within what a buffer's offsets reach)
    const bool direct = (a.K | a.x_m | a.w_n) % 16 == 0 && aligned_to(a.x, 16) && aligned_to(a.w, 16) && a.x_m < (int64_t(1) << 22) && a.w_n < (int64_t(1) << 22);
    const int64_t big = (((int64_t)a.M + 255) / 256) * (((int64_t)a.N + 255) / 256);
    if (direct && big >= 256) return ring_launch<T, FAST, true, 2, 2, 4, 4>(a, stream);
    return direct ? ring_launch<T, FAST, true, 2, 2, 2, 2>(a, stream) : ring_launch<T, FAST, false, 2, 2, 2, 2>(a, stream);
}

}  // namespace

int launch_linear8(const sconv_linear8_desc_t& d, const void* x, const uint8_t* xs, const void* w, const uint8_t* ws, void* y, hipStream_t stream)
{
    LinArgs a = {};
    a.x = (const uint8_t*)x; a.xs = xs; a.w = (const uint8_t*)w; a.ws = ws; a.y = y;
    a.M = d.M; a.N = d.N; a.K = d.K; a.KB = (int)(((int64_t)d.K + 127) / 128);
    a.x_m = d.x_m; a.w_n = d.w_n; a.y_m = d.y_m;
    a.vec = d.y_m % 4 == 0 && aligned_to(y, 16);
    if (d.y_type != SCONV_BF16) return linear_run<float, false>(a, stream);
    return d.exact ? linear_run<bf16, false>(a, stream) : linear_run<bf16, true>(a, stream);
}

}  // namespace sconv
