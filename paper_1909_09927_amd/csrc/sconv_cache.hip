// A paged cache of keys and values: new tokens into its pages, and positions out of them (format and conventions in sconv_serving.h).
//
// Bound by memory, or by latency where a call has few tokens: keys and values share one launch.  A head of a token is a group of LPR lanes
// with eight elements each, whose largest value comes by rotation; a group finds its token's slot by itself: one division by the page size, by
// multiplication, and one read of the table.  A workgroup has a stretch of tokens of a head, then of the next: a page's lines, of which a slot
// of a head is half a line or less, and a slot's scale a byte, are written from one place, whichever of heads and slots lie beside each other.
// (Medians of 8 x 3136 tokens of 8 key heads of 64 and 4 value heads of 128, 16 to 8 bits: 21.8 us written, 21.4 read, 3.5 and 3.6 TB/s; of up to
// 3136, ragged, 14.9 and 14.9.  Heads side by side, tokens apart, the same 8 x 3136 took two fifths longer.)
#include <algorithm>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

struct CacheArgs {
    void* k; void* v; sconv_pages_dev_t dev; const int32_t* starts; const int32_t* counts;
    int Hk, heads, D, Dv, pages, width, tokens, per, chunks;   // heads: keys' and values'; a workgroup has `per` of them
    int64_t k_b, k_s, k_h, v_b, v_s, v_h;
    int64_t kp, ks, kh, vp, vs, vh, kxp, kxs, kxh, vxp, vxs, vxh, table_b;   // pages, scales
    Divide page, by_tokens;
};

constexpr int ROWS = 2;                                // heads at once (four: 8 x 3136 tokens 19.7 -> 22.4 us)

// T: the tokens' type; P: the pages'.
template <typename T, typename P, int LPR, bool WRITE>
__global__ __launch_bounds__(256) void cache_rows(CacheArgs a)
{
    const int tile = blockIdx.x / a.chunks, first = (blockIdx.x - tile * a.chunks) * a.per, last = min(first + a.per, a.heads);
    const int token = tile * (256 / LPR) + threadIdx.x / LPR, d = threadIdx.x % LPR * 8;
    if (token >= a.tokens) return;
    const int b = (int)divided((uint32_t)token, a.by_tokens), i = token - b * (int)a.by_tokens.d;
    const int64_t at = (int64_t)a.starts[b] + i;
    int page = -1, slot = 0;
    if (at >= 0 && at < (int64_t)a.width * a.page.d && (!a.counts || i < a.counts[b])) {
        const uint32_t n = divided((uint32_t)at, a.page);
        slot = (int)((uint32_t)at - n * a.page.d);
        page = a.dev.table[b * a.table_b + n];
    }
    const bool there = page >= 0 && page < a.pages;
    if (WRITE && !there) return;                         // (a token's lanes all alike)
    T* token_k = (T*)a.k + b * a.k_b + i * a.k_s + d;
    T* token_v = (T*)a.v + b * a.v_b + i * a.v_s + d;
    P* page_k = (P*)a.dev.k + (page * a.kp + slot * a.ks) + d;
    P* page_v = (P*)a.dev.v + (page * a.vp + slot * a.vs) + d;
    uint8_t* scale_k = a.dev.ks + (page * a.kxp + slot * a.kxs);
    uint8_t* scale_v = a.dev.vs + (page * a.vxp + slot * a.vxs);
    for (int h0 = first; h0 < last; h0 += ROWS) {
        float v[ROWS][8] = {};
        [[maybe_unused]] u32x2 bytes[ROWS] = {};
        [[maybe_unused]] int s[ROWS] = {};
        T* row[ROWS]; P* kept[ROWS]; uint8_t* scale[ROWS];
        int have[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int head = min(h0 + r, last - 1);
            const bool key = head < a.Hk;
            const int h = key ? head : head - a.Hk;
            have[r] = h0 + r < last ? (key ? a.D : a.Dv) - d : 0;
            row[r] = key ? token_k + h * a.k_h : token_v + h * a.v_h;
            kept[r] = key ? page_k + h * a.kh : page_v + h * a.vh;
            if constexpr (sizeof(P) == 1) scale[r] = key ? scale_k + h * a.kxh : scale_v + h * a.vxh;
            if (have[r] > 0 && there) {
                if constexpr (WRITE) {
                    load8(row[r], have[r], v[r]);
                } else if constexpr (sizeof(P) == 1) {
                    bytes[r] = load8_bytes(kept[r], have[r]);
                    s[r] = *scale[r];
                } else {
                    load8(kept[r], have[r], v[r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if constexpr (WRITE && sizeof(P) == 1) {
                s[r] = scale_byte(lanes_top<(LPR > 16)>(finite_top(v[r])));
                if (have[r] > 0) store8(kept[r], have[r], to_e4m3(v[r], scale_inverse(s[r])));
                if (h0 + r < last && d == 0) *scale[r] = (uint8_t)s[r];
            } else if constexpr (WRITE) {
                if (have[r] > 0) store8(kept[r], have[r], v[r]);
            } else if (have[r] > 0) {
                if constexpr (sizeof(P) == 1)
                    if (there) from_e4m3(bytes[r], scale_of(s[r]), v[r]);
                store8(row[r], have[r], v[r]);
            }
        }
    }
}

template <typename T, typename P, int LPR>
int cache_launch(CacheArgs a, bool write, hipStream_t stream)
{
    // Heads of a workgroup: few where there is little to do, all where a great many workgroups wait (8 key heads of 64 and 4 value heads of 128,
    // 64 tokens, one head, two, all: 8.3, 8.3, 9.1 us; 8 x 3136, two, four, all: 22.8, 19.7, 20.0; 32 x 3136: 96, 78, 68).
    const int64_t tiles = (a.tokens + 256 / LPR - 1) / (256 / LPR), rows = tiles * a.heads;
    a.per = std::min(rows < 1 << 11 ? 2 : rows < 1 << 16 ? 4 : a.heads, a.heads);
    a.chunks = (a.heads + a.per - 1) / a.per;
    const int64_t grid = tiles * a.chunks;
    if (!grid_fits(grid, 256)) return SCONV_EUNSUPPORTED;
    const dim3 blocks((unsigned)grid), threads(256);
    if (write) hipLaunchKernelGGL((cache_rows<T, P, LPR, true>), blocks, threads, 0, stream, a);
    else hipLaunchKernelGGL((cache_rows<T, P, LPR, false>), blocks, threads, 0, stream, a);
    return launch_status();
}

template <typename T, typename P>
int cache_run(const CacheArgs& a, bool write, hipStream_t stream)
{
    return std::max(a.D, a.Dv) <= 128 ? cache_launch<T, P, 16>(a, write, stream) : cache_launch<T, P, 32>(a, write, stream);
}

}  // namespace

int launch_cache(const sconv_cache_desc_t& d, bool write, void* k, void* v, const int32_t* starts, const int32_t* counts,
                 const sconv_pages_dev_t& pages, hipStream_t stream)
{
    const sconv_pages_t& p = d.pages;
    CacheArgs a = {};
    a.k = k; a.v = v; a.dev = pages; a.starts = starts; a.counts = counts;
    a.Hk = p.Hk; a.heads = p.Hk + p.Hv; a.tokens = d.B * d.S; a.D = p.D; a.Dv = p.Dv; a.pages = p.pages; a.width = p.table_width;
    a.k_b = d.k_b; a.k_s = d.k_s; a.k_h = d.k_h; a.v_b = d.v_b; a.v_s = d.v_s; a.v_h = d.v_h;
    a.kp = p.k_p; a.ks = p.k_s; a.kh = p.k_h; a.vp = p.v_p; a.vs = p.v_s; a.vh = p.v_h;
    a.kxp = p.ks_p; a.kxs = p.ks_s; a.kxh = p.ks_h; a.vxp = p.vs_p; a.vxs = p.vs_s; a.vxh = p.vs_h;
    a.table_b = p.table_b; a.page = divide_by((uint32_t)p.page_size);
    a.by_tokens = divide_by((uint32_t)std::max(d.S, 1));
    if (d.type == SCONV_BF16) return p.type == SCONV_E4M3 ? cache_run<bf16, e4m3>(a, write, stream) : cache_run<bf16, bf16>(a, write, stream);
    return p.type == SCONV_E4M3 ? cache_run<float, e4m3>(a, write, stream) : cache_run<float, float>(a, write, stream);
}

}  // namespace sconv
