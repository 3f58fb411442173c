// A paged cache of keys and values: new tokens into its pages, and positions out of them (format and conventions in sconv_serving.h).
//
// Bound by memory, or by latency where a call has few tokens: keys and values share one launch, and a head of a token is a group of
// LPR lanes with eight elements each, whose largest value comes by rotation.  The group finds its slot by itself: one division
// by the page size, by multiplication, and one read of the table.
#include <algorithm>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

struct CacheArgs {
    void* k; void* v; sconv_pages_dev_t dev; const int32_t* starts; const int32_t* counts;
    int S, heads, Hk, D, Dv, pages, width;             // heads: keys' and values'
    int64_t rows;                                      // B * S * heads
    int64_t k_b, k_s, k_h, v_b, v_s, v_h;
    int64_t kp, ks, kh, vp, vs, vh, kxp, kxs, kxh, vxp, vxs, vxh, table_b;   // pages, scales
    Divide page;
};

// T: the tokens' type; P: the pages'.
template <typename T, typename P, int LPR, bool WRITE>
__global__ __launch_bounds__(256) void cache_rows(CacheArgs a)
{
    const uint32_t row = blockIdx.x * (256u / LPR) + threadIdx.x / LPR;      // (fewer than 2^31)
    const bool live = row < (uint32_t)a.rows;
    const uint32_t token = row / (uint32_t)a.heads, b = token / (uint32_t)a.S;
    const int head = (int)(row - token * (uint32_t)a.heads), i = (int)(token - b * (uint32_t)a.S), d = threadIdx.x % LPR * 8;
    const bool key = head < a.Hk;
    const int h = key ? head : head - a.Hk, have = (key ? a.D : a.Dv) - d;
    int page = -1, slot = 0;
    if (live) {
        const int64_t at = (int64_t)a.starts[b] + i;
        if (at >= 0 && at < (int64_t)a.width * a.page.d && (!a.counts || i < a.counts[b])) {
            const uint32_t n = divided((uint32_t)at, a.page);
            slot = (int)((uint32_t)at - n * a.page.d);
            page = a.dev.table[b * a.table_b + n];
        }
    }
    const bool there = page >= 0 && page < a.pages;
    if (!live || (WRITE && !there)) return;              // (a row's lanes all alike)
    T* token_row = key ? (T*)a.k + b * a.k_b + i * a.k_s + h * a.k_h : (T*)a.v + b * a.v_b + i * a.v_s + h * a.v_h;
    const int64_t at = key ? page * a.kp + slot * a.ks + h * a.kh : page * a.vp + slot * a.vs + h * a.vh;
    P* kept = (P*)(key ? a.dev.k : a.dev.v) + at;
    uint8_t* scale = nullptr;
    if constexpr (sizeof(P) == 1) scale = key ? a.dev.ks + page * a.kxp + slot * a.kxs + h * a.kxh : a.dev.vs + page * a.vxp + slot * a.vxs + h * a.vxh;
    float v[8] = {};
    if constexpr (WRITE) {
        if (have > 0) load8(token_row + d, have, v);
        if constexpr (sizeof(P) == 1) {
            const int s = scale_byte(lanes_top<(LPR > 16)>(finite_top(v)));
            if (have > 0) store8(kept + d, have, to_e4m3(v, scale_inverse(s)));
            if (d == 0) *scale = (uint8_t)s;
        } else if (have > 0) {
            store8(kept + d, have, v);
        }
    } else if (have > 0) {
        if (there) {
            if constexpr (sizeof(P) == 1) from_e4m3(load8_bytes(kept + d, have), scale_of(*scale), v);
            else load8(kept + d, have, v);
        }
        store8(token_row + d, have, v);
    }
}

template <typename T, typename P>
int cache_run(const CacheArgs& a, bool write, hipStream_t stream)
{
    const int lpr = std::max(a.D, a.Dv) <= 128 ? 16 : 32;
    const int64_t grid = (a.rows + 256 / lpr - 1) / (256 / lpr);
    if (a.rows >= (int64_t(1) << 31) - 16 || !grid_fits(grid, 256)) return SCONV_EUNSUPPORTED;
    const dim3 blocks((unsigned)grid), threads(256);
    if (write) {
        if (lpr == 16) hipLaunchKernelGGL((cache_rows<T, P, 16, true>), blocks, threads, 0, stream, a);
        else hipLaunchKernelGGL((cache_rows<T, P, 32, true>), blocks, threads, 0, stream, a);
    } else {
        if (lpr == 16) hipLaunchKernelGGL((cache_rows<T, P, 16, false>), blocks, threads, 0, stream, a);
        else hipLaunchKernelGGL((cache_rows<T, P, 32, false>), blocks, threads, 0, stream, a);
    }
    return launch_status();
}

}  // namespace

int launch_cache(const sconv_cache_desc_t& d, bool write, void* k, void* v, const int32_t* starts, const int32_t* counts,
                 const sconv_pages_dev_t& pages, hipStream_t stream)
{
    const sconv_pages_t& p = d.pages;
    CacheArgs a = {};
    a.k = k; a.v = v; a.dev = pages; a.starts = starts; a.counts = counts;
    a.S = d.S; a.Hk = p.Hk; a.heads = p.Hk + p.Hv; a.D = p.D; a.Dv = p.Dv; a.pages = p.pages; a.width = p.table_width;
    a.rows = (int64_t)d.B * d.S * a.heads;
    a.k_b = d.k_b; a.k_s = d.k_s; a.k_h = d.k_h; a.v_b = d.v_b; a.v_s = d.v_s; a.v_h = d.v_h;
    a.kp = p.k_p; a.ks = p.k_s; a.kh = p.k_h; a.vp = p.v_p; a.vs = p.v_s; a.vh = p.v_h;
    a.kxp = p.ks_p; a.kxs = p.ks_s; a.kxh = p.ks_h; a.vxp = p.vs_p; a.vxs = p.vs_s; a.vxh = p.vs_h;
    a.table_b = p.table_b; a.page = divide_by((uint32_t)p.page_size);
    if (d.type == SCONV_BF16) return p.type == SCONV_E4M3 ? cache_run<bf16, e4m3>(a, write, stream) : cache_run<bf16, bf16>(a, write, stream);
    return p.type == SCONV_E4M3 ? cache_run<float, e4m3>(a, write, stream) : cache_run<float, float>(a, write, stream);
}

}  // namespace sconv
