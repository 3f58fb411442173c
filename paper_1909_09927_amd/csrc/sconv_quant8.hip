// Rows into 8 bits with block scales (format in sconv_serving.h).
//
// Bound by memory: x is read once, a byte a value and a byte a block are written.  A block of 128 of a row is 16 lanes with eight values
// each; a block of 128 x 128 is a workgroup, which holds it in registers between its largest value and its bytes.  Medians, 16 bits: rows 6272 x 896
// 5.2 us (3.2 TB/s; 2.5 of it the launch), 7.3 behind another kernel's work, 25088 x 2048 30 (5.1 TB/s); blocks 2048 x 2048 6.9 us, 8192 x 2048 11.8
// (4.3 TB/s), 8192 x 8192 41 (4.9).
#include <algorithm>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

struct QuantArgs { const void* x; e4m3* q; uint8_t* scale; int M, K, KB; int64_t x_m, q_m; };

template <typename T>
__global__ __launch_bounds__(256) void quant_rows(QuantArgs a)
{
    const uint32_t block = blockIdx.x * 16u + (threadIdx.x >> 4);        // (fewer than 2^31)
    const uint32_t m = block / (uint32_t)a.KB, kb = block - m * (uint32_t)a.KB;
    const bool live = m < (uint32_t)a.M;
    const int k = (int)kb * 128 + (threadIdx.x & 15) * 8, have = live ? a.K - k : 0;
    float v[8] = {};
    if (have > 0) load8((const T*)a.x + (int64_t)m * a.x_m + k, have, v);
    const int s = scale_byte(lanes_top<false>(finite_top(v)));
    if (have <= 0) return;
    store8(a.q + (int64_t)m * a.q_m + k, have, to_e4m3(v, scale_inverse(s)));
    if ((threadIdx.x & 15) == 0) a.scale[block] = (uint8_t)s;
}

template <typename T>
__global__ __launch_bounds__(256) void quant_blocks(QuantArgs a)
{
    __shared__ uint32_t tops[16];
    const uint32_t mb = blockIdx.x / (uint32_t)a.KB, kb = blockIdx.x - mb * (uint32_t)a.KB;
    const int k = (int)kb * 128 + (threadIdx.x & 15) * 8, have = a.K - k, m0 = (int)mb * 128 + (threadIdx.x >> 4);
    float v[8][8] = {};
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (have > 0 && m0 + 16 * j < a.M) load8((const T*)a.x + (int64_t)(m0 + 16 * j) * a.x_m + k, have, v[j]);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, finite_top(v[j]));
    top = lanes_top<false>(top);
    if ((threadIdx.x & 15) == 0) tops[threadIdx.x >> 4] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, tops[i]);
    const int s = scale_byte(top);
    if (threadIdx.x == 0) a.scale[blockIdx.x] = (uint8_t)s;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (have > 0 && m0 + 16 * j < a.M) store8(a.q + (int64_t)(m0 + 16 * j) * a.q_m + k, have, to_e4m3(v[j], scale_inverse(s)));
}

}  // namespace

int launch_quant8(const sconv_quant8_desc_t& d, const void* x, void* q, uint8_t* scale, hipStream_t stream)
{
    const QuantArgs a = {x, (e4m3*)q, scale, d.M, d.K, (d.K + 127) / 128, d.x_m, d.q_m};
    const int64_t blocks = (d.block_rows == 1 ? (int64_t)d.M : ((int64_t)d.M + 127) / 128) * a.KB;
    const int64_t grid = d.block_rows == 1 ? (blocks + 15) / 16 : blocks;
    if (blocks >= (int64_t(1) << 31) - 16 || !grid_fits(grid, 256)) return SCONV_EUNSUPPORTED;
    if (d.block_rows == 1) {
        if (d.type == SCONV_BF16) hipLaunchKernelGGL((quant_rows<bf16>), dim3((unsigned)grid), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((quant_rows<float>), dim3((unsigned)grid), dim3(256), 0, stream, a);
    } else {
        if (d.type == SCONV_BF16) hipLaunchKernelGGL((quant_blocks<bf16>), dim3((unsigned)grid), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((quant_blocks<float>), dim3((unsigned)grid), dim3(256), 0, stream, a);
    }
    return launch_status();
}

}  // namespace sconv
