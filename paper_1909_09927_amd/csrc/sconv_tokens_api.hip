// Host side of the token operators: argument checks and dispatch.  No device code here.
#include <math.h>

#include "sconv_tokens_common.h"

namespace sconv {

namespace {

bool aligned_ws(const void* ws, size_t bytes) { return (ws != nullptr) == (bytes != 0) && aligned_to(ws, 16); }

int check_layernorm(const sconv_layernorm_desc_t* d)
{
    if (!d || d->N < 0 || d->S < 0 || d->C < 1) return SCONV_EINVAL;
    if (d->layout != SCONV_LAYOUT_TOKENS && d->layout != SCONV_LAYOUT_MAP) return SCONV_EINVAL;
    if (!type_known(d->x_type) || !type_known(d->y_type) || !type_known(d->w_type)) return SCONV_EINVAL;
    if (d->y_type != d->x_type && !(d->x_type == SCONV_F32 && d->y_type == SCONV_BF16)) return SCONV_EINVAL;
    if (!(d->eps >= 0.0f) || !isfinite(d->eps)) return SCONV_EINVAL;
    if (d->x_n < 0 || d->x_s < 0 || d->y_n < 0 || d->y_s < 0) return SCONV_EINVAL;
    if (d->C > 65536 || (int64_t)d->N * d->S >= (int64_t(1) << 31)) return SCONV_EUNSUPPORTED;
    return SCONV_OK;
}

int check_rotary(const sconv_rotary_desc_t* d)
{
    if (!d || d->B < 0 || d->S < 0 || d->Hq < 0 || d->Hk < 0 || d->D < 1 || !type_known(d->type)) return SCONV_EINVAL;
    if (d->pairs < 1 || d->pairs > d->D / 2 || d->axes < 1) return SCONV_EINVAL;
    if (d->q_b < 0 || d->q_s < 0 || d->q_h < 0 || d->k_b < 0 || d->k_s < 0 || d->k_h < 0 || d->pos_b < 0) return SCONV_EINVAL;
    if (d->qo_b < 0 || d->qo_s < 0 || d->qo_h < 0 || d->ko_b < 0 || d->ko_s < 0 || d->ko_h < 0) return SCONV_EINVAL;
    if (d->D > 1024 || d->pairs > SCONV_ROTARY_MAX_PAIRS || d->axes > SCONV_ROTARY_MAX_AXES) return SCONV_EUNSUPPORTED;
    // (a workgroup's elements are counted in 32 bits, tokens by the grid)
    if ((int64_t)d->B * d->S >= (int64_t(1) << 31) || ((int64_t)d->Hq + d->Hk) * d->D >= (int64_t(1) << 24)) return SCONV_EUNSUPPORTED;
    for (int p = 0; p < d->pairs; ++p)
        if (d->axis[p] >= d->axes) return SCONV_EINVAL;
    return SCONV_OK;
}

int check_diffattn(const sconv_diffattn_desc_t* d)
{
    if (!d || d->B < 0 || d->Sq < 0 || d->Sk < 0 || d->H < 1 || d->Hkv < 1 || d->H % d->Hkv) return SCONV_EINVAL;
    if (d->D < 1 || d->Dv < 1 || !type_known(d->type) || !(d->scale > 0.0f) || !isfinite(d->scale)) return SCONV_EINVAL;
    if (d->q_b < 0 || d->q_s < 0 || d->q_h < 0 || d->k_b < 0 || d->k_s < 0 || d->k_h < 0 || d->v_b < 0 || d->v_s < 0 ||
        d->v_h < 0 || d->mask_b < 0)
        return SCONV_EINVAL;
    if (d->D > 128 || d->Dv > 256) return SCONV_EUNSUPPORTED;
    const int64_t most = int64_t(1) << 30, bh = (int64_t)d->B * d->Hkv, G = d->H / d->Hkv;
    if (d->Sq > most || d->Sk > most || d->Sq * G > most || bh > most) return SCONV_EUNSUPPORTED;
    // (grids: a workgroup a row of the joining kernel, a tile of rows or keys elsewhere)
    if (bh * ((d->Sq * G + 31) / 32) >= (int64_t(1) << 31) || bh * ((d->Sk + 127) / 128) >= (int64_t(1) << 31)) return SCONV_EUNSUPPORTED;
    if ((int64_t)d->B * d->H * (int64_t)d->Sq >= (int64_t(1) << 31)) return SCONV_EUNSUPPORTED;
    const int64_t rows = d->Sq * G, tile = rows > 32 ? 128 : rows > 16 && d->type == SCONV_BF16 ? 32 : 16;   // rows of a forward workgroup
    if (!grid_fits(bh * ((rows + tile - 1) / tile), 256)) return SCONV_EUNSUPPORTED;
    return SCONV_OK;
}

// What the backward kernels' grids take beyond that: 16 rows a workgroup, 128 keys, a head.
int check_diffattn_backward(const sconv_diffattn_desc_t* d)
{
    const int rc = check_diffattn(d);
    if (rc) return rc;
    const bool fits = grid_fits(((int64_t)d->B * d->Sq * d->H + 15) / 16, 256) &&
                      grid_fits((int64_t)d->B * d->Hkv * (((int64_t)d->Sk + 127) / 128), 256) && grid_fits(d->H, 1024);
    return fits ? SCONV_OK : SCONV_EUNSUPPORTED;
}

}  // namespace

}  // namespace sconv

using namespace sconv;

extern "C" {

int sconv_layernorm_workspace_size(const sconv_layernorm_desc_t* desc, size_t* bytes)
{
    const int rc = check_layernorm(desc);
    if (rc) return rc;
    if (!bytes) return SCONV_EINVAL;
    *bytes = layernorm_workspace(*desc);
    return SCONV_OK;
}

int sconv_layernorm_forward(const sconv_layernorm_desc_t* desc, const void* x_dev, const void* w_dev, const void* b_dev,
                            void* y_dev, float* mean_dev, float* rstd_dev, void* hip_stream)
{
    const int rc = check_layernorm(desc);
    if (rc) return rc;
    if (!mean_dev != !rstd_dev) return SCONV_EINVAL;
    if ((int64_t)desc->N * desc->S == 0) return SCONV_OK;
    if (!x_dev || !y_dev) return SCONV_EINVAL;
    return launch_layernorm_forward(*desc, x_dev, w_dev, b_dev, y_dev, mean_dev, rstd_dev, (hipStream_t)hip_stream);
}

int sconv_layernorm_backward(const sconv_layernorm_desc_t* desc, const void* dy_dev, const void* x_dev,
                             const float* mean_dev, const float* rstd_dev, const void* w_dev, void* dx_dev, void* dw_dev,
                             void* db_dev, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    const int rc = check_layernorm(desc);
    if (rc) return rc;
    if (!dw_dev != !db_dev || !aligned_ws(ws_dev, ws_bytes)) return SCONV_EINVAL;
    if (dw_dev && ws_bytes < layernorm_workspace(*desc)) return SCONV_EINVAL;
    if ((int64_t)desc->N * desc->S > 0 && (!dy_dev || !x_dev || !mean_dev || !rstd_dev)) return SCONV_EINVAL;
    return launch_layernorm_backward(*desc, dy_dev, x_dev, mean_dev, rstd_dev, w_dev, dx_dev, dw_dev, db_dev, ws_dev,
                                     (hipStream_t)hip_stream);
}

int sconv_rotary(const sconv_rotary_desc_t* desc, const void* q_dev, const void* k_dev, const int32_t* pos_dev,
                 const float* freq_dev, void* qo_dev, void* ko_dev, void* hip_stream)
{
    const int rc = check_rotary(desc);
    if (rc) return rc;
    if ((int64_t)desc->B * desc->S == 0 || desc->Hq + desc->Hk == 0) return SCONV_OK;
    if (!pos_dev || !freq_dev || (desc->Hq && (!q_dev || !qo_dev)) || (desc->Hk && (!k_dev || !ko_dev))) return SCONV_EINVAL;
    return launch_rotary(*desc, q_dev, k_dev, pos_dev, freq_dev, qo_dev, ko_dev, (hipStream_t)hip_stream);
}

int sconv_diffattn_workspace_size(const sconv_diffattn_desc_t* desc, int backward, size_t* bytes)
{
    const int rc = check_diffattn(desc);
    if (rc) return rc;
    if (!bytes) return SCONV_EINVAL;
    *bytes = backward ? diffattn_backward_workspace(*desc) : diffattn_forward_workspace(*desc);
    return SCONV_OK;
}

int sconv_diffattn_forward(const sconv_diffattn_desc_t* desc, const void* q_dev, const void* k_dev, const void* v_dev,
                           const float* lam_dev, const int32_t* k_lengths_dev, const uint8_t* k_mask_dev, void* out_dev,
                           void* second_dev, float* lse_dev, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    const int rc = check_diffattn(desc);
    if (rc) return rc;
    if (!second_dev != !lse_dev || !aligned_ws(ws_dev, ws_bytes)) return SCONV_EINVAL;
    if (desc->B == 0 || desc->Sq == 0) return SCONV_OK;
    if (!q_dev || !lam_dev || !out_dev || (desc->Sk > 0 && (!k_dev || !v_dev))) return SCONV_EINVAL;
    return launch_diffattn_forward(*desc, q_dev, k_dev, v_dev, lam_dev, k_lengths_dev, k_mask_dev, out_dev, second_dev,
                                   lse_dev, ws_dev, ws_bytes, (hipStream_t)hip_stream);
}

int sconv_diffattn_backward(const sconv_diffattn_desc_t* desc, const void* dout_dev, const void* q_dev, const void* k_dev,
                            const void* v_dev, const float* lam_dev, const int32_t* k_lengths_dev,
                            const uint8_t* k_mask_dev, const void* out_dev, const void* second_dev, const float* lse_dev,
                            void* dq_dev, void* dk_dev, void* dv_dev, float* dlam_dev, void* ws_dev, size_t ws_bytes,
                            void* hip_stream)
{
    const int rc = check_diffattn_backward(desc);
    if (rc) return rc;
    if (!aligned_ws(ws_dev, ws_bytes) || ws_bytes < diffattn_backward_workspace(*desc) || !dlam_dev || !lam_dev) return SCONV_EINVAL;
    const bool queries = desc->B > 0 && desc->Sq > 0, keys = desc->B > 0 && desc->Sk > 0;
    if (queries && (!dout_dev || !q_dev || !out_dev || !second_dev || !lse_dev || !dq_dev)) return SCONV_EINVAL;
    if (keys && (!k_dev || !v_dev || !dk_dev || !dv_dev)) return SCONV_EINVAL;
    return launch_diffattn_backward(*desc, dout_dev, q_dev, k_dev, v_dev, lam_dev, k_lengths_dev, k_mask_dev, out_dev,
                                    second_dev, lse_dev, dq_dev, dk_dev, dv_dev, dlam_dev, ws_dev, (hipStream_t)hip_stream);
}

}  // extern "C"
