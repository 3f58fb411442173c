// Host side of the serving operators: argument checks and dispatch.  No device code here.
#include <math.h>

#include "sconv_serving_common.h"

namespace sconv {

namespace {

bool aligned_ws(const void* ws, size_t bytes) { return (ws != nullptr) == (bytes != 0) && aligned_to(ws, 16); }

int check_rmsnorm(const sconv_rmsnorm_desc_t* d, bool backward)
{
    if (!d || d->rows < 0 || d->C < 1 || !type_known(d->x_type) || !type_known(d->t_type) || !type_known(d->w_type)) return SCONV_EINVAL;
    if (d->t_type != d->x_type && d->t_type != SCONV_F32) return SCONV_EINVAL;
    if (d->y_type != d->x_type && d->y_type != SCONV_BF16 && (backward || d->y_type != SCONV_E4M3)) return SCONV_EINVAL;
    if (!(d->eps >= 0.0f) || !isfinite(d->eps) || d->x_r < 0 || d->res_r < 0 || d->t_r < 0 || d->y_r < 0) return SCONV_EINVAL;
    if (d->C > 16384 || d->rows > 1 << 30) return SCONV_EUNSUPPORTED;
    return SCONV_OK;
}

int check_quant8(const sconv_quant8_desc_t* d)
{
    if (!d || d->M < 0 || d->K < 0 || !type_known(d->type) || (d->block_rows != 1 && d->block_rows != 128) || d->x_m < 0 || d->q_m < 0) return SCONV_EINVAL;
    return d->M > 1 << 30 || d->K > 1 << 30 ? SCONV_EUNSUPPORTED : SCONV_OK;
}

int check_linear8(const sconv_linear8_desc_t* d)
{
    if (!d || d->M < 0 || d->N < 0 || d->K < 0 || !type_known(d->y_type) || d->x_m < 0 || d->w_n < 0 || d->y_m < 0) return SCONV_EINVAL;
    if (d->exact != 0 && d->exact != 1) return SCONV_EINVAL;
    return d->M > 1 << 30 || d->N > 1 << 30 || d->K > 1 << 30 ? SCONV_EUNSUPPORTED : SCONV_OK;
}

int check_pages(const sconv_pages_t& p, int type)
{
    if (p.pages < 0 || p.page_size < 1 || p.table_width < 0 || p.Hk < 1 || p.Hv < 1 || p.D < 1 || p.Dv < 1) return SCONV_EINVAL;
    if (!type_known(type) || (p.type != type && p.type != SCONV_E4M3)) return SCONV_EINVAL;
    for (const int64_t s : {p.k_p, p.k_s, p.k_h, p.v_p, p.v_s, p.v_h, p.ks_p, p.ks_s, p.ks_h, p.vs_p, p.vs_s, p.vs_h, p.table_b})
        if (s < 0) return SCONV_EINVAL;
    if (p.D > 256 || p.Dv > 256 || p.Hk > 1 << 20 || p.Hv > 1 << 20) return SCONV_EUNSUPPORTED;
    if ((int64_t)p.table_width * p.page_size >= int64_t(1) << 31) return SCONV_EUNSUPPORTED;
    return SCONV_OK;
}

// Whether the pages' addresses are there, and their scales where they are wanted and only there.
bool pages_given(const sconv_pages_t& p, const sconv_pages_dev_t* g)
{
    if (!g) return false;
    const bool scales = p.type == SCONV_E4M3;
    if (!scales && (g->ks || g->vs)) return false;
    if (p.table_width > 0 && !g->table) return false;
    return p.pages == 0 || (g->k && g->v && (!scales || (g->ks && g->vs)));
}

int check_cache(const sconv_cache_desc_t* d)
{
    if (!d || d->B < 0 || d->S < 0 || d->k_b < 0 || d->k_s < 0 || d->k_h < 0 || d->v_b < 0 || d->v_s < 0 || d->v_h < 0) return SCONV_EINVAL;
    const int rc = check_pages(d->pages, d->type);
    if (rc) return rc;
    return (int64_t)d->B * d->S >= (int64_t(1) << 31) / (d->pages.Hk + d->pages.Hv) ? SCONV_EUNSUPPORTED : SCONV_OK;
}

int check_paged(const sconv_paged_desc_t* d)
{
    if (!d || d->B < 0 || d->Sq < 0 || d->H < 1 || d->Hkv < 1 || d->H % d->Hkv || !(d->scale > 0.0f) || !isfinite(d->scale)) return SCONV_EINVAL;
    if (d->q_b < 0 || d->q_s < 0 || d->q_h < 0) return SCONV_EINVAL;
    const int rc = check_pages(d->pages, d->type);
    if (rc) return rc;
    if ((int64_t)d->pages.Hk != 2 * (int64_t)d->Hkv || d->pages.Hv != d->Hkv) return SCONV_EINVAL;
    if (d->pages.D > 128 || d->H > 1 << 20 || d->Sq > 1 << 20 || d->B > 1 << 24) return SCONV_EUNSUPPORTED;
    // (a row of the joining kernel is a workgroup of 256, a request's rows of a key head are tiles of 16)
    const int64_t rows = (int64_t)d->Sq * (d->H / d->Hkv);
    if (!grid_fits((int64_t)d->B * d->Sq * d->H, 256) || !grid_fits((int64_t)(d->B > 1024 ? d->B : 1024) * d->Hkv * ((rows + 15) / 16), 256))
        return SCONV_EUNSUPPORTED;
    return SCONV_OK;
}

}  // namespace

}  // namespace sconv

using namespace sconv;

extern "C" {

int sconv_rmsnorm_workspace_size(const sconv_rmsnorm_desc_t* desc, size_t* bytes)
{
    const int rc = check_rmsnorm(desc, true);
    if (rc) return rc;
    if (!bytes) return SCONV_EINVAL;
    *bytes = rmsnorm_workspace(*desc);
    return SCONV_OK;
}

int sconv_rmsnorm_forward(const sconv_rmsnorm_desc_t* desc, const void* x_dev, const void* residual_dev, const void* w_dev, void* y_dev,
                          uint8_t* y_scale_dev, void* total_dev, float* rstd_dev, void* hip_stream)
{
    const int rc = check_rmsnorm(desc, false);
    if (rc) return rc;
    if (desc->rows == 0) return SCONV_OK;
    if (!x_dev || !y_dev || (desc->y_type == SCONV_E4M3) != (y_scale_dev != nullptr) || !residual_dev != !total_dev) return SCONV_EINVAL;
    return launch_rmsnorm_forward(*desc, x_dev, residual_dev, w_dev, y_dev, y_scale_dev, total_dev, rstd_dev, (hipStream_t)hip_stream);
}

int sconv_rmsnorm_backward(const sconv_rmsnorm_desc_t* desc, const void* dy_dev, const void* total_dev, const float* rstd_dev,
                           const void* w_dev, const void* dt_dev, void* dx_dev, void* dres_dev, void* dw_dev, void* ws_dev,
                           size_t ws_bytes, void* hip_stream)
{
    const int rc = check_rmsnorm(desc, true);
    if (rc) return rc;
    if (!aligned_ws(ws_dev, ws_bytes) || (dw_dev && ws_bytes < rmsnorm_workspace(*desc))) return SCONV_EINVAL;
    if (desc->rows > 0 && (!dy_dev || !total_dev || !rstd_dev)) return SCONV_EINVAL;
    return launch_rmsnorm_backward(*desc, dy_dev, total_dev, rstd_dev, w_dev, dt_dev, dx_dev, dres_dev, dw_dev, ws_dev, (hipStream_t)hip_stream);
}

int sconv_quant8(const sconv_quant8_desc_t* desc, const void* x_dev, void* q_dev, uint8_t* scale_dev, void* hip_stream)
{
    const int rc = check_quant8(desc);
    if (rc) return rc;
    if (desc->M == 0 || desc->K == 0) return SCONV_OK;
    if (!x_dev || !q_dev || !scale_dev) return SCONV_EINVAL;
    return launch_quant8(*desc, x_dev, q_dev, scale_dev, (hipStream_t)hip_stream);
}

int sconv_linear8(const sconv_linear8_desc_t* desc, const void* x_dev, const uint8_t* x_scale_dev, const void* w_dev,
                  const uint8_t* w_scale_dev, void* y_dev, void* hip_stream)
{
    const int rc = check_linear8(desc);
    if (rc) return rc;
    if (desc->M == 0 || desc->N == 0) return SCONV_OK;
    if (!y_dev || (desc->K > 0 && (!x_dev || !x_scale_dev || !w_dev || !w_scale_dev))) return SCONV_EINVAL;
    return launch_linear8(*desc, x_dev, x_scale_dev, w_dev, w_scale_dev, y_dev, (hipStream_t)hip_stream);
}

int sconv_cache_write(const sconv_cache_desc_t* desc, const void* k_dev, const void* v_dev, const int32_t* starts_dev,
                      const int32_t* counts_dev, const sconv_pages_dev_t* pages, void* hip_stream)
{
    const int rc = check_cache(desc);
    if (rc) return rc;
    if (!pages_given(desc->pages, pages)) return SCONV_EINVAL;
    if (desc->B == 0 || desc->S == 0) return SCONV_OK;
    if (!k_dev || !v_dev || !starts_dev) return SCONV_EINVAL;
    if (desc->pages.pages == 0 || desc->pages.table_width == 0) return SCONV_OK;
    return launch_cache(*desc, true, const_cast<void*>(k_dev), const_cast<void*>(v_dev), starts_dev, counts_dev, *pages, (hipStream_t)hip_stream);
}

int sconv_cache_read(const sconv_cache_desc_t* desc, const sconv_pages_dev_t* pages, const int32_t* starts_dev,
                     const int32_t* counts_dev, void* k_dev, void* v_dev, void* hip_stream)
{
    const int rc = check_cache(desc);
    if (rc) return rc;
    if (!pages_given(desc->pages, pages)) return SCONV_EINVAL;
    if (desc->B == 0 || desc->S == 0) return SCONV_OK;
    if (!k_dev || !v_dev || !starts_dev) return SCONV_EINVAL;
    return launch_cache(*desc, false, k_dev, v_dev, starts_dev, counts_dev, *pages, (hipStream_t)hip_stream);
}

int sconv_diffattn_paged_workspace_size(const sconv_paged_desc_t* desc, size_t* bytes)
{
    const int rc = check_paged(desc);
    if (rc) return rc;
    if (!bytes) return SCONV_EINVAL;
    *bytes = paged_workspace(*desc);
    return SCONV_OK;
}

int sconv_diffattn_paged(const sconv_paged_desc_t* desc, const void* q_dev, const sconv_pages_dev_t* pages, const float* lam_dev,
                         const int32_t* lengths_dev, void* out_dev, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    const int rc = check_paged(desc);
    if (rc) return rc;
    if (!aligned_ws(ws_dev, ws_bytes) || !pages_given(desc->pages, pages)) return SCONV_EINVAL;
    if (desc->B == 0 || desc->Sq == 0) return SCONV_OK;
    if (!q_dev || !lam_dev || !lengths_dev || !out_dev) return SCONV_EINVAL;
    return launch_paged(*desc, q_dev, *pages, lam_dev, lengths_dev, out_dev, ws_dev, ws_bytes, (hipStream_t)hip_stream);
}

}  // extern "C"
