// C ABI of the operators around the layer: checks of the descriptors, then
// the launches of k_norm.cu, k_scores.cu and k_clip.cu.
#include <cmath>

#include "pmpe_internal.cuh"

namespace pmpe {
namespace {

constexpr int kMaxRows = 1 << 30;  // rows and grid strides past them stay within 32 bits

bool is_type(int t) { return t == PMPE_F32 || t == PMPE_BF16 || t == PMPE_F16; }
bool fits(const void *p, int type) { return ((uintptr_t)p & (type == PMPE_F32 ? 3u : 1u)) == 0; }
bool fits4(const void *p) { return ((uintptr_t)p & 3u) == 0; }
int done(cudaError_t err) { return err == cudaSuccess ? PMPE_OK : PMPE_ERR_CUDA; }

int sm_count(int *n)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PMPE_ERR_CUDA;
    return done(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
}

// Rows of `bytes` bytes each, `pitch` bytes apart.
struct Rows {
    const void *at;
    int64_t n, bytes, pitch;
};
// Whether a run of memory holds a byte of the rows.
bool meets(const void *p, int64_t bytes, const Rows &r)
{
    if (!p || !r.at || r.n == 0) return false;
    const int64_t lo = (int64_t)((uintptr_t)p - (uintptr_t)r.at), hi = lo + bytes;
    const int64_t i = lo < r.bytes ? 0 : (lo - r.bytes) / r.pitch + 1;  // the first row that ends after lo
    return i < r.n && i * r.pitch < hi;
}
// Whether an output without gaps is apart from the rows, or is those rows,
// each of which is read before it is written.
bool may_write(const void *p, int64_t bytes, const Rows &r)
{
    return !meets(p, bytes, r) || (p == r.at && bytes == r.n * r.bytes && (r.n == 1 || r.pitch == r.bytes));
}

bool groups_ok(int pool, int groups, int top, int k)
{
    return groups >= 1 && groups <= 32 && pool % groups == 0 && top >= 1 && top <= groups && top * (pool / groups) >= k;
}

int check_route(const pmpe_route_desc *d)
{
    if (!d || d->T < 0 || d->k < 1 || d->E_pub < d->k || d->E_priv < 0 || (d->E_priv > 0 && d->E_priv < d->k))
        return PMPE_ERR_INVALID_ARG;
    if (!is_type(d->logits_type) || (d->score != PMPE_SCORE_SOFTMAX && d->score != PMPE_SCORE_SIGMOID) ||
        (d->renormalize != 0 && d->renormalize != 1) || !std::isfinite(d->scale) || (d->E_priv == 0 && d->policy) ||
        d->ld < (int64_t)d->E_pub + d->E_priv)
        return PMPE_ERR_INVALID_ARG;
    if (d->k > kMaxTopK || d->E_pub > kMaxPool || d->E_priv > kMaxPool || d->T > kMaxRows) return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (d->T > 0 && (!d->logits || !d->topk_idx)) return PMPE_ERR_INVALID_ARG;
    if (!fits(d->logits, d->logits_type) || !fits4(d->topk_idx)) return PMPE_ERR_UNSUPPORTED_SHAPE;
    return PMPE_OK;
}

}  // namespace
}  // namespace pmpe

using namespace pmpe;

extern "C" {

int pmpe_rms_norm(const pmpe_rms_norm_desc *d, void *stream)
{
    if (!d || d->T < 0 || d->H < 1 || !is_type(d->type) || (d->weight_type != d->type && d->weight_type != PMPE_F32) ||
        d->quant < PMPE_QUANT_NONE || d->quant > PMPE_QUANT_ROW || !(d->eps >= 1e-20f) || !std::isfinite(d->eps))
        return PMPE_ERR_INVALID_ARG;
    if (d->H > PMPE_MAX_NORM_WIDTH || d->T > kMaxRows) return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (d->x_ld < d->H || (d->residual && d->residual_ld < d->H))
        return PMPE_ERR_INVALID_ARG;
    if (d->T == 0) return PMPE_OK;
    if (!d->x || !d->weight || !d->y || (d->quant == PMPE_QUANT_NONE) != !d->scale) return PMPE_ERR_INVALID_ARG;
    if (!fits(d->x, d->type) || !fits(d->residual, d->type) || !fits(d->weight, d->weight_type) || !fits(d->h, d->type) ||
        (d->quant == PMPE_QUANT_NONE && !fits(d->y, d->type)) || !fits4(d->scale) || !fits4(d->rstd))
        return PMPE_ERR_UNSUPPORTED_SHAPE;
    const int64_t T = d->T, H = d->H, e = d->type == PMPE_F32 ? 4 : 2;
    const int64_t h_bytes = T * H * e, y_bytes = d->quant == PMPE_QUANT_NONE ? h_bytes : T * H;
    const Rows x = {d->x, T, H * e, T > 1 ? d->x_ld * e : H * e}, res = {d->residual, T, H * e, T > 1 ? d->residual_ld * e : H * e};
    const Rows w = {d->weight, 1, H * (d->weight_type == PMPE_F32 ? 4 : 2), 1}, h = {d->h, 1, h_bytes, 1};
    // (8-bit rows are another type's, on none of the inputs)
    const bool y_ok = d->quant == PMPE_QUANT_NONE ? may_write(d->y, y_bytes, x) && may_write(d->y, y_bytes, res)
                                                  : !meets(d->y, y_bytes, x) && !meets(d->y, y_bytes, res);
    if (!y_ok || !may_write(d->h, h_bytes, x) || !may_write(d->h, h_bytes, res) || meets(d->h, h_bytes, w) || meets(d->y, y_bytes, w) ||
        meets(d->y, y_bytes, h))
        return PMPE_ERR_INVALID_ARG;
    return done(launch_rms_norm(*d, (cudaStream_t)stream));
}

size_t pmpe_rms_norm_backward_workspace_size(int T, int H)
{
    return T < 0 || T > kMaxRows || H < 1 || H > PMPE_MAX_NORM_WIDTH ? 0 : rms_norm_backward_workspace_bytes(T, H);
}

int pmpe_rms_norm_backward(const pmpe_rms_norm_backward_desc *d, void *stream)
{
    if (!d || d->T < 0 || d->H < 1 || !is_type(d->type) || (d->weight_type != d->type && d->weight_type != PMPE_F32) ||
        (d->dy_type != d->type && d->dy_type != PMPE_F32) || (d->dx_type != d->type && d->dx_type != PMPE_F32))
        return PMPE_ERR_INVALID_ARG;
    if (d->H > PMPE_MAX_NORM_WIDTH || d->T > kMaxRows) return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (!fits4(d->dw)) return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (d->T == 0)  // no rows: the weight's gradient is zero
        return d->dw ? done(cudaMemsetAsync(d->dw, 0, (size_t)d->H * sizeof(float), (cudaStream_t)stream)) : PMPE_OK;
    if (!d->dy || !d->h || !d->weight || !d->rstd || !d->dx) return PMPE_ERR_INVALID_ARG;
    if (!fits(d->dy, d->dy_type) || !fits(d->h, d->type) || !fits(d->weight, d->weight_type) || !fits4(d->rstd) ||
        !fits(d->d_h, d->dx_type) || !fits(d->dx, d->dx_type))
        return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (d->dw && (!d->workspace || ((uintptr_t)d->workspace & 15u) ||
                  d->workspace_bytes < rms_norm_backward_workspace_bytes(d->T, d->H)))
        return PMPE_ERR_WORKSPACE;
    return done(launch_rms_norm_backward(*d, (cudaStream_t)stream));
}

int pmpe_route(const pmpe_route_desc *d, void *stream)
{
    int rc = check_route(d);
    if (rc != PMPE_OK) return rc;
    if ((d->group_score != PMPE_GROUP_MAX && d->group_score != PMPE_GROUP_TOP2) ||
        !groups_ok(d->E_pub, d->groups_pub, d->top_groups_pub, d->k) ||
        (d->E_priv > 0 && !groups_ok(d->E_priv, d->groups_priv, d->top_groups_priv, d->k)) || (d->T > 0 && !d->topk_w))
        return PMPE_ERR_INVALID_ARG;
    if (!fits4(d->bias) || !fits4(d->topk_w) || !fits4(d->load)) return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (d->T == 0) return PMPE_OK;
    int sms = 0;
    if ((rc = sm_count(&sms)) != PMPE_OK) return rc;
    return done(launch_route_scores(*d, sms, (cudaStream_t)stream));
}

int pmpe_route_backward(const pmpe_route_desc *d, const float *dw, void *d_logits, void *stream)
{
    int rc = check_route(d);
    if (rc != PMPE_OK) return rc;
    if (d->T > 0 && (!dw || !d_logits)) return PMPE_ERR_INVALID_ARG;
    if (!fits4(dw) || !fits(d_logits, d->logits_type)) return PMPE_ERR_UNSUPPORTED_SHAPE;
    if (d->T == 0) return PMPE_OK;
    int sms = 0;
    if ((rc = sm_count(&sms)) != PMPE_OK) return rc;
    return done(launch_route_scores_backward(*d, dw, d_logits, sms, (cudaStream_t)stream));
}

size_t pmpe_clip_workspace_size(int n) { return n < 0 || n > kMaxRows ? 0 : clip_workspace_bytes(n); }

int pmpe_clip_grad_norm(const pmpe_grad *grads, int n, float max_norm, float *norm, void *workspace, size_t workspace_bytes,
                        void *stream)
{
    if (n < 0 || (n > 0 && !grads) || !(max_norm >= 0.f) || !norm) return PMPE_ERR_INVALID_ARG;
    if (n > kMaxRows) return PMPE_ERR_UNSUPPORTED_SHAPE;
    for (int i = 0; i < n; ++i) {
        const pmpe_grad &g = grads[i];
        if (g.n < 0 || !is_type(g.type) || (g.n > 0 && !g.grad)) return PMPE_ERR_INVALID_ARG;
        if (g.n > ((int64_t)1 << 44)) return PMPE_ERR_UNSUPPORTED_SHAPE;
        if (!fits(g.grad, g.type) || !fits(g.out, g.type)) return PMPE_ERR_UNSUPPORTED_SHAPE;
    }
    if (!fits4(norm)) return PMPE_ERR_UNSUPPORTED_SHAPE;
    const int ok = clip_tensors_ok(grads, n);
    if (ok <= 0) return ok < 0 ? PMPE_ERR_WORKSPACE : PMPE_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 15u) || workspace_bytes < clip_workspace_bytes(n)) return PMPE_ERR_WORKSPACE;
    return done(launch_clip(grads, n, max_norm, norm, workspace, (cudaStream_t)stream));
}

}  // extern "C"
