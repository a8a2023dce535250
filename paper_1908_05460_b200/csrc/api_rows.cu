// C-ABI entry points for rows of activations: their 8-bit form, filter gradients from it, and the root-mean-square norm.
#include <algorithm>
#include <cstring>
#include <mutex>

#include "gaconv_internal.h"

using namespace gaconv;

namespace {

// Checks a descriptor; strides of 0 become dense ones
gaconv_status_t check_rows(const gaconv_rows_desc_t* d, gaconv_rows_desc_t* out)
{
    if (d == nullptr) return GACONV_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(gaconv_rows_desc_t)) return GACONV_ERR_BAD_DESC;
    if (d->cols < 1 || d->rows < 0) return GACONV_ERR_BAD_DESC;
    if (d->dtype != GACONV_F32 && d->dtype != GACONV_BF16) return GACONV_ERR_BAD_DESC;
    if (d->format != GACONV_ACT_E4M3 && d->format != GACONV_ACT_INT8) return GACONV_ERR_BAD_DESC;
    if (!(d->eps >= 0.f)) return GACONV_ERR_BAD_DESC;
    *out = *d;
    for (int64_t* s : {&out->x_stride, &out->r_stride, &out->s_stride, &out->y_stride}) {
        if (*s == 0) *s = d->cols;
        if (*s < d->cols) return GACONV_ERR_BAD_DESC;
        if (*s > (1ll << 40) || (d->rows > 0 && *s > (1ll << 60) / d->rows)) return GACONV_ERR_UNSUPPORTED;       // (offsets stay below 2^63 bytes)
    }
    return d->rows > 0x7fffffffll || d->cols > (1 << 28) ? GACONV_ERR_UNSUPPORTED : GACONV_OK;
}

template <typename... P>
bool all_aligned16(const P*... p) { return (... && aligned16(p)); }

NormRows norm_rows(const gaconv_rows_desc_t& d)
{
    return NormRows{d.rows, d.x_stride, d.r_stride, d.s_stride, d.y_stride, d.cols, d.format, act_pitch(d.cols), act_groups(d.cols), d.eps, d.dtype == GACONV_BF16};
}
size_t norm_workspace(const NormRows& o) { return std::max<size_t>(256, align_up(sizeof(float) * (size_t)norm_partials(o) * o.cols, 256)); }

// Plan of a linear layer's filter gradient, the quicker of the two kernels' by their estimates.  Plans are kept, by what they depend on (2 us a call otherwise).
struct PlanEntry { long long key[10]; bool used, ok; PackedPlan plan; };
bool plan_linear(const Geom& g, bool npqk, bool tensor_only, PackedPlan* out)
{
    int dev = 0;
    cudaGetDevice(&dev);
    const long long key[10] = {g.n, (long long)g.p * g.q, g.c, g.k, npqk, tensor_only, g.bf16, g.sm_budget, dev,
                               g.r != 1 || g.s != 1 || g.stride_h != 1 || g.stride_w != 1 || g.pad_h != 0 || g.pad_w != 0};
    if (key[9]) return false;
    unsigned long long h = 0;
    for (long long v : key) h = (h ^ (unsigned long long)v) * 0x9E3779B97F4A7C15ull;
    static PlanEntry table[256];
    static std::mutex lock;
    PlanEntry& e = table[h >> 56];
    {
        std::lock_guard<std::mutex> held(lock);
        if (e.used && memcmp(e.key, key, sizeof(key)) == 0) { *out = e.plan; return e.ok; }
    }
    PlanEntry made{};
    memcpy(made.key, key, sizeof(key));
    double tensor = 0, fma = 0;
    PackedPlan other;
    made.used = true;
    made.ok = plan_packed(g, npqk, &made.plan, &tensor);
    if (!tensor_only && plan_packed_fma(g, npqk, &other, &fma) && (!made.ok || fma < tensor)) { made.plan = other; made.ok = true; }
    std::lock_guard<std::mutex> held(lock);
    e = made;
    *out = made.plan;
    return made.ok;
}

// Scratch of a filter gradient from the 8-bit form: the sums of the kernel for linear layers, or what the call on a plain X takes and X itself behind it
struct PackedLayout { size_t inner, total; bool reads, fused; PackedPlan plan; };
gaconv_status_t packed_layout(const gaconv_conv_desc_t* desc, int32_t method, Geom* g, PackedLayout* L)
{
    gaconv_status_t st = make_geom(desc, g);
    if (st != GACONV_OK) return st;
    if (desc->x_layout != GACONV_X_NHWC || (long long)g->n * g->h > 0x7fffffffll / g->w || g->c > (1 << 28)) return GACONV_ERR_UNSUPPORTED;
    L->fused = false;
    L->reads = method != GACONV_METHOD_ZERO && method != GACONV_METHOD_RANDOM;
    // (ALGO_DIRECT and the one-pass TF32 mode name kernels of the plain form)
    if (method == GACONV_METHOD_EXACT && desc->algo != GACONV_ALGO_DIRECT && desc->math == GACONV_MATH_DEFAULT)
        L->fused = plan_linear(*g, desc->dy_layout == GACONV_DY_NPQK, desc->algo == GACONV_ALGO_TENSOR, &L->plan);
    if (L->fused) { L->inner = 0; L->total = align_up(kWsDataOffset, 256) + L->plan.partial_bytes + L->plan.dy_bytes; return GACONV_OK; }
    if ((st = method_workspace(desc, method, kNoLimit, &L->inner)) != GACONV_OK) return st;
    L->inner = align_up(L->inner, 256);
    L->total = L->inner + (L->reads ? align_up((size_t)g->n * g->h * g->w * g->c * (g->bf16 ? 2 : 4), 256) : 0);
    return GACONV_OK;
}

}  // namespace

extern "C" {

gaconv_status_t gaconv_act_sizes(const gaconv_rows_desc_t* desc, size_t* codes_bytes, size_t* scales_bytes)
{
    gaconv_rows_desc_t d;
    const gaconv_status_t st = check_rows(desc, &d);
    if (st != GACONV_OK) return st;
    if (codes_bytes == nullptr || scales_bytes == nullptr) return GACONV_ERR_NULL_POINTER;
    *codes_bytes = (size_t)d.rows * act_pitch(d.cols);
    *scales_bytes = (size_t)d.rows * act_groups(d.cols);
    return GACONV_OK;
}

gaconv_status_t gaconv_act_pack(const void* x, void* codes, void* scales, const gaconv_rows_desc_t* desc, void* stream)
{
    gaconv_rows_desc_t d;
    const gaconv_status_t st = check_rows(desc, &d);
    if (st != GACONV_OK || d.rows == 0) return st;
    if (x == nullptr || codes == nullptr || scales == nullptr) return GACONV_ERR_NULL_POINTER;
    if (!all_aligned16(x, codes, scales)) return GACONV_ERR_MISALIGNED;
    const ActRows a{d.rows, d.x_stride, d.cols, d.format, d.dtype == GACONV_BF16};
    return launch_act_pack(x, codes, scales, a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? GACONV_OK : GACONV_ERR_CUDA;
}

gaconv_status_t gaconv_act_unpack(const void* codes, const void* scales, void* x, const gaconv_rows_desc_t* desc, void* stream)
{
    gaconv_rows_desc_t d;
    const gaconv_status_t st = check_rows(desc, &d);
    if (st != GACONV_OK || d.rows == 0) return st;
    if (x == nullptr || codes == nullptr || scales == nullptr) return GACONV_ERR_NULL_POINTER;
    if (!all_aligned16(x, codes, scales)) return GACONV_ERR_MISALIGNED;
    const ActRows a{d.rows, d.x_stride, d.cols, d.format, d.dtype == GACONV_BF16};
    return launch_act_unpack(codes, scales, x, a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? GACONV_OK : GACONV_ERR_CUDA;
}

gaconv_status_t gaconv_packed_workspace_size(const gaconv_conv_desc_t* desc, int32_t method, size_t* bytes)
{
    if (bytes == nullptr) return GACONV_ERR_NULL_POINTER;
    Geom g;
    PackedLayout L;
    const gaconv_status_t st = packed_layout(desc, method, &g, &L);
    if (st == GACONV_OK) *bytes = L.total;
    return st;
}

gaconv_status_t gaconv_dw_from_packed(int32_t method, const void* codes, const void* scales, int32_t format, const void* dy, float* dw,
                                      const gaconv_conv_desc_t* desc, uint64_t seed, void* stream)
{
    Geom g;
    PackedLayout L;
    gaconv_status_t st = packed_layout(desc, method, &g, &L);
    if (st != GACONV_OK) return st;
    if (format != GACONV_ACT_E4M3 && format != GACONV_ACT_INT8) return GACONV_ERR_BAD_DESC;
    if (!L.reads) return gaconv_dw_approx(method, nullptr, nullptr, dw, desc, seed, stream);
    if (codes == nullptr || scales == nullptr || dy == nullptr || dw == nullptr || desc->workspace == nullptr) return GACONV_ERR_NULL_POINTER;
    if (!all_aligned16(codes, scales, dy, dw, desc->workspace)) return GACONV_ERR_MISALIGNED;
    if (desc->math == GACONV_MATH_TF32 && g.bf16) return GACONV_ERR_BAD_DESC;
    if (desc->workspace_bytes < L.total) return GACONV_ERR_WORKSPACE_TOO_SMALL;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (L.fused) {
        char *ws = static_cast<char*>(desc->workspace), *partial = ws + align_up(kWsDataOffset, 256);
        float* sums = reinterpret_cast<float*>(align_up(reinterpret_cast<size_t>(partial), 256));          // (a workspace starts on 16 bytes; the plans have room)
        const cudaError_t err = L.plan.fma ? launch_packed_fma(codes, scales, format, dy, dw, sums, g, desc->dy_layout == GACONV_DY_NPQK, L.plan, cs)
                                           : launch_packed(codes, scales, format, dy, dw, sums, partial + L.plan.partial_bytes, reinterpret_cast<uint32_t*>(ws), g, L.plan, cs);
        return err == cudaSuccess ? GACONV_OK : GACONV_ERR_CUDA;
    }
    gaconv_conv_desc_t inner = *desc;
    inner.workspace_bytes = L.inner;
    void* x = static_cast<char*>(desc->workspace) + L.inner;
    const ActRows a{(long long)g.n * g.h * g.w, g.c, g.c, format, g.bf16};
    if (launch_act_unpack(codes, scales, x, a, cs) != cudaSuccess) return GACONV_ERR_CUDA;
    return method == GACONV_METHOD_EXACT ? gaconv_dw_exact(x, dy, dw, &inner, stream) : gaconv_dw_approx(method, x, dy, dw, &inner, seed, stream);
}

gaconv_status_t gaconv_rmsnorm_forward(const void* x, const void* residual, const void* weight, void* sum, void* y, void* codes, void* scales, float* rstd,
                                       const gaconv_rows_desc_t* desc, void* stream)
{
    gaconv_rows_desc_t d;
    const gaconv_status_t st = check_rows(desc, &d);
    if (st != GACONV_OK || d.rows == 0) return st;
    if (x == nullptr || weight == nullptr || (residual != nullptr && sum == nullptr) || (codes == nullptr) != (scales == nullptr) || (y == nullptr && codes == nullptr))
        return GACONV_ERR_NULL_POINTER;
    if (!all_aligned16(x, residual, weight, sum, y, codes, scales, rstd)) return GACONV_ERR_MISALIGNED;
    return launch_rmsnorm_forward(norm_rows(d), x, residual, weight, sum, y, codes, scales, rstd, static_cast<cudaStream_t>(stream)) == cudaSuccess ? GACONV_OK : GACONV_ERR_CUDA;
}

gaconv_status_t gaconv_rmsnorm_workspace_size(const gaconv_rows_desc_t* desc, size_t* bytes)
{
    gaconv_rows_desc_t d;
    const gaconv_status_t st = check_rows(desc, &d);
    if (st != GACONV_OK) return st;
    if (bytes == nullptr) return GACONV_ERR_NULL_POINTER;
    *bytes = norm_workspace(norm_rows(d));
    return GACONV_OK;
}

gaconv_status_t gaconv_rmsnorm_backward(const void* dy, const void* dsum, const void* sum, const void* weight, const float* rstd, void* dx, float* dweight,
                                        const gaconv_rows_desc_t* desc, void* workspace, size_t workspace_bytes, void* stream)
{
    gaconv_rows_desc_t d;
    const gaconv_status_t st = check_rows(desc, &d);
    if (st != GACONV_OK) return st;
    const NormRows o = norm_rows(d);
    if (d.rows > 0 && (dy == nullptr || sum == nullptr || weight == nullptr || rstd == nullptr || dx == nullptr || (dweight != nullptr && workspace == nullptr)))
        return GACONV_ERR_NULL_POINTER;
    if (!all_aligned16(dy, dsum, sum, weight, rstd, dx, dweight, workspace)) return GACONV_ERR_MISALIGNED;
    if (d.rows > 0 && dweight != nullptr && workspace_bytes < norm_workspace(o)) return GACONV_ERR_WORKSPACE_TOO_SMALL;
    return launch_rmsnorm_backward(o, dy, dsum, sum, weight, rstd, dx, dweight, static_cast<float*>(workspace), static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? GACONV_OK : GACONV_ERR_CUDA;
}

}  // extern "C"
