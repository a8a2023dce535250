// A layer's input activations in 8 bits and back (the format: act8.cuh).
//
// Both directions move bytes and little else: the bound is HBM.  A lane takes eight neighbouring channels (one 16-byte load or store of bf16), four
// lanes share a scale.  `lanes` threads, a power of two from 4 to 256, walk over a row, so that neither narrow rows leave lanes idle nor few
// rows SMs.
#include "act8.cuh"
#include "gaconv_internal.h"

namespace gaconv {
namespace {

constexpr int kBlock = 256;

struct RowsOp {
    long long rows, stride;     // of the plain tensor, elements
    int cols, pitch, groups;    // channels; bytes and scales of a row of the 8-bit form
    int log_lanes;              // threads of a row
};

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kBlock)
act_pack_kernel(const T* x, uint8_t* codes, uint8_t* scales, const RowsOp o)
{
    pdl_release_next_grid();
    const int lanes = 1 << o.log_lanes, l = threadIdx.x & (lanes - 1);
    const long long row = (long long)blockIdx.x * (kBlock >> o.log_lanes) + (threadIdx.x >> o.log_lanes);
    const bool live = row < o.rows;
    const T* src = x + (live ? row : 0) * o.stride;
    uint8_t* dst = codes + (live ? row : 0) * o.pitch;
    uint8_t* sc = scales + (live ? row : 0) * o.groups;
    pdl_wait_prior_grid();
    const int units = 4 * o.groups;         // (every lane of a warp walks as often: shuffles are warp-wide)
    for (int u0 = 0; u0 < units; u0 += 4 * lanes) {
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = u0 + i * lanes + l;
            load8<VEC>(src + 8 * u, live ? o.cols - 8 * u : 0, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = u0 + i * lanes + l;
            if (u0 + i * lanes >= units) break;
            act_store8<FMT>(v[i], dst + 8 * u, live ? o.pitch - 8 * u : 0, sc + (u >> 2), (u & 3) == 0);
        }
    }
}

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kBlock)
act_unpack_kernel(const uint8_t* codes, const uint8_t* scales, T* x, const RowsOp o)
{
    pdl_release_next_grid();
    const int lanes = 1 << o.log_lanes, l = threadIdx.x & (lanes - 1);
    const long long row = (long long)blockIdx.x * (kBlock >> o.log_lanes) + (threadIdx.x >> o.log_lanes);
    if (row >= o.rows) return;
    const uint8_t* src = codes + row * o.pitch;
    const uint8_t* sc = scales + row * o.groups;
    T* dst = x + row * o.stride;
    pdl_wait_prior_grid();
    const int units = (o.cols + 7) >> 3;
    for (int u0 = l; u0 < units; u0 += 4 * lanes) {
        uint2 q[4];
        uint32_t s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = u0 + i * lanes;
            if (u < units) { q[i] = *reinterpret_cast<const uint2*>(src + 8 * u); s[i] = sc[u >> 2]; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = u0 + i * lanes;
            if (u >= units) break;
            const uint4 d = act_decode8<FMT>(q[i], s[i]);
            const uint32_t w[4] = {d.x, d.y, d.z, d.w};
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
            store8<VEC>(dst + 8 * u, o.cols - 8 * u, v);
        }
    }
}

RowsOp rows_op(const ActRows& a)
{
    RowsOp o;
    o.rows = a.rows; o.stride = a.stride; o.cols = a.cols; o.pitch = act_pitch(a.cols); o.groups = act_groups(a.cols);
    o.log_lanes = 2;
    while (o.log_lanes < 8 && (1 << o.log_lanes) < 4 * o.groups && ((1 << o.log_lanes) < o.groups || a.rows << o.log_lanes < 148 * 1024)) ++o.log_lanes;
    return o;
}
unsigned row_blocks(const RowsOp& o) { return (unsigned)((o.rows + (kBlock >> o.log_lanes) - 1) / (kBlock >> o.log_lanes)); }

template <typename T, int FMT>
cudaError_t pack(const T* x, uint8_t* codes, uint8_t* scales, const RowsOp& o, cudaStream_t stream)
{
    auto kern = o.stride % (16 / (int)sizeof(T)) == 0 ? act_pack_kernel<T, FMT, true> : act_pack_kernel<T, FMT, false>;
    return launch_kernel(kern, dim3(row_blocks(o)), dim3(kBlock), 0, stream, dim3(1, 1, 1), x, codes, scales, o);
}
template <typename T, int FMT>
cudaError_t unpack(const uint8_t* codes, const uint8_t* scales, T* x, const RowsOp& o, cudaStream_t stream)
{
    auto kern = o.stride % (16 / (int)sizeof(T)) == 0 ? act_unpack_kernel<T, FMT, true> : act_unpack_kernel<T, FMT, false>;
    return launch_kernel(kern, dim3(row_blocks(o)), dim3(kBlock), 0, stream, dim3(1, 1, 1), codes, scales, x, o);
}

}  // namespace

cudaError_t launch_act_pack(const void* x, void* codes, void* scales, const ActRows& a, cudaStream_t stream)
{
    const RowsOp o = rows_op(a);
    uint8_t *q = static_cast<uint8_t*>(codes), *s = static_cast<uint8_t*>(scales);
    note_launch();
    if (a.bf16) {
        const auto* p = static_cast<const __nv_bfloat16*>(x);
        return a.format == GACONV_ACT_E4M3 ? pack<__nv_bfloat16, GACONV_ACT_E4M3>(p, q, s, o, stream) : pack<__nv_bfloat16, GACONV_ACT_INT8>(p, q, s, o, stream);
    }
    const auto* p = static_cast<const float*>(x);
    return a.format == GACONV_ACT_E4M3 ? pack<float, GACONV_ACT_E4M3>(p, q, s, o, stream) : pack<float, GACONV_ACT_INT8>(p, q, s, o, stream);
}

cudaError_t launch_act_unpack(const void* codes, const void* scales, void* x, const ActRows& a, cudaStream_t stream)
{
    const RowsOp o = rows_op(a);
    const uint8_t *q = static_cast<const uint8_t*>(codes), *s = static_cast<const uint8_t*>(scales);
    note_launch();
    if (a.bf16) {
        auto* p = static_cast<__nv_bfloat16*>(x);
        return a.format == GACONV_ACT_E4M3 ? unpack<__nv_bfloat16, GACONV_ACT_E4M3>(q, s, p, o, stream) : unpack<__nv_bfloat16, GACONV_ACT_INT8>(q, s, p, o, stream);
    }
    auto* p = static_cast<float*>(x);
    return a.format == GACONV_ACT_E4M3 ? unpack<float, GACONV_ACT_E4M3>(q, s, p, o, stream) : unpack<float, GACONV_ACT_INT8>(q, s, p, o, stream);
}

}  // namespace gaconv
