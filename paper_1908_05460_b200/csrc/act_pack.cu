// A layer's input activations in 8 bits and back (the format: act8.cuh).
//
// Both directions move bytes and little else: the bound is HBM.  A lane takes 16 bytes of a row (rows.cuh), 4 lanes (bf16) or 8 (fp32) share a scale.
// `lanes` threads, a power of two from 8 to 256, walk over a row, so that neither narrow rows leave lanes idle nor few rows SMs; each has the
// loads of kAhead pieces in flight.
#include "act8.cuh"
#include "gaconv_internal.h"
#include "rows.cuh"

namespace gaconv {
namespace {

constexpr int kBlock = 256, kAhead = 4;

struct RowsOp {
    long long rows, stride;     // of the plain tensor, elements
    int cols, pitch, groups;    // channels; bytes and scales of a row of the 8-bit form
    int log_lanes;              // threads of a row
};

template <typename T, int FMT, bool FULL>
__global__ void __launch_bounds__(kBlock)
act_pack_kernel(const T* x, uint8_t* codes, uint8_t* scales, const RowsOp o)
{
    constexpr int N = kPiece<T>;
    pdl_release_next_grid();
    const int lanes = 1 << o.log_lanes, l = threadIdx.x & (lanes - 1);
    const long long row = (long long)blockIdx.x * (kBlock >> o.log_lanes) + (threadIdx.x >> o.log_lanes), r = row < o.rows ? row : 0;
    const int pitch = row < o.rows ? o.pitch : 0;
    const Row<T, FULL> src(x, r, o.stride, o.rows, o.cols, row < o.rows);
    uint8_t* dst = codes + r * o.pitch;
    uint8_t* sc = scales + r * o.groups;
    pdl_wait_prior_grid();
    const int pieces = 32 / N * o.groups;         // (every lane of a warp walks as often: shuffles are warp-wide)
    for (int u0 = 0; u0 < pieces; u0 += kAhead * lanes) {
        Piece<T, FULL> p[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = (u0 + i * lanes + l) * N;
            p[i].start(src, c);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = (u0 + i * lanes + l) * N;
            if (u0 + i * lanes >= pieces) break;
            float v[N];
            to_floats<T>(p[i].value(src, c), v);
            act_store<FMT, N>(v, dst + c, pitch - c, sc + (c >> 5), (c & 31) == 0);
        }
    }
}

template <typename T, int FMT, bool FULL>
__global__ void __launch_bounds__(kBlock)
act_unpack_kernel(const uint8_t* codes, const uint8_t* scales, T* x, const RowsOp o)
{
    constexpr int N = kPiece<T>;
    pdl_release_next_grid();
    const int lanes = 1 << o.log_lanes, l = threadIdx.x & (lanes - 1);
    const long long row = (long long)blockIdx.x * (kBlock >> o.log_lanes) + (threadIdx.x >> o.log_lanes), r = row < o.rows ? row : 0;
    const int cols = row < o.rows ? o.cols : 0;
    const uint8_t* src = codes + r * o.pitch;
    const uint8_t* sc = scales + r * o.groups;
    T* dst = x + r * o.stride;
    pdl_wait_prior_grid();
    const int pieces = (o.cols + N - 1) / N;
    for (int u0 = 0; u0 < pieces; u0 += kAhead * lanes) {
        uint32_t q[kAhead][N / 4], s[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = (u0 + i * lanes + l) * N;
            s[i] = 0;
#pragma unroll
            for (int j = 0; j < N / 4; ++j) q[i][j] = 0;
            if (c < cols) {
                if constexpr (N == 8) { const uint2 t = __ldg(reinterpret_cast<const uint2*>(src + c)); q[i][0] = t.x; q[i][1] = t.y; }
                else q[i][0] = __ldg(reinterpret_cast<const uint32_t*>(src + c));
                s[i] = __ldg(sc + (c >> 5));
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = (u0 + i * lanes + l) * N;
            if (u0 + i * lanes >= pieces) break;
            const uint32_t s2 = act_scale2<FMT>(s[i]);
            uint32_t w[N / 2];
#pragma unroll
            for (int j = 0; j < N / 4; ++j) {
                const uint2 d = act_decode4<FMT>(q[i][j], s2);
                w[2 * j] = d.x; w[2 * j + 1] = d.y;
            }
            if (act_has_rest<FMT>(s[i])) {
                const uint32_t rest = act_rest2(s[i]);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) w[j] = bf2_mul(w[j], rest);
            }
            uint4 v;
            if constexpr (N == 8) v = make_uint4(w[0], w[1], w[2], w[3]);
            else v = make_uint4(w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u);
            store_piece<T, FULL>(dst + c, cols - c, v, o.log_lanes);
        }
    }
}

// threads of a row: one a piece (at most a block), or, where there are rows enough, as few as a quarter of that: a thread then has the kAhead pieces whose loads it keeps in flight
RowsOp rows_op(const ActRows& a)
{
    RowsOp o;
    o.rows = a.rows; o.stride = a.stride; o.cols = a.cols; o.pitch = act_pitch(a.cols); o.groups = act_groups(a.cols);
    const int pieces = o.groups * (a.bf16 ? 4 : 8);
    o.log_lanes = 3;
    while (o.log_lanes < 8 && (1 << o.log_lanes) < pieces && ((kAhead << o.log_lanes) < pieces || a.rows << o.log_lanes < device_sms() * 1024ll)) ++o.log_lanes;
    return o;
}
unsigned row_blocks(const RowsOp& o) { return (unsigned)((o.rows + (kBlock >> o.log_lanes) - 1) / (kBlock >> o.log_lanes)); }

template <typename T, int FMT>
cudaError_t pack(const T* x, uint8_t* codes, uint8_t* scales, const RowsOp& o, cudaStream_t stream)
{
    auto kern = o.stride % kPiece<T> == 0 && o.cols % kPiece<T> == 0 ? act_pack_kernel<T, FMT, true> : act_pack_kernel<T, FMT, false>;
    return launch_kernel(kern, dim3(row_blocks(o)), dim3(kBlock), 0, stream, dim3(1, 1, 1), x, codes, scales, o);
}
template <typename T, int FMT>
cudaError_t unpack(const uint8_t* codes, const uint8_t* scales, T* x, const RowsOp& o, cudaStream_t stream)
{
    auto kern = o.stride % kPiece<T> == 0 && o.cols % kPiece<T> == 0 ? act_unpack_kernel<T, FMT, true> : act_unpack_kernel<T, FMT, false>;
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
