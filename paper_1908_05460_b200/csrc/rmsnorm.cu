// Root-mean-square norm behind the addition of the residual, with its output in 8 bits as well, and its backward pass.
//
//   forward    s = x + r (rounded to the type),  rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd w (rounded once),  codes, scales = y in 8 bits (act8.cuh)
//   backward   h = s rstd,  g = dy w,  dx = ds + rstd (g - h mean(g h)),  dw = sum over rows of dy h
//
// Bound by HBM: every tensor is read and written once.  A team of `lanes` threads holds a row in registers, `NU` pieces of eight channels a
// thread, so that the second use of a row (after its mean) reads nothing.  Sums and means are fp32, in an order that depends on the sizes alone.
#include <algorithm>
#include <type_traits>

#include "act8.cuh"
#include "device_utils.cuh"
#include "gaconv_internal.h"

namespace gaconv {
namespace {

// Sum over the threads of a team, the same bits in each.  `part`: two rows of one float a warp, taken in turn so that one barrier a sum is enough.
__device__ __forceinline__ float team_sum(float v, int log_lanes, float (*part)[16], int& turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (log_lanes > 5) {
        const int warp = threadIdx.x >> 5, team = threadIdx.x >> log_lanes, n = 1 << (log_lanes - 5), first = team << (log_lanes - 5);
        if ((threadIdx.x & 31) == 0) part[turn][warp] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(1 << log_lanes) : "memory");
        v = 0.f;
        for (int i = 0; i < n; ++i) v += part[turn][first + i];
        turn ^= 1;
    }
    return v;
}

template <typename T> __device__ __forceinline__ float act_type_round(float v) { return rounded(v, static_cast<const T*>(nullptr)); }

__device__ __forceinline__ void store_codes(const NormRows& o, const float (&t)[8], uint8_t* codes, uint8_t* scales, long long r, int c, int pitch_left)
{
    uint8_t *q = codes + r * o.pitch + c, *s = scales + r * o.groups + (c >> 5);
    if (o.format == GACONV_ACT_E4M3) act_store8<GACONV_ACT_E4M3>(t, q, pitch_left, s, (c & 31) == 0);
    else act_store8<GACONV_ACT_INT8>(t, q, pitch_left, s, (c & 31) == 0);
}

template <typename T, int NU, bool VEC>
__global__ void __launch_bounds__(512)
rmsnorm_forward_kernel(const NormRows o, const T* x, const T* res, const T* __restrict__ w, T* sum, T* y, uint8_t* codes, uint8_t* scales, float* rstd, int log_lanes)
{
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const int lanes = 1 << log_lanes, l = threadIdx.x & (lanes - 1);
    const long long row = (long long)blockIdx.x * (blockDim.x >> log_lanes) + (threadIdx.x >> log_lanes);
    const bool live = row < o.rows;          // (teams without a row go along: shuffles and barriers are shared)
    const long long r = live ? row : 0;
    const int cols = live ? o.cols : 0;
    int turn = 0;
    pdl_wait_prior_grid();
    float v[NU][8];
#pragma unroll
    for (int i = 0; i < NU; ++i) load8<VEC>(x + r * o.x_stride + 8 * (i * lanes + l), cols - 8 * (i * lanes + l), v[i]);
    if (res != nullptr) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            float t[8];
            load8<VEC>(res + r * o.r_stride + 8 * (i * lanes + l), cols - 8 * (i * lanes + l), t);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = act_type_round<T>(v[i][j] + t[j]);
        }
    }
    if (sum != nullptr) {
#pragma unroll
        for (int i = 0; i < NU; ++i) store8<VEC>(sum + r * o.s_stride + 8 * (i * lanes + l), cols - 8 * (i * lanes + l), v[i]);
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) q = fmaf(v[i][j], v[i][j], q);
    q = team_sum(q, log_lanes, part, turn);
    const float rs = 1.f / sqrtf(q / (float)o.cols + o.eps);
    if (live && l == 0 && rstd != nullptr) rstd[r] = rs;
    const int pitch = live ? o.pitch : 0;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
        const int c = 8 * (i * lanes + l);
        float t[8];
        load8<true>(w + c, o.cols - c, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = act_type_round<T>(v[i][j] * rs * t[j]);
        if (y != nullptr) store8<VEC>(y + r * o.y_stride + c, cols - c, t);
        if (codes != nullptr) store_codes(o, t, codes, scales, r, c, pitch - c);
    }
}

// Rows longer than a team's registers: a block a row, which it reads twice (the second time from L2 or, of very long rows, from memory).
template <typename T, bool VEC>
__global__ void __launch_bounds__(512)
rmsnorm_forward_long_kernel(const NormRows o, const T* x, const T* res, const T* __restrict__ w, T* sum, T* y, uint8_t* codes, uint8_t* scales, float* rstd)
{
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const long long r = blockIdx.x;
    const T *xr = x + r * o.x_stride, *rr = res + (res != nullptr ? r * o.r_stride : 0);
    T* sr = sum + (sum != nullptr ? r * o.s_stride : 0);
    int turn = 0;
    float q = 0.f;
    pdl_wait_prior_grid();
    for (int c = 8 * threadIdx.x; c < o.cols; c += 4096) {
        float v[8], t[8];
        load8<VEC>(xr + c, o.cols - c, v);
        if (res != nullptr) {
            load8<VEC>(rr + c, o.cols - c, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = act_type_round<T>(v[j] + t[j]);
        }
        if (sum != nullptr) store8<VEC>(sr + c, o.cols - c, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) q = fmaf(v[j], v[j], q);
    }
    q = team_sum(q, 9, part, turn);
    const float rs = 1.f / sqrtf(q / (float)o.cols + o.eps);
    if (threadIdx.x == 0 && rstd != nullptr) rstd[r] = rs;
    const T* again = sum != nullptr ? sr : xr;         // (what this thread has written itself)
    for (int c0 = 0; c0 < o.cols; c0 += 4096) {
        const int c = c0 + 8 * threadIdx.x;
        float v[8], t[8];
        load8<VEC>(again + c, o.cols - c, v);
        load8<true>(w + c, o.cols - c, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = act_type_round<T>(v[j] * rs * t[j]);
        if (y != nullptr) store8<VEC>(y + r * o.y_stride + c, o.cols - c, t);
        if (codes != nullptr) store_codes(o, t, codes, scales, r, c, o.pitch - c);
    }
}

// Backward.  A block stays and its teams take rows in turn; a thread keeps the sums over rows of dy h for its channels, which the
// teams of a block add up in order at the end: partial[block][cols].
template <typename T, int NU, bool VEC>
__global__ void __launch_bounds__(512)
rmsnorm_backward_kernel(const NormRows o, const T* dy, const T* ds, const T* s, const T* __restrict__ w, const float* __restrict__ rstd, T* dx, float* __restrict__ partial, int log_lanes)
{
    extern __shared__ float s_dw[];
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const int lanes = 1 << log_lanes, l = threadIdx.x & (lanes - 1), team = threadIdx.x >> log_lanes, teams = blockDim.x >> log_lanes;
    float acc[NU][8];
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    int turn = 0;
    pdl_wait_prior_grid();
    const long long step = (long long)gridDim.x * teams;
    for (long long row = (long long)blockIdx.x * teams + team; row < o.rows; row += step) {
        float g[NU][8], h[NU][8];
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = 8 * (i * lanes + l);
            load8<VEC>(dy + row * o.y_stride + c, o.cols - c, g[i]);
            load8<VEC>(s + row * o.s_stride + c, o.cols - c, h[i]);
        }
        const float rs = rstd[row];
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = 8 * (i * lanes + l);
            float t[8];
            load8<true>(w + c, o.cols - c, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] *= rs;
                acc[i][j] = fmaf(g[i][j], h[i][j], acc[i][j]);
                g[i][j] *= t[j];
                dot = fmaf(g[i][j], h[i][j], dot);
            }
        }
        dot = team_sum(dot, log_lanes, part, turn) / (float)o.cols;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = 8 * (i * lanes + l);
            float t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = 0.f;
            if (ds != nullptr) load8<VEC>(ds + row * o.s_stride + c, o.cols - c, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = fmaf(rs, g[i][j] - h[i][j] * dot, t[j]);
            store8<VEC>(dx + row * o.x_stride + c, o.cols - c, t);
        }
    }
    if (partial == nullptr) return;
    float* out = partial + (size_t)blockIdx.x * o.cols;
    for (int t = 0; t < teams; ++t) {
        if (team == t) {
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int c = 8 * (i * lanes + l);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float v = t == 0 ? acc[i][j] : s_dw[c + j] + acc[i][j];
                    if (t + 1 < teams) s_dw[c + j] = v;
                    else if (c + j < o.cols) out[c + j] = v;
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(512)
rmsnorm_backward_long_kernel(const NormRows o, const T* dy, const T* ds, const T* s, const T* __restrict__ w, const float* __restrict__ rstd, T* dx)
{
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const long long row = blockIdx.x;
    int turn = 0;
    float dot = 0.f;
    pdl_wait_prior_grid();
    const float rs = rstd[row];
    for (int pass = 0; pass < 2; ++pass) {
        for (int c = 8 * threadIdx.x; c < o.cols; c += 4096) {
            float g[8], h[8], t[8];
            load8<VEC>(dy + row * o.y_stride + c, o.cols - c, g);
            load8<VEC>(s + row * o.s_stride + c, o.cols - c, h);
            load8<true>(w + c, o.cols - c, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) { g[j] *= t[j]; h[j] *= rs; }
            if (pass == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) dot = fmaf(g[j], h[j], dot);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = 0.f;
                if (ds != nullptr) load8<VEC>(ds + row * o.s_stride + c, o.cols - c, t);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = fmaf(rs, g[j] - h[j] * dot, t[j]);
                store8<VEC>(dx + row * o.x_stride + c, o.cols - c, t);
            }
        }
        if (pass == 0) dot = team_sum(dot, 9, part, turn) / (float)o.cols;
    }
}
// sums over a range of rows, a thread a channel: grid (channels / 256, ranges)
template <typename T>
__global__ void __launch_bounds__(256)
rmsnorm_weight_long_kernel(const NormRows o, const T* dy, const T* s, const float* __restrict__ rstd, float* __restrict__ partial)
{
    pdl_release_next_grid();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= o.cols) return;
    const long long per = (o.rows + gridDim.y - 1) / gridDim.y, first = blockIdx.y * per, last = min(first + per, o.rows);
    float acc = 0.f;
    pdl_wait_prior_grid();
#pragma unroll 4
    for (long long r = first; r < last; ++r) acc = fmaf(ldf(dy + r * o.y_stride + c), ldf(s + r * o.s_stride + c) * __ldg(rstd + r), acc);
    partial[(size_t)blockIdx.y * o.cols + c] = acc;
}

// ---------------------------------------------------------------- host side
constexpr int kMaxCols = 512 * 4 * 8;          // channels that a team's registers hold

struct Team { int log_lanes, nu; };
// threads of a row: four pieces each, or fewer where that leaves SMs without work
Team team_of(const NormRows& o)
{
    const int units = (o.cols + 7) / 8;
    Team t{5, 0};
    while (t.log_lanes < 9 && 4 << t.log_lanes < units) ++t.log_lanes;
    while (t.log_lanes < 9 && 1 << t.log_lanes < units && o.rows << t.log_lanes < 148 * 512) ++t.log_lanes;
    const int per = (units + (1 << t.log_lanes) - 1) >> t.log_lanes;
    t.nu = per <= 1 ? 1 : per <= 2 ? 2 : 4;
    return t;
}
bool vectors(const NormRows& o, int elem, long long a, long long b, long long c, long long d)
{
    const int n = 16 / elem;
    return a % n == 0 && b % n == 0 && c % n == 0 && d % n == 0;
}
int backward_blocks(const NormRows& o, const Team& t, int threads)
{
    const long long teams = threads >> t.log_lanes, need = (o.rows + teams - 1) / teams;
    return (int)std::min<long long>(need, device_sms() * (1024 / threads));
}
constexpr int kBackwardThreads = 512;

template <typename T>
cudaError_t forward(const NormRows& o, const T* x, const T* res, const T* w, T* sum, T* y, uint8_t* codes, uint8_t* scales, float* rstd, cudaStream_t stream)
{
    const bool vec = vectors(o, sizeof(T), o.x_stride, res ? o.r_stride : 0, sum ? o.s_stride : 0, y ? o.y_stride : 0);
    note_launch();
    if (o.cols > kMaxCols) {
        auto kern = vec ? rmsnorm_forward_long_kernel<T, true> : rmsnorm_forward_long_kernel<T, false>;
        return launch_kernel(kern, dim3((unsigned)o.rows), dim3(512), 0, stream, dim3(1, 1, 1), o, x, res, w, sum, y, codes, scales, rstd);
    }
    const Team t = team_of(o);
    const int threads = std::max(128, 1 << t.log_lanes), teams = threads >> t.log_lanes;
    auto kern = t.nu == 1 ? (vec ? rmsnorm_forward_kernel<T, 1, true> : rmsnorm_forward_kernel<T, 1, false>)
              : t.nu == 2 ? (vec ? rmsnorm_forward_kernel<T, 2, true> : rmsnorm_forward_kernel<T, 2, false>)
                          : (vec ? rmsnorm_forward_kernel<T, 4, true> : rmsnorm_forward_kernel<T, 4, false>);
    return launch_kernel(kern, dim3((unsigned)((o.rows + teams - 1) / teams)), dim3(threads), 0, stream, dim3(1, 1, 1), o, x, res, w, sum, y, codes, scales, rstd, t.log_lanes);
}

template <typename T>
cudaError_t backward(const NormRows& o, const T* dy, const T* ds, const T* s, const T* w, const float* rstd, T* dx, float* dweight, float* partial, cudaStream_t stream)
{
    const bool vec = vectors(o, sizeof(T), o.y_stride, o.s_stride, o.x_stride, 0);
    cudaError_t err;
    int splits;
    note_launch();
    if (o.cols > kMaxCols) {
        if (dweight != nullptr) {
            splits = norm_partials(o);
            err = launch_kernel(rmsnorm_weight_long_kernel<T>, dim3((unsigned)((o.cols + 255) / 256), (unsigned)splits), dim3(256), 0, stream, dim3(1, 1, 1), o, dy, s, rstd, partial);
            if (err != cudaSuccess) return err;
            note_launch();
        }
        auto kern = vec ? rmsnorm_backward_long_kernel<T, true> : rmsnorm_backward_long_kernel<T, false>;
        err = launch_kernel(kern, dim3((unsigned)o.rows), dim3(512), 0, stream, dim3(1, 1, 1), o, dy, ds, s, w, rstd, dx);
    } else {
        const Team t = team_of(o);
        splits = backward_blocks(o, t, kBackwardThreads);
        auto kern = t.nu == 1 ? (vec ? rmsnorm_backward_kernel<T, 1, true> : rmsnorm_backward_kernel<T, 1, false>)
                  : t.nu == 2 ? (vec ? rmsnorm_backward_kernel<T, 2, true> : rmsnorm_backward_kernel<T, 2, false>)
                              : (vec ? rmsnorm_backward_kernel<T, 4, true> : rmsnorm_backward_kernel<T, 4, false>);
        const size_t smem = kBackwardThreads >> t.log_lanes > 1 ? (size_t)t.nu * 32 << t.log_lanes : 0;      // (at most 32 KB)
        err = launch_kernel(kern, dim3((unsigned)splits), dim3(kBackwardThreads), smem, stream, dim3(1, 1, 1), o, dy, ds, s, w, rstd, dx, dweight != nullptr ? partial : nullptr, t.log_lanes);
    }
    if (err != cudaSuccess || dweight == nullptr) return err;
    return reduce_splits(partial, dweight, (size_t)o.cols, splits, 1.f, stream);
}

}  // namespace

// rows of `cols` sums that the backward pass leaves in the workspace
int norm_partials(const NormRows& o)
{
    if (o.rows == 0) return 0;
    if (o.cols <= kMaxCols) return backward_blocks(o, team_of(o), kBackwardThreads);
    return (int)std::min<long long>((o.rows + 31) / 32, 64);
}

cudaError_t launch_rmsnorm_forward(const NormRows& o, const void* x, const void* res, const void* w, void* sum, void* y, void* codes, void* scales, float* rstd, cudaStream_t stream)
{
    if (o.rows == 0) return cudaSuccess;
    auto run = [&](auto* type) {
        typedef typename std::remove_pointer<decltype(type)>::type T;
        return forward<T>(o, static_cast<const T*>(x), static_cast<const T*>(res), static_cast<const T*>(w), static_cast<T*>(sum), static_cast<T*>(y),
                          static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales), rstd, stream);
    };
    return o.bf16 ? run(static_cast<__nv_bfloat16*>(nullptr)) : run(static_cast<float*>(nullptr));
}

cudaError_t launch_rmsnorm_backward(const NormRows& o, const void* dy, const void* ds, const void* s, const void* w, const float* rstd, void* dx, float* dweight, float* partial, cudaStream_t stream)
{
    if (o.rows == 0) return dweight != nullptr ? launch_zero(dweight, (size_t)o.cols, stream) : cudaSuccess;
    auto run = [&](auto* type) {
        typedef typename std::remove_pointer<decltype(type)>::type T;
        return backward<T>(o, static_cast<const T*>(dy), static_cast<const T*>(ds), static_cast<const T*>(s), static_cast<const T*>(w), rstd, static_cast<T*>(dx), dweight, partial, stream);
    };
    return o.bf16 ? run(static_cast<__nv_bfloat16*>(nullptr)) : run(static_cast<float*>(nullptr));
}

}  // namespace gaconv
