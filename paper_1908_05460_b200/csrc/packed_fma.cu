// Filter gradient of a linear layer with X in 8 bits on the FP32 pipes, for problems whose products are few: a launch, or two where rows are split,
// that reads dY as it lies, whatever its type, order and alignment.
//
//   dW[k, c] = alpha * sum over rows t of dY[t, k] * code[t, c] * 2^e[t, c / 32]
//
// The tensor-core kernel (packed_dw.cu) takes 5 to 7 us however small the problem is, and gradients that the copy engine cannot read cost it a packing
// pass before.  Here a block of 256 threads takes TK x TC elements, 4 x 4 a thread, and its share of the rows through shared memory as fp32
// numbers, 32 or 64 rows at a time; the next are on their way in registers meanwhile.  Small tiles leave threads over, which then share the rows
// between them in G groups.  Bound by latency, then by the FP32 pipes.
#include <algorithm>
#include <cstring>

#include "act8.cuh"
#include "device_utils.cuh"
#include "gaconv_internal.h"

namespace gaconv {
namespace {

struct FmaParams {
    const uint8_t *codes, *scales;
    const void* dy;
    float* out;                     // dW, or the sums of a split [split][K * C], in dW's order
    long long out_split, ws_k, ws_c;
    int rows, c, k, pitch, groups, px;       // px: pixels of an image, where dY has them innermost (1: channels last)
    int per_split;                  // rows of a split
    float alpha;
};

template <int TK, int TC> constexpr int kChunk = TK * TC >= 4096 ? 32 : 64;          // rows in shared memory

template <typename T, int FMT, int TK, int TC>
__global__ void __launch_bounds__(256)
packed_fma_kernel(const __grid_constant__ FmaParams P)
{
    constexpr int CH = kChunk<TK, TC>, G = 4096 / (TK * TC), PER = 256 / G;          // rows at a time, groups, threads of a group
    constexpr int ND = TK * CH / 256, NX = TC * CH / 1024;                             // elements of dY, and words of codes, that a thread loads
    __shared__ __align__(16) float s_dy[CH][TK], s_x[CH][TC];
    __shared__ __align__(16) float s_sum[G > 1 ? (G - 1) * PER * 16 : 4];
    pdl_release_next_grid();
    const int t = threadIdx.x, k0 = blockIdx.x * TK, c0 = blockIdx.y * TC;
    const int first = blockIdx.z * P.per_split, last = min(P.rows, first + P.per_split);
    const int u = t % PER, group = t / PER, ck = 4 * (u / (TC / 4)), cc = 4 * (u % (TC / 4));
    const T* dy = static_cast<const T*>(P.dy);
    float vd[ND];
    uint32_t vx[NX], vs[NX];
    auto load = [&](int row0) {
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int e = t + 256 * i, row = row0 + e / TK, k = k0 + e % TK;
            vd[i] = 0.f;
            if (row < last && k < P.k) {
                long long at = (long long)row * P.k + k;
                if (P.px > 1) { const int n = row / P.px; at = ((long long)n * P.k + k) * P.px + (row - n * P.px); }
                vd[i] = ldf(dy + at);
            }
        }
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int e = t + 256 * i, row = row0 + e / (TC / 4), c = c0 + 4 * (e % (TC / 4));
            vx[i] = 0; vs[i] = 127;
            if (row < last && c < P.pitch) {
                vx[i] = __ldg(reinterpret_cast<const uint32_t*>(P.codes + (long long)row * P.pitch + c));
                vs[i] = __ldg(P.scales + (long long)row * P.groups + (c >> 5));
            }
        }
    };
    auto store = [&] {
#pragma unroll
        for (int i = 0; i < ND; ++i) s_dy[(t + 256 * i) / TK][(t + 256 * i) % TK] = vd[i];
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int e = t + 256 * i;
            uint2 d = act_decode4<FMT>(vx[i], act_scale2<FMT>(vs[i]));
            if (act_has_rest<FMT>(vs[i])) { const uint32_t r = act_rest2(vs[i]); d = make_uint2(bf2_mul(d.x, r), bf2_mul(d.y, r)); }
            *reinterpret_cast<float4*>(&s_x[e / (TC / 4)][4 * (e % (TC / 4))]) =
                make_float4(__uint_as_float(d.x << 16), __uint_as_float(d.x & 0xffff0000u), __uint_as_float(d.y << 16), __uint_as_float(d.y & 0xffff0000u));
        }
    };
    float acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
    pdl_wait_prior_grid();
    load(first);
    for (int row0 = first; row0 < last; row0 += CH) {
        if (row0 != first) __syncthreads();
        store();
        __syncthreads();
        if (row0 + CH < last) load(row0 + CH);
        const int n = min(CH, last - row0);
#pragma unroll 8
        for (int r = group; r < n; r += G) {
            const float4 a = *reinterpret_cast<const float4*>(&s_dy[r][ck]), b = *reinterpret_cast<const float4*>(&s_x[r][cc]);
            const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
        }
    }
    if (G > 1) {          // the groups' sums, in order
        float4* sums = reinterpret_cast<float4*>(s_sum);
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[(i * (G - 1) + group - 1) * PER + u] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
        }
        __syncthreads();
        if (group > 0) return;
        for (int q = 0; q < G - 1; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 v = sums[(i * (G - 1) + q) * PER + u];
                acc[i][0] += v.x; acc[i][1] += v.y; acc[i][2] += v.z; acc[i][3] += v.w;
            }
    }
    float* out = P.out + blockIdx.z * P.out_split;
    const int c = c0 + cc;
    const bool quads = P.ws_c == 1 && (P.ws_k & 3) == 0 && (P.out_split & 3) == 0 && c + 4 <= P.c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = k0 + ck + i;
        if (k >= P.k) break;
        float* at = out + k * P.ws_k + c * P.ws_c;
        if (quads) *reinterpret_cast<float4*>(at) = make_float4(P.alpha * acc[i][0], P.alpha * acc[i][1], P.alpha * acc[i][2], P.alpha * acc[i][3]);
        else {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (c + j < P.c) at[j * P.ws_c] = P.alpha * acc[i][j];
        }
    }
}

struct FmaHost { int tk, tc, splits, per_split; };
static_assert(sizeof(FmaHost) <= sizeof(((PackedPlan*)nullptr)->opaque), "opaque");

template <typename T, int FMT>
cudaError_t launch(const FmaHost& H, const FmaParams& P, cudaStream_t stream)
{
    auto kern = H.tk == 64 ? packed_fma_kernel<T, FMT, 64, 64> : H.tk == 32 ? packed_fma_kernel<T, FMT, 32, 32> : packed_fma_kernel<T, FMT, 16, 64>;
    const dim3 grid((unsigned)((P.k + H.tk - 1) / H.tk), (unsigned)((P.c + H.tc - 1) / H.tc), (unsigned)H.splits);
    return launch_kernel(kern, grid, dim3(256), 0, stream, dim3(1, 1, 1), P);
}

}  // namespace

// cycles: the estimate that plan_packed's is compared with.  (us, measured / estimated at 1.9 GHz, tiles of 16 x 64: 6 rows 769->18 2.3 / 2.3, 46 rows
// 1652->439 6.7 / 6.7, 128 rows 499->139 5.4 / 4.9, 2000 rows 300->100 in 16 splits 10.9 / 12.8, where the tensor cores take 10.5 and 10.4 are estimated;
// fp32 1000 rows 100->100 in 16 splits 5.1 / 6.2, there 10.8 / 14; fp32 100 rows 1000->1000 12.1 / 20, there 9.3 / 9.)
bool plan_packed_fma(const Geom& g, bool dy_npqk, PackedPlan* plan, double* cycles)
{
    if (g.r != 1 || g.s != 1 || g.stride_h != 1 || g.stride_w != 1 || g.pad_h != 0 || g.pad_w != 0) return false;
    const long long rows = (long long)g.n * g.p * g.q;
    if (rows > 0x7ff00000ll) return false;          // (a split's last row, rounded up, stays an int)
    const int sms = g.sm_budget > 0 ? std::min(g.sm_budget, device_sms()) : device_sms();
    FmaHost best{};
    double best_cost = 0;
    const int tiles[3][2] = {{16, 64}, {32, 32}, {64, 64}};
    for (const auto& t : tiles) {
        const int chunk = t[0] * t[1] >= 4096 ? kChunk<64, 64> : kChunk<32, 32>;
        const long long blocks = (long long)((g.k + t[0] - 1) / t[0]) * ((g.c + t[1] - 1) / t[1]);
        if ((g.k + t[0] - 1) / t[0] > 65535 || (g.c + t[1] - 1) / t[1] > 65535) continue;
        const long long chunks = (rows + chunk - 1) / chunk;
        for (int want = 0; want <= 4; want = want ? want * 2 : 1) {          // no split, or splits for so many blocks an SM
            const long long room = std::max<long long>(1, (long long)want * sms / blocks);
            const int splits = (int)std::min<long long>(std::min<long long>(chunks, room), 256);
            const long long per = (chunks + splits - 1) / splits;
            const int used = (int)((chunks + per - 1) / per);
            const double rounds = std::max(1.0, (double)blocks * used / (4.0 * sms)), busy = std::min(4.0, std::ceil((double)blocks * used / sms));
            // a chunk of a block alone on an SM, and what each of up to three others sharing it adds
            const double part = std::min(1.0, (double)rows / chunk), alone = 1600 + 1800 * part, shared = (400 + 1400 * part) * (chunk == 32 ? 2.0 : 1.0);
            double cost = 2600 + per * rounds * (alone + shared * (busy - 1)) + 4.0 * g.k * g.c / (sms * (g.c % 4 != 0 ? 8 : 20));
            if (used > 1) cost += 4000 + 4.0 * used * g.k * g.c / (sms * 20);
            if (best.tk != 0 && cost >= best_cost) continue;
            best_cost = cost;
            best = FmaHost{t[0], t[1], used, (int)per * chunk};
        }
    }
    if (best.tk == 0) return false;
    *cycles = best_cost;
    plan->partial_bytes = best.splits == 1 ? 0 : align_up((size_t)best.splits * align_up((size_t)g.k * g.c, 4) * sizeof(float) + 256, 256);
    plan->dy_bytes = 0;
    plan->fma = true;
    (void)dy_npqk;
    memcpy(plan->opaque, &best, sizeof(best));
    return true;
}

cudaError_t launch_packed_fma(const void* codes, const void* scales, int format, const void* dy, float* dw, float* partial, const Geom& g, bool dy_npqk, const PackedPlan& plan,
                              cudaStream_t stream)
{
    FmaHost H;
    memcpy(&H, plan.opaque, sizeof(H));
    const size_t count = (size_t)g.k * g.c;
    FmaParams P{};
    P.codes = static_cast<const uint8_t*>(codes); P.scales = static_cast<const uint8_t*>(scales); P.dy = dy;
    P.out = H.splits > 1 ? partial : dw;
    P.out_split = (long long)count; P.ws_k = g.ws_k; P.ws_c = g.ws_c;
    P.rows = (int)((long long)g.n * g.p * g.q); P.c = g.c; P.k = g.k; P.pitch = act_pitch(g.c); P.groups = act_groups(g.c);
    P.px = dy_npqk || g.k == 1 ? 1 : g.p * g.q;
    P.per_split = H.per_split;
    P.alpha = H.splits > 1 ? 1.f : g.alpha;
    const cudaError_t err = g.bf16 ? (format == GACONV_ACT_E4M3 ? launch<__nv_bfloat16, GACONV_ACT_E4M3>(H, P, stream) : launch<__nv_bfloat16, GACONV_ACT_INT8>(H, P, stream))
                                   : (format == GACONV_ACT_E4M3 ? launch<float, GACONV_ACT_E4M3>(H, P, stream) : launch<float, GACONV_ACT_INT8>(H, P, stream));
    if (err != cudaSuccess) return err;
    note_launch();
    return H.splits > 1 ? reduce_splits(partial, dw, count, H.splits, g.alpha, stream) : cudaSuccess;
}

}  // namespace gaconv
