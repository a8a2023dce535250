// Root-mean-square norm behind the addition of the residual, with its output in 8 bits as well, and its backward pass.
//
//   forward    s = x + r (rounded to the type),  rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd w (fp32, then rounded to the type),  codes, scales = y in 8 bits (act8.cuh)
//   backward   h = s rstd,  g = dy w,  dx = ds + rstd (g - h mean(g h)),  dw = sum over rows of dy h
//
// Bound by HBM.  A team of `lanes` threads holds a row in registers, `NU` pieces of 16 bytes a thread, by columns where rows are whole pieces (FULL) and by
// their frame elsewhere (rows.cuh), so that the second use of a row (after its mean) reads nothing: every tensor is read and written once.  Rows beyond the
// registers, and tensors whose rows lie on different boundaries, take the kernels called long, which read what they need twice: forward its sum (or x), backward dy and the
// sum, and both once more for the weight's gradient.  Sums and means are fp32, in an order that depends on the sizes alone.
#include <algorithm>
#include <type_traits>

#include "act8.cuh"
#include "device_utils.cuh"
#include "gaconv_internal.h"
#include "rows.cuh"

namespace gaconv {
namespace {

// Sum over the threads of a team, the same bits in each.  `part`: two rows of one float a warp, taken in turn so that one barrier a sum is enough.
__device__ __forceinline__ float team_sum(float v, int lanes, int team, float (*part)[16], int& turn)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float other = __shfl_xor_sync(0xffffffffu, v, o);
        if (o < lanes) v += other;
    }
    if (lanes > 32) {
        const int n = lanes >> 5, first = team * n;
        if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(lanes) : "memory");
        v = 0.f;
        for (int i = 0; i < n; ++i) v += part[turn][first + i];
        turn ^= 1;
    }
    return v;
}

template <int N>
__device__ __forceinline__ void store_codes(const NormRows& o, const float (&t)[N], uint8_t* codes, uint8_t* scales, long long r, int c, int pitch_left)
{
    uint8_t *q = codes + r * o.pitch + c, *s = scales + r * o.groups + (c >> 5);
    if (o.format == GACONV_ACT_E4M3) act_store<GACONV_ACT_E4M3, N>(t, q, pitch_left, s, (c & 31) == 0);
    else act_store<GACONV_ACT_INT8, N>(t, q, pitch_left, s, (c & 31) == 0);
}
// x + r, rounded to the type
template <typename T>
__device__ __forceinline__ uint4 add_pieces(const uint4& x, const uint4& r)
{
    float a[kPiece<T>], b[kPiece<T>];
    to_floats<T>(x, a); to_floats<T>(r, b);
#pragma unroll
    for (int j = 0; j < kPiece<T>; ++j) a[j] += b[j];
    return from_floats<T>(a);
}
// N elements of the weight from column c on, zeros outside [0, cols)
template <typename T, bool FULL>
__device__ __forceinline__ uint4 load_weight(const T* __restrict__ w, int c, int cols)
{
    if (FULL) return c < cols ? *reinterpret_cast<const uint4*>(w + c) : make_uint4(0, 0, 0, 0);
    if (c >= 0) {
        const Row<T, false> from(w + c, 0, 0, 1, cols - c, c < cols);
        Piece<T, false> p;
        p.start(from, 0);
        return p.value(from, 0);
    }
    return shifted16(make_uint4(0, 0, 0, 0), load_slowly(w, min(cols, kPiece<T> + c)), 16 + c * (int)sizeof(T));
}

// Blocks stay and their teams take rows in turn, the next one's loads on their way while a row is worked on.  Where rows are not whole pieces a team's
// rows are a multiple of N apart: they have one frame, and the weight's pieces in it stay in registers.
// WIDE: registers for three blocks of 256 threads an SM.  Rows of more than 128 threads gain by it, shorter ones lose (us of calls one behind the other, without
// and with: 16384x4096 bf16 101.6, 99.2; 8192x3584 bf16 52.0, 50.8; 8000x1333 fp32 56.2, 48.7; 16384x1024 bf16 28.0, 29.3; 16000x333 fp32 36.6, 40.4; without codes
// 16384x4096 bf16 90.7, 94.0; bf16 rows that are not whole pieces 8000x3003 66.9, 69.5; few of bf16 512x4096 6.2, 6.4).
template <typename T, int NU, bool FULL, bool WIDE = false>
__global__ void __launch_bounds__(WIDE ? 256 : 512, WIDE ? 3 : 1)
rmsnorm_forward_kernel(const NormRows o, const T* x, const T* res, const T* __restrict__ w, T* sum, T* y, uint8_t* codes, uint8_t* scales, float* rstd, int lanes)
{
    constexpr int N = kPiece<T>;
    __shared__ float part[2][16];
    __shared__ uint4 s_head[FULL ? 1 : 2][FULL ? 1 : NU][16];
    pdl_release_next_grid();
    const int team = threadIdx.x / lanes, l = threadIdx.x - team * lanes, teams = blockDim.x / lanes, warp = threadIdx.x >> 5;
    const long long step = (long long)gridDim.x * teams;
    long long first = (long long)blockIdx.x * teams;          // row of the block's first team; its teams go along in step, with or without a row
    const int shift = FULL ? 0 : (int)((first + team) * o.x_stride % N);          // the frame: columns -shift, N - shift, ...
    const bool edge = lanes >= 32 ? (l & 31) == 31 : l == lanes - 1;                // the next piece of the frame is not a lane up
    int turn = 0, parity = 0;
    pdl_wait_prior_grid();
    uint4 vw[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) vw[i] = load_weight<T, FULL>(w, N * (i * lanes + l) - shift, o.cols);
    uint4 vn[FULL ? 1 : NU];          // a warp's last lane: the weight of the piece behind its own
#pragma unroll
    for (int i = 0; i < (FULL ? 0 : NU); ++i) vn[i] = load_weight<T, FULL>(w, N * (i * lanes + l) - shift + N, edge ? o.cols : 0);
    FramePiece<T, FULL> px[NU], pr[NU];
    auto start = [&](long long row) {
        const Row<T, FULL> rx(x, row, o.x_stride, o.rows, o.cols, row < o.rows), rr(res, row, o.r_stride, o.rows, o.cols, row < o.rows);
#pragma unroll
        for (int i = 0; i < NU; ++i) { px[i].start(rx, N * (i * lanes + l) - shift); pr[i].start(rr, N * (i * lanes + l) - shift); }
    };
    start(first + team);
    for (; first < o.rows; first += step) {
        const long long row = first + team;
        const bool live = row < o.rows;
        const int cols = live ? o.cols : 0, pitch = live ? o.pitch : 0;
        uint4 v[NU];
        {
            const Row<T, FULL> rx(x, row, o.x_stride, o.rows, o.cols, live), rr(res, row, o.r_stride, o.rows, o.cols, live);
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int c = N * (i * lanes + l) - shift;
                v[i] = px[i].value(rx, c);
                if (res != nullptr) v[i] = add_pieces<T>(v[i], pr[i].value(rr, c));
            }
        }
        start(row + step);
        if (sum != nullptr) {
#pragma unroll
            for (int i = 0; i < NU; ++i) store_frame<T, FULL>(sum + row * o.s_stride, N * (i * lanes + l) - shift, cols, v[i]);
        }
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            float f[N], t = 0.f;
            to_floats<T>(v[i], f);
#pragma unroll
            for (int j = 0; j < N; ++j) t = fmaf(f[j], f[j], t);
            q += t;
            if (!FULL && (l & 31) == 0) s_head[parity][i][warp] = v[i];
        }
        if (!FULL) __syncwarp();
        q = team_sum(q, lanes, team, part, turn);          // (and a barrier of the team, where it has several warps)
        const float rs = 1.f / sqrtf(q / (float)o.cols + o.eps);
        if (live && l == 0 && rstd != nullptr) rstd[row] = rs;
        auto output = [&](const uint4& s, const uint4& weight) {
            float f[N], t[N];
            to_floats<T>(weight, t);
            to_floats<T>(s, f);
#pragma unroll
            for (int j = 0; j < N; ++j) t[j] = f[j] * rs * t[j];
            return from_floats<T>(t);
        };
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = N * (i * lanes + l);
            uint4 out = output(v[i], vw[i]);
            if (y != nullptr) store_frame<T, FULL>(y + row * o.y_stride, c - shift, cols, out);
            if (codes != nullptr) {
                if (!FULL) {        // from the frame to columns: with what the next piece of the frame has, a lane up or, for a warp's last lane, of its neighbour's first
                    uint4 next;
                    next.x = __shfl_down_sync(0xffffffffu, out.x, 1); next.y = __shfl_down_sync(0xffffffffu, out.y, 1);
                    next.z = __shfl_down_sync(0xffffffffu, out.z, 1); next.w = __shfl_down_sync(0xffffffffu, out.w, 1);
                    if (edge) {
                        const bool wraps = l == lanes - 1;
                        next = make_uint4(0, 0, 0, 0);
                        if (!wraps || i + 1 < NU) next = output(s_head[parity][wraps && i + 1 < NU ? i + 1 : i][wraps ? warp - (lanes >> 5) + 1 : warp + 1], vn[FULL ? 0 : i]);
                    }
                    out = shifted16(out, next, shift * (int)sizeof(T));
                }
                float t[N];
                to_floats<T>(out, t);
                store_codes<N>(o, t, codes, scales, live ? row : 0, c, pitch - c);
            }
        }
        parity ^= 1;
    }
}

// Rows longer than a team's registers, or tensors whose rows lie on different boundaries: a block a row, which it reads twice (the second time from
// L2 or, of very long rows, from memory), by columns.
template <typename T, bool FULL>
__global__ void __launch_bounds__(512)
rmsnorm_forward_long_kernel(const NormRows o, const T* x, const T* res, const T* __restrict__ w, T* sum, T* y, uint8_t* codes, uint8_t* scales, float* rstd)
{
    constexpr int N = kPiece<T>;
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const long long r = blockIdx.x;
    const Row<T, FULL> rx(x, r, o.x_stride, o.rows, o.cols, true), rr(res, r, o.r_stride, o.rows, o.cols, true);
    T* sr = sum + r * o.s_stride;
    int turn = 0;
    float q = 0.f;
    pdl_wait_prior_grid();
    for (int c0 = 0; c0 < o.cols; c0 += 512 * N) {
        const int c = c0 + N * threadIdx.x;
        float f[N], t = 0.f;
        Piece<T, FULL> px, pr;
        px.start(rx, c);
        pr.start(rr, c);
        uint4 v = px.value(rx, c);
        if (res != nullptr) v = add_pieces<T>(v, pr.value(rr, c));
        if (sum != nullptr) store_piece<T, FULL>(sr + c, o.cols - c, v, 9);
        to_floats<T>(v, f);
#pragma unroll
        for (int j = 0; j < N; ++j) t = fmaf(f[j], f[j], t);
        q += t;
    }
    q = team_sum(q, 512, 0, part, turn);          // (a barrier: the neighbours' stores of a shared 16 bytes are seen below)
    const float rs = 1.f / sqrtf(q / (float)o.cols + o.eps);
    if (threadIdx.x == 0 && rstd != nullptr) rstd[r] = rs;
    const Row<T, FULL> again(sum != nullptr ? sum : x, r, sum != nullptr ? o.s_stride : o.x_stride, o.rows, o.cols, true);
    for (int c0 = 0; c0 < o.cols; c0 += 512 * N) {
        const int c = c0 + N * threadIdx.x;
        float f[N], t[N];
        Piece<T, FULL> pv;
        pv.start(again, c);
        to_floats<T>(load_weight<T, FULL>(w, c, o.cols), t);
        to_floats<T>(pv.value(again, c), f);
#pragma unroll
        for (int j = 0; j < N; ++j) t[j] = f[j] * rs * t[j];
        const uint4 out = from_floats<T>(t);
        if (y != nullptr) store_piece<T, FULL>(y + r * o.y_stride + c, o.cols - c, out, 9);
        if (codes != nullptr) {
            to_floats<T>(out, t);
            store_codes<N>(o, t, codes, scales, r, c, o.pitch - c);
        }
    }
}

constexpr int kChain = 64;          // rows that are added up one by one for dweight, before the sum is added to that of others

// Backward.  A block stays and its teams take rows in turn; a thread keeps the sums over rows of dy h for its channels, which the
// teams of a block add up in order at the end: partial[block][cols].  A team's rows are a multiple of N apart, so that they have one frame, and a thread the
// same channels in each.  (One block writes dweight itself.)  The three tensors of a row are loaded while the row before is worked on, and kept as they are: the products of the first half are
// formed again after the mean.
// CHAINS: a team may have more than kChain rows (where it has not, the looking costs 0.4 us a call: 10x240 fp32 3.6 us without, 4.0 with; 5003x1000 fp32 12.7, 13.4).
template <typename T, int NU, bool FULL, bool CHAINS>
__global__ void __launch_bounds__(512)
rmsnorm_backward_kernel(const NormRows o, const T* dy, const T* ds, const T* s, const T* __restrict__ w, const float* __restrict__ rstd, T* dx, float* __restrict__ partial, int lanes)
{
    constexpr int N = kPiece<T>;
    extern __shared__ float s_dw[];
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const int team = threadIdx.x / lanes, l = threadIdx.x - team * lanes, teams = blockDim.x / lanes;
    float acc[NU][N];
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i][j] = 0.f;
    int turn = 0;
    const long long step = (long long)gridDim.x * teams;
    long long first = (long long)blockIdx.x * teams;          // row of the block's first team; its teams go along in step, with or without a row
    const int shift = FULL ? 0 : (int)((first + team) * o.s_stride % N);
    pdl_wait_prior_grid();
    uint4 vw[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) vw[i] = load_weight<T, FULL>(w, N * (i * lanes + l) - shift, o.cols);
    const float inv = 1.f / (float)o.cols;
    // the team's sums so far, of kChain rows at a time, at s_dw + team * cols; a channel is always the same thread's
    float* mine = s_dw + (size_t)team * o.cols;
    int chain = 0;
    bool begun = false;
    auto add_chain = [&] {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = N * (i * lanes + l) - shift;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (c + j >= 0 && c + j < o.cols) mine[c + j] = CHAINS && begun ? mine[c + j] + acc[i][j] : acc[i][j];
                if (CHAINS) acc[i][j] = 0.f;
            }
        }
        begun = true;
    };
    FramePiece<T, FULL> pg[NU], ps[NU], pd[NU];
    float rs_next = 0.f;
    auto start = [&](long long row) {
        const bool live = row < o.rows;
        const Row<T, FULL> rg(dy, row, o.y_stride, o.rows, o.cols, live), rh(s, row, o.s_stride, o.rows, o.cols, live), rd(ds, row, o.s_stride, o.rows, o.cols, live);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int c = N * (i * lanes + l) - shift;
            pg[i].start(rg, c); ps[i].start(rh, c); pd[i].start(rd, c);
        }
        rs_next = live ? __ldg(rstd + row) : 0.f;          // (a row of nothing adds 0, not 0 times the last row's, which may be infinite)
    };
    start(first + team);
    for (; first < o.rows; first += step) {
        const long long row = first + team;
        const bool live = row < o.rows;
        uint4 vg[NU], vs[NU], vd[NU];
        const float rs = rs_next;
        {
            const Row<T, FULL> rg(dy, row, o.y_stride, o.rows, o.cols, live), rh(s, row, o.s_stride, o.rows, o.cols, live), rd(ds, row, o.s_stride, o.rows, o.cols, live);
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                const int c = N * (i * lanes + l) - shift;
                vg[i] = pg[i].value(rg, c); vs[i] = ps[i].value(rh, c); vd[i] = pd[i].value(rd, c);
            }
        }
        start(row + step);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            float g[N], h[N], t[N], sum = 0.f;
            to_floats<T>(vg[i], g); to_floats<T>(vs[i], h); to_floats<T>(vw[i], t);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float gh = g[j] * (h[j] * rs);
                acc[i][j] += gh;
                sum = fmaf(gh, t[j], sum);
            }
            dot += sum;
        }
        dot = team_sum(dot, lanes, team, part, turn) * inv;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            float g[N], h[N], t[N], d[N];
            to_floats<T>(vg[i], g); to_floats<T>(vs[i], h); to_floats<T>(vw[i], t); to_floats<T>(vd[i], d);
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = fmaf(rs, g[j] * t[j] - h[j] * rs * dot, d[j]);
            store_frame<T, FULL>(dx + row * o.x_stride, N * (i * lanes + l) - shift, live ? o.cols : 0, from_floats<T>(d));
        }
        if (CHAINS && ++chain == kChain) { add_chain(); chain = 0; }
    }
    if (partial == nullptr) return;
    // the teams' sums, in order
    add_chain();
    __syncthreads();
    float* out = partial + (size_t)blockIdx.x * o.cols;
    for (int c = threadIdx.x; c < o.cols; c += blockDim.x) {
        float v = s_dw[c];
        for (int t = 1; t < teams; ++t) v += s_dw[t * o.cols + c];
        out[c] = v;
    }
}

template <typename T, bool FULL>
__global__ void __launch_bounds__(512)
rmsnorm_backward_long_kernel(const NormRows o, const T* dy, const T* ds, const T* s, const T* __restrict__ w, const float* __restrict__ rstd, T* dx)
{
    constexpr int N = kPiece<T>;
    __shared__ float part[2][16];
    pdl_release_next_grid();
    const long long row = blockIdx.x;
    const Row<T, FULL> rg(dy, row, o.y_stride, o.rows, o.cols, true), rh(s, row, o.s_stride, o.rows, o.cols, true), rd(ds, row, o.s_stride, o.rows, o.cols, true);
    int turn = 0;
    float dot = 0.f;
    pdl_wait_prior_grid();
    const float rs = rstd[row];
    for (int pass = 0; pass < 2; ++pass) {
        for (int c0 = 0; c0 < o.cols; c0 += 512 * N) {
            const int c = c0 + N * threadIdx.x;
            float g[N], h[N], t[N], d[N], sum = 0.f;
            Piece<T, FULL> pg, ps, pd;
            pg.start(rg, c);
            ps.start(rh, c);
            if (pass == 1) pd.start(rd, c);
            to_floats<T>(load_weight<T, FULL>(w, c, o.cols), t);
            to_floats<T>(pg.value(rg, c), g);
            to_floats<T>(ps.value(rh, c), h);
            if (pass == 0) {
#pragma unroll
                for (int j = 0; j < N; ++j) sum = fmaf(g[j] * t[j], h[j] * rs, sum);
                dot += sum;
            } else {
                to_floats<T>(pd.value(rd, c), d);
#pragma unroll
                for (int j = 0; j < N; ++j) d[j] = fmaf(rs, g[j] * t[j] - h[j] * rs * dot, d[j]);
                store_piece<T, FULL>(dx + row * o.x_stride + c, o.cols - c, from_floats<T>(d), 9);
            }
        }
        if (pass == 0) dot = team_sum(dot, 512, 0, part, turn) / (float)o.cols;
    }
}
// sums over a range of rows, a thread a channel: grid (channels / 256, ranges).  Ranges grow with the rows; their sums are put together from chains of kChain rows
// (one chain of 16384 rows, of products alike, was off by 1e-4).
template <typename T>
__global__ void __launch_bounds__(256)
rmsnorm_weight_long_kernel(const NormRows o, const T* dy, const T* s, const float* __restrict__ rstd, float* __restrict__ partial)
{
    pdl_release_next_grid();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= o.cols) return;
    const long long per = (o.rows + gridDim.y - 1) / gridDim.y, first = blockIdx.y * per, last = min(first + per, o.rows);
    float total = 0.f, rest = 0.f;          // (the sum is total + rest: what an addition to total rounds off goes to rest)
    pdl_wait_prior_grid();
    for (long long r0 = first; r0 < last; r0 += kChain) {
        const long long end = min(r0 + kChain, last);
        float acc = 0.f;
#pragma unroll 16
        for (long long r = r0; r < end; ++r) acc = fmaf(ldf(dy + r * o.y_stride + c), ldf(s + r * o.s_stride + c) * __ldg(rstd + r), acc);
        const float sum = total + acc, part = sum - total;
        rest += (total - (sum - part)) + (acc - part);
        total = sum;
    }
    // (not finite: total alone, since Inf - Inf in rest would be NaN)
    partial[(size_t)blockIdx.y * o.cols + c] = isfinite(total) ? total + rest : total;
}

// ---------------------------------------------------------------- host side
struct Team { int lanes, nu; bool full; };          // nu = 0: a row by blocks, twice
constexpr int kMaxTeam = 512;
// Threads of a row, a multiple of 32 or, for short rows, 8 or 16: two pieces each, one where that leaves SMs without work, four (forward) for long rows.
// strides: of the tensors in the call.
Team team_of(const NormRows& o, int most, long long a, long long b, long long c, long long d)
{
    const int n = o.bf16 ? 8 : 4;
    Team t{0, 0, o.cols % n == 0 && a % n == 0 && b % n == 0 && c % n == 0 && d % n == 0};
    const int pieces = t.full ? o.cols / n : (o.cols + 2 * n - 2) / n;         // (a frame starts up to n - 1 elements early)
    auto lanes = [&](int nu) { return (pieces + 32 * nu - 1) / (32 * nu) * 32; };
    if (!t.full && (a % n != b % n || a % n != c % n || a % n != d % n)) return t;
    t.nu = lanes(1) == 32 || (lanes(1) <= kMaxTeam && o.rows * lanes(2) < device_sms() * 512ll) ? 1 : lanes(2) <= (most == 4 ? kMaxTeam / 2 : kMaxTeam) ? 2 : lanes(4) <= kMaxTeam && most == 4 ? 4 : 0;
    if (t.nu != 0) t.lanes = pieces <= 8 ? 8 : pieces <= 16 ? 16 : lanes(t.nu);
    return t;
}
// Blocks for teams that stay: as many as fit the SMs, and such that a team's rows have one frame
int team_blocks(const NormRows& o, const Team& t, long long stride, int teams, int most)
{
    const int n = o.bf16 ? 8 : 4;
    const long long need = (o.rows + teams - 1) / teams;
    if (need <= most) return (int)need;
    while (!t.full && most > 1 && (long long)most * teams * stride % n != 0) --most;
    return most;
}
Team backward_team(const NormRows& o) { return team_of(o, 2, o.y_stride, o.s_stride, o.x_stride, o.s_stride); }
int backward_blocks(const NormRows& o, const Team& t) { return team_blocks(o, t, o.s_stride, kMaxTeam / t.lanes, device_sms()); }

template <typename T>
cudaError_t forward(const NormRows& o, const T* x, const T* res, const T* w, T* sum, T* y, uint8_t* codes, uint8_t* scales, float* rstd, cudaStream_t stream)
{
    const Team t = team_of(o, 4, o.x_stride, res ? o.r_stride : o.x_stride, sum ? o.s_stride : o.x_stride, y ? o.y_stride : o.x_stride);
    note_launch();
    if (t.nu == 0) {
        auto kern = t.full ? rmsnorm_forward_long_kernel<T, true> : rmsnorm_forward_long_kernel<T, false>;
        return launch_kernel(kern, dim3((unsigned)o.rows), dim3(512), 0, stream, dim3(1, 1, 1), o, x, res, w, sum, y, codes, scales, rstd);
    }
    const int teams = std::max(1, 128 / t.lanes), threads = teams * t.lanes;
    const bool wide = t.nu == 2 && t.lanes > 128 && codes != nullptr && (sizeof(T) == 4 || (t.full && o.rows > 16ll * device_sms()));          // (two pieces: at most 256 threads)
    auto kern = t.nu == 1 ? (t.full ? rmsnorm_forward_kernel<T, 1, true> : rmsnorm_forward_kernel<T, 1, false>)
              : wide ? (t.full ? rmsnorm_forward_kernel<T, 2, true, true> : rmsnorm_forward_kernel<T, 2, false, sizeof(T) == 4>)
              : t.nu == 2 ? (t.full ? rmsnorm_forward_kernel<T, 2, true> : rmsnorm_forward_kernel<T, 2, false>)
                          : (t.full ? rmsnorm_forward_kernel<T, 4, true> : rmsnorm_forward_kernel<T, 4, false>);
    // blocks that an SM holds, asked once per kernel, size and device (all devices of a process alike)
    static std::atomic<int> resident[2][4][kMaxTeam / 32 + 1];
    std::atomic<int>& known = resident[t.full][wide ? 3 : t.nu / 2][threads / 32];
    int per_sm = known.load(std::memory_order_relaxed);
    if (per_sm == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, threads, 0) != cudaSuccess || per_sm < 1) per_sm = 1;
        known.store(per_sm, std::memory_order_relaxed);
    }
    return launch_kernel(kern, dim3((unsigned)team_blocks(o, t, o.x_stride, teams, per_sm * device_sms())), dim3(threads), 0, stream, dim3(1, 1, 1), o, x, res, w, sum, y, codes, scales, rstd, t.lanes);
}

template <typename T>
cudaError_t backward(const NormRows& o, const T* dy, const T* ds, const T* s, const T* w, const float* rstd, T* dx, float* dweight, float* partial, cudaStream_t stream)
{
    const Team t = backward_team(o);
    cudaError_t err;
    const int splits = norm_partials(o);
    note_launch();
    if (t.nu == 0) {
        if (dweight != nullptr) {
            err = launch_kernel(rmsnorm_weight_long_kernel<T>, dim3((unsigned)((o.cols + 255) / 256), (unsigned)splits), dim3(256), 0, stream, dim3(1, 1, 1), o, dy, s, rstd, partial);
            if (err != cudaSuccess) return err;
            note_launch();
        }
        auto kern = t.full ? rmsnorm_backward_long_kernel<T, true> : rmsnorm_backward_long_kernel<T, false>;
        err = launch_kernel(kern, dim3((unsigned)o.rows), dim3(512), 0, stream, dim3(1, 1, 1), o, dy, ds, s, w, rstd, dx);
    } else {
        const int teams = kMaxTeam / t.lanes;
        const bool chains = o.rows > (long long)kChain * splits * teams;
        auto kern = chains ? (t.nu == 1 ? (t.full ? rmsnorm_backward_kernel<T, 1, true, true> : rmsnorm_backward_kernel<T, 1, false, true>)
                                        : (t.full ? rmsnorm_backward_kernel<T, 2, true, true> : rmsnorm_backward_kernel<T, 2, false, true>))
                           : (t.nu == 1 ? (t.full ? rmsnorm_backward_kernel<T, 1, true, false> : rmsnorm_backward_kernel<T, 1, false, false>)
                                        : (t.full ? rmsnorm_backward_kernel<T, 2, true, false> : rmsnorm_backward_kernel<T, 2, false, false>));
        const size_t smem = sizeof(float) * (size_t)teams * o.cols;          // (at most 512 threads' sums: 32 KB)
        if (splits == 1) partial = dweight;
        err = launch_kernel(kern, dim3((unsigned)splits), dim3((unsigned)(teams * t.lanes)), smem, stream, dim3(1, 1, 1), o, dy, ds, s, w, rstd, dx, dweight != nullptr ? partial : nullptr, t.lanes);
    }
    if (err != cudaSuccess || dweight == nullptr || (t.nu != 0 && splits == 1)) return err;
    return reduce_splits(partial, dweight, (size_t)o.cols, splits, 1.f, stream);
}

}  // namespace

// rows of `cols` sums that the backward pass leaves in the workspace
int norm_partials(const NormRows& o)
{
    if (o.rows == 0) return 0;
    const Team t = backward_team(o);
    if (t.nu != 0) return backward_blocks(o, t);
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
