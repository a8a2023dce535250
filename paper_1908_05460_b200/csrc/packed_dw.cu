// Filter gradient of a linear layer (a 1x1 filter at stride 1) with X in 8 bits, on tcgen05:
//
//   dW[k, c] = alpha * sum over rows t of dY[t, k] * code[t, c] * 2^e[t, c / 32]
//
// The scales belong to the reduction index, so they cannot be taken out of the sum; but a code times its scale is exact in bf16 (act8.cuh).
// So X goes from memory to the SM in 8 bits, is turned into bf16 on the way from one piece of shared memory to another, and lies there in the
// order that the tensor core reads: half the bytes of a bf16 X and no copy of it in memory.  dY is the M side, X the N side, both MN-major (a row of
// shared memory is a row t, 64 channels of it); fp32 gradients are three bf16 planes dY = d0 + d1 + d2 (8 + 8 + 8 bits) whose products add up
// in the same accumulators.  Gradients that the copy engine cannot read as they lie (another order, rows that do not start on 16 bytes) are packed
// into the workspace first, fp32 ones as planes.
//
// fp32 gradients that it can read are split into planes by the threads that turn X, beside it (RAW).  For 64 rows 240 KB then pass through an SM's shared
// memory (128 bytes a cycle), and a stage takes 2300 cycles where one of packed planes takes 1600 (pairs: 2750, 2000); but no pass over dY comes
// first.  us, split inside and packed first: 4096 rows 512 -> 512 19.2, 21.8; 65536 rows 256 -> 256 37, 58; 131072 rows 64 -> 64 24.0, 29.8; 16384
// rows 1024 -> 1024 98, 97; 16384 rows 2048 -> 256 53.6, 48.2; 16384 rows 4096 -> 1024 352, 281.
//
// A CTA pair (CG = 2) shares a tile of 256 x 256: each CTA holds 128 outputs of dY and 128 channels of X, and the pair's MMAs read both halves of X,
// so that a turned element serves 256 outputs.  CG = 1: tiles of 128 x 128, or 128 x 64, for problems that would not fill the GPU with larger ones (us by
// pairs, by 128 x 128, by 128 x 64: 8192 rows 1024 -> 4096 59, 104, -; 16384 rows 100 -> 1000 18.1, 15.7, 18.0; 1000 rows 1000 -> 1000 13.3, 11.7,
// 9.8; 512 rows 512 -> 512 10.5, 8.5, 6.9: an SM writes 21 bytes a cycle, so that small results want many SMs).
//
// What bounds it: 64 rows take the MMAs of a pair 512 cycles, and ~785 pass (16384 rows, 4096 -> 4096, 1065 TFLOP/s where cuBLAS on bf16 operands has 1420;
// tensor pipe 70 % active, shared-memory banks 38 % busy, DRAM 14 %).  Turning 64 x 128 elements takes four warps ~1200 cycles, most of it latency (loads, eight
// chains of five instructions, stores, the fence), two groups of four warps alternate, and every other time the MMAs wait for them.  What helped: rings
// apart for dY, X and X turned; copies of 128 rows, since a warp needs 500 cycles to fill a stage however large it is; looking at a barrier before its
// turn, since that takes 200; no cluster-wide acquire (550 -> 507 us); decoding in five instructions a pair.  A third group of warps has no registers left.
//
// Whoever turns X loads nothing from memory: the fence between its stores and the tensor core waits for every load that the thread has in flight
// (loads two stages ahead in its registers: 1435 us).
//
// The tensor core adds by truncation, so accumulators are handed over every `epoch` stages to eight warps that add them up in fp32 registers; two
// accumulator sets alternate.  CTAs stay and take units (a tile, a range of rows) in turn; pipeline and sets run on from unit to unit, so
// that the writing of one hides behind the next.  The tiles of a last, incomplete round are split over their rows; the splits meet in the workspace,
// added in order by packed_reduce_kernel.
//
// Rows past the end and channels past a row are zeros on both sides.  Every wait is bounded; on expiry the kernel raises the workspace status word,
// lets its copies and MMAs land, frees its tensor memory and returns.
#include <cuda.h>

#include <algorithm>
#include <cstring>

#include "act8.cuh"
#include "device_utils.cuh"
#include "gaconv_internal.h"
#include "tma.cuh"
#include "umma.cuh"

namespace gaconv {
namespace {

constexpr int kRows = 64;                           // rows t that are turned, and multiplied, at a time
constexpr int kTile = kRows * 128;                  // bytes of 64 channels of them in bf16
constexpr int kThreads = 640;                       // warps 0-3: scales, MMAs, copies of X, copies of dY; 4-11 turn X, 12-19 sum
constexpr int kMaxRing = 4;

// Three rings: dY and X in 8 bits as they are copied, `halves` x 64 rows at a time (a warp takes ~500 cycles for its round of wait, byte count and copy, however
// large the copy is, and the MMAs 512 for 64 rows), and X turned, 64 rows at a time.
template <int PLANES> constexpr int kStageRows = PLANES == 3 ? kRows : 2 * kRows;
// XC: channels of X that a CTA turns.  RAW: fp32 gradients as they lie, split into planes beside it.
template <int CG, int PLANES, int XC, bool RAW> struct Config {
    static_assert(!RAW || PLANES == 3, "fp32");
    static constexpr int cols = XC * CG, halves = PLANES == 3 ? 1 : 2, rows = kStageRows<PLANES>, atoms = XC / 64;
    static constexpr int split = RAW ? 2 * PLANES * kTile : 0;      // bytes of dY in a slot of what is turned
    static constexpr int dy_stage = RAW ? kRows * 128 * 4 : 2 * PLANES * halves * kTile, dys = RAW ? 2 : 3;
    static constexpr int turned = split + atoms * kTile, turneds = PLANES == 3 ? 2 : 4, raws = RAW ? 2 : PLANES == 3 ? 4 : 3;
    static constexpr int raw = rows * XC + rows * 8;                // the channels in 8 bits, and the two words around the scales of each row
    static constexpr int turned_at = dys * dy_stage, raw_at = turned_at + turneds * turned, out_at = raw_at + raws * raw, bytes = out_at + 8 * 1024;
    static constexpr int epoch = PLANES == 3 ? 4 : 8;               // stages of dY: chains of 48 or 64 MMAs
    // registers of a thread by role; their sum over the warps is within what the block is launched with (96 each)
    static constexpr int regs_control = 48, regs_turn = CG == 2 ? 56 : 80, regs_sum = CG == 2 ? 160 : 104;
    static_assert(4 * regs_control + 8 * regs_turn + 8 * regs_sum <= 20 * 96, "registers");
    // A wait for a phase is only right once the phase before is over, which a group knows of its own stages alone: no slot passes from one group to the other
    static_assert(turneds % 2 == 0 && raws * halves % 2 == 0 && (!RAW || dys == 2), "two groups turn X");
    static_assert(dys <= kMaxRing && turneds <= kMaxRing && raws <= kMaxRing && bytes <= 225 * 1024 && raw % 128 == 0, "shared memory");
};

struct PackedParams {
    const uint8_t *codes, *scales;
    float *dw, *partial;
    uint32_t* status;
    int rows, c, k, groups;
    long long ws_k, ws_c;
    float alpha;
    int tiles_c;                                    // tile = tk * tiles_c + tc
    int full, splits, units;                        // tiles [0, full) are units of their own; the others `splits` each
    int chunks;                                     // stages of dY in all rows
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
// wait for arrivals of either CTA of a pair
__device__ __forceinline__ bool pair_wait(uint32_t bar, uint32_t parity)
{
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}
// whether a phase is over, without a wait
__device__ __forceinline__ bool mbar_look(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
template <int CG>
__device__ __forceinline__ void arrive_leader(uint32_t bar)
{
    if (CG == 2) {
        asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\tmbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar) : "memory");
    } else {
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
    }
}
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar)       // to the barrier in every CTA of the group
{
    if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
    else umma_commit(bar);
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
    else umma_bf16(d, a, b, idesc, accumulate);
}
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
__device__ __forceinline__ void store_shared16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 load_shared16(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
// asynchronous copy of a word, of which only the first n bytes are read; zeros behind them
__device__ __forceinline__ void copy_word(uint32_t dst, const void* src, int n)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

// The stages of a CTA, unit after unit
struct Walk {
    int unit, left, chunk, k0, c0;
    __device__ __forceinline__ void enter(const PackedParams& P)
    {
        left = 0;
        if (unit >= P.units) return;
        int tile = unit, first = 0, last = P.chunks;
        if (unit >= P.full) {
            const int u = unit - P.full, t = u / P.splits, s = u - t * P.splits;
            tile = P.full + t;
            first = (int)((long long)P.chunks * s / P.splits);
            last = (int)((long long)P.chunks * (s + 1) / P.splits);
        }
        const int tk = tile / P.tiles_c;
        k0 = tk; c0 = tile - tk * P.tiles_c;
        chunk = first; left = last - first;
    }
    __device__ __forceinline__ void start(const PackedParams& P, int first_unit) { unit = first_unit; enter(P); }
    __device__ __forceinline__ bool live() const { return left > 0; }
    __device__ __forceinline__ void next(const PackedParams& P, int step)
    {
        ++chunk;
        if (--left == 0) { unit += step; enter(P); }
    }
};

template <int CG, int PLANES, int XC, bool RAW, int FMT>
__global__ void __launch_bounds__(kThreads, 1)
packed_dw_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ PackedParams P)
{
    typedef Config<CG, PLANES, XC, RAW> C;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_dy[kMaxRing], bar_free_dy[kMaxRing], bar_full[kMaxRing], bar_empty[kMaxRing], bar_raw[kMaxRing], bar_taken[kMaxRing], bar_acc[2], bar_free[2], bar_last;
    __shared__ uint32_t s_tmem;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0, group = blockIdx.x / CG, step = gridDim.x / CG;

    pdl_release_next_grid();
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::dys; ++i) { mbar_init(smem_u32(&bar_dy[i]), rank == 0 && !RAW ? CG : 1); mbar_init(smem_u32(&bar_free_dy[i]), RAW ? 4 : 1); }
        for (int i = 0; i < C::turneds; ++i) { mbar_init(smem_u32(&bar_full[i]), 4 * CG); mbar_init(smem_u32(&bar_empty[i]), 1); }
        for (int i = 0; i < C::raws; ++i) { mbar_init(smem_u32(&bar_raw[i]), 1 + 32); mbar_init(smem_u32(&bar_taken[i]), 4 * C::halves); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&bar_acc[i]), 1); mbar_init(smem_u32(&bar_free[i]), 8 * CG); }
        mbar_init(smem_u32(&bar_last), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_dy) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
    }
    if (warp == 1) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(2 * C::cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(2 * C::cols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    pdl_wait_prior_grid();
    auto give_up = [&] { atomicOr(P.status, 1u); };        // (the other roles' waits run out in turn)

    if (warp < 4) {
        regs_down<C::regs_control>();
        if (warp == 2) {
            // ------------------------------------------------------------ copies of X: 128 channels a stage
            Walk w;
            w.start(P, group);
            int st = 0, ph = 0, n = 0;
            bool ok = true, taken = true;
            for (; w.live(); w.next(P, step)) {
                if (!taken) ok = mbar_wait(smem_u32(&bar_taken[st]), ph ^ 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = smem_u32(&bar_raw[st]);
                    mbar_expect_tx(bar, C::rows * XC);
                    tma_load_3d(base + C::raw_at + st * C::raw, &map_x, bar, (w.c0 * CG + rank) * XC, w.chunk * C::rows, 0);
                }
                __syncwarp();
                if (++st == C::raws) { st = 0; ph ^= 1; }
                ++n;
                taken = n < C::raws || mbar_look(smem_u32(&bar_taken[st]), ph ^ 1);
            }
            if (!ok) give_up();
            // all of X that was copied has been turned; on failure the wait is the time that copies have to land (bounded)
            for (int i = max(0, n - C::raws); i < n; ++i) mbar_wait(smem_u32(&bar_taken[i % C::raws]), (i / C::raws) & 1);
        } else if (warp == 3) {
            // ------------------------------------------------------------ copies of dY: 128 outputs a stage and plane, lane b issues copy b of 64
            Walk w;
            w.start(P, group);
            int st = 0, ph = 0, n = 0;
            bool ok = true, empty = true;
            for (; w.live(); w.next(P, step)) {
                if (!empty) ok = pair_wait(smem_u32(&bar_free_dy[st]), ph ^ 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t bar = smem_u32(&bar_dy[st]);
                if (lane == 0) mbar_expect_tx(bar, C::dy_stage);
                __syncwarp();
                if (RAW) {
                    if (lane < 4) tma_load_3d(base + st * C::dy_stage + lane * kTile, &map_dy, bar, (w.k0 * CG + rank) * 128 + 32 * lane, w.chunk * C::rows, 0);
                } else if (lane < 2 * PLANES)
                    tma_load_3d(base + st * C::dy_stage + lane * C::halves * kTile, &map_dy, bar, (w.k0 * CG + rank) * 128 + 64 * (lane & 1), w.chunk * C::rows, lane >> 1);
                if (++st == C::dys) { st = 0; ph ^= 1; }
                ++n;
                empty = n < C::dys || mbar_look(smem_u32(&bar_free_dy[st]), ph ^ 1);
            }
            if (!ok) give_up();
            // the last commits, which may come from the other CTA, arrive before this one goes; on failure the wait is the time that copies have to land (bounded)
            for (int i = max(0, n - C::dys); i < n; ++i) pair_wait(smem_u32(&bar_free_dy[i % C::dys]), (i / C::dys) & 1);
        } else if (warp == 0) {
            // ------------------------------------------------------------ scales, asynchronous copies too: rows 32 apart a lane
            Walk w;
            w.start(P, group);
            int st = 0, ph = 0, n = 0;
            bool ok = true, taken = true;
            const uint8_t* end = P.scales + (long long)P.rows * P.groups;
            for (; w.live(); w.next(P, step)) {
                if (!taken) ok = mbar_wait(smem_u32(&bar_taken[st]), ph ^ 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t bar = smem_u32(&bar_raw[st]), dst = base + C::raw_at + st * C::raw + C::rows * XC;
                const int g = (w.c0 * CG + rank) * (XC / 32);
#pragma unroll
                for (int i = 0; i < C::rows / 32; ++i) {
                    // a row's scales lie on any byte: the one or two aligned words that hold them, no byte past the end
                    const int r = 32 * i + lane, row = w.chunk * C::rows + r;
                    const bool in = row < P.rows && g < P.groups;
                    const uint8_t* at = P.scales + (in ? (long long)row * P.groups + g : 0);
                    const int off = (int)(reinterpret_cast<uintptr_t>(at) & 3);
                    const int left = (int)min((ptrdiff_t)8, end - (at - off));
                    copy_word(dst + r * 8, at - off, in ? min(4, left) : 0);
                    if ((P.groups & 3) != 0) copy_word(dst + r * 8 + 4, in && off != 0 && left > 4 ? at - off + 4 : P.scales, in && off != 0 ? max(0, left - 4) : 0);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                if (++st == C::raws) { st = 0; ph ^= 1; }
                ++n;
                taken = n < C::raws || mbar_look(smem_u32(&bar_taken[st]), ph ^ 1);
            }
            if (!ok) { give_up(); asm volatile("cp.async.wait_all;" ::: "memory"); }
        } else if (CG == 2 && !RAW && warp == 1 && rank == 1) {
            // ------------------------------------------------------------ tells the leader of this CTA's copies of dY
            Walk w;
            w.start(P, group);
            int st = 0, ph = 0;
            for (; w.live(); w.next(P, step)) {
                if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_dy[st]), ph))) { give_up(); break; }
                if (lane == 0) arrive_leader<CG>(smem_u32(&bar_dy[st]));
                if (++st == C::dys) { st = 0; ph ^= 1; }
            }
        } else if (warp == 1 && rank == 0) {
            // ------------------------------------------------------------ MMAs
            // M = 128 a CTA, N = cols; bf16 operands, both MN-major, fp32 accumulators
            constexpr uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(C::cols / 8) << 17 | (uint32_t)(8 * CG) << 24;
            constexpr uint64_t hi = (uint64_t)(1024 / 16 | 1u << 14 | 2u << 29) << 32;          // eight rows to the next, 128-byte swizzle
            constexpr uint32_t lbo_dy = (uint32_t)(C::halves * kTile / 16) << 16, lbo_x = (uint32_t)(kTile / 16) << 16;         // 64 channels to the next
            // A look at a barrier takes ~200 cycles even where the phase is over, so the next stage's is looked at before this one's MMAs are issued.
            Walk w;
            w.start(P, group);
            int st = 0, ph = 0, ds = 0, dph = 0, set = 0, epochs = 0;
            bool ready = false, ready_dy = false, ok = true;
            while (ok && w.live()) {
                int in_epoch = 0;
                for (int left = w.left; left > 0; --left) {
                    if (in_epoch == 0 && epochs >= 2) ok = pair_wait(smem_u32(&bar_free[set]), ((epochs >> 1) - 1) & 1);
                    if (!RAW && !ready_dy) ok = ok && pair_wait(smem_u32(&bar_dy[ds]), dph);
                    const int next_ds = ds + 1 == C::dys ? 0 : ds + 1;
                    dph ^= next_ds == 0 ? 1 : 0;
                    const bool ends = left == 1 || in_epoch + 1 == C::epoch;
#pragma unroll
                    for (int h = 0; h < C::halves; ++h) {
                        if (!ready) ok = ok && pair_wait(smem_u32(&bar_full[st]), ph);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const int next = st + 1 == C::turneds ? 0 : st + 1;
                        ph ^= next == 0 ? 1 : 0;
                        ready = mbar_look(smem_u32(&bar_full[next]), ph);
                        if (!RAW && h == C::halves - 1) ready_dy = mbar_look(smem_u32(&bar_dy[next_ds]), dph);
                        if (elect_one()) {
                            const uint32_t slot = base + C::turned_at + st * C::turned, a0 = RAW ? slot : base + ds * C::dy_stage + h * kTile, b0 = slot + C::split;
                            const uint64_t a = hi | (lbo_dy | (a0 >> 4)), b = hi | (lbo_x | (b0 >> 4));
                            const uint32_t d = tmem + set * C::cols;
#pragma unroll
                            for (int i = 0; i < kRows / 16; ++i)
#pragma unroll
                                for (int pl = PLANES - 1; pl >= 0; --pl)
                                    mma<CG>(d, a + (pl * 2 * C::halves * kTile + i * 2048) / 16, b + i * 2048 / 16, idesc, in_epoch > 0 || h > 0 || i > 0 || pl < PLANES - 1 ? 1u : 0u);
                            commit<CG>(smem_u32(&bar_empty[st]));
                            if (!RAW && h == C::halves - 1) commit<CG>(smem_u32(&bar_free_dy[ds]));
                            if (h == C::halves - 1 && ends) commit<CG>(smem_u32(&bar_acc[set]));
                        }
                        __syncwarp();
                        st = next;
                    }
                    if (!ok) break;
                    ++in_epoch;
                    if (ends) { in_epoch = 0; set ^= 1; ++epochs; }
                    ds = next_ds;
                }
                w.unit += step;
                w.enter(P);
            }
            if (!ok) {      // the MMAs that were issued end (bounded)
                give_up();
                if (elect_one()) {
                    if (CG == 2) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&bar_last)) : "memory");
                    else umma_commit(smem_u32(&bar_last));
                }
                __syncwarp();
                mbar_wait(smem_u32(&bar_last), 0);
            }
        }
    } else if (warp < 12) {
        // ---------------------------------------------------------------- X: 8 bits -> bf16
        // Four warps take 64 rows, the other four the next.  A thread turns pieces of 16 channels, chunk q of rows `row` + 16 i.  Eight lanes take the
        // lower 64 channels of a row and the upper 64 of its neighbour: then neither their reads nor their writes, whose chunks are permuted by
        // the row, meet in a bank.
        regs_down<C::regs_turn>();
        // (64 channels: four pieces a row, eight lanes take a row and the next.)
        constexpr int pieces = XC / 16, each = kRows * pieces / 128, apart = 128 / pieces;          // of a row; of a thread, so many rows apart
        const int t = threadIdx.x & 127, mine = (warp - 4) >> 2, q = t & (pieces - 1), row = XC == 128 ? (t >> 3) ^ (q >> 2) : t >> 2;
        constexpr int advance = 2 / C::halves;          // stages from this group's rows to its next
        const uint32_t raw = base + C::raw_at, half = C::halves == 2 ? mine * kRows : 0;
        const uint32_t from = raw + (half + row) * XC + 16 * q;
        // (a row's first scale lies at byte (row * groups + its group) % 4 of its two words, the same for rows 4 apart)
        const uint32_t scale = raw + C::rows * XC + (half + row) * 8 + (q >> 1);
        const uint32_t to = base + C::turned_at + C::split + (q >> 2) * kTile + row * 128, x0 = ((2 * (q & 3)) ^ (row & 7)) << 4;
        Walk w;
        w.start(P, group);
        if (C::halves == 1 && mine == 1 && w.live()) w.next(P, step);
        int st = mine, ph = 0, rs = C::halves == 1 ? mine : 0, rph = 0, n = mine;
        int dph = 0;
        bool ok = true, filled = false, empty = true;
        while (w.live()) {
            if (!filled) ok = mbar_wait(smem_u32(&bar_raw[rs]), rph);
            uint4 v[each];
            uint32_t s[each];
            const uint32_t sa = scale + rs * C::raw + ((row * P.groups + (w.c0 * CG + rank) * (XC / 32)) & 3);
#pragma unroll
            for (int i = 0; i < each; ++i) {
                v[i] = load_shared16(from + rs * C::raw + i * apart * XC);
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(s[i]) : "r"(sa + i * apart * 8) : "memory");
            }
            if (!empty) ok = ok && pair_wait(smem_u32(&bar_empty[st]), ph ^ 1);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const uint32_t dst = to + st * C::turned;
            const int old_st = st, old_rs = rs;
            for (st += 2; st >= C::turneds; st -= C::turneds) ph ^= 1;
            for (rs += advance; rs >= C::raws; rs -= C::raws) rph ^= 1;
            n += 2;
            filled = mbar_look(smem_u32(&bar_raw[rs]), rph);
            empty = n < C::turneds || mbar_look(smem_u32(&bar_empty[st]), ph ^ 1);
            uint32_t top = s[0];
#pragma unroll
            for (int i = 1; i < each; ++i) top = max(top, s[i]);
            const bool rest = __any_sync(0xffffffffu, act_has_rest<FMT>(top));
#pragma unroll
            for (int i = 0; i < each; ++i) {
                const uint32_t s2 = act_scale2<FMT>(s[i]);
                uint2 d[4] = {act_decode4<FMT>(v[i].x, s2), act_decode4<FMT>(v[i].y, s2), act_decode4<FMT>(v[i].z, s2), act_decode4<FMT>(v[i].w, s2)};
                if (rest) {
                    const uint32_t r = act_rest2(s[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = make_uint2(bf2_mul(d[j].x, r), bf2_mul(d[j].y, r));
                }
                store_shared16(dst + i * apart * 128 + x0, d[0].x, d[0].y, d[1].x, d[1].y);
                store_shared16(dst + i * apart * 128 + (x0 ^ 16), d[2].x, d[2].y, d[3].x, d[3].y);
            }
            if constexpr (RAW) {
                // dY: eight outputs of row t / 16 + 8 i a thread, three planes of them.  The copies come in boxes of 32 outputs, which eight lanes read two of:
                // those of the second take their 16-byte halves in the other order, into banks that the first leave free.
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_dy[mine]), dph));
                if (!ok) break;
                dph ^= 1;
                const int j = t & 15, swap = j >> 2 & 1;
                const uint32_t src = base + mine * C::dy_stage + (j >> 2) * kTile + (t >> 4) * 128 + (j & 3) * 32;
                const uint32_t out = base + C::turned_at + old_st * C::turned + (j >> 3) * kTile + (t >> 4) * 128 + (((j & 7) ^ (t >> 4 & 7)) << 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4 a = load_shared16(src + i * 1024 + 16 * swap), b = load_shared16(src + i * 1024 + 16 * (swap ^ 1));
                    const uint4 lo = swap ? b : a, hi = swap ? a : b;
                    uint32_t p0[3], p1[3], p2[3], p3[3];
                    split2(__uint_as_float(lo.x), __uint_as_float(lo.y), p0); split2(__uint_as_float(lo.z), __uint_as_float(lo.w), p1);
                    split2(__uint_as_float(hi.x), __uint_as_float(hi.y), p2); split2(__uint_as_float(hi.z), __uint_as_float(hi.w), p3);
#pragma unroll
                    for (int pl = 0; pl < 3; ++pl) store_shared16(out + pl * 2 * kTile + i * 1024, p0[pl], p1[pl], p2[pl], p3[pl]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                arrive_leader<CG>(smem_u32(&bar_full[old_st]));
                arrive(smem_u32(&bar_taken[old_rs]));
                if (RAW) arrive(smem_u32(&bar_free_dy[mine]));
            }
            w.next(P, step);
            if (C::halves == 1 && w.live()) w.next(P, step);
        }
        if (!ok) give_up();
        // the last commits have arrived before this CTA goes (bounded; they may come from the other one)
        if (ok && (warp & 3) == 0)
            for (int i = n - 2; i >= 0 && i + C::turneds >= n; i -= 2) pair_wait(smem_u32(&bar_empty[i % C::turneds]), (i / C::turneds) & 1);
    } else {
        // ---------------------------------------------------------------- sums
        // Warps w and w + 4 share 32 lanes of tensor memory (outputs) and take half of the columns (channels) each.
        regs_up<C::regs_sum>();
        constexpr int H = C::cols / 2;
        const int sp = warp & 3, half = (warp - 12) >> 2, row = 32 * sp + lane;
        float sum[H];
        Walk w;
        w.start(P, group);
        int epochs = 0;
        bool ok = true;
        while (ok && w.live()) {
            int left = w.left;
            const int unit = w.unit, k = (w.k0 * CG + rank) * 128 + row, c0 = w.c0 * C::cols + half * H;
            bool fresh = true;
            for (; left > 0; left -= C::epoch) {
                const int set = epochs & 1;
                ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&bar_acc[set]), (epochs >> 1) & 1));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (!ok) { give_up(); break; }
                const uint32_t src = tmem + set * C::cols + half * H + ((uint32_t)(32 * sp) << 16);
                if (fresh) {
#pragma unroll
                    for (int i = 0; i < H; ++i) sum[i] = 0.f;
                    fresh = false;
                }
#pragma unroll
                for (int i = 0; i < H; i += 16) {
                    float v[16];
                    tmem_ld16_nowait(src + i, v);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum[i + e] += v[e];
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_leader<CG>(smem_u32(&bar_free[set]));
                ++epochs;
            }
            if (!ok) break;
            const bool whole = unit < P.full || P.splits == 1;
            const float a = P.alpha;
            const bool sectors = P.ws_c == 1 && (P.ws_k & 7) == 0 && (P.c & 7) == 0 && (reinterpret_cast<uintptr_t>(P.dw) & 31) == 0;
            if (whole && !sectors && P.ws_c == 1) {
                // Rows of dW on any boundary: eight channels of 32 outputs turn in shared memory, and a store writes eight channels of four outputs (a lane a
                // row, 32 sectors a store, took 12 us longer on 46 rows, 1652 -> 439)
                const uint32_t buf = base + C::out_at + (warp - 12) * 1024;
                float* out = P.dw + (k - lane) * P.ws_k + c0;
#pragma unroll
                for (int i = 0; i < H; i += 8) {
                    store_shared16(buf + lane * 32, __float_as_uint(a * sum[i]), __float_as_uint(a * sum[i + 1]), __float_as_uint(a * sum[i + 2]), __float_as_uint(a * sum[i + 3]));
                    store_shared16(buf + lane * 32 + 16, __float_as_uint(a * sum[i + 4]), __float_as_uint(a * sum[i + 5]), __float_as_uint(a * sum[i + 6]), __float_as_uint(a * sum[i + 7]));
                    __syncwarp();
                    const int c = i + (lane & 7);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int o = 4 * j + (lane >> 3);
                        float v;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(buf + j * 128 + lane * 4) : "memory");
                        if (k - lane + o < P.k && c0 + c < P.c) out[o * P.ws_k + c] = v;
                    }
                    __syncwarp();
                }
            } else if (k < P.k) {
                if (!whole) {
                    // [tail unit][output][channel]
                    float* out = P.partial + ((size_t)(unit - P.full) * (128 * CG) + rank * 128 + row) * C::cols + half * H;
#pragma unroll
                    for (int i = 0; i < H; i += 8)
                        if (c0 + i < P.c)
                            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + i), "f"(sum[i]), "f"(sum[i + 1]), "f"(sum[i + 2]),
                                         "f"(sum[i + 3]), "f"(sum[i + 4]), "f"(sum[i + 5]), "f"(sum[i + 6]), "f"(sum[i + 7]) : "memory");
                } else {
                    float* out = P.dw + k * P.ws_k + c0 * P.ws_c;
#pragma unroll
                    for (int i = 0; i < H; i += 8) {
                        if (sectors && c0 + i < P.c) {
                            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + i), "f"(a * sum[i]), "f"(a * sum[i + 1]), "f"(a * sum[i + 2]),
                                         "f"(a * sum[i + 3]), "f"(a * sum[i + 4]), "f"(a * sum[i + 5]), "f"(a * sum[i + 6]), "f"(a * sum[i + 7]) : "memory");
                        } else if (!sectors) {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (c0 + i + e < P.c) out[(i + e) * P.ws_c] = a * sum[i + e];
                        }
                    }
                }
            }
            w.unit += step;
            w.enter(P);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * C::cols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * C::cols) : "memory");
    }
}

// dW of the split tiles: the sum of their splits in order.  Blocks of 256 threads: 1 << log_g groups of threads take splits g, g + G, ... of
// 256 >> log_g quads of channels; the groups' sums meet in shared memory.  grid (quads / block, tail tiles)
struct PackedReduce {
    const float* partial;
    float* dw;
    long long ws_k, ws_c;
    float alpha;
    int c, k, tile_k, tile_c, tiles_c, full, splits, log_g;
};
__global__ void __launch_bounds__(256)
packed_reduce_kernel(const __grid_constant__ PackedReduce R)
{
    __shared__ float4 s_sum[256];
    pdl_release_next_grid();
    const int G = 1 << R.log_g, per = 256 >> R.log_g, pos = threadIdx.x & (per - 1), g = threadIdx.x / per;
    const int tile = R.full + blockIdx.y, tk = tile / R.tiles_c, tc = tile - tk * R.tiles_c;
    const int quads = R.tile_c >> 2, p = blockIdx.x * per + pos, row = p / quads, q = p - row * quads;
    const int k = tk * R.tile_k + row, c = tc * R.tile_c + 4 * q;
    const bool in = k < R.k && c < R.c;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    pdl_wait_prior_grid();
    if (in) {
        const size_t block = (size_t)R.tile_k * R.tile_c;
        const float* src = R.partial + (size_t)blockIdx.y * R.splits * block + (size_t)row * R.tile_c + 4 * q;
#pragma unroll 4
        for (int s = g; s < R.splits; s += G) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(src + s * block));
            acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        }
    }
    if (G > 1) {
        s_sum[threadIdx.x] = acc;
        __syncthreads();
        if (g != 0) return;
        for (int i = 1; i < G; ++i) {
            const float4 v = s_sum[i * per + pos];
            acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        }
    }
    if (!in) return;
    float* out = R.dw + k * R.ws_k + c * R.ws_c;
    const float v[4] = {R.alpha * acc.x, R.alpha * acc.y, R.alpha * acc.z, R.alpha * acc.w};
    if (R.ws_c == 1 && (R.ws_k & 3) == 0) *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
    else
        for (int e = 0; e < 4; ++e) if (c + e < R.c) out[e * R.ws_c] = v[e];
}

// ---------------------------------------------------------------- host side
int ceil_div(int a, int b) { return (a + b - 1) / b; }

int round_up(int v, int m) { return (v + m - 1) / m * m; }

struct PackedHost { int cg, xc, f32, raw, pack, npqk, full, splits, units, grid, chunks, tiles_c, tail; };
static_assert(sizeof(PackedHost) <= sizeof(((PackedPlan*)nullptr)->opaque), "opaque");

template <int CG, int PLANES, int XC, bool RAW>
cudaError_t launch(const CUtensorMap& map_dy, const CUtensorMap& map_x, const PackedParams& P, int format, int grid, cudaStream_t stream)
{
    auto kern = format == GACONV_ACT_E4M3 ? packed_dw_kernel<CG, PLANES, XC, RAW, GACONV_ACT_E4M3> : packed_dw_kernel<CG, PLANES, XC, RAW, GACONV_ACT_INT8>;
    static std::atomic<unsigned long long> ready[2];
    const cudaError_t err = allow_shared_memory((const void*)kern, ready[format]);
    if (err != cudaSuccess) return err;
    return launch_kernel(kern, dim3((unsigned)grid), dim3(kThreads), (size_t)Config<CG, PLANES, XC, RAW>::bytes + 1024, stream, dim3(CG, 1, 1), map_dy, map_x, P);
}

}  // namespace

// The tiles that are estimated to be quickest, and splits where they are few.
// The estimate counts cycles: stages, and what a round, a split and a packing pass cost beside them (us, measured / estimated at 1.9 GHz: 512 rows 512->512
// 6.9 / 6.9, 8192 rows 1024->4096 58.6 / 56, 4099 rows 1000->1333 27.7 / 28, 131072 rows 64->64 13.4 / 14).
bool plan_packed(const Geom& g, bool dy_npqk, PackedPlan* plan, double* cycles)
{
    if (g.r != 1 || g.s != 1 || g.stride_h != 1 || g.stride_w != 1 || g.pad_h != 0 || g.pad_w != 0) return false;
    const long long rows = (long long)g.n * g.p * g.q;
    if (rows > 0x7fffff00ll || !tensor_maps_available()) return false;
    PackedHost best{};
    double best_cost = 0;
    const int sms = g.sm_budget > 0 ? std::min(g.sm_budget, device_sms()) : device_sms();
    const bool last = dy_npqk || g.k == 1 || g.p * g.q == 1;
    const bool raw_fits = !g.bf16 && last && g.k % 4 == 0;          // fp32 rows that the copy engine can read
    const int variants[6][3] = {{1, 64, 0}, {1, 128, 0}, {2, 128, 0}, {1, 64, 1}, {1, 128, 1}, {2, 128, 1}};          // CTAs of a tile, channels of each, fp32 split inside
    for (const auto& v : variants) {
        const int cg = v[0], tile_k = 128 * cg, tile_c = v[1] * cg;
        const bool raw = v[2] != 0, pack = !raw && (!g.bf16 || g.k % 8 != 0 || !last);
        if ((raw && !raw_fits) || (pack && rows * round_up(g.k, 8) > 0x7fffffffll)) continue;
        PackedHost H{};
        H.cg = cg; H.xc = v[1]; H.f32 = !g.bf16; H.raw = raw; H.pack = pack; H.npqk = last;
        const int stage_rows = g.bf16 ? kStageRows<1> : kStageRows<3>;
        H.chunks = (int)((rows + stage_rows - 1) / stage_rows);
        H.tiles_c = ceil_div(g.c, tile_c);
        const long long tiles = (long long)H.tiles_c * ceil_div(g.k, tile_k);
        if (tiles > 1 << 24) continue;
        const int clusters = std::max(1, sms / cg);
        const double fixed = raw && cg == 1 ? 5000 : 7500, block = 128.0 * tile_c * 4 / 20;
        H.full = (int)(tiles / clusters * clusters);
        const int tail = (int)(tiles - H.full);
        for (int r = 0; r <= 4; ++r) {          // no split, or as many as give the tail r rounds
            const int s = r == 0 || tail == 0 ? 1 : std::min(H.chunks, r * clusters / tail);
            if (s < 1 || (r > 0 && s == 1)) continue;
            const double rounds = std::ceil((double)tail * s / clusters), busy = std::min(1.0, (H.full + (double)tail * s) / clusters);
            // (narrow tiles load as much of dY for half the work: what L2 gives when every SM asks)
            const double stage = raw ? (cg == 2 ? 2750 : v[1] == 128 ? 2300 : 2100)
                               : H.f32 ? (cg == 2 ? 2000 : v[1] == 128 ? 1600 : 1200 + 300 * busy)
                               : cg == 2 ? 1450 : v[1] == 128 ? 1100 : 850 + 300 * busy;
            double cost = (double)(H.full / clusters) * H.chunks * stage + rounds * (ceil_div(H.chunks, s) * stage + 600) + fixed + block;
            if (pack) cost += 3000 + (double)rows * g.k * (g.bf16 ? 4.0 / 2600 : 10.0 / 3600);
            if (s > 1) cost += 5500 + (double)tail * s * tile_k * tile_c * 4 / (clusters * cg) / 20;
            if (best.units != 0 && cost >= best_cost) continue;
            best_cost = cost;
            H.splits = s; H.tail = tail;
            H.units = H.full + tail * s;
            H.grid = std::min(H.units, clusters) * cg;
            best = H;
        }
    }
    if (best.units == 0) return false;
    plan->partial_bytes = best.splits == 1 ? 0 : align_up((size_t)best.tail * best.splits * (128 * best.cg) * (best.xc * best.cg) * sizeof(float) + 256, 256);
    plan->dy_bytes = best.pack ? align_up((size_t)rows * round_up(g.k, 8) * (g.bf16 ? 2 : 6), 256) : 0;
    plan->fma = false;
    *cycles = best_cost;
    memcpy(plan->opaque, &best, sizeof(best));
    return true;
}

cudaError_t launch_packed(const void* codes, const void* scales, int format, const void* dy, float* dw, float* partial, void* dy_scratch, uint32_t* status, const Geom& g,
                          const PackedPlan& plan, cudaStream_t stream)          // partial lies on 32 bytes, dy_scratch on 16
{
    PackedHost H;
    memcpy(&H, plan.opaque, sizeof(H));
    PackedParams P{};
    P.scales = static_cast<const uint8_t*>(scales);
    P.dw = dw; P.partial = partial; P.status = status;
    P.rows = (int)((long long)g.n * g.p * g.q); P.c = g.c; P.k = g.k; P.groups = act_groups(g.c);
    P.ws_k = g.ws_k; P.ws_c = g.ws_c; P.alpha = g.alpha;
    P.tiles_c = H.tiles_c; P.full = H.full; P.splits = H.splits; P.units = H.units; P.chunks = H.chunks;
    const int kp = H.pack ? round_up(g.k, 8) : g.k, planes = H.f32 ? 3 : 1;
    cudaError_t err;
    if (H.pack) {
        if ((err = launch_pack_rows(dy, dy_scratch, g.k, kp, g.p * g.q, g.n, H.npqk != 0, H.f32 != 0, stream)) != cudaSuccess) return err;
        dy = dy_scratch;
    }
    auto encode = [&](CUtensorMap* map, CUtensorMapDataType type, const void* at, int ch, size_t pitch, int third, cuuint32_t box_ch, CUtensorMapSwizzle swz) {
        const cuuint32_t stage_rows = H.f32 ? kStageRows<3> : kStageRows<1>;
        const cuuint64_t dims[3] = {(cuuint64_t)ch, (cuuint64_t)P.rows, (cuuint64_t)third}, strides[2] = {pitch, third > 1 ? pitch * P.rows : pitch};
        const cuuint32_t box[3] = {box_ch, stage_rows, 1}, es[3] = {1, 1, 1};
        return encode_fn()(map, type, 3, const_cast<void*>(at), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swz, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    CUtensorMap map_dy, map_x;
    if (!(H.raw ? encode(&map_dy, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, dy, g.k, (size_t)g.k * 4, 1, 32, CU_TENSOR_MAP_SWIZZLE_NONE)
                : encode(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, g.k, (size_t)kp * 2, planes, 64, CU_TENSOR_MAP_SWIZZLE_128B)) ||
        !encode(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, act_pitch(g.c), act_pitch(g.c), 1, (cuuint32_t)H.xc, CU_TENSOR_MAP_SWIZZLE_NONE))
        return cudaErrorInvalidValue;
    const auto run = [&](auto* bf16, auto* f32, auto* raw) { return (H.raw ? raw : H.f32 ? f32 : bf16)(map_dy, map_x, P, format, H.grid, stream); };
    err = H.cg == 2 ? run(launch<2, 1, 128, false>, launch<2, 3, 128, false>, launch<2, 3, 128, true>)
        : H.xc == 128 ? run(launch<1, 1, 128, false>, launch<1, 3, 128, false>, launch<1, 3, 128, true>)
                      : run(launch<1, 1, 64, false>, launch<1, 3, 64, false>, launch<1, 3, 64, true>);
    if (err != cudaSuccess) return err;
    note_launch();
    if (H.splits == 1) return cudaSuccess;
    PackedReduce R{partial, dw, g.ws_k, g.ws_c, g.alpha, g.c, g.k, 128 * H.cg, H.xc * H.cg, H.tiles_c, H.full, H.splits, 0};
    while (R.log_g < 5 && 4 << R.log_g < H.splits) ++R.log_g;
    const int quads = R.tile_k * R.tile_c / 4, per = 256 >> R.log_g;
    err = launch_kernel(packed_reduce_kernel, dim3((unsigned)(quads / per), (unsigned)H.tail), dim3(256), 0, stream, dim3(1, 1, 1), R);
    if (err == cudaSuccess) note_launch();
    return err;
}

}  // namespace gaconv
