// Rows of fp32 or bf16 in pieces of 16 bytes, on any boundary: what the kernels that read and write rows share.
//
// A piece is 16 bytes of a row, counted from the row's start (8 bf16 or 4 fp32 elements).  Rows that start on 16-byte boundaries are read and written
// piece by piece.  A row of an odd length leaves the next one on another boundary; then a piece is put together from the two aligned
// 16 bytes that it straddles, and written as the aligned 16 bytes that it shares with its neighbour, one lane up: element by element only at the ends of
// a warp's stretch.  (Read and written element by element, 2 bytes at a time, rows of 4095 bf16 took three times as long as rows of 4096.)
//
// No byte past the end of a tensor is read, and none outside a row is written.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace gaconv {

template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);      // elements of a piece

// 16 bytes that start `off` bytes into a, b
__device__ __forceinline__ uint4 shifted16(const uint4& a, const uint4& b, int off)
{
    uint32_t w0 = a.x, w1 = a.y, w2 = a.z, w3 = a.w, w4 = b.x, w5 = b.y, w6 = b.z;
    if (off & 8) { w0 = w2; w1 = w3; w2 = w4; w3 = w5; w4 = w6; w5 = b.w; }
    if (off & 4) { w0 = w1; w1 = w2; w2 = w3; w3 = w4; w4 = w5; }
    const int bits = (off & 3) * 8;
    return make_uint4(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits), __funnelshift_r(w2, w3, bits), __funnelshift_r(w3, w4, bits));
}

template <typename T> __device__ __forceinline__ void to_floats(const uint4& v, float (&f)[kPiece<T>]);
template <> __device__ __forceinline__ void to_floats<float>(const uint4& v, float (&f)[4])
{
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
}
template <> __device__ __forceinline__ void to_floats<__nv_bfloat16>(const uint4& v, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
// rounds to the type
template <typename T> __device__ __forceinline__ uint4 from_floats(const float (&f)[kPiece<T>]);
template <> __device__ __forceinline__ uint4 from_floats<float>(const float (&f)[4])
{
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 from_floats<__nv_bfloat16>(const float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint32_t element_bits(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t element_bits(const __nv_bfloat16* p) { return *reinterpret_cast<const unsigned short*>(p); }
// the first `left` elements at p, one by one; zeros behind them
template <typename T>
__device__ __noinline__ uint4 load_slowly(const T* p, int left)
{
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i)
        if (i < left) w[i * sizeof(T) / 4] |= element_bits(p + i) << (i * sizeof(T) % 4 * 8);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A piece on its way.  VEC: rows start on 16-byte boundaries.  start() only issues loads, so that those of several pieces are in flight together;
// value() puts the piece together.  at: the piece's first element; left: elements of the row from there (may be negative); end: of the tensor.
template <typename T, bool VEC>
struct Piece {
    uint4 lo, hi;
    __device__ __forceinline__ void start(const T* at, int left, const T* end)
    {
        lo = make_uint4(0, 0, 0, 0);
        if (VEC) {
            if (left >= kPiece<T>) lo = *reinterpret_cast<const uint4*>(at);
        } else {
            hi = make_uint4(0, 0, 0, 0);
            const int off = (int)(reinterpret_cast<uintptr_t>(at) & 15);
            const char* from = reinterpret_cast<const char*>(at) - off;
            const bool all = left >= kPiece<T> && from + (off ? 32 : 16) <= reinterpret_cast<const char*>(end);
            if (all) lo = *reinterpret_cast<const uint4*>(from);
            if (all && off) hi = *reinterpret_cast<const uint4*>(from + 16);
        }
    }
    __device__ __forceinline__ uint4 value(const T* at, int left, const T* end) const
    {
        uint4 v = lo;
        if (VEC) {
            if (left > 0 && left < kPiece<T>) v = load_slowly(at, left);
        } else {
            const int off = (int)(reinterpret_cast<uintptr_t>(at) & 15);
            v = shifted16(lo, hi, off);
            if (left > 0 && (left < kPiece<T> || reinterpret_cast<const char*>(at) - off + (off ? 32 : 16) > reinterpret_cast<const char*>(end))) v = load_slowly(at, left);
        }
        return v;
    }
};

template <typename T>
__device__ __noinline__ void store_slowly(T* p, uint4 v, int from, int to)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i)
        if (i >= from && i < to) {
            const uint32_t bits = w[i * sizeof(T) / 4] >> (i * sizeof(T) % 4 * 8);
            if (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p + i) = bits;
            else *reinterpret_cast<unsigned short*>(p + i) = (unsigned short)bits;
        }
}
// Writes the piece at `at`, of which the row has `left` elements.  All lanes of a warp call; neighbours in a stretch of 1 << log_lanes lanes (5: the
// warp) hold neighbouring pieces of a row.
template <typename T, bool VEC>
__device__ __forceinline__ void store_piece(T* at, int left, const uint4& v, int log_lanes)
{
    constexpr int N = kPiece<T>;
    if (VEC) {
        if (left >= N) *reinterpret_cast<uint4*>(at) = v;
        else if (left > 0) store_slowly(at, v, 0, left);
        return;
    }
    const int off = (int)(reinterpret_cast<uintptr_t>(at) & 15), lane = threadIdx.x & ((1 << min(log_lanes, 5)) - 1), last = (1 << min(log_lanes, 5)) - 1;
    const int head = (16 - off) / (int)sizeof(T);            // elements up to the next boundary
    uint4 p;
    p.x = __shfl_up_sync(0xffffffffu, v.x, 1); p.y = __shfl_up_sync(0xffffffffu, v.y, 1);
    p.z = __shfl_up_sync(0xffffffffu, v.z, 1); p.w = __shfl_up_sync(0xffffffffu, v.w, 1);
    const bool whole = off == 0 ? left >= N : lane > 0 && left >= head;      // the 16 bytes that end or start with this piece's head
    const bool next = __shfl_down_sync(0xffffffffu, (int)whole, 1) != 0 && lane < last;
    if (whole) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(at) - off) = off == 0 ? v : shifted16(p, v, 16 - off);
    if (left > 0) {
        const int from = whole ? head : 0, to = off != 0 && next ? head : min(left, N);
        if (from < to) store_slowly(at, v, from, to);
    }
}

}  // namespace gaconv
