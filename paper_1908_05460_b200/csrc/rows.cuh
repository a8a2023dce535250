// Rows of fp32 or bf16 in pieces of 16 bytes, on any boundary: what the kernels that read and write rows share.
//
// A piece is 16 bytes: 8 bf16 or 4 fp32 elements.  Where rows start on 16-byte boundaries and end with a whole piece (FULL), a row is a list of
// pieces.  Otherwise a row of an odd length leaves the next one on another boundary, and there are two ways to look at it:
//   frame    pieces of memory on 16-byte boundaries; the first starts up to N - 1 elements before the row, and elements outside the row are masked.
//            Nothing has to be put together, as long as every tensor of a call has the same boundaries (strides that are alike modulo N).
//   columns  pieces of the row (what a group of an 8-bit scale needs); one is put together from the two pieces of memory that it straddles, and
//            written as the one that it shares with its neighbour, a lane up.
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
// the first `left` elements at p, one by one (all loads in flight together); zeros behind them
template <typename T>
__device__ __forceinline__ uint4 load_slowly(const T* p, int left)
{
    uint32_t e[kPiece<T>];
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) e[i] = i < left ? element_bits(p + i) : 0u;
    if constexpr (sizeof(T) == 4) return make_uint4(e[0], e[1], e[2], e[3]);
    else return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}
// v with zeros in the place of elements before `from` and from `to` on
template <typename T>
__device__ __forceinline__ uint4 only_elements(const uint4& v, int from, int to)
{
    auto word = [&](uint32_t w, int j) {
        if (sizeof(T) == 4) return j >= from && j < to ? w : 0u;
        return (2 * j >= from && 2 * j < to ? w & 0xffffu : 0u) | (2 * j + 1 >= from && 2 * j + 1 < to ? w & 0xffff0000u : 0u);
    };
    return make_uint4(word(v.x, 0), word(v.y, 1), word(v.z, 2), word(v.w, 3));
}

// A row to read: its first element and how far it and the tensor go
template <typename T, bool FULL>
struct Row {
    const T* p;
    int cols, off, room;          // cols: below every column, frames' too, for a row of nothing; off: bytes from the boundary below p; room: bytes from there to the end of the tensor (or 2^30)
    // tensor: nullptr for one that is not there (a row of nothing); live = false: a row of nothing
    __device__ __forceinline__ Row(const T* tensor, long long row, long long stride, long long rows, int columns, bool live)
    {
        live = live && tensor != nullptr;
        cols = live ? columns : -(1 << 30);
        p = tensor + (live ? row * stride : 0);
        off = FULL ? 0 : (int)(reinterpret_cast<uintptr_t>(p) & 15);
        room = FULL ? 0 : (int)min(1ll << 30, ((rows - 1 - row) * stride + columns) * (long long)sizeof(T) + off);
    }
};

// A piece of a row by columns, on its way: start() only issues loads, so that those of several pieces are in flight together; value() puts it together.
template <typename T, bool FULL>
struct Piece {
    uint4 lo, hi;
    static __device__ __forceinline__ bool straddles(const Row<T, FULL>& r, int c) { return !FULL && r.off + min(r.cols - c, kPiece<T>) * (int)sizeof(T) > 16; }
    // (a piece whose 16 or 32 bytes go past the end of the tensor is loaded element by element, in value())
    static __device__ __forceinline__ bool inside(const Row<T, FULL>& r, int c) { return FULL || c * (int)sizeof(T) + (straddles(r, c) ? 32 : 16) <= r.room; }
    __device__ __forceinline__ void start(const Row<T, FULL>& r, int c)
    {
        const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(r.p + c) - r.off);
        const bool in = c < r.cols && inside(r, c);
        lo = make_uint4(0, 0, 0, 0);
        if (in) lo = from[0];
        if (!FULL) {
            hi = make_uint4(0, 0, 0, 0);
            if (in && straddles(r, c)) hi = from[1];
        }
    }
    __device__ __forceinline__ uint4 value(const Row<T, FULL>& r, int c) const
    {
        if (FULL) return lo;
        uint4 v = shifted16(lo, hi, r.off);
        const int left = r.cols - c;
        if (left < kPiece<T>) v = only_elements<T>(v, 0, left);
        if (left > 0 && !inside(r, c)) v = load_slowly(r.p + c, min(left, kPiece<T>));
        return v;
    }
};

// A piece of a row by its frame: N elements from column c on, where c is -off / size, N - off / size, ...
template <typename T, bool FULL>
struct FramePiece {
    uint4 v;
    __device__ __forceinline__ void start(const Row<T, FULL>& r, int c)
    {
        v = make_uint4(0, 0, 0, 0);
        if (c < r.cols && (FULL || c * (int)sizeof(T) + r.off + 16 <= r.room)) v = *reinterpret_cast<const uint4*>(r.p + c);
    }
    __device__ __forceinline__ uint4 value(const Row<T, FULL>& r, int c) const
    {
        if (FULL || (c >= 0 && c + kPiece<T> <= r.cols)) return v;
        uint4 u = v;
        if (c < r.cols && c * (int)sizeof(T) + r.off + 16 > r.room) {        // the last piece of the tensor; c < 0: one row that is shorter than a piece
            u = load_slowly(r.p + max(c, 0), r.cols - max(c, 0));
            if (c < 0) u = shifted16(make_uint4(0, 0, 0, 0), u, 16 + c * (int)sizeof(T));
        }
        return only_elements<T>(u, -c, r.cols - c);
    }
};

// elements [from, to) of a piece
template <typename T>
__device__ __forceinline__ void store_slowly(T* p, const uint4& v, int from, int to)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i)
        if (i >= from && i < to) {
            if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p)[i] = w[i & 3];
            else reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(w[i >> 1] >> 16 * (i & 1));
        }
}
// Writes a piece by columns: at, its first element, of which the row has `left` elements.  All lanes of a warp call; neighbours in a stretch of
// 1 << log_lanes lanes (5: the warp) hold neighbouring pieces of a row.
template <typename T, bool FULL>
__device__ __forceinline__ void store_piece(T* at, int left, const uint4& v, int log_lanes)
{
    constexpr int N = kPiece<T>;
    if (FULL) {
        if (left > 0) *reinterpret_cast<uint4*>(at) = v;
        return;
    }
    const int off = (int)(reinterpret_cast<uintptr_t>(at) & 15), last = (1 << min(log_lanes, 5)) - 1, lane = threadIdx.x & last;
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
// Writes a piece by its frame, N elements from column c on; row: the row's first element
template <typename T, bool FULL>
__device__ __forceinline__ void store_frame(T* row, int c, int cols, const uint4& v)
{
    if (FULL ? c < cols : c >= 0 && c + kPiece<T> <= cols) *reinterpret_cast<uint4*>(row + c) = v;
    else if (!FULL && c < cols) store_slowly(row + c, v, max(0, -c), min(kPiece<T>, cols - c));
}

}  // namespace gaconv
