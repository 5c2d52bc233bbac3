// Vectors of 16 bytes at any element's address: rows of odd lengths start anywhere, and the memory path takes such accesses
// as they are (one instruction; a row that is no whole vectors apart costs the extra cache line it touches).
#pragma once
#include "dev_common.h"

namespace edl {

struct __attribute__((packed, aligned(2))) Loose16 { uint32_t w[4]; };
static_assert(sizeof(Loose16) == 16, "sixteen bytes");

template <typename T> __device__ __forceinline__ Vec16<T> load_loose(const T* p) {
    const Loose16 v = *reinterpret_cast<const Loose16*>(p);
    Vec16<T> r;
    r.u = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    return r;
}
template <typename T> __device__ __forceinline__ void store_loose(T* p, const Vec16<T>& v) {
    Loose16 s;
    s.w[0] = v.u.x; s.w[1] = v.u.y; s.w[2] = v.u.z; s.w[3] = v.u.w;
    *reinterpret_cast<Loose16*>(p) = s;
}

// A [rows][cols] matrix as pieces of kPiece neighbouring elements of a row, one per lane; a block has U times 256 pieces in a row,
// whatever rows they lie in, so that rows shorter and longer than a block fill it alike.
constexpr int kPiece = 8;
struct Pieces {
    int64_t rows, cols, per_row;       // per_row = ceil(cols / kPiece)
};
struct Piece {
    uint32_t row;                      // from the block's first row on: addresses are 32x32-bit products from there
    int64_t col;
};
// The block's first row; `at0` receives its first piece in that row.  One division for the block.
template <int U> __device__ __forceinline__ int64_t block_first_row(const Pieces& p, int64_t& at0, unsigned block) {
    const int64_t item0 = (int64_t)block * (256 * U);
    const int64_t row0 = item0 / p.per_row;
    at0 = item0 - row0 * p.per_row;
    return row0;
}
template <int U> __device__ __forceinline__ Piece piece_of(const Pieces& p, int64_t at0, int u) {
    int64_t at = at0 + u * 256 + (int)threadIdx.x;
    Piece q = {0, 0};
    if (at >= p.per_row) {
        if (p.per_row >= 256 * U) {
            at -= p.per_row;
            q.row = 1;
        } else {                       // at < 2 * 256 * U
            q.row = (unsigned)at / (unsigned)p.per_row;
            at -= q.row * (unsigned)p.per_row;
        }
    }
    q.col = at * kPiece;
    return q;
}

template <typename T> __device__ __forceinline__ void load_piece(const T* p, float (&v)[kPiece]) {
    constexpr int VEC = Elem<T>::VEC;
#pragma unroll
    for (int q = 0; q < kPiece / VEC; ++q) {
        const Vec16<T> t = load_loose(p + q * VEC);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[q * VEC + e] = Elem<T>::to_f32(t.e[e]);
    }
}
// rounded once, to nearest even
__device__ __forceinline__ void store_piece(float* p, const float (&v)[kPiece]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        Vec16<float> t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t.e[e] = v[q * 4 + e];
        store_loose(p + q * 4, t);
    }
}
__device__ __forceinline__ void store_piece(bf16_t* p, const float (&v)[kPiece]) {
    Vec16<bf16_t> t;
    t.u = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
    store_loose(p, t);
}

}  // namespace edl
