// Dropout whose mask is never stored: whether an element stays is a function of (key, row number, column), computed where
// it is needed, forward and backward alike.
//
// The generator is the library's counter-based one (SplitMix64: draw j of a stream is the finaliser of key + (j+1) golden),
// 64 bits for two neighbouring columns: row R has its ceil(cols / 2) draws from R * ceil(cols / 2) on, the low half of a
// draw for its even column, the high half for the odd one.  An element is dropped if its 32 bits are below rate * 2^32.
//
// Bound: the element is read and written once; the arithmetic is close behind (a finaliser is two 64-bit products,
// about 40 issue slots of full-rate instructions for two elements, against the 48 that bf16 traffic at 6 TB/s leaves).
// Measured: 16,384 x 8,192 bf16 100 us (5.4 TB/s; a plain copy reaches 6.2), 2,049 x 4,097 float32 in rows of 4,104 14 us (4.7 TB/s),
// 32 x 4,096 bf16 2.9 us.
#include <algorithm>

#include "graph.h"
#include "operators.h"
#include "profiler.h"
#include "unaligned.h"

namespace edl {

namespace {

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;
static_assert(kPiece == 8, "a lane's piece is four draws");
constexpr int64_t kSmallItems = 1 << 18;   // calls of fewer lanes' worth take one piece per lane

__device__ __forceinline__ uint64_t finalise(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

struct DropoutArgs {
    Pieces m;
    int64_t ldx, ldy;
    uint64_t key1, pairs;      // key + golden; draws per row
    uint64_t first_row;
    uint32_t threshold;
    float scale;
};

// Products stay in float32 and are rounded once, to nearest even.  U = 4 has four loads in flight and divides once for four pieces (the
// division of the block's first piece by the pieces of a row takes as long as half a piece's draws); small calls take
// U = 1, which spreads them over four times the compute units.
template <typename T, int U>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, T* y, DropoutArgs a) {
    int64_t at0;
    const int64_t row0 = block_first_row<U>(a.m, at0, blockIdx.x);
    // addresses and draws from the block's first row on, which are the same for all lanes, in 32x32-bit products
    const T* const x0 = x + row0 * a.ldx;
    T* const y0 = y + row0 * a.ldy;
    const uint64_t j0 = (a.first_row + (uint64_t)row0) * a.pairs;
    const int64_t rows_left = a.m.rows - row0;
    Piece q[U];
    float v[U][kPiece];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        q[u] = piece_of<U>(a.m, at0, u);
        if (q[u].row < rows_left && q[u].col + kPiece <= a.m.cols) load_piece(x0 + (uint64_t)q[u].row * (uint32_t)a.ldx + q[u].col, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (q[u].row >= rows_left) return;
        const uint64_t j = j0 + (uint64_t)q[u].row * (uint32_t)a.pairs + (uint64_t)q[u].col / 2;
        const uint64_t z = a.key1 + j * kGolden;
        uint32_t bits[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece / 2; ++i) {
            const uint64_t d = finalise(z + (uint64_t)i * kGolden);
            bits[2 * i] = (uint32_t)d;
            bits[2 * i + 1] = (uint32_t)(d >> 32);
        }
        T* py = y0 + (uint64_t)q[u].row * (uint32_t)a.ldy + q[u].col;
        if (q[u].col + kPiece <= a.m.cols) {
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[u][e] = bits[e] >= a.threshold ? v[u][e] * a.scale : 0.f;
            store_piece(py, v[u]);
        } else {
            const T* px = x0 + (uint64_t)q[u].row * (uint32_t)a.ldx + q[u].col;
            const int n = (int)(a.m.cols - q[u].col);
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                if (e < n) py[e] = Elem<T>::from_f32(bits[e] >= a.threshold ? Elem<T>::to_f32(px[e]) * a.scale : 0.f);
        }
    }
}

}  // namespace

void launch_dropout(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, float rate, uint64_t key,
                    uint64_t first_row, hipStream_t st) {
    if (rows <= 0 || cols <= 0) return;
    DropoutArgs a;
    a.ldx = ldx;
    a.ldy = ldy;
    a.m = Pieces{rows, cols, (cols + kPiece - 1) / kPiece};
    a.key1 = key + kGolden;
    a.pairs = ((uint64_t)cols + 1) / 2;
    a.first_row = first_row;
    a.threshold = (uint32_t)((double)rate * 4294967296.0);
    a.scale = (float)(1.0 / (1.0 - (double)rate));
    const double esz = dtype == 1 ? 2.0 : 4.0;
    ProfScope ps("dropout", 0.0, 2.0 * esz * (double)rows * (double)cols, st);
    const int64_t items = rows * a.m.per_row;                    // (up to 2^33, as ldx and ldy are below 2^31: checked by the caller)
    const bool small = items < kSmallItems;
    const unsigned grid = (unsigned)((items + (small ? 255 : 1023)) / (small ? 256 : 1024));
#define EDL_DROPOUT(TT, UU) hipLaunchKernelGGL((dropout_kernel<TT, UU>), dim3(grid), dim3(256), 0, st, (const TT*)x, (TT*)y, a)
    if (dtype == 1) { if (small) EDL_DROPOUT(bf16_t, 1); else EDL_DROPOUT(bf16_t, 4); }
    else { if (small) EDL_DROPOUT(float, 1); else EDL_DROPOUT(float, 4); }
#undef EDL_DROPOUT
}

// Streams of keys that differ by a multiple of golden are shifted copies of each other, so keys are draws themselves.
uint64_t dropout_key(uint64_t seed, int64_t step, int layer) {
    return splitmix64_at(splitmix64_at(seed ^ 0x5D6C1F3A9B27E841ull, (uint64_t)step), (uint64_t)layer);
}

}  // namespace edl
