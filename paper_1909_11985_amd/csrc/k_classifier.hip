// Log probabilities of given classes straight from features and classifier weights, and the gradients of both, without
// the logits in memory.
//
//   z = x w^T + b                       [rows][classes], formed tile by tile
//   lse, entropy, log_prob              from each tile's sums (softmax_sums.h), joined over the tiles of a row
//   dz = g (1[c = t] - p) - h p (log p + H),  dx = dz w,  dw = dz^T x,  db = sum of dz over the rows
//
// Four products, one kernel (gemm_kernel) on 32x32 matrix instructions.  An operand lies with the reduction along its rows
// (x and w in z, dz in dx) or across them (dz and x in dw, w in dx); either is brought to LDS as it lies, and a fragment of
// the second kind is read transposed, so nothing is transposed in memory.  z is formed as w x^T: a lane then has one row's
// classes, 16 to a 32x32 tile, and the sums over classes stay inside it.
//
// The gradient forms z again rather than keep it, a piece of the classes at a time.  dz is stored for the two products that
// read it: in float32 as it is, in bf16 as a sum of three bf16 numbers (24 bits), because dw is float32 and a single
// rounding of dz would be its largest error by four orders of magnitude; dx, which is rounded to bf16, takes the first two.
#include <algorithm>
#include <type_traits>

#include "operators.h"
#include "profiler.h"
#include "softmax_sums.h"
#include "unaligned.h"

namespace edl {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;        // of a reduction step along a row
constexpr int kTile = 128, kBigTile = 256;     // rows and columns of a block's tile

// ---- operands ---------------------------------------------------------------------------------------------------------
// 16 bytes per lane from memory to LDS: lane l's go to lds_wave_base + 16 l; lanes whose offset lies past the descriptor's
// extent get zeros.  Issued from assembly, so that the compiler does not wait for it at every LDS access: wait_loads and a
// barrier order it.
constexpr unsigned kNowhere = 0x80000000u;       // past any extent (they are clamped below it)
__device__ __forceinline__ i32x4 extent_of(const char* p, int64_t bytes) {
    const uint64_t a = (uint64_t)p;
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };       // (they are: the compiler has lost track)
    const i32x4 r = {same((int)(uint32_t)a), same((int)(uint32_t)(a >> 32)), same((int)min(bytes, (int64_t)0x7ffffff0)), 0x00020000};
    return r;
}
__device__ __forceinline__ void load16_to_lds(i32x4 extent, unsigned lds_wave_base, unsigned offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_wave_base), "v"(offset), "s"(extent) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// One operand of a product: `rows` of it matter, `k` elements of the reduction.  along: row r's reduction lies at
// p + r * ld; otherwise element (r, k) is at p + k * ld + r.  Bytes; p, ld and the bytes of a row are multiples of 16
// and hold zeros past the operand's elements.
struct Operand {
    const char* p;
    int64_t ld;
    int64_t rows;
};

// A tile of W rows and one reduction step in LDS.
//   along: [W][128 bytes], the 16-byte pieces of a row permuted by the row's bits 1 to 3: of 16 rows, whose same piece the lanes
//     of a read ask for together, each then lies in banks of its own (two rows cover them; by bits 0 to 2, rows 8 apart met)
//   across, bf16: [64 k][W] with the 32-byte pieces of a k permuted by its low bits: a transposing read takes two
//     neighbouring pieces of four consecutive k, which then fall into different banks
//   across, float32: [32 k][W] as it is
template <typename T, bool ALONG, int W, int THREADS> struct Tile {
    static constexpr int ESZ = (int)sizeof(T), STEP = kStepBytes / ESZ, BYTES = W * kStepBytes;
    static constexpr int PIECES = ALONG ? 8 : W * ESZ / 16;            // 16-byte pieces of a line
    static constexpr int LOADS = BYTES / 16 / THREADS;                 // per lane
    static_assert(BYTES % (16 * THREADS) == 0, "whole loads");

    unsigned offset[LOADS];      // this lane's, from the step's start
    unsigned piece_at;           // along: where in the step this lane's pieces lie (the same for all its loads)
    // of the step that is loaded next: where it starts, bytes of the operand from there on, bytes of a row's reduction
    const char* next;
    int64_t left, stride;
    int row_left;

    __device__ __forceinline__ static int swizzle(int k) { return W >= 128 ? (k & 3) << 1 : k & 3; }

    __device__ __forceinline__ void init(const Operand& o, int64_t first_row, int row_bytes) {
        stride = ALONG ? kStepBytes : STEP * o.ld;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int slot = i * THREADS + (int)threadIdx.x, line = slot / PIECES, s = slot % PIECES;
            if (ALONG) {
                const int piece = s ^ ((line >> 1) & 7);
                offset[i] = (unsigned)(line * o.ld) + piece * 16;
                if (i == 0) piece_at = piece * 16;         // (THREADS / 8 lines further on those bits are the same)
            } else {
                const int piece = ESZ == 2 ? ((((s >> 1) ^ swizzle(line)) << 1) | (s & 1)) : s;
                const bool there = first_row * ESZ + piece * 16 < row_bytes;
                offset[i] = there ? (unsigned)(line * o.ld) + piece * 16 : kNowhere;
            }
        }
    }
    // from step s on, of `k` elements of the reduction in all; plane: bytes to the operand's plane
    __device__ __forceinline__ void start(const Operand& o, int64_t plane, int64_t first_row, int row_bytes, int64_t k, int64_t s) {
        k -= s * STEP;
        next = o.p + plane + (ALONG ? first_row * o.ld : first_row * ESZ) + s * stride;
        left = ALONG ? (o.rows - first_row - 1) * o.ld + k * ESZ : (k - 1) * o.ld + row_bytes - first_row * ESZ;
        row_left = (int)min(k * ESZ, (int64_t)0x7ffffff0);
    }
    __device__ __forceinline__ void load(unsigned lds) {
        const i32x4 e = extent_of(next, left);
        const unsigned wave = (unsigned)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            unsigned at = offset[i];
            if (ALONG) at = (int)piece_at < row_left ? at : kNowhere;
            load16_to_lds(e, lds + wave + i * THREADS * 16, at);
        }
        next += stride;
        left -= stride;
        if (ALONG) row_left -= kStepBytes;
    }
    // Fragment of rows [r32, r32 + 32) for the g-th eighth of 16 bytes x 2 of the step: a lane has row r32 + lane % 32 and
    // the half of the group's reduction that lane / 32 names (bf16: 8 elements, float32: 4, each for one of 4 instructions)
    __device__ __forceinline__ static uint4 fragment(const char* tile, int r32, int g, int lane) {
        if constexpr (ALONG) {
            const int r = r32 + (lane & 31);
            return *reinterpret_cast<const uint4*>(tile + r * kStepBytes + (((2 * g + (lane >> 5)) ^ ((r >> 1) & 7)) << 4));
        } else if constexpr (ESZ == 2) {
            // the transposing read hands lane l of 16 lanes element l of the 16 channels of a piece, for four consecutive k
            // whose lines lanes 4q .. 4q + 3 address, eight bytes each
            typedef shortx4 __attribute__((address_space(3))) * lds_ptr;
            const int ch = r32 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3), k = g * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
            auto at = [&](int kk) { return (lds_ptr)(tile + (kk * W + ((((ch >> 4) ^ swizzle(kk)) << 4) | (ch & 15))) * 2); };
            const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k)));
            const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k + 4)));
            return make_uint4(a.x, a.y, b.x, b.y);
        } else {
            const uint32_t* q = reinterpret_cast<const uint32_t*>(tile) + (g * 8 + (lane >> 5) * 4) * W + r32 + (lane & 31);
            return make_uint4(q[0], q[W], q[2 * W], q[3 * W]);
        }
    }
};

template <typename T> __device__ __forceinline__ void multiply(const uint4& a, const uint4& b, floatx16& c) {
    if constexpr (sizeof(T) == 2) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
}
// sum of a fragment's elements of this lane
template <typename T> __device__ __forceinline__ float fragment_sum(const uint4& f) {
    Vec16<T> v;
    v.u = f;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < Elem<T>::VEC; ++e) s += Elem<T>::to_f32(v.e[e]);
    return s;
}
// row of a 32x32 tile that element e of a lane's 16 stands for (its column is lane % 32)
__device__ __forceinline__ int tile_row(int e, int lane) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }

// the next of the bf16 numbers that four floats are the sums of, 8 bits each; what is left of them stays in v
__device__ __forceinline__ uint2 next_bf16(float (&v)[4]) {
    const uint2 b = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
    v[0] -= __uint_as_float(b.x << 16);
    v[1] -= __uint_as_float(b.x & 0xffff0000u);
    v[2] -= __uint_as_float(b.y << 16);
    v[3] -= __uint_as_float(b.y & 0xffff0000u);
    return b;
}

// four neighbouring classes of a row of dz
template <typename T> __device__ __forceinline__ void store_dz(char* p, int64_t plane, const float (&d)[4]) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(d[0], d[1], d[2], d[3]);
    } else {
        float v[4] = {d[0], d[1], d[2], d[3]};
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(p + q * plane) = next_bf16(v);
    }
}

enum Want { SUMS, GRADS, PRODUCT };     // of z: sums over classes, dz; of the others: the product itself

struct GemmArgs {
    Operand a, b;
    int64_t a_k, b_k;          // elements of the reduction that lie there (an operand along it has them up to whole 16 bytes)
    int64_t a_plane;           // bytes between the numbers that a's elements are the sum of
    int planes;
    int a_row_bytes, b_row_bytes;      // of an operand that lies across
    int steps, steps_per_cut;  // of the reduction; a cut of it is a block's
    int tiles_m, tiles_n, group;
    // z: a = w from class `first_class` on, b = x
    const float* bias;
    int64_t first_class, classes, all_classes;     // classes: the end of this launch's
    RowFacts facts;
    float4* sums;              // [tile of classes][rows]: m, s, t
    float* target_z;
    char* dz;                  // [planes][rows][dz_ld], of the classes from first_class on
    int64_t dz_ld, dz_plane;   // bytes
    int dz_classes;            // columns of dz that are written (zeros past the last class)
    // products
    void* out;                 // [cut][a.rows][out_ld]
    int64_t out_ld, out_cut;   // elements
    float* dbias;              // [cut][a.rows] sums of a over the reduction; null: none
    int64_t dbias_cut;
};

// (tile of a's rows, of b's rows, cut).  Consecutive blocks go to the eight dies in turn; a die's blocks are made
// neighbours, `group` tiles of a by all of b, so that what they share stays in its L2.
__device__ __forceinline__ void tile_of(const GemmArgs& g, int& tm, int& tn, int& cut) {
    const unsigned per_cut = (unsigned)g.tiles_m * (unsigned)g.tiles_n, total = gridDim.x;
    const unsigned q = total >> 3, r = total & 7, die = blockIdx.x & 7;
    unsigned l = die * q + min(die, r) + (blockIdx.x >> 3);
    cut = (int)(l / per_cut);
    l -= (unsigned)cut * per_cut;
    const unsigned wide = (unsigned)g.group * (unsigned)g.tiles_n, block = l / wide;
    const unsigned first = block * (unsigned)g.group, high = min((unsigned)g.group, (unsigned)g.tiles_m - first);
    l -= block * wide;
    tn = (int)(l / high);
    tm = (int)(first + l - (unsigned)tn * high);
}

// A block's waves, WM x WN, and a wave's 32x32 tiles, TM x TN.  64x64 to a wave read 4 KB of LDS for every 4 matrix
// instructions, 128x64 read 6 KB for 8; what the larger tile needs is enough of them for the chip.
struct Shape128 { static constexpr int WM = 2, WN = 2, TM = 2, TN = 2; };
struct Shape256 { static constexpr int WM = 2, WN = 4, TM = 4, TN = 2; };

template <typename T, Want WANT, bool A_ALONG, bool B_ALONG, typename OUT, typename SHAPE>
__global__ __launch_bounds__(SHAPE::WM * SHAPE::WN * 64) void gemm_kernel(GemmArgs g) {
    constexpr int WM = SHAPE::WM, WN = SHAPE::WN, TM = SHAPE::TM, TN = SHAPE::TN, THREADS = WM * WN * 64;
    constexpr int MT = WM * TM * 32, NT = WN * TN * 32;
    typedef Tile<T, A_ALONG, MT, THREADS> TA;
    typedef Tile<T, B_ALONG, NT, THREADS> TB;
    constexpr int STAGE = TA::BYTES + TB::BYTES, STEP = TA::STEP;
    __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    int tm, tn, cut;
    tile_of(g, tm, tn, cut);
    const int64_t m0 = (int64_t)tm * MT, n0 = (int64_t)tn * NT;
    TA ta;
    TB tb;
    ta.init(g.a, m0, g.a_row_bytes);
    tb.init(g.b, n0, g.b_row_bytes);
    const int first = cut * g.steps_per_cut, last = min(first + g.steps_per_cut, g.steps), steps = last - first, all = steps * g.planes;
    int at = steps, plane = 0;                              // steps of this plane that are still to be loaded
    ta.start(g.a, 0, m0, g.a_row_bytes, g.a_k, first);
    tb.start(g.b, 0, n0, g.b_row_bytes, g.b_k, first);
    auto load = [&](int stage) {
        if (at == 0) {
            at = steps;
            ++plane;
            ta.start(g.a, plane * g.a_plane, m0, g.a_row_bytes, g.a_k, first);
            tb.start(g.b, 0, n0, g.b_row_bytes, g.b_k, first);
        }
        --at;
        ta.load(lds + stage * STAGE);
        tb.load(lds + stage * STAGE + TA::BYTES);
    };
    floatx16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    float a_sum[TM] = {};
    const bool sum_a = WANT == PRODUCT && g.dbias != nullptr && tn == 0 && wn == 0;
    // Two stages of LDS.  Fragments are read one group of instructions ahead, the first ones of the next step before the last
    // group of this one: by then all waves have read the rest of this step, so the barrier that says the next step is there also
    // frees this one's stage for the step after it.  (The scheduling barriers keep the compiler from moving the reads back.)
    auto contract_all = [&](auto with_sum) {
        if (all <= 0) return;
        uint4 fa[2][TM], fb[2][TN];
        auto read = [&](int stage, int q) {
            const char* const A = smem + stage * STAGE;
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[q & 1][i] = TA::fragment(A, (wm * TM + i) * 32, q, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[q & 1][j] = TB::fragment(A + TA::BYTES, (wn * TN + j) * 32, q, lane);
        };
        load(0);
        wait_loads<0>();
        __syncthreads();
        if (all > 1) load(1);
        read(0, 0);
        for (int t = 0; t < all; ++t) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (q < 3) {
                    read(t & 1, q + 1);
                } else if (t + 1 < all) {
                    wait_loads<0>();
                    __syncthreads();
                    if (t + 2 < all) load(t & 1);
                    read((t + 1) & 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) multiply<T>(fa[q & 1][i], fb[q & 1][j], acc[i][j]);
                if constexpr (decltype(with_sum)::value) {
#pragma unroll
                    for (int i = 0; i < TM; ++i) a_sum[i] += fragment_sum<T>(fa[q & 1][i]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();           // LDS is free
    };
    if (WANT == PRODUCT && sum_a) contract_all(std::true_type{});
    else contract_all(std::false_type{});
    if constexpr (WANT == PRODUCT) {
        OUT* const out = (OUT*)g.out + cut * g.out_cut;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + (wn * TN + j) * 32 + (lane & 31);
            if (n >= g.b.rows) continue;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int64_t m = m0 + (wm * TM + i) * 32 + tile_row(e, lane);
                    if (m < g.a.rows) out[m * g.out_ld + n] = Elem<OUT>::from_f32(acc[i][j][e]);
                }
        }
        if (sum_a) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const float s = a_sum[i] + __shfl_xor(a_sum[i], 32, 64);
                const int64_t m = m0 + (wm * TM + i) * 32 + (lane & 31);
                if (lane < 32 && m < g.a.rows) g.dbias[cut * g.dbias_cut + m] = s;
            }
        }
    } else {
        // z: rows of the tile are classes, columns rows of x
        // class of element e of tile i: c0 + 32 i + 8 (e / 4) + e % 4; those from c0 + left on are none
        const int64_t c0 = g.first_class + m0 + wm * TM * 32 + 4 * (lane >> 5);
        const int left = (int)min((int64_t)4096, g.classes - c0);
        auto place = [](int i, int e) { return 32 * i + 8 * (e >> 2) + (e & 3); };
        float bias[TM][16];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) bias[i][e] = g.bias != nullptr && place(i, e) < left ? g.bias[c0 + place(i, e)] : 0.f;
        if constexpr (WANT == SUMS) {
            __syncthreads();                   // LDS is the sums' now
            float4* const part = reinterpret_cast<float4*>(smem);      // [wm][NT]
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int col = (wn * TN + j) * 32 + (lane & 31);
                const int64_t n = n0 + col;
                const int64_t t = n < g.b.rows && g.facts.targets != nullptr ? g.facts.targets[n] : -1;
                const int hot = t >= c0 && t < c0 + left ? (int)(t - c0) : -1;
                SoftmaxSums s;
                float zt = 0.f;
                bool here = false;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float z = place(i, e) < left ? acc[i][j][e] + bias[i][e] : -INFINITY;
                        acc[i][j][e] = z;
                        s.m = fmaxf(s.m, z);
                        if (place(i, e) == hot) { zt = z; here = true; }
                    }
                const float base = softmax_base(s);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) softmax_add(s, acc[i][j][e], base);
                softmax_join(s, softmax_shuffle(s, 32));
                if (lane < 32) part[wm * NT + col] = make_float4(s.m, s.s, s.t, 0.f);
                if (here) g.target_z[n] = zt;
            }
            __syncthreads();
            if (threadIdx.x < NT && n0 + threadIdx.x < g.b.rows) {
                SoftmaxSums s;
#pragma unroll
                for (int w = 0; w < WM; ++w) {
                    const float4 p = part[w * NT + threadIdx.x];
                    SoftmaxSums o;
                    o.m = p.x; o.s = p.y; o.t = p.z;
                    softmax_join(s, o);
                }
                g.sums[tm * g.b.rows + n0 + threadIdx.x] = make_float4(s.m, s.s, s.t, 0.f);
            }
        } else {
            // dz goes out through LDS, a plane at a time, so that rows are written in whole lines: [NT rows][MT classes] with the
            // 16-byte pieces of a row permuted by its low bits (32 lanes write one piece of 32 rows)
            constexpr int PLANES = sizeof(T) == 2 ? 3 : 1, PIECES = MT * (int)sizeof(T) / 16;
            static_assert(NT * MT * (int)sizeof(T) <= 2 * STAGE, "a plane fits");
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t n = n0 + (wn * TN + j) * 32 + (lane & 31);
                const LogitGrad row = logit_grad(g.facts, min(n, g.b.rows - 1), g.all_classes);
                const int hot = row.target >= c0 && row.target < c0 + left ? (int)(row.target - c0) : -1;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = place(i, e) < left ? row.of(acc[i][j][e] + bias[i][e], place(i, e) == hot) : 0.f;
            }
            const int wide = (int)min((int64_t)MT, g.dz_classes - m0) * (int)sizeof(T) / 16;       // pieces of a row that are written
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                __syncthreads();           // LDS is free: of the product's tiles, then of the plane before
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int r = (wn * TN + j) * 32 + (lane & 31);
                    char* const line = smem + r * (MT * (int)sizeof(T));
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int byte = ((wm * TM + i) * 32 + 8 * q + 4 * (lane >> 5)) * (int)sizeof(T);
                            char* const to = line + (((byte >> 4) ^ (r & (PIECES - 1))) << 4) + (byte & 15);
                            float d[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) d[e] = acc[i][j][4 * q + e];
                            if constexpr (sizeof(T) == 4) {
                                *reinterpret_cast<float4*>(to) = make_float4(d[0], d[1], d[2], d[3]);
                            } else {
                                *reinterpret_cast<uint2*>(to) = next_bf16(d);
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = d[e];
                            }
                        }
                }
                __syncthreads();
                char* const out = g.dz + p * g.dz_plane + n0 * g.dz_ld + m0 * (int64_t)sizeof(T);
                for (int s = threadIdx.x; s < NT * PIECES; s += THREADS) {
                    const int r = s / PIECES, c = s % PIECES;
                    if (n0 + r < g.b.rows && c < wide)
                        *reinterpret_cast<uint4*>(out + r * g.dz_ld + c * 16) = *reinterpret_cast<const uint4*>(smem + (r * PIECES + (c ^ (r & (PIECES - 1)))) * 16);
                }
            }
        }
    }
}

// ---- few tiles ----------------------------------------------------------------------------------------------------------
// Where z has too few tiles to fill the chip it is formed in 32x32 tiles with the reduction cut as well, over a block's four
// waves and over blocks, and its float32 parts are stored: [cut][rows][z_ld].  Fragments come straight from memory (L2: a
// tile is used by few); what that bounds is the latency of the chain of loads, so each wave has eight in flight.
struct ThinArgs {
    Operand w, x;
    int64_t k;                 // up to whole 16 bytes
    int steps, steps_per_wave, tiles_m, tiles_n;
    float* z;
    int64_t z_ld;
};
template <typename T> __global__ __launch_bounds__(256) void thin_logits_kernel(ThinArgs g) {
    __shared__ float part[4][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned l = blockIdx.x;
    const int tn = (int)(l % (unsigned)g.tiles_n);
    l /= (unsigned)g.tiles_n;
    const int tm = (int)(l % (unsigned)g.tiles_m), cut = (int)(l / (unsigned)g.tiles_m);
    const int64_t m = min((int64_t)tm * 32 + (lane & 31), g.w.rows - 1), n = min((int64_t)tn * 32 + (lane & 31), g.x.rows - 1);
    const int first = (cut * 4 + wave) * g.steps_per_wave, last = min(first + g.steps_per_wave, g.steps);
    const int64_t end = g.k * (int64_t)sizeof(T);
    int64_t at = (int64_t)first * kStepBytes + 16 * (lane >> 5);
    const char* const a = g.w.p + m * g.w.ld;
    const char* const b = g.x.p + n * g.x.ld;
    floatx16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    for (int s = first; s < last; ++s, at += kStepBytes) {
        uint4 fa[4], fb[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool in = at + 32 * q < end;
            const int64_t from = in ? at + 32 * q : 0;      // (row starts are always there)
            fa[q] = *reinterpret_cast<const uint4*>(a + from);
            fb[q] = *reinterpret_cast<const uint4*>(b + from);
            if (!in) fa[q] = fb[q] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) multiply<T>(fa[q], fb[q], acc);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) part[wave][e][lane] = acc[e];
    __syncthreads();
    const int64_t row = (int64_t)tn * 32 + (lane & 31);
    if (row >= g.x.rows) return;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = 4 * wave + e;
        v[e] = (part[0][i][lane] + part[1][i][lane]) + (part[2][i][lane] + part[3][i][lane]);
    }
    *reinterpret_cast<float4*>(g.z + (cut * g.x.rows + row) * g.z_ld + tm * 32 + 8 * wave + 4 * (lane >> 5)) = make_float4(v[0], v[1], v[2], v[3]);
}

struct ThinRows {
    const float* z;
    int64_t z_ld, rows, classes;
    int cuts;
    const float* bias;
    RowFacts facts;
};
// four neighbouring logits (classes past the last: whatever lies there)
__device__ __forceinline__ float4 thin_logits(const ThinRows& g, int64_t row, int64_t c) {
    float4 v = *reinterpret_cast<const float4*>(g.z + row * g.z_ld + c);
    for (int q = 1; q < g.cuts; ++q) {
        const float4 p = *reinterpret_cast<const float4*>(g.z + (q * g.rows + row) * g.z_ld + c);
        v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
    }
    if (g.bias != nullptr) {
        v.x += g.bias[c];
        if (c + 1 < g.classes) v.y += g.bias[c + 1];
        if (c + 2 < g.classes) v.z += g.bias[c + 2];
        if (c + 3 < g.classes) v.w += g.bias[c + 3];
    }
    return v;
}
struct RowResults { float *log_prob, *entropy, *lse; };
__device__ __forceinline__ void write_results(const RowResults& out, const int32_t* targets, int64_t classes, int64_t row, const SoftmaxSums& s, float zt) {
    out.lse[row] = softmax_lse(s);
    out.entropy[row] = softmax_entropy(s);
    if (targets == nullptr) return;
    const int32_t t = targets[row];
    out.log_prob[row] = t >= 0 && t < classes ? softmax_log_prob(s, zt) : 0.f;
}
// Sums of a part of a row's classes; of all of them, the results.
__global__ __launch_bounds__(256) void thin_sums_kernel(ThinRows g, int parts, int64_t part, float4* sums, float* target_z, RowResults out) {
    __shared__ float4 wave_sums[4];
    __shared__ float target;
    const int64_t row = blockIdx.x / (unsigned)parts;
    const int p = (int)(blockIdx.x - (unsigned)row * (unsigned)parts);
    const int64_t lo = p * part, hi = min(lo + part, g.classes);
    const int64_t t = g.facts.targets != nullptr ? g.facts.targets[row] : -1;
    SoftmaxSums s;
    for (int64_t c = lo + threadIdx.x * 4; c < hi; c += 1024) {
        const float4 v = thin_logits(g, row, c);
        float z[4] = {v.x, v.y, v.z, v.w}, m = s.m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= hi) z[e] = -INFINITY;
            m = fmaxf(m, z[e]);
            if (c + e == t && c + e < hi) {
                if (parts == 1) target = z[e];
                else target_z[row] = z[e];
            }
        }
        softmax_rebase(s, m);
        const float base = softmax_base(s);
#pragma unroll
        for (int e = 0; e < 4; ++e) softmax_add(s, z[e], base);
    }
    softmax_join_wave(s);
    if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = make_float4(s.m, s.s, s.t, 0.f);
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 4; ++w) {
        SoftmaxSums o;
        o.m = wave_sums[w].x; o.s = wave_sums[w].y; o.t = wave_sums[w].z;
        softmax_join(s, o);
    }
    if (parts == 1) write_results(out, g.facts.targets, g.classes, row, s, target);
    else sums[p * g.rows + row] = make_float4(s.m, s.s, s.t, 0.f);
}
// dz of such logits: a lane has four neighbouring classes
template <typename T> __global__ __launch_bounds__(256) void thin_grads_kernel(ThinRows g, char* dz, int64_t dz_ld, int64_t dz_plane, int dz_classes) {
    const unsigned quads = (unsigned)dz_classes / 4, blocks = (quads + 255) / 256;
    const int64_t row = blockIdx.x / blocks;
    const unsigned quad = (blockIdx.x - (unsigned)row * blocks) * 256 + threadIdx.x;
    if (quad >= quads) return;
    const int64_t c = (int64_t)quad * 4;
    float d[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < g.classes) {
        const float4 v = thin_logits(g, row, c);
        const LogitGrad grad = logit_grad(g.facts, row, g.classes);
        const float z[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = c + e < g.classes ? grad.of(z[e], c + e == grad.target) : 0.f;
    }
    store_dz<T>(dz + row * dz_ld + c * (int64_t)sizeof(T), dz_plane, d);
}

// ---- joins --------------------------------------------------------------------------------------------------------------
// The sums of a row's tiles [tile][rows]: 32 rows by 8 groups of tiles to a block.
__global__ __launch_bounds__(256) void classifier_join_kernel(const float4* __restrict__ sums, int64_t tiles, int64_t rows, const int32_t* targets,
                                                              int64_t classes, const float* target_z, RowResults out) {
    __shared__ float4 part[8][32];
    const int r = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * 32 + r;
    SoftmaxSums s;
    if (row < rows)
        for (int64_t t = group; t < tiles; t += 8) {
            const float4 p = sums[t * rows + row];
            SoftmaxSums o;
            o.m = p.x; o.s = p.y; o.t = p.z;
            softmax_join(s, o);
        }
    part[group][r] = make_float4(s.m, s.s, s.t, 0.f);
    __syncthreads();
    if (group != 0 || row >= rows) return;
    for (int q = 1; q < 8; ++q) {
        const float4 p = part[q][r];
        SoftmaxSums o;
        o.m = p.x; o.s = p.y; o.t = p.z;
        softmax_join(s, o);
    }
    write_results(out, targets, classes, row, s, target_z[row]);      // (without a target: not looked at)
}

// out[r][c] = sum over the slots of part[slot][r][c], in slot order
template <typename OUT>
__global__ __launch_bounds__(256) void sum_slots_kernel(const float* __restrict__ part, int slots, int64_t slot, int64_t cols, int64_t n, OUT* out, int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = part[i];
    for (int q = 1; q < slots; ++q) s += part[q * slot + i];
    const int64_t r = i / cols;
    out[r * ld + (i - r * cols)] = Elem<OUT>::from_f32(s);
}

// rows of `cols` elements, copied to rows of `wide` (whole 16 bytes), zeros past them; a lane has 16 bytes
template <typename T>
__global__ __launch_bounds__(256) void pad_rows_kernel(const T* __restrict__ src, int64_t ld, int64_t cols, T* __restrict__ dst, int64_t wide, int64_t n) {
    constexpr int VEC = Elem<T>::VEC;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t vecs = wide / VEC, row = i / vecs, c = (i - row * vecs) * VEC;
    Vec16<T> v;
    if (c + VEC <= cols) {
        v = load_loose(src + row * ld + c);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v.e[e] = c + e < cols ? src[row * ld + c + e] : (T)0;
    }
    store_vec(dst + row * wide + c, v);
}

// No rows: the gradients of weights and bias are sums of nothing.
__global__ __launch_bounds__(256) void zero_rows_kernel(float* p, int64_t ld, int64_t cols, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i / cols * ld + i % cols] = 0.f;
}

constexpr int64_t kMiB = 1 << 20;
constexpr int64_t kSmallTiles = 192;           // z of fewer tiles is formed in parts (thin_logits_kernel)
constexpr int64_t kDzBytes = 1024 * kMiB;      // of dz at a time
constexpr int64_t kZeroAtOnce = 1ll << 30;     // elements of dw that one launch clears where there are no rows
constexpr int64_t kMostAtOnce = 1 << 20;       // classes of it: 64 rows of dz are counted in 32 bits
constexpr int64_t kWantBlocks = 512;           // two blocks of 128x128 per CU
constexpr int64_t kChip = 256;                 // CUs: one block of 256x256 each
constexpr int64_t kWantWaves = 2048;
constexpr int64_t kThinPart = 4096;            // classes of a part of a row, at least, where rows are few

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// How a product of M x N outputs over `steps` steps is laid out: tiles of 256x256 where they fill most of the chip, the
// reduction cut if need be, and little of them hangs over the edges; else of 128x128, the reduction cut towards two blocks
// per CU, four steps to a cut at least.
struct Layout { bool big; int cuts, per_cut; };
Layout lay_out(int64_t M, int64_t N, int64_t steps, int esz, bool may_cut) {
    Layout l = {};
    const int64_t big = ceil_div(M, kBigTile) * ceil_div(N, kBigTile), tiles = ceil_div(M, kTile) * ceil_div(N, kTile);
    const int64_t big_cuts = may_cut && big < kChip ? std::max<int64_t>(1, std::min<int64_t>(kChip / big, steps / 16)) : 1;
    l.big = esz == 2 && big * big_cuts * 4 >= kChip * 3 && M * N * 4 >= big * kBigTile * kBigTile * 3;
    int64_t want = 1;
    if (l.big) want = big_cuts;
    else if (may_cut && tiles < kWantBlocks / 2) want = std::min<int64_t>(std::max<int64_t>(1, steps / 4), kWantBlocks / tiles);
    l.per_cut = (int)ceil_div(steps, want);
    l.cuts = (int)ceil_div(steps, l.per_cut);
    return l;
}

// everything a call does, from its sizes and alignments alone
struct Plan {
    int esz;
    int64_t wide;              // features up to whole 16 bytes
    bool pad_x, pad_w;
    bool thin;
    int thin_cuts, thin_steps;         // of the reduction: cuts over blocks, steps of a wave
    int64_t z_ld;
    int thin_parts;
    int64_t thin_part;
    int planes, dx_planes;
    int64_t chunk, chunks;     // of classes, in the backward pass
    Layout z, dx, dw;
    int64_t z_tiles;           // of classes
    // workspace
    int64_t x_at, w_at, z_at, sums_at, target_at, dz_at, dz_ld, dz_plane, dx_at, dw_at, db_at, bytes;
};

Plan plan_of(int dtype, int64_t rows, int64_t dim, int64_t classes, bool aligned_x, bool aligned_w, bool backward) {
    Plan p = {};
    p.esz = dtype == 1 ? 2 : 4;
    const int64_t vec = 16 / p.esz, step = kStepBytes / p.esz;
    p.wide = round_up(dim, vec);
    p.pad_x = !aligned_x;
    p.pad_w = !aligned_w;
    const int64_t tiles_r = ceil_div(rows, kTile), tiles_c = ceil_div(classes, kTile);
    int64_t o = 0;
    auto take = [&](int64_t bytes) { const int64_t at = o; o += round_up(bytes, 256); return at; };
    p.x_at = take(p.pad_x ? rows * p.wide * p.esz : 0);
    p.w_at = take(p.pad_w ? classes * p.wide * p.esz : 0);
    p.thin = tiles_r * tiles_c < kSmallTiles;
    if (p.thin) {
        const int64_t steps = ceil_div(p.wide, step), small = ceil_div(rows, 32) * ceil_div(classes, 32);
        const int64_t waves = std::max<int64_t>(4, std::min<int64_t>(kWantWaves / small, steps));
        p.thin_cuts = (int)std::max<int64_t>(1, waves / 4);
        p.thin_steps = (int)ceil_div(steps, p.thin_cuts * 4);
        p.thin_cuts = (int)ceil_div(steps, p.thin_steps * 4);
        p.z_ld = round_up(classes, 32);
        const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(classes, kThinPart), kWantBlocks / rows));
        p.thin_part = round_up(ceil_div(classes, parts), 4);
        p.thin_parts = (int)ceil_div(classes, p.thin_part);
        p.z_at = take(p.thin_cuts * rows * p.z_ld * 4);
    }
    if (!backward) {
        p.z = lay_out(classes, rows, 1, p.esz, false);
        p.z_tiles = ceil_div(classes, p.z.big ? kBigTile : kTile);
        p.sums_at = take(p.thin ? (p.thin_parts > 1 ? p.thin_parts * rows * 16 : 0) : p.z_tiles * rows * 16);
        p.target_at = take(rows * 4);
    } else {
        p.planes = dtype == 1 ? 3 : 1;
        p.dx_planes = dtype == 1 ? 2 : 1;
        const int64_t at_once = std::min(kMostAtOnce, std::max<int64_t>(1, kDzBytes / (rows * p.planes * p.esz * kTile)) * kTile);
        p.chunks = p.thin ? 1 : ceil_div(classes, at_once);
        p.chunk = round_up(ceil_div(classes, p.chunks), kTile);
        p.chunks = ceil_div(classes, p.chunk);
        p.dz_ld = round_up(p.chunk * p.esz, 128);
        p.dz_plane = rows * p.dz_ld;
        p.dz_at = take(p.planes * p.dz_plane);
        const int64_t n = std::min(p.chunk, classes);
        p.z = lay_out(n, rows, 1, p.esz, false);
        p.dx = lay_out(rows, dim, ceil_div(n, step), p.esz, true);
        p.dw = lay_out(n, dim, ceil_div(rows, step), p.esz, true);
        p.dx_at = take(p.chunks * p.dx.cuts > 1 ? p.chunks * p.dx.cuts * rows * dim * 4 : 0);
        p.dw_at = take(p.dw.cuts > 1 ? p.dw.cuts * p.chunk * dim * 4 : 0);
        p.db_at = take(p.dw.cuts > 1 ? p.dw.cuts * p.chunk * 4 : 0);
    }
    p.bytes = o;
    return p;
}

bool lies_aligned(const void* p, int64_t ld, int64_t dim, int esz) {
    return (uintptr_t)p % 16 == 0 && ld * esz % 16 == 0 && dim * esz % 16 == 0 && ld * esz <= (1 << 23);
}

template <typename T> Operand padded(const void* src, int64_t ld, int64_t rows, int64_t dim, const Plan& p, bool pad, int64_t at, char* work, hipStream_t st) {
    if (!pad) return Operand{(const char*)src, ld * p.esz, rows};
    const int64_t n = rows * (p.wide * p.esz / 16);
    ProfScope ps("classifier_pad", 0.0, (double)rows * (dim + p.wide) * p.esz, st);
    hipLaunchKernelGGL((pad_rows_kernel<T>), dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, st, (const T*)src, ld, dim, (T*)(work + at), p.wide, n);
    return Operand{work + at, p.wide * p.esz, rows};
}

template <typename T> ThinRows thin_forward(const Operand& x, const Operand& w, const float* bias, const RowFacts& facts, const Plan& p, char* work, hipStream_t st) {
    ThinArgs t = {};
    t.w = w;
    t.x = x;
    t.k = p.wide;
    t.steps = (int)ceil_div(p.wide * p.esz, kStepBytes);
    t.steps_per_wave = p.thin_steps;
    t.tiles_m = (int)ceil_div(w.rows, 32);
    t.tiles_n = (int)ceil_div(x.rows, 32);
    t.z = (float*)(work + p.z_at);
    t.z_ld = p.z_ld;
    ProfScope ps("classifier_thin_logits", 2.0 * x.rows * w.rows * p.wide, (double)(x.rows + w.rows) * p.wide * p.esz, st);
    hipLaunchKernelGGL((thin_logits_kernel<T>), dim3((unsigned)(t.tiles_m * t.tiles_n * p.thin_cuts)), dim3(256), 0, st, t);
    return ThinRows{t.z, p.z_ld, x.rows, w.rows, p.thin_cuts, bias, facts};
}

GemmArgs product_of(const Operand& a, const Operand& b, int64_t a_k, int64_t b_k, int esz, bool big) {
    GemmArgs g = {};
    g.a = a;
    g.b = b;
    g.a_k = a_k;
    g.b_k = b_k;
    g.planes = 1;
    g.steps = g.steps_per_cut = (int)ceil_div(a_k * esz, kStepBytes);
    g.tiles_m = (int)ceil_div(a.rows, big ? kBigTile : kTile);
    g.tiles_n = (int)ceil_div(b.rows, big ? kBigTile : kTile);
    g.group = big ? 4 : 8;
    return g;
}

template <typename T, Want WANT, bool A_ALONG, bool B_ALONG, typename OUT> void launch_gemm(const GemmArgs& g, int cuts, bool big, hipStream_t st) {
    const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * cuts));
    if constexpr (sizeof(T) == 2) {
        if (big) {
            hipLaunchKernelGGL((gemm_kernel<T, WANT, A_ALONG, B_ALONG, OUT, Shape256>), grid, dim3(512), 0, st, g);
            return;
        }
    }
    hipLaunchKernelGGL((gemm_kernel<T, WANT, A_ALONG, B_ALONG, OUT, Shape128>), grid, dim3(256), 0, st, g);
}

template <typename T> void forward(const ClassifierCall& c, const ClassifierOut& out, hipStream_t st) {
    const Plan p = plan_of(c.dtype, c.rows, c.dim, c.classes, lies_aligned(c.x, c.ldx, c.dim, sizeof(T)), lies_aligned(c.w, c.ldw, c.dim, sizeof(T)), false);
    char* const work = (char*)c.work;
    const Operand x = padded<T>(c.x, c.ldx, c.rows, c.dim, p, p.pad_x, p.x_at, work, st);
    const Operand w = padded<T>(c.w, c.ldw, c.classes, c.dim, p, p.pad_w, p.w_at, work, st);
    RowFacts facts = {};
    facts.targets = c.targets;
    const RowResults res = {out.log_prob, out.entropy, out.lse};
    float4* const sums = (float4*)(work + p.sums_at);
    float* const target_z = (float*)(work + p.target_at);
    int64_t tiles;
    if (p.thin) {
        const ThinRows z = thin_forward<T>(x, w, c.bias, facts, p, work, st);
        ProfScope ps("classifier_thin_sums", 0.0, 4.0 * p.thin_cuts * c.rows * c.classes, st);
        hipLaunchKernelGGL(thin_sums_kernel, dim3((unsigned)(c.rows * p.thin_parts)), dim3(256), 0, st, z, p.thin_parts, p.thin_part, sums, target_z, res);
        tiles = p.thin_parts;
        if (tiles == 1) return;
    } else {
        GemmArgs g = product_of(w, x, p.wide, p.wide, p.esz, p.z.big);
        g.bias = c.bias;
        g.classes = c.classes;
        g.facts = facts;
        g.sums = sums;
        g.target_z = target_z;
        tiles = g.tiles_m;
        ProfScope ps("classifier_sums", 2.0 * c.rows * c.classes * c.dim, (double)(c.rows + c.classes) * c.dim * p.esz, st);
        launch_gemm<T, SUMS, true, true, float>(g, 1, p.z.big, st);
    }
    ProfScope ps("classifier_join", 0.0, 16.0 * tiles * c.rows, st);
    hipLaunchKernelGGL(classifier_join_kernel, dim3((unsigned)ceil_div(c.rows, 32)), dim3(256), 0, st, sums, tiles, c.rows, c.targets, c.classes, target_z, res);
}

template <typename OUT> void sum_slots(const float* part, int64_t slots, int64_t rows, int64_t cols, OUT* out, int64_t ld, hipStream_t st) {
    const int64_t n = rows * cols;
    ProfScope ps("classifier_sum", 0.0, 4.0 * slots * n + sizeof(OUT) * (double)n, st);
    hipLaunchKernelGGL((sum_slots_kernel<OUT>), dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, st, part, (int)slots, n, cols, n, out, ld);
}

template <typename T> void backward(const ClassifierCall& c, const ClassifierGrads& d, hipStream_t st) {
    const Plan p = plan_of(c.dtype, c.rows, c.dim, c.classes, lies_aligned(c.x, c.ldx, c.dim, sizeof(T)), lies_aligned(c.w, c.ldw, c.dim, sizeof(T)), true);
    char* const work = (char*)c.work;
    const Operand x = padded<T>(c.x, c.ldx, c.rows, c.dim, p, p.pad_x, p.x_at, work, st);
    const Operand w = padded<T>(c.w, c.ldw, c.classes, c.dim, p, p.pad_w, p.w_at, work, st);
    const RowFacts facts = {c.targets, d.lse, d.entropy, d.dlog_prob, d.dentropy};
    char* const dz = work + p.dz_at;
    const int64_t slots = p.chunks * p.dx.cuts;
    const int row_bytes = (int)(p.wide * p.esz);
    for (int64_t q = 0; q < p.chunks; ++q) {
        const int64_t from = q * p.chunk, n = std::min(p.chunk, c.classes - from), cols = round_up(n, 16 / p.esz);
        const Operand wq = {w.p + from * w.ld, w.ld, n};
        if (p.thin) {
            const ThinRows z = thin_forward<T>(x, w, c.bias, facts, p, work, st);
            ProfScope ps("classifier_thin_grads", 0.0, (4.0 * p.thin_cuts + p.planes * p.esz) * c.rows * c.classes, st);
            hipLaunchKernelGGL((thin_grads_kernel<T>), dim3((unsigned)(c.rows * ceil_div(cols / 4, 256))), dim3(256), 0, st, z, dz, p.dz_ld, p.dz_plane, (int)cols);
        } else {
            GemmArgs g = product_of(wq, x, p.wide, p.wide, p.esz, p.z.big);
            g.bias = c.bias;
            g.first_class = from;
            g.classes = from + n;
            g.all_classes = c.classes;
            g.facts = facts;
            g.dz = dz;
            g.dz_ld = p.dz_ld;
            g.dz_plane = p.dz_plane;
            g.dz_classes = (int)cols;
            ProfScope ps("classifier_dz", 2.0 * c.rows * n * c.dim, (double)(c.rows + n) * c.dim * p.esz + (double)p.planes * p.esz * c.rows * n, st);
            launch_gemm<T, GRADS, true, true, float>(g, 1, p.z.big, st);
        }
        {
            GemmArgs g = product_of(Operand{dz, p.dz_ld, c.rows}, Operand{wq.p, wq.ld, c.dim}, cols, n, p.esz, p.dx.big);
            g.a_plane = p.dz_plane;
            g.planes = p.dx_planes;
            g.b_row_bytes = row_bytes;
            g.steps_per_cut = p.dx.per_cut;
            const int cuts = (int)ceil_div(g.steps, g.steps_per_cut);
            ProfScope ps("classifier_dx", 2.0 * c.rows * n * c.dim, (double)p.dx_planes * p.esz * c.rows * n + (double)p.esz * (n + c.rows) * c.dim, st);
            if (slots > 1) {
                // (the last chunk may have fewer cuts: the slots it leaves out are not summed, see below)
                g.out = (float*)(work + p.dx_at) + q * p.dx.cuts * c.rows * c.dim;
                g.out_ld = c.dim;
                g.out_cut = c.rows * c.dim;
                launch_gemm<T, PRODUCT, true, false, float>(g, cuts, p.dx.big, st);
            } else {
                g.out = d.dx;
                g.out_ld = d.lddx;
                launch_gemm<T, PRODUCT, true, false, T>(g, cuts, p.dx.big, st);
            }
            if (q + 1 == p.chunks && slots > 1) {
                const int64_t used = (p.chunks - 1) * p.dx.cuts + cuts;
                sum_slots<T>((const float*)(work + p.dx_at), used, c.rows, c.dim, (T*)d.dx, d.lddx, st);
            }
        }
        {
            GemmArgs g = product_of(Operand{dz, p.dz_ld, n}, Operand{x.p, x.ld, c.dim}, c.rows, c.rows, p.esz, p.dw.big);
            g.a_plane = p.dz_plane;
            g.planes = p.planes;
            g.a_row_bytes = (int)(cols * p.esz);
            g.b_row_bytes = row_bytes;
            g.steps_per_cut = p.dw.per_cut;
            const bool cut = p.dw.cuts > 1;
            g.out = cut ? (float*)(work + p.dw_at) : d.dw + from * d.lddw;
            g.out_ld = cut ? c.dim : d.lddw;
            g.out_cut = n * c.dim;
            if (d.dbias != nullptr) {
                g.dbias = cut ? (float*)(work + p.db_at) : d.dbias + from;
                g.dbias_cut = n;
            }
            {
                ProfScope ps("classifier_dw", 2.0 * c.rows * n * c.dim, (double)p.planes * p.esz * c.rows * n + (double)p.esz * c.rows * c.dim + 4.0 * n * c.dim, st);
                launch_gemm<T, PRODUCT, false, false, float>(g, p.dw.cuts, p.dw.big, st);
            }
            if (cut) {
                sum_slots<float>((const float*)(work + p.dw_at), p.dw.cuts, n, c.dim, d.dw + from * d.lddw, d.lddw, st);
                if (d.dbias != nullptr) sum_slots<float>((const float*)(work + p.db_at), p.dw.cuts, 1, n, d.dbias + from, n, st);
            }
        }
    }
}

}  // namespace

size_t classifier_work_bytes(const ClassifierCall& c, bool backward) {
    const int esz = c.dtype == 1 ? 2 : 4;
    const bool ax = c.x == nullptr ? false : lies_aligned(c.x, c.ldx, c.dim, esz), aw = c.w == nullptr ? false : lies_aligned(c.w, c.ldw, c.dim, esz);
    return (size_t)plan_of(c.dtype, c.rows, c.dim, c.classes, ax, aw, backward).bytes;
}

void launch_classifier(const ClassifierCall& c, const ClassifierOut& out, hipStream_t st) {
    if (c.rows <= 0) return;
    if (c.dtype == 1) forward<bf16_t>(c, out, st);
    else forward<float>(c, out, st);
}

void launch_classifier_grads(const ClassifierCall& c, const ClassifierGrads& d, hipStream_t st) {
    if (c.rows <= 0) {
        for (int64_t from = 0; from < c.classes; from += kZeroAtOnce / c.dim) {      // (a launch's work items fit 32 bits)
            const int64_t n = std::min(kZeroAtOnce / c.dim, c.classes - from) * c.dim;
            hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, st, d.dw + from * d.lddw, d.lddw, c.dim, n);
        }
        if (d.dbias != nullptr) hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)ceil_div(c.classes, 256)), dim3(256), 0, st, d.dbias, c.classes, c.classes, c.classes);
        return;
    }
    if (c.dtype == 1) backward<bf16_t>(c, d, st);
    else backward<float>(c, d, st);
}

}  // namespace edl
