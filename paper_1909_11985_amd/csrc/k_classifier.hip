// Log probabilities of given classes straight from features and classifier weights, and the gradients of both, without
// the logits in memory.
//
//   z = x w^T + b                       [rows][classes], formed tile by tile
//   lse, entropy, log_prob              from each tile's sums (softmax_sums.h), joined over the tiles of a row
//   dz = g (1[c = t] - p) - h p (log p + H),  dx = dz w,  dw = dz^T x,  db = sum of dz over the rows
//
// Four products, one kernel (gemm_kernel) on 32x32 bf16 matrix instructions.  An operand lies with the reduction along its
// rows (x and w in z, dz in dx) or across them (dz and x in dw, w in dx); either is brought to LDS as it lies, and a fragment
// of the second kind is read transposed, so nothing is transposed in memory.  z is formed as w x^T: a lane then has one
// row's classes, 16 to a 32x32 tile, and the sums over classes stay inside it.
//
// Float32 operands are sums of three bf16 numbers ("planes", 24 bits together), and a product of two such sums is the six
// products of planes that are not below float32's last place.  The matrix cores do 16 bf16 multiplications in the time of one float32 one,
// so six of them still take less than half of its time.
//
// The gradient forms z again rather than keep it, a piece of the classes at a time.  Rows whose lse is far (softmax_sums.h) need
// their largest logit and sum first: of z in float32 parts, the block that forms their dz sums them up, or of many classes the loss's sums
// and join run once more; on tiles its product and join do, for the tiles that have such a row alone (5 + 2 us of launches that do nothing where there is none).  dz is stored for the two products that
// read it, in both types as three planes: dw is float32, and a single rounding of dz to bf16 would be its largest error by
// four orders of magnitude.  dx of bf16, which is rounded to bf16 itself, takes the first two.
//
// Measured, 4,096 rows of 1,024 bf16 features, 32,768 classes (a large library product reaches 1,386 TFLOP/s on this card): loss 310 us
// (890 TFLOP/s; a third of it is the sums behind the product), dz 440 (of which 130 are its 805 MB), dx 470 (1,170, of two
// planes), dw 600 (1,375, of three).  By the counters the matrix cores are busy for 59 % of dx and 69 % of
// dw; over zeros, for which the chip needs less power, loss and gradient take 18 % less (1,557 -> 1,275 us): part of what bounds them is power.
#include <algorithm>

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

// ---- operands ---------------------------------------------------------------------------------------------------------
// 16 bytes per lane from memory to LDS: lane l's go to lds_wave_base + 16 l; lanes whose offset lies past the descriptor's
// extent get zeros.  Issued from assembly, so that the compiler does not wait for it at every LDS access: wait_loads and a
// barrier order it.
constexpr unsigned kNowhere = 0x80000000u;       // past any extent (they are clamped below it)
__device__ __forceinline__ i32x4 extent_of(const char* p, int64_t bytes) {
    const uint64_t a = (uint64_t)p;
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };       // (they are: the compiler has lost track)
    const i32x4 r = {same((int)(uint32_t)a), same((int)(uint32_t)(a >> 32)), same((int)max((int64_t)0, min(bytes, (int64_t)0x7ffffff0))), 0x00020000};
    return r;
}
__device__ __forceinline__ void load16_to_lds(i32x4 extent, unsigned lds_wave_base, unsigned offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_wave_base), "v"(offset), "s"(extent) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// One operand of a product: element (r, k) of `rows` by `k` of the reduction, bf16.  along: row r's reduction lies at
// p + r * ld; across: k's rows lie at p + k * ld.  A line's elements follow each other, or, of an operand of three planes, in
// groups of 64: the group's first plane, second, third (a line of the caches each).  p and ld are multiples of 16 bytes, a line's
// elements whole pieces of 8 with zeros past the operand's.
constexpr int kGroup = 64;
constexpr int64_t kGroupBytes = 3 * 2 * kGroup;
__host__ __device__ inline int64_t planes_bytes(int64_t n) { return (n + kGroup - 1) / kGroup * kGroupBytes; }
// where element c of such a line has its first plane; the others follow 2 kGroup bytes apart
__host__ __device__ inline int64_t plane_at(int64_t c) { return c / kGroup * kGroupBytes + c % kGroup * 2; }
struct Operand {
    const char* p;
    int64_t ld;                // bytes
    int64_t rows, k;
    int stored;                // planes in memory: 1 or 3
    __host__ __device__ int64_t line_bytes(int64_t n) const { return stored == 1 ? (n + 7) / 8 * 16 : planes_bytes(n); }
    __host__ __device__ int64_t at(int64_t c) const { return stored == 1 ? 2 * c : plane_at(c); }       // of a line's element
};

// Tiles of W rows and one reduction step of KS elements in LDS, one for each of the first P planes.
//   along: [W][KS], the 16-byte pieces of a row permuted by bits of the row's number, such that the 16 rows whose same piece the
//     lanes of a read ask for together lie in banks of their own
//   across: [KS][W], the 32-byte pairs of pieces of a k permuted by its low bits: a transposing read takes two neighbouring
//     pairs of four consecutive k, which then fall into different banks
template <bool ALONG, int W, int P, int KS, int THREADS> struct Tile {
    static constexpr int PLANE = W * KS * 2, BYTES = P * PLANE;
    static constexpr int PIECES = ALONG ? KS / 8 : W / 8;              // 16-byte pieces of a line
    static constexpr int LOADS = BYTES / 16 / THREADS;                 // per lane
    static_assert(BYTES % (16 * THREADS) == 0, "whole loads");
    static_assert(!ALONG || THREADS % (16 * PIECES) == 0, "a lane's loads are of the same piece of their rows");

    unsigned offset[LOADS];      // this lane's, from the step's start
    int piece_k;                 // along: which of the step's elements this lane's pieces hold first
    // of the step that is loaded next: elements of the reduction before it, and with the operand's tile and its bytes where it starts
    int64_t k_at;
    const char* tile;
    int64_t bytes;
    // of the step that is being loaded
    i32x4 extent;
    int k_here;

    __device__ __forceinline__ static int pair_of(int pair, int k) { return pair ^ ((k & 3) << 1); }
    __device__ __forceinline__ static int piece_of(int piece, int row) { return piece ^ ((row * PIECES / 16) & (PIECES - 1)); }

    __device__ __forceinline__ void init(const Operand& o, int64_t first_row) {
        tile = o.p + (ALONG ? first_row * o.ld : o.at(first_row));
        bytes = ALONG ? (o.rows - first_row - 1) * o.ld + o.line_bytes(o.k) : (o.k - 1) * o.ld + o.line_bytes(o.rows) - o.at(first_row);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int slot = i * THREADS + (int)threadIdx.x, plane = slot / (PLANE / 16), line = slot % (PLANE / 16) / PIECES, s = slot % PIECES;
            const int piece = ALONG ? piece_of(s, line) : pair_of(s >> 1, line) << 1 | (s & 1);
            // (a step along does not cross a group: KS divides it)
            const unsigned at = (unsigned)(line * o.ld) + plane * 2 * kGroup + (unsigned)(ALONG ? piece * 16 : o.at(piece * 8));
            offset[i] = ALONG || first_row + piece * 8 < o.rows ? at : kNowhere;
            if (ALONG && i == 0) piece_k = piece * 8;
        }
    }
    // Turns to the next step; there: false past the last one (its loads bring zeros into a stage that nobody reads, so that
    // loads can be counted).
    __device__ __forceinline__ void turn(const Operand& o, bool there) {
        const int64_t at = ALONG ? o.at(k_at) : k_at * o.ld;
        extent = extent_of(tile + at, there ? bytes - at : 0);
        k_here = (int)min(o.k - k_at, (int64_t)KS);
        k_at += KS;
    }
    // the i-th of this step's loads
    __device__ __forceinline__ void load(int i, unsigned lds) const {
        const unsigned wave = (unsigned)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024;
        load16_to_lds(extent, lds + wave + i * THREADS * 16, !ALONG || piece_k < k_here ? offset[i] : kNowhere);
    }
    // Fragment of rows [r32, r32 + 32) and reduction elements [16 q, 16 q + 16) of the step: a lane has row r32 + lane % 32 and
    // the eight elements of half lane / 32
    __device__ __forceinline__ static uint4 fragment(const char* tile, int plane, int r32, int q, int lane) {
        tile += plane * PLANE;
        if constexpr (ALONG) {
            const int r = r32 + (lane & 31);
            return *reinterpret_cast<const uint4*>(tile + r * KS * 2 + piece_of(2 * q + (lane >> 5), r) * 16);
        } else {
            // the transposing read hands lane l of 16 lanes element l of the 16 rows of a pair, for four consecutive k whose
            // lines lanes 4i .. 4i + 3 address, eight bytes each
            typedef shortx4 __attribute__((address_space(3))) * lds_ptr;
            const int row = r32 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3), k = q * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
            auto at = [&](int kk) { return (lds_ptr)(tile + kk * W * 2 + pair_of(row >> 4, kk) * 32 + (row & 15) * 2); };
            const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k)));
            const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(k + 4)));
            return make_uint4(a.x, a.y, b.x, b.y);
        }
    }
};

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
// four neighbouring elements, the first of them number c (a multiple of 4), of a line of three planes
__device__ __forceinline__ void store_planes(char* line, int64_t c, float (&v)[4]) {
    char* const p = line + plane_at(c);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(p + q * 2 * kGroup) = next_bf16(v);
}

enum Want { SUMS, GRADS, PRODUCT, ADDED };     // of z: sums over classes, dz; of the others: the product itself, or added to what is there

struct GemmArgs {
    Operand a, b;
    int steps, steps_per_cut;  // of the reduction; a cut of it is a block's
    int tiles_m, tiles_n, group;
    // z: a = w from class `first_class` on, b = x
    const float* bias;
    int64_t first_class, classes, all_classes;     // classes: the end of this launch's
    RowFacts facts;
    const float2* far;         // dz: of rows whose lse is far, LogitGrad's base and low
    float4* sums;              // [tile of classes][rows]: m, s, t
    float* target_z;           // null: not wanted
    char* dz;                  // [rows][dz_ld bytes] of the classes from first_class on, three planes
    int64_t dz_ld;
    int dz_classes;            // up to whole pairs of pieces (zeros past the last class)
    float* db;                 // [tile of rows][db_ld] sums of dz; null: not wanted
    int64_t db_ld;
    // products
    void* out;                 // [cut][a.rows][out_ld]
    int64_t out_ld, out_cut;   // elements
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

// A block's eight waves, WM x WN, and a wave's 32x32 tiles, TM x TN.  64x32 to a wave read 3 KB of LDS for every 2 matrix
// instructions, 128x64 read 6 KB for 8; what the larger tile needs is enough of them for the chip.  (Four waves of 64x64 read 4 KB
// for 4, but where a CU has one block its matrix cores wait with their only wave: gradients of 333 x 515 x 10,007 float32 115 us, with
// eight 112; 100 x 4,096 x 1,000 bf16 44 and 42; 1,000 x 512 x 6,000 float32 155 and 147; with several blocks to a CU within 2 % either way.)
struct Shape128 { static constexpr int WM = 2, WN = 4, TM = 2, TN = 1, SIDE = 128; };
struct Shape256 { static constexpr int WM = 2, WN = 4, TM = 4, TN = 2, SIDE = 256; };
// Elements of a reduction step and steps in LDS at a time, for PA and PB planes: long steps, because a step's part of a line
// is asked for at once and parts of 32 bytes take the caches twice as long as parts of 64 (dw of 4,096 x 1,024 x 32,768 bf16:
// 880 us with planes in groups of 16 elements, 594 with whole lines), and as many as fit, so that loads of the steps
// to come are always in flight.
template <int PA, int PB, int SIDE> struct Steps {
    static constexpr int KS = (PA + PB == 4 || PA + PB == 6) && SIDE == 256 ? 16 : 32;
    static constexpr int STAGES = PA + PB == 2 || PA + PB == 4 ? 4 : 3;
};

template <int PA, int PB, int SIDE> constexpr int lds_bytes() { return Steps<PA, PB, SIDE>::STAGES * (PA + PB) * SIDE * Steps<PA, PB, SIDE>::KS * 2; }
// One tile, by a block; smem: lds_bytes of LDS.
template <Want WANT, int PA, int PB, bool A_ALONG, bool B_ALONG, typename OUT, typename SHAPE>
__device__ __forceinline__ void gemm_tile(const GemmArgs& g, int tm, int tn, int cut, char* smem) {
    constexpr int WM = SHAPE::WM, WN = SHAPE::WN, TM = SHAPE::TM, TN = SHAPE::TN, THREADS = WM * WN * 64, SIDE = SHAPE::SIDE;
    constexpr int KS = Steps<PA, PB, SIDE>::KS, STAGES = Steps<PA, PB, SIDE>::STAGES;
    typedef Tile<A_ALONG, SIDE, PA, KS, THREADS> TA;
    typedef Tile<B_ALONG, SIDE, PB, KS, THREADS> TB;
    constexpr int STAGE = TA::BYTES + TB::BYTES;
    static_assert(STAGES * STAGE == lds_bytes<PA, PB, SIDE>(), "what the kernel holds");
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const int64_t m0 = (int64_t)tm * SIDE, n0 = (int64_t)tn * SIDE;
    const int first = cut * g.steps_per_cut, all = min(g.steps_per_cut, g.steps - first);
    TA ta;
    TB tb;
    ta.init(g.a, m0);
    tb.init(g.b, n0);
    ta.k_at = tb.k_at = (int64_t)first * KS;
    int asked = 0, to = 0;                                  // steps asked for, and the stage of the one being loaded
    auto turn = [&]() {
        const bool there = asked < all;
        ta.turn(g.a, there);
        tb.turn(g.b, there);
        if (asked > 0) to = to + 1 == STAGES ? 0 : to + 1;
        ++asked;
    };
    constexpr int LOADS = TA::LOADS + TB::LOADS, GROUPS = KS / 16 * PA;
    auto load = [&](int i) {
        if (i < TA::LOADS) ta.load(i, lds + to * STAGE);
        else tb.load(i - TA::LOADS, lds + to * STAGE + TA::BYTES);
    };
    floatx16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
#pragma unroll
    for (int u = 0; u < STAGES - 1; ++u) {
        turn();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(i);
    }
    for (int t = 0, from = 0; t < all; ++t, from = from + 1 == STAGES ? 0 : from + 1) {
        // This step is there for all waves, and all are done with the one before, whose stage is filled now.  (Loads come in
        // order: all but those of the STAGES - 2 younger steps have.)  A wave asks for its part of a step between its groups of
        // matrix instructions: the path to memory takes a load every 16 cycles, and if all waves ask at once the matrix cores
        // wait for that.
        wait_loads<(STAGES - 2) * LOADS>();
        __syncthreads();
        turn();
        const char* const A = smem + from * STAGE;
        const char* const B = A + TA::BYTES;
#pragma unroll
        for (int q = 0; q < KS / 16; ++q) {
            uint4 fb[PB][TN];
#pragma unroll
            for (int b = 0; b < PB; ++b)
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[b][j] = TB::fragment(B, b, (wn * TN + j) * 32, q, lane);
#pragma unroll
            for (int a = 0; a < PA; ++a) {
                uint4 fa[TM];
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[i] = TA::fragment(A, a, (wm * TM + i) * 32, q, lane);
#pragma unroll
                for (int b = 0; b < PB && a + b < (PA > PB ? PA : PB); ++b)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) 
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[i]), __builtin_bit_cast(bf16x8, fb[b][j]), acc[i][j], 0, 0, 0);
                const int group = q * PA + a;
#pragma unroll
                for (int i = group * LOADS / GROUPS; i < (group + 1) * LOADS / GROUPS; ++i) load(i);
            }
        }
    }
    wait_loads<0>();
    __syncthreads();           // LDS is free
    if constexpr (WANT == PRODUCT || WANT == ADDED) {
        OUT* const out = (OUT*)g.out + cut * g.out_cut;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + (wn * TN + j) * 32 + (lane & 31);
            if (n >= g.b.rows) continue;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int64_t top = m0 + (wm * TM + i) * 32;
                if constexpr (WANT == ADDED) {         // (rows past the last: the last one's, so that the loads do not wait for each other)
                    static_assert(sizeof(OUT) == 4, "sums are float32");
                    float was[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) was[e] = out[min(top + tile_row(e, lane), g.a.rows - 1) * g.out_ld + n];
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] += was[e];
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int64_t m = top + tile_row(e, lane);
                    if (m < g.a.rows) out[m * g.out_ld + n] = Elem<OUT>::from_f32(acc[i][j][e]);
                }
            }
        }
    } else {
        // z: rows of the tile are classes, columns rows of x.  Class of element e of tile i: c0 + place(i, e).  Past the last class
        // the bias is -inf, which masks it like any other.
        const int64_t c0 = g.first_class + m0 + wm * TM * 32 + 4 * (lane >> 5);
        auto place = [](int i, int e) { return 32 * i + 8 * (e >> 2) + (e & 3); };
        float* const bias = reinterpret_cast<float*>(smem);
        if (threadIdx.x < SIDE) {
            const int64_t c = g.first_class + m0 + threadIdx.x;
            bias[threadIdx.x] = c >= g.classes ? -INFINITY : g.bias != nullptr ? g.bias[c] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 b = *reinterpret_cast<const float4*>(bias + (wm * TM + i) * 32 + 8 * q + 4 * (lane >> 5));
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    acc[i][j][4 * q] += b.x;
                    acc[i][j][4 * q + 1] += b.y;
                    acc[i][j][4 * q + 2] += b.z;
                    acc[i][j][4 * q + 3] += b.w;
                }
            }
        // where a row's target is among this lane's classes, or -1
        auto place_of = [&](int64_t target) { return target >= c0 && target < min(c0 + TM * 32, g.classes) ? (int)(target - c0) : -1; };
        if constexpr (WANT == SUMS) {
            float4* const part = reinterpret_cast<float4*>(smem + SIDE * 4);      // [wm][SIDE]
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int col = (wn * TN + j) * 32 + (lane & 31);
                const int64_t n = n0 + col;
                const int64_t t = n < g.b.rows && g.facts.targets != nullptr && g.target_z != nullptr ? g.facts.targets[n] : -1;
                const int hot = place_of(t);
                SoftmaxSums s;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s.m = fmaxf(s.m, acc[i][j][e]);
                if (__ballot(hot >= 0) != 0) {     // (few tiles hold a row's target)
                    float zt = 0.f;
                    bool here = false;
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (place(i, e) == hot) { zt = acc[i][j][e]; here = true; }
                    if (here) g.target_z[n] = zt;
                }
                const float base = softmax_base(s);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) softmax_add(s, acc[i][j][e], base);
                softmax_join(s, softmax_shuffle(s, 32));
                if (lane < 32) part[wm * SIDE + col] = make_float4(s.m, s.s, s.t, 0.f);
            }
            __syncthreads();
            if (threadIdx.x < SIDE && n0 + threadIdx.x < g.b.rows) {
                SoftmaxSums s;
#pragma unroll
                for (int w = 0; w < WM; ++w) {
                    const float4 p = part[w * SIDE + threadIdx.x];
                    SoftmaxSums o;
                    o.m = p.x; o.s = p.y; o.t = p.z;
                    softmax_join(s, o);
                }
                g.sums[tm * g.b.rows + n0 + threadIdx.x] = make_float4(s.m, s.s, s.t, 0.f);
            }
        } else {
            // dz goes out through LDS, a plane at a time, so that rows are written in whole pieces: [SIDE rows][SIDE classes] with
            // the 16-byte pieces of a row permuted by its low bits (32 lanes write one piece of 32 rows).  A thread moves the same
            // classes of every (THREADS / PIECES)-th row, whose sum is its part of the bias's gradient.
            constexpr int PIECES = SIDE / 8, ROWS = THREADS / PIECES;
            static_assert(SIDE * SIDE * 2 <= STAGES * STAGE && ROWS * SIDE * 4 <= STAGES * STAGE, "fits");
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t n = n0 + (wn * TN + j) * 32 + (lane & 31);
                LogitGrad row = logit_grad(g.facts, min(n, g.b.rows - 1), g.all_classes);
                const int hot = place_of(row.target);
                if (__ballot(row.far) == 0) {
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[i][j][e] = row.of<false>(acc[i][j][e], place(i, e) == hot);
                    continue;
                }
                if (row.far) {
                    const float2 far = g.far[min(n, g.b.rows - 1)];
                    row.base = far.x;
                    row.low = far.y;
                }
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = row.of<true>(acc[i][j][e], place(i, e) == hot);
            }
            const int c = threadIdx.x % PIECES, rows = (int)min((int64_t)SIDE, g.b.rows - n0);
            const bool wanted = m0 + c * 8 < g.dz_classes;
            float total[8] = {};
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                __syncthreads();           // the biases are read, or the plane before is out
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int r = (wn * TN + j) * 32 + (lane & 31);
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int piece = (wm * TM + i) * 4 + q;
                            float d[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) d[e] = acc[i][j][4 * q + e];
                            *reinterpret_cast<uint2*>(smem + (r * PIECES + (piece ^ (r & (PIECES - 1)))) * 16 + 8 * (lane >> 5)) = next_bf16(d);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = d[e];
                        }
                }
                __syncthreads();
                if (wanted) {
                    char* const out = g.dz + n0 * g.dz_ld + plane_at(m0 + c * 8) + p * 2 * kGroup;
                    for (int r = threadIdx.x / PIECES; r < rows; r += ROWS) {
                        Vec16<bf16_t> v;
                        v.u = *reinterpret_cast<const uint4*>(smem + (r * PIECES + (c ^ (r & (PIECES - 1)))) * 16);
                        *reinterpret_cast<uint4*>(out + r * g.dz_ld) = v.u;
#pragma unroll
                        for (int e = 0; e < 8; ++e) total[e] += bf16_to_f32(v.e[e]);
                    }
                }
            }
            if (g.db != nullptr) {
                __syncthreads();
                float* const part = reinterpret_cast<float*>(smem);        // [ROWS][SIDE]
#pragma unroll
                for (int e = 0; e < 8; ++e) part[threadIdx.x / PIECES * SIDE + c * 8 + e] = total[e];
                __syncthreads();
                if (threadIdx.x < SIDE && g.first_class + m0 + threadIdx.x < g.classes) {
                    float sum = 0.f;
                    for (int r = 0; r < ROWS; ++r) sum += part[r * SIDE + threadIdx.x];
                    g.db[tn * g.db_ld + m0 + threadIdx.x] = sum;
                }
            }
        }
    }
}

template <Want WANT, int PA, int PB, bool A_ALONG, bool B_ALONG, typename OUT, typename SHAPE>
__global__ __launch_bounds__(SHAPE::WM * SHAPE::WN * 64) void gemm_kernel(GemmArgs g) {
    __shared__ __attribute__((aligned(16))) char smem[lds_bytes<PA, PB, SHAPE::SIDE>()];
    int tm, tn, cut;
    tile_of(g, tm, tn, cut);
    gemm_tile<WANT, PA, PB, A_ALONG, B_ALONG, OUT, SHAPE>(g, tm, tn, cut, smem);
}

// z's sums, of tiles with a row whose lse is far.  Mostly there is none: a block looks at the rows of its tiles once, and has all
// tiles of those rows, or every gridDim / tiles_n-th of them.  (With a block to each tile 2,048 of them take 25 us where none
// is wanted, so 5.)
template <int P, typename SHAPE> __global__ __launch_bounds__(SHAPE::WM * SHAPE::WN * 64) void far_sums_kernel(GemmArgs g) {
    __shared__ __attribute__((aligned(16))) char smem[lds_bytes<P, P, SHAPE::SIDE>()];
    const int wide = min(g.tiles_n, (int)gridDim.x), deep = (int)gridDim.x / wide;
    if ((int)blockIdx.x >= wide * deep) return;
    for (int tn = (int)blockIdx.x % wide; tn < g.tiles_n; tn += wide) {
        bool any = false;
        for (int64_t n = (int64_t)tn * SHAPE::SIDE + (threadIdx.x & 63); n < min((int64_t)(tn + 1) * SHAPE::SIDE, g.b.rows); n += 64)
            any = any || row_is_far(g.facts, n, g.all_classes);
        if (__ballot(any) == 0) continue;          // (every wave looks at all of them)
        for (int tm = (int)blockIdx.x / wide; tm < g.tiles_m; tm += deep) {
            gemm_tile<SUMS, P, P, true, true, float, SHAPE>(g, tm, tn, 0, smem);
            __syncthreads();           // the next tile's loads take the place of this one's sums
        }
    }
}

// ---- few tiles ----------------------------------------------------------------------------------------------------------
// Where z has too few tiles to fill the chip its reduction is cut as well and its float32 parts are stored: [cut][rows][z_ld].
// They come from gemm_kernel, or, of up to 32 rows (which would waste most of a tile, and not repay the copies that float32 or
// odd rows need there), from this one: a wave has 32 rows of w and its part of the reduction, as they lie in memory.  What bounds
// it is reading w once: eight lanes take 128 bytes of a row, and fragments are formed through LDS of the wave's own.
constexpr int kStepBytes = 128;        // of a reduction step
struct Matrix { const char* p; int64_t ld, rows; };        // ld in bytes
struct ThinArgs {
    Matrix w, x;
    int64_t row_bytes;
    int steps, steps_per_wave, tiles;
    float* z;
    int64_t z_ld;
};
template <typename T> __device__ __forceinline__ uint4 load_piece_of_row(const char* row, int64_t at, int64_t row_bytes) {
    constexpr int ESZ = (int)sizeof(T);
    if (at + 16 <= row_bytes) return load_loose(reinterpret_cast<const T*>(row + at)).u;
    Vec16<T> v;
#pragma unroll
    for (int e = 0; e < 16 / ESZ; ++e) v.e[e] = at + (e + 1) * ESZ <= row_bytes ? reinterpret_cast<const T*>(row + at)[e] : (T)0;
    return v.u;
}
template <typename T> __global__ __launch_bounds__(256) void thin_logits_kernel(ThinArgs g) {
    __shared__ __attribute__((aligned(16))) char smem[4 * 2 * 32 * kStepBytes];       // a step of w's rows and of x's for each wave
    float (*const part)[16][64] = reinterpret_cast<float (*)[16][64]>(smem);           // ... and then the waves' sums
    static_assert(sizeof(float) * 4 * 16 * 64 <= sizeof(smem), "fits");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tm = (int)(blockIdx.x % (unsigned)g.tiles), cut = (int)(blockIdx.x / (unsigned)g.tiles);
    const int first = (cut * 4 + wave) * g.steps_per_wave, last = min(first + g.steps_per_wave, g.steps), whole = (int)(g.row_bytes / kStepBytes);
    const char *a[4], *b[4];           // rows 8 i + lane / 8
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = g.w.p + min((int64_t)tm * 32 + 8 * i + (lane >> 3), g.w.rows - 1) * g.w.ld;
        b[i] = g.x.p + min((int64_t)8 * i + (lane >> 3), g.x.rows - 1) * g.x.ld;
    }
    char* const mine = smem + wave * (2 * 32 * kStepBytes);
    // 16-byte piece of a row in LDS: the 16 rows whose same piece lanes ask for together lie in banks of their own
    auto slot = [](int row, int piece) { return row * kStepBytes + (piece ^ ((row >> 1) & 7)) * 16; };
    floatx16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    uint4 va[4], vb[4];
    auto load = [&](int s) {
        const int64_t at = (int64_t)s * kStepBytes + 16 * (lane & 7);
        if (s < whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) va[i] = load_loose(reinterpret_cast<const T*>(a[i] + at)).u;
#pragma unroll
            for (int i = 0; i < 4; ++i) vb[i] = load_loose(reinterpret_cast<const T*>(b[i] + at)).u;
        } else {                       // the end of the rows
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                va[i] = load_piece_of_row<T>(a[i], at, g.row_bytes);
                vb[i] = load_piece_of_row<T>(b[i], at, g.row_bytes);
            }
        }
    };
    if (first < last) load(first);
    for (int s = first; s < last; ++s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<uint4*>(mine + slot(8 * i + (lane >> 3), lane & 7)) = va[i];
            *reinterpret_cast<uint4*>(mine + 32 * kStepBytes + slot(8 * i + (lane >> 3), lane & 7)) = vb[i];
        }
        wave_lds_handover();
        if (s + 1 < last) load(s + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 fa = *reinterpret_cast<const uint4*>(mine + slot(lane & 31, 2 * q + (lane >> 5)));
            const uint4 fb = *reinterpret_cast<const uint4*>(mine + 32 * kStepBytes + slot(lane & 31, 2 * q + (lane >> 5)));
            if constexpr (sizeof(T) == 2) {
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa), __builtin_bit_cast(bf16x8, fb), acc, 0, 0, 0);
            } else {
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fa.x), __uint_as_float(fb.x), acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fa.y), __uint_as_float(fb.y), acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fa.z), __uint_as_float(fb.z), acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(fa.w), __uint_as_float(fb.w), acc, 0, 0, 0);
            }
        }
        wave_lds_handover();
    }
    __syncthreads();                   // the steps' memory is the sums' now
#pragma unroll
    for (int e = 0; e < 16; ++e) part[wave][e][lane] = acc[e];
    __syncthreads();
    const int64_t row = lane & 31;
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
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* const z = g.z + row * g.z_ld + c;
    const int64_t cut = g.rows * g.z_ld;
#pragma unroll 8
    for (int q = 0; q < g.cuts; ++q) {         // (unrolled: the loads do not wait for each other)
        const float4 p = *reinterpret_cast<const float4*>(z + q * cut);
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
// Sums of a row's classes [lo, hi), by a block: all of its threads have them.  at(class, logit) is called for each.
template <typename F> __device__ __forceinline__ SoftmaxSums thin_row_sums(const ThinRows& g, int64_t row, int64_t lo, int64_t hi, F at) {
    __shared__ float4 wave_sums[4];
    SoftmaxSums s;
    for (int64_t c = lo + threadIdx.x * 4; c < hi; c += 1024) {
        const float4 v = thin_logits(g, row, c);
        float z[4] = {v.x, v.y, v.z, v.w}, m = s.m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= hi) z[e] = -INFINITY;
            else at(c + e, z[e]);
            m = fmaxf(m, z[e]);
        }
        softmax_rebase(s, m);
        const float base = softmax_base(s);
#pragma unroll
        for (int e = 0; e < 4; ++e) softmax_add(s, z[e], base);
    }
    softmax_join_wave(s);
    if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = make_float4(s.m, s.s, s.t, 0.f);
    __syncthreads();
    SoftmaxSums all;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        SoftmaxSums o;
        o.m = wave_sums[w].x; o.s = wave_sums[w].y; o.t = wave_sums[w].z;
        softmax_join(all, o);
    }
    return all;
}
// Sums of a part of a row's classes; of all of them, the results.  far_only: the sums alone, of rows whose lse is far.
__global__ __launch_bounds__(256) void thin_sums_kernel(ThinRows g, int parts, int64_t part, float4* sums, float* target_z, RowResults out, bool far_only) {
    __shared__ float target;
    const int64_t row = blockIdx.x / (unsigned)parts;
    if (far_only && !row_is_far(g.facts, row, g.classes)) return;
    const int p = (int)(blockIdx.x - (unsigned)row * (unsigned)parts);
    const int64_t lo = p * part, hi = min(lo + part, g.classes);
    const int64_t t = !far_only && g.facts.targets != nullptr ? g.facts.targets[row] : -1;
    const SoftmaxSums s = thin_row_sums(g, row, lo, hi, [&](int64_t c, float z) {
        if (c != t) return;
        if (parts == 1) target = z;
        else target_z[row] = z;
    });
    if (threadIdx.x != 0) return;
    if (parts == 1 && !far_only) write_results(out, g.facts.targets, g.classes, row, s, target);
    else sums[p * g.rows + row] = make_float4(s.m, s.s, s.t, 0.f);
}
// dz of such logits: a lane has four neighbouring classes.  Of a row whose lse is far, every block sums up all of its classes
// (launches less for all calls), unless there are more than kFarHere blocks to a row: their sums are then there, joined, in `far`.  (All
// rows far, 100 x 64 x 24,000 float32: 123 us, 58 where none is; 32 x 64 x 1,000,000: 30 ms by every block, 0.9 from `far`, 0.6.)
constexpr unsigned kFarHere = 32;
__host__ __device__ inline unsigned thin_blocks(int64_t quads) { return (unsigned)((quads + 255) / 256); }
__global__ __launch_bounds__(256) void thin_grads_kernel(ThinRows g, char* dz, int64_t dz_ld, int dz_classes, const float2* far) {
    const unsigned quads = (unsigned)dz_classes / 4, blocks = thin_blocks(quads);
    const int64_t row = blockIdx.x / blocks;
    const unsigned quad = (blockIdx.x - (unsigned)row * blocks) * 256 + threadIdx.x;
    LogitGrad grad = logit_grad(g.facts, row, g.classes);
    if (grad.far) {                    // (the same for the whole block)
        const float2 f = far != nullptr ? far[row] : far_base(thin_row_sums(g, row, 0, g.classes, [](int64_t, float) {}));
        grad.base = f.x;
        grad.low = f.y;
    }
    if (quad >= quads) return;
    const int64_t c = (int64_t)quad * 4;
    float d[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < g.classes) {
        const float4 v = thin_logits(g, row, c);
        const float z[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = c + e < g.classes ? grad.of<true>(z[e], c + e == grad.target) : 0.f;
    }
    store_planes(dz + row * dz_ld, c, d);
}
// Sums of dz over kThinBiasRows rows at a time, [part][classes]: a block has 64 classes, eight to a thread.
constexpr int kThinBiasRows = 512;
__global__ __launch_bounds__(256) void thin_bias_kernel(const char* dz, int64_t dz_ld, int64_t rows, int64_t classes, float* db) {
    __shared__ float part[32][65];
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int64_t first = (int64_t)blockIdx.x * 64, from = (int64_t)blockIdx.y * kThinBiasRows, to = min(from + kThinBiasRows, rows);
    float sum[8] = {};
    if (first + c * 8 < (classes + 15) / 16 * 16) {
        const char* const at = dz + plane_at(first + c * 8);
        for (int64_t row = from + r; row < to; row += 32)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                Vec16<bf16_t> v;
                v.u = *reinterpret_cast<const uint4*>(at + row * dz_ld + p * 2 * kGroup);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += bf16_to_f32(v.e[e]);
            }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[r][c * 8 + e] = sum[e];
    __syncthreads();
    if (threadIdx.x >= 64 || first + threadIdx.x >= classes) return;
    float s = 0.f;
    for (int q = 0; q < 32; ++q) s += part[q][threadIdx.x];
    db[blockIdx.y * classes + first + threadIdx.x] = s;
}

// ---- joins --------------------------------------------------------------------------------------------------------------
// The sums of a row's tiles [tile][rows]: a block has ROWS rows, the rest of its threads share their tiles.  32 rows read half a
// kilobyte at a time; where that leaves few blocks, four.  far: not the results, but, of rows whose lse is far (whose sums alone
// are there), what dz forms log p from.
template <int ROWS>
__global__ __launch_bounds__(256) void classifier_join_kernel(const float4* __restrict__ sums, int64_t tiles, int64_t rows, RowFacts facts,
                                                              int64_t classes, const float* target_z, RowResults out, float2* far) {
    __shared__ float4 part[4][ROWS];
    const int r = threadIdx.x % ROWS, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    SoftmaxSums s;
    bool wanted = row < rows;
    if (far != nullptr && wanted) wanted = row_is_far(facts, row, classes);
    if (wanted) {
#pragma unroll 4
        for (int64_t t = threadIdx.x / ROWS; t < tiles; t += 256 / ROWS) {
            const float4 p = sums[t * rows + row];
            SoftmaxSums o;
            o.m = p.x; o.s = p.y; o.t = p.z;
            softmax_join(s, o);
        }
    }
#pragma unroll
    for (int o = ROWS; o < 64; o <<= 1) softmax_join(s, softmax_shuffle(s, o));
    if (lane < ROWS) part[threadIdx.x >> 6][r] = make_float4(s.m, s.s, s.t, 0.f);
    __syncthreads();
    if (threadIdx.x >= ROWS || row >= rows) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        const float4 p = part[w][r];
        SoftmaxSums o;
        o.m = p.x; o.s = p.y; o.t = p.z;
        softmax_join(s, o);
    }
    if (far == nullptr) write_results(out, facts.targets, classes, row, s, target_z[row]);       // (without a target: not looked at)
    else if (wanted) far[row] = far_base(s);
}

// out[r][c] = sum over the slots of part[slot][r][c]: GROUPS of a block's threads share the slots of 256 / GROUPS elements (one:
// four slots of 4 M elements 16 us, 28 with four; four: for many slots of few elements, whose chain would be the time)
template <typename OUT, int GROUPS>
__global__ __launch_bounds__(256) void sum_slots_kernel(const float* __restrict__ part, int slots, int64_t slot, int64_t cols, int64_t n, OUT* out, int64_t ld) {
    constexpr int WIDE = 256 / GROUPS;
    __shared__ float group[GROUPS][WIDE];
    const int e = threadIdx.x % WIDE;
    const int64_t i = (int64_t)blockIdx.x * WIDE + e;
    float s = 0.f;
    if (i < n) {
#pragma unroll 4
        for (int q = threadIdx.x / WIDE; q < slots; q += GROUPS) s += part[q * slot + i];
    }
    if constexpr (GROUPS > 1) {
        group[threadIdx.x / WIDE][e] = s;
        __syncthreads();
        if (threadIdx.x >= WIDE) return;
        s = 0.f;
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) s += group[q][e];
    }
    if (i >= n) return;
    const int64_t r = i / cols;
    out[r * ld + (i - r * cols)] = Elem<OUT>::from_f32(s);
}

// Copies of x and w (either may be left out: no blocks) in one launch: a block has 256 work items of one of them.
struct CopyOf { const void* src; char* dst; int64_t ld, n; unsigned blocks; };       // n: work items
struct Copies { CopyOf x, w; };
__device__ __forceinline__ bool copy_item(const Copies& a, CopyOf& c, int64_t& i) {
    const bool first = blockIdx.x < a.x.blocks;
    c = first ? a.x : a.w;
    i = (int64_t)(blockIdx.x - (first ? 0 : a.x.blocks)) * 256 + threadIdx.x;
    return i < c.n;
}

// rows of `cols` bf16 elements, copied to rows of `wide` (whole 16 bytes), zeros past them; a lane has 16 bytes
__global__ __launch_bounds__(256) void pad_rows_kernel(Copies a, int64_t cols, int64_t wide) {
    constexpr int VEC = Elem<bf16_t>::VEC;
    CopyOf o;
    int64_t i;
    if (!copy_item(a, o, i)) return;
    const int64_t vecs = wide / VEC, row = i / vecs, c = (i - row * vecs) * VEC;
    const bf16_t* const src = (const bf16_t*)o.src + row * o.ld;
    Vec16<bf16_t> v;
    if (c + VEC <= cols) {
        v = load_loose(src + c);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v.e[e] = c + e < cols ? src[c + e] : (bf16_t)0;
    }
    store_vec((bf16_t*)o.dst + row * wide + c, v);
}

// rows of float32 as three planes, zeros up to whole groups; a lane has four elements.  (What rounds to more than bf16
// holds takes its largest number first.)
__global__ __launch_bounds__(256) void split_rows_kernel(Copies a, int64_t cols, int64_t dst_ld) {
    CopyOf o;
    int64_t i;
    if (!copy_item(a, o, i)) return;
    const int64_t quads = dst_ld / kGroupBytes * (kGroup / 4), row = i / quads, c = (i - row * quads) * 4;
    const float* const p = (const float*)o.src + row * o.ld + c;
    float v[4];
    if (c + 4 <= cols) {
        const Vec16<float> t = load_loose(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = t.e[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c + e < cols ? p[e] : 0.f;
    }
    const float most = __uint_as_float(0x7f7f0000u);
    char* const to = o.dst + row * dst_ld + plane_at(c);
    float high[4], rest[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        high[e] = fminf(fmaxf(v[e], -most), most);
        rest[e] = v[e] - high[e];
    }
    *reinterpret_cast<uint2*>(to) = next_bf16(high);
#pragma unroll
    for (int e = 0; e < 4; ++e) rest[e] += high[e];
    *reinterpret_cast<uint2*>(to + 2 * kGroup) = next_bf16(rest);
    *reinterpret_cast<uint2*>(to + 4 * kGroup) = next_bf16(rest);
}

// No rows: the gradients of weights and bias are sums of nothing.
__global__ __launch_bounds__(256) void zero_rows_kernel(float* p, int64_t ld, int64_t cols, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i / cols * ld + i % cols] = 0.f;
}

constexpr int64_t kMiB = 1 << 20;
constexpr int64_t kTile = 128, kBigTile = 256;
constexpr int64_t kSmallTiles = 192;           // z of fewer 128x128 tiles is formed in float32 parts: by thin_logits_kernel up to 32 rows, else by gemm_kernel
constexpr int64_t kDzBytes = 1024 * kMiB;      // of dz at a time
constexpr int64_t kZeroAtOnce = 1ll << 30;     // elements of dw that one launch clears where there are no rows
constexpr int64_t kMostAtOnce = 1 << 20;       // classes of it: offsets in a tile of dz are counted in 31 bits
constexpr int64_t kWantBlocks = 512;           // of thin_sums_kernel
constexpr int64_t kChip = 256;                 // CUs: a block of a product each
constexpr int64_t kLeastOfZ = 256, kLeastOfGrads = 128;      // elements of the reduction to a cut
constexpr int64_t kWantWaves = 2048;           // of thin_logits_kernel, or more:
// a wave's steps at most.  Of longer ones the last few of many blocks take long alone; shorter ones write more parts: 1 x 4,096 x
// 100,000 float32 353 us without a limit, 314, 313, 324 and 397 with 16, 12, 8 and 4; 3 x 3,782 x 41,732 165, 152, 153, 153 and 162.
constexpr int64_t kMostSteps = 12;
constexpr int64_t kFewRows = 1024;            // a block of classifier_join_kernel has four of them
constexpr int64_t kThinPart = 4096;            // classes of a part of a row, at least, where rows are few

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// How a product of M x N outputs over K is laid out: tiles of 256x256 where they fill most of the chip, the reduction cut
// (into 1,024 elements at least) if need be, and little of them hangs over the edges; else of 128x128, the reduction cut
// towards one block per CU, `least` elements to a cut at least (0: not cut).  Two blocks per CU write twice the parts, which have to be added up: 64 x
// 4,096 x 5,000 float32 83 + 156 us (loss + gradient) with two, 77 + 141 with one, 91 + 173 with a half; 333 x 515 x 10,007 float32 44 + 115, 44 + 108, 44 + 123.
// z's parts are read by two kernels, so that its shortest cut is longer: 100 x 4,096 x 1,000 bf16 16 us with 256, 19 with 128,
// the gradients 45.8 and 43.4.
struct Layout { bool big; int64_t cuts, per_cut; };        // per_cut: elements of the reduction
Layout lay_out(int64_t M, int64_t N, int64_t K, int64_t least) {
    Layout l = {};
    const int64_t big = ceil_div(M, kBigTile) * ceil_div(N, kBigTile), tiles = ceil_div(M, kTile) * ceil_div(N, kTile);
    const int64_t big_cuts = least > 0 && big < kChip ? std::max<int64_t>(1, std::min<int64_t>(kChip / big, K / 1024)) : 1;
    l.big = big * big_cuts * 4 >= kChip * 3 && M * N * 4 >= big * kBigTile * kBigTile * 3;
    int64_t want = 1;
    if (l.big) want = big_cuts;
    else if (least > 0 && tiles < kChip) want = std::min<int64_t>(std::max<int64_t>(1, K / least), kChip / tiles);
    l.per_cut = round_up(ceil_div(K, want), 64);
    l.cuts = ceil_div(K, l.per_cut);
    return l;
}

// everything a call does, from its sizes and alignments alone
struct Plan {
    int esz;
    bool thin;
    // x and w as the products on tiles read them: bf16 where they lie, or copied to whole 16 bytes; float32 copied to three planes
    bool tiles;                // there are such products
    int64_t wide;              // bf16: features up to whole 16 bytes
    bool pad_x, pad_w, split;
    int64_t split_ld;          // bytes
    bool narrow;               // thin_logits_kernel
    int thin_cuts, thin_steps;         // of the reduction: cuts over blocks, steps of a wave of it
    Layout thin_z;
    int64_t z_ld;
    int thin_parts;
    int64_t thin_part;
    bool far_here;             // dz's blocks sum up the rows whose lse is far
    int64_t chunk, chunks;     // of classes, in the backward pass
    Layout sums, z, dx, dw;    // sums: z of all classes; z: of a piece of them
    int64_t sum_tiles, z_tiles;        // of classes; of rows (backward)
    // workspace
    int64_t x_at, w_at, z_at, sums_at, target_at, far_at, dz_at, dz_ld, dx_at, dw_at, db_at, bytes;
};

Plan plan_of(int dtype, int64_t rows, int64_t dim, int64_t classes, bool aligned_x, bool aligned_w, bool backward) {
    Plan p = {};
    p.esz = dtype == 1 ? 2 : 4;
    const int64_t tiles_r = ceil_div(rows, kTile), tiles_c = ceil_div(classes, kTile);
    int64_t o = 0;
    auto take = [&](int64_t bytes) { const int64_t at = o; o += round_up(bytes, 256); return at; };
    // (tiles of 128 rows read w faster where they need no copies of it: 32 rows of 4,096 bf16 features, 50,000 classes 104 us on
    // tiles, 155 by rows; 4 rows, 128,000 classes 200 against 241)
    p.narrow = rows <= 32 && classes <= kMostAtOnce && (dtype != 1 || !aligned_x || !aligned_w || tiles_r * tiles_c < kSmallTiles);
    p.thin = p.narrow || tiles_r * tiles_c < kSmallTiles;
    p.tiles = !p.narrow || backward;
    p.wide = round_up(dim, 8);
    p.pad_x = p.tiles && dtype == 1 && !aligned_x;
    p.pad_w = p.tiles && dtype == 1 && !aligned_w;
    p.split = p.tiles && dtype != 1;
    p.split_ld = planes_bytes(dim);
    p.x_at = take(p.split ? rows * p.split_ld : p.pad_x ? rows * p.wide * p.esz : 0);
    p.w_at = take(p.split ? classes * p.split_ld : p.pad_w ? classes * p.wide * p.esz : 0);
    if (p.thin) {
        if (p.narrow) {
            const int64_t steps = ceil_div(dim * p.esz, kStepBytes);
            const int64_t waves = std::max<int64_t>(4, std::min<int64_t>(std::max(kWantWaves / ceil_div(classes, 32), ceil_div(steps, kMostSteps)), steps));
            p.thin_cuts = (int)std::max<int64_t>(1, waves / 4);
            p.thin_steps = (int)ceil_div(steps, p.thin_cuts * 4);
            p.thin_cuts = (int)ceil_div(steps, p.thin_steps * 4);
        } else {
            p.thin_z = lay_out(rows, classes, dim, kLeastOfZ);
            p.thin_cuts = (int)p.thin_z.cuts;
        }
        p.z_ld = round_up(classes, 32);
        const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(ceil_div(classes, kThinPart), kWantBlocks / rows));
        p.thin_part = round_up(ceil_div(classes, parts), 4);
        p.thin_parts = (int)ceil_div(classes, p.thin_part);
        p.z_at = take(p.thin_cuts * rows * p.z_ld * 4);
    }
    p.sums = lay_out(classes, rows, 1, 0);
    p.sum_tiles = ceil_div(classes, p.sums.big ? kBigTile : kTile);
    if (!backward) {
        p.sums_at = take(p.thin ? (p.thin_parts > 1 ? p.thin_parts * rows * 16 : 0) : p.sum_tiles * rows * 16);
        p.target_at = take(rows * 4);
    } else {
        const int64_t at_once = std::min(kMostAtOnce, std::max<int64_t>(1, kDzBytes / (rows * 6 * kTile)) * kTile);
        p.chunks = p.thin ? 1 : ceil_div(classes, at_once);
        p.chunk = round_up(ceil_div(classes, p.chunks), kTile);
        p.chunks = ceil_div(classes, p.chunk);
        const int64_t n = std::min(p.chunk, classes);
        p.dz_ld = planes_bytes(n);
        p.far_here = p.thin && thin_blocks(round_up(classes, 16) / 4) <= kFarHere;
        p.far_at = take(p.far_here ? 0 : rows * 8);
        // (the far rows' sums are joined before dz is formed)
        p.dz_at = p.sums_at = take(std::max(rows * p.dz_ld, p.far_here ? 0 : (p.thin ? p.thin_parts : p.sum_tiles) * rows * 16));
        p.z = lay_out(n, rows, 1, 0);
        p.z_tiles = p.thin ? ceil_div(rows, kThinBiasRows) : ceil_div(rows, p.z.big ? kBigTile : kTile);
        p.dx = lay_out(rows, dim, n, kLeastOfGrads);
        p.dw = lay_out(n, dim, rows, kLeastOfGrads);
        p.dx_at = take(p.chunks > 1 || p.dx.cuts > 1 ? p.dx.cuts * rows * dim * 4 : 0);
        p.dw_at = take(p.dw.cuts > 1 ? p.dw.cuts * n * dim * 4 : 0);
        p.db_at = take(p.z_tiles > 1 ? p.z_tiles * n * 4 : 0);
    }
    p.bytes = o;
    return p;
}

bool lies_aligned(const void* p, int64_t ld, int64_t dim, int esz) {
    return (uintptr_t)p % 16 == 0 && ld * esz % 16 == 0 && dim * esz % 16 == 0 && ld * esz <= (1 << 23);
}

// x and w as operands whose reduction lies along them
struct Inputs { Operand x, w; };
template <typename T> Inputs inputs_of(const ClassifierCall& c, const Plan& p, char* work, hipStream_t st) {
    if (!p.tiles) return Inputs{};
    const int64_t items = p.split ? p.split_ld / kGroupBytes * (kGroup / 4) : p.wide / 8;        // of a row
    Copies a = {};
    int64_t rows = 0;
    auto operand = [&](const void* src, int64_t ld, int64_t n, bool pad, int64_t copy_at, CopyOf& copy) {
        if (!p.split && !pad) return Operand{(const char*)src, ld * 2, n, p.wide, 1};
        rows += n;
        copy = CopyOf{src, work + copy_at, ld, n * items, (unsigned)ceil_div(n * items, 256)};
        return p.split ? Operand{copy.dst, p.split_ld, n, round_up(c.dim, 16), 3} : Operand{copy.dst, p.wide * 2, n, p.wide, 1};
    };
    Inputs in;
    in.x = operand(c.x, c.ldx, c.rows, p.pad_x, p.x_at, a.x);
    in.w = operand(c.w, c.ldw, c.classes, p.pad_w, p.w_at, a.w);
    const dim3 grid(a.x.blocks + a.w.blocks);
    if (p.split) {
        ProfScope ps("classifier_split", 0.0, (4.0 * c.dim + p.split_ld) * rows, st);
        hipLaunchKernelGGL(split_rows_kernel, grid, dim3(256), 0, st, a, c.dim, p.split_ld);
    } else if (rows > 0) {
        ProfScope ps("classifier_pad", 0.0, 2.0 * rows * (c.dim + p.wide), st);
        hipLaunchKernelGGL(pad_rows_kernel, grid, dim3(256), 0, st, a, c.dim, p.wide);
    }
    return in;
}
// the same memory with its lines the reduction: `rows` outputs (up to whole pieces) by `k` lines
Operand across(const Operand& o, int64_t rows, int64_t k) { return Operand{o.p, o.ld, rows, k, o.stored}; }

// a by b, `cut` elements of the reduction to a block, on tiles as laid out
template <int PA, int PB> void lay_tiles(GemmArgs& g, int64_t cut, bool big) {
    const int64_t side = big ? kBigTile : kTile, KS = big ? Steps<PA, PB, 256>::KS : Steps<PA, PB, 128>::KS;
    g.steps = (int)ceil_div(g.a.k, KS);
    g.steps_per_cut = (int)std::min<int64_t>(g.steps, cut / KS);       // (a cut is a multiple of 64)
    g.tiles_m = (int)ceil_div(g.a.rows, side);
    g.tiles_n = (int)ceil_div(g.b.rows, side);
    g.group = big ? 4 : 8;
}
template <Want WANT, int PA, int PB, bool A_ALONG, bool B_ALONG, typename OUT> void launch_gemm(GemmArgs& g, int64_t cut, bool big, hipStream_t st) {
    lay_tiles<PA, PB>(g, cut, big);
    const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * ceil_div(g.steps, g.steps_per_cut)));
    if (big) hipLaunchKernelGGL((gemm_kernel<WANT, PA, PB, A_ALONG, B_ALONG, OUT, Shape256>), grid, dim3(512), 0, st, g);
    else hipLaunchKernelGGL((gemm_kernel<WANT, PA, PB, A_ALONG, B_ALONG, OUT, Shape128>), grid, dim3(512), 0, st, g);
}
constexpr int64_t kWhole = 1ll << 30;          // no cuts

template <typename T> ThinRows thin_forward(const Inputs& in, const float* bias, const RowFacts& facts, const Plan& p, const ClassifierCall& c, char* work, hipStream_t st) {
    constexpr int P = sizeof(T) == 2 ? 1 : 3;
    float* const z = (float*)(work + p.z_at);
    ProfScope ps("classifier_thin_logits", 2.0 * c.rows * c.classes * c.dim, (double)(c.rows + c.classes) * c.dim * p.esz, st);
    if (p.narrow) {
        ThinArgs t = {};
        t.w = Matrix{(const char*)c.w, c.ldw * p.esz, c.classes};
        t.x = Matrix{(const char*)c.x, c.ldx * p.esz, c.rows};
        t.row_bytes = c.dim * p.esz;
        t.steps = (int)ceil_div(t.row_bytes, kStepBytes);
        t.steps_per_wave = p.thin_steps;
        t.tiles = (int)ceil_div(c.classes, 32);
        t.z = z;
        t.z_ld = p.z_ld;
        hipLaunchKernelGGL((thin_logits_kernel<T>), dim3((unsigned)(t.tiles * p.thin_cuts)), dim3(256), 0, st, t);
    } else {
        GemmArgs g = {};
        g.a = in.x;
        g.b = in.w;
        g.out = z;
        g.out_ld = p.z_ld;
        g.out_cut = c.rows * p.z_ld;
        launch_gemm<PRODUCT, P, P, true, true, float>(g, p.thin_z.per_cut, p.thin_z.big, st);
    }
    return ThinRows{z, p.z_ld, c.rows, c.classes, p.thin_cuts, bias, facts};
}

// z on tiles whose sums go to `sums`
GemmArgs tile_sums(const Inputs& in, const ClassifierCall& c, const RowFacts& facts, float4* sums) {
    GemmArgs g = {};
    g.a = in.w;
    g.b = in.x;
    g.bias = c.bias;
    g.classes = g.all_classes = c.classes;
    g.facts = facts;
    g.sums = sums;
    return g;
}
void launch_join(const float4* sums, int64_t tiles, const ClassifierCall& c, const RowFacts& facts, const float* target_z, const RowResults& res, float2* far,
                 hipStream_t st) {
#define EDL_JOIN(RR) hipLaunchKernelGGL((classifier_join_kernel<RR>), dim3((unsigned)ceil_div(c.rows, RR)), dim3(256), 0, st, sums, tiles, c.rows, facts, c.classes, target_z, res, far)
    if (c.rows <= kFewRows) EDL_JOIN(4);
    else EDL_JOIN(32);
#undef EDL_JOIN
}

template <typename T> void forward(const ClassifierCall& c, const ClassifierOut& out, hipStream_t st) {
    constexpr int P = sizeof(T) == 2 ? 1 : 3;
    const Plan p = plan_of(c.dtype, c.rows, c.dim, c.classes, lies_aligned(c.x, c.ldx, c.dim, sizeof(T)), lies_aligned(c.w, c.ldw, c.dim, sizeof(T)), false);
    char* const work = (char*)c.work;
    const Inputs in = inputs_of<T>(c, p, work, st);
    RowFacts facts = {};
    facts.targets = c.targets;
    const RowResults res = {out.log_prob, out.entropy, out.lse};
    float4* const sums = (float4*)(work + p.sums_at);
    float* const target_z = (float*)(work + p.target_at);
    int64_t tiles = p.sum_tiles;
    if (p.thin) {
        const ThinRows z = thin_forward<T>(in, c.bias, facts, p, c, work, st);
        ProfScope ps("classifier_thin_sums", 0.0, 4.0 * p.thin_cuts * c.rows * c.classes, st);
        hipLaunchKernelGGL(thin_sums_kernel, dim3((unsigned)(c.rows * p.thin_parts)), dim3(256), 0, st, z, p.thin_parts, p.thin_part, sums, target_z, res, false);
        tiles = p.thin_parts;
        if (tiles == 1) return;
    } else {
        GemmArgs g = tile_sums(in, c, facts, sums);
        g.target_z = target_z;
        ProfScope ps("classifier_sums", 2.0 * c.rows * c.classes * c.dim, (double)(c.rows + c.classes) * c.dim * p.esz, st);
        launch_gemm<SUMS, P, P, true, true, float>(g, kWhole, p.sums.big, st);
    }
    ProfScope ps("classifier_join", 0.0, 16.0 * tiles * c.rows, st);
    launch_join(sums, tiles, c, facts, target_z, res, nullptr, st);
}

template <typename OUT> void sum_slots(const float* part, int64_t slots, int64_t rows, int64_t cols, OUT* out, int64_t ld, hipStream_t st) {
    const int64_t n = rows * cols;
    ProfScope ps("classifier_sum", 0.0, 4.0 * slots * n + sizeof(OUT) * (double)n, st);
    if (slots >= 16) hipLaunchKernelGGL((sum_slots_kernel<OUT, 4>), dim3((unsigned)ceil_div(n, 64)), dim3(256), 0, st, part, (int)slots, n, cols, n, out, ld);
    else hipLaunchKernelGGL((sum_slots_kernel<OUT, 1>), dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, st, part, (int)slots, n, cols, n, out, ld);
}

template <typename T> void backward(const ClassifierCall& c, const ClassifierGrads& d, hipStream_t st) {
    constexpr int P = sizeof(T) == 2 ? 1 : 3;
    const Plan p = plan_of(c.dtype, c.rows, c.dim, c.classes, lies_aligned(c.x, c.ldx, c.dim, sizeof(T)), lies_aligned(c.w, c.ldw, c.dim, sizeof(T)), true);
    char* const work = (char*)c.work;
    const Inputs in = inputs_of<T>(c, p, work, st);
    const RowFacts facts = {c.targets, d.lse, d.entropy, d.dlog_prob, d.dentropy};
    char* const dz = work + p.dz_at;
    float2* const far = (float2*)(work + p.far_at);
    if (!p.thin) {
        GemmArgs g = tile_sums(in, c, facts, (float4*)(work + p.sums_at));
        lay_tiles<P, P>(g, kWhole, p.sums.big);
        {
            ProfScope ps("classifier_far_sums", 0.0, 0.0, st);
            const dim3 grid((unsigned)std::min<int64_t>(kChip, (int64_t)g.tiles_m * g.tiles_n));
            if (p.sums.big) hipLaunchKernelGGL((far_sums_kernel<P, Shape256>), grid, dim3(512), 0, st, g);
            else hipLaunchKernelGGL((far_sums_kernel<P, Shape128>), grid, dim3(512), 0, st, g);
        }
        ProfScope ps("classifier_far_join", 0.0, 0.0, st);
        launch_join(g.sums, p.sum_tiles, c, facts, nullptr, RowResults{}, far, st);
    }
    const bool parts_of_dx = p.chunks > 1 || p.dx.cuts > 1;
    for (int64_t q = 0; q < p.chunks; ++q) {
        const int64_t from = q * p.chunk, n = std::min(p.chunk, c.classes - from), cols = round_up(n, 16);
        Operand wq = in.w;
        wq.p += from * wq.ld;
        wq.rows = n;
        float* const db = d.dbias == nullptr ? nullptr : p.z_tiles > 1 ? (float*)(work + p.db_at) : d.dbias + from;
        if (p.thin) {
            const ThinRows z = thin_forward<T>(in, c.bias, facts, p, c, work, st);
            if (!p.far_here) {
                float4* const sums = (float4*)(work + p.sums_at);
                {
                    ProfScope ps("classifier_far_sums", 0.0, 0.0, st);
                    hipLaunchKernelGGL(thin_sums_kernel, dim3((unsigned)(c.rows * p.thin_parts)), dim3(256), 0, st, z, p.thin_parts, p.thin_part, sums, nullptr, RowResults{}, true);
                }
                ProfScope ps("classifier_far_join", 0.0, 0.0, st);
                launch_join(sums, p.thin_parts, c, facts, nullptr, RowResults{}, far, st);
            }
            {
                ProfScope ps("classifier_thin_grads", 0.0, (4.0 * p.thin_cuts + 6.0) * c.rows * c.classes, st);
                hipLaunchKernelGGL(thin_grads_kernel, dim3((unsigned)(c.rows * thin_blocks(cols / 4))), dim3(256), 0, st, z, dz, p.dz_ld, (int)cols,
                                   p.far_here ? nullptr : far);
            }
            if (db != nullptr) {
                ProfScope ps("classifier_thin_bias", 0.0, 6.0 * c.rows * c.classes, st);
                hipLaunchKernelGGL(thin_bias_kernel, dim3((unsigned)ceil_div(n, 64), (unsigned)p.z_tiles), dim3(256), 0, st, dz, p.dz_ld, c.rows, n, db);
            }
        } else {
            GemmArgs g = {};
            g.a = wq;
            g.b = in.x;
            g.bias = c.bias;
            g.first_class = from;
            g.classes = from + n;
            g.all_classes = c.classes;
            g.facts = facts;
            g.far = far;
            g.dz = dz;
            g.dz_ld = p.dz_ld;
            g.dz_classes = (int)cols;
            g.db = db;
            g.db_ld = n;
            ProfScope ps("classifier_dz", 2.0 * c.rows * n * c.dim, (double)(c.rows + n) * c.dim * p.esz + 6.0 * c.rows * n, st);
            launch_gemm<GRADS, P, P, true, true, float>(g, kWhole, p.z.big, st);
        }
        if (db != nullptr && p.z_tiles > 1) sum_slots<float>(db, p.z_tiles, 1, n, d.dbias + from, n, st);
        {
            GemmArgs g = {};
            g.a = Operand{dz, p.dz_ld, c.rows, cols, 3};
            g.b = across(wq, c.dim, n);
            ProfScope ps("classifier_dx", 2.0 * c.rows * n * c.dim, 6.0 * c.rows * n + (double)p.esz * (n + c.rows) * c.dim, st);
            if (parts_of_dx) {         // (later pieces of the classes are added to the first one's cuts, of which the last may have fewer)
                g.out = (float*)(work + p.dx_at);
                g.out_ld = c.dim;
                g.out_cut = c.rows * c.dim;
                if (q == 0) launch_gemm<PRODUCT, P == 1 ? 2 : 3, P, true, false, float>(g, p.dx.per_cut, p.dx.big, st);
                else launch_gemm<ADDED, P == 1 ? 2 : 3, P, true, false, float>(g, p.dx.per_cut, p.dx.big, st);
            } else {
                g.out = d.dx;
                g.out_ld = d.lddx;
                launch_gemm<PRODUCT, P == 1 ? 2 : 3, P, true, false, T>(g, kWhole, p.dx.big, st);
            }
        }
        if (q + 1 == p.chunks && parts_of_dx) sum_slots<T>((const float*)(work + p.dx_at), p.dx.cuts, c.rows, c.dim, (T*)d.dx, d.lddx, st);
        {
            GemmArgs g = {};
            g.a = Operand{dz, p.dz_ld, n, c.rows, 3};
            g.b = across(in.x, c.dim, c.rows);
            const bool cut = p.dw.cuts > 1;
            g.out = cut ? (float*)(work + p.dw_at) : d.dw + from * d.lddw;
            g.out_ld = cut ? c.dim : d.lddw;
            g.out_cut = n * c.dim;
            {
                ProfScope ps("classifier_dw", 2.0 * c.rows * n * c.dim, 6.0 * c.rows * n + (double)p.esz * c.rows * c.dim + 4.0 * n * c.dim, st);
                launch_gemm<PRODUCT, 3, P, false, false, float>(g, p.dw.per_cut, p.dw.big, st);
            }
            if (cut) sum_slots<float>((const float*)(work + p.dw_at), p.dw.cuts, n, c.dim, d.dw + from * d.lddw, d.lddw, st);
        }
    }
}

}  // namespace

size_t classifier_work_bytes(const ClassifierCall& c, bool backward) {
    const int esz = c.dtype == 1 ? 2 : 4;
    // (however they lie: the most of both ways)
    int64_t most = 0;
    for (int way = 0; way < 4; ++way) {
        const bool ax = (way & 1) != 0, aw = (way & 2) != 0;
        if (c.x != nullptr && ax != lies_aligned(c.x, c.ldx, c.dim, esz)) continue;
        if (c.w != nullptr && aw != lies_aligned(c.w, c.ldw, c.dim, esz)) continue;
        most = std::max(most, plan_of(c.dtype, c.rows, c.dim, c.classes, ax, aw, backward).bytes);
    }
    return (size_t)most;
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
