// Log probabilities of given classes, entropy and the most likely classes of rows of logits, in one pass over them, and the
// gradient of the logits.
//
// With the running sums of softmax_sums.h a lane reads each logit once; lanes, waves and parts of a row are then joined.
// Bound: HBM and the vector units together.  A logit costs 9.9 instructions by the counters (conversion, maximum, one exponential at a
// quarter of the rate, two sums), 13 issue slots of the 14 that reading bf16 at 5.5 TB/s leaves; with the best 10 of 49,999 18.4,
// whose slots are all of the kernel's time.
//
// The best k ride along: after a round of loads only vectors that reach the k-th best of what the wave has seen are put aside
// in LDS, and their logits then entered into the wave's list, k log(rounds) of them in random order beside the first
// round's, whose bound is the k-th of the 64 lanes' largest.  Entering them where they lie, in registers, means that code once
// for each of a lane's 32 logits: 11 KB of instructions, whose first fetch alone took most of the 13 us of a call for one row.
//
// Measured: 4,096 x 49,999 bf16 with 10 alternatives 114 us (3.6 TB/s), 8,192 x 32,768 bf16 without 122 us (4.4 TB/s) and their
// gradient 214 us (5.0 TB/s) and 5 for the launch that looks for rows whose lse is far (395 in all if every row is); 1 x 32,000 bf16 with 5 in eight parts 8 + 4 us; 256 x 1,000 float32 with 5, a wave to a row, 6 us.
#include <algorithm>

#include "operators.h"
#include "profiler.h"
#include "softmax_sums.h"
#include "unaligned.h"

namespace edl {

namespace {

struct RowArgs {
    int64_t ld, rows;
    uint32_t classes;
    uint32_t part;             // classes of a part of a row (all of them: rows are not cut)
    int parts, k;
    const int32_t* targets;    // null: none
    float *log_prob, *entropy, *lse, *top_value;
    int32_t* top_class;
    float* sums;               // parts > 1: [rows][parts][4]: m, s, t
    TopKey* keys;              // ... [rows][parts][k]
};

// One wave writes a row's results.  zt: its target's logit, if it has one.
__device__ __forceinline__ void write_row(const RowArgs& a, int64_t row, const SoftmaxSums& sums, bool has_target, float zt, const TopKey& top) {
    const int lane = threadIdx.x & 63;
    if (lane == 0) {
        a.lse[row] = softmax_lse(sums);
        a.entropy[row] = softmax_entropy(sums);
        if (a.targets != nullptr) a.log_prob[row] = has_target ? softmax_log_prob(sums, zt) : 0.f;
    }
    if (lane < a.k) {
        a.top_value[row * a.k + lane] = softmax_log_prob(sums, top_value(top));
        a.top_class[row * a.k + lane] = (int32_t)~top.lo;
    }
}

template <typename T>
__device__ __forceinline__ float target_logit(const RowArgs& a, const T* logits, int64_t row, bool& has) {
    has = false;
    if (a.targets == nullptr) return 0.f;
    const int32_t t = a.targets[row];
    has = t >= 0 && (uint32_t)t < a.classes;
    return has ? Elem<T>::to_f32(logits[row * a.ld + t]) : 0.f;
}

// WAVES = 1: a wave has a row of its own (four to a block); 4: a block has a part of a row.
template <typename T, int WAVES, bool TOP>
__global__ __launch_bounds__(256) void log_probs_kernel(const T* __restrict__ logits, RowArgs a) {
    constexpr int VEC = Elem<T>::VEC, U = 4, WIDE = 64 * VEC, STRIDE = WAVES * WIDE;
    // a wave's vectors of one round that hold candidates, and which of the wave's vectors of the round each is
    __shared__ uint4 aside[TOP ? 4 : 1][TOP ? U * 64 : 1];
    __shared__ uint8_t aside_at[TOP ? 4 : 1][TOP ? U * 64 : 1];
    __shared__ TopKey scratch[TOP ? 4 : 1][TOP ? 64 : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t row;
    int part = 0;
    if (WAVES == 1) {
        row = (int64_t)blockIdx.x * 4 + wave;
        if (row >= a.rows) return;
    } else if (a.parts == 1) {
        row = blockIdx.x;
    } else {
        row = blockIdx.x / (unsigned)a.parts;
        part = (int)(blockIdx.x - (unsigned)row * (unsigned)a.parts);
    }
    const uint32_t lo = (uint32_t)part * a.part, hi = min(lo + a.part, a.classes);
    const T* const z = logits + row * a.ld;
    SoftmaxSums sums;
    TopList top;
    if (TOP) top.clear();
    const uint32_t mine = (WAVES == 1 ? lane : threadIdx.x) * VEC;
    for (uint32_t at = lo; at < hi; at += U * STRIDE) {
        Vec16<T> w[U];
        if (at + U * STRIDE <= hi) {           // (the same for all lanes: the loads follow each other without a branch)
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = load_loose(z + at + u * STRIDE + mine);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t c = at + u * STRIDE + mine;
                if (c + VEC <= hi) {
                    w[u] = load_loose(z + c);
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) w[u].e[e] = c + e < hi ? z[c + e] : Elem<T>::from_f32(-INFINITY);
                }
            }
        }
        float mv[U], round = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mv[u] = Elem<T>::to_f32(w[u].e[0]);
#pragma unroll
            for (int e = 1; e < VEC; ++e) mv[u] = fmaxf(mv[u], Elem<T>::to_f32(w[u].e[e]));
            round = fmaxf(round, mv[u]);
        }
        if (round > sums.m) softmax_rebase(sums, round);
        const float base = softmax_base(sums);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) softmax_add(sums, Elem<T>::to_f32(w[u].e[e]), base);
        }
        if (TOP) {
            if (at == lo) top.expect(at + mine < hi ? top_key(round, 0).hi : 0, a.k);
            const float bar = top.bar();
            if (__ballot(at + mine < hi && !(round < bar)) == 0) continue;
            int n = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = at + u * STRIDE + mine < hi && !(mv[u] < bar);
                const uint64_t who = __ballot(in);
                if (in) {
                    const int to = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                    aside[wave][to] = w[u].u;
                    aside_at[wave][to] = (uint8_t)(u * 64 + lane);
                }
                n += __popcll(who);
            }
            wave_lds_handover();
            for (int i = lane; i - lane < n * VEC; i += 64) {
                TopKey c = {0, 0};
                if (i < n * VEC) {
                    const int p = aside_at[wave][i / VEC];
                    const uint32_t cls = at + (p >> 6) * STRIDE + (WAVES == 1 ? 0 : wave * WIDE) + (p & 63) * VEC + i % VEC;
                    if (cls < hi) c = top_key(Elem<T>::to_f32(reinterpret_cast<const T*>(aside[wave])[i]), cls);
                }
                top.offer(c, a.k, scratch[wave]);
            }
            wave_lds_handover();
        }
    }
    softmax_join_wave(sums);
    if (WAVES == 4) {
        __shared__ float4 wave_sums[4];
        __shared__ TopKey wave_keys[TOP ? 4 * 64 : 1];
        if (lane == 0) wave_sums[wave] = make_float4(sums.m, sums.s, sums.t, 0.f);
        if (TOP && lane < a.k) wave_keys[wave * a.k + lane] = top.mine;
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            SoftmaxSums other;
            other.m = wave_sums[w].x; other.s = wave_sums[w].y; other.t = wave_sums[w].z;
            softmax_join(sums, other);
        }
        if (TOP) {
            // a wave's k-th has k - 1 before it: what is worse than the best of those is none of the block's best
            for (int w = 1; w < 4; ++w) {
                const TopKey t = wave_keys[w * a.k + a.k - 1];
                if (t.hi != 0) top.raise(TopKey{t.hi, t.lo - 1});
            }
            for (int i = a.k; i < 4 * a.k; i += 64) top.offer(i + lane < 4 * a.k ? wave_keys[i + lane] : TopKey{0, 0}, a.k, scratch[0]);
        }
    }
    if (WAVES == 4 && a.parts > 1) {
        const int64_t at = row * a.parts + part;
        if (lane == 0) *reinterpret_cast<float4*>(a.sums + 4 * at) = make_float4(sums.m, sums.s, sums.t, 0.f);
        if (TOP && lane < a.k) a.keys[at * a.k + lane] = top.mine;
        return;
    }
    bool has;
    const float zt = target_logit(a, logits, row, has);
    write_row(a, row, sums, has, zt, top.mine);
}

// The parts of a row: a wave per row.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void log_probs_join_kernel(const T* __restrict__ logits, RowArgs a) {
    __shared__ TopKey scratch[TOP ? 4 : 1][TOP ? 64 : 1];
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.rows) return;
    SoftmaxSums sums;
    if (lane < a.parts) {          // (64 parts at most)
        const float4 p = *reinterpret_cast<const float4*>(a.sums + 4 * (row * a.parts + lane));
        sums.m = p.x; sums.s = p.y; sums.t = p.z;
    }
    softmax_join_wave(sums);
    TopList top;
    if (TOP) {
        top.clear();
        const int n = a.parts * a.k;
        uint32_t best = 0;
        for (int i = lane; i < n; i += 64) best = max(best, a.keys[row * n + i].hi);
        top.expect(best, a.k);
        for (int i = 0; i < n; i += 64) top.offer(i + lane < n ? a.keys[row * n + i + lane] : TopKey{0, 0}, a.k, scratch[threadIdx.x >> 6]);
    }
    bool has;
    const float zt = target_logit(a, logits, row, has);
    write_row(a, row, sums, has, zt, top.mine);
}

struct GradArgs {
    Pieces m;
    int64_t ld, ldd;
    RowFacts facts;
    unsigned far_blocks;       // for the rows whose lse is far
    bool far_by_wave;          // a wave has such a row, else a block
};

// Rows whose lse is far (softmax_sums.h): their sums, then their gradient, by a wave or a block of 256 for each such row, since
// dlogits may lie where the logits do.  Rows are dealt out one by one, so that a run of far ones spreads over the chip; a
// lane looks at one row at a time.
template <typename T, int LANES>
__device__ __forceinline__ void far_rows_by(const T* logits, T* dlogits, const GradArgs& a, unsigned block) {
    constexpr int U = 4, WIDE = LANES * kPiece;
    __shared__ float4 wave_sums[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int me = LANES == 64 ? lane : (int)threadIdx.x;
    const int64_t groups = (int64_t)a.far_blocks * (256 / LANES), group = (int64_t)block * (256 / LANES) + (LANES == 64 ? wave : 0);
    for (int64_t first = group; first < a.m.rows; first += groups * 64) {
        // (each wave of a block looks at the same 64 rows)
        const int64_t look = first + lane * groups;
        for (uint64_t left = __ballot(look < a.m.rows && row_is_far(a.facts, look, a.m.cols)); left != 0; left &= left - 1) {
            const int64_t row = first + (int64_t)__builtin_ctzll(left) * groups;
            const T* const z = logits + row * a.ld;
            T* const d = dlogits + row * a.ldd;
            float v[U][kPiece];
            auto load = [&](int64_t at) {          // (past the row's end: masked)
                if (at + (U - 1) * WIDE + kPiece <= a.m.cols) {
#pragma unroll
                    for (int u = 0; u < U; ++u) load_piece(z + at + u * WIDE, v[u]);
                    return;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t c = at + u * WIDE;
                    if (c + kPiece <= a.m.cols) {
                        load_piece(z + c, v[u]);
                    } else {
#pragma unroll
                        for (int e = 0; e < kPiece; ++e) v[u][e] = c + e < a.m.cols ? Elem<T>::to_f32(z[c + e]) : -INFINITY;
                    }
                }
            };
            SoftmaxSums sums;
            for (int64_t at = me * kPiece; at < a.m.cols; at += U * WIDE) {
                load(at);
                float m = sums.m;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) m = fmaxf(m, v[u][e]);
                softmax_rebase(sums, m);
                const float base = softmax_base(sums);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) softmax_add(sums, v[u][e], base);
            }
            softmax_join_wave(sums);
            if (LANES == 256) {
                if (lane == 0) wave_sums[wave] = make_float4(sums.m, sums.s, sums.t, 0.f);
                __syncthreads();
                SoftmaxSums all;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    SoftmaxSums o;
                    o.m = wave_sums[w].x; o.s = wave_sums[w].y; o.t = wave_sums[w].z;
                    softmax_join(all, o);
                }
                sums = all;
                __syncthreads();       // (the next row writes them again)
            }
            LogitGrad grad = logit_grad(a.facts, row, a.m.cols);
            const float2 far = far_base(sums);
            grad.base = far.x;
            grad.low = far.y;
            for (int64_t at = me * kPiece; at < a.m.cols; at += U * WIDE) {
                load(at);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t c = at + u * WIDE, hot = grad.target - c;
#pragma unroll
                    for (int e = 0; e < kPiece; ++e) v[u][e] = grad.template of<true>(v[u][e], e == hot);
                    if (c + kPiece <= a.m.cols) {
                        store_piece(d + c, v[u]);
                    } else {
#pragma unroll
                        for (int e = 0; e < kPiece; ++e)
                            if (c + e < a.m.cols) d[c + e] = Elem<T>::from_f32(v[u][e]);
                    }
                }
            }
        }
    }
}

template <typename T> __device__ __forceinline__ void far_rows(const T* logits, T* dlogits, const GradArgs& a, unsigned block) {
    if (a.far_by_wave) far_rows_by<T, 64>(logits, dlogits, a, block);
    else far_rows_by<T, 256>(logits, dlogits, a, block);
}
template <typename T> __global__ __launch_bounds__(256) void far_rows_kernel(const T* logits, T* dlogits, GradArgs a) { far_rows(logits, dlogits, a, blockIdx.x); }

// Element-wise once the row's numbers are known, which its lanes read from cache.  Of small calls (U = 1) the first blocks have the rows
// whose lse is far, which spares them a launch; large ones leave those to far_rows_kernel, because with its code beside this
// one 8,192 x 32,768 bf16 takes 250 us, without 216.
template <typename T, int U>
__global__ __launch_bounds__(256) void log_probs_grad_kernel(const T* logits, T* dlogits, GradArgs a) {
    unsigned block = blockIdx.x;
    if constexpr (U == 1) {
        if (block < a.far_blocks) {
            far_rows(logits, dlogits, a, block);
            return;
        }
        block -= a.far_blocks;
    }
    int64_t at0;
    const int64_t row0 = block_first_row<U>(a.m, at0, block);
    const T* const z0 = logits + row0 * a.ld;
    T* const d0 = dlogits + row0 * a.ldd;
    const int64_t rows_left = a.m.rows - row0;
    Piece q[U];
    float v[U][kPiece];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        q[u] = piece_of<U>(a.m, at0, u);
        if (q[u].row < rows_left && q[u].col + kPiece <= a.m.cols) load_piece(z0 + (uint64_t)q[u].row * (uint32_t)a.ld + q[u].col, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (q[u].row >= rows_left) return;
        const LogitGrad row = logit_grad(a.facts, row0 + q[u].row, a.m.cols);
        if (row.far) continue;         // far_rows has it
        const int64_t hot = row.target - q[u].col;
        auto grad = [&](float z, int e) { return row.template of<false>(z, e == hot); };
        T* pd = d0 + (uint64_t)q[u].row * (uint32_t)a.ldd + q[u].col;
        if (q[u].col + kPiece <= a.m.cols) {
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[u][e] = grad(v[u][e], e);
            store_piece(pd, v[u]);
        } else {
            const T* pz = z0 + (uint64_t)q[u].row * (uint32_t)a.ld + q[u].col;
            const int n = (int)(a.m.cols - q[u].col);
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                if (e < n) pd[e] = Elem<T>::from_f32(grad(Elem<T>::to_f32(pz[e]), e));
        }
    }
}

constexpr int64_t kSmallGradItems = 1 << 18;     // (as in k_dropout.hip)
constexpr int64_t kWaveClasses = 1024;           // rows up to this length are a wave's
constexpr int64_t kPartClasses = 4096, kMaxParts = 64, kWantBlocks = 1024;
constexpr int64_t kMostFarBlocks = 1024;         // four to a CU

}  // namespace

// Rows are cut where there are too few to fill the chip: into parts of 4,096 classes at least, towards 1,024 blocks.
LogProbsPlan plan_log_probs(int64_t rows, int64_t classes, int k) {
    LogProbsPlan p;
    p.parts = 1;
    p.part = classes;
    if (classes > kWaveClasses && rows > 0) {
        const int64_t most = std::min<int64_t>(kMaxParts, (classes + kPartClasses - 1) / kPartClasses);
        const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(most, kWantBlocks / rows));
        p.part = ((classes + parts - 1) / parts + 7) / 8 * 8;
        p.parts = (int)((classes + p.part - 1) / p.part);
    }
    p.sums_bytes = p.parts > 1 ? (size_t)rows * p.parts * 16 : 0;
    p.bytes = p.sums_bytes + (p.parts > 1 ? (size_t)rows * p.parts * k * sizeof(TopKey) : 0);
    return p;
}

void launch_log_probs(int dtype, const void* logits, int64_t ld, int64_t rows, int64_t classes, const int32_t* targets, int k,
                      const LogProbsOut& out, void* work, hipStream_t st) {
    if (rows <= 0) return;
    const LogProbsPlan p = plan_log_probs(rows, classes, k);
    RowArgs a = {};
    a.ld = ld;
    a.rows = rows;
    a.classes = (uint32_t)classes;
    a.part = (uint32_t)p.part;
    a.parts = p.parts;
    a.k = k;
    a.targets = targets;
    a.log_prob = out.log_prob; a.entropy = out.entropy; a.lse = out.lse; a.top_value = out.top_value; a.top_class = out.top_class;
    a.sums = (float*)work;
    a.keys = (TopKey*)((char*)work + p.sums_bytes);
    const double esz = dtype == 1 ? 2.0 : 4.0;
    {
        ProfScope ps("log_probs", 0.0, esz * (double)rows * (double)classes, st);
        const bool by_wave = classes <= kWaveClasses;
        const unsigned grid = by_wave ? (unsigned)((rows + 3) / 4) : (unsigned)(rows * p.parts);
#define EDL_LOG_PROBS(TT, WW, KK) hipLaunchKernelGGL((log_probs_kernel<TT, WW, KK>), dim3(grid), dim3(256), 0, st, (const TT*)logits, a)
        if (dtype == 1) {
            if (by_wave) { if (k > 0) EDL_LOG_PROBS(bf16_t, 1, true); else EDL_LOG_PROBS(bf16_t, 1, false); }
            else { if (k > 0) EDL_LOG_PROBS(bf16_t, 4, true); else EDL_LOG_PROBS(bf16_t, 4, false); }
        } else {
            if (by_wave) { if (k > 0) EDL_LOG_PROBS(float, 1, true); else EDL_LOG_PROBS(float, 1, false); }
            else { if (k > 0) EDL_LOG_PROBS(float, 4, true); else EDL_LOG_PROBS(float, 4, false); }
        }
#undef EDL_LOG_PROBS
    }
    if (p.parts == 1) return;
    ProfScope ps("log_probs_join", 0.0, (double)p.bytes, st);
    const dim3 grid((unsigned)((rows + 3) / 4));
#define EDL_LOG_PROBS_JOIN(TT, KK) hipLaunchKernelGGL((log_probs_join_kernel<TT, KK>), grid, dim3(256), 0, st, (const TT*)logits, a)
    if (dtype == 1) { if (k > 0) EDL_LOG_PROBS_JOIN(bf16_t, true); else EDL_LOG_PROBS_JOIN(bf16_t, false); }
    else { if (k > 0) EDL_LOG_PROBS_JOIN(float, true); else EDL_LOG_PROBS_JOIN(float, false); }
#undef EDL_LOG_PROBS_JOIN
}

void launch_log_probs_grad(int dtype, const void* logits, int64_t ld, int64_t rows, int64_t classes, const int32_t* targets, const float* lse,
                           const float* entropy, const float* dlog_prob, const float* dentropy, void* dlogits, int64_t ldd, hipStream_t st) {
    if (rows <= 0) return;
    GradArgs a = {};
    a.m = Pieces{rows, classes, (classes + kPiece - 1) / kPiece};
    a.ld = ld;
    a.ldd = ldd;
    a.facts = RowFacts{targets, lse, entropy, dlog_prob, dentropy};
    const double esz = dtype == 1 ? 2.0 : 4.0;
    const int64_t items = rows * a.m.per_row;
    const bool small = items < kSmallGradItems;
    a.far_by_wave = classes <= kWaveClasses;
    a.far_blocks = (unsigned)std::min(kMostFarBlocks, a.far_by_wave ? (rows + 3) / 4 : rows);
    const unsigned grid = (unsigned)((items + (small ? 255 : 1023)) / (small ? 256 : 1024)) + (small ? a.far_blocks : 0);
    {
        ProfScope ps("log_probs_grad", 0.0, 2.0 * esz * (double)rows * (double)classes, st);
#define EDL_LOG_PROBS_GRAD(TT, UU) hipLaunchKernelGGL((log_probs_grad_kernel<TT, UU>), dim3(grid), dim3(256), 0, st, (const TT*)logits, (TT*)dlogits, a)
        if (dtype == 1) { if (small) EDL_LOG_PROBS_GRAD(bf16_t, 1); else EDL_LOG_PROBS_GRAD(bf16_t, 4); }
        else { if (small) EDL_LOG_PROBS_GRAD(float, 1); else EDL_LOG_PROBS_GRAD(float, 4); }
#undef EDL_LOG_PROBS_GRAD
    }
    if (small) return;
    ProfScope ps("log_probs_far_rows", 0.0, 0.0, st);
    if (dtype == 1) hipLaunchKernelGGL((far_rows_kernel<bf16_t>), dim3(a.far_blocks), dim3(256), 0, st, (const bf16_t*)logits, (bf16_t*)dlogits, a);
    else hipLaunchKernelGGL((far_rows_kernel<float>), dim3(a.far_blocks), dim3(256), 0, st, (const float*)logits, (float*)dlogits, a);
}

}  // namespace edl
