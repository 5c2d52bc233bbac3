// The running sums of a softmax over one row, and the best classes so far, as the kernels of the log-probability operators
// keep them per lane, wave and part of a row.  With m the largest logit and d = (z - m) log2(e):
//   s = sum 2^d,  t = sum 2^d d:   lse = m + log2 s ln 2,  entropy = (log2 s - t / s) ln 2
// all in float32 (s and t are sums of terms relative to the largest, so none is lost to the row's size).  The difference
// comes before the factor: logits as large as the type has (the lowest value as a mask, in a row of nothing else) then stay finite.
// A class at -inf is masked: it adds nothing.  A NaN or +inf makes s NaN and with it everything of the row.
#pragma once
#include "dev_common.h"

namespace edl {

struct SoftmaxSums {
    float m = -INFINITY, s = 0.f, t = 0.f;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Exponents below this are as good as it: 2 to them is 0, and times 0 it stays finite (an infinite one would not).
constexpr float kFarBelow = -300.f;
__device__ __forceinline__ float exp2_of(float d) { return __builtin_amdgcn_exp2f(d); }
// what logits are taken relative to: a maximum of -inf (all classes so far are masked) leaves them at -inf
__device__ __forceinline__ float softmax_base(const SoftmaxSums& a) { return a.m == -INFINITY ? 0.f : a.m; }

// moves the sums to another (larger) maximum
__device__ __forceinline__ void softmax_rebase(SoftmaxSums& a, float m) {
    if (a.m == m) return;
    const float d = fmaxf((a.m - m) * kLog2e, kFarBelow), f = exp2_of(d);
    a.t = f * (a.t + a.s * d);
    a.s = f * a.s;
    a.m = m;
}
// z: at most a.m, or not a number; base: softmax_base(a)
__device__ __forceinline__ void softmax_add(SoftmaxSums& a, float z, float base) {
    const float d = (z - base) * kLog2e, e = exp2_of(d);
    a.s += e;
    a.t = __builtin_fmaf(e, fmaxf(d, kFarBelow), a.t);
}
__device__ __forceinline__ void softmax_join(SoftmaxSums& a, SoftmaxSums b) {
    const float m = fmaxf(a.m, b.m);
    softmax_rebase(a, m);
    softmax_rebase(b, m);
    a.s += b.s;
    a.t += b.t;
}
__device__ __forceinline__ SoftmaxSums softmax_shuffle(const SoftmaxSums& a, int mask) {
    SoftmaxSums b;
    b.m = __shfl_xor(a.m, mask, 64);
    b.s = __shfl_xor(a.s, mask, 64);
    b.t = __shfl_xor(a.t, mask, 64);
    return b;
}
__device__ __forceinline__ void softmax_join_wave(SoftmaxSums& a) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) softmax_join(a, softmax_shuffle(a, o));
}
// (s == 0: every class is masked; the row has no distribution)
__device__ __forceinline__ float softmax_lse(const SoftmaxSums& a) { return a.s == 0.f ? -INFINITY : a.m + log2f(a.s) * kLn2; }
__device__ __forceinline__ float softmax_entropy(const SoftmaxSums& a) { return a.s == 0.f ? 0.f : (log2f(a.s) - a.t / a.s) * kLn2; }
// log probability of a class from its logit: an impossible class of a row without a distribution is as impossible.  (From
// the largest logit, not from lse: exact to a step of its own size, not of the logit's.)
__device__ __forceinline__ float softmax_log_prob(const SoftmaxSums& a, float z) { return a.s == 0.f ? -INFINITY : (z - a.m) - log2f(a.s) * kLn2; }

// ---- the gradient of a logit ---------------------------------------------------------------------------------------------
// What a row's logits need: dz = g (1[c = t] - p) - h p (log p + H), with log p = (z - base) - low.
// Forward leaves lse, one float32: base, with low = 0.  p is then off by up to half a step of lse (2^-24 of it at most), and
// where log s is below lse's last place, p is off by the factor s: rows of the lowest value alone have lse = m, and so p = 1.
// Rows whose lse is at least kFarLse away from 0 take base = m and low = log s instead, summed up again from their logits; below it
// the half step is 2^-18 at most.
constexpr float kFarLse = 128.f;
struct RowFacts {              // of each row; null: none (targets), zeros (gradients)
    const int32_t* targets;
    const float *lse, *entropy, *dlog_prob, *dentropy;
};
struct LogitGrad {
    float g, h, base, low, both;
    int64_t target;            // -1: none
    bool none;                 // zeros, whatever the logits are
    bool far;                  // base and low are yet to be had from the logits

    // FAR: rows may be far, or low is known to be 0 (an operation less for each logit)
    template <bool FAR> __device__ __forceinline__ float of(float z, bool hot) const {
        const float lp = FAR ? (z - base) - low : z - base, p = exp2_of(lp * kLog2e);
        const float d = z == -INFINITY ? 0.f : p * (both - h * fmaxf(lp, kFarBelow));
        return none ? 0.f : hot ? d + g : d;
    }
};
// (infinite or not a number: nothing is gained)
__device__ __forceinline__ bool is_far(float lse) { return fabsf(lse) >= kFarLse && fabsf(lse) < INFINITY; }
__device__ __forceinline__ LogitGrad logit_grad(const RowFacts& f, int64_t row, int64_t classes) {
    LogitGrad r;
    const int32_t t = f.targets != nullptr ? f.targets[row] : -1;
    const bool has = t >= 0 && t < classes;
    r.target = has ? t : -1;
    r.g = has && f.dlog_prob != nullptr ? f.dlog_prob[row] : 0.f;
    r.h = f.dentropy != nullptr ? f.dentropy[row] : 0.f;
    r.base = f.lse[row];
    r.low = 0.f;
    r.both = -(r.g + (r.h != 0.f ? r.h * f.entropy[row] : 0.f));
    r.none = r.g == 0.f && r.h == 0.f;
    r.far = !r.none && is_far(r.base);
    return r;
}
// whether the row is far, by one load where it is not
__device__ __forceinline__ bool row_is_far(const RowFacts& f, int64_t row, int64_t classes) { return is_far(f.lse[row]) && logit_grad(f, row, classes).far; }
// what a row that is far takes, from the sums over all of its logits
__device__ __forceinline__ float2 far_base(const SoftmaxSums& a) { return make_float2(a.m, log2f(a.s) * kLn2); }

// ---- the k largest of a row, one per lane of a wave, best first -------------------------------------------------------
// Ordered by value, then by the lower class: both in one 64-bit key, so that the result does not depend on the order in
// which classes come.  -0 and +0 are equal; a NaN ranks as -inf.  Key 0 is no class.
struct TopKey { uint32_t hi, lo; };
__device__ __forceinline__ bool key_above(const TopKey& a, const TopKey& b) { return a.hi > b.hi || (a.hi == b.hi && a.lo > b.lo); }
__device__ __forceinline__ TopKey top_key(float z, uint32_t cls) {
    z = z == z ? z + 0.f : -INFINITY;
    const uint32_t b = __float_as_uint(z);
    return TopKey{b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u), ~cls};
}
__device__ __forceinline__ float top_value(const TopKey& k) { return __uint_as_float(k.hi ^ ((k.hi >> 31) ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ TopKey key_of_lane(const TopKey& k, int lane) {
    return TopKey{(uint32_t)__builtin_amdgcn_readlane((int)k.hi, lane), (uint32_t)__builtin_amdgcn_readlane((int)k.lo, lane)};
}

struct TopList {
    TopKey mine;        // this lane's entry
    TopKey last;        // what a newcomer has to beat, the same for all lanes: entry k - 1, or more where k better ones are known to come

    __device__ __forceinline__ void clear() { mine = last = TopKey{0, 0}; }
    // as a value: what is below it need not be offered
    __device__ __forceinline__ float bar() const { return top_value(last); }       // (key 0, no class, is a NaN: nothing is below it)
    __device__ __forceinline__ void raise(const TopKey& to) { if (key_above(to, last)) last = to; }

    // A lane's best value so far (its key's high half; 0: none): of 64 lanes' bests, k are at least the k-th, so the best k of
    // all are.  Found bit by bit, to 16 bits: a bound below it does as well.
    __device__ __forceinline__ void expect(uint32_t best, int k) {
        uint32_t at = 0;
        for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
            if (__popcll(__ballot(best >= (at | bit))) >= k) at |= bit;
        raise(TopKey{at, 0});
    }

    // Takes in the candidates (one per lane; key 0: none) that belong to the best k.  All lanes of the wave take part.
    // scratch: 64 keys of LDS for this wave alone.  A few candidates are entered one by one, each step waiting for the one
    // before; of more, every lane counts how many of them are above its candidate and above its entry, which are independent
    // steps, and both go straight to their new places.
    __device__ __forceinline__ void offer(const TopKey& c, int k, TopKey* scratch) {
        const int lane = threadIdx.x & 63;
        uint64_t left = __ballot(key_above(c, last));
        if (left == 0) return;
        if (__popcll(left) <= kOneByOne) {
            do {
                const TopKey n = key_of_lane(c, __builtin_ctzll(left));
                const int at = __popcll(__ballot(key_above(mine, n)));
                // entries from `at` on move up one lane (the hardware's shift by one lane across the wave)
                const uint32_t up_hi = (uint32_t)__builtin_amdgcn_update_dpp((int)mine.hi, (int)mine.hi, 0x138, 0xf, 0xf, false);
                const uint32_t up_lo = (uint32_t)__builtin_amdgcn_update_dpp((int)mine.lo, (int)mine.lo, 0x138, 0xf, 0xf, false);
                if (lane == at) mine = n;
                else if (lane > at) mine = TopKey{up_hi, up_lo};
                left &= left - 1;
            } while (left != 0);
        } else {
            int to = 0, entry_to = lane;       // places of this lane's candidate and of its entry
            for (uint64_t l = left; l != 0; l &= l - 1) {
                const int j = __builtin_ctzll(l);
                const TopKey n = key_of_lane(c, j);
                const int before = __popcll(__ballot(key_above(mine, n)));
                to += (key_above(n, c) ? 1 : 0) + (lane == j ? before : 0);
                entry_to += key_above(n, mine) ? 1 : 0;
            }
            // (the 64 first places are each taken once: what moves past them is dropped)
            if (entry_to < 64) scratch[entry_to] = mine;
            if (((left >> lane) & 1) != 0 && to < 64) scratch[to] = c;
            wave_lds_handover();
            mine = scratch[lane];
            wave_lds_handover();
        }
        raise(key_of_lane(mine, k - 1));
    }
    static constexpr int kOneByOne = 2;
};

}  // namespace edl
