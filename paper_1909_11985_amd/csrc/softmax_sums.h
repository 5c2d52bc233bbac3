// The running sums of a softmax over one row, and the best classes so far, as the kernels of the log-probability operators
// keep them per lane, wave and part of a row.
//   m = max z,  s = sum e^(z-m),  t = sum e^(z-m) (z-m):   lse = m + log s,  entropy = log s - t / s
// all in float32 (s and t are sums of terms relative to the largest, so none is lost to the row's size).  A class at -inf
// is masked: it adds nothing.  A NaN or +inf makes s NaN and with it everything of the row.
#pragma once
#include "dev_common.h"

namespace edl {

struct SoftmaxSums {
    float m = -INFINITY, s = 0.f, t = 0.f;
};

constexpr float kLog2e = 1.4426950408889634f;
// e^x for x <= 0 by the hardware's base-2 exponential: the argument's rounding is relative to x, where the result is small
__device__ __forceinline__ float exp_below(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Differences below this are as good as it: their exponential is 0, and times 0 it stays finite (an infinite one would not).
constexpr float kFarBelow = -200.f;

// moves the sums to another (larger) maximum
__device__ __forceinline__ void softmax_rebase(SoftmaxSums& a, float m) {
    if (a.m == m) return;
    const float d = fmaxf(a.m - m, kFarBelow), f = exp_below(d);
    a.t = f * (a.t + a.s * d);
    a.s = f * a.s;
    a.m = m;
}
// what differences are taken from: a maximum of -inf (all classes so far are masked) leaves them at -inf
__device__ __forceinline__ float softmax_base(const SoftmaxSums& a) { return a.m == -INFINITY ? 0.f : a.m; }
// z: at most a.m, or not a number
__device__ __forceinline__ void softmax_add(SoftmaxSums& a, float z, float base) {
    const float d = z - base, e = exp_below(d);
    a.s += e;
    a.t += e * fmaxf(d, kFarBelow);
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
__device__ __forceinline__ float softmax_lse(const SoftmaxSums& a) { return a.s == 0.f ? -INFINITY : a.m + logf(a.s); }
__device__ __forceinline__ float softmax_entropy(const SoftmaxSums& a) { return a.s == 0.f ? 0.f : logf(a.s) - a.t / a.s; }
// log probability of a class from its logit: an impossible class of a row without a distribution is as impossible
__device__ __forceinline__ float log_prob_of(float z, float lse) { return lse == -INFINITY ? -INFINITY : z - lse; }

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
    TopKey last;        // entry k - 1, the same for all lanes: what a newcomer has to beat
    float bar;          // its value; -inf while there are fewer than k

    __device__ __forceinline__ void clear() { mine = last = TopKey{0, 0}; bar = -INFINITY; }

    // Takes in the candidates (one per lane; key 0: none) that belong to the best k.  All lanes of the wave take part.
    __device__ __forceinline__ void offer(const TopKey& c, int k) {
        const int lane = threadIdx.x & 63;
        uint64_t left = __ballot(key_above(c, last));
        if (left == 0) return;
        do {
            const int from = __builtin_ctzll(left);
            const TopKey n = key_of_lane(c, from);
            const int at = __popcll(__ballot(key_above(mine, n)));
            // entries from `at` on move up one lane (the hardware's shift by one lane across the wave)
            const uint32_t up_hi = (uint32_t)__builtin_amdgcn_update_dpp((int)mine.hi, (int)mine.hi, 0x138, 0xf, 0xf, false);
            const uint32_t up_lo = (uint32_t)__builtin_amdgcn_update_dpp((int)mine.lo, (int)mine.lo, 0x138, 0xf, 0xf, false);
            if (lane == at) mine = n;
            else if (lane > at) mine = TopKey{up_hi, up_lo};
            last = key_of_lane(mine, k - 1);
            left &= left - 1;
            left &= __ballot(key_above(c, last));
        } while (left != 0);
        bar = last.hi == 0 ? -INFINITY : top_value(last);
    }
};

}  // namespace edl
