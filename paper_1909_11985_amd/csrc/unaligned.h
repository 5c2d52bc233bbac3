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

}  // namespace edl
