// Element types of the sequences (DEEPPCR_F32 / _BF16 / _F16): vectors of V
// elements, widened to float32 on reading and rounded to nearest even on
// writing (the compiler's conversions, one instruction on gfx950).
#pragma once

#include <hip/hip_runtime.h>

namespace deeppcr {
namespace {

template <int DT>
struct ElemType;
template <>
struct ElemType<0> {
    typedef float T;
};
template <>
struct ElemType<1> {
    typedef __bf16 T;
};
template <>
struct ElemType<2> {
    typedef _Float16 T;
};
template <int DT>
using elem_t = typename ElemType<DT>::T;

// V consecutive elements, in memory and in registers (V a power of two).
template <int DT, int V>
struct alignas(sizeof(elem_t<DT>) * V) Pack {
    elem_t<DT> e[V];
};

template <int DT, int V>
__device__ __forceinline__ Pack<DT, V> pack_load(const void* base, long long i) {
    return *reinterpret_cast<const Pack<DT, V>*>(reinterpret_cast<const elem_t<DT>*>(base) + i);
}
template <int DT, int V>
__device__ __forceinline__ void pack_store(void* base, long long i, const float (&f)[V]) {
    Pack<DT, V> p;
#pragma unroll
    for (int v = 0; v < V; ++v) p.e[v] = (elem_t<DT>)f[v];
    *reinterpret_cast<Pack<DT, V>*>(reinterpret_cast<elem_t<DT>*>(base) + i) = p;
}

// s = sigmoid(a) and c = 1 - s, each to full relative precision: with
// t = exp(-|a|) in (0, 1] neither overflows nor cancels.  NaN gives NaN.
__device__ __forceinline__ void sigmoid_pair(float a, float* s, float* c) {
    const float t = __expf(-fabsf(a));
    const float big = __builtin_amdgcn_rcpf(1.f + t), small = t * big;
    *s = a >= 0.f ? big : small;
    *c = a >= 0.f ? small : big;
}

}  // namespace
}  // namespace deeppcr
