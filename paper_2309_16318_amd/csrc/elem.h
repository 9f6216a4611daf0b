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

// V consecutive elements as they lie in memory, in whole registers (two 16-bit
// elements each): what a thread holds many of until it uses them.
template <int DT, int V>
struct Raw {
    static constexpr int BYTES = (int)sizeof(elem_t<DT>) * V;
    static constexpr int N = BYTES < 4 ? 1 : BYTES / 4;
    unsigned word[N];
    __device__ __forceinline__ void load(const void* base, long long i) {
        const char* p = (const char*)base + i * (long long)sizeof(elem_t<DT>);
        if constexpr (BYTES == 2) {
            word[0] = *reinterpret_cast<const unsigned short*>(p);
        } else {
            struct alignas(BYTES) Words {
                unsigned w[N];
            };
            const Words q = *reinterpret_cast<const Words*>(p);
#pragma unroll
            for (int j = 0; j < N; ++j) word[j] = q.w[j];
        }
    }
    __device__ __forceinline__ float get(int v) const {
        if constexpr (DT == 0) {
            return __uint_as_float(word[v]);
        } else if constexpr (DT == 1) {
            return __uint_as_float(v & 1 ? word[v / 2] & 0xffff0000u : word[v / 2] << 16);
        } else {
            const unsigned short h = (unsigned short)(v & 1 ? word[v / 2] >> 16 : word[v / 2]);
            return (float)__builtin_bit_cast(_Float16, h);
        }
    }
    // From here on the compiler takes the words for new ones: what was
    // computed from them before is not kept in registers for a second use.
    __device__ __forceinline__ void renew() {
#pragma unroll
        for (int j = 0; j < N; ++j) asm volatile("" : "+v"(word[j]));
    }
};

// s = sigmoid(a) and c = 1 - s: with t = exp(-|a|) in (0, 1] neither overflows
// nor cancels.  NaN gives NaN, a t below 2^-126 zero.  The exponential of the
// rounded product with log2(e) is off by |a| 2^-24, which does for results of 16
// bits (SHORT).  For float32 results FINE brings in what the product's rounding left
// out, five instructions more.  A bfloat16 a has 8 bits, so that its product with the
// first 15 of log2(e) is exact and FINE_BF16 has only the others to bring in, three
// instructions (it leaves out half their square, 1.5 2^-24 at |a| = 85).  A gated
// scan of 8192 x 2048 bfloat16 takes 36.6 us with SHORT, 39.4 with FINE_BF16 and
// 40.0 with FINE, forward and backward of 8 x 2048 x 2048 158, 163 and 165.
enum { SHORT, FINE, FINE_BF16 };
template <int HOW>
__device__ __forceinline__ void sigmoid_pair(float a, float* s, float* c) {
    constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0c00000000p-26f, kLn2 = 0x1.62e43p-1f;
    constexpr float kFirst = 0x1.7154p+0f, kOthers = 0x1.480fb6p-18f;  // the second times ln 2
    const float x = -fabsf(a), h = x * (HOW == FINE_BF16 ? kFirst : kLog2e);
    float t = __builtin_amdgcn_exp2f(h);
    // (of an infinite a t is zero, and any number does for what it is multiplied by)
    if constexpr (HOW == FINE) {
        const float r = fmaxf(fmaf(x, kRest, fmaf(x, kLog2e, -h)), -1.f);
        t = fmaf(t * r, kLn2, t);
    } else if constexpr (HOW == FINE_BF16) {
        t = fmaf(t * fmaxf(x, -1000.f), kOthers, t);
    }
    const float big = __builtin_amdgcn_rcpf(1.f + t), small = t * big;
    *s = a >= 0.f ? big : small;
    *c = a >= 0.f ? small : big;
}

}  // namespace
}  // namespace deeppcr
