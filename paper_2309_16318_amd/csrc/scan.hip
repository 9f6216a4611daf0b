// Gated linear recurrence: x_l = s_l x_{l-1} + r_l channel by channel, its
// backward pass and the single row.
#include <type_traits>

#include "elem.h"
#include "internal.h"

namespace deeppcr {
namespace {

// The multiplier s, the added part r, and c = 1 - s of one element.
template <int GATE>
__device__ __forceinline__ void gate_of(float a, float* s, float* c) {
    if constexpr (GATE == 1) {
        sigmoid_pair(a, s, c);
    } else {
        *s = a;
        *c = 1.f;
    }
}

template <int DT, int GATE>
__global__ void __launch_bounds__(64) scan_walk(ScanArgs k) {
    const long long f = (long long)blockIdx.x * 64 + threadIdx.x;
    if (f >= (long long)k.B * k.w) return;
    const int b = (int)(f / k.w), c = (int)(f % k.w);
    const int n = k.lengths ? min(max(k.lengths[b], 0), k.L) : k.L;
    const long long r0 = (long long)b * k.L;
    float x = k.x0 ? k.x0[f] : 0.f;
    float out[1];
    for (int l = 0; l < n; ++l) {
        float s, q;
        gate_of<GATE>((float)pack_load<DT, 1>(k.a, (r0 + l) * k.lda + c).e[0], &s, &q);
        x = fmaf(s, x, q * (float)pack_load<DT, 1>(k.u, (r0 + l) * k.ldu + c).e[0]);
        out[0] = x;
        pack_store<DT, 1>(k.out0, (r0 + l) * k.w + c, out);
    }
    out[0] = 0.f;
    for (int l = n; l < k.L; ++l) pack_store<DT, 1>(k.out0, (r0 + l) * k.w + c, out);
    if (k.last) k.last[f] = x;
}

template <int DT, int GATE>
__global__ void __launch_bounds__(64) scan_walk_bwd(ScanArgs k) {
    const long long f = (long long)blockIdx.x * 64 + threadIdx.x;
    if (f >= (long long)k.B * k.w) return;
    const int b = (int)(f / k.w), c = (int)(f % k.w);
    const int n = k.lengths ? min(max(k.lengths[b], 0), k.L) : k.L;
    const long long r0 = (long long)b * k.L;
    float out[1] = {0.f};
    for (int l = n; l < k.L; ++l) {
        pack_store<DT, 1>(k.out0, (r0 + l) * k.w + c, out);
        pack_store<DT, 1>(k.out1, (r0 + l) * k.w + c, out);
    }
    float kap = k.g_last ? k.g_last[f] : 0.f;  // s_{l+1} lam_{l+1}
    for (int l = n - 1; l >= 0; --l) {
        float s, q;
        gate_of<GATE>((float)pack_load<DT, 1>(k.a, (r0 + l) * k.lda + c).e[0], &s, &q);
        const float lam = kap + (float)pack_load<DT, 1>(k.g, (r0 + l) * k.ldg + c).e[0];
        float xp = l > 0 ? (float)pack_load<DT, 1>(k.x, (r0 + l - 1) * k.w + c).e[0]
                         : (k.x0 ? k.x0[f] : 0.f);
        if (GATE == 1) xp = (xp - (float)pack_load<DT, 1>(k.u, (r0 + l) * k.ldu + c).e[0]) * s * q;
        out[0] = lam * xp;
        pack_store<DT, 1>(k.out0, (r0 + l) * k.w + c, out);
        out[0] = lam * q;
        pack_store<DT, 1>(k.out1, (r0 + l) * k.w + c, out);
        kap = s * lam;
    }
    if (k.last) k.last[f] = kap;
}

template <int DT, int GATE>
__global__ void __launch_bounds__(256) scan_step(const void* a, long long lda, const void* u,
                                                 long long ldu, const float* state,
                                                 float* state_out, void* x, int B, int w) {
    const long long f = (long long)blockIdx.x * 256 + threadIdx.x;
    if (f >= (long long)B * w) return;
    const long long b = f / w, c = f % w;
    float s, q;
    gate_of<GATE>((float)pack_load<DT, 1>(a, b * lda + c).e[0], &s, &q);
    float out[1] = {fmaf(s, state[f], q * (float)pack_load<DT, 1>(u, b * ldu + c).e[0])};
    state_out[f] = out[0];
    if (x) pack_store<DT, 1>(x, f, out);
}

template <int N>
using Int = std::integral_constant<int, N>;

// f(DT, GATE) with the runtime values as types.
template <class F>
hipError_t by_type(int dtype, int gate, F&& f) {
    switch (dtype * 2 + gate) {
        case 0: return f(Int<0>{}, Int<0>{});
        case 1: return f(Int<0>{}, Int<1>{});
        case 2: return f(Int<1>{}, Int<0>{});
        case 3: return f(Int<1>{}, Int<1>{});
        case 4: return f(Int<2>{}, Int<0>{});
        default: return f(Int<2>{}, Int<1>{});
    }
}

}  // namespace

size_t scan_workspace(int B, int L, int w) { return 256; }

hipError_t launch_scan(bool bwd, const ScanArgs& k, int gate, int dtype, hipStream_t st) {
    const unsigned grid = (unsigned)(((long long)k.B * k.w + 63) / 64);
    return by_type(dtype, gate, [&](auto dt, auto gt) {
        constexpr int DT = decltype(dt)::value, GATE = decltype(gt)::value;
        if (bwd)
            scan_walk_bwd<DT, GATE><<<grid, 64, 0, st>>>(k);
        else
            scan_walk<DT, GATE><<<grid, 64, 0, st>>>(k);
        return hipGetLastError();
    });
}

hipError_t launch_scan_step(const void* a, long long lda, const void* u, long long ldu,
                            const float* state, float* state_out, void* x, int B, int w, int gate,
                            int dtype, hipStream_t st) {
    const unsigned grid = (unsigned)(((long long)B * w + 255) / 256);
    return by_type(dtype, gate, [&](auto dt, auto gt) {
        constexpr int DT = decltype(dt)::value, GATE = decltype(gt)::value;
        scan_step<DT, GATE><<<grid, 256, 0, st>>>(a, lda, u, ldu, state, state_out, x, B, w);
        return hipGetLastError();
    });
}

}  // namespace deeppcr
