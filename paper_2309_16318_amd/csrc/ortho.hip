// Orthogonalised update: X = G / (|G| + eps), then per step A = X X^T,
// B = cb A + cc A A, X = ca X + B X on every matrix of a stack.  A matrix with
// more rows than columns is worked on as its transpose.
#include <algorithm>

#include "elem.h"
#include "internal.h"

namespace deeppcr {
namespace {

constexpr int TS = 32;  // tile side

// One workgroup per matrix: X [k, r] from G [m, n] (transposed where m > n),
// scaled to unit Frobenius norm by way of its largest element, so that no
// square leaves the float32 range.
template <int DT>
__global__ void __launch_bounds__(256) ortho_scale(const void* G, float* X, int m, int n,
                                                   float eps) {
    __shared__ float sm[256];
    const long long sz = (long long)m * n, base = blockIdx.x * sz;
    float top = 0.f;
    for (long long i = threadIdx.x; i < sz; i += 256)
        top = fmaxf(top, fabsf((float)pack_load<DT, 1>(G, base + i).e[0]));
    sm[threadIdx.x] = top;
    __syncthreads();
    for (int s = 128; s > 0; s /= 2) {
        if (threadIdx.x < s) sm[threadIdx.x] = fmaxf(sm[threadIdx.x], sm[threadIdx.x + s]);
        __syncthreads();
    }
    top = sm[0];
    __syncthreads();
    float sum = 0.f;
    for (long long i = threadIdx.x; i < sz; i += 256) {
        const float g = (float)pack_load<DT, 1>(G, base + i).e[0];
        const float v = g == 0.f ? 0.f : g / top;
        sum = fmaf(v, v, sum);
    }
    sm[threadIdx.x] = sum;
    __syncthreads();
    for (int s = 128; s > 0; s /= 2) {
        if (threadIdx.x < s) sm[threadIdx.x] += sm[threadIdx.x + s];
        __syncthreads();
    }
    const float den = sqrtf(sm[0]) + eps / top;
    for (long long i = threadIdx.x; i < sz; i += 256) {
        const float g = (float)pack_load<DT, 1>(G, base + i).e[0];
        const float v = g == 0.f && top == 0.f ? 0.f : g / top / den;
        X[base + (m > n ? (i % n) * m + i / n : i)] = v;
    }
}

template <int DT>
__global__ void __launch_bounds__(256) ortho_store(const float* X, void* out, int m, int n) {
    const long long sz = (long long)m * n, base = blockIdx.x * sz;
    for (long long i = threadIdx.x; i < sz; i += 256) {
        const float v[1] = {X[base + (m > n ? (i % n) * m + i / n : i)]};
        pack_store<DT, 1>(out, base + i, v);
    }
}

// C [k, c] = alpha D + beta P Q (P [k, q]; Q [q, c], or stored [c, q]) for
// matrix blockIdx.z.
template <bool QT>
__global__ void __launch_bounds__(256) ortho_product(const float* P, const float* Q, const float* D,
                                                     float* C, int k, int q, int c, float alpha,
                                                     float beta) {
    __shared__ float p[TS][TS + 1], s[TS][TS + 1];
    const long long z = blockIdx.z;
    P += z * k * q;
    Q += z * q * c;
    C += z * k * c;
    if (D) D += z * k * c;
    const int i0 = blockIdx.y * TS, j0 = blockIdx.x * TS;
    const int tx = threadIdx.x % TS, ty = threadIdx.x / TS;
    float acc[4] = {};
    for (int t0 = 0; t0 < q; t0 += TS) {
        __syncthreads();
        for (int y = ty; y < TS; y += 8) {
            p[y][tx] = i0 + y < k && t0 + tx < q ? P[(long long)(i0 + y) * q + t0 + tx] : 0.f;
            if (QT)
                s[tx][y] = j0 + y < c && t0 + tx < q ? Q[(long long)(j0 + y) * q + t0 + tx] : 0.f;
            else
                s[y][tx] = t0 + y < q && j0 + tx < c ? Q[(long long)(t0 + y) * c + j0 + tx] : 0.f;
        }
        __syncthreads();
        for (int t = 0; t < TS; ++t)
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[u] = fmaf(p[ty + 8 * u][t], s[t][tx], acc[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int i = i0 + ty + 8 * u, j = j0 + tx;
        if (i < k && j < c) {
            const long long at = (long long)i * c + j;
            C[at] = (D ? alpha * D[at] : 0.f) + beta * acc[u];
        }
    }
}

template <bool QT>
hipError_t product(const float* P, const float* Q, const float* D, float* C, int N, int k, int q,
                   int c, float alpha, float beta, hipStream_t st) {
    const dim3 grid((c + TS - 1) / TS, (k + TS - 1) / TS, N);
    ortho_product<QT><<<grid, 256, 0, st>>>(P, Q, D, C, k, q, c, alpha, beta);
    return hipGetLastError();
}

constexpr int kSome = 16384;  // matrices per launch (a grid's third axis ends at 65535)

template <int DT>
hipError_t run(const void* G, void* X, int N, int m, int n, int steps, float ca, float cb, float cc,
               float eps, float* ws, hipStream_t st) {
    const int k = std::min(m, n), r = std::max(m, n);
    const long long sz = (long long)k * r, sq = (long long)k * k;
    for (int at = 0; at < N; at += kSome) {
        const int some = std::min(kSome, N - at);
        float *x = ws, *y = x + some * sz, *A = y + some * sz, *B = A + some * sq;
        const size_t es = sizeof(elem_t<DT>);
        ortho_scale<DT><<<some, 256, 0, st>>>((const char*)G + at * sz * es, x, m, n, eps);
        hipError_t e = hipGetLastError();
        for (int s = 0; s < steps && e == hipSuccess; ++s) {
            e = product<true>(x, x, nullptr, A, some, k, r, k, 0.f, 1.f, st);
            if (e == hipSuccess) e = product<true>(A, A, A, B, some, k, k, k, cb, cc, st);
            if (e == hipSuccess) e = product<false>(B, x, x, y, some, k, k, r, ca, 1.f, st);
            std::swap(x, y);
        }
        if (e != hipSuccess) return e;
        ortho_store<DT><<<some, 256, 0, st>>>(x, (char*)X + at * sz * es, m, n);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t ortho_workspace(int N, int m, int n) {
    const size_t k = std::min(m, n), r = std::max(m, n), some = std::min(N, kSome);
    return some * (2 * k * r + 2 * k * k) * sizeof(float);
}

hipError_t launch_ortho(const void* G, void* X, int N, int m, int n, int steps, float ca, float cb,
                        float cc, float eps, int dtype, void* ws, hipStream_t st) {
    if (dtype == 0) return run<0>(G, X, N, m, n, steps, ca, cb, cc, eps, (float*)ws, st);
    if (dtype == 1) return run<1>(G, X, N, m, n, steps, ca, cb, cc, eps, (float*)ws, st);
    return run<2>(G, X, N, m, n, steps, ca, cb, cc, eps, (float*)ws, st);
}

}  // namespace deeppcr
