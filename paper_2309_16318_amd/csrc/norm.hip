// Residual norm: x_out = x + scale act(z) w_post y / rms(y), h = w_pre x_out /
// rms(x_out) row by row, and its backward pass.
//
// Bound by memory: every sequence is read or written once (forward x, y, z,
// x_out, h), so a row stays in the registers of the threads that own it, 8
// columns each, between its reductions.  Rows of up to 512 columns belong to a
// part of a wave (reduced by lane exchanges, several rows per workgroup),
// wider ones to a workgroup.  Threads keep their columns' weights, and in the
// backward pass their columns' sums over the rows, in registers over many rows;
// the sums of all workgroups are added in a fixed order by a second kernel.
#include <type_traits>

#include "elem.h"
#include "internal.h"

namespace deeppcr {
namespace {

constexpr int E = 8;          // columns per thread
constexpr int kSumLanes = 64;  // threads that add up a column of partial sums
constexpr int kSmallWG = 256;  // threads of a workgroup that holds several rows

// The columns of thread t of a row's G threads: E in a row (VEC: w and the
// row strides are multiples of E and the rows aligned), else G apart.
template <int DT, bool VEC>
struct Cols {
    int c0, step, w;
    __device__ Cols(int t, int G, int w_) : c0(VEC ? t * E : t), step(VEC ? 1 : G), w(w_) {}
    __device__ __forceinline__ bool has(int j) const { return c0 + (VEC ? 0 : j * step) < w; }
    // f = row[columns], zero where there are none
    __device__ __forceinline__ void load(const void* row, long long at, float (&f)[E]) const {
        if constexpr (VEC) {
            Pack<DT, E> p{};
            if (c0 < w) p = pack_load<DT, E>(row, at + c0);
#pragma unroll
            for (int j = 0; j < E; ++j) f[j] = (float)p.e[j];
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j)
                f[j] = has(j) ? (float)pack_load<DT, 1>(row, at + c0 + j * step).e[0] : 0.f;
        }
    }
    // the same, as it lies in memory (not VEC: an element per word)
    struct Held {
        Raw<DT, VEC ? E : 1> r[VEC ? 1 : E];
        __device__ __forceinline__ float get(int j) const {
            return VEC ? r[0].get(VEC ? j : 0) : r[VEC ? 0 : j].get(0);
        }
        __device__ __forceinline__ void renew() {
#pragma unroll
            for (auto& q : r) q.renew();
        }
    };
    __device__ __forceinline__ void hold(const void* row, long long at, Held& h) const {
        if constexpr (VEC) {
            if (c0 < w)
                h.r[0].load(row, at + c0);
            else
                h.r[0] = {};
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (has(j))
                    h.r[j].load(row, at + c0 + j * step);
                else
                    h.r[j] = {};
            }
        }
    }
    __device__ __forceinline__ void store(void* row, long long at, const float (&f)[E]) const {
        if constexpr (VEC) {
            if (c0 < w) pack_store<DT, E>(row, at + c0, f);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float one[1] = {f[j]};
                if (has(j)) pack_store<DT, 1>(row, at + c0 + j * step, one);
            }
        }
    }
    // float32 weights; `none` where there is no array
    __device__ __forceinline__ void weights(const float* p, float none, float (&f)[E]) const {
#pragma unroll
        for (int j = 0; j < E; ++j) f[j] = p ? (has(j) ? p[c0 + j * step] : 0.f) : none;
    }
};

// v + v of the lane that the step pairs this one with: inside 16 lanes by lane
// permutations of the add itself (pairs, quads, then the mirrored half and row),
// beyond by exchanging rows and halves of the wave; no LDS round trips.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(
                   __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
// The sum over the G (a power of two) consecutive lanes of a row.
__device__ __forceinline__ float lanes_sum(float v, int G) {
    if (G > 1) v = dpp_add<0xB1>(v);
    if (G > 2) v = dpp_add<0x4E>(v);
    if (G > 4) v = dpp_add<0x141>(v);
    if (G > 8) v = dpp_add<0x140>(v);
    if (G > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v),
                                                        false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (G > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v),
                                                        false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// Sums of N values over the threads of a row, in every one of them.
template <int N, bool BIG>
struct RowSum {
    float (*sm)[16][N];
    int G, turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
        if constexpr (!BIG) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i], G);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i], 64);
            // two buffers in turn: a wave may be one sum ahead of another
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) sm[turn][threadIdx.x >> 6][i] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.f;
            for (int k = 0; k < (int)(blockDim.x >> 6); ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += sm[turn][k][i];
            turn ^= 1;
        }
    }
};

// The gate's value, and its slope where `slope` is given.
template <int DT>
__device__ __forceinline__ void gate_values(int gate, const float (&z)[E], float (&v)[E],
                                            float* slope) {
    if (gate == 0 || gate == 3) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = gate ? z[j] : 1.f;
            if (slope) slope[j] = 1.f;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        float s, c;
        sigmoid_pair<DT == 0 ? FINE : SHORT>(z[j], &s, &c);
        v[j] = gate == 1 ? s : z[j] * s;
        if (slope) slope[j] = gate == 1 ? s * c : s * fmaf(z[j], c, 1.f);
    }
}

// Where a workgroup's threads stand: thread t of the G of its row, row `sub`
// of the `subs` that the workgroup holds at a time.
template <bool BIG>
struct Place {
    int G, t, sub, subs;
    __device__ explicit Place(int G_) : G(G_) {
        t = BIG ? threadIdx.x : threadIdx.x & (G - 1);
        sub = BIG ? 0 : threadIdx.x / G;
        subs = BIG ? 1 : blockDim.x / G;
    }
};

template <int DT, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT ? MAXT : kSmallWG) norm_fwd(NormArgs k, int G) {
    constexpr bool BIG = MAXT != 0;
    __shared__ float sm[2][16][1];
    const Place<BIG> me(G);
    const Cols<DT, VEC> cols(me.t, G, k.w);
    RowSum<1, BIG> sum{sm, G};
    const float inv = 1.f / (float)k.w;
    const long long rows = (long long)k.B * k.L;
    const long long step = (long long)gridDim.x * me.subs;
    constexpr bool AHEAD = VEC && DT != 0;  // as in the backward pass
    struct Row {
        typename Cols<DT, VEC>::Held x, y, z;
    } now{}, next{};
    auto fetch = [&](long long r0, Row& q) {
        const long long r = r0 + me.sub < rows ? r0 + me.sub : rows - 1;
        cols.hold(k.x, r * k.w, q.x);
        if (k.y) cols.hold(k.y, r * k.ldy, q.y);
        if (k.gate) cols.hold(k.z, (k.z_per_seq ? r / k.L : r) * k.ldz, q.z);
    };
    // the first row is asked for before the weights
    const long long first = (long long)blockIdx.x * me.subs;
    if (first < rows) fetch(first, AHEAD ? next : now);
    float kw[E], pre[E];
    cols.weights(k.w_post, 1.f, kw);
    cols.weights(k.scale, 1.f, pre);
#pragma unroll
    for (int j = 0; j < E; ++j) kw[j] *= pre[j];
    cols.weights(k.w_pre, 1.f, pre);
    // the same number of turns for all threads of the workgroup
    for (long long r0 = first; r0 < rows; r0 += step) {
        const bool live = r0 + me.sub < rows;
        const long long r = live ? r0 + me.sub : rows - 1;
        if constexpr (AHEAD) {
            now = next;
            if (r0 + step < rows) fetch(r0 + step, next);
        } else if (r0 != first) {
            fetch(r0, now);
        }
        float x[E];
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = now.x.get(j);
        if (k.y) {
            float y[E], z[E], v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                y[j] = now.y.get(j);
                z[j] = now.z.get(j);
            }
            gate_values<DT>(k.gate, z, v, nullptr);
            float rp = 1.f;
            if (k.w_post) {
                float s[1] = {0.f};
#pragma unroll
                for (int j = 0; j < E; ++j) s[0] = fmaf(y[j], y[j], s[0]);
                sum(s);
                rp = 1.f / sqrtf(fmaf(s[0], inv, k.eps));
                if (k.rstd_post && me.t == 0 && live) k.rstd_post[r] = rp;
            }
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = fmaf(kw[j] * v[j], y[j] * rp, x[j]);
            if (live) cols.store(k.x_out, r * k.w, x);
        }
        if (k.h) {
            float s[1] = {0.f};
#pragma unroll
            for (int j = 0; j < E; ++j) s[0] = fmaf(x[j], x[j], s[0]);
            sum(s);
            const float rq = 1.f / sqrtf(fmaf(s[0], inv, k.eps));
            if (k.rstd_pre && me.t == 0 && live) k.rstd_pre[r] = rq;
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] *= rq * pre[j];
            if (live) cols.store(k.h, r * k.w, x);
        }
    }
}

// Rows of workgroup blockIdx.x: a consecutive part of all rows, or with one
// gate per sequence a consecutive part of a sequence's rows.
//   m = x_out rstd_pre, n = y rstd_post, e = dh w_pre, c = scale w_post act(z) n
//   dx = d = dx_out + rstd_pre (e - m mean(e m))
//   dy = rstd_post (d c / n - n mean(d c)),  dz = d scale w_post n act'(z)
// with sum(d c) = sum((dx_out + rstd_pre e) c) - rstd_pre mean(e m) sum(m c),
// so that one reduction of three values serves both means.
template <int DT, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT ? MAXT : kSmallWG) norm_bwd(NormArgs k, int G, int parts) {
    constexpr bool BIG = MAXT != 0;
    __shared__ float sm[2][16][3];
    __shared__ float tot[BIG ? 1 : kSmallWG * E];
    const Place<BIG> me(G);
    const Cols<DT, VEC> cols(me.t, G, k.w);
    RowSum<3, BIG> sum{sm, G};
    const float inv = 1.f / (float)k.w;
    // with one gate per sequence `parts` workgroups share a sequence
    const long long rows = k.z_per_seq ? k.L : (long long)k.B * k.L;
    const long long seq = k.z_per_seq ? blockIdx.x / parts : 0;
    const long long part = k.z_per_seq ? blockIdx.x % parts : blockIdx.x;
    const long long base = seq * k.L;
    const long long b0 = base + rows * part / parts, b1 = base + rows * (part + 1) / parts;
    const bool row_gate = k.gate && !k.z_per_seq;
    // A row as read.  The next row's loads are under way while one is worked on,
    // where the registers allow it (16-bit elements, two to a register).
    constexpr bool AHEAD = VEC && DT != 0 && MAXT <= 256;
    struct Row {
        typename Cols<DT, VEC>::Held x, y, z, d, h;
        float rp, rq;
    } now{}, next{};
    auto fetch = [&](long long r0, Row& q) {
        const long long r = r0 + me.sub < b1 ? r0 + me.sub : b1 - 1;
        cols.hold(k.x, r * k.w, q.x);
        if (k.y) cols.hold(k.y, r * k.ldy, q.y);
        if (row_gate) cols.hold(k.z, r * k.ldz, q.z);
        if (k.dx_out) cols.hold(k.dx_out, r * k.w, q.d);
        if (k.dh) cols.hold(k.dh, r * k.w, q.h);
        q.rp = k.w_post ? k.rstd_post[r] : 1.f;
        q.rq = k.w_pre ? k.rstd_pre[r] : 0.f;
    };
    // the first row is asked for before the weights
    fetch(b0, AHEAD ? next : now);
    float acc1[E] = {}, acc2[E] = {};
    float z[E] = {}, v[E], slope[E];
    if (k.gate && k.z_per_seq) cols.load(k.z, seq * k.ldz, z);
    float kw[E], pre[E];
    cols.weights(k.w_post, 1.f, kw);
    cols.weights(k.scale, 1.f, pre);
#pragma unroll
    for (int j = 0; j < E; ++j) kw[j] *= pre[j];
    cols.weights(k.w_pre, 0.f, pre);
    gate_values<DT>(k.gate, z, v, slope);
    for (long long r0 = b0; r0 < b1; r0 += me.subs) {
        const bool live = r0 + me.sub < b1;
        const long long r = live ? r0 + me.sub : b1 - 1;
        if constexpr (AHEAD) {
            now = next;
            if (r0 + me.subs < b1) fetch(r0 + me.subs, next);
        } else if (r0 != b0) {
            fetch(r0, now);
        }
        if (row_gate) {
#pragma unroll
            for (int j = 0; j < E; ++j) z[j] = now.z.get(j);
            gate_values<DT>(k.gate, z, v, slope);
        }
        const float rp = now.rp, rq = now.rq;
        // n, m and d + rq e of a column
        auto terms = [&](int j, float* n, float* c, float* m, float* d) {
            *n = now.y.get(j) * rp;
            *c = kw[j] * v[j] * *n;
            *m = (now.x.get(j) + *c) * rq;
            *d = fmaf(rq * pre[j], now.h.get(j), now.d.get(j));
        };
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < E; ++j) {
            float n, c, m, d;
            terms(j, &n, &c, &m, &d);
            s[0] = fmaf(now.h.get(j) * pre[j], m, s[0]);
            s[1] = fmaf(d, c, s[1]);
            s[2] = fmaf(m, c, s[2]);
        }
        sum(s);
        const float m1 = rq * s[0] * inv;
        const float m2 = k.w_post ? (s[1] - m1 * s[2]) * inv : 0.f;
        now.x.renew();
        now.y.renew();
        now.d.renew();
        now.h.renew();
        float od[E], oy[E], oz[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            float n, c, m, d;
            terms(j, &n, &c, &m, &d);
            d = fmaf(-m1, m, d);
            od[j] = d;
            const float dn = d * n;
            if (live) {
                acc2[j] = fmaf(now.h.get(j), m, acc2[j]);
                acc1[j] = fmaf(dn, k.z_per_seq ? 1.f : v[j], acc1[j]);
            }
            oy[j] = rp * fmaf(d, kw[j] * v[j], -m2 * n);
            oz[j] = dn * kw[j] * slope[j];
        }
        if (live) {
            cols.store(k.dx, r * k.w, od);
            if (k.y) cols.store(k.dy, r * k.w, oy);
            if (row_gate) cols.store(k.dz, r * k.w, oz);
        }
    }
    // the workgroup's sums: over the rows it held at a time, in their order
    auto finish = [&](const float (&a)[E], float* to) {
        if (!to) return;
        to += (long long)blockIdx.x * k.w;
        if constexpr (BIG) {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (cols.has(j)) to[cols.c0 + j * cols.step] = a[j];
        } else {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < E; ++j) tot[j * kSmallWG + threadIdx.x] = a[j];
            __syncthreads();
            if (me.sub == 0)
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    float t = 0.f;
                    for (int i = 0; i < me.subs; ++i) t += tot[j * kSmallWG + i * G + me.t];
                    if (cols.has(j)) to[cols.c0 + j * cols.step] = t;
                }
        }
    };
    finish(acc1, k.part1);
    finish(acc2, k.part2);
}

// Sums over n rows of one column by LANES threads, in a fixed order.
template <int LANES>
__device__ __forceinline__ float column_sum(const float* p, long long n, int w, int c, int lane,
                                            float (*sm)[17]) {
    float t[4] = {};
    if (c < w) {
        long long i = lane;
        for (; i + 3 * LANES < n; i += 4 * LANES)
#pragma unroll
            for (int u = 0; u < 4; ++u) t[u] += p[(i + u * LANES) * w + c];
        for (; i < n; i += LANES) t[0] += p[i * w + c];
    }
    __syncthreads();
    sm[lane][threadIdx.x & 15] = (t[0] + t[1]) + (t[2] + t[3]);
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < LANES; ++i) s += sm[i][threadIdx.x & 15];
    return s;
}

// One gate per sequence: a sequence's sums over its workgroups; dz from them,
// and what they add to the sums over all rows (seq1, seq2 [B, w]).
template <int DT>
__global__ void __launch_bounds__(256) norm_bwd_seq(NormArgs k, int parts, float* seq1,
                                                    float* seq2) {
    __shared__ float sm[16][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
    const long long b = blockIdx.y;
    const float t = column_sum<16>(k.part1 + b * parts * k.w, parts, k.w, c, lane, sm);
    const float u = k.part2 ? column_sum<16>(k.part2 + b * parts * k.w, parts, k.w, c, lane, sm) : 0.f;
    if (lane != 0 || c >= k.w) return;
    float z[E] = {(float)pack_load<DT, 1>(k.z, b * k.ldz + c).e[0]}, v[E], slope[E];
    gate_values<DT>(k.gate, z, v, slope);
    const float kw = (k.w_post ? k.w_post[c] : 1.f) * (k.scale ? k.scale[c] : 1.f);
    const float dz[1] = {t * kw * slope[0]};
    pack_store<DT, 1>(k.dz, b * k.w + c, dz);
    if (seq1) seq1[b * k.w + c] = t * v[0];
    if (seq2) seq2[b * k.w + c] = u;
}

// The weights' gradients from n rows of partial sums.
__global__ void __launch_bounds__(16 * kSumLanes) norm_bwd_sum(NormArgs k, const float* p1, const float* p2,
                                                    long long n) {
    __shared__ float sm[kSumLanes][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
    if (p1) {
        const float t = column_sum<kSumLanes>(p1, n, k.w, c, lane, sm);
        if (lane == 0 && c < k.w) {
            if (k.dscale) k.dscale[c] = t * (k.w_post ? k.w_post[c] : 1.f);
            if (k.dw_post) k.dw_post[c] = t * (k.scale ? k.scale[c] : 1.f);
        }
    }
    if (p2) {
        const float t = column_sum<kSumLanes>(p2, n, k.w, c, lane, sm);
        if (lane == 0 && c < k.w) k.dw_pre[c] = t;
    }
}

// Threads of a row, and whether they are a workgroup.
int row_threads(int w) {
    const int need = (w + E - 1) / E;
    if (need > 64) return (need + 63) / 64 * 64;
    int g = 1;
    while (g < need) g *= 2;
    return g;
}

// Workgroups of the backward pass: enough to fill the chip, few enough that
// their partial sums are a small part of the traffic.  Two of 256 threads for
// each CU, or as many threads in smaller ones, two wider ones: 512, 768, 1024 and
// 1536 of them take, forward and backward of 16384 bfloat16 rows, w 2048 (256
// threads) 187, 190, 198 and 198 us, w 1024 (128) 120, 112, 103 and 101, w 512
// (256, four rows at a time) 57, 59, 63 and 68.
int target_groups(int w) {
    const int g = row_threads(w);
    return g > 64 && g < 256 ? 512 * 256 / g : 512;
}
int parts_of(const NormArgs& k) {
    const long long rows = k.z_per_seq ? k.L : (long long)k.B * k.L;
    const int subs = row_threads(k.w) > 64 ? 1 : kSmallWG / row_threads(k.w);
    const int want = k.z_per_seq ? (target_groups(k.w) + k.B - 1) / k.B : target_groups(k.w);
    const long long most = (rows + subs - 1) / subs;
    return (int)(most < want ? most : want);
}

// f(DT, VEC, MAXT): MAXT = 0 several rows in a workgroup, else its most threads
// (a row of 2048 columns or fewer leaves each thread more registers).
template <class F>
hipError_t by_kind(int dtype, bool vec, int threads, F&& f) {
    auto h = [&](auto dt, auto vc) {
        if (threads <= 64) return f(dt, vc, std::integral_constant<int, 0>{});
        if (threads <= 256) return f(dt, vc, std::integral_constant<int, 256>{});
        return f(dt, vc, std::integral_constant<int, 1024>{});
    };
    auto g = [&](auto dt) { return vec ? h(dt, std::true_type{}) : h(dt, std::false_type{}); };
    if (dtype == 0) return g(std::integral_constant<int, 0>{});
    if (dtype == 1) return g(std::integral_constant<int, 1>{});
    return g(std::integral_constant<int, 2>{});
}

// Rows in packs of E: all row strides multiples of E, all rows aligned (the
// contiguous sequences start on 16 bytes).
bool packed(const NormArgs& k, int dtype) {
    const uintptr_t mask = (dtype == 0 ? 4 : 2) * E - 1;
    auto ok = [&](const void* p, long long ld) { return !p || (((uintptr_t)p & mask) == 0 && ld % E == 0); };
    return k.w % E == 0 && ok(k.x, E) && ok(k.y, k.ldy) && ok(k.z, k.ldz) && ok(k.x_out, E) &&
           ok(k.h, E) && ok(k.dx_out, E) && ok(k.dh, E) && ok(k.dx, E) && ok(k.dy, E) &&
           ok(k.dz, E);
}

}  // namespace

// Partial sums of both kinds per workgroup, and with one gate per sequence
// per sequence.
size_t norm_workspace(int B, int w, bool z_per_seq) {
    const size_t n = z_per_seq ? 2 * (target_groups(w) + (size_t)B) + (size_t)2 * B
                               : (size_t)2 * target_groups(w);
    return n * w * sizeof(float);
}

hipError_t launch_norm_fwd(const NormArgs& k, int dtype, hipStream_t st) {
    const int G = row_threads(k.w);
    const bool big = G > 64;
    const int threads = big ? G : kSmallWG, subs = big ? 1 : kSmallWG / G;
    const long long need = ((long long)k.B * k.L + subs - 1) / subs;
    // as many threads as the registers let a CU hold, 1536: of 16384 bfloat16 rows,
    // w 2048, 512 to 2048 of them a CU take 78, 74 (768), 75 (1024), 71 (1536) and
    // 75 us, of 8192 float32 rows 56, 53, 52, 52 and 56
    const long long most = 256LL * 1536 / threads;
    const unsigned grid = (unsigned)(need < most ? need : most);
    return by_kind(dtype, packed(k, dtype), G, [&](auto dt, auto vec, auto bg) {
        norm_fwd<decltype(dt)::value, decltype(vec)::value, decltype(bg)::value>
            <<<grid, threads, 0, st>>>(k, G);
        return hipGetLastError();
    });
}

hipError_t launch_norm_bwd(const NormArgs& k0, int dtype, hipStream_t st) {
    NormArgs k = k0;
    const int G = row_threads(k.w);
    const bool big = G > 64;
    const int parts = parts_of(k);
    const long long groups = k.z_per_seq ? (long long)parts * k.B : parts;
    const bool want1 = k.dscale || k.dw_post, want2 = k.dw_pre;
    float* ws = (float*)k.ws;
    if (want1 || k.z_per_seq) k.part1 = ws;
    if (want2) k.part2 = ws + groups * k.w;
    hipError_t e = by_kind(dtype, packed(k, dtype), G, [&](auto dt, auto vec, auto bg) {
        norm_bwd<decltype(dt)::value, decltype(vec)::value, decltype(bg)::value>
            <<<(unsigned)groups, big ? G : kSmallWG, 0, st>>>(k, G, parts);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    const float *p1 = want1 ? k.part1 : nullptr, *p2 = k.part2;
    long long n = groups;
    const unsigned cols = (unsigned)((k.w + 15) / 16);
    if (k.z_per_seq) {
        float* s1 = ws + 2 * groups * k.w;
        float* s2 = s1 + (long long)k.B * k.w;
        // a grid's second axis ends at 65535
        for (int b = 0; b < k.B; b += 32768) {
            NormArgs q = k;
            const long long at = (long long)b * k.w;
            q.part1 = k.part1 + at * parts;
            q.part2 = k.part2 ? k.part2 + at * parts : nullptr;
            q.z = (const char*)k.z + (long long)b * k.ldz * (dtype == 0 ? 4 : 2);
            q.dz = (char*)k.dz + at * (dtype == 0 ? 4 : 2);
            const dim3 grid(cols, k.B - b < 32768 ? k.B - b : 32768);
            float *t1 = want1 ? s1 + at : nullptr, *t2 = want2 ? s2 + at : nullptr;
            if (dtype == 0)
                norm_bwd_seq<0><<<grid, 256, 0, st>>>(q, parts, t1, t2);
            else if (dtype == 1)
                norm_bwd_seq<1><<<grid, 256, 0, st>>>(q, parts, t1, t2);
            else
                norm_bwd_seq<2><<<grid, 256, 0, st>>>(q, parts, t1, t2);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        p1 = want1 ? s1 : nullptr;
        p2 = want2 ? s2 : nullptr;
        n = k.B;
    }
    if (p1 || p2) norm_bwd_sum<<<cols, 16 * kSumLanes, 0, st>>>(k, p1, p2, n);
    return hipGetLastError();
}

}  // namespace deeppcr
