// Orthogonalised update: X = G / (|G| + eps), then per step A = X X^T,
// B = cb A + cc A A, X = ca X + B X on every matrix of a stack.  A matrix with
// more rows than columns is worked on as its transpose, X [k, r] with k <= r.
//
// Bound by the matrix cores.  A float32 value is carried by two float16 parts,
// x 2^10 = hi + lo, to 2^-23 of it and not below 2^-35 (half the spacing of float16's
// smallest values): singular values start at most at 1, and the caller has made sure
// that no iterate or polynomial passes 15, so 2^10 x stays in range.  So a matrix as a
// whole keeps the precision of float32 products, and rows or columns far below the
// others do not: 150 x 200 with some rows 1e-4, 1e-6 and 1e-8 of the rest has
// those to 3e-5, 3e-3 and 0.3 of themselves, all by 2e-8 = 2^-35 485, what five steps
// magnify small values by.  A product is hi hi + hi lo + lo hi on the float16 matrix
// cores with float32 accumulation; lo lo is below 2^-22 of it.  (The float32
// instructions have a sixteenth of the float16 ones' rate, against a third.)
// The iterates stay in these parts between the products.  A and A A are
// symmetric: their tiles on and above the diagonal are computed and written
// twice.
//
// A gradient far below eps makes a small X.  It is held as Y = 2^e X with 2^-e a
// bound of its norm, so that its parts keep their bits:
//   Y' = 2^(e'-e) (ca Y + (cb 2^-2e A + cc 2^-4e A A) Y),  A = Y Y^T;
// the bound follows s -> |ca| s + |cb| s^3 + |cc| s^5, which is close where only
// the linear term counts.
#include <algorithm>
#include <type_traits>

#include "elem.h"
#include "internal.h"

namespace deeppcr {
namespace {

typedef _Float16 h16;
typedef h16 h16x8 __attribute__((ext_vector_type(8)));
typedef h16 h16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kScale = 1024.f, kUnscale = 1.f / 1024.f;  // 2^10

// The NP parts of four values that are already multiplied by kScale: a packed
// conversion and a mixed-precision multiply-add each a pair (the matrix cores
// and these instructions share a wave's issue slots).
template <int NP>
__device__ __forceinline__ void split(const float (&s)[4], h16x4 (&part)[NP]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef h16 h16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        f32x2 r{s[i], s[i + 1]};
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const h16x2 h = __builtin_convertvector(r, h16x2);
            part[p][i] = h.x, part[p][i + 1] = h.y;
            r = f32x2{fmaf((float)h.x, -1.f, r.x), fmaf((float)h.y, -1.f, r.y)};
        }
    }
}
// own (hi + lo) + v
__device__ __forceinline__ float add_own(float own, h16 hi, h16 lo, float v) {
    return fmaf((float)hi, own, fmaf((float)lo, own, v));
}

// Four rows of a lane's column <-> row lane % 4 of them, of the four columns of
// the lane's quad (its own inverse): two exchanges inside the quad, elements two to a register.
__device__ __forceinline__ h16x4 quad_turn(h16x4 v) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 w = __builtin_bit_cast(u32x2, v);
    const bool odd = threadIdx.x & 1, upper = threadIdx.x & 2;
    // even lanes: the first of each pair of rows, odd lanes the second
    const unsigned sel = odd ? 0x03020706u : 0x05040100u;
    unsigned a = __builtin_amdgcn_perm(
        __builtin_amdgcn_update_dpp(0u, w.x, 0xB1, 0xF, 0xF, false), w.x, sel);
    unsigned b = __builtin_amdgcn_perm(
        __builtin_amdgcn_update_dpp(0u, w.y, 0xB1, 0xF, 0xF, false), w.y, sel);
    // the lower two lanes keep the first two rows, the upper two the others
    const unsigned got = __builtin_amdgcn_update_dpp(0u, upper ? a : b, 0x4E, 0xF, 0xF, false);
    return __builtin_bit_cast(h16x4, upper ? u32x2{got, b} : u32x2{a, got});
}

// Rows 8 q + 4 half + 0 .. 3 for q = 0, 1 of a lane's column <-> rows 8 half +
// 0 .. 7, by an exchange between the halves of the wave (its own inverse).
__device__ __forceinline__ void half_turn(h16x4* p, h16x4* q) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_bit_cast(u32x2, *p), b = __builtin_bit_cast(u32x2, *q);
    const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
    *p = __builtin_bit_cast(h16x4, u32x2{x[0], y[0]});
    *q = __builtin_bit_cast(h16x4, u32x2{x[1], y[1]});
}

// Reads LDS across its rows (see where it is used).
__device__ __forceinline__ h16x4 read_across(const h16* p) {
    typedef __fp16 f16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) f16x4* Lds;
    return __builtin_bit_cast(h16x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((Lds)p));
}

// ------------------------------------------------------------------ the start
constexpr int kParts = 64;  // most workgroups that share a matrix's norm
// Squares are summed in units of 2^160, 1 and 2^-160; to the next larger unit:
__device__ __forceinline__ float next_unit(float sum) { return sum * 0x1p-80f * 0x1p-80f; }

// Sums of squares of the large, ordinary and small elements of a part of a
// matrix, so that no square and no sum of the at most 2^26 of them leaves the
// float32 range: 2^26 2^100 of the ordinary ones, 2^26 2^96 of the large ones.
template <int DT>
__global__ void __launch_bounds__(256) ortho_norm(const void* G, float4* out, long long sz) {
    __shared__ float sm[3][4];
    constexpr int V = 16 / sizeof(elem_t<DT>);
    const long long base = blockIdx.y * sz;
    // whole packs where the matrices start on 16 bytes, else single elements
    const bool packs = sz % V == 0;
    const long long n = packs ? sz / V : sz;
    const long long b = n * blockIdx.x / gridDim.x, e = n * (blockIdx.x + 1) / gridDim.x;
    float big = 0.f, mid = 0.f, tiny = 0.f;
    auto add = [&](float g) {
        const float a = fabsf(g);
        const bool l = a > 0x1p50f, s = a < 0x1p-60f;
        const float x = l ? g * 0x1p-80f : s ? g * 0x1p80f : g;  // NaN is ordinary
        if (l) big = fmaf(x, x, big);
        if (s) tiny = fmaf(x, x, tiny);
        if (!l && !s) mid = fmaf(x, x, mid);
    };
    if (packs) {
#pragma unroll 4
        for (long long i = b + threadIdx.x; i < e; i += 256) {
            const Pack<DT, V> p = pack_load<DT, V>(G, base + i * V);
#pragma unroll
            for (int v = 0; v < V; ++v) add((float)p.e[v]);
        }
    } else {
        for (long long i = b + threadIdx.x; i < e; i += 256)
            add((float)pack_load<DT, 1>(G, base + i).e[0]);
    }
    for (int m = 1; m < 64; m *= 2) {
        big += __shfl_xor(big, m);
        mid += __shfl_xor(mid, m);
        tiny += __shfl_xor(tiny, m);
    }
    if ((threadIdx.x & 63) == 0) {
        sm[0][threadIdx.x >> 6] = big;
        sm[1][threadIdx.x >> 6] = mid;
        sm[2][threadIdx.x >> 6] = tiny;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        auto all = [&](int i) { return (sm[i][0] + sm[i][1]) + (sm[i][2] + sm[i][3]); };
        out[blockIdx.y * gridDim.x + blockIdx.x] = make_float4(all(0), all(1), all(2), 0.f);
    }
}

// The factors by which a matrix becomes X: g * unit * inv; its norm is
// 2^-depth.
struct Start {
    float unit, inv, depth;
};
__device__ __forceinline__ Start start_of(const float4* parts, int n, float eps) {
    float big = 0.f, mid = 0.f, tiny = 0.f;
    for (int i = 0; i < n; ++i) {
        big += parts[i].x;
        mid += parts[i].y;
        tiny += parts[i].z;
    }
    // the largest elements' unit; two units below there is nothing beside them
    float unit = 1.f, sum = mid + next_unit(tiny);
    if (big > 0.f) {
        unit = 0x1p-80f;
        sum = big + next_unit(mid);
    } else if (mid == 0.f) {
        unit = 0x1p80f;
        sum = tiny;
    }
    // a zero matrix stays zero, whatever eps; a NaN makes all of it NaN
    if (sum == 0.f) return {1.f, 0.f, 0.f};
    const float norm = sqrtf(sum), den = norm + eps * unit;
    return {unit, 1.f / den, log2f(den / norm)};
}

// The polynomial's coefficients' sizes; the bound's logarithm after a step (no
// iterate passes 15); and the shift that goes with it.
struct Growth {
    float a, b, c;
};
__device__ __forceinline__ float grown(float bound, const Growth& g) {
    const float s = exp2f(2.f * bound);
    return fminf(bound + log2f(fmaf(s, fmaf(s, g.c, g.b), g.a)), 4.f);
}
__device__ __forceinline__ int shift_of(float bound) {
    const float e = floorf(-bound);
    return e > 0.f ? (int)fminf(e, 120.f) : 0;  // 0 where the bound is NaN
}
// Of one matrix between the launches: the bound behind the step under way, its
// shift and the next step's.
struct Shift {
    float bound;
    int now, next;
};

// The parts of a stack of matrices [rows, cols], padded to whole tiles with
// zeros, in panels of 16 columns: a row of a panel is 16 hi and 16 lo, and the
// rows of a panel follow each other, so that a tile's share of a step is one run
// of memory.
struct Panels {
    h16* p;
    long long sz;  // rows * cols
    int rows;
    __device__ __forceinline__ h16* at(long long z, int row, int col) const {
        return p + 2 * z * sz + ((long long)(col >> 4) * rows + row) * 32 + (col & 15);
    }
};
constexpr int kLo = 16;  // from hi to lo

// X [kp, rp] from G [m, n] (its transpose where m > n), 64 x 64 at a time.
template <int DT>
__global__ void __launch_bounds__(256) ortho_start(const void* G, Panels X, const float4* parts,
                                                   int nparts, Shift* shifts, int m, int n,
                                                   float eps) {
    __shared__ float t[64][65];
    const long long z = blockIdx.z;
    const Start s = start_of(parts + z * nparts, nparts, eps);
    const int shift = shift_of(-s.depth);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) shifts[z] = {-s.depth, 0, shift};
    const float inv = ldexpf(s.inv, shift);
    const bool tall = m > n;
    // rows i0.. and columns j0.. of G, padded like it
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        const int i = e / 64, j = e % 64;
        float g = 0.f;
        if (i0 + i < m && j0 + j < n)
            g = (float)pack_load<DT, 1>(G, z * (long long)m * n + (long long)(i0 + i) * n + j0 + j).e[0] *
                s.unit * inv;
        t[i][j] = g;
    }
    __syncthreads();
    // four elements of a row
    for (int e = threadIdx.x; e < 64 * 16; e += 256) {
        const int i = e / 16, j = e % 16 * 4;
        h16x4 x[2];
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = kScale * (tall ? t[j + u][i] : t[i][j + u]);
        split(v, x);
        h16* p = tall ? X.at(z, j0 + i, i0 + j) : X.at(z, i0 + i, j0 + j);
        *reinterpret_cast<h16x4*>(p) = x[0];
        *reinterpret_cast<h16x4*>(p + kLo) = x[1];
    }
}

// With no steps: X itself.
template <int DT>
__global__ void __launch_bounds__(256) ortho_scaled(const void* G, void* X, const float4* parts,
                                                    int nparts, long long sz, float eps) {
    const long long z = blockIdx.y;
    const Start s = start_of(parts + z * nparts, nparts, eps);
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < sz; i += gridDim.x * 256LL) {
        const float v[1] = {(float)pack_load<DT, 1>(G, z * sz + i).e[0] * s.unit * s.inv};
        pack_store<DT, 1>(X, z * sz + i, v);
    }
}

// --------------------------------------------------------------- the products
enum { GRAM, POLY, APPLY };

struct Product {
    Panels P, Q;   // C[i, j] = sum_t P[i, t] Q[j, t], APPLY: sum_t P[i, t] Q[t, j]
    Panels C;      // the result; its own term D is A = P = Q, APPLY: X = Q
    void* out;     // last APPLY: X [m, n] instead
    int rows, cols, K;  // padded
    int m, n;
    Shift* shifts;
    Growth growth;
    float own, times;   // own D + times P Q, before the shifts
};

// One tile of BM x BN per workgroup of 2 x 2 waves, in turn over the matrices
// so that an XCD (workgroups go to the 8 of them in turn) works on few.  Steps of
// 16 columns leave room for four workgroups on a CU, which hide each other's
// loads and barriers: 16 matrices of 1024 x 1024 1.35 ms a call in square tiles,
// against 1.49 with two workgroups, steps of 32 and the loads two steps ahead in
// registers.
template <int BM, int BN, int MODE, int OUT>
__global__ void __launch_bounds__(256, 4) ortho_product(Product g, int tiles, long long all) {
    constexpr int BK = 16, MT = BM / 64, NT = BN / 64;  // a wave's tiles of 32 x 32
    // also loads of 64 chunks of an operand per wave
    constexpr int LD[2] = {MT, NT};
    // Steps under way: one beside the one worked on, where large tiles fill the
    // chip; three where small ones leave a CU few workgroups to hide their loads: one of
    // 256 x 256 100 us against 150, two of 1024 x 1024 279 and 451, five of 960 x
    // 960 492 and 613 (of large tiles more than one gained nothing, 8 of 1024 x 1024
    // 683 us and 683).
    constexpr int NB = BM == 64 ? 4 : 2;
    // A matrix instruction cuts its 16 products to the bits that the largest of them
    // and the sum leave them (1 + 15 x 0.9 2^-23 gives 1 + 11 x 2^-23), so that a long
    // sum's error grows in one direction.  Small tiles have registers for five sums: the
    // small terms, and hi hi of every fourth step.  Against float32 products 33 x 8192
    // errs 0.8 times as much (with one sum 2.8), 33 x 1024 1.4 (2.3), 128 x 8192 0.5
    // (2.0), and no sum waits for the one before it: 16 of 64 x 4096 243 us, 270 with
    // one.  Large tiles err 0.9 times as much at most, those of 16 of 1024 x 1024 0.7
    // (with two sums 0.5, and 1452 us a call against 1386).
    constexpr int SUMS = BM == 64 ? 5 : 1, TURNS = SUMS > 1 ? SUMS - 1 : 1;
    __shared__ __attribute__((aligned(16))) h16 sm[NB][(BM + BN) * 2 * BK];  // buffer; both operands
    constexpr int RIGHT = BM * 2 * BK;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long per = (all + 7) / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || id >= all) return;
    const long long z = id / tiles;
    int bi, bj;
    if constexpr (MODE == APPLY) {
        const int nt = g.cols / BN;
        bi = (int)(id % tiles) / nt;
        bj = (int)(id % tiles) % nt;
    } else {
        // tiles on and above the diagonal: of BM columns, column by column, and
        // of those the BM / BN parts
        constexpr int H = BM / BN;
        const int t = (int)(id % tiles) / H;
        bj = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        while (bj * (bj + 1) / 2 > t) --bj;
        while ((bj + 1) * (bj + 2) / 2 <= t) ++bj;
        bi = t - bj * (bj + 1) / 2;
        bj = bj * H + (int)(id % tiles) % H;
    }
    // An operand's tile in a step: BM or BN rows of one panel, or (APPLY's right
    // one) 16 rows of BN / 16 panels, whose columns are read across.
    constexpr bool ACROSS = MODE == APPLY;
    const h16* src[2] = {g.P.at(z, bi * BM, 0),
                         ACROSS ? g.Q.at(z, 0, bj * BN) : g.Q.at(z, bj * BN, 0)};
    const long long ahead[2] = {g.P.rows * 32LL, ACROSS ? 16 * 32LL : g.Q.rows * 32LL};
    // chunk c of a row (2 of hi, 2 of lo) sits at c ^ (row / 4 mod 4): 16 rows
    // that are read together lie in different banks
    auto chunk = [](int row, int c) { return row * 32 + (c ^ ((row >> 2) & 3)) * 8; };
    // A step's tiles go from memory to LDS without passing registers: a wave's
    // load fills 64 chunks in the lanes' order, so each lane asks for the chunk
    // that belongs there.  (Before a read of LDS the compiler waits for all such
    // loads that it knows of; where later ones are under way it is not told of them.
    // They write no register, and the loop waits for them itself.)
    typedef const __attribute__((address_space(1))) void* Global;
    typedef __attribute__((address_space(3))) void* Lds;
    long long from[2][MT];
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int u = 0; u < LD[o]; ++u) {
            const int row = (u * 4 + wave) * 16 + (lane >> 2), c = (lane & 3) ^ ((row >> 2) & 3);
            from[o][u] = ACROSS && o == 1 ? (row >> 4) * (g.Q.rows * 32LL) + (row & 15) * 32 + c * 8
                                          : row * 32 + c * 8;
        }
    auto stage = [&](int buf, int s) {
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int u = 0; u < LD[o]; ++u) {
                const auto* p = src[o] + s * ahead[o] + from[o][u];
                const Lds to = (Lds)&sm[buf][o * RIGHT + (u * 4 + wave) * 512];
                if constexpr (NB == 2) {
                    __builtin_amdgcn_global_load_lds((Global)p, to, 16, 0, 0);
                } else {
                    // (the address of LDS goes by m0, which the compiler sets)
                    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                                 :
                                 : "v"((Global)p), "{m0}"((unsigned)(size_t)to)
                                 : "memory");
                }
            }
    };
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const int r32 = lane & 31, half = lane >> 5;
    // the wave's first row and column; one that lies below the diagonal has
    // nothing to do (of square tiles too few do to ask for it)
    const int r0 = bi * BM + wm, c0 = bj * BN + wn;
    const bool needed = MODE == APPLY || BM == BN || r0 < c0 + BN / 2;
    f32x16 sum[SUMS][MT][NT] = {};
    const int steps = g.K / BK;  // a multiple of four
#pragma unroll
    for (int s = 0; s < NB - 1; ++s)
        if (s < steps) stage(s, s);
    auto step = [&](int s, int turn) {
        // this step's tiles have arrived (the loads of the NB - 2 steps behind it may
        // be under way), and nobody reads the buffer before it any more
        if (NB > 2 && s + NB - 2 < steps)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * (MT + NT)) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int buf = s & (NB - 1);
        h16x8 a[MT][2], b[NT][2];
        if (needed) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    a[t][p] = *reinterpret_cast<const h16x8*>(&sm[buf][chunk(wm + t * 32 + r32, p * 2 + half)]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if constexpr (ACROSS) {
                        // lane 4 i + j of 16 gives row i, columns 4 j .. 4 j + 3 of a 4 x 16
                        // block and gets its column 4 i + j
                        h16x4 v[2];
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int k = wn + t * 32 + (lane & 16) + half * 8 + u * 4 + ((lane & 15) >> 2);
                            v[u] = read_across(&sm[buf][RIGHT + chunk(k, p * 2 + ((lane & 3) >> 1)) + (lane & 1) * 4]);
                        }
                        b[t][p] = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    } else {
                        b[t][p] = *reinterpret_cast<const h16x8*>(&sm[buf][RIGHT + chunk(wn + t * 32 + r32, p * 2 + half)]);
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (s + NB - 1 < steps) stage((s + NB - 1) & (NB - 1), s + NB - 1);
        __builtin_amdgcn_sched_barrier(0);
        if (needed) {
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        f32x16& to = sum[p < 2 ? SUMS - 1 : turn][i][j];
                        to = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][p == 0], b[j][p == 1], to,
                                                                    0, 0, 0);
                    }
        }
    };
    for (int s = 0; s < steps; s += TURNS)
#pragma unroll
        for (int turn = 0; turn < TURNS; ++turn) step(s + turn, turn);
    f32x16(&acc)[MT][NT] = sum[0];
#pragma unroll
    for (int k = 1; k < SUMS; ++k)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] += sum[k][i][j];
    // a lane holds column r32 of each 32 x 32 tile, rows 8 q + 4 half + 0 .. 3
    // values times kScale, as their parts are
    float own = g.own, f = g.times * kUnscale;
    int fin = 0;
    if constexpr (MODE == GRAM) {
        // the step's first launch moves the shifts on; the others read them
        if (id % tiles == 0 && threadIdx.x == 0) {
            Shift s = g.shifts[z];
            s.bound = grown(s.bound, g.growth);
            s.now = s.next;
            s.next = shift_of(s.bound);
            g.shifts[z] = s;
        }
    } else {
        const Shift s = g.shifts[z];
        const int e = s.now;
        if constexpr (MODE == POLY) {
            own = ldexpf(own, -2 * e);
            f = ldexpf(f, -4 * e);
        } else if constexpr (OUT >= 0) {
            fin = -e;  // out of the shift; not in the factors, where it may be subnormal
        } else {
            const int d = s.next - e;
            own = ldexpf(own, d);
            f = ldexpf(f, d);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int row0 = r0 + i * 32, col0 = c0 + j * 32, col = col0 + r32;
            if (MODE != APPLY && row0 > col0) continue;
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                h16x4 own_hi[2], own_lo[2];
                if constexpr (MODE == POLY) {
                    // by symmetry 8 columns of a row: one load
                    const h16* d = g.P.at(z, col, row0 + 8 * (q + half));
                    const h16x8 dh = *reinterpret_cast<const h16x8*>(d);
                    const h16x8 dl = *reinterpret_cast<const h16x8*>(d + kLo);
                    own_hi[0] = dh.lo, own_hi[1] = dh.hi, own_lo[0] = dl.lo, own_lo[1] = dl.hi;
                    half_turn(&own_hi[0], &own_hi[1]);
                    half_turn(&own_lo[0], &own_lo[1]);
                } else if constexpr (MODE == APPLY) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const h16* d = g.Q.at(z, row0 + 8 * (q + u) + 4 * half + (lane & 3), col & ~3);
                        own_hi[u] = quad_turn(*reinterpret_cast<const h16x4*>(d));
                        own_lo[u] = quad_turn(*reinterpret_cast<const h16x4*>(d + kLo));
                    }
                }
                h16x4 hi[2], lo[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int row = row0 + 8 * (q + u) + 4 * half;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = f * acc[i][j][4 * (q + u) + e];
                        if (MODE != GRAM) v[e] = add_own(own, own_hi[u][e], own_lo[u][e], v[e]);
                        if constexpr (OUT >= 0) {
                            const float one[1] = {ldexpf(v[e] * kUnscale, fin)};
                            const bool tall = g.m > g.n;
                            const int r = tall ? col : row + e, c = tall ? row + e : col;
                            if (r < g.m && c < g.n)
                                pack_store<OUT < 0 ? 0 : OUT, 1>(
                                    g.out, (z * g.m + r) * (long long)g.n + c, one);
                        }
                    }
                    if constexpr (OUT < 0) {
                        h16x4 x[2];
                        split(v, x);
                        hi[u] = x[0];
                        lo[u] = x[1];
                    }
                    if (OUT < 0 && (MODE == APPLY || row0 != col0)) {
                        h16* c = g.C.at(z, row + (lane & 3), col & ~3);
                        *reinterpret_cast<h16x4*>(c) = quad_turn(hi[u]);
                        *reinterpret_cast<h16x4*>(c + kLo) = quad_turn(lo[u]);
                    }
                }
                if constexpr (MODE != APPLY) {
                    // by symmetry the tile across the diagonal (one on it only here)
                    half_turn(&hi[0], &hi[1]);
                    half_turn(&lo[0], &lo[1]);
                    h16* c = g.C.at(z, col, row0 + 8 * (q + half));
                    *reinterpret_cast<h16x8*>(c) = __builtin_shufflevector(hi[0], hi[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    *reinterpret_cast<h16x8*>(c + kLo) = __builtin_shufflevector(lo[0], lo[1], 0, 1, 2, 3, 4, 5, 6, 7);
                }
            }
        }
}

// ----------------------------------------------------------- small matrices
// A matrix of up to P x P (P = 32, 64, 128) stays in one workgroup for all
// steps.  Wave v holds the columns 32 v .. 32 v + 31 of X in registers, as the
// products leave them: column lane % 32, rows 8 q + 4 (lane / 32) + e of each 32
// (q, e < 4).  Read as the right operand of a product these are the rows in the
// order 0-3, 8-11 | 4-7, 12-15 of every 16; A and B, which meet them, have their
// columns in LDS in that order, and their symmetry lets a lane write its column
// as a row, four elements at once.  X goes to LDS by rows for the Gram product
// only, then A, then B take its place.
// 1 / (|G| + eps), shifted for the first step, for a matrix whose elements have
// been divided by the largest, `top`, and then have the square sum `sum`; a zero
// matrix stays zero, whatever eps, and NaN stays NaN.
__device__ __forceinline__ float inverse_norm(float top, float sum, float eps, float* bound) {
    *bound = 0.f;
    if (!(top > 0.f)) return sum == sum ? 0.f : sum;
    const float norm = sqrtf(sum), den = norm + eps / top;
    *bound = -log2f(den / norm);
    return ldexpf(1.f / den, shift_of(*bound));
}

// A matrix of up to 16 x 16 in one wave's registers: element e of a lane is row
// 4 (lane / 16) + e of column lane % 16, which is how a product leaves a tile and
// how the next one takes its right operand, and by the symmetry of A and B its
// left one.  X is turned for the Gram product by lane exchanges.  Three parts to
// a value, six terms to a product (as of few rows below).  1024 matrices of 16 x 16
// take 6.0 us (in a graph; in the 32 x 32 kernel a call took 12.4 us when it took 9.0
// here).
template <int DT>
__global__ void __launch_bounds__(64) ortho_tiny(const void* G, void* out, int m, int n, int steps,
                                                 float ca, float cb, float cc, float eps,
                                                 Growth growth) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    constexpr int NP = 3;
    const int lane = threadIdx.x, col = lane & 15, row0 = lane >> 4 << 2;
    const bool tall = m > n;
    const int k = tall ? n : m, r = tall ? m : n;
    const long long base = (long long)blockIdx.x * m * n;
    auto at_of = [&](int row) { return base + (tall ? (long long)col * n + row : (long long)row * n + col); };
    float v[4];
    float top = 0.f, bad = 0.f, sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = row0 + e < k && col < r ? (float)pack_load<DT, 1>(G, at_of(row0 + e)).e[0] : 0.f;
        top = fmaxf(top, fabsf(v[e]));
        bad += v[e] * 0.f;  // NaN where an element is not finite
    }
    for (int s = 1; s < 64; s *= 2) {
        top = fmaxf(top, __shfl_xor(top, s));
        bad += __shfl_xor(bad, s);
    }
    if (top > 0.f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] /= top;
            sum = fmaf(v[e], v[e], sum);
        }
    for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
    float bound;
    const float inv = inverse_norm(top, sum + bad, eps, &bound);
    int e = shift_of(bound);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= inv * kScale;
    h16x4 x[NP];
    split(v, x);
    // lane 16 i + 4 j + l of a quad_turn'ed tile holds row 4 i + l, columns 4 j ..:
    // lane 16 j + 4 i + l is to have it
    const int from = (16 * (col >> 2) + 4 * (lane >> 4) + (col & 3)) * 4;
    auto turned = [&](h16x4 a) {
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        const i32x2 w = __builtin_bit_cast(i32x2, quad_turn(a));
        return __builtin_bit_cast(h16x4, i32x2{__builtin_amdgcn_ds_bpermute(from, w.x),
                                               __builtin_amdgcn_ds_bpermute(from, w.y)});
    };
    auto product = [&](const h16x4 (&l)[NP], const h16x4 (&r)[NP]) {
        f32x4 a[2] = {};  // small terms, and hi hi
#pragma unroll
        for (int order = NP - 1; order >= 0; --order)
#pragma unroll
            for (int p = order; p >= 0; --p)
                a[order == 0] = __builtin_amdgcn_mfma_f32_16x16x16f16(l[p], r[order - p],
                                                                      a[order == 0], 0, 0, 0);
        return a[0] + a[1];
    };
    auto parts = [&](const f32x4& a, h16x4 (&to)[NP]) {
        const float s[4] = {a.x, a.y, a.z, a.w};
        split(s, to);
    };
    const float f = kUnscale;
    for (int s = 0; s < steps; ++s) {
        bound = grown(bound, growth);
        const int next = shift_of(bound);
        h16x4 y[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) y[p] = turned(x[p]);
        const f32x4 A = product(y, y) * f;
        parts(A, y);
        const f32x4 B = A * ldexpf(cb, -2 * e) + product(y, y) * ldexpf(cc * f, -4 * e);
        parts(B, y);
        const bool last = s + 1 == steps;
        const int d = last ? 0 : next - e;
        f32x4 c = product(y, x) * ldexpf(f, d);
        const float own = ldexpf(ca, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) c[i] = fmaf((float)x[p][i], own, c[i]);
            v[i] = last ? ldexpf(c[i], -e) : c[i];
        }
        split(v, x);
        e = next;
    }
    if (steps == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = ldexpf(v[i], -e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float one[1] = {v[i] * kUnscale};
        if (row0 + i < k && col < r) pack_store<DT, 1>(out, at_of(row0 + i), one);
    }
}

// RT = ceil(k / 32) row tiles are in use: known to the compiler, so that nothing
// between the instructions asks whether one is, and symmetric products are
// computed by half (1024 matrices of 128 x 128: 191 us without either, 187
// without the second, 165).
template <int P, int RT, int DT>
__global__ void __launch_bounds__(2 * P, 2) ortho_small(const void* G, void* out, int m, int n,
                                                        int steps, float ca, float cb, float cc,
                                                        float eps, Growth growth) {
    constexpr int NT = P / 32, PITCH = P + 8;  // a row's 16 bytes more spread the banks
    // Sums of few products have no rounding of their own to hide two parts' in
    // (4 x 4 matrices erred by 1.5 times what float32 products do, 11 x 11 by up
    // to 1.7, 4 x 69 by 1.9): there a value has three parts, to 2^-24 of it and not
    // below 2^-35 either, and a product six terms.
    constexpr int NP = RT == 1 ? 3 : 2;
    __shared__ __attribute__((aligned(16))) h16 sm[NP][32 * RT * PITCH];
    __shared__ float red[2][NT];
    const int lane = threadIdx.x & 63;
    // The second workgroup of a CU (256 of them) counts its waves from the other
    // half: the first half of them has more to do, and they share the SIMDs.
    const int wave = (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) +
                      (blockIdx.x >> 8 & 1) * (NT / 2)) % NT;
    const int r32 = lane & 31, half = lane >> 5;
    const bool tall = m > n;
    const int k = tall ? n : m, r = tall ? m : n;
    const int col = 32 * wave + r32;
    const long long base = (long long)blockIdx.x * m * n;
    auto row_of = [&](int t, int q, int e) { return 32 * t + 8 * q + 4 * half + e; };
    auto at_of = [&](int row) { return base + (tall ? (long long)col * n + row : (long long)row * n + col); };

    f32x16 acc[RT];
    float top = 0.f, bad = 0.f;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = row_of(t, i / 4, i % 4);
            acc[t][i] = row < k && col < r ? (float)pack_load<DT, 1>(G, at_of(row)).e[0] : 0.f;
            top = fmaxf(top, fabsf(acc[t][i]));
            bad += acc[t][i] * 0.f;  // NaN where an element is not finite
        }
    for (int s = 1; s < 64; s *= 2) {
        top = fmaxf(top, __shfl_xor(top, s));
        bad += __shfl_xor(bad, s);
    }
    if (lane == 0) red[0][wave] = top, red[1][wave] = bad;
    __syncthreads();
    bad = 0.f;
    for (int v = 0; v < NT; ++v) top = fmaxf(top, red[0][v]), bad += red[1][v];
    __syncthreads();
    float sum = 0.f;
    if (top > 0.f)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                acc[t][i] /= top;
                sum = fmaf(acc[t][i], acc[t][i], sum);
            }
    for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
    if (lane == 0) red[0][wave] = sum;
    __syncthreads();
    sum = bad;
    for (int v = 0; v < NT; ++v) sum += red[0][v];
    float bound;
    const float inv = inverse_norm(top, sum, eps, &bound);
    int e = shift_of(bound);
    h16x8 x[RT][2][NP];
    // X's parts from four values times kScale
    auto keep = [&](int t, int q, const float (&v)[4]) {
        h16x4 part[NP];
        split(v, part);
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[t][q / 2][p][4 * (q & 1) + e] = part[p][e];
    };
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[t][4 * q + e] *= inv, v[e] *= kScale;
            keep(t, q, v);
        }

    // acc[d] = sum over K steps of 16 of the rows of tile tile_of(d) of LDS
    // against `right`, d < D
    // Three parts: hi hi in sums of its own, one or of many steps two (see small tiles
    // above): with one sum for all terms 4 x 128 erred by 1.5 times what float32
    // products do, now 1.1 (1024 of 32 x 128 34.0 us, 35.1).
    auto product = [&](auto D, auto K, auto&& tile_of, auto&& right) {
        constexpr int N = decltype(D)::value;
        constexpr int TURNS = NP < 3 ? 0 : decltype(K)::value < 8 ? 1 : 2;
        constexpr int MORE = TURNS > 0 ? TURNS : 1;
        f32x16 more[MORE][N] = {};
#pragma unroll
        for (int d = 0; d < N; ++d) acc[d] = f32x16{};
#pragma unroll
        for (int s = 0; s < decltype(K)::value; ++s) {
            h16x8 b[NP], a[N][NP];
            right(s, b);
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    a[d][p] = *reinterpret_cast<const h16x8*>(
                        &sm[p][(32 * tile_of(d) + r32) * PITCH + 16 * s + 8 * half]);
#pragma unroll
            for (int order = NP - 1; order >= 0; --order)  // the small terms first
#pragma unroll
                for (int p = order; p >= 0; --p)
#pragma unroll
                    for (int d = 0; d < N; ++d) {
                        f32x16& to = TURNS > 0 && order == 0 ? more[s % MORE][d] : acc[d];
                        to = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[d][p], b[order - p], to, 0, 0,
                                                                    0);
                    }
        }
        if constexpr (TURNS > 0)
#pragma unroll
            for (int t = 0; t < TURNS; ++t)
#pragma unroll
                for (int d = 0; d < N; ++d) acc[d] += more[t][d];
    };
    // The tiles of a symmetric product that a wave below RT computes: those of its
    // column from the diagonal one on, going round, half of them in all (the one
    // half way round by the first half of the waves); it writes each twice.
    constexpr int HALF = RT / 2 + 1, SURE = (RT + 1) / 2;
    auto across = [&](int d) { return (wave + d) % RT; };
    auto mine = [&](int d) { return d < SURE || wave < RT / 2; };
    auto symmetric = [&](auto K, auto&& right) {
        if (HALF == SURE || wave < RT / 2)
            product(std::integral_constant<int, HALF>{}, K, across, right);
        else
            product(std::integral_constant<int, SURE>{}, K, across, right);
    };
    constexpr std::integral_constant<int, 2 * RT> kRows{};
    constexpr std::integral_constant<int, P / 16> kCols{};
    // the wave's 32 rows of LDS as the right operand
    auto own_rows = [&](int s, h16x8 (&b)[NP]) {
#pragma unroll
        for (int p = 0; p < NP; ++p)
            b[p] = *reinterpret_cast<const h16x8*>(&sm[p][col * PITCH + 16 * s + 8 * half]);
    };
    // rows 8 q + 4 half + 0 .. 3 of tile t of the lane's column, by symmetry
    // columns of its row
    auto run_of = [&](int t, int q) {
        return col * PITCH + 32 * t + 16 * (q >> 1) + 4 * (2 * half + (q & 1));
    };
    const float f = kUnscale;  // of a product, for a value times kScale
    // One tile, one wave: A and B are symmetric, so that a lane's column, as a
    // product leaves it, is its row as the left operand too: they never leave the
    // registers.  X crosses LDS for the Gram product.
    auto one_tile = [&](bool last, int e, int next) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const h16x8 h = x[0][q / 2][p];
                *reinterpret_cast<h16x4*>(&sm[p][row_of(0, q, lane & 3) * PITCH + (col & ~3)]) =
                    quad_turn(q & 1 ? h.hi : h.lo);
            }
        wave_sync();
        h16x8 rows[2][NP];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int p = 0; p < NP; ++p)
                rows[c][p] = *reinterpret_cast<const h16x8*>(&sm[p][r32 * PITCH + 16 * c + 8 * half]);
        wave_sync();
        // two accumulators: a product need not wait for the one before it
        auto times_of = [&](const h16x8 (&l)[2][NP], const h16x8 (&r)[2][NP]) {
            f32x16 sum[2] = {};
#pragma unroll
            for (int order = NP - 1; order >= 0; --order)
#pragma unroll
                for (int p = order; p >= 0; --p)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        sum[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[c][p], r[c][order - p],
                                                                        sum[c], 0, 0, 0);
            return sum[0] + sum[1];
        };
        auto parts_of = [&](const f32x16& a, h16x8 (&to)[2][NP]) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                h16x4 part[NP];
                split(v, part);
#pragma unroll
                for (int p = 0; p < NP; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[q / 2][p][4 * (q & 1) + i] = part[p][i];
            }
        };
        const int d = last ? 0 : next - e;
        h16x8 y[2][NP];
        const f32x16 A = times_of(rows, rows) * f;
        parts_of(A, y);
        const f32x16 B = A * ldexpf(cb, -2 * e) + times_of(y, y) * ldexpf(cc * f, -4 * e);
        parts_of(B, y);
        f32x16 v = times_of(y, x[0]) * ldexpf(f, d);
        const float own = ldexpf(ca, d);
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int p = NP - 1; p >= 0; --p)
                v[i] = fmaf((float)x[0][i / 8][p][i % 8], own, v[i]);
        if (last)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[0][i] = ldexpf(v[i] * kUnscale, -e);
        else
            parts_of(v, x[0]);
    };
    int next = e;
    for (int s = 0; s < steps; ++s) {
        e = next;
        bound = grown(bound, growth);
        next = shift_of(bound);
        const bool last = s + 1 == steps;
        if constexpr (NT == 1) {
            one_tile(last, e, next);
            continue;
        }
        const bool square = wave < RT;
        if (s > 0) __syncthreads();  // B has been read
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = row_of(t, q, lane & 3) * PITCH + (col & ~3);
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const h16x8 h = x[t][q / 2][p];
                    *reinterpret_cast<h16x4*>(&sm[p][at]) = quad_turn(q & 1 ? h.hi : h.lo);
                }
            }
        __syncthreads();
        if (square) symmetric(kCols, own_rows);
        __syncthreads();
        auto put = [&](float times) {
#pragma unroll
            for (int d = 0; d < HALF; ++d)
                if (mine(d)) {
                    const int t = across(d);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        h16x4 part[NP];
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = times * acc[d][4 * q + e];
                        split(v, part);
                        // run c of its 16 columns sits at 0, 2, 1, 3
                        const int c = (r32 >> 2) & 3;
                        const int at = row_of(t, q, lane & 3) * PITCH + 32 * wave +
                                       16 * (r32 >> 4) + 4 * (2 * (c & 1) + (c >> 1));
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            *reinterpret_cast<h16x4*>(&sm[p][run_of(t, q)]) = part[p];
                            if (d > 0) *reinterpret_cast<h16x4*>(&sm[p][at]) = quad_turn(part[p]);
                        }
                    }
                }
        };
        if (square) put(f);  // A
        __syncthreads();
        if (square) {
            symmetric(kRows, own_rows);
            const float own = ldexpf(cb, -2 * e), times = ldexpf(cc * f, -4 * e);
#pragma unroll
            for (int d = 0; d < HALF; ++d)
                if (mine(d))
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int at = run_of(across(d), q);
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[d][4 * q + i] *= times;
#pragma unroll
                        for (int p = NP - 1; p >= 0; --p) {
                            const h16x4 part = *reinterpret_cast<const h16x4*>(&sm[p][at]);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                acc[d][4 * q + i] = fmaf((float)part[i], own, acc[d][4 * q + i]);
                        }
                    }
        }
        __syncthreads();
        if (square) put(1.f);  // B
        __syncthreads();
        product(std::integral_constant<int, RT>{}, kRows, [](int d) { return d; },
                [&](int c, h16x8 (&b)[NP]) {
#pragma unroll
                    for (int p = 0; p < NP; ++p) b[p] = x[c / 2][c % 2][p];
                });
        const int d = last ? 0 : next - e;
        const float own = ldexpf(ca, d), times = ldexpf(f, d);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = times * acc[t][4 * q + i];
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        v[i] = fmaf((float)x[t][q / 2][p][4 * (q & 1) + i], own, v[i]);
                }
                if (last)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][4 * q + i] = ldexpf(v[i] * kUnscale, -e);
                else
                    keep(t, q, v);
            }
    }
    if (steps == 0) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][i] = ldexpf(acc[t][i], -e);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = row_of(t, i / 4, i % 4);
            const float v[1] = {acc[t][i]};
            if (row < k && col < r) pack_store<DT, 1>(out, at_of(row), v);
        }
}

// ------------------------------------------------------------ long matrices
// A matrix of at most 32 rows (or columns: its transpose), longer than the kernels
// above hold: products with float32 instructions, because its sums are short (as
// there) and it has little to compute.  One launch a step and no padding: a
// workgroup reduces the partial sums of A that the launch before left, forms
// T = ca I + cb A + cc A A, and takes its columns of X through X' = T X, adding
// up their part of the next A = X' X'^T.  The iterates are float32 [k, r], in their
// own range: no shift.  510 matrices of 755 x 5 157 us a call, one of 24 x 330 61, 20 of
// 32 x 1000 82 (as padded tiles 332, 80 and 126); bound by what a workgroup does before
// its first column (with 128 columns to each instead of 256, 382, 54 and 88).
struct Long {
    const void* G;
    void* out;
    float *X, *sums;        // [k, r]; partial sums of A, [parts, 32, 32]
    const float* before;    // those of the launch before
    const float4* norms;
    int nparts, m, n, parts;
    float ca, cb, cc, eps;
    bool first, step, last;  // X is still G's; there is a step to do; out instead of X
};

template <int DT>
__global__ void __launch_bounds__(256, 3) ortho_long(Long g) {
    constexpr int PITCH = 33;
    __shared__ float A[32 * PITCH], T[32 * PITCH], xs[4][32 * PITCH];
    const int lane = threadIdx.x & 63, r32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool tall = g.m > g.n;
    const int k = tall ? g.n : g.m, r = tall ? g.m : g.n;
    const long long z = blockIdx.y, base = z * g.m * g.n;
    float* X = g.X + base;
    // element 2 u + half of a column is what a lane gives to product u of 16
    float t[16];
    if (g.step) {
        const float* p = g.before + z * g.parts * 1024;
        for (int e = threadIdx.x; e < 1024; e += 256) {
            float s = 0.f;
            for (int i = 0; i < g.parts; ++i) s += p[i * 1024 + e];
            A[(e >> 5) * PITCH + (e & 31)] = s;
        }
        __syncthreads();
        if (wave == 0) {
            f32x16 c = {};
#pragma unroll
            for (int u = 0; u < 16; ++u) {  // A is symmetric
                const float a = A[r32 * PITCH + 2 * u + half];
                c = __builtin_amdgcn_mfma_f32_32x32x2f32(a, a, c, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 8 * (i / 4) + 4 * half + i % 4;
                T[row * PITCH + r32] = fmaf(g.cc, c[i], g.cb * A[row * PITCH + r32]) +
                                       (row == r32 ? g.ca : 0.f);
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 16; ++u) t[u] = T[r32 * PITCH + 2 * u + half];
    }
    Start s{1.f, 1.f, 0.f};
    if (g.first) s = start_of(g.norms + z * g.nparts, g.nparts, g.eps);
    f32x16 sum = {};
    const int tiles = (r + 31) / 32, t0 = tiles * blockIdx.x / g.parts,
              t1 = tiles * (blockIdx.x + 1) / g.parts;
    for (int tile = t0 + wave; tile < t1; tile += 4) {
        const int col = tile * 32 + r32;
        const bool live = col < r;
        auto of_g = [&](int row) { return base + (tall ? (long long)col * k + row : (long long)row * r + col); };
        float x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int row = 2 * u + half;
            x[u] = 0.f;
            if (live && row < k)
                x[u] = g.first ? (float)pack_load<DT, 1>(g.G, of_g(row)).e[0] * s.unit * s.inv
                               : X[(long long)row * r + col];
        }
        if (g.step) {
            f32x16 y = {};
#pragma unroll
            for (int u = 0; u < 16; ++u)
                if (2 * u < k) y = __builtin_amdgcn_mfma_f32_32x32x2f32(t[u], x[u], y, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 8 * (i / 4) + 4 * half + i % 4;
                const float one[1] = {y[i]};
                if (live && row < k) {
                    if (g.last)
                        pack_store<DT, 1>(g.out, of_g(row), one);
                    else
                        X[(long long)row * r + col] = y[i];
                }
                xs[wave][r32 * PITCH + row] = y[i];
            }
        } else {
#pragma unroll
            for (int u = 0; u < 16; ++u) xs[wave][r32 * PITCH + 2 * u + half] = x[u];
        }
        if (!g.last) {
            wave_sync();
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const float a = xs[wave][(2 * u + half) * PITCH + r32];
                sum = __builtin_amdgcn_mfma_f32_32x32x2f32(a, a, sum, 0, 0, 0);
            }
            wave_sync();
        }
    }
    if (g.last) return;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        xs[wave][(8 * (i / 4) + 4 * half + i % 4) * PITCH + r32] = sum[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 1024; e += 256) {
        const int at = (e >> 5) * PITCH + (e & 31);
        g.sums[(z * g.parts + blockIdx.x) * 1024 + e] = (xs[0][at] + xs[1][at]) + (xs[2][at] + xs[3][at]);
    }
}

// ------------------------------------------------------------------- the plan
// Sides are padded to whole tiles of 64.  (Above 64 to tiles of 128: five of 960 x 960
// 520 us, 26 of 448 x 448 416, 192 of 140 x 140 431, against 492, 365 and 282.)
int padded(int n) { return (n + 63) / 64 * 64; }

// Workgroups that share a matrix's norm.
int norm_parts(int m, int n) {
    return (int)std::min<long long>(kParts, ((long long)m * n + 16383) / 16384);
}

struct Plan {
    int k, r, kp, rp, parts;
    long long some;  // matrices at a time
    size_t xs;       // bytes of a matrix's parts
};
Plan plan_of(int N, int m, int n) {
    Plan p;
    p.k = std::min(m, n);
    p.r = std::max(m, n);
    p.kp = padded(p.k);
    p.rp = padded(p.r);
    p.xs = (size_t)p.kp * p.rp * 4;
    p.parts = norm_parts(m, n);
    const size_t each = 3 * p.xs;
    p.some = std::max<long long>(1, std::min<long long>({N, 32768, (long long)((1ull << 30) / each)}));
    return p;
}

template <int MODE, int OUT>
hipError_t product(const Product& g, int some, hipStream_t st) {
    // Tiles of 128, which read LDS and L2 half as much, where there is more than
    // one for every CU: 8 of 1024 x 1024 751 us against 794 with tiles of 64, two of
    // 2048 x 2048 1303 and 1548, 128 of 256 x 256 385 and 404, but 4 of 1024 x 1024
    // 564 and 471.
    // Of symmetric products, which have fewer, 128 x 64: they share the CUs more
    // evenly, and a wave below the diagonal has nothing to do: 16 of 1024 x 1024
    // 1408 us against 1467 with whole tiles, 64 of 512 x 512 851 and 881.
    auto tiles_of = [&](int side) {
        const long long ti = g.rows / side, tj = g.cols / side;
        return (int)(MODE == APPLY ? ti * tj : ti * (ti + 1) / 2);
    };
    auto go = [&](auto bm, auto bn) {
        constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value;
        const int tiles = tiles_of(BM) * (BM / BN);
        const long long all = tiles * (long long)some;
        const unsigned grid = (unsigned)((all + 7) / 8 * 8);
        ortho_product<BM, BN, MODE, OUT><<<grid, 256, 0, st>>>(g, tiles, all);
    };
    constexpr std::integral_constant<int, 64> n64{};
    constexpr std::integral_constant<int, 128> n128{};
    if (g.rows % 128 == 0 && g.cols % 128 == 0 && tiles_of(128) * (long long)some > 256)
        go(n128, std::integral_constant<int, MODE == APPLY ? 128 : 64>{});
    else
        go(n64, n64);
    return hipGetLastError();
}

// Sides up to 128; at most 32 rows or columns beside longer ones.
bool small_side(int m, int n) { return std::max(m, n) <= 128; }
bool long_side(int m, int n) { return std::min(m, n) <= 32; }

// A long matrix's workgroups, two tiles for each wave, and its memory: partial norms,
// partial sums of A twice, X.  At most 8192 matrices at a time.
int long_parts(int m, int n) { return std::min(16, (std::max(m, n) + 255) / 256); }
size_t long_bytes(int m, int n) {
    return kParts * sizeof(float4) + (2 * (size_t)long_parts(m, n) * 1024 + (size_t)m * n) * 4;
}
int long_some(int N) { return std::min(N, 8192); }

template <int DT>
hipError_t run_long(const void* G, void* X, int N, int m, int n, int steps, float ca, float cb,
                    float cc, float eps, char* ws, hipStream_t st) {
    const long long sz = (long long)m * n;
    const int most = long_some(N), parts = long_parts(m, n), norms = norm_parts(m, n);
    for (long long at = 0; at < N; at += most) {
        const int some = (int)std::min<long long>(most, N - at);
        float4* norm = (float4*)ws;
        float* sums = (float*)(norm + (size_t)most * kParts);
        const size_t each = (size_t)most * parts * 1024;
        Long g{};
        g.G = (const char*)G + at * sz * sizeof(elem_t<DT>);
        g.out = (char*)X + at * sz * sizeof(elem_t<DT>);
        g.X = sums + 2 * each;
        g.norms = norm;
        g.nparts = norms;
        g.m = m;
        g.n = n;
        g.parts = parts;
        g.ca = ca;
        g.cb = cb;
        g.cc = cc;
        g.eps = eps;
        ortho_norm<DT><<<dim3(norms, some), 256, 0, st>>>(g.G, norm, sz);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && steps == 0) {
            ortho_scaled<DT><<<dim3(parts, some), 256, 0, st>>>(g.G, g.out, norm, norms, sz, eps);
            e = hipGetLastError();
        }
        for (int s = 0; steps > 0 && s <= steps && e == hipSuccess; ++s) {
            g.first = s <= 1;
            g.step = s > 0;
            g.last = s == steps;
            g.before = sums + (s & 1 ? 0 : each);
            g.sums = sums + (s & 1 ? each : 0);
            ortho_long<DT><<<dim3(parts, some), 256, 0, st>>>(g);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DT>
hipError_t run_small(const void* G, void* X, int N, int m, int n, int steps, float ca, float cb,
                     float cc, float eps, hipStream_t st) {
    const int side = std::max(m, n);
    const Growth growth{fabsf(ca), fabsf(cb), fabsf(cc)};
    const long long sz = (long long)m * n * sizeof(elem_t<DT>);
    // a launch has fewer than 2^32 threads
    for (long long at = 0; at < N; at += 1 << 23) {
        const unsigned some = (unsigned)std::min<long long>(1 << 23, N - at);
        const void* g = (const char*)G + at * sz;
        void* x = (char*)X + at * sz;
        auto go = [&](auto p, auto rt) {
            constexpr int P = decltype(p)::value, RT = decltype(rt)::value;
            ortho_small<P, RT, DT><<<some, 2 * P, 0, st>>>(g, x, m, n, steps, ca, cb, cc, eps, growth);
        };
        constexpr std::integral_constant<int, 1> one{};
        constexpr std::integral_constant<int, 2> two{};
        constexpr std::integral_constant<int, 3> three{};
        constexpr std::integral_constant<int, 4> four{};
        const int rt = (std::min(m, n) + 31) / 32;
        if (side <= 16) {
            ortho_tiny<DT><<<some, 64, 0, st>>>(g, x, m, n, steps, ca, cb, cc, eps, growth);
        } else if (side <= 32) {
            go(std::integral_constant<int, 32>{}, one);
        } else if (side <= 64) {
            constexpr std::integral_constant<int, 64> p{};
            rt == 1 ? go(p, one) : go(p, two);
        } else {
            constexpr std::integral_constant<int, 128> p{};
            rt == 1 ? go(p, one) : rt == 2 ? go(p, two) : rt == 3 ? go(p, three) : go(p, four);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DT>
hipError_t run(const void* G, void* X, int N, int m, int n, int steps, float ca, float cb, float cc,
               float eps, char* ws, hipStream_t st) {
    if (small_side(m, n)) return run_small<DT>(G, X, N, m, n, steps, ca, cb, cc, eps, st);
    if (long_side(m, n))
        return run_long<DT>(G, X, N, m, n, steps, ca, cb, cc, eps, ws, st);
    const Plan p = plan_of(N, m, n);
    const long long sz = (long long)m * n;
    const Growth growth{fabsf(ca), fabsf(cb), fabsf(cc)};
    for (long long at = 0; at < N; at += p.some) {
        const int some = (int)std::min<long long>(p.some, N - at);
        const void* g = (const char*)G + at * sz * sizeof(elem_t<DT>);
        void* out = (char*)X + at * sz * sizeof(elem_t<DT>);
        float4* parts = (float4*)ws;
        Shift* shifts = (Shift*)(parts + p.some * kParts);
        char* q = ws + (size_t)p.some * (kParts + 16) * sizeof(float4);
        // X, A and B take turns in three buffers of X's size
        const long long xn = (long long)p.kp * p.rp, an = (long long)p.kp * p.kp;
        h16* buf[3];
        for (int i = 0; i < 3; ++i) buf[i] = (h16*)(q + i * p.some * p.xs);
        ortho_norm<DT><<<dim3(p.parts, some), 256, 0, st>>>(g, parts, sz);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (steps == 0) {
            const unsigned wg = (unsigned)std::min<long long>(256, (sz + 255) / 256);
            ortho_scaled<DT><<<dim3(wg, some), 256, 0, st>>>(g, out, parts, p.parts, sz, eps);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            continue;
        }
        const int gr = m > n ? p.rp : p.kp, gc = m > n ? p.kp : p.rp;
        ortho_start<DT><<<dim3(gc / 64, gr / 64, some), 256, 0, st>>>(
            g, Panels{buf[0], xn, p.kp}, parts, p.parts, shifts, m, n, eps);
        e = hipGetLastError();
        for (int s = 0; s < steps && e == hipSuccess; ++s) {
            const Panels x{buf[0], xn, p.kp}, A{buf[1], an, p.kp}, B{buf[2], an, p.kp},
                y{buf[1], xn, p.kp};  // over A
            e = product<GRAM, -1>({x, x, A, nullptr, p.kp, p.kp, p.rp, m, n, shifts, growth, 0.f, 1.f},
                                  some, st);
            if (e == hipSuccess)
                e = product<POLY, -1>({A, A, B, nullptr, p.kp, p.kp, p.kp, m, n, shifts, growth, cb, cc},
                                      some, st);
            const Product last{B, x, y, out, p.kp, p.rp, p.kp, m, n, shifts, growth, ca, 1.f};
            if (e == hipSuccess)
                e = s + 1 < steps ? product<APPLY, -1>(last, some, st)
                                  : product<APPLY, DT>(last, some, st);
            std::swap(buf[0], buf[1]);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t ortho_workspace(int N, int m, int n) {
    if (small_side(m, n)) return 256;
    if (long_side(m, n)) return long_some(N) * long_bytes(m, n);
    const Plan p = plan_of(N, m, n);
    return (size_t)p.some * ((kParts + 16) * sizeof(float4) + 3 * p.xs);
}

hipError_t launch_ortho(const void* G, void* X, int N, int m, int n, int steps, float ca, float cb,
                        float cc, float eps, int dtype, void* ws, hipStream_t st) {
    if (dtype == 0) return run<0>(G, X, N, m, n, steps, ca, cb, cc, eps, (char*)ws, st);
    if (dtype == 1) return run<1>(G, X, N, m, n, steps, ca, cb, cc, eps, (char*)ws, st);
    return run<2>(G, X, N, m, n, steps, ca, cb, cc, eps, (char*)ws, st);
}

}  // namespace deeppcr
