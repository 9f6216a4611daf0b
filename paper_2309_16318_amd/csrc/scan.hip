// Gated linear recurrence: x_l = s_l x_{l-1} + r_l channel by channel, its
// backward pass and the single row.
//
// A row maps the state x_in to s x_in + r, so a run of rows maps it to
// A x_in + H with A the product of its multipliers and H its end from zero
// (the diagonal form of the chunk maps P x_in + q of the block solves).  The
// backward pass is the same recurrence on kap_l = s_l lam_l, the adjoint as
// it leaves row l: kap_l = s_l kap_{l+1} + s_l g_l, walked from the last row.  da
// is formed from the states as the forward pass stored them, rounded to the
// sequences' type, which errs by 1.4 times a rounding; forming the float32 states
// again from a and u would read two sequences more beside the five or six that the
// pass moves.
//
// Bound by memory: every input is read once and every output written once.  A
// workgroup of S waves takes a tile of S * R rows by 64 packs of V channels;
// each thread loads its R rows of a pack at once into registers, folds them to
// (A, H), gets its own x_in from the waves before it through LDS, and walks its
// rows again from there, so a value takes its recurrence's order whatever the
// tile.  Where the channels alone do not fill the chip a sequence's tiles run
// at once: each publishes its (A, H) and takes its x_in from those before it.
#include <type_traits>

#include "elem.h"
#include "internal.h"

namespace deeppcr {
namespace {

// Tiles of 64 or 256 rows, packs of 4 and 1 or 4 earlier tiles per wave were
// measured too (sigmoid gates short): one sequence of 65536 rows of 1024 bfloat16 channels, forward
// and backward, 320, 287, 413, 299 and 275 us against 263, 8 of 2048 x 2048 159,
// 169, 200, 156 and 158 against 158, a prompt of 8192 x 2048 40, 42, 48, 40 and
// 38 against 39.
constexpr int R = 16;              // rows per thread
constexpr int S = 8;               // most waves per workgroup
constexpr int T = R * S;           // rows per tile
constexpr int kBack = 2;           // earlier tiles that a wave folds
constexpr int kSuper = kBack * S;  // tiles between two published states
typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
constexpr unsigned long long kEmpty = ~0ull;  // nothing published yet

// The multiplier s, and the factor q of u, of one element: to float32 precision
// of their own whatever the sequences' type, because the states, x_last and dx0
// that they make are float32.
template <int GATE, int DT>
__device__ __forceinline__ void gate_of(float a, float* s, float* q) {
    if constexpr (GATE == 1) {
        sigmoid_pair<DT == 1 ? FINE_BF16 : FINE>(a, s, q);
    } else {
        *s = a;
        *q = 1.f;
    }
}

// A x + H; exactly H at x = 0, also where a long product A has overflowed (a
// multiplier that is infinite or NaN itself makes H NaN).
__device__ __forceinline__ float through(float A, float H, float x) {
    return x == 0.f ? H : fmaf(A, x, H);
}

// A pair as published: one 64-bit word, written and read whole, so that it
// needs no flag beside it.  No pair has kEmpty's bits, because its NaNs are
// made the canonical one.
__device__ __forceinline__ void publish(unsigned long long* p, float A, float H) {
    const unsigned nan = 0x7fc00000u;
    const unsigned a = A == A ? __float_as_uint(A) : nan, h = H == H ? __float_as_uint(H) : nan;
    __hip_atomic_store(p, (unsigned long long)h << 32 | a, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long peek(const unsigned long long* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Waits for a word of a tile with a smaller ticket, given as it was at first:
// that tile's workgroup is running, and what it still waits for has a smaller
// ticket again.  A board that another call writes to at the same time (which the
// interface forbids) may never have the word: the wait ends after kPatience
// looks, some ten seconds, with NaN.
constexpr int kPatience = 1 << 24;
__device__ __forceinline__ void await(const unsigned long long* p, unsigned long long v, float* A,
                                      float* H) {
    for (int i = 0; v == kEmpty && i < kPatience; ++i) {
        __builtin_amdgcn_s_sleep(1);
        v = peek(p);
    }
    // kEmpty itself is a pair of NaN
    *A = __uint_as_float((unsigned)v);
    *H = __uint_as_float((unsigned)(v >> 32));
}

// How tiles talk: pairs [chunks, F, V] of every tile, states [supers, F, V]
// behind every kSuper-th, and the next ticket of each group of 64 packs.
// (Tickets of all groups from one counter: 8 us of a prompt's 44, its atomics
// being done one after the other.)
struct Board {
    unsigned long long *pairs, *states;
    unsigned* tickets;
};
constexpr int kApart = 32;       // words between two groups' tickets, a cache line
// Tiles run at once where there are more than kWalk of them to a sequence and at
// most kMaxGroups groups.  Forward and backward of bfloat16, all at once against
// one after the other: 128 groups of 16 tiles 162 us against 290, 256 of 16 287
// and 325, 512 of 8 266 and 274, 1024 of 4 261 and 267, 512 of 2 69 and 63; of
// float32 8 groups of 8 34 and 76, of 2 34 and 28, 64 of 4 (forward) 16 and 16.
constexpr int kMaxGroups = 512, kWalk = 3;

__global__ void __launch_bounds__(256) scan_clear(unsigned long long* p, long long n,
                                                  unsigned* tickets) {
    // n is even: two words to a store
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 2;
    for (long long i = at; i < n; i += (long long)gridDim.x * 512)
        __builtin_nontemporal_store(u64x2{kEmpty, kEmpty}, reinterpret_cast<u64x2*>(p + i));
    if (at < 2 * kMaxGroups) tickets[at / 2 * kApart] = 0;
}

// SPLIT: one tile per workgroup, by ticket, sequences' tiles side by side;
// else a workgroup walks all tiles of its channels.
template <int DT, int V, int GATE, bool BWD, bool SPLIT>
__global__ void __launch_bounds__(64 * S, 4) scan_tile(ScanArgs k, Board bd, int groups, int chunks) {
    __shared__ float sm[2][S][2][64 * V];   // (A, H) of the waves, two tiles in turn
    __shared__ float lb[S][2][64 * V];      // of the tiles before, as each wave folded them
    __shared__ float start[64 * V];
    __shared__ unsigned ticket;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    // A group's tiles in the order in which its workgroups get their tickets;
    // the groups one further every round, so that no XCD (workgroups go to them
    // in turn) reads the same columns, which lie in few channels of its L2.
    const int grp = SPLIT ? (blockIdx.x + blockIdx.x / groups) % groups : blockIdx.x;
    int c0 = 0;
    if constexpr (SPLIT) {
        if (threadIdx.x == 0) ticket = atomicAdd(bd.tickets + grp * kApart, 1u);
        __syncthreads();
        c0 = __builtin_amdgcn_readfirstlane(ticket);
        if (c0 >= chunks) return;  // only on a board that another call cleared meanwhile
    }
    const int c1 = SPLIT ? c0 + 1 : chunks;
    // pack f of all sequences' channels: sequence b, channels c .. c+V-1
    const int cw = k.w / V, F = k.B * cw;
    const int f = grp * 64 + lane;
    const bool live = f < F;
    const int fc = live ? f : F - 1;
    const int b = fc / cw, c = (fc - b * cw) * V;
    const int n = k.lengths ? min(max(k.lengths[b], 0), k.L) : k.L;
    const long long r0 = (long long)b * k.L;
    const long long fv = (long long)fc * V;

    float K[V];  // the state at the tile's start
#pragma unroll
    for (int v = 0; v < V; ++v) K[v] = 0.f;
    const float* first = BWD ? k.g_last : k.x0;
    if (first && c0 == 0 && (!SPLIT || wave == 0))
#pragma unroll
        for (int v = 0; v < V; ++v) K[v] = first[fv + v];

    for (int ch = c0; ch < c1; ++ch) {
        const int p0 = ch * T + wave * R;  // position in walking order
        // row i of the thread, and whether this lane's sequence has it
        auto row = [&](int i) { return BWD ? k.L - 1 - p0 - i : p0 + i; };
        auto inside = [&](int i) { return BWD ? row(i) >= 0 : row(i) < k.L; };
        auto has = [&](int i) { return row(i) < n && (!BWD || row(i) >= 0); };
        Raw<DT, V> ra[R], ru[R], rx[R], rg[R];
        {
            // rows outside are read at the sequence's ends and not used
            const bool some = (BWD ? row(R - 1) < n && row(0) >= 0 : row(0) < n);
            if (__any(some)) {
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const long long l = r0 + min(max(row(i), 0), k.L - 1);
                    ra[i].load(k.a, l * k.lda + c);
                    if (!BWD || GATE == 1) ru[i].load(k.u, l * k.ldu + c);
                    if (BWD) {
                        rg[i].load(k.g, l * k.ldg + c);
                        const long long m = r0 + min(max(row(i) - 1, 0), k.L - 1);
                        rx[i].load(k.x, m * k.w + c);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < R; ++i) ra[i] = ru[i] = rx[i] = rg[i] = Raw<DT, V>{};
            }
        }
        float A[V], H[V];
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = 1.f, H[v] = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s, q;
                gate_of<GATE, DT>(ra[i].get(v), &s, &q);
                const float r = BWD ? s * rg[i].get(v) : q * ru[i].get(v);
                if (has(i)) {
                    A[v] *= s;
                    H[v] = fmaf(s, H[v], r);
                }
            }
        const int turn = ch & 1;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            sm[turn][wave][0][lane * V + v] = A[v];
            sm[turn][wave][1][lane * V + v] = H[v];
        }
        __syncthreads();
        if constexpr (SPLIT) {
            const int sp = ch / kSuper, at = ch % kSuper;
            const long long tw = (long long)F * V;
            float tA[V], tH[V];
            if (wave == waves - 1) {  // the tile's own pair
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    tA[v] = 1.f;
                    tH[v] = 0.f;
                    for (int j = 0; j < waves; ++j) {
                        const float a = sm[turn][j][0][lane * V + v];
                        tH[v] = through(a, sm[turn][j][1][lane * V + v], tH[v]);
                        tA[v] *= a;
                    }
                    if (live && ch > 0) publish(bd.pairs + ch * tw + fv + v, tA[v], tH[v]);
                }
            }
            // kBack tiles per wave of those between the last published state
            // and this tile, all asked for before one is waited for
            const unsigned long long* board = bd.pairs + (sp * kSuper + kBack * wave) * tw + fv;
            const int mine = min(max(at - kBack * wave, 0), kBack);
            unsigned long long word[kBack][V], prev[V];
#pragma unroll
            for (int j = 0; j < kBack; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (live && j < mine) word[j][v] = peek(board + j * tw + v);
            if (wave == 0 && sp > 0 && live)
#pragma unroll
                for (int v = 0; v < V; ++v) prev[v] = peek(bd.states + (sp - 1) * tw + fv + v);
#pragma unroll
            for (int v = 0; v < V; ++v) A[v] = 1.f, H[v] = 0.f;
#pragma unroll
            for (int j = 0; j < kBack; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (live && j < mine) {
                        float a, h;
                        await(board + j * tw + v, word[j][v], &a, &h);
                        H[v] = through(a, h, H[v]);
                        A[v] *= a;
                    }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                lb[wave][0][lane * V + v] = A[v];
                lb[wave][1][lane * V + v] = H[v];
            }
            if (wave == 0)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float none;
                    if (sp > 0 && live)
                        await(bd.states + (sp - 1) * tw + fv + v, prev[v], &none, &K[v]);
                    start[lane * V + v] = K[v];
                }
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v) {
                K[v] = start[lane * V + v];
                for (int j = 0; j < min(waves, (at + kBack - 1) / kBack); ++j)
                    K[v] = through(lb[j][0][lane * V + v], lb[j][1][lane * V + v], K[v]);
                if (wave == waves - 1 && live) {
                    const float end = through(tA[v], tH[v], K[v]);
                    // the first tile's pair is its end, so that no other tile reads x0
                    if (ch == 0) publish(bd.pairs + fv + v, 0.f, end);
                    if (at == kSuper - 1)
                        publish(bd.states + sp * tw + fv + v, 0.f, end);
                }
            }
        }
        float h[V];  // the state at the thread's first row
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h[v] = K[v];
            for (int j = 0; j < waves; ++j) {
                if (j == wave) h[v] = K[v];
                if (!SPLIT || j < wave)
                    K[v] = through(sm[turn][j][0][lane * V + v], sm[turn][j][1][lane * V + v], K[v]);
            }
            if (SPLIT) h[v] = K[v];
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            ra[i].renew();
            if (BWD) rg[i].renew();
            if (!BWD) ru[i].renew();
            float o0[V], o1[V], xp[V];
            if constexpr (BWD) {
#pragma unroll
                for (int v = 0; v < V; ++v) xp[v] = rx[i].get(v);
                if (row(i) == 0)
#pragma unroll
                    for (int v = 0; v < V; ++v) xp[v] = k.x0 ? k.x0[fv + v] : 0.f;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s, q;
                gate_of<GATE, DT>(ra[i].get(v), &s, &q);
                if constexpr (BWD) {
                    const float lam = h[v] + rg[i].get(v);
                    float d = xp[v];
                    if (GATE == 1) d = (d - ru[i].get(v)) * s * q;
                    o0[v] = has(i) ? lam * d : 0.f;
                    o1[v] = has(i) ? lam * q : 0.f;
                    if (has(i)) h[v] = s * lam;
                } else {
                    if (has(i)) h[v] = fmaf(s, h[v], q * ru[i].get(v));
                    o0[v] = has(i) ? h[v] : 0.f;
                }
            }
            if (inside(i) && live) {
                pack_store<DT, V>(k.out0, (r0 + row(i)) * k.w + c, o0);
                if (BWD) pack_store<DT, V>(k.out1, (r0 + row(i)) * k.w + c, o1);
            }
        }
        if (k.last && ch == chunks - 1 && wave == waves - 1 && live)
#pragma unroll
            for (int v = 0; v < V; ++v) k.last[fv + v] = h[v];
    }
}

// V channels of a sequence per thread.
template <int DT, int V, int GATE>
__global__ void __launch_bounds__(256) scan_step(const void* a, long long lda, const void* u,
                                                 long long ldu, const float* state,
                                                 float* state_out, void* x, int B, int w) {
    const int f = blockIdx.x * 256 + threadIdx.x, cw = w / V;
    if (f >= B * cw) return;
    const int b = f / cw, c = (f - b * cw) * V;
    const long long at = (long long)b * w + c;
    const Pack<DT, V> pa = pack_load<DT, V>(a, b * lda + c), pu = pack_load<DT, V>(u, b * ldu + c);
    const Pack<0, V> ps = pack_load<0, V>(state, at);
    float out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float s, q;
        gate_of<GATE, DT>((float)pa.e[v], &s, &q);
        out[v] = fmaf(s, ps.e[v], q * (float)pu.e[v]);
    }
    pack_store<0, V>(state_out, at, out);
    if (x) pack_store<DT, V>(x, at, out);
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

size_t up(size_t n) { return (n + 255) / 256 * 256; }
long long chunks_of(int L) { return ((long long)L + T - 1) / T; }
bool at_once(long long groups, long long chunks) {
    return chunks > kWalk && groups <= kMaxGroups && groups * chunks < (1 << 22);
}
// Pairs and states, 8 bytes per channel each, if some packs' tiles run at once.
size_t board_words(int B, int L, int w) {
    const long long ch = chunks_of(L), channels = (long long)B * w;
    if (!at_once((channels + 63) / 64, ch) &&
        !(w % 2 == 0 && at_once((channels / 2 + 63) / 64, ch)))
        return 0;
    return ((size_t)(ch + ch / kSuper) * B * w + 1) / 2 * 2;
}

// Whether all rows may be read in packs of V.
bool in_packs(const ScanArgs& k, int dtype, int V) {
    const uintptr_t mask = (dtype == 0 ? 4 : 2) * V - 1;
    auto ok = [&](const void* p, long long ld) { return !p || (((uintptr_t)p & mask) == 0 && ld % V == 0); };
    return k.w % V == 0 && ok(k.a, k.lda) && ok(k.u, k.ldu) && ok(k.g, k.ldg);
}

template <int DT, int V, int GATE, bool BWD>
hipError_t tiles(const ScanArgs& k, hipStream_t st) {
    const long long F = (long long)k.B * (k.w / V), groups = (F + 63) / 64;
    const long long chunks = chunks_of(k.L);
    if (at_once(groups, chunks)) {
        Board bd;
        bd.tickets = (unsigned*)k.ws;
        bd.pairs = (unsigned long long*)((char*)k.ws + kMaxGroups * kApart * 4);
        bd.states = bd.pairs + chunks * F * V;
        const long long n = (long long)board_words(k.B, k.L, k.w);
        const long long wg = (n / 2 + 255) / 256;
        scan_clear<<<(unsigned)(wg < 2 ? 2 : wg < 1024 ? wg : 1024), 256, 0, st>>>(bd.pairs, n, bd.tickets);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        scan_tile<DT, V, GATE, BWD, true>
            <<<(unsigned)(groups * chunks), 64 * S, 0, st>>>(k, bd, (int)groups, (int)chunks);
    } else {
        const int waves = k.L >= T ? S : (k.L + R - 1) / R;
        scan_tile<DT, V, GATE, BWD, false>
            <<<(unsigned)groups, 64 * waves, 0, st>>>(k, Board{}, (int)groups, (int)chunks);
    }
    return hipGetLastError();
}

}  // namespace

size_t scan_workspace(int B, int L, int w) { return kMaxGroups * kApart * 4 + up(board_words(B, L, w) * 8); }

hipError_t launch_scan(bool bwd, const ScanArgs& k, int gate, int dtype, hipStream_t st) {
    return by_type(dtype, gate, [&](auto dt, auto gt) {
        constexpr int DT = decltype(dt)::value, GATE = decltype(gt)::value;
        if constexpr (DT != 0) {
            if (in_packs(k, dtype, 2))
                return bwd ? tiles<DT, 2, GATE, true>(k, st) : tiles<DT, 2, GATE, false>(k, st);
        }
        return bwd ? tiles<DT, 1, GATE, true>(k, st) : tiles<DT, 1, GATE, false>(k, st);
    });
}

hipError_t launch_scan_step(const void* a, long long lda, const void* u, long long ldu,
                            const float* state, float* state_out, void* x, int B, int w, int gate,
                            int dtype, hipStream_t st) {
    // packs of 4 where the rows allow it, and there are threads enough without
    ScanArgs k{};
    k.a = a;
    k.u = u;
    k.lda = lda;
    k.ldu = ldu;
    k.w = w;
    const bool packs = (long long)B * w >= 4 * 256 * 256 && in_packs(k, dtype, 4);
    const long long n = (long long)B * (packs ? w / 4 : w);
    const unsigned grid = (unsigned)((n + 255) / 256);
    return by_type(dtype, gate, [&](auto dt, auto gt) {
        constexpr int DT = decltype(dt)::value, GATE = decltype(gt)::value;
        if (packs)
            scan_step<DT, 4, GATE><<<grid, 256, 0, st>>>(a, lda, u, ldu, state, state_out, x, B, w);
        else
            scan_step<DT, 1, GATE><<<grid, 256, 0, st>>>(a, lda, u, ldu, state, state_out, x, B, w);
        return hipGetLastError();
    });
}

}  // namespace deeppcr
