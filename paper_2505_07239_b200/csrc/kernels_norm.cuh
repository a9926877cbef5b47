// Norms of the heads of shared queries and keys, with the position rotation in the same pass (comet_norm_rotate):
//     x  ->  rotate(gain * x / sqrt(mean(x^2) + eps)),   x a row, i.e. one head of one token,
// composed of Section 2.1's primitives.  Every value is masked and opened once, however many products it enters; D is the length
// of a row, f the fixed point, i the party, tr_b the local truncation by b bits, dv the same by a divisor, sums over j:
//   m_j = open(x_j - U_j),  Q = sum U_j^2 from the dealer:  sq_i = Q_i + sum 2 m_j U_ij + i sum m_j^2
//   s_i = dv(sq_i, D 2^f) + i eps                                                        the mean square
//   Newton for 1 / sqrt(s), y <- y (3 - s y^2) / 2.  The first step, from a public guess g, is local:
//     y_i = tr_{f+1}(g (3 i 2^f - tr_f(s_i g^2)));  every further one is three of Eq. 1:
//     p = tr_f(y y),  w = 3 - tr_f(s p),  y = tr_{f+1}(y w)                               y and s opened once for two products
//   n_j = tr_f(y x_j), x_j's opening used again with the dealer's U_j v (v the mask of y)
//   t_j = tr_f(n_j gain_j)                                                               n and the gain masked and opened
//   (a, b) -> (tr_f(a cos - b sin), tr_f(b cos + a sin)), the angles public: a local step
// One pass: a thread has both parties' words of its elements, which is the exchange, and a row's words stay in registers from
// the first load to the last store.
//
// What bounds it: memory, and the time that a row's registers and shared memory are held.  With gain 8 words per element and party,
// five in (x, U, U v, and the gain's A and C), three out (two messages and the result), 128 bytes an element; beaver_mul_kernel moves
// the same mix at 0.95 of the copy rate.  The root is a chain of 3 (steps - 1) dependent products between a row's first loads and
// its last stores, 0.17 us a step, so what is needed behind it is asked for before it begins: UV, A and C wait in shared
// memory, x's opening and U in registers.  And what a CTA asks for first, x, U and its rows' own words, an earlier CTA has asked the
// L2 for, three CTAs of the SM ahead: the memory works while chains run, and a row is held for less time.
// Measured, ten steps, gain and rotation: 512 tokens x 64 heads x 128 99.7 us, 582 MB, 5.8 TB/s, 0.89 of the copy rate (two steps: 91.5 us,
// 0.90), x 64 60 us (0.81), x 256 178 us (0.97); 32 tokens x 64 heads x 128 13 us, one token 7.5 us, of which the chain 1.6; rows of 4096
// words without rotation, 203 of them, 26 us, 0.63 (two waves of clusters, and the second is not full), 512 of them 62 us (0.67), one 7.9 us.
// What it took, 512 tokens x 64 heads: every warp with its row's chain to itself 135 us (2050 instructions a row, 1500 now), one warp for
// all rows of a CTA 115, a row's own words asked for before the elements 109.  CTAs of four rows: of two or eight 115.  Five CTAs an SM at
// 96 registers: four at 128 125, six at 80 (16 bytes spilled) 111; with 100 bytes spilled 129.  Left out in scratch builds: the chain
// 103, the row's own words 105, the predicates of ragged rows 107.  No difference: another warp of the CTA for the chain, CTAs of the
// first wave begun 1.5 us apart.  Threads dealt to a tile's words whatever the rows' length, instead of whole lanes or warps to a row:
// x 160 189 -> 138 us, x 254, all rotated, 312 -> 229, x 126 147 -> 121 (the latter two in accesses of 16 bytes, too, their pairs
// through shared memory).  The L2 asked ahead (the figures before are without it): 108.5 -> 99.7, x 256 200 -> 178, x 160 133 -> 124,
// without gain 86.7 -> 75.8, 512 rows of 4096 67 -> 62; the rows' own words alone 103.5, x and U alone 106.5; UV, A and C too 103.8; two and
// four CTAs ahead 98.5 and 100.4 (x 64 62.1 and 59.4); five with UV, A and C 107, eight 119; four CTAs an SM 104.5, six 102.4.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "pdl.cuh"

namespace comet {

typedef unsigned long long u64;

namespace norm {
constexpr int MAX_STEPS = 24, MAX_DIM = 8192;
constexpr int TILE_THREADS = 128;                    // at most, of a CTA that has whole rows of up to TILE_DIM words
constexpr int TILE_DIM = 4 * TILE_THREADS, TILE_ROWS = 16;
constexpr int CLUSTER_THREADS = 256, MAX_CLUSTER = 8;   // at most, of a CTA of a cluster that has one; its CTAs
constexpr int TILE_CTAS = 5, CLUSTER_CTAS = 3;       // on an SM
constexpr int TILE_AHEAD = 3, CLUSTER_AHEAD = 2;     // how many CTAs of an SM ahead the L2 is asked for rows
static_assert(4 * MAX_CLUSTER * CLUSTER_THREADS >= MAX_DIM, "a row fits a cluster");
constexpr int PLACE_BYTES = 6 * 2 * 16;              // of shared memory that a thread's four words of UV, A and C of both parties take
__host__ __device__ constexpr int words(int steps) { return 6 * steps - 3; }       // a row's own, from the dealer
__host__ __device__ constexpr int openings(int steps) { return 3 * steps - 1; }    // a row's own, in its message
constexpr int row_bytes(int steps) { return 2 * (words(steps) + openings(steps)) * 8; }    // of shared memory, both parties' of both
// Rows of a tile: a thread has four words, a lane pair of one warp a row's root.
__host__ __device__ constexpr int tile_rows(int quads) { return TILE_THREADS / quads < TILE_ROWS ? TILE_THREADS / quads : TILE_ROWS; }
}  // namespace norm

struct NormArgs {
    const u64* X[2];             // row (t, h) begins at t * x_stride + h * dim
    const u64* U[2]; const u64* row_words[2]; const u64* UV[2];
    const u64* gain[2]; const u64* gain_mask[2]; const u64* A[2]; const u64* C[2];   // gain[0] null: none
    const u64* cos; const u64* sin;                                                  // [table_rows, half]
    const int32_t* positions;                                                        // per token
    u64* M[2]; u64* S[2]; u64* Dm[2]; u64* G[2];                                     // messages
    u64* Z[2];
    int32_t* bad_index;
    long long x_stride;
    u64 guess, first, eps, divisor;      // first = guess^2 / 2^f, divisor = dim * 2^f
    int rows, heads, q_heads, dim;       // rows = tokens * heads; q_heads 0: one gain for all heads
    int half, interleaved, table_rows;   // half = pairs that are rotated, 0: none
    int f, steps, divisor_bits;          // divisor_bits: its logarithm, or -1
    int exchange;                        // tiles: a pair's members are different threads', see norm_tile_kernel
    int ahead;                           // rows from a CTA's or cluster's to those that it asks the L2 for
};

// v >> bits for 1 <= bits <= 32: two instructions, where a shift by any count takes twice as many.
__device__ __forceinline__ u64 norm_shift(u64 v, int bits) {
    const unsigned lo = (unsigned)v, hi = (unsigned)(v >> 32);
    return (u64)__funnelshift_rc(hi, 0u, bits) << 32 | __funnelshift_rc(lo, hi, bits);
}

// Where a thread's four words of a row lie.  A row is dim / 2 pairs, (2P, 2P + 1), or (P, P + half) for the P < half where
// halves are rotated against each other; a thread has two pairs.  VEC: two accesses of 16 bytes, else four of 8.  Neighbouring
// threads' accesses lie side by side: a thread's pairs are neighbours where a pair's members lie apart, else they lie apart
// themselves.  (As neighbours throughout, 32-byte sectors are touched twice: rows of 4096 words, 203 tokens, 38.9 us.)
struct NormPlace {
    int pair[2], at[4];          // elements: first and second of either pair (VEC: at[0] and at[2] of the two accesses)
    bool has[2];                 // either pair exists (VEC: either access)
    bool split;                  // VEC: the accesses are the firsts and the seconds, not the pairs
    bool turned[2];              // either pair is rotated
};
template <bool VEC>
__device__ __forceinline__ NormPlace norm_place(int quad, int dim, int half, int interleaved) {
    NormPlace p;
    const int pairs = dim / 2, apart = VEC && !interleaved ? half : 0;       // (VEC: half is even)
    p.split = 2 * quad < apart;
    const int rest = (pairs - apart + 1) / 2;                                // threads that have the other pairs
    p.pair[0] = p.split ? 2 * quad : quad + apart / 2;
    p.pair[1] = p.pair[0] + (p.split ? 1 : rest);
    p.has[0] = p.split || p.pair[0] < apart + rest;
    p.has[1] = p.has[0] && p.pair[1] < pairs;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int P = p.pair[k];
        p.turned[k] = p.has[k] && P < half;
        const bool far = !interleaved && P < half;
        p.at[2 * k] = far ? P : 2 * P;
        p.at[2 * k + 1] = far ? P + half : 2 * P + 1;
    }
    if (p.split) p.at[2] = p.pair[0] + half;
    return p;
}
// The words of access k (VEC; else of pair k), through L1: what several rows read.
template <bool VEC>
__device__ __forceinline__ void norm_load2(const u64* row, const NormPlace& p, int k, u64 v[2]) {
    if (VEC) {
        const ulonglong2 w = __ldg(reinterpret_cast<const ulonglong2*>(row + p.at[2 * k]));
        v[0] = w.x;
        v[1] = w.y;
    } else {
        v[0] = __ldg(row + p.at[2 * k]);
        v[1] = __ldg(row + p.at[2 * k + 1]);
    }
}
template <bool VEC>
__device__ __forceinline__ void norm_store2(u64* row, const NormPlace& p, int k, const u64 v[2]) {
    if (VEC) {
        __stcs(reinterpret_cast<ulonglong2*>(row + p.at[2 * k]), make_ulonglong2(v[0], v[1]));
    } else {
        __stcs(row + p.at[2 * k], v[0]);
        __stcs(row + p.at[2 * k + 1], v[1]);
    }
}
// All four words, in the order of the accesses, read once.
template <bool VEC>
__device__ __forceinline__ void norm_load(const u64* row, const NormPlace& p, u64 v[4]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v[2 * k] = v[2 * k + 1] = 0ull;
        if (!p.has[k]) continue;
        if (VEC) {
            const ulonglong2 w = __ldcs(reinterpret_cast<const ulonglong2*>(row + p.at[2 * k]));
            v[2 * k] = w.x;
            v[2 * k + 1] = w.y;
        } else {
            v[2 * k] = __ldcs(row + p.at[2 * k]);
            v[2 * k + 1] = __ldcs(row + p.at[2 * k + 1]);
        }
    }
}
template <bool VEC>
__device__ __forceinline__ void norm_store(u64* row, const NormPlace& p, const u64 v[4]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (p.has[k]) norm_store2<VEC>(row, p, k, v + 2 * k);
}

// Public angles of a thread's two pairs.  A position outside the tables is not followed: its pairs become zero.
template <bool VEC>
__device__ __forceinline__ void norm_angles(const NormArgs& a, int token, const NormPlace& p, u64 c[2], u64 s[2]) {
    c[0] = c[1] = s[0] = s[1] = 0ull;
    if (!p.turned[0] && !p.turned[1]) return;
    const int at = __ldg(a.positions + token);
    if (at < 0 || at >= a.table_rows) {
        if (a.bad_index) *a.bad_index = 1;
        return;
    }
    const size_t o = (size_t)at * a.half;
    if (p.split) {                                   // (half is even)
        const ulonglong2 cc = __ldg(reinterpret_cast<const ulonglong2*>(a.cos + o + p.pair[0]));
        const ulonglong2 ss = __ldg(reinterpret_cast<const ulonglong2*>(a.sin + o + p.pair[0]));
        c[0] = cc.x; c[1] = cc.y; s[0] = ss.x; s[1] = ss.y;
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (p.turned[k]) {
                c[k] = __ldg(a.cos + o + p.pair[k]);
                s[k] = __ldg(a.sin + o + p.pair[k]);
            }
    }
}
// Party 1's shares are held negated: its truncation of a share x = -n is -(n >> b), the plain shift of what is held.
__device__ __forceinline__ void norm_turn(u64& x, u64& y, u64 c, u64 s, int f) {
    const u64 one = norm_shift(x * c - y * s, f), two = norm_shift(y * c + x * s, f);
    x = one;
    y = two;
}
__device__ __forceinline__ void norm_rotate_words(u64 v[4], const NormPlace& p, const u64 c[2], const u64 s[2], int f) {
    if (p.split) {
        norm_turn(v[0], v[2], c[0], s[0], f);
        norm_turn(v[1], v[3], c[1], s[1], f);
    } else {
        if (p.turned[0]) norm_turn(v[0], v[1], c[0], s[0], f);
        if (p.turned[1]) norm_turn(v[2], v[3], c[1], s[1], f);
    }
}

// The shares of the root of a row's mean square: even lanes work for party 0, odd ones for party 1, and a pair of lanes exchanges
// its openings.  All of party 1's is held negated here, its words w too, which makes its truncation the plain shift:
//   sq: the party's share of the sum of squares without Q;  w: its words of the row;  o: where its openings go, 3 steps - 1
//   words (`write`: pairs of lanes that share a row let one of them do that).
// Returns the opened y - v.  A chain of 3 steps products, each waiting for the one before, while the CTA waits for it: what a
// step does not have to wait for is made ahead of it.
__device__ __forceinline__ u64 norm_opened(u64 mine, int party) {
    const u64 theirs = __shfl_xor_sync(0xffffffffu, mine, 1);
    return party ? theirs - mine : mine - theirs;
}
__device__ __forceinline__ u64 norm_root(const NormArgs& a, u64 sq, const u64* __restrict__ w, u64* __restrict__ o, bool write, int party) {
    const int f = a.f;
    const u64 only = party ? ~0ull : 0ull, three = only & 3ull << f;     // the public terms are party 1's
    u64 s = sq + w[0];
    s = a.divisor_bits >= 0 ? s >> a.divisor_bits : s / a.divisor;
    s -= only & a.eps;
    u64 y = norm_shift(a.guess * (0ull - three - norm_shift(s * a.first, f)), f + 1);
    const u64 t0 = s - w[1], ds = norm_opened(t0, party), sa = w[1] - (only & ds);
    if (write) o[0] = t0;
    const u64* next = w + 2;
    u64* out = o + 1;
#pragma unroll 1
    for (int k = 1; k < a.steps; ++k) {
        const u64 ya = next[0], yy = next[1], pb = next[2], wb = next[4], yw = next[5], ap = next[3] + ds * pb, ya2 = ya + ya;
        const u64 t1 = y - ya, d = norm_opened(t1, party), own = only & d;
        const u64 p = norm_shift(yy + d * (ya2 - own), f);
        const u64 t2 = p - pb, g = norm_opened(t2, party);
        const u64 x = 0ull - three - norm_shift(ap + g * sa, f);
        const u64 t3 = x - wb, h = norm_opened(t3, party);
        y = norm_shift(yw + d * wb + h * (ya - own), f + 1);
        if (write) {
            out[0] = t1;
            out[1] = t2;
            out[2] = t3;
        }
        next += 6;
        out += 3;
    }
    const u64 t4 = y - *next;
    if (write) *out = t4;
    return norm_opened(t4, party);
}

__device__ __forceinline__ void norm_fetch8(void* dst, const u64* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void norm_fetch16(void* dst, const u64* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void norm_fetch_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Asks the L2 for words that are read later: 16-byte aligned, an even number of them.
__device__ __forceinline__ void norm_ask(const u64* words, int count) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(words), "r"(count * 8) : "memory");
}

// A thread's four words of a row: `open` before the root, `finish` after it.  What `finish` reads is on its way to this thread's
// places in shared memory meanwhile (nobody else reads them): UV, A and C of both parties.
template <bool VEC>
struct NormQuad {
    NormPlace p;
    size_t at;                   // the row in the dense tensors
    u64 m[4], U[2][4];
    ulonglong2* mine;            // pair k of array j, party i: mine[((3 i + j) 2 + k) stride]
    int stride;

    __device__ __forceinline__ void fetch(int array, const u64* row) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            ulonglong2* to = mine + (array * 2 + k) * stride;
            if (!p.has[k]) continue;
            if (VEC) {
                norm_fetch16(to, row + p.at[2 * k]);
            } else {
                norm_fetch8(&to->x, row + p.at[2 * k]);
                norm_fetch8(&to->y, row + p.at[2 * k + 1]);
            }
        }
    }
    __device__ __forceinline__ void fetched(int array, int k, u64 v[2]) const {
        const ulonglong2 w = mine[(array * 2 + k) * stride];
        v[0] = w.x;
        v[1] = w.y;
    }

    // Loads, the first message, and both parties' part of the sum of squares.
    // `beside` runs while the loads are under way.
    template <typename F>
    __device__ __forceinline__ void open(const NormArgs& a, int row, int token, int head, int quad, ulonglong2* place, int place_stride,
                                         u64 sq[2], F&& beside) {
        p = norm_place<VEC>(quad, a.dim, a.half, a.interleaved | a.exchange);
        at = (size_t)row * a.dim;
        mine = place;
        stride = place_stride;
        const size_t x_at = (size_t)token * a.x_stride + (size_t)head * a.dim;
        u64 x[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            norm_load<VEC>(a.X[i] + x_at, p, x[i]);
            norm_load<VEC>(a.U[i] + at, p, U[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fetch(3 * i, a.UV[i] + at);
            if (a.gain[0]) {
                fetch(3 * i + 1, a.A[i] + at);
                fetch(3 * i + 2, a.C[i] + at);
            }
        }
        beside();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[i][k] -= U[i][k];
            norm_store<VEC>(a.M[i] + at, p, x[i]);
        }
        sq[0] = sq[1] = 0ull;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = x[0][k] + x[1][k];                            // the exchange
            sq[0] += m[k] * U[0][k];
            sq[1] += m[k] * (2 * U[1][k] + m[k]);
        }
        sq[0] *= 2;
    }

    // root: the opened y - v; v0, n1: party 0's share of v and party 1's, negated.  `tells`: this row writes the message of its
    // gain.  An access at a time: the registers of both at once would not fit.
    // Leaves the words in U, party 1's negated; `rotate` makes the results of them.
    __device__ __forceinline__ void finish(const NormArgs& a, int head, bool tells, u64 root, u64 v0, u64 n1) {
        const size_t g_at = a.q_heads > 0 && head >= a.q_heads ? a.dim : 0;
        norm_fetch_wait();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (!p.has[k]) continue;
            u64 *x0 = U[0] + 2 * k, *x1 = U[1] + 2 * k, t[2];
            fetched(0, k, t);
#pragma unroll
            for (int j = 0; j < 2; ++j) x0[j] = norm_shift(t[j] + m[2 * k + j] * v0 + root * x0[j], a.f);
            fetched(3, k, t);
#pragma unroll
            for (int j = 0; j < 2; ++j) x1[j] = norm_shift(m[2 * k + j] * n1 - t[j] - root * (x1[j] + m[2 * k + j]), a.f);          // negated
            if (!a.gain[0]) continue;
            u64 A[2][2], d[2], e[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fetched(3 * i + 1, k, A[i]);
                u64 o[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    o[j] = i ? 0ull - (x1[j] + A[1][j]) : x0[j] - A[0][j];
                    d[j] = i ? d[j] + o[j] : o[j];
                }
                norm_store2<VEC>(a.Dm[i] + at, p, k, o);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                norm_load2<VEC>(a.gain[i] + g_at, p, k, t);
                norm_load2<VEC>(a.gain_mask[i] + g_at, p, k, b);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    t[j] -= b[j];
                    e[j] = i ? e[j] + t[j] : t[j];
                }
                if (tells) norm_store2<VEC>(a.G[i] + g_at, p, k, t);
            }
            fetched(5, k, t);
#pragma unroll
            for (int j = 0; j < 2; ++j) x1[j] = norm_shift(0ull - t[j] - d[j] * b[j] - e[j] * (A[1][j] + d[j]), a.f);
            norm_load2<VEC>(a.gain_mask[0] + g_at, p, k, b);
            fetched(2, k, t);
#pragma unroll
            for (int j = 0; j < 2; ++j) x0[j] = norm_shift(t[j] + d[j] * b[j] + e[j] * A[0][j], a.f);
        }
    }
    __device__ __forceinline__ void rotate(const NormArgs& a, int token) {
        u64 c[2], s[2];
        if (a.half) {
            norm_angles<VEC>(a, token, p, c, s);
#pragma unroll
            for (int i = 0; i < 2; ++i) norm_rotate_words(U[i], p, c, s, a.f);
        }
        store(a);
    }
    __device__ __forceinline__ void store(const NormArgs& a) {
#pragma unroll
        for (int k = 0; k < 4; ++k) U[1][k] = 0ull - U[1][k];
#pragma unroll
        for (int i = 0; i < 2; ++i) norm_store<VEC>(a.Z[i] + at, p, U[i]);
    }
    // The same where a pair's members may be any two threads' of a row, whose words lie in shared memory.
    __device__ __forceinline__ void rotate_from(const NormArgs& a, int token, const u64* row0, const u64* row1) {
        if (p.has[0] && p.at[0] < 2 * a.half) {
            const int at_table = __ldg(a.positions + token);
            const bool inside = at_table >= 0 && at_table < a.table_rows;
            if (!inside && a.bad_index) *a.bad_index = 1;
            const size_t o = (size_t)(inside ? at_table : 0) * a.half;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = p.at[k];
                if (!p.has[k >> 1] || j >= 2 * a.half) continue;
                const bool second = j >= a.half;
                const int pair = second ? j - a.half : j, other = second ? pair : j + a.half;
                const u64 c = inside ? __ldg(a.cos + o + pair) : 0ull, t = inside ? __ldg(a.sin + o + pair) : 0ull, s = second ? t : 0ull - t;
                U[0][k] = norm_shift(U[0][k] * c + row0[other] * s, a.f);
                U[1][k] = norm_shift(U[1][k] * c + row1[other] * s, a.f);
            }
        }
        store(a);
    }
};

// Whether a row writes the message of its gain: of the first token the first query head's and the first key head's.
__device__ __forceinline__ bool norm_tells(const NormArgs& a, int token, int head) {
    return token == 0 && (head == 0 || head == a.q_heads);
}
// The sum over a warp's lanes of both parties' sq: even lanes add up party 0's, odd lanes party 1's.
__device__ __forceinline__ u64 norm_lane_sum(const u64 sq[2], int party) {
    u64 sum = (party ? sq[1] : sq[0]) + __shfl_xor_sync(0xffffffffu, party ? sq[0] : sq[1], 1);
#pragma unroll
    for (int o = 2; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}

// The words of a CTA's rows, `total` of them behind one another, on their way to shared memory, party 1's negated: the first N a
// thread are asked for before anything else and put there when the other loads are under way.
template <int N>
struct NormWords {
    u64 v[N][2];
    __device__ __forceinline__ void load(const NormArgs& a, int row, int total, int threads) {
        const size_t at = (size_t)row * norm::words(a.steps);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = threadIdx.x + j * threads;
            if (k < total)
                for (int i = 0; i < 2; ++i) v[j][i] = __ldcs(a.row_words[i] + at + k);
        }
    }
    __device__ __forceinline__ void store(const NormArgs& a, int row, int total, int threads, u64* w0, u64* w1) const {
        const size_t at = (size_t)row * norm::words(a.steps);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = threadIdx.x + j * threads;
            if (k < total) {
                w0[k] = v[j][0];
                w1[k] = 0ull - v[j][1];
            }
        }
        for (int k = threadIdx.x + N * threads; k < total; k += threads) {
            w0[k] = __ldcs(a.row_words[0] + at + k);
            w1[k] = 0ull - __ldcs(a.row_words[1] + at + k);
        }
    }
};

// Rows of up to TILE_DIM words: a tile of as many as its threads cover, a thread per four words whatever the rows' length; one warp
// works out all of the tile's roots, a pair of lanes a row.  Accesses lie side by side in a row, so the members of a rotated pair are one
// thread's if they are neighbours, or if all of a row of a multiple of four words is rotated, halves against each other; else (`exchange`)
// the rows go through shared memory once more.
template <bool VEC>
__global__ void __launch_bounds__(norm::TILE_THREADS, norm::TILE_CTAS)
norm_tile_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ u64 sums[norm::TILE_THREADS][2], root[norm::TILE_ROWS];
    const int quads = (a.dim + 3) / 4, tile = norm::tile_rows(quads);
    const int count = norm::words(a.steps), sent = norm::openings(a.steps);
    ulonglong2* const places = reinterpret_cast<ulonglong2*>(norm_smem);
    u64* const words = reinterpret_cast<u64*>(norm_smem + norm::PLACE_BYTES * blockDim.x);                // [party][row][count]
    u64* const opened = words + 2 * tile * count;                                                         // [party][row][sent]
    u64* const rowed = opened + 2 * tile * sent;                                                          // exchange: [party][row][dim]
    const int first = blockIdx.x * tile, rows = min(tile, a.rows - first);
    const int sub = threadIdx.x / quads, quad = threadIdx.x - sub * quads;
    const bool live = sub < rows;
    const int row = first + (live ? sub : 0);                // threads past the last row have none of its words and write nothing
    const int token = row / a.heads, head = row - token * a.heads;
    pdl_wait();
    pdl_launch_dependents();
    NormWords<3> early;
    early.load(a, first, rows * count, blockDim.x);
    NormQuad<VEC> q;
    u64 sq[2];
    q.open(a, row, token, head, live ? quad : a.dim, places + threadIdx.x, blockDim.x, sq, [&] {
        early.store(a, first, rows * count, blockDim.x, words, words + tile * count);
        if (VEC && threadIdx.x < 32 && a.ahead < a.rows - first) {       // a lane for a row of a party
            const int next = first + a.ahead, many = min(tile, a.rows - next), r = threadIdx.x >> 1, i = threadIdx.x & 1;
            if (r < many) {
                const int at_token = (next + r) / a.heads;
                norm_ask(a.X[i] + (size_t)at_token * a.x_stride + (size_t)(next + r - at_token * a.heads) * a.dim, a.dim);
            }
            if (r == 0) {
                const size_t at = (size_t)next * a.dim, own = (size_t)next * count;
                norm_ask(a.U[i] + at, many * a.dim);
                const u64* w = a.row_words[i] + own;         // 8-byte aligned: the even words between
                const int odd = (int)(reinterpret_cast<uintptr_t>(w) >> 3 & 1);
                norm_ask(w + odd, (many * count - odd) & ~1);
            }
        }
    });
    sums[threadIdx.x][0] = sq[0];
    sums[threadIdx.x][1] = 0ull - sq[1];
    __syncthreads();
    if (threadIdx.x < 32) {
        // lanes 2r and 2r + 1 work for row r; the lanes beyond help with the sums
        const int width = 2 << (32 - __clz(tile - 1));       // lanes that the rows take, a power of two (tile 1: 2)
        const int lane = threadIdx.x, of = lane & (width - 1), party = lane & 1, r = min(of >> 1, tile - 1);
        u64 sum = 0ull;
        for (int k = lane / width; k < quads; k += 32 / width) sum += sums[r * quads + k][party];
        for (int o = width; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const bool mine = lane < 2 * rows;
        const u64 opened_root = norm_root(a, sum, words + (party * tile + r) * count, opened + (party * tile + r) * sent, mine, party);
        if (mine) root[r] = opened_root;
    }
    __syncthreads();
    for (int i = 0; i < 2; ++i)
        for (int k = threadIdx.x; k < rows * sent; k += blockDim.x) {
            const u64 t = opened[i * tile * sent + k];
            __stcs(a.S[i] + (size_t)first * sent + k, i ? 0ull - t : t);
        }
    if (live) {
        q.finish(a, head, norm_tells(a, token, head), root[sub], words[(sub + 1) * count - 1], words[(tile + sub + 1) * count - 1]);
        if (!a.exchange) q.rotate(a, token);
    }
    if (!a.exchange) return;
    u64 *const row0 = rowed + sub * a.dim, *const row1 = row0 + tile * a.dim;
    if (live)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (q.p.has[k >> 1]) {
                row0[q.p.at[k]] = q.U[0][k];
                row1[q.p.at[k]] = q.U[1][k];
            }
    __syncthreads();
    if (live) q.rotate_from(a, token, row0, row1);
}

// Longer rows: a cluster of CTAs per row, a thread per four words.  Every warp's sums are written to every CTA, one barrier of the cluster
// behind them, and every CTA works out the root for itself.  (Sums per CTA, read from each other's behind a barrier: one row of 4096 words
// 8.45 us instead of 7.9, of 8192 8.7 instead of 8.2, 203 rows alike, 512 of 4096 60.7 instead of 61.9.)
template <bool VEC>
__global__ void __launch_bounds__(norm::CLUSTER_THREADS, norm::CLUSTER_CTAS)
norm_cluster_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ u64 partial[norm::MAX_CLUSTER * norm::CLUSTER_THREADS / 32][2], root;        // every warp's of the row
    ulonglong2* const places = reinterpret_cast<ulonglong2*>(norm_smem);
    u64* const words = reinterpret_cast<u64*>(norm_smem + norm::PLACE_BYTES * blockDim.x);               // [party][count]
    uint32_t rank, cluster;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, party = threadIdx.x & 1, warps = blockDim.x >> 5;
    const int count = norm::words(a.steps), sent = norm::openings(a.steps);
    u64* const opened = words + 2 * count;                                                               // [party][sent]
    const int row = (int)(blockIdx.x / cluster), token = row / a.heads, head = row - token * a.heads;
    // (a CTA's shared memory is written to by the others when it has begun)
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    pdl_wait();
    pdl_launch_dependents();
    NormWords<1> early;
    early.load(a, row, count, blockDim.x);
    NormQuad<VEC> q;
    u64 sq[2];
    q.open(a, row, token, head, (int)(rank * blockDim.x + threadIdx.x), places + threadIdx.x, blockDim.x, sq, [&] {
        early.store(a, row, count, blockDim.x, words, words + count);
        if (VEC && threadIdx.x < 4 && threadIdx.x % cluster == rank && a.ahead < a.rows - row) {
            const int next = row + a.ahead, at_token = next / a.heads, i = threadIdx.x & 1;
            if (threadIdx.x < 2) norm_ask(a.X[i] + (size_t)at_token * a.x_stride + (size_t)(next - at_token * a.heads) * a.dim, a.dim);
            else norm_ask(a.U[i] + (size_t)next * a.dim, a.dim);
        }
    });
    u64 sum = norm_lane_sum(sq, party);
    if (cluster > 1) {
        // a warp's sums go to every CTA of the cluster, a lane each
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (lane < 2 * cluster) {
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there)
                         : "r"((uint32_t)__cvta_generic_to_shared(&partial[rank * warps + warp][party])), "r"(lane >> 1));
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(sum) : "memory");
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        if (lane < 2) partial[warp][party] = sum;
        __syncthreads();
    }
    if (warp == 0) {
        sum = 0ull;
        for (int k = 0; k < (int)cluster * warps; ++k) sum += partial[k][party];
        const u64 opened_root = norm_root(a, party ? 0ull - sum : sum, words + party * count, opened + party * sent, lane < 2, party);
        if (lane == 0) root = opened_root;
    }
    __syncthreads();
    if (warp == 0 && rank == 0)
        for (int i = 0; i < 2; ++i)
            for (int k = lane; k < sent; k += 32) {
                const u64 t = opened[i * sent + k];
                __stcs(a.S[i] + (size_t)row * sent + k, i ? 0ull - t : t);
            }
    q.finish(a, head, norm_tells(a, token, head), root, words[count - 1], words[2 * count - 1]);
    q.rotate(a, token);
}

// Rotation without a norm: a thread per four words of a row, both parties.
template <bool VEC>
__global__ void __launch_bounds__(256)
rotate_kernel(const __grid_constant__ NormArgs a, unsigned quads) {
    pdl_wait();
    pdl_launch_dependents();
    const u64 all = (u64)a.rows * quads, stride = (u64)gridDim.x * blockDim.x;
    for (u64 t = (u64)blockIdx.x * blockDim.x + threadIdx.x; t < all; t += stride) {
        const int row = (int)(t / quads), token = row / a.heads, head = row - token * a.heads;
        const NormPlace p = norm_place<VEC>((int)(t - (u64)row * quads), a.dim, a.half, a.interleaved);
        u64 x[2][4], c[2], s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) norm_load<VEC>(a.X[i] + (size_t)token * a.x_stride + (size_t)head * a.dim, p, x[i]);
        norm_angles<VEC>(a, token, p, c, s);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            auto negate = [&] {
#pragma unroll
                for (int k = 0; k < 4; ++k) x[1][k] = 0ull - x[1][k];
            };
            if (i) negate();
            norm_rotate_words(x[i], p, c, s, a.f);
            if (i) negate();
            norm_store<VEC>(a.Z[i] + (size_t)row * a.dim, p, x[i]);
        }
    }
}

}  // namespace comet
