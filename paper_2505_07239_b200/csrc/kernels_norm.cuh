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
// What bounds it: memory.  With gain 8 words per element and party, five in (x, U, U v, and the gain's A and C), three out
// (two messages and the result), 128 bytes an element.  The root is a chain of 3 (steps - 1) dependent products between a row's
// first loads and its last stores, so what is needed behind it is asked for before it begins.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "pdl.cuh"

namespace comet {

typedef unsigned long long u64;

namespace norm {
constexpr int MAX_STEPS = 24, MAX_DIM = 8192;
constexpr int GROUP_WARPS = 4;                       // warps of a CTA that has a row per warp, or several
constexpr int GROUP_DIM = 128;                       // longest row of one warp: four words a lane
constexpr int MAX_CTA_QUADS = 256;                   // longer rows: a thread per four words, a cluster per row
__host__ __device__ constexpr int words(int steps) { return 6 * steps - 3; }       // a row's own, from the dealer
__host__ __device__ constexpr int openings(int steps) { return 3 * steps - 1; }    // a row's own, in its message
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
};

__device__ __forceinline__ u64 norm_negate(u64 v, int party) { return party ? 0ull - v : v; }
__device__ __forceinline__ u64 norm_trunc(u64 v, int party, int bits) { return norm_negate(norm_negate(v, party) >> bits, party); }

// Where a thread's four words of a row lie: pairs P and P + 1, P even, of the row's dim / 2.  A pair is (2P, 2P + 1), or
// (P, P + half) where halves are rotated against each other.  VEC: two accesses of 16 bytes, else four of 8.
struct NormPlace {
    int pair, at[4];             // elements: first and second of either pair (VEC: at[0] and at[2] of the two accesses)
    bool has[2];                 // either pair exists (VEC: either access)
    bool split;                  // VEC: the accesses are the firsts and the seconds, not the pairs
    bool turned[2];              // either pair is rotated
};
template <bool VEC>
__device__ __forceinline__ NormPlace norm_place(int quad, int dim, int half, int interleaved) {
    NormPlace p;
    p.pair = 2 * quad;
    p.has[0] = p.pair < dim / 2;
    p.has[1] = p.pair + 1 < dim / 2;
    p.split = !interleaved && p.pair < half;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int P = p.pair + k;
        p.turned[k] = P < half;
        const bool apart = !interleaved && P < half;
        p.at[2 * k] = apart ? P : 2 * P;
        p.at[2 * k + 1] = apart ? P + half : 2 * P + 1;
    }
    if (VEC && p.split) p.at[2] = p.pair + half;     // half is even: both pairs are apart
    return p;
}
// STREAMED: read once; else through L1, for what several rows read.
template <bool VEC, bool STREAMED>
__device__ __forceinline__ void norm_load(const u64* row, const NormPlace& p, u64 v[4]) {
    if (VEC) {
        ulonglong2 a = make_ulonglong2(0ull, 0ull), b = a;
        const ulonglong2 *pa = reinterpret_cast<const ulonglong2*>(row + p.at[0]), *pb = reinterpret_cast<const ulonglong2*>(row + p.at[2]);
        if (p.has[0]) a = STREAMED ? __ldcs(pa) : __ldg(pa);
        if (p.has[1]) b = STREAMED ? __ldcs(pb) : __ldg(pb);
        v[0] = a.x;
        v[1] = p.split ? b.x : a.y;
        v[2] = p.split ? a.y : b.x;
        v[3] = b.y;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = !p.has[k >> 1] ? 0ull : STREAMED ? __ldcs(row + p.at[k]) : __ldg(row + p.at[k]);
    }
}
template <bool VEC>
__device__ __forceinline__ void norm_store(u64* row, const NormPlace& p, const u64 v[4]) {
    if (VEC) {
        if (p.has[0]) __stcs(reinterpret_cast<ulonglong2*>(row + p.at[0]), make_ulonglong2(v[0], p.split ? v[2] : v[1]));
        if (p.has[1]) __stcs(reinterpret_cast<ulonglong2*>(row + p.at[2]), make_ulonglong2(p.split ? v[1] : v[2], v[3]));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (p.has[k >> 1]) __stcs(row + p.at[k], v[k]);
    }
}

// Public angles of a thread's two pairs.  A position outside the tables is not followed: its pairs become zero.
template <bool VEC>
__device__ __forceinline__ void norm_angles(const NormArgs& a, int token, const NormPlace& p, u64 c[2], u64 s[2]) {
    c[0] = c[1] = s[0] = s[1] = 0ull;
    if (!p.turned[0]) return;
    const int at = __ldg(a.positions + token);
    if (at < 0 || at >= a.table_rows) {
        if (a.bad_index) *a.bad_index = 1;
        return;
    }
    const size_t o = (size_t)at * a.half + p.pair;
    if (VEC) {                                       // half is even
        const ulonglong2 cc = __ldg(reinterpret_cast<const ulonglong2*>(a.cos + o)), ss = __ldg(reinterpret_cast<const ulonglong2*>(a.sin + o));
        c[0] = cc.x; c[1] = cc.y; s[0] = ss.x; s[1] = ss.y;
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (p.turned[k]) {
                c[k] = __ldg(a.cos + o + k);
                s[k] = __ldg(a.sin + o + k);
            }
    }
}
__device__ __forceinline__ void norm_rotate_words(u64 v[4], const NormPlace& p, const u64 c[2], const u64 s[2], int party, int f) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const u64 x = v[2 * k], y = v[2 * k + 1];
        const u64 one = norm_trunc(x * c[k] - y * s[k], party, f), two = norm_trunc(y * c[k] + x * s[k], party, f);
        v[2 * k] = p.turned[k] ? one : x;
        v[2 * k + 1] = p.turned[k] ? two : y;
    }
}

// The shares of the root of a row's mean square, on even lanes party 0's, on odd lanes party 1's (sq: that party's share of the
// sum of squares without Q).  `w` holds the row's words, [party][words(steps)]; the openings take the place of words that have been
// read: the first openings(steps) of each party are then its message.  Every pair of lanes computes the same; `write` for one.
// Returns the opened y - v; *v_own becomes the party's share of v.  All lanes of the warp take part.
__device__ __forceinline__ u64 norm_other(u64 v) { return __shfl_xor_sync(0xffffffffu, v, 1); }
__device__ __forceinline__ u64 norm_root(const NormArgs& a, u64 sq, u64* w, bool write, int party, u64* v_own) {
    const int f = a.f;
    const u64 three = party ? 3ull << f : 0ull;
    w += party * norm::words(a.steps);
    u64 sum = norm_negate(sq + w[0], party);
    sum = a.divisor_bits >= 0 ? sum >> a.divisor_bits : sum / a.divisor;
    const u64 s = norm_negate(sum, party) + (party ? a.eps : 0ull);
    u64 y = norm_trunc(a.guess * (three - norm_trunc(s * a.first, party, f)), party, f + 1);
    const u64 sa = w[1];
    u64 mine = s - sa;
    const u64 ds = mine + norm_other(mine);
    __syncwarp();
    if (write) w[0] = mine;
    const u64* next = w + 2;
    u64* out = w + 1;                // stays behind `next`
    for (int k = 1; k < a.steps; ++k) {
        const u64 ya = next[0], yy = next[1], pb = next[2], apb = next[3], wb = next[4], yw = next[5];
        next += 6;
        const u64 oy = y - ya, d = oy + norm_other(oy);
        const u64 p = norm_trunc(yy + d * (ya + ya + (party ? d : 0ull)), party, f);
        const u64 op = p - pb, g = op + norm_other(op);
        const u64 x = three - norm_trunc(apb + ds * pb + g * (sa + (party ? ds : 0ull)), party, f);
        const u64 ow = x - wb, h = ow + norm_other(ow);
        y = norm_trunc(yw + d * wb + h * (ya + (party ? d : 0ull)), party, f + 1);
        __syncwarp();
        if (write) {
            out[0] = oy;
            out[1] = op;
            out[2] = ow;
        }
        out += 3;
    }
    *v_own = *next;
    mine = y - *v_own;
    __syncwarp();
    if (write) *out = mine;
    return mine + norm_other(mine);
}

__device__ __forceinline__ void norm_fetch_word(u64* dst, const u64* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void norm_fetch_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// A thread's four words of a row: `open` before the root, `finish` after it.
template <bool VEC>
struct NormQuad {
    NormPlace p;
    size_t at;                   // the row in the dense tensors
    u64 m[4], U[2][4], UV[2][4], A[2][4], C[2][4], c[2], s[2];

    // Loads, the first message, and both parties' part of the sum of squares.
    __device__ __forceinline__ void open(const NormArgs& a, int row, int token, int head, int quad, u64 sq[2]) {
        p = norm_place<VEC>(quad, a.dim, a.half, a.interleaved);
        at = (size_t)row * a.dim;
        const size_t x_at = (size_t)token * a.x_stride + (size_t)head * a.dim;
        u64 x[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            norm_load<VEC, true>(a.X[i] + x_at, p, x[i]);
            norm_load<VEC, true>(a.U[i] + at, p, U[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            norm_load<VEC, true>(a.UV[i] + at, p, UV[i]);
            if (a.gain[0]) {
                norm_load<VEC, true>(a.A[i] + at, p, A[i]);
                norm_load<VEC, true>(a.C[i] + at, p, C[i]);
            }
        }
        if (a.half) norm_angles<VEC>(a, token, p, c, s);
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

    // root: the opened y - v; v: both parties' shares of v.  `tells`: this row writes the message of its gain.
    __device__ __forceinline__ void finish(const NormArgs& a, int head, bool tells, u64 root, const u64 v[2]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            U[0][k] = norm_trunc(UV[0][k] + m[k] * v[0] + root * U[0][k], 0, a.f);
            U[1][k] = norm_trunc(UV[1][k] + m[k] * v[1] + root * (U[1][k] + m[k]), 1, a.f);
        }
        if (a.gain[0]) {
            const size_t g_at = a.q_heads > 0 && head >= a.q_heads ? a.dim : 0;
            u64 b[2][4], e[4], g[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                norm_load<VEC, false>(a.gain_mask[i] + g_at, p, b[i]);
                norm_load<VEC, false>(a.gain[i] + g_at, p, g);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    g[k] -= b[i][k];
                    e[k] = i ? e[k] + g[k] : g[k];
                }
                if (tells) norm_store<VEC>(a.G[i] + g_at, p, g);
            }
            u64 d[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    U[i][k] -= A[i][k];
                    d[k] = i ? d[k] + U[i][k] : U[i][k];
                }
                norm_store<VEC>(a.Dm[i] + at, p, U[i]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                U[0][k] = norm_trunc(C[0][k] + d[k] * b[0][k] + e[k] * A[0][k], 0, a.f);
                U[1][k] = norm_trunc(C[1][k] + d[k] * b[1][k] + e[k] * (A[1][k] + d[k]), 1, a.f);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (a.half) norm_rotate_words(U[i], p, c, s, i, a.f);
            norm_store<VEC>(a.Z[i] + at, p, U[i]);
        }
    }
};

// Whether a row writes the message of its gain: of the first token the first query head's and the first key head's.
__device__ __forceinline__ bool norm_tells(const NormArgs& a, int token, int head) {
    return token == 0 && (head == 0 || head == a.q_heads);
}

// Rows of up to GROUP_DIM words: GROUP lanes each, four words a lane.
template <int GROUP, bool VEC>
__global__ void __launch_bounds__(32 * norm::GROUP_WARPS, 4)
norm_group_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ u64 norm_smem[];
    const int sub = threadIdx.x / GROUP, lane = threadIdx.x % GROUP, party = threadIdx.x & 1;
    const int count = norm::words(a.steps), sent = norm::openings(a.steps);
    u64* const w = norm_smem + sub * 2 * count;
    const long long r = (long long)blockIdx.x * (32 * norm::GROUP_WARPS / GROUP) + sub;
    const bool live = r < a.rows;
    const int row = (int)(live ? r : a.rows - 1);            // groups past the last row have none of its words and write nothing
    const int token = row / a.heads, head = row - token * a.heads;
    pdl_wait();
    pdl_launch_dependents();
    for (int i = 0; i < 2; ++i)
        for (int k = lane; k < count; k += GROUP) norm_fetch_word(w + i * count + k, a.row_words[i] + (size_t)row * count + k);
    NormQuad<VEC> q;
    u64 sq[2];
    q.open(a, row, token, head, live ? lane : a.dim, sq);
    // even lanes keep party 0's sum, odd lanes party 1's
    u64 sum = (party ? sq[1] : sq[0]) + norm_other(party ? sq[0] : sq[1]);
#pragma unroll
    for (int o = 2; o < GROUP; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    norm_fetch_wait();
    __syncwarp();
    u64 mine;
    const u64 root = norm_root(a, sum, w, lane < 2, party, &mine), theirs = norm_other(mine);
    const u64 v[2] = {party ? theirs : mine, party ? mine : theirs};
    q.finish(a, head, live && norm_tells(a, token, head), root, v);
    __syncwarp();
    if (live)
        for (int i = 0; i < 2; ++i)
            for (int k = lane; k < sent; k += GROUP) a.S[i][(size_t)row * sent + k] = w[i * count + k];
}

// Longer rows: a cluster of CTAs per row, a thread per four words.
template <bool VEC>
__global__ void __launch_bounds__(norm::MAX_CTA_QUADS, 2)
norm_cluster_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ u64 norm_smem[];
    __shared__ u64 partial[norm::MAX_CTA_QUADS / 32][2], cta_sum[2], told[3];
    uint32_t rank, cluster;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, party = threadIdx.x & 1, warps = blockDim.x >> 5;
    const int count = norm::words(a.steps), sent = norm::openings(a.steps);
    const int row = (int)(blockIdx.x / cluster), token = row / a.heads, head = row - token * a.heads;
    pdl_wait();
    pdl_launch_dependents();
    if (warp == 0)
        for (int i = 0; i < 2; ++i)
            for (int k = lane; k < count; k += 32) norm_fetch_word(norm_smem + i * count + k, a.row_words[i] + (size_t)row * count + k);
    NormQuad<VEC> q;
    u64 sq[2];
    q.open(a, row, token, head, (int)(rank * blockDim.x + threadIdx.x), sq);
    u64 sum = (party ? sq[1] : sq[0]) + norm_other(party ? sq[0] : sq[1]);
#pragma unroll
    for (int o = 2; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane < 2) partial[warp][party] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = 0ull;
        for (int k = 0; k < warps; ++k) sum += partial[k][party];
        if (lane < 2) cta_sum[party] = sum;
    }
    if (cluster > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (warp == 0) {
            sum = 0ull;
            const uint32_t from = (uint32_t)__cvta_generic_to_shared(&cta_sum[party]);
            for (uint32_t k = 0; k < cluster; ++k) {
                uint32_t there;
                u64 v;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(from), "r"(k));
                asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(there) : "memory");
                sum += v;
            }
        }
        __syncwarp();
        // a CTA ends when the others have read its sum
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    if (warp == 0) {
        norm_fetch_wait();
        __syncwarp();
        u64 mine;
        const u64 root = norm_root(a, sum, norm_smem, lane < 2, party, &mine);
        if (lane < 2) told[party] = mine;
        if (lane == 0) told[2] = root;
    }
    __syncthreads();
    const u64 v[2] = {told[0], told[1]};
    q.finish(a, head, norm_tells(a, token, head), told[2], v);
    if (warp == 0 && rank == 0)
        for (int i = 0; i < 2; ++i)
            for (int k = lane; k < sent; k += 32) a.S[i][(size_t)row * sent + k] = norm_smem[i * count + k];
    __syncwarp();
    if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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
        for (int i = 0; i < 2; ++i) norm_load<VEC, true>(a.X[i] + (size_t)token * a.x_stride + (size_t)head * a.dim, p, x[i]);
        norm_angles<VEC>(a, token, p, c, s);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            norm_rotate_words(x[i], p, c, s, i, a.f);
            norm_store<VEC>(a.Z[i] + (size_t)row * a.dim, p, x[i]);
        }
    }
}

}  // namespace comet
