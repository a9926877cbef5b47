// Linear attention with a decay for every head on additive shares (comet_linear_attention, comet_linear_attention_step): products and
// public weights only, so that it needs no comparison.  f the fixed point, i the party, tr the local truncation by f bits, w[n] the public
// n-th power of a key head's decay, P, S, q, k, v, d shared; every value that enters a product is masked and opened once.
//   a prompt, in chunks; of a chunk of L tokens that finds the state S:
//     P[r][s] = tr(w[r - s] tr(q_r . k_s)), s <= r;   O_r = tr(sum_{s <= r} P[r][s] v_s + w[r + 1] tr(q_r S))
//     d_s = tr(w[L - 1 - s] k_s);                     S <- tr(w[L] S + sum_s d_s v_s^T)
//   single tokens:  S <- tr(w S + k v^T),  o = tr(q S)
// Four kernels for a prompt: all values that need no product are opened (open); the products d v^T of all chunks and key heads and the weights P
// of all chunks and query heads (products); the states from chunk to chunk, a word a thread (state); the rows of O (rows).
#pragma once
#include <cstdint>
#include <type_traits>
#include <cuda_runtime.h>

#include "kernels_limb.cuh"
#include "kernels_norm.cuh"
#include "pdl.cuh"

namespace comet {

namespace attn {
constexpr int MAX_CHUNK = 64, MAX_DIM = 256;
constexpr int THREADS = 256;
constexpr int ROWS = 64, COLS = 32, DEPTH = 32;      // of a tile of a product; contraction indices of a step
constexpr int WARP = 16;                             // rows and columns of a warp's part
constexpr int LEFT_BYTES = ROWS * DEPTH * 8, STEP_BYTES = LEFT_BYTES + COLS * DEPTH * 8;
constexpr int STEPS = 4;                             // in shared memory
constexpr int KEPT = 8;                              // words that a thread keeps from one product to the next
constexpr int TILE_SMEM = STEPS * STEP_BYTES + KEPT * THREADS * 8;
constexpr int SLAB = 16;                             // rows of a chunk that a CTA opens
}  // namespace attn

struct AttnArgs {
    const u64* Q[2]; const u64* K[2]; const u64* V[2];                   // token t at t * stride, heads behind one another
    const u64* mq[2]; const u64* mk[2]; const u64* mv[2]; const u64* md[2]; const u64* mp[2]; const u64* ms[2];
    const u64* qk[2]; const u64* pv[2]; const u64* qs[2]; const u64* dv[2];
    const u64* S0[2];                                                    // states, or null: zero
    u64* Eq[2]; u64* Ek[2]; u64* Ev[2]; u64* Ed[2]; u64* Ep[2]; u64* Es[2];
    u64* O[2];
    u64* S1[2];
    u64* kv[2];                                                          // [chunks][kv_heads][k_dim][v_dim]: sum d v^T at scale 2f
    u64* q; u64* k; u64* v; u64* d; u64* s;                              // opened values, as their messages lie
    u64* q1; u64* d1;                                                    // V_1 of Eq. 1: party 1's mask and the opened value
    u64* p; u64* pm[2];                                                  // opened weights, party 0's mask, V_1; zero off the triangle
    const u64* decay;                                                    // [kv_heads][C + 1]
    const int32_t* starts;
    int32_t* bad_starts;
    long long q_stride, k_stride, v_stride;
    int tokens, sequences, q_heads, kv_heads, k_dim, v_dim, C, chunks, f;
    int in_vec;                                                          // 16-byte accesses of Q, K and V
    int* error;                                                          // set where a wait ran out
};

// Tokens of sequence j, which begin at *begin: none where the starts are not ascending or leave the tokens.
__device__ __forceinline__ int attn_length(const AttnArgs& a, int j, int* begin) {
    const int b = a.starts[j], e = a.starts[j + 1];
    *begin = b;
    return b >= 0 && b <= e && e <= a.tokens ? e - b : 0;
}

struct AttnChunk {
    int seq, first, len;                                                 // len 0: there is no such chunk
};

// Chunk `want` of all sequences', by all threads of a CTA.
__device__ __forceinline__ AttnChunk attn_find(const AttnArgs& a, int want) {
    __shared__ AttnChunk found;
    __shared__ int sums[attn::THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    if (tid == 0) found = {0, 0, 0};
    for (int j0 = 0, base = 0; j0 < a.sequences && base <= want; j0 += blockDim.x) {
        const int j = j0 + tid;
        int begin = 0, len = 0;
        if (j < a.sequences) len = attn_length(a, j, &begin);
        const int n = (len + a.C - 1) / a.C;
        int up = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, up, o);
            if (lane >= o) up += t;
        }
        __syncthreads();
        if (lane == 31) sums[warp] = up;
        __syncthreads();
        int before = base, total = 0;
        for (int w = 0; w < warps; ++w) {
            before += w < warp ? sums[w] : 0;
            total += sums[w];
        }
        const int mine = want - (before + up - n);
        if (mine >= 0 && mine < n) found = {j, begin + mine * a.C, min(a.C, len - mine * a.C)};
        base += total;
    }
    __syncthreads();
    return found;
}

template <bool VEC>
__device__ __forceinline__ ulonglong2 attn_load2(const u64* p) {         // words that nobody reads again
    if (VEC) return __ldcs(reinterpret_cast<const ulonglong2*>(p));
    return make_ulonglong2(__ldcs(p), __ldcs(p + 1));
}
template <bool VEC>
__device__ __forceinline__ ulonglong2 attn_keep2(const u64* p) {         // words that the same kernel reads again
    if (VEC) return *reinterpret_cast<const ulonglong2*>(p);
    return make_ulonglong2(p[0], p[1]);
}
template <bool VEC>
__device__ __forceinline__ void attn_send2(u64* p, ulonglong2 v) {       // a message or result: nobody here reads it
    if (VEC) {
        __stcs(reinterpret_cast<ulonglong2*>(p), v);
    } else {
        __stcs(p, v.x);
        __stcs(p + 1, v.y);
    }
}
template <bool VEC>
__device__ __forceinline__ void attn_store2(u64* p, ulonglong2 v) {
    if (VEC) {
        *reinterpret_cast<ulonglong2*>(p) = v;
    } else {
        p[0] = v.x;
        p[1] = v.y;
    }
}

__device__ __forceinline__ ulonglong2 attn_input2(const u64* p, int vec) { return vec ? attn_load2<true>(p) : attn_load2<false>(p); }
__device__ __forceinline__ ulonglong2 attn_sub(ulonglong2 x, ulonglong2 y) { return make_ulonglong2(x.x - y.x, x.y - y.y); }
__device__ __forceinline__ ulonglong2 attn_add(ulonglong2 x, ulonglong2 y) { return make_ulonglong2(x.x + y.x, x.y + y.y); }
__device__ __forceinline__ u64 attn_rescale(u64 v, int party, int f) { return party ? 0ull - norm_shift(0ull - v, f) : norm_shift(v, f); }

// ---------------------------------------------------------------------------
// Products.  A CTA works out tiles of ROWS x COLS words of Z_i = (triple) + E B_i + V_i F, V_i = A_i + i E (Eq. 1), on the int8 tensor cores: a word is
// eight bytes, x = sum_p x_p 2^(8p), and of the 64 products of bytes the 36 with p + q <= 7 matter mod 2^64, summed up by p + q in eight 32-bit
// accumulators (kernels_limb.cuh has why 32 bits are enough).
//
// The words come to shared memory by asynchronous copies, STEPS steps of 32 indices of one product ahead; a warp cuts the words of its 16 rows and 16
// columns into bytes in registers, 72 instructions of 16 x 8 x 32 a step.  Which byte of an operand's registers is which contraction index does not
// matter as long as both operands agree: lane t of four has the indices 8j + 2t, 8j + 2t + 1, j < 4, words that lie side by side.
// ---------------------------------------------------------------------------
template <bool VEC>
__device__ __forceinline__ void attn_copy2(uint32_t to, const u64* from, int words) {        // those behind the words are zero
    if (VEC) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(8 * words) : "memory");
    } else {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(from), "r"(words > 0 ? 8 : 0) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to + 8), "l"(words > 1 ? from + 1 : from), "r"(words > 1 ? 8 : 0) : "memory");
    }
}

// An operand's part of a step, N rows or columns.  Its words lie `step` words from row to row; of a DEEP operand, whose rows lie side by side, from
// index to index.  In shared memory pieces change places so that the reads below meet no bank twice: of a row, whose 256 bytes eight lanes read in
// turns of 64, those halves of 128 bytes that its number says; of an index of a deep operand, of which sixteen lanes read four words of four
// indices, the pieces of 32 bytes.
template <bool DEEP, int N>
struct AttnSide {
    static_assert(N % 16 == 0, "whole passes");
    __device__ __forceinline__ static uint32_t place(int row, int piece) {           // of a pair of words
        return DEEP ? row * (N * 8) + (((piece >> 1) ^ ((row >> 1) & 3)) << 5) + ((piece & 1) << 4)
                    : row * 256 + (((piece >> 2) ^ (row & 1)) << 6) + ((piece & 3) << 4);
    }
    // `size` of the N rows are the operand's, `depth` of the 32 indices
    template <bool VEC>
    __device__ __forceinline__ static void copy(uint32_t to, const u64* x, uint32_t step, int size, int depth) {
        constexpr int PIECES = DEEP ? N / 2 : 16, LINES = DEEP ? attn::DEPTH : N, PASS = attn::THREADS / PIECES;
        const int piece = threadIdx.x % PIECES, first = threadIdx.x / PIECES;
        const int lines = DEEP ? depth : size, words = max(0, min(2, (DEEP ? size : depth) - 2 * piece));
#pragma unroll
        for (int l = first; l < LINES; l += PASS) {
            const int n = l < lines ? words : 0;
            attn_copy2<VEC>(to + place(l, piece), n ? x + (l * step + 2 * piece) : x, n);
        }
    }
    // The eight words of row `row` of lane t of four, cut into bytes: planes[p][h] byte p of the words 4h .. 4h + 3.
    __device__ __forceinline__ static void bytes(const uint8_t* from, int row, int t, uint32_t (&planes)[limb::PLANES][2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u64 w[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (DEEP) {
                    const uint8_t* const at = from + (16 * h + 8 * j + 2 * t) * (N * 8) + (((row >> 2) ^ t) << 5) + ((row & 3) << 3);
                    w[2 * j] = *reinterpret_cast<const u64*>(at);
                    w[2 * j + 1] = *reinterpret_cast<const u64*>(at + N * 8);
                } else {
                    const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(from + row * 256 + (((2 * h + j) ^ (row & 1)) << 6) + (t << 4));
                    w[2 * j] = v.x;
                    w[2 * j + 1] = v.y;
                }
            }
            limb_transpose4((uint32_t)w[0], (uint32_t)w[1], (uint32_t)w[2], (uint32_t)w[3], planes[0][h], planes[1][h], planes[2][h], planes[3][h]);
            limb_transpose4((uint32_t)(w[0] >> 32), (uint32_t)(w[1] >> 32), (uint32_t)(w[2] >> 32), (uint32_t)(w[3] >> 32), planes[4][h], planes[5][h],
                            planes[6][h], planes[7][h]);
        }
    }
};

// A warp's sums: [half of the columns][p + q][register of the instruction].
struct AttnSums {
    uint32_t d[2][limb::PLANES][4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int p = 0; p < limb::PLANES; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) d[n][p][j] = 0u;
    }
    // Pairs of words of a row: f(which of the thread's four pairs, row, column, pair)
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = (warp >> 1) * attn::WARP + (lane >> 2), col = (warp & 1) * attn::WARP + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u64 z[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int e = 2 * h + j;
                    z[j] = limb_recombine(d[n][0][e], d[n][1][e], d[n][2][e], d[n][3][e], d[n][4][e], d[n][5][e], d[n][6][e], d[n][7][e]);
                }
                f(2 * n + h, row + 8 * h, col + 8 * n, make_ulonglong2(z[0], z[1]));
            }
    }
};
__device__ __forceinline__ void attn_mma(uint32_t (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool DEEP_LEFT, bool DEEP_RIGHT>
__device__ __forceinline__ void attn_multiply(const uint8_t* step, AttnSums& sums) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, row = (warp >> 1) * attn::WARP + g, col = (warp & 1) * attn::WARP + g;
    uint32_t a[2][limb::PLANES][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) AttnSide<DEEP_LEFT, attn::ROWS>::bytes(step, row + 8 * h, t, a[h]);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        uint32_t b[limb::PLANES][2];
        AttnSide<DEEP_RIGHT, attn::COLS>::bytes(step + attn::LEFT_BYTES, col + 8 * n, t, b);
#pragma unroll
        for (int p = 0; p < limb::PLANES; ++p)
#pragma unroll
            for (int q = 0; p + q < limb::PLANES; ++q) attn_mma(sums.d[n][p + q], a[0][p][0], a[1][p][0], a[0][p][1], a[1][p][1], b[q][0], b[q][1]);
    }
}
// Steps 0 .. steps - 1 of a CTA: copy(step, where) asks for a step's words, work(step, where) uses them.
template <typename C, typename W>
__device__ __forceinline__ void attn_steps(uint8_t* smem, int steps, C&& copy, W&& work) {
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
#pragma unroll
    for (int n = 0; n < attn::STEPS - 1; ++n) {
        if (n < steps) copy(n, base + n * attn::STEP_BYTES);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
#pragma unroll 1
    for (int n = 0; n < steps; ++n) {
        asm volatile("cp.async.wait_group %0;" ::"n"(attn::STEPS - 2) : "memory");
        __syncthreads();                                     // the step is there, and the one before has been used by all
        const int ahead = n + attn::STEPS - 1;
        if (ahead < steps) copy(ahead, base + ahead % attn::STEPS * attn::STEP_BYTES);
        asm volatile("cp.async.commit_group;" ::: "memory");
        work(n, smem + n % attn::STEPS * attn::STEP_BYTES);
    }
}
__device__ __forceinline__ int attn_blocks(int depth) { return (depth + attn::DEPTH - 1) / attn::DEPTH; }

// The pairs of words of `rows` rows of `cols`, two at a time a thread: load(n, row, column) for both, then finish(n, row, column).
template <typename L, typename F>
__device__ __forceinline__ void attn_pairs(int rows, int cols, L&& load, F&& finish) {
    const int half = cols / 2, all = rows * half;
    for (int t = threadIdx.x; t < all; t += 2 * attn::THREADS) {
        int r[2], j[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int u = t + n * attn::THREADS;
            r[n] = u < all ? u / half : -1;
            j[n] = 2 * (u - r[n] * half);
            if (r[n] >= 0) load(n, r[n], j[n]);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
            if (r[n] >= 0) finish(n, r[n], j[n]);
    }
}

// Messages of q, or of k, v and d, of a head and SLAB rows of a chunk, and the opened values; zeros where no weight is sent.  Bound by memory.
template <bool VEC>
__global__ void __launch_bounds__(attn::THREADS, 2)
attn_open_kernel(const __grid_constant__ AttnArgs a, int slabs) {
    pdl_wait();
    pdl_launch_dependents();
    const int c = blockIdx.x / slabs, r0 = (blockIdx.x - c * slabs) * attn::SLAB;
    const AttnChunk at = attn_find(a, c);
    const int rows = min(attn::SLAB, at.len - r0), first = at.first + r0;
    if (rows <= 0) return;
    if ((int)blockIdx.y < a.kv_heads) {
        const int h = blockIdx.y;
        const size_t k_row = (size_t)a.kv_heads * a.k_dim, v_row = (size_t)a.kv_heads * a.v_dim;
        const size_t k_at = first * k_row + (size_t)h * a.k_dim, v_at = first * v_row + (size_t)h * a.v_dim;
        const u64* const w = a.decay + (size_t)h * (a.C + 1) + at.len - 1 - r0;
        ulonglong2 x[2][2], mk[2][2], md[2][2];
        attn_pairs(rows, a.k_dim, [&](int n, int r, int j) {
            const size_t o = k_at + r * k_row + j, x_at = (size_t)(first + r) * a.k_stride + (size_t)h * a.k_dim + j;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[n][i] = attn_input2(a.K[i] + x_at, a.in_vec);
                mk[n][i] = attn_load2<VEC>(a.mk[i] + o);
                md[n][i] = attn_load2<VEC>(a.md[i] + o);
            }
        }, [&](int n, int r, int j) {
            const size_t o = k_at + r * k_row + j;
            const u64 weight = __ldg(w - r);
            ulonglong2 e[2], g[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e[i] = attn_sub(x[n][i], mk[n][i]);
                g[i] = attn_sub(make_ulonglong2(attn_rescale(x[n][i].x * weight, i, a.f), attn_rescale(x[n][i].y * weight, i, a.f)), md[n][i]);
                attn_send2<VEC>(a.Ek[i] + o, e[i]);
                attn_send2<VEC>(a.Ed[i] + o, g[i]);
            }
            const ulonglong2 d = attn_add(g[0], g[1]);               // the exchange
            attn_store2<VEC>(a.k + o, attn_add(e[0], e[1]));
            attn_store2<VEC>(a.d + o, d);
            attn_store2<VEC>(a.d1 + o, attn_add(md[n][1], d));
        });
        attn_pairs(rows, a.v_dim, [&](int n, int r, int j) {
            const size_t o = v_at + r * v_row + j, x_at = (size_t)(first + r) * a.v_stride + (size_t)h * a.v_dim + j;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[n][i] = attn_input2(a.V[i] + x_at, a.in_vec);
                mk[n][i] = attn_load2<VEC>(a.mv[i] + o);
            }
        }, [&](int n, int r, int j) {
            const size_t o = v_at + r * v_row + j;
            ulonglong2 e[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e[i] = attn_sub(x[n][i], mk[n][i]);
                attn_send2<VEC>(a.Ev[i] + o, e[i]);
            }
            attn_store2<VEC>(a.v + o, attn_add(e[0], e[1]));         // the exchange
        });
    } else {
        const int h = blockIdx.y - a.kv_heads, wide_C = a.C + (a.C & 1);
        const size_t q_row = (size_t)a.q_heads * a.k_dim, p_row = (size_t)a.q_heads * a.C, w_row = (size_t)a.q_heads * wide_C;
        const size_t q_at = first * q_row + (size_t)h * a.k_dim, p_at = first * p_row + (size_t)h * a.C, w_at = first * w_row + (size_t)h * wide_C;
        ulonglong2 x[2][2], m[2][2];
        attn_pairs(rows, a.k_dim, [&](int n, int r, int j) {
            const size_t o = q_at + r * q_row + j, x_at = (size_t)(first + r) * a.q_stride + (size_t)h * a.k_dim + j;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[n][i] = attn_input2(a.Q[i] + x_at, a.in_vec);
                m[n][i] = attn_load2<VEC>(a.mq[i] + o);
            }
        }, [&](int n, int r, int j) {
            const size_t o = q_at + r * q_row + j;
            ulonglong2 e[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e[i] = attn_sub(x[n][i], m[n][i]);
                attn_send2<VEC>(a.Eq[i] + o, e[i]);
            }
            const ulonglong2 q = attn_add(e[0], e[1]);               // the exchange
            attn_store2<VEC>(a.q + o, q);
            attn_store2<VEC>(a.q1 + o, attn_add(m[n][1], q));
        });
        // off the triangle nothing is sent
        for (int t = threadIdx.x; t < rows * wide_C; t += attn::THREADS) {
            const int r = t / wide_C, k = t - r * wide_C;
            if (k <= r0 + r) continue;
            const size_t o = w_at + r * w_row + k;
            a.p[o] = a.pm[0][o] = a.pm[1][o] = 0ull;
            if (k < a.C) a.Ep[0][p_at + r * p_row + k] = a.Ep[1][p_at + r * p_row + k] = 0ull;
        }
    }
}

// A tile of the sum of d v^T of a chunk and key head, [k_dim][v_dim], of one party after the other.
template <bool VEC>
__device__ __forceinline__ void attn_keys(const AttnArgs& a, uint8_t* smem, const AttnChunk& at, int c, int h, int k0, int v0) {
    const uint32_t k_row = (uint32_t)a.kv_heads * a.k_dim, v_row = (uint32_t)a.kv_heads * a.v_dim;
    const size_t k_at = (size_t)at.first * k_row + (size_t)h * a.k_dim + k0, v_at = (size_t)at.first * v_row + (size_t)h * a.v_dim + v0;
    const size_t out = ((size_t)c * a.kv_heads + h) * a.k_dim * a.v_dim + (size_t)k0 * a.v_dim + v0;
    const int rows = min(attn::ROWS, a.k_dim - k0), cols = min(attn::COLS, a.v_dim - v0), half = 2 * attn_blocks(at.len);
    AttnSums sums;
    sums.clear();
    attn_steps(smem, 2 * half, [&](int n, uint32_t to) {
        const int i = n >= half, k = (n - i * half) / 2 * attn::DEPTH;
        const bool first = n % 2 == 0;                       // V_i F, then E B_i
        const u64* const d = (first ? i ? a.d1 : a.md[0] : a.d) + k_at;
        const u64* const v = (first ? a.v : i ? a.mv[1] : a.mv[0]) + v_at;
        AttnSide<true, attn::ROWS>::copy<VEC>(to, d + (size_t)k * k_row, k_row, rows, at.len - k);
        AttnSide<true, attn::COLS>::copy<VEC>(to + attn::LEFT_BYTES, v + (size_t)k * v_row, v_row, cols, at.len - k);
    }, [&](int n, const uint8_t* step) {
        attn_multiply<true, true>(step, sums);
        if ((n + 1) % half) return;
        const u64* const dv = (n < half ? a.dv[0] : a.dv[1]) + out;
        u64* const kv = (n < half ? a.kv[0] : a.kv[1]) + out;
        sums.each([&](int, int row, int col, ulonglong2 z) {
            if (row >= rows || col >= cols) return;
            const int o = row * a.v_dim + col;
            attn_store2<VEC>(kv + o, attn_add(z, attn_load2<VEC>(dv + o)));
        });
        sums.clear();
    });
}
// A tile of the weights of a chunk and query head: P of all rows and the keys from s0 on.
template <bool VEC>
__device__ __forceinline__ void attn_weights(const AttnArgs& a, uint8_t* smem, const AttnChunk& at, int hq, int s0) {
    const int h = hq / (a.q_heads / a.kv_heads), rows = at.len, keys = min(attn::COLS, rows - s0), half = 2 * attn_blocks(a.k_dim);
    const int wide_C = a.C + (a.C & 1);                      // of the opened weights' rows, which begin on 16-byte boundaries
    const uint32_t q_row = (uint32_t)a.q_heads * a.k_dim, k_row = (uint32_t)a.kv_heads * a.k_dim, p_row = (uint32_t)a.q_heads * a.C;
    const uint32_t w_row = (uint32_t)a.q_heads * wide_C;
    const size_t q_at = (size_t)at.first * q_row + (size_t)hq * a.k_dim, k_at = (size_t)(at.first + s0) * k_row + (size_t)h * a.k_dim;
    const size_t p_at = (size_t)at.first * p_row + (size_t)hq * a.C, w_at = (size_t)at.first * w_row + (size_t)hq * wide_C;
    const u64* const w = a.decay + (size_t)h * (a.C + 1);
    const bool pairs = VEC && a.C % 2 == 0;
    ulonglong2* const kept = reinterpret_cast<ulonglong2*>(smem + attn::STEPS * attn::STEP_BYTES) + threadIdx.x;
    const int warp = threadIdx.x >> 5;
    // off the triangle, or behind the rows: nothing to work out
    const bool idle = s0 + (warp & 1) * attn::WARP > (warp >> 1) * attn::WARP + attn::WARP - 1 || (warp >> 1) * attn::WARP >= rows;
    AttnSums sums;
    sums.clear();
    attn_steps(smem, 2 * half, [&](int n, uint32_t to) {
        const int i = n >= half, k = (n - i * half) / 2 * attn::DEPTH;
        const bool first = n % 2 == 0;
        const u64* const q = (first ? i ? a.q1 : a.mq[0] : a.q) + q_at + k;
        const u64* const x = (first ? a.k : i ? a.mk[1] : a.mk[0]) + k_at + k;
        AttnSide<false, attn::ROWS>::copy<VEC>(to, q, q_row, rows, a.k_dim - k);
        AttnSide<false, attn::COLS>::copy<VEC>(to + attn::LEFT_BYTES, x, k_row, keys, a.k_dim - k);
    }, [&](int n, const uint8_t* step) {
        if (idle) return;
        attn_multiply<false, false>(step, sums);
        if ((n + 1) % half) return;
        const bool second = n >= half;
        const u64* const qk = (second ? a.qk[1] : a.qk[0]) + p_at;
        const u64* const mp = (second ? a.mp[1] : a.mp[0]) + p_at;
        u64* const Ep = (second ? a.Ep[1] : a.Ep[0]) + p_at;
        u64* const pm = (second ? a.pm[1] : a.pm[0]) + w_at;
        // (the second word of a pair may lie off the triangle, where everything is zero, and behind an odd row's end)
        sums.each([&](int e, int r, int col, ulonglong2 z) {
            const int key = s0 + col;
            if (key > r || r >= rows) return;
            const bool both = key < r;
            const uint32_t o = r * p_row + key, to = r * w_row + key;
            auto load = [&](const u64* x) { return pairs ? attn_load2<true>(x + o) : make_ulonglong2(__ldcs(x + o), both ? __ldcs(x + o + 1) : 0ull); };
            const ulonglong2 x = load(qk);
            ulonglong2 m = load(mp);
            if (!both) m.y = 0ull;
            const u64 one = attn_rescale(attn_rescale(z.x + x.x, second, a.f) * __ldg(w + r - key), second, a.f) - m.x;
            u64 two = 0ull;
            if (both) two = attn_rescale(attn_rescale(z.y + x.y, second, a.f) * __ldg(w + r - key - 1), second, a.f) - m.y;
            if (pairs) attn_send2<true>(Ep + o, make_ulonglong2(one, two));
            else {
                Ep[o] = one;
                if (both) Ep[o + 1] = two;
            }
            if (!second) {
                kept[e * attn::THREADS] = make_ulonglong2(one, two);
            } else {
                const ulonglong2 open = attn_add(kept[e * attn::THREADS], make_ulonglong2(one, two));    // the exchange
                *reinterpret_cast<ulonglong2*>(a.p + w_at + to) = open;
                m = attn_add(m, open);
            }
            *reinterpret_cast<ulonglong2*>(pm + to) = m;
        });
        sums.clear();
    });
}
template <bool VEC>
__global__ void __launch_bounds__(attn::THREADS, 2)
attn_products_kernel(const __grid_constant__ AttnArgs a, int keys_ctas, int k_tiles, int v_tiles, int s_tiles) {
    extern __shared__ __align__(128) uint8_t attn_smem[];
    pdl_wait();
    pdl_launch_dependents();
    if ((int)blockIdx.x < keys_ctas) {
        const int tiles = k_tiles * v_tiles, ch = blockIdx.x / tiles, tile = blockIdx.x - ch * tiles, c = ch / a.kv_heads, kt = tile / v_tiles;
        const AttnChunk at = attn_find(a, c);
        if (at.len) attn_keys<VEC>(a, attn_smem, at, c, ch - c * a.kv_heads, kt * attn::ROWS, (tile - kt * v_tiles) * attn::COLS);
    } else {
        const int b = blockIdx.x - keys_ctas, ch = b / s_tiles, s0 = (b - ch * s_tiles) * attn::COLS, c = ch / a.q_heads;
        const AttnChunk at = attn_find(a, c);
        if (s0 < at.len) attn_weights<VEC>(a, attn_smem, at, ch - c * a.q_heads, s0);
    }
}

// The state from chunk to chunk of a sequence and key head, two words of both parties a thread; says whether the starts were in order.
template <bool VEC>
__global__ void __launch_bounds__(attn::THREADS)
attn_state_kernel(const __grid_constant__ AttnArgs a, int pieces) {
    __shared__ int before;
    pdl_wait();
    pdl_launch_dependents();
    const int j = blockIdx.x / (a.kv_heads * pieces), rest = blockIdx.x - j * a.kv_heads * pieces, h = rest / pieces;
    const int word = 2 * ((rest - h * pieces) * attn::THREADS + threadIdx.x), words = a.k_dim * a.v_dim;
    if (threadIdx.x == 0) before = 0;
    __syncthreads();
    const bool checks = blockIdx.x == 0;
    int sum = 0, begin;
    bool bad = false;
    for (int s = threadIdx.x; s < (checks ? a.sequences : j); s += attn::THREADS) {
        sum += (attn_length(a, s, &begin) + a.C - 1) / a.C;
        const int end = __ldg(a.starts + s + 1);
        bad |= begin < 0 || end < begin || end > a.tokens;
    }
    if (sum) atomicAdd(&before, sum);
    if (bad && checks && a.bad_starts) *a.bad_starts = 1;
    __syncthreads();
    if (checks && threadIdx.x == 0 && before != a.chunks && a.bad_starts) *a.bad_starts = 1;
    if (word >= words) return;
    const size_t at = ((size_t)j * a.kv_heads + h) * words + word, step = (size_t)a.kv_heads * words;
    const u64* const w = a.decay + (size_t)h * (a.C + 1);
    int c = checks ? 0 : before, left = attn_length(a, j, &begin);
    const int end = min(a.chunks, c + (left + a.C - 1) / a.C);
    ulonglong2 S[2], kv[2], ms[2];
    size_t o = ((size_t)c * a.kv_heads + h) * words + word;
    auto load = [&] {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            kv[i] = attn_load2<VEC>(a.kv[i] + o);
            ms[i] = attn_keep2<VEC>(a.ms[i] + o);
        }
    };
    if (c < end) load();
#pragma unroll
    for (int i = 0; i < 2; ++i) S[i] = a.S0[i] ? attn_load2<VEC>(a.S0[i] + at) : make_ulonglong2(0ull, 0ull);
    for (; c < end; ++c, left -= a.C) {
        const u64 weight = __ldg(w + min(left, a.C));
        ulonglong2 e[2];
        const size_t here = o;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            e[i] = attn_sub(S[i], ms[i]);
            S[i] = make_ulonglong2(attn_rescale(weight * S[i].x + kv[i].x, i, a.f), attn_rescale(weight * S[i].y + kv[i].y, i, a.f));
        }
        o += step;
        if (c + 1 < end) load();
#pragma unroll
        for (int i = 0; i < 2; ++i) attn_send2<VEC>(a.Es[i] + here, e[i]);
        attn_store2<VEC>(a.s + here, attn_add(e[0], e[1]));              // the exchange
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) attn_store2<VEC>(a.S1[i] + at, S[i]);
}

// A tile of the rows of O of a chunk, query head and party: the far part w[r + 1] tr(q S), then the near part P v.
template <bool VEC>
__global__ void __launch_bounds__(attn::THREADS, 2)
attn_rows_kernel(const __grid_constant__ AttnArgs a, int v_tiles) {
    extern __shared__ __align__(128) uint8_t attn_smem[];
    pdl_wait();
    pdl_launch_dependents();
    const int tile = blockIdx.x / 2, ch = tile / v_tiles, c = ch / a.q_heads, hq = ch - c * a.q_heads, h = hq / (a.q_heads / a.kv_heads);
    const int v0 = (tile - ch * v_tiles) * attn::COLS;
    const bool second = blockIdx.x % 2;                      // party
    const AttnChunk at = attn_find(a, c);
    if (at.len == 0) return;
    const int rows = at.len, cols = min(attn::COLS, a.v_dim - v0), far = 2 * attn_blocks(a.k_dim), near = 2 * attn_blocks(rows), wide_C = a.C + (a.C & 1);
    const uint32_t q_row = (uint32_t)a.q_heads * a.k_dim, v_row = (uint32_t)a.kv_heads * a.v_dim, o_row = (uint32_t)a.q_heads * a.v_dim;
    const uint32_t w_row = (uint32_t)a.q_heads * wide_C;
    const size_t q_at = (size_t)at.first * q_row + (size_t)hq * a.k_dim, v_at = (size_t)at.first * v_row + (size_t)h * a.v_dim + v0;
    const size_t s_at = ((size_t)c * a.kv_heads + h) * a.k_dim * a.v_dim + v0;
    const size_t w_at = (size_t)at.first * w_row + (size_t)hq * wide_C, o_at = (size_t)at.first * o_row + (size_t)hq * a.v_dim + v0;
    ulonglong2* const kept = reinterpret_cast<ulonglong2*>(attn_smem + attn::STEPS * attn::STEP_BYTES) + threadIdx.x;
    const int warp_row = (threadIdx.x >> 6) * attn::WARP;
    AttnSums sums;
    sums.clear();
    attn_steps(attn_smem, far + near, [&](int n, uint32_t to) {
        const bool first = n % 2 == 0;
        if (n < far) {
            const int k = n / 2 * attn::DEPTH;
            const u64* const q = (first ? second ? a.q1 : a.mq[0] : a.q) + q_at + k;
            const u64* const S = (first ? a.s : second ? a.ms[1] : a.ms[0]) + s_at + (size_t)k * a.v_dim;
            AttnSide<false, attn::ROWS>::copy<VEC>(to, q, q_row, rows, a.k_dim - k);
            AttnSide<true, attn::COLS>::copy<VEC>(to + attn::LEFT_BYTES, S, a.v_dim, cols, a.k_dim - k);
        } else {
            const int k = (n - far) / 2 * attn::DEPTH;
            const u64* const p = (first ? second ? a.pm[1] : a.pm[0] : a.p) + w_at + k;
            const u64* const v = (first ? a.v : second ? a.mv[1] : a.mv[0]) + v_at + (size_t)k * v_row;
            // (the opened weights' rows are longer than an odd number of keys by a word, zero)
            AttnSide<false, attn::ROWS>::copy<VEC>(to, p, w_row, rows, rows - k);
            AttnSide<true, attn::COLS>::copy<VEC>(to + attn::LEFT_BYTES, v, v_row, cols, rows - k);
        }
    }, [&](int n, const uint8_t* step) {
        if (warp_row >= rows) return;
        // (a key behind all of a warp's rows has no weight)
        if (n < far || (n - far) / 2 * attn::DEPTH < warp_row + attn::WARP) attn_multiply<false, true>(step, sums);
        if (n == far - 1) {
            const u64* const qs = (second ? a.qs[1] : a.qs[0]) + o_at;
            const u64* const pv = (second ? a.pv[1] : a.pv[0]) + o_at;
            const u64* const w = a.decay + (size_t)h * (a.C + 1) + 1;
            sums.each([&](int e, int r, int col, ulonglong2 z) {
                if (r >= rows || col >= cols) return;
                const uint32_t o = r * o_row + col;
                const ulonglong2 x = attn_load2<VEC>(qs + o), y = attn_load2<VEC>(pv + o);
                const u64 weight = __ldg(w + r);
                kept[e * attn::THREADS] = make_ulonglong2(y.x + weight * attn_rescale(z.x + x.x, second, a.f), y.y + weight * attn_rescale(z.y + x.y, second, a.f));
            });
            sums.clear();
        } else if (n == far + near - 1) {
            u64* const O = (second ? a.O[1] : a.O[0]) + o_at;
            sums.each([&](int e, int r, int col, ulonglong2 z) {
                if (r >= rows || col >= cols) return;
                const ulonglong2 x = attn_add(z, kept[e * attn::THREADS]);
                attn_send2<VEC>(O + (r * o_row + col), make_ulonglong2(attn_rescale(x.x, second, a.f), attn_rescale(x.y, second, a.f)));
            });
        }
    });
}

// ---------------------------------------------------------------------------
// Single tokens.  Bound by memory: of every word of a state and party five words, the state, its mask and the product in, the message
// and the new state out.  A CTA has both parties' words of a slice of a state's columns, a thread one pair of columns in every
// row_groups-th row, so every word passes once through the thread that exchanges it; q and k lie in shared memory, what they
// are multiplied with as they are needed.  The sums of o are added up over the row groups at the end.
// ---------------------------------------------------------------------------
struct AttnStepArgs {
    const u64* Q[2]; const u64* K[2]; const u64* V[2];
    const u64* mq[2]; const u64* mk[2]; const u64* mv[2]; const u64* ms[2];
    const u64* kv[2]; const u64* qs[2];
    const u64* S0[2];
    u64* Eq[2]; u64* Ek[2]; u64* Ev[2]; u64* Es[2];
    u64* O[2];
    u64* S1[2];
    const u64* decay;                                                    // [kv_heads]
    long long q_stride, k_stride, v_stride;
    int q_heads, kv_heads, k_dim, v_dim, f;
    int slices, slice_pairs;                                             // of the columns
};

// Dynamic shared memory: a row's opened k and both parties' masks (party 1's with the opened value added: V_i of Eq. 1), the same of q for
// `heads` heads; the sums of o of every thread.
__host__ __device__ constexpr int attn_step_smem(int k_dim, int heads) {
    return 3 * (1 + heads) * k_dim * 8 + heads * attn::THREADS * 2 * 16;
}

// HEADS query heads of a key head's are worked on at a time; those beyond read masks and messages of the state a second time.
template <bool VEC, int HEADS>
__global__ void __launch_bounds__(attn::THREADS)
attn_step_kernel(const __grid_constant__ AttnStepArgs a) {
    extern __shared__ __align__(16) uint8_t step_smem[];
    u64* const keys = reinterpret_cast<u64*>(step_smem);                                 // [k_dim][3]
    u64* const queries = keys + 3 * a.k_dim;                                             // [k_dim][HEADS][3]
    ulonglong2* const sums = reinterpret_cast<ulonglong2*>(queries + 3 * HEADS * a.k_dim);   // [HEADS][2][THREADS]
    const int bh = blockIdx.x / a.slices, slice = blockIdx.x - bh * a.slices, b = bh / a.kv_heads, h = bh - b * a.kv_heads;
    const int group = a.q_heads / a.kv_heads, tid = threadIdx.x, f = a.f;
    const int row_groups = attn::THREADS / a.slice_pairs, rg = tid / a.slice_pairs, pair = slice * a.slice_pairs + tid - rg * a.slice_pairs;
    const bool mine = rg < row_groups && pair < a.v_dim / 2;
    const int col = 2 * (mine ? pair : 0);
    const size_t k_at = (size_t)bh * a.k_dim, v_at = (size_t)bh * a.v_dim, q_at = k_at * group, o_at = v_at * group, s_at = k_at * a.v_dim + col;
    pdl_wait();
    pdl_launch_dependents();
    // a row's words: state, product, mask
    ulonglong2 S[2], kv[2], ms[2];
    auto load = [&](int r) {
        const size_t o = s_at + (size_t)r * a.v_dim;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            S[i] = a.S0[i] ? attn_load2<VEC>(a.S0[i] + o) : make_ulonglong2(0ull, 0ull);
            kv[i] = attn_load2<VEC>(a.kv[i] + o);
            ms[i] = attn_load2<VEC>(a.ms[i] + o);
        }
    };
    if (mine && rg < a.k_dim) load(rg);
    const u64 w = __ldg(a.decay + h);
    ulonglong2 F = make_ulonglong2(0ull, 0ull), mv[2];
    if (mine) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u64* const V = a.V[i] + b * a.v_stride + (long long)h * a.v_dim + col;
            mv[i] = make_ulonglong2(__ldg(a.mv[i] + v_at + col), __ldg(a.mv[i] + v_at + col + 1));
            const ulonglong2 e = make_ulonglong2(__ldg(V) - mv[i].x, __ldg(V + 1) - mv[i].y);
            if (rg == 0) attn_store2<false>(a.Ev[i] + v_at + col, e);
            F.x += e.x;
            F.y += e.y;
        }
    }
    auto open = [&](u64* to, int step, const u64* const x[2], long long x_at, const u64* const m[2], u64* const msg[2], size_t at) {
        for (int r = tid; r < a.k_dim; r += attn::THREADS) {
            u64 mask[2], e[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mask[i] = __ldg(m[i] + at + r);
                e[i] = __ldg(x[i] + x_at + r) - mask[i];
                if (slice == 0) msg[i][at + r] = e[i];
            }
            to[r * step] = e[0] + e[1];
            to[r * step + 1] = mask[0];
            to[r * step + 2] = mask[1] + e[0] + e[1];
        }
    };
    open(keys, 3, a.K, b * a.k_stride + (long long)h * a.k_dim, a.mk, a.Ek, k_at);
    for (int g0 = 0; g0 < group; g0 += HEADS) {
#pragma unroll
        for (int g = 0; g < HEADS; ++g)
            if (g0 + g < group)
                open(queries + 3 * g, 3 * HEADS, a.Q, b * a.q_stride + (long long)(h * group + g0 + g) * a.k_dim, a.mq, a.Eq, q_at + (size_t)(g0 + g) * a.k_dim);
        __syncthreads();
        u64 o[HEADS][2][2];
#pragma unroll
        for (int g = 0; g < HEADS; ++g) o[g][0][0] = o[g][0][1] = o[g][1][0] = o[g][1][1] = 0ull;
        if (mine)
            for (int r = rg; r < a.k_dim; r += row_groups) {
                const size_t at = s_at + (size_t)r * a.v_dim;
                ulonglong2 mask[2], e[2];
                if (g0 == 0) {
                    const u64 E = keys[3 * r];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const u64 A = keys[3 * r + 1 + i];
                        const u64 x = attn_rescale(kv[i].x + E * mv[i].x + A * F.x + w * S[i].x, i, f);
                        const u64 y = attn_rescale(kv[i].y + E * mv[i].y + A * F.y + w * S[i].y, i, f);
                        mask[i] = ms[i];
                        e[i] = make_ulonglong2(x - mask[i].x, y - mask[i].y);
                        attn_store2<VEC>(a.S1[i] + at, make_ulonglong2(x, y));
                        attn_store2<VEC>(a.Es[i] + at, e[i]);
                    }
                    if (r + row_groups < a.k_dim) load(r + row_groups);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        mask[i] = attn_load2<VEC>(a.ms[i] + at);
                        e[i] = make_ulonglong2(a.Es[i][at], a.Es[i][at + 1]);      // this thread's own
                    }
                }
                const u64 ex = e[0].x + e[1].x, ey = e[0].y + e[1].y;
#pragma unroll
                for (int g = 0; g < HEADS; ++g) {
                    const u64* const q = queries + 3 * (r * HEADS + g);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        o[g][i][0] += q[0] * mask[i].x + q[1 + i] * ex;
                        o[g][i][1] += q[0] * mask[i].y + q[1 + i] * ey;
                    }
                }
            }
#pragma unroll
        for (int g = 0; g < HEADS; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) sums[(g * 2 + i) * attn::THREADS + tid] = make_ulonglong2(o[g][i][0], o[g][i][1]);
        __syncthreads();
        for (int t = tid; t < HEADS * 2 * a.slice_pairs; t += attn::THREADS) {
            const int gi = t / a.slice_pairs, p = t - gi * a.slice_pairs, g = gi >> 1, i = gi & 1, c = slice * a.slice_pairs + p;
            if (g0 + g >= group || c >= a.v_dim / 2) continue;
            ulonglong2 z = make_ulonglong2(0ull, 0ull);
            for (int k = 0; k < row_groups; ++k) {
                const ulonglong2 v = sums[gi * attn::THREADS + k * a.slice_pairs + p];
                z.x += v.x;
                z.y += v.y;
            }
            const size_t at = o_at + (size_t)(g0 + g) * a.v_dim + 2 * c;
            z.x += __ldg(a.qs[i] + at);
            z.y += __ldg(a.qs[i] + at + 1);
            attn_store2<false>(a.O[i] + at, make_ulonglong2(attn_rescale(z.x, i, f), attn_rescale(z.y, i, f)));
        }
        __syncthreads();
    }
}

}  // namespace comet
