// Linear attention with a decay for every head on additive shares (comet_linear_attention, comet_linear_attention_step): products and
// public weights only, so that it needs no comparison.  f the fixed point, i the party, tr the local truncation by f bits, w[n] the public
// n-th power of a key head's decay, P, S, q, k, v, d shared; every value that enters a product is masked and opened once.
//   a prompt, in chunks; of a chunk of L tokens that finds the state S:
//     P[r][s] = tr(w[r - s] tr(q_r . k_s)), s <= r;   O_r = tr(sum_{s <= r} P[r][s] v_s + w[r + 1] tr(q_r S))
//     d_s = tr(w[L - 1 - s] k_s);                     S <- tr(w[L] S + sum_s d_s v_s^T)
//   single tokens:  S <- tr(w S + k v^T),  o = tr(q S)
// Four kernels for a prompt: all values that need no product are opened (open); the products d v^T of all chunks and key heads and the weights P
// of all chunks and query heads (products); the states from chunk to chunk, a word a thread (state); the rows of O (rows).  Before them, where it pays, one
// that lists the chunks (list).  What enters a product is
// cut into bytes by the kernel that has it in registers anyway, once, so that those of the products only copy, multiply and add.  (The bytes are
// as many as the words: the same traffic, and no warp of a product's kernel converts.  512 tokens x 32 heads x 128, "the case" below: words cut
// into bytes by warps beside the issuer 438 us, by every warp for its own mma.sync 679, this 371, of which memory's floor is 108.)
// None of these kernels lets the next one's CTAs in before its end (pdl_launch_dependents): they would hold registers and shared memory of SMs that
// still have work, where the kernel that opens the next pass's values holds most.  With it 468 us.
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
constexpr int LEFT = 128, RIGHT = 64;                // rows of a tile's operands at most
constexpr int KC = limb::KC, ROW_BYTES = limb::PLANES * KC;          // of a block of planes: 32 contraction indices
constexpr int SLOTS = 3, LEFT_BYTES = LEFT * ROW_BYTES, SLOT_BYTES = LEFT_BYTES + RIGHT * ROW_BYTES;
constexpr int DRAINERS = 16, PRODUCER = DRAINERS, ISSUER = DRAINERS + 1, TILE_THREADS = 32 * (ISSUER + 1), DRAIN_THREADS = 32 * DRAINERS;
constexpr int ACC_COLS = limb::PLANES * RIGHT;
constexpr int TILE_SMEM = SLOTS * SLOT_BYTES + RIGHT * LEFT * 8 + 128;
constexpr int SLAB = 16;                             // tokens that a CTA opens
constexpr int STATE_THREADS = 128;
constexpr int NOBODY = 1 << 20;                          // behind the last sequence, of which there are no more
constexpr int WINDOW = 1024;                           // tokens that a CTA looks over for rows in no chunk
__host__ __device__ constexpr int up16(int n) { return (n + 15) / 16 * 16; }
__host__ __device__ constexpr int blocks(int n) { return (n + KC - 1) / KC; }
}  // namespace attn

// Blocks of limb planes (kernels_limb.cuh) of an operand: the opened value, party 0's and party 1's mask, or for the operand of a product that takes
// it V_i = mask + i * opened (Eq. 1).  A block has 32 contraction indices of up to 128 rows (left operands: values and states; keys have up to
// 64) or 64 (right ones), rounded up to 16, so that a block's planes lie side by side whatever its rows are.  Contraction indices are in their order.
// Planes of tokens lie behind those of the chunks before, whose rows and blocks are counted: a chunk of one token takes one block's room, not a whole chunk's.
struct AttnPlanes {
    uint8_t* set[3];
};
struct AttnArgs {
    const u64* Q[2]; const u64* K[2]; const u64* V[2];                   // token t at t * stride, heads behind one another
    const u64* mq[2]; const u64* mk[2]; const u64* mv[2]; const u64* md[2]; const u64* mp[2]; const u64* ms[2];
    const u64* qk[2]; const u64* pv[2]; const u64* qs[2]; const u64* dv[2];
    const u64* S0[2];                                                    // states, or null: zero
    u64* Eq[2]; u64* Ek[2]; u64* Ev[2]; u64* Ed[2]; u64* Ep[2]; u64* Es[2];
    u64* O[2];
    u64* S1[2];
    u64* kv[2];                                                          // [chunks][kv_heads][k_dim][v_dim]: sum d v^T at scale 2f
    AttnPlanes q, k, d, v, s, p;
    int4* found;                                                         // [chunks]: first token, 128 x sequence + tokens, rows (in sixteens) and blocks of those before
    int listed;                                                          // whether it is there before the values are opened
    const u64* decay;                                                    // [kv_heads][C + 1]
    const int32_t* starts;
    int32_t* bad_starts;
    long long q_stride, k_stride, v_stride;
    int tokens, sequences, q_heads, kv_heads, k_dim, v_dim, C, chunks, f;
    int row_room, block_room;                                            // sixteens of rows and blocks of all chunks that there is room for
    int in_vec;                                                          // 16-byte accesses of Q, K and V
    int* error;                                                          // set where a wait ran out
    int clears;                                                          // CTAs of the kernel of states that set to zero what nobody writes
};

// Tokens of sequence j, which begin at *begin: none where the starts are not ascending or leave the tokens.
__device__ __forceinline__ int attn_length(const AttnArgs& a, int j, int* begin) {
    const int b = a.starts[j], e = a.starts[j + 1];
    *begin = b;
    return b >= 0 && b <= e && e <= a.tokens ? e - b : 0;
}

struct AttnChunk {
    int4 at;                                             // as in `found`, but y the tokens: none where there is no such chunk, or no room for it
    int owner;                                           // its sequence
};
__device__ __forceinline__ AttnChunk attn_no_chunk() { return {make_int4(0, 0, 0, 0), attn::NOBODY}; }
__device__ __forceinline__ void attn_put(const AttnArgs& a, int c, const AttnChunk& x) { a.found[c] = make_int4(x.at.x, x.owner * 128 + x.at.y, x.at.z, x.at.w); }
__device__ __forceinline__ int4 attn_chunk(const AttnArgs& a, int c) {
    int4 at = a.found[c];
    at.y &= 127;
    return at;
}
__device__ __forceinline__ int attn_owner(const AttnArgs& a, int c) { return a.found[c].y >> 7; }

// Chunks first to last of all sequences', by all threads of a CTA: emit(number, chunk) by whichever thread has its sequence.  Sequences that overlap may have more
// tokens together than there is room for.
template <typename F>
__device__ __forceinline__ void attn_scan(const AttnArgs& a, int first, int last, F&& emit) {
    __shared__ int sums[attn::THREADS / 32][3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int base[3] = {0, 0, 0};                             // chunks, their rows in sixteens, their blocks
    for (int j0 = 0; j0 < a.sequences && base[0] <= last; j0 += attn::THREADS) {
        const int warps = (min(a.sequences - j0, attn::THREADS) + 31) / 32;              // that have any
        const int j = j0 + tid;
        int begin = 0, len = 0;
        if (j < a.sequences) len = attn_length(a, j, &begin);
        const int full = len / a.C, rest = len - full * a.C;
        const int own[3] = {full + (rest > 0), full * (attn::up16(a.C) / 16) + attn::up16(rest) / 16, full * attn::blocks(a.C) + attn::blocks(rest)};
        int up[3] = {own[0], own[1], own[2]};
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int t = __shfl_up_sync(0xffffffffu, up[k], o);
                if (lane >= o) up[k] += t;
            }
        __syncthreads();
        if (lane == 31)
#pragma unroll
            for (int k = 0; k < 3; ++k) sums[warp][k] = up[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) up[k] += base[k] - own[k];
        for (int w = 0; w < warps; ++w)
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int t = sums[w][k];
                up[k] += w < warp ? t : 0;
                base[k] += t;
            }
        for (int c = max(first, up[0]); c <= min(last, up[0] + own[0] - 1); ++c) {
            const int mine = c - up[0], n = min(a.C, len - mine * a.C), rows = up[1] + mine * (attn::up16(a.C) / 16), blocks = up[2] + mine * attn::blocks(a.C);
            const bool room = rows + attn::up16(n) / 16 <= a.row_room && blocks + attn::blocks(n) <= a.block_room;
            emit(c, AttnChunk{room ? make_int4(begin + mine * a.C, n, rows, blocks) : make_int4(0, 0, 0, 0), j});
        }
    }
}

// Chunk `want`, to all threads of a CTA.
__device__ __forceinline__ AttnChunk attn_find(const AttnArgs& a, int want) {
    __shared__ AttnChunk found;
    if (threadIdx.x == 0) found = attn_no_chunk();
    __syncthreads();
    attn_scan(a, want, want, [&](int, const AttnChunk& c) { found = c; });
    __syncthreads();
    return found;
}

// The list of all chunks (AttnArgs::listed): a CTA has as many chunks as threads.  65536 prompts of one token, one head of 2: 11 ms; with every CTA that
// opens values looking through all sequences for itself 181.
__global__ void __launch_bounds__(attn::THREADS)
attn_list_kernel(const __grid_constant__ AttnArgs a) {
    pdl_wait();
    const int first = blockIdx.x * attn::THREADS, last = min(first + attn::THREADS, a.chunks) - 1, c = first + threadIdx.x;
    if (c <= last) attn_put(a, c, attn_no_chunk());
    __syncthreads();
    attn_scan(a, first, last, [&](int k, const AttnChunk& x) { attn_put(a, k, x); });
}

template <bool VEC>
__device__ __forceinline__ ulonglong2 attn_load2(const u64* p) {         // words that nobody reads again
    if (VEC) return __ldcs(reinterpret_cast<const ulonglong2*>(p));
    return make_ulonglong2(__ldcs(p), __ldcs(p + 1));
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
__device__ __forceinline__ ulonglong2 attn_add(ulonglong2 x, ulonglong2 y) { return make_ulonglong2(x.x + y.x, x.y + y.y); }
__device__ __forceinline__ u64 attn_rescale(u64 v, int party, int f) { return party ? 0ull - norm_shift(0ull - v, f) : norm_shift(v, f); }

// Where blocks lie, in bytes from a set's begin.  q, k, p: rows are a chunk's tokens, a head has up to `blocks` blocks; d, v, s: rows are k_dim in tiles of
// 64, or v_dim in tiles of 128, and a head has `blocks` blocks behind the `before` of others.
__device__ __forceinline__ size_t attn_token_block(const int4& found, int heads, int head, int blocks, int b) {
    return ((size_t)found.z * 16 * heads * blocks + (size_t)(head * blocks + b) * attn::up16(found.y)) * attn::ROW_BYTES;
}
__device__ __forceinline__ size_t attn_dim_block(size_t before, int blocks, int b, int dim, int row0, int tile) {
    const int wide = attn::up16(dim);
    return (before * wide + (size_t)row0 * blocks + (size_t)b * min(tile, wide - row0)) * attn::ROW_BYTES;
}
// Blocks of a key head's values or decayed keys start behind this many.
__device__ __forceinline__ size_t attn_before(const int4& found, int heads, int head) { return (size_t)found.w * heads + head * attn::blocks(found.y); }
// Words of a row, `n` of them from index `first` on (a multiple of n), into a block of `rows` rows: n bytes a plane at once.
__device__ __forceinline__ uint8_t* attn_spot(uint8_t* block, int row, int first) {
    return block + (row >> 3) * 256 + (first >> 4) * 128 + (row & 7) * 16 + (first & 15);
}
__device__ __forceinline__ void attn_bytes(const u64* w, uint32_t (&p)[limb::PLANES]) {
    limb_transpose4((uint32_t)w[0], (uint32_t)w[1], (uint32_t)w[2], (uint32_t)w[3], p[0], p[1], p[2], p[3]);
    limb_transpose4((uint32_t)(w[0] >> 32), (uint32_t)(w[1] >> 32), (uint32_t)(w[2] >> 32), (uint32_t)(w[3] >> 32), p[4], p[5], p[6], p[7]);
}
__device__ __forceinline__ void attn_emit(uint8_t* block, int rows, int row, int first, const u64 (&w)[4]) {
    limb_emit4(attn_spot(block, row, first), rows * attn::KC, w);
}
__device__ __forceinline__ void attn_emit(uint8_t* block, int rows, int row, int first, const u64 (&w)[8]) {
    uint32_t lo[limb::PLANES], hi[limb::PLANES];
    attn_bytes(w, lo);
    attn_bytes(w + 4, hi);
    uint8_t* const to = attn_spot(block, row, first);
#pragma unroll
    for (int p = 0; p < limb::PLANES; ++p) *reinterpret_cast<uint2*>(to + p * rows * attn::KC) = make_uint2(lo[p], hi[p]);
}

// Messages of k, d, v or q of a head and SLAB tokens of a chunk, and the planes of what they open; zeros where no weight is sent.  Bound by
// memory: of a word and party two in, one out as a message, and three sets of planes for both parties.  q and k: eight words of a row a thread, four
// threads a row's 32 words.  v and d, whose contraction runs over the tokens: eight tokens of a word a thread, sixteen tokens x sixteen words a
// warp, 128 bytes of a token.  Eight bytes a plane at once either way, 256 bytes a warp, whole sectors.
// The case: 114 us, 570 MB; four bytes a plane at once took 135 us, a third CTA an SM (80 registers) 135 as well.
template <bool VEC>
__global__ void __launch_bounds__(attn::THREADS, 2)
attn_open_kernel(const __grid_constant__ AttnArgs a, int slabs) {
    pdl_wait();
    const int c = blockIdx.x / slabs, t0 = (blockIdx.x - c * slabs) * attn::SLAB;
    int4 at;
    if (a.listed) {
        at = attn_chunk(a, c);
    } else {
        const AttnChunk found = attn_find(a, c);
        at = found.at;
        if (blockIdx.x == c * slabs && blockIdx.y == 0 && threadIdx.x == 0) attn_put(a, c, found);
    }
    const int blocks = attn::blocks(at.y), rows16 = attn::up16(at.y), rows = min(attn::SLAB, at.y - t0), first = at.x + t0;
    if (t0 >= blocks * attn::KC) return;
    const int f = a.f;
    // rows of queries or keys: messages, and the planes of the opened value, party 0's mask, party 1's or V_1
    auto open_rows = [&](const u64* const x[2], long long stride, const u64* const m[2], u64* const msg[2], const AttnPlanes& to, int heads, int head, bool query) {
        const int parts = attn::blocks(a.k_dim) * 4;
        const size_t o0 = ((size_t)first * heads + head) * a.k_dim, block0 = attn_token_block(at, heads, head, parts / 4, 0);
        for (int t = threadIdx.x; t < rows * parts; t += attn::THREADS) {
            const int r = t / parts, part = t - r * parts;
            const size_t o = o0 + (size_t)r * heads * a.k_dim + 8 * part;
            const long long from = (long long)(first + r) * stride + (long long)head * a.k_dim + 8 * part;
            u64 e[2][8], mask[2][8];
#pragma unroll
            for (int h = 0; h < 8; h += 2)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    ulonglong2 v = make_ulonglong2(0ull, 0ull), k = v;
                    if (8 * part + h < a.k_dim) {
                        v = attn_input2(x[i] + from + h, a.in_vec);
                        k = attn_load2<VEC>(m[i] + o + h);
                    }
                    e[i][h] = v.x; e[i][h + 1] = v.y;
                    mask[i][h] = k.x; mask[i][h + 1] = k.y;
                }
#pragma unroll
            for (int h = 0; h < 8; h += 2) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    e[i][h] -= mask[i][h];
                    e[i][h + 1] -= mask[i][h + 1];
                    if (8 * part + h < a.k_dim) attn_send2<VEC>(msg[i] + o + h, make_ulonglong2(e[i][h], e[i][h + 1]));
                }
#pragma unroll
                for (int n = h; n < h + 2; ++n) {
                    e[0][n] += e[1][n];                                                                    // the exchange
                    if (query) mask[1][n] += e[0][n];
                }
            }
            const size_t block = block0 + (size_t)(part / 4 * rows16 * attn::ROW_BYTES);
            attn_emit(to.set[0] + block, rows16, t0 + r, part % 4 * 8, e[0]);
            attn_emit(to.set[1] + block, rows16, t0 + r, part % 4 * 8, mask[0]);
            attn_emit(to.set[2] + block, rows16, t0 + r, part % 4 * 8, mask[1]);
        }
    };
    // values or decayed keys, `dim` words a token in tiles of `tile`; tokens behind the last count as zero
    auto open_dims = [&](const u64* const x[2], long long stride, const u64* const m[2], u64* const msg[2], const AttnPlanes& to, int dim, int tile,
                         int head, const u64* w, bool sum) {
        const int all = attn::up16(dim);
        const size_t o0 = ((size_t)first * a.kv_heads + head) * dim, row = (size_t)a.kv_heads * dim;
        for (int t = threadIdx.x; t < 2 * all; t += attn::THREADS) {
            const int r0 = (t >> 4 & 1) * 8, j = (t & 15) + (t >> 5) * 16;
            u64 e[2][8], mask[2][8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = r0 + k;
                    e[i][k] = mask[i][k] = 0ull;
                    if (r < rows && j < dim) {
                        e[i][k] = __ldcs(x[i] + (long long)(first + r) * stride + (long long)head * dim + j);
                        mask[i][k] = __ldcs(m[i] + o0 + r * row + j);
                    }
                }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = r0 + k;
                const u64 weight = w && r < rows ? __ldg(w - r) : 1ull;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (w) e[i][k] = attn_rescale(e[i][k] * weight, i, f);
                    e[i][k] -= mask[i][k];
                    if (r < rows && j < dim) __stcs(msg[i] + o0 + r * row + j, e[i][k]);
                }
                e[0][k] += e[1][k];                                                                        // the exchange
                if (sum) mask[1][k] += e[0][k];
            }
            const int row0 = j / tile * tile, wide = min(tile, all - row0), token = t0 + r0;
            const size_t block = attn_dim_block(attn_before(at, a.kv_heads, head), blocks, token / attn::KC, dim, row0, tile);
            attn_emit(to.set[0] + block, wide, j - row0, token % attn::KC, e[0]);
            attn_emit(to.set[1] + block, wide, j - row0, token % attn::KC, mask[0]);
            attn_emit(to.set[2] + block, wide, j - row0, token % attn::KC, mask[1]);
        }
    };
    const int what = min(3, (int)blockIdx.y / a.kv_heads), h = blockIdx.y - what * a.kv_heads;
    if (what == 0) {
        open_rows(a.K, a.k_stride, a.mk, a.Ek, a.k, a.kv_heads, h, false);
    } else if (what == 1) {
        open_dims(a.K, a.k_stride, a.md, a.Ed, a.d, a.k_dim, attn::RIGHT, h, a.decay + (size_t)h * (a.C + 1) + at.y - 1 - t0, true);
    } else if (what == 2) {
        open_dims(a.V, a.v_stride, a.mv, a.Ev, a.v, a.v_dim, attn::LEFT, h, nullptr, false);
    } else {
        open_rows(a.Q, a.q_stride, a.mq, a.Eq, a.q, a.q_heads, h, true);
        // off the triangle nothing is sent
        const size_t p_row = (size_t)a.q_heads * a.C, p_at = first * p_row + (size_t)h * a.C;
        for (int t = threadIdx.x; t < rows * a.C; t += attn::THREADS) {
            const int r = t / a.C, k = t - r * a.C;
            if (k > t0 + r) a.Ep[0][p_at + r * p_row + k] = a.Ep[1][p_at + r * p_row + k] = 0ull;
        }
    }
}

// ---------------------------------------------------------------------------
// Products: tiles of up to 128 x 64 words of Z_i - C_i = E B_i + V_i F (Eq. 1) on the int8 tensor cores.  A warp copies blocks of planes to shared memory,
// a warp issues the MMAs, sixteen warps read the sums out of tensor memory to shared memory, which gives tensor memory back for the next tile, and
// add them to what comes from memory.  Left operands are keys, values or states, right ones queries, weights or decayed keys; a left operand
// of less than 128 rows has rows behind it that are whatever lies there, whose sums are never looked at.  Sixteen warps read and add, since what
// they add comes from memory: the case took 2 % longer with eight.  One CTA an SM: the eight accumulators of 64 columns are all of an SM's tensor
// memory, so a tile's products wait until the sums before them have gone to shared memory.
// ---------------------------------------------------------------------------
struct AttnOperand {
    const uint8_t* open; const uint8_t* own;             // the first blocks; V_i or the party's mask
    uint32_t bytes;                                      // of a block; the next one lies behind it
};
struct AttnTile {
    AttnOperand left, right;
    int blocks, rows, cols;                              // rows and columns of the result that are looked at
    bool add;                                            // to what the tile before left in shared memory
};
struct AttnShared {
    uint64_t full[attn::SLOTS], empty[attn::SLOTS], acc_full, acc_empty;
    uint32_t tmem;
    int abort_flag;
};
// Pointers of either party.
template <typename T>
__device__ __forceinline__ T* attn_of(T* const (&x)[2], int i) { return i ? x[1] : x[0]; }
__device__ __forceinline__ AttnOperand attn_operand(const AttnPlanes& p, int i, size_t at, int rows) {
    return {p.set[0] + at, (i ? p.set[2] : p.set[1]) + at, (uint32_t)(rows * attn::ROW_BYTES)};
}

// Asks the L2 for `rows` rows of `words` words, `step` words apart: the draining warps, for what they add to the sums while the products run.
__device__ __forceinline__ void attn_ask(const u64* p, int words, int rows, uint32_t step) {
    const int lines = (words + 15) / 16;
    for (int t = threadIdx.x; t < lines * rows; t += attn::DRAIN_THREADS) {
        const int r = t / lines;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(p + (r * step + 16 * (t - r * lines))));
    }
}

// All tiles of a CTA: items blockIdx.x, blockIdx.x + gridDim.x, ..., of an item's `tiles(item)` the tiles tile(item, n); ask(item, n, tile) and then
// drain(item, n, tile, sums) by the draining warps, with the sums at words[column * LEFT + row].  Every role goes through all of them in the same order.
template <typename N, typename T, typename A, typename D>
__device__ __forceinline__ void attn_tiles(uint8_t* raw, int items, int* error, N&& tiles, T&& tile, A&& ask, D&& drain) {
    using namespace attn;
    __shared__ AttnShared s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* const planes = raw + ((0u - ptx::smem_u32(raw)) & 127u);
    u64* const words = reinterpret_cast<u64*>(planes + SLOTS * SLOT_BYTES);
    if (threadIdx.x == 0) {
        for (int k = 0; k < SLOTS; ++k) {
            ptx::mbar_init(ptx::smem_u32(&s.full[k]), 1);
            ptx::mbar_init(ptx::smem_u32(&s.empty[k]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&s.acc_full), 1);
        ptx::mbar_init(ptx::smem_u32(&s.acc_empty), DRAIN_THREADS);
        s.abort_flag = 0;
        ptx::fence_barrier_init();
    }
    __syncwarp();
    if (warp == ISSUER) {
        ptx::tmem_alloc(ptx::smem_u32(&s.tmem), ACC_COLS);
        ptx::tmem_relinquish();
    }
    ptx::fence_before_sync();
    __syncthreads();
    ptx::fence_after_sync();
    const uint32_t tmem = s.tmem, full0 = ptx::smem_u32(&s.full[0]), empty0 = ptx::smem_u32(&s.empty[0]), planes0 = ptx::smem_u32(planes);
    auto settle = [](uint32_t bar, uint32_t parity) {     // a limit of its own: the abort flag is up
        const long long t0 = clock64();
        while (!ptx::mbar_try_wait(bar, parity) && clock64() - t0 < 20000000ll) {}
    };
    if (warp == PRODUCER) {
        if (ptx::elect_one()) {
            int slot = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int item = blockIdx.x; item < items && ok; item += gridDim.x)
                for (int n = 0, count = tiles(item); n < count && ok; ++n) {
                    const AttnTile x = tile(item, n);
                    for (int b = 0; b < 2 * x.blocks; ++b) {
                        ok = limb_wait(empty0 + 8 * slot, phase ^ 1u, &s.abort_flag);
                        if (!ok) break;
                        const uint32_t bar = full0 + 8 * slot, to = planes0 + slot * SLOT_BYTES;
                        const size_t k = b >> 1;
                        ptx::mbar_expect_tx(bar, x.left.bytes + x.right.bytes);
                        ptx::bulk_g2s(to, (b & 1 ? x.left.own : x.left.open) + k * x.left.bytes, x.left.bytes, bar);
                        ptx::bulk_g2s(to + LEFT_BYTES, (b & 1 ? x.right.open : x.right.own) + k * x.right.bytes, x.right.bytes, bar);
                        ++issued;
                        if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
                    }
                }
            // gave up: let the copies already in flight land before the CTA leaves
            for (int j = 1; j <= min(issued, SLOTS) && !ok; ++j) {
                int k = slot - j;
                uint32_t ph = phase;
                if (k < 0) { k += SLOTS; ph ^= 1u; }
                settle(full0 + 8 * k, ph);
            }
        }
    } else if (warp == ISSUER) {
        if (ptx::elect_one()) {
            constexpr uint32_t IDESC = (2u << 4) | ((uint32_t)(LEFT >> 4) << 24);
            const uint32_t acc_full = ptx::smem_u32(&s.acc_full), acc_empty = ptx::smem_u32(&s.acc_empty), left0 = limb_desc_lo(planes0);
            int slot = 0, issued = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true, sums = false;
            for (int item = blockIdx.x; item < items && ok; item += gridDim.x)
                for (int n = 0, count = tiles(item); n < count && ok; ++n) {
                    const AttnTile x = tile(item, n);
                    const uint32_t cols = x.right.bytes / ROW_BYTES, plane = x.left.bytes / (16 * limb::PLANES);
                    ok = limb_wait(acc_empty, acc_phase ^ 1u, &s.abort_flag);
                    if (!ok) break;
                    ptx::fence_after_sync();
                    for (int b = 0; b < 2 * x.blocks; ++b) {
                        ok = limb_wait(full0 + 8 * slot, phase, &s.abort_flag);
                        if (!ok) break;
                        ptx::fence_after_sync();
                        const uint32_t left = left0 + (slot * SLOT_BYTES >> 4), right = left + (LEFT_BYTES >> 4), first = b > 0 ? 1u : 0u;
#pragma unroll
                        for (int i = 0; i < limb::PLANES; ++i) {
                            // left plane p meets right planes 0 .. 7 - p, whose sums lie side by side; wide and narrow instructions alternate, plane 0,
                            // which overwrites all sums, first
                            const int p = i & 1 ? limb::PLANES - 1 - (i >> 1) : i >> 1;
                            const uint32_t wide = cols * (limb::PLANES - p), at = left + p * plane, to = tmem + cols * p, acc = p == 0 ? first : 1u;
                            if (wide > 256) {
                                ptx::mma_i8_keep_a(to, at, LIMB_DESC_HI, right, LIMB_DESC_HI, IDESC | (256u >> 3 << 17), acc);
                                ptx::mma_i8_reuse_a(to + 256, at, LIMB_DESC_HI, right + (256 * KC >> 4), LIMB_DESC_HI, IDESC | ((wide - 256) >> 3 << 17), acc);
                            } else {
                                ptx::mma_i8(to, at, LIMB_DESC_HI, right, LIMB_DESC_HI, IDESC | (wide >> 3 << 17), acc);
                            }
                        }
                        ptx::mma_commit(empty0 + 8 * slot);
                        ++issued;
                        if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
                    }
                    if (!ok) break;
                    ptx::mma_commit(acc_full);
                    sums = true;
                    acc_phase ^= 1u;
                }
            // the last reports of the tensor core have to find this CTA's memory, also where somebody gave up (else the draining warps have seen those of sums)
            for (int j = 1; j <= min(issued, SLOTS); ++j) {
                int k = slot - j;
                uint32_t ph = phase;
                if (k < 0) { k += SLOTS; ph ^= 1u; }
                if (ok) ok = limb_wait(empty0 + 8 * k, ph, &s.abort_flag);
                if (!ok) settle(empty0 + 8 * k, ph);
            }
            if (!ok && sums) settle(acc_full, acc_phase ^ 1u);
        }
    } else {
        auto meet = [&] {
            __syncwarp();                                // (a warp comes to a barrier as a whole)
            asm volatile("bar.sync 1, %0;" ::"n"(DRAIN_THREADS) : "memory");
        };
        uint32_t acc_phase = 0;
        bool ok = true;
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        for (int item = blockIdx.x; item < items; item += gridDim.x)
            for (int n = 0, count = tiles(item); n < count; ++n) {
                const AttnTile x = tile(item, n);
                const int cols = x.right.bytes / ROW_BYTES;
                ask(item, n, x);
                ok = ok && limb_wait_warp(ptx::smem_u32(&s.acc_full), acc_phase, &s.abort_flag);
                acc_phase ^= 1u;
                meet();                                  // the words before have been used
                if (ok) {
                    ptx::fence_after_sync();
                    if (quarter * 32 < x.rows)
                        for (int c = (warp >> 2) * 8; c < x.cols; c += 2 * DRAINERS) {
                            uint32_t d[limb::PLANES][8];
#pragma unroll
                            for (int p = 0; p < limb::PLANES; ++p) ptx::tmem_ld8(lanes + cols * p + c, d[p]);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                u64* const to = words + (c + j) * LEFT + row;
                                *to = limb_recombine(d[0][j], d[1][j], d[2][j], d[3][j], d[4][j], d[5][j], d[6][j], d[7][j]) + (x.add ? *to : 0ull);
                            }
                            __syncwarp();
                        }
                    ptx::fence_before_sync();
                    ptx::mbar_arrive(ptx::smem_u32(&s.acc_empty));
                }
                meet();
                drain(item, n, x, words);
            }
    }
    __syncwarp();
    ptx::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s.abort_flag) {
        *error = 1;
        __threadfence_system();
    }
    __syncwarp();
    if (warp == ISSUER) {
        ptx::fence_after_sync();
        ptx::tmem_dealloc(tmem, ACC_COLS);
    }
}
// Pairs of rows of a tile's sums, U columns of a thread's at a time: load(row, column, U words) for all of them, then done(row, column, sums, U words).
template <int WORDS, int U, typename L, typename F>
__device__ __forceinline__ void attn_finish(u64* words, int rows, int cols, L&& load, F&& done) {
    const int wide = rows > attn::LEFT / 2 ? 6 : 5, row = 2 * (threadIdx.x & ((1 << wide) - 1)), step = attn::DRAIN_THREADS >> wide;
    if (row < rows)
#pragma unroll 1
        for (int c = threadIdx.x >> wide; c < cols; c += U * step) {
            ulonglong2 x[U][WORDS];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < WORDS; ++k) x[u][k] = c + u * step < cols ? load(row, c + u * step, k) : make_ulonglong2(0ull, 0ull);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c + u * step < cols) done(row, c + u * step, reinterpret_cast<ulonglong2*>(words + (c + u * step) * attn::LEFT + row), x[u]);
        }
}

// Items: chunks and key heads, the sums of d v^T, tiles of party, v_dim and k_dim; then chunks and query heads, the weights, a tile a party.  Both only
// need what was opened, so they share a launch: 97 to 102 us for the case, tensor pipe 36 to 42 %, 410 MB.
template <bool VEC>
__global__ void __launch_bounds__(attn::TILE_THREADS, 1)
attn_products_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ uint8_t attn_smem[];
    pdl_wait();
    using namespace attn;
    const int key_items = a.chunks * a.kv_heads, v_tiles = (a.v_dim + LEFT - 1) / LEFT, k_tiles = (a.k_dim + RIGHT - 1) / RIGHT;
    const int t_blocks = blocks(a.C), k_blocks = blocks(a.k_dim);
    attn_tiles(attn_smem, key_items + a.chunks * a.q_heads, a.error, [&](int item) {
        const int c = item < key_items ? item / a.kv_heads : (item - key_items) / a.q_heads;
        return attn_chunk(a, c).y == 0 ? 0 : item < key_items ? 2 * v_tiles * k_tiles : 2;
    }, [&](int item, int n) {
        AttnTile x;
        x.add = false;
        if (item < key_items) {
            const int i = n & 1, vk = n >> 1, vt = vk / k_tiles, v0 = vt * LEFT, k0 = (vk - vt * k_tiles) * RIGHT, c = item / a.kv_heads;
            const int4 found = attn_chunk(a, c);
            const size_t before = attn_before(found, a.kv_heads, item - c * a.kv_heads);
            x.blocks = blocks(found.y);
            x.left = attn_operand(a.v, i, attn_dim_block(before, x.blocks, 0, a.v_dim, v0, LEFT), min(LEFT, up16(a.v_dim) - v0));
            x.right = attn_operand(a.d, i, attn_dim_block(before, x.blocks, 0, a.k_dim, k0, RIGHT), min(RIGHT, up16(a.k_dim) - k0));
            x.rows = min(LEFT, a.v_dim - v0);
            x.cols = min(RIGHT, a.k_dim - k0);
        } else {
            const int ch = item - key_items, c = ch / a.q_heads, hq = ch - c * a.q_heads;
            const int4 found = attn_chunk(a, c);
            x.left = attn_operand(a.k, n, attn_token_block(found, a.kv_heads, hq / (a.q_heads / a.kv_heads), k_blocks, 0), up16(found.y));
            x.right = attn_operand(a.q, n, attn_token_block(found, a.q_heads, hq, k_blocks, 0), up16(found.y));
            x.blocks = k_blocks;
            x.rows = x.cols = found.y;
        }
        return x;
    }, [&](int item, int n, const AttnTile& x) {
        if (item < key_items) {
            const int vk = n >> 1, vt = vk / k_tiles;
            attn_ask(attn_of(a.dv, n & 1) + ((size_t)item * a.k_dim * a.v_dim + (size_t)(vk - vt * k_tiles) * RIGHT * a.v_dim + vt * LEFT), x.rows, x.cols, a.v_dim);
        } else {
            const int ch = item - key_items, c = ch / a.q_heads;
            const uint32_t p_row = (uint32_t)a.q_heads * a.C;
            const size_t p_at = (size_t)a.found[c].x * p_row + (size_t)(ch - c * a.q_heads) * a.C;
            attn_ask(attn_of(a.qk, n) + p_at, x.rows, x.rows, p_row);
            attn_ask(attn_of(a.mp, n) + p_at, x.rows, x.rows, p_row);
        }
    }, [&](int item, int n, const AttnTile& x, u64* words) {
        if (item < key_items) {
            const int i = n & 1, vk = n >> 1, vt = vk / k_tiles, v0 = vt * LEFT, k0 = (vk - vt * k_tiles) * RIGHT;
            const size_t at = (size_t)item * a.k_dim * a.v_dim + (size_t)k0 * a.v_dim + v0;
            const u64* const dv = attn_of(a.dv, i) + at;
            u64* const kv = attn_of(a.kv, i) + at;
            attn_finish<1, 8>(words, x.rows, x.cols, [&](int row, int col, int) { return attn_load2<VEC>(dv + (col * a.v_dim + row)); },
                              [&](int row, int col, const ulonglong2* z, const ulonglong2* y) { attn_store2<VEC>(kv + (col * a.v_dim + row), attn_add(*z, y[0])); });
            return;
        }
        const int ch = item - key_items, c = ch / a.q_heads, hq = ch - c * a.q_heads, h = hq / (a.q_heads / a.kv_heads), i = n, f = a.f;
        const int4 found = attn_chunk(a, c);
        const int len = found.y, rows16 = up16(len);
        const uint32_t p_row = (uint32_t)a.q_heads * a.C;
        const size_t p_at = (size_t)found.x * p_row + (size_t)hq * a.C;
        const uint32_t row0 = (uint32_t)(found.z * 16 * a.q_heads + hq * rows16) * t_blocks;     // of the planes (chunks x heads are 2^24 at most)
        const u64* const qk = attn_of(a.qk, i) + p_at;
        const u64* const mp = attn_of(a.mp, i) + p_at;
        u64* const Ep = attn_of(a.Ep, i) + p_at;
        const u64* const w = a.decay + (size_t)h * (a.C + 1);
        const bool pairs = VEC && a.C % 2 == 0;
        const int quads = 8 * blocks(len);
        for (int t = threadIdx.x; t < len * quads; t += DRAIN_THREADS) {
            const int r = t / quads, quad = t - r * quads, key0 = 4 * quad;
            u64 z[4], m[4], e[4];
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const int key = key0 + j;
                const uint32_t o = r * p_row + key;
                ulonglong2 x0 = make_ulonglong2(0ull, 0ull), x1 = x0, y = x0;
                if (key <= r) {                          // (the second word of a pair may lie off the triangle, and behind an odd row's end)
                    x0 = pairs ? attn_load2<true>(qk + o) : make_ulonglong2(__ldcs(qk + o), key < r ? __ldcs(qk + o + 1) : 0ull);
                    x1 = pairs ? attn_load2<true>(mp + o) : make_ulonglong2(__ldcs(mp + o), key < r ? __ldcs(mp + o + 1) : 0ull);
                    y = *reinterpret_cast<const ulonglong2*>(words + r * LEFT + key);
                }
                z[j] = x0.x + y.x; z[j + 1] = x0.y + y.y;
                m[j] = x1.x;       m[j + 1] = key < r ? x1.y : 0ull;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = key0 + j;
                e[j] = 0ull;
                if (key <= r) e[j] = attn_rescale(attn_rescale(z[j], i, f) * __ldg(w + r - key), i, f) - m[j];
            }
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const int key = key0 + j;
                const uint32_t o = r * p_row + key;
                if (key > r) continue;
                if (pairs) attn_send2<true>(Ep + o, make_ulonglong2(e[j], e[j + 1]));
                else {
                    Ep[o] = e[j];
                    if (key < r) Ep[o + 1] = e[j + 1];
                }
            }
            // party 0's words wait behind the tile's rows, of which there are 64 at most, for the same thread
            u64* const kept = words + r * LEFT + LEFT / 2 + key0;
            const size_t block = (size_t)(row0 + (quad >> 3) * rows16) * ROW_BYTES;
            if (i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    e[j] += kept[j];                     // the exchange
                    m[j] += e[j];
                }
                attn_emit(a.p.set[0] + block, rows16, r, 4 * (quad & 7), e);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) kept[j] = e[j];
            }
            attn_emit((i ? a.p.set[2] : a.p.set[1]) + block, rows16, r, 4 * (quad & 7), m);
        }
    });
}

// Rows of tokens in no chunk, and messages of states that no chunk finds, are set to zero: CTA `part` of a.clears has a window of tokens and every
// a.clears-th of such states.
__device__ __forceinline__ void attn_clear(const AttnArgs& a, int part) {
    using namespace attn;
    __shared__ uint32_t covered[WINDOW / 32];
    __shared__ int there;                                // chunks that there are: the first ones
    const int tid = threadIdx.x, t0 = part * WINDOW, tokens = min(WINDOW, a.tokens - t0);
    for (int k = tid; k < WINDOW / 32; k += STATE_THREADS) covered[k] = 0u;
    if (tid == 0) there = 0;
    __syncthreads();
    int mine = 0;
    for (int c = tid; c < a.chunks; c += STATE_THREADS) {
        const int4 found = attn_chunk(a, c);
        mine += found.y > 0;
        const int b = max(found.x - t0, 0), e = min(found.x + found.y - t0, tokens);
        for (int k = b >> 5; b < e && 32 * k < e; ++k)
            atomicOr(&covered[k], (~0u << max(b - 32 * k, 0)) & (~0u >> (32 - min(e - 32 * k, 32))));
    }
    if (mine) atomicAdd(&there, mine);
    __syncthreads();
    auto zero = [&](u64* const x[2], size_t row, int words) {
        for (int k = tid; k < words; k += STATE_THREADS) x[0][row * words + k] = x[1][row * words + k] = 0ull;
    };
    const int q = a.q_heads * a.k_dim, k = a.kv_heads * a.k_dim, v = a.kv_heads * a.v_dim, p = a.q_heads * a.C, o = a.q_heads * a.v_dim;
    for (int w = 0; 32 * w < tokens; ++w)
        for (uint32_t left = ~covered[w] & (~0u >> (32 - min(tokens - 32 * w, 32))); left; left &= left - 1) {
            const size_t t = t0 + 32 * w + __ffs(left) - 1;
            zero(a.Eq, t, q);
            zero(a.Ek, t, k);
            zero(a.Ed, t, k);
            zero(a.Ev, t, v);
            zero(a.Ep, t, p);
            zero(a.O, t, o);
        }
    for (int c = there + part; c < a.chunks; c += a.clears) zero(a.Es, c, k * a.v_dim);
}

// The state from chunk to chunk of a sequence and key head, four words of a column and both parties a thread; says whether the starts were in order.
// Bound by memory: the next chunk's words are on their way while this one's are worked on.  50 us for the case, 290 MB (5.8 TB/s).  Carried along by
// the kernel of the products, tile by tile in shared memory, it saved the 134 MB of sums, but left few warps an SM to wait for memory: 152 us for both, where
// the two kernels took 146.
__global__ void __launch_bounds__(attn::STATE_THREADS)
attn_state_kernel(const __grid_constant__ AttnArgs a, int pieces) {
    pdl_wait();
    const int block = (int)blockIdx.x - a.clears;        // (the others are the first ones to begin)
    if (block < 0) {
        attn_clear(a, blockIdx.x);
        return;
    }
    const int j = block / (a.kv_heads * pieces), rest = block - j * a.kv_heads * pieces, h = rest / pieces;
    const int t = (rest - h * pieces) * attn::STATE_THREADS + threadIdx.x, k_blocks = attn::blocks(a.k_dim), wide = attn::up16(a.v_dim);
    // the sequence's first chunk: the first one whose owner it, or a later one, is
    int c = 0, top = a.chunks;
    while (c < top) {
        const int step = (top - c + attn::STATE_THREADS - 1) / attn::STATE_THREADS, at = c + threadIdx.x * step;
        const int n = __syncthreads_count(at < top && attn_owner(a, at) < j);
        if (n == 0) break;
        top = min(top, c + n * step);
        c += (n - 1) * step + 1;
    }
    int begin;
    const int own = (attn_length(a, j, &begin) + a.C - 1) / a.C, end = min(a.chunks, c + own);
    if (rest == 0 && threadIdx.x == 0 && a.bad_starts) {
        const int last = a.starts[j + 1];
        // out of order; more chunks than there are to be; fewer
        if (begin < 0 || last < begin || last > a.tokens || c + own > a.chunks || (j == 0 && a.chunks > 0 && attn_owner(a, a.chunks - 1) == attn::NOBODY)) *a.bad_starts = 1;
    }
    // a warp has four groups of four rows, eight columns: 64 bytes of a row, 128 of a plane
    const int groups = wide / 8, wt = t >> 5, quad = (wt / groups) * 4 + (t >> 3 & 3), col = (wt % groups) * 8 + (t & 7);
    if (quad >= 8 * k_blocks) return;
    const int words = a.k_dim * a.v_dim, row = 4 * quad, word = row * a.v_dim + col;
    const size_t at = ((size_t)j * a.kv_heads + h) * words + word, step = (size_t)a.kv_heads * words;
    const u64* const w = a.decay + (size_t)h * (a.C + 1);
    u64 S[2][4], kv[2][4], ms[2][4];
    size_t o = ((size_t)c * a.kv_heads + h) * words + word;
    auto live = [&](int k) { return col < a.v_dim && row + k < a.k_dim; };
    int len = 0;                                         // of the chunk; none where it had no room: then it and those behind it are not worked out
    auto load = [&](int chunk) {
        len = attn_chunk(a, chunk).y;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                kv[i][k] = live(k) ? __ldcs(a.kv[i] + o + k * a.v_dim) : 0ull;
                ms[i][k] = live(k) ? __ldcs(a.ms[i] + o + k * a.v_dim) : 0ull;
            }
    };
    if (c < end) load(c);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) S[i][k] = a.S0[i] && live(k) ? __ldcs(a.S0[i] + at + k * a.v_dim) : 0ull;
    const int row0 = col / attn::LEFT * attn::LEFT, rows = min(attn::LEFT, wide - row0);
    for (; c < end && len > 0; ++c) {
        const u64 weight = __ldg(w + len);
        const size_t here = o, block = attn_dim_block(((size_t)c * a.kv_heads + h) * k_blocks, k_blocks, quad >> 3, a.v_dim, row0, attn::LEFT);
        attn_emit(a.s.set[1] + block, rows, col - row0, 4 * (quad & 7), ms[0]);
        attn_emit(a.s.set[2] + block, rows, col - row0, 4 * (quad & 7), ms[1]);
        u64 e[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                e[i][k] = S[i][k] - ms[i][k];
                S[i][k] = attn_rescale(weight * S[i][k] + kv[i][k], i, a.f);
            }
        o += step;
        if (c + 1 < end) load(c + 1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (live(k)) __stcs(a.Es[i] + here + k * a.v_dim, e[i][k]);
            e[0][k] += e[1][k];                              // the exchange
        }
        attn_emit(a.s.set[0] + block, rows, col - row0, 4 * (quad & 7), e[0]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (live(k)) a.S1[i][at + k * a.v_dim] = S[i][k];
}

// Items: chunks, query heads and parties, the rows of O: for every tile of v_dim the far part w[r + 1] tr(q S), then the near part P v, which is added to what
// the far part left in shared memory.  81 to 84 us for the case, tensor pipe 34 to 40 %, 360 MB.
template <bool VEC>
__global__ void __launch_bounds__(attn::TILE_THREADS, 1)
attn_rows_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ uint8_t attn_smem[];
    pdl_wait();
    using namespace attn;
    const int v_tiles = (a.v_dim + LEFT - 1) / LEFT, t_blocks = blocks(a.C), k_blocks = blocks(a.k_dim);
    attn_tiles(attn_smem, 2 * a.chunks * a.q_heads, a.error, [&](int item) { return attn_chunk(a, (item >> 1) / a.q_heads).y == 0 ? 0 : 2 * v_tiles; },
               [&](int item, int n) {
        const int i = item & 1, ch = item >> 1, c = ch / a.q_heads, hq = ch - c * a.q_heads, h = hq / (a.q_heads / a.kv_heads);
        const int v0 = (n >> 1) * LEFT, wide = min(LEFT, up16(a.v_dim) - v0);
        const int4 found = attn_chunk(a, c);
        AttnTile x;
        x.add = n & 1;
        if (n & 1) {
            x.blocks = blocks(found.y);
            x.left = attn_operand(a.v, i, attn_dim_block(attn_before(found, a.kv_heads, h), x.blocks, 0, a.v_dim, v0, LEFT), wide);
            x.right = attn_operand(a.p, i, attn_token_block(found, a.q_heads, hq, t_blocks, 0), up16(found.y));
        } else {
            x.blocks = k_blocks;
            x.left = attn_operand(a.s, i, attn_dim_block(((size_t)c * a.kv_heads + h) * k_blocks, k_blocks, 0, a.v_dim, v0, LEFT), wide);
            x.right = attn_operand(a.q, i, attn_token_block(found, a.q_heads, hq, k_blocks, 0), up16(found.y));
        }
        x.rows = min(LEFT, a.v_dim - v0);
        x.cols = found.y;
        return x;
    }, [&](int item, int n, const AttnTile& x) {
        if (n & 1) return;
        const int ch = item >> 1, c = ch / a.q_heads;
        const uint32_t o_row = (uint32_t)a.q_heads * a.v_dim;
        const size_t at = (size_t)a.found[c].x * o_row + (size_t)(ch - c * a.q_heads) * a.v_dim + (n >> 1) * LEFT;
        attn_ask(attn_of(a.qs, item & 1) + at, x.rows, x.cols, o_row);
        attn_ask(attn_of(a.pv, item & 1) + at, x.rows, x.cols, o_row);
    }, [&](int item, int n, const AttnTile& x, u64* words) {
        const int i = item & 1, ch = item >> 1, c = ch / a.q_heads, hq = ch - c * a.q_heads, h = hq / (a.q_heads / a.kv_heads), f = a.f;
        const uint32_t o_row = (uint32_t)a.q_heads * a.v_dim;
        const size_t at = (size_t)a.found[c].x * o_row + (size_t)hq * a.v_dim + (n >> 1) * LEFT;
        if (n & 1) {
            u64* const O = attn_of(a.O, i) + at;
            attn_finish<1, 1>(words, x.rows, x.cols, [&](int, int, int) { return make_ulonglong2(0ull, 0ull); }, [&](int row, int r, const ulonglong2* z, const ulonglong2*) {
                attn_send2<VEC>(O + (r * o_row + row), make_ulonglong2(attn_rescale(z->x, i, f), attn_rescale(z->y, i, f)));
            });
        } else {
            const u64* const qs = attn_of(a.qs, i) + at;
            const u64* const pv = attn_of(a.pv, i) + at;
            const u64* const w = a.decay + (size_t)h * (a.C + 1) + 1;
            attn_finish<2, 4>(words, x.rows, x.cols, [&](int row, int r, int k) { return attn_load2<VEC>((k ? pv : qs) + (r * o_row + row)); },
                              [&](int, int r, ulonglong2* z, const ulonglong2* y) {
                const u64 weight = __ldg(w + r);
                *z = make_ulonglong2(y[1].x + weight * attn_rescale(z->x + y[0].x, i, f), y[1].y + weight * attn_rescale(z->y + y[0].y, i, f));
            });
        }
    });
}

// ---------------------------------------------------------------------------
// Single tokens.  Bound by memory: of every word of a state and party five words, the state, its mask and the product in, the message
// and the new state out.  A CTA has both parties' words of a slice of a state's columns, a thread one pair of columns in every
// row_groups-th row, so every word passes once through the thread that exchanges it; q and k lie in shared memory, what they
// are multiplied with as they are needed.  The sums of o are added up over the row groups at the end.  32 sequences x 32 heads of 128 x 128: 237 us, 0.88
// of the measured copy rate; one sequence of 12 heads of 64 5.5 us, seven of 10 heads on 2 of 80 x 96 9.7 (the call, 16, is the host's).
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
