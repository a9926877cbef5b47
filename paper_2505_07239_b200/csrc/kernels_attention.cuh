// Linear attention with a decay for every head on additive shares (comet_linear_attention, comet_linear_attention_step): products and
// public weights only, so that it needs no comparison.  f the fixed point, i the party, tr the local truncation by f bits, w[n] the public
// n-th power of a key head's decay, P, S, q, k, v, d shared; every value that enters a product is masked and opened once.
//   a prompt, in chunks; of a chunk of L tokens that finds the state S:
//     P[r][s] = tr(w[r - s] tr(q_r . k_s)), s <= r;   O_r = tr(sum_{s <= r} P[r][s] v_s + w[r + 1] tr(q_r S))
//     d_s = tr(w[L - 1 - s] k_s);                     S <- tr(w[L] S + sum_s d_s v_s^T)
//   single tokens:  S <- tr(w S + k v^T),  o = tr(q S)
// Three kernels for a prompt, because only the states depend on one another: the products d v^T of all chunks and key heads at once
// (keys), the states from chunk to chunk, a word a thread (state), then everything else of all chunks and query heads (rows).
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
constexpr int THREADS = 256;                         // of the kernels without products
constexpr int ROWS = 128, TILE = 64;                 // of a tile of a product: rows, columns
constexpr int GROUP = 8;                             // warps that convert one of the two products
constexpr int CONVERTERS = 2 * GROUP, DRAINERS = 8, WORKERS = 32 * (CONVERTERS + DRAINERS), ISSUER = CONVERTERS + DRAINERS;
constexpr int TILE_THREADS = WORKERS + 32;
constexpr int SLOTS = 3;                             // of planes: one of the two products of 32 indices each
constexpr int LEFT_PLANE = ROWS * limb::KC, RIGHT_PLANE = TILE * limb::KC, LEFT_BYTES = limb::PLANES * LEFT_PLANE;
constexpr int SLOT_BYTES = LEFT_BYTES + limb::PLANES * RIGHT_PLANE, ACC_COLS = limb::PLANES * TILE;
constexpr int CELL_ROWS = 32;                        // rows that a group covers at a time
constexpr int AHEAD = 3, BATCH = 4;                  // a draining thread's dealer's words: batches of columns under way, columns of one
constexpr int RING_BYTES = AHEAD * BATCH * 2 * 32 * DRAINERS * 8, TILE_SMEM = SLOTS * SLOT_BYTES + RING_BYTES + 128;
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
    u64* p; u64* pm[2];                                                  // opened weights and their masks, zero off the triangle
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
    const int b = __ldg(a.starts + j), e = __ldg(a.starts + j + 1);
    *begin = b;
    return b >= 0 && b <= e && e <= a.tokens ? e - b : 0;
}

struct AttnChunk {
    int seq, first, len;                                                 // len 0: there is no such chunk
};

// Chunk `want` of all sequences', by all threads of a CTA.
__device__ __forceinline__ AttnChunk attn_find(const AttnArgs& a, int want) {
    __shared__ AttnChunk found;
    __shared__ int sums[attn::TILE_THREADS / 32];
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
__device__ __forceinline__ ulonglong2 attn_load2(const u64* p) {         // words that nobody else reads
    if (VEC) return __ldcs(reinterpret_cast<const ulonglong2*>(p));
    return make_ulonglong2(__ldcs(p), __ldcs(p + 1));
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
// Products on the int8 tensor cores.  A CTA works out tiles of ROWS x TILE words of Z_i = (triple) + E B_i + V_i F, V_i = A_i + i E (Eq. 1), one
// party's after the other's, from words in memory, masks and opened values: two groups of eight warps turn 32 contraction indices of one product each
// into limb planes in shared memory (kernels_limb.cuh has the decomposition and the layout), a warp issues the MMAs, eight warps read the sums out
// of tensor memory.  Left operands are keys, values or states, right ones queries, weights or decayed keys; rows past an operand's are whatever lies
// in shared memory, and their sums are never looked at.
// ---------------------------------------------------------------------------
struct AttnOperand {
    const u64* mask;                     // the party's
    const u64* open;                     // the opened value
    uint32_t step;                       // words from row to row; of a DEEP operand, whose rows lie side by side, from index to index
};
enum AttnWords { MASK, OPEN, BOTH };     // of a plane set: the mask, the opened value, their sum

// A thread's cells of the planes of `rows` rows: four words of a row, indices 2g, 2g + 1, 16 + 2g, 17 + 2g of every 32 (limb_emit4's order), TASKS of
// them, CELL_ROWS rows apart.  Places are counted in 32 bits: an operand spans less than 2^29 words (comet_linear_attention sees to that).
template <bool DEEP, int TASKS>
struct AttnCells {
    uint32_t at;                                 // of the first word, from the operand's on
    int to, row, g;                              // to: in a plane

    __device__ __forceinline__ AttnCells(const AttnOperand& x) {
        const int warp = (threadIdx.x >> 5) % attn::GROUP, lane = threadIdx.x & 31;
        if (DEEP) {
            // eight rows x four groups of indices a warp: 64-byte pieces of memory, 128 bytes of a plane
            row = (warp >> 1) * 8 + (lane & 7);
            g = (warp & 1) * 4 + (lane >> 3);
        } else {
            // lanes of the upper groups take the row four further, against bank conflicts
            g = lane & 7;
            row = 4 * (2 * (warp >> 1) + ((warp & 1) ^ (g >> 2))) + (lane >> 3);
        }
        to = (row >> 3) * 256 + (g >> 2) * 128 + (row & 7) * 16 + (g & 3) * 4;
        at = DEEP ? 2 * g * x.step + row : row * x.step + 2 * g;
    }
    // Of the 32 indices from k0 on; those from `depth` on are zero.
    template <AttnWords WHAT, bool VEC>
    __device__ __forceinline__ void read(const AttnOperand& x, u64 (&w)[TASKS][4], int rows, int k0, int depth) const {
        const uint32_t from = at + (DEEP ? k0 * x.step : k0);
        const int left = depth - k0 - 2 * g;
#pragma unroll
        for (int t = 0; t < TASKS; ++t) {
            const bool live = row + t * attn::CELL_ROWS < rows;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u64 v[2] = {0ull, 0ull};
                if (!DEEP && VEC) {              // (rows are even in length, zero behind an odd depth)
                    if (live && 16 * h < left) {
                        const uint32_t o = from + 16 * h + t * attn::CELL_ROWS * x.step;
                        if (WHAT != MASK) {
                            const ulonglong2 e = *reinterpret_cast<const ulonglong2*>(x.open + o);
                            v[0] = e.x;
                            v[1] = e.y;
                        }
                        if (WHAT != OPEN) {
                            const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(x.mask + o);
                            v[0] += m.x;
                            v[1] += m.y;
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (live && 16 * h + j < left) {
                            const uint32_t o = from + (DEEP ? x.step : 1u) * (16 * h + j) + t * attn::CELL_ROWS * (DEEP ? 1u : x.step);
                            if (WHAT != MASK) v[j] = x.open[o];
                            if (WHAT != OPEN) v[j] += x.mask[o];
                        }
                }
                w[t][2 * h] = v[0];
                w[t][2 * h + 1] = v[1];
            }
        }
    }
    __device__ __forceinline__ void emit(uint8_t* planes, int plane_bytes, const u64 (&w)[TASKS][4], int rows) const {
#pragma unroll
        for (int t = 0; t < TASKS; ++t)
            if (row + t * attn::CELL_ROWS < rows) limb_emit4(planes + to + t * (attn::CELL_ROWS / 8 * 256), plane_bytes, w[t]);
    }
};

// What a CTA's warps share.
struct AttnTile {
    uint64_t full[attn::SLOTS], empty[attn::SLOTS], acc_full, acc_empty, weights;
    uint32_t tmem;
    int abort_flag;
    uint8_t* planes;
};
__device__ __forceinline__ void attn_tile_begin(AttnTile& s, uint8_t* raw) {
    if (threadIdx.x == 0) {
        for (int k = 0; k < attn::SLOTS; ++k) {
            ptx::mbar_init(ptx::smem_u32(&s.full[k]), attn::GROUP);
            ptx::mbar_init(ptx::smem_u32(&s.empty[k]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&s.acc_full), 1);
        ptx::mbar_init(ptx::smem_u32(&s.acc_empty), attn::DRAINERS);
        ptx::mbar_init(ptx::smem_u32(&s.weights), attn::DRAINERS);
        s.abort_flag = 0;
        s.planes = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
        ptx::fence_barrier_init();
    }
    __syncwarp();
    if (threadIdx.x >> 5 == attn::ISSUER) {
        ptx::tmem_alloc(ptx::smem_u32(&s.tmem), attn::ACC_COLS);
        ptx::tmem_relinquish();
    }
    ptx::fence_before_sync();
    __syncthreads();
    ptx::fence_after_sync();
}
// All warps but the issuer wait for one another.  (A warp comes to a barrier, and to a read of tensor memory, as a whole: both are
// undefined for lanes on their own, and what stands before may have parted them.)
__device__ __forceinline__ void attn_meet() {
    __syncwarp();
    asm volatile("bar.sync 1, %0;" ::"n"(attn::WORKERS) : "memory");
}

// Bounded wait, written out where it stands: false, and the CTA's abort flag raised, if the barrier did not flip in time or another warp has given up.
// Not a call: loads and asynchronous copies are under way when a warp comes to wait here.
__device__ __forceinline__ bool attn_wait(uint64_t& bar, uint32_t parity, AttnTile& s) {
    const uint32_t at = ptx::smem_u32(&bar);
    bool ok = ptx::mbar_try_wait(at, parity);
    if (!ok) {
        const long long t0 = clock64();
        volatile int* const abort_flag = &s.abort_flag;
        do {
            ok = ptx::mbar_try_wait(at, parity);
            if (!ok && (*abort_flag || clock64() - t0 > limb::WAIT_CYCLES)) {
                *abort_flag = 1;
                break;
            }
        } while (!ok);
    }
    return ok;
}
// The same for a whole warp.
__device__ __forceinline__ bool attn_wait_warp(uint64_t& bar, uint32_t parity, AttnTile& s) {
    return __all_sync(0xffffffffu, attn_wait(bar, parity, s));
}

// Where a warp is in the order of slots and tiles; all count alike.
struct AttnTurn {
    uint32_t stage = 0, tile = 0;
    bool ok = true;
};
__device__ __forceinline__ int attn_blocks(int depth) { return (depth + limb::KC - 1) / limb::KC; }

// The end of a CTA.  What the tensor core still owes is waited for first: the last stages' slots, which nobody uses again, are reported free through
// shared memory, and a report that comes when the CTA is gone is an access to an address that does not exist.  (It happened, where the last sums were
// drained fast enough.)
__device__ __forceinline__ void attn_tile_end(AttnTile& s, const AttnTurn& turn, int* error) {
    __syncwarp();
    if (threadIdx.x >> 5 == attn::ISSUER && turn.ok)
        for (uint32_t k = 1; k <= attn::SLOTS && k <= turn.stage; ++k) {
            const uint32_t n = turn.stage - k;
            attn_wait(s.empty[n % attn::SLOTS], n / attn::SLOTS & 1u, s);
        }
    __syncwarp();
    ptx::fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s.abort_flag) {
        *error = 1;
        __threadfence_system();
    }
    __syncwarp();
    if (threadIdx.x >> 5 == attn::ISSUER) {
        ptx::fence_after_sync();
        ptx::tmem_dealloc(s.tmem, attn::ACC_COLS);
    }
}

// The issuing warp's part of a tile.
__device__ __forceinline__ void attn_issue(AttnTile& s, AttnTurn& turn, int depth) {
    const int stages = 2 * attn_blocks(depth);
    __syncwarp();
    if (ptx::elect_one() && turn.ok) {
        constexpr uint32_t IDESC = (2u << 4) | ((uint32_t)(attn::ROWS >> 4) << 24);
        bool ok = attn_wait(s.acc_empty, (turn.tile & 1u) ^ 1u, s);
        ptx::fence_after_sync();
        for (int t = 0; t < stages && ok; ++t) {
            const uint32_t n = turn.stage + t, slot = n % attn::SLOTS;
            ok = attn_wait(s.full[slot], n / attn::SLOTS & 1u, s);
            if (!ok) break;
            ptx::fence_after_sync();
            const uint32_t left = limb_desc_lo(ptx::smem_u32(s.planes) + slot * attn::SLOT_BYTES), right = left + (attn::LEFT_BYTES >> 4);
            const uint32_t acc = t > 0 ? 1u : 0u;
#pragma unroll
            for (int i = 0; i < limb::PLANES; ++i) {
                // wide and narrow instructions alternate, plane 0, which overwrites all sums, first
                const int p = i & 1 ? limb::PLANES - 1 - (i >> 1) : i >> 1, n_total = attn::TILE * (limb::PLANES - p);
                const uint32_t at = left + (p * attn::LEFT_PLANE >> 4), acc_p = p == 0 ? acc : 1u;
                if (n_total > 256) {
                    ptx::mma_i8_keep_a(s.tmem + attn::TILE * p, at, LIMB_DESC_HI, right, LIMB_DESC_HI, IDESC | (256u >> 3 << 17), acc_p);
                    ptx::mma_i8_reuse_a(s.tmem + attn::TILE * p + 256, at, LIMB_DESC_HI, right + (256 * limb::KC >> 4), LIMB_DESC_HI,
                                        IDESC | ((uint32_t)(n_total - 256) >> 3 << 17), acc_p);
                } else {
                    ptx::mma_i8(s.tmem + attn::TILE * p, at, LIMB_DESC_HI, right, LIMB_DESC_HI, IDESC | ((uint32_t)n_total >> 3 << 17), acc_p);
                }
            }
            ptx::mma_commit(ptx::smem_u32(&s.empty[slot]));
        }
        if (ok) ptx::mma_commit(ptx::smem_u32(&s.acc_full));
        turn.ok = ok;
    }
    turn.stage += stages;
    ++turn.tile;
}
// The converting warps' part: planes of both products, 32 indices at a time, E B_i by the first group, V_i F by the second.  A stage's words are asked
// for before the wait for its slot, and while one group waits for its words the other puts its own away.
template <bool DEEP_LEFT, bool DEEP_RIGHT, bool VEC>
__device__ __forceinline__ void attn_convert(AttnTile& s, AttnTurn& turn, const AttnOperand& left, int rows, const AttnOperand& right, int cols, int depth,
                                             int party) {
    constexpr int LEFT = DEEP_LEFT ? 4 : 2, RIGHT = 2;       // up to ROWS rows of a deep left operand, MAX_CHUNK of another; TILE rows of a right one
    const int lane = threadIdx.x & 31, second = threadIdx.x / (32 * attn::GROUP);
    const AttnCells<DEEP_LEFT, LEFT> l(left);
    const AttnCells<DEEP_RIGHT, RIGHT> r(right);
#pragma unroll 1
    for (int k0 = 0; k0 < depth; k0 += limb::KC) {
        u64 lw[LEFT][4], rw[RIGHT][4];
        if (second == 0) {
            l.template read<MASK, VEC>(left, lw, rows, k0, depth);
            r.template read<OPEN, VEC>(right, rw, cols, k0, depth);
        } else {
            l.template read<OPEN, VEC>(left, lw, rows, k0, depth);
            if (party) r.template read<BOTH, VEC>(right, rw, cols, k0, depth);
            else r.template read<MASK, VEC>(right, rw, cols, k0, depth);
        }
        const uint32_t n = turn.stage + second, slot = n % attn::SLOTS;
        turn.stage += 2;
        turn.ok = turn.ok && attn_wait_warp(s.empty[slot], (n / attn::SLOTS & 1u) ^ 1u, s);
        if (!turn.ok) continue;
        uint8_t* const at = s.planes + slot * attn::SLOT_BYTES;
        l.emit(at, attn::LEFT_PLANE, lw, rows);
        r.emit(at + attn::LEFT_BYTES, attn::RIGHT_PLANE, rw, cols);
        ptx::fence_proxy_async_smem();                       // the planes are read by the tensor cores
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&s.full[slot]));
    }
}
// Four columns of the eight accumulators, loads and wait in one statement: until the wait is over the hardware may write the registers at any
// time, so nothing may be moved out of them or put into their place before it.
__device__ __forceinline__ void attn_sums(uint32_t at, uint32_t (&d)[limb::PLANES][4]) {
    constexpr int N = attn::TILE;
    __syncwarp();
    asm volatile(
        "{\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%4, %5, %6, %7}, [%33];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%8, %9, %10, %11}, [%34];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%12, %13, %14, %15}, [%35];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%16, %17, %18, %19}, [%36];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%20, %21, %22, %23}, [%37];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%24, %25, %26, %27}, [%38];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%28, %29, %30, %31}, [%39];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n\t}"
        : "=&r"(d[0][0]), "=&r"(d[0][1]), "=&r"(d[0][2]), "=&r"(d[0][3]), "=&r"(d[1][0]), "=&r"(d[1][1]), "=&r"(d[1][2]), "=&r"(d[1][3]),
          "=&r"(d[2][0]), "=&r"(d[2][1]), "=&r"(d[2][2]), "=&r"(d[2][3]), "=&r"(d[3][0]), "=&r"(d[3][1]), "=&r"(d[3][2]), "=&r"(d[3][3]),
          "=&r"(d[4][0]), "=&r"(d[4][1]), "=&r"(d[4][2]), "=&r"(d[4][3]), "=&r"(d[5][0]), "=&r"(d[5][1]), "=&r"(d[5][2]), "=&r"(d[5][3]),
          "=&r"(d[6][0]), "=&r"(d[6][1]), "=&r"(d[6][2]), "=&r"(d[6][3]), "=&r"(d[7][0]), "=&r"(d[7][1]), "=&r"(d[7][2]), "=&r"(d[7][3])
        : "r"(at), "r"(at + N), "r"(at + 2 * N), "r"(at + 3 * N), "r"(at + 4 * N), "r"(at + 5 * N), "r"(at + 6 * N), "r"(at + 7 * N)
        : "memory");
}
// The draining warps' part: the sums of this thread's row, a batch of columns after the other: done(row, column, sum, words, own).  The dealer's
// words, at(k, row, column) the place of the k-th, come into the thread's own places of shared memory AHEAD batches before they are needed, the
// first before the wait for the sums; a word that the thread itself has written, own(row, column), one batch before.
template <int WORDS, typename P, typename O, typename F>
__device__ __forceinline__ void attn_drain(AttnTile& s, AttnTurn& turn, int rows, int cols, P&& at, O&& own, F&& done) {
    using namespace attn;
    const int thread = threadIdx.x - 32 * CONVERTERS, quarter = (thread >> 5) & 3, row = thread & (ROWS - 1);
    const int c0 = thread / ROWS * (TILE / 2), c1 = min(cols, c0 + TILE / 2);                // a half of the columns
    u64* const ring = reinterpret_cast<u64*>(s.planes + SLOTS * SLOT_BYTES) + thread;       // [AHEAD][BATCH][2][threads]
    constexpr int NEXT = 32 * DRAINERS;
    auto fetch = [&](int c) {
        u64* const to = ring + (c / BATCH % AHEAD) * (BATCH * 2 * NEXT);
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
            if (row < rows && c + j < c1)
#pragma unroll
                for (int k = 0; k < WORDS; ++k) {
                    const u64* const from = at(k, row, c + j);
                    if (from) norm_fetch8(to + (2 * j + k) * NEXT, from);
                }
        limb_copy_commit();
    };
    u64 mine[BATCH];
    auto owned = [&](int c) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j) mine[j] = row < rows && c + j < c1 ? own(row, c + j) : 0ull;
    };
    if (WORDS)
#pragma unroll
        for (int b = 0; b < AHEAD; ++b) fetch(c0 + b * BATCH);
    owned(c0);
    __syncwarp();
    turn.ok = turn.ok && attn_wait_warp(s.acc_full, turn.tile & 1u, s);
    ++turn.tile;
    if (turn.ok) {
        ptx::fence_after_sync();
        const uint32_t acc = s.tmem + ((uint32_t)(quarter * 32) << 16);
        if (quarter * 32 < rows) {
#pragma unroll 1
            for (int c = c0; c < c1; c += BATCH) {
                uint32_t d[limb::PLANES][4];
                attn_sums(acc + c, d);
                if (WORDS) limb_copy_wait<AHEAD - 1>();
                u64 here[BATCH], z[BATCH], words[BATCH][WORDS ? WORDS : 1];
                const u64* const from = ring + (c / BATCH % AHEAD) * (BATCH * 2 * NEXT);
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    z[j] = limb_recombine(d[0][j], d[1][j], d[2][j], d[3][j], d[4][j], d[5][j], d[6][j], d[7][j]);
                    here[j] = mine[j];
#pragma unroll
                    for (int k = 0; k < WORDS; ++k) words[j][k] = from[(2 * j + k) * NEXT];
                }
                owned(c + BATCH);
#pragma unroll
                for (int j = 0; j < BATCH; ++j)
                    if (row < rows && c + j < c1) done(row, c + j, z[j], words[j], here[j]);
                if (WORDS) fetch(c + AHEAD * BATCH);             // (the words have been read)
            }
        }
        ptx::fence_before_sync();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(ptx::smem_u32(&s.acc_empty));
    }
    if (WORDS) limb_copy_wait<0>();
}

__device__ __forceinline__ u64 attn_nothing(int, int) { return 0ull; }

// The pairs of words of `rows` rows of `cols`, two at a time a thread of the WORKERS: load(n, row, column) for both, then finish(n, row, column).
template <typename L, typename F>
__device__ __forceinline__ void attn_pairs(int rows, int cols, L&& load, F&& finish) {
    const int half = cols / 2, all = rows * half;
    for (int t = threadIdx.x; t < all; t += 2 * attn::WORKERS) {
        int r[2], j[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int u = t + n * attn::WORKERS;
            r[n] = u < all ? u / half : -1;
            j[n] = 2 * (u - r[n] * half);
            if (r[n] >= 0) load(n, r[n], j[n]);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
            if (r[n] >= 0) finish(n, r[n], j[n]);
    }
}

// Messages of k, v and d of one chunk and key head, and its sum of d v^T.
template <bool VEC>
__global__ void __launch_bounds__(attn::TILE_THREADS, 1)
attn_keys_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ uint8_t attn_smem[];
    __shared__ AttnTile s;
    pdl_wait();
    pdl_launch_dependents();
    const int c = blockIdx.x / a.kv_heads, h = blockIdx.x - c * a.kv_heads, warp = threadIdx.x >> 5;
    const AttnChunk at = attn_find(a, c);
    if (at.len == 0) return;
    attn_tile_begin(s, attn_smem);
    AttnTurn turn;
    const size_t k_row = (size_t)a.kv_heads * a.k_dim, v_row = (size_t)a.kv_heads * a.v_dim;
    const size_t k_at = at.first * k_row + (size_t)h * a.k_dim, v_at = at.first * v_row + (size_t)h * a.v_dim;
    if (warp != attn::ISSUER) {
        const u64* const w = a.decay + (size_t)h * (a.C + 1) + at.len - 1;
        ulonglong2 x[2][2], mk[2][2], md[2][2];
        attn_pairs(at.len, a.k_dim, [&](int n, int r, int j) {
            const size_t o = k_at + r * k_row + j, x_at = (size_t)(at.first + r) * a.k_stride + (size_t)h * a.k_dim + j;
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
                attn_store2<VEC>(a.Ek[i] + o, e[i]);
                attn_store2<VEC>(a.Ed[i] + o, g[i]);
            }
            attn_store2<VEC>(a.k + o, attn_add(e[0], e[1]));         // the exchange
            attn_store2<VEC>(a.d + o, attn_add(g[0], g[1]));
        });
        attn_pairs(at.len, a.v_dim, [&](int n, int r, int j) {
            const size_t o = v_at + r * v_row + j, x_at = (size_t)(at.first + r) * a.v_stride + (size_t)h * a.v_dim + j;
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
                attn_store2<VEC>(a.Ev[i] + o, e[i]);
            }
            attn_store2<VEC>(a.v + o, attn_add(e[0], e[1]));
        });
        attn_meet();
    }
    // the tiles of either party, the same order for every role
    auto tiles = [&](auto&& tile) {
#pragma unroll 1
        for (int i = 0; i < 2; ++i)
#pragma unroll 1
            for (int v0 = 0; v0 < a.v_dim; v0 += attn::ROWS)
#pragma unroll 1
                for (int k0 = 0; k0 < a.k_dim; k0 += attn::TILE) tile(i, v0, k0, min(attn::ROWS, a.v_dim - v0), min(attn::TILE, a.k_dim - k0));
    };
    if (warp == attn::ISSUER) {
        tiles([&](int, int, int, int, int) { attn_issue(s, turn, at.len); });
    } else if (warp < attn::CONVERTERS) {
        tiles([&](int i, int v0, int k0, int rows, int cols) {
            const AttnOperand v = {a.mv[i] + v_at + v0, a.v + v_at + v0, (uint32_t)v_row}, d = {a.md[i] + k_at + k0, a.d + k_at + k0, (uint32_t)k_row};
            attn_convert<true, true, VEC>(s, turn, v, rows, d, cols, at.len, i);
        });
    } else {
        const size_t out = ((size_t)c * a.kv_heads + h) * a.k_dim * a.v_dim;
        tiles([&](int i, int v0, int k0, int rows, int cols) {
            const u64* const dv = a.dv[i] + out + (size_t)k0 * a.v_dim + v0;
            u64* const kv = a.kv[i] + out + (size_t)k0 * a.v_dim + v0;
            attn_drain<1>(s, turn, rows, cols, [&](int, int row, int col) { return dv + col * a.v_dim + row; }, attn_nothing,
                          [&](int row, int col, u64 z, const u64* words, u64) { kv[col * a.v_dim + row] = words[0] + z; });
        });
    }
    attn_tile_end(s, turn, a.error);
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
            ms[i] = attn_load2<VEC>(a.ms[i] + o);
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
        for (int i = 0; i < 2; ++i) attn_store2<VEC>(a.Es[i] + here, e[i]);
        attn_store2<VEC>(a.s + here, attn_add(e[0], e[1]));              // the exchange
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) attn_store2<VEC>(a.S1[i] + at, S[i]);
}

// Everything else of a chunk and query head.
template <bool VEC>
__global__ void __launch_bounds__(attn::TILE_THREADS, 1)
attn_rows_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ uint8_t attn_smem[];
    __shared__ AttnTile s;
    pdl_wait();
    pdl_launch_dependents();
    const int c = blockIdx.x / a.q_heads, hq = blockIdx.x - c * a.q_heads, h = hq / (a.q_heads / a.kv_heads), warp = threadIdx.x >> 5;
    const AttnChunk at = attn_find(a, c);
    if (at.len == 0) return;
    attn_tile_begin(s, attn_smem);
    AttnTurn turn;
    const int rows = at.len, first = at.first;
    const size_t q_row = (size_t)a.q_heads * a.k_dim, p_row = (size_t)a.q_heads * a.C, o_row = (size_t)a.q_heads * a.v_dim;
    const size_t k_row = (size_t)a.kv_heads * a.k_dim, v_row = (size_t)a.kv_heads * a.v_dim;
    const size_t q_at = first * q_row + (size_t)hq * a.k_dim, p_at = first * p_row + (size_t)hq * a.C, o_at = first * o_row + (size_t)hq * a.v_dim;
    const size_t k_at = at.first * k_row + (size_t)h * a.k_dim, v_at = at.first * v_row + (size_t)h * a.v_dim;
    const size_t s_at = ((size_t)c * a.kv_heads + h) * a.k_dim * a.v_dim;
    const int wide_C = a.C + (a.C & 1);                      // of the opened weights' rows, which begin on 16-byte boundaries
    const uint32_t w_row = a.q_heads * wide_C;
    const size_t w_at = (size_t)first * w_row + hq * wide_C;
    const u64* const w = a.decay + (size_t)h * (a.C + 1);
    if (warp != attn::ISSUER) {
        ulonglong2 x[2][2], m[2][2];
        attn_pairs(rows, a.k_dim, [&](int n, int r, int j) {
            const size_t o = q_at + r * q_row + j, x_at = (size_t)(first + r) * a.q_stride + (size_t)hq * a.k_dim + j;
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
                attn_store2<VEC>(a.Eq[i] + o, e[i]);
            }
            attn_store2<VEC>(a.q + o, attn_add(e[0], e[1]));         // the exchange
        });
        // off the triangle nothing is sent
        for (int t = threadIdx.x; t < rows * wide_C; t += attn::WORKERS) {
            const int r = t / wide_C, k = t - r * wide_C;
            if (k <= r) continue;
            const size_t o = w_at + (size_t)r * w_row + k;
            a.p[o] = a.pm[0][o] = a.pm[1][o] = 0ull;
            if (k < a.C) a.Ep[0][p_at + r * p_row + k] = a.Ep[1][p_at + r * p_row + k] = 0ull;
        }
        attn_meet();
    }
    if (warp == attn::ISSUER) {
        attn_issue(s, turn, a.k_dim);
        attn_issue(s, turn, a.k_dim);
#pragma unroll 1
        for (int t = 0; t < 2 * ((a.v_dim + attn::ROWS - 1) / attn::ROWS); ++t) {
            attn_issue(s, turn, a.k_dim);
            attn_issue(s, turn, rows);
        }
    } else if (warp < attn::CONVERTERS) {
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            const AttnOperand k = {a.mk[i] + k_at, a.k + k_at, (uint32_t)k_row}, q = {a.mq[i] + q_at, a.q + q_at, (uint32_t)q_row};
            attn_convert<false, false, VEC>(s, turn, k, rows, q, rows, a.k_dim, i);
        }
        // far part and near part in turn
        const int tiles = (a.v_dim + attn::ROWS - 1) / attn::ROWS;
#pragma unroll 1
        for (int n = 0; n < 4 * tiles; ++n) {
            const bool near = n & 1;
            const int i = n >= 2 * tiles, v0 = (n / 2 - i * tiles) * attn::ROWS;
            if (n == 1) turn.ok = turn.ok && attn_wait_warp(s.weights, 0, s);
            AttnOperand left, right;
            left.mask = (near ? a.mv[i] + v_at : a.ms[i] + s_at) + v0;
            left.open = (near ? a.v + v_at : a.s + s_at) + v0;
            left.step = near ? (uint32_t)v_row : (uint32_t)a.v_dim;
            right.mask = near ? a.pm[i] + w_at : a.mq[i] + q_at;
            right.open = near ? a.p + w_at : a.q + q_at;
            right.step = near ? w_row : (uint32_t)q_row;
            attn_convert<true, false, VEC>(s, turn, left, min(attn::ROWS, a.v_dim - v0), right, rows, near ? rows : a.k_dim, i);
        }
    } else {
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            const u64 *const qk = a.qk[i] + p_at, *const mp = a.mp[i] + p_at;
            u64 *const Ep = a.Ep[i] + p_at, *const p = a.p + w_at, *const pm = a.pm[i] + w_at;
            attn_drain<2>(s, turn, rows, rows, [&](int k, int key, int r) { return key > r ? nullptr : (k ? mp : qk) + (r * p_row + key); },
                          [&](int key, int r) { return i && key <= r ? p[r * w_row + key] : 0ull; }, [&](int key, int r, u64 z, const u64* words, u64 own) {
                if (key > r) return;
                const u64 e = attn_rescale(attn_rescale(z + words[0], i, a.f) * __ldg(w + r - key), i, a.f) - words[1];
                Ep[r * p_row + key] = e;
                pm[r * w_row + key] = words[1];
                p[r * w_row + key] = own + e;                // the exchange
            });
        }
        __syncwarp();
        if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(ptx::smem_u32(&s.weights));
#pragma unroll 1
        for (int i = 0; i < 2; ++i)
#pragma unroll 1
            for (int v0 = 0; v0 < a.v_dim; v0 += attn::ROWS) {
                // what the near part is added to waits in the result's place, where the same thread finds it again
                const int wide = min(attn::ROWS, a.v_dim - v0);
                u64* const O = a.O[i] + o_at + v0;
                const u64 *const qs = a.qs[i] + o_at + v0, *const pv = a.pv[i] + o_at + v0;
                attn_drain<2>(s, turn, wide, rows, [&](int k, int row, int r) { return (k ? pv : qs) + (r * o_row + row); }, attn_nothing,
                              [&](int row, int r, u64 z, const u64* words, u64) {
                    O[r * o_row + row] = words[1] + __ldg(w + r + 1) * attn_rescale(z + words[0], i, a.f);
                });
                attn_drain<0>(s, turn, wide, rows, [&](int, int, int) { return (const u64*)nullptr; }, [&](int row, int r) { return O[r * o_row + row]; },
                              [&](int row, int r, u64 z, const u64*, u64 own) { O[r * o_row + row] = attn_rescale(own + z, i, a.f); });
            }
    }
    attn_tile_end(s, turn, a.error);
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
