// A whole shared linear layer for one to four token rows (the serving form of comet_linear) in one launch: mask, exchange, product
// and what follows it.
//   F_i = W_i - B_i (written), F = F_0 + F_1;  E_i = X_i - A_i (written), E = E_0 + E_1
//   z_0 = C_0 + E B_0^T + A_0 F^T,  z_1 = C_1 + E B_1^T + (A_1 + E) F^T               (Eq. 1), then kernels_linear.cuh's steps
//
// What bounds it: memory, 24 bytes per weight word and party (W_i and B_i in, F_i out); a weight word takes part in four 64-bit
// multiply-adds per token, which the integer ALUs do beside the loads for a few tokens.  No limb planes, no accumulators in tensor
// memory and no partial sums in Z: a CTA has its features' sums to itself, so the bias, the truncation, the activation and the
// residual follow in the same launch.  The streaming kernel (kernels_stream.cuh) takes two launches for the same, three where its
// sums do not lie in parts, and 8.5 us however small the layer.
//
// Measured: one row, 4096 x 4096 139 us, 0.88 of the copy rate; 768 x 768 11.3 us, of which 2.5 are the launch, 4.3 the bytes.  From the
// second row on the multiply-adds show (4096 x 4096: 145 us, four rows 197): comet_api.cu has the rule, with both sides' times.
//
// A CTA (one per SM) takes blocks of features.  Its warps split the contraction index in `slices` parts (8, fewer where the rows are
// short) and the features in 16 / slices.  A lane copies 16 bytes of W_0, W_1, B_0 and B_1 at a time to its own places in shared
// memory, five such steps ahead, 160 KiB under way per SM, across chunks and blocks.  (Three steps ahead in registers, two CTAs of
// eight warps: 4096 x 4096, one token, 176 us.)  E, A_0 and A_1 + E lie in shared memory too, a chunk of the contraction index
// after the other.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kernels_linear.cuh"
#include "pdl.cuh"

namespace comet {

namespace rows {
constexpr int THREADS = 512, WARPS = THREADS / 32, MAX_ROWS = 4, MAX_SLICES = 8, DEPTH = 5;
constexpr int RING_BYTES = THREADS * DEPTH * 64;
constexpr int VECTOR_BYTES = 44 * 1024;              // of E, A_0 and A_1 + E in shared memory
constexpr int MAX_BLOCK = 32;                        // features of a block
// Pairs of words of the contraction index in a chunk: what fits, in whole warps of lanes per slice.
__host__ __device__ constexpr int chunk_pairs(int rows) { return VECTOR_BYTES / (3 * 16 * rows) / 64 * 64; }
}  // namespace rows

struct RowsArgs {
    const u64* X[2]; const u64* A[2]; const u64* W[2]; const u64* B[2]; const u64* C[2];
    u64* E[2]; u64* F[2]; u64* Y[2];
    LinearEnd end;
    int rows, cols, pairs;       // pairs of words of the contraction index
    int slices;                  // 1, 2, 4 or 8
    int block, blocks;           // features of a block, blocks
};

// Sums over a warp's lanes of M values each (a power of two up to 16): afterwards v[0] of every lane is the sum of value
// `lane >> (5 - log2 M)`.
template <int M>
__device__ __forceinline__ void rows_reduce(u64 (&v)[M], int lane) {
#pragma unroll
    for (int s = M / 2, mask = 16; s >= 1; s /= 2, mask /= 2) {
        const bool upper = lane & mask;
#pragma unroll
        for (int j = 0; j < s; ++j) {
            const u64 send = upper ? v[j] : v[j + s], keep = upper ? v[j + s] : v[j];
            v[j] = keep + __shfl_xor_sync(0xffffffffu, send, mask);
        }
    }
#pragma unroll
    for (int mask = 16 / M; mask >= 1; mask /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], mask);
}

// One warp's way through its words: blocks of features, chunks of the contraction index, features, 32 pairs at a time.
struct RowsPlace {
    int blk, chunk, feat, it;    // it: of the iters of this chunk
    int features, p0, here, begin, mine, iters;
    __device__ __forceinline__ void enter(const RowsArgs& a, int capacity, int slice) {
        features = min(a.block, a.cols - blk * a.block);
        p0 = chunk * capacity;
        here = min(capacity, a.pairs - p0);
        const int per = (here + a.slices - 1) / a.slices;
        begin = slice * per;
        mine = max(0, min(per, here - begin));
        iters = (mine + 31) / 32;
    }
};

template <int ROWS>
__global__ void __launch_bounds__(rows::THREADS, 1)
linear_rows_kernel(const __grid_constant__ RowsArgs a) {
    constexpr int M = 2 * ROWS, DEPTH = rows::DEPTH;
    extern __shared__ __align__(16) uint8_t rows_smem[];
    // a lane's four pieces of a step lie 16 THREADS bytes apart; [E | A_0 | A_1 + E][ROWS][pairs of a chunk]
    ulonglong2* const ring = reinterpret_cast<ulonglong2*>(rows_smem) + threadIdx.x;
    ulonglong2* const vec = reinterpret_cast<ulonglong2*>(rows_smem + rows::RING_BYTES);
    __shared__ u64 part[rows::MAX_BLOCK][M][rows::MAX_SLICES];       // a block's sums, per slice
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int slice = warp % a.slices, group = warp / a.slices, groups = rows::WARPS / a.slices;
    const int capacity = min(rows::chunk_pairs(ROWS), a.pairs), chunks = (a.pairs + capacity - 1) / capacity;
    pdl_wait();
    pdl_launch_dependents();

    // the copies run ahead of the work: `ahead` is where they are
    RowsPlace ahead;
    ahead.blk = blockIdx.x;
    ahead.chunk = 0;
    ahead.feat = group;
    ahead.it = 0;
    if (ahead.blk < a.blocks) ahead.enter(a, capacity, slice);
    int load_slot = 0;
    auto load = [&] {
        // the next place with words, if there is one
        while (ahead.blk < a.blocks && (ahead.feat >= ahead.features || ahead.it >= ahead.iters)) {
            if (ahead.feat < ahead.features && ahead.iters > 0) {
                ahead.feat += groups;
                ahead.it = 0;
                continue;
            }
            ahead.feat = group;
            ahead.it = 0;
            if (++ahead.chunk == chunks) {
                ahead.chunk = 0;
                ahead.blk += gridDim.x;
                if (ahead.blk >= a.blocks) break;
            }
            ahead.enter(a, capacity, slice);
        }
        if (ahead.blk < a.blocks) {
            const int p = ahead.it * 32 + lane;
            if (p < ahead.mine) {
                const size_t at = (size_t)(ahead.blk * a.block + ahead.feat) * a.pairs + ahead.p0 + ahead.begin + p;
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring + load_slot * 4 * rows::THREADS);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + k * 16 * rows::THREADS),
                                 "l"(reinterpret_cast<const ulonglong2*>(k < 2 ? a.W[k] : a.B[k - 2]) + at) : "memory");
            }
            ++ahead.it;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");         // one group a step, empty or not
        if (++load_slot == DEPTH) load_slot = 0;
    };
#pragma unroll 1
    for (int j = 0; j < DEPTH - 1; ++j) load();

    int slot = 0;
    RowsPlace now;
    for (now.blk = blockIdx.x; now.blk < a.blocks; now.blk += gridDim.x) {
        const int f0 = now.blk * a.block;
        for (now.chunk = 0; now.chunk < chunks; ++now.chunk) {
            now.enter(a, capacity, slice);
            const int here = now.here;
            if (chunks > 1 || now.blk == (int)blockIdx.x) {
                __syncthreads();                                     // the chunk before this one has been read
                for (int q = threadIdx.x; q < ROWS * here; q += rows::THREADS) {
                    const int t = ROWS == 1 ? 0 : q / here, p = q - t * here;
                    ulonglong2 e = make_ulonglong2(0ull, 0ull), m[2] = {e, e};
                    if (t < a.rows) {
                        const size_t at = (size_t)t * a.pairs + now.p0 + p;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const ulonglong2 x = __ldg(reinterpret_cast<const ulonglong2*>(a.X[i]) + at);
                            m[i] = __ldg(reinterpret_cast<const ulonglong2*>(a.A[i]) + at);
                            const ulonglong2 d = make_ulonglong2(x.x - m[i].x, x.y - m[i].y);
                            // the message: its pieces are dealt out among the CTAs
                            if (now.blk == (int)blockIdx.x && (unsigned)(now.chunk + q / rows::THREADS) % gridDim.x == blockIdx.x)
                                reinterpret_cast<ulonglong2*>(a.E[i])[at] = d;
                            e.x += d.x;                              // the exchange
                            e.y += d.y;
                        }
                    }
                    vec[q] = e;
                    vec[ROWS * here + q] = m[0];
                    vec[2 * ROWS * here + q] = make_ulonglong2(m[1].x + e.x, m[1].y + e.y);
                }
                __syncthreads();
            }
            for (int feat = group; feat < now.features; feat += groups) {
                u64 sum[M];
#pragma unroll
                for (int j = 0; j < M; ++j) sum[j] = 0ull;
                const size_t row = (size_t)(f0 + feat) * a.pairs + now.p0 + now.begin;
                for (int it = 0; it < now.iters; ++it) {
                    load();                                          // (its slot was read a step ago, by this lane alone)
                    asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
                    const int p = it * 32 + lane;
                    const ulonglong2* const from = ring + slot * 4 * rows::THREADS;
                    if (++slot == DEPTH) slot = 0;
                    if (p >= now.mine) continue;
                    ulonglong2 f[2], b[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const ulonglong2 w = from[i * rows::THREADS];
                        b[i] = from[(2 + i) * rows::THREADS];
                        f[i] = make_ulonglong2(w.x - b[i].x, w.y - b[i].y);
                        __stcs(reinterpret_cast<ulonglong2*>(a.F[i]) + row + p, f[i]);
                    }
                    f[0].x += f[1].x;                                // the exchange
                    f[0].y += f[1].y;
#pragma unroll
                    for (int t = 0; t < ROWS; ++t) {
                        const ulonglong2 *v = vec + t * here + now.begin + p, e = v[0], m = v[ROWS * here], n = v[2 * ROWS * here];
                        sum[2 * t] += e.x * b[0].x + e.y * b[0].y + m.x * f[0].x + m.y * f[0].y;
                        sum[2 * t + 1] += e.x * b[1].x + e.y * b[1].y + n.x * f[0].x + n.y * f[0].y;
                    }
                }
                rows_reduce(sum, lane);
                constexpr int SHARE = 32 / M;                        // lanes that hold the same sum
                if (lane % SHARE == 0) {
                    u64* const to = &part[feat][lane / SHARE][slice];
                    *to = now.chunk == 0 ? sum[0] : *to + sum[0];
                }
            }
        }
        __syncthreads();
        const LinearEnd& e = a.end;
        for (int q = threadIdx.x; q < a.rows * now.features; q += rows::THREADS) {
            const int t = ROWS == 1 ? 0 : q / now.features, n = q - t * now.features;
            const size_t at = (size_t)t * a.cols + f0 + n;
            u64 y[2], r[2], m = 0ull;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                y[i] = __ldg(a.C[i] + at);
                for (int k = 0; k < a.slices; ++k) y[i] += part[n][2 * t + i][k];
                if (e.bias[0]) y[i] += __ldg(e.bias[i] + f0 + n) << e.f;
                y[i] = linear_trunc(y[i], i, e.f);
                if (e.R[0]) {
                    r[i] = __ldg(e.R[i] + at);
                    e.M[i][at] = y[i] - r[i];
                    m += y[i] - r[i];                                // the exchange
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (e.R[0]) y[i] = linear_square(y[i], r[i], __ldg(e.Q[i] + at), m, e, i);
                if (e.residual[0]) y[i] += __ldg(e.residual[i] + at);
                a.Y[i][at] = y[i];
            }
        }
        __syncthreads();                                             // the sums are written anew for the next block
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace comet
