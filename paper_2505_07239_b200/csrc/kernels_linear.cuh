// What follows the product of a shared linear layer (comet_linear), element by element, z_i the party's share of X W^T at scale 2f:
//     y_i = tr_f(z_i + 2^f bias_i)                                  (Section 2.1 "Addition" and the local truncation)
//     with an activation k2 y^2 + k1 y + k0, on the dealer's pair (R, Q = R R):
//       [m]_i = y_i - R_i (the message), s_i = tr_f(Q_i + 2 m R_i + i m^2)         (Eq. 1 with both factors y)
//       y_i = tr_f(k2 s_i + k1 y_i) + i k0
//     Y_i = y_i + residual_i
// Bound by memory where it is a pass of its own (behind the kernels that add their sums into Z: one word in and one out per
// element and party, and what the parts that are there read and write); behind the kernel on residues it is part of the
// recombination, which makes the words anyway.  Under ncu: 203 x 1364 with everything 6.6 us (27 MB, 4.0 TB/s); the recombination of
// 512 x 2048 with bias and residual 18.8 us (residue_recombine_kernel alone: 15.8), of 512 x 8192 with the activation 87 us (486 MB, 5.6 TB/s).
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kernels_residue.cuh"
#include "pdl.cuh"

namespace comet {

struct LinearEnd {
    const u64* bias[2];          // [cols], or null
    const u64* residual[2];      // or null
    const u64* R[2]; const u64* Q[2]; u64* M[2];     // R[0] null: no activation
    u64 k0, k1, k2;
    int f;
};

__device__ __forceinline__ u64 linear_trunc(u64 v, int party, int f) { return party ? 0ull - ((0ull - v) >> f) : v >> f; }

// One party's word from the opened m on.
__device__ __forceinline__ u64 linear_square(u64 y, u64 r, u64 q, u64 m, const LinearEnd& e, int party) {
    const u64 s = linear_trunc(q + m * (r + r + (party ? m : 0ull)), party, e.f);
    return linear_trunc(e.k2 * s + e.k1 * y, party, e.f) + (party ? e.k0 : 0ull);
}

// What follows the product for two neighbouring words of both parties, z at pair t of the matrix and pair col of its row.
__device__ __forceinline__ void linear_finish_pair(const LinearEnd& e, ulonglong2 y[2], long long t, int col, u64* const Z[2]) {
    ulonglong2 r[2], q[2], res[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        if (e.R[0]) {
            r[p] = __ldcs(reinterpret_cast<const ulonglong2*>(e.R[p]) + t);
            q[p] = __ldcs(reinterpret_cast<const ulonglong2*>(e.Q[p]) + t);
        }
        res[p] = e.residual[0] ? __ldcs(reinterpret_cast<const ulonglong2*>(e.residual[p]) + t) : make_ulonglong2(0ull, 0ull);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        if (e.bias[0]) {
            const ulonglong2 b = __ldg(reinterpret_cast<const ulonglong2*>(e.bias[p]) + col);
            y[p].x += b.x << e.f;
            y[p].y += b.y << e.f;
        }
        y[p].x = linear_trunc(y[p].x, p, e.f);
        y[p].y = linear_trunc(y[p].y, p, e.f);
    }
    if (e.R[0]) {
        ulonglong2 m = make_ulonglong2(0ull, 0ull);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const ulonglong2 mine = make_ulonglong2(y[p].x - r[p].x, y[p].y - r[p].y);
            __stcs(reinterpret_cast<ulonglong2*>(e.M[p]) + t, mine);
            m.x += mine.x;                                   // the exchange
            m.y += mine.y;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
            y[p] = make_ulonglong2(linear_square(y[p].x, r[p].x, q[p].x, m.x, e, p), linear_square(y[p].y, r[p].y, q[p].y, m.y, e, p));
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) reinterpret_cast<ulonglong2*>(Z[p])[t] = make_ulonglong2(y[p].x + res[p].x, y[p].y + res[p].y);
}

// The pass behind the products whose sums are added into Z: in place.
struct LinearEpilogueArgs {
    LinearEnd end;
    u64* Z[2];
    const u64* C[2]; const u64* sums[2];     // linear_parts_kernel: [parts][rows][cols]
    int parts;
    long long pairs;             // of the whole matrix
    int row_pairs, stride_pairs; // pairs of a row; (gridDim.x * blockDim.x) % row_pairs
};
__global__ void __launch_bounds__(256)
linear_epilogue_kernel(const __grid_constant__ LinearEpilogueArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const long long stride = (long long)gridDim.x * blockDim.x;
    long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    int col = (int)(t % a.row_pairs);
    for (; t < a.pairs; t += stride) {
        ulonglong2 y[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) y[p] = reinterpret_cast<const ulonglong2*>(a.Z[p])[t];
        linear_finish_pair(a.end, y, t, col, a.Z);
        col += a.stride_pairs;
        if (col >= a.row_pairs) col -= a.row_pairs;
    }
}

// The pass behind a product whose sums lie in parts: a pair's parts are dealt to LINEAR_SHARERS lanes, because there are few pairs.  (A
// thread a pair: 20 tokens, 768 x 768, 24 parts, 21.5 us a layer.)
constexpr int LINEAR_SHARERS = 8;
__global__ void __launch_bounds__(256)
linear_parts_kernel(const __grid_constant__ LinearEpilogueArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int PAIRS = 32 / LINEAR_SHARERS;               // of a warp
    const int lane = threadIdx.x & 31, share = lane / PAIRS;
    const long long warps = (long long)gridDim.x * (blockDim.x / 32), all = (a.pairs + PAIRS - 1) / PAIRS;
    for (long long w = (long long)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5); w < all; w += warps) {
        const long long t = w * PAIRS + lane % PAIRS;
        const bool live = t < a.pairs;
        ulonglong2 y[2] = {make_ulonglong2(0ull, 0ull), make_ulonglong2(0ull, 0ull)};
        if (live) {
            if (share == 0)
#pragma unroll
                for (int p = 0; p < 2; ++p) y[p] = __ldcs(reinterpret_cast<const ulonglong2*>(a.C[p]) + t);
#pragma unroll 4
            for (int k = share; k < a.parts; k += LINEAR_SHARERS)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const ulonglong2 v = __ldcs(reinterpret_cast<const ulonglong2*>(a.sums[p]) + k * a.pairs + t);
                    y[p].x += v.x;
                    y[p].y += v.y;
                }
        }
#pragma unroll
        for (int o = PAIRS; o < 32; o *= 2)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                y[p].x += __shfl_xor_sync(0xffffffffu, y[p].x, o);
                y[p].y += __shfl_xor_sync(0xffffffffu, y[p].y, o);
            }
        if (live && share == 0) linear_finish_pair(a.end, y, t, (int)(t % a.row_pairs), a.Z);
    }
}

// The words of a product through residues (see residue_recombine_kernel), finished at once.  A thread makes four words of a row
// (SWAPPED: of a column) of Z, of one party; with an activation of both, which is the exchange.
template <bool SWAPPED, bool QUADRATIC>
__global__ void __launch_bounds__(256)
linear_recombine_kernel(const __grid_constant__ RecombineArgs a, const __grid_constant__ LinearEnd e) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int PARTIES = QUADRATIC ? 2 : 1;
    const size_t plane = (size_t)a.m_groups * a.n_chunks * 512;
    const unsigned pieces = (unsigned)a.m_groups * a.n_chunks * 128;
    for (unsigned piece = blockIdx.x * blockDim.x + threadIdx.x; piece < pieces; piece += gridDim.x * blockDim.x) {
        const unsigned cell = piece >> 7, mg = cell / (unsigned)a.n_chunks, nc = cell - mg * a.n_chunks;
        const unsigned m = SWAPPED ? piece & 31 : piece >> 2 & 31, n = SWAPPED ? piece >> 5 & 3 : piece & 3;
        const unsigned row = SWAPPED ? nc * 16 + n * 4 : mg * 32 + m, col = SWAPPED ? mg * 32 + m : nc * 16 + n * 4;
        if (row >= (unsigned)a.rows || col >= (unsigned)a.cols) continue;
        const size_t at = (size_t)row * (SWAPPED ? a.ld : a.cols) + col;
        // four words of one of the operands that lie like Z
        auto load = [&](const u64* from, u64 v[4]) {
            if (!SWAPPED) {
                const ulonglong2 v0 = __ldcs(reinterpret_cast<const ulonglong2*>(from + at)), v1 = __ldcs(reinterpret_cast<const ulonglong2*>(from + at + 2));
                v[0] = v0.x; v[1] = v0.y; v[2] = v1.x; v[3] = v1.y;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = row + k < (unsigned)a.rows ? __ldcs(from + at + (size_t)k * a.ld) : 0ull;
            }
        };
        auto store = [&](u64* to, const u64 v[4]) {
            if (!SWAPPED) {
                *reinterpret_cast<ulonglong2*>(to + at) = make_ulonglong2(v[0], v[1]);
                *reinterpret_cast<ulonglong2*>(to + at + 2) = make_ulonglong2(v[2], v[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (row + k < (unsigned)a.rows) to[at + (size_t)k * a.ld] = v[k];
            }
        };
        u64 y[PARTIES][4];
#pragma unroll
        for (int j = 0; j < PARTIES; ++j) {
            const int p = QUADRATIC ? j : (int)blockIdx.y;
            u64* sum = y[j];
            load(p ? a.C[1] : a.C[0], sum);
            unsigned quotient[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) quotient[k] = (1u << 23) + (8u << 24) - RESIDUE_QUOTIENT_BIAS;
            const uint8_t* t = (p ? a.T[1] : a.T[0]) + (size_t)cell * 512 + m * 16 + n * 4;
            residue_gather<0>(t, plane, quotient, sum);
            const unsigned x = __ldcs(reinterpret_cast<const unsigned*>(t + residue::MODULI * plane));
            const unsigned z = __ldcs(reinterpret_cast<const unsigned*>(t + (residue::MODULI + 1) * plane));
            const u64* bias = p ? e.bias[1] : e.bias[0];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum[k] -= RESIDUE_BIAS + (u64)(long long)((int)(quotient[k] >> 24) - 8) * residue::product();
                sum[k] += (u64)((x >> (8 * k)) + (z >> (8 * k))) << 56;
                if (bias) sum[k] += __ldg(bias + col + (SWAPPED ? 0 : k)) << e.f;
                sum[k] = linear_trunc(sum[k], p, e.f);
            }
        }
        if (QUADRATIC) {
            u64 r[PARTIES][4], q[4], open[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int p = 0; p < PARTIES; ++p) {
                load(e.R[p], r[p]);
                u64 mine[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    mine[k] = y[p][k] - r[p][k];
                    open[k] += mine[k];                      // the exchange
                }
                store(e.M[p], mine);
            }
#pragma unroll
            for (int p = 0; p < PARTIES; ++p) {
                load(e.Q[p], q);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[p][k] = linear_square(y[p][k], r[p][k], q[k], open[k], e, p);
            }
        }
#pragma unroll
        for (int j = 0; j < PARTIES; ++j) {
            const int p = QUADRATIC ? j : (int)blockIdx.y;
            if (e.residual[0]) {
                u64 v[4];
                load(p ? e.residual[1] : e.residual[0], v);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[j][k] += v[k];
            }
            store(p ? a.Z[1] : a.Z[0], y[j]);
        }
    }
}

}  // namespace comet
