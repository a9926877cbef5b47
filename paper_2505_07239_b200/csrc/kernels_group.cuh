// The norm of groups of neighbouring channels, channels last, with gain, bias and quadratic activation, on additive shares
// (comet_group_norm).  f the fixed point, i the party, tr the local truncation by f bits, div_d the same by a divisor; of every
// sample and group, n words (its positions times its channels):
//   d_i = x_i - div_n(sum x_i),  m = open(d - U),  sq_i = words[0] + sum 2 m U_i + i sum m^2,  s_i = div_{n 2^f}(sq_i) + i eps
//   y ~ 1 / sqrt(s) by Newton's iteration, opened with its mask v                              (norm_root, kernels_norm.cuh)
//   of every channel  t = tr(y gain),  opened with its mask T;  without a gain t = y and T = v
//   z = tr(t d + 2^f bias) by Eq. 1 with the dealer's U T;  then k2 z^2 + k1 z + k0 on the dealer's pair (R, R R)
// The gain meets the root before it meets the words: a product per channel instead of one per word.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kernels_norm.cuh"
#include "pdl.cuh"

namespace comet {

namespace group {
constexpr int THREADS = 256;
}  // namespace group

struct GroupArgs {
    NormArgs root;                       // guess, first, eps, divisor, f, steps: what norm_root reads
    const u64* X[2];                     // position p of sample s at (s * positions + p) * x_stride
    const u64* U[2]; const u64* words[2]; const u64* UT[2];
    const u64* gain[2]; const u64* gain_mask[2]; const u64* T[2]; const u64* VW[2]; const u64* bias[2];   // gain[0] null: none
    const u64* R[2]; const u64* Q[2];                                                                     // R[0] null: no activation
    u64* M[2]; u64* S[2]; u64* D[2]; u64* G[2]; u64* N[2];
    u64* Z[2];
    u64* sums;                           // [2][samples * groups * slabs][2]: of x, of the squares
    u64 k0, k1, k2;
    long long x_stride;
    int positions, channels, groups, per, slabs, slab;                   // slab: positions of one
};

__device__ __forceinline__ u64 group_trunc(u64 v, int party, int bits) {
    return party ? 0ull - ((0ull - v) >> bits) : v >> bits;
}

struct GroupPlace {
    int sample, g, p0, words, slab;      // words of the group in the CTA's slab
    size_t group;
};
__device__ __forceinline__ GroupPlace group_place(const GroupArgs& a) {
    GroupPlace p;
    p.slab = blockIdx.x % a.slabs;
    p.group = blockIdx.x / a.slabs;
    p.sample = (int)(p.group / a.groups);
    p.g = (int)(p.group - (size_t)p.sample * a.groups);
    p.p0 = p.slab * a.slab;
    p.words = min(a.slab, a.positions - p.p0) * a.per;
    return p;
}
// Sums over a CTA's threads of both parties'.
__device__ __forceinline__ void group_reduce(u64 v[2]) {
    __shared__ u64 part[group::THREADS / 32][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int o = 16; o; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) {
        part[threadIdx.x >> 5][0] = v[0];
        part[threadIdx.x >> 5][1] = v[1];
    }
    __syncthreads();
    v[0] = v[1] = 0ull;
    for (int k = 0; k < group::THREADS / 32; ++k) {
        v[0] += part[k][0];
        v[1] += part[k][1];
    }
}
// The sums of a group's slabs.
__device__ __forceinline__ void group_total(const GroupArgs& a, const u64* sums, size_t group, u64 v[2]) {
    v[0] = v[1] = 0ull;
    for (int k = threadIdx.x; k < a.slabs; k += group::THREADS)
        for (int i = 0; i < 2; ++i) v[i] += sums[(group * a.slabs + k) * 2 + i];
    group_reduce(v);
}

__global__ void __launch_bounds__(group::THREADS)
group_sum_kernel(const __grid_constant__ GroupArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const GroupPlace at = group_place(a);
    u64 sum[2] = {0ull, 0ull};
    for (int t = threadIdx.x; t < at.words; t += group::THREADS) {
        const int p = t / a.per, c = t - p * a.per;
        const size_t o = ((size_t)at.sample * a.positions + at.p0 + p) * a.x_stride + (size_t)at.g * a.per + c;
        for (int i = 0; i < 2; ++i) sum[i] += __ldg(a.X[i] + o);
    }
    group_reduce(sum);
    if (threadIdx.x < 2) a.sums[(size_t)blockIdx.x * 2 + threadIdx.x] = sum[threadIdx.x];
}

__global__ void __launch_bounds__(group::THREADS)
group_open_kernel(const __grid_constant__ GroupArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const GroupPlace at = group_place(a);
    u64 mean[2], sq[2] = {0ull, 0ull};
    group_total(a, a.sums, at.group, mean);
    const u64 n = (u64)a.positions * a.per;
    mean[0] = mean[0] / n;
    mean[1] = 0ull - (0ull - mean[1]) / n;
    for (int t = threadIdx.x; t < at.words; t += group::THREADS) {
        const int p = t / a.per, c = t - p * a.per;
        const size_t row = (size_t)at.sample * a.positions + at.p0 + p, col = (size_t)at.g * a.per + c, o = row * a.channels + col;
        u64 u[2], msg[2];
        for (int i = 0; i < 2; ++i) {
            u[i] = __ldg(a.U[i] + o);
            a.M[i][o] = msg[i] = __ldg(a.X[i] + row * a.x_stride + col) - mean[i] - u[i];
        }
        const u64 m = msg[0] + msg[1];
        sq[0] += 2 * m * u[0];
        sq[1] += m * (2 * u[1] + m);
    }
    group_reduce(sq);
    if (threadIdx.x < 2) a.sums[((size_t)gridDim.x + blockIdx.x) * 2 + threadIdx.x] = sq[threadIdx.x];
}

__global__ void __launch_bounds__(group::THREADS)
group_apply_kernel(const __grid_constant__ GroupArgs a) {
    __shared__ u64 words[2][norm::words(norm::MAX_STEPS)], sent[2][norm::openings(norm::MAX_STEPS)], root;
    pdl_wait();
    pdl_launch_dependents();
    const GroupPlace at = group_place(a);
    const int f = a.root.f, count = norm::words(a.root.steps), openings = norm::openings(a.root.steps);
    u64 sq[2];
    group_total(a, a.sums + (size_t)gridDim.x * 2, at.group, sq);
    for (int k = threadIdx.x; k < count; k += group::THREADS)
        for (int i = 0; i < 2; ++i) {
            const u64 v = __ldg(a.words[i] + at.group * count + k);
            words[i][k] = i ? 0ull - v : v;
        }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int party = threadIdx.x & 1;
        const u64 r = norm_root(a.root, party ? 0ull - sq[1] : sq[0], words[party], sent[party], threadIdx.x < 2, party);
        if (threadIdx.x == 0) root = r;
    }
    __syncthreads();
    if (at.slab == 0)
        for (int k = threadIdx.x; k < openings; k += group::THREADS)
            for (int i = 0; i < 2; ++i) a.S[i][at.group * openings + k] = i ? 0ull - sent[1][k] : sent[0][k];
    const u64 v[2] = {words[0][count - 1], 0ull - words[1][count - 1]};
    for (int t = threadIdx.x; t < at.words; t += group::THREADS) {
        const int p = t / a.per, c = t - p * a.per;
        const size_t row = (size_t)at.sample * a.positions + at.p0 + p, col = (size_t)at.g * a.per + c, o = row * a.channels + col;
        u64 mask[2] = {v[0], v[1]}, r = root, bias[2] = {0ull, 0ull};
        if (a.gain[0]) {
            const size_t own = (size_t)at.sample * a.channels + col;
            u64 g[2], b[2];
            for (int i = 0; i < 2; ++i) {
                b[i] = __ldg(a.gain_mask[i] + col);
                g[i] = __ldg(a.gain[i] + col) - b[i];
                if (at.sample == 0 && at.p0 + p == 0) a.G[i][col] = g[i];
            }
            const u64 e = g[0] + g[1];
            u64 opened = 0ull;
            for (int i = 0; i < 2; ++i) {
                const u64 T = group_trunc(__ldg(a.VW[i] + own) + root * (b[i] + (i ? e : 0ull)) + e * v[i], i, f);
                mask[i] = __ldg(a.T[i] + own);
                if (at.p0 + p == 0) a.D[i][own] = T - mask[i];
                opened += T - mask[i];
                bias[i] = __ldg(a.bias[i] + col) << f;
            }
            r = opened;
        }
        const u64 m = a.M[0][o] + a.M[1][o];
        u64 z[2];
        for (int i = 0; i < 2; ++i) z[i] = group_trunc(__ldg(a.UT[i] + o) + m * (mask[i] + (i ? r : 0ull)) + r * __ldg(a.U[i] + o) + bias[i], i, f);
        if (a.R[0]) {
            u64 R[2], msg[2];
            for (int i = 0; i < 2; ++i) {
                R[i] = __ldg(a.R[i] + o);
                a.N[i][o] = msg[i] = z[i] - R[i];
            }
            const u64 b = msg[0] + msg[1];
            for (int i = 0; i < 2; ++i) {
                const u64 square = group_trunc(__ldg(a.Q[i] + o) + b * (2 * R[i] + (i ? b : 0ull)), i, f);
                z[i] = group_trunc(a.k2 * square + a.k1 * z[i], i, f) + (i ? a.k0 : 0ull);
            }
        }
        for (int i = 0; i < 2; ++i) a.Z[i][o] = z[i];
    }
}

}  // namespace comet
