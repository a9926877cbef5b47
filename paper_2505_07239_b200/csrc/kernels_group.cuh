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
constexpr int SLAB_THREADS = 256, SLAB_GROUPS = 32, SLAB_APPLY = 768;  // at most, of a CTA that has a slab of long groups; its groups
constexpr int TILE_THREADS = 128, TILE_WORDS = 4 * TILE_THREADS, TILE_GROUPS = 16, TILE_CTAS = 5;
constexpr int CLUSTER_THREADS = 256, MAX_CLUSTER = 8, CLUSTER_CTAS = 2;
constexpr int TABLE = 1024;                          // channels of a group that a CTA keeps the products of root and gain of
// Groups of a tile: a thread has four words, a lane pair of one warp a group's root.
__host__ __device__ constexpr int tile_groups(int quads) { return TILE_THREADS / quads < TILE_GROUPS ? TILE_THREADS / quads : TILE_GROUPS; }
// What a thread needs behind the root lies in its places of shared memory: per access and party U T, R, Q, and, where a channel's products are
// a word's (one position), V W and T.
__host__ __device__ constexpr int arrays(bool act, bool per_word) { return 1 + (act ? 2 : 0) + (per_word ? 2 : 0); }
}  // namespace group

struct GroupArgs {
    NormArgs root;                       // guess, first, eps, divisor, f, steps: what norm_root reads
    const u64* X[2];                     // position p of sample s at (s * positions + p) * x_stride
    const u64* U[2]; const u64* words[2]; const u64* UT[2];
    const u64* gain[2]; const u64* gain_mask[2]; const u64* T[2]; const u64* VW[2]; const u64* bias[2];   // gain[0] null: none
    const u64* R[2]; const u64* Q[2];                                                                     // R[0] null: no activation
    u64* M[2]; u64* S[2]; u64* D[2]; u64* G[2]; u64* N[2];
    u64* Z[2];
    u64* sums;                           // long groups: [2][all][2], of x, of the squares; zero to begin with
    u64 k0, k1, k2;
    long long x_stride;
    int positions, channels, groups, per;
    int slab, slabs, tiles, tile_groups, parts, units, subs;             // long groups: how they are cut, see group_slab
    int count, all;                      // words of a group, groups of all samples
};

// W words at once, 16 bytes or 8.
template <int W>
__device__ __forceinline__ void group_load(const u64* p, u64* v) {
    if (W == 2) {
        const ulonglong2 t = __ldcs(reinterpret_cast<const ulonglong2*>(p));
        v[0] = t.x;
        v[W - 1] = t.y;
    } else {
        v[0] = __ldcs(p);
    }
}
template <int W>
__device__ __forceinline__ void group_read(const u64* p, u64* v) {                        // what other CTAs read, too
    if (W == 2) {
        const ulonglong2 t = __ldg(reinterpret_cast<const ulonglong2*>(p));
        v[0] = t.x;
        v[W - 1] = t.y;
    } else {
        v[0] = __ldg(p);
    }
}
template <int W>
__device__ __forceinline__ void group_store(u64* p, const u64* v) {
    if (W == 2) __stcs(reinterpret_cast<ulonglong2*>(p), make_ulonglong2(v[0], v[W - 1]));
    else __stcs(p, v[0]);
}
template <int W>
__device__ __forceinline__ void group_fetch(u64* to, const u64* p) {
    if (W == 2) norm_fetch16(to, p);
    else norm_fetch8(to, p);
}

// What a channel's words are multiplied with: the opened t - T, the masks T of both parties (party 1's with the opened value added: V_i of
// Eq. 1), and the bias at scale 2f.
struct GroupScale {
    u64 r, mask[2], bias[2];
};
// Without a gain it is the root's; with one, from the words V W and T of the channel.  Writes the messages of the gain where it is told to.
__device__ __forceinline__ GroupScale group_scale(const GroupArgs& a, u64 root, const u64 v[2], int sample, int channel, const u64 VW[2], const u64 T[2],
                                                  bool tells) {
    GroupScale s;
    if (!a.gain[0]) {
        s.r = root;
        s.mask[0] = v[0];
        s.mask[1] = v[1] + root;
        s.bias[0] = s.bias[1] = 0ull;
        return s;
    }
    const int f = a.root.f;
    u64 g[2], b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        b[i] = __ldg(a.gain_mask[i] + channel);
        g[i] = __ldg(a.gain[i] + channel) - b[i];
        s.bias[i] = __ldg(a.bias[i] + channel) << f;
        if (tells && sample == 0) a.G[i][channel] = g[i];
    }
    const u64 e = g[0] + g[1];
    s.r = 0ull;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u64 t = VW[i] + root * (b[i] + (i ? e : 0ull)) + e * v[i];
        const u64 D = (i ? 0ull - norm_shift(0ull - t, f) : norm_shift(t, f)) - T[i];
        if (tells) a.D[i][(size_t)sample * a.channels + channel] = D;
        s.r += D;
        s.mask[i] = T[i];
    }
    s.mask[1] += s.r;
    return s;
}
// A word's results: m the opened d, U its masks; UT, R, Q the dealer's.
__device__ __forceinline__ void group_word(const GroupArgs& a, const GroupScale& s, u64 m, const u64 U[2], const u64 UT[2], const u64 R[2], const u64 Q[2],
                                           u64 z[2], u64 N[2]) {
    const int f = a.root.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u64 t = UT[i] + m * s.mask[i] + s.r * U[i] + s.bias[i];
        z[i] = i ? 0ull - norm_shift(0ull - t, f) : norm_shift(t, f);
    }
    if (!a.R[0]) return;
    N[0] = z[0] - R[0];
    N[1] = z[1] - R[1];
    const u64 b = N[0] + N[1];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u64 q = Q[i] + b * (2 * R[i] + (i ? b : 0ull)), square = i ? 0ull - norm_shift(0ull - q, f) : norm_shift(q, f);
        const u64 mix = a.k2 * square + a.k1 * z[i];
        z[i] = i ? a.k0 - norm_shift(0ull - mix, f) : norm_shift(mix, f);
    }
}

// A thread's words of a group, ACC accesses of W words: access k is the group's index + k * step of those that there are.
template <int W, int ACC>
struct GroupOwn {
    size_t at[ACC];              // in the dense tensors
    int channel[ACC];
    bool has[ACC], first[ACC];   // first: of the first position
    u64 m[ACC][W], U[2][ACC][W];  // m: party 0's share of x until the mean is known, then the opened d
    u64 x1[ACC][W];              // party 1's share of x
    u64* mine;                   // array j of party i, access k: mine + ((j 2 + i) ACC + k) stride W
    int stride, sample;

    __device__ __forceinline__ u64* place(int array, int i, int k) const { return mine + (size_t)((array * 2 + i) * ACC + k) * stride * W; }

    // Loads, and both parties' sums of x; what `finish` reads is on its way to shared memory meanwhile.  Party 1's masks stay in U[1].
    __device__ __forceinline__ void open(const GroupArgs& a, int group, int index, int step, bool live, u64* places, int place_stride, u64 sum[2]) {
        mine = places;
        stride = place_stride;
        sample = group / a.groups;
        const int base = (group - sample * a.groups) * a.per;
        u64 x[2][ACC][W];
#pragma unroll
        for (int k = 0; k < ACC; ++k) {
            const int e = (index + k * step) * W;
            has[k] = live && e < a.count;
            const int p = has[k] ? e / a.per : 0;
            channel[k] = base + (has[k] ? e - p * a.per : 0);
            first[k] = p == 0;
            const size_t row = (size_t)sample * a.positions + p, from = row * a.x_stride + channel[k];
            at[k] = row * a.channels + channel[k];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int j = 0; j < W; ++j) x[i][k][j] = U[i][k][j] = 0ull;
                if (has[k]) {
                    group_load<W>(a.X[i] + from, x[i][k]);
                    group_load<W>(a.U[i] + at[k], U[i][k]);
                }
            }
        }
        const bool per_word = a.positions == 1 && a.gain[0];
#pragma unroll
        for (int k = 0; k < ACC; ++k)
            if (has[k])
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    group_fetch<W>(place(0, i, k), a.UT[i] + at[k]);
                    if (a.R[0]) {
                        group_fetch<W>(place(1, i, k), a.R[i] + at[k]);
                        group_fetch<W>(place(2, i, k), a.Q[i] + at[k]);
                    }
                    if (per_word) {
                        const int next = a.R[0] ? 3 : 1;
                        group_fetch<W>(place(next, i, k), a.VW[i] + at[k]);
                        group_fetch<W>(place(next + 1, i, k), a.T[i] + at[k]);
                    }
                }
        sum[0] = sum[1] = 0ull;
#pragma unroll
        for (int k = 0; k < ACC; ++k)
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    sum[i] += x[i][k][j];
                    (i ? x1 : m)[k][j] = x[i][k][j];
                }
    }

    // The message, and both parties' part of the sum of squares.
    __device__ __forceinline__ void square(const GroupArgs& a, const u64 mean[2], u64 sq[2]) {
        sq[0] = sq[1] = 0ull;
#pragma unroll
        for (int k = 0; k < ACC; ++k) {
            u64 msg[2][W];
#pragma unroll
            for (int j = 0; j < W; ++j) {
                msg[0][j] = m[k][j] - mean[0] - U[0][k][j];
                msg[1][j] = x1[k][j] - mean[1] - U[1][k][j];
                m[k][j] = has[k] ? msg[0][j] + msg[1][j] : 0ull;                 // the exchange
                sq[0] += m[k][j] * U[0][k][j];
                sq[1] += m[k][j] * (2 * U[1][k][j] + m[k][j]);
            }
            if (has[k])
#pragma unroll
                for (int i = 0; i < 2; ++i) group_store<W>(a.M[i] + at[k], msg[i]);
        }
        sq[0] *= 2;
    }

    // root: the opened y - v, v: both parties' shares of its mask; table: the channels' scales, from channel `base` on, or null.
    __device__ __forceinline__ void finish(const GroupArgs& a, u64 root, const u64 v[2], const GroupScale* table, int base) {
        norm_fetch_wait();
        const bool per_word = a.positions == 1 && a.gain[0];
        const int next = a.R[0] ? 3 : 1;
#pragma unroll
        for (int k = 0; k < ACC; ++k) {
            if (!has[k]) continue;
            u64 z[2][W], N[2][W];
#pragma unroll
            for (int j = 0; j < W; ++j) {
                u64 R[2] = {0ull, 0ull}, Q[2] = {0ull, 0ull}, UT[2], u[2], zz[2], nn[2];
                GroupScale s;
                if (table) {
                    s = table[channel[k] + j - base];
                } else {
                    u64 VW[2] = {0ull, 0ull}, T[2] = {0ull, 0ull};
                    if (a.gain[0])
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const size_t o = (size_t)sample * a.channels + channel[k] + j;
                            VW[i] = per_word ? place(next, i, k)[j] : __ldg(a.VW[i] + o);
                            T[i] = per_word ? place(next + 1, i, k)[j] : __ldg(a.T[i] + o);
                        }
                    s = group_scale(a, root, v, sample, channel[k] + j, VW, T, first[k]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    UT[i] = place(0, i, k)[j];
                    u[i] = U[i][k][j];
                    if (a.R[0]) {
                        R[i] = place(1, i, k)[j];
                        Q[i] = place(2, i, k)[j];
                    }
                }
                group_word(a, s, m[k][j], u, UT, R, Q, zz, nn);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    z[i][j] = zz[i];
                    N[i][j] = nn[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                group_store<W>(a.Z[i] + at[k], z[i]);
                if (a.R[0]) group_store<W>(a.N[i] + at[k], N[i]);
            }
        }
    }
};

// Groups of up to TILE_WORDS words: a CTA has as many as its threads cover, four words a thread; one warp works out their means and roots, a pair
// of lanes a group.  512 tokens x 32 heads of 128 with activation: 91 us, 0.66 of the measured copy rate; a CTA's five sit on an SM, and what they cover for
// one another is a root's chain of products, 0.2 us a step for a group alone on its SM.  Not all of it: with two steps 72 us, with 24 124, of which the steps' own words are
// 8 at the copy rate.  One token of 12 heads of 64: 6.5 us, of which the chain 2.
template <int W>
__global__ void __launch_bounds__(group::TILE_THREADS, group::TILE_CTAS)
group_tile_kernel(const __grid_constant__ GroupArgs a) {
    extern __shared__ __align__(16) uint8_t group_smem[];
    __shared__ u64 sums[group::TILE_THREADS][2], value[group::TILE_GROUPS][2];
    constexpr int ACC = 4 / W;
    const int quads = (a.count + 3) / 4, tile = group::tile_groups(quads), steps = a.root.steps;
    const int count = norm::words(steps), sent = norm::openings(steps);
    u64* const places = reinterpret_cast<u64*>(group_smem);
    u64* const words = places + (size_t)group::arrays(a.R[0], a.positions == 1 && a.gain[0]) * 2 * 4 * blockDim.x;   // [party][group][count], party 1's negated
    u64* const opened = words + 2 * tile * count;                                                                    // [party][group][sent]
    const int first = blockIdx.x * tile, groups = min(tile, a.all - first), sub = threadIdx.x / quads, quad = threadIdx.x - sub * quads;
    const bool live = sub < groups;
    const int group = first + (live ? sub : 0);
    pdl_wait();
    GroupOwn<W, ACC> own;
    u64 sum[2], sq[2];
    own.open(a, group, quad, quads, live, places + threadIdx.x * W, blockDim.x, sum);
    for (int k = threadIdx.x; k < groups * count; k += blockDim.x) {
        words[k] = __ldcs(a.words[0] + (size_t)first * count + k);
        words[tile * count + k] = 0ull - __ldcs(a.words[1] + (size_t)first * count + k);
    }
    // a group's sums: lanes 2g and 2g + 1 have group g's of either party, the lanes beyond help
    const int width = 2 << (32 - __clz(tile - 1)), lane = threadIdx.x & 31, of = lane & (width - 1), party = lane & 1, g = min(of >> 1, tile - 1);
    auto total = [&] {
        u64 t = 0ull;
        for (int k = lane / width; k < quads; k += 32 / width) t += sums[g * quads + k][party];
        for (int o = width; o < 32; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        return t;
    };
    sums[threadIdx.x][0] = sum[0];
    sums[threadIdx.x][1] = sum[1];
    __syncthreads();
    if (threadIdx.x < 32) {
        u64 t = total();
        t = party ? 0ull - (0ull - t) / (u64)a.count : t / (u64)a.count;
        if (lane < 2 * groups) value[g][party] = t;
    }
    __syncthreads();
    own.square(a, value[live ? sub : 0], sq);
    sums[threadIdx.x][0] = sq[0];
    sums[threadIdx.x][1] = 0ull - sq[1];
    __syncthreads();
    if (threadIdx.x < 32) {
        const u64 t = total();
        const bool mine = lane < 2 * groups;
        const u64 root = norm_root(a.root, t, words + (party * tile + g) * count, opened + (party * tile + g) * sent, mine, party);
        if (mine) value[g][0] = root;
    }
    __syncthreads();
    for (int i = 0; i < 2; ++i)
        for (int k = threadIdx.x; k < groups * sent; k += blockDim.x) {
            const u64 t = opened[i * tile * sent + k];
            __stcs(a.S[i] + (size_t)first * sent + k, i ? 0ull - t : t);
        }
    if (!live) return;
    const u64 v[2] = {words[(sub + 1) * count - 1], 0ull - words[(tile + sub + 1) * count - 1]};
    own.finish(a, value[sub][0], v, nullptr, 0);
}

// Longer groups: a cluster of CTAs per group, eight words a thread.  Every warp's sums are written to every CTA of the cluster, and every CTA works
// out mean and root for itself.
template <int W>
__global__ void __launch_bounds__(group::CLUSTER_THREADS, group::CLUSTER_CTAS)
group_cluster_kernel(const __grid_constant__ GroupArgs a) {
    extern __shared__ __align__(16) uint8_t group_smem[];
    __shared__ u64 partial[2][group::MAX_CLUSTER * group::CLUSTER_THREADS / 32][2], value[2];
    constexpr int ACC = 8 / W;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, party = threadIdx.x & 1, warps = blockDim.x >> 5, steps = a.root.steps;
    const int count = norm::words(steps), sent = norm::openings(steps);
    u64* const places = reinterpret_cast<u64*>(group_smem);
    u64* const words = places + (size_t)group::arrays(a.R[0], a.positions == 1 && a.gain[0]) * 2 * 8 * blockDim.x;   // [party][count], party 1's negated
    u64* const opened = words + 2 * count;                                                                           // [party][sent]
    GroupScale* const scales = reinterpret_cast<GroupScale*>(opened + 2 * sent);
    uint32_t rank, cluster;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
    const int group = (int)(blockIdx.x / cluster);
    // (a CTA's shared memory is written to by the others when it has begun)
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    pdl_wait();
    GroupOwn<W, ACC> own;
    u64 sum[2], sq[2];
    own.open(a, group, (int)(rank * blockDim.x + threadIdx.x), (int)(cluster * blockDim.x), true, places + threadIdx.x * W, blockDim.x, sum);
    for (int k = threadIdx.x; k < count; k += blockDim.x) {
        words[k] = __ldcs(a.words[0] + (size_t)group * count + k);
        words[count + k] = 0ull - __ldcs(a.words[1] + (size_t)group * count + k);
    }
    // The cluster's sums, in every CTA: even lanes of its first warp have party 0's, odd lanes party 1's.
    auto total = [&](int round, u64 v[2]) {
        const u64 mine = norm_lane_sum(v, party);
        if (cluster > 1) {
            __syncwarp();
            if (round == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (lane < 2 * cluster) {
                uint32_t there;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there)
                             : "r"((uint32_t)__cvta_generic_to_shared(&partial[round][rank * warps + warp][party])), "r"(lane >> 1));
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(mine) : "memory");
            }
            __syncwarp();
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        } else {
            if (lane < 2) partial[round][warp][party] = mine;
            __syncthreads();
        }
        u64 t = 0ull;
        if (warp == 0) {
            for (int k = lane >> 1; k < (int)cluster * warps; k += 16) t += partial[round][k][party];
#pragma unroll
            for (int o = 2; o < 32; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        }
        return t;
    };
    u64 t = total(0, sum);
    if (warp == 0) {
        t = party ? 0ull - (0ull - t) / (u64)a.count : t / (u64)a.count;
        if (lane < 2) value[party] = t;
    }
    __syncthreads();
    own.square(a, value, sq);
    t = total(1, sq);
    u64* const root = &partial[0][0][0];                     // nobody writes there any more
    if (warp == 0) {
        const u64 opened_root = norm_root(a.root, party ? 0ull - t : t, words + party * count, opened + party * sent, lane < 2, party);
        if (lane == 0) *root = opened_root;
    }
    __syncthreads();
    if (warp == 0 && rank == 0)
        for (int i = 0; i < 2; ++i)
            for (int k = lane; k < sent; k += 32) {
                const u64 s = opened[i * sent + k];
                __stcs(a.S[i] + (size_t)group * sent + k, i ? 0ull - s : s);
            }
    const u64 v[2] = {words[count - 1], 0ull - words[2 * count - 1]};
    // every channel's scale once, where there are several positions
    const bool table = a.positions > 1 && a.per <= group::TABLE;
    const int sample = group / a.groups, base = (group - sample * a.groups) * a.per;
    if (table) {
        for (int c = threadIdx.x; c < a.per; c += blockDim.x) {
            u64 VW[2] = {0ull, 0ull}, T[2] = {0ull, 0ull};
            if (a.gain[0])
                for (int i = 0; i < 2; ++i) {
                    VW[i] = __ldg(a.VW[i] + (size_t)sample * a.channels + base + c);
                    T[i] = __ldg(a.T[i] + (size_t)sample * a.channels + base + c);
                }
            scales[c] = group_scale(a, *root, v, sample, base + c, VW, T, rank == 0);
        }
        __syncthreads();
    }
    own.finish(a, *root, v, table ? scales : nullptr, base);
}

// ---------------------------------------------------------------------------
// Groups that fit no cluster: three passes over slabs of positions, the sums of a group gathered by 64-bit additions, which are exact in any
// order.  What the second and third pass read again is the L2's where it fits.  4096 positions x 320 channels in 32 groups: 11 + 15 + 38 us by themselves, 60 a
// pass; 8 x 1024 x 640 in 32: 19 + 45 + 122, 191.  Of 16 arrays that have to move 6 move twice.
// A CTA has a slab of a tile of channels, whole groups or a part of one, a thread a column of W channels of it in every `subs`-th position.
// ---------------------------------------------------------------------------
struct GroupSlab {
    int sample, group0, groups, part, channel, column, p0, p1, g;        // channel: of this thread's first word, -1: none; g: its group of the tile's
};
template <int W>
__device__ __forceinline__ GroupSlab group_slab(const GroupArgs& a) {
    GroupSlab s;
    const int slab = blockIdx.x % a.slabs, t = blockIdx.x / a.slabs, tile = t % a.tiles, sub = threadIdx.x / a.units;
    s.sample = t / a.tiles;
    s.column = (threadIdx.x - sub * a.units) * W;
    int base, channels;
    if (a.parts == 1) {
        s.group0 = tile * a.tile_groups;
        s.groups = min(a.tile_groups, a.groups - s.group0);
        s.part = 0;
        base = s.group0 * a.per;
        channels = s.groups * a.per;
    } else {
        s.group0 = tile / a.parts;
        s.groups = 1;
        s.part = tile - s.group0 * a.parts;
        base = s.group0 * a.per + s.part * a.units * W;
        channels = min(a.units * W, a.per - s.part * a.units * W);
    }
    const bool has = s.column < channels && sub < a.subs;
    s.channel = has ? base + s.column : -1;
    s.g = has && a.parts == 1 ? s.column / a.per : 0;
    s.p0 = slab * a.slab + sub;
    s.p1 = min((slab + 1) * a.slab, a.positions);
    return s;
}
// Adds both parties' sums of a CTA's threads to those of their groups.
__device__ __forceinline__ void group_gather(const GroupArgs& a, const GroupSlab& s, u64* totals, const u64 v[2]) {
    __shared__ u64 sums[group::SLAB_GROUPS][2];
    for (int k = threadIdx.x; k < 2 * s.groups; k += blockDim.x) sums[k >> 1][k & 1] = 0ull;
    __syncthreads();
    if (s.channel >= 0) {
        atomicAdd(&sums[s.g][0], v[0]);
        atomicAdd(&sums[s.g][1], v[1]);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * s.groups; k += blockDim.x) atomicAdd(totals + ((size_t)s.sample * a.groups + s.group0) * 2 + k, sums[k >> 1][k & 1]);
}

template <int W>
__global__ void __launch_bounds__(group::SLAB_THREADS)
group_sum_kernel(const __grid_constant__ GroupArgs a) {
    pdl_wait();
    const GroupSlab s = group_slab<W>(a);
    u64 sum[2] = {0ull, 0ull};
    if (s.channel >= 0) {
        const size_t at = (size_t)s.sample * a.positions * a.x_stride + s.channel;
#pragma unroll 4
        for (int p = s.p0; p < s.p1; p += a.subs) {
            u64 x[2][W];
#pragma unroll
            for (int i = 0; i < 2; ++i) group_read<W>(a.X[i] + at + (size_t)p * a.x_stride, x[i]);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                sum[0] += x[0][j];
                sum[1] += x[1][j];
            }
        }
    }
    group_gather(a, s, a.sums, sum);
}

template <int W>
__global__ void __launch_bounds__(group::SLAB_THREADS)
group_open_kernel(const __grid_constant__ GroupArgs a) {
    __shared__ u64 means[group::SLAB_GROUPS][2];
    pdl_wait();
    const GroupSlab s = group_slab<W>(a);
    for (int k = threadIdx.x; k < 2 * s.groups; k += blockDim.x) {
        const u64 t = a.sums[((size_t)s.sample * a.groups + s.group0) * 2 + k];
        means[k >> 1][k & 1] = k & 1 ? 0ull - (0ull - t) / (u64)a.count : t / (u64)a.count;
    }
    __syncthreads();
    u64 sq[2] = {0ull, 0ull};
    if (s.channel >= 0) {
        const size_t at = (size_t)s.sample * a.positions, mean0 = means[s.g][0], mean1 = means[s.g][1];
#pragma unroll 2
        for (int p = s.p0; p < s.p1; p += a.subs) {
            const size_t x_at = (at + p) * a.x_stride + s.channel, o = (at + p) * a.channels + s.channel;
            u64 x[2][W], u[2][W];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                group_read<W>(a.X[i] + x_at, x[i]);
                group_read<W>(a.U[i] + o, u[i]);
            }
#pragma unroll
            for (int j = 0; j < W; ++j) {
                x[0][j] -= mean0 + u[0][j];
                x[1][j] -= mean1 + u[1][j];
                const u64 m = x[0][j] + x[1][j];                 // the exchange
                sq[0] += 2 * m * u[0][j];
                sq[1] += m * (2 * u[1][j] + m);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (W == 2) *reinterpret_cast<ulonglong2*>(a.M[i] + o) = make_ulonglong2(x[i][0], x[i][W - 1]);
                else a.M[i][o] = x[i][0];
            }
        }
    }
    group_gather(a, s, a.sums + 2 * (size_t)a.all, sq);
}

// Every CTA works out the roots of its groups, a pair of lanes each; then every thread the scale of its column.  A chain of products that takes some
// microseconds before the first word: so there are no more CTAs than run at once (SLAB_APPLY threads an SM).
template <int W>
__global__ void __launch_bounds__(group::SLAB_THREADS, group::SLAB_APPLY / group::SLAB_THREADS)
group_apply_kernel(const __grid_constant__ GroupArgs a) {
    extern __shared__ __align__(16) uint8_t group_smem[];
    __shared__ u64 roots[group::SLAB_GROUPS];
    const int steps = a.root.steps, count = norm::words(steps), sent = norm::openings(steps);
    u64* const words = reinterpret_cast<u64*>(group_smem);               // [party][group][count], party 1's negated
    u64* const opened = words + 2 * a.tile_groups * count;               // [party][group][sent]
    pdl_wait();
    const GroupSlab s = group_slab<W>(a);
    const size_t first = (size_t)s.sample * a.groups + s.group0;
    for (int k = threadIdx.x; k < s.groups * count; k += blockDim.x) {
        words[k] = __ldg(a.words[0] + first * count + k);
        words[a.tile_groups * count + k] = 0ull - __ldg(a.words[1] + first * count + k);
    }
    __syncthreads();
    if (threadIdx.x < ((2 * s.groups + 31) & ~31)) {
        const int party = threadIdx.x & 1, g = min((int)threadIdx.x >> 1, s.groups - 1);
        const u64 sq = a.sums[2 * (size_t)a.all + (first + g) * 2 + party];
        const u64 root = norm_root(a.root, party ? 0ull - sq : sq, words + (party * a.tile_groups + g) * count, opened + (party * a.tile_groups + g) * sent,
                                   (int)threadIdx.x < 2 * s.groups, party);
        if ((int)threadIdx.x < 2 * s.groups) roots[g] = root;
    }
    __syncthreads();
    const bool tells = blockIdx.x % a.slabs == 0;
    if (tells && s.part == 0)
        for (int i = 0; i < 2; ++i)
            for (int k = threadIdx.x; k < s.groups * sent; k += blockDim.x) {
                const u64 t = opened[i * a.tile_groups * sent + k];
                a.S[i][first * sent + k] = i ? 0ull - t : t;
            }
    if (s.channel < 0) return;
    const u64 v[2] = {words[(s.g + 1) * count - 1], 0ull - words[(a.tile_groups + s.g + 1) * count - 1]};
    GroupScale scale[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
        u64 VW[2] = {0ull, 0ull}, T[2] = {0ull, 0ull};
        if (a.gain[0])
            for (int i = 0; i < 2; ++i) {
                VW[i] = __ldg(a.VW[i] + (size_t)s.sample * a.channels + s.channel + j);
                T[i] = __ldg(a.T[i] + (size_t)s.sample * a.channels + s.channel + j);
            }
        scale[j] = group_scale(a, roots[s.g], v, s.sample, s.channel + j, VW, T, tells && s.p0 == 0);
    }
    const size_t at = (size_t)s.sample * a.positions * a.channels + s.channel;
#pragma unroll 1
    for (int p = s.p0; p < s.p1; p += a.subs) {
        const size_t o = at + (size_t)p * a.channels;
        u64 M[2][W], U[2][W], UT[2][W], R[2][W], Q[2][W], z[2][W], N[2][W];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            group_load<W>(a.M[i] + o, M[i]);
            group_load<W>(a.U[i] + o, U[i]);
            group_load<W>(a.UT[i] + o, UT[i]);
            if (a.R[0]) {
                group_load<W>(a.R[i] + o, R[i]);
                group_load<W>(a.Q[i] + o, Q[i]);
            }
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const u64 u[2] = {U[0][j], U[1][j]}, ut[2] = {UT[0][j], UT[1][j]}, r[2] = {R[0][j], R[1][j]}, q[2] = {Q[0][j], Q[1][j]};
            u64 zz[2], nn[2];
            group_word(a, scale[j], M[0][j] + M[1][j], u, ut, r, q, zz, nn);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                z[i][j] = zz[i];
                N[i][j] = nn[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            group_store<W>(a.Z[i] + o, z[i]);
            if (a.R[0]) group_store<W>(a.N[i] + o, N[i]);
        }
    }
}

}  // namespace comet
