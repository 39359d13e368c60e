// Group norm in one pass: a sample's slab of channels stays on chip between its statistics and its output.
//
// The work item is (sample, slab), a slab being neighbouring whole groups, 128 bytes of channels wide where the groups
// allow it, over all positions.  A cluster of K CTAs holds it in shared memory, each CTA an equal share of the positions,
// each thread up to NV vectors of 16 bytes of one column: x is read once from HBM and y written once, which is the floor
// of the operation.  The clusters are persistent: each keeps one slab and walks over samples, so that what depends on
// the channels is set up once, and while it works on one sample the copies of the next are under way.  A thread copies
// (cp.async) exactly the vectors that it reads itself, so the pipeline needs no barrier and no wait on another thread.
// What a CTA knows of its groups goes to its peers through distributed shared memory, joined in the order of the ranks.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <numeric>

#include "cr_elem.cuh"
#include "cr_tcgen05.cuh"

#ifndef CR_GN_FMIN
#define CR_GN_FMIN 3
#define CR_GN_BMIN 2
#define CR_GN_FNV 8
#define CR_GN_BNV 4
#endif

namespace cr {
namespace {

constexpr int kTH = 256, kWarps = kTH / 32;
constexpr int kMaxCluster = 8;

struct Slab {
    int sc;              // channels of a slab (the last one of a row may have fewer)
    int slabs;           // slabs per row of channels
    int cluster;         // CTAs per item
    int rows_per_cta;
    int cg;
    int channels;
    int samples;
    int walkers;         // clusters that share the samples of a slab
    int entries;         // backward: floats that one sample's sums of the CTA's lines need
    int64_t positions;
};

// Where a thread stands in the items of its cluster.
struct Spot {
    int slab, rank, first_sample, rows, width, vpr, rt, col, j, c0, mine;   // j < 0: idle; mine: rows of this thread
    int groups, cv;                                                       // groups of the slab; vectors per group
};
template <int VEC>
__device__ __forceinline__ Spot spot(const Slab &s) {
    Spot p;
    const uint32_t cluster = blockIdx.x / (uint32_t)s.cluster;
    p.rank = (int)(blockIdx.x % (uint32_t)s.cluster);
    p.first_sample = (int)(cluster / (uint32_t)s.slabs);
    p.slab = (int)(cluster % (uint32_t)s.slabs);
    p.rows = (int)max((int64_t)0, min((int64_t)s.rows_per_cta, s.positions - (int64_t)p.rank * s.rows_per_cta));
    p.width = min(s.sc, s.channels - p.slab * s.sc);
    p.vpr = p.width / VEC;
    p.rt = kTH / p.vpr;
    p.col = (int)threadIdx.x % p.vpr;
    const int j = (int)threadIdx.x / p.vpr;
    p.j = j < p.rt ? j : -1;
    p.c0 = p.slab * s.sc + p.col * VEC;
    p.mine = p.j < 0 || p.j >= p.rows ? 0 : (p.rows - p.j + p.rt - 1) / p.rt;
    p.groups = p.width / s.cg;
    p.cv = s.cg / VEC;
    return p;
}

// Sums the entries [g * per, (g + 1) * per) of `in` into out[g] for g < count: a warp per group, in one order.
__device__ __forceinline__ void fold(const float *in, float *out, int count, int per) {
    const int lane = (int)threadIdx.x & 31;
    for (int g = (int)threadIdx.x >> 5; g < count; g += kWarps) {
        float t = 0.f;
        for (int e = lane; e < per; e += 32) t += in[g * per + e];
#pragma unroll
        for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) out[g] = t;
    }
}

// Adds v over the lanes of the warp that hold the same column: lane, lane + vpr, .. (vpr divides 32).
template <int N>
__device__ __forceinline__ void sum_rows_of_warp(float (&v)[N], int vpr) {
    for (int o = 16; o >= vpr; o >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
}

// Sums over the CTA, by group; every thread gets the sums of its own groups (one where a vector lies inside a group,
// else one per channel of the vector).  `area`: kTH * kG floats, another one in the next call; `sums`: [groups].
// Where a warp holds whole rows and the groups a power of two of vectors, lanes add up the warp and one barrier does;
// otherwise every entry goes through shared memory.
template <int N, int VEC, bool UNI>
__device__ __forceinline__ void sum_groups(float (&acc)[N][UNI ? 1 : VEC], const Spot &p, int cg, float *area, float *sums) {
    constexpr int kG = UNI ? 1 : VEC;
    const int lane = (int)threadIdx.x & 31, warp = (int)threadIdx.x >> 5;
    const bool folded = 32 % p.vpr == 0;
    if (UNI && folded && (p.cv & (p.cv - 1)) == 0) {
        float t[N];
#pragma unroll
        for (int n = 0; n < N; ++n) t[n] = acc[n][0];
        sum_rows_of_warp<N>(t, p.vpr);
        for (int o = 1; o < p.cv; o <<= 1) {
#pragma unroll
            for (int n = 0; n < N; ++n) t[n] += __shfl_xor_sync(0xffffffffu, t[n], o);
        }
        const int g = p.col / p.cv;
        if (lane < p.vpr && p.col == g * p.cv) {
#pragma unroll
            for (int n = 0; n < N; ++n) area[(n * p.groups + g) * kWarps + warp] = t[n];
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float4 *line = reinterpret_cast<const float4 *>(area + (n * p.groups + g) * kWarps);
            const float4 a = line[0], b = line[1];
            acc[n][0] = ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (p.j >= 0) {
#pragma unroll
                for (int i = 0; i < kG; ++i) area[(p.col * kG + i) * p.rt + p.j] = acc[n][i];
            }
            __syncthreads();
            fold(area, sums, p.groups, (UNI ? p.cv : cg) * p.rt);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kG; ++i) acc[n][i] = sums[(p.col * VEC + i) / cg];
            if (n + 1 < N) __syncthreads();
        }
    }
}

// Writes `v` to the place of `mine` in the shared memory of every CTA of the cluster.  Each CTA hands out what it knows
// and reads only its own memory after the one barrier that follows: a read from a peer is a round trip, these are not.
__device__ __forceinline__ void hand_out(const float *mine, float v, int cluster) {
    for (int r = 0; r < cluster; ++r)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(i8::map_to_rank(i8::smem_u32(mine), (uint32_t)r)), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest group have landed (for the thread that issued them).
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
template <typename T>
__device__ __forceinline__ Packed<T, 16 / (int)sizeof(T)> held(uint32_t at) {
    Packed<T, 16 / (int)sizeof(T)> r;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "r"(at) : "memory");
    return r;
}

// z of the activation, for a pair.  Where the activation has a kink (relu) every step is rounded by itself, in the
// forward and the backward pass alike, so that the slope belongs to the z whose value was stored; elsewhere `scaled`
// = rstd gamma goes in one step.
template <int ACT>
__device__ __forceinline__ F2 z_of(F2 centred, F2 rstd, F2 gamma, F2 scaled, F2 beta) {
    if constexpr (ACT == kActRelu) return add2(mul2(mul2(centred, rstd), gamma), beta);
    return fma2(centred, scaled, beta);
}
__device__ __forceinline__ F2 sigmoid2(F2 z) {
    const F2 t = mul2(z, f2(-kLog2e));
    const F2 d = add2({exp2_approx(t.x), exp2_approx(t.y)}, f2(1.f));
    return {recip_approx(d.x), recip_approx(d.y)};
}

// The pair i of a vector, from one value per group (UNI) or per channel.
template <bool UNI, int N>
__device__ __forceinline__ F2 pair_of(const float (&v)[N], int i) {
    if constexpr (UNI) return f2(v[0]);
    else return {v[2 * i], v[2 * i + 1]};
}

// UNI: every vector lies inside one group.
template <typename T, int NV, bool UNI, int ACT>
__global__ void __launch_bounds__(kTH, NV <= 8 ? CR_GN_FMIN : 1) cr_group_norm_kernel(const GroupNormArgs a, const Slab s) {
    constexpr int VEC = 16 / (int)sizeof(T), NP = VEC / 2, kG = UNI ? 1 : VEC;   // kG: groups a thread may touch
    extern __shared__ __align__(16) float sm[];
    const Spot p = spot<VEC>(s);
    if (s.cluster > 1) cluster_meet();         // a CTA's memory may be written from outside once the CTA runs
    const int gmax = s.sc / s.cg;
    float *area = sm + 2 * NV * kTH * 4;       // [2][kTH * kG]
    float *sums = area + 2 * kTH * kG;         // [gmax]
    float *peers = sums + gmax;                // [2][cluster][2][gmax]: sums and centred squares of every CTA, two samples' worth
    const uint32_t mine_at = i8::smem_u32(sm) + threadIdx.x * 16;
    const T *src = static_cast<const T *>(a.x) + (((int64_t)p.first_sample * s.positions + (int64_t)p.rank * s.rows_per_cta + max(p.j, 0)) * a.ld_x + p.c0);
    const int64_t step_x = (int64_t)p.rt * a.ld_x, step_y = (int64_t)p.rt * a.ld_y;
    const int64_t next_x = (int64_t)s.walkers * s.positions * a.ld_x;
    auto fetch = [&](int buf, const T *from) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) copy16(mine_at + (uint32_t)(buf * NV + k) * (kTH * 16), from + k * step_x);
    };
    fetch(0, src);
    copies_issued();
    F2 gamma[NP], beta[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        gamma[i] = a.gamma ? F2{__ldg(a.gamma + p.c0 + 2 * i), __ldg(a.gamma + p.c0 + 2 * i + 1)} : f2(1.f);
        beta[i] = a.beta ? F2{__ldg(a.beta + p.c0 + 2 * i), __ldg(a.beta + p.c0 + 2 * i + 1)} : f2(0.f);
    }
    const float inv = 1.f / fmaxf((float)p.rows * (float)s.cg, 1.f);
    const float all = (float)s.positions * (float)s.cg;
    int buf = 0;
    for (int n = p.first_sample; n < s.samples; n += s.walkers, buf ^= 1) {
        src += next_x;
        if (n + s.walkers < s.samples) fetch(buf ^ 1, src);
        copies_issued();
        copies_landed();
        const uint32_t at = mine_at + (uint32_t)(buf * NV) * (kTH * 16);
        // sums, then squares of the distances from the CTA's own mean
        F2 t[NP];
        float acc[1][kG], mean[kG], rstd[kG];
        auto by_group = [&]() {
            if constexpr (UNI) {
                acc[0][0] = 0.f;
#pragma unroll
                for (int i = 0; i < NP; ++i) acc[0][0] += t[i].x + t[i].y;
            } else {
#pragma unroll
                for (int i = 0; i < NP; ++i) { acc[0][2 * i] = t[i].x; acc[0][2 * i + 1] = t[i].y; }
            }
        };
#pragma unroll
        for (int i = 0; i < NP; ++i) t[i] = f2(0.f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) {
                F2 f[NP];
                unpack2<T, VEC>(held<T>(at + k * (kTH * 16)), f);
#pragma unroll
                for (int i = 0; i < NP; ++i) t[i] = add2(t[i], f[i]);
            }
        by_group();
        sum_groups<1, VEC, UNI>(acc, p, s.cg, area, sums);
#pragma unroll
        for (int i = 0; i < kG; ++i) mean[i] = acc[0][i] * inv;
#pragma unroll
        for (int i = 0; i < NP; ++i) t[i] = f2(0.f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) {
                F2 f[NP];
                unpack2<T, VEC>(held<T>(at + k * (kTH * 16)), f);
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const F2 m = pair_of<UNI>(mean, i), d = add2(f[i], {-m.x, -m.y});
                    t[i] = fma2(d, d, t[i]);
                }
            }
        by_group();
        sum_groups<1, VEC, UNI>(acc, p, s.cg, area + kTH * kG, sums);
        // the first thread of each group speaks for it
        auto leads = [&](int i) { return p.j == 0 && (p.col * VEC + i) % s.cg == 0; };
        if (s.cluster > 1) {
            float *box = peers + (size_t)buf * s.cluster * 2 * gmax;
#pragma unroll
            for (int i = 0; i < kG; ++i)
                if (leads(i)) {
                    const int g = (p.col * VEC + i) / s.cg;
                    hand_out(&box[p.rank * 2 * gmax + g], mean[i], s.cluster);
                    hand_out(&box[(p.rank * 2 + 1) * gmax + g], acc[0][i], s.cluster);
                }
            cluster_meet();
            // join the CTAs: means weighted by their rows, centred squares moved to the common mean
#pragma unroll
            for (int i = 0; i < kG; ++i) {
                const float *in = box + (p.col * VEC + i) / s.cg;
                float total = 0.f, m2 = 0.f;
                for (int r = 0; r < s.cluster; ++r) {
                    const int rows = (int)max((int64_t)0, min((int64_t)s.rows_per_cta, s.positions - (int64_t)r * s.rows_per_cta));
                    total = fmaf((float)rows * (float)s.cg, in[r * 2 * gmax], total);
                }
                mean[i] = total / all;
                for (int r = 0; r < s.cluster; ++r) {
                    const int rows = (int)max((int64_t)0, min((int64_t)s.rows_per_cta, s.positions - (int64_t)r * s.rows_per_cta));
                    const float d = in[r * 2 * gmax] - mean[i];
                    m2 += rows ? fmaf((float)rows * (float)s.cg * d, d, in[(r * 2 + 1) * gmax]) : 0.f;
                }
                acc[0][i] = m2;
            }
        }
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            rstd[i] = 1.f / sqrtf(acc[0][i] / all + a.eps);
            if (a.mean && p.rank == 0 && leads(i)) {
                const int64_t g = (int64_t)n * a.groups + p.slab * gmax + (p.col * VEC + i) / s.cg;
                a.mean[g] = mean[i];
                a.rstd[g] = rstd[i];
            }
        }
        const int64_t row = (int64_t)n * s.positions + (int64_t)p.rank * s.rows_per_cta + max(p.j, 0);
        T *dst = static_cast<T *>(a.y) + (row * a.ld_y + p.c0);
        unsigned long long e = a.drop.offset + (unsigned long long)(row * s.channels + p.c0);
        const unsigned long long step_e = (unsigned long long)p.rt * s.channels;
        F2 scaled[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) scaled[i] = mul2(pair_of<UNI>(rstd, i), gamma[i]);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) {
                F2 f[NP];
                unpack2<T, VEC>(held<T>(at + k * (kTH * 16)), f);
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const F2 m = pair_of<UNI>(mean, i);
                    const F2 z = z_of<ACT>(add2(f[i], {-m.x, -m.y}), pair_of<UNI>(rstd, i), gamma[i], scaled[i], beta[i]);
                    if constexpr (ACT == kActSilu) f[i] = mul2(z, sigmoid2(z));
                    else f[i] = {act_value<ACT>(z.x), act_value<ACT>(z.y)};
                }
                if (a.drop.threshold) {
                    drop_select2<VEC>(f, a.drop, e);
#pragma unroll
                    for (int i = 0; i < NP; ++i) f[i] = mul2(f[i], f2(a.drop.scale));
                    e += step_e;
                }
                store_packed<T, VEC>(dst, pack2<T, VEC>(f));
                dst += step_y;
            }
    }
}

// Backward: x and dy are read once; dz takes the place of dy, in registers.  sum1, sum2 (may be null): the sums of dz and
// of dz xhat of each channel over this CTA's rows of a sample, [samples][cluster] rows of ld_sum.
template <typename T, int NV, bool UNI, int ACT>
__global__ void __launch_bounds__(kTH, NV <= 4 ? CR_GN_BMIN : 1) cr_group_norm_grad_kernel(const GroupNormArgs a, const Slab s, float *sum1, float *sum2, int64_t ld_sum) {
    constexpr int VEC = 16 / (int)sizeof(T), NP = VEC / 2, kG = UNI ? 1 : VEC;
    extern __shared__ __align__(16) float sm[];
    const Spot p = spot<VEC>(s);
    if (s.cluster > 1) cluster_meet();
    const int gmax = s.sc / s.cg;
    float *area = sm + 4 * NV * kTH * 4;       // [2][kTH * max(kG, 2)]: by turns, sample after sample
    float *entries = area + 2 * kTH * (UNI ? 2 : VEC);   // [2][lines][2 * width]
    const bool folded = 32 % p.vpr == 0;
    const int lines = folded ? kWarps : p.rt, line = folded ? (int)threadIdx.x >> 5 : p.j;
    const bool puts = folded ? ((int)threadIdx.x & 31) < p.vpr : p.j >= 0;
    const int both = 2 * p.width;
    float *sums = entries + 2 * s.entries;
    float *peers = sums + gmax;                // [2][cluster][2][gmax]
    const uint32_t mine_at = i8::smem_u32(sm) + threadIdx.x * 16;
    const int64_t row0 = (int64_t)p.first_sample * s.positions + (int64_t)p.rank * s.rows_per_cta + max(p.j, 0);
    const T *src = static_cast<const T *>(a.x) + (row0 * a.ld_x + p.c0);
    const T *up = static_cast<const T *>(a.dy) + (row0 * a.ld_dy + p.c0);
    const int64_t step_x = (int64_t)p.rt * a.ld_x, step_dy = (int64_t)p.rt * a.ld_dy, step_y = (int64_t)p.rt * a.ld_y;
    const int64_t next = (int64_t)s.walkers * s.positions;
    auto fetch = [&](int buf) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) {
                copy16(mine_at + (uint32_t)(buf * 2 * NV + k) * (kTH * 16), src + k * step_x);
                copy16(mine_at + (uint32_t)((buf * 2 + 1) * NV + k) * (kTH * 16), up + k * step_dy);
            }
    };
    fetch(0);
    copies_issued();
    F2 gamma[NP], beta[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        gamma[i] = a.gamma ? F2{__ldg(a.gamma + p.c0 + 2 * i), __ldg(a.gamma + p.c0 + 2 * i + 1)} : f2(1.f);
        beta[i] = a.beta ? F2{__ldg(a.beta + p.c0 + 2 * i), __ldg(a.beta + p.c0 + 2 * i + 1)} : f2(0.f);
    }
    const float all = (float)s.positions * (float)s.cg;
    const bool one = s.positions * s.cg == 1;  // groups of one value have m1 = gamma dz and no gradient at all
    const float kept = a.drop.threshold ? a.drop.scale : 1.f;
    float mean[kG], rstd[kG];
    auto statistics = [&](int n, float (&m)[kG], float (&r)[kG]) {
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            const int64_t g = (int64_t)n * a.groups + (p.c0 + i) / s.cg;
            m[i] = a.mean[g];
            r[i] = a.rstd[g];
        }
    };
    statistics(p.first_sample, mean, rstd);
    int buf = 0;
    for (int n = p.first_sample; n < s.samples; n += s.walkers, buf ^= 1) {
        float mean_next[kG], rstd_next[kG];
        if (n + s.walkers < s.samples) {
            src += next * a.ld_x;
            up += next * a.ld_dy;
            fetch(buf ^ 1);
            statistics(n + s.walkers, mean_next, rstd_next);
        }
        copies_issued();
        copies_landed();
        const uint32_t at_x = mine_at + (uint32_t)(buf * 2 * NV) * (kTH * 16), at_dy = at_x + NV * kTH * 16;
        const int64_t row = (int64_t)n * s.positions + (int64_t)p.rank * s.rows_per_cta + max(p.j, 0);
        unsigned long long e = a.drop.offset + (unsigned long long)(row * s.channels + p.c0);
        const unsigned long long step_e = (unsigned long long)p.rt * s.channels;
        F2 dz[NV][NP], s1[NP], s2[NP], scaled[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            s1[i] = s2[i] = f2(0.f);
            scaled[i] = mul2(gamma[i], pair_of<UNI>(rstd, i));
        }
        // dz without the scale of the kept elements, which the sums and the coefficients of dx take in
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) {
                F2 f[NP];
                unpack2<T, VEC>(held<T>(at_x + k * (kTH * 16)), f);
                unpack2<T, VEC>(held<T>(at_dy + k * (kTH * 16)), dz[k]);
                if (a.drop.threshold) {
                    drop_select2<VEC>(dz[k], a.drop, e);
                    e += step_e;
                }
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const F2 m = pair_of<UNI>(mean, i), centred = add2(f[i], {-m.x, -m.y});
                    if constexpr (ACT != kActNone) {
                        const F2 z = z_of<ACT>(centred, pair_of<UNI>(rstd, i), gamma[i], scaled[i], beta[i]);
                        if constexpr (ACT == kActSilu) {
                            const F2 sg = sigmoid2(z);
                            dz[k][i] = mul2(dz[k][i], mul2(sg, fma2(z, fma2(sg, f2(-1.f), f2(1.f)), f2(1.f))));
                        } else {
                            dz[k][i] = {z.x > 0.f ? dz[k][i].x : 0.f, z.y > 0.f ? dz[k][i].y : 0.f};
                        }
                    }
                    s1[i] = add2(s1[i], dz[k][i]);
                    s2[i] = fma2(dz[k][i], centred, s2[i]);
                }
            }
        if (sum1 || sum2) {     // the channels' sums, on their way while the groups are joined
            float t[2 * VEC];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const F2 r = pair_of<UNI>(rstd, i);
                t[2 * i] = s1[i].x * kept;
                t[2 * i + 1] = s1[i].y * kept;
                t[VEC + 2 * i] = s2[i].x * (r.x * kept);
                t[VEC + 2 * i + 1] = s2[i].y * (r.y * kept);
            }
            if (folded) sum_rows_of_warp<2 * VEC>(t, p.vpr);
            if (puts) {
                float *mine = entries + (buf * lines + line) * both + p.col * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    mine[i] = t[i];
                    mine[p.width + i] = t[VEC + i];
                }
            }
        }
        // the groups' sums of gamma dz and gamma dz xhat
        float acc[2][kG];
#pragma unroll
        for (int i = 0; i < kG; ++i) acc[0][i] = acc[1][i] = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            acc[0][UNI ? 0 : 2 * i] = fmaf(gamma[i].x, s1[i].x, acc[0][UNI ? 0 : 2 * i]);
            acc[0][UNI ? 0 : 2 * i + 1] = fmaf(gamma[i].y, s1[i].y, acc[0][UNI ? 0 : 2 * i + 1]);
            acc[1][UNI ? 0 : 2 * i] = fmaf(gamma[i].x, s2[i].x, acc[1][UNI ? 0 : 2 * i]);
            acc[1][UNI ? 0 : 2 * i + 1] = fmaf(gamma[i].y, s2[i].y, acc[1][UNI ? 0 : 2 * i + 1]);
        }
        sum_groups<2, VEC, UNI>(acc, p, s.cg, area + buf * kTH * (UNI ? 2 : VEC), sums);
        if (sum1 || sum2) {     // sum_groups had a barrier: the entries are there
            for (int c = (int)threadIdx.x; c < both; c += kTH) {
                float t = 0.f;
                const float *in = entries + buf * lines * both + c;
#pragma unroll 8
                for (int r = 0; r < lines; ++r) t += in[r * both];
                float *out = c < p.width ? sum1 : sum2;
                if (out) out[((int64_t)n * s.cluster + p.rank) * ld_sum + p.slab * s.sc + (c < p.width ? c : c - p.width)] = t;
            }
        }
        if (a.y) {
            if (s.cluster > 1) {
                float *box = peers + (size_t)buf * s.cluster * 2 * gmax;
#pragma unroll
                for (int i = 0; i < kG; ++i)
                    if (p.j == 0 && (p.col * VEC + i) % s.cg == 0) {
                        const int g = (p.col * VEC + i) / s.cg;
                        hand_out(&box[p.rank * 2 * gmax + g], acc[0][i], s.cluster);
                        hand_out(&box[(p.rank * 2 + 1) * gmax + g], acc[1][i], s.cluster);
                    }
                cluster_meet();
#pragma unroll
                for (int i = 0; i < kG; ++i) {
                    const float *in = box + (p.col * VEC + i) / s.cg;
                    float t1 = 0.f, t2 = 0.f;
                    for (int r = 0; r < s.cluster; ++r) {
                        t1 += in[r * 2 * gmax];
                        t2 += in[(r * 2 + 1) * gmax];
                    }
                    acc[0][i] = t1;
                    acc[1][i] = t2;
                }
            }
            // dx = rstd (gamma dz - m1 - xhat m2) = (rstd gamma) dz - rstd^3 M2 (x - mean) - rstd m1,  M2 the mean of gamma dz (x - mean)
#pragma unroll
            for (int i = 0; i < kG; ++i) {
                const float r = rstd[i] * kept;
                acc[0][i] = -r * (acc[0][i] / all);
                acc[1][i] = -r * rstd[i] * rstd[i] * (acc[1][i] / all);
            }
            T *dst = static_cast<T *>(a.y) + (row * a.ld_y + p.c0);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (k < p.mine) {
                    F2 f[NP];
                    unpack2<T, VEC>(held<T>(at_x + k * (kTH * 16)), f);
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const F2 m = pair_of<UNI>(mean, i), centred = add2(f[i], {-m.x, -m.y});
                        f[i] = fma2(mul2(scaled[i], f2(kept)), dz[k][i], fma2(pair_of<UNI>(acc[1], i), centred, pair_of<UNI>(acc[0], i)));
                        if (one) f[i] = f2(0.f);
                    }
                    store_packed<T, VEC>(dst, pack2<T, VEC>(f));
                    dst += step_y;
                }
        }
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            mean[i] = mean_next[i];
            rstd[i] = rstd_next[i];
        }
    }
}

template <int V> struct Int { static constexpr int value = V; };

// The slab and the cluster of an item, and the vectors a thread holds: false where an item does not fit.
bool choose(int elem, int channels, int groups, int64_t samples, int64_t positions, int max_nv, Slab &s, int &nv) {
    const int vec = 16 / elem_bytes(elem);
    if (channels % vec || samples > 0x3fffffff) return false;
    s.cg = channels / groups;
    s.channels = channels;
    s.positions = positions;
    s.samples = (int)samples;
    const int unit = std::lcm(s.cg, vec), wanted = 128 / elem_bytes(elem);
    for (int width = std::min(channels, unit * std::max(1, wanted / unit));; width = std::max(unit, width / 2 / unit * unit)) {
        if (width / vec <= kTH) {
            const int rt = kTH / (width / vec);
            const int64_t deep = (positions + rt - 1) / rt;     // vectors of a column, over the whole item
            int cluster = 1;
            while (cluster < kMaxCluster && deep > (int64_t)max_nv * cluster) cluster *= 2;
            if (deep <= (int64_t)max_nv * cluster) {
                s.sc = width;
                s.slabs = (channels + width - 1) / width;
                s.cluster = cluster;
                s.rows_per_cta = (int)((positions + cluster - 1) / cluster);
                nv = 1;
                while ((int64_t)nv * rt < s.rows_per_cta) nv *= 2;
                return nv <= max_nv;
            }
        }
        if (width == unit) return false;
    }
}

// Clusters that are resident together, asked of the runtime once per kernel and cluster size.
template <typename K>
int resident_clusters(K kernel, int cluster, size_t smem, std::atomic<int> *known) {
    int log = 0;
    while (1 << log < cluster) ++log;
    int r = known[log].load(std::memory_order_relaxed);
    if (r) return r;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)cluster);
    cfg.blockDim = dim3(kTH);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&r, kernel, &cfg) != cudaSuccess || r < 1) {
        (void)cudaGetLastError();
        r = 1;
    }
    known[log].store(r, std::memory_order_relaxed);
    return r;
}

template <typename K, typename... More>
cudaError_t launch(K kernel, std::atomic<int> *known, Slab s, size_t smem, cudaStream_t stream, int64_t *launches, const GroupNormArgs &a, More... more) {
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    // as many clusters as fit, in equal numbers per slab; each walks over every walkers-th sample
    const int64_t rounds = std::max(1, resident_clusters(kernel, s.cluster, smem, known) / s.slabs);
    s.walkers = (int)std::min<int64_t>(s.samples, rounds);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)s.walkers * (unsigned)s.slabs * (unsigned)s.cluster);
    cfg.blockDim = dim3(kTH);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = s.cluster > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, s, more...);
    if (e == cudaSuccess) ++*launches;
    return e;
}

constexpr int kForwardNV = CR_GN_FNV, kBackwardNV = CR_GN_BNV;

template <int Low, int High, typename F>
cudaError_t by_nv(int nv, F &&f) {
    if (nv <= Low) return f(Int<Low>{});
    if constexpr (Low < High) return by_nv<Low * 2, High>(nv, f);
    return cudaErrorInvalidValue;
}

template <typename F>
cudaError_t by_type_act(int elem, int act, F &&f) {
    auto with = [&](auto t) {
        switch (act) {
            case kActNone: return f(t, Int<kActNone>{});
            case kActRelu: return f(t, Int<kActRelu>{});
            default: return f(t, Int<kActSilu>{});
        }
    };
    switch (elem) {
        case kElemF32: return with(float{});
        case kElemBF16: return with(__nv_bfloat16{});
        default: return with(__half{});
    }
}

}  // namespace

bool group_norm_on_chip(int64_t samples, int64_t positions, int channels, int groups, int elem) {
    Slab s;
    int nv;
    return choose(elem, channels, groups, samples, positions, kForwardNV, s, nv);
}
int group_norm_backward_on_chip(int64_t samples, int64_t positions, int channels, int groups, int elem) {
    Slab s;
    int nv;
    return choose(elem, channels, groups, samples, positions, kBackwardNV, s, nv) ? s.cluster : 0;
}

cudaError_t launch_group_norm_on_chip(const GroupNormArgs &a, cudaStream_t stream, int64_t *launches) {
    Slab s;
    int nv;
    if (!choose(a.elem, a.channels, a.groups, a.samples, a.positions, kForwardNV, s, nv)) return cudaErrorInvalidValue;
    return by_type_act(a.elem, a.act, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T), ACT = decltype(act)::value;
        const int gmax = s.sc / s.cg;
        return by_nv<2, kForwardNV>(nv, [&](auto n) {
            constexpr int NV = decltype(n)::value;
            auto go = [&](auto uni) {
                constexpr bool UNI = decltype(uni)::value != 0;
                static std::atomic<int> known[4];
                const size_t smem = (size_t)2 * NV * kTH * 16 + ((size_t)2 * kTH * (UNI ? 1 : VEC) + gmax + (size_t)4 * s.cluster * gmax) * 4;
                return launch(cr_group_norm_kernel<T, NV, UNI, ACT>, known, s, smem, stream, launches, a);
            };
            return s.cg % VEC == 0 ? go(Int<1>{}) : go(Int<0>{});
        });
    });
}

cudaError_t launch_group_norm_grad_on_chip(const GroupNormArgs &a, float *sum1, float *sum2, int64_t ld_sum, cudaStream_t stream, int64_t *launches) {
    Slab s;
    int nv;
    if (!choose(a.elem, a.channels, a.groups, a.samples, a.positions, kBackwardNV, s, nv)) return cudaErrorInvalidValue;
    return by_type_act(a.elem, a.act, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T), ACT = decltype(act)::value;
        const int gmax = s.sc / s.cg;
        const int last = s.channels - (s.slabs - 1) * s.sc;     // a narrow last slab may need what a full one does not
        s.entries = 32 % (s.sc / VEC) == 0 && 32 % (last / VEC) == 0 ? kWarps * 2 * s.sc : kTH * 2 * VEC;
        return by_nv<2, kBackwardNV>(nv, [&](auto n) {
            constexpr int NV = decltype(n)::value;
            auto go = [&](auto uni) {
                constexpr bool UNI = decltype(uni)::value != 0;
                static std::atomic<int> known[4];
                const size_t smem = (size_t)4 * NV * kTH * 16 + ((size_t)2 * kTH * (UNI ? 2 : VEC) + 2 * (size_t)s.entries + gmax + (size_t)4 * s.cluster * gmax) * 4;
                return launch(cr_group_norm_grad_kernel<T, NV, UNI, ACT>, known, s, smem, stream, launches, a, sum1, sum2, ld_sum);
            };
            return s.cg % VEC == 0 ? go(Int<1>{}) : go(Int<0>{});
        });
    });
}

}  // namespace cr
