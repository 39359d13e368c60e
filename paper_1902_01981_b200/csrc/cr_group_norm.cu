// Group norm in one pass: a sample's slab of channels stays on chip between its statistics and its output.
//
// The work item is (sample, slab), a slab being neighbouring whole groups, 128 bytes of channels wide where the groups
// allow it, over all positions.  A cluster of K CTAs holds it in registers, each CTA an equal share of the positions,
// each thread up to NV vectors of 16 bytes of one column: x is read once and y written once, which is the floor of the
// operation.  What a CTA knows of its groups (mean and centred square sum; in the backward pass the channels' sums) goes
// to the others through distributed shared memory, in an order fixed by the ranks.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <numeric>

#include "cr_elem.cuh"
#include "cr_tcgen05.cuh"

namespace cr {
namespace {

struct Slab {
    int sc;              // channels of a slab (the last one of a row may have fewer)
    int slabs;           // slabs per row of channels
    int cluster;         // CTAs per item
    int rows_per_cta;
    int cg;
    int channels;
    int64_t positions;
};

// Where a thread stands in its item.
struct Spot {
    int64_t n;
    int slab, rank, rows, width, vpr, rt, col, j, c0;   // j < 0: idle
    int64_t row0;                                       // first row of the CTA, counted over the whole tensor
};
template <int VEC, int TH>
__device__ __forceinline__ Spot spot(const Slab &s) {
    Spot p;
    const uint32_t item = blockIdx.x / (uint32_t)s.cluster;
    p.rank = (int)(blockIdx.x % (uint32_t)s.cluster);
    p.n = item / (uint32_t)s.slabs;
    p.slab = (int)(item % (uint32_t)s.slabs);
    const int64_t first = (int64_t)p.rank * s.rows_per_cta;
    p.rows = (int)max((int64_t)0, min((int64_t)s.rows_per_cta, s.positions - first));
    p.row0 = p.n * s.positions + first;
    p.width = min(s.sc, s.channels - p.slab * s.sc);
    p.vpr = p.width / VEC;
    p.rt = TH / p.vpr;
    p.col = (int)threadIdx.x % p.vpr;
    const int j = (int)threadIdx.x / p.vpr;
    p.j = j < p.rt ? j : -1;
    p.c0 = p.slab * s.sc + p.col * VEC;
    return p;
}

// Sums the entries [g * per, (g + 1) * per) of `in` into out[g] for g < count: a warp per group, in one order.
template <int TH>
__device__ __forceinline__ void fold(const float *in, float *out, int count, int per) {
    const int lane = (int)threadIdx.x & 31;
    for (int g = (int)threadIdx.x >> 5; g < count; g += TH / 32) {
        float t = 0.f;
        for (int e = lane; e < per; e += 32) t += in[g * per + e];
#pragma unroll
        for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) out[g] = t;
    }
}

__device__ __forceinline__ float peer_float(const float *mine, int rank) {
    return __int_as_float(i8::load_cluster(i8::map_to_rank(i8::smem_u32(mine), (uint32_t)rank)));
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// z of the activation.  Where the activation has a kink (relu) every step is rounded by itself, in the forward and the
// backward pass alike, so that the slope belongs to the z whose value was stored.
template <int ACT>
__device__ __forceinline__ float z_of(float centred, float rstd, float gamma, float beta) {
    if constexpr (ACT == kActRelu) return __fadd_rn(__fmul_rn(__fmul_rn(centred, rstd), gamma), beta);
    return fmaf(centred, rstd * gamma, beta);
}

// UNI: every vector lies inside one group.
template <typename T, int NV, int TH, bool UNI, int ACT>
__global__ void __launch_bounds__(TH) cr_group_norm_kernel(const GroupNormArgs a, const Slab s) {
    constexpr int VEC = 16 / (int)sizeof(T), kG = UNI ? 1 : VEC;   // kG: groups a thread may touch
    extern __shared__ float sm[];
    const Spot p = spot<VEC, TH>(s);
    const int groups = p.width / s.cg, per = (UNI ? s.cg / VEC : s.cg) * p.rt;
    float *entries = sm;                       // [TH * kG]: partial sums, group by group
    float *sums = sm + TH * kG;                // [3][groups of a slab]: sum or mean, centred squares, final rstd
    const int gmax = s.sc / s.cg;
    Packed<T, VEC> v[NV];
    const T *src = static_cast<const T *>(a.x) + ((p.row0 + max(p.j, 0)) * a.ld_x + p.c0);
    const int mine = p.j < 0 || p.j >= p.rows ? 0 : (p.rows - p.j + p.rt - 1) / p.rt;   // rows of this thread
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k < mine) v[k] = load_packed<T, VEC>(src + (int64_t)k * p.rt * a.ld_x);
    // sums, then distances from the CTA's own mean
    float acc[kG], mean[kG];
#pragma unroll
    for (int i = 0; i < kG; ++i) acc[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k < mine) {
            float f[VEC];
            unpack<T, VEC>(v[k], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[UNI ? 0 : i] += f[i];
        }
    auto put = [&]() {
        if (p.j >= 0) {
#pragma unroll
            for (int i = 0; i < kG; ++i) entries[(p.col * kG + i) * p.rt + p.j] = acc[i];
        }
        __syncthreads();
    };
    put();
    fold<TH>(entries, sums, groups, per);
    __syncthreads();
    const float inv = 1.f / fmaxf((float)p.rows * (float)s.cg, 1.f);
#pragma unroll
    for (int i = 0; i < kG; ++i) {
        mean[i] = sums[(p.col * VEC + i) / s.cg] * inv;
        acc[i] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k < mine) {
            float f[VEC];
            unpack<T, VEC>(v[k], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = f[i] - mean[UNI ? 0 : i];
                acc[UNI ? 0 : i] = fmaf(d, d, acc[UNI ? 0 : i]);
            }
        }
    put();
    fold<TH>(entries, sums + gmax, groups, per);
    float gamma[VEC], beta[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        gamma[i] = a.gamma ? __ldg(a.gamma + p.c0 + i) : 1.f;
        beta[i] = a.beta ? __ldg(a.beta + p.c0 + i) : 0.f;
    }
    __syncthreads();
    if (s.cluster > 1) {
        cluster_arrive();
        cluster_wait();
    }
    // join the CTAs: means weighted by their rows, centred squares moved to the common mean
    float final_mean = 0.f, final_rstd = 0.f;
    const int g = (int)threadIdx.x;
    if (g < groups) {
        float total = 0.f, m2 = 0.f;
        for (int r = 0; r < s.cluster; ++r) total += s.cluster > 1 ? peer_float(&sums[g], r) : sums[g];
        const float all = (float)s.positions * (float)s.cg;
        final_mean = total / all;
        for (int r = 0; r < s.cluster; ++r) {
            const float rows = (float)max((int64_t)0, min((int64_t)s.rows_per_cta, s.positions - (int64_t)r * s.rows_per_cta));
            const float count = rows * (float)s.cg;
            const float d = count > 0.f ? (s.cluster > 1 ? peer_float(&sums[g], r) : sums[g]) * (1.f / count) - final_mean : 0.f;
            m2 += (s.cluster > 1 ? peer_float(&sums[gmax + g], r) : sums[gmax + g]) + count * d * d;
        }
        final_rstd = 1.f / sqrtf(m2 / all + a.eps);
        if (p.rank == 0 && a.mean) {
            const int64_t at = p.n * a.groups + p.slab * gmax + g;
            a.mean[at] = final_mean;
            a.rstd[at] = final_rstd;
        }
    }
    if (s.cluster > 1) cluster_arrive();    // this CTA has read its peers; they may leave once all have
    float *ready = sums + 2 * gmax;         // [2][groups]
    if (g < groups) {
        ready[g] = final_mean;
        ready[gmax + g] = final_rstd;
    }
    __syncthreads();
    float rstd[kG];
#pragma unroll
    for (int i = 0; i < kG; ++i) {
        mean[i] = ready[(p.col * VEC + i) / s.cg];
        rstd[i] = ready[gmax + (p.col * VEC + i) / s.cg];
    }
    const int64_t row = p.row0 + max(p.j, 0);
    T *dst = static_cast<T *>(a.y) + (row * a.ld_y + p.c0);
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k < mine) {
            float f[VEC];
            unpack<T, VEC>(v[k], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = act_value<ACT>(z_of<ACT>(f[i] - mean[UNI ? 0 : i], rstd[UNI ? 0 : i], gamma[i], beta[i]));
            if (a.drop.threshold) drop<VEC>(f, a.drop, a.drop.offset + (unsigned long long)((row + (int64_t)k * p.rt) * s.channels + p.c0));
            store_packed<T, VEC>(dst + (int64_t)k * p.rt * a.ld_y, pack<T, VEC>(f));
        }
    if (s.cluster > 1) cluster_wait();
}

// Backward: x and dy are read once; dz takes the place of dy in registers.  per_sample: where the sums of each sample's
// channels go (dbeta, dgamma), [samples][channels] unless every partition is one sample.
template <typename T, int NV, int TH, bool UNI, int ACT>
__global__ void __launch_bounds__(TH) cr_group_norm_grad_kernel(const GroupNormArgs a, const Slab s, float *sum1, float *sum2, int64_t ld_sum) {
    constexpr int VEC = 16 / (int)sizeof(T), kG = UNI ? 1 : VEC;
    extern __shared__ float sm[];
    const Spot p = spot<VEC, TH>(s);
    float *entries = sm;                               // [TH * VEC]
    float *chan = sm + TH * VEC;                       // [2][sc]: this CTA's sums of dz and dz (x - mean) rstd
    float *whole = chan + 2 * s.sc;                    // [2][sc]: the item's
    float *coef = whole + 2 * s.sc;                    // [2][groups]
    const int gmax = s.sc / s.cg, groups = p.width / s.cg;
    const int64_t row = p.row0 + max(p.j, 0);
    const int mine = p.j < 0 || p.j >= p.rows ? 0 : (p.rows - p.j + p.rt - 1) / p.rt;
    Packed<T, VEC> v[NV], w[NV];
    const T *src = static_cast<const T *>(a.x) + (row * a.ld_x + p.c0);
    const T *up = static_cast<const T *>(a.dy) + (row * a.ld_dy + p.c0);
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k < mine) {
            v[k] = load_packed<T, VEC>(src + (int64_t)k * p.rt * a.ld_x);
            w[k] = load_packed<T, VEC>(up + (int64_t)k * p.rt * a.ld_dy);
        }
    float mean[kG], rstd[kG], gamma[VEC], beta[VEC];
#pragma unroll
    for (int i = 0; i < kG; ++i) {
        const int64_t at = p.n * a.groups + (p.c0 + i) / s.cg;
        mean[i] = a.mean[at];
        rstd[i] = a.rstd[at];
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        gamma[i] = a.gamma ? __ldg(a.gamma + p.c0 + i) : 1.f;
        beta[i] = a.beta ? __ldg(a.beta + p.c0 + i) : 0.f;
    }
    float dz[NV][VEC], s1[VEC], s2[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k < mine) {
            float f[VEC];
            unpack<T, VEC>(v[k], f);
            unpack<T, VEC>(w[k], dz[k]);
            if (a.drop.threshold) drop<VEC>(dz[k], a.drop, a.drop.offset + (unsigned long long)((row + (int64_t)k * p.rt) * s.channels + p.c0));
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float centred = f[i] - mean[UNI ? 0 : i];
                if constexpr (ACT != kActNone) dz[k][i] *= act_slope<ACT>(z_of<ACT>(centred, rstd[UNI ? 0 : i], gamma[i], beta[i]));
                s1[i] += dz[k][i];
                s2[i] = fmaf(dz[k][i], centred, s2[i]);
            }
        }
    // channel sums over the CTA's rows, one array after the other through the same memory
    auto put = [&](const float (&t)[VEC], bool scaled, float *out) {
        if (p.j >= 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) entries[(p.col * VEC + i) * p.rt + p.j] = scaled ? t[i] * rstd[UNI ? 0 : i] : t[i];
        }
        __syncthreads();
        fold<TH>(entries, out, p.width, p.rt);
        __syncthreads();
    };
    put(s1, false, chan);
    put(s2, true, chan + s.sc);
    if (s.cluster > 1) {
        cluster_arrive();
        cluster_wait();
    }
    for (int e = (int)threadIdx.x; e < 2 * p.width; e += TH) {
        const int c = e < p.width ? e : e - p.width + s.sc;
        float t = 0.f;
        for (int r = 0; r < s.cluster; ++r) t += s.cluster > 1 ? peer_float(&chan[c], r) : chan[c];
        whole[c] = t;
        float *out = e < p.width ? sum1 : sum2;
        if (p.rank == 0 && out) out[p.n * ld_sum + p.slab * s.sc + (e < p.width ? e : e - p.width)] = t;
    }
    if (s.cluster > 1) cluster_arrive();
    if (a.y) {
        __syncthreads();
        const int lane = (int)threadIdx.x & 31;
        const float all = (float)s.positions * (float)s.cg;
        for (int g = (int)threadIdx.x >> 5; g < groups; g += TH / 32) {
            float t1 = 0.f, t2 = 0.f;
            for (int c = g * s.cg + lane; c < (g + 1) * s.cg; c += 32) {
                const float wgt = a.gamma ? __ldg(a.gamma + p.slab * s.sc + c) : 1.f;
                t1 = fmaf(wgt, whole[c], t1);
                t2 = fmaf(wgt, whole[s.sc + c], t2);
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                t1 += __shfl_xor_sync(0xffffffffu, t1, o);
                t2 += __shfl_xor_sync(0xffffffffu, t2, o);
            }
            if (lane == 0) {
                coef[g] = t1 / all;
                coef[gmax + g] = t2 / all;
            }
        }
        __syncthreads();
        // dx = rstd (gamma dz - m1 - xhat m2); a group of one value has m1 = gamma dz and no gradient at all
        const bool one = s.positions * s.cg == 1;
        float b1[kG], b2[kG];
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            const int at = (p.col * VEC + i) / s.cg;
            b1[i] = -rstd[i] * coef[at];
            b2[i] = -rstd[i] * rstd[i] * coef[gmax + at];
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) gamma[i] *= rstd[UNI ? 0 : i];
        T *dst = static_cast<T *>(a.y) + (row * a.ld_y + p.c0);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < mine) {
                float f[VEC];
                unpack<T, VEC>(v[k], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    f[i] = fmaf(gamma[i], dz[k][i], fmaf(b2[UNI ? 0 : i], f[i] - mean[UNI ? 0 : i], b1[UNI ? 0 : i]));
                    if (one) f[i] = 0.f;
                }
                store_packed<T, VEC>(dst + (int64_t)k * p.rt * a.ld_y, pack<T, VEC>(f));
            }
    }
    if (s.cluster > 1) cluster_wait();
}

template <int V> struct Int { static constexpr int value = V; };

constexpr int kTH = 256;
constexpr int kMaxCluster = 8;

// The slab and the cluster of an item, and the vectors a thread holds: false where an item does not fit.
bool choose(int elem, int channels, int groups, int64_t positions, int max_nv, Slab &s, int &nv) {
    const int vec = 16 / elem_bytes(elem);
    if (channels % vec) return false;
    s.cg = channels / groups;
    s.channels = channels;
    s.positions = positions;
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

template <typename K>
cudaError_t launch(K kernel, const Slab &s, int64_t samples, size_t smem, cudaStream_t stream, int64_t *launches, const GroupNormArgs &a,
                   float *sum1, float *sum2, int64_t ld_sum) {
    (void)sum1; (void)sum2; (void)ld_sum;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(samples * s.slabs * s.cluster));
    cfg.blockDim = dim3(kTH);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = s.cluster > 1 ? 1 : 0;
    cudaError_t e;
    if constexpr (std::is_invocable_v<K, const GroupNormArgs, const Slab>) e = cudaLaunchKernelEx(&cfg, kernel, a, s);
    else e = cudaLaunchKernelEx(&cfg, kernel, a, s, sum1, sum2, ld_sum);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

constexpr int kForwardNV = 16, kBackwardNV = 8;

bool group_norm_on_chip(const GroupNormArgs &a) {
    Slab s;
    int nv;
    return choose(a.elem, a.channels, a.groups, a.positions, kForwardNV, s, nv) && a.samples * s.slabs * s.cluster <= 0x7fffffffll;
}
bool group_norm_backward_on_chip(const GroupNormArgs &a) {
    Slab s;
    int nv;
    return choose(a.elem, a.channels, a.groups, a.positions, kBackwardNV, s, nv) && a.samples * s.slabs * s.cluster <= 0x7fffffffll;
}

template <int Low, typename F>
static cudaError_t by_nv(int nv, F &&f) {
    if (nv <= Low) return f(Int<Low>{});
    if constexpr (Low < 16) return by_nv<Low * 2>(nv, f);
    return cudaErrorInvalidValue;
}

template <typename F>
static cudaError_t by_type_act(int elem, int act, F &&f) {
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

cudaError_t launch_group_norm_on_chip(const GroupNormArgs &a, cudaStream_t stream, int64_t *launches) {
    Slab s;
    int nv;
    if (!choose(a.elem, a.channels, a.groups, a.positions, kForwardNV, s, nv)) return cudaErrorInvalidValue;
    return by_type_act(a.elem, a.act, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T), ACT = decltype(act)::value;
        const bool uni = s.cg % VEC == 0;
        const size_t smem = ((size_t)kTH * (uni ? 1 : VEC) + 4 * (size_t)(s.sc / s.cg)) * 4;
        return by_nv<2>(nv, [&](auto n) {
            constexpr int NV = decltype(n)::value;
            return uni ? launch(cr_group_norm_kernel<T, NV, kTH, true, ACT>, s, a.samples, smem, stream, launches, a, nullptr, nullptr, 0)
                       : launch(cr_group_norm_kernel<T, NV, kTH, false, ACT>, s, a.samples, smem, stream, launches, a, nullptr, nullptr, 0);
        });
    });
}

cudaError_t launch_group_norm_grad_on_chip(const GroupNormArgs &a, float *sum1, float *sum2, int64_t ld_sum, cudaStream_t stream, int64_t *launches) {
    Slab s;
    int nv;
    if (!choose(a.elem, a.channels, a.groups, a.positions, kBackwardNV, s, nv)) return cudaErrorInvalidValue;
    return by_type_act(a.elem, a.act, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T), ACT = decltype(act)::value;
        const bool uni = s.cg % VEC == 0;
        const size_t smem = ((size_t)kTH * VEC + 4 * (size_t)s.sc + 2 * (size_t)(s.sc / s.cg)) * 4;
        return by_nv<2>(nv, [&](auto n) {
            constexpr int NV = decltype(n)::value;
            if constexpr (NV > kBackwardNV) return cudaErrorInvalidValue;
            else
                return uni ? launch(cr_group_norm_grad_kernel<T, NV, kTH, true, ACT>, s, a.samples, smem, stream, launches, a, sum1, sum2, ld_sum)
                           : launch(cr_group_norm_grad_kernel<T, NV, kTH, false, ACT>, s, a.samples, smem, stream, launches, a, sum1, sum2, ld_sum);
        });
    });
}

}  // namespace cr
