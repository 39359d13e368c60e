// Group norm with an activation and dropout, channels last, forward and backward; dropout by itself.
//
// For sample n and group g (C / G neighbouring channels, all positions; K = positions * C / G values):
//   mean = sum x / K,  var = sum (x - mean)^2 / K,  rstd = 1 / sqrt(var + eps),  xhat = (x - mean) rstd,
//   z = gamma_c xhat + beta_c,  y = drop(act(z));
//   dz = drop(dy) act'(z),  dbeta_c = sum dz,  dgamma_c = sum dz xhat  (over a partition's samples),
//   dx = rstd (gamma_c dz - m1 - xhat m2),  m1 = sum gamma_c dz / K,  m2 = sum gamma_c dz xhat / K.
// Statistics and sums are held in 32 bits whatever the elements' type; a value is rounded to it once, when it is
// stored.  No atomics: every sum has one order.  The order follows the sizes, the element type and whether all tensors of
// the call lie in 16-byte vectors (which decides between the forms), not the samples beside it, the strides themselves or
// the machine: every worker that holds a partition in such a layout gets the same bits.
//
// z is formed as ((x - mean) * rstd) * gamma + beta: in this file, and for relu everywhere, with each step rounded, in the
// forward and the backward pass alike.  Where the activation has a kink its slope then belongs to the very z that the
// forward pass used.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <numeric>

#include "cr_elem.cuh"

namespace cr {

DropSpec make_drop(double p, uint64_t seed, int64_t offset) {
    DropSpec d;
    d.threshold = (uint32_t)(p * 65536.0 + 0.5);
    d.scale = d.threshold >= 65536u ? 0.f : (float)(65536.0 / (65536.0 - (double)d.threshold));
    d.key = mix64(seed);
    d.offset = (unsigned long long)offset;
    return d;
}

namespace {

constexpr int kThreads = 256;

// Blocks of the streaming kernels that an SM holds, by the registers that a thread's channels take (elements of its
// vector, arrays it reads).
__host__ __device__ constexpr int blocks_per_sm(int vec, int arrays) { return vec < 8 ? 4 : arrays == 1 ? 3 : 2; }

// Which part of the tensor a block of the streaming kernels has: sample, tile of channels, chunk of positions.  A tile
// is a run of whole groups of up to 256 vectors, or one of `parts` pieces of a group that is wider than that.  A thread
// keeps its vector of channels and walks every rt-th row of the chunk.
struct Split {
    int64_t positions, rows_per_chunk;
    int channels, groups, cg, width, tiles, parts, chunks;
};
struct Place {
    int64_t n, row0;
    int rows, chunk, part, c_start, width, vecs, rt, col, j;   // j: this thread's first row of the chunk; -1: no work
    int c0, g0, groups;                                        // its first channel; the tile's groups
};
template <int VEC>
__device__ __forceinline__ Place place(const Split &s) {
    Place p;
    const uint32_t b = blockIdx.x;
    p.chunk = (int)(b % (uint32_t)s.chunks);
    const uint32_t r = b / (uint32_t)s.chunks;
    const int tile = (int)(r % (uint32_t)s.tiles);
    p.n = r / (uint32_t)s.tiles;
    p.row0 = (int64_t)p.chunk * s.rows_per_chunk;
    p.rows = (int)min(s.rows_per_chunk, s.positions - p.row0);
    p.part = tile % s.parts;
    if (s.parts > 1) {
        p.g0 = tile / s.parts;
        p.groups = 1;
        p.c_start = p.g0 * s.cg + p.part * s.width;
        p.width = min(s.width, s.cg - p.part * s.width);
    } else {
        p.c_start = tile * s.width;
        p.width = min(s.width, s.channels - p.c_start);
        p.g0 = p.c_start / s.cg;
        p.groups = p.width / s.cg;
    }
    p.vecs = p.width / VEC;
    p.rt = kThreads / p.vecs;
    p.col = (int)threadIdx.x % p.vecs;
    const int j = (int)threadIdx.x / p.vecs;
    p.j = j < p.rt ? j : -1;
    p.c0 = p.c_start + p.col * VEC;
    return p;
}
// The partial results of (sample, group): one per chunk and piece, next to each other.
__device__ __forceinline__ int64_t entries_of(const Split &s, int64_t n, int g) { return (n * s.groups + g) * s.chunks * s.parts; }

// Sums sm[j * width + c] over j < rt into sm[c], for c < width, both planes; `plane` floats apart.  Up to 16 threads share
// a channel, so that a narrow tile does not leave its sums to a few threads.
__device__ __forceinline__ void fold_rows(float *sm, int plane, int width, int rt) {
    int share = 1;
    while (share < 16 && share * 2 <= rt && share * 2 * width <= kThreads) share *= 2;
    __syncthreads();
    if (share > 1) {
        const int c = (int)threadIdx.x % width, q = (int)threadIdx.x / width;
        if (q < share) {
            float t1 = 0.f, t2 = 0.f;
            for (int j = q; j < rt; j += share) {
                t1 += sm[j * width + c];
                t2 += sm[plane + j * width + c];
            }
            sm[q * width + c] = t1;            // row q is this thread's own
            sm[plane + q * width + c] = t2;
        }
        __syncthreads();
        rt = share;
    }
    for (int c = threadIdx.x; c < width; c += kThreads) {
        float t1 = 0.f, t2 = 0.f;
        for (int j = 0; j < rt; ++j) {
            t1 += sm[j * width + c];
            t2 += sm[plane + j * width + c];
        }
        sm[c] = t1;
        sm[plane + c] = t2;
    }
    __syncthreads();
}
// Vectors that a thread requests before it works on the first of them.  An
// output may be the input's own buffer, so the compiler does not move a load over a store and the batches are made here.
__host__ __device__ constexpr int in_flight(int vec, int arrays) { return (vec == 1 ? 8 : 4) / arrays; }

// f(vector, k) for the thread's k-th row of the chunk, whose first lies at `src`, `step` elements apart.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void walk_one(const Place &p, const T *src, int64_t step, F &&f) {
    constexpr int U = in_flight(VEC, 1);
    const int mine = p.j < p.rows ? (p.rows - p.j + p.rt - 1) / p.rt : 0;
    int k = 0;
    for (; k + U <= mine; k += U, src += U * step) {
        Packed<T, VEC> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_packed<T, VEC>(src + u * step);
#pragma unroll
        for (int u = 0; u < U; ++u) f(raw[u], k + u);
    }
    for (; k < mine; ++k, src += step) f(load_packed<T, VEC>(src), k);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---- forward, streaming: mean and centred square sum of each group over a chunk -------------------------------------
//
// Sums are taken of x - k, k the channel's value in the chunk's first row: the squares then carry the spread and not the
// mean.  Where that value lies more than eight standard deviations off the channel's mean over the chunk (first rows of
// zeros, say), the squares have lost digits to it, or their sum has left the range of a float, and the block walks its
// chunk once more around the means: what is lost otherwise stays below 64 x 2^-24 of the variance, and ordinary data, whose
// values do not lie that far out, are walked once.  Channels, chunks and pieces are joined by mean and centred square sum.
// This form serves what the one-pass form does not take: odd rows, and items beyond a cluster's shared memory, whose
// second read comes from L2 where the tensor fits it.  Two samples of 65536 x 64 f16 (floor 5.2 us): 11 us here and 13 us
// in the apply pass.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(VEC, 1)) cr_group_norm_stats_kernel(const T *x, int64_t ld, const Split s, float2 *partial) {
    __shared__ float sm[2 * kThreads * VEC];
    __shared__ float around[kThreads * VEC];     // the channels' means, where the chunk is walked again
    constexpr int kPlane = kThreads * VEC;
    const Place p = place<VEC>(s);
    const T *first = x + ((p.n * s.positions + p.row0) * ld + p.c0);
    // The sums around k, by channel, in `sm`.
    auto sums_around = [&](const float (&k)[VEC]) {
        float s1[VEC], s2[VEC];
        const T *src = first + p.j * ld;
        const int64_t step = (int64_t)p.rt * ld;
#pragma unroll
        for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
        walk_one<T, VEC>(p, src, step, [&](const Packed<T, VEC> &raw, int) {
            float v[VEC];
            unpack<T, VEC>(raw, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float dlt = v[i] - k[i];
                s1[i] += dlt;
                s2[i] = fmaf(dlt, dlt, s2[i]);
            }
        });
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int at = (p.j * p.vecs + p.col) * VEC + i;
            sm[at] = s1[i];
            sm[kPlane + at] = s2[i];
        }
    };
    if (p.j >= 0) {
        float k[VEC];
        unpack<T, VEC>(load_packed<T, VEC>(first), k);
        sums_around(k);
    }
    fold_rows(sm, kPlane, p.width, p.rt);
    const float rows = (float)p.rows, inv = 1.f / rows;
    bool far = false;
    for (int c = threadIdx.x; c < p.width; c += kThreads) {
        const float t1 = sm[c], t2 = sm[kPlane + c], off = t1 * inv, m2 = not_below_zero(fmaf(-t1, off, t2));
        far = far || m2 * 64.f < t2 || isinf(t2);
        sm[kPlane + c] = m2;
        sm[c] = to_float(x[(p.n * s.positions + p.row0) * ld + p.c_start + c]) + off;
    }
    if (__syncthreads_or(far)) {
        float k[VEC];
        if (p.j >= 0) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) k[i] = sm[p.col * VEC + i];
        }
        for (int c = threadIdx.x; c < p.width; c += kThreads) around[c] = sm[c];
        __syncthreads();
        if (p.j >= 0) sums_around(k);
        fold_rows(sm, kPlane, p.width, p.rt);
        for (int c = threadIdx.x; c < p.width; c += kThreads) {
            const float t1 = sm[c], off = t1 * inv;
            sm[kPlane + c] = not_below_zero(fmaf(-t1, off, sm[kPlane + c]));
            sm[c] = around[c] + off;
        }
        __syncthreads();
    }
    const int lane = threadIdx.x & 31, per = p.width / p.groups;
    for (int g = threadIdx.x >> 5; g < p.groups; g += kThreads / 32) {
        float sum = 0.f, m2 = 0.f;
        for (int c = g * per + lane; c < (g + 1) * per; c += 32) sum += sm[c];
        const float mean = warp_sum(sum) / (float)per;
        for (int c = g * per + lane; c < (g + 1) * per; c += 32) {
            const float d = sm[c] - mean;
            m2 += sm[kPlane + c] + rows * d * d;
        }
        m2 = warp_sum(m2);
        if (lane == 0) partial[entries_of(s, p.n, p.g0 + g) + p.chunk * s.parts + p.part] = make_float2(mean, m2);
    }
}

// What a thread keeps of its channels.
template <int VEC>
struct Affine {
    float mean[VEC], rstd[VEC], gamma[VEC], beta[VEC];
    __device__ __forceinline__ void parameters(const Place &p, const float *gamma_in, const float *beta_in) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            gamma[i] = gamma_in ? __ldg(gamma_in + p.c0 + i) : 1.f;
            beta[i] = beta_in ? __ldg(beta_in + p.c0 + i) : 0.f;
        }
    }
    __device__ __forceinline__ float xhat(float x, int i) const { return __fmul_rn(x - mean[i], rstd[i]); }
    __device__ __forceinline__ float z(float xh, int i) const { return __fadd_rn(__fmul_rn(xh, gamma[i]), beta[i]); }
};

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(VEC, 1)) cr_group_norm_apply_kernel(const GroupNormArgs a, const Split s, const Split own, const float2 *partial) {
    __shared__ float2 ready[kThreads * VEC];     // mean and rstd of the tile's groups
    const Place p = place<VEC>(own);             // `s`: how the partial results were cut
    Affine<VEC> f;
    if (p.j >= 0) f.parameters(p, a.gamma, a.beta);
    // every block joins the chunks of its groups for itself: a warp per group, in one order
    const int lane = threadIdx.x & 31, entries = s.chunks * s.parts;
    const float total = (float)s.positions * (float)s.cg;
    for (int g = threadIdx.x >> 5; g < p.groups; g += kThreads / 32) {
        const float2 *in = partial + entries_of(s, p.n, p.g0 + g);
        auto count = [&](int e) {
            const int chunk = e / s.parts, part = e - chunk * s.parts;
            const float rows = (float)min(s.rows_per_chunk, s.positions - chunk * s.rows_per_chunk);
            return rows * (float)(s.parts > 1 ? min(s.width, s.cg - part * s.width) : s.cg);
        };
        float sum = 0.f, m2 = 0.f;
#pragma unroll 8
        for (int e = lane; e < entries; e += 32) sum = fmaf(count(e), in[e].x, sum);
        const float mean = warp_sum(sum) / total;
#pragma unroll 8
        for (int e = lane; e < entries; e += 32) {
            const float2 v = in[e];
            const float d = v.x - mean;
            m2 += fmaf(count(e) * d, d, v.y);
        }
        m2 = warp_sum(m2);
        if (lane == 0) {
            const float rstd = 1.f / sqrtf(m2 / total + a.eps);
            ready[g] = make_float2(mean, rstd);
            if (a.mean && p.chunk == 0 && p.part == 0) {
                a.mean[p.n * s.groups + p.g0 + g] = mean;
                a.rstd[p.n * s.groups + p.g0 + g] = rstd;
            }
        }
    }
    __syncthreads();
    if (p.j < 0) return;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float2 v = ready[(p.c0 + i) / s.cg - p.g0];
        f.mean[i] = v.x;
        f.rstd[i] = v.y;
    }
    const int64_t first = p.n * s.positions + p.row0 + p.j;
    T *y = static_cast<T *>(a.y) + (first * a.ld_y + p.c0);
    const int64_t step_y = (int64_t)p.rt * a.ld_y;
    unsigned long long e = a.drop.offset + (unsigned long long)(first * s.channels + p.c0);
    walk_one<T, VEC>(p, static_cast<const T *>(a.x) + (first * a.ld_x + p.c0), (int64_t)p.rt * a.ld_x, [&](const Packed<T, VEC> &raw, int) {
        float v[VEC];
        unpack<T, VEC>(raw, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = act_value<ACT>(f.z(f.xhat(v[i], i), i));
        if (a.drop.threshold) {
            drop<VEC>(v, a.drop, e);
            e += (unsigned long long)p.rt * s.channels;
        }
        store_packed<T, VEC>(y, pack<T, VEC>(v));
        y += step_y;
    });
}

// ---- backward, streaming -----------------------------------------------------------------------------------------

template <int VEC>
__device__ __forceinline__ void statistics(Affine<VEC> &f, const Place &p, const Split &s, const GroupNormArgs &a) {
    f.parameters(p, a.gamma, a.beta);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int64_t at = p.n * s.groups + (p.c0 + i) / s.cg;
        f.mean[i] = a.mean[at];
        f.rstd[i] = a.rstd[at];
    }
}

// dz of a vector of elements, and their xhat; `e`: index of the first element.
template <typename T, int VEC, int ACT>
__device__ __forceinline__ void slopes(const GroupNormArgs &a, const Affine<VEC> &f, const Packed<T, VEC> &x, const Packed<T, VEC> &dy, int64_t e,
                                       float (&dz)[VEC], float (&xh)[VEC]) {
    unpack<T, VEC>(x, xh);
    unpack<T, VEC>(dy, dz);
    if (a.drop.threshold) drop<VEC>(dz, a.drop, a.drop.offset + (unsigned long long)e);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        xh[i] = f.xhat(xh[i], i);
        if constexpr (ACT != kActNone) dz[i] = act_gradient<ACT>(dz[i], f.z(xh[i], i));
    }
}

// Walks the thread's rows of the chunk in batches: f(dz, xhat).
template <typename T, int VEC, int ACT, typename F>
__device__ __forceinline__ void walk(const GroupNormArgs &a, const Split &s, const Place &p, const Affine<VEC> &aff, F &&f) {
    const int64_t first = p.n * s.positions + p.row0 + p.j;
    const T *x = static_cast<const T *>(a.x) + (first * a.ld_x + p.c0);
    const T *dy = static_cast<const T *>(a.dy) + (first * a.ld_dy + p.c0);
    const int64_t step_x = (int64_t)p.rt * a.ld_x, step_dy = (int64_t)p.rt * a.ld_dy, step_e = (int64_t)p.rt * s.channels;
    int64_t e = first * s.channels + p.c0;
    constexpr int U = in_flight(VEC, 2);
    const int mine = p.j < p.rows ? (p.rows - p.j + p.rt - 1) / p.rt : 0;
    auto one = [&](const Packed<T, VEC> &raw_x, const Packed<T, VEC> &raw_dy) {
        float dz[VEC], xh[VEC];
        slopes<T, VEC, ACT>(a, aff, raw_x, raw_dy, e, dz, xh);
        e += step_e;
        f(dz, xh);
    };
    int k = 0;
    for (; k + U <= mine; k += U, x += U * step_x, dy += U * step_dy) {
        Packed<T, VEC> raw_x[U], raw_dy[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw_x[u] = load_packed<T, VEC>(x + u * step_x);
            raw_dy[u] = load_packed<T, VEC>(dy + u * step_dy);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) one(raw_x[u], raw_dy[u]);
    }
    for (; k < mine; ++k, x += step_x, dy += step_dy) one(load_packed<T, VEC>(x), load_packed<T, VEC>(dy));
}

// The channels' sums of dz (part1) and dz xhat (part2) over a chunk, [samples][chunks] rows of `channels`, and the
// groups' sums of gamma dz and gamma dz xhat.
template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(VEC, 2)) cr_group_norm_grad_sums_kernel(const GroupNormArgs a, const Split s, float *part1, float *part2, float2 *partial) {
    __shared__ float sm[2 * kThreads * VEC];
    constexpr int kPlane = kThreads * VEC;
    const Place p = place<VEC>(s);
    if (p.j >= 0) {
        Affine<VEC> f;
        statistics<VEC>(f, p, s, a);
        float s1[VEC], s2[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
        walk<T, VEC, ACT>(a, s, p, f, [&](const float (&dz)[VEC], const float (&xh)[VEC]) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                s1[i] += dz[i];
                s2[i] = fmaf(dz[i], xh[i], s2[i]);
            }
        });
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            sm[(p.j * p.vecs + p.col) * VEC + i] = s1[i];
            sm[kPlane + (p.j * p.vecs + p.col) * VEC + i] = s2[i];
        }
    }
    fold_rows(sm, kPlane, p.width, p.rt);
    for (int c = threadIdx.x; c < p.width; c += kThreads) {
        const int64_t at = (p.n * s.chunks + p.chunk) * s.channels + p.c_start + c;
        part1[at] = sm[c];
        part2[at] = sm[kPlane + c];
    }
    const int lane = threadIdx.x & 31, per = p.width / p.groups;
    for (int g = threadIdx.x >> 5; g < p.groups; g += kThreads / 32) {
        float t1 = 0.f, t2 = 0.f;
        for (int c = g * per + lane; c < (g + 1) * per; c += 32) {
            const float w = a.gamma ? __ldg(a.gamma + p.c_start + c) : 1.f;
            t1 = fmaf(w, sm[c], t1);
            t2 = fmaf(w, sm[kPlane + c], t2);
        }
        t1 = warp_sum(t1);
        t2 = warp_sum(t2);
        if (lane == 0) partial[entries_of(s, p.n, p.g0 + g) + p.chunk * s.parts + p.part] = make_float2(t1, t2);
    }
}

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(VEC, 2)) cr_group_norm_grad_apply_kernel(const GroupNormArgs a, const Split s, const Split own, const float2 *partial) {
    __shared__ float2 ready[kThreads * VEC];     // m1 and m2 of the tile's groups
    const Place p = place<VEC>(own);             // `s`: how the partial results were cut
    const int lane = threadIdx.x & 31, entries = s.chunks * s.parts;
    const float total = (float)s.positions * (float)s.cg;
    for (int g = threadIdx.x >> 5; g < p.groups; g += kThreads / 32) {
        float t1 = 0.f, t2 = 0.f;
        const float2 *in = partial + entries_of(s, p.n, p.g0 + g);
#pragma unroll 8
        for (int e = lane; e < entries; e += 32) {
            const float2 v = in[e];
            t1 += v.x;
            t2 += v.y;
        }
        t1 = warp_sum(t1);
        t2 = warp_sum(t2);
        if (lane == 0) ready[g] = make_float2(t1 / total, t2 / total);
    }
    __syncthreads();
    if (p.j < 0) return;
    Affine<VEC> f;
    statistics<VEC>(f, p, s, a);
    float b1[VEC], b2[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float2 v = ready[(p.c0 + i) / s.cg - p.g0];
        b1[i] = v.x;
        b2[i] = v.y;
    }
    const int64_t row = p.n * s.positions + p.row0 + p.j, step_y = (int64_t)p.rt * a.ld_y;
    T *y = static_cast<T *>(a.y) + (row * a.ld_y + p.c0);
    walk<T, VEC, ACT>(a, s, p, f, [&](float (&dz)[VEC], const float (&xh)[VEC]) {
        // gamma dz is rounded before m1 leaves it: a group of one value has m1 = gamma dz and so a gradient of zero
#pragma unroll
        for (int i = 0; i < VEC; ++i) dz[i] = f.rstd[i] * fmaf(-xh[i], b2[i], __fmul_rn(f.gamma[i], dz[i]) - b1[i]);
        store_packed<T, VEC>(y, pack<T, VEC>(dz));
        y += step_y;
    });
}

// Parameter gradients of a partition: the sums over the rows (one or more a sample) of its samples, 32 channels a block, eight threads to a channel.
__global__ void __launch_bounds__(kThreads) cr_group_norm_params_kernel(const float *sum1, const float *sum2, int64_t per, int channels,
                                                                        int64_t ld, float *dbeta, float *dgamma) {
    __shared__ float sm[2][8][32];
    const int lane = threadIdx.x & 31, j = threadIdx.x >> 5;
    const int tiles = (channels + 31) / 32;
    const int c = (int)(blockIdx.x % (unsigned)tiles) * 32 + lane;
    const int64_t part = blockIdx.x / (unsigned)tiles;
    float t1 = 0.f, t2 = 0.f;
    if (c < channels) {
#pragma unroll 4
        for (int64_t k = j; k < per; k += 8) {
            const int64_t at = (part * per + k) * channels + c;
            t1 += sum1[at];
            t2 += sum2[at];
        }
    }
    sm[0][j][lane] = t1;
    sm[1][j][lane] = t2;
    __syncthreads();
    if (j == 0 && c < channels) {
        t1 = t2 = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            t1 += sm[0][k][lane];
            t2 += sm[1][k][lane];
        }
        if (dbeta) dbeta[part * ld + c] = t1;
        if (dgamma) dgamma[part * ld + c] = t2;
    }
}

__global__ void cr_zero_params_kernel(int64_t count, int channels, int64_t ld, float *dbeta, float *dgamma) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= count) return;
    if (dbeta) dbeta[i / channels * ld + i % channels] = 0.f;
    if (dgamma) dgamma[i / channels * ld + i % channels] = 0.f;
}

// ---- dropout ---------------------------------------------------------------------------------------------------------

// Division by an invariant number (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994),
// for 32-bit dividends.
struct Divide {
    uint32_t by, mul, shift;
    explicit Divide(uint32_t d) : by(d), mul(0), shift(0) {
        while (shift < 32 && (1ull << shift) < d) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
        if (shift == 0) return n;
        const uint32_t t = __umulhi(mul, n);
        return (t + ((n - t) >> 1)) >> (shift - 1);
    }
};

// The elements of a row-major [rows][cols] tensor as 16-byte vectors; a thread takes kUnroll of them, a block apart.
// Where the row strides are the width, the caller passes one long row and no division is made.  Bound by memory: 16384 x
// 4096 bf16 with a residual, 403 MB, 57 us (1.09 of the measured copy bandwidth; 61-65 us in a loop); the generator's 8
// instructions an element hide under the loads, of which four vectors (eight with a residual) a thread are under way.
template <typename T, int VEC, typename I>
__global__ void __launch_bounds__(kThreads) cr_dropout_kernel(const T *x, const T *residual, T *y, I nvec, I vecs_per_row, const Divide divide,
                                                              int64_t ld_x, int64_t ld_r, int64_t ld_y, const DropSpec d) {
    constexpr int kUnroll = 4;
    const I v0 = (I)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
    Packed<T, VEC> px[kUnroll], pr[kUnroll];
    int64_t row[kUnroll], col[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const I v = v0 + u * kThreads;
        I r = 0;
        if (vecs_per_row != nvec) r = sizeof(I) == 4 ? (I)divide((uint32_t)v) : v / vecs_per_row;
        row[u] = (int64_t)r;
        col[u] = (int64_t)(v - r * vecs_per_row) * VEC;
        if (v < nvec) {
            px[u] = load_packed<T, VEC>(x + row[u] * ld_x + col[u]);
            if (residual) pr[u] = load_packed<T, VEC>(residual + row[u] * ld_r + col[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const I v = v0 + u * kThreads;
        if (v >= nvec) break;
        float f[VEC];
        unpack<T, VEC>(px[u], f);
        if (d.threshold) drop<VEC>(f, d, d.offset + (unsigned long long)v * VEC);
        if (residual) {
            float g[VEC];
            unpack<T, VEC>(pr[u], g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] += g[i];
        }
        store_packed<T, VEC>(y + row[u] * ld_y + col[u], pack<T, VEC>(f));
    }
}

// Element by element, for rows that no vector fits.  A warp has 128 consecutive elements, the first one's index a multiple
// of four: lane l makes the output of elements 4 l .. 4 l + 3, and every lane fetches its 16 bits from the lane that made
// them, so that neighbouring lanes still read and write neighbouring elements.  8596 rows of 2245 f16 (77 MB): 43 us, bound by
// 2-byte accesses; with a generator output for every element 57 us.
template <typename T, typename I>
__global__ void __launch_bounds__(kThreads) cr_dropout_elements_kernel(const T *x, const T *residual, T *y, I count, I cols, const Divide divide,
                                                                       int64_t ld_x, int64_t ld_r, int64_t ld_y, const DropSpec d) {
    const int lane = threadIdx.x & 31;
    const I ahead = (I)(d.offset & 3);                     // elements of the first four that lie before the tensor
    const I start = ((I)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * 128;    // counted with those
    const unsigned long long w = drop_word(d.key, (d.offset >> 2) + (unsigned long long)(start >> 2) + (unsigned)lane);
    const uint32_t lo = (uint32_t)w, hi = (uint32_t)(w >> 32);
    const bool all_go = d.scale == 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int from = q * 8 + (lane >> 2);
        const uint32_t a = __shfl_sync(0xffffffffu, lo, from), b = __shfl_sync(0xffffffffu, hi, from);
        const uint32_t half = lane & 2 ? b : a, number = lane & 1 ? half >> 16 : half & 0xffffu;
        const I counted = start + (I)(q * 32 + lane);
        if (counted < ahead || counted - ahead >= count) continue;
        const I i = counted - ahead;
        I r = 0;
        if (cols != count) r = sizeof(I) == 4 ? (I)divide((uint32_t)i) : i / cols;
        const int64_t row = (int64_t)r, col = (int64_t)(i - r * cols);
        float v = to_float(x[row * ld_x + col]);
        if (d.threshold) v = all_go || number < d.threshold ? 0.f : v * d.scale;
        if (residual) v += to_float(residual[row * ld_r + col]);
        y[row * ld_y + col] = from_float<T>(v);
    }
}

Split make_split(int64_t positions, int channels, int groups, int vec) {
    Split s;
    s.positions = positions;
    s.channels = channels;
    s.groups = groups;
    s.cg = channels / groups;
    const int most = kThreads * vec, unit = std::lcm(s.cg, vec);
    if (unit <= most) {
        s.parts = 1;
        s.width = std::min(channels, most / unit * unit);
        s.tiles = (channels + s.width - 1) / s.width;
    } else {
        s.parts = (s.cg + most - 1) / most;
        s.width = most;
        s.tiles = groups * s.parts;
    }
    // Chunks of 32 vectors (64 single elements) a thread, at most 148 (this machine's SMs) for a sample.  Neither the number
    // of samples nor the device's own count may enter: the chunks set the order of the sums, and a worker that holds a
    // partition alone, wherever, has to get the bits of the whole batch.  Forward, us, at 16 / 32 / 64 a thread: 8 samples of 65536 x 64 in vectors 72 / 64 / -, 64 samples of
    // 1024 x 256 in odd rows 76 / 59 / 49; two samples of 65536 x 64 spend 9.3 / 10.9 / - on the sums.
    const int64_t least = (vec == 1 ? 64ll : 32ll) * (kThreads / std::min(kThreads, s.width / vec));
    const int64_t chunks = std::min<int64_t>(148, std::max<int64_t>(1, positions / least));
    s.rows_per_chunk = (positions + chunks - 1) / chunks;
    // a block counts its rows in 32 bits, and a float holds the count of a group without rounding far beyond this
    s.rows_per_chunk = std::min<int64_t>(s.rows_per_chunk, 1 << 24);
    s.chunks = (int)((positions + s.rows_per_chunk - 1) / s.rows_per_chunk);
    return s;
}
// The same tiles in chunks for a pass without sums of its own, whose order does not matter: one round of blocks.
Split recut(Split s, int64_t samples, int vec, int arrays) {
    const int64_t least = 4ll * (kThreads / std::min(kThreads, s.width / vec));
    int64_t chunks = std::max<int64_t>(1, 148 * blocks_per_sm(vec, arrays) / std::max<int64_t>(1, samples * s.tiles));
    chunks = std::min(chunks, std::max<int64_t>(1, s.positions / least));
    s.rows_per_chunk = std::min<int64_t>((s.positions + chunks - 1) / chunks, 1 << 24);
    s.chunks = (int)((s.positions + s.rows_per_chunk - 1) / s.rows_per_chunk);
    return s;
}
// Elements of a vector of the streaming kernels: 16 bytes where the rows allow it and no group wider than a tile is cut
// inside a vector.
int split_vec(bool wide, int elem, int channels, int groups) {
    const int vec = 16 / elem_bytes(elem), cg = channels / groups;
    return wide && (cg % vec == 0 || std::lcm(cg, vec) <= kThreads * vec) ? vec : 1;
}

template <typename F>
cudaError_t by_act(int act, F &&f) {
    switch (act) {
        case kActNone: return f(Int<kActNone>{});
        case kActRelu: return f(Int<kActRelu>{});
        default: return f(Int<kActSilu>{});
    }
}

}  // namespace

bool group_norm_vector_rows(const GroupNormArgs &a) {
    return vector_rows(a.elem, a.channels, {a.x, a.dy, a.y}, {a.ld_x, a.dy ? a.ld_dy : 0, a.y ? a.ld_y : 0});
}

size_t group_norm_workspace_bytes(int64_t samples, int64_t positions, int channels, int groups, int elem, bool vectors) {
    if (samples < 1 || (vectors && group_norm_on_chip(samples, positions, channels, groups, elem))) return 0;
    const Split s = make_split(positions, channels, groups, split_vec(vectors, elem, channels, groups));
    return (size_t)s.chunks * groups * s.parts * (size_t)samples * 8;
}

size_t group_norm_backward_workspace_bytes(int64_t samples, int64_t positions, int channels, int groups, int elem, bool vectors) {
    if (samples < 1) return 0;
    if (const int rows = vectors ? group_norm_backward_on_chip(samples, positions, channels, groups, elem) : 0)
        return (size_t)rows * channels * (size_t)samples * 8;
    const Split s = make_split(positions, channels, groups, split_vec(vectors, elem, channels, groups));
    return (size_t)s.chunks * (channels + (size_t)groups * s.parts) * (size_t)samples * 8;
}

cudaError_t launch_group_norm(const GroupNormArgs &a, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (a.samples == 0) return cudaSuccess;
    const bool wide = group_norm_vector_rows(a);
    if (wide && group_norm_on_chip(a.samples, a.positions, a.channels, a.groups, a.elem)) return launch_group_norm_on_chip(a, stream, launches);
    const int vec = split_vec(wide, a.elem, a.channels, a.groups);
    const Split s = make_split(a.positions, a.channels, a.groups, vec);
    float2 *partial = reinterpret_cast<float2 *>(a.workspace);
    const Split own = recut(s, a.samples, vec, 1);
    if (a.samples * s.tiles > 0x7fffffffll / std::max(s.chunks, own.chunks)) return cudaErrorInvalidValue;
    const unsigned blocks = (unsigned)(a.samples * s.tiles * s.chunks), own_blocks = (unsigned)(a.samples * own.tiles * own.chunks);
    auto run = [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        cr_group_norm_stats_kernel<T, VEC><<<blocks, kThreads, 0, stream>>>(static_cast<const T *>(a.x), a.ld_x, s, partial);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        e = by_act(a.act, [&](auto act) {
            cr_group_norm_apply_kernel<T, VEC, decltype(act)::value><<<own_blocks, kThreads, 0, stream>>>(a, s, own, partial);
            return cudaGetLastError();
        });
        if (e == cudaSuccess) *launches += 2;
        return e;
    };
    return by_type(a.elem, [&](auto t) { return vec > 1 ? run(t, Int<16 / (int)sizeof(t)>{}) : run(t, Int<1>{}); });
}

static cudaError_t launch_params(const GroupNormArgs &a, const float *sum1, const float *sum2, int rows_per_sample, cudaStream_t stream,
                                 int64_t *launches) {
    const unsigned tiles = (unsigned)((a.channels + 31) / 32);
    cr_group_norm_params_kernel<<<tiles * (unsigned)a.partitions, kThreads, 0, stream>>>(sum1, sum2, a.samples / a.partitions * rows_per_sample, a.channels,
                                                                                      a.ld_param, a.dbeta, a.dgamma);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t launch_group_norm_backward(const GroupNormArgs &a, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (a.samples == 0) {
        const int64_t count = a.partitions * a.channels;
        if (!(a.dgamma || a.dbeta) || count == 0) return cudaSuccess;
        cr_zero_params_kernel<<<(unsigned)((count + 255) / 256), 256, 0, stream>>>(count, a.channels, a.ld_param, a.dbeta, a.dgamma);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    }
    const bool wide = group_norm_vector_rows(a);
    const bool params = a.dgamma || a.dbeta;
    const size_t plane = (size_t)a.samples * a.channels;
    float *sum1 = a.workspace;
    cudaError_t e;
    if (const int rows = wide ? group_norm_backward_on_chip(a.samples, a.positions, a.channels, a.groups, a.elem) : 0) {
        // a partition of one sample that one CTA holds has its sums where they belong
        if (a.partitions == a.samples && rows == 2) return launch_group_norm_grad_on_chip(a, a.dbeta, a.dgamma, a.ld_param, true, stream, launches);
        float *sum2 = sum1 + plane * rows;
        e = launch_group_norm_grad_on_chip(a, params ? sum1 : nullptr, params ? sum2 : nullptr, a.channels, false, stream, launches);
        if (e != cudaSuccess || !params) return e;
        return launch_params(a, sum1, sum2, rows, stream, launches);
    }
    const int vec = split_vec(wide, a.elem, a.channels, a.groups);
    const Split s = make_split(a.positions, a.channels, a.groups, vec);
    float *sum2 = sum1 + plane * s.chunks;
    float2 *partial = reinterpret_cast<float2 *>(sum2 + plane * s.chunks);
    const Split own = recut(s, a.samples, vec, 2);
    if (a.samples * s.tiles > 0x7fffffffll / std::max(s.chunks, own.chunks)) return cudaErrorInvalidValue;
    const unsigned blocks = (unsigned)(a.samples * s.tiles * s.chunks), own_blocks = (unsigned)(a.samples * own.tiles * own.chunks);
    auto run = [&](auto t, auto v, auto act) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value, ACT = decltype(act)::value;
        cr_group_norm_grad_sums_kernel<T, VEC, ACT><<<blocks, kThreads, 0, stream>>>(a, s, sum1, sum2, partial);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        ++*launches;
        if (a.y) {
            cr_group_norm_grad_apply_kernel<T, VEC, ACT><<<own_blocks, kThreads, 0, stream>>>(a, s, own, partial);
            e = cudaGetLastError();
            if (e != cudaSuccess) return e;
            ++*launches;
        }
        return cudaSuccess;
    };
    e = by_type(a.elem, [&](auto t) {
        return by_act(a.act, [&](auto act) { return vec > 1 ? run(t, Int<16 / (int)sizeof(t)>{}, act) : run(t, Int<1>{}, act); });
    });
    if (e != cudaSuccess || !params) return e;
    return launch_params(a, sum1, sum2, s.chunks, stream, launches);
}

cudaError_t launch_dropout(const void *x, const void *residual, void *y, int64_t rows, int64_t cols, int64_t ld_x,
                           int64_t ld_r, int64_t ld_y, int elem, const DropSpec &drop, const DeviceInfo &,
                           cudaStream_t stream, int64_t *launches) {
    if (rows == 0 || cols == 0) return cudaSuccess;
    if (!residual) ld_r = ld_x;
    if (rows == 1 || (ld_x == cols && ld_r == cols && ld_y == cols)) {   // one long row
        cols *= rows;
        rows = 1;
        ld_x = ld_r = ld_y = cols;
    }
    return by_type(elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const T *px = static_cast<const T *>(x), *pr = static_cast<const T *>(residual);
        T *py = static_cast<T *>(y);
        const bool one = rows == 1;   // a long row's stride does not count
        const bool vectors = vector_rows(elem, cols, {x, residual, y}, {one ? 0 : ld_x, one ? 0 : ld_r, one ? 0 : ld_y});
        const int64_t units = vectors ? rows * (cols / VEC) : rows * cols, per_row = vectors ? cols / VEC : cols;
        const int64_t blocks = (units + 3 + kThreads * 4 - 1) / (kThreads * 4);    // + 3: elements counted before the first
        if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
        const Divide divide((uint32_t)std::min<int64_t>(per_row, 0x7fffffff));
        auto go = [&](auto i) {
            using I = decltype(i);
            if (vectors)
                cr_dropout_kernel<T, VEC, I><<<(unsigned)blocks, kThreads, 0, stream>>>(px, pr, py, (I)units, (I)per_row, divide, ld_x, ld_r, ld_y, drop);
            else
                cr_dropout_elements_kernel<T, I><<<(unsigned)blocks, kThreads, 0, stream>>>(px, pr, py, (I)units, (I)per_row, divide, ld_x, ld_r, ld_y, drop);
        };
        if (units < (1ll << 31) - 8192) go(uint32_t{});
        else go(uint64_t{});
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

}  // namespace cr
