// Group norm with an activation and dropout, channels last, forward and backward; dropout by itself.
//
// For sample n and group g (C / G neighbouring channels, all positions; K = positions * C / G values):
//   mean = sum x / K,  var = sum (x - mean)^2 / K,  rstd = 1 / sqrt(var + eps),  xhat = (x - mean) rstd,
//   z = gamma_c xhat + beta_c,  y = drop(act(z));
//   dz = drop(dy) act'(z),  dbeta_c = sum dz,  dgamma_c = sum dz xhat  (over a partition's samples),
//   dx = rstd (gamma_c dz - m1 - xhat m2),  m1 = sum gamma_c dz / K,  m2 = sum gamma_c dz xhat / K.
// Statistics and sums are held in 32 bits whatever the elements' type; a value is rounded to it once, when it is
// stored.  No atomics: every sum has one order, so every worker that holds a partition gets the same bits.
//
// z is formed as ((x - mean) * rstd) * gamma + beta with each step rounded, in the forward and the backward pass
// alike: where the activation has a kink its slope then belongs to the very z that the forward pass used.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

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

// Which part of the tensor a block of the streaming kernels has: sample, tile of up to 256 vectors of channels,
// chunk of positions.  A thread keeps its vector of channels and walks every rt-th row of the chunk.
struct Split {
    int64_t positions;
    int channels, cg, nvec, tiles, chunks;
    int64_t rows_per_chunk;
};
struct Place {
    int64_t n, row0;
    int rows, tile, chunk, vecs, rt, col, j;   // j: this thread's first row of the chunk; -1: no work
    int c0;                                    // its first channel
};
template <int VEC>
__device__ __forceinline__ Place place(const Split &s) {
    Place p;
    const uint32_t b = blockIdx.x;
    p.chunk = (int)(b % (uint32_t)s.chunks);
    const uint32_t r = b / (uint32_t)s.chunks;
    p.tile = (int)(r % (uint32_t)s.tiles);
    p.n = r / (uint32_t)s.tiles;
    p.row0 = (int64_t)p.chunk * s.rows_per_chunk;
    p.rows = (int)min(s.rows_per_chunk, s.positions - p.row0);
    p.vecs = min(kThreads, s.nvec - p.tile * kThreads);
    p.rt = kThreads / p.vecs;
    p.col = (int)threadIdx.x % p.vecs;
    const int j = (int)threadIdx.x / p.vecs;
    p.j = j < p.rt ? j : -1;
    p.c0 = (p.tile * kThreads + p.col) * VEC;
    return p;
}
__device__ __forceinline__ int rows_of(const Place &p, int j) { return j < p.rows ? (p.rows - j + p.rt - 1) / p.rt : 0; }

// ---- forward, streaming: statistics of each channel over a chunk ----------------------------------------------
//
// Sums are taken of x - k, k the thread's first value of the channel: the squares then carry the spread and not the
// mean.  Threads and chunks are joined by mean and centred square sum.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) cr_group_norm_stats_kernel(const T *x, int64_t ld, const Split s, float *part_mean, float *part_m2) {
    __shared__ float sm[2][kThreads * VEC];
    const Place p = place<VEC>(s);
    if (p.j >= 0) {
        float k[VEC], s1[VEC], s2[VEC];
        const int cnt = rows_of(p, p.j);
        const T *src = x + ((p.n * s.positions + p.row0 + p.j) * ld + p.c0);
        const int64_t step = (int64_t)p.rt * ld;
        if (cnt > 0) unpack<T, VEC>(load_packed<T, VEC>(src), k);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
#pragma unroll 4
        for (int r = 1; r < cnt; ++r) {
            float v[VEC];
            unpack<T, VEC>(load_packed<T, VEC>(src + r * step), v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float dlt = v[i] - k[i];
                s1[i] += dlt;
                s2[i] = fmaf(dlt, dlt, s2[i]);
            }
        }
        const float inv = cnt > 0 ? 1.f / (float)cnt : 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int at = (p.j * p.vecs + p.col) * VEC + i;
            sm[0][at] = cnt > 0 ? fmaf(s1[i], inv, k[i]) : 0.f;
            sm[1][at] = cnt > 0 ? fmaxf(s2[i] - s1[i] * s1[i] * inv, 0.f) : 0.f;
        }
    }
    __syncthreads();
    const int width = p.vecs * VEC;
    for (int c = threadIdx.x; c < width; c += kThreads) {
        float sum = 0.f;
        for (int j = 0; j < p.rt; ++j) sum += (float)rows_of(p, j) * sm[0][j * width + c];
        const float mean = sum / (float)p.rows;
        float m2 = 0.f;
        for (int j = 0; j < p.rt; ++j) {
            const float dlt = sm[0][j * width + c] - mean;
            m2 += sm[1][j * width + c] + (float)rows_of(p, j) * dlt * dlt;
        }
        const int64_t at = (p.n * s.chunks + p.chunk) * s.channels + p.tile * kThreads * VEC + c;
        part_mean[at] = mean;
        part_m2[at] = m2;
    }
}

__device__ __forceinline__ float block_sum_128(float v, float *sm) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    return (sm[0] + sm[1]) + (sm[2] + sm[3]);
}

// One block of 128 threads per (sample, group) joins the chunks' statistics.
__global__ void __launch_bounds__(128) cr_group_norm_join_kernel(const float *part_mean, const float *part_m2, const Split s, int groups,
                                                                 float eps, float *mean_out, float *rstd_out) {
    __shared__ float sm[4];
    const int64_t n = blockIdx.x / (unsigned)groups;
    const int g = (int)(blockIdx.x % (unsigned)groups);
    const int64_t base = n * s.chunks * (int64_t)s.channels + (int64_t)g * s.cg;
    const int entries = s.chunks * s.cg;
    float sum = 0.f;
    for (int e = threadIdx.x; e < entries; e += 128) {
        const int k = e / s.cg;
        const float rows = (float)min(s.rows_per_chunk, s.positions - k * s.rows_per_chunk);
        sum = fmaf(rows, part_mean[base + (int64_t)k * s.channels + e % s.cg], sum);
    }
    const float total = (float)s.positions * (float)s.cg;
    const float mean = block_sum_128(sum, sm) / total;
    float m2 = 0.f;
    for (int e = threadIdx.x; e < entries; e += 128) {
        const int k = e / s.cg;
        const float rows = (float)min(s.rows_per_chunk, s.positions - k * s.rows_per_chunk);
        const int64_t at = base + (int64_t)k * s.channels + e % s.cg;
        const float dlt = part_mean[at] - mean;
        m2 += part_m2[at] + rows * dlt * dlt;
    }
    m2 = block_sum_128(m2, sm);
    if (threadIdx.x == 0) {
        mean_out[blockIdx.x] = mean;
        rstd_out[blockIdx.x] = 1.f / sqrtf(m2 / total + eps);
    }
}

// What a thread keeps of its channels.
template <int VEC>
struct Affine {
    float mean[VEC], rstd[VEC], gamma[VEC], beta[VEC];
    __device__ __forceinline__ void load(const Place &p, const Split &s, int groups, const float *mean_in, const float *rstd_in,
                                         const float *gamma_in, const float *beta_in) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = p.c0 + i;
            const int64_t at = p.n * groups + c / s.cg;
            mean[i] = mean_in[at];
            rstd[i] = rstd_in[at];
            gamma[i] = gamma_in ? __ldg(gamma_in + c) : 1.f;
            beta[i] = beta_in ? __ldg(beta_in + c) : 0.f;
        }
    }
    __device__ __forceinline__ float xhat(float x, int i) const { return __fmul_rn(x - mean[i], rstd[i]); }
    __device__ __forceinline__ float z(float xh, int i) const { return __fadd_rn(__fmul_rn(xh, gamma[i]), beta[i]); }
};

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads) cr_group_norm_apply_kernel(const GroupNormArgs a, const Split s) {
    const Place p = place<VEC>(s);
    if (p.j < 0) return;
    Affine<VEC> f;
    f.load(p, s, a.groups, a.mean, a.rstd, a.gamma, a.beta);
    const int64_t first = p.n * s.positions + p.row0;
#pragma unroll 2
    for (int r = p.j; r < p.rows; r += p.rt) {
        float v[VEC];
        unpack<T, VEC>(load_packed<T, VEC>(static_cast<const T *>(a.x) + ((first + r) * a.ld_x + p.c0)), v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = act_value<ACT>(f.z(f.xhat(v[i], i), i));
        if (a.drop.threshold) drop<VEC>(v, a.drop, a.drop.offset + (unsigned long long)((first + r) * s.channels + p.c0));
        store_packed<T, VEC>(static_cast<T *>(a.y) + ((first + r) * a.ld_y + p.c0), pack<T, VEC>(v));
    }
}

// ---- backward, streaming -----------------------------------------------------------------------------------------

// dz of a vector of elements, and their xhat.
template <typename T, int VEC, int ACT>
__device__ __forceinline__ void slopes(const GroupNormArgs &a, const Affine<VEC> &f, int64_t row, int c0, int channels,
                                       float (&dz)[VEC], float (&xh)[VEC]) {
    unpack<T, VEC>(load_packed<T, VEC>(static_cast<const T *>(a.x) + (row * a.ld_x + c0)), xh);
    unpack<T, VEC>(load_packed<T, VEC>(static_cast<const T *>(a.dy) + (row * a.ld_dy + c0)), dz);
    if (a.drop.threshold) drop<VEC>(dz, a.drop, a.drop.offset + (unsigned long long)(row * channels + c0));
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        xh[i] = f.xhat(xh[i], i);
        if constexpr (ACT != kActNone) dz[i] *= act_slope<ACT>(f.z(xh[i], i));
    }
}

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads) cr_group_norm_grad_sums_kernel(const GroupNormArgs a, const Split s, float *part1, float *part2) {
    __shared__ float sm[2][kThreads * VEC];
    const Place p = place<VEC>(s);
    if (p.j >= 0) {
        Affine<VEC> f;
        f.load(p, s, a.groups, a.mean, a.rstd, a.gamma, a.beta);
        float s1[VEC], s2[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) s1[i] = s2[i] = 0.f;
        const int64_t first = p.n * s.positions + p.row0;
#pragma unroll 2
        for (int r = p.j; r < p.rows; r += p.rt) {
            float dz[VEC], xh[VEC];
            slopes<T, VEC, ACT>(a, f, first + r, p.c0, s.channels, dz, xh);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                s1[i] += dz[i];
                s2[i] = fmaf(dz[i], xh[i], s2[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            sm[0][(p.j * p.vecs + p.col) * VEC + i] = s1[i];
            sm[1][(p.j * p.vecs + p.col) * VEC + i] = s2[i];
        }
    }
    __syncthreads();
    const int width = p.vecs * VEC;
    for (int c = threadIdx.x; c < width; c += kThreads) {
        float t1 = 0.f, t2 = 0.f;
        for (int j = 0; j < p.rt; ++j) {
            t1 += sm[0][j * width + c];
            t2 += sm[1][j * width + c];
        }
        const int64_t at = (p.n * s.chunks + p.chunk) * s.channels + p.tile * kThreads * VEC + c;
        part1[at] = t1;
        part2[at] = t2;
    }
}

// One block per sample: the channels' sums over the chunks, then m1 and m2 of its groups.
__global__ void __launch_bounds__(kThreads) cr_group_norm_grad_join_kernel(const float *part1, const float *part2, const Split s, int groups,
                                                                           const float *gamma, float *sum1, float *sum2,
                                                                           float *m1, float *m2) {
    const int64_t n = blockIdx.x;
    for (int c = threadIdx.x; c < s.channels; c += kThreads) {
        float t1 = 0.f, t2 = 0.f;
        for (int k = 0; k < s.chunks; ++k) {
            t1 += part1[(n * s.chunks + k) * s.channels + c];
            t2 += part2[(n * s.chunks + k) * s.channels + c];
        }
        sum1[n * s.channels + c] = t1;
        sum2[n * s.channels + c] = t2;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const float total = (float)s.positions * (float)s.cg;
    for (int g = threadIdx.x >> 5; g < groups; g += kThreads / 32) {
        float t1 = 0.f, t2 = 0.f;
        for (int c = g * s.cg + lane; c < (g + 1) * s.cg; c += 32) {
            const float w = gamma ? gamma[c] : 1.f;
            t1 = fmaf(w, sum1[n * s.channels + c], t1);
            t2 = fmaf(w, sum2[n * s.channels + c], t2);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            t1 += __shfl_xor_sync(0xffffffffu, t1, o);
            t2 += __shfl_xor_sync(0xffffffffu, t2, o);
        }
        if (lane == 0) {
            m1[n * groups + g] = t1 / total;
            m2[n * groups + g] = t2 / total;
        }
    }
}

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads) cr_group_norm_grad_apply_kernel(const GroupNormArgs a, const Split s, const float *m1, const float *m2) {
    const Place p = place<VEC>(s);
    if (p.j < 0) return;
    Affine<VEC> f;
    f.load(p, s, a.groups, a.mean, a.rstd, a.gamma, a.beta);
    float b1[VEC], b2[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int64_t at = p.n * a.groups + (p.c0 + i) / s.cg;
        b1[i] = m1[at];
        b2[i] = m2[at];
    }
    const int64_t first = p.n * s.positions + p.row0;
    for (int r = p.j; r < p.rows; r += p.rt) {
        float dz[VEC], xh[VEC];
        slopes<T, VEC, ACT>(a, f, first + r, p.c0, s.channels, dz, xh);
        // gamma dz is rounded before m1 leaves it: a group of one value has m1 = gamma dz and so a gradient of zero
#pragma unroll
        for (int i = 0; i < VEC; ++i) dz[i] = f.rstd[i] * fmaf(-xh[i], b2[i], __fmul_rn(f.gamma[i], dz[i]) - b1[i]);
        store_packed<T, VEC>(static_cast<T *>(a.y) + ((first + r) * a.ld_y + p.c0), pack<T, VEC>(dz));
    }
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

// The elements of a row-major [rows][cols] tensor as vectors; a thread takes kUnroll of them, a block apart.  Where the
// row strides are the width, the caller passes one long row and no division is made.
template <typename T, int VEC, typename I>
__global__ void __launch_bounds__(kThreads) cr_dropout_kernel(const T *x, const T *residual, T *y, I nvec, I vecs_per_row, int64_t ld_x,
                                                              int64_t ld_r, int64_t ld_y, const DropSpec d) {
    constexpr int kUnroll = 4;
    const I v0 = (I)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
    Packed<T, VEC> px[kUnroll], pr[kUnroll];
    int64_t row[kUnroll], col[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const I v = v0 + u * kThreads;
        const I r = vecs_per_row == nvec ? 0 : v / vecs_per_row;
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

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

Split make_split(int64_t samples, int64_t positions, int channels, int groups, int vec) {
    Split s;
    s.positions = positions;
    s.channels = channels;
    s.cg = channels / groups;
    s.nvec = channels / vec;
    s.tiles = (s.nvec + kThreads - 1) / kThreads;
    // chunks of at least 32 rows a thread-row, about 2048 blocks in all
    const int vecs = std::min(kThreads, s.nvec);
    const int64_t least = 32ll * (kThreads / vecs);
    int64_t chunks = std::max<int64_t>(1, 2048 / std::max<int64_t>(1, samples * s.tiles));
    chunks = std::min(chunks, std::max<int64_t>(1, positions / least));
    s.rows_per_chunk = (positions + chunks - 1) / chunks;
    // a block counts its rows in 32 bits, and a float holds the count of a group without rounding far beyond this
    s.rows_per_chunk = std::min<int64_t>(s.rows_per_chunk, 1 << 24);
    s.chunks = (int)((positions + s.rows_per_chunk - 1) / s.rows_per_chunk);
    return s;
}

template <typename F>
cudaError_t by_type(int elem, F &&f) {
    switch (elem) {
        case kElemF32: return f(float{});
        case kElemBF16: return f(__nv_bfloat16{});
        default: return f(__half{});
    }
}
template <int V> struct Int { static constexpr int value = V; };
template <typename F>
cudaError_t by_act(int act, F &&f) {
    switch (act) {
        case kActNone: return f(Int<kActNone>{});
        case kActRelu: return f(Int<kActRelu>{});
        default: return f(Int<kActSilu>{});
    }
}

// The vector form needs whole 16-byte vectors in every row.
bool vector_rows(int elem, int64_t channels, std::initializer_list<const void *> ptrs, std::initializer_list<int64_t> lds) {
    const int vec = 16 / elem_bytes(elem);
    if (channels % vec) return false;
    for (const void *p : ptrs)
        if (p && !aligned16(p)) return false;
    for (int64_t ld : lds)
        if (ld % vec) return false;
    return true;
}

}  // namespace

size_t group_norm_workspace_bytes(int64_t samples, int64_t positions, int channels, int groups, int elem) {
    if (samples < 1) return 0;
    size_t most = 0;
    for (int vec : {1, 16 / elem_bytes(elem)}) {
        if (channels % vec) continue;
        const Split s = make_split(samples, positions, channels, groups, vec);
        most = std::max(most, ((size_t)s.chunks * channels + groups) * (size_t)samples * 8);
    }
    return most;
}

size_t group_norm_backward_workspace_bytes(int64_t samples, int64_t positions, int channels, int groups, int elem) {
    if (samples < 1) return 0;
    size_t most = 0;
    for (int vec : {1, 16 / elem_bytes(elem)}) {
        if (channels % vec) continue;
        const Split s = make_split(samples, positions, channels, groups, vec);
        most = std::max(most, ((size_t)(s.chunks + 1) * channels + groups) * (size_t)samples * 8);
    }
    // the one-pass form's rows of sums
    return std::max(most, (size_t)group_norm_backward_on_chip(samples, positions, channels, groups, elem) * channels * (size_t)samples * 8);
}

cudaError_t launch_group_norm(const GroupNormArgs &in, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (in.samples == 0) return cudaSuccess;
    GroupNormArgs a = in;
    const bool wide = vector_rows(a.elem, a.channels, {a.x, a.y}, {a.ld_x, a.ld_y});
    if (wide && group_norm_on_chip(a.samples, a.positions, a.channels, a.groups, a.elem)) return launch_group_norm_on_chip(a, stream, launches);
    const Split s = make_split(a.samples, a.positions, a.channels, a.groups, wide ? 16 / elem_bytes(a.elem) : 1);
    float *part_mean = a.workspace;
    float *part_m2 = part_mean + (size_t)a.samples * s.chunks * a.channels;
    if (!a.mean) a.mean = part_m2 + (size_t)a.samples * s.chunks * a.channels;
    if (!a.rstd) a.rstd = part_m2 + (size_t)a.samples * s.chunks * a.channels + (size_t)a.samples * a.groups;
    const unsigned blocks = (unsigned)(a.samples * s.tiles * s.chunks);
    auto run = [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        cr_group_norm_stats_kernel<T, VEC><<<blocks, kThreads, 0, stream>>>(static_cast<const T *>(a.x), a.ld_x, s, part_mean, part_m2);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        cr_group_norm_join_kernel<<<(unsigned)(a.samples * a.groups), 128, 0, stream>>>(part_mean, part_m2, s, a.groups, a.eps, a.mean, a.rstd);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        e = by_act(a.act, [&](auto act) {
            cr_group_norm_apply_kernel<T, VEC, decltype(act)::value><<<blocks, kThreads, 0, stream>>>(a, s);
            return cudaGetLastError();
        });
        if (e == cudaSuccess) *launches += 3;
        return e;
    };
    return by_type(a.elem, [&](auto t) { return wide ? run(t, Int<16 / (int)sizeof(t)>{}) : run(t, Int<1>{}); });
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
    const bool wide = vector_rows(a.elem, a.channels, {a.x, a.dy, a.y}, {a.ld_x, a.ld_dy, a.y ? a.ld_y : 0});
    const Split s = make_split(a.samples, a.positions, a.channels, a.groups, wide ? 16 / elem_bytes(a.elem) : 1);
    const size_t plane = (size_t)a.samples * a.channels;
    float *sum1 = a.workspace, *sum2 = sum1 + plane;
    float *part1 = sum2 + plane, *part2 = part1 + plane * s.chunks;
    float *m1 = part2 + plane * s.chunks, *m2 = m1 + (size_t)a.samples * a.groups;
    const unsigned blocks = (unsigned)(a.samples * s.tiles * s.chunks);
    const bool params = a.dgamma || a.dbeta;
    cudaError_t e;
    if (const int rows = wide ? group_norm_backward_on_chip(a.samples, a.positions, a.channels, a.groups, a.elem) : 0) {
        // a partition of one sample that one CTA holds has its sums where they belong
        if (a.partitions == a.samples && rows == 2) return launch_group_norm_grad_on_chip(a, a.dbeta, a.dgamma, a.ld_param, true, stream, launches);
        sum2 = sum1 + plane * rows;
        e = launch_group_norm_grad_on_chip(a, params ? sum1 : nullptr, params ? sum2 : nullptr, a.channels, false, stream, launches);
        if (e != cudaSuccess || !params) return e;
        return launch_params(a, sum1, sum2, rows, stream, launches);
    }
    auto run = [&](auto t, auto v, auto act) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value, ACT = decltype(act)::value;
        cr_group_norm_grad_sums_kernel<T, VEC, ACT><<<blocks, kThreads, 0, stream>>>(a, s, part1, part2);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        cr_group_norm_grad_join_kernel<<<(unsigned)a.samples, kThreads, 0, stream>>>(part1, part2, s, a.groups, a.gamma, sum1, sum2, m1, m2);
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        *launches += 2;
        if (a.y) {
            cr_group_norm_grad_apply_kernel<T, VEC, ACT><<<blocks, kThreads, 0, stream>>>(a, s, m1, m2);
            e = cudaGetLastError();
            if (e != cudaSuccess) return e;
            ++*launches;
        }
        return cudaSuccess;
    };
    e = by_type(a.elem, [&](auto t) {
        return by_act(a.act, [&](auto act) { return wide ? run(t, Int<16 / (int)sizeof(t)>{}, act) : run(t, Int<1>{}, act); });
    });
    if (e != cudaSuccess || !params) return e;
    return launch_params(a, sum1, sum2, 1, stream, launches);
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
    auto run = [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        const int64_t per_row = cols / VEC, nvec = rows * per_row;
        const int64_t blocks = (nvec + kThreads * 4 - 1) / (kThreads * 4);
        if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
        auto go = [&](auto i) {
            using I = decltype(i);
            cr_dropout_kernel<T, VEC, I><<<(unsigned)blocks, kThreads, 0, stream>>>(
                static_cast<const T *>(x), static_cast<const T *>(residual), static_cast<T *>(y), (I)nvec, (I)per_row, ld_x, ld_r, ld_y, drop);
        };
        if (nvec < (1ll << 31)) go(uint32_t{});
        else go(uint64_t{});
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    };
    return by_type(elem, [&](auto t) {
        // one long row may end inside a vector: the scalar form takes it whole
        constexpr int VEC = 16 / (int)sizeof(t);
        const bool one = rows == 1;
        return vector_rows(elem, cols, {x, residual, y}, {one ? 0 : ld_x, one ? 0 : ld_r, one ? 0 : ld_y}) ? run(t, Int<VEC>{}) : run(t, Int<1>{});
    });
}

}  // namespace cr
