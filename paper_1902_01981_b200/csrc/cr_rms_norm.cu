// Root-mean-square norm of rows, with the residual's addition in front and 8-bit codes behind, and its gradient.
//
//   h = x + r,  rstd = 1 / sqrt(sum_c h_c^2 / C + eps),  y_c = h_c rstd gamma_c,  or codes of y: q_c = rint(127 y_c / max |y|)
//   g = dy gamma,  xhat = h rstd,  dx = dh + rstd (g - xhat (sum_c g_c xhat_c) / C),  dgamma = sum over a partition's rows of dy xhat
//
// x and r may lie in 16 bits: their sum is held in 32, the norm is taken of that, and h is rounded once, where it is stored.
// Sums are fp32; the order of a row's sum follows from its length, the element type and whether all tensors lie in 16-byte
// vectors; that of dgamma from the partition's rows besides.  No atomics.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cr_elem.cuh"

namespace cr {
namespace {

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sum over a block of whole warps, the same in every thread; `sm` holds 32 floats and is free again after the next barrier.
__device__ __forceinline__ float block_sum(float v, float *sm) {
    v = warp_sum(v);
    const int warps = (int)blockDim.x / 32;
    if (warps == 1) return v;
    if (threadIdx.x % 32 == 0) sm[threadIdx.x / 32] = v;
    __syncthreads();
    const int lane = (int)threadIdx.x % 32;
    return warp_sum(lane < warps ? sm[lane] : 0.f);
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *sm) {
    v = __reduce_max_sync(0xffffffffu, v);
    const int warps = (int)blockDim.x / 32;
    if (warps == 1) return v;
    if (threadIdx.x % 32 == 0) sm[threadIdx.x / 32] = v;
    __syncthreads();
    const int lane = (int)threadIdx.x % 32;
    return __reduce_max_sync(0xffffffffu, lane < warps ? sm[lane] : 0u);
}

template <int VEC>
__device__ __forceinline__ void load_floats(const float *p, float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        v[0] = *p;
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
            const float4 f = reinterpret_cast<const float4 *>(p)[i];
            v[4 * i] = f.x; v[4 * i + 1] = f.y; v[4 * i + 2] = f.z; v[4 * i + 3] = f.w;
        }
    }
}

// Vectors of a row that a thread keeps in registers.
template <int VEC> __host__ __device__ constexpr int held_vectors() { return VEC == 1 ? 16 : 4; }

// One block a row.  The first vectors of each thread stay in registers as fp32 sums between the statistics and the output;
// longer rows are read again (from L2).  Everything is read before the block's first barrier or by the thread that
// writes it, so outputs may be the inputs' own buffers.
template <typename T, int VEC, bool CODES>
__global__ void __launch_bounds__(1024) cr_rms_norm_kernel(const RmsNormArgs a) {
    constexpr int kHeld = held_vectors<VEC>();
    __shared__ float sums[32];
    __shared__ uint32_t tops[32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ld_residual : nullptr;
    T *h = a.h ? static_cast<T *>(a.h) + row * a.ld_h : nullptr;
    const int64_t nvec = a.cols / VEC;
    const int nt = (int)blockDim.x, tid = (int)threadIdx.x;
    auto sum_at = [&](int64_t v, float (&f)[VEC]) {
        unpack<T, VEC>(load_packed<T, VEC>(x + v * VEC), f);
        if (r) {
            float g[VEC];
            unpack<T, VEC>(load_packed<T, VEC>(r + v * VEC), g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] += g[i];
        }
    };
    float held[kHeld][VEC];
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) sum_at(tid + u * nt, held[u]);
    float squares = 0.f;
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) squares = fmaf(held[u][i], held[u][i], squares);
        }
    for (int64_t v = tid + (int64_t)kHeld * nt; v < nvec; v += nt) {
        float f[VEC];
        sum_at(v, f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) squares = fmaf(f[i], f[i], squares);
    }
    const float rstd = 1.f / sqrtf(block_sum(squares, sums) / (float)a.cols + a.eps);
    if (a.rstd && tid == 0) a.rstd[row] = rstd;
    // y of vector v in place of its sum
    auto norm = [&](int64_t v, const float (&f)[VEC], float (&z)[VEC]) {
        float g[VEC];
        if (a.gamma) load_floats<VEC>(a.gamma + v * VEC, g);
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = f[i] * rstd * (a.gamma ? g[i] : 1.f);
    };
    RowScale rs = {0.f, 0.f};
    bool dead = false;
    if constexpr (CODES) {
        uint32_t top = 0;
        auto widen = [&](const float (&z)[VEC]) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) top = max(top, __float_as_uint(z[i]) & 0x7fffffffu);
        };
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (tid + u * nt < nvec) {
                float z[VEC];
                norm(tid + u * nt, held[u], z);
                widen(z);
            }
        for (int64_t v = tid + (int64_t)kHeld * nt; v < nvec; v += nt) {
            float f[VEC], z[VEC];
            sum_at(v, f);
            norm(v, f, z);
            widen(z);
        }
        top = block_max(top, tops);
        rs = row_scale(top);
        dead = top >= 0x7f800000u;
        if (tid == 0) a.scale[row] = rs.scale;
    }
    auto put = [&](int64_t v, const float (&f)[VEC]) {
        float z[VEC];
        norm(v, f, z);
        if (h) store_packed<T, VEC>(h + v * VEC, pack<T, VEC>(f));
        if constexpr (CODES) {
            int8_t *q = a.q + row * a.ld_q + v * VEC;
            if constexpr (VEC == 1) {
                *q = dead ? (int8_t)0 : (int8_t)code(z[0], rs.mult);
            } else {
                uint32_t w[VEC / 4];
#pragma unroll
                for (int i = 0; i < VEC / 4; ++i) {
                    const uint32_t lo = __byte_perm(code(z[4 * i], rs.mult), code(z[4 * i + 1], rs.mult), 0x0040);
                    const uint32_t hi = __byte_perm(code(z[4 * i + 2], rs.mult), code(z[4 * i + 3], rs.mult), 0x0040);
                    w[i] = dead ? 0u : __byte_perm(lo, hi, 0x5410);
                }
                if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(q) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t *>(q) = w[0];
            }
        } else {
            store_packed<T, VEC>(static_cast<T *>(a.y) + row * a.ld_y + v * VEC, pack<T, VEC>(z));
        }
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) put(tid + u * nt, held[u]);
    for (int64_t v = tid + (int64_t)kHeld * nt; v < nvec; v += nt) {
        float f[VEC];
        sum_at(v, f);
        put(v, f);
    }
}

// ---- gradient ------------------------------------------------------------------------------------------------------------

// A row's (sum g xhat) / C.
template <typename T, int VEC>
__global__ void __launch_bounds__(1024) cr_rms_norm_dots_kernel(const RmsNormArgs a, float *dots) {
    __shared__ float sums[32];
    const int64_t row = blockIdx.x;
    const T *dy = static_cast<const T *>(a.dy) + row * a.ld_dy, *h = static_cast<const T *>(a.h) + row * a.ld_h;
    const int64_t nvec = a.cols / VEC;
    const float rstd = a.rstd[row];
    float dot = 0.f;
    for (int64_t v = threadIdx.x; v < nvec; v += blockDim.x) {
        float g[VEC], x[VEC], w[VEC];
        unpack<T, VEC>(load_packed<T, VEC>(dy + v * VEC), g);
        unpack<T, VEC>(load_packed<T, VEC>(h + v * VEC), x);
        if (a.gamma) load_floats<VEC>(a.gamma + v * VEC, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) dot = fmaf(a.gamma ? g[i] * w[i] : g[i], x[i] * rstd, dot);
    }
    dot = block_sum(dot, sums);
    if (threadIdx.x == 0) dots[row] = dot / (float)a.cols;
}

// Rows of a partition that one block adds up: the partition's rows in at most 256 chunks of 4 to 64 rows.
int64_t chunk_rows(int64_t rows) { return std::min<int64_t>(64, std::max<int64_t>(4, (rows + 255) / 256)); }

// dx of a chunk of rows for a slab of columns, and the chunk's sums of dy xhat.
template <typename T, int VEC>
__global__ void __launch_bounds__(128) cr_rms_norm_grad_kernel(const RmsNormArgs a, const float *dots, float *partial, int64_t ld_partial, int64_t rows_each,
                                                               int chunk, int chunks, int slabs) {
    const unsigned item = blockIdx.x / (unsigned)slabs;
    const int64_t v = (int64_t)(blockIdx.x % (unsigned)slabs) * blockDim.x + threadIdx.x;
    const int64_t part = item / (unsigned)chunks, c = item % (unsigned)chunks;
    if (v >= a.cols / VEC) return;
    const int64_t first = c * chunk, count = min((int64_t)chunk, rows_each - first);
    float w[VEC], acc[VEC] = {};
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[i] = 1.f;
    if (a.gamma) load_floats<VEC>(a.gamma + v * VEC, w);
    for (int64_t k = 0; k < count; ++k) {
        const int64_t row = part * rows_each + first + k;
        const float rstd = a.rstd[row];
        float g[VEC], x[VEC];
        unpack<T, VEC>(load_packed<T, VEC>(static_cast<const T *>(a.dy) + row * a.ld_dy + v * VEC), g);
        unpack<T, VEC>(load_packed<T, VEC>(static_cast<const T *>(a.h) + row * a.ld_h + v * VEC), x);
        float d[VEC] = {};
        if (a.y && a.dh) unpack<T, VEC>(load_packed<T, VEC>(static_cast<const T *>(a.dh) + row * a.ld_dh + v * VEC), d);
        const float dot = a.y ? dots[row] : 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float xhat = x[i] * rstd;
            acc[i] = fmaf(g[i], xhat, acc[i]);
            d[i] = fmaf(rstd, fmaf(-xhat, dot, g[i] * w[i]), d[i]);
        }
        if (a.y) store_packed<T, VEC>(static_cast<T *>(a.y) + row * a.ld_y + v * VEC, pack<T, VEC>(d));
    }
    if (partial) {
        float *out = partial + item * ld_partial + v * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = acc[i];
    }
}

// dgamma of a partition from its chunks' sums: eight warps take every eighth chunk and are summed in order.
__global__ void __launch_bounds__(256) cr_rms_norm_params_kernel(const float *partial, int chunks, int64_t cols, float *dgamma, int64_t ld, unsigned slabs) {
    __shared__ float sm[8][32];
    const int64_t part = blockIdx.x / slabs;
    const int lane = (int)threadIdx.x % 32, warp = (int)threadIdx.x / 32;
    const int64_t col = (int64_t)(blockIdx.x % slabs) * 32 + lane;
    float sum = 0.f;
    if (col < cols)
        for (int c = warp; c < chunks; c += 8) sum += partial[(part * chunks + c) * cols + col];
    sm[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || col >= cols) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += sm[w][lane];
    dgamma[part * ld + col] = sum;
}

__global__ void cr_rms_norm_zero_kernel(float *dgamma, int64_t partitions, int64_t cols, int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < partitions * cols) dgamma[i / cols * ld + i % cols] = 0.f;
}

template <typename T, int VEC>
int row_threads(int64_t cols) {
    const int64_t nvec = cols / VEC, held = held_vectors<VEC>();
    return (int)std::min<int64_t>(1024, (nvec + held * 32 - 1) / (held * 32) * 32);
}

}  // namespace

cudaError_t launch_rms_norm(const RmsNormArgs &a, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    return by_type(a.elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        bool wide = vector_rows(a.elem, a.cols, {a.x, a.residual, a.h, a.y, a.gamma},
                                {a.ld_x, a.residual ? a.ld_residual : 0, a.h ? a.ld_h : 0, a.y ? a.ld_y : 0});
        if (a.q) wide = wide && reinterpret_cast<uintptr_t>(a.q) % VEC == 0 && a.ld_q % VEC == 0;
        auto go = [&](auto v, auto codes) {
            constexpr int V = decltype(v)::value;
            cr_rms_norm_kernel<T, V, decltype(codes)::value != 0><<<(unsigned)a.rows, row_threads<T, V>(a.cols), 0, stream>>>(a);
        };
        if (wide) a.q ? go(Int<VEC>{}, Int<1>{}) : go(Int<VEC>{}, Int<0>{});
        else a.q ? go(Int<1>{}, Int<1>{}) : go(Int<1>{}, Int<0>{});
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

size_t rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t partitions) {
    if (rows == 0 || partitions == 0) return 0;
    const int64_t each = rows / partitions, chunk = chunk_rows(each), chunks = (each + chunk - 1) / chunk;
    return ((size_t)rows * 4 + 15) / 16 * 16 + (size_t)(chunks > 1 ? partitions * chunks * cols * 4 : 0);
}

cudaError_t launch_rms_norm_backward(const RmsNormArgs &a, float *workspace, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) {
        const int64_t count = a.partitions * a.cols;
        if (!a.dgamma || count == 0) return cudaSuccess;
        if ((count + 255) / 256 > 0x7fffffffll) return cudaErrorInvalidValue;
        cr_rms_norm_zero_kernel<<<(unsigned)((count + 255) / 256), 256, 0, stream>>>(a.dgamma, a.partitions, a.cols, a.ld_gamma);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    }
    const int64_t each = a.rows / a.partitions;
    const int chunk = (int)chunk_rows(each), chunks = (int)((each + chunk - 1) / chunk);
    float *dots = workspace, *partial = workspace + (a.rows + 3) / 4 * 4;
    cudaError_t e = by_type(a.elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const bool wide = vector_rows(a.elem, a.cols, {a.dy, a.dh, a.h, a.y, a.gamma}, {a.ld_dy, a.dh ? a.ld_dh : 0, a.ld_h, a.y ? a.ld_y : 0});
        auto go = [&](auto v) {
            constexpr int V = decltype(v)::value;
            if (a.y) {
                cr_rms_norm_dots_kernel<T, V><<<(unsigned)a.rows, row_threads<T, V>(a.cols), 0, stream>>>(a, dots);
                const cudaError_t e = cudaGetLastError();
                if (e != cudaSuccess) return e;
                ++*launches;
            }
            const int64_t nvec = a.cols / V;
            const int threads = (int)std::min<int64_t>(128, (nvec + 31) / 32 * 32);
            const int64_t slabs = (nvec + threads - 1) / threads;
            if (a.partitions * chunks > 0x7fffffffll / slabs) return cudaErrorInvalidValue;
            float *sums = !a.dgamma ? nullptr : chunks > 1 ? partial : a.dgamma;
            cr_rms_norm_grad_kernel<T, V><<<(unsigned)(a.partitions * chunks * slabs), threads, 0, stream>>>(
                a, dots, sums, chunks > 1 ? a.cols : a.ld_gamma, each, chunk, chunks, (int)slabs);
            const cudaError_t e = cudaGetLastError();
            if (e == cudaSuccess) ++*launches;
            return e;
        };
        return wide ? go(Int<VEC>{}) : go(Int<1>{});
    });
    if (e != cudaSuccess || !a.dgamma || chunks == 1) return e;
    const int64_t slabs = (a.cols + 31) / 32;
    if (a.partitions > 0x7fffffffll / slabs) return cudaErrorInvalidValue;
    cr_rms_norm_params_kernel<<<(unsigned)(a.partitions * slabs), 256, 0, stream>>>(partial, chunks, a.cols, a.dgamma, a.ld_gamma, (unsigned)slabs);
    e = cudaGetLastError();
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cr
