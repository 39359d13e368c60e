// Products of 8-bit integer matrices with a scale for each token and each channel, and the quantiser of tokens:
//   s_t = max_k |x_tk| / 127,  q_tk = rint(x_tk * (127 / max_k |x_tk|)),
//   y_tn = (sum_k q_tk w_nk) * (s_t s_n) + bias_n.
// The sum is taken in 32-bit integers (|sum| <= 2^14 k: exact for every k the entry point takes), so it has no order
// and no rounding: the tiles, the split over k and the machine do not show in the result.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cr_elem.cuh"

namespace cr {
namespace {

// ---- quantiser ------------------------------------------------------------------------------------------------------

// Rows whose largest magnitude is below 2^-120 count as zero (127 / max would leave the range of a float); a row with an
// infinity or a NaN gets the scale NaN, which its outputs then show.
struct RowScale {
    float mult, scale;
};
__device__ __forceinline__ RowScale row_scale(uint32_t largest_bits) {
    const float largest = __uint_as_float(largest_bits);
    if (largest_bits >= 0x7f800000u) return {0.f, __uint_as_float(0x7fc00000u)};
    if (largest < 0x1p-120f) return {0.f, 0.f};
    return {__fdiv_rn(127.f, largest), __fdiv_rn(largest, 127.f)};
}
__device__ __forceinline__ int code(float x, float mult) {
    return mult == 0.f ? 0 : max(-127, min(127, __float2int_rn(x * mult)));
}

// One block per row.  The row's first kHeld vectors of each thread stay in registers between the search for the
// largest magnitude and the rounding; longer rows are read a second time (from L2).
template <typename T, int VEC>
__global__ void __launch_bounds__(512) cr_quantize_rows_kernel(const T *x, int64_t cols, int64_t ld_x, int8_t *q, int64_t ld_q, float *scale) {
    constexpr int kHeld = 4;
    __shared__ uint32_t sm[16];
    const T *row = x + (int64_t)blockIdx.x * ld_x;
    int8_t *out = q + (int64_t)blockIdx.x * ld_q;
    const int64_t nvec = cols / VEC;
    const int nt = (int)blockDim.x, tid = (int)threadIdx.x;
    Packed<T, VEC> held[kHeld];
    uint32_t top = 0;
    // magnitudes are compared as integers: the order is the same, and a NaN is larger than everything
    auto look = [&](const Packed<T, VEC> &pv) {
        float v[VEC];
        unpack<T, VEC>(pv, v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) held[u] = load_packed<T, VEC>(row + (int64_t)(tid + u * nt) * VEC);
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) look(held[u]);
    for (int64_t v = tid + kHeld * nt; v < nvec; v += nt) look(load_packed<T, VEC>(row + v * VEC));
    for (int64_t c = nvec * VEC + tid; c < cols; c += nt) top = max(top, __float_as_uint(to_float(row[c])) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if ((tid & 31) == 0) sm[tid >> 5] = top;
    __syncthreads();
    top = sm[0];
    for (int w = 1; w < nt / 32; ++w) top = max(top, sm[w]);
    const RowScale rs = row_scale(top);
    if (tid == 0) scale[blockIdx.x] = rs.scale;
    auto put = [&](const Packed<T, VEC> &pv, int64_t v) {
        float f[VEC];
        unpack<T, VEC>(pv, f);
        if constexpr (VEC == 1) {
            out[v] = (int8_t)code(f[0], rs.mult);
        } else {
            uint32_t w[VEC / 4];
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i) {
                uint32_t b = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) b |= ((uint32_t)code(f[4 * i + k], rs.mult) & 0xffu) << (8 * k);
                w[i] = b;
            }
            if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(out + v * 8) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(out + v * 4) = w[0];
        }
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) put(held[u], tid + u * nt);
    for (int64_t v = tid + kHeld * nt; v < nvec; v += nt) put(load_packed<T, VEC>(row + v * VEC), v);
    for (int64_t c = nvec * VEC + tid; c < cols; c += nt) out[c] = (int8_t)code(to_float(row[c]), rs.mult);
}

// ---- product, any alignment --------------------------------------------------------------------------------------------
//
// 64 x 64 outputs a block, 64 bytes of k at a time through shared memory, four-way byte products.  It serves rows that
// do not start on 16-byte boundaries, which the copy engine cannot fetch.
template <typename T>
__global__ void __launch_bounds__(256) cr_int8_product_bytes_kernel(const Int8ProductArgs a) {
    constexpr int kTile = 64, kWords = 16;
    __shared__ int sx[kTile][kWords + 1], sw[kTile][kWords + 1];
    const int64_t tiles_n = (a.outer + kTile - 1) / kTile;
    const int64_t m0 = (int64_t)blockIdx.x / tiles_n * kTile, n0 = (int64_t)blockIdx.x % tiles_n * kTile;
    const int tid = (int)threadIdx.x, tm = tid / 16, tn = tid % 16;
    int acc[4][4] = {};
    for (int64_t k0 = 0; k0 < a.inner; k0 += 4 * kWords) {
        // a byte a thread, 64 threads to a row: neighbouring threads read neighbouring bytes
        for (int e = tid; e < kTile * 4 * kWords; e += 256) {
            const int r = e / (4 * kWords), b = e % (4 * kWords);
            const bool in = k0 + b < a.inner;
            reinterpret_cast<int8_t *>(&sx[r][0])[b] = in && m0 + r < a.tokens ? a.x[(m0 + r) * a.ld_x + k0 + b] : (int8_t)0;
            reinterpret_cast<int8_t *>(&sw[r][0])[b] = in && n0 + r < a.outer ? a.w[(n0 + r) * a.ld_w + k0 + b] : (int8_t)0;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            int xv[4], wv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                xv[i] = sx[tm + 16 * i][w];
                wv[i] = sw[tn + 16 * i][w];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(xv[i], wv[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + tm + 16 * i;
        if (m >= a.tokens) continue;
        const float s = a.x_scale[m];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + tn + 16 * j;
            if (n >= a.outer) continue;
            static_cast<T *>(a.y)[m * a.ld_y + n] = from_float<T>(fmaf((float)acc[i][j], s * a.w_scale[n], a.bias ? a.bias[n] : 0.f));
        }
    }
}

template <typename F>
cudaError_t by_type(int elem, F &&f) {
    switch (elem) {
        case kElemF32: return f(float{});
        case kElemBF16: return f(__nv_bfloat16{});
        default: return f(__half{});
    }
}

}  // namespace

cudaError_t launch_quantize_rows(const void *x, int64_t rows, int64_t cols, int64_t ld_x, int elem, int8_t *q, int64_t ld_q,
                                 float *scale, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (rows == 0) return cudaSuccess;
    return by_type(elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ld_x % VEC == 0 && (reinterpret_cast<uintptr_t>(q) & (VEC - 1)) == 0 &&
                          ld_q % VEC == 0;
        const int64_t nvec = wide ? (cols + VEC - 1) / VEC : cols;
        const int threads = (int)std::min<int64_t>(512, std::max<int64_t>(32, (nvec + 127) / 128 * 32));   // about four vectors a thread
        if (wide) cr_quantize_rows_kernel<T, VEC><<<(unsigned)rows, threads, 0, stream>>>(static_cast<const T *>(x), cols, ld_x, q, ld_q, scale);
        else cr_quantize_rows_kernel<T, 1><<<(unsigned)rows, threads, 0, stream>>>(static_cast<const T *>(x), cols, ld_x, q, ld_q, scale);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

cudaError_t launch_int8_product(const Int8ProductArgs &a, int *, const DeviceInfo &, const Tuning &, EncodeTiledFn,
                                cudaStream_t stream, int64_t *launches) {
    if (a.tokens == 0 || a.outer == 0) return cudaSuccess;
    const int64_t blocks = ((a.tokens + 63) / 64) * ((a.outer + 63) / 64);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    return by_type(a.elem, [&](auto t) {
        cr_int8_product_bytes_kernel<decltype(t)><<<(unsigned)blocks, 256, 0, stream>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

}  // namespace cr
