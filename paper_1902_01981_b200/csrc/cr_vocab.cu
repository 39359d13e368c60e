// Rows of logits over a vocabulary: log probabilities of given tokens with entropy and the best alternatives, distillation from a
// teacher's top logits, and their gradients.
//
//   z = x / T,  lse = log sum_v e^{z_v},  logp = z_id - lse,  H = lse - sum_v p_v z_v,  p_v = e^{z_v - lse}
//   dx_v = (1/T) (a (1[v = id] - p_v) - b p_v (log p_v + H))                      a = d logp, b = d H
//   t = softmax over the teacher's k logits / T,  loss = T^2 sum_j t_j (log t_j - log p_{id_j}),  dx_v = w T (p_v - sum_{j: id_j = v} t_j)
//
// With c = log2(e) / T and the row's largest logit m, e^{z_v - m/T} = 2^{(x_v - m) c}.  The difference comes first: it is exact
// near m, and a row whose logits are all the type's lowest value stays in range.  What a row keeps for its gradient is m and
// log sum_v e^{(x_v - m)/T}, not their sum, which would round the second one away where m is large.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cr_elem.cuh"

namespace cr {
namespace {

constexpr int kThreads = 256;
constexpr float kLn2 = 0.6931471805599453f;
// Exponents below this are zero in fp32; the clamp keeps 0 * -infinity out of the entropy.
constexpr float kLeast = -160.f;

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <typename F>
__device__ __forceinline__ float block_reduce(float v, float *sm, F f) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if (threadIdx.x % 32 == 0) sm[threadIdx.x / 32] = v;
    __syncthreads();
    v = sm[0];
    for (int w = 1; w < kThreads / 32; ++w) v = f(v, sm[w]);
    return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// Position in the order of the alternatives: the larger value first, then the lower index; a NaN above everything.
__device__ __forceinline__ unsigned long long rank_key(float x, uint32_t index) {
    const uint32_t b = __float_as_uint(x + 0.f);     // -0 counts as 0
    const uint32_t order = x != x ? 0xffffffffu : (b >> 31) ? ~b : b | 0x80000000u;
    return (unsigned long long)order << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(unsigned long long key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float((order >> 31) ? order & 0x7fffffffu : ~order);
}

__device__ __forceinline__ int64_t id_at(const void *ids, int id_bytes, int64_t i) {
    return id_bytes == 4 ? (int64_t)static_cast<const int32_t *>(ids)[i] : (int64_t)static_cast<const long long *>(ids)[i];
}

struct RowStats {
    float m, base, sum, turn;    // the largest logit; the same, 0 for an infinity; sum of 2^u, u = (x - base) c; sum of 2^u u
};

template <typename T, int VEC>
__device__ __forceinline__ RowStats row_stats(const T *x, int64_t vocab, float c, float *sm) {
    const int64_t nvec = vocab / VEC;
    float m = -INFINITY;
    for (int64_t v = threadIdx.x; v < nvec; v += kThreads) {
        float f[VEC];
        unpack<T, VEC>(load_packed<T, VEC>(x + v * VEC), f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) m = max_nan(m, f[i]);
    }
    m = block_reduce(m, sm, max_nan);
    RowStats r;
    r.m = m;
    r.base = isinf(m) ? 0.f : m;
    float s = 0.f, t = 0.f;
    for (int64_t v = threadIdx.x; v < nvec; v += kThreads) {
        float f[VEC];
        unpack<T, VEC>(load_packed<T, VEC>(x + v * VEC), f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float u = max_nan((f[i] - r.base) * c, kLeast), e = exp2_approx(u);
            s += e;
            t = fmaf(e, u, t);
        }
    }
    r.sum = block_reduce(s, sm, add);
    r.turn = block_reduce(t, sm, add);
    return r;
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) cr_token_log_probs_kernel(const VocabArgs a) {
    __shared__ float sm[kThreads / 32];
    __shared__ unsigned long long keys[kThreads / 32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    const float c = a.inverse * kLog2e;
    const RowStats r = row_stats<T, VEC>(x, a.vocab, c, sm);
    const bool nothing = r.sum == 0.f;
    const float log_sum = log2f(r.sum);
    if (threadIdx.x == 0) {
        if (a.stats) reinterpret_cast<float2 *>(a.stats)[row] = make_float2(r.m, kLn2 * log_sum);
        if (a.entropy) a.entropy[row] = nothing ? 0.f : kLn2 * (log_sum - r.turn / r.sum);
        if (a.logp) {
            const int64_t id = id_at(a.ids, a.id_bytes, row);
            a.logp[row] = id < 0 || id >= a.vocab ? 0.f : nothing ? -INFINITY : kLn2 * ((to_float(x[id]) - r.base) * c - log_sum);
        }
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        unsigned long long best = 0;
        for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) {
            const unsigned long long key = rank_key(to_float(x[v]), (uint32_t)v);
            if ((k == 0 || key < last) && key > best) best = key;
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        __syncthreads();
        if (threadIdx.x % 32 == 0) keys[threadIdx.x / 32] = best;
        __syncthreads();
        for (int w = 0; w < kThreads / 32; ++w) best = max(best, keys[w]);
        last = best;
        if (threadIdx.x == 0) {
            const uint32_t id = 0xffffffffu - (uint32_t)best;
            if (a.id_bytes == 4) static_cast<int32_t *>(a.top_ids)[row * a.top + k] = (int32_t)id;
            else static_cast<long long *>(a.top_ids)[row * a.top + k] = (long long)id;
            a.top_logp[row * a.top + k] = nothing ? -INFINITY : kLn2 * ((key_value(best) - r.base) * c - log_sum);
        }
    }
}

// A tile of a row a block.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) cr_token_log_probs_grad_kernel(const VocabArgs a, unsigned tiles) {
    constexpr int kUnroll = 4;
    const int64_t row = blockIdx.x / tiles, first = (int64_t)(blockIdx.x % tiles) * kThreads * kUnroll;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    T *d = static_cast<T *>(a.dlogits) + row * a.ld_d;
    const int64_t nvec = a.vocab / VEC;
    const float c = a.inverse * kLog2e;
    const float m = a.stats[2 * row], base = isinf(m) ? 0.f : m, log_sum = a.stats[2 * row + 1] * kLog2e;
    int64_t id = a.dlogp ? id_at(a.ids, a.id_bytes, row) : -1;
    if (id < 0 || id >= a.vocab) id = -1;
    const float ga = id >= 0 ? a.dlogp[row] * a.inverse : 0.f, gb = a.dentropy ? a.dentropy[row] * a.inverse : 0.f;
    const bool none = (ga == 0.f && gb == 0.f) || m == -INFINITY;
    const float level = gb != 0.f ? fmaf(gb, a.entropy[row], ga) : ga, turn = gb * kLn2;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int64_t v = first + u * kThreads + (int)threadIdx.x;
        if (v >= nvec) break;
        float f[VEC] = {};
        if (!none) {
            unpack<T, VEC>(load_packed<T, VEC>(x + v * VEC), f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float w = max_nan((f[i] - base) * c - log_sum, kLeast);     // log2 p
                f[i] = (v * VEC + i == id ? ga : 0.f) - exp2_approx(w) * fmaf(turn, w, level);
            }
        }
        store_packed<T, VEC>(d + v * VEC, pack<T, VEC>(f));
    }
}

// ---- distillation --------------------------------------------------------------------------------------------------------

constexpr int kMostTop = 1024;

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) cr_distill_kernel(const VocabArgs a) {
    __shared__ float sm[kThreads / 32];
    __shared__ float share[kMostTop], logit[kMostTop];
    __shared__ int32_t named[kMostTop];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    T *d = a.dlogits ? static_cast<T *>(a.dlogits) + row * a.ld_d : nullptr;
    const float c = a.inverse * kLog2e;
    const float w = a.weight ? a.weight[row] : 1.f;
    // the teacher
    float best = -INFINITY;
    for (int j = threadIdx.x; j < a.top; j += kThreads) {
        const int64_t id = id_at(a.ids, a.id_bytes, row * a.top + j);
        const bool there = id >= 0 && id < a.vocab;
        named[j] = there ? (int32_t)id : -1;
        logit[j] = there ? to_float(x[id]) : 0.f;
        share[j] = there ? a.teacher[row * a.top + j] * c : -INFINITY;
        best = max_nan(best, share[j]);
    }
    best = block_reduce(best, sm, max_nan);
    const bool left_out = best == -INFINITY;
    float mass = 0.f;
    for (int j = threadIdx.x; j < a.top; j += kThreads) mass += exp2_approx(share[j] - best);
    mass = block_reduce(mass, sm, add);
    RowStats r = {0.f, 0.f, 1.f, 0.f};
    if (!left_out && (a.loss || (d && w != 0.f))) r = row_stats<T, VEC>(x, a.vocab, c, sm);
    const float log_sum = log2f(r.sum), log_mass = log2f(mass);
    float loss = 0.f;
    for (int j = threadIdx.x; j < a.top; j += kThreads) {
        const float u = share[j] - best, p = left_out ? 0.f : exp2_approx(u) / mass;
        share[j] = p;
        if (p != 0.f) loss += p * ((u - log_mass) - (r.sum == 0.f ? -INFINITY : (logit[j] - r.base) * c - log_sum));
    }
    loss = block_reduce(loss, sm, add);
    if (threadIdx.x == 0 && a.loss) a.loss[row] = left_out ? 0.f : a.temperature * a.temperature * kLn2 * loss;
    if (!d) return;
    const int64_t nvec = a.vocab / VEC;
    const bool none = left_out || w == 0.f;
    const float scale = w * a.temperature, factor = r.sum == 0.f ? 0.f : scale / r.sum;
    for (int64_t v = threadIdx.x; v < nvec; v += kThreads) {
        float f[VEC] = {};
        if (!none) {
            unpack<T, VEC>(load_packed<T, VEC>(x + v * VEC), f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = exp2_approx((f[i] - r.base) * c) * factor;
        }
        store_packed<T, VEC>(d + v * VEC, pack<T, VEC>(f));
    }
    if (none) return;
    __syncthreads();
    for (int j = threadIdx.x; j < a.top; j += kThreads) {
        if (named[j] < 0) continue;
        float p = 0.f;     // a token may be named more than once
        for (int i = 0; i < a.top; ++i) p += named[i] == named[j] ? share[i] : 0.f;
        d[named[j]] = from_float<T>(fmaf(exp2_approx((logit[j] - r.base) * c), factor, -scale * p));
    }
}

template <typename F>
cudaError_t by_form(const VocabArgs &a, F &&f) {
    return by_type(a.elem, [&](auto t) {
        constexpr int VEC = 16 / (int)sizeof(t);
        if (vector_rows(a.elem, a.vocab, {a.logits, a.dlogits}, {a.ld, a.dlogits ? a.ld_d : 0})) return f(t, Int<VEC>{});
        return f(t, Int<1>{});
    });
}

}  // namespace

cudaError_t launch_token_log_probs(const VocabArgs &a, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    return by_form(a, [&](auto t, auto v) {
        cr_token_log_probs_kernel<decltype(t), decltype(v)::value><<<(unsigned)a.rows, kThreads, 0, stream>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

cudaError_t launch_token_log_probs_backward(const VocabArgs &a, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    return by_form(a, [&](auto t, auto v) {
        const int64_t nvec = a.vocab / decltype(v)::value, tiles = (nvec + kThreads * 4 - 1) / (kThreads * 4);
        if (a.rows > 0x7fffffffll / tiles) return cudaErrorInvalidValue;
        cr_token_log_probs_grad_kernel<decltype(t), decltype(v)::value><<<(unsigned)(a.rows * tiles), kThreads, 0, stream>>>(a, (unsigned)tiles);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

cudaError_t launch_distill(const VocabArgs &a, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    return by_form(a, [&](auto t, auto v) {
        cr_distill_kernel<decltype(t), decltype(v)::value><<<(unsigned)a.rows, kThreads, 0, stream>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

}  // namespace cr
