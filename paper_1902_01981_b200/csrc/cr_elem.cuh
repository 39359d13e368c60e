// Vectors of 32-, bf16- and f16-elements, and the counter-based generator of the dropout masks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "cr_layers.hpp"

namespace cr {

// `VEC` consecutive elements as they lie in memory: 16 bytes, or one element.
template <typename T, int VEC>
struct Packed {
    static constexpr int kWords = VEC * (int)sizeof(T) / 4;
    uint32_t w[kWords];
};
template <typename T>
struct Packed<T, 1> {
    T e;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// A difference that cannot be negative but for rounding.  A NaN stays one (a maximum with zero would hide it).
__device__ __forceinline__ float not_below_zero(float v) { return v < 0.f ? 0.f : v; }

// Ordinary accesses, which the compiler may move past one another: an output may be the input's own buffer, so nothing
// goes through the read-only path.
template <typename T, int VEC>
__device__ __forceinline__ Packed<T, VEC> load_packed(const T *p) {
    Packed<T, VEC> r;
    if constexpr (VEC == 1) {
        r.e = *p;
    } else {
        static_assert(sizeof(r) == 16, "a vector is 16 bytes");
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    }
    return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_packed(T *p, const Packed<T, VEC> &r) {
    if constexpr (VEC == 1) *p = r.e;
    else *reinterpret_cast<uint4 *>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
}
template <typename T, int VEC>
__device__ __forceinline__ void unpack(const Packed<T, VEC> &r, float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        v[0] = to_float(r.e);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (__is_same(T, __nv_bfloat16)) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&r.w[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}
template <typename T, int VEC>
__device__ __forceinline__ Packed<T, VEC> pack(const float (&v)[VEC]) {
    Packed<T, VEC> r;
    if constexpr (VEC == 1) {
        r.e = from_float<T>(v[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) r.w[i] = __float_as_uint(v[i]);
    } else if constexpr (__is_same(T, __nv_bfloat16)) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            r.w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
            r.w[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
    return r;
}

// ---- the generator -------------------------------------------------------------------------------
//
// SplitMix64 (Steele, Lea, Flood, "Fast splittable pseudorandom number generators", 2014) read by index: the i-th
// output of the stream that starts at `key` is a function of key and i alone, so every element's number can be had
// anywhere, in any order, and no mask is stored.  One 64-bit output serves four consecutive elements with 16 bits each
// (the lowest bits the first).  About 20 integer instructions per output, 5 per element: under the time the element's
// bytes take from HBM, which a cipher-like generator with its ten rounds would not be.

constexpr unsigned long long kMixGamma = 0x9E3779B97F4A7C15ull;
__host__ __device__ __forceinline__ unsigned long long mix64(unsigned long long z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
__device__ __forceinline__ unsigned long long drop_word(unsigned long long key, unsigned long long i) {
    return mix64(key + (i + 1) * kMixGamma);
}

// v[i] = kept ? v[i] : 0 for the VEC elements from index e on; the scale is left to the caller.  A dropped element is
// selected away, not multiplied by zero: an infinity or a NaN in its place leaves a zero.
template <int VEC>
__device__ __forceinline__ void drop_select(float (&v)[VEC], const DropSpec &d, unsigned long long e) {
    const unsigned long long first = e >> 2;
    const uint32_t shift = (uint32_t)e & 3u;
    if (d.scale == 0.f) {   // threshold 65536: everything goes
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = 0.f;
        return;
    }
    const uint32_t limit = d.threshold << 16;
    if constexpr (VEC == 1) {
        const uint32_t lane = (uint32_t)(drop_word(d.key, first) >> (16 * shift)) & 0xffffu;
        v[0] = lane >= d.threshold ? v[0] : 0.f;
    } else {
        // z of output `first`; the following ones are one addition away
        unsigned long long z = d.key + (first + 1) * kMixGamma;
        uint32_t w[VEC / 2 + 2];
#pragma unroll
        for (int j = 0; j < VEC / 4; ++j, z += kMixGamma) {
            const unsigned long long o = mix64(z);
            w[2 * j] = (uint32_t)o;
            w[2 * j + 1] = (uint32_t)(o >> 32);
        }
        if (shift) {   // the vector straddles one output more: move its 16-bit numbers into place
            const unsigned long long o = mix64(z);
            w[VEC / 2] = (uint32_t)o;
            w[VEC / 2 + 1] = (uint32_t)(o >> 32);
            const bool whole = shift & 2u;
#pragma unroll
            for (int j = 0; j <= VEC / 2; ++j) w[j] = whole ? w[j + 1] : w[j];
            const uint32_t bits = (shift & 1u) * 16u;
#pragma unroll
            for (int j = 0; j < VEC / 2; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], bits);
        }
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
            v[2 * j] = (w[j] << 16) >= limit ? v[2 * j] : 0.f;
            v[2 * j + 1] = w[j] >= limit ? v[2 * j + 1] : 0.f;   // the low half cannot lift it over the limit
        }
    }
}
template <int VEC>
__device__ __forceinline__ void drop(float (&v)[VEC], const DropSpec &d, unsigned long long e) {
    drop_select<VEC>(v, d, e);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] *= d.scale;
}

// ---- pairs -------------------------------------------------------------------------------------------
//
// Two fp32 operations in one instruction (add, mul, fma .f32x2): half the issue slots of the element-wise arithmetic.  A
// pair is kept as one 64-bit value, so that it stays in an aligned register pair between operations.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 f2(float x, float y) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(x, x); }
__device__ __forceinline__ float low(F2 a) { return __uint_as_float((uint32_t)a.v); }
__device__ __forceinline__ float high(F2 a) { return __uint_as_float((uint32_t)(a.v >> 32)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// Elements as pairs.
template <typename T, int VEC>
__device__ __forceinline__ void unpack2(const Packed<T, VEC> &r, F2 (&v)[VEC / 2]) {
    float f[VEC];
    unpack<T, VEC>(r, f);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
}
template <typename T, int VEC>
__device__ __forceinline__ Packed<T, VEC> pack2(const F2 (&v)[VEC / 2]) {
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) { f[2 * i] = low(v[i]); f[2 * i + 1] = high(v[i]); }
    return pack<T, VEC>(f);
}

template <int VEC>
__device__ __forceinline__ void drop_select2(F2 (&v)[VEC / 2], const DropSpec &d, unsigned long long e) {
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) { f[2 * i] = low(v[i]); f[2 * i + 1] = high(v[i]); }
    drop_select<VEC>(f, d, e);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
}

// ---- activations -----------------------------------------------------------------------------------
//
// 2^t and 1 / t to about one unit in the last place, subnormal numbers as zero: e^-z then leaves the range at
// |z| = 87, where the sigmoid has long become 0 or 1.  t = -z log2(e) is rounded, so e^-z carries a relative error of about
// |z| 2^-24 besides (silu measured: 2e-7 at z = -5, 9e-7 at -20, 4e-6 at -80), in a tail whose value is |z| e^-|z|: against
// the other outputs of a call it is far below their own rounding.
__device__ __forceinline__ float exp2_approx(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float recip_approx(float t) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float sigmoid(float z) { return recip_approx(1.f + exp2_approx(-kLog2e * z)); }

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;   // a NaN stays one
    if constexpr (ACT == kActSilu) return z * sigmoid(z);
    return z;
}
// dy times the derivative of the activation at z.  Where relu is off the gradient is selected away, not multiplied by zero:
// an infinity or a NaN in dy there leaves a zero.
template <int ACT>
__device__ __forceinline__ float act_gradient(float dy, float z) {
    if constexpr (ACT == kActRelu) return z > 0.f ? dy : 0.f;
    if constexpr (ACT == kActSilu) {
        const float s = sigmoid(z);
        return dy * (s * fmaf(z, 1.f - s, 1.f));
    }
    return dy;
}

}  // namespace cr
