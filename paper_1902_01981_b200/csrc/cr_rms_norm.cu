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

// A row is cut into pieces that a warp takes at once: kHeld vectors (or elements, where rows do not lie in vectors) a lane, a
// warp's width apart, so that the addresses differ by constants.
template <int VEC> __host__ __device__ constexpr int held_vectors() { return VEC == 1 ? 16 : 4; }
template <typename T, int VEC>
struct RowPiece {
    static constexpr int kHeld = held_vectors<VEC>();
    float f[kHeld][VEC];

    // Vectors of this lane of piece `piece` that lie in a row of nvec.
    static __device__ __forceinline__ int have(int64_t piece, int64_t nvec) {
        const int64_t left = nvec - piece * kHeld * 32 - (int)threadIdx.x % 32;
        return left >= (kHeld - 1) * 32 + 1 ? kHeld : left <= 0 ? 0 : (int)(left + 31) / 32;
    }
    static __device__ __forceinline__ int64_t offset(int64_t piece) { return (piece * kHeld * 32 + (int)threadIdx.x % 32) * VEC; }

    // x + r of the piece; zeros where there is no more row.  x and r point at the lane's first vector.
    __device__ __forceinline__ void load(const T *x, const T *r, int n) {
        Packed<T, VEC> px[kHeld], pr[kHeld];
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (n == kHeld || u < n) px[u] = load_packed<T, VEC>(x + u * 32 * VEC);
        if (r) {
#pragma unroll
            for (int u = 0; u < kHeld; ++u)
                if (n == kHeld || u < n) pr[u] = load_packed<T, VEC>(r + u * 32 * VEC);
        }
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            const bool in = n == kHeld || u < n;
            float g[VEC];
            unpack<T, VEC>(px[u], f[u]);
            if (r) unpack<T, VEC>(pr[u], g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[u][i] = in ? (r ? f[u][i] + g[i] : f[u][i]) : 0.f;
        }
    }
    __device__ __forceinline__ float squares() const {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s = fmaf(f[u][i], f[u][i], s);
        return s;
    }
    __device__ __forceinline__ void store(T *p, int n) const {
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (n == kHeld || u < n) store_packed<T, VEC>(p + u * 32 * VEC, pack<T, VEC>(f[u]));
    }
    // The sums times rstd and gamma.
    __device__ __forceinline__ void norm(const float *gamma, float rstd, int n) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            float g[VEC];
            if (gamma && (n == kHeld || u < n)) load_floats<VEC>(gamma + u * 32 * VEC, g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[u][i] = f[u][i] * rstd * (gamma ? g[i] : 1.f);
        }
    }
    __device__ __forceinline__ uint32_t largest(int n) const {
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (n == kHeld || u < n) top = max(top, __float_as_uint(f[u][i]) & 0x7fffffffu);
        return top;
    }
    __device__ __forceinline__ void store_codes(int8_t *q, float mult, bool dead, int n) const {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (n != kHeld && u >= n) continue;
            if constexpr (VEC == 1) {
                q[u * 32] = dead ? (int8_t)0 : (int8_t)code(f[u][0], mult);
            } else {
                uint32_t w[VEC / 4];
#pragma unroll
                for (int i = 0; i < VEC / 4; ++i) {
                    const uint32_t lo = __byte_perm(code(f[u][4 * i], mult), code(f[u][4 * i + 1], mult), 0x0040);
                    const uint32_t hi = __byte_perm(code(f[u][4 * i + 2], mult), code(f[u][4 * i + 3], mult), 0x0040);
                    w[i] = dead ? 0u : __byte_perm(lo, hi, 0x5410);
                }
                if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(q + u * 32 * 8) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t *>(q + u * 32 * 4) = w[0];
            }
        }
    }
};

// One block a row.  A warp's piece stays in registers between the statistics and the output; rows of more pieces than a block
// has warps (LONG) are read again for each (from L2).  Everything is read before the block's first barrier or by the thread
// that writes it, so outputs may be the inputs' own buffers.  Bound by memory: 16384 x 4096 bf16 with residual into codes, 470 MB, 70 us
// (6.7 TB/s); 8192 x 4096 fp32 81 us (6.6 TB/s); 16-bit elements in odd rows about half of that.
constexpr int kRowWarps = 16;
template <typename T, int VEC, bool CODES, bool LONG>
__global__ void __launch_bounds__(32 * kRowWarps) cr_rms_norm_kernel(const RmsNormArgs a) {
    using P = RowPiece<T, VEC>;
    __shared__ float sums[32];
    __shared__ uint32_t tops[32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ld_residual : nullptr;
    T *h = a.h ? static_cast<T *>(a.h) + row * a.ld_h : nullptr;
    const int64_t nvec = a.cols / VEC, pieces = (nvec + P::kHeld * 32 - 1) / (P::kHeld * 32);
    const int warps = (int)blockDim.x / 32, warp = (int)threadIdx.x / 32;
    P p;
    auto load = [&](int64_t piece) { p.load(x + P::offset(piece), r ? r + P::offset(piece) : nullptr, P::have(piece, nvec)); };
    // f(piece) for the warp's pieces
    auto each = [&](auto &&f) {
        if constexpr (LONG)
            for (int64_t piece = warp; piece < pieces; piece += warps) f(piece);
        else
            f((int64_t)warp);
    };
    float squares = 0.f;
    each([&](int64_t piece) {
        load(piece);
        squares += p.squares();
    });
    const float rstd = 1.f / sqrtf(block_sum(squares, sums) / (float)a.cols + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    // y of the piece in the place of the sums, which are stored
    auto norm = [&](int64_t piece, bool store) {
        const int n = P::have(piece, nvec);
        if (store && h) p.store(h + P::offset(piece), n);
        p.norm(a.gamma ? a.gamma + P::offset(piece) : nullptr, rstd, n);
    };
    if constexpr (CODES) {
        uint32_t top = 0;
        each([&](int64_t piece) {
            if constexpr (LONG) load(piece);
            norm(piece, !LONG);
            top = max(top, p.largest(P::have(piece, nvec)));
        });
        top = block_max(top, tops);
        const RowScale rs = row_scale(top);
        const bool dead = top >= 0x7f800000u;      // an infinity or a NaN: codes 0
        if (threadIdx.x == 0) a.scale[row] = rs.scale;
        int8_t *q = a.q + row * a.ld_q;
        each([&](int64_t piece) {
            if constexpr (LONG) {
                load(piece);
                norm(piece, true);
            }
            p.store_codes(q + P::offset(piece), rs.mult, dead, P::have(piece, nvec));
        });
    } else {
        T *y = static_cast<T *>(a.y) + row * a.ld_y;
        each([&](int64_t piece) {
            if constexpr (LONG) load(piece);
            norm(piece, true);
            p.store(y + P::offset(piece), P::have(piece, nvec));
        });
    }
}

// ---- gradient ------------------------------------------------------------------------------------------------------------

// Rows of a partition that one block adds up: 4 to 64, so that up to 16384 rows make 256 chunks at most; longer partitions have
// a chunk for every 64 rows (a longer chain in the sums of the chunks: an eighth of them, one after the other).
int64_t chunk_rows(int64_t rows) { return std::min<int64_t>(64, std::max<int64_t>(4, (rows + 255) / 256)); }

// One block a chunk of rows: a thread keeps its columns' gamma and sums of dy xhat in registers over the rows.  Rows of up to
// grad_held vectors a thread.  Each thread copies its own vectors of the rows to come into shared memory
// (cp.async, four rows ahead, two of fp32; no barrier, since nobody else reads them); elements that do not lie in vectors are
// fetched a row ahead into registers.  Bound by memory: 16384 x 4096 bf16 with the stream's gradient, 537 MB, 88 us (6.1 TB/s); rows
// fetched one ahead into registers 119 us (16 warps an SM cannot ask for enough), three blocks an SM with 80 registers 117.
template <int VEC> __host__ __device__ constexpr int grad_threads() { return VEC == 1 ? 1024 : 512; }
template <int VEC> __host__ __device__ constexpr int grad_stages() { return VEC == 1 ? 1 : VEC == 4 ? 2 : 4; }
template <int VEC> __host__ __device__ constexpr int grad_held() { return VEC == 8 ? 2 : 4; }
template <int VEC> __host__ __device__ constexpr int64_t grad_held_cols() { return (int64_t)grad_threads<VEC>() * grad_held<VEC>() * VEC; }

template <typename T, int VEC>
struct RowsAhead {
    static constexpr int kHeld = grad_held<VEC>();
    uint4 *mine;                                // this thread's first slot; slots are a block apart
    Packed<T, VEC> next[VEC == 1 ? 3 * kHeld : 1];

    // Asks for tensor t's vectors of a row: `have` of them, a warp's width apart.
    __device__ __forceinline__ void fetch(int stage, int t, const T *row, int have) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u >= have) continue;
            if constexpr (VEC == 1) {
                next[t * kHeld + u] = load_packed<T, 1>(row + u * 32);
            } else {
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine + ((stage * 3 + t) * kHeld + u) * blockDim.x);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + u * 32 * VEC) : "memory");
            }
        }
    }
    __device__ __forceinline__ void asked() const {
        if constexpr (VEC > 1) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // Waits for all but the latest grad_stages - 1 rows asked for.
    __device__ __forceinline__ void arrived() const {
        if constexpr (VEC > 1) asm volatile("cp.async.wait_group %0;" ::"n"(grad_stages<VEC>() - 1) : "memory");
    }
    __device__ __forceinline__ void take(int stage, int t, int u, float (&f)[VEC]) const {
        if constexpr (VEC == 1) {
            unpack<T, 1>(next[t * kHeld + u], f);
        } else {
            const uint4 q = mine[((stage * 3 + t) * kHeld + u) * blockDim.x];
            Packed<T, VEC> p;
            p.w[0] = q.x; p.w[1] = q.y; p.w[2] = q.z; p.w[3] = q.w;
            unpack<T, VEC>(p, f);
        }
    }
};

template <typename T, int VEC, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 2 : 1) cr_rms_norm_grad_rows_kernel(const RmsNormArgs a, float *partial, int64_t ld_partial, int64_t rows_each,
                                                                             int chunk, int chunks) {
    constexpr int kHeld = grad_held<VEC>(), kAhead = grad_stages<VEC>();
    extern __shared__ uint4 staged[];
    __shared__ float sums[2][32];
    let_next_begin();
    const int64_t part = blockIdx.x / (unsigned)chunks, first = (int64_t)(blockIdx.x % (unsigned)chunks) * chunk;
    const int count = (int)min((int64_t)chunk, rows_each - first);
    const int64_t row0 = part * rows_each + first;
    const int lane = (int)threadIdx.x % 32, v0 = (int)(threadIdx.x / 32) * kHeld * 32 + lane;      // this thread's first vector
    const int left = (int)(a.cols / VEC) - v0, have = left <= 0 ? 0 : min(kHeld, (left + 31) / 32), col = v0 * VEC;
    const T *dh = static_cast<const T *>(a.dh);
    T *dx = static_cast<T *>(a.y);
    const float over = 1.f / (float)a.cols;
    RowsAhead<T, VEC> ahead;
    ahead.mine = staged + threadIdx.x;
    auto fetch = [&](int k) {
        const int64_t row = row0 + k;
        const int stage = k % kAhead;
        if (k < count) {
            ahead.fetch(stage, 0, static_cast<const T *>(a.dy) + row * a.ld_dy + col, have);
            ahead.fetch(stage, 1, static_cast<const T *>(a.h) + row * a.ld_h + col, have);
            if (dh) ahead.fetch(stage, 2, dh + row * a.ld_dh + col, have);
        }
        ahead.asked();
    };
    for (int k = 0; k < kAhead; ++k) fetch(k);
    float w[kHeld][VEC], acc[kHeld][VEC] = {};
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[u][i] = 1.f;
        if (a.gamma && u < have) load_floats<VEC>(a.gamma + col + u * 32 * VEC, w[u]);
    }
    float rstd_ahead = a.rstd[row0];
    for (int k = 0; k < count; ++k) {
        const float rstd = rstd_ahead;
        if (k + 1 < count) rstd_ahead = a.rstd[row0 + k + 1];
        float fg[kHeld][VEC], fx[kHeld][VEC], d[kHeld][VEC] = {}, dot = 0.f;
        ahead.arrived();
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u >= have) continue;
            ahead.take(k % kAhead, 0, u, fg[u]);
            ahead.take(k % kAhead, 1, u, fx[u]);
            if (dh && VEC == 1) ahead.take(k % kAhead, 2, u, d[u]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                fx[u][i] *= rstd;
                acc[u][i] = fmaf(fg[u][i], fx[u][i], acc[u][i]);
                fg[u][i] *= w[u][i];
                dot = fmaf(fg[u][i], fx[u][i], dot);
            }
        }
        // a row's dx may be its own dy, h or dh, which have arrived by now; the rows asked for are not written yet
        if (VEC == 1) fetch(k + 1);
        if (dx) {
            dot = block_sum(dot, sums[k & 1]) * over;
#pragma unroll
            for (int u = 0; u < kHeld; ++u) {
                if (u >= have) continue;
                if (dh && VEC > 1) ahead.take(k % kAhead, 2, u, d[u]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) d[u][i] = fmaf(rstd, fmaf(-fx[u][i], dot, fg[u][i]), d[u][i]);
                store_packed<T, VEC>(dx + (row0 + k) * a.ld_y + col + u * 32 * VEC, pack<T, VEC>(d[u]));
            }
        }
        if (VEC > 1) fetch(k + kAhead);       // into the slots just read
    }
    if (!partial) return;
    float *out = partial + blockIdx.x * ld_partial + col;
    const bool aligned = VEC > 1 && ld_partial % 4 == 0 && (reinterpret_cast<uintptr_t>(partial) & 15u) == 0;
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
        if (u >= have) continue;
        if (aligned) {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) *reinterpret_cast<float4 *>(out + u * 32 * VEC + i) = make_float4(acc[u][i], acc[u][i + 1 < VEC ? i + 1 : 0], acc[u][i + 2 < VEC ? i + 2 : 0], acc[u][i + 3 < VEC ? i + 3 : 0]);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) out[u * 32 * VEC + i] = acc[u][i];
        }
    }
}

// Longer rows in two kernels.  The first leaves a row's (sum g xhat) / C.
constexpr int kDotWarps = 8;
template <typename T, int VEC>
__global__ void __launch_bounds__(32 * kDotWarps, 3) cr_rms_norm_dots_kernel(const RmsNormArgs a, float *dots) {
    using P = RowPiece<T, VEC>;
    __shared__ float sums[32];
    let_next_begin();
    const int64_t row = blockIdx.x;
    const T *dy = static_cast<const T *>(a.dy) + row * a.ld_dy, *h = static_cast<const T *>(a.h) + row * a.ld_h;
    const int64_t nvec = a.cols / VEC, pieces = (nvec + P::kHeld * 32 - 1) / (P::kHeld * 32);
    float dot = 0.f;
    for (int64_t piece = threadIdx.x / 32; piece < pieces; piece += blockDim.x / 32) {
        const int n = P::have(piece, nvec);
        const int64_t o = P::offset(piece);
        P g, x;
        x.load(h + o, nullptr, n);
        g.load(dy + o, nullptr, n);
        g.norm(a.gamma ? a.gamma + o : nullptr, 1.f, n);
#pragma unroll
        for (int u = 0; u < P::kHeld; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (n == P::kHeld || u < n) dot = fmaf(g.f[u][i], x.f[u][i], dot);
    }
    dot = block_sum(dot, sums);
    if (threadIdx.x == 0) dots[row] = dot * a.rstd[row] / (float)a.cols;
}

// The second one dx of a chunk of rows for a slab of columns, and the chunk's sums of dy xhat.  A thread takes slab_held vectors
// of columns, a warp's width apart, and asks for the next row's before it writes this row's dx.
constexpr int kSlabThreads = 128;
template <int VEC> __host__ __device__ constexpr int slab_held() { return VEC == 1 ? 4 : 1; }
template <typename T, int VEC>
__global__ void __launch_bounds__(kSlabThreads) cr_rms_norm_grad_kernel(const RmsNormArgs a, const float *dots, float *partial, int64_t ld_partial,
                                                                        int64_t rows_each, int chunk, int chunks, int slabs) {
    constexpr int kHeld = slab_held<VEC>();
    let_next_begin();
    if (dots) wait_for_previous();       // null: no dx is wanted, and nothing was launched before
    const unsigned item = blockIdx.x / (unsigned)slabs;
    const int lane = (int)threadIdx.x % 32;
    const int64_t v0 = ((int64_t)(blockIdx.x % (unsigned)slabs) * kSlabThreads + threadIdx.x / 32 * 32) * kHeld + lane, left = a.cols / VEC - v0;
    const int64_t part = item / (unsigned)chunks, c = item % (unsigned)chunks;
    if (left <= 0) return;
    const int have = (int)min((int64_t)kHeld, (left + 31) / 32);
    const int64_t first = c * chunk, col = v0 * VEC;
    const int count = (int)min((int64_t)chunk, rows_each - first);
    const int64_t row0 = part * rows_each + first;
    const bool stream = a.y && a.dh;
    float w[kHeld][VEC], acc[kHeld][VEC] = {};
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[u][i] = 1.f;
        if (a.gamma && u < have) load_floats<VEC>(a.gamma + col + u * 32 * VEC, w[u]);
    }
    Packed<T, VEC> g[kHeld], x[kHeld], s[kHeld];
    float rstd = 0.f, dot = 0.f;
    auto fetch = [&](int k) {
        const int64_t row = row0 + k;
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u >= have) continue;
            g[u] = load_packed<T, VEC>(static_cast<const T *>(a.dy) + row * a.ld_dy + col + u * 32 * VEC);
            x[u] = load_packed<T, VEC>(static_cast<const T *>(a.h) + row * a.ld_h + col + u * 32 * VEC);
            if (stream) s[u] = load_packed<T, VEC>(static_cast<const T *>(a.dh) + row * a.ld_dh + col + u * 32 * VEC);
        }
        rstd = a.rstd[row];
        if (a.y) dot = dots[row];
    };
    fetch(0);
    for (int k = 0; k < count; ++k) {
        Packed<T, VEC> out[kHeld];
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u >= have) continue;
            float fg[VEC], fx[VEC], d[VEC] = {};
            unpack<T, VEC>(g[u], fg);
            unpack<T, VEC>(x[u], fx);
            if (stream) unpack<T, VEC>(s[u], d);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xhat = fx[i] * rstd;
                acc[u][i] = fmaf(fg[i], xhat, acc[u][i]);
                d[i] = fmaf(rstd, fmaf(-xhat, dot, fg[i] * w[u][i]), d[i]);
            }
            out[u] = pack<T, VEC>(d);
        }
        // a row's dx may be its own dy, h or dh: the next row is another one
        if (k + 1 < count) fetch(k + 1);
        if (!a.y) continue;
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (u < have) store_packed<T, VEC>(static_cast<T *>(a.y) + (row0 + k) * a.ld_y + col + u * 32 * VEC, out[u]);
    }
    if (!partial) return;
    float *sums = partial + item * ld_partial + col;
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (u < have) sums[u * 32 * VEC + i] = acc[u][i];
}

// dgamma of a partition from its chunks' sums: eight warps take every eighth chunk and are summed in order.
__global__ void __launch_bounds__(256) cr_rms_norm_params_kernel(const float *partial, int chunks, int64_t cols, float *dgamma, int64_t ld, unsigned slabs) {
    __shared__ float sm[8][32];
    wait_for_previous();
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
            constexpr bool kCodes = decltype(codes)::value != 0;
            const int64_t pieces = (a.cols / V + held_vectors<V>() * 32 - 1) / (held_vectors<V>() * 32);
            if (pieces <= kRowWarps) cr_rms_norm_kernel<T, V, kCodes, false><<<(unsigned)a.rows, 32 * (unsigned)pieces, 0, stream>>>(a);
            else cr_rms_norm_kernel<T, V, kCodes, true><<<(unsigned)a.rows, 32 * (unsigned)kRowWarps, 0, stream>>>(a);
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
            float *sums = !a.dgamma ? nullptr : chunks > 1 ? partial : a.dgamma;
            const int64_t ld_sums = chunks > 1 ? a.cols : a.ld_gamma;
            if (a.cols <= grad_held_cols<V>()) {
                if (a.partitions * chunks > 0x7fffffffll) return cudaErrorInvalidValue;
                const int64_t nvec = a.cols / V, held = grad_held<V>();
                const int threads = (int)std::max<int64_t>(32, (nvec + held * 32 - 1) / (held * 32) * 32);
                const size_t smem = V == 1 ? 0 : (size_t)grad_stages<V>() * 3 * held * threads * 16;
                auto kernel = threads <= 256 ? cr_rms_norm_grad_rows_kernel<T, V, 256> : cr_rms_norm_grad_rows_kernel<T, V, grad_threads<V>()>;
                if (smem > 32 * 1024) {       // 48 KB without asking, of which the block's sums take some
                    static std::atomic<uint64_t> told[2] = {};     // one for each of the two kernels
                    const cudaError_t e = allow_most_smem(reinterpret_cast<const void *>(kernel), told[threads <= 256]);
                    if (e != cudaSuccess) return e;
                }
                kernel<<<(unsigned)(a.partitions * chunks), threads, smem, stream>>>(a, sums, ld_sums, each, chunk, chunks);
                const cudaError_t e = cudaGetLastError();
                if (e == cudaSuccess) ++*launches;
                return e;
            }
            if (a.y) {
                cr_rms_norm_dots_kernel<T, V><<<(unsigned)a.rows, 32 * kDotWarps, 0, stream>>>(a, dots);
                const cudaError_t e = cudaGetLastError();
                if (e != cudaSuccess) return e;
                ++*launches;
            }
            const int64_t slab = kSlabThreads * slab_held<V>(), slabs = (a.cols / V + slab - 1) / slab;
            if (a.partitions * chunks > 0x7fffffffll / slabs) return cudaErrorInvalidValue;
            const unsigned blocks = (unsigned)(a.partitions * chunks * slabs);
            cudaError_t e;
            if (a.y) {
                e = launch_next(cr_rms_norm_grad_kernel<T, V>, blocks, kSlabThreads, stream, a, dots, sums, ld_sums, each, chunk, chunks, (int)slabs);
            } else {
                cr_rms_norm_grad_kernel<T, V><<<blocks, kSlabThreads, 0, stream>>>(a, nullptr, sums, ld_sums, each, chunk, chunks, (int)slabs);
                e = cudaGetLastError();
            }
            if (e == cudaSuccess) ++*launches;
            return e;
        };
        return wide ? go(Int<VEC>{}) : go(Int<1>{});
    });
    if (e != cudaSuccess || !a.dgamma || chunks == 1) return e;
    const int64_t slabs = (a.cols + 31) / 32;
    if (a.partitions > 0x7fffffffll / slabs) return cudaErrorInvalidValue;
    e = launch_next(cr_rms_norm_params_kernel, (unsigned)(a.partitions * slabs), 256, stream, partial, chunks, a.cols, a.dgamma, a.ld_gamma, (unsigned)slabs);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cr
