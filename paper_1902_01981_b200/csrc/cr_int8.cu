// Products of 8-bit integer matrices with a scale for each token and each channel, and the quantiser of tokens:
//   s_t = max_k |x_tk| / 127,  q_tk = rint(x_tk * (127 / max_k |x_tk|)),
//   y_tn = (sum_k q_tk w_nk) * (s_t s_n) + bias_n.
// The sum is taken in 32-bit integers (|sum| <= 2^14 k: exact for every k the entry point takes), so it has no order
// and no rounding: the tiles, the split over k and the machine do not show in the result.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "cr_elem.cuh"
#include "cr_tcgen05.cuh"

namespace cr {
namespace {

// ---- quantiser ------------------------------------------------------------------------------------------------------

// The largest magnitude of a vector, as the bits of a float.  Magnitudes are compared as integers: the order is the same,
// and a NaN is larger than everything.  16-bit elements are compared two at a time.
template <typename T, int VEC>
__device__ __forceinline__ uint32_t largest(const Packed<T, VEC> &pv, uint32_t top) {
    if constexpr (VEC == 1) {
        return max(top, __float_as_uint(to_float(pv.e)) & 0x7fffffffu);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = max(top, pv.w[i] & 0x7fffffffu);
        return top;
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) top = __vmaxu2(top, pv.w[i] & 0x7fff7fffu);
        return top;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ uint32_t float_bits(uint32_t top) {
    if constexpr (VEC == 1 || sizeof(T) == 4) {
        return top;
    } else {
        const unsigned short h = (unsigned short)max(top & 0xffffu, top >> 16);
        if constexpr (__is_same(T, __nv_bfloat16)) return (uint32_t)h << 16;
        else return __float_as_uint(__half2float(__ushort_as_half(h)));
    }
}

// One block per row.  The row's first kHeld vectors of each thread stay in registers between the search for the
// largest magnitude and the rounding; longer rows are read a second time (from L2).  Bound by memory: 16384 rows of 4096
// bf16, 201 MB, 31.5 us (6.4 TB/s); with clamped conversions (cvt and two comparisons an element) 42 us.
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
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) held[u] = load_packed<T, VEC>(row + (int64_t)(tid + u * nt) * VEC);
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) top = largest<T, VEC>(held[u], top);
    for (int64_t v = tid + kHeld * nt; v < nvec; v += nt) top = largest<T, VEC>(load_packed<T, VEC>(row + v * VEC), top);
    top = float_bits<T, VEC>(top);
    for (int64_t c = nvec * VEC + tid; c < cols; c += nt) top = max(top, __float_as_uint(to_float(row[c])) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if (nt > 32) {
        if ((tid & 31) == 0) sm[tid >> 5] = top;
        __syncthreads();
        top = sm[0];
        for (int w = 1; w < nt / 32; ++w) top = max(top, sm[w]);
    }
    const RowScale rs = row_scale(top);
    const bool dead = top >= 0x7f800000u;     // an infinity or a NaN: codes 0
    if (tid == 0) scale[blockIdx.x] = rs.scale;
    auto put = [&](const Packed<T, VEC> &pv, int64_t v) {
        float f[VEC];
        unpack<T, VEC>(pv, f);
        if constexpr (VEC == 1) {
            out[v] = dead ? (int8_t)0 : (int8_t)code(f[0], rs.mult);
        } else {
            uint32_t w[VEC / 4];
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i) {
                const uint32_t a = __byte_perm(code(f[4 * i], rs.mult), code(f[4 * i + 1], rs.mult), 0x0040);
                const uint32_t b = __byte_perm(code(f[4 * i + 2], rs.mult), code(f[4 * i + 3], rs.mult), 0x0040);
                w[i] = dead ? 0u : __byte_perm(a, b, 0x5410);
            }
            if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(out + v * 8) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(out + v * 4) = w[0];
        }
    };
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
        if (tid + u * nt < nvec) put(held[u], tid + u * nt);
    for (int64_t v = tid + kHeld * nt; v < nvec; v += nt) put(load_packed<T, VEC>(row + v * VEC), v);
    for (int64_t c = nvec * VEC + tid; c < cols; c += nt) out[c] = dead ? (int8_t)0 : (int8_t)code(to_float(row[c]), rs.mult);
}

// ---- product, any alignment --------------------------------------------------------------------------------------------
//
// 64 x 64 outputs a block, 64 bytes of k at a time through shared memory, four-way byte products.  It serves rows that
// do not start on 16-byte boundaries, which the copy engine cannot fetch.  2048 x 4096 x 4096: 1.6 ms (43 TOP/s), bound by the
// byte-wise fill of shared memory: a caller that can choose its strides should.
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

// ---- product on the tensor cores ------------------------------------------------------------------------------------------
//
// The weights are the matrix operand of 128 rows, the tokens the columns: D[channel][token], 128 x TN 32-bit integers in
// tensor memory, so one token needs a tile of 16 columns and not of 128 rows, and a warp that reads a column out holds
// 32 neighbouring channels of one token, which it stores as they lie in y.
// Warp 0 streams boxes of 128 bytes of k (128 weight rows, TN token rows, 128-byte swizzle) into a ring; one thread of
// warp 1 issues four tcgen05.mma (kind::i8, 32 bytes of k each) per box into one of two accumulators; the others read
// the other one, scale it and store it.  CTAs are persistent over the tiles.
// One token through 4096 x 32768 weights, 134 MB: 28.7 us cold (4.7 TB/s); 4096 x 4096: 10 us, the latency of launch, copies
// and the cluster's two meetings.
// Where there are fewer tiles than SMs a cluster of `splits` CTAs shares a tile, each with its part of k: they leave
// their integer sums in shared memory and every one of them adds up and stores its share of the tokens.

struct TcArgs {
    const float *x_scale, *w_scale, *bias;
    void *y;
    long long ld_y;
    int tokens, outer;
    int tiles_m, tiles_n;   // tiles of TN tokens, of 128 channels
    int chunks;             // 128-byte chunks of k
    int stages;
    int *status;
    unsigned long long wait_ns;
};

constexpr int kChunk = 128;           // bytes of k per box
constexpr int kRows = 128;            // channels per tile
constexpr int kBand = 12;             // tiles of tokens that share a sweep over the channels (L2 holds their rows)

// Tiles are numbered so that CTAs which run together cover a near-square patch of the output.
__device__ __forceinline__ void tile_at(const TcArgs &a, int t, int &tm, int &tn) {
    const int per_band = kBand * a.tiles_n;
    const int band = t / per_band, in = t - band * per_band;
    const int height = min(kBand, a.tiles_m - band * kBand);
    tn = in / height;
    tm = band * kBand + in - tn * height;
}

template <typename T>
__device__ __forceinline__ void store_output(const TcArgs &a, int token, int channel, int sum, float xs, float ws, float b) {
    static_cast<T *>(a.y)[(long long)token * a.ld_y + channel] = from_float<T>(fmaf((float)sum, xs * ws, b));
}

// Warps that read accumulators out: with 8 of them two share a quarter of the lanes and halve the tokens, which keeps the
// read-out of a 256-token tile under the MMAs of the next one (int to float conversion alone takes 2048 cycles a tile).
__host__ __device__ constexpr int drain_warps(int tn) { return tn >= 128 ? 8 : 4; }

// Scales and stores the accumulator columns [c0, c1) of a tile for this thread's lane (channel); `scales`: shared memory of
// this warp for c1 - c0 floats.
template <typename T, int COLS>
__device__ __forceinline__ void drain(const TcArgs &a, uint32_t taddr, int token0, int channel, float *scales) {
    const int lane = (int)threadIdx.x & 31;
    const bool mine = channel < a.outer;
    const float ws = mine ? __ldg(a.w_scale + channel) : 0.f;
    const float b = mine && a.bias ? __ldg(a.bias + channel) : 0.f;
    for (int c = lane; c < COLS; c += 32) scales[c] = token0 + c < a.tokens ? __ldg(a.x_scale + token0 + c) : 0.f;
    __syncwarp();
    T *out = static_cast<T *>(a.y) + ((long long)token0 * a.ld_y + channel);
    const int count = min(COLS, a.tokens - token0);
#pragma unroll 1
    for (int c = 0; c < count; c += 16) {
        int r[16];
        __syncwarp();
        i8::tmem_load_16(taddr + (uint32_t)c, r);
        float xs[16];
#pragma unroll
        for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4 *>(&xs[j]) = *reinterpret_cast<const float4 *>(scales + c + j);
        if (!mine) continue;
        if (c + 16 <= count) {
#pragma unroll
            for (int j = 0; j < 16; ++j, out += a.ld_y) *out = from_float<T>(fmaf((float)r[j], xs[j] * ws, b));
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j, out += a.ld_y)
                if (c + j < count) *out = from_float<T>(fmaf((float)r[j], xs[j] * ws, b));
        }
    }
    __syncwarp();
}

template <typename T, int TN>
__global__ void __launch_bounds__(64 + 32 * drain_warps(TN), 1)
cr_int8_product_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const TcArgs a, const int splits) {
    using namespace i8;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    constexpr uint32_t kWBytes = kRows * kChunk, kStage = kWBytes + TN * kChunk;
    constexpr int kDrain = drain_warps(TN), kThreads = 64 + 32 * kDrain, kCols1 = TN * 4 / kDrain;   // tokens a warp reads out
    constexpr uint32_t kCols = 2 * TN < 32 ? 32 : 2 * TN;
    __shared__ __align__(16) float scales[kDrain][kCols1];
    const int S = a.stages;
    unsigned char *ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t *full = reinterpret_cast<uint64_t *>(ring + (size_t)S * kStage);
    uint64_t *empty = full + S;
    uint64_t *acc_full = empty + S, *acc_empty = acc_full + 2;
    uint64_t *settled = acc_empty + 2;                                       // used after a wait has run out
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(settled + 1);
    volatile int *flags = reinterpret_cast<volatile int *>(tmem_slot + 1);   // [0] someone gave up, [1] never set

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = splits > 1 ? (int)cluster_rank() : 0;
    const int first = (int)blockIdx.x / splits, step = (int)gridDim.x / splits;
    const int tiles = a.tiles_m * a.tiles_n;
    const int k0 = (int)((long long)a.chunks * rank / splits), k1 = (int)((long long)a.chunks * (rank + 1) / splits);

    if (tid == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], kDrain); }
        mbar_init(settled, 1);
        flags[0] = 0; flags[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(tmem_slot, kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    int issued = 0;                          // boxes that thread 0 has asked for

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 1;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                int tm, tn;
                tile_at(a, t, tm, tn);
                for (int k = k0; k < k1; ++k) {
                    if (!mbar_wait(&empty[s], phase, &flags[0], a.wait_ns)) { ok = false; break; }
                    unsigned char *st = ring + (size_t)s * kStage;
                    mbar_expect_tx(&full[s], kStage);
                    tma_load_2d(st, &map_w, k * kChunk, tn * kRows, &full[s]);
                    tma_load_2d(st + kWBytes, &map_x, k * kChunk, tm * TN, &full[s]);
                    ++issued;
                    if (++s == S) { s = 0; phase ^= 1; }
                }
            }
            if (!ok) { flags[0] = 1; atomicExch(a.status, 1); }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = instr_desc(kRows, TN);
            int s = 0, use = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step, ++use) {
                const int set = use & 1;
                if (!mbar_wait(&acc_empty[set], (uint32_t)(((use >> 1) & 1) ^ 1), &flags[0], a.wait_ns)) { ok = false; break; }
                tc_fence_after();
                for (int k = k0; k < k1; ++k) {
                    if (!mbar_wait(&full[s], phase, &flags[0], a.wait_ns)) { ok = false; break; }
                    tc_fence_after();
                    const unsigned char *st = ring + (size_t)s * kStage;
#pragma unroll
                    for (int q = 0; q < kChunk / 32; ++q)
                        mma_i8(tmem + (uint32_t)(set * TN), smem_desc(st + q * 32), smem_desc(st + kWBytes + q * 32), idesc, (k > k0 || q > 0) ? 1u : 0u);
                    mma_commit(&empty[s]);
                    if (++s == S) { s = 0; phase ^= 1; }
                }
                if (ok) mma_commit(&acc_full[set]);
            }
            if (!ok) { flags[0] = 1; atomicExch(a.status, 1); }
        }
    } else {
        const int q = warp & 3, c0 = (warp - 2) / 4 * kCols1;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c0;
        int use = 0;
        for (int t = first; t < tiles; t += step, ++use) {
            const int set = use & 1;
            int tm, tn;
            tile_at(a, t, tm, tn);
            const bool ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[set], (uint32_t)((use >> 1) & 1), &flags[0], a.wait_ns) ? 1 : 0) != 0;
            if (!ok) {
                if (lane == 0) { flags[0] = 1; atomicExch(a.status, 1); }
                break;
            }
            tc_fence_after();
            if (splits > 1) {
                // every MMA that read the ring has finished: its memory takes the sums
                int *sums = reinterpret_cast<int *>(ring) + c0 * kRows + q * 32 + lane;
#pragma unroll 1
                for (int c = 0; c < kCols1; c += 16) {
                    int r[16];
                    tmem_load_16(lanes + (uint32_t)(set * TN + c), r);
#pragma unroll
                    for (int j = 0; j < 16; ++j) sums[(c + j) * kRows] = r[j];
                }
            } else {
                drain<T, kCols1>(a, lanes + (uint32_t)(set * TN), tm * TN + c0, tn * kRows + q * 32 + lane, scales[warp - 2]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[set]);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (flags[0]) {
        // somebody gave up (whoever it was): boxes and MMAs may be under way that nobody has waited for
        if (tid == 0)
            for (int i = issued > S ? issued - S : 0; i < issued; ++i) mbar_wait(&full[i % S], (uint32_t)((i / S) & 1), &flags[1], kSettleNs);
        if (tid == 32) {                     // the thread that issued the MMAs
            mma_commit(settled);
            mbar_wait(settled, 0, &flags[1], kSettleNs);
        }
        __syncthreads();
    }
    // tensor memory goes back before the cluster meets: a CTA that holds some never waits for another CTA
    if (warp == 1) tmem_free(tmem, kCols);
    __syncthreads();
    if (splits > 1) {
        cluster_sync();      // all sums of the cluster are in place
        int tm, tn;
        tile_at(a, first, tm, tn);
        const int c0 = TN * rank / splits, c1 = TN * (rank + 1) / splits;
        for (int e = tid; e < (c1 - c0) * kRows; e += kThreads) {
            const int c = c0 + e / kRows, l = e % kRows;
            const int token = tm * TN + c, channel = tn * kRows + l;
            if (token >= a.tokens || channel >= a.outer) continue;
            const uint32_t at = smem_u32(ring) + (uint32_t)(c * kRows + l) * 4;
            int sum = 0;
            for (int r = 0; r < splits; ++r) sum += load_cluster(map_to_rank(at, (uint32_t)r));
            store_output<T>(a, token, channel, sum, __ldg(a.x_scale + token), __ldg(a.w_scale + channel), a.bias ? __ldg(a.bias + channel) : 0.f);
        }
        cluster_sync();      // nobody leaves while its sums may be read
    }
}

// Large products: two CTAs on neighbouring SMs share a tile of 256 channels x 256 tokens (cta_group::2).  Each brings its
// half of the channels and its half of the tokens, so a byte that crosses from L2 serves twice the products that it
// serves in the kernel above, which L2 paces there (13.8 TB/s at 58 % of the tensor cores' cycles on 8192 x 4096 x 8192).
// 16384 x 4096 x 8192: 356 us (3.1 POP/s, tensor pipe active 76 % of the cycles) against 448 with single CTAs; with four
// read-out warps instead of eight 425.
// The even CTA's thread issues the MMAs for both; its barriers count both CTAs' copies, its commits free both CTAs'
// stages, and each CTA reads its own 128 channels out of its own tensor memory.
constexpr int kPairStages = 6, kPairDrain = 8, kPairThreads = 64 + 32 * kPairDrain;

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
cr_int8_product_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const TcArgs a) {
    using namespace i8;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    constexpr uint32_t kWBytes = kRows * kChunk, kXBytes = 128 * kChunk, kStage = kWBytes + kXBytes;
    constexpr int S = kPairStages, TN = 256, kCols1 = TN * 4 / kPairDrain;
    __shared__ __align__(16) float scales[kPairDrain][kCols1];
    unsigned char *ring = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t *full = reinterpret_cast<uint64_t *>(ring + (size_t)S * kStage);   // used in the even CTA
    uint64_t *empty = full + S;
    uint64_t *acc_full = empty + S, *acc_empty = acc_full + 2;                  // acc_empty: used in the even CTA
    uint64_t *settled = acc_empty + 2;                                          // used after a wait has run out
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(settled + 1);
    volatile int *flags = reinterpret_cast<volatile int *>(tmem_slot + 1);      // [0] someone gave up, [1] never set, [2] boxes of the odd CTA

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)cluster_rank();
    const int first = (int)blockIdx.x >> 1, step = (int)gridDim.x >> 1;
    const int tiles = a.tiles_m * a.tiles_n;
    if (tid == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], 2 * kPairDrain); }
        mbar_init(settled, 1);
        flags[0] = 0; flags[1] = 0; flags[2] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_pair(tmem_slot, 2 * TN);
    tc_fence_before();
    __syncthreads();
    cluster_sync();          // both CTAs' barriers and tensor memory are there
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    int issued = 0;                          // boxes that thread 0 has asked for

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 1;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                int tm, tn;
                tile_at(a, t, tm, tn);
                for (int k = 0; k < a.chunks; ++k) {
                    if (!mbar_wait(&empty[s], phase, &flags[0], a.wait_ns)) { ok = false; break; }
                    unsigned char *st = ring + (size_t)s * kStage;
                    if (rank == 0) mbar_expect_tx(&full[s], 2 * kStage);
                    const uint32_t bar = map_to_rank(smem_u32(&full[s]), 0);
                    tma_load_2d_pair(st, &map_w, k * kChunk, tn * 2 * kRows + rank * kRows, bar);
                    tma_load_2d_pair(st + kWBytes, &map_x, k * kChunk, tm * TN + rank * 128, bar);
                    ++issued;
                    if (++s == S) { s = 0; phase ^= 1; }
                }
            }
            // the commits of the last stages have arrived before this CTA may end
            for (int i = issued > S ? issued - S : 0; i < issued && ok; ++i) ok = mbar_wait(&empty[i % S], (uint32_t)((i / S) & 1), &flags[0], a.wait_ns);
            if (!ok) { flags[0] = 1; atomicExch(a.status, 1); }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = instr_desc(2 * kRows, TN);
            int s = 0, use = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step, ++use) {
                const int set = use & 1;
                if (!mbar_wait(&acc_empty[set], (uint32_t)(((use >> 1) & 1) ^ 1), &flags[0], a.wait_ns)) { ok = false; break; }
                tc_fence_after();
                for (int k = 0; k < a.chunks; ++k) {
                    if (!mbar_wait(&full[s], phase, &flags[0], a.wait_ns)) { ok = false; break; }
                    tc_fence_after();
                    const unsigned char *st = ring + (size_t)s * kStage;
#pragma unroll
                    for (int q = 0; q < kChunk / 32; ++q)
                        mma_i8_pair(tmem + (uint32_t)(set * TN), smem_desc(st + q * 32), smem_desc(st + kWBytes + q * 32), idesc, (k > 0 || q > 0) ? 1u : 0u);
                    mma_commit_pair(&empty[s]);
                    if (++s == S) { s = 0; phase ^= 1; }
                }
                if (ok) mma_commit_pair(&acc_full[set]);
            }
            if (!ok) { flags[0] = 1; atomicExch(a.status, 1); }
        }
    } else {
        const int q = warp & 3, c0 = (warp - 2) / 4 * kCols1;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c0;
        int use = 0;
        for (int t = first; t < tiles; t += step, ++use) {
            const int set = use & 1;
            int tm, tn;
            tile_at(a, t, tm, tn);
            const bool ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[set], (uint32_t)((use >> 1) & 1), &flags[0], a.wait_ns) ? 1 : 0) != 0;
            if (!ok) {
                if (lane == 0) { flags[0] = 1; atomicExch(a.status, 1); }
                break;
            }
            tc_fence_after();
            drain<T, kCols1>(a, lanes + (uint32_t)(set * TN), tm * TN + c0, tn * 2 * kRows + rank * kRows + q * 32 + lane, scales[warp - 2]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_rank(smem_u32(&acc_empty[set]), 0));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && flags[0]) store_cluster(map_to_rank(smem_u32(const_cast<int *>(flags)), (uint32_t)(rank ^ 1)), 1);
    cluster_sync();          // neither CTA ends while the other one's MMAs or commits may reach it
    if (flags[0]) {
        // One of the two gave up: boxes and MMAs may be under way that nobody has waited for.  Both CTAs' boxes count on the
        // even CTA's barriers, which expect two halves a stage; the CTAs may have stopped up to a ring apart.
        if (tid == 0 && rank == 1) store_cluster(map_to_rank(smem_u32(const_cast<int *>(flags + 2)), 0), issued);
        __syncthreads();
        cluster_sync();
        if (tid == 0 && rank == 0) {
            const int other = flags[2], last = max(issued, other);
            for (int i = min(issued, other); i < last; ++i) {
                if (i >= issued) mbar_expect_tx(&full[i % S], kStage);      // the odd CTA's half comes alone
                else mbar_complete_tx(&full[i % S], kStage);                // the odd CTA's half does not come
            }
            for (int i = last > S ? last - S : 0; i < last; ++i) mbar_wait(&full[i % S], (uint32_t)((i / S) & 1), &flags[1], kSettleNs);
        }
        if (tid == 32) {
            if (rank == 0) mma_commit_pair(settled);                        // the thread that issued the MMAs
            mbar_wait(settled, 0, &flags[1], kSettleNs);
        }
        __syncthreads();
        cluster_sync();
    }
    if (warp == 1) tmem_free_pair(tmem, 2 * TN);
}

// Whether rows of codes start on 16-byte boundaries; one row by itself has no stride to ask for.
bool rows_on_16(const void *p, int64_t rows, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows == 1 || ld % 16 == 0); }

CUresult encode_codes(EncodeTiledFn encode, CUtensorMap *map, const void *base, int64_t cols, int64_t rows, int64_t ld, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows == 1 ? (cols + 15) / 16 * 16 : ld)};
    const cuuint32_t box[2] = {kChunk, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

constexpr int kStaticSmem = 8 * 128 * 4;   // at most: the scales of eight read-out warps

TcArgs tc_args(const Int8ProductArgs &p, int tile_tokens, int tile_channels, int *status, const Tuning &tune) {
    TcArgs a;
    a.x_scale = p.x_scale; a.w_scale = p.w_scale; a.bias = p.bias; a.y = p.y; a.ld_y = p.ld_y;
    a.tokens = (int)p.tokens; a.outer = (int)p.outer;
    a.tiles_m = (int)((p.tokens + tile_tokens - 1) / tile_tokens);
    a.tiles_n = (int)((p.outer + tile_channels - 1) / tile_channels);
    a.chunks = (int)((p.inner + kChunk - 1) / kChunk);
    a.stages = 0;
    a.status = status; a.wait_ns = tune.wait_limit_ns;
    return a;
}

template <typename T>
cudaError_t launch_pair(const Int8ProductArgs &p, int *status, const DeviceInfo &dev, const Tuning &tune, EncodeTiledFn encode,
                        cudaStream_t stream, int64_t *launches) {
    const TcArgs a = tc_args(p, 256, 2 * kRows, status, tune);
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
    CUtensorMap map_w, map_x;
    if (encode_codes(encode, &map_w, p.w, p.inner, p.outer, p.ld_w, kRows) != CUDA_SUCCESS ||
        encode_codes(encode, &map_x, p.x, p.inner, p.tokens, p.ld_x, 128) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> told{0};
    cudaError_t e = allow_most_smem(reinterpret_cast<const void *>(cr_int8_product_pair_kernel<T>), told);
    if (e != cudaSuccess) return e;
    const size_t smem = (size_t)kPairStages * (kRows + 128) * kChunk + (2 * kPairStages + 5) * 8 + 16 + 1024;
    const unsigned pairs = (unsigned)std::min<int64_t>(tiles, dev.sm_count / 2);
    cr_int8_product_pair_kernel<T><<<2 * pairs, kPairThreads, smem, stream>>>(map_w, map_x, a);
    e = cudaGetLastError();
    if (e == cudaSuccess) ++*launches;
    return e;
}

template <typename T, int TN>
cudaError_t launch_tc(const Int8ProductArgs &p, int *status, const DeviceInfo &dev, const Tuning &tune, EncodeTiledFn encode,
                      cudaStream_t stream, int64_t *launches) {
    TcArgs a = tc_args(p, TN, kRows, status, tune);
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
    int splits = 1;
    while (splits < 8 && tiles * splits * 2 <= dev.sm_count && a.chunks >= 2 * splits * 2) splits *= 2;
    constexpr size_t kStage = (kRows + TN) * kChunk;
    const size_t tail = 1024 + 256 + kStaticSmem;   // alignment, barriers, scales
    const size_t room = (size_t)dev.smem_optin - tail;
    int stages = (int)std::min<size_t>(8, room / kStage);
    const int per_cta = (a.chunks + splits - 1) / splits;
    // a ring no deeper than the CTA's work, but large enough for the sums of a split tile
    if (tiles * splits <= dev.sm_count) stages = std::min(stages, std::max(per_cta, (int)((TN * kRows * 4 + kStage - 1) / kStage)));
    a.stages = stages;
    const size_t smem = stages * kStage + (2 * stages + 5) * 8 + 16 + 1024;
    CUtensorMap map_w, map_x;
    if (encode_codes(encode, &map_w, p.w, p.inner, p.outer, p.ld_w, kRows) != CUDA_SUCCESS ||
        encode_codes(encode, &map_x, p.x, p.inner, p.tokens, p.ld_x, TN) != CUDA_SUCCESS)
        return cudaErrorInvalidValue;
    static std::atomic<uint64_t> told{0};
    cudaError_t e = allow_most_smem(reinterpret_cast<const void *>(cr_int8_product_kernel<T, TN>), told);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(splits > 1 ? tiles * splits : std::min<int64_t>(tiles, dev.sm_count)));
    cfg.blockDim = dim3(64 + 32 * drain_warps(TN));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = splits > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, cr_int8_product_kernel<T, TN>, map_w, map_x, a, splits);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

cudaError_t launch_quantize_rows(const void *x, int64_t rows, int64_t cols, int64_t ld_x, int elem, int8_t *q, int64_t ld_q,
                                 float *scale, const DeviceInfo &, cudaStream_t stream, int64_t *launches) {
    if (rows == 0) return cudaSuccess;
    return by_type(elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const bool wide = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (reinterpret_cast<uintptr_t>(q) & (VEC - 1)) == 0 &&
                          (rows == 1 || (ld_x % VEC == 0 && ld_q % VEC == 0));
        const int64_t nvec = wide ? (cols + VEC - 1) / VEC : cols;
        const int threads = (int)std::min<int64_t>(512, std::max<int64_t>(32, (nvec + 127) / 128 * 32));   // about four vectors a thread
        if (wide) cr_quantize_rows_kernel<T, VEC><<<(unsigned)rows, threads, 0, stream>>>(static_cast<const T *>(x), cols, ld_x, q, ld_q, scale);
        else cr_quantize_rows_kernel<T, 1><<<(unsigned)rows, threads, 0, stream>>>(static_cast<const T *>(x), cols, ld_x, q, ld_q, scale);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

cudaError_t launch_int8_product(const Int8ProductArgs &a, int *status, const DeviceInfo &dev, const Tuning &tune, EncodeTiledFn encode,
                                cudaStream_t stream, int64_t *launches) {
    if (a.tokens == 0 || a.outer == 0) return cudaSuccess;
    if (encode && rows_on_16(a.x, a.tokens, a.ld_x) && rows_on_16(a.w, a.outer, a.ld_w)) {
        return by_type(a.elem, [&](auto t) {
            using T = decltype(t);
            if (a.tokens <= 16) return launch_tc<T, 16>(a, status, dev, tune, encode, stream, launches);
            if (a.tokens <= 32) return launch_tc<T, 32>(a, status, dev, tune, encode, stream, launches);
            if (a.tokens <= 64) return launch_tc<T, 64>(a, status, dev, tune, encode, stream, launches);
            if (a.tokens <= 128) return launch_tc<T, 128>(a, status, dev, tune, encode, stream, launches);
            // rounds of tiles times what L2 lets a round take, in its unit of 32 KB a chunk: 128 x 128 on one SM, 256 x 256 on two
            const int64_t tn = (a.outer + 127) / 128, sms = dev.sm_count;
            const int64_t single = ((a.tokens + 127) / 128 * tn + sms - 1) / sms;
            const int64_t pair = ((a.tokens + 255) / 256 * ((tn + 1) / 2) + sms / 2 - 1) / (sms / 2);
            // one round of small tiles has L2 to itself and takes half the MMA cycles of one of large tiles
            if (single < pair || single == 1) return launch_tc<T, 128>(a, status, dev, tune, encode, stream, launches);
            return launch_pair<T>(a, status, dev, tune, encode, stream, launches);
        });
    }
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
