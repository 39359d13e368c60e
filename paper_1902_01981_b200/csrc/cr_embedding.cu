// Embedding: rows of a table by token number, scaled, and the table's gradient.
//
//   y_t = s E[id_t]            dE_p[v] = s sum_{t in partition p, id_t = v} dy_t
//
// A number outside the table names nothing: its row of y is zero, and it has no gradient.  The gradient of every partition is
// written whole (rows that no token names are zero): it is a partial gradient as the aggregation takes it.
//
// The gradient's sums have one order.  A partition's tokens are sorted by number, equal numbers in the order of their
// positions (a radix sort, exact), the sorted sequence is cut into tiles, and a token number's sum is the sum of its
// tiles' pieces in one order.  The tiles depend on the partition's own tokens, so a partition gets the same bits alone and
// in a batch.  Sums are fp32; the scale is applied once, to the sum.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cr_elem.cuh"

namespace cr {
namespace {

// ---- lookup ------------------------------------------------------------------------------------------------------------

constexpr int kLookupThreads = 256;

// `per_row` threads take a row (several rows a warp, or several warps a row), lookup_held vectors each at a time, which lie a
// warp's width apart.  Bound by memory: 65536 rows of 2048 bf16, 57 us for 268 MB written and a table of 131 MB.
template <int VEC> __host__ __device__ constexpr int lookup_held() { return VEC == 1 ? 16 : 4; }
template <typename T, int VEC, typename I>
__global__ void __launch_bounds__(kLookupThreads) cr_embedding_kernel(const I *ids, const T *table, int64_t ld_table, T *y, int64_t ld_y, int64_t tokens,
                                                                      int64_t vocab, int nvec, int per_row, float scale) {
    constexpr int kHeld = lookup_held<VEC>();
    const int64_t t = (int64_t)blockIdx.x * (kLookupThreads / per_row) + (int)threadIdx.x / per_row;
    if (t >= tokens) return;
    const int64_t id = (int64_t)ids[t];
    const bool named = id >= 0 && id < vocab;
    const int j = (int)threadIdx.x % per_row, step = min(per_row, 32), v0 = j / step * step * kHeld + j % step;
    const T *row = table + (named ? id : 0) * ld_table + (int64_t)v0 * VEC;
    T *out = y + t * ld_y + (int64_t)v0 * VEC;
    for (int left = nvec - v0; left > 0; left -= per_row * kHeld, row += per_row * kHeld * VEC, out += per_row * kHeld * VEC) {
        Packed<T, VEC> r[kHeld];
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (named && u * step < left) r[u] = load_packed<T, VEC>(row + u * step * VEC);
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (u * step >= left) break;
            float f[VEC] = {};
            if (named) {
                unpack<T, VEC>(r[u], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[i] *= scale;
            }
            store_packed<T, VEC>(out + u * step * VEC, pack<T, VEC>(f));
        }
    }
}

// ---- sorting a partition's tokens -----------------------------------------------------------------------------------------

constexpr int kDigitBits = 8, kBins = 1 << kDigitBits, kMaxCluster = 8, kSortOneCta = 2048;

__device__ __forceinline__ void sort_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Word `w` of a shared array of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t peer_word(const uint32_t *w, int rank) {
    uint32_t addr, v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"((uint32_t)__cvta_generic_to_shared(w)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

struct GradArgs {
    const void *dy;
    float *dtable, *pieces;      // pieces [partitions][tiles][width]: what a tile adds to a sum that began before it
    uint2 *pairs;                // [partitions][2][tokens]
    int32_t *bounds;             // [partitions][tiles + 1]: where the tiles begin
    int32_t *far;                // [partitions][1 + tiles]: count and tiles where a sum first goes on from the tile before
    uint32_t *named;             // [partitions][words]: a bit a number, set if a token names it; null: no tokens
    int64_t tokens, vocab, padding, ld_dy, ld_row, ld_partition;
    int width, tile, tiles, passes, words;
    float scale;
};

template <int VEC>
__device__ __forceinline__ void store_floats(float *p, const float (&v)[VEC], float scale) {
    if constexpr (VEC == 1) {
        *p = v[0] * scale;
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i)
            reinterpret_cast<float4 *>(p)[i] = make_float4(v[4 * i] * scale, v[4 * i + 1] * scale, v[4 * i + 2] * scale, v[4 * i + 3] * scale);
    }
}

// Sums of up to this many tokens are not cut.
constexpr int kWhole = 64;

// Where a tile begins: at position i0, or, where a number of at most kWhole tokens lies across it, at that number's first one.
// `cut`: a longer one lies across it.  For a warp.
__device__ __forceinline__ int tile_begin(const uint2 *pairs, int i0, int n, bool &cut) {
    const int lane = (int)threadIdx.x % 32;
    const uint32_t number = pairs[i0].x;
    int back = 0, on = 0;
#pragma unroll
    for (int k = 0; k < kWhole / 32; ++k) {
        const int b = i0 - 1 - k * 32 - lane, f = i0 + k * 32 + lane;
        const uint32_t same_back = __ballot_sync(0xffffffffu, b >= 0 && pairs[max(b, 0)].x == number);
        const uint32_t same_on = __ballot_sync(0xffffffffu, f < n && pairs[min(f, n - 1)].x == number);
        if (back == k * 32) back += same_back == 0xffffffffu ? 32 : __ffs(~same_back) - 1;
        if (on == k * 32) on += same_on == 0xffffffffu ? 32 : __ffs(~same_on) - 1;
    }
    cut = back > 0 && back + on > kWhole;
    return cut ? i0 : i0 - back;
}

// The lanes that hold this lane's digit, by a vote a bit (the match instruction in its place: 51 instead of 46 us for 65536
// tokens).  Without meaning for a lane that has none.
__device__ __forceinline__ uint32_t same_digit(uint32_t d, bool has) {
    uint32_t peers = __ballot_sync(0xffffffffu, has);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const bool one = d >> b & 1u;
        const uint32_t m = __ballot_sync(0xffffffffu, one);
        peers &= one ? m : ~m;
    }
    return peers;
}

// This thread's bin: what the warps before each warp have counted, in place of each warp's count; returns the sum.
__device__ __forceinline__ uint32_t sum_warps(uint32_t (*hist)[kBins], int warps) {
    uint32_t sum = 0;
#pragma unroll
    for (int w0 = 0; w0 < 32; w0 += 8) {
        uint32_t c[8];
#pragma unroll
        for (int w = 0; w < 8; ++w) c[w] = w0 + w < warps ? hist[w0 + w][threadIdx.x] : 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (w0 + w < warps) hist[w0 + w][threadIdx.x] = sum;
            sum += c[w];
        }
    }
    return sum;
}

// Marks the numbers that occur, and cuts the sorted sequence into tiles: the threads of a partition, `first` among `all`, and its
// warps.  a.named is zero and far[0] is zero by now.
__device__ __forceinline__ void cut_tiles(const GradArgs &a, int64_t part, const uint2 *sorted, int count, int first, int all) {
    uint32_t *named = a.named + part * a.words;
    for (int i = first; i < count; i += all) {
        const uint32_t v = sorted[i].x;
        if (i == 0 || sorted[i - 1].x != v) atomicOr(&named[v / 32], 1u << (v % 32));
    }
    int32_t *bounds = a.bounds + part * (a.tiles + 1), *far = a.far + part * (a.tiles + 1);
    for (int64_t t = first / 32; t <= a.tiles; t += all / 32) {
        const int64_t i0 = t * a.tile;
        int begin = (int)min(i0, (int64_t)count);
        if (t > 0 && i0 < count) {
            bool cut;
            begin = tile_begin(sorted, (int)i0, count, cut);
            if (cut && first % 32 == 0) {
                // the first tile into which the number reaches: only from a number's first tile on does a sum go on
                const int64_t earlier = i0 - a.tile;
                if (earlier == 0 || sorted[earlier - 1].x != sorted[i0].x) far[1 + atomicAdd(&far[0], 1)] = (int32_t)t;
            }
        }
        if (first % 32 == 0) bounds[t] = begin;
    }
}

// Sorts (number, position) of the tokens of a partition that name a row, by number, then position: digits of 8 bits from
// the lowest up, each pass stable.  Up to 1024 EACH tokens, one CTA, everything on the chip: a thread holds EACH entries, lanes with
// one digit find each other, which gives an entry its rank among its warp's; the counts of the warps and digits
// are summed up, and the entries go to their places in shared memory.  Then the sequence is cut into tiles.  Bound by latency,
// a few dependent steps an entry and pass.
template <typename I, int EACH>
__global__ void __launch_bounds__(1024, 1) cr_token_sort_kernel(const GradArgs a, const I *ids) {
    extern __shared__ uint2 entries[];           // [32 EACH warps]
    __shared__ uint32_t hist[32][kBins], base[kBins], scan[kBins / 32];
    let_next_begin();
    const int64_t part = blockIdx.x;
    const int tid = (int)threadIdx.x, nt = (int)blockDim.x, warp = tid / 32, lane = tid % 32, warps = nt / 32;
    const uint32_t below = (1u << lane) - 1u;
    const int mine = warp * 32 * EACH + lane;    // this thread's entries are 32 apart
    ids += part * a.tokens;
    if (tid == 0) a.far[part * (a.tiles + 1)] = 0;
    for (int w = tid; w < a.words; w += nt) a.named[part * a.words + w] = 0;
    uint32_t key[EACH], place[EACH];             // a place: position in the low half, rank in the high half
    bool in[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int i = mine + k * 32;
        const int64_t id = i < a.tokens ? (int64_t)ids[i] : -1;
        in[k] = id >= 0 && id < a.vocab && id != a.padding;
        key[k] = (uint32_t)id;
        place[k] = (uint32_t)i;
    }
    int count = 0;
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * kDigitBits;
        for (int b = lane; b < kBins; b += 32) hist[warp][b] = 0;
        __syncwarp();
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const uint32_t d = in[k] ? (key[k] >> shift) & (kBins - 1) : kBins;
            const uint32_t peers = same_digit(d, in[k]);
            const uint32_t before = in[k] ? hist[warp][d] : 0;
            place[k] = (place[k] & 0xffffu) | (before + __popc(peers & below)) << 16;
            __syncwarp();
            if (in[k] && (peers & below) == 0) hist[warp][d] = before + __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        uint32_t sum = 0, inclusive = 0;
        if (tid < kBins) {
            sum = sum_warps(hist, warps);
            inclusive = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, inclusive, o);
                if (lane >= o) inclusive += v;
            }
            if (lane == 31) scan[warp] = inclusive;
        }
        __syncthreads();
        uint32_t before = 0;
        count = 0;
#pragma unroll
        for (int w = 0; w < kBins / 32; ++w) {
            if (w < warp) before += scan[w];
            count += (int)scan[w];
        }
        if (tid < kBins) base[tid] = before + inclusive - sum;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (!in[k]) continue;
            const uint32_t d = (key[k] >> shift) & (kBins - 1);
            entries[base[d] + hist[warp][d] + (place[k] >> 16)] = make_uint2(key[k], place[k] & 0xffffu);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int i = mine + k * 32;
            in[k] = i < count;
            if (!in[k]) continue;
            key[k] = entries[i].x;
            place[k] = entries[i].y;
        }
    }
    uint2 *pairs = a.pairs + part * 2 * a.tokens;
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (in[k]) pairs[mine + k * 32] = make_uint2(key[k], place[k] & 0xffffu);
    cut_tiles(a, part, entries, count, tid, nt);
}

// More tokens: a cluster of CTAs takes a partition; each warp owns a run of consecutive entries and goes over it twice a
// pass, first counting, then putting them in place, kBatch times 32 of them in flight.  The buffers are in global memory (L2).
// Bound by latency: four partitions of 16384 tokens 18 us, of 65536 39 us, of 4000 14 us (one CTA 13.5: the border is at 2048).
template <typename I>
__global__ void __launch_bounds__(1024, 1) cr_token_sort_cluster_kernel(const GradArgs a, const I *ids) {
    constexpr int WARPS = 32, cluster = kMaxCluster;
    static_assert(WARPS * 32 >= kBins, "a thread a bin");
    __shared__ uint32_t hist[WARPS][kBins];
    __shared__ uint32_t total[kBins], base[kBins], scan[kBins / 32];
    let_next_begin();
    const int64_t part = blockIdx.x / (unsigned)cluster;
    const int rank = (int)(blockIdx.x % (unsigned)cluster), tid = (int)threadIdx.x, warp = tid / 32, lane = tid % 32;
    const uint32_t below = (1u << lane) - 1u;
    ids += part * a.tokens;
    uint2 *buffer[2] = {a.pairs + part * 2 * a.tokens, a.pairs + (part * 2 + 1) * a.tokens};
    if (rank == 0 && tid == 0) a.far[part * (a.tiles + 1)] = 0;
    uint32_t *named = a.named + part * a.words;
    for (int w = rank * WARPS * 32 + tid; w < a.words; w += cluster * WARPS * 32) named[w] = 0;
    int count = (int)a.tokens;
    for (int pass = 0; pass < a.passes; ++pass) {
        // the last pass writes into buffer 0
        const int into = (a.passes - 1 - pass) & 1;
        const uint2 *from = buffer[into ^ 1];
        uint2 *to = buffer[into];
        constexpr unsigned kShares = 32 * cluster * WARPS;
        const unsigned each = ((unsigned)count + kShares - 1) / kShares * 32;      // positions and sums of a few fit 32 bits unsigned
        const unsigned begin = min((unsigned)count, (unsigned)(rank * WARPS + warp) * each), end = min((unsigned)count, begin + each);
        auto entry = [&](unsigned i, uint2 &e) -> uint32_t {      // the digit; kBins: no entry
            if (i >= end) return kBins;
            if (pass == 0) {
                const int64_t id = (int64_t)ids[i];
                if (id < 0 || id >= a.vocab || id == a.padding) return kBins;
                e = make_uint2((uint32_t)id, i);
            } else {
                e = from[i];
            }
            return (e.x >> (pass * kDigitBits)) & (kBins - 1);
        };
        for (int b = lane; b < kBins; b += 32) hist[warp][b] = 0;
        __syncwarp();
        constexpr int kBatch = 4;
        for (unsigned i = begin; i < end; i += 32 * kBatch) {
            uint2 e;
            uint32_t d[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) d[k] = entry(i + k * 32 + lane, e);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i + k * 32 >= end) break;
                const uint32_t peers = same_digit(d[k], d[k] < kBins);
                if (d[k] < kBins && (peers & below) == 0) hist[warp][d[k]] += __popc(peers);
                __syncwarp();
            }
        }
        __syncthreads();
        if (tid < kBins) total[tid] = sum_warps(hist, WARPS);
        sort_meet();
        uint32_t mine = 0, before = 0, inclusive = 0;
        if (tid < kBins) {
            uint32_t v[cluster];
#pragma unroll
            for (int r = 0; r < cluster; ++r) v[r] = peer_word(&total[tid], r);
#pragma unroll
            for (int r = 0; r < cluster; ++r) {
                if (r < rank) before += v[r];
                mine += v[r];
            }
            inclusive = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, inclusive, o);
                if (lane >= o) inclusive += v;
            }
            if (lane == 31) scan[warp] = inclusive;
        }
        __syncthreads();
        uint32_t all = 0;
#pragma unroll
        for (int w = 0; w < kBins / 32; ++w) {
            if (w < warp) before += scan[w];
            all += scan[w];
        }
        if (tid < kBins) base[tid] = before + inclusive - mine;
        __syncthreads();
        for (unsigned i = begin; i < end; i += 32 * kBatch) {
            uint2 e[kBatch];
            uint32_t d[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) d[k] = entry(i + k * 32 + lane, e[k]);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                if (i + k * 32 >= end) break;
                const uint32_t peers = same_digit(d[k], d[k] < kBins);
                if (d[k] < kBins) to[base[d[k]] + hist[warp][d[k]] + __popc(peers & below)] = e[k];
                __syncwarp();
                if (d[k] < kBins && (peers & below) == 0) hist[warp][d[k]] += __popc(peers);
                __syncwarp();
            }
        }
        count = (int)all;
        sort_meet();     // the entries are in place, and nobody reads a peer's counts any more
    }
    cut_tiles(a, part, buffer[0], count, rank * WARPS * 32 + tid, cluster * WARPS * 32);
}

// ---- sums ---------------------------------------------------------------------------------------------------------------

constexpr int kSumThreads = 128;

// A tile of the sorted tokens for a slab of columns: `across` threads, kHeld vectors of columns each, walk the tile's tokens and
// write a sum wherever the number changes: into the table's row where the number's first token is in this tile, into the
// tile's row of pieces where it is not.  The pairs of the next tokens are fetched with the rows of these.
template <int VEC> __host__ __device__ constexpr int sum_held() { return VEC == 1 ? 4 : 1; }
template <typename T, int VEC>
__device__ __forceinline__ void sum_tile(const GradArgs &a, unsigned block, int across, int slabs) {
    constexpr int kUnroll = 8, kHeld = sum_held<VEC>();
    const int per_block = kSumThreads / across;
    const int groups = (a.tiles + per_block - 1) / per_block;
    const unsigned item = block / (unsigned)slabs;
    const int slab = (int)(block % (unsigned)slabs);
    const int64_t part = item / (unsigned)groups;
    const int tile = (int)(item % (unsigned)groups) * per_block + (int)threadIdx.x / across;
    const int col = (slab * kHeld * across + (int)threadIdx.x % across) * VEC, step = across * VEC;
    if (tile >= a.tiles || col >= a.width) return;
    bool in[kHeld];
#pragma unroll
    for (int q = 0; q < kHeld; ++q) in[q] = col + q * step < a.width;
    const int32_t *bounds = a.bounds + part * (a.tiles + 1) + tile;
    const int64_t first = bounds[0];
    const int count = bounds[1] - bounds[0];
    if (count <= 0) return;
    const uint2 *pairs = a.pairs + part * 2 * a.tokens + first;
    const T *dy = static_cast<const T *>(a.dy) + part * a.tokens * a.ld_dy + col;
    float *table = a.dtable + part * a.ld_partition + col;
    float *piece = a.pieces + (part * a.tiles + tile) * a.width + col;
    uint2 e[kUnroll + 1];
    bool began_before = first > 0 && pairs[-1].x == pairs[0].x;
    float acc[kHeld][VEC] = {};
#pragma unroll
    for (int u = 0; u <= kUnroll; ++u) e[u] = u < count ? pairs[u] : make_uint2(0xffffffffu, 0);
    for (int t0 = 0; t0 < count; t0 += kUnroll) {
        Packed<T, VEC> r[kUnroll][kHeld];
        uint2 next[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const T *row = dy + (int64_t)e[u].y * a.ld_dy;
#pragma unroll
            for (int q = 0; q < kHeld; ++q)
                if (t0 + u < count && in[q]) r[u][q] = load_packed<T, VEC>(row + q * step);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) next[u] = t0 + kUnroll + 1 + u < count ? pairs[t0 + kUnroll + 1 + u] : make_uint2(0xffffffffu, 0);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (t0 + u >= count) break;
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                float f[VEC];
                unpack<T, VEC>(r[u][q], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[q][i] += f[i];
            }
            if (e[u + 1].x != e[u].x) {
                float *out = began_before ? piece : table + (int64_t)e[u].x * a.ld_row;
                const float scale = began_before ? 1.f : a.scale;
                began_before = false;
#pragma unroll
                for (int q = 0; q < kHeld; ++q) {
                    if (in[q]) store_floats<VEC>(out + q * step, acc[q], scale);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[q][i] = 0.f;
                }
            }
        }
        e[0] = e[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) e[u + 1] = next[u];
    }
}

// Zeroes those of 32 rows that no token names, a warp a row: vectors from the row's first 16-byte boundary on.
__device__ __forceinline__ void zero_rows(const GradArgs &a, unsigned block) {
    const int64_t part = block / (unsigned)a.words, word = block % (unsigned)a.words;
    const uint32_t named = a.named ? a.named[part * a.words + word] : 0;
    const int rows = (int)min((int64_t)32, a.vocab - word * 32), lane = (int)threadIdx.x % 32;
    for (int r = (int)threadIdx.x / 32; r < rows; r += kSumThreads / 32) {
        if (named >> r & 1u) continue;
        float *out = a.dtable + part * a.ld_partition + (word * 32 + r) * a.ld_row;
        const int head = min(a.width, (int)((16 - (reinterpret_cast<uintptr_t>(out) & 15u)) / 4) % 4), body = (a.width - head) / 4 * 4;
        if (lane < head) out[lane] = 0.f;
#pragma unroll 4
        for (int c = lane * 4; c < body; c += 128) *reinterpret_cast<float4 *>(out + head + c) = make_float4(0.f, 0.f, 0.f, 0.f);
        if (lane < a.width - head - body) out[head + body + lane] = 0.f;
    }
}

// Sums and zeroes in one grid: the first `sum_blocks` blocks take tiles.  Bound by memory: 4 x 16384 tokens, tables of 32000 x 1024 from
// bf16, 659 MB, 98 us (6.7 TB/s).
template <typename T, int VEC>
__global__ void __launch_bounds__(kSumThreads) cr_embedding_sums_kernel(const GradArgs a, unsigned sum_blocks, int across, int slabs) {
    let_next_begin();
    if (a.named) wait_for_previous();        // null: nothing was launched before
    if (blockIdx.x < sum_blocks) sum_tile<T, VEC>(a, blockIdx.x, across, slabs);
    else zero_rows(a, blockIdx.x - sum_blocks);
}

// Numbers whose tokens reach into further tiles: the tiles' pieces are added to the row.  `across` threads take a vector of
// columns each; the block's threads / across of them that share a column take every such piece each and are summed in order.
constexpr int kJoinThreads = 256;
template <int VEC>
__device__ __forceinline__ void join_pieces(const GradArgs &a, int64_t part, int64_t tile, int slab, int across, float *sm) {
    constexpr int kUnroll = 4;
    const int deep = kJoinThreads / across, col0 = (int)threadIdx.x % across, row = (int)threadIdx.x / across;
    const int col = (slab * across + col0) * VEC;
    const int32_t *bounds = a.bounds + part * (a.tiles + 1);
    const uint2 *pairs = a.pairs + part * 2 * a.tokens;
    const int64_t n = bounds[a.tiles];
    const uint32_t number = pairs[tile * a.tile].x;
    const bool in = col < a.width;
    const float *pieces = a.pieces + part * a.tiles * a.width + col;
    float sum[VEC] = {};
    for (int64_t t0 = tile + row;; t0 += deep * kUnroll) {
        float f[kUnroll][VEC] = {};
        bool more = true;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t t = t0 + u * deep;
            const bool reaches = t * a.tile < n && pairs[t * a.tile].x == number;
            more = reaches;
            if (!reaches || !in) continue;
            if constexpr (VEC == 4) {
                const float4 p = *reinterpret_cast<const float4 *>(pieces + t * a.width);
                f[u][0] = p.x; f[u][1] = p.y; f[u][2] = p.z; f[u][3] = p.w;
            } else {
                f[u][0] = pieces[t * a.width];
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum[i] += f[u][i];
        if (!more) break;
    }
    __syncthreads();             // the memory is free again
#pragma unroll
    for (int i = 0; i < VEC; ++i) sm[(int)threadIdx.x * VEC + i] = sum[i];
    __syncthreads();
    if (row != 0 || !in) return;
    for (int r = 1; r < deep; ++r)
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += sm[(r * across + col0) * VEC + i];
    float *out = a.dtable + part * a.ld_partition + (int64_t)number * a.ld_row + col;
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[i] += a.scale * sum[i];
}
template <int VEC>
__global__ void __launch_bounds__(kJoinThreads) cr_embedding_join_kernel(const GradArgs a, int across, int slabs, unsigned walkers) {
    __shared__ float sm[kJoinThreads * VEC];
    wait_for_previous();
    const unsigned item = blockIdx.x / (unsigned)slabs;
    const int64_t part = item / walkers;
    const int32_t *far = a.far + part * (a.tiles + 1);
    const int count = far[0];
    for (int k = (int)(item % walkers); k < count; k += (int)walkers) join_pieces<VEC>(a, part, far[1 + k], (int)(blockIdx.x % (unsigned)slabs), across, sm);
}

int tile_tokens(int64_t tokens) {
    // 32 tokens; longer tiles where there would be more than 4096 of them to join
    int64_t tile = 32;
    while (tokens / tile > 4096) tile *= 2;
    return (int)tile;
}
size_t align16(size_t b) { return (b + 15) / 16 * 16; }

}  // namespace

// pairs, bounds, far, named, pieces
size_t embedding_backward_workspace_bytes(int64_t tokens, int64_t partitions, int64_t vocab, int64_t width) {
    if (tokens == 0) return 0;
    const int64_t tile = tile_tokens(tokens), tiles = (tokens + tile - 1) / tile;
    return (size_t)(partitions * tokens * 16) + 2 * align16((size_t)(partitions * (tiles + 1)) * 4) + align16((size_t)(partitions * ((vocab + 31) / 32)) * 4) +
           (size_t)(tokens > kWhole ? partitions * tiles * width * 4 : 0);
}

cudaError_t launch_embedding(const EmbeddingArgs &a, cudaStream_t stream, int64_t *launches) {
    if (a.tokens == 0 || a.width == 0) return cudaSuccess;
    return by_type(a.elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const bool wide = vector_rows(a.elem, a.width, {a.table, a.y}, {a.ld_table, a.ld_y});
        const int nvec = (int)(wide ? a.width / VEC : a.width);
        const int held = wide ? lookup_held<VEC>() : lookup_held<1>();
        int per_row = 1;
        while (per_row < kLookupThreads && per_row * held < nvec) per_row *= 2;
        const int rows = kLookupThreads / per_row;
        const unsigned blocks = (unsigned)((a.tokens + rows - 1) / rows);
        auto go = [&](auto v, auto i) {
            using I = decltype(i);
            cr_embedding_kernel<T, decltype(v)::value, I><<<blocks, kLookupThreads, 0, stream>>>(
                static_cast<const I *>(a.ids), static_cast<const T *>(a.table), a.ld_table, static_cast<T *>(a.y), a.ld_y, a.tokens, a.vocab, nvec, per_row,
                a.scale);
        };
        auto by_ids = [&](auto v) { a.id_bytes == 4 ? go(v, int32_t{}) : go(v, (long long){}); };
        if (wide) by_ids(Int<VEC>{});
        else by_ids(Int<1>{});
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    });
}

cudaError_t launch_embedding_backward(const EmbeddingArgs &a, void *workspace, const DeviceInfo &dev, cudaStream_t stream, int64_t *launches) {
    if (a.partitions == 0 || a.vocab == 0 || a.width == 0) return cudaSuccess;
    GradArgs g = {};
    g.dy = a.dy; g.dtable = a.dtable; g.tokens = a.tokens; g.vocab = a.vocab;
    g.ld_dy = a.ld_dy; g.ld_row = a.ld_row; g.ld_partition = a.ld_partition;
    g.width = (int)a.width; g.scale = a.scale;
    const bool table16 = aligned16(a.dtable) && a.ld_row % 4 == 0 && (a.partitions == 1 || a.ld_partition % 4 == 0);
    g.padding = a.padding;
    g.tile = tile_tokens(a.tokens);
    g.tiles = (int)((a.tokens + g.tile - 1) / g.tile);
    g.words = (int)((a.vocab + 31) / 32);
    // the grid of the sums and zeroes
    const int vec = 16 / elem_bytes(a.elem);
    const bool wide = table16 && vector_rows(a.elem, a.width, {a.dy}, {a.ld_dy});
    const int nvec = g.width / (wide ? vec : 1), held = wide ? 1 : sum_held<1>();
    int across = 1;
    while (across < kSumThreads && across * held < nvec) across *= 2;
    const int slabs = (nvec + across * held - 1) / (across * held);
    const int64_t groups = (g.tiles + kSumThreads / across - 1) / (kSumThreads / across);
    if (a.partitions * groups > ((1ll << 29) - 1) / slabs) return cudaErrorInvalidValue;     // more than the gradients that fit a device
    const unsigned sums = (unsigned)(a.partitions * groups * slabs), blocks = sums + (unsigned)(a.partitions * g.words);
    if (a.tokens > 0) {
        char *p = static_cast<char *>(workspace);
        const size_t table = align16((size_t)(a.partitions * (g.tiles + 1)) * 4);
        g.pairs = reinterpret_cast<uint2 *>(p);
        g.bounds = reinterpret_cast<int32_t *>(p += a.partitions * a.tokens * 16);
        g.far = reinterpret_cast<int32_t *>(p += table);
        g.named = reinterpret_cast<uint32_t *>(p += table);
        g.pieces = reinterpret_cast<float *>(p += align16((size_t)(a.partitions * g.words) * 4));
        int bits = 1;
        while (bits < 31 && (1ll << bits) < a.vocab) ++bits;
        g.passes = (bits + kDigitBits - 1) / kDigitBits;
        cudaError_t e;
        auto by_ids = [&](auto &&f) { return a.id_bytes == 4 ? f(int32_t{}) : f((long long){}); };
        if (a.tokens <= kSortOneCta) {
            e = by_ids([&](auto i) {
                using I = decltype(i);
                auto go = [&](auto each, auto kernel) -> cudaError_t {
                    constexpr int EACH = decltype(each)::value;
                    const int warps = std::max(kBins / 32, (int)((a.tokens + 32 * EACH - 1) / (32 * EACH)));
                    const size_t smem = (size_t)warps * 32 * EACH * sizeof(uint2);
                    if (smem > 8 * 1024) {       // beside the counters' 34 KB
                        static std::atomic<uint64_t> told{0};      // one for each EACH and type of ids
                        const cudaError_t e = allow_most_smem(reinterpret_cast<const void *>(kernel), told);
                        if (e != cudaSuccess) return e;
                    }
                    kernel<<<(unsigned)a.partitions, 32 * warps, smem, stream>>>(g, static_cast<const I *>(a.ids));
                    return cudaGetLastError();
                };
                if (a.tokens <= 1024) return go(Int<1>{}, cr_token_sort_kernel<I, 1>);
                return go(Int<2>{}, cr_token_sort_kernel<I, 2>);
            });
        } else {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(a.partitions * kMaxCluster));
            cfg.blockDim = dim3(1024);
            cfg.stream = stream;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = kMaxCluster;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            e = by_ids([&](auto i) { return cudaLaunchKernelEx(&cfg, cr_token_sort_cluster_kernel<decltype(i)>, g, static_cast<const decltype(i) *>(a.ids)); });
        }
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    cudaError_t e = by_type(a.elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        auto kernel = wide ? cr_embedding_sums_kernel<T, VEC> : cr_embedding_sums_kernel<T, 1>;
        if (a.tokens > 0) return launch_next(kernel, blocks, kSumThreads, stream, g, sums, across, slabs);
        kernel<<<blocks, kSumThreads, 0, stream>>>(g, sums, across, slabs);
        return cudaGetLastError();
    });
    if (e != cudaSuccess) return e;
    ++*launches;
    if (a.tokens > kWhole) {      // otherwise no sum is cut
        const bool four = table16 && g.width % 4 == 0;
        const int join_nvec = four ? g.width / 4 : g.width;
        int join_across = 1;
        while (join_across < 64 && join_across < join_nvec) join_across *= 2;
        const int join_slabs = (join_nvec + join_across - 1) / join_across;
        const int64_t walkers = std::min<int64_t>(a.tokens / kWhole, std::max<int64_t>(1, 4 * dev.sm_count / a.partitions));
        if (a.partitions * walkers > 0x7fffffffll / join_slabs) return cudaErrorInvalidValue;
        const unsigned joins = (unsigned)(a.partitions * walkers * join_slabs);
        e = launch_next(four ? cr_embedding_join_kernel<4> : cr_embedding_join_kernel<1>, joins, kJoinThreads, stream, g, join_across, join_slabs,
                        (unsigned)walkers);
        if (e == cudaSuccess) ++*launches;
    }
    return e;
}

}  // namespace cr
