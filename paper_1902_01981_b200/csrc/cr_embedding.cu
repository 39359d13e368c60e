// Embedding: rows of a table by token number, scaled, and the table's gradient.
//
//   y_t = s E[id_t]            dE_p[v] = s sum_{t in partition p, id_t = v} dy_t
//
// A number outside the table names nothing: its row of y is zero, and it has no gradient.  The gradient of every partition is
// written whole (rows that no token names are zero): it is a partial gradient as the aggregation takes it.
//
// The gradient's sums have one order.  A partition's tokens are sorted by number, equal numbers in the order of their
// positions (a radix sort, exact), the sorted sequence is cut into tiles, and a token number's sum is the sum of its
// tiles' pieces in ascending order.  The tiles depend on the partition's length alone, so a partition gets the same bits
// alone and in a batch.  Sums are fp32; the scale is applied once, to the sum.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cr_elem.cuh"

namespace cr {
namespace {

// ---- lookup ------------------------------------------------------------------------------------------------------------

constexpr int kLookupThreads = 256;

// `per_row` threads take a row, four vectors each at a time.
template <typename T, int VEC, typename I>
__global__ void __launch_bounds__(kLookupThreads) cr_embedding_kernel(const I *ids, const T *table, int64_t ld_table, T *y, int64_t ld_y, int64_t tokens,
                                                                      int64_t vocab, int nvec, int per_row, float scale) {
    constexpr int kUnroll = 4;
    const int64_t t = (int64_t)blockIdx.x * (kLookupThreads / per_row) + (int)threadIdx.x / per_row;
    if (t >= tokens) return;
    const int64_t id = (int64_t)ids[t];
    const bool named = id >= 0 && id < vocab;
    const T *row = table + (named ? id : 0) * ld_table;
    T *out = y + t * ld_y;
    for (int v0 = (int)threadIdx.x % per_row; v0 < nvec; v0 += per_row * kUnroll) {
        Packed<T, VEC> r[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int v = v0 + u * per_row;
            if (named && v < nvec) r[u] = load_packed<T, VEC>(row + (int64_t)v * VEC);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int v = v0 + u * per_row;
            if (v >= nvec) break;
            float f[VEC] = {};
            if (named) {
                unpack<T, VEC>(r[u], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[i] *= scale;
            }
            store_packed<T, VEC>(out + (int64_t)v * VEC, pack<T, VEC>(f));
        }
    }
}

// ---- sorting a partition's tokens -----------------------------------------------------------------------------------------

constexpr int kDigitBits = 8, kBins = 1 << kDigitBits, kMaxCluster = 8;

__device__ __forceinline__ void sort_meet(int cluster) {
    if (cluster == 1) {
        __syncthreads();
        return;
    }
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

// (number, position) of the tokens of a partition that name a row, sorted by number, then position: digits of 8 bits from
// the lowest up, each pass stable.  A cluster of CTAs takes a partition; each warp owns a run of consecutive entries, counts
// its digits (lanes with one digit find each other by match), and after the counts of all warps have been summed up it
// puts its entries in place in order.  The buffers are in global memory (L2).  Bound by latency: a few dependent steps a pass.
template <typename I, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) cr_token_sort_kernel(const I *ids, int tokens, int64_t vocab, int64_t padding, int passes, uint2 *pairs,
                                                                   int32_t *counts, int cluster) {
    static_assert(WARPS * 32 >= kBins, "a thread a bin");
    __shared__ uint32_t hist[WARPS][kBins];
    __shared__ uint32_t total[kBins], scan[kBins / 32];
    const int64_t part = blockIdx.x / (unsigned)cluster;
    const int rank = (int)(blockIdx.x % (unsigned)cluster), tid = (int)threadIdx.x, warp = tid / 32, lane = tid % 32;
    const uint32_t below = (1u << lane) - 1u;
    ids += part * tokens;
    uint2 *buffer[2] = {pairs + part * 2 * tokens, pairs + (part * 2 + 1) * tokens};
    int count = tokens;
    for (int pass = 0; pass < passes; ++pass) {
        // the last pass writes into buffer 0
        const int into = (passes - 1 - pass) & 1;
        const uint2 *from = buffer[into ^ 1];
        uint2 *to = buffer[into];
        const int64_t warps = (int64_t)cluster * WARPS;
        const int64_t each = (count + warps * 32 - 1) / (warps * 32) * 32;
        const int64_t begin = min((int64_t)count, (rank * WARPS + warp) * each), end = min((int64_t)count, begin + each);
        auto entry = [&](int64_t i, uint2 &e) -> uint32_t {      // the digit; kBins: no entry
            if (i >= end) return kBins;
            if (pass == 0) {
                const int64_t id = (int64_t)ids[i];
                if (id < 0 || id >= vocab || id == padding) return kBins;
                e = make_uint2((uint32_t)id, (uint32_t)i);
            } else {
                e = from[i];
            }
            return (e.x >> (pass * kDigitBits)) & (kBins - 1);
        };
        for (int b = lane; b < kBins; b += 32) hist[warp][b] = 0;
        __syncwarp();
        for (int64_t i = begin; i < end; i += 32) {
            uint2 e;
            const uint32_t d = entry(i + lane, e);
            const uint32_t peers = __match_any_sync(0xffffffffu, d);
            if (d < kBins && (peers & below) == 0) hist[warp][d] += __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        uint32_t column[WARPS], sum = 0;         // a bin's counts, all in flight at once
        if (tid < kBins) {
#pragma unroll
            for (int w = 0; w < WARPS; ++w) column[w] = hist[w][tid];
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const uint32_t t = column[w];
                column[w] = sum;
                sum += t;
            }
            total[tid] = sum;
        }
        sort_meet(cluster);
        uint32_t mine = 0, before = 0, inclusive = 0;
        if (tid < kBins) {
            if (cluster == 1) {
                mine = sum;
            } else {
                uint32_t v[kMaxCluster];
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r) v[r] = r < cluster ? peer_word(&total[tid], r) : 0;
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r) {
                    if (r < rank) before += v[r];
                    mine += v[r];
                }
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
        if (tid < kBins) {
            before += inclusive - mine;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) hist[w][tid] = before + column[w];
        }
        __syncthreads();
        for (int64_t i = begin; i < end; i += 32) {
            uint2 e;
            const uint32_t d = entry(i + lane, e);
            const uint32_t peers = __match_any_sync(0xffffffffu, d);
            if (d < kBins) to[hist[warp][d] + __popc(peers & below)] = e;
            __syncwarp();
            if (d < kBins && (peers & below) == 0) hist[warp][d] += __popc(peers);
            __syncwarp();
        }
        count = (int)all;
        sort_meet(cluster);     // the entries are in place, and nobody reads a peer's counts any more
    }
    if (rank == 0 && tid == 0) counts[part] = count;
}

// ---- sums ---------------------------------------------------------------------------------------------------------------

struct GradArgs {
    const void *dy;
    float *dtable, *pieces;      // pieces [partitions][tiles][width]: what a tile adds to a sum that began before it
    const uint2 *pairs;
    const int32_t *counts;       // null: no tokens
    int64_t tokens, vocab, ld_dy, ld_row, ld_partition;
    int width, tile, tiles;
    float scale;
};

constexpr int kSumThreads = 128;

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

// A tile of the sorted tokens for a slab of columns: `across` threads, a vector of columns each, walk the tile's tokens and
// write a sum wherever the number changes: into the table's row where the number's first token is in this tile, into the
// tile's row of pieces where it is not.
template <typename T, int VEC>
__device__ __forceinline__ void sum_tile(const GradArgs &a, unsigned block, int across, int slabs) {
    constexpr int kUnroll = 8;
    const int per_block = kSumThreads / across;
    const int groups = (a.tiles + per_block - 1) / per_block;
    const unsigned item = block / (unsigned)slabs;
    const int slab = (int)(block % (unsigned)slabs);
    const int64_t part = item / (unsigned)groups;
    const int tile = (int)(item % (unsigned)groups) * per_block + (int)threadIdx.x / across;
    const int col = (slab * across + (int)threadIdx.x % across) * VEC;
    const int64_t first = (int64_t)tile * a.tile, n = a.counts[part];
    if (first >= n || col >= a.width) return;
    const int count = (int)min((int64_t)a.tile, n - first);
    const uint2 *pairs = a.pairs + part * 2 * a.tokens + first;
    const T *dy = static_cast<const T *>(a.dy) + part * a.tokens * a.ld_dy + col;
    float *table = a.dtable + part * a.ld_partition + col;
    float *piece = a.pieces + (part * a.tiles + tile) * a.width + col;
    bool began_before = first > 0 && pairs[-1].x == pairs[0].x;
    float acc[VEC] = {};
    for (int t0 = 0; t0 < count; t0 += kUnroll) {
        uint2 e[kUnroll + 1];
        Packed<T, VEC> r[kUnroll];
#pragma unroll
        for (int u = 0; u <= kUnroll; ++u) e[u] = t0 + u < count ? pairs[t0 + u] : make_uint2(0xffffffffu, 0);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (t0 + u < count) r[u] = load_packed<T, VEC>(dy + (int64_t)e[u].y * a.ld_dy);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (t0 + u >= count) break;
            float f[VEC];
            unpack<T, VEC>(r[u], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += f[i];
            if (e[u + 1].x != e[u].x) {
                if (began_before) store_floats<VEC>(piece, acc, 1.f);
                else store_floats<VEC>(table + (int64_t)e[u].x * a.ld_row, acc, a.scale);
                began_before = false;
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
            }
        }
    }
}

// Rows that no token names.  A block looks its 32 numbers up in the sorted tokens.
constexpr int kZeroRows = 32;
template <int VEC>
__device__ __forceinline__ void zero_rows(const GradArgs &a, unsigned block, unsigned ranges) {
    __shared__ uint32_t named;
    const int64_t part = block / ranges, v0 = (int64_t)(block % ranges) * kZeroRows;
    const int rows = (int)min((int64_t)kZeroRows, a.vocab - v0);
    if (threadIdx.x == 0) named = 0;
    if (a.counts) {
        const uint2 *pairs = a.pairs + part * 2 * a.tokens;
        const int64_t n = a.counts[part];
        int64_t low = 0, high = n;
        while (low < high) {
            const int64_t mid = (low + high) / 2;
            if ((int64_t)pairs[mid].x < v0) low = mid + 1;
            else high = mid;
        }
        __syncthreads();
        for (int64_t i = low + (int)threadIdx.x; i < n; i += kSumThreads) {
            const int64_t v = (int64_t)pairs[i].x - v0;
            if (v >= rows) break;
            atomicOr(&named, 1u << v);
        }
    }
    __syncthreads();
    const int nvec = a.width / VEC;
    const float zero[VEC] = {};
    const uint32_t bits = named;
    for (int r = 0; r < rows; ++r) {
        if (bits >> r & 1u) continue;
        float *out = a.dtable + part * a.ld_partition + (v0 + r) * a.ld_row;
        for (int v = (int)threadIdx.x; v < nvec; v += kSumThreads) store_floats<VEC>(out + v * VEC, zero, 1.f);
    }
}

// Both in one grid: the first `sum_blocks` blocks take tiles, the others ranges of rows.  Bound by memory.
template <typename T, int VEC, int ZERO>
__global__ void __launch_bounds__(kSumThreads) cr_embedding_sums_kernel(const GradArgs a, unsigned sum_blocks, int across, int slabs, unsigned ranges) {
    if (blockIdx.x < sum_blocks) sum_tile<T, VEC>(a, blockIdx.x, across, slabs);
    else zero_rows<ZERO>(a, blockIdx.x - sum_blocks, ranges);
}

// Numbers whose tokens reach into further tiles: the block of the first such tile adds the tiles' pieces to the row.  `across`
// threads take a vector of columns each; the block's threads / across of them that share a column take every such piece each
// and are summed in order.
constexpr int kJoinThreads = 256;
template <int VEC>
__global__ void __launch_bounds__(kJoinThreads) cr_embedding_join_kernel(const GradArgs a, int across, int slabs) {
    constexpr int kUnroll = 4;
    __shared__ float sm[kJoinThreads * VEC];
    const unsigned item = blockIdx.x / (unsigned)slabs;
    const int deep = kJoinThreads / across, col0 = (int)threadIdx.x % across, row = (int)threadIdx.x / across;
    const int col = ((int)(blockIdx.x % (unsigned)slabs) * across + col0) * VEC;
    const int64_t part = item / (unsigned)(a.tiles - 1);
    const int64_t tile = item % (unsigned)(a.tiles - 1) + 1, n = a.counts[part];
    const uint2 *pairs = a.pairs + part * 2 * a.tokens;
    if (tile * a.tile >= n) return;
    const uint32_t number = pairs[tile * a.tile].x, earlier = pairs[tile * a.tile - 1].x;
    const uint32_t before = tile > 1 ? pairs[(tile - 1) * a.tile - 1].x : 0xffffffffu;
    if (earlier != number || before == number) return;       // nothing reaches into this tile, or it comes from further back
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

int tile_tokens(int64_t tokens) {
    // 32 tokens; longer tiles where there would be more than 4096 of them to join
    int64_t tile = 32;
    while (tokens / tile > 4096) tile *= 2;
    return (int)tile;
}
size_t align16(size_t b) { return (b + 15) / 16 * 16; }

}  // namespace

size_t embedding_backward_workspace_bytes(int64_t tokens, int64_t partitions, int64_t width) {
    if (tokens == 0) return 0;
    const int64_t tile = tile_tokens(tokens), tiles = (tokens + tile - 1) / tile;
    return align16((size_t)(partitions * tokens * 16)) + align16((size_t)partitions * 4) + (size_t)(tiles > 1 ? partitions * tiles * width * 4 : 0);
}

cudaError_t launch_embedding(const EmbeddingArgs &a, cudaStream_t stream, int64_t *launches) {
    if (a.tokens == 0 || a.width == 0) return cudaSuccess;
    return by_type(a.elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const bool wide = vector_rows(a.elem, a.width, {a.table, a.y}, {a.ld_table, a.ld_y});
        const int nvec = (int)(wide ? a.width / VEC : a.width);
        int per_row = 1;
        while (per_row < kLookupThreads && per_row * 4 < nvec) per_row *= 2;
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

cudaError_t launch_embedding_backward(const EmbeddingArgs &a, void *workspace, cudaStream_t stream, int64_t *launches) {
    if (a.partitions == 0 || a.vocab == 0 || a.width == 0) return cudaSuccess;
    GradArgs g = {};
    g.dy = a.dy; g.dtable = a.dtable; g.tokens = a.tokens; g.vocab = a.vocab;
    g.ld_dy = a.ld_dy; g.ld_row = a.ld_row; g.ld_partition = a.ld_partition;
    g.width = (int)a.width; g.scale = a.scale;
    cudaError_t e;
    const bool table16 = aligned16(a.dtable) && a.ld_row % 4 == 0 && (a.partitions == 1 || a.ld_partition % 4 == 0);
    if (a.tokens > 0) {
        g.tile = tile_tokens(a.tokens);
        g.tiles = (int)((a.tokens + g.tile - 1) / g.tile);
        uint2 *pairs = static_cast<uint2 *>(workspace);
        int32_t *counts = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + align16((size_t)(a.partitions * a.tokens * 16)));
        g.pairs = pairs;
        g.counts = counts;
        g.pieces = reinterpret_cast<float *>(reinterpret_cast<char *>(counts) + align16((size_t)a.partitions * 4));
        int bits = 1;
        while (bits < 31 && (1ll << bits) < a.vocab) ++bits;
        const int passes = (bits + kDigitBits - 1) / kDigitBits;
        // a CTA's warps take 32 tokens at a time: eight warps a partition up to 1024 tokens, from there on 32 warps a CTA
        const bool small = a.tokens <= 1024;
        int cluster = 1;
        while (!small && cluster < kMaxCluster && a.tokens > (int64_t)cluster * 2048) cluster *= 2;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(a.partitions * cluster));
        cfg.blockDim = dim3(small ? 256 : 1024);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 1 : 0;
        auto sort = [&](auto i, auto kernel) {
            return cudaLaunchKernelEx(&cfg, kernel, static_cast<const decltype(i) *>(a.ids), (int)a.tokens, a.vocab, a.padding, passes, pairs, counts, cluster);
        };
        if (a.id_bytes == 4) e = small ? sort(int32_t{}, cr_token_sort_kernel<int32_t, 8>) : sort(int32_t{}, cr_token_sort_kernel<int32_t, 32>);
        else e = small ? sort((long long){}, cr_token_sort_kernel<long long, 8>) : sort((long long){}, cr_token_sort_kernel<long long, 32>);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    const int64_t ranges = (a.vocab + kZeroRows - 1) / kZeroRows;
    e = by_type(a.elem, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T);
        const bool wide = table16 && vector_rows(a.elem, a.width, {a.dy}, {a.ld_dy});
        const int nvec = g.width / (wide ? VEC : 1);
        int across = 1;
        while (across < kSumThreads && across < nvec) across *= 2;
        const int slabs = (nvec + across - 1) / across;
        const int64_t groups = (g.tiles + kSumThreads / across - 1) / (kSumThreads / across);
        if (a.partitions * groups > 0x3fffffffll / slabs || a.partitions > 0x3fffffffll / ranges) return cudaErrorInvalidValue;
        const unsigned sums = (unsigned)(a.partitions * groups * slabs), blocks = sums + (unsigned)(a.partitions * ranges);
        const bool zero4 = table16 && g.width % 4 == 0;
        if (wide) cr_embedding_sums_kernel<T, VEC, 4><<<blocks, kSumThreads, 0, stream>>>(g, sums, across, slabs, (unsigned)ranges);
        else if (zero4) cr_embedding_sums_kernel<T, 1, 4><<<blocks, kSumThreads, 0, stream>>>(g, sums, across, slabs, (unsigned)ranges);
        else cr_embedding_sums_kernel<T, 1, 1><<<blocks, kSumThreads, 0, stream>>>(g, sums, across, slabs, (unsigned)ranges);
        return cudaGetLastError();
    });
    if (e != cudaSuccess) return e;
    ++*launches;
    if (g.tiles > 1) {
        const bool four = table16 && g.width % 4 == 0;
        const int nvec = four ? g.width / 4 : g.width;
        int across = 1;
        while (across < 64 && across < nvec) across *= 2;
        const int slabs = (nvec + across - 1) / across;
        if (a.partitions * (g.tiles - 1) > 0x7fffffffll / slabs) return cudaErrorInvalidValue;
        const unsigned blocks = (unsigned)(a.partitions * (g.tiles - 1) * slabs);
        if (four) cr_embedding_join_kernel<4><<<blocks, kJoinThreads, 0, stream>>>(g, across, slabs);
        else cr_embedding_join_kernel<1><<<blocks, kJoinThreads, 0, stream>>>(g, across, slabs);
        e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
    }
    return e;
}

}  // namespace cr
