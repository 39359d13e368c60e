// Rows of logits over a vocabulary: log probabilities of given tokens with entropy and the best alternatives, distillation from a
// teacher's top logits, and their gradients.
//
//   z = x / T,  lse = log sum_v e^{z_v},  logp = z_id - lse,  H = lse - sum_v p_v z_v,  p_v = e^{z_v - lse}
//   dx_v = (1/T) (a (1[v = id] - p_v) - b p_v (log p_v + H))                      a = d logp, b = d H
//   t = softmax over the teacher's k logits / T,  loss = T^2 sum_j t_j (log t_j - log p_{id_j}),  dx_v = w T (p_v - sum_{j: id_j = v} t_j)
//
// With c = log2(e) / T and the row's largest logit m, e^{z_v - m/T} = 2^{(x_v - m) c}.  The difference comes first: it is exact
// near m, and a row whose logits are all the type's lowest value stays in range; the teacher's logits are taken relative to their
// largest in the same way, and a log p is formed without base two, which would take the lowest value out of range.  What a row keeps for its gradient is m and
// log sum_v e^{(x_v - m)/T}, not their sum, which would round the second one away where m is large.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "cr_elem.cuh"

namespace cr {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
// Exponents below this are zero in fp32; the clamp keeps 0 * -infinity out of the entropy.
constexpr float kLeast = -160.f;
constexpr int kMaxCluster = 8, kScoreWarps = 8, kDistillWarps = 8;

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_nan(float v) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float finite_base(float m) { return isinf(m) ? 0.f : m; }
// log p of a logit from the logarithm to base two of its row's sum.  Without the detour over base two for the logit itself: that of
// one at the type's lowest value, times log2(e), would leave the range.
__device__ __forceinline__ float natural_log_p(float x, float base, float inverse, float log2_sum) { return (x - base) * inverse - kLn2 * log2_sum; }

// ---- a cluster of CTAs on a row --------------------------------------------------------------------------------------------

__device__ __forceinline__ void arrive(int cluster) {
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void wait(int cluster) {
    if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void meet(int cluster) {
    if (cluster > 1) {
        arrive(cluster);
        wait(cluster);
    } else {
        __syncthreads();
    }
}
__device__ __forceinline__ uint32_t address_at(const void *p, int rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}

// ---- pieces of a row ---------------------------------------------------------------------------------------------------------
//
// A row is cut into chunks that a warp takes at once, all loads first: kUnroll vectors (or elements, where rows do not lie in
// vectors) a lane, 4 KB of 16-byte vectors.  A chunk yields its largest logit m, sum 2^u and sum 2^u u with u = (x - m) c; they
// go into slots (chunk modulo kSlots, in ascending order where a row is longer than that) and are joined over the slots in
// a fixed order.  So the result depends on the row's length alone, and any number of warps and CTAs may share a row.
constexpr int kSlots = 1024;

template <typename T, int VEC>
struct Chunk {
    static constexpr int kUnroll = VEC == 1 ? 32 : 8;
    static constexpr int kElements = 32 * kUnroll * VEC;
    static constexpr int kLane = kUnroll * VEC;      // elements of a lane
    Packed<T, VEC> r[kUnroll];

    // The index of element i of vector u of a lane.
    static __device__ __forceinline__ int64_t index(int64_t chunk, int lane, int u, int i) { return ((chunk * kUnroll + u) * 32 + lane) * VEC + i; }

    __device__ __forceinline__ void load(const T *x, int64_t vocab, int64_t chunk) {
        const int lane = (int)threadIdx.x % 32;
        const T *p = x + index(chunk, lane, 0, 0);
        if ((chunk + 1) * kElements <= vocab) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) r[u] = load_packed<T, VEC>(p + u * 32 * VEC);
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                float none[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) none[i] = -INFINITY;
                r[u] = index(chunk, lane, u, 0) < vocab ? load_packed<T, VEC>(p + u * 32 * VEC) : pack<T, VEC>(none);
            }
        }
    }
    // The lane's largest logit (NaN if it has one).
    __device__ __forceinline__ float largest() const {
        if constexpr (VEC == 1 || sizeof(T) == 4) {
            float m = -INFINITY;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                float f[VEC];
                unpack<T, VEC>(r[u], f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) m = max_nan(m, f[i]);
            }
            return m;
        } else if constexpr (__is_same(T, __nv_bfloat16)) {
            __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162 *>(&r[0].w[0]);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) m = __hmax2_nan(m, *reinterpret_cast<const __nv_bfloat162 *>(&r[u].w[i]));
            return max_nan(__low2float(m), __high2float(m));
        } else {
            __half2 m = *reinterpret_cast<const __half2 *>(&r[0].w[0]);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) m = __hmax2_nan(m, *reinterpret_cast<const __half2 *>(&r[u].w[i]));
            return max_nan(__low2float(m), __high2float(m));
        }
    }
    // f(a pair of the lane's logits) for all of them.
    template <typename F>
    __device__ __forceinline__ void for_pairs(F &&f) const {
        if constexpr (VEC == 1) {
#pragma unroll
            for (int u = 0; u < kUnroll; u += 2) f(f2(to_float(r[u].e), to_float(r[u + 1].e)));
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                F2 v[VEC / 2];
                unpack2<T, VEC>(r[u], v);
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) f(v[i]);
            }
        }
    }
    // The lane's sum of 2^u, and of 2^u u where it is wanted.
    template <bool TURN>
    __device__ __forceinline__ float2 sums(float base, float c) const {
        const F2 shift = f2(-base), factor = f2(c);
        F2 s = f2(0.f), t = f2(0.f);
        for_pairs([&](F2 v) {
            F2 w = mul2(add2(v, shift), factor);
            if constexpr (TURN) w = f2(max_nan(low(w), kLeast), max_nan(high(w), kLeast));
            const F2 e = f2(exp2_approx(low(w)), exp2_approx(high(w)));
            s = add2(s, e);
            if constexpr (TURN) t = fma2(e, w, t);
        });
        return make_float2(low(s) + high(s), low(t) + high(t));
    }
    // Puts f(pair) in the places of the lane's pairs, in a row of the chunk's layout.
    template <typename F>
    __device__ __forceinline__ void store(T *d, int64_t vocab, int64_t chunk, F &&f) const {
        const int lane = (int)threadIdx.x % 32;
        T *p = d + index(chunk, lane, 0, 0);
        const bool full = (chunk + 1) * kElements <= vocab;
        // vectors (or elements) of the lane that lie in the row
        const int have = full ? kUnroll : (int)max((int64_t)0, min((int64_t)kUnroll, (vocab / VEC - chunk * kUnroll * 32 - lane + 31) / 32));
        if constexpr (VEC == 1) {
#pragma unroll
            for (int u = 0; u < kUnroll; u += 2) {
                const F2 v = f(f2(to_float(r[u].e), to_float(r[u + 1].e)));
                if (full || u < have) p[u * 32] = from_float<T>(low(v));
                if (full || u + 1 < have) p[(u + 1) * 32] = from_float<T>(high(v));
            }
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                F2 v[VEC / 2];
                unpack2<T, VEC>(r[u], v);
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) v[i] = f(v[i]);
                if (full || u < have) store_packed<T, VEC>(p + u * 32 * VEC, pack2<T, VEC>(v));
            }
        }
    }
};

struct Piece {
    float m, sum, turn, unused;
};
// b's numbers added to a's, relative to a's largest logit.
template <bool TURN>
__device__ __forceinline__ void add_piece(Piece &a, const Piece &b, float c) {
    if (b.m == -INFINITY) return;
    const float d = max_nan((finite_base(b.m) - finite_base(a.m)) * c, kLeast), f = exp2_approx(d);
    a.sum = fmaf(b.sum, f, a.sum);
    if constexpr (TURN) a.turn = fmaf(fmaf(b.sum, d, b.turn), f, a.turn);
}
// Joins the slots; every lane gets the result.
template <bool TURN>
__device__ __forceinline__ Piece join(const Piece *slots, int count, float c) {
    const int lane = (int)threadIdx.x % 32;
    float m = -INFINITY;
    for (int j = lane; j < count; j += 32) m = max_nan(m, slots[j].m);
    Piece a = {warp_max_nan(m), 0.f, 0.f, 0.f};
    for (int j = lane; j < count; j += 32) add_piece<TURN>(a, slots[j], c);
    a.sum = warp_sum(a.sum);
    if constexpr (TURN) a.turn = warp_sum(a.turn);
    return a;
}

__device__ __forceinline__ int64_t id_at(const void *ids, int id_bytes, int64_t i) {
    return id_bytes == 4 ? (int64_t)static_cast<const int32_t *>(ids)[i] : (int64_t)static_cast<const long long *>(ids)[i];
}

// ---- the best alternatives ------------------------------------------------------------------------------------------------

// Position in the order of the alternatives: the larger value first, then the lower index; a NaN above everything.
// No logit has the place 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);     // -0 counts as 0
    return x != x ? 0xffffffffu : (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long rank_key(uint32_t order, uint32_t index) { return (unsigned long long)order << 32 | (0xffffffffu - index); }
__device__ __forceinline__ float key_value(unsigned long long key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float((order >> 31) ? order & 0x7fffffffu : ~order);
}

// 32 values in descending order, one a lane.
__device__ __forceinline__ uint32_t sort_list(uint32_t v) {
    const int lane = (int)threadIdx.x % 32;
#pragma unroll
    for (int k = 2; k <= 32; k *= 2)
#pragma unroll
        for (int j = k / 2; j > 0; j /= 2) {
            const uint32_t o = __shfl_xor_sync(0xffffffffu, v, j);
            v = ((lane & k) == 0) == ((lane & j) == 0) ? max(v, o) : min(v, o);
        }
    return v;
}
// The 32 largest of two sorted lists, sorted.
__device__ __forceinline__ uint32_t merge_lists(uint32_t a, uint32_t b) {
    const int lane = (int)threadIdx.x % 32;
    uint32_t v = max(a, __shfl_sync(0xffffffffu, b, 31 - lane));
#pragma unroll
    for (int j = 16; j > 0; j /= 2) {
        const uint32_t o = __shfl_xor_sync(0xffffffffu, v, j);
        v = (lane & j) == 0 ? max(v, o) : min(v, o);
    }
    return v;
}

// A warp keeps this many logits that reach the bound; where ties bring more, it goes over them again with a sorted list.
constexpr int kKept = 64;

// Log probability, entropy and alternatives.  Phase one: a warp a chunk; besides the sums each lane leaves the place of its
// largest logit, and each warp sorts its lanes' largest.  The k-th of these, merged over the warps, is a bound that at least k
// logits reach, and hardly more than k do.  Phase two: only the lanes whose largest reaches the bound have their elements
// read again (32 or 64 each, from L2), four lanes' at a time; what reaches the bound is kept, and as all keys differ, counting
// the larger ones gives each its rank.  The CTAs of a cluster hand the leader their k best.  4096 x 32000 bf16: 52 us without
// alternatives (5.0 TB/s), 72 with 20 of them, whose steps are short and wait for each other.  Five blocks of eight warps leave 48
// registers, of which 72 to 96 bytes are spilled.
template <typename T, int VEC>
__global__ void __launch_bounds__(32 * kScoreWarps, 5) cr_token_log_probs_kernel(const VocabArgs a, int cluster, int slots) {
    using C = Chunk<T, VEC>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ uint32_t lists[kScoreWarps][32];
    __shared__ int found;
    __shared__ unsigned long long keys[kScoreWarps][kKept], together[kScoreWarps * kKept], ranked[kMaxCluster * 32];
    Piece *pieces = reinterpret_cast<Piece *>(dynamic);                                    // [slots], the leader's are used
    uint32_t *tops = reinterpret_cast<uint32_t *>(pieces + slots);                         // [own slots][32]
    const int rank = (int)(blockIdx.x % (unsigned)cluster);
    const int64_t row = blockIdx.x / (unsigned)cluster;
    const int warps = (int)blockDim.x / 32, warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x % 32;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    const float c = a.inverse * kLog2e;
    const int64_t chunks = (a.vocab + C::kElements - 1) / C::kElements;
    const int own = (slots - rank + cluster - 1) / cluster;
    if (a.top > 0) {
        for (int i = threadIdx.x; i < kMaxCluster * 32; i += blockDim.x) ranked[i] = 0;
        if (threadIdx.x == 0) found = 0;
    }
    arrive(cluster);                     // a CTA's memory may be written from outside only once it runs
    int64_t id = -1;
    float picked = 0.f;
    if (a.logp && rank == 0 && warp == 0) {
        id = id_at(a.ids, a.id_bytes, row);
        if (id < 0 || id >= a.vocab) id = -1;
        else picked = to_float(x[id]);
    }
    bool started = false;
    uint32_t best = 0;
    for (int k = warp; k < own; k += warps) {
        const int slot = k * cluster + rank;
        Piece p = {-INFINITY, 0.f, 0.f, 0.f};
        uint32_t lane_top = 0;
        for (int64_t chunk = slot; chunk < chunks; chunk += kSlots) {
            C d;
            d.load(x, a.vocab, chunk);
            const float lm = d.largest();
            Piece q = {warp_max_nan(lm), 0.f, 0.f, 0.f};
            const float2 s = a.entropy ? d.template sums<true>(finite_base(q.m), c) : d.template sums<false>(finite_base(q.m), c);
            q.sum = warp_sum(s.x);
            if (a.entropy) q.turn = warp_sum(s.y);
            if (q.m == -INFINITY) q.sum = q.turn = 0.f;
            if (chunk == slot) {
                p = q;
            } else {
                Piece all = {max_nan(p.m, q.m), 0.f, 0.f, 0.f};
                add_piece<true>(all, p, c);
                add_piece<true>(all, q, c);
                p = all;
            }
            if (C::index(chunk, lane, 0, 0) < a.vocab) lane_top = max(lane_top, order_of(lm));
        }
        if (a.top > 0) {
            tops[k * 32 + lane] = lane_top;
            best = max(best, lane_top);
        }
        if (!started) wait(cluster);
        started = true;
        if (lane == 0) {
            if (cluster == 1) {
                pieces[slot] = p;
            } else {
                asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(address_at(&pieces[slot], 0)), "f"(p.m), "f"(p.sum), "f"(p.turn), "f"(0.f)
                             : "memory");
            }
        }
    }
    if (!started) wait(cluster);
    if (a.top > 0) lists[warp][lane] = best = sort_list(best);
    meet(cluster);
    __shared__ float result[2];
    if (rank == 0 && warp == 0) {
        const Piece all = join<true>(pieces, slots, c);
        const float base = finite_base(all.m), log_sum = log2f(all.sum);
        const bool nothing = all.m == -INFINITY;
        if (lane == 0) {
            if (a.stats) reinterpret_cast<float2 *>(a.stats)[row] = make_float2(all.m, kLn2 * log_sum);
            if (a.entropy) a.entropy[row] = nothing ? 0.f : kLn2 * (log_sum - all.turn / all.sum);
            if (a.logp) a.logp[row] = id < 0 ? 0.f : nothing ? -INFINITY : natural_log_p(picked, base, a.inverse, log_sum);
            result[0] = base;
            result[1] = log_sum;
        }
    }
    if (a.top == 0) return;
    for (int half = kScoreWarps / 2; half > 0; half /= 2) {
        if (half >= warps) continue;
        if (warp < half && warp + half < warps) lists[warp][lane] = best = merge_lists(best, lists[warp + half][lane]);
        __syncthreads();
    }
    const uint32_t bound = max(1u, lists[0][a.top - 1]);
    const float bound_value = key_value((unsigned long long)bound << 32);
    int count = 0;
    const uint32_t below = (1u << lane) - 1u;
    constexpr int kGroups = 32 / C::kUnroll;          // lanes' elements that the warp looks at together, a vector a lane
    for (int k = warp; k < own; k += warps) {
        const int slot = k * cluster + rank;
        uint32_t groups = __ballot_sync(0xffffffffu, tops[k * 32 + lane] >= bound);
        while (groups) {
            int g = -1;
#pragma unroll
            for (int b = 0; b < kGroups; ++b) {
                if (lane / C::kUnroll == b) g = __ffs(groups) - 1;
                groups &= groups - 1;
            }
            for (int64_t chunk = slot; chunk < chunks; chunk += kSlots) {
                const int64_t v = C::index(chunk, g, lane % C::kUnroll, 0);
                const bool in = g >= 0 && v < a.vocab;
                float f[VEC];
                if (in) unpack<T, VEC>(load_packed<T, VEC>(x + v), f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const bool reaches = in && !(f[i] < bound_value);      // a NaN does
                    const uint32_t some = __ballot_sync(0xffffffffu, reaches);
                    if (some == 0) continue;
                    const int at = count + __popc(some & below);
                    if (reaches && at < kKept) keys[warp][at] = rank_key(order_of(f[i]), (uint32_t)(v + i));
                    count += __popc(some);
                }
            }
        }
    }
    if (count > kKept) {
        // the warp's best in a sorted list, and the a.top-th of them
        unsigned long long list = 0, last = 0;
        for (int k = warp; k < own; k += warps) {
            const int slot = k * cluster + rank;
            const uint32_t t = tops[k * 32 + lane];
            for (uint32_t groups = __ballot_sync(0xffffffffu, t >= bound); groups; groups &= groups - 1) {
                const int g = __ffs(groups) - 1;
                // the best that this lane's elements can be
                if (rank_key(__shfl_sync(0xffffffffu, t, g), (uint32_t)C::index(slot, g, 0, 0)) <= last) continue;
                for (int64_t chunk = slot; chunk < chunks; chunk += kSlots) {
#pragma unroll 1
                    for (int q = 0; q < C::kLane; q += 32) {
                        const int64_t v = C::index(chunk, g, (q + lane) / VEC, (q + lane) % VEC);
                        const unsigned long long key = v < a.vocab ? rank_key(order_of(to_float(x[v])), (uint32_t)v) : 0;
                        for (uint32_t some = __ballot_sync(0xffffffffu, key > last); some; some &= some - 1) {
                            const unsigned long long next = __shfl_sync(0xffffffffu, key, __ffs(some) - 1);
                            if (next <= last) continue;
                            const int place = __popc(__ballot_sync(0xffffffffu, list > next));
                            const unsigned long long up = __shfl_up_sync(0xffffffffu, list, 1);
                            list = lane < place ? list : lane == place ? next : up;
                            last = __shfl_sync(0xffffffffu, list, a.top - 1);
                        }
                    }
                }
            }
        }
        __syncwarp();
        keys[warp][lane] = list;
        count = a.top;
    }
    __syncwarp();
    int at = 0;
    if (lane == 0 && count > 0) at = atomicAdd(&found, count);
    at = __shfl_sync(0xffffffffu, at, 0);
    for (int i = lane; i < count; i += 32) together[at + i] = keys[warp][i];
    __syncthreads();
    auto put = [&](unsigned long long key, int place) {
        const uint32_t v = 0xffffffffu - (uint32_t)key;
        if (a.id_bytes == 4) static_cast<int32_t *>(a.top_ids)[row * a.top + place] = (int32_t)v;
        else static_cast<long long *>(a.top_ids)[row * a.top + place] = (long long)v;
        const float f = key_value(key);
        a.top_logp[row * a.top + place] = isinf(result[1]) && result[1] < 0.f ? -INFINITY : natural_log_p(f, result[0], a.inverse, result[1]);
    };
    const int n = found;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const unsigned long long key = together[i];
        int place = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) place += together[j] > key;
        if (place >= a.top) continue;
        if (cluster == 1) put(key, place);
        else asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(address_at(&ranked[rank * 32 + place], 0)), "l"(key) : "memory");
    }
    if (cluster == 1) return;
    meet(cluster);
    if (rank != 0) return;
    for (int i = threadIdx.x; i < cluster * 32; i += blockDim.x) {
        const unsigned long long key = ranked[i];
        if (key == 0) continue;
        int place = 0;
        for (int j = 0; j < cluster * 32; ++j) place += ranked[j] > key;
        if (place < a.top) put(key, place);
    }
}

// ---- their gradient ---------------------------------------------------------------------------------------------------------

constexpr int kGradWarps = 8;

// A warp a chunk of a row; all loads come before the first store, which may go to the same memory.  Nothing is summed, so rows off
// the 16-byte boundaries (PEEL) may be taken from their first boundary on, which x and dx have in one place: the elements
// in front of it and behind the last vector are the first chunk's.  Bound by memory: 2048 x 32000 bf16 42 us (6.2 TB/s), 2048 x
// 32001 48 us (67 by elements), 1024 x 50257 fp32 63 us (6.5 TB/s).
template <typename T, int VEC, bool PEEL>
__global__ void __launch_bounds__(32 * kGradWarps, 4) cr_token_log_probs_grad_kernel(const VocabArgs a, unsigned chunks, int64_t items) {
    using C = Chunk<T, VEC>;
    const int64_t item = (int64_t)blockIdx.x * kGradWarps + threadIdx.x / 32;
    if (item >= items) return;
    const int64_t row = item < 0x7fffffffll ? (unsigned)item / chunks : item / chunks, chunk = item - row * chunks;
    const int lane = (int)threadIdx.x % 32;
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    T *d = static_cast<T *>(a.dlogits) + row * a.ld_d;
    int head = 0;
    if constexpr (PEEL) head = (int)min(a.vocab, (int64_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15u)) % 16 / sizeof(T)));
    const int64_t body = PEEL ? (a.vocab - head) / VEC * VEC : a.vocab;
    C data;
    data.load(x + head, body, chunk);
    // lanes 0 .. 7 the head's, 8 .. 15 the tail's (fewer than eight each)
    const int64_t edge = lane < 8 ? (lane < head ? lane : a.vocab) : head + body + lane - 8;
    const bool at_edge = PEEL && chunk == 0 && lane < 16 && edge < a.vocab;
    const float edge_logit = at_edge ? to_float(x[edge]) : 0.f;
    int64_t id = a.dlogp ? id_at(a.ids, a.id_bytes, row) : -1;
    if (id >= a.vocab) id = -1;
    const bool here = id >= head && id < head + body && (id - head) / C::kElements == chunk;
    const float picked = here ? to_float(x[id]) : 0.f;
    const float2 stats = reinterpret_cast<const float2 *>(a.stats)[row];
    const float ga = id >= 0 ? a.dlogp[row] * a.inverse : 0.f, gb = a.dentropy ? a.dentropy[row] * a.inverse : 0.f;
    const bool none = (ga == 0.f && gb == 0.f) || stats.x == -INFINITY;
    // log2 p = (x - base) c - log_sum;  dx = -p (ga + gb (log p + H)), and ga more at the token
    const float c = a.inverse * kLog2e, base = finite_base(stats.x), log_sum = stats.y * kLog2e;
    const float level = gb != 0.f ? fmaf(gb, a.entropy[row], ga) : ga, turn = gb * kLn2;
    auto one = [&](float v, bool token) {
        const float w = max_nan(fmaf(v - base, c, -log_sum), kLeast);
        return (token ? ga : 0.f) + exp2_approx(w) * fmaf(-turn, w, -level);
    };
    __syncwarp();        // every lane has read what the stores may overwrite
    if (at_edge) d[edge] = from_float<T>(none ? 0.f : one(edge_logit, edge == id));
    if (none) {
        data.store(d + head, body, chunk, [](F2) { return f2(0.f); });
        return;
    }
    const F2 shift = f2(-base), factor = f2(c), minus_log = f2(-log_sum), minus_turn = f2(-turn), minus_level = f2(-level);
    data.store(d + head, body, chunk, [&](F2 v) {
        F2 w = fma2(add2(v, shift), factor, minus_log);
        w = f2(max_nan(low(w), kLeast), max_nan(high(w), kLeast));
        return mul2(f2(exp2_approx(low(w)), exp2_approx(high(w))), fma2(minus_turn, w, minus_level));
    });
    if (!here) return;
    __syncwarp();
    if (lane == 0) d[id] = from_float<T>(one(picked, true));
}

// ---- distillation --------------------------------------------------------------------------------------------------------

// Words of the teacher warp's marks: 64 bits a token, so that few of them share one with another.
__host__ __device__ constexpr uint32_t seen_words(int top) {
    uint32_t w = 64;
    while (w < 2u * (uint32_t)top) w *= 2;
    return w;
}

// One warp takes the teacher: its shares, and the loss once the row's sums are there.  The others take a chunk each, keep it in
// registers over the exchange of the sums (the last one, where a warp has several) and write the gradient; then they put in the
// elements of their own chunk that the teacher names, which its warp has worked out.  8192 x 32000 bf16, 64 named: 204 us (5.1 TB/s
// of the bytes that it cannot do without), between the two powers of two an element (113 us of their unit, 16 a clock and SM at
// 1965 MHz) and the memory (163): eight warps a row and four rows an SM hide them best (16 warps 263, 4 warps 217).
template <typename T, int VEC>
__global__ void __launch_bounds__(32 * (kDistillWarps + 1), VEC == 1 ? 3 : 4) cr_distill_kernel(const VocabArgs a, int cluster, int slots, uint32_t words) {
    using C = Chunk<T, VEC>;
    extern __shared__ __align__(16) unsigned char dynamic[];
    Piece *pieces = reinterpret_cast<Piece *>(dynamic);               // [slots]
    float *share = reinterpret_cast<float *>(pieces + slots);         // [top]
    float *logit = share + a.top;
    float *mended = logit + a.top;
    int32_t *named = reinterpret_cast<int32_t *>(mended + a.top);
    __shared__ int wanted;
    uint32_t *seen = reinterpret_cast<uint32_t *>(named + a.top), *twice = seen + words;     // [words] each
    const int rank = (int)(blockIdx.x % (unsigned)cluster);
    const int64_t row = blockIdx.x / (unsigned)cluster;
    const int warps = (int)blockDim.x / 32 - 1, warp = (int)threadIdx.x / 32 - 1, lane = (int)threadIdx.x % 32;   // warp -1: the teacher's
    const T *x = static_cast<const T *>(a.logits) + row * a.ld;
    T *d = a.dlogits ? static_cast<T *>(a.dlogits) + row * a.ld_d : nullptr;
    const float c = a.inverse * kLog2e;
    const float w = a.weight ? a.weight[row] : 1.f;
    const int64_t chunks = (a.vocab + C::kElements - 1) / C::kElements;
    const int own = (slots - rank + cluster - 1) / cluster;
    C data;
    float mass = 0.f, best = -INFINITY;
    arrive(cluster);
    if (warp < 0) {
        for (uint32_t i = lane; d && i < words; i += 32) seen[i] = twice[i] = 0;
#pragma unroll 4
        for (int j = lane; j < a.top; j += 32) {
            const int64_t id = id_at(a.ids, a.id_bytes, row * a.top + j);
            const bool there = id >= 0 && id < a.vocab;
            named[j] = there ? (int32_t)id : -1;
            logit[j] = there ? to_float(x[id]) : 0.f;
            share[j] = there ? a.teacher[row * a.top + j] : -INFINITY;      // as it is: its difference to the largest comes first
            best = max_nan(best, share[j]);
        }
        __syncwarp();
        for (int j = lane; d && j < a.top; j += 32) {
            if (named[j] < 0) continue;
            const uint32_t bit = 1u << (named[j] % 32), word = (uint32_t)(named[j] / 32) % words;
            if (atomicOr(&seen[word], bit) & bit) atomicOr(&twice[word], bit);
        }
        __syncwarp();
        best = warp_max_nan(best);
        for (int j = lane; j < a.top; j += 32) mass += exp2_approx((share[j] - best) * c);
        mass = warp_sum(mass);
        if (lane == 0) wanted = best != -INFINITY;
        wait(cluster);
    } else {
        bool started = false;
        for (int k = warp; k < own; k += warps) {
            const int slot = k * cluster + rank;
            Piece p = {-INFINITY, 0.f, 0.f, 0.f};
            for (int64_t chunk = slot; chunk < chunks; chunk += kSlots) {
                data.load(x, a.vocab, chunk);
                Piece q = {warp_max_nan(data.largest()), 0.f, 0.f, 0.f};
                q.sum = warp_sum(data.template sums<false>(finite_base(q.m), c).x);
                if (q.m == -INFINITY) q.sum = 0.f;
                if (chunk == slot) {
                    p = q;
                } else {
                    Piece all = {max_nan(p.m, q.m), 0.f, 0.f, 0.f};
                    add_piece<false>(all, p, c);
                    add_piece<false>(all, q, c);
                    p = all;
                }
            }
            if (!started) wait(cluster);
            started = true;
            if (cluster == 1) {
                if (lane == 0) pieces[slot] = p;
            } else if (lane < cluster) {
                asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(address_at(&pieces[slot], lane)), "f"(p.m), "f"(p.sum), "f"(0.f), "f"(0.f)
                             : "memory");
            }
        }
        if (!started) wait(cluster);
    }
    meet(cluster);
    const Piece all = join<false>(pieces, slots, c);
    const float base = finite_base(all.m), log_sum = log2f(all.sum);
    const bool left_out = !wanted, empty = all.m == -INFINITY;
    const float scale = w * a.temperature, factor = empty ? 0.f : scale / all.sum;
    // the shares, the loss, and for all warps the gradient at the elements that the teacher names
    if (warp < 0) {
        // T sum_j t_j (log t_j - log p_j): logits are not divided by T here, so that large differences under T < 1 stay in range
        const float between = a.temperature * kLn2 * (log_sum - log2f(mass));
        float loss = 0.f;
        for (int j = lane; j < a.top; j += 32) {
            const float u = share[j] - best, p = left_out ? 0.f : exp2_approx(u * c) / mass;
            share[j] = p;
            if (p != 0.f) loss += p * (empty ? INFINITY : u - (logit[j] - base) + between);
        }
        loss = warp_sum(loss);
        __syncwarp();
        // A token that is named more than once: each of its places gets the sum, in one order.  `seen` has the tokens' bits, `twice`
        // those that came again: few others share a bit with them.
        for (int j0 = 0; d && j0 < a.top; j0 += 32) {
            const int j = j0 + lane;
            const bool again = j < a.top && named[j] >= 0 && (twice[(uint32_t)(named[j] / 32) % words] >> (named[j] % 32) & 1u);
            for (uint32_t some = __ballot_sync(0xffffffffu, again); some; some &= some - 1) {
                const int k = j0 + __ffs(some) - 1;
                float p = 0.f;
                for (int i = lane; i < a.top; i += 32) p += named[i] == named[k] ? share[i] : 0.f;
                p = warp_sum(p);
                if (lane == 0) mended[k] = p;
            }
            __syncwarp();
            if (j < a.top) {      // the gradient there
                const float p = again ? mended[j] : share[j];
                mended[j] = fmaf(exp2_approx((logit[j] - base) * c), factor, -scale * p);
            }
        }
        if (lane == 0 && rank == 0 && a.loss) a.loss[row] = left_out ? 0.f : a.temperature * loss;
    }
    if (!d) return;
    const bool none = left_out || w == 0.f;
    if (!none) __syncthreads();
    if (warp < 0 || warp >= own) return;
    // the warp's slots from the last one back: that one's last chunk is still in registers
    const int last = warp + (own - 1 - warp) / warps * warps;
    bool held = true;
    for (int k = last; k >= 0; k -= warps) {
        const int slot = k * cluster + rank;
        for (int64_t chunk = slot + (chunks - 1 - slot) / kSlots * kSlots; chunk >= 0; chunk -= kSlots) {
            if (!held && !none) data.load(x, a.vocab, chunk);
            held = false;
            if (none) {
                data.store(d, a.vocab, chunk, [](F2) { return f2(0.f); });
                continue;
            }
            data.store(d, a.vocab, chunk, [&](F2 v) {
                const F2 w = mul2(add2(v, f2(-base)), f2(c));
                return mul2(f2(exp2_approx(low(w)), exp2_approx(high(w))), f2(factor));
            });
            __syncwarp();
            const uint32_t first = (uint32_t)chunk * C::kElements;
            for (int j = lane; j < a.top; j += 32)       // a place that names nothing is 2^32 - 1, beyond every chunk's last element
                if ((uint32_t)named[j] - first < (uint32_t)C::kElements) d[named[j]] = from_float<T>(mended[j]);
        }
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

// How a row is shared.  The result does not depend on it.
struct Share {
    int cluster, warps, slots;
};
Share share_row(int64_t rows, int64_t vocab, int64_t chunk_elements, int most_warps, int sm_count) {
    Share s;
    s.slots = (int)std::min<int64_t>(kSlots, (vocab + chunk_elements - 1) / chunk_elements);
    // as many CTAs as leave every SM at most one, while there are slots for them.  That leaves SMs idle where
    // rows are few: 39 rows of 128000 bf16 (two CTAs each) 16.4 us, 75 rows (one) 22.5, no less than 148 rows
    s.cluster = 1;
    while (s.cluster < kMaxCluster && s.cluster * 2 <= s.slots && rows * s.cluster * 2 <= sm_count) s.cluster *= 2;
    const int own = (s.slots + s.cluster - 1) / s.cluster, turns = (own + most_warps - 1) / most_warps;
    s.warps = (own + turns - 1) / turns;       // the fewest that need no more turns
    return s;
}

template <typename K, typename... More>
cudaError_t launch(K kernel, std::atomic<uint64_t> &told, const VocabArgs &a, const Share &s, int threads, size_t smem, cudaStream_t stream, int64_t *launches, More... more) {
    if (a.rows > 0x7fffffffll / s.cluster) return cudaErrorInvalidValue;
    if (smem > 32 * 1024) {
        const cudaError_t e = allow_most_smem(reinterpret_cast<const void *>(kernel), told);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * s.cluster));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = s.cluster > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, s.cluster, s.slots, more...);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

cudaError_t launch_token_log_probs(const VocabArgs &a, const DeviceInfo &dev, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    return by_form(a, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        // Many rows: half the warps a row, so that while one row joins its pieces and ranks its alternatives others are read (4096 x
        // 32000, 20 alternatives: 71 us, with eight warps 77); few rows: as many as fit (128000 x 1 in a cluster: 10 us, with four 13).
        const Share s = share_row(a.rows, a.vocab, Chunk<T, VEC>::kElements, a.rows >= 4 * dev.sm_count ? kScoreWarps / 2 : kScoreWarps, dev.sm_count);
        const size_t smem = (size_t)s.slots * sizeof(Piece) + (a.top > 0 ? (size_t)((s.slots + s.cluster - 1) / s.cluster) * 128 : 0);
        static std::atomic<uint64_t> told{0};
        return launch(cr_token_log_probs_kernel<T, VEC>, told, a, s, 32 * s.warps, smem, stream, launches);
    });
}

cudaError_t launch_token_log_probs_backward(const VocabArgs &a, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    auto go = [&](auto t, auto v, auto peel) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        const int64_t chunks = (a.vocab + Chunk<T, VEC>::kElements - 1) / Chunk<T, VEC>::kElements, items = a.rows * chunks;
        if ((items + kGradWarps - 1) / kGradWarps > 0x7fffffffll) return cudaErrorInvalidValue;
        cr_token_log_probs_grad_kernel<T, VEC, decltype(peel)::value != 0><<<(unsigned)((items + kGradWarps - 1) / kGradWarps), 32 * kGradWarps, 0, stream>>>(
            a, (unsigned)chunks, items);
        const cudaError_t e = cudaGetLastError();
        if (e == cudaSuccess) ++*launches;
        return e;
    };
    return by_form(a, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        if constexpr (VEC == 1 && sizeof(T) == 2) {      // for fp32 the elements alone are as fast (65 against 67 us)
            const uintptr_t apart = reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.dlogits);
            if (apart % 16 == 0 && (a.ld - a.ld_d) * 2 % 16 == 0) return go(t, Int<8>{}, Int<1>{});
        }
        return go(t, v, Int<0>{});
    });
}

cudaError_t launch_distill(const VocabArgs &a, const DeviceInfo &dev, cudaStream_t stream, int64_t *launches) {
    if (a.rows == 0) return cudaSuccess;
    return by_form(a, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int VEC = decltype(v)::value;
        const Share s = share_row(a.rows, a.vocab, Chunk<T, VEC>::kElements, kDistillWarps, dev.sm_count);
        const uint32_t words = seen_words(a.top);
        static std::atomic<uint64_t> told{0};
        return launch(cr_distill_kernel<T, VEC>, told, a, s, 32 * (s.warps + 1), (size_t)s.slots * sizeof(Piece) + (size_t)a.top * 16 + words * 8, stream, launches, words);
    });
}

}  // namespace cr
