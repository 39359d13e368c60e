// Group norm in one pass: a sample's slab of channels stays on chip between its statistics and its output.
//
// The work item is (sample, slab), a slab being neighbouring whole groups, 64 or 128 bytes of channels wide where the
// groups allow it, over all positions.  A cluster of K CTAs holds it in shared memory, each CTA an equal share of the positions,
// each thread up to NV vectors of 16 bytes of one column: x is read once from HBM and y written once, which is the floor
// of the operation.  The clusters are persistent: each keeps one slab and walks over samples, so that what depends on
// the channels is set up once, and while it works on one sample the copies of the next are under way.  A thread copies
// (cp.async) exactly the vectors that it reads itself, so the pipeline needs no barrier and no wait on another thread.
// What a CTA knows of its groups goes to its peers through distributed shared memory, joined in the order of the ranks.
// Measured (floor at the copy bandwidth): forward, 256 samples of 1024 x 256, fp32 98 us (83), bf16 62 (42), bf16 with
// dropout 90; backward, 192 of them, fp32 124 (94), bf16 112 (47), with dropout 134.  fp32 is near the memory.  16-bit
// elements are bound by latency at low occupancy: 20 (forward) and 13 warps an SM fill 2.1 and 1.8 of 4 issue slots a cycle with
// DRAM at a fifth of its peak, and wait for their own previous results and at the two barriers and the exchange of a sample.
// What is issued is about 15 instructions an element forward and 8.5 more for the dropout mask.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <numeric>

#include "cr_elem.cuh"
#include "cr_tcgen05.cuh"

namespace cr {
namespace {

constexpr int kMaxCluster = 8;

// Threads of a CTA, vectors a thread holds at most, and the CTAs an SM is to hold.  A thread's work per vector has to
// carry what it does once per sample (sums, exchange, addresses: about 300 instructions), and the CTAs of an SM have to
// cover each other's barriers, so small CTAs with many vectors a thread win, as far as shared memory (two samples in
// flight) and registers (dz) go.  Measured on 256 samples of 1024 x 256 (forward) and 192 (backward), bf16, us:
// forward 256 threads 3 CTAs 71, 128 threads 6 CTAs 67, 5 CTAs 73; 4 vectors 82; backward 256 threads 2 CTAs 117,
// 128 threads 4 CTAs 114, 5 CTAs 166 (spills).  fp32 has half the elements in a vector and wants twice the vectors in
// the backward pass: 165 with 4, 125 with 8.
constexpr int kTH = 128, kForwardNV = 8, kForwardCTAs = 6;
constexpr int backward_nv(int elem_size) { return elem_size == 4 ? 8 : 4; }
constexpr int backward_ctas(int elem_size) { return elem_size == 4 ? 3 : 4; }
// Bytes of channels of a slab, where the groups allow it.  Wide slabs need more CTAs for an item, narrow ones more
// sectors for a row: forward 74 / 67 / 74 us at 128 / 64 / 32 bytes; fp32 backward 125 at 128 bytes, 136 at 64.
constexpr int kForwardBytes = 64;
constexpr int backward_bytes(int elem_size) { return elem_size == 4 ? 128 : 64; }

struct Slab {
    int sc;              // channels of a slab (the last one of a row may have fewer)
    int slabs;           // slabs per row of channels
    int cluster;         // CTAs per item
    int rows_per_cta;
    int cg;
    int channels;
    int samples;
    int walkers;         // clusters that share the samples of a slab
    int64_t positions;
};

// Where a thread stands in the items of its cluster.
struct Spot {
    int slab, rank, first_sample, rows, width, vpr, rt, col, j, c0, mine;   // j < 0: idle; mine: rows of this thread
    int groups, cv, cv_log;                                               // groups of the slab; vectors per group, its logarithm
    int lanes;           // bit o: lanes that differ in bit o hold rows or columns of the same group; -1: not that simple
    bool full;           // every thread has all its rows
};
template <int VEC, int NV>
__device__ __forceinline__ Spot spot(const Slab &s) {
    Spot p;
    const uint32_t cluster = blockIdx.x / (uint32_t)s.cluster;
    p.rank = (int)(blockIdx.x % (uint32_t)s.cluster);
    p.first_sample = (int)(cluster / (uint32_t)s.slabs);
    p.slab = (int)(cluster % (uint32_t)s.slabs);
    p.rows = (int)max((int64_t)0, min((int64_t)s.rows_per_cta, s.positions - (int64_t)p.rank * s.rows_per_cta));
    p.width = min(s.sc, s.channels - p.slab * s.sc);
    p.vpr = p.width / VEC;
    p.rt = kTH / p.vpr;
    p.col = (int)threadIdx.x % p.vpr;
    const int j = (int)threadIdx.x / p.vpr;
    p.j = j < p.rt ? j : -1;
    p.c0 = p.slab * s.sc + p.col * VEC;
    p.mine = p.j < 0 || p.j >= p.rows ? 0 : (p.rows - p.j + p.rt - 1) / p.rt;
    p.groups = p.width / s.cg;
    p.cv = s.cg / VEC;
    p.cv_log = 31 - __clz(max(p.cv, 1));
    // whole rows in a warp and a power of two of vectors in a group: column bits below cv, row bits from vpr on
    p.lanes = 32 % p.vpr == 0 && s.cg % VEC == 0 && (p.cv & (p.cv - 1)) == 0 ? (p.cv - 1) | (31 & ~(p.vpr - 1)) : -1;
    p.full = kTH % p.vpr == 0 && p.rows == NV * p.rt;
    return p;
}

// Sums the entries [g * per, (g + 1) * per) of `in` into out[g] for g < count: a warp per group, in one order.
template <int kWarps>
__device__ __forceinline__ void fold(const float *in, float *out, int count, int per) {
    const int lane = (int)threadIdx.x & 31;
    for (int g = (int)threadIdx.x >> 5; g < count; g += kWarps) {
        float t = 0.f;
        for (int e = lane; e < per; e += 32) t += in[g * per + e];
#pragma unroll
        for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) out[g] = t;
    }
}

// Sums over the CTA, by group, of N numbers a thread has for each of its groups (one group where a vector lies inside
// it, else one per channel of the vector).  After the barrier in it, group_sum gives any thread any group's sum.
// Where a warp holds whole rows and the groups a power of two of vectors, lanes add up the warp and one number a warp and
// group goes through shared memory; otherwise every entry does.  `lanes`: the lane bits to add over (-1: not that
// simple), `group`: the thread's group.  `area`: kTH * N * kG floats.
template <int N, int VEC, bool UNI, int kWarps>
__device__ __forceinline__ void put_groups(float (&acc)[N][UNI ? 1 : VEC], const Spot &p, int lanes, int group, int cg, float *area, float *sums) {
    constexpr int kG = UNI ? 1 : VEC;
    if (UNI && lanes >= 0) {
        float t[N];
#pragma unroll
        for (int n = 0; n < N; ++n) t[n] = acc[n][0];
#pragma unroll
        for (int b = 0; b < 5; ++b)
            if (lanes >> b & 1) {
#pragma unroll
                for (int n = 0; n < N; ++n) t[n] += __shfl_xor_sync(0xffffffffu, t[n], 1 << b);
            }
        if (((int)threadIdx.x & 31 & lanes) == 0) {
            float *mine = area + group * (N * kWarps) + ((int)threadIdx.x >> 5);
#pragma unroll
            for (int n = 0; n < N; ++n) mine[n * kWarps] = t[n];
        }
        __syncthreads();
    } else {
        if (p.j >= 0) {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < kG; ++i) area[((n * p.vpr + p.col) * kG + i) * p.rt + p.j] = acc[n][i];
        }
        __syncthreads();
        fold<kWarps>(area, sums, N * p.groups, (UNI ? p.cv : cg) * p.rt);
        __syncthreads();
    }
}
template <int N, bool UNI, int kWarps>
__device__ __forceinline__ float group_sum(int n, int g, const Spot &p, const float *area, const float *sums) {
    if (UNI && p.lanes >= 0) {
        const float4 *line = reinterpret_cast<const float4 *>(area + (g * N + n) * kWarps);
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps / 4; ++w) {
            const float4 v = line[w];
            t += (v.x + v.y) + (v.z + v.w);
        }
        return t;
    }
    return sums[n * p.groups + g];
}

__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// The CTAs of a cluster tell each other two numbers per group.  Each writes its numbers into the memory of every CTA
// (itself too) and the write itself counts on that CTA's barrier, so that only the threads that join the numbers wait,
// and nothing is fenced; a barrier of the cluster would wait for the stores of the previous sample as well.  Two boxes
// by turns: a CTA writes into a box again only after it has heard from everybody about the exchange in between, which
// they take part in after they have read this one.
template <int KM>   // KM: most groups of a slab
struct Exchange {
    struct Memory {
        float2 box[2][kMaxCluster][KM];
        uint64_t bars[2];
        int given_up, unused;
    };
    Memory *m;
    int turn = 0;

    // Sets the barriers up; the cluster meets once, since a CTA's memory may be written from outside only once it runs.
    __device__ __forceinline__ void open(Memory *memory, int cluster) {
        m = memory;
        if (cluster > 1) {
            if (threadIdx.x == 0) {
                i8::mbar_init(&m->bars[0], 1);
                i8::mbar_init(&m->bars[1], 1);
                m->given_up = 0;
                asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            }
            cluster_meet();
        }
    }
    // by one thread, before the others' numbers are waited for
    __device__ __forceinline__ void expect(int groups, int cluster) const {
        i8::mbar_expect_tx(&m->bars[turn & 1], (uint32_t)(groups * cluster * 8));
    }
    __device__ __forceinline__ void tell(float2 v, int rank, int g, int cluster) const {
        const uint32_t to = i8::smem_u32(&m->box[turn & 1][rank][g]), bar = i8::smem_u32(&m->bars[turn & 1]);
        for (int r = 0; r < cluster; ++r)
            asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                         ::"r"(i8::map_to_rank(to, (uint32_t)r)), "f"(v.x), "f"(v.y), "r"(i8::map_to_rank(bar, (uint32_t)r)) : "memory");
    }
    // The sums over the cluster of group g, in the order of the ranks.  A wait that runs out is reported, and the numbers are
    // then waited for with a limit of their own: every CTA of the cluster runs and tells its numbers whatever it hears, so they
    // come, and a CTA that went on without them would arrive on a barrier whose phase is not over, decide unlike its
    // peers about a second sum, and might end while a peer's numbers are on their way into its memory.
    __device__ __forceinline__ float2 hear(int g, int cluster, int *status, unsigned long long wait_ns) const {
        uint64_t *bar = &m->bars[turn & 1];
        const uint32_t parity = (uint32_t)((turn >> 1) & 1);
        if (!i8::mbar_wait(bar, parity, &m->given_up, wait_ns)) {
            atomicExch(status, 1);
            if (!i8::mbar_wait(bar, parity, &m->given_up, i8::kSettleNs)) m->given_up = 1;
        }
        float2 t = make_float2(0.f, 0.f);
        for (int r = 0; r < cluster; ++r) {
            const float2 v = m->box[turn & 1][r][g];
            t.x += v.x;
            t.y += v.y;
        }
        return t;
    }
};

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest group have landed (for the thread that issued them).
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
template <typename T>
__device__ __forceinline__ Packed<T, 16 / (int)sizeof(T)> held(const uint4 *at) {
    const uint4 v = *at;
    Packed<T, 16 / (int)sizeof(T)> r;
    r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    return r;
}

// z of the activation, for a pair.  Where the activation has a kink (relu) every step is rounded by itself, in the
// forward and the backward pass alike, so that the slope belongs to the z whose value was stored; elsewhere `scaled`
// = rstd gamma goes in one step.
template <int ACT>
__device__ __forceinline__ F2 z_of(F2 centred, F2 rstd, F2 gamma, F2 scaled, F2 beta) {
    if constexpr (ACT == kActRelu) return add2(mul2(mul2(centred, rstd), gamma), beta);
    return fma2(centred, scaled, beta);
}
__device__ __forceinline__ F2 sigmoid2(F2 z) {
    const F2 t = mul2(z, f2(-kLog2e));
    const F2 d = add2(f2(exp2_approx(low(t)), exp2_approx(high(t))), f2(1.f));
    return f2(recip_approx(low(d)), recip_approx(high(d)));
}

// The pair i of a vector, from one value per group (UNI) or per channel.
template <bool UNI, int N>
__device__ __forceinline__ F2 pair_of(const float (&v)[N], int i) {
    if constexpr (UNI) return f2(v[0]);
    else return f2(v[2 * i], v[2 * i + 1]);
}

// Most groups of a slab: a slab is at most 32 channels wide, or one run of groups that no shorter run aligns (at most
// as many as a vector has elements).  Where vectors lie inside groups these have 4 (fp32) or 8 channels at least.
template <bool UNI>
__host__ __device__ constexpr int most_groups() { return UNI ? 8 : 32; }
// Shared memory of the two kernels behind the vectors; every array at a fixed place, which costs no register.
template <int VEC, bool UNI>
struct ForwardMemory {
    float area[2][kTH * 2 * (UNI ? 1 : VEC)];                // by turns
    float ready[2][most_groups<UNI>()];                      // mean, rstd
    float sums[2 * most_groups<UNI>()];
    int again[2];                                            // by turns
    typename Exchange<most_groups<UNI>()>::Memory exchange;
};
template <int VEC, bool UNI>
struct BackwardMemory {
    float entries[2 * kTH * VEC];                            // [rt][2 * width]: channel sums of the thread rows
    float area[2][kTH * 2 * (UNI ? 1 : VEC)];                // by turns
    float ready[2][2][most_groups<UNI>()];                   // by turns
    float sums[2 * most_groups<UNI>()];
    typename Exchange<most_groups<UNI>()>::Memory exchange;
};

// The vectors of a thread: all NV of them where the CTA's share is full (no branches), else the first `mine`.
template <int NV, typename F>
__device__ __forceinline__ void for_rows(const Spot &p, F &&f) {
    if (p.full) {
#pragma unroll
        for (int k = 0; k < NV; ++k) f(k);
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k < p.mine) f(k);
    }
}

// Sums and squares of 16-bit elements on the tensor cores, four elements of every lane an instruction and no conversion:
// with the lanes' registers r0, r1 as rows 0..7 of A and at the same time as B, entry (i, i) of A B is the sum of the
// squares of what the four lanes of quad i hold, and with ones in rows 8..15 every entry (8 + ., i) is their plain sum.
// (The other entries are not used.)  Products of 16-bit elements are exact in fp32; the accumulator is fp32.
template <typename T>
__device__ __forceinline__ void add_moments(float (&d)[4], uint32_t r0, uint32_t r1) {
    if constexpr (__is_same(T, __nv_bfloat16)) {
        constexpr uint32_t kOnes = 0x3f803f80u;
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %6, %5, %6}, {%4, %5}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(r0), "r"(r1), "r"(kOnes));
    } else {
        constexpr uint32_t kOnes = 0x3c003c00u;
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %6, %5, %6}, {%4, %5}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(r0), "r"(r1), "r"(kOnes));
    }
}

// Forward.  Sums and squares are taken of x - pivot, the pivot being the mean of the group's very first vector (16-bit
// elements: its first value; zero where the tensor cores take the sums: 16-bit elements, up to 8 vectors a row): one pass over the vectors and one exchange.  Where the pivot turns out to lie more than four standard deviations off the mean, the
// squares have lost digits to it, and where their sum has left the range of a float they have lost everything: the item is
// then summed once more around the mean itself (all CTAs of the cluster see the same numbers and decide alike).
// UNI: every vector lies inside one group.
template <typename T, int NV, bool UNI, int ACT>
__global__ void __launch_bounds__(kTH, kForwardCTAs) cr_group_norm_kernel(const GroupNormArgs a, const Slab s) {
    constexpr int VEC = 16 / (int)sizeof(T), NP = VEC / 2, kG = UNI ? 1 : VEC;   // kG: groups a thread may touch
    extern __shared__ __align__(16) float sm[];
    const Spot p = spot<VEC, NV>(s);
    constexpr int KM = most_groups<UNI>();
    ForwardMemory<VEC, UNI> &mem = *reinterpret_cast<ForwardMemory<VEC, UNI> *>(sm + 2 * NV * kTH * 4);
    Exchange<KM> ex;
    ex.open(&mem.exchange, s.cluster);
    const uint32_t mine_at = i8::smem_u32(sm) + threadIdx.x * 16;
    const int64_t row0 = (int64_t)p.first_sample * s.positions + (int64_t)p.rank * s.rows_per_cta + max(p.j, 0);
    const T *src = static_cast<const T *>(a.x) + (row0 * a.ld_x + p.c0);
    T *dst = static_cast<T *>(a.y) + (row0 * a.ld_y + p.c0);
    const int64_t step_x = (int64_t)p.rt * a.ld_x, step_y = (int64_t)p.rt * a.ld_y;
    const int64_t next_x = (int64_t)s.walkers * s.positions * a.ld_x, next_y = (int64_t)s.walkers * s.positions * a.ld_y;
    auto fetch = [&](int buf) {
        const T *from = src;
        for_rows<NV>(p, [&](int k) {
            copy16(mine_at + (uint32_t)(buf * NV + k) * (kTH * 16), from);
            from += step_x;
        });
    };
    fetch(0);
    copies_issued();
    F2 gamma[NP], beta[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        gamma[i] = a.gamma ? f2(__ldg(a.gamma + p.c0 + 2 * i), __ldg(a.gamma + p.c0 + 2 * i + 1)) : f2(1.f);
        beta[i] = a.beta ? f2(__ldg(a.beta + p.c0 + 2 * i), __ldg(a.beta + p.c0 + 2 * i + 1)) : f2(0.f);
    }
    const float inv_all = 1.f / ((float)s.positions * (float)s.cg);
    const int g = (int)threadIdx.x;            // the group this thread joins, if g < p.groups
    int mine_g[kG];
#pragma unroll
    for (int i = 0; i < kG; ++i) mine_g[i] = (p.col * VEC + i) / s.cg;
    // first values of the thread's groups, and of the group it joins
    const T *firsts = static_cast<const T *>(a.x) + ((int64_t)p.first_sample * s.positions * a.ld_x + p.slab * s.sc);
    constexpr int kFirst = UNI && sizeof(T) == 4 ? VEC : 1;   // (16-bit elements hardly come here, and registers are short)
    Packed<T, kFirst> pivots[kG], pivot_g;
    auto pivot_of = [](const Packed<T, kFirst> &first) {
        float f[kFirst], t = 0.f;
        unpack<T, kFirst>(first, f);
#pragma unroll
        for (int i = 0; i < kFirst; ++i) t += f[i];
        return t * (1.f / kFirst);
    };
    constexpr bool kMoments = UNI && sizeof(T) == 2;
    // Quad i of a warp takes the moments of column i % vpr, the rows 4 (i / vpr) + 0..3 of the warp: the slots of other
    // lanes of the same warp.  (Copying in that order would cost a sector a lane.)
    const bool moments = kMoments && p.vpr <= 8 && p.lanes >= 0;
    const int lane = (int)threadIdx.x & 31, quad = lane >> 2;
    const int quad_col = quad % p.vpr, quad_row = quad / p.vpr * 4 + (lane & 3);
    const int quad_slot = (int)threadIdx.x - lane + quad_row * p.vpr + quad_col;
    const int quad_j = ((int)threadIdx.x >> 5) * (32 / p.vpr) + quad_row;
    const int quad_mine = quad_j < p.rows ? (p.rows - quad_j + p.rt - 1) / p.rt : 0;
    const int quad_group = kMoments ? quad_col * VEC / s.cg : 0;
    const int quad_lanes = 31 & ~(4 * (p.vpr - 1)) | 4 * (p.cv - 1);
    auto look_ahead = [&]() {
        if (moments) return;
#pragma unroll
        for (int i = 0; i < kG; ++i) pivots[i] = load_packed<T, kFirst>(firsts + mine_g[i] * s.cg);
        pivot_g = load_packed<T, kFirst>(firsts + (g < p.groups ? g : 0) * s.cg);
        firsts += next_x;
    };
    look_ahead();
    int buf = 0;
    for (int n = p.first_sample; n < s.samples; n += s.walkers, buf ^= 1) {
        float m[kG];
#pragma unroll
        for (int i = 0; i < kG; ++i) m[i] = moments ? 0.f : -pivot_of(pivots[i]);
        float pivot = moments ? 0.f : pivot_of(pivot_g);
        src += next_x;
        if (n + s.walkers < s.samples) {
            fetch(buf ^ 1);
            look_ahead();
        }
        copies_issued();
        copies_landed();
        const uint4 *at = reinterpret_cast<const uint4 *>(sm) + buf * NV * kTH + threadIdx.x;
        F2 less[NP];                           // minus the pivot, then minus the mean
#pragma unroll
        for (int i = 0; i < NP; ++i) less[i] = pair_of<UNI>(m, i);
        for (int pass = 0;; ++pass) {
            float acc[2][kG];
            const bool by_quads = kMoments && moments && pass == 0;
            if (by_quads) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                const uint4 *from = reinterpret_cast<const uint4 *>(sm) + buf * NV * kTH + quad_slot;
                __syncwarp();                  // the lanes' copies have landed, for all lanes
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (p.full || k < quad_mine) v = from[k * kTH];
                    if constexpr (kMoments) {
                        add_moments<T>(d, v.x, v.y);
                        add_moments<T>(d, v.z, v.w);
                    }
                }
                // lane 4 i + i / 2 holds what belongs to quad i
                const bool holds = (lane & 3) == quad >> 1;
                acc[0][0] = holds ? (quad & 1 ? d[3] : d[2]) : 0.f;
                acc[1][0] = holds ? (quad & 1 ? d[1] : d[0]) : 0.f;
            } else {
                F2 t1[NP], t2[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) t1[i] = t2[i] = f2(0.f);
                for_rows<NV>(p, [&](int k) {
                    F2 f[NP];
                    unpack2<T, VEC>(held<T>(at + k * kTH), f);
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const F2 d = add2(f[i], less[i]);
                        t1[i] = add2(t1[i], d);
                        t2[i] = fma2(d, d, t2[i]);
                    }
                });
                if constexpr (UNI) {
#pragma unroll
                    for (int i = 1; i < NP; ++i) {
                        t1[0] = add2(t1[0], t1[i]);
                        t2[0] = add2(t2[0], t2[i]);
                    }
                    acc[0][0] = low(t1[0]) + high(t1[0]);
                    acc[1][0] = low(t2[0]) + high(t2[0]);
                } else {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        acc[0][2 * i] = low(t1[i]);
                        acc[0][2 * i + 1] = high(t1[i]);
                        acc[1][2 * i] = low(t2[i]);
                        acc[1][2 * i + 1] = high(t2[i]);
                    }
                }
            }
            float *my_area = mem.area[ex.turn & 1];
            if (threadIdx.x == 0) {
                mem.again[ex.turn & 1] = 0;
                if (s.cluster > 1) ex.expect(p.groups, s.cluster);
            }
            put_groups<2, VEC, UNI, kTH / 32>(acc, p, by_quads ? quad_lanes : p.lanes, by_quads ? quad_group : p.col >> p.cv_log, s.cg, my_area, mem.sums);
            if (g < p.groups) {
                float total = group_sum<2, UNI, kTH / 32>(0, g, p, my_area, mem.sums), squares = group_sum<2, UNI, kTH / 32>(1, g, p, my_area, mem.sums);
                if (s.cluster > 1) {
                    // y may be x: the peer that holds the first row writes over it once it has heard from this thread, so the
                    // pivot is here before that (the other threads' pivots have gone into the sums)
                    asm volatile("" ::"f"(pivot) : "memory");
                    ex.tell(make_float2(total, squares), p.rank, g, s.cluster);
                    const float2 all = ex.hear(g, s.cluster, a.status, a.wait_ns);
                    total = all.x;
                    squares = all.y;
                }
                const float off = total * inv_all, m2 = not_below_zero(fmaf(-total, off, squares));
                if (pass == 0 && (m2 * 16.f < squares || isinf(squares))) mem.again[ex.turn & 1] = 1;
                const float mean = pivot + off, rstd = 1.f / sqrtf(fmaf(m2, inv_all, a.eps));
                pivot = mean;
                mem.ready[0][g] = mean;
                mem.ready[1][g] = rstd;
                if (a.mean && p.rank == 0) {
                    const int64_t to = (int64_t)n * a.groups + p.slab * (s.sc / s.cg) + g;
                    a.mean[to] = mean;
                    a.rstd[to] = rstd;
                }
            }
            __syncthreads();
            const int more = *const_cast<volatile int *>(&mem.again[ex.turn & 1]);
            ++ex.turn;
#pragma unroll
            for (int i = 0; i < kG; ++i) m[i] = -mem.ready[0][mine_g[i]];
#pragma unroll
            for (int i = 0; i < NP; ++i) less[i] = pair_of<UNI>(m, i);
            if (!more) break;
        }
        F2 scaled[NP], spread[NP];
#pragma unroll
        for (int i = 0; i < kG; ++i) m[i] = mem.ready[1][mine_g[i]];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            spread[i] = pair_of<UNI>(m, i);
            scaled[i] = mul2(spread[i], gamma[i]);
        }
        unsigned long long e = a.drop.offset + (unsigned long long)((row0 + (int64_t)(n - p.first_sample) * s.positions) * s.channels + p.c0);
        T *to = dst;
        for_rows<NV>(p, [&](int k) {
            F2 f[NP];
            unpack2<T, VEC>(held<T>(at + k * kTH), f);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const F2 z = z_of<ACT>(add2(f[i], less[i]), spread[i], gamma[i], scaled[i], beta[i]);
                if constexpr (ACT == kActSilu) f[i] = mul2(z, sigmoid2(z));
                else f[i] = f2(act_value<ACT>(low(z)), act_value<ACT>(high(z)));
            }
            if (a.drop.threshold) {
                drop_select2<VEC>(f, a.drop, e);
#pragma unroll
                for (int i = 0; i < NP; ++i) f[i] = mul2(f[i], f2(a.drop.scale));
                e += (unsigned long long)p.rt * s.channels;
            }
            store_packed<T, VEC>(to, pack2<T, VEC>(f));
            to += step_y;
        });
        dst += next_y;
    }
    if (s.cluster > 1) cluster_meet();         // nobody leaves while a peer may still write to it
}

// Rows of channel sums that a CTA leaves for each sample: the lines of the CTA in this many shares.
constexpr int kShares = 2;

// Backward: x and dy are read once; dz takes the place of dy, in registers.  sum1, sum2 (may be null): the sums of dz and
// of dz xhat of each channel over a share of this CTA's rows of a sample, [samples][cluster][shares] rows of ld_sum;
// `whole`: one row per sample, cluster = 1.
template <typename T, int NV, bool UNI, int ACT>
__global__ void __launch_bounds__(kTH, backward_ctas(sizeof(T))) cr_group_norm_grad_kernel(const GroupNormArgs a, const Slab s, float *sum1, float *sum2, int64_t ld_sum, int whole) {
    constexpr int VEC = 16 / (int)sizeof(T), NP = VEC / 2, kG = UNI ? 1 : VEC;
    extern __shared__ __align__(16) float sm[];
    const Spot p = spot<VEC, NV>(s);
    constexpr int KM = most_groups<UNI>();
    BackwardMemory<VEC, UNI> &mem = *reinterpret_cast<BackwardMemory<VEC, UNI> *>(sm + 4 * NV * kTH * 4);
    Exchange<KM> ex;
    ex.open(&mem.exchange, s.cluster);
    const int both = 2 * p.width;
    const uint32_t mine_at = i8::smem_u32(sm) + threadIdx.x * 16;
    const int64_t row0 = (int64_t)p.first_sample * s.positions + (int64_t)p.rank * s.rows_per_cta + max(p.j, 0);
    const T *src = static_cast<const T *>(a.x) + (row0 * a.ld_x + p.c0);
    const T *up = static_cast<const T *>(a.dy) + (row0 * a.ld_dy + p.c0);
    T *dst = static_cast<T *>(a.y) + (row0 * a.ld_y + p.c0);
    const int64_t step_x = (int64_t)p.rt * a.ld_x, step_dy = (int64_t)p.rt * a.ld_dy, step_y = (int64_t)p.rt * a.ld_y;
    const int64_t next = (int64_t)s.walkers * s.positions;
    auto fetch = [&](int buf) {
        const T *from = src, *from_dy = up;
        for_rows<NV>(p, [&](int k) {
            copy16(mine_at + (uint32_t)(buf * 2 * NV + k) * (kTH * 16), from);
            copy16(mine_at + (uint32_t)((buf * 2 + 1) * NV + k) * (kTH * 16), from_dy);
            from += step_x;
            from_dy += step_dy;
        });
    };
    fetch(0);
    copies_issued();
    const float inv_all = 1.f / ((float)s.positions * (float)s.cg);
    const bool one = s.positions * s.cg == 1;  // groups of one value have m1 = gamma dz and no gradient at all
    const float kept = a.drop.threshold ? a.drop.scale : 1.f;
    const int g = (int)threadIdx.x;            // the group this thread joins, if g < p.groups
    // the group of a channel of the thread: formed anew where it is needed, registers are what this kernel lacks (keeping
    // it: 114 -> 127 us on 192 samples of 1024 x 256, bf16)
    auto group_of = [&](int i) { return (p.col * VEC + i) / s.cg; };
    const float *mean_in = a.mean + (int64_t)p.first_sample * a.groups + p.slab * (s.sc / s.cg);
    const float *rstd_in = a.rstd + (int64_t)p.first_sample * a.groups + p.slab * (s.sc / s.cg);
    float mean[kG], rstd[kG];
    auto look_ahead = [&]() {
#pragma unroll
        for (int i = 0; i < kG; ++i) {
            mean[i] = mean_in[group_of(i)];
            rstd[i] = rstd_in[group_of(i)];
        }
        mean_in += (int64_t)s.walkers * a.groups;
        rstd_in += (int64_t)s.walkers * a.groups;
    };
    look_ahead();
    int buf = 0;
    for (int n = p.first_sample; n < s.samples; n += s.walkers, buf ^= 1) {
        F2 dz[NV][NP], s1[NP], s2[NP], scaled[NP], gamma[ACT == kActRelu ? NP : 1], beta[NP], less[NP], spread[NP];
        {
            float m[kG];
#pragma unroll
            for (int i = 0; i < kG; ++i) m[i] = -mean[i];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                s1[i] = s2[i] = f2(0.f);
                less[i] = pair_of<UNI>(m, i);
                spread[i] = pair_of<UNI>(rstd, i);
                // the parameters are fetched for each sample (from L1): kept, they cost registers that this kernel lacks
                const F2 weight = a.gamma ? f2(__ldg(a.gamma + p.c0 + 2 * i), __ldg(a.gamma + p.c0 + 2 * i + 1)) : f2(1.f);
                if constexpr (ACT == kActRelu) gamma[i] = weight;
                beta[i] = a.beta ? f2(__ldg(a.beta + p.c0 + 2 * i), __ldg(a.beta + p.c0 + 2 * i + 1)) : f2(0.f);
                scaled[i] = mul2(weight, spread[i]);
            }
        }
        if (n + s.walkers < s.samples) {
            src += next * a.ld_x;
            up += next * a.ld_dy;
            fetch(buf ^ 1);
            look_ahead();
        }
        copies_issued();
        copies_landed();
        const uint4 *at_x = reinterpret_cast<const uint4 *>(sm) + buf * 2 * NV * kTH + threadIdx.x, *at_dy = at_x + NV * kTH;
        unsigned long long e = a.drop.offset + (unsigned long long)((row0 + (int64_t)(n - p.first_sample) * s.positions) * s.channels + p.c0);
        // dz without the scale of the kept elements, which the sums and the coefficients of dx take in
        for_rows<NV>(p, [&](int k) {
            F2 f[NP];
            unpack2<T, VEC>(held<T>(at_x + k * kTH), f);
            unpack2<T, VEC>(held<T>(at_dy + k * kTH), dz[k]);
            if (a.drop.threshold) {
                drop_select2<VEC>(dz[k], a.drop, e);
                e += (unsigned long long)p.rt * s.channels;
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const F2 centred = add2(f[i], less[i]);
                if constexpr (ACT != kActNone) {
                    const F2 z = z_of<ACT>(centred, spread[i], gamma[ACT == kActRelu ? i : 0], scaled[i], beta[i]);
                    if constexpr (ACT == kActSilu) {
                        const F2 sg = sigmoid2(z);
                        dz[k][i] = mul2(dz[k][i], mul2(sg, fma2(z, fma2(sg, f2(-1.f), f2(1.f)), f2(1.f))));
                    } else {
                        dz[k][i] = f2(low(z) > 0.f ? low(dz[k][i]) : 0.f, high(z) > 0.f ? high(dz[k][i]) : 0.f);
                    }
                }
                s1[i] = add2(s1[i], dz[k][i]);
                s2[i] = fma2(dz[k][i], centred, s2[i]);
            }
        });
        // the channels' sums, on their way while the groups are joined
        float *my_entries = mem.entries;
        if ((sum1 || sum2) && p.j >= 0) {
            float *mine = my_entries + p.j * both + p.col * VEC;
#pragma unroll
            for (int i = 0; i < NP; i += 2) {
                const F2 u1 = mul2(s1[i], f2(kept)), v1 = mul2(s1[i + 1], f2(kept));
                const F2 u2 = mul2(s2[i], mul2(spread[i], f2(kept))), v2 = mul2(s2[i + 1], mul2(spread[i + 1], f2(kept)));
                *reinterpret_cast<float4 *>(mine + 2 * i) = make_float4(low(u1), high(u1), low(v1), high(v1));
                *reinterpret_cast<float4 *>(mine + p.width + 2 * i) = make_float4(low(u2), high(u2), low(v2), high(v2));
            }
        }
        // the groups' sums of rstd gamma dz and rstd gamma dz (x - mean)
        float acc[2][kG];
        if constexpr (UNI) {
            F2 u1 = mul2(scaled[0], s1[0]), u2 = mul2(scaled[0], s2[0]);
#pragma unroll
            for (int i = 1; i < NP; ++i) {
                u1 = fma2(scaled[i], s1[i], u1);
                u2 = fma2(scaled[i], s2[i], u2);
            }
            acc[0][0] = low(u1) + high(u1);
            acc[1][0] = low(u2) + high(u2);
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const F2 u1 = mul2(scaled[i], s1[i]), u2 = mul2(scaled[i], s2[i]);
                acc[0][2 * i] = low(u1);
                acc[0][2 * i + 1] = high(u1);
                acc[1][2 * i] = low(u2);
                acc[1][2 * i + 1] = high(u2);
            }
        }
        if (s.cluster > 1 && a.y && threadIdx.x == 0) ex.expect(p.groups, s.cluster);
        float *my_area = mem.area[buf];
        put_groups<2, VEC, UNI, kTH / 32>(acc, p, p.lanes, p.col >> p.cv_log, s.cg, my_area, mem.sums);
        // a thread per group joins the CTAs.  dx = rstd (gamma dz - m1 - xhat m2)
        //   = (rstd gamma) dz - M1 - rstd^2 M2 (x - mean),  M1, M2 the means of rstd gamma dz and rstd gamma dz (x - mean)
        if (a.y && g < p.groups) {
            float t1 = group_sum<2, UNI, kTH / 32>(0, g, p, my_area, mem.sums), t2 = group_sum<2, UNI, kTH / 32>(1, g, p, my_area, mem.sums);
            if (s.cluster > 1) {
                ex.tell(make_float2(t1, t2), p.rank, g, s.cluster);
                const float2 all = ex.hear(g, s.cluster, a.status, a.wait_ns);
                t1 = all.x;
                t2 = all.y;
            }
            mem.ready[buf][0][g] = t1 * inv_all;
            mem.ready[buf][1][g] = t2 * inv_all;
        }
        ++ex.turn;
        if (sum1 || sum2) {     // put_groups had a barrier: the entries are there
            if (whole) {
                for (int c = (int)threadIdx.x; c < both; c += kTH) {
                    float t = 0.f;
#pragma unroll 8
                    for (int r = 0; r < p.rt; ++r) t += my_entries[r * both + c];
                    float *out = c < p.width ? sum1 : sum2;
                    if (out) out[(int64_t)n * ld_sum + p.slab * s.sc + (c < p.width ? c : c - p.width)] = t;
                }
            } else {
                for (int w = (int)threadIdx.x; w < kShares * both; w += kTH) {
                    const int share = w / both, c = w - share * both;
                    float t = 0.f;
#pragma unroll 8
                    for (int r = share * p.rt / kShares; r < (share + 1) * p.rt / kShares; ++r) t += my_entries[r * both + c];
                    float *out = c < p.width ? sum1 : sum2;
                    if (out)
                        out[(((int64_t)n * s.cluster + p.rank) * kShares + share) * ld_sum + p.slab * s.sc + (c < p.width ? c : c - p.width)] = t;
                }
            }
        }
        if (a.y) {
            __syncthreads();
            float acc1[kG], acc2[kG];
#pragma unroll
            for (int i = 0; i < kG; ++i) {
                const float r = UNI ? low(spread[0]) : (i & 1 ? high(spread[i / 2]) : low(spread[i / 2]));
                acc1[i] = -kept * mem.ready[buf][0][group_of(i)];
                acc2[i] = -kept * r * r * mem.ready[buf][1][group_of(i)];
            }
            F2 c1[NP], c2[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                c1[i] = pair_of<UNI>(acc1, i);
                c2[i] = pair_of<UNI>(acc2, i);
                scaled[i] = mul2(scaled[i], f2(kept));
            }
            T *to = dst;
            for_rows<NV>(p, [&](int k) {
                F2 f[NP];
                unpack2<T, VEC>(held<T>(at_x + k * kTH), f);
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    f[i] = fma2(scaled[i], dz[k][i], fma2(c2[i], add2(f[i], less[i]), c1[i]));
                    if (one) f[i] = f2(0.f);
                }
                store_packed<T, VEC>(to, pack2<T, VEC>(f));
                to += step_y;
            });
            dst += next * a.ld_y;
        } else {
            __syncthreads();    // the entries are free again
        }
    }
    if (s.cluster > 1) cluster_meet();
}

template <int V> struct Int { static constexpr int value = V; };

// The slab and the cluster of an item, and the vectors a thread holds: false where an item does not fit.
bool choose(int elem, int channels, int groups, int64_t samples, int64_t positions, int bytes, int max_nv, Slab &s, int &nv) {
    const int vec = 16 / elem_bytes(elem);
    if (channels % vec || samples > 0x3fffffff) return false;
    s.cg = channels / groups;
    s.channels = channels;
    s.positions = positions;
    s.samples = (int)samples;
    const int unit = std::lcm(s.cg, vec), wanted = bytes / elem_bytes(elem);
    for (int width = std::min(channels, unit * std::max(1, wanted / unit));; width = std::max(unit, width / 2 / unit * unit)) {
        if (width / vec <= kTH) {
            const int rt = kTH / (width / vec);
            const int64_t deep = (positions + rt - 1) / rt;     // vectors of a column, over the whole item
            int cluster = 1;
            while (cluster < kMaxCluster && deep > (int64_t)max_nv * cluster) cluster *= 2;
            if (deep <= (int64_t)max_nv * cluster) {
                s.sc = width;
                s.slabs = (channels + width - 1) / width;
                s.cluster = cluster;
                s.rows_per_cta = (int)((positions + cluster - 1) / cluster);
                nv = 1;
                while ((int64_t)nv * rt < s.rows_per_cta) nv *= 2;
                return nv <= max_nv;
            }
        }
        if (width == unit) return false;
    }
}

// What a kernel needs to be told once per device, and the clusters that are resident together, asked of the runtime once
// per kernel, device and cluster size.
struct Known {
    static constexpr int kDevices = 16;
    std::atomic<int> resident[kDevices][4] = {};
};
template <typename K>
cudaError_t resident_clusters(K kernel, Known &known, int device, const cudaLaunchConfig_t &cfg, int cluster, int &r) {
    int log = 0;
    while (1 << log < cluster) ++log;
    std::atomic<int> *place = device < Known::kDevices ? &known.resident[device][log] : nullptr;
    r = place ? place->load(std::memory_order_relaxed) : 0;
    if (r) return cudaSuccess;
    // the largest shared memory a block may have, so that the attribute need not follow the call's sizes
    int most = 0;
    cudaError_t e = cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, device);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e == cudaSuccess && cluster > 1) {
        e = cudaOccupancyMaxActiveClusters(&r, kernel, &cfg);
    } else if (e == cudaSuccess) {
        int sms = 0;
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&r, kernel, (int)cfg.blockDim.x, cfg.dynamicSmemBytes);
        r *= sms;
    }
    if (e != cudaSuccess) return e;
    r = std::max(r, 1);
    if (place) place->store(r, std::memory_order_relaxed);
    return cudaSuccess;
}

template <typename K, typename... More>
cudaError_t launch(K kernel, Known &known, Slab s, size_t smem, cudaStream_t stream, int64_t *launches, const GroupNormArgs &a, More... more) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)s.cluster);
    cfg.blockDim = dim3(kTH);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = s.cluster > 1 ? 1 : 0;
    int resident = 0;
    cudaError_t e = resident_clusters(kernel, known, a.device, cfg, s.cluster, resident);
    if (e != cudaSuccess) return e;
    // as many clusters as fit, in equal numbers per slab; each walks over every walkers-th sample
    s.walkers = (int)std::min<int64_t>(s.samples, std::max(1, resident / s.slabs));
    cfg.gridDim = dim3((unsigned)s.walkers * (unsigned)s.slabs * (unsigned)s.cluster);
    e = cudaLaunchKernelEx(&cfg, kernel, a, s, more...);
    if (e == cudaSuccess) ++*launches;
    return e;
}

template <int Low, int High, typename F>
cudaError_t by_nv(int nv, F &&f) {
    if (nv <= Low) return f(Int<Low>{});
    if constexpr (Low < High) return by_nv<Low * 2, High>(nv, f);
    return cudaErrorInvalidValue;
}

template <typename F>
cudaError_t by_type_act(int elem, int act, F &&f) {
    auto with = [&](auto t) {
        switch (act) {
            case kActNone: return f(t, Int<kActNone>{});
            case kActRelu: return f(t, Int<kActRelu>{});
            default: return f(t, Int<kActSilu>{});
        }
    };
    switch (elem) {
        case kElemF32: return with(float{});
        case kElemBF16: return with(__nv_bfloat16{});
        default: return with(__half{});
    }
}

}  // namespace

bool group_norm_on_chip(int64_t samples, int64_t positions, int channels, int groups, int elem) {
    Slab s;
    int nv;
    return choose(elem, channels, groups, samples, positions, kForwardBytes, kForwardNV, s, nv);
}
int group_norm_backward_on_chip(int64_t samples, int64_t positions, int channels, int groups, int elem) {
    Slab s;
    int nv;
    return choose(elem, channels, groups, samples, positions, backward_bytes(elem_bytes(elem)), backward_nv(elem_bytes(elem)), s, nv) ? s.cluster * kShares : 0;
}

cudaError_t launch_group_norm_on_chip(const GroupNormArgs &a, cudaStream_t stream, int64_t *launches) {
    Slab s;
    int nv;
    if (!choose(a.elem, a.channels, a.groups, a.samples, a.positions, kForwardBytes, kForwardNV, s, nv)) return cudaErrorInvalidValue;
    return by_type_act(a.elem, a.act, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T), ACT = decltype(act)::value;
        return by_nv<2, kForwardNV>(nv, [&](auto n) {
            constexpr int NV = decltype(n)::value;
            auto go = [&](auto uni) {
                constexpr bool UNI = decltype(uni)::value != 0;
                static Known known;
                constexpr size_t smem = (size_t)2 * NV * kTH * 16 + sizeof(ForwardMemory<VEC, UNI>);
                return launch(cr_group_norm_kernel<T, NV, UNI, ACT>, known, s, smem, stream, launches, a);
            };
            return s.cg % VEC == 0 ? go(Int<1>{}) : go(Int<0>{});
        });
    });
}

cudaError_t launch_group_norm_grad_on_chip(const GroupNormArgs &a, float *sum1, float *sum2, int64_t ld_sum, bool whole, cudaStream_t stream,
                                           int64_t *launches) {
    Slab s;
    int nv;
    if (!choose(a.elem, a.channels, a.groups, a.samples, a.positions, backward_bytes(elem_bytes(a.elem)), backward_nv(elem_bytes(a.elem)), s, nv)) return cudaErrorInvalidValue;
    return by_type_act(a.elem, a.act, [&](auto t, auto act) {
        using T = decltype(t);
        constexpr int VEC = 16 / (int)sizeof(T), ACT = decltype(act)::value;
        return by_nv<2, backward_nv(sizeof(T))>(nv, [&](auto n) {
            constexpr int NV = decltype(n)::value;
            auto go = [&](auto uni) {
                constexpr bool UNI = decltype(uni)::value != 0;
                static Known known;
                constexpr size_t smem = (size_t)4 * NV * kTH * 16 + sizeof(BackwardMemory<VEC, UNI>);
                return launch(cr_group_norm_grad_kernel<T, NV, UNI, ACT>, known, s, smem, stream, launches, a, sum1, sum2, ld_sum, whole ? 1 : 0);
            };
            return s.cg % VEC == 0 ? go(Int<1>{}) : go(Int<0>{});
        });
    });
}

}  // namespace cr
