// The choice of a token from its logits: temperature, top-k, top-p, min-p and one given number per row (include/dip.h has the definition).
//
// A row is shared out over a cluster of up to eight blocks.  Where the blocks' parts fit in shared memory beside what else a block has there (parts of up to
// 67 KB with two blocks on an SM, 175 KB with one), the row is read from global memory once and stays there.  Longer parts, as in large batches of long
// rows, are not copied: the maximum, the histogram, the list and the draw each walk through global memory, all but the first of them mostly out of L2.  Weights are
// exp((z - max) / temperature) as whole multiples of 2^-45 of the largest one, computed in binary64: sums of them are exact whatever their order,
// so results depend neither on how a row is shared out nor on the order of atomics, and a row's 2^18 weights fit 64 bits.
//
// Top-k and top-p both keep the front of the row's order (logit descending, index ascending), which ends at some element: its key and
// its index.  A histogram of counts says in which bin that is (bins of bfloat16 are its values, so their weights are known exactly; bins of
// binary32 are of equal width, with the sum of what is left in each, and their weights are known to some 10^-5, which is checked).
//   few   what is left up to that bin is at most SP_LIST elements: they go to the row's first block, which does the rest by itself
//   many  the elements of the bin (binary32: of the bins where the border can be) go there, which finds the border; or, ties of one
//         bfloat16 value, they are counted in order of index; then all blocks draw
//   else  (a crowd in one bin, borders that the check refuses, a long top-k with a top-p behind it) histograms of weights over ever fewer keys
// Several thousand elements in shared memory are searched by histograms of their own (`reach`).
// The draw adds up the kept weights per warp (whose elements are consecutive), then looks closer where the sum crosses the number.
// Bound, for few rows, by a chain of some dozen steps of 0.3 to 2 us (block scans, barriers of a cluster, reads between SMs, which take tens of cycles per
// 128 bytes): 12 to 27 us whatever the size.  For many rows by the work on each logit.  512 rows of 151001 bfloat16 logits by top-p take 280 us (155 MB are 24 us);
// two blocks' rows on each of 148 SMs are 296 at a time, and a block needs, in us, 15 for the maximum, 34 for the histogram (an atomic each), 7 for the cuts, 24 for the list or
// the ties, 35 for the draw (106 at most) or 5 for a list's end.  256 rows of 50257 binary32 logits without a filter 40 us (8): 12 until the maximum is known,
// 26 for the draw, a weight each.  64 rows of 102400 with mixed settings 61 us: 9, 6 for the histogram, 5, 9, and 13 for the draw or 16 for a long list's end.
// (The kernels have 64 registers a thread, for two blocks on an SM, and spill 8 bytes; bfloat16's 52.)
#include <initializer_list>

#include <cuda_bf16.h>

#include "common.cuh"
#include "gemv_common.cuh"

namespace {

constexpr int SP_THREADS = 512, SP_WARPS = SP_THREADS / 32;
constexpr int SP_CLUSTER = 8;                   // most blocks per row
constexpr int SP_BINS = 2048;                   // of a histogram of weights
constexpr int SP_PAIRS = 512;                   // elements that are compared pair by pair
constexpr int SP_LIST = 2048;                   // elements that one block looks after
constexpr int SP_FEW = SP_THREADS / 4;          // of them, that are compared with one another
constexpr int SP_REACH = SP_THREADS;            // bins by which it does
constexpr int SP_TABLE = 512;                   // 2^(j / 512)
constexpr int SP_ONE_BITS = 45;                 // the largest weight is 2^45
constexpr float SP_SPREAD = 64.f;               // logits further below the largest one share the last bin of the first histogram

typedef unsigned long long u64;

struct SampleParams {
    const void *logits;
    size_t pitch;
    int vocab, slice, resident;                 // whether a block's part of the row is copied to shared memory
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
    u64 *tr;
};

struct SampleBorder {
    float z;
    int index;
};

struct SampleList {
    u64 mass[SP_LIST];
    unsigned key[SP_LIST];
    int index[SP_LIST];
};
struct SampleWeights {                          // the last resort's
    u64 mass[SP_BINS];
    unsigned count[SP_BINS];
    u64 list_mass[SP_PAIRS];
    unsigned list_key[SP_PAIRS];
    int list_index[SP_PAIRS];
};

struct __align__(16) SampleSmem {
    double table[SP_TABLE];
    union {
        unsigned bins[8192];                    // counts; binary32: 4096 of them and what is left in each (1/1024 of a bin's width)
        u64 bin_mass[4096];                     // bfloat16, for the draw: of the bins from the largest logit's on
        SampleList list;
        SampleWeights weights;
    };
    u64 reach[SP_REACH];
    unsigned reach_count[SP_REACH];
    int final_slot[32];
    int finals, reached, listed;
    u64 reach_before;
    u64 tiny[2];
    u64 scan[SP_WARPS + 1];
    // what the blocks of a cluster tell one another
    u64 total[SP_CLUSTER], sums[3], part[3][SP_WARPS], of_all;
    float top, low;
    int first[SP_CLUSTER];
    unsigned key_lo[SP_CLUSTER], key_hi[SP_CLUSTER];
    struct {
        int bin;
        unsigned count;
        u64 before;
    } found;
    struct {
        int bin;
        unsigned count;                         // of its elements, and of those in front of it
        unsigned in_front;
        u64 before, want;                       // and the weight of those; what is reached in it
    } cut[2];
    struct {
        int coarse;
        u64 before_c, before_w, want;
    } near[2];                                  // the neighbouring bins among which a cut is
    unsigned coarse_count[128];
    u64 coarse_weight[128];
    u64 all_count, all_weight;                  // (bfloat16: exact)
    SampleBorder border;
    float block_top[SP_WARPS], block_low[SP_WARPS];
    int block_first[SP_WARPS];
};

__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned cluster_size()
{
    unsigned n;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}
__device__ __forceinline__ void cluster_sync(unsigned blocks)
{
    if (blocks == 1) __syncthreads();
    else asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Where block `rank` has what is at p here.
__device__ __forceinline__ uint32_t at_rank(const void *p, unsigned rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void put32(uint32_t a, unsigned v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void put64(uint32_t a, u64 v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }
// The same as an ordinary address (reads through it may go out together).
template <typename V>
__device__ __forceinline__ const V *of_rank(const V *p, unsigned rank)
{
    const V *q;
    asm("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(rank));
    return q;
}

__device__ __forceinline__ unsigned key_of(float z)
{
    const unsigned u = __float_as_uint(z);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float value_of_key(unsigned key) { return __uint_as_float(key ^ (~(unsigned)((int)key >> 31) | 0x80000000u)); }

// The larger ones of two pairs of bfloat16 (a number beside what is none).
__device__ __forceinline__ unsigned max2(unsigned a, unsigned b)
{
    unsigned m;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
}
__device__ __forceinline__ float larger(unsigned pair) { return fmaxf(__uint_as_float(pair << 16), __uint_as_float(pair & 0xffff0000u)); }

__device__ __forceinline__ float item_value(const float *p, int i) { return p[i] + 0.f; }          // (-0 is 0)
__device__ __forceinline__ float item_value(const uint16_t *p, int i) { return __uint_as_float((unsigned)p[i] << 16) + 0.f; }

// To a sum in shared memory, by its halves (the lower one says whether it ran over).
__device__ __forceinline__ void add64(u64 *sum, u64 q)
{
    unsigned *w = reinterpret_cast<unsigned *>(sum);
    const unsigned lo = (unsigned)q, was = atomicAdd(w, lo), hi = (unsigned)(q >> 32) + (was + lo < lo);
    if (hi) atomicAdd(w + 1, hi);
}

template <typename T>
struct Row {
    SampleSmem &s;
    const T *items;                             // this block's, in shared memory or where they came from
    int n, begin;                               // how many; the first one's index
    unsigned rank, blocks;
    float top;                                  // the largest logit
    double steps;                               // 512 log2(e) / temperature; below a logit of +infinity, so many that nothing else weighs
    double top_wide;
    float steps_f;
    float scale;                                // bins per unit
    int head, vectors;                          // items in front of the first boundary of 16 bytes; whole pieces of 16 bytes from there on

    __device__ __forceinline__ float value(int i) const { return item_value(items, i); }

    // Pieces of 16 bytes (-infinity for what is not there).
    static constexpr int PER = 16 / sizeof(T);
    __device__ __forceinline__ void decode(const uint4 &a, float (&z)[PER]) const
    {
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (sizeof(T) == 2) {
                z[2 * j] = __uint_as_float(w[j] << 16) + 0.f;
                z[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u) + 0.f;
            } else {
                z[j] = __uint_as_float(w[j]) + 0.f;
            }
        }
    }
    // f(piece, place of its first logit) for the pieces first, first + step, ..., below last (all: of the block's threads), with the next one under
    // way.  (HALF: pieces without a logit from `least` up are passed over.)
    template <class F>
    __device__ __forceinline__ void walk(int first, int last, int step, const F &f, float least = -INFINITY) const
    {
        const uint4 *from = reinterpret_cast<const uint4 *>(items + head);
        uint4 a = first < last ? from[first] : make_uint4(0u, 0u, 0u, 0u);
        for (int v = first; v < last; v += step) {
            const uint4 next = v + step < last ? from[v + step] : a;
            if (sizeof(T) == 4 || larger(max2(max2(a.x, a.y), max2(a.z, a.w))) >= least) f(a, head + v * PER);
            a = next;
        }
    }
    // (what is in front of the first whole piece and behind the last one comes as a piece filled up with -infinity)
    template <class F>
    __device__ __forceinline__ void walk_all(const F &f) const
    {
        walk(threadIdx.x, vectors, SP_THREADS, f);
        if (threadIdx.x < 2) {
            const int first = threadIdx.x ? head + vectors * PER : 0, last = threadIdx.x ? n : head;
            unsigned w[4] = {};
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const unsigned bits = __float_as_uint(first + j < last ? value(first + j) : -INFINITY);
                if (sizeof(T) == 2) w[j >> 1] |= j & 1 ? bits & 0xffff0000u : bits >> 16;
                else w[j] = bits;
            }
            f(make_uint4(w[0], w[1], w[2], w[3]), first);
        }
    }

    // A number's bits in a binary64 number's places: 2^-896 times it (infinity comes as 2^128; what is no number as one, too).  A conversion takes four times as
    // long as other instructions.
    static __device__ __forceinline__ double wide(float z)
    {
        return __hiloint2double((__float_as_int(z) >> 3) & 0x8fffffff, __float_as_int(z) << 29);
    }
    // exp((z - top) / temperature) times 2^45, of an open logit: 2^(k / 512) from the table times the third-order sum for what is left (within 10^-14).
    // Ten binary64 operations, at half of binary32's rate.
    __device__ __forceinline__ double weight(float z) const
    {
        constexpr double STEP = 0.69314718055994530942 / SP_TABLE, magic = 6755399441055744.0;
        const double d = fma(wide(z), 0x1p896, -top_wide), k = fma(d, steps, magic), f = fma(d, steps, magic - k);
        const int i = __double2loint(k);
        const double t = s.table[i & (SP_TABLE - 1)];
        const double e = fma(t, f * fma(f, fma(f, STEP * STEP * STEP / 6, STEP * STEP / 2), STEP), t);
        const double w = __hiloint2double(__double2hiint(e) + ((i >> 9) << 20), __double2loint(e));
        // (asked in binary64, where neither the difference nor the steps leave the range)
        return k > magic - 60.0 * SP_TABLE ? w : 0.0;
    }
    // Whether min_p (above 0) keeps a logit.  From 1 on it keeps the largest alone; that is not asked of weights, since a weight that
    // is smaller by less than 2^-53 is rounded to the largest one's.
    __device__ __forceinline__ bool likely(float z, float min_p) const
    {
        return min_p < 1.f ? !(weight(z) < (double)min_p * (double)(1ull << SP_ONE_BITS)) : z == top;
    }
    __device__ __forceinline__ u64 mass(float z) const
    {
        return (u64)__double_as_longlong(weight(z) + 4503599627370496.0) & 0xfffffffffffffull;
    }
    // whether the element is open and in front of the border (or it; the border of all is (-infinity, -1))
    __device__ __forceinline__ bool kept(float z, int i, const SampleBorder &b) const { return z > b.z || (z == b.z && begin + i <= b.index); }

    // Bins in order of falling logits.  bfloat16: one per value from 2^-12 to 2^20 either way, the first, the last and the two in the middle
    // for all beyond.  (Places are such that a thread's consecutive bins and its neighbours' fall on different banks.)
    static constexpr bool HALF = sizeof(T) == 2;
    static constexpr int BINS = HALF ? 8192 : 4096, HALF_FIRST = 115 << 7;
    static constexpr float REST = 1024.f;
    __device__ __forceinline__ int place(int bin) const { return bin ^ (bin >> 4 & 15); }
    __device__ __forceinline__ int bin_of(float z) const
    {
        if (HALF) {
            const int m = min(max((int)(__float_as_uint(z) >> 16 & 0x7fffu) - HALF_FIRST, 0), 4095);
            return __float_as_int(z) < 0 ? 4096 + m : 4095 - m;
        }
        return min(BINS - 1, (int)((top - z) * scale * 2.f));
    }
    __device__ __forceinline__ bool middle(int bin) const { return bin == 4095 || bin == 4096; }           // (HALF)
    __device__ __forceinline__ bool mixed(int bin) const { return HALF ? middle(bin) || bin == 0 || bin == 8191 : true; }
    __device__ __forceinline__ float value_of(int bin) const
    {
        return __uint_as_float(bin < 4096 ? (unsigned)(HALF_FIRST + 4095 - bin) << 16 : ((unsigned)(HALF_FIRST + bin - 4096) << 16) | 0x80000000u);
    }
    // The weight of a bin's elements.  HALF: exact (the last bin's are 0: see `plain` below); else as if each had the middle one's.
    __device__ __forceinline__ u64 bin_mass(int bin, unsigned count, unsigned rest, const u64 *tiny) const
    {
        if (HALF) return middle(bin) ? tiny[bin - 4095] : bin == 8191 ? 0 : count * mass(value_of(bin));
        const float below = ((float)bin + ((float)rest + 0.5f * count) / (REST * count)) / (2.f * scale);
        return __float2ull_rn(exp2f(below * steps_f * (-1.f / SP_TABLE)) * (float)count * 1099511627776.f);       // (times 2^40)
    }
    __device__ __forceinline__ void histogram(bool weights) const
    {
        for (int i = threadIdx.x; i < 8192 / 4; i += SP_THREADS) reinterpret_cast<uint4 *>(s.bins)[i] = make_uint4(0u, 0u, 0u, 0u);
        if (threadIdx.x < 2) s.tiny[threadIdx.x] = 0;
        __syncthreads();
        walk_all([&](const uint4 &a, int) {
            if (HALF) {
                const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const unsigned raw = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu, size = raw & 0x7fffu;
                    if (size - (HALF_FIRST + 1) < 0x7f80u - (HALF_FIRST + 1)) {
                        const int m = min((int)size - HALF_FIRST, 4095), bin = 4096 + (m ^ ((int)(raw >> 15) - 1));
                        atomicAdd(&s.bins[place(bin)], 1u);
                    } else {
                        // next to zero, infinite, or none
                        const float z = __uint_as_float(raw << 16) + 0.f;
                        if (z > -INFINITY) {
                            const int bin = bin_of(z);
                            atomicAdd(&s.bins[place(bin)], 1u);
                            if (middle(bin)) add64(&s.tiny[bin - 4095], mass(z));
                        }
                    }
                }
            } else {
                float z[PER];
                decode(a, z);
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if (!(z[j] > -INFINITY)) continue;
                    const int bin = bin_of(z[j]);
                    atomicAdd(&s.bins[place(bin)], 1u);
                    if (weights) {
                        const float at = (top - z[j]) * scale * 2.f;
                        atomicAdd(&s.bins[BINS + place(bin)], (unsigned)(fminf(at - (float)bin, 1.f) * REST));
                    }
                }
            }
        });
        __syncthreads();
    }
    // The bins where a count (top_k > 0), or a weight, is reached: the latter (HALF) exactly, or between cut[0] and cut[1] if all is well.
    // Every block finds them for itself, from the others' sums of 64 (32) neighbouring bins and then from their bins: between SMs 128 bytes take
    // tens of cycles, so not all bins are read.  Ends with a cluster barrier (the bins have been read).
    static constexpr int COARSE = 128, FINE = BINS / COARSE;
    __device__ __forceinline__ void cuts(int top_k, float top_p) const
    {
        constexpr int EACH = BINS / SP_THREADS, SHARE = SP_THREADS / COARSE;
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        u64 weight = 0, count = 0;
#pragma unroll 4
        for (int j = 0; j < EACH; ++j) {
            const int bin = tid * EACH + j;
            const unsigned c = s.bins[place(bin)];
            count += c;
            if (top_k == 0 && c) weight += bin_mass(bin, c, HALF ? 0 : s.bins[BINS + place(bin)], s.tiny);
        }
#pragma unroll
        for (int o = 1; o < SHARE; o <<= 1) {
            count += __shfl_xor_sync(0xffffffffu, count, o);
            weight += __shfl_xor_sync(0xffffffffu, weight, o);
        }
        if (tid % SHARE == 0) {
            s.coarse_count[tid / SHARE] = (unsigned)count;
            s.coarse_weight[tid / SHARE] = weight;
        }
        cluster_sync(blocks);
        count = weight = 0;
        if (tid < COARSE) {
            unsigned c[SP_CLUSTER];
            u64 w[SP_CLUSTER];
#pragma unroll
            for (unsigned r = 0; r < SP_CLUSTER; ++r) {
                c[r] = r < blocks ? *of_rank(&s.coarse_count[tid], r) : 0;
                w[r] = r < blocks && top_k == 0 ? *of_rank(&s.coarse_weight[tid], r) : 0;
            }
#pragma unroll
            for (unsigned r = 0; r < SP_CLUSTER; ++r) {
                count += c[r];
                weight += w[r];
            }
        }
        u64 all_c, all_w = 0;
        const u64 before_c = scan(count, all_c), before_w = top_k == 0 ? scan(weight, all_w) : 0;
        const double goal = fmax((double)top_p, 0.0) * (double)all_w;
#pragma unroll
        for (int c = 0; c < (HALF ? 1 : 2); ++c) {
            const u64 want = top_k ? min((u64)top_k, all_c)
                             : HALF ? max(1ull, (u64)ceil(goal)) : min(all_w, max(1ull, (u64)(c ? goal * (1 + 1.0 / 2048) + 2 : goal * (1 - 1.0 / 2048))));
            const u64 before = top_k ? before_c : before_w, here = top_k ? count : weight;
            if (before < want && want <= before + here) s.near[c] = {tid, before_c, before_w, want};
        }
        if (tid == 0) {
            s.all_count = all_c;
            s.all_weight = all_w;
        }
        __syncthreads();
        if (warp < (HALF ? 1 : 2) && s.near[warp].coarse >= 0) {
            const auto near = s.near[warp];
            constexpr int PER = FINE / 32;
            unsigned c[PER];
            u64 w[PER], bc = 0, bw = 0;
            unsigned k[PER][SP_CLUSTER], rest[PER][SP_CLUSTER];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int at = place(near.coarse * FINE + lane * PER + j);
#pragma unroll
                for (unsigned r = 0; r < SP_CLUSTER; ++r) {
                    k[j][r] = r < blocks ? *of_rank(&s.bins[at], r) : 0;
                    rest[j][r] = !HALF && top_k == 0 && r < blocks ? *of_rank(&s.bins[BINS + at], r) : 0;
                }
            }
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int bin = near.coarse * FINE + lane * PER + j;
                c[j] = 0;
                w[j] = 0;
#pragma unroll
                for (unsigned r = 0; r < SP_CLUSTER; ++r) {
                    c[j] += k[j][r];
                    if (top_k == 0 && !HALF && k[j][r]) w[j] += bin_mass(bin, k[j][r], rest[j][r], nullptr);
                }
                if (top_k == 0 && HALF && c[j]) {
                    if (middle(bin))
                        for (unsigned r = 0; r < blocks; ++r) w[j] += *of_rank(&s.tiny[bin - 4095], r);
                    else w[j] = bin_mass(bin, c[j], 0, s.tiny);
                }
                bc += c[j];
                bw += w[j];
            }
            const u64 own_c = bc, own_w = bw;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 x = __shfl_up_sync(0xffffffffu, bc, o), y = __shfl_up_sync(0xffffffffu, bw, o);
                if (lane >= o) {
                    bc += x;
                    bw += y;
                }
            }
            bc += near.before_c - own_c;
            bw += near.before_w - own_w;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const u64 b = top_k ? bc : bw, u = top_k ? c[j] : w[j];
                if (b < near.want && near.want <= b + u) s.cut[warp] = {near.coarse * FINE + lane * PER + j, c[j], (unsigned)bc, bw, near.want};
                bc += c[j];
                bw += w[j];
            }
        }
        cluster_sync(blocks);
    }

    // Brings the elements of the bins first .. last into the first block's list, if there are at most SP_LIST: the number of them comes back
    // (each block lists its own, then the first one fetches them).  sums: [0] the weight of all elements in front of them, [1] their own, [2]
    // of all, if `weigh`.  Ends with a cluster barrier.
    __device__ __forceinline__ unsigned collect(int first, int last, bool weigh, u64 (&sums)[3]) const
    {
        u64 mine[3] = {0, 0, 0};
        walk_all([&](const uint4 &a, int i0) {
            float z[PER];
            decode(a, z);
            int bin[PER];
            bool any = weigh;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                bin[j] = z[j] > -INFINITY ? bin_of(z[j]) : BINS;
                any |= bin[j] >= first && bin[j] <= last;
            }
            if (!any) return;
            // (four weights side by side, for the latency of binary64)
#pragma unroll
            for (int j0 = 0; j0 < PER; j0 += 4) {
                u64 q[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) q[j] = mass(z[j0 + j]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = bin[j0 + j];
                    mine[2] += at < BINS ? q[j] : 0;
                    if (first > 0) mine[0] += at < first ? q[j] : 0;
                    if (at >= first && at <= last) {
                        mine[1] += q[j];
                        const int slot = atomicAdd(&s.listed, 1);
                        if (slot < SP_LIST) {
                            s.list.key[slot] = key_of(z[j0 + j]);
                            s.list.index[slot] = begin + i0 + j0 + j;
                            s.list.mass[slot] = q[j];
                        }
                    }
                }
            }
        });
        if (weigh) {
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
            for (int j = 0; j < 3; ++j) {
#pragma unroll
                for (int o = 16; o; o >>= 1) mine[j] += __shfl_xor_sync(0xffffffffu, mine[j], o);
                if (lane == 0) s.part[j][warp] = mine[j];
            }
            __syncthreads();
            if (threadIdx.x < 3) {
                u64 sum = 0;
                for (int w = 0; w < SP_WARPS; ++w) sum += s.part[threadIdx.x][w];
                s.sums[threadIdx.x] = sum;
            }
        }
        cluster_sync(blocks);
        unsigned counts[SP_CLUSTER], all = 0;
#pragma unroll
        for (unsigned r = 0; r < SP_CLUSTER; ++r) counts[r] = r < blocks ? *of_rank(&s.listed, r) : 0;
#pragma unroll
        for (unsigned r = 0; r < SP_CLUSTER; ++r) all += counts[r];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            sums[j] = 0;
            if (weigh) {
                u64 a[SP_CLUSTER];
#pragma unroll
                for (unsigned r = 0; r < SP_CLUSTER; ++r) a[r] = r < blocks ? *of_rank(&s.sums[j], r) : 0;
#pragma unroll
                for (unsigned r = 0; r < SP_CLUSTER; ++r) sums[j] += a[r];
            }
        }
        if (rank == 0 && all <= SP_LIST) {
            for (unsigned i = counts[0] + threadIdx.x; i < all; i += SP_THREADS) {
                unsigned r = 0, j = i;
#pragma unroll
                for (unsigned k = 0; k < SP_CLUSTER - 1; ++k)
                    if (r == k && j >= counts[k]) {
                        j -= counts[k];
                        ++r;
                    }
                const unsigned key = *of_rank(&s.list.key[j], r);
                const int index = *of_rank(&s.list.index[j], r);
                const u64 q = *of_rank(&s.list.mass[j], r);
                s.list.key[i] = key;
                s.list.index[i] = index;
                s.list.mass[i] = q;
            }
        }
        cluster_sync(blocks);
        return all;
    }

    // Of m elements, each with a number of its own (lo to hi) and a share (0: none), the one at which the sum of shares in order of the
    // numbers reaches `want` (1 up to the sum of all).  By one block.
    template <class Number, class Share>
    __device__ int reach(int m, const Number &number, const Share &share, u64 want, u64 lo, u64 hi) const
    {
        const int tid = threadIdx.x;
        u64 before = 0;
        for (;;) {
            const int bits = lo == hi ? 0 : 64 - __clzll(hi - lo), shift = max(0, bits - 9);
            s.reach[tid] = 0;
            s.reach_count[tid] = 0;
            if (tid == 0) s.finals = s.reached = 0;
            __syncthreads();
            for (int i = tid; i < m; i += SP_THREADS) {
                const u64 q = share(i), a = number(i);
                if (!q || a < lo || a > hi) continue;
                const int bin = (int)((a - lo) >> shift);
                atomicAdd(&s.reach_count[bin], 1u);
                add64(&s.reach[bin], q);
            }
            __syncthreads();
            u64 ignored;
            const u64 here = s.reach[tid], b = before + scan(here, ignored);
            if (b < want && want <= b + here) {
                s.reached = tid;
                s.reach_before = b;
            }
            __syncthreads();
            before = s.reach_before;            // (there is one: 1 <= want <= the sum)
            const int few = s.reach_count[s.reached];
            lo += (u64)s.reached << shift;
            hi = min(hi, lo + ((1ull << shift) - 1));
            if (few <= 32) break;
            __syncthreads();
        }
        for (int i = tid; i < m; i += SP_THREADS)
            if (share(i) && number(i) >= lo && number(i) <= hi) s.final_slot[atomicAdd(&s.finals, 1)] = i;
        __syncthreads();
        if (tid < s.finals) {
            const int i = s.final_slot[tid];
            const u64 a = number(i);
            u64 b = before;
            for (int j = 0; j < s.finals; ++j)
                if (number(s.final_slot[j]) < a) b += share(s.final_slot[j]);
            if (b < want && want <= b + share(i)) s.reached = i;
        }
        __syncthreads();
        return s.reached;
    }
    __device__ __forceinline__ u64 number_in_order(int i) const { return ((u64)(key_of(top) - s.list.key[i]) << 18) | (unsigned)s.list.index[i]; }
    // (no number of an element down to logit z is above)
    __device__ __forceinline__ u64 last_number(float z) const { return ((u64)(key_of(top) - key_of(z)) << 18) | 0x3ffffu; }

    // The sum over the block's threads.
    __device__ __forceinline__ u64 block_sum(u64 v) const
    {
#pragma unroll
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s.scan[threadIdx.x >> 5] = v;
        __syncthreads();
        v = s.scan[threadIdx.x & (SP_WARPS - 1)];
#pragma unroll
        for (int o = SP_WARPS / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    // finish() for at most SP_FEW elements: everyone compared with everyone, by several threads each.  (One row of 1000 by top-p 12.4 us, by three searches
    // with histograms 15.0; with two threads each for up to 256 elements, a row of 102400 by top-k 26 us, by searches 22.)
    __device__ __forceinline__ void finish_few(int m, int top_k, float top_p, float min_p, float u, u64 all, int32_t *token, float *prob) const
    {
        const int each = m <= SP_THREADS / 32 ? 32 : m <= SP_THREADS / 8 ? 8 : 4, e = threadIdx.x / each, part = threadIdx.x % each;
        const bool there = e < m;
        const unsigned key = there ? s.list.key[e] : 0u;
        const int index = there ? s.list.index[e] : 0;
        const u64 mass = there ? s.list.mass[e] : 0;
        const auto together = [&](u64 v) {
            for (int o = each / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            return v;
        };
        // what is in front in the row's order: how many, what weight
        unsigned rank_of = 0;
        u64 before = 0;
#pragma unroll 8
        for (int j = part; j < m; j += each) {
            const unsigned k = s.list.key[j];
            const bool first = k > key || (k == key & s.list.index[j] < index);
            rank_of += first;
            before += first ? s.list.mass[j] : 0;
        }
        rank_of = (unsigned)together(rank_of);
        before = together(before);
        bool left = there && (top_k == 0 || rank_of < (unsigned)top_k);
        if (top_p < 1.f) {
            if (top_k) all = block_sum(left && part == 0 ? mass : 0);
            left &= before < max(1ull, (u64)ceil(fmax((double)top_p, 0.0) * (double)all));
        }
        const double weight_of = weight(value_of_key(key));
        if (min_p > 0.f) left &= likely(value_of_key(key), min_p);
        const u64 sum = block_sum(left && part == 0 ? mass : 0), mark = min(sum - 1, (u64)(fmax((double)u, 0.0) * (double)sum));
        // in order of index, of those that are left
        if (there && part == 0 && !left) s.list.mass[e] = 0;
        __syncthreads();
        before = 0;
#pragma unroll 8
        for (int j = part; j < m; j += each) before += s.list.index[j] < index ? s.list.mass[j] : 0;
        before = together(before);
        if (left && part == 0 && before <= mark && mark < before + mass) {
            *token = index;
            if (prob) *prob = (float)(weight_of / (double)sum);
        }
    }

    // The first block has all that can be left in its list: everything else.  all: the weight that top_p is a share of (top_k > 0: of what
    // that leaves).
    __device__ __forceinline__ void finish(int m, int top_k, float top_p, float min_p, float u, u64 all, float lowest, int vocab, int32_t *token,
                                           float *prob) const
    {
        u64 last = last_number(lowest);         // the border's number
        const auto number = [&](int i) { return number_in_order(i); };
        const auto weight_in = [&](int i) -> u64 { return number_in_order(i) <= last ? s.list.mass[i] : 0; };
        const auto sum_of = [&](const auto &share) {
            u64 mine = 0, sum;
            for (int i = threadIdx.x; i < m; i += SP_THREADS) mine += share(i);
            scan(mine, sum);
            return sum;
        };
        if (top_k) {
            last = number(reach(m, number, [](int) { return 1ull; }, min(top_k, m), 0, last));
            if (top_p < 1.f) all = sum_of(weight_in);
        }
        if (top_p < 1.f) last = number(reach(m, number, weight_in, max(1ull, (u64)ceil(fmax((double)top_p, 0.0) * (double)all)), 0, last));
        const auto drawn = [&](int i) -> u64 {
            if (min_p > 0.f) {
                const unsigned k = s.list.key[i];
                if (!likely(value_of_key(k), min_p)) return 0;
            }
            return weight_in(i);
        };
        const u64 sum = sum_of(drawn), mark = min(sum - 1, (u64)(fmax((double)u, 0.0) * (double)sum));
        const int i = reach(m, [&](int j) { return (u64)s.list.index[j]; }, drawn, mark + 1, 0, vocab - 1);
        if (threadIdx.x == 0) {
            const unsigned k = s.list.key[i];
            *token = s.list.index[i];
            if (prob) *prob = (float)(weight(value_of_key(k)) / (double)sum);
        }
    }

    // Of all elements in order of index, each with a share, the one at which the sum of shares exceeds mark(sum of all): found(its place in
    // this block, its logit, the sum of all), by one thread of one block.  shares(piece, place): those of a piece's elements together;
    // none below `least` has any.
    // A warp's elements are consecutive; those of the warp that has it are shared out among the warps in turn, until there are few for each thread.
    template <class Shares, class Share, class Mark, class Found>
    __device__ __forceinline__ void in_order(float least, const Shares &shares, const Share &share, const Mark &mark, const Found &found) const
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        int p0 = 0, p1 = vectors;               // pieces
        bool front = true, back = true;         // with what is in front of the first one, behind the last one
        u64 at = 0, want = 0;
        for (bool first = true;; first = false) {
            const int each = (p1 - p0 + SP_WARPS - 1) / SP_WARPS, v0 = min(p1, p0 + warp * each), v1 = min(p1, v0 + each);
            u64 sum = 0;
            walk(v0 + lane, v1, 32, [&](const uint4 &a, int i) { sum += shares(a, i); }, least);
            if (warp == 0 && front && lane < head) sum += share(value(lane), lane);
            const int behind = head + vectors * PER + lane;
            if (warp == SP_WARPS - 1 && back && behind < n) sum += share(value(behind), behind);
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            __syncthreads();
            if (lane == 0) s.part[0][warp] = sum;
            __syncthreads();
            if (first) {
                u64 block_sum = 0, all;
                for (int w = 0; w < SP_WARPS; ++w) block_sum += s.part[0][w];
                at = gather(block_sum, all);
                want = mark(all);
                if (!(at <= want && want < at + block_sum)) return;
                s.of_all = all;
            }
            int w = 0;
            for (; w < SP_WARPS - 1 && at + s.part[0][w] <= want; ++w) at += s.part[0][w];
            p0 = min(p1, p0 + w * each);
            p1 = min(p1, p0 + each);
            front &= w == 0;
            back &= w == SP_WARPS - 1;
            if ((p1 - p0 + 2) * PER <= 8 * SP_THREADS) break;
        }
        const int begin_at = front ? 0 : head + p0 * PER, end = back ? n : head + p1 * PER, each = (end - begin_at + SP_THREADS - 1) / SP_THREADS;
        const int i0 = min(end, begin_at + (int)threadIdx.x * each), i1 = min(end, i0 + each);
        u64 mine = 0, ignored;
        for (int i = i0; i < i1; ++i) mine += share(value(i), i);
        at += scan(mine, ignored);
        if (at <= want && want < at + mine) {
            int i = i0;
            for (u64 q; at + (q = share(value(i), i)) <= want; ++i) at += q;
            found(i, value(i), s.of_all);
        }
    }
    // The border is the nth (from 1) in order of index among the elements of that logit (HALF; not 0, which has two forms).
    __device__ __forceinline__ void among_ties(float tie, u64 nth) const
    {
        in_order(
            tie, [&](const uint4 &a, int) -> u64 {
                const unsigned w[4] = {a.x, a.y, a.z, a.w}, both = (__float_as_uint(tie) & 0xffff0000u) | __float_as_uint(tie) >> 16;
                unsigned here = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) here += (((w[j] ^ both) & 0xffffu) == 0) + (((w[j] ^ both) >> 16) == 0);
                return here;
            },
            [&](float z, int) -> u64 { return z == tie; }, [&](u64) { return nth - 1; }, [&](int i, float z, u64) { tell(z, begin + i); });
        cluster_sync(blocks);
    }
    __device__ __forceinline__ void tell(float z, int index) const
    {
        for (unsigned r = 0; r < blocks; ++r) {
            put32(at_rank(&s.border.z, r), __float_as_uint(z));
            put32(at_rank(&s.border.index, r), index);
        }
    }

    // Exclusive sums over the block's threads; `sum`: of all.
    __device__ __forceinline__ u64 scan(u64 v, u64 &sum) const
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        u64 incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 a = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += a;
        }
        __syncthreads();                        // (the sums in front have been read)
        if (lane == 31) s.scan[warp] = incl;
        __syncthreads();
        u64 sums = s.scan[lane & (SP_WARPS - 1)];
        const u64 own = sums;
#pragma unroll
        for (int o = 1; o < SP_WARPS; o <<= 1) {
            const u64 a = __shfl_up_sync(0xffffffffu, sums, o, SP_WARPS);
            if ((lane & (SP_WARPS - 1)) >= o) sums += a;
        }
        sum = __shfl_sync(0xffffffffu, sums, SP_WARPS - 1);
        const u64 before = __shfl_sync(0xffffffffu, sums - own, warp);
        return before + incl - v;
    }
    // The same over the cluster, given this block's sum: what is in front of this block, and all.  Ends with a cluster barrier.
    __device__ __forceinline__ u64 gather(u64 mine, u64 &all) const
    {
        if (threadIdx.x < blocks) put64(at_rank(&s.total[rank], threadIdx.x), mine);
        cluster_sync(blocks);
        u64 before = 0;
        all = 0;
        for (unsigned r = 0; r < blocks; ++r) {
            before += r < rank ? s.total[r] : 0;
            all += s.total[r];
        }
        return before;
    }

    __device__ __forceinline__ void clear() const
    {
        for (int i = threadIdx.x; i < SP_BINS; i += SP_THREADS) {
            s.weights.mass[i] = 0;
            s.weights.count[i] = 0;
        }
        if (threadIdx.x == 0) s.listed = 0;
        __syncthreads();
    }
    template <bool MASS>
    __device__ __forceinline__ void add(int bin, float z) const
    {
        atomicAdd(&s.weights.count[bin], 1u);
        if (MASS) {
            add64(&s.weights.mass[bin], mass(z));
        }
    }

    // The bins' sums over the cluster are in order: the bin in which `want` (counted from 1) is reached, with what is in front of it and how
    // many elements it has, in s.found of every block.  want == 0: goal(sum of all bins) says.
    template <bool MASS, class Goal>
    __device__ __forceinline__ u64 locate(u64 want, const Goal &goal) const
    {
        cluster_sync(blocks);                         // (all blocks have counted)
        const int mine = SP_BINS / blocks, each = (mine + SP_THREADS - 1) / SP_THREADS, b0 = rank * mine + threadIdx.x * each;
        const int in = max(0, min(each, (int)((rank + 1) * mine) - b0));
        u64 unit[SP_BINS / SP_THREADS], sum = 0;
        unsigned count[SP_BINS / SP_THREADS];
#pragma unroll
        for (int j = 0; j < SP_BINS / SP_THREADS; ++j) {
            unit[j] = 0;
            count[j] = 0;
            if (j < in) {
                for (unsigned r = 0; r < blocks; ++r) {
                    count[j] += *of_rank(&s.weights.count[b0 + j], r);
                    if (MASS) unit[j] += *of_rank(&s.weights.mass[b0 + j], r);
                }
                if (!MASS) unit[j] = count[j];
                sum += unit[j];
            }
        }
        u64 block_sum, all;
        u64 before = scan(sum, block_sum);
        before += gather(block_sum, all);
        if (want == 0) want = goal(all);
        if (before < want && want <= before + sum) {
#pragma unroll
            for (int j = 0; j < SP_BINS / SP_THREADS; ++j) {
                if (before < want && want <= before + unit[j]) {
                    for (unsigned r = 0; r < blocks; ++r) {
                        put32(at_rank(&s.found.bin, r), b0 + j);
                        put32(at_rank(&s.found.count, r), count[j]);
                        put64(at_rank(&s.found.before, r), before);
                    }
                    want = 0;                   // (no other)
                }
                before += unit[j];
            }
            want = ~0ull;
        }
        cluster_sync(blocks);
        return want;
    }

    // Moves the border to the front's end: the element at which the count, or the weight, of the elements kept so far reaches goal(all of it).
    template <bool MASS, class Goal>
    __device__ void shorten(SampleBorder &border, const Goal &goal) const
    {
        clear();
        const auto first_bin = [&](float z) { return min(SP_BINS - 1, (int)((top - z) * scale)); };
        for (int i = threadIdx.x; i < n; i += SP_THREADS) {
            const float z = value(i);
            if (kept(z, i, border)) add<MASS>(first_bin(z), z);
        }
        u64 want = 0;
        const auto remember = [&](u64 all) { return want = goal(all); };
        locate<MASS>(0, remember);
        int bin = s.found.bin;
        u64 before = s.found.before;
        unsigned lo = 0, hi = 0xffffffffu;      // keys among which the border's is
        bool by_bin = true;
        while (s.found.count > SP_PAIRS) {
            if (by_bin) {
                // the keys of that bin
                unsigned a = 0xffffffffu, z = 0u;
                for (int i = threadIdx.x; i < n; i += SP_THREADS) {
                    const float v = value(i);
                    if (kept(v, i, border) && first_bin(v) == bin) {
                        a = min(a, key_of(v));
                        z = max(z, key_of(v));
                    }
                }
                a = __reduce_min_sync(0xffffffffu, a);
                z = __reduce_max_sync(0xffffffffu, z);
                if (threadIdx.x == 0) {
                    s.key_lo[0] = 0xffffffffu;
                    s.key_hi[0] = 0u;
                }
                __syncthreads();
                if ((threadIdx.x & 31) == 0) {
                    atomicMin(&s.key_lo[0], a);
                    atomicMax(&s.key_hi[0], z);
                }
                cluster_sync(blocks);
                lo = 0xffffffffu;
                hi = 0u;
                for (unsigned r = 0; r < blocks; ++r) {
                    lo = min(lo, *of_rank(&s.key_lo[0], r));
                    hi = max(hi, *of_rank(&s.key_hi[0], r));
                }
                cluster_sync(blocks);
                by_bin = false;
            }
            if (lo == hi) break;
            const int shift = max(0, 32 - __clz(hi - lo) - 11);
            clear();
            for (int i = threadIdx.x; i < n; i += SP_THREADS) {
                const float z = value(i);
                const unsigned k = key_of(z);
                if (k >= lo && k <= hi && kept(z, i, border)) add<MASS>((hi - k) >> shift, z);
            }
            locate<MASS>(want - before, goal);
            before += s.found.before;
            hi -= (unsigned)s.found.bin << shift;
            lo = max(lo, hi - ((1u << shift) - 1u));
        }
        const auto there = [&](float z, int i) {
            const unsigned k = key_of(z);
            return kept(z, i, border) && (by_bin ? first_bin(z) == bin : k >= lo && k <= hi);
        };
        if (s.found.count > SP_PAIRS) {
            // ties: the one of them in order of index at which it is reached
            u64 nth = want - before;
            if (MASS) {
                const u64 q = mass(value_of_key(lo));
                nth = (nth + q - 1) / q;
            }
            // (a thread's elements are consecutive)
            const int each = (n + SP_THREADS - 1) / SP_THREADS, i0 = min(n, threadIdx.x * each), i1 = min(n, i0 + each);
            int here = 0;
            for (int i = i0; i < i1; ++i) here += there(value(i), i);
            u64 block_sum, all;
            u64 in_front = scan(here, block_sum);
            in_front += gather(block_sum, all);
            if (in_front < nth && nth <= in_front + here) {
                for (int i = i0; i < i1; ++i)
                    if (there(value(i), i) && ++in_front == nth) {
                        tell(value_of_key(lo), begin + i);
                    }
            }
        } else {
            // all of them to the first block
            const uint32_t listed = at_rank(&s.listed, 0);
            for (int i = threadIdx.x; i < n; i += SP_THREADS) {
                const float z = value(i);
                if (!there(z, i)) continue;
                unsigned slot;
                asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;" : "=r"(slot) : "r"(listed) : "memory");
                put32(at_rank(&s.weights.list_key[slot], 0), key_of(z));
                put32(at_rank(&s.weights.list_index[slot], 0), begin + i);
                if (MASS) put64(at_rank(&s.weights.list_mass[slot], 0), mass(z));
            }
            cluster_sync(blocks);
            if (rank == 0) {
                const int m = s.listed;
                if (threadIdx.x < m) {
                    const unsigned key = s.weights.list_key[threadIdx.x];
                    const int index = s.weights.list_index[threadIdx.x];
                    const u64 own = MASS ? s.weights.list_mass[threadIdx.x] : 1;
                    u64 b = before;
                    for (int j = 0; j < m; ++j) {
                        const unsigned k = s.weights.list_key[j];
                        if (k > key || (k == key && s.weights.list_index[j] < index)) b += MASS ? s.weights.list_mass[j] : 1;
                    }
                    if (b < want && want <= b + own) {
                        tell(value_of_key(key), index);
                    }
                }
            }
        }
        cluster_sync(blocks);
        border = s.border;
    }
};

template <typename T>
__global__ void __launch_bounds__(SP_THREADS, 2)
sample_kernel(const SampleParams p)
{
    extern __shared__ __align__(16) unsigned char sp_smem_raw[];
    SampleSmem &s = *reinterpret_cast<SampleSmem *>(sp_smem_raw);
    constexpr int PER = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    DIP_TRACE_MIN(p.tr, 0);
    s.table[tid] = exp2((double)tid / SP_TABLE) * (double)(1ull << SP_ONE_BITS);
    dip_grid_dependency_wait();
    DIP_TRACE_MIN(p.tr, 1);
    const unsigned blocks = cluster_size(), rank = cluster_rank();
    const int row = blockIdx.x / blocks, begin = min(p.vocab, (int)rank * p.slice), n = min(p.slice, p.vocab - begin);
    // the block's part of the row, at the same place within 16 bytes as in global memory
    const T *from = static_cast<const T *>(p.logits) + (size_t)row * p.pitch + begin;
    const int skew = (int)(((uintptr_t)from & 15) / sizeof(T));
    T *copy = reinterpret_cast<T *>(sp_smem_raw + sizeof(SampleSmem)) + skew;
    const T *items = p.resident ? copy : from;
    const int head = min(n, (PER - skew) % PER), vectors = (n - head) / PER;
    // (on the way: the largest logit, and binary32's lowest one that is open)
    float top = -INFINITY, low = sizeof(T) == 2 ? -3.402823466e38f : INFINITY;
    unsigned tops = 0xff80ff80u;
    const auto look = [&](float z) {
        top = fmaxf(top, z);                    // (NaN is not taken)
        low = fminf(low, z > -INFINITY ? z : INFINITY);
    };
    {
        const uint4 *v = reinterpret_cast<const uint4 *>(from + head);
        uint4 *to = reinterpret_cast<uint4 *>(copy + head);
        constexpr int U = 4;
        for (int i = tid; i < vectors; i += U * SP_THREADS) {
            uint4 a[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * SP_THREADS < vectors) a[u] = __ldcg(v + i + u * SP_THREADS);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * SP_THREADS < vectors) {
                    if (p.resident) to[i + u * SP_THREADS] = a[u];
                    if (sizeof(T) == 2) {
                        tops = max2(tops, max2(max2(a[u].x, a[u].y), max2(a[u].z, a[u].w)));
                    } else {
                        look(__uint_as_float(a[u].x));
                        look(__uint_as_float(a[u].y));
                        look(__uint_as_float(a[u].z));
                        look(__uint_as_float(a[u].w));
                    }
                }
        }
        const int done = head + vectors * PER;
        for (int i = tid; i < head + n - done; i += SP_THREADS) {
            const int at = i < head ? i : done + i - head;
            const T one = from[at];
            if (p.resident) copy[at] = one;
            look(item_value(&one, 0));
        }
    }
    if (sizeof(T) == 2) top = fmaxf(top, larger(tops));
    top += 0.f;                                 // (-0 is 0)
    dip_launch_dependents();
    const float temperature = p.temperature ? p.temperature[row] : 1.f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, u = p.uniform[row];
    const float min_p = p.min_p && temperature < INFINITY ? p.min_p[row] : 0.f;        // (all alike: it leaves all)
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
    if (lane == 0) {
        s.block_top[warp] = top;
        s.block_low[warp] = low;
    }
    if (tid == 0) {
        s.listed = 0;
        s.cut[0].bin = s.cut[1].bin = -1;
        s.near[0].coarse = s.near[1].coarse = -1;
    }
    __syncthreads();
    for (int w = 0; w < SP_WARPS; ++w) {
        top = fmaxf(top, s.block_top[w]);
        low = fminf(low, s.block_low[w]);
    }
    if (blocks > 1) {
        if (tid == 0) {
            s.top = top;
            s.low = low;
        }
        cluster_sync(blocks);
        const unsigned r = lane & (SP_CLUSTER - 1);
        if (r < blocks) {
            top = *of_rank(&s.top, r);
            low = *of_rank(&s.low, r);
        }
#pragma unroll
        for (int o = SP_CLUSTER / 2; o; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
        }
    }
    if (top == -INFINITY) {
        if (rank == 0 && tid == 0) {
            p.token[row] = -1;
            if (p.prob) p.prob[row] = 0.f;
        }
        cluster_sync(blocks);                   // (the others have read this block's)
        DIP_TRACE_MAX(p.tr, 2);
        return;
    }
    if (!(temperature > 0.f)) {
        int first = 0x7fffffff;
        for (int i = tid; i < n && first == 0x7fffffff; i += SP_THREADS)
            if (item_value(items, i) == top) first = begin + i;
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) s.block_first[warp] = first;
        __syncthreads();
        for (int w = 0; w < SP_WARPS; ++w) first = min(first, s.block_first[w]);
        if (tid == 0) put32(at_rank(&s.first[rank], 0), (unsigned)first);
        cluster_sync(blocks);
        if (rank == 0 && tid == 0) {
            for (unsigned r = 0; r < blocks; ++r) first = min(first, s.first[r]);
            p.token[row] = first;
            if (p.prob) p.prob[row] = 1.f;
        }
        DIP_TRACE_MAX(p.tr, 2);
        return;
    }

    const float spread = fminf(top - low, SP_SPREAD);
    const double steps = SP_TABLE * 1.4426950408889634074 / (double)temperature;
    const Row<T> r = {s, items, n, begin, rank, blocks, top, top < INFINITY ? steps : 1e300, Row<T>::wide(top) * 0x1p896, (float)steps,
                      spread > 1e-30f ? (SP_BINS - 1) / spread : 0.f, head, vectors};
    SampleBorder border = {-INFINITY, -1};
    const bool by_count = top_k > 0 && top_k < p.vocab, by_weight = top_p < 1.f;
    const auto share_of = [&](u64 all) { return max(1ull, (u64)ceil(fmax((double)top_p, 0.0) * (double)all)); };
    const auto count_of = [&](u64 all) { return min((u64)top_k, all); };
    // (bfloat16, weights by bins: the last bin's elements, from -2^20 down, weigh nothing)
    const bool counted = (by_count || by_weight) && r.scale > 0.f && (by_count || !Row<T>::HALF || (temperature <= 1000.f && fabsf(top) < 524288.f));
    bool count_done = !by_count, weight_done = !by_weight, alone = false;
    u64 all_weight = 0;
    unsigned listed = 0;
    if (counted) {
        r.histogram(!by_count);
        r.cuts(by_count ? top_k : 0, top_p);
        const auto first = s.cut[0], last = s.cut[Row<T>::HALF || by_count ? 0 : 1];
        const unsigned up_to = last.in_front + last.count;
        if (first.bin >= 0 && last.bin >= 0) {
            u64 sums[3];
            if (up_to <= SP_LIST) {
                // (binary32 by weight: the sum of all is not known yet, nor that the border is among these)
                const bool weigh = !by_count && !Row<T>::HALF;
                all_weight = s.all_weight;
                listed = r.collect(0, last.bin, weigh, sums);
                if (weigh) all_weight = sums[2];
                alone = !weigh || share_of(all_weight) <= sums[1];
            } else if (Row<T>::HALF) {
                if (!r.mixed(last.bin)) {
                    const float z = r.value_of(last.bin);
                    u64 nth = count_of(s.all_count) - last.in_front;
                    if (!by_count) {
                        const u64 q = r.mass(z);
                        nth = (last.want - last.before + q - 1) / q;
                    }
                    r.among_ties(z, nth);
                    border = s.border;
                    (by_count ? count_done : weight_done) = true;
                }
            } else if (up_to - first.in_front <= SP_LIST) {
                const bool weigh = !by_count;
                listed = r.collect(first.bin, last.bin, weigh, sums);
                const u64 want = weigh ? share_of(sums[2]) : count_of(s.all_count) - last.in_front;
                if (!weigh || (sums[0] < want && want <= sums[0] + sums[1])) {
                    if (rank == 0) {
                        const int i = r.reach(listed, [&](int j) { return r.number_in_order(j); }, [&](int j) { return weigh ? s.list.mass[j] : 1ull; },
                                              want - (weigh ? sums[0] : 0), 0, r.last_number(low));
                        if (tid == 0) r.tell(value_of_key(s.list.key[i]), s.list.index[i]);
                    }
                    cluster_sync(blocks);
                    border = s.border;
                    (by_count ? count_done : weight_done) = true;
                }
            }
        }
    } else if (min_p > 0.f && !by_count && !by_weight) {
        // (a little lower than need be: what is left out weighs less than min_p for certain)
        const float far = -temperature * logf(fminf(min_p, 1.f));
        u64 ignored[3];
        listed = r.collect(0, r.bin_of(top - far * 1.0001f - 1e-5f * fabsf(top) - 1e-37f), false, ignored);
        alone = listed <= SP_LIST;
    }
    if (alone) {
        if (rank == 0 && listed <= SP_FEW)
            r.finish_few(listed, by_count ? top_k : 0, top_p, min_p, u, all_weight, p.token + row, p.prob ? p.prob + row : nullptr);
        else if (rank == 0)
            r.finish(listed, by_count ? top_k : 0, top_p, min_p, u, all_weight, low, p.vocab, p.token + row, p.prob ? p.prob + row : nullptr);
        DIP_TRACE_MAX(p.tr, 2);
        return;
    }
    if (!count_done) r.template shorten<false>(border, count_of);
    if (!weight_done) r.template shorten<true>(border, share_of);

    // The draw.  Where a block has more bfloat16 logits than there are values of them that count, their weights
    // are worked out once.
    const int top_bin = r.bin_of(top);
    int known = 0;                              // bins whose weights are in s.bin_mass
    if (Row<T>::HALF && n > 4096 && fabsf(top) < INFINITY) {
        known = min(4096, 8191 - top_bin);
        if (border.z > -INFINITY) known = min(known, r.bin_of(border.z) - top_bin + 1);
        __syncthreads();
        for (int i = tid; i < known; i += SP_THREADS) s.bin_mass[i] = r.mass(r.value_of(top_bin + i));
        __syncthreads();
    }
    // (what min_p leaves, too, is the front of the order; only within a hair of its end does it take the weight itself to tell)
    const float cut = min_p > 0.f ? temperature * logf(fminf(min_p, 1.f)) : -INFINITY, hair = 1e-4f * -cut + 1e-5f * fabsf(top) + 1e-37f;
    const float sure = min_p > 0.f ? top + cut + hair : -INFINITY, doubtful = min_p > 0.f ? top + cut - hair : -INFINITY;
    const auto left = [&](float z, int i) {
        return r.kept(z, i, border) && (z >= sure || z == top || (z >= doubtful && r.likely(z, min_p)));
    };
    const auto drawn = [&](float z, int i) -> u64 { return left(z, i) ? r.mass(z) : 0; };
    constexpr int PIECE = Row<T>::PER;
    // (bfloat16 above zero, all of whose weights are known: the weight of the nth value below the largest is the nth, so that a logit takes a difference
    // and a look; what is behind the border, which is a tie, is taken away again)
    const unsigned top_raw = __float_as_uint(top) >> 16;
    const bool by_value = Row<T>::HALF && known > 0 && known < 4096 && border.z > 0.f && r.bin_of(border.z) == top_bin + known - 1 && top_bin > 0 &&
                          r.bin_of(border.z) < 4095 && min_p <= 0.f;
    if (by_value) {
        __syncthreads();
        if (tid == 0) s.bin_mass[known] = 0;
        __syncthreads();
    }
    r.in_order(
        border.z, [&](const uint4 &a, int i) -> u64 {
            u64 sum = 0;
            if (by_value) {
                const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned p0 = min(top_raw - (w[j] & 0xffffu), (unsigned)known), p1 = min(top_raw - (w[j] >> 16), (unsigned)known);
                    sum += s.bin_mass[p0] + s.bin_mass[p1];
                    if (p0 == known - 1 && begin + i + 2 * j > border.index) sum -= s.bin_mass[known - 1];
                    if (p1 == known - 1 && begin + i + 2 * j + 1 > border.index) sum -= s.bin_mass[known - 1];
                }
                return sum;
            }
            float z[PIECE];
            r.decode(a, z);
            u64 q[PIECE];
            bool in[PIECE], any = false, unknown = !Row<T>::HALF;
#pragma unroll
            for (int j = 0; j < PIECE; ++j) any |= in[j] = left(z[j], i + j);
            if (!any) return 0;
            if (Row<T>::HALF) {
#pragma unroll
                for (int j = 0; j < PIECE; ++j) {
                    const int bin = r.bin_of(z[j]), at = bin - top_bin;
                    unknown |= in[j] && (at >= known || r.mixed(bin));
                    q[j] = in[j] && at < known ? s.bin_mass[at] : 0;
                }
            }
            if (unknown) {
#pragma unroll
                for (int j = 0; j < PIECE; ++j) q[j] = r.mass(z[j]);
#pragma unroll
                for (int j = 0; j < PIECE; ++j) q[j] = in[j] ? q[j] : 0;
            }
#pragma unroll
            for (int j = 0; j < PIECE; ++j) sum += q[j];
            return sum;
        },
        drawn,
        // the smallest index at which the sum in order of index is above u of all
        [&](u64 all) { return min(all - 1, (u64)(fmax((double)u, 0.0) * (double)all)); },
        [&](int i, float z, u64 all) {
            p.token[row] = begin + i;
            if (p.prob) p.prob[row] = (float)(r.weight(z) / (double)all);
        });
    DIP_TRACE_MAX(p.tr, 2);
}

template <typename T>
cudaError_t launch(dip_ctx *ctx, int rows, int blocks, cudaStream_t stream, const SampleParams &p)
{
    static dip_per_device_once once;
    const size_t smem = sizeof(SampleSmem) + (p.resident ? ((size_t)p.slice * sizeof(T) + 31) / 16 * 16 : 0);
    cudaError_t e = dip_raise_smem_limit(once, ctx->device, sample_kernel<T>, 227 * 1024);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)rows * blocks);
    cfg.blockDim = dim3(SP_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T>, p);
}

// What is written, and what must not share memory with it.
struct Bytes {
    const void *p;
    size_t n;
};
bool apart(std::initializer_list<Bytes> written, std::initializer_list<Bytes> read)
{
    const auto meet = [](const Bytes &a, const Bytes &b) {
        return a.p && b.p && (uintptr_t)a.p < (uintptr_t)b.p + b.n && (uintptr_t)b.p < (uintptr_t)a.p + a.n;
    };
    for (const Bytes *w = written.begin(); w != written.end(); ++w) {
        for (const Bytes &r : read)
            if (meet(*w, r)) return false;
        for (const Bytes *o = written.begin(); o != w; ++o)
            if (meet(*w, *o)) return false;
    }
    return true;
}
// Whether a piece meets any of n rows of `each` bytes, whose starts are `pitch` bytes apart (what lies between them is not read).
bool meets_rows(const Bytes &a, const void *rows, size_t n, size_t each, size_t pitch)
{
    const uintptr_t r = (uintptr_t)rows, at = (uintptr_t)a.p;
    if (!a.p || at + a.n <= r) return false;
    const size_t first = at > r ? at - r : 0, row = first / pitch;
    return row < n && (first - row * pitch < each || (row + 1 < n && (row + 1) * pitch < at + a.n - r));
}

}  // namespace

extern "C" dip_status dip_sample_tokens(dip_ctx *ctx, const void *logits, int logits_bf16, int n_rows, int vocab, int64_t pitch,
                                        const dip_sampling *how, const float *uniform, int32_t *token, float *prob, void *stream)
{
    if (!dip_ctx_current(ctx) || !logits || !uniform || !token || (uintptr_t)logits % (logits_bf16 ? 2 : 4)) return DIP_ERR_INVALID_ARG;
    if (n_rows < 1 || n_rows > DIP_MAX_TOKENS || vocab < 1 || vocab > DIP_MAX_OUT || pitch < vocab || pitch > (int64_t)1 << 40)
        return DIP_ERR_INVALID_ARG;
    const dip_sampling none = {};
    if (!how) how = &none;
    for (const void *q : {(const void *)how->temperature, (const void *)how->top_k, (const void *)how->top_p, (const void *)how->min_p,
                          (const void *)uniform, (const void *)token, (const void *)prob})
        if ((uintptr_t)q % 4) return DIP_ERR_INVALID_ARG;
    const size_t item = logits_bf16 ? 2 : 4, each = (size_t)n_rows * 4;
    if (!apart({{token, each}, {prob, each}}, {{how->temperature, each}, {how->top_k, each}, {how->top_p, each}, {how->min_p, each}, {uniform, each}}) ||
        meets_rows({token, each}, logits, n_rows, vocab * item, pitch * item) || meets_rows({prob, each}, logits, n_rows, vocab * item, pitch * item))
        return DIP_ERR_INVALID_ARG;
    // As many blocks per row as find room (two per SM), if each has 1024 logits and more.  (1, 2, 4, 8 blocks, us: a row of 1000 bfloat16 logits 12.1, 13.8,
    // 13.9, 14.8, of 9000 16.3, 16.4, 14.7, 15.0, of 32064 22.5, 19.0, 16.4, 15.2; a row of 102400 binary32 ones 40.0, 28.0, 20.3, 17.0, 64 rows 120, 75, 60.5, 61.7.)
    // Their parts of the rows stay in shared memory if they fit beside what else is there, and
    // are read again, out of L2, if not.
    int blocks = 1;
    while (blocks < SP_CLUSTER && n_rows * blocks * 2 <= 2 * ctx->sm_count && vocab > 2048 * blocks) blocks *= 2;
    const int slice = ((vocab + blocks - 1) / blocks + 31) & ~31;
    SampleParams p = {};
    p.logits = logits;
    p.pitch = (size_t)pitch;
    p.vocab = vocab;
    p.slice = slice;
    p.resident = (size_t)slice * item + 64 + sizeof(SampleSmem) <= (n_rows * blocks <= ctx->sm_count ? 220 : 112) * 1024;
    p.temperature = how->temperature;
    p.top_k = how->top_k;
    p.top_p = how->top_p;
    p.min_p = how->min_p;
    p.uniform = uniform;
    p.token = token;
    p.prob = prob;
    p.tr = dip_trace_slot(ctx, 12);
    const cudaStream_t s = (cudaStream_t)stream;
    DIP_CUDA_TRY(ctx, logits_bf16 ? launch<uint16_t>(ctx, n_rows, blocks, s, p) : launch<float>(ctx, n_rows, blocks, s, p));
    return DIP_OK;
}
