// The choice of a token from its logits: temperature, top-k, top-p, min-p and one given number per row (include/dip.h has the definition).
//
// A row is read once, into the shared memory of a cluster of up to eight blocks, and stays there.  Weights are
// exp((z - max) / temperature) as whole multiples of 2^-45 of the largest one, computed in binary64: sums of them are exact whatever their order,
// so results depend neither on how a row is shared out nor on the order of atomics, and a row's 2^18 weights fit 64 bits.
//
// Top-k and top-p both keep the front of the row's order (logit descending, index ascending), which ends at some element: its key and
// its index.  Finding it is a histogram (of counts, or of weights) over bins of equal width below the largest logit, whose bins
// each block adds up a part of; then, in the bin where the front ends, either all pairs of its elements compared (up to
// SP_LIST), or histograms of the keys' next bits until one key is left, and a count in order of index among its ties.
// The draw adds up the kept weights per warp (whose elements are consecutive), then looks closer where the sum crosses the number.
#include <initializer_list>

#include "common.cuh"
#include "gemv_common.cuh"

namespace {

constexpr int SP_THREADS = 512, SP_WARPS = SP_THREADS / 32;
constexpr int SP_CLUSTER = 8;                   // most blocks per row
constexpr int SP_BINS = 2048;
constexpr int SP_LIST = 512;                    // elements that are compared pair by pair
constexpr int SP_TABLE = 512;                   // 2^(j / 512)
constexpr int SP_ONE_BITS = 45;                 // the largest weight is 2^45
constexpr float SP_SPREAD = 64.f;               // logits further below the largest one share the last bin of the first histogram

typedef unsigned long long u64;

struct SampleParams {
    const void *logits;
    size_t pitch;
    int vocab, slice;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
    u64 *tr;
};

struct SampleBorder {
    unsigned key;
    int index;
};

struct __align__(16) SampleSmem {
    double table[SP_TABLE];
    u64 mass[SP_BINS];
    unsigned count[SP_BINS];
    u64 list_mass[SP_LIST];
    unsigned list_key[SP_LIST];
    int list_index[SP_LIST];
    int listed;
    u64 scan[SP_WARPS + 1];
    // what the blocks of a cluster tell one another
    u64 total[SP_CLUSTER];
    float top[SP_CLUSTER], low[SP_CLUSTER];
    int first[SP_CLUSTER];
    unsigned key_lo[SP_CLUSTER], key_hi[SP_CLUSTER];
    struct {
        int bin;
        unsigned count;
        u64 before;
    } found;
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
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
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
__device__ __forceinline__ unsigned get32(uint32_t a)
{
    unsigned v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ u64 get64(uint32_t a)
{
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ unsigned key_of(float z)
{
    const unsigned u = __float_as_uint(z);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float item_value(const float *p, int i) { return p[i] + 0.f; }          // (-0 is 0)
__device__ __forceinline__ float item_value(const uint16_t *p, int i) { return __uint_as_float((unsigned)p[i] << 16) + 0.f; }

template <typename T>
struct Row {
    SampleSmem &s;
    const T *items;                             // this block's, in shared memory
    int n, begin;                               // how many; the first one's index
    unsigned rank, blocks;
    float top;                                  // the largest logit
    double steps;                               // 512 log2(e) / temperature
    float scale;                                // bins per unit

    __device__ __forceinline__ float value(int i) const { return item_value(items, i); }

    // exp((z - top) / temperature): 2^(k / 512) from the table times the third-order sum for what is left (within 10^-14)
    __device__ __forceinline__ double weight(float z) const
    {
        if (z == top) return 1.0;
        if (top == INFINITY) return 0.0;
        const double y = ((double)z - (double)top) * steps;
        if (!(y > -60.0 * SP_TABLE)) return 0.0;
        const double magic = 6755399441055744.0, k = y + magic;
        const int i = __double2loint(k);
        const double f = (y - (k - magic)) * (0.69314718055994530942 / SP_TABLE);
        const double t = s.table[i & (SP_TABLE - 1)];
        const double e = fma(t, f * fma(f, fma(f, 1.0 / 6.0, 0.5), 1.0), t);
        return __hiloint2double(__double2hiint(e) + ((i >> 9) << 20), __double2loint(e));
    }
    __device__ __forceinline__ u64 mass(float z) const
    {
        const double q = weight(z) * (double)(1ull << SP_ONE_BITS) + 4503599627370496.0;
        return (u64)__double_as_longlong(q) & 0xfffffffffffffull;
    }
    // whether the element is open and in front of the border (or it)
    __device__ __forceinline__ bool kept(float z, int i, const SampleBorder &b) const
    {
        const unsigned k = key_of(z);
        return z > -INFINITY && (k > b.key || (k == b.key && begin + i <= b.index));
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
        u64 before = 0;
        sum = 0;
        for (int w = 0; w < SP_WARPS; ++w) {
            const u64 a = s.scan[w];
            before += w < warp ? a : 0;
            sum += a;
        }
        return before + incl - v;
    }
    // The same over the cluster, given this block's sum: what is in front of this block, and all.  Ends with a cluster barrier.
    __device__ __forceinline__ u64 gather(u64 mine, u64 &all) const
    {
        if (threadIdx.x < blocks) put64(at_rank(&s.total[rank], threadIdx.x), mine);
        cluster_sync();
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
            s.mass[i] = 0;
            s.count[i] = 0;
        }
        if (threadIdx.x == 0) s.listed = 0;
        __syncthreads();
    }
    template <bool MASS>
    __device__ __forceinline__ void add(int bin, float z) const
    {
        atomicAdd(&s.count[bin], 1u);
        if (MASS) {
            const u64 q = mass(z);
            unsigned *w = reinterpret_cast<unsigned *>(&s.mass[bin]);
            const unsigned lo = (unsigned)q, was = atomicAdd(w, lo), hi = (unsigned)(q >> 32) + (was + lo < lo);
            if (hi) atomicAdd(w + 1, hi);
        }
    }

    // The bins' sums over the cluster are in order: the bin in which `want` (counted from 1) is reached, with what is in front of it and how
    // many elements it has, in s.found of every block.  want == 0: goal(sum of all bins) says.
    template <bool MASS, class Goal>
    __device__ __forceinline__ u64 locate(u64 want, const Goal &goal) const
    {
        cluster_sync();                         // (all blocks have counted)
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
                    count[j] += get32(at_rank(&s.count[b0 + j], r));
                    if (MASS) unit[j] += get64(at_rank(&s.mass[b0 + j], r));
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
        cluster_sync();
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
        while (s.found.count > SP_LIST) {
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
                cluster_sync();
                lo = 0xffffffffu;
                hi = 0u;
                for (unsigned r = 0; r < blocks; ++r) {
                    lo = min(lo, get32(at_rank(&s.key_lo[0], r)));
                    hi = max(hi, get32(at_rank(&s.key_hi[0], r)));
                }
                cluster_sync();
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
        if (s.found.count > SP_LIST) {
            // ties: the one of them in order of index at which it is reached
            u64 nth = want - before;
            if (MASS) {
                const unsigned u = lo ^ (~(unsigned)((int)lo >> 31) | 0x80000000u);
                const u64 q = mass(__uint_as_float(u));
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
                        for (unsigned r = 0; r < blocks; ++r) {
                            put32(at_rank(&s.border.key, r), lo);
                            put32(at_rank(&s.border.index, r), begin + i);
                        }
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
                put32(at_rank(&s.list_key[slot], 0), key_of(z));
                put32(at_rank(&s.list_index[slot], 0), begin + i);
                if (MASS) put64(at_rank(&s.list_mass[slot], 0), mass(z));
            }
            cluster_sync();
            if (rank == 0) {
                const int m = s.listed;
                if (threadIdx.x < m) {
                    const unsigned key = s.list_key[threadIdx.x];
                    const int index = s.list_index[threadIdx.x];
                    const u64 own = MASS ? s.list_mass[threadIdx.x] : 1;
                    u64 b = before;
                    for (int j = 0; j < m; ++j) {
                        const unsigned k = s.list_key[j];
                        if (k > key || (k == key && s.list_index[j] < index)) b += MASS ? s.list_mass[j] : 1;
                    }
                    if (b < want && want <= b + own) {
                        for (unsigned r = 0; r < blocks; ++r) {
                            put32(at_rank(&s.border.key, r), key);
                            put32(at_rank(&s.border.index, r), index);
                        }
                    }
                }
            }
        }
        cluster_sync();
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
    s.table[tid] = exp2((double)tid / SP_TABLE);
    dip_grid_dependency_wait();
    DIP_TRACE_MIN(p.tr, 1);
    const unsigned blocks = cluster_size(), rank = cluster_rank();
    const int row = blockIdx.x / blocks, begin = min(p.vocab, (int)rank * p.slice), n = min(p.slice, p.vocab - begin);
    // the block's part of the row, at the same place within 16 bytes as in global memory
    const T *from = static_cast<const T *>(p.logits) + (size_t)row * p.pitch + begin;
    const int skew = (int)(((uintptr_t)from & 15) / sizeof(T));
    T *items = reinterpret_cast<T *>(sp_smem_raw + sizeof(SampleSmem)) + skew;
    const int head = min(n, (PER - skew) % PER), vectors = (n - head) / PER;
    {
        const uint4 *v = reinterpret_cast<const uint4 *>(from + head);
        uint4 *to = reinterpret_cast<uint4 *>(items + head);
        constexpr int U = 4;
        for (int i = tid; i < vectors; i += U * SP_THREADS) {
            uint4 a[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * SP_THREADS < vectors) a[u] = __ldcs(v + i + u * SP_THREADS);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * SP_THREADS < vectors) to[i + u * SP_THREADS] = a[u];
        }
        if (tid < head) items[tid] = from[tid];
        const int done = head + vectors * PER;
        if (tid < n - done) items[done + tid] = from[done + tid];
    }
    dip_launch_dependents();
    const float temperature = p.temperature ? p.temperature[row] : 1.f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f, u = p.uniform[row];
    __syncthreads();

    // the largest logit, the first one of them, and how far below it the others are
    float top = -INFINITY, low = INFINITY;
    for (int i = tid; i < n; i += SP_THREADS) {
        const float z = item_value(items, i);
        top = fmaxf(top, z);                    // (NaN is not taken)
        if (z > -INFINITY) low = fminf(low, z);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
    if (lane == 0) {
        s.block_top[warp] = top;
        s.block_low[warp] = low;
    }
    __syncthreads();
    for (int w = 0; w < SP_WARPS; ++w) {
        top = fmaxf(top, s.block_top[w]);
        low = fminf(low, s.block_low[w]);
    }
    cluster_sync();                             // (all blocks are there)
    if (tid < (int)blocks) {
        put32(at_rank(&s.top[rank], tid), __float_as_uint(top));
        put32(at_rank(&s.low[rank], tid), __float_as_uint(low));
    }
    cluster_sync();
    for (unsigned r = 0; r < blocks; ++r) {
        top = fmaxf(top, s.top[r]);
        low = fminf(low, s.low[r]);
    }
    if (top == -INFINITY) {
        if (rank == 0 && tid == 0) {
            p.token[row] = -1;
            if (p.prob) p.prob[row] = 0.f;
        }
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
        cluster_sync();
        if (rank == 0 && tid == 0) {
            for (unsigned r = 0; r < blocks; ++r) first = min(first, s.first[r]);
            p.token[row] = first;
            if (p.prob) p.prob[row] = 1.f;
        }
        DIP_TRACE_MAX(p.tr, 2);
        return;
    }

    const float spread = fminf(top - low, SP_SPREAD);
    const Row<T> r = {s, items, n, begin, rank, blocks, top, SP_TABLE * 1.4426950408889634074 / (double)temperature,
                      spread > 1e-30f ? (SP_BINS - 1) / spread : 0.f};
    SampleBorder border = {0u, 0x7fffffff};
    if (top_k > 0 && top_k < p.vocab)
        r.template shorten<false>(border, [&](u64 all) { return min((u64)top_k, all); });
    if (top_p < 1.f)
        r.template shorten<true>(border, [&](u64 all) { return max(1ull, (u64)ceil(fmax((double)top_p, 0.0) * (double)all)); });

    // the draw: a warp's elements are consecutive
    const double least = fmin((double)min_p, 1.0);
    const auto drawn = [&](int i) -> u64 {
        const float z = r.value(i);
        return r.kept(z, i, border) && !(min_p > 0.f && r.weight(z) < least) ? r.mass(z) : 0;
    };
    const int each = ((n + SP_WARPS - 1) / SP_WARPS + 31) & ~31, i0 = min(n, warp * each), i1 = min(n, i0 + each);
    u64 sum = 0;
    for (int i = i0 + lane; i < i1; i += 32) sum += drawn(i);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s.scan[warp] = sum;
    __syncthreads();
    u64 block_sum = 0, all;
    for (int w = 0; w < SP_WARPS; ++w) block_sum += s.scan[w];
    const u64 before = r.gather(block_sum, all);
    // the smallest index at which the sum in order of index is above u of all
    const u64 mark = min(all - 1, (u64)(fmax((double)u, 0.0) * (double)all));
    if (before <= mark && mark < before + block_sum) {
        u64 at = before;
        int w = 0;
        for (; at + s.scan[w] <= mark; ++w) at += s.scan[w];
        const int j0 = min(n, w * each), j1 = min(n, j0 + each), part = (each + SP_THREADS - 1) / SP_THREADS;
        const int k0 = min(j1, j0 + tid * part), k1 = min(j1, k0 + part);
        u64 mine = 0, ignored;
        for (int i = k0; i < k1; ++i) mine += drawn(i);
        at += r.scan(mine, ignored);
        if (at <= mark && mark < at + mine) {
            int i = k0;
            for (u64 q; at + (q = drawn(i)) <= mark; ++i) at += q;
            p.token[row] = begin + i;
            if (p.prob) p.prob[row] = (float)(r.weight(r.value(i)) * (double)(1ull << SP_ONE_BITS) / (double)all);
        }
    }
    DIP_TRACE_MAX(p.tr, 2);
}

template <typename T>
cudaError_t launch(dip_ctx *ctx, int rows, int blocks, cudaStream_t stream, const SampleParams &p)
{
    static dip_per_device_once once;
    const size_t smem = sizeof(SampleSmem) + ((size_t)p.slice * sizeof(T) + 31) / 16 * 16;
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
    if (!apart({{token, each}, {prob, each}}, {{logits, ((size_t)(n_rows - 1) * pitch + vocab) * item}, {how->temperature, each}, {how->top_k, each},
                                               {how->top_p, each}, {how->min_p, each}, {uniform, each}}))
        return DIP_ERR_INVALID_ARG;
    // As many blocks per row as its items need (two blocks share an SM), and more where SMs are idle.
    const size_t room = 110 * 1024 - sizeof(SampleSmem) - 64;
    int blocks = 1;
    while (blocks < SP_CLUSTER && ((size_t)vocab * item > room * blocks || ((long long)n_rows * blocks * 2 <= ctx->sm_count && vocab > 2048 * blocks)))
        blocks *= 2;
    SampleParams p = {};
    p.logits = logits;
    p.pitch = (size_t)pitch;
    p.vocab = vocab;
    p.slice = ((vocab + blocks - 1) / blocks + 31) & ~31;
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
