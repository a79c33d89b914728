// Operators that pick entries out of rows of vocabulary logits:
//   sample_rows_kernel  one token per row from a given uniform, under temperature, top-k, top-p and min-p;
//   top_rows_kernel     the K largest logits of a row, their ids, and the row's log-sum-exp.
//
// Both rest on one order of a row's entries -- larger logit first, lower id first among equals -- and on finding
// the entry at which the running count, or the running mass, of that order passes a given value.  Masses are whole
// numbers: entry i weighs w_i = rint(2^31 exp((l_i - max) / T)), so that every sum is exact and the same in whatever
// order, block or split it is taken, and a draw does not depend on the batch it is part of.
//
// A cluster of 1 to 8 CTAs shares a row; what a step needs of the whole row goes through distributed shared memory.
//   Streaming pass.  The row is read from HBM once: the largest logit of each of four groups of units per thread, and
//   the thread's sum of exponentials.
//   Top-k (a list of at most 1024).  The r-th largest of the groups' largest logits bounds the r-th largest logit from
//   below, because r groups hold one at least as large: a threshold without a histogram.  The few groups that reach
//   it are read again (from L2), their entries at or above it -- not many more than r -- go to the cluster's first CTA,
//   which sorts them and is left with a short list.
//   Masses (no top-k).  A second pass (from L2) adds the weights up in 1024 bins of the exponent.  The bin in which the
//   wanted mass lies is a range of keys; its entries, or all from there on up where they are few, are the list.
//   Where a list would be too long (ties, nearly flat rows, a top-k beyond 1024), the cluster narrows the interval of
//   keys, then of ids, by counting in 64 bins a level.
//
// Bound: for few rows the chain of steps.  1 x 151936 bf16 with top-k and nucleus 12 us: pass 2.5, exchange 2.1, list 2.5, sort 2.1,
// draw 1.4.  16 x 151936 fp32, nothing cut off, 24 us: pass 2.5, exchange 1.4, masses 7.1, bin 2.8, list 2.8, narrowing 1.7.  For many
// the two passes over the row: 256 x 151936 bf16, mixed settings, 95 us, of which a row without top-k takes 70 (pass 16, masses 40 to
// 45, the search 7 to 10), one with top-k 25, and a greedy one 35 (14 of them listing the largest among its own units again).
#include "row_picks.cuh"

namespace specs {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kGroups = 4;                   // groups of a thread's units, one running maximum each
constexpr int kMaxCluster = 8;
constexpr int kListCap = 2048, kPer = kListCap / kThreads;   // entries of the first CTA's list; of a thread
constexpr int kMassBins = 1024, kCoarse = 64, kFine = kMassBins / kCoarse;
constexpr float kBinsPerUnit = 45.0f;        // bins per unit of the exponent: weights end at 22.2, bin 999
constexpr int kBins = 64, kMaxLevels = 12;   // narrowing: 32 bits of a key and 19 of an id, 6 a level, take 10 at most
constexpr int kLeastUnits = 1024, kLongUnits = 16000;
constexpr uint32_t kHighestKey = 0xffffffffu, kKeyOfMinusZero = 0x7fffffffu;   // order_key has both zeros at 0x80000000

// Temperature in the exponent.  NaN and what is too small to weigh anything become -30, so that no special case remains.
__device__ __forceinline__ float scaled(float l, float top, float inv_t) { return fmaxf((l - top) * inv_t, -30.0f); }
// exp(z) for -30 <= z <= 0, of two exponents at a time: the product z log2(e) in two parts, the larger of them through the
// special-function unit.  Relative error 2^-22; 1 for 0.
__device__ __forceinline__ float2 powers_of(float2 z) {
    auto both = [](float v) { return make_float2(v, v); };
    const float2 x = __fmul2_rn(z, both(1.44269502f));
    const float2 lost = __ffma2_rn(z, both(1.44269502f), make_float2(-x.x, -x.y));
    const float2 m = __ffma2_rn(lost, both(0.693147181f), __fmul2_rn(z, both(1.3349706e-8f)));      // log2(e) has that much more
    const float2 e = make_float2(fast_exp2(x.x), fast_exp2(x.y));
    return __ffma2_rn(e, m, e);
}
// The weight of a power below 2^-8, which rounds to 2^23 at most, by adding 2^23: spares the slow conversion.
constexpr float kSmallPower = 0.00390625f;
__device__ __forceinline__ uint32_t small_weight(float scaled_up) { return __float_as_uint(scaled_up) - 0x4b000000u; }
__device__ __forceinline__ uint32_t weight_of(float z) {
    return __float2uint_rn(powers_of(make_float2(z, z)).x * 2147483648.0f);
}
__device__ __forceinline__ uint32_t place_weight(uint64_t place, float top, float inv_t) {
    return weight_of(scaled(key_value(place_key(place)), top, inv_t));
}
// Bin of an exponent: adding 2^21 leaves z kBinsPerUnit in quarters in the low bits.
constexpr float kBinShift = 2097152.0f;
__device__ __forceinline__ uint32_t bin_of(float z) {
    return (__float_as_uint(fmaf(z, -kBinsPerUnit, kBinShift)) - 0x4a000000u) >> 2;
}

// Entries that a search still considers: keys lo .. hi and ids first .. last, with what precedes them in the order.
struct Interval { uint32_t lo, hi; int first, last; uint64_t count_before, mass_before; };
struct Bin { uint64_t mass; uint32_t count; };
struct Narrow { uint32_t count[kBins], low[kBins], high[kBins]; };   // sums of w & 0xffff and of w >> 16
struct MassPart { uint64_t allowed; uint32_t weighted; };

struct Shared {
    union {
        uint64_t list[kListCap];                             // first CTA: the entries to sort
        struct { uint32_t count[kBins][32], low[kBins][32], high[kBins][32]; } h;   // narrowing: one column per lane
    };
    struct { uint32_t low[kMassBins], high[kMassBins]; } mass;   // sums of weights, and their carries
    uint16_t flags[kThreads * kGroups];                      // groups to read again
    Bin bins[2][kBins];                                      // the CTA's totals, by the parity of the level
    uint64_t coarse[kMaxCluster][kCoarse];                   // every CTA's masses, kFine bins at a time
    uint32_t group_key[kThreads * kGroups];                  // the groups' (or the threads') largest, for the bound
    uint32_t part_key[kMaxCluster], part_bound[kMaxCluster]; // every CTA's largest key, and bound
    float part_sum[kMaxCluster];                             // ... and sum of exponentials relative to its largest
    MassPart rest[kMaxCluster];
    uint32_t listed[2][kMaxCluster];                         // entries each CTA has pushed, by the parity of the round
    uint64_t red64[kWarps];
    float warp_top[kWarps], warp_sum[kWarps];
    uint32_t red32[kWarps];
    union { uint32_t rank[256]; uint32_t weight[kListCap]; };  // first CTA: ranks while it sorts, or what its entries weigh
    Narrow narrow;
    uint32_t ends[4][kWarps];                                // of the keys and ids in question
    uint32_t filled;                                         // first CTA: entries in its list
    uint32_t count, flagged, in_bin, complete;
    Interval at;
    uint64_t found_place, found_before, allowed, total;
    uint32_t* status;                                        // of the checked build
};

// By this name, and not by a reference handed down, so that out-of-line functions know that it is shared memory.
__device__ __forceinline__ Shared& shared() {
    extern __shared__ __align__(16) uint8_t smem[];
    return *reinterpret_cast<Shared*>(smem);
}

// The checked build's index checks report to the status word, which functions find in shared memory.  (Before the first barrier.)
__device__ __forceinline__ void report_to(Shared& s, uint32_t* status) {
#ifdef SPECS_DEBUG
    if (threadIdx.x == 0) s.status = status;
#endif
}

// What a thread knows of its row's cluster.
struct Cluster {
    int ranks, rank;
    __device__ Cluster() {
        asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    }
    __device__ __forceinline__ void sync() const {
        if (ranks > 1) asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
        else __syncthreads();
    }
    // the same shared memory in another CTA of the cluster, as a generic address
    __device__ __forceinline__ Shared* peer(Shared& s, int r) const {
        uint64_t there;
        asm("mapa.u64 %0, %1, %2;" : "=l"(there) : "l"(reinterpret_cast<uint64_t>(&s)), "r"(r));
        return reinterpret_cast<Shared*>(there);
    }
};

// Unit i * kThreads + t of the slice belongs to thread t and to its group i % kGroups.
template <typename T> using Slice = RowSlice<T, kThreads>;

// The block's sum, in every thread; `scratch` may be written again after the next barrier.
template <typename V>
__device__ __forceinline__ V block_sum(V v, V* scratch) {
    v = warp_reduce(v, AddOp());
    const int lane = threadIdx.x & 31;
    if (lane == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_reduce(lane < kWarps ? scratch[lane] : V(0), AddOp());
}

// ---- streaming pass -----------------------------------------------------------------------------
struct Streamed { uint32_t group_key[kGroups]; };

template <typename T>
__device__ __forceinline__ Streamed stream_slice(const Slice<T>& slice, bool want_sum, float c, Shared& s) {
    GroupMaxima<T, kGroups> row(c);
    slice.template each_batch<kGroups>([&](const uint4* q, int) { row.add(q, want_sum); });
    Streamed out;
    row.of_warp(want_sum, out.group_key, s.warp_top[threadIdx.x >> 5], s.warp_sum[threadIdx.x >> 5]);
    return out;
}

struct RowPart { uint32_t key, bound; float top; };

// What all CTAs know after the first exchange: the row's largest logit, and with `want` > 0 a key that at least that many of
// the row's groups reach.
__device__ RowPart exchange_parts(const Cluster& c, Shared& s, const Streamed& st, float scale, uint32_t want) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t share = (want + c.ranks - 1) / c.ranks;
    // The threads' largest will do where no more than 5/8 of them are wanted: that many reach a bound that about as many
    // entries again as are wanted reach at most.
    const bool many = share > kThreads / 8 * 5;
    if (many)
        reinterpret_cast<uint4*>(s.group_key)[threadIdx.x] = make_uint4(st.group_key[0], st.group_key[1], st.group_key[2], st.group_key[3]);
    else if (want > 0)
        s.group_key[threadIdx.x] = max(max(st.group_key[0], st.group_key[1]), max(st.group_key[2], st.group_key[3]));
    // a CTA may write to another's shared memory only once that one runs: they arrived when they started
    if (c.ranks > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    __syncthreads();
    if (warp == 0) {
        const float top = lane < kWarps ? s.warp_top[lane] : -INFINITY;
        const float most = warp_reduce(top, MaxOp());
        const float factor = top == -INFINITY || top == most ? 1.0f : fast_exp2((top - most) * scale);
        const float sum = warp_reduce(lane < kWarps ? s.warp_sum[lane] * factor : 0.0f, AddOp());
        if (lane < c.ranks) {
            Shared* peer = c.peer(s, lane);
            peer->part_key[c.rank] = order_key(most);
            peer->part_sum[c.rank] = sum;
        }
    } else if (warp == 1 && want > 0) {
        const uint32_t bound = bound_of_rank(s.group_key, many, share);
        if (lane < c.ranks) c.peer(s, lane)->part_bound[c.rank] = bound;
    }
    c.sync();
    RowPart row;
    row.key = __reduce_max_sync(kAllLanes, lane < c.ranks ? s.part_key[lane] : 0u);
    row.bound = want > 0 ? __reduce_min_sync(kAllLanes, lane < c.ranks ? s.part_bound[lane] : 0xffffffffu) : 0u;
    row.top = row.key >= kLowestKey ? key_value(row.key) : -INFINITY;
    return row;
}

// One warp: the logarithm of the row's sum of exponentials relative to its largest logit.
__device__ float log_row_sum(const Cluster& c, const Shared& s, const RowPart& row, float scale) {
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    if (lane < c.ranks) {
        const uint32_t key = s.part_key[lane];
        sum = (double)s.part_sum[lane] * (key < kLowestKey || key == row.key ? 1.0f : fast_exp2((key_value(key) - row.top) * scale));
    }
    return logf((float)warp_reduce(sum, AddOp()));
}

// Sorts the first n entries of the list, largest first (n <= kListCap).  Up to 256 entries: every entry's rank is counted,
// the threads sharing out the comparisons (256 entries: 64 16-byte loads a thread).  More: bitonic.
__device__ __noinline__ void sort_list(int n) {
    Shared& s = shared();
    if (!SPECS_IN_BOUNDS(n, kListCap + 1, s.status)) return;
    const int tid = threadIdx.x;
    int size = 32;
    while (size < n) size <<= 1;
    uint64_t* list = s.list;
    for (int i = n + tid; i < size; i += kThreads) list[i] = 0;
    uint32_t* rank = s.rank;
    if (size <= 256 && tid < size) rank[tid] = 0;
    __syncthreads();
    if (size <= 256) {
        const int i = tid & (size - 1), part = kThreads / size, span = size / part;      // span entries each
        const uint64_t v = list[i];
        uint32_t larger = 0;
        const ulonglong2* two = reinterpret_cast<const ulonglong2*>(list + (tid / size) * span);
#pragma unroll 4
        for (int k = 0; k < span / 2; ++k) {                 // span is 2 at least
            const ulonglong2 w = two[k];
            larger += (w.x > v) + (w.y > v);
        }
        if (larger) atomicAdd(&rank[i], larger);
        __syncthreads();
        const uint32_t at = tid < n ? rank[tid] : 0;
        __syncthreads();
        if (tid < n && SPECS_IN_BOUNDS(at, n, s.status)) list[at] = v;     // places are distinct, and so are the ranks
    } else if (size <= kThreads) {
        // a thread holds one entry: partners less than a warp apart swap by shuffles
        uint64_t v = list[tid];
        for (int k = 2; k <= size; k <<= 1) {
            for (int j = k >> 1; j > 0; j >>= 1) {
                uint64_t w;
                if (j < 32) {
                    w = __shfl_xor_sync(kAllLanes, v, j);
                } else {
                    __syncthreads();
                    list[tid] = v;
                    __syncthreads();
                    w = list[tid ^ j];
                }
                const bool larger = ((tid & k) == 0) == ((tid & j) == 0);
                v = larger == (v > w) ? v : w;
            }
        }
        __syncthreads();
        list[tid] = v;
    } else {
        for (int k = 2; k <= size; k <<= 1) {
            for (int j = k >> 1; j > 0; j >>= 1) {
                for (int t = tid; t < size / 2; t += kThreads) {
                    const int a = 2 * t - (t & (j - 1)), b = a + j;
                    const uint64_t x = list[a], y = list[b];
                    if ((x < y) == ((a & k) == 0)) { list[a] = y; list[b] = x; }
                }
                __syncthreads();
            }
        }
    }
    __syncthreads();
}

// Exclusive sum over the block's threads, in thread order; *total gets the sum.
template <typename V>
__device__ V block_before(V v, V* scratch, V* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V run = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V up = __shfl_up_sync(kAllLanes, run, o);
        if (lane >= o) run += up;
    }
    if (lane == 31) scratch[warp] = run;
    __syncthreads();
    V before = 0, sum = 0;
    for (int i = 0; i < kWarps; ++i) {
        if (i < warp) before += scratch[i];
        sum += scratch[i];
    }
    __syncthreads();
    *total = sum;
    return before + run - v;
}

// ---- the list -----------------------------------------------------------------------------------
__device__ __forceinline__ void push_entry(Shared& s, Shared* home, uint32_t key, int id, int V) {
    if (!SPECS_IN_BOUNDS(id, V, s.status)) return;
    atomicAdd(&s.count, 1u);
    const uint32_t pos = atomicAdd(&home->filled, 1u);
    if (pos < kListCap) home->list[pos] = place_of(key, id);
}

template <typename T>
__device__ __forceinline__ void push_unit(Shared& s, Shared* home, int V, const uint4& q, int id, uint32_t lo, uint32_t hi,
                                          int first, int last) {
    // (as numbers; an interval that ends at the key of -0, which no entry has, ends at the number below the zeros)
    const float least = key_value(lo), most = hi == kHighestKey ? INFINITY : key_value(hi == kKeyOfMinusZero ? hi - 1 : hi);
    float f[Elem<T>::kWidth];
    uint32_t in = 0;
    Elem<T>::widen(q, f);
#pragma unroll
    for (int e = 0; e < Elem<T>::kWidth; ++e) in |= (f[e] >= least && f[e] <= most ? 1u : 0u) << e;
    while (in) {                                             // few units have any
        const int e = __ffs(in) - 1;
        in &= in - 1;
        float v = f[0];
#pragma unroll
        for (int k = 1; k < Elem<T>::kWidth; ++k) v = e == k ? f[k] : v;
        if (id + e >= first && id + e <= last) push_entry(s, home, order_key(v), id + e, V);
    }
}

// Pushes the CTA's entries with keys lo .. hi and ids first .. last to the first CTA's list.  Where hi is open, only groups
// whose largest key reaches lo can hold any: those are shared out over the block unit by unit.  Else every thread looks its
// own units through.  Entries beyond the list's end are only counted.  Returns, in every CTA, how many the whole row has.
template <typename T>
__device__ __noinline__ uint32_t push_entries(const Cluster c, const Slice<T> slice, const Streamed st, uint32_t lo, uint32_t hi,
                                              int first, int last, int round) {
    Shared& s = shared();
    Shared* home = c.peer(s, 0);
    __syncthreads();
    if (threadIdx.x == 0) { s.count = 0; s.flagged = 0; }
    __syncthreads();
    if (hi == kHighestKey) {
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
            if (st.group_key[j] >= lo) {
                const uint32_t at = atomicAdd(&s.flagged, 1u);
                if (SPECS_IN_BOUNDS(at, kThreads * kGroups, s.status)) s.flags[at] = (uint16_t)(threadIdx.x * kGroups + j);
            }
        __syncthreads();
        const int per = (slice.row.units + kGroups * slice.step - 1) / (kGroups * slice.step);   // units of a group, at most
        const int work = (int)s.flagged * per;
        for (int w = threadIdx.x; w < work; w += kThreads) {
            const int flag = s.flags[w / per], n = w % per;
            const int u = slice.start(flag / kGroups) + (n * kGroups + flag % kGroups) * slice.step;
            if (u < slice.row.units && SPECS_IN_BOUNDS(u, slice.row.units, s.status))
                push_unit<T>(s, home, slice.row.V, slice.row.load(u), slice.row.first(u), lo, hi, first, last);
        }
    } else {
        slice.template each_batch<kGroups>([&](const uint4* q, int u) {
#pragma unroll 1
            for (int j = 0; j < kGroups; ++j)
                push_unit<T>(s, home, slice.row.V, j == 0 ? q[0] : j == 1 ? q[1] : j == 2 ? q[2] : q[3],
                             slice.row.first(u + j * slice.step), lo, hi, first, last);
        });
    }
    __syncthreads();
    if (threadIdx.x < c.ranks) c.peer(s, threadIdx.x)->listed[round & 1][c.rank] = s.count;
    c.sync();
    uint32_t n = 0;
    for (int r = 0; r < c.ranks; ++r) n += s.listed[round & 1][r];
    return n;
}

// The first CTA: what the entries of its list weigh.
__device__ __forceinline__ void weigh_list(Shared& s, int n, float top, float inv_t) {
    for (int i = threadIdx.x; i < n; i += kThreads) s.weight[i] = place_weight(s.list[i], top, inv_t);
}

// The first CTA: the entry at which the running mass (or, without by_mass, count) of its list first exceeds `goal`.  A round
// sorts the entries in question into 64 bins of their keys, or of their ids where the keys are all the same, until one is
// left.  s.found_before gets the list's mass before it.
__device__ __noinline__ void narrow_list(int n, bool by_mass, uint64_t goal) {
    Shared& s = shared();
    if (!SPECS_IN_BOUNDS(n, kListCap + 1, s.status)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t live = 0;
    __syncthreads();                                         // the weights are there
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int at = threadIdx.x + i * kThreads;
        if (at < n) live |= 1u << i;
    }
    uint64_t run = 0, mass_before = 0;
    for (int round = 0; round < kMaxLevels; ++round) {
        uint32_t least = 0xffffffffu, most = 0, first = 0xffffffffu, last = 0;     // of keys and of ids
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if ((live >> i) & 1u) {
                const uint64_t place = s.list[threadIdx.x + i * kThreads];
                const uint32_t key = place_key(place), id = (uint32_t)place_id(place);
                least = min(least, key); most = max(most, key);
                first = min(first, id); last = max(last, id);
            }
        least = __reduce_min_sync(kAllLanes, least); most = __reduce_max_sync(kAllLanes, most);
        first = __reduce_min_sync(kAllLanes, first); last = __reduce_max_sync(kAllLanes, last);
        if (lane == 0) { s.ends[0][warp] = least; s.ends[1][warp] = most; s.ends[2][warp] = first; s.ends[3][warp] = last; }
        if (threadIdx.x < kBins) s.narrow.count[threadIdx.x] = s.narrow.low[threadIdx.x] = s.narrow.high[threadIdx.x] = 0;
        __syncthreads();
        const int w = lane & (kWarps - 1);
        least = __reduce_min_sync(kAllLanes, s.ends[0][w]); most = __reduce_max_sync(kAllLanes, s.ends[1][w]);
        first = __reduce_min_sync(kAllLanes, s.ends[2][w]); last = __reduce_max_sync(kAllLanes, s.ends[3][w]);
        const bool by_key = least < most;
        const uint32_t range = by_key ? most - least : last - first;
        const int shift = max(0, 32 - __clz(range) - 6);     // range >> shift < 64
        uint32_t digit[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            digit[i] = kBins;
            if ((live >> i) & 1u) {
                const uint64_t place = s.list[threadIdx.x + i * kThreads];
                const uint32_t w = s.weight[threadIdx.x + i * kThreads];
                digit[i] = (by_key ? most - place_key(place) : (uint32_t)place_id(place) - first) >> shift;
                if (!SPECS_IN_BOUNDS(digit[i], kBins, s.status)) continue;
                atomicAdd(&s.narrow.count[digit[i]], 1u);
                atomicAdd(&s.narrow.low[digit[i]], w & 0xffffu);
                if (w >> 16) atomicAdd(&s.narrow.high[digit[i]], w >> 16);
            }
        }
        __syncthreads();
        // every warp scans for itself: two bins a lane
        uint64_t m[2];
        uint32_t count[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            m[i] = (uint64_t)s.narrow.low[2 * lane + i] + ((uint64_t)s.narrow.high[2 * lane + i] << 16);
            count[i] = s.narrow.count[2 * lane + i];
        }
        uint64_t mb = m[0] + m[1];
        uint32_t nb = count[0] + count[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t um = __shfl_up_sync(kAllLanes, mb, o);
            const uint32_t un = __shfl_up_sync(kAllLanes, nb, o);
            if (lane >= o) { mb += um; nb += un; }
        }
        mb -= m[0] + m[1];
        nb -= count[0] + count[1];
        int hit = 2;
        uint64_t hit_run = 0, hit_mass = 0;
        uint32_t hit_count = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t at = run + (by_mass ? mb : (uint64_t)nb), step = by_mass ? m[i] : (uint64_t)count[i];
            if (at <= goal && goal < at + step) { hit = i; hit_run = at; hit_mass = mb; hit_count = count[i]; }
            mb += m[i];
            nb += count[i];
        }
        const unsigned who = __ballot_sync(kAllLanes, hit < 2);
        if (!who) break;                                     // goal is beyond the list: the caller's arithmetic rules that out
        const int from = __ffs(who) - 1;
        const uint32_t bin = 2 * from + __shfl_sync(kAllLanes, hit, from);
        run = __shfl_sync(kAllLanes, hit_run, from);
        mass_before += __shfl_sync(kAllLanes, hit_mass, from);
        hit_count = __shfl_sync(kAllLanes, hit_count, from);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (((live >> i) & 1u) && digit[i] != bin) live &= ~(1u << i);
        if (hit_count == 1) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if ((live >> i) & 1u) { s.found_place = s.list[threadIdx.x + i * kThreads]; s.found_before = mass_before; }
            break;
        }
        __syncthreads();                                     // the bins are read by all
    }
    __syncthreads();
}

// The first CTA: running masses of the sorted list, four entries a thread.
struct Running { uint64_t place[4]; uint32_t w[4]; uint64_t before; uint64_t total; };
__device__ Running run_list(Shared& s, int n, float top, float inv_t) {
    Running r;
    uint64_t sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = threadIdx.x * 4 + i;
        r.place[i] = at < n ? s.list[at] : 0;
        r.w[i] = at < n ? place_weight(r.place[i], top, inv_t) : 0;
        sum += r.w[i];
    }
    r.before = block_before(sum, s.red64, &r.total);
    return r;
}
// The entry at which the running mass first exceeds `goal` (a mass relative to the list's start).
__device__ void find_in(Shared& s, const Running& r, uint64_t goal) {
    uint64_t run = r.before;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (run <= goal && goal < run + r.w[i]) { s.found_place = r.place[i]; s.found_before = run; }
        run += r.w[i];
    }
    __syncthreads();
}

// The running mass that closes the nucleus, and the one a draw has to exceed.
__device__ __forceinline__ uint64_t nucleus_goal(uint64_t kept, float top_p) {
    const double goal = floor((double)kept * (double)top_p);
    return goal >= 1.0 ? (uint64_t)goal - 1 : 0;
}
__device__ __forceinline__ uint64_t draw_goal(uint64_t kept, float u) { return (uint64_t)floor((double)kept * (double)u); }

// The mass up to and with the entry that was found.
__device__ __forceinline__ uint64_t mass_upto(const Shared& s, float top, float inv_t) {
    return s.found_before + place_weight(s.found_place, top, inv_t);
}

// The whole cluster: the entry of the interval s.at (already the same in every CTA) at which the running mass or count
// first exceeds `goal`.  Every CTA gets s.found_place and s.found_before.
template <typename T>
__device__ __noinline__ void search(const Cluster c, const Slice<T> slice, const Streamed st, bool by_mass, uint64_t goal, float top,
                                    float inv_t, int round) {
    Shared& s = shared();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) s.found_place = 0;
    for (int level = 0; level < kMaxLevels; ++level) {
        const Interval at = s.at;
        const bool by_key = at.lo < at.hi;
        const uint32_t range = by_key ? at.hi - at.lo : (uint32_t)(at.last - at.first);
        const int shift = max(0, 32 - __clz(range) - 6);     // range >> shift < 64
        __syncthreads();
        for (int i = tid; i < kBins * 32; i += kThreads) {
            (&s.h.count[0][0])[i] = 0; (&s.h.low[0][0])[i] = 0; (&s.h.high[0][0])[i] = 0;
        }
        __syncthreads();
        for (int u = slice.start(tid); u < slice.row.units; u += slice.step) {
            float f[Elem<T>::kWidth];
            Elem<T>::widen(slice.row.load(u), f);
#pragma unroll 1
            for (int e = 0; e < Elem<T>::kWidth; ++e) {      // (rolled: rare, and long)
                float v = f[0];
#pragma unroll
                for (int k = 1; k < Elem<T>::kWidth; ++k) v = e == k ? f[k] : v;
                const uint32_t key = order_key(v);
                const int id = slice.row.first(u) + e;
                if (key < at.lo || key > at.hi || id < at.first || id > at.last) continue;
                const uint32_t d = (by_key ? at.hi - key : (uint32_t)(id - at.first)) >> shift;
                if (!SPECS_IN_BOUNDS(d, kBins, s.status)) continue;
                const uint32_t w = weight_of(scaled(v, top, inv_t));
                atomicAdd(&s.h.count[d][lane], 1u);
                atomicAdd(&s.h.low[d][lane], w & 0xffffu);   // a column gets a 32nd of the slice: below 2^15 entries
                atomicAdd(&s.h.high[d][lane], w >> 16);
            }
        }
        __syncthreads();
        for (int b = warp; b < kBins; b += kWarps) {
            const uint32_t n = __reduce_add_sync(kAllLanes, s.h.count[b][lane]);
            const uint64_t m = warp_reduce((uint64_t)s.h.low[b][lane] + ((uint64_t)s.h.high[b][lane] << 16), AddOp());
            if (lane == 0) { s.bins[level & 1][b].mass = m; s.bins[level & 1][b].count = n; }
        }
        if (tid == 0) { s.filled = 0; s.in_bin = 0; }
        c.sync();
        if (warp == 0) {                                     // two bins per lane, in the order of the entries
            uint64_t mass[2] = {0, 0}, count[2] = {0, 0};
            for (int r = 0; r < c.ranks; ++r) {
                const Bin* b = c.peer(s, r)->bins[level & 1] + 2 * lane;
                mass[0] += b[0].mass; count[0] += b[0].count;
                mass[1] += b[1].mass; count[1] += b[1].count;
            }
            const uint64_t m = mass[0] + mass[1], n = count[0] + count[1];
            uint64_t mb = m, cb = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t um = __shfl_up_sync(kAllLanes, mb, o), uc = __shfl_up_sync(kAllLanes, cb, o);
                if (lane >= o) { mb += um; cb += uc; }
            }
            mb += at.mass_before - m;
            cb += at.count_before - n;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t run = by_mass ? mb : cb, step = by_mass ? mass[i] : count[i];
                if (run <= goal && goal < run + step) {
                    const uint32_t d = 2 * lane + i;
                    Interval next = at;
                    next.mass_before = mb;
                    next.count_before = cb;
                    if (by_key) {
                        next.hi = at.hi - (d << shift);
                        next.lo = next.hi - min(next.hi - at.lo, (1u << shift) - 1);
                    } else {
                        next.first = at.first + (int)(d << shift);
                        next.last = min(at.last, next.first + (int)((1u << shift) - 1));
                    }
                    s.at = next;
                    s.in_bin = (uint32_t)count[i];
                }
                mb += mass[i];
                cb += count[i];
            }
        }
        __syncthreads();
        if (s.in_bin <= kListCap) break;
    }
    const Interval at = s.at;
    const int n = (int)push_entries(c, slice, st, at.lo, at.hi, at.first, at.last, round);
    if (c.rank == 0) {
        weigh_list(s, min(n, kListCap), top, inv_t);
        narrow_list(min(n, kListCap), by_mass, goal - (by_mass ? at.mass_before : at.count_before));
        if (tid < c.ranks) {
            Shared* peer = c.peer(s, tid);
            const uint64_t place = s.found_place, before = s.found_before + at.mass_before;
            __syncwarp((1u << c.ranks) - 1);                 // one of the peers is this CTA itself
            peer->found_place = place;
            peer->found_before = before;
        }
        if (tid == 0) s.filled = 0;
    }
    c.sync();
}

// ---- masses -------------------------------------------------------------------------------------
// The CTA's weights, added up by bins of their exponent, and the sums of kFine bins at a time sent to every CTA.  With
// `allowed` the mass of the entries that min_p allows, with `weighted` the number of entries that weigh anything.
// A bin's 32 bits wrap; whoever makes them wrap, as the atomic's result tells, adds a carry: exact, and one atomic an entry
// where sums of halves take two (151936 bf16 x 256 rows, mixed settings, on two CTAs each: 86 us, with halves and expf 103).
// Bound: about 20 instructions per entry.
template <typename T>
__device__ void add_masses(const Cluster& c, Shared& s, const Slice<T>& slice, float top, float inv_t, float low,
                           bool allowed, bool weighted) {
    const int tid = threadIdx.x;
    for (int i = tid; i < kMassBins; i += kThreads) s.mass.low[i] = s.mass.high[i] = 0;
    __syncthreads();
    MassPart mine = {0, 0};
    constexpr int kUnits = 16 / Elem<T>::kWidth, kWidth = Elem<T>::kWidth;
    auto bin = [](uint32_t* bins, uint32_t bits) {
        return reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(bins) + (bits & (4 * kMassBins - 4)));
    };
    slice.template each_batch<kUnits>([&](const uint4* q, int) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            float2 z[kWidth / 2], ex[kWidth / 2], at[kWidth / 2];
            uint32_t w[kWidth], sum[kWidth];
            float most = 0.0f;
            Elem<T>::widen(q[j], reinterpret_cast<float*>(z));
#pragma unroll
            for (int i = 0; i < kWidth / 2; ++i) {           // (as `scaled` and `bin_of` have it)
                z[i] = __fmul2_rn(__fadd2_rn(z[i], make_float2(-top, -top)), make_float2(inv_t, inv_t));
                z[i] = make_float2(fmaxf(z[i].x, -30.0f), fmaxf(z[i].y, -30.0f));
                ex[i] = powers_of(z[i]);
                at[i] = __ffma2_rn(z[i], make_float2(-kBinsPerUnit, -kBinsPerUnit), make_float2(kBinShift, kBinShift));
                most = fmaxf(most, fmaxf(ex[i].x, ex[i].y));
            }
            const float* power = reinterpret_cast<const float*>(ex);
            const float* bits = reinterpret_cast<const float*>(at);
            if (most < kSmallPower) {
#pragma unroll
                for (int e = 0; e < kWidth; ++e) w[e] = small_weight(fmaf(power[e], 2147483648.0f, 8388608.0f));
            } else {
#pragma unroll
                for (int e = 0; e < kWidth; ++e) w[e] = __float2uint_rn(power[e] * 2147483648.0f);
            }
            // (what weighs nothing lies beyond the bins)
#pragma unroll
            for (int e = 0; e < kWidth; ++e) {
                sum[e] = 0;
                if (w[e] && SPECS_IN_BOUNDS((__float_as_uint(bits[e]) - 0x4a000000u) >> 2, kMassBins, s.status))
                    sum[e] = atomicAdd(bin(s.mass.low, __float_as_uint(bits[e])), w[e]);
            }
            bool carry = false;
#pragma unroll
            for (int e = 0; e < kWidth; ++e) carry |= sum[e] + w[e] < w[e];
            if (carry) {
#pragma unroll
                for (int e = 0; e < kWidth; ++e)
                    if (sum[e] + w[e] < w[e]) atomicAdd(bin(s.mass.high, __float_as_uint(bits[e])), 1u);
            }
            if (allowed || weighted) {
                const float* zs = reinterpret_cast<const float*>(z);
#pragma unroll
                for (int e = 0; e < kWidth; ++e) {
                    if (zs[e] >= low) mine.allowed += w[e];
                    mine.weighted += w[e] != 0;
                }
            }
        }
    });
    if (allowed) mine.allowed = block_sum(mine.allowed, s.red64);
    if (weighted) mine.weighted = block_sum(mine.weighted, s.red32);
    __syncthreads();
    // two bins a thread, eight threads a sum
    uint64_t m = (uint64_t)s.mass.low[2 * tid] + s.mass.low[2 * tid + 1] +
                 (((uint64_t)s.mass.high[2 * tid] + s.mass.high[2 * tid + 1]) << 32);
#pragma unroll
    for (int o = 1; o < kFine / 2; o <<= 1) m += __shfl_xor_sync(kAllLanes, m, o);
    if (tid % (kFine / 2) == 0)
        for (int r = 0; r < c.ranks; ++r) c.peer(s, r)->coarse[c.rank][tid / (kFine / 2)] = m;
    if (tid < c.ranks) c.peer(s, tid)->rest[c.rank] = mine;
    c.sync();
}
static_assert(kMassBins == 2 * kThreads && kCoarse == 64 && kFine == 16, "add_masses and find_bin share the bins out");

// One warp: the lowest key of the row whose bin is at most b (bins fall as keys rise; that of `key`, the largest, is 0).
__device__ uint32_t lowest_key_of_bin(uint32_t b, uint32_t key, float top, float inv_t) {
    auto bin_at = [&](uint32_t k) { return bin_of(scaled(key_value(k), top, inv_t)); };
    uint32_t lo = kKeyNegInf, hi = key;                      // bin(lo) > b >= bin(hi)
    // the bound lies where the formula puts it, give or take its rounding
    const float at = top - ((float)b + 0.875f) / (kBinsPerUnit * inv_t), slack = (fabsf(at) + fabsf(top)) * 4e-6f;
    const uint32_t below = order_key(at - slack), above = order_key(at + slack);
    if (below > lo && below < hi && bin_at(below) > b) lo = below;
    if (above > lo && above < hi && bin_at(above) <= b) hi = above;
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 31) / 32;
        const uint64_t k = (uint64_t)lo + (uint64_t)step * ((threadIdx.x & 31) + 1);
        const bool in = k >= hi || bin_at((uint32_t)k) <= b;
        const int first = __ffs(__ballot_sync(kAllLanes, in)) - 1;          // the last lane is at hi or beyond
        hi = (uint32_t)min((uint64_t)hi, (uint64_t)lo + (uint64_t)step * (first + 1));
        lo = lo + step * first;
    }
    return hi;
}

// Where the running mass first exceeds `goal`: s.at gets the keys of that bin and the mass before it -- or, where all
// entries from the largest down to it are few enough for the list, the keys from that bin up (s.complete).
__device__ void find_bin(const Cluster& c, Shared& s, uint64_t goal, uint32_t key, float top, float inv_t, int V) {
    const int lane = threadIdx.x & 31;
    __syncthreads();
    if (threadIdx.x < 32) {
        uint64_t m[2] = {0, 0};
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
            if (r < c.ranks) { m[0] += s.coarse[r][2 * lane]; m[1] += s.coarse[r][2 * lane + 1]; }
        // at most so many entries: a bin's mass over its smallest weight
        float n[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            n[i] = (float)m[i] / fmaxf(1.0f, 2147483648.0f * fast_exp2(-kLog2e / kBinsPerUnit * ((2 * lane + i + 1) * kFine)));
        uint64_t before = m[0] + m[1];
        float entries = n[0] + n[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t um = __shfl_up_sync(kAllLanes, before, o);
            const float un = __shfl_up_sync(kAllLanes, entries, o);
            if (lane >= o) { before += um; entries += un; }
        }
        before -= m[0] + m[1];
        const int mine = before <= goal && goal < before + m[0] ? 0 : before + m[0] <= goal && goal < before + m[0] + m[1] ? 1 : 2;
        const unsigned who = __ballot_sync(kAllLanes, mine < 2);
        if (who) {
            const int from = __ffs(who) - 1;
            const int half = __shfl_sync(kAllLanes, mine, from);
            uint64_t run = __shfl_sync(kAllLanes, before, from) + (half ? __shfl_sync(kAllLanes, m[0], from) : 0);
            const float upto = __shfl_sync(kAllLanes, entries, from);
            const int first = (2 * from + half) * kFine;
            // the CTAs' fine bins, all asked for at once: a half-warp has half the CTAs
            uint32_t low[kMaxCluster / 2], high[kMaxCluster / 2];
#pragma unroll
            for (int k = 0; k < kMaxCluster / 2; ++k) {
                const int r = (lane / kFine) * (kMaxCluster / 2) + k;
                low[k] = high[k] = 0;
                if (r < c.ranks) {
                    const Shared* p = c.peer(s, r);
                    low[k] = p->mass.low[first + lane % kFine];
                    high[k] = p->mass.high[first + lane % kFine];
                }
            }
            uint64_t fine = 0;
#pragma unroll
            for (int k = 0; k < kMaxCluster / 2; ++k) fine += (uint64_t)low[k] + ((uint64_t)high[k] << 32);
            fine += __shfl_xor_sync(kAllLanes, fine, kFine);
            if (lane >= kFine) fine = 0;
            uint64_t sum = fine;
#pragma unroll
            for (int o = 1; o < kFine; o <<= 1) {
                const uint64_t up = __shfl_up_sync(kAllLanes, sum, o);
                if (lane >= o) sum += up;
            }
            run += sum - fine;
            const unsigned hit = __ballot_sync(kAllLanes, lane < kFine && run <= goal && goal < run + fine);
            const int at = hit ? __ffs(hit) - 1 : 0;
            run = __shfl_sync(kAllLanes, run, at);
            const uint32_t b = first + at;
            const bool complete = upto <= kListCap - 64;
            Interval next;
            next.lo = lowest_key_of_bin(b, key, top, inv_t);
            next.hi = complete || b == 0 ? kHighestKey : lowest_key_of_bin(b - 1, key, top, inv_t) - 1;
            next.first = 0; next.last = V - 1;
            next.count_before = 0;
            next.mass_before = complete ? 0 : run;
            if (lane == 0) { s.at = next; s.complete = complete; }
        }
    }
    __syncthreads();
}

// ---- the kernels --------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kThreads, 2) top_rows_kernel(const TopArgs a) {
    Shared& s = shared();
    const Cluster c;
    if (c.ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x / c.ranks;
    if (tid == 0) s.filled = 0;
    report_to(s, a.status);
    const Slice<T> slice(static_cast<const T*>(a.logits) + r * a.row_stride, a.V, __ffs(c.ranks) - 1, c.rank);
    const float scale = a.inv_t * kLog2e;
    const Streamed st = stream_slice(slice, a.lse != nullptr, scale, s);
    const RowPart row = exchange_parts(c, s, st, scale, a.K);

    int n = 0;
    if (row.key >= kLowestKey) {
        n = (int)push_entries(c, slice, st, row.bound, kHighestKey, 0, a.V - 1, 0);
        if (n > kListCap) {                                  // ties: find the K-th entry, list what comes up to it
            if (tid == 0) s.at = {row.bound, row.key, 0, a.V - 1, 0, 0};
            __syncthreads();
            search<T>(c, slice, st, false, (uint64_t)a.K - 1, row.top, a.inv_t, 1);
            const uint32_t key = place_key(s.found_place);
            const int id = place_id(s.found_place);
            n = (int)push_entries(c, slice, st, key + 1, kHighestKey, 0, a.V - 1, 0);
            n = min(kListCap, n + (int)push_entries(c, slice, st, key, key, 0, id, 1));
        }
    }
    if (c.rank != 0) return;
    if (a.lse && tid >= kThreads - 32) {                     // a warp that has least to do with a short list
        const float ln_sum = log_row_sum(c, s, row, scale);
        if (tid == kThreads - 1) a.lse[r] = (float)((double)row.top * a.inv_t64 + (double)ln_sum);
    }
    if (n > 0) sort_list(n);
    int32_t* ids = a.ids + r * a.K;
    float* values = a.values + r * a.K;
    for (int j = tid; j < a.K; j += kThreads) {
        const uint64_t p = j < n ? s.list[j] : 0;
        if (j < n && !SPECS_IN_BOUNDS(place_id(p), a.V, a.status)) continue;
        ids[j] = j < n ? place_id(p) : -1;
        values[j] = j < n ? key_value(place_key(p)) : -INFINITY;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_rows_kernel(const SampleArgs a) {
    Shared& s = shared();
    const Cluster c;
    if (c.ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int tid = threadIdx.x;
    const int64_t r = blockIdx.x / c.ranks;
    if (tid == 0) { s.filled = 0; s.found_place = 0; s.found_before = 0; }
    report_to(s, a.status);

    // the row's settings
    const float temp = a.temperature ? a.temperature[r] : 1.0f;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f;
    const float u = fminf(fmaxf(a.uniforms[r], 0.0f), 1.0f - 5.9604645e-8f);
    float inv_t = 1.0f / temp;
    int k = a.top_k ? a.top_k[r] : 0;
    if (k >= a.V) k = 0;
    if (!(temp > 0.0f) || inv_t == INFINITY) { inv_t = 1.0f; k = 1; }
    const float low = min_p > 0.0f ? logf(fminf(min_p, 1.0f)) : -INFINITY;

    const Slice<T> slice(static_cast<const T*>(a.logits) + r * a.row_stride, a.V, __ffs(c.ranks) - 1, c.rank);
    const Streamed st = stream_slice(slice, a.tok_logprob != nullptr, kLog2e, s);
    const uint32_t want = k > 1 && k <= kMaxTopLogits ? k : 0;
    const RowPart row = exchange_parts(c, s, st, kLog2e, want);
    const float top = row.top;
    if (top == INFINITY) k = 1;                              // takes everything
    const Interval everything = {kLowestKey, row.key, 0, a.V - 1, 0, 0};

    uint64_t kept = 0;                                       // 0: the draw was certain
    bool drawn = row.key < kLowestKey;                       // nothing to draw from: the place found stays 0
    if (!drawn && k == 1) {
        const int n = (int)push_entries(c, slice, st, row.key, row.key, 0, a.V - 1, 0);
        if (n <= kListCap) {
            if (c.rank != 0) return;
            sort_list(n);
            if (tid == 0) s.found_place = s.list[0];
            __syncthreads();
        } else {
            if (tid == 0) { s.at = everything; s.at.lo = row.key; }
            __syncthreads();
            search<T>(c, slice, st, false, 0, top, inv_t, 1);
        }
        drawn = true;
    } else if (!drawn && want > 0) {
        const int n = (int)push_entries(c, slice, st, row.bound, kHighestKey, 0, a.V - 1, 0);
        if (n <= kListCap) {
            if (c.rank != 0) return;
            sort_list(n);
            const Running list = run_list(s, min(n, k), top, inv_t);
            kept = list.total;
            if (top_p < 1.0f) {
                find_in(s, list, nucleus_goal(kept, top_p));
                kept = min(kept, mass_upto(s, top, inv_t));
            }
            if (min_p > 0.0f) {
                uint64_t allowed = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (list.w[i] && scaled(key_value(place_key(list.place[i])), top, inv_t) >= low) allowed += list.w[i];
                kept = min(kept, block_sum(allowed, s.red64));
            }
            __syncthreads();
            find_in(s, list, draw_goal(kept, u));
            drawn = true;
        } else if (tid == 0) {                               // more ties at the bound than the list holds: given up
            s.filled = 0;
        }
    }
    if (!drawn && a.V <= kListCap) {                         // a short row is a list as it is
        const int n = (int)push_entries(c, slice, st, kLowestKey, kHighestKey, 0, a.V - 1, 2);
        if (c.rank != 0) return;
        weigh_list(s, n, top, inv_t);
        uint64_t sum = 0, allowed = 0;
        for (int i = tid; i < n; i += kThreads) {            // (a thread's own weights)
            sum += s.weight[i];
            if (scaled(key_value(place_key(s.list[i])), top, inv_t) >= low) allowed += s.weight[i];
        }
        kept = block_sum(sum, s.red64);
        __syncthreads();
        allowed = block_sum(allowed, s.red64);
        if (k > 0 && k < n) {
            narrow_list(n, false, (uint64_t)k - 1);
            kept = mass_upto(s, top, inv_t);
        }
        if (top_p < 1.0f) {
            narrow_list(n, true, nucleus_goal(kept, top_p));
            kept = min(kept, mass_upto(s, top, inv_t));
        }
        kept = min(kept, allowed);
        narrow_list(n, true, draw_goal(kept, u));
        drawn = true;
    }
    if (!drawn) {
        add_masses(c, s, slice, top, inv_t, low, min_p > 0.0f, k > 0);
        uint64_t allowed = 0;
        uint32_t weighted = 0;
        for (int i = 0; i < c.ranks; ++i) { allowed += s.rest[i].allowed; weighted += s.rest[i].weighted; }
        if (tid < 32) {
            uint64_t m = 0;
            for (int i = tid; i < c.ranks * kCoarse; i += 32) m += s.coarse[0][i];
            m = warp_reduce(m, AddOp());
            if (tid == 0) s.total = m;
        }
        __syncthreads();
        kept = s.total;
        int round = 2;
        if (k > 0 && (uint32_t)k < weighted) {
            if (tid == 0) s.at = everything;
            __syncthreads();
            search<T>(c, slice, st, false, (uint64_t)k - 1, top, inv_t, round++);
            kept = mass_upto(s, top, inv_t);
        }
        // the nucleus first, then the draw: the same search for another mass
        bool alone = false;                                  // the first CTA has it all in its list
        int listed = 0;
        for (int step = top_p < 1.0f ? 0 : 1; step < 2; ++step) {
            if (step == 1 && min_p > 0.0f) kept = min(kept, allowed);
            const uint64_t goal = step == 0 ? nucleus_goal(kept, top_p) : draw_goal(kept, u);
            if (alone) {
                narrow_list(listed, true, goal);
                continue;
            }
            find_bin(c, s, goal, row.key, top, inv_t, a.V);
            const Interval at = s.at;
            const bool complete = s.complete != 0;
            const int n = (int)push_entries(c, slice, st, at.lo, at.hi, 0, a.V - 1, round++);
            if (n > kListCap) {                              // many entries of the same size: narrow the bin down
                search<T>(c, slice, st, true, goal, top, inv_t, round++);
            } else if (complete || step == 1) {
                if (c.rank != 0) return;
                alone = true;
                listed = n;
                weigh_list(s, n, top, inv_t);
                narrow_list(n, true, goal - at.mass_before);
            } else {
                if (c.rank == 0) {
                    weigh_list(s, n, top, inv_t);
                    narrow_list(n, true, goal - at.mass_before);
                    if (tid < c.ranks) {
                        const uint64_t place = s.found_place, before = s.found_before + at.mass_before;
                        __syncwarp((1u << c.ranks) - 1);
                        c.peer(s, tid)->found_place = place;
                        c.peer(s, tid)->found_before = before;
                    }
                    if (tid == 0) s.filled = 0;
                }
                c.sync();
            }
            if (step == 0) kept = min(kept, mass_upto(s, top, inv_t));
        }
    }
    if (c.rank == 0 && tid < 32) {
        const float nan = __int_as_float(0x7fc00000);
        const uint64_t place = s.found_place;
        const float l = place ? key_value(place_key(place)) : nan;
        const float ln_sum = log_row_sum(c, s, row, kLog2e);
        if (tid == 0) {
            a.tokens[r] = place && SPECS_IN_BOUNDS(place_id(place), a.V, a.status) ? place_id(place) : -1;
            if (a.tok_logprob) a.tok_logprob[r] = (l - top) - ln_sum;
            if (a.draw_logprob)
                a.draw_logprob[r] = !place ? nan : kept == 0 ? 0.0f
                                  : (l - top) * inv_t - logf((float)((double)kept * (1.0 / 2147483648.0)));
        }
    }
}

// CTAs of a row: as many as the device holds at once (two on an SM), but none without 1024 units, two a thread.  Measured, 32768
// bf16, nothing cut off / nucleus / top-k (us): 111 rows on 222 CTAs 26 / 36 / 15, on 444 37 / 54 / 24; 256 rows on 256 CTAs
// 34 / 45 / 16, on 512 45 / 64 / 26; 60 rows of 151936 on 240 38 / 51 / 18, on 480 50 / 74 / 27.  With 256 or 512 units a CTA
// the exchanges cost more than the shorter passes save (37 x 32003 fp16, nucleus: 35 us instead of 26).
// Rows of 16000 units and more get two CTAs as long as there are no more than 3/2 of them an SM: with one each, half of the SMs or
// more would have a single CTA, and a long row takes long.  Measured with one / two (us, nothing cut off, nucleus, top-k, min-p,
// and the four of them mixed): 128256 bf16, 210 rows 88 119 34 73 88 / 80 109 42 73 65, 230 rows 86 116 35 73 88 / 89 114 42 86 73;
// 151936 bf16, 170 rows 100 137 37 85 88 / 88 115 40 81 68, 256 rows 105 143 40 87 103 / 105 135 48 99 89; 65536 bf16, 170 rows
// 47 62 24 44 44 / 51 67 30 48 40.
int cluster_size(int64_t rows, int units, int num_sms) {
    int ranks = 1;
    while (ranks < kMaxCluster && units > ranks * kLeastUnits && rows * 2 * ranks <= 2 * num_sms) ranks *= 2;
    return ranks == 1 && units >= kLongUnits && 2 * rows <= 3 * num_sms ? 2 : ranks;
}

template <typename Args>
int launch(void (*kernel)(const Args), const Args& args, int ranks, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(args.rows * ranks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Shared);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, args));
}

}  // namespace

bool prepare_pick_rows() {
    const void* kernels[] = {(const void*)top_rows_kernel<float>, (const void*)top_rows_kernel<__nv_bfloat16>,
                             (const void*)top_rows_kernel<__half>, (const void*)sample_rows_kernel<float>,
                             (const void*)sample_rows_kernel<__nv_bfloat16>, (const void*)sample_rows_kernel<__half>};
    for (const void* k : kernels)
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) != cudaSuccess) return false;
    return true;
}

int launch_sample_rows(const SampleArgs& a, int dtype, cudaStream_t stream) {
    const int ranks = cluster_size(a.rows, a.V / (dtype == SPECS_F32 ? 4 : 8), a.num_sms);
    return launch(dtype == SPECS_F32 ? sample_rows_kernel<float>
                  : dtype == SPECS_BF16 ? sample_rows_kernel<__nv_bfloat16> : sample_rows_kernel<__half>, a, ranks, stream);
}

// Many rows stream through one persistent CTA per SM (top_stream.cu) as soon as there are more of them than SMs, if they have as
// many units as that kernel has half its groups, and lists that half of those can bound.  Measured, 16384 and 131072 bf16 (us,
// clusters / streamed): 148 rows K = 64 13 / 12 and 17 / 17, 200 rows 19 / 12 and 25 / 24, 1184 rows 38 / 27 and 85 / 65,
// with K = 512 99 / 56 and 162 / 104; against it 296 rows, which clusters take in one wave: 12 / 13 and 23 / 25.  8192 entries
// are too few for K = 512: 48 / 244, most rows there being listed as ties.
int launch_top_rows(const TopArgs& a, int dtype, cudaStream_t stream) {
    if (a.rows > a.num_sms && a.V / (dtype == SPECS_F32 ? 4 : 8) >= kStreamUnits && a.K <= kStreamTop)
        return launch_top_stream(a, dtype, stream);
    const int ranks = cluster_size(a.rows, a.V / (dtype == SPECS_F32 ? 4 : 8), a.num_sms);
    return launch(dtype == SPECS_F32 ? top_rows_kernel<float>
                  : dtype == SPECS_BF16 ? top_rows_kernel<__nv_bfloat16> : top_rows_kernel<__half>, a, ranks, stream);
}

}  // namespace specs
