// The K largest logits of many rows, and their log-sum-exps: one persistent CTA per SM.
//
// Each CTA takes whole rows, one after the other.  One thread fills a ring of 32 KB stages with bulk copies and runs ahead
// of everyone.  16 warps take the stages: they keep the largest logit of each of 4096 groups of a row's units and the sums of
// exponentials, and hand these over.  Three teams of four warps pick, a row each: the K-th largest of the groups' largest
// bounds the K-th largest logit from below; the groups that reach it are read again (from L2), and the entries at or above
// it, not many more than K, are ranked by counting.  So nobody who streams waits for a pick, and HBM stays busy.
//
// Bound: HBM and the exponentials beside it.  1024 x 151936 bf16, K = 64: 70 us, 4.5 TB/s (56 us without the log-sum-exp, which
// takes an exponential per entry; clusters that stream and pick in turn: 87 us).  fp32 rows of as many bytes: 59 us, 5.3 TB/s.
// A pick takes 4 us for K = 64 and 18 us for K = 400, most of it the groups read again while HBM is busy; three teams have
// three rows' time for it.
#include <cstddef>

#include "bulk_ring.cuh"
#include "row_picks.cuh"

namespace specs {
namespace {

constexpr int kSharedPerBlock = 232448;                    // 227 KB
constexpr int kTakers = 512, kTakeWarps = kTakers / 32, kTake = kStageUnits / kTakers;
constexpr int kTeams = 3, kTeam = 128, kTeamWarps = kTeam / 32;
constexpr int kStreamBlock = kTakers + kTeams * kTeam + 32;   // and the filling warp
// Groups: a taking thread has two pairs of neighbouring units (32 bytes, what memory is read by) of a stage, and two groups for
// every quarter of a row's stages.
constexpr int kTurns = 4, kRuns = 2 * kTurns, kGroups = kRuns * kTakers, kHalf = kStageUnits / 2;
constexpr int kRingMax = 4;                                // a deeper ring only makes what the teams read wait longer
constexpr int kListCap = 1024;
constexpr int kOwn = 4;                                    // units a thread reads again at a time
constexpr int kBins = 64, kMaxLevels = 12;                 // ties: 32 bits of a key and 19 of an id, 6 a level, take 10 at most
static_assert(kTake == 4 && kTakers == 4 * kTeam, "pairs, and four places of each run a thread of a team");
static_assert(kTeam == 128 && kGroups == 32 * kTeam, "a bin a thread, and a bit for each of its groups");
static_assert(kListCap >= 2 * kStreamTop && kStreamUnits >= kStageUnits, "a list has room for K entries and as many beyond");

// What a team has of its row.
struct alignas(16) Slot {                                  // read 16 bytes at a time
    union {
        uint32_t group_key[kGroups];                       // by the taking warps
        uint16_t flags[kGroups];                           // ... then the groups to read again
        uint32_t bins[kBins][32];                          // ties: one column per lane
        uint64_t binned[kListCap];                         // the list by bins of its keys
    };
    uint64_t list[kListCap];
    float top[kTakeWarps], sum[kTakeWarps];
    uint32_t total[kTeam], warp_total[kTeamWarps];
    uint32_t reached[2][kTeamWarps];                       // while the bound is searched
    uint32_t bound, key, filled, flagged, go;
};
struct StreamShared {
    Ring ring;
    uint64_t taken[kTeams], free[kTeams];
    Slot slot[kTeams];
    uint32_t abort;
};
static_assert(sizeof(Slot) % 16 == 0 && offsetof(Slot, list) % 16 == 0 && offsetof(StreamShared, slot) % 16 == 0, "16-byte loads");

__device__ __forceinline__ int stages_of_turn(int count) { return (count + kTurns * kStageUnits - 1) / (kTurns * kStageUnits); }

__device__ __forceinline__ void team_meets(int team) {
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(kTeam) : "memory");
}

__device__ __forceinline__ void push(Slot& slot, uint64_t place) {
    const uint32_t at = atomicAdd(&slot.filled, 1u);
    if (at < kListCap) slot.list[at] = place;
}

// Room for n of each lane in a list: where the lane's begin.  One atomic for the warp.
__device__ __forceinline__ uint32_t warp_room(uint32_t& filled, uint32_t n) {
    const int lane = threadIdx.x & 31;
    uint32_t upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(kAllLanes, upto, o);
        if (lane >= o) upto += up;
    }
    uint32_t begin = 0;
    if (lane == 31 && upto) begin = atomicAdd(&filled, upto);
    return __shfl_sync(kAllLanes, begin, 31) + upto - n;
}

// Ties at the bound: the interval of keys from `bound` to the row's largest, then of ids, is narrowed by counting in 64 bins a
// level until the entries up to its end fit the list.  Rare, and as long as a few passes over the row by four warps.
template <typename T>
__device__ __noinline__ void list_ties(const TopArgs& a, int64_t r, Slot& slot, int team) {
    const int t = (threadIdx.x - kTakers) % kTeam, lane = t & 31, warp = t >> 5;
    const RowUnits<T> row(static_cast<const T*>(a.logits) + r * a.row_stride, a.V);
    uint32_t lo = slot.bound, hi = slot.key, before = 0;
    int first = 0, last = a.V - 1;
    for (int level = 0; level < kMaxLevels; ++level) {
        const bool by_key = lo < hi;
        const uint32_t range = by_key ? hi - lo : (uint32_t)(last - first);
        const int shift = max(0, 32 - __clz(range) - 6);   // range >> shift < 64
        team_meets(team);
        for (int i = t; i < kBins * 32; i += kTeam) (&slot.bins[0][0])[i] = 0;
        team_meets(team);
        for (int u = t; u < row.units; u += kTeam) {
            float f[Elem<T>::kWidth];
            Elem<T>::widen(row.load(u), f);
#pragma unroll
            for (int e = 0; e < Elem<T>::kWidth; ++e) {
                const uint32_t key = order_key(f[e]);
                const int id = row.first(u) + e;
                if (key >= lo && key <= hi && id >= first && id <= last)
                    atomicAdd(&slot.bins[(by_key ? hi - key : (uint32_t)(id - first)) >> shift][lane], 1u);
            }
        }
        team_meets(team);
        for (int b = warp; b < kBins; b += kTeamWarps) {
            const uint32_t n = __reduce_add_sync(kAllLanes, slot.bins[b][lane]);
            if (lane == 0) slot.total[b] = n;
        }
        team_meets(team);
        uint32_t d = 0, n = 0;
        for (; d < kBins; ++d) {                           // the bin that holds the K-th entry
            n = slot.total[d];
            if (before + n >= (uint32_t)a.K) break;
            before += n;
        }
        if (d == kBins) break;                             // fewer than K in all: the caller's arithmetic rules that out
        if (by_key) {
            hi -= d << shift;
            lo = hi - min(hi - lo, (1u << shift) - 1);
        } else {
            first += (int)(d << shift);
            last = min(last, first + (int)((1u << shift) - 1));
        }
        if (before + n <= kListCap) break;
    }
    team_meets(team);
    if (t == 0) slot.filled = 0;
    team_meets(team);
    const uint64_t least = place_of(lo, last);
    for (int u = t; u < row.units; u += kTeam) {
        float f[Elem<T>::kWidth];
        Elem<T>::widen(row.load(u), f);
#pragma unroll
        for (int e = 0; e < Elem<T>::kWidth; ++e) {
            const uint64_t place = place_of(order_key(f[e]), row.first(u) + e);
            if (place >= least) push(slot, place);
        }
    }
    team_meets(team);
}

// The row's log-sum-exp, by one warp: 16 parts, and the elements of partial units.
template <typename T>
__device__ __forceinline__ void sum_row(const TopArgs& a, int64_t r, const StreamRow<T>& row, const Slot& slot, float scale) {
    const int lane = threadIdx.x & 31;
    float top = -INFINITY, sum = 0.0f;
    if (lane < kTakeWarps) {
        top = slot.top[lane];
        sum = slot.sum[lane];
    } else {
        const int v = row.edge_element(lane - kTakeWarps);
        if (v >= 0) {                                      // an entry by itself: its sum is 1 (NaN for NaN and inf, 0 for -inf)
            const float logit = Elem<T>::to_float(row.row.row[v]);
            top = fmaxf(logit, -INFINITY);
            sum = logit == -INFINITY ? 0.0f : 1.0f + (logit - logit);
        }
    }
    const float most = warp_reduce(top, MaxOp());
    sum = warp_reduce(sum * (top == -INFINITY || top == most ? 1.0f : fast_exp2((top - most) * scale)), AddOp());
    if (lane == 0) a.lse[r] = (float)((double)most * a.inv_t64 + (double)logf(sum));
}

// The team: a key that at least K groups reach, and not many more.  The largest of a thread's groups will do for as many as 5/8
// of the threads: that many reach a bound that about as many entries again as are wanted reach at most.  For more, two groups
// are taken as one.
__device__ __forceinline__ uint32_t team_bound(Slot& slot, int K, int team) {
    const int t = (threadIdx.x - kTakers) % kTeam, lane = t & 31, warp = t >> 5;
    const bool many = K > kTakers / 8 * 5;
    uint4 k[kTurns];
    auto larger = [](const uint4& a, const uint4& b) {
        return make_uint4(max(a.x, b.x), max(a.y, b.y), max(a.z, b.z), max(a.w, b.w));
    };
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const uint4* keys = reinterpret_cast<const uint4*>(slot.group_key) + t;
        k[i] = larger(keys[i * kTeam], keys[(i + kTurns) * kTeam]);
    }
    if (!many) {
        k[0] = larger(larger(k[0], k[1]), larger(k[2], k[3]));
#pragma unroll
        for (int i = 1; i < kTurns; ++i) k[i] = make_uint4(0, 0, 0, 0);
    }
    int round = 0;
    auto gather = [&](uint32_t v) {                        // the warps' values, in four lanes each
        if (lane == 0) slot.reached[round][warp] = v;
        team_meets(team);
        v = slot.reached[round][lane % kTeamWarps];
        round ^= 1;
        return v;
    };
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) most = max(max(most, max(k[i].x, k[i].y)), max(k[i].z, k[i].w));
    most = __reduce_max_sync(kAllLanes, gather(__reduce_max_sync(kAllLanes, most)));
    if (t == 0) slot.key = most;
    return search_bound((uint32_t)K, most, [&](uint32_t key) {
        uint32_t n = (k[0].x >= key) + (k[0].y >= key) + (k[0].z >= key) + (k[0].w >= key);
        if (many)
#pragma unroll
            for (int i = 1; i < kTurns; ++i) n += (k[i].x >= key) + (k[i].y >= key) + (k[i].z >= key) + (k[i].w >= key);
        const uint32_t all = gather(__reduce_add_sync(kAllLanes, n));
        return __reduce_add_sync(kAllLanes, lane < kTeamWarps ? all : 0u);
    });
}

// The team's list in order, to the output.  The keys from the bound up fall into 128 bins; an entry's rank is the number of entries
// in higher bins and of larger ones in its own.
__device__ __forceinline__ void rank_list(const TopArgs& a, int64_t r, Slot& slot, int team) {
    const int t = (threadIdx.x - kTakers) % kTeam, lane = t & 31, warp = t >> 5;
    const int n = (int)slot.filled;
    const uint32_t least = slot.bound, range = slot.key - least;
    const int shift = max(0, 32 - __clz(range) - 7);       // range >> shift < kTeam
    uint32_t* end = slot.total;
    end[t] = 0;
    team_meets(team);
    for (int i = t; i < n; i += kTeam) atomicAdd(&end[kTeam - 1 - ((place_key(slot.list[i]) - least) >> shift)], 1u);
    team_meets(team);
    uint32_t before = end[t];                              // of the bins up to this one, the highest keys first
    const uint32_t mine = before;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(kAllLanes, before, o);
        if (lane >= o) before += up;
    }
    if (lane == 31) slot.warp_total[warp] = before;
    team_meets(team);
    for (int w = 0; w < warp; ++w) before += slot.warp_total[w];
    end[t] = before - mine;                                // the bin's first place, and its end when all are in
    team_meets(team);
    for (int i = t; i < n; i += kTeam) {
        const uint64_t place = slot.list[i];
        slot.binned[atomicAdd(&end[kTeam - 1 - ((place_key(place) - least) >> shift)], 1u)] = place;
    }
    team_meets(team);
    int32_t* ids = a.ids + r * a.K;
    float* values = a.values + r * a.K;
    for (int i = t; i < n; i += kTeam) {
        const uint64_t place = slot.binned[i];
        const uint32_t bin = kTeam - 1 - ((place_key(place) - least) >> shift);
        const int last = (int)end[bin];
        int rank = bin > 0 ? (int)end[bin - 1] : 0;
        for (int k = rank; k < last && rank < a.K; ++k) rank += slot.binned[k] > place;
        if (rank < a.K && SPECS_IN_BOUNDS(place_id(place), a.V, a.status)) {
            ids[rank] = place_id(place);
            values[rank] = key_value(place_key(place));
        }
    }
    for (int j = n + t; j < a.K; j += kTeam) { ids[j] = -1; values[j] = -INFINITY; }
}

template <typename T>
__device__ void pick_row(const TopArgs& a, int64_t r, Slot& slot, int team, float scale) {
    const int t = (threadIdx.x - kTakers) % kTeam, lane = t & 31, warp = t >> 5;
    const StreamRow<T> row(static_cast<const T*>(a.logits) + r * a.row_stride, a.V);
    if (t == 0) slot.filled = slot.flagged = 0;
    const uint32_t bound = team_bound(slot, a.K, team);
    if (t == 0) slot.bound = bound;
    uint32_t in[kGroups / kTeam / 4];
#pragma unroll
    for (int i = 0; i < kGroups / kTeam / 4; ++i) {
        const uint4 k = reinterpret_cast<const uint4*>(slot.group_key)[i * kTeam + t];
        in[i] = (k.x >= bound) | (k.y >= bound) << 1 | (k.z >= bound) << 2 | (k.w >= bound) << 3;
    }
    uint32_t own = 0;
#pragma unroll
    for (int i = 0; i < kGroups / kTeam / 4; ++i) own |= in[i] << (4 * i);
    const uint32_t at_flags = warp_room(slot.flagged, __popc(own));
    team_meets(team);                                      // the flags go where the keys were
    for (uint32_t m = own, pos = at_flags; m; m &= m - 1, ++pos) {
        const int bit = __ffs(m) - 1;
        if (SPECS_IN_BOUNDS(pos, kGroups, a.status)) slot.flags[pos] = (uint16_t)((bit / 4 * kTeam + t) * 4 + bit % 4);
    }
    const int edge = t < 16 ? row.edge_element(t) : -1;
    if (edge >= 0) {
        const uint32_t key = order_key(Elem<T>::to_float(row.row.row[edge]));
        if (key >= bound) push(slot, place_of(key, edge));
        atomicMax(&slot.key, key);
    }
    team_meets(team);
    const int per_turn = stages_of_turn(row.count), per = 2 * per_turn, work = (int)slot.flagged * per;   // units of a group, at most
    const uint4* units = reinterpret_cast<const uint4*>(row.from());
    const int first = row.row.first(row.begin);
    const float least = key_value(bound);
    for (int w = t; w - lane < work; w += kOwn * kTeam) {  // kOwn loads at a time, whole warps
        uint4 q[kOwn];
        int at[kOwn];
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int x = w + j * kTeam;
            const uint32_t ninf = Elem<T>::kNegInfWord;
            q[j] = make_uint4(ninf, ninf, ninf, ninf);
            const int g = x < work ? slot.flags[x / per] : 0, n = x % per;
            at[j] = ((n >> 1) + g / (2 * kTakers) * per_turn) * kStageUnits + g / kTakers % 2 * kHalf + g % kTakers * 2 + (n & 1);
            if (x >= work) at[j] = row.count;
            if (at[j] < row.count && SPECS_IN_BOUNDS(at[j], row.count, a.status)) q[j] = units[at[j]];
        }
        // a lane's hits, a bit each
        constexpr int kWidth = Elem<T>::kWidth;
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            float f[kWidth];
            Elem<T>::widen(q[j], f);
#pragma unroll
            for (int e = 0; e < kWidth; ++e) hits |= (f[e] >= least ? 1u : 0u) << (j * kWidth + e);
        }
        __syncwarp();
        uint32_t pos = warp_room(slot.filled, __popc(hits));
        for (; hits; hits &= hits - 1, ++pos) {
            const int bit = __ffs(hits) - 1, j = bit / kWidth, e = bit % kWidth;
            const uint4 v = j == 0 ? q[0] : j == 1 ? q[1] : j == 2 ? q[2] : q[3];
            const int u = j == 0 ? at[0] : j == 1 ? at[1] : j == 2 ? at[2] : at[3];
            if (pos < kListCap) slot.list[pos] = place_of(order_key(unit_element<T>(v, e)), first + u * kWidth + e);
        }
    }
    team_meets(team);
    if (slot.filled > kListCap) list_ties<T>(a, r, slot, team);
    rank_list(a, r, slot, team);
    if (a.lse && warp == kTeamWarps - 1) sum_row(a, r, row, slot, scale);
}

template <typename T>
__device__ __forceinline__ bool take_row(StreamShared& s, const uint8_t* stages, int stage_count, RingPlace& at,
                                         const StreamRow<T>& row, bool want_sum, const BoundedWait& wait, GroupMaxima<T, kRuns>& out) {
    const int per_turn = stages_of_turn(row.count);
    int turn = 0, left = per_turn;
    float2 now = make_float2(-INFINITY, -INFINITY);
    for (int base = 0; base < row.count; base += kStageUnits) {
        if (!wait(&s.ring.full[at.stage], at.phase)) return false;
        const uint4* in = reinterpret_cast<const uint4*>(stages + (size_t)at.stage * kStageBytes);
        // neighbouring threads swap their pairs' units by fours: no two of eight in the same banks
        const int own = 2 * threadIdx.x, swap = (threadIdx.x >> 2) & 1;
        const uint32_t ninf = Elem<T>::kNegInfWord;
        uint4 q[kTake];
        if (base + kStageUnits <= row.count) {
#pragma unroll
            for (int j = 0; j < kTake; ++j) q[j] = in[j / 2 * kHalf + own + ((j & 1) ^ swap)];
        } else {
#pragma unroll
            for (int j = 0; j < kTake; ++j) {
                const int k = j / 2 * kHalf + own + ((j & 1) ^ swap);
                q[j] = base + k < row.count ? in[k] : make_uint4(ninf, ninf, ninf, ninf);
            }
        }
        ring_release(s.ring, at, stage_count);
        out.add_pairs(q, now, want_sum);
        if (--left == 0 || base + kStageUnits >= row.count) {
            out.set_pair(turn++, now);
            now = make_float2(-INFINITY, -INFINITY);
            left = per_turn;
        }
    }
    return true;
}

template <typename T>
__global__ void __launch_bounds__(kStreamBlock, 1) top_stream_kernel(const TopArgs a, int stage_count) {
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* stages = smem;
    StreamShared& s = *reinterpret_cast<StreamShared*>(smem + (size_t)stage_count * kStageBytes);
    const float scale = a.inv_t * kLog2e;
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        ring_init(s.ring, stage_count, kTakeWarps);
        for (int i = 0; i < kTeams; ++i) { barrier_init(&s.taken[i], kTakeWarps); barrier_init(&s.free[i], 1); }
        s.abort = 0;
        barriers_ready();
    }
    __syncthreads();
    const BoundedWait wait = {&s.abort, a.status};
    const T* logits = static_cast<const T*>(a.logits);

    if (threadIdx.x >= kTakers + kTeams * kTeam) {         // ---- the filling thread
        if (lane != 0) return;
        RingPlace at;
        bool fine = true;
        for (int64_t r = blockIdx.x; r < a.rows && fine; r += gridDim.x) {
            const StreamRow<T> row(logits + r * a.row_stride, a.V);
            const T* from = row.from();
            for (int base = 0; base < row.count && fine; base += kStageUnits)
                fine = ring_fill(s.ring, at, stage_count, stages, from + (size_t)base * Elem<T>::kWidth,
                                 min(kStageUnits, row.count - base), wait);
        }
        ring_drain(s.ring, at, stage_count, wait);
    } else if (threadIdx.x < kTakers) {                    // ---- the taking warps
        const int warp = threadIdx.x >> 5;
        RingPlace at;
        int team = 0;
        uint32_t phase = 0;
        for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
            const StreamRow<T> row(logits + r * a.row_stride, a.V);
            GroupMaxima<T, kRuns> best(scale);
            if (!take_row(s, stages, stage_count, at, row, a.lse != nullptr, wait, best)) return;
            if (!wait(&s.free[team], phase ^ 1u)) return;
            Slot& slot = s.slot[team];
            uint32_t key[kRuns];
            __syncwarp();
            best.of_warp(a.lse != nullptr, key, slot.top[warp], slot.sum[warp]);
#pragma unroll
            for (int j = 0; j < kRuns; ++j) slot.group_key[j * kTakers + threadIdx.x] = key[j];
            __syncwarp();
            if (lane == 0) barrier_arrive(&s.taken[team]);
            if (++team == kTeams) { team = 0; phase ^= 1u; }
        }
    } else {                                               // ---- the teams
        const int team = (threadIdx.x - kTakers) / kTeam, t = (threadIdx.x - kTakers) % kTeam;
        Slot& slot = s.slot[team];
        uint32_t phase = 0;
        for (int64_t r = blockIdx.x + (int64_t)team * gridDim.x; r < a.rows; r += (int64_t)kTeams * gridDim.x, phase ^= 1u) {
            if (t < 32) {                                  // one warp waits, and tells the others how that went
                const bool fine = __all_sync(kAllLanes, wait(&s.taken[team], phase));
                if (t == 0) slot.go = fine;
            }
            team_meets(team);
            if (!slot.go) return;
            pick_row<T>(a, r, slot, team, scale);
            team_meets(team);
            if (t == 0) barrier_arrive(&s.free[team]);
        }
    }
}

template <typename T>
int launch_stream(const TopArgs& a, cudaStream_t stream) {
    const int room = (kSharedPerBlock - (int)sizeof(StreamShared)) / kStageBytes, stages = room < kRingMax ? room : kRingMax;
    const int bytes = stages * kStageBytes + (int)sizeof(StreamShared);
    const int grid = a.rows < a.num_sms ? (int)a.rows : a.num_sms;
    top_stream_kernel<T><<<grid, kStreamBlock, bytes, stream>>>(a, stages);
    return cuda_status(cudaGetLastError());
}

}  // namespace

bool prepare_top_stream() {
    const void* kernels[] = {(const void*)top_stream_kernel<float>, (const void*)top_stream_kernel<__nv_bfloat16>,
                             (const void*)top_stream_kernel<__half>};
    for (const void* k : kernels)
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedPerBlock) != cudaSuccess) return false;
    return true;
}

int launch_top_stream(const TopArgs& a, int dtype, cudaStream_t stream) {
    return dtype == SPECS_F32 ? launch_stream<float>(a, stream)
         : dtype == SPECS_BF16 ? launch_stream<__nv_bfloat16>(a, stream) : launch_stream<__half>(a, stream);
}

}  // namespace specs
