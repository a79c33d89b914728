// What the kernels share that pick entries out of rows of vocabulary logits (sample_rows.cu, top_stream.cu): the order of
// a row's entries, the streaming pass with its groups' maxima, and the bound that these give.
#pragma once

#include "logit_rows.cuh"

namespace specs {

constexpr uint32_t kLowestKey = kKeyNegInf + 1;

// An entry's place in the order as one number: the larger comes first.
__device__ __forceinline__ uint64_t place_of(uint32_t key, int id) {
    return ((uint64_t)key << 32) | (uint64_t)(0xffffffffu - (uint32_t)id);
}
__device__ __forceinline__ int place_id(uint64_t place) { return (int)(0xffffffffu - (uint32_t)place); }
__device__ __forceinline__ uint32_t place_key(uint64_t place) { return (uint32_t)(place >> 32); }

// A thread's streaming pass: the largest logit of each of its kGroups groups of units and, if wanted, the sum of
// exp2((l - top) c), top being the largest of them all.
template <typename T, int kGroups>
struct GroupMaxima {
    float best[kGroups], top, c;
    Exponent ex;
    float2 sums;
    __device__ explicit GroupMaxima(float c_) : top(-INFINITY), c(c_), ex(0.0f, c_), sums(make_float2(0.0f, 0.0f)) {
#pragma unroll
        for (int j = 0; j < kGroups; ++j) best[j] = -INFINITY;
    }
    // a unit of each group
    __device__ __forceinline__ void add(const uint4* q, bool want_sum) {
#pragma unroll
        for (int j = 0; j < kGroups; ++j) best[j] = unit_max<T>(q[j], best[j]);
        if (!want_sum) return;
        float most = best[0];
#pragma unroll
        for (int j = 1; j < kGroups; ++j) most = fmaxf(most, best[j]);
        add_sum<kGroups>(q, most);
    }
    // two units of one group, and two of another, which are told later
    __device__ __forceinline__ void add_pairs(const uint4* q, float2& now, bool want_sum) {
        const float a = units_max<T, 2>(q, -INFINITY), b = units_max<T, 2>(q + 2, -INFINITY);
        now = make_float2(fmaxf(now.x, a), fmaxf(now.y, b));
        if (want_sum) add_sum<4>(q, fmaxf(a, b));
    }
    __device__ __forceinline__ void set_pair(int pair, const float2& now) {
#pragma unroll
        for (int w = 0; w < kGroups / 2; ++w)
            if (w == pair) { best[2 * w] = now.x; best[2 * w + 1] = now.y; }
    }
    template <int kUnits>
    __device__ __forceinline__ void add_sum(const uint4* q, float most) {
        if (most > top) {
            const float scale = ex.raise(top, most);
            if (top != -INFINITY) sums = __fmul2_rn(sums, make_float2(scale, scale));
            top = most;
        }
        if (ex.shift == 0.0f) add_powers<kUnits, false>(q);  // (decided here: within the loop it costs 5 instructions a unit)
        else add_powers<kUnits, true>(q);
    }
    template <int kUnits, bool kShift>
    __device__ __forceinline__ void add_powers(const uint4* q) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            float2 e[Elem<T>::kWidth / 2];
            ex.of_unit<T, kShift>(q[j], e);
#pragma unroll
            for (int i = 1; i < Elem<T>::kWidth / 2; ++i) e[0] = __fadd2_rn(e[0], e[i]);
            sums = __fadd2_rn(sums, e[0]);
        }
    }
    // the groups' largest keys, and by lane 0 the warp's largest logit and its sum relative to that
    __device__ __forceinline__ void of_warp(bool want_sum, uint32_t* group_key, float& warp_top, float& warp_sum) {
        float most = best[0], sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kGroups; ++j) {
            group_key[j] = order_key(best[j]);
            most = fmaxf(most, best[j]);
        }
        const float all = warp_reduce(most, MaxOp());
        if (want_sum) {
            sum = (sums.x + sums.y) * (most == -INFINITY ? 1.0f : fast_exp2((most - all) * c) * ex.mend);
            sum = warp_reduce(sum, AddOp());
        }
        if ((threadIdx.x & 31) == 0) { warp_top = all; warp_sum = sum; }
    }
};

// A key that at least `rank` of a set of keys reach, and not many more, by bisection; reach(key) counts them, `most` is the
// largest.  kLowestKey where fewer are of entries at all.
template <typename Reach>
__device__ __forceinline__ uint32_t search_bound(uint32_t rank, uint32_t most, const Reach& reach) {
    if (reach(kLowestKey) < rank) return kLowestKey;
    uint32_t lo = kLowestKey, hi = most + 1, n;              // reach(lo) >= rank > reach(hi)
    // values an eighth of an octave and more below the largest: a start close by
    for (int down = 20; down < 26; ++down) {
        const uint32_t mid = most - (1u << down);
        if (mid >= most || mid <= lo) break;
        if ((n = reach(mid)) >= rank) { lo = mid; break; }
        hi = mid;
    }
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        n = reach(mid);
        if (n >= rank) lo = mid; else hi = mid;
        if (n >= rank && n <= rank + rank / 8 + 1) break;
    }
    return lo;
}

// One warp: such a key for the keys given: they are kBoundKeys (in registers), or with `many` four times as many.
constexpr int kBoundKeys = 512, kBoundRuns = 4;
__device__ __forceinline__ uint32_t bound_of_rank(const uint32_t* keys, bool many, uint32_t rank) {
    constexpr int kLoads = kBoundKeys / 128;
    const int lane = threadIdx.x & 31;
    const uint4* wide = reinterpret_cast<const uint4*>(keys) + lane;
    uint4 k[kLoads];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        k[i] = wide[i * 32];
        most = max(max(most, max(k[i].x, k[i].y)), max(k[i].z, k[i].w));
    }
    if (many)
        for (int i = kLoads; i < kBoundRuns * kLoads; ++i) {
            const uint4 v = wide[i * 32];
            most = max(max(most, max(v.x, v.y)), max(v.z, v.w));
        }
    most = __reduce_max_sync(kAllLanes, most);
    auto reach = [&](uint32_t key) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) n += (k[i].x >= key) + (k[i].y >= key) + (k[i].z >= key) + (k[i].w >= key);
        if (many)
#pragma unroll 4
            for (int i = kLoads; i < kLoads * kBoundRuns; ++i) {
                const uint4 v = wide[i * 32];
                n += (v.x >= key) + (v.y >= key) + (v.z >= key) + (v.w >= key);
            }
        return __reduce_add_sync(kAllLanes, n);
    };
    return search_bound(rank, most, reach);
}

}  // namespace specs
