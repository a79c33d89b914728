// A ring of shared-memory stages filled by bulk copies: one thread of a CTA asks for runs of 16-byte units of
// global memory, in order, and the CTA's other warps take them in the same order.  A stage is full when its bytes have
// arrived and empty when every taking warp has read it.
//
// Every wait is bounded: after two seconds the CTA's abort flag and SPECS_DEV_TIMEOUT are raised, and every role leaves.
#pragma once

#include "logit_rows.cuh"

namespace specs {

constexpr unsigned long long kRingWaitNs = 2000000000ull;      // per wait
constexpr unsigned long long kRingDrainNs = 20000000ull;       // per stage, for copies in flight after an abort

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(bar)) : "memory");
}
__device__ __forceinline__ bool barrier_passed(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(shared_address(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long timer_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// False when the wait ran out, or another role's did.
struct BoundedWait {
    volatile uint32_t* abort;      // in shared memory
    uint32_t* status;
    __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity) const {
        if (barrier_passed(bar, parity)) return true;
        const unsigned long long start = timer_ns();
        for (;;) {
            if (barrier_passed(bar, parity)) return true;
            if (*abort) return false;
            if (timer_ns() - start > kRingWaitNs) {
                *abort = 1;
                atomicOr(status, SPECS_DEV_TIMEOUT);
                return false;
            }
        }
    }
    // For copies in flight: gives up quietly.
    __device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) const {
        const unsigned long long start = timer_ns();
        while (!barrier_passed(bar, parity) && timer_ns() - start <= kRingDrainNs) {}
    }
};

constexpr int kStageUnits = 2048, kStageBytes = kStageUnits * 16;
constexpr int kRingStages = 6;                                // at most

struct Ring {
    uint64_t full[kRingStages], empty[kRingStages];
};
// A role's place in the ring.
struct RingPlace {
    int stage = 0;
    uint32_t phase = 0;
    bool wrapped = false;
    __device__ __forceinline__ void next(int stages) {
        if (++stage == stages) { stage = 0; phase ^= 1u; wrapped = true; }
    }
};

__device__ __forceinline__ void ring_init(Ring& ring, int stages, uint32_t takers) {
    for (int i = 0; i < stages; ++i) { barrier_init(&ring.full[i], 1); barrier_init(&ring.empty[i], takers); }
}
// After the barriers' initialisation, before anyone uses them (and a block barrier).
__device__ __forceinline__ void barriers_ready() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// The filling thread: the next stage gets `units` (at most kStageUnits) from `from`, a 16-byte boundary.
__device__ __forceinline__ bool ring_fill(Ring& ring, RingPlace& at, int stages, uint8_t* smem, const void* from, int units,
                                          const BoundedWait& wait) {
    if (!wait(&ring.empty[at.stage], at.phase ^ 1u)) return false;
    const uint32_t bar = shared_address(&ring.full[at.stage]), bytes = (uint32_t)units * 16u;
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     shared_address(smem + (size_t)at.stage * kStageBytes)),
                 "l"(from), "r"(bytes), "r"(bar) : "memory");
    at.next(stages);
    return true;
}
// A taking warp, whole, has read the stage it is at.  The copy that comes next writes through another proxy than the one that the
// warp read through: without the fence a read that still waits (behind a queue of scattered stores, say) may find that copy's data.
__device__ __forceinline__ void ring_release(Ring& ring, RingPlace& at, int stages) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if ((threadIdx.x & 31) == 0) barrier_arrive(&ring.empty[at.stage]);
    at.next(stages);
}
// The filling thread, before it leaves: no copy may still be under way.  `at` is where the next fill would have gone.
__device__ __forceinline__ void ring_drain(Ring& ring, const RingPlace& at, int stages, const BoundedWait& wait) {
    for (int i = 0; i < stages; ++i) {
        const bool this_round = i < at.stage;
        if (!this_round && !at.wrapped) continue;            // never filled
        wait.drain(&ring.full[i], this_round ? at.phase : at.phase ^ 1u);
    }
}

// A row as a streaming kernel sees it: whole units from memory, the first of them at from(), and the elements of up to
// two partial ones.
template <typename T>
struct StreamRow {
    RowUnits<T> row;
    int begin, count;                                      // whole units
    __device__ StreamRow(const T* p, int V) : row(p, V) {
        begin = row.lead > 0 ? 1 : 0;
        count = max(0, (V + row.lead) / RowUnits<T>::kWidth - begin);
    }
    __device__ const T* from() const { return row.row + row.first(begin); }
    // i = 0 .. 7: elements of a partial first unit, 8 .. 15: of a partial last one; -1: there is none
    __device__ int edge_element(int i) const {
        const int u = i < 8 ? 0 : row.units - 1, e = i & 7, v = row.first(u) + e;
        const bool partial = e < Elem<T>::kWidth && (u < begin || u >= begin + count) && !(i >= 8 && u == 0 && begin == 1);
        return partial && v >= 0 && v < row.V ? v : -1;
    }
};

}  // namespace specs
