// Distillation from a teacher's top logits, many rows (the formulas are in distill.cuh): one persistent CTA per SM.
//
// Each CTA takes whole rows, one after the other.  One thread fills a ring of 32 KB stages with bulk copies and runs
// ahead of everyone, through the end of a row into the next one.  16 warps take the stages.  Four more have the lists: they
// fetch those of the rows to come.  One finishes the rows.  So nothing but the sums of a row that its gradient needs is waited
// for, and HBM stays busy during that.  specs_distill_step asks for a row's units twice: the second time they are in L2 (148
// rows of 304 KB, and as much being written).
//
// Listed entries: the 32 units that a warp has of a stage in one register are a group; a group's listed entries are chained,
// a bit per group says whether there are any.  A warp that meets one walks the chain together: the lane that holds
// the entry leaves it out of its sum (the list warps have those), or writes its gradient after the unit's.
//
// Bound: HBM, and the exponentials beside it, which overlap with the copies in part: neither pipe is full.  151936 bf16, 64
// listed, the remaining mass held against the others: 1024 rows forward 69 us, 4.5 TB/s; backward (152064, 100 listed) 117 us,
// 5.4 TB/s; 4096 rows step 535 us, 4.7 TB/s.  A gradient whose rows lie otherwise on 16-byte boundaries than the logits' is written
// element by element, and that is what bounds it then: 1024 x 151936 bf16, backward 115 -> 371 us, step 145 -> 437 us; 333 x 50021
// fp32, 31 -> 32 and 45 -> 48 us.
#include "bulk_ring.cuh"
#include "distill.cuh"

namespace specs {
namespace {

constexpr int kSharedPerBlock = 232448;                    // 227 KB
constexpr int kTakers = 512, kTakeWarps = kTakers / 32;
constexpr int kListers = 128, kListWarps = kListers / 32;
constexpr int kSlots = 3;                                  // rows under way: streamed, being finished, being fetched
constexpr int kStreamBlock = kTakers + kListers + 64;     // and the finishing warp, and the filling one
constexpr int kTake = kStageUnits / kTakers;               // units of a stage that a taking thread has
constexpr int kFlagWords = (kMaxRowVocab / 4 / kStageUnits + 1) * kTake / 32 + 1;
static_assert(kTake * kTakers == kStageUnits && 32 % kTake == 0, "stages are shared out evenly");

// A row's list, with what the taking warps need of the row.
struct Slot {
    int pos[kMaxTopLogits];                                // element of the row's whole units, -1: in none of them
    float q[kMaxTopLogits];
    uint16_t next[kMaxTopLogits];                          // 1 + the next listed entry of the group, 0: none
    Part part[kListWarps];
    Row row;
    float weight, scale;
    float edge[16];                                        // elements of the row's partial units
    int edge_id[16];                                       // -1: none
    double edge_q[16];                                     // what the list gives them, < 0: not listed
    uint32_t flags[kTakeWarps][kFlagWords];                // which of a warp's units, 32 at a time, have listed entries
    float top[kTakeWarps], rest[kTakeWarps], listed[kListWarps];    // sums of the taking warps, and of the list warps' entries
    int skip, bad;
};
struct StreamShared {
    Ring ring;
    uint64_t list_full[kSlots], sums_full[kSlots], row_full[kSlots], done[kSlots];
    Slot slot[kSlots];
    uint32_t abort;
    int go;
};
// A row's slot, and how often that has been used before.
struct SlotPlace {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++slot == kSlots) { slot = 0; phase ^= 1u; }
    }
};

// Calls each(entry, element) for the listed entries of a group that this lane holds; all lanes walk the chain.
template <typename T, typename Each>
__device__ __forceinline__ void walk_group(const Slot& slot, const uint32_t* head, int group, const Each& each) {
    for (uint32_t entry = head[group]; entry; entry = slot.next[entry - 1]) {
        const int pos = slot.pos[entry - 1];
        if (((pos / Elem<T>::kWidth) & 31) == (int)(threadIdx.x & 31)) each((int)entry - 1, pos % Elem<T>::kWidth);
    }
}

// The taking warps' pass over a row: work(units, first unit's index, flags) for the kTake units of each stage -- fewer
// are told by `limit`, the number of whole units --, units and their indexes kTakers apart.
template <typename T, typename Work>
__device__ __forceinline__ bool take_row(StreamShared& s, const Slot& slot, const uint8_t* stages, int stage_count, RingPlace& at,
                                         const StreamRow<T>& row, const BoundedWait& wait, const Work& work) {
    const uint32_t* flags = slot.flags[threadIdx.x >> 5];
    for (int base = 0, chunk = 0; base < row.count; base += kStageUnits, ++chunk) {
        if (!wait(&s.ring.full[at.stage], at.phase)) return false;
        const uint4* in = reinterpret_cast<const uint4*>(stages + (size_t)at.stage * kStageBytes) + threadIdx.x;
        const uint32_t flag = (flags[chunk * kTake / 32] >> (chunk * kTake % 32)) & ((1u << kTake) - 1);
        const int k = base + (int)threadIdx.x;
        uint4 q[kTake];
        if (base + kStageUnits <= row.count) {
#pragma unroll
            for (int j = 0; j < kTake; ++j) q[j] = in[j * kTakers];
        } else {
            const uint32_t ninf = Elem<T>::kNegInfWord;
#pragma unroll
            for (int j = 0; j < kTake; ++j)
                q[j] = k + j * kTakers < row.count ? in[j * kTakers] : make_uint4(ninf, ninf, ninf, ninf);
        }
        ring_release(s.ring, at, stage_count);
        work(q, k, flag);
    }
    return true;
}

template <typename T>
__device__ bool take_sums(StreamShared& s, const Slot& slot, const uint32_t* head, const uint8_t* stages, int stage_count,
                          RingPlace& at, const StreamRow<T>& row, float c, const BoundedWait& wait, bool lists, Part& part) {
    RunningSums<T> sums(c);
    const bool fine = take_row(s, slot, stages, stage_count, at, row, wait, [&](uint4* q, int k, uint32_t flag) {
        if (!lists) flag = 0;
        sums.template add<kTake>(q, [&](int j) { return ((flag >> j) & 1u) != 0; }, [&](int j) {
            uint32_t bits = 0;
            walk_group<T>(slot, head, (k + j * kTakers) >> 5, [&](int, int e) { bits |= 1u << e; });
            return bits;
        });
    });
    sums.of_warp(part);
    return fine;
}

template <typename T>
__device__ bool take_gradient(StreamShared& s, const Slot& slot, const uint32_t* head, const uint8_t* stages, int stage_count,
                              RingPlace& at, const StreamRow<T>& row, T* grad, float c, const BoundedWait& wait) {
    const Gradient g(slot.row, c, slot.scale);
    const RowUnits<T> out(grad, row.row.V);
    const bool alike = out.lead == row.row.lead, zero = slot.bad != 0;
    T* first = grad + row.row.first(row.begin);
    return take_row(s, slot, stages, stage_count, at, row, wait, [&](const uint4* q, int k, uint32_t flag) {
#pragma unroll
        for (int j = 0; j < kTake; ++j) {
            const int u = k + j * kTakers;
            T* to = first + (size_t)u * Elem<T>::kWidth;
            if (u < row.count) {
                uint4 v = g.template unit<T>(q[j]);
                if (zero) v = make_uint4(0, 0, 0, 0);
                if (alike) {
                    *reinterpret_cast<uint4*>(to) = v;
                } else {                                   // the two rows lie differently on 16-byte boundaries
                    union { uint4 q; T e[Elem<T>::kWidth]; } w;
                    w.q = v;
#pragma unroll
                    for (int e = 0; e < Elem<T>::kWidth; ++e) to[e] = w.e[e];
                }
            }
            if ((flag >> j) & 1u)                          // over what the same thread has just written
                walk_group<T>(slot, head, u >> 5, [&](int entry, int e) {
                    to[e] = Elem<T>::from_float(zero ? 0.0f : g.listed(unit_element<T>(q[j], e), slot.q[entry]));
                });
        }
    });
}

__device__ __forceinline__ void listers_meet() { asm volatile("bar.sync 1, %0;" ::"n"(kListers) : "memory"); }

// The list warps: everything of a row's list that does not need the student's sums.
template <typename T, int kMode>
__device__ void load_list(const DistillArgs& a, int64_t r, Slot& slot, uint32_t* head) {
    constexpr int kPer = kMaxTopLogits / kListers;
    const int t = threadIdx.x - kTakers, lane = t & 31, warp = t >> 5;
    const StreamRow<T> row(static_cast<const T*>(a.logits) + r * a.row_stride, a.V);
    const float weight = a.row_weight ? a.row_weight[r] : 1.0f;
    int id[kPer];
    float value[kPer], logit[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = t + i * kListers;
        id[i] = -1;
        value[i] = -INFINITY;
        if (j < a.K) { id[i] = a.top_ids[r * a.K + j]; value[i] = a.top_values[r * a.K + j]; }
    }
    if (t == 0) {
        slot.weight = weight;
        slot.skip = weight == 0.0f;
        slot.bad = 0;
        slot.scale = kMode == kForward ? 0.0f : weight * (a.grad_loss ? a.grad_loss[r] : 1.0f) * a.inv_t;
    }
    if (t < 16) {                                          // the partial units' elements
        const int v = row.edge_element(t);
        slot.edge_id[t] = v;
        slot.edge[t] = v >= 0 && weight != 0.0f ? Elem<T>::to_float(row.row.row[v]) : -INFINITY;
        slot.edge_q[t] = -1.0;
    }
    for (int i = t; i < kTakeWarps * kFlagWords; i += kListers) (&slot.flags[0][0])[i] = 0;
    for (int i = t; i < (row.count + 31) / 32; i += kListers) head[i] = 0;
    listers_meet();
    if (weight == 0.0f) return;
    float most = -INFINITY, near = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = t + i * kListers;
        if (id[i] >= a.V) { slot.bad = 1; id[i] = -1; }
        logit[i] = -INFINITY;
        int pos = id[i] + row.row.lead - row.begin * Elem<T>::kWidth;
        if (id[i] < 0 || pos < 0 || pos >= row.count * Elem<T>::kWidth) pos = -1;
        if (j < a.K) slot.pos[j] = pos;
        if (pos >= 0 && SPECS_IN_BOUNDS(pos, row.count * Elem<T>::kWidth, a.status)) {   // into its group's chain
            const int k = pos / Elem<T>::kWidth, flag = k / kStageUnits * kTake + k % kStageUnits / kTakers;
            slot.next[j] = (uint16_t)atomicExch(&head[k >> 5], (uint32_t)j + 1);
            atomicOr(&slot.flags[k % kTakers / 32][flag / 32], 1u << (flag % 32));
        }
        if (id[i] < 0) continue;
        if (kMode != kBackward && SPECS_IN_BOUNDS(id[i], a.V, a.status)) logit[i] = Elem<T>::to_float(row.row.row[id[i]]);
        most = fmaxf(most, value[i]);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) near = fmaxf(near, logit[i]);
    Part part = no_part();
    warp_maxima(most, near);
    part.near = near;
    near = finite_or_zero(near);
    part.ref = a.top_lse ? (double)a.top_lse[r] : over_t(a, most);
    part.mass = part.cross = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (id[i] < 0 || value[i] == -INFINITY) continue;
        const double x = over_t(a, value[i]) - part.ref, e = exp(x);
        part.mass += e;
        if (kMode == kBackward || e == 0.0) continue;
        if (logit[i] == -INFINITY) part.lost = fmaxf(part.lost, value[i]);
        else part.cross += e * (x - ((double)logit[i] - (double)near) * a.inv_t64);
    }
    warp_sums(part.mass, part.cross);
    warp_maxima(part.lost);
    if (lane == 0) slot.part[warp] = part;
    listers_meet();
    if (kMode != kBackward && a.top_lse) {                 // the student's sum over the listed ids, each of them once
        float listed = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = t + i * kListers;
            if (j >= a.K || slot.pos[j] < 0) continue;
            bool first = true;
            for (uint32_t entry = head[slot.pos[j] / Elem<T>::kWidth >> 5]; entry; entry = slot.next[entry - 1])
                first &= slot.pos[entry - 1] != slot.pos[j] || (int)entry - 1 >= j;
            if (first) listed += fast_exp2((logit[i] - near) * (a.inv_t * kLog2e));
        }
        listed = warp_reduce(listed, AddOp());
        if (lane == 0) slot.listed[warp] = listed;
    }
    Row known;
    combine_teacher(a, lane < kListWarps ? slot.part[lane] : no_part(), known);
    if (t == 0) {
        if (kMode == kBackward) student_from_stats(a, r, known);
        slot.row = known;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = t + i * kListers;
        const float q = id[i] >= 0 && kMode != kForward ? teacher_q(a, value[i], known) : 0.0f;
        if (j < a.K) slot.q[j] = q;
        if (id[i] >= 0 && slot.pos[j] < 0) {               // an element of a partial unit
            for (int e = 0; e < 16; ++e)
                if (slot.edge_id[e] == id[i]) {
                    atomicMax(reinterpret_cast<long long*>(&slot.edge_q[e]), 0ll);   // from -1 to 0, as bits
                    atomicAdd(&slot.edge_q[e], (double)q);
                }
        }
    }
    listers_meet();
    if (kMode != kForward) {                               // an id that is listed more than once has the sum of its q
        float sum[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int j = t + i * kListers;
            sum[i] = 0.0f;
            if (j >= a.K || slot.pos[j] < 0) continue;
            double q = 0.0;                                // exact for a few floats, in any order
            for (uint32_t entry = head[slot.pos[j] / Elem<T>::kWidth >> 5]; entry; entry = slot.next[entry - 1])
                if (slot.pos[entry - 1] == slot.pos[j]) q += (double)slot.q[entry - 1];
            sum[i] = (float)q;
        }
        listers_meet();
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (t + i * kListers < a.K) slot.q[t + i * kListers] = sum[i];
        listers_meet();
    }
}

// The finishing warp: the row's sums, which the gradient pass waits for; its loss; the partial units' gradient.  What the list
// alone gives is worked out while the taking warps are still at it.  False when a wait ran out.
template <typename T, int kMode>
__device__ bool finish_row(const DistillArgs& a, int64_t r, Slot& slot, const SlotPlace& place, StreamShared& s, float c,
                           const BoundedWait& wait) {
    const int lane = threadIdx.x & 31;
    const int edge = lane >= 16 ? slot.edge_id[lane - 16] : -1;
    const float logit = edge >= 0 ? slot.edge[lane - 16] : -INFINITY;
    const double edge_q = edge >= 0 ? slot.edge_q[lane - 16] : -1.0;
    const bool bad = slot.bad != 0;
    Row row = slot.row;
    Part p = no_part();
    Listed listed = {-INFINITY, 0.0f};
    if (kMode != kBackward) {
        if (lane < kListWarps && a.top_lse) { p.near = slot.part[lane].near; p.listed = slot.listed[lane]; }
        if (edge >= 0) {                                   // an entry by itself: its sum is 1 (NaN for NaN and inf, 0 for -inf)
            const float most = fmaxf(logit, -INFINITY), sum = logit == -INFINITY ? 0.0f : 1.0f + (logit - logit);
            if (a.top_lse && edge_q >= 0.0) { p.near = most; p.listed = sum; } else { p.top = most; p.rest = sum; }
        }
        listed = combine_listed(p, c);
    }
    if (!__all_sync(kAllLanes, wait(&s.sums_full[place.slot], place.phase))) return false;
    if (kMode != kBackward) {
        if (lane < kTakeWarps) { p.top = slot.top[lane]; p.rest = slot.rest[lane]; }
        combine_student(a, p, listed, c, row);
        if (kMode == kStep) {
            if (lane == 0) { slot.row = row; barrier_arrive(&s.row_full[place.slot]); }
            __syncwarp();
        }
        const float loss = row_loss(a, lane < kListWarps ? slot.part[lane] : no_part(), row);
        if (lane == 0) {
            a.loss[r] = bad ? __int_as_float(0x7fc00000) : slot.weight * loss;
            if (kMode == kForward && a.stats) {
                a.stats[3 * r] = bad ? 0.0f : row.top;
                a.stats[3 * r + 1] = bad ? 0.0f : row.sum;
                a.stats[3 * r + 2] = bad ? 0.0f : rest_to_stats(a, row);
            }
        }
    }
    if (lane == 0 && bad) atomicOr(a.status, SPECS_DEV_TOKEN_RANGE);
    if (kMode != kForward && edge >= 0) {
        const Gradient g(row, c, slot.scale);
        float v = edge_q >= 0.0 ? g.listed(logit, (float)edge_q) : g.unlisted(logit);
        if (bad) v = 0.0f;
        (static_cast<T*>(a.grad) + r * a.grad_stride)[edge] = Elem<T>::from_float(v);
    }
    return true;
}

template <typename T, int kMode>
__global__ void __launch_bounds__(kStreamBlock, 1)
distill_stream_kernel(const DistillArgs a, int stage_count, int groups) {
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t* stages = smem;
    StreamShared& s = *reinterpret_cast<StreamShared*>(smem + (size_t)stage_count * kStageBytes);
    uint32_t* heads = reinterpret_cast<uint32_t*>(&s + 1);     // of each slot's groups
    const float c = a.inv_t * kLog2e;
    if (threadIdx.x == 0) {
        ring_init(s.ring, stage_count, kTakeWarps);
        for (int i = 0; i < kSlots; ++i) {
            barrier_init(&s.list_full[i], 1);
            barrier_init(&s.sums_full[i], kTakeWarps);
            barrier_init(&s.row_full[i], 1);
            barrier_init(&s.done[i], kTakeWarps + 1);
        }
        s.abort = 0;
        barriers_ready();
    }
    __syncthreads();
    const BoundedWait wait = {&s.abort, a.status};
    const T* logits = static_cast<const T*>(a.logits);

    if (threadIdx.x >= kTakers + kListers + 32) {          // ---- the filling thread
        if (threadIdx.x != kTakers + kListers + 32) return;
        RingPlace at;
        bool fine = true;
        float weight = a.row_weight && blockIdx.x < a.rows ? a.row_weight[blockIdx.x] : 1.0f;
        for (int64_t r = blockIdx.x; r < a.rows && fine; r += gridDim.x) {
            const float mine = weight;
            if (a.row_weight && r + gridDim.x < a.rows) weight = a.row_weight[r + gridDim.x];
            if (mine == 0.0f) continue;
            const StreamRow<T> row(logits + r * a.row_stride, a.V);
            const T* from = row.from();
            for (int pass = 0; pass < (kMode == kStep ? 2 : 1) && fine; ++pass)
                for (int base = 0; base < row.count && fine; base += kStageUnits)
                    fine = ring_fill(s.ring, at, stage_count, stages, from + (size_t)base * Elem<T>::kWidth,
                                     min(kStageUnits, row.count - base), wait);
        }
        ring_drain(s.ring, at, stage_count, wait);
        return;
    }
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < kTakers) {                           // ---- the taking warps
        const int warp = threadIdx.x >> 5;
        RingPlace at;
        SlotPlace place;
        for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, place.next()) {
            Slot& slot = s.slot[place.slot];
            const uint32_t* head = heads + place.slot * groups;
            if (!wait(&s.list_full[place.slot], place.phase)) return;
            const StreamRow<T> row(logits + r * a.row_stride, a.V);
            T* grad = static_cast<T*>(a.grad) + r * a.grad_stride;
            const bool skip = slot.skip != 0;
            if (skip) {
                if (kMode != kForward) {
                    const RowUnits<T> out(grad, a.V);
                    for (int u = threadIdx.x; u < out.units; u += kTakers) out.store(u, make_uint4(0, 0, 0, 0));
                }
            } else if (kMode != kBackward) {
                Part part;
                if (!take_sums(s, slot, head, stages, stage_count, at, row, c, wait, a.top_lse != nullptr, part)) return;
                if (lane == 0) {
                    slot.top[warp] = part.top;
                    slot.rest[warp] = part.rest;
                }
            }
            __syncwarp();
            if (lane == 0) barrier_arrive(&s.sums_full[place.slot]);
            if (kMode != kForward && !skip) {
                if (kMode == kStep && !wait(&s.row_full[place.slot], place.phase)) return;
                if (!take_gradient(s, slot, head, stages, stage_count, at, row, grad, c, wait)) return;
            }
            __syncwarp();
            if (lane == 0) barrier_arrive(&s.done[place.slot]);
        }
        return;
    }
    if (threadIdx.x >= kTakers + kListers) {               // ---- the finishing warp
        SlotPlace place;
        for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, place.next()) {
            Slot& slot = s.slot[place.slot];
            if (!__all_sync(kAllLanes, wait(&s.list_full[place.slot], place.phase))) return;
            if (!slot.skip) {
                if (!finish_row<T, kMode>(a, r, slot, place, s, c, wait)) return;
            } else {
                if (!__all_sync(kAllLanes, wait(&s.sums_full[place.slot], place.phase))) return;
                if (lane == 0 && kMode == kStep) barrier_arrive(&s.row_full[place.slot]);
                if (lane == 0 && kMode != kBackward) a.loss[r] = 0.0f;
                if (lane < 3 && kMode == kForward && a.stats) a.stats[3 * r + lane] = 0.0f;
            }
            __syncwarp();
            if (lane == 0) barrier_arrive(&s.done[place.slot]);
        }
        return;
    }
    // ---- the list warps
    const int t = threadIdx.x - kTakers;
    SlotPlace place;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, place.next()) {
        if (t < 32) {                                      // one warp waits, and tells the others how that went
            const bool fine = __all_sync(kAllLanes, wait(&s.done[place.slot], place.phase ^ 1u));
            if (t == 0) s.go = fine;
        }
        listers_meet();
        if (!s.go) return;
        load_list<T, kMode>(a, r, s.slot[place.slot], heads + place.slot * groups);
        listers_meet();
        if (t == 0) barrier_arrive(&s.list_full[place.slot]);
    }
}

template <typename T, int kMode>
int launch_stream(const DistillArgs& a, cudaStream_t stream) {
    const int groups = (a.V / Elem<T>::kWidth + 31) / 32;
    const int fixed = (int)sizeof(StreamShared) + kSlots * groups * 4;
    const int room = (kSharedPerBlock - fixed) / kStageBytes, stages = room < kRingStages ? room : kRingStages;
    const int bytes = stages * kStageBytes + fixed;
    const int grid = a.rows < a.num_sms ? (int)a.rows : a.num_sms;
    distill_stream_kernel<T, kMode><<<grid, kStreamBlock, bytes, stream>>>(a, stages, groups);
    return cuda_status(cudaGetLastError());
}

template <typename T>
bool prepare_typed() {
    const void* kernels[] = {(const void*)distill_stream_kernel<T, kForward>, (const void*)distill_stream_kernel<T, kBackward>,
                             (const void*)distill_stream_kernel<T, kStep>};
    for (const void* k : kernels)
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedPerBlock) != cudaSuccess) return false;
    return true;
}

template <int kMode>
int launch_mode(const DistillArgs& a, int dtype, cudaStream_t stream) {
    switch (dtype) {
        case SPECS_F32: return launch_stream<float, kMode>(a, stream);
        case SPECS_BF16: return launch_stream<__nv_bfloat16, kMode>(a, stream);
        default: return launch_stream<__half, kMode>(a, stream);
    }
}

}  // namespace

bool prepare_distill_stream() { return prepare_typed<float>() && prepare_typed<__nv_bfloat16>() && prepare_typed<__half>(); }

int launch_distill_stream(const DistillArgs& a, int dtype, int mode, cudaStream_t stream) {
    return mode == kForward ? launch_mode<kForward>(a, dtype, stream)
         : mode == kBackward ? launch_mode<kBackward>(a, dtype, stream) : launch_mode<kStep>(a, dtype, stream);
}

}  // namespace specs
