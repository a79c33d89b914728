// Distillation from a teacher's top logits, few rows (the formulas are in distill.cuh).
//
// A cluster of up to 8 CTAs shares a row; in each, eight warps stream a slice of the student's logits, once, with a
// running maximum per thread, and a ninth warp has the list: it marks the slice's listed ids, and adds up its CTA's
// share of the sums over the list.  Everything the row needs is such a sum -- with a_j = t_j / T and b_j = l_{id_j} / T,
//   sum_j q_j (ln q_j - ln p_{id_j}) = e^-norm sum_j e^{a_j} (a_j - b_j) + (sum_j q_j) (ln sum_v e^{l_v / T} - norm),
// each sum taken relative to a value of its own -- so that one exchange through distributed shared memory is all.  The
// gradient pass of specs_distill_step then reads the slice again: the CTAs of a row are in flight together, so the second
// read comes from L2, and HBM sees each logit once in and each gradient once out.
//
// Bound: a launch and the exchange for small rows (64 x 1024 fp32 forward 4.6 us, with the remaining mass 5.3), then the latency of
// a CTA's steps, list and stream in turn, for its share of a row: 592 rows of 16384 bf16, forward 13 us, 1.5 TB/s, step 15 us,
// 2.6 TB/s.  A gradient whose rows lie otherwise on 16-byte boundaries than the logits' is written element by element: 592 x 16384,
// backward 13 -> 45 us, step 15 -> 47; 37 x 131072, 7 -> 20 and 11 -> 30.
#include <cooperative_groups.h>

#include "distill.cuh"

namespace specs {
namespace {

namespace cg = cooperative_groups;

constexpr int kStreamers = 256, kStreamWarps = kStreamers / 32;   // threads that stream the student's logits
constexpr int kThreads = kStreamers + 32;                  // and the list's warp
constexpr int kBatch = 4;                                  // units a thread has in flight
constexpr int kMaxCluster = 8;
constexpr int kResident = 3;                               // CTAs of an SM, at least
constexpr int kLeastUnits = 1024, kPersistent = 12288, kPersistentBackward = 8192;

extern __shared__ uint32_t listed_bits[];                  // a byte per unit of the slice, up to a whole number of batches
__host__ __device__ constexpr int padded_units(int count) {
    return (count + kBatch * kStreamers - 1) / (kBatch * kStreamers) * (kBatch * kStreamers);
}

struct Shared {
    Part part[kMaxCluster];
    float top[kStreamWarps], rest[kStreamWarps];
    float listed_logit[kMaxTopLogits];                     // the slice's listed entries' own logits
    int bad, twice;
};

template <int kValue> struct Count { static constexpr int value = kValue; };

template <typename T>
struct Slice : RowSlice<T, kStreamers> {
    __device__ Slice(const T* p, int V, int shift, int rank) : RowSlice<T, kStreamers>(p, V, shift, rank) {}
    // where the unit of a listed entry stands, -1 for entries that are not there or another CTA's
    __device__ int index_of(int id) const {
        return id >= 0 && id < this->row.V ? this->index((id + this->row.lead) / Elem<T>::kWidth) : -1;
    }
};

__device__ __forceinline__ uint32_t unit_bits(int i) { return reinterpret_cast<const uint8_t*>(listed_bits)[i]; }

// ---- the list's warp ----------------------------------------------------------------------------
// Marks the slice's listed ids; notes whether an id is listed twice, or lies outside the vocabulary.  Returns which of the lane's
// entries (a bit each) are the first of their id.
template <typename T>
__device__ uint32_t mark_listed(const DistillArgs& a, int64_t r, const Slice<T>& slice, Shared& s) {
    uint32_t first = 0, mine = 1;
    for (int j = threadIdx.x & 31; j < a.K; j += 32, mine <<= 1) {
        const int id = a.top_ids[r * a.K + j];
        if (id >= a.V) s.bad = 1;
        const int i = slice.index_of(id);
        if (i < 0) continue;
        if (!SPECS_IN_BOUNDS(i, slice.count(), a.status)) continue;
        const uint32_t bit = 1u << ((i & 3) * 8 + (id + slice.row.lead) % Elem<T>::kWidth);
        if (atomicOr(&listed_bits[i >> 2], bit) & bit) s.twice = 1;
        else first |= mine;
    }
    return first;
}
static_assert(kMaxTopLogits <= 32 * 32, "a bit for each of a lane's entries");

// The teacher's sums: with `student` over the slice's entries, with their part in the student's and the cross sums; else over all.
template <typename T>
__device__ void list_sums(const DistillArgs& a, int64_t r, const Slice<T>& slice, bool student, uint32_t firsts, float c, Shared& s,
                          Part& part) {
    const int32_t* ids = a.top_ids + r * a.K;
    const float* t = a.top_values + r * a.K;
    auto missing = [&](int id) { return student ? slice.index_of(id) < 0 : id < 0 || id >= a.V; };
    float most = -INFINITY, near = -INFINITY;
    for (int j = threadIdx.x & 31; j < a.K; j += 32) {
        const int id = ids[j];
        if (missing(id)) continue;
        most = fmaxf(most, t[j]);
        if (!student || !SPECS_IN_BOUNDS(id, a.V, a.status) || !SPECS_IN_BOUNDS(j, kMaxTopLogits, a.status)) continue;
        const float logit = Elem<T>::to_float(slice.row.row[id]);
        s.listed_logit[j] = logit;
        near = fmaxf(near, logit);
    }
    warp_maxima(most, near);
    part.near = near;
    part.ref = a.top_lse ? (double)a.top_lse[r] : over_t(a, most);
    part.mass = part.cross = 0.0;
    part.lost = -INFINITY;
    part.listed = 0.0f;
    const float from = finite_or_zero(part.near);
    for (int j = threadIdx.x & 31; j < a.K; j += 32, firsts >>= 1) {
        if (missing(ids[j])) continue;
        if (student && a.top_lse && (firsts & 1u)) part.listed += fast_exp2((s.listed_logit[j] - from) * c);
        if (t[j] == -INFINITY) continue;
        const double x = over_t(a, t[j]) - part.ref, e = exp(x);
        part.mass += e;
        if (!student || e == 0.0) continue;
        const float logit = s.listed_logit[j];
        if (logit == -INFINITY) part.lost = fmaxf(part.lost, t[j]);
        else part.cross += e * (x - ((double)logit - (double)from) * a.inv_t64);
    }
    warp_sums(part.listed, part.mass, part.cross);
    warp_maxima(part.lost);
}

// ---- the streaming warps ------------------------------------------------------------------------
// The first batch of a thread's units, asked for before anything else is done.
template <typename T>
__device__ __forceinline__ void first_batch(const Slice<T>& slice, uint4* q) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) q[j] = slice.whole_or_masked(slice.start(threadIdx.x) + j * slice.step);
}

// One pass over the slice, the first batch being there already: the warp's sums.
template <typename T>
__device__ __forceinline__ void read_slice(const DistillArgs& a, const Slice<T>& slice, uint4* q, bool lists, float c, Part& part) {
    RunningSums<T> sums(c);
    const int step = slice.step;
    int u = slice.start(threadIdx.x), i = threadIdx.x;
    auto add = [&](auto count, uint4* units) {       // units whose bits stand kStreamers apart
        constexpr int kUnits = decltype(count)::value;
        uint32_t bits[kUnits];
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            const int at = i + j * kStreamers;
            bits[j] = lists && SPECS_IN_BOUNDS(at, padded_units(slice.count()), a.status) ? unit_bits(at) : 0;
        }
        sums.template add<kUnits>(units, [&](int j) { return bits[j] != 0; }, [&](int j) { return bits[j]; });
    };
    if (u < slice.end) {
        add(Count<kBatch>(), q);
        u += kBatch * step;
        i += kBatch * kStreamers;
    }
    for (; u + (kBatch - 1) * step < slice.end; u += kBatch * step, i += kBatch * kStreamers) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) q[j] = slice.whole(u + j * step);
        add(Count<kBatch>(), q);
    }
    for (; u < slice.end; u += step, i += kStreamers) {
        q[0] = slice.whole(u);
        add(Count<1>(), q);
    }
    for (int k = 0; k < 2; ++k) {
        u = slice.edge(k);
        if (u < 0) continue;
        q[0] = slice.row.load(u);
        i = slice.index(u);
        add(Count<1>(), q);
    }
    sums.of_warp(part);
}

// The list's warp: the streaming warps' sums as the CTA's.
__device__ __forceinline__ void block_sums(const Shared& s, float c, Part& part) {
    const int lane = threadIdx.x & 31;
    const float top = lane < kStreamWarps ? s.top[lane] : -INFINITY;
    part.top = warp_reduce(top, MaxOp());
    part.rest = (float)warp_reduce(lane < kStreamWarps ? (double)s.rest[lane] * moved(top, part.top, c) : 0.0, AddOp());
}

// The slice as if nothing were listed; the first batch is there already if it is wanted at all.
template <typename T>
__device__ __forceinline__ void write_unlisted(const Slice<T>& slice, uint4* q, T* grad, const Gradient& g) {
    const RowUnits<T> out(grad, slice.row.V);
    const int step = slice.step;
    int u = slice.start(threadIdx.x);
    if (out.lead != slice.row.lead) {                      // the two rows lie differently on 16-byte boundaries
        for (; u < slice.row.units; u += step)
            for (int e = 0; e < Elem<T>::kWidth; ++e) {
                const int v = slice.row.first(u) + e;
                if (v >= 0 && v < slice.row.V)
                    grad[v] = Elem<T>::from_float(g.unlisted(Elem<T>::to_float(slice.row.row[v])));
            }
        return;
    }
    auto put = [&](int at, const uint4& v) { *reinterpret_cast<uint4*>(grad + out.first(at)) = v; };
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
        if (u + j * step >= slice.begin && u + j * step < slice.end) put(u + j * step, g.template unit<T>(q[j]));
    for (u += kBatch * step; u + (kBatch - 1) * step < slice.end; u += kBatch * step) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) q[j] = slice.whole(u + j * step);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) put(u + j * step, g.template unit<T>(q[j]));
    }
    for (; u < slice.end; u += step) put(u, g.template unit<T>(slice.whole(u)));
    for (int k = 0; k < 2; ++k) {
        const int at = slice.edge(k);
        if (at >= 0) out.store(at, g.template unit<T>(slice.row.load(at)));
    }
}

template <typename T, int kMode>
__global__ void __launch_bounds__(kThreads, kResident) distill_rows_kernel(const DistillArgs a, int shift) {
    __shared__ Shared s;
    const int ranks = 1 << shift, rank = (int)(blockIdx.x & (ranks - 1));
    const int64_t r = blockIdx.x >> shift;
    const bool clustered = kMode != kBackward && ranks > 1, lists = threadIdx.x >= kStreamers;
    if (clustered) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const Slice<T> slice(static_cast<const T*>(a.logits) + r * a.row_stride, a.V, shift, rank);
    T* grad = kMode == kForward ? nullptr : static_cast<T*>(a.grad) + r * a.grad_stride;
    const float c = a.inv_t * kLog2e;

    uint4 q[kBatch];
    if (!lists) {
        first_batch(slice, q);
        for (int i = threadIdx.x; i < padded_units(slice.count()) / 4; i += kStreamers) listed_bits[i] = 0;
    } else if (threadIdx.x == kStreamers) {
        s.twice = 0;
        s.bad = 0;
    }
    const float weight = a.row_weight ? a.row_weight[r] : 1.0f;
    __syncthreads();
    uint32_t firsts = 0;
    if (lists && weight != 0.0f) firsts = mark_listed(a, r, slice, s);
    __syncthreads();
    const bool bad = s.bad != 0, skip = weight == 0.0f || bad;        // the same in all CTAs of the row

    Part part = no_part();
    if (!skip) {
        if (lists) {
            // (backward: the whole list, there is no exchange)
            list_sums(a, r, slice, kMode != kBackward, firsts, c, s, part);
            if (kMode == kBackward)                        // before anything is written: the gradient may replace the logits
                for (int j = threadIdx.x & 31; j < a.K; j += 32) {
                    const int id = a.top_ids[r * a.K + j];
                    if (slice.index_of(id) >= 0) s.listed_logit[j] = Elem<T>::to_float(slice.row.row[id]);
                }
        } else if (kMode != kBackward) {
            read_slice(a, slice, q, a.top_lse != nullptr, c, part);
            if ((threadIdx.x & 31) == 0) {
                const int w = threadIdx.x >> 5;
                s.top[w] = part.top;
                s.rest[w] = part.rest;
            }
        }
    }
    __syncthreads();
    if (lists && !skip && kMode != kBackward) block_sums(s, c, part);
    if (clustered) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // the others run: their memory may be written
    if (lists && (threadIdx.x & 31) < (kMode == kBackward ? 1 : ranks)) {
        if (clustered) cg::this_cluster().map_shared_rank(&s, threadIdx.x & 31)->part[rank] = part;
        else s.part[0] = part;
    }
    if (kMode == kStep && !lists && !skip) first_batch(slice, q);      // for the gradient, while the CTAs meet
    if (clustered) cg::this_cluster().sync(); else __syncthreads();

    if (skip) {                                            // not trained on, or names no entry
        if (threadIdx.x == 0 && rank == 0) {
            if (bad) atomicOr(a.status, SPECS_DEV_TOKEN_RANGE);
            if (kMode != kBackward) a.loss[r] = bad ? __int_as_float(0x7fc00000) : 0.0f;
            if (kMode == kForward && a.stats) a.stats[3 * r] = a.stats[3 * r + 1] = a.stats[3 * r + 2] = 0.0f;
        }
        if (kMode != kForward && !lists) {
            const Slice<T> out(grad, a.V, shift, rank);
            for (int u = out.start(threadIdx.x); u < out.row.units; u += out.step) out.row.store(u, make_uint4(0, 0, 0, 0));
        }
        return;
    }
    if (kMode == kForward && !(lists && rank == 0)) return;
    const int lane = threadIdx.x & 31;
    const Part mine = lane < (kMode == kBackward ? 1 : ranks) ? s.part[lane] : no_part();
    Row row;
    if (kMode != kBackward) combine_row(a, mine, c, row); else combine_teacher(a, mine, row);
    if (kMode == kBackward) student_from_stats(a, r, row);
    if (kMode != kBackward && lists && rank == 0) {
        const float loss = row_loss(a, mine, row);
        if (threadIdx.x == kStreamers) {
            a.loss[r] = weight * loss;
            if (kMode == kForward && a.stats) {
                a.stats[3 * r] = row.top;
                a.stats[3 * r + 1] = row.sum;
                a.stats[3 * r + 2] = rest_to_stats(a, row);
            }
        }
    }
    if (kMode == kForward) return;

    const Gradient g(row, c, weight * (a.grad_loss ? a.grad_loss[r] : 1.0f) * a.inv_t);
    if (!lists) write_unlisted(slice, q, grad, g);
    __syncthreads();
    for (int j = threadIdx.x; j < a.K; j += kThreads) {    // then the listed ones over it
        const int id = a.top_ids[r * a.K + j];
        if (slice.index_of(id) < 0 || !SPECS_IN_BOUNDS(id, a.V, a.status)) continue;
        float q_id = 0.0f;
        if (s.twice) {
            for (int i = 0; i < a.K; ++i)
                if (a.top_ids[r * a.K + i] == id) q_id += teacher_q(a, a.top_values[r * a.K + i], row);
        } else {
            q_id = teacher_q(a, a.top_values[r * a.K + j], row);
        }
        grad[id] = Elem<T>::from_float(g.listed(s.listed_logit[j], q_id));
    }
}

// CTAs of a row: as many as two a SM allow, but none without kLeastUnits units.  Measured, 131072 bf16, backward / step: 37 rows on
// 296 CTAs 8 / 11 us, on 148 8 / 13; 74 rows on 296 10 / 16, on 592 14 / 20; and 592 rows of 16384 on as many CTAs 16 / 17, on four
// times as many 53 / 93: more CTAs than the device holds wait for their clusters to fit.  512 or 2048 units change little.
template <typename T, int kMode>
int launch_typed(const DistillArgs& a, cudaStream_t stream) {
    const int units = a.V / Elem<T>::kWidth + 2;             // at most, whatever the alignment
    int shift = 0;
    while ((1 << shift) < kMaxCluster && units > (kLeastUnits << shift) && (a.rows << (shift + 1)) <= 2 * a.num_sms) ++shift;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows << shift));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)padded_units(((((units + 31) >> 5) + (1 << shift) - 1) >> shift) * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kMode == kBackward ? 1u : 1u << shift;      // the backward pass exchanges nothing
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, distill_rows_kernel<T, kMode>, a, shift));
}

template <typename T>
bool prepare_typed() {
    constexpr int kMost = padded_units((kMaxRowVocab / Elem<T>::kWidth + 2 + 31) / 32 * 32);      // a whole row of the longest
    const void* kernels[] = {(const void*)distill_rows_kernel<T, kForward>, (const void*)distill_rows_kernel<T, kBackward>,
                             (const void*)distill_rows_kernel<T, kStep>};
    for (const void* k : kernels)
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) != cudaSuccess) return false;
    return true;
}

// One persistent CTA per SM (distill_stream.cu) for more rows than SMs that are long enough for its lists to be fetched behind
// them.  Measured, clusters / streamed, forward, backward and step (us): 131072 bf16, 180 rows 22 / 24, 27 / 25, 39 / 42; 1184 rows
// 72 / 67, 118 / 115, 170 / 142; 98304, 1184 rows 59 / 56, 93 / 89, 128 / 118; 65536, 592 rows 29 / 30, 40 / 33, 47 / 52; 32768, 592
// rows 19 / 28, 23 / 26, 26 / 37; 49152 fp32, 592 rows 34 / 29, 52 / 45, 71 / 56.
template <int kMode>
int launch(const DistillArgs& a, int dtype, cudaStream_t stream) {
    const int units = a.V / (dtype == SPECS_F32 ? 4 : 8);
    if (a.rows > a.num_sms &&
        (units >= kPersistent || (kMode == kBackward && a.rows >= 2 * a.num_sms && units >= kPersistentBackward)))
        return launch_distill_stream(a, dtype, kMode, stream);
    switch (dtype) {
        case SPECS_F32: return launch_typed<float, kMode>(a, stream);
        case SPECS_BF16: return launch_typed<__nv_bfloat16, kMode>(a, stream);
        default: return launch_typed<__half, kMode>(a, stream);
    }
}

}  // namespace

bool prepare_distill_rows() { return prepare_typed<float>() && prepare_typed<__nv_bfloat16>() && prepare_typed<__half>(); }

int launch_distill_forward(const DistillArgs& a, int dtype, cudaStream_t stream) { return launch<kForward>(a, dtype, stream); }
int launch_distill_backward(const DistillArgs& a, int dtype, cudaStream_t stream) { return launch<kBackward>(a, dtype, stream); }
int launch_distill_step(const DistillArgs& a, int dtype, cudaStream_t stream) { return launch<kStep>(a, dtype, stream); }

}  // namespace specs
