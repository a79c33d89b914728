// Distillation from a teacher's top logits: Kullback-Leibler divergence of the student's softmax p over the
// whole vocabulary from the teacher's probabilities q on a list of K entries, and its gradient.
//
//   q_j  = exp(t_j / T - norm), norm = the teacher's own log-sum-exp, or that of the list alone
//   q_r  = 1 - sum_j q_j        what the list leaves out (0 when the list is normalised by itself)
//   KL   = sum_j q_j (ln q_j - ln p_{id_j}) + q_r (ln q_r - ln p_r),   p_r = 1 - p of the listed ids
//   dKL/dl_v = (p_v S - sum of q_j with id_j = v) / T   for a listed id v,    S = sum_j q_j + q_r
//            = p_v (S - q_r / p_r) / T                  elsewhere
//
// p_r is summed over the entries that are not listed, not taken as 1 - the others: a student that is sure of a
// listed word leaves a p_r far below the rounding of 1.  Membership is a bit per element in shared memory.
//
//
// This header has the arithmetic that the kernels share; distill_rows.cu the kernel for few rows, distill_stream.cu the one for
// many.
#pragma once

#include "logit_rows.cuh"

namespace specs {

enum { kForward, kBackward, kStep };

// A part of a row.  Student, over some of the logits: the largest, sums of exp((l - top) / T) over all and over the
// unlisted entries.  Teacher, over its share of the list: sums of e_j = exp(a_j - ref) and of
// e_j ((a_j - ref) - (b_j - near / T)), the latter without entries that the student rules out (b_j = -inf): of those the largest
// t_j is kept, `lost`.  They make the loss infinite where q_j > 0 and are nothing where q_j = 0, which only the row's norm tells: a
// share of negligible entries has e_j = 1 all the same.
struct Part { float top, all, rest, near, lost; double ref, mass, cross; };

__device__ __forceinline__ Part no_part() { return {-INFINITY, 0.0f, 0.0f, 0.0f, -INFINITY, -INFINITY, 0.0, 0.0}; }

// The row's: the student's as above, and norm, sum of q_j (`listed`) and q_r (`left`) of the teacher.
struct Row { float top, sum, rest, left; double norm, listed; };

// q_j for the gradient: the exponent in 64 bits, rounded once.
__device__ __forceinline__ float teacher_q(float t, float inv_t, double norm) {
    return expf((float)((double)t * (double)inv_t - norm));
}

// The factor that takes a part's teacher sums to the row's reference.
__device__ __forceinline__ double teacher_scale(const Part& p, double ref) {
    return p.ref == ref ? 1.0 : p.mass == 0.0 ? 0.0 : exp(p.ref - ref);
}

// One warp, a part per lane (no_part where there is none): the teacher of the row, in every lane.
__device__ __forceinline__ void combine_teacher(const DistillArgs& a, const Part& p, Row& row) {
    const double ref = warp_reduce(p.ref, MaxOp());
    const double mass = warp_reduce(p.mass * teacher_scale(p, ref), AddOp());
    if (a.top_lse) {
        row.norm = ref;
        row.listed = mass;
        row.left = (float)fmax(0.0, 1.0 - mass);
    } else {                                               // q sums to 1, or nothing is listed
        row.norm = mass == 0.0 ? INFINITY : ref + log(mass);
        row.listed = mass == 0.0 ? 0.0 : mass != mass ? mass : 1.0;
        row.left = 0.0f;
    }
}
// ... and the student.
__device__ __forceinline__ void combine_student(const DistillArgs& a, const Part& p, float c, Row& row) {
    row.top = warp_reduce(p.top, MaxOp());
    const double f = p.top == -INFINITY || p.top == row.top ? 1.0 : (double)fast_exp2((p.top - row.top) * c);
    row.sum = (float)warp_reduce((double)p.all * f, AddOp());
    row.rest = a.top_lse ? (float)warp_reduce((double)p.rest * f, AddOp()) : 0.0f;
}

// One warp: the row's loss, in lane 0.
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Part& p, const Row& row) {
    const double ln_sum = log((double)row.sum);
    const bool none = row.top == -INFINITY && row.sum == 0.0f;      // a student without any entry: all that is listed is lost
    const double share = p.mass != 0.0 ? exp(p.ref - row.norm) : 0.0;
    double loss = 0.0;
    if (share != 0.0 && !none)
        loss = share * (p.cross + p.mass * ((p.ref - row.norm) - ((double)p.near - (double)row.top) * (double)a.inv_t + ln_sum));
    if (p.lost != -INFINITY && exp((double)p.lost * (double)a.inv_t - row.norm) > 0.0) loss += INFINITY;
    loss = warp_reduce(loss, AddOp());
    if (row.left > 0.0f && row.rest > 0.0f)
        loss += (double)row.left * (log((double)row.left) - (log((double)row.rest) - ln_sum));
    return (float)loss;
}

// A thread's running sums of 2^((l - top) c), up to the exponents' common error: over listed entries and over the
// others.  Where nothing but -inf (and NaN) has been seen the exponentials are taken from 0, which makes them 0 (NaN).
template <typename T>
struct RunningSums {
    static constexpr int kPairs = Elem<T>::kWidth / 2;
    float c, top = -INFINITY, listed = 0.0f;
    float2 rest = make_float2(0.0f, 0.0f);
    Exponent ex;
    __device__ explicit RunningSums(float c_) : c(c_), ex(0.0f, c_) {}

    __device__ __forceinline__ void raise(float most) {
        if (most > top) {
            if (top != -INFINITY) {
                const float scale = fast_exp2((top - most) * c) * ex.mend;
                listed *= scale;
                rest = __fmul2_rn(rest, make_float2(scale, scale));
            }
            top = most;
            ex = Exponent(top, c);
        }
    }
    // kUnits units; flagged(j): unit j may have listed entries, which bits_of(j) then has as a mask.
    template <int kUnits, typename Flagged, typename BitsOf>
    __device__ __forceinline__ void add(const uint4* q, const Flagged& flagged, const BitsOf& bits_of) {
        raise(units_max<T, kUnits>(q, top));
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            float2 e[kPairs];
            ex.of_unit<T>(q[j], e);
            if (flagged(j)) {
                const uint32_t bits = bits_of(j);
#pragma unroll
                for (int k = 0; k < kPairs; ++k) {
                    const bool x = (bits >> (2 * k)) & 1u, y = (bits >> (2 * k + 1)) & 1u;
                    listed += (x ? e[k].x : 0.0f) + (y ? e[k].y : 0.0f);
                    e[k] = make_float2(x ? 0.0f : e[k].x, y ? 0.0f : e[k].y);
                }
            }
            float2 sum = e[0];
#pragma unroll
            for (int k = 1; k < kPairs; ++k) sum = __fadd2_rn(sum, e[k]);
            rest = __fadd2_rn(rest, sum);
        }
    }
    // The warp's sums, in every lane.
    __device__ __forceinline__ void of_warp(Part& part) const {
        part.top = warp_reduce(top, MaxOp());
        const float scale = top == -INFINITY ? 1.0f : fast_exp2((top - part.top) * c) * ex.mend;
        part.rest = warp_reduce((rest.x + rest.y) * scale, AddOp());
        part.all = part.rest + warp_reduce(listed * scale, AddOp());
    }
};

// What makes the gradient of an entry from its logit.
struct Gradient {
    Exponent ex;
    float inv_sum, S, rest;                                // of an unlisted entry: rest 2^exponent
    float scale;
    __device__ Gradient(const Row& row, float c, float scale_) : ex(row.top == -INFINITY ? 0.0f : row.top, c), scale(scale_) {
        inv_sum = row.sum == 0.0f ? 0.0f : ex.mend / row.sum;
        const float left = row.rest > 0.0f ? row.left : 0.0f;
        S = (float)row.listed + left;
        rest = scale * inv_sum * (left > 0.0f ? S - left * (row.sum / row.rest) : S);
    }
    template <typename T>
    __device__ __forceinline__ uint4 unit(const uint4& q) const {
        float2 e[Elem<T>::kWidth / 2];
        ex.of_unit<T>(q, e);
#pragma unroll
        for (int i = 0; i < Elem<T>::kWidth / 2; ++i) e[i] = __fmul2_rn(e[i], make_float2(rest, rest));
        return Elem<T>::narrow(reinterpret_cast<const float*>(e));
    }
};

int launch_distill_stream(const DistillArgs& a, int dtype, int mode, cudaStream_t stream);

}  // namespace specs
