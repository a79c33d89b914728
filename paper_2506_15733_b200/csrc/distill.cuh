// Distillation from a teacher's top logits: Kullback-Leibler divergence of the student's softmax p over the
// whole vocabulary from the teacher's probabilities q on a list of K entries, and its gradient.
//
//   q_j  = exp(t_j / T - norm), norm = the teacher's own log-sum-exp, or that of the list alone
//   q_r  = 1 - sum_j q_j        what the list leaves out (0 when the list is normalised by itself)
//   KL   = sum_j q_j (ln q_j - ln p_{id_j}) + q_r (ln q_r - ln p_r),   p_r = 1 - p of the listed ids
//   dKL/dl_v = (p_v S - sum of q_j with id_j = v) / T   for a listed id v,    S = sum_j q_j + q_r
//            = p_v (S - q_r / p_r) / T                  elsewhere
//
// p_r is summed over the entries that are not listed, not taken as 1 - the others, and relative to the largest of them, not
// of the row: a student that is sure of a listed word leaves a p_r far below the rounding of 1, and below the range of a float.
// Where the largest unlisted logit lies more than kLeastRest T below the row's largest, p_r counts as 0.
//
// This header has the arithmetic that the kernels share; distill_rows.cu the kernel for few rows, distill_stream.cu the one for
// many.
#pragma once

#include "logit_rows.cuh"

namespace specs {

enum { kForward, kBackward, kStep };

// A part of a row.  Student, over some of the logits: the largest unlisted one, `top`, and the sum of exp((l - top) / T) over
// the unlisted ones; the largest listed one, `near`, and the sum over those (each id once) relative to it.  Without a normaliser
// (top_lse) nothing is held against the remaining mass, and all logits count as unlisted.
// Teacher, over its share of the list: sums of e_j = exp(a_j - ref) and of e_j ((a_j - ref) - (b_j - near / T)), the latter
// without entries that the student rules out (b_j = -inf): of those the largest t_j is kept, `lost`.  They make the loss infinite
// where q_j > 0 and are nothing where q_j = 0, which only the row's norm tells: a share of negligible entries has e_j = 1 all the
// same.
struct Part { float top, rest, near, listed, lost; double ref, mass, cross; };

__device__ __forceinline__ Part no_part() { return {-INFINITY, 0.0f, -INFINITY, 0.0f, -INFINITY, -INFINITY, 0.0, 0.0}; }
__device__ __forceinline__ float finite_or_zero(float v) { return v == -INFINITY ? 0.0f : v; }

// The row's.  Student: the largest logit, the sum over all entries relative to it, and of that the unlisted part (which may have
// underflowed); the largest unlisted logit, and the sum over the unlisted ones relative to it.  Teacher: norm = ref + ln_mass (never
// added up: next to a lowest value the logarithm would be lost), the sum of q_j (`listed`), and q_r where it counts (`left`).
struct Row { float top, sum, rest, rest_top, rest_own, left; double ref, ln_mass, listed; };

constexpr double kLeastRest = 690.0;                       // exp() of it: 1e-300, well inside the range of a double
constexpr float kNearRest = 1e-17f;                        // `rest` from here on: fp32 relative to the row's largest logit will do

// A logit over T, rounded by itself: fused into a difference, a lowest value's would not be that of its equals.
__device__ __forceinline__ double over_t(const DistillArgs& a, float v) { return __dmul_rn((double)v, a.inv_t64); }

// q_j for the gradient: the exponent in 64 bits, rounded once.
__device__ __forceinline__ float teacher_q(const DistillArgs& a, float t, const Row& row) {
    return expf((float)((over_t(a, t) - row.ref) - row.ln_mass));
}

// The factor that takes a part's teacher sums to the row's reference.
__device__ __forceinline__ double teacher_scale(const Part& p, double ref) {
    return p.ref == ref ? 1.0 : p.mass == 0.0 ? 0.0 : exp(p.ref - ref);
}

// The row from sums over all parts.  Teacher:
__device__ __forceinline__ void set_teacher(const DistillArgs& a, double ref, double mass, Row& row) {
    if (a.top_lse) {
        row.ref = ref;
        row.ln_mass = 0.0;
        row.listed = mass;
        row.left = (float)fmax(0.0, 1.0 - mass);
    } else {                                               // q sums to 1, or nothing is listed
        row.ref = mass == 0.0 ? 0.0 : ref;
        row.ln_mass = mass == 0.0 ? INFINITY : log(mass);
        row.listed = mass == 0.0 ? 0.0 : mass != mass ? mass : 1.0;
        row.left = 0.0f;
    }
}
// What takes a sum of exponentials relative to one logit to another, larger one.
__device__ __forceinline__ float moved(float from, float to, float c) {
    return from == -INFINITY || from == to ? 1.0f : fast_exp2((from - to) * c);
}
// Student, after the teacher: the largest listed logit with the sum relative to it, and the same of the unlisted ones.
struct Listed { float near, sum; };
__device__ __forceinline__ void set_student(const DistillArgs& a, const Listed& listed, float top, float rest, float c, Row& row) {
    row.rest_top = top;
    row.rest_own = rest;
    row.top = fmaxf(top, listed.near);                     // (without top_lse all of these are in `top`, and listed.sum is 0)
    row.rest = rest * moved(top, row.top, c);
    row.sum = row.rest + listed.sum * moved(listed.near, row.top, c);
    const bool none = rest == 0.0f || ((double)row.top - (double)top) * a.inv_t64 > kLeastRest;
    if (none && rest == rest) row.left = 0.0f;             // (NaN stays one)
}

// One warp, a part per lane (no_part where there is none), the results in every lane: the teacher of the row ...
__device__ __forceinline__ void combine_teacher(const DistillArgs& a, const Part& p, Row& row) {
    const double ref = warp_reduce(p.ref, MaxOp());
    set_teacher(a, ref, warp_reduce(p.mass * teacher_scale(p, ref), AddOp()), row);
}
// ... the student's listed entries, and the student with these ...
__device__ __forceinline__ Listed combine_listed(const Part& p, float c) {
    const float near = warp_reduce(p.near, MaxOp());
    return {near, (float)warp_reduce((double)p.listed * moved(p.near, near, c), AddOp())};
}
__device__ __forceinline__ void combine_student(const DistillArgs& a, const Part& p, const Listed& listed, float c, Row& row) {
    const float top = warp_reduce(p.top, MaxOp());
    set_student(a, listed, top, (float)warp_reduce((double)p.rest * moved(p.top, top, c), AddOp()), c, row);
}
// ... or all at once.
__device__ __forceinline__ void combine_row(const DistillArgs& a, const Part& p, float c, Row& row) {
    double ref = p.ref;
    float top = p.top, near = p.near;
    warp_maxima(ref, top, near);
    double mass = p.mass * teacher_scale(p, ref), rest = (double)p.rest * moved(p.top, top, c),
           listed = (double)p.listed * moved(p.near, near, c);
    warp_sums(mass, rest, listed);
    set_teacher(a, ref, mass, row);
    set_student(a, {near, (float)listed}, top, (float)rest, c, row);
}

// What the forward pass leaves of the unlisted part for the backward pass: itself, or its logarithm where it is below the normal
// floats (which is negative, while it is not); 0 where it does not count.
__device__ __forceinline__ float rest_to_stats(const DistillArgs& a, const Row& row) {
    if (!a.top_lse || row.rest_own == 0.0f) return 0.0f;
    if (row.rest >= kNearRest) return row.rest;
    if (row.rest_own != row.rest_own) return row.rest_own;
    const double down = ((double)row.rest_top - (double)row.top) * a.inv_t64;
    if (down < -kLeastRest) return 0.0f;
    const double rest = (double)row.rest_own * exp(down);
    return rest < 1.1754943508222875e-38 ? (float)(log((double)row.rest_own) + down) : (float)rest;
}
__device__ __forceinline__ void student_from_stats(const DistillArgs& a, int64_t r, Row& row) {
    row.top = row.rest_top = a.stats[3 * r];
    row.sum = a.stats[3 * r + 1];
    const float rest = a.stats[3 * r + 2];
    row.rest = row.rest_own = rest < 0.0f ? 0.0f : rest;
    if (rest == 0.0f) {
        row.left = 0.0f;
    } else if (rest < kNearRest) {                         // relative to a logit about as large as the largest unlisted one
        const double ln_rest = rest < 0.0f ? (double)rest : log((double)rest);
        row.rest_top = (float)((double)row.top + ln_rest / a.inv_t64);
        row.rest_own = (float)exp(ln_rest - ((double)row.rest_top - (double)row.top) * a.inv_t64);
    }
}

// One warp: the row's loss, in lane 0.
__device__ __forceinline__ float row_loss(const DistillArgs& a, const Part& p, const Row& row) {
    const double ln_sum = log((double)row.sum);
    const bool none = row.top == -INFINITY && row.sum == 0.0f;      // a student without any entry: all that is listed is lost
    const double ln_share = (p.ref - row.ref) - row.ln_mass, share = p.mass != 0.0 ? exp(ln_share) : 0.0;
    double loss = 0.0;
    if (share != 0.0 && !none)
        loss = share * (p.cross + p.mass * (ln_share -
                                             ((double)finite_or_zero(p.near) - (double)row.top) * a.inv_t64 +
                                             ln_sum));
    if (p.lost != -INFINITY && exp((over_t(a, p.lost) - row.ref) - row.ln_mass) > 0.0) loss += INFINITY;
    loss = warp_reduce(loss, AddOp());
    if (row.left > 0.0f)
        loss += (double)row.left * (log((double)row.left) - (log((double)row.rest_own) +
                                                             ((double)row.rest_top - (double)row.top) * a.inv_t64 - ln_sum));
    return (float)loss;
}

// A unit without the elements whose bits are set: they become -inf.
template <typename T>
__device__ __forceinline__ void hide(uint4& q, uint32_t bits) {
    constexpr int kPerWord = 4 / sizeof(T);
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t mask;
        if (kPerWord == 1) mask = (bits >> i) & 1u ? 0xffffffffu : 0u;
        else mask = ((bits >> (2 * i)) & 1u ? 0xffffu : 0u) | ((bits >> (2 * i + 1)) & 1u ? 0xffff0000u : 0u);
        w[i] = (w[i] & ~mask) | (Elem<T>::kNegInfWord & mask);
    }
    q = make_uint4(w[0], w[1], w[2], w[3]);
}

// A thread's running sum of 2^((l - top) c) over unlisted entries, up to the exponents' common error.  Where nothing but -inf
// (and NaN) has been seen the exponentials are taken from 0, which makes them 0 (NaN).
template <typename T>
struct RunningSums {
    static constexpr int kPairs = Elem<T>::kWidth / 2;
    float c, top = -INFINITY;
    float2 rest = make_float2(0.0f, 0.0f);
    Exponent ex;
    __device__ explicit RunningSums(float c_) : c(c_), ex(0.0f, c_) {}

    __device__ __forceinline__ void raise(float most) {
        if (most > top) {
            const float scale = ex.raise(top, most);
            if (top != -INFINITY) rest = __fmul2_rn(rest, make_float2(scale, scale));
            top = most;
        }
    }
    // kUnits units, which are changed; flagged(j): unit j may have listed entries, which bits_of(j) then has as a mask.
    template <int kUnits, typename Flagged, typename BitsOf>
    __device__ __forceinline__ void add(uint4* q, const Flagged& flagged, const BitsOf& bits_of) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < kUnits; ++j) any |= flagged(j);
        if (any) {
#pragma unroll
            for (int j = 0; j < kUnits; ++j)
                if (flagged(j)) hide<T>(q[j], bits_of(j));
        }
        raise(units_max<T, kUnits>(q, top));
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            float2 e[kPairs];
            ex.of_unit<T>(q[j], e);
#pragma unroll
            for (int k = 1; k < kPairs; ++k) e[0] = __fadd2_rn(e[0], e[k]);
            rest = __fadd2_rn(rest, e[0]);
        }
    }
    // The warp's, in every lane.
    __device__ __forceinline__ void of_warp(Part& part) const {
        part.top = warp_reduce(top, MaxOp());
        const float scale = top == -INFINITY ? 1.0f : fast_exp2((top - part.top) * c) * ex.mend;
        part.rest = warp_reduce((rest.x + rest.y) * scale, AddOp());
    }
};

// What makes the gradient of an entry from its logit: of an unlisted one rest 2^exponent, the exponent relative to the row's largest
// logit, or to the largest unlisted one where that is so far below it that its powers would underflow.  (Listed entries may
// overflow then; they get their own gradient.)
struct Gradient {
    Exponent ex;
    float rest, top, inv_sum, S, scale;
    __device__ Gradient(const Row& row, float c, float scale_) : ex(0.0f, c), scale(scale_) {
        top = finite_or_zero(row.top);
        const bool far = row.left > 0.0f && !(row.rest >= kNearRest);
        const float ref = far ? row.rest_top : top;
        ex = Exponent(ref, c);
        inv_sum = row.sum == 0.0f ? 0.0f : 1.0f / row.sum;
        S = (float)row.listed + row.left;
        const float share = row.left > 0.0f ? row.left / (far ? row.rest_own : row.rest) : 0.0f;
        rest = scale * (ex.mend * (S * inv_sum * moved(ref, top, c) - share));
    }
    template <typename T>
    __device__ __forceinline__ uint4 unit(const uint4& q) const {
        float2 e[Elem<T>::kWidth / 2];
        ex.of_unit<T>(q, e);
#pragma unroll
        for (int i = 0; i < Elem<T>::kWidth / 2; ++i) e[i] = __fmul2_rn(e[i], make_float2(rest, rest));
        return Elem<T>::narrow(reinterpret_cast<const float*>(e));
    }
    __device__ __forceinline__ float unlisted(float logit) const { return rest * ex.of_logit(logit); }
    __device__ __forceinline__ float listed(float logit, float q) const {
        return scale * (fast_exp2((logit - top) * ex.c) * inv_sum * S - q);
    }
};

int launch_distill_stream(const DistillArgs& a, int dtype, int mode, cudaStream_t stream);

}  // namespace specs
