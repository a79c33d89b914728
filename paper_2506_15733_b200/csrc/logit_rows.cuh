// Device helpers shared by the kernels that work on rows of vocabulary logits (sample_rows.cu,
// top_stream.cu, distill_rows.cu, distill_stream.cu): element types, a row seen as aligned 16-byte units, exponents, reductions.
#pragma once

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "specs_internal.h"

namespace specs {

constexpr float kLog2e = 1.4426950408889634f;
constexpr unsigned kAllLanes = 0xffffffffu;

// ---- element types ------------------------------------------------------------------------------
// A unit is 16 bytes of a row: `kWidth` elements, widened to fp32 on use (exact for all three types).
template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kWidth = 4;
    static constexpr uint32_t kNegInfWord = 0xff800000u;
    __device__ static void widen(const uint4& q, float* f) {
        f[0] = __uint_as_float(q.x); f[1] = __uint_as_float(q.y); f[2] = __uint_as_float(q.z); f[3] = __uint_as_float(q.w);
    }
    __device__ static float to_float(float v) { return v; }
    __device__ static uint4 narrow(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    __device__ static float from_float(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kWidth = 8;
    static constexpr uint32_t kNegInfWord = 0xff80ff80u;
    __device__ static void widen(const uint4& q, float* f) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ static uint4 narrow(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
    static constexpr int kWidth = 8;
    static constexpr uint32_t kNegInfWord = 0xfc00fc00u;
    __device__ static void widen(const uint4& q, float* f) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        }
    }
    __device__ static float to_float(__half v) { return __half2float(v); }
    __device__ static uint4 narrow(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static __half from_float(float v) { return __float2half_rn(v); }
};

// ---- a row as units -----------------------------------------------------------------------------
// Units lie on 16-byte boundaries of memory, so a row that starts anywhere else has a first unit that only
// partly belongs to it (`lead` elements of it lie before the row), and nearly every row has such a last
// unit.  Whole units are read and written 16 bytes at a time, partial ones element by element: nothing
// outside the row is ever touched.  Elements that a partial unit lacks read as -inf, which no operator counts.
template <typename T>
struct RowUnits {
    static constexpr int kWidth = Elem<T>::kWidth;
    T* row;
    int V, lead, units;

    __device__ RowUnits(const T* p, int V_) : row(const_cast<T*>(p)), V(V_) {
        lead = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
        units = (V + lead + kWidth - 1) / kWidth;
    }
    // the row index of a unit's first element (negative in a partial first unit)
    __device__ int first(int u) const { return u * kWidth - lead; }
    __device__ bool whole(int u) const { return first(u) >= 0 && first(u) + kWidth <= V; }
    __device__ __forceinline__ uint4 load(int u) const {
        const int e0 = first(u);
        return whole(u) ? *reinterpret_cast<const uint4*>(row + e0) : partial(row, V, e0);
    }
    // (kept out of line: it is rare, and long)
    __device__ static __noinline__ uint4 partial(const T* row, int V, int e0) {
        union { uint4 q; T e[kWidth]; uint32_t w[4]; } v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = Elem<T>::kNegInfWord;
#pragma unroll
        for (int i = 0; i < kWidth; ++i)
            if (e0 + i >= 0 && e0 + i < V) v.e[i] = row[e0 + i];
        return v.q;
    }
    __device__ __forceinline__ void store(int u, const uint4& q) const {
        const int e0 = first(u);
        if (whole(u)) *reinterpret_cast<uint4*>(row + e0) = q;
        else store_partial(row, V, e0, q);
    }
    __device__ static __noinline__ void store_partial(T* row, int V, int e0, const uint4 q) {
        union { uint4 q; T e[kWidth]; } v;
        v.q = q;
#pragma unroll
        for (int i = 0; i < kWidth; ++i)
            if (e0 + i >= 0 && e0 + i < V) row[e0 + i] = v.e[i];
    }
};

// The units of a row that one CTA of a cluster works on: every ranks-th run of 32, so that a vocabulary sorted by
// frequency loads all CTAs alike.  Thread t has the units start(t), start(t) + step, ..., warps read 512 bytes at a time.
// Loops take the whole units of memory in batches without any special case; the up to two partial ones of the row
// (`edge`) are left to the threads that have them.
template <typename T, int kThreads>
struct RowSlice {
    static_assert((kThreads & (kThreads - 1)) == 0, "units are dealt out by masks");
    RowUnits<T> row;
    int shift, rank, step, begin, end;                       // 2^shift CTAs; whole units: begin .. end - 1
    __device__ RowSlice(const T* p, int V, int shift_, int rank_) : row(p, V), shift(shift_), rank(rank_) {
        step = kThreads << shift;
        begin = row.lead > 0 ? 1 : 0;
        end = (V + row.lead) / RowUnits<T>::kWidth;
    }
    __device__ int start(int t) const { return ((((t >> 5) << shift) + rank) << 5) + (t & 31); }
    __device__ uint4 whole(int u) const { return *reinterpret_cast<const uint4*>(row.row + row.first(u)); }
    __device__ uint4 whole_or_masked(int u) const {
        const uint32_t ninf = Elem<T>::kNegInfWord;
        uint4 q = make_uint4(ninf, ninf, ninf, ninf);
        if (u >= begin && u < end) q = whole(u);
        return q;
    }
    // the row's partial units: the first (which = 0) and the last (1) one; -1 where this thread has none
    __device__ int edge(int which) const {
        const int u = which == 0 ? 0 : row.units - 1;
        if (which == 0 ? begin == 0 : (end == row.units || (u == 0 && begin == 1))) return -1;
        return (u & (step - 1)) == start(threadIdx.x) ? u : -1;
    }
    // Calls body(units, first unit) for the thread's units, kBatch at a time and step apart; units that are not there are
    // masked.  A partial unit comes by itself, in the place of the batch that its number has.  One copy of the body.
    template <int kBatch, typename Body>
    __device__ __forceinline__ void each_batch(const Body& body) const {
        int u = start(threadIdx.x), which = 0;
        for (;;) {
            uint4 q[kBatch];
            int at = u;
            if (u >= begin && u + (kBatch - 1) * step < end) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) q[j] = whole(u + j * step);
                u += kBatch * step;
            } else if (u < end) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) q[j] = whole_or_masked(u + j * step);
                u += kBatch * step;
            } else if (which < 2) {
                const int partial = edge(which++);
                if (partial < 0) continue;
                const uint32_t ninf = Elem<T>::kNegInfWord;
                const int n = (partial - start(threadIdx.x)) / step % kBatch;
                const uint4 v = row.load(partial);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) q[j] = j == n ? v : make_uint4(ninf, ninf, ninf, ninf);
                at = partial - n * step;
            } else {
                break;
            }
            body(q, at);
        }
    }
    // where a unit stands among the CTA's (thread t's n-th one at n * kThreads + t), -1 for another CTA's
    __device__ int index(int u) const {
        const int run = u >> 5;
        return (run & ((1 << shift) - 1)) == rank ? ((run >> shift) << 5) + (u & 31) : -1;
    }
    __device__ int count() const { return (((((row.units + 31) >> 5) - rank - 1) >> shift) + 1) * 32; }   // at most
};

// Element e of a unit.
template <typename T>
__device__ __forceinline__ float unit_element(const uint4& q, int e) {
    constexpr int kPerWord = 4 / sizeof(T);
    const int w = e / kPerWord;
    const uint32_t word = w == 0 ? q.x : w == 1 ? q.y : w == 2 ? q.z : q.w;
    if (kPerWord == 1) return __uint_as_float(word);
    const uint16_t half = (uint16_t)(word >> (16 * (e % kPerWord)));
    T v;
    memcpy(&v, &half, sizeof(T) < sizeof(half) ? sizeof(T) : sizeof(half));
    return Elem<T>::to_float(v);
}

// The largest element of a unit, and `best` (NaN is passed over).
template <typename T> __device__ __forceinline__ float unit_max(const uint4& q, float best) {
    float f[4];
    Elem<float>::widen(q, f);
    return fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), best);
}
template <> __device__ __forceinline__ float unit_max<__nv_bfloat16>(const uint4& q, float best) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(fmaxf(__low2float(m), __high2float(m)), best);
}
template <> __device__ __forceinline__ float unit_max<__half>(const uint4& q, float best) {
    const __half2* h = reinterpret_cast<const __half2*>(&q);
    const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(fmaxf(__low2float(m), __high2float(m)), best);
}

// The largest element of several units, and `best`.
template <typename T2, int kUnits>
__device__ __forceinline__ T2 halves_max(const uint4* q) {
    T2 m[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
        const T2* h = reinterpret_cast<const T2*>(&q[j]);
        m[j] = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    }
#pragma unroll
    for (int j = 1; j < kUnits; ++j) m[0] = __hmax2(m[0], m[j]);
    return m[0];
}
template <typename T, int kUnits>
__device__ __forceinline__ float units_max(const uint4* q, float best) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j) best = unit_max<T>(q[j], best);
        return best;
    } else {
        using T2 = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
        const T2 m = halves_max<T2, kUnits>(q);
        return fmaxf(fmaxf(__low2float(m), __high2float(m)), best);
    }
}

// ---- arithmetic ---------------------------------------------------------------------------------
// 2^x with a relative error of about 2^-22 (the special-function unit); 0 for -inf.
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Exponents in one multiply-add: 2^(f c - offset) = 2^((f - ref) c) 2^error.  The product offset = ref c is rounded, and
// `error` is what that loses; a sum of such powers is put right at its end, by the factor `mend` = 2^-error.  Where ref c is
// so large that its rounding would swamp the exponents (rows of the type's lowest values, vanishing temperatures), ref is
// subtracted first.
struct Exponent {
    float c, offset, shift, mend;
    __device__ Exponent(float ref, float c_) : c(c_) {
        const bool large = !(fabsf(ref) * c <= 65536.0f);
        shift = large ? ref : 0.0f;
        offset = large ? 0.0f : ref * c;
        const float y = large ? 0.0f : 0.69314718f * fmaf(ref, c, -offset);      // |error| < 2^-8: two terms will do
        mend = fmaf(y, fmaf(y, 0.5f, -1.0f), 1.0f);
    }
    // a unit's elements, two per instruction up to the special-function unit; kShift: `shift` may be other than 0
    template <typename T, bool kShift = true>
    __device__ __forceinline__ void of_unit(const uint4& q, float2* out) const {
        float2 f[Elem<T>::kWidth / 2];
        Elem<T>::widen(q, reinterpret_cast<float*>(f));
        if (kShift && shift != 0.0f) {
#pragma unroll
            for (int i = 0; i < Elem<T>::kWidth / 2; ++i) f[i] = __fadd2_rn(f[i], make_float2(-shift, -shift));
        }
#pragma unroll
        for (int i = 0; i < Elem<T>::kWidth / 2; ++i) {
            const float2 x = __ffma2_rn(f[i], make_float2(c, c), make_float2(-offset, -offset));
            out[i] = make_float2(fast_exp2(x.x), fast_exp2(x.y));
        }
    }
    // Makes the exponents relative to a larger `ref`, and returns what a sum of powers so far has to be multiplied by: it was made
    // with the old error, and will be put right for the new one.
    __device__ __forceinline__ float raise(float from, float ref) {
        const float old = mend;
        *this = Exponent(ref, c);
        const float d = 1.0f - mend;                        // below 2^-8: 1 / mend = 1 + d + d^2, to 2^-24
        return fast_exp2((from - ref) * c) * (old * (1.0f + fmaf(d, d, d)));
    }
    __device__ __forceinline__ float operator()(float f) const { return fast_exp2(fmaf(f, c, -offset)); }
    __device__ __forceinline__ float of_logit(float f) const { return operator()(f - shift); }
};

// An unsigned key with the order of the floats: -0 and +0 share one, NaN comes below everything.
__device__ __forceinline__ uint32_t order_key(float f) {
    const uint32_t u = __float_as_uint(f + 0.0f);
    if (f != f) return 0u;
    return u ^ ((u & 0x80000000u) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
    return __uint_as_float(key ^ ((key & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kKeyNegInf = 0x007fffffu;         // order_key(-inf): keys up to this one are masked entries

// ---- warp reductions ----------------------------------------------------------------------------
template <typename V, typename Op>
__device__ __forceinline__ V warp_reduce(V v, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(kAllLanes, v, o));
    return v;
}
struct MaxOp { template <typename V> __device__ V operator()(V a, V b) const { return a > b ? a : b; } };
struct AddOp { template <typename V> __device__ V operator()(V a, V b) const { return a + b; } };
// Several at a time: their shuffles do not wait for one another.
template <typename... V>
__device__ __forceinline__ void warp_maxima(V&... v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ((v = MaxOp()(v, __shfl_xor_sync(kAllLanes, v, o))), ...);
}
template <typename... V>
__device__ __forceinline__ void warp_sums(V&... v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ((v += __shfl_xor_sync(kAllLanes, v, o)), ...);
}

}  // namespace specs
