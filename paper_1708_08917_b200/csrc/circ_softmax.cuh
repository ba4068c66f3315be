// Softmax statistics of rows in one pass: exponentials relative to a running maximum, joined over the lanes of a warp.
#pragma once
#include "circ_rows.cuh"

namespace circ {

// exp(z - top) summed up, with the sum's own `top`: the pair that a pass over a row carries along.
struct Softmax {
    float top, sum;
};
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp2_of(float d) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    return r;
}
// The exponentials of a row relative to `top`: exp(z - top) 2^shift = 2^(z log2(e) - base), one multiply-add and one exponential an
// element.  base is top log2(e) rounded, shift what the rounding left: up to |top| 2^-23, so scores beyond 2^20 (a row that a mask's
// lowest value fills) take the difference to the top first, and shift is 0.  A top of -inf counts as 0.  Scores of a temperature tau
// stand for z / tau: `scale` is log2(e) / tau then.
struct Exponent {
    float top, base, shift, scale;
    bool plain;
    __device__ __forceinline__ explicit Exponent(float t, float k = kLog2e) : scale(k) {
        top = t == -INFINITY ? 0.f : t;
        plain = !(fabsf(top * k) <= 1048576.f * kLog2e);
        base = plain ? 0.f : top * k;
        shift = plain ? 0.f : fmaf(top, k, -base);
    }
    template <bool PLAIN, int N>
    __device__ __forceinline__ void powers(const float (&z)[N], float (&e)[N]) const {
        if constexpr (PLAIN) {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = exp2_of((z[i] - top) * scale);
        } else if constexpr (N % 2 == 0) {
            const Pair k = pair_of(scale, scale), b = pair_of(-base, -base);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                split(pair_fma(pair_of(z[i], z[i + 1]), k, b), e[i], e[i + 1]);
                e[i] = exp2_of(e[i]);
                e[i + 1] = exp2_of(e[i + 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = exp2_of(fmaf(z[i], scale, -base));
        }
    }
    template <int N>
    __device__ __forceinline__ void of(const float (&z)[N], float (&e)[N]) const {
        if (plain) powers<true>(z, e);
        else powers<false>(z, e);
    }
};
// Two pairs as one.  A part whose top is -inf has the sum 0 or, from a NaN, NaN.
__device__ __forceinline__ Softmax join(Softmax a, Softmax b, float scale) {
    const float top = fmaxf(a.top, b.top);
    return Softmax{top, a.sum * (a.top == -INFINITY ? 0.f : exp2_of((a.top - top) * scale)) +
                            b.sum * (b.top == -INFINITY ? 0.f : exp2_of((b.top - top) * scale))};
}
// The lanes' pairs as one: the top first, so that every lane takes one exponential.
__device__ __forceinline__ Softmax warp_join(Softmax v, float scale = kLog2e) {
    float top = v.top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    // a part whose top is -inf has the sum 0 or, from a NaN, NaN
    return Softmax{top, warp_sum(v.sum * (v.top == -INFINITY ? 0.f : exp2_of((v.top - top) * scale)))};
}
// The largest element of some vectors; bfloat16 ones are compared in pairs as they lie.
template <int VEC, int N>
__device__ __forceinline__ float most_of(const RawVec<float, VEC> (&raw)[N]) {
    float most = raw[0].get(0);
#pragma unroll
    for (int i = 1; i < N * VEC; ++i) most = fmaxf(most, raw[i / VEC].get(i % VEC));
    return most;
}
template <int VEC, int N>
__device__ __forceinline__ float most_of(const RawVec<__nv_bfloat16, VEC> (&raw)[N]) {
    constexpr int W = VEC / 2;
    __nv_bfloat162 most = *reinterpret_cast<const __nv_bfloat162*>(&raw[0].w[0]);
#pragma unroll
    for (int i = 1; i < N * W; ++i) most = __hmax2(most, *reinterpret_cast<const __nv_bfloat162*>(&raw[i / W].w[i % W]));
    return fmaxf(__low2float(most), __high2float(most));
}
// A thread's part of a row: vectors in any order, one exponential an element and one more where the top rises.
struct Running {
    float top = -INFINITY, sum = 0.f;      // sum of exp(z - top) 2^shift
    Exponent ex;
    float limit;                           // the top goes no higher: with FLT_MAX a score of +inf makes the sum +inf, without a limit NaN
    __device__ __forceinline__ explicit Running(float scale = kLog2e, float l = INFINITY) : ex(-INFINITY, scale), limit(l) {}
    __device__ __forceinline__ void rise(float most) {
        if (!(most > top)) return;
        most = most > limit ? limit : most;
        const Exponent to(most, ex.scale);
        sum *= top == -INFINITY ? 0.f : exp2_of((top - most) * ex.scale + (to.shift - ex.shift));
        top = most;
        ex = to;
    }
    template <int VEC>
    __device__ __forceinline__ void take(const float (&z)[VEC]) {
        float most = z[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) most = fmaxf(most, z[e]);
        rise(most);
        float e[VEC], part = 0.f;
        ex.of(z, e);
#pragma unroll
        for (int i = 0; i < VEC; ++i) part += e[i];
        sum += part;
    }
    // N vectors as loaded: one look at the top for all of them.
    template <typename T, int VEC, int N>
    __device__ __forceinline__ void take(const RawVec<T, VEC> (&raw)[N]) {
        rise(most_of(raw));
        if (ex.plain) add<true>(raw);      // one branch for all of them
        else add<false>(raw);
    }
    template <bool PLAIN, typename T, int VEC, int N>
    __device__ __forceinline__ void add(const RawVec<T, VEC> (&raw)[N]) {
        Pair part[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float z[VEC], e[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) z[i] = raw[u].get(i);
            ex.powers<PLAIN>(z, e);
            part[u] = pair_of(e[0], e[1]);
#pragma unroll
            for (int i = 2; i < VEC; i += 2) part[u] = pair_add(part[u], pair_of(e[i], e[i + 1]));
        }
#pragma unroll
        for (int u = 1; u < N; ++u) part[0] = pair_add(part[0], part[u]);
        float lo, hi;
        split(part[0], lo, hi);
        sum += lo + hi;
    }
    __device__ __forceinline__ Softmax done() const { return Softmax{top, sum * exp2_of(-ex.shift)}; }
};
// Elements of a vector as scores; those beside the row's own are -inf.
template <typename T, int VEC, typename SPAN>
__device__ __forceinline__ void scores(const SPAN& span, int v, const RawVec<T, VEC>& raw, float (&z)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) z[e] = raw.get(e);
    if (span.any(v) && span.whole(v)) return;
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (!span.any(v) || e < span.lo(v) || e >= span.hi(v)) z[e] = -INFINITY;
}

}  // namespace circ
