// Group norm with an activation on channel-last tensors [N][pixels][C]: over the m = pixels D values of an image and a group of D channels
//   mean, variance = mean((x - mean)^2), rstd = 1 / sqrt(variance + eps), v = gain_c (x - mean) rstd + bias_c, y = act(v)
// and its gradients, with u = (x - mean) rstd and g = grad_y act'(v):
//   grad_x = rstd (gain g - (A + u B) / m), A = sum of gain g over the group, B = sum of gain g u
//   grad_gain_c = sum of g u, grad_bias_c = sum of g over images and pixels.
#include <algorithm>
#include <new>
#include <type_traits>

#include "circ_rows.cuh"

namespace circ {

struct Gnorm {
    int device;
    int channels, groups;
    float eps;
    int x_dtype, y_dtype, act;
    Scratch ws;
    long images_held;       // that the workspace is laid out for
};

struct GnormArgs {
    const float *gain, *bias;
    float *mean, *rstd;       // [N][groups]
    int channels, groups, depth;      // depth: channels a group
    int images, pixels;
    float eps;
    double inv_m, inv_depth;  // 1 / (pixels depth), 1 / depth
    // a block's part: `columns` vectors of channels (all, or a tile of them), and pixels of one image
    int columns, tiles, pieces, per;
    int act;
    // workspace
    unsigned* arrived;        // [N] parts of an image that are summed up (0 before and after a call)
    double2* group_parts;     // [N][pieces][groups] the pieces' sums of the groups
    float2* parts;            // [N][pieces][C] forward: mean, less the channel's first value, and sum of squares around it; backward: sum of g, of g u
    float2* means;            // [N][groups] backward: A / m, B / m
};

constexpr int kGnormThreads = 256;

// 1 / (1 + exp(-v)): one exponential, one reciprocal.  Below -87 the exponential is infinite and the sigmoid 0.  The exponent is a rounded product, which costs |v| 2^-24 of the
// result, as much as rounding v itself.
__device__ __forceinline__ float sigmoid_of(float v) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}

template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if constexpr (ACT == CIRC_ACT_RELU) return max_nan(v, 0.f);
    if constexpr (ACT == CIRC_ACT_SILU) return v * sigmoid_of(v);
    return v;
}

template <typename F>
__device__ __forceinline__ void with_act_of(int act, F&& f) {
    if (act == CIRC_ACT_RELU) f(std::integral_constant<int, CIRC_ACT_RELU>{});
    else if (act == CIRC_ACT_SILU) f(std::integral_constant<int, CIRC_ACT_SILU>{});
    else f(std::integral_constant<int, CIRC_ACT_NONE>{});
}

// Values that a thread adds up in float32 at a time (and up to a round of loads more); the sums of longer walks are joined in float64, so that what rounding
// costs does not grow with the pixels.  A walk's squares are taken around the mean of its first values (at most kPivot), those of later runs around the mean so
// far: a value far from the others in the first place is lost in neither.  (Variance of 264 normal values, the first 100 deviations out: relative error 5e-6 at most
// in 60 draws, 3e-4 around the first one alone; 3e-3 and more without runs from 12800 values on.)
constexpr int kRun = 256;
constexpr int kPivot = 8;
// The mean of some values, less a reference, and the sum of squares around the mean.
struct Moments {
    double mean, m2;
    // Those of n values (`inv`: 1 / n) whose sums around `pivot` (less the reference) are s1 and s2.
    __device__ __forceinline__ static Moments of(double inv, double pivot, float s1, float s2) {
        const double d = (double)s1 * inv;
        return Moments{pivot + d, (double)s2 - (double)s1 * d};
    }
    // Both: of n0 values, and of n1 more that are `part` of all.
    __device__ __forceinline__ static Moments join(double n0, Moments a, double part, Moments b) {
        const double d = b.mean - a.mean;
        return Moments{a.mean + d * part, a.m2 + b.m2 + d * d * (n0 * part)};
    }
};
// The sum of squares around the mean, in float32; squares beyond its range stay +inf.
__device__ __forceinline__ float around_mean(float s1, float s2, float inv) { return s2 == INFINITY ? s2 : s2 - s1 * s1 * inv; }
// A float64 value in the place of two float32 ones.
__device__ __forceinline__ float2 as_float2(double v) { return make_float2(__int_as_float(__double2loint(v)), __int_as_float(__double2hiint(v))); }
__device__ __forceinline__ double as_double(float2 v) { return __hiloint2double(__float_as_int(v.y), __float_as_int(v.x)); }

// What a channel's values go through: v = (x - mean) (rstd gain) + bias.
struct Channel {
    float mean, rstd, gain, bias;
    __device__ __forceinline__ float unit(float x) const { return (x - mean) * rstd; }
    // act'(v) for a value.  Which side of 0 a value lies on does not depend on rounding: near it the sign comes from float64.
    template <int ACT>
    __device__ __forceinline__ float slope(float x, float u) const {
        if constexpr (ACT == CIRC_ACT_RELU) {
            const float t = u * gain, v = t + bias;
            if (fabsf(v) <= 1e-6f * (fabsf(t) + fabsf(bias)))
                return ((double)x - (double)mean) * ((double)rstd * (double)gain) + (double)bias > 0.0 ? 1.f : 0.f;
            return v > 0.f ? 1.f : v != v ? v : 0.f;
        }
        if constexpr (ACT == CIRC_ACT_SILU) {
            const float v = fmaf(u, gain, bias), s = sigmoid_of(v);
            return s * fmaf(v, 1.f - s, 1.f);
        }
        return 1.f;
    }
};

// Whether v is above 0.  A call for single channels: in line, its registers cost the other activations of the same kernels (SiLU gradient of 32 x 56 x 56 x 255
// bfloat16: 102 us, and 93 with the call; ReLU 112 and 120, and 149 with float64 for every value).
__device__ __noinline__ bool above_zero(float x, float mean, float rstd, float gain, float bias) {
    return ((double)x + (double)mean) * ((double)rstd * (double)gain) + (double)bias > 0.0;
}
// The same for a vector of channels, arithmetic in pairs.
template <int VEC>
struct Channels {
    static constexpr int N = VEC > 1 ? VEC / 2 : 1;
    Pair mean[N], rstd[N], gain[N], bias[N];       // mean: less than 0
    __device__ __forceinline__ void set(int e, float m, float r, float g, float b) {
        put(mean[e / 2], e % 2, -m);
        put(rstd[e / 2], e % 2, r);
        put(gain[e / 2], e % 2, g);
        put(bias[e / 2], e % 2, b);
    }
    __device__ __forceinline__ static void put(Pair& p, int half, float v) {
        float lo, hi;
        split(p, lo, hi);
        p = half ? pair_of(lo, v) : pair_of(v, VEC > 1 ? hi : 0.f);
    }
    // u and g = grad_y act'(v) of two values.
    template <int ACT>
    __device__ __forceinline__ void slopes(int i, Pair x, Pair grad_y, Pair& u, Pair& g) const {
        u = pair_mul(pair_add(x, mean[i]), rstd[i]);
        g = grad_y;
        if constexpr (ACT == CIRC_ACT_NONE) return;
        const Pair t = pair_mul(u, gain[i]), v = pair_add(t, bias[i]);
        float v0, v1;
        split(v, v0, v1);
        if constexpr (ACT == CIRC_ACT_RELU) {
            float t0, t1, b0, b1, g0, g1;
            split(t, t0, t1);
            split(bias[i], b0, b1);
            split(g, g0, g1);
            // near 0 the sides come from float64
            auto near = [](float v, float t, float b) { return fabsf(v) <= 1e-6f * (fabsf(t) + fabsf(b)); };
            bool on0 = v0 > 0.f, on1 = v1 > 0.f;
            if (near(v0, t0, b0) || (VEC > 1 && near(v1, t1, b1))) {
                float x0, x1, m0, m1, r0, r1, a0, a1;
                split(x, x0, x1);
                split(mean[i], m0, m1);
                split(rstd[i], r0, r1);
                split(gain[i], a0, a1);
                if constexpr (VEC == 1) {
                    on0 = above_zero(x0, m0, r0, a0, b0);
                } else {
                    on0 = ((double)x0 + (double)m0) * ((double)r0 * (double)a0) + (double)b0 > 0.0;
                    on1 = ((double)x1 + (double)m1) * ((double)r1 * (double)a1) + (double)b1 > 0.0;
                }
            }
            g0 = on0 ? g0 : v0 != v0 ? v0 : 0.f;
            if constexpr (VEC > 1) g1 = on1 ? g1 : v1 != v1 ? v1 : 0.f;
            g = pair_of(g0, VEC > 1 ? g1 : 0.f);
        } else {
            const Pair s = pair_of(sigmoid_of(v0), VEC > 1 ? sigmoid_of(v1) : 0.f), one = pair_of(1.f, 1.f);
            g = pair_mul(g, pair_mul(s, pair_fma(v, pair_fma(s, pair_of(-1.f, -1.f), one), one)));
        }
    }
};

// ---- any tensor: a thread a channel, two launches ----
// Which channel and which pixels a thread works on.
struct GnormPlace {
    int image, piece, tile, column, lane, lanes, from, to;      // pixels from + lane, + lanes, ... below `to`
    bool live;
    __device__ __forceinline__ explicit GnormPlace(const GnormArgs& a) {
        const int part = blockIdx.x % (a.pieces * a.tiles);
        image = blockIdx.x / (a.pieces * a.tiles);
        piece = part / a.tiles;
        tile = part % a.tiles;
        lanes = kGnormThreads / a.columns;
        lane = threadIdx.x / a.columns;
        column = tile * a.columns + threadIdx.x % a.columns;
        from = piece * a.per;
        to = min(a.pixels, from + a.per);
        live = lane < lanes && column < a.channels;
    }
    __device__ __forceinline__ size_t at(const GnormArgs& a, int pixel) const { return ((size_t)image * a.pixels + pixel) * a.channels + column; }
    __device__ __forceinline__ Channel channel(const GnormArgs& a) const {
        const size_t g = (size_t)image * a.groups + column / a.depth;
        return Channel{a.mean[g], a.rstd[g], a.gain ? a.gain[column] : 1.f, a.bias ? a.bias[column] : 0.f};
    }
};

// The block that is last to finish an image's parts.  All threads call it.
__device__ __forceinline__ bool last_of_image(const GnormArgs& a, int image) {
    __shared__ bool last;
    __syncthreads();
    if (a.pieces * a.tiles == 1) return true;
    if (threadIdx.x == 0) {
        __threadfence();
        const unsigned parts = (unsigned)(a.pieces * a.tiles);
        last = atomicAdd(a.arrived + image, 1u) == parts - 1;
        if (last) a.arrived[image] = 0;
    }
    __syncthreads();
    if (last) __threadfence();
    return last;
}

// Sums over `entries` entries for every group, by a warp each, or the block for few groups: term(group, entry) -> double2, f(group, sum).
template <typename TERM, typename F>
__device__ __forceinline__ void over_groups(const GnormArgs& a, int entries, TERM term, F f) {
    __shared__ double2 red[kGnormThreads / 32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = kGnormThreads / 32;
    const bool wide = a.groups < warps;
    for (int g = wide ? 0 : warp; g < a.groups; g += wide ? 1 : warps) {
        double2 s = make_double2(0.0, 0.0);
#pragma unroll 4
        for (int i = wide ? threadIdx.x : lane; i < entries; i += wide ? kGnormThreads : 32) {
            const double2 v = term(g, i);
            s.x += v.x;
            s.y += v.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
            s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
        }
        if (wide) {
            __syncthreads();
            if (lane == 0) red[warp] = s;
            __syncthreads();
            s = red[0];
            for (int w = 1; w < warps; ++w) {
                s.x += red[w].x;
                s.y += red[w].y;
            }
        }
        if (wide ? threadIdx.x == 0 : lane == 0) f(g, s);
    }
}

// Means are kept as differences from the channel's first value in the image, so that a large offset costs no digits, until they are joined in float64.
// LONG: some threads have more than kRun pixels.
template <typename T, bool LONG>
__global__ void __launch_bounds__(kGnormThreads) gnorm_any_stats_kernel(const T* __restrict__ x, GnormArgs a) {
    __shared__ float2 sums[kGnormThreads];
    __shared__ Moments totals[LONG ? kGnormThreads : 1];      // of a thread's runs that are done
    pdl_begin();
    const GnormPlace at(a);
    if (at.live) {
        const float first = to_float(x[at.at(a, 0)]);
        const int p0 = at.from + at.lane;
        float pivot = 0.f, s1 = 0.f, s2 = 0.f, head[kPivot];
        auto take = [&](float v) {
            const float d = v - pivot;
            s1 += d;
            s2 = fmaf(d, d, s2);
        };
        int n = 0, before = 0;      // values of the run, and of those before it
#pragma unroll
        for (int i = 0; i < kPivot; ++i) {
            head[i] = p0 + i * at.lanes < at.to ? to_float(x[at.at(a, p0 + i * at.lanes)]) : 0.f;
            pivot += head[i];
            n += p0 + i * at.lanes < at.to;
        }
        pivot *= n ? 1.f / (float)n : 0.f;
#pragma unroll
        for (int i = 0; i < kPivot; ++i)
            if (i < n) take(head[i]);
        int p = p0 + kPivot * at.lanes;
        if constexpr (LONG) {
            auto fold = [&]() {
                Moments all = Moments::of(1.0 / n, (double)pivot - (double)first, s1, s2);
                if (before) all = Moments::join(before, totals[threadIdx.x], (double)n / (double)(before + n), all);
                totals[threadIdx.x] = all;
                before += n;
            };
            while (p < at.to) {
                const int end = min(at.to, p + (kRun - n) * at.lanes);
#pragma unroll 4
                for (; p < end; p += at.lanes, ++n) take(to_float(x[at.at(a, p)]));
                if (p >= at.to) break;
                fold();
                pivot = (float)(totals[threadIdx.x].mean + (double)first);
                s1 = s2 = 0.f;
                n = 0;
            }
            if (before) fold();
        } else {
#pragma unroll 4
            for (; p < at.to; p += at.lanes, ++n) take(to_float(x[at.at(a, p)]));
        }
        if (LONG && before) {
            sums[threadIdx.x] = make_float2((float)totals[threadIdx.x].mean, (float)totals[threadIdx.x].m2);
        } else {
            const float inv = n ? 1.f / (float)n : 0.f;
            sums[threadIdx.x] = make_float2(fmaf(s1, inv, pivot - first), around_mean(s1, s2, inv));
        }
    }
    __syncthreads();
    const int c = at.tile * a.columns + threadIdx.x;
    if ((int)threadIdx.x < a.columns && c < a.channels) {
        auto pixels = [&](int l) { return (at.to - at.from - l + at.lanes - 1) / at.lanes; };
        float count = (float)pixels(0), mean = sums[threadIdx.x].x, m2 = sums[threadIdx.x].y;
        for (int l = 1; l < at.lanes && pixels(l) > 0; ++l) {
            const float2 v = sums[l * a.columns + threadIdx.x];
            const float mine = (float)pixels(l), all = count + mine, d = v.x - mean, part = mine / all;
            mean = fmaf(d, part, mean);
            m2 += v.y + d * d * count * part;
            count = all;
        }
        a.parts[((size_t)at.image * a.pieces + at.piece) * a.channels + c] = make_float2(mean, m2);
    }
    if (!last_of_image(a, at.image)) return;
    const T* first = x + (size_t)at.image * a.pixels * a.channels;
    over_groups(a, a.pieces * a.depth,
                [&](int g, int i) {
                    const int piece = i / a.depth, c0 = g * a.depth, k = c0 + i - piece * a.depth;
                    const float2 v = __ldcg(a.parts + ((size_t)at.image * a.pieces + piece) * a.channels + k);
                    const double n = (double)(min(a.pixels, (piece + 1) * a.per) - piece * a.per);
                    const double d = (double)v.x + ((double)to_float(first[k]) - (double)to_float(first[c0]));
                    return make_double2(n * d, (double)v.y + n * d * d);
                },
                [&](int g, double2 s) {
                    const double mean = s.x * a.inv_m, var = s.y * a.inv_m - mean * mean;
                    a.mean[(size_t)at.image * a.groups + g] = (float)(mean + (double)to_float(first[g * a.depth]));
                    a.rstd[(size_t)at.image * a.groups + g] = 1.f / sqrtf((var < 0.0 ? 0.f : (float)var) + a.eps);
                });
}
template <typename T, typename U>
__global__ void __launch_bounds__(kGnormThreads) gnorm_any_apply_kernel(const T* x, U* y, GnormArgs a) {
    pdl_begin();
    const GnormPlace at(a);
    if (!at.live) return;
    const Channel c = at.channel(a);
    const float scale = c.rstd * c.gain;
    with_act_of(a.act, [&](auto act) {
#pragma unroll 4
        for (int p = at.from + at.lane; p < at.to; p += at.lanes)
            store_one(y + at.at(a, p), activate<decltype(act)::value>(fmaf(to_float(x[at.at(a, p)]) - c.mean, scale, c.bias)));
    });
}
template <typename T, typename U, bool LONG>
__global__ void __launch_bounds__(kGnormThreads) gnorm_any_sums_kernel(const T* __restrict__ x, const U* __restrict__ grad_y, GnormArgs a) {
    __shared__ float2 sums[kGnormThreads];
    pdl_begin();
    const GnormPlace at(a);
    if (at.live) {
        const Channel ch = at.channel(a);
        float s1 = 0.f, s2 = 0.f;
        double2 all = make_double2(0.0, 0.0);       // of the runs that are done
        with_act_of(a.act, [&](auto act) {
            int p = at.from + at.lane;
            for (;;) {
                const int end = LONG ? min(at.to, p + kRun * at.lanes) : at.to;
#pragma unroll 4
                for (; p < end; p += at.lanes) {
                    const float v = to_float(x[at.at(a, p)]), u = ch.unit(v), g = to_float(grad_y[at.at(a, p)]) * ch.template slope<decltype(act)::value>(v, u);
                    s1 += g;
                    s2 = fmaf(g, u, s2);
                }
                if (!LONG) break;
                all.x += (double)s1;
                all.y += (double)s2;
                s1 = s2 = 0.f;
                if (p >= at.to) break;
            }
        });
        sums[threadIdx.x] = LONG ? make_float2((float)all.x, (float)all.y) : make_float2(s1, s2);
    }
    __syncthreads();
    const int c = at.tile * a.columns + threadIdx.x;
    if ((int)threadIdx.x < a.columns && c < a.channels) {
        float2 s = make_float2(0.f, 0.f);
        for (int l = 0; l < at.lanes; ++l) {
            s.x += sums[l * a.columns + threadIdx.x].x;
            s.y += sums[l * a.columns + threadIdx.x].y;
        }
        a.parts[((size_t)at.image * a.pieces + at.piece) * a.channels + c] = s;
    }
    if (!last_of_image(a, at.image)) return;
    over_groups(a, a.pieces * a.depth,
                [&](int g, int i) {
                    const int piece = i / a.depth, k = g * a.depth + i - piece * a.depth;
                    const float2 v = __ldcg(a.parts + ((size_t)at.image * a.pieces + piece) * a.channels + k);
                    const double gain = a.gain ? (double)a.gain[k] : 1.0;
                    return make_double2(gain * v.x, gain * v.y);
                },
                [&](int g, double2 s) { a.means[(size_t)at.image * a.groups + g] = make_float2((float)(s.x * a.inv_m), (float)(s.y * a.inv_m)); });
}
template <typename T, typename U>
__global__ void __launch_bounds__(kGnormThreads) gnorm_any_grad_kernel(const T* x, const U* grad_y, T* grad_x, GnormArgs a) {
    pdl_begin();
    const GnormPlace at(a);
    if (!at.live) return;
    const Channel ch = at.channel(a);
    const float2 m = a.means[(size_t)at.image * a.groups + at.column / a.depth];
    with_act_of(a.act, [&](auto act) {
#pragma unroll 4
        for (int p = at.from + at.lane; p < at.to; p += at.lanes) {
            const float v = to_float(x[at.at(a, p)]), u = ch.unit(v), g = to_float(grad_y[at.at(a, p)]) * ch.template slope<decltype(act)::value>(v, u);
            store_one(grad_x + at.at(a, p), ch.rstd * (fmaf(g, ch.gain, -m.x) - u * m.y));
        }
    });
}

// ---- tensors up to 256 vectors of channels wide ----
// Two launches: the sums of pieces of the images (the block that is last to finish an image's joins them), and the output, which goes the same way back: what
// was read last is still in L2.  A thread has one vector of channels, its constants in registers, and R pixels on their way at a time.
// 32 x 112 x 112 x 256 bfloat16 with SiLU take 118 us: the sums read 206 MB at 5.1 TB/s (40 us), the output reads and writes 411 at 5.4, with the XU pipe
// 69 % busy (two of its instructions an element).  The gradients of 64 x 56 x 56 x 256 take 110 us, 4 XU instructions an element.  Small calls are two
// launches (10 us with the call), or one where a block has a whole image.  (Rounds of one pixel a thread for few images, so that more blocks share them, were slower in 86 of
// 176 sizes, up to 65 %, and faster in 7, up to 9 %.)
// (One launch, whose blocks took sums and outputs from a counter and waited for an image's sums, read every image once, but an image's counting, waiting
// and joining by small tasks cost more than the second reading: 145 us for 32 x 112 x 112 x 256 bfloat16.)
// A piece takes every pieces-th round of `per` pixels (R of each thread): the blocks that run at once read neighbouring memory.
struct PieceSize {
    int full, rest;      // whole rounds, and pixels of one that is not
    __device__ __forceinline__ PieceSize(const GnormArgs& a, int piece) {
        const int whole = a.pixels / a.per;
        full = piece < whole ? (whole - piece + a.pieces - 1) / a.pieces : 0;
        rest = whole % a.pieces == piece ? a.pixels - whole * a.per : 0;
    }
    __device__ __forceinline__ int pixels(const GnormArgs& a) const { return full * a.per + rest; }
};
template <int VEC>
struct Stretch {
    int image, piece, lanes, lane, column;
    PieceSize size;
    int last, mine;           // this thread's pixels: of the round that is not whole, and all
    bool live;
    size_t at, step, jump;    // element of the first, between two pixels, between two rounds
    __device__ __forceinline__ Stretch(const GnormArgs& a, unsigned block, int r) : size(a, block % a.pieces) {
        image = block / a.pieces;
        piece = block % a.pieces;
        lanes = kGnormThreads / a.columns;
        lane = threadIdx.x / a.columns;
        column = threadIdx.x % a.columns;
        live = lane < lanes;
        last = live ? (size.rest - lane + lanes - 1) / lanes : 0;
        mine = live ? size.full * r + last : 0;
        at = ((size_t)image * a.pixels + (size_t)piece * a.per + lane) * a.channels + (size_t)column * VEC;
        step = (size_t)lanes * a.channels;
        jump = (size_t)a.pieces * a.per * a.channels;
    }
};
// Sums over an image's parts for every group: f(group, sum of x-terms, sum of y-terms), in float64.  `red`: [kGnormThreads] double2.
template <typename TERM, typename F>
__device__ __forceinline__ void join_groups(const GnormArgs& a, int image, double2* red, TERM term, F f) {
    const int wide = min(a.groups, kGnormThreads), rows = kGnormThreads / wide, r = threadIdx.x / wide;
    for (int g0 = 0; g0 < a.groups; g0 += wide) {
        const int g = g0 + threadIdx.x % wide;
        double2 s = make_double2(0.0, 0.0);
        if (r < rows && g < a.groups) {
            const double2* p = a.group_parts + (size_t)image * a.pieces * a.groups + g;
#pragma unroll 4
            for (int t = r; t < a.pieces; t += rows) {
                const double2 v = term(t, __ldcg(p + (size_t)t * a.groups));
                s.x += v.x;
                s.y += v.y;
            }
        }
        __syncthreads();
        red[threadIdx.x] = s;
        __syncthreads();
        if (r == 0 && g < a.groups) {
            for (int i = 1; i < rows; ++i) {
                s.x += red[i * wide + threadIdx.x].x;
                s.y += red[i * wide + threadIdx.x].y;
            }
            f(g, s);
        }
    }
}
// Every group's channels in shared memory, by as many lanes of a warp as there are channels in one: f(group, lane of that many, their number, whether
// the group is one).
template <typename F>
__device__ __forceinline__ void each_group(const GnormArgs& a, F f) {
    int shift = 0;
    while (1 << shift < a.depth && shift < 5) ++shift;
    for (int g0 = 0; g0 < a.groups; g0 += kGnormThreads >> shift) {
        const int g = g0 + (threadIdx.x >> shift);
        f(g, threadIdx.x & ((1 << shift) - 1), 1 << shift, g < a.groups);
    }
}
template <typename T>
__device__ __forceinline__ T lanes_sum(T v, int wide) {
    for (int o = wide / 2; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename T, int VEC>
__device__ __forceinline__ Pair two(const RawVec<T, VEC>& r, int i) {
    if constexpr (VEC > 1) return r.get2(2 * i);
    else return pair_of(r.get(0), 0.f);
}
__device__ __forceinline__ float half(Pair p, int e) {
    float lo, hi;
    split(p, lo, hi);
    return e % 2 ? hi : lo;
}
// The threads' sums of a channel lie `columns` apart and those of a vector's elements a block's threads apart, so that neither side's accesses meet in a
// bank.  Calls f(channel, element, column) for a block's channels, by one thread each.
template <int VEC, typename F>
__device__ __forceinline__ void each_channel(const GnormArgs& a, F f) {
    for (int i = threadIdx.x; i < a.channels; i += kGnormThreads) {
        const int e = i / a.columns, column = i - e * a.columns;
        f(column * VEC + e, e, column);
    }
}
// Calls load(i, element) for a thread's pixels, R at a time, and take(i, element) for each of them behind.  BACK: from the last round to the first.
// start(pixels) (STARTS): between the first round's loads and takes, with its number of pixels.  fold(pixels) (FOLDS): between every kRun pixels and more, with
// the number of those before them.
template <int R, bool BACK, bool STARTS, bool FOLDS, int VEC, typename LOAD, typename TAKE, typename START, typename FOLD>
__device__ __forceinline__ void walk_pixels(const Stretch<VEC>& st, LOAD load, TAKE take, START start, FOLD fold) {
    auto rest = [&]() {
        if (st.last <= 0) return;
        const size_t at = st.at + st.size.full * st.jump;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < st.last) load(i, at + i * st.step);
        if (STARTS && st.size.full == 0) start(st.last);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < st.last) take(i, at + i * st.step);
    };
    auto round = [&](int n, bool head) {
        const size_t at = st.at + (BACK ? st.size.full - 1 - n : n) * st.jump;
#pragma unroll
        for (int i = 0; i < R; ++i) load(i, at + i * st.step);
        if (head) start(R);
#pragma unroll
        for (int i = 0; i < R; ++i) take(i, at + i * st.step);
    };
    if (BACK) rest();
    int n = 0;
    if (STARTS && n < st.size.full) round(n++, true);
    for (;;) {
        const int end = FOLDS ? min(st.size.full, (n + kRun / R) / (kRun / R) * (kRun / R)) : st.size.full;
        for (; n < end; ++n) round(n, false);
        if (!FOLDS || n >= st.size.full) break;
        fold(n * R - kRun);
    }
    if (!BACK) rest();
}
template <int R, bool BACK, int VEC, typename LOAD, typename TAKE>
__device__ __forceinline__ void walk_pixels(const Stretch<VEC>& st, LOAD load, TAKE take) {
    walk_pixels<R, BACK, false, false>(st, load, take, [](int) {}, [](int) {});
}
// Pixels of a walk that fold() is called for.
template <int R, int VEC>
__device__ __forceinline__ int folded_pixels(const Stretch<VEC>& st) {
    return st.size.full > 0 ? (st.size.full - 1) / (kRun / R) * kRun : 0;
}

// VEC channels' values of a vector of one a channel (NULL: `none`), and of one a group.
template <int VEC>
__device__ __forceinline__ void of_channels(const float* p, int c, float none, float (&v)[VEC]) {
    if (VEC >= 4 && p && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
        for (int e = 0; e + 3 < VEC; e += 4) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p + c + e));
            v[e] = f.x; v[e + 1] = f.y; v[e + 2] = f.z; v[e + 3] = f.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = p ? __ldg(p + c + e) : none;
}
template <int VEC, typename V, typename F>
__device__ __forceinline__ void of_groups(const GnormArgs& a, const Stretch<VEC>& st, const V* p, F set) {
    p += (size_t)st.image * a.groups;
    const int c = st.column * VEC, g = c / a.depth;
    if (a.depth % VEC == 0) {
        const V v = p[g];
#pragma unroll
        for (int e = 0; e < VEC; ++e) set(e, v);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) set(e, p[(c + e) / a.depth]);
    }
}
template <int VEC>
__device__ __forceinline__ void load_channels(const GnormArgs& a, const Stretch<VEC>& st, Channels<VEC>& ch) {
    float gain[VEC], bias[VEC], mean[VEC], rstd[VEC];
    of_channels<VEC>(a.gain, st.column * VEC, 1.f, gain);
    of_channels<VEC>(a.bias, st.column * VEC, 0.f, bias);
    of_groups<VEC>(a, st, a.mean, [&](int e, float v) { mean[e] = v; });
    of_groups<VEC>(a, st, a.rstd, [&](int e, float v) { rstd[e] = v; });
#pragma unroll
    for (int e = 0; e < VEC; ++e) ch.set(e, mean[e], rstd[e], gain[e], bias[e]);
}

template <typename T, typename U, int VEC, int R>
__device__ __forceinline__ void apply_stretch(const T* x, U* y, const GnormArgs& a, const Stretch<VEC>& st) {
    if (!st.live) return;
    Channels<VEC> ch;
    load_channels(a, st, ch);
#pragma unroll
    for (int k = 0; k < Channels<VEC>::N; ++k) ch.rstd[k] = pair_mul(ch.rstd[k], ch.gain[k]);
    with_act_of(a.act, [&](auto act) {
        RawVec<T, VEC> raw[R];
        walk_pixels<R, true>(st, [&](int i, size_t o) { raw[i].load(x + o); },
                       [&](int i, size_t o) {
                           float v[VEC > 1 ? VEC : 2], out[VEC];
#pragma unroll
                           for (int k = 0; k < Channels<VEC>::N; ++k)
                               split(pair_fma(pair_add(two(raw[i], k), ch.mean[k]), ch.rstd[k], ch.bias[k]), v[2 * k], v[2 * k + 1]);
#pragma unroll
                           for (int e = 0; e < VEC; ++e) out[e] = activate<decltype(act)::value>(v[e]);
                           store_vec_once<VEC>(y + o, out);
                       });
    });
}

// A piece's sums: a thread's (see kRun; what came before a run waits in shared memory), those of the threads that share a channel, and those of a group's
// channels, each around their joint mean.  Means are kept as differences from the image's first pixel, so that a large offset costs no digits, and joined in float64, so
// that a mean that is small beside that pixel keeps its own: each thread's is off by 2^-24 of the difference, and those errors average out.
// WHOLE: a block has a whole image, and writes its output too.  LONG: some threads have more than kRun pixels (a kernel of its own: its registers cost the
// others 2 to 9 %).
template <typename T, typename U, int VEC, int R, bool WHOLE, bool LONG>
__global__ void __launch_bounds__(kGnormThreads, 3) gnorm_stats_kernel(const T* x, U* y, GnormArgs a) {
    constexpr int N = Channels<VEC>::N;
    static_assert(R <= kPivot && kRun % R == 0, "");
    __shared__ float2 sums[kGnormThreads * VEC], joined[kGnormThreads * VEC];
    __shared__ float firsts[kGnormThreads * VEC];
    __shared__ double2 red[kGnormThreads];
    pdl_begin();
    const Stretch<VEC> st(a, blockIdx.x, R);
    const T* first = x + (size_t)st.image * a.pixels * a.channels;
    if (st.live) {
        RawVec<T, VEC> raw[R], zero;
        Pair pivot[N], s1[N], s2[N];       // pivot: less than 0
#pragma unroll
        for (int i = 0; i < N; ++i) pivot[i] = s1[i] = s2[i] = pair_of(0.f, 0.f);
        // values around `p` joined to those before, of which the thread's shared words have the moments
        auto joined_run = [&](int before, double inv, double part, float f, float p, float sum, float square, int e) {
            const Moments run = Moments::of(inv, (double)p - (double)f, sum, square);
            if (before == 0) return run;
            const int at = e * kGnormThreads + threadIdx.x;
            return Moments::join(before, Moments{as_double(sums[at]), as_double(joined[at])}, part, run);
        };
        walk_pixels<R, false, true, LONG>(st, [&](int i, size_t o) { raw[i].load(x + o); },
                       [&](int i, size_t) {
#pragma unroll
                           for (int k = 0; k < N; ++k) {
                               const Pair d = pair_add(two(raw[i], k), pivot[k]);
                               s1[k] = pair_add(s1[k], d);
                               s2[k] = pair_fma(d, d, s2[k]);
                           }
                       },
                       [&](int n) {
                           const float inv = -1.f / (float)n;
#pragma unroll
                           for (int i = 0; i < R; ++i)
                               if (i < n)
#pragma unroll
                                   for (int k = 0; k < N; ++k) pivot[k] = pair_add(pivot[k], two(raw[i], k));
#pragma unroll
                           for (int k = 0; k < N; ++k) pivot[k] = pair_mul(pivot[k], pair_of(inv, inv));
                       },
                       [&](int before) {
                           zero.load(first + st.column * VEC);
                           const double part = (double)kRun / (double)(before + kRun);
#pragma unroll
                           for (int e = 0; e < VEC; ++e) {
                               const Moments m = joined_run(before, 1.0 / kRun, part, zero.get(e), -half(pivot[e / 2], e), half(s1[e / 2], e), half(s2[e / 2], e), e);
                               sums[e * kGnormThreads + threadIdx.x] = as_float2(m.mean);
                               joined[e * kGnormThreads + threadIdx.x] = as_float2(m.m2);
                               Channels<VEC>::put(pivot[e / 2], e % 2, -(float)(m.mean + (double)zero.get(e)));
                           }
#pragma unroll
                           for (int i = 0; i < N; ++i) s1[i] = s2[i] = pair_of(0.f, 0.f);
                       });
        zero.load(first + st.column * VEC);
        const int before = LONG ? folded_pixels<R>(st) : 0;
        const float inv = st.mine > 0 ? 1.f / (float)st.mine : 0.f;
        double inv_run = 0.0, part = 0.0;
        if (before > 0) {
            inv_run = 1.0 / (double)(st.mine - before);
            part = (double)(st.mine - before) / (double)st.mine;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float f = zero.get(e), p = -half(pivot[e / 2], e), sum = half(s1[e / 2], e), square = half(s2[e / 2], e);
            float2 both;
            if (before > 0) {
                const Moments m = joined_run(before, inv_run, part, f, p, sum, square, e);
                both = make_float2((float)m.mean, (float)m.m2);
            } else {
                both = make_float2(fmaf(sum, inv, p - f), around_mean(sum, square, inv));
            }
            sums[e * kGnormThreads + threadIdx.x] = both;
            if (st.lane == 0) firsts[st.column * VEC + e] = f;
        }
    }
    const int here = st.size.pixels(a), least = st.size.full * R + st.size.rest / st.lanes, more = st.size.rest % st.lanes;      // pixels of lane l: least + (l < more)
    const double inv_here = 1.0 / (double)here, some = (double)least;
    const int lanes = least > 0 ? st.lanes : more;      // that have pixels
    __syncthreads();
    // A channel's mean goes to its first thread's place, which no other channel reads, in float64.
    each_channel<VEC>(a, [&](int c, int e, int column) {
        float2* v = sums + e * kGnormThreads + column;
        double part[4] = {};      // (chains that do not wait for one another, and loads that go together)
        auto take = [&](int l, int u) { part[u] = fma(l < more ? some + 1.0 : some, (double)v[l * a.columns].x, part[u]); };
        int l = 0;
        for (; l + 4 <= lanes; l += 4)
#pragma unroll
            for (int u = 0; u < 4; ++u) take(l + u, u);
        for (; l < lanes; ++l) take(l, 0);
        const double mean = ((part[0] + part[1]) + (part[2] + part[3])) * inv_here;
        const float near = (float)mean;
        float q = 0.f;
#pragma unroll 4
        for (int l = 0; l < lanes; ++l) {
            const float2 one = v[l * a.columns];
            const float d = one.x - near;
            q += fmaf(d * d, (float)(least + (l < more)), one.y);
        }
        v[0] = as_float2(mean);
        joined[c].y = q;
    });
    __syncthreads();
    each_group(a, [&](int g, int l, int wide, bool one) {
        const int c0 = g * a.depth, end = one ? a.depth : 0;
        const double f = one ? (double)firsts[c0] : 0.0;
        auto mean_of = [&](int c) { return as_double(sums[c % VEC * kGnormThreads + c / VEC]) + ((double)firsts[c] - f); };
        double s = 0.0;
        float q = 0.f;
        for (int i = l; i < end; i += wide) s += mean_of(c0 + i);
        const double mean = lanes_sum(s, wide) * a.inv_depth;
        for (int i = l; i < end; i += wide) {
            const float d = (float)(mean_of(c0 + i) - mean);
            q += fmaf(d * d, (float)here, joined[c0 + i].y);
        }
        q = lanes_sum(q, wide);
        if (one && l == 0) a.group_parts[((size_t)st.image * a.pieces + st.piece) * a.groups + g] = make_double2(mean, (double)q);
    });
    if (!last_of_image(a, st.image)) return;
    join_groups(a, st.image, red,
                [&](int t, double2 v) {
                    const double k = (double)PieceSize(a, t).pixels(a) * a.depth, mean = v.x;
                    return make_double2(k * mean, v.y + k * mean * mean);
                },
                [&](int g, double2 s) {
                    const double mean = s.x * a.inv_m, var = s.y * a.inv_m - mean * mean;
                    a.mean[(size_t)st.image * a.groups + g] = (float)(mean + (double)to_float(first[g * a.depth]));
                    a.rstd[(size_t)st.image * a.groups + g] = 1.f / sqrtf((var < 0.0 ? 0.f : (float)var) + a.eps);
                });
    if constexpr (WHOLE) {
        __syncthreads();
        apply_stretch<T, U, VEC, R>(x, y, a, st);
    }
}

template <typename T, typename U, int VEC, int R>
__global__ void __launch_bounds__(kGnormThreads, 3) gnorm_apply_kernel(const T* x, U* y, GnormArgs a) {
    pdl_begin();
    apply_stretch<T, U, VEC, R>(x, y, a, Stretch<VEC>(a, gridDim.x - 1 - blockIdx.x, R));
}

template <typename T, typename U, int VEC, int R>
__device__ __forceinline__ void grad_stretch(const T* x, const U* grad_y, T* grad_x, const GnormArgs& a, const Stretch<VEC>& st) {
    constexpr int N = Channels<VEC>::N;
    if (!st.live) return;
    Channels<VEC> ch;
    load_channels(a, st, ch);
    Pair mean_a[N], mean_b[N];       // less than 0
    of_groups<VEC>(a, st, a.means, [&](int e, float2 m) {
        Channels<VEC>::put(mean_a[e / 2], e % 2, -m.x);
        Channels<VEC>::put(mean_b[e / 2], e % 2, -m.y);
    });
    with_act_of(a.act, [&](auto act) {
        RawVec<T, VEC> raw[R];
        RawVec<U, VEC> graw[R];
        walk_pixels<R, true>(st,
                       [&](int i, size_t o) {
                           raw[i].load(x + o);
                           graw[i].load(grad_y + o);
                       },
                       [&](int i, size_t o) {
                           float v[VEC > 1 ? VEC : 2], out[VEC];
#pragma unroll
                           for (int k = 0; k < N; ++k) {
                               Pair u, g;
                               ch.template slopes<decltype(act)::value>(k, two(raw[i], k), two(graw[i], k), u, g);
                               split(pair_mul(ch.rstd[k], pair_fma(u, mean_b[k], pair_fma(g, ch.gain[k], mean_a[k]))), v[2 * k], v[2 * k + 1]);
                           }
#pragma unroll
                           for (int e = 0; e < VEC; ++e) out[e] = v[e];
                           store_vec_once<VEC>(grad_x + o, out);
                       });
    });
}

// Backward: the channels' sums of the pieces go to `parts`; the gain's and the bias's gradients are added up from them.
// LONG: some threads have more than kRun pixels; sums of their runs wait in shared memory.
template <typename T, typename U, int VEC, int R, bool WHOLE, bool LONG>
__global__ void __launch_bounds__(kGnormThreads, 3) gnorm_sums_kernel(const T* x, const U* grad_y, T* grad_x, GnormArgs a) {
    constexpr int N = Channels<VEC>::N;
    __shared__ float2 sums[kGnormThreads * VEC], joined[kGnormThreads * VEC];
    __shared__ double2 red[kGnormThreads];
    pdl_begin();
    const Stretch<VEC> st(a, blockIdx.x, R);
    if (st.live) {
        Channels<VEC> ch;
        load_channels(a, st, ch);
        Pair s1[N], s2[N];
#pragma unroll
        for (int i = 0; i < N; ++i) s1[i] = s2[i] = pair_of(0.f, 0.f);
        const int at = threadIdx.x;
        with_act_of(a.act, [&](auto act) {
            RawVec<T, VEC> raw[R];
            RawVec<U, VEC> graw[R];
            walk_pixels<R, false, false, LONG>(st,
                           [&](int i, size_t o) {
                               raw[i].load(x + o);
                               graw[i].load(grad_y + o);
                           },
                           [&](int i, size_t) {
#pragma unroll
                               for (int k = 0; k < N; ++k) {
                                   Pair u, g;
                                   ch.template slopes<decltype(act)::value>(k, two(raw[i], k), two(graw[i], k), u, g);
                                   s1[k] = pair_add(s1[k], g);
                                   s2[k] = pair_fma(g, u, s2[k]);
                               }
                           },
                           [](int) {},
                           [&](int before) {
#pragma unroll
                               for (int e = 0; e < VEC; ++e) {
                                   const double old1 = before ? as_double(sums[e * kGnormThreads + at]) : 0.0, old2 = before ? as_double(joined[e * kGnormThreads + at]) : 0.0;
                                   sums[e * kGnormThreads + at] = as_float2(old1 + (double)half(s1[e / 2], e));
                                   joined[e * kGnormThreads + at] = as_float2(old2 + (double)half(s2[e / 2], e));
                               }
#pragma unroll
                               for (int i = 0; i < N; ++i) s1[i] = s2[i] = pair_of(0.f, 0.f);
                           });
        });
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            float2 both = make_float2(half(s1[e / 2], e), half(s2[e / 2], e));
            if (LONG && folded_pixels<R>(st) > 0)
                both = make_float2((float)(as_double(sums[e * kGnormThreads + at]) + (double)both.x), (float)(as_double(joined[e * kGnormThreads + at]) + (double)both.y));
            sums[e * kGnormThreads + at] = both;
        }
    }
    __syncthreads();
    each_channel<VEC>(a, [&](int c, int e, int column) {
        const float2* v = sums + e * kGnormThreads + column;
        float2 s = v[0];
        for (int l = 1; l < st.lanes; ++l) {
            s.x += v[l * a.columns].x;
            s.y += v[l * a.columns].y;
        }
        joined[c] = s;
        a.parts[((size_t)st.image * a.pieces + st.piece) * a.channels + c] = s;
    });
    __syncthreads();
    each_group(a, [&](int g, int l, int wide, bool one) {
        float s = 0.f, q = 0.f;
        for (int i = l; i < (one ? a.depth : 0); i += wide) {
            const int c = g * a.depth + i;
            const float gain = a.gain ? __ldg(a.gain + c) : 1.f;
            s = fmaf(gain, joined[c].x, s);
            q = fmaf(gain, joined[c].y, q);
        }
        s = lanes_sum(s, wide);
        q = lanes_sum(q, wide);
        if (one && l == 0) a.group_parts[((size_t)st.image * a.pieces + st.piece) * a.groups + g] = make_double2((double)s, (double)q);
    });
    if (!last_of_image(a, st.image)) return;
    join_groups(a, st.image, red, [&](int, double2 v) { return v; },
                [&](int g, double2 s) { a.means[(size_t)st.image * a.groups + g] = make_float2((float)(s.x * a.inv_m), (float)(s.y * a.inv_m)); });
    if constexpr (WHOLE) {
        if (!grad_x) return;
        __syncthreads();
        grad_stretch<T, U, VEC, R>(x, grad_y, grad_x, a, st);
    }
}
// The gradients of kTotalWide channels of the gain and the bias, by one block, from all pieces' sums.
constexpr int kTotalWide = 8;
__device__ __forceinline__ void total_of_channels(const GnormArgs& a, int block, float* grad_gain, float* grad_bias, double2* red) {
    const int c = block * kTotalWide + threadIdx.x % kTotalWide, r = threadIdx.x / kTotalWide, rows = a.images * a.pieces;
    double2 s = make_double2(0.0, 0.0);
    if (c < a.channels)
#pragma unroll 8
        for (int t = r; t < rows; t += kGnormThreads / kTotalWide) {
            const float2 v = a.parts[(size_t)t * a.channels + c];
            s.x += (double)v.x;
            s.y += (double)v.y;
        }
    red[threadIdx.x] = s;
    __syncthreads();
    if (r != 0 || c >= a.channels) return;
    for (int i = 1; i < kGnormThreads / kTotalWide; ++i) {
        s.x += red[i * kTotalWide + threadIdx.x].x;
        s.y += red[i * kTotalWide + threadIdx.x].y;
    }
    if (grad_bias) grad_bias[c] = (float)s.x;
    if (grad_gain) grad_gain[c] = (float)s.y;
}

// Its first `totals` blocks add up the gradients of the gain and the bias meanwhile.
template <typename T, typename U, int VEC, int R>
__global__ void __launch_bounds__(kGnormThreads, 3) gnorm_grad_kernel(const T* x, const U* grad_y, T* grad_x, float* grad_gain, float* grad_bias, int totals, GnormArgs a) {
    __shared__ double2 red[kGnormThreads];
    pdl_begin();
    if ((int)blockIdx.x < totals) {
        total_of_channels(a, blockIdx.x, grad_gain, grad_bias, red);
        return;
    }
    grad_stretch<T, U, VEC, R>(x, grad_y, grad_x, a, Stretch<VEC>(a, gridDim.x - 1 - blockIdx.x, R));
}

__global__ void __launch_bounds__(kGnormThreads) gnorm_total_kernel(float* grad_gain, float* grad_bias, GnormArgs a) {
    __shared__ double2 red[kGnormThreads];
    pdl_begin();
    total_of_channels(a, blockIdx.x, grad_gain, grad_bias, red);
}

constexpr int kGnormTarget = 148 * 8;       // blocks that fill the machine
constexpr double kEndRounds = 3.0;
// Rounds up to which a block takes a whole image, in one launch.  Forward, 256 channels bfloat16, in pieces and whole: 64 images of 1 round 7.7 and 6.1 us, of 4
// rounds 13.2 and 9.9, of 6 rounds 13.5 and 12.3; 4 images of 3 rounds 8.9 and 8.4, of 4 rounds 8.9 and 9.6, of 6 rounds 9.0 and 11.8.  Backward with ReLU: 148 images of 2
// rounds 11.1 and 9.9, of 4 rounds 13.6 and 13.4; 64 of 4 rounds 11.1 and 11.7 (SiLU 10.7 and 9.9).  With few images a round's slopes and the second reading make the whole one
// slow: 4 of 2 rounds 8.0 and 8.2, of 4 rounds 8.3 and 11.1 (SiLU 8.0 and 9.3; without an activation 7.5 and 7.7; single channels, 8 of 86 x 12 x 2 of 3 rounds, 8.0 and 7.2).
constexpr int kWholeRounds = 4, kWholeRoundsFew = 2, kFewImages = 32;
// Images from which on a block takes a whole one of any size: what it has read last is still near.  In pieces and whole, bfloat16: forward 1776 of 28 x 28 x 64 102 and 78 us (900
// of them 57 and 47: fewer would gain as well), backward 6000 of 14 x 14 x 256 without an activation 528 and 516, 1776 of 28 x 28 x 64 with ReLU 193 and 199.
constexpr int kManyImages = 148 * 12;

// How a call is run.
struct GnormPlan {
    int vec, r;             // elements a vector, pixels a thread; vec 0: any tensor
    int columns, tiles, pieces, per;
    bool whole;             // a block an image, in one launch
    bool runs;              // a thread may have more than kRun pixels
};
static GnormPlan plan_of(const Gnorm* g, int images, int pixels, bool backward, uintptr_t addresses) {
    const size_t xb = dtype_bytes(g->x_dtype), yb = dtype_bytes(g->y_dtype), small = xb < yb ? xb : yb;
    GnormPlan p{};
    // 16 bytes of the smaller type (backward 4 elements: with 8 the constants leave room for two blocks an SM, 64 x 56 x 56 x 256 SiLU: 116 against 110 us),
    // 4 elements, or single ones
    const int widest = small == 2 && !backward ? 8 : 4;
    for (int vec : {widest, 4, 1})
        if (g->channels % vec == 0 && g->channels / vec <= kGnormThreads && addresses % std::min(vec * xb, (size_t)16) == 0 && addresses % std::min(vec * yb, (size_t)16) == 0) {
            p.vec = vec;
            break;
        }
    if (p.vec) {
        p.columns = g->channels / p.vec;
        p.tiles = 1;
        const int lanes = kGnormThreads / p.columns;
        p.r = backward || (p.vec == 8 && xb == 4) ? 4 : 8;
        // a round of loads a piece at least, and no more pieces than fill the machine twice over
        p.per = lanes * p.r;
        const int rounds = (pixels + p.per - 1) / p.per;
        const bool slow_rounds = backward && p.vec > 1 && g->act != CIRC_ACT_NONE;
        p.whole = rounds <= (slow_rounds && images < kFewImages ? kWholeRoundsFew : kWholeRounds) || images >= kManyImages;
        if (p.whole) {
            p.pieces = 1;
            p.runs = pixels / p.per * p.r > kRun;
            return p;
        }
        // As many pieces an image as take the least time: blocks that run at once (three an SM) take the pieces in turns, and a block's beginning and end
        // take as long as some rounds.
        const long slots = 148 * 3, most = std::min((long)rounds, (kGnormTarget + images) / (long)images);
        double best = 0.0;
        p.pieces = 1;
        for (long k = 1; k <= most; ++k) {
            const double cost = (double)((images * k + slots - 1) / slots) * ((double)((rounds + k - 1) / k) + kEndRounds);
            if (k == 1 || cost < best) {
                best = cost;
                p.pieces = (int)k;
            }
        }
        p.runs = (pixels / p.per + p.pieces - 1) / p.pieces * p.r > kRun;
    } else {
        p.columns = kGnormThreads < g->channels ? kGnormThreads : g->channels;
        p.tiles = (g->channels + p.columns - 1) / p.columns;
        const int lanes = kGnormThreads / p.columns;
        const long want = (kGnormTarget + (long)images * p.tiles - 1) / ((long)images * p.tiles), can = (pixels + 8L * lanes - 1) / (8L * lanes);
        const long pieces = std::min({want, can, 64L});       // one block joins them
        p.per = (int)((pixels + pieces - 1) / pieces);
        p.pieces = (pixels + p.per - 1) / p.per;
        p.runs = p.per > kRun * lanes;
    }
    return p;
}
// Pieces that any call of up to `images` images has at most, all images together.
static long pieces_of(long images) { return kGnormTarget + images; }

// Workspace: the images' counters, the pieces' sums, the groups' means, and mean and rstd where the caller keeps
// none.
struct GnormSpace {
    size_t group_parts, parts, means, stats, bytes;
};
static GnormSpace space_of(const Gnorm* g, long images) {
    const long pieces = pieces_of(images);
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    GnormSpace s;
    s.group_parts = up(sizeof(unsigned) * images);
    s.parts = s.group_parts + up(sizeof(double2) * pieces * g->groups);
    s.means = s.parts + up(sizeof(float2) * pieces * g->channels);
    s.stats = s.means + up(sizeof(float2) * images * g->groups);
    s.bytes = s.stats + up(2 * sizeof(float) * images * g->groups);
    return s;
}
// Clears what it has just allocated, nothing else: the counters of a workspace in use are 0 between calls, and numbers of images that need the same bytes
// have the same layout, since no section shrinks as the images grow.
static int ensure_gnorm(Gnorm* g, long images, cudaStream_t s) {
    const long held = images > g->images_held ? images : g->images_held;
    const GnormSpace space = space_of(g, held);
    const bool fresh = g->ws.bytes < space.bytes;
    const int rc = ensure_scratch(g->ws, space.bytes, s, "circ_gnorm_reserve");
    if (rc != CIRC_OK) {
        if (!g->ws.ptr) g->images_held = 0;
        return rc;
    }
    g->images_held = held;
    if (!fresh) return CIRC_OK;
    if (cudaMemsetAsync(g->ws.ptr, 0, space.group_parts, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaFree(g->ws.ptr);      // this one alone: graphs may hold earlier ones
        g->ws.ptr = nullptr;
        g->ws.bytes = 0;
        g->images_held = 0;
        set_error(CIRC_ERR_CUDA, "clearing the workspace failed: %s", cudaGetErrorString(cudaGetLastError()));
        return CIRC_ERR_CUDA;
    }
    return CIRC_OK;
}

// Calls f(vector elements, pixels a thread) as constants.
template <typename T, bool BACKWARD, typename F>
static void with_plan(const GnormPlan& p, F&& f) {
    auto with_r = [&](auto vec) {
        constexpr int VEC = decltype(vec)::value, R = BACKWARD || (VEC == 8 && sizeof(T) == 4) ? 4 : 8;
        f(vec, std::integral_constant<int, R>{});
    };
    if constexpr (!BACKWARD)
        if (p.vec == 8) {
            with_r(std::integral_constant<int, 8>{});
            return;
        }
    if (p.vec == 4) with_r(std::integral_constant<int, 4>{});
    else with_r(std::integral_constant<int, 1>{});
}
static int check_gnorm(const Gnorm* g, int N, int H, int W) {
    if (!g) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (N < 0 || N > (1 << 20) || H < 1 || W < 1 || (long)H * W > (1L << 28)) {
        set_error(CIRC_ERR_SHAPE, "N=%d must be in [0, 2^20], H=%d and W=%d at least 1 and their product at most 2^28", N, H, W);
        return CIRC_ERR_SHAPE;
    }
    return CIRC_OK;
}
template <typename T, typename U>
static cudaError_t run_forward(const GnormPlan& p, const GnormArgs& a, const T* x, U* y, cudaStream_t s) {
    cudaError_t err = cudaSuccess;
    if (p.vec == 0) {
        const dim3 grid((unsigned)((long)a.images * a.pieces * a.tiles));
        const auto stats = p.runs ? gnorm_any_stats_kernel<T, true> : gnorm_any_stats_kernel<T, false>;
        if ((err = launch_row(stats, grid, dim3(kGnormThreads), 0, s, x, a)) == cudaSuccess)
            err = launch_row(gnorm_any_apply_kernel<T, U>, grid, dim3(kGnormThreads), 0, s, x, y, a);
        return err;
    }
    with_plan<T, false>(p, [&](auto vec, auto r) {
        constexpr int VEC = decltype(vec)::value, R = decltype(r)::value;
        const dim3 grid((unsigned)((long)a.images * a.pieces));
        if (p.whole) {
            err = launch_row(p.runs ? gnorm_stats_kernel<T, U, VEC, R, true, true> : gnorm_stats_kernel<T, U, VEC, R, true, false>, grid, dim3(kGnormThreads), 0,
                             s, x, y, a);
            return;
        }
        const auto stats = p.runs ? gnorm_stats_kernel<T, U, VEC, R, false, true> : gnorm_stats_kernel<T, U, VEC, R, false, false>;
        if ((err = launch_row(stats, grid, dim3(kGnormThreads), 0, s, x, y, a)) == cudaSuccess)
            err = launch_row(gnorm_apply_kernel<T, U, VEC, R>, grid, dim3(kGnormThreads), 0, s, x, y, a);
    });
    return err;
}
template <typename T, typename U>
static cudaError_t run_backward(const GnormPlan& p, const GnormArgs& a, const T* x, const U* grad_y, T* grad_x, float* grad_gain, float* grad_bias,
                                cudaStream_t s, int* launches) {
    cudaError_t err = cudaSuccess;
    const int totals = grad_gain || grad_bias ? (a.channels + kTotalWide - 1) / kTotalWide : 0;
    const dim3 grid((unsigned)((long)a.images * a.pieces * a.tiles)), threads(kGnormThreads);
    bool done = false;
    *launches = 1;
    if (p.vec == 0) {
        const auto sums = p.runs ? gnorm_any_sums_kernel<T, U, true> : gnorm_any_sums_kernel<T, U, false>;
        if ((err = launch_row(sums, grid, threads, 0, s, x, grad_y, a)) == cudaSuccess && grad_x) {
            err = launch_row(gnorm_any_grad_kernel<T, U>, grid, threads, 0, s, x, grad_y, grad_x, a);
            ++*launches;
        }
    } else {
        with_plan<T, true>(p, [&](auto vec, auto r) {
            constexpr int VEC = decltype(vec)::value, R = decltype(r)::value;
            if (p.whole) {
                err = launch_row(p.runs ? gnorm_sums_kernel<T, U, VEC, R, true, true> : gnorm_sums_kernel<T, U, VEC, R, true, false>, grid, threads, 0, s, x, grad_y,
                                 grad_x, a);
                return;
            }
            const auto sums = p.runs ? gnorm_sums_kernel<T, U, VEC, R, false, true> : gnorm_sums_kernel<T, U, VEC, R, false, false>;
            if ((err = launch_row(sums, grid, threads, 0, s, x, grad_y, grad_x, a)) == cudaSuccess && grad_x) {
                err = launch_row(gnorm_grad_kernel<T, U, VEC, R>, dim3(grid.x + totals), threads, 0, s, x, grad_y, grad_x, grad_gain, grad_bias, totals, a);
                done = true;
                ++*launches;
            }
        });
    }
    if (err == cudaSuccess && totals && !done) {
        err = launch_row(gnorm_total_kernel, dim3((unsigned)totals), threads, 0, s, grad_gain, grad_bias, a);
        ++*launches;
    }
    return err;
}

static GnormArgs args_of(const Gnorm* g, const GnormPlan& p, const float* gain, const float* bias, const float* mean, const float* rstd, int N, int pixels) {
    const GnormSpace space = space_of(g, g->images_held);
    char* ws = static_cast<char*>(g->ws.ptr);
    GnormArgs a{};
    a.gain = gain;
    a.bias = bias;
    float* stats = reinterpret_cast<float*>(ws + space.stats);
    a.mean = mean ? const_cast<float*>(mean) : stats;
    a.rstd = rstd ? const_cast<float*>(rstd) : stats + (size_t)g->images_held * g->groups;
    a.channels = g->channels;
    a.groups = g->groups;
    a.depth = g->channels / g->groups;
    a.images = N;
    a.pixels = pixels;
    a.eps = g->eps;
    a.inv_m = 1.0 / ((double)pixels * a.depth);
    a.inv_depth = 1.0 / (double)a.depth;
    a.columns = p.columns;
    a.tiles = p.tiles;
    a.pieces = p.pieces;
    a.per = p.per;
    a.act = g->act;
    a.arrived = reinterpret_cast<unsigned*>(ws);
    a.group_parts = reinterpret_cast<double2*>(ws + space.group_parts);
    a.parts = reinterpret_cast<float2*>(ws + space.parts);
    a.means = reinterpret_cast<float2*>(ws + space.means);
    return a;
}
static uintptr_t address(const void* p) { return reinterpret_cast<uintptr_t>(p); }

}  // namespace circ

using namespace circ;

extern "C" {

circ_gnorm_handle circ_gnorm_create(int channels, int groups, float eps) {
    if (channels < 1 || channels > (1 << 16) || groups < 1 || channels % groups != 0 || !(eps >= 0.f)) {
        set_error(CIRC_ERR_SHAPE, "channels=%d must be in [1, 2^16], groups=%d a divisor of it, eps=%g not negative", channels, groups, (double)eps);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Gnorm* g = new (std::nothrow) Gnorm{device, channels, groups, eps, CIRC_F32, CIRC_F32, CIRC_ACT_NONE, {}, 0};
    if (!g) set_error(CIRC_ERR_ALLOC, "host allocation failed");
    return reinterpret_cast<circ_gnorm_handle>(g);
}

void circ_gnorm_destroy(circ_gnorm_handle h) {
    Gnorm* g = reinterpret_cast<Gnorm*>(h);
    if (!g) return;
    free_on(g->device, g->ws);
    delete g;
}

int circ_gnorm_set_dtypes(circ_gnorm_handle h, int x_dtype, int y_dtype) {
    Gnorm* g = reinterpret_cast<Gnorm*>(h);
    if (!g || !float_dtype(x_dtype) || !float_dtype(y_dtype)) {
        set_error(CIRC_ERR_ARG, "bad handle or type codes (%d, %d)", x_dtype, y_dtype);
        return CIRC_ERR_ARG;
    }
    g->x_dtype = x_dtype;
    g->y_dtype = y_dtype;
    return CIRC_OK;
}

int circ_gnorm_set_activation(circ_gnorm_handle h, int activation) {
    Gnorm* g = reinterpret_cast<Gnorm*>(h);
    if (!g || activation < CIRC_ACT_NONE || activation > CIRC_ACT_SILU) {
        set_error(CIRC_ERR_ARG, "bad handle or activation %d", activation);
        return CIRC_ERR_ARG;
    }
    g->act = activation;
    return CIRC_OK;
}

int circ_gnorm_reserve(circ_gnorm_handle h, int N, int H, int W) {
    Gnorm* g = reinterpret_cast<Gnorm*>(h);
    const int rc = check_gnorm(g, N, H, W);
    return rc != CIRC_OK || N == 0 ? rc : ensure_gnorm(g, N, 0);
}

int circ_gnorm_forward(circ_gnorm_handle h, const void* x, const float* gain, const float* bias, void* y, float* mean, float* rstd, int N, int H,
                       int W, void* stream) {
    Gnorm* g = reinterpret_cast<Gnorm*>(h);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc = check_gnorm(g, N, H, W);
    if (rc != CIRC_OK || N == 0) return rc;
    if (!x || !y || (x == y && g->x_dtype != g->y_dtype)) {
        set_error(CIRC_ERR_ARG, "x and y must be non-NULL; y in the place of x needs its type");
        return CIRC_ERR_ARG;
    }
    if (misaligned(x, dtype_bytes(g->x_dtype)) || misaligned(y, dtype_bytes(g->y_dtype)) || misaligned(gain, 4) || misaligned(bias, 4) ||
        misaligned(mean, 4) || misaligned(rstd, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    const GnormPlan p = plan_of(g, N, H * W, false, address(x) | address(y));
    if ((rc = ensure_gnorm(g, N, s)) != CIRC_OK) return rc;
    const GnormArgs a = args_of(g, p, gain, bias, mean, rstd, N, H * W);
    cudaError_t err = cudaSuccess;
    with_dtype(g->x_dtype, [&](auto* t) {
        with_dtype(g->y_dtype, [&](auto* u) {
            using T = tag_type<decltype(t)>;
            using U = tag_type<decltype(u)>;
            err = run_forward(p, a, static_cast<const T*>(x), static_cast<U*>(y), s);
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(p.whole ? 1 : 2);
    return CIRC_OK;
}

int circ_gnorm_backward(circ_gnorm_handle h, const void* x, const float* gain, const float* bias, const float* mean, const float* rstd,
                        const void* grad_y, void* grad_x, float* grad_gain, float* grad_bias, int N, int H, int W, void* stream) {
    Gnorm* g = reinterpret_cast<Gnorm*>(h);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc = check_gnorm(g, N, H, W);
    if (rc != CIRC_OK) return rc;
    if (misaligned(gain, 4) || misaligned(bias, 4) || misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(grad_gain, 4) || misaligned(grad_bias, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    if (N == 0) {
        if (grad_gain) CIRC_CUDA_TRY(cudaMemsetAsync(grad_gain, 0, sizeof(float) * g->channels, s), CIRC_ERR_CUDA);
        if (grad_bias) CIRC_CUDA_TRY(cudaMemsetAsync(grad_bias, 0, sizeof(float) * g->channels, s), CIRC_ERR_CUDA);
        return CIRC_OK;
    }
    if (!x || !grad_y || !mean || !rstd || (!grad_x && !grad_gain && !grad_bias) || (g->x_dtype != g->y_dtype && grad_x == grad_y)) {
        set_error(CIRC_ERR_ARG, "x, grad_y, mean, rstd and one of the gradients must be non-NULL; grad_x in the place of grad_y needs its type");
        return CIRC_ERR_ARG;
    }
    if (misaligned(x, dtype_bytes(g->x_dtype)) || misaligned(grad_x, dtype_bytes(g->x_dtype)) || misaligned(grad_y, dtype_bytes(g->y_dtype))) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    const GnormPlan p = plan_of(g, N, H * W, true, address(x) | address(grad_y) | address(grad_x));
    if ((rc = ensure_gnorm(g, N, s)) != CIRC_OK) return rc;
    const GnormArgs a = args_of(g, p, gain, bias, mean, rstd, N, H * W);
    cudaError_t err = cudaSuccess;
    int launches = 0;
    with_dtype(g->x_dtype, [&](auto* t) {
        with_dtype(g->y_dtype, [&](auto* u) {
            using T = tag_type<decltype(t)>;
            using U = tag_type<decltype(u)>;
            err = run_backward(p, a, static_cast<const T*>(x), static_cast<const U*>(grad_y), static_cast<T*>(grad_x), grad_gain, grad_bias, s, &launches);
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(launches);
    return CIRC_OK;
}

}  // extern "C"
