// Group norm with an activation on channel-last tensors [N][pixels][C]: over the m = pixels D values of an image and a group of D channels
//   mean, variance = mean((x - mean)^2), rstd = 1 / sqrt(variance + eps), v = gain_c (x - mean) rstd + bias_c, y = act(v)
// and its gradients, with u = (x - mean) rstd and g = grad_y act'(v):
//   grad_x = rstd (gain g - (A + u B) / m), A = sum of gain g over the group, B = sum of gain g u
//   grad_gain_c = sum of g u, grad_bias_c = sum of g over images and pixels.
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
    int images_held;        // images that the workspace is laid out for
};

struct GnormArgs {
    const float *gain, *bias;
    float *mean, *rstd;       // [N][groups]
    int channels, groups, depth;      // depth: channels a group
    int images, pixels;
    float eps;
    // a block's part: `columns` vectors of channels (all, or a tile of them), and pixels of one image
    int columns, tiles, pieces, per;
    // workspace
    unsigned* arrived;        // [N] parts of an image that are summed up (0 before and after a call)
    float2* parts;            // [N][pieces][C] forward: mean, less the channel's first value, and sum of squares around it; backward: sum of g, of g u
    float2* totals;           // [N][C] backward: the same over the image
    float2* means;            // [N][groups] backward: A / m, B / m
};

constexpr int kGnormThreads = 256;

__device__ __forceinline__ float sigmoid_of(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if constexpr (ACT == CIRC_ACT_RELU) return v > 0.f ? v : v != v ? v : 0.f;
    if constexpr (ACT == CIRC_ACT_SILU) return v * sigmoid_of(v);
    return v;
}

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

// Which vectors of channels and which pixels a thread works on.
template <int VEC>
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
        live = lane < lanes && column * VEC < a.channels;
    }
    __device__ __forceinline__ size_t at(const GnormArgs& a, int pixel) const {
        return ((size_t)image * a.pixels + pixel) * a.channels + (size_t)column * VEC;
    }
    __device__ __forceinline__ Channel channel(const GnormArgs& a, int e) const {
        const int c = column * VEC + e, g = c / a.depth;
        return Channel{a.mean[(size_t)image * a.groups + g], a.rstd[(size_t)image * a.groups + g], a.gain ? a.gain[c] : 1.f, a.bias ? a.bias[c] : 0.f};
    }
};

// The block that is last to finish an image's parts.  All threads call it.
__device__ __forceinline__ bool last_of_image(const GnormArgs& a, int image) {
    __shared__ bool last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        const unsigned parts = (unsigned)(a.pieces * a.tiles);
        last = parts == 1 || atomicAdd(a.arrived + image, 1u) == parts - 1;
        if (last && parts > 1) a.arrived[image] = 0;
    }
    __syncthreads();
    if (last) __threadfence();
    return last;
}

// A thread's sums of a channel run around the thread's first value, which bounds what the difference of the two sums loses; means are kept as
// differences from the channel's first value in the image, so that a large offset costs no digits, until they are joined in float64.
template <typename T, int VEC>
__global__ void __launch_bounds__(kGnormThreads) gnorm_stats_kernel(const T* __restrict__ x, GnormArgs a) {
    __shared__ float2 sums[kGnormThreads * VEC];
    pdl_begin();
    const GnormPlace<VEC> at(a);
    float pivot[VEC], s1[VEC], s2[VEC];
    int n = 0;
    if (at.live) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) pivot[e] = s1[e] = s2[e] = 0.f;
        for (int p = at.from + at.lane; p < at.to; p += at.lanes, ++n) {
            RawVec<T, VEC> raw;
            raw.load(x + at.at(a, p));
            if (n == 0)
#pragma unroll
                for (int e = 0; e < VEC; ++e) pivot[e] = raw.get(e);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = raw.get(e) - pivot[e];
                s1[e] += d;
                s2[e] = fmaf(d, d, s2[e]);
            }
        }
        const float inv = n ? 1.f / (float)n : 0.f;
        RawVec<T, VEC> first;
        first.load(x + at.at(a, 0));
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            sums[(at.lane * a.columns + threadIdx.x % a.columns) * VEC + e] = make_float2(fmaf(s1[e], inv, pivot[e] - first.get(e)), s2[e] - s1[e] * s1[e] * inv);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.columns * VEC; i += kGnormThreads) {
        const int c = at.tile * a.columns * VEC + i;
        if (c >= a.channels) continue;
        float count = 0.f, mean = 0.f, m2 = 0.f;
        for (int l = 0; l < at.lanes; ++l) {
            const int mine = (at.to - at.from - l + at.lanes - 1) / at.lanes;
            if (mine <= 0) break;
            const float2 v = sums[l * a.columns * VEC + i];
            const float all = count + (float)mine, d = v.x - mean, part = (float)mine / all;
            mean = fmaf(d, part, mean);
            m2 += v.y + d * d * count * part;
            count = all;
        }
        a.parts[((size_t)at.image * a.pieces + at.piece) * a.channels + c] = make_float2(mean, m2);
    }
    if (!last_of_image(a, at.image)) return;
    // a warp a group
    const int lane = threadIdx.x % 32, entries = a.pieces * a.depth;
    const double m = (double)a.pixels * a.depth;
    for (int g = threadIdx.x / 32; g < a.groups; g += kGnormThreads / 32) {
        const float2* p = a.parts + (size_t)at.image * a.pieces * a.channels + g * a.depth;
        const T* first = x + (size_t)at.image * a.pixels * a.channels + g * a.depth;
        double sum = 0.0, m2 = 0.0;
        for (int i = lane; i < entries; i += 32) {
            const int piece = i / a.depth;
            const float2 v = __ldcg(p + (size_t)piece * a.channels + i % a.depth);
            sum += ((double)v.x + (double)to_float(first[i % a.depth])) * (min(a.pixels, (piece + 1) * a.per) - piece * a.per);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const double mean = sum / m;
        for (int i = lane; i < entries; i += 32) {
            const int piece = i / a.depth;
            const float2 v = __ldcg(p + (size_t)piece * a.channels + i % a.depth);
            const double d = (double)v.x + (double)to_float(first[i % a.depth]) - mean;
            m2 += (double)v.y + d * d * (min(a.pixels, (piece + 1) * a.per) - piece * a.per);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
        if (lane == 0) {
            a.mean[(size_t)at.image * a.groups + g] = (float)mean;
            a.rstd[(size_t)at.image * a.groups + g] = (float)(1.0 / sqrt(m2 / m + (double)a.eps));
        }
    }
}

template <typename T, typename U, int VEC, int ACT>
__global__ void __launch_bounds__(kGnormThreads) gnorm_apply_kernel(const T* x, U* y, GnormArgs a) {
    pdl_begin();
    const GnormPlace<VEC> at(a);
    if (!at.live) return;
    float mean[VEC], scale[VEC], bias[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const Channel c = at.channel(a, e);
        mean[e] = c.mean;
        scale[e] = c.rstd * c.gain;
        bias[e] = c.bias;
    }
    for (int p = at.from + at.lane; p < at.to; p += at.lanes) {
        RawVec<T, VEC> raw;
        float v[VEC];
        raw.load(x + at.at(a, p));
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = activate<ACT>(fmaf(raw.get(e) - mean[e], scale[e], bias[e]));
        store_vec<VEC>(y + at.at(a, p), v);
    }
}

template <typename T, typename U, int VEC, int ACT>
__global__ void __launch_bounds__(kGnormThreads) gnorm_sums_kernel(const T* __restrict__ x, const U* __restrict__ grad_y, GnormArgs a) {
    __shared__ float2 sums[kGnormThreads * VEC];
    pdl_begin();
    const GnormPlace<VEC> at(a);
    if (at.live) {
        Channel ch[VEC];
        float s1[VEC], s2[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            ch[e] = at.channel(a, e);
            s1[e] = s2[e] = 0.f;
        }
        for (int p = at.from + at.lane; p < at.to; p += at.lanes) {
            RawVec<T, VEC> raw;
            RawVec<U, VEC> graw;
            raw.load(x + at.at(a, p));
            graw.load(grad_y + at.at(a, p));
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float v = raw.get(e), u = ch[e].unit(v), g = graw.get(e) * ch[e].template slope<ACT>(v, u);
                s1[e] += g;
                s2[e] = fmaf(g, u, s2[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[(at.lane * a.columns + threadIdx.x % a.columns) * VEC + e] = make_float2(s1[e], s2[e]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.columns * VEC; i += kGnormThreads) {
        const int c = at.tile * a.columns * VEC + i;
        if (c >= a.channels) continue;
        float2 s = make_float2(0.f, 0.f);
        for (int l = 0; l < at.lanes; ++l) {
            const float2 v = sums[l * a.columns * VEC + i];
            s.x += v.x;
            s.y += v.y;
        }
        a.parts[((size_t)at.image * a.pieces + at.piece) * a.channels + c] = s;
    }
    if (!last_of_image(a, at.image)) return;
    for (int c = threadIdx.x; c < a.channels; c += kGnormThreads) {
        double s1 = 0.0, s2 = 0.0;
        for (int piece = 0; piece < a.pieces; ++piece) {
            const float2 v = __ldcg(a.parts + ((size_t)at.image * a.pieces + piece) * a.channels + c);
            s1 += (double)v.x;
            s2 += (double)v.y;
        }
        a.totals[(size_t)at.image * a.channels + c] = make_float2((float)s1, (float)s2);
    }
    __syncthreads();
    const int lane = threadIdx.x % 32;
    const double m = (double)a.pixels * a.depth;
    for (int g = threadIdx.x / 32; g < a.groups; g += kGnormThreads / 32) {
        double s1 = 0.0, s2 = 0.0;
        for (int i = lane; i < a.depth; i += 32) {
            const int c = g * a.depth + i;
            const float2 v = a.totals[(size_t)at.image * a.channels + c];
            const double gain = a.gain ? (double)a.gain[c] : 1.0;
            s1 += gain * v.x;
            s2 += gain * v.y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s1 += __shfl_xor_sync(0xffffffffu, s1, o);
            s2 += __shfl_xor_sync(0xffffffffu, s2, o);
        }
        if (lane == 0) a.means[(size_t)at.image * a.groups + g] = make_float2((float)(s1 / m), (float)(s2 / m));
    }
}

// The blocks behind those of the pixels add up the gain's and the bias's gradients over the images, 32 channels each.
template <typename T, typename U, int VEC, int ACT>
__global__ void __launch_bounds__(kGnormThreads) gnorm_grad_kernel(const T* x, const U* grad_y, T* grad_x, float* grad_gain, float* grad_bias, GnormArgs a) {
    __shared__ double2 red[kGnormThreads / 32][32];
    pdl_begin();
    const unsigned blocks = grad_x ? (unsigned)a.images * a.pieces * a.tiles : 0;
    if (blockIdx.x >= blocks) {
        const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = (int)(blockIdx.x - blocks) * 32 + lane;
        double2 s = make_double2(0.0, 0.0);
        if (c < a.channels)
            for (int n = warp; n < a.images; n += kGnormThreads / 32) {
                const float2 v = a.totals[(size_t)n * a.channels + c];
                s.x += (double)v.x;
                s.y += (double)v.y;
            }
        red[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && c < a.channels) {
            for (int w = 1; w < kGnormThreads / 32; ++w) {
                s.x += red[w][lane].x;
                s.y += red[w][lane].y;
            }
            if (grad_bias) grad_bias[c] = (float)s.x;
            if (grad_gain) grad_gain[c] = (float)s.y;
        }
        return;
    }
    const GnormPlace<VEC> at(a);
    if (!at.live) return;
    Channel ch[VEC];
    float mean_a[VEC], mean_b[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        ch[e] = at.channel(a, e);
        const float2 m = a.means[(size_t)at.image * a.groups + (at.column * VEC + e) / a.depth];
        mean_a[e] = m.x;
        mean_b[e] = m.y;
    }
    for (int p = at.from + at.lane; p < at.to; p += at.lanes) {
        RawVec<T, VEC> raw;
        RawVec<U, VEC> graw;
        float out[VEC];
        raw.load(x + at.at(a, p));
        graw.load(grad_y + at.at(a, p));
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float v = raw.get(e), u = ch[e].unit(v), g = graw.get(e) * ch[e].template slope<ACT>(v, u);
            out[e] = ch[e].rstd * (fmaf(g, ch[e].gain, -mean_a[e]) - u * mean_b[e]);
        }
        store_vec<VEC>(grad_x + at.at(a, p), out);
    }
}

constexpr int kGnormTarget = 148 * 8;       // blocks that fill the machine

static void lay_out(GnormArgs& a, int vec) {
    const int vectors = a.channels / vec;
    a.columns = vectors < kGnormThreads ? vectors : kGnormThreads;
    a.tiles = (vectors + a.columns - 1) / a.columns;
    const int lanes = kGnormThreads / a.columns;
    const long want = (kGnormTarget + (long)a.images * a.tiles - 1) / ((long)a.images * a.tiles), can = (a.pixels + 4L * lanes - 1) / (4L * lanes);
    const long pieces = want < can ? want : can;
    a.per = (int)((a.pixels + pieces - 1) / pieces);
    a.pieces = (a.pixels + a.per - 1) / a.per;
}

// Workspace: the images' counters, the parts' sums, the images' totals, the groups' means, and mean and rstd where the caller keeps none.
struct GnormSpace {
    size_t parts, totals, means, stats, bytes;
};
static GnormSpace space_of(const Gnorm* g, long images) {
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    GnormSpace s;
    s.parts = up(sizeof(unsigned) * images);
    s.totals = s.parts + up(sizeof(float2) * (images * g->channels + kGnormTarget * (long)(g->channels < kGnormThreads * 8 ? g->channels : kGnormThreads * 8)));
    s.means = s.totals + up(sizeof(float2) * images * g->channels);
    s.stats = s.means + up(sizeof(float2) * images * g->groups);
    s.bytes = s.stats + up(2 * sizeof(float) * images * g->groups);
    return s;
}
static int ensure_gnorm(Gnorm* g, int images, cudaStream_t s) {
    if (images <= g->images_held) return ensure_scratch(g->ws, space_of(g, g->images_held).bytes, s, "circ_gnorm_reserve");
    const int rc = ensure_scratch(g->ws, space_of(g, images).bytes, s, "circ_gnorm_reserve");
    g->images_held = rc == CIRC_OK ? images : g->ws.ptr ? g->images_held : 0;
    if (rc != CIRC_OK) return rc;
    if (cudaMemsetAsync(g->ws.ptr, 0, space_of(g, images).parts, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaFree(g->ws.ptr);      // this one alone: graphs may hold earlier ones
        g->ws.ptr = nullptr;
        g->ws.bytes = 0;
        g->images_held = 0;
        set_error(CIRC_ERR_CUDA, "clearing the workspace failed: %s", cudaGetErrorString(cudaGetLastError()));
        return CIRC_ERR_CUDA;
    }
    return CIRC_OK;
}

template <typename F>
static void with_act(int act, F&& f) {
    if (act == CIRC_ACT_RELU) f(std::integral_constant<int, CIRC_ACT_RELU>{});
    else if (act == CIRC_ACT_SILU) f(std::integral_constant<int, CIRC_ACT_SILU>{});
    else f(std::integral_constant<int, CIRC_ACT_NONE>{});
}
// Vectors of 8 elements (4 where both tensors are float32) where every one of them is aligned, else single elements.
template <typename T, typename U, typename F>
static void with_vectors(bool aligned, int channels, F&& f) {
    constexpr int VEC = sizeof(T) == 4 && sizeof(U) == 4 ? 4 : 8;
    if (aligned && channels % VEC == 0) f(std::integral_constant<int, VEC>{});
    else f(std::integral_constant<int, 1>{});
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
static GnormArgs args_of(const Gnorm* g, const float* gain, const float* bias, const float* mean, const float* rstd, int N, int H, int W) {
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
    a.pixels = H * W;
    a.eps = g->eps;
    a.arrived = reinterpret_cast<unsigned*>(ws);
    a.parts = reinterpret_cast<float2*>(ws + space.parts);
    a.totals = reinterpret_cast<float2*>(ws + space.totals);
    a.means = reinterpret_cast<float2*>(ws + space.means);
    return a;
}

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
    if ((rc = ensure_gnorm(g, N, s)) != CIRC_OK) return rc;
    GnormArgs a = args_of(g, gain, bias, mean, rstd, N, H, W);
    cudaError_t err = cudaSuccess;
    with_dtype(g->x_dtype, [&](auto* t) {
        with_dtype(g->y_dtype, [&](auto* u) {
            using T = tag_type<decltype(t)>;
            using U = tag_type<decltype(u)>;
            with_vectors<T, U>(!misaligned(x, 16) && !misaligned(y, 16), a.channels, [&](auto vec) {
                constexpr int VEC = decltype(vec)::value;
                lay_out(a, VEC);
                const dim3 grid((unsigned)((long)a.images * a.pieces * a.tiles));
                if ((err = launch_row(gnorm_stats_kernel<T, VEC>, grid, dim3(kGnormThreads), 0, s, static_cast<const T*>(x), a)) != cudaSuccess) return;
                with_act(g->act, [&](auto act) {
                    err = launch_row(gnorm_apply_kernel<T, U, VEC, decltype(act)::value>, grid, dim3(kGnormThreads), 0, s, static_cast<const T*>(x),
                                     static_cast<U*>(y), a);
                });
            });
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(2);
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
    if ((rc = ensure_gnorm(g, N, s)) != CIRC_OK) return rc;
    GnormArgs a = args_of(g, gain, bias, mean, rstd, N, H, W);
    cudaError_t err = cudaSuccess;
    with_dtype(g->x_dtype, [&](auto* t) {
        with_dtype(g->y_dtype, [&](auto* u) {
            using T = tag_type<decltype(t)>;
            using U = tag_type<decltype(u)>;
            with_vectors<T, U>(!misaligned(x, 16) && !misaligned(grad_y, 16) && !misaligned(grad_x, 16), a.channels, [&](auto vec) {
                constexpr int VEC = decltype(vec)::value;
                lay_out(a, VEC);
                with_act(g->act, [&](auto act) {
                    constexpr int ACT = decltype(act)::value;
                    const unsigned blocks = (unsigned)((long)a.images * a.pieces * a.tiles), sums = grad_gain || grad_bias ? (a.channels + 31) / 32 : 0;
                    err = launch_row(gnorm_sums_kernel<T, U, VEC, ACT>, dim3(blocks), dim3(kGnormThreads), 0, s, static_cast<const T*>(x),
                                     static_cast<const U*>(grad_y), a);
                    if (err != cudaSuccess) return;
                    err = launch_row(gnorm_grad_kernel<T, U, VEC, ACT>, dim3((grad_x ? blocks : 0) + sums), dim3(kGnormThreads), 0, s,
                                     static_cast<const T*>(x), static_cast<const U*>(grad_y), static_cast<T*>(grad_x), grad_gain, grad_bias, a);
                });
            });
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(2);
    return CIRC_OK;
}

}  // extern "C"
