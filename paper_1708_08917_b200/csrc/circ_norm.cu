// Root-mean-square norm between circulant layers, with the residual's addition in front of it:
//   s = x + residual,  rstd = 1 / sqrt(mean(s^2) + eps),  y = s rstd gain
// and its gradients, with u = grad_y gain and h = s rstd:
//   grad_x = grad_residual = rstd (u - h mean(u h)) + grad_sum,     grad_gain = sum over rows of grad_y h.
// y in 8 bits (e4m3): values of a group are divided by scale = max|y| / 448 (448: the type's largest value) and rounded.
#include <cuda_fp8.h>

#include <new>
#include <type_traits>

#include "circ_rows.cuh"

namespace circ {

constexpr float kE4m3Max = 448.f;

struct Norm {
    int device;
    int dim;
    float eps;
    int x_dtype, y_dtype, group;
    Scratch ws;
};

__device__ __forceinline__ uint8_t to_e4m3(float v) { return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float from_e4m3(uint8_t v) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)v, __NV_E4M3)));
}

// The scale of a group whose largest magnitude is `top`: 1 for a group of zeros, NaN where a value is not finite (the
// group's values have no meaning then, and the NaN says so), at least the smallest normal number so that it has an inverse.
__device__ __forceinline__ float group_scale(float top) {
    const float scale = fmaxf(top * (1.f / kE4m3Max), 1.17549435e-38f);
    return top == 0.f ? 1.f : top <= 3.402823466e38f ? scale : NAN;
}
__device__ __forceinline__ float inverse(float v) {     // of a normal number, within one unit of the last place
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The e4m3 codes of VEC values, packed (`mine`: the values' lanes that exist).
template <int VEC>
__device__ __forceinline__ void pack_e4m3(const float (&v)[VEC], uint32_t (&w)[VEC / 4]) {
#pragma unroll
    for (int e = 0; e < VEC; e += 4) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[e], v[e + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[e + 2], v[e + 3]), __NV_SATFINITE, __NV_E4M3);
        w[e / 4] = lo | hi << 16;
    }
}

struct NormForward {
    const float* gain;
    float* y_scale;
    float* rstd;
    long rows;
    int dim, group, group_bits;     // group = 2^group_bits unless it is the row
    float eps;
};

// One row per `threads` threads (a warp: several rows a block), every value read once and kept in registers until the row's sum
// is known: the memory traffic is the floor's.  The sum of the residual stream leaves before the reduction.  A whole-row scale comes
// with the same reduction as the mean, from max|s gain| (y = rstd s gain, and rstd > 0).  Bound by memory: 8192 x 9216 bfloat16 with residual
// to 8 bits in groups of 128: 87 us, 6.1 TB/s.  Rows that are not aligned: 117 us against 80 at 16384 x 4095 and 4096.
template <typename TX, typename TY, int VEC, int ITEMS, bool ALIGNED>
__global__ void __launch_bounds__(512) norm_forward_kernel(const TX* x, const TX* residual, TX* sum, TY* y, NormForward a) {
    constexpr bool E4M3 = std::is_same<TY, uint8_t>::value;
    __shared__ float red[2][16];
    pdl_begin();
    const int threads = blockDim.x, tid = threadIdx.x;
    const long row = (long)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= a.rows) return;       // whole warps; blocks of several rows have one warp a row and no barrier
    const RowSpan<VEC, ALIGNED> span(row, a.dim);
    float s[ITEMS][VEC];
    {
        RawVec<TX, VEC> xr[ITEMS], rr[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) span.load(xr[i], x, tid + i * threads);
        if (residual) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) span.load(rr[i], residual, tid + i * threads);
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) rr[i].clear();
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < VEC; e += 2) split(pair_add(xr[i].get2(e), rr[i].get2(e)), s[i][e], s[i][e + 1]);
    }
    if (sum)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) span.store(sum, tid + i * threads, s[i]);
    const bool row_scale = E4M3 && a.group == a.dim;
    Pair squares = pair_of(0.f, 0.f);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) squares = pair_fma(pair_of(s[i][e], s[i][e + 1]), pair_of(s[i][e], s[i][e + 1]), squares);
        if (row_scale) {
            float g[VEC];
            span.load_columns(g, a.gain, tid + i * threads);
#pragma unroll
            for (int e = 0; e < VEC; ++e) top = max_nan(top, fabsf(s[i][e] * g[e]));
        }
    }
    float sq, odd;
    split(squares, sq, odd);
    sq = warp_sum(sq + odd);
    if (row_scale) top = warp_max_nan(top);
    if (threads > 32) {
        const int warps = threads / 32, lane = tid % 32;
        if (lane == 0) {
            red[0][tid / 32] = sq;
            red[1][tid / 32] = top;
        }
        __syncthreads();
        sq = warp_sum(lane < warps ? red[0][lane] : 0.f);
        if (row_scale) top = warp_max_nan(lane < warps ? red[1][lane] : 0.f);
    }
    const float rstd = rsqrtf(sq / (float)a.dim + a.eps);
    if (a.rstd && tid == 0) a.rstd[row] = rstd;
    float inv = 0.f;
    if (row_scale) {
        const float scale = group_scale(top * rstd);
        inv = inverse(scale);
        if (tid == 0) a.y_scale[row] = scale;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int v = tid + i * threads;
        float out[VEC];
        span.load_columns(out, a.gain, v);
#pragma unroll
        for (int e = 0; e < VEC; e += 2)
            split(pair_mul(pair_mul(pair_of(s[i][e], s[i][e + 1]), pair_of(rstd, rstd)), pair_of(out[e], out[e + 1])), out[e], out[e + 1]);
        if constexpr (E4M3) {
            if (!row_scale) {      // the lanes of a group (32, 64 or 128 elements) are neighbours in the warp, and groups do not cross rows
                float t = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) t = max_nan(t, fabsf(out[e]));
                for (int o = a.group / VEC / 2; o > 0; o >>= 1) t = max_nan(t, __shfl_xor_sync(0xffffffffu, t, o));
                const float scale = group_scale(t);
                inv = inverse(scale);
                const int c = span.col(v);
                if (span.any(v) && (c & (a.group - 1)) == 0) a.y_scale[row * (a.dim >> a.group_bits) + (c >> a.group_bits)] = scale;
            }
            // times 1 / scale instead of a division by scale: at most the rounding of a value that lies in the middle between two
            // codes changes
#pragma unroll
            for (int e = 0; e < VEC; e += 2) split(pair_mul(pair_of(out[e], out[e + 1]), pair_of(inv, inv)), out[e], out[e + 1]);
            uint32_t w[VEC / 4];
            pack_e4m3<VEC>(out, w);
            if (!span.any(v)) continue;
            uint8_t* dst = y + span.at(v);
            if (span.whole(v)) {
                if constexpr (VEC == 8)
                    *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
                else
                    *reinterpret_cast<uint32_t*>(dst) = w[0];
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (e >= span.lo(v) && e < span.hi(v)) dst[e] = (uint8_t)(w[e / 4] >> (e % 4 * 8));
            }
        } else {
            span.store(y, v, out);
        }
    }
}

// Rows that do not fit the registers of a block, or tensors that do not start on 16-byte boundaries: element by element, rows
// read again (from L1 / L2) for each step: 211 us against 80 at 16384 x 4096 bfloat16.
template <typename TX, typename TY>
__global__ void __launch_bounds__(512) norm_forward_any_kernel(const TX* x, const TX* residual, TX* sum, TY* y, NormForward a) {
    __shared__ float red[33];
    pdl_begin();
    const int dim = a.dim, group = a.group;
    const size_t row = blockIdx.x, base = row * dim;
    auto value = [&](int c) { return to_float(x[base + c]) + (residual ? to_float(residual[base + c]) : 0.f); };
    auto gained = [&](int c, float rstd) { return value(c) * rstd * (a.gain ? a.gain[c] : 1.f); };
    float sq = 0.f;
    for (int c = threadIdx.x; c < dim; c += blockDim.x) {
        const float v = value(c);
        sq = fmaf(v, v, sq);
    }
    const float rstd = rsqrtf(block_sum(sq, red) / (float)dim + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    if constexpr (std::is_same<TY, uint8_t>::value) {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
        if (group == dim) {
            float top = 0.f;
            for (int c = threadIdx.x; c < dim; c += blockDim.x) top = max_nan(top, fabsf(gained(c, rstd)));
            top = warp_max_nan(top);
            __syncthreads();
            if (lane == 0) red[warp] = top;
            __syncthreads();
            const float scale = group_scale(warp_max_nan(lane < warps ? red[lane] : 0.f));
            if (threadIdx.x == 0) a.y_scale[row] = scale;
            for (int c = threadIdx.x; c < dim; c += blockDim.x) y[base + c] = to_e4m3(gained(c, rstd) * inverse(scale));
        } else {
            for (int g = warp; g < dim / group; g += warps) {
                float top = 0.f;
                for (int c = lane; c < group; c += 32) top = max_nan(top, fabsf(gained(g * group + c, rstd)));
                const float scale = group_scale(warp_max_nan(top));
                if (lane == 0) a.y_scale[row * (dim / group) + g] = scale;
                for (int c = g * group + lane; c < (g + 1) * group; c += 32) y[base + c] = to_e4m3(gained(c, rstd) * inverse(scale));
            }
        }
        __syncthreads();    // sum may be x or residual
        if (sum)
            for (int c = threadIdx.x; c < dim; c += blockDim.x) store_one(sum + base + c, value(c));
    } else {
        for (int c = threadIdx.x; c < dim; c += blockDim.x) {
            const float v = value(c);
            store_one(y + base + c, v * rstd * (a.gain ? a.gain[c] : 1.f));
            if (sum) store_one(sum + base + c, v);
        }
    }
}

// ---- backward ------------------------------------------------------------------------------------------------
// One pass over the tensors gives both gradients: a block walks rows blockIdx.x, + gridDim.x, ..., holds a row in registers while its
// mean(u h) is summed up, and adds grad_y h to its own columns' share of grad_gain, in registers.  The shares of the blocks go to
// `part` [blocks][dim], and a second kernel adds them up in the blocks' order.  16384 x 4096 bfloat16 with grad_sum: 89 us, 6.0 TB/s, issue slots
// two thirds busy; the second kernel takes 6 us more.  16384 x 4095: 121 us together.
struct NormBackward {
    const float* gain;
    const float* rstd;
    float* part;        // NULL: grad_gain is not wanted
    long rows;
    int dim;
};

// A row's reduction waits for all of its loads, so the loads of the next rows must be in flight meanwhile.  RING (a vector a thread, rows
// of at most 16 KB a tensor): they go to a ring of kRowsAhead rows in shared memory, in which every thread copies and reads its own vectors.
// Rows that are not aligned: the blocks are a multiple of VEC, so all rows of a block start at the same place within a vector, and a
// thread has the same columns in each of them.  A vector that is shared with the neighbouring row is copied whole, and what is not the
// row's own is cleared when it is read; only the tensor's last vector, which may end behind it, goes by element.
constexpr int kRowsAhead = 4;

template <typename TX, typename TY, int VEC, int ITEMS, bool ALIGNED, bool RING>
__global__ void __launch_bounds__(RING ? 1024 : 512) norm_backward_kernel(const TX* __restrict__ sum, const TY* __restrict__ dy, const TX* ds, TX* dx, NormBackward a) {
    constexpr int XB = VEC * (int)sizeof(TX), YB = VEC * (int)sizeof(TY), BYTES = 2 * XB + YB;
    static_assert(!RING || ITEMS == 1, "a vector a thread");
    __shared__ __align__(16) float red[2][32];
    pdl_begin();
    const int threads = blockDim.x, tid = threadIdx.x, lane = tid % 32;
    for (int i = tid; i < 2 * 32; i += threads) (&red[0][0])[i] = 0.f;
    __syncthreads();
    extern __shared__ __align__(16) unsigned char smem[];      // the ring
    auto place = [&](int slot, int i, int off) { return smem + (size_t)(slot * ITEMS + i) * BYTES * threads + (size_t)off * threads; };
    Pair acc[ITEMS][VEC / 2];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) acc[i][e] = pair_of(0.f, 0.f);
    const size_t size = (size_t)a.rows * a.dim;
    long ahead = blockIdx.x;
    int slot_in = 0, slot = 0;
    auto fetch = [&]() {
        if (ahead < a.rows) {
            const RowSpan<VEC, ALIGNED> span(ahead, a.dim);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int v = tid + i * threads;
                if (!span.any(v) || (!ALIGNED && span.at(v) + VEC > size)) continue;
                copy_async<XB>(place(slot_in, i, 0) + tid * XB, sum + span.at(v));
                copy_async<YB>(place(slot_in, i, XB) + tid * YB, dy + span.at(v));
                if (ds && dx) copy_async<XB>(place(slot_in, i, XB + YB) + tid * XB, ds + span.at(v));
            }
            ahead += gridDim.x;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        slot_in = slot_in + 1 == kRowsAhead ? 0 : slot_in + 1;
    };
    if constexpr (RING)
#pragma unroll 1
        for (int u = 0; u < kRowsAhead; ++u) fetch();
    // a thread's columns of the gain are the same for every row: they stay in registers where it has one vector
    float kept[VEC];
    if constexpr (RING) RowSpan<VEC, ALIGNED>(blockIdx.x, a.dim).load_columns(kept, a.gain, tid);
    auto gain_of = [&](const RowSpan<VEC, ALIGNED>& span, float (&g)[VEC], int v) {
        if constexpr (RING) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) g[e] = kept[e];
        } else {
            span.load_columns(g, a.gain, v);
        }
    };
    int flip = 0;
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
        RawVec<TX, VEC> sr[ITEMS], cr[ITEMS];
        RawVec<TY, VEC> yr[ITEMS];
        const RowSpan<VEC, ALIGNED> span(row, a.dim);
        const float rstd = __ldg(a.rstd + row);
        if constexpr (RING) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRowsAhead - 1) : "memory");
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int v = tid + i * threads;
                if (!span.any(v) || (!ALIGNED && span.at(v) + VEC > size)) {
                    span.load(sr[i], sum, v);
                    span.load(yr[i], dy, v);
                    if (ds && dx) span.load(cr[i], ds, v);
                    else cr[i].clear();
                    continue;
                }
                sr[i].load(reinterpret_cast<const TX*>(place(slot, i, 0)) + tid * VEC);
                yr[i].load(reinterpret_cast<const TY*>(place(slot, i, XB)) + tid * VEC);
                if (ds && dx) cr[i].load(reinterpret_cast<const TX*>(place(slot, i, XB + YB)) + tid * VEC);
                else cr[i].clear();
                if (!span.whole(v)) {
                    sr[i].keep(span.lo(v), span.hi(v));
                    yr[i].keep(span.lo(v), span.hi(v));
                }
            }
            slot = slot + 1 == kRowsAhead ? 0 : slot + 1;
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) span.load(sr[i], sum, tid + i * threads);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) span.load(yr[i], dy, tid + i * threads);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                if (ds && dx) span.load(cr[i], ds, tid + i * threads);
                else cr[i].clear();
            }
        }
        // grad_y s once for both sums: times the gain for mean(u h), whose factor rstd waits for the end, and times rstd for grad_gain
        Pair dots = pair_of(0.f, 0.f);
        const Pair rs = pair_of(rstd, rstd);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int v = tid + i * threads;
            float g[VEC];
            gain_of(span, g, v);
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const Pair ys = pair_mul(yr[i].get2(e), sr[i].get2(e));
                dots = pair_fma(ys, pair_of(g[e], g[e + 1]), dots);
                acc[i][e / 2] = pair_fma(ys, rs, acc[i][e / 2]);
            }
        }
        float lo, hi;
        split(dots, lo, hi);
        float dot = lo + hi;
        if constexpr (RING) fetch();                  // this row's vectors are in registers
        dot = warp_sum(dot);
        if (lane == 0) red[flip][tid / 32] = dot;
        __syncthreads();                              // the other half of `red` serves the next row
        float mean = 0.f;
        for (int w = 0; w < threads / 32; w += 4) {     // entries of warps that do not exist are zero
            const float4 t = *reinterpret_cast<const float4*>(&red[flip][w]);
            mean += (t.x + t.y) + (t.z + t.w);
        }
        mean *= rstd / (float)a.dim;
        if (!dx) continue;
        // rstd (u - h mean) + grad_sum = rstd u + (grad_sum - s (rstd rstd mean))
        const float back = -rstd * rstd * mean;
        const Pair bk = pair_of(back, back);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float g[VEC];
            gain_of(span, g, tid + i * threads);
#pragma unroll
            for (int e = 0; e < VEC; e += 2)
                split(pair_fma(pair_mul(yr[i].get2(e), pair_of(g[e], g[e + 1])), rs, pair_fma(sr[i].get2(e), bk, cr[i].get2(e))), g[e], g[e + 1]);
            span.store(dx, tid + i * threads, g);
        }
    }
    if (!a.part) return;
    float* part = a.part + (size_t)blockIdx.x * a.dim;
    const RowSpan<VEC, ALIGNED> span(blockIdx.x, a.dim);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int v = tid + i * threads;
        if (!span.any(v)) continue;
        float out[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e += 2) split(acc[i][e / 2], out[e], out[e + 1]);
        if constexpr (ALIGNED) {
            store_vec<VEC>(part + span.col(v), out);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e >= span.lo(v) && e < span.hi(v)) part[span.col(v) + e] = out[e];
        }
    }
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(512) norm_backward_any_kernel(const TX* __restrict__ sum, const TY* __restrict__ dy, const TX* ds, TX* dx, NormBackward a) {
    __shared__ float red[33];
    pdl_begin();
    const int dim = a.dim;
    const size_t row = blockIdx.x, base = row * dim;
    const float rstd = a.rstd[row];
    auto gain = [&](int c) { return a.gain ? a.gain[c] : 1.f; };
    float dot = 0.f;
    for (int c = threadIdx.x; c < dim; c += blockDim.x) dot = fmaf(to_float(dy[base + c]) * gain(c), to_float(sum[base + c]) * rstd, dot);
    dot = block_sum(dot, red) / (float)dim;
    for (int c = threadIdx.x; c < dim; c += blockDim.x)
        store_one(dx + base + c, rstd * (to_float(dy[base + c]) * gain(c) - to_float(sum[base + c]) * rstd * dot) + (ds ? to_float(ds[base + c]) : 0.f));
}
template <typename TX, typename TY>
__global__ void __launch_bounds__(256) norm_gain_any_kernel(const TX* __restrict__ sum, const TY* __restrict__ dy, NormBackward a) {
    pdl_begin();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.dim) return;
    float acc = 0.f;
#pragma unroll 4
    for (long r = blockIdx.y; r < a.rows; r += gridDim.y) acc = fmaf(to_float(dy[r * a.dim + c]), to_float(sum[r * a.dim + c]) * __ldg(a.rstd + r), acc);
    a.part[(size_t)blockIdx.y * a.dim + c] = acc;
}

// grad_gain[c] = part[0][c] + part[1][c] + ...: a block has 32 columns, its warps take consecutive parts.
__global__ void __launch_bounds__(512) norm_gain_kernel(const float* __restrict__ part, float* __restrict__ dgain, int parts, int dim) {
    __shared__ float sums[16][33];
    pdl_begin();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, c = blockIdx.x * 32 + lane;
    const int per = (parts + 15) / 16, from = warp * per, to = from + per < parts ? from + per : parts;
    float s = 0.f;
    if (c < dim)
#pragma unroll 8
        for (int i = from; i < to; ++i) s += part[(size_t)i * dim + c];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < dim) {
#pragma unroll
        for (int w = 1; w < 16; ++w) s += sums[w][lane];
        dgain[c] = s;
    }
}

constexpr int kNormParts = 148 * 4, kGainParts = 64;      // shares of grad_gain: of rows in registers at most, and of others
constexpr int kNormLongest = 32768;                       // longest row that a block's registers hold (512 threads x 8 vectors x 8 elements; 4 beside float32)

// Launch shape of a row kernel: `items` vectors a thread (1, 2, 4 or 8), `threads` a multiple of 32 (at most 512); items 0: the row
// does not fit.  Rows of one warp are put several in a block.
struct RowShape {
    int items, threads;
};
static RowShape row_shape(int vectors, int want_items) {
    for (int items = want_items; items <= 8; items *= 2) {
        const int threads = ((vectors + items - 1) / items + 31) / 32 * 32;
        if (threads <= 512) return RowShape{items, threads};
    }
    return RowShape{0, 0};
}
template <typename F>
static void with_items(int items, F&& f) {
    if (items == 1) f(std::integral_constant<int, 1>{});
    else if (items == 2) f(std::integral_constant<int, 2>{});
    else if (items == 4) f(std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 8>{});
}

// Sixteen values a thread where the tensors allow it; those of a group of 32 or more share their scale.  8192 x 9216 to bfloat16: 41 us,
// 5.6 TB/s.
template <typename TO>
__global__ void __launch_bounds__(256) norm_unpack_kernel(const uint8_t* __restrict__ y, const float* __restrict__ scale, TO* __restrict__ out,
                                                          long count, int group_bits) {
    pdl_begin();
    const long v = blockIdx.x * 256L + threadIdx.x;
    if (v * 16 >= count) return;
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(y) + v);
    const float s = __ldg(scale + (v * 16 >> group_bits));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = from_e4m3((uint8_t)(w[e / 4] >> (e % 4 * 8))) * s;
    store_vec<16>(out + v * 16, x);
}
// Whole-row scales, or tensors that are not aligned.
template <typename TO>
__global__ void __launch_bounds__(256) norm_unpack_any_kernel(const uint8_t* __restrict__ y, const float* __restrict__ scale, TO* __restrict__ out,
                                                              long rows, int dim, int group) {
    pdl_begin();
    for (long row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint8_t* src = y + row * dim;
        const float* sc = scale + row * (dim / group);
        TO* dst = out + row * dim;
#pragma unroll 4
        for (int c = threadIdx.x; c < dim; c += 256) store_one(dst + c, from_e4m3(src[c]) * __ldg(sc + c / group));
    }
}

static int check_norm(const Norm* n, long rows) {
    if (!n) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (rows < 0 || rows > INT32_MAX) {
        set_error(CIRC_ERR_SHAPE, "rows=%ld must be in [0, 2^31)", rows);
        return CIRC_ERR_SHAPE;
    }
    return CIRC_OK;
}
static int norm_group(const Norm* n) { return n->group ? n->group : n->dim; }
static size_t norm_scratch(const Norm* n) { return sizeof(float) * (size_t)(n->dim <= kNormLongest ? kNormParts : kGainParts) * n->dim; }

}  // namespace circ

using namespace circ;

extern "C" {

circ_norm_handle circ_norm_create(int dim, float eps) {
    if (dim < 1 || dim > (1 << 24)) {
        set_error(CIRC_ERR_SHAPE, "dim=%d must be in [1, 2^24]", dim);
        return nullptr;
    }
    if (!(eps >= 0.f) || isinf(eps)) {
        set_error(CIRC_ERR_ARG, "eps=%g must be finite and >= 0", (double)eps);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Norm* n = new (std::nothrow) Norm{device, dim, eps, CIRC_F32, CIRC_F32, 0, {}};
    if (!n) set_error(CIRC_ERR_ALLOC, "host allocation failed");
    return reinterpret_cast<circ_norm_handle>(n);
}

void circ_norm_destroy(circ_norm_handle h) {
    Norm* n = reinterpret_cast<Norm*>(h);
    if (!n) return;
    free_on(n->device, n->ws);
    delete n;
}

int circ_norm_set_dtypes(circ_norm_handle h, int x_dtype, int y_dtype) {
    Norm* n = reinterpret_cast<Norm*>(h);
    if (!n || !float_dtype(x_dtype) || !(float_dtype(y_dtype) || y_dtype == CIRC_E4M3)) {
        set_error(CIRC_ERR_ARG, "bad handle or dtype codes (%d, %d)", x_dtype, y_dtype);
        return CIRC_ERR_ARG;
    }
    n->x_dtype = x_dtype;
    n->y_dtype = y_dtype;
    return CIRC_OK;
}

int circ_norm_set_group(circ_norm_handle h, int group) {
    Norm* n = reinterpret_cast<Norm*>(h);
    if (!n) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (group != 0 && (!(group == 32 || group == 64 || group == 128) || n->dim % group)) {
        set_error(CIRC_ERR_SHAPE, "group=%d must be 0 (a whole row), 32, 64 or 128 and divide dim=%d", group, n->dim);
        return CIRC_ERR_SHAPE;
    }
    n->group = group;
    return CIRC_OK;
}

int circ_norm_reserve(circ_norm_handle h) {
    Norm* n = reinterpret_cast<Norm*>(h);
    const int rc = check_norm(n, 0);
    return rc != CIRC_OK ? rc : ensure_scratch(n->ws, norm_scratch(n), 0, "circ_norm_reserve");
}

int circ_norm_forward(circ_norm_handle h, const void* x, const void* residual, const float* gain, void* sum, void* y, float* y_scale,
                      float* rstd, long rows, void* stream) {
    Norm* n = reinterpret_cast<Norm*>(h);
    int rc = check_norm(n, rows);
    if (rc != CIRC_OK || rows == 0) return rc;
    const bool e4m3 = n->y_dtype == CIRC_E4M3;
    if (!x || !y || y == x || y == residual || y == sum || (e4m3 && !y_scale)) {
        set_error(CIRC_ERR_ARG, "x and y (y_scale too for an 8-bit y) must be non-NULL, y distinct from x, residual and sum");
        return CIRC_ERR_ARG;
    }
    const size_t xb = dtype_bytes(n->x_dtype);
    if (misaligned(x, xb) || misaligned(residual, xb) || misaligned(sum, xb) || misaligned(y, dtype_bytes(n->y_dtype)) || misaligned(gain, 4) ||
        misaligned(y_scale, 4) || misaligned(rstd, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t err = cudaSuccess;
    const NormForward a{gain, y_scale, rstd, rows, n->dim, norm_group(n), n->group == 32 ? 5 : n->group == 64 ? 6 : 7, n->eps};
    with_dtype(n->x_dtype, [&](auto* t) {
        using TX = tag_type<decltype(t)>;
        auto go = [&](auto* o) {
            using TY = tag_type<decltype(o)>;
            // 16 bytes a vector; 8 elements only where no tensor is wider than 16 bits
            constexpr int VEC = std::is_same<TX, float>::value || std::is_same<TY, float>::value ? 4 : 8;
            const TX *xs = static_cast<const TX*>(x), *rs = static_cast<const TX*>(residual);
            TX* ss = static_cast<TX*>(sum);
            TY* ys = static_cast<TY*>(y);
            auto launch = [&](auto aligned) {
                constexpr bool ALIGNED = decltype(aligned)::value;
                const int vectors = RowSpan<VEC, ALIGNED>::most(n->dim);
                // few rows: as many threads as possible, each waits for one vector; many: four vectors in flight a thread
                const RowShape shape = row_shape(vectors, rows <= 148 ? 1 : vectors >= 128 ? 4 : vectors > 32 ? 2 : 1);
                if (!shape.items) return false;
                const int per_block = shape.threads == 32 ? (rows < 148 * 4 ? 1 : 4) : 1;
                with_items(shape.items, [&](auto items) {
                    err = launch_row(norm_forward_kernel<TX, TY, VEC, decltype(items)::value, ALIGNED>, dim3((unsigned)((rows + per_block - 1) / per_block)),
                                     dim3(shape.threads, per_block), 0, s, xs, rs, ss, ys, a);
                });
                return true;
            };
            const bool bases = !misaligned(x, 16) && !misaligned(residual, 16) && !misaligned(sum, 16) && !misaligned(y, 16);
            const bool done = bases && (n->dim % VEC == 0 && !misaligned(gain, 16) ? launch(std::true_type{}) : launch(std::false_type{}));
            if (!done) err = launch_row(norm_forward_any_kernel<TX, TY>, dim3((unsigned)rows), dim3(512), 0, s, xs, rs, ss, ys, a);
        };
        if (e4m3)
            go(static_cast<uint8_t*>(nullptr));
        else
            with_dtype(n->y_dtype, go);
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(1);
    return CIRC_OK;
}

int circ_norm_backward(circ_norm_handle h, const void* sum, const float* gain, const float* rstd, const void* grad_y, const void* grad_sum,
                       void* grad_x, float* grad_gain, long rows, void* stream) {
    Norm* n = reinterpret_cast<Norm*>(h);
    int rc = check_norm(n, rows);
    if (rc != CIRC_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        if (grad_gain) CIRC_CUDA_TRY(cudaMemsetAsync(grad_gain, 0, sizeof(float) * n->dim, s), CIRC_ERR_CUDA);
        return CIRC_OK;
    }
    if (!sum || !rstd || !grad_y || (!grad_x && !grad_gain) || grad_x == sum || grad_x == grad_y) {
        set_error(CIRC_ERR_ARG, "sum, rstd, grad_y and one of grad_x, grad_gain must be non-NULL, grad_x distinct from sum and grad_y");
        return CIRC_ERR_ARG;
    }
    const int gy = n->y_dtype == CIRC_E4M3 ? n->x_dtype : n->y_dtype;
    const size_t xb = dtype_bytes(n->x_dtype);
    if (misaligned(sum, xb) || misaligned(grad_sum, xb) || misaligned(grad_x, xb) || misaligned(grad_y, dtype_bytes(gy)) || misaligned(gain, 4) ||
        misaligned(rstd, 4) || misaligned(grad_gain, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    if (grad_gain && (rc = ensure_scratch(n->ws, norm_scratch(n), s, "circ_norm_reserve")) != CIRC_OK) return rc;
    const NormBackward a{gain, rstd, grad_gain ? static_cast<float*>(n->ws.ptr) : nullptr, rows, n->dim};
    int parts = 0, launches = 0;
    cudaError_t err = cudaSuccess;
    with_dtype(n->x_dtype, [&](auto* t) {
        with_dtype(gy, [&](auto* o) {
            using TX = tag_type<decltype(t)>;
            using TY = tag_type<decltype(o)>;
            constexpr int VEC = std::is_same<TX, float>::value || std::is_same<TY, float>::value ? 4 : 8;
            const TX *ss = static_cast<const TX*>(sum), *cs = static_cast<const TX*>(grad_sum);
            const TY* ys = static_cast<const TY*>(grad_y);
            TX* xs = static_cast<TX*>(grad_x);
            auto launch = [&](auto aligned) {
                constexpr bool ALIGNED = decltype(aligned)::value;
                const int vectors = RowSpan<VEC, ALIGNED>::most(n->dim);
                const RowShape shape = vectors <= 1024 ? RowShape{1, (vectors + 31) / 32 * 32} : row_shape(vectors, 4);
                if (!shape.items) return false;
                auto go = [&](auto items) {
                    constexpr int ITEMS = decltype(items)::value;
                    constexpr bool RING = ITEMS == 1;
                    constexpr int BYTES = VEC * (2 * (int)sizeof(TX) + (int)sizeof(TY));
                    auto kernel = norm_backward_kernel<TX, TY, VEC, ITEMS, ALIGNED, RING>;
                    const size_t smem = RING ? (size_t)kRowsAhead * ITEMS * BYTES * shape.threads : 0;
                    // a wave of blocks that walk the rows, some rows each, and no more shares than kNormParts
                    int per_sm = 1;
                    if ((err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024)) != cudaSuccess) return;
                    if ((err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, shape.threads, smem)) != cudaSuccess) return;
                    const long wave = 148L * (per_sm < 1 ? 1 : per_sm > 4 ? 4 : per_sm), some = (rows + 3) / 4 > 148 ? (rows + 3) / 4 : rows < 148 ? rows : 148;
                    parts = (int)(some < wave ? some : wave);
                    if (!ALIGNED && parts < rows) parts = parts / VEC * VEC;
                    err = launch_row(kernel, dim3(parts), dim3(shape.threads), smem, s, ss, ys, cs, xs, a);
                    ++launches;
                };
                shape.items == 1 ? go(std::integral_constant<int, 1>{}) : shape.items == 4 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 8>{});
                return true;
            };
            const bool bases = !misaligned(sum, 16) && !misaligned(grad_y, 16) && !misaligned(grad_sum, 16) && !misaligned(grad_x, 16);
            const bool done = bases && (n->dim % VEC == 0 && !misaligned(gain, 16) ? launch(std::true_type{}) : launch(std::false_type{}));
            if (done || err != cudaSuccess) return;
            if (grad_x) {
                err = launch_row(norm_backward_any_kernel<TX, TY>, dim3((unsigned)rows), dim3(512), 0, s, ss, ys, cs, xs, a);
                ++launches;
            }
            if (grad_gain && err == cudaSuccess) {
                parts = rows < kGainParts ? (int)rows : kGainParts;
                err = launch_row(norm_gain_any_kernel<TX, TY>, dim3((n->dim + 255) / 256, parts), dim3(256), 0, s, ss, ys, a);
                ++launches;
            }
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    if (grad_gain) {
        CIRC_CUDA_TRY(launch_row(norm_gain_kernel, dim3((n->dim + 31) / 32), dim3(512), 0, s, a.part, grad_gain, parts, n->dim), CIRC_ERR_CUDA);
        ++launches;
    }
    count_launches(launches);
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

int circ_norm_unpack(circ_norm_handle h, const void* y, const float* y_scale, void* out, int out_dtype, long rows, void* stream) {
    Norm* n = reinterpret_cast<Norm*>(h);
    int rc = check_norm(n, rows);
    if (rc != CIRC_OK || rows == 0) return rc;
    if (!y || !y_scale || !out || y == out || !float_dtype(out_dtype) || misaligned(y_scale, 4) || misaligned(out, dtype_bytes(out_dtype))) {
        set_error(CIRC_ERR_ARG, "y, y_scale and out must be non-NULL and aligned to their element sizes, out_dtype CIRC_F32 or CIRC_BF16");
        return CIRC_ERR_ARG;
    }
    const long count = rows * n->dim;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t err = cudaSuccess;
    with_dtype(out_dtype, [&](auto* o) {
        using TO = tag_type<decltype(o)>;
        const uint8_t* q = static_cast<const uint8_t*>(y);
        TO* x = static_cast<TO*>(out);
        if (n->group && !misaligned(y, 16) && !misaligned(out, 16) && count / 16 < (1L << 31) * 256)
            err = launch_row(norm_unpack_kernel<TO>, dim3((unsigned)((count / 16 + 255) / 256)), dim3(256), 0, s, q, y_scale, x, count,
                             n->group == 32 ? 5 : n->group == 64 ? 6 : 7);
        else
            err = launch_row(norm_unpack_any_kernel<TO>, dim3((unsigned)(rows < 148 * 8 ? rows : 148 * 8)), dim3(256), 0, s, q, y_scale, x, rows, n->dim,
                             norm_group(n));
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(1);
    return CIRC_OK;
}

}  // extern "C"
