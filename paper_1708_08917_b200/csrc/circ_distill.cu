// Distillation from a teacher's top logits: the divergence of softmax(z / tau) from the teacher's probabilities, of which a short list of
// classes a row is given, and its gradient (formulas: circ_lists.cuh).
//   mean = sum_r w_r loss_r / sum w;  rows whose weight is not above 0 are not read.
#include <new>
#include <type_traits>

#include "circ_lists.cuh"

namespace circ {

struct Distill {
    int device;
    int classes, count;
    int dtype, values_dtype, ids_type;
    float temperature;
    bool rest, add;
    Scratch ws;
    long rows_held;      // rows that the workspace is laid out for ...
    long lists_held;     // ... and rows that it has room for the lists of
};

// A row's part of the gradient kernel's work.
struct RowPlan {
    float top, factor;   // of the classes outside the list
    float weight;        // 0: nothing to add, zeros to write
    int listed;          // entries of the list that count
};
struct Listed {
    int id;
    float grad;          // before the factor that all rows share
};

struct DistillArgs {
    ListSide side;
    long ld, grad_ld;
    const float* weights;
    float *row_loss, *student_lse, *mean;
    float grad_mean;
    int rows;
    int pieces, per;          // pieces a row, vectors a piece (0: all)
    bool add;
    // workspace
    unsigned* done;           // groups of rows that are finished (0 before and after a call)
    double *weight_sum, *weight_total;      // found with the mean; found beforehand
    unsigned* arrived;        // [rows] pieces that are summed up (0 before and after a call)
    unsigned* grouped;        // [rows / 64] rows that are finished (0 before and after a call)
    double2* sums;            // [rows] weight loss, weight
    double2* group_sums;      // [rows / 64]
    RowPlan* plans;           // [rows]
    Listed* listed;           // [rows][count]
    Softmax* parts;           // [rows][pieces]
};

constexpr int kPieceBits = 32768;        // classes a piece, at most: a bit each says which are listed
constexpr int kPieceThreads = 256;       // of the gradient's pieces

template <int VEC>
struct Piece {
    RowSpan<VEC, false> span;
    int from, to;                        // vectors
    __device__ __forceinline__ Piece(const DistillArgs& a, long row, int piece) : span(row, a.side.classes, a.ld) {
        const int vectors = (a.side.classes - span.shift + VEC - 1) / VEC;
        from = piece * a.per;
        to = a.per ? min(vectors, from + a.per) : vectors;
    }
    // Place of a class in the piece, or -1.
    __device__ __forceinline__ int place(long id) const {
        const long at = id - span.col(from);
        return id >= 0 && id < span.dim && at >= 0 && at < (long)(to - from) * VEC ? (int)at : -1;
    }
};
template <int VEC>
__device__ __forceinline__ unsigned marks_of(const uint32_t* marks, int v) {       // v: vector of the piece
    if constexpr (VEC == 8) return reinterpret_cast<const unsigned char*>(marks)[v];
    else return (marks[v * VEC / 32] >> (v * VEC % 32)) & ((1u << VEC) - 1);
}
// The marked elements of a vector become -inf.
template <typename T, int VEC>
__device__ __forceinline__ void strike(RawVec<T, VEC>& raw, unsigned m) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (m >> e & 1) {
            if constexpr (sizeof(T) == 4) raw.w[e] = 0xff800000u;
            else raw.w[e / 2] = e % 2 ? (raw.w[e / 2] & 0xffffu) | 0xff800000u : (raw.w[e / 2] & 0xffff0000u) | 0xff80u;
        }
}

// The mean: every row leaves weight * loss and weight; the warp that is last in a group of 64 rows adds up the group's, the one that is last of
// all the groups', in their order, in float64.  All lanes of one warp call it.  With many rows the sums are left to a kernel of its own: the counting
// takes a row's last warp 2000 cycles (16384 x 8192 bfloat16: 112 us with it).
constexpr int kMeanGroup = 64;
constexpr int kMeanAlone = 2048;
__device__ __forceinline__ void finish_mean(const DistillArgs& a, int row, double loss, double weight) {
    if (a.rows >= kMeanAlone) {
        if (threadIdx.x % 32 == 0) a.sums[row] = make_double2(weight * loss, weight);
        return;
    }
    const int lane = threadIdx.x % 32, group = row / kMeanGroup, groups = (a.rows + kMeanGroup - 1) / kMeanGroup;
    bool last = false;
    if (lane == 0) {
        a.sums[row] = make_double2(weight * loss, weight);
        __threadfence();
        const unsigned size = min(kMeanGroup, a.rows - group * kMeanGroup);
        last = atomicAdd(a.grouped + group, 1u) == size - 1;
        if (last) a.grouped[group] = 0;
    }
    if (!__shfl_sync(0xffffffffu, last, 0)) return;
    __threadfence();
    double s = 0.0, w = 0.0;
#pragma unroll
    for (int i = 0; i < kMeanGroup; i += 32)
        if (group * kMeanGroup + i + lane < a.rows) {
            const double2 v = __ldcg(a.sums + group * kMeanGroup + i + lane);
            s += v.x;
            w += v.y;
        }
    s = warp_sum(s);
    w = warp_sum(w);
    if (lane == 0) {
        a.group_sums[group] = make_double2(s, w);
        __threadfence();
        last = atomicAdd(a.done, 1u) == (unsigned)groups - 1;
        if (last) *a.done = 0;
    }
    if (!__shfl_sync(0xffffffffu, last, 0)) return;
    __threadfence();
    s = w = 0.0;
#pragma unroll 8
    for (int i = lane; i < groups; i += 32) {
        const double2 v = __ldcg(a.group_sums + i);
        s += v.x;
        w += v.y;
    }
    s = warp_sum(s);
    w = warp_sum(w);
    if (lane == 0) {
        if (a.mean) *a.mean = w > 0.0 ? (float)(s / w) : 0.f;
        *a.weight_sum = w;
    }
}
__global__ void __launch_bounds__(1024) distill_mean_kernel(DistillArgs a) {
    __shared__ double2 part[32];
    pdl_begin();
    double s = 0.0, w = 0.0;
#pragma unroll 8
    for (int r = threadIdx.x; r < a.rows; r += 1024) {
        const double2 v = a.sums[r];
        s += v.x;
        w += v.y;
    }
    s = warp_sum(s);
    w = warp_sum(w);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = make_double2(s, w);
    __syncthreads();
    if (threadIdx.x >= 32) return;
    s = warp_sum(part[threadIdx.x].x);
    w = warp_sum(part[threadIdx.x].y);
    if (threadIdx.x == 0) {
        if (a.mean) *a.mean = w > 0.0 ? (float)(s / w) : 0.f;
        *a.weight_sum = w;
    }
}
// The sum of the weights above 0, for a gradient that is written along with the losses.
__global__ void __launch_bounds__(1024) distill_weights_kernel(DistillArgs a) {
    __shared__ double part[32];
    pdl_begin();
    double w = 0.0;
#pragma unroll 8
    for (int r = threadIdx.x; r < a.rows; r += 1024) {
        const float v = a.weights[r];
        w += v > 0.f ? (double)v : 0.0;
    }
    w = warp_sum(w);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = w;
    __syncthreads();
    if (threadIdx.x < 32) {
        w = warp_sum(part[threadIdx.x]);
        if (threadIdx.x == 0) *a.weight_total = w;
    }
}
constexpr int kWeightsAlone = 512;       // rows from which on a kernel of its own adds up the weights
// The factor that a row's gradients share; one warp calls it.
__device__ __forceinline__ float shared_factor(const DistillArgs& a, float weight) {
    double total = (double)a.rows;
    if (a.weights && a.rows > kWeightsAlone) {
        total = __ldcg(a.weight_total);
    } else if (a.weights) {
        total = 0.0;
#pragma unroll 4
        for (int r = threadIdx.x % 32; r < a.rows; r += 32) {
            const float v = a.weights[r];
            total += v > 0.f ? (double)v : 0.0;
        }
        total = warp_sum(total);
    }
    return (float)((double)a.grad_mean * (double)weight / total * a.side.inv_tau);
}

// Gradients of a vector: exponentials * factor, on top of what is there if `add`.
template <bool PLAIN, typename T, int VEC>
__device__ __forceinline__ void slopes(const RawVec<T, VEC>& raw, const Exponent& ex, float factor, bool add, const T* old, float (&g)[VEC]) {
    float s[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = raw.get(e);
    ex.powers<PLAIN>(s, g);
    if (add) {
        RawVec<T, VEC> was;
        was.load(old);
#pragma unroll
        for (int e = 0; e < VEC; ++e) g[e] = fmaf(g[e], factor, was.get(e));
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) g[e] *= factor;
    }
}

// ---- rows, or pieces of them, a block each ----
// Bound by memory for long rows: 4096 x 50001 bfloat16 without a gradient 86 us (one in ten rows without weight; 4.3 TB/s of what is read), by the list's
// chain of dependent steps (6 us) for those of a few thousand classes.  With a gradient 8192 x 50001 bfloat16 take 363 us (4.3 TB/s): two exponentials an
// element keep the XU pipe half busy, and blocks wait at the barriers between their phases; rows held in shared memory (as the cross entropy's are) take
// the same time.
// THREADS threads sum up the classes that are not listed, four vectors at a time (the first four are on their way before the list is known); one more
// warp has the list: it marks its classes, works out the teacher's side meanwhile, and then the row's loss.  GRAD: the row is read a second time, from
// L2, where its block's neighbours have left room for it, and the gradient written; the list's own elements follow behind a barrier.
// PIECES: the warp that is last to finish a row's pieces works out its loss, and with `plans` what distill_grad_kernel needs.
template <int WARPS, int MOST, bool PIECES>
struct RowSpace {
    ListSpace<MOST> list;
    uint32_t table[PIECES ? 2 * MOST : 1];
    Softmax part[WARPS];
    float top, factor;
    bool zero;
};
constexpr int kAhead = 4;

template <typename T, typename V, typename ID, int VEC, int THREADS, int MOST, bool GRAD, bool PIECES>
__global__ void __launch_bounds__(THREADS + 32, PIECES ? 1 : 1280 / (THREADS + 32))
    distill_rows_kernel(const T* z, const V* __restrict__ values, const ID* __restrict__ ids, T* grad, DistillArgs a) {
    static_assert(!(GRAD && PIECES) && (VEC > 1 || PIECES), "");
    constexpr int WARPS = THREADS / 32;
    extern __shared__ __align__(16) uint32_t marks[];
    __shared__ RowSpace<WARPS, MOST, PIECES> space;
    pdl_begin();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int row = PIECES ? blockIdx.x / a.pieces : blockIdx.x, piece = PIECES ? blockIdx.x % a.pieces : 0;
    const float weight = a.weights ? a.weights[row] : 1.f;
    const bool live = weight > 0.f;
    const Piece<VEC> p(a, row, piece);
    const int w0 = p.span.whole(p.from) ? p.from : p.from + 1, w1 = p.to > w0 && !p.span.whole(p.to - 1) ? p.to - 1 : p.to, whole = w1 - w0;
    const T* zr = z + (size_t)row * a.ld;
    // the vectors that are not whole: one for each of the first two threads, or -1
    const int rest = tid == 0 && w0 > p.from ? p.from : tid == 1 && w1 < p.to ? p.to - 1 : -1;
    if (warp == WARPS) {
        TeacherList<MOST> list(space.list);
        if (live) {
            list.fetch(a.side, values, ids, (size_t)row, zr);
            __syncthreads();
            auto mark = [&](int id) {      // false: it is marked already
                const int at = p.place(id);
                return at >= 0 && !(atomicOr(marks + at / 32, 1u << at % 32) >> at % 32 & 1);
            };
            if constexpr (PIECES) {        // the marks are those of the piece
                for (int k = lane; k < a.side.count; k += 32) mark(list.at.id[k]);
                __syncthreads();
                list.keep_first(a.side, space.table);
            } else {
                list.keep_first(a.side, mark);
                __syncthreads();
            }
            list.prepare(a.side);
        }
        const float scale = GRAD && live ? shared_factor(a, weight) : 0.f;
        double loss = 0.0, lse = 0.0;
        RowPlan plan{-INFINITY, 0.f, 0.f, 0};
        ListRow r{};
        bool zero = true;
        if (live || PIECES) {
            Softmax outside{-INFINITY, 0.f};
            if (live) {
                __syncthreads();
                outside = warp_join(lane < WARPS ? space.part[lane] : outside, a.side.scale);
            }
            if (PIECES && a.pieces > 1) {
                bool last = false;
                if (lane == 0) {
                    a.parts[(size_t)row * a.pieces + piece] = outside;
                    __threadfence();
                    last = atomicAdd(a.arrived + row, 1u) == (unsigned)a.pieces - 1;
                    if (last) a.arrived[row] = 0;
                }
                if (!__shfl_sync(0xffffffffu, last, 0)) return;
                __threadfence();
                outside = Softmax{-INFINITY, 0.f};
                for (int i = lane; i < a.pieces; i += 32) {
                    const float2 other = __ldcg(reinterpret_cast<const float2*>(a.parts) + (size_t)row * a.pieces + i);
                    outside = join(outside, Softmax{other.x, other.y}, a.side.scale);
                }
                outside = warp_join(outside, a.side.scale);
            }
            if (live) {
                r = list.finish(a.side, outside);
                zero = r.zero;
                if (GRAD && lane == 0) {
                    space.top = r.top;
                    space.factor = r.factor * scale;
                    space.zero = zero;
                }
                if (GRAD && a.add && !zero)      // what is there now, before the others write over it
                    for (int k = lane; k < a.side.count; k += 32)
                        if (list.at.id[k] >= 0) list.at.t[k] = fmaf(list.slope(r, k), scale, to_float(grad[(size_t)row * a.grad_ld + list.at.id[k]]));
                if (GRAD) __syncthreads();
                list.losses(a.side, r, loss, lse);
                if (PIECES && a.plans) {
                    int n = 0;
                    for (int k0 = 0; k0 < a.side.count; k0 += 32) {
                        const int k = k0 + lane, id = k < a.side.count ? list.at.id[k] : -1;
                        const unsigned have = __ballot_sync(0xffffffffu, id >= 0);
                        if (id >= 0) a.listed[(size_t)row * a.side.count + n + __popc(have & ((1u << lane) - 1))] = Listed{id, list.slope(r, k)};
                        n += __popc(have);
                    }
                    plan = RowPlan{r.top, r.factor, zero ? 0.f : weight, n};
                }
            }
        }
        if (lane == 0) {
            if (a.row_loss) a.row_loss[row] = (float)loss;
            if (a.student_lse) a.student_lse[row] = (float)lse;
            if (PIECES && a.plans) a.plans[row] = plan;
        }
        finish_mean(a, row, loss, live ? (double)weight : 0.0);
        if (GRAD && live) {
            __syncthreads();
            if (!zero)
                for (int k = lane; k < a.side.count; k += 32)
                    if (list.at.id[k] >= 0) store_one(grad + (size_t)row * a.grad_ld + list.at.id[k], a.add ? list.at.t[k] : list.slope(r, k) * scale);
        }
        return;
    }
    const T* src = z + p.span.at(w0) + (size_t)tid * VEC;
    if (live) {
        RawVec<T, VEC> raw[kAhead];
        const bool full = tid + (kAhead - 1) * THREADS < whole;
        if (full)
#pragma unroll
            for (int u = 0; u < kAhead; ++u) raw[u].load(src + u * THREADS * VEC);
        for (int i = tid; i < ((p.to - p.from) * VEC + 31) / 32; i += THREADS) marks[i] = 0;
        __syncthreads();
        __syncthreads();      // the list is marked
        Running run(a.side.scale);
        auto take = [&](auto& some) {
            if constexpr (VEC > 1) {
                run.take(some);
            } else {
                float s[sizeof(some) / sizeof(some[0])];
#pragma unroll
                for (int u = 0; u < (int)(sizeof(some) / sizeof(some[0])); ++u) s[u] = some[u].get(0);
                run.take(s);
            }
        };
        int i = tid;
        for (bool ready = full; i + (kAhead - 1) * THREADS < whole; i += kAhead * THREADS, ready = false) {
            if (!ready)
#pragma unroll
                for (int u = 0; u < kAhead; ++u) raw[u].load(src + (size_t)(i - tid + u * THREADS) * VEC);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const unsigned m = marks_of<VEC>(marks, w0 - p.from + i + u * THREADS);
                if (m) strike(raw[u], m);
            }
            take(raw);
        }
        if (i < whole) {      // the last vectors together too
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                raw[u].fill_lowest();
                if (i + u * THREADS < whole) raw[u].load(src + (size_t)(i - tid + u * THREADS) * VEC);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (i + u * THREADS < whole) {
                    const unsigned m = marks_of<VEC>(marks, w0 - p.from + i + u * THREADS);
                    if (m) strike(raw[u], m);
                }
            take(raw);
        }
        if (rest >= 0) {
            RawVec<T, VEC> one;
            float s[VEC];
            p.span.load(one, z, rest);
            strike(one, marks_of<VEC>(marks, rest - p.from));
            scores(p.span, rest, one, s);
            run.take(s);
        }
        const Softmax all = warp_join(run.done(), a.side.scale);
        if (lane == 0) space.part[warp] = all;
        __syncthreads();
    }
    if constexpr (GRAD) {
        bool zero = true;
        float factor = 0.f;
        Exponent ex(-INFINITY, a.side.scale);
        if (live) {
            __syncthreads();
            zero = space.zero;
            factor = space.factor;
            ex = Exponent(space.top, a.side.scale);
        }
        T* const g0 = grad + (size_t)row * a.grad_ld + p.span.shift;
        T* dst = g0 + (size_t)(w0 + tid) * VEC;
        if (zero) {
            if (!a.add) {
                const float none[VEC] = {};
                for (int i = tid; i < whole; i += THREADS) store_vec_once<VEC>(dst + (size_t)(i - tid) * VEC, none);
            }
        } else {
            auto put = [&](auto plain) {
                int i = tid;
                for (; i + (kAhead - 1) * THREADS < whole; i += kAhead * THREADS) {
                    RawVec<T, VEC> raw[kAhead];
                    const size_t o = (size_t)(i - tid) * VEC;
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) raw[u].load(src + o + u * THREADS * VEC);
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        float g[VEC];
                        slopes<decltype(plain)::value>(raw[u], ex, factor, a.add, dst + o + u * THREADS * VEC, g);
                        store_vec_once<VEC>(dst + o + u * THREADS * VEC, g);
                    }
                }
                if (i < whole) {
                    RawVec<T, VEC> raw[kAhead];
                    const size_t o = (size_t)(i - tid) * VEC;
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (i + u * THREADS < whole) raw[u].load(src + o + u * THREADS * VEC);
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (i + u * THREADS < whole) {
                            float g[VEC];
                            slopes<decltype(plain)::value>(raw[u], ex, factor, a.add, dst + o + u * THREADS * VEC, g);
                            store_vec_once<VEC>(dst + o + u * THREADS * VEC, g);
                        }
                }
            };
            if (ex.plain) put(std::true_type{});
            else put(std::false_type{});
        }
        if (rest >= 0 && !(zero && a.add)) {
            RawVec<T, VEC> raw;
            float s[VEC], g[VEC];
            if (zero) raw.clear();
            else p.span.load(raw, z, rest);
            scores(p.span, rest, raw, s);
            ex.of(s, g);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e >= p.span.lo(rest) && e < p.span.hi(rest)) {
                    T* at = g0 + (size_t)rest * VEC + e;
                    store_one(at, zero ? 0.f : a.add ? fmaf(g[e], factor, to_float(*at)) : g[e] * factor);
                }
        }
        if (live) __syncthreads();
    }
}

// ---- short rows: a warp holds one in registers ----
// Bound by the list's chain of dependent steps: 128 x 1024 float32 with gradient 8.9 us a call, 16384 x 200 34 us.
template <typename T, typename V, typename ID, int VEC, int N, int MOST, bool GRAD>
__global__ void __launch_bounds__(128) distill_warp_kernel(const T* z, const V* __restrict__ values, const ID* __restrict__ ids, T* grad, DistillArgs a) {
    __shared__ uint32_t marks_of_warp[4][N * VEC];
    __shared__ ListSpace<MOST> lists[4];
    pdl_begin();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, row = blockIdx.x * 4 + warp;
    if (row >= a.rows) return;
    uint32_t* marks = marks_of_warp[warp];
    const float weight = a.weights ? a.weights[row] : 1.f;
    const bool live = weight > 0.f;
    const Piece<VEC> p(a, row, 0);
    const auto& span = p.span;
    T* const gr = GRAD ? grad + (size_t)row * a.grad_ld : nullptr;
    double loss = 0.0, lse = 0.0;
    bool zero = true;
    if (live) {
        RawVec<T, VEC> raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) span.load(raw[i], z, i * 32 + lane);
        for (int i = lane; i < N * VEC; i += 32) marks[i] = 0;
        TeacherList<MOST> list(lists[warp]);
        list.fetch(a.side, values, ids, (size_t)row, z + (size_t)row * a.ld);
        __syncwarp();
        list.keep_first(a.side, [&](int id) {
            const int at = p.place(id);
            return !(atomicOr(marks + at / 32, 1u << at % 32) >> at % 32 & 1);
        });
        __syncwarp();
        Running run(a.side.scale);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int v = i * 32 + lane;
            if (span.any(v)) strike(raw[i], marks_of<VEC>(marks, v));
            float s[VEC];
            scores(span, v, raw[i], s);
            run.take(s);
        }
        const Softmax outside = warp_join(run.done(), a.side.scale);
        list.prepare(a.side);
        const ListRow r = list.finish(a.side, outside);
        list.losses(a.side, r, loss, lse);
        zero = r.zero;
        if (GRAD && !zero) {
            const float scale = shared_factor(a, weight), factor = r.factor * scale;
            const Exponent ex(r.top, a.side.scale);
            for (int k = lane; k < a.side.count; k += 32)
                if (list.at.id[k] >= 0) list.at.t[k] = a.add ? fmaf(list.slope(r, k), scale, to_float(gr[list.at.id[k]])) : list.slope(r, k) * scale;
            __syncwarp();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int v = i * 32 + lane;
                if (!span.any(v)) continue;
                float s[VEC], g[VEC];
                scores(span, v, raw[i], s);
                ex.of(s, g);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const bool in = e >= span.lo(v) && e < span.hi(v);
                    g[e] = a.add && in ? fmaf(g[e], factor, to_float(gr[span.col(v) + e])) : g[e] * factor;
                }
                if (span.whole(v)) {
                    store_vec_once<VEC>(gr + span.col(v), g);
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (e >= span.lo(v) && e < span.hi(v)) store_one(gr + span.col(v) + e, g[e]);
                }
            }
            __syncwarp();
            for (int k = lane; k < a.side.count; k += 32)
                if (list.at.id[k] >= 0) store_one(gr + list.at.id[k], list.at.t[k]);
        }
    }
    if (GRAD && zero && !a.add)
        for (int c = lane; c < a.side.classes; c += 32) store_one(gr + c, 0.f);
    if (lane == 0) {
        if (a.row_loss) a.row_loss[row] = (float)loss;
        if (a.student_lse) a.student_lse[row] = (float)lse;
    }
    finish_mean(a, row, loss, live ? (double)weight : 0.0);
}

// One bit for each listed class of the piece.
template <int VEC, typename ID>
__device__ __forceinline__ void mark_listed(const DistillArgs& a, const Piece<VEC>& p, const ID* __restrict__ ids, size_t row, uint32_t* marks) {
    for (int i = threadIdx.x; i < kPieceBits / 32; i += kPieceThreads) marks[i] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < a.side.count; k += kPieceThreads) {
        const int at = p.place((long)ids[row * a.side.count + k]);
        if (at >= 0) atomicOr(marks + at / 32, 1u << at % 32);
    }
    __syncthreads();
}

// The gradient of pieces of rows, from the rows' plans.
template <typename T, typename ID, int VEC>
__global__ void __launch_bounds__(kPieceThreads) distill_grad_kernel(const T* z, const ID* __restrict__ ids, T* grad, DistillArgs a) {
    __shared__ uint32_t marks[kPieceBits / 32];
    pdl_begin();
    const int tid = threadIdx.x, row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
    const RowPlan plan = a.plans[row];
    const bool zero = plan.weight == 0.f;
    if (zero && a.add) return;
    const Piece<VEC> p(a, row, piece);
    const float shared_factor = (float)((double)a.grad_mean * (double)plan.weight / *a.weight_sum * a.side.inv_tau);
    const Exponent ex(plan.top, a.side.scale);
    const float factor = plan.factor * shared_factor;
    T* g = grad + (size_t)row * a.grad_ld;
    if (!zero) mark_listed(a, p, ids, (size_t)row, marks);
    for (int v0 = p.from + tid; v0 < p.to; v0 += kAhead * kPieceThreads) {
        RawVec<T, VEC> raw[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            raw[u].clear();
            if (!zero && v0 + u * kPieceThreads < p.to) p.span.load(raw[u], z, v0 + u * kPieceThreads);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int v = v0 + u * kPieceThreads, col = p.span.col(v);
            if (v >= p.to) break;
            const unsigned m = zero ? 0 : marks_of<VEC>(marks, v - p.from);
            float s[VEC], out[VEC];
            scores(p.span, v, raw[u], s);
            ex.of(s, out);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                out[e] = zero ? 0.f : out[e] * factor;
                if (a.add && !(m >> e & 1) && col + e >= 0 && col + e < a.side.classes) out[e] += to_float(g[col + e]);
            }
            if (VEC > 1 && p.span.whole(v) && !m) {
                store_vec<VEC>(g + col, out);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (col + e >= 0 && col + e < a.side.classes && !(m >> e & 1)) store_one(g + col + e, out[e]);
            }
        }
    }
    if (zero) return;
    for (int k = tid; k < plan.listed; k += kPieceThreads) {
        const Listed l = a.listed[(size_t)row * a.side.count + k];
        if (p.place(l.id) >= 0) {
            const float v = l.grad * shared_factor;
            store_one(g + l.id, a.add ? v + to_float(g[l.id]) : v);
        }
    }
}

constexpr long kPieceTarget = 148 * 8;      // blocks that fill the machine
// Fewer rows, each longer, are cut into pieces: with so few a block's own time for a row is longer than that of pieces and their joining.  Blocks and pieces, us: 140000
// classes float32 without gradient, 1 row 14.8 and 11.4, 12 rows 15.4 and 11.4, 24 rows 15.7 and 13.5; with gradient 24.5 and 15.7, 24.4 and 19.4, 25.2 and 24.8; bfloat16 with
// gradient 18.1 and 16.5, 18.0 and 18.8, 18.1 and 21.6.  8 rows of 50000 float32 (200 KB): 10.6 and 10.9, with gradient 13.0 and 15.9; of 80000: 12.0 and 11.0, 15.8 and 16.3.
constexpr int kFewRows = 16;
constexpr size_t kFewBytes = 256 * 1024;
constexpr size_t kMarksMost = 48 * 1024 * 8;      // classes a row whose marks a block holds

// Pieces a row: enough for the marks, and more while the rows do not fill the machine (4 vectors a thread left at least).
static int pieces_of(long rows, int classes, int vec, int* per) {
    const long vectors = ((long)classes + 2 * vec - 2) / vec, most = kPieceBits / vec;
    long pieces = (vectors + most - 1) / most;
    const long want = (kPieceTarget / 2 + rows - 1) / rows, can = vectors / (kAhead * kPieceThreads);
    const long split = want < can ? want : can;
    if (split > pieces) pieces = split;
    if (pieces < 1) pieces = 1;
    *per = (int)((vectors + pieces - 1) / pieces);
    return (int)((vectors + *per - 1) / *per);
}

// How a call is run: rows, or pieces of them by vectors or by elements.
enum class Walk { rows, pieces, elements };
static Walk walk_of(const Distill* d, const void* z, long ld, const void* grad, long grad_ld, long rows) {
    const int vec = 16 / (int)dtype_bytes(d->dtype);
    if (misaligned(z, 16) || misaligned(grad, 16) || (grad && (ld - grad_ld) % vec)) return Walk::elements;
    const long vectors = ((long)d->classes + 2 * vec - 2) / vec;
    int per;
    const bool few = vectors > 256 && pieces_of(rows, d->classes, vec, &per) > 1 && rows < kFewRows && (size_t)vectors * 16 > kFewBytes;
    return few || (size_t)vectors * vec > kMarksMost ? Walk::pieces : Walk::rows;
}

// Workspace: counters (256 bytes), the rows' counters, their sums and plans, and the pieces' sums, for `rows` rows; the lists' gradients for `lists` rows.
struct DistillSpace {
    size_t arrived, grouped, sums, group_sums, plans, parts, listed, bytes;
};
static DistillSpace space_of(const Distill* d, long rows, long lists) {
    DistillSpace s;
    const size_t least = ((size_t)d->classes + kPieceBits / 2 - 1) / (kPieceBits / 2) + 1;      // pieces a row where rows fill the machine
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    s.arrived = 256;
    s.grouped = s.arrived + up(sizeof(unsigned) * rows);
    s.sums = s.grouped + up(sizeof(unsigned) * (rows / kMeanGroup + 1));
    s.group_sums = s.sums + up(sizeof(double2) * rows);
    s.plans = s.group_sums + up(sizeof(double2) * (rows / kMeanGroup + 1));
    s.parts = s.plans + up(sizeof(RowPlan) * rows);
    s.listed = s.parts + up(sizeof(Softmax) * (rows * least + 2 * kPieceTarget));
    s.bytes = s.listed + up(sizeof(Listed) * lists * d->count);
    return s;
}
// Only calls in pieces use the lists' room.  Others hold it up to this size all the same, for a call that follows; a forward call over 2^20 rows with lists of 256
// would hold 2 GB.
constexpr size_t kListsAnyway = 64 << 20;
// Clears what it has just allocated, nothing else: the counters of a workspace in use are 0 between calls, and numbers of rows and lists that need the same bytes
// have the same layout, since no section shrinks as they grow.
static int ensure_distill(Distill* d, long rows, bool pieces, cudaStream_t s) {
    const long held = rows > d->rows_held ? rows : d->rows_held, want = pieces || sizeof(Listed) * rows * d->count <= kListsAnyway ? rows : 0;
    const long lists = want > d->lists_held ? want : d->lists_held;
    const DistillSpace space = space_of(d, held, lists);
    const bool fresh = d->ws.bytes < space.bytes;
    const int rc = ensure_scratch(d->ws, space.bytes, s, "circ_distill_reserve");
    if (rc != CIRC_OK) {
        if (!d->ws.ptr) d->rows_held = d->lists_held = 0;
        return rc;
    }
    d->rows_held = held;
    d->lists_held = lists;
    if (!fresh) return CIRC_OK;
    if (cudaMemsetAsync(d->ws.ptr, 0, space.sums, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaFree(d->ws.ptr);      // this one alone: graphs may hold earlier ones
        d->ws.ptr = nullptr;
        d->ws.bytes = 0;
        d->rows_held = d->lists_held = 0;
        set_error(CIRC_ERR_CUDA, "clearing the workspace failed: %s", cudaGetErrorString(cudaGetLastError()));
        return CIRC_ERR_CUDA;
    }
    return CIRC_OK;
}

// The kernel for a call, by the rows' length, their number and the alignment.
template <typename T, typename V, typename ID>
static cudaError_t dispatch_distill(Walk walk, const T* z, const V* values, const ID* ids, T* grad, DistillArgs a, cudaStream_t s, int* launches) {
    constexpr int VEC = 16 / (int)sizeof(T);
    cudaError_t err = cudaSuccess;
    auto go = [&](auto kernel, long blocks, int threads, size_t smem, auto... args) {
        if (err != cudaSuccess) return;
        if (blocks >= 1L << 31) {
            err = cudaErrorInvalidConfiguration;
            return;
        }
        if (smem > 32 * 1024) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (err == cudaSuccess) err = launch_row(kernel, dim3((unsigned)blocks), dim3(threads), smem, s, args..., a);
        ++*launches;
    };
    auto with_list = [&](auto f) {
        if (a.side.count <= 64) f(std::integral_constant<int, 64>{});
        else f(std::integral_constant<int, kListMost>{});
    };
    auto in_pieces = [&](auto vec) {
        constexpr int N = decltype(vec)::value;
        a.pieces = pieces_of(a.rows, a.side.classes, N, &a.per);
        const long blocks = (long)a.rows * a.pieces;
        with_list([&](auto most) {
            go(distill_rows_kernel<T, V, ID, N, kPieceThreads, decltype(most)::value, false, true>, blocks, kPieceThreads + 32,
               ((size_t)a.per * N + 31) / 32 * 4, z, values, ids, static_cast<T*>(nullptr));
        });
        if (a.rows >= kMeanAlone) go(distill_mean_kernel, 1, 1024, 0);
        if (grad) go(distill_grad_kernel<T, ID, N>, blocks, kPieceThreads, 0, z, ids, grad);
    };
    if (walk == Walk::elements) {
        in_pieces(std::integral_constant<int, 1>{});
        return err;
    }
    if (walk == Walk::pieces) {
        in_pieces(std::integral_constant<int, VEC>{});
        return err;
    }
    const int vectors = RowSpan<VEC, false>::most(a.side.classes);
    const size_t marks = ((size_t)vectors * VEC + 31) / 32 * 4, bytes = (size_t)vectors * 16;
    a.pieces = 1;
    a.per = 0;
    auto with_grad = [&](auto gradient) {
        constexpr bool GRAD = decltype(gradient)::value;
        if (GRAD && a.weights && a.rows > kWeightsAlone) go(distill_weights_kernel, 1, 1024, 0);
        with_list([&](auto most) {
            constexpr int MOST = decltype(most)::value;
            auto rows = [&](auto threads) {
                constexpr int THREADS = decltype(threads)::value;
                go(distill_rows_kernel<T, V, ID, VEC, THREADS, MOST, GRAD, false>, a.rows, THREADS + 32, marks, z, values, ids, grad);
            };
            auto warps = [&](auto n) {
                go(distill_warp_kernel<T, V, ID, VEC, decltype(n)::value, MOST, GRAD>, (a.rows + 3L) / 4, 128, 0, z, values, ids, grad);
            };
            if (vectors <= 32) warps(std::integral_constant<int, 1>{});
            else if (vectors <= 64) warps(std::integral_constant<int, 2>{});
            else if (vectors <= 128) warps(std::integral_constant<int, 4>{});
            else if (vectors <= 256) warps(std::integral_constant<int, 8>{});
            // small blocks, whose waits overlap; with a gradient no more of them than L2 holds the rows of
            else if (a.rows < 148 * 2) rows(std::integral_constant<int, 512>{});      // (fewer than the machine holds: a row's own time counts)
            else if (!GRAD || bytes <= 32 * 1024) rows(std::integral_constant<int, 128>{});
            else if (bytes <= 128 * 1024) rows(std::integral_constant<int, 256>{});
            else rows(std::integral_constant<int, 512>{});
        });
        if (a.rows >= kMeanAlone && a.mean) go(distill_mean_kernel, 1, 1024, 0);
    };
    grad ? with_grad(std::true_type{}) : with_grad(std::false_type{});
    return err;
}

static int run_distill(Distill* d, const void* z, long ld, const void* values, const void* ids, const float* lse, const float* weights, float* row_loss,
                       float* student_lse, float* mean, void* grad, long grad_ld, float grad_mean, long rows, cudaStream_t s) {
    if (!d) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (rows < 0 || rows > (1L << 24) || ld < d->classes || (grad && grad_ld < d->classes)) {
        set_error(CIRC_ERR_SHAPE, "rows=%ld must be in [0, 2^24] and the strides (%ld, %ld) at least classes=%d", rows, ld, grad_ld, d->classes);
        return CIRC_ERR_SHAPE;
    }
    if (rows == 0) {
        if (mean) CIRC_CUDA_TRY(cudaMemsetAsync(mean, 0, sizeof(float), s), CIRC_ERR_CUDA);
        return CIRC_OK;
    }
    if (!z || !values || !ids || (d->rest ? !lse : lse != nullptr)) {
        set_error(CIRC_ERR_ARG, "logits, values and ids must be non-NULL, and the teacher's lse with the rest, NULL without");
        return CIRC_ERR_ARG;
    }
    if (grad == z && (grad_ld != ld || d->add)) {
        set_error(CIRC_ERR_ARG, "a gradient in the place of the logits needs their stride, and cannot be added to them");
        return CIRC_ERR_ARG;
    }
    const size_t zb = dtype_bytes(d->dtype);
    if (misaligned(z, zb) || misaligned(grad, zb) || misaligned(values, dtype_bytes(d->values_dtype)) || misaligned(ids, d->ids_type == CIRC_I64 ? 8 : 4) ||
        misaligned(lse, 4) || misaligned(weights, 4) || misaligned(row_loss, 4) || misaligned(student_lse, 4) || misaligned(mean, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    const Walk walk = walk_of(d, z, ld, grad, grad_ld, rows);
    const int rc = ensure_distill(d, rows, walk != Walk::rows, s);
    if (rc != CIRC_OK) return rc;
    const DistillSpace space = space_of(d, d->rows_held, d->lists_held);
    char* ws = static_cast<char*>(d->ws.ptr);
    DistillArgs a{};
    a.side = ListSide{lse, 1.0 / (double)d->temperature, (float)(1.4426950408889634 / (double)d->temperature), d->classes, d->count, d->rest};
    a.ld = ld;
    a.grad_ld = grad_ld;
    a.weights = weights;
    a.row_loss = row_loss;
    a.student_lse = student_lse;
    a.mean = mean;
    a.grad_mean = grad_mean;
    a.rows = (int)rows;
    a.add = d->add;
    a.done = reinterpret_cast<unsigned*>(ws);
    a.weight_sum = reinterpret_cast<double*>(ws + 8);
    a.weight_total = reinterpret_cast<double*>(ws + 16);
    a.grouped = reinterpret_cast<unsigned*>(ws + space.grouped);
    a.group_sums = reinterpret_cast<double2*>(ws + space.group_sums);
    a.arrived = reinterpret_cast<unsigned*>(ws + space.arrived);
    a.sums = reinterpret_cast<double2*>(ws + space.sums);
    a.plans = grad ? reinterpret_cast<RowPlan*>(ws + space.plans) : nullptr;
    a.listed = reinterpret_cast<Listed*>(ws + space.listed);
    a.parts = reinterpret_cast<Softmax*>(ws + space.parts);
    cudaError_t err = cudaSuccess;
    int launches = 0;
    with_dtype(d->dtype, [&](auto* t) {
        with_dtype(d->values_dtype, [&](auto* v) {
            with_index_type(d->ids_type, [&](auto* i) {
                using T = tag_type<decltype(t)>;
                using V = tag_type<decltype(v)>;
                using ID = tag_type<decltype(i)>;
                err = dispatch_distill<T, V, ID>(walk, static_cast<const T*>(z), static_cast<const V*>(values), static_cast<const ID*>(ids),
                                                 static_cast<T*>(grad), a, s, &launches);
            });
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(launches);
    return CIRC_OK;
}

}  // namespace circ

using namespace circ;

extern "C" {

circ_distill_handle circ_distill_create(int classes, int count) {
    if (classes < 1 || classes > (1 << 28) || count < 1 || count > kListMost) {
        set_error(CIRC_ERR_SHAPE, "classes=%d must be in [1, 2^28] and count=%d in [1, %d]", classes, count, kListMost);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Distill* d = new (std::nothrow) Distill{device, classes, count, CIRC_F32, CIRC_F32, CIRC_I64, 1.f, false, false, {}, 0, 0};
    if (!d) set_error(CIRC_ERR_ALLOC, "host allocation failed");
    return reinterpret_cast<circ_distill_handle>(d);
}

void circ_distill_destroy(circ_distill_handle h) {
    Distill* d = reinterpret_cast<Distill*>(h);
    if (!d) return;
    free_on(d->device, d->ws);
    delete d;
}

int circ_distill_set_dtypes(circ_distill_handle h, int logits_dtype, int values_dtype, int ids_type) {
    Distill* d = reinterpret_cast<Distill*>(h);
    if (!d || !float_dtype(logits_dtype) || !float_dtype(values_dtype) || (ids_type != CIRC_I32 && ids_type != CIRC_I64)) {
        set_error(CIRC_ERR_ARG, "bad handle or type codes (%d, %d, %d)", logits_dtype, values_dtype, ids_type);
        return CIRC_ERR_ARG;
    }
    d->dtype = logits_dtype;
    d->values_dtype = values_dtype;
    d->ids_type = ids_type;
    return CIRC_OK;
}

int circ_distill_set_temperature(circ_distill_handle h, float temperature) {
    Distill* d = reinterpret_cast<Distill*>(h);
    if (!d || !(temperature >= 1e-6f && temperature <= 1e6f)) {
        set_error(CIRC_ERR_ARG, "bad handle, or temperature %g outside [1e-6, 1e6]", (double)temperature);
        return CIRC_ERR_ARG;
    }
    d->temperature = temperature;
    return CIRC_OK;
}

int circ_distill_set_rest(circ_distill_handle h, int rest) {
    Distill* d = reinterpret_cast<Distill*>(h);
    if (!d) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    d->rest = rest != 0;
    return CIRC_OK;
}

int circ_distill_set_add(circ_distill_handle h, int add) {
    Distill* d = reinterpret_cast<Distill*>(h);
    if (!d) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    d->add = add != 0;
    return CIRC_OK;
}

int circ_distill_reserve(circ_distill_handle h, long max_rows) {
    Distill* d = reinterpret_cast<Distill*>(h);
    if (!d || max_rows < 0 || max_rows > (1L << 24)) {
        set_error(CIRC_ERR_ARG, "bad handle or max_rows %ld", max_rows);
        return CIRC_ERR_ARG;
    }
    return ensure_distill(d, max_rows, true, 0);
}

int circ_distill_forward(circ_distill_handle h, const void* logits, long stride, const void* values, const void* ids, const float* lse,
                         const float* weights, float* row_loss, float* student_lse, float* mean, long rows, void* stream) {
    if (!row_loss && !student_lse && !mean) {
        set_error(CIRC_ERR_ARG, "one of row_loss, student_lse and mean must be non-NULL");
        return CIRC_ERR_ARG;
    }
    return run_distill(reinterpret_cast<Distill*>(h), logits, stride, values, ids, lse, weights, row_loss, student_lse, mean, nullptr, 0, 0.f, rows,
                       static_cast<cudaStream_t>(stream));
}

int circ_distill_backward(circ_distill_handle h, const void* logits, long stride, const void* values, const void* ids, const float* lse,
                          const float* weights, float* row_loss, float* student_lse, float* mean, void* grad_logits, long grad_stride,
                          float grad_mean, long rows, void* stream) {
    if (!grad_logits && rows != 0) {
        set_error(CIRC_ERR_ARG, "grad_logits is NULL");
        return CIRC_ERR_ARG;
    }
    return run_distill(reinterpret_cast<Distill*>(h), logits, stride, values, ids, lse, weights, row_loss, student_lse, mean, grad_logits, grad_stride,
                       grad_mean, rows, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
