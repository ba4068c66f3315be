// Softmax cross entropy over the outputs ("classes") of a network's last layer, and its gradient:
//   lse_t = log sum_v exp(z_tv),   loss_t = lse_t - z_t,target(t)   (0 for a row without a target)
//   mean  = sum_t loss_t / count,  count = rows with a target (a mean over no row is 0)
//   grad_tv = (exp(z_tv - lse_t) - [v = target(t)]) grad_mean / count, 0 for a row without a target.
// A row all of whose classes are -inf has lse = -inf, loss = +inf and a zero gradient; a NaN or +inf makes its row NaN.
#include <new>
#include <type_traits>

#include "circ_rows.cuh"

namespace circ {

struct Loss {
    int device;
    int classes;
    int dtype, ids_type;
    long ignore;
    Scratch ws;
};

template <typename ID>
__device__ __forceinline__ bool has_target(ID t, int classes, long ignore) { return t >= 0 && (long)t < classes && (long)t != ignore; }

struct LossArgs {
    long ld, grad_ld;
    float *row_loss, *lse, *mean;
    int* count;          // rows with a target, from loss_count_kernel; NULL: the block counts them itself
    unsigned* done;      // blocks that have written their sums (0 before and after a call)
    double2* sums;       // [blocks] sum of a block's row losses, and its rows with a target
    float grad_mean;
    int rows, classes;
    long ignore;
};

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
// lowest value fills) take the difference to the top first, and shift is 0.  A top of -inf counts as 0.
struct Exponent {
    float top, base, shift;
    bool plain;
    __device__ __forceinline__ explicit Exponent(float t) {
        top = t == -INFINITY ? 0.f : t;
        plain = !(fabsf(top) <= 1048576.f);
        base = plain ? 0.f : top * kLog2e;
        shift = plain ? 0.f : fmaf(top, kLog2e, -base);
    }
    template <bool PLAIN, int N>
    __device__ __forceinline__ void powers(const float (&z)[N], float (&e)[N]) const {
        if constexpr (PLAIN) {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = exp2_of((z[i] - top) * kLog2e);
        } else if constexpr (N % 2 == 0) {
            const Pair k = pair_of(kLog2e, kLog2e), b = pair_of(-base, -base);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                split(pair_fma(pair_of(z[i], z[i + 1]), k, b), e[i], e[i + 1]);
                e[i] = exp2_of(e[i]);
                e[i + 1] = exp2_of(e[i + 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = exp2_of(fmaf(z[i], kLog2e, -base));
        }
    }
    template <int N>
    __device__ __forceinline__ void of(const float (&z)[N], float (&e)[N]) const {
        if (plain) powers<true>(z, e);
        else powers<false>(z, e);
    }
};
// The lanes' pairs as one: the top first, so that every lane takes one exponential.
__device__ __forceinline__ Softmax warp_join(Softmax v) {
    float top = v.top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    // a part whose top is -inf has the sum 0 or, from a NaN, NaN
    return Softmax{top, warp_sum(v.sum * (v.top == -INFINITY ? 0.f : exp2_of((v.top - top) * kLog2e)))};
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
    Exponent ex{-INFINITY};
    __device__ __forceinline__ void rise(float most) {
        if (!(most > top)) return;
        const Exponent to(most);
        sum *= top == -INFINITY ? 0.f : exp2_of((top - most) * kLog2e + (to.shift - ex.shift));
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

// What is the same for a whole row once its sum is known.
struct RowResult {
    Exponent ex;
    float factor;      // gradient = exponential * factor, less `hot` at the target
    float hot;
    bool zero;         // no gradient
    bool valid;        // has a target
    float loss;        // 0 without one
};
template <typename ID>
__device__ __forceinline__ RowResult finish_row(const LossArgs& a, int row, Softmax all, ID target, float target_score, int count, bool writes) {
    RowResult r{Exponent(all.top), 0.f, 0.f, false, has_target(target, a.classes, a.ignore), 0.f};
    if (writes) {
        const float log_sum = logf(all.sum), lse = r.ex.top + log_sum;
        // the difference of the two scores first: it is small where both are large
        if (r.valid) r.loss = target_score == -INFINITY && lse == lse ? INFINITY : (r.ex.top - target_score) + log_sum;
        if (a.lse) a.lse[row] = lse;
        if (a.row_loss) a.row_loss[row] = r.loss;
    }
    r.zero = !r.valid || all.sum == 0.f;
    r.hot = a.grad_mean / (float)(count < 1 ? 1 : count);
    r.factor = r.hot / (all.sum * exp2_of(r.ex.shift));
    return r;
}
// The gradient of a vector whose first element is `t` columns before the target (t outside [0, VEC): the target is not in it).
template <int VEC>
__device__ __forceinline__ void gradient(const float (&z)[VEC], const RowResult& r, int t, float (&g)[VEC]) {
    r.ex.of(z, g);
#pragma unroll
    for (int e = 0; e < VEC; ++e) g[e] *= r.factor;
    if ((unsigned)t < (unsigned)VEC)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e == t) g[e] -= r.hot;
    if (r.zero)
#pragma unroll
        for (int e = 0; e < VEC; ++e) g[e] = 0.f;
}
template <typename T, int VEC, typename SPAN>
__device__ __forceinline__ void write_gradient(const SPAN& span, T* grad, size_t first, int v, const float (&z)[VEC], const RowResult& r, int target) {
    float g[VEC];
    gradient(z, r, target - span.col(v), g);
    T* dst = grad + first + (size_t)v * VEC;
    if (span.whole(v)) {
        store_vec_once<VEC>(dst, g);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e >= span.lo(v) && e < span.hi(v)) store_one(dst + e, g[e]);
    }
}

template <typename ID>
__device__ __forceinline__ int targets_of(const LossArgs& a, const ID* __restrict__ targets, int from, int step) {
    int n = 0;
#pragma unroll 16
    for (int r = from; r < a.rows; r += step) n += has_target(targets[r], a.classes, a.ignore);
    return n;
}
template <typename ID>
__global__ void __launch_bounds__(1024) loss_count_kernel(LossArgs a, const ID* __restrict__ targets) {
    __shared__ int part[32];
    pdl_begin();
    const int n = __reduce_add_sync(0xffffffffu, targets_of(a, targets, threadIdx.x, 1024));
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = n;
    __syncthreads();
    if (threadIdx.x < 32) {
        const int all = __reduce_add_sync(0xffffffffu, part[threadIdx.x]);
        if (threadIdx.x == 0) *a.count = all;
    }
}

// The mean: every block leaves the sum of its rows' losses and the number of its rows with a target (`loss` and `rows` of thread 0), and
// the block that is last to do so adds them up in the blocks' order, in float64.  All threads call it.
__device__ __forceinline__ void finish_mean(const LossArgs& a, unsigned block, unsigned blocks, double loss, int rows) {
    __shared__ bool last;
    __shared__ double part[2][32];
    if (!a.mean) return;
    if (threadIdx.x == 0) {
        a.sums[block] = make_double2(loss, (double)rows);
        __threadfence();
        last = atomicAdd(a.done, 1u) == blocks - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0, n = 0.0;
#pragma unroll 8
    for (unsigned b = threadIdx.x; b < blocks; b += blockDim.x) {
        const double2 v = __ldcg(a.sums + b);
        s += v.x;
        n += v.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        n += __shfl_xor_sync(0xffffffffu, n, o);
    }
    if (threadIdx.x % 32 == 0) {
        part[0][threadIdx.x / 32] = s;
        part[1][threadIdx.x / 32] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < (int)blockDim.x / 32; ++w) {
            s += part[0][w];
            n += part[1][w];
        }
        *a.mean = n > 0.0 ? (float)(s / n) : 0.f;
        *a.done = 0;
    }
}

// ---- short rows: a warp holds one in registers ----
// 65536 x 1000 bfloat16: 88 us with gradient, 48 without; a row of 2 KB does not keep a warp's loads in flight for long.
template <typename T, typename ID, int VEC, int ITEMS, bool ALIGNED, bool GRAD>
__global__ void __launch_bounds__(256) loss_warp_kernel(const T* z, const ID* __restrict__ targets, T* grad, LossArgs a) {
    __shared__ int part[8];
    __shared__ float losses[8];
    __shared__ int valid[8];
    pdl_begin();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, row = blockIdx.x * 8 + warp;
    const bool live = row < a.rows;
    const RowSpan<VEC, ALIGNED> span(live ? row : 0, live ? a.classes : 0, a.ld);
    float s[ITEMS][VEC];
    {
        RawVec<T, VEC> raw[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) span.load(raw[i], z, lane + i * 32);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) scores(span, lane + i * 32, raw[i], s[i]);
    }
    const ID target = live ? targets[row] : (ID)-1;
    const float target_score = live && has_target(target, a.classes, a.ignore) ? to_float(z[(size_t)row * a.ld + target]) : 0.f;
    int count = 1;
    if (GRAD && !a.count) {
        const int n = __reduce_add_sync(0xffffffffu, targets_of(a, targets, threadIdx.x, 256));
        if (lane == 0) part[warp] = n;
        __syncthreads();
        count = __reduce_add_sync(0xffffffffu, lane < 8 ? part[lane] : 0);
    }
    Running run;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) run.take(s[i]);
    const Softmax all = warp_join(run.done());
    if (GRAD && a.count) count = __ldcg(a.count);
    if (lane == 0) {
        losses[warp] = 0.f;
        valid[warp] = 0;
    }
    if (live) {
        const RowResult r = finish_row(a, row, all, target, target_score, count, lane == 0);
        if (lane == 0) {
            losses[warp] = r.loss;
            valid[warp] = r.valid;
        }
        if constexpr (GRAD) {
            const size_t first = (size_t)row * a.grad_ld + span.shift;
            __syncwarp();      // every lane has its scores and the target's: grad may be z
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (span.any(lane + i * 32)) write_gradient<T, VEC>(span, grad, first, lane + i * 32, s[i], r, (int)target);
        }
    }
    __syncthreads();
    double sum = 0.0;
    int rows = 0;
    for (int w = 0; w < 8; ++w) {
        sum += (double)losses[w];
        rows += valid[w];
    }
    finish_mean(a, blockIdx.x, gridDim.x, sum, rows);
}

// ---- long rows: a block, or the blocks of a cluster, hold one ----
// GRAD: the row is copied to shared memory as it arrives, summed up from there, and read there a second time for the gradient, so that
// it crosses the memory bus once.  Every thread copies and reads its own vectors, so a vector's place is free for the next row's as
// soon as its gradient is out: the blocks walk over the rows, and the next row streams in behind the gradient of this one.  Without a
// gradient nothing is kept.  What bounds it next to the bus: two exponentials an element, at 16 a cycle on an SM (8192 x 50001 bfloat16: 358 us,
// 4.6 TB/s, XU pipe 56 % busy; 306 us without any exponential; 174 us for the loss alone).  The loops run over
// whole vectors; a row's first and last elements beside them (odd strides) are one thread's each.
constexpr int kLossChunk = 4;     // vectors a thread in a group of copies

__device__ __forceinline__ void wait_copies(int groups) {      // until at most `groups` groups of copies are in flight (exact up to 7)
    switch (groups) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
        case 4: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
        case 5: asm volatile("cp.async.wait_group 5;" ::: "memory"); break;
        case 6: asm volatile("cp.async.wait_group 6;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 7;" ::: "memory"); break;
    }
}

// A block's part of a row.
template <int VEC>
struct LossPart {
    RowSpan<VEC, false> span;
    int vectors, w0, w1;      // vectors of the row, and the range of its whole ones
    int from, mine;           // this block's: `mine` whole ones from `from` on; a thread's are every threads-th of them
    __device__ __forceinline__ LossPart(const LossArgs& a, long row, int rank, int cluster) : span(row, a.classes, a.ld) {
        vectors = (a.classes - span.shift + VEC - 1) / VEC;
        w0 = span.whole(0) ? 0 : 1;
        w1 = span.whole(vectors - 1) ? vectors : vectors - 1;
        const int per = (w1 - w0 + cluster - 1) / cluster;
        from = w0 + rank * per;
        mine = min(w1 - from, per);
    }
};

template <typename T, typename ID, int VEC, bool GRAD>
__global__ void __launch_bounds__(512, GRAD ? 2 : 3) loss_block_kernel(const T* z, const ID* __restrict__ targets, T* grad, LossArgs a, int cluster) {
    extern __shared__ __align__(16) unsigned char held[];
    __shared__ Softmax part[2][16];
    __shared__ Softmax peers[2][8];
    __shared__ int counts[16];
    pdl_begin();
    const int threads = blockDim.x, tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = threads / 32;
    const int rank = blockIdx.x % cluster, rows_apart = gridDim.x / cluster;
    T* kept = reinterpret_cast<T*>(held) + (size_t)tid * VEC;
    const int step = threads * VEC;
    // the peers' shared memory may be written once their blocks run: arrived here, waited for in front of the first such write
    if (cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    if (lane == 0) counts[warp] = 0;
    if constexpr (GRAD) {
        const LossPart<VEC> p(a, blockIdx.x / cluster, rank, cluster);
        const T* src = z + p.span.at(p.from) + (size_t)tid * VEC;
        for (int i = tid; i < p.mine; i += kLossChunk * threads) {
#pragma unroll
            for (int u = 0; u < kLossChunk; ++u)
                if (i + u * threads < p.mine) copy_async<16>(kept + (i - tid) * VEC + u * step, src + (size_t)(i - tid) * VEC + u * step);
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        const int n = a.count ? 0 : __reduce_add_sync(0xffffffffu, targets_of(a, targets, tid, threads));
        if (lane == 0) counts[warp] = n;
    }
    int count = 0, flip = 0, valid = 0;
    double losses = 0.0;
    for (int row = blockIdx.x / cluster; row < a.rows; row += rows_apart, flip ^= 1) {
        const LossPart<VEC> p(a, row, rank, cluster);
        // the vectors that are not whole: the row's first block's thread 0 or 1 has one, or -1
        const int rest = rank != 0 ? -1 : tid == 0 && p.w0 == 1 ? 0 : tid == 1 && p.w1 < p.vectors ? p.vectors - 1 : -1;
        const ID target = targets[row];
        const float target_score = has_target(target, a.classes, a.ignore) ? to_float(z[(size_t)row * a.ld + target]) : 0.f;
        Running run;
        if constexpr (GRAD) {
            int groups = (p.mine - tid + kLossChunk * threads - 1) / (kLossChunk * threads);
            for (int i = tid; i < p.mine; i += kLossChunk * threads) {
                const T* k = kept + (i - tid) * VEC;
                wait_copies(--groups);
                if (i + (kLossChunk - 1) * threads < p.mine) {
                    RawVec<T, VEC> raw[kLossChunk];
#pragma unroll
                    for (int u = 0; u < kLossChunk; ++u) raw[u].load(k + u * step);
                    run.take(raw);
                } else {
                    for (int j = 0; i + j * threads < p.mine; ++j) {
                        RawVec<T, VEC> raw[1];
                        raw[0].load(k + j * step);
                        run.take(raw);
                    }
                }
            }
        } else {
            const T* src = z + p.span.at(p.from) + (size_t)tid * VEC;
            int i = tid;
            for (; i + (kLossChunk - 1) * threads < p.mine; i += kLossChunk * threads) {
                RawVec<T, VEC> raw[kLossChunk];
#pragma unroll
                for (int u = 0; u < kLossChunk; ++u) raw[u].load(src + (size_t)(i - tid) * VEC + u * step);
                run.take(raw);
            }
            for (; i < p.mine; i += threads) {
                RawVec<T, VEC> raw[1];
                raw[0].load(src + (size_t)(i - tid) * VEC);
                run.take(raw);
            }
        }
        if (rest >= 0) {
            RawVec<T, VEC> raw;
            float s[VEC];
            p.span.load(raw, z, rest);
            scores(p.span, rest, raw, s);
            run.take(s);
        }
        Softmax all = warp_join(run.done());
        if (lane == 0) part[flip][warp] = all;
        __syncthreads();                    // the other halves of `part` and `peers` serve the next row
        all = warp_join(lane < warps ? part[flip][lane] : Softmax{-INFINITY, 0.f});
        if (cluster > 1) {
            if (row == (int)blockIdx.x / cluster) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (tid < cluster) {            // this block's pair to every block of the cluster
                uint32_t dst;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"((uint32_t)__cvta_generic_to_shared(&peers[flip][rank])), "r"(tid));
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dst), "f"(all.top), "f"(all.sum) : "memory");
            }
            asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
            all = warp_join(lane < cluster ? peers[flip][lane] : Softmax{-INFINITY, 0.f});
        }
        if (GRAD && count == 0) {
            count = a.count ? __ldcg(a.count) : __reduce_add_sync(0xffffffffu, lane < warps ? counts[lane] : 0);
            count = count < 1 ? 1 : count;
        }
        const RowResult r = finish_row(a, row, all, target, target_score, count, rank == 0 && tid == 0);
        losses += (double)r.loss;
        valid += r.valid;
        if constexpr (GRAD) {
            const size_t first = (size_t)row * a.grad_ld + p.span.shift;
            T* dst = grad + first + (size_t)(p.from + tid) * VEC;
            const bool more = row + rows_apart < a.rows;
            const LossPart<VEC> q(a, more ? row + rows_apart : row, rank, cluster);
            const T* src = z + q.span.at(q.from) + (size_t)tid * VEC;
            const int next = more ? q.mine : 0, last = next > p.mine ? next : p.mine;
            const Pair factor = pair_of(r.factor, r.factor);
            auto put = [&](int o, auto plain) {           // the gradient of the vector that is kept at o
                RawVec<T, VEC> raw;
                float s[VEC], g[VEC];
                raw.load(kept + o);
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[e] = raw.get(e);
                r.ex.template powers<decltype(plain)::value>(s, g);
#pragma unroll
                for (int e = 0; e < VEC; e += 2) split(pair_mul(pair_of(g[e], g[e + 1]), factor), g[e], g[e + 1]);
                store_vec_once<VEC>(dst + o, g);
            };
            for (int i = tid; i < last; i += kLossChunk * threads) {
                const int o = (i - tid) * VEC, behind = i + (kLossChunk - 1) * threads;
                if (behind < p.mine && !r.zero && !r.ex.plain) {
#pragma unroll
                    for (int u = 0; u < kLossChunk; ++u) put(o + u * step, std::false_type{});
                } else {
#pragma unroll 1
                    for (int u = 0; u < kLossChunk && i + u * threads < p.mine; ++u) {
                        const float g[VEC] = {};
                        if (r.zero) store_vec_once<VEC>(dst + o + u * step, g);
                        else if (r.ex.plain) put(o + u * step, std::true_type{});
                        else put(o + u * step, std::false_type{});
                    }
                }
                // behind the stores, which have taken what lay there
                if (behind < next) {
#pragma unroll
                    for (int u = 0; u < kLossChunk; ++u) copy_async<16>(kept + o + u * step, src + o + u * step);
                } else {
#pragma unroll 1
                    for (int u = 0; i + u * threads < next; ++u) copy_async<16>(kept + o + u * step, src + o + u * step);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
            const int t = (int)target - p.span.col(p.from);       // the target's element once more, by the thread that has written its vector
            if (!r.zero && t >= 0 && t / VEC < p.mine && t / VEC % threads == tid) {
                const float s[1] = {target_score};
                float g[1];
                gradient(s, r, 0, g);
                store_one(grad + first + (size_t)p.from * VEC + t, g[0]);
            }
            if (rest >= 0) {     // read again: where grad is z, these elements are this thread's own
                RawVec<T, VEC> raw;
                float s[VEC];
                p.span.load(raw, z, rest);
                scores(p.span, rest, raw, s);
                write_gradient<T, VEC>(p.span, grad, first, rest, s, r, (int)target);
            }
        }
    }
    if (rank == 0) finish_mean(a, blockIdx.x / cluster, rows_apart, losses, valid);
}

// ---- anything else (unaligned tensors, strides of the two matrices that do not go together, rows longer than a cluster holds) ----
template <typename T, typename ID>
__global__ void __launch_bounds__(512) loss_any_kernel(const T* z, const ID* __restrict__ targets, T* grad, LossArgs a) {
    __shared__ Softmax part[2][16];
    __shared__ int counts[16];
    pdl_begin();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int n = grad && !a.count ? __reduce_add_sync(0xffffffffu, targets_of(a, targets, tid, 512)) : 0;
    if (lane == 0) counts[warp] = n;
    int flip = 0, valid = 0;
    double losses = 0.0;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
        const T* zr = z + (size_t)row * a.ld;
        Running run;
        for (int c0 = tid; c0 < a.classes; c0 += 512 * 8) {
            float s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = c0 + e * 512 < a.classes ? to_float(zr[c0 + e * 512]) : -INFINITY;
            run.take(s);
        }
        const ID target = targets[row];
        const float target_score = has_target(target, a.classes, a.ignore) ? to_float(zr[target]) : 0.f;
        Softmax all = warp_join(run.done());
        if (lane == 0) part[flip][warp] = all;
        __syncthreads();         // every thread has read the target's score: grad may be z
        all = warp_join(lane < 16 ? part[flip][lane] : Softmax{-INFINITY, 0.f});
        const int count = a.count ? __ldcg(a.count) : __reduce_add_sync(0xffffffffu, lane < 16 ? counts[lane] : 0);
        const RowResult r = finish_row(a, row, all, target, target_score, count, tid == 0);
        losses += (double)r.loss;
        valid += r.valid;
        if (!grad) continue;
        T* gr = grad + (size_t)row * a.grad_ld;
        for (int c = tid; c < a.classes; c += 512) {
            const float s[1] = {to_float(zr[c])};
            float g[1];
            gradient(s, r, (int)target - c, g);
            store_one(gr + c, g[0]);
        }
    }
    finish_mean(a, blockIdx.x, gridDim.x, losses, valid);
}

constexpr int kLossWalkers = 148 * 16;             // blocks that walk over long rows, at most
constexpr int kCountAlone = 1024;                  // rows from which on a kernel of its own counts the targets
constexpr size_t kLossHeld = 110 * 1024;           // bytes of a row that a block holds: two blocks an SM
constexpr size_t kLossMost = 216 * 1024;           // one block an SM

template <typename... KArgs, typename... Args>
static cudaError_t launch_loss(int cluster, void (*kernel)(KArgs...), unsigned blocks, int threads, size_t smem, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// The kernel for a call, by the rows' length, their number and the alignment.
template <typename T, typename ID>
static cudaError_t dispatch_loss(const T* z, const ID* targets, T* grad, const LossArgs& a, cudaStream_t s) {
    constexpr int VEC = 16 / (int)sizeof(T);
    cudaError_t err = cudaErrorNotSupported;
    auto with_rows = [&](auto aligned, auto gradient) {
        constexpr bool ALIGNED = decltype(aligned)::value, GRAD = decltype(gradient)::value;
        const int vectors = RowSpan<VEC, ALIGNED>::most(a.classes);
        if (vectors <= 128) {
            const unsigned blocks = (unsigned)((a.rows + 7L) / 8);
            auto go = [&](auto items) {
                err = launch_loss(1, loss_warp_kernel<T, ID, VEC, decltype(items)::value, ALIGNED, GRAD>, blocks, 256, 0, s, z, targets, grad, a);
            };
            vectors <= 32 ? go(std::integral_constant<int, 1>{}) : vectors <= 64 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
            return;
        }
        // blocks a row: enough to hold it, and more while the rows do not fill the machine (4 vectors a thread left at least)
        int cluster = 1;
        auto bytes = [&]() { return (size_t)((vectors + cluster - 1) / cluster) * 16; };
        while (cluster < 8 && ((GRAD && bytes() > kLossHeld) || ((long)a.rows * cluster < 148 && vectors / cluster > 2048))) cluster *= 2;
        if (GRAD && bytes() > kLossMost) return;
        const int each = (vectors + cluster - 1) / cluster, threads = each <= 512 ? 128 : each <= 2048 ? 256 : 512;
        auto kernel = loss_block_kernel<T, ID, VEC, GRAD>;
        if (GRAD && (err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLossMost)) != cudaSuccess) return;
        int per_sm = 1;
        if ((err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, GRAD ? bytes() : 0)) != cudaSuccess) return;
        const long wave = 148L * (per_sm < 1 ? 1 : per_sm) / cluster, walkers = wave < 1 ? 1 : a.rows < wave ? a.rows : wave;
        err = launch_loss(cluster, kernel, (unsigned)(walkers * cluster), threads, GRAD ? bytes() : 0, s, z, targets, grad, a, cluster);
    };
    auto with_alignment = [&](auto gradient) {
        if (misaligned(z, 16) || misaligned(grad, 16) || (grad && (a.ld - a.grad_ld) % VEC)) return;
        if (a.classes % VEC == 0 && a.ld % VEC == 0) with_rows(std::true_type{}, gradient);
        else with_rows(std::false_type{}, gradient);
    };
    grad ? with_alignment(std::true_type{}) : with_alignment(std::false_type{});
    if (err == cudaErrorNotSupported) err = launch_loss(1, loss_any_kernel<T, ID>, (unsigned)(a.rows < kLossWalkers ? a.rows : kLossWalkers), 512, 0, s, z, targets, grad, a);
    return err;
}

// Workspace: the counters (256 bytes), then the blocks' sums.
static int ensure_loss(Loss* l, long rows, cudaStream_t s) {
    const long blocks = (rows + 7) / 8 > kLossWalkers ? (rows + 7) / 8 : kLossWalkers;
    const size_t need = 256 + sizeof(double2) * (size_t)blocks;
    const bool fresh = l->ws.bytes < need;
    const int rc = ensure_scratch(l->ws, need, s, "circ_loss_reserve");
    if (rc != CIRC_OK || !fresh) return rc;
    if (cudaMemsetAsync(l->ws.ptr, 0, 256, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaFree(l->ws.ptr);      // this one alone: graphs may hold earlier ones
        l->ws.ptr = nullptr;
        l->ws.bytes = 0;
        set_error(CIRC_ERR_CUDA, "clearing the workspace failed: %s", cudaGetErrorString(cudaGetLastError()));
        return CIRC_ERR_CUDA;
    }
    return CIRC_OK;
}

static int run_loss(Loss* l, const void* z, long ld, const void* targets, float* row_loss, float* lse, float* mean, void* grad, long grad_ld,
                    float grad_mean, long rows, cudaStream_t s) {
    if (!l) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (rows < 0 || rows > (1L << 30) || ld < l->classes || (grad && grad_ld < l->classes)) {
        set_error(CIRC_ERR_SHAPE, "rows=%ld must be in [0, 2^30] and the strides (%ld, %ld) at least classes=%d", rows, ld, grad_ld, l->classes);
        return CIRC_ERR_SHAPE;
    }
    if (rows == 0) {
        if (mean) CIRC_CUDA_TRY(cudaMemsetAsync(mean, 0, sizeof(float), s), CIRC_ERR_CUDA);
        return CIRC_OK;
    }
    if (!z || !targets || (grad == z && grad_ld != ld)) {
        set_error(CIRC_ERR_ARG, "logits and targets must be non-NULL; a gradient in the place of the logits needs their stride");
        return CIRC_ERR_ARG;
    }
    const size_t zb = dtype_bytes(l->dtype);
    if (misaligned(z, zb) || misaligned(grad, zb) || misaligned(targets, l->ids_type == CIRC_I64 ? 8 : 4) || misaligned(row_loss, 4) ||
        misaligned(lse, 4) || misaligned(mean, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    const bool count_alone = grad && rows > kCountAlone;
    const int rc = ensure_loss(l, rows, s);
    if (rc != CIRC_OK) return rc;
    unsigned* words = static_cast<unsigned*>(l->ws.ptr);
    const LossArgs a{ld, grad_ld, row_loss, lse, mean, count_alone ? reinterpret_cast<int*>(words + 1) : nullptr, words,
                     reinterpret_cast<double2*>(static_cast<char*>(l->ws.ptr) + 256), grad_mean, (int)rows,
                     l->classes, l->ignore};
    cudaError_t err = cudaSuccess;
    with_dtype(l->dtype, [&](auto* t) {
        with_index_type(l->ids_type, [&](auto* i) {
            using T = tag_type<decltype(t)>;
            using ID = tag_type<decltype(i)>;
            const ID* ids = static_cast<const ID*>(targets);
            if (count_alone) {
                if ((err = launch_row(loss_count_kernel<ID>, dim3(1), dim3(1024), 0, s, a, ids)) != cudaSuccess) return;
            }
            err = dispatch_loss<T, ID>(static_cast<const T*>(z), ids, static_cast<T*>(grad), a, s);
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(1 + count_alone);
    return CIRC_OK;
}

}  // namespace circ

using namespace circ;

extern "C" {

circ_loss_handle circ_loss_create(int classes) {
    if (classes < 1 || classes > (1 << 28)) {
        set_error(CIRC_ERR_SHAPE, "classes=%d must be in [1, 2^28]", classes);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Loss* l = new (std::nothrow) Loss{device, classes, CIRC_F32, CIRC_I64, -100, {}};
    if (!l) set_error(CIRC_ERR_ALLOC, "host allocation failed");
    return reinterpret_cast<circ_loss_handle>(l);
}

void circ_loss_destroy(circ_loss_handle h) {
    Loss* l = reinterpret_cast<Loss*>(h);
    if (!l) return;
    free_on(l->device, l->ws);
    delete l;
}

int circ_loss_set_dtypes(circ_loss_handle h, int logits_dtype, int ids_type) {
    Loss* l = reinterpret_cast<Loss*>(h);
    if (!l || !float_dtype(logits_dtype) || (ids_type != CIRC_I32 && ids_type != CIRC_I64)) {
        set_error(CIRC_ERR_ARG, "bad handle or type codes (%d, %d)", logits_dtype, ids_type);
        return CIRC_ERR_ARG;
    }
    l->dtype = logits_dtype;
    l->ids_type = ids_type;
    return CIRC_OK;
}

int circ_loss_set_ignore(circ_loss_handle h, long ignore) {
    Loss* l = reinterpret_cast<Loss*>(h);
    if (!l) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    l->ignore = ignore;
    return CIRC_OK;
}

int circ_loss_reserve(circ_loss_handle h, long max_rows) {
    Loss* l = reinterpret_cast<Loss*>(h);
    if (!l || max_rows < 0 || max_rows > (1L << 30)) {
        set_error(CIRC_ERR_ARG, "bad handle or max_rows %ld", max_rows);
        return CIRC_ERR_ARG;
    }
    return ensure_loss(l, max_rows, 0);
}

int circ_loss_forward(circ_loss_handle h, const void* logits, long stride, const void* targets, float* row_loss, float* lse, float* mean,
                      long rows, void* stream) {
    if (!row_loss && !lse && !mean) {
        set_error(CIRC_ERR_ARG, "one of row_loss, lse and mean must be non-NULL");
        return CIRC_ERR_ARG;
    }
    return run_loss(reinterpret_cast<Loss*>(h), logits, stride, targets, row_loss, lse, mean, nullptr, 0, 0.f, rows, static_cast<cudaStream_t>(stream));
}

int circ_loss_backward(circ_loss_handle h, const void* logits, long stride, const void* targets, float* row_loss, float* lse, float* mean,
                       void* grad_logits, long grad_stride, float grad_mean, long rows, void* stream) {
    if (!grad_logits && rows != 0) {
        set_error(CIRC_ERR_ARG, "grad_logits is NULL");
        return CIRC_ERR_ARG;
    }
    return run_loss(reinterpret_cast<Loss*>(h), logits, stride, targets, row_loss, lse, mean, grad_logits, grad_stride, grad_mean, rows,
                    static_cast<cudaStream_t>(stream));
}

}  // extern "C"
