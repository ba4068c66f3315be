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
    long rows_held;      // rows that the workspace is laid out for
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
    int pieces, per;          // pieces a row, vectors a piece
    bool add;
    // workspace
    unsigned* done;           // rows that are finished (0 before and after a call)
    double* weight_sum;
    unsigned* arrived;        // [rows] pieces that are summed up (0 before and after a call)
    double2* sums;            // [rows] weight loss, weight
    RowPlan* plans;           // [rows]
    Listed* listed;           // [rows][count]
    Softmax* parts;           // [rows][pieces]
};

constexpr int kPieceBits = 32768;        // classes a piece, at most: a bit each says which are listed
constexpr int kPieceThreads = 256;

template <int VEC>
struct Piece {
    RowSpan<VEC, false> span;
    int from, to;                        // vectors
    __device__ __forceinline__ Piece(const DistillArgs& a, long row, int piece) : span(row, a.side.classes, a.ld) {
        const int vectors = (a.side.classes - span.shift + VEC - 1) / VEC;
        from = piece * a.per;
        to = min(vectors, from + a.per);
    }
    // Place of a class in the piece, or -1.
    __device__ __forceinline__ int place(long id) const {
        const long at = id - span.col(from);
        return id >= 0 && id < span.dim && at >= 0 && at < (long)(to - from) * VEC ? (int)at : -1;
    }
};
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
template <int VEC>
__device__ __forceinline__ unsigned marks_of(const uint32_t* marks, int v) {       // v: vector of the piece
    return (marks[v * VEC / 32] >> (v * VEC % 32)) & ((1u << VEC) - 1);
}

// Pieces of rows, summed up without the listed classes; the block that is last to finish a row's pieces works out its loss, and the one
// that is last to finish a row the mean.
template <typename T, typename V, typename ID, int VEC, int ITEMS>
__global__ void __launch_bounds__(kPieceThreads) distill_sum_kernel(const T* z, const V* __restrict__ values, const ID* __restrict__ ids, DistillArgs a) {
    __shared__ uint32_t marks[kPieceBits / 32];
    __shared__ Softmax part[kPieceThreads / 32];
    __shared__ bool last;
    __shared__ double2 red[kPieceThreads / 32];
    pdl_begin();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
    const float weight = a.weights ? a.weights[row] : 1.f;
    const bool live = weight > 0.f;
    if (live) {
        const Piece<VEC> p(a, row, piece);
        mark_listed(a, p, ids, (size_t)row, marks);
        Running run(a.side.scale);
        for (int v = p.from + tid; v < p.to; v += kPieceThreads) {
            RawVec<T, VEC> raw;
            float s[VEC];
            p.span.load(raw, z, v);
            scores(p.span, v, raw, s);
            const unsigned m = marks_of<VEC>(marks, v - p.from);
            if (m)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (m >> e & 1) s[e] = -INFINITY;
            run.take(s);
        }
        const Softmax all = warp_join(run.done(), a.side.scale);
        if (lane == 0) part[warp] = all;
        __syncthreads();
        if (warp == 0) {
            const Softmax block = warp_join(lane < kPieceThreads / 32 ? part[lane] : Softmax{-INFINITY, 0.f}, a.side.scale);
            if (lane == 0) a.parts[(size_t)row * a.pieces + piece] = block;
        }
    }
    if (tid == 0) {
        __threadfence();
        last = a.pieces == 1 || atomicAdd(a.arrived + row, 1u) == (unsigned)a.pieces - 1;
        if (last && a.pieces > 1) a.arrived[row] = 0;
    }
    __syncthreads();
    if (!last) return;
    if (warp == 0) {
        __threadfence();
        RowPlan plan{-INFINITY, 0.f, 0.f, 0};
        double loss = 0.0, lse = 0.0;
        if (live) {
            Softmax outside{-INFINITY, 0.f};
            for (int i = lane; i < a.pieces; i += 32) {
                const float2 other = __ldcg(reinterpret_cast<const float2*>(a.parts) + (size_t)row * a.pieces + i);
                outside = join(outside, Softmax{other.x, other.y}, a.side.scale);
            }
            outside = warp_join(outside, a.side.scale);
            TeacherList<ITEMS> list;
            list.load(a.side, values, ids, (size_t)row, marks);
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) list.s[j] = list.id[j] >= 0 ? to_float(z[(size_t)row * a.ld + list.id[j]]) : -INFINITY;
            float q[ITEMS];
            const ListRow r = list.finish(a.side, outside, q);
            loss = r.loss;
            lse = r.lse;
            if (a.plans) {
                int n = 0;
#pragma unroll
                for (int j = 0; j < ITEMS; ++j) {
                    const unsigned have = __ballot_sync(0xffffffffu, list.id[j] >= 0);
                    if (list.id[j] >= 0) a.listed[(size_t)row * a.side.count + n + __popc(have & ((1u << lane) - 1))] = Listed{list.id[j], q[j]};
                    n += __popc(have);
                }
                plan = RowPlan{outside.top, r.factor, r.zero ? 0.f : weight, n};
            }
        }
        if (lane == 0) {
            if (a.row_loss) a.row_loss[row] = (float)loss;
            if (a.student_lse) a.student_lse[row] = (float)lse;
            if (a.plans) a.plans[row] = plan;
            a.sums[row] = live ? make_double2(weight * loss, (double)weight) : make_double2(0.0, 0.0);
            __threadfence();
            last = atomicAdd(a.done, 1u) == (unsigned)a.rows - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0, w = 0.0;
    for (int r = tid; r < a.rows; r += kPieceThreads) {
        const double2 v = __ldcg(a.sums + r);
        s += v.x;
        w += v.y;
    }
    s = warp_sum(s);
    w = warp_sum(w);
    if (lane == 0) red[warp] = make_double2(s, w);
    __syncthreads();
    if (tid == 0) {
        s = w = 0.0;
        for (int i = 0; i < kPieceThreads / 32; ++i) {
            s += red[i].x;
            w += red[i].y;
        }
        if (a.mean) *a.mean = w > 0.0 ? (float)(s / w) : 0.f;
        *a.weight_sum = w;
        *a.done = 0;
    }
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
    for (int v = p.from + tid; v < p.to; v += kPieceThreads) {
        float out[VEC], old[VEC];
        const unsigned m = zero ? 0 : marks_of<VEC>(marks, v - p.from);
        if (zero) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[e] = 0.f;
        } else {
            RawVec<T, VEC> raw;
            float s[VEC];
            p.span.load(raw, z, v);
            scores(p.span, v, raw, s);
            ex.of(s, out);
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[e] *= factor;
        }
        const int col = p.span.col(v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) old[e] = a.add && !(m >> e & 1) && col + e >= 0 && col + e < a.side.classes ? to_float(g[col + e]) : 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) out[e] += old[e];
        if (VEC > 1 && p.span.whole(v) && !m) {
            store_vec<VEC>(g + col, out);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (col + e >= 0 && col + e < a.side.classes && !(m >> e & 1)) store_one(g + col + e, out[e]);
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

// Pieces a row: enough for the marks, and more while the rows do not fill the machine (4 vectors a thread left at least).
static int pieces_of(long rows, int classes, int vec, int* per) {
    const long vectors = ((long)classes + 2 * vec - 2) / vec, most = kPieceBits / vec;
    long pieces = (vectors + most - 1) / most;
    const long want = (kPieceTarget + rows - 1) / rows, can = vectors / (4 * kPieceThreads);
    const long split = want < can ? want : can;
    if (split > pieces) pieces = split;
    if (pieces < 1) pieces = 1;
    *per = (int)((vectors + pieces - 1) / pieces);
    return (int)((vectors + *per - 1) / *per);
}

// Workspace: counters (256 bytes), the rows' counters, their sums, plans and lists, and the pieces' sums, for `rows` rows.
struct DistillSpace {
    size_t arrived, sums, plans, listed, parts, bytes;
};
static DistillSpace space_of(const Distill* d, long rows) {
    DistillSpace s;
    const size_t least = ((size_t)d->classes + kPieceBits / 2 - 1) / (kPieceBits / 2) + 1;      // pieces a row where rows fill the machine
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    s.arrived = 256;
    s.sums = s.arrived + up(sizeof(unsigned) * rows);
    s.plans = s.sums + up(sizeof(double2) * rows);
    s.listed = s.plans + up(sizeof(RowPlan) * rows);
    s.parts = s.listed + up(sizeof(Listed) * rows * d->count);
    s.bytes = s.parts + up(sizeof(Softmax) * (rows * least + 2 * kPieceTarget));
    return s;
}
static int ensure_distill(Distill* d, long rows, cudaStream_t s) {
    if (rows <= d->rows_held) return ensure_scratch(d->ws, space_of(d, d->rows_held).bytes, s, "circ_distill_reserve");
    const int rc = ensure_scratch(d->ws, space_of(d, rows).bytes, s, "circ_distill_reserve");
    d->rows_held = rc == CIRC_OK ? rows : d->ws.ptr ? d->rows_held : 0;
    if (rc != CIRC_OK) return rc;
    if (cudaMemsetAsync(d->ws.ptr, 0, space_of(d, rows).sums, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaFree(d->ws.ptr);      // this one alone: graphs may hold earlier ones
        d->ws.ptr = nullptr;
        d->ws.bytes = 0;
        d->rows_held = 0;
        set_error(CIRC_ERR_CUDA, "clearing the workspace failed: %s", cudaGetErrorString(cudaGetLastError()));
        return CIRC_ERR_CUDA;
    }
    return CIRC_OK;
}

template <typename T, typename V, typename ID>
static cudaError_t dispatch_distill(const T* z, const V* values, const ID* ids, T* grad, DistillArgs a, cudaStream_t s, int* launches) {
    constexpr int VEC = 16 / (int)sizeof(T);
    cudaError_t err = cudaSuccess;
    auto split = [&](auto vec) {
        constexpr int N = decltype(vec)::value;
        a.pieces = pieces_of(a.rows, a.side.classes, N, &a.per);
        const long blocks = (long)a.rows * a.pieces;
        if (blocks >= 1L << 31) {
            err = cudaErrorInvalidConfiguration;
            return;
        }
        auto sum = [&](auto items) {
            err = launch_row(distill_sum_kernel<T, V, ID, N, decltype(items)::value>, dim3((unsigned)blocks), dim3(kPieceThreads), 0, s, z, values, ids, a);
        };
        a.side.count <= 64 ? sum(std::integral_constant<int, 2>{}) : sum(std::integral_constant<int, kListLanes>{});
        *launches = 1;
        if (err != cudaSuccess || !grad) return;
        err = launch_row(distill_grad_kernel<T, ID, N>, dim3((unsigned)blocks), dim3(kPieceThreads), 0, s, z, ids, grad, a);
        *launches = 2;
    };
    if (misaligned(z, 16) || misaligned(grad, 16) || (grad && (a.ld - a.grad_ld) % VEC)) split(std::integral_constant<int, 1>{});
    else split(std::integral_constant<int, VEC>{});
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
    const int rc = ensure_distill(d, rows, s);
    if (rc != CIRC_OK) return rc;
    const DistillSpace space = space_of(d, d->rows_held);
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
                err = dispatch_distill<T, V, ID>(static_cast<const T*>(z), static_cast<const V*>(values), static_cast<const ID*>(ids),
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
    Distill* d = new (std::nothrow) Distill{device, classes, count, CIRC_F32, CIRC_F32, CIRC_I64, 1.f, false, false, {}, 0};
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
    return ensure_distill(d, max_rows, 0);
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
