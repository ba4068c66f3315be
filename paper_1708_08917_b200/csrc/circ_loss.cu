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

template <typename T, typename ID>
__global__ void __launch_bounds__(256) loss_kernel(const T* z, long ld, const ID* __restrict__ targets, float* row_loss, float* lse_out, T* grad,
                                                   long grad_ld, float grad_mean, int rows, int classes, long ignore) {
    __shared__ float red[33];
    const int row = blockIdx.x;
    const T* zr = z + row * ld;
    float top = -INFINITY;
    for (int c = threadIdx.x; c < classes; c += blockDim.x) top = fmaxf(top, to_float(zr[c]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = top;
    __syncthreads();
    for (int w = 0; w < 8; ++w) top = fmaxf(top, red[w]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int c = threadIdx.x; c < classes; c += blockDim.x) sum += expf(to_float(zr[c]) - base);
    sum = block_sum(sum, red);
    const float lse = base + logf(sum);
    const ID target = targets[row];
    const bool valid = has_target(target, classes, ignore);
    float loss = 0.f;
    if (valid) {
        const float zt = to_float(zr[target]);
        loss = zt == -INFINITY && lse == lse ? INFINITY : lse - zt;
    }
    float count = 0.f;
    if (grad) {
        for (int r = threadIdx.x; r < rows; r += blockDim.x) count += has_target(targets[r], classes, ignore) ? 1.f : 0.f;
        count = block_sum(count, red);
    }
    __syncthreads();    // every thread has read the target's score: grad may be z
    if (threadIdx.x == 0) {
        if (row_loss) row_loss[row] = loss;
        if (lse_out) lse_out[row] = lse;
    }
    if (!grad) return;
    T* gr = grad + row * grad_ld;
    const float w = valid ? grad_mean / count : 0.f, inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int c = threadIdx.x; c < classes; c += blockDim.x) {
        const float p = expf(to_float(zr[c]) - base) * inv;
        store_one(gr + c, valid && sum != 0.f ? (p - (c == (long)target ? 1.f : 0.f)) * w : valid ? 0.f * sum : 0.f);
    }
}

template <typename ID>
__global__ void __launch_bounds__(1024) loss_mean_kernel(const float* __restrict__ row_loss, const ID* __restrict__ targets, float* mean, int rows,
                                                         int classes, long ignore) {
    __shared__ double sums[1024];
    __shared__ int counts[1024];
    double s = 0.0;
    int n = 0;
    for (int r = threadIdx.x; r < rows; r += 1024)
        if (has_target(targets[r], classes, ignore)) {
            s += row_loss[r];
            ++n;
        }
    sums[threadIdx.x] = s;
    counts[threadIdx.x] = n;
    __syncthreads();
    for (int o = 512; o > 0; o >>= 1) {
        if (threadIdx.x < o) {
            sums[threadIdx.x] += sums[threadIdx.x + o];
            counts[threadIdx.x] += counts[threadIdx.x + o];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) *mean = counts[0] ? (float)(sums[0] / counts[0]) : 0.f;
}

static int run_loss(Loss* l, const void* z, long ld, const void* targets, float* row_loss, float* lse, float* mean, void* grad, long grad_ld,
                    float grad_mean, long rows, cudaStream_t s) {
    if (!l) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (rows < 0 || rows > INT32_MAX || ld < l->classes || (grad && grad_ld < l->classes)) {
        set_error(CIRC_ERR_SHAPE, "rows=%ld must be in [0, 2^31) and the strides (%ld, %ld) at least classes=%d", rows, ld, grad_ld, l->classes);
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
    if (mean && !row_loss) {
        const int rc = ensure_scratch(l->ws, (size_t)rows * sizeof(float), s, "circ_loss_reserve");
        if (rc != CIRC_OK) return rc;
        row_loss = static_cast<float*>(l->ws.ptr);
    }
    with_dtype(l->dtype, [&](auto* t) {
        with_index_type(l->ids_type, [&](auto* i) {
            using T = tag_type<decltype(t)>;
            using ID = tag_type<decltype(i)>;
            loss_kernel<T, ID><<<(unsigned)rows, 256, 0, s>>>(static_cast<const T*>(z), ld, static_cast<const ID*>(targets), row_loss, lse,
                                                              static_cast<T*>(grad), grad_ld, grad_mean, (int)rows, l->classes, l->ignore);
            if (mean)
                loss_mean_kernel<ID><<<1, 1024, 0, s>>>(row_loss, static_cast<const ID*>(targets), mean, (int)rows, l->classes, l->ignore);
        });
    });
    count_launches(1 + (mean != nullptr));
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

}  // namespace circ

using namespace circ;

extern "C" {

circ_loss_handle circ_loss_create(int classes) {
    if (classes < 1) {
        set_error(CIRC_ERR_SHAPE, "classes=%d must be >= 1", classes);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Loss* l = new (std::nothrow) Loss{device, classes, CIRC_F32, CIRC_I64, -100, {nullptr, 0}};
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
    if (!l || max_rows < 0 || max_rows > INT32_MAX) {
        set_error(CIRC_ERR_ARG, "bad handle or max_rows %ld", max_rows);
        return CIRC_ERR_ARG;
    }
    return ensure_scratch(l->ws, (size_t)max_rows * sizeof(float), 0, "circ_loss_reserve");
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
