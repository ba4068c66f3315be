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
// group's values have no meaning then, and the NaN says so).
__device__ __forceinline__ float group_scale(float top) { return top == 0.f ? 1.f : top <= 3.402823466e38f ? top / kE4m3Max : NAN; }

template <typename TX, typename TY>
__global__ void __launch_bounds__(256) norm_forward_kernel(const TX* x, const TX* residual, const float* __restrict__ gain, TX* sum, TY* y,
                                                           float* y_scale, float* rstd_out, int dim, int group, float eps) {
    __shared__ float red[33];
    const size_t row = blockIdx.x, base = row * dim;
    auto value = [&](int c) { return to_float(x[base + c]) + (residual ? to_float(residual[base + c]) : 0.f); };
    float sq = 0.f;
    for (int c = threadIdx.x; c < dim; c += blockDim.x) {
        const float v = value(c);
        sq = fmaf(v, v, sq);
    }
    const float rstd = rsqrtf(block_sum(sq, red) / (float)dim + eps);
    if (rstd_out && threadIdx.x == 0) rstd_out[row] = rstd;
    if constexpr (std::is_same<TY, uint8_t>::value) {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        for (int g = warp; g < dim / group; g += blockDim.x / 32) {
            float top = 0.f;
            for (int c = lane; c < group; c += 32) top = max_nan(top, fabsf(value(g * group + c) * rstd * (gain ? gain[g * group + c] : 1.f)));
            const float scale = group_scale(warp_max_nan(top));
            if (lane == 0) y_scale[row * (dim / group) + g] = scale;
            for (int c = g * group + lane; c < (g + 1) * group; c += 32)
                y[base + c] = to_e4m3(value(c) * rstd * (gain ? gain[c] : 1.f) / scale);
        }
        __syncthreads();    // sum may be x or residual
        if (sum)
            for (int c = threadIdx.x; c < dim; c += blockDim.x) store_one(sum + base + c, value(c));
    } else {
        for (int c = threadIdx.x; c < dim; c += blockDim.x) {
            const float v = value(c);
            store_one(y + base + c, v * rstd * (gain ? gain[c] : 1.f));
            if (sum) store_one(sum + base + c, v);
        }
    }
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(256) norm_backward_kernel(const TX* __restrict__ sum, const float* __restrict__ gain,
                                                            const float* __restrict__ rstd_in, const TY* __restrict__ dy, const TX* ds, TX* dx, int dim) {
    __shared__ float red[33];
    const size_t row = blockIdx.x, base = row * dim;
    const float rstd = rstd_in[row];
    float dot = 0.f;
    for (int c = threadIdx.x; c < dim; c += blockDim.x)
        dot = fmaf(to_float(dy[base + c]) * (gain ? gain[c] : 1.f), to_float(sum[base + c]) * rstd, dot);
    dot = block_sum(dot, red) / (float)dim;
    for (int c = threadIdx.x; c < dim; c += blockDim.x) {
        const float u = to_float(dy[base + c]) * (gain ? gain[c] : 1.f), hh = to_float(sum[base + c]) * rstd;
        store_one(dx + base + c, rstd * (u - hh * dot) + (ds ? to_float(ds[base + c]) : 0.f));
    }
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(256) norm_gain_kernel(const TX* __restrict__ sum, const float* __restrict__ rstd, const TY* __restrict__ dy,
                                                        float* __restrict__ dgain, long rows, int dim) {
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c >= dim) return;
    float acc = 0.f;
    for (long r = 0; r < rows; ++r) acc = fmaf(to_float(dy[r * dim + c]), to_float(sum[r * dim + c]) * rstd[r], acc);
    dgain[c] = acc;
}

template <typename TO>
__global__ void __launch_bounds__(256) norm_unpack_kernel(const uint8_t* __restrict__ y, const float* __restrict__ scale, TO* __restrict__ out,
                                                          long count, int group) {
    for (long i = blockIdx.x * (long)blockDim.x + threadIdx.x; i < count; i += (long)gridDim.x * blockDim.x)
        store_one(out + i, from_e4m3(y[i]) * scale[i / group]);
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

}  // namespace circ

using namespace circ;

extern "C" {

circ_norm_handle circ_norm_create(int dim, float eps) {
    if (dim < 1) {
        set_error(CIRC_ERR_SHAPE, "dim=%d must be >= 1", dim);
        return nullptr;
    }
    if (!(eps >= 0.f) || isinf(eps)) {
        set_error(CIRC_ERR_ARG, "eps=%g must be finite and >= 0", (double)eps);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Norm* n = new (std::nothrow) Norm{device, dim, eps, CIRC_F32, CIRC_F32, 0, {nullptr, 0}};
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
    return check_norm(n, 0);
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
    with_dtype(n->x_dtype, [&](auto* t) {
        using TX = tag_type<decltype(t)>;
        auto go = [&](auto* o) {
            using TY = tag_type<decltype(o)>;
            norm_forward_kernel<TX, TY><<<(unsigned)rows, 256, 0, s>>>(static_cast<const TX*>(x), static_cast<const TX*>(residual), gain,
                                                                       static_cast<TX*>(sum), static_cast<TY*>(y), y_scale, rstd, n->dim,
                                                                       norm_group(n), n->eps);
        };
        if (e4m3)
            go(static_cast<uint8_t*>(nullptr));
        else
            with_dtype(n->y_dtype, go);
    });
    count_launches(1);
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
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
    with_dtype(n->x_dtype, [&](auto* t) {
        with_dtype(gy, [&](auto* o) {
            using TX = tag_type<decltype(t)>;
            using TY = tag_type<decltype(o)>;
            if (grad_x)
                norm_backward_kernel<TX, TY><<<(unsigned)rows, 256, 0, s>>>(static_cast<const TX*>(sum), gain, rstd, static_cast<const TY*>(grad_y),
                                                                            static_cast<const TX*>(grad_sum), static_cast<TX*>(grad_x), n->dim);
            if (grad_gain)
                norm_gain_kernel<TX, TY><<<(unsigned)((n->dim + 255) / 256), 256, 0, s>>>(static_cast<const TX*>(sum), rstd,
                                                                                          static_cast<const TY*>(grad_y), grad_gain, rows, n->dim);
        });
    });
    count_launches((grad_x != nullptr) + (grad_gain != nullptr));
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
    const long count = rows * n->dim, need = (count + 255) / 256;
    const unsigned blocks = (unsigned)(need < 148L * 32 ? need : 148L * 32);
    with_dtype(out_dtype, [&](auto* o) {
        using TO = tag_type<decltype(o)>;
        norm_unpack_kernel<TO><<<blocks, 256, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<const uint8_t*>(y), y_scale, static_cast<TO*>(out),
                                                                                      count, norm_group(n));
    });
    count_launches(1);
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

}  // extern "C"
