// Clipping of a network's gradients by their global norm, many tensors in one call:
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / (norm + 1e-6)).
// Two launches: sums of squares (one partial sum per thread block), then the scaled copies; every block of the second
// adds the partial sums up itself, in the same fixed order.  A norm that is not finite follows the formula (a NaN makes
// every output NaN, an infinity makes them 0 and NaN): the caller sees it in `norm`.
#include <new>
#include <type_traits>
#include <vector>

#include "circ_rows.cuh"

namespace circ {

constexpr float kClipEps = 1e-6f;
constexpr int kClipThreads = 256;

// A stretch of one tensor: the unit of work.
struct ClipPiece {
    const void* grad;
    void* out;
    int count;
    int types;     // bit 0: grad is bfloat16, bit 1: out is bfloat16
};

struct Clip {
    int device;
    std::vector<long> sizes;
    std::vector<int> types;
    std::vector<ClipPiece> pieces;
    bool set;
    Scratch plan, partial;
};

constexpr int kPieceElems = 16384;

__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(const ClipPiece* __restrict__ pieces, int count, double* __restrict__ partial) {
    __shared__ float red[33];
    double total = 0.0;
    for (int i = blockIdx.x; i < count; i += gridDim.x) {
        const ClipPiece p = pieces[i];
        float sum = 0.f;
        for (int c = threadIdx.x; c < p.count; c += kClipThreads) {
            const float g = p.types & 1 ? to_float(static_cast<const __nv_bfloat16*>(p.grad)[c]) : static_cast<const float*>(p.grad)[c];
            sum = fmaf(g, g, sum);
        }
        total += block_sum(sum, red);
    }
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

__global__ void __launch_bounds__(kClipThreads) clip_scale_kernel(const ClipPiece* __restrict__ pieces, int count, const double* __restrict__ partial,
                                                                  int partials, float max_norm, float* norm_out) {
    double total = 0.0;
    for (int i = 0; i < partials; ++i) total += partial[i];
    const float norm = (float)sqrt(total);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    const float ratio = max_norm / (norm + kClipEps), factor = ratio > 1.f ? 1.f : ratio;   // a NaN stays
    for (int i = blockIdx.x; i < count; i += gridDim.x) {
        const ClipPiece p = pieces[i];
        for (int c = threadIdx.x; c < p.count; c += kClipThreads) {
            const float g = p.types & 1 ? to_float(static_cast<const __nv_bfloat16*>(p.grad)[c]) : static_cast<const float*>(p.grad)[c];
            if (p.types & 2)
                store_one(static_cast<__nv_bfloat16*>(p.out) + c, g * factor);
            else
                static_cast<float*>(p.out)[c] = g * factor;
        }
    }
}

constexpr int kClipBlocks = 148 * 4;

}  // namespace circ

using namespace circ;

extern "C" {

circ_clip_handle circ_clip_create(int count, const long* sizes, const int* grad_dtypes, const int* out_dtypes) {
    if (count < 1 || !sizes || !grad_dtypes || !out_dtypes) {
        set_error(CIRC_ERR_ARG, "count=%d must be >= 1 and the arrays non-NULL", count);
        return nullptr;
    }
    long pieces = 0;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > (1L << 40)) {
            set_error(CIRC_ERR_SHAPE, "size %ld of tensor %d is out of range", sizes[i], i);
            return nullptr;
        }
        if (!float_dtype(grad_dtypes[i]) || !float_dtype(out_dtypes[i])) {
            set_error(CIRC_ERR_ARG, "bad dtype codes (%d, %d) of tensor %d", grad_dtypes[i], out_dtypes[i], i);
            return nullptr;
        }
        pieces += (sizes[i] + kPieceElems - 1) / kPieceElems;
    }
    if (pieces > INT32_MAX) {
        set_error(CIRC_ERR_SHAPE, "too many elements");
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Clip* c = nullptr;
    try {
        c = new Clip{device, {}, {}, {}, false, {nullptr, 0}, {nullptr, 0}};
        c->sizes.assign(sizes, sizes + count);
        for (int i = 0; i < count; ++i) c->types.push_back((grad_dtypes[i] == CIRC_BF16 ? 1 : 0) | (out_dtypes[i] == CIRC_BF16 ? 2 : 0));
        c->pieces.resize(pieces);
    } catch (const std::bad_alloc&) {
        delete c;
        set_error(CIRC_ERR_ALLOC, "host allocation failed");
        return nullptr;
    }
    if (ensure_scratch(c->plan, sizeof(ClipPiece) * (size_t)(pieces ? pieces : 1), 0, "circ_clip_create") != CIRC_OK ||
        ensure_scratch(c->partial, sizeof(double) * kClipBlocks, 0, "circ_clip_create") != CIRC_OK) {
        circ_clip_destroy(reinterpret_cast<circ_clip_handle>(c));
        return nullptr;
    }
    return reinterpret_cast<circ_clip_handle>(c);
}

void circ_clip_destroy(circ_clip_handle h) {
    Clip* c = reinterpret_cast<Clip*>(h);
    if (!c) return;
    free_on(c->device, c->plan);
    free_on(c->device, c->partial);
    delete c;
}

int circ_clip_set_tensors(circ_clip_handle h, const void* const* grads, void* const* outs, void* stream) {
    Clip* c = reinterpret_cast<Clip*>(h);
    if (!c || !grads) {
        set_error(CIRC_ERR_ARG, "handle or grads is NULL");
        return CIRC_ERR_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (stream_is_capturing(s)) {
        set_error(CIRC_ERR_UNSUPPORTED, "circ_clip_set_tensors copies from host memory: call it before the capture");
        return CIRC_ERR_UNSUPPORTED;
    }
    const int count = (int)c->sizes.size();
    for (int i = 0; i < count; ++i) {
        const size_t gb = c->types[i] & 1 ? 2 : 4, ob = c->types[i] & 2 ? 2 : 4;
        const void* out = outs ? outs[i] : grads[i];
        if (c->sizes[i] > 0 && (!grads[i] || !out)) {
            set_error(CIRC_ERR_ARG, "tensor %d is NULL", i);
            return CIRC_ERR_ARG;
        }
        if (misaligned(grads[i], gb) || misaligned(out, ob)) {
            set_error(CIRC_ERR_ARG, "tensor %d is not aligned to its element size", i);
            return CIRC_ERR_ARG;
        }
        if (c->sizes[i] > 0 && out == grads[i] && gb != ob) {
            set_error(CIRC_ERR_ARG, "tensor %d: clipping in place needs equal types", i);
            return CIRC_ERR_ARG;
        }
    }
    size_t n = 0;
    for (int i = 0; i < count; ++i) {
        const size_t gb = c->types[i] & 1 ? 2 : 4, ob = c->types[i] & 2 ? 2 : 4;
        const char* g = static_cast<const char*>(grads[i]);
        char* o = outs ? static_cast<char*>(outs[i]) : const_cast<char*>(g);
        for (long at = 0; at < c->sizes[i]; at += kPieceElems, ++n) {
            const long left = c->sizes[i] - at;
            c->pieces[n] = ClipPiece{g + at * gb, o + at * ob, (int)(left < kPieceElems ? left : kPieceElems), c->types[i]};
        }
    }
    c->set = false;
    if (n) CIRC_CUDA_TRY(cudaMemcpyAsync(c->plan.ptr, c->pieces.data(), sizeof(ClipPiece) * n, cudaMemcpyHostToDevice, s), CIRC_ERR_CUDA);
    c->set = true;
    return CIRC_OK;
}

int circ_clip_forward(circ_clip_handle h, float max_norm, float* norm, void* stream) {
    Clip* c = reinterpret_cast<Clip*>(h);
    if (!c || !c->set || misaligned(norm, 4)) {
        set_error(CIRC_ERR_ARG, "bad handle, no tensors set, or misaligned norm");
        return CIRC_ERR_ARG;
    }
    if (!(max_norm >= 0.f)) {
        set_error(CIRC_ERR_ARG, "max_norm=%g must be >= 0", (double)max_norm);
        return CIRC_ERR_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int pieces = (int)c->pieces.size(), blocks = pieces < kClipBlocks ? (pieces ? pieces : 1) : kClipBlocks;
    const ClipPiece* plan = static_cast<const ClipPiece*>(c->plan.ptr);
    double* partial = static_cast<double*>(c->partial.ptr);
    clip_norm_kernel<<<blocks, kClipThreads, 0, s>>>(plan, pieces, partial);
    clip_scale_kernel<<<blocks, kClipThreads, 0, s>>>(plan, pieces, partial, blocks, max_norm, norm);
    count_launches(2);
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

}  // extern "C"
