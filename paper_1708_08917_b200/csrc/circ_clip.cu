// Clipping of a network's gradients by their global norm, many tensors in one call:
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / (norm + 1e-6)).
// Two launches: sums of squares (one partial sum per thread block), then the scaled copies; every block of the second
// adds the partial sums up itself, in the same fixed order.  A norm that is not finite follows the formula (a NaN makes
// every output NaN, an infinity makes them 0 and NaN): the caller sees it in `norm`.  Bound by memory with two reads: 676 million bfloat16 into
// float32 in 215 + 640 us (6.3 TB/s both); 21 million float32, half of whose second read comes from L2, in 15 + 24 us.
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
    int same_types;     // ClipPiece::types of every tensor, or -1
    bool set;
    Scratch plan, partial;
};

// A piece is a block's unit of work: 256 threads take 32 elements each, in 16-byte vectors of the gradients that are all in flight
// together.  Pieces start on 16-byte boundaries of their tensor's gradient, but for its first one, which has up to 7 elements more in
// front.  A tensor's number of pieces follows from its size alone (the last one may be empty), so that a captured call stays valid for
// other addresses.
constexpr int kPieceElems = 8192;
static long pieces_of(long size) { return (size + kPieceElems - 1) / kPieceElems; }

// Elements in front of the first 16-byte boundary.
template <typename T>
__device__ __forceinline__ int head_of(const T* p) {
    constexpr unsigned VEC = 16 / sizeof(T);
    return (int)((VEC - (unsigned)(reinterpret_cast<uintptr_t>(p) / sizeof(T)) % VEC) % VEC);
}

// The sum of squares of a thread's elements of a piece; consecutive threads take consecutive vectors.  Squares that float32 does not hold
// (a sum beyond its range, or so small that squares below the normal numbers count) are taken again of the elements times 2^-96 or
// 2^96, which are still in registers.
constexpr float kSquareFactor = 7.9228162514264338e28f;      // 2^96
constexpr float kSquaresLow = 1.2621774483536189e-29f;       // 2^-96: what subnormal squares lose is below 2^-45 of a sum from here on

template <typename TG>
__device__ __forceinline__ double piece_squares(const TG* g, int count) {
    constexpr int VEC = 16 / (int)sizeof(TG), DEPTH = kPieceElems / kClipThreads / VEC;
    const int tid = threadIdx.x, front = head_of(g), head = front < count ? front : count;
    const float first = tid < head ? to_float(g[tid]) : 0.f;
    float last = 0.f;
    g += head;
    count -= head;
    RawVec<TG, VEC> raw[DEPTH];
    if (count == kPieceElems) {
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) raw[u].load(g + (u * kClipThreads + tid) * VEC);
    } else {
        const int whole = count / VEC, c = whole * VEC + tid;
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (u * kClipThreads + tid < whole) raw[u].load(g + (u * kClipThreads + tid) * VEC);
            else raw[u].clear();
        }
        if (c < count) last = to_float(g[c]);
    }
    float part[4] = {first * first, last * last, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < DEPTH; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) part[e % 4] = fmaf(raw[u].get(e), raw[u].get(e), part[e % 4]);
    const float sum = (part[0] + part[1]) + (part[2] + part[3]);
    if (sum >= kSquaresLow && sum < INFINITY) return (double)sum;
    const float k = sum < 1.f ? kSquareFactor : 1.f / kSquareFactor;
    float again = first * k * (first * k) + last * k * (last * k);
#pragma unroll
    for (int u = 0; u < DEPTH; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) again = fmaf(raw[u].get(e) * k, raw[u].get(e) * k, again);
    return (double)again / ((double)k * (double)k);
}

// Pieces are walked in order here and in reverse order by the second kernel, which so finds the last ones in the L2 cache.
__global__ void __launch_bounds__(kClipThreads) clip_norm_kernel(const ClipPiece* __restrict__ pieces, int count, double* __restrict__ partial) {
    __shared__ double sums[kClipThreads / 32];
    pdl_begin();
    double total = 0.0;
    for (int i = blockIdx.x; i < count; i += gridDim.x) {
        const ClipPiece p = pieces[i];
        total += p.types & 1 ? piece_squares(static_cast<const __nv_bfloat16*>(p.grad), p.count) : piece_squares(static_cast<const float*>(p.grad), p.count);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kClipThreads / 32; ++w) total += sums[w];
        partial[blockIdx.x] = total;
    }
}

constexpr int kScaleBlocks = 4;       // of the second kernel on an SM, 64 KB in flight

// Vectors where gradient and output are aligned together (the same number of elements in front of their boundaries), else by element.
template <typename TG, typename TO>
__device__ __forceinline__ void piece_scale(const TG* g, TO* out, int count, float factor) {
    constexpr int VEC = sizeof(TG) == 2 && sizeof(TO) == 2 ? 8 : 4, DEPTH = 4;     // four vectors in flight a thread
    const int tid = threadIdx.x, front = head_of(g), head = front < count ? front : count;
    if (((reinterpret_cast<uintptr_t>(g + front) | reinterpret_cast<uintptr_t>(out + front)) & 15u) == 0) {
        if (tid < head) store_one(out + tid, to_float(g[tid]) * factor);
        g += head;
        out += head;
        count -= head;
        const int whole = count / VEC, c = whole * VEC + tid;
#pragma unroll 1
        for (int v = tid; v < whole; v += DEPTH * kClipThreads) {
            RawVec<TG, VEC> raw[DEPTH];
#pragma unroll
            for (int u = 0; u < DEPTH; ++u)
                if (v + u * kClipThreads < whole) raw[u].load(g + (v + u * kClipThreads) * VEC);
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                if (v + u * kClipThreads >= whole) break;
                float x[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = raw[u].get(e) * factor;
                store_vec_once<VEC>(out + (v + u * kClipThreads) * VEC, x);
            }
        }
        if (c < count) store_one(out + c, to_float(g[c]) * factor);
    } else {
#pragma unroll 4
        for (int c = tid; c < count; c += kClipThreads) store_one(out + c, to_float(g[c]) * factor);
    }
}

// TYPES: those of all pieces (ClipPiece::types), or -1 where they differ.
template <int TYPES>
__global__ void __launch_bounds__(kClipThreads, kScaleBlocks) clip_scale_kernel(const ClipPiece* __restrict__ pieces, int count, const double* __restrict__ partial,
                                                                  int partials, float max_norm, float* norm_out) {
    __shared__ double sums[kClipThreads / 32];
    pdl_begin();
    double total = 0.0;
    for (int i = threadIdx.x; i < partials; i += kClipThreads) total += __ldcg(partial + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = total;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / 32; ++w) total += sums[w];
    const float norm = (float)sqrt(total);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    const float ratio = max_norm / (norm + kClipEps), factor = ratio > 1.f ? 1.f : ratio;   // a NaN stays
    for (int i = count - 1 - (int)blockIdx.x; i >= 0; i -= (int)gridDim.x) {
        const ClipPiece p = pieces[i];
        if (factor == 1.f && p.grad == p.out) continue;       // nothing to clip, in place
        const float* gf = static_cast<const float*>(p.grad);
        const __nv_bfloat16* gb = static_cast<const __nv_bfloat16*>(p.grad);
        float* of = static_cast<float*>(p.out);
        __nv_bfloat16* ob = static_cast<__nv_bfloat16*>(p.out);
        const int types = TYPES < 0 ? p.types : TYPES;
        if (types == 0) piece_scale(gf, of, p.count, factor);
        else if (types == 1) piece_scale(gb, of, p.count, factor);
        else if (types == 2) piece_scale(gf, ob, p.count, factor);
        else piece_scale(gb, ob, p.count, factor);
    }
}

constexpr int kClipBlocks = 148 * 8;   // a wave of eight blocks an SM

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
        pieces += pieces_of(sizes[i]);
    }
    if (pieces > INT32_MAX) {
        set_error(CIRC_ERR_SHAPE, "too many elements");
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Clip* c = nullptr;
    try {
        c = new Clip{device, {}, {}, {}, -1, false, {}, {}};
        c->sizes.assign(sizes, sizes + count);
        for (int i = 0; i < count; ++i) c->types.push_back((grad_dtypes[i] == CIRC_BF16 ? 1 : 0) | (out_dtypes[i] == CIRC_BF16 ? 2 : 0));
        c->pieces.resize(pieces);
        c->same_types = c->types[0];
        for (int t : c->types)
            if (t != c->types[0]) c->same_types = -1;
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
        const long pieces = pieces_of(c->sizes[i]);
        long most = kPieceElems + (long)((16 - reinterpret_cast<uintptr_t>(g) % 16) % 16 / gb), at = 0;
        for (long k = 0; k < pieces; ++k, ++n, most = kPieceElems) {
            const long left = c->sizes[i] - at, len = left < most ? left : most;
            c->pieces[n] = ClipPiece{g + at * gb, o + at * ob, (int)len, c->types[i]};
            at += len;
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
    CIRC_CUDA_TRY(launch_row(clip_norm_kernel, dim3(blocks), dim3(kClipThreads), 0, s, plan, pieces, partial), CIRC_ERR_CUDA);
    auto* kernel = c->same_types < 0 ? clip_scale_kernel<-1> : c->same_types == 0 ? clip_scale_kernel<0> : c->same_types == 1 ? clip_scale_kernel<1>
                   : c->same_types == 2 ? clip_scale_kernel<2> : clip_scale_kernel<3>;
    const int scale_blocks = pieces < 148 * kScaleBlocks ? blocks : 148 * kScaleBlocks;
    CIRC_CUDA_TRY(launch_row(kernel, dim3(scale_blocks), dim3(kClipThreads), 0, s, plan, pieces, partial, blocks, max_norm, norm), CIRC_ERR_CUDA);
    count_launches(2);
    return CIRC_OK;
}

}  // extern "C"
