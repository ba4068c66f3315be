// Shared pieces of the row operators around the circulant layers (embedding, norm, loss, gradient clipping): element
// types chosen at run time, class indices, sums over a thread block in a fixed order, and workspaces of their handles.
#pragma once
#include <math.h>

#include "circ_common.cuh"
#include "circ_io.cuh"

namespace circ {

inline size_t dtype_bytes(int dtype) { return dtype == CIRC_F32 ? 4 : dtype == CIRC_BF16 ? 2 : 1; }
inline bool float_dtype(int dtype) { return dtype == CIRC_F32 || dtype == CIRC_BF16; }
inline bool misaligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Calls f with a null pointer of the element type as its tag: f(static_cast<float*>(nullptr)) or the bfloat16 one.
template <typename F>
inline void with_dtype(int dtype, F&& f) {
    if (dtype == CIRC_BF16)
        f(static_cast<__nv_bfloat16*>(nullptr));
    else
        f(static_cast<float*>(nullptr));
}
template <typename F>
inline void with_index_type(int type, F&& f) {
    if (type == CIRC_I64)
        f(static_cast<int64_t*>(nullptr));
    else
        f(static_cast<int32_t*>(nullptr));
}
template <typename T>
using tag_type = std::remove_pointer_t<T>;

// Sum over the lanes of a warp, the same bits in every lane.
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// The larger value, NaN if either is (fmaxf drops a NaN).
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// Sum over a thread block of whole warps, in a fixed order, the result in every thread.  `red`: 33 floats of shared
// memory that the call may use until its second barrier.
__device__ __forceinline__ float block_sum(float v, float* red) {
    const int warps = (blockDim.x + 31) / 32;
    v = warp_sum(v);
    if (warps == 1) return v;
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = threadIdx.x % 32 < warps ? red[threadIdx.x % 32] : 0.f;
    return warp_sum(v);
}

// A workspace that a handle owns: grows when a call needs more, never while the stream is being captured.
struct Scratch {
    void* ptr;
    size_t bytes;
};
inline int ensure_scratch(Scratch& s, size_t need, cudaStream_t stream, const char* reserve_call) {
    if (s.bytes >= need) return CIRC_OK;
    if (stream_is_capturing(stream)) {
        set_error(CIRC_ERR_UNSUPPORTED, "the workspace (%zu bytes) is too small for this call (%zu bytes) and the stream is being "
                  "captured: call %s before the capture", s.bytes, need, reserve_call);
        return CIRC_ERR_UNSUPPORTED;
    }
    cudaFree(s.ptr);   // implicit synchronisation: earlier calls have finished with it
    s.ptr = nullptr;
    s.bytes = 0;
    if (dev_alloc(&s.ptr, need) != cudaSuccess) {
        cudaGetLastError();
        s.ptr = nullptr;
        set_error(CIRC_ERR_ALLOC, "workspace allocation of %zu bytes failed", need);
        return CIRC_ERR_ALLOC;
    }
    s.bytes = need;
    return CIRC_OK;
}
// Frees what a handle owns on the device it was created on.
inline void free_on(int device, Scratch& s) {
    if (!s.ptr) return;
    int prev = -1;
    cudaGetDevice(&prev);
    if (prev != device) cudaSetDevice(device);
    cudaFree(s.ptr);
    if (prev != device && prev >= 0) cudaSetDevice(prev);
    s.ptr = nullptr;
    s.bytes = 0;
}
// The current device for a new handle; false (with the error set) when there is none.
inline bool current_device(int* device) {
    if (cudaGetDevice(device) == cudaSuccess) return true;
    set_error(CIRC_ERR_CUDA, "no CUDA device: %s", cudaGetErrorString(cudaGetLastError()));
    return false;
}

}  // namespace circ
