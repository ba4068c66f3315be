// Shared pieces of the row operators around the circulant layers (embedding, norm, loss, gradient clipping): element
// types chosen at run time, class indices, sums over a thread block in a fixed order, and workspaces of their handles.
#pragma once
#include <math.h>

#include <new>
#include <type_traits>

#include "circ_common.cuh"
#include "circ_io.cuh"

namespace circ {

// Every kernel of these operators starts with pdl_begin() and is launched by launch_row: its blocks may be scheduled while the stream's
// previous kernel still runs (which hides the launch), and touch global memory only once that one has finished.
__device__ __forceinline__ void pdl_begin() {
    pdl_wait();
    pdl_trigger();
}
template <typename... KArgs, typename... Args>
inline cudaError_t launch_row(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, Args&&... args) {
    return launch_kernel(PDL_EARLY, kernel, grid, block, smem, stream, args...);
}

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

// Two float32 values a register pair: additions, products and multiply-adds of both in one instruction.
struct Pair {
    uint64_t v;
};
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p.v)); }
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Pair pair_add(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair pair_mul(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

// VEC float32 registers to consecutive elements: 16-byte accesses (the address must be 16-byte aligned; 8 bytes for four bfloat16), or
// VEC = 1.
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1)
        store_one(p, v[0]);
    else
        store_run<VEC>(p, v);
}

// The same for outputs that this kernel does not read again (first to leave the L2 cache).
template <int VEC>
__device__ __forceinline__ void store_vec_once(float* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1)
        __stcs(p, v[0]);
    else
#pragma unroll
        for (int r = 0; r < VEC; r += 4) __stcs(reinterpret_cast<float4*>(p + r), make_float4(v[r], v[r + 1], v[r + 2], v[r + 3]));
}
template <int VEC>
__device__ __forceinline__ void store_vec_once(__nv_bfloat16* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1)
        store_one(p, v[0]);
    else if constexpr (VEC == 4)
        __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])));
    else
#pragma unroll
        for (int r = 0; r < VEC; r += 8)
            __stcs(reinterpret_cast<uint4*>(p + r), make_uint4(pack_bf16(v[r], v[r + 1]), pack_bf16(v[r + 2], v[r + 3]),
                                                              pack_bf16(v[r + 4], v[r + 5]), pack_bf16(v[r + 6], v[r + 7])));
}

// The same, kept as loaded until an element is asked for (half the registers of bfloat16 data in flight).
template <typename T, int VEC>
struct RawVec {
    static constexpr int WORDS = (int)(VEC * sizeof(T) + 3) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void fill_lowest() {      // -inf
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    }
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VEC == 1) {
            w[0] = sizeof(T) == 4 ? *reinterpret_cast<const uint32_t*>(p) : (uint32_t)*reinterpret_cast<const uint16_t*>(p);
        } else if constexpr (WORDS == 1) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (WORDS == 2) {
            const uint2 t = *reinterpret_cast<const uint2*>(p);
            w[0] = t.x; w[1] = t.y;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i += 4) {
                const uint4 t = *reinterpret_cast<const uint4*>(p + i * 4 / (int)sizeof(T));
                w[i] = t.x; w[i + 1] = t.y; w[i + 2] = t.z; w[i + 3] = t.w;
            }
        }
    }
    // Elements lo <= e < hi only, zeros beside them.
    __device__ __forceinline__ void load_part(const T* p, int lo, int hi) {
        clear();
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e >= lo && e < hi) {
                if constexpr (sizeof(T) == 4)
                    w[e] = *reinterpret_cast<const uint32_t*>(p + e);
                else
                    w[e / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + e) << (e % 2 * 16);
            }
    }
    // Keeps elements lo <= e < hi of a whole vector, zeros beside them.
    __device__ __forceinline__ void keep(int lo, int hi) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < lo || e >= hi) {
                if constexpr (sizeof(T) == 4)
                    w[e] = 0;
                else
                    w[e / 2] &= e % 2 ? 0x0000ffffu : 0xffff0000u;
            }
    }
    __device__ __forceinline__ Pair get2(int e) const { return pair_of(get(e), get(e + 1)); }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(w[e]);
        else      // a bfloat16 is the upper half of a float32
            return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
};

// Copies BYTES from global to shared memory without waiting where that is possible (4, 8 or 16 bytes).
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else if constexpr (BYTES >= 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(BYTES) : "memory");
    else
        *static_cast<uint16_t*>(dst) = *static_cast<const uint16_t*>(src);
}

// A row of `dim` elements seen as vectors that are aligned in the whole tensor.  ALIGNED: every row starts and ends with a whole
// vector.  Otherwise its first and last vectors are shared with the neighbouring rows; those are read and written by element.
// All tensors of a call that have the row's shape and a 16-byte aligned start can be walked with the same spans (VEC elements are
// at most 16 bytes in a 16-bit type, and two 16-byte pieces in float32).
template <int VEC, bool ALIGNED>
struct RowSpan {
    size_t first;      // element index of vector 0 in the tensor
    int shift, dim;    // column of its first element, <= 0
    __host__ __device__ __forceinline__ RowSpan(long row, int d) : RowSpan(row, d, d) {}
    __host__ __device__ __forceinline__ RowSpan(long row, int d, long stride) {
        const size_t base = (size_t)row * stride;
        first = ALIGNED ? base : base / VEC * VEC;
        shift = ALIGNED ? 0 : -(int)(base - first);
        dim = d;
    }
    __host__ __device__ __forceinline__ int col(int v) const { return v * VEC + shift; }
    __host__ __device__ __forceinline__ size_t at(int v) const { return first + (size_t)v * VEC; }
    __host__ __device__ __forceinline__ bool any(int v) const { return col(v) < dim; }
    __host__ __device__ __forceinline__ bool whole(int v) const { return ALIGNED || (col(v) >= 0 && col(v) + VEC <= dim); }
    __host__ __device__ __forceinline__ int lo(int v) const { return col(v) < 0 ? -col(v) : 0; }
    __host__ __device__ __forceinline__ int hi(int v) const { return dim - col(v) < VEC ? dim - col(v) : VEC; }
    // The aligned loads of VEC + 4 columns around a vector, from its first column down to a multiple of 4, stay within the row's columns.
    __host__ __device__ __forceinline__ bool turns(int v) const { return whole(v) && (col(v) & ~3) + VEC + 4 <= dim; }
    template <typename T>
    __device__ __forceinline__ void load(RawVec<T, VEC>& r, const T* p, int v) const {
        if (!any(v)) r.clear();
        else if (whole(v)) r.load(p + at(v));
        else r.load_part(p + at(v), lo(v), hi(v));
    }
    template <typename T>
    __device__ __forceinline__ void store(T* p, int v, const float (&x)[VEC]) const {
        if (!any(v)) return;
        if (whole(v)) {
            store_vec<VEC>(p + at(v), x);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e >= lo(v) && e < hi(v)) store_one(p + at(v) + e, x[e]);
        }
    }
    // A vector that all rows share (`p` indexed by column); NULL: ones.
    __device__ __forceinline__ void load_columns(float (&g)[VEC], const float* __restrict__ p, int v) const {
#pragma unroll
        for (int e = 0; e < VEC; ++e) g[e] = 1.f;
        if (!p || !any(v)) return;
        if (ALIGNED) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                const float4 t = __ldg(reinterpret_cast<const float4*>(p + col(v) + e));
                g[e] = t.x; g[e + 1] = t.y; g[e + 2] = t.z; g[e + 3] = t.w;
            }
        } else if (turns(v) && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
            // aligned loads around the vector, turned by what its first column is behind a boundary: the same for the whole row
            float t[VEC + 4];
            const int turn = col(v) & 3;
            const float* q = p + col(v) - turn;
#pragma unroll
            for (int e = 0; e < VEC + 4; e += 4) {
                const float4 f = __ldg(reinterpret_cast<const float4*>(q + e));
                t[e] = f.x; t[e + 1] = f.y; t[e + 2] = f.z; t[e + 3] = f.w;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) g[e] = turn == 0 ? t[e] : turn == 1 ? t[e + 1] : turn == 2 ? t[e + 2] : t[e + 3];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e >= lo(v) && e < hi(v)) g[e] = __ldg(p + col(v) + e);
        }
    }
    // Vectors that a row of d elements may have.
    static __host__ __device__ int most(int d) { return ALIGNED ? d / VEC : (d + 2 * VEC - 2) / VEC; }
};

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

// A workspace that a handle owns: grows when a call needs more, never while the stream is being captured.  One that a captured graph
// holds is not freed when it is outgrown, since replays of the graph write there: it stays until the handle is destroyed.
struct Scratch {
    void* ptr;
    size_t bytes;
    bool in_graph;      // a call that was captured uses it
    Scratch* outgrown;  // earlier ones that graphs hold
};
inline int ensure_scratch(Scratch& s, size_t need, cudaStream_t stream, const char* reserve_call) {
    const bool capturing = stream_is_capturing(stream);
    if (s.bytes >= need) {
        s.in_graph = s.in_graph || capturing;
        return CIRC_OK;
    }
    if (capturing) {
        set_error(CIRC_ERR_UNSUPPORTED, "the workspace (%zu bytes) is too small for this call (%zu bytes) and the stream is being "
                  "captured: call %s before the capture", s.bytes, need, reserve_call);
        return CIRC_ERR_UNSUPPORTED;
    }
    if (s.in_graph) {
        Scratch* old = new (std::nothrow) Scratch(s);
        if (!old) {
            set_error(CIRC_ERR_ALLOC, "host allocation failed");
            return CIRC_ERR_ALLOC;
        }
        s = Scratch{nullptr, 0, false, old};
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
    if (!s.ptr && !s.outgrown) return;
    int prev = -1;
    cudaGetDevice(&prev);
    if (prev != device) cudaSetDevice(device);
    cudaFree(s.ptr);
    while (Scratch* old = s.outgrown) {
        cudaFree(old->ptr);
        s.outgrown = old->outgrown;
        delete old;
    }
    if (prev != device && prev >= 0) cudaSetDevice(prev);
    s = Scratch{};
}
// The current device for a new handle; false (with the error set) when there is none.
inline bool current_device(int* device) {
    if (cudaGetDevice(device) == cudaSuccess) return true;
    set_error(CIRC_ERR_CUDA, "no CUDA device: %s", cudaGetErrorString(cudaGetLastError()));
    return false;
}

}  // namespace circ
