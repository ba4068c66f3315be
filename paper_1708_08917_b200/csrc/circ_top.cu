// The `count` largest of a row's scores in descending order, equal ones by their class, and log sum exp(z / tau) over the whole row.
#include <new>
#include <type_traits>

#include "circ_softmax.cuh"

namespace circ {

constexpr int kTopMost = 256;      // scores a row

struct Top {
    int device;
    int classes, count;
    int dtype, ids_type;
    float temperature;
    Scratch ws;
};

struct TopArgs {
    long ld;
    void *values, *ids;
    float* lse;
    float scale;         // log2(e) / tau
    double inv_tau;
    int rows, classes, count;
};

// Whole numbers in the order of the scores; the zeros are equal, and a NaN is above all.  Of a bfloat16 the lower half is 0.
template <typename T>
__device__ __forceinline__ uint32_t order_of(T score) {
    const float z = to_float(score) + 0.f;
    const uint32_t b = __float_as_uint(z), o = z != z ? 0xffffffffu : b >> 31 ? ~b : b | 0x80000000u;
    return sizeof(T) == 4 ? o : o & 0xffff0000u;
}

// What has been found of a row, in any order; written in its final order: a score's place is the number of those before it.
struct Found {
    uint64_t key[kTopMost];      // order of the score, then the complement of the class
    __device__ __forceinline__ static uint64_t key_of(uint32_t order, int id) { return (uint64_t)order << 32 | (uint32_t)~id; }
    template <typename T, typename ID>
    __device__ __forceinline__ void write(const TopArgs& a, const T* __restrict__ zr, int row) const {
        for (int k = threadIdx.x; k < a.count; k += blockDim.x) {
            const uint64_t mine = key[k];
            int place = 0;
            for (int i = 0; i < a.count; ++i) place += key[i] > mine;
            const size_t at = (size_t)row * a.count + place;
            const int id = (int)~(uint32_t)mine;
            if (a.values) static_cast<T*>(a.values)[at] = zr[id];
            if (a.ids) static_cast<ID*>(a.ids)[at] = (ID)id;
        }
    }
};

// Any row: the order of its count-th score by digits of 8 bits from the top, then those above it, and of those equal to it the first.
template <typename T, typename ID>
__global__ void __launch_bounds__(512) top_any_kernel(const T* __restrict__ z, TopArgs a) {
    __shared__ Found found;
    __shared__ unsigned digits[256];
    __shared__ unsigned prefix, left, taken, warps[16];
    __shared__ Softmax part[16];
    pdl_begin();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* zr = z + (size_t)row * a.ld;
        if (a.lse) {
            Running run(a.scale);
            for (int c0 = tid; c0 < a.classes; c0 += 512 * 8) {
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = c0 + e * 512 < a.classes ? to_float(zr[c0 + e * 512]) : -INFINITY;
                run.take(s);
            }
            Softmax all = warp_join(run.done(), a.scale);
            if (lane == 0) part[warp] = all;
            __syncthreads();
            if (warp == 0) {
                all = warp_join(lane < 16 ? part[lane] : Softmax{-INFINITY, 0.f}, a.scale);
                const double base = all.top == -INFINITY ? 0.0 : (double)all.top;
                if (lane == 0) a.lse[row] = (float)(base * a.inv_tau + log((double)all.sum));
            }
        }
        if (tid == 0) {
            prefix = 0;
            left = a.count;
            taken = 0;
        }
        for (int shift = 24; shift >= 32 - 8 * (int)sizeof(T); shift -= 8) {
            if (tid < 256) digits[tid] = 0;
            __syncthreads();
            const uint32_t known = shift == 24 ? 0u : ~0u << (shift + 8), want = prefix;
            for (int c = tid; c < a.classes; c += 512) {
                const uint32_t o = order_of(zr[c]);
                if ((o & known) == want) atomicAdd(digits + (o >> shift & 255), 1u);
            }
            __syncthreads();
            if (tid == 0) {
                unsigned rest = left;
                int d = 255;
                while (d > 0 && digits[d] < rest) rest -= digits[d--];
                left = rest;
                prefix = want | (uint32_t)d << shift;
            }
            __syncthreads();
        }
        const uint32_t last = prefix;
        const int above = a.count - (int)left;
        for (int c = tid; c < a.classes; c += 512) {
            const uint32_t o = order_of(zr[c]);
            if (o > last) found.key[atomicAdd(&taken, 1u)] = Found::key_of(o, c);
        }
        __syncthreads();
        int have = above;
        for (int c0 = 0; c0 < a.classes && have < a.count; c0 += 512) {
            const int c = c0 + tid;
            const uint32_t o = c < a.classes ? order_of(zr[c]) : 0u;
            const bool equal = c < a.classes && o == last;
            const unsigned lanes = __ballot_sync(0xffffffffu, equal);
            if (lane == 0) warps[warp] = __popc(lanes);
            __syncthreads();
            int before = 0, all = 0;
            for (int w = 0; w < 16; ++w) {
                before += w < warp ? (int)warps[w] : 0;
                all += (int)warps[w];
            }
            const int at = have + before + __popc(lanes & ((1u << lane) - 1));
            if (equal && at < a.count) found.key[at] = Found::key_of(o, c);
            have += all;
            __syncthreads();
        }
        __syncthreads();
        found.write<T, ID>(a, zr, row);
        __syncthreads();
    }
}

template <typename T, typename ID>
static cudaError_t dispatch_top(const T* z, const TopArgs& a, cudaStream_t s) {
    return launch_row(top_any_kernel<T, ID>, dim3((unsigned)(a.rows < 148 * 16 ? a.rows : 148 * 16)), dim3(512), 0, s, z, a);
}

static int run_top(Top* t, const void* z, long ld, void* values, void* ids, float* lse, long rows, cudaStream_t s) {
    if (!t) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (rows < 0 || rows > (1L << 24) || ld < t->classes) {
        set_error(CIRC_ERR_SHAPE, "rows=%ld must be in [0, 2^24] and the stride %ld at least classes=%d", rows, ld, t->classes);
        return CIRC_ERR_SHAPE;
    }
    if (rows == 0) return CIRC_OK;
    if (!z || (!values && !ids && !lse)) {
        set_error(CIRC_ERR_ARG, "logits and one of values, ids and lse must be non-NULL");
        return CIRC_ERR_ARG;
    }
    const size_t zb = dtype_bytes(t->dtype);
    if (misaligned(z, zb) || misaligned(values, zb) || misaligned(ids, t->ids_type == CIRC_I64 ? 8 : 4) || misaligned(lse, 4)) {
        set_error(CIRC_ERR_ARG, "every pointer must be aligned to its element size");
        return CIRC_ERR_ARG;
    }
    const TopArgs a{ld, values, ids, lse, (float)(1.4426950408889634 / (double)t->temperature), 1.0 / (double)t->temperature, (int)rows, t->classes, t->count};
    cudaError_t err = cudaSuccess;
    with_dtype(t->dtype, [&](auto* e) {
        with_index_type(t->ids_type, [&](auto* i) {
            using T = tag_type<decltype(e)>;
            using ID = tag_type<decltype(i)>;
            err = dispatch_top<T, ID>(static_cast<const T*>(z), a, s);
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(1);
    return CIRC_OK;
}

}  // namespace circ

using namespace circ;

extern "C" {

circ_top_handle circ_top_create(int classes, int count) {
    if (classes < 1 || classes > (1 << 28) || count < 1 || count > kTopMost || count > classes) {
        set_error(CIRC_ERR_SHAPE, "classes=%d must be in [1, 2^28], count=%d in [1, %d] and at most classes", classes, count, kTopMost);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Top* t = new (std::nothrow) Top{device, classes, count, CIRC_F32, CIRC_I64, 1.f, {}};
    if (!t) set_error(CIRC_ERR_ALLOC, "host allocation failed");
    return reinterpret_cast<circ_top_handle>(t);
}

void circ_top_destroy(circ_top_handle h) {
    Top* t = reinterpret_cast<Top*>(h);
    if (!t) return;
    free_on(t->device, t->ws);
    delete t;
}

int circ_top_set_dtypes(circ_top_handle h, int logits_dtype, int ids_type) {
    Top* t = reinterpret_cast<Top*>(h);
    if (!t || !float_dtype(logits_dtype) || (ids_type != CIRC_I32 && ids_type != CIRC_I64)) {
        set_error(CIRC_ERR_ARG, "bad handle or type codes (%d, %d)", logits_dtype, ids_type);
        return CIRC_ERR_ARG;
    }
    t->dtype = logits_dtype;
    t->ids_type = ids_type;
    return CIRC_OK;
}

int circ_top_set_temperature(circ_top_handle h, float temperature) {
    Top* t = reinterpret_cast<Top*>(h);
    if (!t || !(temperature >= 1e-6f && temperature <= 1e6f)) {
        set_error(CIRC_ERR_ARG, "bad handle, or temperature %g outside [1e-6, 1e6]", (double)temperature);
        return CIRC_ERR_ARG;
    }
    t->temperature = temperature;
    return CIRC_OK;
}

int circ_top_reserve(circ_top_handle h, long max_rows) {
    Top* t = reinterpret_cast<Top*>(h);
    if (!t || max_rows < 0 || max_rows > (1L << 24)) {
        set_error(CIRC_ERR_ARG, "bad handle or max_rows %ld", max_rows);
        return CIRC_ERR_ARG;
    }
    return CIRC_OK;
}

int circ_top_forward(circ_top_handle h, const void* logits, long stride, void* values, void* ids, float* lse, long rows, void* stream) {
    return run_top(reinterpret_cast<Top*>(h), logits, stride, values, ids, lse, rows, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
