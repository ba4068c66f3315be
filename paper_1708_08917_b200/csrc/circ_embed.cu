// Embedding table in front of a network of circulant layers:
//   forward   y[t] = scale * table[ids[t]]                          (a zero row where ids[t] is the padding id or outside the table)
//   backward  grad_table[v] = scale * sum over { t : ids[t] = v } of grad_y[t]     (zero where no token has id v)
#include <new>
#include <type_traits>

#include "circ_rows.cuh"

namespace circ {

struct Embed {
    int device;
    int vocab, dim;
    int table_dtype, y_dtype, ids_type;
    float scale;
    long padding;
    Scratch ws;
};

template <typename TT, typename TY, typename ID>
__global__ void __launch_bounds__(256) embed_forward_kernel(const TT* __restrict__ table, const ID* __restrict__ ids, TY* __restrict__ y,
                                                            int vocab, int dim, float scale, long padding) {
    const long t = blockIdx.x;
    const long id = (long)ids[t];
    const bool row = id >= 0 && id < vocab && id != padding;
    for (int c = threadIdx.x; c < dim; c += blockDim.x)
        store_one(y + t * dim + c, row ? scale * to_float(table[id * dim + c]) : 0.f);
}

// One thread block per table row: every thread walks all ids in order and adds up its columns of the matching rows.
template <typename TT, typename TY, typename ID>
__global__ void __launch_bounds__(256) embed_backward_kernel(const ID* __restrict__ ids, const TY* __restrict__ dy, TT* __restrict__ dt,
                                                             long tokens, int dim, float scale, long padding) {
    const long v = blockIdx.x;
    for (int c = threadIdx.x; c < dim; c += blockDim.x) {
        float sum = 0.f;
        if (v != padding)
            for (long t = 0; t < tokens; ++t)
                if ((long)ids[t] == v) sum += to_float(dy[t * dim + c]);
        store_one(dt + v * dim + c, scale * sum);
    }
}

static int check_embed(const Embed* e, long tokens) {
    if (!e) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (tokens < 0 || tokens > INT32_MAX) {
        set_error(CIRC_ERR_SHAPE, "tokens=%ld must be in [0, 2^31)", tokens);
        return CIRC_ERR_SHAPE;
    }
    return CIRC_OK;
}

}  // namespace circ

using namespace circ;

extern "C" {

circ_embed_handle circ_embed_create(int vocab, int dim) {
    if (vocab < 1 || dim < 1) {
        set_error(CIRC_ERR_SHAPE, "vocab=%d and dim=%d must be >= 1", vocab, dim);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Embed* e = new (std::nothrow) Embed{device, vocab, dim, CIRC_F32, CIRC_F32, CIRC_I64, 1.f, -1, {nullptr, 0}};
    if (!e) set_error(CIRC_ERR_ALLOC, "host allocation failed");
    return reinterpret_cast<circ_embed_handle>(e);
}

void circ_embed_destroy(circ_embed_handle h) {
    Embed* e = reinterpret_cast<Embed*>(h);
    if (!e) return;
    free_on(e->device, e->ws);
    delete e;
}

int circ_embed_set_dtypes(circ_embed_handle h, int table_dtype, int y_dtype, int ids_type) {
    Embed* e = reinterpret_cast<Embed*>(h);
    if (!e || !float_dtype(table_dtype) || !float_dtype(y_dtype) || (ids_type != CIRC_I32 && ids_type != CIRC_I64)) {
        set_error(CIRC_ERR_ARG, "bad handle or type codes (%d, %d, %d)", table_dtype, y_dtype, ids_type);
        return CIRC_ERR_ARG;
    }
    e->table_dtype = table_dtype;
    e->y_dtype = y_dtype;
    e->ids_type = ids_type;
    return CIRC_OK;
}

int circ_embed_set_scale(circ_embed_handle h, float scale) {
    Embed* e = reinterpret_cast<Embed*>(h);
    if (!e) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    e->scale = scale;
    return CIRC_OK;
}

int circ_embed_set_padding(circ_embed_handle h, long padding) {
    Embed* e = reinterpret_cast<Embed*>(h);
    if (!e || padding < -1 || padding >= e->vocab) {
        set_error(CIRC_ERR_ARG, "bad handle or padding id %ld (-1: none)", padding);
        return CIRC_ERR_ARG;
    }
    e->padding = padding;
    return CIRC_OK;
}

int circ_embed_reserve(circ_embed_handle h, long max_tokens) {
    Embed* e = reinterpret_cast<Embed*>(h);
    return check_embed(e, max_tokens);
}

int circ_embed_forward(circ_embed_handle h, const void* table, const void* ids, void* y, long tokens, void* stream) {
    Embed* e = reinterpret_cast<Embed*>(h);
    int rc = check_embed(e, tokens);
    if (rc != CIRC_OK || tokens == 0) return rc;
    if (!table || !ids || !y || table == y || ids == y) {
        set_error(CIRC_ERR_ARG, "table, ids and y must be non-NULL and y distinct");
        return CIRC_ERR_ARG;
    }
    if (misaligned(table, dtype_bytes(e->table_dtype)) || misaligned(y, dtype_bytes(e->y_dtype)) || misaligned(ids, e->ids_type == CIRC_I64 ? 8 : 4)) {
        set_error(CIRC_ERR_ARG, "table, ids and y must be aligned to their element sizes");
        return CIRC_ERR_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    with_dtype(e->table_dtype, [&](auto* t) {
        with_dtype(e->y_dtype, [&](auto* o) {
            with_index_type(e->ids_type, [&](auto* i) {
                using TT = tag_type<decltype(t)>;
                using TY = tag_type<decltype(o)>;
                using ID = tag_type<decltype(i)>;
                embed_forward_kernel<TT, TY, ID><<<(unsigned)tokens, 256, 0, s>>>(
                    static_cast<const TT*>(table), static_cast<const ID*>(ids), static_cast<TY*>(y), e->vocab, e->dim, e->scale, e->padding);
            });
        });
    });
    count_launches(1);
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

int circ_embed_backward(circ_embed_handle h, const void* ids, const void* grad_y, void* grad_table, long tokens, void* stream) {
    Embed* e = reinterpret_cast<Embed*>(h);
    int rc = check_embed(e, tokens);
    if (rc != CIRC_OK) return rc;
    if (!grad_table || (tokens > 0 && (!ids || !grad_y)) || grad_table == grad_y || grad_table == ids) {
        set_error(CIRC_ERR_ARG, "ids, grad_y and grad_table must be non-NULL and grad_table distinct");
        return CIRC_ERR_ARG;
    }
    if (misaligned(grad_table, dtype_bytes(e->table_dtype)) || misaligned(grad_y, dtype_bytes(e->y_dtype)) ||
        misaligned(ids, e->ids_type == CIRC_I64 ? 8 : 4)) {
        set_error(CIRC_ERR_ARG, "ids, grad_y and grad_table must be aligned to their element sizes");
        return CIRC_ERR_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    with_dtype(e->table_dtype, [&](auto* t) {
        with_dtype(e->y_dtype, [&](auto* o) {
            with_index_type(e->ids_type, [&](auto* i) {
                using TT = tag_type<decltype(t)>;
                using TY = tag_type<decltype(o)>;
                using ID = tag_type<decltype(i)>;
                embed_backward_kernel<TT, TY, ID><<<(unsigned)e->vocab, 256, 0, s>>>(
                    static_cast<const ID*>(ids), static_cast<const TY*>(grad_y), static_cast<TT*>(grad_table), tokens, e->dim, e->scale,
                    e->padding);
            });
        });
    });
    count_launches(1);
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

}  // extern "C"
