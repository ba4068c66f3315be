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

// ---- forward -------------------------------------------------------------------------------------------------
// Pure data movement.  The output is walked as one run of vectors (VEC elements, 16 bytes or more per access when the rows
// allow it): a thread takes UNROLL of them, a thread block apart, so that several rows' loads are in flight behind their ids.
// 8192 tokens of 4096 from a float32 table into bfloat16: 22 us, 5.6 TB/s of table rows and output.
// (step_rows, step_vecs): 256 vectors as whole rows and vectors, so that a thread divides once.
template <typename TT, typename TY, typename ID, int VEC, int UNROLL>
__global__ void __launch_bounds__(256) embed_forward_kernel(const TT* __restrict__ table, const ID* __restrict__ ids, TY* __restrict__ y, int tokens,
                                                            unsigned vec_per_row, unsigned step_rows, unsigned step_vecs, unsigned vocab, int dim,
                                                            float scale, unsigned padding) {
    pdl_begin();
    const long first = (long)blockIdx.x * (256 * UNROLL);
    const long row0 = first / vec_per_row;         // the block's first vector; the rest is small-integer arithmetic
    const unsigned k = (unsigned)(first - row0 * vec_per_row) + threadIdx.x, rows = k / vec_per_row;
    unsigned c = k - rows * vec_per_row;
    long t = row0 + rows;
    RawVec<TT, VEC> raw[UNROLL];
    unsigned col[UNROLL];
    long token[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        col[u] = c * VEC;
        token[u] = t;
        raw[u].clear();
        if (t < tokens) {
            const ID id = __ldg(ids + t);
            const unsigned lo = (unsigned)id;
            bool row = lo < vocab && lo != padding;
            if constexpr (sizeof(ID) == 8) row = row && (unsigned)((uint64_t)id >> 32) == 0;
            if (row) raw[u].load(table + (size_t)lo * dim + col[u]);
        }
        t += step_rows;
        c += step_vecs;
        if (c >= vec_per_row) {
            c -= vec_per_row;
            ++t;
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        if (token[u] >= tokens) break;
        float v[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = raw[u].get(e) * scale;
        store_vec<VEC>(y + token[u] * dim + col[u], v);
    }
}

// Rows that do not lie on 16-byte boundaries: a block has a stretch of one row, by element, eight in flight a thread.  8192 tokens of
// 4095: 38 us (vectors, at 4096: 23).
template <typename TT, typename TY, typename ID>
__global__ void __launch_bounds__(256) embed_forward_any_kernel(const TT* __restrict__ table, const ID* __restrict__ ids, TY* __restrict__ y, unsigned chunks,
                                                                unsigned vocab, int dim, float scale, unsigned padding) {
    pdl_begin();
    const unsigned t = blockIdx.x / chunks;
    const int c0 = (int)(blockIdx.x - t * chunks) * (8 * blockDim.x) + threadIdx.x;
    const ID id = __ldg(ids + t);
    const unsigned lo = (unsigned)id;
    bool row = lo < vocab && lo != padding;
    if constexpr (sizeof(ID) == 8) row = row && (unsigned)((uint64_t)id >> 32) == 0;
    const TT* src = table + (size_t)(row ? lo : 0) * dim;
    TY* dst = y + (size_t)t * dim;
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int c = c0 + u * (int)blockDim.x;
        v[u] = row && c < dim ? to_float(src[c]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int c = c0 + u * (int)blockDim.x;
        if (c < dim) store_one(dst + c, v[u] * scale);
    }
}

// ---- backward ------------------------------------------------------------------------------------------------
// The tokens are sorted by id (1), then every table row is the sum of its run of sorted tokens (2), and runs that were
// cut for balance are put together (3).  Nothing is added through atomics: the order of every sum follows from the ids.
//
// (1) A thread block owns a class of table rows, the ids equal to it modulo the number of classes, and reads all ids: with its
// counts per (warp, row) it knows the place of each of its tokens in the whole order without hearing from another block, since the
// tokens in front of its class are those of lower classes.  (Classes and not ranges: ids are commonly handed out by frequency, and
// a block with the first 1/128 of the ids had half of the tokens.)  Warps take consecutive parts of the tokens, so that equal ids
// stay in the order of their positions.  Reading the ids is what takes the time (every block reads all of them from L2), so it is done once:
// a warp lists its tokens as it finds them.  32768 64-bit ids: 17 us, of which 4 are launch and set-up.  The rows' order behind is (class, id); `slot` numbers the rows in that order.
// (2) The work is the list of all rows, each with its reads and then its write, laid out on a line whose unit is a byte of
// traffic per column; `workers` groups of GROUP threads take equal stretches of it, whatever the ids are.  A stretch that ends in
// a run of more than kWholeRun tokens cuts it (the part before goes to `carry`, the part in which the row ends to `tail`); shorter
// runs go whole to the worker they end with.  32768 tokens of 2048 bfloat16 into 65536 float32 rows: 122 us, 5.4 TB/s; waiting for memory
// (the same table is cleared at 7.3 TB/s).  Where a stretch begins is found by the sort, by the block that knows its row.
constexpr int kWholeRun = 16, kLongChain = 6;

struct Bound {
    int row, read;         // reads before `read` and slots before `row` lie before the bound
};
struct EmbedSum {
    int* start;            // [slots + 1] first sorted token of a slot
    int* order;            // [tokens]
    Bound* bound;          // [workers + 1]
    long* stretch;         // [1] length of a stretch: worker p begins at p * stretch
    float* carry;          // [workers][dim]
    float* tail;           // [workers][dim]
    int* cuts;             // [2] rows that are put together from parts: from few, from more than kLongChain
    int4* cut;             // [2][workers] (row, first worker that holds a part of it, the one in which it ends, 0), in any order
    int vocab, dim, workers;
    int bits, per_class, slots;     // slot = (id mod 2^bits) * per_class + id / 2^bits; those of ids >= vocab are empty
    int read_cost, row_cost;
    float scale;
};
__device__ __forceinline__ int slot_id(const EmbedSum& a, int slot) { return ((slot % a.per_class) << a.bits) + slot / a.per_class; }

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortUnroll = 16;
constexpr int kSortRows = 1280;              // table rows of a block at most: 32 warps x 1280 counts are 160 KB of shared memory
constexpr size_t kSortShared = 200 * 1024;   // what the counts leave of it holds the warps' lists of tokens

// The row's number within class `cls` of 2^bits classes; kNotOurs for an id of another class or for no token.  `less`, `all`: counts of
// tokens of lower classes and of all classes.  Negative ids are above every row as unsigned numbers.
constexpr unsigned kNotOurs = 0xffffffffu;
template <typename ID>
__device__ __forceinline__ unsigned class_row(ID id, unsigned cls, int bits, unsigned vocab, unsigned padding, int& less, int& all) {
    const unsigned lo = (unsigned)id, own = lo & ((1u << bits) - 1);
    bool token = lo < vocab && lo != padding;
    if constexpr (sizeof(ID) == 8) token = token && (unsigned)((uint64_t)id >> 32) == 0;
    less += token && own < cls;
    all += token;
    return token && own == cls ? lo >> bits : kNotOurs;
}

template <typename ID>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const ID* __restrict__ ids, int tokens, unsigned padding, int room, EmbedSum a) {
    const int rows_per_block = a.per_class;
    extern __shared__ __align__(16) int count[];   // [warp][rows_per_block], first counts, then places; then the warps' lists
    __shared__ int part[kSortWarps], below[kSortWarps], valid[kSortWarps];
    pdl_begin();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int per_warp = ((tokens + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    const int begin = warp * per_warp < tokens ? warp * per_warp : tokens, end = begin + per_warp < tokens ? begin + per_warp : tokens;
    int* mine = count + warp * rows_per_block;
    // the warp's tokens of this class, in order: (row, token); where they are more than the list has room for they are found again
    int2* list = reinterpret_cast<int2*>(count + kSortWarps * rows_per_block) + warp * room;
    int less = 0, all = 0, listed = 0;
    // the rows of the next 16 x 32 tokens, 0xffffffff where they are not ours
    auto fetch = [&](int t0, unsigned (&row)[kSortUnroll]) {
        ID id[kSortUnroll];
#pragma unroll
        for (int u = 0; u < kSortUnroll; ++u) id[u] = t0 + u * 32 + lane < end ? __ldg(ids + t0 + u * 32 + lane) : (ID)-1;
#pragma unroll
        for (int u = 0; u < kSortUnroll; ++u) row[u] = class_row(id[u], blockIdx.x, a.bits, (unsigned)a.vocab, padding, less, all);
    };
    for (int i = threadIdx.x; i < kSortWarps / 4 * rows_per_block; i += kSortThreads) reinterpret_cast<int4*>(count)[i] = make_int4(0, 0, 0, 0);
    if (blockIdx.x == 0 && threadIdx.x < 2) a.cuts[threadIdx.x] = 0;
    __syncthreads();
    for (int t0 = begin; t0 < end; t0 += 32 * kSortUnroll) {
        unsigned row[kSortUnroll];
        fetch(t0, row);
#pragma unroll
        for (int u = 0; u < kSortUnroll; ++u) {
            const bool ours = row[u] != kNotOurs;
            const unsigned some = __ballot_sync(0xffffffffu, ours);
            if (!some) continue;
            const int at = listed + __popc(some & ((1u << lane) - 1));
            if (ours) {
                atomicAdd(mine + row[u], 1);
                if (at < room) list[at] = make_int2((int)row[u], t0 + u * 32 + lane);
            }
            listed += __popc(some);
        }
    }
    less = __reduce_add_sync(0xffffffffu, less);
    all = __reduce_add_sync(0xffffffffu, all);
    if (lane == 0) {
        below[warp] = less;
        valid[warp] = all;
    }
    __syncthreads();
    // exclusive sums over the block's rows; a thread takes consecutive ones
    const int rpt = (rows_per_block + kSortThreads - 1) / kSortThreads;
    int sum = 0;
    for (int i = 0; i < rpt; ++i) {
        const int r = threadIdx.x * rpt + i;
        if (r < rows_per_block)
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) sum += count[w * rows_per_block + r];
    }
    int scan = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += up;
    }
    if (lane == 31) part[warp] = scan;
    __syncthreads();
    int place = scan - sum + __reduce_add_sync(0xffffffffu, below[lane] + (lane < warp ? part[lane] : 0));
    const long total = (long)__reduce_add_sync(0xffffffffu, valid[lane]) * a.read_cost + (long)a.slots * a.row_cost, stretch = total / a.workers + 1;
    for (int i = 0; i < rpt; ++i) {
        const int r = threadIdx.x * rpt + i, slot = blockIdx.x * rows_per_block + r, first = place;
        const bool row = r < rows_per_block;
        long p0 = 0, p1 = 0;                    // the stretches that begin in this slot, which is [from, to) on the line
        if (row) {
            a.start[slot] = first;
            int n[kSortWarps];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) n[w] = count[w * rows_per_block + r];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                count[w * rows_per_block + r] = place;
                place += n[w];
            }
            const long from = (long)first * a.read_cost + (long)slot * a.row_cost, to = (long)place * a.read_cost + (long)(slot + 1) * a.row_cost;
            p0 = (from + stretch - 1) / stretch;
            p1 = (to + stretch - 1) / stretch;
            if (slot == a.slots - 1) {          // the end of the line, and stretches behind it
                a.start[a.slots] = place;
                for (long p = p1; p <= a.workers; ++p) a.bound[p] = Bound{a.slots, place};
                *a.stretch = stretch;
            }
        }
        // a slot with many stretches has the whole warp's help
        for (unsigned left = __ballot_sync(0xffffffffu, p1 > p0); left; left &= left - 1) {
            const int src = __ffs(left) - 1, sl = __shfl_sync(0xffffffffu, slot, src), s0 = __shfl_sync(0xffffffffu, first, src);
            const int cnt = __shfl_sync(0xffffffffu, place, src) - s0;
            const long q0 = __shfl_sync(0xffffffffu, p0, src), q1 = __shfl_sync(0xffffffffu, p1, src);
            const long from = (long)s0 * a.read_cost + (long)sl * a.row_cost;
            for (long p = q0 + lane; p < q1; p += 32) {
                const long into = (p * stretch - from + a.read_cost - 1) >> (a.read_cost == 4 ? 2 : 1);     // a read costs 2 or 4
                a.bound[p] = Bound{sl, cnt <= kWholeRun ? s0 : s0 + (int)(into < cnt ? into : cnt)};
            }
        }
    }
    __syncthreads();
    // 32 tokens in their order to their rows' places; called by whole warps
    auto deal = [&](unsigned row, int token) {
        const bool ours = row != kNotOurs;
        const unsigned some = __ballot_sync(0xffffffffu, ours);
        if (ours) {
            const unsigned same = __match_any_sync(some, row);
            const int rank = __popc(same & ((1u << lane) - 1)), base = mine[row];
            __syncwarp(some);
            if (rank == 0) mine[row] = base + __popc(same);
            a.order[base + rank] = token;
        }
        __syncwarp();
    };
    if (listed <= room) {
        for (int i = 0; i < listed; i += 32) {
            const int2 e = i + lane < listed ? list[i + lane] : make_int2(-1, 0);
            deal((unsigned)e.x, e.y);
        }
    } else {
        for (int t0 = begin; t0 < end; t0 += 32 * kSortUnroll) {
            unsigned row[kSortUnroll];
            fetch(t0, row);
#pragma unroll
            for (int u = 0; u < kSortUnroll; ++u) deal(row[u], t0 + u * 32 + lane);
        }
    }
}

// A thread has PARTS vectors of a row, GROUP vectors apart: enough bytes a row that the walk over rows costs little next to them.
constexpr int kSumBlocks = 4;        // resident blocks of 256 threads on an SM, 48 KB of ring each
constexpr int ring_depth(int bytes) { return bytes <= 16 ? 12 : 6; }
template <typename TT, typename TY, int VEC, int PARTS, int GROUP>
__global__ void __launch_bounds__(256, kSumBlocks) embed_sum_kernel(EmbedSum a, const TY* __restrict__ dy, TT* __restrict__ dt) {
    // Loads run ahead of the sums over the sorted tokens, whatever the rows they belong to: DEPTH tokens are in flight in a ring of
    // shared memory in which every thread copies and reads its own vectors (no barrier between threads is needed).
    constexpr int BYTES = VEC * (int)sizeof(TY), DEPTH = ring_depth(PARTS * BYTES);
    extern __shared__ __align__(16) unsigned char ring[];
    auto place = [&](int slot, int c) { return ring + ((size_t)(slot * PARTS + c) * 256 + threadIdx.x) * BYTES; };
    pdl_begin();
    const int p = blockIdx.x * (256 / GROUP) + threadIdx.x / GROUP, lane = threadIdx.x % 32;
    if (p >= a.workers) return;      // whole warps: GROUP is a multiple of 32
    const int col = (int)(blockIdx.y * (PARTS * GROUP) + threadIdx.x % GROUP) * VEC;
    const Bound from = a.bound[p], to = a.bound[p + 1];
    int j = from.read, ahead = j, tokens = 0, slot = 0, slot_in = 0;      // `tokens`: 32 sorted tokens, one a lane, of which `ahead` is next
    auto fetch = [&]() {
        if (ahead < to.read) {
            const int k = (ahead - from.read) % 32;
            if (k == 0) tokens = ahead + lane < to.read ? __ldg(a.order + ahead + lane) : 0;
            const TY* src = dy + (long)__shfl_sync(0xffffffffu, tokens, k) * a.dim + col;
#pragma unroll
            for (int c = 0; c < PARTS; ++c)
                if (col + c * GROUP * VEC < a.dim) copy_async<BYTES>(place(slot_in, c), src + c * GROUP * VEC);
            ++ahead;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        slot_in = slot_in + 1 == DEPTH ? 0 : slot_in + 1;
    };
#pragma unroll 1
    for (int u = 0; u < DEPTH; ++u) fetch();
    int in_class = from.row % a.per_class, id = slot_id(a, from.row), ends = 0;
    bool begun = from.read > __ldg(a.start + from.row);     // the first row began in an earlier stretch
    for (int v = from.row;; ++v) {
        const int k = (v - from.row) % 32;
        if (k == 0) ends = __ldg(a.start + (v + lane < a.slots ? v + lane + 1 : a.slots));
        const bool open = v == to.row;                      // the part of a row that ends in a later stretch
        const int end = open ? to.read : __shfl_sync(0xffffffffu, ends, k);
        if (open && end == j && !(begun && v == from.row)) break;
        float sum[PARTS][VEC];
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[c][e] = 0.f;
#pragma unroll 1
        for (; j < end; ++j) {
            asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
#pragma unroll
            for (int c = 0; c < PARTS; ++c)
                if (col + c * GROUP * VEC < a.dim) {
                    RawVec<TY, VEC> raw;
                    raw.load(reinterpret_cast<const TY*>(place(slot, c)));
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[c][e] += raw.get(e);
                }
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
            fetch();
        }
        if (open || begun) {
            float* part = (open ? a.carry : a.tail) + (size_t)p * a.dim + col;
#pragma unroll
            for (int c = 0; c < PARTS; ++c)
                if (col + c * GROUP * VEC < a.dim) store_vec<VEC>(part + c * GROUP * VEC, sum[c]);
            if (open) break;
            begun = false;
            if (blockIdx.y == 0 && threadIdx.x % GROUP == 0) {
                // the stretch that holds the row's first read
                const int q = (int)(((long)__ldg(a.start + v) * a.read_cost + (long)v * a.row_cost) / *a.stretch);
                const int many = p - q > kLongChain;
                a.cut[(size_t)many * a.workers + atomicAdd(a.cuts + many, 1)] = make_int4(id, q, p, 0);
            }
        } else if (id < a.vocab) {
            TT* row = dt + (size_t)id * a.dim + col;
#pragma unroll
            for (int c = 0; c < PARTS; ++c)
                if (col + c * GROUP * VEC < a.dim) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[c][e] *= a.scale;
                    store_vec_once<VEC>(row + c * GROUP * VEC, sum[c]);
                }
        }
        id += 1 << a.bits;
        if (++in_class == a.per_class) {
            in_class = 0;
            id = (v + 1) / a.per_class;
        }
    }
}

// (3) Rows that were cut: carry of the stretches before, in their order, and the tail.  A warp takes 128 columns of a row; where
// the row has many parts, a block takes 32 columns and its 8 warps share the parts, so that a row with most of the tokens is no
// chain of loads.  7 us behind the sums above (107 rows cut), 3 us with none.

template <typename TT>
__global__ void __launch_bounds__(256) embed_join_kernel(EmbedSum a, TT* __restrict__ dt) {
    pdl_begin();
    __shared__ float parts[8][33];
    const int few = a.cuts[0], many = a.cuts[1], warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int slices = (a.dim + 127) / 128, thin = (a.dim + 31) / 32;
    for (int item = blockIdx.x * 8 + warp; item < few * slices; item += gridDim.x * 8) {
        const int4 cut = a.cut[item / slices];
        const int col = item % slices * 128 + lane;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int q = cut.y; q <= cut.z; ++q) {
            const float* src = (q < cut.z ? a.carry : a.tail) + (size_t)q * a.dim;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + 32 * e < a.dim) sum[e] += src[col + 32 * e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + 32 * e < a.dim) store_one(dt + (size_t)cut.x * a.dim + col + 32 * e, a.scale * sum[e]);
    }
    for (int item = blockIdx.x; item < many * thin; item += gridDim.x) {
        const int4 cut = a.cut[a.workers + item / thin];
        const int col = item % thin * 32 + lane, per = (cut.z - cut.y + 7) / 8;
        const int from = cut.y + warp * per, to = from + per < cut.z ? from + per : cut.z;
        float sum = 0.f;
        if (col < a.dim)
#pragma unroll 8
            for (int q = from; q < to; ++q) sum += a.carry[(size_t)q * a.dim + col];
        parts[warp][lane] = sum;
        __syncthreads();
        if (warp == 0 && col < a.dim) {
#pragma unroll
            for (int w = 1; w < 8; ++w) sum += parts[w][lane];
            store_one(dt + (size_t)cut.x * a.dim + col, a.scale * (sum + a.tail[(size_t)cut.z * a.dim + col]));
        }
        __syncthreads();
    }
}

// ---- few tokens: one launch ----
// A thread block owns the table rows equal to its number modulo the blocks, for a slice of 2 x 32 vectors of columns, and picks its
// tokens out of all ids in their order.  Its warps write a row each: most are zero.  A row with many tokens is left to all warps
// together, each with an eighth of the block's tokens, added up in order.  Reading all ids in every block is what limits it to kFewTokens.
// 513 tokens of 1000 into 10007 rows of float32: 10.4 us a call, 2048 of 2048 into 65536: 92 us, 5.9 TB/s.
constexpr int kFewTokens = 2048, kFewRows = 2048, kFewLong = 16;

template <typename TT, typename TY, typename ID, int VEC>
__global__ void __launch_bounds__(256, 4) embed_few_kernel(const ID* __restrict__ ids, const TY* __restrict__ dy, TT* __restrict__ dt, int tokens, int vocab,
                                                           unsigned padding, int dim, float scale) {
    constexpr int PARTS = 2, PER = kFewTokens / 256, WIDTH = PARTS * 32 * VEC;
    __shared__ int tok[kFewTokens], row[kFewTokens], count[kFewRows], found[PER * 8], longs[kFewTokens / kFewLong], many;
    __shared__ __align__(16) float sums[8][WIDTH];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const unsigned blocks = gridDim.x, b = blockIdx.x;
    pdl_begin();
    const int rows = (int)((vocab - b + blocks - 1) / blocks);
    unsigned own[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = i * 256 + tid;
        const ID id = t < tokens ? __ldg(ids + t) : (ID)-1;
        const unsigned lo = (unsigned)id;
        bool mine = lo < (unsigned)vocab && lo != padding;
        if constexpr (sizeof(ID) == 8) mine = mine && (unsigned)((uint64_t)id >> 32) == 0;
        own[i] = mine && lo % blocks == b ? lo / blocks : kNotOurs;
    }
    for (int i = tid; i < rows; i += 256) count[i] = 0;
    if (tid == 0) many = 0;
    unsigned hits[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        hits[i] = __ballot_sync(0xffffffffu, own[i] != kNotOurs);
        if (lane == 0) found[i * 8 + warp] = __popc(hits[i]);
    }
    __syncthreads();
    // places in the order of the tokens: exclusive sums over (i, warp), two a lane
    const int f0 = found[2 * lane], f1 = found[2 * lane + 1];
    int scan = f0 + f1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += up;
    }
    const int n = __shfl_sync(0xffffffffu, scan, 31), before = scan - f0 - f1;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = i * 8 + warp, at0 = __shfl_sync(0xffffffffu, before, k / 2), at1 = __shfl_sync(0xffffffffu, before + f0, k / 2);
        if (own[i] != kNotOurs) {
            const int at = (k % 2 ? at1 : at0) + __popc(hits[i] & ((1u << lane) - 1));
            tok[at] = i * 256 + tid;
            row[at] = (int)own[i];
            atomicAdd(&count[own[i]], 1);
        }
    }
    __syncthreads();
    const int col = blockIdx.y * WIDTH + lane * VEC;
    float sum[PARTS][VEC];
    auto clear = [&]() {
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[c][e] = 0.f;
    };
    // adds the block's tokens from..to that belong to row r, up to four in flight
    auto add_tokens = [&](int from, int to, int r) {
        for (int base = from; base < to; base += 32) {
            const bool in = base + lane < to && row[base + lane] == r;
            const int mine = in ? tok[base + lane] : 0;
            unsigned m = __ballot_sync(0xffffffffu, in);
            while (m) {
                RawVec<TY, VEC> raw[4][PARTS];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int k = m ? __ffs(m) - 1 : 0;
                    const TY* src = dy + (size_t)__shfl_sync(0xffffffffu, mine, k) * dim + col;
#pragma unroll
                    for (int c = 0; c < PARTS; ++c) {
                        if (m && col + c * 32 * VEC < dim) raw[u][c].load(src + c * 32 * VEC);
                        else raw[u][c].clear();
                    }
                    m &= m - 1;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int c = 0; c < PARTS; ++c)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) sum[c][e] += raw[u][c].get(e);
            }
        }
    };
    for (int r = warp; r < rows; r += 8) {
        const int c0 = count[r];
        if (c0 > kFewLong) {
            if (lane == 0) longs[atomicAdd(&many, 1)] = r;
            continue;
        }
        clear();
        if (c0) add_tokens(0, n, r);
        TT* dst = dt + ((size_t)r * blocks + b) * dim + col;
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
            if (col + c * 32 * VEC < dim) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[c][e] *= scale;
                store_vec_once<VEC>(dst + c * 32 * VEC, sum[c]);
            }
    }
    __syncthreads();
    const int long_rows = many;
    for (int k = 0; k < long_rows; ++k) {
        const int r = longs[k], per = (n + 7) / 8, from = warp * per;
        clear();
        add_tokens(from, from + per < n ? from + per : n, r);
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sums[warp][(c * 32 + lane) * VEC + e] = sum[c][e];
        __syncthreads();
        for (int i = tid; i < WIDTH; i += 256) {
            float t = sums[0][i];
#pragma unroll
            for (int w = 1; w < 8; ++w) t += sums[w][i];
            const int c = blockIdx.y * WIDTH + i;
            if (c < dim) store_one(dt + ((size_t)r * blocks + b) * dim + c, scale * t);
        }
        __syncthreads();
    }
}

// Launch shape of a backward call and its pieces of the workspace.
struct EmbedPlan {
    int bits, rows_per_block, blocks, vec, parts, group, slices, workers;
    size_t order_at, bound_at, carry_at, tail_at, cut_at, bytes;
};
static EmbedPlan plan_embed(const Embed* e, long tokens, bool aligned) {
    EmbedPlan pl;
    pl.bits = 7;     // 128 classes: a block on most of the SMs, and no division
    while (((e->vocab - 1) >> pl.bits) + 1 > kSortRows) ++pl.bits;
    pl.blocks = 1 << pl.bits;
    pl.rows_per_block = ((e->vocab - 1) >> pl.bits) + 1;
    // 16-byte accesses of the wider type: whole lines for a warp on both sides
    const int wide = e->y_dtype == CIRC_BF16 && e->table_dtype == CIRC_BF16 ? 8 : 4;
    pl.vec = aligned && e->dim % 8 == 0 ? wide : 1;
    const int vectors = (e->dim + pl.vec - 1) / pl.vec;
    pl.parts = vectors <= 32 ? 1 : pl.vec == 1 ? 4 : 2;      // single elements: more of them a thread
    const int threads = (vectors + pl.parts - 1) / pl.parts;
    pl.group = threads <= 32 ? 32 : threads <= 64 ? 64 : threads <= 128 ? 128 : 256;
    pl.slices = (threads + pl.group - 1) / pl.group;
    // stretches of equal traffic, two for each place on the machine: reads take longer than writes of the same size, and the second
    // round evens that out (one / two / four rounds: 160 / 144 / 138 us at 32768 tokens of 2048, 65536 rows); a few rows each at least
    long workers = 2 * 148L * kSumBlocks * 256 / pl.group / pl.slices;
    const long most = (tokens + (long)pl.blocks * pl.rows_per_block + 3) / 4;
    if (workers > most) workers = most;
    pl.workers = (int)(workers < 1 ? 1 : workers);
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    pl.order_at = up(sizeof(int) * ((size_t)pl.blocks * pl.rows_per_block + 1));
    pl.bound_at = pl.order_at + up(sizeof(int) * (size_t)(tokens ? tokens : 1));
    pl.carry_at = pl.bound_at + up(sizeof(Bound) * ((size_t)pl.workers + 1));
    pl.tail_at = pl.carry_at + up(sizeof(float) * (size_t)pl.workers * e->dim);
    pl.cut_at = pl.tail_at + up(sizeof(float) * (size_t)pl.workers * e->dim);
    pl.bytes = pl.cut_at + 256 + up(2 * sizeof(int4) * (size_t)pl.workers);
    return pl;
}
// The one-launch kernel's shape, where it serves a call.
struct FewPlan {
    bool fits;
    int vec, slices, blocks;
};
static FewPlan plan_few(const Embed* e, long tokens, bool aligned) {
    FewPlan f;
    f.vec = !aligned || e->dim % 8 ? 1 : e->y_dtype == CIRC_BF16 && e->table_dtype == CIRC_BF16 ? 8 : 4;
    const int width = 64 * f.vec;                           // columns of a block: 32 lanes, 2 vectors each
    f.slices = (e->dim + width - 1) / width;
    f.blocks = (148 * 8 + f.slices - 1) / f.slices;        // two rounds of blocks on the machine
    if (f.blocks > e->vocab) f.blocks = e->vocab;
    f.fits = tokens <= kFewTokens && f.slices <= 65535 && (e->vocab + f.blocks - 1) / f.blocks <= kFewRows;
    return f;
}
// What a call of up to this many tokens needs, whatever the alignment of its pointers.
static size_t embed_bytes(const Embed* e, long tokens) {
    if (plan_few(e, tokens, true).fits && plan_few(e, tokens, false).fits) return 0;
    const size_t a = plan_embed(e, tokens, true).bytes, b = plan_embed(e, tokens, false).bytes;
    return a > b ? a : b;
}

static int check_embed(const Embed* e, long tokens) {
    if (!e) {
        set_error(CIRC_ERR_ARG, "handle is NULL");
        return CIRC_ERR_ARG;
    }
    if (tokens < 0 || tokens > (1L << 30)) {
        set_error(CIRC_ERR_SHAPE, "tokens=%ld must be in [0, 2^30]", tokens);
        return CIRC_ERR_SHAPE;
    }
    return CIRC_OK;
}

}  // namespace circ

using namespace circ;

extern "C" {

circ_embed_handle circ_embed_create(int vocab, int dim) {
    if (vocab < 1 || vocab > (1 << 30) || dim < 1 || dim > (1 << 24)) {
        set_error(CIRC_ERR_SHAPE, "vocab=%d must be in [1, 2^30], dim=%d in [1, 2^24]", vocab, dim);
        return nullptr;
    }
    int device;
    if (!current_device(&device)) return nullptr;
    Embed* e = new (std::nothrow) Embed{device, vocab, dim, CIRC_F32, CIRC_F32, CIRC_I64, 1.f, -1, {}};
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
    const int rc = check_embed(e, max_tokens);
    return rc != CIRC_OK ? rc : ensure_scratch(e->ws, embed_bytes(e, max_tokens), 0, "circ_embed_reserve");
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
    if (tokens * ((e->dim + 2047) / 2048) > INT32_MAX) {      // thread blocks: of 1024 vectors of 8 elements, or of a row's 2048 elements
        set_error(CIRC_ERR_SHAPE, "tokens=%ld of %d elements are too many", tokens, e->dim);
        return CIRC_ERR_SHAPE;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool vec = e->dim % 8 == 0 && !misaligned(table, 16) && !misaligned(y, 16);
    cudaError_t err = cudaSuccess;
    with_dtype(e->table_dtype, [&](auto* t) {
        with_dtype(e->y_dtype, [&](auto* o) {
            with_index_type(e->ids_type, [&](auto* i) {
                using TT = tag_type<decltype(t)>;
                using TY = tag_type<decltype(o)>;
                using ID = tag_type<decltype(i)>;
                auto go = [&](auto kernel, int vec, int unroll) {
                    const int per_row = e->dim / vec;
                    const long vectors = tokens * per_row, blocks = (vectors + 256L * unroll - 1) / (256L * unroll);
                    err = launch_row(kernel, dim3((unsigned)blocks), dim3(256), 0, s, static_cast<const TT*>(table), static_cast<const ID*>(ids),
                                     static_cast<TY*>(y), (int)tokens, per_row, 256 / per_row, 256 % per_row, e->vocab, e->dim, e->scale,
                                     (unsigned)e->padding);
                };
                if (vec)
                    tokens * (e->dim / 8) <= 148L * 256 ? go(embed_forward_kernel<TT, TY, ID, 8, 1>, 8, 1)    // one vector a thread fills the machine
                                                        : go(embed_forward_kernel<TT, TY, ID, 8, 4>, 8, 4);
                else {
                    const int threads = e->dim >= 2048 ? 256 : (e->dim + 255) / 256 * 32;
                    const long chunks = (e->dim + 8L * threads - 1) / (8L * threads);
                    err = launch_row(embed_forward_any_kernel<TT, TY, ID>, dim3((unsigned)(tokens * chunks)), dim3(threads), 0, s,
                                     static_cast<const TT*>(table), static_cast<const ID*>(ids), static_cast<TY*>(y), (unsigned)chunks, e->vocab, e->dim,
                                     e->scale, (unsigned)e->padding);
                }
            });
        });
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(1);
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
    const bool aligned = !misaligned(grad_y, 16) && !misaligned(grad_table, 16);
    // Up to 2048 tokens in one launch, in microseconds against the three launches: 92 / 100 (65536 rows of 2048), 10 / 18 (1000 of 512),
    // 28 / 34 (131072 of 256); only with every token in one row the three are ahead (30 / 17 at 1000 of 512).
    const FewPlan few = plan_few(e, tokens, aligned);
    cudaError_t err = cudaSuccess;
    if (few.fits) {
        with_dtype(e->table_dtype, [&](auto* t) {
            with_dtype(e->y_dtype, [&](auto* o) {
                with_index_type(e->ids_type, [&](auto* i) {
                    using TT = tag_type<decltype(t)>;
                    using TY = tag_type<decltype(o)>;
                    using ID = tag_type<decltype(i)>;
                    constexpr int WIDE = std::is_same<TY, __nv_bfloat16>::value && std::is_same<TT, __nv_bfloat16>::value ? 8 : 4;
                    auto go = [&](auto kernel) {
                        err = launch_row(kernel, dim3((unsigned)few.blocks, few.slices), dim3(256), 0, s, static_cast<const ID*>(ids),
                                         static_cast<const TY*>(grad_y), static_cast<TT*>(grad_table), (int)tokens, e->vocab, (unsigned)e->padding,
                                         e->dim, e->scale);
                    };
                    few.vec == 1 ? go(embed_few_kernel<TT, TY, ID, 1>) : go(embed_few_kernel<TT, TY, ID, WIDE>);
                });
            });
        });
        CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
        count_launches(1);
        return CIRC_OK;
    }
    if ((rc = ensure_scratch(e->ws, embed_bytes(e, tokens), s, "circ_embed_reserve")) != CIRC_OK) return rc;
    const EmbedPlan pl = plan_embed(e, tokens, aligned);
    char* ws = static_cast<char*>(e->ws.ptr);
    const EmbedSum a{reinterpret_cast<int*>(ws), reinterpret_cast<int*>(ws + pl.order_at), reinterpret_cast<Bound*>(ws + pl.bound_at),
                     reinterpret_cast<long*>(ws + pl.cut_at + 16), reinterpret_cast<float*>(ws + pl.carry_at), reinterpret_cast<float*>(ws + pl.tail_at),
                     reinterpret_cast<int*>(ws + pl.cut_at), reinterpret_cast<int4*>(ws + pl.cut_at + 256), e->vocab, e->dim, pl.workers, pl.bits,
                     pl.rows_per_block, pl.blocks * pl.rows_per_block, (int)dtype_bytes(e->y_dtype), (int)dtype_bytes(e->table_dtype), e->scale};
    const int per_warp = (int)((tokens + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    int room = (int)((kSortShared - sizeof(int) * kSortWarps * pl.rows_per_block) / (sizeof(int2) * kSortWarps));
    if (room > per_warp) room = per_warp;
    const size_t smem = kSortWarps * (sizeof(int) * (size_t)pl.rows_per_block + sizeof(int2) * room);
    with_index_type(e->ids_type, [&](auto* i) {
        using ID = tag_type<decltype(i)>;
        err = cudaFuncSetAttribute(embed_sort_kernel<ID>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSortShared);
        if (err != cudaSuccess) return;
        err = launch_row(embed_sort_kernel<ID>, dim3(pl.blocks), dim3(kSortThreads), smem, s, static_cast<const ID*>(ids), (int)tokens,
                         (unsigned)e->padding, room, a);
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    with_dtype(e->table_dtype, [&](auto* t) {
        using TT = tag_type<decltype(t)>;
        with_dtype(e->y_dtype, [&](auto* o) {
            using TY = tag_type<decltype(o)>;
            constexpr int WIDE = std::is_same<TY, __nv_bfloat16>::value && std::is_same<TT, __nv_bfloat16>::value ? 8 : 4;
            auto go = [&](auto kernel) {
                const int per_block = 256 / pl.group, bytes = pl.parts * pl.vec * (int)sizeof(TY);
                const size_t ring = (size_t)ring_depth(bytes) * bytes * 256;
                err = launch_row(kernel, dim3((pl.workers + per_block - 1) / per_block, pl.slices), dim3(256), ring, s, a,
                                    static_cast<const TY*>(grad_y), static_cast<TT*>(grad_table));
            };
            auto by_group = [&](auto vec, auto parts) {
                constexpr int V = decltype(vec)::value, P = decltype(parts)::value;
                pl.group == 32 ? go(embed_sum_kernel<TT, TY, V, P, 32>) : pl.group == 64 ? go(embed_sum_kernel<TT, TY, V, P, 64>)
                    : pl.group == 128 ? go(embed_sum_kernel<TT, TY, V, P, 128>) : go(embed_sum_kernel<TT, TY, V, P, 256>);
            };
            using One = std::integral_constant<int, 1>;
            using Two = std::integral_constant<int, 2>;
            using Four = std::integral_constant<int, 4>;
            using Wide = std::integral_constant<int, WIDE>;
            if (pl.parts == 1)     // at most 32 vectors a row
                pl.vec == 1 ? go(embed_sum_kernel<TT, TY, 1, 1, 32>) : go(embed_sum_kernel<TT, TY, WIDE, 1, 32>);
            else
                pl.vec == 1 ? by_group(One{}, Four{}) : by_group(Wide{}, Two{});
        });
        if (err == cudaSuccess && tokens > kWholeRun)
            err = launch_row(embed_join_kernel<TT>, dim3(148 * 4), dim3(256), 0, s, a, static_cast<TT*>(grad_table));
    });
    CIRC_CUDA_TRY(err, CIRC_ERR_CUDA);
    count_launches(2 + (tokens > kWholeRun));
    CIRC_CUDA_TRY(cudaGetLastError(), CIRC_ERR_CUDA);
    return CIRC_OK;
}

}  // extern "C"
