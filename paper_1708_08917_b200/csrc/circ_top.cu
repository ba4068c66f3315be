// The `count` largest of a row's scores in descending order, equal ones by their class, and log sum exp(z / tau) over the whole row.
#include <float.h>

#include <algorithm>
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
    int pieces, per;     // pieces of a row, and vectors a piece
    // workspace
    unsigned* arrived;   // [rows] pieces that are done (0 before and after a call)
    int* overflow;       // [rows] a piece has more ties than its lists hold (0 before and after a call)
    Softmax* parts;      // [rows][pieces]
    uint64_t* keys;      // [rows][pieces][count]
};

// Whole numbers in the order of the scores; the zeros are equal, and a NaN is above all.  Of a bfloat16 the lower half is 0.  No score has 0.
__device__ __forceinline__ uint32_t order_of(float score) {
    const float z = score + 0.f;
    const uint32_t b = __float_as_uint(z);
    return z != z ? 0xffffffffu : b >> 31 ? ~b : b | 0x80000000u;
}
template <typename T>
__device__ __forceinline__ uint32_t order_in(float score) {
    return sizeof(T) == 4 ? order_of(score) : order_of(score) & 0xffff0000u;
}
__device__ __forceinline__ float score_of(uint32_t order) { return __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order); }

// The threads that work on a row together: a warp, the block, or some warps of it with a barrier of their own.
template <int THREADS, int BARRIER>       // BARRIER 0: the block's; above: a named one
struct Team {
    static constexpr int WARPS = THREADS / 32;
    uint2 (*red)[WARPS];                  // [2][WARPS] in shared memory
    int flip = 0;
    int rank;                             // of the thread
    __device__ __forceinline__ void sync() const {
        if constexpr (WARPS == 1) __syncwarp();
        else if constexpr (BARRIER == 0) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"n"(BARRIER), "n"(THREADS) : "memory");
    }
    // Over all threads: the sum of a word, the least and the largest.
    __device__ __forceinline__ unsigned sum(unsigned x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if constexpr (WARPS > 1) {
            share(make_uint2(x, 0));
            x = __reduce_add_sync(0xffffffffu, rank % 32 < WARPS ? red[flip][rank % 32].x : 0u);
            flip ^= 1;
        }
        return x;
    }
    __device__ __forceinline__ uint2 range(unsigned x) {
        uint2 v = make_uint2(__reduce_min_sync(0xffffffffu, x), __reduce_max_sync(0xffffffffu, x));
        if constexpr (WARPS > 1) {
            share(v);
            v = rank % 32 < WARPS ? red[flip][rank % 32] : make_uint2(0xffffffffu, 0);
            v = make_uint2(__reduce_min_sync(0xffffffffu, v.x), __reduce_max_sync(0xffffffffu, v.y));
            flip ^= 1;
        }
        return v;
    }
    __device__ __forceinline__ void share(uint2 v) const {
        if (rank % 32 == 0) red[flip][rank / 32] = v;
        sync();
    }
    // Where this thread's `n` entries of a list begin; `length`: the list's, in shared memory.
    __device__ __forceinline__ unsigned append(unsigned n, unsigned* length) const {
        unsigned before = n;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const unsigned v = __shfl_up_sync(0xffffffffu, before, o);
            if (rank % 32 >= o) before += v;
        }
        unsigned base = 0;
        if (rank % 32 == 31 && before) base = atomicAdd(length, before);
        return __shfl_sync(0xffffffffu, base, 31) + before - n;
    }
};

// The largest bound that at least `want` orders reach (of which there are that many), or a lower one that no more than `enough` do; `reach`: how many
// do.  Halves the scores' range, and where that does not get on (infinities, values far apart) the orders' range.
template <typename T, int N, typename TEAM>
__device__ __forceinline__ uint32_t find_bound(TEAM& team, const uint32_t (&order)[N], unsigned want, unsigned enough, unsigned& reach) {
    constexpr uint32_t UNIT = sizeof(T) == 4 ? 1u : 0x10000u;
    auto reaching = [&](uint32_t bound) {
        unsigned n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += order[i] >= bound;
        return team.sum(n);
    };
    uint32_t mine = order[0];
#pragma unroll
    for (int i = 1; i < N; ++i) mine = max(mine, order[i]);
    const uint2 ends = team.range(mine);
    uint32_t low = UNIT, high = ends.y;
    if ((int)want <= TEAM::WARPS * 32) low = max(low, ends.x);       // every thread has one that reaches it
    reach = ~0u;
    bool looked = false;        // at `high` itself
    for (int step = 0; high - low > UNIT; ++step) {
        uint32_t middle = low + (high - low) / 2;
        const float m = 0.5f * score_of(low) + 0.5f * score_of(high);
        if (step < 12 && fabsf(m) < INFINITY) middle = order_of(m);      // NaN: no
        if (UNIT > 1) middle &= 0xffff0000u;
        middle = min(max(middle, low + UNIT), high - UNIT);
        const unsigned n = reaching(middle);
        if (n >= want) {
            low = middle;
            reach = n;
            if (n <= enough) return low;
        } else {
            high = middle;
            looked = true;
        }
    }
    if (!looked) {              // the largest order, which want of them may have
        const unsigned n = reaching(high);
        if (n >= want) {
            reach = n;
            return high;
        }
    }
    if (reach == ~0u) reach = reaching(low);
    return low;
}
// A bound that at least `want` of a block's N THREADS groups reach, from the largest order of each: found by its first warp from `most`, a word of shared
// memory for each.  The same in every thread.
template <typename T, int THREADS, int N>
__device__ __forceinline__ uint32_t block_bound(const uint32_t* most, unsigned want, uint32_t* bound) {
    __syncthreads();
    if (threadIdx.x < 32) {
        Team<32, 0> team{nullptr, 0, (int)threadIdx.x};
        uint32_t order[N * THREADS / 32];
#pragma unroll
        for (int i = 0; i < N * THREADS / 32; ++i) order[i] = most[i * 32 + threadIdx.x];
        unsigned reach;
        const uint32_t found = find_bound<T>(team, order, want, want + want / 4 + 4, reach);
        if (threadIdx.x == 0) *bound = found;
    }
    __syncthreads();
    return *bound;
}

// What may belong to a row's top, in any order: the order of the score, then the complement of the class.
__device__ __forceinline__ uint64_t key_of(uint32_t order, int id) { return (uint64_t)order << 32 | (uint32_t)~id; }

// Hands the first `count` of `found` keys to out(place, key); `keys` has room for a multiple of 32.  A warp sorts 32 of them in its registers; a key's
// place is the number of those above it, from a binary search in each of the other sorted runs.  (Counting by comparison with every key took
// 300 of them 13000 to 19000 cycles.)
template <typename TEAM, typename OUT>
__device__ __forceinline__ void put_in_order(const TEAM& team, uint64_t* keys, int found, int count, OUT out) {
    const int lane = team.rank % 32, warp = team.rank / 32, runs = (found + 31) / 32;
    for (int r = warp; r < runs; r += TEAM::WARPS) {
        uint64_t key = r * 32 + lane < found ? keys[r * 32 + lane] : 0;
#pragma unroll
        for (int k = 2; k <= 32; k *= 2)
#pragma unroll
            for (int j = k / 2; j > 0; j /= 2) {
                const uint64_t other = __shfl_xor_sync(0xffffffffu, key, j);
                const bool larger = ((lane & j) == 0) == ((lane & k) == 0 || k == 32);      // this lane keeps the larger one
                key = (other > key) == larger ? other : key;
            }
        if (runs == 1 && lane < count) out(lane, key);
        keys[r * 32 + lane] = key;
    }
    if (runs == 1) return;
    team.sync();
    for (int r = warp; r < runs; r += TEAM::WARPS) {
        const uint64_t mine = keys[r * 32 + lane];
        int place = lane;
        for (int o = 0; o < runs; ++o) {
            if (o == r) continue;
            const uint64_t* run = keys + o * 32;
            int above = 0;
#pragma unroll
            for (int b = 16; b > 0; b /= 2) above += run[above + b - 1] > mine ? b : 0;
            above += run[above] > mine;
            place += above;
        }
        if (mine != 0 && place < count) out(place, mine);
    }
}
template <typename T, typename ID>
__device__ __forceinline__ void write_one(const TopArgs& a, size_t row, int place, uint64_t key) {
    const size_t at = row * a.count + place;
    if (a.values) {
        const uint32_t bits = __float_as_uint(score_of((uint32_t)(key >> 32)));      // of a bfloat16 below zero the lower half is all ones
        store_one(static_cast<T*>(a.values) + at, __uint_as_float(sizeof(T) == 4 ? bits : bits & 0xffff0000u));
    }
    if (a.ids) static_cast<ID*>(a.ids)[at] = (ID)(int)~(uint32_t)key;
}
__device__ __forceinline__ void write_lse(const TopArgs& a, size_t row, Softmax all) {
    const double base = all.top == -INFINITY ? 0.0 : (double)all.top;
    a.lse[row] = (float)(base * a.inv_tau + log((double)all.sum));
}

// Any row, by a team: the order of its count-th score by digits of 8 bits from the top, then those above it, and of those equal to it the first.
template <int WARPS>
struct AnySpace {
    unsigned digits[256];
    unsigned prefix, left, taken, warps[WARPS];
};
template <typename T, typename ID, typename TEAM>
__device__ __forceinline__ void select_any(const TopArgs& a, const T* __restrict__ zr, size_t row, uint64_t* keys, AnySpace<TEAM::WARPS>& space, TEAM& team) {
    constexpr int THREADS = TEAM::WARPS * 32;
    const int rank = team.rank, warp = rank / 32, lane = rank % 32;
    team.sync();
    if (rank == 0) {
        space.prefix = 0;
        space.left = a.count;
        space.taken = 0;
    }
    for (int shift = 24; shift >= 32 - 8 * (int)sizeof(T); shift -= 8) {
        for (int i = rank; i < 256; i += THREADS) space.digits[i] = 0;
        team.sync();
        const uint32_t known = shift == 24 ? 0u : ~0u << (shift + 8), want = space.prefix;
        for (int c = rank; c < a.classes; c += THREADS) {
            const uint32_t o = order_in<T>(to_float(zr[c]));
            if ((o & known) == want) atomicAdd(space.digits + (o >> shift & 255), 1u);
        }
        team.sync();
        if (rank == 0) {
            unsigned rest = space.left;
            int d = 255;
            while (d > 0 && space.digits[d] < rest) rest -= space.digits[d--];
            space.left = rest;
            space.prefix = want | (uint32_t)d << shift;
        }
        team.sync();
    }
    const uint32_t last = space.prefix;
    int have = a.count - (int)space.left;
    for (int c = rank; c < a.classes; c += THREADS) {
        const uint32_t o = order_in<T>(to_float(zr[c]));
        if (o > last) keys[atomicAdd(&space.taken, 1u)] = key_of(o, c);
    }
    for (int c0 = 0; c0 < a.classes && have < a.count; c0 += THREADS) {
        const int c = c0 + rank;
        const bool equal = c < a.classes && order_in<T>(to_float(zr[c])) == last;
        const unsigned lanes = __ballot_sync(0xffffffffu, equal);
        if (lane == 0) space.warps[warp] = __popc(lanes);
        team.sync();
        int before = 0, all = 0;
        for (int w = 0; w < TEAM::WARPS; ++w) {
            before += w < warp ? (int)space.warps[w] : 0;
            all += (int)space.warps[w];
        }
        const int at = have + before + __popc(lanes & ((1u << lane) - 1));
        if (equal && at < a.count) keys[at] = key_of(last, c);
        have += all;
        team.sync();
    }
    team.sync();
    put_in_order(team, keys, a.count, a.count, [&](int place, uint64_t key) { write_one<T, ID>(a, row, place, key); });
}

constexpr int kAnyThreads = 512;
// Tensors that are not aligned.
template <typename T, typename ID>
__global__ void __launch_bounds__(kAnyThreads) top_any_kernel(const T* __restrict__ z, TopArgs a) {
    __shared__ uint64_t keys[kTopMost];
    __shared__ AnySpace<kAnyThreads / 32> space;
    __shared__ uint2 red[2][kAnyThreads / 32];
    __shared__ Softmax part[kAnyThreads / 32];
    pdl_begin();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    Team<kAnyThreads, 0> team{red, 0, tid};
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* zr = z + (size_t)row * a.ld;
        if (a.lse) {
            Running run(a.scale, FLT_MAX);
            for (int c0 = tid; c0 < a.classes; c0 += kAnyThreads * 8) {
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = c0 + e * kAnyThreads < a.classes ? to_float(zr[c0 + e * kAnyThreads]) : -INFINITY;
                run.take(s);
            }
            Softmax all = warp_join(run.done(), a.scale);
            __syncthreads();
            if (lane == 0) part[warp] = all;
            __syncthreads();
            if (warp == 0) {
                all = warp_join(lane < kAnyThreads / 32 ? part[lane] : Softmax{-INFINITY, 0.f}, a.scale);
                if (lane == 0) write_lse(a, (size_t)row, all);
            }
        }
        if (a.values || a.ids) select_any<T, ID>(a, zr, (size_t)row, keys, space, team);
    }
}

// The top of orders that a team holds, N a thread, into `keys` (in any order, `taken` of them): those that reach a bound that at least `want` do, and few
// more.  Of more than kHeldKeys, which are ties at the want-th score, the lowest classes.  id(i): the class of the thread's i-th.
constexpr int kHeldKeys = 512;
template <int N, typename TEAM, typename FID>
__device__ __forceinline__ bool collect_from(TEAM& team, const uint32_t (&order)[N], uint32_t bound, int cut, uint64_t* keys, unsigned* taken, FID id) {
    if (team.rank == 0) *taken = 0;
    team.sync();
    unsigned mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) mine += order[i] > bound || (order[i] == bound && (cut == 0x7fffffff || id(i) <= cut));
    unsigned at = team.append(mine, taken);
    if (mine)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (order[i] > bound || (order[i] == bound && (cut == 0x7fffffff || id(i) <= cut))) {
                if (at < kHeldKeys) keys[at] = key_of(order[i], id(i));
                ++at;
            }
    team.sync();
    return *taken <= kHeldKeys;
}
template <typename T, int N, typename TEAM, typename FID>
__device__ __forceinline__ void collect(TEAM& team, const uint32_t (&order)[N], unsigned want, uint64_t* keys, unsigned* taken, int classes, FID id) {
    unsigned reach, enough = 64;
    while (enough < want) enough *= 2;
    if (TEAM::WARPS > 1) enough = min((unsigned)kHeldKeys, want + want / 4 + 16);
    const uint32_t bound = find_bound<T>(team, order, want, enough, reach);
    int cut = 0x7fffffff;                          // classes up to it, of those at the bound
    if (reach > kHeldKeys) {
        unsigned above = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) above += order[i] > bound;
        above = team.sum(above);
        int low = -1, high = classes - 1;          // classes up to `high` are enough
        while (high - low > 1) {
            const int middle = low + (high - low) / 2;
            unsigned n = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) n += order[i] == bound && id(i) <= middle;
            if (above + team.sum(n) >= want) high = middle;
            else low = middle;
        }
        cut = high;
    }
    collect_from(team, order, bound, cut, keys, taken, id);
}

// ---- short rows: a team holds one in registers ----
// In a block the bound comes from the largest of each thread's first, second, third and fourth quarter, found by one warp, if that is a good one
// (kGroups THREADS groups, twice as many as scores are wanted); in a warp from the scores themselves.
constexpr int kGroups = 4;
template <typename T, typename ID, int THREADS, int N>      // N vectors a thread
__global__ void __launch_bounds__(THREADS < 128 ? 128 : THREADS) top_held_kernel(const T* __restrict__ z, TopArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), ROWS = THREADS < 128 ? 128 / THREADS : 1, WARPS = THREADS / 32;
    __shared__ uint64_t keys_of[ROWS][kHeldKeys];
    __shared__ unsigned taken_of[ROWS];
    __shared__ uint2 red[2][WARPS];
    __shared__ Softmax part[WARPS];
    __shared__ uint32_t most[WARPS > 1 ? kGroups * THREADS : 1], shared_bound;
    pdl_begin();
    const int rank = threadIdx.x % THREADS, team_of = threadIdx.x / THREADS, lane = rank % 32, row = blockIdx.x * ROWS + team_of;
    if (row >= a.rows) return;      // a whole team
    Team<THREADS, 0> team{red, 0, rank};
    const RowSpan<VEC, false> span(row, a.classes, a.ld);
    uint32_t order[N * VEC];
    {
        RawVec<T, VEC> raw[N];
        Running run(a.scale, FLT_MAX);
#pragma unroll
        for (int i = 0; i < N; ++i) span.load(raw[i], z, i * THREADS + rank);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int v = i * THREADS + rank;
            float s[VEC];
            scores(span, v, raw[i], s);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int c = span.col(v) + e;
                order[i * VEC + e] = c >= 0 && c < a.classes ? order_in<T>(s[e]) : 0u;
            }
            if (a.lse) run.take(s);
        }
        if (a.lse) {
            Softmax all = warp_join(run.done(), a.scale);
            if constexpr (WARPS > 1) {
                if (lane == 0) part[rank / 32] = all;
                __syncthreads();
                if (rank < 32) all = warp_join(lane < WARPS ? part[lane] : Softmax{-INFINITY, 0.f}, a.scale);
            }
            if (rank == 0) write_lse(a, (size_t)row, all);
        }
    }
    if (!a.values && !a.ids) return;
    auto id = [&](int i) { return span.col(i / VEC * THREADS + rank) + i % VEC; };
    bool done = false;
    if constexpr (WARPS > 1) {
        constexpr int EACH = N * VEC / kGroups;
        // groups without a score have the order 0, which a bound does not count: at least half of the groups have one
        if (2 * a.count <= kGroups * THREADS / 2) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < EACH; ++i) m = max(m, order[g * EACH + i]);
                most[g * THREADS + rank] = m;
            }
            const uint32_t bound = block_bound<T, THREADS, kGroups>(most, (unsigned)a.count, &shared_bound);
            done = collect_from(team, order, bound, 0x7fffffff, keys_of[team_of], &taken_of[team_of], id);
        }
    }
    if (!done) collect<T>(team, order, (unsigned)a.count, keys_of[team_of], &taken_of[team_of], a.classes, id);
    put_in_order(team, keys_of[team_of], (int)taken_of[team_of], a.count, [&](int place, uint64_t key) { write_one<T, ID>(a, (size_t)row, place, key); });
}

// ---- long rows: a block a row, or a piece of one, read once ----
// A thread keeps the largest scores of the first, second, third and fourth vectors that it takes at a time: at least `count` scores reach a bound that
// `count` threads' largest do.  One warp finds that bound (halving it by the whole block took 2.5 times the instructions of the reading).  Only the
// vectors behind a maximum that reaches it are read again (from L2), and the few scores that do are put in order.  A row with more of them than the
// lists hold (ties) goes through select_any.
// Bound by memory where few scores are wanted (8192 x 50000 bfloat16, top 8 and the sum: 149 us, 5.5 TB/s); with 64 of them (219 us) by the waits between
// reading, finding the bound, reading again and sorting, which more and smaller blocks hide only in part.
// Pieces leave their top and their sum in the workspace, and the block that is last to finish a row's takes the top of those.
constexpr int kKept = 4;
constexpr int kHits = 512, kRowKeys = 1024;
constexpr int kRowThreads = 1280;   // resident on an SM
constexpr int kMergeEach = 16;     // keys that a thread takes when a row's pieces are put together

// The largest of some vectors, NaN if one is.
template <int VEC, int N>
__device__ __forceinline__ float most_nan(const RawVec<float, VEC> (&raw)[N]) {
    float most = raw[0].get(0);
#pragma unroll
    for (int i = 1; i < N * VEC; ++i) most = max_nan(most, raw[i / VEC].get(i % VEC));
    return most;
}
template <int VEC, int N>
__device__ __forceinline__ float most_nan(const RawVec<__nv_bfloat16, VEC> (&raw)[N]) {
    constexpr int W = VEC / 2;
    __nv_bfloat162 most = *reinterpret_cast<const __nv_bfloat162*>(&raw[0].w[0]);
#pragma unroll
    for (int i = 1; i < N * W; ++i) most = __hmax2_nan(most, *reinterpret_cast<const __nv_bfloat162*>(&raw[i / W].w[i % W]));
    return max_nan(__low2float(most), __high2float(most));
}

template <typename T, int VEC>
__device__ __forceinline__ float most_nan(const RawVec<T, VEC>& one) {
    return most_nan(reinterpret_cast<const RawVec<T, VEC>(&)[1]>(one));
}

template <typename T, typename ID, int THREADS, bool PIECES>
__global__ void __launch_bounds__(THREADS, PIECES ? 1 : kRowThreads / THREADS) top_rows_kernel(const T* __restrict__ z, TopArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), WARPS = THREADS / 32;
    __shared__ uint64_t keys[kRowKeys];
    __shared__ uint16_t hits[kHits];
    __shared__ unsigned hit, taken;
    __shared__ uint32_t most_of_thread[THREADS], shared_bound;
    __shared__ uint2 red[2][WARPS];
    __shared__ Softmax part[WARPS];
    __shared__ AnySpace<WARPS> any;
    __shared__ bool last;
    pdl_begin();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const bool wanted = a.values || a.ids;
    Team<THREADS, 0> team{red, 0, tid};
    const int row = PIECES ? blockIdx.x / a.pieces : blockIdx.x;
    const RowSpan<VEC, false> span(row, a.classes, a.ld);
    const int vectors = (a.classes - span.shift + VEC - 1) / VEC, piece = PIECES ? blockIdx.x % a.pieces : 0;
    const int v0 = piece * a.per, v1 = PIECES ? min(vectors, v0 + a.per) : vectors;
    const int w0 = span.whole(v0) ? v0 : v0 + 1, w1 = span.whole(v1 - 1) ? v1 : v1 - 1, whole = w1 - w0;
    const T* src = z + span.at(w0) + (size_t)tid * VEC;
    float best[kKept];
#pragma unroll
    for (int u = 0; u < kKept; ++u) best[u] = -INFINITY;
    Running run(a.scale, FLT_MAX);
    for (int i = tid; i < whole; i += kKept * THREADS) {
        const T* from = src + (size_t)(i - tid) * VEC;
        RawVec<T, VEC> raw[kKept];
        if (i + (kKept - 1) * THREADS < whole) {
#pragma unroll
            for (int u = 0; u < kKept; ++u) raw[u].load(from + u * THREADS * VEC);
        } else {
#pragma unroll
            for (int u = 0; u < kKept; ++u) {
                raw[u].fill_lowest();
                if (i + u * THREADS < whole) raw[u].load(from + u * THREADS * VEC);
            }
        }
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < kKept; ++u) {
            const float one = most_nan(raw[u]);
            best[u] = max_nan(best[u], one);
            most = max_nan(most, one);
        }
        if (a.lse) {
            run.rise(most);
            if (run.ex.plain) run.template add<true>(raw);
            else run.template add<false>(raw);
        }
    }
    // the first and last elements beside the whole vectors
    const int rest = tid == 0 && w0 > v0 ? v0 : tid == 1 && w1 < v1 && (w1 > v0 || w0 == v0) ? v1 - 1 : -1;
    float edge[VEC];
    if (rest >= 0) {
        RawVec<T, VEC> raw;
        span.load(raw, z, rest);
        scores(span, rest, raw, edge);
        if (a.lse) run.take(edge);
    }
    if (tid == 0) hit = taken = 0;
    if (a.lse) {
        Softmax all = warp_join(run.done(), a.scale);
        if (lane == 0) part[warp] = all;
        __syncthreads();
        if (warp == 0) {
            all = warp_join(lane < WARPS ? part[lane] : Softmax{-INFINITY, 0.f}, a.scale);
            if (lane == 0) {
                if (PIECES) a.parts[(size_t)row * a.pieces + piece] = all;
                else write_lse(a, (size_t)row, all);
            }
        }
    }
    if (wanted) {
        uint32_t order[kKept], most = 0;
#pragma unroll
        for (int u = 0; u < kKept; ++u) {
            order[u] = tid + u * THREADS < whole ? order_in<T>(best[u]) : 0u;
            most = max(most, order[u]);
        }
        most_of_thread[tid] = most;
        const uint32_t bound = block_bound<T, THREADS, 1>(most_of_thread, (unsigned)a.count, &shared_bound);
        unsigned mine = 0;
#pragma unroll
        for (int u = 0; u < kKept; ++u) mine += order[u] >= bound;
        unsigned at = team.append(mine, &hit);
#pragma unroll
        for (int u = 0; u < kKept; ++u)
            if (order[u] >= bound) {
                if (at < kHits) hits[at] = (uint16_t)(u * THREADS + tid);
                ++at;
            }
        __syncthreads();
        bool listed = hit <= kHits;
        if (listed) {
            const int each = (whole + kKept * THREADS - 1) / (kKept * THREADS), items = (int)hit * each;       // vectors behind a hit
            for (int i0 = 0; i0 < items; i0 += THREADS) {
                const int i = i0 + tid;
                float s[VEC];
                int c0 = 0;
                unsigned above = 0;
                if (i < items) {
                    const int h = hits[i / each], v = (i % each * kKept + h / THREADS) * THREADS + h % THREADS;
                    if (v < whole) {
                        RawVec<T, VEC> raw;
                        raw.load(z + span.at(w0 + v));
                        c0 = span.col(w0 + v);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            s[e] = raw.get(e);
                            above |= (unsigned)(order_in<T>(s[e]) >= bound) << e;
                        }
                    }
                }
                unsigned at = team.append(__popc(above), &taken);
                if (above)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (above >> e & 1) {
                            if (at < kRowKeys) keys[at] = key_of(order_in<T>(s[e]), c0 + e);
                            ++at;
                        }
            }
            if (rest >= 0)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int c = span.col(rest) + e;
                    if (c < 0 || c >= a.classes || order_in<T>(edge[e]) < bound) continue;
                    const unsigned at = atomicAdd(&taken, 1u);
                    if (at < kRowKeys) keys[at] = key_of(order_in<T>(edge[e]), c);
                }
            __syncthreads();
            listed = taken <= kRowKeys;
        }
        if (PIECES && !listed) a.overflow[row] = 1;
        if (PIECES) {
            uint64_t* out = a.keys + ((size_t)row * a.pieces + piece) * a.count;
            if (listed) put_in_order(team, keys, (int)taken, a.count, [&](int place, uint64_t key) { out[place] = key; });
        } else if (listed) {
            put_in_order(team, keys, (int)taken, a.count, [&](int place, uint64_t key) { write_one<T, ID>(a, (size_t)row, place, key); });
        } else {
            select_any<T, ID>(a, z + (size_t)row * a.ld, (size_t)row, keys, any, team);
        }
    }
    __syncthreads();
    if (!PIECES) return;
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(a.arrived + row, 1u) == (unsigned)a.pieces - 1;
        if (last) a.arrived[row] = 0;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (a.lse && warp == 0) {
        Softmax all{-INFINITY, 0.f};
        for (int i = lane; i < a.pieces; i += 32) {
            const float2 p = __ldcg(reinterpret_cast<const float2*>(a.parts) + (size_t)row * a.pieces + i);
            all = join(all, Softmax{p.x, p.y}, a.scale);
        }
        all = warp_join(all, a.scale);
        if (lane == 0) write_lse(a, (size_t)row, all);
    }
    if (!wanted) return;
    const bool over = __ldcg(a.overflow + row) != 0;
    __syncthreads();
    if (over) {
        if (tid == 0) a.overflow[row] = 0;
        select_any<T, ID>(a, z + (size_t)row * a.ld, (size_t)row, keys, any, team);
        return;
    }
    const unsigned long long* in = reinterpret_cast<const unsigned long long*>(a.keys) + (size_t)row * a.pieces * a.count;
    const int total = a.pieces * a.count;
    uint32_t merged[kMergeEach];
#pragma unroll
    for (int i = 0; i < kMergeEach; ++i) merged[i] = i * THREADS + tid < total ? (uint32_t)(__ldcg(in + i * THREADS + tid) >> 32) : 0u;
    collect<T>(team, merged, (unsigned)a.count, keys, &taken, a.classes,
               [&](int i) { return i * THREADS + tid < total ? (int)~(uint32_t)__ldcg(in + i * THREADS + tid) : 0x7fffffff; });
    put_in_order(team, keys, (int)taken, a.count, [&](int place, uint64_t key) { write_one<T, ID>(a, (size_t)row, place, key); });
    return;
}

// ---- many rows of middling length: the same by a warp, without a barrier ----
// 256 maxima a row: eight a lane, of the four vectors that it takes at a time in even turns and in odd ones.
constexpr int kWarpKeys = 256;
template <typename T, typename ID>
__global__ void __launch_bounds__(128, 10) top_warp_kernel(const T* __restrict__ z, TopArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T);
    __shared__ uint64_t keys_of[4][kWarpKeys];
    __shared__ uint16_t hits_of[4][2 * kKept * 32];
    __shared__ unsigned lengths[4][2];
    __shared__ AnySpace<1> any[4];
    pdl_begin();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, row = blockIdx.x * 4 + warp;
    if (row >= a.rows) return;
    Team<32, 0> team{nullptr, 0, lane};
    uint64_t* keys = keys_of[warp];
    uint16_t* hits = hits_of[warp];
    unsigned *hit = &lengths[warp][0], *taken = &lengths[warp][1];
    const RowSpan<VEC, false> span(row, a.classes, a.ld);
    const int vectors = (a.classes - span.shift + VEC - 1) / VEC, w0 = span.whole(0) ? 0 : 1, w1 = span.whole(vectors - 1) ? vectors : vectors - 1, whole = w1 - w0;
    const T* src = z + span.at(w0) + (size_t)lane * VEC;
    float best[2][kKept];
#pragma unroll
    for (int u = 0; u < 2 * kKept; ++u) best[u / kKept][u % kKept] = -INFINITY;
    Running run(a.scale, FLT_MAX);
    for (int i = 0; i < whole; i += 2 * kKept * 32)
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const int at = i + odd * kKept * 32;
            if (at >= whole) break;
            RawVec<T, VEC> raw[kKept];
#pragma unroll
            for (int u = 0; u < kKept; ++u) {
                raw[u].fill_lowest();
                if (at + u * 32 + lane < whole) raw[u].load(src + (size_t)(at + u * 32) * VEC);
            }
            float most = -INFINITY;
#pragma unroll
            for (int u = 0; u < kKept; ++u) {
                const float one = most_nan(raw[u]);
                best[odd][u] = max_nan(best[odd][u], one);
                most = max_nan(most, one);
            }
            if (a.lse) {
                run.rise(most);
                if (run.ex.plain) run.template add<true>(raw);
                else run.template add<false>(raw);
            }
        }
    const int rest = lane == 0 && w0 == 1 ? 0 : lane == 1 && w1 < vectors && (w1 > 0 || w0 == 0) ? vectors - 1 : -1;
    float edge[VEC];
    if (rest >= 0) {
        RawVec<T, VEC> raw;
        span.load(raw, z, rest);
        scores(span, rest, raw, edge);
        if (a.lse) run.take(edge);
    }
    if (a.lse) {
        const Softmax all = warp_join(run.done(), a.scale);
        if (lane == 0) write_lse(a, (size_t)row, all);
    }
    if (!a.values && !a.ids) return;
    uint32_t order[2 * kKept];
#pragma unroll
    for (int u = 0; u < 2 * kKept; ++u) order[u] = lane + u * 32 < whole ? order_in<T>(best[u / kKept][u % kKept]) : 0u;
    unsigned reach;
    const uint32_t bound = find_bound<T>(team, order, (unsigned)a.count, (unsigned)(a.count + a.count / 4 + 4), reach);
    if (lane == 0) *hit = *taken = 0;
    __syncwarp();
    unsigned mine = 0;
#pragma unroll
    for (int u = 0; u < 2 * kKept; ++u) mine += order[u] >= bound;
    unsigned at = team.append(mine, hit);
#pragma unroll
    for (int u = 0; u < 2 * kKept; ++u)
        if (order[u] >= bound) hits[at++] = (uint16_t)(u * 32 + lane);
    __syncwarp();
    const int each = (whole + 2 * kKept * 32 - 1) / (2 * kKept * 32), items = (int)*hit * each;
    for (int i0 = 0; i0 < items; i0 += 32) {
        const int i = i0 + lane;
        float s[VEC];
        int c0 = 0;
        unsigned above = 0;
        if (i < items) {
            const int v = i % each * (2 * kKept * 32) + hits[i / each];
            if (v < whole) {
                RawVec<T, VEC> raw;
                raw.load(z + span.at(w0 + v));
                c0 = span.col(w0 + v);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    s[e] = raw.get(e);
                    above |= (unsigned)(order_in<T>(s[e]) >= bound) << e;
                }
            }
        }
        unsigned to = team.append(__popc(above), taken);
        if (above)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (above >> e & 1) {
                    if (to < kWarpKeys) keys[to] = key_of(order_in<T>(s[e]), c0 + e);
                    ++to;
                }
    }
    if (rest >= 0)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = span.col(rest) + e;
            if (c < 0 || c >= a.classes || order_in<T>(edge[e]) < bound) continue;
            const unsigned to = atomicAdd(taken, 1u);
            if (to < kWarpKeys) keys[to] = key_of(order_in<T>(edge[e]), c);
        }
    __syncwarp();
    if (*taken <= kWarpKeys)
        put_in_order(team, keys, (int)*taken, a.count, [&](int place, uint64_t key) { write_one<T, ID>(a, (size_t)row, place, key); });
    else
        select_any<T, ID>(a, z + (size_t)row * a.ld, (size_t)row, keys, any[warp], team);
}

constexpr int kTopPieces = 64;                 // a row, at most
// Rows below this many, and longer than kTopFewBytes, are cut into pieces (24 x 131072 float32, top 64: 22 us in pieces, 16 by blocks).
constexpr int kTopFew = 48;
constexpr size_t kTopFewBytes = 1024 * 1024;
static bool may_cut(int classes, long rows, int element) {
    const int vec = 16 / element;
    return rows < kTopFew && (size_t)(classes + 2 * vec - 2) / vec * 16 > kTopFewBytes;
}

// The kernel for a call, by the rows' length, their number and the alignment.
template <typename T, typename ID>
static cudaError_t dispatch_top(const T* z, TopArgs a, cudaStream_t s) {
    constexpr int VEC = 16 / (int)sizeof(T), MOST = 32 / VEC;      // vectors a thread holds
    cudaError_t err = cudaSuccess;
    if (misaligned(z, 16))
        return launch_row(top_any_kernel<T, ID>, dim3((unsigned)std::min(a.rows, 148 * 16)), dim3(kAnyThreads), 0, s, z, a);
    const int vectors = RowSpan<VEC, false>::most(a.classes);
    auto held = [&](auto threads, auto n) {
        constexpr int THREADS = decltype(threads)::value, ROWS = THREADS < 128 ? 128 / THREADS : 1;
        err = launch_row(top_held_kernel<T, ID, THREADS, decltype(n)::value>, dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), dim3(THREADS < 128 ? 128 : THREADS), 0, s,
                         z, a);
    };
    auto held_by = [&](auto threads) {
        const int each = (vectors + decltype(threads)::value - 1) / decltype(threads)::value;
        if (each == 1) held(threads, std::integral_constant<int, 1>{});
        else if (each == 2) held(threads, std::integral_constant<int, 2>{});
        else if (each <= 4) held(threads, std::integral_constant<int, 4>{});
        else held(threads, std::integral_constant<int, MOST>{});
    };
    auto rows = [&](auto threads, auto pieces, int blocks) {
        constexpr int THREADS = decltype(threads)::value;
        err = launch_row(top_rows_kernel<T, ID, THREADS, decltype(pieces)::value>, dim3((unsigned)blocks), dim3(THREADS), 0, s, z, a);
    };
    using Threads32 = std::integral_constant<int, 32>;
    using Threads128 = std::integral_constant<int, 128>;
    using Threads256 = std::integral_constant<int, 256>;
    using Threads512 = std::integral_constant<int, 512>;
    // Rows that fill the machine by a warp each, where its 256 maxima are four for each score.  Longer rows are better with a block each (4096 x 8192
    // bfloat16, 32 of each: 36 us against 26; of 3000 float32, 2000 of them: 13 us by warps, 21 by blocks), and so are few (700: 10 against 9).
    const bool warps = a.count <= 64 && vectors <= 768 && vectors - 2 >= 3 * a.count && a.rows >= 148 * 10;
    if (vectors <= 32 * MOST && !(warps && vectors >= 64)) {
        held_by(Threads32{});
    } else if (warps) {
        err = launch_row(top_warp_kernel<T, ID>, dim3((unsigned)((a.rows + 3) / 4)), dim3(128), 0, s, z, a);
    } else if (vectors <= 128 * MOST) {
        held_by(Threads128{});
    } else if (vectors - 2 < 3 * a.count) {      // with fewer than three vectors for each score too many scores would reach the vectors' bound
        if constexpr (VEC == 8) held(Threads256{}, std::integral_constant<int, MOST>{});       // (never so for float32)
    } else {
        // few rows: as many pieces as fill the machine twice over, as keep four vectors a thread and three for each score, and as the joining block holds
        const int most = std::min({kTopPieces, kMergeEach * 512 / a.count, vectors / std::max(1024, 3 * a.count + 2)});
        const int pieces = std::min(most, (2 * 148 + a.rows - 1) / a.rows);
        if (may_cut(a.classes, a.rows, (int)sizeof(T)) && pieces > 1) {
            a.per = (vectors + pieces - 1) / pieces;
            a.pieces = (vectors + a.per - 1) / a.per;
            if (vectors - (a.pieces - 1) * a.per >= 3 * a.count + 2) {      // the last piece is the shortest
                rows(Threads512{}, std::true_type{}, a.rows * a.pieces);
                return err;
            }
        }
        // Small blocks, whose waits overlap, but at least two threads for each score, and four where a maximum stands for many vectors, which are
        // read again (64 of 50001 bfloat16: 262 us with 128 threads, 217 with 256; of 8192: 135 with 128, 161 with 256).
        if (a.rows < 148 * 2) rows(Threads512{}, std::false_type{}, a.rows);      // (fewer than the machine holds: a row's own time counts)
        else if (a.count <= 32 || (a.count <= 64 && vectors <= 4 * kKept * 128)) rows(Threads128{}, std::false_type{}, a.rows);
        else if (a.count <= 64 || (a.count <= 128 && vectors <= 4 * kKept * 256)) rows(Threads256{}, std::false_type{}, a.rows);
        else rows(Threads512{}, std::false_type{}, a.rows);
    }
    return err;
}

// Workspace: the counters, keys and sums of rows in pieces.
static int ensure_top(Top* t, cudaStream_t s) {
    const size_t blocks = (size_t)kTopFew * kTopPieces, need = 2048 + blocks * (sizeof(Softmax) + sizeof(uint64_t) * t->count);
    const bool fresh = t->ws.bytes < need;
    const int rc = ensure_scratch(t->ws, need, s, "circ_top_reserve");
    if (rc != CIRC_OK || !fresh) return rc;
    if (cudaMemsetAsync(t->ws.ptr, 0, 2048, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaFree(t->ws.ptr);
        t->ws.ptr = nullptr;
        t->ws.bytes = 0;
        set_error(CIRC_ERR_CUDA, "clearing the workspace failed: %s", cudaGetErrorString(cudaGetLastError()));
        return CIRC_ERR_CUDA;
    }
    return CIRC_OK;
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
    const bool cut = may_cut(t->classes, rows, (int)zb);      // else no workspace is used
    const int rc = cut ? ensure_top(t, s) : CIRC_OK;
    if (rc != CIRC_OK) return rc;
    char* ws = static_cast<char*>(t->ws.ptr);
    TopArgs a{};
    a.ld = ld;
    a.values = values;
    a.ids = ids;
    a.lse = lse;
    a.scale = (float)(1.4426950408889634 / (double)t->temperature);
    a.inv_tau = 1.0 / (double)t->temperature;
    a.rows = (int)rows;
    a.classes = t->classes;
    a.count = t->count;
    if (cut) {
        a.arrived = reinterpret_cast<unsigned*>(ws);
        a.overflow = reinterpret_cast<int*>(ws + 1024);
        a.keys = reinterpret_cast<uint64_t*>(ws + 2048);
        a.parts = reinterpret_cast<Softmax*>(a.keys + (size_t)kTopFew * kTopPieces * t->count);
    }
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
    return max_rows > 0 && may_cut(t->classes, 1, 4) ? ensure_top(t, 0) : CIRC_OK;      // (whatever type the logits get)
}

int circ_top_forward(circ_top_handle h, const void* logits, long stride, void* values, void* ids, float* lse, long rows, void* stream) {
    return run_top(reinterpret_cast<Top*>(h), logits, stride, values, ids, lse, rows, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
