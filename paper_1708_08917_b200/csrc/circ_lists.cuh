// A teacher's list of classes for one row, held by a warp: which of its entries count, their probabilities, and what the row's loss and
// gradient become once the student's other classes are summed up.
//   p_k = exp(t_k / tau - T) over the entries that count; T = log sum exp(t_k / tau), or the teacher's own lse where the other classes
//   count as one class more ("the rest", p_rest = max(0, 1 - sum p)).
//   a = log of the student's sum over the classes outside the list, lse = log(exp(a) + sum over the list), q_rest = exp(a - lse)
//   loss = sum p_k (log p_k - s_k / tau + lse) + p_rest (log p_rest - a + lse)
//   gradient, times tau: P q_k - p_k on the list, exp(s / tau - a) (P q_rest - p_rest) outside, with P = sum p_k + p_rest.
// The sum over the outside is taken without the listed classes, not as a difference: q_rest keeps its digits where the list holds nearly all.
// The teacher's side is float64: what the list leaves over, and the loss of a student that has learnt it, are small differences.  The student's exponentials
// and their sums are float32 (a few 2^-24 of its probabilities, no more than a float32 logit's rounding makes of them); logarithms and the loss are float64 again.
#pragma once
#include "circ_softmax.cuh"

namespace circ {

constexpr int kListMost = 256;                   // entries
constexpr uint32_t kNoId = 0xffffffffu;

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Slots of the table that finds repeated ids: at least twice the entries.
__host__ __device__ inline int list_table(int count) {
    int n = 64;
    while (n < 2 * count) n *= 2;
    return n;
}

struct ListSide {
    const float* lse;       // the teacher's, or NULL
    double inv_tau;
    float scale;            // log2(e) / tau
    int classes, count;
    bool rest;
};

// What a row's gradient needs, and its loss further on; the same in every lane.
struct ListRow {
    float top;              // of the classes outside the list ...
    float factor;           // ... whose gradient is 2^(s scale - base) * factor (Exponent), before grad_mean weight / (sum of weights tau)
    bool zero;              // no gradient
    bool empty;             // nothing outside the list
    float base, total, sum; // exponentials relative to base, all of them; of those outside relative to their own top
    double p_rest, all;
};

// A list in shared memory; a lane of its warp works on the entries lane, lane + 32, ...  (In registers they cost the kernel's other warps
// occupancy, and where those were spilled, every use of one a trip through an L1 cache that the rows stream through: 5000 to 17000 cycles a row.)
template <int MOST>
struct ListSpace {
    double p[MOST];
    float t[MOST], s[MOST];     // the teacher's values (later the entries' gradients), the student's logits
    int id[MOST];               // -1: does not count
};

template <int MOST>
struct TeacherList {
    ListSpace<MOST>& at;
    double mass, own, left;     // sum p, this lane's part of sum p (t / tau - T), p_rest
    float given;                // the teacher's lse
    bool none;                  // no teacher
    __device__ __forceinline__ explicit TeacherList(ListSpace<MOST>& space) : at(space) {}

    // The list as it lies in memory, with the student's logits of it; an id outside the classes does not count.
    template <typename T, typename V, typename ID>
    __device__ __forceinline__ void fetch(const ListSide& a, const V* __restrict__ values, const ID* __restrict__ ids, size_t row, const T* zr) {
        const int lane = threadIdx.x % 32;
        constexpr int N = MOST / 32;
        int c[N];
        float t[N], s[N];
        given = a.rest ? a.lse[row] : 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            c[j] = -1;
            if (j * 32 + lane < a.count) {
                const ID i = ids[row * a.count + j * 32 + lane];
                if (i >= 0 && i < (ID)a.classes) c[j] = (int)i;
                t[j] = to_float(values[row * a.count + j * 32 + lane]);
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c[j] >= 0) s[j] = to_float(zr[c[j]]);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j * 32 + lane < a.count) {
                at.id[j * 32 + lane] = c[j];
                at.t[j * 32 + lane] = t[j];
                at.s[j * 32 + lane] = c[j] >= 0 ? s[j] : -INFINITY;
            }
    }
    // Calls take(id), by the first lane of each id, for the entries in their order; the entries that it does not want, and those behind a first one,
    // no longer count.
    template <typename F>
    __device__ __forceinline__ void keep_first(const ListSide& a, F take) {
        const int lane = threadIdx.x % 32;
        for (int k0 = 0; k0 < a.count; k0 += 32) {
            const int k = k0 + lane, id = k < a.count ? at.id[k] : -1;
            const unsigned same = __match_any_sync(0xffffffffu, id);
            bool first = false;
            if (id >= 0 && lane == __ffs(same) - 1) first = take(id);
            __syncwarp();
            if (id >= 0 && !first) at.id[k] = -1;
        }
    }
    // The same by a table of list_table(count) words of shared memory.
    __device__ __forceinline__ void keep_first(const ListSide& a, uint32_t* table) {
        const int slots = list_table(a.count);
        for (int i = threadIdx.x % 32; i < slots; i += 32) table[i] = kNoId;
        __syncwarp();
        keep_first(a, [&](int id) {
            uint32_t slot = ((uint32_t)id * 2654435761u) >> 16;
            for (int tries = 0; tries < slots; ++tries, ++slot) {      // the table is at most half full
                slot &= (uint32_t)slots - 1;
                const uint32_t old = atomicCAS(table + slot, kNoId, (uint32_t)id);
                if (old == kNoId) return true;
                if (old == (uint32_t)id) return false;
            }
            return false;
        });
    }
    // The teacher's side.
    __device__ __forceinline__ void prepare(const ListSide& a) {
        const int lane = threadIdx.x % 32;
        float top = -INFINITY;
        for (int k = lane; k < a.count; k += 32)
            if (at.id[k] >= 0) top = fmaxf(top, at.t[k]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const double base = top == -INFINITY ? 0.0 : (double)top;
        double sum = 0.0;
        for (int k = lane; k < a.count; k += 32) {
            const double e = at.id[k] >= 0 ? exp(((double)at.t[k] - base) * a.inv_tau) : 0.0;
            at.p[k] = e;
            sum += e;
        }
        // e / exp(T - base / tau)
        double log_all, part;
        if (a.rest) {
            log_all = (double)given - base * a.inv_tau;
            part = exp(-log_all);
            none = given == -INFINITY;
        } else {
            sum = warp_sum(sum);
            log_all = log(sum);
            part = 1.0 / sum;
            none = sum == 0.0;
        }
        mass = own = 0.0;
        for (int k = lane; k < a.count; k += 32) {
            const double e = at.p[k], p = e != 0.0 && !none ? e * part : 0.0;
            at.p[k] = p;
            mass += p;
            if (p != 0.0) own += p * (((double)at.t[k] - base) * a.inv_tau - log_all);
        }
        mass = warp_sum(mass);
        left = a.rest && !none && !(mass >= 1.0) ? 1.0 - mass : 0.0;
    }

    // `outside`: the student's classes outside the list.  The entries' own gradients, before the same factor, take the place of the teacher's values.
    __device__ __forceinline__ ListRow finish(const ListSide& a, Softmax outside) const {
        const int lane = threadIdx.x % 32;
        float top = outside.top;
        for (int k = lane; k < a.count; k += 32)
            if (at.id[k] >= 0) top = fmaxf(top, at.s[k]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        ListRow r;
        r.base = top == -INFINITY ? 0.f : top;
        float listed = 0.f;
        for (int k = lane; k < a.count; k += 32) {
            const float q = at.id[k] >= 0 ? exp2_of((at.s[k] - r.base) * a.scale) : 0.f;
            at.t[k] = q;
            listed += q;
        }
        listed = warp_sum(listed);
        const float rest = outside.top == -INFINITY && outside.sum == 0.f ? 0.f : outside.sum * exp2_of((outside.top - r.base) * a.scale);
        r.top = outside.top;
        r.sum = outside.sum;
        r.total = rest + listed;
        r.empty = outside.sum == 0.f;                       // its term is left out
        r.p_rest = r.empty ? 0.0 : left;
        r.all = mass + r.p_rest;
        r.zero = none || r.total == 0.f || r.all == 0.0;
        r.factor = 0.f;
        if (!r.zero && !r.empty) r.factor = (float)(r.all * (double)(rest / r.total) - r.p_rest) / (outside.sum * exp2_of(Exponent(outside.top, a.scale).shift));
        return r;
    }
    // The gradient of entry k, before the factor that all rows share.
    __device__ __forceinline__ float slope(const ListRow& r, int k) const { return (float)(r.all * (double)(at.t[k] / r.total) - at.p[k]); }
    __device__ __forceinline__ void losses(const ListSide& a, const ListRow& r, double& loss, double& lse) const {
        const double log_total = log((double)r.total);
        lse = (double)r.base * a.inv_tau + log_total;
        double mine = 0.0;
        for (int k = threadIdx.x % 32; k < a.count; k += 32)
            if (at.p[k] != 0.0) mine += at.p[k] * ((double)at.s[k] - (double)r.base);
        mine = warp_sum(own - mine * a.inv_tau);
        if (none || r.all == 0.0) {
            loss = 0.0;
        } else if (r.total == 0.f) {
            loss = INFINITY;
        } else {
            loss = mine + log_total * mass;
            if (r.p_rest != 0.0) loss += r.p_rest * (log(r.p_rest * ((double)r.total / (double)r.sum)) - ((double)r.top - (double)r.base) * a.inv_tau);
        }
    }
};

}  // namespace circ
