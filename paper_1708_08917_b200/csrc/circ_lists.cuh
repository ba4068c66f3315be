// A teacher's list of classes for one row, held by a warp: which of its entries count, their probabilities, and what the row's loss and
// gradient become once the student's other classes are summed up.
//   p_k = exp(t_k / tau - T) over the entries that count; T = log sum exp(t_k / tau), or the teacher's own lse where the other classes
//   count as one class more ("the rest", p_rest = max(0, 1 - sum p)).
//   a = log of the student's sum over the classes outside the list, lse = log(exp(a) + sum over the list), q_rest = exp(a - lse)
//   loss = sum p_k (log p_k - s_k / tau + lse) + p_rest (log p_rest - a + lse)
//   gradient, times tau: P q_k - p_k on the list, exp(s / tau - a) (P q_rest - p_rest) outside, with P = sum p_k + p_rest.
// The sum over the outside is taken without the listed classes, not as a difference: q_rest keeps its digits where the list holds nearly all.
// The teacher's side is float64: what the list leaves over, and the loss of a student that has learnt it, are small differences.
#pragma once
#include "circ_softmax.cuh"

namespace circ {

constexpr int kListMost = 256;                   // entries
constexpr int kListLanes = kListMost / 32;       // a lane's entries: lane, lane + 32, ...
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

// ITEMS: entries a lane (the list has at most 32 ITEMS).
template <int ITEMS>
struct TeacherList {
    int id[ITEMS];          // -1: does not count
    double p[ITEMS];
    float t[ITEMS], s[ITEMS];      // the teacher's values, the student's logits
    float given;            // the teacher's lse
    double mass, own, left; // sum p, sum p (t / tau - T), p_rest
    bool none;              // no teacher

    // The list as it lies in memory, with the student's logits of it; an id outside the classes does not count.
    template <typename T, typename V, typename ID>
    __device__ __forceinline__ void fetch(const ListSide& a, const V* __restrict__ values, const ID* __restrict__ ids, size_t row, const T* zr) {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const int k = j * 32 + lane;
            id[j] = -1;
            t[j] = s[j] = -INFINITY;
            if (k < a.count) {
                const ID c = ids[row * a.count + k];
                if (c >= 0 && c < (ID)a.classes) id[j] = (int)c;
                t[j] = to_float(values[row * a.count + k]);
            }
        }
        given = a.rest ? a.lse[row] : 0.f;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (id[j] >= 0) s[j] = to_float(zr[id[j]]);
    }
    // The teacher's side.  `table`: list_table(count) words of shared memory of this warp's own.
    __device__ __forceinline__ void prepare(const ListSide& a, uint32_t* table) {
        const int lane = threadIdx.x % 32, slots = list_table(a.count);
        __syncwarp();       // the row before is done with the table
        for (int i = lane; i < slots; i += 32) table[i] = kNoId;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            if (j * 32 >= a.count) break;
            const unsigned same = __match_any_sync(0xffffffffu, id[j]);
            bool first = false;
            if (id[j] >= 0 && lane == __ffs(same) - 1) {
                uint32_t slot = ((uint32_t)id[j] * 2654435761u) >> 16;
                for (int tries = 0; tries < slots; ++tries) {     // the table is at most half full
                    slot &= (uint32_t)slots - 1;
                    const uint32_t old = atomicCAS(table + slot, kNoId, (uint32_t)id[j]);
                    first = old == kNoId;
                    if (first || old == (uint32_t)id[j]) break;
                    ++slot;
                }
            }
            __syncwarp();   // earlier entries come first
            if (!first) id[j] = -1;
        }
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (id[j] >= 0) top = fmaxf(top, t[j]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        double e[ITEMS], sum = 0.0;
        const double base = top == -INFINITY ? 0.0 : (double)top;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            e[j] = 0.0;
            if (j * 32 >= a.count) break;
            if (id[j] >= 0) e[j] = exp(((double)t[j] - base) * a.inv_tau);
            sum += e[j];
        }
        sum = warp_sum(sum);
        // e / exp(T - base / tau)
        const double log_all = a.rest ? (double)given - base * a.inv_tau : log(sum), part = a.rest ? exp(-log_all) : 1.0 / sum;
        none = a.rest ? given == -INFINITY : sum == 0.0;
        mass = own = 0.0;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            p[j] = 0.0;
            if (j * 32 >= a.count) break;
            if (id[j] >= 0 && !none && e[j] != 0.0) {
                p[j] = e[j] * part;
                mass += p[j];
                own += p[j] * (((double)t[j] - base) * a.inv_tau - log_all);
            }
        }
        mass = warp_sum(mass);
        own = warp_sum(own);
        left = a.rest && !none && !(mass >= 1.0) ? 1.0 - mass : 0.0;
    }

    // `outside`: the student's classes outside the list; s holds its logits on the list.  q: the list's own gradients, before the same factor.
    __device__ __forceinline__ ListRow finish(const ListSide& a, Softmax outside, float (&q)[ITEMS]) const {
        float top = outside.top;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (id[j] >= 0) top = fmaxf(top, s[j]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        ListRow r;
        r.base = top == -INFINITY ? 0.f : top;
        float listed = 0.f;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            q[j] = 0.f;
            if (j * 32 >= a.count) break;
            if (id[j] >= 0) q[j] = exp2_of((s[j] - r.base) * a.scale);
            listed += q[j];
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
        if (!r.zero) {
            const float inv = 1.f / r.total;
            if (!r.empty) r.factor = (float)(r.all * (double)(rest / r.total) - r.p_rest) / (outside.sum * exp2_of(Exponent(outside.top, a.scale).shift));
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) q[j] = (float)(r.all * (double)(q[j] * inv) - p[j]);
        }
        return r;
    }
    __device__ __forceinline__ void losses(const ListSide& a, const ListRow& r, double& loss, double& lse) const {
        const double log_total = log((double)r.total);
        lse = (double)r.base * a.inv_tau + log_total;
        double cross = 0.0;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            if (j * 32 >= a.count) break;
            if (id[j] >= 0 && p[j] != 0.0) cross += p[j] * ((double)s[j] - (double)r.base);
        }
        cross = warp_sum(cross) * a.inv_tau;
        if (none || r.all == 0.0) {
            loss = 0.0;
        } else if (r.total == 0.f) {
            loss = INFINITY;
        } else {
            loss = own - cross + log_total * mass;
            if (r.p_rest != 0.0) loss += r.p_rest * (log(r.p_rest) - log((double)r.sum) - ((double)r.top - (double)r.base) * a.inv_tau + log_total);
        }
    }
};

}  // namespace circ
