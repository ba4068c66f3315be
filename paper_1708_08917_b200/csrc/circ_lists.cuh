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

// What one row's loss and gradient need; the same in every lane.
struct ListRow {
    double loss, lse;
    Exponent ex;            // of the classes outside the list ...
    float factor;           // ... whose gradient is exponential * factor, before grad_mean weight / (sum of weights tau)
    bool zero;              // no gradient
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

    // `outside`: the student's classes outside the list; s holds its logits on the list.
    __device__ __forceinline__ ListRow finish(const ListSide& a, Softmax outside, float (&q)[ITEMS]) const {
        float top = outside.top;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (id[j] >= 0) top = fmaxf(top, s[j]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float base = top == -INFINITY ? 0.f : top;
        float listed = 0.f;
        double cross = 0.0;
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            q[j] = 0.f;
            if (j * 32 >= a.count) break;
            if (id[j] >= 0) {
                q[j] = exp2_of((s[j] - base) * a.scale);
                if (p[j] != 0.0) cross += p[j] * ((double)s[j] - (double)base);
            }
            listed += q[j];
        }
        listed = warp_sum(listed);
        cross = warp_sum(cross) * a.inv_tau;
        const float rest = outside.top == -INFINITY && outside.sum == 0.f ? 0.f : outside.sum * exp2_of((outside.top - base) * a.scale);
        const float total = rest + listed;
        ListRow r{0.0, 0.0, Exponent(outside.top, a.scale), 0.f, false};
        const double log_total = log((double)total);
        r.lse = (double)base * a.inv_tau + log_total;
        const bool empty = outside.sum == 0.f;                       // its term is left out
        const double p_rest = empty ? 0.0 : left, all = mass + p_rest;
        r.zero = none || total == 0.f || all == 0.0;
        if (none || all == 0.0) {
            r.loss = 0.0;
        } else if (total == 0.f) {
            r.loss = INFINITY;
        } else {
            r.loss = own - cross + log_total * mass;
            if (p_rest != 0.0) r.loss += p_rest * (log(p_rest) - log((double)outside.sum) - ((double)outside.top - (double)base) * a.inv_tau + log_total);
        }
        if (!r.zero) {
            const float inv = 1.f / total;
            r.factor = empty ? 0.f : (float)(all * (double)(rest / total) - p_rest) / (outside.sum * exp2_of(r.ex.shift));
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) q[j] = (float)(all * (double)(q[j] * inv) - p[j]);
        }
        return r;
    }
};

}  // namespace circ
