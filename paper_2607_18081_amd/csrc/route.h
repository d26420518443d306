// The choice of a token's experts from its logits (k_route.hip), for the kernels that make it.
#pragma once

#include "common.h"

namespace si {

// What a choice reads and how it ranks. part: float64 logits [KS][T][E], to be added in order.
struct Choice {
    const double* part;
    int KS, T, E;
    int EP;  // E rounded up to a power of two, at least 64
    const float* bias;
    int k, sigmoid, renorm;
    float scale;
    const int32_t* n_valid;
};

template <int MAXE>
struct ChoiceLds {
    uint64_t keys[MAXE];
    int rank[MAXE];
    double red[16];
    double chosen[32];
    int id[32];
};

// order key: unsigned order equals the order of the values, -0 = +0, NaN below every number
__device__ __forceinline__ uint64_t key_of(double v) {
    if (!(v == v)) return 1u;
    v += 0.0;  // -0 -> +0
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

// Fixed-order sum or maximum over the work-group's values
template <bool MAX>
__device__ __forceinline__ double group_reduce(double v, double* red) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        const double o = __shfl_xor(v, m, kWave);
        v = MAX ? fmax(v, o) : v + o;
    }
    const int n = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int i = 1; i < n; ++i) v = MAX ? fmax(v, red[i]) : v + red[i];
    return v;
}

// Chooses the experts of token t with the whole work-group (a multiple of EP threads, at least
// E): s.id[r] is the expert of rank r afterwards, -1 for a token past n_valid. With publish the ids
// and weights are written too (the weights are not computed without).
//
// Thread i < EP owns expert i; an expert's rank is the number of experts before it in the order,
// counted by blockDim / EP threads an expert from the keys in LDS: one exchange, where k rounds of
// a maximum over the work-group would take several each. Softmax weights that are divided by their
// chosen sum need no sum over the others: exp(z - top) / sum of the chosen, k exponentials.
template <int MAXE>
__device__ __forceinline__ void choose_experts(const Choice& a, int t, bool publish,
                                               int32_t* __restrict__ ids,
                                               float* __restrict__ weights, ChoiceLds<MAXE>& s) {
    const int i = threadIdx.x, E = a.E, k = a.k;
    if (a.n_valid && t >= *a.n_valid) {
        if (i < k) {
            s.id[i] = -1;
            if (publish) {
                ids[(int64_t)t * k + i] = -1;
                weights[(int64_t)t * k + i] = 0.0f;
            }
        }
        __syncthreads();
        return;
    }
    const bool mine = i < E;
    double z = 0.0;
    if (mine) {
        // (four loads at once: one after the other they cost a memory latency each)
        const double* part = a.part + (int64_t)t * E + i;
        const int64_t plane = (int64_t)a.T * E;
        for (int q = 0; q < a.KS; q += 4) {
            double v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = part[min(q + j, a.KS - 1) * plane];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (q + j < a.KS) z += v[j];
        }
    }
    // the score of a softmax by its logit alone, until the chosen are known
    const bool late = !a.sigmoid && a.renorm && !a.bias;
    double p = z;
    if (a.sigmoid) {
        p = 1.0 / (1.0 + exp(-z));
    } else if (!late) {
        const double top = group_reduce<true>(mine ? z : -HUGE_VAL, s.red);
        p = mine ? exp(z - top) : 0.0;
        p /= group_reduce<false>(p, s.red);
    }
    if (i < a.EP) {
        s.keys[i] = mine ? key_of(a.bias ? p + (double)a.bias[i] : z) : 0u;  // 0: below every one
        s.rank[i] = 0;
    }
    const bool nan = __syncthreads_or(mine && !(z == z));
    // thread i counts for expert i % EP over the i / EP-th part of the experts
    const int me = i & (a.EP - 1);
    if (me < E) {
        const int parts = (int)blockDim.x / a.EP, per = (E + parts - 1) / parts;
        const int lo = min(E, (i / a.EP) * per), hi = min(E, lo + per);
        const uint64_t m = s.keys[me];
        // (an equal key goes first from a lower expert; on which side of a lane's own an expert is,
        // is open only among the wave's own 64: 200 tokens, 256 experts 20.9 -> 19.0 us)
        const int own = __builtin_amdgcn_readfirstlane(me & ~63);
        int n = 0;
        auto count = [&](int from, int to, uint64_t past) {
#pragma unroll 8
            for (int j = from; j < to; ++j) n += s.keys[j] > past;
        };
        count(lo, min(hi, own), m - 1u);
#pragma unroll 8
        for (int j = max(lo, own); j < min(hi, own + 64); ++j)
            n += s.keys[j] > m - (uint64_t)(j < me);
        count(max(lo, own + 64), hi, m);
        if (n) atomicAdd(&s.rank[me], n);  // whole numbers: the order of the additions is free
    }
    __syncthreads();
    const int r = mine ? s.rank[i] : k;
    if (r < k) {
        s.chosen[r] = p;
        s.id[r] = i;
    }
    __syncthreads();
    if (!publish) return;
    if (late) {
        // (a NaN logit makes every score NaN, as in the softmax over all experts)
        const double top = s.chosen[0];
        const double e = i < k ? (nan ? __longlong_as_double(0x7ff8000000000000ll)
                                      : exp(s.chosen[i] - top))
                               : 0.0;
        __syncthreads();
        if (i < k) s.chosen[i] = e;
        __syncthreads();
    }
    if (i >= k) return;  // thread i: the expert of rank i
    double w = s.chosen[i], sum = 0.0;
    if (a.renorm)
        for (int j = 0; j < k; ++j) sum += s.chosen[j];
    if (a.renorm) w = sum > 0.0 || !(sum == sum) ? w / sum : 0.0;
    ids[(int64_t)t * k + i] = s.id[i];
    weights[(int64_t)t * k + i] = (float)(w * (double)a.scale);
}

}  // namespace si
