// The router of a mixture-of-experts layer: logits z = W x, the k experts of each token, and
// their weights.
//
//   score p = softmax(z) over the experts, or sigmoid(z)
//   key     = z, or p + bias where a choice bias is given
//   chosen  : the k largest keys, equal keys to the lower expert, NaN after every number
//   weight  = scale * p / (sum of the chosen p, in rank order)   (or scale * p)
//
// Which experts a token takes is a comparison of sums, so the sums are kept from depending on
// their order as far as it costs nothing: MFMAs of 16-bit data add 32 products in float32, and
// those short sums are added in float64, as are the parts of a split reduction. Scores, keys and
// weights are float64 too (E of them a token) and the weights are rounded once.
#include "common.h"
#include "launch.h"
#include "mfma.h"
#include "route.h"

namespace si {

namespace {

// ---- logits ------------------------------------------------------------------------------
// One K step: 16 bytes of a weight row a lane (four lanes a row: 32 values of 16-bit data, 16 of
// float32), and the same columns of a token.
template <typename XT, typename WT>
struct Step {  // a float32 router over 16-bit activations
    static constexpr int K = 16;
    __device__ __forceinline__ static V16 tokens(__amdgpu_buffer_rsrc_t xr, int xo) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(xr, xo, 0, 0);
        return V16{{(uint32_t)v[0], (uint32_t)v[1], 0u, 0u}};
    }
    __device__ __forceinline__ static f32x4_t mma(const V16& w, const V16& x) {
        float f[8];
        Elem<XT>::unpack(x, f);
        f32x4_t z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            z = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w[e]), f[e], z, 0, 0, 0);
        return z;
    }
};
template <typename T>
struct Step<T, T> {
    static constexpr int K = 4 * Elem<T>::V;
    __device__ __forceinline__ static V16 tokens(__amdgpu_buffer_rsrc_t xr, int xo) {
        return bload16(xr, xo);
    }
    __device__ __forceinline__ static f32x4_t mma(const V16& w, const V16& x) {
        f32x4_t z = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                z = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w[e]),
                                                         __uint_as_float(x.w[e]), z, 0, 0, 0);
        } else {
            z = Mfma<T>::mma(Mfma<T>::vec(w), Mfma<T>::vec(x), z);
        }
        return z;
    }
};

// One work-group of 4 waves a tile of 16 experts x 16 tokens and a K chunk, of which each wave
// takes a run. The experts' rows are the MFMA's M operand, tokens its N operand. U steps' loads
// are issued before the first product.
constexpr int kLogitWaves = 4;

template <typename XT, typename WT>
__global__ __launch_bounds__(kLogitWaves * 64) void route_logits(
    const XT* __restrict__ x, const WT* __restrict__ w, int T, int E, int64_t d, int kchunk,
    double* __restrict__ part) {
    using S = Step<XT, WT>;
    constexpr int U = 8;
    __shared__ double red[kLogitWaves][256];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
    // rows of the two operand tiles only: 32-bit offsets hold for any number of tokens, and rows
    // past the last lie past the descriptor's end and read zeros
    const auto wr = make_rsrc(w + (int64_t)e0 * d, (int64_t)min(16, E - e0) * d * sizeof(WT));
    const auto xr = make_rsrc(x + (int64_t)t0 * d, (int64_t)min(16, T - t0) * d * sizeof(XT));
    const int run = kchunk / kLogitWaves;
    const int k0 = blockIdx.z * kchunk + wave * run, k1 = min((int)d, k0 + run);
    constexpr int V = S::K / 4;  // values a lane
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    for (int k = k0; k < k1; k += U * S::K) {
        V16 a[U], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = k + u * S::K + V * g;
            a[u] = bload16(wr, c < k1 ? (int)((row * d + c) * sizeof(WT)) : kOOB);
            b[u] = S::tokens(xr, c < k1 ? (int)((row * d + c) * sizeof(XT)) : kOOB);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const f32x4_t s = S::mma(a[u], b[u]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += (double)s[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[wave][row * 16 + 4 * g + i] = acc[i];  // [token][expert]
    __syncthreads();
    const int t = threadIdx.x >> 4, e = threadIdx.x & 15;
    double s = red[0][threadIdx.x];
#pragma unroll
    for (int v = 1; v < kLogitWaves; ++v) s += red[v][threadIdx.x];
    if (t0 + t < T && e0 + e < E)
        part[((int64_t)blockIdx.z * T + t0 + t) * E + e0 + e] = s;
}

// ---- choice ------------------------------------------------------------------------------

// One work-group a token
__global__ __launch_bounds__(1024) void route_choose(Choice a, int32_t* __restrict__ ids,
                                                    float* __restrict__ weights) {
    __shared__ ChoiceLds<1024> s;
    choose_experts<1024>(a, blockIdx.x, true, ids, weights, s);
}

template <typename XT, typename WT>
void logits(const void* x, const void* w, int64_t T, int64_t E, int64_t d, int kchunk, int KS,
            double* part, hipStream_t s) {
    const dim3 grid((unsigned)((E + 15) / 16), (unsigned)((T + 15) / 16), (unsigned)KS);
    route_logits<XT, WT><<<grid, kLogitWaves * 64, 0, s>>>(
        static_cast<const XT*>(x), static_cast<const WT*>(w), (int)T, (int)E, d, kchunk, part);
}

}  // namespace

// K chunks of the logits: enough work-groups to spread the call over the chip (512 columns each
// at least), one chunk where the tiles of experts and tokens do that alone. (200 tokens, 256
// experts, d = 5120: 2 to 5 chunks, one to four expert tiles a work-group and one to eight steps
// ahead all take 11 to 13 us, 8 of them without any load.)
int route_chunks(int64_t T, int64_t E, int64_t d) {
    const int64_t tiles = ((E + 15) / 16) * ((T + 15) / 16);
    int64_t ks = (512 + tiles - 1) / tiles;
    const int64_t most = (d + 511) / 512;
    if (ks > most) ks = most;
    if (ks > 16) ks = 16;
    return (int)ks;
}

size_t route_workspace(int64_t T, int64_t E, int64_t d) {
    return (size_t)route_chunks(T, E, d) * T * E * sizeof(double);
}

Choice route_logits_of(const void* x, int xdt, int64_t T, int64_t d, const void* w, int wdt,
                       int64_t E, const float* bias, int64_t k, int sigmoid, int renorm,
                       float scale, const int32_t* n_valid, void* ws, hipStream_t s) {
    const int KS = route_chunks(T, E, d);
    // chunks of whole 64-value runs of the waves (whole lines of 16-bit data)
    constexpr int kRun = 64 * kLogitWaves;
    const int kchunk = (int)(((d + KS - 1) / KS + kRun - 1) / kRun * kRun);
    double* part = static_cast<double*>(ws);
    if (xdt == 0)
        logits<float, float>(x, w, T, E, d, kchunk, KS, part, s);
    else if (xdt == 1 && wdt == 1)
        logits<bf16_t, bf16_t>(x, w, T, E, d, kchunk, KS, part, s);
    else if (xdt == 1)
        logits<bf16_t, float>(x, w, T, E, d, kchunk, KS, part, s);
    else if (wdt == 2)
        logits<f16_t, f16_t>(x, w, T, E, d, kchunk, KS, part, s);
    else
        logits<f16_t, float>(x, w, T, E, d, kchunk, KS, part, s);
    int EP = 64;
    while (EP < E) EP *= 2;
    return Choice{part, KS, (int)T, (int)E, EP, bias, (int)k, sigmoid, renorm, scale, n_valid};
}

hipError_t launch_choose(const Choice& c, int32_t* ids, float* weights, hipStream_t s) {
    // more threads an expert where there are many to compare
    route_choose<<<dim3((unsigned)c.T), c.EP <= 128 ? 512 : 1024, 0, s>>>(c, ids, weights);
    return hipGetLastError();
}

}  // namespace si
