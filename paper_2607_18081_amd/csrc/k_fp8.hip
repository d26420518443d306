// Products of block-scaled 8-bit matrices:
//
//   y[m][n] = sum over blocks b of xs[m][b] * ws[n / 128][b] * sum over k in block b of
//             x[m][k] * w[n][k]
//
// x [M][K] codes with a scale for each 1 x 128 block, w [N][K] codes with a scale for each
// 128 x 128 block (k_quant.hip). One v_mfma_f32_16x16x128_f8f6f4 takes exactly one scale block
// of 16 weight rows and 16 tokens from a zero accumulator; its four results a lane belong to one
// token and four weight rows, so they are scaled into the float32 total by one factor.
//
// The 8-bit MFMA does not sum its products in full float32: measured on random codes, it aligns
// them to the largest and drops what lies 2^-14 below it, a relative error of 1.5e-5 of a result
// (bf16 MFMAs of the same codes: 9e-9). Below the rounding of a bf16 (1.7e-3) or half (2.1e-4)
// output that is invisible, and the 8-bit MFMA has twice the rate; a float32 output takes the
// codes as bf16, which holds them exactly.
#include "common.h"
#include "launch.h"
#include "mfma.h"

namespace si {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

constexpr int kBlk = 128;

__device__ __forceinline__ i32x8_t join(const V16& a, const V16& b) {
    return i32x8_t{(int)a.w[0], (int)a.w[1], (int)a.w[2], (int)a.w[3],
                   (int)b.w[0], (int)b.w[1], (int)b.w[2], (int)b.w[3]};
}
// An operand of one scale block: 32 codes a lane, as they are or as four bf16 vectors
template <bool EXACT>
struct Op {
    typedef i32x8_t type;
    __device__ __forceinline__ static type make(const V16& lo, const V16& hi) {
        return join(lo, hi);
    }
    // 16 rows x 16 tokens x 128 values, from zero (unit hardware scales)
    __device__ __forceinline__ static f32x4_t mma(const type& a, const type& b) {
        const f32x4_t z = {0.0f, 0.0f, 0.0f, 0.0f};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, z, 0, 0, 0, 0, 0, 0);
    }
};
template <>
struct Op<true> {
    struct type {
        Mfma<bf16_t>::vec8 v[4];
    };
    __device__ __forceinline__ static type make(const V16& lo, const V16& hi) {
        type t;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const V16& s = i < 2 ? lo : hi;
            t.v[i] = Mfma<bf16_t>::vec(e4m3_to_bf16(s.w[2 * (i & 1)], s.w[2 * (i & 1) + 1]));
        }
        return t;
    }
    __device__ __forceinline__ static f32x4_t mma(const type& a, const type& b) {
        f32x4_t c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) c = Mfma<bf16_t>::mma(a.v[i], b.v[i], c);
        return c;
    }
};

__device__ __forceinline__ void put(float* y, float v) { *y = v; }
__device__ __forceinline__ void put(bf16_t* y, float v) {
    *y = __builtin_bit_cast(uint16_t, (__bf16)v);
}
__device__ __forceinline__ void put(f16_t* y, float v) { *y = (f16_t)v; }

// ---- few tokens: the weights are streamed once ----------------------------------------------
// Work-group: 16 weight rows and up to 16 NT tokens; its waves take the scale blocks in turn.
constexpr int kWaves = 4;

template <typename YT, int NT, bool EXACT>
__global__ __launch_bounds__(kWaves * 64) void fp8_rows(
    const uint8_t* __restrict__ x, const float* __restrict__ xs, int M, int K,
    const uint8_t* __restrict__ w, const float* __restrict__ ws, int N, YT* __restrict__ y) {
    __shared__ f32x4_t red[kWaves * NT * 64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * NT;
    const int kb = (K + kBlk - 1) / kBlk;
    // descriptors of the tile's own rows: 32-bit offsets hold whatever M and N are
    const auto wr = make_rsrc(w + (int64_t)n0 * K, (int64_t)min(16, N - n0) * K);
    const int mt = min(16 * NT, M - m0);
    const auto xr = make_rsrc(x + (int64_t)m0 * K, (int64_t)mt * K);
    const float* wsc = ws + (int64_t)(n0 / kBlk) * kb;
    f32x4_t acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int wo = n0 + row < N ? row * K : kOOB;
    int xo[NT];
    const float* xsc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int t = 16 * n + row;
        xo[n] = t < mt ? t * K : kOOB;
        xsc[n] = xs + (int64_t)(m0 + min(t, mt - 1)) * kb;
    }
    for (int b = wave; b < kb; b += kWaves) {
        const int o = b * kBlk + 32 * g;
        const auto a = Op<EXACT>::make(bload16(wr, (o < K) & (wo >= 0) ? wo + o : kOOB),
                                       bload16(wr, (o + 16 < K) & (wo >= 0) ? wo + o + 16 : kOOB));
        const float sw = wsc[b];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const auto v =
                Op<EXACT>::make(bload16(xr, (o < K) & (xo[n] >= 0) ? xo[n] + o : kOOB),
                                bload16(xr, (o + 16 < K) & (xo[n] >= 0) ? xo[n] + o + 16 : kOOB));
            const f32x4_t t = Op<EXACT>::mma(a, v);
            const float s = sw * xsc[n][b];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = fmaf(s, t[i], acc[n][i]);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) red[(wave * NT + n) * 64 + lane] = acc[n];
    __syncthreads();
    for (int n = wave; n < NT; n += kWaves) {
        f32x4_t s = red[n * 64 + lane];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) {
            const f32x4_t p = red[(v * NT + n) * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += p[i];
        }
        const int t = 16 * n + row;
        if (t < mt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = n0 + 4 * g + i;
                if (c < N) put(y + (int64_t)(m0 + t) * N + c, s[i]);
            }
        }
    }
}

template <typename YT>
void run(const uint8_t* x, const float* xs, int64_t M, int64_t K, const uint8_t* w,
         const float* ws, int64_t N, YT* y, hipStream_t s) {
    constexpr bool EXACT = sizeof(YT) == 4;
    const unsigned gn = (unsigned)((N + 15) / 16);
    if (M <= 16)
        fp8_rows<YT, 1, EXACT><<<dim3(gn), kWaves * 64, 0, s>>>(x, xs, (int)M, (int)K, w, ws, (int)N, y);
    else
        fp8_rows<YT, 4, EXACT><<<dim3(gn, (unsigned)((M + 63) / 64)), kWaves * 64, 0, s>>>(
            x, xs, (int)M, (int)K, w, ws, (int)N, y);
}

}  // namespace

size_t fp8_workspace(int64_t M, int64_t N, int64_t K) { return 0; }

hipError_t launch_matmul_fp8(const uint8_t* x, const float* xs, int64_t M, int64_t K,
                             const uint8_t* w, const float* ws, int64_t N, void* y, int ydt,
                             void* wsp, hipStream_t s) {
    if (ydt == 0)
        run(x, xs, M, K, w, ws, N, static_cast<float*>(y), s);
    else if (ydt == 1)
        run(x, xs, M, K, w, ws, N, static_cast<bf16_t*>(y), s);
    else
        run(x, xs, M, K, w, ws, N, static_cast<f16_t*>(y), s);
    return hipGetLastError();
}

}  // namespace si
