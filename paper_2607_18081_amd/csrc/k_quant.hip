// Block quantisation to 8 bits: e4m3 codes with one float32 scale for each block of 1 x 128
// (activations) or 128 x 128 (weights) values of a row-major matrix.
//
//   a = max(max |x| of the block, 2^-60),  scale = a / 448,  code = e4m3(x * (448 / a))
//
// in float32, the code rounded to nearest even; 448 is the largest e4m3 value. The floor keeps
// 448 / a finite (a block of zeros gets codes 0). A block that holds a NaN or an infinity has no
// scale that its other values survive: its scale and all its codes are NaN, so the loss shows.
//
// Bound by HBM: 2 (4) bytes read and 1 written per value, each once. The maximum is taken on the
// bits of |x| (integer order equals float order there, and puts infinities and NaN on top), so
// one integer maximum also finds the blocks without a scale.
#include "common.h"
#include "launch.h"

namespace si {

namespace {

constexpr int kBlk = 128;           // columns (and rows) of a scale block
constexpr float kE4m3Max = 448.0f;
constexpr uint32_t kAmaxMin = 0x21800000u;  // 2^-60
constexpr uint32_t kInf = 0x7f800000u;
constexpr uint32_t kNan = 0x7fc00000u;
constexpr uint32_t kCodeNan = 0x7f7f7f7fu;  // four e4m3 NaN codes

// 8 consecutive values as loaded: one 16-byte vector of 16-bit data, two of float32
template <typename XT>
struct Eight {
    static constexpr int NV = 8 / Elem<XT>::V;
    V16 v[NV];
    __device__ __forceinline__ void load(const XT* p) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = ld16(p + i * Elem<XT>::V);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = V16{{0u, 0u, 0u, 0u}};
    }
    __device__ __forceinline__ void unpack(float* f) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) Elem<XT>::unpack(v[i], f + i * Elem<XT>::V);
    }
    __device__ __forceinline__ uint32_t amax() const {
        float f[8];
        unpack(f);
        uint32_t m = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7fffffffu);
        return m;
    }
};

// scale and 448 / a of a block by the bits of its largest |x|
__device__ __forceinline__ void block_scale(uint32_t am, float& scale, float& inv) {
    const float a = __uint_as_float(max(am, kAmaxMin));
    scale = am >= kInf ? __uint_as_float(kNan) : __fdiv_rn(a, kE4m3Max);
    inv = __fdiv_rn(kE4m3Max, a);
}

// the 8 codes; |x| * inv may pass 448 by a rounding, which the conversion would round back to
// 448 (the next code would be 480), so nothing is clamped
template <typename XT>
__device__ __forceinline__ void store_codes(const Eight<XT>& x, float inv, bool nan, uint8_t* q) {
    float f[8];
    x.unpack(f);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * inv, f[4 * i + 1] * inv, 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * inv, f[4 * i + 3] * inv, c, true);
        w[i] = nan ? kCodeNan : (uint32_t)c;
    }
    *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
}

// 1 x 128 blocks. 16 lanes hold a block, 8 values each; a wave's load covers 4 blocks (1 KB of
// 16-bit data). Block b is row b / nb, columns 128 (b % nb) on.
template <typename XT>
__global__ __launch_bounds__(256) void quant_rows(const XT* __restrict__ x, int64_t C, int64_t nb,
                                                  int64_t nblocks, uint8_t* __restrict__ codes,
                                                  float* __restrict__ scales) {
    const int64_t b = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (b >= nblocks) return;  // whole groups of 16 lanes
    const int64_t r = b / nb;
    const int64_t c = (b - r * nb) * kBlk + 8 * (threadIdx.x & 15);
    Eight<XT> v;
    if (c < C)
        v.load(x + r * C + c);
    else
        v.zero();
    uint32_t am = v.amax();
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) am = max(am, (uint32_t)__shfl_xor((int)am, m, 16));
    float scale, inv;
    block_scale(am, scale, inv);
    if (c < C) store_codes(v, inv, am >= kInf, codes + r * C + c);
    if ((threadIdx.x & 15) == 0) scales[b] = scale;
}

// 128 x 128 blocks of G matrices [R][C]: one work-group of 512 threads a block, the block's
// values in registers (4 loads of 8 values a thread) between the maximum and the codes.
template <typename XT>
__global__ __launch_bounds__(512) void quant_tiles(const XT* __restrict__ x, int64_t R, int64_t C,
                                                   int64_t nr, int64_t nc,
                                                   uint8_t* __restrict__ codes,
                                                   float* __restrict__ scales) {
    __shared__ uint32_t red[8];
    const int64_t b = blockIdx.x;
    const int64_t br = b / nc;           // row of blocks over all matrices
    const int64_t g = br / nr;
    const int64_t r0 = (br - g * nr) * kBlk + (threadIdx.x >> 4);
    const int64_t c = (b - br * nc) * kBlk + 8 * (threadIdx.x & 15);
    const int64_t base = (g * R + r0) * C + c;
    Eight<XT> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (c < C && r0 + 32 * i < R)
            v[i].load(x + base + 32 * i * C);
        else
            v[i].zero();
    }
    uint32_t am = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) am = max(am, v[i].amax());
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) am = max(am, (uint32_t)__shfl_xor((int)am, m, kWave));
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = am;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) am = max(am, red[w]);
    float scale, inv;
    block_scale(am, scale, inv);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c < C && r0 + 32 * i < R)
            store_codes(v[i], inv, am >= kInf, codes + base + 32 * i * C);
    if (threadIdx.x == 0) scales[b] = scale;
}

template <typename XT>
hipError_t launch(const void* x, int64_t G, int64_t R, int64_t C, int block_rows, uint8_t* codes,
                  float* scales, hipStream_t s) {
    const XT* p = static_cast<const XT*>(x);
    const int64_t nc = (C + kBlk - 1) / kBlk;
    if (block_rows == 1) {
        const int64_t nblocks = G * R * nc;
        quant_rows<XT><<<dim3((unsigned)((nblocks + 15) / 16)), 256, 0, s>>>(p, C, nc, nblocks,
                                                                            codes, scales);
    } else {
        const int64_t nr = (R + kBlk - 1) / kBlk;
        quant_tiles<XT><<<dim3((unsigned)(G * nr * nc)), 512, 0, s>>>(p, R, C, nr, nc, codes,
                                                                     scales);
    }
    return hipGetLastError();
}

}  // namespace

int64_t quant_blocks(int64_t G, int64_t R, int64_t C, int block_rows) {
    return G * ((R + block_rows - 1) / block_rows) * ((C + kBlk - 1) / kBlk);
}

hipError_t launch_quant(const void* x, int xdt, int64_t G, int64_t R, int64_t C, int block_rows,
                        uint8_t* codes, float* scales, hipStream_t s) {
    if (xdt == 0) return launch<float>(x, G, R, C, block_rows, codes, scales, s);
    if (xdt == 1) return launch<bf16_t>(x, G, R, C, block_rows, codes, scales, s);
    return launch<f16_t>(x, G, R, C, block_rows, codes, scales, s);
}

}  // namespace si
