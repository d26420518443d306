// The experts of a mixture-of-experts layer for few tokens:
//
//   y[t] = sum over r < k of w[t][r] * D_e (SiLU(G_e x[t]) * (U_e x[t])),   e = ids[t][r]
//
// gate_up [E][2][I][d] and down [E][d][I] are read where they lie, each chosen expert once per 64
// of its tokens: with few tokens the time is that of streaming the chosen experts' weights, and
// every product runs on MFMAs whose token operand is mostly padding (16 tokens a tile), which is
// free below the weights' rate. Three kernels: gate/up with SiLU(g) * u, down, weighted sum.
//
// A pair is an entry p = t * k + r of ids. A work-group takes one expert and a tile of weight
// rows, finds the expert's pairs by reading ids itself (no list kernel, no launch that waits for
// one), and its waves split K. An id outside [0, E) belongs to no expert: nothing is read for it
// and it adds nothing.
//
// Element types: float32, bf16, half, or e4m3 codes with a float32 scale for each 128 x 128
// weights. Codes become the 16-bit type of x (exactly); a scale block's products are summed in
// float32 and then scaled into the total. h enters the down product in parts of 16 bits: bf16
// hi + lo (16 bits), hi + mid + lo (24 bits) when y is float32, and half hi + lo (22 bits); the
// extra MFMAs are free for the same reason.
#include <type_traits>

#include "common.h"
#include "launch.h"
#include "mfma.h"

namespace si {

namespace {

constexpr int kWaves = 4;           // a work-group's waves, which split K
constexpr int kLine = 128;          // bytes of a weight row a wave takes at a step
constexpr int kMaxNT = 4;           // token tiles of 16 served by one pass over the weights

// The 16-byte operand chunks that one 16-byte chunk of a weight row becomes, and the matrix
// product of one chunk pair.
template <typename XT, bool FP8>
struct Core {
    static constexpr int XC = 1;                        // operand chunks of a weight chunk
    static constexpr int KL = kLine / 16 * Elem<XT>::V; // values of a line
    typedef typename Mfma<XT>::vec8 vec;
    __device__ __forceinline__ static void widen(const V16& a, vec (&o)[1]) {
        o[0] = Mfma<XT>::vec(a);
    }
    __device__ __forceinline__ static f32x4_t mma(const vec& a, const V16& b, const f32x4_t& c) {
        return Mfma<XT>::mma(a, Mfma<XT>::vec(b), c);
    }
};
template <>
struct Core<float, false> {
    static constexpr int XC = 1;
    static constexpr int KL = 32;
    typedef V16 vec;
    __device__ __forceinline__ static void widen(const V16& a, vec (&o)[1]) { o[0] = a; }
    __device__ __forceinline__ static f32x4_t mma(const vec& a, const V16& b, f32x4_t c) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[e]),
                                                     __uint_as_float(b.w[e]), c, 0, 0, 0);
        return c;
    }
};
__device__ __forceinline__ V16 codes8(uint32_t lo, uint32_t hi, const bf16_t*) {
    return e4m3_to_bf16(lo, hi);
}
__device__ __forceinline__ V16 codes8(uint32_t lo, uint32_t hi, const f16_t*) {
    return e4m3_to_f16(lo, hi);
}
template <typename XT>
struct Core<XT, true> {
    static constexpr int XC = 2;
    static constexpr int KL = kLine;  // one scale block
    typedef typename Mfma<XT>::vec8 vec;
    __device__ __forceinline__ static void widen(const V16& a, vec (&o)[2]) {
        o[0] = Mfma<XT>::vec(codes8(a.w[0], a.w[1], (const XT*)nullptr));
        o[1] = Mfma<XT>::vec(codes8(a.w[2], a.w[3], (const XT*)nullptr));
    }
    __device__ __forceinline__ static f32x4_t mma(const vec& a, const V16& b, const f32x4_t& c) {
        return Mfma<XT>::mma(a, Mfma<XT>::vec(b), c);
    }
};

// The pairs of this work-group's expert, ascending, into list[]; their number. Every thread of
// the work-group calls it. by_pair: the grid's slot is a pair, and the work-group serves that
// pair's expert only if no earlier pair has it (else 0); otherwise the slot is the expert.
__device__ int expert_pairs(const int32_t* __restrict__ ids, int npairs, int E, int slot,
                            int by_pair, int& e, uint16_t* list, int* cnt) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    e = slot;
    if (by_pair) {
        e = ids[slot];
        if ((unsigned)e >= (unsigned)E) return 0;
    }
    // wave w scans a run of the pairs: count, then place after the earlier waves' pairs
    const int per = ((npairs + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int lo = wave * per, hi = min(npairs, lo + per);
    int n = 0;
    bool earlier = false;
    for (int b = lo; b < hi; b += 64) {
        const bool hit = b + lane < hi && ids[b + lane] == e;
        earlier |= hit && by_pair && b + lane < slot;
        n += __popcll(__ballot(hit));
    }
    if (lane == 0) cnt[wave] = n;
    if (__syncthreads_or(earlier)) return 0;
    int at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) at += cnt[w];
        total += cnt[w];
    }
    for (int b = lo; b < hi; b += 64) {
        const bool hit = b + lane < hi && ids[b + lane] == e;
        const unsigned long long m = __ballot(hit);
        if (hit) list[at + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)(b + lane);
        at += __popcll(m);
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(total);
}

// acc[r][n] += the product of RT row tiles and NT token tiles over this wave's lines.
//   wr, woff[r]   the expert's weights and the byte offset of this lane's row of tile r (kOOB:
//                 no such row), rb the bytes of a row
//   xr, xoff[n]   the token operand (PARTS planes, `plane` bytes apart) and the byte offset of
//                 this lane's token row of tile n (kOOB: none); xb its bytes
//   sc[r]         scales of tile r's rows, one a line (FP8)
// Lane (i, g) of a wave holds row i of a tile and columns 16 g .. of each half line, of the
// weights and of the tokens alike.
template <typename XT, bool FP8, int RT, int NT, int PARTS, int U>
__device__ __forceinline__ void lines(f32x4_t (&acc)[RT][NT], __amdgpu_buffer_rsrc_t wr,
                                      const int (&woff)[RT], int rb, __amdgpu_buffer_rsrc_t xr,
                                      const int (&xoff)[NT], int xb, int plane,
                                      const float* const (&sc)[RT], int l0, int l1) {
    using C = Core<XT, FP8>;
    const int g = (threadIdx.x & 63) >> 4;
    for (int l = l0; l < l1; l += U) {
        V16 a[U][RT][2], b[U][NT][PARTS][2 * C::XC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int o = (l + u) * kLine + 64 * h + 16 * g;
                const bool in = (l + u < l1) & (o < rb);
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    a[u][r][h] = bload16(wr, (in & (woff[r] >= 0)) ? woff[r] + o : kOOB);
            }
#pragma unroll
            for (int c = 0; c < 2 * C::XC; ++c) {
                const int o = C::XC == 1 ? (l + u) * kLine + 64 * c + 16 * g
                                         : (l + u) * 2 * kLine + 128 * (c >> 1) + 32 * g +
                                               16 * (c & 1);
                const bool in = (l + u < l1) & (o < xb);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
                        b[u][n][p][c] =
                            bload16(xr, (in & (xoff[n] >= 0)) ? xoff[n] + p * plane + o : kOOB);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f32x4_t blk[RT][NT];
            if (FP8) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int n = 0; n < NT; ++n) blk[r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    typename C::vec w[C::XC];
                    C::widen(a[u][r][h], w);
#pragma unroll
                    for (int c = 0; c < C::XC; ++c)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int p = 0; p < PARTS; ++p) {
                                f32x4_t& t = FP8 ? blk[r][n] : acc[r][n];
                                t = C::mma(w[c], b[u][n][p][h * C::XC + c], t);
                            }
                }
            if (FP8 && l + u < l1) {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const float s = sc[r][l + u];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[r][n][i] = fmaf(s, blk[r][n][i], acc[r][n][i]);
                }
            }
        }
    }
}

// lines of this wave: equal runs, in whole lines
__device__ __forceinline__ void wave_lines(int nl, int wave, int& l0, int& l1) {
    const int per = (nl + kWaves - 1) / kWaves;
    l0 = min(nl, wave * per);
    l1 = min(nl, l0 + per);
}

// element type and parts of h as the down product takes it
template <typename XT, bool FP8>
struct HType {
    typedef XT type;
};
template <>
struct HType<f16_t, true> {
    typedef bf16_t type;  // codes are exact in either type, and bf16 parts have no range limit
};

// h of half weights is kept as h / 256, so that it may reach 2^24 instead of 65504; the parts
// below the first carry a factor 2^11 each, which keeps them from being subnormal
constexpr float kHalfDown = 1.0f / 256.0f, kHalfUp = 256.0f;

__device__ __forceinline__ void put_h(float h, int64_t at, int64_t plane, int parts, float* o) {
    o[at] = h;
}
__device__ __forceinline__ uint16_t rne_bf16(float f) {
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}
__device__ __forceinline__ void put_h(float h, int64_t at, int64_t plane, int parts, bf16_t* o) {
    for (int p = 0; p < parts; ++p) {
        const uint16_t b = rne_bf16(h);
        o[p * plane + at] = b;
        h -= bf16_to_f32(b);
        // an infinite or NaN h stays in the first part alone
        if (!(fabsf(h) < HUGE_VALF)) h = 0.0f;
    }
}
__device__ __forceinline__ void put_h(float h, int64_t at, int64_t plane, int parts, f16_t* o) {
    h *= kHalfDown;
    for (int p = 0; p < parts; ++p) {
        const f16_t b = (f16_t)h;
        o[p * plane + at] = b;
        h = (h - (float)b) * 2048.0f;
        if (!(fabsf(h) < HUGE_VALF)) h = 0.0f;
    }
}

// ---- gate and up, SiLU(g) * u -> h ---------------------------------------------------------
// Work-group: 16 neurons (their gate and up rows) of one expert.
template <typename XT, bool FP8, int NT, int U>
__device__ __forceinline__ void gate_up_pass(
    const XT* x, int64_t xbytes, int d, int k, const uint8_t* gu, const float* gus, int I, int n0,
    const uint16_t* list, int m, typename HType<XT, FP8>::type* H, int64_t plane, int parts,
    f32x4_t* red) {
    constexpr int WB = FP8 ? 1 : (int)sizeof(XT);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int rb = d * WB;
    const auto wr = make_rsrc(gu, (int64_t)2 * I * rb);
    const auto xr = make_rsrc(x, xbytes);
    int woff[2], xoff[NT];
    woff[0] = n0 + row < I ? (n0 + row) * rb : kOOB;
    woff[1] = n0 + row < I ? (I + n0 + row) * rb : kOOB;
#pragma unroll
    for (int n = 0; n < NT; ++n)
        xoff[n] = 16 * n + row < m ? (list[16 * n + row] / k) * d * (int)sizeof(XT) : kOOB;
    const int nl = (rb + kLine - 1) / kLine;
    const int nb = (I + 127) / 128;
    const float* sc[2] = {nullptr, nullptr};
    if (FP8) {
        sc[0] = gus + (int64_t)(n0 / 128) * nl;
        sc[1] = gus + (int64_t)(nb + n0 / 128) * nl;
    }
    int l0, l1;
    wave_lines(nl, wave, l0, l1);
    f32x4_t acc[2][NT];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    lines<XT, FP8, 2, NT, 1, U>(acc, wr, woff, rb, xr, xoff, d * (int)sizeof(XT), 0, sc, l0, l1);
    __syncthreads();  // the last pass's reads of red are done
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) red[((wave * 2 + r) * NT + n) * 64 + lane] = acc[r][n];
    __syncthreads();
    // wave w finishes token tiles w, w + kWaves, ...
    for (int n = wave; n < NT; n += kWaves) {
        f32x4_t s[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            s[r] = red[(r * NT + n) * 64 + lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                const f32x4_t v = red[((w * 2 + r) * NT + n) * 64 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][i] += v[i];
            }
        }
        // lane (i, g) holds token i, neurons 4 g ..
        if (16 * n + row < m) {
            const int64_t pair = list[16 * n + row];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = n0 + 4 * g + i;
                if (j < I) put_h(silu_f32(s[0][i]) * s[1][i], pair * I + j, plane, parts, H);
            }
        }
    }
}

template <typename XT, bool FP8, int U>
__global__ __launch_bounds__(kWaves * 64) void moe_gate_up(
    const XT* __restrict__ x, int64_t T, int d, const int32_t* __restrict__ ids, int npairs, int k,
    const uint8_t* __restrict__ gate_up, const float* __restrict__ scales, int E, int I,
    int by_pair, typename HType<XT, FP8>::type* __restrict__ H, int parts) {
    extern __shared__ uint16_t list[];
    __shared__ f32x4_t red[kWaves * 2 * kMaxNT * 64];
    __shared__ int cnt[kWaves];
    int e;
    const int m = expert_pairs(ids, npairs, E, blockIdx.y, by_pair, e, list, cnt);
    if (m == 0) return;
    constexpr int WB = FP8 ? 1 : (int)sizeof(XT);
    const uint8_t* gu = gate_up + (int64_t)e * 2 * I * d * WB;
    const float* gs = FP8 ? scales + (int64_t)e * 2 * ((I + 127) / 128) * ((d + 127) / 128) : nullptr;
    const int n0 = blockIdx.x * 16;
    const int64_t plane = (int64_t)npairs * I;
    for (int c = 0; c < m; c += 16 * kMaxNT) {
        const int mc = min(m - c, 16 * kMaxNT);
        const int64_t xb = T * d * (int64_t)sizeof(XT);
        if (mc <= 16)
            gate_up_pass<XT, FP8, 1, U>(x, xb, d, k, gu, gs, I, n0, list + c, mc, H, plane, parts, red);
        else if (mc <= 32)
            gate_up_pass<XT, FP8, 2, U / 2>(x, xb, d, k, gu, gs, I, n0, list + c, mc, H, plane, parts, red);
        else
            gate_up_pass<XT, FP8, 4, U / 4>(x, xb, d, k, gu, gs, I, n0, list + c, mc, H, plane, parts, red);
    }
}

// ---- down -----------------------------------------------------------------------------------
// Work-group: 32 rows of one expert's down matrix (32 columns of y) -> z[pair][d] float32.
constexpr int kDownTiles = 2;

// factor of part p of h in the sum (half: see kHalfDown)
template <typename HT>
__device__ __forceinline__ float part_factor(int p) {
    return 1.0f;
}
template <>
__device__ __forceinline__ float part_factor<f16_t>(int p) {
    return p == 0 ? kHalfUp : kHalfUp / 2048.0f;
}

template <typename HT, bool FP8, int PARTS, int NT, int U>
__device__ __forceinline__ void down_pass(const HT* H, int64_t plane, int npairs, int d,
                                          const uint8_t* dn, const float* dns, int I, int c0,
                                          const uint16_t* list, int m, float* z, f32x4_t* red) {
    constexpr int RT = kDownTiles;
    constexpr int WB = FP8 ? 1 : (int)sizeof(HT);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int rb = I * WB;
    const auto wr = make_rsrc(dn, (int64_t)d * rb);
    const int hb = I * (int)sizeof(HT);
    const auto hr = make_rsrc(H, (int64_t)PARTS * plane * sizeof(HT));
    const int pl = (int)(plane * sizeof(HT));
    int woff[RT], xoff[NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        woff[r] = c0 + 16 * r + row < d ? (c0 + 16 * r + row) * rb : kOOB;
#pragma unroll
    for (int n = 0; n < NT; ++n)
        xoff[n] = 16 * n + row < m ? (int)list[16 * n + row] * hb : kOOB;
    const int nl = (rb + kLine - 1) / kLine;
    const float* sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        sc[r] = FP8 ? dns + (int64_t)(min(c0 + 16 * r, d - 1) / 128) * nl : nullptr;
    int l0, l1;
    wave_lines(nl, wave, l0, l1);
    f32x4_t acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (std::is_same<HT, f16_t>::value) {
        // parts of different weight: one product each
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p) {
            f32x4_t t[RT][NT];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n) t[r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            int xp[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) xp[n] = xoff[n] >= 0 ? xoff[n] + p * pl : kOOB;
            lines<HT, FP8, RT, NT, 1, U>(t, wr, woff, rb, hr, xp, hb, 0, sc, l0, l1);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[r][n][i] = fmaf(part_factor<HT>(p), t[r][n][i], acc[r][n][i]);
        }
    } else {
        lines<HT, FP8, RT, NT, PARTS, U>(acc, wr, woff, rb, hr, xoff, hb, pl, sc, l0, l1);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) red[((wave * RT + r) * NT + n) * 64 + lane] = acc[r][n];
    __syncthreads();
    for (int q = wave; q < RT * NT; q += kWaves) {
        const int r = q / NT, n = q - r * NT;
        f32x4_t s = red[q * 64 + lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            const f32x4_t v = red[(w * RT * NT + q) * 64 + lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += v[i];
        }
        const int c = c0 + 16 * r + 4 * g;
        // d is a multiple of 4: a lane's four columns are all in or all out
        if (16 * n + row < m && c < d)
            *reinterpret_cast<f32x4_t*>(z + (int64_t)list[16 * n + row] * d + c) = s;
    }
}

template <typename HT, bool FP8, int PARTS, int U>
__global__ __launch_bounds__(kWaves * 64) void moe_down(
    const HT* __restrict__ H, int d, const int32_t* __restrict__ ids, int npairs,
    const uint8_t* __restrict__ down, const float* __restrict__ scales, int E, int I, int by_pair,
    float* __restrict__ z) {
    extern __shared__ uint16_t list[];
    __shared__ f32x4_t red[kWaves * kDownTiles * kMaxNT * 64];
    __shared__ int cnt[kWaves];
    int e;
    const int m = expert_pairs(ids, npairs, E, blockIdx.y, by_pair, e, list, cnt);
    if (m == 0) return;
    constexpr int WB = FP8 ? 1 : (int)sizeof(HT);
    const uint8_t* dn = down + (int64_t)e * d * I * WB;
    const float* ds = FP8 ? scales + (int64_t)e * ((d + 127) / 128) * ((I + 127) / 128) : nullptr;
    const int c0 = blockIdx.x * 16 * kDownTiles;
    const int64_t plane = (int64_t)npairs * I;
    for (int c = 0; c < m; c += 16 * kMaxNT) {
        const int mc = min(m - c, 16 * kMaxNT);
        if (mc <= 16)
            down_pass<HT, FP8, PARTS, 1, U>(H, plane, npairs, d, dn, ds, I, c0, list + c, mc, z, red);
        else if (mc <= 32)
            down_pass<HT, FP8, PARTS, 2, U / 2>(H, plane, npairs, d, dn, ds, I, c0, list + c, mc, z, red);
        else
            down_pass<HT, FP8, PARTS, 4, U / 4>(H, plane, npairs, d, dn, ds, I, c0, list + c, mc, z, red);
    }
}

// ---- weighted sum ----------------------------------------------------------------------------
// y[t][c] = sum of w[t][r] * z[t k + r][c] over the r whose expert exists, in order of r
__device__ __forceinline__ void put4(float* y, const float (&v)[4]) {
    *reinterpret_cast<f32x4_t*>(y) = f32x4_t{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void put4(bf16_t* y, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(y) =
        make_uint2(rne_bf16(v[0]) | ((uint32_t)rne_bf16(v[1]) << 16),
                   rne_bf16(v[2]) | ((uint32_t)rne_bf16(v[3]) << 16));
}
__device__ __forceinline__ void put4(f16_t* y, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(y) =
        make_uint2(f32_to_f16_rne(v[0]) | (f32_to_f16_rne(v[1]) << 16),
                   f32_to_f16_rne(v[2]) | (f32_to_f16_rne(v[3]) << 16));
}

template <typename YT>
__global__ __launch_bounds__(256) void moe_sum(const float* __restrict__ z,
                                               const int32_t* __restrict__ ids,
                                               const float* __restrict__ w, int k, int E, int d,
                                               YT* __restrict__ y) {
    const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
    const int64_t t = blockIdx.y;
    if (c >= d) return;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int r = 0; r < k; ++r) {
        const int64_t p = t * k + r;
        if ((unsigned)ids[p] >= (unsigned)E) continue;
        const float f = w[p];
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(z + p * d + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fmaf(f, v[i], s[i]);
    }
    put4(y + t * d + c, s);
}

struct Plan {
    int64_t pairs;
    int parts, hbytes;  // parts of h and bytes of an element of one
    size_t off_z, total;
};
Plan moe_plan(int64_t T, int64_t k, int64_t d, int64_t I, int xdt, int wdt, int ydt) {
    Plan p;
    p.pairs = T * k;
    if (xdt == 0) {
        p.parts = 1;
        p.hbytes = 4;
    } else {
        p.hbytes = 2;
        p.parts = (xdt == 2 && wdt == 2) ? 2 : (ydt == 0 ? 3 : 2);
    }
    p.off_z = ((size_t)p.pairs * I * p.parts * p.hbytes + 255) / 256 * 256;
    p.total = p.off_z + (size_t)p.pairs * d * sizeof(float);
    return p;
}

struct Args {
    const void* x;
    int64_t T, d;
    const int32_t* ids;
    const float* w;
    int64_t k;
    const uint8_t* gate_up;
    const float* gus;
    const uint8_t* down;
    const float* dns;
    int64_t E, I;
    void* ws;
    Plan p;
    hipStream_t s;
};

template <typename XT, bool FP8, int PARTS>
void experts(const Args& a) {
    typedef typename HType<XT, FP8>::type HT;
    HT* H = static_cast<HT*>(a.ws);
    float* z = reinterpret_cast<float*>(static_cast<char*>(a.ws) + a.p.off_z);
    const int np = (int)a.p.pairs;
    // fewer pairs than experts: a slot a pair, so that no work-group is without an expert but
    // those of repeated ones; else a slot an expert
    const int by_pair = np <= a.E;
    const unsigned slots = (unsigned)(by_pair ? np : a.E);
    const size_t lds = ((size_t)np * sizeof(uint16_t) + 15) / 16 * 16;
    constexpr int U = 4;
    moe_gate_up<XT, FP8, U><<<dim3((unsigned)((a.I + 15) / 16), slots), kWaves * 64, lds, a.s>>>(
        static_cast<const XT*>(a.x), a.T, (int)a.d, a.ids, np, (int)a.k, a.gate_up, a.gus,
        (int)a.E, (int)a.I, by_pair, H, a.p.parts);
    constexpr int rows = 16 * kDownTiles;
    moe_down<HT, FP8, PARTS, U>
        <<<dim3((unsigned)((a.d + rows - 1) / rows), slots), kWaves * 64, lds, a.s>>>(
            H, (int)a.d, a.ids, np, a.down, a.dns, (int)a.E, (int)a.I, by_pair, z);
}

template <typename YT>
void sum(const Args& a, void* y) {
    const float* z = reinterpret_cast<const float*>(static_cast<char*>(a.ws) + a.p.off_z);
    moe_sum<YT><<<dim3((unsigned)((a.d + 1023) / 1024), (unsigned)a.T), 256, 0, a.s>>>(
        z, a.ids, a.w, (int)a.k, (int)a.E, (int)a.d, static_cast<YT*>(y));
}

}  // namespace

size_t moe_workspace(int64_t T, int64_t k, int64_t d, int64_t I, int xdt, int wdt, int ydt) {
    return moe_plan(T, k, d, I, xdt, wdt, ydt).total;
}

// planes of h, an expert's weights and x are addressed by 32-bit byte offsets
bool moe_supported(int64_t T, int64_t k, int64_t d, int64_t I, int xdt, int wdt, int ydt) {
    const int64_t top = ((int64_t)1 << 31) - 1;
    const int wb = wdt == 3 ? 1 : (wdt == 0 ? 4 : 2);
    const Plan p = moe_plan(T, k, d, I, xdt, wdt, ydt);
    return 2 * I * d * wb <= top && T * d * 4 <= top && p.pairs * I * p.parts * p.hbytes <= top;
}

hipError_t launch_moe(const void* x, int xdt, int64_t T, int64_t d, const int32_t* ids,
                      const float* w, int64_t k, const void* gate_up, const float* gus,
                      const void* down, const float* dns, int64_t E, int64_t I, int wdt, void* y,
                      int ydt, void* ws, hipStream_t s) {
    const Args a{x, T, d, ids, w, k, static_cast<const uint8_t*>(gate_up), gus,
                 static_cast<const uint8_t*>(down), dns, E, I, ws,
                 moe_plan(T, k, d, I, xdt, wdt, ydt), s};
    const bool three = a.p.parts == 3;
    if (wdt == 0)
        experts<float, false, 1>(a);
    else if (wdt == 2)
        experts<f16_t, false, 2>(a);
    else if (wdt == 1)
        three ? experts<bf16_t, false, 3>(a) : experts<bf16_t, false, 2>(a);
    else if (xdt == 1)
        three ? experts<bf16_t, true, 3>(a) : experts<bf16_t, true, 2>(a);
    else
        three ? experts<f16_t, true, 3>(a) : experts<f16_t, true, 2>(a);
    if (ydt == 0)
        sum<float>(a, y);
    else if (ydt == 1)
        sum<bf16_t>(a, y);
    else
        sum<f16_t>(a, y);
    return hipGetLastError();
}

}  // namespace si
