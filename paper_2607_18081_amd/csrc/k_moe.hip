// The experts of a mixture-of-experts layer for few tokens:
//
//   y[t] = sum over r < k of w[t][r] * D_e (SiLU(G_e x[t]) * (U_e x[t])),   e = ids[t][r]
//
// gate_up [E][2][I][d] and down [E][d][I] are read where they lie, each chosen expert once per 16
// to 128 of its tokens: with few tokens the time is that of streaming the chosen experts' weights,
// and every product runs on MFMAs whose token operand is mostly padding (16 tokens a tile), which
// is free below the weights' rate. Three kernels: gate/up with SiLU(g) * u, down, weighted sum; two
// for one token, the router's choice included; two others for many tokens an expert, whose waves
// share the tokens' operand. Half weights take one more between gate/up and down (moe_h_parts).
//
// A pair is an entry p = t * k + r of ids. A work-group takes one expert and a tile of weight
// rows, finds the expert's pairs by reading ids itself (no list kernel, no launch that waits for
// one), and its waves share rows and K. An id outside [0, E) belongs to no expert: nothing is read
// for it and it adds nothing.
//
// Rates (weights of the experts that were chosen): 48 tokens over 8 experts of 14336 x 4096 in bf16
// 486 us, 5.8 TB/s; 13 tokens over 64 8-bit experts of 1408 x 4096 157 us, 5.1 TB/s; one token
// through 8 of 128 experts of 768 x 2048 24.5 us, of which three launches cost about 7.
//
// Element types: float32, bf16, half, or e4m3 codes with a float32 scale for each 128 x 128
// weights. Codes become the 16-bit type of x (exactly); a scale block's products are summed in
// float32 and then scaled into the total. h enters the down product in parts of 16 bits: bf16
// hi + lo (16 bits), hi + mid + lo (24 bits) when y is float32, and half hi + lo (22 bits) of h
// times a power of two by the pair's largest |h|; the extra MFMAs are free for the same reason.
#include <type_traits>

#include "common.h"
#include "launch.h"
#include "mfma.h"
#include "pipe.h"
#include "route.h"

namespace si {

namespace {

constexpr int kLine = 128;  // bytes of a weight row a wave takes at a step

// The 16-byte operand chunks that one 16-byte chunk of a weight row becomes, and the matrix
// product of one chunk pair.
template <typename XT, bool FP8>
struct Core {
    static constexpr int XC = 1;  // operand chunks of a weight chunk
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
template <int W>
__device__ __forceinline__ int expert_pairs(const int32_t* __restrict__ ids, int npairs, int E,
                                            int slot, int by_pair, int& e, uint16_t* list,
                                            int* cnt) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    e = slot;
    if (by_pair) {
        e = ids[slot];
        if ((unsigned)e >= (unsigned)E) return 0;
    }
    // wave w scans a run of the pairs: count, then place after the earlier waves' pairs
    const int per = ((npairs + W - 1) / W + 63) / 64 * 64;
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
    for (int v = 0; v < W; ++v) {
        if (v < wave) at += cnt[v];
        total += cnt[v];
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

// LDS reads of operand tiles: 16 bytes at addr0 + O and at addr1 + O for each of N tiles 2048 bytes
// apart, waited for in place. (Not ordinary loads: the compiler would wait for every load into LDS
// in flight before each of them, since it cannot tell the stages of a wave's ring apart.)
template <int N, int O>
__device__ __forceinline__ void lds_tiles(uint32_t addr0, uint32_t addr1, V16 (*out)[2]) {
    u32x4_t v0, v1;
    if constexpr (N == 1) {
        asm volatile(
            "ds_read_b128 %0, %2 offset:%4\n\t"
            "ds_read_b128 %1, %3 offset:%4\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v0), "=&v"(v1)
            : "v"(addr0), "v"(addr1), "n"(O)
            : "memory");
    } else {
        u32x4_t v2, v3;
        asm volatile(
            "ds_read_b128 %0, %4 offset:%6\n\t"
            "ds_read_b128 %1, %5 offset:%6\n\t"
            "ds_read_b128 %2, %4 offset:%7\n\t"
            "ds_read_b128 %3, %5 offset:%7\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3)
            : "v"(addr0), "v"(addr1), "n"(O), "n"(O + 2048)
            : "memory");
        out[1][0] = __builtin_bit_cast(V16, v2);
        out[1][1] = __builtin_bit_cast(V16, v3);
    }
    out[0][0] = __builtin_bit_cast(V16, v0);
    out[0][1] = __builtin_bit_cast(V16, v1);
    if constexpr (N > 2) lds_tiles<N - 2, O + 4096>(addr0, addr1, out + 2);
}
__device__ __forceinline__ uint32_t lds_addr(const char* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

// 1 KB loads into LDS that one line takes: two of 8 rows for each row tile, and for each token
// tile, part and 128 bytes of its columns
template <bool FP8, int RT, int NT, int PARTS>
constexpr int line_loads() {
    return 2 * RT + 2 * NT * PARTS * (FP8 ? 2 : 1);
}

// acc += the products of one line: operands a of the row tiles, b of the token tiles (by tile, part
// and, for codes, 128 bytes of columns), scales sc[r][l]
template <typename XT, bool FP8, int RT, int NT, int PARTS, int SUMS>
__device__ __forceinline__ void line_product(f32x4_t (&acc)[SUMS][RT][NT], const V16 (&a)[RT][2],
                                             const V16 (&b)[NT * PARTS * Core<XT, FP8>::XC][2],
                                             const float* const (&sc)[RT], int l) {
    using C = Core<XT, FP8>;
    constexpr int XC = C::XC;
    f32x4_t blk[SUMS][RT][NT];
    if (FP8) {
#pragma unroll
        for (int q = 0; q < SUMS; ++q)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n) blk[q][r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            typename C::vec w[XC];
            C::widen(a[r][h], w);
#pragma unroll
            for (int c = 0; c < XC; ++c)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        f32x4_t& t = FP8 ? blk[p % SUMS][r][n] : acc[p % SUMS][r][n];
                        t = C::mma(w[c],
                                   XC == 1 ? b[n * PARTS + p][h]
                                           : b[(n * PARTS + p) * XC + h * (XC - 1)][c], t);
                    }
        }
    if (FP8) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const float f = sc[r][l];
#pragma unroll
            for (int q = 0; q < SUMS; ++q)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[q][r][n][e] = fmaf(f, blk[q][r][n][e], acc[q][r][n][e]);
        }
    }
}

// acc[q][r][n] += the product of RT row tiles and NT token tiles over the lines [l0, l1): one total
// for all parts, or (half, whose parts differ in weight) one for each, SUMS = PARTS.
//   wr, woff[r]   the expert's weights and the byte offset of row lane / 8 of tile r, in woff[r][1]
//                 that of row lane / 8 + 8 (kOOB: no such row); rb the bytes of a row
//   xr, xoff[n]   the same for the token operand (PARTS planes, `plane` bytes apart), xb its bytes
//   sc[r]         scales of tile r's rows, one a line (FP8)
//   ring          this wave's own LDS: D stages of line_loads() KB
// A line goes from memory to LDS in whole 128-byte rows (8 rows a load), D lines ahead; chunk c of
// row r lies at c ^ (r % 8), so that the 16-row reads do not conflict. Loads straight into
// registers in the operand's shape, 64 bytes of 16 rows each, streamed at 3.4 to 4.4 TB/s. Lane
// (i, g) takes chunks g and 4 + g of row i.
template <typename XT, bool FP8, int RT, int NT, int PARTS, int SUMS, int D>
__device__ __forceinline__ void lines(f32x4_t (&acc)[SUMS][RT][NT], __amdgpu_buffer_rsrc_t wr,
                                      const int (&woff)[RT][2], int rb, __amdgpu_buffer_rsrc_t xr,
                                      const int (&xoff)[NT][2], int xb, int plane,
                                      const float* const (&sc)[RT], int l0, int l1, char* ring) {
    using C = Core<XT, FP8>;
    constexpr int XC = C::XC;
    constexpr int L = line_loads<FP8, RT, NT, PARTS>();
    static_assert(D >= 1 && (D - 1) * L <= 63, "outstanding loads");
    const int lane = threadIdx.x & 63;
    const int i = lane & 15, g = lane >> 4;
    const int lcol = ((lane & 7) ^ (lane >> 3)) * 16;
    auto load = [&](int l, char* at) {
        // lines past the run and columns past the row read zeros
        const bool in = (l < l1) & (l * kLine + lcol < rb);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                load_lds16<kNonTemporal>(wr, at + (2 * r + h) * 1024,
                                         (in & (woff[r][h] >= 0)) ? woff[r][h] + lcol : kOOB,
                                         l * kLine);
#pragma unroll
        for (int c = 0; c < XC; ++c) {
            const int o = (l * XC + c) * kLine;
            const bool xin = (l < l1) & (o + lcol < xb);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        load_lds16(xr, at + (2 * RT + 2 * ((n * PARTS + p) * XC + c) + h) * 1024,
                                   (xin & (xoff[n][h] >= 0)) ? xoff[n][h] + lcol : kOOB,
                                   p * plane + o);
        }
    };
#pragma unroll
    for (int d = 0; d < D; ++d) load(l0 + d, ring + d * L * 1024);
    const uint32_t base = lds_addr(ring) + i * kLine;
    // positions of this lane's chunks: g and 4 + g, or, of the tokens of a code line, 2 g and
    // 2 g + 1 of each half
    const uint32_t a0 = base + (g ^ (i & 7)) * 16, a1 = base + ((4 + g) ^ (i & 7)) * 16;
    const uint32_t x0 = XC == 1 ? a0 : base + ((2 * g) ^ (i & 7)) * 16;
    const uint32_t x1 = XC == 1 ? a1 : base + ((2 * g + 1) ^ (i & 7)) * 16;
    int slot = 0;
    for (int l = l0; l < l1; ++l) {
        wait_vm_lds<(D - 1) * L>();
        V16 a[RT][2], b[NT * PARTS * XC][2];
        const uint32_t at = slot * L * 1024;
        lds_tiles<RT, 0>(a0 + at, a1 + at, a);
        lds_tiles<NT * PARTS * XC, 2048 * RT>(x0 + at, x1 + at, b);
        load(l + D, ring + at);
        slot = slot + 1 == D ? 0 : slot + 1;
        line_product<XT, FP8, RT, NT, PARTS, SUMS>(acc, a, b, sc, l);
    }
    wait_vm_lds<0>();  // the ring is free again
}

// lines of a wave: equal runs, in whole lines
template <int WK>
__device__ __forceinline__ void wave_lines(int nl, int wk, int& l0, int& l1) {
    const int per = (nl + WK - 1) / WK;
    l0 = min(nl, wk * per);
    l1 = min(nl, l0 + per);
}

// element type and parts of h as the down product takes it
template <typename XT, bool FP8>
struct HType {
    typedef XT type;
};
template <>
struct HType<f16_t, true> {
    typedef bf16_t type;  // codes are exact in either type, and bf16 parts need no scale
};

// What gate and up write: the parts of h, or, of half weights, h itself. A half holds 11 bits from
// 2^-14 to 2^16 alone, so their parts are those of h * 2^e, by the largest finite |h| of the pair
// (half_scale): hi, and what hi leaves out times 2^11. That is 22 bits of each value down to 2^-27
// of the largest, and below that a step of 2^-49 of it, whatever the size of h. The largest is known
// when the pair's last neuron is, so the parts are a kernel of their own (moe_h_parts).
// (Parts of h / 256, without the maximum, lost bits below 2^-6 and everything below 2^-28.)
template <typename XT, bool FP8>
struct GateOut {
    typedef typename HType<XT, FP8>::type type;
};
template <>
struct GateOut<f16_t, false> {
    typedef float type;
};

constexpr float kLoUp = 2048.0f, kLoDown = 1.0f / 2048.0f;

// bits of |v|, 0 for an infinity or a NaN
__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
// up = 2^e that takes the largest |h| (by its bits) to [2^14, 2^15), and down = 2^-e; e <= 126
// keeps both normal
__device__ __forceinline__ void half_scale(uint32_t top, float& up, float& down) {
    const int e = min(126, 141 - (int)(top >> 23));
    up = __uint_as_float((uint32_t)(127 + e) << 23);
    down = __uint_as_float((uint32_t)(127 - e) << 23);
}
// the two parts of v = h * 2^e; an infinite or NaN h stays in the first alone
__device__ __forceinline__ void half_parts(float v, f16_t& hi, f16_t& lo) {
    hi = (f16_t)v;
    const float r = (v - (float)hi) * kLoUp;
    lo = (f16_t)(fabsf(r) < HUGE_VALF ? r : 0.0f);
}

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
// h of four neurons, at a multiple of 4 (rows of h hold a multiple of 4 too)
__device__ __forceinline__ void put_h4(const f32x4_t& h, int64_t at, int64_t plane, int parts,
                                       float* o) {
    *reinterpret_cast<f32x4_t*>(o + at) = h;
}
__device__ __forceinline__ void put_h4(const f32x4_t& h, int64_t at, int64_t plane, int parts,
                                       bf16_t* o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) put_h(h[e], at + e, plane, parts, o);
}

// LDS of a wave: its ring, which the sums of the waves reuse. Passes of 16, 32 and 64 tokens keep
// as many lines in flight as fit it.
template <int RING, bool FP8, int RT, int NT, int PARTS>
constexpr int ring_depth() {
    constexpr int by_lds = RING / 1024 / line_loads<FP8, RT, NT, PARTS>();
    constexpr int by_count = 63 / line_loads<FP8, RT, NT, PARTS>() + 1;
    constexpr int d = by_lds < by_count ? by_lds : by_count;
    return d < 4 ? d : 4;
}
// token tiles a pass: 4, or what leaves two lines in flight
template <int RING, bool FP8, int RT, int PARTS>
constexpr int max_tiles() {
    return ring_depth<RING, FP8, RT, 4, PARTS>() >= 2
               ? 4
               : (ring_depth<RING, FP8, RT, 2, PARTS>() >= 2 ? 2 : 1);
}

// Sums acc over the WK waves that split K of one row group, in order; on return out(q, s) has been
// called for this wave's share of the NQ tiles, each with its sum.
template <int WK, int NQ, typename F>
__device__ __forceinline__ void join_waves(const f32x4_t* acc, f32x4_t* red, int wk, int lane,
                                           F out) {
    if constexpr (WK == 1) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) out(q, acc[q]);
    } else {
        __syncthreads();  // the rings are done with
#pragma unroll
        for (int q = 0; q < NQ; ++q) red[(wk * NQ + q) * 64 + lane] = acc[q];
        __syncthreads();
        for (int q = wk; q < NQ; q += WK) {
            f32x4_t s = red[q * 64 + lane];
#pragma unroll
            for (int w = 1; w < WK; ++w) {
                const f32x4_t v = red[(w * NQ + q) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] += v[e];
            }
            out(q, s);
        }
        __syncthreads();  // before the next pass's loads
    }
}

// ---- gate and up, SiLU(g) * u -> h ---------------------------------------------------------
// Work-group: 16 NR neurons (their gate and up rows) of one expert, K split over WK waves.
template <typename XT, bool FP8, int RING, int WK, int NR, int NT>
__device__ __forceinline__ void gate_up_pass(
    const XT* x, int64_t xbytes, int d, int k, const uint8_t* gu, const float* gus, int I, int n0,
    const uint16_t* list, int m, typename GateOut<XT, FP8>::type* H, int64_t plane, int parts,
    int wk, char* ring, f32x4_t* red) {
    constexpr int WB = FP8 ? 1 : (int)sizeof(XT);
    constexpr int RT = 2 * NR;  // tile 2 q: gate rows of neurons 16 q .., 2 q + 1: their up rows
    constexpr int D = ring_depth<RING, FP8, RT, NT, 1>();
    const int lane = threadIdx.x & 63;
    const int row = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int rb = d * WB;
    const auto wr = make_rsrc(gu, (int64_t)2 * I * rb);
    const auto xr = make_rsrc(x, xbytes);
    int woff[RT][2], xoff[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int j = n0 + 16 * (r >> 1) + 8 * h + lr;
            woff[r][h] = j < I ? ((r & 1) * I + j) * rb : kOOB;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int t = 16 * n + 8 * h + lr;
            xoff[n][h] = t < m ? (list[t] / k) * d * (int)sizeof(XT) : kOOB;
        }
    }
    const int nl = (rb + kLine - 1) / kLine;
    const int nb = (I + 127) / 128;
    const float* sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        sc[r] = FP8 ? gus + (int64_t)((r & 1) * nb + min(n0 + 16 * (r >> 1), I - 1) / 128) * nl
                    : nullptr;
    int l0, l1;
    wave_lines<WK>(nl, wk, l0, l1);
    f32x4_t sums[1][RT][NT];
    auto& acc = sums[0];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    lines<XT, FP8, RT, NT, 1, 1, D>(sums, wr, woff, rb, xr, xoff, d * (int)sizeof(XT), 0, sc, l0,
                                    l1, ring);
    auto finish = [&](int q, const f32x4_t& sg, const f32x4_t& su) {
        // lane (i, g) holds token i, neurons 4 g ..
        const int nr = q / NT, n = q - nr * NT;
        if (16 * n + row < m) {
            const int64_t pair = list[16 * n + row];
            const int j = n0 + 16 * nr + 4 * g;
            f32x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = silu_f32(sg[e]) * su[e];
            if (j < I) put_h4(h, pair * I + j, plane, parts, H);
        }
    };
    constexpr int NQ = NR * NT;
    __syncthreads();  // the rings are done with
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int r = 0; r < 2; ++r)
            red[((wk * NQ + q) * 2 + r) * 64 + lane] = acc[2 * (q / NT) + r][q % NT];
    __syncthreads();
    for (int q = wk; q < NQ; q += WK) {
        f32x4_t s[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            s[r] = red[(q * 2 + r) * 64 + lane];
#pragma unroll
            for (int w = 1; w < WK; ++w) {
                const f32x4_t v = red[((w * NQ + q) * 2 + r) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r][e] += v[e];
            }
        }
        finish(q, s[0], s[1]);
    }
    __syncthreads();  // before the next pass's loads
}

template <typename XT, bool FP8, int RING, int WK, int NR>
__global__ __launch_bounds__(WK * 64) void moe_gate_up(
    const XT* __restrict__ x, int64_t T, int d, const int32_t* __restrict__ ids, int npairs, int k,
    const uint8_t* __restrict__ gate_up, const float* __restrict__ scales, int E, int I,
    int by_pair, typename GateOut<XT, FP8>::type* __restrict__ H, int parts) {
    extern __shared__ uint16_t list[];
    constexpr int MT = max_tiles<RING, FP8, 2 * NR, 1>();
    __shared__ __align__(1024) char rings[WK * RING];
    __shared__ int cnt[WK];
    int e;
    const int m = expert_pairs<WK>(ids, npairs, E, blockIdx.y, by_pair, e, list, cnt);
    if (m == 0) return;
    const int wk = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int WB = FP8 ? 1 : (int)sizeof(XT);
    const uint8_t* gu = gate_up + (int64_t)e * 2 * I * d * WB;
    const int nb = (I + 127) / 128;
    const float* gs = FP8 ? scales + (int64_t)e * 2 * nb * ((d + 127) / 128) : nullptr;
    const int n0 = blockIdx.x * 16 * NR;
    const int64_t plane = (int64_t)npairs * I;
    char* const ring = rings + wk * RING;
    f32x4_t* const red = reinterpret_cast<f32x4_t*>(rings);
    const int64_t xb = T * d * (int64_t)sizeof(XT);
    for (int c = 0; c < m; c += 16 * MT) {
        const int mc = min(m - c, 16 * MT);
        auto pass = [&](auto tiles) {
            gate_up_pass<XT, FP8, RING, WK, NR, decltype(tiles)::value>(
                x, xb, d, k, gu, gs, I, n0, list + c, mc, H, plane, parts, wk, ring, red);
        };
        if (mc <= 16)
            pass(std::integral_constant<int, 1>());
        else if (MT < 4 || mc <= 32)
            pass(std::integral_constant<int, MT < 2 ? MT : 2>());
        else
            pass(std::integral_constant<int, MT>());
    }
}

// ---- parts of h, half weights ----------------------------------------------------------------
// One work-group a pair: its largest finite |h|, then the parts of h * 2^e into two planes, and
// 2^-e into hs. The row stays in registers between the two, V vectors of each of TH threads. It
// costs its launch, 2.2 us of a layer's 25.4 for one token, and 4 bytes written, read and written a
// value: 48 to 96 tokens over 8 experts of 14336 x 4096, from 1% less to 3% more than parts without
// a scale. (Done by each work-group of moe_down_one in LDS, 2.3 us for one token.)
template <int TH, int V>
__global__ __launch_bounds__(TH) void moe_h_parts(const float* __restrict__ h,
                                                  const int32_t* __restrict__ ids, int E, int I,
                                                  int64_t plane, f16_t* __restrict__ H,
                                                  float* __restrict__ hs) {
    __shared__ uint32_t red[TH / kWave];
    const int64_t pair = blockIdx.x;
    if ((unsigned)ids[pair] >= (unsigned)E) return;  // no expert: no h was written
    const f32x4_t* row = reinterpret_cast<const f32x4_t*>(h + pair * I);
    const int n = I / 4;  // I is a multiple of 8
    f32x4_t v[V];
    uint32_t m = 0u;
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int i = threadIdx.x + u * TH;
        v[u] = i < n ? row[i] : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int u = 0; u < V; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = max(m, finite_bits(v[u][e]));
#pragma unroll
    for (int q = 1; q < kWave; q <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, q, kWave));
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TH / kWave; ++q) m = max(m, red[q]);
    float up, down;
    half_scale(m, up, down);
    f16_t* const o = H + pair * I;
#pragma unroll
    for (int u = 0; u < V; ++u) {
        const int i = threadIdx.x + u * TH;
        if (i < n) {
            f16_t p[2][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) half_parts(v[u][e] * up, p[0][e], p[1][e]);
#pragma unroll
            for (int q = 0; q < 2; ++q) __builtin_memcpy(o + q * plane + 4 * i, p[q], 8);
        }
    }
    if (threadIdx.x == 0) hs[pair] = down;
}

// ---- down -----------------------------------------------------------------------------------
// Work-group: WR groups of 16 RT rows of one expert's down matrix (columns of y), K split over WK
// waves -> z[pair][d] float32.

// acc[0] = the sum of the parts' totals (half: the lower part counts 2^-11)
template <int SUMS, int RT, int NT>
__device__ __forceinline__ void join_parts(f32x4_t (&acc)[SUMS][RT][NT]) {
    if constexpr (SUMS > 1) {
        static_assert(SUMS == 2, "hi and lo");
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[0][r][n][e] = fmaf(kLoDown, acc[1][r][n][e], acc[0][r][n][e]);
    }
}

// four columns of z of a pair, whose h of half weights was taken times 1 / hs[pair]
template <typename HT>
__device__ __forceinline__ void put_z(float* z, int64_t pair, int d, int c, const float* hs,
                                      f32x4_t s) {
    if constexpr (std::is_same<HT, f16_t>::value) {
        const float f = hs[pair];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] *= f;
    }
    *reinterpret_cast<f32x4_t*>(z + pair * d + c) = s;
}

template <typename HT, bool FP8, int PARTS, int RING, int WK, int RT, int NT>
__device__ __forceinline__ void down_pass(const HT* H, int64_t plane, int d, const uint8_t* dn,
                                          const float* dns, int I, int c0, const uint16_t* list,
                                          int m, const float* hs, float* z, int wk, char* ring,
                                          f32x4_t* red) {
    constexpr int WB = FP8 ? 1 : (int)sizeof(HT);
    const int lane = threadIdx.x & 63;
    const int row = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int rb = I * WB;
    const auto wr = make_rsrc(dn, (int64_t)d * rb);
    const int hb = I * (int)sizeof(HT);
    const auto hr = make_rsrc(H, (int64_t)PARTS * plane * sizeof(HT));
    const int pl = (int)(plane * sizeof(HT));
    int woff[RT][2], xoff[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int c = c0 + 16 * r + 8 * h + lr;
            woff[r][h] = c < d ? c * rb : kOOB;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int t = 16 * n + 8 * h + lr;
            xoff[n][h] = t < m ? (int)list[t] * hb : kOOB;
        }
    }
    const int nl = (rb + kLine - 1) / kLine;
    const float* sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        sc[r] = FP8 ? dns + (int64_t)(min(c0 + 16 * r, d - 1) / 128) * nl : nullptr;
    int l0, l1;
    wave_lines<WK>(nl, wk, l0, l1);
    constexpr int SUMS = std::is_same<HT, f16_t>::value ? PARTS : 1;
    constexpr int D = ring_depth<RING, FP8, RT, NT, PARTS>();
    f32x4_t acc[SUMS][RT][NT];
#pragma unroll
    for (int q = 0; q < SUMS; ++q)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[q][r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    lines<HT, FP8, RT, NT, PARTS, SUMS, D>(acc, wr, woff, rb, hr, xoff, hb, pl, sc, l0, l1, ring);
    join_parts(acc);
    join_waves<WK, RT * NT>(&acc[0][0][0], red, wk, lane, [&](int q, const f32x4_t& s) {
        const int r = q / NT, n = q - r * NT;
        const int c = c0 + 16 * r + 4 * g;
        // d is a multiple of 4: a lane's four columns are all in or all out
        if (16 * n + row < m && c < d)
            put_z<HT>(z, list[16 * n + row], d, c, hs, s);
    });
}

template <typename HT, bool FP8, int PARTS, int RING, int WK, int WR, int RT>
__global__ __launch_bounds__(WK * WR * 64) void moe_down(
    const HT* __restrict__ H, int d, const int32_t* __restrict__ ids, int npairs,
    const uint8_t* __restrict__ down, const float* __restrict__ scales, int E, int I, int by_pair,
    const float* __restrict__ hs, float* __restrict__ z) {
    extern __shared__ uint16_t list[];
    constexpr int W = WK * WR;
    constexpr int MT = max_tiles<RING, FP8, RT, PARTS>();
    __shared__ __align__(1024) char rings[W * RING];
    __shared__ int cnt[W];
    int e;
    const int m = expert_pairs<W>(ids, npairs, E, blockIdx.y, by_pair, e, list, cnt);
    if (m == 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave / WK, wk = wave - wr * WK;
    constexpr int WB = FP8 ? 1 : (int)sizeof(HT);
    const uint8_t* dn = down + (int64_t)e * d * I * WB;
    const float* ds = FP8 ? scales + (int64_t)e * ((d + 127) / 128) * ((I + 127) / 128) : nullptr;
    const int c0 = (blockIdx.x * WR + wr) * 16 * RT;
    const int64_t plane = (int64_t)npairs * I;
    char* const ring = rings + wave * RING;
    f32x4_t* const red = reinterpret_cast<f32x4_t*>(rings + wr * WK * RING);
    for (int c = 0; c < m; c += 16 * MT) {
        const int mc = min(m - c, 16 * MT);
        auto pass = [&](auto tiles) {
            down_pass<HT, FP8, PARTS, RING, WK, RT, decltype(tiles)::value>(
                H, plane, d, dn, ds, I, c0, list + c, mc, hs, z, wk, ring, red);
        };
        if (mc <= 16)
            pass(std::integral_constant<int, 1>());
        else if (MT < 4 || mc <= 32)
            pass(std::integral_constant<int, MT < 2 ? MT : 2>());
        else
            pass(std::integral_constant<int, MT>());
    }
}

// ---- many tokens an expert: waves that share the tokens' operand --------------------------------
// acc as for lines(), of RT row tiles of each of W waves over all lines of K. A stage holds every
// wave's rows and, once, the token operand, of which each wave loads its share; S stages. One
// barrier a line: past it every wave's loads of the line have landed, and the stage of the line
// before is free.
template <bool FP8, int RT, int NT, int PARTS, int W>
constexpr int wide_stage() {
    return W * 2 * RT + 2 * NT * PARTS * (FP8 ? 2 : 1);
}
template <typename XT, bool FP8, int RT, int NT, int PARTS, int SUMS, int W, int S>
__device__ __forceinline__ void wide_lines(f32x4_t (&acc)[SUMS][RT][NT], __amdgpu_buffer_rsrc_t wr,
                                           const int (&woff)[RT][2], int rb,
                                           __amdgpu_buffer_rsrc_t xr, const uint16_t* list, int m,
                                           int div, int xb, int plane,
                                           const float* const (&sc)[RT], int nl, char* lds) {
    using C = Core<XT, FP8>;
    constexpr int XC = C::XC, XL = 2 * NT * PARTS * XC / W;  // token loads of a wave
    constexpr int LPW = 2 * RT + XL, STAGE = wide_stage<FP8, RT, NT, PARTS, W>() * 1024;
    static_assert(XL * W == 2 * NT * PARTS * XC && (S - 2) * LPW <= 63, "loads");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int lcol = ((lane & 7) ^ lr) * 16;
    // token load q of the stage: 8 tokens (half h of tile n), part p, 128 bytes c of their columns
    int xo[XL], xc[XL], xp[XL];
#pragma unroll
    for (int u = 0; u < XL; ++u) {
        const int q = wave * XL + u, h = q & 1, c = (q >> 1) % XC, p = (q >> 1) / XC % PARTS;
        const int n = (q >> 1) / (XC * PARTS), t = 16 * n + 8 * h + lr;
        xo[u] = t < m ? (int)list[t] / div * xb + lcol : kOOB;
        xc[u] = c * kLine;
        xp[u] = p * plane;
    }
    auto load = [&](int l, char* at) {
        const bool in = (l < nl) & (l * kLine + lcol < rb);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                load_lds16<kNonTemporal>(wr, at + (wave * 2 * RT + 2 * r + h) * 1024,
                                         (in & (woff[r][h] >= 0)) ? woff[r][h] + lcol : kOOB,
                                         l * kLine);
#pragma unroll
        for (int u = 0; u < XL; ++u) {
            const int o = l * XC * kLine + xc[u];
            load_lds16(xr, at + (W * 2 * RT + wave * XL + u) * 1024,
                       ((l < nl) & (o + lcol < xb) & (xo[u] >= 0)) ? xo[u] : kOOB, xp[u] + o);
        }
    };
#pragma unroll
    for (int d = 0; d < S - 1; ++d) load(d, lds + d * STAGE);
    const uint32_t base = lds_addr(lds) + i * kLine;
    const uint32_t a0 = base + wave * 2048 * RT + (g ^ (i & 7)) * 16;
    const uint32_t a1 = base + wave * 2048 * RT + ((4 + g) ^ (i & 7)) * 16;
    const uint32_t xbase = base + W * 2048 * RT;
    const uint32_t x0 = xbase + (XC == 1 ? (g ^ (i & 7)) : ((2 * g) ^ (i & 7))) * 16;
    const uint32_t x1 = xbase + (XC == 1 ? ((4 + g) ^ (i & 7)) : ((2 * g + 1) ^ (i & 7))) * 16;
    int cur = 0, free = S - 1;
    for (int l = 0; l < nl; ++l) {
        wait_vm_lds<(S - 2) * LPW>();
        wg_barrier();
        load(l + S - 1, lds + free * STAGE);
        free = cur;
        const uint32_t at = cur * STAGE;
        cur = cur + 1 == S ? 0 : cur + 1;
        V16 a[RT][2], b[NT * PARTS * XC][2];
        lds_tiles<RT, 0>(a0 + at, a1 + at, a);
        lds_tiles<NT * PARTS * XC, 0>(x0 + at, x1 + at, b);
        line_product<XT, FP8, RT, NT, PARTS, SUMS>(acc, a, b, sc, l);
    }
    wait_vm_lds<0>();
    __syncthreads();  // the stages are free again
}

constexpr int kWide = 4, kWideStages = 3;  // waves

// most token tiles a pass, by the LDS that three stages of them take
template <bool FP8, int PARTS>
constexpr int wide_tiles() {
    return FP8 ? (PARTS == 3 ? 2 : 4) : (PARTS == 3 ? 4 : 8);
}
// LDS that the two kernels take beside the pairs' list (1 KB: counts, and what __syncthreads_or
// keeps there)
template <bool FP8, int PARTS>
constexpr size_t wide_lds() {
    constexpr int g = wide_stage<FP8, 4, wide_tiles<FP8, 1>(), 1, kWide>();
    constexpr int h = wide_stage<FP8, 2, wide_tiles<FP8, PARTS>(), PARTS, kWide>();
    return (size_t)(kWideStages * (g > h ? g : h) + 1) * 1024;
}

// m pairs in passes of up to NTM tiles, the fewest tiles of 2, 4 and 8 that hold a pass:
// pass(tiles, first pair, pairs)
template <int NTM, typename F>
__device__ __forceinline__ void wide_passes(int m, F pass) {
    for (int c = 0; c < m; c += 16 * NTM) {
        const int mc = min(m - c, 16 * NTM);
        if (NTM == 2 || mc <= 32)
            pass(std::integral_constant<int, 2>(), c, mc);
        else if (NTM == 4 || mc <= 64)
            pass(std::integral_constant<int, NTM < 4 ? NTM : 4>(), c, mc);
        else
            pass(std::integral_constant<int, NTM>(), c, mc);
    }
}

// Work-group: 64 NR neurons (16 NR a wave) of one expert. NR = 1 takes passes of up to 64 tokens in
// 72 KB of LDS, so that two work-groups share a CU; NR = 2 of up to 128 (8-bit weights 64).

template <typename XT, bool FP8, int NR, int NT, int S>
__device__ __forceinline__ void gate_up_wide_pass(
    const XT* x, int64_t xbytes, int d, int k, const uint8_t* gu, const float* gus, int I, int n0,
    const uint16_t* list, int m, typename GateOut<XT, FP8>::type* H, int64_t plane, int parts,
    char* lds) {
    constexpr int RT = 2 * NR;
    const int lane = threadIdx.x & 63;
    const int row = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int rb = d * (FP8 ? 1 : (int)sizeof(XT));
    int woff[RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int j = n0 + 16 * (r >> 1) + 8 * h + lr;
            woff[r][h] = j < I ? ((r & 1) * I + j) * rb : kOOB;
        }
    const int nl = (rb + kLine - 1) / kLine, nb = (I + 127) / 128;
    const float* sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        sc[r] = FP8 ? gus + (int64_t)((r & 1) * nb + min(n0 + 16 * (r >> 1), I - 1) / 128) * nl
                    : nullptr;
    f32x4_t acc[1][RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[0][r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    wide_lines<XT, FP8, RT, NT, 1, 1, kWide, S>(
        acc, make_rsrc(gu, (int64_t)2 * I * rb), woff, rb, make_rsrc(x, xbytes), list, m, k,
        d * (int)sizeof(XT), 0, sc, nl, lds);
#pragma unroll
    for (int q = 0; q < NR * NT; ++q) {
        const int nr = q / NT, n = q - nr * NT;
        if (16 * n + row < m) {
            const int64_t pair = list[16 * n + row];
            const int j = n0 + 16 * nr + 4 * g;
            f32x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                h[e] = silu_f32(acc[0][2 * nr][n][e]) * acc[0][2 * nr + 1][n][e];
            if (j < I) put_h4(h, pair * I + j, plane, parts, H);
        }
    }
}

template <typename XT, bool FP8, int NR>
__global__ __launch_bounds__(kWide * 64) void moe_gate_up_wide(
    const XT* __restrict__ x, int64_t T, int d, const int32_t* __restrict__ ids, int npairs, int k,
    const uint8_t* __restrict__ gate_up, const float* __restrict__ scales, int E, int I,
    int by_pair, typename GateOut<XT, FP8>::type* __restrict__ H, int parts) {
    extern __shared__ uint16_t list[];
    constexpr int NTM = NR == 1 ? 4 : wide_tiles<FP8, 1>(), S = kWideStages;
    __shared__ __align__(1024) char lds[S * wide_stage<FP8, 2 * NR, NTM, 1, kWide>() * 1024];
    __shared__ int cnt[kWide];
    int e;
    const int m = expert_pairs<kWide>(ids, npairs, E, blockIdx.y, by_pair, e, list, cnt);
    if (m == 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int WB = FP8 ? 1 : (int)sizeof(XT);
    const uint8_t* gu = gate_up + (int64_t)e * 2 * I * d * WB;
    const int nb = (I + 127) / 128;
    const float* gs = FP8 ? scales + (int64_t)e * 2 * nb * ((d + 127) / 128) : nullptr;
    const int n0 = (blockIdx.x * kWide + wave) * 16 * NR;
    const int64_t plane = (int64_t)npairs * I, xb = T * d * (int64_t)sizeof(XT);
    wide_passes<NTM>(m, [&](auto tiles, int c, int mc) {
        gate_up_wide_pass<XT, FP8, NR, decltype(tiles)::value, S>(x, xb, d, k, gu, gs, I, n0,
                                                                  list + c, mc, H, plane, parts,
                                                                  lds);
    });
}

// Work-group: 128 rows (32 a wave) of one expert's down matrix.
template <typename HT, bool FP8, int PARTS, int NT, int S>
__device__ __forceinline__ void down_wide_pass(const HT* H, int64_t plane, int d, const uint8_t* dn,
                                               const float* dns, int I, int c0,
                                               const uint16_t* list, int m, const float* hs,
                                               float* z, char* lds) {
    constexpr int RT = 2, SUMS = std::is_same<HT, f16_t>::value ? PARTS : 1;
    const int lane = threadIdx.x & 63;
    const int row = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int rb = I * (FP8 ? 1 : (int)sizeof(HT));
    int woff[RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int c = c0 + 16 * r + 8 * h + lr;
            woff[r][h] = c < d ? c * rb : kOOB;
        }
    const int nl = (rb + kLine - 1) / kLine;
    const float* sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        sc[r] = FP8 ? dns + (int64_t)(min(c0 + 16 * r, d - 1) / 128) * nl : nullptr;
    f32x4_t acc[SUMS][RT][NT];
#pragma unroll
    for (int q = 0; q < SUMS; ++q)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[q][r][n] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    wide_lines<HT, FP8, RT, NT, PARTS, SUMS, kWide, S>(
        acc, make_rsrc(dn, (int64_t)d * rb), woff, rb,
        make_rsrc(H, (int64_t)PARTS * plane * sizeof(HT)), list, m, 1, I * (int)sizeof(HT),
        (int)(plane * sizeof(HT)), sc, nl, lds);
    join_parts(acc);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int c = c0 + 16 * r + 4 * g;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // d is a multiple of 4: a lane's four columns are all in or all out
            if (16 * n + row < m && c < d)
                put_z<HT>(z, list[16 * n + row], d, c, hs, acc[0][r][n]);
        }
    }
}

template <typename HT, bool FP8, int PARTS>
__global__ __launch_bounds__(kWide * 64) void moe_down_wide(
    const HT* __restrict__ H, int d, const int32_t* __restrict__ ids, int npairs,
    const uint8_t* __restrict__ down, const float* __restrict__ scales, int E, int I, int by_pair,
    const float* __restrict__ hs, float* __restrict__ z) {
    extern __shared__ uint16_t list[];
    constexpr int NTM = wide_tiles<FP8, PARTS>(), S = kWideStages;
    __shared__ __align__(1024) char lds[S * wide_stage<FP8, 2, NTM, PARTS, kWide>() * 1024];
    __shared__ int cnt[kWide];
    int e;
    const int m = expert_pairs<kWide>(ids, npairs, E, blockIdx.y, by_pair, e, list, cnt);
    if (m == 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint8_t* dn = down + (int64_t)e * d * I * (FP8 ? 1 : (int)sizeof(HT));
    const float* ds = FP8 ? scales + (int64_t)e * ((d + 127) / 128) * ((I + 127) / 128) : nullptr;
    const int c0 = (blockIdx.x * kWide + wave) * 32;
    const int64_t plane = (int64_t)npairs * I;
    wide_passes<NTM>(m, [&](auto tiles, int c, int mc) {
        down_wide_pass<HT, FP8, PARTS, decltype(tiles)::value, S>(H, plane, d, dn, ds, I, c0,
                                                                  list + c, mc, hs, z, lds);
    });
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

// ---- one token -------------------------------------------------------------------------------
// The token's operand lies in LDS, and every MFMA column holds it: a lane reads its chunks without
// regard to its column, and column 0 is the result. So only weights pass through the waves' rings.
// most LDS that the operand may take (x: two work-groups share a CU)
constexpr int kOneH = 48 * 1024, kOneX = 8 * 1024;
constexpr int one_pitch(int64_t n, int bytes) { return (int)((n * bytes + 1023) / 1024 * 1024); }

// n bytes of row `pr` of a matrix of rows of rb bytes to LDS, in whole KB with zeros behind: the
// KBs q, q + W, ... of `rows` such rows, for wave q of W
template <int W>
__device__ __forceinline__ void stage_rows(__amdgpu_buffer_rsrc_t r, int rows, int rb, int pitch,
                                           char* to, int wave, int lane) {
    const int kbs = pitch >> 10;
    for (int q = wave; q < rows * kbs; q += W) {
        const int pr = q / kbs, o = (q - pr * kbs) * 1024 + lane * 16;
        load_lds16(r, to + q * 1024, o < rb ? pr * rb + o : kOOB, 0);
    }
}

// acc[r][p] += the product of RT row tiles and part p of the token over the lines [l0, l1).
// hbase: LDS address of this lane's chunk of line 0 of part 0, parts `ppitch` apart; staged() is
// called once the first D lines' loads are issued. The rest as for lines().
template <typename XT, bool FP8, int RT, int PARTS, int D, typename F>
__device__ __forceinline__ void lines_one(f32x4_t (&acc)[RT][PARTS], __amdgpu_buffer_rsrc_t wr,
                                          const int (&woff)[RT][2], int rb, uint32_t hbase,
                                          int ppitch, const float* const (&sc)[RT], int l0, int l1,
                                          char* ring, F staged) {
    using C = Core<XT, FP8>;
    constexpr int XC = C::XC, L = 2 * RT;
    static_assert((D - 1) * L <= 63, "outstanding loads");
    const int lane = threadIdx.x & 63;
    const int i = lane & 15, g = lane >> 4;
    const int lcol = ((lane & 7) ^ (lane >> 3)) * 16;
    auto load = [&](int l, char* at) {
        const bool in = (l < l1) & (l * kLine + lcol < rb);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                load_lds16<kNonTemporal>(wr, at + (2 * r + h) * 1024,
                                         (in & (woff[r][h] >= 0)) ? woff[r][h] + lcol : kOOB,
                                         l * kLine);
    };
#pragma unroll
    for (int t = 0; t < D; ++t) load(l0 + t, ring + t * L * 1024);
    staged();
    const uint32_t base = lds_addr(ring) + i * kLine;
    const uint32_t a0 = base + (g ^ (i & 7)) * 16, a1 = base + ((4 + g) ^ (i & 7)) * 16;
    int slot = 0;
    for (int l = l0; l < l1; ++l) {
        wait_vm_lds<(D - 1) * L>();
        V16 a[RT][2], b[PARTS][XC][2];
        lds_tiles<RT, 0>(a0 + slot * L * 1024, a1 + slot * L * 1024, a);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const uint32_t at = hbase + p * ppitch + l * kLine * XC;
            if constexpr (XC == 1) {
                lds_tiles<1, 0>(at, at + 64, b[p]);
            } else {
                lds_tiles<1, 0>(at, at + 16, b[p]);
                lds_tiles<1, 128>(at, at + 16, b[p] + 1);
            }
        }
        load(l + D, ring + slot * L * 1024);
        slot = slot + 1 == D ? 0 : slot + 1;
        f32x4_t blk[RT][PARTS];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) blk[r][p] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                typename C::vec w[XC];
                C::widen(a[r][h], w);
#pragma unroll
                for (int c = 0; c < XC; ++c)
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) {
                        f32x4_t& t = FP8 ? blk[r][p] : acc[r][p];
                        t = C::mma(w[c], XC == 1 ? b[p][0][h] : b[p][h * (XC - 1)][c], t);
                    }
            }
        if (FP8) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float s = sc[r][l];
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[r][p][e] = fmaf(s, blk[r][p][e], acc[r][p][e]);
            }
        }
    }
    wait_vm_lds<0>();  // the ring is free again
}

// Gate and up, SiLU(g) * u -> h. Work-group: 16 neurons of the expert of one rank, K split over 4
// waves. With CHOOSE each work-group makes the token's choice itself, from the logits (the first
// one also writes ids and weights): the same arithmetic in each, and a launch less.
// (8 of 128 experts: 28.2 us a layer with a choice kernel, 25.6 without. Above 256 experts the
// comparisons, E^2 / 256 a thread, would take longer than the launch they save.)
constexpr int kOneMaxE = 256;

template <typename XT, bool FP8, bool CHOOSE>
__global__ __launch_bounds__(256) void moe_gate_up_one(
    const XT* __restrict__ x, int d, Choice choice, int32_t* __restrict__ ids,
    float* __restrict__ weights, int k, const uint8_t* __restrict__ gate_up,
    const float* __restrict__ scales, int E, int I, typename GateOut<XT, FP8>::type* __restrict__ H,
    int parts) {
    constexpr int W = 4, D = 4, RT = 2;
    __shared__ __align__(1024) char rings[W * D * 2 * RT * 1024];
    __shared__ ChoiceLds<CHOOSE ? kOneMaxE : 1> cs;
    extern __shared__ __align__(1024) char hs[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int r = blockIdx.y, n0 = blockIdx.x * 16;
    constexpr int WB = FP8 ? 1 : (int)sizeof(XT);
    const int rb = d * WB, xb = d * (int)sizeof(XT);
    stage_rows<W>(make_rsrc(x, xb), 1, xb, one_pitch(d, sizeof(XT)), hs, wave, lane);
    int e;
    if constexpr (CHOOSE) {
        choose_experts<kOneMaxE>(choice, 0, blockIdx.x == 0 && r == 0, ids, weights, cs);
        e = __builtin_amdgcn_readfirstlane(cs.id[r]);
    } else {
        e = __builtin_amdgcn_readfirstlane(ids[r]);
    }
    if ((unsigned)e >= (unsigned)E) {
        wait_vm_lds<0>();  // no load may land in LDS after the work-group's end
        return;
    }
    const int nl = (rb + kLine - 1) / kLine, nb = (I + 127) / 128;
    const auto wr = make_rsrc(gate_up + (int64_t)e * 2 * I * rb, (int64_t)2 * I * rb);
    int woff[RT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = n0 + 8 * h + lr;
        woff[0][h] = j < I ? j * rb : kOOB;
        woff[1][h] = j < I ? (I + j) * rb : kOOB;
    }
    const float* sc[RT];
    sc[0] = FP8 ? scales + ((int64_t)e * 2 * nb + n0 / 128) * nl : nullptr;
    sc[1] = FP8 ? sc[0] + (int64_t)nb * nl : nullptr;
    int l0, l1;
    wave_lines<W>(nl, wave, l0, l1);
    f32x4_t acc[RT][1];
#pragma unroll
    for (int q = 0; q < RT; ++q) acc[q][0] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    lines_one<XT, FP8, RT, 1, D>(acc, wr, woff, rb, lds_addr(hs) + (FP8 ? 32 * g : 16 * g), 0, sc,
                                 l0, l1, rings + wave * D * 2 * RT * 1024, [&]() {
                                     // every wave's part of x has landed (the weights may fly)
                                     wait_vm_lds<D * 2 * RT>();
                                     wg_barrier();
                                 });
    f32x4_t* const red = reinterpret_cast<f32x4_t*>(rings);
    __syncthreads();  // the rings are done with
    if (row == 0) {
        red[(wave * 2) * 4 + g] = acc[0][0];
        red[(wave * 2 + 1) * 4 + g] = acc[1][0];
    }
    __syncthreads();
    // thread j: neuron n0 + j
    const int j = threadIdx.x;
    if (j < 16 && n0 + j < I) {
        const float* f = reinterpret_cast<const float*>(red);
        float sg = f[j], su = f[16 + j];
#pragma unroll
        for (int w = 1; w < W; ++w) {
            sg += f[w * 32 + j];
            su += f[w * 32 + 16 + j];
        }
        put_h(silu_f32(sg) * su, (int64_t)r * I + n0 + j, (int64_t)k * I, parts, H);
    }
}

// Down and the weighted sum. Work-group: 16 rows of every chosen expert's down matrix (16 columns
// of y). A wave takes an expert, or one of kc runs of K of it where there are fewer experts than
// waves; the waves' sums are weighted and added in order, and y is written at once. (With h in the
// rings too, as for more tokens, 10.3 us where this takes 7.6: 8 experts of 768 x 2048.)
constexpr int kOneWaves = 8;

template <typename HT, bool FP8, int PARTS, typename YT>
__global__ __launch_bounds__(kOneWaves * 64) void moe_down_one(
    const HT* __restrict__ H, const float* __restrict__ hscale, int d,
    const int32_t* __restrict__ ids, const float* __restrict__ weights, int k, int kc,
    const uint8_t* __restrict__ down, const float* __restrict__ scales, int E, int I,
    YT* __restrict__ y) {
    constexpr int D = 6;
    __shared__ __align__(1024) char rings[kOneWaves * D * 2 * 1024];
    extern __shared__ __align__(1024) char hs[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4, lr = lane >> 3;
    const int c0 = blockIdx.x * 16;
    constexpr int WB = FP8 ? 1 : (int)sizeof(HT);
    const int rb = I * WB, hb = I * (int)sizeof(HT), pitch = one_pitch(I, sizeof(HT));
    const int nl = (rb + kLine - 1) / kLine, per = (nl + kc - 1) / kc;
    // row r of part p of h at (p k + r) pitch
    stage_rows<kOneWaves>(make_rsrc(H, (int64_t)PARTS * k * I * sizeof(HT)), PARTS * k, hb, pitch,
                          hs, wave, lane);
    const int woff[1][2] = {{c0 + lr < d ? (c0 + lr) * rb : kOOB,
                             c0 + 8 + lr < d ? (c0 + 8 + lr) * rb : kOOB}};
    bool ready = false;
    f32x4_t tot = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int u = wave; u < k * kc; u += kOneWaves) {
        const int r = u / kc, q = u - r * kc;
        const int e = __builtin_amdgcn_readfirstlane(ids[r]);
        const bool some = (unsigned)e < (unsigned)E;
        const int ex = some ? e : 0;
        const auto wr = make_rsrc(down + (int64_t)ex * d * rb, (int64_t)d * rb);
        const float* sc[1] = {
            FP8 ? scales + ((int64_t)ex * ((d + 127) / 128) + c0 / 128) * nl : nullptr};
        const int l0 = min(nl, q * per), l1 = some ? min(nl, l0 + per) : l0;
        f32x4_t acc[1][PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) acc[0][p] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        lines_one<HT, FP8, 1, PARTS, D>(acc, wr, woff, rb,
                                        lds_addr(hs) + r * pitch + (FP8 ? 32 * g : 16 * g),
                                        k * pitch, sc, l0, l1, rings + wave * D * 2 * 1024, [&]() {
                                            if (ready) return;
                                            // every wave's part of h has landed
                                            wait_vm_lds<D * 2>();
                                            wg_barrier();
                                            ready = true;
                                        });
        if (some) {
            const float f = weights[r];
            if constexpr (std::is_same<HT, f16_t>::value) {
                const float back = hscale[r];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    tot[i] = fmaf(f, fmaf(kLoDown, acc[0][1][i], acc[0][0][i]) * back, tot[i]);
            } else {
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) tot[i] = fmaf(f, acc[0][p][i], tot[i]);
            }
        }
    }
    if (!ready) {  // a wave without work meets the same barrier, its part of h landed
        wait_vm_lds<0>();
        wg_barrier();
    }
    f32x4_t* const red = reinterpret_cast<f32x4_t*>(rings);
    __syncthreads();  // the rings are done with
    if (row == 0) red[wave * 4 + g] = tot;
    __syncthreads();
    // thread g: columns 4 g .. (d is a multiple of 4)
    if (threadIdx.x < 4 && c0 + 4 * (int)threadIdx.x < d) {
        f32x4_t s = red[threadIdx.x];
#pragma unroll
        for (int w = 1; w < kOneWaves; ++w) {
            const f32x4_t v = red[w * 4 + threadIdx.x];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += v[i];
        }
        const float o[4] = {s[0], s[1], s[2], s[3]};
        put4(y + c0 + 4 * threadIdx.x, o);
    }
}

struct Plan {
    int64_t pairs;
    int parts, hbytes;  // parts of h and bytes of an element of one
    size_t off_z, off_h, off_s, total;  // (half weights: h in float32, and the pairs' scales)
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
    p.off_h = p.off_z + ((size_t)p.pairs * d * sizeof(float) + 255) / 256 * 256;
    const bool half = xdt == 2 && wdt == 2;
    p.off_s = p.off_h + (half ? ((size_t)p.pairs * I * sizeof(float) + 255) / 256 * 256 : 0);
    p.total = p.off_s + (half ? (size_t)p.pairs * sizeof(float) : 0);
    return p;
}

struct Args {
    const void* x;
    int64_t T, d;
    int32_t* ids;
    float* w;
    int64_t k;
    const uint8_t* gate_up;
    const float* gus;
    const uint8_t* down;
    const float* dns;
    int64_t E, I;
    void* y;
    int ydt;
    void* ws;
    Plan p;
    const Choice* choice;
    hipStream_t s;
};

template <typename YT>
void sum(const Args& a, YT* y) {
    const float* z = reinterpret_cast<const float*>(static_cast<char*>(a.ws) + a.p.off_z);
    moe_sum<YT><<<dim3((unsigned)((a.d + 1023) / 1024), (unsigned)a.T), 256, 0, a.s>>>(
        z, a.ids, a.w, (int)a.k, (int)a.E, (int)a.d, y);
}

// Lines of a weight row from which it counts as long: more waves then share one row group, so that
// fewer work-groups take more of a row at a time (48 tokens over 8 experts of 14336 x 4096: gate
// and up by 4 waves 525 us a layer, by 2 542; down by 2 518, by 1 541; 13 tokens over 8-bit experts
// with rows of 1408, 11 lines: down by 1 wave 159, by 2 187).
constexpr int kLongRow = 64;

// Pairs an expert from which the tokens' operand weighs: waves that share it, instead of each
// loading it for its own rows. Microseconds by the kernels of few and of many tokens:
//   8 experts of 14336 x 4096, bf16: 12 pairs each 472 and 494, 16: 512 and 496, 32: 862 and 530;
//   128 of 768 x 2048, bf16: 8: 253 and 251, 12: 284 and 262, 16: 315 and 272
//   64 of 1408 x 4096, 8-bit: 9: 253 and 270, 12: 280 and 275, 18: 356 and 294, 37: 703 and 379
//   half, 8 of 8192 x 4096: 12: 279 and 314, 16: 296 and 318, 32: 495 and 326;  64 of 1024 x 1024:
//     12: 114 and 87
// One number for every shape, right for rows of kLongRow lines and more; below, layers of 8 to 16
// pairs an expert lose by it (12 pairs: 8% and 31% above). float32 weights have no such kernels: 200
// tokens, 2 of 16 experts of 2048 x 2048 take 211 us, their bytes 155.
constexpr int64_t kManyPairs = 16;

// Pairs an expert up to which gate and up take two work-groups a CU and passes of 64 tokens: 8
// experts of 14336 x 4096, 24 pairs 483 us, by wider ones 522; 48: 549 and 571; 64, where half of
// the experts take two passes: 819 and 682. (8-bit weights: no difference. Down with two
// work-groups a CU, by half the rows or two stages: from 6% less to 18% more.)
constexpr int64_t kWidePairs = 48;

template <typename XT, bool FP8, int PARTS>
void experts(const Args& a) {
    typedef typename HType<XT, FP8>::type HT;
    typedef typename GateOut<XT, FP8>::type GT;
    constexpr bool HALF = std::is_same<HT, f16_t>::value;
    HT* H = static_cast<HT*>(a.ws);
    float* z = reinterpret_cast<float*>(static_cast<char*>(a.ws) + a.p.off_z);
    // what gate and up write
    GT* G = reinterpret_cast<GT*>(static_cast<char*>(a.ws) + (HALF ? a.p.off_h : 0));
    float* hs = reinterpret_cast<float*>(static_cast<char*>(a.ws) + a.p.off_s);
    const int np = (int)a.p.pairs;
    // fewer pairs than experts: a slot a pair, so that no work-group is without an expert but
    // those of repeated ones; else a slot an expert
    const int by_pair = np <= a.E;
    const unsigned slots = (unsigned)(by_pair ? np : a.E);
    const size_t lds = ((size_t)np * sizeof(uint16_t) + 15) / 16 * 16;
    const int gl = (int)((a.d * (FP8 ? 1 : (int)sizeof(XT)) + kLine - 1) / kLine);
    const int dl = (int)((a.I * (FP8 ? 1 : (int)sizeof(HT)) + kLine - 1) / kLine);
    constexpr bool kMany = sizeof(XT) == 2;
    // (lists of more than 7680 pairs do not fit beside the stages of 8-bit weights)
    const bool many =
        kMany && (int64_t)np >= kManyPairs * a.E && wide_lds<FP8, PARTS>() + lds <= 160 * 1024;
    const XT* x = static_cast<const XT*>(a.x);
    const int64_t xlds = one_pitch(a.d, sizeof(XT));
    if (a.T == 1 && xlds <= kOneX) {
        const dim3 grid((unsigned)((a.I + 15) / 16), (unsigned)a.k);
        if (a.choice)
            moe_gate_up_one<XT, FP8, true><<<grid, 256, (size_t)xlds, a.s>>>(
                x, (int)a.d, *a.choice, a.ids, a.w, (int)a.k, a.gate_up, a.gus, (int)a.E, (int)a.I,
                G, a.p.parts);
        else
            moe_gate_up_one<XT, FP8, false><<<grid, 256, (size_t)xlds, a.s>>>(
                x, (int)a.d, Choice{}, a.ids, a.w, (int)a.k, a.gate_up, a.gus, (int)a.E, (int)a.I,
                G, a.p.parts);
    } else {
        auto gate = [&](auto kernel, int rows, int threads) {
            kernel<<<dim3((unsigned)((a.I + rows - 1) / rows), slots), threads, lds, a.s>>>(
                x, a.T, (int)a.d, a.ids, np, (int)a.k, a.gate_up, a.gus, (int)a.E, (int)a.I,
                by_pair, G, a.p.parts);
        };
        if (many) {
            if constexpr (FP8) {
                gate(moe_gate_up_wide<XT, true, 2>, 32 * kWide, kWide * 64);
            } else if constexpr (kMany) {
                if (np <= kWidePairs * a.E)
                    gate(moe_gate_up_wide<XT, false, 1>, 16 * kWide, kWide * 64);
                else
                    gate(moe_gate_up_wide<XT, false, 2>, 32 * kWide, kWide * 64);
            }
        } else if (gl >= kLongRow) {
            gate(moe_gate_up<XT, FP8, 16 * 1024, 4, 1>, 16, 256);
        } else {
            gate(moe_gate_up<XT, FP8, 24 * 1024, 2, 1>, 16, 128);
        }
    }
    if constexpr (HALF) {
        auto parts = [&](auto kernel, int threads) {
            kernel<<<dim3((unsigned)np), threads, 0, a.s>>>(G, a.ids, (int)a.E, (int)a.I,
                                                            (int64_t)np * a.I, H, hs);
        };
        // (rows up to 65536 values; short ones by the large work-group: 128 tokens, 6 of 64 experts
        // of 1024 x 1024 132 us instead of 124, one token, 8 of 768 x 2048 27.3 instead of 25.4)
        if (a.I <= 4096)
            parts(moe_h_parts<256, 4>, 256);
        else
            parts(moe_h_parts<1024, 16>, 1024);
    }
    // f(y) with y's type: bf16 parts number 3 for a float32 y and 2 for one of 16 bits
    auto to_y = [&](auto f) {
        constexpr bool kF32 = PARTS != 2 || HALF;
        if constexpr (PARTS == 2) {
            if (!kF32 || a.ydt != 0) return f(static_cast<XT*>(a.y));
        }
        if constexpr (kF32) f(static_cast<float*>(a.y));
    };
    const int64_t hlds = (int64_t)PARTS * a.k * one_pitch(a.I, sizeof(HT));
    if (a.T == 1 && hlds <= kOneH) {
        // one token: as many runs of K as keep the waves busy
        const int kc = a.k >= kOneWaves ? 1 : (int)(kOneWaves / a.k);
        const dim3 grid((unsigned)((a.d + 15) / 16));
        auto one = [&](auto* y) {
            typedef typename std::remove_pointer<decltype(y)>::type YT;
            moe_down_one<HT, FP8, PARTS, YT><<<grid, kOneWaves * 64, (size_t)hlds, a.s>>>(
                H, hs, (int)a.d, a.ids, a.w, (int)a.k, kc, a.down, a.dns, (int)a.E, (int)a.I, y);
        };
        to_y(one);
        return;
    }
    auto down = [&](auto kernel, int rows, int threads) {
        kernel<<<dim3((unsigned)((a.d + rows - 1) / rows), slots), threads, lds, a.s>>>(
            H, (int)a.d, a.ids, np, a.down, a.dns, (int)a.E, (int)a.I, by_pair, hs, z);
    };
    if (many) {
        if constexpr (kMany) down(moe_down_wide<HT, FP8, PARTS>, 32 * kWide, kWide * 64);
    } else if (dl >= kLongRow) {
        down(moe_down<HT, FP8, PARTS, 24 * 1024, 2, 2, 2>, 64, 256);
    } else {
        down(moe_down<HT, FP8, PARTS, 24 * 1024, 1, 2, 2>, 64, 128);
    }
    to_y([&](auto* y) { sum(a, y); });
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

bool moe_chooses(int64_t T, int64_t d, int64_t E, int xdt) {
    return T == 1 && E <= kOneMaxE && one_pitch(d, xdt == 0 ? 4 : 2) <= kOneX;
}

hipError_t launch_moe(const void* x, int xdt, int64_t T, int64_t d, int32_t* ids, float* w,
                      int64_t k, const void* gate_up, const float* gus, const void* down,
                      const float* dns, int64_t E, int64_t I, int wdt, void* y, int ydt, void* ws,
                      hipStream_t s, const Choice* choice) {
    const Args a{x, T, d, ids, w, k, static_cast<const uint8_t*>(gate_up), gus,
                 static_cast<const uint8_t*>(down), dns, E, I, y, ydt, ws,
                 moe_plan(T, k, d, I, xdt, wdt, ydt), choice, s};
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
    return hipGetLastError();
}

}  // namespace si
