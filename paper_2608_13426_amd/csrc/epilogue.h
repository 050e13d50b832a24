// The products' epilogue: Y = act(acc + bias[n]) + rs * R[m][n], evaluated in
// fp32 from the fp32 accumulator and rounded once to the output type.
#pragma once

#include <type_traits>

#include "device_common.h"

namespace rmm {

// act: the rmm_act values; bias, res: of the product's type, or null
struct Epilogue {
    const void *bias, *res;
    int64_t ldr;          // residual row stride (elements), units M * ldr apart
    float rs;
    int act;
};

// Y of a kernel that may have an epilogue (EP): it may then be the residual itself,
// which the same threads read through ep.res
template <bool EP, class T>
using OutPtr = std::conditional_t<EP, T *, T *__restrict__>;

constexpr int kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3, kActGeluTanh = 4;

// T: the output's type.  Where it is bf16 gelu's negative side a Phi(-a) is off by 3e-5
// of itself and the forms below by at most 3e-5 of their value (the rounding: 2^-8 of it),
// in as few operations as that takes: they run on every output of a tile while its matrix
// cores wait (8192 x 14336 outputs of 2048 retained indices: 406 us as a plain product,
// 428 with bias and silu).  fp32 gelu is 1 + erf: exact to the argument's size, not to its
// own where that is far smaller.
template <int ACT, class T>
__device__ __forceinline__ float activate(float x) {
    constexpr bool kFast = sizeof(T) == 2;
    if constexpr (ACT == kActRelu) return x < 0.f ? 0.f : x;          // NaN stays
    if constexpr (ACT == kActSilu) return x * __builtin_amdgcn_rcpf(1.f + __expf(-x));
    if constexpr (ACT == kActGelu && !kFast) return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
    if constexpr (ACT == kActGelu && kFast) {
        // x Phi(x) = max(x, 0) - a Phi(-a), a = |x|; log2 Phi(-a) as a polynomial of
        // degree 8, least largest error on [0, 10] (of Phi: 1.9e-5, with the fp32 steps'
        // rounding 2.8e-5); past 10, a Phi(-a) < 1e-22
        const float a = fminf(fabsf(x), 10.f);
        float p = 6.003541844e-08f;
        p = fmaf(p, a, -3.129991683e-06f);
        p = fmaf(p, a, 7.174348139e-05f);
        p = fmaf(p, a, -9.613548173e-04f);
        p = fmaf(p, a, 8.502015844e-03f);
        p = fmaf(p, a, -5.372728780e-02f);
        p = fmaf(p, a, -4.589110017e-01f);
        p = fmaf(p, a, -1.150986195f);
        p = fmaf(p, a, -1.000023842f);
        return fmaf(-a, __builtin_amdgcn_exp2f(p), x < 0.f ? 0.f : x);
    }
    // 0.5 x (1 + tanh u) = x / (1 + e^(-2u)),  u = sqrt(2/pi) (x + 0.044715 x^3)
    if constexpr (ACT == kActGeluTanh) {
        const float w = x * fmaf(x * x, -0.10294324f, -2.3022082f);   // -2 u log2(e)
        return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(w));
    }
    return x;
}

template <class T>
__device__ __forceinline__ float activate(float x, int act) {
    switch (act) {
    case kActRelu: return activate<kActRelu, T>(x);
    case kActSilu: return activate<kActSilu, T>(x);
    case kActGelu: return activate<kActGelu, T>(x);
    case kActGeluTanh: return activate<kActGeluTanh, T>(x);
    default: return x;
    }
}

// f(std::integral_constant<int, ACT>) for the call's activation: one uniform
// branch around it
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
    case kActRelu: f(std::integral_constant<int, kActRelu>{}); break;
    case kActSilu: f(std::integral_constant<int, kActSilu>{}); break;
    case kActGelu: f(std::integral_constant<int, kActGelu>{}); break;
    case kActGeluTanh: f(std::integral_constant<int, kActGeluTanh>{}); break;
    default: f(std::integral_constant<int, kActNone>{}); break;
    }
}

__device__ __forceinline__ float ep_load(const uint16_t *p, int64_t i) { return bf16_to_f32(p[i]); }
__device__ __forceinline__ float ep_load(const float *p, int64_t i) { return p[i]; }

// one output at column n; row: its row over all units
template <class T>
__device__ __forceinline__ float ep_value(const Epilogue &ep, float acc, int64_t row, int n) {
    if (ep.bias) acc += ep_load(static_cast<const T *>(ep.bias), n);
    acc = activate<T>(acc, ep.act);
    if (ep.res) acc = fmaf(ep.rs, ep_load(static_cast<const T *>(ep.res), row * ep.ldr + n), acc);
    return acc;
}

// 16 bytes at any address (global memory takes them at every alignment)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void ep_unpack(const u32x4_t &q, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(q[e] << 16);
        v[2 * e + 1] = __uint_as_float(q[e] & 0xffff0000u);
    }
}

// eight values at p, of which the first n exist
__device__ __forceinline__ u32x4_t ep_load8(const uint16_t *p, int n) {
    if (n >= 8) return *reinterpret_cast<const u32x4_any *>(p);
    u32x4_t q = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) q[e >> 1] |= static_cast<uint32_t>(p[e]) << (16 * (e & 1));
    return q;
}

// Where a pass's fp32 sum of row r and column n (of BN) lies in row r's LDS: 16-byte
// chunk cc = n / 4 at (cc / 2) ^ (r % 16) of the row's first or second half as cc is
// even or odd, so that both the fragments' writes and the rows' reads fall on
// distinct banks.
template <int BN>
constexpr int ep_swizzle = BN / 8 < 16 ? BN / 8 - 1 : 15;
template <int BN>
__device__ __forceinline__ char *ep_at(char *row, int r, int n) {
    const int cc = n >> 2;
    return row + 16 * (((cc >> 1) ^ (r & ep_swizzle<BN>)) + BN / 8 * (cc & 1)) + 4 * (n & 3);
}

// The epilogue of a tile of BN columns held as fp32 sums by NW waves, 2 x NW/2 of
// them, each TM rows of its own columns.  The sums go through LDS 64 rows at a time:
// put(p) writes, for rows r = 32 wm .. + 31 of pass p (tile rows wm * TM + 32 p ..),
// the wave's columns to ep_at(obj(r), r, n).  A thread then holds 8 neighbouring
// columns of a row: bias and residual come in 16 bytes a lane, one rounding, 16
// bytes out.  No access needs alignment; only the chunk that N cuts goes element by
// element.  (Residual added on the fragments, 8 bytes a lane in 32 rows, and outputs
// staged as bf16: 420 us for 8192 x 4096 of 7168 retained indices; so: 404.  With
// rows off 16-byte boundaries, 2 x 1001 x 4097 of 610, the same tiles: 111, 35.)
// Every wave's reads of the ring and loads into it have ended before the call.
// left: rows from the tile's origin on; row0: the origin's row over all units.
template <int BN, int NW, int PASSES, int TM, class Put, class Obj>
__device__ __forceinline__ void ep_tile(const Epilogue &ep, Put put, Obj obj, int wave, int lane, uint16_t *Y,
                                        int64_t ldy, bool aligned16, int n0, int N, int left, int64_t row0) {
    constexpr int LPR = BN / 8, RPI = 64 / LPR, Q = 64 / (NW * RPI);     // lanes per row, rows per step
    const int c = lane % LPR, nc = N - n0 - 8 * c;
    auto tile_row = [&](int r, int p) { return (r / 32) * TM + 32 * p + r % 32; };
    auto step_row = [&](int q) { return RPI * (NW * q + wave) + lane / LPR; };
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.f;
    if (ep.bias && nc > 0) ep_unpack(ep_load8(static_cast<const uint16_t *>(ep.bias) + n0 + 8 * c, nc), bias);
    const uint16_t *src = static_cast<const uint16_t *>(ep.res) + row0 * ep.ldr + n0 + 8 * c;
    uint16_t *dst = Y + row0 * ldy + n0 + 8 * c;
    u32x4_t res[Q];
    auto fetch = [&](int p) {
        if (!ep.res) return;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int ml = tile_row(step_row(q), p);
            if (ml < left && nc > 0) res[q] = ep_load8(src + ml * ep.ldr, nc);
        }
    };
    fetch(0);
    lds_barrier();
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        put(p);
        lds_barrier();
        u32x4_t now[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) now[q] = res[q];
        if (p + 1 < PASSES) fetch(p + 1);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int r = step_row(q), ml = tile_row(r, p);
            const f32x4_t lo = *reinterpret_cast<const f32x4_t *>(ep_at<BN>(obj(r), r, 8 * c));
            const f32x4_t hi = *reinterpret_cast<const f32x4_t *>(ep_at<BN>(obj(r), r, 8 * c + 4));
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = lo[e] + bias[e]; v[4 + e] = hi[e] + bias[4 + e]; }
            with_activation(ep.act, [&](auto A) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = activate<decltype(A)::value, uint16_t>(v[e]);
            });
            if (ep.res) {
                float add[8];
                ep_unpack(now[q], add);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(ep.rs, add[e], v[e]);
            }
            if (ml >= left || nc <= 0) continue;
            const u32x4_t out = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                 pack_bf16x2(v[6], v[7])};
            uint16_t *d = dst + ml * ldy;
            if (nc >= 8) {
                // whole lines go past L2 (streaming); pieces of lines are joined there
                if (aligned16) __builtin_nontemporal_store(out, reinterpret_cast<u32x4_t *>(d));
                else *reinterpret_cast<u32x4_any *>(d) = out;
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < nc) d[e] = static_cast<uint16_t>(out[e >> 1] >> (16 * (e & 1)));
            }
        }
        if (p + 1 < PASSES) lds_barrier();        // the next pass overwrites the staged rows
    }
}

// put() of the K-major kernels, whose fragments are transposed: acc[j][i][4*gq + r] is
// row wm*TM + 32i + lane%32 and column wn*32*FN + 32j + 8gq + 4*(lane/32) + r.
template <int BN, int NW, int FN, int FM, class Obj>
__device__ __forceinline__ void ep_put_rows(const f32x16_t (&acc)[FN][FM], int p, Obj obj, int wave, int lane) {
    const int wm = wave / (NW / 2), wn = wave % (NW / 2), r = 32 * wm + (lane & 31);
    char *o = obj(r);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq)
            *reinterpret_cast<f32x4_t *>(ep_at<BN>(o, r, 32 * (FN * wn + j) + 8 * gq + 4 * (lane >> 5))) =
                f32x4_t{acc[j][p][4 * gq], acc[j][p][4 * gq + 1], acc[j][p][4 * gq + 2], acc[j][p][4 * gq + 3]};
}

// and of the row-major ones: acc[i][j][v] is row wm*TM + 32i + 8*(v/4) + 4*(lane/32) +
// v%4 and column wn*32*FN + 32j + lane%32.
template <int BN, int NW, int FM, int FN, class Obj>
__device__ __forceinline__ void ep_put_columns(const f32x16_t (&acc)[FM][FN], int p, Obj obj, int wave, int lane) {
    const int wm = wave / (NW / 2), wn = wave % (NW / 2);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int r = 32 * wm + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
#pragma unroll
        for (int j = 0; j < FN; ++j)
            *reinterpret_cast<float *>(ep_at<BN>(obj(r), r, 32 * (FN * wn + j) + (lane & 31))) = acc[p][j][v];
    }
}

}  // namespace rmm
