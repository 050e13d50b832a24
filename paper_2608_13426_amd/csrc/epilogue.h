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
    int vec;              // bf16 bias and residual rows are 8-byte aligned
};

constexpr int kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3, kActGeluTanh = 4;

template <int ACT>
__device__ __forceinline__ float activate(float x) {
    if constexpr (ACT == kActRelu) return x < 0.f ? 0.f : x;          // NaN stays
    if constexpr (ACT == kActSilu) return x / (1.f + __expf(-x));
    if constexpr (ACT == kActGelu) return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
    // 0.5 x (1 + tanh u) = x / (1 + e^(-2u)),  u = sqrt(2/pi) (x + 0.044715 x^3)
    if constexpr (ACT == kActGeluTanh)
        return x / (1.f + __expf(-1.5957691216057308f * (x + 0.044715f * x * x * x)));
    return x;
}

__device__ __forceinline__ float activate(float x, int act) {
    switch (act) {
    case kActRelu: return activate<kActRelu>(x);
    case kActSilu: return activate<kActSilu>(x);
    case kActGelu: return activate<kActGelu>(x);
    case kActGeluTanh: return activate<kActGeluTanh>(x);
    default: return x;
    }
}

// f(std::integral_constant<int, ACT>) for the call's activation: one uniform
// branch around a whole pass over the accumulators
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
    acc = activate(acc, ep.act);
    if (ep.res) acc = fmaf(ep.rs, ep_load(static_cast<const T *>(ep.res), row * ep.ldr + n), acc);
    return acc;
}

// The same on the Y^T fragments of the K-major kernels: acc[j][i][4*gq + r] is
// row m = mrow + 32i + lane%32 and column n = ncol + 32j + 8gq + 4*(lane/32) + r.
// rows: how many rows are left from mrow's tile origin; row0: the tile origin's
// row over all units.
template <int FN, int FM>
__device__ __forceinline__ void ep_fragments(const Epilogue &ep, f32x16_t (&acc)[FN][FM], int lane, int mrow,
                                             int ncol, int rows, int64_t row0, int N) {
    const bool vec = ep.vec;
    const int lr = lane & 31, lh = lane >> 5;
    if (ep.bias) {
        const uint16_t *bias = static_cast<const uint16_t *>(ep.bias);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq) {
                const int n = ncol + 32 * j + 8 * gq + 4 * lh;
                float b[4];
                if (vec && n + 4 <= N) {
                    const uint2 v = *reinterpret_cast<const uint2 *>(bias + n);
                    b[0] = __uint_as_float(v.x << 16); b[1] = __uint_as_float(v.x & 0xffff0000u);
                    b[2] = __uint_as_float(v.y << 16); b[3] = __uint_as_float(v.y & 0xffff0000u);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) b[r] = n + r < N ? bf16_to_f32(bias[n + r]) : 0.f;
                }
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[j][i][4 * gq + r] += b[r];
            }
    }
    with_activation(ep.act, [&](auto A) {
        if constexpr (decltype(A)::value != kActNone) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[j][i][v] = activate<decltype(A)::value>(acc[j][i][v]);
        }
    });
    if (ep.res) {
        const uint16_t *res = static_cast<const uint16_t *>(ep.res) + row0 * ep.ldr;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m = mrow + 32 * i + lr;
            if (m >= rows) continue;
            const uint16_t *p = res + m * ep.ldr;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const int n = ncol + 32 * j + 8 * gq + 4 * lh;
                    if (vec && n + 4 <= N) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(p + n);
                        acc[j][i][4 * gq] = fmaf(ep.rs, __uint_as_float(v.x << 16), acc[j][i][4 * gq]);
                        acc[j][i][4 * gq + 1] = fmaf(ep.rs, __uint_as_float(v.x & 0xffff0000u), acc[j][i][4 * gq + 1]);
                        acc[j][i][4 * gq + 2] = fmaf(ep.rs, __uint_as_float(v.y << 16), acc[j][i][4 * gq + 2]);
                        acc[j][i][4 * gq + 3] = fmaf(ep.rs, __uint_as_float(v.y & 0xffff0000u), acc[j][i][4 * gq + 3]);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (n + r < N) acc[j][i][4 * gq + r] = fmaf(ep.rs, bf16_to_f32(p[n + r]), acc[j][i][4 * gq + r]);
                    }
                }
        }
    }
}

}  // namespace rmm
