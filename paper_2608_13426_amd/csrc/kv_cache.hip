// Per-head norm and position rotation of queries and keys, and the paged
// key/value cache: appending to it (the keys normed and rotated on the way) and
// reading tokens back.
//
//   y   = x * r * gamma,  r = 1 / sqrt(mean x^2 + eps)                 (optional)
//   out = pairs (a, b) of y -> (a cos - b sin, b cos + a sin), cos and sin of the
//         token's position and the pair's index; the dims past `rot` pass through
//
// One pass, bound by reading and writing each element once.  A head's D values
// lie in D / 16 lanes, two 8-element pieces per lane chosen so that a rotation
// pair never leaves its lane: no exchange but the norm's sum.  A wave takes
// 1024 / D heads of one token (they share its cos and sin), a workgroup four
// tokens at a time.  8192 tokens, 32 + 8 heads of 128 (168 MB read and written):
// 40 us, 4.2 TB/s, where a large copy moves 4.9; one token per sequence: 3 to 5 us.
//
// Numerics: the mean square and its root in float64 (squares of bf16 are exact
// there, so the order of the sum does not show), r rounded to fp32; every
// product and sum of the norm and the rotation rounded separately in fp32 (no
// fused multiply-add: the result is the same whatever the compiler fuses), one
// rounding to the stored type.  4-bit codes are made from the fp32 value.
//
// Column energies of the rotated queries (the score of the per-head
// selection): each lane keeps float64 sums of its 16 columns over its tokens,
// the workgroup's four waves are added in order, a second kernel adds the
// workgroups' sums in order.
#include <algorithm>

#include "device_common.h"
#include "kernels.h"
#include "kv_cache.h"

namespace rmm {

namespace {

constexpr int kThreads = 256, kWaves = 4;
// A grid holds fewer than 2^32 threads along an axis (a larger one is launched cut to
// its low 32 bits): workgroups past this many go on along z.
constexpr int kGridX = 1 << 22;

// ---- 8 elements of a head
template <typename T>
struct alignas(16) Raw8 {
    T x[8];
};
__device__ __forceinline__ void load8(const uint16_t *p, float (&x)[8]) {
    const uint4 q = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
// stores the rounded values and leaves them in x
__device__ __forceinline__ void store8(uint16_t *p, float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float *p, float (&x)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// ---- 4-bit groups (MXFP4: 32 elements, one power-of-two scale)
// scale byte of a group with largest magnitude amax: the smallest scale at
// which amax rounds to at most 6 (magnitudes from 7 on round to 8), kept in
// 8 .. 252 so that every value is a normal bf16; 255 (NaN) when amax is not finite
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    const int e = static_cast<int>(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) >= 0x600000u ? 1 : 0);
    return static_cast<uint32_t>(min(max(e, 8), 252));
}
// round to nearest, ties to the even code, magnitudes over 6 to 6
__device__ __forceinline__ uint32_t mx_codes8(const float (&x)[8], float scale) {
    uint32_t w = 0;
#if defined(__HIP_DEVICE_COMPILE__)
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
#endif
    return w;
}

struct Piece {
    int c1, c2, on;      // the lane's two 8-element pieces; whether they rotate with each other / inside
};
// Pieces of lane j of a head (D / 16 lanes).  Halves: pieces c and c + rot/16
// hold the pairs (i, i + rot/2).  Adjacent pairs lie inside a piece.  The rest
// is dealt out in order.
template <int D>
__device__ __forceinline__ Piece piece_of(int j, int rot, int interleaved) {
    const int h = interleaved ? D / 16 : rot / 16;
    if (interleaved || j < h) return {j, j + h, 1};
    const int n = D / 8 - 2 * h, r = j - h;
    return {2 * h + r, 2 * h + n / 2 + r, 0};
}

// 1 / sqrt(x) for x >= 0: the hardware's estimate and two Newton steps, within a
// few float64 roundings (its fp32 rounding is the correct one but for about one
// value in 2^27); 0 for infinity
__device__ __forceinline__ double rsqrt64(double x) {
#if defined(__HIP_DEVICE_COMPILE__)
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = fma(0.5 * r, fma(-x * r, r, 1.0), r);
    return __builtin_isinf(x) ? 0.0 : r;
#else
    return x;
#endif
}

__device__ __forceinline__ void turn(float &a, float &b, float c, float s) {
#pragma clang fp contract(off)
    const float x = a * c - b * s, y = b * c + a * s;
    a = x;
    b = y;
}

}  // namespace

// KV: 0 no cache, 1 bf16 cache, 2 4-bit cache
template <typename T, int D, int KV, bool NORM, bool ENERGY>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a, int TB, int64_t blocks) {
    constexpr int LPH = D / 16, VPW = 64 / LPH;            // lanes per head, heads per wave
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = lane % LPH, nv = a.q.n + a.k.n + a.v.n;
    const int vec = static_cast<int>(blockIdx.y) * VPW + lane / LPH;
    const bool act = vec < nv;
    // which list the lane's head is in
    const int kind = !act ? 3 : vec < a.q.n ? 0 : vec < a.q.n + a.k.n ? 1 : 2;
    const int head = kind == 0 ? vec : kind == 1 ? vec - a.q.n : kind == 2 ? vec - a.q.n - a.k.n : 0;
    const Piece pc = piece_of<D>(j, a.rot, a.interleaved);
    // idle lanes read the first head along
    const bool fq = kind == 0 || (kind == 3 && a.q.n > 0), fv = kind == 2;
    const int64_t isb = fq ? a.q.sb : fv ? a.v.sb : a.k.sb, ist = fq ? a.q.st : fv ? a.v.st : a.k.st;
    const T *in = static_cast<const T *>(fq ? a.q.p : fv ? a.v.p : a.k.p) + head * (fq ? a.q.sh : fv ? a.v.sh : a.k.sh);
    const int64_t osb = kind == 0 ? a.qo.sb : a.ko.sb, ost = kind == 0 ? a.qo.st : a.ko.st;
    T *out = static_cast<T *>(kind == 0 ? a.qo.p : a.ko.p) + head * (kind == 0 ? a.qo.sh : a.ko.sh);
    const bool direct = kind == 0 || (kind == 1 && KV == 0);

    float g1[8], g2[8];
    const void *gam = kind == 0 ? a.gq : kind == 1 ? a.gk : nullptr;
    if constexpr (NORM) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g1[i] = g2[i] = 1.f;
        if (gam) {
            load8(static_cast<const T *>(gam) + 8 * pc.c1, g1);
            load8(static_cast<const T *>(gam) + 8 * pc.c2, g2);
        }
    }
    double e1[8], e2[8];
    if constexpr (ENERGY) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e1[i] = e2[i] = 0.0;
    }
    __shared__ __attribute__((aligned(16))) uint32_t amax_of[KV == 2 ? kThreads * 2 : 4];

    // tokens of this workgroup: block `blk` of the batch entry (without
    // energies the whole call is one entry of T tokens), at most 64
    const int64_t place = static_cast<int64_t>(blockIdx.z) * kGridX + blockIdx.x;
    const int64_t unit = place / blocks, blk = place % blocks;
    const int64_t per = ENERGY ? a.L : a.T, t0 = unit * per + blk * TB;
    if (t0 >= a.T) return;
    const int n = static_cast<int>(min(static_cast<int64_t>(TB), per - blk * TB));
    // lane i holds the position and slot of token i
    int pos_of = 0, slot_of = -1;
    if (lane < n) {
        if (a.rot) pos_of = a.pos[t0 + lane];
        if constexpr (KV != 0) slot_of = a.slots[t0 + lane];
    }
    auto where = [&](int i, int64_t &b, int64_t &l) __attribute__((always_inline)) {
        const int64_t t = t0 + i;
        b = ENERGY ? unit : static_cast<int64_t>(static_cast<uint32_t>(t) / static_cast<uint32_t>(a.L));
        l = t - b * a.L;
    };
    // a token's values, and the cos and sin that the lane's pairs take: of its first
    // piece's eight pairs, or (adjacent pairs) of both pieces' four
    struct Token {
        Raw8<T> r1, r2;
        float4 c1, c2, s1, s2;
    };
    const int ca = a.interleaved ? 4 * pc.c1 : 8 * pc.c1, cb = a.interleaved ? 4 * pc.c2 : 8 * pc.c1 + 4;
    const bool turn1 = kind < 2 && a.rot && (a.interleaved ? 8 * pc.c1 < a.rot : pc.on);
    const bool turn2 = kind < 2 && a.rot && (a.interleaved ? 8 * pc.c2 < a.rot : pc.on);
    auto load = [&](Token &k, int i) __attribute__((always_inline)) {
        int64_t b, l;
        where(i, b, l);
        const T *x = in + b * isb + l * ist;
        k.r1 = *reinterpret_cast<const Raw8<T> *>(x + 8 * pc.c1);
        k.r2 = *reinterpret_cast<const Raw8<T> *>(x + 8 * pc.c2);
        if (a.rot) {
            const int p = __builtin_amdgcn_readlane(pos_of, i);
            const int64_t row = static_cast<int64_t>(p >= 0 && p < a.n_pos ? p : 0) * (a.rot / 2);
            if (turn1) {
                k.c1 = *reinterpret_cast<const float4 *>(a.cs + row + ca);
                k.s1 = *reinterpret_cast<const float4 *>(a.sn + row + ca);
            }
            if (turn2) {
                k.c2 = *reinterpret_cast<const float4 *>(a.cs + row + cb);
                k.s2 = *reinterpret_cast<const float4 *>(a.sn + row + cb);
            }
        }
    };
    auto token = [&](const Token &k, int i) __attribute__((always_inline)) {
        int64_t b, l;
        where(i, b, l);
        float x1[8], x2[8];
        load8(k.r1.x, x1);
        load8(k.r2.x, x2);
        if constexpr (NORM) {
#pragma clang fp contract(off)
            double ss = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double u = x1[i], v = x2[i];
                ss = ss + u * u;
                ss = ss + v * v;
            }
            ss += dpp_f64<0xB1>(ss);
            ss += dpp_f64<0x4E>(ss);
            if constexpr (LPH == 8) ss += dpp_f64<0x141>(ss);
            const float r = static_cast<float>(rsqrt64(ss / D + static_cast<double>(a.eps)));
            if (gam) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x1[i] = x1[i] * r * g1[i];
                    x2[i] = x2[i] * r * g2[i];
                }
            }
        }
        if (a.rot) {
            // a position outside the tables gives NaN
            const int p = __builtin_amdgcn_readlane(pos_of, i);
            const float bad = p >= 0 && p < a.n_pos ? 1.f : __builtin_nanf("");
            const float c[8] = {k.c1.x, k.c1.y, k.c1.z, k.c1.w, k.c2.x, k.c2.y, k.c2.z, k.c2.w};
            const float s[8] = {k.s1.x, k.s1.y, k.s1.z, k.s1.w, k.s2.x, k.s2.y, k.s2.z, k.s2.w};
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (turn1) turn(x1[2 * j], x1[2 * j + 1], c[j] * bad, s[j] * bad);
                    if (turn2) turn(x2[2 * j], x2[2 * j + 1], c[4 + j] * bad, s[4 + j] * bad);
                }
            } else if (turn1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) turn(x1[j], x2[j], c[j] * bad, s[j] * bad);
            }
        }
        if (act && direct) {
            T *o = out + b * osb + l * ost;
            store8(o + 8 * pc.c1, x1);
            store8(o + 8 * pc.c2, x2);
            if constexpr (ENERGY) {
                if (kind == 0) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const double u = x1[i], v = x2[i];
                        e1[i] += u * u;
                        e2[i] += v * v;
                    }
                }
            }
        }
        if constexpr (KV != 0) {
            const int slot = __builtin_amdgcn_readlane(slot_of, i);
            const int page = slot >> a.kv.lg_page, off = slot & ((1 << a.kv.lg_page) - 1);
            const bool held = slot >= 0 && page < a.kv.n_pages && (kind == 1 || kind == 2);
            const int64_t row = (static_cast<int64_t>(head) << a.kv.lg_page) + off;
            if constexpr (KV == 1) {
                if (held) {
                    uint8_t *pg = kind == 1 ? a.kv.k + page * a.kv.k_page : a.kv.v + page * a.kv.v_page;
                    uint16_t *o = reinterpret_cast<uint16_t *>(pg) + row * D;
                    store8(o + 8 * pc.c1, x1);
                    store8(o + 8 * pc.c2, x2);
                }
            } else {
                // magnitudes as bit patterns: they order as numbers, NaN above infinity
                uint32_t m1 = 0, m2 = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m1 = max(m1, __float_as_uint(x1[i]) & 0x7fffffffu);
                    m2 = max(m2, __float_as_uint(x2[i]) & 0x7fffffffu);
                }
                // the pieces' maxima meet in the wave's own corner of LDS: a
                // group's four pieces can lie in any of the head's lanes
                uint32_t *mine = amax_of + (threadIdx.x / LPH) * (2 * LPH);
                __builtin_amdgcn_wave_barrier();
                mine[pc.c1] = m1;
                mine[pc.c2] = m2;
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                const uint4 q1 = *reinterpret_cast<const uint4 *>(mine + (pc.c1 & ~3));
                const uint4 q2 = *reinterpret_cast<const uint4 *>(mine + (pc.c2 & ~3));
                const uint32_t s1 = mx_scale_byte(max(max(q1.x, q1.y), max(q1.z, q1.w)));
                const uint32_t s2 = mx_scale_byte(max(max(q2.x, q2.y), max(q2.z, q2.w)));
                const uint32_t w1 = s1 == 255u ? 0u : mx_codes8(x1, __uint_as_float(s1 << 23));
                const uint32_t w2 = s2 == 255u ? 0u : mx_codes8(x2, __uint_as_float(s2 << 23));
                if (held) {
                    uint8_t *pg = kind == 1 ? a.kv.k + page * a.kv.k_page : a.kv.v + page * a.kv.v_page;
                    uint8_t *sg = kind == 1 ? a.kv.ks + page * a.kv.ks_page : a.kv.vs + page * a.kv.vs_page;
                    uint32_t *o = reinterpret_cast<uint32_t *>(pg + row * (D / 2));
                    o[pc.c1] = w1;
                    o[pc.c2] = w2;
                    uint8_t *so = sg + row * (D / 32);
                    if ((pc.c1 & 3) == 0) so[pc.c1 >> 2] = static_cast<uint8_t>(s1);
                    if ((pc.c2 & 3) == 0) so[pc.c2 >> 2] = static_cast<uint8_t>(s2);
                }
            }
        }
    };
    // the next token is on its way while one is worked on
    Token cur, next;
    if (wave < n) load(cur, wave);
    for (int i = wave; i < n; i += kWaves) {               // wave-uniform
        if (i + kWaves < n) load(next, i + kWaves);
        token(cur, i);
        cur = next;
    }

    if constexpr (ENERGY) {
        __shared__ double part[kWaves][64 * 16];
        double *mine = part[wave] + (lane / LPH) * D;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            mine[8 * pc.c1 + i] = e1[i];
            mine[8 * pc.c2 + i] = e2[i];
        }
        __syncthreads();
        const int HD = a.q.n * D, c0 = static_cast<int>(blockIdx.y) * VPW * D;
        double *o = a.partials + (unit * blocks + blk) * HD;
        for (int i = threadIdx.x; i < VPW * D && c0 + i < HD; i += kThreads)
            o[c0 + i] = ((part[0][i] + part[1][i]) + part[2][i]) + part[3][i];
    }
}

// Cached tokens as bf16 rows: 8 elements of each of U rows per thread (an exact
// widening of the 4-bit codes), all U slots and then all U pieces asked for at once.
// Bound by the writes of many tokens, by latency for few.  From 4 bits, 8 + 8 heads of
// 128, with 1 / 2 / 4 / 8 rows per thread: 8198 tokens 12.2 / 11.1 / 11.0 / 11.6 us, 2000
// tokens 4.8 / 5.1 / 5.6 / 7.1; 32 + 32 heads, 8198 tokens (170 MB) 46 / 42 / 38 / 38, the
// last two 4.5 TB/s: four from 4096 workgroups of one row per thread on.
template <int D, int U>
__global__ __launch_bounds__(kThreads) void kv_gather_kernel(KvPages kv, const int32_t *__restrict__ slots, uint32_t rows,
                                                             Heads k, Heads v) {
    constexpr int CH = D / 8, PER = kThreads / CH;
    const uint32_t i0 = blockIdx.x * (PER * U) + threadIdx.x / CH;           // row: token, key or value head
    const int c = threadIdx.x % CH, H2 = 2 * kv.Hkv;
    uint32_t t[U], q[U], sc[U];
    int hv[U], slot[U];
    bool on[U];
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = i0 + u * PER;
        on[u] = i < rows && i >= i0;
        t[u] = (on[u] ? i : 0u) / static_cast<uint32_t>(H2);
        hv[u] = static_cast<int>((on[u] ? i : 0u) - t[u] * H2);
        slot[u] = slots[t[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool key = hv[u] < kv.Hkv;
        const int page = slot[u] >> kv.lg_page, off = slot[u] & ((1 << kv.lg_page) - 1);
        q[u] = sc[u] = 0u;                                 // codes of zeros
        w[u] = make_uint4(0, 0, 0, 0);
        if (slot[u] >= 0 && page < kv.n_pages) {
            const uint8_t *pg = key ? kv.k + page * kv.k_page : kv.v + page * kv.v_page;
            const int64_t row = (static_cast<int64_t>(key ? hv[u] : hv[u] - kv.Hkv) << kv.lg_page) + off;
            if (!kv.mx) {
                w[u] = reinterpret_cast<const uint4 *>(pg + row * (2 * D))[c];
            } else {
                const uint8_t *sg = key ? kv.ks + page * kv.ks_page : kv.vs + page * kv.vs_page;
                q[u] = reinterpret_cast<const uint32_t *>(pg + row * (D / 2))[c];
                sc[u] = sg[row * (D / 32) + (c >> 2)];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#if defined(__HIP_DEVICE_COMPILE__)
        if (kv.mx) {
            const float s = __uint_as_float(sc[u] << 23);
            w[u].x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[u], s, 0));
            w[u].y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[u], s, 1));
            w[u].z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[u], s, 2));
            w[u].w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[u], s, 3));
        }
#endif
        const bool key = hv[u] < kv.Hkv;
        const Heads &d = key ? k : v;
        if (on[u])
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(d.p) + t[u] * d.st + (key ? hv[u] : hv[u] - kv.Hkv) * d.sh + 8 * c) = w[u];
    }
}

namespace {

// Tokens per workgroup.  With energies each workgroup writes a float64 row of
// columns and adds up its waves: 256 workgroups at least, else as many tokens as
// that leaves (kernel + final sum, us, for 256 / 512 / 1024: 8192 tokens x 32 + 8 heads
// 41 + 5 / 42 + 5 / 42 + 5; 2 x 1001 x 32 + 8 15 + 4 / 17 + 4 / 20 + 6; the same x 16 + 8
// with norms 13 + 4 / 15 + 6 / 15 + 6).  Without, 2048 (512 / 1024 / 2048 / 4096: 8192 x 32 +
// 8 heads 41 / 45 / 40 / 43, 6000 tokens appended with their queries 40 / 37 / 36 / 39).
int rotate_tokens(int64_t T, int64_t heads, int D, bool energy) {
    const int64_t groups = (heads + 1024 / D - 1) / (1024 / D);
    int tb = kWaves;
    while (tb < 64 && T / (2 * tb) * groups >= (energy ? 256 : 2048)) tb *= 2;
    return tb;
}

template <typename T, int D, int KV, bool ENERGY>
hipError_t launch(const RotateArgs &a, hipStream_t stream) {
    const int nv = a.q.n + a.k.n + a.v.n, groups = (nv + 1024 / D - 1) / (1024 / D);
    const int TB = rotate_tokens(a.T, ENERGY ? a.q.n : nv, D, ENERGY);
    const int64_t per = ENERGY ? a.L : a.T, blocks = (per + TB - 1) / TB, units = ENERGY ? a.T / a.L : 1;
    const int64_t all = units * blocks, nz = (all + kGridX - 1) / kGridX;
    const dim3 grid(static_cast<uint32_t>(nz > 1 ? kGridX : all), static_cast<uint32_t>(groups), static_cast<uint32_t>(nz));
    if (a.gq || a.gk) rotate_kernel<T, D, KV, true, ENERGY><<<grid, kThreads, 0, stream>>>(a, TB, blocks);
    else rotate_kernel<T, D, KV, false, ENERGY><<<grid, kThreads, 0, stream>>>(a, TB, blocks);
    return hipGetLastError();
}

}  // namespace

int64_t rotate_blocks(int64_t batch, int64_t L, int64_t heads, int D) {
    const int TB = rotate_tokens(batch * L, heads, D, true);
    return (L + TB - 1) / TB;
}

hipError_t launch_rotate(const RotateArgs &a, bool bf16, int D, hipStream_t stream) {
    const bool e = a.partials != nullptr;
    if (bf16) {
        if (D == 128) return e ? launch<uint16_t, 128, 0, true>(a, stream) : launch<uint16_t, 128, 0, false>(a, stream);
        return e ? launch<uint16_t, 64, 0, true>(a, stream) : launch<uint16_t, 64, 0, false>(a, stream);
    }
    if (D == 128) return e ? launch<float, 128, 0, true>(a, stream) : launch<float, 128, 0, false>(a, stream);
    return e ? launch<float, 64, 0, true>(a, stream) : launch<float, 64, 0, false>(a, stream);
}

hipError_t launch_kv_append(const RotateArgs &a, int D, hipStream_t stream) {
    if (a.kv.mx)
        return D == 128 ? launch<uint16_t, 128, 2, false>(a, stream) : launch<uint16_t, 64, 2, false>(a, stream);
    return D == 128 ? launch<uint16_t, 128, 1, false>(a, stream) : launch<uint16_t, 64, 1, false>(a, stream);
}

hipError_t launch_kv_gather(const KvPages &kv, const int32_t *slots, int64_t T, const Heads &k, const Heads &v, int D,
                            hipStream_t stream) {
    const uint32_t rows = static_cast<uint32_t>(T * 2 * kv.Hkv), per = kThreads / (D / 8);
    const bool many = rows / per >= 4096;                  // workgroups of one row per thread
    const uint32_t each = many ? 4 * per : per, grid = rows / each + (rows % each != 0);
    if (D == 128 && many) kv_gather_kernel<128, 4><<<grid, kThreads, 0, stream>>>(kv, slots, rows, k, v);
    else if (D == 128) kv_gather_kernel<128, 1><<<grid, kThreads, 0, stream>>>(kv, slots, rows, k, v);
    else if (many) kv_gather_kernel<64, 4><<<grid, kThreads, 0, stream>>>(kv, slots, rows, k, v);
    else kv_gather_kernel<64, 1><<<grid, kThreads, 0, stream>>>(kv, slots, rows, k, v);
    return hipGetLastError();
}

}  // namespace rmm
