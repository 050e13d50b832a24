// The join of a block's output with the residual stream, and the norm that feeds
// the next block's reduced projection (Sec. 3.2 scores from the projection's own
// input, whose column energies come with it):
//
//   y' = y,  or  y * r(y) * gamma_post               (a norm after the block)
//   h  = s R + gate * y'                             stored in the stream's type
//   x  = h * r(h) * gamma_pre                        (the norm before the next)
//   r(v) = 1 / sqrt(mean_j v_j^2 + eps)
//
// The mean squares are float64 sums, r is rounded to fp32 once, and every other
// step is one fp32 operation, rounded by itself: x and the energies then do not
// depend on how a row is split over lanes (but for an r whose float64 value lies
// within float64 rounding of an fp32 border: one row in 10^7 or so).  h is rounded to the stream's type
// before its norm, which is of the stored stream, and x once, to its type.
#include <type_traits>

#include "block.h"
#include "device_common.h"
#include "kernels.h"

namespace rmm {

namespace {

// eight values as they lie in memory
template <typename T>
struct Raw8 {
    uint4 q[sizeof(T) / 2];
};
// 16 bytes at any address (global memory takes them at every alignment)
typedef uint32_t any16 __attribute__((ext_vector_type(4), aligned(2)));
// the first n of them exist, the others are zeros; without TAIL all or none do
template <bool TAIL = false, typename T>
__device__ __forceinline__ Raw8<T> load_raw(const T *p, int n = 8) {
    Raw8<T> r = {};
    if (TAIL ? n >= 8 : n > 0) {
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; ++i) {
            const any16 v = reinterpret_cast<const any16 *>(p)[i];
            r.q[i] = make_uint4(v.x, v.y, v.z, v.w);
        }
    } else if constexpr (TAIL) {
        uint32_t *w = &r.q[0].x;
#pragma unroll
        for (int e = 0; e < 7; ++e) {
            if (e >= n) continue;
            if constexpr (sizeof(T) == 2) w[e >> 1] |= static_cast<uint32_t>(p[e]) << (16 * (e & 1));
            else w[e] = __float_as_uint(p[e]);
        }
    }
    return r;
}
__device__ __forceinline__ void unpack(const Raw8<uint16_t> &r, float (&v)[8]) {
    const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw8<float> &r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(r.q[i].x);
        v[4 * i + 1] = __uint_as_float(r.q[i].y);
        v[4 * i + 2] = __uint_as_float(r.q[i].z);
        v[4 * i + 3] = __uint_as_float(r.q[i].w);
    }
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) { unpack(load_raw(p), v); }
template <bool TAIL>
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8], int n) {
    const any16 q = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    if (TAIL ? n >= 8 : n > 0) {
        *reinterpret_cast<any16 *>(p) = q;
    } else if constexpr (TAIL) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = static_cast<uint16_t>(q[e >> 1] >> (16 * (e & 1)));
    }
}
template <bool TAIL>
__device__ __forceinline__ void store8(float *p, const float (&v)[8], int n) {
    typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
    if (TAIL ? n >= 8 : n > 0) {
        reinterpret_cast<f32x4_any *>(p)[0] = f32x4_any{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f32x4_any *>(p)[1] = f32x4_any{v[4], v[5], v[6], v[7]};
    } else if constexpr (TAIL) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = v[e];
    }
}
template <class T>
__device__ __forceinline__ float rounded(float v) {
    return std::is_same<T, uint16_t>::value ? bf16_to_f32(f32_to_bf16(v)) : v;
}

// One workgroup per row: thread t holds elements 8 (t + NT c) .. + 7, c < C.  The
// stream is asked for after the block's sum, all chunks together: asked for before
// it, everything took 5 to 12 % longer (8192 x 4096 50 / 54 us, 2002 x 8192 29 / 33).
template <typename TY, typename TS, bool TAIL, int NT, int C>
__global__ __launch_bounds__(NT) void join_rows_kernel(JoinArgs a) {
#pragma clang fp contract(off)
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    const int K = a.K;
    const int64_t unit = row / a.M, m = row - unit * a.M;
    const TY *y = a.y ? static_cast<const TY *>(a.y) + row * a.ldy : nullptr;
    const TS *r = a.r ? static_cast<const TS *>(a.r) + row * a.ldr : nullptr;
    const TY *gate = a.gate ? static_cast<const TY *>(a.gate) + unit * a.gate_unit + m * a.gate_row : nullptr;
    const TY *gpost = static_cast<const TY *>(a.gpost), *gpre = static_cast<const TY *>(a.gpre);
    auto first = [&](int c) { return 8 * (t + NT * c); };
    // chunk c of a row; absent elements are zeros
    auto load = [&](auto *p, int c, float (&v)[8]) { unpack(load_raw<TAIL>(p + first(c), K - first(c)), v); };
    auto store = [&](auto *p, int c, const float (&v)[8]) { store8<TAIL>(p + first(c), v, K - first(c)); };
    Raw8<TY> yq[C];
    Raw8<TS> rq[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        yq[c] = {};
        if (y) yq[c] = load_raw<TAIL>(y + first(c), K - first(c));
    }
    __shared__ double red[2][NT / 64];
    // 1 / rms of the row's values, the same in every thread
    auto inv_rms = [&](const float (&v)[C][8], int slot) {
        double s = 0.0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma(static_cast<double>(v[c][e]), static_cast<double>(v[c][e]), s);
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1) s += __shfl_xor(s, sh);
        if constexpr (NT > 64) {
            if ((t & 63) == 0) red[slot][t >> 6] = s;
            __syncthreads();
            s = red[slot][0];
#pragma unroll
            for (int w = 1; w < NT / 64; ++w) s += red[slot][w];
        }
        return static_cast<float>(1.0 / sqrt(s / K + static_cast<double>(a.eps)));
    };

    float h[C][8];
    if (y) {
#pragma unroll
        for (int c = 0; c < C; ++c) unpack(yq[c], h[c]);
        if (a.post) {
            const float ry = inv_rms(h, 0);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float g[8];
                if (gpost) load(gpost, c, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[c][e] = gpost ? h[c][e] * ry * g[e] : h[c][e] * ry;
            }
        }
        if (gate) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float g[8];
                load(gate, c, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[c][e] = h[c][e] * g[e];
            }
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        rq[c] = {};
        if (r) rq[c] = load_raw<TAIL>(r + first(c), K - first(c));
    }
    if (r) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float v[8];
            unpack(rq[c], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[c][e] = y ? a.rs * v[e] + h[c][e] : a.rs * v[e];
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (a.h) store(static_cast<TS *>(a.h) + row * a.ldh, c, h[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = rounded<TS>(h[c][e]);
    }
    if (!a.x && !a.rscale) return;
    const float rh = inv_rms(h, 1);
    if (a.rscale) {
        if (t == 0) a.rscale[row] = rh;
        return;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float g[8];
        if (gpre) load(gpre, c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = gpre ? h[c][e] * rh * g[e] : h[c][e] * rh;
        store(static_cast<TY *>(a.x) + row * a.ldx, c, h[c]);
    }
}

// The K-major half: a wave takes 64 columns of a run of rows, 64 at a time.  Lane
// 8 mc + jc holds rows 8 mc .. + 7 and columns 8 jc .. + 7 of each 64 x 64 tile,
// transposes its 8 x 8 block in registers and writes 16 bytes (8 tokens) of each
// of 8 Xt rows, so that the 8 lanes of one jc fill 128 bytes.  LINES: these are
// whole lines; they go past the caches, which then still hold the stream (8192 x
// 4096, both launches: 74 us without, 66 so; where lines are shared by two tiles,
// 2002 x 8192, 41 and 47).
template <typename TS, bool LINES>
__global__ __launch_bounds__(256) void join_kmajor_kernel(
    const TS *__restrict__ H, int64_t ldh, const float *__restrict__ rscale, const uint16_t *__restrict__ gpre,
    int64_t M, int K, int64_t rps, uint16_t *__restrict__ Xt, int64_t ldxt, double *__restrict__ out) {
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int jc = lane & 7, mc = lane >> 3;
    const int j = (blockIdx.x * 4 + wave) * 64 + 8 * jc;
    const int64_t unit = blockIdx.z, s = blockIdx.y;
    const int64_t m_end = min(M, (s + 1) * rps);
    const bool live = j < K;                        // K % 8 == 0
    float g[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = 1.f;
    if (gpre && live) load8(gpre + j, g);
    double acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0;
    for (int64_t m0 = s * rps + 8 * mc; live && m0 < m_end; m0 += 64) {
        const int n = static_cast<int>(min<int64_t>(8, m_end - m0));
        uint32_t w[8][4];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float v[8];
            float sc = 0.f;
            if (r < n) {
                load8(H + (unit * M + m0 + r) * ldh + j, v);
                sc = rscale[unit * M + m0 + r];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float xa = v[2 * e] * sc, xb = v[2 * e + 1] * sc;
                if (gpre) { xa = xa * g[2 * e]; xb = xb * g[2 * e + 1]; }
                w[r][e] = pack_bf16x2(xa, xb);
                const double ya = static_cast<double>(__uint_as_float(w[r][e] << 16));
                const double yb = static_cast<double>(__uint_as_float(w[r][e] & 0xffff0000u));
                if (r < n) {
                    acc[2 * e] = fma(ya, ya, acc[2 * e]);
                    acc[2 * e + 1] = fma(yb, yb, acc[2 * e + 1]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = __builtin_amdgcn_perm(w[2 * q + 1][e >> 1], w[2 * q][e >> 1], sel);
            uint16_t *dst = Xt + (unit * K + j + e) * ldxt + m0;
            if (n == 8) {
                typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
                const u32x4 v = {o[0], o[1], o[2], o[3]};
                if (LINES) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(dst));
                else *reinterpret_cast<u32x4 *>(dst) = v;
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < n) dst[r] = static_cast<uint16_t>(o[r >> 1] >> (16 * (r & 1)));
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        acc[e] += __shfl_xor(acc[e], 8);
        acc[e] += __shfl_xor(acc[e], 16);
        acc[e] += __shfl_xor(acc[e], 32);
    }
    if (mc == 0 && live) {
        double *o = out + (unit * gridDim.y + s) * K + j;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = acc[e];
    }
}

// TAIL: K % 8 != 0
template <typename TY, typename TS, bool TAIL>
hipError_t launch_rows(const JoinArgs &a, hipStream_t stream) {
    auto go = [&](auto kernel, int nt) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(a.rows)), dim3(nt), 0, stream, a);
        return hipGetLastError();
    };
    // Few rows: as many threads as chunks, for the shortest wait (64 x 4096, 512 x 1 /
    // 256 x 2 / 128 x 4: 4.6 / 5.0 / 6.3 us).  From 4096 waves on: two to four chunks per
    // thread (8192 x 4096 bf16, 512 x 1 / 256 x 2 / 128 x 4 / 64 x 8: 63 / 56 / 58 / 66 us;
    // 8192 x 2048, 512 x 1 / 256 x 2 / 64 x 4: 46 / 36 / 32; 2002 x 8192 with an fp32
    // stream, 1024 x 1 / 512 x 2 / 256 x 4: 45.6 / 44.8 / 48.8).  Past 16384 a row is still
    // held whole, eight chunks a thread, most of them absent just past it: 45 to 112 of its 128
    // registers go to scratch, and its time is far from the copy's (2^25 bf16 in all, K =
    // 16384 53 us; 16392 217, 20480 188, 32768 133, 65536 98).
    const auto many = [&](int waves) { return a.rows * waves >= 4096; };
    if (a.K <= 64 * 8) return go(join_rows_kernel<TY, TS, TAIL, 64, 1>, 64);
    if (a.K <= 128 * 8) return many(1) ? go(join_rows_kernel<TY, TS, TAIL, 64, 2>, 64) : go(join_rows_kernel<TY, TS, TAIL, 128, 1>, 128);
    if (a.K <= 256 * 8) return many(1) ? go(join_rows_kernel<TY, TS, TAIL, 64, 4>, 64) : go(join_rows_kernel<TY, TS, TAIL, 256, 1>, 256);
    if (a.K <= 512 * 8) return many(4) ? go(join_rows_kernel<TY, TS, TAIL, 256, 2>, 256) : go(join_rows_kernel<TY, TS, TAIL, 512, 1>, 512);
    if (a.K <= 1024 * 8) return many(8) ? go(join_rows_kernel<TY, TS, TAIL, 512, 2>, 512) : go(join_rows_kernel<TY, TS, TAIL, 1024, 1>, 1024);
    if (a.K <= 1024 * 16) return many(8) ? go(join_rows_kernel<TY, TS, TAIL, 512, 4>, 512) : go(join_rows_kernel<TY, TS, TAIL, 1024, 2>, 1024);
    return go(join_rows_kernel<TY, TS, TAIL, 1024, 8>, 1024);
}

constexpr int64_t kJoinRows = 64;                   // rows of a K-major tile

// whole tiles per split, enough splits for about eight workgroups per CU
int64_t rows_per_split(int64_t B, int64_t M, int64_t K) {
    const int64_t tiles = (M + kJoinRows - 1) / kJoinRows, cols = (K + 255) / 256 * B;
    const int64_t want = (2048 + cols - 1) / cols;
    const int64_t splits = tiles < want ? tiles : want;
    return (tiles + splits - 1) / splits * kJoinRows;
}

}  // namespace

hipError_t launch_join_rows(const JoinArgs &a, bool y_bf16, bool stream_bf16, hipStream_t stream) {
    auto go = [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if (y_bf16)
            return stream_bf16 ? launch_rows<uint16_t, uint16_t, TAIL>(a, stream) : launch_rows<uint16_t, float, TAIL>(a, stream);
        return launch_rows<float, float, TAIL>(a, stream);
    };
    return a.K % 8 ? go(std::true_type{}) : go(std::false_type{});
}

int64_t join_splits(int64_t B, int64_t M, int64_t K) {
    const int64_t rps = rows_per_split(B, M, K);
    return (M + rps - 1) / rps;
}

hipError_t launch_join_kmajor(const void *H, bool stream_bf16, int64_t ldh, const float *rscale, const uint16_t *gpre,
                              int64_t B, int64_t M, int64_t K, uint16_t *Xt, int64_t ldxt, double *partials,
                              double *energy, hipStream_t stream) {
    const int64_t rps = rows_per_split(B, M, K), S = join_splits(B, M, K);
    const dim3 grid(static_cast<unsigned>((K + 255) / 256), static_cast<unsigned>(S), static_cast<unsigned>(B));
    double *out = S == 1 ? energy : partials;
    auto go = [&](auto kernel, const auto *h) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, h, ldh, rscale, gpre, M, static_cast<int>(K), rps, Xt, ldxt,
                           out);
    };
    const uint16_t *hb = static_cast<const uint16_t *>(H);
    const float *hf = static_cast<const float *>(H);
    if (ldxt % kJoinRows == 0 && reinterpret_cast<uintptr_t>(Xt) % 128 == 0)
        stream_bf16 ? go(join_kmajor_kernel<uint16_t, true>, hb) : go(join_kmajor_kernel<float, true>, hf);
    else
        stream_bf16 ? go(join_kmajor_kernel<uint16_t, false>, hb) : go(join_kmajor_kernel<float, false>, hf);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || S == 1) return e;
    return launch_score_finalize_grouped(partials, B, S, K, energy, stream);
}

}  // namespace rmm
