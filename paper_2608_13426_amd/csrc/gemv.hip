// Reduced product with few rows per unit (a decode step: one token, or a
// handful, per sequence)   (Sec. 3.2 definition of RMM; App. A: during
// decoding the retained set follows the current decoding state).
//
//   Y[b][m][:] = sum_{t < k} X[b][m][I_b[t]] * W[I_b[t]][:],   m < M <= 8
//
// With so few rows the product is bound by reading the retained rows of W
// (k*N*2 bytes per unit): each retained index is one contiguous weight row,
// so the kernel streams exactly those rows.  Work is split over
// (512-column chunk, slice of the retained list, unit): a workgroup stages
// its slice's row offsets and activations in LDS, its four waves take every
// fourth row, each lane holding 8 columns (one 16-byte load per row, 8 rows
// in flight), and the waves' sums are added in a fixed order in LDS.  Slices write fp32 partials that a second kernel adds in slice
// order (or, with one slice, the workgroup writes Y directly), so results
// are bit-reproducible.
#include <type_traits>

#include "device_common.h"
#include "epilogue.h"
#include "kernels.h"
#include "span.h"

namespace rmm {

namespace {

namespace gv {
constexpr int NW = 4, NT = NW * 64;
constexpr int CW = 512;            // columns per workgroup (64 lanes x 8)
constexpr int RB = 256;            // retained rows staged per pass
constexpr int TARGET_BLOCKS = 512;
constexpr int MIN_SLICE = 64;      // retained rows per slice at least
}  // namespace gv

// One workgroup's share: columns chunk*CW .., slice s of unit b's retained
// list; DIRECT writes Y, otherwise the slice's fp32 partials.
template <int MR, bool VEC, bool EP = false>
__device__ __forceinline__ void gemv_tile(
    const uint16_t *__restrict__ X, const uint16_t *__restrict__ W, const int32_t *__restrict__ idx,
    float *__restrict__ P, OutPtr<EP, uint16_t> Y, int M, int N, int K, int k, int64_t ldx,
    int64_t ldw, int64_t ldy, int SR, int S, int chunk, int s, int b, bool DIRECT,
    const Epilogue &ep = Epilogue{}) {
    using namespace gv;
    __shared__ uint32_t roff[RB];              // byte offset of each staged row in W
    __shared__ float xs[RB][MR];               // its activation value per row m
    __shared__ float red[NW - 1][MR][CW];      // sums of waves 1..3

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = chunk * CW;
    const int t0 = s * SR, t1 = min(k, t0 + SR);
    const int32_t *I = idx + static_cast<int64_t>(b) * k;
    const uint16_t *Xb = X + static_cast<int64_t>(b) * M * ldx;
    // the whole of W from this chunk's first column on: a row's columns past N read
    // padding or the next row, and past the last row's end zeros
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(W + n0), 0,
        static_cast<uint32_t>(span_bytes(K, ldw, N, VEC) - n0 * 2), 0x00020000);

    float acc[MR][8];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[m][e] = 0.f;

    for (int base = t0; base < t1; base += RB) {
        const int nr = min(RB, t1 - base);
        for (int r = tid; r < nr; r += NT) {
            const int j = I[base + r];
            roff[r] = static_cast<uint32_t>(j * ldw * 2);
#pragma unroll
            for (int m = 0; m < MR; ++m)
                xs[r][m] = m < M ? bf16_to_f32(Xb[m * ldx + j]) : 0.f;
        }
        __syncthreads();
        // rows wave, wave + 4, ... of this pass; 8 loads in flight per lane
        for (int r0 = wave; r0 < nr; r0 += 8 * NW) {
            uint32_t w[8][4];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int r = r0 + NW * u;
                if (VEC) {
                    const uint32_t o = r < nr ? roff[r] + 16u * lane : 0x80000000u;
                    const auto v = __builtin_amdgcn_raw_buffer_load_b128(wr, o, 0, 0);
                    w[u][0] = v[0]; w[u][1] = v[1]; w[u][2] = v[2]; w[u][3] = v[3];
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t o = r < nr ? roff[r] + 16u * lane + 4u * q : 0x80000000u;
                        const uint32_t lo = __builtin_amdgcn_raw_buffer_load_b16(wr, o, 0, 0);
                        const uint32_t hi = __builtin_amdgcn_raw_buffer_load_b16(wr, o + 2u, 0, 0);
                        w[u][q] = lo | (hi << 16);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int r = r0 + NW * u;
                if (r < nr) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float wl = __uint_as_float(w[u][q] << 16);
                        const float wh = __uint_as_float(w[u][q] & 0xffff0000u);
#pragma unroll
                        for (int m = 0; m < MR; ++m) {
                            acc[m][2 * q] = __builtin_fmaf(xs[r][m], wl, acc[m][2 * q]);
                            acc[m][2 * q + 1] = __builtin_fmaf(xs[r][m], wh, acc[m][2 * q + 1]);
                        }
                    }
                }
            }
        }
        __syncthreads();                       // staged rows are reused by the next pass
    }

    // waves 1..3 hand their sums to wave 0, which adds them in wave order
    if (wave > 0) {
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int e = 0; e < 8; ++e) red[wave - 1][m][8 * lane + e] = acc[m][e];
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 0; w < NW - 1; ++w)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[m][e] += red[w][m][8 * lane + e];
    const int nb = n0 + 8 * lane;
#pragma unroll
    for (int m = 0; m < MR; ++m) {
        if (m >= M) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int n = nb + e;
            if (n < N) {
                if (DIRECT) {
                    const int64_t row = static_cast<int64_t>(b) * M + m;
                    if constexpr (EP) acc[m][e] = ep_value<uint16_t>(ep, acc[m][e], row, n);
                    Y[row * ldy + n] = f32_to_bf16(acc[m][e]);
                } else
                    P[((static_cast<int64_t>(b) * S + s) * M + m) * N + n] = acc[m][e];
            }
        }
    }
}

// Two to eight rows per unit on the matrix cores: v_mfma_f32_4x4x4_16b_bf16 holds
// 16 products of 4 rows of X by 4 columns of W over 4 retained indices, a column
// per lane, so each lane multiplies the columns it has loaded and W passes through
// no LDS.  A wave takes every fourth group of four retained rows; four groups (16
// KiB) are on their way while two are multiplied: 16 byte permutations bring a
// group's four values of each column together, and 8 (up to 4 rows) or 16
// products follow, against 4 * (8 + 8 M) operations in the form above.
// Three units of 5 x 4096 -> 6144, a set of 2048 each: 39 us in that form, 20 so (21
// with two groups on their way); 8 x 14336 -> 4096, k = 7168: 29 and 17 (4 rows: 18 and
// 16; 2 rows: 15 both).
template <int MG, bool EP>
__global__ __launch_bounds__(gv::NT) void gemv_quad_kernel(
    const uint16_t *__restrict__ X, const uint16_t *__restrict__ W, const int32_t *__restrict__ idx,
    float *__restrict__ P, OutPtr<EP, uint16_t> Y, int M, int N, int K, int k, int64_t ldx,
    int64_t ldw, int64_t ldy, int SR, int S, Epilogue ep) {
    using namespace gv;
    constexpr int MR = 4 * MG, XS = RB + 4;    // xs rows apart in LDS (elements)
    __shared__ __attribute__((aligned(16))) uint32_t roff[RB];
    __shared__ __attribute__((aligned(16))) uint16_t xs[MR * XS];
    __shared__ __attribute__((aligned(16))) float red[2][MR][CW];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * CW, s = blockIdx.y, b = blockIdx.z;
    const int t0 = s * SR, t1 = min(k, t0 + SR);
    const int32_t *I = idx + static_cast<int64_t>(b) * k;
    const uint16_t *Xb = X + static_cast<int64_t>(b) * M * ldx;
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t *>(W + n0), 0,
        static_cast<uint32_t>(span_bytes(K, ldw, N) - n0 * 2), 0x00020000);

    f32x4_t acc[MG][8];                        // [rows 4g ..][the lane's column]
#pragma unroll
    for (int g = 0; g < MG; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[g][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

    for (int base = t0; base < t1; base += RB) {
        const int nr = min(RB, t1 - base);
        // rows past the slice: out of range (zeros) times zero
        static_assert(RB == NT, "a row per thread");
        const bool row_in = tid < nr;
        const int j = row_in ? I[base + tid] : 0;
        roff[tid] = row_in ? static_cast<uint32_t>(j * ldw * 2) : 0x80000000u;
        lds_barrier();
        uint16_t xv[MR];
#pragma unroll
        for (int m = 0; m < MR; ++m) xv[m] = row_in && m < M ? Xb[m * ldx + j] : uint16_t(0);
        const int groups = (nr + 3) / 4;
        u32x4 w[3][2][4];
        auto fetch = [&](int g, u32x4 (&q)[2][4]) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = min(4 * (g + NW * u), RB - 4);
                const u32x4 o = *reinterpret_cast<const u32x4 *>(&roff[r]);
                const bool in = g + NW * u < groups;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    q[u][i] = __builtin_amdgcn_raw_buffer_load_b128(wr, in ? o[i] + 16u * lane : 0x80000000u, 0, 0);
            }
        };
        auto multiply = [&](int g, const u32x4 (&q)[2][4]) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = min(4 * (g + NW * u), RB - 4);
                s16x4_t x[MG];
#pragma unroll
                for (int h = 0; h < MG; ++h) x[h] = *reinterpret_cast<const s16x4_t *>(&xs[(4 * h + (lane & 3)) * XS + r]);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;
                    const uint2 d = make_uint2(__builtin_amdgcn_perm(q[u][1][c >> 1], q[u][0][c >> 1], sel),
                                               __builtin_amdgcn_perm(q[u][3][c >> 1], q[u][2][c >> 1], sel));
#pragma unroll
                    for (int h = 0; h < MG; ++h)
                        acc[h][c] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(x[h], __builtin_bit_cast(s16x4_t, d), acc[h][c], 0, 0, 0);
                }
            }
        };
        // groups past the last one load nothing (out of range) and add zeros; the
        // first two pairs are on their way while X's values arrive
        fetch(wave, w[0]);
        fetch(wave + 2 * NW, w[1]);
#pragma unroll
        for (int m = 0; m < MR; ++m) xs[m * XS + tid] = xv[m];
        lds_barrier();
        for (int g = wave; g < groups; g += 6 * NW) {
            fetch(g + 4 * NW, w[2]);
            multiply(g, w[0]);
            if (g + 2 * NW >= groups) break;
            fetch(g + 6 * NW, w[0]);
            multiply(g + 2 * NW, w[1]);
            if (g + 4 * NW >= groups) break;
            fetch(g + 8 * NW, w[1]);
            multiply(g + 4 * NW, w[2]);
        }
        lds_barrier();                         // staged rows are reused by the next pass
    }

    // waves 2 and 3 hand their sums to 0 and 1, then 1 to 0
    auto put = [&](float (&to)[MR][CW]) {
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4_t *>(&to[m][256 * h + 4 * lane]) =
                    f32x4_t{acc[m / 4][4 * h][m % 4], acc[m / 4][4 * h + 1][m % 4], acc[m / 4][4 * h + 2][m % 4],
                            acc[m / 4][4 * h + 3][m % 4]};
    };
    auto add = [&](const float (&from)[MR][CW]) {
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4_t v = *reinterpret_cast<const f32x4_t *>(&from[m][256 * h + 4 * lane]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m / 4][4 * h + e][m % 4] += v[e];
            }
    };
    if (wave >= 2) put(red[wave - 2]);
    __syncthreads();
    if (wave < 2) add(red[wave]);
    __syncthreads();
    if (wave == 1) put(red[0]);
    __syncthreads();
    if (wave != 0) return;
    add(red[0]);
    const int nb = n0 + 8 * lane;
#pragma unroll
    for (int m = 0; m < MR; ++m) {
        if (m >= M) break;
        const int64_t row = static_cast<int64_t>(b) * M + m;
        if (S > 1) {
            float *p = P + ((static_cast<int64_t>(b) * S + s) * M + m) * N + nb;
            if (N % 4 == 0 && nb + 8 <= N) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<f32x4_t *>(p + 4 * h) =
                        f32x4_t{acc[m / 4][4 * h][m % 4], acc[m / 4][4 * h + 1][m % 4], acc[m / 4][4 * h + 2][m % 4],
                                acc[m / 4][4 * h + 3][m % 4]};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (nb + e < N) p[e] = acc[m / 4][e][m % 4];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (nb + e >= N) continue;
                float y = acc[m / 4][e][m % 4];
                if constexpr (EP) y = ep_value<uint16_t>(ep, y, row, nb + e);
                Y[row * ldy + nb + e] = f32_to_bf16(y);
            }
        }
    }
}

template <int MR, bool VEC, bool DIRECT, bool EP = false>
__global__ __launch_bounds__(gv::NT) void gemv_partial_kernel(
    const uint16_t *__restrict__ X, const uint16_t *__restrict__ W, const int32_t *__restrict__ idx,
    float *__restrict__ P, OutPtr<EP, uint16_t> Y, int M, int N, int K, int k, int64_t ldx,
    int64_t ldw, int64_t ldy, int SR, int S, Epilogue ep = {}) {
    gemv_tile<MR, VEC, EP>(X, W, idx, P, Y, M, N, K, k, ldx, ldw, ldy, SR, S, blockIdx.x, blockIdx.y,
                           blockIdx.z, DIRECT, ep);
}

// Several independent one-row products in one launch: the workgroups of
// group g are g's (chunk, slice, unit) triples, numbered from first[g].
__global__ __launch_bounds__(gv::NT) void gemv_partial_grouped_kernel(GemvGroups G) {
    int g = 0;
    while (g + 1 < G.n && static_cast<int>(blockIdx.x) >= G.g[g + 1].first) ++g;
    const GemvGroup &q = G.g[g];
    const int local = static_cast<int>(blockIdx.x) - q.first;
    const int chunk = local % q.chunks, s = (local / q.chunks) % q.S, b = local / (q.chunks * q.S);
    gemv_tile<1, true>(q.X, q.W, q.idx, q.P, q.Y, 1, q.N, q.K, q.k, q.ldx, q.ldw, q.ldy, q.SR, q.S,
                       chunk, s, b, q.S == 1);
}

// The slice reduction of one 64-column piece: the 256 threads are 64
// columns (one per lane) x 4 waves; wave w adds slices [w*S/4, (w+1)*S/4)
// in slice order (eight loads in flight), and the four quarter sums are
// added in wave order (AHEAD: the last ones' loads, fewer than eight, go out together too).  p points at slice 0 of the lane's column; slice s
// is st floats further.  Returns the sum in wave 0 (other waves: garbage).
template <bool AHEAD = false>
__device__ __forceinline__ float reduce_slices(const float *__restrict__ p, int64_t st, int S,
                                               bool col_ok) {
    __shared__ float quarter[3][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int s0 = w * S / 4, s1 = (w + 1) * S / 4;
    float sum = 0.f;
    if (col_ok) {
        int s = s0;
        for (; s + 8 <= s1; s += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p[(s + u) * st];
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u];
        }
        if constexpr (AHEAD) {                 // the last few too
            float v[7];
#pragma unroll
            for (int u = 0; u < 7; ++u) v[u] = s + u < s1 ? p[(s + u) * st] : 0.f;
#pragma unroll
            for (int u = 0; u < 7; ++u) sum += v[u];
        } else {
            for (; s < s1; ++s) sum += p[s * st];
        }
    }
    if (w > 0) quarter[w - 1][lane] = sum;
    __syncthreads();
    if (w == 0) sum = ((sum + quarter[0][lane]) + quarter[1][lane]) + quarter[2][lane];
    return sum;
}

// Y[b][m][n] = the slices' partials P[b][s][m][n] added in the order of
// reduce_slices; workgroup (x, m, b) covers columns 64x .. 64x+63
template <bool EP = false>
__global__ __launch_bounds__(256) void gemv_reduce_kernel(const float *__restrict__ P,
                                                          OutPtr<EP, uint16_t> Y, int M, int N,
                                                          int S, int64_t ldy, Epilogue ep = {}) {
    const int n = blockIdx.x * 64 + (threadIdx.x & 63);
    const int m = blockIdx.y, b = blockIdx.z;
    const float *p = P + (static_cast<int64_t>(b) * S * M + m) * N + n;
    float sum = reduce_slices<EP>(p, static_cast<int64_t>(M) * N, S, n < N);
    if (threadIdx.x < 64 && n < N) {
        const int64_t row = static_cast<int64_t>(b) * M + m;
        if constexpr (EP) sum = ep_value<uint16_t>(ep, sum, row, n);
        Y[row * ldy + n] = f32_to_bf16(sum);
    }
}

// the slice reduction of every group with more than one slice: workgroup
// blockIdx.x of group g covers 64 columns of one unit, numbered from rfirst[g]
__global__ __launch_bounds__(256) void gemv_reduce_grouped_kernel(GemvGroups G) {
    int g = -1;
    for (int i = 0; i < G.n; ++i)
        if (G.g[i].S > 1 && static_cast<int>(blockIdx.x) >= G.g[i].rfirst) g = i;
    const GemvGroup &q = G.g[g];
    const int local = static_cast<int>(blockIdx.x) - q.rfirst;
    const int nb = (q.N + 63) / 64;
    const int b = local / nb, n = (local % nb) * 64 + static_cast<int>(threadIdx.x & 63);
    const float *p = q.P + static_cast<int64_t>(b) * q.S * q.N + n;
    const float sum = reduce_slices(p, q.N, q.S, n < q.N);
    if (threadIdx.x < 64 && n < q.N) q.Y[static_cast<int64_t>(b) * q.ldy + n] = f32_to_bf16(sum);
}

template <int MR, bool VEC, bool EP>
hipError_t launch_mr(const uint16_t *X, const uint16_t *W, const int32_t *idx, int64_t B, int64_t M,
                     int64_t N, int64_t K, int64_t k, int64_t ldx, int64_t ldw, uint16_t *Y,
                     int64_t ldy, float *P, int SR, int S, const Epilogue &ep, hipStream_t stream) {
    using namespace gv;
    dim3 grid(static_cast<unsigned>((N + CW - 1) / CW), static_cast<unsigned>(S), static_cast<unsigned>(B));
    if (S == 1) {
        hipLaunchKernelGGL((gemv_partial_kernel<MR, VEC, true, EP>), grid, dim3(NT), 0, stream, X, W, idx,
                           P, Y, static_cast<int>(M), static_cast<int>(N), static_cast<int>(K),
                           static_cast<int>(k), ldx, ldw, ldy, SR, S, ep);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((gemv_partial_kernel<MR, VEC, false>), grid, dim3(NT), 0, stream, X, W, idx,
                       P, Y, static_cast<int>(M), static_cast<int>(N), static_cast<int>(K),
                       static_cast<int>(k), ldx, ldw, ldy, SR, S, Epilogue{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    dim3 rgrid(static_cast<unsigned>((N + 63) / 64), static_cast<unsigned>(M), static_cast<unsigned>(B));
    hipLaunchKernelGGL(gemv_reduce_kernel<EP>, rgrid, dim3(256), 0, stream, P, Y, static_cast<int>(M),
                       static_cast<int>(N), S, ldy, ep);
    return hipGetLastError();
}

template <bool VEC, bool EP>
hipError_t launch_vec(const uint16_t *X, const uint16_t *W, const int32_t *idx, int64_t B, int64_t M,
                      int64_t N, int64_t K, int64_t k, int64_t ldx, int64_t ldw, uint16_t *Y,
                      int64_t ldy, float *P, int SR, int S, const Epilogue &ep, hipStream_t stream) {
    auto go = [&](auto mr) {
        return launch_mr<decltype(mr)::value, VEC, EP>(X, W, idx, B, M, N, K, k, ldx, ldw, Y, ldy, P, SR, S, ep, stream);
    };
    if (M == 1) return go(std::integral_constant<int, 1>{});
    if constexpr (VEC && EP) {
        const dim3 grid(static_cast<unsigned>((N + gv::CW - 1) / gv::CW), static_cast<unsigned>(S), static_cast<unsigned>(B));
        auto quads = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(gv::NT), 0, stream, X, W, idx, P, Y, static_cast<int>(M),
                               static_cast<int>(N), static_cast<int>(K), static_cast<int>(k), ldx, ldw, ldy, SR, S, ep);
            return hipGetLastError();
        };
        const hipError_t e = M <= 4 ? quads(gemv_quad_kernel<1, EP>) : quads(gemv_quad_kernel<2, EP>);
        if (e != hipSuccess || S == 1) return e;
        hipLaunchKernelGGL(gemv_reduce_kernel<EP>, dim3(static_cast<unsigned>((N + 63) / 64), static_cast<unsigned>(M),
                                                       static_cast<unsigned>(B)), dim3(256), 0, stream, P, Y,
                           static_cast<int>(M), static_cast<int>(N), S, ldy, ep);
        return hipGetLastError();
    } else {
        if (M == 2) return go(std::integral_constant<int, 2>{});
        if (M <= 4) return go(std::integral_constant<int, 4>{});
        return go(std::integral_constant<int, 8>{});
    }
}

}  // namespace

// Rows per slice (a multiple of 4) and slice count: enough workgroups to
// keep every CU streaming, at least MIN_SLICE rows per slice.
void gemv_slices(int64_t B, int64_t N, int64_t k, int *SR, int *S) {
    const int64_t chunks = (N + gv::CW - 1) / gv::CW;
    int64_t s = (gv::TARGET_BLOCKS + B * chunks - 1) / (B * chunks);
    const int64_t smax = (k + gv::MIN_SLICE - 1) / gv::MIN_SLICE;
    if (s > smax) s = smax;
    if (s < 1) s = 1;
    int64_t sr = (k + s - 1) / s;
    sr = (sr + 3) / 4 * 4;
    *SR = static_cast<int>(sr);
    *S = static_cast<int>((k + sr - 1) / sr);
}

size_t gemv_workspace_bytes(int64_t B, int64_t M, int64_t N, int64_t k) {
    int SR, S;
    gemv_slices(B, N, k, &SR, &S);
    return S == 1 ? 0 : static_cast<size_t>(B) * S * M * N * sizeof(float);
}

hipError_t launch_gemv_grouped_bf16(GemvGroups G, int64_t B, hipStream_t stream) {
    int blocks = 0, rblocks = 0;
    for (int i = 0; i < G.n; ++i) {
        GemvGroup &q = G.g[i];
        gemv_slices(B, q.N, q.k, &q.SR, &q.S);
        q.chunks = (q.N + gv::CW - 1) / gv::CW;
        q.first = blocks;
        blocks += q.chunks * q.S * static_cast<int>(B);
        q.rfirst = rblocks;
        if (q.S > 1) rblocks += (q.N + 63) / 64 * static_cast<int>(B);
    }
    hipLaunchKernelGGL(gemv_partial_grouped_kernel, dim3(static_cast<unsigned>(blocks)), dim3(gv::NT), 0,
                       stream, G);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || rblocks == 0) return e;
    hipLaunchKernelGGL(gemv_reduce_grouped_kernel, dim3(static_cast<unsigned>(rblocks)), dim3(256), 0,
                       stream, G);
    return hipGetLastError();
}

hipError_t launch_gemv_bf16(const uint16_t *X, const uint16_t *W, const int32_t *idx, int64_t B,
                            int64_t M, int64_t N, int64_t K, int64_t k, int64_t ldx, int64_t ldw,
                            uint16_t *Y, int64_t ldy, void *workspace, const Epilogue *ep,
                            hipStream_t stream) {
    int SR, S;
    gemv_slices(B, N, k, &SR, &S);
    const bool vec = ldw % 8 == 0 && reinterpret_cast<uintptr_t>(W) % 16 == 0;
    float *P = static_cast<float *>(workspace);
    auto go = [&](auto kernels, const Epilogue &e) {
        return kernels(X, W, idx, B, M, N, K, k, ldx, ldw, Y, ldy, P, SR, S, e, stream);
    };
    if (ep) return vec ? go(launch_vec<true, true>, *ep) : go(launch_vec<false, true>, *ep);
    return vec ? go(launch_vec<true, false>, Epilogue{}) : go(launch_vec<false, false>, Epilogue{});
}

}  // namespace rmm
