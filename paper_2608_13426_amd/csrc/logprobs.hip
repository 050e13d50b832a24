// Log probabilities of given tokens, entropy and the most likely tokens of rows
// of logits z, read once (the read-out of a reduced output projection):
//
//   t_i = c (z_i - b),  c = scale log2(e),  S = sum 2^t_i,  D = sum t_i 2^t_i
//   log p_i = ln2 (c (z_i - b) - log2 S),   entropy = ln2 (log2 S - D / S)
//
// with one base b per wave, the largest logit it has seen: it moves about ln n
// times over n chunks, and the largest logit's weight is 1 without an error.
// z_i - b is formed before the product with c: a row whose logits are
// all the type's lowest value keeps its weights.  The lanes' fp32 sums are
// added in float64 and the logarithm is float64.
// Entropy is a sum of two terms of one sign: no cancellation.
//
// The largest logits are kept as 64-bit keys (the logit in the order of whole
// numbers, then the complement of its index: ties go to the lower index, -0
// equals +0, NaN above +infinity) in one sorted list per wave, lane i holding
// the i-th; a chunk of 512 logits whose maximum is not above the list's last
// costs one comparison.
//
// One workgroup per row, or per piece of a row where there are few rows; then a
// second launch joins the pieces.
#include <algorithm>

#include "block.h"
#include "device_common.h"

namespace rmm {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kChunk = 512;              // logits per wave step: 8 per lane
constexpr double kLn2 = 0.69314718055994530942;

struct Part {                            // one piece of a row
    double S, D;
    float b;
    int set;                             // whether b is (some logit above -infinity)
};

__device__ __forceinline__ uint32_t order32(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.f);          // -0 becomes +0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
// never 0, which stands for no key
__device__ __forceinline__ uint64_t make_key(float x, int i) {
    return (static_cast<uint64_t>(order32(x)) << 32) | (0x7fffffffu - static_cast<uint32_t>(i));
}
__device__ __forceinline__ int key_index(uint64_t k) { return static_cast<int>(0x7fffffffu - static_cast<uint32_t>(k)); }
// the key's logit; -0 reads as +0, any NaN as one
__device__ __forceinline__ float key_logit(uint64_t k) {
    const uint32_t o = static_cast<uint32_t>(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o == 0xffffffffu ? o : o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ uint64_t lane_key(uint64_t v, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), lane);
    return (static_cast<uint64_t>(hi) << 32) | lo;
}

// A wave's `top` largest keys, descending over its lanes.
struct TopList {
    uint64_t key;                        // this lane's
    uint64_t last;                       // the top-th, 0 while there are fewer
    float lim;                           // its logit: only what is above can enter
    int top;
    __device__ void init(int n) { key = 0; last = 0; lim = -__builtin_inff(); top = n; }
    __device__ bool full() const { return last != 0; }
    // every lane offers one key (0: none)
    __device__ void offer(uint64_t cand) {
        const int lane = threadIdx.x & 63;
        uint64_t todo = __ballot(cand > last);
        while (todo) {
            const int from = __builtin_ctzll(todo);
            const uint64_t k = lane_key(cand, from);
            const int pos = __popcll(__ballot(key > k));
            const uint64_t prev = __shfl_up(key, 1);
            key = lane < pos ? key : lane == pos ? k : prev;
            last = lane_key(key, top - 1);
            if (lane == from) cand = 0;
            todo = __ballot(cand > last);
        }
        lim = last ? key_logit(last) : -__builtin_inff();
    }
};

// A wave's softmax sums of the logits it has seen: b shared, s and d per lane.
struct Sums {
    float b, bmax, s, d;                 // bmax: b, or -infinity while it is not set
    bool set;
    __device__ void init() { b = 0.f; bmax = -__builtin_inff(); s = 0.f; d = 0.f; set = false; }
    // moves b to the largest of the lanes' values
    __device__ void rebase(float cm, float c) {
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1) cm = fmaxf(cm, __shfl_xor(cm, sh));
        if (set) {
            const float delta = (b - cm) * c, f = __builtin_amdgcn_exp2f(delta);
            d = f > 0.f ? (d + s * delta) * f : 0.f;
            s *= f;
        }
        b = bmax = cm;
        set = true;
    }
    template <bool ENT>
    __device__ void add(const float (&x)[8], float c) {
        float e[8], t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (x[i] - b) * c;
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(t[i]);
        s += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        if constexpr (ENT) {
            // a weight of zero (a logit of -infinity, or far below) adds nothing
#pragma unroll
            for (int i = 0; i < 8; ++i) d = fmaf(e[i], fmaxf(t[i], -1e30f), d);
        }
    }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) v += __shfl_xor(v, sh);
    return v;
}

// Sums of n parts, in order: the same in every thread.
__device__ __forceinline__ Part join_parts(const Part *p, int n, float c) {
    Part r = {0.0, 0.0, 0.f, 0};
    for (int i = 0; i < n; ++i) {
        if (!p[i].set) continue;
        if (!r.set || p[i].b > r.b) r.b = p[i].b;
        r.set = 1;
    }
    for (int i = 0; i < n; ++i) {
        if (!p[i].set) continue;
        const double delta = (static_cast<double>(p[i].b) - r.b) * c;
        const double f = delta == 0.0 ? 1.0 : exp2(delta);
        if (f == 0.0) continue;                              // nothing left of it
        r.S += f * p[i].S;
        r.D += f * (p[i].D + p[i].S * delta);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ float logit(const T *z, int64_t i) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(z[i]); else return z[i];
}

// A row's results from its sums and its list (thread i < top holds key i).
template <typename T>
__device__ __forceinline__ void write_row(const LogprobArgs &a, int64_t row, const Part &p, uint64_t key) {
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    const double ls = log2(p.S);
    // a row without a logit above -infinity has no weights: -infinity for every token
    auto logp = [&](float x) {
        if (!p.set) return -__builtin_inff();
        return static_cast<float>(((static_cast<double>(x) - p.b) * a.c - ls) * kLn2);
    };
    const int t = threadIdx.x;
    if (t == 0 && a.entropy) a.entropy[row] = p.set ? static_cast<float>((ls - p.D / p.S) * kLn2) : 0.f;
    for (int i = t; i < a.given; i += blockDim.x) {
        const int tok = a.tokens[row * a.given + i];
        a.logp[row * a.given + i] = tok >= 0 && tok < a.V ? logp(logit(z, tok)) : tok == -1 ? 0.f : __builtin_nanf("");
    }
    if (t < a.top) {
        a.top_idx[row * a.top + t] = key_index(key);
        a.top_logp[row * a.top + t] = logp(key_logit(key));
    }
}

// The workgroup's four lists as one: key i of the result in thread i < top.
__device__ __forceinline__ uint64_t join_lists(uint64_t key, int top) {
    __shared__ uint64_t lists[kWaves][kMaxTop], out[kMaxTop];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x < kMaxTop) out[threadIdx.x] = 0;
    lists[wave][lane] = lane < top ? key : 0;
    __syncthreads();
    if (lane < top && key != 0) {
        int rank = 0;
        for (int w = 0; w < kWaves; ++w)
            for (int i = 0; i < top; ++i) rank += lists[w][i] > key;
        if (rank < top) out[rank] = key;
    }
    __syncthreads();
    return threadIdx.x < kMaxTop ? out[threadIdx.x] : 0;
}

template <typename T, bool VEC, bool ENT>
__global__ __launch_bounds__(kThreads) void logprob_kernel(LogprobArgs a) {
    const int64_t row = blockIdx.x / a.pieces;
    const int piece = static_cast<int>(blockIdx.x - row * a.pieces);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    const int chunks = (a.V + kChunk - 1) / kChunk, full = a.V / kChunk;
    const int c0 = static_cast<int>(static_cast<int64_t>(chunks) * piece / a.pieces);
    const int c1 = static_cast<int>(static_cast<int64_t>(chunks) * (piece + 1) / a.pieces);
    Sums sums;
    sums.init();
    TopList list;
    list.init(a.top > 0 ? a.top : 1);

    // element e of this lane in chunk ch
    auto index = [&](int ch, int e) { return ch * kChunk + (VEC ? 8 * lane + e : lane + 64 * e); };
    auto load = [&](int ch, float (&x)[8]) {
        if (VEC && ch < full) {
            if constexpr (sizeof(T) == 2) {
                const uint4 q = *reinterpret_cast<const uint4 *>(z + index(ch, 0));
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[2 * e] = __uint_as_float(w[e] << 16);
                    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                }
            } else {
                const f32x4_t *p = reinterpret_cast<const f32x4_t *>(z + index(ch, 0));
                const f32x4_t u = p[0], v = p[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[e] = u[e]; x[4 + e] = v[e]; }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = index(ch, e);
                x[e] = i < a.V ? logit(z, i) : -__builtin_inff();
            }
        }
    };
    auto take = [&](int ch, const float (&x)[8]) {
        float cm = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) cm = fmaxf(cm, x[e]);
        if (__ballot(cm > sums.bmax)) sums.rebase(cm, a.c);
        sums.template add<ENT>(x, a.c);
        // a NaN among them has made s one
        if (a.top > 0 && (!list.full() || __ballot(cm > list.lim || sums.s != sums.s))) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = index(ch, e);
                list.offer(i < a.V ? make_key(x[e], i) : 0);
            }
        }
    };
    for (int ch = c0 + wave; ch < c1; ch += kWaves) {
        float x[8];
        load(ch, x);
        take(ch, x);
    }

    __shared__ Part parts[kWaves];
    const double S = wave_sum(sums.s), D = wave_sum(sums.d);
    if (lane == 0) parts[wave] = {S, D, sums.b, sums.set || S != S};
    const uint64_t key = a.top > 0 ? join_lists(list.key, a.top) : 0;
    __syncthreads();
    const Part p = join_parts(parts, kWaves, a.c);
    if (a.pieces == 1) {
        write_row<T>(a, row, p, key);
        return;
    }
    Part *out = static_cast<Part *>(a.part);
    uint64_t *keys = reinterpret_cast<uint64_t *>(out + a.T * a.pieces);
    if (threadIdx.x == 0) out[blockIdx.x] = p;
    if (threadIdx.x < a.top) keys[static_cast<int64_t>(blockIdx.x) * a.top + threadIdx.x] = key;
}

// The pieces of one row.
template <typename T>
__global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobArgs a) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Part *in = static_cast<const Part *>(a.part) + row * a.pieces;
    const uint64_t *keys = reinterpret_cast<const uint64_t *>(static_cast<const Part *>(a.part) + a.T * a.pieces) +
                           row * a.pieces * a.top;
    uint64_t key = 0;
    if (a.top > 0) {
        TopList list;
        list.init(a.top);
        for (int i = wave; i < a.pieces; i += kWaves) list.offer(lane < a.top ? keys[i * a.top + lane] : 0);
        key = join_lists(list.key, a.top);
    }
    write_row<T>(a, row, join_parts(in, a.pieces, a.c), key);
}

template <typename T, bool VEC>
hipError_t launch(const LogprobArgs &a, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.T * a.pieces));
    if (a.entropy)
        hipLaunchKernelGGL((logprob_kernel<T, VEC, true>), grid, dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((logprob_kernel<T, VEC, false>), grid, dim3(kThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.pieces == 1) return e;
    hipLaunchKernelGGL(logprob_join_kernel<T>, dim3(static_cast<unsigned>(a.T)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

// pieces of at least four chunks per wave, until there are about 1024 workgroups
int logprob_pieces(int64_t T, int64_t V) {
    const int64_t most = std::max<int64_t>(1, V / (4 * kWaves * kChunk));
    return static_cast<int>(std::max<int64_t>(1, std::min(most, 1024 / T)));
}

size_t logprob_workspace_bytes(int64_t T, int64_t V, int64_t top) {
    const int64_t n = logprob_pieces(T, V);
    return n == 1 ? 0 : static_cast<size_t>(T * n) * (sizeof(Part) + 8 * static_cast<size_t>(top));
}

hipError_t launch_logprobs(const LogprobArgs &a, bool bf16, bool vec, hipStream_t stream) {
    if (bf16) return vec ? launch<uint16_t, true>(a, stream) : launch<uint16_t, false>(a, stream);
    return vec ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace rmm
