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
#include <type_traits>

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
    int set;                             // some logit is above -infinity, or NaN
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

// the key of the lane before (lane 0: 0)
__device__ __forceinline__ uint64_t key_before(uint64_t k) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(k), 0x138, 0xF, 0xF, true);          // wave_shr:1
    const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(k >> 32), 0x138, 0xF, 0xF, true);
    return (static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo);
#else
    return k;
#endif
}

// LDS accesses of a wave's lanes stay in this order (the hardware keeps a wave's LDS
// accesses in program order)
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wave's `top` largest keys, descending over its lanes.
struct TopList {
    uint64_t key;                        // this lane's
    uint64_t last;                       // the top-th, 0 while there are fewer
    float lim;                           // its logit: only what is above can enter
    int top;
    uint64_t *scratch;                   // 64 keys of LDS, this wave's alone, 16-byte aligned
    __device__ void init(int n, uint64_t *lds) { key = 0; last = 0; lim = -__builtin_inff(); top = n; scratch = lds; }
    __device__ bool full() const { return last != 0; }
    __device__ void bound() {
        last = lane_key(key, top - 1);
        lim = last ? key_logit(last) : -__builtin_inff();
    }
    // every lane offers one key (0: none) to an empty list: each goes to the lane
    // that as many keys are larger.  Two keys per LDS read that all lanes share (1900
    // cycles; one by one from the other lanes' registers 3300)
    __device__ void fill(uint64_t cand) {
        const int lane = threadIdx.x & 63;
        scratch[lane] = cand;
        wave_lds_order();
        int rank = 0;
#pragma unroll 16
        for (int i = 0; i < 64; i += 2) {
            const ulonglong2 k = *reinterpret_cast<const ulonglong2 *>(scratch + i);
            rank += k.x > cand;
            rank += k.y > cand;
        }
        const int held = 64 - __popcll(__ballot(cand == 0));
        wave_lds_order();
        if (cand != 0) scratch[rank] = cand;
        wave_lds_order();
        key = lane < held ? scratch[lane] : 0;
        bound();
    }
    // every lane offers one key (0: none)
    __device__ void offer(uint64_t cand) {
        uint64_t todo = __ballot(cand > last);
        if (!todo) return;
        const int lane = threadIdx.x & 63;
        do {
            const int from = __builtin_ctzll(todo);
            const uint64_t k = lane_key(cand, from);
            const int pos = __popcll(__ballot(key > k));
            const uint64_t prev = key_before(key);
            key = lane < pos ? key : lane == pos ? k : prev;
            last = lane_key(key, top - 1);
            if (lane == from) cand = 0;
            todo = __ballot(cand > last);
        } while (todo);
        lim = last ? key_logit(last) : -__builtin_inff();
    }
};

template <int CTRL>
__device__ __forceinline__ float dpp_f32(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __uint_as_float(static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(x)), CTRL, 0xF, 0xF, false)));
#else
    return x;
#endif
}
__device__ __forceinline__ float lane_f32(float v, int lane) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
// over the wave, the same in every lane: lane ^ 1, lane ^ 2, mirrors of 8 and 16
// lanes, then the four rows of 16
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_f32<0xB1>(v));
    v = fmaxf(v, dpp_f32<0x4E>(v));
    v = fmaxf(v, dpp_f32<0x141>(v));
    v = fmaxf(v, dpp_f32<0x140>(v));
    return fmaxf(fmaxf(lane_f32(v, 0), lane_f32(v, 16)), fmaxf(lane_f32(v, 32), lane_f32(v, 48)));
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
    return __longlong_as_double(static_cast<long long>(lane_key(static_cast<uint64_t>(__double_as_longlong(v)), lane)));
}
__device__ __forceinline__ double wave_sum(double v) {
    v += dpp_f64<0xB1>(v);
    v += dpp_f64<0x4E>(v);
    v += dpp_f64<0x141>(v);
    v += dpp_f64<0x140>(v);
    return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}

// A wave's softmax sums of the logits it has seen: the base shared, s and d per
// lane.  As long as it can, t = fma(z, c, -base) with base = b c rounded to fp32
// (what that rounds is known, and taken out again at the end); in a wave that has
// met a logit of -infinity (0 times infinity in d) or a base past 4096, t =
// c (z - b), kept above -1e30: 8.5 operations per logit, an exponential
// counted as four, against 10.5.
struct Sums {
    float b, bmax, base, s, d;           // bmax: b, or -infinity while it is not set
    bool set, careful;
    __device__ void init() {
        b = 0.f; bmax = -__builtin_inff(); base = 0.f; s = 0.f; d = 0.f;
        set = false; careful = false;
    }
    // what base lacks of b c
    __device__ float rest(float c) const { return careful ? 0.f : fmaf(b, c, -base); }
    __device__ void take_care(float c) {
        const float r = rest(c), f = __builtin_amdgcn_exp2f(-r);
        d = (d - r * s) * f;
        s *= f;
        careful = true;
    }
    // moves b to the largest of the lanes' values
    __device__ void rebase(float cm, float c) {
        cm = wave_max(cm);
        const float nb = cm * c;
        if (!careful && !(fabsf(nb) < 4096.f)) take_care(c);
        if (set) {
            const float delta = careful ? (b - cm) * c : base - nb, f = __builtin_amdgcn_exp2f(delta);
            d = f > 0.f ? (d + s * delta) * f : 0.f;
            s *= f;
        }
        b = bmax = cm;
        base = nb;
        set = true;
    }
    template <bool ENT, bool CAREFUL>
    __device__ void add(const float (&x)[8], float c) {
        float e[8], t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = CAREFUL ? (x[i] - b) * c : fmaf(x[i], c, -base);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(t[i]);
        s += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        if constexpr (ENT) {
#pragma unroll
            for (int i = 0; i < 8; ++i) d = fmaf(e[i], CAREFUL ? fmaxf(t[i], -1e30f) : t[i], d);
        }
    }
};

// the largest float below x; NaN, which nothing compares with, for -infinity and NaN
__device__ __forceinline__ float below(float x) {
    const int u = static_cast<int>(__float_as_uint(x));
    if (!(x > -__builtin_inff())) return __builtin_nanf("");
    if (x == 0.f) return __uint_as_float(0x80000001u);
    return __uint_as_float(static_cast<uint32_t>(u > 0 ? u - 1 : u + 1));
}

// 2^delta for the weight of one base against another (delta <= 0): fp32, whose
// relative error 2^-24 |delta| meets a weight of 2^delta
__device__ __forceinline__ double base_weight(float b, float to, float c) {
    return b == to ? 1.0 : static_cast<double>(__builtin_amdgcn_exp2f((b - to) * c));
}

// The sums of n parts (n <= 64: lane i of every wave holds part i): the same in
// every lane.
__device__ __forceinline__ Part join_parts(Part mine, float c) {
    const float b = wave_max(mine.set ? mine.b : -__builtin_inff());
    Part r = {0.0, 0.0, b, __ballot(mine.set) != 0};
    // A NaN among a part's logits is in its S, never in its base (the largest of the
    // others, 0 without any): it reaches the row whatever that base weighs.
    const double f = mine.set ? base_weight(mine.b, b, c) : 0.0;
    const bool some = mine.set && (f != 0.0 || mine.S != mine.S);
    r.S = wave_sum(some ? f * mine.S : 0.0);
    r.D = wave_sum(some ? f * (mine.D + mine.S * static_cast<double>((mine.b - b) * c)) : 0.0);
    return r;
}

template <typename T>
__device__ __forceinline__ float logit(const T *z, int64_t i) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(z[i]); else return z[i];
}

// A row's results from its sums and its list (thread i < top holds key i).
template <typename T>
__device__ __forceinline__ void write_row(const LogprobArgs &a, int64_t row, const Part &p, uint64_t key) {
    const int t = threadIdx.x;
    if (t > 0 && t >= a.given && t >= a.top) return;
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    const double ls = log2(p.S);
    // a row without a logit above -infinity has no weights: -infinity for every token
    auto logp = [&](float x) {
        if (!p.set) return -__builtin_inff();
        const double v = ((static_cast<double>(x) - p.b) * a.c - ls) * kLn2;
        return v > 0.0 ? 0.f : static_cast<float>(v);        // what rounding left above 1
    };
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
    __shared__ __attribute__((aligned(16))) uint64_t lists[kWaves][kMaxTop], out[kMaxTop];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x < kMaxTop) out[threadIdx.x] = 0;
    lists[wave][lane] = lane < top ? key : 0;            // descending
    __syncthreads();
    if (lane < top && key != 0) {
        // its place: its own, and in each other list how many are larger
        int rank = lane;
        if (top <= 8) {                                      // by one read of each
#pragma unroll
            for (int w = 1; w < kWaves; ++w)
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const ulonglong2 k = *reinterpret_cast<const ulonglong2 *>(&lists[(wave + w) % kWaves][i]);
                    rank += k.x > key;
                    rank += k.y > key;
                }
        } else {                                             // by bisection
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                const uint64_t *l = lists[(wave + w) % kWaves];
                int n = 0;
#pragma unroll
                for (int step = kMaxTop / 2; step > 0; step /= 2) n += l[n + step - 1] > key ? step : 0;
                rank += n + (l[n] > key);
            }
        }
        if (rank < top) out[rank] = key;
    }
    __syncthreads();
    return threadIdx.x < kMaxTop ? out[threadIdx.x] : 0;
}

// 16 bytes at any address (global memory takes them at every alignment)
typedef uint32_t any16 __attribute__((ext_vector_type(4), aligned(2)));

// One chunk of a row: 8 logits of each lane, as loaded.
template <typename T>
struct Raw {
    static constexpr int N = sizeof(T) / 2;              // 16-byte loads
    uint4 q[N];
    __device__ float get(int e) const {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = (&q[0].x)[e >> 1];
            return __uint_as_float((e & 1) ? w & 0xffff0000u : w << 16);
        } else {
            return __uint_as_float((&q[e >> 2].x)[e & 3]);
        }
    }
};

// chunks per step of a wave: 64 bytes per lane
template <typename T>
constexpr int group_of = sizeof(T) == 2 ? 4 : 2;

template <typename T, bool ENT, int kGroup>
__global__ __launch_bounds__(kThreads) void logprob_kernel(LogprobArgs a) {
    const int64_t row = blockIdx.x / a.pieces;
    const int piece = static_cast<int>(blockIdx.x - row * a.pieces);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T *z = static_cast<const T *>(a.z) + row * a.ld;
    const int chunks = (a.V + kChunk - 1) / kChunk;
    const int c0 = static_cast<int>(static_cast<int64_t>(chunks) * piece / a.pieces);
    const int c1 = static_cast<int>(static_cast<int64_t>(chunks) * (piece + 1) / a.pieces);
    const int whole = min(c1, a.V / kChunk);             // chunks before this one are whole
    Sums sums;
    sums.init();
    TopList list;
    __shared__ __attribute__((aligned(16))) uint64_t scratch[kWaves][64];
    list.init(a.top > 0 ? a.top : 1, scratch[wave]);
    bool fresh = a.top > 0;

    // element e of this lane in chunk ch
    auto index = [&](int ch, int e) { return ch * kChunk + 8 * lane + e; };
    constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;   // -infinity
    auto load = [&](int ch, Raw<T> &r) {
        if (ch < whole) {
            const any16 *p = reinterpret_cast<const any16 *>(z + index(ch, 0));
#pragma unroll
            for (int i = 0; i < Raw<T>::N; ++i) r.q[i] = make_uint4(p[i].x, p[i].y, p[i].z, p[i].w);
            return;
        }
        uint32_t w[4 * Raw<T>::N];
#pragma unroll
        for (int i = 0; i < 4 * Raw<T>::N; ++i) w[i] = kNone;
        if (ch < c1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = index(ch, e);
                const float x = i < a.V ? logit(z, i) : -__builtin_inff();
                if constexpr (sizeof(T) == 2) {
                    const uint32_t u = __float_as_uint(x) >> 16;
                    w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xffffu) | (u << 16) : (w[e >> 1] & 0xffff0000u) | u;
                } else {
                    w[e] = __float_as_uint(x);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < Raw<T>::N; ++i) r.q[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    };
    // What the waves know of the row's top-th logit: nothing below the largest of their
    // own top-th (first half), nor below the smallest of their (top / 4)-th (second
    // half: the four hold that many above it together) can be among the top ones; what
    // equals it can, with a lower index.  Read whenever: an older value only lets more
    // through.  (The second half: 2048 rows of 128000, the 20 and 64 largest, 152 -> 135
    // and 239 -> 186 us; without any 101, the 5 largest 116.)
    __shared__ __attribute__((aligned(16))) volatile float limits[2 * kWaves];
    const int quarter = (a.top + kWaves - 1) / kWaves;
    auto publish = [&]() {
        const uint64_t k = lane_key(list.key, quarter - 1);
        const float q = k ? key_logit(k) : -__builtin_inff();
        if (lane == 0) {
            limits[wave] = list.lim;
            limits[kWaves + wave] = q == q ? q : __builtin_inff();       // NaN: above them all
        }
    };
    auto known = [&]() {
        static_assert(kWaves == 4, "two 16-byte reads");
        const f32x4_t l = *reinterpret_cast<const volatile f32x4_t *>(limits);
        const f32x4_t q = *reinterpret_cast<const volatile f32x4_t *>(limits + kWaves);
        return below(fmaxf(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])), fminf(fminf(q[0], q[1]), fminf(q[2], q[3]))));
    };
    __shared__ uint32_t words[kWaves][64 * 4 * Raw<T>::N * kGroup];
    if (lane < 2) limits[kWaves * lane + wave] = -__builtin_inff();
    // chunks ch, ch + kWaves, ... of a step; those past c1 are all -infinity
    auto take = [&](int ch, const Raw<T> (&r)[kGroup]) {
        float gm = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) gm = fmaxf(gm, r[u].get(e));
        if (__ballot(gm > sums.bmax)) sums.rebase(gm, a.c);
        auto add = [&](auto careful) {
#pragma unroll
            for (int u = 0; u < kGroup; ++u) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = r[u].get(e);
                sums.template add<ENT, decltype(careful)::value>(x, a.c);
            }
        };
        if (!sums.careful) {
            const float s0 = sums.s, d0 = sums.d;
            add(std::false_type{});
            if (ENT && __ballot(sums.d != sums.d)) {
                sums.s = s0;
                sums.d = d0;
                sums.take_care(a.c);
                add(std::true_type{});
            }
        } else {
            add(std::true_type{});
        }
        if (a.top == 0) return;
        // A NaN has made s one: from its first on every logit of the wave is offered (2048 x
        // 128000, the 5 largest: 108 us, with one NaN at the start of one row 136, of every row 305)
        const bool nan = __ballot(sums.s != sums.s) != 0;
        // nothing compares with a limit of NaN: all pass
        float lim = __builtin_nanf("");
        if (!nan && !fresh) {
            lim = known();
            if (list.full()) lim = fmaxf(list.lim, lim);
            if (!__ballot(!(gm <= lim))) return;
        }
        uint64_t best = 0;
        if (!nan) {
            // the lane's largest, the first of equal ones
            int i = index(ch, 0);
#pragma unroll
            for (int u = kGroup - 1; u >= 0; --u)
#pragma unroll
                for (int e = 7; e >= 0; --e) i = r[u].get(e) == gm ? index(ch + kWaves * u, e) : i;
            best = i < a.V && !(gm <= lim) ? make_key(gm, i) : 0;
            if (fresh) {
                // in order; few others are above the top-th of them (or equal to it,
                // with a lower index)
                list.fill(best);
                publish();
                lim = list.full() ? fmaxf(below(list.lim), known()) : known();
            } else {
                list.offer(best);
            }
        }
        fresh = false;
        int n = 0;
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) n += !(r[u].get(e) <= lim);
        // a lane's second, third ... are rare: in a short loop over LDS
        if (nan || __ballot(n > 1)) {
#pragma unroll
            for (int u = 0; u < kGroup; ++u)
#pragma unroll
                for (int i = 0; i < 4 * Raw<T>::N; ++i) words[wave][(4 * Raw<T>::N * u + i) * 64 + lane] = (&r[u].q[0].x)[i];
#pragma unroll 1
            for (int u = 0; u < kGroup; ++u) {
                Raw<T> t;
#pragma unroll
                for (int i = 0; i < 4 * Raw<T>::N; ++i) (&t.q[0].x)[i] = words[wave][(4 * Raw<T>::N * u + i) * 64 + lane];
                int more = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) more |= nan || !(t.get(e) <= lim) ? 1 << e : 0;
                if (n < 2 && !nan) more = 0;
                while (__ballot(more != 0)) {                // each lane's next
                    const int e = __builtin_ctz(more | 256);
                    float x = t.get(0);
#pragma unroll
                    for (int q = 1; q < 8; ++q) x = q == e ? t.get(q) : x;
                    const int i = index(ch + kWaves * u, e);
                    const uint64_t k = more != 0 && i < a.V && ch + kWaves * u < c1 ? make_key(x, i) : 0;
                    list.offer(k != best ? k : 0);
                    more &= more - 1;
                }
            }
        }
        publish();
    };
    Raw<T> cur[kGroup], next[kGroup];
    auto load_group = [&](int ch, Raw<T> (&r)[kGroup]) {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) load(ch + kWaves * u, r[u]);
    };
    constexpr int kStep = kGroup * kWaves;
    int ch = c0 + wave;
    if (ch < c1) load_group(ch, cur);
    lds_barrier();                       // the limits are set
    for (; ch < c1; ch += kStep) {
        if (ch + kStep < c1) load_group(ch + kStep, next);
        take(ch, cur);
#pragma unroll
        for (int u = 0; u < kGroup; ++u) cur[u] = next[u];
    }

    __shared__ Part parts[kWaves];
    const double r = sums.rest(a.c), f = 1.0 - kLn2 * r;         // 2^-r: r is at most 2^-12
    const double S0 = wave_sum(sums.s), S = f * S0, D = f * (wave_sum(sums.d) - r * S0);
    if (lane == 0) parts[wave] = {S, D, sums.b, sums.set || S != S};
    const uint64_t key = a.top > 0 ? join_lists(list.key, a.top) : 0;
    __syncthreads();
    if (wave > 0 && (a.pieces > 1 || (64 * wave >= a.given && 64 * wave >= a.top))) return;
    const Part p = join_parts(lane < kWaves ? parts[lane] : Part{0.0, 0.0, 0.f, 0}, a.c);
    if (a.pieces == 1) {
        write_row<T>(a, row, p, key);
        return;
    }
    Part *out = static_cast<Part *>(a.part);
    uint64_t *keys = reinterpret_cast<uint64_t *>(out + a.T * a.pieces);
    if (lane == 0) out[blockIdx.x] = p;
    if (lane < a.top) keys[row * a.pieces * a.top + lane * a.pieces + piece] = key;
}

// The pieces (at most kMaxPieces) of one row, by one wave.  The keys lie by rank,
// then by piece: 64 in a row hold one of every piece at least, so that once none
// of them enters nothing behind them can.
constexpr int kMaxPieces = 64;
template <typename T>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const Part *in = static_cast<const Part *>(a.part) + row * a.pieces;
    const int n = a.pieces * a.top;
    const uint64_t *keys = reinterpret_cast<const uint64_t *>(static_cast<const Part *>(a.part) + a.T * a.pieces) + row * n;
    auto read = [&](int i) -> uint64_t { return i + lane < n ? keys[i + lane] : 0; };
    uint64_t k = read(0), next = read(64);
    const Part p = join_parts(lane < a.pieces ? in[lane] : Part{0.0, 0.0, 0.f, 0}, a.c);
    __shared__ __attribute__((aligned(16))) uint64_t scratch[64];
    TopList list;
    list.init(a.top > 0 ? a.top : 1, scratch);
    if (a.top > 0) {
        list.fill(k);
        for (int i = 64; i < n; i += 64) {
            k = next;
            next = read(i + 64);
            if (!__ballot(k > list.last)) break;
            list.offer(k);
        }
    }
    write_row<T>(a, row, p, list.key);
}

// Up to 512 workgroups (2048 waves): one chunk per wave and step, so one step each up to
// 64 pieces' 131072 logits.  Beyond, steps of 64 bytes per lane.
bool one_step(int64_t T, int64_t V) { return T * std::min<int64_t>(kMaxPieces, (V + kWaves * kChunk - 1) / (kWaves * kChunk)) <= 512; }

template <typename T>
hipError_t launch(const LogprobArgs &a, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.T * a.pieces));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
        return hipGetLastError();
    };
    constexpr int G = group_of<T>;
    const hipError_t e = one_step(a.T, a.V) ? a.entropy ? go(logprob_kernel<T, true, 1>) : go(logprob_kernel<T, false, 1>)
                                            : a.entropy ? go(logprob_kernel<T, true, G>) : go(logprob_kernel<T, false, G>);
    if (e != hipSuccess || a.pieces == 1) return e;
    hipLaunchKernelGGL(logprob_join_kernel<T>, dim3(static_cast<unsigned>(a.T)), dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

// otherwise pieces of four chunks per wave or more, until there are about 1024 workgroups
int logprob_pieces(int64_t T, int64_t V) {
    const int64_t per = kWaves * kChunk * (one_step(T, V) ? 1 : 4), most = (V + per - 1) / per;
    return static_cast<int>(std::max<int64_t>(1, std::min({most, one_step(T, V) ? most : 1024 / T, int64_t(kMaxPieces)})));
}

size_t logprob_workspace_bytes(int64_t T, int64_t V, int64_t top) {
    const int64_t n = logprob_pieces(T, V);
    return n == 1 ? 0 : static_cast<size_t>(T * n) * (sizeof(Part) + 8 * static_cast<size_t>(top));
}

hipError_t launch_logprobs(const LogprobArgs &a, bool bf16, hipStream_t stream) {
    return bf16 ? launch<uint16_t>(a, stream) : launch<float>(a, stream);
}

}  // namespace rmm
