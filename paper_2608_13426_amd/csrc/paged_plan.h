// How the work of an attention call over the paged cache lies on one line, and
// what a workgroup finds at a place of it.  Plain arithmetic: the host compiles
// it too, so that the cover can be checked without a GPU.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_cache.h"

namespace rmm {

namespace {

namespace pg {
// Units of at most kShort blocks, no more of them than workgroups, are never cut
// (the host then leaves out the joining launch).  One token, 32 heads of 128 on 8:
// 500 keys uncut 11.3 us, cut 9.9 + 3.9 and a launch; 1000 keys uncut 16.4, cut
// 10.0 + 3.9, which is even with the launch and leaves the card to others.
constexpr int kShort = 16;

// x, which is the same in every lane, in a scalar register
__host__ __device__ __forceinline__ int uniform(int x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_readfirstlane(x);
#else
    return x;
#endif
}
// a / b of non-negative values
__host__ __device__ __forceinline__ int quot(int a, int b) {
    return uniform(static_cast<int>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)));
}

// ---- the line.  TK keys per block, ROWS query rows per unit.  The host keeps its
// length below 2^30 (paged_line_fits).
struct Seq {
    int q0, n, len;                       // first token, new tokens, keys
    int bad;                              // longer than its row of the page table
};
template <int TK, int ROWS>
struct Plan {
    int grp, causal, Hkv;
    bool whole;                           // units count one each (all are short)

    __host__ __device__ __forceinline__ Seq load(const PagedArgs &a, int b) const {
        Seq s;
        int q1;
        if (a.q_start) {
            s.q0 = min(max(a.q_start[b], 0), static_cast<int>(a.T));
            q1 = min(a.q_start[b + 1], static_cast<int>(a.T));
        } else {
            s.q0 = b;
            q1 = b + 1;
        }
        s.n = max(q1 - s.q0, 0);
        const int cap = a.width << a.kv.lg_page, len = max(a.lens[b], 0);
        s.bad = len > cap;
        s.len = min(len, cap);
        return s;
    }
    __host__ __device__ __forceinline__ int tiles(const Seq &s) const {
        return static_cast<int>((static_cast<uint32_t>(s.n * grp) + ROWS - 1) / ROWS);
    }
    // keys that some row of a tile sees (at most; the last token of the tile given)
    __host__ __device__ __forceinline__ int keys(const Seq &s, int last_tok) const {
        return causal ? min(max(s.len - s.n + last_tok + 1, 0), s.len) : s.len;
    }
    __host__ __device__ __forceinline__ int last_token(const Seq &s, int tile) const {
        return min(static_cast<int>((static_cast<uint32_t>(tile) * ROWS + ROWS - 1) / static_cast<uint32_t>(grp)), s.n - 1);
    }
    __host__ __device__ __forceinline__ int blocks(const Seq &s, int tile) const {
        return max((keys(s, last_token(s, tile)) + TK - 1) / TK, 1);
    }
    // length on the line of a pair of tiles (p, 2 np - 1 - p)
    __host__ __device__ __forceinline__ int pair(const Seq &s, int np) const {
        if (np == 1 || !causal) return blocks(s, 0) + blocks(s, 2 * np - 1);
        const int tok = static_cast<int>((static_cast<uint32_t>(np) * 2 * ROWS - 1) / static_cast<uint32_t>(grp));    // of a full last tile
        const int k = min(max(s.len - s.n + tok + 1, 1), s.len + ROWS);
        return blocks(s, 0) + (k + TK - 1) / TK + 2;
    }
    __host__ __device__ __forceinline__ int units(const Seq &s) const { return tiles(s) * Hkv; }
    // a sequence's share of the line per kv head
    __host__ __device__ __forceinline__ int head_work(const Seq &s) const {
        const int t = tiles(s), np = t >> 1;
        if (whole) return t;
        int w = np > 0 ? np * pair(s, np) : 0;
        if (t & 1) w += blocks(s, t - 1);
        return w;
    }
    __host__ __device__ __forceinline__ int work(const Seq &s) const { return head_work(s) * Hkv; }
    __host__ __device__ __forceinline__ int longest(const Seq &s) const {
        return s.n > 0 ? blocks(s, tiles(s) - 1) : 0;
    }
    // of two units that are neighbours when none is cut
    __host__ __device__ __forceinline__ int longest_pair(const Seq &s) const {
        const int t = tiles(s);
        return t > 1 ? blocks(s, 0) + blocks(s, t - 1) : 2 * longest(s);
    }
};

// A workgroup's place on the line
template <int TK, int ROWS>
struct Walk {
    Plan<TK, ROWS> pl;
    int wg;                               // the workgroup's place among the runs
    bool over;                            // sequences of more than T tokens between them: no line
    int x, begin, end, run;               // position, the workgroup's run, run length
    int b, f;                             // the sequence at x, where it begins
    Seq s;
    // the unit at x
    int kvh, tile, c0, c1;                // blocks [c0, c1) of it are in the run
    int u0, u1;                           // its place on the line

    // false: no work for this workgroup
    // min_run: shortest run; cut_cost: what cutting units costs, in blocks
    // (in paged_attn.hip: the wave's lanes look at the sequences together)
    __device__ bool init(const PagedArgs &a, int min_run, int cut_cost);
    // the unit at x (false: x is at no unit and has moved on, or at the end)
    __host__ __device__ __forceinline__ bool locate(const PagedArgs &a) {
        const int hw = pl.head_work(s);
        if (x >= f + hw * pl.Hkv) {       // the next sequence with work
            f += hw * pl.Hkv;
            const Seq q = pl.load(a, ++b);
            s = {uniform(q.q0), uniform(q.n), uniform(q.len), uniform(q.bad)};
            return false;
        }
        kvh = quot(x - f, hw);
        const int y = x - f - kvh * hw;
        if (pl.whole) {                   // one place per unit, late and early tiles in turn
            tile = y & 1 ? y >> 1 : hw - 1 - (y >> 1);
            u0 = x;
            u1 = x + 1;
            c0 = 0;
            c1 = pl.blocks(s, tile);
            return true;
        }
        const int t = pl.tiles(s), np = t >> 1;
        const int pr = np > 0 ? pl.pair(s, np) : 0;
        int off;
        if (y < np * pr) {
            const int p = quot(y, pr);
            off = y - p * pr;
            tile = p;
            const int wa = pl.blocks(s, p);
            if (off >= wa) {
                tile = 2 * np - 1 - p;
                const int wb = pl.blocks(s, tile);
                if (off >= wa + wb) {     // the rest of the pair's length is empty
                    x += pr - off;
                    return false;
                }
                off -= wa;
            }
        } else {
            tile = t - 1;
            off = y - np * pr;
        }
        u0 = x - off;
        u1 = u0 + pl.blocks(s, tile);
        c0 = off;
        c1 = min(end, u1) - u0;
        return true;
    }
    __host__ __device__ __forceinline__ void advance() { x = min(end, u1); }
    __host__ __device__ __forceinline__ bool complete() const { return u0 >= begin && u1 <= end; }
    // 1: the piece of a cut unit that begins in this run, 0: of one that began before it
    __host__ __device__ __forceinline__ int part() const { return u0 >= begin ? 1 : 0; }
};

}  // namespace pg

namespace few {
constexpr int kWaves = 4, kThreads = 64 * kWaves, TK = 32;
// Workgroups: two per CU, what the registers allow at once.  More wait their turn:
// 64 sequences of up to 1000 keys 43 us with 512, 54 with 768, 51 with 1024.
constexpr int kGroups = 512;
// Chunks in a run at least: two rounds of the four waves.  Half of it is 1 us
// faster at 1000 keys (9.1 for 10.0) and 3 slower at 8192 in the joining launch
// (7.4 for 4.8); twice is slower at both (12.5; 14.8 for 13.0).
constexpr int kMinRun = 8;
// What a cut unit costs, in chunks: 64 sequences of up to 1000 keys 43 us, 47 with
// 4, 43 with 16 (a unit's halves then end later than whole units elsewhere).
constexpr int kCutCost = 8;
}  // namespace few

namespace rowsk {
constexpr int NW = 8, NT = 64 * NW;       // waves of 32 query rows
constexpr int ROWS = 32 * NW, TK = 64, NS = 4;    // rows per unit, keys per tile, ring slots
constexpr int kGroups = 256;              // workgroups: one per CU
// In tiles.  Cutting costs a unit's 256 rows of partial sums written and read: a
// prompt of 4096 tokens, 32 heads, takes 166 + 5 us uncut and 192 + 42 cut.  Three
// sequences of 700 tokens behind up to 3300: cut 102 + 20, uncut (cost 32) 123 + 5.
constexpr int kMinRun = 4, kCutCost = 16;
}  // namespace rowsk

// Query rows per unit, by the average sequence's.  A unit reads its keys once, so
// small ones repeat reads (partly from a cache) and large ones spend matrix work and
// registers on rows that are not there.  Measured (us, heads of 128, 8 sequences of
// up to 9000 keys unless said, without the joining launch):
//   bf16    16 rows: 16 per unit 37, 32: 38;   24 rows: 42, 41;   40 rows: 64, 46
//   bf16    32 rows: 32 per unit 40, 256: 44;  64 rows: 49, 46;  128 rows: 72, 51
//           64 sequences: 24 rows 80, 93;  40 rows 122, 98;  128 rows 210, 116
//   4-bit   64 sequences: 24 rows, 16 per unit 59, 32: 50, 64: 60;  40 rows: 82, 81, 72
//   4-bit   64 per unit against 256: 128 rows 54, 72;  256 rows 57, 74;  32 sequences
//           of 256 rows 192, 179;  512 rows 100, 104.  Heads of 64: 40 rows 28, 30;
//           64 rows 91, 121;  128 rows 42, 34
// With a bf16 cache units of 64 rows were no better than 32 or 256 anywhere (40 rows
// 47, 128 rows 66, 64 sequences of 40 rows 95): there is none.  A 4-bit cache keeps
// them, since a 256-row unit turns every key into bf16 through registers into LDS.
int unit_rows(int64_t T, int64_t B, int64_t grp, bool mx, int D) {
    const int64_t rows = (T * grp + B - 1) / B;
    if (rows <= 16) return 16;
    if (rows <= 32) return 32;
    return mx && rows <= (D == 128 ? 256 : 64) ? 64 : rowsk::ROWS;
}
int workgroups(int rows) { return rows <= 64 ? few::kGroups : rowsk::kGroups; }
int block_keys(int rows) { return rows <= 64 ? few::TK : rowsk::TK; }
// units at most: full row tiles, and a last one per sequence
int64_t most_units(int64_t T, int64_t B, int64_t H, int64_t Hkv, int rows) {
    return T * H / rows + (T < B ? T : B) * Hkv;
}

// whether the joining launch is left out: no unit is cut whatever the lengths
bool never_cut(const PagedArgs &a, int rows) {
    return (static_cast<int64_t>(a.width) << a.kv.lg_page) <= pg::kShort * block_keys(rows) &&
           most_units(a.T, a.B, a.q.n, a.kv.Hkv, rows) <= a.nw;
}

}  // namespace

}  // namespace rmm
