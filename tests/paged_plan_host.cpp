// Host program over the arithmetic that lays an attention call's work on its line
// (csrc/paged_plan.h).  Per case of the input it walks every workgroup's run and
// checks that each key block of each unit is covered exactly once, that no unit is
// cut more finely than its pieces' places say, and prints what the case reaches.
//
// Input, numbers apart by white space: type (0 bf16, 1 4-bit), D, H, Hkv, causal,
// page size, page table width, T, B, 1 or 0 (q_start given), lengths [B], q_start
// [B + 1] if given.  Output per case, one line:
//   rows host_whole whole units run longest_piece most_units_of_a_workgroup cut blocks
// "over" where the sequences have more than T tokens between them, or "error ..." for a
// cover that is not exact.
#include <cstdio>
#include <map>
#include <tuple>
#include <vector>

#include "../paper_2608_13426_amd/csrc/paged_plan.h"

using namespace rmm;

namespace {

int error(const char *what, long a, long b) {
    std::printf("error %s %ld %ld\n", what, a, b);
    return 1;
}

// the sums over all sequences that a workgroup's lanes form together
template <int TK, int ROWS>
bool start(pg::Walk<TK, ROWS> &w, const PagedArgs &a, int wg, int min_run, int cut_cost, long &units, long &blocks) {
    auto &pl = w.pl;
    pl.grp = a.q.n / a.kv.Hkv;
    pl.causal = a.causal;
    pl.Hkv = a.kv.Hkv;
    pl.whole = false;
    long total = 0, tokens = 0;
    int most = 0, most2 = 0;
    units = 0;
    for (int b = 0; b < a.B; ++b) {
        const pg::Seq s = pl.load(a, b);
        most = max(most, pl.longest(s));
        most2 = max(most2, pl.longest_pair(s));
        total += pl.work(s);
        units += pl.units(s);
        tokens += s.n;
    }
    w.wg = wg;
    w.over = a.q_start && tokens > a.T;
    if (w.over) return false;
    blocks = total;
    const long rounds = (units + a.nw - 1) / a.nw, room = total / a.nw + cut_cost;
    pl.whole = a.whole || (rounds >> 1) * most2 + (rounds & 1) * most <= room;
    if (pl.whole) total = units;
    if (total >= 1l << 30) return false;
    w.run = static_cast<int>((total + a.nw - 1) / a.nw);
    w.run = pl.whole ? max(w.run, 1) : (max(w.run, min_run) + 3) / 4 * 4;
    const int runs = static_cast<int>((total + w.run - 1) / w.run), per = (runs + 7) >> 3;
    if ((wg >> 3) < per) w.wg = (wg & 7) * per + (wg >> 3);
    if ((wg >> 3) >= per || w.wg >= runs) return false;
    w.begin = w.x = w.wg * w.run;
    w.end = min(static_cast<int>(total) - w.x, w.run) + w.x;
    long f = 0;
    for (int b = 0;; ++b) {
        w.s = pl.load(a, b);
        if (f + pl.work(w.s) > w.x) {
            w.b = b;
            w.f = static_cast<int>(f);
            return true;
        }
        f += pl.work(w.s);
    }
}

template <int TK, int ROWS>
int check(const PagedArgs &a, int min_run, int cut_cost) {
    struct Piece {
        int c0, c1, n, first, slot;
        bool complete;
    };
    std::map<std::tuple<int, int, int>, std::map<int, Piece>> seen;     // (sequence, kv head, tile) -> by workgroup
    long units = 0, blocks = 0, piece = 0, most = 0, cut = 0;
    int run = 0, whole = 0;
    std::vector<int> places(a.nw, 0);
    for (int i = 0; i < a.nw; ++i) {
        pg::Walk<TK, ROWS> w;
        const bool any = start(w, a, i, min_run, cut_cost, units, blocks);
        if (w.over) {
            std::printf("over\n");
            return 0;
        }
        if (w.wg < 0 || w.wg >= a.nw || places[w.wg]++) return error("place", i, w.wg);
        run = w.run;
        whole = w.pl.whole;
        long n = 0, steps = 0;
        for (bool more = any; more; more = w.x < w.end) {
            if (++steps > 4l * a.B + 4 * (w.end - w.begin) + 16) return error("stuck", i, w.x);
            if (!w.locate(a)) continue;
            if (w.b >= a.B || w.kvh < 0 || w.kvh >= a.kv.Hkv || w.tile < 0 || w.tile >= w.pl.tiles(w.s) || w.c1 <= w.c0)
                return error("unit", i, w.x);
            const int first = w.u0 / w.run, last = (w.u1 - 1) / w.run;
            const Piece p = {w.c0, w.c1, last - first + 1, first, w.part(), w.complete()};
            if (!seen[{w.b, w.kvh, w.tile}].emplace(w.wg, p).second) return error("twice", i, w.x);
            piece = std::max(piece, static_cast<long>(w.c1 - w.c0));
            ++n;
            w.advance();
        }
        most = std::max(most, n);
    }
    long want = 0;
    pg::Plan<TK, ROWS> pl = {a.q.n / a.kv.Hkv, a.causal, a.kv.Hkv, false};
    for (int b = 0; b < a.B; ++b) {
        const pg::Seq s = pl.load(a, b);
        for (int h = 0; h < a.kv.Hkv; ++h)
            for (int t = 0; t < pl.tiles(s); ++t) {
                ++want;
                const auto it = seen.find({b, h, t});
                if (it == seen.end()) return error("missing", b, t);
                // every key that some row of the tile sees lies in the unit's blocks
                const int rows = min(ROWS, s.n * pl.grp - t * ROWS), tok = (t * ROWS + rows - 1) / pl.grp;
                const int keys = a.causal ? s.len - s.n + tok + 1 : s.len;
                if (pl.blocks(s, t) * TK < keys || (pl.blocks(s, t) - 1) * TK >= max(keys, 1)) return error("blocks", b, t);
                int c = 0, k = 0;
                const int n = static_cast<int>(it->second.size()), first = it->second.begin()->first;
                for (const auto &[wg, p] : it->second) {
                    if (p.c0 != c) return error("gap", b, t);
                    c = p.c1;
                    if (p.complete != (n == 1)) return error("complete", b, t);
                    if (n > 1 && (p.n != n || p.first != first || wg != first + k || p.slot != (k == 0))) return error("piece", b, t);
                    ++k;
                }
                if (c != pl.blocks(s, t)) return error("end", b, t);
                cut += n > 1;
            }
    }
    if (want != units || seen.size() != static_cast<size_t>(want)) return error("count", want, units);
    if (units > most_units(a.T, a.B, a.q.n, a.kv.Hkv, ROWS)) return error("units", units, 0);
    std::printf("%d %d %d %ld %d %ld %ld %ld %ld\n", ROWS, a.whole, whole, units, run, piece, most, cut, blocks);
    return 0;
}

}  // namespace

int main() {
    long mx, D, H, Hkv, causal, page, width, T, B, given;
    while (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld %ld %ld", &mx, &D, &H, &Hkv, &causal, &page, &width, &T, &B, &given) == 10) {
        std::vector<int32_t> lens(B), q_start(B + 1);
        for (auto &x : lens)
            if (std::scanf("%d", &x) != 1) return 2;
        if (given)
            for (auto &x : q_start)
                if (std::scanf("%d", &x) != 1) return 2;
        PagedArgs a = {};
        a.q.n = static_cast<int>(H);
        a.kv.Hkv = static_cast<int>(Hkv);
        while ((1l << a.kv.lg_page) < page) ++a.kv.lg_page;
        a.lens = lens.data();
        a.q_start = given ? q_start.data() : nullptr;
        a.width = static_cast<int>(width);
        a.B = static_cast<int>(B);
        a.T = T;
        a.causal = static_cast<int>(causal);
        const int rows = unit_rows(T, B, H / Hkv, mx != 0, static_cast<int>(D));
        a.nw = workgroups(rows);
        a.whole = never_cut(a, rows);
        if (rows == 16) check<few::TK, 16>(a, few::kMinRun, few::kCutCost);
        else if (rows == 32) check<few::TK, 32>(a, few::kMinRun, few::kCutCost);
        else if (rows == 64) check<few::TK, 64>(a, few::kMinRun, few::kCutCost);
        else check<rowsk::TK, rowsk::ROWS>(a, rowsk::kMinRun, rowsk::kCutCost);
        std::fflush(stdout);
    }
    return 0;
}
