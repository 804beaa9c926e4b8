// Work lists of the matrix products, walked on the host: every tile, or every part of a divided one, is one workgroup's in one round, and a workgroup's list has no
// gaps.  Grids of the planners over many sizes, and the room that their parts take.  Host code only.
#include <cstdio>
#include <cstdlib>
#include <ctime>
#include <random>
#include <vector>

#include "wlb_dense.h"

static int cus = 256;
namespace wlb {
int compute_units() { return cus; }
}  // namespace wlb
using namespace wlb;

static long long grids = 0, divided = 0, items = 0;

// lists that are walked item by item: larger ones would take minutes, and none is where plans are timed
static bool walking = true;
static bool walkable(const GemmGrid& g) { return walking && (long long)g.ntm * g.ntn <= 20000; }

static void walk(const GemmGrid& g, const char* what) {
    const int tiles = g.ntm * g.ntn, steps = (g.depth + kStepK - 1) / kStepK;
    ++grids;
    divided += g.left > 0;
    auto wrong = [&](const char* text, int a, int b) {
        printf("%s: %s (%d, %d): %d x %d tiles, depth %d, %d workgroups, %d whole, %d in %d parts\n", what, text, a, b, g.ntm, g.ntn, g.depth, g.workgroups, g.whole, g.left, g.parts);
        exit(1);
    };
    if (g.workgroups < kLists || g.workgroups % kLists || g.whole < 0 || g.left < 0 || g.parts < 1 || g.whole + g.left != tiles) wrong("grid", tiles, 0);
    std::vector<int> covered(tiles, 0), places(g.left * g.parts, 0);
    for (int b = 0; b < g.workgroups; ++b) {
        GemmItem it;
        int round = 0;
        for (; g.item(b, round, it); ++round) {
            ++items;
            if (it.tm < 0 || it.tm >= g.ntm || it.tn < 0 || it.tn >= g.ntn) wrong("place", it.tm, it.tn);
            if (it.part < 0) {
                if (it.k0 != 0 || it.depth != g.depth) wrong("whole tile's depth", it.k0, it.depth);
                covered[it.tn * g.ntm + it.tm] += std::max(steps, 1);
            } else {
                if (it.part >= g.left * g.parts) wrong("part", it.part, 0);
                if (it.k0 % kStepK || it.k0 + it.depth > g.depth || it.depth < 0) wrong("part's depth", it.k0, it.depth);
                // a tile's parts lie side by side, in the order of k
                GemmItem tile;
                g.place(g.whole + it.part / g.parts, tile);
                if (tile.tm != it.tm || tile.tn != it.tn) wrong("tile of a part", it.part, it.tm);
                if (it.k0 / kStepK != (int)((long long)steps * (it.part % g.parts) / g.parts)) wrong("order of parts", it.part, it.k0);
                covered[it.tn * g.ntm + it.tm] += (it.depth + kStepK - 1) / kStepK;
                ++places[it.part];
            }
        }
        for (int later = 1; later <= 2; ++later)
            if (g.item(b, round + later, it)) wrong("gap in the list of workgroup", b, round);
    }
    for (int t = 0; t < tiles; ++t)
        if (covered[t] != std::max(steps, 1)) wrong("steps of a tile, instead of each once", covered[t], steps);
    for (int p = 0; p < g.left * g.parts; ++p)
        if (places[p] != 1) wrong("times that a part is computed", places[p], p);
}

static ProductArgs product(int pm, int qn, int depth, int twin = 0) {
    ProductArgs a = {};
    a.pm = pm; a.qn = qn; a.depth = depth; a.twin = twin;
    return a;
}

static int groups[8] = {}, tiles[6] = {};
static size_t room = 0, largest_need = 0;         // bytes for parts in the calls of the operator that is looked at, and what its plans took most

static void takes(int kind, const GemmGrid& g, const char* what) {
    const size_t need = parts_bytes(kind, g);
    largest_need = std::max(largest_need, need);
    if (need > room) { printf("%s: parts of %zu bytes, room for %zu\n", what, need, room); exit(1); }
}
static void alone(Kinds kinds, const ProductArgs& a, const char* what) {
    const Tiling t = plan_product(kinds, a);
    ++tiles[t.kind];
    takes(t.kind, t.grid, what);
    if (walkable(t.grid)) walk(t.grid, what);
}
static void slots(Kinds kinds, int pm, int rows, int depth, int end, const char* what) {
    const Tiling t = plan_slots(kinds, pm, rows, depth, end);
    ++tiles[t.kind];
    takes(t.kind, t.grid, what);
    if (walkable(t.grid)) walk(t.grid, what);
}

// The gradients of an operator, as the calls plan them.
static void gradients(int rows, int twin, int dx_pm, int dx_depth, std::vector<std::pair<int, int>> weights, const char* what) {
    GroupArgs g = {};
    g.n = 1;
    if (dx_pm) g.a[0] = product(dx_pm, rows, dx_depth, twin);
    for (auto& w : weights) g.a[g.n++] = product(w.first, w.second, rows);
    const Group kind = plan_gradients(g);
    ++groups[kind];
    if (kind == kApart) {
        if (dx_pm) alone(Kinds::MK, g.a[0], what);
        for (int k = 1; k < g.n; ++k) alone(Kinds::MM, g.a[k], what);
        return;
    }
    for (int k = 0; k < g.n; ++k) takes(group_tiles(kind), g.a[k].grid, what);
    for (int k = 0; k < g.n; ++k)
        if (g.a[k].qn && walkable(g.a[k].grid)) {
            if (g.a[k].grid.workgroups != g.a[g.n - 1].grid.workgroups || g.turn[k] < 0 || g.turn[k] >= g.a[k].grid.workgroups / kLists) { printf("%s: launch\n", what); exit(1); }
            if (g.a[k].grid.left && k != (rows <= kFewSlots ? 0 : g.n - 1)) { printf("%s: a product that no join follows is divided\n", what); exit(1); }
            walk(g.a[k].grid, what);
        }
}
// All launches of an operator's calls, with any of their outputs left out.
static void linear(int n, int n_in, int n_out, int act) {
    const int twin = act && n <= kExactSlots ? n : 0, rows = twin ? 2 * n : n;
    room = linear_parts_bytes(n, n_in, n_out, act);
    largest_need = 0;
    ProductArgs y = product(n_out, n, n_in);
    y.act = act;
    alone(Kinds::KK, y, "product");
    __bf16 some;
    y.residual = &some;
    alone(Kinds::KK, y, "product with a residual");
    gradients(rows, twin, n_in, n_out, {{n_in, n_out}}, "gradients of a product");
    gradients(rows, twin, n_in, n_out, {}, "gradient of x");
    gradients(rows, twin, 0, 0, {{n_in, n_out}}, "gradient of the weight");
}
static void ffn(int n, int hidden, int inner, int act) {
    const int twin = n <= kExactSlots ? n : 0, rows = twin ? 2 * n : n;
    room = ffn_parts_bytes(n, hidden, inner);
    largest_need = 0;
    for (int end : {0, 2000, 8000, 11000}) slots(Kinds::KK, 2 * inner, n, hidden, end, "gate");
    ProductArgs y = product(hidden, rows, inner, twin);
    alone(Kinds::KK, y, "product with Wd");
    __bf16 some;
    y.residual = &some;
    alone(Kinds::KK, y, "product with Wd and a residual");
    slots(Kinds::MK, inner, n, hidden, 20000, "inner gradient");
    for (int which = 1; which < 8; ++which) {
        std::vector<std::pair<int, int>> w;
        if (which & 2) w.push_back({hidden, 2 * inner});
        if (which & 4) w.push_back({inner, hidden});
        gradients(rows, twin, which & 1 ? hidden : 0, 2 * inner, w, "gradients of a feed-forward block");
    }
}

// What plan_group says a group should take, against the time of every workgroup of an XCD added up tile by tile.
template <class S>
static void group_time(GroupArgs g, const TileCost& c) {
    const long long said = plan_group<S>(g, c);
    const int side = wide_workgroups() * (S::RING ? 1 : 2) / kLists;
    std::vector<long long> load(side, 0);
    long long most = 0, last = 0;
    for (int k = 0; k < g.n; ++k) {
        const GemmGrid& q = g.a[k].grid;
        if (g.a[k].qn == 0) continue;
        const long long steps = std::max(2, (q.depth + kStepK - 1) / kStepK), per = (q.whole + kLists - 1) / kLists;
        for (long long i = 0; i < per; ++i) load[(g.turn[k] + i) % side] += steps * c.step + c.end;
        most = *std::max_element(load.begin(), load.end());
        if (q.left) {
            const int parts = q.left * q.parts, share = (parts + kLists - 1) / kLists, from = g.turn[k] + (int)(per % side) + q.lead;
            for (int i = 0; i < std::min(share, side); ++i) last = std::max(last, load[(from + i) % side]);
            most = std::max(most, last + (steps + q.parts - 1) / q.parts * c.step + c.end) + kJoinLaunch + (long long)parts * c.join;
        }
    }
    if (said != most) { printf("a group's time: %lld, tile by tile %lld\n", said, most); exit(1); }
}
static void group_times(int n, int hidden, int inner) {
    GroupArgs g = {};
    g.n = 3;
    g.a[0] = product(hidden, n, 2 * inner); g.a[1] = product(hidden, 2 * inner, n); g.a[2] = product(inner, hidden, n);
    group_time<Wide<true, true>>(g, kWideCost);
    group_time<Small<true, true>>(g, kSmallCost);
    group_time<Tiny<true, true>>(g, kTinyCost);
}

// The largest calls: a plan is a few divisions, whatever the number of tiles.
static int largest() {
    walking = false;
    const clock_t start = clock();
    for (int k = 0; k < 10; ++k) {
        linear(1990000, 1 << 20, 1 << 20, true);
        ffn(1990000, 2040, 1 << 19, 7);
    }
    const double ms = 1e3 * (double)(clock() - start) / CLOCKS_PER_SEC / 20;
    printf("plans of a largest call, with any of its outputs left out: %.4f ms\n", ms);
    return ms < 5 ? 0 : 1;
}

int main(int argc, char** argv) {
    if (argc > 1) return largest();
    std::mt19937 rng(5);
    auto spread = [&](int lo, int hi) { return (int)std::exp(std::uniform_real_distribution<double>(std::log((double)lo), std::log(hi + 1.0))(rng)); };
    auto width = [&](int hi) { return std::max(8, spread(8, hi) / 8 * 8); };

    // sizes whose last product is divided in a group, with workgroups that have no whole tile in the last round
    ffn(7680, 1024, 4096, 2);
    ffn(5376, 1024, 4096, 2);
    ffn(4096, 3080, 8192, 2);
    ffn(7168, 4096, 14336, 2);
    ffn(7691, 2624, 1328, 2);
    ffn(5061, 152, 2600, 2);
    linear(4189, 1544, 5000, 3);
    int full = 0;
    for (int i = 0; i < 3000; ++i) {
        cus = i % 8 == 6 ? 32 : i % 8 == 7 ? 304 : 256;
        const int n = spread(1, i % 3 ? 40000 : 200);
        linear(n, width(16384), width(16384), i % 4);
        full += largest_need == room;
        ffn(n, width(8192), width(16384), 2);
        full += largest_need == room;
    }
    cus = 256;
    for (int i = 0; i < 2000; ++i) group_times(spread(1, 20000), width(4096), width(8192));
    for (int i = 0; i < 3000; ++i) {
        const int pm = width(32768), qn = spread(1, 40000), depth = spread(1, 32768);
        const Tiling t = best_tiling(pm, qn, depth, (int)(rng() % 3) * 6000);
        if (walkable(t.grid)) walk(t.grid, "tiling");
        const GemmGrid g = planned_grid((pm + 255) / 256, (qn + 255) / 256, depth, 256, kWideParts, kWideRounds);
        const GemmGrid same((pm + 255) / 256, (qn + 255) / 256, depth, 256, kWideParts, kWideRounds);
        if (g.whole != same.whole || g.left != same.left || g.parts != same.parts) { printf("the host's grid is not the device's\n"); return 1; }
        if (walkable(g)) walk(g, "wide tiles");
        long long cost = 0;
        for (int most : {0, 256}) {
            walk(narrow_grid(kTinyCost, pm, 64, depth, cost, true, most), "joined tiles");
            walk(narrow_grid(kSmallCost, pm, 300, depth, cost, false, most), "narrow tiles");
        }
        walk(few_grid((pm + 127) / 128, depth), "few slots");
        walk(joined_grid((pm + 127) / 128, depth, 256), "few slots, joined");
    }
    // any grid that a planner could come to
    for (int i = 0; i < 20000; ++i) {
        GemmGrid g;
        g.ntm = spread(1, 60); g.ntn = spread(1, 60);
        g.workgroups = kLists * spread(1, 64);
        g.left = (int)(rng() % 2) * (int)(rng() % (g.ntm * g.ntn + 1));
        g.whole = g.ntm * g.ntn - g.left;
        g.parts = g.left ? spread(1, kMaxParts) : 1;
        g.lead = (int)(rng() % (g.workgroups / kLists));
        g.depth = spread(1, 20000);
        walk(g, "any grid");
    }
    for (int k = 0; k < 6; ++k)
        if (!tiles[k]) { printf("tiles that no size here has: %d\n", k); return 1; }
    // small calls take little: 65 slots, 1024 x 1024, 2 MiB of parts, one of 64 x 64 its own tiles alone
    if (linear_parts_bytes(65, 1024, 1024, 0) > 4u << 20 || linear_parts_bytes(1, 64, 64, 0) > 0 || ffn_parts_bytes(1, 64, 64) > 64u << 10) {
        printf("room of small calls: %zu %zu %zu\n", linear_parts_bytes(65, 1024, 1024, 0), linear_parts_bytes(1, 64, 64, 0), ffn_parts_bytes(1, 64, 64));
        return 1;
    }
    printf("room taken as a whole: %d of 6000; work lists: ok: %lld grids, %lld divided, %lld items; gradients", full, grids, divided, items);
    for (int k = 0; k < 8; ++k) printf(" %d", groups[k]);
    printf("\n");
    for (int k = 0; k < 8; ++k)
        if (!groups[k]) { printf("a kind of launch that no size here has\n"); return 1; }
    return 0;
}
