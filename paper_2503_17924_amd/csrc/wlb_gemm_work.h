// Work lists, joins and launches of the matrix products of wlb_gemm.h.
#pragma once
#include <algorithm>

#include "wlb_gemm.h"
#include "wlb_internal.h"

namespace wlb {

// Tiles.  `Slots32` .. `Slots128` serve calls of few slots: four wavefronts side by side along the words (or columns).
template <bool MP, bool MQ> using Wide = GemmShape<2, 2, 8, 8, MP, MQ>;
template <bool MP, bool MQ> using Half = GemmShape<2, 2, 4, 4, MP, MQ>;
template <bool MP, bool MQ> using Slots128 = GemmShape<4, 1, 4, 8, MP, MQ>;
template <bool MP, bool MQ> using Slots64 = GemmShape<4, 1, 4, 4, MP, MQ>;
template <bool MP, bool MQ> using Slots32 = GemmShape<4, 1, 4, 2, MP, MQ>;

// ------------------------------------------------------------------------------------------
// Products and their work lists.  A wide tile is divided along k (GemmGrid) into parts of kWideParts steps and more, in up to kWideRounds rounds; narrow ones, which
// few slots leave to a few workgroups, into parts of kNarrowParts and more for dX, else never.
constexpr int kWideParts = 8, kWideRounds = 2, kNarrowParts = 4, kNever = 1 << 30;

struct Work : GemmGrid {
    const __bf16 *p_at, *q_at;
    long long ldp, ldq;
    int pm, qn;                      // rows or columns of the operands
    const int32_t* list;             // rows of q, or null
    int tile_m, tile_n;
    bool p_down, q_down;             // operand kind M: k runs down the rows
    template <class S>
    static __device__ __forceinline__ Work make(const __bf16* p, long long ldp, int pm, const __bf16* q, long long ldq, int qn, const int32_t* list, int depth,
                                                int workgroups, int narrow_parts) {
        Work w(GemmGrid((pm + S::TM - 1) / S::TM, (qn + S::TN - 1) / S::TN, depth, workgroups, S::RING ? kWideParts : narrow_parts,
                        S::RING ? kWideRounds : 1));
        w.p_at = p; w.q_at = q; w.ldp = ldp; w.ldq = ldq; w.pm = pm; w.qn = qn; w.list = list;
        w.tile_m = S::TM; w.tile_n = S::TN; w.p_down = S::MP; w.q_down = S::MQ;
        return w;
    }
    __device__ __forceinline__ explicit Work(const GemmGrid& g) : GemmGrid(g) {}
    __device__ __forceinline__ GemmOperand p(const GemmItem& i) const {
        const int m0 = i.tm * tile_m;
        return GemmOperand{p_down ? p_at + (long long)i.k0 * ldp + m0 : p_at + (long long)m0 * ldp + i.k0, pm - m0, nullptr};
    }
    __device__ __forceinline__ GemmOperand q(const GemmItem& i) const {
        const int n0 = i.tn * tile_n;
        if (list) return GemmOperand{q_at + i.k0, qn - n0, list + n0};
        return GemmOperand{q_down ? q_at + (long long)i.k0 * ldq + n0 : q_at + (long long)n0 * ldq + i.k0, qn - n0, nullptr};
    }
};

// Joins the parts of divided tiles in order: f(tm, tn, n, m, four sums).  A row n of a tile is a wavefront's, of a narrow tile, which has up to kMaxParts parts, a
// workgroup's, whose wavefronts add up a quarter of the parts each.
template <class S, class W, class F>
__device__ __forceinline__ void join_parts(const W& w, const float* parts, F f) {
    static_assert(S::TM == 256, "four columns a lane");
    __shared__ f32x4 s_sum[3][64];
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), id = S::RING ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x;
    GemmItem it;
    if (id >= w.left * S::TN) return;
    w.place(w.whole + id / S::TN, it);
    const int n = id % S::TN;
    if (it.tn * S::TN + n >= w.qn) return;
    const int first = S::RING ? 0 : w.parts * wave / 4, end = S::RING ? w.parts : w.parts * (wave + 1) / 4;
    const f32x4* from = reinterpret_cast<const f32x4*>(parts + ((size_t)(id / S::TN) * w.parts * S::TN + n) * S::TM) + lane;
    f32x4 sum = {0, 0, 0, 0};
    constexpr int kAhead = 8;
    for (int k = first; k < end; k += kAhead) {
        f32x4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = from[(size_t)min(k + i, end - 1) * (S::TN * S::TM / 4)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (k + i < end) sum += v[i];
    }
    if (!S::RING) {
        if (wave > 0) s_sum[wave - 1][lane] = sum;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int i = 0; i < 3; ++i) sum += s_sum[i][lane];
    }
    f(it.tm, it.tn, n, lane * 4, sum);
}

// The same for tiles of 128 or 64 columns: half or a quarter of a wavefront to a row.  twin: rows behind the first `twin` are added to those (0: none are)
// where they are numbers: beside an infinite operand, which makes infinite what it meets in the first, the little or nothing that it meets in the others says nothing.
template <class S, class W, class F>
__device__ __forceinline__ void join_parts_narrow(const W& w, const float* parts, F f, int twin) {
    constexpr int LANES = S::TM / 4;
    static_assert(LANES == 32 || LANES == 16, "four columns a lane");
    const int lane = (int)threadIdx.x % LANES, id = (int)blockIdx.x * (256 / LANES) + (int)threadIdx.x / LANES;
    if (id >= w.left * S::TN) return;
    GemmItem it;
    w.place(w.whole + uniform(id / S::TN), it);         // a wavefront's rows lie in one tile
    const int n = id % S::TN;
    if (twin && n >= twin) return;
    const f32x4* from = reinterpret_cast<const f32x4*>(parts + ((size_t)(id / S::TN) * w.parts * S::TN + n) * S::TM) + lane;
    f32x4 sum = {0, 0, 0, 0}, rest = {0, 0, 0, 0};
    constexpr int kAhead = 8;
    for (int k = 0; k < w.parts; k += kAhead) {
        f32x4 v[kAhead], t[kAhead] = {};
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = from[(size_t)min(k + i, w.parts - 1) * (S::TN * S::TM / 4)];
        if (twin) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) t[i] = from[(size_t)min(k + i, w.parts - 1) * (S::TN * S::TM / 4) + (size_t)twin * (S::TM / 4)];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (k + i < w.parts) { sum += v[i]; rest += t[i]; }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __builtin_isfinite(rest[i]) ? rest[i] : 0.f;
    f(it.tm, it.tn, n, lane * 4, sum);
}

template <class S, class W, class F>
__device__ __forceinline__ void join_any(const W& w, const float* parts, F f, int twin = 0) {
    if constexpr (S::TM < 256) join_parts_narrow<S>(w, parts, f, twin);
    else join_parts<S>(w, parts, f);
}

// ------------------------------------------------------------------------------------------
// What the ends of tiles share.
// What belongs to a wavefront's rows n is loaded once for every row, 64 to a register, and fetched from the lane that holds it.
template <class S> constexpr int row_regs() { return (S::BN * 16 + 63) / 64; }
template <class S>
__device__ __forceinline__ int row_held(const Gemm<S>& g, const GemmItem& it, int k) { return it.tn * S::TN + g.wn * (S::BN * 16) + k * 64 + g.lane % (S::BN * 16); }
template <class T, int N>
__device__ __forceinline__ T of_row(const T (&regs)[N], int j, int lane) { return __shfl(regs[j / 4], (j % 4) * 16 + lane % 16); }

// Stores of a wavefront's part in rows_out<Bytes>, 1 KiB each, where no row or column lies past the end.
template <class S, int Bytes> constexpr int row_stores() { return S::BM * 16 * S::BN * 16 * Bytes / 1024; }

struct NothingAhead {
    struct Ahead {};
    template <class G>
    __device__ __forceinline__ Ahead load(const G&, const GemmItem&) const { return Ahead{}; }
};

// ------------------------------------------------------------------------------------------
// Launches.
inline int slot_tile(int n_q) { return n_q <= 32 ? 32 : n_q <= 64 ? 64 : n_q <= 128 ? 128 : 256; }

inline unsigned tile_grid(long long tiles) { return (unsigned)((tiles + kLists - 1) / kLists * kLists); }
// Workgroups of a launch of wide tiles, and of a product that narrow tiles divide along k: one to a compute unit (two, with twice as many parts, took
// longer: dX of 65 slots, 32768 words, hidden 1024, and its join 37 us, with one 27).
inline int wide_workgroups() { return std::max(kLists, compute_units() / kLists * kLists); }

// Wide tiles: one workgroup to a compute unit, and a join of the divided tiles where `depth` is long enough (half as many as there are workgroups at most, in one
// round; two thirds, in two: two rounds of halves save nothing).
template <class K, class J, class A>
void launch_wide(K kernel, J join, A& a, int depth, hipStream_t stream) {
    a.workgroups = wide_workgroups();
    kernel<<<a.workgroups, 256, 0, stream>>>(a);
    if (depth > (2 * kWideParts - 1) * kStepK) join<<<a.workgroups * 2 / 3 * 256 / 4, 256, 0, stream>>>(a);
}

// Narrow tiles of shape S, none of them divided.
template <class S, class K, class A>
void launch_narrow(K kernel, A& a, long long tiles, hipStream_t stream) {
    a.workgroups = (int)std::min((long long)tile_grid(tiles), (long long)wide_workgroups() * S::PER_CU);
    kernel<<<a.workgroups, 256, 0, stream>>>(a);
}

// Narrow tiles along the columns, all divided along the words.  tile: slots of one
template <class K, class J, class A>
void launch_divided(K kernel, J join, A& a, int tile, int tiles, hipStream_t stream) {
    a.workgroups = wide_workgroups();
    kernel<<<a.workgroups, 256, 0, stream>>>(a);
    join<<<std::min(tiles, a.workgroups / 2) * tile, 256, 0, stream>>>(a);
}

// The grid of a product whose sizes the host knows: GemmGrid's rule, so that the join of divided tiles is as large as there is something to join, or left out.
inline GemmGrid planned_grid(int ntm, int ntn, int depth, int workgroups, int part_steps, int rounds) {
    GemmGrid g;
    g.ntm = ntm; g.ntn = ntn; g.depth = depth; g.workgroups = workgroups;
    const int tiles = ntm * ntn, steps = (depth + kStepK - 1) / kStepK, most = std::min(kMaxParts, steps / part_steps);
    g.left = tiles % workgroups;
    g.parts = 1;
    int least = rounds > 1 ? steps + kEndSteps : 1 << 30;
    for (int r = 1; g.left > 0 && r <= rounds; ++r) {
        const int p = std::min(r * workgroups / g.left, most);
        if (p < 2) continue;
        const int cost = r * (steps / p + kEndSteps) + g.left * p / 10 + kJoinSteps;
        if (cost < least) { least = cost; g.parts = p; }
    }
    if (g.parts == 1) g.left = 0;
    g.whole = tiles - g.left;
    return g;
}
// workgroups of the join of a grid's divided tiles
template <class S> unsigned join_grid(const GemmGrid& g) { return (unsigned)(S::RING ? (g.left * S::TN + 3) / 4 : S::TM < 256 ? (g.left * S::TN * (S::TM / 4) + 255) / 256 : g.left * S::TN); }

// Tiles of 128 x 128 and of 64 x 64, two to a compute unit, for products that leave wide tiles' workgroups without work.  Of one round or less tiles are divided along k where
// that pays.
template <bool MP, bool MQ> using Small = GemmShape<2, 2, 4, 4, MP, MQ, kDivSmall>;
template <bool MP, bool MQ> using Tiny = GemmShape<2, 2, 2, 2, MP, MQ, kDivTiny>;
// What products take, in ns: of a step of 64 along k, where two tiles share a compute unit and where one has it alone, of a tile's end, and of a divided tile's join for
// each part.
struct TileCost { int tile, step, alone, end, join; };
constexpr TileCost kWideCost = {256, 1060, 1060, 10400, 55}, kSmallCost = {128, 900, 800, 2400, 14}, kTinyCost = {64, 430, 285, 2300, 3};
constexpr int kJoinLaunch = 6700, kNextLaunch = 2000, kNarrowSteps = 4;          // one more launch, in ns; steps of a part
inline long long narrow_cost(const TileCost& c, long long items, int steps, int cus) {
    const long long full = items / (2 * cus), rest = items % (2 * cus);
    return full * ((long long)steps * c.step + c.end) + (rest == 0 ? 0 : (long long)steps * (rest <= cus ? c.alone : c.step) + c.end);
}
// joined: every tile in parts, of which there may be but one: where the join has more to do than to add them.
// most: workgroups that parts may fill, 0: all.
inline GemmGrid narrow_grid(const TileCost& c, int pm, int qn, int depth, long long& cost, bool joined = false, int most = 0) {
    const int cus = wide_workgroups(), steps = std::max(2, (depth + kStepK - 1) / kStepK);
    GemmGrid g;
    g.ntm = (pm + c.tile - 1) / c.tile; g.ntn = (qn + c.tile - 1) / c.tile; g.depth = depth;
    g.workgroups = 2 * cus;
    const int tiles = g.ntm * g.ntn;
    g.left = 0; g.parts = 1; g.whole = tiles;
    cost = narrow_cost(c, tiles, steps, cus);
    if (joined) { g.left = tiles; g.whole = 0; }
    if (most == 0) most = 2 * cus;
    for (int p = 2; p <= most / std::max(tiles, 1) && steps / p >= kNarrowSteps; ++p) {
        const long long t = narrow_cost(c, (long long)tiles * p, (steps + p - 1) / p, cus) + kJoinLaunch + (long long)tiles * p * c.join;
        if (t < cost) { cost = t; g.left = tiles; g.parts = p; g.whole = 0; }
    }
    return g;
}
inline long long wide_cost(const TileCost& c, const GemmGrid& g) {
    const int steps = std::max(2, (g.depth + kStepK - 1) / kStepK), cus = g.workgroups;
    long long cost = (long long)((g.whole + cus - 1) / cus) * ((long long)steps * c.step + c.end);
    if (g.left) cost += (long long)((g.left * g.parts + cus - 1) / cus) * ((steps + g.parts - 1) / g.parts * (long long)c.step + c.end) + kJoinLaunch + (long long)g.left * g.parts * c.join;
    return cost;
}
// Which tiles a product should take least with.  end: what a wide tile's end takes beyond a plain one's, in ns; the others' ends, of a quarter and a sixteenth of the values, run
// beside another workgroup's steps.
enum { kWideTiles, kSmallTiles, kTinyTiles, kFewTiles32, kFewTiles64, kFewTiles128 };
struct Tiling { int kind; GemmGrid grid; long long cost; };
inline Tiling best_tiling(int pm, int qn, int depth, int end = 0) {
    TileCost wide = kWideCost, narrow[2] = {kSmallCost, kTinyCost};
    wide.end += end;
    narrow[0].end += end / 8;
    narrow[1].end += end / 32;
    Tiling best = {kWideTiles, planned_grid((pm + 255) / 256, (qn + 255) / 256, depth, wide_workgroups(), kWideParts, kWideRounds), 0};
    best.cost = wide_cost(wide, best.grid);
    for (int kind = kSmallTiles; kind <= kTinyTiles; ++kind) {
        long long cost = 0;
        const GemmGrid g = narrow_grid(narrow[kind - kSmallTiles], pm, qn, depth, cost);
        if (cost < best.cost) best = Tiling{kind, g, cost};
    }
    return best;
}

// Tiles of 128 columns for few slots (up to 16 BN) and a large weight, of which a compute unit holds as many buffers as fit: bound by the weight's bytes, of which enough have
// to be under way.  Parts of kFewParts steps and more fill the chip; one product of up to kFewWhole steps is done before a join would be.  Tiles of 64 x 64 against these, us,
// weights from memory: 17 slots, 28672 x 4096, kinds KK and MK 46.7, 54.9 and 43.1, 49.4; 4096 x 4096 14.3, 16.3 and 15.0, 14.2; 8192 x 1024 8.9, 9.2 and 11.3, 11.0.
constexpr int kFewSlots = 128;
inline bool few_slots(bool mp, int n_rows, int pm, int depth) { return n_rows <= kFewSlots && (long long)pm * depth >= (mp ? 1 << 24 : 1 << 25); }
template <int BN, bool MP> using Few = GemmShape<4, 1, 2, BN, MP, false, kDivDeep>;
constexpr int kFewParts = 6, kFewWhole = 16;
inline GemmGrid few_grid(int ntm, int depth) { return planned_grid(ntm, 1, depth, wide_workgroups(), depth <= kFewWhole * kStepK ? kNever : kFewParts, 1); }
// Every tile in parts, of which there may be but one: where the join has more to do than to add them.
inline GemmGrid joined_grid(int ntm, int depth, int workgroups) {
    GemmGrid g = planned_grid(ntm, 1, depth, workgroups, kFewParts, 1);
    if (g.whole > 0) {
        g.left += g.whole;
        g.whole = 0;
        g.parts = 1;
    }
    return g;
}
inline int few_tiles(int n_rows) { return n_rows <= 32 ? kFewTiles32 : n_rows <= 64 ? kFewTiles64 : kFewTiles128; }

// Bytes of the parts of a product's divided tiles.
inline size_t tile_bytes(int kind) {
    constexpr int values[] = {256 * 256, 128 * 128, 64 * 64, 128 * 32, 128 * 64, 128 * 128};
    return sizeof(float) * values[kind];
}
inline size_t parts_bytes(int kind, const GemmGrid& g) { return tile_bytes(kind) * (size_t)g.left * g.parts; }
// At most as many as any of the plans above has, for a product by itself or in a group: a launch of parts, and no part of fewer steps than each has at least.
// joined: in narrow tiles all of them are in parts, of which there may be but one.
inline size_t parts_bytes_at_most(int pm, int qn, int depth, bool joined) {
    const long long steps = std::max(2, (depth + kStepK - 1) / kStepK), cus = wide_workgroups();
    auto items = [](long long tiles, long long parts, long long most, bool all) { return (size_t)std::max(parts < 2 ? 0 : std::min(most, tiles * parts), all ? tiles : 0); };
    auto tiles = [&](int tm, int tn) { return (long long)((pm + tm - 1) / tm) * ((qn + tn - 1) / tn); };
    const long long wide = tiles(256, 256), wide_parts = steps / kWideParts, narrow_parts = steps / kNarrowSteps;
    // by itself up to kWideRounds rounds of the tiles that are left behind whole rounds, in a group one
    size_t bytes = tile_bytes(kWideTiles) * std::max(items(wide % cus, wide_parts, kWideRounds * cus, false), items(wide, wide_parts, cus, false));
    bytes = std::max(bytes, tile_bytes(kSmallTiles) * items(tiles(128, 128), narrow_parts, 2 * cus, false));
    bytes = std::max(bytes, tile_bytes(kTinyTiles) * items(tiles(64, 64), narrow_parts, 2 * cus, joined));
    if (qn <= kFewSlots) bytes = std::max(bytes, tile_bytes(few_tiles(qn)) * items((pm + 127) / 128, steps / kFewParts, cus, joined));
    return bytes;
}
}  // namespace wlb
