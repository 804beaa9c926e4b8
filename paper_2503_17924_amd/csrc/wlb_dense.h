// What the layer's matrix products share: the product with its epilogue, activations, rows of slots.
#pragma once
#include <hip/hip_runtime.h>

#include "wlb_gemm_work.h"
#include "wlb_vocab.h"

namespace wlb {

typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

// A product out[n][m] = act(sum_k P[m][k] Q[n][k] + bias[m]) + residual[n][m].  An operand lies with k along its rows (kind K) or down them (kind M).
struct ProductArgs {
    const __bf16 *p, *q;
    long long ldp, ldq, ldo;         // elements between rows
    int pm, qn, depth;
    int twin;                        // 0, or half of qn: rows behind the first `twin` are added to those
    const int32_t* to;               // rows of out and residual, numbers below out_limit; or null: n
    int out_limit;
    __bf16* out;
    const __bf16 *bias, *residual;   // or null
    int act;
    _Float16* kept;                  // [qn][pm]: the activation's slopes, or null
    float* parts;                    // divided tiles
    GemmGrid grid;
};

enum class Kinds { KK, MK, MM };     // of p and q

// Launches the product (with an epilogue only where the kinds are KK).  a.parts: parts_bytes_at_most(a.pm, a.qn, a.depth, a.twin) bytes, here and in a gradient.
void launch_product(Kinds kinds, ProductArgs& a, hipStream_t stream);
// Launches the products of a gradient that wait for nothing of each other: one of kinds MK (or null) and up to two of kinds MM, side by side where that pays.
void launch_gradients(ProductArgs* dx, ProductArgs* const* dw, int n_dw, hipStream_t stream);

// Up to this many slots an operand that is rounded to bf16 has a second set of rows with what that leaves out: their few roundings find little to average out with, and
// such products are bound by the weight's bytes.
constexpr int kExactSlots = 32;
inline int operand_rows(int n_rows) { return n_rows <= kExactSlots ? 2 * n_rows : n_rows; }
// What bf16 leaves out of a value: nothing, beside one that is not finite.
__device__ __forceinline__ float rest_of(float v) {
#pragma clang fp contract(off)          // of v as it was rounded, whichever product it came from: the same with what is kept and without
    const float rest = v - (float)(__bf16)v;
    return __builtin_isfinite(rest) ? rest : 0.f;
}

// ------------------------------------------------------------------------------------------
// Plans.
// What activations add to a wide tile's end, in ns, and rows in 32 bits with something beside them (4189 slots, 1544 x 5000, two rounds of wide tiles: 83 us plain, silu 87, gelu
// 97; with a residual or slopes that are kept 12 more; 128 x 128 tiles 99 to 107).
inline int activation_end(int act) { return act == WLB_ACT_GELU ? 6000 : act == WLB_ACT_SILU ? 2000 : 0; }
constexpr int kRowsEnd = 6000;

// The tiles that a product by itself should take least with.
inline Tiling plan_product(Kinds kinds, const ProductArgs& a) {
    const bool mp = kinds != Kinds::KK;
    if (kinds != Kinds::MM && few_slots(mp, a.qn, a.pm, a.depth)) {
        const int ntm = (a.pm + 127) / 128;
        return Tiling{few_tiles(a.qn), a.twin ? joined_grid(ntm, a.depth, wide_workgroups()) : few_grid(ntm, a.depth), 0};
    }
    if (a.twin) {
        Tiling t = {kTinyTiles, {}, 0};
        t.grid = narrow_grid(kTinyCost, a.pm, a.qn, a.depth, t.cost, true);
        return t;
    }
    return best_tiling(a.pm, a.qn, a.depth, activation_end(a.act) + (a.residual || a.kept ? kRowsEnd : 0));
}
// The same of the products that leave rows of h, dg and du: of those that have a second set of rows where there is one.
inline Tiling plan_slots(Kinds kinds, int pm, int n_rows, int depth, int end) {
    if (few_slots(kinds != Kinds::KK, n_rows, pm, depth)) return Tiling{few_tiles(n_rows), few_grid((pm + 127) / 128, depth), 0};
    Tiling t = best_tiling(pm, n_rows, depth, end);
    if (n_rows <= kExactSlots) {
        t.kind = kTinyTiles;
        t.grid = narrow_grid(kTinyCost, pm, n_rows, depth, t.cost);
    }
    return t;
}

// ------------------------------------------------------------------------------------------
// Several products in one launch: a workgroup takes its items of one after the other, and those of the next product begin with the workgroups that the last one
// left without any, so that three products which each leave part of the chip idle share it.  None of them is divided along k but the last one's tiles
// past whole rounds (or, of few slots, the first).
struct GroupArgs {
    ProductArgs a[3];                // the first of kinds MK, if there is one (its qn is 0 otherwise), then those of kinds MM
    int n;
    int turn[3];                     // workgroups of an XCD by which a product's first one is moved
};

// A group of whole tiles, and what it should take: every workgroup of an XCD has its items' time, and the last product's tiles past whole rounds may be divided.
template <class S>
long long plan_group(GroupArgs& g, const TileCost& cost) {
    const int per_cu = S::RING ? 1 : 2, workgroups = wide_workgroups() * per_cu, side = workgroups / kLists;
    long long all = 0, load[256] = {};         // of every workgroup of an XCD, and beside that
    int at = 0;
    for (int k = 0; k < g.n; ++k) {
        ProductArgs& a = g.a[k];
        if (a.qn == 0) continue;
        const int ntm = (a.pm + S::TM - 1) / S::TM, ntn = (a.qn + S::TN - 1) / S::TN, steps = std::max(2, (a.depth + kStepK - 1) / kStepK);
        a.grid.ntm = ntm; a.grid.ntn = ntn; a.grid.depth = a.depth; a.grid.workgroups = workgroups;
        a.grid.whole = ntm * ntn; a.grid.left = 0; a.grid.parts = 1; a.grid.lead = 0;
        long long part = 0, join = 0;
        if (k == g.n - 1) {
            // the tiles of a last round that a quarter of the launch at most would have
            const int before = at, per = (a.grid.whole + kLists - 1) / kLists, over = (before + per) % side;
            const int most = std::min(kMaxParts, steps / kWideParts);
            if (over > 0 && over <= side / 4 && over < per && before + per > side) {
                const int whole = (per - over) * kLists, left = a.grid.whole - whole, p = left > 0 ? std::min(workgroups / left, most) : 0;
                if (p >= 2 && (long long)left * p * S::TM * S::TN <= (long long)workgroups * S::TM * S::TN) {
                    a.grid.whole = whole; a.grid.left = left; a.grid.parts = p;
                    part = (long long)((steps + p - 1) / p) * cost.step + cost.end;
                    join = kJoinLaunch + (long long)left * p * cost.join;
                }
            }
        }
        const int per = (a.grid.whole + kLists - 1) / kLists;
        g.turn[k] = at % side;
        // whole rounds, and one more tile from the workgroup `turn` on
        const long long tile = (long long)steps * cost.step + cost.end;
        all += per / side * tile;
        for (int i = 0, n = per % side, w = g.turn[k]; i < n; ++i, w = w + 1 < side ? w + 1 : 0) load[w] += tile;
        at += per;
        if (part) {
            // An XCD's parts go to the workgroups that are done first of those where a product begins or ends: at equal loads behind the last whole tile, but where
            // products' steps differ beside the one with fewer (4189 slots, 1544 x 5000, dx's 79 and dW's 66: 145 us, behind dx's tiles 157).
            const int share = (a.grid.left * a.grid.parts + kLists - 1) / kLists, end = at % side;
            long long least = 0;
            for (int c = k + 1; c >= 0; --c) {
                const int from = c > k ? end : g.a[c].qn ? g.turn[c] : end;
                long long most = 0;
                for (int i = 0; i < std::min(share, side); ++i) most = std::max(most, load[(from + i) % side]);
                if (c > k || most < least) {
                    least = most;
                    a.grid.lead = (from - end + side) % side;
                }
            }
            return all + std::max(*std::max_element(load, load + side), least + part) + join;
        }
    }
    return all + *std::max_element(load, load + side);
}

// Bytes for the parts of divided tiles in the calls of an operator, one product or launch after the other: y, dx and dW; (g, u), y, dh, dx, dW_in and dW_out.
inline size_t linear_parts_bytes(int n_rows, int n_in, int n_out, int activation) {
    const int dz = activation != WLB_ACT_NONE ? operand_rows(n_rows) : n_rows;
    return std::max({parts_bytes_at_most(n_out, n_rows, n_in, false), parts_bytes_at_most(n_in, dz, n_out, dz > n_rows), parts_bytes_at_most(n_in, n_out, dz, false)});
}
inline size_t ffn_parts_bytes(int n_rows, int hidden, int inner) {
    const int both = operand_rows(n_rows);
    const bool joined = both > n_rows;
    return std::max({parts_bytes_at_most(2 * inner, n_rows, hidden, false), parts_bytes_at_most(hidden, both, inner, joined), parts_bytes_at_most(inner, n_rows, hidden, false),
                     parts_bytes_at_most(hidden, both, 2 * inner, joined), parts_bytes_at_most(hidden, 2 * inner, both, false), parts_bytes_at_most(inner, hidden, both, false)});
}

// How the products of a gradient, which wait for nothing of each other, are launched: one after the other, or in one launch of wide, small or tiny tiles; few slots' weights in
// small tiles, dx in tiles of 128 columns and up to 32, 64 or 128 slots, or in tiny ones.
enum Group { kApart, kWideGroup, kSmallGroup, kTinyGroup, kFewGroup32, kFewGroup64, kFewGroup128, kFewGroupTiny };
inline int group_tiles(Group kind) {          // of the divided product
    constexpr int kinds[] = {kWideTiles, kWideTiles, kSmallTiles, kTinyTiles, kFewTiles32, kFewTiles64, kFewTiles128, kTinyTiles};
    return kinds[kind];
}
inline Group plan_gradients(GroupArgs& g) {
    const bool dx = g.a[0].qn > 0;
    const int rows = dx ? g.a[0].qn : g.n > 1 ? g.a[1].depth : 0;
    if (rows == 0 || (dx ? 1 : 0) + g.n - 1 < 2) return kApart;
    if (rows <= kFewSlots) {
        // the weights' gradients in tiles of 128 x 128, which are bound by what they write; dx as its product by itself would be
        const int workgroups = 2 * wide_workgroups(), ntm = (g.a[0].pm + 127) / 128;
        const bool few = dx && few_slots(true, rows, g.a[0].pm, g.a[0].depth);
        long long unused = 0;
        // dx in parts for half of the workgroups, beside which the others begin with the weights' tiles
        const int half = wide_workgroups();
        if (few) g.a[0].grid = g.a[0].twin ? joined_grid(ntm, g.a[0].depth, half) : planned_grid(ntm, 1, g.a[0].depth, half, kFewParts, 1);
        else if (dx) g.a[0].grid = narrow_grid(kTinyCost, g.a[0].pm, rows, g.a[0].depth, unused, g.a[0].twin > 0, half);
        g.a[0].grid.workgroups = workgroups;
        int at = dx ? (g.a[0].grid.whole + g.a[0].grid.left * g.a[0].grid.parts + kLists - 1) / kLists : 0;
        for (int k = 1; k < g.n; ++k) {
            g.a[k].grid = narrow_grid(kSmallCost, g.a[k].pm, g.a[k].qn, g.a[k].depth, unused);
            g.a[k].grid.whole += g.a[k].grid.left;
            g.a[k].grid.left = 0;
            g.a[k].grid.parts = 1;
            g.turn[k] = at % (workgroups / kLists);
            at += (g.a[k].grid.whole + kLists - 1) / kLists;
        }
        const int tile = few ? slot_tile(rows) : 0;
        return tile == 32 ? kFewGroup32 : tile == 64 ? kFewGroup64 : tile == 128 ? kFewGroup128 : kFewGroupTiny;
    }
    long long apart = 0;
    for (int k = 0; k < g.n; ++k)
        if (g.a[k].qn) apart += best_tiling(g.a[k].pm, g.a[k].qn, g.a[k].depth).cost + kNextLaunch;
    GroupArgs wide = g, small = g, tiny = g;
    const long long wide_time = plan_group<Wide<true, true>>(wide, kWideCost), small_time = plan_group<Small<true, true>>(small, kSmallCost), tiny_time = plan_group<Tiny<true, true>>(tiny, kTinyCost);
    const long long least = std::min({apart, wide_time, small_time, tiny_time});
    if (apart == least) return kApart;
    g = wide_time == least ? wide : small_time == least ? small : tiny;
    return wide_time == least ? kWideGroup : small_time == least ? kSmallGroup : kTinyGroup;
}

// ------------------------------------------------------------------------------------------
// Rows of `src` that are listed, one behind the other in `dst` (null: nothing is copied), for up to two tensors; and zeros in the rows of `zero` that are not.
struct GatherArgs {
    const uint4* src[2];
    uint4* dst[2];
    int chunks[2];                   // of 16 bytes, to a row
    uint4* zero;
    int zero_chunks;
    const int32_t* rows;             // [n_q]: those that are listed, then the others
    int n_q, n_rows;
};
void launch_gather(const GatherArgs& a, hipStream_t stream);

// What can be said of a descriptor of either operator.
wlb_status check_rows(const char* call, int32_t n_q, int32_t n_rows, int32_t a, int32_t b, int32_t activation);
// rows is given where not every slot holds a token
wlb_status check_list(const char* call, int32_t n_q, int32_t n_rows, const int32_t* rows);

// Few slots' rows twice, for the products over slots whose other operand has a second set of rows: as they are, and behind them with zeros in place of what is not finite (a zero
// among what bf16 leaves out would make an infinity undefined).
struct TwiceArgs {
    const uint4* src[2];             // [rows][chunks of 8 values], or null
    uint4* dst[2];                   // [2 rows][chunks]
    int rows, chunks;
};
__device__ __forceinline__ uint32_t finite2(uint32_t v) {
    if ((v & 0x7f800000u) == 0x7f800000u) v &= 0x0000ffffu;
    if ((v & 0x00007f80u) == 0x00007f80u) v &= 0xffff0000u;
    return v;
}
__device__ __forceinline__ void write_twice(const TwiceArgs& a, int thread, int threads) {
    const int n = a.rows * a.chunks;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (a.src[k])
            for (int i = thread; i < n; i += threads) {
                const uint4 v = a.src[k][i];
                a.dst[k][i] = v;
                a.dst[k][n + i] = uint4{finite2(v.x), finite2(v.y), finite2(v.z), finite2(v.w)};
            }
}
void launch_twice(const TwiceArgs& a, hipStream_t stream);

// ------------------------------------------------------------------------------------------
// Activations and their slopes.  Silu z p with p = 1 / (1 + e^-z); gelu z q with q the normal distribution's share below z.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(-1.4426950408889634f * z)); }
// The share above |z| is e R with e = e^(-z^2 / 2) and, t = 1 / (1 + 0.28 |z|), R = t times a polynomial fitted to it (least largest relative error, 1.7e-7; with
// the roundings of float 2e-6 up to |z| = 6, 8e-6 at 13, where it leaves the range of float).  erfcf in its place made a wide tile's end too long to keep in registers.
__device__ __forceinline__ float normal_share(float z, float& e) {
    const float x = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.28f, x, 1.f));
    constexpr float c[9] = {0.11170385777950287f, 0.11169980466365814f, 0.10308466851711273f, 0.0836307480931282f, 0.07277520000934601f, -0.006449663545936346f,
                            0.0924287810921669f, -0.09359358996152878f, 0.024720102548599243f};
    float p = c[8];
#pragma unroll
    for (int k = 7; k >= 0; --k) p = __builtin_fmaf(p, t, c[k]);
    e = fast_exp2(-0.72134752044448170f * x * x);
    const float above = p * t * e;
    return z < 0.f ? above : 1.f - above;
}

template <int Act>
__device__ __forceinline__ float activated(float z) {
    if (Act == WLB_ACT_RELU) return z > 0.f || z != z ? z : 0.f;          // NaN stays
    if (Act == WLB_ACT_SILU) return z * logistic(z);
    if (Act == WLB_ACT_GELU) {
        float e;
        return z * normal_share(z, e);
    }
    return z;
}
// the activation and its slope
template <int Act>
__device__ __forceinline__ void activated(float z, float& value, float& slope) {
    value = z;
    slope = 1.f;
    if (Act == WLB_ACT_RELU) {
        value = activated<Act>(z);
        slope = z > 0.f ? 1.f : 0.f;
    } else if (Act == WLB_ACT_SILU) {
        const float p = logistic(z);
        value = z * p;
        slope = p + value * (1.f - p);
    } else if (Act == WLB_ACT_GELU) {
        float e;
        const float q = normal_share(z, e);
        value = z * q;
        slope = q + z * 0.3989422804014327f * e;
    }
}

template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
    switch (act) {
    case WLB_ACT_RELU: f(std::integral_constant<int, WLB_ACT_RELU>{}); break;
    case WLB_ACT_SILU: f(std::integral_constant<int, WLB_ACT_SILU>{}); break;
    case WLB_ACT_GELU: f(std::integral_constant<int, WLB_ACT_GELU>{}); break;
    default: f(std::integral_constant<int, WLB_ACT_NONE>{});
    }
}

}  // namespace wlb
