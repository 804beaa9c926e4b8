// Gated feed-forward block of a rank's slots and its gradient (wlb_ffn_fwd / wlb_ffn_bwd).
//
//   forward   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T + r
//   backward  dh = dy Wd, dg = dh a, du = dh b with a = u act'(g), b = act(g); dWd = dy^T h, (dWg, dWu) = (dg, du)^T x, dx = (dg, du) (Wg, Wu)
// Products of 6 n H F operations forward and 12 n H F backward, which bound it (up to about 64 slots the weights' bytes do).  The two products that
// meet in an elementwise function are one kernel each: a tile of the first has rows of Wg and of Wu by turns, so that a lane holds g and u of the same place;
// the one of dh has a and b loaded at its end and leaves dg and du.  The others are plain products (wlb_linear.hip).
//
// Up to kExactSlots slots h, dg and du have a second set of rows with what bf16 leaves out of the first, and results are exact but for their own rounding.
//
// What the forward keeps: h, and a and b in pieces of four in fp16 below a common power of two, rounded by 2^-11 of themselves: an eighth of what dg and du lose
// when they are rounded for their products (2^-40 of the power where they lie far below it).  At a tile's end all compute units move their operands and results at once, so bytes are time: with g
// and u in 32 bits (8192 slots, hidden 4096, inner 14336) the product with Wg and Wu took 1503 us, the one of dh, which made h again, 892.
#include "wlb_dense.h"

namespace wlb {

// a and b as they leave the accumulators: blocks of 16 columns x 16 slots of 16 bytes a lane, four of a and four of b; lane l of a block has columns 4 (l / 16) .. + 3 of slot
// l % 16.  Their exponents lie apart, two bytes a lane, four blocks of a lane's one behind the other.
struct Kept {
    __bf16* h;                       // [n_rows][inner], up to kExactSlots slots with as many rows of what bf16 leaves out behind them
    char* values;                    // [slots / 16][columns / 16] blocks of 1 KiB
    char* exponents;                 // [slots / 16][columns / 64] of 512 bytes
    int inner;
    __host__ __device__ static size_t blocks(int n, int of) { return (size_t)((n + of - 1) / of); }
    __device__ __forceinline__ size_t block(int row, int col) const { return (size_t)(row / 16) * blocks(inner, 16) + col / 16; }
    __device__ __forceinline__ char* value_at(int row, int col, int lane) const { return values + block(row, col) * 1024 + lane * 16; }
    __device__ __forceinline__ char* exponent_at(int row, int col, int lane) const {
        return exponents + ((size_t)(row / 16) * blocks(inner, 64) + col / 64) * 512 + lane * 8 + col % 64 / 16 * 2;
    }
};
// lane of a block that has columns col .. + 3 (col a multiple of 4) of slot row
__device__ __forceinline__ int piece_lane(int row, int col) { return col % 16 / 4 * 16 + row % 16; }

// Four floats in fp16, multiplied by 2^(15 - e), and e - 1, which is e of the largest finite one, in 8 bits.
__device__ __forceinline__ f16x4 lowered(const f32x4& v, int& e) {
    float most = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
    if (__builtin_isinf(most)) {                    // it stays infinite beside the others
        most = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) most = __builtin_isinf(v[k]) ? most : fmaxf(most, fabsf(v[k]));
    }
    e = max(__builtin_amdgcn_frexp_expf(most), -126);
    f16x4 out;
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = (_Float16)__builtin_amdgcn_ldexpf(v[k], 15 - e);
    return out;
}
__device__ __forceinline__ uint16_t exponents(int ea, int eb) { return (uint16_t)(((ea - 1) & 0xff) | ((eb - 1) & 0xff) << 8); }
// the factors that undo it
__device__ __forceinline__ void factors(uint16_t e, float& fa, float& fb) {
    fa = __builtin_amdgcn_ldexpf(1.f, (int)(int8_t)(e & 0xff) - 14);
    fb = __builtin_amdgcn_ldexpf(1.f, (int)(int8_t)(e >> 8) - 14);
}
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
struct Piece { f16x4 a, b; };

// From g and u of a piece: h rounded, what that leaves out, and a and b as they are kept.
template <int Act>
__device__ __forceinline__ bf16x4 gated(const f32x4& g, const f32x4& u, Piece& kept, uint16_t& e, bf16x4& rest) {
    f32x4 a, b;
    bf16x4 h;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float value, slope;
        activated<Act>(g[k], value, slope);
        a[k] = u[k] * slope;
        b[k] = value;
        h[k] = (__bf16)(value * u[k]);
        rest[k] = (__bf16)rest_of(value * u[k]);
    }
    int ea, eb;
    kept.a = lowered(a, ea);
    kept.b = lowered(b, eb);
    e = exponents(ea, eb);
    return h;
}

// tiles that may have up to kExactSlots slots alone
template <class S> constexpr bool kMayExact = S::TN <= kExactSlots || S::TM == 64;

// What the bytes that are kept add to a wide tile's end, and those that dg and du are made of and leave, in ns.
constexpr int kKeptEnd = 8000, kInnerEnd = 20000;

struct GateArgs {
    const __bf16 *x, *w_in;
    int n_rows, hidden, inner;
    Kept to;                         // h alone, or all
    float* parts;                    // divided tiles
    GemmGrid grid;
};

template <class S>
struct GateWork : GemmGrid {
    static constexpr int COLS = S::TM / 2;             // columns of h to a tile
    const GateArgs& a;
    int qn;
    long long ldp, ldq;
    __device__ __forceinline__ explicit GateWork(const GateArgs& a_) : GemmGrid(a_.grid), a(a_), qn(a_.n_rows), ldp(a_.hidden), ldq(a_.hidden) {}
    __device__ __forceinline__ GemmPaired p(const GemmItem& i) const {
        const int f0 = i.tm * COLS;
        return GemmPaired{a.w_in + (long long)f0 * ldp + i.k0, a.inner - f0, S::BM * 8, (uint32_t)a.inner};
    }
    __device__ __forceinline__ GemmOperand q(const GemmItem& i) const {
        const int n0 = i.tn * S::TN;
        return GemmOperand{a.x + (long long)n0 * ldq + i.k0, a.n_rows - n0, nullptr};
    }
};

template <class S, int Act, bool Keep>
struct GateDone : NothingAhead {
    const GateArgs& a;
    __device__ __forceinline__ explicit GateDone(const GateArgs& a_) : a(a_) {}
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, Ahead, uint32_t room) const {
        constexpr int B = S::BM / 2, COLS = S::TM / 2;
        if (it.part >= 0) {
            g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), a.n_rows - it.tn * S::TN);
            return 0;
        }
        const int f0 = it.tm * COLS, n0 = it.tn * S::TN;
        const bool full = n0 + S::TN <= a.n_rows && f0 + COLS <= a.inner;
        constexpr bool MayExact = kMayExact<S>;
        const bool exact = MayExact && a.n_rows <= kExactSlots;
        auto put = [&](int n, int m, const i32x4& v, int o = 0) __attribute__((always_inline)) {
            if (n0 + n < a.n_rows && f0 + m < a.inner) *reinterpret_cast<i32x4*>(a.to.h + (size_t)(n0 + n + (o ? a.n_rows : 0)) * a.inner + f0 + m) = v;
        };
        if constexpr (!Keep) {
            g.template rows_out<2, B>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return activated<Act>(g.sum(i, j, r)) * g.sum(B + i, j, r); },
                                      [&](int n, int m, const i32x4& v, int) __attribute__((always_inline)) { put(n, m, v); });
            if constexpr (MayExact)
                if (exact) g.template rows_out<2, B>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return rest_of(activated<Act>(g.sum(i, j, r)) * g.sum(B + i, j, r)); },
                                          [&](int n, int m, const i32x4& v, int) __attribute__((always_inline)) { put(n, m, v, 1); });
            return full ? S::BN * B / 2 : 0;            // of 1 KiB, two blocks each
        } else {
            const int n1 = n0 + g.wn * (S::BN * 16), f1 = f0 + g.wm * (B * 16), rows = a.n_rows - n1, cols = a.inner - f1;
            char* values = a.to.value_at(n1, f1, g.lane);
            char* exps = a.to.exponent_at(n1, f1, g.lane);
            const size_t down = Kept::blocks(a.inner, 16) * 1024, exps_down = Kept::blocks(a.inner, 64) * 512;
            uint16_t e[B];
            struct None {};
            constexpr int OUTS = MayExact ? 2 : 1;
            g.template rows_out_many<OUTS, B>(
                room, [&](int, int) __attribute__((always_inline)) { return None{}; },
                [&](int i, int j, int, None, bf16x4 (&out)[OUTS]) __attribute__((always_inline)) {
                    Piece kept;
                    bf16x4 rest;
                    out[0] = gated<Act>(f32x4{g.sum(i, j, 0), g.sum(i, j, 1), g.sum(i, j, 2), g.sum(i, j, 3)},
                                        f32x4{g.sum(B + i, j, 0), g.sum(B + i, j, 1), g.sum(B + i, j, 2), g.sum(B + i, j, 3)}, kept, e[i], rest);
                    if constexpr (MayExact) out[1] = rest;
                    if (j * 16 < rows && i * 16 < cols) *reinterpret_cast<Piece*>(values + j * down + i * 1024) = kept;
                    if (i == B - 1 && j * 16 < rows) {
                        if constexpr (B == 4) {
                            // a wavefront's columns are 64: eight bytes of exponents a lane, of blocks that exist or not
                            if (0 < cols) *reinterpret_cast<u32x2*>(exps + j * exps_down) = u32x2{e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16};
                        } else {
#pragma unroll
                            for (int k = 0; k < B; ++k)
                                if (k * 16 < cols) *reinterpret_cast<uint16_t*>(exps + j * exps_down + k * 2) = e[k];
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                },
                [&](int o, int n, int m, const i32x4& v) __attribute__((always_inline)) { if (o == 0 || exact) put(n, m, v, o); });
            return full ? S::BN * B : 0;                // values
        }
    }
};

template <class S, int Act, bool Keep>
__global__ void __launch_bounds__(256, S::PER_CU) gate_kernel(GateArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const GateWork<S> w(a);
    Gemm<S> gemm;
    gemm.run(smem, w, GateDone<S, Act, Keep>(a));
}

template <class S, int Act>
__global__ void __launch_bounds__(256) gate_join_kernel(GateArgs a) {
    const GateWork<S> w(a);
    join_any<S>(w, a.parts, [&](int tm, int tn, int n, int m, const f32x4& v) __attribute__((always_inline)) {
        // columns m of a tile: of 2 * half the first half are g's, u's lie half a turn on
        constexpr int HALF = S::BM * 8;
        const int row = tn * S::TN + n, t = m % (2 * HALF), col = tm * (S::TM / 2) + m / (2 * HALF) * HALF + t;
        f32x4 u;
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = __shfl(v[k], (int)(threadIdx.x & 63) + HALF / 4);
        if (t >= HALF || row >= a.n_rows || col >= a.inner) return;
        Piece kept;
        uint16_t e;
        bf16x4 rest;
        *reinterpret_cast<bf16x4*>(a.to.h + (size_t)row * a.inner + col) = gated<Act>(v, u, kept, e, rest);
        if (kMayExact<S> && a.n_rows <= kExactSlots) *reinterpret_cast<bf16x4*>(a.to.h + (size_t)(a.n_rows + row) * a.inner + col) = rest;
        if (a.to.values) {
            const int lane = piece_lane(row, col);
            *reinterpret_cast<Piece*>(a.to.value_at(row, col, lane)) = kept;
            *reinterpret_cast<uint16_t*>(a.to.exponent_at(row, col, lane)) = e;
        }
    });
}

template <class S, int Act>
static void launch_gate_tiles(GateArgs& a, hipStream_t stream) {
    if (a.to.values) gate_kernel<S, Act, true><<<a.grid.workgroups, 256, 0, stream>>>(a);
    else gate_kernel<S, Act, false><<<a.grid.workgroups, 256, 0, stream>>>(a);
    if (a.grid.left) gate_join_kernel<S, Act><<<join_grid<S>(a.grid), 256, 0, stream>>>(a);
}
template <int Act>
static void launch_gate(GateArgs& a, hipStream_t stream) {
    if (a.n_rows == 0) return;
    const Tiling t = plan_slots(Kinds::KK, 2 * a.inner, a.n_rows, a.hidden, activation_end(Act) / 2 + (a.to.values ? kKeptEnd : 0));
    a.grid = t.grid;
    if (t.kind == kWideTiles) launch_gate_tiles<Wide<false, false>, Act>(a, stream);
    else if (t.kind == kSmallTiles) launch_gate_tiles<Small<false, false>, Act>(a, stream);
    else if (t.kind == kTinyTiles) launch_gate_tiles<Tiny<false, false>, Act>(a, stream);
    else if (t.kind == kFewTiles32) launch_gate_tiles<Few<2, false>, Act>(a, stream);
    else if (t.kind == kFewTiles64) launch_gate_tiles<Few<4, false>, Act>(a, stream);
    else launch_gate_tiles<Few<8, false>, Act>(a, stream);
}

// ------------------------------------------------------------------------------------------
// dh = dy Wd and, with a and b, dg and du.
struct InnerArgs {
    const __bf16 *w_out, *dy;        // [hidden][inner], [n_rows][hidden]
    int n_rows, hidden, inner;
    Kept kept;
    __bf16* d;                       // [n_rows][2 inner]: dg, then du; rows of what bf16 leaves out as of h
    float* parts;
    GemmGrid grid;
    TwiceArgs twice;                 // x and dy of few slots, for the products behind this one
};

template <class S>
struct InnerWork : GemmGrid {
    const InnerArgs& a;
    int qn;
    long long ldp, ldq;
    __device__ __forceinline__ explicit InnerWork(const InnerArgs& a_) : GemmGrid(a_.grid), a(a_), qn(a_.n_rows), ldp(a_.inner), ldq(a_.hidden) {}
    __device__ __forceinline__ GemmOperand p(const GemmItem& i) const {
        const int m0 = i.tm * S::TM;
        return GemmOperand{a.w_out + (long long)i.k0 * ldp + m0, a.inner - m0, nullptr};
    }
    __device__ __forceinline__ GemmOperand q(const GemmItem& i) const {
        const int n0 = i.tn * S::TN;
        return GemmOperand{a.dy + (long long)n0 * ldq + i.k0, a.n_rows - n0, nullptr};
    }
};

// dg and du of four values, and (Outs = 4) what bf16 leaves out of them
template <int Outs>
__device__ __forceinline__ void inner_gradient(const f32x4& dh, const Piece& kept, uint16_t e, bf16x4 (&out)[Outs]) {
    float fa, fb;
    factors(e, fa, fb);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float dg = dh[k] * ((float)kept.a[k] * fa), du = dh[k] * ((float)kept.b[k] * fb);
        out[0][k] = (__bf16)dg;
        out[1][k] = (__bf16)du;
        if constexpr (Outs == 4) {
            out[2][k] = (__bf16)rest_of(dg);
            out[3][k] = (__bf16)rest_of(du);
        }
    }
}

template <class S>
struct InnerDone : NothingAhead {
    const InnerArgs& a;
    __device__ __forceinline__ explicit InnerDone(const InnerArgs& a_) : a(a_) {}
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, Ahead, uint32_t room) const {
        if (it.part >= 0) {
            g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), a.n_rows - it.tn * S::TN);
            return 0;
        }
        const int m0 = it.tm * S::TM, n0 = it.tn * S::TN, n1 = n0 + g.wn * (S::BN * 16), m1 = m0 + g.wm * (S::BM * 16), rows = a.n_rows - n1, cols = a.inner - m1;
        const char* values = a.kept.value_at(n1, m1, g.lane);
        const char* exps = a.kept.exponent_at(n1, m1, g.lane);
        const size_t down = Kept::blocks(a.inner, 16) * 1024, exps_down = Kept::blocks(a.inner, 64) * 512;
        constexpr int OUTS = kMayExact<S> ? 4 : 2, G = Gemm<S>::template out_group<>();
        struct Pieces { Piece piece[G]; uint32_t e[G / 2]; };
        static_assert(G == 4 || G == 2, "exponents of two or four blocks at a time");
        g.template rows_out_many<OUTS>(
            room,
            [&](int i0, int j) __attribute__((always_inline)) {
                Pieces t = {};
                if (j * 16 < rows && i0 * 16 < cols) {
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        if ((i0 + i) * 16 < cols) t.piece[i] = *reinterpret_cast<const Piece*>(values + j * down + (i0 + i) * 1024);
                    // of blocks that are not there too: their bytes are
                    const char* from = exps + j * exps_down + i0 / 4 * 512 + i0 % 4 * 2;
#pragma unroll
                    for (int i = 0; i < G / 2; ++i) t.e[i] = reinterpret_cast<const uint32_t*>(from)[i];
                }
                return t;
            },
            [&](int i, int j, int k, const Pieces& t, bf16x4 (&out)[OUTS]) __attribute__((always_inline)) {
                inner_gradient<OUTS>(f32x4{g.sum(i, j, 0), g.sum(i, j, 1), g.sum(i, j, 2), g.sum(i, j, 3)}, t.piece[k], (uint16_t)(t.e[k / 2] >> (k % 2 * 16)), out);
            },
            [&](int o, int n, int m, const i32x4& v) __attribute__((always_inline)) {
                if (n0 + n < a.n_rows && m0 + m < a.inner && (o < 2 || a.n_rows <= kExactSlots)) *reinterpret_cast<i32x4*>(a.d + (size_t)(n0 + n + (o / 2 ? a.n_rows : 0)) * (2 * (size_t)a.inner) + (o % 2 ? a.inner : 0) + m0 + m) = v;
            });
        return n0 + S::TN <= a.n_rows && m0 + S::TM <= a.inner ? 2 * row_stores<S, 2>() : 0;
    }
};

template <class S>
__global__ void __launch_bounds__(256, S::PER_CU) inner_kernel(InnerArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const InnerWork<S> w(a);
    // first the workgroups that have no tile, which are the last
    if constexpr (kMayExact<S>) write_twice(a.twice, (int)((gridDim.x - 1 - blockIdx.x) * 256 + threadIdx.x), (int)gridDim.x * 256);
    Gemm<S> gemm;
    gemm.run(smem, w, InnerDone<S>(a));
}

template <class S>
__global__ void __launch_bounds__(256) inner_join_kernel(InnerArgs a) {
    const InnerWork<S> w(a);
    join_any<S>(w, a.parts, [&](int tm, int tn, int n, int m, const f32x4& dh) __attribute__((always_inline)) {
        const int row = tn * S::TN + n, col = tm * S::TM + m;
        if (row >= a.n_rows || col >= a.inner) return;
        const int lane = piece_lane(row, col);
        constexpr int OUTS = kMayExact<S> ? 4 : 2;
        bf16x4 out[OUTS];
        inner_gradient<OUTS>(dh, *reinterpret_cast<const Piece*>(a.kept.value_at(row, col, lane)), *reinterpret_cast<const uint16_t*>(a.kept.exponent_at(row, col, lane)), out);
        __bf16* d = a.d + (size_t)row * (2 * (size_t)a.inner) + col;
        *reinterpret_cast<bf16x4*>(d) = out[0];
        *reinterpret_cast<bf16x4*>(d + a.inner) = out[1];
        if (OUTS == 4 && a.n_rows <= kExactSlots) {
            d += (size_t)a.n_rows * (2 * (size_t)a.inner);
            *reinterpret_cast<bf16x4*>(d) = out[OUTS - 2];
            *reinterpret_cast<bf16x4*>(d + a.inner) = out[OUTS - 1];
        }
    });
}

template <class S>
static void launch_inner_tiles(InnerArgs& a, hipStream_t stream) {
    inner_kernel<S><<<a.grid.workgroups, 256, 0, stream>>>(a);
    if (a.grid.left) inner_join_kernel<S><<<join_grid<S>(a.grid), 256, 0, stream>>>(a);
}
static void launch_inner(InnerArgs& a, hipStream_t stream) {
    if (a.n_rows == 0) return;
    const Tiling t = plan_slots(Kinds::MK, a.inner, a.n_rows, a.hidden, kInnerEnd);
    a.grid = t.grid;
    if (t.kind == kWideTiles) launch_inner_tiles<Wide<true, false>>(a, stream);
    else if (t.kind == kSmallTiles) launch_inner_tiles<Small<true, false>>(a, stream);
    else if (t.kind == kTinyTiles) launch_inner_tiles<Tiny<true, false>>(a, stream);
    else if (t.kind == kFewTiles32) launch_inner_tiles<Few<2, true>>(a, stream);
    else if (t.kind == kFewTiles64) launch_inner_tiles<Few<4, true>>(a, stream);
    else launch_inner_tiles<Few<8, true>>(a, stream);
}

static void launch_gate(int act, GateArgs& a, hipStream_t stream) {
    if (act == WLB_ACT_RELU) launch_gate<WLB_ACT_RELU>(a, stream);
    else if (act == WLB_ACT_SILU) launch_gate<WLB_ACT_SILU>(a, stream);
    else if (act == WLB_ACT_GELU) launch_gate<WLB_ACT_GELU>(a, stream);
    else launch_gate<WLB_ACT_NONE>(a, stream);
}

// ------------------------------------------------------------------------------------------
static wlb_status check_ffn(const wlb_ffn_desc* d, const char* call) {
    if (!d) return fail(WLB_ERR_INVALID_ARG, "%s: null desc", call);
    if (wlb_status st = check_rows(call, d->n_q, d->n_rows, d->hidden, d->inner, d->activation)) return st;
    // rows of Wu are addressed from those of Wg with 32-bit offsets
    if ((int64_t)(d->inner + 256) * d->hidden >= (1ll << 31) - (1 << 20)) return fail(WLB_ERR_UNSUPPORTED, "%s: inner=%d times hidden=%d of 2^31 or more", call, d->inner, d->hidden);
    return WLB_OK;
}

struct FfnLayout {
    size_t off_parts, off_h, fwd_bytes, off_d, off_x, off_dy, off_x2, off_dy2, bwd_bytes, off_kept, kept_bytes;
    size_t off_values, off_exponents;          // in what is kept, behind h
};
static FfnLayout ffn_layout(const wlb_ffn_desc& d) {
    FfnLayout L;
    const size_t n = d.n_rows, f = d.inner, h = d.hidden, operand = operand_rows(d.n_rows);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    const bool gaps = d.n_rows < d.n_q;
    L.off_parts = take(std::max<size_t>(1, ffn_parts_bytes(d.n_rows, d.hidden, d.inner)));          // a workspace of no bytes would have no address
    L.off_x = take(gaps ? 2 * n * h : 0);
    L.off_h = at;                    // where nothing is kept
    L.fwd_bytes = at + align_up(2 * operand * f, 256);
    L.off_d = take(4 * operand * f);
    L.off_dy = take(gaps ? 2 * n * h : 0);
    L.off_x2 = take(operand > n ? 4 * n * h : 0);
    L.off_dy2 = take(operand > n ? 4 * n * h : 0);
    L.bwd_bytes = at;
    L.off_values = align_up(2 * operand * f, 256);
    L.off_exponents = L.off_values + 1024 * Kept::blocks(d.n_rows, 16) * Kept::blocks(d.inner, 16);
    L.kept_bytes = L.off_exponents + 512 * Kept::blocks(d.n_rows, 16) * Kept::blocks(d.inner, 64);
    L.off_kept = at;                 // where the backward makes what the forward has not kept
    return L;
}
static Kept kept_at(const void* at, const FfnLayout& L, int inner) {
    char* p = (char*)at;
    return Kept{(__bf16*)p, p + L.off_values, p + L.off_exponents, inner};
}

}  // namespace wlb

using namespace wlb;

extern "C" wlb_status wlb_ffn_workspace_size(const wlb_ffn_desc* desc, size_t* kept_bytes, size_t* fwd_bytes, size_t* bwd_bytes) {
    if (wlb_status st = check_ffn(desc, "wlb_ffn_workspace_size")) return st;
    const FfnLayout L = ffn_layout(*desc);
    if (kept_bytes) *kept_bytes = L.kept_bytes;
    if (fwd_bytes) *fwd_bytes = L.fwd_bytes;
    if (bwd_bytes) *bwd_bytes = L.bwd_bytes;
    return WLB_OK;
}

extern "C" wlb_status wlb_ffn_fwd(const wlb_ffn_desc* desc, const void* x, const int32_t* rows, const void* w_in, const void* w_out, const void* residual, void* y, void* kept,
                                  void* workspace, size_t workspace_bytes, void* stream_) {
    const char* call = "wlb_ffn_fwd";
    if (wlb_status st = check_ffn(desc, call)) return st;
    const wlb_ffn_desc& d = *desc;
    if (!x || !w_in || !w_out || !y || !workspace) return fail(WLB_ERR_INVALID_ARG, "%s: null pointer", call);
    if (misaligned(x, 16) || misaligned(w_in, 16) || misaligned(w_out, 16) || misaligned(residual, 16) || misaligned(y, 16) || misaligned(kept, 16) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    if (wlb_status st = check_list(call, d.n_q, d.n_rows, rows)) return st;
    const FfnLayout L = ffn_layout(d);
    if (workspace_bytes < L.fwd_bytes) return fail(WLB_ERR_BUFFER_TOO_SMALL, "%s: workspace %zu < %zu bytes", call, workspace_bytes, L.fwd_bytes);
    hipStream_t stream = (hipStream_t)stream_;
    char* ws = (char*)workspace;
    float* parts = (float*)(ws + L.off_parts);
    const Kept to = kept ? kept_at(kept, L, d.inner) : Kept{(__bf16*)(ws + L.off_h), nullptr, nullptr, d.inner};
    if (rows) {
        GatherArgs z = {};
        z.src[0] = (const uint4*)x; z.dst[0] = (uint4*)(ws + L.off_x); z.chunks[0] = d.hidden / 8;
        z.zero = (uint4*)y; z.zero_chunks = d.hidden / 8; z.rows = rows; z.n_q = d.n_q; z.n_rows = d.n_rows;
        launch_gather(z, stream);
        x = z.dst[0];
    }
    GateArgs g = {(const __bf16*)x, (const __bf16*)w_in, d.n_rows, d.hidden, d.inner, to, parts, {}};
    launch_gate(d.activation, g, stream);
    ProductArgs a = {};
    a.p = (const __bf16*)w_out; a.ldp = d.inner; a.pm = d.hidden;
    a.q = to.h; a.ldq = d.inner; a.qn = operand_rows(d.n_rows); a.twin = a.qn > d.n_rows ? d.n_rows : 0; a.depth = d.inner;
    a.to = rows; a.out_limit = d.n_q; a.out = (__bf16*)y; a.ldo = d.hidden; a.residual = (const __bf16*)residual; a.act = WLB_ACT_NONE; a.parts = parts;
    launch_product(Kinds::KK, a, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "feed-forward launch: %s", hipGetErrorString(e));
    return WLB_OK;
}

extern "C" wlb_status wlb_ffn_bwd(const wlb_ffn_desc* desc, const void* x, const int32_t* rows, const void* w_in, const void* w_out, const void* kept, const void* dy, void* dx,
                                  void* dw_in, void* dw_out, void* workspace, size_t workspace_bytes, void* stream_) {
    const char* call = "wlb_ffn_bwd";
    if (wlb_status st = check_ffn(desc, call)) return st;
    const wlb_ffn_desc& d = *desc;
    if (!x || !w_in || !w_out || !dy || !workspace) return fail(WLB_ERR_INVALID_ARG, "%s: null pointer", call);
    if (misaligned(x, 16) || misaligned(w_in, 16) || misaligned(w_out, 16) || misaligned(kept, 16) || misaligned(dy, 16) || misaligned(dx, 16) || misaligned(dw_in, 16) ||
        misaligned(dw_out, 16) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    if (wlb_status st = check_list(call, d.n_q, d.n_rows, rows)) return st;
    const FfnLayout L = ffn_layout(d);
    const size_t need = L.bwd_bytes + (kept ? 0 : L.kept_bytes);
    if (workspace_bytes < need) return fail(WLB_ERR_BUFFER_TOO_SMALL, "%s: workspace %zu < %zu bytes", call, workspace_bytes, need);
    hipStream_t stream = (hipStream_t)stream_;
    char* ws = (char*)workspace;
    float* parts = (float*)(ws + L.off_parts);
    __bf16* dgu = (__bf16*)(ws + L.off_d);
    const __bf16 *xs = (const __bf16*)x, *dys = (const __bf16*)dy;
    if (rows) {
        GatherArgs g = {};
        g.src[0] = (const uint4*)x; g.dst[0] = (uint4*)(ws + L.off_x); g.chunks[0] = d.hidden / 8;
        g.src[1] = (const uint4*)dy; g.dst[1] = (uint4*)(ws + L.off_dy); g.chunks[1] = d.hidden / 8;
        g.zero = (uint4*)dx; g.zero_chunks = d.hidden / 8; g.rows = rows; g.n_q = d.n_q; g.n_rows = d.n_rows;
        launch_gather(g, stream);
        xs = (const __bf16*)(ws + L.off_x);
        dys = (const __bf16*)(ws + L.off_dy);
    }
    const Kept from = kept_at(kept ? kept : ws + L.off_kept, L, d.inner);
    if (!kept) {
        GateArgs g = {xs, (const __bf16*)w_in, d.n_rows, d.hidden, d.inner, from, parts, {}};
        launch_gate(d.activation, g, stream);
    }
    const int operand = operand_rows(d.n_rows), twin = operand > d.n_rows ? d.n_rows : 0;
    TwiceArgs twice = {{twin && dw_in ? (const uint4*)xs : nullptr, twin && dw_out ? (const uint4*)dys : nullptr}, {(uint4*)(ws + L.off_x2), (uint4*)(ws + L.off_dy2)}, d.n_rows, d.hidden / 8};
    if (dw_in || dx) {
        InnerArgs i = {(const __bf16*)w_out, dys, d.n_rows, d.hidden, d.inner, from, dgu, parts, {}, twice};
        launch_inner(i, stream);
    } else if (twin && dw_out) {
        launch_twice(twice, stream);
    }
    if (twin) {
        xs = (const __bf16*)twice.dst[0];
        dys = (const __bf16*)twice.dst[1];
    }
    ProductArgs to_x = {}, to_in = {}, to_out = {}, *to_weights[2];
    int n_weights = 0;
    if (dx) {
        ProductArgs& a = to_x;
        a.p = (const __bf16*)w_in; a.ldp = d.hidden; a.pm = d.hidden;
        a.q = dgu; a.ldq = 2ll * d.inner; a.qn = operand; a.twin = twin; a.depth = 2 * d.inner;
        a.to = rows; a.out_limit = d.n_q; a.out = (__bf16*)dx; a.ldo = d.hidden; a.parts = parts;
    }
    if (dw_in) {
        ProductArgs& a = to_in;
        a.p = xs; a.ldp = d.hidden; a.pm = d.hidden;
        a.q = dgu; a.ldq = 2ll * d.inner; a.qn = 2 * d.inner; a.depth = operand;
        a.out = (__bf16*)dw_in; a.ldo = d.hidden; a.parts = parts;
        to_weights[n_weights++] = &to_in;
    }
    if (dw_out) {
        ProductArgs& a = to_out;
        a.p = from.h; a.ldp = d.inner; a.pm = d.inner;
        a.q = dys; a.ldq = d.hidden; a.qn = d.hidden; a.depth = operand;
        a.out = (__bf16*)dw_out; a.ldo = d.inner; a.parts = parts;
        to_weights[n_weights++] = &to_out;
    }
    launch_gradients(dx ? &to_x : nullptr, to_weights, n_weights, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "feed-forward gradient launch: %s", hipGetErrorString(e));
    return WLB_OK;
}
