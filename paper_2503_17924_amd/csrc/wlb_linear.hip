// Product of a rank's slots with a weight, with bias, activation and residual in its epilogue, and its gradient (wlb_linear_fwd / wlb_linear_bwd); and the
// products without an epilogue that the feed-forward block consists of.
//
//   forward   z = x W^T + b, y = act(z) + r
//   backward  dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum of dz's rows
// Only slots that hold a token take part: where there is padding, products take their rows from a copy without gaps (in the launch that clears the padding's rows of the
// result: fetched by a list inside the products they cost 2 us a tile) and leave theirs in the slots.  dz is rounded to bf16 where there is an activation (up to
// kExactSlots slots in two parts).  The forward keeps the slopes, of the unrounded z, in fp16: they lie between -0.2 and 1.2, so its 2^-11 of them (2^-25 below
// 2^-14) are an eighth of dz's own rounding.
// Bound by the matrix products, by the weight's bytes up to about 64 slots.
#include "wlb_dense.h"

namespace wlb {

struct ProductWork : GemmGrid {
    const ProductArgs& a;
    int qn;
    long long ldp, ldq;
    __device__ __forceinline__ explicit ProductWork(const ProductArgs& a_) : GemmGrid(a_.grid), a(a_), qn(a_.qn), ldp(a_.ldp), ldq(a_.ldq) {}
};

template <class S>
struct ProductOperands : ProductWork {
    __device__ __forceinline__ explicit ProductOperands(const ProductArgs& a_) : ProductWork(a_) {}
    __device__ __forceinline__ GemmOperand p(const GemmItem& i) const {
        const int m0 = i.tm * S::TM;
        return GemmOperand{S::MP ? a.p + (long long)i.k0 * ldp + m0 : a.p + (long long)m0 * ldp + i.k0, a.pm - m0, nullptr};
    }
    __device__ __forceinline__ GemmOperand q(const GemmItem& i) const {
        const int n0 = i.tn * S::TN;
        return GemmOperand{S::MQ ? a.q + (long long)i.k0 * ldq + n0 : a.q + (long long)n0 * ldq + i.k0, a.qn - n0, nullptr};
    }
};

// Whether slopes are kept: known when compiled (wide tiles' ends are long), or by the arguments.
enum { kKeepNot, kKeep, kKeepAsked };
// N values of a row n of the product, from column m on, on their way to row `slot` of the output, with the bias's and the residual's.
template <class T, int N> using vec = T __attribute__((ext_vector_type(N)));
template <int Act, int Keep, int N>
__device__ __forceinline__ void finish(const ProductArgs& a, int n, int m, vec<float, N> v, int slot, const vec<__bf16, N>& bias, const vec<__bf16, N>& residual) {
    if (m >= a.pm || (unsigned)slot >= (unsigned)a.out_limit) return;
    vec<__bf16, N> out;
    if (Act != WLB_ACT_NONE && Keep != kKeepNot && (Keep == kKeep || a.kept)) {
        vec<_Float16, N> s;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float value, slope;
            activated<Act>(v[k] + (float)bias[k], value, slope);
            out[k] = (__bf16)(value + (float)residual[k]);
            s[k] = (_Float16)slope;
        }
        *reinterpret_cast<vec<_Float16, N>*>(a.kept + (size_t)n * a.pm + m) = s;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = (__bf16)(activated<Act>(v[k] + (float)bias[k]) + (float)residual[k]);
    }
    *reinterpret_cast<vec<__bf16, N>*>(a.out + (size_t)slot * a.ldo + m) = out;
}
template <int N>
__device__ __forceinline__ vec<__bf16, N> some(const __bf16* at, bool there) {
    vec<__bf16, N> v = {};
    if (at && there) v = *reinterpret_cast<const vec<__bf16, N>*>(at);
    return v;
}

// What a kernel's epilogue has: nothing, bias and activation, or with those what moves rows in 32 bits: a residual, and slopes that are kept.
enum { kPlain, kBias, kRows, kRowsKept };

template <class S, int Epilogue, int Act>
struct ProductDone {
    const ProductArgs& a;
    const ProductWork& w;
    struct Ahead { int slot[row_regs<S>()]; };
    __device__ __forceinline__ Ahead load(const Gemm<S>& g, const GemmItem& it) const {
        Ahead h;
#pragma unroll
        for (int k = 0; k < row_regs<S>(); ++k) {
            const int row = row_held<S>(g, it, k);
            h.slot[k] = row >= a.qn || (a.twin && row >= a.twin) ? -1 : a.to ? a.to[row] : row;
        }
        return h;
    }
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, const Ahead& h, uint32_t room) const {
        if constexpr (S::DIVIDES)
            if (it.part >= 0) {
                g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), a.qn - it.tn * S::TN);
                return 0;
            }
        const int m0 = it.tm * S::TM, n0 = it.tn * S::TN;
        const bool full = !a.to && n0 + S::TN <= a.qn && m0 + S::TM <= a.pm;
        auto slot_of = [&](int n, int j) __attribute__((always_inline)) { return __shfl(h.slot[j / 4], n - g.wn * (S::BN * 16) - j / 4 * 64); };
        auto there = [&](int slot, int m) __attribute__((always_inline)) { return (unsigned)slot < (unsigned)a.out_limit && m0 + m < a.pm; };
        auto put = [&](int n, int m, const i32x4& v, int j) __attribute__((always_inline)) {
            const int slot = slot_of(n, j);
            if (there(slot, m)) *reinterpret_cast<i32x4*>(a.out + (size_t)slot * a.ldo + m0 + m) = v;
        };
        if constexpr (Epilogue == kPlain) {
            g.template rows_out<2>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return g.sum(i, j, r); }, put);
            return full ? row_stores<S, 2>() : 0;
        } else if constexpr (Epilogue == kBias) {
            const int first = m0 + g.wm * (S::BM * 16) + (g.lane / 16) * 4;         // column of register 0 of block 0
            float bias[S::BM][4];
#pragma unroll
            for (int i = 0; i < S::BM; ++i) {
                const bf16x4 b = some<4>(a.bias ? a.bias + first + i * 16 : nullptr, first + i * 16 < a.pm);
#pragma unroll
                for (int r = 0; r < 4; ++r) bias[i][r] = (float)b[r];
            }
            g.template rows_out<2>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return activated<Act>(g.sum(i, j, r) + bias[i][r]); }, put);
            return full ? row_stores<S, 2>() : 0;
        } else {
            // a lane's columns are the same in every row: one or two groups of 8
            constexpr int G = S::BM < 4 ? S::BM : 4;
            bf16x8 bias[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int m = m0 + g.wm * (S::BM * 16) + i * 64 + g.lane % (G * 2) * 8;
                bias[i] = some<8>(a.bias ? a.bias + m : nullptr, i * 4 < S::BM && m < a.pm);
            }
            g.rows_out_beside(room, [&](int i, int j, int r) __attribute__((always_inline)) { return g.sum(i, j, r); },
                              [&](int n, int m, int j) __attribute__((always_inline)) {
                                  const int slot = slot_of(n, j);
                                  return some<8>(a.residual ? a.residual + (size_t)slot * a.ldo + m0 + m : nullptr, there(slot, m));
                              },
                              [&](int n, int m, const f32x4& low, const f32x4& high, int j, int part, const bf16x8& r) __attribute__((always_inline)) {
                                  finish<Act, S::RING ? (Epilogue == kRowsKept ? kKeep : kKeepNot) : kKeepAsked, 8>(
                                      a, n0 + n, m0 + m, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7), slot_of(n, j), bias[part], r);
                              });
            return full ? row_stores<S, 2>() : 0;
        }
    }
};

template <class S, int Epilogue, int Act>
__global__ void __launch_bounds__(256, S::PER_CU) product_kernel(ProductArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const ProductOperands<S> w(a);
    Gemm<S> gemm;
    gemm.run(smem, w, ProductDone<S, Epilogue, Act>{a, w});
}

template <class S>
__global__ void __launch_bounds__(256) product_join_kernel(ProductArgs a) {
    const ProductWork w(a);
    auto join = [&](int tm, int tn, int n, int m, const f32x4& v) __attribute__((always_inline)) {
        const int row = tn * S::TN + n, col = tm * S::TM + m;
        if (row >= a.qn || (a.twin && row >= a.twin)) return;
        const int slot = a.to ? a.to[row] : row;
        const bool there = col < a.pm && (unsigned)slot < (unsigned)a.out_limit;
        const bf16x4 b = some<4>(a.bias ? a.bias + col : nullptr, there), r = some<4>(a.residual ? a.residual + (size_t)slot * a.ldo + col : nullptr, there);
        with_activation(a.act, [&](auto act) __attribute__((always_inline)) { finish<decltype(act)::value, kKeepAsked, 4>(a, row, col, v, slot, b, r); });
    };
    join_any<S>(w, a.parts, join, a.twin);
}

template <class S, int Epilogue, int Act>
static void launch_one(ProductArgs& a, hipStream_t stream) {
    product_kernel<S, Epilogue, Act><<<a.grid.workgroups, 256, 0, stream>>>(a);
    if (a.grid.left) product_join_kernel<S><<<join_grid<S>(a.grid), 256, 0, stream>>>(a);
}
template <class S, int Act>
static void launch_activated(ProductArgs& a, hipStream_t stream) {
    if constexpr (S::RING) {
        if (Act != WLB_ACT_NONE && a.kept) return launch_one<S, kRowsKept, Act>(a, stream);
        if (!a.residual) return launch_one<S, kBias, Act>(a, stream);
    }
    launch_one<S, kRows, Act>(a, stream);
}
template <class S>
static void launch_epilogue(ProductArgs& a, hipStream_t stream) {
    if constexpr (S::MP || S::MQ) return launch_one<S, kPlain, WLB_ACT_NONE>(a, stream);
    else if (a.act == WLB_ACT_RELU) launch_activated<S, WLB_ACT_RELU>(a, stream);
    else if (a.act == WLB_ACT_SILU) launch_activated<S, WLB_ACT_SILU>(a, stream);
    else if (a.act == WLB_ACT_GELU) launch_activated<S, WLB_ACT_GELU>(a, stream);
    else if (a.bias || a.residual) launch_activated<S, WLB_ACT_NONE>(a, stream);
    else launch_one<S, kPlain, WLB_ACT_NONE>(a, stream);
}
template <bool MP, bool MQ>
static void launch_tiles(int kind, ProductArgs& a, hipStream_t stream) {
    if (kind == kWideTiles) launch_epilogue<Wide<MP, MQ>>(a, stream);
    else if (kind == kSmallTiles) launch_epilogue<Small<MP, MQ>>(a, stream);
    else if (kind == kTinyTiles) launch_epilogue<Tiny<MP, MQ>>(a, stream);
    if constexpr (!MQ) {
        if (kind == kFewTiles32) launch_epilogue<Few<2, MP>>(a, stream);
        else if (kind == kFewTiles64) launch_epilogue<Few<4, MP>>(a, stream);
        else if (kind == kFewTiles128) launch_epilogue<Few<8, MP>>(a, stream);
    }
}

void launch_product(Kinds kinds, ProductArgs& a, hipStream_t stream) {
    if (a.qn == 0 || a.pm == 0) return;
    if (!a.to) a.out_limit = a.twin ? a.twin : a.qn;
    const Tiling t = plan_product(kinds, a);
    a.grid = t.grid;
    if (kinds == Kinds::KK) launch_tiles<false, false>(t.kind, a, stream);
    else if (kinds == Kinds::MK) launch_tiles<true, false>(t.kind, a, stream);
    else launch_tiles<true, true>(t.kind, a, stream);
}

// ------------------------------------------------------------------------------------------
// Several products in one launch (GroupArgs).
// Few slots: two workgroups to a compute unit, as of the small tiles that run beside them.
template <int BN> using FewBeside = GemmShape<4, 1, 2, BN, true, false, kDivSmall>;

template <class MK, class MM>
__global__ void __launch_bounds__(256, MM::PER_CU < MK::PER_CU ? MM::PER_CU : MK::PER_CU) group_kernel(GroupArgs g) {
    constexpr int BYTES = MK::LDS_BYTES > MM::LDS_BYTES ? MK::LDS_BYTES : MM::LDS_BYTES;
    __shared__ __attribute__((aligned(1024))) char smem[BYTES];
    const int side = (int)gridDim.x / kLists, x = (int)blockIdx.x % kLists, i = (int)blockIdx.x / kLists;
    auto block = [&](int turn) { return uniform((i + side - turn) % side * kLists + x); };
    if (g.a[0].qn > 0) {
        const ProductOperands<MK> w(g.a[0]);
        Gemm<MK> gemm;
        gemm.run(smem, w, ProductDone<MK, kPlain, WLB_ACT_NONE>{g.a[0], w}, block(g.turn[0]));
    }
    for (int k = 1; k < g.n; ++k) {
        __syncthreads();
        const ProductOperands<MM> w(g.a[k]);
        Gemm<MM> gemm;
        gemm.run(smem, w, ProductDone<MM, kPlain, WLB_ACT_NONE>{g.a[k], w}, block(g.turn[k]));
    }
}

template <class S>
static void join_last(const ProductArgs& a, hipStream_t stream) {
    if (a.grid.left) product_join_kernel<S><<<join_grid<S>(a.grid), 256, 0, stream>>>(a);
}

void launch_gradients(ProductArgs* dx, ProductArgs* const* dw, int n_dw, hipStream_t stream) {
    GroupArgs g = {};
    g.n = 1;
    if (dx) g.a[0] = *dx;
    for (int k = 0; k < n_dw; ++k) g.a[g.n++] = *dw[k];
    for (int k = 0; k < g.n; ++k)
        if (!g.a[k].to) g.a[k].out_limit = g.a[k].twin ? g.a[k].twin : g.a[k].qn;
    auto launch = [&](auto first, auto others) {
        group_kernel<decltype(first), decltype(others)><<<g.a[g.n - 1].grid.workgroups, 256, 0, stream>>>(g);
    };
    switch (plan_gradients(g)) {
    case kApart:
        if (dx) launch_product(Kinds::MK, *dx, stream);
        for (int k = 0; k < n_dw; ++k) launch_product(Kinds::MM, *dw[k], stream);
        break;
    case kWideGroup:
        launch(Wide<true, false>{}, Wide<true, true>{});
        join_last<Wide<true, true>>(g.a[g.n - 1], stream);
        break;
    case kSmallGroup:
        launch(Small<true, false>{}, Small<true, true>{});
        join_last<Small<true, true>>(g.a[g.n - 1], stream);
        break;
    case kTinyGroup:
        launch(Tiny<true, false>{}, Tiny<true, true>{});
        join_last<Tiny<true, true>>(g.a[g.n - 1], stream);
        break;
    // of few slots dx may be divided, beside the weights' whole tiles
    case kFewGroup32:
        launch(FewBeside<2>{}, Small<true, true>{});
        join_last<FewBeside<2>>(g.a[0], stream);
        break;
    case kFewGroup64:
        launch(FewBeside<4>{}, Small<true, true>{});
        join_last<FewBeside<4>>(g.a[0], stream);
        break;
    case kFewGroup128:
        launch(FewBeside<8>{}, Small<true, true>{});
        join_last<FewBeside<8>>(g.a[0], stream);
        break;
    case kFewGroupTiny:
        launch(Tiny<true, false>{}, Small<true, true>{});
        join_last<Tiny<true, false>>(g.a[0], stream);
        break;
    }
}

// ------------------------------------------------------------------------------------------
// Rows.
constexpr int kRowsGrid = 1 << 20;          // workgroups at most

__global__ void __launch_bounds__(256) gather_kernel(GatherArgs a) {
    const int lane = threadIdx.x & 63, first = a.dst[0] || a.dst[1] ? 0 : a.n_rows;
    for (int i = first + (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6); i < a.n_q; i += (int)gridDim.x * 4) {
        const int slot = a.rows[i];
        const bool in = (unsigned)slot < (unsigned)a.n_q;
        if (i < a.n_rows) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (!a.dst[k]) continue;
                for (int c = lane; c < a.chunks[k]; c += 64) a.dst[k][(size_t)i * a.chunks[k] + c] = in ? a.src[k][(size_t)slot * a.chunks[k] + c] : uint4{0, 0, 0, 0};
            }
        } else if (a.zero && in) {
            for (int c = lane; c < a.zero_chunks; c += 64) a.zero[(size_t)slot * a.zero_chunks + c] = uint4{0, 0, 0, 0};
        }
    }
}

void launch_gather(const GatherArgs& a, hipStream_t stream) {
    const int n = a.n_q - (a.dst[0] || a.dst[1] ? 0 : a.n_rows);
    if (n > 0) gather_kernel<<<std::min((n + 3) / 4, kRowsGrid), 256, 0, stream>>>(a);
}

__global__ void __launch_bounds__(256) twice_kernel(TwiceArgs a) { write_twice(a, (int)(blockIdx.x * 256 + threadIdx.x), (int)gridDim.x * 256); }
void launch_twice(const TwiceArgs& a, hipStream_t stream) { twice_kernel<<<std::min((a.rows * a.chunks + 255) / 256, 2 * wide_workgroups()), 256, 0, stream>>>(a); }

// dz = dy act'(z), rows without gaps, and the sums of its columns.  A workgroup has 512 columns, 8 to a lane, of a piece of the rows; the pieces are summed in order
// by a second launch.  Sums are of dz before it is rounded.
struct SlopeArgs {
    const _Float16* slope;           // [n_rows][width], or null: 1
    const __bf16* dy;                // [n_q][width]
    __bf16* dz;                      // or null
    int rest;                        // 0, or n_rows: behind that many rows of dz stands what bf16 leaves out of them
    float* sums;                     // [pieces][width], or null
    const int32_t* rows;             // or null
    int n_q, n_rows, width, pieces;
    TwiceArgs twice;
};
__global__ void __launch_bounds__(256) slope_kernel(SlopeArgs a) {
    write_twice(a.twice, (int)((blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x), (int)(gridDim.x * gridDim.y) * 256);
    __shared__ float s_sum[4][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = (int)blockIdx.x * 512 + lane * 8, piece = blockIdx.y;
    const int first = (int)((long long)a.n_rows * piece / a.pieces), end = (int)((long long)a.n_rows * (piece + 1) / a.pieces);
    float sum[8] = {};
    constexpr int kAhead = 4;
    if (col < a.width)
        for (int i0 = first + wave; i0 < end; i0 += 4 * kAhead) {
            bf16x8 d[kAhead];
            f16x8 s[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = i0 + 4 * k;
                d[k] = {};
                s[k] = {};
                if (i >= end) continue;
                const int slot = a.rows ? a.rows[i] : i;
                if ((unsigned)slot >= (unsigned)a.n_q) continue;          // its slopes were not written either
                d[k] = *reinterpret_cast<const bf16x8*>(a.dy + (size_t)slot * a.width + col);
                if (a.slope) s[k] = *reinterpret_cast<const f16x8*>(a.slope + (size_t)i * a.width + col);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = i0 + 4 * k;
                if (i >= end) continue;
                bf16x8 rest;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float v = a.slope ? (float)d[k][c] * (float)s[k][c] : (float)d[k][c];
                    sum[c] += v;
                    rest[c] = a.rest ? (__bf16)rest_of(v) : (__bf16)0.f;
                    d[k][c] = (__bf16)v;
                }
                if (a.dz) *reinterpret_cast<bf16x8*>(a.dz + (size_t)i * a.width + col) = d[k];
                if (a.dz && a.rest) *reinterpret_cast<bf16x8*>(a.dz + (size_t)(a.rest + i) * a.width + col) = rest;
            }
        }
    if (!a.sums) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) s_sum[wave][lane * 8 + k] = sum[k];
    __syncthreads();
    for (int c = threadIdx.x; c < 512; c += 256)
        if ((int)blockIdx.x * 512 + c < a.width) a.sums[(size_t)piece * a.width + blockIdx.x * 512 + c] = (s_sum[0][c] + s_sum[1][c]) + (s_sum[2][c] + s_sum[3][c]);
}
// Enough workgroups to fill the chip, of 16 rows at least.
constexpr int kSumPieces = 256;
static int sum_pieces(int n_rows, int width) { return std::min({kSumPieces, (n_rows + 15) / 16, std::max(64, 1024 / ((width + 511) / 512))}); }

// 32 columns to a workgroup, 8 threads to a column.
__global__ void __launch_bounds__(256) column_join_kernel(const float* part, __bf16* out, int width, int pieces) {
    __shared__ float s_sum[8][32];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = (int)blockIdx.x * 32 + x;
    constexpr int kAhead = 8;
    float sum = 0.f;
    if (col < width)
        for (int p0 = y; p0 < pieces; p0 += 8 * kAhead) {
            float v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) v[k] = p0 + 8 * k < pieces ? part[(size_t)(p0 + 8 * k) * width + col] : 0.f;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) sum += v[k];
        }
    s_sum[y][x] = sum;
    __syncthreads();
    if (y > 0 || col >= width) return;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += s_sum[k][x];
    out[col] = (__bf16)sum;
}

// ------------------------------------------------------------------------------------------
wlb_status check_rows(const char* call, int32_t n_q, int32_t n_rows, int32_t a, int32_t b, int32_t activation) {
    if (n_q < 1 || n_rows < 0 || n_rows > n_q || a < 1 || b < 1) return fail(WLB_ERR_INVALID_ARG, "%s: n_q=%d n_rows=%d widths %d and %d", call, n_q, n_rows, a, b);
    if (activation < WLB_ACT_NONE || activation > WLB_ACT_GELU) return fail(WLB_ERR_INVALID_ARG, "%s: activation %d", call, activation);
    if (a % 8 != 0 || b % 8 != 0 || a > (1 << 20) || b > (1 << 20)) return fail(WLB_ERR_UNSUPPORTED, "%s: widths %d and %d (multiples of 8 up to 2^20)", call, a, b);
    if (n_q > (1 << 30)) return fail(WLB_ERR_UNSUPPORTED, "%s: n_q=%d above 2^30", call, n_q);
    if ((int64_t)(std::max(a, b) / 64 + 1) * (n_q / 32 + 1) > (1 << 30) || (int64_t)(a / 64 + 1) * (b / 64 + 1) > (1 << 30))
        return fail(WLB_ERR_UNSUPPORTED, "%s: n_q=%d for widths %d and %d", call, n_q, a, b);
    return WLB_OK;
}

wlb_status check_list(const char* call, int32_t n_q, int32_t n_rows, const int32_t* rows) {
    if ((n_rows < n_q) != (rows != nullptr)) return fail(WLB_ERR_INVALID_ARG, "%s: rows goes with slots that hold no token (n_q=%d n_rows=%d)", call, n_q, n_rows);
    if (misaligned(rows, 4)) return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    return WLB_OK;
}

static wlb_status check_linear(const wlb_linear_desc* d, const char* call) {
    if (!d) return fail(WLB_ERR_INVALID_ARG, "%s: null desc", call);
    return check_rows(call, d->n_q, d->n_rows, d->n_in, d->n_out, d->activation);
}

struct LinearLayout {
    size_t off_parts, fwd_bytes, off_x, off_twice, off_dz, off_sums, bwd_bytes, off_kept, kept_bytes;
};
static LinearLayout linear_layout(const wlb_linear_desc& d) {
    LinearLayout L;
    const size_t n = d.n_rows, out = d.n_out;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    L.off_parts = take(std::max<size_t>(1, linear_parts_bytes(d.n_rows, d.n_in, d.n_out, d.activation)));          // a workspace of no bytes would have no address
    const bool gaps = d.n_rows < d.n_q;
    L.off_x = take(gaps ? 2 * n * d.n_in : 0);
    L.fwd_bytes = at;
    L.off_dz = take(d.activation != WLB_ACT_NONE ? 2 * (size_t)operand_rows(d.n_rows) * out : gaps ? 2 * n * out : 0);
    L.off_twice = take(d.activation != WLB_ACT_NONE && operand_rows(d.n_rows) > d.n_rows ? 4 * n * d.n_in : 0);
    L.off_sums = take(4 * (size_t)sum_pieces(d.n_rows, d.n_out) * out);
    L.bwd_bytes = at;
    L.kept_bytes = d.activation != WLB_ACT_NONE ? align_up(2 * n * out, 256) : 0;
    L.off_kept = at;                 // where the backward makes what the forward has not kept
    return L;
}

static ProductArgs forward_args(const wlb_linear_desc& d, const void* x, const void* weight, const void* bias) {
    ProductArgs a = {};
    a.p = (const __bf16*)weight; a.ldp = d.n_in; a.pm = d.n_out;
    a.q = (const __bf16*)x; a.ldq = d.n_in; a.qn = d.n_rows; a.depth = d.n_in;
    a.ldo = d.n_out; a.bias = (const __bf16*)bias; a.act = d.activation;
    return a;
}

}  // namespace wlb

using namespace wlb;

extern "C" wlb_status wlb_linear_workspace_size(const wlb_linear_desc* desc, size_t* kept_bytes, size_t* fwd_bytes, size_t* bwd_bytes) {
    if (wlb_status st = check_linear(desc, "wlb_linear_workspace_size")) return st;
    const LinearLayout L = linear_layout(*desc);
    if (kept_bytes) *kept_bytes = L.kept_bytes;
    if (fwd_bytes) *fwd_bytes = L.fwd_bytes;
    if (bwd_bytes) *bwd_bytes = L.bwd_bytes;
    return WLB_OK;
}

extern "C" wlb_status wlb_linear_fwd(const wlb_linear_desc* desc, const void* x, const int32_t* rows, const void* weight, const void* bias, const void* residual, void* y,
                                     void* kept, void* workspace, size_t workspace_bytes, void* stream_) {
    const char* call = "wlb_linear_fwd";
    if (wlb_status st = check_linear(desc, call)) return st;
    const wlb_linear_desc& d = *desc;
    if (!x || !weight || !y || !workspace) return fail(WLB_ERR_INVALID_ARG, "%s: null pointer", call);
    if (misaligned(x, 16) || misaligned(weight, 16) || misaligned(bias, 16) || misaligned(residual, 16) || misaligned(y, 16) || misaligned(kept, 16) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    if (kept && d.activation == WLB_ACT_NONE) return fail(WLB_ERR_INVALID_ARG, "%s: nothing is kept without an activation", call);
    if (wlb_status st = check_list(call, d.n_q, d.n_rows, rows)) return st;
    const LinearLayout L = linear_layout(d);
    if (workspace_bytes < L.fwd_bytes) return fail(WLB_ERR_BUFFER_TOO_SMALL, "%s: workspace %zu < %zu bytes", call, workspace_bytes, L.fwd_bytes);
    hipStream_t stream = (hipStream_t)stream_;
    if (rows) {
        GatherArgs g = {};
        g.src[0] = (const uint4*)x; g.dst[0] = (uint4*)((char*)workspace + L.off_x); g.chunks[0] = d.n_in / 8;
        g.zero = (uint4*)y; g.zero_chunks = d.n_out / 8; g.rows = rows; g.n_q = d.n_q; g.n_rows = d.n_rows;
        launch_gather(g, stream);
        x = g.dst[0];
    }
    ProductArgs a = forward_args(d, x, weight, bias);
    a.to = rows; a.out_limit = d.n_q; a.out = (__bf16*)y; a.residual = (const __bf16*)residual;
    a.kept = (_Float16*)kept; a.parts = (float*)((char*)workspace + L.off_parts);
    launch_product(Kinds::KK, a, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "linear launch: %s", hipGetErrorString(e));
    return WLB_OK;
}

extern "C" wlb_status wlb_linear_bwd(const wlb_linear_desc* desc, const void* x, const int32_t* rows, const void* weight, const void* bias, const void* kept, const void* dy,
                                     void* dx, void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream_) {
    const char* call = "wlb_linear_bwd";
    if (wlb_status st = check_linear(desc, call)) return st;
    const wlb_linear_desc& d = *desc;
    if (!x || !weight || !dy || !workspace) return fail(WLB_ERR_INVALID_ARG, "%s: null pointer", call);
    if (misaligned(x, 16) || misaligned(weight, 16) || misaligned(bias, 16) || misaligned(kept, 16) || misaligned(dy, 16) || misaligned(dx, 16) || misaligned(dweight, 16) ||
        misaligned(dbias, 16) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    const bool act = d.activation != WLB_ACT_NONE, again = act && !kept;
    if (kept && !act) return fail(WLB_ERR_INVALID_ARG, "%s: nothing is kept without an activation", call);
    if (wlb_status st = check_list(call, d.n_q, d.n_rows, rows)) return st;
    const LinearLayout L = linear_layout(d);
    const size_t need = L.bwd_bytes + (again ? L.kept_bytes : 0);
    if (workspace_bytes < need) return fail(WLB_ERR_BUFFER_TOO_SMALL, "%s: workspace %zu < %zu bytes", call, workspace_bytes, need);
    hipStream_t stream = (hipStream_t)stream_;
    char* ws = (char*)workspace;
    float* parts = (float*)(ws + L.off_parts);
    __bf16* dz_room = (__bf16*)(ws + L.off_dz);
    const __bf16 *xs = (const __bf16*)x, *dz = (const __bf16*)dy;
    if (rows) {
        GatherArgs g = {};
        g.src[0] = (const uint4*)x; g.dst[0] = dweight || again ? (uint4*)(ws + L.off_x) : nullptr; g.chunks[0] = d.n_in / 8;
        g.zero = (uint4*)dx; g.zero_chunks = d.n_in / 8; g.rows = rows; g.n_q = d.n_q; g.n_rows = d.n_rows;
        launch_gather(g, stream);
        xs = (const __bf16*)(ws + L.off_x);
    }
    if (again && d.n_rows > 0) {
        // the activation's output goes where dz is written afterwards
        ProductArgs a = forward_args(d, xs, weight, bias);
        a.out = dz_room; a.kept = (_Float16*)(ws + L.off_kept); a.parts = parts;
        launch_product(Kinds::KK, a, stream);
        kept = a.kept;
    }
    const int pieces = sum_pieces(d.n_rows, d.n_out);
    float* sums = (float*)(ws + L.off_sums);
    const bool own_dz = rows || act;
    const int dz_rows = act ? operand_rows(d.n_rows) : d.n_rows, twin = dz_rows > d.n_rows ? d.n_rows : 0;
    const TwiceArgs twice = {{twin && dweight ? (const uint4*)xs : nullptr, nullptr}, {(uint4*)(ws + L.off_twice), nullptr}, d.n_rows, d.n_in / 8};
    if (d.n_rows > 0 && (own_dz || dbias)) {
        const SlopeArgs s = {act ? (const _Float16*)kept : nullptr, (const __bf16*)dy, own_dz ? dz_room : nullptr, twin, dbias ? sums : nullptr, rows, d.n_q, d.n_rows, d.n_out, pieces, twice};
        slope_kernel<<<dim3((d.n_out + 511) / 512, pieces), 256, 0, stream>>>(s);
    }
    if (own_dz) dz = dz_room;
    if (dbias) column_join_kernel<<<(d.n_out + 31) / 32, 256, 0, stream>>>(sums, (__bf16*)dbias, d.n_out, pieces);
    ProductArgs to_x = {}, to_weight = {}, *to_weights[1] = {&to_weight};
    if (dx) {
        ProductArgs& a = to_x;
        a.p = (const __bf16*)weight; a.ldp = d.n_in; a.pm = d.n_in;
        a.q = dz; a.ldq = d.n_out; a.qn = dz_rows; a.twin = twin; a.depth = d.n_out;
        a.to = rows; a.out_limit = d.n_q; a.out = (__bf16*)dx; a.ldo = d.n_in; a.parts = parts;
    }
    if (dweight) {
        ProductArgs& a = to_weight;
        a.p = twin ? (const __bf16*)twice.dst[0] : xs; a.ldp = d.n_in; a.pm = d.n_in;
        a.q = dz; a.ldq = d.n_out; a.qn = d.n_out; a.depth = dz_rows;
        a.out = (__bf16*)dweight; a.ldo = d.n_in; a.parts = parts;
    }
    launch_gradients(dx ? &to_x : nullptr, to_weights, dweight ? 1 : 0, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "linear gradient launch: %s", hipGetErrorString(e));
    return WLB_OK;
}
