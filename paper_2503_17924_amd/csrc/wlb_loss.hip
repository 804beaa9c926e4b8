// Cross entropy of a rank's slots over the whole vocabulary, and its gradient, without the logits ever being kept
// (wlb_loss_fwd / wlb_loss_bwd).
//
// With c = scale, l = <x, E_v> in fp32 sums of the MFMAs, n labelled slots:
//   forward   one product l = X E^T.  A tile of 256 words x up to 256 slots leaves per slot its maximum and its sum of exp(c (l - max)), and the
//             target's l where the tile holds it; loss_join_kernel combines a slot's tiles: lse = c max + ln sum, loss = c (max - l_t) + ln sum.
//   backward  D = w (exp(c l - lse) - [v = target]) with w = d_loss / G, G the largest |d_loss|, in bf16, for one piece of the vocabulary at a
//             time; then dE = c G D^T X for the piece's rows and dX += D E over the pieces, in fp32; dX is scaled by c G at the end.
//             G keeps the factor that most training steps have in common (1 / tokens) out of the rounding of D.
// Slots without a target are left out of everything: the others are listed in order (rows), and products run over that list.
// Bound by the matrix products: 2 n V H operations forward, 6 n V H backward, where 64 slots or more share the table's
// rows; by the table's bytes below that.
#include <algorithm>
#include <cmath>

#include "wlb_gemm.h"
#include "wlb_vocab.h"

namespace wlb {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWordTile = 256;                 // words (forward, D) and columns of hidden (dX) per tile
constexpr int kRowsThreads = 1024;

// ------------------------------------------------------------------------------------------
// The labelled slots.
struct RowsArgs {
    const int32_t *tokens, *q_idx, *cu;
    int32_t *slot_target;            // [n_q] target of a slot, -1: none
    int32_t *block_count;            // [blocks] labelled slots of each block of kRowsThreads
    float *block_max;                // [blocks] largest |d_loss| of them
    int32_t *rows, *target;          // [labelled] slot and target, by row
    float *row_lse, *row_weight;     // backward: [labelled]
    int32_t *count;                  // labelled slots
    float *factor;                   // backward: c G
    const float *lse_in, *d_loss;    // backward, else null
    float *loss_out, *lse_out;       // forward, else null
    int n_q, t_kv, n_docs, vocab, blocks;
    float scale;
};

__device__ __forceinline__ int slot_target(const RowsArgs& a, int i) {
    const int g = a.q_idx[i];
    if ((unsigned)g >= (unsigned)a.t_kv || g + 1 >= a.t_kv) return -1;
    int lo = 0, hi = a.n_docs + 1;                  // first offset above g: the end of g's document
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid] <= g) lo = mid + 1; else hi = mid;
    }
    if (lo > a.n_docs || lo == 0 || g + 1 >= a.cu[lo]) return -1;
    const int t = a.tokens[g + 1];
    return (unsigned)t < (unsigned)a.vocab ? t : -1;
}

__device__ __forceinline__ void block_sum_max(int& sum, float& most, int* s_sum, float* s_max) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o);
        most = fmaxf(most, __shfl_xor(most, o));
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { s_sum[threadIdx.x >> 6] = sum; s_max[threadIdx.x >> 6] = most; }
    __syncthreads();
    sum = 0; most = 0;
    for (int w = 0; w < kRowsThreads / 64; ++w) { sum += s_sum[w]; most = fmaxf(most, s_max[w]); }
}

__global__ void __launch_bounds__(kRowsThreads) loss_targets_kernel(RowsArgs a) {
    __shared__ int s_sum[kRowsThreads / 64];
    __shared__ float s_max[kRowsThreads / 64];
    const int i = (int)(blockIdx.x * kRowsThreads + threadIdx.x);
    const int t = i < a.n_q ? slot_target(a, i) : -1;
    if (i < a.n_q) a.slot_target[i] = t;
    int sum = t >= 0;
    float most = t >= 0 && a.d_loss ? fabsf(a.d_loss[i]) : 0.f;
    block_sum_max(sum, most, s_sum, s_max);
    if (threadIdx.x == 0) { a.block_count[blockIdx.x] = sum; a.block_max[blockIdx.x] = most; }
}

// One: a single block that finds the targets as well.
template <bool One>
__global__ void __launch_bounds__(kRowsThreads) loss_rows_kernel(RowsArgs a) {
    __shared__ int s_sum[kRowsThreads / 64];
    __shared__ float s_max[kRowsThreads / 64];
    const int i = (int)(blockIdx.x * kRowsThreads + threadIdx.x), wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int t = -1;
    if (i < a.n_q) t = One ? slot_target(a, i) : a.slot_target[i];
    if (One && i < a.n_q) a.slot_target[i] = t;
    int before = 0, total = 0;
    float most = 0;
    if (One) {
        total = t >= 0;
        most = t >= 0 && a.d_loss ? fabsf(a.d_loss[i]) : 0.f;
        block_sum_max(total, most, s_sum, s_max);
    } else {
        for (int b = threadIdx.x; b < a.blocks; b += kRowsThreads) {
            const int n = a.block_count[b];
            if (b < (int)blockIdx.x) before += n;
            total += n;
            most = fmaxf(most, a.block_max[b]);
        }
        float unused = 0;
        block_sum_max(total, most, s_sum, s_max);
        block_sum_max(before, unused, s_sum, s_max);
    }
    const unsigned long long has = __ballot(t >= 0);
    __syncthreads();
    if (lane == 0) s_sum[wave] = __popcll(has);
    __syncthreads();
    int row = before + __popcll(has & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) row += s_sum[w];
    // the largest |d_loss| is taken out of the weights where it is a number to divide by
    const bool divide = most > 0.f && most <= 3.0e38f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *a.count = total;
        if (a.d_loss) *a.factor = divide ? a.scale * most : a.scale;
    }
    if (i >= a.n_q) return;
    if (t < 0) {
        if (a.loss_out) { a.loss_out[i] = 0.f; a.lse_out[i] = -INFINITY; }
        return;
    }
    a.rows[row] = i;
    a.target[row] = t;
    if (a.d_loss) {
        a.row_lse[row] = a.lse_in[i];
        a.row_weight[row] = divide ? a.d_loss[i] / most : a.d_loss[i];
    }
}

// ------------------------------------------------------------------------------------------
// Workgroup -> tile of an ntm x ntn grid.  Workgroup b runs on XCD b % 8; each XCD takes a consecutive share of the tiles in bands of
// kBand tiles along n, so that the workgroups that run side by side on it share kBand operand tiles along n and a few along m in its L2.
constexpr int kBand = 8;
__device__ __forceinline__ bool find_tile(int ntm, int ntn, int layers, int& tm, int& tn, int& layer) {
    const int plane = ntm * ntn, all = plane * layers, per = (all + kLists - 1) / kLists, i = (int)blockIdx.x / kLists;
    int t = ((int)blockIdx.x % kLists) * per + i;
    if (i >= per || t >= all) return false;
    layer = t / plane;
    t -= layer * plane;
    const int band = t / (kBand * ntm), high = min(kBand, ntn - band * kBand);
    t -= band * kBand * ntm;
    tm = t / high;
    tn = band * kBand + t % high;
    return true;
}
static unsigned tile_grid(long long tiles) { return (unsigned)((tiles + kLists - 1) / kLists * kLists); }

// ------------------------------------------------------------------------------------------
struct StatsArgs {
    const __bf16 *x, *table;
    const int32_t *rows, *target, *count;
    float2* part;                    // [word tiles][pitch]: maximum of l and sum of exp(c (l - maximum)) of a row in a tile
    float* target_logit;             // [labelled]
    int vocab, hidden, pitch;
    float c2;                        // scale * log2(e)
};

template <class S>
__global__ void __launch_bounds__(256, S::LDS_BYTES > 81920 ? 1 : 2) loss_stats_kernel(StatsArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const int n_rows = ld_const(a.count);
    int tm, tn, unused;
    if (!find_tile((a.vocab + S::TM - 1) / S::TM, (n_rows + S::TN - 1) / S::TN, 1, tm, tn, unused)) return;
    const int m0 = tm * S::TM, n0 = tn * S::TN;
    Gemm<S> g;
    g.start(smem);
    g.run(GemmOperand{a.table + (size_t)m0 * a.hidden, a.hidden, a.vocab - m0, nullptr}, GemmOperand{a.x, a.hidden, n_rows - n0, a.rows + n0}, a.hidden);
    const int first = m0 + g.wm * (S::BM * 32) + (g.lane / 32) * 4;       // word of register 0 of block 0
    if (m0 + S::TM > a.vocab) {
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int j = 0; j < S::BN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (first + i * 32 + (r / 4) * 8 + r % 4 >= a.vocab) g.acc[i][j][r] = -INFINITY;
    }
    float2* s_part = (float2*)smem;                                       // [WM][TN]
#pragma unroll
    for (int j = 0; j < S::BN; ++j) {
        const int n = g.wn * (S::BN * 32) + j * 32 + g.lane % 32;
        const int t = n0 + n < n_rows ? a.target[n0 + n] - first : -1;    // register that holds the target, if this lane has it
        float most = -INFINITY, at_target = 0.f;
        bool mine = false;
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, g.acc[i][j][r]);
        most = fmaxf(most, xhalf(most));
        if (__any(t >= 0 && t < S::BM * 32)) {
#pragma unroll
            for (int i = 0; i < S::BM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (t == i * 32 + (r / 4) * 8 + r % 4) { mine = true; at_target = g.acc[i][j][r]; }
            if (mine) a.target_logit[n0 + n] = at_target;
        }
        const float ref = most == -INFINITY ? 0.f : most;                 // a wavefront all of whose words lie past the end
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += fast_exp2((g.acc[i][j][r] - ref) * a.c2);
        sum += xhalf(sum);
        if (g.lane < 32) s_part[g.wm * S::TN + n] = float2{most, sum};
    }
    __syncthreads();
    for (int n = threadIdx.x; n < S::TN; n += 256) {
        if (n0 + n >= n_rows) continue;
        float most = s_part[n].x, sum = 0.f;
#pragma unroll
        for (int w = 1; w < S::WM; ++w) most = fmaxf(most, s_part[w * S::TN + n].x);
#pragma unroll
        for (int w = 0; w < S::WM; ++w) {
            const float2 p = s_part[w * S::TN + n];
            sum += p.x == -INFINITY ? p.y : p.y * fast_exp2((p.x - most) * a.c2);      // p.y is 0 where every word lies past the end, or NaN
        }
        a.part[(size_t)tm * a.pitch + n0 + n] = float2{most, sum};
    }
}

// A slot's tiles combined: 32 rows to a workgroup, 8 threads to a row.
__global__ void __launch_bounds__(256) loss_join_kernel(const float2* part, const float* target_logit, const int32_t* rows, const int32_t* count, float* loss,
                                                        float* lse, int tiles, int pitch, float scale) {
    __shared__ float2 s_part[8][32];
    const int n_rows = *count, x = threadIdx.x & 31, y = threadIdx.x >> 5, row = (int)blockIdx.x * 32 + x;
    const float c2 = scale * kLog2e;
    if ((int)blockIdx.x * 32 >= n_rows) return;
    float most = -INFINITY, sum = 0.f;
    if (row < n_rows)
        for (int t = y; t < tiles; t += 8) {
            const float2 p = part[(size_t)t * pitch + row];
            const float m = fmaxf(most, p.x);
            sum = (most == -INFINITY ? sum : sum * fast_exp2((most - m) * c2)) + (p.x == -INFINITY ? p.y : p.y * fast_exp2((p.x - m) * c2));
            most = m;
        }
    s_part[y][x] = float2{most, sum};
    __syncthreads();
    if (y != 0 || row >= n_rows) return;
    for (int w = 1; w < 8; ++w) most = fmaxf(most, s_part[w][x].x);
    sum = 0.f;
    for (int w = 0; w < 8; ++w) {
        const float2 p = s_part[w][x];
        sum += p.x == -INFINITY ? p.y : p.y * fast_exp2((p.x - most) * c2);
    }
    const float ln = logf(sum);
    const int slot = rows[row];
    lse[slot] = scale * most + ln;
    loss[slot] = scale * (most - target_logit[row]) + ln;
}

// ------------------------------------------------------------------------------------------
// Backward.  The labelled rows of x one behind the other, and zeros in dx of the other slots.
__global__ void __launch_bounds__(256) loss_gather_kernel(const uint4* x, uint4* rows_x, uint4* dx, const int32_t* rows, const int32_t* slot_target,
                                                          const int32_t* count, int n_q, int chunks) {
    const int i = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= n_q) return;
    const bool row = i < *count, none = slot_target[i] < 0;
    const size_t from = row ? (size_t)rows[i] * chunks : 0;
    for (int c = lane; c < chunks; c += 64) {
        if (row) rows_x[(size_t)i * chunks + c] = x[from + c];
        if (none) dx[(size_t)i * chunks + c] = uint4{0, 0, 0, 0};
    }
}

struct GradArgs {
    const __bf16 *table;
    __bf16 *rows_x;                  // [labelled][hidden]
    __bf16 *d;                       // [labelled][pitch]: D of the piece
    __bf16 *dx, *dtable;
    float *part;                     // [splits][n_q][hidden]: dX so far
    const int32_t *rows, *target, *count;
    const float *row_lse, *row_weight, *factor;
    int vocab, hidden, n_q, pitch;
    int piece0, piece_n;             // words of the piece
    int splits;                      // of the piece along the words, for dX
    int add, final;                  // dX: there are earlier pieces; this piece is the last and not split
    float c2;
};

template <class S>
__global__ void __launch_bounds__(256, S::LDS_BYTES > 81920 ? 1 : 2) loss_d_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const int n_rows = ld_const(a.count);
    int tm, tn, unused;
    if (!find_tile((a.piece_n + S::TM - 1) / S::TM, (n_rows + S::TN - 1) / S::TN, 1, tm, tn, unused)) return;
    const int m0 = tm * S::TM, n0 = tn * S::TN, v0 = a.piece0 + m0;
    Gemm<S> g;
    g.start(smem);
    g.run(GemmOperand{a.table + (size_t)v0 * a.hidden, a.hidden, a.vocab - v0, nullptr},
          GemmOperand{a.rows_x + (size_t)n0 * a.hidden, a.hidden, n_rows - n0, nullptr}, a.hidden);
    const int first = v0 + g.wm * (S::BM * 32) + (g.lane / 32) * 4;
    if (v0 + S::TM > a.vocab) {                     // words past the end: D is 0
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int j = 0; j < S::BN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (first + i * 32 + (r / 4) * 8 + r % 4 >= a.vocab) g.acc[i][j][r] = -INFINITY;
    }
    float lse2[S::BN], weight[S::BN];
    int target[S::BN];
#pragma unroll
    for (int j = 0; j < S::BN; ++j) {
        const int n = n0 + g.wn * (S::BN * 32) + j * 32 + g.lane % 32;
        const bool on = n < n_rows;
        lse2[j] = on ? a.row_lse[n] * kLog2e : 0.f;
        weight[j] = on ? a.row_weight[n] : 0.f;
        target[j] = on ? a.target[n] - first : -1;
    }
    g.template rows_out<2>(
        [&](int i, int j, int r) __attribute__((always_inline)) {
            const float p = fast_exp2(g.acc[i][j][r] * a.c2 - lse2[j]);
            return weight[j] * (target[j] == i * 32 + (r / 4) * 8 + r % 4 ? p - 1.f : p);
        },
        [&](int n, int m, const i32x4& v) __attribute__((always_inline)) {
            if (n0 + n < n_rows) *reinterpret_cast<i32x4*>(a.d + (size_t)(n0 + n) * a.pitch + m0 + m) = v;
        });
}

// dE of the piece: D^T X, both operands with the sum's index (the row) outermost.
template <class S>
__global__ void __launch_bounds__(256, S::LDS_BYTES > 81920 ? 1 : 2) loss_dtable_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    int tm, tn, unused;
    if (!find_tile((a.hidden + S::TM - 1) / S::TM, (a.piece_n + S::TN - 1) / S::TN, 1, tm, tn, unused)) return;
    const int n_rows = ld_const(a.count), m0 = tm * S::TM, n0 = tn * S::TN;
    Gemm<S> g;
    g.start(smem);
    g.run(GemmOperand{a.rows_x + m0, a.hidden, a.hidden - m0, nullptr}, GemmOperand{a.d + n0, a.pitch, a.pitch - n0, nullptr}, n_rows);
    const float factor = n_rows > 0 ? *a.factor : 0.f;
    g.template rows_out<2>([&](int i, int j, int r) __attribute__((always_inline)) { return factor * g.acc[i][j][r]; },
                           [&](int n, int m, const i32x4& v) __attribute__((always_inline)) {
                               if (n0 + n < a.piece_n && m0 + m < a.hidden)
                                   *reinterpret_cast<i32x4*>(a.dtable + (size_t)(a.piece0 + n0 + n) * a.hidden + m0 + m) = v;
                           });
}

// dX: D E over the piece's words (or a split's share of them), added to what earlier pieces left.
template <class S>
__global__ void __launch_bounds__(256, S::LDS_BYTES > 81920 ? 1 : 2) loss_dx_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const int n_rows = ld_const(a.count);
    int tm, tn, split;
    if (!find_tile((a.hidden + S::TM - 1) / S::TM, (n_rows + S::TN - 1) / S::TN, a.splits, tm, tn, split)) return;
    const int steps = (a.piece_n + kStepK - 1) / kStepK, per = (steps + a.splits - 1) / a.splits;
    const int k0 = min(split * per * kStepK, a.piece_n), k1 = min(k0 + per * kStepK, a.piece_n), m0 = tm * S::TM, n0 = tn * S::TN;
    Gemm<S> g;
    g.start(smem);
    g.run(GemmOperand{a.table + (size_t)(a.piece0 + k0) * a.hidden + m0, a.hidden, a.hidden - m0, nullptr},
          GemmOperand{a.d + (size_t)n0 * a.pitch + k0, a.pitch, n_rows - n0, nullptr}, k1 - k0);
    const float factor = *a.factor;
    g.template rows_out<4>([&](int i, int j, int r) __attribute__((always_inline)) { return g.acc[i][j][r]; },
                           [&](int n, int m, const i32x4& bits) __attribute__((always_inline)) {
                               const int row = n0 + n, col = m0 + m;
                               if (row >= n_rows || col >= a.hidden) return;
                               f32x4 v = __builtin_bit_cast(f32x4, bits);
                               f32x4* part = reinterpret_cast<f32x4*>(a.part + ((size_t)split * a.n_q + row) * a.hidden + col);
                               if (a.add) v += *part;
                               if (a.final) *reinterpret_cast<bf16x4*>(a.dx + (size_t)a.rows[row] * a.hidden + col) = pack4(factor * v[0], factor * v[1], factor * v[2], factor * v[3]);
                               else *part = v;
                           });
}

__global__ void __launch_bounds__(256) loss_dx_join_kernel(GradArgs a) {
    const int chunks = a.hidden / 8, strips = (chunks + 255) / 256, row = (int)blockIdx.x / strips, c = ((int)blockIdx.x % strips) * 256 + (int)threadIdx.x;
    if (row >= *a.count || c >= chunks) return;
    const float factor = *a.factor;
    f32x4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    for (int s = 0; s < a.splits; ++s) {
        const f32x4* from = reinterpret_cast<const f32x4*>(a.part + ((size_t)s * a.n_q + row) * a.hidden + c * 8);
        u += from[0];
        v += from[1];
    }
    *reinterpret_cast<bf16x8*>(a.dx + (size_t)a.rows[row] * a.hidden + c * 8) =
        pack8(factor * u[0], factor * u[1], factor * u[2], factor * u[3], factor * v[0], factor * v[1], factor * v[2], factor * v[3]);
}

// ------------------------------------------------------------------------------------------
// Tiles.  `Slots32` .. `Slots128` serve calls of few slots: four wavefronts side by side along the words (or columns).
template <bool MP, bool MQ> using Wide = GemmShape<2, 2, 4, 4, MP, MQ>;
template <bool MP, bool MQ> using Half = GemmShape<2, 2, 2, 2, MP, MQ>;
template <bool MP, bool MQ> using Slots128 = GemmShape<4, 1, 2, 4, MP, MQ>;
template <bool MP, bool MQ> using Slots64 = GemmShape<4, 1, 2, 2, MP, MQ>;
template <bool MP, bool MQ> using Slots32 = GemmShape<4, 1, 2, 1, MP, MQ>;

static int slot_tile(int n_q) { return n_q <= 32 ? 32 : n_q <= 64 ? 64 : n_q <= 128 ? 128 : 256; }

// Words to a piece: D of a piece takes up to kPieceBytes, and dX's partial sums (8 bytes of traffic a piece, slot and column) stay below 3 % of the
// time of the products where a piece has kPieceMin words.
constexpr size_t kPieceBytes = 512u << 20;
constexpr int kPieceMin = 16384;

struct LossLayout {
    size_t off_count, off_factor, off_slot_target, off_block_count, off_block_max, off_rows, off_target, off_row_lse, off_row_weight;
    size_t off_part, off_target_logit, fwd_bytes;                 // forward
    size_t off_rows_x, off_d, off_dx_part, bwd_bytes;             // backward
    int blocks, tile, word_tiles, pitch_rows, piece, pieces, splits;
};

static LossLayout loss_layout(const wlb_vocab_desc& d) {
    LossLayout L;
    const size_t n_q = d.n_q, v = d.vocab, h = d.hidden;
    L.blocks = (d.n_q + kRowsThreads - 1) / kRowsThreads;
    L.tile = slot_tile(d.n_q);
    L.word_tiles = (d.vocab + kWordTile - 1) / kWordTile;
    L.pitch_rows = (int)align_up(n_q, 64);
    const size_t words = align_up(v, kWordTile);
    size_t piece = std::max((size_t)kPieceMin, kPieceBytes / (2 * n_q) / kWordTile * kWordTile);
    L.piece = (int)std::min(words, piece);
    L.pieces = (int)((v + L.piece - 1) / L.piece);
    const long long tiles = (long long)((d.hidden + kWordTile - 1) / kWordTile) * ((d.n_q + L.tile - 1) / L.tile);
    const int slots = compute_units() * (L.tile <= 64 ? 2 : 1), steps = (int)((std::min((size_t)L.piece, v) + kStepK - 1) / kStepK);
    L.splits = (int)std::max(1LL, std::min(slots / tiles, (long long)steps / 4));
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    L.off_count = take(4);
    L.off_factor = take(4);
    L.off_slot_target = take(4 * n_q);
    L.off_block_count = take(4 * (size_t)L.blocks);
    L.off_block_max = take(4 * (size_t)L.blocks);
    L.off_rows = take(4 * n_q);
    L.off_target = take(4 * n_q);
    L.off_row_lse = take(4 * n_q);
    L.off_row_weight = take(4 * n_q);
    const size_t common = at;
    L.off_part = take(sizeof(float2) * (size_t)L.word_tiles * L.pitch_rows);
    L.off_target_logit = take(4 * n_q);
    L.fwd_bytes = at;
    at = common;
    L.off_rows_x = take(2 * n_q * h);
    L.off_d = take(2 * n_q * (size_t)L.piece);
    L.off_dx_part = take(L.pieces > 1 || L.splits > 1 ? 4 * n_q * h * (size_t)L.splits : 0);
    L.bwd_bytes = at;
    return L;
}

size_t loss_fwd_bytes(const wlb_vocab_desc& d) { return loss_layout(d).fwd_bytes; }
size_t loss_bwd_bytes(const wlb_vocab_desc& d) { return loss_layout(d).bwd_bytes; }

static wlb_status check_loss(const wlb_vocab_desc* desc, const char* call) {
    if (wlb_status st = check_vocab(desc, call, 0)) return st;
    // rows of x are addressed with 32-bit offsets
    if ((uint64_t)desc->n_q * desc->hidden * 2 >= (1ull << 32) - (1u << 20))
        return fail(WLB_ERR_UNSUPPORTED, "%s: x of 4 GiB or more is not supported", call);
    if ((int64_t)(desc->vocab / kWordTile + 1) * (desc->n_q / 32 + 1) > (1 << 30))
        return fail(WLB_ERR_UNSUPPORTED, "%s: vocab=%d words for n_q=%d slots", call, desc->vocab, desc->n_q);
    return WLB_OK;
}

static RowsArgs rows_args(const wlb_vocab_desc& d, const LossLayout& L, char* ws, const int32_t* tokens, const int32_t* q_idx, const int32_t* cu) {
    RowsArgs a = {};
    a.tokens = tokens; a.q_idx = q_idx; a.cu = cu;
    a.slot_target = (int32_t*)(ws + L.off_slot_target);
    a.block_count = (int32_t*)(ws + L.off_block_count);
    a.block_max = (float*)(ws + L.off_block_max);
    a.rows = (int32_t*)(ws + L.off_rows);
    a.target = (int32_t*)(ws + L.off_target);
    a.row_lse = (float*)(ws + L.off_row_lse);
    a.row_weight = (float*)(ws + L.off_row_weight);
    a.count = (int32_t*)(ws + L.off_count);
    a.factor = (float*)(ws + L.off_factor);
    a.n_q = d.n_q; a.t_kv = d.t_kv; a.n_docs = d.n_docs; a.vocab = d.vocab; a.blocks = L.blocks; a.scale = d.scale;
    return a;
}

static void launch_rows(const RowsArgs& a, hipStream_t stream) {
    if (a.blocks == 1) {
        loss_rows_kernel<true><<<1, kRowsThreads, 0, stream>>>(a);
    } else {
        loss_targets_kernel<<<a.blocks, kRowsThreads, 0, stream>>>(a);
        loss_rows_kernel<false><<<a.blocks, kRowsThreads, 0, stream>>>(a);
    }
}

}  // namespace wlb

using namespace wlb;

extern "C" wlb_status wlb_vocab_workspace_size(const wlb_vocab_desc* desc, size_t* embed_bwd, size_t* loss_fwd, size_t* loss_bwd) {
    if (wlb_status st = check_vocab(desc, "wlb_vocab_workspace_size", WLB_VOCAB_ACCUMULATE)) return st;
    if (embed_bwd) *embed_bwd = embed_bwd_bytes(*desc);
    if (loss_fwd) *loss_fwd = loss_fwd_bytes(*desc);
    if (loss_bwd) *loss_bwd = loss_bwd_bytes(*desc);
    return WLB_OK;
}

extern "C" wlb_status wlb_loss_fwd(const wlb_vocab_desc* desc, const void* x, const void* table, const int32_t* tokens, const int32_t* q_idx,
                                   const int32_t* cu_seqlens_k, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream_) {
    if (wlb_status st = check_loss(desc, "wlb_loss_fwd")) return st;
    if (!x || !table || !tokens || !q_idx || !cu_seqlens_k || !loss || !lse || !workspace) return fail(WLB_ERR_INVALID_ARG, "wlb_loss_fwd: null pointer");
    if (misaligned(x, 16) || misaligned(table, 16) || misaligned(tokens, 4) || misaligned(q_idx, 4) || misaligned(cu_seqlens_k, 4) || misaligned(loss, 4) ||
        misaligned(lse, 4) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "wlb_loss_fwd: misaligned pointer");
    const wlb_vocab_desc& d = *desc;
    const LossLayout L = loss_layout(d);
    if (workspace_bytes < L.fwd_bytes) return fail(WLB_ERR_BUFFER_TOO_SMALL, "wlb_loss_fwd: workspace %zu < %zu bytes", workspace_bytes, L.fwd_bytes);
    hipStream_t stream = (hipStream_t)stream_;
    char* ws = (char*)workspace;
    RowsArgs r = rows_args(d, L, ws, tokens, q_idx, cu_seqlens_k);
    r.loss_out = loss; r.lse_out = lse;
    launch_rows(r, stream);
    StatsArgs a;
    a.x = (const __bf16*)x; a.table = (const __bf16*)table;
    a.rows = r.rows; a.target = r.target; a.count = r.count;
    a.part = (float2*)(ws + L.off_part); a.target_logit = (float*)(ws + L.off_target_logit);
    a.vocab = d.vocab; a.hidden = d.hidden; a.pitch = L.pitch_rows; a.c2 = d.scale * kLog2e;
    const unsigned grid = tile_grid((long long)L.word_tiles * ((d.n_q + L.tile - 1) / L.tile));
    if (L.tile == 32) loss_stats_kernel<Slots32<false, false>><<<grid, 256, 0, stream>>>(a);
    else if (L.tile == 64) loss_stats_kernel<Slots64<false, false>><<<grid, 256, 0, stream>>>(a);
    else if (L.tile == 128) loss_stats_kernel<Slots128<false, false>><<<grid, 256, 0, stream>>>(a);
    else loss_stats_kernel<Wide<false, false>><<<grid, 256, 0, stream>>>(a);
    loss_join_kernel<<<(d.n_q + 31) / 32, 256, 0, stream>>>(a.part, a.target_logit, a.rows, a.count, loss, lse, L.word_tiles, L.pitch_rows, d.scale);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "loss launch: %s", hipGetErrorString(e));
    return WLB_OK;
}

extern "C" wlb_status wlb_loss_bwd(const wlb_vocab_desc* desc, const void* x, const void* table, const int32_t* tokens, const int32_t* q_idx,
                                   const int32_t* cu_seqlens_k, const float* lse, const float* d_loss, void* dx, void* dtable, void* workspace,
                                   size_t workspace_bytes, void* stream_) {
    if (wlb_status st = check_loss(desc, "wlb_loss_bwd")) return st;
    if (!x || !table || !tokens || !q_idx || !cu_seqlens_k || !lse || !d_loss || !dx || !dtable || !workspace)
        return fail(WLB_ERR_INVALID_ARG, "wlb_loss_bwd: null pointer");
    if (misaligned(x, 16) || misaligned(table, 16) || misaligned(tokens, 4) || misaligned(q_idx, 4) || misaligned(cu_seqlens_k, 4) || misaligned(lse, 4) ||
        misaligned(d_loss, 4) || misaligned(dx, 16) || misaligned(dtable, 16) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "wlb_loss_bwd: misaligned pointer");
    const wlb_vocab_desc& d = *desc;
    const LossLayout L = loss_layout(d);
    if (workspace_bytes < L.bwd_bytes) return fail(WLB_ERR_BUFFER_TOO_SMALL, "wlb_loss_bwd: workspace %zu < %zu bytes", workspace_bytes, L.bwd_bytes);
    hipStream_t stream = (hipStream_t)stream_;
    char* ws = (char*)workspace;
    RowsArgs r = rows_args(d, L, ws, tokens, q_idx, cu_seqlens_k);
    r.lse_in = lse; r.d_loss = d_loss;
    launch_rows(r, stream);
    GradArgs a = {};
    a.table = (const __bf16*)table; a.rows_x = (__bf16*)(ws + L.off_rows_x); a.d = (__bf16*)(ws + L.off_d);
    a.dx = (__bf16*)dx; a.dtable = (__bf16*)dtable; a.part = (float*)(ws + L.off_dx_part);
    a.rows = r.rows; a.target = r.target; a.count = r.count; a.row_lse = r.row_lse; a.row_weight = r.row_weight; a.factor = r.factor;
    a.vocab = d.vocab; a.hidden = d.hidden; a.n_q = d.n_q; a.pitch = L.piece; a.splits = L.splits; a.c2 = d.scale * kLog2e;
    loss_gather_kernel<<<(d.n_q + 3) / 4, 256, 0, stream>>>((const uint4*)x, (uint4*)a.rows_x, (uint4*)dx, a.rows, r.slot_target, a.count, d.n_q, d.hidden / 8);
    const long long slot_tiles = (d.n_q + L.tile - 1) / L.tile;
    for (int p = 0; p < L.pieces; ++p) {
        a.piece0 = p * L.piece;
        a.piece_n = std::min(L.piece, d.vocab - a.piece0);
        a.add = p > 0;
        a.final = p == L.pieces - 1 && L.splits == 1;
        const unsigned d_grid = tile_grid((long long)((a.piece_n + kWordTile - 1) / kWordTile) * slot_tiles);
        if (L.tile == 32) loss_d_kernel<Slots32<false, false>><<<d_grid, 256, 0, stream>>>(a);
        else if (L.tile == 64) loss_d_kernel<Slots64<false, false>><<<d_grid, 256, 0, stream>>>(a);
        else if (L.tile == 128) loss_d_kernel<Slots128<false, false>><<<d_grid, 256, 0, stream>>>(a);
        else loss_d_kernel<Wide<false, false>><<<d_grid, 256, 0, stream>>>(a);
        const long long wide = (long long)((a.piece_n + 255) / 256) * ((d.hidden + 255) / 256);
        if (wide >= compute_units()) loss_dtable_kernel<Wide<true, true>><<<tile_grid(wide), 256, 0, stream>>>(a);
        else loss_dtable_kernel<Half<true, true>><<<tile_grid((long long)((a.piece_n + 127) / 128) * ((d.hidden + 127) / 128)), 256, 0, stream>>>(a);
        const unsigned dx_grid = tile_grid((long long)((d.hidden + kWordTile - 1) / kWordTile) * slot_tiles * L.splits);
        if (L.tile == 32) loss_dx_kernel<Slots32<true, false>><<<dx_grid, 256, 0, stream>>>(a);
        else if (L.tile == 64) loss_dx_kernel<Slots64<true, false>><<<dx_grid, 256, 0, stream>>>(a);
        else if (L.tile == 128) loss_dx_kernel<Slots128<true, false>><<<dx_grid, 256, 0, stream>>>(a);
        else loss_dx_kernel<Wide<true, false>><<<dx_grid, 256, 0, stream>>>(a);
    }
    if (L.splits > 1) loss_dx_join_kernel<<<(unsigned)d.n_q * ((d.hidden / 8 + 255) / 256), 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "loss gradient launch: %s", hipGetErrorString(e));
    return WLB_OK;
}
