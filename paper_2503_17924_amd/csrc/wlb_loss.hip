// Cross entropy of a rank's slots over the whole vocabulary, and its gradient, without the logits ever being kept
// (wlb_loss_fwd / wlb_loss_bwd).
//
// With c = scale, l = <x, E_v> in fp32 sums of the MFMAs, n labelled slots:
//   forward   one product l = X E^T.  A tile of up to 256 words and 256 slots leaves per slot its maximum and its sum of exp(c (l - max)), and the
//             target's l where the tile holds it; loss_join_kernel combines a slot's tiles: lse = c max + ln sum, loss = c (max - l_t) + ln sum.
//   backward  D = w (exp(c l - lse) - [v = target]) with w = d_loss / G, G the largest |d_loss|, in bf16, for one piece of the vocabulary at a
//             time; then dE = c G D^T X for the piece's rows and dX += D E over the pieces, in fp32; dX is scaled by c G at the end.
//             G keeps the factor that most training steps have in common (1 / tokens) out of the rounding of D.  What bf16 leaves out of D at a row's
//             target, the largest of its entries, is added to dX in fp32.  dE keeps D's roundings, up to 2^-8 of each term of its sums: as much as its own rounding
//             where one row makes up the sum, less where many rows' roundings average out.  Up to kExactRows rows, which fill half of a step of its
//             sum, D has a second set of rows with all that bf16 leaves out of the first, and dE is exact but for its own rounding.
// Slots without a target are left out of everything: the others are listed in order (rows), and products run over that list.
// Bound by the matrix products: 2 n V H operations forward, 6 n V H backward, where 64 slots or more share the table's
// rows; by the table's bytes below that.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "wlb_gemm.h"
#include "wlb_vocab.h"

namespace wlb {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWordTile = 256;                 // words (forward, D) and columns of hidden (dX) per tile; some tiles of few slots have less
constexpr int kRowsThreads = 1024;
constexpr int kExactRows = kStepK / 2;         // labelled slots up to which D has a second set of rows

// Tiles.  `Slots32` .. `Slots128` serve calls of few slots: four wavefronts side by side along the words (or columns).
template <bool MP, bool MQ> using Wide = GemmShape<2, 2, 8, 8, MP, MQ>;
template <bool MP, bool MQ> using Half = GemmShape<2, 2, 4, 4, MP, MQ>;
template <bool MP, bool MQ> using Slots128 = GemmShape<4, 1, 4, 8, MP, MQ>;
template <bool MP, bool MQ> using Slots64 = GemmShape<4, 1, 4, 4, MP, MQ>;
template <bool MP, bool MQ> using Slots32 = GemmShape<4, 1, 4, 2, MP, MQ>;
// the same with tiles of 128 words
using Slots128Low = GemmShape<4, 1, 2, 8, false, false>;
using Slots64Low = GemmShape<4, 1, 2, 4, false, false>;
using Slots32Low = GemmShape<4, 1, 2, 2, false, false>;

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
template <class S, class F>
__device__ __forceinline__ void join_parts(const Work& w, const float* parts, F f) {
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

// ------------------------------------------------------------------------------------------
// Forward.  Exponents are in units of log2, relative to a tile's reference: its largest l times c2, rounded.  What the rounding
// is off by cancels, since the reference is what the sum is stored with.  An infinite reference cannot be subtracted: there the exponents are taken as they
// are, and 2^inf stays in the sum (a logit of +inf), or nothing does (all of them -inf, or words past the end).
__device__ __forceinline__ float subtracted(float ref) { return __builtin_isinf(ref) ? 0.f : ref; }
// a tile's sum, relative to a reference that is at least the tile's
__device__ __forceinline__ float rescaled(float2 part, float ref) { return part.x == ref ? part.y : part.y * fast_exp2(part.x - ref); }

struct StatsArgs {
    const __bf16 *x, *table;
    const int32_t *rows, *target, *count;
    float2* part;                    // [word tiles][pitch]: reference r of a row in a tile, and sum of 2^(c2 l - r)
    float* target_logit;             // [labelled] l of the target
    float* parts;                    // divided tiles
    int vocab, hidden, pitch, workgroups;
    float c2;                        // scale * log2(e)
};

template <class S>
__device__ __forceinline__ Work stats_work(const StatsArgs& a) {
    const int n_rows = ld_const(a.count);
    return Work::make<S>(a.table, a.hidden, a.vocab, a.x, a.hidden, n_rows, a.rows, a.hidden, a.workgroups, kNever);
}

// exchange a value with the lane 16 away, inside a half of the wavefront
__device__ __forceinline__ float xrow(float x) {
    const int xi = __builtin_bit_cast(int, x);
    const auto r = __builtin_amdgcn_permlane16_swap(xi, xi, false, false);
    return __builtin_bit_cast(float, (int)((threadIdx.x & 16) ? r[0] : r[1]));
}

// What belongs to a wavefront's rows n is loaded once for every row, 64 to a register, and fetched from the lane that holds it.
template <class S> constexpr int row_regs() { return (S::BN * 16 + 63) / 64; }
template <class S>
__device__ __forceinline__ int row_held(const Gemm<S>& g, const GemmItem& it, int k) { return it.tn * S::TN + g.wn * (S::BN * 16) + k * 64 + g.lane % (S::BN * 16); }
template <class T, int N>
__device__ __forceinline__ T of_row(const T (&regs)[N], int j, int lane) { return __shfl(regs[j / 4], (j % 4) * 16 + lane % 16); }

// Stores of a wavefront's part in rows_out<Bytes>, 1 KiB each, where no row or column lies past the end.
template <class S, int Bytes> constexpr int row_stores() { return S::BM * 16 * S::BN * 16 * Bytes / 1024; }

template <class S>
struct StatsDone {
    const StatsArgs& a;
    const Work& w;
    char* smem;
    struct Ahead { int target[row_regs<S>()]; };        // -1: no row
    __device__ __forceinline__ Ahead load(const Gemm<S>& g, const GemmItem& it) const {
        Ahead h;
#pragma unroll
        for (int k = 0; k < row_regs<S>(); ++k) {
            const int row = row_held<S>(g, it, k);
            h.target[k] = row < w.qn ? a.target[row] : -1;
        }
        return h;
    }
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, const Ahead& ahead, uint32_t room) const {
        if constexpr (S::OUT_WAVE == 8192)          // other tiles are never divided
            if (it.part >= 0) {
                g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), w.qn - it.tn * S::TN);
                return 0;
            }
        const int m0 = it.tm * S::TM, n0 = it.tn * S::TN, n_rows = w.qn;
        const int first = m0 + g.wm * (S::BM * 16) + (g.lane / 16) * 4;       // word of register 0 of block 0
        float2* s_part = (float2*)(smem + (room - g.lds));                    // [WM][TN]
        int target[S::BN];                                                    // register that holds the target, if this lane has it
#pragma unroll
        for (int j = 0; j < S::BN; ++j) {
            const int word = of_row(ahead.target, j, g.lane);
            target[j] = word < 0 ? -1 : word - first;
        }
        auto block = [&](int j, auto edge) __attribute__((always_inline)) {   // edge: words of the tile lie past the end
            const int n = g.wn * (S::BN * 16) + j * 16 + g.lane % 16;
            float logit[S::BM][4];
#pragma unroll
            for (int i = 0; i < S::BM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float l = g.sum(i, j, r);
                    logit[i][r] = edge && first + i * 16 + r >= a.vocab ? -INFINITY : l;
                }
            const int t = target[j];
            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < S::BM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) most[r] = fmaxf(most[r], logit[i][r]);
            float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            top = fmaxf(top, xrow(top));
            top = fmaxf(top, xhalf(top));
            if (__any(t >= 0 && t < S::BM * 16)) {
                float l = 0.f;
                bool mine = false;
#pragma unroll
                for (int i = 0; i < S::BM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool here = t == i * 16 + r;
                        l = here ? logit[i][r] : l;
                        mine |= here;
                    }
                if (mine) a.target_logit[n0 + n] = l;
            }
            const float ref = top * a.c2, from = subtracted(ref);
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < S::BM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] += fast_exp2(__builtin_fmaf(logit[i][r], a.c2, -from));
            float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            all += xrow(all);
            all += xhalf(all);
            if (g.lane < 16) s_part[g.wm * S::TN + n] = float2{ref, all};
            __builtin_amdgcn_sched_barrier(0);
        };
        if (m0 + S::TM > a.vocab) {
#pragma unroll
            for (int j = 0; j < S::BN; ++j) block(j, std::true_type{});
        } else {
#pragma unroll
            for (int j = 0; j < S::BN; ++j) block(j, std::false_type{});
        }
        __syncthreads();
        for (int n = threadIdx.x; n < S::TN; n += 256) {
            if (n0 + n >= n_rows) continue;
            float ref = s_part[n].x, sum = 0.f;
#pragma unroll
            for (int k = 1; k < S::WM; ++k) ref = fmaxf(ref, s_part[k * S::TN + n].x);
#pragma unroll
            for (int k = 0; k < S::WM; ++k) sum += rescaled(s_part[k * S::TN + n], ref);
            a.part[(size_t)it.tm * a.pitch + n0 + n] = float2{ref, sum};
        }
        __syncthreads();
        return 0;
    }
};

template <class S>
__global__ void __launch_bounds__(256, S::PER_CU) loss_stats_kernel(StatsArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const Work w = stats_work<S>(a);
    Gemm<S> gemm;
    gemm.run(smem, w, StatsDone<S>{a, w, smem});
}

// The same for a row of a divided tile.
template <class S>
__global__ void __launch_bounds__(256) loss_stats_parts_kernel(StatsArgs a) {
    const Work w = stats_work<S>(a);
    join_parts<S>(w, a.parts, [&](int tm, int tn, int n, int m, const f32x4& l) __attribute__((always_inline)) {
        const int row = tn * S::TN + n, word = tm * S::TM + m;
        if (row >= w.qn) return;
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) most = word + k < a.vocab ? fmaxf(most, l[k]) : most;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float ref = most * a.c2, from = subtracted(ref);
        const int t = a.target[row] - word;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (word + k < a.vocab) sum += fast_exp2(__builtin_fmaf(l[k], a.c2, -from));
            if (t == k) a.target_logit[row] = l[k];
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if ((threadIdx.x & 63) == 0) a.part[(size_t)tm * a.pitch + row] = float2{ref, sum};
    });
}

// A slot's tiles combined: R rows to a workgroup, 256 / R threads to a row (few rows have few workgroups, and more tiles).
template <int R>
__global__ void __launch_bounds__(256) loss_join_kernel(const float2* part, const float* target_logit, const int32_t* rows, const int32_t* count, float* loss,
                                                        float* lse, int tiles, int pitch, float c2) {
    constexpr int W = 256 / R;
    __shared__ float2 s_part[W][R];
    const int n_rows = *count, x = threadIdx.x % R, y = threadIdx.x / R, row = (int)blockIdx.x * R + x;
    constexpr float kLn2 = 0.6931471805599453f;
    if ((int)blockIdx.x * R >= n_rows) return;
    constexpr int kAhead = 8;
    float ref = -INFINITY, sum = 0.f;
    if (row < n_rows)
        for (int t = y; t < tiles; t += W * kAhead) {
            float2 p[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) p[k] = t + W * k < tiles ? part[(size_t)(t + W * k) * pitch + row] : float2{-INFINITY, 0.f};
            float r = ref;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) r = fmaxf(r, p[k].x);
            sum = rescaled(float2{ref, sum}, r);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) sum += rescaled(p[k], r);
            ref = r;
        }
    s_part[y][x] = float2{ref, sum};
    __syncthreads();
    if (y != 0 || row >= n_rows) return;
    for (int k = 1; k < W; ++k) ref = fmaxf(ref, s_part[k][x].x);
    sum = 0.f;
    for (int k = 0; k < W; ++k) sum += rescaled(s_part[k][x], ref);
    const float log_sum = log2f(sum);
    const int slot = rows[row];
    lse[slot] = kLn2 * (ref + log_sum);
    loss[slot] = kLn2 * (log_sum - __builtin_fmaf(target_logit[row], c2, -ref));
}

// ------------------------------------------------------------------------------------------
// Backward.  The labelled rows of x one behind the other (few of them once more, for D's second set of rows), and zeros in dx of the other slots.
constexpr int kGatherMost = 1 << 20;           // workgroups at most
__global__ void __launch_bounds__(256) loss_gather_kernel(const uint4* x, uint4* rows_x, uint4* dx, const int32_t* rows, const int32_t* slot_target,
                                                          const int32_t* count, int n_q, int chunks) {
    const int lane = threadIdx.x & 63, n = *count;
    for (int i = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6); i < n_q; i += kGatherMost * 4) {
        const bool row = i < n, none = slot_target[i] < 0;
        const size_t from = row ? (size_t)rows[i] * chunks : 0;
        for (int c = lane; c < chunks; c += 64) {
            if (row) rows_x[(size_t)i * chunks + c] = x[from + c];
            if (row && n <= kExactRows) rows_x[(size_t)(n + i) * chunks + c] = x[from + c];
            if (none) dx[(size_t)i * chunks + c] = uint4{0, 0, 0, 0};
        }
    }
}

struct GradArgs {
    const __bf16 *table;
    __bf16 *rows_x;                  // [labelled][hidden], up to kExactRows rows twice
    __bf16 *d;                       // [labelled][pitch]: D of the piece; behind up to kExactRows rows what bf16 leaves out of them
    __bf16 *dx, *dtable;
    float *dx_sum;                   // [n_q][hidden]: dX of the pieces so far, where there are several
    float *parts;                    // divided tiles
    const int32_t *rows, *target, *count;
    const float *row_lse, *row_weight, *factor;
    float *target_rest;              // [labelled]: what bf16 leaves out of D at the row's target
    int vocab, hidden, n_q, pitch, workgroups;
    int piece0, piece_n;             // words of the piece
    int add, final;                  // dX: there are earlier pieces; this piece is the last
    float c2;
};

template <class S>
__device__ __forceinline__ Work d_work(const GradArgs& a) {
    return Work::make<S>(a.table + (size_t)a.piece0 * a.hidden, a.hidden, a.piece_n, a.rows_x, a.hidden, ld_const(a.count), nullptr, a.hidden, a.workgroups, kNever);
}

// What bf16 leaves out of d: nothing, beside a value that is not finite.
__device__ __forceinline__ float left_out(float d) {
    const float rest = d - (float)(__bf16)d;
    return __builtin_isfinite(rest) ? rest : 0.f;
}

template <class S>
struct DDone {
    const GradArgs& a;
    const Work& w;
    struct Ahead { float lse2[row_regs<S>()], weight[row_regs<S>()]; int target[row_regs<S>()]; };
    __device__ __forceinline__ Ahead load(const Gemm<S>& g, const GemmItem& it) const {
        Ahead h;
#pragma unroll
        for (int k = 0; k < row_regs<S>(); ++k) {
            const int row = row_held<S>(g, it, k);
            const bool on = row < w.qn;
            h.lse2[k] = on ? a.row_lse[row] : 0.f;
            h.weight[k] = on ? a.row_weight[row] : 0.f;
            h.target[k] = on ? a.target[row] : -1;
        }
        return h;
    }
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, const Ahead& h, uint32_t room) const {
        if constexpr (S::OUT_WAVE == 8192)          // other tiles are never divided
            if (it.part >= 0) {
                g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), w.qn - it.tn * S::TN);
                return 0;
            }
        const int m0 = it.tm * S::TM, n0 = it.tn * S::TN;
        const int first = m0 + g.wm * (S::BM * 16) + (g.lane / 16) * 4;     // word of register 0 of block 0, in the piece
        float lse2[S::BN], weight[S::BN];
        int target[S::BN];
#pragma unroll
        for (int j = 0; j < S::BN; ++j) {
            lse2[j] = of_row(h.lse2, j, g.lane) * kLog2e;
            weight[j] = of_row(h.weight, j, g.lane);
            target[j] = of_row(h.target, j, g.lane) - a.piece0 - first;         // register that holds the target, if this lane has it
        }
        auto share = [&](float l, int j) __attribute__((always_inline)) { return fast_exp2(__builtin_fmaf(l, a.c2, -lse2[j])); };
        // edge: words of the tile lie past the end, D is 0 there
        auto out = [&](auto edge) __attribute__((always_inline)) {
            g.template rows_out<2>(
                room,
                [&](int i, int j, int r) __attribute__((always_inline)) {
                    const float e = weight[j] * share(g.sum(i, j, r), j);
                    return edge && first + i * 16 + r >= a.piece_n ? 0.f : e;
                },
                [&](int n, int m, const i32x4& v, int) __attribute__((always_inline)) {
                    if (n0 + n < w.qn) *reinterpret_cast<i32x4*>(a.d + (size_t)(n0 + n) * a.pitch + m0 + m) = v;
                },
                // the few targets among the words, from the unrounded probability (comparing every word with its row's target took 2.7 us a tile)
                [&](int j, auto set) __attribute__((always_inline)) {
                    const int t = target[j];
                    if (!__any(t >= 0 && t < S::BM * 16)) return;
                    float l = 0.f;
                    bool mine = false;
#pragma unroll
                    for (int i = 0; i < S::BM; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const bool here = t == i * 16 + r;
                            l = here ? g.sum(i, j, r) : l;
                            mine |= here;
                        }
                    if (!mine) return;
                    const float d = weight[j] * (share(l, j) - 1.f);
                    set(t + (g.lane / 16) * 4, d);
                    a.target_rest[n0 + g.wn * (S::BN * 16) + j * 16 + g.lane % 16] = left_out(d);
                });
            if (S::RING || w.qn > kExactRows) return;
            g.template rows_out<2>(
                room,
                [&](int i, int j, int r) __attribute__((always_inline)) {
                    const float p = share(g.sum(i, j, r), j), d = weight[j] * (target[j] == i * 16 + r ? p - 1.f : p);
                    return edge && first + i * 16 + r >= a.piece_n ? 0.f : left_out(d);
                },
                [&](int n, int m, const i32x4& v, int) __attribute__((always_inline)) {
                    if (n0 + n < w.qn) *reinterpret_cast<i32x4*>(a.d + (size_t)(w.qn + n0 + n) * a.pitch + m0 + m) = v;
                });
        };
        if (m0 + S::TM > a.piece_n) out(std::true_type{});
        else out(std::false_type{});
        return n0 + S::TN <= w.qn ? row_stores<S, 2>() : 0;
    }
};

template <class S>
__global__ void __launch_bounds__(256, S::PER_CU) loss_d_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    if constexpr (S::RING) {
        // few labelled slots among many: a wide tile's end with a second set of rows took twice as long, also for the calls that have none (16408 slots, 65536
        // words, hidden 4096: 1795 us a piece, without it 1620)
        using Few = Slots32<false, false>;
        static_assert(Few::TN >= kExactRows && Few::LDS_BYTES <= S::LDS_BYTES, "one tile along the rows, in the same LDS");
        if (ld_const(a.count) <= kExactRows) {
            const Work w = d_work<Few>(a);
            Gemm<Few> gemm;
            gemm.run(smem, w, DDone<Few>{a, w});
            return;
        }
    }
    const Work w = d_work<S>(a);
    Gemm<S> gemm;
    gemm.run(smem, w, DDone<S>{a, w});
}

template <class S>
__global__ void __launch_bounds__(256) loss_d_parts_kernel(GradArgs a) {
    const Work w = d_work<S>(a);
    if (w.qn <= kExactRows) return;
    join_parts<S>(w, a.parts, [&](int tm, int tn, int n, int m, const f32x4& l) __attribute__((always_inline)) {
        const int row = tn * S::TN + n, word = tm * S::TM + m;
        if (row >= w.qn) return;
        const float lse2 = a.row_lse[row] * kLog2e, weight = a.row_weight[row];
        const int t = a.target[row] - a.piece0 - word;
        float d[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float p = word + k < a.piece_n ? fast_exp2(__builtin_fmaf(l[k], a.c2, -lse2)) : 0.f;
            d[k] = weight * (t == k ? p - 1.f : p);
            if (t == k) a.target_rest[row] = left_out(d[k]);
        }
        *reinterpret_cast<bf16x4*>(a.d + (size_t)row * a.pitch + word) = pack4(d[0], d[1], d[2], d[3]);
    });
}

// dE of the piece: D^T X, both operands with the sum's index (the row) outermost.
template <class S>
__device__ __forceinline__ Work dtable_work(const GradArgs& a) {
    const int n = ld_const(a.count);
    return Work::make<S>(a.rows_x, a.hidden, a.hidden, a.d, a.pitch, a.piece_n, nullptr, n <= kExactRows ? 2 * n : n, a.workgroups, kNever);
}

struct NothingAhead {
    struct Ahead {};
    template <class G>
    __device__ __forceinline__ Ahead load(const G&, const GemmItem&) const { return Ahead{}; }
};

template <class S>
struct DtableDone : NothingAhead {
    const GradArgs& a;
    const Work& w;
    float factor;
    __device__ __forceinline__ DtableDone(const GradArgs& a_, const Work& w_) : a(a_), w(w_), factor(*a_.factor) {}
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, Ahead, uint32_t room) const {
        if constexpr (S::OUT_WAVE == 8192)          // other tiles are never divided
            if (it.part >= 0) {
                g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), w.qn - it.tn * S::TN);
                return 0;
            }
        const int m0 = it.tm * S::TM, n0 = it.tn * S::TN;
        g.template rows_out<2>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return factor * g.sum(i, j, r); },
                               [&](int n, int m, const i32x4& v, int) __attribute__((always_inline)) {
                                   if (n0 + n < a.piece_n && m0 + m < a.hidden)
                                       *reinterpret_cast<i32x4*>(a.dtable + (size_t)(a.piece0 + n0 + n) * a.hidden + m0 + m) = v;
                               });
        return n0 + S::TN <= a.piece_n && m0 + S::TM <= a.hidden ? row_stores<S, 2>() : 0;
    }
};

template <class S>
__global__ void __launch_bounds__(256, S::PER_CU) loss_dtable_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const Work w = dtable_work<S>(a);
    Gemm<S> gemm;
    gemm.run(smem, w, DtableDone<S>(a, w));
}

template <class S>
__global__ void __launch_bounds__(256) loss_dtable_parts_kernel(GradArgs a) {
    const Work w = dtable_work<S>(a);
    const float factor = *a.factor;
    join_parts<S>(w, a.parts, [&](int tm, int tn, int n, int m, const f32x4& v) __attribute__((always_inline)) {
        const int word = tn * S::TN + n, col = tm * S::TM + m;
        if (word < a.piece_n && col < a.hidden)
            *reinterpret_cast<bf16x4*>(a.dtable + (size_t)(a.piece0 + word) * a.hidden + col) = pack4(factor * v[0], factor * v[1], factor * v[2], factor * v[3]);
    });
}

// dX: D E over the piece's words, added to what earlier pieces left.
template <class S>
__device__ __forceinline__ Work dx_work(const GradArgs& a) {
    return Work::make<S>(a.table + (size_t)a.piece0 * a.hidden, a.hidden, a.hidden, a.d, a.pitch, ld_const(a.count), nullptr, a.piece_n, a.workgroups, kNarrowParts);
}

// In the last piece with what bf16 left out of D at the row's target, the largest of its entries and a rounding that nothing in the row averages out with
// (up to 2^-8 of all its gradient).  slot, target, rest: the row's, used in the last piece alone.
__device__ __forceinline__ void put_dx(const GradArgs& a, float factor, int row, int col, f32x4 v, int slot, int target, float rest) {
    f32x4* sum = reinterpret_cast<f32x4*>(a.dx_sum + (size_t)row * a.hidden + col);
    if (a.add) v += *sum;
    if (a.final) {
        const bf16x4 e = *reinterpret_cast<const bf16x4*>(a.table + (size_t)target * a.hidden + col);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float more = rest * (float)e[k];
            v[k] += __builtin_isfinite(more) ? more : 0.f;       // beside an entry that is not finite the sum is what it is already
        }
        *reinterpret_cast<bf16x4*>(a.dx + (size_t)slot * a.hidden + col) = pack4(factor * v[0], factor * v[1], factor * v[2], factor * v[3]);
    } else {
        *sum = v;
    }
}

template <class S>
struct DxDone : NothingAhead {
    const GradArgs& a;
    const Work& w;
    float factor;
    __device__ __forceinline__ DxDone(const GradArgs& a_, const Work& w_) : a(a_), w(w_), factor(*a_.factor) {}
    __device__ __forceinline__ int operator()(Gemm<S>& g, const GemmItem& it, Ahead, uint32_t room) const {
        if constexpr (S::OUT_WAVE == 8192)          // other tiles are never divided
            if (it.part >= 0) {
                g.part_out(room, a.parts + (size_t)it.part * (S::TM * S::TN), w.qn - it.tn * S::TN);
                return 0;
            }
        int slot[row_regs<S>()], target[row_regs<S>()];
        float rest[row_regs<S>()];
#pragma unroll
        for (int k = 0; k < row_regs<S>(); ++k) {
            const int row = row_held<S>(g, it, k);
            const bool on = a.final && row < w.qn;
            slot[k] = on ? a.rows[row] : 0;
            target[k] = on ? a.target[row] : 0;
            rest[k] = on ? a.target_rest[row] : 0.f;
        }
        const int m0 = it.tm * S::TM, n0 = it.tn * S::TN;
        g.template rows_out<4>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return g.sum(i, j, r); },
                               [&](int n, int m, const i32x4& v, int j) __attribute__((always_inline)) {
                                   const int from = n - g.wn * (S::BN * 16) - j / 4 * 64;       // lane that holds the row's values
                                   const int s = __shfl(slot[j / 4], from), t = __shfl(target[j / 4], from);
                                   const float r = __shfl(rest[j / 4], from);
                                   if (n0 + n < w.qn && m0 + m < a.hidden) put_dx(a, factor, n0 + n, m0 + m, __builtin_bit_cast(f32x4, v), s, t, r);
                               });
        return n0 + S::TN <= w.qn && m0 + S::TM <= a.hidden ? row_stores<S, 4>() : 0;
    }
};

template <class S>
__global__ void __launch_bounds__(256, S::PER_CU) loss_dx_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const Work w = dx_work<S>(a);
    Gemm<S> gemm;
    gemm.run(smem, w, DxDone<S>(a, w));
}

template <class S>
__global__ void __launch_bounds__(256) loss_dx_parts_kernel(GradArgs a) {
    const Work w = dx_work<S>(a);
    const float factor = *a.factor;
    join_parts<S>(w, a.parts, [&](int tm, int tn, int n, int m, const f32x4& v) __attribute__((always_inline)) {
        const int row = tn * S::TN + n, col = tm * S::TM + m;
        if (row < w.qn && col < a.hidden) put_dx(a, factor, row, col, v, a.rows[row], a.target[row], a.final ? a.target_rest[row] : 0.f);
    });
}

// ------------------------------------------------------------------------------------------
static int slot_tile(int n_q) { return n_q <= 32 ? 32 : n_q <= 64 ? 64 : n_q <= 128 ? 128 : 256; }

// Words to a piece: D of a piece takes up to kPieceBytes, but a piece has kPieceMin words at least (above 16384 slots that is more: 4 GiB at 131072 slots), with
// which dX's partial sums (8 bytes of traffic a piece, slot and column) stay below 3 % of the time of the products.
constexpr size_t kPieceBytes = 512u << 20;
constexpr int kPieceMin = 16384;

static unsigned tile_grid(long long tiles) { return (unsigned)((tiles + kLists - 1) / kLists * kLists); }
// Workgroups of a launch of wide tiles, and of a product that narrow tiles divide along k: one to a compute unit (two, with twice as many parts, took
// longer: dX of 65 slots, 32768 words, hidden 1024, and its join 37 us, with one 27).
static int wide_workgroups() { return std::max(kLists, compute_units() / kLists * kLists); }

struct LossLayout {
    size_t off_count, off_factor, off_slot_target, off_block_count, off_block_max, off_rows, off_target, off_row_lse, off_row_weight, off_target_rest, off_parts;
    size_t off_part, off_target_logit, fwd_bytes;                 // forward
    size_t off_rows_x, off_d, off_dx_sum, bwd_bytes;              // backward
    int blocks, tile, word_tile, word_tiles, pitch_rows, piece, pieces;
};

static LossLayout loss_layout(const wlb_vocab_desc& d) {
    LossLayout L;
    const size_t n_q = d.n_q, v = d.vocab, h = d.hidden;
    L.blocks = (d.n_q + kRowsThreads - 1) / kRowsThreads;
    L.tile = slot_tile(d.n_q);
    // Few slots: tiles of 128 words where those of 256 are fewer than the compute units (32768 words, hidden 1024, 65 slots: statistics 19 us, with 256 33).
    L.word_tile = L.tile < 256 && (d.vocab + kWordTile - 1) / kWordTile < compute_units() ? kWordTile / 2 : kWordTile;
    L.word_tiles = (d.vocab + L.word_tile - 1) / L.word_tile;
    L.pitch_rows = (int)align_up(n_q, 64);
    const size_t words = align_up(v, kWordTile);
    size_t piece = std::max((size_t)kPieceMin, kPieceBytes / (2 * n_q) / kWordTile * kWordTile);
    L.piece = (int)std::min(words, piece);
    L.pieces = (int)((v + L.piece - 1) / L.piece);
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
    L.off_target_rest = take(4 * n_q);
    // parts of divided tiles
    L.off_parts = take(sizeof(float) * kWordTile * (size_t)L.tile * wide_workgroups() * (L.tile < 256 ? 1 : kWideRounds));
    const size_t common = at;
    L.off_part = take(sizeof(float2) * (size_t)L.word_tiles * L.pitch_rows);
    L.off_target_logit = take(4 * n_q);
    L.fwd_bytes = at;
    at = common;
    const size_t rows = n_q + std::min(n_q, (size_t)kExactRows);         // how many slots have a target is known on the device
    L.off_rows_x = take(2 * rows * h);
    L.off_d = take(2 * rows * (size_t)L.piece);
    L.off_dx_sum = take(L.pieces > 1 ? 4 * n_q * h : 0);
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
    if ((int64_t)(desc->vocab / (kWordTile / 2) + 1) * (desc->n_q / 32 + 1) > (1 << 30))
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

// Wide tiles: one workgroup to a compute unit, and a join of the divided tiles where `depth` is long enough (half as many as there are workgroups at most, in one
// round; two thirds, in two: two rounds of halves save nothing).
template <class K, class J, class A>
static void launch_wide(K kernel, J join, A& a, int depth, hipStream_t stream) {
    a.workgroups = wide_workgroups();
    kernel<<<a.workgroups, 256, 0, stream>>>(a);
    if (depth > (2 * kWideParts - 1) * kStepK) join<<<a.workgroups * 2 / 3 * 256 / 4, 256, 0, stream>>>(a);
}

// Narrow tiles of shape S, none of them divided.
template <class S, class K, class A>
static void launch_narrow(K kernel, A& a, long long tiles, hipStream_t stream) {
    a.workgroups = (int)std::min((long long)tile_grid(tiles), (long long)wide_workgroups() * S::PER_CU);
    kernel<<<a.workgroups, 256, 0, stream>>>(a);
}

// Narrow tiles along the columns, all divided along the words.  tile: slots of one
template <class K, class J, class A>
static void launch_divided(K kernel, J join, A& a, int tile, int tiles, hipStream_t stream) {
    a.workgroups = wide_workgroups();
    kernel<<<a.workgroups, 256, 0, stream>>>(a);
    join<<<std::min(tiles, a.workgroups / 2) * tile, 256, 0, stream>>>(a);
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
    a.parts = (float*)(ws + L.off_parts);
    const bool low = L.word_tile < kWordTile;
    if (L.tile == 32) low ? launch_narrow<Slots32Low>(loss_stats_kernel<Slots32Low>, a, L.word_tiles, stream)
                           : launch_narrow<Slots32<false, false>>(loss_stats_kernel<Slots32<false, false>>, a, L.word_tiles, stream);
    else if (L.tile == 64) low ? launch_narrow<Slots64Low>(loss_stats_kernel<Slots64Low>, a, L.word_tiles, stream)
                           : launch_narrow<Slots64<false, false>>(loss_stats_kernel<Slots64<false, false>>, a, L.word_tiles, stream);
    else if (L.tile == 128) low ? launch_narrow<Slots128Low>(loss_stats_kernel<Slots128Low>, a, L.word_tiles, stream)
                           : launch_narrow<Slots128<false, false>>(loss_stats_kernel<Slots128<false, false>>, a, L.word_tiles, stream);
    else launch_wide(loss_stats_kernel<Wide<false, false>>, loss_stats_parts_kernel<Wide<false, false>>, a, d.hidden, stream);
    if (L.tile < 256) loss_join_kernel<4><<<(d.n_q + 3) / 4, 256, 0, stream>>>(a.part, a.target_logit, a.rows, a.count, loss, lse, L.word_tiles, L.pitch_rows, a.c2);
    else loss_join_kernel<32><<<(d.n_q + 31) / 32, 256, 0, stream>>>(a.part, a.target_logit, a.rows, a.count, loss, lse, L.word_tiles, L.pitch_rows, a.c2);
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
    a.dx = (__bf16*)dx; a.dtable = (__bf16*)dtable; a.dx_sum = (float*)(ws + L.off_dx_sum);
    a.rows = r.rows; a.target = r.target; a.count = r.count; a.row_lse = r.row_lse; a.row_weight = r.row_weight; a.factor = r.factor;
    a.target_rest = (float*)(ws + L.off_target_rest);
    a.vocab = d.vocab; a.hidden = d.hidden; a.n_q = d.n_q; a.pitch = L.piece; a.c2 = d.scale * kLog2e;
    loss_gather_kernel<<<std::min((d.n_q + 3) / 4, kGatherMost), 256, 0, stream>>>((const uint4*)x, (uint4*)a.rows_x, (uint4*)dx, a.rows, r.slot_target, a.count, d.n_q, d.hidden / 8);
    a.parts = (float*)(ws + L.off_parts);
    const bool low = L.word_tile < kWordTile;
    for (int p = 0; p < L.pieces; ++p) {
        a.piece0 = p * L.piece;
        a.piece_n = std::min(L.piece, d.vocab - a.piece0);
        a.add = p > 0;
        a.final = p == L.pieces - 1;
        const int word_tiles = (a.piece_n + kWordTile - 1) / kWordTile, column_tiles = (d.hidden + kWordTile - 1) / kWordTile;
        const int few_tiles = (a.piece_n + L.word_tile - 1) / L.word_tile;
        if (L.tile == 32) low ? launch_narrow<Slots32Low>(loss_d_kernel<Slots32Low>, a, few_tiles, stream)
                               : launch_narrow<Slots32<false, false>>(loss_d_kernel<Slots32<false, false>>, a, few_tiles, stream);
        else if (L.tile == 64) low ? launch_narrow<Slots64Low>(loss_d_kernel<Slots64Low>, a, few_tiles, stream)
                               : launch_narrow<Slots64<false, false>>(loss_d_kernel<Slots64<false, false>>, a, few_tiles, stream);
        else if (L.tile == 128) low ? launch_narrow<Slots128Low>(loss_d_kernel<Slots128Low>, a, few_tiles, stream)
                               : launch_narrow<Slots128<false, false>>(loss_d_kernel<Slots128<false, false>>, a, few_tiles, stream);
        else launch_wide(loss_d_kernel<Wide<false, false>>, loss_d_parts_kernel<Wide<false, false>>, a, d.hidden, stream);
        // tiles of 128 x 128 where wide ones neither fill the launch nor have rows enough to be divided, and where there is but one step, in front of
        // and behind which nothing runs beside a wide tile (33 slots, 65536 words, hidden 2048: 66 us, wide 71; 128 slots: 84 and 73)
        if (d.n_q > kStepK && ((long long)word_tiles * column_tiles >= wide_workgroups() || d.n_q > (2 * kWideParts - 1) * kStepK))
            launch_wide(loss_dtable_kernel<Wide<true, true>>, loss_dtable_parts_kernel<Wide<true, true>>, a, d.n_q, stream);
        else launch_narrow<Half<true, true>>(loss_dtable_kernel<Half<true, true>>, a, (long long)((a.piece_n + 127) / 128) * ((d.hidden + 127) / 128), stream);
        if (L.tile == 32) launch_divided(loss_dx_kernel<Slots32<true, false>>, loss_dx_parts_kernel<Slots32<true, false>>, a, 32, column_tiles, stream);
        else if (L.tile == 64) launch_divided(loss_dx_kernel<Slots64<true, false>>, loss_dx_parts_kernel<Slots64<true, false>>, a, 64, column_tiles, stream);
        else if (L.tile == 128) launch_divided(loss_dx_kernel<Slots128<true, false>>, loss_dx_parts_kernel<Slots128<true, false>>, a, 128, column_tiles, stream);
        else launch_wide(loss_dx_kernel<Wide<true, false>>, loss_dx_parts_kernel<Wide<true, false>>, a, a.piece_n, stream);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "loss gradient launch: %s", hipGetErrorString(e));
    return WLB_OK;
}
